"""GPU: the paged cache through the C ABI against the float64 oracle: attention with and without a window, append, the
page operators and a decode loop of them together.

Tolerance of attention outputs, from the roundings: bf16's half step is 2^-8 of a value.  The output is rounded once
(2^-8 |o|); the probabilities are rounded to bf16, in the sum over V and in the normaliser, so the result moves by at
most 2^-8 (w + |o|) <= 2^-7 w, w the same weighted sum over |v|; the logits' 32-bit sums of D products and the 32-bit
exponentials stay below 2^-10 in relative size of a probability for the logits drawn here (|s| < 60: 60 x D x 2^-24
even if every rounding fell the same way)."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2609_26368_amd import hs2

pytestmark = pytest.mark.gpu

BF16_HALF = torch.finfo(torch.bfloat16).eps / 2


def check_out(got, want, weight, what=""):
    got = got.double().cpu().numpy()
    tol = BF16_HALF * np.abs(want) + (2 * BF16_HALF + 2.0 ** -10) * weight + 1e-30
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / tol):.3g} of the tolerance"


class Setup:
    """A pool in one of the layouts with random rows where the sequences' tokens are and NaN everywhere else."""

    def __init__(self, seed, kv, D, Hkv, page, lens, layout="record", spare=3, max_pages=None, poison=True):
        rng = np.random.default_rng(seed)
        self.kv, self.D, self.Hkv, self.page, self.lens = kv, D, Hkv, page, [int(x) for x in lens]
        B = len(lens)
        n_of = [-(-x // page) for x in self.lens]
        self.max_pages = M = max_pages or max(1, max(n_of) + 1)
        self.n_pages = P = sum(n_of) + spare
        order, at = rng.permutation(P), 0
        self.table = np.full((B, M), -1, np.int32)
        for b, n in enumerate(n_of):
            self.table[b, :n] = order[at:at + n]
            at += n
        fp8 = kv == "e4m3"
        dtype = torch.uint8 if fp8 else torch.bfloat16
        if layout == "record":
            kvp = torch.empty(P, Hkv, page, 2 * D, dtype=dtype, device="cuda")
            self.K, self.V = kvp[..., :D], kvp[..., D:]
        elif layout == "token":
            self.K, self.V = (torch.empty(P, page, Hkv, D, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2))
        else:  # rows and pages further apart than they have to be
            self.K, self.V = (torch.empty(P, Hkv + 1, page, D + 32, dtype=dtype, device="cuda")[:, :Hkv, :, :D]
                              for _ in range(2))
        gen = torch.Generator(device="cuda").manual_seed(seed)
        valid = torch.zeros(P, page, dtype=torch.bool, device="cuda")
        for b, L in enumerate(self.lens):
            for j in range(n_of[b]):
                valid[int(self.table[b, j]), :min(page, L - j * page)] = True
        self.scales = None
        self.f64 = []
        if fp8:
            self.scales = tuple(torch.rand(Hkv, device="cuda", generator=gen) * 0.01 + 0.008 for _ in range(2))
        for i, X in enumerate((self.K, self.V)):
            x = torch.randn(P, Hkv, page, D, device="cuda", generator=gen)
            if fp8:
                x = (x / self.scales[i][:, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                v = x.view(torch.float8_e4m3fn).float().double() * self.scales[i].double()[:, None, None]
            else:
                x = x.to(torch.bfloat16)
                v = x.double()
            self.f64.append(torch.where(valid[:, None, :, None], v, 0.0).cpu().numpy())
            if poison:
                x = torch.where(valid[:, None, :, None], x, torch.full_like(x, 0x7F if fp8 else math.nan))
            X.copy_(x)
        self.dtable = torch.from_numpy(self.table).cuda()
        self.dlen = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.gen = gen

    def dims(self, C, Hq, scale=0.0):
        return hs2.make_paged_dims(len(self.lens), C, Hq, self.Hkv, self.D, self.page, self.n_pages, self.max_pages,
                                   tuple(self.K.stride()[:3]), scale)

    def queries(self, C, Hq, extras):
        q = torch.randn(len(self.lens), C, Hq, self.D, device="cuda", generator=self.gen).to(torch.bfloat16)
        if not extras:
            return q, None, None
        return (q, torch.randn(Hq, device="cuda", generator=self.gen),
                torch.randn(q.shape, device="cuda", generator=self.gen).to(torch.bfloat16))

    def attend(self, q, sink, gate, window=None, first=0, out=None, ws=None, stream=None):
        d = self.dims(q.shape[1], q.shape[2])
        out = torch.full_like(q, math.nan) if out is None else out
        ws = torch.empty(hs2.hs2_paged_workspace_bytes(d), dtype=torch.uint8, device="cuda") if ws is None else ws
        span = () if window is None else (window, first)
        name = "hs2_paged_attn" if window is None else "hs2_paged_window_attn"
        sc = () if self.scales is None else self.scales
        getattr(hs2, name + ("" if self.scales is None else "_fp8"))(d, q, self.K, self.V, *sc, self.dtable, self.dlen,
                                                                     *span, sink, gate, out, ws, stream)
        return out

    def reference(self, q, sink, gate, window=None, first=0, pairs=None):
        f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        return PO.attention(f(q), *self.f64, self.table, self.lens, self.page, 1 / math.sqrt(self.D), window, first,
                            f(sink), f(gate), pairs)

    def check(self, C, Hq, window=None, first=0, extras=False):
        q, sink, gate = self.queries(C, Hq, extras)
        out = self.attend(q, sink, gate, window, first)
        check_out(out, *self.reference(q, sink, gate, window, first))


HEADS = [(1, 1), (3, 1), (16, 2), (24, 4), (5, 5), (32, 2), (40, 2), (64, 1), (128, 2)]


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_heads(kv, D, Hq, Hkv):
    s = Setup(Hq * 7 + D, kv, D, Hkv, 32, [0, 1, 31, 33, 200, 517], layout="record")
    s.check(1, Hq, extras=Hq % 2 == 0)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("C,Hq,Hkv", [(2, 16, 2), (3, 24, 4), (5, 3, 3), (8, 16, 2), (16, 8, 1), (16, 3, 1), (4, 64, 2),
                                      (2, 64, 1), (7, 12, 2)])
def test_chunks(kv, D, C, Hq, Hkv):
    """Queries of a chunk see different tokens, some of a short sequence none."""
    s = Setup(C * 11 + D, kv, D, Hkv, 16, [0, 1, C - 1, C, C + 1, 64, 150, 333], layout="token")
    s.check(C, Hq, extras=C % 2 == 1)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["record", "token", "apart"])
def test_pages_and_layouts(kv, page, layout):
    s = Setup(page, kv, 128, 2, page, [page - 1, page, page + 1, 3 * page + 7, 900], layout=layout)
    s.check(1, 8)
    s.check(2, 8, window=page + 5, first=3)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("C", [1, 3, 16])
@pytest.mark.parametrize("window,first", [(1, 0), (1, 1), (2, 0), (15, 4), (16, 16), (17, 1), (64, 33), (127, 0), (128, 4),
                                          (300, 65), (600, 0), (1 << 27, 0), (1, 1 << 27), (40, 500)])
def test_windows(kv, C, window, first):
    s = Setup(window % 97 + C, kv, 128, 2, 16, [0, 1, 2, 17, 40, 130, 500, 555], layout="record")
    s.check(C, 8, window=window, first=first, extras=window % 2 == 0)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,Hq,Hkv,C", [(128, 8, 1, 1), (256, 8, 1, 1), (128, 32, 1, 1), (128, 64, 1, 1), (256, 64, 1, 1),
                                        (128, 8, 1, 16), (256, 32, 1, 4), (128, 32, 1, 4)])
def test_long(kv, D, Hq, Hkv, C):
    """Few sequences, many splits: one long among short ones, and a window that is itself long."""
    s = Setup(D + C, kv, D, Hkv, 64, [9001, 3, 700], layout="record")
    s.check(C, Hq)
    s.check(C, Hq, window=5003, first=70, extras=True)


def test_many_heads_ragged():
    """More (sequence, KV head) pairs than the grid holds at once."""
    rng = np.random.default_rng(5)
    s = Setup(5, "bf16", 128, 8, 16, [int(x) for x in rng.integers(0, 200, 150)] + [4000], layout="token")
    q, _, _ = s.queries(1, 16, False)
    out = s.attend(q, None, None)
    pairs = {(b, b % 8) for b in range(151)} | {(150, g) for g in range(8)}
    want, weight = s.reference(q, None, None, pairs=pairs)
    for b, g in pairs:
        h = slice(2 * g, 2 * g + 2)
        check_out(out[b, :, h], want[b, :, h], weight[b, :, h], f"sequence {b} head {g}")


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("C", [1, 4])
def test_entries_that_are_no_page(kv, C):
    """Their tokens count for nobody; a row of nothing else gives 0."""
    s = Setup(3, kv, 128, 2, 16, [400, 90, 33, 40], layout="record")
    s.table[0, [0, 5, 6, 24]] = [-1, s.n_pages, 2 ** 31 - 1, -2 ** 31]
    s.table[1, 5] = -1  # the last page, the new tokens among it
    s.table[2, :] = -1
    s.dtable = torch.from_numpy(s.table).cuda()
    s.check(C, 8)
    s.check(C, 8, window=70, first=20)
    q, _, _ = s.queries(C, 8, False)
    assert not s.attend(q, None, None)[2].any()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,Hq", [(128, 8), (128, 32), (256, 8)])
@pytest.mark.parametrize("poison", ["nan", "inf"])
def test_what_only_some_queries_see(kv, D, Hq, poison):
    """A token's NaN or infinity reaches the queries that see the token and no other, in windows' first tokens too."""
    if kv == "e4m3" and poison == "inf":
        pytest.skip("E4M3 has no infinities")
    C, L = 4, 300
    s = Setup(11, kv, D, 1, 16, [L, L], layout="record")
    bad = 0x7F if kv == "e4m3" else float(poison)
    q, sink, gate = s.queries(C, Hq, True)
    for X, rows in ((s.K, (L - 1,)), (s.V, (L - 2,))):
        for t in rows:
            X[int(s.table[0, t // 16]), :, t % 16] = bad
    out = s.attend(q, sink, gate)
    want, weight = s.reference(q, sink, gate)
    check_out(out[1], want[1], weight[1])
    check_out(out[0, :2], want[0, :2], weight[0, :2])
    assert not torch.isfinite(out[0, 2:]).any()
    # a window of 50: t = L - 52 is seen by the queries 0 and 1 (pos - 50 < t), the first tokens by all
    s = Setup(12, kv, D, 1, 16, [L], layout="record")
    for X in (s.K, s.V):
        X[int(s.table[0, (L - 52) // 16]), :, (L - 52) % 16] = bad
        X[int(s.table[0, 0]), :, 7] = bad
    out = s.attend(q[:1], sink, gate[:1], window=50, first=7)
    want, weight = s.reference(q[:1], sink, gate[:1], window=50, first=7)
    check_out(out[0, 2:], want[0, 2:], weight[0, 2:])
    assert torch.isfinite(out[0, 2:]).all() and not torch.isfinite(out[0, :2]).any()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,D", [(8, 128), (32, 128), (8, 256), (64, 256)])
@pytest.mark.parametrize("C", [1, 2])
def test_tokens_that_nobody_sees_hold_nan(kv, Hq, D, C):
    """Between the first tokens and the windows, also within one 16-token block."""
    window, first, lens = 5, 3, [9, 17, 20, 30, 47, 250]
    s = Setup(21, kv, D, 1, 16, lens, layout="record")
    bad = 0x7F if kv == "e4m3" else math.nan
    for b, L in enumerate(lens):
        seen = set(np.concatenate([PO.visible(L - C + c, window, first) for c in range(C)]).tolist())
        for t in set(range(L)) - seen:
            for X in (s.K, s.V):
                X[int(s.table[b, t // 16]), :, t % 16] = bad
    s.check(C, Hq, window=window, first=first)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("C,Hq,D", [(2, 8, 128), (3, 16, 128), (2, 64, 256), (16, 8, 128), (16, 8, 256)])
def test_queries_apart(kv, C, Hq, D):
    """Each query alone among tokens that only the others of the chunk see, all of them NaN."""
    L, window, first = 90, 21, 2
    bad = 0x7F if kv == "e4m3" else math.nan
    for c in range(0, C, max(1, C // 4)):
        s = Setup(22, kv, D, 1, 16, [L], layout="token")
        q, sink, gate = s.queries(C, Hq, True)
        want, weight = s.reference(q, sink, gate, window, first)
        seen = set(PO.visible(L - C + c, window, first).tolist())
        for t in set(range(L)) - seen:
            for X in (s.K, s.V):
                X[int(s.table[0, t // 16]), :, t % 16] = bad
        out = s.attend(q, sink, gate, window, first)
        check_out(out[:, c], want[:, c], weight[:, c], f"query {c}")


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("C,Hq,D", [(1, 8, 128), (2, 32, 128), (1, 64, 256)])
def test_cache_policies_give_the_same_bits(kv, C, Hq, D, monkeypatch):
    s = Setup(23, kv, D, 2, 16, [3000, 3000, 40, 700, 3001], layout="record")
    s.table[1, :100] = s.table[0, :100]  # a common prompt
    s.dtable = torch.from_numpy(s.table).cuda()
    q, sink, gate = s.queries(C, Hq, True)
    outs = []
    for v in ("0", "1"):
        monkeypatch.setenv("HS2_PAGED_STREAM", v)
        outs.append((s.attend(q, sink, gate), s.attend(q, sink, gate, 1000, 5)))
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    check_out(outs[1][0], *s.reference(q, sink, gate))


def test_negative_and_excessive_lengths():
    s = Setup(13, "bf16", 128, 2, 16, [100, 100, 112], max_pages=7)
    q, _, _ = s.queries(1, 8, False)
    s.dlen = torch.tensor([-5, 100, 1 << 30], dtype=torch.int32, device="cuda")
    out = s.attend(q, None, None)
    s.lens = [0, 100, 112]
    check_out(out, *s.reference(q, None, None))


def test_offsets_past_32_bits():
    """Pages 2^27 + 64 elements apart: byte offsets up to 5 GB."""
    D, P, stride = 128, 20, (1 << 27) + 64
    s = Setup(14, "bf16", D, 1, 16, [300], layout="record", spare=1)
    big = torch.empty((P - 1) * stride + 16 * 2 * D, dtype=torch.bfloat16, device="cuda")
    K = big.as_strided((P, 1, 16, D), (stride, 16 * 2 * D, 2 * D, 1))
    V = big.as_strided((P, 1, 16, D), (stride, 16 * 2 * D, 2 * D, 1), D)
    K.copy_(s.K), V.copy_(s.V)
    s.K, s.V = K, V
    s.check(1, 8)
    k = torch.randn(1, 40, 1, D, device="cuda").to(torch.bfloat16)
    s.dlen.fill_(320 - 20)
    hs2.hs2_paged_append(s.dims(1, 8), k, k * 2, None, s.dtable, s.dlen, K, V)
    row = torch.cat([K[int(p), 0] for p in s.table[0, :19]])[260:300]
    assert torch.equal(row, k[0, :, 0])
    moves = torch.tensor([[int(s.table[0, 18]), int(s.table[0, 0]), 16]], dtype=torch.int32, device="cuda")
    n = torch.ones(1, dtype=torch.int32, device="cuda")
    hs2.hs2_pages_copy(s.dims(1, 8), moves, n, K, V)
    a, e = moves[0, :2].tolist()
    assert torch.equal(K[a].view(torch.int16), K[e].view(torch.int16)) and torch.equal(V[a].view(torch.int16), V[e].view(torch.int16))


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_same_bits_again_and_on_another_stream(kv):
    s = Setup(15, kv, 128, 2, 64, [5000, 20, 777], layout="record")
    q, sink, gate = s.queries(2, 16, True)
    a = s.attend(q, sink, gate)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.full((hs2.hs2_paged_workspace_bytes(s.dims(2, 16)),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    b = s.attend(q, sink, gate, ws=ws, out=torch.empty_like(q), stream=side)
    side.synchronize()
    assert torch.equal(a, b)


def test_graphs_that_share_a_workspace():
    s = Setup(16, "bf16", 128, 2, 64, [6000, 300], layout="record")
    q, sink, gate = s.queries(1, 16, True)
    ws = torch.empty(hs2.hs2_paged_workspace_bytes(s.dims(1, 16)), dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.empty_like(q) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    spans = [(None, 0), (2000, 4)]
    for span, out in zip(spans, outs):
        s.attend(q, sink, gate, *span, out=out, ws=ws)
    torch.cuda.synchronize()
    for g, span, out in zip(graphs, spans, outs):
        with torch.cuda.graph(g):
            s.attend(q, sink, gate, *span, out=out, ws=ws)
    for rep in range(3):
        q.copy_(torch.randn_like(q))
        s.dlen.copy_(torch.tensor([6000 - 50 * rep, 300 - rep], dtype=torch.int32))
        for g in graphs + graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for span, out in zip(spans, outs):
            assert torch.equal(out, s.attend(q, sink, gate, *span))
            torch.cuda.synchronize()


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("T,ragged", [(1, False), (2, True), (70, False), (70, True)])
@pytest.mark.parametrize("layout", ["record", "token", "apart"])
def test_append(kv, D, T, ragged, layout):
    s = Setup(T + D, kv, D, 3, 16, [0, 1, 69, 71, 160, 100], layout=layout, poison=False)
    s.table[3, 2] = -1  # dropped
    s.table[4, 9] = s.n_pages
    s.dtable = torch.from_numpy(s.table).cuda()
    if ragged:
        n_new = torch.tensor([3, 1, 0, -4, 1 << 30, 40], dtype=torch.int32, device="cuda")
    else:
        n_new = None
    wide = torch.randn(6, T, 5, 3, D, device="cuda", generator=s.gen).to(torch.bfloat16)  # slices of a wider projection
    k, v = wide[:, :, 1], wide[:, :, 4]
    want = [X.clone().cpu() for X in (s.K, s.V)]
    scales = None if s.scales is None else [x.double().cpu().numpy() for x in s.scales]

    def convert(row, g, which):
        return row if scales is None else torch.from_numpy(PO.to_e4m3(row.double().numpy(), float(scales[which][g])))
    PO.append(*want, k.cpu(), v.cpu(), None if n_new is None else n_new.tolist(), s.table, s.lens, 16, convert)
    sc = () if s.scales is None else s.scales
    f = hs2.hs2_paged_append if s.scales is None else hs2.hs2_paged_append_fp8
    f(s.dims(1, 3), k, v, n_new, *sc, s.dtable, s.dlen, s.K, s.V)
    for X, Y in zip((s.K, s.V), want):
        bits = (lambda t: t.contiguous().view(torch.uint8)) if s.scales is not None else (lambda t: t.contiguous().view(torch.int16))
        assert torch.equal(bits(X.cpu()), bits(Y))


def test_append_of_one_token_and_one_sequence_has_any_stride():
    """Extents of one carry any stride."""
    s = Setup(31, "bf16", 128, 2, 16, [33], layout="record", poison=False)
    raw = torch.randn(2, 2, 128, device="cuda").to(torch.bfloat16)
    k, v = torch.as_strided(raw[0], (1, 1, 2, 128), (3, 5, 128, 1)), raw[1].view(1, 1, 2, 128)
    hs2.hs2_paged_append(s.dims(1, 2), k, v, None, s.dtable, s.dlen, s.K, s.V)
    p = int(s.table[0, 2])
    assert torch.equal(s.K[p, :, 0], raw[0]) and torch.equal(s.V[p, :, 0], raw[1])
    with pytest.raises(hs2.HS2Error):
        wide = torch.zeros(1, 2, 2, 132, dtype=torch.bfloat16, device="cuda")[..., :128]
        hs2.hs2_paged_append(s.dims(1, 2), wide, wide, None, s.dtable, s.dlen, s.K, s.V)


def test_binding_refusals():
    s = Setup(32, "bf16", 128, 2, 16, [33, 7], layout="record")
    q, sink, gate = s.queries(1, 8, True)
    out, d = torch.empty_like(q), s.dims(1, 8)
    ws = torch.empty(hs2.hs2_paged_workspace_bytes(d), dtype=torch.uint8, device="cuda")

    def call(**kw):
        a = dict(q=q, K=s.K, V=s.V, table=s.dtable, len=s.dlen, sink=sink, gate=gate, out=out, ws=ws)
        a.update(kw)
        hs2.hs2_paged_attn(d, *a.values())
    call()
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(q=q[:1]), dict(q=q.transpose(2, 3)), dict(K=s.K[:-1, :1, :1].clone()),
                dict(V=s.V.view(torch.float16)), dict(table=s.dtable.long()), dict(table=s.dtable[:, :-1]),
                dict(len=s.dlen.cpu()), dict(sink=sink[:-1]), dict(sink=sink.double()), dict(gate=gate[..., :64]),
                dict(out=out.transpose(0, 1)), dict(ws=None), dict(ws=ws[::2])):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(hs2.HS2Error) as e:
        call(ws=ws[:0])
    assert e.value.status == hs2.HS2_ERR_WORKSPACE or e.value.status == hs2.HS2_ERR_NULL
    with pytest.raises(hs2.HS2Error):
        hs2.hs2_paged_window_attn(d, q, s.K, s.V, s.dtable, s.dlen, 0, 0, None, None, out, ws)


@pytest.mark.parametrize("scale", [1.0, 0.0123, 1 / 3, 7.7e-3, 3.0e5, 1e-30])
def test_every_bf16_value_to_e4m3(scale):
    """All 65536 bit patterns: ties, subnormals, saturation, infinities, NaN."""
    D, page = 128, 256
    pool = torch.zeros(2, 1, page, D, dtype=torch.uint8, device="cuda")
    V = torch.zeros_like(pool)
    bits = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16)
    k = bits.view(torch.bfloat16).view(1, 512, 1, D)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([512], dtype=torch.int32, device="cuda")
    s = torch.tensor([scale], device="cuda")
    d = hs2.make_paged_dims(1, 1, 1, 1, D, page, 2, 2)
    hs2.hs2_paged_append_fp8(d, k, k, None, s, s, table, lens, pool, V)
    got = torch.cat([pool[1, 0], pool[0, 0]]).flatten().cpu().numpy()
    x = k.float().double().flatten().cpu().numpy()
    want = PO.to_e4m3(x, float(s.double()))
    nan = np.isnan(x)
    assert ((got[nan] & 0x7F) == 0x7F).all()
    np.testing.assert_array_equal(got[~nan], want[~nan])
    assert torch.equal(pool, V)


# ------------------------------------------------------------------ page operators
def state(rng, R, M, P, page, shared=0.2):
    """A consistent random state: some rows share leading pages, some pages are held from outside."""
    order, at = rng.permutation(P), 0
    table, lens = np.full((R, M), -1, np.int32), np.zeros(R, np.int32)
    for b in range(R):
        n = min(int(rng.integers(0, M * page + 1)), (P - at) // 2 // max(1, R // 8) * page)
        lens[b] = n
        pages, k = -(-n // page), 0
        if b and rng.random() < shared:
            k = min(int(lens[b - 1]) // page, n // page)
            table[b, :k] = table[b - 1, :k]
        table[b, k:pages] = order[at:at + pages - k]
        at += pages - k
    refs = np.bincount(table[table >= 0], minlength=P)
    held = order[at:][rng.random(P - at) < 0.2]
    refs[held] = 1
    return table, lens, refs.astype(np.int32)


def dev(*arrays):
    return [torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda() for a in arrays]


STATES = [(1, 3, 5, 16), (1, 1, 1, 16), (7, 9, 50, 32), (40, 30, 700, 16), (300, 20, 4096, 64), (65, 33, 4097, 16), (64, 200, 9000, 16),
          (3, 2000, 20001, 16)]


def ws_for(d):
    return torch.full((hs2.hs2_paged_workspace_bytes(d),), 255, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("R,M,P,page", STATES)
def test_extend(R, M, P, page, inplace):
    rng = np.random.default_rng(R * 31 + P)
    table, lens, refs = state(rng, R, M, P, page)
    for more in (1, page, M * page):  # the last: more than the pool has, most of the time
        want = np.minimum(lens + rng.integers(0, more + 1, R), M * page)
        d = hs2.make_paged_dims(R, 1, 1, 1, 128, page, P, M)
        t, n, r = dev(table, want, refs)
        to, ro = (t, r) if inplace else (torch.full_like(t, 77), torch.full_like(r, 77))
        counts = torch.full((2,), 77, dtype=torch.int32, device="cuda")
        hs2.hs2_pages_extend(d, t, n, r, to, ro, counts, ws_for(d))
        et, er, ec = PO.extend(table.tolist(), want.tolist(), refs.tolist(), page)
        assert counts.tolist() == ec and to.tolist() == et and ro.tolist() == er


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("R,M,P,page", STATES)
@pytest.mark.parametrize("kind", ["beams", "random", "one", "nothing", "keep", "all_free"])
def test_reorder(R, M, P, page, inplace, kind):
    rng = np.random.default_rng(R * 17 + P + len(kind))
    table, lens, refs = state(rng, R, M, P, page)
    parent = {"beams": np.minimum(np.arange(R) // 4 * 4 + rng.integers(0, 4, R), R - 1),
              "random": rng.integers(-1, R + 1, R), "one": np.full(R, R // 2), "nothing": np.full(R, -1),
              "keep": np.arange(R), "all_free": np.where(rng.random(R) < 0.5, 2 ** 31 - 1, -2 ** 31)}[kind]
    if R > 2 and kind == "random":  # a hole in a row, and in the place of a partial page
        if lens[1] > page:
            refs[table[1, 0]] -= 1
            table[1, 0] = -1
        if lens[2] % page:
            refs[table[2, lens[2] // page]] -= 1
            table[2, lens[2] // page] = -1
    d = hs2.make_paged_dims(R, 1, 1, 1, 128, page, P, M)
    pa, t, n, r = dev(parent, table, lens, refs)
    to, no = torch.full_like(t, 77), torch.full_like(n, 77)
    ro = r if inplace else torch.full_like(r, 77)
    moves, counts = torch.full((R + 3, 3), 77, dtype=torch.int32, device="cuda"), torch.full((2,), 77, dtype=torch.int32, device="cuda")
    hs2.hs2_pages_reorder(d, pa, t, n, r, to, no, ro, moves, counts, ws_for(d))
    et, en, er, em, ec = PO.reorder(parent.tolist(), table.tolist(), lens.tolist(), refs.tolist(), page)
    assert counts.tolist() == ec and to.tolist() == et and no.tolist() == en and ro.tolist() == er
    assert moves[:ec[0]].tolist() == em and (moves[ec[0]:] == 77).all()
    assert t.tolist() == table.tolist() and n.tolist() == lens.tolist()


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("R,M,P,page", STATES)
def test_compact(R, M, P, page, inplace):
    rng = np.random.default_rng(R * 13 + P)
    table, lens, refs = state(rng, R, M, P, page)
    drop = rng.random(R) < 0.4  # finished sequences leave holes
    for b in np.flatnonzero(drop):
        np.subtract.at(refs, table[b][table[b] >= 0], 1)
        table[b] = -1
    if M > 1:
        table[-1, -1] = 2 ** 31 - 1  # no page: stays what it is
    d = hs2.make_paged_dims(R, 1, 1, 1, 128, page, P, M)
    t, r = dev(table, refs)
    to, ro = (t, r) if inplace else (torch.full_like(t, 77), torch.full_like(r, 77))
    moves = torch.full((P // 2 + 1, 3), 77, dtype=torch.int32, device="cuda")
    counts = torch.full((2,), 77, dtype=torch.int32, device="cuda")
    hs2.hs2_pages_compact(d, t, r, to, ro, moves, counts, ws_for(d))
    et, er, em, ec = PO.compact(table.tolist(), refs.tolist(), page)
    assert counts.tolist() == ec and to.tolist() == et and ro.tolist() == er
    assert moves[:ec[0]].tolist() == em and (moves[ec[0]:] == 77).all()


@pytest.mark.parametrize("P", [4096, 8192, 12289])
@pytest.mark.parametrize("used", ["front", "back", "all", "none", "every_other"])
def test_compact_at_chunk_edges(P, used):
    refs = np.zeros(P, np.int32)
    refs[{"front": slice(0, 4096), "back": slice(P - 4096, P), "all": slice(0, P), "none": slice(0, 0), "every_other": slice(0, P, 2)}[used]] = 2
    table = np.arange(P, dtype=np.int32)[None]
    d = hs2.make_paged_dims(1, 1, 1, 1, 128, 16, P, P)
    t, r = dev(table, refs)
    moves, counts = torch.full((P // 2, 3), 77, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    to, ro = torch.empty_like(t), torch.empty_like(r)
    hs2.hs2_pages_compact(d, t, r, to, ro, moves, counts, ws_for(d))
    et, er, em, ec = PO.compact(table.tolist(), refs.tolist(), 16)
    assert counts.tolist() == ec and to.tolist() == et and ro.tolist() == er and moves[:ec[0]].tolist() == em


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.uint8])
@pytest.mark.parametrize("D,Hkv,page", [(128, 3, 16), (256, 1, 64), (128, 8, 256)])
@pytest.mark.parametrize("layout", ["record", "token"])
def test_copy(dtype, D, Hkv, page, layout):
    P, rng = 60, np.random.default_rng(D + page)
    shape = (P, Hkv, page, 2 * D) if layout == "record" else (2, P, page, Hkv, D)
    raw = torch.randint(0, 256, (*shape[:-1], shape[-1] * dtype.itemsize), dtype=torch.uint8, device="cuda").view(dtype)
    K, V = (raw[..., :D], raw[..., D:]) if layout == "record" else (raw[0].transpose(1, 2), raw[1].transpose(1, 2))
    order = rng.permutation(P)
    moves = np.stack([order[:25], order[25:50], rng.integers(0, page + 1, 25)], 1)
    moves[3, 2], moves[4, 2], moves[5, 2] = page, -3, page + 9
    moves[6, 0], moves[7, 1], moves[8, 0], moves[9, 1] = -1, P, 2 ** 31 - 1, -2 ** 31
    before = [X.clone().contiguous().view(torch.uint8) for X in (K, V)]
    d = hs2.make_paged_dims(1, 1, Hkv, Hkv, D, page, P, 1, tuple(K.stride()[:3]))
    m, = dev(moves)
    for n, done in ((0, 0), (-4, 0), (20, 20), (1000, 25)):
        hs2.hs2_pages_copy(d, m, torch.tensor([n], dtype=torch.int32, device="cuda"), K, V)
        want = [x.clone() for x in before]
        for a, e, tokens in moves[:done]:
            if 0 <= a < P and 0 <= e < P:
                tokens = min(max(tokens, 0), page)
                for x in want:
                    x[e, :, :tokens] = x[a, :, :tokens]
        for X, x in zip((K, V), want):
            assert torch.equal(X.contiguous().view(torch.uint8), x)


@pytest.mark.parametrize("dtype,P", [(torch.bfloat16, 80), (torch.uint8, 150)])
def test_copy_past_the_caches(dtype, P):
    """Moves on both sides of half the last-level cache (32 and 64 of these pages), pages of odd lengths among them."""
    D, Hkv, page = 256, 8, 256
    raw = torch.randint(0, 256, (P, Hkv, page, 2 * D * dtype.itemsize), dtype=torch.uint8, device="cuda").view(dtype)
    K, V = raw[..., :D], raw[..., D:]
    before = raw.view(torch.uint8).clone()
    order = np.random.default_rng(P).permutation(P)
    n = P // 2
    tokens = np.full(n, page)
    tokens[1], tokens[2], tokens[5], tokens[n - 1] = 0, 1, 37, 255
    moves = np.stack([order[:n], order[n:2 * n], tokens], 1)
    d = hs2.make_paged_dims(1, 1, Hkv, Hkv, D, page, P, 1, tuple(K.stride()[:3]))
    m, = dev(moves)
    edge = 32 if dtype == torch.bfloat16 else 64
    for k in (edge, edge + 1, n):
        hs2.hs2_pages_copy(d, m, torch.tensor([k], dtype=torch.int32, device="cuda"), K, V)
        want = before.clone()
        for a, e, t in moves[:k]:
            want[e, :, :t] = want[a, :, :t]
        assert torch.equal(raw.view(torch.uint8), want)


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("graph", [False, True])
def test_decode_loop_with_beams(kv, graph):
    """Prompts, then steps of extend, append, both kinds of attention, a beam reorder and now and then a compaction,
    against sequences that the test keeps as whole float64 arrays."""
    B, Hq, Hkv, D, page, M = 6, 8, 2, 128, 16, 12
    gen = torch.Generator(device="cuda").manual_seed(3)
    rng = np.random.default_rng(3)
    scales = None if kv == "bf16" else (torch.tensor([0.011, 0.013], device="cuda"), torch.tensor([0.012, 0.009], device="cuda"))
    cache = hs2.PagedCache(B, Hq, Hkv, D, page, n_pages=70, max_pages=M, kv_scales=scales)
    for X in (cache.K, cache.V):
        X.copy_(torch.full_like(X, math.nan if kv == "bf16" else 0x7F))
    sink = torch.randn(Hq, device="cuda", generator=gen)

    def stored(x, which):
        if scales is None:
            return x.double().cpu().numpy()
        x = (x.double() / scales[which].double()[:, None]).cpu().numpy()
        return PO.e4m3_values()[PO.to_e4m3(x, 1.0)] * scales[which].double().cpu().numpy()[:, None]
    seqs = [[np.zeros((0, Hkv, D)) for _ in range(2)] for _ in range(B)]
    T = 50
    k, v = (torch.randn(B, T, Hkv, D, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
    n_new = torch.tensor([50, 3, 17, 32, 1, 16], dtype=torch.int32, device="cuda")
    cache.extend(n_new)
    cache.append(k, v, n_new)
    for b, n in enumerate(n_new.tolist()):
        seqs[b] = [np.concatenate([seqs[b][i], stored(x[b, :n], i)]) for i, x in enumerate((k, v))]
    C = 2
    q = torch.empty(B, C, Hq, D, dtype=torch.bfloat16, device="cuda")
    kn, vn = (torch.empty(B, C, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    parent = torch.zeros(B, dtype=torch.int32, device="cuda")
    outs = [torch.empty_like(q) for _ in range(2)]
    missing = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step():
        cache.reorder(parent)
        missing.add_(cache.counts[1:])
        cache.extend(C)
        missing.add_(cache.counts[1:])
        cache.append(kn, vn)
        cache.attend(q, sink=sink, out=outs[0])
        cache.attend(q, window=20, first=3, sink=sink, out=outs[1])
    g = None
    for i in range(12):
        for x in (q, kn, vn):
            x.copy_(torch.randn(x.shape, device="cuda", generator=gen))
        par = [int(rng.integers(0, B)) if rng.random() < 0.4 else b for b in range(B)]
        par[int(rng.integers(0, B))] = -1
        parent.copy_(torch.tensor(par, dtype=torch.int32))
        if graph and i == 0:  # the capture records the work, the replay does it
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
        if graph:
            g.replay()
        else:
            step()
        torch.cuda.synchronize()
        seqs = [[np.concatenate([seqs[p][i] if p >= 0 else np.zeros((0, Hkv, D)), stored(x[b], i)])
                 for i, x in enumerate((kn, vn))] for b, p in enumerate(par)]
        assert missing.item() == 0 and cache.len.tolist() == [len(s[0]) for s in seqs]
        for b in range(B):
            Kp, Vp = (np.ascontiguousarray(x.transpose(1, 0, 2))[None] for x in seqs[b])
            for out, span in zip(outs, ((None, 0), (20, 3))):
                want, weight = PO.attention(q[b:b + 1].double().cpu().numpy(), Kp, Vp, [[0]], [Kp.shape[2]], Kp.shape[2],
                                            1 / math.sqrt(D), *span, sink=sink.double().cpu().numpy())
                check_out(out[b:b + 1], want, weight, f"step {i} sequence {b}")
        if i % 4 == 3:
            cache.compact()
            used = cache.counts.tolist()[1]
            assert (cache.refs[:used] > 0).all() and not cache.refs[used:].any()
