"""The paged cache without a GPU: sizes and refusals of the C ABI, the binding's checks, the oracle's own pins."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2609_26368_amd import hs2

FAKE = 1 << 20  # a 256-byte aligned non-null address; never dereferenced on the error paths
N, S, U, W, A = (hs2.HS2_ERR_NULL, hs2.HS2_ERR_SHAPE, hs2.HS2_ERR_UNSUPPORTED, hs2.HS2_ERR_WORKSPACE, hs2.HS2_ERR_ALIGN)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hs2.LIB_PATH):
        from paper_2609_26368_amd import _build
        _build.build()
    return hs2.load()


def dims(**kw):
    base = dict(batch=2, n_queries=1, n_q_heads=32, n_kv_heads=4, head_dim=128, page=64, n_pages=100, max_pages=40,
                kv_strides=None, scale=0.0)
    base.update(kw)
    return hs2.make_paged_dims(**base)


BAD_DIMS = [(dict(page=8), S), (dict(page=48), S), (dict(page=512), S), (dict(n_pages=0), S),
            (dict(n_pages=(1 << 24) + 1), S), (dict(max_pages=0), S), (dict(max_pages=(1 << 21) + 1), S),
            (dict(batch=0), S), (dict(n_queries=0), S), (dict(n_queries=17), S), (dict(n_q_heads=30), S),
            (dict(head_dim=64), U), (dict(n_q_heads=65 * 4), U), (dict(n_queries=16, n_q_heads=64), U),
            (dict(batch=20000), U), (dict(scale=float("nan")), S), (dict(kv_strides=(-8, 128, 128)), A),
            (dict(kv_strides=(8196, 128, 128)), A), (dict(kv_strides=(8192, 132, 128)), A),
            (dict(kv_strides=(8192, 128, 120)), A), (dict(kv_strides=(8192, 128, (1 << 24) + 8)), U)]


def _p(v):
    return ctypes.c_void_p(v)


def call(lib, name, d, **kw):
    """Calls `name` with FAKE addresses but for those in kw."""
    orders = {
        "hs2_paged_attn": "q K V table len sink gate out ws WS stream",
        "hs2_paged_attn_fp8": "q K V ks vs table len sink gate out ws WS stream",
        "hs2_paged_window_attn": "q K V table len WINDOW FIRST sink gate out ws WS stream",
        "hs2_paged_window_attn_fp8": "q K V ks vs table len WINDOW FIRST sink gate out ws WS stream",
        "hs2_paged_append": "k_new v_new SB ST SH TOKENS n_new table len K V stream",
        "hs2_paged_append_fp8": "k_new v_new SB ST SH TOKENS n_new ks vs table len K V stream",
        "hs2_pages_extend": "table len refs table_out refs_out counts ws WS stream",
        "hs2_pages_reorder": "parent table len refs table_out len_out refs_out moves MOVES counts ws WS stream",
        "hs2_pages_compact": "table refs table_out refs_out moves MOVES counts ws WS stream",
        "hs2_pages_copy": "moves n_moves MOVES ELEM K V stream"}
    values = dict(WINDOW=128, FIRST=4, SB=4096, ST=512, SH=128, TOKENS=1, WS=1 << 40, MOVES=1000, ELEM=2, sink=None, gate=None,
                  n_new=None, stream=None, table_out=2 * FAKE, len_out=2 * FAKE)
    values.update(kw)
    args = [values.get(a, FAKE) for a in orders[name].split()]
    args = [v if a.isupper() else _p(v) for a, v in zip(orders[name].split(), args)]
    return getattr(lib, name)(None if d is None else ctypes.byref(d), *args)


CALLS = ["hs2_paged_attn", "hs2_paged_attn_fp8", "hs2_paged_window_attn", "hs2_paged_window_attn_fp8",
         "hs2_paged_append", "hs2_paged_append_fp8", "hs2_pages_extend", "hs2_pages_reorder", "hs2_pages_compact",
         "hs2_pages_copy"]


@pytest.mark.parametrize("name", CALLS)
def test_bad_dims(lib, name):
    assert call(lib, name, None) == N
    for bad, status in BAD_DIMS:
        assert call(lib, name, dims(**bad)) == status, bad
        assert hs2.hs2_last_error()


def test_workspace_bytes(lib):
    n = hs2.hs2_paged_workspace_bytes(dims())
    assert n > 0 and n % 256 == 0
    assert hs2.hs2_paged_workspace_bytes(dims(n_pages=1 << 24)) > n
    for bad, _ in BAD_DIMS:
        assert hs2.hs2_paged_workspace_bytes(dims(**bad)) == 0, bad


REQUIRED = {"hs2_paged_attn": "q K V table len out ws", "hs2_paged_attn_fp8": "q K V ks vs table len out ws",
            "hs2_paged_window_attn": "q K V table len out ws",
            "hs2_paged_window_attn_fp8": "q K V ks vs table len out ws",
            "hs2_paged_append": "k_new v_new table len K V", "hs2_paged_append_fp8": "k_new v_new ks vs table len K V",
            "hs2_pages_extend": "table len refs table_out refs_out counts ws",
            "hs2_pages_reorder": "parent table len refs table_out len_out refs_out moves counts ws",
            "hs2_pages_compact": "table refs table_out refs_out moves counts ws", "hs2_pages_copy": "moves n_moves K V"}


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned(lib, name):
    for arg in REQUIRED[name].split():
        assert call(lib, name, dims(), **{arg: None}) == N, arg
        assert call(lib, name, dims(), **{arg: FAKE + 2}) == A, arg
    if "ws" in REQUIRED[name].split():
        assert call(lib, name, dims(), WS=100) == W


def test_other_refusals(lib):
    d = dims()
    for name in ("hs2_paged_attn", "hs2_paged_window_attn"):
        assert call(lib, name, d, sink=FAKE + 2) == A
        assert call(lib, name, d, gate=FAKE + 4) == A
    for name in ("hs2_paged_window_attn", "hs2_paged_window_attn_fp8"):
        for bad in (dict(WINDOW=0), dict(WINDOW=-1), dict(WINDOW=(1 << 27) + 1), dict(FIRST=-1), dict(FIRST=(1 << 27) + 1)):
            assert call(lib, name, d, **bad) == S
    for name in ("hs2_paged_append", "hs2_paged_append_fp8"):
        assert call(lib, name, d, TOKENS=0) == S
        assert call(lib, name, d, TOKENS=1 << 26) == S
        assert call(lib, name, d, TOKENS=(1 << 27) // d.n_kv_heads) == S
        for bad in (dict(SB=4), dict(ST=-8), dict(SH=12), dict(n_new=FAKE + 1)):
            assert call(lib, name, d, **bad) == A
    for name in ("hs2_paged_attn_fp8", "hs2_paged_window_attn_fp8", "hs2_paged_append_fp8"):  # 16-element strides
        assert call(lib, name, dims(kv_strides=(8200, 128, 128))) == A
        assert call(lib, name, dims(kv_strides=(8192, 136, 128))) == A
        assert call(lib, name, dims(kv_strides=(8192, 128, 136))) == A
    assert call(lib, "hs2_pages_reorder", d, table_out=FAKE) == S  # the table itself
    assert call(lib, "hs2_pages_reorder", d, len_out=FAKE) == S
    assert call(lib, "hs2_pages_reorder", d, MOVES=1) == S
    assert call(lib, "hs2_pages_compact", d, MOVES=49) == S
    assert call(lib, "hs2_pages_copy", d, MOVES=-1) == S
    assert call(lib, "hs2_pages_copy", d, ELEM=4) == S
    assert call(lib, "hs2_pages_copy", dims(kv_strides=(8200, 128, 128)), ELEM=1) == A


def test_binding_refuses_tensors_elsewhere(lib):
    d = dims()
    q = torch.zeros(2, 1, 32, 128, dtype=torch.bfloat16)
    K = torch.zeros(100, 4, 64, 128, dtype=torch.bfloat16)
    table, lens = torch.zeros(2, 40, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    refs, counts, ws = torch.zeros(100, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(1 << 20)
    moves = torch.zeros(50, 3, dtype=torch.int32)
    new = torch.zeros(2, 1, 4, 128, dtype=torch.bfloat16)
    for f in (lambda: hs2.hs2_paged_attn(d, q, K, K, table, lens, None, None, q, ws),
              lambda: hs2.hs2_paged_window_attn(d, q, K, K, table, lens, 5, 0, None, None, q, ws),
              lambda: hs2.hs2_paged_append(d, new, new, None, table, lens, K, K),
              lambda: hs2.hs2_pages_extend(d, table, lens, refs, table, refs, counts, ws),
              lambda: hs2.hs2_pages_reorder(d, lens, table, lens, refs, table, lens, refs, moves, counts, ws),
              lambda: hs2.hs2_pages_compact(d, table, refs, table, refs, moves, counts, ws),
              lambda: hs2.hs2_pages_copy(d, moves, counts, K, K)):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            f()


# ------------------------------------------------------------------ the oracle
def test_e4m3_bytes_agree_with_torch():
    every = np.arange(256, dtype=np.uint8)
    got = torch.from_numpy(every).view(torch.float8_e4m3fn).float().double().numpy()
    np.testing.assert_array_equal(got, PO.e4m3_values())
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(0, 60, 4000), PO.e4m3_values()[:127], [0.0, -0.0, 1e9, -1e9, 2.0 ** -10, 3 * 2.0 ** -10]])
    x = x.astype(np.float32)
    want = torch.from_numpy(np.clip(x, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(PO.to_e4m3(x, 1.0), want)
    assert PO.to_e4m3(np.array([np.nan]), 1.0)[0] & 0x7F == 0x7F


def test_visible_tokens():
    assert PO.visible(-1, None, 0).size == 0
    assert list(PO.visible(5, 2, 1)) == [0, 4, 5]
    assert list(PO.visible(5, 100, 3)) == list(range(6))
    assert list(PO.visible(5, 1, 0)) == [5]
    assert list(PO.visible(5, 2, 9)) == list(range(6))


def test_attention_pins():
    rng = np.random.default_rng(1)
    K, V, q = rng.normal(size=(3, 1, 16, 128)), rng.normal(size=(3, 1, 16, 128)), rng.normal(size=(1, 1, 2, 128))
    out, _ = PO.attention(q, K, V, [[2, 0]], [1], 16, 0.1)
    np.testing.assert_allclose(out[0, 0, 0], V[2, 0, 0])  # one token: its value
    out, _ = PO.attention(q * 0, K, V, [[2, 0]], [18], 16, 0.1)
    np.testing.assert_allclose(out[0, 0, 1], np.concatenate([V[2, 0], V[0, 0, :2]]).mean(0))  # equal logits: the mean
    out, _ = PO.attention(q * 0, K, V, [[7, 0]], [18], 16, 0.1)  # the first page is none
    np.testing.assert_allclose(out[0, 0, 1], V[0, 0, :2].mean(0))
    out, _ = PO.attention(q, K, V, [[2, 0]], [0], 16, 0.1, sink=np.zeros(2))
    assert not out.any()
    out, _ = PO.attention(q * 0, K, V, [[2, 0]], [1], 16, 0.1, sink=np.zeros(2), gate=np.zeros((1, 1, 2, 128)))
    np.testing.assert_allclose(out[0, 0, 0], V[2, 0, 0] / 4)  # the sink's half, the gate's half


def test_page_operators_keep_the_counts():
    """refs is always how many entries name a page, through a random run of all three."""
    rng = np.random.default_rng(2)
    page, R, M, P = 16, 7, 6, 30
    table, lens, refs = [[-1] * M for _ in range(R)], [0] * R, [0] * P
    for step in range(200):
        lens = [min(M * page, n + int(rng.integers(0, 20))) for n in lens]
        table, refs, (given, missing) = PO.extend(table, lens, refs, page)
        lens = [min(n, page * sum(p >= 0 for p in r)) for n, r in zip(lens, table)]
        parent = [int(rng.integers(-1, R)) if rng.random() < 0.3 else b for b in range(R)]
        table, lens, refs, moves, _ = PO.reorder(parent, table, lens, refs, page)
        assert len({m[1] for m in moves}) == len(moves)
        table, refs, moves, (n, used) = PO.compact(table, refs, page)
        flat = [p for r in table for p in r if p >= 0]
        assert [flat.count(p) for p in range(P)] == refs and all(r > 0 for r in refs[:used]) and not any(refs[used:])
        for n, r in zip(lens, table):
            assert all(p >= 0 for p in r[:-(-n // page)])
