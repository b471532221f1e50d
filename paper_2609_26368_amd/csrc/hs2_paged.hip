// HIP kernels of the paged KV cache (gfx950).
//
//   k_paged_attn     attention of the new tokens over a sequence's pages, split over
//                    its length; k_paged_merge joins the splits
//   k_paged_append   new K and V rows to their slots (bf16, or quantised to E4M3)
//   k_pages_scan     lists the free pages of each chunk of the pool (compaction:
//                    counts the used ones) and what each table row wants
//   k_pages_extend   gives rows free pages
//   k_pages_reorder  rows take over their parents' entries
//   k_pages_list, k_pages_compact   moves that pack the pool; table and counts after them
//   k_pages_copy     the moves' contents
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "hs2_device.h"
#include "hs2_launch.h"

namespace hs2 {
namespace {

constexpr int NTP = 256;  // threads per workgroup of this file's kernels

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline int paged_len(const PagedPool& p, int b) {
  const int L = p.len[b], cap = p.page * p.max_pages;
  return L < 0 ? 0 : (L > cap ? cap : L);
}
__device__ inline bool is_page(int id, int n_pages) { return (uint32_t)id < (uint32_t)n_pages; }

// ============================================================================ attention
// Softmax attention of a chunk's queries over the pages of their sequence,
// one pass over K and V with a running maximum and sum per query row:
//   s_t = c2 <q, k_t>,  m' = max(m, s_t),  l' = l 2^(m - m') + 2^(s_t - m'),
//   o' = o 2^(m - m') + 2^(s_t - m') v_t,  out = o / l   (c2 = scale log2 e).
// Bound by reading K and V once: G C operations a byte of a bf16 cache, far
// below the matrix units' rate.  2 x 512K tokens (4.3 GB) 630 us, 6.8 TB/s; 64
// sequences of 1000 to 12000 (1.7 GB) 271 to 280 us.  E4M3 with several row
// tiles is bound by the vector work of the conversions (4 x 128K tokens, 64 rows
// a KV head, 0.54 GB: 121 to 128 us, 4.2 to 4.4 TB/s).
//
// Tokens are taken in blocks of 16, which never straddle a page.  The blocks
// that some query of the chunk sees are numbered through: nf blocks of first
// tokens, then those from the start of the earliest query's window on.  A
// sequence's blocks are cut into splits of S (PagedSplit); a workgroup takes
// one split of one KV head.  Its TGW token groups take every TGW-th tile of
// TW tokens through an LDS ring of their own, and the NWV waves of a group
// share its tiles, RPW row tiles of 16 query rows each.  A group of one wave
// needs no barrier.  The groups meet in LDS; a KV head of one split is
// finished there, of more it leaves partial rows for k_paged_merge.
//
// What a query does not see must not reach it, and 0 x NaN is NaN: rows that no
// query sees are never loaded (they repeat a visible row of their block, or are
// zero rows), and a tile of which the queries see different rows (the last
// tokens of a chunk, the starts of its windows) whose V is not finite is
// emptied and left to a second loop, which takes the queries one by one.  (With
// both products in one loop the compiler kept O twice, 154 registers a lane
// for one row tile of head dim 128 instead of 120.)

// What stands in for rows that are not loaded.
__device__ const uint4 zero_row[32] = {};

// The visible blocks of a sequence with Lv tokens.
struct PagedSpan {
  int nf, w0, n;  // blocks of first tokens, first block of the window, all of them
  int lo;         // the earliest token of any window
};
__device__ inline PagedSpan paged_span(const PagedAttnArgs& a, int Lv) {
  PagedSpan s;
  const int pos0 = max(0, Lv - a.C);  // the earliest query that sees anything
  s.lo = a.window > 0 ? max(0, pos0 - a.window + 1) : 0;
  s.w0 = s.lo / 16;
  s.nf = min((a.first + 15) / 16, s.w0);
  s.n = s.nf + (Lv + 15) / 16 - s.w0;
  return s;
}
__device__ inline int token_block(const PagedSpan& s, int i) { return i < s.nf ? i : i - s.nf + s.w0; }

// Sums over the wave of a value per sequence; f(blocks) of sequences lane, lane + 64, ...
template <class F>
__device__ inline int wave_sum_sequences(const PagedAttnArgs& a, int n0, F&& f) {
  const int lane = threadIdx.x & 63;
  int s = lane < a.p.B ? f(n0) : 0;
  for (int b = lane + 64; b < a.p.B; b += 64) s += f(paged_span(a, paged_len(a.p, b)).n);
  return wave_sum(s);
}
__device__ inline int splits_at(int n, int S) { return max(1, (int)((uint32_t)(n + S - 1) / (uint32_t)S)); }

// Blocks per split, 0 if workgroup `item` has nothing to do.  Either the longest
// sequence's (every KV head is one split), or the shortest multiple of align, at
// least min_blocks, whose (sequence, KV head, split) items number at most what
// paged_items says (few tokens: down to align).  items(S) lies between total / S
// and total / S + units, which brackets the search.
__device__ inline int paged_split_blocks(const PagedAttnArgs& a, int n0, int item) {
  const PagedSplit& sp = a.sp;
  if (sp.fixed) return sp.fixed;
  const int units = a.p.B * a.p.Hkv;
  float tot = 0.f;
  int longest = 0;
  {
    const int lane = threadIdx.x & 63;
    if (lane < a.p.B) tot = (float)(longest = n0);
    for (int b = lane + 64; b < a.p.B; b += 64) {
      const int n = paged_span(a, paged_len(a.p, b)).n;
      tot += (float)n;
      longest = max(longest, n);
    }
    tot = wave_sum(tot) * (float)a.p.Hkv;
    longest = wave_max(longest);
  }
  const int n_items = paged_items(sp, tot, units, (float)longest);
  if (n_items == 0) return item < units ? max(1, longest) : 0;
  if (item >= n_items) return 0;
  const bool few = n_items == sp.few_items && tot <= (float)sp.min_blocks * (float)n_items;
  const float n = (float)n_items, al = (float)sp.align;
  int lo = max(few ? 1 : sp.min_blocks / sp.align, (int)(tot * (0.9999f / (n * al))));
  int hi = (sp.cap_blocks + sp.align - 1) / sp.align;
  if (n_items > units) hi = min(hi, (int)fminf(tot * (1.0001f / ((n - (float)units) * al)), 1e9f) + 1);
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(max(hi, lo));
  while (lo < hi) {
    const int mid = (lo + hi) / 2, S = mid * sp.align;
    if (wave_sum_sequences(a, n0, [&](int k) { return splits_at(k, S); }) * a.p.Hkv <= n_items)
      hi = mid;
    else
      lo = mid + 1;
  }
  return hi * sp.align;
}

// The (sequence, KV head, split) of a workgroup, how many splits that KV head
// has; false past the last item.
struct PagedItem {
  int b, g, split, n_splits;
};
__device__ inline bool paged_locate(const PagedAttnArgs& a, int n0, int S, int item, PagedItem& it) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < a.p.B; b0 += 64) {
    const int b = b0 + lane;
    const int k = b < a.p.B ? splits_at(b0 == 0 ? n0 : paged_span(a, paged_len(a.p, b)).n, S) : 0;
    const int incl = wave_scan(k * a.p.Hkv);
    const unsigned long long hit = __ballot(incl > item);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;
      it.n_splits = __builtin_amdgcn_readlane(k, l);
      const int r = item - (__builtin_amdgcn_readlane(incl, l) - it.n_splits * a.p.Hkv);
      it.b = b0 + l;
      it.g = (int)((uint32_t)r / (uint32_t)it.n_splits);
      it.split = r - it.g * it.n_splits;
      return true;
    }
    item -= __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// A wave's running state: the reference maximum and O as in WaveState, and the
// normalisers as a column of O would be, the product of the probabilities with
// ones: they sum the rounded probabilities (so that the weights sum to one)
// without vector instructions, in the row layout of O.
template <int RPW, int HDIM>
struct PagedState : WaveState<RPW, HDIM> {
  f32x4 z[RPW];
  __device__ inline void init() {
    WaveState<RPW, HDIM>::init();
#pragma unroll
    for (int r = 0; r < RPW; ++r) z[r] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
};

// Running softmax with BPW blocks of products q k (-inf: not seen), c2 > 0
// times which are the logits in log2 units; returns the probabilities as A
// operands of P V, rounded to bf16, the cache's type (half a step, 2^-8).  m is
// raised only past LAZY_MARGIN.
template <int RPW, int BPW, int HDIM>
__device__ inline void paged_softmax(PagedState<RPW, HDIM>& st, const f32x4 (&S)[BPW][RPW], float c2,
                                     PFrags<BPW, RPW>& pf, int lane) {
#pragma unroll
  for (int rr = 0; rr < RPW; ++rr) {
    float mx = -INFINITY;
#pragma unroll
    for (int bi = 0; bi < BPW; ++bi)
      mx = fmaxf(mx, fmaxf(fmaxf(S[bi][rr][0], S[bi][rr][1]), fmaxf(S[bi][rr][2], S[bi][rr][3])));
    mx = max_xor32(max_xor16(mx)) * c2;
    if (__ballot(mx > st.m[rr] + LAZY_MARGIN)) {
      const float mnew = fmaxf(st.m[rr], mx);
      const float alpha = mnew == -INFINITY ? 1.f : fast_exp2(st.m[rr] - mnew);  // m = -inf -> 0
      st.m[rr] = mnew;
      float a4[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a4[i] = __shfl(alpha, 4 * (lane >> 4) + i);
#pragma unroll
      for (int i = 0; i < 4; ++i) st.z[rr][i] *= a4[i];
#pragma unroll
      for (int nb = 0; nb < WaveState<RPW, HDIM>::NBC; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[rr][nb][i] *= a4[i];
    }
    const float msub = st.m[rr] == -INFINITY ? 0.f : st.m[rr];
#pragma unroll
    for (int bi = 0; bi < BPW; ++bi) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = fast_exp2(__builtin_fmaf(S[bi][rr][i], c2, -msub));
      pf.set(bi, rr, pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]));
    }
  }
  constexpr uint32_t ONES = 0x3F803F80u;
  constexpr bool K32 = BPW % 2 == 0;
#pragma unroll
  for (int i = 0; i < (K32 ? BPW / 2 : BPW); ++i)
#pragma unroll
    for (int rr = 0; rr < RPW; ++rr) {
      if constexpr (K32)
        st.z[rr] = mfma_k32(pf.w[i][rr], make_uint4(ONES, ONES, ONES, ONES), st.z[rr]);
      else
        st.z[rr] = mfma_k16(pf.h[i][rr], make_uint2(ONES, ONES), st.z[rr]);
    }
}

// Whether a staged tile of bytes holds an infinity or NaN (bf16: exponent of
// ones, E4M3: 0x7F), looked at by the whole wave.
template <bool KV8, int BYTES>
__device__ inline bool any_not_finite(const unsigned char* tile, int lane) {
  uint32_t bad = 0;
#pragma unroll
  for (int k = 0; k < BYTES / 1024; ++k) {
    const uint4 v = *(const uint4*)(tile + 1024 * k + 16 * lane);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      bad |= KV8 ? ((w[j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u
                 : ((w[j] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
  }
  return __any(bad != 0);
}

// V operand(s) of blocks of a tile: blocks 2 i and 2 i + 1 (K32) or block i.
template <bool KV8, bool K32, int HDIM, int RB>
__device__ inline uint4 v_operand(const unsigned char* v, int i, int nb, int lane) {
  if constexpr (K32 && KV8) {
    return v_operand_e4m3_pair<RB>(v, i, nb, lane);
  } else if constexpr (K32) {
    const uint2 x = v_operand_tr_at<HDIM>(v, 2 * i, nb, lane), y = v_operand_tr_at<HDIM>(v, 2 * i + 1, nb, lane);
    return make_uint4(x.x, x.y, y.x, y.y);
  } else if constexpr (KV8) {
    const uint2 x = v_operand_e4m3<RB>(v, i, nb, lane);
    return make_uint4(x.x, x.y, 0, 0);
  } else {
    const uint2 x = v_operand_tr_at<HDIM>(v, i, nb, lane);
    return make_uint4(x.x, x.y, 0, 0);
  }
}

// O += P V of a tile of which the queries see different rows and some V is not
// finite: a product with a probability of 0 would carry a NaN into the rows of
// the queries that do not see it.  One pass per query, with the rows that it
// does not see taken as 0, kept in that query's rows only.
// seen(bi, j, c): whether query c sees the lane's token j of block bi.
template <int RPW, int NB, int HDIM, bool KV8, int RB, class Seen>
__device__ inline void pv_apart(PagedState<RPW, HDIM>& st, const PFrags<NB, RPW>& pf, const unsigned char* v, int C,
                                int gp_shift, int rt0, int lane, Seen&& seen) {
  constexpr bool K32 = NB % 2 == 0;
  int c = 0;
  do {
    uint32_t mine[RPW][4];  // the rows of query c
#pragma unroll
    for (int rr = 0; rr < RPW; ++rr)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        mine[rr][k] = (16 * (rt0 + rr) + 4 * (lane >> 4) + k) >> gp_shift == c ? 0xFFFFFFFFu : 0u;
#pragma unroll
    for (int i = 0; i < (K32 ? NB / 2 : NB); ++i) {
      uint32_t keep[4];  // of the lane's tokens, two a word, in the operand's order
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int bi = K32 ? 2 * i + (j >> 1) : i, t = 2 * (j & 1);
        keep[j] = (seen(bi, t, c) ? 0xFFFFu : 0u) | (seen(bi, t + 1, c) ? 0xFFFF0000u : 0u);
      }
#pragma unroll
      for (int nb = 0; nb < HDIM / 16; ++nb) {
        uint4 x = v_operand<KV8, K32, HDIM, RB>(v, i, nb, lane);
        x.x &= keep[0];
        x.y &= keep[1];
        x.z &= keep[2];
        x.w &= keep[3];
#pragma unroll
        for (int rr = 0; rr < RPW; ++rr) {
          f32x4 d = {0.f, 0.f, 0.f, 0.f};
          if constexpr (K32)
            d = mfma_k32(pf.w[i][rr], x, d);
          else
            d = mfma_k16(pf.h[i][rr], make_uint2(x.x, x.y), d);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            st.o[rr][nb][k] += __uint_as_float(__float_as_uint(d[k]) & mine[rr][k]);
        }
        __builtin_amdgcn_sched_barrier(0);  // one operand at a time: a rare loop is not to cost the other registers
      }
    }
  } while (++c < C);
}

// Shapes: LDS of a workgroup and what follows from the template's numbers.
template <int RPW_, int NWV_, int TGW_, int TW_, int NS_, bool KV8, int HDIM>
struct PagedShape {
  static constexpr int RPW = RPW_, NWV = NWV_, TGW = TGW_, TW = TW_, NS = NS_;
  static constexpr int RT = RPW * NWV, NW = NWV * TGW, ROWS = 16 * RT;
  static constexpr int RB = KV8 ? HDIM : 2 * HDIM;       // bytes of a staged cache row
  static constexpr int SB = 2 * TW * RB;                 // stage: K rows, then V rows
  static constexpr int LPM = TW * RB / 1024 / NWV;       // 1 KB loads per matrix per stage per wave
  // E4M3 tiles of more than two waves are converted once into shared bf16 tiles;
  // two waves convert in registers, each for itself (4 x 128K tokens, 64 rows: 129
  // us, with shared tiles 142)
  static constexpr bool KCONV = KV8 && NWV > 2;
  static constexpr int GB = NS * SB + (KCONV ? 2 * TW * 2 * HDIM : 0);
  // blocks described per wave, in two halves (a refill waits for every load in
  // flight); where the ring leaves room for one workgroup only, more
  static constexpr int IDS = TGW * GB > 80 * 1024 && NW == 4 ? 256 : 128;
  // columns per exchange of the groups' outputs
  static constexpr int CW = TGW * ROWS * (HDIM + 4) * 4 <= (TGW * GB > 70000 ? TGW * GB : 70000) ? HDIM : HDIM / 2;
  static constexpr int EXCH = TGW * ROWS * (CW + 4) * 4;
  static constexpr int RING = TGW * GB > EXCH ? TGW * GB : EXCH;
  static constexpr int LDS = RING + NW * IDS * 16;
  static constexpr int LDS_ALL = LDS + TGW * ROWS * 8 + ROWS * 4;  // with the row statistics
  static_assert(LPM >= 1 && TW * RB == 1024 * LPM * NWV && TW <= 32, "whole 1 KB loads for every wave and stage, two blocks");
  static_assert(LDS_ALL <= 160 * 1024, "fits a compute unit");
};

// Weight of a part with maximum m against the common maximum M (0 where it
// has seen nothing; a NaN of its sums stays one).
__device__ inline float merge_weight(float m, float M) { return m == -INFINITY ? 0.f : fast_exp2(m - M); }

// Four columns of a finished row: over Z, times the cache's scale and the
// gate's sigmoid, rounded to bf16.
__device__ inline void paged_store4(float4 o, float Z, float v_scale, bool gated, uint2 gb, uint16_t* out) {
  const float inv = (Z > 0.f || Z != Z ? 1.f / Z : 0.f) * v_scale;
  float x[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
  if (gated) {
    const float gv[4] = {bf16_bits_to_f32(gb.x & 0xFFFFu), bf16_bits_to_f32(gb.x >> 16),
                         bf16_bits_to_f32(gb.y & 0xFFFFu), bf16_bits_to_f32(gb.y >> 16)};
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] *= 1.f / (1.f + fast_exp2(-gv[j] * 1.4426950408889634f));
  }
  *(uint2*)out = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
}

template <int RPW, int NWV, int TGW, int TW, int NS, bool KV8, int HDIM>
__global__ __launch_bounds__(64 * NWV * TGW) void k_paged_attn(PagedAttnArgs a) {
  using P = PagedShape<RPW, NWV, TGW, TW, NS, KV8, HDIM>;
  constexpr int NB = TW / 16, NKK = HDIM / 32, RB = P::RB, SB = P::SB, LPM = P::LPM, CPR = RB / 16, RPL = 1024 / RB;
  constexpr int SRB = 2 * HDIM, NTH = 64 * P::NW, ROWS = P::ROWS, IDS = P::IDS;
  constexpr bool KCONV = P::KCONV;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float s_m[TGW][ROWS], s_l[TGW][ROWS], s_sink[ROWS];

  const int lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tg = wid / NWV, wave = wid % NWV, rt0 = wave * RPW;
  PagedItem it;
  int S;
  if (a.sp.single) {  // one split per KV head
    it = PagedItem{(int)(blockIdx.x / (uint32_t)a.p.Hkv), (int)(blockIdx.x % (uint32_t)a.p.Hkv), 0, 1};
    S = a.sp.fixed;
  } else {
    const int n0 = lane < a.p.B ? paged_span(a, paged_len(a.p, lane)).n : 0;
    S = __builtin_amdgcn_readfirstlane(paged_split_blocks(a, n0, blockIdx.x));
    if (S == 0 || !paged_locate(a, n0, S, blockIdx.x, it)) return;
  }
  const int b = __builtin_amdgcn_readfirstlane(it.b), g = __builtin_amdgcn_readfirstlane(it.g);
  const int split = __builtin_amdgcn_readfirstlane(it.split), n_splits = __builtin_amdgcn_readfirstlane(it.n_splits);
  const int Lv = __builtin_amdgcn_readfirstlane(paged_len(a.p, b));
  const PagedSpan span = paged_span(a, Lv);
  const int i0 = split * S;                                  // this split's blocks
  const int n_blocks = max(0, min(span.n - i0, S));
  const int all_tiles = (n_blocks + NB - 1) / NB;
  // tiles tg, tg + TGW, ...; a group without one takes a tile of zero rows, so
  // that the loop always runs (see below)
  const int ntiles = max(1, (all_tiles - tg + TGW - 1) / TGW);

  uint4 q[RPW][NKK];
#pragma unroll
  for (int rr = 0; rr < RPW; ++rr) {
    const int r = 16 * (rt0 + rr) + (lane & 15), c = r >> a.gp_shift, h = r & ((1 << a.gp_shift) - 1);
    const bool real = c < a.C && h < a.G;
    const uint16_t* p = a.q + (((int64_t)b * a.C + (real ? c : 0)) * a.Hq + g * a.G + (real ? h : 0)) * HDIM;
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) {
      q[rr][kk] = *(const uint4*)(p + q_koff(kk, lane));
      if (!real) q[rr][kk] = make_uint4(0, 0, 0, 0);
    }
  }
  const bool whole = n_splits == 1;  // this workgroup writes the output
  for (int r = threadIdx.x; r < ROWS; r += NTH) {
    const int h = r & ((1 << a.gp_shift) - 1);
    s_sink[r] = whole && a.sink && h < a.G ? a.sink[g * a.G + h] * 1.4426950408889634f : -INFINITY;
  }
  float c2 = KV8 ? a.c2 * a.k_scale[g] : a.c2;
  if (c2 < FLT_MIN) c2 = FLT_MIN;  // -inf times it stays -inf
  const unsigned char* Kg = a.p.K + g * a.p.stride_h;
  const unsigned char* Vg = a.p.V + g * a.p.stride_h;
  unsigned char* ring_p = smem + tg * P::GB;
  const uint32_t ring = lds_addr(ring_p);
  unsigned char* tile_k = ring_p + NS * SB;   // KCONV: the converted tiles
  unsigned char* tile_v = tile_k + TW * SRB;
  uint4* blocks = (uint4*)(smem + P::RING) + wid * IDS;

  // Tiles apart, of which the queries see different rows: those with the starts
  // of the later queries' windows (or where first tokens end and a window begins
  // in one block) and those with the chunk's own tokens; at most two of each.
  int a0 = 0, a1 = -1, e0 = 0, e1 = -1;
  {
    const bool gap = a.window > 0 && (a.first + 15) / 16 > span.w0 && a.first < span.lo;
    const int last = a.window > 0 ? Lv - 1 - a.window : -1;  // the last token that the last query does not see any more
    auto tile_of = [&](int block) { return (block - span.w0 + span.nf - i0) >> (NB - 1); };  // rounded down
    if (n_blocks > 0 && (gap || (a.C > 1 && last >= span.lo))) {
      a0 = max(0, tile_of(span.w0));
      a1 = min(all_tiles - 1, tile_of(max(span.w0, last >= 0 ? last / 16 : 0)));
    }
    if (n_blocks > 0 && a.C > 1) {
      e0 = max(0, tile_of(max(0, Lv - a.C + 1) / 16));
      e1 = min(all_tiles - 1, tile_of((Lv - 1) / 16));
    }
  }
  auto is_apart = [&](int T) { return (T >= a0 && T <= a1) || (T >= e0 && T <= e1); };
  auto round_apart = [&](int i) {  // a tile apart among the groups' tiles i
    const int T0 = i * TGW, T1 = T0 + TGW - 1;
    return (a0 <= min(a1, T1) && a1 >= T0) || (e0 <= min(e1, T1) && e1 >= T0);
  };
  // whether the query at pos sees the token
  auto sees = [&](int pos, int t) { return t <= pos && (a.window == 0 || t > pos - a.window || t < a.first); };
  bool deferred = false;

  // Blocks are described IDS / 2 at a time, a lane each, in LDS: x, y: byte offset of
  // the first row in the pool; z: the rows [lo, hi] that some query sees, lo +
  // 256 hi (rows outside repeat one of them), or NONE (zero rows: no page); w:
  // first token, and CACHED.  The loop over tiles then needs a few scalars a block.
  //
  // Rows of pools past the last-level cache are read non-temporal (64 sequences
  // of 8000 tokens 351 -> 310 us) but for pages that the sequence before or
  // behind has too (a common prompt, beams), which the caches are to keep for it
  // (4 beams each sharing nine tenths 195 us non-temporal, 163 cacheable).
  constexpr uint32_t ALL = 15u << 8, NONE = 16u, CACHED = 1u << 31;
  auto describe = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
    for (int more = 0; more < IDS / 128; ++more) {
      const int e = tile * NB + 64 * more + lane;         // block of the group
      const int T = (e / NB) * TGW + tg, i = T * NB + e % NB;  // tile and block of the split
      uint4 d = make_uint4(0, 0, NONE, 0);
      // (without a window the entry is known, and loaded, before the length is)
      const int v = i0 + i, most = a.p.max_pages - 1;
      int t0;
      const int32_t* entry = a.p.table + (int64_t)b * a.p.max_pages;
      if (a.window == 0) {
        t0 = 16 * v;
        entry += min(t0 >> a.p.page_shift, most);
      } else {
        t0 = 16 * token_block(span, v);
        entry += min(max(t0 >> a.p.page_shift, 0), most);
      }
      const int id = *entry;
      uint32_t cached = CACHED;
      if (a.stream) {
        const int before = b > 0 ? entry[-(int64_t)a.p.max_pages] : -1, behind = b + 1 < a.p.B ? entry[a.p.max_pages] : -1;
        if (id != before && id != behind) cached = 0;
      }
      if (i < n_blocks) {
        if (is_page(id, a.p.n_pages)) {
          const int64_t off = id * a.p.stride_p + (t0 & (a.p.page - 1)) * a.p.stride_t;
          const int lo = t0 < a.first ? 0 : max(0, span.lo - t0);
          const int hi = min(15, (v < span.nf ? min(a.first, Lv) : Lv) - 1 - t0);
          d = make_uint4((uint32_t)off, (uint32_t)(off >> 32), (uint32_t)(lo | hi << 8), (uint32_t)t0 | cached);
        }
      }
      blocks[e % IDS] = d;
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    asm volatile("" ::: "memory");
  };
  auto rows_of = [&](int tile, int bi) __attribute__((always_inline)) {
    return (uint32_t)__builtin_amdgcn_readfirstlane(blocks[(tile * NB + bi) % IDS].z);
  };
  const int lrow = lane / CPR;  // this lane's row of a 1 KB load
  auto lane_offset = [&](int row, int from) __attribute__((always_inline)) {
    return (uint32_t)(from * (int)a.p.stride_t) +
           16u * (uint32_t)((lane % CPR) ^ (KV8 ? raw_swz<RB>(row) : stage_swz(row)));
  };
  uint32_t lane_off[LPM];  // from a block's first row
#pragma unroll
  for (int u = 0; u < LPM; ++u) {
    const int row = RPL * (wave * LPM + u) + lrow;
    lane_off[u] = lane_offset(row, row & 15);
  }
  // (every stage issues all its loads: the waits count them)
  constexpr int WB = NWV > 1 ? 1 : NB;                // blocks that a wave loads rows of
  const int wb0 = NWV > 1 ? wave * NB / NWV : 0;      // its first
  static_assert(NWV == 1 || NWV % NB == 0, "a wave's rows are of one block");
  auto issue_to = [&](int tile, int stage) __attribute__((always_inline)) {
    const uint32_t base = ring + (uint32_t)(stage * SB) + 1024u * (uint32_t)(wave * LPM);
    const unsigned char *kp[WB], *vp[WB];
    uint32_t z[WB], cached = 0;
    bool all = true;
#pragma unroll
    for (int k = 0; k < WB; ++k) {
      const uint4 d = blocks[(tile * NB + wb0 + k) % IDS];
      z[k] = (uint32_t)__builtin_amdgcn_readfirstlane(d.z);
      cached |= (uint32_t)__builtin_amdgcn_readfirstlane(d.w);
      const uint64_t off = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(d.x) |
                           (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(d.y) << 32;
      kp[k] = z[k] == NONE ? (const unsigned char*)zero_row : Kg + off;
      vp[k] = z[k] == NONE ? (const unsigned char*)zero_row : Vg + off;
      all &= z[k] == ALL;
    }
    uint32_t from[LPM];
#pragma unroll
    for (int u = 0; u < LPM; ++u) {
      from[u] = lane_off[u];
      if (!all) {
        const int row = RPL * (wave * LPM + u) + lrow;
        const uint32_t r = z[WB > 1 ? RPL * u / 16 : 0];
        from[u] = lane_offset(row, r == NONE ? 0 : max((int)(r & 255u), min(row & 15, (int)(r >> 8))));
      }
    }
    auto load = [&](auto nt) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < LPM; ++u) {
        const int k = WB > 1 ? RPL * u / 16 : 0;
        dma16_s<decltype(nt)::value>(kp[k], from[u], __builtin_amdgcn_readfirstlane(base + 1024 * u));
        dma16_s<decltype(nt)::value>(vp[k], from[u], __builtin_amdgcn_readfirstlane(base + TW * RB + 1024 * u));
      }
    };
    if (!(cached & CACHED))
      load(std::true_type{});
    else
      load(std::false_type{});
  };
  auto issue = [&](int tile) __attribute__((always_inline)) {
    if (tile % (IDS / 2 / NB) == 0) describe(tile);
    issue_to(tile, tile % NS);
  };
  auto logits = [&](const unsigned char* stg, f32x4 (&Sx)[NB][RPW]) __attribute__((always_inline)) {
#pragma unroll
    for (int bi = 0; bi < NB; ++bi) {
      if constexpr (KCONV)
        qk_block_swz<RPW>(tile_k, bi, q, Sx[bi], lane);
      else if constexpr (KV8)
        qk_block_e4m3<RPW, RB>(stg, bi, q, Sx[bi], lane);
      else
        qk_block_swz<RPW>(stg, bi, q, Sx[bi], lane);
    }
  };
  auto convert = [&](const unsigned char* stg) __attribute__((always_inline)) {
    if constexpr (KCONV) {
      convert_rows_e4m3<TW, 64 * NWV, HDIM>(stg, tile_k, 64 * wave + lane);
      convert_rows_e4m3<TW, 64 * NWV, HDIM>(stg + TW * RB, tile_v, 64 * wave + lane);
      __syncthreads();
    }
  };

  PagedState<RPW, HDIM> st;
  st.init();
  // a group of one wave refills a stage as soon as it has read it; the waves
  // of a shared ring meet once a stage, which leaves NS - 1 stages in flight
  constexpr int AHEAD = NWV == 1 ? NS : NS - 1;
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (i < ntiles) issue(i);
  __builtin_assume(ntiles >= 1);
  for (int i = 0; i < ntiles; ++i) {
    wait_ring<2 * LPM>(min(AHEAD - 1, ntiles - 1 - i));
    asm volatile("" ::: "memory");
    if constexpr (NWV > 1) {
      __syncthreads();
      if (i + AHEAD < ntiles) issue(i + AHEAD);
    }
    const unsigned char* stg = ring_p + (i % NS) * SB;
    convert(stg);
    f32x4 Sx[NB][RPW];
    logits(stg, Sx);
    uint32_t z[NB];  // rows that the queries see
    bool full = true;
#pragma unroll
    for (int bi = 0; bi < NB; ++bi) {
      z[bi] = rows_of(i, bi);
      full &= z[bi] == ALL;
    }
    const bool apart = is_apart(i * TGW + tg);
    if (!full || apart) {
#pragma unroll
      for (int bi = 0; bi < NB; ++bi)
#pragma unroll
        for (int ii = 0; ii < 4; ++ii) {
          const int row = 4 * (lane >> 4) + ii;
          const bool out = row < (int)(z[bi] & 255u) || row > (int)(z[bi] >> 8);
#pragma unroll
          for (int rr = 0; rr < RPW; ++rr) Sx[bi][rr][ii] = out ? -INFINITY : Sx[bi][rr][ii];
        }
    }
    if (NWV == 1 ? apart : round_apart(i)) {
      unsigned char* v = ring_p + (i % NS) * SB + TW * RB;
      const bool bad = apart && any_not_finite<KV8, TW * RB>(v, lane);
      if constexpr (NWV > 1) __syncthreads();  // every wave of the group has looked
      if (apart) {
#pragma unroll
        for (int bi = 0; bi < NB; ++bi) {
          const int t0 = (int)(__builtin_amdgcn_readfirstlane(blocks[(i * NB + bi) % IDS].w) & ~CACHED) + 4 * (lane >> 4);
#pragma unroll
          for (int rr = 0; rr < RPW; ++rr) {
            const int pos = Lv - a.C + min((16 * (rt0 + rr) + (lane & 15)) >> a.gp_shift, a.C - 1);
#pragma unroll
            for (int ii = 0; ii < 4; ++ii) Sx[bi][rr][ii] = !bad && sees(pos, t0 + ii) ? Sx[bi][rr][ii] : -INFINITY;
          }
        }
        if (bad) {  // empty: probabilities and V are 0
          deferred = true;
          unsigned char* x = KCONV ? tile_v : v;
#pragma unroll
          for (int k = 0; k < TW * (KCONV ? SRB : RB) / 1024; ++k) *(uint4*)(x + 1024 * k + 16 * lane) = make_uint4(0, 0, 0, 0);
          asm volatile("" ::: "memory");
        }
      }
    }
    PFrags<NB, RPW> pf;
    paged_softmax(st, Sx, c2, pf, lane);
    const unsigned char* vt = KCONV ? tile_v : stg + TW * RB;
    if constexpr (KV8 && !KCONV)
      pv_tile_e4m3<RPW, NB, HDIM, RB>(st, pf, vt, lane);
    else
      pv_tile<RPW, NB, HDIM>(st, pf, vt, lane);
    if constexpr (NWV == 1) {
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the stage has been read
      asm volatile("" ::: "memory");
      if (i + NS < ntiles) issue(i + NS);
    }
  }
  if constexpr (NWV > 1 && TGW > 1)  // the other groups' barriers
    for (int i = ntiles; i < (all_tiles + TGW - 1) / TGW; ++i) {
      __syncthreads();
      if (KCONV) __syncthreads();
      if (round_apart(i)) __syncthreads();
    }

  // the tiles left out, through stage 0 of their group's ring
  if constexpr (NWV > 1) {
    if (a1 >= a0 || e1 >= e0) deferred = __syncthreads_or(deferred);
  }
  if (deferred)
    for (int T = a0; T <= max(a1, e1); ++T) {
      if (T > a1 && T < e0) T = e0;
      if (!is_apart(T)) continue;
      if constexpr (NWV > 1) __syncthreads();  // the ring's last stage has been read
      const int i = T / TGW;
      const bool mine = T % TGW == tg;
      const unsigned char* stg = ring_p;
      if (mine) {
        describe(i);
        issue_to(i, 0);
        wait_ring<2 * LPM>(0);
        asm volatile("" ::: "memory");
      }
      if constexpr (NWV > 1) __syncthreads();
      convert(stg);  // (KCONV: a group that has no tile converts what its ring holds)
      if (!mine || !any_not_finite<KV8, TW * RB>(stg + TW * RB, lane)) continue;
      f32x4 Sx[NB][RPW];
      logits(stg, Sx);
      int t0[NB];
      bool there[NB];
#pragma unroll
      for (int bi = 0; bi < NB; ++bi) {
        t0[bi] = (int)(__builtin_amdgcn_readfirstlane(blocks[(i * NB + bi) % IDS].w) & ~CACHED) + 4 * (lane >> 4);
        there[bi] = rows_of(i, bi) != NONE;
      }
#pragma unroll
      for (int rr = 0; rr < RPW; ++rr) {
        const int pos = Lv - a.C + min((16 * (rt0 + rr) + (lane & 15)) >> a.gp_shift, a.C - 1);
#pragma unroll
        for (int bi = 0; bi < NB; ++bi)
#pragma unroll
          for (int ii = 0; ii < 4; ++ii)
            Sx[bi][rr][ii] = there[bi] && sees(pos, t0[bi] + ii) ? Sx[bi][rr][ii] : -INFINITY;
      }
      PFrags<NB, RPW> pf;
      paged_softmax(st, Sx, c2, pf, lane);
      pv_apart<RPW, NB, HDIM, KV8 && !KCONV, RB>(
          st, pf, KCONV ? tile_v : stg + TW * RB, a.C, a.gp_shift, rt0, lane,
          [&](int bi, int j, int c) { return there[bi] && sees(Lv - a.C + c, t0[bi] + j); });
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the stage has been read
      asm volatile("" ::: "memory");
    }

  // the groups' rows against their common maximum, summed; with one split the
  // sink's logit takes part and the output is written
  constexpr int CW = P::CW, XS = CW + 4, NQ = CW / 4;
  const int items = (a.C << a.gp_shift) * NQ;  // column quads of the rows
  auto real_row = [&](int e, int& c, int& h) {
    const int r = e / NQ;
    c = r >> a.gp_shift;
    h = r & ((1 << a.gp_shift) - 1);
    return h < a.G;
  };
  auto out_at = [&](int e, int c, int h, int d0) {
    return (((int64_t)b * a.C + c) * a.Hq + g * a.G + h) * HDIM + d0 + 4 * (e % NQ);
  };
  // gates on their way while the groups exchange their rows
  constexpr int EPT = ROWS * NQ / NTH;
  constexpr bool EARLY = EPT <= 4 && CW == HDIM;
  uint2 gates[EARLY ? EPT : 1] = {};
  if (EARLY && whole && a.gate)
#pragma unroll
    for (int k = 0; k < (EARLY ? EPT : 1); ++k) {
      int c, h;
      const int e = threadIdx.x + NTH * k;
      if (e < items && real_row(e, c, h)) gates[k] = *(const uint2*)(a.gate + out_at(e, c, h, 0));
    }
#pragma unroll
  for (int rr = 0; rr < RPW; ++rr) {
    if (lane < 16) s_m[tg][16 * (rt0 + rr) + lane] = st.m[rr];
    if ((lane & 15) == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_l[tg][16 * (rt0 + rr) + 4 * (lane >> 4) + i] = st.z[rr][i];
  }
  const float v_scale = KV8 ? a.v_scale[g] : 1.f;
  __syncthreads();  // and every ring is free
  auto row_max = [&](int r) {
    float M = s_sink[r];
#pragma unroll
    for (int w = 0; w < TGW; ++w) M = fmaxf(M, s_m[w][r]);
    return M;
  };
  float* xo = (float*)smem;  // [TGW][ROWS][XS]
#pragma unroll
  for (int d0 = 0; d0 < HDIM; d0 += CW) {
    if (d0) __syncthreads();
#pragma unroll
    for (int rr = 0; rr < RPW; ++rr)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 16 * (rt0 + rr) + 4 * (lane >> 4) + i;
        const float f = merge_weight(s_m[tg][r], row_max(r));
#pragma unroll
        for (int nb = 0; nb < CW / 16; ++nb)
          xo[(tg * ROWS + r) * XS + 16 * nb + (lane & 15)] = st.o[rr][d0 / 16 + nb][i] * f;
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < EPT; ++k) {
      const int e = threadIdx.x + NTH * k, r = e / NQ, d = 4 * (e % NQ);
      int c, h;
      if (e >= items || !real_row(e, c, h)) continue;
      const float M = row_max(r);
      float Z = merge_weight(s_sink[r], M);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < TGW; ++w) {
        Z += s_l[w][r] * merge_weight(s_m[w][r], M);
        const float4 x = *(const float4*)(xo + (w * ROWS + r) * XS + d);
        o.x += x.x;
        o.y += x.y;
        o.z += x.z;
        o.w += x.w;
      }
      if (whole) {
        const int64_t at = out_at(e, c, h, d0);
        uint2 gate = gates[EARLY ? k : 0];
        if (!EARLY && a.gate) gate = *(const uint2*)(a.gate + at);
        paged_store4(o, Z, v_scale, a.gate != nullptr, gate, a.out + at);
      } else {
        const int64_t row = (int64_t)blockIdx.x * ROWS + r;
        *(float4*)(a.part_o + row * HDIM + d0 + d) = o;
        if (d0 + d == 0) *(float2*)(a.part_ml + 2 * row) = make_float2(M, Z);
      }
    }
  }
  if (!a.sp.single && split == 0 && threadIdx.x == 0)
    *(int2*)(a.unit_items + 2 * ((int64_t)b * a.p.Hkv + g)) = make_int2(blockIdx.x, n_splits);
}

// Joins the splits' partial rows.  grid (row groups, B Hkv); NQ threads take a
// row's column quads, SG such teams share a row's splits and meet in LDS.  Bound
// by two memory latencies: 3.5 to 7.0 us.
template <int HDIM, int SG>
__global__ __launch_bounds__(NTP) void k_paged_merge(PagedAttnArgs a) {
  constexpr int NQ = HDIM / 4, TEAMS = NTP / NQ, RPG = TEAMS / SG;  // rows per workgroup
  __shared__ float s_m[TEAMS], s_l[TEAMS];
  __shared__ float4 s_o[SG > 1 ? TEAMS : 1][NQ];
  const int unit = blockIdx.y, g = unit % a.p.Hkv, b = unit / a.p.Hkv;
  const int2 items = *(const int2*)(a.unit_items + 2 * (int64_t)unit);
  if (items.y < 2) return;  // its one workgroup has written the output
  const int team = threadIdx.x / NQ, dq = threadIdx.x % NQ;
  const int r = blockIdx.x * RPG + team / SG, part = team % SG;
  const bool real = r < a.C * a.G;
  const int c = real ? r / a.G : 0, h = real ? r % a.G : 0;
  const int64_t row0 = (int64_t)items.x * a.part_rows + (c << a.gp_shift) + h;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int U = 4;
  for (int s0 = part; s0 < items.y; s0 += U * SG) {
    float2 ml[U];
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u * SG;
      const int64_t row = row0 + (int64_t)min(s, items.y - 1) * a.part_rows;
      ml[u] = *(const float2*)(a.part_ml + 2 * row);
      x[u] = *(const float4*)(a.part_o + row * HDIM + 4 * dq);
      if (s >= items.y) ml[u] = make_float2(-INFINITY, 0.f);
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) mn = fmaxf(mn, ml[u].x);
    const float f = merge_weight(m, mn);
    m = mn;
    l *= f;
    o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float w = merge_weight(ml[u].x, mn);
      l += ml[u].y * w;
      o.x += x[u].x * w;
      o.y += x[u].y * w;
      o.z += x[u].z * w;
      o.w += x[u].w * w;
    }
  }
  if constexpr (SG > 1) {
    if (dq == 0) {
      s_m[team] = m;
      s_l[team] = l;
    }
    s_o[team][dq] = o;
    __syncthreads();
    if (part) return;
    float M = m;
#pragma unroll
    for (int w = 1; w < SG; ++w) M = fmaxf(M, s_m[team + w]);
    const float f = merge_weight(m, M);
    l *= f;
    o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
#pragma unroll
    for (int w = 1; w < SG; ++w) {
      const float e = merge_weight(s_m[team + w], M);
      const float4 x = s_o[team + w][dq];
      l += s_l[team + w] * e;
      o.x += x.x * e;
      o.y += x.y * e;
      o.z += x.z * e;
      o.w += x.w * e;
    }
    m = M;
  }
  if (!real) return;
  if (a.sink) {
    const float s = a.sink[g * a.G + h] * 1.4426950408889634f, M = fmaxf(m, s);
    const float f = merge_weight(m, M);
    l = l * f + merge_weight(s, M);
    o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
  }
  const int64_t at = (((int64_t)b * a.C + c) * a.Hq + g * a.G + h) * HDIM + 4 * dq;
  const uint2 gate = a.gate ? *(const uint2*)(a.gate + at) : make_uint2(0, 0);
  paged_store4(o, l, a.v_scale ? a.v_scale[g] : 1.f, a.gate != nullptr, gate, a.out + at);
}

// ============================================================================ append
// The E4M3 value nearest to x / s: the 32-bit quotient (x times the reciprocal,
// corrected once: one of the two neighbours of the exact one) is rounded to odd:
// where it is not exact, its residual tells on which side the exact quotient
// lies, and of the two neighbours the one with an odd last bit stands for it.
// The conversion, which rounds to 4 bits, then sees no tie that is none.
struct E4m3Scale {
  float s, inv, most;
  __device__ explicit E4m3Scale(float s_) : s(s_), inv(1.f / s_), most(fminf(449.f * s_, FLT_MAX)) {}
};
__device__ inline float quotient_odd(float x, const E4m3Scale& k) {
  const float y = __builtin_amdgcn_fmed3f(x, -k.most, k.most);  // saturates (449 becomes 448)
  const float q0 = y * k.inv;
  const float q = __builtin_fmaf(__builtin_fmaf(-q0, k.s, y), k.inv, q0);
  const float r = __builtin_fmaf(-q, k.s, y);
  const uint32_t u = __float_as_uint(q), odd = (u - ((__float_as_uint(r) ^ u) >> 31)) | 1u;
  const float z = copysignf(__uint_as_float(r != 0.f ? odd : u), x);  // (a zero keeps its sign)
  return x != x ? x : z;
}
// 8 bf16 values (low first) over the scale, as 8 bytes
__device__ inline uint2 quantise8(const uint4& v, const E4m3Scale& k) {
  auto two = [&](uint32_t w) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(quotient_odd(bf16_bits_to_f32(w), k),
                                                     quotient_odd(__uint_as_float(w & 0xFFFF0000u), k), 0, false) & 0xFFFFu;
  };
  return make_uint2(two(v.x) | two(v.y) << 16, two(v.z) | two(v.w) << 16);
}

// grid (rows (token, KV head) / rows per workgroup, B); a thread takes 16
// bytes of a K row and of its V row in the pool.  Bound by memory, E4M3 nearly as
// much by the conversions: 8 x 4096 tokens of 8 heads (268 MB; E4M3 201) 30 us,
// E4M3 26.  Stored non-temporally (else 37 and 30 us; an attention that follows
// takes what it did).  Several rows a thread were slower (2: 38 us, 4: 49).
template <bool KV8, int HDIM>
__global__ __launch_bounds__(NTP) void k_paged_append(PagedAppendArgs a) {
  constexpr int CPR = KV8 ? HDIM / 16 : HDIM / 8;  // 16-byte pieces of a pool row
  const int b = blockIdx.y, piece = threadIdx.x % CPR;
  const uint32_t row = blockIdx.x * (uint32_t)(NTP / CPR) + threadIdx.x / CPR;
  const uint32_t i = row / (uint32_t)a.p.Hkv, g = row % (uint32_t)a.p.Hkv;
  const int n = a.n_new ? min(max(a.n_new[b], 0), a.n_tokens) : a.n_tokens;
  if (i >= (uint32_t)n) return;
  const int t = paged_len(a.p, b) - n + (int)i;
  if (t < 0) return;
  const int id = a.p.table[(int64_t)b * a.p.max_pages + (t >> a.p.page_shift)];
  const int64_t src = b * a.stride_b + i * a.stride_t + g * a.stride_h + piece * (KV8 ? 16 : 8);
  const int64_t dst = id * a.p.stride_p + g * a.p.stride_h + (t & (a.p.page - 1)) * a.p.stride_t + 16 * piece;
  auto store = [](uint4 x, unsigned char* p) { __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), (u32x4*)p); };
  if constexpr (KV8) {
    const uint4 k0 = *(const uint4*)(a.k_new + src), k1 = *(const uint4*)(a.k_new + src + 8);
    const uint4 v0 = *(const uint4*)(a.v_new + src), v1 = *(const uint4*)(a.v_new + src + 8);
    if (!is_page(id, a.p.n_pages)) return;
    const E4m3Scale ks(a.k_scale[g]), vs(a.v_scale[g]);
    const uint2 ka = quantise8(k0, ks), kb = quantise8(k1, ks), va = quantise8(v0, vs), vb = quantise8(v1, vs);
    store(make_uint4(ka.x, ka.y, kb.x, kb.y), a.p.K + dst);
    store(make_uint4(va.x, va.y, vb.x, vb.y), a.p.V + dst);
  } else {
    const uint4 k = *(const uint4*)(a.k_new + src), v = *(const uint4*)(a.v_new + src);
    if (!is_page(id, a.p.n_pages)) return;
    store(k, a.p.K + dst);
    store(v, a.p.V + dst);
  }
}

// ============================================================================ page operators
// Sums over a workgroup's threads (sh: a word per wave; free again on return).
__device__ inline int block_sum(int v, int* sh) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  int s = 0;
#pragma unroll
  for (int w = 0; w < NTP / 64; ++w) s += sh[w];
  __syncthreads();
  return s;
}

// The pages of chunk `chunk` with which(refs) true, as bits of ballots: wave w
// holds 1024 consecutive pages, word k of it 64.  f(page, refs, true or not,
// how many of the chunk before it).  Returns how many there are.
template <class Which, class F>
__device__ inline int chunk_pages(const PagesArgs& a, int chunk, int* sh, Which&& which, F&& f) {
  constexpr int PER = PAGES_CHUNK / NTP;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int p0 = chunk * PAGES_CHUNK + wave * (64 * PER) + lane;
  int v[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) v[k] = p0 + 64 * k < a.n_pages ? a.refs[p0 + 64 * k] : 0;
  unsigned long long bits[PER];
  int n = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    bits[k] = __ballot(p0 + 64 * k < a.n_pages && which(v[k]));
    n += __popcll(bits[k]);
  }
  if (lane == 0) sh[wave] = n;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NTP / 64; ++w) {
    if (w < wave) before += sh[w];
    all += sh[w];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const bool hit = (bits[k] >> lane) & 1;
    if (p0 + 64 * k < a.n_pages) f(p0 + 64 * k, v[k], hit, before + __popcll(bits[k] & ((1ull << lane) - 1)));
    before += __popcll(bits[k]);
  }
  return all;
}

enum { ROW_HEIR = 1, ROW_CHILDLESS = 2 };

__device__ inline int pages_len(const PagesArgs& a, int b) {
  const int L = a.len[b], cap = a.page * a.max_pages;
  return L < 0 ? 0 : (L > cap ? cap : L);
}

// grid: one workgroup per chunk of the pool, then (but for a compaction) one
// per table row.  A chunk's free pages are listed in order, its counts copied
// to refs_out; a row finds what it wants.
template <PagesOp OP>
__global__ __launch_bounds__(NTP) void k_pages_scan(PagesArgs a) {
  __shared__ int sh[NTP / 64];
  if ((int)blockIdx.x < a.n_chunks) {
    const int chunk = blockIdx.x;
    int n;
    if constexpr (OP == PagesOp::compact)
      n = chunk_pages(a, chunk, sh, [](int r) { return r > 0; }, [](int, int, bool, int) {});
    else
      n = chunk_pages(a, chunk, sh, [](int r) { return r <= 0; }, [&](int p, int r, bool free, int at) {
        if (a.refs_out != a.refs) a.refs_out[p] = r;
        if (free) a.list[(int64_t)chunk * PAGES_CHUNK + at] = p;
      });
    if (threadIdx.x == 0) a.chunk_n[chunk] = n;
    return;
  }
  const int b = blockIdx.x - a.n_chunks;
  if constexpr (OP == PagesOp::extend) {
    int have = 0;
    const int32_t* row = a.table + (int64_t)b * a.max_pages;
    for (int j = threadIdx.x; j < a.max_pages; j += NTP)
      if (is_page(row[j], a.n_pages)) have = j + 1;
    have = wave_max(have);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = have;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < NTP / 64; ++w) have = max(have, sh[w]);
      const int L = pages_len(a, b);
      a.row_have[b] = have;
      a.row_need[b] = max(0, L / a.page + (L % a.page != 0) - have);
    }
  } else if constexpr (OP == PagesOp::reorder) {
    const int p = a.parent[b];
    int heir = a.B, child = 0;
    for (int j = threadIdx.x; j < a.B; j += NTP) {
      const int pj = a.parent[j];
      if (pj == p) heir = min(heir, j);
      child |= pj == b;
    }
    heir = a.B - wave_max(a.B - heir);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = heir;
    child = __syncthreads_or(child);
    if (threadIdx.x == 0) {
      for (int w = 1; w < NTP / 64; ++w) heir = min(heir, sh[w]);
      bool is_heir = false, wants = false;
      if ((uint32_t)p < (uint32_t)a.B) {
        is_heir = b == (a.parent[p] == p ? p : heir);
        const int L = pages_len(a, p);
        wants = !is_heir && L % a.page != 0 && is_page(a.table[(int64_t)p * a.max_pages + L / a.page], a.n_pages);
      }
      a.row_need[b] = wants;
      a.row_have[b] = (is_heir ? ROW_HEIR : 0) | (child ? 0 : ROW_CHILDLESS);
    }
  }
}

// Pages that the rows before b want, and all rows; and the chunks' free pages
// as prefix sums in pre[0 .. n_chunks].
struct PagesPlace {
  int before, wanted, free;
};
__device__ inline PagesPlace pages_place(const PagesArgs& a, int b, int* pre, int* sh) {
  int before = 0, wanted = 0;
  for (int j = threadIdx.x; j < a.B; j += NTP) {
    const int n = a.row_need[j];
    wanted += n;
    if (j < b) before += n;
  }
  PagesPlace at;
  at.before = block_sum(before, sh);
  at.wanted = block_sum(wanted, sh);
  // a thread's chunks are consecutive: their sum, then the scan of the threads' sums
  const int per = (a.n_chunks + NTP - 1) / NTP, c0 = threadIdx.x * per;
  int own = 0;
  for (int c = c0; c < min(c0 + per, a.n_chunks); ++c) own += a.chunk_n[c];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_scan(own);
  if (lane == 63) sh[wave] = incl;
  __syncthreads();
  int base = incl - own;
  at.free = 0;
#pragma unroll
  for (int w = 0; w < NTP / 64; ++w) {
    if (w < wave) base += sh[w];
    at.free += sh[w];
  }
  for (int c = c0; c < min(c0 + per, a.n_chunks); ++c) {
    pre[c] = base;
    base += a.chunk_n[c];
  }
  if (threadIdx.x == 0) pre[a.n_chunks] = at.free;
  __syncthreads();
  return at;
}
// the r-th free page of the pool, r < pre[n_chunks]
__device__ inline int free_page(const PagesArgs& a, const int* pre, int r) {
  int lo = 0, hi = a.n_chunks - 1;  // the last chunk whose pages begin at or before r
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (pre[mid] <= r)
      lo = mid;
    else
      hi = mid - 1;
  }
  return a.list[(int64_t)lo * PAGES_CHUNK + r - pre[lo]];
}

// grid (B): row b's entries, the pages that it is given behind them.
__global__ __launch_bounds__(NTP) void k_pages_extend(PagesArgs a) {
  extern __shared__ int pre[];
  __shared__ int sh[NTP / 64];
  const int b = blockIdx.x;
  const int need = a.row_need[b], have = a.row_have[b];
  PagesPlace at{0, 0, 0};
  if (need > 0 || b == 0) at = pages_place(a, b, pre, sh);
  if (b == 0 && threadIdx.x == 0) {
    a.counts[0] = min(at.wanted, at.free);
    a.counts[1] = at.wanted - min(at.wanted, at.free);
  }
  const int32_t* row = a.table + (int64_t)b * a.max_pages;
  int32_t* out = a.table_out + (int64_t)b * a.max_pages;
  for (int j = threadIdx.x; j < a.max_pages; j += NTP) {
    int v = row[j];
    const int r = at.before + j - have;
    if (j >= have && j < have + need && r < at.free) {
      v = free_page(a, pre, r);
      a.refs_out[v] = 1;
    }
    out[j] = v;
  }
}

// grid (B): row b's new entries and length from its parent's; counts of the
// pages that it shares, and of those that the old row b gives up.  Integer
// atomics: their order changes nothing.
__global__ __launch_bounds__(NTP) void k_pages_reorder(PagesArgs a) {
  extern __shared__ int pre[];
  __shared__ int sh[NTP / 64];
  const int b = blockIdx.x;
  const int wants = a.row_need[b], part = a.row_have[b], p = a.parent[b];
  PagesPlace at{0, 0, 0};
  if (wants || b == 0) at = pages_place(a, b, pre, sh);
  if (b == 0 && threadIdx.x == 0) {
    a.counts[0] = min(at.wanted, at.free);
    a.counts[1] = at.wanted - min(at.wanted, at.free);
  }
  const bool alive = (uint32_t)p < (uint32_t)a.B;
  const int L = alive ? pages_len(a, p) : 0;
  const int full = L / a.page;
  const bool gets = wants && at.before < at.free;
  const bool heir = part & ROW_HEIR;
  const int32_t* from = a.table + (int64_t)(alive ? p : 0) * a.max_pages;
  const int32_t* old = a.table + (int64_t)b * a.max_pages;
  int32_t* out = a.table_out + (int64_t)b * a.max_pages;
  for (int j = threadIdx.x; j < a.max_pages; j += NTP) {
    int v = -1;
    if (heir) {
      v = from[j];
    } else if (alive && j < full) {
      v = from[j];
      if (is_page(v, a.n_pages)) atomicAdd(a.refs_out + v, 1);
    } else if (gets && j == full) {
      v = free_page(a, pre, at.before);
      a.refs_out[v] = 1;
      int32_t* move = a.moves + 3 * (int64_t)at.before;
      move[0] = from[j];
      move[1] = v;
      move[2] = L % a.page;
    }
    out[j] = v;
    if (part & ROW_CHILDLESS) {
      const int x = old[j];
      if (is_page(x, a.n_pages)) atomicSub(a.refs_out + x, 1);
    }
  }
  if (threadIdx.x == 0) a.len_out[b] = wants && !gets ? full * a.page : L;
}

// grid (chunks): with n_used pages in use, the free pages before n_used are
// the holes, the used ones from n_used on move there, rank by rank.  list[p]:
// the rank of a page that moves, -2 for a hole, -1 for any other page.
// ALONE: pools of at most PAGES_ALONE chunks, whose pages every workgroup counts
// itself, without a launch before this one: a bit each of every 256th.
constexpr int PAGES_ALONE = 4;
template <bool ALONE>
__global__ __launch_bounds__(NTP) void k_pages_list(PagesArgs a) {
  __shared__ int sh[NTP / 64];
  const int chunk = blockIdx.x;
  int before = 0, n_used = 0, stay = 0;  // used pages: before this chunk, all, before n_used
  if constexpr (ALONE) {
    constexpr int PER = PAGES_CHUNK / NTP;
    static_assert(PAGES_ALONE * PER <= 64 && PAGES_ALONE * PAGES_CHUNK < 1 << 15, "bits of a word, half a word a count");
    unsigned long long bits = 0;
    auto count = [&](int n) { return __popcll(n < 64 ? bits & ((1ull << n) - 1) : bits); };  // among the first n
    for (int k0 = 0; k0 * NTP < a.n_pages; k0 += 2 * PER) {
      int v[2 * PER];
#pragma unroll
      for (int k = 0; k < 2 * PER; ++k) v[k] = a.refs[min((k0 + k) * NTP + (int)threadIdx.x, a.n_pages - 1)];
#pragma unroll
      for (int k = 0; k < 2 * PER; ++k)
        bits |= (unsigned long long)((k0 + k) * NTP + (int)threadIdx.x < a.n_pages && v[k] > 0) << (k0 + k);
    }
    const int both = block_sum(__popcll(bits) << 16 | count(chunk * PER), sh);
    before = both & 0xFFFF;
    n_used = both >> 16;
    stay = block_sum(count(max(0, n_used - (int)threadIdx.x + NTP - 1) / NTP), sh);
  } else {
    for (int c = threadIdx.x; c < a.n_chunks; c += NTP) {
      const int n = a.chunk_n[c];
      n_used += n;
      if (c < chunk) before += n;
    }
    before = block_sum(before, sh);
    n_used = block_sum(n_used, sh);
    const int c0 = n_used / PAGES_CHUNK;
    for (int c = threadIdx.x; c < c0; c += NTP) stay += a.chunk_n[c];
#pragma unroll 8
    for (int p = c0 * PAGES_CHUNK + threadIdx.x; p < n_used; p += NTP) stay += a.refs[p] > 0;
    stay = block_sum(stay, sh);
  }
  if (chunk == 0 && threadIdx.x == 0) {
    a.counts[0] = n_used - stay;
    a.counts[1] = n_used;
  }
  chunk_pages(a, chunk, sh, [](int r) { return r > 0; }, [&](int p, int, bool used, int in_chunk) {
    const int u = before + in_chunk;  // used pages before p
    int what = -1;
    if (p < n_used && !used) {
      what = -2;
      a.moves[3 * (int64_t)(p - u) + 1] = p;
    } else if (p >= n_used && used) {
      what = u - stay;
      a.moves[3 * (int64_t)what] = p;
      a.moves[3 * (int64_t)what + 2] = a.page;
    }
    a.list[p] = what;
  });
}

// Counts and table entries follow the moves (each may be written in place:
// a page's count is read by the thread that writes it or clears it).
__global__ __launch_bounds__(NTP) void k_pages_compact(PagesArgs a) {
  const int64_t entries = (int64_t)a.B * a.max_pages, step = (int64_t)gridDim.x * NTP;
  for (int64_t i = (int64_t)blockIdx.x * NTP + threadIdx.x; i < a.n_pages + entries; i += step) {
    if (i < a.n_pages) {
      const int what = a.list[i];
      if (what == -2) continue;  // the page that moves here writes it
      const int r = a.refs[i];
      if (what >= 0) a.refs_out[a.moves[3 * (int64_t)what + 1]] = r;
      a.refs_out[i] = what >= 0 ? 0 : r;
    } else {
      const int64_t e = i - a.n_pages;
      int v = a.table[e];
      if (is_page(v, a.n_pages)) {
        const int what = a.list[v];
        if (what >= 0) v = a.moves[3 * (int64_t)what + 1];
      }
      a.table_out[e] = v;
    }
  }
}

// A workgroup copies the K and V rows of one KV head of one move at a time.
// Bound by memory: 2000 pages (262 MB read, 262 written) 94 us, 5.6 TB/s; a large
// library copy 5.2.  From stream_moves moves on, half the last-level cache's bytes,
// nothing is kept there (123 MB moved 50.0 -> 43.8 us, 61 level, 31 17.7 -> 18.8).
template <bool STREAM>
__device__ inline void copy_rows(const PagesCopyArgs& a, int64_t src, int64_t dst, int pieces, int cpr_shift) {
  constexpr int U = 2;  // rows of K and of V on their way (1: 105, 4: as 2, pages of 16 tokens slower by 4 %)
  auto load = [](const unsigned char* p) {
    return STREAM ? __builtin_nontemporal_load((const u32x4*)p) : *(const u32x4*)p;
  };
  auto store = [](u32x4 x, unsigned char* p) {
    if (STREAM)
      __builtin_nontemporal_store(x, (u32x4*)p);
    else
      *(u32x4*)p = x;
  };
  for (int i0 = threadIdx.x; i0 < pieces; i0 += NTP * U) {
    u32x4 k[U], v[U];
    int64_t off[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * NTP, pieces - 1);
      off[u] = (i >> cpr_shift) * a.p.stride_t + 16 * (i & ((1 << cpr_shift) - 1));
      k[u] = load(a.p.K + src + off[u]);
      v[u] = load(a.p.V + src + off[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * NTP < pieces) {
        store(k[u], a.p.K + dst + off[u]);
        store(v[u], a.p.V + dst + off[u]);
      }
  }
}
__global__ __launch_bounds__(NTP) void k_pages_copy(PagesCopyArgs a) {
  const int cpr_shift = 31 - __clz(a.p.hd * a.esz / 16);  // 16-byte pieces of a row: a power of two
  const int n = min(max(a.n_moves[0], 0), a.max_moves);
  const int64_t units = (int64_t)n * a.p.Hkv;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int32_t* move = a.moves + 3 * (u / a.p.Hkv);
    const int from = move[0], to = move[1], tokens = min(max(move[2], 0), a.p.page);
    if (!is_page(from, a.p.n_pages) || !is_page(to, a.p.n_pages) || from == to) continue;
    const int64_t head = (u % a.p.Hkv) * a.p.stride_h;
    const int64_t src = from * a.p.stride_p + head, dst = to * a.p.stride_p + head;
    const int pieces = tokens << cpr_shift;
    if (n > a.stream_moves)
      copy_rows<true>(a, src, dst, pieces, cpr_shift);
    else
      copy_rows<false>(a, src, dst, pieces, cpr_shift);
  }
}

}  // namespace

// ============================================================================ host launchers
// Shapes by query row tiles, cache format and head dim.  Columns: RT, E4M3, head
// dim, row tiles per wave, waves per ring, token groups, rows and stages of a
// ring.  Of one workgroup a compute unit (head dim 256), two groups of four waves
// rather than one: another wave to each SIMD while one waits at its ring's barrier
// (64 rows; 256 KV heads of 2000 tokens, E4M3 99 -> 78 us; 128 of 300 to 3000 63 -> 56); at head
// dim 128, where two workgroups fit, 5 to 20 % slower.
#define HS2_PAGED_SHAPES(X)                                                        \
  X(1, false, 128, 1, 1, 4, 16, 2) X(2, false, 128, 2, 1, 4, 16, 2)          \
  X(4, false, 128, 2, 2, 2, 32, 2) X(8, false, 128, 2, 4, 1, 32, 2)          \
  X(1, false, 256, 1, 1, 4, 16, 2) X(2, false, 256, 1, 2, 2, 32, 2)          \
  X(4, false, 256, 1, 4, 2, 16, 3) X(8, false, 256, 1, 8, 1, 32, 4)          \
  X(1, true, 128, 1, 1, 4, 32, 2) X(2, true, 128, 2, 1, 4, 32, 2)            \
  X(4, true, 128, 2, 2, 2, 32, 2) X(8, true, 128, 2, 4, 1, 32, 2)            \
  X(1, true, 256, 1, 1, 4, 16, 2) X(2, true, 256, 1, 2, 4, 32, 2)            \
  X(4, true, 256, 1, 4, 2, 32, 2) X(8, true, 256, 1, 8, 1, 32, 4)

PagedAttnShape paged_attn_shape(int RT, bool kv8, int hd) {
#define HS2_PAGED_SHAPE(rt, f8, hdim, rpw, nwv, tgw, tw, ns)             \
  if (RT == rt && kv8 == f8 && hd == hdim) {                             \
    using P = PagedShape<rpw, nwv, tgw, tw, ns, f8, hdim>;               \
    return PagedAttnShape{P::ROWS, tgw * tw / 16, 160 * 1024 / (P::LDS_ALL + 1024)};  \
  }
  HS2_PAGED_SHAPES(HS2_PAGED_SHAPE)
#undef HS2_PAGED_SHAPE
  return PagedAttnShape{0, 0, 0};
}

// Workgroups resident on a compute unit: the runtime's figure, each with 1 KB
// of LDS to spare (as occupancy_capped of the full attention).
hipError_t paged_attn_wgs(int RT, bool kv8, int hd, int* wgs) {
#define HS2_PAGED_WGS(rt, f8, hdim, rpw, nwv, tgw, tw, ns)                                                \
  if (RT == rt && kv8 == f8 && hd == hdim) {                                                              \
    using P = PagedShape<rpw, nwv, tgw, tw, ns, f8, hdim>;                                                \
    const hipError_t e = hipOccupancyMaxActiveBlocksPerMultiprocessor(                                    \
        wgs, (const void*)k_paged_attn<rpw, nwv, tgw, tw, ns, f8, hdim>, 64 * P::NW, P::LDS);       \
    *wgs = std::min(*wgs, 160 * 1024 / (P::LDS_ALL + 1024));                                              \
    return e;                                                                                             \
  }
  HS2_PAGED_SHAPES(HS2_PAGED_WGS)
#undef HS2_PAGED_WGS
  return hipErrorInvalidValue;
}

hipError_t set_paged_smem_limits() {
  hipError_t e = hipSuccess;
#define HS2_PAGED_ATTR(rt, f8, hdim, rpw, nwv, tgw, tw, ns)                                               \
  if (e == hipSuccess)                                                                                    \
    e = hipFuncSetAttribute((const void*)k_paged_attn<rpw, nwv, tgw, tw, ns, f8, hdim>,                   \
                            hipFuncAttributeMaxDynamicSharedMemorySize,                                   \
                            PagedShape<rpw, nwv, tgw, tw, ns, f8, hdim>::LDS);
  HS2_PAGED_SHAPES(HS2_PAGED_ATTR)
#undef HS2_PAGED_ATTR
  return e;
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, int RT, hipStream_t s) {
  const unsigned grid = a.sp.single ? a.p.B * a.p.Hkv : a.sp.n_items;
  const bool kv8 = a.k_scale != nullptr;
#define HS2_PAGED_LAUNCH(rt, f8, hdim, rpw, nwv, tgw, tw, ns)                                             \
  if (RT == rt && kv8 == f8 && a.p.hd == hdim) {                                                          \
    using P = PagedShape<rpw, nwv, tgw, tw, ns, f8, hdim>;                                                \
    k_paged_attn<rpw, nwv, tgw, tw, ns, f8, hdim><<<grid, 64 * P::NW, P::LDS, s>>>(a);                    \
    return hipGetLastError();                                                                             \
  }
  HS2_PAGED_SHAPES(HS2_PAGED_LAUNCH)
#undef HS2_PAGED_LAUNCH
  return hipErrorInvalidValue;
}

hipError_t launch_paged_merge(const PagedAttnArgs& a, hipStream_t s) {
  const int units = a.p.B * a.p.Hkv, rows = a.C * a.G;
  const int teams = NTP / (a.p.hd / 4);
  // a team per row where a KV head has few splits on average
  const bool shared = a.sp.n_items > 8 * units;
  const dim3 grid(shared ? rows : (rows + teams - 1) / teams, units);
  if (a.p.hd == 128) {
    if (shared) k_paged_merge<128, 8><<<grid, NTP, 0, s>>>(a); else k_paged_merge<128, 1><<<grid, NTP, 0, s>>>(a);
  } else {
    if (shared) k_paged_merge<256, 4><<<grid, NTP, 0, s>>>(a); else k_paged_merge<256, 1><<<grid, NTP, 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t s) {
  const int per = NTP / (a.k_scale ? a.p.hd / 16 : a.p.hd / 8);  // rows per workgroup
  const dim3 grid((unsigned)(((int64_t)a.n_tokens * a.p.Hkv + per - 1) / per), a.p.B);
#define HS2_PAGED_APPEND(kv8, hdim) k_paged_append<kv8, hdim><<<grid, NTP, 0, s>>>(a)
  if (a.k_scale) {
    if (a.p.hd == 128) HS2_PAGED_APPEND(true, 128); else HS2_PAGED_APPEND(true, 256);
  } else {
    if (a.p.hd == 128) HS2_PAGED_APPEND(false, 128); else HS2_PAGED_APPEND(false, 256);
  }
#undef HS2_PAGED_APPEND
  return hipGetLastError();
}

hipError_t launch_pages_scan(const PagesArgs& a, PagesOp op, hipStream_t s) {
  if (op == PagesOp::extend) k_pages_scan<PagesOp::extend><<<a.n_chunks + a.B, NTP, 0, s>>>(a);
  if (op == PagesOp::reorder) k_pages_scan<PagesOp::reorder><<<a.n_chunks + a.B, NTP, 0, s>>>(a);
  if (op == PagesOp::compact && a.n_chunks > PAGES_ALONE) k_pages_scan<PagesOp::compact><<<a.n_chunks, NTP, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t s) {
  k_pages_extend<<<a.B, NTP, sizeof(int) * (a.n_chunks + 1), s>>>(a);
  return hipGetLastError();
}
hipError_t launch_pages_reorder(const PagesArgs& a, hipStream_t s) {
  k_pages_reorder<<<a.B, NTP, sizeof(int) * (a.n_chunks + 1), s>>>(a);
  return hipGetLastError();
}
hipError_t launch_pages_list(const PagesArgs& a, hipStream_t s) {
  if (a.n_chunks <= PAGES_ALONE)
    k_pages_list<true><<<a.n_chunks, NTP, 0, s>>>(a);
  else
    k_pages_list<false><<<a.n_chunks, NTP, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s) {
  const int64_t n = (a.n_pages + (int64_t)a.B * a.max_pages + NTP - 1) / NTP;
  k_pages_compact<<<(unsigned)(n < 4096 ? n : 4096), NTP, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.max_moves * a.p.Hkv;
  // (one unit a workgroup while the grid is small; 2048 107 us, 8192 103, 32768 the same)
  k_pages_copy<<<(unsigned)(n < 8192 ? n : 8192), NTP, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace hs2
