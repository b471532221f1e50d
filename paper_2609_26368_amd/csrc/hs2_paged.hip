// HIP kernels of the paged KV cache (gfx950).
//
//   k_paged_attn     attention of the new tokens over a sequence's pages
//   k_paged_append   new K and V rows to their slots (bf16, or quantised to E4M3)
//   k_pages_scan     lists the free pages of each chunk of the pool (compaction:
//                    counts the used ones) and what each table row wants
//   k_pages_extend   gives rows free pages
//   k_pages_reorder  rows take over their parents' entries
//   k_pages_list, k_pages_compact   moves that pack the pool; table and counts after them
//   k_pages_copy     the moves' contents
#include "hs2_device.h"
#include "hs2_launch.h"

namespace hs2 {
namespace {

constexpr int NTP = 256;  // threads per workgroup of this file's kernels

__device__ inline int paged_len(const PagedPool& p, int b) {
  const int L = p.len[b], cap = p.page * p.max_pages;
  return L < 0 ? 0 : (L > cap ? cap : L);
}
__device__ inline bool is_page(int id, int n_pages) { return (uint32_t)id < (uint32_t)n_pages; }

// ============================================================================ attention
// grid (Hq, C, B), 4 waves: wave w takes every fourth token that the query
// sees, a lane HDIM / 64 of its head dims; the waves meet in LDS.
template <bool KV8, int HDIM>
__global__ __launch_bounds__(NTP) void k_paged_attn(PagedAttnArgs a) {
  constexpr int EPL = HDIM / 64, NW = NTP / 64;
  __shared__ float s_m[NW], s_l[NW], s_o[NW][HDIM];
  const int h = blockIdx.x, c = blockIdx.y, b = blockIdx.z, g = h / a.G;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int pos = paged_len(a.p, b) - a.C + c;
  const int64_t orow = ((int64_t)b * a.C + c) * a.Hq + h;
  // the tokens seen: [0, nf), then [w0, pos]
  const int w0 = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  const int nf = min(a.first, w0);
  const int n = pos < 0 ? 0 : nf + pos + 1 - w0;
  float q[EPL], o[EPL];
#pragma unroll
  for (int j = 0; j < EPL; ++j) {
    q[j] = bf16_bits_to_f32(a.q[orow * HDIM + lane * EPL + j]) * a.c2 * (KV8 ? a.k_scale[g] : 1.f);
    o[j] = 0.f;
  }
  auto load = [&](const unsigned char* row, float (&x)[EPL]) {
    if constexpr (KV8) {
#pragma unroll
      for (int j = 0; j < EPL; j += 2) {
        const uint32_t v = e4m3x2_to_bf16x2(*(const uint16_t*)(row + lane * EPL + j));
        x[j] = bf16_bits_to_f32(v & 0xFFFFu);
        x[j + 1] = bf16_bits_to_f32(v >> 16);
      }
    } else {
#pragma unroll
      for (int j = 0; j < EPL; ++j) x[j] = bf16_bits_to_f32(((const uint16_t*)row)[lane * EPL + j]);
    }
  };
  float m = -INFINITY, l = 0.f;
  for (int u = wave; u < n; u += NW) {
    const int t = u < nf ? u : u - nf + w0;
    const int id = a.p.table[(int64_t)b * a.p.max_pages + (t >> a.p.page_shift)];
    if (!is_page(id, a.p.n_pages)) continue;
    const int64_t off = id * a.p.stride_p + g * a.p.stride_h + (t & (a.p.page - 1)) * a.p.stride_t;
    float k[EPL], v[EPL], s = 0.f;
    load(a.p.K + off, k);
    load(a.p.V + off, v);
#pragma unroll
    for (int j = 0; j < EPL; ++j) s += q[j] * k[j];
#pragma unroll
    for (int w = 1; w < 64; w *= 2) s += __shfl_xor(s, w);
    const float mn = fmaxf(m, s);
    const float f = mn == -INFINITY ? 0.f : fast_exp2(m - mn), p = mn == -INFINITY ? 0.f : fast_exp2(s - mn);
    m = mn;
    l = l * f + p;
#pragma unroll
    for (int j = 0; j < EPL; ++j) o[j] = o[j] * f + p * v[j];
  }
  if (lane == 0) {
    s_m[wave] = m;
    s_l[wave] = l;
  }
#pragma unroll
  for (int j = 0; j < EPL; ++j) s_o[wave][lane * EPL + j] = o[j];
  __syncthreads();
  const int d = threadIdx.x;
  if (d >= HDIM) return;
  const float sink = a.sink ? a.sink[h] * 1.4426950408889634f : -INFINITY;
  float M = sink;
  for (int w = 0; w < NW; ++w) M = fmaxf(M, s_m[w]);
  float Z = 0.f, x = 0.f;
  if (M != -INFINITY) {
    Z = fast_exp2(sink - M);
    for (int w = 0; w < NW; ++w) {
      const float f = fast_exp2(s_m[w] - M);
      Z += s_l[w] * f;
      x += s_o[w][d] * f;
    }
  }
  x *= (Z > 0.f ? 1.f / Z : 0.f) * (KV8 ? a.v_scale[g] : 1.f);
  if (a.gate) x *= 1.f / (1.f + fast_exp2(-bf16_bits_to_f32(a.gate[orow * HDIM + d]) * 1.4426950408889634f));
  a.out[orow * HDIM + d] = (uint16_t)pack_bf16x2(x, x);
}

// ============================================================================ append
// The E4M3 value nearest to x / s in 64 bits' sense: the 32-bit quotient is
// rounded to odd (where it is not exact, the residual tells on which side the
// quotient lies, and the neighbour with an odd last bit takes its place), so
// that the conversion, which rounds to 4 bits, sees no tie that is none.
__device__ inline float quotient_odd(float x, float s) {
  const float q = x / s;
  uint32_t u = __float_as_uint(q);
  const uint32_t mag = u & 0x7FFFFFFFu;
  if (mag > 0x7F800000u) return q;                                // NaN stays NaN
  if (mag >= 0x43E00000u) return copysignf(448.f, q);             // from 448 on: saturated
  const float r = __builtin_fmaf(-q, s, x);
  if (r != 0.f && !(u & 1u)) u += ((__float_as_uint(r) ^ u) >> 31) ? 0xFFFFFFFFu : 1u;
  return __uint_as_float(u);
}
__device__ inline uint32_t to_e4m3x2(float a, float b) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}
// 8 bf16 values (low first) over s, as 8 bytes
__device__ inline uint2 quantise8(const uint4& v, float s) {
  auto four = [&](uint32_t lo, uint32_t hi) {
    return to_e4m3x2(quotient_odd(bf16_bits_to_f32(lo & 0xFFFFu), s), quotient_odd(bf16_bits_to_f32(lo >> 16), s)) |
           to_e4m3x2(quotient_odd(bf16_bits_to_f32(hi & 0xFFFFu), s), quotient_odd(bf16_bits_to_f32(hi >> 16), s)) << 16;
  };
  return make_uint2(four(v.x, v.y), four(v.z, v.w));
}

// grid (rows (token, KV head) / rows per workgroup, B); a thread takes 16
// bytes of a K row and of its V row in the pool.
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
  if (!is_page(id, a.p.n_pages)) return;
  const int64_t src = b * a.stride_b + i * a.stride_t + g * a.stride_h + piece * (KV8 ? 16 : 8);
  const int64_t dst = id * a.p.stride_p + g * a.p.stride_h + (t & (a.p.page - 1)) * a.p.stride_t + 16 * piece;
  if constexpr (KV8) {
    const uint4 k0 = *(const uint4*)(a.k_new + src), k1 = *(const uint4*)(a.k_new + src + 8);
    const uint4 v0 = *(const uint4*)(a.v_new + src), v1 = *(const uint4*)(a.v_new + src + 8);
    const float ks = a.k_scale[g], vs = a.v_scale[g];
    const uint2 ka = quantise8(k0, ks), kb = quantise8(k1, ks), va = quantise8(v0, vs), vb = quantise8(v1, vs);
    *(uint4*)(a.p.K + dst) = make_uint4(ka.x, ka.y, kb.x, kb.y);
    *(uint4*)(a.p.V + dst) = make_uint4(va.x, va.y, vb.x, vb.y);
  } else {
    const uint4 k = *(const uint4*)(a.k_new + src), v = *(const uint4*)(a.v_new + src);
    *(uint4*)(a.p.K + dst) = k;
    *(uint4*)(a.p.V + dst) = v;
  }
}

// ============================================================================ page operators
// Sums over a workgroup's threads (sh: a word per wave; free again on return).
__device__ inline int block_sum(int v, int* sh) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) v += __shfl_xor(v, w);
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
#pragma unroll
    for (int w = 1; w < 64; w *= 2) have = max(have, __shfl_xor(have, w));
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
#pragma unroll
    for (int w = 1; w < 64; w *= 2) heir = min(heir, __shfl_xor(heir, w));
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
  int incl = own;
#pragma unroll
  for (int w = 1; w < 64; w *= 2) {
    const int x = __shfl_up(incl, w);
    if (lane >= w) incl += x;
  }
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
__global__ __launch_bounds__(NTP) void k_pages_list(PagesArgs a) {
  __shared__ int sh[NTP / 64];
  const int chunk = blockIdx.x;
  int before = 0, n_used = 0;
  for (int c = threadIdx.x; c < a.n_chunks; c += NTP) {
    const int n = a.chunk_n[c];
    n_used += n;
    if (c < chunk) before += n;
  }
  before = block_sum(before, sh);
  n_used = block_sum(n_used, sh);
  int stay = 0;  // used pages before n_used
  const int c0 = n_used / PAGES_CHUNK;
  for (int c = threadIdx.x; c < c0; c += NTP) stay += a.chunk_n[c];
  for (int p = c0 * PAGES_CHUNK + threadIdx.x; p < n_used; p += NTP) stay += a.refs[p] > 0;
  stay = block_sum(stay, sh);
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
    for (int i = threadIdx.x; i < pieces; i += NTP) {
      const int64_t off = (i >> cpr_shift) * a.p.stride_t + 16 * (i & ((1 << cpr_shift) - 1));
      const uint4 k = *(const uint4*)(a.p.K + src + off), v = *(const uint4*)(a.p.V + src + off);
      *(uint4*)(a.p.K + dst + off) = k;
      *(uint4*)(a.p.V + dst + off) = v;
    }
  }
}

}  // namespace

// ============================================================================ host launchers
hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid(a.Hq, a.C, a.p.B);
#define HS2_PAGED_ATTN(kv8, hdim) k_paged_attn<kv8, hdim><<<grid, NTP, 0, s>>>(a)
  if (a.k_scale) {
    if (a.p.hd == 128) HS2_PAGED_ATTN(true, 128); else HS2_PAGED_ATTN(true, 256);
  } else {
    if (a.p.hd == 128) HS2_PAGED_ATTN(false, 128); else HS2_PAGED_ATTN(false, 256);
  }
#undef HS2_PAGED_ATTN
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
  if (op == PagesOp::compact) k_pages_scan<PagesOp::compact><<<a.n_chunks, NTP, 0, s>>>(a);
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
  k_pages_list<<<a.n_chunks, NTP, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s) {
  const int64_t n = (a.n_pages + (int64_t)a.B * a.max_pages + NTP - 1) / NTP;
  k_pages_compact<<<(unsigned)(n < 4096 ? n : 4096), NTP, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.max_moves * a.p.Hkv;
  k_pages_copy<<<(unsigned)(n < 2048 ? n : 2048), NTP, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace hs2
