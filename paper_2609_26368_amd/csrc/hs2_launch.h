// Internal interface between the C ABI (hs2_api.hip) and the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

namespace hs2 {

// Token splits of the full-attention pass: fixed > 0 fixes the split
// length; else every workgroup derives the balanced length from len[]: the
// shortest multiple of align, at least min_split, whose (sequence, KV head,
// split) items number at most even_items; where that is over four times the
// mean length, at most n_items, the grid size; when min_split would give fewer
// than few_items items, the shortest multiple of align whose items number at
// most few_items.  A length that is a multiple of avoid (a power of two, or 0:
// none) is made `longer` tokens longer (from 8192 tokens on longer + align).
struct FaSplitPlan {
  int fixed, align, min_split, even_items, n_items, few_items, avoid, longer;
};

struct FaArgs {
  const uint16_t* q;
  const uint16_t* K;
  const uint16_t* V;
  const int32_t* len;
  float* part_o;   // [n_items][16 RT][HD]
  float* part_ml;  // [n_items][16 RT][4]: (m ref, l, m true, 0)
  int64_t stride_b, stride_h, stride_t;
  float c2;        // softmax scale * log2(e)
  int B, C, Hq, Hkv, G, Gp, max_len;
  FaSplitPlan sp;  // grid: sp.n_items workgroups, one (sequence, KV head, split) item each
  float* logits;   // [B*Hkv][C*G][logit_stride] logits in log2 units (ring kernels), or null
  int64_t logit_stride;
  const float* k_scale;  // [Hkv] for an E4M3 cache (K, V are then byte arrays), else null
  int cache_policy;      // ring kernels: FaCachePolicy of the stage loads
  int k_keep_pct;        // FA_STREAM_K_HEAD: the last k_keep_pct % of each token group's K rows stay
                         // cacheable, the rows before them are non-temporal
};

// Cache policy of the full-attention ring kernel's loads.  Non-temporal
// rows stream past the caches: for rows read once, so that they do not
// evict lines a later pass reads again.
enum FaCachePolicy {
  FA_CACHE_DEFAULT = 0,  // every row cacheable
  FA_STREAM_V = 1,       // V non-temporal, K cacheable
  FA_STREAM_KV = 2,      // K and V non-temporal
  FA_STREAM_K_HEAD = 3,  // V non-temporal, K non-temporal in the leading part of each token group
};
// Policies built for each query row tile count: one row tile takes no
// per-tile branch (it is latency-sensitive), more row tiles take the split one.
constexpr bool fa_cache_policy_built(int rt, int kp) {
  return kp == FA_CACHE_DEFAULT || (rt == 1 ? (kp == FA_STREAM_V || kp == FA_STREAM_KV) : kp == FA_STREAM_K_HEAD);
}

struct CombineArgs {
  const float* part_o;
  const float* part_ml;
  const int32_t* len;
  uint16_t* out;        // [B, C, Hq, HD] bf16
  float* stats_log2;    // [B, C, Hq, 2] (reference max M in log2 units, Z against it) or null
  float* stats_user;    // [B, C, Hq, 2] (M in natural units, Z) or null
  int B, C, Hq, Hkv, G, Gp, max_len;
  int rows;             // partial rows per slot
  int nslot;            // partial slots per unit
  FaSplitPlan sp;       // FA only: the full-attention pass's splits (the partial of item i at slot i)
  int sa_mode;
  uint4* clear;         // 16-byte words zeroed by the kernel as a side job, or null
  int64_t n_clear;
  const float* sink;    // [Hq] sink logits (natural units of the scaled logits) or null
  const uint16_t* gate; // [B, C, Hq, D] bf16 output gate logits or null
  const float* v_scale; // [Hkv] E4M3 cache: output scale of each KV head, or null
  int hd;               // head dim (128 or 256)
};

struct PoolArgs {
  const uint16_t* q;
  const uint16_t* K;
  const int32_t* len;
  const float* stats_log2;
  float* scores;        // [rows][score_stride]
  uint32_t* hist;       // [rows][NBINS]
  const float* logits;  // [B*Hkv][C*G][logit_stride] (k_pool_logits)
  int64_t logit_stride;
  const float* k_scale;  // [Hkv] for an E4M3 cache, else null
  int hd;                // head dim (128 or 256)
  int64_t stride_b, stride_h, stride_t;
  int64_t score_stride;
  float c2;
  int B, C, Hq, Hkv, G, Gp, max_len, W;
  int split_tokens, n_split;
  int k_stream;          // k_pool: K rows are read non-temporal (the last pass over them)
};

struct SelArgs {
  const float* scores;
  const int32_t* len;
  uint32_t* hist;       // [rows][NBINS]
  int32_t* state;       // [rows][8]
  uint64_t* bitmap;     // [rows][bitmap_words]
  uint32_t* cand_key;   // [rows][cand_cap]
  int32_t* cand_idx;    // [rows][cand_cap]
  int32_t* idx;         // [rows][S]
  int64_t rows, score_stride, bitmap_words, cand_cap;
  int B, C, Hkv, max_len, k, W, S;
  int chunk;
};

struct BlockSelArgs {
  const float* scores;  // [rows][score_stride]
  const int32_t* len;
  int32_t* idx;         // [rows][S]
  uint32_t* keys;       // [rows][key_stride] block score keys (workspace)
  int64_t rows, score_stride, key_stride;
  int C, Hkv, max_len, k, W, S;
  int block;            // tokens per block, a power of two in [16, 256]; ceil(max_len / block) <= 16384
};

struct SaArgs {
  const uint16_t* q;
  const uint16_t* K;
  const uint16_t* V;
  const int32_t* len;
  const int32_t* idx;   // [B*Hkv*C][idx_stride]
  float* part_o;
  float* part_ml;
  int64_t stride_b, stride_h, stride_t, idx_stride;
  float c2;
  int B, C, Hq, Hkv, G, max_len;
  int n_slots, split_slots, n_split;
  const float* k_scale;  // [Hkv] for an E4M3 cache, else null
  int hd;                // head dim (128 or 256)
  // launch_sa_unit: partial rows per split (n_split > 1), or with one split
  // the output and what the merge would apply to it
  int part_rows;
  uint16_t* out;         // [B, C, Hq, D] bf16
  const float* sink;     // [Hq] sink logits or null
  const uint16_t* gate;  // [B, C, Hq, D] bf16 output gate logits or null
  const float* v_scale;  // [Hkv] E4M3 cache: output scale of each KV head, or null
  int stream;            // launch_sa_unit: cache rows are gathered non-temporal
};

constexpr int kFaVariants = 9;             // full-attention kernel shapes (see HS2_RING_VARIANTS)
int fa_split_align(int RT, int variant);   // split lengths are multiples of this many tokens
// head dim served by full-attention kernel (RT, variant) for the cache format, 0 if there is none
int fa_variant_head_dim(int RT, int variant, bool kv8);
// workgroups of the full-attention kernel (RT, variant) resident per compute
// unit on the current device (0 if that kernel does not exist)
hipError_t fa_wgs_per_cu(int RT, int variant, bool kv8, int* wgs);
hipError_t launch_fa_split(const FaArgs& a, int RT, int variant, hipStream_t s);  // a.k_scale: E4M3 cache
hipError_t launch_combine(const CombineArgs& a, int rows_per_unit, int64_t units, hipStream_t s);
hipError_t launch_pool(const PoolArgs& a, int RT, hipStream_t s);
hipError_t launch_pool_logits(const PoolArgs& a, hipStream_t s);
// workgroups of k_pool (RT, Gp, cache format, head dim) with C queries resident per compute unit
hipError_t pool_wgs_per_cu(int RT, int Gp, int C, bool kv8, int hd, int* wgs);
hipError_t set_pool_smem_limits();
hipError_t launch_sel_init(const SelArgs& a, hipStream_t s);
hipError_t launch_sel_hist(const SelArgs& a, int nchunks, hipStream_t s);
hipError_t launch_select(const SelArgs& a, hipStream_t s);
// scores from the stored logits and selection in one launch, for rows of at
// most 16384 tokens (score_select_serves); pa.scores: where the scores go, or null
bool score_select_serves(int max_len);
hipError_t launch_score_select(const SelArgs& a, const PoolArgs& pa, hipStream_t s);
hipError_t launch_block_select(const BlockSelArgs& a, hipStream_t s);  // block sums + selection
hipError_t launch_sa_split(const SaArgs& a, int RT, hipStream_t s);
// sparse layer with one workgroup of NW (4 or 8) waves per (sequence, KV head,
// query, 16-head tile, split of at most kSaUnitSlots slots); with one split it
// writes the output, else one partial per split for launch_combine
constexpr int kSaUnitSlots = 4096;      // as many as a split of the split kernel: never more splits than it needs
constexpr int kSaUnitSlotsShort = 2304;  // up to here a lane holds fewer indices (see k_sa_unit)
constexpr int kSaUnitSlotsPair = 3584;  // two workgroups of 4 waves with so many slots fit a compute unit's LDS
hipError_t launch_sa_unit(const SaArgs& a, int NW, hipStream_t s);
// streaming-read probe over n16 16-byte words (mode: 0 register loads, 1
// non-temporal register loads, 2 direct-to-LDS loads, 3 non-temporal
// direct-to-LDS loads); workgroup w stores a fold of its slice to sink[w]
constexpr int STREAM_PROBE_WORKGROUPS = 4096;
hipError_t launch_stream_probe(const void* src, int64_t n16, int mode, uint32_t* sink, hipStream_t s);

// ---------------------------------------------------------------- paged cache
// A pool of pages with the tables of its sequences; strides in bytes.
struct PagedPool {
  unsigned char* K;
  unsigned char* V;
  int64_t stride_p, stride_h, stride_t;
  const int32_t* table;  // [B][max_pages]
  const int32_t* len;    // [B]
  int B, Hkv, hd, page, page_shift, n_pages, max_pages;
};

// Splits of the paged attention, in blocks of 16 tokens: fixed > 0 fixes their
// length (single: one a KV head, the grid's workgroups are the KV heads, no
// merge is launched); else every workgroup derives it from len[]
// (paged_split_blocks).
//
// The estimate of a call's time, in the time that a block takes a workgroup
// while all of them stream (0.5 - 0.7 us): with `resident` workgroups at once, a
// workgroup alone takes its blocks `alone` times faster; what a split costs
// besides its blocks (its start, its partial written and read again) is
// `item` blocks, the merge's launch `merge`.  A third of the longest item's time
// is left over at the end, less where the device is filled in one round with
// splits of one length: by few KV heads, or by sequences of one length.  Measured, us, one split a KV head / as many splits as
// resident workgroups / 2 / 4 times as many: 512 KV heads of 1000-12000 tokens 304 /
// 329 / 286 / 285, of 6000 243 / 247 / 250 / 254, 1600 of 100-2000 146 / 157 / 158 / 166,
// 64 of 30000 316 / 158 / 158 / 158; 64 rows of head dim 256, 256 heads of 1500 71 / 82
// / 103 / 135, 200 of 1000-4000 152 / 179 / 132 / 158.
struct PagedSplit {
  int fixed, align, min_blocks, n_items, few_items, cap_blocks, resident;
  bool single;
  float alone, item, merge;
};
__host__ __device__ inline float paged_over(float x, float y) {  // x / y, nearly
#ifdef __HIP_DEVICE_COMPILE__
  return x * __builtin_amdgcn_rcpf(y);
#else
  return x / y;
#endif
}
__host__ __device__ inline float paged_time(const PagedSplit& sp, float total, float longest, float left) {
  const float t = paged_over(total, (float)sp.resident), last = paged_over(longest, sp.alone);
  return (t > last ? t : last) + left * last;
}
// The (sequence, KV head, split) items that the splits may number at most, 0: one
// for each of the `units` KV heads.  total: blocks of all, longest: of one.
__host__ __device__ inline int paged_items(const PagedSplit& sp, float total, int units, float longest) {
  constexpr float LEFT = 0.35f;
  float best = paged_time(sp, total, longest, LEFT);
  int n = 0;
  auto consider = [&](int items, float least, float left) {
    const float u = 0.5f * (float)units;  // a KV head's last split is half full
    const float s = paged_over(total, (float)items - u > 1.f ? (float)items - u : 1.f), S = s > least ? s : least;
    const float all = paged_over(total, S) + u;
    const float t = paged_time(sp, total + sp.item * (all < (float)items ? all : (float)items), S, left) + sp.merge;
    if (t < best) {
      best = t;
      n = items;
    }
  };
  // few tokens: short splits, at most one item per compute unit
  if (sp.few_items > units && total <= (float)sp.min_blocks * (float)sp.few_items) {
    consider(sp.few_items, (float)sp.align, LEFT);
  } else {
    const float many = fminf(1.f, paged_over(2.f * (float)units, (float)sp.resident));
    const float ragged = fminf(1.f, paged_over(longest * (float)units, fmaxf(total, 1.f)) - 0.75f);
    for (int k = 1; k <= 4; k *= 2) {
      const int more = units + sp.resident / 4, items = k * sp.resident > more ? k * sp.resident : more;
      consider(items < sp.n_items ? items : sp.n_items, (float)sp.min_blocks, k == 1 ? LEFT * many * ragged : LEFT);
    }
  }
  return n;
}

struct PagedAttnArgs {
  PagedPool p;
  PagedSplit sp;
  float* part_o;           // [n_items][part_rows][hd]: splits' unnormalised outputs
  float* part_ml;          // [n_items][part_rows][2]: (m, l)
  int32_t* unit_items;     // [B * Hkv][2]: first item and number of items of each KV head
  int part_rows;
  const uint16_t* q;
  uint16_t* out;           // [B, C, Hq, hd]
  float c2;                // softmax scale * log2(e)
  int C, Hq, G, gp_shift;  // query rows c * 2^gp_shift + h
  int window, first;       // window 0: every token is seen
  int stream;              // pool rows are read non-temporal
  const float* k_scale;    // [Hkv] for an E4M3 pool, else null
  const float* v_scale;
  const float* sink;       // [Hq] or null
  const uint16_t* gate;    // [B, C, Hq, hd] or null
};
struct PagedAttnShape {
  int rows, align, wgs;  // partial rows, blocks that splits are multiples of, workgroups per compute unit (by LDS)
};
hipError_t paged_attn_wgs(int RT, bool kv8, int hd, int* wgs);  // on the current device
PagedAttnShape paged_attn_shape(int RT, bool kv8, int hd);
hipError_t set_paged_smem_limits();
hipError_t launch_paged_attn(const PagedAttnArgs& a, int RT, hipStream_t s);
hipError_t launch_paged_merge(const PagedAttnArgs& a, hipStream_t s);

struct PagedAppendArgs {
  PagedPool p;
  const uint16_t* k_new;
  const uint16_t* v_new;
  int64_t stride_b, stride_t, stride_h;  // elements
  int n_tokens;
  const int32_t* n_new;    // [B] or null
  const float* k_scale;    // [Hkv] for an E4M3 pool, else null
  const float* v_scale;
};
hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t s);

// Page operators: free (or used) pages are listed in chunks of
// PAGES_CHUNK pages, one workgroup each.
constexpr int PAGES_CHUNK = 4096;
struct PagesArgs {
  const int32_t* table;
  const int32_t* len;
  const int32_t* refs;
  const int32_t* parent;   // reorder
  int32_t* table_out;
  int32_t* len_out;        // reorder
  int32_t* refs_out;
  int32_t* moves;          // [][3] reorder, compact
  int32_t* counts;
  int B, page, n_pages, max_pages, n_chunks;
  // workspace
  int32_t* chunk_n;        // [n_chunks] pages listed of each chunk
  int32_t* list;           // [n_chunks * PAGES_CHUNK] extend, reorder: the free pages of each chunk in order; compact: what
                           // becomes of each page
  int32_t* row_need;       // [B] extend, reorder: pages that the row wants
  int32_t* row_have;       // [B] extend: entries that it has; reorder: its part (ROW_HEIR, ROW_CHILDLESS)
};
enum class PagesOp { extend, reorder, compact };
hipError_t launch_pages_scan(const PagesArgs& a, PagesOp op, hipStream_t s);  // first launch of each operator
hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_reorder(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_list(const PagesArgs& a, hipStream_t s);     // compact: second launch
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s);  // third

struct PagesCopyArgs {
  PagedPool p;
  const int32_t* moves;
  const int32_t* n_moves;
  int max_moves, esz;
  int64_t stream_moves;  // more moves than this go past the caches
};
hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t s);

}  // namespace hs2
