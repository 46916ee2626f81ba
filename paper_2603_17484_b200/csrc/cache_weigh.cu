// Weights of the cached keys (l2a_cache_weigh): W_j += sum over the counted new tokens and the heads of a KV group of what the soft-max over all
// keys up to the token gives key j.  The maximum and sum of a row have to be known before any of its weights is:
//
//   sequences of few rows (cache_few.cu): scores to the workspace in one pass over the keys, a second small kernel sums them up.
//   others, here: the counted rows are compacted, 128 of a KV group to a block, and the products Q K^T are taken twice.
//
// weigh_plan_kernel : one CTA lists the counted tokens and the blocks of rows; the others decode the keys of an 8- or 4-bit cache to bf16.
// weigh_rows_kernel : the blocks' rows of Q side by side.
// weigh_pass_kernel : up to four blocks of rows of a KV head stay in shared memory, 128 keys at a time pass and are multiplied with all of them
//                     (tcgen05, tiles of 128 x 128 scores in TMEM, one for each of four warpgroups, a lane to a thread, 32 columns at a time).
//     first pass    : S = Q K^T, a thread has a row, its running maximum and sum.
//     second pass   : S^T = K Q^T, a thread has a key and sums the weights of its column; another warp adds up the blocks' sums.
//                     The key tiles of the call, laid end to end and weighed by the blocks of their sequence, are cut into even ranges, one a CTA:
//                     in the first pass a range leaves a part of the rows' sums, which weigh_join_kernel joins; in the second it owns its keys, so
//                     that a weight is made by one CTA in a fixed order: bit-reproducible.
// Bound by the exponentials: 16384 a tile, 1024 clk on the special-function unit, next to 512 clk of products; a quarter of them is computed on the
// FMA pipe.  With one block kept and keys streamed past it (32 KB from L2 a tile) L2 was the bound: 4 sequences of up to 16384 keys, 400 tokens of
// the longest, 30 % counted (28/4 heads): 40 and 58 us for the passes.
#include <math.h>

#include <algorithm>

#include "cache_common.cuh"

namespace l2a {

namespace {

constexpr int kCtas = kSplitSms;
constexpr int kPlanThreads = 1024;
constexpr int kKept = 4;                     // blocks of rows, and warpgroups
constexpr int kSumWarps = 4 * kKept, kTmaWarp = kSumWarps, kMmaWarp = kSumWarps + 1, kAddWarp = kSumWarps + 2, kPassThreads = (kSumWarps + 3) * 32;
constexpr int kKStages = 2, kSumBufs = 2;
constexpr int kBoxBytes = 128 * 128;         // 128 rows of 128 bytes

// A block of 128 counted rows of a sequence: packed row r is that of token list[list + r / G], head r % G of the group
struct alignas(16) RowBlock {
  int b, list, row0, n_rows;
  int base, tiles, last;         // position = base + token; key tiles that some row sees; position of the last row
  int first_pos;                 // of the first row: keys up to there are seen by all
};
// A unit: a key tile, times the blocks of rows of its sequence (one where there are none)
struct WeighPlan { int n_blocks, most; int64_t units, share; };     // blocks; most of a sequence; units of a KV head; of a CTA

struct WeighArgs {
  CacheFwdArgs f;                // f.c: the bf16 cache or the decoded copy
  CacheView codes;               // the cache itself
  WeighPlan* plan;
  RowBlock* blocks;
  int* list;                     // counted tokens
  int *list_start, *list_end;    // of a sequence
  int* block_start;              // first block of a sequence, [B + 1],
  int64_t* unit_start;           // units of the sequences before it, [B + 1]
  bf16* rows;                    // [Hkv][most_blocks * 128][D]
  int* row_pos;                  // [most_blocks * 128], -1: no row
  float* minus_lse;              // [Hkv][most_blocks * 128], minus infinity: no row, or one whose sum is NaN,
  int4* nan_last;                // whose position is here: [Hkv][most_blocks], the last one of each 32 rows, -1: none
  float2* part;                  // maximum and sum of 128 rows, from a range,
  int64_t parts;                 // bound of them
  int most_blocks;               // bound
  int clear;                     // no kernel ahead has cleared the status word
};

__device__ __forceinline__ bool here(const CacheFwdArgs& a, int n) { return (int64_t)n * a.G > a.few_rows; }
// New tokens of a sequence, 0 where it is not taken here
__device__ __forceinline__ int sequence(const CacheFwdArgs& a, int b, int& first, int& length) {
  const int n = cache_new(a.c, b, first);
  length = cache_length(a.c, b);
  return here(a, n) ? n : 0;
}
// The last i with v[i] <= x, of n > 0 ascending ones with v[0] <= x
template <class T>
__device__ __forceinline__ int last_not_above(const T* v, int n, T x) {
  int lo = 0;
  while (n - lo > 1) {
    const int mid = (lo + n) >> 1;
    if (v[mid] <= x) lo = mid; else n = mid;
  }
  return lo;
}
// Inclusive scan over the CTA's threads, in place; returns the sum
template <class T>
__device__ __forceinline__ T block_scan(T& x, T* sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T u = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += u;
  }
  __syncthreads();
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  T u = sums[lane];                                    // (as many warps as lanes)
  const T mine = u;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, u, o);
    if (lane >= o) u += y;
  }
  x += __shfl_sync(0xffffffffu, u - mine, warp);
  return __shfl_sync(0xffffffffu, u, 31);
}

// ------------------------------------------------------------------------------------------------------------- plan
__device__ void make_plan(const WeighArgs& p, int* sums, int64_t* sums2) {
  const CacheFwdArgs& a = p.f;
  const CacheView& c = a.c;
  const int tid = threadIdx.x;
  // (lists of new tokens that do not ascend: nothing is stored)
  bool bad = false;
  if (c.cu_new != nullptr)
    for (int b = tid; b < c.B; b += kPlanThreads) bad |= c.cu_new[b] > c.cu_new[b + 1];
  bad = __syncthreads_or(bad);
  // ---- counted tokens
  int base = 0;
  for (int64_t t0 = 0; t0 < c.n_tokens; t0 += kPlanThreads) {
    const int64_t t = t0 + tid;
    int b = -1, first = 0, n = 0, length = 0;
    if (t < c.n_tokens && !bad && (c.cu_new == nullptr || t >= c.cu_new[0])) {
      b = c.cu_new == nullptr ? (int)t / c.Lq : last_not_above(c.cu_new, c.B, (int)t);
      n = sequence(a, b, first, length);
      if (n == 0 || t < first || t >= first + n) b = -1;
    }
    const int take = b >= 0 && (a.every || a.d[t] != 0) && length - n + (t - first) >= 0;
    int x = take;
    const int all = block_scan(x, sums), at = base + x - take;
    if (take && dbg_in_range(at < c.n_tokens, a.status)) p.list[at] = (int)t;
    if (b >= 0 && t == first) p.list_start[b] = at;
    if (b >= 0 && t == first + n - 1) p.list_end[b] = at + take;
    base += all;
  }
  __syncthreads();
  // ---- blocks of rows and units of every sequence
  int block_base = 0, most = 1;
  int64_t unit_base = 0;
  for (int b0 = 0; b0 < c.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int first, length = 0, n = 0;
    if (b < c.B && !bad) n = sequence(a, b, first, length);
    const int blocks = n > 0 ? compact_tiles(p.list_end[b] - p.list_start[b], a.G) : 0;
    const int64_t units = n > 0 ? (int64_t)((length + kTileN - 1) / kTileN) * max(blocks, 1) : 0;
    int x = blocks;
    int64_t y = units;
    const int all = block_scan(x, sums);
    const int64_t all_units = block_scan(y, sums2);
    if (b < c.B) {
      p.block_start[b] = block_base + x - blocks;
      p.unit_start[b] = unit_base + y - units;
    }
    block_base += all;
    unit_base += all_units;
    most = max(most, blocks);
  }
  most = __reduce_max_sync(0xffffffffu, most);
  __syncthreads();
  if ((tid & 31) == 0) sums[tid >> 5] = most;
  __syncthreads();
  most = __reduce_max_sync(0xffffffffu, sums[tid & 31]);
  if (tid == 0) {
    p.block_start[c.B] = block_base;
    p.unit_start[c.B] = unit_base;
    // (a CTA has the tiles whose first unit is in its range; with a tile's units or more a range has one wherever it begins)
    *p.plan = WeighPlan{block_base, most, unit_base, max((int64_t)most, (unit_base * c.Hkv + kCtas - 1) / kCtas)};
  }
  __syncthreads();
  // ---- the blocks
  for (int q = tid; q < block_base; q += kPlanThreads) {
    RowBlock r;
    int first, length;
    r.b = last_not_above(p.block_start, c.B, q);       // (the last: it has blocks)
    const int n = sequence(a, r.b, first, length);
    r.list = p.list_start[r.b];
    r.row0 = (q - p.block_start[r.b]) * kTileM;
    r.n_rows = min(kTileM, (p.list_end[r.b] - r.list) * a.G - r.row0);
    r.base = length - n - first;
    r.first_pos = r.base + p.list[r.list + r.row0 / a.G];
    r.last = r.base + p.list[r.list + (r.row0 + r.n_rows - 1) / a.G];
    r.tiles = r.last / kTileN + 1;
    if (dbg_in_range(q < p.most_blocks && r.n_rows > 0 && r.last < length, a.status)) p.blocks[q] = r;
  }
}

// Keys of an 8- or 4-bit cache as bf16, pages of 128 tokens [page][KV head][128][D].  A lane brings 16 codes, a warp 512 / D keys at a time, 32
// keys of a head in all.
constexpr int kDecodeKeys = 32, kDecodeParts = kTileN / kDecodeKeys;
template <int D, int kKind>
__device__ __forceinline__ void decode_keys(const WeighArgs& p, int64_t item, int b) {
  constexpr bool kE2M1 = kKind == L2A_CACHE_E2M1;
  constexpr int kLanes = D / 16, kRows = 32 / kLanes, kSteps = kDecodeKeys / kRows;
  const CacheFwdArgs& a = p.f;
  const CacheView &c = p.codes, &out = a.c;
  const int lane = threadIdx.x & 31, sub = lane % kLanes;
  int first, length;
  const int n = sequence(a, b, first, length);
  if (n == 0) return;
  const int part = (int)(item % kDecodeParts), head = (int)(item / kDecodeParts % c.Hkv);
  const int64_t block = item / kDecodeParts / c.Hkv, key0 = block * kTileN + part * kDecodeKeys;
  const bool inside = key0 < length;
  uint4 x[kSteps];
  uint32_t e[kSteps], t[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int64_t key = key0 + i * kRows + lane / kLanes;
    const int page = inside && key < length ? cache_page(c, b, (int)key) : -1;
    const int in_page = (int)key & ((1 << c.page_shift) - 1);
    const uint8_t* row = c.K + page * c.page_bytes + (((int64_t)head << c.page_shift) + in_page) * row_bytes(kKind, D);
    const uint8_t* scales = c.ks + page * c.scale_stride;
    if (kE2M1) {
      const uint2 y = page >= 0 ? *reinterpret_cast<const uint2*>(row + sub * 8) : make_uint2(0u, 0u);
      x[i] = make_uint4(y.x, y.y, 0u, 0u);
      t[i] = page >= 0 ? scales[blocks_at<D>(c, head, in_page) + sub] : 0u;
    } else {
      x[i] = page >= 0 ? *reinterpret_cast<const uint4*>(row + sub * 16) : make_uint4(0, 0, 0, 0);
    }
    e[i] = page >= 0 ? scales[exponent_at<D, kKind>(c, head, in_page)] : 0u;
  }
  // (looked up while the codes are on their way)
  bool counts = a.every;
  if (!a.every)
    for (int i = threadIdx.x; i < n; i += kPlanThreads) counts |= a.d[first + i] != 0;
  counts = __syncthreads_or(counts);
  if (!inside || !counts) return;
  if (!dbg_in_range(block < out.table_stride && b < out.B, a.status)) return;
  uint8_t* dst = out.K + ((int64_t)b * out.table_stride + block) * out.page_bytes + ((int64_t)head * kTileN + part * kDecodeKeys) * (2 * D);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    uint32_t o[8];
    if (kE2M1) decode_16(make_uint2(x[i].x, x[i].y), e4m3_value(t[i]) * scale_of_exponent(e[i]), o);
    else decode_16(x[i], scale_of_exponent(e[i]), o);
    store_32(dst + (i * kRows + lane / kLanes) * (2 * D) + sub * 32, true, o);
  }
}

template <int D, int kKind>
__global__ void __launch_bounds__(kPlanThreads) weigh_plan_kernel(const WeighArgs p) {
  dependency_wait();
  dependents_release();
  if (blockIdx.x == 0) {
    if (blockIdx.y != 0) return;
    __shared__ int sums[kPlanThreads / 32];
    __shared__ int64_t sums2[kPlanThreads / 32];
    if (p.clear && threadIdx.x == 0) *p.f.status = 0;
    make_plan(p, sums, sums2);
    return;
  }
  if (kKind != L2A_CACHE_BF16) decode_keys<D, kKind>(p, (int64_t)(blockIdx.x - 1) * (kPlanThreads / 32) + (threadIdx.x >> 5), blockIdx.y);
}

// A block of rows of one KV head, 16 bytes a thread and step; zeros behind the last
constexpr int kRowsThreads = 256;
template <int D>
__global__ void __launch_bounds__(kRowsThreads) weigh_rows_kernel(const WeighArgs p) {
  const CacheFwdArgs& a = p.f;
  const int q = blockIdx.x, g = blockIdx.y, tid = threadIdx.x;
  dependency_wait();
  dependents_release();
  if (q >= p.plan->n_blocks) return;
  const RowBlock r = p.blocks[q];
  if (!dbg_in_range(r.b < a.c.B && r.list + (r.row0 + r.n_rows - 1) / a.G < a.c.n_tokens, a.status)) return;
  constexpr int kPieces = D / 8, kSteps = kTileM * kPieces / kRowsThreads;
  bf16* dst = p.rows + ((int64_t)g * p.most_blocks + q) * kTileM * D;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int row = (i * kRowsThreads + tid) / kPieces, piece = tid % kPieces, x = r.row0 + row, token = x / a.G;
    uint4 v = make_uint4(0, 0, 0, 0);
    const int t = row < r.n_rows ? p.list[r.list + token] : 0;
    if (row < r.n_rows && dbg_in_range(t >= 0 && t < a.c.n_tokens, a.status))
      v = reinterpret_cast<const uint4*>(a.q + t * a.q_t + (int64_t)(g * a.G + x - token * a.G) * D)[piece];
    reinterpret_cast<uint4*>(dst + row * D)[piece] = v;
  }
  if (g == 0 && tid < kTileM) p.row_pos[q * kTileM + tid] = tid < r.n_rows ? r.base + p.list[r.list + (r.row0 + tid) / a.G] : -1;
}

// ------------------------------------------------------------------------------------------------------------- passes
// A piece of work: some key tiles of a KV head of a sequence, by their places in the line
struct WeighPiece {
  int b, g, k0, k1;
  int tiles, length;       // of the sequence
  int q0, blocks;          // its blocks of rows
};
// Early tiles are seen by all rows, late ones by few: places take them from both ends in turn
__device__ __forceinline__ int tile_of(const WeighPiece& w, int k) { return k & 1 ? w.tiles - 1 - (k >> 1) : k >> 1; }

struct WeighWalk {
  int64_t at, end, units;
  __device__ __forceinline__ void init(const WeighArgs& p) {
    const WeighPlan plan = *p.plan;
    units = plan.units;
    const int64_t total = units * p.f.c.Hkv;
    at = min(total, blockIdx.x * plan.share);
    end = min(total, at + plan.share);
  }
  __device__ __forceinline__ bool next(const WeighArgs& p, WeighPiece& w) {
    while (at < end) {
      const int64_t in = at % units;
      w.g = (int)(at / units);
      w.b = last_not_above(p.unit_start, p.f.c.B, in);                   // (the last: it has units)
      w.length = cache_length(p.f.c, w.b);
      w.tiles = (w.length + kTileN - 1) / kTileN;
      w.q0 = p.block_start[w.b];
      w.blocks = p.block_start[w.b + 1] - w.q0;
      const int64_t first = p.unit_start[w.b], last = p.unit_start[w.b + 1], of_tile = max(w.blocks, 1);
      w.k0 = (int)((in - first + of_tile - 1) / of_tile);
      w.k1 = (int)((min(in + (end - at), last) - first + of_tile - 1) / of_tile);
      at += min(end - at, last - in);
      if (w.k0 < w.k1) return true;
    }
    return false;
  }
};
// The blocks that are kept at a time: n of them from q on.  One tile of keys takes `width` warpgroups (block i: warpgroup i of those), so that `wide` tiles
// are under way together.
struct Kept {
  int q, n, width, wide;
  int tiles[kKept];        // that each of them sees (ascending; 0: no block)
  __device__ __forceinline__ Kept(const WeighArgs& p, const WeighPiece& w, int i0) {
    q = w.q0 + i0;
    n = min(kKept, w.blocks - i0);
    width = n <= 1 ? 1 : n == 2 ? 2 : 4;
    wide = kKept / width;
#pragma unroll
    for (int i = 0; i < kKept; ++i) tiles[i] = i < n ? p.blocks[q + i].tiles : 0;
  }
  __device__ __forceinline__ int seen() const { return max(max(tiles[0], tiles[1]), max(tiles[2], tiles[3])); }
};

struct PassBars {
  uint64_t q_full, q_empty, k_full[kKStages], k_empty[kKStages], s_full[kKept], s_empty[kKept], sum_full[kSumBufs], sum_empty[kSumBufs];
  uint32_t tmem_base;
  int abort_flag;
};
template <int D>
struct PassSmem {
  static constexpr int kTileBytes = 128 * D * 2;
  static constexpr int kKOff = kKept * kTileBytes, kStageOff = kKOff + kKStages * kTileBytes;
  static constexpr int kSumOff = kStageOff + kSumWarps * 1024;           // (a warp's copy of what its columns need)
  static constexpr int kSumBytes = kKept * 128 * 8;                      // first pass: maxima and sums; second: two buffers of sums
  static constexpr int kBarOff = kSumOff + kSumBytes;
  static constexpr int kTotal = kBarOff + 256 + 1024 /* alignment slack */;
};
static_assert(sizeof(PassBars) <= 256, "barriers");

// kSum: the second pass
template <int D, bool kSum>
__global__ void __launch_bounds__(kPassThreads, 1)
weigh_pass_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const WeighArgs p) {
  using SM = PassSmem<D>;
  const CacheFwdArgs& a = p.f;
  const CacheView& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  PassBars* bar = reinterpret_cast<PassBars*>(smem + SM::kBarOff);
  volatile int* abort_flag = &bar->abort_flag;
  if (tid == kTmaWarp * 32) {
    mbar_init(&bar->q_full, 1);
    mbar_init(&bar->q_empty, 1);
    for (int i = 0; i < kKStages; ++i) { mbar_init(&bar->k_full[i], 1); mbar_init(&bar->k_empty[i], 1); }
    for (int i = 0; i < kKept; ++i) { mbar_init(&bar->s_full[i], 1); mbar_init(&bar->s_empty[i], 4); }
    for (int i = 0; i < kSumBufs; ++i) { mbar_init(&bar->sum_full[i], kSumWarps); mbar_init(&bar->sum_empty[i], 1); }
    bar->abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(&bar->tmem_base, 512);
    tmem_relinquish();
  }
  dependency_wait();
  dependents_release();
  const bool lost = kSum && *a.status != 0;      // a wait ran out in the first pass: nothing more is stored
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bar->tmem_base;
  WeighWalk walk;
  walk.init(p);
  if (lost) walk.at = walk.end;
  WeighPiece w;
  bool ok = true;

  if (warp == kTmaWarp) {
    // =========================================================================== TMA producer
    if (lane == 0) {
      tma_prefetch_desc(&mapQ);
      tma_prefetch_desc(&mapK);
    }
    const int copies = 128 >> c.page_shift, u = lane % copies, piece = lane / copies;
    const uint32_t bytes = (1u << c.page_shift) * 128;
    uint32_t q_cnt = 0, k_cnt = 0;
    while (ok && walk.next(p, w)) {
      const int last_entry = (w.length - 1) >> c.page_shift;
      auto page_of = [&](int k) -> int {         // of this lane's rows of the tile at place k, -1: none
        const int entry = (int)(((int64_t)tile_of(w, k) * kTileN) >> c.page_shift) + u;
        return k < w.k1 && piece < D / 64 && entry <= last_entry ? cache_page(c, w.b, entry << c.page_shift) : -1;
      };
      for (int i0 = 0; ok && i0 < w.blocks; i0 += kKept) {
        const Kept kept(p, w, i0);
        const int seen = kept.seen();
        ok = mbar_wait_warp(&bar->q_empty, (q_cnt & 1) ^ 1, abort_flag);
        if (!ok) break;
        ++q_cnt;
        if (lane == 0) {
          mbar_expect_tx(&bar->q_full, kept.n * SM::kTileBytes);
          for (int i = 0; i < kept.n; ++i) tma_load_4d(smem + i * SM::kTileBytes, &mapQ, &bar->q_full, 0, (kept.q + i) * kTileM, 0, w.g);
        }
        __syncwarp();
        int page = page_of(w.k0), next = page_of(w.k0 + 1);              // (looked up two tiles ahead)
        for (int k = w.k0; k < w.k1; ++k) {
          const int later = page_of(k + 2);
          if (tile_of(w, k) < seen) {
            const int s = k_cnt % kKStages;
            ok = mbar_wait_warp(&bar->k_empty[s], ((k_cnt / kKStages) & 1) ^ 1, abort_flag);
            if (!ok) break;
            ++k_cnt;
            const uint32_t expect = __popc(__ballot_sync(0xffffffffu, page >= 0)) * bytes;
            if (lane == 0) mbar_expect_tx(&bar->k_full[s], expect);
            __syncwarp();
            if (page >= 0)
              tma_load_page(smem + SM::kKOff + s * SM::kTileBytes + piece * kBoxBytes + u * bytes, &mapK, &bar->k_full[s], false, piece, 0, w.g, page);
          }
          page = next;
          next = later;
        }
      }
    }
  } else if (warp == kMmaWarp) {
    // =========================================================================== MMA issuer
    if (elect_one()) {
      constexpr uint32_t idesc = idesc_bf16_f32(128, 128, 0, 0);
      const uint64_t dq = smem_desc_sw128(smem_u32(smem), 16, 1024), dk = smem_desc_sw128(smem_u32(smem + SM::kKOff), 16, 1024);
      uint32_t q_cnt = 0, k_cnt = 0, phases = 0;         // bit wg: phase of its scores' buffer
      while (ok && walk.next(p, w)) {
        for (int i0 = 0; ok && i0 < w.blocks; i0 += kKept) {
          const Kept kept(p, w, i0);
          const int seen = kept.seen();
          if (!mbar_spin(&bar->q_full, q_cnt & 1, abort_flag)) { ok = false; break; }
          ++q_cnt;
          for (int k = w.k0; ok && k < w.k1; ++k) {
            const int t = tile_of(w, k), wg0 = (k - w.k0) % kept.wide * kept.width;
            if (t >= seen) continue;
            const uint32_t s = k_cnt % kKStages;
            if (!mbar_spin(&bar->k_full[s], (k_cnt / kKStages) & 1, abort_flag)) { ok = false; break; }
            ++k_cnt;
#pragma unroll
            for (int i = 0; i < kKept; ++i) {
              if (t >= kept.tiles[i]) continue;
              const int wg = wg0 + i;
              if (!mbar_spin(&bar->s_empty[wg], ((phases >> wg) & 1) ^ 1, abort_flag)) { ok = false; break; }
              phases ^= 1u << wg;
              tc_fence_after();
              const uint64_t x = dq + i * (SM::kTileBytes >> 4), y = dk + s * (SM::kTileBytes >> 4);
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t o = ((kk >> 2) * kBoxBytes + (kk & 3) * 32) >> 4;
                mma_ss(tmem + wg * 128, (kSum ? y : x) + o, (kSum ? x : y) + o, idesc, kk > 0);
              }
              tc_commit(&bar->s_full[wg]);
            }
            tc_commit(&bar->k_empty[s]);
          }
          tc_commit(&bar->q_empty);
        }
      }
    }
    __syncwarp();
  } else if (warp == kAddWarp) {
    // =========================================================================== second pass: the sums of a tile's blocks onto the keys' weights
    uint32_t rounds = 0;
    while (kSum && ok && walk.next(p, w)) {
      int first;
      const int fresh = w.length - cache_new(c, w.b, first);
      for (int i0 = 0; ok && i0 < max(w.blocks, 1); i0 += kKept) {
        const Kept kept(p, w, i0);
        const int hi = kept.n > 0 ? p.blocks[kept.q + kept.n - 1].last : -1;
        int nan_last = -1;
        for (int i = 0; i < kept.n; ++i) {
          const int4 x = p.nan_last[(int64_t)w.g * p.most_blocks + kept.q + i];
          nan_last = max(nan_last, max(max(x.x, x.y), max(x.z, x.w)));
        }
        for (int k = w.k0; k < w.k1; k += kept.wide, ++rounds) {
          const int buf = rounds % kSumBufs;
          if (!mbar_wait_warp(&bar->sum_full[buf], (rounds / kSumBufs) & 1, abort_flag)) { ok = false; break; }
          const float* sums = reinterpret_cast<const float*>(smem + SM::kSumOff) + buf * (kKept * 128);
          for (int x = 0; x < kept.wide && k + x < w.k1; ++x) {
            float four[4] = {};
            for (int i = 0; i < kept.width; ++i) {
              const float4 y = reinterpret_cast<const float4*>(sums + (x * kept.width + i) * 128)[lane];
              four[0] += y.x; four[1] += y.y; four[2] += y.z; four[3] += y.w;
            }
            const int key = tile_of(w, k + x) * kTileN + 4 * lane;
            if (key <= nan_last) {
#pragma unroll
              for (int i = 0; i < 4; ++i) four[i] = key + i <= nan_last ? NAN : four[i];
            }
            add_weights(a, p.codes, w.b, w.g, key, w.length, i0 == 0 ? fresh : w.length, hi, four);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&bar->sum_empty[buf]);
        }
      }
    }
  } else {
    // =========================================================================== soft-max
    const int wg = warp >> 2, r = (warp & 3) * 32 + lane;       // row of the A operand == TMEM lane
    const uint32_t s_addr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + wg * 128;
    float* stage = reinterpret_cast<float*>(smem + SM::kStageOff + warp * 1024);
    const int* stage_pos = reinterpret_cast<const int*>(stage + 128);
    const float2 scale = make_float2(a.scale_log2, a.scale_log2);
    uint32_t s_cnt = 0, rounds = 0;
    while (ok && walk.next(p, w)) {
      for (int i0 = 0; ok && i0 < max(w.blocks, kSum ? 1 : 0); i0 += kKept) {
        const Kept kept(p, w, i0);
        const int i = wg % kept.width, slot = wg / kept.width, q = kept.q + i;
        const bool mine = i < kept.n;
        int seen = 0, row_pos = -1, first_pos = 0;
#pragma unroll
        for (int x = 0; x < kKept; ++x) seen = x == i ? kept.tiles[x] : seen;
        if (mine && !kSum) row_pos = p.row_pos[q * kTileM + r];
        if (mine && kSum) {
          first_pos = p.blocks[q].first_pos;
          __syncwarp();
          reinterpret_cast<float4*>(stage)[lane] = reinterpret_cast<const float4*>(p.minus_lse + ((int64_t)w.g * p.most_blocks + q) * kTileM)[lane];
          reinterpret_cast<int4*>(stage + 128)[lane] = reinterpret_cast<const int4*>(p.row_pos + q * kTileM)[lane];
          __syncwarp();
        }
        float m = -INFINITY, l = 0.f;
        for (int k = w.k0; k < w.k1; k += kept.wide) {
          const int t = k + slot < w.k1 ? tile_of(w, k + slot) : 0x7fffffff;
          if (kSum) l = 0.f;
          if (t < seen) {
            const int pos = kSum ? t * kTileN + r : row_pos;
            // some pair of the tile is not seen
            const bool partial = kSum ? t * kTileN + kTileN - 1 > first_pos : __any_sync(0xffffffffu, t * kTileN + kTileN - 1 > pos);
            if (!mbar_wait_warp(&bar->s_full[wg], s_cnt & 1, abort_flag)) { ok = false; break; }
            ++s_cnt;
            tc_fence_after();
            // 32 columns are computed with while the next ones come
            uint32_t v[2][32];
            tmem_ld32(s_addr, v[0]);
            float2 sum[2] = {};
#pragma unroll
            for (int col = 0; col < 4; ++col) {
              uint32_t (&x)[32] = v[col & 1];
              tmem_ld_wait();
              if (col < 3) {
                tmem_ld32(s_addr + (col + 1) * 32, v[(col + 1) & 1]);
              } else {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar->s_empty[wg]);
              }
              if (kSum) {
                if (partial) {
#pragma unroll
                  for (int e = 0; e < 32; ++e) x[e] = stage_pos[col * 32 + e] >= pos ? x[e] : 0xff800000u;
                }
                const uint32_t at = smem_u32(stage) + col * 128;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const float4 z = lds128(at + e * 16);
                  const float2 y0 = __ffma2_rn(make_float2(__uint_as_float(x[4 * e]), __uint_as_float(x[4 * e + 1])), scale, make_float2(z.x, z.y));
                  const float2 y1 = __ffma2_rn(make_float2(__uint_as_float(x[4 * e + 2]), __uint_as_float(x[4 * e + 3])), scale, make_float2(z.z, z.w));
                  sum[0] = __fadd2_rn(sum[0], make_float2(fast_exp2(y0.x), fast_exp2(y0.y)));
                  sum[1] = __fadd2_rn(sum[1], e % 2 ? exp2_fma2(y1) : make_float2(fast_exp2(y1.x), fast_exp2(y1.y)));
                }
              } else {
                if (partial) {
                  const uint32_t visible = bit_range(0, pos + 1 - t * kTileN - col * 32);
#pragma unroll
                  for (int e = 0; e < 32; ++e) x[e] = (visible >> e) & 1u ? x[e] : 0xff800000u;
                }
                float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                  mx[0] = fmax3(mx[0], __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                  mx[1] = fmax3(mx[1], __uint_as_float(x[e + 2]), __uint_as_float(x[e + 3]));
                }
                const float m_new = fmaxf(m, fmaxf(mx[0], mx[1]) * a.scale_log2);
                const float neg = m_new == -INFINITY ? 0.f : -m_new;
                sum[0] = sum[1] = make_float2(0.f, 0.f);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const float2 y = __ffma2_rn(make_float2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), scale, make_float2(neg, neg));
                  sum[e & 1] = __fadd2_rn(sum[e & 1], e % 4 == 3 ? exp2_fma2(y) : make_float2(fast_exp2(y.x), fast_exp2(y.y)));
                }
                l = l * fast_exp2(m + neg) + ((sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
                m = m_new;
              }
            }
            if (kSum) l = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
          }
          if (kSum) {
            const int buf = rounds % kSumBufs;
            if (!mbar_wait_warp(&bar->sum_empty[buf], ((rounds / kSumBufs) & 1) ^ 1, abort_flag)) { ok = false; break; }
            ++rounds;
            reinterpret_cast<float*>(smem + SM::kSumOff)[(buf * kKept + wg) * 128 + r] = l;
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar->sum_full[buf]);
          }
        }
        if (!kSum) {
          // ---- the warpgroups that had the same rows, in one part.  (All warps leave together where a wait ran out.)
          float2* sums = reinterpret_cast<float2*>(smem + SM::kSumOff);
          sums[wg * 128 + r] = make_float2(m, l);
          ok = named_barrier_all(1, kSumWarps * 32, ok);
          if (ok && slot == 0 && mine) {
            for (int x = 1; x < kept.wide; ++x) {
              const float2 y = sums[(x * kept.width + i) * 128 + r];
              const float M = fmaxf(m, y.x), base = M == -INFINITY ? 0.f : M;
              l = l * fast_exp2(m - base) + y.y * fast_exp2(y.x - base);
              m = M;
            }
            // (a range that begins inside the sequence's head is its CTA's first)
            const int64_t at = w.k0 == 0 ? (int64_t)w.g * p.plan->n_blocks + q : (int64_t)c.Hkv * p.plan->n_blocks + (int64_t)blockIdx.x * p.plan->most + q - w.q0;
            if (dbg_in_range(at < p.parts && q < p.plan->n_blocks && w.g < c.Hkv, a.status)) p.part[at * kTileM + r] = make_float2(m, l);
          }
          ok = named_barrier_all(1, kSumWarps * 32, ok);
        }
      }
    }
  }

  // ---- teardown
  tc_fence_before();
  __syncthreads();
  if (bar->abort_flag) {
    // a bounded wait ran out: give copies still in flight time to land before shared memory is released
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    if (tid == 0) atomicExch(a.status, 1);
    __syncthreads();
  }
  if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

// Minus log2 of the sum of a row's weights, from the ranges that have seen a part of its keys
__global__ void __launch_bounds__(kTileM) weigh_join_kernel(const WeighArgs p) {
  const int q = blockIdx.x, g = blockIdx.y, r = threadIdx.x;
  dependency_wait();
  dependents_release();
  const WeighPlan plan = *p.plan;
  if (q >= plan.n_blocks) return;
  const int b = p.blocks[q].b, q0 = p.block_start[b];
  const int64_t first = g * plan.units + p.unit_start[b], units = p.unit_start[b + 1] - p.unit_start[b], of_tile = p.block_start[b + 1] - q0;
  const int64_t c0 = first / plan.share, c1 = (first + units - of_tile) / plan.share;
  float2 x = p.part[((int64_t)g * plan.n_blocks + q) * kTileM + r];
  float m = x.x, l = x.y;
  const float2* rest = p.part + ((int64_t)p.f.c.Hkv * plan.n_blocks + q - q0) * kTileM + r;
  constexpr int kAhead = 8;                // parts under way together
  for (int64_t cta = c0 + 1; cta <= c1; cta += kAhead) {
    float2 y[kAhead];
    float M = m;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) y[i] = cta + i <= c1 ? rest[(cta + i) * plan.most * kTileM] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) M = fmaxf(M, y[i].x);
    const float base = M == -INFINITY ? 0.f : M;
    l *= fast_exp2(m - base);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) l += y[i].y * fast_exp2(y[i].x - base);
    m = M;
  }
  const bool row = r < p.blocks[q].n_rows;
  const int64_t block = (int64_t)g * p.most_blocks + q;
  // A row with NaN gives it to the keys that it sees, no others: behind its position the second pass is not to meet it
  const int nan_last = __reduce_max_sync(0xffffffffu, row && isnan(l) ? p.row_pos[q * kTileM + r] : -1);
  if (r % 32 == 0) reinterpret_cast<int*>(p.nan_last + block)[r / 32] = nan_last;
  p.minus_lse[block * kTileM + r] = row && l != 0.f && !isnan(l) ? -(m + log2f(l)) : -INFINITY;
}

// ------------------------------------------------------------------------------------------------------------- host
int64_t most_blocks(const l2a_params* p, int n_tokens) { return ((int64_t)n_tokens * (p->Hq / p->Hkv) + kTileM - 1) / kTileM + p->B; }
int64_t most_of_one(const l2a_params* p) { return ((int64_t)p->Lq * (p->Hq / p->Hkv) + kTileM - 1) / kTileM; }
int64_t key_tiles(int Lk) { return ((int64_t)Lk + kTileN - 1) / kTileN; }
size_t layout(const l2a_params* p, int kind, int n_tokens, uint8_t* base, WeighArgs* w, uint8_t** copy) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    uint8_t* x = base + at;
    at += align_up(bytes, 256);
    return x;
  };
  const size_t blocks = (size_t)most_blocks(p, n_tokens), B = p->B, Hkv = p->Hkv;
  WeighArgs x = {};
  x.plan = reinterpret_cast<WeighPlan*>(take(sizeof(WeighPlan)));
  x.blocks = reinterpret_cast<RowBlock*>(take(blocks * sizeof(RowBlock)));
  x.list = reinterpret_cast<int*>(take((size_t)n_tokens * 4));
  x.list_start = reinterpret_cast<int*>(take(B * 4));
  x.list_end = reinterpret_cast<int*>(take(B * 4));
  x.block_start = reinterpret_cast<int*>(take((B + 1) * 4));
  x.unit_start = reinterpret_cast<int64_t*>(take((B + 1) * 8));
  x.row_pos = reinterpret_cast<int*>(take(blocks * kTileM * 4));
  x.minus_lse = reinterpret_cast<float*>(take(Hkv * blocks * kTileM * 4));
  x.nan_last = reinterpret_cast<int4*>(take(Hkv * blocks * sizeof(int4)));
  x.parts = (int64_t)(Hkv * blocks + kCtas * (size_t)most_of_one(p));
  x.part = reinterpret_cast<float2*>(take((size_t)x.parts * kTileM * 8));
  x.rows = reinterpret_cast<bf16*>(take(Hkv * blocks * kTileM * p->D * 2));
  x.most_blocks = (int)blocks;
  uint8_t* decoded = take(kind == L2A_CACHE_BF16 ? 0 : B * Hkv * (size_t)key_tiles(p->Lk) * kTileN * p->D * 2);
  if (w) {
    *w = x;
    *copy = decoded;
  }
  return at;
}

// Rows of a sequence up to which its scores are kept: as many as the kernel of the few rows takes, for bf16, where the blocks need no decoded copy,
// three quarters; less where the workspace for the scores of all sequences would pass kMostScores.  us scores kept / blocks: 64 rows of each of eight
// sequences of 32K (32/8 heads, half counted) bf16 448 / 248, e2m1 378 / 406, of one e2m1 99 / 78; 49 rows of four of 16K (28/4) e4m3 63 / 78; 35 of
// two of 100K e2m1 128 / 188; 28 of eight of 32K bf16 107 / 144.
constexpr int64_t kMostScores = 4ll << 30;
int kept_rows(const l2a_params* p, int kind) {
  const int64_t G = p->Hq / p->Hkv, all = (int64_t)p->Lq * G;
  for (int rows = (kind == L2A_CACHE_BF16 ? 3 : kRowBlocks) * kBlockRows; rows >= kBlockRows; rows -= kBlockRows)
    if (rows >= G && (double)p->B * p->Hkv * (double)std::min<int64_t>(rows, all) * (p->Lk + 64.0) * 4 <= (double)kMostScores) return rows;
  return 0;
}
static_assert(kRowBlocks == 4, "three quarters");
int most_kept(const l2a_params* p, int kind) { return (int)std::min<int64_t>(kept_rows(p, kind), (int64_t)p->Lq * (p->Hq / p->Hkv)); }
size_t few_bytes(const l2a_params* p, int kind) {
  const int rows = most_kept(p, kind);
  return rows > 0 ? align_up(cache_few_weigh_ws_bytes(p, rows), 256) : 0;
}
// The most of them for any smaller Lq and Lk.  More rows are kept of shorter sequences, so that these can need more: for each number of rows as many
// keys as kMostScores allows.
size_t most_few_bytes(const l2a_params* p, int kind) {
  const int64_t G = p->Hq / p->Hkv, top = std::min<int64_t>((kind == L2A_CACHE_BF16 ? 3 : kRowBlocks) * kBlockRows, (int64_t)p->Lq * G);
  size_t most = 0;
  for (int64_t rows = G; rows <= top; ++rows) {
    l2a_params x = *p;
    x.Lk = (int)std::min<int64_t>(p->Lk, kMostScores / (4 * (int64_t)p->B * p->Hkv * rows) - 64);
    if (x.Lk > 0) most = std::max(most, align_up(cache_few_weigh_ws_bytes(&x, (int)rows), 256));
  }
  return most;
}
bool has_blocks(const l2a_params* p, int kind) { return (int64_t)p->Lq * (p->Hq / p->Hkv) > kept_rows(p, kind); }

template <int D, bool kSum>
cudaError_t launch_pass(const CUtensorMap& mapQ, const CUtensorMap& mapK, const WeighArgs& p, cudaStream_t s) {
  constexpr int smem = PassSmem<D>::kTotal;
  static PerDeviceOnce once;
  const cudaError_t e = once.run([] { return cudaFuncSetAttribute(weigh_pass_kernel<D, kSum>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); });
  return e != cudaSuccess ? e : launch_dependent(weigh_pass_kernel<D, kSum>, dim3(kCtas), kPassThreads, smem, s, true, mapQ, mapK, p);
}

template <int D, int kKind>
cudaError_t launch_plan(const WeighArgs& p, bool first, cudaStream_t s) {
  const int64_t items = kKind == L2A_CACHE_BF16 ? 0 : (int64_t)p.f.c.table_stride * p.f.c.Hkv * kDecodeParts, per = kPlanThreads / 32;
  return launch_dependent(weigh_plan_kernel<D, kKind>, dim3((unsigned)(1 + (items + per - 1) / per), items ? p.f.c.B : 1), kPlanThreads, 0, s, !first, p);
}

template <int D>
cudaError_t launch_blocks(const WeighArgs& p, bool first, cudaStream_t s) {
  CUtensorMap mapQ, mapK;
  if (!encode_rows_map(&mapQ, p.rows, p.f.c.Hkv, p.most_blocks * kTileM, D, kTileM, D) || !encode_pool_map(&mapK, p.f.c, p.f.c.K, 1 << p.f.c.page_shift, 1))
    return cudaErrorUnknown;
  cudaError_t e = p.codes.kind == L2A_CACHE_BF16   ? launch_plan<D, L2A_CACHE_BF16>(p, first, s)
                  : p.codes.kind == L2A_CACHE_E4M3 ? launch_plan<D, L2A_CACHE_E4M3>(p, first, s)
                                                   : launch_plan<D, L2A_CACHE_E2M1>(p, first, s);
  const dim3 grid(p.most_blocks, p.f.c.Hkv);
  if (e == cudaSuccess) e = launch_dependent(weigh_rows_kernel<D>, grid, kRowsThreads, 0, s, true, p);
  if (e == cudaSuccess) e = launch_pass<D, false>(mapQ, mapK, p, s);
  if (e == cudaSuccess) e = launch_dependent(weigh_join_kernel, grid, kTileM, 0, s, true, p);
  if (e == cudaSuccess) e = launch_pass<D, true>(mapQ, mapK, p, s);
  return e;
}

int64_t row_stride(const int64_t (&s)[2], int row_elems) {
  if (s[0] != 0 || s[1] < 0) return 0;
  const int64_t t = s[1] ? s[1] : row_elems;
  return t >= row_elems && t % 8 == 0 ? t : 0;
}

l2a_status check_weigh(const l2a_params* p, const l2a_cache* c, int n_tokens, CacheView* v) {
  const int32_t some = 0;
  const l2a_status st = cache_view(p, c, &some, n_tokens, v);
  if (st != L2A_OK) return st;
  if (p->flags & ~L2A_FLAG_SHARED_WINDOW) return L2A_ERR_INVALID_ARG;
  if ((int64_t)n_tokens * p->Hq >= (1ll << 31) - 32 || p->B > 65535 || p->Hkv > 65535) return L2A_ERR_UNSUPPORTED;
  if (most_kept(p, c->kind) > 0 && !cache_few_counts(p, c->kind, true)) return L2A_ERR_UNSUPPORTED;
  // (slots and rows of the blocks are counted in 32 bits, as are the CTAs that decode)
  if (has_blocks(p, c->kind) && ((most_blocks(p, n_tokens) * p->Hkv) >= (1ll << 31) || most_blocks(p, n_tokens) >= (1ll << 31) / kTileM ||
                        key_tiles(p->Lk) * p->Hkv >= (1ll << 31)))
    return L2A_ERR_UNSUPPORTED;
  return L2A_OK;
}
size_t block_bytes(const l2a_params* p, int kind, int n_tokens) { return has_blocks(p, kind) ? layout(p, kind, n_tokens, nullptr, nullptr, nullptr) : 0; }
// What a call takes
size_t weigh_ws_bytes(const l2a_params* p, int kind, int n_tokens) { return kWsHeaderBytes + few_bytes(p, kind) + block_bytes(p, kind, n_tokens); }

}  // namespace
}  // namespace l2a

using namespace l2a;

extern "C" l2a_status l2a_cache_weigh_workspace_bytes(const l2a_params* p, const l2a_cache* c, int n_tokens, size_t* ws_bytes) {
  CacheView v;
  const l2a_status st = check_weigh(p, c, n_tokens, &v);
  if (st != L2A_OK) return st;
  if (!ws_bytes) return L2A_ERR_INVALID_ARG;
  *ws_bytes = kWsHeaderBytes + most_few_bytes(p, c->kind) + block_bytes(p, c->kind, n_tokens);      // (the blocks' part grows with all three)
  return L2A_OK;
}

extern "C" l2a_status l2a_cache_weigh(const l2a_params* p, const l2a_cache* c, const void* Q, const int32_t* cu_new, int n_tokens,
                                      const uint8_t* d, float* weights, int64_t weight_stride, void* ws, size_t ws_bytes, void* stream) {
  CacheFwdArgs a = {};
  l2a_status st = check_weigh(p, c, n_tokens, &a.c);
  if (st == L2A_OK) st = cache_view(p, c, cu_new, n_tokens, &a.c);
  if (st != L2A_OK) return st;
  a.q_t = row_stride(p->q_stride, p->Hq * p->D);
  if (a.q_t == 0) return L2A_ERR_INVALID_ARG;
  const int64_t dense = (int64_t)p->Hkv * c->page_size;
  a.w_page = weight_stride ? weight_stride : dense;
  if (a.w_page < dense) return L2A_ERR_INVALID_ARG;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) % 256) != 0 || ws_bytes < weigh_ws_bytes(p, c->kind, n_tokens)) return L2A_ERR_WORKSPACE;
  if (n_tokens == 0) return L2A_OK;
  if (!Q || !weights || (reinterpret_cast<uintptr_t>(Q) & 15) || (reinterpret_cast<uintptr_t>(weights) & 3)) return L2A_ERR_INVALID_ARG;
  a.Hq = p->Hq;
  a.G = p->Hq / p->Hkv;
  a.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)p->D)) * 1.4426950408889634f;
  a.global = 1;
  a.every = d == nullptr;
  a.q = static_cast<const bf16*>(Q);
  a.d = d;
  a.weights = weights;
  a.status = static_cast<int*>(ws);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint8_t* at = static_cast<uint8_t*>(ws) + kWsHeaderBytes;
  a.few_rows = kept_rows(p, c->kind);
  const bool blocks = has_blocks(p, c->kind);
  // With as many tokens as there can be no sequence is expected to have few rows (as in l2a_cache_forward)
  const bool few = a.few_rows > 0 && !(blocks && (int64_t)p->B * p->Lq == n_tokens);
  if (!few) a.few_rows = 0;
  cudaError_t e = few ? launch_cache_few_weigh(a, at, s) : cudaSuccess;
  if (e == cudaSuccess && blocks) {
    WeighArgs w;
    uint8_t* copy;
    layout(p, c->kind, n_tokens, at + few_bytes(p, c->kind), &w, &copy);
    w.f = a;
    w.codes = a.c;
    w.clear = !few;
    if (c->kind != L2A_CACHE_BF16) {
      CacheView& v = w.f.c;
      v.kind = L2A_CACHE_BF16;
      v.K = copy;
      v.page_bytes = (int64_t)v.Hkv * kTileN * v.D * 2;
      v.page_shift = 7;
      v.table = nullptr;
      v.table_stride = (int)key_tiles(p->Lk);
      v.n_pages = v.B * v.table_stride;
    }
    e = p->D == 128 ? launch_blocks<128>(w, !few, s) : launch_blocks<64>(w, !few, s);
  }
  return e == cudaSuccess ? L2A_OK : L2A_ERR_CUDA;
}
