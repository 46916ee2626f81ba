// Attention over the paged cache for sequences with more query rows (the next chunk of a prompt): rows are the new tokens of
// a sequence times the G heads of a KV group, packed (row i * G + h), 256 of them to a group.  Two kinds of groups:
//   segment 0: all rows; keys max(0, p - W) .. p (Local Attention)
//   segment 1: the rows of routed tokens, compacted; keys 0 .. p - W - 1 (with segment 0 what Global Attention sees)
// so that the scores inside a window are computed once.  s and a are weighted sums of both segments' results.
//
// cache_prepare_kernel: the plan, by one CTA.  Compacts the routed tokens, lists the groups with their key blocks (of 128), and divides the key
//                       blocks of all groups and KV heads, laid end to end, evenly among the CTAs.  Other CTAs, where every key is used
//                       by many rows: an 8-bit cache decoded to bf16 in the workspace, which the rest then reads.
// cache_chunk_kernel  : one CTA an SM takes its range, a few pieces of (group, KV head).  A row whose piece is all there is leaves
//                       finished; other rows go to the piece's slot of the workspace, unnormalised.
// cache_join_kernel   : joins the slots of a row.
//
// A piece: two query tiles of 128 rows share the stream of key blocks; a group of at most 128 rows is in both tiles, which then
// take every other key block each.
//   warps 0-7   : soft-max, correction and epilogue, one thread a row; they also gather the rows of Q
//   warp 8      : TMA producer, one copy a page (and 64 columns in bf16)
//   warp 9      : tcgen05 MMA issuer and TMEM owner
//   warps 12-15 : one thread a key.  e4m3: decode keys and values to the bf16 tiles that the products read, exactly (code * 2^e), so that
//                 both kinds of caches share all that follows, to the bit.  Both kinds: zeros for the values of keys that no row of the
//                 group sees (their slots may hold anything).
// Weights enter the second product as bf16, one term (8 bits; the sum of the weights is taken before), as in l2a_forward: a second term would be
// half as many products again.
//
// Measured, 2000 tokens on 34768 keys (32/8 heads, D = 128, window 4096, a fifth routed; 21.5K key blocks of two tiles): call 352 us from
// an 8-bit cache (decoded once: 42 us for 213 MB), in a shorter run 341 next to 329 from bf16; 329 GFLOP = 0.93 to 1.00 PFLOP/s.  A key block
// takes 2900 clk, 2048 of them its products; the tensor pipe is active 62 % of a launch and the special-function unit 46 %.  A piece takes
// about 9600 clk besides: look-up 100, first scores 540, last products 2900, store of Q and results 6050.
// In a long loop the power cap lowers the clock (388 us at 1.67 of 1.965 GHz; 409 in another run).
// Decoding in the products' kernel, four sequences of 16384 keys, 383 tokens each (32/8 heads): 366 us next to 208 from bf16, 262 for an
// earlier form with K as 8-bit operands (Q in two e4m3 terms) and values relative to the largest of 32 keys in fp16: there a large value
// took bits from rows that do not see it, and small elements of Q were lost.  Tried for the decoding: codes spread to bf16 by integer
// operations 446 us, codes in a ring of their own with two stages of K 400, six warps instead of four 353.
#include <math.h>

#include <algorithm>

#include "cache_common.cuh"
#include "cache_ranges.h"

namespace l2a {

namespace {

constexpr int kKStages = 3, kVStages = 2;
constexpr int kSoftmaxWarps = 8, kTmaWarp = 8, kMmaWarp = 9, kConvWarp = 12, kConvWarps = 4;
constexpr int kChunkThreads = 512;
// The launch has 16 warps of 128 registers; the two warpgroups that do not compute rows give most of theirs away (with 184 and 72 the
// soft-max spills 136 bytes instead of 16).
constexpr int kSoftmaxRegs = 200, kOtherRegs = 56;
static_assert(kSoftmaxWarps * kSoftmaxRegs + 8 * kOtherRegs <= 16 * 128, "register shares exceed the launch allocation");
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr int kBoxBytes = 128 * 128;       // 128 rows of 128 bytes
constexpr int kPlanThreads = 1024;
constexpr int kCtas = kSplitSms;

// A group of rows
struct alignas(16) Group {
  int b, seg, dual, first;       // sequence, segment, one tile twice, its first row of the token axis,
  int off, list, row0, n_rows;   // position of that row; segment 1: its list of routed tokens starts here; first packed row; rows
  int jlo, jhi, key_lo, key_hi;  // keys that some row sees, and their blocks (jhi < jlo: none)
  int64_t base;                  // first key block of the group's heads in the call
  int hi0, lo1;                  // last block of tile 0, first of tile 1
  int min_hi0, min_hi1, max_lo0, max_lo1;      // of each tile: keys from max_lo to min_hi are seen by all its rows
};
static_assert(sizeof(Group) == 80, "copied by 16 bytes");
struct alignas(16) Start { int blocks, group, head, block; };   // a CTA's range: its key blocks, and where it begins

struct Plan {
  int n_groups, ctas;
  int64_t at[kCtas + 1];         // first key block, of the call's, of every CTA's range
  Start start[kCtas];
};

// What the join has to know of a token
struct alignas(16) TokenInfo {
  int index, rank;         // among the new tokens of its sequence (-1: of none here), among the routed ones that see keys before
                           // their window (-1: not one)
  int group[2];            // first group of the sequence in both segments
};

// Workspace: plan, groups, then per token: its info, list of routed tokens; per sequence: first group of both segments, its part
// of the list.
struct ChunkWs {
  Plan* plan;
  Group* groups;
  TokenInfo* token;
  int* list;
  int *first_group, *list_start, *list_end;   // [2][B], [B], [B]
  int64_t* group_cost;             // of the groups before each
  float* part;
};

__host__ __device__ inline int64_t most_groups(int n_tokens, int G, int B) {
  return 2 * (((int64_t)n_tokens * G + kRowsPerCta - 1) / kRowsPerCta + B);
}
__host__ __device__ constexpr size_t slot_floats(int D) { return (size_t)kRowsPerCta * (D + 2); }

struct ChunkArgs {
  CacheFwdArgs f;
  ChunkWs w;
  CacheView codes;       // the 8-bit cache that f.c is the decoded copy of
  int clear;             // no kernel ahead has cleared the status word
  int wide;              // the call's key blocks may cost more than 32 bits count
};

// ------------------------------------------------------------------------------------------------------------- plan
__device__ __forceinline__ bool is_chunk(const CacheFwdArgs& a, int n) { return (int64_t)n * a.G > a.few_rows; }

// Inclusive scans of kN values over the CTA's threads, in place; all: the sums.  Two barriers.
template <int kN, class T>
__device__ __forceinline__ void block_scan(T (&x)[kN], T (*sums)[kPlanThreads / 32], T (&all)[kN]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      const T u = __shfl_up_sync(0xffffffffu, x[k], o);
      if (lane >= o) x[k] += u;
    }
  }
  __syncthreads();
  if (lane == 31)
    for (int k = 0; k < kN; ++k) sums[k][warp] = x[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    const T mine = sums[k][lane];                      // (as many warps as lanes)
    T u = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T i = __shfl_up_sync(0xffffffffu, u, o);
      if (lane >= o) u += i;
    }
    all[k] = __shfl_sync(0xffffffffu, u, 31);
    x[k] += __shfl_sync(0xffffffffu, u - mine, warp);
  }
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

// Bound by latencies: what is searched lies in shared memory where it fits (kKeep sequences, kKeepCosts groups), else in the workspace.
constexpr int kKeep = 1024, kKeepCosts = 512;
struct PlanSmem {
  int64_t cost[kKeepCosts], base[kKeepCosts], at[kCtas + 1], sums2[2][kPlanThreads / 32];     // (T)
  int blocks[kKeepCosts];
  int first[kKeep], n[kKeep], length[kKeep], group[2 * kKeep], start[kKeep], end[kKeep], sums[1][kPlanThreads / 32];
};
// T: what key blocks and costs are summed in
template <class T>
__device__ void make_plan(const ChunkArgs& p, PlanSmem& sm) {
  const CacheFwdArgs& a = p.f;
  const CacheView& c = a.c;
  const ChunkWs& w = p.w;
  int *keep_first = sm.first, *keep_n = sm.n, *keep_length = sm.length, *keep_blocks = sm.blocks;
  T *keep_cost = reinterpret_cast<T*>(sm.cost), *keep_base = reinterpret_cast<T*>(sm.base);
  static_assert(kPlanThreads == 1024, "block_scan");
  const int tid = threadIdx.x;
  const bool small = c.B <= kKeep;
  int* first_group = small ? sm.group : w.first_group;
  int* list_start = small ? sm.start : w.list_start;
  int* list_end = small ? sm.end : w.list_end;
  // ---- the sequences.  (Lists of new tokens that do not ascend: no groups, nothing is stored.)
  bool bad = false;
  if (c.cu_new != nullptr)
    for (int b = tid; b < c.B; b += kPlanThreads) bad |= c.cu_new[b] > c.cu_new[b + 1];
  bad = __syncthreads_or(bad);
  auto sequence = [&](int b, int& first, int& length) -> int {       // new tokens, 0: none here
    const int n = bad ? 0 : cache_new(c, b, first);
    length = cache_length(c, b);
    return is_chunk(a, n) ? n : 0;
  };
  if (small && tid < c.B) {
    int first = 0, length = 0;
    keep_n[tid] = sequence(tid, first, length);
    keep_first[tid] = c.cu_new != nullptr ? c.cu_new[tid] : first;   // (ascending, whatever else is wrong with a sequence)
    keep_length[tid] = length;
  }
  __syncthreads();
  auto sequence_of = [&](int t, int& first, int& n, int& length) -> int {      // -1: of none here
    const int b = c.cu_new == nullptr ? t / c.Lq : small ? last_not_above(keep_first, c.B, t) : last_not_above(c.cu_new, c.B, t);
    if (small) {
      first = keep_first[b];
      n = keep_n[b];
      length = keep_length[b];
    } else {
      n = sequence(b, first, length);
    }
    return n > 0 && t >= first && t < first + n ? b : -1;
  };
  // ---- compact the routed tokens that see keys before their windows
  int base = 0, x[1], all[1];
  for (int t0 = 0; t0 < c.n_tokens; t0 += kPlanThreads) {
    const int t = t0 + tid;
    int b = -1, first = 0, n = 0, length = 0;
    const bool routed = a.global && a.d != nullptr && t < c.n_tokens && a.d[t] != 0;
    if (t < c.n_tokens && !bad && (c.cu_new == nullptr || t >= (small ? keep_first[0] : c.cu_new[0]))) b = sequence_of(t, first, n, length);
    const int take = b >= 0 && routed && length - n + (t - first) - a.shift >= 0;
    x[0] = take;
    block_scan(x, sm.sums, all);
    const int at = base + x[0] - take;
    if (t < c.n_tokens) w.token[t] = TokenInfo{b >= 0 ? t - first : -1, take ? at : -1, {b, 0}};      // (completed below)
    if (b >= 0 && t == first) list_start[b] = at;
    if (b >= 0 && t == first + n - 1) list_end[b] = at + take;
    if (take) w.list[at] = t;
    base += all[0];
  }
  __syncthreads();
  // ---- groups of both segments, sequence by sequence
  base = 0;
  for (int b0 = 0; b0 < c.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int first, length, n = 0, loc = 0, out = 0;
    if (b < c.B) n = small ? keep_n[b] : sequence(b, first, length);
    if (n > 0) {
      loc = a.local ? (int)compact_groups(n, a.G) : 0;
      out = (int)compact_groups(list_end[b] - list_start[b], a.G);
    }
    x[0] = loc + out;
    block_scan(x, sm.sums, all);
    const int at = base + x[0] - loc - out;
    if (b < c.B) {
      first_group[b] = at;
      first_group[c.B + b] = at + loc;
    }
    base += all[0];
  }
  const int n_groups = base;
  __syncthreads();
  for (int t = tid; t < c.n_tokens; t += kPlanThreads) {
    TokenInfo x = w.token[t];                          // (written by this thread)
    if (x.index < 0) continue;
    const int b = x.group[0];
    if (x.rank >= 0) x.rank -= list_start[b];
    x.group[0] = first_group[b];
    x.group[1] = first_group[c.B + b];
    w.token[t] = x;
  }
  // ---- the groups, their key blocks and costs laid end to end
  const bool few_groups = n_groups <= kKeepCosts;
  T* cost_before = few_groups ? keep_cost : reinterpret_cast<T*>(w.group_cost);
  T base_blocks = 0, base_cost = 0;
  for (int q0 = 0; q0 < n_groups; q0 += kPlanThreads) {
    const int q = q0 + tid;
    Group g;
    g.dual = 0;
    int x = 0;
    if (q < n_groups) {
      const int b = last_not_above(first_group, c.B, q), out0 = first_group[c.B + b];      // (the last: it has groups)
      int length;
      int n;
      if (small) {
        g.first = keep_first[b];
        n = keep_n[b];
        length = keep_length[b];
      } else {
        n = sequence(b, g.first, length);
      }
      g.b = b;
      g.seg = q >= out0;
      g.off = length - n;
      g.list = g.seg ? list_start[b] : 0;
      g.row0 = (q - (g.seg ? out0 : first_group[b])) * kRowsPerCta;
      g.n_rows = min(kRowsPerCta, (g.seg ? list_end[b] - g.list : n) * a.G - g.row0);
      g.dual = g.n_rows <= kTileM;
      const int shift = g.seg ? a.shift : 0;
      auto pos = [&](int r) {                          // position of packed row r of the group
        const int i = (g.row0 + r) / a.G;
        return g.off + (g.seg ? w.list[g.list + i] - g.first : i);
      };
      auto low = [&](int y) { return g.seg ? 0 : max(0, y - a.window); };
      const int i1 = g.dual ? g.n_rows - 1 : kTileM - 1, i2 = g.dual ? 0 : kTileM;
      const int p0 = pos(0), p1 = pos(i1), p2 = pos(i2), p3 = pos(g.n_rows - 1);
      g.key_lo = low(p0);
      g.key_hi = p3 - shift;
      g.jlo = g.key_lo / kTileN;
      g.jhi = g.key_hi >= 0 ? g.key_hi / kTileN : g.jlo - 1;
      g.hi0 = g.dual ? g.jhi : p1 - shift >= 0 ? (p1 - shift) / kTileN : g.jlo - 1;
      g.lo1 = g.dual ? g.jlo : low(p2) / kTileN;
      g.min_hi0 = p0 - shift;
      g.min_hi1 = p2 - shift;
      g.max_lo0 = low(p1);
      g.max_lo1 = low(p3);
      x = g.jhi - g.jlo + 1;
    }
    const T blocks = (T)x * c.Hkv, cost = (T)group_cost(x, g.dual, c.Hkv);
    T at[2] = {blocks, cost}, both[2];
    block_scan(at, reinterpret_cast<T(*)[kPlanThreads / 32]>(sm.sums2), both);
    if (q < n_groups) {
      g.base = base_blocks + at[0] - blocks;
      w.groups[q] = g;
      cost_before[q] = base_cost + at[1] - cost;
      if (few_groups) { keep_base[q] = g.base; keep_blocks[q] = g.dual ? -x : x; }
    }
    base_blocks += both[0];
    base_cost += both[1];
  }
  __syncthreads();
  // ---- the CTAs' ranges
  const int ctas = (int)max((T)1, min((T)kCtas, base_blocks));
  if (tid == 0) { w.plan->n_groups = n_groups; w.plan->ctas = ctas; }
  Start start = {0, 0, 0, 0};
  T* range_at = reinterpret_cast<T*>(sm.at);
  if (tid <= kCtas) {
    T at = tid == 0 ? 0 : base_blocks;
    if (tid > 0 && tid < ctas) {
      const T cost = (T)range_cost(tid, ctas, base_cost);
      start.group = last_not_above(cost_before, n_groups, cost);         // (the last: it has blocks)
      const Group& g = w.groups[start.group];
      const int kept = few_groups ? keep_blocks[start.group] : (g.jhi - g.jlo + 1) * (g.dual ? -1 : 1);
      const RangePlace place = range_place(cost - cost_before[start.group], abs(kept), kept < 0);
      start.head = place.head;
      start.block = place.block;
      at = (T)range_first(few_groups ? keep_base[start.group] : g.base, place, abs(kept));
    }
    range_at[tid] = at;
    w.plan->at[tid] = at;
  }
  __syncthreads();
  if (tid < kCtas) {
    start.blocks = (int)(range_at[tid + 1] - range_at[tid]);
    w.plan->start[tid] = start;
  }
}

// Decoded copy: pages of 128 tokens, [page][KV head][128][D] of K and of V.  A lane brings 16 codes, a warp 512 / D keys at a time, 32
// keys of a head of K or V in all.  HBM-bound: 3 bytes a code, of the keys that some row sees.
constexpr int kDecodeKeys = 32, kDecodeParts = kTileN / kDecodeKeys;
template <int D, int kKind>
__device__ __forceinline__ void decode_cache(const ChunkArgs& p, int item, int b) {
  constexpr bool kE2M1 = kKind == L2A_CACHE_E2M1;
  constexpr int kLanes = D / 16, kRows = 32 / kLanes, kSteps = kDecodeKeys / kRows;
  const CacheFwdArgs& a = p.f;
  const CacheView &c = p.codes, &out = a.c;
  const int lane = threadIdx.x & 31, sub = lane % kLanes;
  int first;
  const int n = cache_new(c, b, first), length = cache_length(c, b);
  if (!is_chunk(a, n)) return;
  const int value = item & 1, part = (item >> 1) % kDecodeParts, row = item / (2 * kDecodeParts), head = row % c.Hkv, block = row / c.Hkv;
  const int key0 = block * kTileN + part * kDecodeKeys, window = max(0, length - n - a.window);
  const bool may_route = a.global && a.d != nullptr, inside = key0 < length && (may_route || key0 + kDecodeKeys > window);
  const uint8_t *src = value ? c.V : c.K, *exps = value ? c.vs : c.ks;
  uint4 x[kSteps];                 // (e2m1: half of it)
  uint32_t e[kSteps], t[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int key = key0 + i * kRows + lane / kLanes;
    const int page = inside && key < length && (may_route || key >= window) ? cache_page(c, b, key) : -1;
    const int in_page = key & ((1 << c.page_shift) - 1);
    const int64_t slot = ((int64_t)head << c.page_shift) + in_page;
    const uint8_t* row = src + page * c.page_bytes + slot * row_bytes(kKind, D);
    if (kE2M1) {
      const uint2 y = page >= 0 ? *reinterpret_cast<const uint2*>(row + sub * 8) : make_uint2(0u, 0u);
      x[i] = make_uint4(y.x, y.y, 0u, 0u);
      t[i] = page >= 0 ? exps[page * c.scale_stride + blocks_at<D>(c, head, in_page) + sub] : 0u;
    } else {
      x[i] = page >= 0 ? *reinterpret_cast<const uint4*>(row + sub * 16) : make_uint4(0, 0, 0, 0);
    }
    e[i] = page >= 0 ? exps[page * c.scale_stride + exponent_at<D, kKind>(c, head, in_page)] : 0u;
  }
  // all keys where a token is routed, else those of the windows (looked up while the codes are on their way)
  bool routed = false;
  if (may_route)
    for (int i = threadIdx.x; i < n; i += kPlanThreads) routed |= a.d[first + i] != 0;
  routed = __syncthreads_or(routed);
  if (!inside || (!routed && key0 + kDecodeKeys <= window)) return;
  uint8_t* dst = (value ? out.V : out.K) + (int64_t)(b * out.table_stride + block) * out.page_bytes +
                 ((int64_t)head * kTileN + part * kDecodeKeys) * (2 * D);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    uint32_t o[8];
    if (kE2M1) decode_16(make_uint2(x[i].x, x[i].y), e4m3_value(t[i]) * scale_of_exponent(e[i]), o);
    else decode_16(x[i], scale_of_exponent(e[i]), o);
    store_32(dst + (i * kRows + lane / kLanes) * (2 * D) + sub * 32, true, o);
  }
}

// The first CTA plans; the others, a row of the grid for each sequence, decode: 213 MB in 42 us (35K tokens, 8 heads, D = 128), two CTAs of
// half the registers an SM 48.
template <int D, int kKind>
__global__ void __launch_bounds__(kPlanThreads) cache_prepare_kernel(const ChunkArgs p) {
  dependency_wait();
  dependents_release();
  if (blockIdx.x == 0) {
    if (blockIdx.y != 0) return;
    if (p.clear && threadIdx.x == 0) *p.f.status = 0;
    __shared__ PlanSmem sm;
    if (p.wide) make_plan<int64_t>(p, sm);
    else make_plan<int>(p, sm);
    return;
  }
  decode_cache<D, kKind>(p, (blockIdx.x - 1) * (kPlanThreads / 32) + (threadIdx.x >> 5), blockIdx.y);
}

// ------------------------------------------------------------------------------------------------------------- pieces
struct ChunkPiece {
  int head, j0, j1;        // KV head; key blocks j0 .. j1
  bool whole;              // all of the group's blocks
  int item;                // group * Hkv + head
};
// The pieces of a CTA's range in order; every warp walks through them by itself, and reads of a group what it needs (few
// registers: those of the soft-max warps are taken by the scores).
constexpr int kKeepGroups = 16;
struct ChunkWalk {
  int left, group, head, block, n_groups;      // key blocks of the range that are left, and where it has come to
  const Group* kept;       // the first kKeepGroups of the range, in shared memory
  int kept_from;
  __device__ __forceinline__ const Group& group_now(const ChunkWs& w) const {
    return group - kept_from < kKeepGroups ? kept[group - kept_from] : w.groups[group];
  }
  __device__ __forceinline__ bool init(const ChunkWs& w, const Group* keep) {
    const int cta = blockIdx.x;
    kept = keep;
    n_groups = w.plan->n_groups;
    const int4 s = *reinterpret_cast<const int4*>(&w.plan->start[cta]);
    left = s.x;
    group = kept_from = s.y;
    head = s.z;
    block = s.w;
    return cta < w.plan->ctas && left > 0 && group < n_groups;
  }
  __device__ __forceinline__ bool next(const ChunkWs& w, int Hkv, ChunkPiece& p) {
    if (left <= 0) return false;
    int n, jlo;
    for (;;) {
      const int2 j = *reinterpret_cast<const int2*>(&group_now(w).jlo);
      jlo = j.x;
      n = j.y - j.x + 1;
      if (head < Hkv && block < n) break;
      block = 0;
      if (++head >= Hkv || n <= 0) {
        head = 0;
        if (++group >= n_groups) return false;
      }
    }
    const int take = min(n - block, left);
    p.head = head;
    p.j0 = jlo + block;
    p.j1 = p.j0 + take - 1;
    p.whole = take == n;
    p.item = group * Hkv + head;
    left -= take;
    block += take;
    return true;
  }
};
// First and last block of tile t in the piece (first > last: none), and their distance
struct TileBlocks { int first, last, step; };
__device__ __forceinline__ TileBlocks tile_blocks(const Group& g, const ChunkPiece& p, int t) {
  TileBlocks x;
  if (g.dual) {
    x.first = p.j0 + ((p.j0 ^ t) & 1);
    x.last = p.j1 - ((p.j1 ^ t) & 1);
    x.step = 2;
  } else {
    x.first = t ? max(p.j0, g.lo1) : p.j0;
    x.last = t ? p.j1 : min(p.j1, g.hi0);
    x.step = 1;
  }
  return x;
}

constexpr int kBarBytes = 512;
template <int D, int kKind>
struct ChunkSmem {
  static constexpr int kQTileBytes = kTileM * D * 2;
  static constexpr int kKTileBytes = kTileN * D * 2;
  static constexpr int kVTileBytes = kTileN * D * 2;
  // Codes land where their bf16 tile will be: with D = 128 on its second 64 columns, a key's 128 codes on the same 128 bytes that its
  // values take there, so that a thread finds its row and leaves it without the others.  Rows of 64 codes do not fit that way.  e2m1: the rows,
  // behind them the scales of their blocks and their exponents; they are read by all threads before the first writes.
  static constexpr int kCodes = kTileN * row_bytes(kKind, D);
  static constexpr int kBlocks = kTileN * (D / 16);
  static constexpr bool kApart = kKind == L2A_CACHE_E4M3 && D == 64;
  static constexpr int kKOff = 2 * kQTileBytes;
  static constexpr int kVOff = kKOff + kKStages * kKTileBytes;
  static constexpr int kRawOff = kVOff + kVStages * kVTileBytes;
  static constexpr int kBarOff = kRawOff + (kApart ? (kKStages + kVStages) * kCodes : 0);
  static __device__ __forceinline__ uint8_t* k_codes(uint8_t* smem, int s) {
    return kApart ? smem + kRawOff + s * kCodes : smem + kKOff + s * kKTileBytes + (D == 128 ? kBoxBytes : 0);
  }
  static __device__ __forceinline__ uint8_t* v_codes(uint8_t* smem, int s) {
    return kApart ? smem + kRawOff + (kKStages + s) * kCodes : smem + kVOff + s * kVTileBytes + (D == 128 ? kBoxBytes : 0);
  }
  static constexpr int kGroupOff = kBarOff + kBarBytes;
  static constexpr int kTotal = kGroupOff + kKeepGroups * (int)sizeof(Group) + 1024 /* alignment slack */;
};

struct ChunkBars {
  uint64_t q_full[2];
  uint64_t k_full[kKStages], k_empty[kKStages], v_full[kVStages], v_empty[kVStages];
  uint64_t s_full[2], p_half[2], p_full[2], o_final[2];
  uint64_t k_raw[kKStages], v_raw[kVStages];             // e4m3: codes; bf16: V before the clearing
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(ChunkBars) <= kBarBytes, "barriers");

__device__ __forceinline__ void sts128(uint32_t saddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(saddr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// A soft-max thread's row in a piece
struct RowOf {
  TileBlocks tb;
  int token, head, lo, hi;       // first and last key that it sees
  int min_hi, max_lo;            // of the tile
  int slot;
  bool valid, seg, whole;        // whole: the piece holds all of the row's keys in this segment
  int rank;                      // segment 0: whether other keys are to be joined (>= 0),
  uint8_t routed;                // and the routing decision; looked up here, needed at the piece's end
};

template <int D, int kKind>
__global__ void __launch_bounds__(kChunkThreads, 1)
cache_chunk_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const ChunkArgs p) {
  using SM = ChunkSmem<D, kKind>;
  constexpr bool kCoded = kKind != L2A_CACHE_BF16, kE2M1 = kKind == L2A_CACHE_E2M1;
  constexpr int kKSteps = D / 16;      // MMA k-steps of Q*K^T
  constexpr int kOCol0 = 2 * kTileN;   // first TMEM column of the O accumulators
  const CacheFwdArgs& a = p.f;
  const CacheView& c = a.c;
  const ChunkWs& w = p.w;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;
  uint8_t* sK = smem + SM::kKOff;
  uint8_t* sV = smem + SM::kVOff;
  ChunkBars* bar = reinterpret_cast<ChunkBars*>(smem + SM::kBarOff);
  Group* sGroups = reinterpret_cast<Group*>(smem + SM::kGroupOff);
  volatile int* abort_flag = &bar->abort_flag;

  if (tid == kTmaWarp * 32) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(&bar->q_full[t], kTileM);
      mbar_init(&bar->s_full[t], 1);
      mbar_init(&bar->p_half[t], kTileM);
      mbar_init(&bar->p_full[t], kTileM);
      mbar_init(&bar->o_final[t], 1);
    }
    for (int s = 0; s < kKStages; ++s) {
      mbar_init(&bar->k_raw[s], 1);
      mbar_init(&bar->k_full[s], kCoded ? kConvWarps * 32 : 1);
      mbar_init(&bar->k_empty[s], 1);
    }
    for (int s = 0; s < kVStages; ++s) {
      mbar_init(&bar->v_full[s], kConvWarps * 32);
      mbar_init(&bar->v_empty[s], 1);
      mbar_init(&bar->v_raw[s], 1);
    }
    bar->abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(&bar->tmem_base, 512);
    tmem_relinquish();
  }
  dependency_wait();
  dependents_release();
  {
    constexpr int kWords = sizeof(Group) / 16;
    const int from = w.plan->start[blockIdx.x].group, n = min(kKeepGroups, w.plan->n_groups - from);
    for (int i = tid; i < n * kWords; i += kChunkThreads)
      reinterpret_cast<uint4*>(sGroups)[i] = reinterpret_cast<const uint4*>(w.groups + from)[i];
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bar->tmem_base;
  if (tmem != 0) {
    // all 512 columns were requested, so the allocation must start at column 0 (the MMA warp relies on it)
    __syncthreads();
    if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
    if (tid == 0) atomicExch(a.status, 3);
    return;
  }

  if (warp == kTmaWarp) {
    // =========================================================================== TMA producer
    setmaxnreg_dec<kOtherRegs>();
    if (lane == 0) {
      tma_prefetch_desc(&mapK);
      tma_prefetch_desc(&mapV);
    }
    ChunkWalk walk;
    ChunkPiece pc;
    bool ok = walk.init(w, sGroups);
    // a lane copies the rows of page `u` of a block, in bf16 64 columns of them
    const int rows = 1 << c.page_shift, copies = 128 >> c.page_shift, u = lane % copies, piece = lane / copies;
    // (e2m1: the codes, the scales of their blocks, the exponents)
    const bool active = piece < (kE2M1 ? 3 : kCoded ? 1 : D / 64);
    const uint32_t bytes = rows * (kE2M1 ? (piece == 0 ? D / 2 : piece == 1 ? D / 16 : 1) : kCoded ? D : 128);
    uint32_t k_slot = 0, k_ph = 1, v_cnt = 0;
    while (ok && walk.next(w, c.Hkv, pc)) {
      const Group& g = walk.group_now(w);
      const int b = g.b, key_lo = g.key_lo, key_hi = g.key_hi, step = g.dual ? 2 : 1;
      const int first_entry = key_lo >> c.page_shift, last_entry = key_hi >> c.page_shift;
      int entry0 = -512, page_ids = -1;
      // pages of block j, 32 of them at a time (a block of V lies `step` blocks behind that of K)
      auto copy = [&](int j, uint8_t* dst, const CUtensorMap* map, const uint8_t* scales, uint64_t* full) {
        const int key = j * kTileN + u * rows, entry = key >> c.page_shift;
        if (((j * kTileN) >> c.page_shift) < entry0 || ((j * kTileN + kTileN - 1) >> c.page_shift) - entry0 >= 32) {
          entry0 = (max(j - step, 0) * kTileN) >> c.page_shift;
          const int e = entry0 + lane;
          page_ids = e >= first_entry && e <= last_entry ? cache_page(c, b, e << c.page_shift) : -1;
        }
        const int page = __shfl_sync(0xffffffffu, page_ids, entry - entry0);
        const bool load = active && page >= 0 && key <= key_hi && key + rows > key_lo;
        const uint32_t expect = kE2M1 ? __reduce_add_sync(0xffffffffu, load ? bytes : 0u) : __popc(__ballot_sync(0xffffffffu, load)) * bytes;
        if (lane == 0) mbar_expect_tx(full, expect);
        __syncwarp();
        if (!load) return;
        if (kE2M1 && piece > 0) {
          const uint8_t* src = scales + page * c.scale_stride + (piece == 1 ? blocks_at<D>(c, pc.head, 0) : exponent_at<D, kKind>(c, pc.head, 0));
          bulk_load(dst + SM::kCodes + (piece == 1 ? u * rows * (D / 16) : SM::kBlocks + u * rows), src, bytes, full);
        } else {
          tma_load_page(dst + (kCoded ? u * rows * row_bytes(kKind, D) : piece * kBoxBytes + u * rows * 128), map, full, kCoded, piece, 0,
                        pc.head, page);
        }
      };
      auto copy_v = [&](int j) -> bool {
        const int s = v_cnt & 1;
        if (!mbar_wait_warp(&bar->v_empty[s], ((v_cnt >> 1) & 1) ^ 1, abort_flag)) return false;
        copy(j, kCoded ? SM::v_codes(smem, s) : sV + s * SM::kVTileBytes, &mapV, c.vs, &bar->v_raw[s]);
        ++v_cnt;
        return true;
      };
      auto copy_k = [&](int j) -> bool {
        if (!mbar_wait_warp(&bar->k_empty[k_slot], k_ph, abort_flag)) return false;
        copy(j, kCoded ? SM::k_codes(smem, k_slot) : sK + k_slot * SM::kKTileBytes, &mapK, c.ks, kCoded ? &bar->k_raw[k_slot] : &bar->k_full[k_slot]);
        if (++k_slot == kKStages) { k_slot = 0; k_ph ^= 1; }
        return true;
      };
      // In the order in which the products take them.  e4m3: in that of the decoding, which has K done while V is on its way.
      for (int j = pc.j0 - step; ok && j <= pc.j1; ++j) {
        if (!kCoded && j >= pc.j0) ok = copy_v(j);
        if (ok && j + step <= pc.j1) ok = copy_k(j + step);
        if (kCoded && ok && j >= pc.j0) ok = copy_v(j);
      }
    }
  } else if (warp == kMmaWarp) {
    // =========================================================================== MMA issuer
    setmaxnreg_dec<kOtherRegs>();
    if (elect_one()) {
      constexpr uint32_t tmem = 0;   // checked above: TMEM operand addresses are immediates in this loop
      constexpr uint32_t idesc_qk = idesc_bf16_f32(kTileM, kTileN, 0, 0), idesc_pv = idesc_bf16_f32(kTileM, D, 0, 1);
      auto k_major = [](const uint8_t* tile) { return smem_desc_sw128(smem_u32(tile), 16, 1024); };
      const uint64_t dq0 = k_major(sQ), dq1 = k_major(sQ + SM::kQTileBytes), dk0 = k_major(sK);
      const uint64_t dv0 = smem_desc_sw128(smem_u32(sV), kBoxBytes, 1024);
      const uint64_t dv1 = smem_desc_sw128(smem_u32(sV + SM::kVTileBytes), kBoxBytes, 1024);
      uint32_t p_cnt[2] = {0, 0}, q_cnt[2] = {0, 0};
      bool started[2];

      auto issue_qk = [&](int t, int s) {
        const uint64_t qd = t ? dq1 : dq0, kd = dk0 + s * (SM::kKTileBytes >> 4);
        const uint32_t d = tmem + t * kTileN;
#pragma unroll
        for (int kk = 0; kk < kKSteps; ++kk) {
          const uint32_t o = ((kk >> 2) * kBoxBytes + (kk & 3) * 32) >> 4;
          mma_ss(d, qd + o, kd + o, idesc_qk, kk > 0);
        }
        tc_commit(&bar->s_full[t]);
      };
      auto issue_pv = [&](int t, int s, int half, uint32_t acc) {   // P*V of 64 keys
        const uint64_t vd = s ? dv1 : dv0;
        const uint32_t d = tmem + kOCol0 + t * D, q = tmem + t * kTileN + half * 64;
#pragma unroll
        for (int kk = 0; kk < kTileN / 32; ++kk)
          mma_ts(d, q + kk * 8, vd + (((half * 4 + kk) * 2048) >> 4), idesc_pv, kk > 0 ? 1u : acc);
      };

      uint32_t k_slot = 0, k_ph = 0;
      ChunkWalk walk;
      ChunkPiece pc;
      bool ok = walk.init(w, sGroups);
      uint32_t it = 0;
      while (ok && walk.next(w, c.Hkv, pc)) {
        const TileBlocks tb[2] = {tile_blocks(walk.group_now(w), pc, 0), tile_blocks(walk.group_now(w), pc, 1)};
        const bool dual = walk.group_now(w).dual;
        auto takes = [&](int t, int j) {
          return t ? j >= tb[1].first && j <= tb[1].last && (!dual || (j & 1)) : j >= tb[0].first && j <= tb[0].last && (!dual || !(j & 1));
        };
        // scores of block j for tile t; the tile's rows of Q arrive with its first block
        auto scores = [&](int t, int j, int s) {
          if (!started[t]) {
            if (!mbar_spin(&bar->q_full[t], q_cnt[t] & 1, abort_flag)) { ok = false; return; }
            ++q_cnt[t];
            started[t] = true;
            tc_fence_after();
          }
          issue_qk(t, s);
        };
        started[0] = started[1] = false;
        // Each tile has the scores of one block under way: the next block's, or where the tiles take turns those of
        // the two next blocks.
        const int step = dual ? 2 : 1;
        auto k_done = [&]() {
          tc_commit(&bar->k_empty[k_slot]);
          if (++k_slot == kKStages) { k_slot = 0; k_ph ^= 1; }
        };
        for (int i = 0; ok && i < step && pc.j0 + i <= pc.j1; ++i) {
          if (!mbar_spin(&bar->k_full[k_slot], k_ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
#pragma unroll
          for (int t = 0; t < 2; ++t)
            if (ok && takes(t, pc.j0 + i)) scores(t, pc.j0 + i, k_slot);
          if (ok) k_done();
        }
        for (int j = pc.j0; ok && j <= pc.j1; ++j, ++it) {
          const int s = it & 1;
          const bool more = j + step <= pc.j1;
          // Both operand blocks of this step are waited for ahead of the probabilities (a wait between the products, even one already
          // satisfied, is part of a tile's serial chain); where the tiles take turns there is time in between.
          if (!mbar_spin(&bar->v_full[s], (it >> 1) & 1, abort_flag)) { ok = false; break; }
          if (more && !dual && !mbar_spin(&bar->k_full[k_slot], k_ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (ok && takes(t, j)) {
              const uint32_t pp = p_cnt[t] & 1;
              if (!mbar_spin(&bar->p_half[t], pp, abort_flag)) { ok = false; break; }
              tc_fence_after();
              issue_pv(t, s, 0, j > tb[t].first ? 1u : 0u);
              if (!mbar_spin(&bar->p_full[t], pp, abort_flag)) { ok = false; break; }
              ++p_cnt[t];
              tc_fence_after();
              issue_pv(t, s, 1, 1u);
              if (j == tb[t].last) tc_commit(&bar->o_final[t]);
            }
            if (ok && more && takes(t, j + step)) {
              if (dual && !mbar_spin(&bar->k_full[k_slot], k_ph, abort_flag)) { ok = false; break; }
              tc_fence_after();
              scores(t, j + step, k_slot);
            }
          }
          if (!ok) break;
          tc_commit(&bar->v_empty[s]);
          if (more) k_done();
        }
      }
    }
    __syncwarp();
  } else if (warp >= kConvWarp) {
    // =========================================================================== decoding and clearing
    setmaxnreg_dec<kOtherRegs>();
    const int row = (warp - kConvWarp) * 32 + lane;      // this thread's key of a block
    ChunkWalk walk;
    ChunkPiece pc;
    bool ok = walk.init(w, sGroups);
    uint32_t it = 0, k_slot = 0, k_ph = 0;
    while (ok && walk.next(w, c.Hkv, pc)) {
      const Group& g = walk.group_now(w);
      const int b = g.b, key_lo = g.key_lo, key_hi = g.key_hi, step = g.dual ? 2 : 1;
      auto seen = [&](int j) { return j * kTileN + row >= key_lo && j * kTileN + row <= key_hi; };
      if (!kCoded) {
        for (int j = pc.j0; ok && j <= pc.j1; ++j, ++it) {
          const int s = it & 1;
          if (!mbar_wait_warp(&bar->v_raw[s], (it >> 1) & 1, abort_flag)) { ok = false; break; }
          if (!seen(j)) {
            const uint32_t dst = smem_u32(sV + s * SM::kVTileBytes) + row * 128;
#pragma unroll
            for (int k = 0; k < D / 8; ++k) sts128(dst + (k >> 3) * kBoxBytes + ((k & 7) << 4), 0u, 0u, 0u, 0u);
            fence_async_smem();
          }
          mbar_arrive(&bar->v_full[s]);
        }
        continue;
      }
      if (kE2M1) {
        // this thread's row of a block of codes, times its blocks' scales and 2^e, to its tile
        auto decode = [&](const uint8_t* codes, uint8_t* tile, uint64_t* raw, uint32_t ph, uint64_t* full, bool zero) -> bool {
          constexpr int kPieces = D / 32;                      // of 32 codes
          const bool here = mbar_wait_warp(raw, ph, abort_flag);
          const uint32_t src = smem_u32(codes), dst = smem_u32(tile) + row * 128;
          uint4 x[kPieces];
          uint32_t t[2] = {}, e = 0;
          if (here) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
              const float4 y = lds128(src + row * (D / 2) + ((D == 128 ? i ^ ((row >> 1) & 3) : i ^ ((row >> 2) & 1)) << 4));
              x[i] = zero ? make_uint4(0u, 0u, 0u, 0u)
                          : make_uint4(__float_as_uint(y.x), __float_as_uint(y.y), __float_as_uint(y.z), __float_as_uint(y.w));
            }
            const uint8_t* scales = codes + SM::kCodes;
            if (!zero) {
              t[0] = *reinterpret_cast<const volatile uint32_t*>(scales + row * (D / 16));
              if (D == 128) t[1] = *reinterpret_cast<const volatile uint32_t*>(scales + row * (D / 16) + 4);
              e = *reinterpret_cast<const volatile uint8_t*>(scales + SM::kBlocks + row);
            }
          }
          // (all leave together where a wait ran out)
          if (!named_barrier_all(2, kConvWarps * 32, here)) return false;
          const float scale = scale_of_exponent(e);
#pragma unroll
          for (int i = 0; i < kPieces; ++i) {
            uint32_t lo, hi;
            e4m3x4_to_f16(t[i / 2] >> (i % 2) * 16 & 0xffffu, lo, hi);
            const float2 f = f16x2_to_float2(lo);
            const uint32_t at = dst + i / 2 * kBoxBytes;
            uint32_t o[8];
            decode_16(make_uint2(x[i].x, x[i].y), f.x * scale, o);
            sts128(at + ((((i & 1) * 4) ^ (row & 7)) << 4), o[0], o[1], o[2], o[3]);
            sts128(at + ((((i & 1) * 4 + 1) ^ (row & 7)) << 4), o[4], o[5], o[6], o[7]);
            decode_16(make_uint2(x[i].z, x[i].w), f.y * scale, o);
            sts128(at + ((((i & 1) * 4 + 2) ^ (row & 7)) << 4), o[0], o[1], o[2], o[3]);
            sts128(at + ((((i & 1) * 4 + 3) ^ (row & 7)) << 4), o[4], o[5], o[6], o[7]);
          }
          fence_async_smem();
          mbar_arrive(full);
          return true;
        };
        for (int j = pc.j0 - step; ok && j <= pc.j1; ++j) {
          if (j + step <= pc.j1) {
            ok = decode(SM::k_codes(smem, k_slot), sK + k_slot * SM::kKTileBytes, &bar->k_raw[k_slot], k_ph, &bar->k_full[k_slot], false);
            if (++k_slot == kKStages) { k_slot = 0; k_ph ^= 1; }
          }
          if (ok && j >= pc.j0) {
            const int s = it & 1;
            ok = decode(SM::v_codes(smem, s), sV + s * SM::kVTileBytes, &bar->v_raw[s], (it >> 1) & 1, &bar->v_full[s], !seen(j));
            ++it;
          }
        }
        continue;
      }
      // Of this thread's key in block j: its entry of the table (-1: none is needed), and from that the exponents of its rows of K and V.  What
      // is loaded is looked at a block later.
      auto entry_of = [&](int j) -> int {
        return seen(j) ? c.table[(int64_t)b * c.table_stride + ((j * kTileN + row) >> c.page_shift)] : -1;
      };
      auto exponents = [&](int j, int entry, uint32_t& k, uint32_t& v) {
        k = v = 0u;
        if (entry < 0 || entry >= c.n_pages) return;
        const int64_t at = entry * c.scale_stride + ((int64_t)pc.head << c.page_shift) + ((j * kTileN + row) & ((1 << c.page_shift) - 1));
        k = c.ks[at];
        v = c.vs[at];
      };
      // this thread's row of a block of codes, times 2^e, to its tile
      auto decode = [&](const uint8_t* codes, uint8_t* tile, uint64_t* raw, uint32_t ph, uint64_t* full, uint32_t e, bool zero) -> bool {
        if (!mbar_wait_warp(raw, ph, abort_flag)) return false;
        const uint32_t src = smem_u32(codes) + row * D, dst = smem_u32(tile) + row * 128;
        const float scale = scale_of_exponent(e);
#pragma unroll 1
        for (int half = 0; half < D / 64; ++half) {          // (64 columns at a time: the second half of the codes is overwritten last)
          uint4 x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 y = lds128(src + ((D == 128 ? (half * 4 + i) ^ (row & 7) : i ^ ((row >> 1) & 3)) << 4));
            x[i] = zero ? make_uint4(0u, 0u, 0u, 0u)
                        : make_uint4(__float_as_uint(y.x), __float_as_uint(y.y), __float_as_uint(y.z), __float_as_uint(y.w));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t o[8];
            decode_16(x[i], scale, o);
            const uint32_t at = dst + half * kBoxBytes;
            sts128(at + (((2 * i) ^ (row & 7)) << 4), o[0], o[1], o[2], o[3]);
            sts128(at + (((2 * i + 1) ^ (row & 7)) << 4), o[4], o[5], o[6], o[7]);
          }
        }
        fence_async_smem();
        mbar_arrive(full);
        return true;
      };
      // Pages are looked up three blocks ahead of K, exponents two; those of V wait until its block comes, `step` behind that of K.
      uint32_t k_now, k_next, v_now, v_next, v_back1 = 0, v_back2 = 0;
      exponents(pc.j0, entry_of(pc.j0), k_now, v_now);
      exponents(pc.j0 + 1, entry_of(pc.j0 + 1), k_next, v_next);
      int entry = entry_of(pc.j0 + 2);
      for (int j = pc.j0 - step; ok && j <= pc.j1; ++j) {
        const int x = j + step;
        if (x <= pc.j1) {
          ok = decode(SM::k_codes(smem, k_slot), sK + k_slot * SM::kKTileBytes, &bar->k_raw[k_slot], k_ph, &bar->k_full[k_slot], k_now, false);
          if (++k_slot == kKStages) { k_slot = 0; k_ph ^= 1; }
        }
        if (ok && j >= pc.j0) {
          const int s = it & 1;
          ok = decode(SM::v_codes(smem, s), sV + s * SM::kVTileBytes, &bar->v_raw[s], (it >> 1) & 1, &bar->v_full[s],
                      step == 2 ? v_back2 : v_back1, !seen(j));
          ++it;
        }
        v_back2 = v_back1;
        v_back1 = v_now;
        k_now = k_next;
        v_now = v_next;
        exponents(x + 2, entry, k_next, v_next);
        entry = entry_of(x + 3);
      }
    }
  } else if (warp > kMmaWarp) {
    setmaxnreg_dec<kOtherRegs>();     // idle warps of the third warpgroup
  } else {
    // =========================================================================== soft-max warpgroups
    setmaxnreg_inc<kSoftmaxRegs>();
    const int t = warp >> 2;                 // tile of this warpgroup
    const int r = (warp & 3) * 32 + lane;    // row inside the tile == TMEM lane
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lane_base + t * kTileN;        // this row's 128 score columns
    const uint32_t o_addr = tmem + lane_base + kOCol0 + t * D;    // its D accumulator columns
    ChunkWalk walk;
    ChunkPiece pc;
    RowOf me;
    constexpr int kPieces = D / 8, kRowsPerStep = 32 / kPieces;
    const int piece = lane % kPieces;
    // The next piece and this thread's row of it
    auto advance = [&]() -> bool {
      if (!walk.next(w, c.Hkv, pc)) return false;
      const Group& g = walk.group_now(w);
      me.tb = tile_blocks(g, pc, t);
      me.min_hi = t ? g.min_hi1 : g.min_hi0;
      me.max_lo = t ? g.max_lo1 : g.max_lo0;
      const int dual = g.dual, seg = g.seg, tile_row = (dual ? 0 : t * kTileM) + r;
      me.valid = tile_row < g.n_rows;
      me.seg = seg;
      me.whole = pc.whole && !dual;
      me.rank = seg && a.local ? 0 : -1;
      me.routed = 0;
      me.slot = pc.item + blockIdx.x;
      me.token = me.head = 0;
      me.lo = 0x3fffffff;
      me.hi = -1;
      if (me.valid) {
        const int x = g.row0 + tile_row, i = x / a.G;
        me.token = seg ? w.list[g.list + i] : g.first + i;
        me.head = pc.head * a.G + x - i * a.G;
        const int pos = g.off + me.token - g.first;
        me.hi = pos - (seg ? a.shift : 0);
        me.lo = seg ? 0 : pos - a.window;
        if (!seg) {
          me.rank = w.token[me.token].rank;
          if (a.global && a.d != nullptr) me.routed = a.d[me.token];
        }
      }
      if (me.valid) {
        const bf16* q = a.q + me.token * a.q_t + (int64_t)me.head * D;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(q));
        if (D == 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + 64));
      }
      return true;
    };
    // The warp's 32 rows of Q, 16-byte pieces, to where a TMA copy would leave them
    auto store_q = [&]() {
      uint4 qx[kPieces];
      const bf16* src = me.valid ? a.q + me.token * a.q_t + (int64_t)me.head * D : nullptr;
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const bf16* q = reinterpret_cast<const bf16*>(
            __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(src), k * kRowsPerStep + lane / kPieces));
        qx[k] = q != nullptr ? __ldcg(reinterpret_cast<const uint4*>(q) + piece) : make_uint4(0, 0, 0, 0);
      }
      const uint32_t base = smem_u32(sQ + t * SM::kQTileBytes);
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const int rr = (warp & 3) * 32 + k * kRowsPerStep + lane / kPieces;
        sts128(base + (piece >> 3) * kBoxBytes + rr * 128 + (((piece & 7) ^ (rr & 7)) << 4), qx[k].x, qx[k].y, qx[k].z, qx[k].w);
      }
      fence_async_smem();
      mbar_arrive(&bar->q_full[t]);
    };

    bool ok = walk.init(w, sGroups);
    bool more = ok && advance();
    if (more && me.tb.first <= me.tb.last) store_q();
    uint32_t s_cnt = 0, o_cnt = 0;
    while (more) {
      const RowOf cur = me;
      const TileBlocks tb = cur.tb;
      const bool any = tb.first <= tb.last, warp_has_rows = __any_sync(0xffffffffu, cur.valid);
      float m_use = -INFINITY;   // reference maximum, exp2 domain
      float l = 0.f;             // row sum
      for (int j = tb.first; j <= tb.last; j += tb.step) {
        // warp-uniform outcome: the TMEM loads/stores below are warp-collective
        if (!mbar_wait_warp(&bar->s_full[t], s_cnt & 1, abort_flag)) { ok = false; break; }
        ++s_cnt;
        tc_fence_after();
        if (!warp_has_rows) {    // nothing of these rows is ever stored
          mbar_arrive(&bar->p_half[t]);
          mbar_arrive(&bar->p_full[t]);
          continue;
        }
        const int k0 = j * kTileN;
        const bool partial = k0 + kTileN - 1 > cur.min_hi || k0 < cur.max_lo;
        uint32_t v[4][32];       // the row's scores of this key block
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32(s_addr + q * 32, v[q]);
        tmem_ld_wait();
        if (partial) {
          // the row's visible keys are one range, hence one bit per column; a masked score becomes -inf whatever it was
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t visible = bit_range(cur.lo - k0 - q * 32, cur.hi + 1 - k0 - q * 32);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[q][e] = (visible >> e) & 1u ? v[q][e] : 0xff800000u;
          }
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
#pragma unroll
          for (int q = 0; q < 4; ++q) mx[q] = fmax3(mx[q], __uint_as_float(v[q][e]), __uint_as_float(v[q][e + 1]));
        }
        const float m_new = fmaxf(m_use, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2);
        // rescale the running sum and the TMEM accumulator only when the maximum moved a lot
        const bool need = j == tb.first ? false : m_new - m_use > kRescaleThreshold;
        if (j == tb.first) m_use = m_new;
        if (__any_sync(0xffffffffu, need)) {
          const float alpha = need ? fast_exp2(m_use - m_new) : 1.0f;
          l *= alpha;
#pragma unroll 1
          for (int q = 0; q < D / 32; ++q) {
            uint32_t o[32];
            tmem_ld32(o_addr + q * 32, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            tmem_st32(o_addr + q * 32, o);
          }
          if (need) m_use = m_new;
        }
        const float neg_m = m_use == -INFINITY ? 0.f : -m_use;
        // probabilities; the 16-bit P of keys 64h .. 64h+63 overwrites score columns 64h .. 64h+31, a quarter of the
        // exponentials on the FMA pipe, and the first half is handed over while the second is computed
        float2 sum2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t pk[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float2 y = __ffma2_rn(make_float2(__uint_as_float(v[q][2 * e]), __uint_as_float(v[q][2 * e + 1])),
                                        make_float2(a.scale_log2, a.scale_log2), make_float2(neg_m, neg_m));
            const float2 z = e % 4 == 3 ? exp2_fma2(y) : make_float2(fast_exp2(y.x), fast_exp2(y.y));
            sum2 = __fadd2_rn(sum2, z);
            pk[e] = pack_bf16(z.x, z.y);
          }
          tmem_st16(s_addr + (q >> 1) * 64 + (q & 1) * 16, pk);
          if (q == 1) {
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(&bar->p_half[t]);
          }
        }
        l += sum2.x + sum2.y;
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&bar->p_full[t]);
      }
      // The next piece is looked up while this one's last products run, and its rows of Q are in place before this one's results are
      // stored, so that its first scores are computed meanwhile.
      if (!ok) break;
      more = advance();
      if (any) {
        if (!mbar_wait_warp(&bar->o_final[t], o_cnt & 1, abort_flag)) { ok = false; break; }
        ++o_cnt;
      }
      tc_fence_after();
      if (more && me.tb.first <= me.tb.last) store_q();

      // ---- a row that has nothing else to be joined with leaves finished, others go to the piece's slot
      const bool valid = cur.valid, finished = cur.whole && cur.rank < 0;
      float* slot = w.part + (size_t)cur.slot * slot_floats(D) + t * kTileM * (D + 2);
      const bool here = finished && valid && dbg_in_range(cur.token >= 0 && cur.token < c.n_tokens && cur.head < a.Hq, a.status);
      bf16* dst = here ? a.O + cur.token * a.o_t + (int64_t)cur.head * D : nullptr;
      const float inv_l = l != 0.f ? (cur.routed != 0 ? 2.f : 1.f) / l : 0.f;      // (finished and routed: no key before the window, a = s)
      // Four lanes, four rows: each lane stores the same 16 bytes of all four, so that a store covers 64 bytes of a row
      bf16* rows[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        rows[k] = reinterpret_cast<bf16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(dst), (lane & ~3) + k));
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        uint32_t o[32];
        if (any) {
          tmem_ld32(o_addr + q * 32, o);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0u;                      // no block of this tile: the accumulator was never written
        }
        if (valid && !finished) {
#pragma unroll
          for (int x = 0; x < 8; ++x)
            *reinterpret_cast<float4*>(slot + ((q * 8 + x) * kTileM + r) * 4) =
                make_float4(__uint_as_float(o[4 * x]), __uint_as_float(o[4 * x + 1]), __uint_as_float(o[4 * x + 2]), __uint_as_float(o[4 * x + 3]));
        }
        if (__any_sync(0xffffffffu, dst != nullptr)) {
          float2 old[16];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint4 u = a.add && dst != nullptr ? reinterpret_cast<const uint4*>(dst + q * 32)[x] : make_uint4(0, 0, 0, 0);
            const uint32_t ow[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) old[4 * x + e] = make_float2(__uint_as_float(ow[e] << 16), __uint_as_float(ow[e] & 0xffff0000u));
          }
          uint32_t pk[4][4];
#pragma unroll
          for (int e = 0; e < 16; ++e)
            pk[e / 4][e % 4] = pack_bf16(fmaf(__uint_as_float(o[2 * e]), inv_l, old[e].x), fmaf(__uint_as_float(o[2 * e + 1]), inv_l, old[e].y));
#pragma unroll
          for (int step = 1; step <= 2; step *= 2) {
            const bool up = lane & step;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              if (x & step) continue;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? pk[x][e] : pk[x + step][e], step);
                if (up) pk[x][e] = got; else pk[x + step][e] = got;
              }
            }
          }
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (rows[k] != nullptr) reinterpret_cast<uint4*>(rows[k] + q * 32)[lane & 3] = make_uint4(pk[k][0], pk[k][1], pk[k][2], pk[k][3]);
        }
      }
      if (valid && !finished) {
        slot[kTileM * D + r] = m_use;
        slot[kTileM * (D + 1) + r] = any ? l : 0.f;
      }
      tc_fence_before();       // the accumulators have been read; the next piece's products come behind this warp's arrivals
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

// ------------------------------------------------------------------------------------------------------------- join
// The parts of one row in the slots of its (group, KV head)
struct RowParts {
  const float* tile;     // half of the first slot that has the row,
  int r;                 // its lane
  int n, tiles;          // slots, halves of each
  bool complete;         // one part only
};
template <int D>
__device__ __forceinline__ RowParts row_parts(const ChunkWs& w, int group, int Hkv, int head, int row, const int* starts, int ctas, bool wide) {
  RowParts x;
  const int64_t base = w.groups[group].base;
  const int blocks = w.groups[group].jhi - w.groups[group].jlo + 1, dual = w.groups[group].dual;
  x.tiles = dual ? 2 : 1;
  x.r = row % kTileM;
  x.n = 0;
  x.tile = nullptr;
  x.complete = false;
  if (blocks <= 0) return x;
  int c0, c1;
  if (wide) {
    const int64_t lo = base + (int64_t)head * blocks;
    c0 = last_not_above(w.plan->at, ctas, lo);
    c1 = last_not_above(w.plan->at, ctas, lo + blocks - 1);
  } else {
    const int lo = (int)base + head * blocks;
    c0 = last_not_above(starts, ctas, lo);
    c1 = last_not_above(starts, ctas, lo + blocks - 1);
  }
  x.n = c1 - c0 + 1;
  x.complete = x.n == 1 && !dual;
  x.tile = w.part + (size_t)(group * Hkv + head + c0) * slot_floats(D) + row / kTileM * (kTileM * (D + 2));
  return x;
}

// A CTA takes 32 packed rows of the token axis and one KV head, a thread kPieces times four columns of a row.  Bound by latencies: the
// loads of kAhead parts are in flight together, maxima, sums and accumulators in one pass.
template <int D, int kPieces, int kAhead>
__global__ void __launch_bounds__(256) cache_join_kernel(const ChunkArgs p) {
  const CacheFwdArgs& a = p.f;
  const ChunkWs& w = p.w;
  __shared__ int starts[kCtas];
  const int row = blockIdx.x * 32 + (threadIdx.x & 31);
  const int piece0 = (blockIdx.z * 8 + (threadIdx.x >> 5)) * kPieces, head = blockIdx.y, t = row / a.G, h = row - t * a.G;
  const bool inside = t < a.c.n_tokens;
  dependency_wait();
  TokenInfo tok = {-1, -1, {0, 0}};
  bool routed = false;
  if (inside) {
    *reinterpret_cast<int4*>(&tok) = *reinterpret_cast<const int4*>(w.token + t);
    routed = a.global && a.d != nullptr && a.d[t] != 0;
  }
  const int ctas = w.plan->ctas, status = *a.status;
  if (threadIdx.x < kCtas) starts[threadIdx.x] = (int)w.plan->at[threadIdx.x];
  __syncthreads();
  if (tok.index < 0 || (a.add && !routed)) return;
  RowParts part[2] = {};
  if (a.local) {
    const int x = tok.index * a.G + h;
    part[0] = row_parts<D>(w, tok.group[0] + x / kRowsPerCta, a.c.Hkv, head, x % kRowsPerCta, starts, ctas, p.wide);
    if (part[0].complete && tok.rank < 0) return;
  }
  if (tok.rank >= 0) {
    const int x = tok.rank * a.G + h;
    part[1] = row_parts<D>(w, tok.group[1] + x / kRowsPerCta, a.c.Hkv, head, x % kRowsPerCta, starts, ctas, p.wide);
    if (part[1].complete && !a.local) return;
  }
  if (status != 0) return;                 // a wait ran out: nothing more is stored
  if (!dbg_in_range(tok.index < a.c.Lq && tok.rank < a.c.n_tokens && head * a.G + h < a.Hq, a.status)) return;
  // of the window and of what lies before it
  constexpr size_t kSlot = (size_t)kRowsPerCta * (D + 2), kHalf = (size_t)kTileM * (D + 2);
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float4 f[2][kPieces] = {};
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int n = part[s].n * part[s].tiles, r = part[s].r;
    for (int i0 = 0; i0 < n; i0 += kAhead) {
      float ls[kAhead], ms[kAhead], m_new = m[s];
      float4 v[kAhead][kPieces];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = min(i0 + u, n - 1);
        const float* x = part[s].tile + (part[s].tiles == 2 ? (i >> 1) * kSlot + (i & 1) * kHalf : i * kSlot);
        ms[u] = x[kTileM * D + r];
        ls[u] = i0 + u < n ? x[kTileM * (D + 1) + r] : 0.f;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) v[u][k] = *reinterpret_cast<const float4*>(x + ((piece0 + k) * kTileM + r) * 4);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (ls[u] != 0.f) m_new = fmaxf(m_new, ms[u]);       // (0: no key of that part is visible to the row)
      if (m_new == -INFINITY) {                // no key, or scores that are NaN: so is the result then
#pragma unroll
        for (int u = 0; u < kAhead; ++u) l[s] += ls[u];
        continue;
      }
      const float old = fast_exp2(m[s] - m_new);
      l[s] *= old;
#pragma unroll
      for (int k = 0; k < kPieces; ++k) { f[s][k].x *= old; f[s][k].y *= old; f[s][k].z *= old; f[s][k].w *= old; }
      m[s] = m_new;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (ls[u] == 0.f) continue;
        const float g = fast_exp2(ms[u] - m_new);
        l[s] = fmaf(ls[u], g, l[s]);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
          f[s][k].x = fmaf(g, v[u][k].x, f[s][k].x);
          f[s][k].y = fmaf(g, v[u][k].y, f[s][k].y);
          f[s][k].z = fmaf(g, v[u][k].z, f[s][k].z);
          f[s][k].w = fmaf(g, v[u][k].w, f[s][k].w);
        }
      }
    }
  }
  const float m_all = fmaxf(m[0], m[1]);
  const float k0 = l[0] != 0.f ? fast_exp2(m[0] - m_all) : 0.f, k1 = l[1] != 0.f ? fast_exp2(m[1] - m_all) : 0.f;
  const float l_all = fmaf(k0, l[0], k1 * l[1]);
  const float g_all = routed && l_all != 0.f ? 1.f / l_all : 0.f;
  const float w0 = (a.local && l[0] != 0.f ? 1.f / l[0] : 0.f) + g_all * k0, w1 = g_all * k1;
  uint2* dst = reinterpret_cast<uint2*>(a.O + t * a.o_t + (int64_t)(head * a.G + h) * D) + piece0;
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    float4 o = make_float4(fmaf(w0, f[0][k].x, w1 * f[1][k].x), fmaf(w0, f[0][k].y, w1 * f[1][k].y),
                           fmaf(w0, f[0][k].z, w1 * f[1][k].z), fmaf(w0, f[0][k].w, w1 * f[1][k].w));
    if (a.add) {
      const uint2 old = dst[k];
      o.x += __uint_as_float(old.x << 16); o.y += __uint_as_float(old.x & 0xffff0000u);
      o.z += __uint_as_float(old.y << 16); o.w += __uint_as_float(old.y & 0xffff0000u);
    }
    dst[k] = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
  }
}

// ------------------------------------------------------------------------------------------------------------- host
// A cache of codes is decoded once where a sequence can have kDecodeRows rows of a KV head or more: each 256 of them would decode its keys
// again.  us decoded in the products' kernel / once (window 4096, a fifth routed), 8 bits: 560 rows of each of eight sequences of 32K (28/4 heads) 246 /
// 283, 800 of one (32/8) 94 / 97, 1050 of one (28/4) 65 / 67, of four of 16K 120 / 123, of one of 6000 42 / 39, 1200 of four of 4000 (32/8)
// 127 / 114, 1470 of one of 64K (28/4) 134 / 116, 1532 of four of 16K (32/8) 366 / 269.  Not for copies beyond kMostDecoded bytes.
// 4 bits take longer to decode there, so that the copy is worth it sooner: 280 rows of one of 32K (28/4) 64 / 70, 560 of each of eight 339 / 303, 800 of
// one (32/8) 123 / 106, 1050 of one of 6000 (28/4) 52 / 45, of four of 16K 182 / 131, 1532 of four (32/8) 472 / 284.
constexpr int64_t kDecodeRows = 1024, kDecodeRows4 = 512, kMostDecoded = 4ll << 30;
int decoded_pages(int Lk) { return (Lk + kTileN - 1) / kTileN; }
int64_t decoded_bytes(int B, int Lk, int Hkv, int D) { return 2ll * B * decoded_pages(Lk) * Hkv * kTileN * D * 2; }
size_t layout(int B, int n_tokens, int G, int Hkv, int D, uint8_t* base, ChunkWs* w) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    uint8_t* p = base + at;
    at += align_up(bytes, 256);
    return p;
  };
  const size_t groups = (size_t)most_groups(n_tokens, G, B), tokens = n_tokens;
  ChunkWs x;
  x.plan = reinterpret_cast<Plan*>(take(sizeof(Plan)));
  x.groups = reinterpret_cast<Group*>(take(groups * sizeof(Group)));
  x.group_cost = reinterpret_cast<int64_t*>(take(groups * 8));
  x.token = reinterpret_cast<TokenInfo*>(take(tokens * sizeof(TokenInfo)));
  x.list = reinterpret_cast<int*>(take(tokens * 4));
  x.first_group = reinterpret_cast<int*>(take((size_t)B * 8));
  x.list_start = reinterpret_cast<int*>(take((size_t)B * 4));
  x.list_end = reinterpret_cast<int*>(take((size_t)B * 4));
  x.part = reinterpret_cast<float*>(take((groups * Hkv + kCtas) * slot_floats(D) * sizeof(float)));
  if (w) *w = x;
  return at;
}

template <int D, int kKind>
cudaError_t launch_prepare(const ChunkArgs& p, bool decode, bool first, cudaStream_t s) {
  const unsigned items = decode ? (unsigned)(p.f.c.table_stride * p.f.c.Hkv * 2 * kDecodeParts) : 0, per = kPlanThreads / 32;
  return launch_dependent(cache_prepare_kernel<D, kKind>, dim3(1 + (items + per - 1) / per, decode ? p.f.c.B : 1), kPlanThreads, 0, s, !first, p);
}

template <int D, int kKind>
cudaError_t launch_chunk(const ChunkArgs& p, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t s) {
  constexpr int smem = ChunkSmem<D, kKind>::kTotal;
  static PerDeviceOnce once;
  cudaError_t e = once.run([] {
    return cudaFuncSetAttribute(cache_chunk_kernel<D, kKind>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  });
  if (e != cudaSuccess) return e;
  e = launch_dependent(cache_chunk_kernel<D, kKind>, dim3(kCtas), kChunkThreads, smem, s, true, mapK, mapV, p);
  if (e != cudaSuccess) return e;
  // Few rows have many parts each: their columns over several CTAs, and more parts in flight.  Many rows have two or three parts, and
  // registers are CTAs that an SM has room for.  Whole call, four parts in flight / two: 2000 tokens on 34K keys (32/8 heads) 363 / 353 us, 290
  // on 1253 (28/4, two sequences) 33 / 35.
  const unsigned rows = (unsigned)(((int64_t)p.f.c.n_tokens * p.f.G + 31) / 32), heads = p.f.c.Hkv;
  const int64_t ctas = (int64_t)rows * heads;
  if (ctas <= kSplitSms) return launch_dependent(cache_join_kernel<D, 1, 8>, dim3(rows, heads, D / 32), 256, 0, s, true, p);
  if (ctas <= 4 * kSplitSms) return launch_dependent(cache_join_kernel<D, D / 32, 4>, dim3(rows, heads), 256, 0, s, true, p);
  return launch_dependent(cache_join_kernel<D, D / 32, 2>, dim3(rows, heads), 256, 0, s, true, p);
}

template <int D>
cudaError_t launch_both(const ChunkArgs& p, const CUtensorMap& mapK, const CUtensorMap& mapV, bool decode, bool first, cudaStream_t s) {
  const cudaError_t e = p.codes.kind == L2A_CACHE_E2M1 ? launch_prepare<D, L2A_CACHE_E2M1>(p, decode, first, s)
                                                       : launch_prepare<D, L2A_CACHE_E4M3>(p, decode, first, s);
  if (e != cudaSuccess) return e;
  return p.f.c.kind == L2A_CACHE_BF16   ? launch_chunk<D, L2A_CACHE_BF16>(p, mapK, mapV, s)
         : p.f.c.kind == L2A_CACHE_E4M3 ? launch_chunk<D, L2A_CACHE_E4M3>(p, mapK, mapV, s)
                                        : launch_chunk<D, L2A_CACHE_E2M1>(p, mapK, mapV, s);
}

}  // namespace

size_t cache_chunk_ws_bytes(const l2a_params* p, int n_tokens) {
  return layout(p->B, n_tokens, p->Hq / p->Hkv, p->Hkv, p->D, nullptr, nullptr);
}

size_t cache_copy_bytes(const l2a_params* p, int kind) {
  const int64_t rows = (int64_t)p->Lq * (p->Hq / p->Hkv), least = kind == L2A_CACHE_E2M1 ? kDecodeRows4 : kDecodeRows;
  if (kind == L2A_CACHE_BF16 || rows < least || p->B > 65535) return 0;
  const int64_t bytes = decoded_bytes(p->B, p->Lk, p->Hkv, p->D);
  return bytes <= kMostDecoded ? (size_t)bytes : 0;
}

bool cache_chunk_counts(const l2a_params* p, int n_tokens) {
  return most_blocks(most_groups(n_tokens, p->Hq / p->Hkv, p->B), p->Hkv, p->Lk) < kMostBlocks;
}

cudaError_t launch_cache_chunk(const CacheFwdArgs& a, bool first, void* ws, bool decode, cudaStream_t s) {
  ChunkArgs p;
  p.f = a;
  p.clear = first;
  p.wide = most_cost(most_groups(a.c.n_tokens, a.G, a.c.B), a.c.Hkv, a.c.max_keys) >= (double)(1u << 31);
  const size_t at = layout(a.c.B, a.c.n_tokens, a.G, a.c.Hkv, a.c.D, static_cast<uint8_t*>(ws), &p.w);
  p.codes = a.c;
  if (decode) {
    CacheView& c = p.f.c;
    c.kind = L2A_CACHE_BF16;
    c.K = static_cast<uint8_t*>(ws) + at;
    c.V = c.K + decoded_bytes(c.B, c.max_keys, c.Hkv, c.D) / 2;
    c.ks = c.vs = nullptr;
    c.page_bytes = (int64_t)c.Hkv * kTileN * c.D * 2;
    c.page_shift = 7;
    c.table = nullptr;
    c.table_stride = decoded_pages(c.max_keys);
    c.n_pages = c.B * c.table_stride;
  }
  const CacheView& c = p.f.c;
  CUtensorMap mapK, mapV;
  const int rows = 1 << c.page_shift;
  if (!encode_pool_map(&mapK, c, c.K, rows, 1) || !encode_pool_map(&mapV, c, c.V, rows, 1)) return cudaErrorUnknown;
  return c.D == 128 ? launch_both<128>(p, mapK, mapV, decode, first, s) : launch_both<64>(p, mapK, mapV, decode, first, s);
}

}  // namespace l2a
