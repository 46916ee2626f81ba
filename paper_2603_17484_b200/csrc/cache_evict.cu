// Eviction from a paged cache (l2a_cache_evict): of every sequence and KV head the first tokens, the last ones and those of the highest
// weights in between move, in order, into the pages of another table.
//
// cache_select_kernel: a cluster takes a KV head of a sequence, each of its CTAs a range of the positions, whose weights it keeps in shared
//                      memory as whole numbers of the same order.  The least weight that stays is found digit by digit (11, 11 and 10 bits): a
//                      CTA counts its numbers by digit, and every CTA adds up the counts of all.  Then each lists what stays, at its place.
//                      Equal weights stay from the lowest position on, whatever the number of CTAs.  Bound by latencies: 32K positions a head, 16 x 8
//                      heads in clusters of four 26 to 30 us, one sequence of 9001 15 (digits of 8 bits: 33 and 21).
// cache_move_kernel  : 64 rows of 256 bytes of a head a CTA (128 of 128, else 256), 16 bytes a thread; nothing is computed.
//                      16 sequences of up to 32K tokens, 40 % kept (8 heads, D = 128, e2m1): 38 us for 177 MB = 4.7 TB/s; with 64 rows a CTA 53.
#include "cache_common.cuh"

namespace l2a {

namespace {

constexpr int kSelectThreads = 1024, kSelectWarps = kSelectThreads / 32;
constexpr int kMostCluster = 8;              // CTAs of a cluster (portable)
constexpr int kShareKeys = 8192;             // positions of a CTA where the cluster may grow (with 4096, clusters of eight, 32K positions take longer),
constexpr int kKeepKeys = 48 * 1024;         // and the most that it keeps in shared memory; beyond, weights are read again
constexpr int kMoveThreads = 256;
// Rows of a CTA: four dependent loads lead to a row, so that a thread has several of them under way
__host__ __device__ constexpr int move_rows(int row_bytes) { return row_bytes >= 256 ? 64 : row_bytes == 128 ? 128 : 256; }

struct EvictArgs {
  CacheView c, to;
  const float* w;
  float* w_to;
  int64_t w_page, w_to_page;     // elements of a page of weights
  const int32_t* keep;
  int sinks, recent, most;       // most: tokens of a sequence that can stay
  int32_t *kept, *count, *lengths;
  int* status;                   // the workspace's status word
};

// What stays of a sequence: its first tokens, the last, and the best in between
struct Kept { int length, all, first, last, middle; };
__device__ __forceinline__ Kept kept_of(const EvictArgs& a, int b) {
  Kept k;
  k.length = cache_length(a.c, b);
  k.all = min(min(max(a.keep[b], 0), a.most), k.length);
  k.last = min(a.recent, k.all);
  k.first = min(a.sinks, k.all - k.last);
  k.middle = k.all - k.last - k.first;
  return k;
}
// Whole numbers in the order of the weights; both zeros alike, NaN below all
__device__ __forceinline__ uint32_t ordered(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return isnan(w) ? 0u : u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ uint32_t remote_u32(const uint32_t* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_map(smem_u32(p), rank)));
  return v;
}
__device__ __forceinline__ uint2 remote_u64(const uint32_t* p, uint32_t rank) {
  uint2 v;
  asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(cluster_map(smem_u32(p), rank)));
  return v;
}

constexpr int kRounds = 3, kDigits = 2048;
struct SelectSmem {
  alignas(8) uint32_t counts[kRounds][kDigits];     // of each digit
  uint32_t warp_sum[kSelectWarps];
  uint32_t digit, left;
  uint32_t above[kSelectWarps], equal[kSelectWarps];
  uint32_t cta_above, cta_equal;
};

// Bound by latencies: three rounds of counting with a cluster barrier each.  (The counts of a digit fall into few places, since weights have few
// exponents; atomics without a result that meet in a warp are one.)
template <bool kKeep>
__global__ void __launch_bounds__(kSelectThreads) cache_select_kernel(const EvictArgs a) {
  extern __shared__ uint32_t keys[];
  __shared__ SelectSmem sm;
  const CacheView& c = a.c;
  const int ctas = gridDim.x, rank = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  dependents_release();
  const Kept k = kept_of(a, b);
  int32_t* out = a.kept + ((int64_t)b * c.Hkv + g) * a.most;
  if (rank == 0 && g == 0 && tid == 0) {
    a.count[b] = k.all;
    if (b == 0) *a.status = 0;
  }
  // what stays whatever its weight, and no positions behind it
  const int from = k.first, to = k.length - k.last;        // the positions in between
  for (int64_t i = rank * kSelectThreads + tid; i < a.most; i += ctas * kSelectThreads) {
    if (i < k.first) out[i] = (int32_t)i;
    else if (i >= k.all) out[i] = -1;
    else if (i >= k.all - k.last || k.all == k.length) out[i] = k.length - k.all + (int32_t)i;
  }
  if (k.middle == 0 || k.all == k.length) return;          // (the same for the whole cluster)
  for (int i = tid; i < kRounds * kDigits; i += kSelectThreads) sm.counts[0][i] = 0u;
  // ---- this CTA's range, in parts of 32 positions for each warp
  const int n = to - from, parts = n / 32 + (n % 32 != 0), share = (parts + ctas - 1) / ctas;
  auto edge = [&](int r) { return from + (int)min((int64_t)n, (int64_t)r * share * 32); };
  const int first = edge(rank), mine = edge(rank + 1) - first;
  auto load = [&](int i) -> uint32_t {
    const int pos = first + i, page = cache_page(c, b, pos);
    if (page < 0) return 0u;
    return ordered(a.w[page * a.w_page + ((int64_t)g << c.page_shift) + (pos & ((1 << c.page_shift) - 1))]);
  };
  auto key = [&](int i) { return kKeep ? keys[i] : load(i); };
  if (kKeep) {
#pragma unroll 4
    for (int64_t i = tid; i < mine; i += kSelectThreads) keys[i] = load((int)i);
  }
  __syncthreads();
  // ---- digit by digit: `left` of the numbers that begin with `prefix` stay, and all above them
  uint32_t prefix = 0, left = k.middle;
#pragma unroll 1
  for (int round = 0; round < kRounds; ++round) {
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0;
    const uint32_t mask = round == 0 ? 0u : round == 1 ? 0xffe00000u : 0xfffffc00u, digits = round == 2 ? 1023u : 2047u;
    for (int64_t i = tid; i < mine; i += kSelectThreads) {
      const uint32_t x = key((int)i);
      if (((x ^ prefix) & mask) == 0u) atomicAdd(&sm.counts[round][x >> shift & digits], 1u);
    }
    cluster_sync();
    // two digits a thread, the highest first
    static_assert(kDigits == 2 * kSelectThreads, "two digits a thread");
    const int d = kDigits - 1 - 2 * tid;
    uint2 got[kMostCluster];
#pragma unroll
    for (int r = 0; r < kMostCluster; ++r) got[r] = r < ctas ? remote_u64(&sm.counts[round][d - 1], r) : make_uint2(0u, 0u);
    uint32_t high = 0, low = 0;
#pragma unroll
    for (int r = 0; r < kMostCluster; ++r) { low += got[r].x; high += got[r].y; }
    uint32_t before = high + low;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += y;
    }
    if (lane == 31) sm.warp_sum[warp] = before;
    before -= high + low;
    __syncthreads();
    before += __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_sum[lane] : 0u);
    if (before < left && left <= before + high + low) {
      const bool second = left > before + high;
      sm.digit = d - second;
      sm.left = left - before - (second ? high : 0u);
    }
    __syncthreads();
    prefix |= sm.digit << shift;
    left = sm.left;
  }
  // ---- what each warp's range, then each CTA's, has above the number and equal to it
  const int per = (share + kSelectWarps - 1) / kSelectWarps * 32, w0 = (int)min((int64_t)mine, (int64_t)warp * per), w1 = min(mine - w0, per) + w0;
  uint32_t above = 0, equal = 0;
  for (int i = w0 + lane; i < w1; i += 32) {
    const uint32_t x = key(i);
    above += x > prefix;
    equal += x == prefix;
  }
  above = __reduce_add_sync(0xffffffffu, above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) {
    sm.above[warp] = above;
    sm.equal[warp] = equal;
  }
  __syncthreads();
  if (warp == 0) {
    const uint32_t x = sm.above[lane], y = sm.equal[lane];
    uint32_t sx = x, sy = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t ux = __shfl_up_sync(0xffffffffu, sx, o), uy = __shfl_up_sync(0xffffffffu, sy, o);
      if (lane >= o) { sx += ux; sy += uy; }
    }
    sm.above[lane] = sx - x;
    sm.equal[lane] = sy - y;
    if (lane == 31) { sm.cta_above = sx; sm.cta_equal = sy; }
  }
  cluster_sync();
  uint32_t at_above = sm.above[warp], at_equal = sm.equal[warp];
  for (int r = 0; r < rank; ++r) {
    at_above += remote_u32(&sm.cta_above, r);
    at_equal += remote_u32(&sm.cta_equal, r);
  }
  // ---- the list, in order
  const uint32_t below = (1u << lane) - 1u;
  for (int i0 = w0; i0 < w1; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t x = i < w1 ? key(i) : 0u;
    const bool is_above = i < w1 && x > prefix, is_equal = i < w1 && x == prefix;
    const uint32_t ba = __ballot_sync(0xffffffffu, is_above), be = __ballot_sync(0xffffffffu, is_equal);
    const uint32_t ea = at_above + __popc(ba & below), ee = at_equal + __popc(be & below);
    if (is_above || (is_equal && ee < left)) {
      const uint32_t at = k.first + ea + min(ee, left);
      if (at < (uint32_t)a.most) out[at] = first + i;
    }
    at_above += __popc(ba);
    at_equal += __popc(be);
  }
  cluster_sync();                // (no CTA leaves while another reads its counts)
}

// HBM-bound.
template <int kRowBytes, int kScaleBlocks>
__global__ void __launch_bounds__(kMoveThreads) cache_move_kernel(const EvictArgs a) {
  constexpr int kLanes = kRowBytes / 16, kMoveRows = move_rows(kRowBytes);
  const int g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  __shared__ int64_t from[kMoveRows], to[kMoveRows];       // page << 32 | token in it; -1: none
  dependency_wait();
  dependents_release();
  const int count = a.count[b];
  if (blockIdx.x == 0 && g == 0 && tid == 0) a.lengths[b] = count;
  const int64_t t0 = (int64_t)blockIdx.x * kMoveRows;
  if (t0 >= count) return;
  const CacheView &c = a.c, &n = a.to;
  if (tid < kMoveRows) {
    int64_t x = -1, y = -1;
    if (t0 + tid < count) {
      const int t = (int)t0 + tid;
      const int32_t* kept = a.kept + ((int64_t)b * c.Hkv + g) * a.most;
      const int pos = kept[t];
      const bool inside = pos >= 0 && pos < c.max_keys;
      if (dbg_in_range(inside && t < a.most && (t == 0 || kept[t - 1] < pos), a.status) && inside) {
        const int p = cache_page(c, b, pos), q = cache_page(n, b, t);
        if (p >= 0 && q >= 0) {
          x = (int64_t)p << 32 | (pos & ((1 << c.page_shift) - 1));
          y = (int64_t)q << 32 | (t & ((1 << n.page_shift) - 1));
        }
      }
    }
    from[tid] = x;
    to[tid] = y;
  }
  __syncthreads();
  constexpr int kSteps = kMoveRows * kLanes / kMoveThreads, kRowSteps = (2 * kMoveRows + kMoveThreads - 1) / kMoveThreads;
  constexpr int kBytes = 1 + kScaleBlocks;                 // of a row's scales
  uint4 k[kSteps], v[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int x = i * kMoveThreads + tid, row = x / kLanes, piece = x % kLanes;
    k[i] = v[i] = make_uint4(0, 0, 0, 0);
    if (from[row] < 0) continue;
    const int64_t at = (from[row] >> 32) * c.page_bytes + (((int64_t)g << c.page_shift) + (int)from[row]) * kRowBytes + piece * 16;
    k[i] = *reinterpret_cast<const uint4*>(c.K + at);
    v[i] = *reinterpret_cast<const uint4*>(c.V + at);
  }
  // scales and weights: two threads a row, one for K and the weight, one for V
  uint32_t exponent[kRowSteps];
  uint2 blocks[kRowSteps];
  float weight[kRowSteps];
#pragma unroll
  for (int i = 0; i < kRowSteps; ++i) {
    const int x = i * kMoveThreads + tid, row = x >> 1, value = x & 1;
    exponent[i] = 0u;
    blocks[i] = make_uint2(0u, 0u);
    weight[i] = 0.f;
    if (row >= kMoveRows || from[row] < 0) continue;
    const int64_t p = from[row] >> 32;
    const int in_page = (int)from[row];
    if (!value) weight[i] = a.w[p * a.w_page + ((int64_t)g << c.page_shift) + in_page];
    if (kScaleBlocks < 0) continue;
    const uint8_t* src = (value ? c.vs : c.ks) + p * c.scale_stride + (((int64_t)g * kBytes) << c.page_shift);
    exponent[i] = src[in_page];
    src += (1 << c.page_shift) + in_page * kScaleBlocks;
    if (kScaleBlocks == 8) blocks[i] = *reinterpret_cast<const uint2*>(src);
    if (kScaleBlocks == 4) blocks[i].x = *reinterpret_cast<const uint32_t*>(src);
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int x = i * kMoveThreads + tid, row = x / kLanes, piece = x % kLanes;
    if (from[row] < 0) continue;
    const int64_t at = (to[row] >> 32) * n.page_bytes + (((int64_t)g << n.page_shift) + (int)to[row]) * kRowBytes + piece * 16;
    *reinterpret_cast<uint4*>(n.K + at) = k[i];
    *reinterpret_cast<uint4*>(n.V + at) = v[i];
  }
#pragma unroll
  for (int i = 0; i < kRowSteps; ++i) {
    const int x = i * kMoveThreads + tid, row = x >> 1, value = x & 1;
    if (row >= kMoveRows || from[row] < 0) continue;
    const int64_t q = to[row] >> 32;
    const int in_page = (int)to[row];
    if (!value) a.w_to[q * a.w_to_page + ((int64_t)g << n.page_shift) + in_page] = weight[i];
    if (kScaleBlocks < 0) continue;
    uint8_t* dst = (value ? n.vs : n.ks) + q * n.scale_stride + (((int64_t)g * kBytes) << n.page_shift);
    dst[in_page] = (uint8_t)exponent[i];
    dst += (1 << n.page_shift) + in_page * kScaleBlocks;
    if (kScaleBlocks == 8) *reinterpret_cast<uint2*>(dst) = blocks[i];
    if (kScaleBlocks == 4) *reinterpret_cast<uint32_t*>(dst) = blocks[i].x;
  }
}

template <bool kKeep>
cudaError_t launch_select(const EvictArgs& a, int ctas, size_t smem, cudaStream_t s) {
  static PerDeviceOnce once;
  cudaError_t e = once.run([] {
    return cudaFuncSetAttribute(cache_select_kernel<kKeep>, cudaFuncAttributeMaxDynamicSharedMemorySize, kKeep ? kKeepKeys * 4 : 0);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = ctas;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas, a.c.Hkv, a.c.B);
  cfg.blockDim = dim3(kSelectThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, cache_select_kernel<kKeep>, a);
}

template <int kRowBytes, int kScaleBlocks>
cudaError_t launch_move(const EvictArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.most + move_rows(kRowBytes) - 1) / move_rows(kRowBytes)), a.c.Hkv, a.c.B);
  return launch_dependent(cache_move_kernel<kRowBytes, kScaleBlocks>, grid, kMoveThreads, 0, s, true, a);
}
cudaError_t launch_move_kind(const EvictArgs& a, cudaStream_t s) {
  const bool wide = a.c.D == 128;
  if (a.c.kind == L2A_CACHE_BF16) return wide ? launch_move<256, -1>(a, s) : launch_move<128, -1>(a, s);
  if (a.c.kind == L2A_CACHE_E4M3) return wide ? launch_move<128, 0>(a, s) : launch_move<64, 0>(a, s);
  return wide ? launch_move<64, 8>(a, s) : launch_move<32, 4>(a, s);
}

size_t count_bytes(int B) { return align_up((size_t)B * 4, 256); }
size_t evict_ws_bytes(const l2a_params* p) { return kWsHeaderBytes + count_bytes(p->B) + align_up((size_t)p->B * p->Hkv * p->Lq * 4, 256); }

l2a_status check_evict(const l2a_params* p, const l2a_cache* c, CacheView* v) {
  const int32_t none = 0;
  const l2a_status st = cache_view(p, c, &none, 0, v);
  if (st != L2A_OK) return st;
  return p->B > 65535 || p->Hkv > 65535 ? L2A_ERR_UNSUPPORTED : L2A_OK;
}

}  // namespace
}  // namespace l2a

using namespace l2a;

extern "C" l2a_status l2a_cache_evict_workspace_bytes(const l2a_params* p, const l2a_cache* c, size_t* ws_bytes) {
  CacheView v;
  const l2a_status st = check_evict(p, c, &v);
  if (st != L2A_OK) return st;
  if (!ws_bytes) return L2A_ERR_INVALID_ARG;
  *ws_bytes = evict_ws_bytes(p);
  return L2A_OK;
}

extern "C" l2a_status l2a_cache_evict(const l2a_params* p, const l2a_cache* c, const float* weights, int64_t weight_stride,
                                      const int32_t* keep, int sinks, int recent, const l2a_cache* to, float* to_weights,
                                      int64_t to_weight_stride, int32_t* to_lengths, int32_t* kept, void* ws, size_t ws_bytes,
                                      void* stream) {
  EvictArgs a;
  l2a_status st = check_evict(p, c, &a.c);
  if (st != L2A_OK) return st;
  l2a_params room = *p;                    // what the other table has room for
  room.Lk = p->Lq;
  st = check_evict(&room, to, &a.to);
  if (st != L2A_OK) return st;
  if (to->kind != c->kind || (to->K == c->K && to->page_table == c->page_table)) return L2A_ERR_INVALID_ARG;
  if (!weights || !keep || !to_weights || !to_lengths || sinks < 0 || recent < 0) return L2A_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(weights) | reinterpret_cast<uintptr_t>(to_weights)) & 3) return L2A_ERR_INVALID_ARG;
  const int64_t dense = (int64_t)p->Hkv * c->page_size, to_dense = (int64_t)p->Hkv * to->page_size;
  a.w_page = weight_stride ? weight_stride : dense;
  a.w_to_page = to_weight_stride ? to_weight_stride : to_dense;
  if (a.w_page < dense || a.w_to_page < to_dense) return L2A_ERR_INVALID_ARG;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) % 256) != 0 || ws_bytes < evict_ws_bytes(p)) return L2A_ERR_WORKSPACE;
  a.w = weights;
  a.w_to = to_weights;
  a.keep = keep;
  a.sinks = sinks;
  a.recent = recent;
  a.most = p->Lq;
  a.status = static_cast<int*>(ws);
  uint8_t* at = static_cast<uint8_t*>(ws) + kWsHeaderBytes;
  a.count = reinterpret_cast<int32_t*>(at);
  a.kept = kept ? kept : reinterpret_cast<int32_t*>(at + count_bytes(p->B));
  a.lengths = to_lengths;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int ctas = 1;
  while (ctas < kMostCluster && p->Lk > (int64_t)ctas * kShareKeys) ctas *= 2;
  const int64_t share = (((int64_t)p->Lk + 31) / 32 + ctas - 1) / ctas * 32;
  cudaError_t e = share <= kKeepKeys ? launch_select<true>(a, ctas, (size_t)share * 4, s) : launch_select<false>(a, ctas, 0, s);
  if (e == cudaSuccess) e = launch_move_kind(a, s);
  return e == cudaSuccess ? L2A_OK : L2A_ERR_CUDA;
}
