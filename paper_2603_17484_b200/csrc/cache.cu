// Paged key/value cache: argument checks, the write of new tokens (l2a_cache_append) and the read back (l2a_cache_read).
#include <math.h>

#include "cache_common.cuh"
#include "sm100_prims.cuh"

namespace l2a {

l2a_status cache_view(const l2a_params* p, const l2a_cache* c, const int32_t* cu_new, int n_tokens, CacheView* v) {
  if (!p || !c) return L2A_ERR_INVALID_ARG;
  if (p->B <= 0 || p->Lq <= 0 || p->Lk <= 0 || p->Hq <= 0 || p->Hkv <= 0 || p->D <= 0 || n_tokens < 0) return L2A_ERR_INVALID_ARG;
  if (p->Hq % p->Hkv != 0 || p->window < 0 || p->seq_bounds != nullptr) return L2A_ERR_INVALID_ARG;
  if (!(p->softmax_scale >= 0.f) || isinf(p->softmax_scale)) return L2A_ERR_INVALID_ARG;
  if (p->D != 64 && p->D != 128) return L2A_ERR_UNSUPPORTED;
  if (c->kind != L2A_CACHE_BF16 && c->kind != L2A_CACHE_E4M3) return L2A_ERR_UNSUPPORTED;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return L2A_ERR_UNSUPPORTED;
  if (c->n_pages <= 0 || c->table_stride <= 0 || (int64_t)c->table_stride * c->page_size < p->Lk) return L2A_ERR_INVALID_ARG;
  if (!c->K || !c->V || !c->page_table || !c->lengths) return L2A_ERR_INVALID_ARG;
  const bool e4m3 = c->kind == L2A_CACHE_E4M3;
  const int64_t elem = e4m3 ? 1 : 2, page = (int64_t)p->Hkv * c->page_size * p->D, scales = (int64_t)p->Hkv * c->page_size;
  const int64_t ps = c->page_stride ? c->page_stride : page, ss = c->scale_stride ? c->scale_stride : scales;
  if (ps < page || ps * elem % 16 != 0 || ss < scales || ss % 16 != 0) return L2A_ERR_INVALID_ARG;
  uintptr_t bits = reinterpret_cast<uintptr_t>(c->K) | reinterpret_cast<uintptr_t>(c->V);
  if (e4m3) {
    if (!c->k_scale || !c->v_scale) return L2A_ERR_INVALID_ARG;
    bits |= reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale);
  }
  if (bits & 15) return L2A_ERR_INVALID_ARG;
  if (!cu_new && (int64_t)p->B * p->Lq != n_tokens) return L2A_ERR_INVALID_ARG;
  v->K = static_cast<uint8_t*>(c->K); v->V = static_cast<uint8_t*>(c->V);
  v->ks = c->k_scale; v->vs = c->v_scale;
  v->page_bytes = ps * elem;
  v->scale_stride = ss;
  v->kind = c->kind;
  v->n_pages = c->n_pages;
  v->page_shift = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7;
  v->table_stride = c->table_stride;
  v->max_keys = p->Lk;
  v->table = c->page_table; v->lengths = c->lengths;
  v->cu_new = cu_new;
  v->B = p->B; v->Lq = p->Lq; v->Hkv = p->Hkv; v->D = p->D; v->n_tokens = n_tokens;
  return L2A_OK;
}

bool encode_pool_map(CUtensorMap* map, const CacheView& c, const void* pool, int box_rows, int box_pieces) {
  const cuuint64_t page = 1ull << c.page_shift, D = c.D, pages = c.n_pages, stride = c.page_bytes;
  const cuuint32_t rows = box_rows;
  if (c.kind == L2A_CACHE_E4M3) {
    const cuuint64_t dims[4] = {D, page, (cuuint64_t)c.Hkv, pages}, strides[3] = {D, page * D, stride};
    const cuuint32_t box[4] = {(cuuint32_t)c.D, rows, 1, 1};
    return encode_tiled_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, pool, dims, strides, box,
                            c.D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
  }
  const cuuint64_t dims[5] = {64, page, D / 64, (cuuint64_t)c.Hkv, pages}, strides[4] = {2 * D, 128, 2 * page * D, stride};
  const cuuint32_t box[5] = {64, rows, (cuuint32_t)box_pieces, 1, 1};
  return encode_tiled_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, pool, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

namespace {

constexpr int kRowsThreads = 256;

// Token stride of a tensor on the token axis, 0: not usable
int64_t token_stride(const int64_t (&s)[2], int row_elems) {
  if (s[0] != 0 || s[1] < 0) return 0;
  const int64_t t = s[1] ? s[1] : row_elems;
  return t >= row_elems && t % 8 == 0 ? t : 0;
}

struct AppendArgs {
  CacheView c;
  const bf16 *K, *V;
  int64_t k_t, v_t;
  int wide, wide_pool;     // 32-byte accesses to K and V, to a bf16 pool
};

// Biased exponent of the least 2^e with amax <= 448 * 2^e = 1.75 * 2^(8 + e), from the bits of the bf16 amax
__device__ __forceinline__ uint32_t exponent_for(uint32_t amax) {
  const int e = (int)(amax >> 7) - 8 + ((amax & 0x7fu) > 0x60u ? 1 : 0);
  return amax == 0 ? 127u : (uint32_t)max(e, 1);
}
// The two magnitudes of a bf16 pair, 0 for those that are not finite
__device__ __forceinline__ uint32_t finite_magnitudes(uint32_t x) {
  x &= 0x7fff7fffu;
  return __vcmpltu2(x, 0x7f807f80u) & x;
}
// A CTA takes kTokens tokens, all heads of K and V; a lane holds 16 values of a row, D / 16 lanes a row, a warp 512 / D tokens of a head of K
// or V at a time, so that the CTA reads whole token rows and the exponents of neighbours in a page leave in one sector.
// Where the tokens go takes four dependent loads (list, length, table): looked up once for the CTA, by one warp, while the
// first rows are on their way.  What bounds it then is the instructions of the conversion: 18380 tokens (8 heads, D = 128, e4m3) take
// 24.8 us (113 MB: 4.6 TB/s), with 16-byte loads, products one by one and indices by division 30.6.
constexpr int kAppendAhead = 4;
template <int D, bool kE4M3, int kTokens>
__global__ void __launch_bounds__(kRowsThreads) cache_append_kernel(const AppendArgs a) {
  constexpr int kLanes = D / 16, kRows = 32 / kLanes, kGroups = kTokens / kRows, kWarps = kRowsThreads / 32;
  const CacheView& c = a.c;
  __shared__ int to_page[kTokens], to_slot[kTokens];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % kLanes;
  const int heads = 2 * c.Hkv, t0 = blockIdx.x * kTokens;
  const int groups = min(kGroups, (c.n_tokens - t0 + kRows - 1) / kRows);       // of kRows tokens
  // step s of the CTA: head s % heads, tokens s / heads; this warp's next one, and the one whose rows it has
  int hv = warp, group = 0, done_hv, done_group;
  auto next = [&](int& x, int& y) {
    for (x += kWarps; x >= heads; x -= heads) ++y;
  };
  for (; hv >= heads; hv -= heads) ++group;
  done_hv = hv;
  done_group = group;
  uint32_t w[kAppendAhead][8];
  for (bool first_batch = true; first_batch || group < groups; first_batch = false) {
#pragma unroll
    for (int i = 0; i < kAppendAhead; ++i) {
      if (group < groups) {
        const int64_t t = min(t0 + group * kRows + lane / kLanes, c.n_tokens - 1);
        load_32((hv & 1 ? a.V + t * a.v_t : a.K + t * a.k_t) + (hv >> 1) * D + sub * 16, a.wide, w[i]);
      }
      next(hv, group);
    }
    if (first_batch) {
      if (warp == 0) {
        // the sequence of a token: the last b with cu_new[b] <= t
        const int t = t0 + lane;
        int b = 0, first = 0, page = -1, pos = 0;
        if (c.cu_new == nullptr) {
          b = t / c.Lq;
        } else {
          for (int b0 = 0; b0 < c.B; b0 += 32) {
            const int cu = b0 + lane < c.B ? c.cu_new[b0 + lane] : 0x7fffffff;
            int seen = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) seen += __shfl_sync(0xffffffffu, cu, i) <= t;
            b += seen;
            if (__all_sync(0xffffffffu, seen < 32)) break;
          }
          b = max(b - 1, 0);
        }
        if (lane < kTokens && t < c.n_tokens) {
          const int n = cache_new(c, b, first);
          pos = c.lengths[b] - n + (t - first);
          if (t >= first && t - first < n && pos >= 0 && pos < c.max_keys) page = cache_page(c, b, pos);
        }
        if (lane < kTokens) {
          to_page[lane] = page;
          to_slot[lane] = pos & ((1 << c.page_shift) - 1);
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kAppendAhead; ++i) {
      if (done_group >= groups) break;
      const bool value = done_hv & 1;
      const int row = done_group * kRows + lane / kLanes, page = to_page[row];
      const int64_t slot = ((int64_t)(done_hv >> 1) << c.page_shift) + to_slot[row];
      uint8_t* dst = (value ? c.V : c.K) + page * c.page_bytes + slot * (kE4M3 ? D : 2 * D);
      next(done_hv, done_group);
      if (kE4M3) {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = __vmaxu2(m, w[i][k] & 0x7fff7fffu);
        if (__any_sync(0xffffffffu, (m & 0xffffu) >= 0x7f80u || m >= 0x7f800000u)) {      // values that are not finite do not count
          m = 0;
#pragma unroll
          for (int k = 0; k < 8; ++k) m = __vmaxu2(m, finite_magnitudes(w[i][k]));
        }
        m = max(m & 0xffffu, m >> 16);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const uint32_t e = exponent_for(m);
        const float f = __uint_as_float((254u - e) << 23);         // 2^-e; e + 127 is 1 .. 247
        const float2 inv = make_float2(f, f);
        uint32_t code[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t u = w[i][2 * k], v = w[i][2 * k + 1];
          const float2 x = __fmul2_rn(make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)), inv);
          const float2 y = __fmul2_rn(make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)), inv);
          code[k] = __byte_perm(pack_e4m3(x.x, x.y), pack_e4m3(y.x, y.y), 0x5410);
        }
        if (page >= 0) {
          *reinterpret_cast<uint4*>(dst + sub * 16) = make_uint4(code[0], code[1], code[2], code[3]);
          if (sub == 0) (value ? c.vs : c.ks)[page * c.scale_stride + slot] = (uint8_t)e;
        }
      } else if (page >= 0) {
        store_32(dst + sub * 32, a.wide_pool, w[i]);
      }
    }
  }
}

struct ReadArgs {
  CacheView c;
  const int32_t* first;
  bf16 *K, *V;
  RowStrides k_st, v_st;
  int wide, wide_pool;     // 32-byte accesses to K and V, to a bf16 pool
};

// The same shape for the way back: a lane brings 16 values of a position, a warp 512 / D positions of a head at a time.  HBM-bound: 1.34 GB
// (eight sequences, 127K tokens of 262K rows, 8 heads, D = 128, e4m3) in 196 us = 6.8 TB/s, with 16-byte accesses 251.
template <int D, bool kE4M3, int kSteps>
__global__ void __launch_bounds__(kRowsThreads) cache_read_kernel(const ReadArgs a) {
  constexpr int kLanes = D / 16, kRows = 32 / kLanes, kTokens = kRows * kSteps;
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 31, b = blockIdx.y, sub = lane % kLanes;
  const int64_t item = ((int64_t)blockIdx.x * kRowsThreads + threadIdx.x) >> 5;
  const int heads = 2 * c.Hkv, hv = (int)(item % heads), h = hv >> 1;
  const bool value = hv & 1;
  const int64_t t0 = item / heads * kTokens + lane / kLanes;
  if (item / heads * kTokens >= c.max_keys) return;
  const int start = a.first ? a.first[b] : 0, length = cache_length(c, b);
  uint32_t x[kSteps][8];         // (e4m3: the first four)
  uint32_t e[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int64_t pos = start + t0 + i * kRows;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[i][k] = 0u;
    e[i] = 127;
    if (pos < 0 || pos >= length) continue;
    const int page = cache_page(c, b, (int)pos);
    if (page < 0) continue;
    const int64_t slot = ((int64_t)h << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
    const uint8_t* src = (value ? c.V : c.K) + page * c.page_bytes + slot * (kE4M3 ? D : 2 * D);
    if (kE4M3) {
      const uint4 y = *reinterpret_cast<const uint4*>(src + sub * 16);
      x[i][0] = y.x; x[i][1] = y.y; x[i][2] = y.z; x[i][3] = y.w;
      e[i] = (value ? c.vs : c.ks)[page * c.scale_stride + slot];
    } else {
      load_32(src + sub * 32, a.wide_pool, x[i]);
    }
  }
  const RowStrides st = value ? a.v_st : a.k_st;
  bf16* out = (value ? a.V : a.K) + b * st.b + h * D + sub * 16;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int64_t t = t0 + i * kRows;
    if (t >= c.max_keys) continue;
    if (kE4M3) {
      uint32_t o[8];
      decode_16(make_uint4(x[i][0], x[i][1], x[i][2], x[i][3]), scale_of_exponent(e[i]), o);
      store_32(out + t * st.t, a.wide, o);
    } else {
      store_32(out + t * st.t, a.wide, x[i]);
    }
  }
}

template <int D, bool kE4M3>
cudaError_t launch_append(const AppendArgs& a, cudaStream_t s) {
  // 16 tokens a CTA, or as many as a warp takes at once up to two waves of CTAs of the former an SM (8 heads, D = 128, e4m3: 32 tokens 5.7 /
  // 3.1 us, 2000 6.1 / 4.6, 4000 7.8 / 7.6, 8000 13.9 / 15.7)
  constexpr int kFew = 512 / D;
  if (a.c.n_tokens < 2 * 16 * kSplitSms) cache_append_kernel<D, kE4M3, kFew><<<ceil_div(a.c.n_tokens, kFew), kRowsThreads, 0, s>>>(a);
  else cache_append_kernel<D, kE4M3, 16><<<ceil_div(a.c.n_tokens, 16), kRowsThreads, 0, s>>>(a);
  return cudaGetLastError();
}
template <int D, bool kE4M3>
cudaError_t launch_read(const ReadArgs& a, cudaStream_t s) {
  constexpr int kSteps = 2, kTokens = 512 / D * kSteps;
  const int64_t warps = ((int64_t)a.c.max_keys + kTokens - 1) / kTokens * 2 * a.c.Hkv;
  const dim3 grid((unsigned)((warps * 32 + kRowsThreads - 1) / kRowsThreads), a.c.B);
  cache_read_kernel<D, kE4M3, kSteps><<<grid, kRowsThreads, 0, s>>>(a);
  return cudaGetLastError();
}

// Whether rows of two tensors (of elem bytes, any number of elements of the strides apart) all start at multiples of 32 bytes
bool all_wide(const void* p, const void* q, int64_t elem, int64_t s0, int64_t s1, int64_t s2 = 0, int64_t s3 = 0) {
  return ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & 31) == 0 && ((s0 | s1 | s2 | s3) * elem) % 32 == 0;
}
bool misaligned(const void* p, const void* q) { return (reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & 15; }

}  // namespace
}  // namespace l2a

using namespace l2a;

extern "C" l2a_status l2a_cache_append(const l2a_params* p, const l2a_cache* c, const void* K, const void* V,
                                       const int32_t* cu_new, int n_tokens, void* stream) {
  AppendArgs a;
  const l2a_status st = cache_view(p, c, cu_new, n_tokens, &a.c);
  if (st != L2A_OK) return st;
  if (n_tokens == 0) return L2A_OK;
  a.k_t = token_stride(p->k_stride, p->Hkv * p->D);
  a.v_t = token_stride(p->v_stride, p->Hkv * p->D);
  if (!K || !V || misaligned(K, V) || a.k_t == 0 || a.v_t == 0) return L2A_ERR_INVALID_ARG;
  a.K = static_cast<const bf16*>(K);
  a.V = static_cast<const bf16*>(V);
  a.wide = all_wide(K, V, 2, a.k_t, a.v_t);
  a.wide_pool = all_wide(c->K, c->V, 1, a.c.page_bytes, 0);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool e4m3 = c->kind == L2A_CACHE_E4M3;
  const cudaError_t e = p->D == 128 ? (e4m3 ? launch_append<128, true>(a, s) : launch_append<128, false>(a, s))
                                    : (e4m3 ? launch_append<64, true>(a, s) : launch_append<64, false>(a, s));
  return e == cudaSuccess ? L2A_OK : L2A_ERR_CUDA;
}

extern "C" l2a_status l2a_cache_read(const l2a_params* p, const l2a_cache* c, const int32_t* first, void* K_out, void* V_out,
                                     void* stream) {
  ReadArgs a;
  const int32_t no_tokens = 0;      // (the new tokens play no part)
  const l2a_status st = cache_view(p, c, &no_tokens, 0, &a.c);
  if (st != L2A_OK) return st;
  if (!K_out || !V_out || misaligned(K_out, V_out)) return L2A_ERR_INVALID_ARG;
  if (!strides_ok(p->k_stride, p->Lk, p->Hkv * p->D) || !strides_ok(p->v_stride, p->Lk, p->Hkv * p->D)) return L2A_ERR_INVALID_ARG;
  if (p->B > 65535) return L2A_ERR_UNSUPPORTED;
  a.c.cu_new = nullptr;
  a.first = first;
  a.K = static_cast<bf16*>(K_out);
  a.V = static_cast<bf16*>(V_out);
  a.k_st = resolve_strides(p->k_stride, p->Lk, p->Hkv * p->D);
  a.v_st = resolve_strides(p->v_stride, p->Lk, p->Hkv * p->D);
  a.wide = all_wide(K_out, V_out, 2, a.k_st.b, a.k_st.t, a.v_st.b, a.v_st.t);
  a.wide_pool = all_wide(c->K, c->V, 1, a.c.page_bytes, 0);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool e4m3 = c->kind == L2A_CACHE_E4M3;
  const cudaError_t e = p->D == 128 ? (e4m3 ? launch_read<128, true>(a, s) : launch_read<128, false>(a, s))
                                    : (e4m3 ? launch_read<64, true>(a, s) : launch_read<64, false>(a, s));
  return e == cudaSuccess ? L2A_OK : L2A_ERR_CUDA;
}
