// Attention of the new tokens over the paged cache (l2a_cache_forward): o = s + d * a for every row, both parts from one pass.
#include <math.h>

#include "cache_common.cuh"
#include "sm100_prims.cuh"

namespace l2a {

namespace {

constexpr int kWarps = 4;

// One CTA = one query row of one head; a warp takes every fourth key, a lane D / 32 elements.
template <int D>
__global__ void __launch_bounds__(kWarps * 32) cache_forward_kernel(const CacheFwdArgs a) {
  constexpr int kE = D / 32;
  const CacheView& c = a.c;
  const int t = blockIdx.x, h = blockIdx.y, g = h / a.G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (a.G > kFewRows && t == 0 && h == 0 && threadIdx.x == 0) *a.status = 0;
  int b = 0, first, n = 0;
  if (c.cu_new == nullptr) b = t / c.Lq;
  else while (b + 1 < c.B && c.cu_new[b + 1] <= t) ++b;
  n = cache_new(c, b, first);
  if (n * a.G <= kFewRows) return;
  const int i = t - first;
  const int pos = i >= 0 && i < n ? cache_length(c, b) - n + i : -1;
  const bool routed = a.global && a.d != nullptr && a.d[t] != 0;
  if (a.add && !routed) return;
  float q[kE];
#pragma unroll
  for (int k = 0; k < kE; ++k) q[k] = __bfloat162float(a.q[t * a.q_t + h * D + lane * kE + k]) * a.scale_log2;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, acc[2][kE] = {};
  for (int j = (routed ? 0 : max(0, pos - a.window)) + warp; j <= pos; j += kWarps) {
    const int page = cache_page(c, b, j);
    const int64_t slot = ((int64_t)g << c.page_shift) + (j & ((1 << c.page_shift) - 1));
    float k[kE], v[kE];
    for (int x = 0; x < kE; ++x) {
      const int64_t at = slot * D + lane * kE + x;
      if (page < 0) {
        k[x] = v[x] = 0.f;
      } else if (c.kind == L2A_CACHE_E4M3) {
        k[x] = f16x2_to_float2(e4m3x2_to_f16x2(c.K[page * c.page_bytes + at])).x * scale_of_exponent(c.ks[page * c.scale_stride + slot]);
        v[x] = f16x2_to_float2(e4m3x2_to_f16x2(c.V[page * c.page_bytes + at])).x * scale_of_exponent(c.vs[page * c.scale_stride + slot]);
      } else {
        k[x] = __bfloat162float(reinterpret_cast<const bf16*>(c.K + page * c.page_bytes)[at]);
        v[x] = __bfloat162float(reinterpret_cast<const bf16*>(c.V + page * c.page_bytes)[at]);
      }
    }
    float s = 0.f;
#pragma unroll
    for (int x = 0; x < kE; ++x) s = fmaf(q[x], k[x], s);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
#pragma unroll
    for (int w = 0; w < 2; ++w) {            // 0: the window, 1: all keys
      if (w == 0 && j < pos - a.window) continue;
      const float m_new = fmaxf(m[w], s), alpha = exp2f(m[w] - m_new), p = exp2f(s - m_new);
      m[w] = m_new;
      l[w] = l[w] * alpha + p;
#pragma unroll
      for (int x = 0; x < kE; ++x) acc[w][x] = acc[w][x] * alpha + p * v[x];
    }
  }
  __shared__ float sm[2][kWarps], sl[2][kWarps], sa[2][kWarps][D];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    if (lane == 0) { sm[w][warp] = m[w]; sl[w][warp] = l[w]; }
#pragma unroll
    for (int x = 0; x < kE; ++x) sa[w][warp][lane * kE + x] = acc[w][x];
  }
  __syncthreads();
  for (int x = threadIdx.x; x < D; x += kWarps * 32) {
    float o = 0.f;
    bf16* dst = a.O + t * a.o_t + h * D + x;
    if (a.add) o = __bfloat162float(*dst);
    for (int w = 0; w < 2; ++w) {
      if (!(w == 0 ? a.local : routed)) continue;
      float M = -INFINITY, L = 0.f, A = 0.f;
      for (int k = 0; k < kWarps; ++k) M = fmaxf(M, sm[w][k]);
      for (int k = 0; k < kWarps; ++k) {
        const float f = sm[w][k] == -INFINITY ? 0.f : exp2f(sm[w][k] - M);
        L += f * sl[w][k];
        A += f * sa[w][k][x];
      }
      if (L > 0.f) o += A / L;
    }
    *dst = __float2bfloat16(o);
  }
}

int64_t row_stride(const int64_t (&s)[2], int row_elems) {
  if (s[0] != 0 || s[1] < 0) return 0;
  const int64_t t = s[1] ? s[1] : row_elems;
  return t >= row_elems && t % 8 == 0 ? t : 0;
}

l2a_status check_forward(const l2a_params* p, const l2a_cache* c, int n_tokens, CacheView* v) {
  const int32_t some = 0;
  const l2a_status st = cache_view(p, c, &some, n_tokens, v);
  if (st != L2A_OK) return st;
  const uint32_t known = L2A_FLAG_SKIP_LOCAL | L2A_FLAG_SKIP_GLOBAL | L2A_FLAG_GLOBAL_PHASE | L2A_FLAG_SHARED_WINDOW;
  const uint32_t modes = p->flags & known & ~L2A_FLAG_SHARED_WINDOW;
  return (p->flags & ~known) || (modes & (modes - 1)) ? L2A_ERR_INVALID_ARG : L2A_OK;
}

}  // namespace
}  // namespace l2a

using namespace l2a;

extern "C" l2a_status l2a_cache_workspace_bytes(const l2a_params* p, const l2a_cache* c, int n_tokens, size_t* ws_bytes) {
  CacheView v;
  const l2a_status st = check_forward(p, c, n_tokens, &v);
  if (st != L2A_OK) return st;
  if (!ws_bytes) return L2A_ERR_INVALID_ARG;
  *ws_bytes = kWsHeaderBytes + cache_few_ws_bytes(p);
  return L2A_OK;
}

extern "C" l2a_status l2a_cache_forward(const l2a_params* p, const l2a_cache* c, const void* Q, const int32_t* cu_new, int n_tokens,
                                        const uint8_t* d, void* O, void* ws, size_t ws_bytes, void* stream) {
  CacheFwdArgs a;
  l2a_status st = check_forward(p, c, n_tokens, &a.c);
  if (st == L2A_OK) st = cache_view(p, c, cu_new, n_tokens, &a.c);
  if (st != L2A_OK) return st;
  a.q_t = row_stride(p->q_stride, p->Hq * p->D);
  a.o_t = row_stride(p->o_stride, p->Hq * p->D);
  if (a.q_t == 0 || a.o_t == 0) return L2A_ERR_INVALID_ARG;
  size_t need = 0;
  st = l2a_cache_workspace_bytes(p, c, n_tokens, &need);
  if (st != L2A_OK) return st;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) % 256) != 0 || ws_bytes < need) return L2A_ERR_WORKSPACE;
  if (n_tokens == 0) return L2A_OK;
  if (!Q || !O || ((reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(O)) & 15)) return L2A_ERR_INVALID_ARG;
  a.Hq = p->Hq; a.G = p->Hq / p->Hkv;
  a.window = p->window < p->Lk ? p->window : p->Lk;       // (no key is further away)
  a.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)p->D)) * 1.4426950408889634f;
  a.add = (p->flags & L2A_FLAG_GLOBAL_PHASE) != 0;
  a.local = !a.add && !(p->flags & L2A_FLAG_SKIP_LOCAL);
  a.global = !(p->flags & L2A_FLAG_SKIP_GLOBAL);
  a.shift = a.local ? a.window + 1 : 0;
  a.q = static_cast<const bf16*>(Q);
  a.d = d;
  a.O = static_cast<bf16*>(O);
  a.status = static_cast<int*>(ws);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.G <= kFewRows) {
    const cudaError_t e = launch_cache_few(a, static_cast<uint8_t*>(ws) + kWsHeaderBytes, s);
    if (e != cudaSuccess) return L2A_ERR_CUDA;
    if ((int64_t)p->Lq * a.G <= kFewRows) return L2A_OK;
  }
  const dim3 grid(n_tokens, p->Hq);
  if (p->D == 128) cache_forward_kernel<128><<<grid, kWarps * 32, 0, s>>>(a);
  else cache_forward_kernel<64><<<grid, kWarps * 32, 0, s>>>(a);
  return cudaGetLastError() == cudaSuccess ? L2A_OK : L2A_ERR_CUDA;
}
