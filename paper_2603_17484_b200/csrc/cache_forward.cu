// Attention of the new tokens over the paged cache (l2a_cache_forward): o = s + d * a for every row, both parts from one pass.
#include <math.h>

#include <algorithm>

#include "cache_common.cuh"
#include "sm100_prims.cuh"

namespace l2a {

namespace {

// Workspace: header, then the part of the few rows, then that of the others
bool has_few(const l2a_params* p) { return p->Hq / p->Hkv <= kRowBlocks * kBlockRows; }
bool has_chunks(const l2a_params* p) { return (int64_t)p->Lq * (p->Hq / p->Hkv) > kBlockRows; }
// Most rows of a sequence that the kernel of the few rows takes: those of one block, or of kRowBlocks where reading the keys once for each
// block costs less than the launches of the other path (125 MB, less what that path reads itself).  Blocks by the average sequence, keys
// by the longest.  us with one block / four (window 4096, a fifth routed; 28/4 heads): 5 tokens of one sequence of 32K e4m3 51 / 37, of
// four 65 / 71, of eight 99 / 148, of eight ragged ones (18 tokens in all) 81 / 56, 9 tokens of one of 9000 42 / 23; (32/8) 8 tokens of eight
// of 8000 e4m3 81 / 73, bf16 66 / 87; 16 of one of 100K e4m3 101 / 192.
int few_rows(const l2a_params* p, const l2a_cache* c, int n_tokens) {
  const int G = p->Hq / p->Hkv;
  const double blocks = std::max<double>(p->B, (double)n_tokens * G / kBlockRows);
  const double pass = (double)p->Lk * p->Hkv * p->D * (c->kind == L2A_CACHE_E4M3 ? 2 : 4);
  return (blocks - 1.15 * p->B) * pass < 125e6 ? kRowBlocks * kBlockRows : kBlockRows;
}

// Without the decoded copy of an 8-bit cache, which a smaller workspace does without
size_t least_ws_bytes(const l2a_params* p, int n_tokens) {
  return kWsHeaderBytes + (has_few(p) ? cache_few_ws_bytes(p) : 0) + (has_chunks(p) ? cache_chunk_ws_bytes(p, n_tokens) : 0);
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
  if ((p->flags & ~known) || (modes & (modes - 1))) return L2A_ERR_INVALID_ARG;
  if ((int64_t)n_tokens * p->Hq >= (1ll << 31) - 32) return L2A_ERR_UNSUPPORTED;      // (rows are counted in 32 bits)
  return (!has_few(p) || cache_few_counts(p)) && (!has_chunks(p) || cache_chunk_counts(p, n_tokens)) ? L2A_OK : L2A_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace l2a

using namespace l2a;

extern "C" l2a_status l2a_cache_workspace_bytes(const l2a_params* p, const l2a_cache* c, int n_tokens, size_t* ws_bytes) {
  CacheView v;
  const l2a_status st = check_forward(p, c, n_tokens, &v);
  if (st != L2A_OK) return st;
  if (!ws_bytes) return L2A_ERR_INVALID_ARG;
  *ws_bytes = least_ws_bytes(p, n_tokens) + cache_copy_bytes(p, c->kind);
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
  const size_t need = least_ws_bytes(p, n_tokens), copy = cache_copy_bytes(p, c->kind);
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
  uint8_t* at = static_cast<uint8_t*>(ws) + kWsHeaderBytes;
  cudaError_t e = cudaSuccess;
  bool first = true;
  a.few_rows = few_rows(p, c, n_tokens);
  const bool few = p->Hq / p->Hkv <= a.few_rows, chunks = (int64_t)p->Lq * a.G > a.few_rows;
  if (has_few(p)) {
    // With as many tokens as there can be no sequence is expected to have few rows: no launch for those.  The list may say otherwise (the
    // device alone reads it, and the token axis may be longer than what it lists), so the path of the chunks then takes every sequence.
    first = !few || ((int64_t)p->B * p->Lq == n_tokens && chunks);
    if (!first) e = launch_cache_few(a, at, s);
    else if (few) a.few_rows = 0;
    at += cache_few_ws_bytes(p);
  }
  if (e == cudaSuccess && chunks) e = launch_cache_chunk(a, first, at, copy > 0 && ws_bytes >= need + copy, s);
  return e == cudaSuccess ? L2A_OK : L2A_ERR_CUDA;
}
