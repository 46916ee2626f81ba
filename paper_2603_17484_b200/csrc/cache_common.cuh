// What the kernels of the paged key/value cache share: the cache as the device sees it, positions of the new tokens, the
// conversion of 8-bit rows.
#pragma once
#include "l2a_common.cuh"
#include "sm100_prims.cuh"

namespace l2a {

struct CacheView {
  uint8_t *K, *V;              // pools, as bytes
  uint8_t *ks, *vs;            // exponents + 127 (E4M3)
  int64_t page_bytes, scale_stride;
  int kind, n_pages, page_shift, table_stride;
  int max_keys;                // positions that the table and p->Lk allow
  const int32_t *table, *lengths;
  const int32_t* cu_new;       // NULL: every sequence has Lq new tokens
  int B, Lq, Hkv, D, n_tokens;
};

// Host side: checks a cache call's parameters and fills the view.
l2a_status cache_view(const l2a_params* p, const l2a_cache* c, const int32_t* cu_new, int n_tokens, CacheView* v);

__device__ __forceinline__ int cache_length(const CacheView& c, int b) { return min(max(c.lengths[b], 0), c.max_keys); }

// New tokens of sequence b: first row of the token axis and their number (0 where cu_new breaks its bounds)
__device__ __forceinline__ int cache_new(const CacheView& c, int b, int& first) {
  if (c.cu_new == nullptr) {
    first = b * c.Lq;
    return c.Lq;
  }
  first = c.cu_new[b];
  const int n = c.cu_new[b + 1] - first;
  return first >= 0 && n > 0 && n <= c.Lq && first <= c.n_tokens - n ? n : 0;
}

// Page of a position of sequence b, -1: none.  Without a table (a copy in the workspace) the pages of a sequence follow each other.
__device__ __forceinline__ int cache_page(const CacheView& c, int b, int pos) {
  if (c.table == nullptr) return b * c.table_stride + (pos >> c.page_shift);
  const int page = c.table[(int64_t)b * c.table_stride + (pos >> c.page_shift)];
  return page >= 0 && page < c.n_pages ? page : -1;
}

// A forward call over the cache.
struct CacheFwdArgs {
  CacheView c;
  int Hq, G, window;
  float scale_log2;
  int local, global, add;      // which modules run; add: O holds s already
  int shift;                   // a routed row at position p sees the keys 0 .. p - shift besides what Local Attention sees:
                               // window + 1 where that runs, else 0
  const bf16* q;               // [n_tokens, Hq, D], token strides q_t, o_t
  int64_t q_t, o_t;
  const uint8_t* d;            // routing decisions, NULL: none
  bf16* O;
  int* status;                 // workspace: status word,
  int* plan;                   // few rows: tiles of a CTA, first tile of every sequence;
  float* part;                 // rows of the parts
  int few_rows;                // most rows of a sequence there, and
  int row_blocks;              // blocks of rows that it can have
  int clear;                   // few rows: no launch ahead has cleared the status word
};

// Sequences whose new tokens have at most few_rows rows (tokens x heads of a KV group), one block of rows or kRowBlocks of them:
// cache_few.cu
constexpr int kBlockRows = 16, kRowBlocks = 4;
size_t cache_few_ws_bytes(const l2a_params* p);     // plan and parts
bool cache_few_counts(const l2a_params* p);         // whether it can count the tiles of one sequence
cudaError_t launch_cache_few(const CacheFwdArgs& a, void* ws, cudaStream_t s);

// All others: cache_chunk.cu
size_t cache_chunk_ws_bytes(const l2a_params* p, int n_tokens);          // plan and parts,
size_t cache_copy_bytes(const l2a_params* p, int kind);                  // behind them the decoded copy, 0: none is made
bool cache_chunk_counts(const l2a_params* p, int n_tokens);      // whether it can count the key blocks of such a call
// first: no kernel of the call ahead; copy: the workspace has room for the decoded copy
cudaError_t launch_cache_chunk(const CacheFwdArgs& a, bool first, void* ws, bool copy, cudaStream_t s);

// Tensor map over a pool: {elements of 128 bytes at most, tokens, (pieces of a row,) heads, pages}; one copy brings box_rows
// tokens of one head of one page, box_pieces * 64 elements of each (bf16) or the whole row of codes.
bool encode_pool_map(CUtensorMap* map, const CacheView& c, const void* pool, int box_rows, int box_pieces);

// The four e4m3 codes of a word as fp16, exactly
__device__ __forceinline__ void e4m3x4_to_f16(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}"
      : "=r"(lo), "=r"(hi) : "r"(codes));
}
__device__ __forceinline__ float2 f16x2_to_float2(uint32_t v) {
  float2 f;
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}" : "=f"(f.x), "=f"(f.y) : "r"(v));
  return f;
}
// Two values as e4m3, to nearest even
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Copies from one page: K or V rows of a head; untiled for their exponents (16 bytes or a multiple, 16-byte aligned)
__device__ __forceinline__ void tma_load_page(void* dst, const CUtensorMap* map, uint64_t* bar, bool e4m3, int piece, int row,
                                              int head, int page) {
  if (e4m3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(0), "r"(row), "r"(head), "r"(page) : "memory");
  } else {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(0), "r"(row), "r"(piece), "r"(head), "r"(page) : "memory");
  }
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// 32 bytes of a lane: one access where the address allows it, so that a warp's access covers whole sectors
__device__ __forceinline__ void load_32(const void* p, bool wide, uint32_t (&x)[8]) {
  if (wide) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]) : "l"(p));
  } else {
    const uint4 a = static_cast<const uint4*>(p)[0], b = static_cast<const uint4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}
__device__ __forceinline__ void store_32(void* p, bool wide, const uint32_t (&x)[8]) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]) : "memory");
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(x[0], x[1], x[2], x[3]);
    static_cast<uint4*>(p)[1] = make_uint4(x[4], x[5], x[6], x[7]);
  }
}
// 2^e of a stored exponent (0 and 255, which no row is written with, stand for 0 and infinity)
__device__ __forceinline__ float scale_of_exponent(uint32_t biased) { return __uint_as_float(biased << 23); }

// 16 codes times 2^e as bf16 (exact but for overflow and underflow)
__device__ __forceinline__ void decode_16(const uint4& codes, float scale, uint32_t (&o)[8]) {
  const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t l, h;
    e4m3x4_to_f16(w[k], l, h);
    const float2 both = make_float2(scale, scale), lo = __fmul2_rn(f16x2_to_float2(l), both), hi = __fmul2_rn(f16x2_to_float2(h), both);
    o[2 * k] = pack_bf16(lo.x, lo.y);
    o[2 * k + 1] = pack_bf16(hi.x, hi.y);
  }
}

}  // namespace l2a
