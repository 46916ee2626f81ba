// What the kernels of the paged key/value cache share: the cache as the device sees it, positions of the new tokens, the
// conversion of 8-bit rows.
#pragma once
#include "l2a_common.cuh"
#include "sm100_prims.cuh"

namespace l2a {

struct CacheView {
  uint8_t *K, *V;              // pools, as bytes
  uint8_t *ks, *vs;            // E4M3, E2M1: of a page and head the exponents + 127, [page]; E2M1: behind them block scales, [page][D / 16]
  int64_t page_bytes, scale_stride;
  int kind, n_pages, page_shift, table_stride;
  int max_keys;                // positions that the table and p->Lk allow
  const int32_t *table, *lengths;
  const int32_t* cu_new;       // NULL: every sequence has Lq new tokens
  int B, Lq, Hkv, D, n_tokens;
};

// Bytes of a row of codes or values, and of the scales of a row
__host__ __device__ constexpr int row_bytes(int kind, int D) { return kind == L2A_CACHE_BF16 ? 2 * D : kind == L2A_CACHE_E4M3 ? D : D / 2; }
__host__ __device__ constexpr int scale_bytes(int kind, int D) { return kind == L2A_CACHE_BF16 ? 0 : kind == L2A_CACHE_E4M3 ? 1 : 1 + D / 16; }
// Offsets, inside a page's scales, of the exponent of a token of a head and of the scales of its blocks (E2M1)
template <int D, int kKind>
__device__ __forceinline__ int64_t exponent_at(const CacheView& c, int head, int in_page) {
  return (((int64_t)head * scale_bytes(kKind, D)) << c.page_shift) + in_page;
}
template <int D>
__device__ __forceinline__ int64_t blocks_at(const CacheView& c, int head, int in_page) {
  return ((((int64_t)head * scale_bytes(L2A_CACHE_E2M1, D)) + 1) << c.page_shift) + in_page * (D / 16);
}

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

// A call of the attention over the cache, or of the weights of its keys.
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
  // the weights of the keys (l2a_cache_weigh); global is set, local and add are not
  int every;                   // every row counts, whatever d
  float* weights;              // pool [pages, Hkv, page], w_page elements a page
  int64_t w_page;
  float* scores;               // few rows: of a sequence's KV head score_rows rows of score_pitch keys
  int score_rows;
  int64_t score_pitch;
};

// Sequences whose new tokens have at most few_rows rows (tokens x heads of a KV group), one block of rows or kRowBlocks of them:
// cache_few.cu
constexpr int kBlockRows = 16, kRowBlocks = 4;
size_t cache_few_ws_bytes(const l2a_params* p, int kind);     // plan and parts
bool cache_few_counts(const l2a_params* p, int kind, bool weigh);         // whether it can count the tiles of one sequence
cudaError_t launch_cache_few(const CacheFwdArgs& a, void* ws, cudaStream_t s);

// The weights of the keys from those sequences, up to `rows` rows of each
size_t cache_few_weigh_ws_bytes(const l2a_params* p, int rows);
cudaError_t launch_cache_few_weigh(const CacheFwdArgs& a, void* ws, cudaStream_t s);

// All others: cache_chunk.cu
size_t cache_chunk_ws_bytes(const l2a_params* p, int n_tokens);          // plan and parts,
size_t cache_copy_bytes(const l2a_params* p, int kind);                  // behind them the decoded copy, 0: none is made
bool cache_chunk_counts(const l2a_params* p, int n_tokens);      // whether it can count the key blocks of such a call
// first: no kernel of the call ahead; copy: the workspace has room for the decoded copy
cudaError_t launch_cache_chunk(const CacheFwdArgs& a, bool first, void* ws, bool copy, cudaStream_t s);

// Adds sum[i] to the weights of keys key .. key + 3 of a sequence's KV head, key a multiple of four; those of its new tokens (from `fresh` on)
// had none.  Keys behind hi that are not new keep what they have.  The memory adds: a page may be in the tables of several sequences, whose CTAs
// know nothing of each other.  (A key's sums of one sequence come from one thread, in order.  Weights of four chunks of 400 on 16K: 101.5 us a call
// with loads and stores here, 99.3 with this.)
__device__ __forceinline__ void add_weights(const CacheFwdArgs& a, const CacheView& c, int b, int g, int key, int length, int fresh, int hi,
                                            const float (&sum)[4]) {
  const int last = min(length - 1, key + 3);
  if (key > last || (key > hi && last < fresh)) return;
  const int page = cache_page(c, b, key);              // (a page holds a multiple of four tokens)
  if (page < 0) return;
  if (!dbg_in_range(key >= 0 && key % 4 == 0 && last < c.max_keys && g < c.Hkv && b < c.B, a.status)) return;
  float* w = a.weights + page * a.w_page + ((int64_t)g << c.page_shift) + (key & ((1 << c.page_shift) - 1));
  if (last == key + 3 && key + 3 < fresh && (reinterpret_cast<uintptr_t>(w) & 15) == 0) {
    asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(w), "f"(sum[0]), "f"(sum[1]), "f"(sum[2]), "f"(sum[3]) : "memory");
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (key + i > last) break;
    if (key + i >= fresh) w[i] = sum[i];
    else if (key + i <= hi) atomicAdd(w + i, sum[i]);
  }
}

// Tensor map over a pool: {elements of 128 bytes at most, tokens, (pieces of a row,) heads, pages}; one copy brings box_rows
// tokens of one head of one page, box_pieces * 64 elements of each (bf16) or the whole row of codes (swizzled over the row's bytes).
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
// e2m1 codes, two a byte, the even element in the low half.  Those of a word as fp16, exactly
__device__ __forceinline__ void e2m1x8_to_f16(uint32_t codes, uint32_t (&h)[4]) {
  asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
      " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
}
// Eight values as e2m1, to nearest even, at most 6
__device__ __forceinline__ uint32_t pack_e2m1(const float2 (&x)[4]) {
  uint32_t r;
  asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}"
      : "=r"(r) : "f"(x[0].x), "f"(x[0].y), "f"(x[1].x), "f"(x[1].y), "f"(x[2].x), "f"(x[2].y), "f"(x[3].x), "f"(x[3].y));
  return r;
}
// The two e4m3 bytes of a half as fp16; an e4m3 byte's value
__device__ __forceinline__ uint32_t e4m3x2_to_f16(uint32_t bytes) {
  uint32_t r;
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(r) : "r"(bytes));
  return r;
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) { return f16x2_to_float2(e4m3x2_to_f16(byte)).x; }
// Copies from one page: K or V rows of a head; untiled for their exponents (16 bytes or a multiple, 16-byte aligned)
__device__ __forceinline__ void tma_load_page(void* dst, const CUtensorMap* map, uint64_t* bar, bool codes, int piece, int row,
                                              int head, int page) {
  if (codes) {
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
// 16 bytes by this thread's own asynchronous copy, and the arrival of the thread (one that the barrier counts) once all of its copies are there
__device__ __forceinline__ void copy_16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void arrive_after_copies(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
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
// 16 e2m1 codes times the scale of their block, 2^e in it, as bf16 (the same)
__device__ __forceinline__ void decode_16(const uint2& codes, float scale, uint32_t (&o)[8]) {
  const uint32_t w[2] = {codes.x, codes.y};
  const float2 both = make_float2(scale, scale);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t h[4];
    e2m1x8_to_f16(w[k], h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = __fmul2_rn(f16x2_to_float2(h[i]), both);
      o[4 * k + i] = pack_bf16(x.x, x.y);
    }
  }
}

}  // namespace l2a
