// Attention over the paged cache for sequences with few query rows: the new tokens of a sequence times the heads of a KV group
// are at most few_rows (decode, a few drafted tokens).  Rows are taken in blocks of 16, each with its own pass over the keys that some row
// of the sequence sees: HBM-bound with one block, the passes of further blocks find their keys in L2.
//
// Keys come in tiles of 64 from position 0 on.  For every sequence and KV head there are up to two segments of tiles: those
// of Local Attention (from the first row's window on; all rows) and, where a token is routed, those before its window.
// Every key block a routed row sees thus enters one set of partial soft-max results, and s and a are weighted sums of
// the sets.  All segments of the call, laid end to end, are cut into equal ranges of tiles, one to a CTA (two CTAs
// an SM), whatever the lengths of the sequences: a range is a few pieces of segments, a piece leaves its rows
// (acc, max, sum) in a slot of the workspace, and cache_few_combine_kernel joins the slots of a row.  A sequence that is one
// piece stores its result itself.
//
//   producer warp : the tiles through a ring of shared-memory stages, one TMA copy a page, and the exponents of 8-bit rows
//                   by untiled copies.  Page numbers come 32 at a time, one a lane.
//   compute warps : 16 keys of every tile each.  Rows are the 16 rows of mma.sync A fragments.
//                   bf16: S = Q K^T from ldmatrix'd rows, P rounded to bf16 and the part that is cut off (in rows 8 .. 15 where those
//                   are free, else in a product of their own) times V from transposed ldmatrix.
//                   e4m3: codes become fp16, exactly, one conversion for two of them (mma.sync of e4m3 operands is made of the same
//                   conversions here, those of Q among them).  A lane loads 16 codes of a key at once and takes them as its elements
//                   of successive products: the order of the head's elements does not matter as long as Q has the same.  V: two
//                   keys' codes of a column are put side by side by byte permutes.  The keys' scales multiply the
//                   scores in fp32, the values' scales go into the weights: w = 2^(s + e - M) with a running maximum M of s + e,
//                   beside the sum of 2^(s - m) with its own.  fp16 has 11 bits against bf16's 8, but less range: Q is scaled by a
//                   power of two for each row, w lies at 2^10 .. 2^14 where it counts and is dropped at 2^-38 of that.
//
// Measured (captured calls back to back, milliseconds long): 16 sequences of 128K keys (32/8 heads, D = 128, four routed) e4m3 196 to 202 us for
// 1.18 GB = 5.9 to 6.0 TB/s, bf16 346 us for 2.35 GB = 6.8 TB/s; 32 ragged ones of up to 8000, a quarter routed, bf16 69 us (394 MB: 5.7 TB/s).
// The 8-bit passes take 355 instructions a warp for 16 keys of a head, 176 of them on the integer pipe (48 % of its rate, 44 % of the issue
// slots; 445 with mma.sync of e4m3 operands), and slow down with the clock in a long loop (218 us at 1.83 of 1.965 GHz; 230 to 236 in others).
// A lone short sequence is latency (9001 keys: 13.3 us, of which this kernel 9.2; the dense l2a_decode, which knows its lengths on the host,
// takes 7.6 in 16 bits): lists, lengths and decisions are read by every CTA ahead of its first copy.  Tried: two chains of products 206 us
// against 196; the loads of V ahead of the soft-max, no change; pieces and rows of Q handed over by the producer, 14.2 against 13.0 for 9001 keys.
#include <math.h>

#include <algorithm>

#include "cache_common.cuh"

namespace l2a {

namespace {

constexpr int kTile = 64;
constexpr int kComputeWarps = kTile / 16;
constexpr int kThreads = (kComputeWarps + 1) * 32;
constexpr int kMaxStages = 6;
constexpr int kMinTiles = 4;                 // tiles of a CTA at least (9001 keys, 28/4 heads: 12.6 us; with 2 14.1, 3 13.1, 6 13.8)
constexpr int kCtas = 2 * kSplitSms;
constexpr float kWeightTop = 10.f;           // log2 of the largest weight when the reference is new (fp16 operands)
constexpr float kLag = 4.f;                  // the reference follows the maximum when it is more than this behind

struct FewBars {
  uint64_t full[kMaxStages], empty[kMaxStages];
  int abort_flag;
  int warp_sum[kThreads / 32], warp_pairs[kThreads / 32];
  int found_b, found_base;   // sequence of the CTA's first tile, and that sequence's first
  int found[9];              // ... and what it takes part with (FewSeq)
};

// What a sequence takes part with: its new tokens and the tiles of its two segments
struct FewSeq {
  int first, n;            // rows of the token axis; n = 0: none here
  int length;
  int lo, n_loc;           // first key and tiles of Local Attention
  int hi, n_out;           // last key (-1: none) and tiles before the windows
  int blocks;              // of 16 rows
  __device__ int tiles() const { return n_loc + n_out; }       // of a KV head and block of rows
};
static_assert(sizeof(FewSeq) <= sizeof(FewBars::found), "kept in shared memory");
__device__ __forceinline__ FewSeq few_seq(const CacheFwdArgs& a, int b) {
  FewSeq s;
  s.n = cache_new(a.c, b, s.first);
  if ((int64_t)s.n * a.G > a.few_rows) s.n = 0;
  s.blocks = (s.n * a.G + kBlockRows - 1) / kBlockRows;
  s.length = cache_length(a.c, b);
  s.lo = max(0, s.length - s.n - a.window);
  s.n_loc = a.local && s.n > 0 && s.length > 0 ? (s.length - 1) / kTile - s.lo / kTile + 1 : 0;
  s.hi = -1;
  if (a.global && a.d != nullptr)
    for (int i = 0; i < s.n; ++i)
      if (a.d[s.first + i] != 0) s.hi = s.length - s.n + i - a.shift;
  s.hi = max(s.hi, -1);
  s.n_out = s.hi / kTile + (s.hi >= 0 ? 1 : 0);
  return s;
}

__device__ __forceinline__ void ldsm_x4(uint32_t saddr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(saddr));
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t saddr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(saddr));
}
// C += A B, A 16 x 16 (row), B 16 x 8 (col), fp32 accumulators
template <bool kHalf>
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&x)[4], uint32_t b0, uint32_t b1) {
  if (kHalf)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t lds32(uint32_t saddr) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(saddr));
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t saddr) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(saddr));
  return v;
}

template <int D, bool kE4M3>
struct FewSmem {
  static constexpr int kTileBytes = kTile * D * (kE4M3 ? 1 : 2);
  static constexpr int kStageBytes = 2 * kTileBytes;                       // K, then V
  static constexpr int kScaleBytes = kE4M3 ? 2 * kTile : 0;                // exponents of K, then of V
  static __host__ __device__ constexpr int red_bytes(int rows) { return kComputeWarps * rows * (D + 4) * 4; }
  static __host__ __device__ constexpr int total(int stages, int rows) {
    return stages * (kStageBytes + kScaleBytes) + red_bytes(rows) + (int)sizeof(FewBars);
  }
};

// A piece: part of one segment
struct Piece {
  int b, g, block, seg;    // KV head, block of rows; seg 0: Local Attention, 1: before the windows
  int t0, t1;              // tiles [t0, t1)
  int lo, hi;              // keys of the segment
  bool alone;              // the sequence's head has no other piece
};

// Tiles of a CTA, for `total` tiles of `pairs` blocks of rows and KV heads: an even share, but at least kMinTiles of them or all of a pair
// (a part more costs the combination about what a tile does), and where it covers several pairs of the average length, whole ones, whose
// results need no combination.
__device__ __forceinline__ int tiles_per_cta(int total, int pairs) {
  const int share = max(1, (total + kCtas - 1) / kCtas), pair = max(1, total / max(pairs, 1));
  return share >= pair ? (share + pair - 1) / pair * pair : max(share, min(kMinTiles, pair));
}

// The pieces of a CTA's range of tiles, in order: every warp walks through them by itself.
struct Walk {
  int at, end;             // tiles of the call, laid end to end
  int b, base;             // sequence and its first tile
  FewSeq s;
};
__device__ __forceinline__ bool next_piece(const CacheFwdArgs& a, Walk& w, Piece& p) {
  if (w.at >= w.end) return false;
  while (w.at >= w.base + w.s.tiles() * w.s.blocks * a.c.Hkv) {
    w.base += w.s.tiles() * w.s.blocks * a.c.Hkv;
    if (++w.b >= a.c.B) return false;
    w.s = few_seq(a, w.b);
  }
  const int per = w.s.tiles(), in = w.at - w.base, x = in % per;
  p.b = w.b;
  p.g = in / per / w.s.blocks;
  p.block = in / per % w.s.blocks;
  p.seg = x >= w.s.n_loc;
  const int skip = p.seg ? w.s.n_loc : 0, n = p.seg ? w.s.n_out : w.s.n_loc, first = p.seg ? 0 : w.s.lo / kTile;
  const int i0 = x - skip, i1 = min(n, i0 + w.end - w.at);
  p.t0 = first + i0;
  p.t1 = first + i1;
  p.lo = p.seg ? 0 : w.s.lo;
  p.hi = p.seg ? w.s.hi : w.s.length - 1;
  p.alone = i1 - i0 == per;
  w.at += i1 - i0;
  return true;
}

// kHigh: more than eight rows.
template <int D, bool kE4M3, bool kHigh>
__global__ void __launch_bounds__(kThreads, 2)
cache_few_kernel(const CacheFwdArgs a, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                 const int stages) {
  using SM = FewSmem<D, kE4M3>;
  constexpr int kRows = kHigh ? 16 : 8, kHalves = kHigh ? 2 : 1;
  constexpr int kCols = D / 8;                   // e4m3: columns of V of a lane's group, and column tiles
  const CacheView& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  dependents_release();
  if (a.clear && blockIdx.x == 0 && tid == 0) *a.status = 0;

  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* scales = smem + stages * SM::kStageBytes;
  float* red = reinterpret_cast<float*>(scales + stages * SM::kScaleBytes);
  FewBars* bar = reinterpret_cast<FewBars*>(reinterpret_cast<uint8_t*>(red) + SM::red_bytes(kRows));
  volatile int* abort_flag = &bar->abort_flag;

  if (tid == kThreads - 1) {
    tma_prefetch_desc(&mapK);
    tma_prefetch_desc(&mapV);
    for (int s = 0; s < stages; ++s) {
      mbar_init(&bar->full[s], 1);
      mbar_init(&bar->empty[s], kComputeWarps);
    }
    bar->abort_flag = (smem_u32(smem) & 1023u) != 0 ? 2 : 0;       // the swizzled tiles need a 1024-byte aligned base
    fence_mbar_init();
  }
  // ---- the plan: tiles of every sequence, a CTA's range of them.  The first CTA leaves it for the combination.
  const int mine = blockIdx.x;
  int total = 0, per_cta = 0, all_pairs = 0;
  FewSeq own = {};                               // the thread's sequence, of the last kThreads ones
  for (int pass = 0; pass < 2; ++pass) {         // sum, then search
    int base = 0;
    if (pass == 1) per_cta = tiles_per_cta(total, all_pairs);
    for (int b0 = 0; b0 < c.B; b0 += kThreads) {
      const int b = b0 + tid;
      if (b < c.B && (pass == 0 || c.B > kThreads)) own = few_seq(a, b);
      const int pairs = b < c.B && own.tiles() > 0 ? own.blocks * c.Hkv : 0, n = own.tiles() * pairs;
      int x = n;
      if (pass == 0) {
        const int warp_pairs = __reduce_add_sync(0xffffffffu, pairs);
        if (lane == 0) bar->warp_pairs[warp] = warp_pairs;
      }
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (lane == 31) bar->warp_sum[warp] = x;
      __syncthreads();
      int all = 0;
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) x += bar->warp_sum[w];
        all += bar->warp_sum[w];
        if (pass == 0) all_pairs += bar->warp_pairs[w];
      }
      x += base;
      if (pass == 1 && b < c.B) {
        if (mine == 0) {
          // for the combination: tiles before the sequence, and the sequence
          reinterpret_cast<int4*>(a.plan)[2 + 2 * b] = make_int4(x - n, own.first, own.n, own.n_loc);
          a.plan[8 + 8 * b + 4] = own.n_out;
        }
        const int at = mine * per_cta;
        if (at >= x - n && at < x) {
          bar->found_b = b;
          bar->found_base = x - n;
          *reinterpret_cast<FewSeq*>(bar->found) = own;
        }
      }
      base += all;
      __syncthreads();
    }
    total = base;
  }
  if (mine == 0 && tid == 0) a.plan[0] = per_cta;
  Walk walk;
  walk.at = mine * per_cta;
  if (walk.at >= total) return;
  walk.end = min(total, walk.at + per_cta);
  walk.b = bar->found_b;
  walk.base = bar->found_base;
  walk.s = *reinterpret_cast<const FewSeq*>(bar->found);

  bool ok = *abort_flag == 0;
  const int rows_shift = min(c.page_shift, 6), rows = 1 << rows_shift, copies = kTile >> rows_shift;   // of a page, pages of a tile

  if (warp == kComputeWarps) {
    // ================================================================= producer
    // lane -> what it copies of a tile: page `u` of K, V, their exponents
    const int what = lane / copies, u = lane % copies;
    const uint32_t bytes = what < 2 ? rows * D * (kE4M3 ? 1 : 2) : what < (kE4M3 ? 4 : 2) ? rows : 0;
    int s = 0, ph = 1;
    Piece p;
    while (ok && next_piece(a, walk, p)) {
      const int last_entry = p.hi >> c.page_shift, first_entry = p.lo >> c.page_shift;
      int entry0 = -64, page_ids = -1;
      for (int t = p.t0; t < p.t1; ++t) {
        const int key = t * kTile + u * rows, entry = key >> c.page_shift;
        const int last_of_tile = (t * kTile + kTile - 1) >> c.page_shift;
        if (last_of_tile - entry0 >= 32) {
          entry0 = (t * kTile) >> c.page_shift;
          const int e = entry0 + lane;
          page_ids = e >= first_entry && e <= last_entry ? cache_page(c, p.b, e << c.page_shift) : -1;
        }
        const int page = __shfl_sync(0xffffffffu, page_ids, entry - entry0);
        const bool load = bytes > 0 && page >= 0 && key <= p.hi && key + rows > p.lo;
        const uint32_t expect = __reduce_add_sync(0xffffffffu, load ? bytes : 0u);
        if (!mbar_wait_warp(&bar->empty[s], ph, abort_flag)) { ok = false; break; }
        if (lane == 0) mbar_expect_tx(&bar->full[s], expect);
        __syncwarp();
        if (load) {
          const int in_page = key & ((1 << c.page_shift) - 1);
          if (what < 2) {
            tma_load_page(smem + s * SM::kStageBytes + what * SM::kTileBytes + u * (SM::kTileBytes / copies), what ? &mapV : &mapK,
                          &bar->full[s], kE4M3, 0, in_page, p.g, page);
          } else {
            bulk_load(scales + s * SM::kScaleBytes + (what - 2) * kTile + u * rows,
                      (what == 2 ? c.ks : c.vs) + page * c.scale_stride + ((int64_t)p.g << c.page_shift) + in_page, rows,
                      &bar->full[s]);
          }
        }
        if (++s == stages) { s = 0; ph ^= 1; }
      }
    }
  } else {
    // ================================================================= compute warps
    const int hr = lane >> 2, t4 = lane & 3;           // row of the fragments (and row + 8); pair of elements or keys
    const int r0 = warp * 16;                          // this warp's keys of a tile
    int s = 0, ph = 0;
    Piece p;
    while (next_piece(a, walk, p)) {
      // ---- rows: bounds of the keys that each sees in this segment
      int row_lo[kHalves], row_hi[kHalves];
      bool row_ok[kHalves];
      int token[kHalves], head[kHalves];
      int every_lo = p.lo, every_hi = p.hi;            // keys that every row sees
#pragma unroll
      for (int x = 0; x < kHalves; ++x) {
        const int r = p.block * kBlockRows + hr + 8 * x, i = r / a.G;
        row_ok[x] = i < walk.s.n;
        token[x] = walk.s.first + (row_ok[x] ? i : 0);
        head[x] = p.g * a.G + r % a.G;
        const int pos = walk.s.length - walk.s.n + i;
        row_lo[x] = 0;
        row_hi[x] = -1;
        if (row_ok[x]) {
          if (p.seg == 0) {
            row_lo[x] = pos - a.window;
            row_hi[x] = pos;
          } else if (a.d[token[x]] != 0) {
            row_hi[x] = pos - a.shift;
          }
          every_lo = max(every_lo, row_lo[x]);
          every_hi = min(every_hi, row_hi[x]);
        }
      }
      every_lo = __reduce_max_sync(0xffffffffu, every_lo);
      every_hi = __reduce_min_sync(0xffffffffu, every_hi);

      // ---- A fragments of Q
      uint32_t qa[D / 16][4];
      float row_scale[kHalves];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (x >= kHalves) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) qa[k][1] = qa[k][3] = 0u;
          continue;
        }
        constexpr int kLast = kHalves - 1;
        const int y = x < kLast ? x : kLast;
        const bf16* qrow = a.q + token[y] * a.q_t + (int64_t)head[y] * D;
        if (kE4M3) {
          // a lane's elements: those of the 16-byte pieces of a key's codes that it loads (below)
          constexpr int kPieces = D / 64;
          uint32_t v[kPieces][8];
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < kPieces; ++i) {
            load_32(qrow + (t4 * kPieces + i) * 16, false, v[i]);
#pragma unroll
            for (int k = 0; k < 8; ++k) top = __vmaxu2(top, v[i][k] & 0x7fff7fffu);
          }
          top = max(top & 0xffffu, top >> 16);
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          // largest element to 2^14 .. 2^15: the others keep all their bits down to 2^-28 of it
          const int up = min(max(14 + 127 - (int)(top >> 7), -113), 100);
          const float f = row_ok[y] ? __uint_as_float((uint32_t)(up + 127) << 23) : 0.f;
          row_scale[y] = a.scale_log2 * __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
          for (int i = 0; i < kPieces; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k)
              qa[i * 4 + k / 2][(k & 1) * 2 + x] = pack_f16(__uint_as_float(v[i][k] << 16) * f, __uint_as_float(v[i][k] & 0xffff0000u) * f);
        } else {
          row_scale[y] = a.scale_log2;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t v0 = *reinterpret_cast<const uint32_t*>(qrow + k * 16 + 2 * t4);
            const uint32_t v1 = *reinterpret_cast<const uint32_t*>(qrow + k * 16 + 8 + 2 * t4);
            qa[k][x] = row_ok[y] ? v0 : 0u;
            qa[k][2 + x] = row_ok[y] ? v1 : 0u;
          }
        }
      }

      float m[kHalves], l[kHalves], ref[kHalves];      // maximum and sum of the weights; reference of the accumulators
#pragma unroll
      for (int x = 0; x < kHalves; ++x) { m[x] = ref[x] = -INFINITY; l[x] = 0.f; }
      float acc[D / 8][4];
#pragma unroll
      for (int j = 0; j < D / 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;

      for (int t = p.t0; ok && t < p.t1; ++t) {
        if (!mbar_wait_warp(&bar->full[s], ph, abort_flag)) { ok = false; break; }
        const uint32_t tK = smem_u32(smem + s * SM::kStageBytes), tV = tK + SM::kTileBytes;
        const int key0 = t * kTile + r0;               // first key of this warp's 16
        if (key0 <= p.hi && key0 + 15 >= p.lo) {
          const bool edge = key0 < every_lo || key0 + 15 > every_hi;
          // ---- S = Q K^T for two times eight keys; this lane's are key0 + 2 t4 + {0, 1, 8, 9}
          float sc[2][4] = {};
          uint32_t ev[2] = {};
          if (kE4M3) {
            constexpr int kPieces = D / 64;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int row = r0 + x * 8 + hr;
#pragma unroll
              for (int i = 0; i < kPieces; ++i) {
                const int piece = t4 * kPieces + i;
                const float4 y = lds128(tK + row * D + ((D == 128 ? piece ^ (row & 7) : piece ^ ((row >> 1) & 3)) << 4));
                const uint32_t w[4] = {__float_as_uint(y.x), __float_as_uint(y.y), __float_as_uint(y.z), __float_as_uint(y.w)};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  uint32_t lo, hi;
                  e4m3x4_to_f16(w[k], lo, hi);
                  mma_16816<true>(sc[x], qa[i * 4 + k], lo, hi);
                }
              }
              const uint32_t at = smem_u32(scales) + s * SM::kScaleBytes + r0 + x * 8 + 2 * t4;
              const uint32_t ek = lds16(at);
              ev[x] = lds16(at + kTile);
              const float f0 = scale_of_exponent(ek & 0xffu), f1 = scale_of_exponent(ek >> 8);
              sc[x][0] *= f0; sc[x][1] *= f1; sc[x][2] *= f0; sc[x][3] *= f1;
            }
          } else {
            const int lm = lane >> 3, row = r0 + (lm >> 1) * 8 + (lane & 7);
            const uint32_t base = tK + (row >> rows_shift) * (SM::kTileBytes / copies) + (row & (rows - 1)) * 128;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const int chunk = k * 2 + (lm & 1);
              uint32_t kb[4];
              ldsm_x4(base + (chunk >> 3) * (rows * 128) + (((chunk & 7) ^ (row & 7)) << 4), kb);
              mma_16816<false>(sc[0], qa[k], kb[0], kb[1]);
              mma_16816<false>(sc[1], qa[k], kb[2], kb[3]);
            }
          }
          // e4m3: a lane's share of the codes of one of its four keys' values (key0 + 2 t4 + {0, 1, 8, 9})
          constexpr int kWords = kCols / 4;
          auto value_codes = [&](int y, uint32_t (&w)[kWords]) {
            const int row = r0 + 2 * t4 + (y & 1) + (y >> 1) * 8;
            if (D == 128) {
              const float4 z = lds128(tV + row * 128 + ((hr ^ (row & 7)) << 4));
              w[0] = __float_as_uint(z.x); w[1] = __float_as_uint(z.y);
              w[kWords - 2] = __float_as_uint(z.z); w[kWords - 1] = __float_as_uint(z.w);
            } else {
              const uint32_t at = tV + row * 64 + (((hr >> 1) ^ ((row >> 1) & 3)) << 4) + (hr & 1) * 8;
              w[0] = lds32(at);
              w[1] = lds32(at + 4);
            }
          };
          // ---- weights: u is what they are two to the power of, relative to the reference
          float u[kHalves][4], top[kHalves];
          auto row_max = [](const float (&y)[4]) {
            const float z = fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), q = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, 1));
            return fmaxf(q, __shfl_xor_sync(0xffffffffu, q, 2));
          };
          bool grow = false;
#pragma unroll
          for (int x = 0; x < kHalves; ++x) {
            float v[4] = {sc[0][2 * x] * row_scale[x], sc[0][2 * x + 1] * row_scale[x], sc[1][2 * x] * row_scale[x],
                          sc[1][2 * x + 1] * row_scale[x]};
            if (edge) {
              const int k = key0 + 2 * t4;
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const int j = k + (y & 1) + (y >> 1) * 8;
                if (j < row_lo[x] || j > row_hi[x]) v[y] = -INFINITY;
              }
            }
            if (kE4M3) {
              const float m_new = fmaxf(m[x], row_max(v)), base = m_new == -INFINITY ? 0.f : m_new;
              l[x] = l[x] * fast_exp2(m[x] - base) + ((fast_exp2(v[0] - base) + fast_exp2(v[1] - base)) +
                                                       (fast_exp2(v[2] - base) + fast_exp2(v[3] - base)));
              m[x] = m_new;
            }
#pragma unroll
            for (int y = 0; y < 4; ++y)
              u[x][y] = kE4M3 ? v[y] + (float)((int)(y & 1 ? ev[y >> 1] >> 8 : ev[y >> 1] & 0xffu) - 127) : v[y];
            top[x] = row_max(u[x]);
            grow |= top[x] > ref[x] + kLag;            // (the same for the four lanes of a row)
          }
          uint32_t pa[4], pb[4];                       // A fragments of the weights, and of what their rounding cut off
          if (__any_sync(0xffffffffu, grow)) {
            // Values of zeros have exponent 0 however small all others are: they must not become the reference, which would push the
            // weights of the others out of fp16's range.  They get the least exponent.
            if (kE4M3 && __any_sync(0xffffffffu, __vcmpeq4(ev[0] | ev[1] << 16, 0x7f7f7f7fu) != 0)) {
              uint32_t some = 0;                       // bit y: key y has a value that is not zero
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                uint32_t w[kWords], any = 0;
                value_codes(y, w);
#pragma unroll
                for (int i = 0; i < kWords; ++i) any |= w[i] & 0x7f7f7f7fu;
                some |= any != 0 ? 1u << y : 0u;
              }
#pragma unroll
              for (int o = 4; o < 32; o <<= 1) some |= __shfl_xor_sync(0xffffffffu, some, o);
#pragma unroll
              for (int x = 0; x < kHalves; ++x) {
#pragma unroll
                for (int y = 0; y < 4; ++y) u[x][y] -= some >> y & 1u ? 0.f : 127.f;
                top[x] = row_max(u[x]);
              }
            }
            float alpha[2] = {1.f, 1.f};
#pragma unroll
            for (int x = 0; x < kHalves; ++x) {
              if (top[x] > ref[x] + kLag) {
                alpha[x] = fast_exp2(ref[x] - top[x]);           // 0 the first time
                ref[x] = top[x];
                if (!kE4M3) l[x] *= alpha[x];
              }
            }
            if (!kHigh) alpha[1] = alpha[0];
#pragma unroll
            for (int j = 0; j < D / 8; ++j) { acc[j][0] *= alpha[0]; acc[j][1] *= alpha[0]; acc[j][2] *= alpha[1]; acc[j][3] *= alpha[1]; }
          }
#pragma unroll
          for (int x = 0; x < kHalves; ++x) {
            const float zero = (ref[x] == -INFINITY ? 0.f : ref[x]) - (kE4M3 ? kWeightTop : 0.f);
            float w[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) w[y] = fast_exp2(u[x][y] - zero);
            if (kE4M3) {
              pa[x] = pack_f16(w[0], w[1]);
              pa[2 + x] = pack_f16(w[2], w[3]);
            } else {
              l[x] += (w[0] + w[1]) + (w[2] + w[3]);
              const uint32_t h0 = pack_bf16(w[0], w[1]), h1 = pack_bf16(w[2], w[3]);
              pa[x] = h0;
              pa[2 + x] = h1;
              const uint32_t l0 = pack_bf16(w[0] - __uint_as_float(h0 << 16), w[1] - __uint_as_float(h0 & 0xffff0000u));
              const uint32_t l1 = pack_bf16(w[2] - __uint_as_float(h1 << 16), w[3] - __uint_as_float(h1 & 0xffff0000u));
              pb[x] = l0;
              pb[2 + x] = l1;
            }
          }
          if (!kHigh) {
            pa[1] = kE4M3 ? 0u : pb[0];
            pa[3] = kE4M3 ? 0u : pb[2];
          }
          // ---- O += P V.  Slots outside the segment's keys may hold anything: their values are made zeros.
          const bool clear = key0 < p.lo || key0 + 15 > p.hi;
          bool out[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int j = key0 + 2 * t4 + (y & 1) + (y >> 1) * 8;
            out[y] = j < p.lo || j > p.hi;
          }
          if (kE4M3) {
            uint32_t w[4][kWords];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              value_codes(y, w[y]);
              if (clear && out[y]) {
#pragma unroll
                for (int i = 0; i < kWords; ++i) w[y][i] = 0u;
              }
            }
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
              const uint32_t a0 = __byte_perm(w[0][i], w[1][i], 0x5140), a1 = __byte_perm(w[0][i], w[1][i], 0x7362);
              const uint32_t b0 = __byte_perm(w[2][i], w[3][i], 0x5140), b1 = __byte_perm(w[2][i], w[3][i], 0x7362);
              uint32_t p0, p1, p2, p3, q0, q1, q2, q3;
              e4m3x4_to_f16(a0, p0, p1);
              e4m3x4_to_f16(a1, p2, p3);
              e4m3x4_to_f16(b0, q0, q1);
              e4m3x4_to_f16(b1, q2, q3);
              mma_16816<true>(acc[4 * i], pa, p0, q0);
              mma_16816<true>(acc[4 * i + 1], pa, p1, q1);
              mma_16816<true>(acc[4 * i + 2], pa, p2, q2);
              mma_16816<true>(acc[4 * i + 3], pa, p3, q3);
            }
          } else {
            const int lm = lane >> 3, row = r0 + (lm & 1) * 8 + (lane & 7);
            const uint32_t base = tV + (row >> rows_shift) * (SM::kTileBytes / copies) + (row & (rows - 1)) * 128;
            const uint32_t vm0 = (out[0] ? 0u : 0x0000ffffu) | (out[1] ? 0u : 0xffff0000u);
            const uint32_t vm1 = (out[2] ? 0u : 0x0000ffffu) | (out[3] ? 0u : 0xffff0000u);
#pragma unroll
            for (int jj = 0; jj < D / 16; ++jj) {
              const int chunk = jj * 2 + (lm >> 1);
              uint32_t vb[4];
              ldsm_x4_t(base + (chunk >> 3) * (rows * 128) + (((chunk & 7) ^ (row & 7)) << 4), vb);
              if (clear) { vb[0] &= vm0; vb[1] &= vm1; vb[2] &= vm0; vb[3] &= vm1; }
              mma_16816<false>(acc[2 * jj], pa, vb[0], vb[1]);
              mma_16816<false>(acc[2 * jj + 1], pa, vb[2], vb[3]);
              if (kHigh) {
                mma_16816<false>(acc[2 * jj], pb, vb[0], vb[1]);
                mma_16816<false>(acc[2 * jj + 1], pb, vb[2], vb[3]);
              }
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar->empty[s]);
        if (++s == stages) { s = 0; ph ^= 1; }
      }

      // ---- join the four warps, then store the result or the part
      constexpr int kPitch = D + 4;
      float* mine_red = red + warp * kRows * kPitch;
      named_barrier(1, kComputeWarps * 32);            // the piece before has been read
#pragma unroll
      for (int x = 0; x < kHalves; ++x) {
        float* row = mine_red + (hr + 8 * x) * kPitch;
        float sum = l[x];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (t4 == 0) { row[D] = kE4M3 ? m[x] : ref[x]; row[D + 1] = sum; row[D + 2] = ref[x]; }
#pragma unroll
        for (int j = 0; j < D / 8; ++j) {
          float v0 = acc[j][2 * x], v1 = acc[j][2 * x + 1];
          if (!kHigh && !kE4M3) {
            // (an infinite value stays what it is: the part cut off may have the other sign or be zero)
            if (isfinite(v0)) v0 += acc[j][2];
            if (isfinite(v1)) v1 += acc[j][3];
          }
          if (kE4M3) {                                 // column tile j, columns 2 t4 and 2 t4 + 1 of it
            row[2 * t4 * kCols + j] = v0;
            row[(2 * t4 + 1) * kCols + j] = v1;
          } else {
            row[j * 8 + 2 * t4] = v0;
            row[j * 8 + 2 * t4 + 1] = v1;
          }
        }
      }
      named_barrier(1, kComputeWarps * 32);
      const bool failed = *abort_flag != 0;
      const int row0 = p.block * kBlockRows, n_rows = min(kBlockRows, walk.s.n * a.G - row0);
      for (int i = tid; i < n_rows * (D / 4); i += kComputeWarps * 32) {
        const int r = i / (D / 4), c4 = i % (D / 4);
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < kComputeWarps; ++w) M = fmaxf(M, red[(w * kRows + r) * kPitch + D]);
        const float base = M == -INFINITY ? 0.f : M;
        float L = 0.f;
        float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kComputeWarps; ++w) {
          const float* row = red + (w * kRows + r) * kPitch;
          const float mw = row[D], rw = row[D + 2];
          L += row[D + 1] * exp2f(mw - base);
          if (rw == -INFINITY) continue;
          const float f = exp2f(rw - (kE4M3 ? kWeightTop : 0.f) - base);
          const float4 v = *reinterpret_cast<const float4*>(row + c4 * 4);
          A.x += v.x * f; A.y += v.y * f; A.z += v.z * f; A.w += v.w * f;
        }
        if (!p.alone) {
          float* slot = a.part + (((int64_t)(p.b * c.Hkv + p.g) * a.row_blocks + p.block) * 2 + p.seg + blockIdx.x) * (kRows * kPitch) +
                        r * kPitch;
          *reinterpret_cast<float4*>(slot + c4 * 4) = A;
          // (a sum of NaN comes with a maximum above all others, so that the combination cannot pass it over)
          if (c4 == 0) *reinterpret_cast<float2*>(slot + D) = make_float2(isnan(L) ? INFINITY : M, failed ? -1.f : L);
        } else if (!failed) {
          const int t = walk.s.first + (row0 + r) / a.G;
          const bool routed = a.global && a.d != nullptr && a.d[t] != 0;
          if ((a.add && !routed) || !dbg_in_range(t >= 0 && t < c.n_tokens, a.status)) continue;
          const float k = L != 0.f ? (float)((a.local ? 1 : 0) + (routed ? 1 : 0)) / L : 0.f;
          uint2* dst = reinterpret_cast<uint2*>(a.O + t * a.o_t + (int64_t)(p.g * a.G + (row0 + r) % a.G) * D) + c4;
          float4 old = make_float4(0.f, 0.f, 0.f, 0.f);
          if (a.add) {
            const uint2 x = *dst;
            old = make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
                              __uint_as_float(x.y & 0xffff0000u));
          }
          *dst = make_uint2(pack_bf16(fmaf(k, A.x, old.x), fmaf(k, A.y, old.y)), pack_bf16(fmaf(k, A.z, old.z), fmaf(k, A.w, old.w)));
        }
      }
    }
  }
  __syncthreads();
  if (bar->abort_flag) {
    // a bounded wait ran out: give copies still in flight time to land before shared memory is released
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    if (tid == 0) atomicExch(a.status, bar->abort_flag);
    __syncthreads();
  }
}

// Joins the parts of one head of one new token:
//   o = sum_loc acc_i 2^(m_i - M_loc) / L_loc + d sum_all acc_i 2^(m_i - M_all) / L_all
// Bound by latencies: every thread asks for its share of the first kAhead * 128 / (D / 4) parts before the weights are known.
constexpr int kCombineThreads = 128, kAhead = 12, kMaxParts = kCtas + 2;
template <int D, int kRows>
__global__ void __launch_bounds__(kCombineThreads) cache_few_combine_kernel(const CacheFwdArgs a) {
  constexpr int kLanes = D / 4, kGroups = kCombineThreads / kLanes, kPitch = D + 4;
  __shared__ float weight[kMaxParts];
  __shared__ float4 red[kGroups][kLanes];
  __shared__ float4 stat[kCombineThreads / 32];
  const CacheView& c = a.c;
  const int h = blockIdx.x, b = blockIdx.y, i = blockIdx.z, g = h / a.G;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c4 = tid % kLanes, grp = tid / kLanes;
  dependency_wait();
  dependents_release();
  const int per_cta = a.plan[0];
  const int4 seq = reinterpret_cast<const int4*>(a.plan)[2 + 2 * b];
  FewSeq s;
  s.first = seq.y;
  s.n = seq.z;
  s.n_loc = seq.w;
  s.n_out = a.plan[8 + 8 * b + 4];
  if (i >= s.n) return;
  const int row_of = i * a.G + h % a.G, block = row_of / kBlockRows, blocks = (s.n * a.G + kBlockRows - 1) / kBlockRows;
  const int at = seq.x + (g * blocks + block) * s.tiles();
  const int loc0 = at / per_cta, n_loc = s.n_loc ? (at + s.n_loc - 1) / per_cta - loc0 + 1 : 0;
  const int out0 = (at + s.n_loc) / per_cta, n_out = s.n_out ? (at + s.tiles() - 1) / per_cta - out0 + 1 : 0;
  if (n_loc + n_out == 1) return;                      // stored by its only piece
  const int t = s.first + i;
  const bool routed = a.global && a.d != nullptr && a.d[t] != 0;
  if ((a.add && !routed) || !dbg_in_range(t >= 0 && t < c.n_tokens && n_loc + n_out <= kMaxParts, a.status)) return;
  const int n = n_loc + (routed ? n_out : 0);
  const int64_t seg = ((int64_t)(b * c.Hkv + g) * a.row_blocks + block) * 2;
  const float* row = a.part + row_of % kBlockRows * kPitch;
  auto slot = [&](int k) { return row + (k < n_loc ? seg + loc0 + k : seg + 1 + out0 + k - n_loc) * (kRows * kPitch); };
  float4 v[kAhead];
#pragma unroll
  for (int x = 0; x < kAhead; ++x) {
    const int k = grp + x * kGroups;
    v[x] = k < n ? __ldcg(reinterpret_cast<const float4*>(slot(k)) + c4) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  constexpr int kMine = (kMaxParts + kCombineThreads - 1) / kCombineThreads;
  float2 ml[kMine];
  float m_loc = -INFINITY, m_all = -INFINITY, least = 0.f;
#pragma unroll
  for (int x = 0; x < kMine; ++x) {
    const int k = tid + x * kCombineThreads;
    ml[x] = k < n ? __ldcg(reinterpret_cast<const float2*>(slot(k) + D)) : make_float2(-INFINITY, 0.f);
    m_all = fmaxf(m_all, ml[x].x);
    if (k < n_loc) m_loc = fmaxf(m_loc, ml[x].x);
    least = fminf(least, ml[x].y);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    m_loc = fmaxf(m_loc, __shfl_xor_sync(0xffffffffu, m_loc, o));
    m_all = fmaxf(m_all, __shfl_xor_sync(0xffffffffu, m_all, o));
    least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
  }
  if (lane == 0) stat[warp] = make_float4(m_loc, m_all, least, 0.f);
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kCombineThreads / 32; ++w) {
    m_loc = fmaxf(m_loc, stat[w].x);
    m_all = fmaxf(m_all, stat[w].y);
    least = fminf(least, stat[w].z);
  }
  __syncthreads();
  float l_loc = 0.f, l_all = 0.f;
#pragma unroll
  for (int x = 0; x < kMine; ++x) {
    if (ml[x].x == -INFINITY) continue;                // no key of that part is visible to the row
    l_all += ml[x].y * exp2f(ml[x].x - m_all);
    if (tid + x * kCombineThreads < n_loc) l_loc += ml[x].y * exp2f(ml[x].x - m_loc);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    l_loc += __shfl_xor_sync(0xffffffffu, l_loc, o);
    l_all += __shfl_xor_sync(0xffffffffu, l_all, o);
  }
  if (lane == 0) stat[warp] = make_float4(l_loc, l_all, 0.f, 0.f);
  __syncthreads();
  l_loc = l_all = 0.f;
#pragma unroll
  for (int w = 0; w < kCombineThreads / 32; ++w) { l_loc += stat[w].x; l_all += stat[w].y; }
#pragma unroll
  for (int x = 0; x < kMine; ++x) {
    const int k = tid + x * kCombineThreads;
    if (k >= n) continue;
    float w = 0.f;
    if (ml[x].x != -INFINITY) {
      if (k < n_loc) w = exp2f(ml[x].x - m_loc) / l_loc;
      if (routed) w += exp2f(ml[x].x - m_all) / l_all;
    }
    weight[k] = w;
  }
  __syncthreads();
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](int k, const float4& x) {
    const float w = weight[k];
    o.x = fmaf(w, x.x, o.x);
    o.y = fmaf(w, x.y, o.y);
    o.z = fmaf(w, x.z, o.z);
    o.w = fmaf(w, x.w, o.w);
  };
#pragma unroll
  for (int x = 0; x < kAhead; ++x)
    if (grp + x * kGroups < n) add(grp + x * kGroups, v[x]);
#pragma unroll 4
  for (int k = grp + kAhead * kGroups; k < n; k += kGroups) add(k, __ldcg(reinterpret_cast<const float4*>(slot(k)) + c4));
  red[grp][c4] = o;
  __syncthreads();
  if (grp != 0 || least < 0.f) return;                 // a wait ran out in a part: nothing is stored
#pragma unroll
  for (int x = 1; x < kGroups; ++x) {
    const float4 y = red[x][c4];
    o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
  }
  uint2* dst = reinterpret_cast<uint2*>(a.O + t * a.o_t + (int64_t)h * D) + c4;
  if (a.add) {
    const uint2 x = *dst;
    o.x += __uint_as_float(x.x << 16); o.y += __uint_as_float(x.x & 0xffff0000u);
    o.z += __uint_as_float(x.y << 16); o.w += __uint_as_float(x.y & 0xffff0000u);
  }
  *dst = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
}

constexpr int kSmemPerCta = 113 * 1024;          // two CTAs an SM

template <int D, bool kE4M3, bool kHigh>
cudaError_t launch(const CacheFwdArgs& a, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t s) {
  using SM = FewSmem<D, kE4M3>;
  constexpr int kRows = kHigh ? 16 : 8;
  constexpr int kFit = (kSmemPerCta - SM::total(0, kRows)) / (SM::kStageBytes + SM::kScaleBytes);
  constexpr int kStages = kFit < kMaxStages ? kFit : kMaxStages;
  constexpr int smem = SM::total(kStages, kRows);
  static PerDeviceOnce once;
  cudaError_t e = once.run([] {
    return cudaFuncSetAttribute(cache_few_kernel<D, kE4M3, kHigh>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  });
  if (e != cudaSuccess) return e;
  cache_few_kernel<D, kE4M3, kHigh><<<kCtas, kThreads, smem, s>>>(a, mapK, mapV, kStages);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const dim3 grid(a.Hq, a.c.B, std::max(1, std::min(a.c.Lq, a.few_rows / a.G)));
  return launch_dependent(cache_few_combine_kernel<D, kRows>, grid, kCombineThreads, 0, s, true, a);
}

int slot_rows(const l2a_params* p) { return (int64_t)p->Lq * (p->Hq / p->Hkv) > 8 ? kBlockRows : 8; }
int row_blocks(int64_t rows) { return (int)(std::min<int64_t>(rows, kRowBlocks * kBlockRows) + kBlockRows - 1) / kBlockRows; }
size_t plan_bytes(int B) { return align_up(((size_t)B + 1) * 8 * sizeof(int), 256); }
// Sequences of a launch, 0: not even one.  A launch counts its tiles in 32 bits (up to one more for a segment that begins inside a tile, and
// up to one pair's more a CTA behind the last range), and the combination has a row of its grid for each.
int batch_of(int Lk, int Hkv, int blocks) {
  const int64_t pair = ((int64_t)Lk + kTile - 1) / kTile + 1, one = pair * Hkv * blocks, most = (1ll << 31) - 1 - (kCtas + 1) * (pair + 1);
  return (int)std::max<int64_t>(0, std::min<int64_t>(65535, most / one));
}

}  // namespace

size_t cache_few_ws_bytes(const l2a_params* p) {
  return plan_bytes(p->B) + align_up((2 * (size_t)p->B * p->Hkv * row_blocks((int64_t)p->Lq * (p->Hq / p->Hkv)) + kCtas) * slot_rows(p) * (p->D + 4) * sizeof(float), 256);
}

bool cache_few_counts(const l2a_params* p) { return batch_of(p->Lk, p->Hkv, row_blocks((int64_t)p->Lq * (p->Hq / p->Hkv))) > 0; }

cudaError_t launch_cache_few(const CacheFwdArgs& args, void* ws, cudaStream_t s) {
  CacheFwdArgs a = args;
  const bool high = (int64_t)a.c.Lq * a.G > 8, e4m3 = a.c.kind == L2A_CACHE_E4M3;
  a.plan = static_cast<int*>(ws);
  a.row_blocks = row_blocks((int64_t)a.c.Lq * a.G);
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + plan_bytes(a.c.B));
  CUtensorMap mapK, mapV;
  const int rows = std::min(1 << a.c.page_shift, kTile);
  if (!encode_pool_map(&mapK, a.c, a.c.K, rows, a.c.D / 64) || !encode_pool_map(&mapV, a.c, a.c.V, rows, a.c.D / 64))
    return cudaErrorUnknown;
  const int B = a.c.B, batch = batch_of(a.c.max_keys, a.c.Hkv, row_blocks(std::min<int64_t>((int64_t)a.c.Lq * a.G, a.few_rows)));
  cudaError_t e = batch > 0 ? cudaSuccess : cudaErrorInvalidValue;
  for (int b = 0; e == cudaSuccess && b < B; b += batch) {
    a.clear = b == 0;
    a.c.B = std::min(batch, B - b);
    a.c.table = args.c.table + (int64_t)b * a.c.table_stride;
    a.c.lengths = args.c.lengths + b;
    if (a.c.cu_new != nullptr) {
      a.c.cu_new = args.c.cu_new + b;
    } else {
      const int64_t t = (int64_t)b * a.c.Lq;
      a.c.n_tokens = a.c.B * a.c.Lq;
      a.q = args.q + t * a.q_t;
      a.O = args.O + t * a.o_t;
      if (a.d != nullptr) a.d = args.d + t;
    }
    if (a.c.D == 128) {
      if (e4m3) e = high ? launch<128, true, true>(a, mapK, mapV, s) : launch<128, true, false>(a, mapK, mapV, s);
      else e = high ? launch<128, false, true>(a, mapK, mapV, s) : launch<128, false, false>(a, mapK, mapV, s);
    } else {
      if (e4m3) e = high ? launch<64, true, true>(a, mapK, mapV, s) : launch<64, true, false>(a, mapK, mapV, s);
      else e = high ? launch<64, false, true>(a, mapK, mapV, s) : launch<64, false, false>(a, mapK, mapV, s);
    }
  }
  return e;
}

}  // namespace l2a
