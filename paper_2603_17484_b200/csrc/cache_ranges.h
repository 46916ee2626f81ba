// How the key blocks of a call over the paged cache are divided among the CTAs of its chunks (cache_chunk.cu): whole numbers only, so that
// the same functions run in the plan's kernel and on the host.  Sums over a call are 64 bits wide where they have to be: a million routed
// tokens on a million keys are 2^29 blocks, and 2^32 of the units below.
#pragma once
#include <stdint.h>

#ifndef __CUDACC__
#define __host__
#define __device__
#endif

namespace l2a {

// Costs, in eighths of a key block of two tiles (2900 clk): a block that one tile takes (1800), a piece besides its blocks
constexpr int kBlockCost = 8, kDualCost = 5, kItemCost = 40;
constexpr int64_t kMostBlocks = 1ll << 38;       // of a call: a CTA's share of them is counted in 32 bits

__host__ __device__ inline int block_cost(bool dual) { return dual ? kDualCost : kBlockCost; }
// One KV head of a group of `blocks` key blocks, all of them
__host__ __device__ inline int64_t head_cost(int blocks, bool dual) {
  return blocks > 0 ? (int64_t)blocks * block_cost(dual) + kItemCost : 0;
}
__host__ __device__ inline int64_t group_cost(int blocks, bool dual, int Hkv) { return head_cost(blocks, dual) * Hkv; }

// a / b of numbers that are not negative, in 32 bits where they are small (the plan is bound by latencies)
__host__ __device__ inline int64_t quotient(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// Cost at which the range of a CTA begins, of `total` divided evenly
__host__ __device__ inline int64_t range_cost(int cta, int ctas, int64_t total) { return quotient(cta * total, ctas); }
// The place of a cost `in` inside its group (0 <= in < group_cost, blocks > 0)
struct RangePlace { int head, block; };
__host__ __device__ inline RangePlace range_place(int64_t in, int blocks, bool dual) {
  const int64_t per = head_cost(blocks, dual), head = quotient(in, per), rest = in - head * per - kItemCost;
  return RangePlace{(int)head, rest > 0 ? (int)((uint32_t)rest / (uint32_t)block_cost(dual)) : 0};
}
// First key block of a place, of a group whose blocks begin at `base`
__host__ __device__ inline int64_t range_first(int64_t base, RangePlace p, int blocks) { return base + (int64_t)p.head * blocks + p.block; }

// Most key blocks of a call from the host's bounds: both segments of every group, over all keys
inline double most_blocks(int64_t groups, int Hkv, int Lk) { return (double)groups * Hkv * (Lk / 128 + 1); }
inline double most_cost(int64_t groups, int Hkv, int Lk) { return (double)groups * Hkv * ((Lk / 128 + 1.0) * kBlockCost + kItemCost); }

}  // namespace l2a
