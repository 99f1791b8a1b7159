// What the kernels of espo_attention share: sizes, workspace, arguments, and device helpers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "espo.h"
#include "espo_device.cuh"
#include "espo_host.h"

namespace espo {
namespace {

constexpr int kTile = 64;                 // tokens per tile of a row
constexpr int kPrefixTile = 128;          // tokens per tile of a prefix
constexpr int kPrefixBlocks = 148;        // one per SM
constexpr int kOwnBlocks = 444;           // three per SM: rows of up to eight queries a key/value head
constexpr int kWideBlocks = 296;          // two per SM: rows of more
constexpr int kComputeWarps = 4;
constexpr int kMaxPerKv = 64;             // query heads per key/value head
constexpr int kPrefixQueries = 128;       // queries per prefix item
constexpr int kFoldBits = 15;             // e4m3: folded weights are 2^15 times larger, see above
constexpr int kMinTiles = 2;              // a piece of the rows' line is no shorter than this

// ---------------------------------------------------------------------------------------------- workspace

// Everything the kernels share, by offset from the workspace's start.
struct Work {
  int32_t* n_active;      // [1]
  int32_t* n_segments;    // [1]
  int64_t* own_total;     // [1] own tiles of all active rows
  int64_t* prefix_total;  // [1] tiles x query blocks of all segments
  int32_t *row, *slot, *len, *segment;       // per active row
  int32_t *group, *prefix_len;               // per active row (scratch of the plan)
  int64_t* own_off;                          // [n_rows + 1] tiles before the row
  int32_t *seg_first, *seg_end, *seg_group, *seg_len;
  int64_t* seg_off;                          // [n_rows + 1] tiles before the segment
  float2* prefix_ml;      // [n_rows][heads]  (m, l) of the first part of each query's prefix item
  float* prefix_o;        // [n_rows][heads][dim]
  float2* extra_ml;       // [kPrefixBlocks][kPrefixQueries]  later parts of prefix items
  float* extra_o;         // [kPrefixBlocks][kPrefixQueries][dim]
  float2* whole_ml;       // [n_rows][heads]  own results of rows that have a prefix and are not cut
  float* whole_o;         // [n_rows][heads][dim]
  float2* own_ml;         // [kOwnBlocks][2][per_kv]  parts of own items: continued from / into the neighbour block's piece
  float* own_o;           // [kOwnBlocks][2][per_kv][dim]
};

__host__ __device__ inline int64_t work_layout(Work& w, char* base, int64_t n_rows, int64_t heads, int64_t per_kv,
                                              int64_t dim) {
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    char* p = base + at;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  char* head = take(256);
  w.own_total = reinterpret_cast<int64_t*>(head);
  w.prefix_total = reinterpret_cast<int64_t*>(head + 8);
  w.n_active = reinterpret_cast<int32_t*>(head + 16);
  w.n_segments = reinterpret_cast<int32_t*>(head + 20);
  w.row = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.slot = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.len = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.segment = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.group = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.prefix_len = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.own_off = reinterpret_cast<int64_t*>(take((n_rows + 1) * 8));
  w.seg_first = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.seg_end = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.seg_group = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.seg_len = reinterpret_cast<int32_t*>(take(n_rows * 4));
  w.seg_off = reinterpret_cast<int64_t*>(take((n_rows + 1) * 8));
  w.prefix_ml = reinterpret_cast<float2*>(take(n_rows * heads * 8));
  w.prefix_o = reinterpret_cast<float*>(take(n_rows * heads * dim * 4));
  w.extra_ml = reinterpret_cast<float2*>(take(int64_t(kPrefixBlocks) * kPrefixQueries * 8));
  w.extra_o = reinterpret_cast<float*>(take(int64_t(kPrefixBlocks) * kPrefixQueries * dim * 4));
  w.whole_ml = reinterpret_cast<float2*>(take(n_rows * heads * 8));
  w.whole_o = reinterpret_cast<float*>(take(n_rows * heads * dim * 4));
  w.own_ml = reinterpret_cast<float2*>(take(int64_t(kOwnBlocks) * 2 * per_kv * 8));
  w.own_o = reinterpret_cast<float*>(take(int64_t(kOwnBlocks) * 2 * per_kv * dim * 4));
  return at;
}

struct AttnArgs {
  espo_kv_cache cache;
  espo_sequences seqs;
  Work work;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  int64_t q_stride, out_stride;
  const int32_t* row_ids;
  uint32_t* status_out;
  float to_log2;              // scale * log2(e)
  int32_t n_q_heads, n_rows;
  int32_t per_kv;             // query heads per key/value head
  int32_t own_blocks;         // blocks that share the rows' line
  int32_t rows_per_block;     // rows whose queries share a prefix item
};

__device__ __forceinline__ void wait_for_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// a / b for a >= 0, b > 0; the 64-bit division's hundred instructions only where they are needed.
__host__ __device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  if (static_cast<uint64_t>(a | b) >> 32 == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
  return a / b;
}

// How many tiles of the line a block takes.
__device__ __forceinline__ int64_t piece_length(int64_t line, int blocks, int least) {
  return max(quotient(line + blocks - 1, blocks), static_cast<int64_t>(least));
}

// A segment's part of the prefixes' line: query block after query block, each with every tile of the prefix.  In 64 bits: a
// prefix of 2^29 tokens has 2^22 tiles, and 512 query blocks of it pass 31 bits.
//
// Tiles before the query block of the segment's row `row`.
__host__ __device__ __forceinline__ int64_t tiles_before_row(int row, int rows_per_block, int tiles) {
  return static_cast<int64_t>(row / rows_per_block) * tiles;
}
// The query block and the tile of the prefix that lie `at` tiles into the part.
__host__ __device__ __forceinline__ void block_and_tile(int64_t at, int tiles, int& block, int& tile) {
  block = static_cast<int>(quotient(at, tiles));
  tile = static_cast<int>(at - static_cast<int64_t>(block) * tiles);
}

__device__ __forceinline__ void tma_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          smem_addr(dst)), "l"(map), "r"(x), "r"(y), "r"(smem_addr(bar)) : "memory");
}

// A bounded wait whose outcome is the same for the whole warp.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(kFullMask, mbar_wait_bounded(bar, parity, abort_flag));
}

// The warps that `bar` counts meet: what each wrote before is seen by all after it.  False if one of them does not come; a warp
// that has given up elsewhere raises the flag, so the others never wait for it at length (as they would at a barrier of the
// block).  `parity` is the warp's own, 0 before the first meeting.
__device__ __forceinline__ bool warps_meet(uint64_t* bar, uint32_t& parity, volatile int* abort_flag) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
  // (a meeting that took place counts, however soon the flag was raised after it)
  const bool ok = warp_wait(bar, parity, abort_flag) || __all_sync(kFullMask, mbar_try_wait(bar, parity));
  parity ^= 1;
  return ok;
}

// Last index i in [0, n) with off[i] <= x (off ascending, off[0] <= x): 32 probes a step, one per lane.
__device__ __forceinline__ int warp_find(const int64_t* off, int n, int64_t x) {
  const int lane = threadIdx.x & 31;
  int lo = 0, size = n;
  while (size > 1) {
    const int step = (size + 31) / 32;
    const int at = lo + lane * step;
    const unsigned ok = __ballot_sync(kFullMask, at < lo + size && at < n && __ldcg(off + at) <= x);
    const int hit = 31 - __clz(ok | 1u);
    lo += hit * step;
    size = min(step, n - lo);
  }
  return lo;
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}

}  // namespace
}  // namespace espo
