// Attention of one query token per row over a shared prefix and the row's own tokens.
//
// Mathematics.  With t_j = scale log2(e) q.k_j, running maximum m, sum l = sum 2^(t_j - m) and o = sum 2^(t_j - m) v_j, two
// partial results over disjoint tokens join as  m = max(m1, m2),  l = l1 2^(m1-m) + l2 2^(m2-m),  o likewise;  out = o / l.
// An e4m3 cache adds one exponent per vector: the key's multiplies its score, the value's, 2^e_j, is folded into the weight.
// There m runs over t_j + e_j, so that the folded weight 2^(t_j + e_j - m) is at most 1 however far the values' sizes are
// apart, while the plain weight 2^(t_j - m) that l adds up is at most 2^64.  As fp16 the folded weight is taken 2^15 times
// larger (o too, until the end): weights down to 2^-29 of the largest keep all bits, and the rounding step never exceeds
// 2^-39 of it.  Against a bf16 cache the weights are bf16 (off by 2^-8 of each at most), the type of the values in the same
// instruction.  The sum l takes the weights before either rounding.
//
// What bounds it: a row's own tokens are read once for the few query heads of one key/value head (7 heads: 7 multiply-adds a
// byte of bf16), far below the tensor cores' ratio, so those are bound by HBM; a prefix is read once for the query heads of
// all its rows.
//
// Work split.  Up to four kernels on one stream, each set up while the one before it winds down (programmatic dependent
// launch):
//   plan     one block: the active rows in order, their own tiles of 64 tokens and the prefix segments (runs of rows of one
//            group), as running sums.
//   prefix   (batches with groups) tiles of every segment against 128 queries -- as many whole rows as fit -- and one
//            key/value head.  Results stay partial, in 32 bits.
//   own      tiles of every row against its own query heads; writes the output where that is all there is to a row.
//   join     a warp per remaining row and query head joins its partial results.
// In the middle two the tiles of all items, item after item, head after head, form one line that is cut into equal pieces, one
// per resident block: no imbalance from ragged lengths, and a single long row still uses the whole GPU.  An item cut by a
// piece's end leaves its parts in the blocks' scratch; they are joined in line order, so the result does not depend on timing.
//
// Inside a block one warp or two copy tiles into a ring of shared-memory stages with tensor-map copies (128-byte swizzle) and four
// warps compute with m16n8k16 matrix instructions.  With up to 16 queries an item's tile is split over the warps by tokens,
// so that a warp depends on no other until the item ends, and the queries are the eight columns of the instruction rather
// than its 16 rows: 7 queries a key/value head leave one column idle, not nine rows.  With more, the tile is split by queries.
//
// Measured.  512 rows of up to 4096 own tokens, 28 query heads on 4 of 128 dims, e4m3: 152 us for 903 MB, 6.0 TB/s; 12 on 2,
// bf16: 168 us for 1058 MB, 6.3 TB/s.  Short items of small tiles are bound by their ends and by latency instead: 256 rows of up
// to 1000 tokens, 8 heads of 64 dims, pages of 16, e4m3, 51 us for 123 MB (48 with a second copying warp).
#include "espo_attn_common.cuh"
#include "espo_attn_prefix.cuh"

namespace espo {
namespace {

// ---------------------------------------------------------------------------------------------- plan

constexpr int kPlanThreads = 1024;

// Exclusive running sums of v over the block; total receives the sum.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* scratch, int64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t n = __shfl_up_sync(kFullMask, upto, o);
    if (lane >= o) upto += n;
  }
  __syncthreads();
  if (lane == 31) scratch[warp] = upto;
  __syncthreads();
  if (warp == 0) {
    int64_t s = scratch[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t n = __shfl_up_sync(kFullMask, s, o);
      if (lane >= o) s += n;
    }
    scratch[lane] = s;
  }
  __syncthreads();
  total = scratch[31];
  return upto - v + (warp ? scratch[warp - 1] : 0);
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const AttnArgs A) {
  __shared__ int64_t scratch[32];
  let_next_kernel_start();
  const espo_sequences& S = A.seqs;
  const Work& W = A.work;
  const int page = A.cache.page_size;
  const int max_own = S.max_pages * page, max_prefix = S.max_prefix_pages * page;
  uint32_t bad = 0;
  int active_before = 0;
  int64_t tiles_before = 0, total;
  for (int base = 0; base < A.n_rows; base += kPlanThreads) {
    const int r = base + threadIdx.x;
    int slot = -1, len = 0, group = -1, prefix = 0;
    bool on = false;
    if (r < A.n_rows) {
      slot = A.row_ids ? A.row_ids[r] : r;
      if (slot < 0 || slot >= S.capacity) {
        bad |= ESPO_DEV_BAD_SLOT;
      } else {
        // (asked for together: one trip to memory)
        const uint8_t status = S.status ? S.status[slot] : ESPO_ROW_ACTIVE;
        len = S.length[slot];
        group = S.group ? S.group[slot] : -1;
        on = status == ESPO_ROW_ACTIVE;
      }
      if (on) {
        if (len < 0 || len > max_own) bad |= ESPO_DEV_BAD_LENGTHS;
        len = min(max(len, 0), max_own);
        if (group >= S.n_groups) {
          bad |= ESPO_DEV_BAD_PAGE;
          group = -1;
        }
        if (group >= 0) {
          prefix = S.prefix_length[group];
          if (prefix < 0 || prefix > max_prefix) bad |= ESPO_DEV_BAD_LENGTHS;
          prefix = min(max(prefix, 0), max_prefix);
          if (prefix == 0) group = -1;
        }
      }
    }
    // a row without tokens still has one (empty) tile: the visit that writes its output
    const int64_t tiles = on ? max((len + kTile - 1) / kTile, 1) : 0;
    // both sums at once: a row has at most 2^24 tiles, 1024 rows fewer than 2^40
    constexpr int kShift = 40;
    const int64_t before = block_scan(tiles | (on ? 1ll << kShift : 0), scratch, total);
    const int a = active_before + static_cast<int>(before >> kShift);
    const int64_t off = tiles_before + (before & ((1ll << kShift) - 1));
    active_before += static_cast<int>(total >> kShift);
    tiles_before += total & ((1ll << kShift) - 1);
    if (on) {
      W.row[a] = r;
      W.slot[a] = slot;
      W.len[a] = len;
      W.group[a] = group;
      W.prefix_len[a] = prefix;
      W.own_off[a] = off;
      W.segment[a] = -1;
    }
  }
  if (bad && A.status_out) atomicOr(A.status_out, bad);
  const int n = active_before;
  int n_seg = 0;
  int64_t seg_tiles = 0;
  if (S.group) {
    __syncthreads();        // (also makes the arrays above visible to the block)
    for (int base = 0; base < n; base += kPlanThreads) {
      const int a = base + threadIdx.x;
      const int g = a < n ? W.group[a] : -1;
      const bool first = g >= 0 && (a == 0 || W.group[a - 1] != g);
      const bool last = g >= 0 && (a == n - 1 || W.group[a + 1] != g);
      const int idx = n_seg + static_cast<int>(block_scan(first ? 1 : 0, scratch, total)) + (first ? 1 : 0) - 1;
      n_seg += static_cast<int>(total);
      if (g >= 0) W.segment[a] = idx;
      if (first) {
        W.seg_first[idx] = a;
        W.seg_group[idx] = g;
        W.seg_len[idx] = W.prefix_len[a];
      }
      if (last) W.seg_end[idx] = a + 1;
    }
    __syncthreads();
    for (int base = 0; base < n_seg; base += kPlanThreads) {
      const int s = base + threadIdx.x;
      int64_t tiles = 0;
      if (s < n_seg) {
        const int rows = W.seg_end[s] - W.seg_first[s];
        tiles = static_cast<int64_t>((rows + A.rows_per_block - 1) / A.rows_per_block) * ((W.seg_len[s] + kPrefixTile - 1) / kPrefixTile);
      }
      const int64_t off = seg_tiles + block_scan(tiles, scratch, total);
      seg_tiles += total;
      if (s < n_seg) W.seg_off[s] = off;
    }
  }
  if (threadIdx.x == 0) {
    *W.n_active = n;
    *W.n_segments = n_seg;
    *W.own_total = tiles_before;
    *W.prefix_total = seg_tiles;
    W.own_off[n] = tiles_before;
    W.seg_off[n_seg] = seg_tiles;
  }
}

// ---------------------------------------------------------------------------------------------- matrix instructions

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool kHalf>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (kHalf)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four e4m3 codes as two pairs of halves; exact.
__device__ __forceinline__ void e4m3x4_to_f16(uint32_t four, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(four));
}
// An 8 x 8 matrix of 16-bit numbers transposed across the warp (a lane holds two neighbours of row lane/4).
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool kHalf>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t w;
  if constexpr (kHalf) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}

// ---------------------------------------------------------------------------------------------- tiles in shared memory

template <int kDim, bool kE4M3>
struct Tile {
  static constexpr int kRowBytes = kDim * (kE4M3 ? 1 : 2);
  static constexpr int kPartBytes = kRowBytes < 128 ? kRowBytes : 128;      // bytes of a row that lie together
  static constexpr int kParts = kRowBytes / kPartBytes;
  static constexpr int kMatrix = kTile * kRowBytes;                         // one of K, V
  static constexpr int kStage = 2 * kMatrix + (kE4M3 ? 1024 : 0);           // exponents in a kilobyte of their own
  // Stages of a block where two blocks share an SM, and where three do.
  static constexpr int kStagesOfTwo = kStage >= 32768 ? 3 : kStage >= 16384 ? 5 : 8;
  static constexpr int kStagesOfThree = kStage >= 32768 ? 2 : kStage > 16384 ? 3 : kStage == 16384 ? 4 : 6;

  // Address of 16-byte chunk `chunk` of row `row` relative to the matrix (the swizzle of the tensor-map copies).
  static __device__ __forceinline__ uint32_t at(int row, int chunk) {
    if constexpr (kPartBytes == 128) return (chunk >> 3) * (kTile * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
    else return row * 64 + (((chunk & 3) ^ ((row >> 1) & 3)) << 4);
  }
};

// What the copying warp tells the computing warps about a stage.
struct StageInfo {
  uint64_t valid;         // bit per token of the tile
  int32_t item;           // active row
  int32_t head;           // key/value head
  int32_t flags;          // 1: first tile of the item in this piece; 2: last one; 4: no more tiles; 8: the item starts before
                          // this piece; 16: the item goes on after it
  int32_t pad;
};

struct Queue {            // shared memory beside the stages
  uint64_t full[8], empty[8];
  uint64_t meeting;       // of the computing warps
  StageInfo info[8];
  float2 ml[kComputeWarps][16];
  int abort_flag;
};

// ---------------------------------------------------------------------------------------------- rows' own tokens

// One warp's running result, in fragments of the matrix instruction.  Two layouts with one interface: a lane holds kQ queries
// (query(i) within the warp's) with their m and l, and each(f) calls f(i, dim, value) for every number of o it holds.
//
// Rows: queries are the rows of the left operand, 16 a warp; a lane holds rows lane/4 and lane/4 + 8.
template <int kDim, bool kE4M3>
struct RowAcc {
  static constexpr int kQ = 2;
  float o[kDim / 8][4];
  float m[2], l[2];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kDim / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.0f;
  }
  static __device__ __forceinline__ int query(int i) { return ((threadIdx.x & 31) >> 2) + 8 * i; }
  static __device__ __forceinline__ bool writes_ml() { return (threadIdx.x & 3) == 0; }
  // The dims of fragment i's two columns.  e4m3 pairs of dims come out of a transposed 16-bit load, so an even fragment holds
  // even dims and the odd one beside it the odd dims.
  static __device__ __forceinline__ int dim(int i, int col) {
    const int c = threadIdx.x & 3;
    if constexpr (kE4M3) return (i >> 1) * 16 + 4 * c + 2 * col + (i & 1);
    else return i * 8 + 2 * c + col;
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int i = 0; i < kDim / 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) f(j >> 1, dim(i, j & 1), o[i][j]);
  }
  __device__ __forceinline__ void sum_l() {      // a lane summed its own columns' tokens
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(kFullMask, l[r], 1);
      l[r] += __shfl_xor_sync(kFullMask, l[r], 2);
    }
  }
};

// Columns: queries are the columns of the right operand, kTiles times eight a warp; dims are the rows of the product.  A lane
// holds columns 2c and 2c + 1 (c = lane % 4) of each tile, and rows lane/4 and lane/4 + 8 of every 16 dims.
template <int kDim, bool kE4M3, int kTiles>
struct ColAcc {
  static constexpr int kQ = 2 * kTiles;
  float o[kDim / 16][kTiles][4];
  float m[kQ], l[kQ];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kDim / 16; ++i)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) o[i][t][0] = o[i][t][1] = o[i][t][2] = o[i][t][3] = 0.0f;
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      m[q] = -INFINITY;
      l[q] = 0.0f;
    }
  }
  static __device__ __forceinline__ int query(int i) { return (i >> 1) * 8 + 2 * (threadIdx.x & 3) + (i & 1); }
  static __device__ __forceinline__ bool writes_ml() { return (threadIdx.x & 31) < 4; }
  static __device__ __forceinline__ int dim(int i, int half) {
    const int g = (threadIdx.x & 31) >> 2;
    return kE4M3 ? i * 16 + 2 * g + half : i * 16 + g + 8 * half;
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int i = 0; i < kDim / 16; ++i)
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) f(2 * t + (j & 1), dim(i, j >> 1), o[i][t][j]);
  }
  __device__ __forceinline__ void sum_l() {      // a lane summed its own rows' tokens
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      l[q] += __shfl_xor_sync(kFullMask, l[q], 4);
      l[q] += __shfl_xor_sync(kFullMask, l[q], 8);
      l[q] += __shfl_xor_sync(kFullMask, l[q], 16);
    }
  }
};

// Query fragments of 16 queries as the left operand, and the factor that turns a product into a score, per row of the lane.
template <int kDim, bool kE4M3>
struct RowQueries {
  uint32_t a[kDim / 16][4];
  float factor[2];
};

// The power of two 2^e that brings numbers of magnitude up to `top` into [2^14, 2^15), fp16's upper end: -113 for the largest
// finite numbers, and for infinities, which stay what they are; at most 126, so that 2^-e is a normal number too.
__device__ __forceinline__ int fp16_exponent(float top) {
  return min(max(14 + 127 - static_cast<int>(__float_as_uint(top) >> 23), -113), 126);
}

template <int kDim, bool kE4M3>
__device__ __forceinline__ void load_queries(RowQueries<kDim, kE4M3>& Q, const AttnArgs& A, int item, int head, int q0) {
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const __nv_bfloat16* src[2];
  bool on[2];
  const int row = __ldcg(A.work.row + item);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int j = q0 + g + 8 * r;
    on[r] = j < A.per_kv;
    src[r] = A.q + row * A.q_stride + (head * A.per_kv + (on[r] ? j : 0)) * kDim;
    Q.factor[r] = A.to_log2;
  }
  if constexpr (!kE4M3) {
#pragma unroll
    for (int k = 0; k < kDim / 16; ++k)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(src[r] + k * 16);
        Q.a[k][r] = on[r] ? p[c] : 0u;
        Q.a[k][r + 2] = on[r] ? p[c + 4] : 0u;
      }
  } else {
    // Keys come as e4m3 turned into fp16, so queries are fp16 too: scaled by a power of two that brings the row's largest
    // magnitude to [2^14, 2^15); what lies 2^29 below it loses bits of no weight in the sum.  A lane's four dims of each
    // 16 lie together, as the four bytes of a key's word do.
    uint2 w[2][kDim / 16];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float top = 0.0f;
#pragma unroll
      for (int k = 0; k < kDim / 16; ++k) {
        w[r][k] = on[r] ? *reinterpret_cast<const uint2*>(src[r] + k * 16 + 4 * c) : make_uint2(0u, 0u);
        top = fmaxf(top, fmaxf(fmaxf(fabsf(bf16_lo(w[r][k].x)), fabsf(bf16_hi(w[r][k].x))),
                               fmaxf(fabsf(bf16_lo(w[r][k].y)), fabsf(bf16_hi(w[r][k].y)))));
      }
      top = fmaxf(top, __shfl_xor_sync(kFullMask, top, 1));
      top = fmaxf(top, __shfl_xor_sync(kFullMask, top, 2));
      const int e = fp16_exponent(top);
      const float up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
      Q.factor[r] *= __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
      for (int k = 0; k < kDim / 16; ++k) {
        Q.a[k][r] = pack2<true>(bf16_lo(w[r][k].x) * up, bf16_hi(w[r][k].x) * up);
        Q.a[k][r + 2] = pack2<true>(bf16_lo(w[r][k].y) * up, bf16_hi(w[r][k].y) * up);
      }
    }
  }
}

// Queries as the right operand, eight a tile; a lane's fragments belong to query lane/4 of each tile, its factors to the
// queries of its accumulators.
template <int kDim, bool kE4M3, int kTiles>
struct ColQueries {
  uint32_t b[kDim / 16][kTiles][2];
  float factor[2 * kTiles];
};

template <int kDim, bool kE4M3, int kTiles>
__device__ __forceinline__ void load_queries(ColQueries<kDim, kE4M3, kTiles>& Q, const AttnArgs& A, int item, int head,
                                             int) {
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int row = __ldcg(A.work.row + item);
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int j = t * 8 + g;
    const bool on = j < A.per_kv;
    const __nv_bfloat16* src = A.q + row * A.q_stride + (head * A.per_kv + (on ? j : 0)) * kDim;
    if constexpr (!kE4M3) {
#pragma unroll
      for (int k = 0; k < kDim / 16; ++k) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(src + k * 16);
        Q.b[k][t][0] = on ? p[c] : 0u;
        Q.b[k][t][1] = on ? p[c + 4] : 0u;
      }
      Q.factor[2 * t] = Q.factor[2 * t + 1] = A.to_log2;
    } else {
      // as fp16, scaled like the row form's; a lane's four dims of each 16 lie together, as a key's four codes do
      uint2 w[kDim / 16];
      float top = 0.0f;
#pragma unroll
      for (int k = 0; k < kDim / 16; ++k) {
        w[k] = on ? *reinterpret_cast<const uint2*>(src + k * 16 + 4 * c) : make_uint2(0u, 0u);
        top = fmaxf(top, fmaxf(fmaxf(fabsf(bf16_lo(w[k].x)), fabsf(bf16_hi(w[k].x))),
                               fmaxf(fabsf(bf16_lo(w[k].y)), fabsf(bf16_hi(w[k].y)))));
      }
      top = fmaxf(top, __shfl_xor_sync(kFullMask, top, 1));
      top = fmaxf(top, __shfl_xor_sync(kFullMask, top, 2));
      const int e = fp16_exponent(top);
      const float up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
#pragma unroll
      for (int k = 0; k < kDim / 16; ++k) {
        Q.b[k][t][0] = pack2<true>(bf16_lo(w[k].x) * up, bf16_hi(w[k].x) * up);
        Q.b[k][t][1] = pack2<true>(bf16_lo(w[k].y) * up, bf16_hi(w[k].y) * up);
      }
      const float down = A.to_log2 * __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
      for (int i = 0; i < 2; ++i) Q.factor[2 * t + i] = __shfl_sync(kFullMask, down, (2 * c + i) * 4);
    }
  }
}

// 16 tokens (rows t0 .. t0+15 of the tile, all present but those that `valid` leaves out, whose values are zero) against the
// warp's queries: scores as tokens x queries, weights turned round by a matrix transpose, values as dims x tokens.
template <int kDim, bool kE4M3, int kTiles>
__device__ __forceinline__ void chunk(ColAcc<kDim, kE4M3, kTiles>& X, const ColQueries<kDim, kE4M3, kTiles>& Q, uint32_t k_base,
                                      uint32_t v_base, const uint8_t* exps, int t0, uint32_t valid) {
  using T = Tile<kDim, kE4M3>;
  const int lane = threadIdx.x & 31, g = lane >> 2;
  const int row = t0 + (lane & 15);
  float s[kTiles][4];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.0f;
  if constexpr (!kE4M3) {
#pragma unroll
    for (int k = 0; k < kDim / 16; ++k) {
      uint32_t a[4];
      ldmatrix4(a, k_base + T::at(row, 2 * k + (lane >> 4)));
#pragma unroll
      for (int t = 0; t < kTiles; ++t) mma<false>(s[t], a, Q.b[k][t][0], Q.b[k][t][1]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < kDim / 16; k += 2) {
      uint32_t r[4];
      ldmatrix4(r, k_base + T::at(row, k + (lane >> 4)));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t a[4];
        e4m3x4_to_f16(r[2 * h], a[0], a[2]);
        e4m3x4_to_f16(r[2 * h + 1], a[1], a[3]);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) mma<true>(s[t], a, Q.b[k + h][t][0], Q.b[k + h][t][1]);
      }
    }
  }
  // tokens g and g + 8
  float kup[2] = {1.0f, 1.0f}, vup[2], add[2] = {0.0f, 0.0f};
  const bool on[2] = {((valid >> g) & 1u) != 0, ((valid >> (g + 8)) & 1u) != 0};
  if constexpr (kE4M3) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const uint32_t ke = exps[t0 + g + 8 * r], ve = exps[kTile + t0 + g + 8 * r];
      kup[r] = __uint_as_float(ke << 23);
      vup[r] = on[r] ? __uint_as_float((ve + kFoldBits) << 23) : 0.0f;      // a masked token's byte may be anything
      add[r] = static_cast<float>(static_cast<int>(ve) - 127);
    }
  }
  float top[2 * kTiles];
  bool moved = false;
#pragma unroll
  for (int q = 0; q < 2 * kTiles; ++q) {
    float* x = s[q >> 1];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float& y = x[2 * r + (q & 1)];
      y = on[r] ? y * (Q.factor[q] * kup[r]) : -INFINITY;
    }
    top[q] = fmaxf(x[q & 1] + add[0], x[2 + (q & 1)] + add[1]);
    top[q] = fmaxf(top[q], __shfl_xor_sync(kFullMask, top[q], 4));
    top[q] = fmaxf(top[q], __shfl_xor_sync(kFullMask, top[q], 8));
    top[q] = fmaxf(top[q], __shfl_xor_sync(kFullMask, top[q], 16));
    moved |= top[q] > X.m[q];
  }
  if (__any_sync(kFullMask, moved)) {
    float keep[2 * kTiles];
#pragma unroll
    for (int q = 0; q < 2 * kTiles; ++q) {
      const float m = fmaxf(X.m[q], top[q]);
      keep[q] = X.m[q] == m ? 1.0f : ex2_approx(X.m[q] - m);      // also where both are -inf
      X.m[q] = m;
      X.l[q] *= keep[q];
    }
    X.each([&](int q, int, float& v) { v *= keep[q]; });
  }
  uint32_t p[kTiles][2];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int q = 2 * t + i;
        const float m = X.m[q] == -INFINITY ? 0.0f : X.m[q];      // nothing seen yet: every weight is zero
        w[i] = ex2_approx(s[t][2 * r + i] - m);
        X.l[q] += w[i];
        if constexpr (kE4M3) w[i] *= vup[r];
      }
      p[t][r] = transpose8x8(pack2<kE4M3>(w[0], w[1]));
    }
#pragma unroll
  for (int i = 0; i < kDim / 16; i += kE4M3 ? 2 : 1) {
    uint32_t r[4];
    if constexpr (!kE4M3) {
      ldmatrix4_trans(r, v_base + T::at(t0 + (lane & 7) + 8 * (lane >> 4), 2 * i + ((lane >> 3) & 1)));
#pragma unroll
      for (int t = 0; t < kTiles; ++t) mma<false>(X.o[i][t], r, p[t][0], p[t][1]);
    } else {
      // a 16-bit column of a transposed load is two dims: their codes are separated, even dims to rows 0-7, odd to 8-15
      ldmatrix4_trans(r, v_base + T::at(t0 + (lane & 15), i + (lane >> 4)));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t a[4];
        e4m3x4_to_f16(__byte_perm(r[2 * h], 0, 0x3120), a[0], a[1]);
        e4m3x4_to_f16(__byte_perm(r[2 * h + 1], 0, 0x3120), a[2], a[3]);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) mma<true>(X.o[i + h][t], a, p[t][0], p[t][1]);
      }
    }
  }
}

// Zero weight times a masked token's NaN or infinity would be NaN, so the values of tokens that `valid` (16 bits from row t0)
// leaves out are cleared in the tile before it is used.
template <int kDim, bool kE4M3>
__device__ __forceinline__ void clear_values(uint8_t* v_tile, int t0, uint32_t valid) {
  using T = Tile<kDim, kE4M3>;
  const int lane = threadIdx.x & 31;
  for (int i = lane; i < 16 * (T::kRowBytes / 16); i += 32) {
    const int row = i / (T::kRowBytes / 16);
    if (!((valid >> row) & 1u)) *reinterpret_cast<uint4*>(v_tile + T::at(t0 + row, i % (T::kRowBytes / 16))) = make_uint4(0, 0, 0, 0);
  }
  __syncwarp();
}

// 16 tokens (rows t0 .. t0+15 of the tile; the values of those that `valid` leaves out are zero) against 16 queries.
template <int kDim, bool kE4M3>
__device__ __forceinline__ void chunk(RowAcc<kDim, kE4M3>& X, const RowQueries<kDim, kE4M3>& Q, uint32_t k_base, uint32_t v_base,
                                      const uint8_t* exps, int t0, uint32_t valid) {
  using T = Tile<kDim, kE4M3>;
  const int lane = threadIdx.x & 31, c = lane & 3;
  float s[2][4] = {};
  // scores: tokens are the columns
  if constexpr (!kE4M3) {
#pragma unroll
    for (int k = 0; k < kDim / 16; k += 2) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t b[4];
        ldmatrix4(b, k_base + T::at(t0 + 8 * j + (lane & 7), 2 * k + (lane >> 3)));
        mma<false>(s[j], Q.a[k], b[0], b[1]);
        mma<false>(s[j], Q.a[k + 1], b[2], b[3]);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < kDim / 16; k += 4) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t b[4];
        ldmatrix4(b, k_base + T::at(t0 + 8 * j + (lane & 7), k + (lane >> 3)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t b0, b1;
          e4m3x4_to_f16(b[i], b0, b1);
          mma<true>(s[j], Q.a[k + i], b0, b1);
        }
      }
    }
  }
  float vexp[2][2];                      // the values' factors 2^e of this lane's four columns
  float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float up = 1.0f, add = 0.0f;
      if constexpr (kE4M3) {
        const int t = t0 + 8 * j + 2 * c + i;
        const uint32_t ve = exps[kTile + t];
        up = __uint_as_float(static_cast<uint32_t>(exps[t]) << 23);
        vexp[j][i] = __uint_as_float((ve + kFoldBits) << 23);
        add = static_cast<float>(static_cast<int>(ve) - 127);
      }
      const bool on = (valid >> (8 * j + 2 * c + i)) & 1u;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float& x = s[j][i + 2 * r];
        x = on ? x * (Q.factor[r] * up) : -INFINITY;
        top[r] = fmaxf(top[r], x + add);
      }
    }
  bool moved = false;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    top[r] = fmaxf(top[r], __shfl_xor_sync(kFullMask, top[r], 1));
    top[r] = fmaxf(top[r], __shfl_xor_sync(kFullMask, top[r], 2));
    moved |= top[r] > X.m[r];
  }
  if (__any_sync(kFullMask, moved)) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float m = fmaxf(X.m[r], top[r]);
      const float keep = X.m[r] == m ? 1.0f : ex2_approx(X.m[r] - m);      // also where both are -inf
      X.m[r] = m;
      X.l[r] *= keep;
#pragma unroll
      for (int i = 0; i < kDim / 8; ++i) {
        X.o[i][2 * r] *= keep;
        X.o[i][2 * r + 1] *= keep;
      }
    }
  }
  uint32_t p[4];                         // weights as the left operand: rows g, g+8 x tokens 2c, 2c+1 | +8
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float m = X.m[r] == -INFINITY ? 0.0f : X.m[r];      // nothing seen yet: every weight below is zero
      float w0 = ex2_approx(s[j][2 * r] - m), w1 = ex2_approx(s[j][2 * r + 1] - m);
      X.l[r] += w0 + w1;
      if constexpr (kE4M3) {
        // a masked token's exponent byte may be anything: its weight is zero and must stay zero
        w0 = s[j][2 * r] == -INFINITY ? 0.0f : w0 * vexp[j][0];
        w1 = s[j][2 * r + 1] == -INFINITY ? 0.0f : w1 * vexp[j][1];
      }
      p[2 * j + r] = pack2<kE4M3>(w0, w1);
    }
  const int row = t0 + (lane & 15);
#pragma unroll
  for (int i = 0; i < T::kRowBytes / 16; i += 2) {
    uint32_t b[4];                       // tokens 0-7 and 8-15 of chunk i, then of chunk i + 1
    ldmatrix4_trans(b, v_base + T::at(row, i + (lane >> 4)));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (!kE4M3) {
        mma<false>(X.o[i + h], p, b[2 * h], b[2 * h + 1]);
      } else {
        uint32_t e0, o0, e1, o1;       // even and odd dims, tokens 0-7 and 8-15
        e4m3x4_to_f16(__byte_perm(b[2 * h], 0, 0x3120), e0, o0);
        e4m3x4_to_f16(__byte_perm(b[2 * h + 1], 0, 0x3120), e1, o1);
        mma<true>(X.o[2 * (i + h)], p, e0, e1);
        mma<true>(X.o[2 * (i + h) + 1], p, o0, o1);
      }
    }
  }
}

// One over the sum of weights; no tokens: zero, so that the output is zero; NaN stays NaN.
__device__ __forceinline__ float reciprocal(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }

// Query i of the lane becomes entry q[i] of arrays [..] and [..][dim].
template <int kDim, typename Acc>
__device__ __forceinline__ void store_part(Acc& X, float2* ml, float* o, const int64_t (&q)[Acc::kQ], const bool (&on)[Acc::kQ]) {
#pragma unroll
  for (int i = 0; i < Acc::kQ; ++i)
    if (on[i] && X.writes_ml()) ml[q[i]] = make_float2(X.m[i], X.l[i]);
  X.each([&](int i, int d, float& v) {
    if (on[i]) o[q[i] * kDim + d] = v;
  });
}

// The rows' own tokens.  kColTiles: 0: the warps split an item's queries, 16 each, and each walks all tokens; else they split
// its tokens and each has all queries, up to kColTiles times eight.  256 rows of 3000 tokens, 4 key/value heads of 128: with
// 4 queries each in the three forms 1, 2, 0: 247, 248, 310 us of bf16 and 137, 182, 356 of e4m3; with 12 in the forms 2, 0: 256,
// 320 and 193, 368 (one copying warp throughout).  Two copying warps, one for keys and one for values, serve the two blocks of
// forms 2 and 0 better (12 queries 182 us of e4m3, not 193; 24 queries 332 and 379, not 389 and 487) and the three of form 1
// worse (8 queries 145 of e4m3, not 141).
__host__ __device__ constexpr int copying_warps(int col_tiles) { return col_tiles == 1 ? 1 : 2; }
__host__ __device__ constexpr int tile_threads(int col_tiles) { return (kComputeWarps + copying_warps(col_tiles)) * 32; }
template <int kDim, bool kE4M3, int kColTiles>
__global__ void __launch_bounds__(tile_threads(kColTiles), kColTiles == 1 ? 3 : 2)
    tile_kernel(const AttnArgs A, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using T = Tile<kDim, kE4M3>;
  constexpr bool kByQuery = kColTiles == 0;
  constexpr int kStages = kColTiles == 1 ? T::kStagesOfThree : T::kStagesOfTwo;
  constexpr int kBlocks = kColTiles == 1 ? kOwnBlocks : kWideBlocks;
  using Acc = std::conditional_t<kByQuery, RowAcc<kDim, kE4M3>, ColAcc<kDim, kE4M3, kByQuery ? 1 : kColTiles>>;
  using Queries = std::conditional_t<kByQuery, RowQueries<kDim, kE4M3>, ColQueries<kDim, kE4M3, kByQuery ? 1 : kColTiles>>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* stages = smem;
  float* reduce = reinterpret_cast<float*>(smem + kStages * T::kStage);               // [2][8 kColTiles][kDim]
  Queue& Z = *reinterpret_cast<Queue*>(smem + kStages * T::kStage + 2 * 8 * kColTiles * kDim * 4);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Work& W = A.work;
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&Z.full[s], copying_warps(kColTiles));
      mbar_init(&Z.empty[s], kComputeWarps);
    }
    mbar_init(&Z.meeting, kComputeWarps);
    Z.abort_flag = 0;
    mbar_init_fence();
  }
  __syncthreads();
  let_next_kernel_start();
  wait_for_previous_kernel();

  const int n_heads = A.cache.n_kv_heads;
  const int64_t total = __ldcg(W.own_total);
  const int64_t line = total * n_heads;
  const int64_t per = piece_length(line, kBlocks, kMinTiles);
  const int64_t x_begin = blockIdx.x * per, x_end = min(x_begin + per, line);
  if (x_begin >= x_end) return;
  volatile int* abort_flag = &Z.abort_flag;

  if (warp >= kComputeWarps) {
    // ------------------------------------------------------------------ the copying warps: one for both, or keys and values
    constexpr int kEach = 2 / copying_warps(kColTiles);      // matrices a warp copies
    const int first_matrix = kEach == 2 ? 0 : warp - kComputeWarps;      // 0: keys, 1: values
    const bool leads = warp == kComputeWarps;
    const int page = A.cache.page_size;
    const int box = min(page, kTile);
    const int copies = kTile / box;                       // copies of `box` tokens per tile
    const int page_shift = 31 - __clz(page);
    const int my_token = (lane & 3) * box;                // lane i copies tokens [i * box, (i + 1) * box) of the tile
    uint32_t bad = 0;
    int stage = 0, filled = 0;
    uint32_t parity = 0;
    bool ok = true;
    int head = static_cast<int>(quotient(x_begin, total));
    int64_t x = x_begin;
    const int n_items = __ldcg(W.n_active);
    int item = warp_find(W.own_off, n_items, x - head * total);
    while (x < x_end && ok) {
      const int64_t begin = head * total + __ldcg(W.own_off + item);
      const int len = __ldcg(W.len + item);
      const int tiles = max((len + kTile - 1) / kTile, 1);
      const int32_t* table = A.seqs.pages + static_cast<int64_t>(__ldcg(W.slot + item)) * A.seqs.max_pages;
      const int n_pages = (len + page - 1) >> page_shift;
      int page_base = -64, my_page = -1;                  // lane i holds page page_base + i of the table
      for (; x < min(begin + tiles, x_end) && ok; ++x) {
        const int t = static_cast<int>(x - begin);
        const int p0 = t * kTile >> page_shift;           // the tile's first page
        if (p0 < page_base || p0 + copies > page_base + 32) {
          page_base = p0;
          my_page = p0 + lane < n_pages ? table[p0 + lane] : -1;
        }
        if (filled >= kStages) ok = warp_wait(&Z.empty[stage], parity ^ 1, abort_flag);
        if (!ok) break;
        const int mine = __shfl_sync(kFullMask, my_page, p0 + (lane < copies ? lane : 0) - page_base);
        const int left = len - t * kTile;                 // tokens from the tile's first on
        const bool wanted = lane < copies && my_token < left;
        const bool good = wanted && mine >= 0 && mine < A.cache.n_pages;
        if (wanted && !good) bad |= ESPO_DEV_BAD_PAGE;
        const unsigned copied = __ballot_sync(kFullMask, good);
        const int n_copied = __popc(copied);
        uint64_t valid = ~0ull;
        if (left < kTile || n_copied != copies) {
          valid = 0;
          for (int i = 0; i < copies; ++i) {
            const int n = min(max(left - i * box, 0), box);
            if ((copied >> i) & 1u) valid |= (n == 64 ? ~0ull : (1ull << n) - 1) << (i * box);
          }
        }
        uint8_t* dst = stages + stage * T::kStage;
        if (lane == 0) {
          if (leads) {
            StageInfo& I = Z.info[stage];
            const bool first_here = x == x_begin || t == 0, last_here = x == x_end - 1 || t == tiles - 1;
            I.valid = valid;
            I.item = item;
            I.head = head;
            I.flags = (first_here ? 1 : 0) | (last_here ? 2 : 0) | (begin < x_begin ? 8 : 0) | (begin + tiles > x_end ? 16 : 0);
          }
          mbar_arrive_expect_tx(&Z.full[stage], n_copied * box * kEach * (T::kRowBytes + (kE4M3 ? 1 : 0)));
        }
        __syncwarp();
        if (good) {
          const int64_t entry = ((static_cast<int64_t>(mine) * n_heads + head) << page_shift) + ((t * kTile + my_token) & (page - 1));
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            const bool values = first_matrix + i != 0;
            const CUtensorMap* map = values ? &v_map : &k_map;
            uint8_t* to = dst + (values ? T::kMatrix : 0) + my_token * T::kPartBytes;
#pragma unroll
            for (int part = 0; part < T::kParts; ++part)
              tma_2d(to + part * (kTile * 128), map, part * 64, static_cast<int>(entry), &Z.full[stage]);
            if constexpr (kE4M3)
              bulk_copy_g2s(dst + 2 * T::kMatrix + (values ? kTile : 0) + my_token, (values ? A.cache.v_exp : A.cache.k_exp) + entry,
                            box, &Z.full[stage]);
          }
        }
        ++filled;
        if (++stage == kStages) {
          stage = 0;
          parity ^= 1;
        }
      }
      if (++item == n_items) {
        item = 0;
        ++head;
      }
    }
    if (ok) {
      if (filled >= kStages) ok = warp_wait(&Z.empty[stage], parity ^ 1, abort_flag);
      if (ok && lane == 0) {
        if (leads) Z.info[stage].flags = 4;
        mbar_arrive(&Z.full[stage]);
      }
    }
    if (!ok) {
      *abort_flag = 1;
      bad |= ESPO_DEV_TIMEOUT;
    }
    // Copies in flight write to this block's shared memory, and the computing warps may give up before they arrive: the block
    // lasts until they have (bounded too).  Without such a mishap the last tiles are waited for anyhow.  `stage` itself has
    // been used up, unless the wait for it ran out.
    for (int i = 0; i < min(filled, ok ? kStages - 1 : kStages); ++i) {
      if (--stage < 0) {
        stage = kStages - 1;
        parity ^= 1;
      }
      if (!warp_wait(&Z.full[stage], parity, nullptr)) bad |= ESPO_DEV_TIMEOUT;
    }
    bad = __reduce_or_sync(kFullMask, bad);
    if (bad && lane == 0 && A.status_out) atomicOr(A.status_out, bad);
    return;
  }

  // -------------------------------------------------------------------- the computing warps
  Acc X;
  Queries Q;
  X.clear();
  const int q0 = kByQuery ? warp * 16 : 0;
  int stage = 0;
  uint32_t parity = 0, meeting_parity = 0;
  bool ok = true;
  auto meet = [&]() { return ok = warps_meet(&Z.meeting, meeting_parity, abort_flag); };
  for (;;) {
    // A warp whose wait runs out leaves the loop, although the tile may still come and be seen by the others: they meet
    // bounded too, and leave at the next meeting.
    ok = warp_wait(&Z.full[stage], parity, abort_flag);
    if (!ok) break;
    const StageInfo I = Z.info[stage];
    if (I.flags & 4) break;
    const bool busy = q0 < A.per_kv;
    if (I.flags & 1) {
      X.clear();
      if (busy) load_queries(Q, A, I.item, I.head, q0);
    }
    uint8_t* base = stages + stage * T::kStage;
    const uint32_t k_base = smem_addr(base), v_base = k_base + T::kMatrix;
    const uint8_t* exps = base + 2 * T::kMatrix;
    if constexpr (kByQuery) {
      if (I.valid != ~0ull) {            // each warp clears a quarter for all
        clear_values<kDim, kE4M3>(base + T::kMatrix, warp * 16, static_cast<uint32_t>(I.valid >> (16 * warp)) & 0xffffu);
        fence_proxy_async();             // the stage is the copies' again afterwards
        if (!meet()) break;
      }
      if (busy) {
#pragma unroll 1
        for (int ch = 0; ch < kTile / 16; ++ch) {
          const uint32_t valid = static_cast<uint32_t>(I.valid >> (16 * ch)) & 0xffffu;
          if (valid) chunk(X, Q, k_base, v_base, exps, ch * 16, valid);
        }
      }
    } else {
      const uint32_t valid = static_cast<uint32_t>(I.valid >> (16 * warp)) & 0xffffu;
      if (valid != 0xffffu) {
        clear_values<kDim, kE4M3>(base + T::kMatrix, warp * 16, valid);
        fence_proxy_async();
      }
      if (valid) chunk(X, Q, k_base, v_base, exps, warp * 16, valid);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&Z.empty[stage]);
    if (++stage == kStages) {
      stage = 0;
      parity ^= 1;
    }
    if (!(I.flags & 2)) continue;

    // ---------------------------------------------------------------- the item's last tile in this piece
    X.sum_l();
    bool mine = busy;
    if constexpr (!kByQuery) {
      // the four warps' results become warp 0's: each scales its own to the common maximum, then two pairwise additions
      if (X.writes_ml()) {
#pragma unroll
        for (int i = 0; i < Acc::kQ; ++i) Z.ml[warp][X.query(i)] = make_float2(X.m[i], X.l[i]);
      }
      if (!meet()) break;
      float keep[Acc::kQ];
#pragma unroll
      for (int i = 0; i < Acc::kQ; ++i) {
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < kComputeWarps; ++w) m = fmaxf(m, Z.ml[w][X.query(i)].x);
#pragma unroll
        for (int w = 0; w < kComputeWarps; ++w) {
          const float2 p = Z.ml[w][X.query(i)];
          l += p.x == m ? p.y : p.y * ex2_approx(p.x - m);
        }
        keep[i] = X.m[i] == m ? 1.0f : ex2_approx(X.m[i] - m);
        X.m[i] = m;
        X.l[i] = l;
      }
      X.each([&](int i, int, float& v) { v *= keep[i]; });
      float4* half = reinterpret_cast<float4*>(reduce) + (warp & 1) * (2 * kColTiles * kDim);
      auto put = [&]() {
#pragma unroll
        for (int i = 0; i < kDim / 16; ++i)
#pragma unroll
          for (int t = 0; t < kColTiles; ++t)
            half[(i * kColTiles + t) * 32 + lane] = make_float4(X.o[i][t][0], X.o[i][t][1], X.o[i][t][2], X.o[i][t][3]);
      };
      auto add = [&](const float4* from) {
#pragma unroll
        for (int i = 0; i < kDim / 16; ++i)
#pragma unroll
          for (int t = 0; t < kColTiles; ++t) {
            const float4 v = from[(i * kColTiles + t) * 32 + lane];
            X.o[i][t][0] += v.x;
            X.o[i][t][1] += v.y;
            X.o[i][t][2] += v.z;
            X.o[i][t][3] += v.w;
          }
      };
      if (warp >= 2) put();
      if (!meet()) break;
      if (warp < 2) add(half);
      if (!meet()) break;
      if (warp == 1) put();
      if (!meet()) break;
      if (warp == 0) add(reinterpret_cast<float4*>(reduce) + 2 * kColTiles * kDim);
      mine = warp == 0;
    }
    if (!mine) continue;
    bool on[Acc::kQ];
    int64_t q[Acc::kQ];
#pragma unroll
    for (int i = 0; i < Acc::kQ; ++i) on[i] = q0 + X.query(i) < A.per_kv;
    if (I.flags & 24) {              // the row is cut
#pragma unroll
      for (int i = 0; i < Acc::kQ; ++i) q[i] = (static_cast<int64_t>(blockIdx.x) * 2 + (I.flags & 8 ? 0 : 1)) * A.per_kv + q0 + X.query(i);
      store_part<kDim>(X, W.own_ml, W.own_o, q, on);
    } else if (A.seqs.group && __ldcg(W.segment + I.item) >= 0) {
#pragma unroll
      for (int i = 0; i < Acc::kQ; ++i) q[i] = static_cast<int64_t>(I.item) * A.n_q_heads + I.head * A.per_kv + q0 + X.query(i);
      store_part<kDim>(X, W.whole_ml, W.whole_o, q, on);
    } else {
      const int row = __ldcg(W.row + I.item);
      float inv[Acc::kQ];
      __nv_bfloat16* dst[Acc::kQ];
#pragma unroll
      for (int i = 0; i < Acc::kQ; ++i) {
        inv[i] = reciprocal(X.l[i]) * (kE4M3 ? 1.0f / (1 << kFoldBits) : 1.0f);
        dst[i] = A.out + row * A.out_stride + (I.head * A.per_kv + q0 + X.query(i)) * kDim;
      }
      X.each([&](int i, int d, float& v) {
        if (on[i]) dst[i][d] = __float2bfloat16(v * inv[i]);
      });
    }
  }
  if (!ok) {
    *abort_flag = 1;
    if (lane == 0 && A.status_out) atomicOr(A.status_out, ESPO_DEV_TIMEOUT);
  }
}

// ---------------------------------------------------------------------------------------------- joining parts

// A warp per row and query head whose result lies in several parts: its own tokens' (cut between blocks or not) and its
// prefix's.  In a fixed order: own parts along the line, then the prefix's.
template <int kDim, bool kE4M3>
__global__ void __launch_bounds__(256) join_kernel(const AttnArgs A, const __grid_constant__ CUtensorMap, const __grid_constant__ CUtensorMap) {
  constexpr int kN = kDim / 32;
  const Work& W = A.work;
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int64_t a = quotient(at, A.n_q_heads);
  const int h = static_cast<int>(at - a * A.n_q_heads);
  if (a >= __ldcg(W.n_active)) return;
  const int head = h / A.per_kv, q = h % A.per_kv;
  const int seg = A.seqs.group ? __ldcg(W.segment + a) : -1;
  const int64_t own_total = __ldcg(W.own_total);
  const int64_t own_per = piece_length(own_total * A.cache.n_kv_heads, A.own_blocks, kMinTiles);
  const int64_t b0 = quotient(head * own_total + __ldcg(W.own_off + a), own_per);
  const int64_t b1 = quotient(head * own_total + __ldcg(W.own_off + a + 1) - 1, own_per);
  if (b0 == b1 && seg < 0) return;                       // written already
  const int n_own = static_cast<int>(b1 - b0) + 1;
  int n_prefix = 0;
  int64_t p0 = 0, in_block = 0;
  if (seg >= 0) {
    const int64_t total = __ldcg(W.prefix_total);
    const int64_t per = piece_length(total * A.cache.n_kv_heads, kPrefixBlocks, 1);
    const int in_seg = static_cast<int>(a) - __ldcg(W.seg_first + seg);
    const int tiles = (__ldcg(W.seg_len + seg) + kPrefixTile - 1) / kPrefixTile;
    const int64_t x0 = head * total + __ldcg(W.seg_off + seg) + tiles_before_row(in_seg, A.rows_per_block, tiles);
    p0 = quotient(x0, per);
    n_prefix = static_cast<int>(quotient(x0 + tiles - 1, per) - p0) + 1;
    in_block = in_seg % A.rows_per_block * A.per_kv + q;
  }
  float m = -INFINITY, l = 0.0f, o[kN] = {};
  for (int first = 0; first < n_own + n_prefix; first += 32) {
    // a lane per part
    const int i = first + lane, n = min(32, n_own + n_prefix - first);
    const float2* ml = nullptr;
    const float* src = nullptr;
    float times = 1.0f;
    if (i < n_own) {
      const int64_t e = n_own == 1 ? at : ((b0 + i) * 2 + (i == 0 ? 1 : 0)) * A.per_kv + q;
      ml = (n_own == 1 ? W.whole_ml : W.own_ml) + e;
      src = (n_own == 1 ? W.whole_o : W.own_o) + e * kDim;
      if constexpr (kE4M3) times = 1.0f / (1 << kFoldBits);
    } else if (i < n_own + n_prefix) {
      const int64_t e = i == n_own ? at : (p0 + i - n_own) * kPrefixQueries + in_block;
      ml = (i == n_own ? W.prefix_ml : W.extra_ml) + e;
      src = (i == n_own ? W.prefix_o : W.extra_o) + e * kDim;
    }
    const float2 mine = ml ? __ldcg(ml) : make_float2(-INFINITY, 0.0f);
    const float to = fmaxf(m, warp_max(mine.x));
    const float keep = m == to ? 1.0f : ex2_approx(m - to), take = mine.x == to ? 1.0f : ex2_approx(mine.x - to);
    m = to;
    l = l * keep + warp_sum(ml ? mine.y * take : 0.0f);
#pragma unroll
    for (int d = 0; d < kN; ++d) o[d] *= keep;
    const float factor = take * times;
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      const float* p = reinterpret_cast<const float*>(__shfl_sync(kFullMask, reinterpret_cast<unsigned long long>(src), j));
      const float f = __shfl_sync(kFullMask, factor, j);
      if constexpr (kN == 4) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(p) + lane);
        o[0] += v.x * f;
        o[1] += v.y * f;
        o[2] += v.z * f;
        o[3] += v.w * f;
      } else {
        const float2 v = __ldcg(reinterpret_cast<const float2*>(p) + lane);
        o[0] += v.x * f;
        o[1] += v.y * f;
      }
    }
  }
  const float inv = reciprocal(l);
  __nv_bfloat16* dst = A.out + __ldcg(W.row + a) * A.out_stride + h * kDim + lane * kN;
  if constexpr (kN == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
  else *reinterpret_cast<uint32_t*>(dst) = pack_bf16x2(o[0] * inv, o[1] * inv);
}

// ---------------------------------------------------------------------------------------------- host side

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

// The cache as a matrix of n_pages * n_kv_heads * page_size rows; a copy takes up to 64 rows of one page, 128 bytes wide.
int make_map(CUtensorMap* map, const espo_kv_cache& c, void* base) {
  EncodeTiled encode = encode_tiled();
  if (!encode) return record_cuda_error(cudaErrorNotSupported);
  const bool e = c.dtype == ESPO_E4M3;
  const cuuint64_t rows = static_cast<cuuint64_t>(c.n_pages) * c.n_kv_heads * c.page_size;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(c.head_dim), rows};
  const cuuint64_t stride[1] = {static_cast<cuuint64_t>(c.head_dim) * (e ? 1 : 2)};
  const cuuint32_t width = e ? c.head_dim : 64;
  const cuuint32_t box[2] = {width, static_cast<cuuint32_t>(c.page_size < kTile ? c.page_size : kTile)};
  const cuuint32_t one[2] = {1, 1};
  const CUresult rc = encode(map, e ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, stride, box,
                             one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                             e && c.head_dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return rc == CUDA_SUCCESS ? ESPO_OK : record_cuda_error(cudaErrorInvalidValue);
}

// Launches a kernel that may be set up while the one before it in the stream winds down.
int launch_chained(void (*f)(AttnArgs, CUtensorMap, CUtensorMap), int blocks, int threads, int smem, const AttnArgs& a,
                   const CUtensorMap& k, const CUtensorMap& v, cudaStream_t st) {
  if (smem > 48 * 1024) ESPO_CUDA_TRY(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  ESPO_CUDA_TRY(cudaLaunchKernelEx(&cfg, f, a, k, v));
  return ESPO_OK;
}

template <int kDim, bool kE4M3, int kColTiles>
int launch_tiles(const AttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t st) {
  using T = Tile<kDim, kE4M3>;
  constexpr int kSmem = (kColTiles == 1 ? T::kStagesOfThree : T::kStagesOfTwo) * T::kStage + 2 * 8 * kColTiles * kDim * 4 + sizeof(Queue);
  static_assert(kSmem + 1024 <= 228 * 1024 / (kColTiles == 1 ? 3 : 2), "two or three blocks share an SM's 228 KB");
  return launch_chained(tile_kernel<kDim, kE4M3, kColTiles>, kColTiles == 1 ? kOwnBlocks : kWideBlocks, tile_threads(kColTiles), kSmem, a, k, v, st);
}

template <int kDim, bool kE4M3>
int launch_prefix(const AttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t st) {
  constexpr int kSmem = PrefixShape<kDim, kE4M3>::kBytes + sizeof(PrefixShared);
  static_assert(kSmem <= 227 * 1024, "one block on an SM");
  return launch_chained(prefix_kernel<kDim, kE4M3>, kPrefixBlocks, kPrefixThreads, kSmem, a, k, v, st);
}

template <int kDim, bool kE4M3>
int launch_attention(const AttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t st) {
  if (a.seqs.group) {
    const int rc = launch_prefix<kDim, kE4M3>(a, k, v, st);
    if (rc != ESPO_OK) return rc;
  }
  const int rc = a.per_kv <= 8    ? launch_tiles<kDim, kE4M3, 1>(a, k, v, st)
                 : a.per_kv <= 16 ? launch_tiles<kDim, kE4M3, 2>(a, k, v, st)
                                  : launch_tiles<kDim, kE4M3, 0>(a, k, v, st);
  if (rc != ESPO_OK) return rc;
  const int64_t warps = static_cast<int64_t>(a.n_rows) * a.n_q_heads;
  return launch_chained(join_kernel<kDim, kE4M3>, static_cast<int>((warps + 7) / 8), 256, 0, a, k, v, st);
}

int check_heads(const espo_kv_cache* cache, int32_t n_q_heads) {
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads || n_q_heads / cache->n_kv_heads > kMaxPerKv) return ESPO_ERR_BAD_SHAPE;
  return ESPO_OK;
}

}  // namespace
}  // namespace espo

using namespace espo;

extern "C" {

int espo_attention_workspace(const espo_kv_cache* cache, int32_t n_rows, int32_t n_q_heads, int64_t* bytes_out) {
  if (!bytes_out) return ESPO_ERR_NULL;
  int rc = check_kv_cache(cache);
  if (rc == ESPO_OK) rc = check_heads(cache, n_q_heads);
  if (rc != ESPO_OK) return rc;
  if (n_rows < 0) return ESPO_ERR_BAD_SHAPE;
  Work w;
  *bytes_out = work_layout(w, nullptr, n_rows, n_q_heads, n_q_heads / cache->n_kv_heads, cache->head_dim);
  return ESPO_OK;
}

int espo_attention(const espo_kv_cache* cache, const espo_sequences* seqs, const void* q, int64_t q_stride,
                   int32_t n_q_heads, const int32_t* row_ids, int32_t n_rows, float scale, void* out, int64_t out_stride,
                   void* workspace, int64_t workspace_bytes, uint32_t* status_out, void* stream) {
  int64_t need = 0;
  int rc = espo_attention_workspace(cache, n_rows, n_q_heads, &need);
  if (rc == ESPO_OK) rc = check_sequences(seqs);
  if (rc != ESPO_OK) return rc;
  if (!workspace || (n_rows > 0 && (!q || !out))) return ESPO_ERR_NULL;
  if (!(fabsf(scale) <= 0x1p127f)) return ESPO_ERR_BAD_PARAM;      // NaN too; times log2(e) it has to stay finite
  const int64_t row = static_cast<int64_t>(n_q_heads) * cache->head_dim;
  if (q_stride < row || out_stride < row) return ESPO_ERR_BAD_SHAPE;
  if (q_stride % 8 || out_stride % 8 || !aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256) ||
      !aligned(row_ids, 4) || !aligned(status_out, 4))
    return ESPO_ERR_ALIGN;
  if (workspace_bytes < need || n_rows > seqs->capacity) return ESPO_ERR_CAPACITY;
  if (n_rows == 0) return ESPO_OK;
  AttnArgs a = {};
  a.cache = *cache;
  a.seqs = *seqs;
  work_layout(a.work, static_cast<char*>(workspace), n_rows, n_q_heads, n_q_heads / cache->n_kv_heads, cache->head_dim);
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.row_ids = row_ids;
  a.status_out = status_out;
  a.to_log2 = scale * 1.44269504088896340736f;
  a.n_q_heads = n_q_heads;
  a.n_rows = n_rows;
  a.per_kv = n_q_heads / cache->n_kv_heads;
  a.own_blocks = a.per_kv <= 8 ? kOwnBlocks : kWideBlocks;
  a.rows_per_block = kPrefixQueries / a.per_kv;
  CUtensorMap k, v;
  rc = make_map(&k, *cache, cache->k);
  if (rc == ESPO_OK) rc = make_map(&v, *cache, cache->v);
  if (rc != ESPO_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  plan_kernel<<<1, kPlanThreads, 0, st>>>(a);
  ESPO_CUDA_TRY(cudaGetLastError());
  const bool e = cache->dtype == ESPO_E4M3;
  if (cache->head_dim == 128) return e ? launch_attention<128, true>(a, k, v, st) : launch_attention<128, false>(a, k, v, st);
  return e ? launch_attention<64, true>(a, k, v, st) : launch_attention<64, false>(a, k, v, st);
}

}  // extern "C"
