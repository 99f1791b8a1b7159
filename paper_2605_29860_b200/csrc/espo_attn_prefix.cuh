// The shared prefixes: every tile of 128 tokens of a segment's prefix against 128 queries -- as many whole rows of the segment
// as fit -- of one key/value head, on the fifth-generation tensor cores.
//
// Mathematics.  S = Q K^T and O += P V are matrix products with 32-bit accumulators in tensor memory; the softmax between
// them is one row per thread.  Even and odd tiles of an item form two independent streams, each with its own O, running
// maximum and sum (joined when the item ends), so that one's products run beside the other's softmax.  The softmax hands its
// weights over in halves of 64 tokens.  A maximum is only moved when a score exceeds it by more than 8 doublings, which is
// rare after the first tiles: until then weights are at most 2^8, and O need not be read back and rescaled.
//
// Roundings.  The weights become bf16 for the product with the values (at most 2^-8 of each; the sum l takes them unrounded), since
// one instruction's operands share a type, and the values are bf16: a cache's own, or e4m3 codes with exponents that no other 16-bit
// type holds.  For an e4m3 prefix fp16 weights would be eight times finer; they need the values' exponents folded into them.
//
// What bounds it: a stream's chain of product, softmax (1200 clocks a half: loading scores 300, maximum 100, exponentials
// 740) and product, 4100 clocks for a tile of each of the two streams, against 1024 a tile for the exponentials alone (16 a
// clock and SM) and 768 for the products.  e4m3 pages add the conversion (by instruction to half
// and float, on to bf16): about 2700 clocks a tile; moving the codes' bits into place instead took 3700, on the integer pipe that
// the softmax needs too (8 groups of 32, 64 dims: 67 us, now 54).  Before an item's first product lie about 8 us: the plan, the walk to the item, its queries.
// One group of 64 rows, 28 query heads on 4 of 128 dims, 40000 tokens of bf16: 60 us, 580 TFLOP/s, tensor
// pipe 31 % active; 64 groups of 8 with up to 700 tokens: bf16 24 us, e4m3 42.  All 128 registers that 512 threads leave each are
// taken, with 28 bytes spilled.  Measured and dropped: one
// warp for both operands' copies (79 us: 1750 clocks to issue a unit), products of 64 keys (62), a second set of four
// converting warps with 96 registers a thread (while codes were still moved by bits: 64 groups of 8 on e4m3 pages 241 us against
// 237, 64-dim heads 137 against 141).
//
// Roles of the block's 16 warps: 0-3 and 4-7 the softmax of the even and the odd tiles; 8-11 load the queries, turn e4m3
// keys and values into bf16 (exact: a code has 4 significant bits and its scale is a power of two) and clear the values of
// absent tokens; 12 copies keys and 15 values; 13 issues the products with the keys, 14 those with the values (one warp for
// both spent as long between products as in them).  Keys and values travel through one ring of 128-token units in the order
// of use: K0 K1 V0 K2 V1 K3 V2 ...
#pragma once

#include <cuda_fp8.h>

#include "espo_attn_common.cuh"

namespace espo {
namespace {

constexpr int kPrefixThreads = 16 * 32;

template <int kDim, bool kE4M3>
struct PrefixShape {
  static constexpr int kUnit = kPrefixTile * kDim * 2;                     // bf16
  static constexpr int kRaw = kE4M3 ? kPrefixTile * kDim + 1024 : 0;       // codes, then the exponents in a kilobyte of their own
  static constexpr int kUnits = kDim == 128 ? (kE4M3 ? 4 : 6) : 8;
  static constexpr int kRaws = kE4M3 ? (kDim == 128 ? 3 : 4) : 0;
  static constexpr int kQBytes = 128 * kDim * 2;
  static constexpr int kBytes = kQBytes + kUnits * kUnit + kRaws * kRaw;
};

struct PrefixShared {
  uint64_t loaded[8];        // a copied unit (bf16) or raw unit (e4m3) has arrived
  uint64_t free[8];          // the products have read a unit (bf16: and the clearing warps and the other copying warp are past it)
  uint64_t raw_free[4];      // e4m3: a raw unit has been converted, and the copying warp that did not fill it is past it
  uint64_t ready[8];         // e4m3: a unit is converted; bf16: an incomplete value unit is cleared
  uint64_t scores[2];        // S of a stream's tile is complete
  uint64_t weights[2][2];    // P of a stream's half tile is written
  uint64_t used[2][2];       // and its product with the values complete
  uint64_t queries;          // Q is in place
  uint64_t done;             // the item's products are complete
  uint64_t odd;              // the odd stream's maxima and sums are in place
  uint64_t written;          // the item's result has been read from tensor memory
  uint64_t drained[2];       // the products of each issuing warp are complete, at the block's end
  uint64_t valid[8][2];      // by unit slot (e4m3: raw slot): a bit per token
  uint64_t tile_valid[8][2]; // the same for the softmax, by the block's running tile number: a tile's entry is written again
                             // with the eighth tile after it, whose key unit finds room only once this tile's product with
                             // the values is complete
  float2 ml[128];
  float factor;              // |scale| log2(e), its sign is in Q; for a scale of zero Q is zero and this 1
  uint32_t tmem;
  int abort_flag;
};

// One item of the block's piece of the line, found by every role for itself.
struct PrefixItem {
  int head, seg, block;
  int first, rows;           // its active rows
  int tile0, tiles;          // its tiles inside the piece
  int len;                   // tokens of the prefix
  bool from_before;          // its first tile lies in an earlier piece
};

struct PrefixWalk {
  int64_t x, x_end, total;
  int head, seg, n_seg;
  // Whole warps call this.
  __device__ __forceinline__ void start(const AttnArgs& A) {
    const Work& W = A.work;
    total = __ldcg(W.prefix_total);
    const int64_t line = total * A.cache.n_kv_heads;
    const int64_t per = piece_length(line, kPrefixBlocks, 1);
    x = min(blockIdx.x * per, line);
    x_end = min(x + per, line);
    if (x >= x_end) return;
    n_seg = __ldcg(W.n_segments);
    head = static_cast<int>(quotient(x, total));
    seg = warp_find(W.seg_off, n_seg, x - head * total);
  }
  __device__ __forceinline__ bool next(const AttnArgs& A, PrefixItem& I) {
    if (x >= x_end) return false;
    const Work& W = A.work;
    if (x - head * total >= __ldcg(W.seg_off + seg + 1)) {
      if (++seg == n_seg) {
        seg = 0;
        ++head;
      }
    }
    I.len = __ldcg(W.seg_len + seg);
    const int tiles = (I.len + kPrefixTile - 1) / kPrefixTile;
    I.head = head;
    I.seg = seg;
    block_and_tile(x - head * total - __ldcg(W.seg_off + seg), tiles, I.block, I.tile0);
    I.tiles = static_cast<int>(min(static_cast<int64_t>(tiles - I.tile0), x_end - x));
    I.first = __ldcg(W.seg_first + seg) + I.block * A.rows_per_block;
    I.rows = min(A.rows_per_block, __ldcg(W.seg_end + seg) - I.first);
    I.from_before = I.tile0 > 0;
    x += I.tiles;
    return true;
  }
};

// The ring's order for an item of n tiles, K0 K1 V0 K2 V1 K3 ...; the keys end first: position of a tile's keys and values.
__device__ __forceinline__ int key_unit(int t) { return t < 2 ? t : 2 * t - 1; }
__device__ __forceinline__ int value_unit(int t, int n) { return t < n - 2 ? 2 * t + 2 : t + n; }
__device__ __forceinline__ void unit_at(int p, int n, bool& is_key, int& tile) {
  const int i = (p - 2) >> 1;
  if (p < 2 && p < n) {
    is_key = true;
    tile = p;
  } else if (p >= 2 && i < n - 2) {
    is_key = (p & 1) != 0;
    tile = is_key ? i + 2 : i;
  } else {
    is_key = false;
    tile = p - n;
  }
}

// ---- tensor memory and products

__device__ __forceinline__ void tmem_alloc(uint32_t* out, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(out)), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Waits for the warp's loads from tensor memory; the registers pass through so that no use of them moves ahead of the wait.
template <int kN>
__device__ __forceinline__ void tmem_wait_ld(float (&v)[kN]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < kN; ++i) asm volatile("" : "+f"(v[i]));
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of the lane's row; tmem_wait_ld() comes before their use.
__device__ __forceinline__ void tmem_load32(uint32_t at, float* v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
      "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at) : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at) : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(v[0]),
      "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
      "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float m;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
  return m;
}
// 32 bytes, a whole sector: the lanes' rows lie far apart.
__device__ __forceinline__ void store_sector(float* p, const float* v) {
  asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]),
               "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}

// Shared-memory matrix of rows of 64 bf16 (128 bytes, 128-byte swizzle), eight rows a kilobyte; wider matrices continue
// `group` bytes further on.  Bits: address and the two strides in 16 bytes, version 1, swizzle mode 2.
__device__ __forceinline__ uint64_t matrix_descriptor(uint32_t addr, uint32_t group) {
  return static_cast<uint64_t>((addr >> 4) & 0x3fffu) | (static_cast<uint64_t>((group >> 4) & 0x3fffu) << 16) |
         (static_cast<uint64_t>(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// bf16 x bf16 -> 32-bit, 128 rows, n columns; `across`: the right operand's columns lie together (values), not its depth (keys).
__device__ __forceinline__ constexpr uint32_t product_descriptor(int n, bool across) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (across ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) | (8u << 24);
}
__device__ __forceinline__ void product_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
               "l"(a), "l"(b), "r"(desc), "r"(add ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
               "r"(a), "l"(b), "r"(desc), "r"(add ? 1u : 0u) : "memory");
}
// One thread of the warp, in a form that lets the compiler keep the products' operands in uniform registers (half the time
// to issue eight of them, against a test of the lane's number).
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0;
}
// Arrives on the barrier once everything issued so far is complete.
__device__ __forceinline__ void products_arrive(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// Waits (bounded) until everything the warp has issued is complete: nothing reads shared or tensor memory after that, whoever
// gives up.  `bar` serves this one time.
__device__ __forceinline__ bool products_end(uint64_t* bar) {
  __syncwarp();
  if (elect_one()) products_arrive(bar);
  __syncwarp();
  return warp_wait(bar, 0, nullptr);
}

// Two bf16 numbers times zero: zeros, or NaN.
__device__ __forceinline__ uint32_t times_zero(uint32_t w) { return pack_bf16x2(bf16_lo(w) * 0.0f, bf16_hi(w) * 0.0f); }

// Byte offset of 16-byte chunk `chunk` (of eight numbers) of row `row` in a 128-row matrix of bf16.
__device__ __forceinline__ uint32_t unit_offset(int row, int chunk) {
  return (chunk >> 3) * (128 * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
}

template <int kDim, bool kE4M3>
__global__ void __launch_bounds__(kPrefixThreads, 1)
    prefix_kernel(const AttnArgs A, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using P = PrefixShape<kDim, kE4M3>;
  constexpr uint32_t kTmemColumns = 512;
  constexpr int kChunks = kDim / 8;                  // 16-byte chunks of a bf16 row
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* q_tile = smem;
  uint8_t* units = smem + P::kQBytes;
  uint8_t* raws = units + P::kUnits * P::kUnit;
  PrefixShared& Z = *reinterpret_cast<PrefixShared*>(smem + P::kBytes);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile int* abort_flag = &Z.abort_flag;
  if (tid == 0) {
    for (int i = 0; i < 8; ++i) {
      mbar_init(&Z.loaded[i], 1);
      mbar_init(&Z.free[i], kE4M3 ? 1 : 6);
      mbar_init(&Z.ready[i], 4);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&Z.raw_free[i], 5);
    for (int i = 0; i < 2; ++i) mbar_init(&Z.scores[i], 1);
    for (int i = 0; i < 4; ++i) {
      mbar_init(&Z.weights[0][0] + i, 4);
      mbar_init(&Z.used[0][0] + i, 1);
    }
    mbar_init(&Z.queries, 4);
    mbar_init(&Z.done, 1);
    mbar_init(&Z.odd, 4);
    mbar_init(&Z.written, 4);
    mbar_init(&Z.drained[0], 1);
    mbar_init(&Z.drained[1], 1);
    Z.abort_flag = 0;
    Z.factor = A.to_log2 != 0.0f ? fabsf(A.to_log2) : 1.0f;      // not zero: a masked score has to stay -inf
    mbar_init_fence();
  }
  __syncthreads();
  let_next_kernel_start();
  if (warp == 13) tmem_alloc(&Z.tmem, kTmemColumns);
  wait_for_previous_kernel();
  PrefixWalk walk;
  walk.start(A);
  if (walk.x >= walk.x_end) {                        // the whole block
    if (warp == 13) tmem_free(Z.tmem, kTmemColumns);
    return;
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = Z.tmem;
  // tensor memory: S of stream w, half h at column 128 w + 64 h (P in the same place), O of stream w behind them
  const uint32_t o_at[2] = {tmem + 256, tmem + 256 + kDim};
  PrefixItem I;
  bool ok = true;
  uint32_t bad = 0;

  if (warp == 12 || warp == 15) {
    // ---------------------------------------------------------------- copies of keys (12) and of values (15)
    constexpr int kSlots = kE4M3 ? P::kRaws : P::kUnits;
    const bool keys = warp == 12;
    const int page = A.cache.page_size, shift = 31 - __clz(page), box = min(page, 64);      // a tile is whole pages
    const int copies = kPrefixTile / box;                          // at most eight
    const int my_token = lane * box;                               // lane i copies the i-th box
    const int in_page = my_token & (page - 1);
    const CUtensorMap* map = keys ? &k_map : &v_map;
    const uint8_t* exps = keys ? A.cache.k_exp : A.cache.v_exp;
    int slot = 0, tile = 0;
    uint32_t parity = 0, filled = 0, filled_parity = 0;            // filled: a bit per slot this warp filled last, and the phase
    for (; ok && walk.next(A, I); tile += I.tiles) {
      const int32_t* table = A.seqs.prefix_pages + static_cast<int64_t>(__ldcg(A.work.seg_group + I.seg)) * A.seqs.max_prefix_pages;
      // Page ids four tiles at a time, lane 8 i + j for box j of the i-th, loaded four tiles before they are used.
      auto load_ids = [&](int batch) {
        const int token = (I.tile0 + 4 * batch + (lane >> 3)) * kPrefixTile + (lane & 7) * box;
        return (lane & 7) < copies && token < I.len ? __ldg(table + (token >> shift)) : -1;
      };
      int ids = load_ids(0), next_ids = load_ids(1);
      for (int p = 0; p < 2 * I.tiles && ok; ++p) {
        bool is_key;
        int t;
        unit_at(p, I.tiles, is_key, t);
        // for every unit, the other warp's too: a phase passed over could be taken for the next of its parity
        if (2 * tile + p >= kSlots) ok = warp_wait(kE4M3 ? &Z.raw_free[slot] : &Z.free[slot], parity ^ 1, abort_flag);
        if (!ok) break;
        filled &= ~(1u << slot);                                   // what was there is free
        if (is_key == keys) {
          if (t > 0 && (t & 3) == 0) {
            ids = next_ids;
            next_ids = load_ids((t >> 2) + 1);
          }
          const int left = I.len - (I.tile0 + t) * kPrefixTile;         // tokens from the tile's first on
          const int id = __shfl_sync(kFullMask, ids, 8 * (t & 3) + (lane & 7));
          const bool wanted = lane < copies && my_token < left;
          const bool good = wanted && id >= 0 && id < A.cache.n_pages;
          if (wanted && !good) bad |= ESPO_DEV_BAD_PAGE;
          const unsigned copied = __ballot_sync(kFullMask, good);
          const int n_copied = __popc(copied);
          uint64_t valid = ~0ull;
          if (left < kPrefixTile || n_copied != copies) {
            valid = 0;
            for (int i = 0; i < 64 / box; ++i) {
              const int b = (lane & 1) * (64 / box) + i;
              const int n = min(max(left - b * box, 0), box);
              if ((copied >> b) & 1u) valid |= (n == 64 ? ~0ull : (1ull << n) - 1) << (i * box);
            }
          }
          if (lane < 2) {
            Z.valid[slot][lane] = valid;
            if (keys) Z.tile_valid[(tile + t) & 7][lane] = valid;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive_expect_tx(&Z.loaded[slot], n_copied * box * (kE4M3 ? kDim + 1 : kDim * 2));
          __syncwarp();
          if (good) {
            const int64_t entry = ((static_cast<int64_t>(id) * A.cache.n_kv_heads + I.head) << shift) + in_page;
            if constexpr (kE4M3) {
              uint8_t* dst = raws + slot * P::kRaw;
              tma_2d(dst + my_token * kDim, map, 0, static_cast<int>(entry), &Z.loaded[slot]);
              bulk_copy_g2s(dst + kPrefixTile * kDim + my_token, exps + entry, box, &Z.loaded[slot]);
            } else {
              uint8_t* dst = units + slot * P::kUnit;
#pragma unroll
              for (int h = 0; h < kDim / 64; ++h)
                tma_2d(dst + h * (128 * 128) + my_token * 128, map, h * 64, static_cast<int>(entry), &Z.loaded[slot]);
            }
          }
          filled |= 1u << slot;
          filled_parity = (filled_parity & ~(1u << slot)) | (parity << slot);
        } else if (lane == 0) {
          // The slot is not free again before this warp has passed it: two phases on, the wait above would not know its own.
          mbar_arrive(kE4M3 ? &Z.raw_free[slot] : &Z.free[slot]);
        }
        if (++slot == kSlots) {
          slot = 0;
          parity ^= 1;
        }
      }
    }
    // Copies in flight write to this block's shared memory, and another warp may give up before they arrive: the block lasts
    // until they have (bounded too).
    for (int i = 0; i < kSlots; ++i)
      if ((filled >> i) & 1u) ok &= warp_wait(&Z.loaded[i], (filled_parity >> i) & 1u, nullptr);
    bad = __reduce_or_sync(kFullMask, bad);
  } else if (warp == 13) {
    // ---------------------------------------------------------------- scores: S = Q K^T
    constexpr uint32_t kDesc = product_descriptor(kPrefixTile, false);
    const uint64_t q_desc = matrix_descriptor(smem_addr(q_tile), 0);
    uint32_t item_parity = 0;
    uint32_t products[2] = {0, 0};                       // value products of a stream before this item's
    uint32_t base = 0;                                   // units before this item's
    for (; ok && walk.next(A, I); base += 2 * I.tiles) {
      ok = warp_wait(&Z.queries, item_parity, abort_flag);
      for (int t = 0; t < I.tiles && ok; ++t) {
        const int w = t & 1;
        const uint32_t unit = base + key_unit(t), slot = unit % P::kUnits;
        ok = warp_wait(kE4M3 ? &Z.ready[slot] : &Z.loaded[slot], (unit / P::kUnits) & 1u, abort_flag);
        // the P of the stream's tile before, in S's place, has been used
        if (t >= 2 && ok) ok = warp_wait(&Z.used[w][1], (products[w] + (t >> 1) - 1) & 1u, abort_flag);
        if (!ok) break;
        tmem_fence_after();
        const uint64_t k_desc = matrix_descriptor(smem_addr(units + slot * P::kUnit), 0);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < kDim / 16; ++k) {          // 16 dims are 32 bytes of a row; 64 dims further on the next group
            const uint64_t step = (k >> 2) * (128 * 128 / 16) + (k & 3) * 2;
            product_ss(tmem + 128 * w, q_desc + step, k_desc + step, kDesc, k > 0);
          }
          products_arrive(&Z.scores[w]);
          products_arrive(&Z.free[slot]);
        }
        __syncwarp();
      }
      products[0] += (I.tiles + 1) >> 1;
      products[1] += I.tiles >> 1;
      item_parity ^= 1;
    }
    ok &= products_end(&Z.drained[0]);
  } else if (warp == 14) {
    // ---------------------------------------------------------------- values: O += P V
    constexpr uint32_t kDesc = product_descriptor(kDim, true);
    uint32_t ready_parity = 0;                           // bf16: a bit per slot, moved when a unit was cleared
    uint32_t item_parity = 0, weight_parity[2] = {0, 0};
    uint32_t base = 0;                                   // units before this item's
    for (; ok && walk.next(A, I); base += 2 * I.tiles) {
      if (base > 0) ok = warp_wait(&Z.written, item_parity ^ 1, abort_flag);      // O of the item before has been read
      for (int t = 0; t < I.tiles && ok; ++t) {
        const int w = t & 1;
        const uint32_t unit = base + value_unit(t, I.tiles), slot = unit % P::kUnits, parity = (unit / P::kUnits) & 1u;
        if constexpr (kE4M3) {
          ok = warp_wait(&Z.ready[slot], parity, abort_flag);
        } else {
          ok = warp_wait(&Z.loaded[slot], parity, abort_flag);
          if (ok && (Z.valid[slot][0] & Z.valid[slot][1]) != ~0ull) {
            ok = warp_wait(&Z.ready[slot], (ready_parity >> slot) & 1u, abort_flag);
            ready_parity ^= 1u << slot;
          }
        }
        const uint64_t v_desc = matrix_descriptor(smem_addr(units + slot * P::kUnit), 128 * 128);
#pragma unroll
        for (int h = 0; h < 2 && ok; ++h) {
          ok = warp_wait(&Z.weights[w][h], weight_parity[w], abort_flag);
          if (!ok) break;
          tmem_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < kPrefixTile / 32; ++k)     // 16 tokens: eight columns of P, two kilobytes of V
              product_ts(o_at[w], tmem + 128 * w + 64 * h + k * 8, v_desc + (h * 4 + k) * (2048 / 16), kDesc, t >= 2 || h > 0 || k > 0);
            products_arrive(&Z.used[w][h]);
            if (h == 1) products_arrive(&Z.free[slot]);
            if (h == 1 && t == I.tiles - 1) products_arrive(&Z.done);
          }
          __syncwarp();
        }
        weight_parity[w] ^= 1;
      }
      item_parity ^= 1;
    }
    ok &= products_end(&Z.drained[1]);
  } else if (warp >= 8) {
    // ---------------------------------------------------------------- queries, conversion, clearing
    const int r = (warp & 3) * 32 + lane;
    int slot = 0, raw = 0, filled = 0;
    uint32_t slot_parity = 0, raw_parity = 0, done_parity = 0;
    bool first_item = true;
    while (ok && walk.next(A, I)) {
      // query r: head r % per_kv of the item's row r / per_kv; the sign of the scale goes here, exact, and a scale of zero (an
      // infinity times zero is NaN, as in the formula)
      if (!first_item) {
        ok = warp_wait(&Z.done, done_parity, abort_flag);      // the item before has used Q
        done_parity ^= 1;
      }
      first_item = false;
      if (!ok) break;
      const int row = r / A.per_kv;
      const bool on = row < I.rows;
      const uint4* src = reinterpret_cast<const uint4*>(
          A.q + (on ? __ldcg(A.work.row + I.first + row) : 0) * A.q_stride + (I.head * A.per_kv + r % A.per_kv) * kDim);
      auto put = [&](auto scaled) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          uint4 v = make_uint4(0, 0, 0, 0);
          if (on) {
            v = __ldg(src + c);
            v = make_uint4(scaled(v.x), scaled(v.y), scaled(v.z), scaled(v.w));
          }
          *reinterpret_cast<uint4*>(q_tile + unit_offset(r, c)) = v;
        }
      };
      // (one test for all chunks: a test in each keeps their loads from being in flight together, 5 us)
      const uint32_t flip = A.to_log2 < 0.0f ? 0x80008000u : 0u;
      if (A.to_log2 != 0.0f) put([&](uint32_t w) { return w ^ flip; });
      else put([](uint32_t w) { return times_zero(w); });
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&Z.queries);
      for (int p = 0; p < 2 * I.tiles && ok; ++p) {
        bool is_key;
        int t;
        unit_at(p, I.tiles, is_key, t);
        if constexpr (kE4M3) {
          ok = warp_wait(&Z.loaded[raw], raw_parity, abort_flag);
          if (ok && filled >= P::kUnits) ok = warp_wait(&Z.free[slot], slot_parity ^ 1, abort_flag);
          if (!ok) break;
          const uint8_t* codes = raws + raw * P::kRaw;
          const uint64_t valid = Z.valid[raw][r >> 6];
          const bool on = (valid >> (r & 63)) & 1u;
          // token r: code * 2^(exp - 127), zeros if it is absent.  Every step is exact: code to half, half to float, the product
          // with a power of two, and 4 significant bits as bf16; a NaN stays one.
          const uint32_t e = codes[kPrefixTile * kDim + r];
          const float up = on ? __uint_as_float(e ? e << 23 : 0x400000u) : 0.0f;      // (nothing was copied there)
          const uint32_t there = on ? ~0u : 0u;
          uint8_t* dst = units + slot * P::kUnit;
#pragma unroll
          for (int c = 0; c < kDim / 16; ++c) {            // 16 codes of the row
            uint4 w;
            if constexpr (kDim == 128) w = *reinterpret_cast<const uint4*>(codes + r * 128 + ((c ^ (r & 7)) << 4));
            else w = *reinterpret_cast<const uint4*>(codes + r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
            const uint32_t in[4] = {w.x & there, w.y & there, w.z & there, w.w & there};
            uint32_t out[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const __nv_fp8x2_storage_t two = static_cast<__nv_fp8x2_storage_t>(in[i >> 1] >> (16 * (i & 1)));
              const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3)));
              out[i] = pack_bf16x2(f.x * up, f.y * up);
            }
            *reinterpret_cast<uint4*>(dst + unit_offset(r, 2 * c)) = make_uint4(out[0], out[1], out[2], out[3]);
            *reinterpret_cast<uint4*>(dst + unit_offset(r, 2 * c + 1)) = make_uint4(out[4], out[5], out[6], out[7]);
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&Z.raw_free[raw]);
            mbar_arrive(&Z.ready[slot]);
          }
          ++filled;
          if (++raw == P::kRaws) {
            raw = 0;
            raw_parity ^= 1;
          }
        } else {
          ok = warp_wait(&Z.loaded[slot], slot_parity, abort_flag);
          if (!ok) break;
          if (!is_key && (Z.valid[slot][0] & Z.valid[slot][1]) != ~0ull) {
            if (!((Z.valid[slot][r >> 6] >> (r & 63)) & 1u))
#pragma unroll
              for (int c = 0; c < kChunks; ++c)
                *reinterpret_cast<uint4*>(units + slot * P::kUnit + unit_offset(r, c)) = make_uint4(0, 0, 0, 0);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&Z.ready[slot]);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&Z.free[slot]);
        }
        if (++slot == P::kUnits) {
          slot = 0;
          slot_parity ^= 1;
        }
      }
    }
  } else {
    // ---------------------------------------------------------------- softmax: a row per thread, stream `w`
    const int w = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_row = tmem + 128 * w + lanes;
    const float factor = Z.factor;
    int tile = 0;                                            // the item's first in the block's count
    uint32_t score_parity = 0, item_parity = 0;
    while (ok && walk.next(A, I)) {
      float m = -INFINITY, l = 0.0f;
      for (int t = w; t < I.tiles && ok; t += 2) {
        ok = warp_wait(&Z.scores[w], score_parity, abort_flag);
        if (!ok) break;
        tmem_fence_after();
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          float x[64];
          tmem_load32(s_row + h * 64, x);
          tmem_load32(s_row + h * 64 + 32, x + 32);
          tmem_wait_ld(x);
          const uint64_t valid = Z.tile_valid[(tile + t) & 7][h];
          if (valid != ~0ull) {
#pragma unroll
            for (int i = 0; i < 64; ++i) x[i] = (valid >> i) & 1u ? x[i] : -INFINITY;
          }
          float tops[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) tops[i] = x[i];
#pragma unroll
          for (int i = 4; i < 64; i += 2) tops[(i >> 1) & 3] = max3(tops[(i >> 1) & 3], x[i], x[i + 1]);
          const float top = max3(tops[0], tops[1], fmaxf(tops[2], tops[3])) * factor;
          // move the maximum, and what was summed under the old one, where it is exceeded by more than 8 doublings
          const bool move = top > m + 8.0f;
          if (__any_sync(kFullMask, move)) {
            const float to = move ? top : m;
            const float keep = m == to ? 1.0f : ex2_approx(m - to);
            m = to;
            l *= keep;
            // O as the products before this step left it: the one with this step's predecessor may still be running
            const bool any_before = t >= 2 || h > 0;
            if (any_before) {
              ok = warp_wait(&Z.used[w][h ^ 1], h ? score_parity : score_parity ^ 1, abort_flag);
              if (!ok) break;
              tmem_fence_after();
#pragma unroll
              for (int c = 0; c < kDim / 16; ++c) {
                float y[16];
                tmem_load16(o_at[w] + lanes + c * 16, y);
                tmem_wait_ld(y);
                uint32_t z[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] = __float_as_uint(y[i] * keep);
                tmem_store16(o_at[w] + lanes + c * 16, z);
              }
            }
          }
          const float base = m == -INFINITY ? 0.0f : m;
          float sum[4] = {};
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t p[16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float a = ex2_approx(fmaf(x[c * 32 + i], factor, -base)), b = ex2_approx(fmaf(x[c * 32 + i + 1], factor, -base));
              sum[(i >> 1) & 3] += a + b;
              p[i >> 1] = pack_bf16x2(a, b);
            }
            tmem_store16(s_row + h * 64 + c * 16, p);      // P takes S's place
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          tmem_wait_st();
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&Z.weights[w][h]);
        }
        score_parity ^= 1;
      }
      if (!ok) break;
      tile += I.tiles;
      // ---- the item's end: the even stream joins both and writes the part
      if (w == 1) {
        Z.ml[r] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) mbar_arrive(&Z.odd);
        ok = warp_wait(&Z.written, item_parity, abort_flag);      // before the next item's odd numbers go there
      } else {
        ok = warp_wait(&Z.odd, item_parity, abort_flag) && warp_wait(&Z.done, item_parity, abort_flag);
        if (!ok) break;
        tmem_fence_after();
        const float2 other = Z.ml[r];
        const float to = fmaxf(m, other.x);
        const float keep = m == to ? 1.0f : ex2_approx(m - to), take = I.tiles < 2 ? 0.0f : other.x == to ? 1.0f : ex2_approx(other.x - to);
        const int row = r / A.per_kv, q = r % A.per_kv;
        const bool on = row < I.rows;
        const Work& W = A.work;
        const int64_t at = I.from_before ? static_cast<int64_t>(blockIdx.x) * kPrefixQueries + r
                                         : static_cast<int64_t>(I.first + row) * A.n_q_heads + I.head * A.per_kv + q;
        float* dst = (I.from_before ? W.extra_o : W.prefix_o) + at * kDim;
        if (on) (I.from_before ? W.extra_ml : W.prefix_ml)[at] = make_float2(to, l * keep + other.y * take);
#pragma unroll
        for (int c = 0; c < kDim / 32; ++c) {
          float x[32];
          tmem_load32(o_at[0] + lanes + c * 32, x);
          tmem_wait_ld(x);
          if (I.tiles > 1) {
            float y[32];
            tmem_load32(o_at[1] + lanes + c * 32, y);
            tmem_wait_ld(y);
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = x[i] * keep + y[i] * take;
          }
          if (on) {
#pragma unroll
            for (int i = 0; i < 32; i += 8) store_sector(dst + c * 32 + i, x + i);
          }
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&Z.written);
      }
      item_parity ^= 1;
    }
  }
  if (!ok) {
    *abort_flag = 1;
    bad |= ESPO_DEV_TIMEOUT;
  }
  if (bad && lane == 0 && A.status_out) atomicOr(A.status_out, bad);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (warp == 13) tmem_free(tmem, kTmemColumns);
}

}  // namespace
}  // namespace espo
