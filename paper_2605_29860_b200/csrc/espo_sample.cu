// Sampling from given random numbers with per-row temperature, top-k, top-p and min-p.
//
// Mathematics.  w_a = exp((x_a - M) / T) in 64 bits, kept as an integer multiple of 2^-42: sums of integers do not depend on
// their order, and a comparison next to a border (a mass against top_p Z, a running sum against u W) is decided by 42 bits.
// The support is a threshold on the logit: mass and number of strictly larger logits grow as the logit falls, so the ids
// that pass top_p, top_k and min_p are those at or above one value, the "floor", of an order-preserving key.
//
// Work split, three kernels, each set up while the one before it winds down:
//   chunk  a block per 16384 bf16 or 8192 fp32 ids, held in registers from the one read of HBM on: largest logit; the sum of
//          weights relative to it, in 64 bits, for rows that need one (top_p, or no filter at all); and, for rows with a
//          filter, the ids at or above the chunk's own cut, in order.  The cut is the lowest, among the warps, of the values
//          that a few of the lanes reach, so the list is short (about 600 ids a row) and complete down to the cut.
//   row    a block per row: finds the floor among the listed ids by bisection and draws.  Rows whose support reaches below
//          some chunk's cut (wide supports) are left to the third kernel.
//   wide   clusters of eight blocks sweep such rows again, from L2: a histogram of counts over 1/32nds of a doubling of the
//          weight brackets the floor, then histograms of exact masses over ever shorter ranges of keys (1024 bins) find it.
// Every path ends at the same floor and token.
//
// What bounds it: HBM, one read of the logits; for 64-bit sums the 64-bit pipe (13 operations an id, 64 a clock and SM), which
// is why ids are only summed where a sum is needed; issue slots are scarcer still (39 an id, 72 % taken), so a logit becomes a
// double by the conversion instruction, not by four integer ones (200 x 151669 fp32: 58.0 -> 53.7 us).  With top_k or min_p alone
// nothing is summed in 64 bits, and a block's own chain bounds it (one load of its chunk, the search for its cut, two to four
// barriers, the list, the listed logits read again), the other three blocks of its SM being all that hides it.  512 rows of
// 152064 bf16 ids: 64 us with top_k alone, 62 with min_p, 101 without a filter, the mode 32; mixed filters 92 us in the first
// kernel (64-bit pipe 43 % active, issuing 62 %), 15 in the second, 58 in the third, which its sweeps' latency bounds (issuing
// 11 %; at 64 registers a thread it spills 378 bytes); 512 wide supports 730 us.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "espo.h"
#include "espo_device.cuh"
#include "espo_host.h"

namespace espo {
namespace {

namespace cg = cooperative_groups;

constexpr double kOne = 4398046511104.0;    // 2^42
constexpr int kMaxVocab = 1 << 19;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxChunks = 64;              // of 8192 fp32 or 16384 bf16 ids
constexpr int kListTotal = 2048;            // ids that all chunks' lists of a row hold together
constexpr int kPerThread = 4;               // listed ids per thread when a floor is sought
constexpr int kListed = kThreads * kPerThread;
constexpr int kCluster = 8;                 // with four, some 120 wide rows of 152064 ids took 104 us, not 57, and 512 of them 579, not 730
constexpr int kClusters = 74;               // of the third kernel: four blocks on every SM
constexpr int kParts = kCluster * kWarps / 32;      // of the cluster's warps, per lane of one
constexpr int kMaxRows = 2048;              // rows per three launches: what the workspace is sized for
constexpr int kNear = 128;                  // keys a warp keeps of a bracket
constexpr int kBins = 1024;
constexpr float kBinsPerUnit = 32.0f;       // bins per doubling of the weight
constexpr int kMaxRounds = 16;              // of sweeps: a histogram, a guessed bracket, then at most four times 10 bits of key
struct ChunkStat {
  double sum[kWarps];      // of exp((x - max) / T) over each eighth of the chunk; 0 if the row needs none
  float max;               // NaN if the chunk holds one
  int32_t listed;          // ids in the chunk's list
  uint32_t cut;            // every id of the chunk at or above this key is listed
  uint32_t pad;
};

struct Listed {
  uint32_t key;
  int32_t id;
};

// What the second kernel leaves to the third.
struct Order {
  int action;
  uint32_t lo, hi;        // kZoom: keys [lo, hi), in bins of 2^shift keys; kDraw: the floor lo
  int shift;
  int sum_above;          // kZoom: whether the mass at or above hi is wanted too
};
struct WideRow {
  int32_t in_batch;
  Order order;
};

struct SampleArgs {
  const void* logits;
  int64_t row_stride;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t *top_k, *row_ids;
  const uint8_t* status;
  int32_t* tokens_out;
  float* logp_out;
  uint32_t* status_out;
  ChunkStat* stats;          // [rows][chunks]
  Listed* lists;             // [rows][chunks][list_cap]
  unsigned* n_wide;          // [1]
  WideRow* wide;             // [rows]
  int32_t row0, V, capacity;
  int32_t chunks, list_cap;
  int32_t cut_rank;          // how many of a warp's lanes reach its cut with their largest logit; above 32: list all ids
  int32_t warp_pieces;       // 16-byte pieces per warp of a chunk, at most 32 * kPieces
  int32_t slice;             // ids per block of a cluster, a multiple of 8
};

// An order-preserving key: larger key = larger logit; -0 and +0 share one.  16 bits say all about a bf16 logit.
template <typename T>
struct Key;
template <>
struct Key<float> {
  static constexpr uint32_t kLowest = 0x00800000u;      // of the lowest finite number; -inf lies below
  static constexpr int kCoarse = 16;                    // low bits that a chunk's cut leaves out
  static __device__ __forceinline__ uint32_t of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ ((b & 0x80000000u) ? 0xffffffffu : 0x80000000u);
  }
  static __device__ __forceinline__ float value(uint32_t key) {
    return __uint_as_float(key ^ ((key & 0x80000000u) ? 0x80000000u : 0xffffffffu));
  }
};
template <>
struct Key<__nv_bfloat16> {
  static constexpr uint32_t kLowest = 0x0080u;
  static constexpr int kCoarse = 0;
  static __device__ __forceinline__ uint32_t of(float x) { return Key<float>::of(x) >> 16; }
  static __device__ __forceinline__ float value(uint32_t key) {
    return __uint_as_float((key & 0x8000u ? key ^ 0x8000u : key ^ 0xffffu) << 16);
  }
};

// 2^t for t = d c in [-1000, 1]: t = n + f with |f| <= 1/2; 2^f by a polynomial of degree 8, 1 + f q(f) with q through
// (2^f - 1) / f at the eight Chebyshev nodes of [-1/2, 1/2]: relative error below 2^-38.7, none at f = 0.
__device__ __forceinline__ double power_of_two(double d, double c) {
  constexpr double kShift = 6755399441055744.0;                           // 1.5 * 2^52: adding it rounds to an integer
  const double shifted = fma(d, c, kShift);
  const int n = __double2loint(shifted);
  const double f = fma(d, c, -(shifted - kShift));
  double p = fma(1.325080551750225e-06, f, 1.5303700711365693e-05);
  p = fma(p, f, 0.00015403475186530786);
  p = fma(p, f, 0.0013333478473685416);
  p = fma(p, f, 0.00961812913523614);
  p = fma(p, f, 0.055504109063258665);
  p = fma(p, f, 0.24022650695888503);
  p = fma(p, f, 0.6931471805568324);
  p = fma(p, f, 1.0);
  return __hiloint2double(__double2hiint(p) + n * 1048576, __double2loint(p));
}

// Weights exp((x - top) / T) of a row or a part of it: 2^((x - top) c).
struct Weights {
  double top, c;
  float least;            // logits below weigh at most 2^-200, and are taken as this one to keep the exponent in range
  __device__ __forceinline__ void set(float largest, float temperature) {
    // A temperature so low that the next float below the largest logit weighs nothing stays in range too.
    const uint32_t b = __float_as_uint(largest);
    const float below = largest == 0.0f ? -1e-37f : __uint_as_float(largest > 0.0f ? b - 1 : b + 1);
    const double gap = static_cast<double>(largest) - below;
    c = fmin(1.4426950408889634 / static_cast<double>(temperature), 900.0 / gap);
    least = fmaxf(static_cast<float>(fmin(static_cast<double>(largest) - 200.0 / c, static_cast<double>(below))), -3.402823466e38f);
    top = static_cast<double>(largest);
  }
  __device__ __forceinline__ double operator()(float x) const { return power_of_two(static_cast<double>(fmaxf(x, least)) - top, c); }
  // in units of 2^-42
  __device__ __forceinline__ uint64_t fixed(float x) const {
    return static_cast<uint64_t>(__double_as_longlong(fma((*this)(x), kOne, 4503599627370496.0))) & 0xfffffffffffffull;   // + 2^52
  }
};

template <typename T> struct Vec;
template <> struct Vec<float> { static constexpr int kN = 4; };
template <> struct Vec<__nv_bfloat16> { static constexpr int kN = 8; };

__device__ __forceinline__ void unpack(const float*, const uint4& v, float (&x)[4]) {
  x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void unpack(const __nv_bfloat16*, const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(w[i]);
    x[2 * i + 1] = bf16_hi(w[i]);
  }
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float c;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(a), "f"(b));
  return c;
}
// Largest of a 16-byte piece; NaN if one is.
__device__ __forceinline__ float piece_max(const float*, const uint4& v) {
  return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
}
__device__ __forceinline__ float piece_max(const __nv_bfloat16*, const uint4& v) {
  uint32_t a, b;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
  return max_nan(bf16_lo(a), bf16_hi(a));
}

__device__ __forceinline__ uint32_t raw(float x) { return __float_as_uint(x); }
__device__ __forceinline__ uint32_t raw(__nv_bfloat16 x) { return __bfloat16_as_ushort(x); }

// A piece of -inf.
__device__ __forceinline__ uint4 lowest_piece(const float*) { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
__device__ __forceinline__ uint4 lowest_piece(const __nv_bfloat16*) { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }

// Ids [p * kN, (p + 1) * kN) of a row, -inf beyond its end.  `whole`: the row starts on a 16-byte boundary.
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* row, int p, int V, bool whole) {
  constexpr int kN = Vec<T>::kN;
  if (whole && (p + 1) * kN <= V) return __ldg(reinterpret_cast<const uint4*>(row) + p);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kN == 4) {
      w[i] = p * 4 + i < V ? raw(row[p * 4 + i]) : 0xff800000u;
    } else {
      const int a = p * 8 + 2 * i;
      w[i] = (a < V ? raw(row[a]) : 0xff80u) | ((a + 1 < V ? raw(row[a + 1]) : 0xff80u) << 16);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

struct RowParams {
  float u, temperature, top_p, min_p;      // top_p 2, min_p 0: no filter
  uint32_t top_k;                          // 2^31: no filter
  bool fine, greedy;
};
__device__ __forceinline__ RowParams row_params(const SampleArgs& A, int r) {
  RowParams P;
  P.temperature = A.temperature ? A.temperature[r] : 1.0f;
  P.u = A.u[r];
  const float p = A.top_p ? A.top_p[r] : 1.0f;
  P.top_p = p > 0.0f && p < 1.0f ? p : 2.0f;
  const int k = A.top_k ? A.top_k[r] : 0;
  P.top_k = k > 0 && k < A.V ? static_cast<uint32_t>(k) : 1u << 31;
  const float m = A.min_p ? A.min_p[r] : 0.0f;
  P.min_p = m > 0.0f && m <= 1.0f ? m : 0.0f;
  P.greedy = P.temperature == 0.0f;
  P.fine = P.u >= 0.0f && P.u < 1.0f && P.temperature >= 0.0f && P.temperature <= 1e30f;
  return P;
}
// Whether the row takes part; false with a slot outside the state too.
__device__ __forceinline__ bool row_active(const SampleArgs& A, int r, bool& bad_slot) {
  bad_slot = false;
  if (!A.status) return true;
  const int slot = A.row_ids ? A.row_ids[r] : r;
  bad_slot = slot < 0 || slot >= A.capacity;
  return !bad_slot && A.status[slot] == ESPO_ROW_ACTIVE;
}

// ---------------------------------------------------------------------------------------------- chunks

// Which of a piece's ids reach the cut: bit i for id i.
__device__ __forceinline__ uint32_t reach(const float*, const uint4& v, float cut) {
  return (__uint_as_float(v.x) >= cut ? 1u : 0u) | (__uint_as_float(v.y) >= cut ? 2u : 0u) |
         (__uint_as_float(v.z) >= cut ? 4u : 0u) | (__uint_as_float(v.w) >= cut ? 8u : 0u);
}
__device__ __forceinline__ uint32_t reach(const __nv_bfloat16*, const uint4& v, float cut) {
  const __nv_bfloat162 c = __float2bfloat162_rn(cut);      // the cut is a bf16
  auto ge = [&](uint32_t w) { return __hge2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w), c); };
  const uint32_t m = (ge(v.x) & 0x00020001u) | (ge(v.y) & 0x00080004u) | (ge(v.z) & 0x00200010u) | (ge(v.w) & 0x00800040u);
  return (m | (m >> 16)) & 0xffu;
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

constexpr int kPieces = 8;      // 16-byte pieces per thread
template <typename T>
constexpr int kChunk = kThreads * kPieces * Vec<T>::kN;

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) chunk_kernel(const SampleArgs A) {
  constexpr int kN = Vec<T>::kN;
  using K = Key<T>;
  __shared__ float s_max[kWarps];
  __shared__ uint32_t s_cut[kWarps];
  __shared__ int s_id[kListTotal];      // a list's ids: at most list_cap
  __shared__ int s_count[2][kWarps];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int r = A.row0 + static_cast<int>(blockIdx.x / A.chunks), chunk = static_cast<int>(blockIdx.x % A.chunks);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const T* row = static_cast<const T*>(A.logits) + static_cast<int64_t>(r) * A.row_stride;
  const bool whole = reinterpret_cast<uintptr_t>(row) % 16 == 0;
  if (blockIdx.x == 0 && tid == 0) *A.n_wide = 0;
  bool bad_slot;
  if (!row_active(A, r, bad_slot)) return;

  uint4 v[kPieces];
  const int p0 = (chunk * kWarps + warp) * A.warp_pieces + lane;      // a warp's pieces lie together
  if (whole && (chunk + 1) * kWarps * A.warp_pieces * kN <= A.V) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
      v[j] = j * 32 + lane < A.warp_pieces ? __ldg(reinterpret_cast<const uint4*>(row) + p0 + j * 32) : lowest_piece(row);
  } else {
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
      v[j] = j * 32 + lane < A.warp_pieces ? load_piece(row, p0 + j * 32, A.V, whole) : lowest_piece(row);
  }
  const RowParams P = row_params(A, r);

  float mine = piece_max(row, v[0]);
#pragma unroll
  for (int j = 1; j < kPieces; ++j) mine = max_nan(mine, piece_max(row, v[j]));
  const bool filtered = P.top_p <= 1.0f || P.top_k < (1u << 31) || P.min_p > 0.0f;
  float m = mine;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(kFullMask, m, o));
  uint32_t warp_cut = K::kLowest >> K::kCoarse;
  if (filtered && A.cut_rank <= 32) {
    // largest coarse key that cut_rank of the warp's lanes reach with their largest logit
    const uint32_t key = K::of(mine) >> K::kCoarse;
    uint32_t yes = __reduce_min_sync(kFullMask, key), no = __reduce_max_sync(kFullMask, key) + 1;
    while (no - yes > 1) {
      const uint32_t probe = yes + (no - yes) / 2;
      if (__popc(__ballot_sync(kFullMask, key >= probe)) >= A.cut_rank) yes = probe;
      else no = probe;
    }
    warp_cut = max(yes, warp_cut);
  }
  if (lane == 0) {
    s_max[warp] = m;
    s_cut[warp] = warp_cut;
  }
  __syncthreads();
  m = s_max[0];
  uint32_t cut = s_cut[0], high_cut = s_cut[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) {
    m = max_nan(m, s_max[w]);
    cut = min(cut, s_cut[w]);
    high_cut = max(high_cut, s_cut[w]);
  }
  cut <<= K::kCoarse;
  high_cut <<= K::kCoarse;
  const bool usable = P.fine && !P.greedy && m > -INFINITY && m < INFINITY;
  const bool listing = usable && filtered, summing = usable && (P.top_p <= 1.0f || !filtered);

  double sum = 0.0;
  if (summing) {
    Weights weight;
    weight.set(m, P.temperature);
    double s[2] = {0.0, 0.0};
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      float x[kN];
      unpack(row, v[j], x);
#pragma unroll
      for (int i = 0; i < kN; ++i) s[i & 1] += weight(x[i]);
    }
    sum = s[0] + s[1];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFullMask, sum, o);
  }
  int listed = 0;
  if (listing) {
    // ids at or above the cut, in order: warp by warp, piece by piece, lane by lane; the highest of the warps' cuts if the
    // lowest lists too many
    uint32_t hits[kPieces];
    int before[kPieces];      // of the lane's hits, within the warp
    int mine_from = 0;
    for (int attempt = 0; attempt < 2; ++attempt) {
      const float cut_x = K::value(cut);
      const bool any = mine >= cut_x;
      int total = 0;
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        hits[j] = any ? reach(row, v[j], cut_x) : 0u;
        const unsigned some = __ballot_sync(kFullMask, hits[j] != 0), more = __ballot_sync(kFullMask, (hits[j] & (hits[j] - 1)) != 0);
        before[j] = total;
        if (more) {             // some lane holds several
          const int c = __popc(hits[j]);
          int upto = c;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int n = __shfl_up_sync(kFullMask, upto, o);
            if (lane >= o) upto += n;
          }
          before[j] += upto - c;
          total += __shfl_sync(kFullMask, upto, 31);
        } else {
          before[j] += __popc(some & ((1u << lane) - 1u));
          total += __popc(some);
        }
      }
      if (lane == 0) s_count[attempt][warp] = total;
      __syncthreads();
      mine_from = listed = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const int n = s_count[attempt][w];
        if (w < warp) mine_from += n;
        listed += n;
      }
      if (listed <= A.list_cap || cut == high_cut) break;
      cut = high_cut;
    }
    if (listed > A.list_cap) {
      listed = 0;                  // too many equal logits at the cut: no list, and nothing is known to be listed
      cut = 0xffffffffu;
    } else {
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        uint32_t h = hits[j];
        int to = mine_from + before[j];
        while (h) {
          s_id[to++] = (p0 + j * 32) * kN + __ffs(h) - 1;
          h &= h - 1;
        }
      }
      __syncthreads();
      Listed* list = A.lists + (static_cast<int64_t>(r - A.row0) * A.chunks + chunk) * A.list_cap;
      for (int e = tid; e < listed; e += kThreads) {
        const int id = s_id[e];
        list[e] = Listed{K::of(to_float(row[id])), id};
      }
    }
  }
  ChunkStat* stat = A.stats + static_cast<int64_t>(r - A.row0) * A.chunks + chunk;
  if (lane == 0) stat->sum[warp] = sum;
  if (tid == 0) {
    stat->max = m;
    stat->listed = listed;
    stat->cut = m == -INFINITY ? 0u : listing ? cut : 0xffffffffu;
  }
}

// ---------------------------------------------------------------------------------------------- rows

enum Action : int { kDone, kHistogram, kZoom, kDraw };

// The order for keys [lo, hi).
__device__ __forceinline__ Order zoom(uint32_t lo, uint32_t hi, bool sum_above) {
  int shift = 0;
  while ((hi - lo - 1) >> shift >= static_cast<uint32_t>(kBins)) ++shift;
  return {kZoom, lo, hi, shift, sum_above ? 1 : 0};
}

struct Crossing {
  uint64_t mass;          // at or above the bin's end
  uint32_t count;
  int32_t bin;            // -1: none
};

// A block's shared memory; peers of the cluster read it, the first block writes the order.
struct Shared {
  union {
    struct {
      unsigned long long mass[kBins];
      uint32_t count[kBins];
    };
    Listed compact[kListed];
  };
  uint64_t above_mass[kWarps];      // exact mass and number at or above the bracket
  uint32_t above_count[kWarps];
  uint64_t exact_sum[kWarps];
  float queue[kWarps][64];
  uint32_t near[kWarps][kNear];     // keys inside the bracket
  int32_t n_near[kWarps];
  Order order;
  Crossing crossing;
  int32_t starts[kMaxChunks + 1];
  int32_t max_id;         // lowest id found: of the largest logit, or by a draw from the sums
  int32_t bin_crossed, bin_clear;
  uint64_t scratch64[kWarps];
  uint32_t scratch32[kWarps];
  float scratch_f[kWarps];
};

__device__ __forceinline__ uint64_t warp_sum64(uint64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFullMask, v, o);
  return v;
}

template <typename V>
__device__ __forceinline__ V warp_scan(V v) {      // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V n = __shfl_up_sync(kFullMask, v, o);
    if ((threadIdx.x & 31) >= o) v += n;
  }
  return v;
}

// Sums over the block, the same for every thread.
__device__ __forceinline__ void block_sum(uint64_t& mass, uint32_t& count, Shared& S) {
  mass = warp_sum64(mass);
  count = __reduce_add_sync(kFullMask, count);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) {
    S.scratch64[threadIdx.x >> 5] = mass;
    S.scratch32[threadIdx.x >> 5] = count;
  }
  __syncthreads();
  mass = 0;
  count = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    mass += S.scratch64[w];
    count += S.scratch32[w];
  }
}

// Per-row numbers that every thread of the cluster holds alike.
struct Row {
  int r;
  float top;              // largest logit
  float k;                // log2(e) / T
  Weights weight;
  double inv_t;
  double z;               // sum of weights
  double top_p;           // > 1: no filter
  uint32_t top_k;         // no filter: 2^31
  uint32_t min_key;       // floor of min_p, or the lowest finite key
  uint32_t top_key;
  double u;
  bool bounded;           // by top_p or top_k
  // log-probability of an id among ids of weight `total`
  __device__ __forceinline__ float logp(float x, double total) const {
    return static_cast<float>((static_cast<double>(x) - top) * inv_t - log(total));
  }
  // whether a level with this mass and number of strictly larger logits passes top_p and top_k
  __device__ __forceinline__ bool passes(uint64_t mass, uint32_t count) const {
    return count < top_k && (top_p > 1.0 || static_cast<double>(mass) < top_p * z * kOne);
  }
};

// Ids in id order, kPerThread a thread; id -1: none.
struct List {
  uint32_t key[kPerThread];
  uint64_t f[kPerThread];
  int id[kPerThread];
};

// The list holds every id at or above lo.  Finds the smallest key at which a level would pass top_p and top_k, the ids
// strictly above it being few and light enough; false if levels below lo pass too (and lo is not the lowest possible floor).
__device__ __forceinline__ bool find_floor(const List& L, const Row& R, uint32_t lo, uint32_t& floor_key, Shared& S) {
  uint64_t mass = 0;
  uint32_t count = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i)
    if (L.id[i] >= 0) {
      ++count;
      mass += L.f[i];
    }
  block_sum(mass, count, S);
  if (R.passes(mass, count)) {      // a level just below lo
    floor_key = lo;
    return lo == R.min_key;
  }
  uint32_t pass_key = R.top_key, fail_key = lo - 1;
  while (pass_key - fail_key > 1) {
    const uint32_t mid = fail_key + (pass_key - fail_key) / 2;
    mass = 0;
    count = 0;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
      if (L.id[i] >= 0 && L.key[i] > mid) {
        ++count;
        mass += L.f[i];
      }
    block_sum(mass, count, S);
    if (R.passes(mass, count)) pass_key = mid;
    else fail_key = mid;
  }
  floor_key = pass_key;
  return true;
}

__device__ __forceinline__ void emit(const SampleArgs& A, int r, int id, float logp) {
  A.tokens_out[r] = id;
  if (A.logp_out) A.logp_out[r] = logp;
}

// Draws among the listed ids at or above the floor: the whole support.
template <typename T>
__device__ __forceinline__ void draw_listed(const SampleArgs& A, List& L, const Row& R, uint32_t floor_key, Shared& S) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t own = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    if (L.id[i] < 0 || L.key[i] < floor_key) L.f[i] = 0;
    own += L.f[i];
  }
  const uint64_t upto = warp_scan(own);
  __syncthreads();
  if (lane == 31) S.scratch64[warp] = upto;
  __syncthreads();
  uint64_t total = 0, before = upto - own;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += S.scratch64[w];
    total += S.scratch64[w];
  }
  const double target = R.u * static_cast<double>(total);
  if (static_cast<double>(before) <= target && target < static_cast<double>(before + own)) {      // one thread
    bool taken = false;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      before += L.f[i];
      if (!taken && L.f[i] && target < static_cast<double>(before)) {
        taken = true;
        emit(A, R.r, L.id[i], R.logp(Key<T>::value(L.key[i]), static_cast<double>(total) / kOne));
      }
    }
  }
}

// Entry i of a List becomes v, if its key is at or above lo.
template <typename T>
__device__ __forceinline__ void put_entry(List& L, const Row& R, int i, bool on, const Listed& v) {
  L.key[i] = on ? v.key : 0;
  L.id[i] = on ? v.id : -1;
  L.f[i] = on ? R.weight.fixed(Key<T>::value(v.key)) : 0;
}

// Which of the 64 segments whose running starts stand in S.starts holds entry e.
__device__ __forceinline__ int segment_of(const Shared& S, int e) {
  int s = 0;
#pragma unroll
  for (int step = 32; step > 0; step >>= 1)
    if (S.starts[s + step] <= e) s += step;
  return s;
}

// Writes the running starts of 64 counts, two a lane (every warp holds them alike), and returns their sum.
__device__ __forceinline__ int put_starts(int c0, int c1, Shared& S) {
  const int lane = threadIdx.x & 31;
  const int upto0 = warp_scan(c0), half = __shfl_sync(kFullMask, upto0, 31);
  const int upto1 = half + warp_scan(c1), sum = __shfl_sync(kFullMask, upto1, 31);
  if (threadIdx.x < 32) {
    S.starts[lane] = upto0 - c0;
    S.starts[32 + lane] = upto1 - c1;
    if (lane == 31) S.starts[kMaxChunks] = sum;
  }
  __syncthreads();
  return sum;
}

// A block's part of the row: pieces of 16 bytes, a warp's range of them contiguous.
template <typename T>
struct Slice {
  const T* row;
  int V;
  bool whole;
  int first, count;       // the block's pieces
  __device__ __forceinline__ uint4 piece(int p) const { return load_piece(row, p, V, whole); }
  __device__ __forceinline__ int begin(int warp) const { return first + static_cast<int>(static_cast<int64_t>(count) * warp / kWarps); }
};

// Calls f(piece, its 16 bytes, whether it exists) for the pieces [begin, end) in groups of 32, lane by lane; four groups'
// loads are in flight at a time.
template <typename T, typename F>
__device__ __forceinline__ void sweep(const Slice<T>& L, int begin, int end, F f) {
  constexpr int kBatch = 4;
  const int lane = threadIdx.x & 31;
  for (int base = begin; base < end; base += 32 * kBatch) {
    uint4 v[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int p = base + j * 32 + lane;
      v[j] = p < end ? L.piece(p) : lowest_piece(L.row);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (base + j * 32 < end) f(base + j * 32 + lane, v[j]);
  }
}

// Calls f(logit, whether there is one) for the logits at or above floor_x in pieces [begin, end), 32 at a time: the few that
// matter are brought together in the warp's queue first, so that 64-bit arithmetic is not spent on lanes without one.  Their
// order is of no account to sums of integers.
template <typename T, typename F>
__device__ __forceinline__ void sweep_dense(const Slice<T>& L, int begin, int end, float floor_x, float* queue, F f) {
  const int lane = threadIdx.x & 31;
  int waiting = 0;
  __syncwarp();
  sweep(L, begin, end, [&](int, const uint4& v) {
    if (!__any_sync(kFullMask, piece_max(L.row, v) >= floor_x)) return;
    float x[Vec<T>::kN];
    unpack(L.row, v, x);
#pragma unroll
    for (int i = 0; i < Vec<T>::kN; ++i) {
      const bool on = x[i] >= floor_x;
      const unsigned who = __ballot_sync(kFullMask, on);
      if (on) queue[waiting + __popc(who & ((1u << lane) - 1u))] = x[i];
      waiting += __popc(who);
      if (waiting >= 32) {
        __syncwarp();
        const float first = queue[lane], second = queue[32 + lane];
        __syncwarp();
        waiting -= 32;
        if (lane < waiting) queue[lane] = second;
        __syncwarp();                // the next logit may be put there by another lane
        f(first, true);
      }
    }
  });
  __syncwarp();
  f(lane < waiting ? queue[lane] : 0.0f, lane < waiting);
  __syncwarp();
}

// Exact mass of the ids at or above the floor in pieces [begin, end) (the whole warp gets it).
template <typename T>
__device__ __forceinline__ uint64_t exact_mass(const Slice<T>& L, const Row& R, uint32_t floor_key, int begin, int end, float* queue) {
  uint64_t s = 0;
  sweep_dense(L, begin, end, Key<T>::value(floor_key), queue, [&](float x, bool on) {
    const uint64_t f = R.weight.fixed(x);
    s += on ? f : 0;
  });
  return warp_sum64(s);
}

// The row swept again by its cluster, order after order; the first block keeps the search.
template <typename T>
__device__ __forceinline__ void sweep_row(const SampleArgs& A, const Row& R, Order now, Shared& S) {
  constexpr int kN = Vec<T>::kN;
  using K = Key<T>;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank());
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Slice<T> L;
  L.row = static_cast<const T*>(A.logits) + static_cast<int64_t>(R.r) * A.row_stride;
  L.V = A.V;
  L.whole = reinterpret_cast<uintptr_t>(L.row) % 16 == 0;
  L.first = min(rank * (A.slice / kN), (A.V + kN - 1) / kN);
  L.count = min((rank + 1) * (A.slice / kN), (A.V + kN - 1) / kN) - L.first;
  uint32_t low = R.min_key, high = R.top_key + 1;      // first block: the floor lies in [low, high)
  uint64_t base_mass = 0;                              // and what lies at or above the bracket, once it is known
  uint32_t base_count = 0;
  uint64_t warp_above = 0;                             // this warp's exact mass at or above above_key; S.near holds its keys
  uint32_t above_key = 0, above_low = 0;               // in [above_low, above_key)
  for (int round = 0; now.action == kHistogram || now.action == kZoom; ++round) {
    // ---- every block carries the order out on its slice
    for (int b = tid; b < kBins; b += kThreads) {
      S.count[b] = 0;
      S.mass[b] = 0;
    }
    __syncthreads();
    if (now.action == kHistogram) {
      const float scale = R.k * kBinsPerUnit;
      sweep(L, L.begin(warp), L.begin(warp + 1), [&](int, const uint4& v) {
        float x[kN];
        unpack(L.row, v, x);
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          const float d = (R.top - x[i]) * scale;
          if (d < static_cast<float>(kBins)) atomicAdd(&S.count[static_cast<int>(d)], 1u);
        }
      });
    } else {
      const float lo_x = K::value(now.lo), hi_x = K::value(now.hi);
      uint64_t above = 0;
      uint32_t n_above = 0;
      if (now.sum_above && lane == 0) S.n_near[warp] = 0;
      __syncwarp();
      auto bin = [&](float x, uint64_t f) {
        const uint32_t key = K::of(x), b = (key - now.lo) >> now.shift;
        atomicAdd(&S.count[b], 1u);
        atomicAdd(&S.mass[b], static_cast<unsigned long long>(f));
        if (now.sum_above) {            // kept for the draw
          const int at = atomicAdd(&S.n_near[warp], 1);
          if (at < kNear) S.near[warp][at] = key;
        }
      };
      if (now.sum_above) {
        sweep_dense(L, L.begin(warp), L.begin(warp + 1), lo_x, S.queue[warp], [&](float x, bool on) {
          const uint64_t f = R.weight.fixed(x);
          if (on && x >= hi_x) {
            above += f;
            ++n_above;
          } else if (on) {
            bin(x, f);
          }
        });
      } else {
        sweep(L, L.begin(warp), L.begin(warp + 1), [&](int, const uint4& v) {
          if (!__any_sync(kFullMask, piece_max(L.row, v) >= lo_x)) return;
          float x[kN];
          unpack(L.row, v, x);
#pragma unroll
          for (int i = 0; i < kN; ++i)
            if (x[i] >= lo_x && x[i] < hi_x) bin(x[i], R.weight.fixed(x[i]));
        });
      }
      if (now.sum_above) {
        above = warp_sum64(above);
        n_above = __reduce_add_sync(kFullMask, n_above);
        warp_above = above;
        above_key = now.hi;
        above_low = now.lo;
        if (lane == 0) {
          S.above_mass[warp] = above;
          S.above_count[warp] = n_above;
        }
      }
    }
    cluster.sync();
    // each block adds up its share of the bins and hands the sums to the first
    {
      constexpr int kShare = kBins / kCluster;
      uint32_t count = 0;
      unsigned long long mass = 0;
      const int b = rank * kShare + tid;
      if (tid < kShare) {
#pragma unroll
        for (int c = 0; c < kCluster; ++c) {
          const Shared* P = cluster.map_shared_rank(&S, c);
          count += P->count[b];
          mass += P->mass[b];
        }
      }
      cluster.sync();
      if (tid < kShare) {
        Shared* F = cluster.map_shared_rank(&S, 0);
        F->count[b] = count;
        F->mass[b] = mass;
      }
      cluster.sync();
    }

    // ---- the first block looks at the sums
    if (rank == 0) {
      Order next = {kDone, 0, 0, 0, 0};
      constexpr int kOwn = kBins / kThreads;
      if (now.action == kHistogram) {
        // Number and mass of the ids above each thread's bins, the masses at the bins' centres: off by 1.1 % at most, and the
        // bracket is wide enough for that.
        float mass = 0.0f;
        uint32_t count = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const uint32_t c = S.count[tid * kOwn + i];
          count += c;
          mass += c * ex2_approx(-(tid * kOwn + i + 0.5f) / kBinsPerUnit);
        }
        const float mass_upto = warp_scan(mass);
        const uint32_t count_upto = warp_scan(count);
        if (lane == 31) {
          S.scratch_f[warp] = mass_upto;
          S.scratch32[warp] = count_upto;
        }
        if (tid == 0) {
          S.bin_crossed = kBins;       // first bin by whose end a border has been crossed
          S.bin_clear = 0;             // last bin at whose start none has
        }
        __syncthreads();
        mass = mass_upto - mass;
        count = count_upto - count;
        for (int w = 0; w < warp; ++w) {
          mass += S.scratch_f[w];
          count += S.scratch32[w];
        }
        const float limit = static_cast<float>(R.top_p * R.z);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const int b = tid * kOwn + i;
          const uint32_t c = S.count[b];
          if (count < R.top_k && (R.top_p > 1.0 || mass < limit * 0.985f)) atomicMax(&S.bin_clear, b);
          count += c;
          mass += c * ex2_approx(-(b + 0.5f) / kBinsPerUnit);
          if (count >= R.top_k || (R.top_p <= 1.0 && mass >= limit * 1.015f)) atomicMin(&S.bin_crossed, b);
        }
        __syncthreads();
        const int b1 = S.bin_crossed, b0 = S.bin_clear;
        // bin b holds (top - x) k 32 in [b, b + 1); a bin more on either side covers the rounding of that product
        const double unit = 1.0 / (R.weight.c * kBinsPerUnit);
        uint32_t lo = b1 >= kBins ? low : K::of(static_cast<float>(fmax(R.top - (b1 + 2) * unit, -3.0e38)));
        uint32_t hi = b0 <= 1 ? high : K::of(static_cast<float>(fmax(R.top - (b0 - 1) * unit, -3.0e38)));
        lo = min(max(lo, low), high - 1);
        hi = min(max(hi, lo + 1), high);
        next = zoom(lo, hi, true);
      } else {
        if (now.sum_above) {
          uint64_t above = 0;
          uint32_t n_above = 0;
#pragma unroll
          for (int i = 0; i < kParts; ++i) {
            const int w = lane * kParts + i;
            const Shared* P = cluster.map_shared_rank(&S, w / kWarps);
            above += P->above_mass[w % kWarps];
            n_above += P->above_count[w % kWarps];
          }
          base_mass = warp_sum64(above);
          base_count = __reduce_add_sync(kFullMask, n_above);
        }
        // bins from the highest keys down: what lies above each of the thread's
        uint64_t mass = 0;
        uint32_t count = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          mass += S.mass[kBins - 1 - (tid * kOwn + i)];
          count += S.count[kBins - 1 - (tid * kOwn + i)];
        }
        const uint64_t mass_upto = warp_scan(mass);
        const uint32_t count_upto = warp_scan(count);
        if (lane == 31) {
          S.scratch64[warp] = mass_upto;
          S.scratch32[warp] = count_upto;
        }
        if (tid == 0) S.crossing.bin = -1;
        __syncthreads();
        mass = base_mass + mass_upto - mass;
        count = base_count + count_upto - count;
        for (int w = 0; w < warp; ++w) {
          mass += S.scratch64[w];
          count += S.scratch32[w];
        }
        // the one bin before which a level passes, and after which it does not
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const int b = kBins - 1 - (tid * kOwn + i);
          const uint64_t m1 = mass + S.mass[b];
          const uint32_t c1 = count + S.count[b];
          if (R.passes(mass, count) && !R.passes(m1, c1)) S.crossing = {mass, count, b};
          mass = m1;
          count = c1;
        }
        __syncthreads();
        const Crossing at = S.crossing;
        if (at.bin >= 0) {
          const uint32_t lo = now.lo + (static_cast<uint32_t>(at.bin) << now.shift);
          const uint32_t hi = min(lo + (1u << now.shift), now.hi);
          if (hi - lo == 1) {
            next = {kDraw, lo, 0, 0, 0};                     // the floor
          } else {
            low = lo;
            high = hi;
            base_mass = at.mass;
            base_count = at.count;
            next = zoom(lo, hi, false);
          }
        } else if (!R.passes(base_mass, base_count)) {       // the guess was too low
          low = now.hi;
          next = zoom(low, high, true);
        } else if (now.lo <= low) {
          next = {kDraw, low, 0, 0, 0};                      // nothing stands in the way down to the lowest possible floor
        } else {
          high = now.lo;
          next = zoom(low, high, true);
        }
      }
      if (round == kMaxRounds && next.action != kDone) {      // not reached; a bound all the same
        next.action = kDone;
        if (tid == 0) {
          emit(A, R.r, 0, __int_as_float(0x7fffffff));
          if (A.status_out) atomicOr(A.status_out, ESPO_DEV_TIMEOUT);
        }
      }
      __syncthreads();
      if (tid < kCluster) cluster.map_shared_rank(&S, tid)->order = next;
    }
    cluster.sync();
    now = S.order;
  }
  if (now.action == kDone) return;

  // ---- the draw over the ids at or above the floor: the warps' exact masses, then inside the range that holds the target
  {
    uint64_t s = 0;
    if (above_key > now.lo && above_low <= now.lo && S.n_near[warp] <= kNear) {      // the last sweep but some kept what it takes
      for (int i = lane; i < S.n_near[warp]; i += 32)
        if (S.near[warp][i] >= now.lo) s += R.weight.fixed(K::value(S.near[warp][i]));
      s = warp_sum64(s) + warp_above;
    } else {
      s = exact_mass(L, R, now.lo, L.begin(warp), L.begin(warp + 1), S.queue[warp]);
    }
    if (lane == 0) S.exact_sum[warp] = s;
  }
  cluster.sync();
  uint64_t part[kParts], own = 0;
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    const int w = lane * kParts + i;
    part[i] = cluster.map_shared_rank(&S, w / kWarps)->exact_sum[w % kWarps];
    own += part[i];
  }
  cluster.sync();          // nobody reads a peer's memory after this
  const uint64_t upto = warp_scan(own), total = __shfl_sync(kFullMask, upto, 31);
  const double target = R.u * static_cast<double>(total);
  const unsigned beyond = __ballot_sync(kFullMask, target < static_cast<double>(upto));
  if (!beyond) return;             // (the total is at least one unit and u below 1)
  int at = __ffs(beyond) - 1;
  uint64_t before = __shfl_sync(kFullMask, upto - own, at);
  {
    int i = 0;
#pragma unroll
    for (int j = 0; j < kParts - 1; ++j) {
      const uint64_t next = __shfl_sync(kFullMask, part[j], at);
      if (i == j && target >= static_cast<double>(before + next)) {
        before += next;
        ++i;
      }
    }
    at = at * kParts + i;
  }
  if (at / kWarps != rank) return;
  const int b = L.begin(at % kWarps), n = L.begin(at % kWarps + 1) - b;
  const int b0 = b + n * warp / kWarps, b1 = b + n * (warp + 1) / kWarps;
  const uint64_t mine = exact_mass(L, R, now.lo, b0, b1, S.queue[warp]);
  if (lane == 0) S.scratch64[warp] = mine;
  __syncthreads();
  for (int w = 0; w < warp; ++w) before += S.scratch64[w];
  if (static_cast<double>(before) > target || target >= static_cast<double>(before + mine)) return;
  const float floor_x = K::value(now.lo);
  bool done = false;
  sweep(L, b0, b1, [&](int p, const uint4& v) {
    if (done) return;
    float x[kN];
    unpack(L.row, v, x);
    uint64_t f[kN], own = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      f[i] = R.weight.fixed(x[i]);
      if (!(x[i] >= floor_x)) f[i] = 0;
      own += f[i];
    }
    const uint64_t upto = warp_scan(own), step = __shfl_sync(kFullMask, upto, 31);
    if (target < static_cast<double>(before + step)) {
      done = true;
      uint64_t c = before + upto - own;
      if (static_cast<double>(c) <= target && target < static_cast<double>(c + own)) {
        bool taken = false;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          c += f[i];
          if (!taken && f[i] && target < static_cast<double>(c)) {
            taken = true;
            emit(A, R.r, p * kN + i, R.logp(x[i], static_cast<double>(total) / kOne));
          }
        }
      }
    }
    before += step;
  });
}

// Draws a row without a filter from the chunks' sums, all in 64 bits: chunk, eighth of it, then the thread's piece.  False
// if the last bits of two orders of addition disagree (the integers decide then).  scaled: the chunks' sums relative to the
// row's largest logit, two a lane; c_max their largest logits.
template <typename T>
__device__ __forceinline__ bool pick(const SampleArgs& A, const Row& R, const ChunkStat* stats, const double (&scaled)[2],
                                     const float (&c_max)[2], Shared& S) {
  constexpr int kN = Vec<T>::kN;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const double target = R.u * R.z;
  const double upto0 = warp_scan(scaled[0]), half = __shfl_sync(kFullMask, upto0, 31);
  const double upto1 = half + warp_scan(scaled[1]);
  const unsigned in0 = __ballot_sync(kFullMask, target < upto0), in1 = __ballot_sync(kFullMask, target < upto1);
  if (!(in0 | in1)) return false;
  const int l = in0 ? __ffs(in0) - 1 : __ffs(in1) - 1;
  const int c = in0 ? l : 32 + l;
  double before = __shfl_sync(kFullMask, in0 ? upto0 - scaled[0] : upto1 - scaled[1], l);
  const double factor = R.weight(__shfl_sync(kFullMask, in0 ? c_max[0] : c_max[1], l));
  int eighth = 0;
  for (; eighth < kWarps - 1; ++eighth) {
    const double part = stats[c].sum[eighth] * factor;
    if (target < before + part) break;
    before += part;
  }
  const T* row = static_cast<const T*>(A.logits) + static_cast<int64_t>(R.r) * A.row_stride;
  const int p = (c * kWarps + eighth) * A.warp_pieces + tid;
  float x[kN];
  double own = 0.0;
  if (tid < A.warp_pieces && p * kN < A.V) {
    unpack(row, load_piece(row, p, A.V, reinterpret_cast<uintptr_t>(row) % 16 == 0), x);
#pragma unroll
    for (int i = 0; i < kN; ++i) own += R.weight(x[i]);
  }
  const double upto = warp_scan(own);
  double* sums = reinterpret_cast<double*>(S.scratch64);
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  for (int w = 0; w < warp; ++w) before += sums[w];
  double at = before + upto - own;
  // The borders between threads are rounded on either side for themselves, so the target may seem to lie in two threads'
  // pieces: the lowest id is the token.
  int mine = 0x7fffffff;
  float mine_x = 0.0f;
  if (own > 0.0 && at <= target && target < before + upto) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const double w = R.weight(x[i]);
      if (mine == 0x7fffffff && target < at + w && x[i] > -INFINITY) {
        mine = p * kN + i;
        mine_x = x[i];
      }
      at += w;
    }
    if (mine != 0x7fffffff) atomicMin(&S.max_id, mine);
  }
  __syncthreads();
  const int token = S.max_id;
  if (token == 0x7fffffff) return false;
  if (mine == token) emit(A, R.r, token, R.logp(mine_x, R.z));
  return true;
}

// The row's numbers from its chunks': a lane holds chunks lane and lane + 32, every warp alike.
struct Chunks {
  float max[2];
  double scaled[2];       // sums relative to the row's largest logit
  int listed[2];
  uint32_t cut;           // the highest of the chunks' cuts
};
enum Kind : int { kUnusable, kGreedy, kSampled };

template <typename T>
__device__ __forceinline__ Kind read_row(const SampleArgs& A, int in_batch, const RowParams& P, Chunks& C, Row& R) {
  using K = Key<T>;
  const int lane = threadIdx.x & 31;
  const ChunkStat* stats = A.stats + static_cast<int64_t>(in_batch) * A.chunks;
  C.cut = 0;
#pragma unroll
  for (int h = 0; h < kMaxChunks / 32; ++h) {
    C.max[h] = -INFINITY;
    C.scaled[h] = 0.0;
    C.listed[h] = 0;
    const int c = h * 32 + lane;
    if (c < A.chunks) {
      C.max[h] = stats[c].max;
      C.listed[h] = stats[c].listed;
      C.cut = max(C.cut, stats[c].cut);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) C.scaled[h] += stats[c].sum[w];
    }
  }
  C.cut = __reduce_max_sync(kFullMask, C.cut);
  R.r = A.row0 + in_batch;
  R.top = max_nan(C.max[0], C.max[1]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) R.top = max_nan(R.top, __shfl_xor_sync(kFullMask, R.top, o));
  // (so close to the lowest float that a logit 140 T below has no place there, a masked id could not be told from it)
  const bool room = static_cast<double>(R.top) - 140.0 * P.temperature > -3.4028234663852886e38;
  if (!(P.fine && room && R.top < INFINITY)) return kUnusable;      // NaN fails too
  if (P.greedy) return kGreedy;
  R.inv_t = 1.0 / static_cast<double>(P.temperature);
  R.k = static_cast<float>(fmin(1.4426950408889634 * R.inv_t, 3e38));
  R.weight.set(R.top, P.temperature);
  R.u = P.u;
  R.top_p = P.top_p;
  R.top_k = P.top_k;
  R.bounded = P.top_p <= 1.0f || P.top_k < (1u << 31);
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (C.scaled[h] > 0.0) C.scaled[h] *= R.weight(C.max[h]);
  R.z = C.scaled[0] + C.scaled[1];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) R.z += __shfl_xor_sync(kFullMask, R.z, o);
  R.top_key = K::of(R.top);
  R.min_key = K::kLowest;
  if (P.min_p > 0.0f) {
    // The smallest key whose logit lies at most -T ln(min_p) below the largest, sought from the lowest key to the largest
    // logit's (which passes), 32 probes a step.  In 64 bits, and by the logits, not by their keys' distance from a rounded
    // border: next to zero thousands of keys lie closer together than any rounding of it.
    const double least = log(static_cast<double>(P.min_p)) * static_cast<double>(P.temperature);
    uint32_t lo = K::kLowest, hi = R.top_key;
    while (lo < hi) {
      const uint32_t step = (hi - lo + 31) / 32;
      const uint32_t probe = min(lo + lane * step, hi);
      const bool enough = static_cast<double>(K::value(probe)) - static_cast<double>(R.top) >= least;
      const unsigned ok = __ballot_sync(kFullMask, enough);
      if (ok) {
        const int first = __ffs(ok) - 1;
        hi = __shfl_sync(kFullMask, probe, first);
        if (first) lo += (first - 1) * step + 1;
        else lo = hi;
      } else {
        lo += 31 * step + 1;
      }
    }
    R.min_key = hi;
  }
  return kSampled;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) row_kernel(const SampleArgs A) {
  constexpr int kN = Vec<T>::kN;
  using K = Key<T>;
  const int in_batch = blockIdx.x, r = A.row0 + in_batch;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __shared__ Shared S;
  if (tid == 0) S.max_id = 0x7fffffff;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  bool bad_slot;
  if (!row_active(A, r, bad_slot)) {
    if (tid == 0) {
      A.tokens_out[r] = -1;
      if (bad_slot && A.status_out) atomicOr(A.status_out, ESPO_DEV_BAD_SLOT);
    }
    return;
  }
  const RowParams P = row_params(A, r);
  Chunks C;
  Row R;
  const Kind kind = read_row<T>(A, in_batch, P, C, R);
  if (kind == kUnusable) {
    if (tid == 0) {
      emit(A, r, 0, __int_as_float(0x7fffffff));
      if (A.status_out) atomicOr(A.status_out, ESPO_DEV_BAD_ROW);
    }
    return;
  }
  if (kind == kGreedy) {
    const unsigned h0 = __ballot_sync(kFullMask, C.max[0] == R.top), h1 = __ballot_sync(kFullMask, C.max[1] == R.top);
    const int c = h0 ? __ffs(h0) - 1 : 32 + __ffs(h1) - 1;
    const T* row = static_cast<const T*>(A.logits) + static_cast<int64_t>(r) * A.row_stride;
    const bool whole = reinterpret_cast<uintptr_t>(row) % 16 == 0;
    int best = 0x7fffffff;
    const int n = kWarps * A.warp_pieces;
    for (int p = c * n + tid; p < (c + 1) * n && best == 0x7fffffff; p += kThreads) {
      if (p * kN >= A.V) break;
      float x[kN];
      unpack(row, load_piece(row, p, A.V, whole), x);
#pragma unroll
      for (int i = kN - 1; i >= 0; --i)
        if (x[i] == R.top) best = p * kN + i;
    }
    __syncthreads();
    if (best != 0x7fffffff) atomicMin(&S.max_id, best);
    __syncthreads();
    if (tid == 0) emit(A, r, S.max_id, 0.0f);
    return;
  }

  Order next = {kDone, 0, 0, 0, 0};
  if (!R.bounded && !(P.min_p > 0.0f)) {
    __syncthreads();
    if (!pick<T>(A, R, A.stats + static_cast<int64_t>(in_batch) * A.chunks, C.scaled, C.max, S)) next = {kDraw, K::kLowest, 0, 0, 0};
  } else {
    const uint32_t lo = max(C.cut, R.min_key);      // the lists are complete down to every chunk's cut
    const int listed = put_starts(C.listed[0], C.listed[1], S);
    const bool usable = lo <= R.top_key;
    int kept = 0;                                   // listed ids at or above lo, brought together in order
    if (usable && (R.bounded || lo == R.min_key)) {
      constexpr int kEach = kListTotal / kThreads;
      Listed v[kEach];
      int s = segment_of(S, tid * kEach), mine = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int e = tid * kEach + i;
        v[i].key = 0;
        if (e < listed) {
          while (S.starts[s + 1] <= e) ++s;
          v[i] = A.lists[(static_cast<int64_t>(in_batch) * A.chunks + s) * A.list_cap + (e - S.starts[s])];
        }
        mine += v[i].key >= lo;
      }
      const int upto = warp_scan(mine);
      if (lane == 31) S.scratch32[warp] = upto;
      __syncthreads();
      int to = upto - mine;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const int n = static_cast<int>(S.scratch32[w]);
        if (w < warp) to += n;
        kept += n;
      }
      if (kept <= kListed) {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
          if (v[i].key >= lo) S.compact[to++] = v[i];
      }
      __syncthreads();
    }
    if (!R.bounded && !(usable && lo == R.min_key && kept <= kListed)) {
      next = {kDraw, R.min_key, 0, 0, 0};           // min_p alone: the floor is known
    } else if (!usable || kept > kListed) {
      next = {kHistogram, 0, 0, 0, 0};
    } else {
      List list;
#pragma unroll
      for (int i = 0; i < kPerThread; ++i) {
        const int e = tid * kPerThread + i;
        Listed v = {0, 0};
        if (e < kept) v = S.compact[e];
        put_entry<T>(list, R, i, e < kept, v);
      }
      uint32_t floor_key = R.min_key;
      if (!R.bounded || find_floor(list, R, lo, floor_key, S)) draw_listed<T>(A, list, R, floor_key, S);
      else next = {kHistogram, 0, 0, 0, 0};
    }
  }
  if (next.action != kDone && tid == 0) A.wide[atomicAdd(A.n_wide, 1u)] = {in_batch, next};
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) wide_kernel(const SampleArgs A) {
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ Shared S;
  cluster.barrier_arrive();          // a block may touch a peer's memory only once the peer runs
  asm volatile("griddepcontrol.wait;" ::: "memory");
  cluster.barrier_wait();
  const unsigned n = *A.n_wide;
  for (unsigned i = blockIdx.x / kCluster; i < n; i += gridDim.x / kCluster) {
    const WideRow W = A.wide[i];
    Chunks C;
    Row R;
    read_row<T>(A, W.in_batch, row_params(A, A.row0 + W.in_batch), C, R);
    sweep_row<T>(A, R, W.order, S);
    cluster.sync();                  // the next row's sweeps overwrite what the peers read
  }
}

// ---------------------------------------------------------------------------------------------- host side

struct Plan {
  int chunks, warp_pieces, cut_rank, list_cap, batch;
  int64_t stat_bytes, list_bytes, bytes;
};
Plan plan_sample(int32_t n_rows, int32_t V, int32_t dtype) {
  Plan p;
  const int ids = dtype == ESPO_F32 ? kChunk<float> : kChunk<__nv_bfloat16>;
  p.chunks = (V + ids - 1) / ids;
  const int pieces = (V + ids / (kThreads * kPieces) - 1) / (ids / (kThreads * kPieces));
  p.warp_pieces = (pieces + p.chunks * kWarps - 1) / (p.chunks * kWarps);
  // About 600 listed ids a row are expected, 2048 fit (a vocabulary of half that is listed whole).  The lowest of eight warps'
  // cuts at rank 4 of 32 lanes lies near rank 7 of 32 (ten chunks: 56 lanes a chunk), and differs little from chunk to chunk,
  // so most of what is listed lies above the highest cut of the row.
  const int lanes = p.warp_pieces < 32 ? p.warp_pieces : 32;
  p.list_cap = kListTotal / p.chunks;
  p.cut_rank = 40 / p.chunks < (lanes + 1) / 2 ? 40 / p.chunks : (lanes + 1) / 2;
  if (p.cut_rank < 1) p.cut_rank = 1;
  if (V <= kListed) p.cut_rank = 33;
  p.batch = n_rows < kMaxRows ? n_rows : kMaxRows;
  p.stat_bytes = (static_cast<int64_t>(p.batch) * p.chunks * sizeof(ChunkStat) + 255) / 256 * 256;
  p.list_bytes = (static_cast<int64_t>(p.batch) * p.chunks * p.list_cap * static_cast<int64_t>(sizeof(Listed)) + 255) / 256 * 256;
  p.bytes = 256 + p.stat_bytes + p.list_bytes + static_cast<int64_t>(p.batch) * static_cast<int64_t>(sizeof(WideRow));
  return p;
}

template <typename T>
int launch_sample(SampleArgs a, int n_rows, const Plan& plan, cudaStream_t st) {
  for (int row0 = 0; row0 < n_rows; row0 += plan.batch) {
    const int rows = n_rows - row0 < plan.batch ? n_rows - row0 : plan.batch;
    a.row0 = row0;
    chunk_kernel<T><<<static_cast<unsigned>(rows) * plan.chunks, kThreads, 0, st>>>(a);
    ESPO_CUDA_TRY(cudaGetLastError());
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ESPO_CUDA_TRY(cudaLaunchKernelEx(&cfg, row_kernel<T>, a));
    a.slice = ((a.V + kCluster - 1) / kCluster + 7) / 8 * 8;
    cfg.gridDim = dim3(static_cast<unsigned>(rows < kClusters ? rows : kClusters) * kCluster);
    cfg.numAttrs = 2;
    ESPO_CUDA_TRY(cudaLaunchKernelEx(&cfg, wide_kernel<T>, a));
  }
  return ESPO_OK;
}

}  // namespace
}  // namespace espo

using namespace espo;

extern "C" {

int espo_sample_workspace(int32_t n_rows, int32_t V, int64_t* bytes_out) {
  if (!bytes_out) return ESPO_ERR_NULL;
  if (n_rows < 0 || V < 1) return ESPO_ERR_BAD_SHAPE;
  if (V > kMaxVocab) return ESPO_ERR_CAPACITY;
  const int64_t f = plan_sample(n_rows, V, ESPO_F32).bytes, b = plan_sample(n_rows, V, ESPO_BF16).bytes;
  *bytes_out = f > b ? f : b;      // either element type
  return ESPO_OK;
}

int espo_sample(const void* logits, int32_t logits_dtype, int64_t row_stride, int32_t n_rows, int32_t V, const float* u,
                const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                const int32_t* row_ids, const uint8_t* status, int32_t capacity, int32_t* tokens_out, float* logp_out,
                void* workspace, int64_t workspace_bytes, uint32_t* status_out, void* stream) {
  if (n_rows > 0 && (!logits || !u || !tokens_out || !workspace)) return ESPO_ERR_NULL;
  if (logits_dtype != ESPO_F32 && logits_dtype != ESPO_BF16) return ESPO_ERR_BAD_DTYPE;
  if (n_rows < 0 || V < 1 || row_stride < V || (status && capacity < 1)) return ESPO_ERR_BAD_SHAPE;
  if (V > kMaxVocab) return ESPO_ERR_CAPACITY;
  if (!aligned(logits, logits_dtype == ESPO_F32 ? 4 : 2) || !aligned(u, 4) || !aligned(temperature, 4) ||
      !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(row_ids, 4) || !aligned(tokens_out, 4) ||
      !aligned(logp_out, 4) || !aligned(workspace, 256) || !aligned(status_out, 4))
    return ESPO_ERR_ALIGN;
  const Plan plan = plan_sample(n_rows, V, logits_dtype);
  if (n_rows > 0 && workspace_bytes < plan.bytes) return ESPO_ERR_CAPACITY;
  if (n_rows == 0) return ESPO_OK;
  SampleArgs a = {};
  a.logits = logits;
  a.row_stride = row_stride;
  a.u = u;
  a.temperature = temperature;
  a.top_p = top_p;
  a.min_p = min_p;
  a.top_k = top_k;
  a.row_ids = row_ids;
  a.status = status;
  a.tokens_out = tokens_out;
  a.logp_out = logp_out;
  a.status_out = status_out;
  a.V = V;
  a.capacity = capacity;
  char* at = static_cast<char*>(workspace);
  a.n_wide = reinterpret_cast<unsigned*>(at);
  a.stats = reinterpret_cast<ChunkStat*>(at + 256);
  a.lists = reinterpret_cast<Listed*>(at + 256 + plan.stat_bytes);
  a.wide = reinterpret_cast<WideRow*>(at + 256 + plan.stat_bytes + plan.list_bytes);
  a.chunks = plan.chunks;
  a.list_cap = plan.list_cap;
  a.cut_rank = plan.cut_rank;
  a.warp_pieces = plan.warp_pieces;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return logits_dtype == ESPO_F32 ? launch_sample<float>(a, n_rows, plan, st) : launch_sample<__nv_bfloat16>(a, n_rows, plan, st);
}

}  // extern "C"
