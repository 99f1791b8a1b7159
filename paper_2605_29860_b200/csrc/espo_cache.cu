// The paged key/value cache: writing tokens (rotary positions, 8-bit codes with a power-of-two scale per vector) and
// reading them back.
//
// Mathematics.  A head's vector is cut into units of four rotary pairs (eight numbers): in the half layout four dims from
// [0, rot/2) with their partners rot/2 further on, in the interleaved layout eight adjacent dims; the dims beyond rot_dim
// are paired the same way with an angle of zero.  One lane owns one unit, so head_dim/8 lanes hold a head, the pair's two
// numbers sit in one lane, and the largest magnitude of the vector is a butterfly over those lanes.  The angles are the same
// for every head of a token: the warp computes each of them once and hands every lane its four.
//
// What bounds it: HBM for a prompt, launch latency for a decode step.  Every number is read and written once.  20000 tokens,
// 16 query and 8 cache heads of 64, fp32 to bf16: 46.3 us, 6.2 TB/s; 8191 tokens, 28 and 4 heads of 128, bf16 to e4m3: 34 us,
// 4.2 TB/s, half of the clocks issuing instructions and the rest waiting for loads of 8 bytes a lane.  Reading back, 12 us of the
// latter and 20.5 of the former (issuing 25 to 30 %), waits for one token's loads a warp at a time.  The decode form in a graph:
// 3.2 us for 8 rows of bf16, 5.4 for 512 of e4m3.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "espo.h"
#include "espo_device.cuh"
#include "espo_host.h"

namespace espo {
namespace {

struct AppendArgs {
  espo_kv_cache cache;
  espo_rope rope;               // rot_dim 0: no rotation
  espo_sequences seqs;          // decode form only
  const void *key, *value, *q;
  void* q_out;
  int64_t key_stride, value_stride, q_stride, q_out_stride;
  const int32_t *cache_slots, *positions, *row_ids;
  uint32_t* status_out;
  int32_t n_tokens, n_q_heads;
};

__device__ __forceinline__ void flag(uint32_t* status_out, uint32_t bits) {
  if (status_out) atomicOr(status_out, bits);
}

// Four adjacent numbers of a row as floats.
template <typename T>
__device__ __forceinline__ float4 load4(const T* p);
template <>
__device__ __forceinline__ float4 load4<float>(const float* p) { return __ldcs(reinterpret_cast<const float4*>(p)); }
template <>
__device__ __forceinline__ float4 load4<__nv_bfloat16>(const __nv_bfloat16* p) {
  const uint2 w = __ldcs(reinterpret_cast<const uint2*>(p));
  return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

// Smallest e in [-64, 63] with amax <= 448 * 2^e (448 = 1.75 * 2^8): amax = f * 2^k with f in [1, 2) needs k - 8, or one
// more if f > 1.75.  A subnormal or zero amax ends at -64, an infinite one at 63.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, -64), 63);
}

__device__ __forceinline__ uint32_t pack_e4m3(float4 v, float s) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v.x * s, v.y * s), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v.z * s, v.w * s), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// (a.x, b.x), (a.y, b.y), ... are the four pairs.
struct Unit {
  float4 a, b;
};

__device__ __forceinline__ void turn(Unit& u, const float4& c, const float4& s) {
  const float4 a = u.a, b = u.b;
  u.a = make_float4(a.x * c.x - b.x * s.x, a.y * c.y - b.y * s.y, a.z * c.z - b.z * s.z, a.w * c.w - b.w * s.w);
  u.b = make_float4(b.x * c.x + a.x * s.x, b.y * c.y + a.y * s.y, b.z * c.z + a.z * s.z, b.w * c.w + a.w * s.w);
}

// Where a lane's unit lies in the head: two runs of four dims.
struct UnitPlace {
  int first, second;   // dims of the two runs
  bool adjacent;       // pairs are adjacent dims: run = (a0 b0 a1 b1)
  bool rotated;
};

__device__ __forceinline__ UnitPlace unit_place(int unit, int head_dim, const espo_rope& rope) {
  UnitPlace p;
  const int units_rot = rope.rot_dim / 8;
  p.rotated = unit < units_rot;
  p.adjacent = rope.interleaved != 0 || !p.rotated;
  if (p.adjacent) {
    p.first = unit * 8;
    p.second = p.first + 4;
  } else {
    p.first = unit * 4;
    p.second = p.first + rope.rot_dim / 2;
  }
  return p;
}

template <typename T>
__device__ __forceinline__ Unit load_unit(const T* head, const UnitPlace& p) {
  Unit u;
  u.a = load4(head + p.first);
  u.b = load4(head + p.second);
  return u;
}

// From the order in memory to pairs and back (its own inverse is the other direction below).
__device__ __forceinline__ void to_pairs(Unit& u, bool adjacent) {
  if (!adjacent) return;
  const Unit m = u;
  u.a = make_float4(m.a.x, m.a.z, m.b.x, m.b.z);
  u.b = make_float4(m.a.y, m.a.w, m.b.y, m.b.w);
}
__device__ __forceinline__ void from_pairs(Unit& u, bool adjacent) {
  if (!adjacent) return;
  const Unit m = u;
  u.a = make_float4(m.a.x, m.b.x, m.a.y, m.b.y);
  u.b = make_float4(m.a.z, m.b.z, m.a.w, m.b.w);
}

// Cosine and sine of position * inv_freq, times mscale, in 64 bits and rounded once.  The product and its reduction to a part
// of a turn need 64 bits (at position 10^6 a 32-bit product would be off by 0.06 rad).  The functions take them for the entries
// next to a border between two codes: with 32-bit ones 1709 of 41 million bf16 keys were rounded to the other side (20000 fp32
// tokens, four batches), now 763, which the 32-bit rotation leaves; 8191 tokens to e4m3 take 41.5 us with their read-back, not 40.5.
__device__ __forceinline__ void angle_of(int position, double inv_freq, float mscale, float& c, float& s) {
  const double turns = static_cast<double>(position) * inv_freq * 0.15915494309189533577;   // 1 / (2 pi)
  double sine, cosine;
  sincospi(2.0 * (turns - rint(turns)), &sine, &cosine);                                     // of at most half a turn
  c = static_cast<float>(cosine * static_cast<double>(mscale));
  s = static_cast<float>(sine * static_cast<double>(mscale));
}

constexpr int kAppendWarps = 8;

// kPerBlock tokens share a block of eight warps: one token's heads are spread over eight, two or one of them.
template <typename T, int kHeadDim, bool kE4M3, bool kRows, int kPerBlock>
__global__ void __launch_bounds__(kAppendWarps * 32) append_kernel(const AppendArgs A) {
  constexpr int kLanes = kHeadDim / 8;          // lanes per head
  constexpr int kHeadsPerWarp = 32 / kLanes;
  constexpr int kWarpsPerToken = kAppendWarps / kPerBlock;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int token = blockIdx.x * kPerBlock + warp / kWarpsPerToken;
  const int sub = warp % kWarpsPerToken;
  const espo_kv_cache& C = A.cache;

  bool live = token < A.n_tokens;
  int64_t slot = -1;
  int position = 0;
  int seq = -1, len = 0;
  if (live) {
    if constexpr (kRows) {
      const espo_sequences& S = A.seqs;
      seq = A.row_ids ? A.row_ids[token] : token;
      uint32_t bad = 0;
      if (seq < 0 || seq >= S.capacity) {
        bad = ESPO_DEV_BAD_SLOT;
        live = false;
      } else if (S.status && S.status[seq] != ESPO_ROW_ACTIVE) {
        live = false;
      } else {
        len = S.length[seq];
        const int group = S.group ? S.group[seq] : -1;
        const int64_t room = static_cast<int64_t>(S.max_pages) * C.page_size;
        int prefix = 0;
        if (group >= S.n_groups) bad |= ESPO_DEV_BAD_PAGE;
        else if (group >= 0) prefix = S.prefix_length[group];
        if (len < 0 || len > room || prefix < 0 || prefix > S.max_prefix_pages * C.page_size) bad |= ESPO_DEV_BAD_LENGTHS;
        else if (len == room) bad |= ESPO_DEV_CACHE_FULL;
        if (!bad) {
          const int page = S.pages[static_cast<int64_t>(seq) * S.max_pages + len / C.page_size];
          if (page < 0 || page >= C.n_pages) bad = ESPO_DEV_BAD_PAGE;
          else slot = static_cast<int64_t>(page) * C.page_size + len % C.page_size;
        }
        position = prefix + len;
      }
      if (bad && sub == 0 && lane == 0) flag(A.status_out, bad);
    } else {
      slot = A.cache_slots[token];
      position = A.rope.rot_dim ? A.positions[token] : 0;
      if (slot >= static_cast<int64_t>(C.n_pages) * C.page_size) {
        if (sub == 0 && lane == 0) flag(A.status_out, ESPO_DEV_BAD_PAGE);
        slot = -1;
      }
    }
  }

  if (live) {
    const int unit = lane % kLanes;
    const UnitPlace place = unit_place(unit, kHeadDim, A.rope);
    float4 c, s;
    {
      // the token's rot_dim / 2 angles, each by one lane, then the unit's four from their lanes
      constexpr int kEach = kHeadDim / 64;
      float mine_c[kEach], mine_s[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        mine_c[i] = mine_s[i] = 0.0f;
        const int j = kEach * lane + i;
        if (j < A.rope.rot_dim / 2) angle_of(position, A.rope.inv_freq[j], A.rope.mscale, mine_c[i], mine_s[i]);
      }
      float of_c[4], of_s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        of_c[i] = __shfl_sync(kFullMask, mine_c[i % kEach], (4 * unit + i) / kEach);
        of_s[i] = __shfl_sync(kFullMask, mine_s[i % kEach], (4 * unit + i) / kEach);
      }
      c = make_float4(of_c[0], of_c[1], of_c[2], of_c[3]);
      s = make_float4(of_s[0], of_s[1], of_s[2], of_s[3]);
    }
    const int n_q = A.n_q_heads, n_kv = C.n_kv_heads;
    const int first_head = sub * kHeadsPerWarp + lane / kLanes;
    constexpr int kStep = kWarpsPerToken * kHeadsPerWarp;

    const T* q = static_cast<const T*>(A.q) + token * A.q_stride;
    T* q_out = static_cast<T*>(A.q_out) + token * A.q_out_stride;
#pragma unroll 4
    for (int h = first_head; h < n_q; h += kStep) {
      Unit u = load_unit(q + h * kHeadDim, place);
      to_pairs(u, place.adjacent);
      if (place.rotated) turn(u, c, s);
      from_pairs(u, place.adjacent);
      store4(q_out + h * kHeadDim + place.first, u.a);
      store4(q_out + h * kHeadDim + place.second, u.b);
    }

    // keys are heads 0 .. n_kv-1, values the n_kv after them; a warp's lanes stay together for the butterfly
    const int64_t page = slot < 0 ? 0 : slot / C.page_size;
    const int offset = slot < 0 ? 0 : static_cast<int>(slot % C.page_size);
    for (int base = sub * kHeadsPerWarp; base < 2 * n_kv; base += kStep) {
      const int hv = base + lane / kLanes;
      const bool on = slot >= 0 && hv < 2 * n_kv;
      const bool is_key = hv < n_kv;
      const int h = is_key ? hv : hv - n_kv;
      Unit u = {};
      if (on) {
        const T* src = is_key ? static_cast<const T*>(A.key) + token * A.key_stride
                              : static_cast<const T*>(A.value) + token * A.value_stride;
        u = load_unit(src + h * kHeadDim, place);
        to_pairs(u, place.adjacent);
        if (is_key && place.rotated) turn(u, c, s);
        from_pairs(u, place.adjacent);
      }
      const int64_t entry = (page * n_kv + h) * C.page_size + offset;
      if constexpr (kE4M3) {
        float amax = fmaxf(fmaxf(fmaxf(fabsf(u.a.x), fabsf(u.a.y)), fmaxf(fabsf(u.a.z), fabsf(u.a.w))),
                           fmaxf(fmaxf(fabsf(u.b.x), fabsf(u.b.y)), fmaxf(fabsf(u.b.z), fabsf(u.b.w))));
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(kFullMask, amax, o));
        const int e = scale_exponent(amax);
        if (on) {
          const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);     // 2^-e
          uint8_t* dst = static_cast<uint8_t*>(is_key ? C.k : C.v) + entry * kHeadDim;
          *reinterpret_cast<uint32_t*>(dst + place.first) = pack_e4m3(u.a, down);
          *reinterpret_cast<uint32_t*>(dst + place.second) = pack_e4m3(u.b, down);
          if (unit == 0) (is_key ? C.k_exp : C.v_exp)[entry] = static_cast<uint8_t>(e + 127);
        }
      } else if (on) {
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(is_key ? C.k : C.v) + entry * kHeadDim;
        store4(dst + place.first, u.a);
        store4(dst + place.second, u.b);
      }
    }
  }
  if constexpr (kRows) {
    __syncthreads();      // every warp of the token has read the length
    if (live && slot >= 0 && sub == 0 && lane == 0) A.seqs.length[seq] = len + 1;
  }
}

template <typename T, int kHeadDim, bool kE4M3, bool kRows>
void launch_append(const AppendArgs& a, cudaStream_t st) {
  // A token's heads are spread over eight warps while tokens are few, over two while one warp each would leave room on the
  // 148 SMs of 64 warps, else one warp takes them all.  Append and gather of 28 query and 4 cache heads of 128, bf16 to e4m3,
  // with eight, two and one: 512 tokens 7.5, 8.5, 10.8 us; 768: 9.6, 9.6, 11.2; 8192: 51.8, 40.9, 43.4; 12288: 78, 63.9, 58.8.
  // The same order at 16 and 8 heads of 64, fp32 to bf16: 512 tokens 6.8, 7.1, 7.5; 8192: 34.8, 26.5, 27.5; 12288: 51.2, 42.2, 39.7.
  constexpr int kSpread = 600, kShared = 148 * 64;
  if (a.n_tokens <= kSpread) {
    append_kernel<T, kHeadDim, kE4M3, kRows, 1><<<a.n_tokens, kAppendWarps * 32, 0, st>>>(a);
  } else if (a.n_tokens <= kShared) {
    append_kernel<T, kHeadDim, kE4M3, kRows, 4><<<(a.n_tokens + 3) / 4, kAppendWarps * 32, 0, st>>>(a);
  } else {
    append_kernel<T, kHeadDim, kE4M3, kRows, kAppendWarps>
        <<<(a.n_tokens + kAppendWarps - 1) / kAppendWarps, kAppendWarps * 32, 0, st>>>(a);
  }
}

template <bool kRows>
int dispatch_append(const AppendArgs& a, int dtype, cudaStream_t st) {
  const bool e = a.cache.dtype == ESPO_E4M3, d = a.cache.head_dim == 128, f = dtype == ESPO_F32;
#define ESPO_APPEND(T, D, E) launch_append<T, D, E, kRows>(a, st)
  if (f) {
    if (d) { if (e) ESPO_APPEND(float, 128, true); else ESPO_APPEND(float, 128, false); }
    else   { if (e) ESPO_APPEND(float, 64, true); else ESPO_APPEND(float, 64, false); }
  } else {
    if (d) { if (e) ESPO_APPEND(__nv_bfloat16, 128, true); else ESPO_APPEND(__nv_bfloat16, 128, false); }
    else   { if (e) ESPO_APPEND(__nv_bfloat16, 64, true); else ESPO_APPEND(__nv_bfloat16, 64, false); }
  }
#undef ESPO_APPEND
  ESPO_CUDA_TRY(cudaGetLastError());
  return ESPO_OK;
}

// ---------------------------------------------------------------------------------------------- reading back

struct GatherArgs {
  espo_kv_cache cache;
  const int32_t* cache_slots;
  void *k_out, *v_out;
  uint32_t* status_out;
  int32_t n_tokens;
};

__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                                                 pack_bf16(v[6], v[7])));
}

// A warp per token, a lane per eight numbers of a key or value vector.  (A thread per eight numbers of all tokens, with the
// token and the page found by division each time, was bound by those instructions: 20000 tokens of 8 heads of 64 bf16 dims
// 25.2 us.)
template <typename T, bool kE4M3>
__global__ void __launch_bounds__(256) gather_kernel(const GatherArgs A) {
  const espo_kv_cache& C = A.cache;
  const int lane = threadIdx.x & 31;
  const int dim_shift = C.head_dim == 128 ? 7 : 6, page_shift = 31 - __clz(C.page_size);
  const int units = C.n_kv_heads << (dim_shift - 3);        // of the keys, and as many of the values
  const int64_t row = static_cast<int64_t>(C.n_kv_heads) << dim_shift;
  for (int64_t token = blockIdx.x * 8ll + (threadIdx.x >> 5); token < A.n_tokens; token += gridDim.x * 8ll) {
    int slot = A.cache_slots[token];
    if (slot >= 0 && (slot >> page_shift) >= C.n_pages) {
      if (lane == 0) flag(A.status_out, ESPO_DEV_BAD_PAGE);
      slot = -1;
    }
    const int64_t first = ((static_cast<int64_t>(slot >> page_shift) * C.n_kv_heads) << page_shift) + (slot & (C.page_size - 1));
#pragma unroll 4
    for (int i = lane; i < 2 * units; i += 32) {
      const bool is_key = i < units;
      const int r = is_key ? i : i - units;
      T* out = static_cast<T*>(is_key ? A.k_out : A.v_out);
      if (!out) continue;
      float v[8] = {};
      if (slot >= 0) {
        const int64_t entry = first + (static_cast<int64_t>(r >> (dim_shift - 3)) << page_shift);
        const int64_t at = (entry << dim_shift) + ((r << 3) & (C.head_dim - 1));
        if constexpr (kE4M3) {
          const int e = (is_key ? C.k_exp : C.v_exp)[entry];
          const uint2 w = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(is_key ? C.k : C.v) + at));
          const float up = __uint_as_float(e ? static_cast<uint32_t>(e) << 23 : 0x400000u);    // 2^(e - 127)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __nv_fp8x2_storage_t two = (j < 2 ? w.x : w.y) >> (16 * (j & 1));
            const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3)));
            v[2 * j] = f.x * up;
            v[2 * j + 1] = f.y * up;
          }
        } else {
          const uint4 w = __ldcs(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(is_key ? C.k : C.v) + at));
          const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[2 * j] = bf16_lo(x[j]);
            v[2 * j + 1] = bf16_hi(x[j]);
          }
        }
      }
      store8(out + token * row + (static_cast<int64_t>(r) << 3), v);
    }
  }
}

int check_append(const espo_kv_cache* cache, const espo_rope* rope, const void* key, int64_t key_stride,
                 const void* value, int64_t value_stride, int32_t dtype, int32_t n, const void* q, int64_t q_stride,
                 int32_t n_q_heads, void* q_out, int64_t q_out_stride, uint32_t* status_out) {
  const int rc = check_kv_cache(cache);
  if (rc != ESPO_OK) return rc;
  if (n < 0 || n_q_heads < 0) return ESPO_ERR_BAD_SHAPE;
  if (n > 0 && (!key || !value || (n_q_heads > 0 && (!q || !q_out)))) return ESPO_ERR_NULL;
  if (dtype != ESPO_F32 && dtype != ESPO_BF16) return ESPO_ERR_BAD_DTYPE;
  const int64_t kv = static_cast<int64_t>(cache->n_kv_heads) * cache->head_dim;
  const int64_t qn = static_cast<int64_t>(n_q_heads) * cache->head_dim;
  if (key_stride < kv || value_stride < kv || (n_q_heads > 0 && (q_stride < qn || q_out_stride < qn)) || n_q_heads > 65536)
    return ESPO_ERR_BAD_SHAPE;
  if (key_stride % 8 || value_stride % 8 || (n_q_heads > 0 && (q_stride % 8 || q_out_stride % 8))) return ESPO_ERR_ALIGN;
  if (!aligned(key, 16) || !aligned(value, 16) || !aligned(q, 16) || !aligned(q_out, 16) || !aligned(status_out, 4))
    return ESPO_ERR_ALIGN;
  if (rope) {
    if (!rope->inv_freq) return ESPO_ERR_NULL;
    if (rope->rot_dim < 8 || rope->rot_dim % 8 || rope->rot_dim > cache->head_dim || !isfinite(rope->mscale))
      return ESPO_ERR_BAD_PARAM;
    if (!aligned(rope->inv_freq, 8)) return ESPO_ERR_ALIGN;
  }
  return ESPO_OK;
}

AppendArgs pack_append(const espo_kv_cache* cache, const espo_rope* rope, const void* key, int64_t key_stride,
                       const void* value, int64_t value_stride, int32_t n, const void* q, int64_t q_stride,
                       int32_t n_q_heads, void* q_out, int64_t q_out_stride, uint32_t* status_out) {
  AppendArgs a = {};
  a.cache = *cache;
  if (rope) a.rope = *rope;
  a.key = key; a.key_stride = key_stride;
  a.value = value; a.value_stride = value_stride;
  a.q = q; a.q_stride = q_stride; a.n_q_heads = n_q_heads;
  a.q_out = q_out; a.q_out_stride = q_out_stride;
  a.status_out = status_out;
  a.n_tokens = n;
  return a;
}

}  // namespace

int check_kv_cache(const espo_kv_cache* c) {
  if (!c || !c->k || !c->v) return ESPO_ERR_NULL;
  if (c->dtype != ESPO_BF16 && c->dtype != ESPO_E4M3) return ESPO_ERR_BAD_DTYPE;
  if (c->dtype == ESPO_E4M3 && (!c->k_exp || !c->v_exp)) return ESPO_ERR_NULL;
  if (c->n_pages < 1 || c->n_kv_heads < 1) return ESPO_ERR_BAD_SHAPE;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return ESPO_ERR_BAD_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128) return ESPO_ERR_BAD_SHAPE;
  // bounds one factor at a time: n_pages * n_kv_heads fits 62 bits, and only if it is below 2^31 is it multiplied again
  const int64_t vectors = static_cast<int64_t>(c->n_pages) * c->n_kv_heads;
  if (vectors >= (1ll << 31) || vectors * c->page_size >= (1ll << 31)) return ESPO_ERR_CAPACITY;
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return ESPO_ERR_ALIGN;
  if (c->dtype == ESPO_E4M3 && (!aligned(c->k_exp, 16) || !aligned(c->v_exp, 16))) return ESPO_ERR_ALIGN;
  return ESPO_OK;
}

int check_sequences(const espo_sequences* s) {
  if (!s) return ESPO_ERR_NULL;
  if (s->capacity < 1 || s->max_pages < 0 || s->n_groups < 0 || s->max_prefix_pages < 0) return ESPO_ERR_BAD_SHAPE;
  if (!s->length || (s->max_pages > 0 && !s->pages)) return ESPO_ERR_NULL;
  if (s->group && s->n_groups > 0 && (!s->prefix_length || (s->max_prefix_pages > 0 && !s->prefix_pages))) return ESPO_ERR_NULL;
  // 2^30 own tokens and 2^29 of a prefix at 128 a page: their sum fits 31 bits
  if (s->max_pages > (1 << 23) || s->max_prefix_pages > (1 << 22)) return ESPO_ERR_CAPACITY;
  if (!aligned(s->pages, 4) || !aligned(s->length, 4) || !aligned(s->group, 4) || !aligned(s->prefix_pages, 4) ||
      !aligned(s->prefix_length, 4))
    return ESPO_ERR_ALIGN;
  return ESPO_OK;
}

}  // namespace espo

using namespace espo;

extern "C" {

int espo_rope_frequencies(int32_t kind, double theta, int32_t rot_dim, double factor, double original_length,
                          double fast_turns, double slow_turns, double* inv_freq_out, float* mscale_out) {
  if (!inv_freq_out) return ESPO_ERR_NULL;
  if (kind < ESPO_ROPE_PLAIN || kind > ESPO_ROPE_BY_PARTS) return ESPO_ERR_BAD_PARAM;
  if (!(theta > 1.0) || !isfinite(theta) || rot_dim < 8 || rot_dim % 8) return ESPO_ERR_BAD_PARAM;
  if (kind != ESPO_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return ESPO_ERR_BAD_PARAM;
  double lo = 0.0, hi = 0.0;
  if (kind == ESPO_ROPE_BY_PARTS) {
    if (!(original_length >= 1.0) || !(slow_turns > 0.0) || !(fast_turns > slow_turns) || !isfinite(original_length) ||
        !isfinite(fast_turns))
      return ESPO_ERR_BAD_PARAM;
    const double two_pi = 6.283185307179586477;
    lo = floor(rot_dim * log(original_length / (two_pi * fast_turns)) / (2.0 * log(theta)));
    hi = ceil(rot_dim * log(original_length / (two_pi * slow_turns)) / (2.0 * log(theta)));
    if (lo < 0.0) lo = 0.0;
    if (hi > rot_dim - 1) hi = rot_dim - 1;
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double plain = pow(theta, -2.0 * i / rot_dim);
    double f = plain;
    if (kind == ESPO_ROPE_LINEAR) f = plain / factor;
    if (kind == ESPO_ROPE_BY_PARTS) {
      double ramp = (i - lo) / (hi - lo > 0.001 ? hi - lo : 0.001);
      ramp = ramp < 0.0 ? 0.0 : ramp > 1.0 ? 1.0 : ramp;
      f = plain / factor * ramp + plain * (1.0 - ramp);
    }
    inv_freq_out[i] = f;
  }
  if (mscale_out) *mscale_out = kind == ESPO_ROPE_BY_PARTS ? static_cast<float>(0.1 * log(factor) + 1.0) : 1.0f;
  return ESPO_OK;
}

int espo_kv_append(const espo_kv_cache* cache, const espo_rope* rope, const void* key, int64_t key_stride,
                   const void* value, int64_t value_stride, int32_t dtype, const int32_t* cache_slots,
                   const int32_t* positions, int32_t n_tokens, const void* q, int64_t q_stride, int32_t n_q_heads,
                   void* q_out, int64_t q_out_stride, uint32_t* status_out, void* stream) {
  const int rc = check_append(cache, rope, key, key_stride, value, value_stride, dtype, n_tokens, q, q_stride, n_q_heads,
                              q_out, q_out_stride, status_out);
  if (rc != ESPO_OK) return rc;
  if (n_tokens > 0 && (!cache_slots || (rope && !positions))) return ESPO_ERR_NULL;
  if (!aligned(cache_slots, 4) || !aligned(positions, 4)) return ESPO_ERR_ALIGN;
  if (n_tokens == 0) return ESPO_OK;
  AppendArgs a = pack_append(cache, rope, key, key_stride, value, value_stride, n_tokens, q, q_stride, n_q_heads, q_out,
                             q_out_stride, status_out);
  a.cache_slots = cache_slots;
  a.positions = positions;
  return dispatch_append<false>(a, dtype, static_cast<cudaStream_t>(stream));
}

int espo_kv_append_rows(const espo_kv_cache* cache, const espo_rope* rope, const void* key, int64_t key_stride,
                        const void* value, int64_t value_stride, int32_t dtype, const espo_sequences* seqs,
                        const int32_t* row_ids, int32_t n_rows, const void* q, int64_t q_stride, int32_t n_q_heads,
                        void* q_out, int64_t q_out_stride, uint32_t* status_out, void* stream) {
  int rc = check_append(cache, rope, key, key_stride, value, value_stride, dtype, n_rows, q, q_stride, n_q_heads, q_out,
                        q_out_stride, status_out);
  if (rc != ESPO_OK) return rc;
  rc = check_sequences(seqs);
  if (rc != ESPO_OK) return rc;
  if (!aligned(row_ids, 4)) return ESPO_ERR_ALIGN;
  if (n_rows > seqs->capacity) return ESPO_ERR_CAPACITY;
  if (n_rows == 0) return ESPO_OK;
  AppendArgs a = pack_append(cache, rope, key, key_stride, value, value_stride, n_rows, q, q_stride, n_q_heads, q_out,
                             q_out_stride, status_out);
  a.seqs = *seqs;
  a.row_ids = row_ids;
  return dispatch_append<true>(a, dtype, static_cast<cudaStream_t>(stream));
}

int espo_kv_gather(const espo_kv_cache* cache, const int32_t* cache_slots, int32_t n_tokens, void* k_out, void* v_out,
                   int32_t dtype, uint32_t* status_out, void* stream) {
  const int rc = check_kv_cache(cache);
  if (rc != ESPO_OK) return rc;
  if (n_tokens < 0) return ESPO_ERR_BAD_SHAPE;
  if (n_tokens > 0 && !cache_slots) return ESPO_ERR_NULL;
  if (dtype != ESPO_F32 && dtype != ESPO_BF16) return ESPO_ERR_BAD_DTYPE;
  if (!aligned(cache_slots, 4) || !aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(status_out, 4)) return ESPO_ERR_ALIGN;
  if (n_tokens == 0 || (!k_out && !v_out)) return ESPO_OK;
  GatherArgs a = {*cache, cache_slots, k_out, v_out, status_out, n_tokens};
  const int grid = std::min((n_tokens - 1) / 8 + 1, 148 * 64);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool e = cache->dtype == ESPO_E4M3;
  if (dtype == ESPO_F32) {
    if (e) gather_kernel<float, true><<<grid, 256, 0, st>>>(a);
    else gather_kernel<float, false><<<grid, 256, 0, st>>>(a);
  } else {
    if (e) gather_kernel<__nv_bfloat16, true><<<grid, 256, 0, st>>>(a);
    else gather_kernel<__nv_bfloat16, false><<<grid, 256, 0, st>>>(a);
  }
  ESPO_CUDA_TRY(cudaGetLastError());
  return ESPO_OK;
}

}  // extern "C"
