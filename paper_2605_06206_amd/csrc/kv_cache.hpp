// Device helpers of the 8-bit key/value cache (layouts and rules in foe.h).
#pragma once

#include "foe_common.hpp"

namespace foe {

constexpr int kPage = FOE_CACHE_PAGE;      // tokens per page
constexpr int kSub = 16;                   // tokens per group of the value layout
// from this magnitude on the code nearest to a value, 256 * 2^120, stands for 2^128
constexpr float kTooLarge = 0x1.fp127f;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// 8 e4m3 codes times a power of two, as bf16: both conversions are exact (four
// significant bits, and bf16 has the exponents), so the products of the matrix
// instructions see the cache's own values.
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// four values (at most 448 in magnitude, or NaN) as e4m3, nearest even
__device__ __forceinline__ uint32_t to_codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// four codes in units of another scale (ratio = old / new); exact unless a
// value falls among the new scale's subnormals.  The codes of a key that is not
// finite (all NaN) stay as they are, sign and all.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float ratio) {
  if ((w & 0x7f7f7f7fu) == 0x7f7f7f7fu) return w;
  return to_codes4(__builtin_amdgcn_cvt_f32_fp8(w, 0) * ratio,
                   __builtin_amdgcn_cvt_f32_fp8(w, 1) * ratio,
                   __builtin_amdgcn_cvt_f32_fp8(w, 2) * ratio,
                   __builtin_amdgcn_cvt_f32_fp8(w, 3) * ratio);
}

// Smallest power of two s >= 2^-100 with amax <= 448 s (amax finite, >= 0):
// 448 = 1.75 * 2^8, so with amax = f * 2^E, 1 <= f < 2, it is 2^(E-8) up to
// f = 1.75 and 2^(E-7) above.
__device__ __forceinline__ float block_scale(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)max(e, 127 - 100) << 23);
}
// 1 / s of a power of two
__device__ __forceinline__ float pow2_inv(float s) {
  return __uint_as_float((254u << 23) - __float_as_uint(s));
}
// old / new scale.  Where it passes fp32, the codes that it multiplies are zeros or NaN
// (others, at least 2^-9, would have made the new scale larger), and 0 * inf is NaN.
__device__ __forceinline__ float scale_ratio(float old, float inv_new) {
  return fminf(old * inv_new, 0x1p127f);
}

// A call's sequences.  Lengths and tables are the caller's device data and are
// not trusted: rows are cut to the batch, lengths to the table, and pages
// outside the pool count as absent.
struct CacheBatch {
  int H, B, N, nq, n_pages, max_blocks;
  const int32_t* table;      // [B][max_blocks]
  const int32_t* ctx;        // [B]
  const int32_t* row_start;  // [B + 1]

  __device__ __forceinline__ int cap() const { return max_blocks * kPage; }
  __device__ __forceinline__ int context(int b) const { return min(max(ctx[b], 0), cap()); }
  __device__ __forceinline__ int first_row(int b) const { return min(max(row_start[b], 0), N); }
  __device__ __forceinline__ int rows(int b) const {
    return max(min(max(row_start[b + 1], 0), N) - first_row(b), 0);
  }
  __device__ __forceinline__ int page(int b, int blk) const {
    const int p = blk < max_blocks ? table[(size_t)b * max_blocks + blk] : -1;
    return p >= 0 && p < n_pages ? p : -1;
  }
};

// Sequence b and tile `local` of it that tile number `tile` of the batch is,
// when sequence b has count(b) >= 0 tiles: every thread of the workgroup calls
// this; false past the last tile.
template <int NT, typename Count>
__device__ __forceinline__ bool find_tile(int B, int tile, Count count, int& b, int& local) {
  constexpr int NW = NT / kWave;
  __shared__ int wave_sum[NW];
  __shared__ int found[2];
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) found[0] = -1;
  int before = 0;
  for (int base = 0; base < B; base += NT) {
    const int i = base + (int)threadIdx.x;
    const int c = i < B ? count(i) : 0;
    int incl = c;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int up = __shfl_up(incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == kWave - 1) wave_sum[wave] = incl;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if (w < wave) incl += wave_sum[w];
      total += wave_sum[w];
    }
    const int t = tile - before;
    if (t >= incl - c && t < incl) {
      found[0] = i;
      found[1] = t - (incl - c);
    }
    before += total;
    __syncthreads();
    if (tile < before) break;
  }
  __syncthreads();
  b = found[0];
  local = found[1];
  return b >= 0;
}

// largest value of a workgroup of NT threads, in every thread
template <int NT>
__device__ __forceinline__ float2 block_max(float2 v) {
  constexpr int NW = NT / kWave;
  __shared__ float2 part[NW];
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) {
    v.x = fmaxf(v.x, __shfl_xor(v.x, o));
    v.y = fmaxf(v.y, __shfl_xor(v.y, o));
  }
  if (lane_id() == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) {
    v.x = fmaxf(v.x, part[w].x);
    v.y = fmaxf(v.y, part[w].y);
  }
  return v;
}

}  // namespace foe
