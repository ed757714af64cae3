// Values in 8 bits (e4m3) with a power of two for each block of 128, as hm_quantize_* write and the experts' products
// read them: where things lie, and the rounding.
#pragma once

#include "hm_device.h"

namespace hm {

constexpr int kBlock8 = 128;   // values of a block

// Bytes of a row of C values, and bytes of a row's scales.
__host__ __device__ static inline int64_t row8_bytes(int64_t C) { return (C + 127) / 128 * 128; }
__host__ __device__ static inline int64_t scale8_bytes(int64_t C) { return (C + 511) / 512 * 4; }
__host__ __device__ static inline int64_t blocks8(int64_t C) { return (C + 127) / 128; }
// Blocks in the columns layout of `rows` rows in `segments` segments, and a segment's first: never below the blocks of
// the segments before it, whose ceilings add up to at most offset / 128 + segment.
__host__ __device__ static inline int64_t column8_blocks(int64_t rows, int64_t segments) {
  return rows / 128 + segments;
}
__device__ __forceinline__ int first_block8(int offset, int segment) { return offset / 128 + segment; }

// Rows of a segment, kept inside [0,rows] whatever the offsets say.
struct Segment8 {
  int from, to;
};
__device__ __forceinline__ Segment8 segment8(const int32_t *__restrict__ offsets, int segment, int rows) {
  const int from = min(max(offsets[segment], 0), rows);
  return {from, min(max(offsets[segment + 1], from), rows)};
}

constexpr uint32_t kInfinityBits = 0x7F800000u;

// Scale code of a block whose largest finite value has these bits: the least exponent e with amax <= 448 * 2^e, + 127.
// 448 = 1.75 * 2^8, so the mantissa decides between two.
__device__ __forceinline__ int scale_code8(uint32_t amax_bits) {
  return max((int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0), 0);
}
// 2^(127 - code): what a block's values are multiplied by; normal for every code that scale_code8 gives.
__device__ __forceinline__ float inverse_scale8(int code) {
  return __builtin_bit_cast(float, (uint32_t)(254 - code) << 23);
}

// Largest magnitude among a thread's values of a block, as bits: those order as the magnitudes do.  NaN and infinities,
// which are seen by bits that are too large, do not count and become NaN.
template <int N>
__device__ __forceinline__ uint32_t largest_bits(float (&v)[N]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) most = max(most, __builtin_bit_cast(uint32_t, v[i]) & 0x7FFFFFFFu);
  if (most >= kInfinityBits) {
    most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t bits = __builtin_bit_cast(uint32_t, v[i]) & 0x7FFFFFFFu;
      if (bits >= kInfinityBits) v[i] = __builtin_nanf("");
      else most = max(most, bits);
    }
  }
  return most;
}
// Four values times a power of two, rounded to nearest even, in order.
__device__ __forceinline__ uint32_t pack8(float a, float b, float c, float d, float by) {
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a * by, b * by, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * by, d * by, low, true);
}

typedef f32x4 f32x4_align4 __attribute__((aligned(4)));
typedef uint32_t u32x2_align2 __attribute__((ext_vector_type(2), aligned(2)));
// N = 4 or 8 consecutive elements as fp32; any alignment of the elements.
template <int N>
__device__ __forceinline__ void load_floats(const uint16_t *__restrict__ p, float (&v)[N]) {
  uint32_t w[N / 2];
  if constexpr (N == 8) {
    const u32x4 t = *(const u32x4_align2 *)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = t[i];
  } else {
    const u32x2_align2 t = *(const u32x2_align2 *)p;
    w[0] = t[0];
    w[1] = t[1];
  }
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    v[2 * i] = bf16_lo(w[i]);
    v[2 * i + 1] = bf16_hi(w[i]);
  }
}
template <int N>
__device__ __forceinline__ void load_floats(const float *__restrict__ p, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x4 t = *(const f32x4_align4 *)(p + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i + j] = t[j];
  }
}
__device__ __forceinline__ float load_float(const uint16_t *p) { return bf16_lo(*p); }
__device__ __forceinline__ float load_float(const float *p) { return *p; }
// Elements c to c + N - 1 of a row of C, zeros behind its end.  A vector that would pass the end is loaded from before
// it and moved down: loads one by one, each waited for, cost a kernel's tail 10 us.
template <int N, typename IN>
__device__ __forceinline__ void load_row_end(const IN *__restrict__ row, int c, int C, float (&v)[N]) {
  if (C < N) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = c + i < C ? load_float(row + c + i) : 0.0f;
    return;
  }
  const int at = min(c, C - N), by = c - at;
  load_floats<N>(row + at, v);
#pragma unroll
  for (int bit = 1; bit < N; bit *= 2)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = by & bit ? (i + bit < N ? v[i + bit] : 0.0f) : v[i];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = by < N ? v[i] : 0.0f;
}

static inline bool buffers8_aligned(const void *q, const void *scale) {
  return ((uintptr_t)q & 15) == 0 && ((uintptr_t)scale & 3) == 0;
}
static inline bool dtype_known(hm_dtype dtype) { return dtype == HM_BF16 || dtype == HM_F32; }
constexpr int kMostSegments8 = 1024, kMostColumns8 = 1 << 20;
// Sizes of rows ordered by expert, common to the calls that take offsets.
static inline bool segments8_ok(int32_t segments, int64_t rows) {
  return segments >= 1 && segments <= kMostSegments8 && rows >= 0 && rows <= 2147483647LL - 128LL * segments;
}

}  // namespace hm
