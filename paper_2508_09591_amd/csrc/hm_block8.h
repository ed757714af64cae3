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

// The segment that owns block b, the last whose first block is not behind it, and its rows; called by whole waves.
// Both offsets of a lane's segment are loaded together: what follows waits for one trip to memory.
struct BlockOwner8 {
  int segment;   // -1: none
  Segment8 rows;
};
__device__ __forceinline__ BlockOwner8 owner_of_block8(const int32_t *__restrict__ offsets, int segments, int rows,
                                                       int b) {
  const int lane = lane_id();
  BlockOwner8 owner = {-1, {0, 0}};
  for (int e0 = 0; e0 < segments; e0 += kWave) {
    const int e = e0 + lane;
    const Segment8 s = segment8(offsets, min(e, segments - 1), rows);
    const uint64_t upto = __ballot(e < segments && first_block8(s.from, e) <= b);
    if (upto == 0) break;
    const int l = 63 - __builtin_clzll(upto);
    owner = {e0 + l, {read_lane(s.from, l), read_lane(s.to, l)}};
  }
  return owner;
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

// Largest value of the sixteen lanes of a row, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, true));
}

// Eight values a lane of the 512 columns from 512 `part` on of a row in 8 bits: the row's bytes, `width` of them, and its
// scales; sixteen lanes have a block.  What lies behind the row's end is zero.  Called by whole waves.
__device__ __forceinline__ void store_piece8(uint8_t *q, uint8_t *scale, int part, int width, float (&v)[8]) {
  const int lane = lane_id(), c = part * 512 + lane * 8;
  const int code = scale_code8(max16(largest_bits(v)));
  const float by = inverse_scale8(code);
  if (c < width)
    *(uint64_t *)(q + c) = (uint64_t)pack8(v[4], v[5], v[6], v[7], by) << 32 | pack8(v[0], v[1], v[2], v[3], by);
  const uint32_t mine = c < width ? (uint32_t)code : 0u;   // behind the last block zeros
  const uint32_t codes = (uint32_t)read_lane((int)mine, 0) | (uint32_t)read_lane((int)mine, 16) << 8 |
                         (uint32_t)read_lane((int)mine, 32) << 16 | (uint32_t)read_lane((int)mine, 48) << 24;
  if (lane == 0) *(uint32_t *)(scale + part * 4) = codes;
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

// Eight elements as they were loaded.
template <typename IN>
struct Eight;
template <>
struct Eight<uint16_t> {
  u32x4 w;
  Eight() = default;
  __device__ __forceinline__ explicit Eight(const uint16_t *p) : w(*(const u32x4_align2 *)p) {}
  __device__ __forceinline__ float at(int i) const { return i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]); }
  // What has been computed from them is forgotten, not kept in registers.
  __device__ __forceinline__ void forget() { __asm__("" : "+v"(w)); }
  __device__ __forceinline__ float times(const Eight &v, float sum) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = fmaf(bf16_hi(w[i]), bf16_hi(v.w[i]), fmaf(bf16_lo(w[i]), bf16_lo(v.w[i]), sum));
    return sum;
  }
};
template <>
struct Eight<float> {
  f32x4 a, b;
  Eight() = default;
  __device__ __forceinline__ explicit Eight(const float *p)
      : a(*(const f32x4_align4 *)p), b(*(const f32x4_align4 *)(p + 4)) {}
  __device__ __forceinline__ float at(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ __forceinline__ void forget() { __asm__("" : "+v"(a), "+v"(b)); }
  __device__ __forceinline__ float times(const Eight &v, float sum) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = fmaf(b[i], v.b[i], fmaf(a[i], v.a[i], sum));
    return sum;
  }
};
// Those of a row of C from column c on, zeros behind its end; `whole` (uniform): none of the wave's reach it.
__device__ __forceinline__ Eight<uint16_t> eight_of_row(const uint16_t *__restrict__ row, int c, int C, bool whole) {
  if (whole) return Eight<uint16_t>(row + c);
  float v[8];
  load_row_end<8>(row, c, C, v);
  Eight<uint16_t> e;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    e.w[i] = __builtin_bit_cast(uint32_t, v[2 * i]) >> 16 | (__builtin_bit_cast(uint32_t, v[2 * i + 1]) & 0xFFFF0000u);
  return e;
}
__device__ __forceinline__ Eight<float> eight_of_row(const float *__restrict__ row, int c, int C, bool whole) {
  if (whole) return Eight<float>(row + c);
  float v[8];
  load_row_end<8>(row, c, C, v);
  Eight<float> e;
  e.a = f32x4{v[0], v[1], v[2], v[3]};
  e.b = f32x4{v[4], v[5], v[6], v[7]};
  return e;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
// Eight values as bf16, times their block's power of two, of which the conversion takes the exponent (code 0 too is
// 2^-127).  Exact down to the least subnormal, 2^-133: values are multiples of 2^-9, so that codes from 3 on lose
// nothing.  2^128, to which what lies next to fp32's largest number is rounded (256 under code 247), is infinite.
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, uint32_t code) {
  const float power = __builtin_bit_cast(float, (code & 0xFFu) << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, true);
  return {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// N consecutive elements, to nearest even; any alignment of the elements.
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t round_bf16x2(float lo, float hi) {   // two an instruction
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}
__device__ __forceinline__ void store_floats(uint16_t *p, const float (&v)[8]) {
  *(u32x4_align2 *)p = u32x4{round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3]), round_bf16x2(v[4], v[5]),
                             round_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void store_floats(uint16_t *p, const float (&v)[4]) {
  *(u32x2_align2 *)p = u32x2_align2{round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3])};
}
template <int N>
__device__ __forceinline__ void store_floats(float *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *(f32x4_align4 *)(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}
__device__ __forceinline__ void store_float(uint16_t *p, float v) { *p = (uint16_t)round_bf16x2(v, v); }
__device__ __forceinline__ void store_float(float *p, float v) { *p = v; }
// Elements c to c + N - 1 of a row of C.
template <int N, typename OUT>
__device__ __forceinline__ void store_row(OUT *row, int c, int C, const float (&v)[N]) {
  if (c + N <= C) {
    store_floats(row + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < C) store_float(row + c + i, v[i]);
  }
}
// The same loaded, zeros behind the row's end; `whole` (uniform): none of the wave's reach it.
template <typename IN>
__device__ __forceinline__ void load_row(const IN *__restrict__ row, int c, int C, bool whole, float (&v)[8]) {
  if (whole) load_floats<8>(row + c, v);
  else load_row_end<8>(row, c, C, v);
}
// Rounded to the type of OUT, as fp32.
__device__ __forceinline__ void round_to(const uint16_t *, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t w = round_bf16x2(v[i], v[i + 1]);
    v[i] = bf16_lo(w);
    v[i + 1] = bf16_hi(w);
  }
}
__device__ __forceinline__ void round_to(const float *, float (&)[8]) {}

static inline bool buffers8_aligned(const void *q, const void *scale) {
  return ((uintptr_t)q & 15) == 0 && ((uintptr_t)scale & 3) == 0;
}
static inline bool aligned_as(hm_dtype dtype, const void *at) {
  return ((uintptr_t)at & (dtype == HM_F32 ? 3 : 1)) == 0;
}
static inline bool dtype_known(hm_dtype dtype) { return dtype == HM_BF16 || dtype == HM_F32; }
constexpr int kMostSegments8 = 1024, kMostColumns8 = 1 << 20;
// Sizes of rows ordered by expert, common to the calls that take offsets.
static inline bool segments8_ok(int32_t segments, int64_t rows) {
  return segments >= 1 && segments <= kMostSegments8 && rows >= 0 && rows <= 2147483647LL - 128LL * segments;
}

}  // namespace hm
