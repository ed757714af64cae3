// The norm in front of a layer: s = x + residual, y = s m^-1/2 w with m = mean(s^2) + eps, as values and in 8 bits, and the
// way back:
//     u = gy w,   gs = m^-1/2 (u - s mean(u s) / m) + gtotal,   gw = sum over the rows of gy s m^-1/2.
// Both need a row's sums before they can write the row, so a row stays in registers between: THREADS threads have VEC
// vectors of eight values of it, the k-th of thread i being vector k THREADS + i.  A wave's vectors are 512 neighbouring
// columns, four blocks of 8 bits.  Memory bounds both: 8,192 rows of 7,168 bf16 with a residual, values and 8 bits written, take
// 106 us (528 MB, 5.0 TB/s; a copy of it 103), with an fp32 residual 146 (764 MB; 149), all in fp32 166 (881 MB; 172); the way back 97
// (470 MB, 4.9 TB/s; 92), in fp32 155 (822 MB; 160).  One row is a launch, a trip to memory and a barrier (4.3 us).
#include "hm_block8.h"

namespace hm {

constexpr int kMostNormColumns = 32768;   // 1,024 threads of four vectors

struct NormParams {
  const void *x, *residual, *weight;
  void *total, *y;
  uint8_t *q, *scale;
  int64_t ld, residual_ld, total_ld, rows;
  int32_t C;
  float eps;
  bool weight_bf16, y_bf16;
};

// The sums over a row's threads, in all of them; `sums` has a place for every wave, another one from call to call, so that one
// barrier is enough.  Lanes add in fp32, waves in 64 bits.
template <int THREADS, int N>
__device__ __forceinline__ void row_sums(const float (&v)[N], float (&sums)[2][N][THREADS / kWave], int turn, double (&sum)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const float s = wave_sum(v[n]);
    if constexpr (THREADS > kWave) {
      if (lane_id() == 0) sums[turn][n][threadIdx.x / kWave] = s;
    } else {
      sum[n] = (double)s;
    }
  }
  if constexpr (THREADS > kWave) {
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      sum[n] = 0.0;
#pragma unroll
      for (int w = 0; w < THREADS / kWave; ++w) sum[n] += (double)sums[turn][n][w];
    }
  }
}
// m^-1/2 and what it is short of the exact value, from one step of Newton's in 64 bits: every value of a row would share its error.
// With it a value is rounded once, where the root's, the product's and the weight's roundings would be three.
struct Inverse {
  float root, rest;
};
__device__ __forceinline__ Inverse inverse_root(double m) {
  const float r = 1.0f / sqrtf((float)m);
  const float rest = r * (float)(0.5 * (1.0 - m * (double)r * (double)r));
  return {r, fabsf(rest) < __builtin_inff() ? rest : 0.0f};   // none of 0 and of what is no number
}

// A vector of the weight of either type.
__device__ __forceinline__ void load_weight(const void *weight, bool bf16, int c, int C, float (&v)[8]) {
  if (bf16) load_row_end<8>((const uint16_t *)weight, c, C, v);
  else load_row_end<8>((const float *)weight, c, C, v);
}

// Threads of a workgroup: a row's, or four rows of a wave each.
template <int THREADS>
constexpr int norm_block() { return THREADS < 256 ? 256 : THREADS; }

// 8,192 rows of 7,168 take 84 registers (99 with an fp32 residual), five (four) waves a SIMD; held to 80 for six they spilled 20 (68) bytes a
// thread: 111 (168) us instead of 106 (146), of 5,000 columns 97 (144) and 90 (117).
template <typename IN, typename SUM, int VEC, int THREADS>
__global__ __launch_bounds__(norm_block<THREADS>()) void rms_norm_kernel(NormParams p) {
  constexpr int kRows = norm_block<THREADS>() / THREADS;   // of a workgroup
  __shared__ float sums[2][1][THREADS / kWave];
  const int tid = threadIdx.x % THREADS, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int first_part = THREADS < 256 ? 0 : wave;   // the wave's pieces of 512 columns: this one, and every kStep-th behind it
  constexpr int kStep = THREADS / kWave;
  const int width = (int)row8_bytes(p.C);
  float w[VEC][8];
#pragma unroll
  for (int k = 0; k < VEC; ++k) load_weight(p.weight, p.weight_bf16, (k * THREADS + tid) * 8, p.C, w[k]);
  const double per_C = 1.0 / (double)p.C;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (THREADS < 256 ? wave : 0); row < p.rows; row += (int64_t)gridDim.x * kRows) {
    float v[VEC][8], squares[1] = {0.0f};
    const IN *x = (const IN *)p.x + row * p.ld;
    Eight<IN> own[VEC];   // as they were loaded: half the registers of fp32
    Eight<SUM> add[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) own[k] = eight_of_row(x, (k * THREADS + tid) * 8, p.C, (first_part + k * kStep) * 512 + 512 <= p.C);
    if (p.residual) {
      const SUM *r = (const SUM *)p.residual + row * p.residual_ld;
#pragma unroll
      for (int k = 0; k < VEC; ++k) add[k] = eight_of_row(r, (k * THREADS + tid) * 8, p.C, (first_part + k * kStep) * 512 + 512 <= p.C);
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] = p.residual ? own[k].at(i) + add[k].at(i) : own[k].at(i);
      if (p.residual) round_to((const SUM *)nullptr, v[k]);   // what is normed is the sum as it is kept, so that the way back sees the same
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) squares[0] = fmaf(v[k][i], v[k][i], squares[0]);
    double sum[1];
    row_sums<THREADS>(squares, sums, turn, sum);
    turn ^= 1;
    const Inverse by = inverse_root(sum[0] * per_C + (double)p.eps);
    // Stores come behind the barrier: outputs may take the place of the row's inputs, of which a thread at a row's end reads more
    // than it has.
    if (p.residual) {
      SUM *total = (SUM *)p.total + row * p.total_ld;
#pragma unroll
      for (int k = 0; k < VEC; ++k) store_row(total, (k * THREADS + tid) * 8, p.C, v[k]);
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const int c = (k * THREADS + tid) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {   // one rounding in the end, for three instructions more
        const float normed = v[k][i] * by.root, rest = fmaf(v[k][i], by.rest, fmaf(v[k][i], by.root, -normed));
        v[k][i] = fmaf(normed, w[k][i], rest * w[k][i]);
      }
      if (p.y) {
        if (p.y_bf16) store_row((uint16_t *)p.y + row * p.C, c, p.C, v[k]);
        else store_row((float *)p.y + row * p.C, c, p.C, v[k]);
      }
      const int part = first_part + k * kStep;
      if (p.q && part * 512 < p.C) store_piece8(p.q + row * width, p.scale + row * scale8_bytes(p.C), part, width, v[k]);
    }
  }
}

struct NormBackParams {
  const void *gy, *s, *weight, *gtotal;
  void *gx;
  float *gweight;   // of the weight, or parts [groups, C] of it
  int64_t gy_ld, s_ld, gtotal_ld, gx_ld, rows;
  int32_t C, groups;
  float eps;
  bool weight_bf16;
};

// THREADS threads are a group, which takes every groups-th row and adds up its part of the weight's gradient in registers; the parts
// are added up in order by a second launch (5 us for 512 of 7,168 columns), so the result does not depend on who is first.  With a
// row in fp32 registers half as many waves fit a CU: 160 us for 8,192 rows, 92 as it is; with the next row on its way the same.
template <typename GY, typename IN, int VEC, int THREADS>
__global__ __launch_bounds__(norm_block<THREADS>()) void rms_norm_backward_kernel(NormBackParams p) {
  constexpr int kGroups = norm_block<THREADS>() / THREADS;   // of a workgroup
  __shared__ float sums[2][2][THREADS / kWave];
  const int tid = threadIdx.x % THREADS, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int group = (int)blockIdx.x * kGroups + (THREADS < 256 ? wave : 0);
  if (group >= p.groups) return;   // whole waves; workgroups of one group have none too many
  const int first_part = THREADS < 256 ? 0 : wave;
  constexpr int kStep = THREADS / kWave;
  float w[VEC][8], gw[VEC][8];
#pragma unroll
  for (int k = 0; k < VEC; ++k) {
    load_weight(p.weight, p.weight_bf16, (k * THREADS + tid) * 8, p.C, w[k]);
#pragma unroll
    for (int i = 0; i < 8; ++i) gw[k][i] = 0.0f;
  }
  const double per_C = 1.0 / (double)p.C;
  int turn = 0;
  for (int64_t row = group; row < p.rows; row += p.groups) {
    Eight<IN> s[VEC], t[VEC];   // as they were loaded: half the registers of fp32, for twice the waves
    Eight<GY> g[VEC];
    float parts[2] = {0.0f, 0.0f};
    const IN *from_s = (const IN *)p.s + row * p.s_ld, *from_t = (const IN *)p.gtotal + row * p.gtotal_ld;
    const GY *from_g = (const GY *)p.gy + row * p.gy_ld;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const bool whole = (first_part + k * kStep) * 512 + 512 <= p.C;
      s[k] = eight_of_row(from_s, (k * THREADS + tid) * 8, p.C, whole);
      g[k] = eight_of_row(from_g, (k * THREADS + tid) * 8, p.C, whole);
      if (p.gtotal) t[k] = eight_of_row(from_t, (k * THREADS + tid) * 8, p.C, whole);
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        parts[0] = fmaf(s[k].at(i), s[k].at(i), parts[0]);
        parts[1] = fmaf(g[k].at(i) * w[k][i], s[k].at(i), parts[1]);
      }
    double sum[2];
    row_sums<THREADS>(parts, sums, turn, sum);
    turn ^= 1;
    const float by = 1.0f / sqrtf((float)(sum[0] * per_C + (double)p.eps)), mean = by * by * (float)(sum[1] * per_C);
    IN *gx = (IN *)p.gx + row * p.gx_ld;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      s[k].forget();
      g[k].forget();
      float out[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = s[k].at(i), u = g[k].at(i);
        gw[k][i] = fmaf(u, v * by, gw[k][i]);
        out[i] = by * (u * w[k][i] - v * mean);
        if (p.gtotal) out[i] += t[k].at(i);
      }
      store_row(gx, (k * THREADS + tid) * 8, p.C, out);
    }
  }
  if (p.gweight) {
    float *to = p.gweight + (int64_t)group * p.C;
#pragma unroll
    for (int k = 0; k < VEC; ++k) store_row(to, (k * THREADS + tid) * 8, p.C, gw[k]);
  }
}

// The parts of the weight's gradient added up: a workgroup takes 64 columns, a wave every 16th part in four sums of fp32, and the sums
// are added up in 64 bits.  One sum a wave, and theirs in fp32: 1,237 x 1,030 off by 1.5e-7 of its norm, now by 0.9e-7, in
// the same time.
constexpr int kPartWaves = 16, kPartSums = 4;
__global__ __launch_bounds__(kPartWaves * kWave) void rms_norm_weight_grad_kernel(const float *__restrict__ parts, int groups, int C,
                                                                                  float *__restrict__ gweight) {
  __shared__ double sums[kPartWaves][kWave];
  const int lane = lane_id(), wave = threadIdx.x / kWave, c = (int)blockIdx.x * kWave + lane;
  float sum[kPartSums] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c < C) {
    int g = wave;
#pragma unroll 2
    for (; g + (kPartSums - 1) * kPartWaves < groups; g += kPartSums * kPartWaves) {
#pragma unroll
      for (int i = 0; i < kPartSums; ++i) sum[i] += parts[(int64_t)(g + i * kPartWaves) * C + c];
    }
    for (; g < groups; g += kPartWaves) sum[0] += parts[(int64_t)g * C + c];
  }
  sums[wave][lane] = ((double)sum[0] + (double)sum[1]) + ((double)sum[2] + (double)sum[3]);
  __syncthreads();
  if (wave == 0 && c < C) {
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < kPartWaves; ++w) all += sums[w][lane];
    gweight[c] = (float)all;
  }
}

// Groups of rows that have a part of the weight's gradient each.  More hide each other's trips to memory, and are more parts to add
// up: 8,192 x 7,168 with 256, 512 and 1,024 113 + 5, 100 + 5 and 105 + 9 us, 1,237 x 1,030 fp32 11.5 + 3.9, 9.3 + 4.0 and 8.6 + 5.8.
// Short rows have a wave each, four to a workgroup.
static int norm_groups(int64_t rows, int32_t C) {
  const int64_t most = C <= 1024 ? 1024 : 512;
  return (int)(rows < most ? rows : most);
}

// Calls launch(vectors, threads) with the threads of a row and the vectors that each has of it.  Few rows leave most CUs without
// one, and the fewer vectors a thread has the sooner a row is done; many rows hide each other's trips to memory, and a row of fewer
// waves waits less for its own.  us forward (back), bf16 with a residual, few's shape against many's: one row of 1,024 3.1 (3.3) and 3.7
// (3.2), of 7,168 4.3 (4.5) and 5.1 (5.1); 512 rows 4.2 (8.1) and 4.4 (8.1), 10.0 (17.1) and 10.0 (17.9); 1,024 rows 5.2 (11.4) and
// 4.8 (11.2), 17.5 (23.5) and 16.0 (21.0); 8,192 rows 19.8 (27.3) and 14.0 (21.2), 114 (108) and 106 (97).  One wave a row up to 512
// columns: 8,192 rows 8.7 (16.0), two vectors of it 13.0 (23.8).  Between 8,193 and 16,384 columns 512 threads of four vectors take
// one row 7.3 (6.7), two of 1,024 6.0 (5.8), and 8,192 of 16,384 231 (212) and 220 (207).  Beyond, 1,024 threads are all there
// are: 32 values of a thread, which on the way back, with weight, gradient and two or three rows, pass its 128 registers by 180 to 300 bytes.  Of
// 32,768 columns one row takes 10.5 (18.9), in fp32 12.6 (27.1); 4,096 rows 234 (344), in fp32 411 (708), where copies take 236 (209)
// and 393 (366).
template <typename LAUNCH>
static void norm_shape(int64_t rows, int32_t C, LAUNCH launch) {
#define HM_NORM_SHAPE(v, t) launch(std::integral_constant<int, v>(), std::integral_constant<int, t>())
  const bool few = rows <= 512;
  if (C <= 512) HM_NORM_SHAPE(1, 64);
  else if (C <= 1024 && !few) HM_NORM_SHAPE(2, 64);
  else if (C <= 2048) HM_NORM_SHAPE(1, 256);
  else if (C <= 4096) HM_NORM_SHAPE(1, 512);
  else if (C <= 8192 && !few) HM_NORM_SHAPE(2, 512);
  else if (C <= 8192) HM_NORM_SHAPE(1, 1024);
  else if (C <= 16384) HM_NORM_SHAPE(2, 1024);
  else HM_NORM_SHAPE(4, 1024);
#undef HM_NORM_SHAPE
}

template <typename IN, typename SUM>
static void launch_norm(const NormParams &p, hipStream_t stream) {
  norm_shape(p.rows, p.C, [&](auto vec, auto threads) {
    constexpr int kRows = norm_block<threads()>() / threads();
    const int64_t blocks = (p.rows + kRows - 1) / kRows;
    hipLaunchKernelGGL((rms_norm_kernel<IN, SUM, vec(), threads()>), dim3((unsigned)(blocks < 2048 ? blocks : 2048)),
                       dim3(norm_block<threads()>()), 0, stream, p);
  });
}
template <typename GY, typename IN>
static void launch_norm_backward(const NormBackParams &p, hipStream_t stream) {
  norm_shape(p.rows, p.C, [&](auto vec, auto threads) {
    constexpr int kGroups = norm_block<threads()>() / threads();
    hipLaunchKernelGGL((rms_norm_backward_kernel<GY, IN, vec(), threads()>), dim3((unsigned)((p.groups + kGroups - 1) / kGroups)),
                       dim3(norm_block<threads()>()), 0, stream, p);
  });
}

}  // namespace hm

extern "C" hm_status hm_rms_norm(const void *x, hm_dtype dtype, int64_t ld, const void *residual, hm_dtype total_dtype,
                                 int64_t residual_ld, const void *weight, hm_dtype weight_dtype, float eps, int64_t rows, int32_t C,
                                 void *total, int64_t total_ld, void *y, hm_dtype y_dtype, uint8_t *q, uint8_t *scale,
                                 void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!dtype_known(dtype) || !dtype_known(total_dtype) || !dtype_known(weight_dtype) || !dtype_known(y_dtype)) return HM_ERR_SHAPE;
  if (rows < 0 || rows > 2147483647LL || C < 1 || C > kMostNormColumns || !(eps >= 0.0f)) return HM_ERR_SHAPE;
  if (rows > 1 && (ld < C || (residual && (residual_ld < C || total_ld < C)))) return HM_ERR_SHAPE;
  if (!aligned_as(dtype, x) || !aligned_as(total_dtype, residual) || !aligned_as(total_dtype, total)) return HM_ERR_SHAPE;
  if (!aligned_as(weight_dtype, weight) || !aligned_as(y_dtype, y) || !buffers8_aligned(q, scale)) return HM_ERR_SHAPE;
  if (rows == 0) return HM_OK;
  if (!residual != !total || !q != !scale || (!y && !q)) return HM_ERR_NULL;
  if (!x || !weight) return HM_ERR_NULL;
  const NormParams p = {x, residual, weight, total, y, q, scale, ld, residual_ld, total_ld, rows, C, eps, weight_dtype == HM_BF16,
                        y_dtype == HM_BF16};
  const hipStream_t stream = (hipStream_t)hip_stream;
  const bool same = !residual || total_dtype == dtype;   // without a residual its type is not looked at
  if (dtype == HM_BF16) same ? launch_norm<uint16_t, uint16_t>(p, stream) : launch_norm<uint16_t, float>(p, stream);
  else same ? launch_norm<float, float>(p, stream) : launch_norm<float, uint16_t>(p, stream);
  return hm_launch_status();
}

extern "C" size_t hm_rms_norm_backward_workspace_bytes(int64_t rows, int32_t C) {
  if (rows < 0 || C < 1 || C > hm::kMostNormColumns) return 0;
  const int groups = hm::norm_groups(rows, C);
  return groups > 1 ? (size_t)groups * C * 4 : 0;
}

extern "C" hm_status hm_rms_norm_backward(const void *gy, hm_dtype gy_dtype, int64_t gy_ld, const void *s, hm_dtype dtype,
                                          int64_t s_ld, const void *weight, hm_dtype weight_dtype, float eps, int64_t rows,
                                          int32_t C, const void *gtotal, int64_t gtotal_ld, void *gx, int64_t gx_ld,
                                          float *gweight, void *workspace, size_t workspace_bytes, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!dtype_known(gy_dtype) || !dtype_known(dtype) || !dtype_known(weight_dtype)) return HM_ERR_SHAPE;
  if (rows < 0 || rows > 2147483647LL || C < 1 || C > kMostNormColumns || !(eps >= 0.0f)) return HM_ERR_SHAPE;
  if (rows > 1 && (gy_ld < C || s_ld < C || gx_ld < C || (gtotal && gtotal_ld < C))) return HM_ERR_SHAPE;
  if (!aligned_as(gy_dtype, gy) || !aligned_as(dtype, s) || !aligned_as(weight_dtype, weight)) return HM_ERR_SHAPE;
  if (!aligned_as(dtype, gtotal) || !aligned_as(dtype, gx) || ((uintptr_t)gweight & 3)) return HM_ERR_SHAPE;
  if (!gweight) return HM_ERR_NULL;
  NormBackParams p = {gy, s, weight, gtotal, gx, gweight, gy_ld, s_ld, gtotal_ld, gx_ld, rows, C, norm_groups(rows, C), eps,
                      weight_dtype == HM_BF16};
  const hipStream_t stream = (hipStream_t)hip_stream;
  const bool parts = p.groups != 1;   // no rows: the sum of no parts
  if (rows > 0) {
    if (!gy || !s || !weight || !gx) return HM_ERR_NULL;
    if (parts) {
      if (!workspace || workspace_bytes < hm_rms_norm_backward_workspace_bytes(rows, C) || ((uintptr_t)workspace & 15))
        return HM_ERR_WORKSPACE;
      p.gweight = (float *)workspace;
    }
    if (gy_dtype == HM_BF16) dtype == HM_BF16 ? launch_norm_backward<uint16_t, uint16_t>(p, stream)
                                              : launch_norm_backward<uint16_t, float>(p, stream);
    else dtype == HM_BF16 ? launch_norm_backward<float, uint16_t>(p, stream) : launch_norm_backward<float, float>(p, stream);
    const hm_status launched = hm_launch_status();
    if (launched != HM_OK || !parts) return launched;
  }
  hipLaunchKernelGGL(rms_norm_weight_grad_kernel, dim3((unsigned)((C + kWave - 1) / kWave)), dim3(kPartWaves * kWave), 0, stream,
                     (const float *)workspace, p.groups, C, gweight);
  return hm_launch_status();
}
