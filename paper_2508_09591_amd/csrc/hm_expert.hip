// The experts' products in 8 bits: rows ordered by expert times their expert's weights, and the weights' gradient.
//
// Both are D[q][p] = sum_k Q[q][k] P[p][k] with operands whose rows run along k in blocks of 128 that have a power of two each.
//   rows:   Q = rows of a segment, P = the expert's weights, k = columns
//   dw:     Q = columns of gy, P = columns of x, k = rows of the segment, padded to whole blocks with zeros
//
// Two ways to sum.  The matrix unit's products of 8 bits (32 x 32 x 64) apply the powers of two by themselves, but align the
// products of a step to the largest and drop what lies more than 2^13 below it: 1.5e-5 of the result, a hundredth of what
// rounding to bf16 costs.  So bf16 results take them.  fp32 results have their operands turned into bf16 in registers, which is
// exact and takes the power of two along, and products of 16 bits, which are summed in 32 (1e-8 per step).
#include "hm_block8.h"

namespace hm {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct ProductParams {
  const uint8_t *q, *q_scale, *p, *p_scale;
  const int32_t *offsets;
  int32_t experts, rows, N, H;   // rows: D is [segment, N], k = H; dw: D is [N, H], k = rows of the segment
  void *out;
};

// Where a workgroup's tile lies.
struct Tile {
  int expert, q0, q_end, p0;   // first and last row of D, first column; q_end <= q0: none
};

// The tile of a workgroup among those of all segments, counted on the device: an expert's tiles lie together, the tiles of
// neighbouring rows next to one another, and every die gets a run of them, so that it reads few weights and rows.
template <int TQ, int TP>
__device__ __forceinline__ Tile tile_of_rows(const ProductParams &p) {
  const int lane = lane_id(), wide = (p.N + TP - 1) / TP;
  int total = 0;
  for (int e0 = 0; e0 < p.experts; e0 += kWave) {
    const int e = e0 + lane;
    const Segment8 s = segment8(p.offsets, min(e, p.experts - 1), p.rows);
    total += read_lane(lane_scan(e < p.experts ? (s.to - s.from + TQ - 1) / TQ : 0), kWave - 1);
  }
  const int64_t tiles = (int64_t)total * wide, run = (tiles + 7) / 8;
  const int64_t at = (blockIdx.x & 7) * run + (blockIdx.x >> 3);
  if ((int64_t)(blockIdx.x >> 3) >= run || at >= tiles) return {0, 0, 0, 0};
  const int strip = (int)(at / wide);   // lies among the strips of the tile's own expert
  int before = 0;
  for (int e0 = 0; e0 < p.experts; e0 += kWave) {
    const int e = e0 + lane;
    const Segment8 s = segment8(p.offsets, min(e, p.experts - 1), p.rows);
    const int n = e < p.experts ? (s.to - s.from + TQ - 1) / TQ : 0, upto = before + lane_scan(n);
    const uint64_t behind = __ballot(upto > strip);
    if (behind) {
      const int l = __builtin_ctzll(behind), strips = read_lane(n, l);
      const int64_t local = at - (int64_t)(read_lane(upto, l) - strips) * wide;
      const int column = (int)(local / strips);
      return {e0 + l, read_lane(s.from, l) + (int)(local - (int64_t)column * strips) * TQ, read_lane(s.to, l), column * TP};
    }
    before = read_lane(upto, kWave - 1);
  }
  return {0, 0, 0, 0};
}

template <typename OUT>
__device__ __forceinline__ void store4(OUT *at, int n, const f32x4 &v) {
  OUT o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(OUT) == 2) o[i] = (OUT)f32_to_bf16(v[i]);
    else o[i] = v[i];
  }
  if (n >= 4) {
    __builtin_memcpy(at, o, sizeof(o));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) at[i] = o[i];
  }
}

// Eight values of a block as bf16, times the block's power of two.
__device__ __forceinline__ bf16x8 widen(int lo, int hi, float power) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, true);
  return {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// FQ x FP fragments of 32 x 32 in a wave, WQ x WP waves.  LDS holds two steps of 128 bytes of the tile's rows, filled
// straight from memory while the other is multiplied; a row's eight 16-byte pieces are stored at places exchanged by the row
// number, so that the rows of a fragment spread over all banks.  Lane l has
// row l % 32 of a fragment and its pieces 4 (l / 32) to 4 (l / 32) + 3; which values meet in an instruction does not matter as
// long as both operands' lanes hold the same ones.
template <int FQ, int FP, int WQ, int WP, bool DW, typename OUT>
__global__ __launch_bounds__(WQ * WP * kWave) void product_kernel(ProductParams p) {
  constexpr int kWaves = WQ * WP, TQ = FQ * WQ * 32, TP = FP * WP * 32;
  constexpr bool kFull = sizeof(OUT) == 4;
  constexpr int kLoadsQ = TQ / 8 / kWaves, kLoadsP = TP / 8 / kWaves;
  __shared__ __attribute__((aligned(128))) uint8_t stage[2][(TQ + TP) * 128];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wq = wave / WP, wp = wave % WP;
  Tile t;
  int steps, q_rows, p_rows;
  const uint8_t *q, *ps;
  int64_t q_pitch, p_pitch;
  int block0 = 0;
  if constexpr (DW) {
    const int e = (int)blockIdx.z;
    const Segment8 s = segment8(p.offsets, e, p.rows);
    steps = (s.to - s.from + 127) / 128;
    block0 = first_block8(s.from, e);
    t = {e, (int)blockIdx.y * TQ, p.N, (int)blockIdx.x * TP};
    q_pitch = p_pitch = column8_blocks(p.rows, p.experts) * 128;
    q = p.q + (int64_t)block0 * 128;
    ps = p.p + (int64_t)block0 * 128;
    q_rows = p.N;
    p_rows = p.H;
  } else {
    t = tile_of_rows<TQ, TP>(p);
    if (t.q0 >= t.q_end) return;
    steps = (int)blocks8(p.H);
    q_pitch = p_pitch = row8_bytes(p.H);
    q = p.q;
    ps = p.p + (int64_t)t.expert * p.N * p_pitch;
    q_rows = t.q_end;
    p_rows = p.N;
  }
  // places of this lane's pieces; rows behind the last are read from the last, their products are not stored
  const uint8_t *from_q[kLoadsQ], *from_p[kLoadsP];
  const int row8 = lane >> 3, piece = ((lane & 7) ^ row8) * 16;
#pragma unroll
  for (int i = 0; i < kLoadsQ; ++i) from_q[i] = q + (int64_t)min(t.q0 + (wave + i * kWaves) * 8 + row8, q_rows - 1) * q_pitch + piece;
#pragma unroll
  for (int i = 0; i < kLoadsP; ++i) from_p[i] = ps + (int64_t)min(t.p0 + (wave + i * kWaves) * 8 + row8, p_rows - 1) * p_pitch + piece;
  auto load = [&](int s, int k) {
#pragma unroll
    for (int i = 0; i < kLoadsQ; ++i)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from_q[i] + (int64_t)k * 128),
                                       (__attribute__((address_space(3))) void *)(stage[s] + (wave + i * kWaves) * 1024), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < kLoadsP; ++i)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from_p[i] + (int64_t)k * 128),
                                       (__attribute__((address_space(3))) void *)(stage[s] + (TQ / 8 + wave + i * kWaves) * 1024), 16, 0, 0);
  };
  // scales of this lane's row of each fragment
  const int64_t scale_q = DW ? 0 : scale8_bytes(p.H);
  const uint8_t *sq[FQ], *sp[FP];
#pragma unroll
  for (int i = 0; i < FQ; ++i) {
    const int r = min(t.q0 + (wq * FQ + i) * 32 + (lane & 31), q_rows - 1);
    sq[i] = p.q_scale + (DW ? (int64_t)block0 * p.N + r : (int64_t)r * scale_q);
  }
#pragma unroll
  for (int i = 0; i < FP; ++i) {
    const int r = min(t.p0 + (wp * FP + i) * 32 + (lane & 31), p_rows - 1);
    sp[i] = p.p_scale + (DW ? (int64_t)block0 * p.H + r : ((int64_t)t.expert * blocks8(p.N) + r / 128) * scale_q);
  }
  f32x16 acc[FQ][FP];
#pragma unroll
  for (int i = 0; i < FQ; ++i)
#pragma unroll
    for (int j = 0; j < FP; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
  if (steps > 0) load(0, 0);
  const int at = (lane & 31) * 128 + (((lane >> 5) * 4) ^ (lane & 7)) * 16;   // piece 4 (l / 32); the others are exchanged with it
  for (int k = 0; k < steps; ++k) {
    int scale_of_q[FQ], scale_of_p[FP];
#pragma unroll
    for (int i = 0; i < FQ; ++i) scale_of_q[i] = sq[i][DW ? (int64_t)k * p.N : k];
#pragma unroll
    for (int i = 0; i < FP; ++i) scale_of_p[i] = sp[i][DW ? (int64_t)k * p.H : k];
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): the wave's own pieces are in LDS
    __syncthreads();
    if (k + 1 < steps) load((k + 1) & 1, k + 1);
    const uint8_t *tile_q = stage[k & 1] + wq * FQ * 4096, *tile_p = stage[k & 1] + TQ * 128 + wp * FP * 4096;
    if constexpr (kFull) {
      float power_of_q[FQ], power_of_p[FP];
#pragma unroll
      for (int i = 0; i < FQ; ++i) power_of_q[i] = __builtin_bit_cast(float, scale_of_q[i] << 23);
#pragma unroll
      for (int j = 0; j < FP; ++j) power_of_p[j] = __builtin_bit_cast(float, scale_of_p[j] << 23);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        i32x4 a[FQ], b[FP];
#pragma unroll
        for (int i = 0; i < FQ; ++i) a[i] = *(const i32x4 *)(tile_q + i * 4096 + (at ^ (s * 16)));
#pragma unroll
        for (int j = 0; j < FP; ++j) b[j] = *(const i32x4 *)(tile_p + j * 4096 + (at ^ (s * 16)));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 wide[FP];
#pragma unroll
          for (int j = 0; j < FP; ++j) wide[j] = widen(b[j][2 * h], b[j][2 * h + 1], power_of_p[j]);
#pragma unroll
          for (int i = 0; i < FQ; ++i) {
            const bf16x8 row = widen(a[i][2 * h], a[i][2 * h + 1], power_of_q[i]);
#pragma unroll
            for (int j = 0; j < FP; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wide[j], row, acc[i][j], 0, 0, 0);
          }
        }
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        auto piece8 = [&](const uint8_t *tile) {
          const i32x4 lo = *(const i32x4 *)(tile + (at ^ (s * 32))), hi = *(const i32x4 *)(tile + (at ^ (s * 32 + 16)));
          return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        };
        i32x8 b[FP];
#pragma unroll
        for (int j = 0; j < FP; ++j) b[j] = piece8(tile_p + j * 4096);
#pragma unroll
        for (int i = 0; i < FQ; ++i) {
          const i32x8 a = piece8(tile_q + i * 4096);
#pragma unroll
          for (int j = 0; j < FP; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[j], a, acc[i][j], 0, 0, 0, scale_of_p[j], 0, scale_of_q[i]);   // 0, 0: e4m3
        }
      }
    }
  }
  // a lane has row l % 32 of a fragment and of every eight columns the first or the last four
#pragma unroll
  for (int i = 0; i < FQ; ++i) {
    const int r = t.q0 + (wq * FQ + i) * 32 + (lane & 31);
    if (r >= q_rows) continue;
    OUT *row = (OUT *)p.out + (DW ? ((int64_t)t.expert * p.N + r) * p.H : (int64_t)r * p.N);
#pragma unroll
    for (int j = 0; j < FP; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = t.p0 + (wp * FP + j) * 32 + g * 8 + (lane >> 5) * 4;
        if (c < p_rows) store4(row + c, p_rows - c, f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]});
      }
  }
}

static hm_status check_products(const void *a, const void *as, const void *b, const void *bs, const int32_t *offsets, int32_t experts, int64_t rows,
                                int32_t N, int32_t H, const void *out, hm_dtype dtype, bool none) {
  if (!dtype_known(dtype) || !segments8_ok(experts, rows) || N < 1 || N > kMostColumns8 || H < 1 || H > kMostColumns8) return HM_ERR_SHAPE;
  if (!buffers8_aligned(a, as) || !buffers8_aligned(b, bs) || ((uintptr_t)out & (dtype == HM_F32 ? 3 : 1))) return HM_ERR_SHAPE;
  if (none) return HM_OK;
  if (!a || !as || !b || !bs || !offsets || !out) return HM_ERR_NULL;
  return HM_OK;
}

}  // namespace hm

extern "C" hm_status hm_expert_matmul(const uint8_t *x, const uint8_t *x_scale, const uint8_t *w, const uint8_t *w_scale, const int32_t *offsets,
                                      int32_t experts, int64_t rows, int32_t N, int32_t H, void *out, hm_dtype out_dtype, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  const hm_status bad = check_products(x, x_scale, w, w_scale, offsets, experts, rows, N, H, out, out_dtype, rows == 0);
  if (bad != HM_OK) return bad;
  if (rows == 0) return HM_OK;
  const ProductParams p = {x, x_scale, w, w_scale, offsets, experts, (int32_t)rows, N, H, out};
  const int64_t tiles = (rows / 128 + experts) * ((N + 127) / 128) + 8;
  if (tiles > (1 << 23)) return HM_ERR_SHAPE;
  const auto kernel = out_dtype == HM_BF16 ? product_kernel<2, 2, 2, 2, false, uint16_t> : product_kernel<2, 2, 2, 2, false, float>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(256), 0, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}

extern "C" hm_status hm_expert_matmul_dw(const uint8_t *gy, const uint8_t *gy_scale, const uint8_t *x, const uint8_t *x_scale,
                                         const int32_t *offsets, int32_t experts, int64_t rows, int32_t N, int32_t H, void *dw,
                                         hm_dtype dw_dtype, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  const hm_status bad = check_products(gy, gy_scale, x, x_scale, offsets, experts, rows, N, H, dw, dw_dtype, false);
  if (bad != HM_OK) return bad;
  const ProductParams p = {gy, gy_scale, x, x_scale, offsets, experts, (int32_t)rows, N, H, dw};
  const auto kernel = dw_dtype == HM_BF16 ? product_kernel<2, 2, 2, 2, true, uint16_t> : product_kernel<2, 2, 2, 2, true, float>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((H + 127) / 128), (unsigned)((N + 127) / 128), (unsigned)experts), dim3(256), 0, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}
