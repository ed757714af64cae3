// Values in 8 bits with a power of two for each block of 128: rows, transposed columns of segments, weights both ways.
#include "hm_block8.h"

namespace hm {

constexpr int kQuantThreads = 256;

struct RowParams {
  const void *x;
  int64_t ld, pieces;   // pieces of 512 columns of all rows
  int32_t C, per_row;   // pieces of a row
  uint8_t *q, *scale;
};

// A wave takes 512 columns of a row, a lane eight of them, sixteen lanes a block.  Bound by memory: 8,192 x 7,168 bf16
// 34 us, 5.2 TB/s.
template <typename IN>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(RowParams p) {
  const int lane = lane_id();
  const int64_t piece = (int64_t)blockIdx.x * (kQuantThreads / kWave) + threadIdx.x / kWave;
  if (piece >= p.pieces) return;
  const int64_t r = piece / p.per_row;
  const int part = (int)(piece - r * p.per_row), c = part * 512 + lane * 8;
  const int64_t width = row8_bytes(p.C);
  float v[8];
  const IN *row = (const IN *)p.x + r * p.ld;
  if (part * 512 + 512 <= p.C) load_floats<8>(row + c, v);   // the whole wave
  else load_row_end<8>(row, c, p.C, v);
  store_piece8(p.q + r * width, p.scale + r * scale8_bytes(p.C), part, (int)width, v);
}

struct ColumnParams {
  const void *x;
  int64_t ld;
  const int32_t *offsets;
  int32_t segments, rows, C, blocks, tiles;   // blocks of rows; tiles of columns
  uint8_t *q, *scale;
};

// A workgroup takes a block of 128 rows and 64 columns: a thread eight rows of four columns, whose bytes it turns in
// registers; LDS puts a column's 128 bytes together.  6,001 rows of 2,056 bf16 in 16 segments 11 us, 3.3 TB/s: one
// generation of workgroups, whose offsets, rows and stores wait for one another (23 with scalar loads, 14 with
// neighbouring tiles on any die).
constexpr int kColumnTile = 64, kColumnPitch = 128 + 8;
template <typename IN>
__global__ __launch_bounds__(kQuantThreads) void quantize_columns_kernel(ColumnParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[kColumnTile * kColumnPitch];
  __shared__ uint32_t most_of[kQuantThreads / kWave][kColumnTile];
  // a die gets neighbouring tiles: they share the lines that rows off a line's alignment have in common
  const int64_t per_die = ((int64_t)p.blocks * p.tiles + 7) / 8, at = (blockIdx.x & 7) * per_die + (blockIdx.x >> 3);
  if ((int64_t)(blockIdx.x >> 3) >= per_die || at >= (int64_t)p.blocks * p.tiles) return;
  const int b = (int)(at / p.tiles);
  const BlockOwner8 owner = owner_of_block8(p.offsets, p.segments, p.rows, b);
  if (owner.segment < 0) return;
  const Segment8 s = owner.rows;
  const int first = s.from + (b - first_block8(s.from, owner.segment)) * 128;
  if (first >= s.to) return;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
  const int c0 = (int)(at - (int64_t)b * p.tiles) * kColumnTile, cl = (tid & 15) * 4, c = c0 + cl, r0 = (tid >> 4) * 8;
  float v[8][4], column[4][8];
  uint32_t most[4];
  // rows behind the segment are read from its last and count as zeros; whole tiles without branches, so that a thread's
  // loads are on their way together
  const IN *from[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) from[i] = (const IN *)p.x + (int64_t)min(first + r0 + i, s.to - 1) * p.ld;
  if (c0 + kColumnTile <= p.C) {
#pragma unroll
    for (int i = 0; i < 8; ++i) load_floats<4>(from[i] + c, v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) load_row_end<4>(from[i], c, p.C, v[i]);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int i = 0; i < 8; ++i) column[j][i] = first + r0 + i < s.to ? v[i][j] : 0.0f;
    most[j] = largest_bits(column[j]);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    most[j] = max(most[j], (uint32_t)__shfl_xor((int)most[j], 16, kWave));
    most[j] = max(most[j], (uint32_t)__shfl_xor((int)most[j], 32, kWave));
    if (lane < 16) most_of[wave][cl + j] = most[j];
  }
  __syncthreads();
  float by[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < kQuantThreads / kWave; ++w) m = max(m, most_of[w][cl + j]);
    const int code = scale_code8(m);
    by[j] = inverse_scale8(code);
    if (tid < 16 && c + j < p.C) p.scale[(int64_t)b * p.C + c + j] = (uint8_t)code;
    const float (&u)[8] = column[j];
    const uint64_t out = (uint64_t)pack8(u[4], u[5], u[6], u[7], by[j]) << 32 | pack8(u[0], u[1], u[2], u[3], by[j]);
    *(uint64_t *)(turned + (cl + j) * kColumnPitch + r0) = out;
  }
  __syncthreads();
  const int col = tid >> 2, part = (tid & 3) * 32;
  if (c0 + col < p.C) {
    const int64_t width = column8_blocks(p.rows, p.segments) * 128;
    uint8_t *out = p.q + (int64_t)(c0 + col) * width + (int64_t)b * 128 + part;
    const uint64_t *in = (const uint64_t *)(turned + col * kColumnPitch + part);
#pragma unroll
    for (int i = 0; i < 4; ++i) ((uint64_t *)out)[i] = in[i];
  }
}

struct WeightParams {
  const void *w;
  int32_t N, C;
  uint8_t *q, *scale, *qt, *scale_t;
};

// A workgroup takes a block of 128 x 128: a thread eight rows of eight columns.  Bound by memory: 32 x 2,048 x 2,048
// fp32, both layouts, 145 us, 5.6 TB/s.
template <typename IN>
__global__ __launch_bounds__(kQuantThreads) void quantize_weights_kernel(WeightParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[128 * kColumnPitch];
  __shared__ uint32_t most_of[kQuantThreads / kWave];
  const int tid = threadIdx.x, cl = (tid & 15) * 8, rl = (tid >> 4) * 8;
  const int n0 = (int)blockIdx.y * 128, c0 = (int)blockIdx.x * 128;
  const int64_t e = blockIdx.z;
  float v[8][8];
  const IN *from[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) from[i] = (const IN *)p.w + (e * p.N + min(n0 + rl + i, p.N - 1)) * p.C;
  if (c0 + 128 <= p.C) {   // as above
#pragma unroll
    for (int i = 0; i < 8; ++i) load_floats<8>(from[i] + c0 + cl, v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) load_row_end<8>(from[i], c0 + cl, p.C, v[i]);
  }
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = n0 + rl + i < p.N ? v[i][j] : 0.0f;
    most = max(most, largest_bits(v[i]));
  }
  most = max16(most);
  most = max(most, (uint32_t)__shfl_xor((int)most, 16, kWave));
  most = max(most, (uint32_t)__shfl_xor((int)most, 32, kWave));
  if (lane_id() == 0) most_of[tid / kWave] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQuantThreads / kWave; ++w) most = max(most, most_of[w]);
  const int code = scale_code8(most);
  const float by = inverse_scale8(code);
  const int64_t width = row8_bytes(p.C), width_t = row8_bytes(p.N);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (n0 + rl + i >= p.N) continue;
    const uint64_t out = (uint64_t)pack8(v[i][4], v[i][5], v[i][6], v[i][7], by) << 32 |
                         pack8(v[i][0], v[i][1], v[i][2], v[i][3], by);
    *(uint64_t *)(p.q + (e * p.N + n0 + rl + i) * width + c0 + cl) = out;
  }
  // a row's scales end with zeros up to a multiple of four; the last block of a row writes them
  const int blocks_n = (int)blocks8(p.N), blocks_c = (int)blocks8(p.C);
  const int wide = (int)scale8_bytes(p.C), wide_t = (int)scale8_bytes(p.N);
  if (tid < 4) {
    const int k = (int)blockIdx.x + tid;
    if (tid == 0 || ((int)blockIdx.x == blocks_c - 1 && k < wide))
      p.scale[(e * blocks_n + blockIdx.y) * wide + k] = tid == 0 ? (uint8_t)code : 0;
  }
  if (!p.qt) return;
  if (tid < 4) {
    const int k = (int)blockIdx.y + tid;
    if (tid == 0 || ((int)blockIdx.y == blocks_n - 1 && k < wide_t))
      p.scale_t[(e * blocks_c + blockIdx.x) * wide_t + k] = tid == 0 ? (uint8_t)code : 0;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint64_t out = (uint64_t)pack8(v[4][j], v[5][j], v[6][j], v[7][j], by) << 32 |
                         pack8(v[0][j], v[1][j], v[2][j], v[3][j], by);
    *(uint64_t *)(turned + (cl + j) * kColumnPitch + rl) = out;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = i * 32 + (tid >> 3), part = (tid & 7) * 16;
    if (c0 + c >= p.C) continue;
    const uint64_t *in = (const uint64_t *)(turned + c * kColumnPitch + part);
    uint64_t *out = (uint64_t *)(p.qt + (e * p.C + c0 + c) * width_t + n0 + part);
    out[0] = in[0];
    out[1] = in[1];
  }
}

}  // namespace hm

extern "C" hm_status hm_quantize_rows(const void *x, hm_dtype dtype, int64_t ld, int64_t rows, int32_t C, uint8_t *q,
                                      uint8_t *scale, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!dtype_known(dtype) || C < 1 || C > kMostColumns8 || rows < 0 || rows > 2147483647LL) return HM_ERR_SHAPE;
  if ((ld < C && rows > 1) || !buffers8_aligned(q, scale)) return HM_ERR_SHAPE;
  if (rows == 0) return HM_OK;
  if (!x || !q || !scale) return HM_ERR_NULL;
  RowParams p;
  p.x = x;
  p.ld = ld;
  p.C = C;
  p.per_row = (C + 511) / 512;
  p.pieces = rows * p.per_row;
  p.q = q;
  p.scale = scale;
  const int64_t blocks = (p.pieces + kQuantThreads / kWave - 1) / (kQuantThreads / kWave);
  if (blocks > (1 << 23)) return HM_ERR_SHAPE;
  const auto kernel = dtype == HM_BF16 ? quantize_rows_kernel<uint16_t> : quantize_rows_kernel<float>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kQuantThreads), 0, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}

extern "C" hm_status hm_quantize_columns(const void *x, hm_dtype dtype, int64_t ld, const int32_t *offsets,
                                         int32_t segments, int64_t rows, int32_t C, uint8_t *q, uint8_t *scale,
                                         void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!dtype_known(dtype) || C < 1 || C > kMostColumns8 || !segments8_ok(segments, rows)) return HM_ERR_SHAPE;
  if ((ld < C && rows > 1) || !buffers8_aligned(q, scale)) return HM_ERR_SHAPE;
  if (rows == 0) return HM_OK;
  if (!x || !offsets || !q || !scale) return HM_ERR_NULL;
  ColumnParams p;
  p.x = x;
  p.ld = ld;
  p.offsets = offsets;
  p.segments = segments;
  p.rows = (int32_t)rows;
  p.C = C;
  p.q = q;
  p.scale = scale;
  const auto kernel = dtype == HM_BF16 ? quantize_columns_kernel<uint16_t> : quantize_columns_kernel<float>;
  p.blocks = (int32_t)column8_blocks(rows, segments);
  p.tiles = (C + kColumnTile - 1) / kColumnTile;
  const int64_t workgroups = ((int64_t)p.blocks * p.tiles + 7) / 8 * 8;
  if (workgroups > (1 << 23)) return HM_ERR_SHAPE;
  hipLaunchKernelGGL(kernel, dim3((unsigned)workgroups), dim3(kQuantThreads), 0, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}

extern "C" hm_status hm_quantize_weights(const void *w, hm_dtype dtype, int32_t experts, int32_t N, int32_t C,
                                         uint8_t *q, uint8_t *scale, uint8_t *qt, uint8_t *scale_t,
                                         void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!w || !q || !scale || (!qt != !scale_t)) return HM_ERR_NULL;
  if (!dtype_known(dtype) || experts < 1 || experts > kMostSegments8) return HM_ERR_SHAPE;
  if (N < 1 || N > kMostColumns8 || C < 1 || C > kMostColumns8) return HM_ERR_SHAPE;
  if (!buffers8_aligned(q, scale) || !buffers8_aligned(qt, scale_t)) return HM_ERR_SHAPE;
  WeightParams p = {w, N, C, q, scale, qt, scale_t};
  const auto kernel = dtype == HM_BF16 ? quantize_weights_kernel<uint16_t> : quantize_weights_kernel<float>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks8(C), (unsigned)blocks8(N), (unsigned)experts), dim3(kQuantThreads),
                     0, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}
