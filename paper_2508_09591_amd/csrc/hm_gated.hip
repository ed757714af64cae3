// The activation between an expert's two products: rows h = [gate | up] of 2 F values, a = silu(gate) up, and the way back
//     g_gate = ga up s (1 + gate (1 - s)),   g_up = ga gate s,   s = 1 / (1 + exp(-gate)),
// written in the layouts that the products behind it read: rows in 8 bits, and on the way back also columns in 8 bits.
#include "hm_block8.h"

namespace hm {

constexpr int kGatedThreads = 256, kGatedWaves = kGatedThreads / kWave;

struct GatedParams {
  const void *h;
  int64_t ld;
  const int32_t *offsets;   // rows of segments; NULL: all rows
  int32_t segments;
  int64_t rows;
  int32_t F, parts;   // pieces of 512 columns of a row
  void *a;
  uint8_t *q, *scale;
  bool a_bf16;
};

// The kernels round alike, whichever writes a value: no products and sums are joined but where it says so.
__device__ __forceinline__ float gated_value(float gate, float up) {
#pragma clang fp contract(off)
  return gate / (1.0f + expf(-gate)) * up;
}

// First and last row of all segments.
__device__ __forceinline__ void rows_of_segments(const int32_t *__restrict__ offsets, int segments, int64_t rows, int64_t &from, int64_t &to) {
  from = 0;
  to = rows;
  if (offsets) {
    from = min(max((int64_t)offsets[0], (int64_t)0), rows);
    to = min(max((int64_t)offsets[segments], from), rows);
  }
}

// A wave takes 512 columns of a of ROWS rows.
template <typename IN, int ROWS>
__global__ __launch_bounds__(kGatedThreads) void gated_kernel(GatedParams p) {
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const uint32_t block = blockIdx.x / (uint32_t)p.parts;
  const int part = (int)(blockIdx.x - block * (uint32_t)p.parts), c = part * 512 + lane * 8;
  const int64_t first = ((int64_t)block * kGatedWaves + wave) * ROWS;
  const bool whole = part * 512 + 512 <= p.F;
  const int width = (int)row8_bytes(p.F);
  int64_t from, to;
  rows_of_segments(p.offsets, p.segments, p.rows, from, to);
  float gate[ROWS][8], up[ROWS][8];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {   // rows behind the last are read from it
    const IN *row = (const IN *)p.h + min(first + i, p.rows - 1) * p.ld;
    load_row(row, c, p.F, whole, gate[i]);
    load_row(row + p.F, c, p.F, whole, up[i]);
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int64_t r = first + i;
    if (r < from || r >= to) continue;   // the same for the wave
#pragma unroll
    for (int j = 0; j < 8; ++j) gate[i][j] = gated_value(gate[i][j], up[i][j]);
    if (p.a) {
      if (p.a_bf16) store_row((uint16_t *)p.a + r * p.F, c, p.F, gate[i]);
      else store_row((float *)p.a + r * p.F, c, p.F, gate[i]);
    }
    if (p.q) store_piece8(p.q + r * width, p.scale + r * scale8_bytes(p.F), part, width, gate[i]);
  }
}

struct GatedBackParams {
  const void *h, *ga;
  int64_t ld, ga_ld;
  const int32_t *offsets;
  int32_t segments;
  int64_t rows;
  int32_t F, parts;   // parts: pieces of 512 columns of a row of 2 F
  void *gh;
  bool gh_bf16;
  uint8_t *q, *scale, *q_columns, *scale_columns, *a_columns, *a_scale;
  int32_t blocks, tiles;   // of 128 rows of a segment; of 128 columns
};

struct GatedGradient {
  float gate, up;
};
__device__ __forceinline__ GatedGradient gated_gradient(float gate, float up, float ga) {
#pragma clang fp contract(off)
  const float s = 1.0f / (1.0f + expf(-gate));
  return {ga * up * s * fmaf(gate, 1.0f - s, 1.0f), ga * gate * s};
}

// Rows of [g_gate | g_up]: a wave takes 512 columns of ROWS rows, of either half or of both.
template <typename IN, int ROWS>
__global__ __launch_bounds__(kGatedThreads) void gated_backward_rows_kernel(GatedBackParams p) {
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const uint32_t block = blockIdx.x / (uint32_t)p.parts;
  const int part = (int)(blockIdx.x - block * (uint32_t)p.parts), c = part * 512 + lane * 8, F = p.F;
  const int64_t first = ((int64_t)block * kGatedWaves + wave) * ROWS;
  const int width = (int)row8_bytes(2 * (int64_t)F);
  int64_t from, to;
  rows_of_segments(p.offsets, p.segments, p.rows, from, to);
  // columns c to c + 7 of the gradient are those from `at` on of one half, or the first `mine` of them are g_gate's last
  const bool upper = c >= F;
  const int at = upper ? c - F : c, mine = upper ? 0 : min(F - c, 8);
  const bool whole = (part * 512 + 512 <= F) || (part * 512 >= F && part * 512 + 512 <= 2 * (int64_t)F);
  float v[ROWS][8];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int64_t r = min(first + i, p.rows - 1);
    const IN *h = (const IN *)p.h + r * p.ld, *from_ga = (const IN *)p.ga + r * p.ga_ld;
    float gate[8], up[8], ga[8];
    load_row(h, at, F, whole, gate);
    load_row(h + F, at, F, whole, up);
    load_row(from_ga, at, F, whole, ga);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const GatedGradient g = gated_gradient(gate[j], up[j], ga[j]);
      v[i][j] = upper ? g.up : g.gate;
    }
    if (!whole && mine < 8 && mine > 0) {   // g_up's first behind g_gate's last
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j >= mine && j - mine < F) {
          const int n = j - mine;
          v[i][j] = gated_gradient(load_float(h + n), load_float(h + F + n), load_float(from_ga + n)).up;
        }
    }
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int64_t r = first + i;
    if (r < from || r >= to) continue;
    if (p.gh) {
      if (p.gh_bf16) store_row((uint16_t *)p.gh + r * 2 * F, c, 2 * F, v[i]);
      else store_row((float *)p.gh + r * 2 * F, c, 2 * F, v[i]);
    }
    if (p.q) store_piece8(p.q + r * width, p.scale + r * scale8_bytes(2 * (int64_t)F), part, width, v[i]);
  }
}

// A workgroup takes a block of 128 rows of a segment and 128 columns of each half; a thread four rows of eight columns.
// g_gate, g_up and a one after the other: rows leave from registers, columns are turned in LDS.
constexpr int kTurnThreads = 512, kTurnPitch = 128 + 8;
template <typename IN>
__global__ __launch_bounds__(kTurnThreads) void gated_backward_kernel(GatedBackParams p) {
  constexpr int kWaves = kTurnThreads / kWave;
  __shared__ __attribute__((aligned(16))) uint8_t turned[128 * kTurnPitch];
  __shared__ uint32_t most_of[kWaves][128];
  const int64_t all = (int64_t)p.blocks * p.tiles, per_die = (all + 7) / 8;
  const int64_t at = (blockIdx.x & 7) * per_die + (blockIdx.x >> 3);   // a die gets neighbouring tiles
  if ((int64_t)(blockIdx.x >> 3) >= per_die || at >= all) return;
  const int b = (int)(at / p.tiles), tile = (int)(at - (int64_t)b * p.tiles);
  const BlockOwner8 owner = owner_of_block8(p.offsets, p.segments, (int)p.rows, b);
  if (owner.segment < 0) return;
  const int first = owner.rows.from + (b - first_block8(owner.rows.from, owner.segment)) * 128, end = owner.rows.to;
  if (first >= end) return;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave, F = p.F;
  const int c0 = tile * 128, cl = (tid & 15) * 8, c = c0 + cl, rl = (tid >> 4) * 4;
  const bool whole = c0 + 128 <= F;
  float gate[4][8], up[4][8], ga[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {   // rows behind the segment are read from its last and count as zeros
    const int64_t r = min(first + rl + i, end - 1);
    const IN *h = (const IN *)p.h + r * p.ld;
    load_row(h, c, F, whole, gate[i]);
    load_row(h + F, c, F, whole, up[i]);
    load_row((const IN *)p.ga + r * p.ga_ld, c, F, whole, ga[i]);
  }
  const int64_t width = row8_bytes(2 * (int64_t)F), scales = scale8_bytes(2 * (int64_t)F);
#pragma unroll
  for (int plane = 0; plane < 3; ++plane) {
    const int half = plane == 1 ? F : 0;   // first column of this half
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const GatedGradient g = gated_gradient(gate[i][j], up[i][j], ga[i][j]);
        const float x = plane == 0 ? g.gate : plane == 1 ? g.up : gated_value(gate[i][j], up[i][j]);
        v[i][j] = first + rl + i < end ? x : 0.0f;
      }
    if (plane < 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t r = first + rl + i;
        if (p.gh && r < end) {
          if (p.gh_bf16) store_row((uint16_t *)p.gh + r * 2 * F + half, c, F, v[i]);
          else store_row((float *)p.gh + r * 2 * F + half, c, F, v[i]);
        }
        if (p.q) {   // whole blocks of both halves: F is a multiple of 128
          float u[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) u[j] = v[i][j];
          const int code = scale_code8(max16(largest_bits(u)));
          const float by = inverse_scale8(code);
          if (r < end) {
            *(uint64_t *)(p.q + r * width + half + c) =
                (uint64_t)pack8(u[4], u[5], u[6], u[7], by) << 32 | pack8(u[0], u[1], u[2], u[3], by);
            const int k = (half + c0) / 128;
            if ((lane & 15) == 0) p.scale[r * scales + k] = (uint8_t)code;
            if ((lane & 15) < 3 && k == 2 * F / 128 - 1 && k + 1 + (lane & 15) < scales)
              p.scale[r * scales + k + 1 + (lane & 15)] = 0;   // zeros behind the last
          }
        }
      }
    }
    uint8_t *to = plane < 2 ? p.q_columns : p.a_columns, *to_scale = plane < 2 ? p.scale_columns : p.a_scale;
    if (!to) continue;
    const int64_t C = plane < 2 ? 2 * (int64_t)F : F;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float u[4] = {v[0][j], v[1][j], v[2][j], v[3][j]};
      uint32_t most = largest_bits(u);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i][j] = u[i];
      most = max(most, (uint32_t)__shfl_xor((int)most, 16, kWave));
      most = max(most, (uint32_t)__shfl_xor((int)most, 32, kWave));
      if (lane < 16) most_of[wave][cl + j] = most;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t m = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = max(m, most_of[w][cl + j]);
      const int code = scale_code8(m);
      if (tid < 16 && c + j < F) to_scale[(int64_t)b * C + half + c + j] = (uint8_t)code;
      *(uint32_t *)(turned + (cl + j) * kTurnPitch + rl) = pack8(v[0][j], v[1][j], v[2][j], v[3][j], inverse_scale8(code));
    }
    __syncthreads();
    const int col = tid >> 2, piece = (tid & 3) * 32;
    if (c0 + col < F) {
      const int64_t row_bytes = column8_blocks(p.rows, p.segments) * 128;
      uint64_t *out = (uint64_t *)(to + (int64_t)(half + c0 + col) * row_bytes + (int64_t)b * 128 + piece);
      const uint64_t *in = (const uint64_t *)(turned + col * kTurnPitch + piece);
#pragma unroll
      for (int i = 0; i < 4; ++i) out[i] = in[i];
    }
    // the next plane writes `turned` behind its first barrier and `most_of`, which is read before this one's second
  }
}

static bool segments_given_ok(const int32_t *offsets, int32_t segments, int64_t rows) {
  return !offsets || segments8_ok(segments, rows);
}
// Rows of a wave: one where few rows would not fill the chip otherwise.
static int rows_of_wave(int64_t rows, int32_t parts) { return rows * parts >= 32768 ? 4 : 1; }
constexpr int64_t kMostGatedPieces = 1 << 25;   // of 512 columns, of all rows

}  // namespace hm

extern "C" hm_status hm_gated(const void *h, hm_dtype dtype, int64_t ld, const int32_t *offsets, int32_t segments, int64_t rows,
                              int32_t F, void *a, hm_dtype a_dtype, uint8_t *q, uint8_t *scale, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!dtype_known(dtype) || !dtype_known(a_dtype) || F < 1 || F > kMostColumns8) return HM_ERR_SHAPE;
  if (rows < 0 || rows > 2147483647LL || !segments_given_ok(offsets, segments, rows)) return HM_ERR_SHAPE;
  if ((ld < 2 * (int64_t)F && rows > 1) || !aligned_as(dtype, h) || !aligned_as(a_dtype, a)) return HM_ERR_SHAPE;
  if (!buffers8_aligned(q, scale) || ((uintptr_t)offsets & 3)) return HM_ERR_SHAPE;
  if (rows == 0) return HM_OK;
  if (!q != !scale || (!a && !q)) return HM_ERR_NULL;
  if (!h) return HM_ERR_NULL;
  const int32_t parts = (F + 511) / 512;
  const GatedParams p = {h, ld, offsets, segments, rows, F, parts, a, q, scale, a_dtype == HM_BF16};
  const int each = rows_of_wave(rows, parts);
  const int64_t blocks = (rows + kGatedWaves * each - 1) / (kGatedWaves * each) * parts;
  if (rows * parts > kMostGatedPieces) return HM_ERR_SHAPE;
  const auto kernel = dtype == HM_BF16 ? each == 4 ? gated_kernel<uint16_t, 4> : gated_kernel<uint16_t, 1>
                                       : each == 4 ? gated_kernel<float, 4> : gated_kernel<float, 1>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kGatedThreads), 0, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}

extern "C" hm_status hm_gated_backward(const void *h, const void *ga, hm_dtype dtype, int64_t ld, int64_t ga_ld,
                                       const int32_t *offsets, int32_t segments, int64_t rows, int32_t F, void *gh,
                                       hm_dtype gh_dtype, uint8_t *q, uint8_t *scale, uint8_t *q_columns, uint8_t *scale_columns,
                                       uint8_t *a_columns, uint8_t *a_scale, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!dtype_known(dtype) || !dtype_known(gh_dtype) || F < 1 || F > kMostColumns8 / 2) return HM_ERR_SHAPE;
  if (rows < 0 || rows > 2147483647LL || !segments_given_ok(offsets, segments, rows)) return HM_ERR_SHAPE;
  if (((ld < 2 * (int64_t)F || ga_ld < F) && rows > 1) || !aligned_as(dtype, h) || !aligned_as(dtype, ga)) return HM_ERR_SHAPE;
  if (!aligned_as(gh_dtype, gh) || !buffers8_aligned(q, scale) || !buffers8_aligned(q_columns, scale_columns) ||
      !buffers8_aligned(a_columns, a_scale) || ((uintptr_t)offsets & 3))
    return HM_ERR_SHAPE;
  if (rows == 0) return HM_OK;
  const bool columns = q_columns || a_columns;
  if (!q != !scale || !q_columns != !scale_columns || !a_columns != !a_scale || (!gh && !q && !columns)) return HM_ERR_NULL;
  if (columns && !offsets) return HM_ERR_NULL;
  if (!h || !ga) return HM_ERR_NULL;
  GatedBackParams p = {h, ga, ld, ga_ld, offsets, segments, rows, F, (2 * F + 511) / 512, gh, gh_dtype == HM_BF16, q, scale,
                       q_columns, scale_columns, a_columns, a_scale, 0, (F + 127) / 128};
  // blocks of 8 bits of a row that lie in both halves are not the tiles'
  const bool by_rows = !columns || (q && F % 128 != 0);
  const int each = rows_of_wave(rows, p.parts);
  const int64_t row_blocks = (rows + kGatedWaves * each - 1) / (kGatedWaves * each) * p.parts;
  if (rows * p.parts > kMostGatedPieces) return HM_ERR_SHAPE;
  if (columns) {
    p.blocks = (int32_t)column8_blocks(rows, segments);
    const int64_t workgroups = ((int64_t)p.blocks * p.tiles + 7) / 8 * 8;
    if (workgroups > (1 << 22)) return HM_ERR_SHAPE;
    GatedBackParams tiles = p;
    if (by_rows) tiles.q = nullptr;
    const auto kernel = dtype == HM_BF16 ? gated_backward_kernel<uint16_t> : gated_backward_kernel<float>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)workgroups), dim3(kTurnThreads), 0, (hipStream_t)hip_stream, tiles);
    const hm_status launched = hm_launch_status();
    if (launched != HM_OK || !by_rows) return launched;
    p.gh = nullptr;   // written
  }
  const auto kernel = dtype == HM_BF16 ? each == 4 ? gated_backward_rows_kernel<uint16_t, 4> : gated_backward_rows_kernel<uint16_t, 1>
                                       : each == 4 ? gated_backward_rows_kernel<float, 4> : gated_backward_rows_kernel<float, 1>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)row_blocks), dim3(kGatedThreads), 0, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}
