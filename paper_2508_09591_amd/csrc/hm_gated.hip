// The activation between an expert's two products: rows h = [gate | up] of 2 F values, a = silu(gate) up, and the way back
//     g_gate = ga up s (1 + gate (1 - s)),   g_up = ga gate s,   s = 1 / (1 + exp(-gate)),
// written in the layouts that the products behind it read: rows in 8 bits, and on the way back also columns in 8 bits, with a itself
// computed again instead of kept.
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

// s = 1 / (1 + exp(-gate)) and gate s.  exp(-x) = 2^(-x log2 e), of whose exponent the part that is lost to its rounding is
// multiplied back in: three instructions more than the bare power, and right to two units in the last place for every x.  The
// reciprocal has one Newton step.  Beyond 88 in size s is 1 or at most e^-88.  All kernels round alike, whichever writes a value: no product and
// sum are joined but where it says so.
struct Gate {
  float s, times;
};
__device__ __forceinline__ Gate gate_of(float gate) {
#pragma clang fp contract(off)
  constexpr float kLog2E = 1.44269502f, kRest = 1.92596299e-8f, kLn2 = 0.693147181f;   // log2 e = the first and the second
  const float x = __builtin_amdgcn_fmed3f(gate, -88.0f, 88.0f), t = -x * kLog2E;
  const float lost = fmaf(-x, kRest, fmaf(-x, kLog2E, -t)), power = __builtin_amdgcn_exp2f(t);
  const float y = 1.0f + fmaf(power, lost * kLn2, power), r = __builtin_amdgcn_rcpf(y);   // y is finite: r may be 0, not NaN
  const float s = fmaf(fmaf(-y, r, 1.0f), r, r);
  return {s, gate * s};
}
__device__ __forceinline__ float gated_value(float gate, float up) { return gate_of(gate).times * up; }

// First and last row of all segments.
__device__ __forceinline__ void rows_of_segments(const int32_t *__restrict__ offsets, int segments, int64_t rows, int64_t &from, int64_t &to) {
  from = 0;
  to = rows;
  if (offsets) {
    from = min(max((int64_t)offsets[0], (int64_t)0), rows);
    to = min(max((int64_t)offsets[segments], from), rows);
  }
}

// A wave takes 512 columns of a row of a; neighbouring waves take neighbouring pieces, so that a row's lines are asked for together:
// 65,536 rows of 2 x 2,048 bf16 to 8 bits in 124 to 130 us (672 MB, 5.2 to 5.4 TB/s: memory), 173 where a workgroup took several rows
// in turn.  To bf16 values 138 us (5.9 TB/s), from fp32 rows to 8 bits 217 (5.6), of three quarters of the rows 100.  64 rows 3.7 us: a
// launch and a trip to memory.
template <typename IN>
__global__ __launch_bounds__(kGatedThreads) void gated_kernel(GatedParams p) {
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const uint32_t piece = blockIdx.x * (uint32_t)kGatedWaves + (uint32_t)wave, r = piece / (uint32_t)p.parts;
  const int part = (int)(piece - r * (uint32_t)p.parts), c = part * 512 + lane * 8;
  int64_t from, to;
  rows_of_segments(p.offsets, p.segments, p.rows, from, to);
  if (r < from || r >= to) return;
  const bool whole = part * 512 + 512 <= p.F;
  const IN *row = (const IN *)p.h + r * p.ld;
  float a[8], up[8];
  load_row(row, c, p.F, whole, a);
  load_row(row + p.F, c, p.F, whole, up);
#pragma unroll
  for (int j = 0; j < 8; ++j) a[j] = gated_value(a[j], up[j]);
  if (p.a) {
    if (p.a_bf16) store_row((uint16_t *)p.a + (int64_t)r * p.F, c, p.F, a);
    else store_row((float *)p.a + (int64_t)r * p.F, c, p.F, a);
  }
  if (p.q) store_piece8(p.q + r * row8_bytes(p.F), p.scale + r * scale8_bytes(p.F), part, (int)row8_bytes(p.F), a);
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

// The gradient's two halves: ga up s (1 + gate (1 - s)) and ga gate s.  Of bf16 inputs ga gate is exact, and multiplied first would leave
// g_up off by 0.67 units of 2^-24 on average instead of 0.76; 32,768 rows of F = 768 would take 0.7 us more.
__device__ __forceinline__ float gradient_of_gate(const Gate &g, float up, float ga) {
#pragma clang fp contract(off)
  return ga * up * fmaf(g.times, 1.0f - g.s, g.s);
}
__device__ __forceinline__ float gradient_of_up(const Gate &g, float ga) { return ga * g.times; }

// Rows of [g_gate | g_up]: a wave takes 512 columns of a row, of either half or of both.  Where columns are wanted too, this is for
// rows in 8 bits of an F that is no multiple of 128 alone, whose blocks lie in both halves: 5,003 rows of F = 1,001 fp32 17 us.
// Waves of either half read gate, up and ga and compute the gate, which shows where F is large: 65,536 rows of F = 2,048 bf16 to values
// alone 310 us, which copied would be 262, to rows in 8 bits 281 (210); 32,768 of F = 768 57 (49) and 55 (39), fp32 100 (98) and 68 (69).
template <typename IN>
__global__ __launch_bounds__(kGatedThreads) void gated_backward_rows_kernel(GatedBackParams p) {
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), F = p.F;
  const uint32_t piece = blockIdx.x * (uint32_t)kGatedWaves + (uint32_t)wave, r = piece / (uint32_t)p.parts;
  const int part = (int)(piece - r * (uint32_t)p.parts), c = part * 512 + lane * 8;
  int64_t from, to;
  rows_of_segments(p.offsets, p.segments, p.rows, from, to);
  if (r < from || r >= to) return;
  // columns c to c + 7 of the gradient are those from `at` on of one half, or the first `mine` of them are g_gate's last
  const bool upper = c >= F;
  const int at = upper ? c - F : c, mine = upper ? 0 : min(F - c, 8);
  const bool whole = part * 512 + 512 <= F || (part * 512 >= F && part * 512 + 512 <= 2 * F);
  const IN *h = (const IN *)p.h + r * p.ld, *from_ga = (const IN *)p.ga + r * p.ga_ld;
  float v[8], up[8], ga[8];
  load_row(h, at, F, whole, v);
  load_row(h + F, at, F, whole, up);
  load_row(from_ga, at, F, whole, ga);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const Gate g = gate_of(v[j]);
    v[j] = upper ? gradient_of_up(g, ga[j]) : gradient_of_gate(g, up[j], ga[j]);
  }
  if (!whole && mine < 8 && mine > 0) {   // g_up's first behind g_gate's last
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= mine && j - mine < F) v[j] = gradient_of_up(gate_of(load_float(h + j - mine)), load_float(from_ga + j - mine));
  }
  if (p.gh) {
    if (p.gh_bf16) store_row((uint16_t *)p.gh + (int64_t)r * 2 * F, c, 2 * F, v);
    else store_row((float *)p.gh + (int64_t)r * 2 * F, c, 2 * F, v);
  }
  if (p.q) store_piece8(p.q + r * row8_bytes(2 * (int64_t)F), p.scale + r * scale8_bytes(2 * (int64_t)F), part, (int)row8_bytes(2 * (int64_t)F), v);
}

// Four values as they were loaded, zeros behind a row's end.
template <typename IN>
struct Four;
template <>
struct Four<uint16_t> {
  uint32_t w[2];
  // columns c to c + 3 of the row of C that begins `at` elements, less than 2^30, behind `rows`
  __device__ __forceinline__ void load(const uint16_t *rows, uint32_t at, int c, int C, bool whole) {
    if (whole) {
      const u32x2_align2 t = *(const u32x2_align2 *)((const char *)rows + (at + (uint32_t)c) * 2u);
      w[0] = t[0];
      w[1] = t[1];
    } else {
      float v[4];
      load_row_end<4>(rows + at, c, C, v);
#pragma unroll
      for (int i = 0; i < 2; ++i) w[i] = __builtin_bit_cast(uint32_t, v[2 * i]) >> 16 | __builtin_bit_cast(uint32_t, v[2 * i + 1]);
    }
  }
  __device__ __forceinline__ float at(int i) const { return i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]); }
  __device__ __forceinline__ void keep(bool there) {   // or zeros
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = there ? w[i] : 0u;
  }
};
template <>
struct Four<float> {
  float v[4];
  __device__ __forceinline__ void load(const float *rows, uint32_t at, int c, int C, bool whole) {
    if (whole) load_floats<4>((const float *)((const char *)rows + (at + (uint32_t)c) * 4u), v);
    else load_row_end<4>(rows + at, c, C, v);
  }
  __device__ __forceinline__ float at(int i) const { return v[i]; }
  __device__ __forceinline__ void keep(bool there) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = there ? v[i] : 0.0f;
  }
};
// The larger of each pair of lanes 16, or 32, apart, in both.
__device__ __forceinline__ uint32_t max_16_apart(uint32_t v) {
  const auto t = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return max((uint32_t)t[0], (uint32_t)t[1]);
}
__device__ __forceinline__ uint32_t max_32_apart(uint32_t v) {
  const auto t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max((uint32_t)t[0], (uint32_t)t[1]);
}

// The values of one element: g_gate, g_up and a.
struct Three {
  float v[3];
};
__device__ __forceinline__ Three three_of(float gate, float up, float ga) {
  const Gate g = gate_of(gate);
  return {{gradient_of_gate(g, up, ga), gradient_of_up(g, ga), g.times * up}};
}
__device__ __forceinline__ float finite_size(float v) { return fabsf(v) < __builtin_inff() ? fabsf(v) : 0.0f; }   // 0 of others

// A tile is a block of 128 rows of a segment and 128 columns of each half; a thread has four rows of four columns.  Rows leave from
// registers and the columns' largest values meet in LDS, and behind a barrier the values are turned in LDS and stored as columns.
// What a thread loads for the next tile is on its way meanwhile, so a workgroup goes through several; one fills a CU.
// 32,768 rows of F = 768 bf16 in all 8-bit layouts: 77 to 81 us, 277 MB at 3.5 TB/s, which copied would be 54; the vector unit is busy
// for 47 of them.  A workgroup a tile, nothing ahead, g_gate, g_up and a through LDS one after the other, took 194.  fp32 has twice
// the registers on their way and 72 to 104 bytes of a thread in scratch: loads later instead make no difference (5,003 rows of F =
// 1,001 53 us, two generations of tiles for 256 workgroups, of which the first waits for memory alone).
constexpr int kTurnThreads = 1024, kTurnPitch = 128 + 4, kTurnRows = 4, kTurnGroups = 256;
// Everybody's accesses of LDS are done; loads from memory stay on their way.
__device__ __forceinline__ void lds_barrier() {
  __asm__ volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  __asm__ volatile("" ::: "memory");
}
template <typename IN, bool VALUES>   // whether gh is wanted: stores of any alignment are much code, which runs cold
__global__ __launch_bounds__(kTurnThreads, 4) void gated_backward_kernel(GatedBackParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[3][128 * kTurnPitch];
  __shared__ uint32_t most_of[2][3][4][32];   // of every other tile: column 4 i + j at [j][i]
  __shared__ int32_t offsets[kMostSegments8 + 1];
  const int tid = threadIdx.x, lane = lane_id(), F = p.F;
  const int i32 = tid & 31, cl = i32 * 4, rl = (tid >> 5) * kTurnRows;
  for (int i = tid; i <= p.segments; i += kTurnThreads) offsets[i] = p.offsets[i];
  if (tid < 3 * 128) (&most_of[0][0][0][0])[tid] = 0;
  lds_barrier();
  const int64_t all = (int64_t)p.blocks * p.tiles, per_die = (all + 7) / 8;   // a die gets neighbouring tiles
  const int64_t last = min((int64_t)((blockIdx.x & 7) + 1) * per_die, all);
  int64_t at = (int64_t)(blockIdx.x & 7) * per_die + (blockIdx.x >> 3);
  struct Place {
    int b, c0, first, end;
  };
  auto next_place = [&](Place &t) {   // the next tile with rows; false: none is left
    for (; at < last; at += gridDim.x >> 3) {
      t.b = (int)(at / p.tiles);
      t.c0 = (int)(at - (int64_t)t.b * p.tiles) * 128;
      const BlockOwner8 owner = owner_of_block8(offsets, p.segments, (int)p.rows, t.b);
      t.end = owner.rows.to;
      t.first = owner.segment < 0 ? t.end : owner.rows.from + (t.b - first_block8(owner.rows.from, owner.segment)) * 128;
      if (t.first < t.end) {
        at += gridDim.x >> 3;
        t.b = __builtin_amdgcn_readfirstlane(t.b);
        t.c0 = __builtin_amdgcn_readfirstlane(t.c0);
        t.first = __builtin_amdgcn_readfirstlane(t.first);
        t.end = __builtin_amdgcn_readfirstlane(t.end);
        return true;
      }
    }
    return false;
  };
  Four<IN> gate[kTurnRows], up[kTurnRows], ga[kTurnRows];
  auto load = [&](const Place &t) {
    // uniform bases and offsets of 32 bits: addresses of 64 bits would take as many registers again as what they load
    const IN *from_h = (const IN *)p.h + (int64_t)t.first * p.ld, *from_ga = (const IN *)p.ga + (int64_t)t.first * p.ga_ld;
    const bool whole = t.c0 + 128 <= F;
#pragma unroll
    for (int i = 0; i < kTurnRows; ++i) {   // rows behind the segment are read from its last and count as zeros
      const uint32_t r = (uint32_t)min(rl + i, t.end - 1 - t.first);
      const uint32_t at_h = r * (uint32_t)p.ld, at_ga = r * (uint32_t)p.ga_ld;
      gate[i].load(from_h, at_h, t.c0 + cl, F, whole);
      up[i].load(from_h + F, at_h, t.c0 + cl, F, whole);
      ga[i].load(from_ga, at_ga, t.c0 + cl, F, whole);
    }
  };
  const int64_t width = row8_bytes(2 * (int64_t)F), scales = scale8_bytes(2 * (int64_t)F);
  const int64_t row_bytes = column8_blocks(p.rows, p.segments) * 128;
  Place place;
  if (!next_place(place)) return;
  load(place);
  for (int turn = 0;; turn ^= 1) {
    const int c = place.c0 + cl;
    float v[3][kTurnRows][4], column[3][4];
#pragma unroll
    for (int n = 0; n < 3; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) column[n][j] = 0.0f;
#pragma unroll
    for (int i = 0; i < kTurnRows; ++i) {
      const int64_t r = place.first + rl + i;
      const bool there = r < place.end;
      gate[i].keep(there);
      up[i].keep(there);
      ga[i].keep(there);
      float most[2] = {0.0f, 0.0f};   // a NaN does not count
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Three t = three_of(gate[i].at(j), up[i].at(j), ga[i].at(j));
#pragma unroll
        for (int n = 0; n < 3; ++n) {
          v[n][i][j] = t.v[n];
          column[n][j] = fmaxf(column[n][j], fabsf(t.v[n]));
          __asm__("" : "+v"(column[n][j]), "+v"(v[n][i][j]));   // now: put off, what they are computed from would take more registers
        }
#pragma unroll
        for (int n = 0; n < 2; ++n) most[n] = fmaxf(most[n], fabsf(t.v[n]));
      }
      if (VALUES && there) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          if (p.gh_bf16) store_row((uint16_t *)p.gh + r * 2 * F + n * F, c, F, v[n][i]);
          else store_row((float *)p.gh + r * 2 * F + n * F, c, F, v[n][i]);
        }
      }
      if (p.q) {   // whole blocks of both halves: F is a multiple of 128
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          if (most[n] == __builtin_inff()) {   // nor does an infinity; both become NaN in 8 bits
            most[n] = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) most[n] = fmaxf(most[n], finite_size(v[n][i][j]));
          }
          const int code = scale_code8(max_16_apart(max16(__builtin_bit_cast(uint32_t, most[n]))));
          if (there) {
            const int k = (n * F + place.c0) / 128;
            *(uint32_t *)(p.q + r * width + n * F + c) = pack8(v[n][i][0], v[n][i][1], v[n][i][2], v[n][i][3], inverse_scale8(code));
            if (i32 == 0) p.scale[r * scales + k] = (uint8_t)code;
            if (i32 < 3 && k == 2 * F / 128 - 1 && k + 1 + i32 < scales) p.scale[r * scales + k + 1 + i32] = 0;   // zeros behind the last
          }
        }
      }
    }
#pragma unroll
    for (int n = 0; n < 3; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (column[n][j] == __builtin_inff()) {
          column[n][j] = 0.0f;
#pragma unroll
          for (int i = 0; i < kTurnRows; ++i) column[n][j] = fmaxf(column[n][j], finite_size(v[n][i][j]));
        }
        const uint32_t most = max_32_apart(__builtin_bit_cast(uint32_t, column[n][j]));
        if (lane < 32) atomicMax(&most_of[turn][n][j][i32], most);
      }
    const Place here = place;
    const bool more = next_place(place);
    if (more) load(place);
    lds_barrier();
#pragma unroll
    for (int n = 0; n < 3; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int code = scale_code8(most_of[turn][n][j][i32]);
        *(uint32_t *)(turned[n] + (cl + j) * kTurnPitch + rl) = pack8(v[n][0][j], v[n][1][j], v[n][2][j], v[n][3][j], inverse_scale8(code));
      }
    if (tid < 128 && here.c0 + tid < F) {
#pragma unroll
      for (int n = 0; n < 3; ++n) {
        uint8_t *to = n < 2 ? p.scale_columns : p.a_scale;
        const int64_t C = n < 2 ? 2 * (int64_t)F : F;
        if (to) to[(int64_t)here.b * C + (n == 1 ? F : 0) + here.c0 + tid] = (uint8_t)scale_code8(most_of[turn][n][tid & 3][tid >> 2]);
      }
    }
    if (tid < 3 * 128) (&most_of[turn ^ 1][0][0][0])[tid] = 0;   // nobody has read it since the last tile's second barrier
    lds_barrier();
    const int col = tid >> 3, piece = (tid & 7) * 16;
    if (here.c0 + col < F) {
#pragma unroll
      for (int n = 0; n < 3; ++n) {
        uint8_t *to = n < 2 ? p.q_columns : p.a_columns;
        if (!to) continue;
        const uint32_t *in = (const uint32_t *)(turned[n] + col * kTurnPitch + piece);
        *(u32x4 *)(to + (int64_t)((n == 1 ? F : 0) + here.c0 + col) * row_bytes + (int64_t)here.b * 128 + piece) =
            u32x4{in[0], in[1], in[2], in[3]};
      }
    }
    if (!more) return;   // the same for the workgroup
  }
}

static bool segments_given_ok(const int32_t *offsets, int32_t segments, int64_t rows) {
  return !offsets || segments8_ok(segments, rows);
}
static unsigned gated_blocks(int64_t rows, int32_t parts) { return (unsigned)((rows * parts + kGatedWaves - 1) / kGatedWaves); }
constexpr int64_t kMostTurnPitch = 1 << 22;   // 128 rows of it within offsets of 32 bits
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
  if (rows * parts > kMostGatedPieces) return HM_ERR_SHAPE;
  const auto kernel = dtype == HM_BF16 ? gated_kernel<uint16_t> : gated_kernel<float>;
  hipLaunchKernelGGL(kernel, dim3(gated_blocks(rows, parts)), dim3(kGatedThreads), 0, (hipStream_t)hip_stream, p);
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
  if (rows * p.parts > kMostGatedPieces) return HM_ERR_SHAPE;
  if (columns) {
    p.blocks = (int32_t)column8_blocks(rows, segments);
    const int64_t workgroups = ((int64_t)p.blocks * p.tiles + 7) / 8 * 8;
    if (workgroups > (1 << 22) || ld > kMostTurnPitch || ga_ld > kMostTurnPitch) return HM_ERR_SHAPE;
    GatedBackParams tiles = p;
    if (by_rows) tiles.q = nullptr;
    const auto kernel = dtype == HM_BF16 ? gh ? gated_backward_kernel<uint16_t, true> : gated_backward_kernel<uint16_t, false>
                                         : gh ? gated_backward_kernel<float, true> : gated_backward_kernel<float, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(workgroups < kTurnGroups ? workgroups : kTurnGroups)), dim3(kTurnThreads), 0, (hipStream_t)hip_stream, tiles);
    const hm_status launched = hm_launch_status();
    if (launched != HM_OK || !by_rows) return launched;
    p.gh = nullptr;   // written
  }
  const auto kernel = dtype == HM_BF16 ? gated_backward_rows_kernel<uint16_t> : gated_backward_rows_kernel<float>;
  hipLaunchKernelGGL(kernel, dim3(gated_blocks(rows, p.parts)), dim3(kGatedThreads), 0, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}
