// The experts' products in 8 bits: rows ordered by expert times their expert's weights, and the weights' gradient.
//
// Both are D[q][p] = sum_k Q[q][k] P[p][k] with operands whose rows run along k in blocks of 128 that have a power of
// two each.
//   rows:   Q = rows of a segment, P = the expert's weights, k = columns
//   dw:     Q = columns of gy, P = columns of x, k = rows of the segment, padded to whole blocks with zeros
//
// Two ways to sum.  The matrix unit's products of 8 bits (32 x 32 x 64) apply the powers of two by themselves, but
// align the 64 products of a step to the largest and drop what lies more than 2^13 below it, and only then add in 32
// bits.  At most that is 2^-7 of a step's largest product.  Measured before the rounding, as a part of the results'
// norm (2,048 x 1,024 sums of 4,096 products): 1.5e-5 of normally distributed values, 4.5e-5, 7.1e-5 and 9.2e-5 where 8
// columns are 30, 100 and 1,000 times as large, 7.5e-5 of log-normal values (sigma 2), 5.1e-5 of bytes drawn evenly
// from all codes.  Rounding to bf16 costs 1.7e-3 in all of them, so that their error with and without the loss is the
// same in three digits; but where large products cancel nothing of the small ones is left.  So bf16 results of tiles
// take these products, which are twice as fast, unless the caller wants sums in 32 bits. Those, fp32 results, and bf16
// results of few rows, which memory bounds, have their operands turned into bf16 in registers, which is exact and takes
// the power of two along, and products of 16 bits, which are summed in 32 (1e-8 a step): 65,536 rows, 32 experts, 4,096
// x 7,168 3,110 us for 1,520.
#include "hm_block8.h"

namespace hm {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

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

// The tile of a workgroup among those of all segments, counted on the device: an expert's tiles lie together, the tiles
// of neighbouring rows next to one another, and every die gets a run of them, so that it reads few weights and rows.
template <int TQ, int TP>
__device__ __forceinline__ Tile tile_of_rows(const ProductParams &p) {
  const int lane = lane_id(), wide = (p.N + TP - 1) / TP;
  // the lane's segment of the first 64, which are most often all: one trip to memory
  const Segment8 mine = segment8(p.offsets, min(lane, p.experts - 1), p.rows);
  auto segment_at = [&](int e0) { return e0 == 0 ? mine : segment8(p.offsets, min(e0 + lane, p.experts - 1), p.rows); };
  auto strips_of = [&](int e0, const Segment8 &s) { return e0 + lane < p.experts ? (s.to - s.from + TQ - 1) / TQ : 0; };
  int total = 0;
  for (int e0 = 0; e0 < p.experts; e0 += kWave) total += read_lane(lane_scan(strips_of(e0, segment_at(e0))), kWave - 1);
  const int64_t tiles = (int64_t)total * wide, run = (tiles + 7) / 8;
  const int64_t at = (blockIdx.x & 7) * run + (blockIdx.x >> 3);
  if ((int64_t)(blockIdx.x >> 3) >= run || at >= tiles) return {0, 0, 0, 0};
  const int strip = (int)(at / wide);   // lies among the strips of the tile's own expert
  int before = 0;
  for (int e0 = 0; e0 < p.experts; e0 += kWave) {
    const Segment8 s = segment_at(e0);
    const int n = strips_of(e0, s), upto = before + lane_scan(n);
    const uint64_t behind = __ballot(upto > strip);
    if (behind) {
      const int l = __builtin_ctzll(behind), strips = read_lane(n, l);
      const int64_t local = at - (int64_t)(read_lane(upto, l) - strips) * wide;
      const int column = (int)(local / strips);
      const int q0 = read_lane(s.from, l) + (int)(local - (int64_t)column * strips) * TQ;
      return {e0 + l, q0, read_lane(s.to, l), column * TP};
    }
    before = read_lane(upto, kWave - 1);
  }
  return {0, 0, 0, 0};
}

template <typename OUT>
__device__ __forceinline__ void store4(OUT *at, const f32x4 &v) {   // at a multiple of four elements
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  // to nearest even, two an instruction
  if constexpr (sizeof(OUT) == 2) *(bf16x4 *)at = __builtin_convertvector(v, bf16x4);
  else *(f32x4 *)at = v;
}

// What a lane holds of a fragment's row for one part of a step, and its products.
template <bool FULL>
struct Slice;
template <>
struct Slice<false> {   // 32 values: one instruction, half a step
  i32x8 v;
  __device__ __forceinline__ void read(const uint8_t *lds, const uint32_t (&at)[4], int fragment, int part) {
    const i32x4 lo = *(const i32x4 *)(lds + at[2 * part] + fragment);
    const i32x4 hi = *(const i32x4 *)(lds + at[2 * part + 1] + fragment);
    v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  }
  static constexpr int kProducts = 1;
  __device__ __forceinline__ void times(const Slice &q, uint32_t code_p, uint32_t code_q, f32x16 &acc, int) const {
    // 0, 0: e4m3
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v, q.v, acc, 0, 0, 0, (int)code_p, 0, (int)code_q);
  }
};
template <>
struct Slice<true> {   // 16 values: two instructions, a quarter of a step
  i32x4 v;
  __device__ __forceinline__ void read(const uint8_t *lds, const uint32_t (&at)[4], int fragment, int part) {
    v = *(const i32x4 *)(lds + at[part] + fragment);
  }
  static constexpr int kProducts = 2;
  __device__ __forceinline__ void times(const Slice &q, uint32_t code_p, uint32_t code_q, f32x16 &acc, int h) const {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(v[2 * h], v[2 * h + 1], code_p),
                                                  widen8(q.v[2 * h], q.v[2 * h + 1], code_q), acc, 0, 0, 0);
  }
};

// A buffer from `at` on, as far as an offset of 32 bits goes: kernels keep their rows inside by themselves.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_resource(const uint8_t *at) {
  return __builtin_amdgcn_make_buffer_rsrc((void *)at, 0, (int)0xFFFFFFFFu, 0x00027000);
}

// All but the last LATER of the wave's loads have arrived in LDS, and then everybody's have; nobody has reads of LDS
// left.
template <int LATER>
__device__ __forceinline__ void arrived() {
  static_assert(LATER < 64, "the counter's range");
  __asm__ volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (LATER & 15) | (LATER >> 4) << 14);   // vmcnt(LATER) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  __asm__ volatile("" ::: "memory");
}

// One code of scale, or four.
template <bool ONE>
__device__ __forceinline__ uint32_t codes_at(__amdgpu_buffer_rsrc_t base, uint32_t at) {
  if constexpr (ONE) return __builtin_amdgcn_raw_buffer_load_b8(base, (int)at, 0, 0);
  else return __builtin_amdgcn_raw_buffer_load_b32(base, (int)at, 0, 0);
}

// FQ x FP fragments of 32 x 32 in a wave, WQ x WP waves.
//
// LDS is a ring of five units, a unit being one operand's rows of the tile for one step: Q0 P0 Q1 P1 Q2, then P2 in
// place of Q0 and so on, filled straight from memory.  Behind a step its two units are free; the next P is loaded into
// the one, the Q after the next into the other, so that the one has a step's time to arrive and the other two.  Whole
// rows of 128 bytes: of half the size (and twice the stages) they took the L2 nearly twice the requests.  A row's eight
// 16-byte pieces are stored at places exchanged by half the row number, so that sixteen rows of a fragment, which are
// read together, spread over all 64 banks.  Lane l has row l % 32 of a fragment and its pieces 4 (l / 32) to 4 (l / 32)
// + 3; which values meet in an instruction does not matter as long as both operands' lanes hold the same ones.
//
// 65,536 rows, 32 experts, 4,096 x 7,168, bf16 results 1,570 us (2.45 PFLOP/s; the products alone take 1,000, without
// loads 1,375: the unit's clock falls with what the rest draws); 32,768 rows, 16 experts, gradient of 1,536 x 2,048 in
// fp32 189 (1.09 PFLOP/s).
constexpr int kUnits = 5;
template <int FQ, int FP, int WQ, int WP, bool DW, bool kFull, typename OUT>
__global__ __launch_bounds__(WQ * WP * kWave, FQ * FP < 16 ? 2 : 1) void product_kernel(ProductParams p) {
  constexpr int kWaves = WQ * WP, TQ = FQ * WQ * 32, TP = FP * WP * 32;
  constexpr int kSlices = kFull ? 4 : 2, kUnitBytes = TQ * 128;
  static_assert(TQ == TP && kWaves % 2 == 0, "units of one size; the pieces' places go by the wave's number");
  constexpr int kLoads = TQ / 8 / kWaves;   // of a wave for a unit
  __shared__ __attribute__((aligned(128))) uint8_t ring[kUnits * kUnitBytes];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wq = wave / WP, wp = wave % WP;
  Tile t;
  int steps, q_rows, p_rows;
  const uint8_t *q, *ps;
  int64_t pitch;
  const int64_t scale_pitch = scale8_bytes(p.H);
  int block0 = 0;
  if constexpr (DW) {
    const int e = (int)blockIdx.z;
    const Segment8 s = segment8(p.offsets, e, p.rows);
    steps = (s.to - s.from + 127) / 128;
    block0 = first_block8(s.from, e);
    t = {e, (int)blockIdx.y * TQ, p.N, (int)blockIdx.x * TP};
    pitch = column8_blocks(p.rows, p.experts) * 128;
    q = p.q + (int64_t)block0 * 128;
    ps = p.p + (int64_t)block0 * 128;
    q_rows = p.N;
    p_rows = p.H;
  } else {
    t = tile_of_rows<TQ, TP>(p);
    if (t.q0 >= t.q_end) return;
    steps = (int)blocks8(p.H);
    pitch = row8_bytes(p.H);
    q = p.q;
    ps = p.p + (int64_t)t.expert * p.N * pitch;
    q_rows = t.q_end;
    p_rows = p.N;
  }
  // places of this lane's pieces; rows behind the last are read from the last, their products are not stored
  uint32_t from_q[kLoads], from_p[kLoads];
  // of row 8 (wave + i kWaves) + row8: half the row, modulo 8
  const int row8 = lane >> 3, piece = ((lane & 7) ^ ((lane >> 4) + 4 * (wave & 1))) * 16;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    from_q[i] = (uint32_t)min((wave + i * kWaves) * 8 + row8, q_rows - 1 - t.q0) * (uint32_t)pitch + piece;
    from_p[i] = (uint32_t)min((wave + i * kWaves) * 8 + row8, p_rows - 1 - t.p0) * (uint32_t)pitch + piece;
  }
  // uniform bases and 32-bit offsets: addresses of 64 bits per piece would not fit beside the sums
  const auto base_q = tile_resource(q + (int64_t)t.q0 * pitch), base_p = tile_resource(ps + (int64_t)t.p0 * pitch);
  // the i-th load of a unit; behind the last step the last again, which nobody reads
  auto load_q = [&](int at, int k, int i) {
    uint8_t *to = ring + at + (wave + i * kWaves) * 1024;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(base_q, (__attribute__((address_space(3))) void *)to, 16, (int)from_q[i],
                                             min(k, steps - 1) * 128, 0, 0);
  };
  auto load_p = [&](int at, int k, int i) {
    uint8_t *to = ring + at + (wave + i * kWaves) * 1024;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(base_p, (__attribute__((address_space(3))) void *)to, 16, (int)from_p[i],
                                             min(k, steps - 1) * 128, 0, 0);
  };
  // scales of this lane's row of each fragment; codes of a step in the lowest byte, rows: those of four steps are
  // loaded together
  uint32_t from_sq[FQ], from_sp[FP], scale_of_q[FQ], scale_of_p[FP], next_q[FQ], next_p[FP];
#pragma unroll
  for (int i = 0; i < FQ; ++i) {
    const int r = min((wq * FQ + i) * 32 + (lane & 31), q_rows - 1 - t.q0);
    from_sq[i] = (uint32_t)r * (uint32_t)(DW ? 1 : scale_pitch);
  }
#pragma unroll
  for (int i = 0; i < FP; ++i) {
    const int r = min((wp * FP + i) * 32 + (lane & 31), p_rows - 1 - t.p0);
    // the tile begins with a block, or one of 64 lies inside one
    from_sp[i] = DW ? (uint32_t)r : (uint32_t)(r / 128) * (uint32_t)scale_pitch;
  }
  auto load_scales = [&](int k) {
    const uint8_t *sq = p.q_scale + (DW ? (int64_t)(block0 + k) * p.N + t.q0 : (int64_t)t.q0 * scale_pitch + k);
    const uint8_t *sp = p.p_scale + (DW ? (int64_t)(block0 + k) * p.H + t.p0
                                        : ((int64_t)t.expert * blocks8(p.N) + t.p0 / 128) * scale_pitch + k);
#pragma unroll
    for (int i = 0; i < FQ; ++i) next_q[i] = codes_at<DW>(tile_resource(sq), from_sq[i]);
#pragma unroll
    for (int i = 0; i < FP; ++i) next_p[i] = codes_at<DW>(tile_resource(sp), from_sp[i]);
  };
  f32x16 acc[FQ][FP];
#pragma unroll
  for (int i = 0; i < FQ; ++i)
#pragma unroll
    for (int j = 0; j < FP; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
  // A step is a row of items: part item / FQ of fragment item % FQ of Q, times all of the wave's fragments of P.  An
  // item's operands are read two items ahead, so that the matrix unit always has some.
  constexpr int kItems = kSlices * FQ, kAhead = 2;
  Slice<kFull> of_q[4], of_p[2][FP];
  // piece 4 (l / 32) of this lane's row and those exchanged with it, in the units that are read
  uint32_t to_q[4], to_p[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const uint32_t at = (uint32_t)((lane & 31) * 128 + (((lane >> 5) * 4) ^ (lane >> 1 & 7) ^ v) * 16);
    to_q[v] = at + (uint32_t)(wq * FQ * 4096);
    to_p[v] = at + (uint32_t)(kUnitBytes + wp * FP * 4096);
  }
  auto read = [&](int item) {
    const int part = item / FQ;
    if (item % FQ == 0) {
#pragma unroll
      for (int j = 0; j < FP; ++j) of_p[part & 1][j].read(ring, to_p, j * 4096, part);
    }
    of_q[item & 3].read(ring, to_q, item % FQ * 4096, part);
  };
  auto two_on = [](int unit) { return unit + (unit >= 3 * kUnitBytes ? -3 * kUnitBytes : 2 * kUnitBytes); };
  // read; filled with the P of the next step and the Q after it
  int q_unit = 0, p_unit = kUnitBytes, free_p = 3 * kUnitBytes, free_q = 4 * kUnitBytes;
  // The loads are spread over the items since the last turn of the ring: a wave that issues many waits for the others'
  // before it multiplies on.  P, which is needed first, in the first half; `k`: the step of P.
  auto fill = [&](int from, int to, int k) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int when = i * (kItems / 2) / kLoads;
      if (when >= from && when < to) load_p(free_p, k, i);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int when = kItems / 2 + i * (kItems / 2) / kLoads;
      if (when >= from && when < to) load_q(free_q, k + 1, i);
    }
  };
  constexpr int kBefore = kAhead * 2 * kLoads / kItems;   // loads due in the items before a turn of the ring
  static_assert(kAhead * 2 * kLoads % kItems == 0 && kAhead <= kItems / 2, "whole loads, all of them P's");
  if (steps > 0) {   // arrived() counts the loads behind those that are needed, so their order is the program's
    load_scales(0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_q(0, 0, i);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_p(kUnitBytes, 0, i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_q(2 * kUnitBytes, 1, i);
    __builtin_amdgcn_sched_barrier(0);
    fill(0, kAhead, 1);
    arrived<kLoads + kBefore>();
#pragma unroll
    for (int item = 0; item < kAhead; ++item) read(item);
  }
  auto step = [&](int k) {
#pragma unroll
    for (int item = 0; item < kItems; ++item) {
      const Slice<kFull> mine = of_q[item & 3];
      Slice<kFull> other[FP];
#pragma unroll
      for (int j = 0; j < FP; ++j) other[j] = of_p[(item / FQ) & 1][j];
      // what is loaded and read ahead of the last step is not used: a branch around it would part the products from the
      // reads
      if (item + kAhead == kItems) {
        arrived<kLoads>();   // the next step, but for the Q after it; of this one nothing is left to read
        // five units: the P of step k + 2 takes the place of the Q of step k, the Q of k + 3 that of the P
        free_p = q_unit;
        free_q = p_unit;
        const int next_q_unit = two_on(q_unit), next_p_unit = two_on(p_unit);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          to_q[v] += (uint32_t)(next_q_unit - q_unit);
          to_p[v] += (uint32_t)(next_p_unit - p_unit);
        }
        q_unit = next_q_unit;
        p_unit = next_p_unit;
      }
      const int since = (item + kAhead) % kItems;
      fill(since, since + 1, item + kAhead < kItems ? k + 1 : k + 2);
      read((item + kAhead) % kItems);
      // one product after the other with other sums: one that waits for its own sum's last leaves the unit idle
#pragma unroll
      for (int h = 0; h < Slice<kFull>::kProducts; ++h)
#pragma unroll
        for (int j = 0; j < FP; ++j) other[j].times(mine, scale_of_p[j], scale_of_q[item % FQ], acc[item % FQ][j], h);
      // keeps the loads' order; and else the compiler reads all items at once and runs out of registers
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  constexpr int kScaled = DW ? 1 : 4;   // steps whose codes are loaded together, as long before their use
  auto shift_codes = [&] {
#pragma unroll
    for (int i = 0; i < FQ; ++i) scale_of_q[i] >>= 8;
#pragma unroll
    for (int i = 0; i < FP; ++i) scale_of_p[i] >>= 8;
  };
  auto take_codes = [&] {
#pragma unroll
    for (int i = 0; i < FQ; ++i) scale_of_q[i] = next_q[i];
#pragma unroll
    for (int i = 0; i < FP; ++i) scale_of_p[i] = next_p[i];
  };
  int k = 0;
  for (; k + kScaled <= steps; k += kScaled) {
    take_codes();
    load_scales(k + kScaled < steps ? k + kScaled : 0);
#pragma unroll
    for (int u = 0; u < kScaled; ++u) {
      if (u > 0) shift_codes();
      step(k + u);
    }
  }
  // what is left of the last four; one loop with an exit behind each step costs copies of the sums
  if constexpr (!DW) {
    take_codes();
#pragma unroll 1
    for (; k < steps; ++k) {
      step(k);
      shift_codes();
    }
  }
  // The wave's part of the tile through LDS, 32 rows at a time, so that stores are whole lines: a lane has row l % 32
  // of a fragment and of every eight columns the first or the last four.
  arrived<0>();   // nothing is on its way to LDS, nobody reads it
  constexpr int kCols = FP * 32, kRowBytes = kCols * (int)sizeof(OUT), kPitch = kRowBytes + 16;
  constexpr int kVec = 16 / (int)sizeof(OUT);
  static_assert(kWaves * 32 * kPitch <= kUnits * kUnitBytes, "the waves' rows fit the ring");
  uint8_t *mine = ring + wave * 32 * kPitch;
  const int c0 = t.p0 + wp * kCols, r_first = t.q0 + wq * FQ * 32;
  const int64_t out_pitch = DW ? p.H : p.N;
  OUT *out = (OUT *)p.out + (DW ? (int64_t)t.expert * p.N : 0) * out_pitch + c0;
  const bool vectors = ((uintptr_t)p.out & 15) == 0 && out_pitch % kVec == 0;   // of every row
#pragma unroll
  for (int i = 0; i < FQ; ++i) {
    const int r0 = r_first + i * 32;
#pragma unroll
    for (int j = 0; j < FP; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        store4((OUT *)(mine + (lane & 31) * kPitch) + j * 32 + g * 8 + (lane >> 5) * 4,
               f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]});
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (vectors) {
      constexpr int kLanes = kRowBytes / 16, kRows = kWave / kLanes;   // of a row; rows stored together
      const int c = lane % kLanes * kVec;
#pragma unroll
      for (int n = 0; n < 32 / kRows; ++n) {
        const int r = n * kRows + lane / kLanes;
        if (r0 + r < q_rows && c0 + c < p_rows) {
          const u32x4 v = *(const u32x4 *)(mine + r * kPitch + c * (int)sizeof(OUT));
          *(u32x4 *)(out + (int64_t)(r0 + r) * out_pitch + c) = v;
        }
      }
    } else {
#pragma unroll 1
      for (int n = lane; n < 32 * kCols; n += kWave) {
        const int r = n / kCols, c = n % kCols;
        if (r0 + r < q_rows && c0 + c < p_rows)
          out[(int64_t)(r0 + r) * out_pitch + c] = ((const OUT *)(mine + r * kPitch))[c];
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// ---- few rows ------------------------------------------------------------------------------------------
// The weights are all there is to read, once: 16 of their rows a workgroup, straight from memory into the operands of
// products of 16 x 16 x 32 in 16 bits, no LDS between; its four waves take every fourth group of four steps (512 bytes
// of a row, four codes of scale) and add up in LDS.  A lane has row l % 16 of the weights and of the segment, bytes 32
// (l / 16) to 32 (l / 16) + 31 of a step.  All results are sums in 32 bits: 8 rows for 8 experts of 4,096 x 7,168 42.7
// us, 5.5 TB/s (40.4 with the unit's products of 8 bits, whose sums lose bits), 32 rows for 32 experts 94.
constexpr int kThinWaves = 4, kGroupSteps = 4;
template <typename OUT>
__global__ __launch_bounds__(kThinWaves * kWave) void thin_product_kernel(ProductParams p) {
  __shared__ f32x4 sums[kThinWaves][kWave];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const Tile t = tile_of_rows<16, 16>(p);
  if (t.q0 >= t.q_end) return;
  const int steps = (int)blocks8(p.H), groups = (steps + kGroupSteps - 1) / kGroupSteps;
  const int64_t pitch = row8_bytes(p.H), scale_pitch = scale8_bytes(p.H);
  const int row = min(t.q0 + (lane & 15), t.q_end - 1), col = min(t.p0 + (lane & 15), p.N - 1);
  const uint8_t *q = p.q + (int64_t)row * pitch + (lane >> 4) * 32;
  const uint8_t *w = p.p + ((int64_t)t.expert * p.N + col) * pitch + (lane >> 4) * 32;
  const uint8_t *sq = p.q_scale + (int64_t)row * scale_pitch;
  const uint8_t *sp = p.p_scale + ((int64_t)t.expert * blocks8(p.N) + t.p0 / 128) * scale_pitch;
  struct Group {
    i32x8 q[kGroupSteps], w[kGroupSteps];
    uint32_t sq, sp;
  };
  auto load = [&](Group &g, int group) {   // steps behind the last are the last: their products are left out
#pragma unroll
    for (int s = 0; s < kGroupSteps; ++s) {
      const int64_t at = (int64_t)min(group * kGroupSteps + s, steps - 1) * 128;
      __builtin_memcpy(&g.w[s], __builtin_assume_aligned(w + at, 16), 32);
      __builtin_memcpy(&g.q[s], __builtin_assume_aligned(q + at, 16), 32);
    }
    g.sq = *(const uint32_t *)(sq + group * kGroupSteps);
    g.sp = *(const uint32_t *)(sp + group * kGroupSteps);
  };
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  auto multiply = [&](const Group &g, int group) {
#pragma unroll
    for (int s = 0; s < kGroupSteps; ++s) {
      if (group * kGroupSteps + s >= steps) break;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            widen8(g.w[s][2 * i], g.w[s][2 * i + 1], g.sp >> 8 * s),
            widen8(g.q[s][2 * i], g.q[s][2 * i + 1], g.sq >> 8 * s), acc, 0, 0, 0);
    }
  };
  Group a, b;   // one on its way while the other is multiplied
  int group = wave;
  if (group < groups) load(a, group);
  for (; group < groups; group += 2 * kThinWaves) {
    if (group + kThinWaves < groups) load(b, group + kThinWaves);
    multiply(a, group);
    if (group + kThinWaves < groups) {
      if (group + 2 * kThinWaves < groups) load(a, group + 2 * kThinWaves);
      multiply(b, group + kThinWaves);
    }
  }
  sums[wave][lane] = acc;
  __syncthreads();
  // thread: row / 16, column % 16 of the tile; lane l had row l % 16 and columns 4 (l / 16) to 4 (l / 16) + 3
  const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
  float sum = 0.0f;
#pragma unroll
  for (int v = 0; v < kThinWaves; ++v) sum += ((const float *)&sums[v][(c >> 2) * 16 + r])[c & 3];
  if (t.q0 + r < t.q_end && t.p0 + c < p.N) {
    OUT *out = (OUT *)p.out + (int64_t)(t.q0 + r) * p.N + t.p0 + c;
    if constexpr (sizeof(OUT) == 4) *out = sum;
    else *out = (OUT)f32_to_bf16(sum);
  }
}

static hm_status check_products(const void *a, const void *as, const void *b, const void *bs, const int32_t *offsets,
                                int32_t experts, int64_t rows, int32_t N, int32_t H, const void *out, hm_dtype dtype,
                                bool none) {
  if (!dtype_known(dtype) && dtype != HM_BF16_SUM_F32) return HM_ERR_SHAPE;
  if (!segments8_ok(experts, rows) || N < 1 || N > kMostColumns8 || H < 1 || H > kMostColumns8) return HM_ERR_SHAPE;
  if (!buffers8_aligned(a, as) || !buffers8_aligned(b, bs)) return HM_ERR_SHAPE;
  if ((uintptr_t)out & (dtype == HM_F32 ? 3 : 1)) return HM_ERR_SHAPE;
  if (none) return HM_OK;
  if (!a || !as || !b || !bs || !offsets || !out) return HM_ERR_NULL;
  return HM_OK;
}

// Rows and columns of a tile, from the tiles that there would be of 256 and of 128.  256 read the operands least often,
// but a CU holds one, so they need 400 and segments that fill them (us, 256 against 128: 16,384 rows, 16 experts, 1,536
// x 2,048 60.7 and 75.9; 8,192, 8, 4,096 x 7,168 241 and 282; 8,192, 32, 2,048 x 2,048 58.6 and 62.5, but 56.3 and 48.2
// where operands stay in the last-level cache); with fp32 sums, bound by products of 16 bits and by widening, 128 are
// as fast or faster, two to a CU (8,192, 8, 4,096 x 7,168 453 and 416), but for the gradient of the weights (32,768,
// 16, 1,536 x 2,048 191 and 207).  Tiles of 64 for few (64 against 128): 300 rows, 1, 4,096 x 7,168 39.3 and 44.0;
// 1,000, 1, 500 x 700 8.9 and 11.8; 2,048, 4, 1,024 x 2,048 14.8 and 15.9; 1,024, 8, 2,048 x 2,048 17.5 and 16.9; but
// 4,096, 2, 1,000 x 2,056 (256 tiles of 128) 27.5 and 19.4, 2,048, 32, 2,048 x 2,048 (512) 41.5 and 28.8.  Measured
// with operands in turn, so that they come from memory.
static int tile_side(bool large, int64_t tiles128) { return large ? 256 : tiles128 >= 200 ? 128 : 64; }

template <int FQ, int FP, int WQ, int WP, bool DW>
static hm_status launch_tiles(const ProductParams &p, hm_dtype dtype, dim3 grid, void *stream) {
  const auto kernel = dtype == HM_F32            ? product_kernel<FQ, FP, WQ, WP, DW, true, float>
                      : dtype == HM_BF16_SUM_F32 ? product_kernel<FQ, FP, WQ, WP, DW, true, uint16_t>
                                                 : product_kernel<FQ, FP, WQ, WP, DW, false, uint16_t>;
  hipLaunchKernelGGL(kernel, grid, dim3(WQ * WP * kWave), 0, (hipStream_t)stream, p);
  return hm_launch_status();
}
template <bool DW>
static hm_status launch_products(const ProductParams &p, int side, hm_dtype dtype, dim3 grid, void *stream) {
  if (side == 256) {
    if constexpr (DW) return launch_tiles<4, 4, 2, 2, true>(p, dtype, grid, stream);
    hipLaunchKernelGGL((product_kernel<4, 4, 2, 2, false, false, uint16_t>), grid, dim3(256), 0,
                       (hipStream_t)stream, p);
    return hm_launch_status();
  }
  if (side == 128) return launch_tiles<2, 2, 2, 2, DW>(p, dtype, grid, stream);
  return launch_tiles<2, 1, 1, 2, DW>(p, dtype, grid, stream);
}

}  // namespace hm

extern "C" hm_status hm_expert_matmul(const uint8_t *x, const uint8_t *x_scale, const uint8_t *w,
                                      const uint8_t *w_scale, const int32_t *offsets, int32_t experts, int64_t rows,
                                      int32_t N, int32_t H, void *out, hm_dtype out_dtype, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  const hm_status bad = check_products(x, x_scale, w, w_scale, offsets, experts, rows, N, H, out, out_dtype, rows == 0);
  if (bad != HM_OK) return bad;
  if (rows == 0) return HM_OK;
  // strips of 16 rows are counted in 32 bits, also where offsets overlap
  if (rows * experts >= 1LL << 35) return HM_ERR_SHAPE;
  const ProductParams p = {x, x_scale, w, w_scale, offsets, experts, (int32_t)rows, N, H, out};
  // Few rows: up to four an expert, or 32 in all (us, strips against tiles with sums in 32 bits and in the unit's 8-bit
  // products, operands from memory: 32 experts of 4,096 x 7,168, 32 rows 94, 137 and 126; 128 rows 165, 212 and 158;
  // 256 rows 190, 213 and 158; 32 of 2,048 x 2,048, 128 rows 34, 33 and 27; one of 4,096 x 7,168, 32 rows 17.7, 43 and
  // 38; 64 rows 28.8, 43 and 38; one of 7,168 x 2,048, 32 rows 11.9, 15 and 13; 48 rows 15.8, 15 and 13). More strips
  // than a launch has workgroups go by tiles, with the same sums.
  const bool few = rows <= 4LL * experts || rows <= 32;
  const int64_t strips = (rows / 16 + (rows < experts ? rows : experts)) * ((N + 15) / 16) + 8;
  if (few && out_dtype == HM_BF16) out_dtype = HM_BF16_SUM_F32;
  if (few && strips <= 1 << 23) {
    const auto kernel = out_dtype == HM_F32 ? thin_product_kernel<float> : thin_product_kernel<uint16_t>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)strips), dim3(kThinWaves * kWave), 0, (hipStream_t)hip_stream, p);
    return hm_launch_status();
  }
  const bool large = out_dtype == HM_BF16 && rows / experts >= 512 &&
                     (rows / 256 + experts / 2) * ((N + 255) / 256) >= 400;
  const int side = tile_side(large, (rows / 128 + experts / 2) * ((N + 127) / 128));
  const int64_t tiles = (rows / side + experts) * ((N + side - 1) / side) + 8;
  if (tiles > (1 << 23)) return HM_ERR_SHAPE;
  return launch_products<false>(p, side, out_dtype, dim3((unsigned)tiles), hip_stream);
}

extern "C" hm_status hm_expert_matmul_dw(const uint8_t *gy, const uint8_t *gy_scale, const uint8_t *x,
                                         const uint8_t *x_scale, const int32_t *offsets, int32_t experts, int64_t rows,
                                         int32_t N, int32_t H, void *dw, hm_dtype dw_dtype, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  const hm_status bad = check_products(gy, gy_scale, x, x_scale, offsets, experts, rows, N, H, dw, dw_dtype, false);
  if (bad != HM_OK) return bad;
  if (column8_blocks(rows, experts) >= (1 << 17)) return HM_ERR_SHAPE;   // 256 rows of a tile within offsets of 32 bits
  const ProductParams p = {gy, gy_scale, x, x_scale, offsets, experts, (int32_t)rows, N, H, dw};
  const bool large = (int64_t)((H + 255) / 256) * ((N + 255) / 256) * experts >= 256;
  const int side = tile_side(large, (int64_t)((H + 127) / 128) * ((N + 127) / 128) * experts);
  const dim3 grid((unsigned)((H + side - 1) / side), (unsigned)((N + side - 1) / side), (unsigned)experts);
  return launch_products<true>(p, side, dw_dtype, grid, hip_stream);
}
