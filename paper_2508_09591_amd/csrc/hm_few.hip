// A whole layer for a few tokens: choice, both products, activation and weighted sum, without a plan and without rows in 8 bits.
//     out[t] = sum_k w[t,k] w2_e (silu(gate) up),   [gate; up] = w13_e x[t],   e = ids[t,k] - first
// The weights of the experts hit are all there is to read, once: 16 of their rows a workgroup, straight from memory into the
// operands of products of 16 x 16 x 32 in 16 bits, as for the products of few rows.  Values in 8 bits times their block's power of
// two are exact in bf16, x is bf16; activations go between the two products as sums of two or three bf16 numbers, so that what
// they lose is far below the output's rounding (2^-17 of each, 2^-25 for fp32 outputs).
// us, and weights a second: a token's 8 experts of 7,168 x 2,048 74 (353 MB, 4.8 TB/s), of 2,048 x 768 18 (38 MB: two launches of two
// trips to memory each); 64 tokens on 32 experts of the former 230 (1.23 GB, 5.3 TB/s).
#include "hm_choice.h"

namespace hm {

constexpr int kMostFewTokens = 64, kMostFewSlots = 1024;

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct FewParams {
  const uint16_t *x;
  int64_t ld;
  int32_t *ids;            // [T,K]
  float *weights;
  int32_t T, K, first, experts, H, F;
  uint32_t per_K;          // ceil(2^20 / K)
  const uint8_t *w13, *s13, *w2, *s2;
  uint16_t *a;             // [planes, T K, up(F,128)]
  float *y;                // [T K, H]
  void *out;
};

// A workgroup's expert and the slots that chose it.  There are as many workgroups' shares as experts here, or, if those are fewer,
// as slots: a slot's are taken where no slot before it has chosen the same expert.
__device__ __forceinline__ int expert_here(const FewParams &p, int slot) {   // -1: none or elsewhere
  const int e = p.ids[slot] - p.first;
  return (unsigned)e < (unsigned)p.experts ? e : -1;
}
// Writes the slots, ascending, to `list`, one of the wave's own: at most one of a token's.  0: nothing to do.  By whole waves.
// `expert_of` says what expert_here does.
template <typename EXPERT>
__device__ __forceinline__ int slots_of_share(const FewParams &p, int share, EXPERT expert_of, int &e, int *list) {
  const int lane = lane_id(), slots = p.T * p.K;
  const bool by_slot = slots < p.experts;
  e = by_slot ? expert_of(share) : share;
  int n = 0;
  auto take = [&](int s, int expert) {
    const uint64_t all = __ballot(s < slots && expert == e);
    const int at = n + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));   // before this lane
    if (s < slots && expert == e && at < kMostFewTokens) list[at] = s;
    n += __popcll(all);
  };
  if (slots <= kWave) {
    take(lane, expert_of(min(lane, slots - 1)));
  } else {
    constexpr int kTogether = 4;   // loads on their way
    for (int s0 = 0; s0 < slots; s0 += kTogether * kWave) {
      int expert[kTogether];
#pragma unroll
      for (int i = 0; i < kTogether; ++i) expert[i] = expert_of(min(s0 + i * kWave + lane, slots - 1));
#pragma unroll
      for (int i = 0; i < kTogether; ++i) take(s0 + i * kWave + lane, expert[i]);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (e < 0 || n == 0 || (by_slot && __builtin_amdgcn_readfirstlane(list[0]) != share)) return 0;
  return min(n, kMostFewTokens);
}

// slot / K: slots are below 2^10, so that what per_K is too large by does not reach the next multiple.
__device__ __forceinline__ int token_of(const FewParams &p, int slot) { return (int)((uint32_t)slot * p.per_K >> 20); }

// 32 bytes of a weight's row, 32 bf16 numbers.
__device__ __forceinline__ i32x8 load32(const uint8_t *p) {
  i32x8 v;
  __builtin_memcpy(&v, __builtin_assume_aligned(p, 16), 32);
  return v;
}
struct Wide {
  bf16x8 v[4];
};
__device__ __forceinline__ Wide load_wide(const uint16_t *p) {   // at any alignment of the elements
  Wide w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w.v[i] = __builtin_bit_cast(bf16x8, (u32x4)*(const u32x4_align2 *)(p + 8 * i));
  return w;
}
// The same of a row of H from column c on, zeros behind its end: vectors that would pass it are loaded from before it and moved down.
__device__ __forceinline__ Wide load_wide_end(const uint16_t *row, int c, int H) {
  Wide w;
#pragma unroll
  for (int i = 0; i < 4; ++i, c += 8) {
    u32x4 v = {0, 0, 0, 0};
    if (H < 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j / 2] |= c + j < H ? (uint32_t)row[c + j] << 16 * (j & 1) : 0u;
    } else {
      const int at = min(c, H - 8), by = c - at;
      v = *(const u32x4_align2 *)(row + at);
      v = by & 4 ? u32x4{v[2], v[3], 0, 0} : v;
      v = by & 2 ? u32x4{v[1], v[2], v[3], 0} : v;
      v = by & 1 ? u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16} : v;
      v = by < 8 ? v : u32x4{0, 0, 0, 0};
    }
    w.v[i] = __builtin_bit_cast(bf16x8, v);
  }
  return w;
}
__device__ __forceinline__ Wide zero_wide() {
  Wide w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w.v[i] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
  return w;
}

// ---- the first product and the activation --------------------------------------------------------------
// A workgroup takes an expert and 16 columns of its activation: as many rows of the gate's weights and of the up's.  Its four
// waves share the steps of 128 columns of x and add up in LDS.  A lane has row l % 16 of the weights and of the slots, bytes
// 32 (l / 16) to 32 (l / 16) + 31 of a step.  Two strips of columns a workgroup, eight waves, x in LDS and loads past the caches
// were no faster.
constexpr int kUpWaves = 4;

// GROUPS: of 16 slots each that one reading of the weights serves.
// N: with up to four tokens every workgroup makes the choice by itself, lists of N, 16 lanes a token in its first wave, which takes it
// less time than another launch would; the first one writes it down.  0: it has been made.
constexpr int kChoosingTokens = kWave / 16;
template <typename LOGIT, int N, int GROUPS, int PLANES>
__global__ __launch_bounds__(kUpWaves * kWave) void few_up_kernel(FewParams p, RouteParams route, int lanes_per_group, int run) {
  __shared__ int lists[kUpWaves][kMostFewTokens];
  __shared__ f32x4 sums[kUpWaves][2][kWave];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int width_a = (int)row8_bytes(p.F), slots = p.T * p.K;
  const int *list = lists[wave];
  const int share = (int)blockIdx.y, f0 = (int)blockIdx.x * 16;
  int e, all;
  if constexpr (N > 0) {
    __shared__ int chosen[kWave];
    if (wave == 0) {
      const int t = lane >> 4;
      choose_by_lists<LOGIT, 16, N>(route, t, lanes_per_group, run, [&](int k, int expert, float weight) {
        const int slot = t * p.K + k, here = expert - p.first;
        chosen[slot] = (unsigned)here < (unsigned)p.experts ? here : -1;
        if (blockIdx.x == 0 && blockIdx.y == 0) {
          p.ids[slot] = expert;
          p.weights[slot] = weight;
        }
      });
    }
    __syncthreads();
    all = slots_of_share(p, share, [&](int slot) { return chosen[slot]; }, e, lists[wave]);
  } else {
    all = slots_of_share(p, share, [&](int slot) { return expert_here(p, slot); }, e, lists[wave]);
  }
  if (all == 0) return;   // the same for the workgroup
  const int row = lane & 15, part = (lane >> 4) * 32, steps = (int)blocks8(p.H);
  const int64_t pitch = row8_bytes(p.H), scale_pitch = scale8_bytes(p.H);
  const uint8_t *w = p.w13 + (int64_t)e * 2 * p.F * pitch + part, *s = p.s13 + (int64_t)e * blocks8(2 * (int64_t)p.F) * scale_pitch;
  const uint8_t *from[2], *scale[2];   // of gate and up
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int n = min(f0 + row, p.F - 1) + h * p.F;
    from[h] = w + n * pitch;
    scale[h] = s + (n / 128) * scale_pitch;
  }
  for (int first = 0; first < all; first += 16 * GROUPS) {   // more slots than that read the weights again
    const int n = all - first;
    const uint16_t *x[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) x[g] = p.x + (int64_t)token_of(p, list[first + min(g * 16 + row, n - 1)]) * p.ld;
    f32x4 acc[GROUPS][2];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) acc[g][0] = acc[g][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    struct Step {
      i32x8 w[2];
      uint32_t scale[2];
      Wide x[GROUPS];
    };
    auto load = [&](Step &t, int k) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        t.w[h] = load32(from[h] + (int64_t)k * 128);
        t.scale[h] = scale[h][k];
      }
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        t.x[g] = zero_wide();
        if (g * 16 >= n) continue;
        if (g * 16 + row >= n) continue;
        if (k * 128 + 128 <= p.H) t.x[g] = load_wide(x[g] + k * 128 + part);
        else t.x[g] = load_wide_end(x[g], k * 128 + part, p.H);
      }
    };
    auto multiply = [&](const Step &t) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8 u = widen8(t.w[h][2 * i], t.w[h][2 * i + 1], t.scale[h]);
#pragma unroll
          for (int g = 0; g < GROUPS; ++g)
            if (g * 16 < n) acc[g][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, t.x[g].v[i], acc[g][h], 0, 0, 0);
        }
    };
    Step a, b;   // one on its way while the other is multiplied
    int k = wave;
    if (k < steps) load(a, k);
    for (; k < steps; k += 2 * kUpWaves) {
      if (k + kUpWaves < steps) load(b, k + kUpWaves);
      multiply(a);
      if (k + kUpWaves < steps) {
        if (k + 2 * kUpWaves < steps) load(a, k + 2 * kUpWaves);
        multiply(b);
      }
    }
    // thread: slot / 16, column % 16 of a group; lane l had slot l % 16 and columns 4 (l / 16) to 4 (l / 16) + 3
    const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      if (g * 16 >= n) break;   // the same for the workgroup
      if (first + g > 0) __syncthreads();
      sums[wave][0][lane] = acc[g][0];
      sums[wave][1][lane] = acc[g][1];
      __syncthreads();
      if (g * 16 + r >= n) continue;
      float v[2] = {0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < kUpWaves; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] += ((const float *)&sums[u][h][(c >> 2) * 16 + r])[c & 3];
      const int column = f0 + c;
      float rest = column < p.F ? v[0] / (1.0f + expf(-v[0])) * v[1] : 0.0f;   // zeros up to a whole block
      const int64_t at = (int64_t)list[first + g * 16 + r] * width_a + column;
#pragma unroll
      for (int plane = 0; plane < PLANES; ++plane) {
        const uint32_t bits = round_bf16x2(rest, rest);
        p.a[(int64_t)plane * slots * width_a + at] = (uint16_t)bits;
        const float part_of = bf16_lo(bits);
        rest = fabsf(part_of) < __builtin_inff() ? rest - part_of : 0.0f;   // an infinity's or a NaN's rest is none
      }
    }
  }
}

// ---- the second product and the sum over a token's experts ---------------------------------------------
// Few slots: a workgroup takes up to 16 columns of the output, all activations stand in its LDS, and its waves share the weights'
// rows of all experts hit evenly, in pieces of four steps; behind an expert's pieces a wave adds what its slots get, times their
// weights, to its own sums of the tokens, which are added up in the end.  Activations read from memory in between would come behind the
// weights that are on their way, as loads return in order: 41 us for a token's 8 experts of 7,168 x 2,048, 28 from LDS.
constexpr int kDownWaves = 8, kPieceSteps = 4;
template <int PLANES, typename OUT>
__global__ __launch_bounds__(kDownWaves * kWave, PLANES == 2 ? 4 : 2) void few_down_kernel(FewParams p, int columns) {
  extern __shared__ __attribute__((aligned(16))) float sums[];   // [waves][T][16], and the activations behind them
  __shared__ int lists[kDownWaves][kWave];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int width_a = (int)row8_bytes(p.F), slots = p.T * p.K, row = lane & 15, part = (lane >> 4) * 32, h0 = (int)blockIdx.x * columns;
  const int mine_is = lane < slots ? expert_here(p, lane) : -1;   // at most 64 slots
  const int pitch_a = width_a + 8;   // of a row in LDS: rows read together lie in different banks
  uint16_t *staged = (uint16_t *)(sums + kDownWaves * p.T * 16);
  uint64_t hit = 0;   // slots that are their expert's first
  for (int s = 0; s < slots; ++s) {
    const int e = read_lane(mine_is, s);
    hit |= (uint64_t)(e >= 0 && __builtin_ctzll(__ballot(mine_is == e)) == s) << s;
  }
  const int steps = (int)blocks8(p.F), pieces = (steps + kPieceSteps - 1) / kPieceSteps, h = min(h0 + min(row, columns - 1), p.H - 1);
  const int64_t pitch = row8_bytes(p.F), scale_pitch = scale8_bytes(p.F);
  const int all = __popcll(hit) * pieces, end = (int)((int64_t)all * (wave + 1) / kDownWaves);
  int at = (int)((int64_t)all * wave / kDownWaves);
  for (int skip = at / pieces; skip > 0; --skip) hit &= hit - 1;
  struct Piece {
    i32x8 w[kPieceSteps];
    uint32_t scales;
  };
  auto load = [&](Piece &t, int e, int piece) {   // steps behind the last are the last: their products are left out
    const uint8_t *w = p.w2 + ((int64_t)e * p.H + h) * pitch + part;
#pragma unroll
    for (int s = 0; s < kPieceSteps; ++s) {
      t.w[s] = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
      if (row < columns) t.w[s] = load32(w + (int64_t)min(piece * kPieceSteps + s, steps - 1) * 128);
    }
    t.scales = *(const uint32_t *)(p.s2 + ((int64_t)e * blocks8(p.H) + h / 128) * scale_pitch + piece * kPieceSteps);
  };
  Piece x, y;   // one on its way while the other is multiplied
  if (at < end) load(x, read_lane(mine_is, __builtin_ctzll(hit)), at % pieces);
  const int vectors = width_a / 8;
  for (int i = threadIdx.x; i < PLANES * slots * vectors; i += kDownWaves * kWave) {   // those of slots elsewhere nobody reads
    const int r = i / vectors, c = i - r * vectors;
    *(u32x4 *)(staged + r * pitch_a + c * 8) = *(const u32x4 *)(p.a + (int64_t)i * 8);
  }
  for (int i = threadIdx.x; i < kDownWaves * p.T * 16; i += kDownWaves * kWave) sums[i] = 0.0f;
  __syncthreads();
  int *list = lists[wave];
  float *mine = sums + wave * p.T * 16;
  while (at < end) {
    const int from = at % pieces, to = min(pieces, from + end - at);
    const int e = read_lane(mine_is, __builtin_ctzll(hit));
    const uint64_t chosen = __ballot(mine_is == e);
    const int n = __popcll(chosen);
    if (chosen >> lane & 1) list[__popcll(chosen & ((1ull << lane) - 1))] = lane;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    at += to - from;
    hit &= hit - 1;
    for (int first = 0; first < n; first += 16) {   // more than 16 slots of an expert: its weights again
      if (first > 0) load(x, e, from);
      const int slot = first + row < n ? list[first + row] : -1;
      const float by = slot >= 0 ? p.weights[slot] : 0.0f;
      const uint16_t *a = staged + max(slot, 0) * pitch_a + part;
      f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
      auto multiply = [&](const Piece &t, int piece) {
#pragma unroll
        for (int s = 0; s < kPieceSteps; ++s) {
          const int step = piece * kPieceSteps + s;
          if (step >= steps) break;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bf16x8 u = widen8(t.w[s][2 * i], t.w[s][2 * i + 1], t.scales >> 8 * s);
#pragma unroll
            for (int plane = 0; plane < PLANES; ++plane) {
              const bf16x8 v = *(const bf16x8 *)(a + plane * slots * pitch_a + step * 128 + i * 8);
              acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, v, acc, 0, 0, 0);
            }
          }
        }
      };
      for (int piece = from; piece < to; piece += 2) {
        if (piece + 1 < to) load(y, e, piece + 1);
        multiply(x, piece);
        if (piece + 1 < to) {
          if (piece + 2 < to) load(x, e, piece + 2);
          multiply(y, piece + 1);
        }
      }
      if (first + 16 >= n && at < end) load(x, read_lane(mine_is, __builtin_ctzll(hit)), 0);   // the next expert's
      if (slot >= 0) {   // lane: slot l % 16, columns 4 (l / 16) to 4 (l / 16) + 3; a token has one slot of an expert
        float *to_token = mine + token_of(p, slot) * 16 + (lane >> 4) * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) to_token[i] = fmaf(by, acc[i], to_token[i]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.T * 16; i += kDownWaves * kWave) {
    const int t = i >> 4, c = i & 15;
    if (c >= columns || h0 + c >= p.H) continue;
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < kDownWaves; ++u) sum += sums[(u * p.T + t) * 16 + c];
    store_float((OUT *)p.out + (int64_t)t * p.H + h0 + c, sum);
  }
}

// The same by experts: a workgroup takes one and FRAGS times 16 columns of the output, and leaves what its slots get; its four waves
// take every fourth step.  64 tokens on 32 experts of 7,168 x 2,048 79 to 89 us (5.3 to 6 TB/s) and the sum's 5; all slots' activations do
// not fit LDS there, and with all of a workgroup's experts in turn it took 453.
template <int PLANES, int FRAGS>
__global__ __launch_bounds__(kUpWaves * kWave) void few_down_slots_kernel(FewParams p) {
  __shared__ int lists[kUpWaves][kMostFewTokens];
  __shared__ f32x4 sums[kUpWaves][FRAGS][kWave];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int slots = p.T * p.K, width_a = (int)row8_bytes(p.F);
  const int *list = lists[wave];
  const int share = (int)blockIdx.y, h0 = (int)blockIdx.x * 16 * FRAGS;
  int e;
  const int n = slots_of_share(p, share, [&](int slot) { return expert_here(p, slot); }, e, lists[wave]);
  if (n == 0) return;   // the same for the workgroup
  const int row = lane & 15, part = (lane >> 4) * 32, steps = (int)blocks8(p.F);
  const int64_t pitch = row8_bytes(p.F), scale_pitch = scale8_bytes(p.F);
  const uint8_t *w[FRAGS], *scale[FRAGS];
#pragma unroll
  for (int f = 0; f < FRAGS; ++f) {
    const int h = min(h0 + f * 16 + row, p.H - 1);
    w[f] = p.w2 + ((int64_t)e * p.H + h) * pitch + part;
    scale[f] = p.s2 + ((int64_t)e * blocks8(p.H) + h / 128) * scale_pitch;
  }
  for (int first = 0; first < n; first += 16) {
    const int slot = first + row < n ? list[first + row] : -1;
    const uint16_t *a = p.a + (int64_t)max(slot, 0) * width_a + part;
    struct Step {
      i32x8 w[FRAGS];
      uint32_t scale[FRAGS];
      Wide a[PLANES];
    };
    f32x4 acc[FRAGS];
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) acc[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto load = [&](Step &t, int k) {
#pragma unroll
      for (int f = 0; f < FRAGS; ++f) {
        t.w[f] = load32(w[f] + (int64_t)k * 128);
        t.scale[f] = scale[f][k];
      }
#pragma unroll
      for (int plane = 0; plane < PLANES; ++plane) {
        t.a[plane] = zero_wide();
        if (slot >= 0) t.a[plane] = load_wide(a + (int64_t)plane * slots * width_a + k * 128);
      }
    };
    auto multiply = [&](const Step &t) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) {
          const bf16x8 u = widen8(t.w[f][2 * i], t.w[f][2 * i + 1], t.scale[f]);
#pragma unroll
          for (int plane = 0; plane < PLANES; ++plane)
            acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, t.a[plane].v[i], acc[f], 0, 0, 0);
        }
    };
    Step x, y;   // one on its way while the other is multiplied
    int k = wave;
    if (k < steps) load(x, k);
    for (; k < steps; k += 2 * kUpWaves) {
      if (k + kUpWaves < steps) load(y, k + kUpWaves);
      multiply(x);
      if (k + kUpWaves < steps) {
        if (k + 2 * kUpWaves < steps) load(x, k + 2 * kUpWaves);
        multiply(y);
      }
    }
    if (first > 0) __syncthreads();
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) sums[wave][f][lane] = acc[f];
    __syncthreads();
    const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) {
      float sum = 0.0f;
#pragma unroll
      for (int u = 0; u < kUpWaves; ++u) sum += ((const float *)&sums[u][f][(c >> 2) * 16 + r])[c & 3];
      const int h = h0 + f * 16 + c;
      if (first + r < n && h < p.H) p.y[(int64_t)list[first + r] * p.H + h] = sum;
    }
  }
}
// out[t] = sum over k of w[t,k] y[t,k], k ascending.
template <typename OUT>
__global__ __launch_bounds__(256) void few_sum_kernel(FewParams p) {
  const int h = (int)blockIdx.x * 256 + (int)threadIdx.x, t = (int)blockIdx.y;
  if (h >= p.H) return;
  float sum = 0.0f;
#pragma unroll 8
  for (int k = 0; k < p.K; ++k) {
    const int slot = t * p.K + k;
    if ((unsigned)(p.ids[slot] - p.first) < (unsigned)p.experts) sum = fmaf(p.weights[slot], p.y[(int64_t)slot * p.H + h], sum);
  }
  store_float((OUT *)p.out + (int64_t)t * p.H + h, sum);
}

template <typename LOGIT, int N, int GROUPS, int PLANES>
static void launch_few_up(const FewParams &p, const RouteParams &route, int64_t shares, hipStream_t stream) {
  int lanes_per_group = 0, run = 0;
  if (N > 0) {   // of the choice by lists, which has at most 16 groups; other routers have more groups than lanes
    lanes_per_group = 16 / route.r.groups;
    run = (route.r.E / route.r.groups + lanes_per_group - 1) / lanes_per_group;
  }
  hipLaunchKernelGGL((few_up_kernel<LOGIT, N, GROUPS, PLANES>), dim3((unsigned)(row8_bytes(p.F) / 16), (unsigned)shares),
                     dim3(kUpWaves * kWave), 0, stream, p, route, lanes_per_group, run);
}
// The choice by the workgroups of the first product, as far as it goes.
static bool chooses_itself(const RouteParams &route) {
  return route.T <= kChoosingTokens && list_lanes(route.r, route.bias != nullptr, route.T) == 16;
}
template <typename LOGIT, int PLANES>
static void launch_choosing_up(const FewParams &p, const RouteParams &route, int64_t shares, hipStream_t stream) {
  if (p.K <= 8) launch_few_up<LOGIT, 8, 1, PLANES>(p, route, shares, stream);
  else launch_few_up<LOGIT, 16, 1, PLANES>(p, route, shares, stream);
}
// Dynamic LDS that few_down_kernel may have, more than a kernel gets by default.  It takes in the eight slots of one token of
// 2,048 columns, and leaves room for two workgroups a CU.
constexpr int kMostStaged = 66 * 1024;
template <int PLANES, typename OUT>
static int64_t staged_limit() {
  static LdsGrant grant;
  return lds_granted(grant, (const void *)few_down_kernel<PLANES, OUT>, kMostStaged) ? kMostStaged : 65536 - 4096;   // beside what it has anyway
}
template <int PLANES, typename OUT>
static hm_status launch_few(const FewParams &p, const RouteParams &route, hm_dtype logits, int64_t shares, hipStream_t stream) {
  // The choice inside the first product: one token of 128 experts of 2,048 x 768 18.2 us, with a launch of its own 19.6.
  // Four groups of slots take registers, hence waves, one reads an expert's weights again where there are more.  us with one and four:
  // 8 experts of 7,168 x 2,048 and 5, 8, 10, 16 slots each (of 20 to 64 tokens) 81 and 88, 93 and 97, 100 and 98, 165 and 128; 32 experts
  // and 8, 10, 16 of 8 a token 324 and 332, 335 and 344, 478 and 432; of 2,048 x 768 50 and 54, 54 and 58, 77 and 73.  Two groups
  // are like four.  Up to 16 tokens no expert has more than one.
  if (chooses_itself(route)) {
    if (logits == HM_BF16) launch_choosing_up<uint16_t, PLANES>(p, route, shares, stream);
    else launch_choosing_up<float, PLANES>(p, route, shares, stream);
  } else if (p.T <= 16 || p.T * p.K <= 10 * route.r.E) {
    launch_few_up<float, 0, 1, PLANES>(p, route, shares, stream);
  } else {
    launch_few_up<float, 0, 4, PLANES>(p, route, shares, stream);
  }
  const hm_status up = hm_launch_status();
  if (up != HM_OK) return up;
  const int64_t slots = (int64_t)p.T * p.K, staged = PLANES * slots * (row8_bytes(p.F) + 8) * 2, sums = (int64_t)kDownWaves * p.T * 16 * 4;
  // by columns while the activations fit: a token's 8 experts of 7,168 x 2,048 28 us, by experts 30.5 and the sum's 4.8
  if (slots <= kWave && staged + sums <= staged_limit<PLANES, OUT>()) {
    // half the columns leave the matrix unit half empty, but a workgroup for each CU: 2,048 columns 7.8 to 8.5 us with 8, 8.7 to 9.4
    // with 16, 7,168 35 and 28
    const int columns = p.H < 4096 ? 8 : 16;
    hipLaunchKernelGGL((few_down_kernel<PLANES, OUT>), dim3((unsigned)((p.H + columns - 1) / columns)), dim3(kDownWaves * kWave),
                       (size_t)(sums + staged), stream, p, columns);
    return hm_launch_status();
  }
  // wide strips keep more loads on their way, narrow ones are more workgroups: 32 experts of 7,168 columns (3,584 wide strips) 85 and
  // 95 us, 60 of 1,030 (1,020) 28.6 and 25.2
  const bool wide = shares * ((p.H + 63) / 64) >= 2048;
  const int64_t strip = wide ? 64 : 32;
  hipLaunchKernelGGL((wide ? few_down_slots_kernel<PLANES, 4> : few_down_slots_kernel<PLANES, 2>),
                     dim3((unsigned)((p.H + strip - 1) / strip), (unsigned)shares), dim3(kUpWaves * kWave), 0, stream, p);
  const hm_status down = hm_launch_status();
  if (down != HM_OK) return down;
  hipLaunchKernelGGL((few_sum_kernel<OUT>), dim3((unsigned)((p.H + 255) / 256), (unsigned)p.T), dim3(256), 0, stream, p);
  return hm_launch_status();
}
}  // namespace hm

extern "C" size_t hm_layer_few_workspace_bytes(int32_t T, int32_t K, int32_t H, int32_t F) {
  if (T < 0 || T > hm::kMostFewTokens || K < 1 || (int64_t)T * K > hm::kMostFewSlots) return 0;
  if (H < 1 || H > hm::kMostColumns8 || F < 1 || F > hm::kMostColumns8 / 2) return 0;
  return (size_t)T * K * (3 * 2 * hm::row8_bytes(F) + 4 * (size_t)H);
}

extern "C" hm_status hm_layer_few(const void *x, int64_t ld, const void *logits, hm_dtype logits_dtype, int64_t logits_ld,
                                  const float *bias, int32_t T, const hm_router *router, const uint8_t *w13, const uint8_t *w13_scale,
                                  const uint8_t *w2, const uint8_t *w2_scale, int32_t first, int32_t experts, int32_t H, int32_t F,
                                  int32_t *topk_ids, float *topk_weights, void *out, hm_dtype out_dtype, void *workspace,
                                  size_t workspace_bytes, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!router) return HM_ERR_NULL;
  if (T < 0 || T > kMostFewTokens || router->K < 1 || (int64_t)T * router->K > kMostFewSlots) return HM_ERR_SHAPE;
  if (experts < 1 || experts > kMostSegments8 || first < 0 || (int64_t)first + experts > router->E) return HM_ERR_SHAPE;
  if (H < 1 || H > kMostColumns8 || F < 1 || F > kMostColumns8 / 2 || !dtype_known(out_dtype) || (ld < H && T > 1)) return HM_ERR_SHAPE;
  if (((uintptr_t)x & 1) || ((uintptr_t)out & (out_dtype == HM_F32 ? 3 : 1))) return HM_ERR_SHAPE;
  if (!buffers8_aligned(w13, w13_scale) || !buffers8_aligned(w2, w2_scale)) return HM_ERR_SHAPE;
  const int64_t hit = experts < (int64_t)T * router->K ? experts : (int64_t)T * router->K;
  if (hit * (row8_bytes(F) / 16) > (1 << 23)) return HM_ERR_SHAPE;
  if (T > 0 && (!x || !w13 || !w13_scale || !w2 || !w2_scale || !out)) return HM_ERR_NULL;
  if (T > 0 && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < hm_layer_few_workspace_bytes(T, router->K, H, F)))
    return HM_ERR_WORKSPACE;
  // what hm_route looks at, which makes the choice for more than a few tokens
  const RouteParams route = {logits, logits_ld, bias, T, *router, topk_ids, topk_weights};
  const hm_status fits = check_router(router);
  if (fits != HM_OK) return fits;
  if (!dtype_known(logits_dtype) || (logits_ld < router->E && T > 1)) return HM_ERR_SHAPE;
  if (T == 0) return HM_OK;
  if (!logits || !topk_ids || !topk_weights) return HM_ERR_NULL;
  if (!chooses_itself(route)) {
    const hm_status routed = hm_route(logits, logits_dtype, logits_ld, bias, T, router, topk_ids, topk_weights, hip_stream);
    if (routed != HM_OK) return routed;
  }
  const FewParams p = {(const uint16_t *)x, ld, topk_ids, topk_weights, T, router->K, first, experts, H, F,
                       ((1u << 20) + router->K - 1) / router->K, w13, w13_scale, w2, w2_scale, (uint16_t *)workspace,
                       (float *)((char *)workspace + (int64_t)T * router->K * 6 * row8_bytes(F)), out};
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (out_dtype == HM_F32) return launch_few<3, float>(p, route, logits_dtype, hit, stream);
  return launch_few<2, uint16_t>(p, route, logits_dtype, hit, stream);
}
