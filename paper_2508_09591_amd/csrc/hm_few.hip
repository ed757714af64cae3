// A whole layer for a few tokens: choice, both products, activation and weighted sum, without a plan and without rows in 8 bits.
//     out[t] = sum_k w[t,k] w2_e (silu(gate) up),   [gate; up] = w13_e x[t],   e = ids[t,k] - first
// The weights of the experts hit are all there is to read, once: 16 of their rows a workgroup, straight from memory into the
// operands of products of 16 x 16 x 32 in 16 bits, as for the products of few rows.  Values in 8 bits times their block's power of
// two are exact in bf16, x is bf16; activations go between the two products as sums of two or three bf16 numbers, so that what
// they lose is far below the output's rounding (2^-17 of each, 2^-25 for fp32 outputs).
#include "hm_block8.h"

namespace hm {

constexpr int kMostFewTokens = 64, kMostFewSlots = 1024;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct FewParams {
  const uint16_t *x;
  int64_t ld;
  const int32_t *ids;      // [T,K]
  const float *weights;
  int32_t T, K, first, experts, H, F;
  const uint8_t *w13, *s13, *w2, *s2;
  uint16_t *a;             // [planes, T K, up(F,128)]
  void *out;
};

// The experts that are here and that a slot has chosen, as bits in LDS; called by all threads, before a barrier of theirs is
// left.
constexpr int kHitWords = kMostSegments8 / 32;
__device__ __forceinline__ int local_expert(const FewParams &p, int slot) {   // -1: not here
  const int e = slot < p.T * p.K ? p.ids[slot] - p.first : -1;
  return (unsigned)e < (unsigned)p.experts ? e : -1;
}
__device__ __forceinline__ void find_hits(const FewParams &p, uint32_t *hits, int16_t *expert_of) {
  for (int i = threadIdx.x; i < kHitWords; i += blockDim.x) hits[i] = 0;
  __syncthreads();
  for (int s = threadIdx.x; s < p.T * p.K; s += blockDim.x) {
    const int e = local_expert(p, s);
    expert_of[s] = (int16_t)e;
    if (e >= 0) atomicOr(&hits[e >> 5], 1u << (e & 31));
  }
  __syncthreads();
}
// The n-th of them in ascending order, -1 if there are fewer; and how many there are.  By whole waves.
__device__ __forceinline__ int nth_hit(const uint32_t *hits, int n, int &count) {
  const int lane = lane_id();
  const uint32_t mine = lane < kHitWords ? hits[lane] : 0u;
  const int upto = lane_scan(__popc(mine));
  count = read_lane(upto, kWave - 1);
  if (n >= count) return -1;
  const int word = __builtin_ctzll(__ballot(upto > n));
  uint32_t bits = (uint32_t)read_lane((int)mine, word);
  for (int skip = n - (read_lane(upto, word) - __popc(bits)); skip > 0; --skip) bits &= bits - 1;
  return word * 32 + __builtin_ctz(bits);
}
// The slots of an expert, ascending, into `list`; at most one of a token's, so at most kMostFewTokens.  By one wave.
__device__ __forceinline__ int slots_of(const int16_t *expert_of, int slots, int e, int *list) {
  const int lane = lane_id();
  int n = 0;
  for (int s0 = 0; s0 < slots; s0 += kWave) {
    const bool mine = s0 + lane < slots && expert_of[s0 + lane] == e;
    const uint64_t all = __ballot(mine);
    const int at = n + __popcll(all & ((1ull << lane) - 1));
    if (mine && at < kMostFewTokens) list[at] = s0 + lane;
    n += __popcll(all);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return min(n, kMostFewTokens);
}

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
__device__ __forceinline__ Wide zero_wide() {
  Wide w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w.v[i] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
  return w;
}

// ---- the first product and the activation --------------------------------------------------------------
// A workgroup takes an expert and 16 columns of its activation: as many rows of the gate's weights and of the up's.  Its four
// waves take every fourth step of 128 columns of x and add up in LDS.  A lane has row l % 16 of the weights and of the slots,
// bytes 32 (l / 16) to 32 (l / 16) + 31 of a step.
constexpr int kUpWaves = 4;
template <int GROUPS, int PLANES>
__global__ __launch_bounds__(kUpWaves * kWave) void few_up_kernel(FewParams p) {
  __shared__ uint32_t hits[kHitWords];
  __shared__ int16_t expert_of[kMostFewSlots];
  __shared__ int lists[kUpWaves][kMostFewTokens];
  __shared__ f32x4 sums[kUpWaves][2][kWave];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int width_a = (int)row8_bytes(p.F), strips = width_a / 16, slots = p.T * p.K;
  find_hits(p, hits, expert_of);
  int count;
  const int e = nth_hit(hits, (int)(blockIdx.x / (uint32_t)strips), count);
  if (e < 0) return;
  const int n = slots_of(expert_of, slots, e, lists[wave]);
  const int *list = lists[wave];
  const int f0 = (int)(blockIdx.x % (uint32_t)strips) * 16, row = lane & 15, part = (lane >> 4) * 32;
  const int steps = (int)blocks8(p.H);
  const int64_t pitch = row8_bytes(p.H), scale_pitch = scale8_bytes(p.H);
  const int gate = min(f0 + row, p.F - 1), up = p.F + gate;
  const uint8_t *w = p.w13 + (int64_t)e * 2 * p.F * pitch + part, *s = p.s13 + (int64_t)e * blocks8(2 * (int64_t)p.F) * scale_pitch;
  const uint8_t *from_gate = w + gate * pitch, *from_up = w + up * pitch;
  const uint8_t *scale_gate = s + (gate / 128) * scale_pitch, *scale_up = s + (up / 128) * scale_pitch;
  const uint16_t *x[GROUPS];
  bool there[GROUPS];
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    there[g] = g * 16 + row < n;
    x[g] = p.x + (int64_t)(list[min(g * 16 + row, n - 1)] / p.K) * p.ld + part;
  }
  f32x4 acc[GROUPS][2];
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) acc[g][0] = acc[g][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  struct Step {
    i32x8 gate, up;
    uint32_t scale_gate, scale_up;
    Wide x[GROUPS];
  };
  auto load = [&](Step &t, int k) {
    t.gate = load32(from_gate + (int64_t)k * 128);
    t.up = load32(from_up + (int64_t)k * 128);
    t.scale_gate = scale_gate[k];
    t.scale_up = scale_up[k];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      t.x[g] = zero_wide();
      if (g * 16 >= n) continue;
      if (k * 128 + 128 <= p.H) {
        if (there[g]) t.x[g] = load_wide(x[g] + k * 128);
      } else if (there[g]) {   // the row's end: zeros behind it
#pragma unroll
        for (int i = 0; i < 32; ++i)
          t.x[g].v[i / 8][i % 8] = k * 128 + part + i < p.H ? __builtin_bit_cast(__bf16, x[g][k * 128 + i]) : (__bf16)0.0f;
      }
    }
  };
  auto multiply = [&](const Step &t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x8 wg = widen8(t.gate[2 * i], t.gate[2 * i + 1], t.scale_gate), wu = widen8(t.up[2 * i], t.up[2 * i + 1], t.scale_up);
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        if (g * 16 >= n) continue;
        acc[g][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wg, t.x[g].v[i], acc[g][0], 0, 0, 0);
        acc[g][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wu, t.x[g].v[i], acc[g][1], 0, 0, 0);
      }
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
  const int r = threadIdx.x >> 4, c = threadIdx.x & 15, f = f0 + c;
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    if (g * 16 >= n) break;   // the same for the workgroup
    if (g > 0) __syncthreads();
    sums[wave][0][lane] = acc[g][0];
    sums[wave][1][lane] = acc[g][1];
    __syncthreads();
    float v[2] = {0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < kUpWaves; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) v[h] += ((const float *)&sums[u][h][(c >> 2) * 16 + r])[c & 3];
    if (g * 16 + r < n) {
      float rest = f < p.F ? v[0] / (1.0f + expf(-v[0])) * v[1] : 0.0f;   // zeros up to a whole block
      const int64_t at = (int64_t)list[g * 16 + r] * width_a + f;
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
// A workgroup takes 16 columns of the output.  Its waves share the steps of all experts hit evenly; behind an expert's steps a
// wave adds what its slots get, times their weights, to its own sums of the tokens in LDS, which are added up in the end.
template <int GROUPS, int PLANES, typename OUT>
__global__ __launch_bounds__(512) void few_down_kernel(FewParams p, int columns) {
  extern __shared__ float sums[];   // [waves][T][16]
  __shared__ uint32_t hits[kHitWords];
  __shared__ int16_t expert_of[kMostFewSlots];
  __shared__ int lists[8][kMostFewTokens];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), waves = blockDim.x / kWave;
  const int width_a = (int)row8_bytes(p.F), slots = p.T * p.K, row = lane & 15, part = (lane >> 4) * 32, h0 = (int)blockIdx.x * columns;
  for (int i = threadIdx.x; i < waves * p.T * 16; i += blockDim.x) sums[i] = 0.0f;
  find_hits(p, hits, expert_of);
  int count;
  nth_hit(hits, 0, count);
  const int steps = (int)blocks8(p.F), h = min(h0 + min(row, columns - 1), p.H - 1);
  const int64_t pitch = row8_bytes(p.F), scale_pitch = scale8_bytes(p.F), all = (int64_t)count * steps;
  int64_t at = all * wave / waves;
  const int64_t end = all * (wave + 1) / waves;
  int *list = lists[wave];
  float *mine = sums + wave * p.T * 16;
  struct Step {
    i32x8 w;
    uint32_t scale;
    Wide a[GROUPS][PLANES];
  };
  while (at < end) {
    const int j = (int)(at / steps), from = (int)(at - (int64_t)j * steps), to = (int)min((int64_t)steps, from + end - at);
    int unused;
    const int e = nth_hit(hits, j, unused);
    const int n = slots_of(expert_of, slots, e, list);
    const uint8_t *w = p.w2 + ((int64_t)e * p.H + h) * pitch + part;
    const uint8_t *scale = p.s2 + ((int64_t)e * blocks8(p.H) + h / 128) * scale_pitch;
    int slot[GROUPS];
    f32x4 acc[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      slot[g] = g * 16 + row < n ? list[g * 16 + row] : -1;
      acc[g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    auto load = [&](Step &t, int k) {
      t.w = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
      if (row < columns) t.w = load32(w + (int64_t)k * 128);
      t.scale = scale[k];
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int plane = 0; plane < PLANES; ++plane) {
          t.a[g][plane] = zero_wide();
          if (slot[g] >= 0) t.a[g][plane] = load_wide(p.a + ((int64_t)plane * slots + slot[g]) * width_a + k * 128 + part);
        }
    };
    auto multiply = [&](const Step &t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x8 v = widen8(t.w[2 * i], t.w[2 * i + 1], t.scale);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          if (g * 16 >= n) continue;
#pragma unroll
          for (int plane = 0; plane < PLANES; ++plane)
            acc[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, t.a[g][plane].v[i], acc[g], 0, 0, 0);
        }
      }
    };
    Step a, b;
    int k = from;
    load(a, k);
    for (; k < to; k += 2) {
      if (k + 1 < to) load(b, k + 1);
      multiply(a);
      if (k + 1 < to) {
        if (k + 2 < to) load(a, k + 2);
        multiply(b);
      }
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
      if (slot[g] >= 0) {   // lane: slot l % 16, columns 4 (l / 16) to 4 (l / 16) + 3; a token has one slot of an expert
        const float by = p.weights[slot[g]];
        float *to_token = mine + (slot[g] / p.K) * 16 + (lane >> 4) * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) to_token[i] = fmaf(by, acc[g][i], to_token[i]);
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    at += to - from;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.T * 16; i += blockDim.x) {
    const int t = i >> 4, c = i & 15;
    if (c >= columns || h0 + c >= p.H) continue;
    float sum = 0.0f;
    for (int u = 0; u < waves; ++u) sum += sums[(u * p.T + t) * 16 + c];
    store_float((OUT *)p.out + (int64_t)t * p.H + h0 + c, sum);
  }
}

static int few_planes(hm_dtype out) { return out == HM_F32 ? 3 : 2; }

template <int GROUPS, int PLANES, typename OUT>
static hm_status launch_few(const FewParams &p, int64_t experts, hipStream_t stream) {
  const int64_t strips = row8_bytes(p.F) / 16;
  hipLaunchKernelGGL((few_up_kernel<GROUPS, PLANES>), dim3((unsigned)(experts * strips)), dim3(kUpWaves * kWave), 0, stream, p);
  const hm_status up = hm_launch_status();
  if (up != HM_OK) return up;
  const int columns = 16, waves = 8;
  hipLaunchKernelGGL((few_down_kernel<GROUPS, PLANES, OUT>), dim3((unsigned)((p.H + columns - 1) / columns)), dim3(waves * kWave),
                     (size_t)waves * p.T * 16 * 4, stream, p, columns);
  return hm_launch_status();
}
template <int PLANES, typename OUT>
static hm_status launch_few_groups(const FewParams &p, int64_t experts, hipStream_t stream) {
  if (p.T <= 16) return launch_few<1, PLANES, OUT>(p, experts, stream);
  if (p.T <= 32) return launch_few<2, PLANES, OUT>(p, experts, stream);
  return launch_few<4, PLANES, OUT>(p, experts, stream);
}

}  // namespace hm

extern "C" size_t hm_layer_few_workspace_bytes(int32_t T, int32_t K, int32_t F) {
  if (T < 0 || T > hm::kMostFewTokens || K < 1 || (int64_t)T * K > hm::kMostFewSlots || F < 1 || F > hm::kMostColumns8 / 2) return 0;
  return (size_t)3 * T * K * hm::row8_bytes(F) * 2;
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
  if (T > 0 && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < hm_layer_few_workspace_bytes(T, router->K, F)))
    return HM_ERR_WORKSPACE;
  const hm_status routed = hm_route(logits, logits_dtype, logits_ld, bias, T, router, topk_ids, topk_weights, hip_stream);
  if (routed != HM_OK || T == 0) return routed;
  const FewParams p = {(const uint16_t *)x, ld, topk_ids, topk_weights, T, router->K, first, experts, H, F, w13, w13_scale, w2, w2_scale,
                       (uint16_t *)workspace, out};
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (out_dtype == HM_F32) return launch_few_groups<3, float>(p, hit, stream);
  return launch_few_groups<2, uint16_t>(p, hit, stream);
}
