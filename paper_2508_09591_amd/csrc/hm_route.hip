// The router in front of the dispatch: logits -> expert ids and weights, and the way back.
#include "hm_choice.h"

namespace hm {

constexpr int kRouteThreads = 256, kRouteWaves = kRouteThreads / kWave;

// The largest of the wave's values and the lowest index that has it.
__device__ __forceinline__ void wave_first(float &v, int &i) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float u = __shfl_xor(v, d, kWave);
    const int j = __shfl_xor(i, d, kWave);
    const bool take = u > v || (u == v && j < i);
    v = take ? u : v;
    i = take ? j : i;
  }
}

// What the choice by lists (hm_choice.h) does not take: K > 16, groups that are no power of two up to 16, a softmax with a
// bias, many experts.  A wave takes a token; its choices stand in LDS and the largest is taken K times: 65,536 tokens
// of 256 experts 178 us where the lists take 30.
template <typename IN>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(RouteParams p) {
  extern __shared__ float choices[];
  const int lane = lane_id(), wave = threadIdx.x / kWave, E = p.r.E, K = p.r.K;
  const int64_t t = (int64_t)blockIdx.x * (blockDim.x / kWave) + wave;
  if (t >= p.T) return;
  float *c = choices + wave * E;
  const IN *x = (const IN *)p.logits + t * p.ld;
  const bool softmax = p.r.score == HM_SCORE_SOFTMAX;
  float best = kNone();
  for (int e = lane; e < E; e += kWave) best = fmaxf(best, usable(logit_at(x, e)));
  best = wave_max(best);
  float sum = 0.0f;
  const bool whole = softmax && (!p.r.renormalise || p.bias);   // the softmax's own sum
  if (whole) {
    for (int e = lane; e < E; e += kWave) {
      const float v = usable(logit_at(x, e));
      sum += v == kNone() ? 0.0f : expf(v - best);
    }
    sum = wave_sum(sum);
  }
  for (int e = lane; e < E; e += kWave) {
    const float v = usable(logit_at(x, e));
    float choice = v;
    if (v != kNone() && p.bias) choice = (softmax ? expf(v - best) / sum : logistic(v)) + p.bias[e];
    c[e] = choice == choice ? choice : kNone();
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (p.r.groups > 1) {
    const int per = E / p.r.groups;
    // a lane scores groups lane, lane + 64, ...; the scores stand behind the choices of all waves
    float *g = choices + (blockDim.x / kWave) * E + wave * p.r.groups;
    for (int j = lane; j < p.r.groups; j += kWave) {
      float a = kNone(), b = kNone();
      for (int e = j * per; e < (j + 1) * per; ++e) {
        float v = c[e];
        if (v == kNone()) continue;
        if (!p.bias) v = softmax ? expf(v - best) : logistic(v);
        if (v > a) {
          b = a;
          a = v;
        } else if (v > b) {
          b = v;
        }
      }
      g[j] = p.r.group_best == 2 && b != kNone() ? a + b : a;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int j = 0; j < p.r.groups; ++j) {
      const float mine = g[j];
      int better = 0;
      for (int i = lane; i < p.r.groups; i += kWave) better += g[i] > mine || (g[i] == mine && i < j);
      better = (int)wave_sum((float)better);
      if (better >= p.r.top_groups)
        for (int e = j * per + lane; e < (j + 1) * per; e += kWave) c[e] = kNone();
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  int id = -1;   // of slot `lane`
  for (int k = 0; k < K; ++k) {
    float v = kNone();
    int i = 0x7FFFFFFF;
    for (int e = lane; e < E; e += kWave) {
      const float u = c[e];
      if (u > v) {
        v = u;
        i = e;
      }
    }
    wave_first(v, i);
    if (v == kNone()) break;
    if (lane == k) id = i;
    if (lane == (i & (kWave - 1))) c[i] = kNone();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  float score = 0.0f;
  if (id >= 0) {
    const float v = usable(logit_at(x, id));
    score = softmax ? expf(v - best) : logistic(v);
  }
  const float by = p.r.renormalise ? wave_sum(score) : softmax ? sum : 1.0f;
  if (lane < K) {
    p.ids[t * K + lane] = id;
    p.weights[t * K + lane] = by > 0.0f ? score / by * p.r.scale : 0.0f;
  }
}

template <typename IN, int L, int N>
__global__ __launch_bounds__(kRouteThreads) void route_lists_kernel(RouteParams p, int lanes_per_group, int run) {
  const int64_t t = (int64_t)blockIdx.x * (kRouteThreads / L) + threadIdx.x / L;
  choose_by_lists<IN, L, N>(p, t, lanes_per_group, run, [&](int k, int expert, float weight) {
    p.ids[t * p.r.K + k] = expert;
    p.weights[t * p.r.K + k] = weight;
  });
}

struct RouteBackParams {
  const void *logits;
  int64_t ld, grad_ld;
  const int32_t *ids;
  const float *grad_weights;
  int32_t T;
  hm_router r;
  void *grad_logits;
};

__device__ __forceinline__ void put(uint16_t *x, float v) { *x = (uint16_t)f32_to_bf16(v); }
__device__ __forceinline__ void put(float *x, float v) { *x = v; }

// A wave takes a token, a lane a slot; the row is put together in LDS.  8,192 x 256 fp32 6 us, the stores of 8 MB and a
// launch.
template <typename IN>
__global__ __launch_bounds__(kRouteThreads) void route_backward_kernel(RouteBackParams p) {
  extern __shared__ float rows[];
  const int lane = lane_id(), wave = threadIdx.x / kWave, E = p.r.E, K = p.r.K;
  const int64_t t = (int64_t)blockIdx.x * (blockDim.x / kWave) + wave;
  if (t >= p.T) return;
  float *row = rows + wave * E;
  const IN *x = (const IN *)p.logits + t * p.ld;
  const bool softmax = p.r.score == HM_SCORE_SOFTMAX, dense = softmax && !p.r.renormalise;
  int id = lane < K ? p.ids[t * K + lane] : -1;
  if ((unsigned)id >= (unsigned)E) id = -1;
  float v = id >= 0 ? usable(logit_at(x, id)) : kNone();
  if (v == kNone()) id = -1;
  const float g = id >= 0 ? p.grad_weights[t * K + lane] : 0.0f;
  float best = v, sum = 1.0f;
  if (dense)
    for (int e = lane; e < E; e += kWave) best = fmaxf(best, usable(logit_at(x, e)));
  best = wave_max(best);
  if (dense) {
    sum = 0.0f;
    for (int e = lane; e < E; e += kWave) {
      const float u = usable(logit_at(x, e)), s = u == kNone() ? 0.0f : expf(u - best);
      row[e] = s;
      sum += s;
    }
    sum = wave_sum(sum);
    if (sum == 0.0f) sum = 1.0f;   // nothing can be chosen
  } else {
    for (int e = lane; e < E; e += kWave) row[e] = 0.0f;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // score, and its derivative by the logit over the score (1 - s of a logistic without cancellation)
  float s = 0.0f, slope = 1.0f;
  if (id >= 0) {
    if (softmax) {
      s = expf(v - best) / sum;
    } else {
      const float small = expf(-fabsf(v)), half = 1.0f / (1.0f + small);
      s = v >= 0.0f ? half : small * half;
      slope = v >= 0.0f ? small * half : half;
    }
  }
  float d;
  if (p.r.renormalise) {
    const float total = wave_sum(s), u = total > 0.0f ? s / total : 0.0f;
    d = p.r.scale * u * (g - wave_sum(g * u)) * slope;
  } else if (softmax) {
    const float mean = wave_sum(g * s);
    for (int e = lane; e < E; e += kWave) row[e] = -p.r.scale * (row[e] / sum) * mean;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    d = p.r.scale * s * (g - mean);
  } else {
    d = p.r.scale * g * s * slope;
  }
  if (id >= 0) row[id] = d;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  IN *out = (IN *)p.grad_logits + t * p.grad_ld;
  for (int e = lane; e < E; e += kWave) put(out + e, row[e]);
}

struct WeightGradParams {
  const void *gout, *y;
  int64_t y_rows;
  const int32_t *slot_row;
  int32_t T, K, H;
  float *grad;
  int32_t *status;
};

// A wave takes a part of a token's row and SLOTS of its slots at a time: its gradient's row once, the slots' rows
// beside it, all loads of 512 elements on their way together.  Where a row is split, the parts' sums meet in LDS.  What
// bounds it is memory, (K + 1) rows a token: 8,192 tokens, K = 8, 7,168 bf16 180 us, 5.9 TB/s; few tokens wait for one
// trip after the other (1,237 tokens, K = 6, 1,030 fp32 9 us).
template <typename IN, int PARTS, int SLOTS>
__global__ __launch_bounds__(kRouteThreads) void combine_weight_grad_kernel(WeightGradParams p) {
  __shared__ float parts[kRouteWaves][SLOTS];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), part = wave % PARTS;
  const int64_t t = (int64_t)blockIdx.x * (kRouteWaves / PARTS) + wave / PARTS;
  // the same for the waves of a token; with several parts nobody leaves before the barriers
  const bool there_t = t < p.T;
  if (PARTS == 1 && !there_t) return;
  const int64_t token = there_t ? t : 0;
  const IN *gout = (const IN *)p.gout + token * p.H;
  constexpr int kStep = kWave * 8;
  for (int k0 = 0; k0 < p.K; k0 += SLOTS) {
    const IN *row[SLOTS];
    bool there[SLOTS], bad = false;
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      const int64_t r = k0 + j < p.K ? p.slot_row[token * p.K + k0 + j] : -1;
      there[j] = r >= 0 && r < p.y_rows;
      bad = bad || r >= p.y_rows;
      row[j] = there[j] ? (const IN *)p.y + r * p.H : gout;   // something to read in place of a row that is not there
    }
    if (bad && lane == 0 && there_t) flag(p.status, HM_ERR_CAPACITY);
    float sum[SLOTS];
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) sum[j] = 0.0f;
    int h = part * kStep + lane * 8;
    for (int first = part * kStep; first + kStep <= p.H; first += PARTS * kStep, h += PARTS * kStep) {
      Eight<IN> g(gout + h), v[SLOTS];
#pragma unroll
      for (int j = 0; j < SLOTS; ++j)
        if (k0 + j < p.K) v[j] = Eight<IN>(row[j] + h);
#pragma unroll
      for (int j = 0; j < SLOTS; ++j)
        if (k0 + j < p.K) sum[j] = g.times(v[j], sum[j]);
    }
    // The row's last, shorter step is the part's whose turn it is: vectors that would pass the end lie before it, and
    // what the vector before them has had counts as zero.
    const int begin = h - lane * 8;
    if (begin < p.H && begin + kStep > p.H) {
      if (p.H >= 8) {
        if (h < p.H) {
          const int at = min(h, p.H - 8), had = h - at;
          float g[8];
          load_floats<8>(gout + at, g);
          Eight<IN> v[SLOTS];
#pragma unroll
          for (int j = 0; j < SLOTS; ++j)
            if (k0 + j < p.K) v[j] = Eight<IN>(row[j] + at);
#pragma unroll
          for (int j = 0; j < SLOTS; ++j)
            if (k0 + j < p.K) {
#pragma unroll
              for (int i = 0; i < 8; ++i) sum[j] = i < had ? sum[j] : fmaf(g[i], v[j].at(i), sum[j]);
            }
        }
      } else if (lane < p.H) {
        const float g = load_float(gout + lane);
#pragma unroll
        for (int j = 0; j < SLOTS; ++j)
          if (k0 + j < p.K) sum[j] = fmaf(g, load_float(row[j] + lane), sum[j]);
      }
    }
    float mine = 0.0f;
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      const float s = wave_sum(sum[j]);
      mine = lane == j && there[j] ? s : mine;
    }
    if (PARTS > 1) {
      if (lane < SLOTS) parts[wave][lane] = mine;
      __syncthreads();
      mine = 0.0f;
      if (lane < SLOTS)
        for (int w = 0; w < PARTS; ++w) mine += parts[wave - part + w][lane];
      __syncthreads();
    }
    if (part == 0 && there_t && lane < SLOTS && k0 + lane < p.K) p.grad[token * p.K + k0 + lane] = mine;
  }
}

template <typename IN, int L>
static void launch_lists(const RouteParams &p, hipStream_t stream) {
  const int K = p.r.K, lanes_per_group = L / p.r.groups;
  const int run = (p.r.E / p.r.groups + lanes_per_group - 1) / lanes_per_group;
  const auto kernel = K <= 2   ? route_lists_kernel<IN, L, 2>
                      : K <= 4 ? route_lists_kernel<IN, L, 4>
                      : K <= 8 ? route_lists_kernel<IN, L, 8>
                               : route_lists_kernel<IN, L, 16>;
  const int64_t per_block = kRouteThreads / L;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((p.T + per_block - 1) / per_block)), dim3(kRouteThreads), 0, stream, p,
                     lanes_per_group, run);
}
// Whether a launch has threads for T tokens of so many: it has less than 2^32, in whole workgroups.
static bool threads_suffice(int64_t T, int each) { return T * each <= (1LL << 32) - kRouteThreads; }
// Tokens of a workgroup whose rows of `floats` fit 64 KiB.
static int tokens_per_group(int floats) {
  int n = kRouteWaves;
  while (n > 1 && n * floats * 4 > 65536) n >>= 1;
  return n;
}

}  // namespace hm

extern "C" hm_status hm_route(const void *logits, hm_dtype dtype, int64_t ld, const float *bias, int32_t T,
                              const hm_router *router, int32_t *topk_ids, float *topk_weights, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  const hm_status bad = check_router(router);
  if (bad != HM_OK) return bad;
  const hm_status shape = hm_check_tk(T, router->K);
  if (shape != HM_OK) return shape;
  if (!dtype_known(dtype) || (ld < router->E && T > 1)) return HM_ERR_SHAPE;
  if (T == 0) return HM_OK;
  if (!logits || !topk_ids || !topk_weights) return HM_ERR_NULL;
  const RouteParams p = {logits, ld, bias, T, *router, topk_ids, topk_weights};
  const int lanes = list_lanes(p.r, bias != nullptr, T);
  if (!threads_suffice(T, lanes ? lanes : kWave)) return HM_ERR_SHAPE;
  if (lanes) {
    const hipStream_t stream = (hipStream_t)hip_stream;
    if (dtype == HM_BF16) lanes == 8 ? launch_lists<uint16_t, 8>(p, stream) : launch_lists<uint16_t, 16>(p, stream);
    else lanes == 8 ? launch_lists<float, 8>(p, stream) : launch_lists<float, 16>(p, stream);
    return hm_launch_status();
  }
  const int floats = router->E + (router->groups > 1 ? router->groups : 0), n = tokens_per_group(floats);
  const auto kernel = dtype == HM_BF16 ? route_kernel<uint16_t> : route_kernel<float>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((T + (int64_t)n - 1) / n)), dim3((unsigned)(n * kWave)),
                     (size_t)n * floats * 4, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}

extern "C" hm_status hm_route_backward(const void *logits, hm_dtype dtype, int64_t ld, const int32_t *topk_ids,
                                       const float *grad_weights, int32_t T, const hm_router *router,
                                       void *grad_logits, int64_t grad_ld, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  const hm_status bad = check_router(router);
  if (bad != HM_OK) return bad;
  const hm_status shape = hm_check_tk(T, router->K);
  if (shape != HM_OK) return shape;
  if (!dtype_known(dtype) || ((ld < router->E || grad_ld < router->E) && T > 1)) return HM_ERR_SHAPE;
  if (!threads_suffice(T, kWave)) return HM_ERR_SHAPE;
  if (T == 0) return HM_OK;
  if (!logits || !topk_ids || !grad_weights || !grad_logits) return HM_ERR_NULL;
  const RouteBackParams p = {logits, ld, grad_ld, topk_ids, grad_weights, T, *router, grad_logits};
  const int n = tokens_per_group(router->E);
  const auto kernel = dtype == HM_BF16 ? route_backward_kernel<uint16_t> : route_backward_kernel<float>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((T + (int64_t)n - 1) / n)), dim3((unsigned)(n * kWave)),
                     (size_t)n * router->E * 4, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}

extern "C" hm_status hm_combine_weight_grad(const void *gout, const void *y, hm_dtype dtype, int64_t y_rows, int32_t T,
                                            int32_t K, int32_t H, const hm_plan_out *plan, float *grad_weights,
                                            void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!plan || !plan->slot_row || !plan->status) return HM_ERR_NULL;
  const hm_status shape = hm_check_tk(T, K);
  if (shape != HM_OK) return shape;
  if (!dtype_known(dtype) || H < 1 || y_rows < 0 || !threads_suffice(T, kWave)) return HM_ERR_SHAPE;
  if (T == 0) return HM_OK;
  if (!gout || !grad_weights || (!y && y_rows > 0)) return HM_ERR_NULL;
  const WeightGradParams p = {gout, y, y_rows, plan->slot_row, T, K, H, grad_weights, plan->status};
  // A token's row in four parts where there are few tokens.  Eight slots at a time read the gradient's row once for
  // most K; fp32 rows take the registers of four waves a SIMD for that, so they go four at a time (8,192 x 2,048, K =
  // 8: 125 us and 137) but where rows are long (8,192 x 7,168: 395 and 356).
  const int parts = T <= 4096 && H > 512 ? kRouteWaves : 1, tokens = kRouteWaves / parts;
  const auto whole = dtype == HM_BF16 ? combine_weight_grad_kernel<uint16_t, 1, 8>
                     : H >= 4096      ? combine_weight_grad_kernel<float, 1, 8>
                                      : combine_weight_grad_kernel<float, 1, 4>;
  const auto split = dtype == HM_BF16 ? combine_weight_grad_kernel<uint16_t, kRouteWaves, 8>
                                      : combine_weight_grad_kernel<float, kRouteWaves, 4>;
  hipLaunchKernelGGL((parts == 1 ? whole : split), dim3((unsigned)((T + tokens - 1) / tokens)), dim3(kRouteThreads), 0,
                     (hipStream_t)hip_stream, p);
  return hm_launch_status();
}
