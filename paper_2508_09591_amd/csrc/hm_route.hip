// The router in front of the dispatch: logits -> expert ids and weights, and the way back.
#include "hm_block8.h"

namespace hm {

constexpr int kRouteThreads = 256, kRouteWaves = kRouteThreads / kWave;
constexpr int kMostExperts = 4096, kMostSlots = 64;

struct RouteParams {
  const void *logits;
  int64_t ld;
  const float *bias;
  int32_t T;
  hm_router r;
  int32_t *ids;
  float *weights;
};

__device__ __forceinline__ float logit_at(const uint16_t *x, int64_t i) { return bf16_lo(x[i]); }
__device__ __forceinline__ float logit_at(const float *x, int64_t i) { return x[i]; }
// What an expert that is never chosen has in place of its logit and its choice.
__device__ __forceinline__ float kNone() { return -__builtin_inff(); }
__device__ __forceinline__ float usable(float x) { return x == x ? fminf(x, 3.402823466e38f) : kNone(); }
__device__ __forceinline__ float logistic(float x) { return 1.0f / (1.0f + expf(-x)); }

template <typename OP>
__device__ __forceinline__ float wave_all(float v, OP op) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = op(v, __shfl_xor(v, d, kWave));
  return v;
}
__device__ __forceinline__ float wave_max(float v) { return wave_all(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_sum(float v) { return wave_all(v, [](float a, float b) { return a + b; }); }

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

// A wave takes a token; its choices stand in LDS and the largest is taken K times.
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

// A wave takes a token, a lane a slot; the row is put together in LDS.
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

// A wave takes a token and eight of its slots at a time: its gradient's row once, the eight rows beside it.
template <typename IN>
__global__ __launch_bounds__(kRouteThreads) void combine_weight_grad_kernel(WeightGradParams p) {
  const int lane = lane_id();
  const int64_t t = (int64_t)blockIdx.x * kRouteWaves + threadIdx.x / kWave;
  if (t >= p.T) return;
  const IN *gout = (const IN *)p.gout + t * p.H;
  for (int k0 = 0; k0 < p.K; k0 += 8) {
    const IN *row[8];
    bool there[8], bad = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t r = k0 + j < p.K ? p.slot_row[t * p.K + k0 + j] : -1;
      there[j] = r >= 0 && r < p.y_rows;
      bad = bad || r >= p.y_rows;
      row[j] = (const IN *)p.y + (there[j] ? r : 0) * p.H;
    }
    if (bad && lane == 0) flag(p.status, HM_ERR_CAPACITY);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int h = lane * 8; h < p.H; h += kWave * 8) {
      float g[8];
      load8(gout + h, p.H - h, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!there[j]) continue;
        float v[8];
        load8(row[j] + h, p.H - h, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[j] = fmaf(g[i], v[i], sum[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float s = wave_sum(sum[j]);
      if (lane == j && k0 + j < p.K) p.grad[t * p.K + k0 + j] = s;
    }
  }
}

static hm_status check_router(const hm_router *r) {
  if (!r) return HM_ERR_NULL;
  if (r->E < 1 || r->E > kMostExperts || r->K < 1 || r->K > kMostSlots) return HM_ERR_SHAPE;
  if (r->score != HM_SCORE_SOFTMAX && r->score != HM_SCORE_SIGMOID) return HM_ERR_SHAPE;
  if (r->groups < 1 || r->groups > r->E || r->E % r->groups || r->top_groups < 1 || r->top_groups > r->groups) return HM_ERR_SHAPE;
  if (r->group_best < 1 || r->group_best > 2 || r->group_best > r->E / r->groups) return HM_ERR_SHAPE;
  if (r->K > r->E / r->groups * r->top_groups) return HM_ERR_SHAPE;
  return HM_OK;
}
// Tokens of a workgroup whose rows of `floats` fit 64 KiB.
static int tokens_per_group(int floats) {
  int n = kRouteWaves;
  while (n > 1 && n * floats * 4 > 65536) n >>= 1;
  return n;
}

}  // namespace hm

extern "C" hm_status hm_route(const void *logits, hm_dtype dtype, int64_t ld, const float *bias, int32_t T, const hm_router *router,
                              int32_t *topk_ids, float *topk_weights, void *hip_stream) {
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
  const int floats = router->E + (router->groups > 1 ? router->groups : 0), n = tokens_per_group(floats);
  const auto kernel = dtype == HM_BF16 ? route_kernel<uint16_t> : route_kernel<float>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((T + (int64_t)n - 1) / n)), dim3((unsigned)(n * kWave)), (size_t)n * floats * 4, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}

extern "C" hm_status hm_route_backward(const void *logits, hm_dtype dtype, int64_t ld, const int32_t *topk_ids, const float *grad_weights,
                                       int32_t T, const hm_router *router, void *grad_logits, int64_t grad_ld, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  const hm_status bad = check_router(router);
  if (bad != HM_OK) return bad;
  const hm_status shape = hm_check_tk(T, router->K);
  if (shape != HM_OK) return shape;
  if (!dtype_known(dtype) || ((ld < router->E || grad_ld < router->E) && T > 1)) return HM_ERR_SHAPE;
  if (T == 0) return HM_OK;
  if (!logits || !topk_ids || !grad_weights || !grad_logits) return HM_ERR_NULL;
  const RouteBackParams p = {logits, ld, grad_ld, topk_ids, grad_weights, T, *router, grad_logits};
  const int n = tokens_per_group(router->E);
  const auto kernel = dtype == HM_BF16 ? route_backward_kernel<uint16_t> : route_backward_kernel<float>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((T + (int64_t)n - 1) / n)), dim3((unsigned)(n * kWave)), (size_t)n * router->E * 4, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}

extern "C" hm_status hm_combine_weight_grad(const void *gout, const void *y, hm_dtype dtype, int64_t y_rows, int32_t T, int32_t K, int32_t H,
                                            const hm_plan_out *plan, float *grad_weights, void *hip_stream) {
  HM_ENTRY_SCOPE;
  using namespace hm;
  if (!plan || !plan->slot_row || !plan->status) return HM_ERR_NULL;
  const hm_status shape = hm_check_tk(T, K);
  if (shape != HM_OK) return shape;
  if (!dtype_known(dtype) || H < 1 || y_rows < 0) return HM_ERR_SHAPE;
  if (T == 0) return HM_OK;
  if (!gout || !grad_weights || (!y && y_rows > 0)) return HM_ERR_NULL;
  const WeightGradParams p = {gout, y, y_rows, plan->slot_row, T, K, H, grad_weights, plan->status};
  const auto kernel = dtype == HM_BF16 ? combine_weight_grad_kernel<uint16_t> : combine_weight_grad_kernel<float>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((T + kRouteWaves - 1) / kRouteWaves)), dim3(kRouteThreads), 0, (hipStream_t)hip_stream, p);
  return hm_launch_status();
}
