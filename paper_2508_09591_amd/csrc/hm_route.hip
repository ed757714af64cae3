// The router in front of the dispatch: logits -> expert ids and weights, and the way back.
#include <type_traits>

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
// 1 / (1 + exp(-x)), the quotient rounded as a division rounds it: one Newton step from a reciprocal good to a unit in
// the last place (Markstein), compared with the division for every y from 1 to 2^126; beyond scores are 0.  The
// division takes eight instructions more for each of a token's experts: 65,536 x 256 with a bias 43 -> 31 us.
__device__ __forceinline__ float reciprocal(float y) {   // of y >= 1
  const float r = __builtin_amdgcn_rcpf(y);
  const float better = __builtin_fmaf(__builtin_fmaf(-y, r, 1.0f), r, r);
  return y < 8.50705917e37f ? better : 0.0f;
}
__device__ __forceinline__ float logistic(float x) { return reciprocal(1.0f + expf(-x)); }

// Over all lanes, the result in each: within rows of sixteen by rotations, then the four rows.
template <typename OP>
__device__ __forceinline__ float wave_all(float v, OP op) {
  auto turned = [](float x, auto control) {
    const int from = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), control(), 0xF, 0xF, true);
    return __builtin_bit_cast(float, from);
  };
  v = op(v, turned(v, std::integral_constant<int, 0x128>()));
  v = op(v, turned(v, std::integral_constant<int, 0x124>()));
  v = op(v, turned(v, std::integral_constant<int, 0x122>()));
  v = op(v, turned(v, std::integral_constant<int, 0x121>()));
  return op(op(read_lane(v, 0), read_lane(v, 16)), op(read_lane(v, 32), read_lane(v, 48)));
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

// What the choice by lists (below) does not take: K > 16, groups that are no power of two up to 16, a softmax with a
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

// ---- choice by sorted lists ----------------------------------------------------------------------------
// A choice and its expert as one number of 64 bits that orders as the definition does: the fp32 choice is the high word
// of a double, whose order is that of the floats (a float's bits with anything behind them are a finite double, -inf's
// and +inf's too), and the low word puts the lower of two equal experts first.  The largest and the smaller of two are
// one instruction each.
__device__ __forceinline__ double key_of(int32_t high, int e) {
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)high << 32 | (uint32_t)(~e ^ (high >> 31)));
}
constexpr int32_t kNoneBits = (int32_t)0xFF800000u;   // -inf
// Of a logit: NaN and -inf are none, +inf the largest number, -0 is 0.
__device__ __forceinline__ double key_of_logit(float x, int e) {
  const int32_t high = min(__builtin_bit_cast(int32_t, x + 0.0f), 0x7F7FFFFF);
  return key_of(x > kNone() ? high : kNoneBits, e);
}
// Of a logistic score and a bias: none where the logit is, and where the sum is none.  The sum is never -0.
__device__ __forceinline__ double key_of_sum(float x, float bias, int e) {
  const float c = logistic(x) + bias;
  // two selects: with `and` the compiler branches
  const int32_t high = c > kNone() ? __builtin_bit_cast(int32_t, c) : kNoneBits;
  return key_of(x > kNone() ? high : kNoneBits, e);
}
__device__ __forceinline__ float choice_of(double key) {
  return __builtin_bit_cast(float, (uint32_t)(__builtin_bit_cast(uint64_t, key) >> 32));
}
__device__ __forceinline__ int expert_of(double key) {
  const uint64_t k = __builtin_bit_cast(uint64_t, key);
  return (int64_t)k < 0 ? (int)(uint32_t)k : ~(int)(uint32_t)k;
}
// -inf
__device__ __forceinline__ double none_key() { return __builtin_bit_cast(double, (uint64_t)0xFF800000u << 32); }
// as it is, without the compiler's care for signalling NaN
__device__ __forceinline__ double larger(double a, double b) {
  double r;
  __asm__("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ double smaller(double a, double b) {
  double r;
  __asm__("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ void order(double &a, double &b) {
  const double high = larger(a, b);
  b = smaller(a, b);
  a = high;
}
// N keys, descending; N a power of two.  Merge exchange (Batcher), then a bitonic merge of what rises and falls.
template <int N>
__device__ __forceinline__ void sort(double (&k)[N]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int q = p; q >= 1; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < N; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < N && (i + j) / (2 * p) == (i + j + q) / (2 * p)) order(k[i + j], k[i + j + q]);
}
// The N largest of two descending lists, descending, in `k`.
template <int N>
__device__ __forceinline__ void merge(double (&k)[N], const double (&other)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) k[i] = larger(k[i], other[N - 1 - i]);
#pragma unroll
  for (int d = N / 2; d >= 1; d /= 2)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!(i & d)) order(k[i], k[i + d]);
}
// From a lane of the other half of 2 D lanes, D = 1, 2, 4, 8, where all lanes of a half hold the same.
template <int D>
__device__ __forceinline__ int other_half(int v) {
  // quads 1 0 3 2 and 2 3 0 1; mirrors of eight and sixteen
  constexpr int kControl = D == 1 ? 0xB1 : D == 2 ? 0x4E : D == 4 ? 0x141 : 0x140;
  return __builtin_amdgcn_update_dpp(0, v, kControl, 0xF, 0xF, true);
}
template <int D>
__device__ __forceinline__ float other_half(float v) {
  return __builtin_bit_cast(float, other_half<D>(__builtin_bit_cast(int, v)));
}
template <int D>
__device__ __forceinline__ double other_half(double v) {
  const uint64_t k = __builtin_bit_cast(uint64_t, v);
  const uint32_t high = (uint32_t)other_half<D>((int)(k >> 32)), low = (uint32_t)other_half<D>((int)k);
  return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
// op(v, what the other half has) for halves of FROM up to half of UPTO lanes.
template <int FROM, int UPTO, typename OP>
__device__ __forceinline__ void over_halves(OP op) {
  if constexpr (FROM < UPTO) {
    op(std::integral_constant<int, FROM>());
    over_halves<2 * FROM, UPTO>(op);
  }
}

// N consecutive elements, none's from the n-th on.
template <int N, typename IN>
__device__ __forceinline__ void load_logits(const IN *p, int n, float (&v)[N]) {
  if (n >= N) {
    IN raw[N];
    __builtin_memcpy(raw, p, sizeof(raw));
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = logit_at(raw, i);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? logit_at(p, i) : kNone();
  }
}

// L lanes take a token, each a run of its experts, of which it keeps the N >= K largest; the lists of the lanes are
// then merged pairwise.  With groups the L lanes are shared among them, so that a lane's run lies in one group, and
// the two largest of its list give the group's score: lists of groups that are not taken are emptied before the merges.
// What bounds it are vector instructions: about 27 an expert for a logistic score, 4 for its key and 9 for sorting (N =
// 8), against 4 bytes read.  us: 65,536 tokens, 256 experts, logistic with bias and groups 30 (2.4 TB/s), softmax 24,
// bf16 18; one token 5.3. 8 lanes a token from 16,384 tokens on: 65,536 x 64 8.4 and, with 16 lanes, 14.7; 8,192 x 256
// 8.3 and 6.9.
template <typename IN, int L, int N>
__global__ __launch_bounds__(kRouteThreads) void route_lists_kernel(RouteParams p, int lanes_per_group, int run) {
  const int sub = (int)threadIdx.x & (L - 1);
  const int64_t t = (int64_t)blockIdx.x * (kRouteThreads / L) + threadIdx.x / L;
  const bool there = t < p.T;
  const int E = p.r.E, K = p.r.K, per = E / p.r.groups, group = sub / lanes_per_group;
  const IN *x = (const IN *)p.logits + (there ? t : p.T - 1) * p.ld;
  const bool softmax = p.r.score == HM_SCORE_SOFTMAX;   // then there is no bias
  const int e = group * per + (sub - group * lanes_per_group) * run;
  const int end = min(e + run, (group + 1) * per);
  double list[N];
#pragma unroll
  for (int i = 0; i < N; ++i) list[i] = none_key();
  float v[N], b[N];
  load_logits<N>(x + e, end - e, v);
  if (p.bias) load_logits<N>(p.bias + e, end - e, b);
  for (int first = e; first < end; first += N) {
    float next[N], next_b[N];   // on their way while this batch is sorted
    load_logits<N>(x + first + N, end - first - N, next);
    if (p.bias) load_logits<N>(p.bias + first + N, end - first - N, next_b);
    double batch[N];
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < N; ++i) batch[i] = key_of_sum(v[i], b[i], first + i);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) batch[i] = key_of_logit(v[i], first + i);
    }
    sort(batch);
    merge(list, batch);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = next[i];
      b[i] = next_b[i];
    }
  }
  float best = choice_of(list[0]);   // the softmax's largest logit: of all experts
  if (softmax) over_halves<1, L>([&](auto d) { best = fmaxf(best, other_half<d()>(best)); });
  if (p.r.groups > 1) {
    const bool pair = p.r.group_best == 2;
    auto score_of = [&](double key) {
      const float c = choice_of(key);
      return c == kNone() || p.bias ? c : softmax ? expf(c - best) : logistic(c);
    };
    float a = score_of(list[0]), b = pair ? score_of(list[1]) : kNone();
    over_halves<1, L>([&](auto d) {
      if (d() < lanes_per_group) {
        const float c = other_half<d()>(a), f = other_half<d()>(b);
        b = fmaxf(fminf(a, c), fmaxf(b, f));
        a = fmaxf(a, c);
      }
    });
    const float mine = b != kNone() ? a + b : a;
    int better = 0;
    for (int g = 1; g < p.r.groups; ++g) {
      const int other_group = (group + g) & (p.r.groups - 1);
      const float c = __shfl(pair ? mine : a, (lane_id() & ~(L - 1)) + other_group * lanes_per_group, kWave);
      const float m = pair ? mine : a;
      better += c > m || (c == m && other_group < group);
    }
    if (better >= p.r.top_groups) {
#pragma unroll
      for (int i = 0; i < N; ++i) list[i] = none_key();
    }
  }
  over_halves<1, L>([&](auto d) {
    double other[N];
#pragma unroll
    for (int i = 0; i < N; ++i) other[i] = other_half<d()>(list[i]);
    merge(list, other);
  });
  // Slot k is lane k's; with fewer lanes than slots a lane has several.
  constexpr int kMine = N > L ? N / L : 1;
  float score[kMine], total = 0.0f;
  int id[kMine];
#pragma unroll
  for (int m = 0; m < kMine; ++m) {
    const int k = sub + m * L;
    double key = none_key();
#pragma unroll
    for (int i = m * L; i < min(N, (m + 1) * L); ++i) key = i == k ? list[i] : key;
    const float c = choice_of(key);
    const bool chosen = k < K && c != kNone();
    id[m] = chosen ? expert_of(key) : -1;
    const float logit = p.bias ? (chosen ? usable(logit_at(x, id[m])) : kNone()) : c;
    score[m] = !chosen ? 0.0f : softmax ? expf(logit - choice_of(list[0])) : logistic(logit);
    total += score[m];
  }
  float by = 1.0f;
  if (p.r.renormalise) {
    over_halves<1, L>([&](auto d) { total += other_half<d()>(total); });
    by = total;
  } else if (softmax) {   // over all experts, once more through them; scores are relative to the largest of all
    const float first = choice_of(list[0]), shift = first == kNone() ? 1.0f : expf(first - best);
    float sum = 0.0f;
    for (int at = e; at < end; at += N) {
      float v[N];
      load_logits<N>(x + at, end - at, v);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float u = usable(v[i]);
        sum += u == kNone() ? 0.0f : expf(u - best);
      }
    }
    over_halves<1, L>([&](auto d) { sum += other_half<d()>(sum); });
    by = sum;
#pragma unroll
    for (int m = 0; m < kMine; ++m) score[m] *= shift;
  }
#pragma unroll
  for (int m = 0; m < kMine; ++m) {
    const int k = sub + m * L;
    if (there && k < K) {
      p.ids[t * K + k] = id[m];
      p.weights[t * K + k] = by > 0.0f ? score[m] / by * p.r.scale : 0.0f;
    }
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

// Eight elements as they were loaded.
template <typename IN>
struct Eight;
template <>
struct Eight<uint16_t> {
  u32x4 w;
  Eight() = default;
  __device__ __forceinline__ explicit Eight(const uint16_t *p) : w(*(const u32x4_align2 *)p) {}
  __device__ __forceinline__ float at(int i) const { return i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]); }
  __device__ __forceinline__ float times(const Eight &v, float sum) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = fmaf(bf16_hi(w[i]), bf16_hi(v.w[i]), fmaf(bf16_lo(w[i]), bf16_lo(v.w[i]), sum));
    return sum;
  }
};
template <>
struct Eight<float> {
  f32x4 a, b;
  Eight() = default;
  __device__ __forceinline__ explicit Eight(const float *p)
      : a(*(const f32x4_align4 *)p), b(*(const f32x4_align4 *)(p + 4)) {}
  __device__ __forceinline__ float at(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ __forceinline__ float times(const Eight &v, float sum) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = fmaf(b[i], v.b[i], fmaf(a[i], v.a[i], sum));
    return sum;
  }
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

static hm_status check_router(const hm_router *r) {
  if (!r) return HM_ERR_NULL;
  if (r->E < 1 || r->E > kMostExperts || r->K < 1 || r->K > kMostSlots) return HM_ERR_SHAPE;
  if (r->score != HM_SCORE_SOFTMAX && r->score != HM_SCORE_SIGMOID) return HM_ERR_SHAPE;
  if (r->groups < 1 || r->groups > r->E || r->E % r->groups) return HM_ERR_SHAPE;
  if (r->top_groups < 1 || r->top_groups > r->groups) return HM_ERR_SHAPE;
  if (r->group_best < 1 || r->group_best > 2 || r->group_best > r->E / r->groups) return HM_ERR_SHAPE;
  if (r->K > r->E / r->groups * r->top_groups) return HM_ERR_SHAPE;
  return HM_OK;
}
// Lanes of a token for the choice by lists, 0 where it is not made: groups share the lanes, and a softmax with a bias
// needs its sum before the choice.
static int list_lanes(const hm_router &r, bool biased, int64_t T) {
  if (r.K > 16 || (r.groups & (r.groups - 1)) || r.groups > 16 || (biased && r.score == HM_SCORE_SOFTMAX)) return 0;
  if (T >= 16384 && r.groups <= 8 && r.E <= 64 * 8) return 8;
  return r.E <= 64 * 16 ? 16 : 0;
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
