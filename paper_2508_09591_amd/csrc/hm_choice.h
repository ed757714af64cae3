// The choice of a token's experts by sorted lists, as hm_route makes it and the layer for a few tokens makes it inside.
#pragma once

#include "hm_block8.h"

namespace hm {

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

// L lanes take token t, each a run of its experts, of which it keeps the N >= K largest; the lists of the lanes are
// then merged pairwise.  With groups the L lanes are shared among them, so that a lane's run lies in one group, and
// the two largest of its list give the group's score: lists of groups that are not taken are emptied before the merges.
// What bounds it are vector instructions: about 27 an expert for a logistic score, 4 for its key and 9 for sorting (N =
// 8), against 4 bytes read.  us: 65,536 tokens, 256 experts, logistic with bias and groups 30 (2.4 TB/s), softmax 24,
// bf16 18; one token 5.3. 8 lanes a token from 16,384 tokens on: 65,536 x 64 8.4 and, with 16 lanes, 14.7; 8,192 x 256
// 8.3 and 6.9.
// store(k, expert, weight) is called for each slot of a token that is there, by the lane that holds it.
template <typename IN, int L, int N, typename STORE>
__device__ __forceinline__ void choose_by_lists(const RouteParams &p, int64_t t, int lanes_per_group, int run,
                                                STORE store) {
  const int sub = (int)threadIdx.x & (L - 1);
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
    __builtin_amdgcn_sched_barrier(0);   // else the bias comes behind the wait for the logits: 65,536 x 256 30 -> 34 us
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
    const float choice = choice_of(key);
    const bool chosen = k < K && choice != kNone();
    id[m] = chosen ? expert_of(key) : -1;
    const float logit = p.bias ? (chosen ? usable(logit_at(x, id[m])) : kNone()) : choice;
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
    if (there && k < K) store(k, id[m], by > 0.0f ? score[m] / by * p.r.scale : 0.0f);
  }
}

constexpr int kMostExperts = 4096, kMostSlots = 64;
static inline hm_status check_router(const hm_router *r) {
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
static inline int list_lanes(const hm_router &r, bool biased, int64_t T) {
  if (r.K > 16 || (r.groups & (r.groups - 1)) || r.groups > 16 || (biased && r.score == HM_SCORE_SOFTMAX)) return 0;
  if (T >= 16384 && r.groups <= 8 && r.E <= 64 * 8) return 8;
  return r.E <= 64 * 16 ? 16 : 0;
}

}  // namespace hm
