// Clipped policy loss over the response tokens of packed groups, with its gradient.
//
// A row of a packed batch is a prompt and K sampled responses.  For every counted token
// t of a response, with d = logp_t - old_t, r = e^d and its advantage A:
//
//   surrogate  min(r A, clip(r, 1 - clip_low, 1 + clip_high) A), and for A < 0 with a dual
//              clip c no less than c A
//   KL         x = ref_t - logp_t:  k1 -x,  k2 x^2 / 2,  k3 e^x - 1 - x
//   loss       sum_t w_t (-surrogate + kl_coef KL - ent_coef entropy_t)
//   gradient   w_t (-A r, 0 where the clip holds, + kl_coef dKL/dlogp), -ent_coef w_t
//
// with w_t = 1 / (counted tokens), 1 / (responses x the response's counted tokens), or
// 1 / norm.  Bytes are few (33 per token at most), so launches and latency set the time:
//
//   policy_small    one workgroup does it all: up to kPolicySmall tokens
//   policy_records  the responses' records to the workspace, and their counted tokens
//   policy_tokens   the terms, token by token, and a workgroup's sums
//   policy_reduce   the sums in workgroup order (no atomics on results)
//
// A token's terms and all sums are 64 bits, so a result is as good as its rounding to fp32,
// what counts as clipped is what the exact ratio says, and a ratio past fp32 that a small
// weight or advantage brings back counts as what it is.  The 64-bit units multiply and add
// at fp32's plain rate, and one short exponential serves the ratio and the KL term:
// policy_tokens takes 15.4 us for 1.2M tokens (13.7 with fp32 terms), a call as long as then.

#include <hip/hip_runtime.h>
#include <math.h>

#include "pp_device.h"
#include "pp_launch.h"

namespace pp {
namespace {

constexpr int kThreads = kPolicyThreads;

// Responses ride in the launch's arguments when they are few.  A launch with 3 KB of
// arguments takes the host 4.3 us, one with 500 bytes 3.5 and one with 64 bytes 2.5, so
// there are two sizes, and none.
template <int N>
struct InlineSlots {
  static constexpr int kSlots = N;
  PolicySlot slot[N];
};

struct NoSlots {
  static constexpr int kSlots = 0;
};

__device__ __forceinline__ double wave_sum_d(double x) {
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}
__device__ __forceinline__ int wave_sum_i(int x) {
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

// Counted tokens of a response, by a wave.
__device__ __forceinline__ int count_tokens(const PolicyParams& p, const PolicySlot& sl) {
  if (!p.mask) return sl.len;
  const uint8_t* m = p.mask + sl.begin;
  constexpr int U = 16;  // bytes in flight a lane: most responses in one go
  int n = 0;
  for (int j = threadIdx.x & 63; j < sl.len; j += 64 * U) {
    uint8_t v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = j + 64 * u < sl.len ? m[j + 64 * u] : (uint8_t)0;
#pragma unroll
    for (int u = 0; u < U; ++u) n += v[u] != 0;
  }
  return wave_sum_i(n);
}

// A wave a response; `from`: records in mapped host memory, or null (inl, or in place).
// It also notes, for the workgroups of policy_tokens (chunk tokens each) that start
// between the end of the response ahead and its own, that it is the first they meet.
template <typename Inline>
__global__ __launch_bounds__(kThreads) void policy_records_kernel(PolicyParams p, const PolicySlot* from, int chunk, Inline inl) {
  const int i = (int)((blockIdx.x * kThreads + threadIdx.x) >> 6), lane = threadIdx.x & 63;
  if (i >= p.n_slots) return;
  auto at = [&](int k) {
    if constexpr (Inline::kSlots > 0) return inl.slot[k];
    else return from ? from[k] : p.slots[k];
  };
  const PolicySlot sl = at(i);
  const int64_t from_t = i > 0 ? (int64_t)at(i - 1).begin + at(i - 1).len : 0, to_t = (int64_t)sl.begin + sl.len;
  const int chunks = (int)((p.sumT + chunk - 1) / chunk);
  const int c_first = (int)((from_t + chunk - 1) / chunk), c_end = min(chunks, (int)((to_t + chunk - 1) / chunk));
  for (int c = c_first + lane; c < c_end; c += 64) p.first[c] = i;
  if (i == p.n_slots - 1)
    for (int c = c_end + lane; c < chunks; c += 64) p.first[c] = p.n_slots;
  const int n = count_tokens(p, sl);
  if (lane == 0) {
    if (!p.in_place) p.slots[i] = sl;
    p.slot_counts[i] = n;
  }
}

__device__ __forceinline__ void write_results(const PolicyParams& p, const PolicyPartial& t) {
  double loss = t.sum[0];
  if (p.kl_coef != 0) loss += p.kl_coef * t.sum[1];
  if (p.ent_coef != 0) loss -= p.ent_coef * t.sum[2];
  *p.loss = (float)loss;
  if (p.stats)
    for (int i = 0; i < 4; ++i) p.stats[i] = (float)t.sum[i];
  if (p.counts) {
    p.counts[0] = t.counted;
    p.counts[1] = t.clipped;
  }
}

// The workgroup's sums in a fixed order, valid in thread 0.
template <int THREADS>
__device__ __forceinline__ PolicyPartial block_sum(PolicyPartial t) {
  __shared__ PolicyPartial part[THREADS / 64];
#pragma unroll
  for (int i = 0; i < 4; ++i) t.sum[i] = wave_sum_d(t.sum[i]);
  t.counted = wave_sum_i(t.counted);
  t.clipped = wave_sum_i(t.clipped);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < THREADS / 64; ++w) {
#pragma unroll
      for (int i = 0; i < 4; ++i) t.sum[i] += part[w].sum[i];
      t.counted += part[w].counted;
      t.clipped += part[w].clipped;
    }
  }
  return t;
}

// e^x as 2^k (1 + r + q): x = k ln 2 + r with |r| <= ln 2 / 2, and q = e^r - 1 - r from its
// series, whose first missing term is 2^-53 of it.  So e^x - 1 = r + q and e^x - 1 - x = q
// keep all their digits where k = 0, and elsewhere little cancels.
struct Exp {
  double e;         // e^x
  double m1, m1x;   // e^x - 1, e^x - 1 - x
};
__device__ __forceinline__ Exp exp_of(double x) {
  const double c = x < -800.0 ? -800.0 : x > 800.0 ? 800.0 : x;  // 0 and infinity; NaN stays
  const double k = rint(c * 1.4426950408889634);
  // ln 2 in two parts (Cody and Waite): its first 40 bits, whose products with k are exact, and the rest
  double r = fma(k, -0x1.62e42fefa2000p-1, c);
  r = fma(k, -0x1.9ef35793c7673p-41, r);
  double p = 1.0 / 6227020800;  // 1 / 13!
  p = fma(p, r, 1.0 / 479001600);
  p = fma(p, r, 1.0 / 39916800);
  p = fma(p, r, 1.0 / 3628800);
  p = fma(p, r, 1.0 / 362880);
  p = fma(p, r, 1.0 / 40320);
  p = fma(p, r, 1.0 / 5040);
  p = fma(p, r, 1.0 / 720);
  p = fma(p, r, 1.0 / 120);
  p = fma(p, r, 1.0 / 24);
  p = fma(p, r, 1.0 / 6);
  p = fma(p, r, 0.5);
  const double q = p * (r * r);
  Exp y;
  y.e = ldexp(1.0 + (r + q), k == k ? (int)k : 0);
  y.m1 = k == 0.0 ? r + q : y.e - 1.0;
  y.m1x = k == 0.0 ? q : y.m1 - x;
  return y;
}

// What a counted token adds, before its weight.
struct PolicyTerms {
  double grad;       // of the unweighted loss, but for the entropy
  double surr, kl, ratio;
  bool clipped;
};

__device__ __forceinline__ PolicyTerms policy_terms(const PolicyParams& p, double lp, double old, double ref, double A) {
  PolicyTerms t;
  const double d_lp = p.old ? lp - old : 0.0;
  t.ratio = p.old ? exp_of(d_lp).e : 1.0;
  double used = t.ratio;
  t.clipped = false;
  auto clip = [&](double end) {
    t.clipped = true;
    used = end;
  };
  if (p.old) {
    if (A > 0.0 && t.ratio > 1.0 + p.clip_high) clip(1.0 + p.clip_high);
    else if (A < 0.0 && t.ratio < 1.0 - p.clip_low) clip(1.0 - p.clip_low);
    else if (A < 0.0 && p.dual_clip > 0 && t.ratio > p.dual_clip) clip(p.dual_clip);
  }
  if (A == 0.0 && d_lp < __builtin_inf()) used = 0.0;  // no advantage of a ratio past 64 bits
  t.surr = used * A;
  t.grad = t.clipped ? 0.0 : -A * used;
  t.kl = 0.0;
  if (p.ref) {
    const double x = ref - lp;
    double d;
    if (p.kl == PP_KL_K1) {
      t.kl = -x;
      d = 1.0;
    } else if (p.kl == PP_KL_K2) {
      t.kl = 0.5 * x * x;
      d = -x;
    } else {
      const Exp y = exp_of(x);
      t.kl = y.m1x;
      d = -y.m1;
    }
    if (p.kl_coef != 0) t.grad = fma(p.kl_coef, d, t.grad);
  }
  return t;
}

// A token's share of the sums.
__device__ __forceinline__ void add_token(PolicyPartial& sum, const PolicyTerms& t, double w, float ent, bool with_ent) {
  sum.sum[0] -= w * t.surr;
  sum.sum[1] += w * t.kl;
  if (with_ent) sum.sum[2] += w * ent;
  sum.sum[3] += w * t.ratio;
  sum.counted += 1;
  sum.clipped += t.clipped;
}

// The weight of a response's tokens: `some` responses have a counted one, `total` tokens
// are counted, n of this response.
__device__ __forceinline__ double slot_weight(const PolicyParams& p, int64_t total, int some, int n) {
  if (p.reduction == PP_REDUCE_SUM) return 1.0 / p.norm;
  if (p.reduction == PP_REDUCE_TOKEN) return 1.0 / (double)(total > 0 ? total : 1);
  return n > 0 ? 1.0 / ((double)some * n) : 0.0;
}

// The first response that ends behind position c: 64 probes a round.
template <typename At>
__device__ __forceinline__ int first_slot(int n_slots, int64_t c, At&& at) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n_slots;
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    bool before = false;
    if (i < hi) {
      const PolicySlot s = at(i);
      before = (int64_t)s.begin + s.len <= c;
    }
    const int n = __popcll(__ballot(before));
    if (n == 0) return lo;
    hi = min(hi, lo + n * step);
    lo = lo + (n - 1) * step + 1;
  }
  return lo;
}

// TPT consecutive tokens a thread; their values are on the way while the responses that
// they belong to are found.  Records that come with the launch are those of an unmasked
// batch: there are no counts to read.
template <int TPT, typename Inline>
__global__ __launch_bounds__(kThreads) void policy_tokens_kernel(PolicyParams p, Inline inl) {
  constexpr bool IN_ARGS = Inline::kSlots > 0;
  constexpr int CH = kThreads * TPT;
  __shared__ int s_begin[CH], s_end[CH], s_out[CH], s_count[CH];
  __shared__ double s_w[CH];
  __shared__ int s_first, s_n, s_total, s_some;
  const int tid = threadIdx.x;
  const bool masked = !IN_ARGS && p.mask != nullptr;
  const int64_t c0 = (int64_t)blockIdx.x * CH, c1 = c0 + CH < p.sumT ? c0 + CH : p.sumT;
  auto slot_at = [&](int i) {
    if constexpr (IN_ARGS) return inl.slot[i];
    else return p.slots[i];
  };
  const int64_t t0 = c0 + (int64_t)tid * TPT;
  typedef float fvec __attribute__((ext_vector_type(TPT)));
  const bool whole = t0 + TPT <= p.sumT;
  float lp[TPT], old[TPT], ref[TPT], ent[TPT], adv[TPT];
  uint8_t keep[TPT];
  auto load = [&](const float* src, float* dst) {
#pragma unroll
    for (int e = 0; e < TPT; ++e) dst[e] = 0.f;
    if (!src) return;
    if (TPT > 1 && whole) {
      const fvec v = *reinterpret_cast<const fvec*>(src + t0);
#pragma unroll
      for (int e = 0; e < TPT; ++e) dst[e] = v[e];
    } else {
#pragma unroll
      for (int e = 0; e < TPT; ++e)
        if (t0 + e < p.sumT) dst[e] = src[t0 + e];
    }
  };
  load(p.logp, lp);
  load(p.old, old);
  load(p.ref, ref);
  load(p.entropy, ent);
  load(p.adv_per_token ? p.adv : nullptr, adv);
  if (masked) {
    if (TPT == 4 && whole) {  // 4-byte aligned here
      const uint32_t v = *reinterpret_cast<const uint32_t*>(p.mask + t0);
#pragma unroll
      for (int e = 0; e < TPT; ++e) keep[e] = (uint8_t)(v >> (8 * e));
    } else {
#pragma unroll
      for (int e = 0; e < TPT; ++e) keep[e] = t0 + e < p.sumT ? p.mask[t0 + e] : (uint8_t)0;
    }
  }
  if (tid == 0) s_n = s_total = s_some = 0;
  // what the mask counts of all the batch, eight responses in flight a thread
  int total = 0, some = 0;
  if (masked && p.reduction != PP_REDUCE_SUM) {
    constexpr int U = 8;
    for (int i = tid; i < p.n_slots; i += kThreads * U) {
      int v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = i + kThreads * u < p.n_slots ? p.slot_counts[i + kThreads * u] : 0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        total += v[u];
        some += v[u] > 0;
      }
    }
  }
  int first;
  if constexpr (IN_ARGS) {
    if (tid < 64) {
      const int f = first_slot(p.n_slots, c0, slot_at);
      if (tid == 0) s_first = f;
    }
    __syncthreads();
    first = s_first;
  } else {
    first = p.n_slots > 0 ? p.first[blockIdx.x] : 0;
    __syncthreads();
  }
  if (masked && p.reduction != PP_REDUCE_SUM) {
    total = wave_sum_i(total);
    some = wave_sum_i(some);
    if ((tid & 63) == 0) {
      atomicAdd(&s_total, total);
      atomicAdd(&s_some, some);
    }
  }
  // the responses that reach into [c0, c1): CH at most, none being empty
  for (int i = tid; i < CH && first + i < p.n_slots; i += kThreads) {
    const PolicySlot sl = slot_at(first + i);
    if (sl.begin >= c1) break;
    s_begin[i] = sl.begin;
    s_end[i] = sl.begin + sl.len;
    s_out[i] = sl.out;
    s_count[i] = masked ? p.slot_counts[first + i] : sl.len;
    atomicMax(&s_n, i + 1);
  }
  __syncthreads();
  const int n = s_n;
  for (int i = tid; i < n; i += kThreads)
    s_w[i] = slot_weight(p, masked ? (int64_t)s_total : p.tokens, masked ? s_some : p.n_slots, s_count[i]);
  __syncthreads();

  PolicyPartial sum{};
  if (t0 < c1) {
    float out_lp[TPT], out_ent[TPT];
    // the last response that begins at or ahead of t0
    int lo = 0, hi = n;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_begin[mid] <= t0) lo = mid + 1;
      else hi = mid;
    }
    int i = lo - 1;
#pragma unroll
    for (int e = 0; e < TPT; ++e) {
      const int64_t t = t0 + e;
      if (i + 1 < n && s_begin[i + 1] <= t) ++i;
      out_lp[e] = out_ent[e] = 0.f;
      if (i < 0 || t >= s_end[i] || t >= c1 || (masked && !keep[e])) continue;
      const double w = s_w[i];
      const PolicyTerms x = policy_terms(p, lp[e], old[e], ref[e], p.adv_per_token ? adv[e] : p.adv[s_out[i]]);
      out_lp[e] = (float)(w * x.grad);
      out_ent[e] = (float)(-p.ent_coef * w);
      add_token(sum, x, w, ent[e], p.entropy != nullptr);
    }
    auto store = [&](float* dst, const float* src) {
      if (!dst) return;
      if (TPT > 1 && whole) {
        fvec v;
#pragma unroll
        for (int e = 0; e < TPT; ++e) v[e] = src[e];
        *reinterpret_cast<fvec*>(dst + t0) = v;
      } else {
#pragma unroll
        for (int e = 0; e < TPT; ++e)
          if (t0 + e < p.sumT) dst[t0 + e] = src[e];
      }
    };
    store(p.dlogp, out_lp);
    store(p.dentropy, out_ent);
  }
  sum = block_sum<kThreads>(sum);
  if (tid == 0) p.part[blockIdx.x] = sum;
}

// Few tokens of few responses: a call of one launch.  16 waves count the responses'
// tokens, then every thread takes each 1024th token, its response found by stepping on.
constexpr int kSmallThreads = 1024;
template <typename Inline>
__global__ __launch_bounds__(kSmallThreads) void policy_small_kernel(PolicyParams p, Inline inl) {
  constexpr int S = Inline::kSlots;
  __shared__ int s_begin[S], s_end[S], s_out[S], s_n[S];
  __shared__ double s_w[S];
  __shared__ int s_total, s_some;
  const int tid = threadIdx.x, wave = tid >> 6;
  if (tid == 0) s_total = s_some = 0;
  for (int i = wave; i < p.n_slots; i += kSmallThreads / 64) {
    const PolicySlot sl = inl.slot[i];
    const int n = count_tokens(p, sl);
    if ((tid & 63) == 0) {
      s_begin[i] = sl.begin;
      s_end[i] = sl.begin + sl.len;
      s_out[i] = sl.out;
      s_n[i] = n;
    }
  }
  __syncthreads();
  if (tid < p.n_slots && s_n[tid] > 0) {
    atomicAdd(&s_total, s_n[tid]);
    atomicAdd(&s_some, 1);
  }
  __syncthreads();
  if (tid < p.n_slots) s_w[tid] = slot_weight(p, s_total, s_some, s_n[tid]);
  __syncthreads();
  PolicyPartial sum{};
  constexpr int U = 4;  // tokens in flight a thread
  int i = 0;
  for (int t0 = tid; t0 < (int)p.sumT; t0 += kSmallThreads * U) {
    float lp[U], old[U], ref[U], ent[U], adv[U];
    int slot[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * kSmallThreads;
      while (i < p.n_slots && s_end[i] <= t) ++i;
      slot[u] = t < (int)p.sumT && i < p.n_slots && t >= s_begin[i] ? i : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = slot[u] < 0 ? 0 : t0 + u * kSmallThreads;
      if (p.mask && !p.mask[t]) slot[u] = -1;
      lp[u] = p.logp[t];
      old[u] = p.old ? p.old[t] : 0.f;
      ref[u] = p.ref ? p.ref[t] : 0.f;
      ent[u] = p.entropy ? p.entropy[t] : 0.f;
      adv[u] = slot[u] < 0 ? 0.f : p.adv[p.adv_per_token ? t : s_out[slot[u]]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * kSmallThreads;
      if (t >= (int)p.sumT) break;
      float out_lp = 0.f, out_ent = 0.f;
      if (slot[u] >= 0) {
        const double w = s_w[slot[u]];
        const PolicyTerms x = policy_terms(p, lp[u], old[u], ref[u], adv[u]);
        out_lp = (float)(w * x.grad);
        out_ent = (float)(-p.ent_coef * w);
        add_token(sum, x, w, ent[u], p.entropy != nullptr);
      }
      if (p.dlogp) p.dlogp[t] = out_lp;
      if (p.dentropy) p.dentropy[t] = out_ent;
    }
  }
  sum = block_sum<kSmallThreads>(sum);
  if (tid == 0) write_results(p, sum);
}

__global__ __launch_bounds__(kThreads) void policy_reduce_kernel(PolicyParams p, int n) {
  PolicyPartial t{};
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const PolicyPartial x = p.part[i];
#pragma unroll
    for (int c = 0; c < 4; ++c) t.sum[c] += x.sum[c];
    t.counted += x.counted;
    t.clipped += x.clipped;
  }
  t = block_sum<kThreads>(t);
  if (threadIdx.x == 0) write_results(p, t);
}

template <typename Inline>
hipError_t launch_policy_t(const PolicyLaunch& a, const Inline& inl, hipStream_t s) {
  PolicyParams p = a;
  hipError_t e = hipSuccess;
  constexpr bool in_args = Inline::kSlots > 0;
  if constexpr (in_args) {
    if (policy_small(a.sumT, a.n_slots)) {
      TimingScope t("pp_policy_tokens", s);
      hipLaunchKernelGGL(policy_small_kernel<Inline>, dim3(1), dim3(kSmallThreads), 0, s, p, inl);
      return hipGetLastError();
    }
  }
  uintptr_t any = 0;
  for (const void* x : {(const void*)a.logp, (const void*)a.old, (const void*)a.ref, (const void*)a.entropy,
                        a.adv_per_token ? (const void*)a.adv : nullptr, (const void*)a.dlogp, (const void*)a.dentropy})
    any |= reinterpret_cast<uintptr_t>(x);
  const bool vec = (any & 15) == 0 && (reinterpret_cast<uintptr_t>(a.mask) & 3) == 0 && a.sumT >= 1 << 18;
  const int64_t ch = kThreads * (vec ? 4 : 1);
  const int blocks = (int)((a.sumT + ch - 1) / ch);
  const bool plain = in_args && !a.mask;  // no records to stage, nothing to count
  if (a.n_slots > 0 && !plain) {
    TimingScope t("pp_policy_records", s);
    p.in_place = !a.from && !in_args;
    const int per = kThreads / 64;
    hipLaunchKernelGGL(policy_records_kernel<Inline>, dim3((a.n_slots + per - 1) / per), dim3(kThreads), 0, s, p, a.from, (int)ch,
                       inl);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  {
    TimingScope t("pp_policy_tokens", s);
    auto launch = [&](auto kernel, auto& records) {
      hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, s, p, records);
    };
    const NoSlots none;
    if (plain && vec) launch(policy_tokens_kernel<4, Inline>, inl);
    else if (plain) launch(policy_tokens_kernel<1, Inline>, inl);
    else if (vec) launch(policy_tokens_kernel<4, NoSlots>, none);
    else launch(policy_tokens_kernel<1, NoSlots>, none);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  TimingScope t("pp_policy_reduce", s);
  hipLaunchKernelGGL(policy_reduce_kernel, dim3(1), dim3(kThreads), 0, s, p, blocks);
  return hipGetLastError();
}

template <int N>
hipError_t launch_policy_inline(const PolicyLaunch& a, hipStream_t s) {
  InlineSlots<N> inl;
  for (int i = 0; i < N; ++i) inl.slot[i] = i < a.n_slots ? a.host_slots[i] : PolicySlot{};
  return launch_policy_t(a, inl, s);
}

}  // namespace

hipError_t launch_policy(const PolicyLaunch& a, hipStream_t s) {
  if (a.n_slots <= 40) return launch_policy_inline<40>(a, s);
  if (policy_inline(a.n_slots)) return launch_policy_inline<kPolicyInline>(a, s);
  return launch_policy_t(a, NoSlots{}, s);
}

}  // namespace pp
