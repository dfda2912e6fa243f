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
// 1 / norm.  Kernels:
//
//   policy_count    counted tokens of every response, where a mask decides
//   policy_tokens   the terms, token by token, and a workgroup's sums
//   policy_reduce   the sums in workgroup order (no atomics)
//
// Bytes are few (33 per token at most), so launches and latency set the time.  A token's terms are formed
// in 64 bits: whether a clip holds is then decided by the ratio and not by its rounding to
// fp32, and e^x - 1 - x keeps its digits for small x; sums too.

#include <hip/hip_runtime.h>
#include <math.h>

#include "pp_device.h"
#include "pp_launch.h"

namespace pp {
namespace {

constexpr int kThreads = kPolicyThreads;

// Responses ride in the launch's arguments when they are few.
struct InlineSlots {
  PolicySlot slot[kPolicyInline];
};

__device__ __forceinline__ PolicySlot slot_of(const PolicyParams& p, const InlineSlots& inl, int i) {
  return p.slots ? p.slots[i] : inl.slot[i];
}

__device__ __forceinline__ double wave_sum_d(double x) {
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}
__device__ __forceinline__ int wave_sum_i(int x) {
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

// A wave a response.
__global__ __launch_bounds__(kThreads) void policy_count_kernel(PolicyParams p, InlineSlots inl) {
  const int i = (int)((blockIdx.x * kThreads + threadIdx.x) >> 6), lane = threadIdx.x & 63;
  if (i >= p.n_slots) return;
  const PolicySlot sl = slot_of(p, inl, i);
  int n = 0;
  for (int j = lane; j < sl.len; j += 64) n += p.mask[(int64_t)sl.begin + j] != 0;
  n = wave_sum_i(n);
  if (lane == 0) p.slot_counts[i] = n;
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
__device__ __forceinline__ PolicyPartial block_sum(PolicyPartial t) {
  __shared__ PolicyPartial part[kThreads / 64];
#pragma unroll
  for (int i = 0; i < 4; ++i) t.sum[i] = wave_sum_d(t.sum[i]);
  t.counted = wave_sum_i(t.counted);
  t.clipped = wave_sum_i(t.clipped);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) {
#pragma unroll
      for (int i = 0; i < 4; ++i) t.sum[i] += part[w].sum[i];
      t.counted += part[w].counted;
      t.clipped += part[w].clipped;
    }
  }
  return t;
}

// The first response that ends behind position c: 64 probes a round.
__device__ __forceinline__ int first_slot(const PolicyParams& p, const InlineSlots& inl, int64_t c) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = p.n_slots;
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    bool before = false;
    if (i < hi) {
      const PolicySlot s = slot_of(p, inl, i);
      before = (int64_t)s.begin + s.len <= c;
    }
    const int n = __popcll(__ballot(before));
    if (n == 0) return lo;
    hi = min(hi, lo + n * step);
    lo = lo + (n - 1) * step + 1;
  }
  return lo;
}

// TPT consecutive tokens a thread.
template <int TPT>
__global__ __launch_bounds__(kThreads) void policy_tokens_kernel(PolicyParams p, InlineSlots inl) {
  constexpr int CH = kThreads * TPT;
  __shared__ int s_begin[CH + 1], s_end[CH + 1], s_out[CH + 1];
  __shared__ double s_w[CH + 1];
  __shared__ int s_first, s_n, s_total, s_some;
  const int tid = threadIdx.x;
  const int64_t c0 = (int64_t)blockIdx.x * CH, c1 = c0 + CH < p.sumT ? c0 + CH : p.sumT;
  if (tid == 0) s_n = s_total = s_some = 0;
  if (tid < 64) {
    const int f = first_slot(p, inl, c0);
    if (tid == 0) s_first = f;
  }
  __syncthreads();
  const int first = s_first;
  const bool masked = p.mask != nullptr;
  if (masked && p.reduction != PP_REDUCE_SUM) {  // what the mask counts of all the batch
    int total = 0, some = 0;
    for (int i = tid; i < p.n_slots; i += kThreads) {
      const int n = p.slot_counts[i];
      total += n;
      some += n > 0;
    }
    total = wave_sum_i(total);
    some = wave_sum_i(some);
    if ((tid & 63) == 0) {
      atomicAdd(&s_total, total);
      atomicAdd(&s_some, some);
    }
  }
  // the responses that reach into [c0, c1): CH at most, none being empty
  for (int i = tid; i < CH && first + i < p.n_slots; i += kThreads) {
    const PolicySlot sl = slot_of(p, inl, first + i);
    if (sl.begin >= c1) break;
    s_begin[i] = sl.begin;
    s_end[i] = sl.begin + sl.len;
    s_out[i] = sl.out;
    atomicMax(&s_n, i + 1);
  }
  __syncthreads();
  const int n = s_n;
  {
    const double total = masked ? (double)s_total : (double)p.tokens;
    const double some = masked ? (double)s_some : (double)p.n_slots;
    for (int i = tid; i < n; i += kThreads) {
      double w = 1.0 / p.norm;
      if (p.reduction == PP_REDUCE_TOKEN) w = 1.0 / fmax(total, 1.0);
      else if (p.reduction == PP_REDUCE_SEQ)
        w = 1.0 / (some * (double)max(1, masked ? p.slot_counts[first + i] : s_end[i] - s_begin[i]));
      s_w[i] = w;
    }
  }
  __syncthreads();

  const int64_t t0 = c0 + (int64_t)tid * TPT;
  PolicyPartial sum{};
  if (t0 < c1) {
    typedef float fvec __attribute__((ext_vector_type(TPT)));
    float out_lp[TPT], out_ent[TPT];
    float lp[TPT], old[TPT], ref[TPT], ent[TPT], adv[TPT];
    uint8_t keep[TPT];
    const bool whole = t0 + TPT <= p.sumT;
    auto load = [&](const float* src, float* dst) {
      if (!src) return;
      if (TPT > 1 && whole) {
        const fvec v = *reinterpret_cast<const fvec*>(src + t0);
#pragma unroll
        for (int e = 0; e < TPT; ++e) dst[e] = v[e];
      } else {
#pragma unroll
        for (int e = 0; e < TPT; ++e) dst[e] = t0 + e < p.sumT ? src[t0 + e] : 0.f;
      }
    };
    load(p.logp, lp);
    load(p.old, old);
    load(p.ref, ref);
    load(p.entropy, ent);
    if (p.adv_per_token) load(p.adv, adv);
    if (masked) {
#pragma unroll
      for (int e = 0; e < TPT; ++e) keep[e] = t0 + e < p.sumT ? p.mask[t0 + e] : (uint8_t)0;
    }
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
      const double A = p.adv_per_token ? adv[e] : p.adv[s_out[i]];
      const double ratio = p.old ? exp((double)lp[e] - (double)old[e]) : 1.0;
      double used = ratio;
      bool off = false;
      if (A > 0 && ratio > 1.0 + p.clip_high) {
        off = true;
        used = 1.0 + p.clip_high;
      } else if (A < 0 && ratio < 1.0 - p.clip_low) {
        off = true;
        used = 1.0 - p.clip_low;
      } else if (A < 0 && p.dual_clip > 0 && ratio > p.dual_clip) {
        off = true;
        used = p.dual_clip;
      }
      double g = off ? 0.0 : -A * ratio;
      double kl = 0.0;
      if (p.ref) {
        const double x = (double)ref[e] - (double)lp[e];
        double dkl;
        if (p.kl == PP_KL_K1) {
          kl = -x;
          dkl = 1.0;
        } else if (p.kl == PP_KL_K2) {
          kl = 0.5 * x * x;
          dkl = -x;
        } else {
          const double em = expm1(x);
          kl = em - x;
          dkl = -em;
        }
        if (p.kl_coef != 0) g += p.kl_coef * dkl;
      }
      out_lp[e] = (float)(w * g);
      out_ent[e] = (float)(-p.ent_coef * w);
      sum.sum[0] -= w * (used * A);
      sum.sum[1] += w * kl;
      if (p.entropy) sum.sum[2] += w * (double)ent[e];
      sum.sum[3] += w * ratio;
      sum.counted += 1;
      sum.clipped += off;
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
  sum = block_sum(sum);
  if (tid == 0) {
    if (gridDim.x == 1) write_results(p, sum);
    else p.part[blockIdx.x] = sum;
  }
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
  t = block_sum(t);
  if (threadIdx.x == 0) write_results(p, t);
}

}  // namespace

hipError_t launch_policy(const PolicyLaunch& a, hipStream_t s) {
  const PolicyParams p = a;
  InlineSlots inl{};
  if (!a.slots)
    for (int i = 0; i < a.n_slots; ++i) inl.slot[i] = a.host_slots[i];
  hipError_t e = hipSuccess;
  if (a.mask && a.n_slots > 0 && a.reduction != PP_REDUCE_SUM) {
    TimingScope t("pp_policy_count", s);
    const int per = kThreads / 64;
    hipLaunchKernelGGL(policy_count_kernel, dim3((a.n_slots + per - 1) / per), dim3(kThreads), 0, s, p, inl);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  uintptr_t any = 0;
  for (const void* x : {(const void*)a.logp, (const void*)a.old, (const void*)a.ref, (const void*)a.entropy,
                        a.adv_per_token ? (const void*)a.adv : nullptr, (const void*)a.dlogp, (const void*)a.dentropy})
    any |= reinterpret_cast<uintptr_t>(x);
  const bool vec = (any & 15) == 0 && a.sumT >= 1 << 18;
  const int64_t ch = kThreads * (vec ? 4 : 1);
  const int blocks = a.sumT > 0 ? (int)((a.sumT + ch - 1) / ch) : 1;
  {
    TimingScope t("pp_policy_tokens", s);
    if (vec) hipLaunchKernelGGL(policy_tokens_kernel<4>, dim3(blocks), dim3(kThreads), 0, s, p, inl);
    else hipLaunchKernelGGL(policy_tokens_kernel<1>, dim3(blocks), dim3(kThreads), 0, s, p, inl);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (blocks > 1) {
    TimingScope t("pp_policy_reduce", s);
    hipLaunchKernelGGL(policy_reduce_kernel, dim3(1), dim3(kThreads), 0, s, p, blocks);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace pp
