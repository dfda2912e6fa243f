// Verification of drafted tokens, on gfx950: which nodes of a drafted tree stay, and the token
// that follows them.
//
// Node 0 of a sequence is its last token, nodes above it were drafted: a child of node i from
// q = softmax(draft_i / T).  With p = softmax(target_i / T), the children y of a node are
// tried in order, each with its number u:
//
//   w = p, Z = 1, a = 0;  y stays if u q(y) Z < w(y);  else a += Z, w = max(p - a q, 0), Z = sum w
//
// (w / Z is what is left of p: after a rejection the distribution is max(w / Z - q, 0), made 1
// again; in this form a step needs one sum over the vocabulary.)  Without draft logits the
// drafts are given: y stays if u Z < w(y), else w(y) = 0.  From a node that none of its
// children follow the next token is the first x at which the running sum of w passes u_0 Z.
//
//   draft_rows     a workgroup for 8192 entries of a row: maximum, sum, where the maximum is
//   draft_residual Z after a rejected child that has siblings behind it, one launch a sibling
//   draft_walk     every workgroup walks the tree on its own (nothing but LDS by then) and sums
//                  its entries of w at the node where the walk ends
//   draft_sample   a workgroup a sequence: the entry at which the running sum passes
//
// Probabilities are 64 bits throughout: numbers are compared with given ones, and a running
// sum over 10^5 entries in 32 bits passes a number u elsewhere in one case of some hundred.
// Bound by reading the rows once.

#include <hip/hip_runtime.h>
#include <math.h>

#include "pp_device.h"
#include "pp_sample.h"

namespace pp {
namespace {

constexpr int kThreads = 256;
constexpr int kWavesD = kThreads / 64;

template <typename T>
constexpr int kVec = 16 / sizeof(T);  // entries of a 16-byte load
template <typename T>
constexpr int kLoads = kDraftChunk / (kThreads * kVec<T>);  // a thread's

__device__ __forceinline__ float to_float(uint16_t x) { return bf16_bits_to_f32(x); }
__device__ __forceinline__ float to_float(float x) { return x; }
template <typename T>
__device__ __forceinline__ float lowest();
template <>
__device__ __forceinline__ float lowest<uint16_t>() {
  return bf16_bits_to_f32(0xff7f);
}
template <>
__device__ __forceinline__ float lowest<float>() {
  return -3.4028234663852886e38f;
}

// e^y for y <= 0 in 64 bits: e^y = 2^n e^r, |r| <= ln 2 / 2, by the series of e^r through r^13
// (the rest is below 2^-57 of it).
__device__ __forceinline__ double exp_neg(double y) {
  const double n = rint(fmax(y, -1000.0) * 1.4426950408889634);
  double r = fma(n, -0.6931471805599453, fmax(y, -1000.0));
  r = fma(n, -2.3190468138462996e-17, r);  // ln 2 less its 64-bit value
  double s = 1.0 / 6227020800.0;
  s = fma(s, r, 1.0 / 479001600.0);
  s = fma(s, r, 1.0 / 39916800.0);
  s = fma(s, r, 1.0 / 3628800.0);
  s = fma(s, r, 1.0 / 362880.0);
  s = fma(s, r, 1.0 / 40320.0);
  s = fma(s, r, 1.0 / 5040.0);
  s = fma(s, r, 1.0 / 720.0);
  s = fma(s, r, 1.0 / 120.0);
  s = fma(s, r, 1.0 / 24.0);
  s = fma(s, r, 1.0 / 6.0);
  s = fma(s, r, 0.5);
  s = fma(s, r, 1.0);
  s = fma(s, r, 1.0);
  return ldexp(s, (int)n);
}

// A thread's entries of one chunk of a row: load u holds entries at(u) .. + kVec - 1, -inf
// where masked or outside the row.  Loads lie on the row's 16-byte boundaries; those that
// reach over an end of the row are taken entry by entry.
template <typename T>
struct ChunkOf {
  const T* row;
  int64_t first;  // entry of the thread's first load
  int vocab;

  __device__ __forceinline__ void init(const T* r, int v, int chunk, int thread) {
    row = r;
    vocab = v;
    const int ahead = (int)((reinterpret_cast<uintptr_t>(r) / sizeof(T)) % kVec<T>);
    first = (int64_t)chunk * kDraftChunk + thread * kVec<T> - ahead;
  }
  __device__ __forceinline__ int64_t at(int u) const { return first + (int64_t)u * kThreads * kVec<T>; }
  __device__ __forceinline__ void load(int u, float (&x)[kVec<T>]) const {
    const int64_t e = at(u);
    if (e >= 0 && e + kVec<T> <= vocab) {
      typedef T Raw __attribute__((ext_vector_type(kVec<T>)));
      const Raw v = *reinterpret_cast<const Raw*>(row + e);
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) x[i] = to_float(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) x[i] = e + i >= 0 && e + i < vocab ? to_float(row[e + i]) : kNegInf;
    }
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) x[i] = x[i] == lowest<T>() ? kNegInf : x[i];
  }
};

__device__ __forceinline__ double wave_sum_d(double x) {
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

// A sequence's tree: lane l of a wave looks at node l.
struct TreeOf {
  int count;      // nodes
  uint64_t kids;  // lane's children, at most max_children of them
  int up, rank;   // the lane's parent (-1: none, or never reached) and its place among that one's children
};
__device__ __forceinline__ TreeOf tree_of(const DraftShape& d, const int32_t* parents, const int32_t* count, int s, int lane) {
  TreeOf t;
  t.count = max(0, min(count ? count[s] : d.nodes, d.nodes));
  int up = lane > 0 && lane < t.count ? (parents ? parents[(int64_t)s * d.nodes + lane] : lane - 1) : -1;
  if (up >= lane) up = -1;
  t.kids = 0;
  t.rank = 0;
  for (int j = 1; j < t.count; ++j) {
    const int uj = __builtin_amdgcn_readlane(up, j);
    if (uj < 0) continue;
    const int before = __popcll(__builtin_amdgcn_readlane((int)(t.kids >> 32), uj) & 0xffffffffu) +
                       __popcll(__builtin_amdgcn_readlane((int)t.kids, uj) & 0xffffffffu);
    if (lane == j) t.rank = before;
    if (before >= d.max_children) {
      if (lane == j) up = -1;
    } else if (lane == uj) {
      t.kids |= 1ull << j;
    }
  }
  t.up = up;
  return t;
}

__device__ __forceinline__ double inv_temp(const float* temperature, int s) {
  const double t = temperature ? (double)temperature[s] : 1.0;
  return t > 0 ? 1.0 / t : 1.0;
}
__device__ __forceinline__ bool greedy(const float* temperature, int s) { return temperature && !(temperature[s] > 0); }

template <typename T>
__global__ __launch_bounds__(kThreads) void draft_rows_kernel(DraftParams p) {
  __shared__ float s_m[kWavesD];
  __shared__ int s_arg[kWavesD];
  __shared__ double s_sum[kWavesD];
  __shared__ int s_bad;
  const DraftShape& d = p.shape;
  const int row = blockIdx.y, chunk = blockIdx.x, s = row / d.nodes, node = row - s * d.nodes;
  const bool is_draft = blockIdx.z != 0;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = max(0, min(p.count ? p.count[s] : d.nodes, d.nodes));
  if (node >= n) return;
  if (is_draft) {
    if (greedy(p.temperature, s)) return;
    bool kid = false;  // only nodes with children have drafts
    for (int j = node + 1 + lane; j < n; j += 64)
      kid = kid || (p.parents ? p.parents[(int64_t)s * d.nodes + j] == node : j == node + 1);
    if (!__any(kid)) return;
  }
  if (tid == 0) s_bad = 0;
  ChunkOf<T> c;
  c.init((const T*)(is_draft ? p.draft : p.target) + (int64_t)row * d.vocab, d.vocab, chunk, tid);
  float x[kLoads<T>][kVec<T>];
#pragma unroll
  for (int u = 0; u < kLoads<T>; ++u) c.load(u, x[u]);
  float m = kNegInf;
  int arg = 0x7fffffff;
  bool bad = false;
#pragma unroll
  for (int u = 0; u < kLoads<T>; ++u)
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) {
      bad = bad || !(x[u][i] < -kNegInf);  // NaN and +inf
      if (x[u][i] > m) {
        m = x[u][i];
        arg = (int)(c.at(u) + i);
      }
    }
  const float wm = wave_max(m);
  int wa = m == wm ? arg : 0x7fffffff;
  for (int off = 32; off > 0; off >>= 1) wa = min(wa, __shfl_xor(wa, off, 64));
  if (lane == 0) {
    s_m[wave] = wm;
    s_arg[wave] = wa;
  }
  __syncthreads();
  if (bad) s_bad = 1;
  float top = kNegInf;
#pragma unroll
  for (int w = 0; w < kWavesD; ++w) top = fmaxf(top, s_m[w]);
  const double it = inv_temp(p.temperature, s);
  double sum = 0;
  if (top > kNegInf) {
#pragma unroll
    for (int u = 0; u < kLoads<T>; ++u)
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) sum += x[u][i] > kNegInf ? exp_neg(((double)x[u][i] - (double)top) * it) : 0.0;
  }
  sum = wave_sum_d(sum);
  if (lane == 0) s_sum[wave] = sum;
  __syncthreads();
  if (tid == 0) {
    DraftPart out;
    out.sum = 0;
    out.arg = 0x7fffffff;
    for (int w = 0; w < kWavesD; ++w) {
      out.sum += s_sum[w];
      if (s_m[w] == top) out.arg = min(out.arg, s_arg[w]);
    }
    out.max = s_bad ? __builtin_nanf("") : top;
    p.part[((int64_t)blockIdx.z * d.n * d.nodes + row) * d.chunks + chunk] = out;
  }
}

// A row's distribution: e^((x - max) / T) / sum.
struct RowDist {
  float max;
  double sum;
  int arg;
  bool usable;
};
// By a wave, from the parts of the row's chunks.
__device__ __forceinline__ RowDist row_dist(const DraftPart* part, int chunks, double it, int lane) {
  float m = kNegInf;
  bool bad = false;
  for (int c = lane; c < chunks; c += 64) {
    const float x = part[c].max;
    bad = bad || x != x;
    m = fmaxf(m, x);
  }
  RowDist r;
  r.max = wave_max(m);
  r.usable = !__any(bad) && r.max > kNegInf;
  double s = 0;
  int arg = 0x7fffffff;
  if (r.usable)
    for (int c = lane; c < chunks; c += 64) {
      const float x = part[c].max;
      if (x > kNegInf) s += part[c].sum * exp_neg(((double)x - (double)r.max) * it);
      if (x == r.max) arg = min(arg, part[c].arg);
    }
  r.sum = wave_sum_d(s);
  for (int off = 32; off > 0; off >>= 1) arg = min(arg, __shfl_xor(arg, off, 64));
  r.arg = arg;
  return r;
}
__device__ __forceinline__ double prob(float x, const RowDist& r, double it) {
  return x > kNegInf ? exp_neg(((double)x - (double)r.max) * it) / r.sum : 0.0;
}
__device__ __forceinline__ double weight(float x, const RowDist& r, double it, double inv_sum) {
  return x > kNegInf ? exp_neg(((double)x - (double)r.max) * it) * inv_sum : 0.0;
}

// Sum over a chunk of max(p - a q, 0), valid in thread 0.
template <typename T>
__device__ __forceinline__ double residual_sum(const DraftParams& p, int row, int chunk, const RowDist& tp, const RowDist& tq, double a,
                                               double it, double* s_sum) {
  const DraftShape& d = p.shape;
  const int tid = threadIdx.x;
  ChunkOf<T> c;
  double sum = 0;
  const double ip = 1.0 / tp.sum, iq = a / tq.sum;
  // the two rows may lie differently on 16-byte boundaries: entries are taken where the target's lie
  c.init((const T*)p.target + (int64_t)row * d.vocab, d.vocab, chunk, tid);
  const T* q = (const T*)p.draft + (int64_t)row * d.vocab;
  const bool alike = ((reinterpret_cast<uintptr_t>(q) ^ reinterpret_cast<uintptr_t>(c.row)) & 15) == 0;
  ChunkOf<T> cq = c;
  cq.row = q;
  for (int u = 0; u < kLoads<T>; ++u) {
    float x[kVec<T>], y[kVec<T>];
    c.load(u, x);
    if (alike) {
      cq.load(u, y);
    } else {
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) {
        const int64_t e = c.at(u) + i;
        y[i] = e >= 0 && e < d.vocab ? to_float(q[e]) : kNegInf;
        y[i] = y[i] == lowest<T>() ? kNegInf : y[i];
      }
    }
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) sum += fmax(weight(x[i], tp, it, ip) - weight(y[i], tq, it, iq), 0.0);
  }
  sum = wave_sum_d(sum);
  __syncthreads();
  if ((tid & 63) == 0) s_sum[tid >> 6] = sum;
  __syncthreads();
  sum = 0;
  for (int w = 0; w < kWavesD; ++w) sum += s_sum[w];
  return sum;
}

// Z after child j is rejected, the chunk's share: for children of rank `round` that have a
// sibling behind them.
template <typename T>
__global__ __launch_bounds__(kThreads) void draft_residual_kernel(DraftParams p, int round) {
  __shared__ double s_sum[kWavesD];
  const DraftShape& d = p.shape;
  const int chunk = blockIdx.x, s = blockIdx.y / d.nodes, j = blockIdx.y - s * d.nodes, lane = threadIdx.x & 63;
  if (greedy(p.temperature, s)) return;
  const TreeOf t = tree_of(d, p.parents, p.count, s, lane);
  if (j >= t.count) return;
  const int up = __builtin_amdgcn_readlane(t.up, j);
  if (up < 0 || __builtin_amdgcn_readlane(t.rank, j) != round) return;
  const uint64_t kids = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(t.kids >> 32), up) << 32 |
                        (uint32_t)__builtin_amdgcn_readlane((int)t.kids, up);
  if ((kids >> j) == 1) return;  // the last
  const double it = inv_temp(p.temperature, s);
  const int row = s * d.nodes + up;
  const int64_t rows = (int64_t)d.n * d.nodes;
  const RowDist tp = row_dist(p.part + (int64_t)row * d.chunks, d.chunks, it, lane);
  const RowDist tq = row_dist(p.part + (rows + row) * d.chunks, d.chunks, it, lane);
  if (!tp.usable || !tq.usable) return;
  double a = 1.0;
  for (uint64_t m = kids & ((1ull << j) - 1); m; m &= m - 1) {  // the siblings rejected ahead of it
    const int64_t at = (int64_t)s * d.nodes + __ffsll((unsigned long long)m) - 1;
    double z = 0;
    for (int c = lane; c < d.chunks; c += 64) z += p.left[at * d.chunks + c];
    a += wave_sum_d(z);
  }
  const double sum = residual_sum<T>(p, row, chunk, tp, tq, a, it, s_sum);
  if (threadIdx.x == 0) p.left[(int64_t)blockIdx.y * d.chunks + chunk] = sum;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void draft_walk_kernel(DraftParams p) {
  __shared__ RowDist s_p[kTreeNodes], s_q[kTreeNodes];
  __shared__ double s_py[kTreeNodes], s_qy[kTreeNodes], s_left[kTreeNodes], s_sum[kWavesD];
  __shared__ float s_u[kTreeNodes], s_logp[kTreeNodes];
  __shared__ int s_tok[kTreeNodes], s_up[kTreeNodes], s_path[kTreeNodes];
  __shared__ DraftEnd s_end;
  const DraftShape& d = p.shape;
  const int s = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const TreeOf t = tree_of(d, p.parents, p.count, s, lane);
  const int n = t.count;
  const int64_t row0 = (int64_t)s * d.nodes, rows = (int64_t)d.n * d.nodes;
  if (n == 0) {
    if (chunk == 0 && tid < d.nodes) {
      p.out_tokens[row0 + tid] = p.out_path[row0 + tid] = -1;
      p.out_logp[row0 + tid] = 0.f;
    }
    if (chunk == 0 && tid == 0) {
      p.out_count[s] = 0;
      p.end[s].node = -1;
    }
    return;
  }
  const bool argmax = greedy(p.temperature, s), sampled = p.draft != nullptr && !argmax;
  const double it = inv_temp(p.temperature, s);
  for (int i = wave; i < n; i += kWavesD) {
    const RowDist r = row_dist(p.part + (row0 + i) * d.chunks, d.chunks, it, lane);
    const uint64_t kids = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(t.kids >> 32), i) << 32 |
                          (uint32_t)__builtin_amdgcn_readlane((int)t.kids, i);
    RowDist q{};
    if (sampled && kids) q = row_dist(p.part + (rows + row0 + i) * d.chunks, d.chunks, it, lane);
    const int up = __builtin_amdgcn_readlane(t.up, i);
    double z = 0;
    if (sampled && up >= 0) {
      const uint64_t sib = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(t.kids >> 32), up) << 32 |
                           (uint32_t)__builtin_amdgcn_readlane((int)t.kids, up);
      if (sib >> i != 1) {
        for (int c = lane; c < d.chunks; c += 64) z += p.left[(row0 + i) * d.chunks + c];
        z = wave_sum_d(z);
      }
    }
    if (lane == 0) {
      s_p[i] = r;
      s_q[i] = q;
      s_left[i] = z;
    }
  }
  __syncthreads();
  if (tid < n) {  // (the first wave)
    const int y = p.tokens[row0 + tid];
    s_up[tid] = t.up;
    s_tok[tid] = y;
    s_u[tid] = p.u[row0 + tid];
    s_py[tid] = s_qy[tid] = 0;
    if (t.up >= 0 && y >= 0 && y < d.vocab) {
      const int64_t at = (row0 + t.up) * d.vocab + y;
      auto value = [&](const void* x) {
        const float v = to_float(((const T*)x)[at]);
        return v == lowest<T>() ? kNegInf : v;
      };
      if (s_p[t.up].usable) s_py[tid] = prob(value(p.target), s_p[t.up], it);
      if (sampled && s_q[t.up].usable) s_qy[tid] = prob(value(p.draft), s_q[t.up], it);
    }
  }
  __syncthreads();
  if (tid == 0) {
    // children of a node come behind it, so one pass over the nodes sees every step of the walk
    int at = 0, len = 1, tried = 0, last = -1;
    double Z = 1.0, a = 0.0;
    s_path[0] = 0;
    for (int j = 1; j < n; ++j) {
      if (s_up[j] != at) continue;
      const int y = s_tok[j];
      bool stays;
      double w = s_py[j];
      if (!s_p[at].usable || (sampled && !s_q[at].usable)) {
        continue;  // nothing to try it against
      } else if (argmax) {
        stays = y == s_p[at].arg;
      } else if (sampled) {
        w = fmax(w - a * s_qy[j], 0.0);
        stays = (double)s_u[j] * s_qy[j] * Z < w;
      } else {
        for (int i = at + 1; i < j; ++i)
          if (s_up[i] == at && s_tok[i] == y) w = 0;  // tried already
        stays = (double)s_u[j] * Z < w;
      }
      if (stays) {
        s_logp[len - 1] = (float)log(s_py[j]);
        s_path[len++] = j;
        at = j;
        Z = 1.0;
        a = 0.0;
        tried = 0;
        last = -1;
      } else if (!argmax) {
        ++tried;
        last = j;
        a += Z;  // (its Z: of the last one the sum is still to be formed, and not needed here)
        Z = sampled ? s_left[j] : Z - w;
      }
    }
    s_end.node = at;
    s_end.len = len;
    s_end.a = sampled && tried ? a : 0.0;
    s_end.tried = tried;
    s_end.last = last;
    s_end.max = s_p[at].max;
    s_end.sum = s_p[at].sum;
    s_end.arg = s_p[at].usable ? s_p[at].arg : -1;
    s_end.greedy = argmax;
    if (chunk == 0) {
      p.end[s] = s_end;
      p.out_count[s] = len;
    }
  }
  __syncthreads();
  if (chunk == 0 && tid < d.nodes) {
    const int len = s_end.len;
    p.out_path[row0 + tid] = tid < len ? s_path[tid] : -1;
    if (tid != len - 1) {  // (draft_sample writes the last)
      p.out_tokens[row0 + tid] = tid < len - 1 ? s_tok[s_path[tid + 1]] : -1;
      p.out_logp[row0 + tid] = tid < len - 1 ? s_logp[tid] : 0.f;
    }
  }
  if (!(s_end.a > 0)) return;
  const int at = s_end.node;
  const double sum = residual_sum<T>(p, (int)row0 + at, chunk, s_p[at], s_q[at], s_end.a, it, s_sum);
  if (tid == 0) p.ends[(int64_t)s * d.chunks + chunk] = sum;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void draft_sample_kernel(DraftParams p) {
  constexpr int PER = kDraftChunk / kVec<T> / 64;  // loads of the chunk a lane of the last search has
  __shared__ double s_w[kDraftChunk / kVec<T>];
  __shared__ double s_target, s_total;
  __shared__ int s_chunk, s_tok;
  const DraftShape& d = p.shape;
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const DraftEnd e = p.end[s];
  if (e.node < 0) return;
  const int64_t row0 = (int64_t)s * d.nodes, row = row0 + e.node;
  auto finish = [&](int y, double logp) {
    p.out_tokens[row0 + e.len - 1] = y;
    p.out_logp[row0 + e.len - 1] = (float)logp;
  };
  const double it = inv_temp(p.temperature, s);
  if (e.arg < 0) {
    if (tid == 0) finish(-1, (double)__builtin_nanf(""));
    return;
  }
  if (e.greedy) {
    if (tid == 0) finish(e.arg, -log(e.sum));
    return;
  }
  RowDist tp;
  tp.max = e.max;
  tp.sum = e.sum;
  tp.usable = true;
  const T* target = (const T*)p.target + row * d.vocab;
  const T* draft = (const T*)p.draft + (p.draft ? row * d.vocab : 0);
  bool residual = e.a > 0;
  const DraftPart* part = p.part + row * d.chunks;
  const DraftPart* qpart = p.part + ((int64_t)d.n * d.nodes + row) * d.chunks;
  const RowDist tq = residual ? row_dist(qpart, d.chunks, it, lane) : RowDist{};
  const int n = max(0, min(p.count ? p.count[s] : d.nodes, d.nodes));
  // given drafts: is y one of the tried children?
  const bool given = !residual && e.tried > 0;
  auto tried = [&](int64_t y) {
    for (int j = e.node + 1; j <= e.last && j < n; ++j)
      if ((p.parents ? p.parents[row0 + j] : j - 1) == e.node && p.tokens[row0 + j] == y) return true;
    return false;
  };
  auto entry = [&](const T* r, int64_t y) {
    const float v = to_float(r[y]);
    return v == lowest<T>() ? kNegInf : v;
  };
  if (tid == 0) {
    auto share = [&](int c) {  // of chunk c in Z
      if (residual) return p.ends[(int64_t)s * d.chunks + c];
      const float m = part[c].max;
      return m > kNegInf ? part[c].sum * exp_neg(((double)m - (double)e.max) * it) / e.sum : 0.0;
    };
    auto less = [&](int c) {  // what tried tokens take off it
      double x = 0;
      if (!given) return x;
      const int ahead = (int)((reinterpret_cast<uintptr_t>(target) / sizeof(T)) % kVec<T>);
      for (int j = e.node + 1; j <= e.last && j < n; ++j) {
        if ((p.parents ? p.parents[row0 + j] : j - 1) != e.node) continue;
        const int y = p.tokens[row0 + j];
        if (y < 0 || y >= d.vocab || (y + ahead) / kDraftChunk != c) continue;
        bool again = false;
        for (int i = e.node + 1; i < j; ++i)
          again = again || ((p.parents ? p.parents[row0 + i] : i - 1) == e.node && p.tokens[row0 + i] == y);
        if (!again) x += prob(entry(target, y), tp, it);
      }
      return x;
    };
    double total = 0;
    for (int c = 0; c < d.chunks; ++c) total += fmax(share(c) - less(c), 0.0);
    if (!(total > 0)) {  // nothing is left: from p itself
      residual = false;
      total = 0;
      for (int c = 0; c < d.chunks; ++c) total += share(c);
      s_total = -total;
    } else {
      s_total = total;
    }
    const bool whole = s_total < 0;
    const double target_sum = (double)p.u[row0] * total;
    double before = 0;
    int pick = -1;
    double ahead_of = 0;
    for (int c = 0; c < d.chunks; ++c) {
      const double x = fmax(share(c) - (whole ? 0.0 : less(c)), 0.0);
      if (x > 0) {  // (the last one that has any, should none pass)
        pick = c;
        ahead_of = before;
      }
      before += x;
      if (before > target_sum) break;
    }
    s_chunk = pick;
    s_target = target_sum - ahead_of;
  }
  __syncthreads();
  const bool whole = s_total < 0;
  if (whole) residual = false;
  const bool drop = given && !whole;
  ChunkOf<T> c;
  c.init(target, d.vocab, s_chunk, tid);
  const double ip = 1.0 / tp.sum, iq = residual ? e.a / tq.sum : 0.0;
  auto left = [&](int64_t y) {
    if (y < 0 || y >= d.vocab) return 0.0;
    const double w = weight(entry(target, y), tp, it, ip);
    if (residual) return fmax(w - weight(entry(draft, y), tq, it, iq), 0.0);
    return drop && tried(y) ? 0.0 : w;
  };
  for (int u = 0; u < kLoads<T>; ++u) {
    double sum = 0;
    for (int i = 0; i < kVec<T>; ++i) sum += left(c.at(u) + i);
    s_w[u * kThreads + tid] = sum;
  }
  __syncthreads();
  if (tid >= 64) return;
  // one wave: which load, then which entry
  double mine = 0;
  for (int i = 0; i < PER; ++i) mine += s_w[lane * PER + i];
  double upto = mine;
  for (int off = 1; off < 64; off <<= 1) {
    const double y = __shfl_up(upto, off, 64);
    if (lane >= off) upto += y;
  }
  const double want = s_target;
  const uint64_t past = __ballot(upto > want && mine > 0), some = __ballot(mine > 0);
  const int who = past ? __ffsll((unsigned long long)past) - 1 : some ? 63 - __clzll((long long)some) : 0;
  if (lane != who) return;
  double at = upto - mine;
  const int64_t first = c.first - (int64_t)tid * kVec<T>;  // the chunk's first entry
  int64_t best = -1;
  for (int i = lane * PER; i < lane * PER + PER; ++i) {
    const bool here = at + s_w[i] > want;
    if (s_w[i] > 0) {
      double run = at;
      for (int v = 0; v < kVec<T>; ++v) {
        const int64_t y = first + (int64_t)i * kVec<T> + v;
        const double w = left(y);
        run += w;
        if (w > 0) {
          best = y;
          if (here && run > want) break;
        }
      }
    }
    if (here) break;
    at += s_w[i];
  }
  finish((int)best, best >= 0 ? ((double)entry(target, best) - (double)tp.max) * it - log(tp.sum) : (double)__builtin_nanf(""));
}

template <typename T>
hipError_t launch_draft_t(const DraftParams& p, hipStream_t s) {
  const DraftShape& d = p.shape;
  hipError_t e;
  {
    TimingScope t("pp_verify_draft_rows", s);
    hipLaunchKernelGGL((draft_rows_kernel<T>), dim3(d.chunks, d.n * d.nodes, p.draft ? 2 : 1), dim3(kThreads), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  for (int round = 0; p.draft && round + 1 < d.max_children; ++round) {
    TimingScope t("pp_verify_draft_residual", s);
    hipLaunchKernelGGL((draft_residual_kernel<T>), dim3(d.chunks, d.n * d.nodes), dim3(kThreads), 0, s, p, round);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  {
    TimingScope t("pp_verify_draft_walk", s);
    hipLaunchKernelGGL((draft_walk_kernel<T>), dim3(p.draft ? d.chunks : 1, d.n), dim3(kThreads), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  TimingScope t("pp_verify_draft_sample", s);
  hipLaunchKernelGGL((draft_sample_kernel<T>), dim3(d.n), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify_draft(const DraftParams& p, int dtype, hipStream_t s) {
  return dtype == kBF16 ? launch_draft_t<uint16_t>(p, s) : launch_draft_t<float>(p, s);
}

}  // namespace pp
