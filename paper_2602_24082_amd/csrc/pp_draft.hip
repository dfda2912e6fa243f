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
template <typename T>
constexpr uint32_t kInfBits = sizeof(T) == 2 ? 0x7f80u : 0x7f800000u;

// 2^t for t <= 0 in 64 bits: 2^n by the exponent's bits, 2^f, |f| <= 1/2, by the polynomial of
// degree 9 through Chebyshev's points, good to 2e-14 of it (degree 14 of the series takes five
// more multiplications).  n comes out of the low bits of t + 1.5 2^52.  Below 2^-1000, and for
// -inf and NaN, 2^-1000.
constexpr double kTiny = -1000.0;
__device__ __forceinline__ double exp2_neg(double t) {
  t = fmax(t, kTiny);
  const double u = t + 6755399441055744.0;
  const double f = t - (u - 6755399441055744.0);
  double s = 1.0205757125041537e-07;
  s = fma(s, f, 1.325968083523609e-06);
  s = fma(s, f, 1.5252674538194317e-05);
  s = fma(s, f, 0.00015403433618713555);
  s = fma(s, f, 0.001333355819593412);
  s = fma(s, f, 0.009618129194074796);
  s = fma(s, f, 0.05550410866470368);
  s = fma(s, f, 0.2402265069563986);
  s = fma(s, f, 0.6931471805599446);
  s = fma(s, f, 1.0000000000000135);
  return __hiloint2double(__double2hiint(s) + (__double2loint(u) << 20), __double2loint(s));
}

// A thread's entries of one chunk of a row: load u holds entries at(u) .. + kVec - 1, -inf
// outside the row.  Loads lie on the row's 16-byte boundaries; those that reach over an end of
// the row are taken entry by entry.
template <typename T>
struct ChunkOf {
  typedef T Raw __attribute__((ext_vector_type(kVec<T>)));
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
  __device__ __forceinline__ Raw load(int u) const {
    const int64_t e = at(u);
    if (e >= 0 && e + kVec<T> <= vocab) return *reinterpret_cast<const Raw*>(row + e);
    Raw x;
    const T none = sizeof(T) == 2 ? (T)0xff80 : (T)kNegInf;
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) x[i] = e + i >= 0 && e + i < vocab ? row[e + i] : none;
    return x;
  }
};

// The largest of the entries' bits without their signs: NaN and infinities lie at the top.
__device__ __forceinline__ void track_bits(ChunkOf<uint16_t>::Raw& most, const ChunkOf<uint16_t>::Raw& x) {
  most = __builtin_elementwise_max(most, x & (uint16_t)0x7fff);
}
__device__ __forceinline__ void track_bits(uint32_t& most, const ChunkOf<float>::Raw& x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
}
__device__ __forceinline__ uint32_t most_bits(const ChunkOf<uint16_t>::Raw& m) {
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) r = max(r, (uint32_t)m[i]);
  return r;
}
__device__ __forceinline__ uint32_t most_bits(uint32_t m) { return m; }
template <typename T>
struct BitsOf {
  using Type = uint32_t;
};
template <>
struct BitsOf<uint16_t> {
  using Type = ChunkOf<uint16_t>::Raw;
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

// log2(e) / T.  T is taken as at most 10^6, where masked entries still come out as 0.
__device__ __forceinline__ double inv_temp(const float* temperature, int s) {
  const double t = temperature ? (double)temperature[s] : 1.0;
  return 1.4426950408889634 / (t > 0 ? fmin(t, 1e6) : 1.0);
}
__device__ __forceinline__ bool greedy(const float* temperature, int s) { return temperature && !(temperature[s] > 0); }

template <typename T>
__global__ __launch_bounds__(kThreads) void draft_rows_kernel(DraftParams p) {
  __shared__ float s_m[kWavesD];
  __shared__ int s_arg[kWavesD], s_bad[kWavesD];
  __shared__ double s_sum[kWavesD];
  const DraftShape& d = p.shape;
  const int row = blockIdx.y, chunk = blockIdx.x, s = row / d.nodes, node = row - s * d.nodes;
  const bool is_draft = blockIdx.z != 0, argmax = greedy(p.temperature, s);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = max(0, min(p.count ? p.count[s] : d.nodes, d.nodes));
  if (node >= n) return;
  if (is_draft) {
    if (argmax) return;
    bool kid = false;  // only nodes with children have drafts
    for (int j = node + 1 + lane; j < n; j += 64)
      kid = kid || (p.parents ? p.parents[(int64_t)s * d.nodes + j] == node : j == node + 1);
    if (!__any(kid)) return;
  }
  ChunkOf<T> c;
  c.init((const T*)(is_draft ? p.draft : p.target) + (int64_t)row * d.vocab, d.vocab, chunk, tid);
  typename ChunkOf<T>::Raw x[kLoads<T>];
#pragma unroll
  for (int u = 0; u < kLoads<T>; ++u) x[u] = c.load(u);
  float m = kNegInf;
  typename BitsOf<T>::Type bits{};
#pragma unroll
  for (int u = 0; u < kLoads<T>; ++u) {
    track_bits(bits, x[u]);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) m = fmaxf(m, to_float(x[u][i]));
  }
  m = wave_max(m);
  const bool nan = __any(most_bits(bits) > kInfBits<T>);
  if (lane == 0) {
    s_m[wave] = m;
    s_bad[wave] = nan;
  }
  __syncthreads();
  float top = kNegInf;
  bool bad = false;
#pragma unroll
  for (int w = 0; w < kWavesD; ++w) {
    top = fmaxf(top, s_m[w]);
    bad = bad || s_bad[w];
  }
  bad = bad || top == -kNegInf;
  const double a = inv_temp(p.temperature, s), b = -(double)top * a;
  double sum = 0;
  int arg = 0x7fffffff;
  if (top > lowest<T>() && !bad) {
#pragma unroll
    for (int u = 0; u < kLoads<T>; ++u)
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) sum += exp2_neg(fma((double)to_float(x[u][i]), a, b));
    sum = wave_sum_d(sum);
    if (argmax) {
#pragma unroll
      for (int u = 0; u < kLoads<T>; ++u)
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i)
          if (to_float(x[u][i]) == top) arg = min(arg, (int)(c.at(u) + i));
      for (int off = 32; off > 0; off >>= 1) arg = min(arg, __shfl_xor(arg, off, 64));
    }
  }
  if (lane == 0) {
    s_sum[wave] = sum;
    s_arg[wave] = arg;
  }
  __syncthreads();
  if (tid == 0) {
    DraftPart out;
    out.sum = 0;
    out.arg = 0x7fffffff;
    for (int w = 0; w < kWavesD; ++w) {
      out.sum += s_sum[w];
      out.arg = min(out.arg, s_arg[w]);
    }
    out.max = bad ? __builtin_nanf("") : top > lowest<T>() ? top : kNegInf;
    p.part[((int64_t)blockIdx.z * d.n * d.nodes + row) * d.chunks + chunk] = out;
  }
}

// A row's distribution, 2^(a x + b) / sum, a = log2(e) / T.
struct RowDist {
  double a, b, sum;
  float max;
  int arg;
  bool usable;
  // e^((x - max) / T); 0 where masked (or below 2^-999)
  __device__ __forceinline__ double raw(float x) const {
    const double t = fma((double)x, a, b);
    return t > kTiny + 1 ? exp2_neg(t) : 0.0;
  }
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
  r.a = it;
  r.b = -(double)r.max * it;
  double s = 0;
  int arg = 0x7fffffff;
  if (r.usable)
    for (int c = lane; c < chunks; c += 64) {
      const float x = part[c].max;
      if (x > kNegInf) s += part[c].sum * r.raw(x);
      if (x == r.max) arg = min(arg, part[c].arg);
    }
  r.sum = wave_sum_d(s);
  for (int off = 32; off > 0; off >>= 1) arg = min(arg, __shfl_xor(arg, off, 64));
  r.arg = arg;
  return r;
}

// What is left of a row's distribution: max(p - a q, 0), or p where there is no q.
template <typename T>
struct LeftOf {
  ChunkOf<T> c;   // the target's row
  const T* q;     // or null
  RowDist tp, tq;
  double ip, iq;  // 1 / sum, a / sum
  bool alike;     // the rows lie alike on 16-byte boundaries

  __device__ __forceinline__ void init(const DraftParams& p, int64_t row, int chunk, const RowDist& p_, const RowDist& q_, double a) {
    tp = p_;
    tq = q_;
    c.init((const T*)p.target + row * p.shape.vocab, p.shape.vocab, chunk, threadIdx.x);
    q = a > 0 ? (const T*)p.draft + row * p.shape.vocab : nullptr;
    ip = 1.0 / tp.sum;
    iq = a > 0 ? a / tq.sum : 0.0;
    alike = ((reinterpret_cast<uintptr_t>(q) ^ reinterpret_cast<uintptr_t>(c.row)) & 15) == 0;
  }
  __device__ __forceinline__ double of(float x, float y) const {
    const double w = tp.raw(x) * ip;
    return q ? fmax(fma(-tq.raw(y), iq, w), 0.0) : w;
  }
  // weights of load u's entries
  __device__ __forceinline__ void load(int u, double (&w)[kVec<T>]) const {
    const typename ChunkOf<T>::Raw x = c.load(u);
    typename ChunkOf<T>::Raw y = x;
    if (q) {
      if (alike) {
        ChunkOf<T> cq = c;
        cq.row = q;
        y = cq.load(u);
      } else {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) {
          const int64_t e = c.at(u) + i;
          if (e >= 0 && e < c.vocab) y[i] = q[e];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) w[i] = of(to_float(x[i]), to_float(y[i]));
  }
};

// Sum over a chunk of max(p - a q, 0), valid in every thread.
template <typename T>
__device__ __forceinline__ double residual_sum(const DraftParams& p, int64_t row, int chunk, const RowDist& tp, const RowDist& tq,
                                               double a, double* s_sum) {
  LeftOf<T> left;
  left.init(p, row, chunk, tp, tq, a);
  double sum = 0;
#pragma unroll 2
  for (int u = 0; u < kLoads<T>; ++u) {
    double w[kVec<T>];
    left.load(u, w);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) sum += w[i];
  }
  sum = wave_sum_d(sum);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
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
  const double sum = residual_sum<T>(p, row, chunk, tp, tq, a, s_sum);
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
      if (s_p[t.up].usable) s_py[tid] = s_p[t.up].raw(to_float(((const T*)p.target)[at])) / s_p[t.up].sum;
      if (sampled && s_q[t.up].usable) s_qy[tid] = s_q[t.up].raw(to_float(((const T*)p.draft)[at])) / s_q[t.up].sum;
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
  const double sum = residual_sum<T>(p, row0 + at, chunk, s_p[at], s_q[at], s_end.a, s_sum);
  if (tid == 0) p.ends[(int64_t)s * d.chunks + chunk] = sum;
}

// The first lane whose running sum passes `want`, or the last that adds anything; `before`: the
// sum ahead of it.  -1: no lane adds anything.  `upto`: the lane's running sum.
__device__ __forceinline__ int pass_lane(double mine, double start, double want, int lane, double& before, bool& passed) {
  double upto = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double y = __shfl_up(upto, off, 64);
    if (lane >= off) upto += y;
  }
  upto += start;
  const uint64_t past = __ballot(upto > want && mine > 0), some = __ballot(mine > 0);
  passed = past != 0;
  const int who = past ? __ffsll((unsigned long long)past) - 1 : some ? 63 - __clzll((long long)some) : -1;
  before = who > 0 ? __shfl(upto, who - 1, 64) : start;
  return who;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void draft_sample_kernel(DraftParams p) {
  constexpr int VPC = kDraftChunk / kVec<T>, PER = VPC / 64;  // loads of a chunk, and a lane's
  __shared__ double s_w[VPC];
  __shared__ double s_want;
  __shared__ int s_chunk, s_whole, s_gone[kTreeNodes], s_n_gone;
  const DraftShape& d = p.shape;
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const DraftEnd e = p.end[s];
  if (e.node < 0) return;
  const int64_t row0 = (int64_t)s * d.nodes, row = row0 + e.node;
  auto finish = [&](int64_t y, double logp) {
    p.out_tokens[row0 + e.len - 1] = (int32_t)y;
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
  RowDist tp{};
  tp.max = e.max;
  tp.sum = e.sum;
  tp.a = it;
  tp.b = -(double)e.max * it;
  bool residual = e.a > 0;
  const DraftPart* part = p.part + row * d.chunks;
  RowDist tq{};
  if (residual) tq = row_dist(p.part + ((int64_t)d.n * d.nodes + row) * d.chunks, d.chunks, it, lane);
  const T* target = (const T*)p.target + row * d.vocab;
  if (tid < 64) {
    // given drafts: the tokens of the children that were tried are gone, a lane each
    double gone = 0;
    int gone_at = -1, y = -1;
    if (!residual && e.tried > 0) {
      const TreeOf t = tree_of(d, p.parents, p.count, s, lane);
      bool is = t.up == e.node && lane <= e.last;
      y = is ? p.tokens[row0 + lane] : -1;
      is = is && y >= 0 && y < d.vocab;
      for (uint64_t m = __ballot(is); m; m &= m - 1) {
        const int j = __ffsll((unsigned long long)m) - 1;
        if (lane > j && __builtin_amdgcn_readlane(y, j) == y) is = false;  // the same again
      }
      if (is) {
        const int ahead = (int)((reinterpret_cast<uintptr_t>(target) / sizeof(T)) % kVec<T>);
        gone_at = (y + ahead) / kDraftChunk;
        gone = tp.raw(to_float(target[y])) / tp.sum;
      }
    }
    uint64_t takes = __ballot(gone_at >= 0);
    auto share = [&](int c) {  // of chunk c in what is left
      const bool is = c < d.chunks;
      if (residual) return is ? p.ends[(int64_t)s * d.chunks + c] : 0.0;
      double x = is && part[c].max > kNegInf ? part[c].sum * tp.raw(part[c].max) / tp.sum : 0.0;
      for (uint64_t m = takes; m; m &= m - 1) {  // (all lanes: they read each other's)
        const int j = __ffsll((unsigned long long)m) - 1;
        const double off = __shfl(gone, j, 64);
        if (__shfl(gone_at, j, 64) == c) x -= off;
      }
      return fmax(x, 0.0);
    };
    double total = 0;
    for (int c0 = 0; c0 < d.chunks; c0 += 64) total += share(c0 + lane);
    total = wave_sum_d(total);
    if (!(total > 0)) {  // nothing is left: from p itself
      residual = false;
      takes = 0;
      total = 0;
      for (int c0 = 0; c0 < d.chunks; c0 += 64) total += share(c0 + lane);
      total = wave_sum_d(total);
    }
    const double want = (double)p.u[row0] * total;
    double start = 0, ahead = 0;
    int pick = -1;
    for (int c0 = 0; c0 < d.chunks; c0 += 64) {
      const double x = share(c0 + lane);
      double before;
      bool passed;
      const int who = pass_lane(x, start, want, lane, before, passed);
      if (who >= 0) {  // (the last chunk that has any, should none pass)
        pick = c0 + who;
        ahead = before;
      }
      if (passed) break;
      start += wave_sum_d(x);
    }
    const bool here = gone_at == pick && (takes >> lane & 1);
    const uint64_t in_chunk = __ballot(here);
    if (here) s_gone[__popcll(in_chunk & ((1ull << lane) - 1))] = y;
    if (lane == 0) {
      s_n_gone = __popcll(in_chunk);
      s_chunk = pick;
      s_want = want - ahead;
      s_whole = !residual;
    }
  }
  __syncthreads();
  LeftOf<T> left;
  left.init(p, row, s_chunk, tp, tq, s_whole ? 0.0 : e.a);
  const int n_gone = s_n_gone;
  auto is_gone = [&](int64_t y) {
    for (int i = 0; i < n_gone; ++i)
      if (s_gone[i] == y) return true;
    return false;
  };
  for (int u = 0; u < kLoads<T>; ++u) {
    double w[kVec<T>], sum = 0;
    left.load(u, w);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) sum += n_gone && is_gone(left.c.at(u) + i) ? 0.0 : w[i];
    s_w[u * kThreads + tid] = sum;
  }
  __syncthreads();
  if (tid >= 64) return;
  // one wave: a lane's loads, then the load, then the entry
  double mine = 0, before;
  bool passed;
  for (int i = 0; i < PER; ++i) mine += s_w[lane * PER + i];
  const double want = s_want;
  const int who = pass_lane(mine, 0.0, want, lane, before, passed);
  int load = 0;
  double ahead = before;
  if (who >= 0) {
    double run = before;
    for (int i = who * PER; i < who * PER + PER; ++i) {
      const double w = s_w[i];
      if (w > 0) {  // (the last one that has any, should none pass)
        load = i;
        ahead = run;
      }
      run += w;
      if (w > 0 && run > want) break;
    }
  }
  const int64_t y = left.c.first - (int64_t)tid * kVec<T> + (int64_t)load * kVec<T> + lane;  // (first: the thread's)
  double w = 0;
  if (who >= 0 && lane < kVec<T> && y >= 0 && y < d.vocab && !(n_gone && is_gone(y)))
    w = left.of(to_float(left.c.row[y]), left.q ? to_float(left.q[y]) : 0.f);
  const int last = pass_lane(w, ahead, want, lane, before, passed);
  if (last < 0) {
    if (lane == 0) finish(-1, (double)__builtin_nanf(""));
  } else if (lane == last) {
    finish(y, fma((double)to_float(left.c.row[y]), tp.a, tp.b) * 0.6931471805599453 - log(tp.sum));
  }
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
