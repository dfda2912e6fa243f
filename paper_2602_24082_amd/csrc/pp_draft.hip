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
//   draft_rows      a wave for 2048 entries of a row: maximum, sum, where the maximum is
//   draft_edges     a workgroup a sequence: rows' sums joined, p and q of every drafted token,
//                   and which nodes can be reached at all: a first child's fate is known here
//   draft_residual  Z after a rejected child that has siblings behind it and can be reached; one
//                   launch for each place among siblings
//   draft_end       a workgroup for 2048 entries of w at the node where the walk ends, which each
//                   finds by walking again (a few steps in registers); the last of a sequence's
//                   searches the entry at which the running sum passes
//
// Probabilities are 64 bits throughout: numbers are compared with given ones, and a running
// sum over 10^5 entries in 32 bits passes a number u elsewhere in one case of some hundred.
// Bound by vector issue: 19 instructions an entry, nine 64-bit and three others of them for its exponential
// and the sum.  33 million entries, 66 MB of logits, take 24 to 27 us: the compute units hold waves for some
// 20 of them, and their vector units are busy for 81% of that (LDS, with its conflicts, for 28%).

#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "pp_device.h"
#include "pp_sample.h"

namespace pp {
namespace {

constexpr int kThreads = 256;
constexpr int kWavesD = kThreads / 64;

template <typename T>
constexpr int kVec = 16 / sizeof(T);  // entries of a 16-byte load
template <typename T, int THREADS>
constexpr int kLoads = kDraftChunk / (THREADS * kVec<T>);  // a thread's of a chunk

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

// 2^(i / 256), in LDS.  Their upper words are lower by i << 12: k << 12 on top makes entry k & 255
// 2^(k / 256).
constexpr int kRoots = 256;
struct RootTable {
  double of[kRoots];
};
constexpr RootTable root_table() {
  RootTable t{};
  for (int i = 0; i < kRoots; ++i) {
    const double x = i * (0.6931471805599453 / kRoots);
    double sum = 0.0;
    for (int n = 18; n > 0; --n) sum = (1.0 + sum) * x / n;  // e^x - 1
    t.of[i] = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, 1.0 + sum) - ((uint64_t)i << 44));
  }
  return t;
}
__device__ const RootTable kRootTable = root_table();
__device__ __forceinline__ double* exp2_roots() {
  __shared__ double roots[kRoots];
  return roots;
}
__device__ __forceinline__ void fill_roots() {
  if (threadIdx.x < kRoots) exp2_roots()[threadIdx.x] = kRootTable.of[threadIdx.x];
  lds_barrier();
}
// 2^t for t <= 0 in 64 bits: with k the whole number next to 256 t and f = t - k / 256,
// |f| <= 1/512, 2^(k / 256) from the table, 2^f by the polynomial of degree 3 through 1 at 0 and
// Chebyshev's points, good to 3.5e-14 of it (and to ln 2 times what t is off by).  k comes out of the
// low bits of t + 1.5 2^44.  Below 2^-1000, and for -inf, 2^-1000; without CLAMP t has to be above.
// NaN stays.
constexpr double kTiny = -1000.0;
struct Exp2 {
  double root, p;  // whose product it is
};
template <bool CLAMP = true>
__device__ __forceinline__ Exp2 exp2_parts(double t) {
  constexpr double shift = 1.5 * (1ull << 44);
  if (CLAMP && t < kTiny) t = kTiny;
  const double u = t + shift;
  const int k = __double2loint(u);
  const double base = exp2_roots()[k & (kRoots - 1)];
  const double f = t - (u - shift);
  Exp2 x;
  x.root = __hiloint2double(__double2hiint(base) + (k << 12), __double2loint(base));
  x.p = fma(fma(fma(0.05550411247958329, f, 0.24022653447679007), f, 0.6931471805599453), f, 1.0);
  return x;
}
template <bool CLAMP = true>
__device__ __forceinline__ double exp2_neg(double t) {
  const Exp2 x = exp2_parts<CLAMP>(t);
  return x.root * x.p;
}

template <typename T>
using RawOf = T __attribute__((ext_vector_type(kVec<T>)));

// A thread's entries of one chunk of a row, of THREADS threads: load u holds entries at(u) .. + kVec - 1, -inf
// outside the row.  Loads lie on the row's 16-byte boundaries; those that reach over an end of
// the row are taken entry by entry.
template <typename T, int THREADS>
struct ChunkOf {
  using Raw = RawOf<T>;
  const T* row;
  int64_t first;  // entry of the thread's first load
  int vocab, ahead;  // ahead: of the row, from a 16-byte boundary on

  __device__ __forceinline__ void init(const T* r, int v, int chunk, int thread) {
    row = r;
    vocab = v;
    ahead = (int)((reinterpret_cast<uintptr_t>(r) / sizeof(T)) % kVec<T>);
    first = (int64_t)chunk * kDraftChunk + thread * kVec<T> - ahead;
  }
  __device__ __forceinline__ int64_t at(int u) const { return first + u * (THREADS * kVec<T>); }
  // the whole chunk lies in the row
  __device__ __forceinline__ bool inside(int chunk) const {
    const int64_t e = (int64_t)chunk * kDraftChunk - ahead;
    return e >= 0 && e + kDraftChunk <= vocab;
  }
  __device__ __forceinline__ Raw load_inside(int u) const { return *reinterpret_cast<const Raw*>(row + at(u)); }
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

__device__ __forceinline__ double lane_d(double x, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane), __builtin_amdgcn_readlane(__double2loint(x), lane));
}
__device__ __forceinline__ float lane_f(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(x), lane));
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t x, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}

// Running sums over the wave's lanes, in registers (DPP: lanes 1, 2, 4, 8 to the left within rows
// of 16, then the rows' last lanes), a sixth of the time of exchanges through LDS.
template <int CTRL, int ROWS>
__device__ __forceinline__ double add_moved(double x) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, ROWS, 0xf, false);
  return x + __hiloint2double(hi, lo);
}
__device__ __forceinline__ double wave_scan_d(double x) {
  x = add_moved<0x111, 0xf>(x);
  x = add_moved<0x112, 0xf>(x);
  x = add_moved<0x114, 0xf>(x);
  x = add_moved<0x118, 0xf>(x);
  x = add_moved<0x142, 0xa>(x);
  return add_moved<0x143, 0xc>(x);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float max_moved(float x) {
  const int own = (int)__float_as_uint(x);
  return fmaxf(x, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(own, own, CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float wave_max_f(float x) {
  x = max_moved<0x111, 0xf>(x);
  x = max_moved<0x112, 0xf>(x);
  x = max_moved<0x114, 0xf>(x);
  x = max_moved<0x118, 0xf>(x);
  x = max_moved<0x142, 0xa>(x);
  return lane_f(max_moved<0x143, 0xc>(x), 63);
}
__device__ __forceinline__ double wave_sum_d(double x) { return lane_d(wave_scan_d(x), 63); }

// A sequence's tree: lane l of a wave looks at node l.
struct TreeOf {
  int count;      // nodes
  uint64_t kids;  // lane's children, at most max_children of them
  int up, rank;   // the lane's parent (-1: none, or never reached) and its place among that one's children
};
__device__ __forceinline__ TreeOf tree_of(const DraftShape& d, const int32_t* parents, const int32_t* count, int s, int lane) {
  TreeOf t;
  int up = !parents ? lane - 1 : lane < d.nodes ? parents[(int64_t)s * d.nodes + lane] : -1;  // (on its way with the count)
  t.count = max(0, min(count ? count[s] : d.nodes, d.nodes));
  if (lane == 0 || lane >= t.count || up >= lane) up = -1;
  t.kids = 0;
  t.rank = 0;
  for (int j = 1; j < t.count; ++j) {
    const int uj = __builtin_amdgcn_readlane(up, j);
    if (uj < 0) continue;
    const int before = __popcll(lane_u64(t.kids, uj));
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

// The greatest of a wave's entries (NaN left out), and a number that none of the lane's is below.
// As whole numbers bf16 ones rise where they are positive and fall where they are negative, so two
// entries at a time can be compared: with sign the greatest of those that have none, if there is one, and
// without it the lowest of those that have one.
__device__ __forceinline__ float extremes(const RawOf<uint16_t> (&x)[4], float& low) {
  typedef int16_t Signed __attribute__((ext_vector_type(8)));
  typedef int16_t Two __attribute__((ext_vector_type(2)));
  typedef uint16_t UTwo __attribute__((ext_vector_type(2)));
  typedef uint16_t UFour __attribute__((ext_vector_type(4)));
  typedef int16_t Four __attribute__((ext_vector_type(4)));
  Signed hi = __builtin_bit_cast(Signed, x[0]);
  RawOf<uint16_t> lo = x[0];
#pragma unroll
  for (int u = 1; u < 4; ++u) {
    hi = __builtin_elementwise_max(hi, __builtin_bit_cast(Signed, x[u]));
    lo = __builtin_elementwise_max(lo, x[u]);
  }
  const Four h4 = __builtin_elementwise_max(hi.lo, hi.hi);
  const UFour l4 = __builtin_elementwise_max(lo.lo, lo.hi);
  const Two h2 = __builtin_elementwise_max(h4.lo, h4.hi);
  const UTwo l2 = __builtin_elementwise_max(l4.lo, l4.hi);
  const int h = max((int)h2.x, (int)h2.y);
  const uint32_t l = max((uint32_t)l2.x, (uint32_t)l2.y);
  low = l & 0x8000u ? bf16_bits_to_f32((uint16_t)l) : 0.f;
  if (wave_any(h >= 0)) return wave_max_f(h >= 0 ? bf16_bits_to_f32((uint16_t)h) : kNegInf);
  uint32_t least = 0xffffu;  // all have a sign (or are NaN)
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) least = min(least, (uint32_t)x[u][i]);
  return wave_max_f(least & 0x8000u ? bf16_bits_to_f32((uint16_t)least) : kNegInf);
}
__device__ __forceinline__ float extremes(const RawOf<float> (&x)[8], float& low) {
  float m = kNegInf;
  low = -kNegInf;
#pragma unroll
  for (int u = 0; u < 8; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m = fmaxf(m, x[u][i]);
      low = fminf(low, x[u][i]);
    }
  return wave_max_f(m);
}

// A wave a chunk.
template <typename T>
__global__ __launch_bounds__(kThreads) void draft_rows_kernel(DraftParams p) {
  constexpr int L = kLoads<T, 64>;
  const DraftShape& d = p.shape;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.y, chunk = blockIdx.x * kWavesD + wave, s = row / d.nodes, node = row - s * d.nodes;
  const bool is_draft = blockIdx.z != 0, argmax = greedy(p.temperature, s);
  const int n = max(0, min(p.count ? p.count[s] : d.nodes, d.nodes));
  const double a = inv_temp(p.temperature, s);
  if (node == 0 && chunk == 0 && !is_draft && lane == 0) p.arrived[s * kOwnLine] = 0;
  if (node >= n) return;
  if (is_draft) {
    if (argmax) return;
    // only nodes with children have drafts
    const bool later = lane > node && lane < n;
    const int up = !later ? -1 : p.parents ? p.parents[(int64_t)s * d.nodes + lane] : lane - 1;
    if (!__any(up == node)) return;
  }
  ChunkOf<T, 64> c;
  c.init((const T*)(is_draft ? p.draft : p.target) + (int64_t)row * d.vocab, d.vocab, min(chunk, d.chunks - 1), lane);
  RawOf<T> x[L];
  if (c.inside(chunk)) {
#pragma unroll
    for (int u = 0; u < L; ++u) x[u] = c.load_inside(u);
  } else {
#pragma unroll
    for (int u = 0; u < L; ++u) x[u] = c.load(u);
  }
  fill_roots();
  if (chunk >= d.chunks) return;
  float low;  // none of the thread's entries is below
  const float top = extremes(x, low);
  bool bad = top == -kNegInf;  // or a NaN among them
  double sum = 0;
  int arg = 0x7fffffff;
  if (top > lowest<T>() && !bad) {
    // (x - top) a, as one operation where the rounding of top a is below 2^-45
    const double b = -(double)top * a;
    auto add_all = [&](auto careful) {
#pragma unroll
      for (int u = 0; u < L; ++u) {
        asm volatile("" : "+v"(x[u]));  // (else both loops' numbers are made ahead of them, in registers)
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) {
          const double y = (double)to_float(x[u][i]);
          const Exp2 e = careful.value ? exp2_parts<true>((y - (double)top) * a) : exp2_parts<false>(fma(y, a, b));
          sum = fma(e.root, e.p, sum);
        }
      }
    };
    if (__any(!(fma((double)low, a, b) > kTiny)) || !(fabs(b) < 256.0)) add_all(std::true_type{});
    else add_all(std::false_type{});
    sum = wave_sum_d(sum);
    bad = sum != sum;
    if (argmax) {
#pragma unroll
      for (int u = 0; u < L; ++u)
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i)
          if (to_float(x[u][i]) == top) arg = min(arg, (int)(c.at(u) + i));
      for (int off = 32; off > 0; off >>= 1) arg = min(arg, __shfl_xor(arg, off, 64));
    }
  } else {
#pragma unroll
    for (int u = 0; u < L; ++u)
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) bad = bad || to_float(x[u][i]) != to_float(x[u][i]);
    bad = __any(bad);
  }
  if (lane) return;
  DraftPart out;
  out.sum = sum;
  out.arg = arg;
  out.max = bad ? __builtin_nanf("") : top > lowest<T>() ? top : kNegInf;
  p.part[((int64_t)blockIdx.z * d.n * d.nodes + row) * d.chunks + chunk] = out;
}

// A row's distribution, 2^(a (x - max)) / sum, a = log2(e) / T.
struct RowDist {
  double a, sum;
  float max;
  int arg;
  bool usable;
  // e^((x - max) / T); 0 where masked (or below 2^-999)
  __device__ __forceinline__ double raw(float x) const {
    const double t = ((double)x - (double)max) * a;
    return t > kTiny + 1 ? exp2_neg<false>(t) : 0.0;
  }
};
__device__ __forceinline__ RowDist row_dist(const DraftRow& x, double it) {
  RowDist r;
  r.max = x.max;
  r.sum = x.sum;
  r.arg = x.arg;
  r.usable = x.arg >= 0;
  r.a = it;
  return r;
}
// The parts of a row's first 128 chunks, two a lane.
struct RowParts {
  DraftPart a, b;
  __device__ __forceinline__ void load(const DraftPart* part, int chunks, int lane) {
    a.sum = b.sum = 0;
    a.max = b.max = kNegInf;
    a.arg = b.arg = 0x7fffffff;
    if (lane < chunks) a = part[lane];
    if (lane + 64 < chunks) b = part[lane + 64];
  }
};
// By a wave, from the parts of the row's chunks.
__device__ __forceinline__ RowDist row_dist(const RowParts& first, const DraftPart* part, int chunks, double it, bool argmax, int lane) {
  float m = fmaxf(first.a.max, first.b.max);
  bool bad = first.a.max != first.a.max || first.b.max != first.b.max;
  for (int c = lane + 128; c < chunks; c += 64) {
    const float x = part[c].max;
    bad = bad || x != x;
    m = fmaxf(m, x);
  }
  RowDist r;
  r.max = wave_max_f(m);
  r.usable = !__any(bad) && r.max > kNegInf;
  r.a = it;
  r.sum = 0;
  r.arg = 0x7fffffff;
  if (!r.usable) return r;
  double s = 0;
  int arg = 0x7fffffff;
  auto add = [&](const DraftPart& x) {
    if (x.max > kNegInf) s = fma(x.sum, r.raw(x.max), s);
    if (x.max == r.max) arg = min(arg, x.arg);
  };
  add(first.a);
  add(first.b);
  for (int c = lane + 128; c < chunks; c += 64) add(part[c]);
  r.sum = wave_sum_d(s);
  r.arg = 0;
  if (argmax) {
    for (int off = 32; off > 0; off >>= 1) arg = min(arg, __shfl_xor(arg, off, 64));
    r.arg = arg;
  }
  return r;
}

// What is left of a row's distribution: max(p - a q, 0), or p where there is no q.
template <typename T>
struct LeftOf {
  static constexpr int L = kLoads<T, kThreads>;
  ChunkOf<T, kThreads> c;  // the target's row
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
  // use(load, entry of it, weight) for the thread's entries; all loads ahead
  template <typename Use>
  __device__ __forceinline__ void each(Use&& use) const {
    RawOf<T> x[L], y[L];
    ChunkOf<T, kThreads> cq = c;
    cq.row = q;
#pragma unroll
    for (int u = 0; u < L; ++u) x[u] = c.load(u);
    if (q && alike) {
#pragma unroll
      for (int u = 0; u < L; ++u) y[u] = cq.load(u);
    } else if (q) {
#pragma unroll
      for (int u = 0; u < L; ++u) {
        y[u] = x[u];
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) {
          const int64_t e = c.at(u) + i;
          if (e >= 0 && e < c.vocab) y[u][i] = q[e];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < L; ++u)
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) use(u, i, of(to_float(x[u][i]), q ? to_float(y[u][i]) : 0.f));
  }
};

// Sum over a chunk of max(p - a q, 0), valid in every thread.
template <typename T>
__device__ __forceinline__ double residual_sum(const DraftParams& p, int64_t row, int chunk, const RowDist& tp, const RowDist& tq,
                                               double a, double* s_sum) {
  LeftOf<T> left;
  left.init(p, row, chunk, tp, tq, a);
  double sum = 0;
  left.each([&](int, int, double w) { sum += w; });
  sum = wave_sum_d(sum);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = 0;
  for (int w = 0; w < kWavesD; ++w) sum += s_sum[w];
  return sum;
}

// Of a drafted token, a lane each, and the lane's own rows (lanes behind the count hold
// anything).
struct EdgeOf {
  double p, q;
  float u;
  int tok;
  DraftRow rp, rq;
};
__device__ __forceinline__ EdgeOf edge_of(const DraftParams& p, int64_t row0, int lane) {
  EdgeOf e{};
  e.tok = -1;
  if (lane < p.shape.nodes) {
    const DraftEdge x = p.edge[row0 + lane];
    e.rp = p.row[row0 + lane];
    e.rq = p.row[(int64_t)p.shape.n * p.shape.nodes + row0 + lane];
    e.p = x.p;
    e.q = x.q;
    e.u = p.u[row0 + lane];
    e.tok = p.tokens[row0 + lane];
  }
  return e;
}
__device__ __forceinline__ DraftRow lane_row(const DraftRow& r, int lane) {
  DraftRow x;
  x.sum = lane_d(r.sum, lane);
  x.max = lane_f(r.max, lane);
  x.arg = __builtin_amdgcn_readlane(r.arg, lane);
  return x;
}

// Z after a node is rejected, by a wave.
__device__ __forceinline__ double left_after(const DraftParams& p, int64_t node, int lane) {
  double z = 0;
  for (int c = lane; c < p.shape.chunks; c += 64) z += p.left[node * p.shape.chunks + c];
  return wave_sum_d(z);
}

constexpr int kEdgeThreads = 1024;  // a wave a row, as far as they reach

template <typename T>
__global__ __launch_bounds__(kEdgeThreads) void draft_edges_kernel(DraftParams p) {
  __shared__ DraftRow s_p[kTreeNodes], s_q[kTreeNodes];
  const DraftShape& d = p.shape;
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row0 = (int64_t)s * d.nodes, rows = (int64_t)d.n * d.nodes;
  // what does not wait for anything else: tokens, numbers, the parts of the wave's first row
  auto part_of = [&](int i) { return p.part + ((i & 1) * rows + row0 + (i >> 1)) * d.chunks; };
  int y = lane < d.nodes ? p.tokens[row0 + lane] : -1;
  const float u32 = lane < d.nodes ? p.u[row0 + lane] : 0.f;
  RowParts ahead;
  if (wave < 2 * d.nodes) ahead.load(part_of(wave), d.chunks, lane);
  const TreeOf t = tree_of(d, p.parents, p.count, s, lane);
  const int n = t.count;
  if (lane >= n) y = -1;
  const bool argmax = greedy(p.temperature, s), sampled = p.draft != nullptr && !argmax;
  const double it = inv_temp(p.temperature, s);
  // the drafted tokens' logits
  float xp = 0.f, xq = 0.f;
  if (tid < 64 && t.up >= 0 && y >= 0 && y < d.vocab) {
    const int64_t at = (row0 + t.up) * d.vocab + y;
    xp = to_float(((const T*)p.target)[at]);
    if (sampled) xq = to_float(((const T*)p.draft)[at]);
  }
  // the rows, each one's parts fetched ahead
  auto next = [&](int i) {  // the wave's next row from i on that is looked at
    while (i < 2 * n && (i & 1) && !(sampled && lane_u64(t.kids, i >> 1))) i += kEdgeThreads / 64;
    return i;
  };
  int i = next(wave);
  if (i != wave && i < 2 * n) ahead.load(part_of(i), d.chunks, lane);
  fill_roots();
  while (i < 2 * n) {
    const int node = i >> 1, is_q = i & 1, then = next(i + kEdgeThreads / 64);
    const RowParts mine = ahead;
    if (then < 2 * n) ahead.load(part_of(then), d.chunks, lane);
    const RowDist r = row_dist(mine, part_of(i), d.chunks, it, argmax, lane);
    i = then;
    if (lane == 0) {
      DraftRow x;
      x.sum = r.sum;
      x.max = r.max;
      x.arg = r.usable ? r.arg : -1;
      (is_q ? s_q : s_p)[node] = x;
      p.row[is_q * rows + row0 + node] = x;
    }
  }
  __syncthreads();
  if (tid >= 64) return;
  DraftEdge e{};
  bool tried = false, stays = false;  // as a first child
  if (lane < n && t.up >= 0) {
    const DraftRow rp = s_p[t.up], rq = sampled ? s_q[t.up] : rp;
    tried = rp.arg >= 0 && rq.arg >= 0;
    if (tried && y >= 0 && y < d.vocab) {
      e.p = row_dist(rp, it).raw(xp) / rp.sum;
      if (sampled) e.q = row_dist(rq, it).raw(xq) / rq.sum;
    }
    const double u = (double)u32;
    stays = tried && (sampled ? u * e.q < e.p : argmax ? y == rp.arg : u < e.p);
  }
  // a node can be reached if its edge can be taken, and its parent's, ..: a first child's if it
  // stays, another's if the first does not
  const int up = t.up;
  const uint64_t kids = __shfl(t.kids, max(up, 0), 64);
  const int first = up >= 0 ? __ffsll((unsigned long long)kids) - 1 : 0;
  const int first_stays = __shfl((int)stays, max(first, 0), 64);
  int ok = lane == 0 ? 1 : up >= 0 && tried && (t.rank == 0 ? stays : !first_stays);
  int to = up;
  for (int i = 0; i < 6; ++i) {
    const int from = max(to, 0);
    const int ok2 = __shfl(ok, from, 64), to2 = __shfl(to, from, 64);
    if (to >= 0) {
      ok &= ok2;
      to = to2;
    }
  }
  ok &= to < 0;
  const int parent_ok = __shfl(ok, max(up, 0), 64);
  e.need = up >= 0 && sampled && tried && !stays && t.rank == 0 && parent_ok && (kids >> lane) != 1;
  if (lane < n) p.edge[row0 + lane] = e;
}

// Z after a child of rank `round` is rejected that has a sibling behind it, a chunk's
// share, for every node where it may be asked for.
template <typename T>
__global__ __launch_bounds__(kThreads) void draft_residual_kernel(DraftParams p, int round) {
  __shared__ double s_sum[kWavesD];
  const DraftShape& d = p.shape;
  const int chunk = blockIdx.x, s = blockIdx.y, lane = threadIdx.x & 63;
  const int64_t row0 = (int64_t)s * d.nodes;
  const int n = max(0, min(p.count ? p.count[s] : d.nodes, d.nodes));
  uint64_t need = __ballot(lane < n && p.edge[row0 + lane].need);
  if (need == 0) return;
  const TreeOf t = tree_of(d, p.parents, p.count, s, lane);
  const EdgeOf e = edge_of(p, row0, lane);
  const double it = inv_temp(p.temperature, s);
  fill_roots();
  for (; need; need &= need - 1) {
    const int first = __ffsll((unsigned long long)need) - 1, up = __builtin_amdgcn_readlane(t.up, first);
    const uint64_t kids = lane_u64(t.kids, up);
    const int j_rank = __popcll(kids) - 1;
    if (j_rank <= round) continue;  // none, or the last
    // the siblings up to it, all rejected?
    double a = 0, Z = 1.0;
    int j = first, rank = 0;
    bool stays = false;
    for (uint64_t m = kids; m; m &= m - 1, ++rank) {
      j = __ffsll((unsigned long long)m) - 1;
      const double q = lane_d(e.q, j), w = fmax(fma(-a, q, lane_d(e.p, j)), 0.0);  // (as draft_end)
      stays = (double)lane_f(e.u, j) * q * Z < w;
      a += Z;
      if (stays || rank == round) break;
      Z = left_after(p, row0 + j, lane);
    }
    if (stays) continue;
    const RowDist tp = row_dist(lane_row(e.rp, up), it), tq = row_dist(lane_row(e.rq, up), it);
    const double sum = residual_sum<T>(p, row0 + up, chunk, tp, tq, a, s_sum);
    if (threadIdx.x == 0) p.left[(row0 + j) * d.chunks + chunk] = sum;
  }
}

// The first lane whose running sum passes `want`, or the last that adds anything; `before`: the
// sum ahead of it.  -1: no lane adds anything.  `upto`: the lane's running sum.
__device__ __forceinline__ int pass_lane(double mine, double start, double want, int lane, double& before, bool& passed) {
  const double upto = wave_scan_d(mine) + start;
  const uint64_t past = __ballot(upto > want && mine > 0), some = __ballot(mine > 0);
  passed = past != 0;
  const int who = past ? __ffsll((unsigned long long)past) - 1 : some ? 63 - __clzll((long long)some) : -1;
  before = who > 0 ? lane_d(upto, who - 1) : start;
  return who;
}

// Where to look for the next token: a chunk, what its running sum has to pass, and tokens in
// it that are gone.
struct PickOf {
  double want;
  int chunk, n_gone, gone[kTreeNodes];
};
struct Picked {
  bool mine;  // the thread that has it
  int64_t y;  // -1: nothing there
  double logp;
};
// By the workgroup: the entry of the chunk at which the running sum of what is left passes; s_w,
// s_sum: room for the entries' weights and the sums of the chunk's loads.
template <typename T>
__device__ __forceinline__ Picked pick_entry(const DraftParams& p, int64_t row, const RowDist& tp, const RowDist& tq, double a,
                                             const PickOf& pick, double* s_w, double* s_sum) {
  constexpr int VPC = kDraftChunk / kVec<T>, PER = VPC / 64, L = kLoads<T, kThreads>;  // loads of a chunk, a lane's, a thread's
  const int tid = threadIdx.x, lane = tid & 63;
  Picked out{false, -1, (double)__builtin_nanf("")};
  LeftOf<T> left;
  left.init(p, row, pick.chunk, tp, tq, a);
  const int n_gone = pick.n_gone;
  auto is_gone = [&](int64_t y) {
    for (int i = 0; i < n_gone; ++i)
      if (pick.gone[i] == y) return true;
    return false;
  };
  double sums[L] = {};
  left.each([&](int u, int i, double w) {
    if (n_gone && is_gone(left.c.at(u) + i)) w = 0.0;
    const int at = (u * kThreads + tid) * kVec<T> + i;
    s_w[at] = w;
    sums[u] += w;
  });
#pragma unroll
  for (int u = 0; u < L; ++u) s_sum[u * kThreads + tid] = sums[u];
  __syncthreads();
  if (tid >= 64) return out;
  // one wave: a lane's loads, then the load, then the entry
  double mine = 0, before;
  bool passed;
#pragma unroll
  for (int i = 0; i < PER; ++i) mine += s_sum[lane * PER + i];
  const int who = pass_lane(mine, 0.0, pick.want, lane, before, passed);
  int load = 0;
  double ahead = before;
  if (who >= 0) {
    double run = before;
    for (int i = who * PER; i < who * PER + PER; ++i) {
      const double w = s_sum[i];
      if (w > 0) {  // (the last one that has any, should none pass)
        load = i;
        ahead = run;
      }
      run += w;
      if (w > 0 && run > pick.want) break;
    }
  }
  const int64_t y = left.c.first - (int64_t)tid * kVec<T> + (int64_t)load * kVec<T> + lane;  // (first: the thread's)
  const bool entry = who >= 0 && lane < kVec<T>;
  const double w = entry ? s_w[load * kVec<T> + lane] : 0.0;
  const float x = entry && y >= 0 && y < p.shape.vocab ? to_float(left.c.row[y]) : 0.f;
  const int last = pass_lane(w, ahead, pick.want, lane, before, passed);
  out.mine = lane == max(last, 0);
  if (lane == last) {
    out.y = y;
    out.logp = ((double)x - (double)tp.max) * tp.a * 0.6931471805599453 - log(tp.sum);
  }
  return out;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void draft_end_kernel(DraftParams p) {
  __shared__ double s_w[kDraftChunk], s_sum[kDraftChunk / kVec<T>];
  __shared__ PickOf s_pick;
  __shared__ int s_whole, s_last;
  const DraftShape& d = p.shape;
  const int s = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int64_t row0 = (int64_t)s * d.nodes;
  const EdgeOf e = edge_of(p, row0, lane);
  const TreeOf t = tree_of(d, p.parents, p.count, s, lane);
  const int n = t.count;
  if (n == 0) {
    if (chunk == 0 && tid < d.nodes) {
      p.out_tokens[row0 + tid] = p.out_path[row0 + tid] = -1;
      p.out_logp[row0 + tid] = 0.f;
    }
    if (chunk == 0 && tid == 0) p.out_count[s] = 0;
    return;
  }
  const bool argmax = greedy(p.temperature, s), sampled = p.draft != nullptr && !argmax;
  const double it = inv_temp(p.temperature, s);
  fill_roots();

  // the walk, by every wave on its own
  int at = 0, len = 1, order = lane == 0 ? 0 : -1;
  double a = 0;
  uint64_t gone = 0;  // children of `at` that were tried
  for (bool moved = true; moved;) {
    moved = false;
    double Z = 1.0;
    a = 0;
    gone = 0;
    const int p_arg = __builtin_amdgcn_readlane(e.rp.arg, at);
    const uint64_t kids = lane_u64(t.kids, at);
    if (kids == 0 || p_arg < 0 || (sampled && __builtin_amdgcn_readlane(e.rq.arg, at) < 0)) break;  // nothing to try
    for (uint64_t m = kids; m; m &= m - 1) {
      const int j = __ffsll((unsigned long long)m) - 1;
      const int y = __builtin_amdgcn_readlane(e.tok, j);
      const double u = (double)lane_f(e.u, j);
      double w = lane_d(e.p, j);
      bool stays;
      if (argmax) {
        stays = y == p_arg;
      } else if (sampled) {
        const double q = lane_d(e.q, j);
        w = fmax(fma(-a, q, w), 0.0);
        stays = u * q * Z < w;
      } else {
        if (__ballot((gone >> lane & 1) && e.tok == y)) w = 0;  // tried already
        stays = u * Z < w;
      }
      if (stays) {
        if (lane == j) order = len;
        ++len;
        at = j;
        moved = true;
        break;
      }
      if (argmax) continue;
      gone |= 1ull << j;
      a += Z;
      if (!sampled) {
        Z -= w;
      } else if (m & (m - 1)) {  // (the last one's sum is still to be formed)
        Z = left_after(p, row0 + j, lane);
      }
    }
  }
  bool residual = sampled && gone != 0;
  if (!residual) a = 0;
  if (chunk == 0 && tid < 64) {
    if (order >= 0) {
      p.out_path[row0 + order] = lane;
      if (order > 0) {
        p.out_tokens[row0 + order - 1] = e.tok;
        p.out_logp[row0 + order - 1] = (float)log(e.p);
      }
    }
    if (lane >= len && lane < d.nodes) {
      p.out_path[row0 + lane] = p.out_tokens[row0 + lane] = -1;
      p.out_logp[row0 + lane] = 0.f;
    }
    if (lane == 0) p.out_count[s] = len;
  }
  const int64_t row = row0 + at;
  const RowDist tp = row_dist(lane_row(e.rp, at), it);
  auto finish = [&](int64_t y, double logp) {
    p.out_tokens[row0 + len - 1] = (int32_t)y;
    p.out_logp[row0 + len - 1] = (float)logp;
  };
  if (!tp.usable || argmax) {
    if (chunk == 0 && tid == 0) {
      if (tp.usable) finish(tp.arg, -log(tp.sum));
      else finish(-1, (double)__builtin_nanf(""));
    }
    return;
  }
  RowDist tq{};
  if (residual) {
    tq = row_dist(lane_row(e.rq, at), it);
    const double sum = residual_sum<T>(p, row, chunk, tp, tq, a, s_sum);
    if (tid == 0) {
      // written through to where all XCDs see it, and waited for, ahead of the count: a fence
      // would write back the whole L2
      __hip_atomic_store(p.ends + (int64_t)s * d.chunks + chunk, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      s_last = __hip_atomic_fetch_add(p.arrived + s * kOwnLine, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == d.chunks - 1;
    }
    __syncthreads();
    if (!s_last) return;
  } else if (chunk != 0) {
    return;
  }

  const DraftPart* part = p.part + row * d.chunks;
  const T* target = (const T*)p.target + row * d.vocab;
  if (tid < 64) {
    // given drafts: the tokens of the children that were tried are gone, a lane each
    double off = 0;
    int off_at = -1;
    if (!sampled && gone) {
      bool is = (gone >> lane & 1) && e.tok >= 0 && e.tok < d.vocab;
      for (uint64_t m = __ballot(is); m; m &= m - 1) {
        const int j = __ffsll((unsigned long long)m) - 1;
        if (lane > j && __builtin_amdgcn_readlane(e.tok, j) == e.tok) is = false;  // the same again
      }
      if (is) {
        const int ahead = (int)((reinterpret_cast<uintptr_t>(target) / sizeof(T)) % kVec<T>);
        off_at = (e.tok + ahead) / kDraftChunk;
        off = e.p;
      }
    }
    uint64_t takes = __ballot(off_at >= 0), firsts = 0;
    auto part_share = [&](int c) { return part[c].max > kNegInf ? part[c].sum * tp.raw(part[c].max) / tp.sum : 0.0; };
    // A chunk's share without them (the first such lane holds it) is its own less theirs; where that is all
    // but nothing it is summed from the entries, since a rest of mere rounding would end the search in a
    // chunk that has no entry left.
    double rest = 0;
    for (uint64_t todo = takes; todo;) {
      const int j = __ffsll((unsigned long long)todo) - 1, c = __builtin_amdgcn_readlane(off_at, j);
      const uint64_t same = __ballot(off_at == c);
      todo &= ~same;
      firsts |= 1ull << j;
      const double whole = part_share(c);
      double x = whole;
      for (uint64_t m = same; m; m &= m - 1) x -= lane_d(off, __ffsll((unsigned long long)m) - 1);
      if (x < whole * 0x1p-20) {
        ChunkOf<T, 64> entries;
        entries.init(target, d.vocab, c, lane);
        const double ip = 1.0 / tp.sum;
        x = 0;
#pragma unroll 1
        for (int u = 0; u < kLoads<T, 64>; ++u) {
          const RawOf<T> v = entries.load(u);
#pragma unroll
          for (int i = 0; i < kVec<T>; ++i) {
            bool is_gone = false;
            for (uint64_t m = same; m; m &= m - 1)
              is_gone = is_gone || entries.at(u) + i == __builtin_amdgcn_readlane(e.tok, __ffsll((unsigned long long)m) - 1);
            if (!is_gone) x += tp.raw(to_float(v[i])) * ip;
          }
        }
        x = wave_sum_d(x);
      }
      if (lane == j) rest = x;
    }
    auto share = [&](int c) {  // of chunk c in what is left
      const bool is = c < d.chunks;
      if (residual) return is ? __hip_atomic_load(p.ends + (int64_t)s * d.chunks + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
      double x = is ? part_share(c) : 0.0;
      for (uint64_t m = firsts; m; m &= m - 1) {  // (all lanes: they read each other's)
        const int j = __ffsll((unsigned long long)m) - 1;
        const double left = lane_d(rest, j);
        if (__builtin_amdgcn_readlane(off_at, j) == c) x = left;
      }
      return x;
    };
    double near[2];  // the first 128 chunks' shares, looked up once
    auto share_from = [&](int c0) { return c0 < 128 ? c0 ? near[1] : near[0] : share(c0 + lane); };
    auto whole_sum = [&]() {
      near[0] = share(lane);
      near[1] = share(64 + lane);
      double x = 0;
      for (int c0 = 0; c0 < d.chunks; c0 += 64) x += share_from(c0);
      return wave_sum_d(x);
    };
    double total = whole_sum();
    if (!(total > 0)) {  // nothing is left: from p itself
      residual = false;
      takes = firsts = 0;
      total = whole_sum();
    }
    const double want = (double)p.u[row0] * total;
    double start = 0, ahead = 0;
    int pick = -1;
    for (int c0 = 0; c0 < d.chunks; c0 += 64) {
      const double x = share_from(c0);
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
    const bool here = off_at == pick && (takes >> lane & 1);
    const uint64_t in_chunk = __ballot(here);
    if (here) s_pick.gone[__popcll(in_chunk & ((1ull << lane) - 1))] = e.tok;
    if (lane == 0) {
      s_pick.n_gone = __popcll(in_chunk);
      s_pick.chunk = pick;
      s_pick.want = want - ahead;
      s_whole = !residual;
    }
  }
  __syncthreads();
  const Picked got = pick_entry<T>(p, row, tp, tq, s_whole ? 0.0 : a, s_pick, s_w, s_sum);
  if (got.mine) finish(got.y, got.logp);
}

template <typename T>
hipError_t launch_draft_t(const DraftParams& p, hipStream_t s) {
  const DraftShape& d = p.shape;
  hipError_t e;
  {
    TimingScope t("pp_verify_draft_rows", s);
    hipLaunchKernelGGL((draft_rows_kernel<T>), dim3((d.chunks + kWavesD - 1) / kWavesD, d.n * d.nodes, p.draft ? 2 : 1), dim3(kThreads), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  {
    TimingScope t("pp_verify_draft_edges", s);
    hipLaunchKernelGGL((draft_edges_kernel<T>), dim3(d.n), dim3(kEdgeThreads), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  for (int round = 0; p.draft && round + 1 < d.max_children; ++round) {
    TimingScope t("pp_verify_draft_residual", s);
    hipLaunchKernelGGL((draft_residual_kernel<T>), dim3(d.chunks, d.n), dim3(kThreads), 0, s, p, round);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  TimingScope t("pp_verify_draft_end", s);
  hipLaunchKernelGGL((draft_end_kernel<T>), dim3(p.draft ? d.chunks : 1, d.n), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify_draft(const DraftParams& p, int dtype, hipStream_t s) {
  return dtype == kBF16 ? launch_draft_t<uint16_t>(p, s) : launch_draft_t<float>(p, s);
}

}  // namespace pp
