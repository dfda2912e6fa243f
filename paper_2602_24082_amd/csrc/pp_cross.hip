// Cross attention of packed rows to an encoder's states, forward and backward, on gfx950.
//
// Every real token of packed row b -- prompt and responses alike -- looks at the row's
// encoder states: keys and values [0, E_b), or the part [begin_t, end_t) of them.  There
// is no order among the two axes, so the tokens of a row and the G query heads of one
// kv-head are one list of T_b G rows, row r = token r / G, head r % G:
//
//   S = Q K^T scale (visible keys),  P = softmax(S),  O = P V
//   dV = P^T dO,  dS = P (dO V^T - delta),  delta = dO . O
//   dQ = scale dS K,  dK = scale dS^T Q
//
// which is one matrix of rows against keys per (packed row, kv-head): one token of an
// 8-fold group fills 8 rows of a tile that reads its keys once, and the shared heads'
// dK and dV sum up in the accumulators.  Kernels:
//
//   cross_fwd      one workgroup = 128 rows (four waves of 32), walking tiles of keys
//   cross_few      one workgroup = 32 rows, its waves walking different keys
//   cross_combine  joins forwards whose keys were split over workgroups
//   cross_dq       delta and -lse log2(e), then dQ, shaped as cross_fwd
//   cross_dkdv     key-major: one workgroup = 128 keys, walking the rows
//   cross_sum      adds dQ of split keys, dK and dV of split rows
//
// No atomics: the sums' order depends on the batch's shape alone.  All matrix products
// run on the 32 x 32 MFMAs with fp32 accumulation: bf16 inputs on v_mfma_f32_32x32x16_bf16
// with P and dS rounded to bf16 (nearest even; half a step of 2^-8 relative each, as small
// as the rounding of the results), fp32 numbers as sums of three of bf16 on the same
// instruction, which loses nothing that an fp32 product would keep (see Split3).

#include <hip/hip_runtime.h>

#include "pp_device.h"
#include "pp_launch.h"

namespace pp {
namespace {

constexpr float kRescaleSlack = 8.0f;  // log2 units

// What a kernel does with 8 elements along the contraction axis: lane l of a fragment
// holds elements 8 (l / 32) + 0..7 of its row (see pp_device.h).
template <typename T>
struct Ops;

template <>
struct Ops<__bf16> {
  using Frag = bf16x8;
  template <int D>
  static constexpr int kRowD = D;  // the row as 2-byte elements, for the DMA and its swizzle
  static __device__ __forceinline__ Frag load(const __bf16* p) { return *reinterpret_cast<const Frag*>(p); }
  using Held = Frag;  // a fragment that stays in registers
  static __device__ __forceinline__ const Frag& use(const Held& x) { return x; }
  static __device__ __forceinline__ f32x16 mma(const Frag& a, const Frag& b, const f32x16& c) { return mfma32(a, b, c); }
  static __device__ __forceinline__ Frag from_acc(const f32x16& acc, int s) { return acc_half_to_bf16(acc, s); }
  template <int D>
  static __device__ __forceinline__ Held row8(const __bf16* tile, int r, int lc) {
    return lds_row8<D>(tile, r, lc);
  }
  template <int D>
  static __device__ __forceinline__ Frag tr8(const __bf16* tile, int row16, int col0, int lane) {
    return lds_tr8<D>(tile, row16, col0, lane);
  }
};

// fp32 on the bf16 matrix units: x = h + m + l, three bf16 numbers that hold all 24 bits
// of it (each the rest rounded to nearest: |m| <= 2^-9 |x|, |l| <= 2^-18 |x|).  Of the
// nine products of two such sums the six above 2^-26 of the whole are taken, smallest
// first, so a product is as good as an fp32 one: 6 x 32 cycles for 16 steps of the
// contraction, against 8 x 64 on v_mfma_f32_32x32x2_f32.
struct Split3 {
  bf16x8 h, m, l;
};
__device__ __forceinline__ Split3 split3(const f32x8& x) {
  Split3 s;
  s.h = __builtin_convertvector(x, bf16x8);
  const f32x8 r = x - __builtin_convertvector(s.h, f32x8);
  s.m = __builtin_convertvector(r, bf16x8);
  s.l = __builtin_convertvector(r - __builtin_convertvector(s.m, f32x8), bf16x8);
  return s;
}

template <>
struct Ops<float> {
  using Frag = Split3;
  template <int D>
  static constexpr int kRowD = 2 * D;
  static __device__ __forceinline__ Frag load(const float* p) { return split3(*reinterpret_cast<const f32x8*>(p)); }
  using Held = f32x8;  // whole: 64 registers of K and V at head size 128 instead of 96, split at each use
  static __device__ __forceinline__ Frag use(const Held& x) { return split3(x); }
  static __device__ __forceinline__ const Frag& use(const Frag& x) { return x; }
  static __device__ __forceinline__ f32x16 mma(const Frag& a, const Frag& b, f32x16 c) {
    c = mfma32(a.l, b.h, c);
    c = mfma32(a.h, b.l, c);
    c = mfma32(a.m, b.m, c);
    c = mfma32(a.m, b.h, c);
    c = mfma32(a.h, b.m, c);
    return mfma32(a.h, b.h, c);
  }
  static __device__ __forceinline__ Frag from_acc(const f32x16& acc, int s) {
    f32x8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = acc[8 * s + e];
    return split3(f);
  }
  template <int D>
  static __device__ __forceinline__ Held row8(const float* tile, int r, int lc) {
    const int sw = swz<2 * D>(r);
    const f32x4 a = *reinterpret_cast<const f32x4*>(tile + r * D + (((2 * lc) ^ sw) << 2));
    const f32x4 b = *reinterpret_cast<const f32x4*>(tile + r * D + (((2 * lc + 1) ^ sw) << 2));
    return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
  // column col0 + l % 32 of the rows that from_acc's elements stand for
  template <int D>
  static __device__ __forceinline__ Frag tr8(const float* tile, int row16, int col0, int lane) {
    const int c = col0 + (lane & 31), h = lane >> 5;
    f32x8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = row16 + 8 * (e >> 2) + 4 * h + (e & 3);
      f[e] = tile[r * D + (((c >> 2) ^ swz<2 * D>(r)) << 2) + (c & 3)];
    }
    return split3(f);
  }
};

// A fragment read ahead of its products.  fp32 at head size 64 keeps it whole, which leaves two
// workgroups of the forward and of dQ room on a compute unit (dQ 632 -> 505 us on 6 rows of
// 16/4 heads); at head size 128, with one a unit, it is split at once (dQ 2355 us, whole 2452).
template <int D, typename T>
__device__ __forceinline__ auto ahead(const typename Ops<T>::Held& x) {
  if constexpr (sizeof(T) == 4 && D == 128) return Ops<T>::use(x);
  else return x;
}

// Wave-cooperative DMA of NR rows of D elements of T (see TileDma).
template <typename T, int D, int NR>
using RowDma = TileDma<Ops<T>::template kRowD<D>, NR>;
template <bool ONCE = false, int RD, int NR, typename T>
__device__ __forceinline__ void dma_rows(const TileDma<RD, NR>& d, T* lds_tile, const T* src, int rows_valid) {
  d.template issue<ONCE>(reinterpret_cast<__bf16*>(lds_tile), reinterpret_cast<const __bf16*>(src), rows_valid);
}

// A lane's 16 columns 8 r4 + 4 hf + 0..3 of a row's block of 32, times sc, or zeros.  As bf16
// the wave's halves exchange groups of four first, so that a lane writes 16 bytes and the
// two lanes of a row 32: half the requests of 8-byte stores (17 rows of 12/12 heads with one
// to five states, the forward 52 -> 43 us, dQ 116 -> 107; dK and dV, few beside what their
// walks read, gain nothing from it).
template <typename T>
__device__ __forceinline__ void store_block(T* dst, int hf, const f32x16& x, float sc, bool some) {
  f32x4 v[4];
#pragma unroll
  for (int r4 = 0; r4 < 4; ++r4) {
    v[r4] = f32x4{};
    if (some) v[r4] = f32x4{x[4 * r4] * sc, x[4 * r4 + 1] * sc, x[4 * r4 + 2] * sc, x[4 * r4 + 3] * sc};
  }
  if constexpr (sizeof(T) == 2) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int r4 = 0; r4 < 4; r4 += 2) {
      const u32x2 a = __builtin_bit_cast(u32x2, __builtin_convertvector(v[r4], bf16x4));
      const u32x2 b = __builtin_bit_cast(u32x2, __builtin_convertvector(v[r4 + 1], bf16x4));
      const auto x0 = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
      const auto x1 = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
      *reinterpret_cast<u32x4*>(dst + 8 * r4 + 8 * hf) = u32x4{x0[0], x1[0], x0[1], x1[1]};
    }
  } else {
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) store4<T>(dst + 8 * r4 + 4 * hf, v[r4]);
  }
}

template <typename T>
struct CrossParams {
  const T* q;
  const T* k;
  const T* v;
  const T* dout;
  const T* o_in;           // backward
  T* o;                    // forward: o; dQ: dq
  T* dk;
  T* dv;
  float* lse;              // forward: out
  const float* lse_in;
  const CrossItem* items;  // null: in inl
  const CrossKvItem* kv_items;
  const int32_t* kbeg;     // per token, or null
  const int32_t* kend;
  float* part;             // partial sums of split items
  float* part_ml;          // forward: (maximum, sum) of the partial rows
  float* ndelta;           // [hkv][sumT G]: -delta and -lse log2(e) of every row
  float* nlse2;
  CrossRange* ranges;      // per block of 32 rows: least and greatest begin and end
  int hq, hkv, G, sumT;
  uint32_t g_magic;
  float scale;
  float scale_log2;
};

// Few items ride in the launch's arguments, so that a small call needs no copy ahead of
// its kernels.
template <int N>
struct InlineItems {
  CrossItem item[N];
};

template <typename P, int N>
__device__ __forceinline__ CrossItem cross_item(const P& p, const InlineItems<N>& inl, int idx) {
  if (p.items) return load_uniform(p.items + idx);
  return inl.item[idx];
}

// One lane's row of an item and what it sees.
struct RowOf {
  bool in_tile, live;
  int tok, head;  // flat token, query head
  int lo, hi;     // visible keys of the item's part
  int all_lo, all_hi;  // and of all the states, if any
};

template <bool RANGES, typename P>
__device__ __forceinline__ RowOf row_of(const P& p, const CrossItem& it, int g, int r) {
  RowOf w;
  w.in_tile = r < it.rows;
  w.live = r < it.live;
  const int i = (int)((unsigned)r / (unsigned)p.G);
  w.tok = it.tok0 + i;
  w.head = g * p.G + (r - i * p.G);
  w.lo = it.k_begin;
  w.hi = w.live ? it.k_end : it.k_begin;
  w.all_lo = 0;
  w.all_hi = w.live ? it.elen : 0;
  if (RANGES && w.live) {
    const int lo = p.kbeg[w.tok], hi = p.kend[w.tok];
    w.lo = max(w.lo, lo);
    w.hi = min(w.hi, hi);
    w.all_lo = max(0, lo);
    w.all_hi = min(it.elen, hi);
  }
  if (w.hi <= w.lo) w.lo = w.hi = it.k_begin;
  return w;
}

__device__ __forceinline__ int wave_min_i(int x) {
  for (int off = 32; off > 0; off >>= 1) x = min(x, __shfl_xor(x, off, 64));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max_i(int x) {
  for (int off = 32; off > 0; off >>= 1) x = max(x, __shfl_xor(x, off, 64));
  return __builtin_amdgcn_readfirstlane(x);
}

// What a wave's 32 rows see of the keys, as wave-uniform bounds: no row sees a key
// outside [any_lo, any_hi), every live row sees all of [all_lo, all_hi).
struct WaveKeys {
  int any_lo, any_hi, all_lo, all_hi;
  __device__ __forceinline__ bool none(int k0, int k1) const { return k1 <= any_lo || k0 >= any_hi; }
  __device__ __forceinline__ bool every(int k0, int k1) const { return k0 >= all_lo && k1 <= all_hi; }
};

template <bool RANGES>
__device__ __forceinline__ WaveKeys wave_keys(const CrossItem& it, const RowOf& w, int wave_r0) {
  if constexpr (!RANGES) {
    const bool any = wave_r0 < it.live && it.k_end > it.k_begin;
    return {it.k_begin, any ? it.k_end : it.k_begin, it.k_begin, it.k_end};
  } else {
    const bool some = w.hi > w.lo;
    return {wave_min_i(some ? w.lo : 0x7fffffff), wave_max_i(some ? w.hi : 0), wave_max_i(w.live ? w.lo : 0),
            wave_min_i(w.live ? w.hi : 0x7fffffff)};
  }
}

// S^T of masked pairs becomes -inf: key k0 + 4 hf + off is seen iff lo <= it < hi.
template <int KB>
__device__ __forceinline__ void mask_keys(f32x16 (&s)[KB], int k0, int hf, int lo, int hi) {
  static_assert(KB <= 2, "64 bits");
  const uint64_t vis = bits_below64(hi - k0 - 4 * hf) & ~bits_below64(lo - k0 - 4 * hf);
  const uint32_t w[2] = {(uint32_t)vis, (uint32_t)(vis >> 32)};
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[kb][r] = keep_or_neginf(s[kb][r], w[kb], 8 * (r >> 2) + (r & 3));
}

// A row's running softmax: reference maximum (scaled, log2 units), this lane's share of
// the denominator, and O^T.  The reference is only raised when a tile exceeds it by more
// than 2^8, so most tiles do not rescale.
template <int D>
struct RowState {
  f32x16 o[D / 32];
  float m_ref, l;

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int m = 0; m < D / 32; ++m) o[m] = f32x16{};
    m_ref = kNegInf;
    l = 0.f;
  }

  // turns the block's scores into probabilities relative to the reference
  template <int KB>
  __device__ __forceinline__ void probabilities(f32x16 (&s)[KB], float c2) {
    float mx = kNegInf;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
    mx = half_swap_max(mx) * c2;
    const bool raise = mx > m_ref + kRescaleSlack;
    if (wave_any(raise)) {
      const float m_new = raise ? mx : m_ref;
      const float alpha = (m_ref == kNegInf) ? 0.f : fast_exp2(m_ref - m_new);  // nothing seen yet: O = l = 0
      l *= alpha;
#pragma unroll
      for (int m = 0; m < D / 32; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[m][r] *= alpha;
      m_ref = m_new;
    }
    const float mref = (m_ref == kNegInf) ? 0.f : m_ref;
    float ps[2] = {0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[kb][r] = fast_exp2(fmaf(s[kb][r], c2, -mref));
        ps[r & 1] += s[kb][r];
      }
    l += ps[0] + ps[1];
  }
};

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------

// Keys per tile and tiles in flight: 64 keys of bf16 (32 KB of K and V at head size 128),
// 32 of fp32; two workgroups a compute unit.
template <typename T>
constexpr int kKeys = sizeof(T) == 2 ? 64 : 32;
constexpr int kStages = 2;
constexpr int kWaves = 4;
template <int D, typename T>
constexpr int kFwdPerCu = sizeof(T) == 4 ? (D == 64 ? 2 : 1) : D == 64 ? 4 : 2;  // workgroups a compute unit
template <int D, typename T>
constexpr int kDqPerCu = sizeof(T) == 4 ? (D == 64 ? 2 : 1) : D == 64 ? 3 : 2;
static_assert(32 * kWaves == kCrossRows, "rows a workgroup");

// A range of keys, from tile-aligned t0 on; none: t1 = t0 = 0.
struct TileKeys {
  int t0, t1;
};

// What the kWaves waves of a workgroup need together of N ranges that each has: lo[i] <
// hi[i], or no key of it.
template <int N, int BN>
__device__ __forceinline__ void block_join(const int (&lo)[N], const int (&hi)[N], int wave, TileKeys (&out)[N]) {
  __shared__ int s_lo[N][kWaves], s_hi[N][kWaves];
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s_lo[i][wave] = lo[i];
      s_hi[i][wave] = hi[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    int l = s_lo[i][0], h = s_hi[i][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
      l = min(l, s_lo[i][w]);
      h = max(h, s_hi[i][w]);
    }
    l = __builtin_amdgcn_readfirstlane(l);
    h = __builtin_amdgcn_readfirstlane(h);
    out[i] = h > l ? TileKeys{l / BN * BN, h} : TileKeys{0, 0};
  }
}

// The keys that a workgroup walks.
template <bool RANGES, int BN>
__device__ __forceinline__ TileKeys block_keys(const CrossItem& it, const WaveKeys& wk, int wave) {
  TileKeys t[1] = {{it.k_begin, it.k_end}};
  if constexpr (RANGES) {
    const int lo[1] = {wk.any_lo}, hi[1] = {wk.any_hi};
    block_join<1, BN>(lo, hi, wave, t);
  }
  return t[0];
}

template <int D, typename T, bool RANGES, int N>
__global__ __launch_bounds__(kWaves * 64, (kFwdPerCu<D, T>)) void cross_fwd_kernel(CrossParams<T> p, InlineItems<N> inl) {
  using O = Ops<T>;
  using Frag = typename O::Frag;
  using Ahead = decltype(ahead<D, T>(typename O::Held{}));
  constexpr int BN = kKeys<T>, KB = BN / 32, RPW = BN / kWaves;
  using Dma = RowDma<T, D, RPW>;
  __shared__ __attribute__((aligned(1024))) T sKV[kStages][2][BN * D];

  const int item_idx = blockIdx.x / p.hkv, g = blockIdx.x - item_idx * p.hkv;
  const CrossItem it = cross_item(p, inl, item_idx);
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, ln = lane & 31, hf = lane >> 5;
  const RowOf w = row_of<RANGES>(p, it, g, it.r0 + wave * 32 + ln);
  const WaveKeys wk = wave_keys<RANGES>(it, w, it.r0 + wave * 32);
  const int64_t qrow = ((int64_t)w.tok * p.hq + w.head) * D;
  Frag qf[D / 16];
#pragma unroll
  for (int c = 0; c < D / 16; ++c)
    qf[c] = w.live ? O::load(p.q + qrow + 16 * c + 8 * hf) : Frag{};

  const TileKeys tk = block_keys<RANGES, BN>(it, wk, wave);
  const int key0 = tk.t0, n_tiles = (tk.t1 - tk.t0 + BN - 1) / BN;
  const int64_t kv_stride = (int64_t)p.hkv * D;
  const T* kbase = p.k + ((int64_t)it.e0 * p.hkv + g) * D;
  const T* vbase = p.v + ((int64_t)it.e0 * p.hkv + g) * D;
  Dma dma;
  dma.init(wave * RPW, kv_stride * (sizeof(T) / 2), lane);
  auto issue = [&](int t) {
    const int k0 = key0 + t * BN;
    const int rows = min(BN, it.elen - k0);
    dma_rows(dma, sKV[t % kStages][0], kbase + k0 * kv_stride, rows);
    dma_rows(dma, sKV[t % kStages][1], vbase + k0 * kv_stride, rows);
  };
#pragma unroll
  for (int t = 0; t < kStages - 1; ++t)
    if (t < n_tiles) issue(t);

  RowState<D> st;
  st.init();
  const float c2 = p.scale_log2;
  for (int t = 0; t < n_tiles; ++t) {
    const int k0 = key0 + t * BN;
    wait_tile<kStages, 2 * Dma::N>(t, n_tiles);
    __syncthreads();  // tile t landed for every wave; the stage of tile t-1 is free
    if (t + kStages - 1 < n_tiles) issue(t + kStages - 1);
    if (wk.none(k0, k0 + BN)) continue;
    const T* sK = sKV[t % kStages][0];
    const T* sV = sKV[t % kStages][1];
    // S^T = K Q^T: lane = row, registers = keys; K fragments read PD steps ahead
    f32x16 s[KB];
    {
      constexpr int NC = D / 16, NI = KB * NC, PD = sizeof(T) == 4 && D == 64 ? 1 : 3;
      Ahead a[PD + 1];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] = f32x16{};
#pragma unroll
      for (int n = 0; n < PD; ++n) a[n] = ahead<D, T>(O::template row8<D>(sK, (n / NC) * 32 + ln, 2 * (n % NC) + hf));
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        if (n + PD < NI)
          a[(n + PD) % (PD + 1)] =
              ahead<D, T>(O::template row8<D>(sK, ((n + PD) / NC) * 32 + ln, 2 * ((n + PD) % NC) + hf));
        s[n / NC] = O::mma(O::use(a[n % (PD + 1)]), qf[n % NC], s[n / NC]);
      }
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int n = 0; n < PD; ++n) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 1, 0);
#pragma unroll
        for (int n = 0; n < NI; ++n) {
          if (n + PD < NI) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 1, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
        }
      }
    }
    if (!wk.every(k0, k0 + BN)) mask_keys<KB>(s, k0, hf, w.lo, w.hi);
    st.probabilities(s, c2);
    // O^T += V^T P^T over 16-key chunks
#pragma unroll
    for (int ch = 0; ch < 2 * KB; ++ch) {
      const Frag pb = O::from_acc(s[ch >> 1], ch & 1);
#pragma unroll
      for (int m = 0; m < D / 32; ++m) st.o[m] = O::mma(O::template tr8<D>(sV, 16 * ch, 32 * m, lane), pb, st.o[m]);
    }
  }

  if (!w.in_tile) return;
  const float l_tot = half_swap_sum(st.l);
  if (it.slot >= 0) {
    if (!w.live) return;
    const int64_t prow = ((int64_t)it.slot * p.hkv + g) * kCrossRows + wave * 32 + ln;
#pragma unroll
    for (int m = 0; m < D / 32; ++m)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<f32x4*>(p.part + prow * D + 32 * m + 8 * r4 + 4 * hf) =
            f32x4{st.o[m][4 * r4], st.o[m][4 * r4 + 1], st.o[m][4 * r4 + 2], st.o[m][4 * r4 + 3]};
    if (hf == 0) {
      p.part_ml[2 * prow] = st.m_ref;
      p.part_ml[2 * prow + 1] = l_tot;
    }
    return;
  }
  const bool seen = w.hi > w.lo;
  const float inv = seen ? 1.f / l_tot : 0.f;
#pragma unroll
  for (int m = 0; m < D / 32; ++m) store_block<T>(p.o + qrow + 32 * m, hf, st.o[m], inv, seen);
  if (hf == 0) p.lse[(int64_t)w.head * p.sumT + w.tok] = seen ? (st.m_ref + __log2f(l_tot)) * (1.0f / kLog2e) : 0.f;
}

// ---------------------------------------------------------------------------
// Forward of a few rows: sampling, a token or a few of each packed row
// ---------------------------------------------------------------------------

// Up to 32 rows a packed row leave three of cross_fwd's waves without any, and its one
// barrier a tile makes a stream of keys wait for the slowest.  Here all waves hold the
// same 32 rows and walk 32-key blocks of their own, w, w + NW, ..., each through a ring in
// its own part of LDS that nobody else touches: no barrier until the waves' softmaxes are
// joined.  Bound by reading keys and values once: 6.3 TB/s on 471 MB.
template <int D, typename T>
constexpr int kFewWaves = D * sizeof(T) > 256 ? 2 : 4;  // 128 KB of LDS at most

template <int D, typename T, bool RANGES, int N>
__global__ __launch_bounds__((kFewWaves<D, T> * 64), 1) void cross_few_kernel(CrossParams<T> p, InlineItems<N> inl) {
  using O = Ops<T>;
  using Frag = typename O::Frag;
  constexpr int NW = kFewWaves<D, T>, NC = D / 16;
  using Dma = RowDma<T, D, 32>;
  struct Join {
    f32x4 o[D / 8][64];
  };
  union Smem {
    T kv[NW][2][2][32 * D];  // [wave][stage][K / V]
    Join join[NW];
  };
  __shared__ __attribute__((aligned(1024))) Smem sm;
  __shared__ float s_m[NW][32], s_l[NW][32];

  const int item_idx = blockIdx.x / p.hkv, g = blockIdx.x - item_idx * p.hkv;
  const CrossItem it = cross_item(p, inl, item_idx);
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, ln = lane & 31, hf = lane >> 5;
  const RowOf w = row_of<RANGES>(p, it, g, it.r0 + ln);
  const WaveKeys wk = wave_keys<RANGES>(it, w, it.r0);
  const int key0 = RANGES ? (wk.any_hi > 0 ? wk.any_lo / 32 * 32 : 0) : it.k_begin;
  const int nb = (wk.any_hi - key0 + 31) / 32;
  const int64_t kv_stride = (int64_t)p.hkv * D;
  const T* kbase = p.k + ((int64_t)it.e0 * p.hkv + g) * D;
  const T* vbase = p.v + ((int64_t)it.e0 * p.hkv + g) * D;
  Dma dma;
  dma.init(0, kv_stride * (sizeof(T) / 2), lane);
  // Block i of this wave: its K and V in stage i & 1, each refilled with block i + 2's as
  // soon as it has been read, so three quarters of the ring are in flight.
  auto key_of = [&](int i) { return key0 + (wave + i * NW) * 32; };
  auto issue = [&](int i, int kv, const T* base) {
    const int k0 = key_of(i);
    dma_rows<true>(dma, sm.kv[wave][i & 1][kv], base + k0 * kv_stride, min(32, it.elen - k0));
  };
  const int n = wave < nb ? (nb - wave + NW - 1) / NW : 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (i < n) {
      issue(i, 0, kbase);
      issue(i, 1, vbase);
    }
  }
  const int64_t qrow = ((int64_t)w.tok * p.hq + w.head) * D;
  Frag qf[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c)
    qf[c] = w.live ? O::load(p.q + qrow + 16 * c + 8 * hf) : Frag{};
  RowState<D> st;
  st.init();
  for (int i = 0; i < n; ++i) {
    // in flight behind K(i): V(i), and K and V of block i + 1 if there is one (at the
    // first block Q's loads too, which then are waited for as well)
    if (i == 0) wait_vmem<0>();
    else if (i + 1 < n) wait_vmem<3 * Dma::N>();
    else wait_vmem<Dma::N>();
    asm volatile("" ::: "memory");
    const int k0 = key_of(i);
    const T* sK = sm.kv[wave][i & 1][0];
    const T* sV = sm.kv[wave][i & 1][1];
    f32x16 s[1] = {f32x16{}};
#pragma unroll
    for (int c = 0; c < NC; ++c) s[0] = O::mma(O::use(O::template row8<D>(sK, ln, 2 * c + hf)), qf[c], s[0]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K's reads have returned
    if (i + 2 < n) issue(i + 2, 0, kbase);
    if (!wk.every(k0, k0 + 32)) mask_keys<1>(s, k0, hf, w.lo, w.hi);
    st.probabilities(s, p.scale_log2);
    if (i + 2 < n) wait_vmem<3 * Dma::N>();  // behind V(i): K and V of i + 1, K of i + 2
    else if (i + 1 < n) wait_vmem<2 * Dma::N>();
    else wait_vmem<0>();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ch = 0; ch < 2; ++ch) {
      const Frag pb = O::from_acc(s[0], ch);
#pragma unroll
      for (int m = 0; m < D / 32; ++m) st.o[m] = O::mma(O::template tr8<D>(sV, 16 * ch, 32 * m, lane), pb, st.o[m]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V's too
    if (i + 2 < n) issue(i + 2, 1, vbase);
  }
  // the waves' shares, in wave order; wave w finishes D / 8 / NW groups of four columns
  const float l_own = half_swap_sum(st.l);
  __syncthreads();
#pragma unroll
  for (int q = 0; q < D / 8; ++q)
    sm.join[wave].o[q][lane] = f32x4{st.o[q >> 2][4 * (q & 3)], st.o[q >> 2][4 * (q & 3) + 1], st.o[q >> 2][4 * (q & 3) + 2],
                                     st.o[q >> 2][4 * (q & 3) + 3]};
  if (hf == 0) {
    s_m[wave][ln] = st.m_ref;
    s_l[wave][ln] = l_own;
  }
  __syncthreads();
  float m = kNegInf, l = 0.f, a[NW];
#pragma unroll
  for (int i = 0; i < NW; ++i) m = fmaxf(m, s_m[i][ln]);
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    const float li = s_l[i][ln];
    a[i] = li == 0.f ? 0.f : fast_exp2(s_m[i][ln] - (m == kNegInf ? 0.f : m));  // 0: the wave saw no key of the row
    l = fmaf(li, a[i], l);
  }
  if (!w.in_tile) return;
  const bool seen = w.hi > w.lo;
  const float inv = it.slot >= 0 ? 1.f : seen ? 1.f / l : 0.f;
  const int64_t prow = ((int64_t)it.slot * p.hkv + g) * 32 + ln;
  if (it.slot >= 0 && !w.live) return;
#pragma unroll
  for (int i = 0; i < D / 8 / NW; ++i) {
    const int q = wave * (D / 8 / NW) + i, col = 8 * q + 4 * hf;
    f32x4 v = f32x4{};
#pragma unroll
    for (int j = 0; j < NW; ++j) v += sm.join[j].o[q][lane] * a[j];
    v *= inv;
    if (it.slot >= 0) *reinterpret_cast<f32x4*>(p.part + prow * D + col) = v;
    else store4<T>(p.o + qrow + col, seen ? v : f32x4{});
  }
  if (wave != 0 || hf != 0) return;
  if (it.slot >= 0) {
    p.part_ml[2 * prow] = m;
    p.part_ml[2 * prow + 1] = l;
  } else {
    p.lse[(int64_t)w.head * p.sumT + w.tok] = seen ? (m + __log2f(l)) * (1.0f / kLog2e) : 0.f;
  }
}

// Joins the parts of rows whose keys were split, in part order: a row is D / 4 lanes,
// four parts' loads in flight.
template <int D, typename T, int N>
__global__ __launch_bounds__(256) void cross_combine_kernel(CrossParams<T> p, const CrossSplit* splits, CrossSplitList<N> inl,
                                                            int bm) {
  constexpr int LPR = D / 4, RPB = 256 / LPR;
  const int si = blockIdx.x / p.hkv, g = blockIdx.x - si * p.hkv;
  const CrossSplit sp = splits ? load_uniform(splits + si) : inl.split[si];
  const int lr = blockIdx.y * RPB + threadIdx.x / LPR, c = (threadIdx.x % LPR) * 4;
  const int r = sp.r0 + lr;
  if (lr >= bm || r >= sp.rows) return;
  const int i = (int)((unsigned)r / (unsigned)p.G);
  const int tok = sp.tok0 + i, head = g * p.G + (r - i * p.G);
  f32x4 acc = f32x4{};
  float m = kNegInf, l = 0.f;
  if (r < sp.live) {
    constexpr int NP = 4;
    const int64_t stride = (int64_t)p.hkv * bm;  // rows between slots
    int64_t prow = ((int64_t)sp.slot0 * p.hkv + g) * bm + lr;
    for (int n0 = 0; n0 < sp.parts; n0 += NP, prow += NP * stride) {
      f32x4 x[NP];
      float pm[NP], pl[NP];
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        const bool on = n0 + n < sp.parts;
        const int64_t row = prow + (on ? n : 0) * stride;
        x[n] = *reinterpret_cast<const f32x4*>(p.part + row * D + c);
        pm[n] = p.part_ml[2 * row];
        pl[n] = on ? p.part_ml[2 * row + 1] : 0.f;
      }
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        if (pl[n] == 0.f) continue;  // a part without a visible key
        const float mn = fmaxf(m, pm[n]);
        const float a = m == kNegInf ? 0.f : fast_exp2(m - mn), b = fast_exp2(pm[n] - mn);
        l = l * a + pl[n] * b;
        acc = acc * a + x[n] * b;
        m = mn;
      }
    }
  }
  const bool seen = l != 0.f;
  const float inv = seen ? 1.f / l : 0.f;
  store4<T>(p.o + ((int64_t)tok * p.hq + head) * D + c, seen ? acc * inv : f32x4{});
  if (c == 0) p.lse[(int64_t)head * p.sumT + tok] = seen ? (m + __log2f(l)) * (1.0f / kLog2e) : 0.f;
}

// ---------------------------------------------------------------------------
// dQ
// ---------------------------------------------------------------------------

template <int D, typename T, bool RANGES>
__global__ __launch_bounds__(kWaves * 64, (kDqPerCu<D, T>)) void cross_dq_kernel(CrossParams<T> p) {
  using O = Ops<T>;
  using Frag = typename O::Frag;
  using Ahead = decltype(ahead<D, T>(typename O::Held{}));
  constexpr int BN = kKeys<T>, KB = BN / 32, RPW = BN / kWaves;
  using Dma = RowDma<T, D, RPW>;
  __shared__ __attribute__((aligned(1024))) T sKV[kStages][2][BN * D];

  const int item_idx = blockIdx.x / p.hkv, g = blockIdx.x - item_idx * p.hkv;
  const CrossItem it = load_uniform(p.items + item_idx);
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, ln = lane & 31, hf = lane >> 5;
  const int r = it.r0 + wave * 32 + ln;
  const RowOf w = row_of<RANGES>(p, it, g, r);
  const WaveKeys wk = wave_keys<RANGES>(it, w, it.r0 + wave * 32);
  const int64_t qrow = ((int64_t)w.tok * p.hq + w.head) * D;
  Frag qf[D / 16], df[D / 16];
  // Q, then dO, then O: eight loads pass over a row's two cache lines, which the first level
  // keeps that long for one tensor, but not for two; the first keys are on their way behind
  // them, ahead of delta (12 rows with 129 to 349 states 256 -> 240 us, 24 ragged rows of head
  // size 64 87 -> 79)
#pragma unroll
  for (int c = 0; c < D / 16; ++c) qf[c] = w.live ? O::load(p.q + qrow + 16 * c + 8 * hf) : Frag{};
#pragma unroll
  for (int c = 0; c < D / 16; ++c) df[c] = w.live ? O::load(p.dout + qrow + 16 * c + 8 * hf) : Frag{};
  // delta = dO . O and -lse log2(e) of the lane's row, kept for the dK/dV pass.  O as stored is
  // rounded to bf16, and where a row sees few keys dP - delta is small beside delta: a row of at
  // most BN keys gets delta = sum P dP.  Where they lie in one tile (a bit of `single`) that is
  // formed in the tile's step; where they lie across a border (`two`) the workgroup goes over
  // those tiles once before its walk.  dQ and dK at about two keys are off by 0.0024 of them
  // instead of 0.0037.  It costs short walks 2%, the backward of texts whose images of 64 states
  // start off the borders 7% (221 us for 206 on 8 rows of 32/8 heads of 128), others nothing.
  float dlt = 0.f;
  uint64_t single = 0, two = 0;
  auto stat = [&] { return (int64_t)g * p.sumT * p.G + (int64_t)it.tok0 * p.G + (it.r0 + wave * 32 + (threadIdx.x & 31)); };
  if constexpr (sizeof(T) == 2) {
    const bool few = w.all_hi > w.all_lo && w.all_hi - w.all_lo <= BN;
    single = __ballot(few && w.all_lo / BN == (w.all_hi - 1) / BN);
    two = RANGES ? __ballot(few) & ~single : 0;
  }
  const int64_t kv_stride = (int64_t)p.hkv * D;
  const T* kbase = p.k + ((int64_t)it.e0 * p.hkv + g) * D;
  const T* vbase = p.v + ((int64_t)it.e0 * p.hkv + g) * D;
  Dma dma;
  dma.init(wave * RPW, kv_stride * (sizeof(T) / 2), lane);
  auto issue = [&](int k0, int t) {
    const int rows = min(BN, it.elen - k0);
    dma_rows(dma, sKV[t % kStages][0], kbase + k0 * kv_stride, rows);
    dma_rows(dma, sKV[t % kStages][1], vbase + k0 * kv_stride, rows);
  };
  // S^T = K Q^T and dP^T = V dO^T of a tile, fragments read PD ahead
  auto products = [&](const T* sK, const T* sV, f32x16 (&s)[KB], f32x16 (&dp)[KB]) {
    constexpr int NC = D / 16, NI = 2 * KB * NC, PD = 3;
    auto frag = [&](int n) {
      return ahead<D, T>(O::template row8<D>(((n / NC) & 1) ? sV : sK, (n / (2 * NC)) * 32 + ln, 2 * (n % NC) + hf));
    };
    Ahead a[PD + 1];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      s[kb] = f32x16{};
      dp[kb] = f32x16{};
    }
#pragma unroll
    for (int n = 0; n < PD; ++n) a[n] = frag(n);
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      if (n + PD < NI) a[(n + PD) % (PD + 1)] = frag(n + PD);
      const int kb = n / (2 * NC), c = n % NC;
      if ((n / NC) & 1) dp[kb] = O::mma(O::use(a[n % (PD + 1)]), df[c], dp[kb]);
      else s[kb] = O::mma(O::use(a[n % (PD + 1)]), qf[c], s[kb]);
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int n = 0; n < PD; ++n) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 1, 0);
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        if (n + PD < NI) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
      }
    }
  };
  auto sum_products = [&](const f32x16 (&s)[KB], const f32x16 (&dp)[KB]) {
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum = fmaf(s[kb][e], dp[kb][e], sum);
    return sum;
  };

  TileKeys tk;
  if constexpr (RANGES && sizeof(T) == 2) {
    // rows of `two` with keys in this part; their tiles may lie in the next or the last one,
    // and every part that has a row's keys sums the same numbers in the same order
    const bool mine = (two >> lane & 1) && w.hi > w.lo;
    const int lo[2] = {wk.any_lo, wave_min_i(mine ? w.all_lo : 0x7fffffff)}, hi[2] = {wk.any_hi, wave_max_i(mine ? w.all_hi : 0)};
    TileKeys t[2];
    block_join<2, BN>(lo, hi, wave, t);
    tk = t[0];
    const int n_ahead = (t[1].t1 - t[1].t0 + BN - 1) / BN;
    if (n_ahead > 0) {
      const float nl = mine ? -p.lse_in[(int64_t)w.head * p.sumT + w.tok] * kLog2e : 0.f;
      float sum = 0.f;
      issue(t[1].t0, 0);
#pragma unroll 1
      for (int i = 0; i < n_ahead; ++i) {
        const int k0 = t[1].t0 + i * BN;
        wait_vmem<0>();
        __syncthreads();
        if (i + 1 < n_ahead) issue(k0 + BN, i + 1);
        if (k0 + BN <= lo[1] || k0 >= hi[1]) continue;
        f32x16 s[KB], dp[KB];
        products(sKV[i % kStages][0], sKV[i % kStages][1], s, dp);
        mask_keys<KB>(s, k0, hf, mine ? w.all_lo : 0, mine ? w.all_hi : 0);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[kb][e] = fast_exp2(fmaf(s[kb][e], p.scale_log2, nl));
        sum += sum_products(s, dp);
      }
      dlt = half_swap_sum(sum);
      if (mine && hf == 0 && w.all_lo == w.lo) p.ndelta[stat()] = -dlt;  // the part of its first key writes
      __syncthreads();  // the stages are free
    }
  } else {
    tk = block_keys<RANGES, BN>(it, wk, wave);
  }
  const int key0 = tk.t0, n_tiles = (tk.t1 - tk.t0 + BN - 1) / BN;
#pragma unroll
  for (int t = 0; t < kStages - 1; ++t)
    if (t < n_tiles) issue(key0 + t * BN, t);

  float nlse2 = 0.f;
  {
    float acc = 0.f;
    if (w.live) {
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        typedef T vec8 __attribute__((ext_vector_type(8)));
        vec8 a;
        if constexpr (sizeof(T) == 2) a = df[c];
        else a = *reinterpret_cast<const vec8*>(p.dout + qrow + 16 * c + 8 * hf);
        const vec8 b = *reinterpret_cast<const vec8*>(p.o_in + qrow + 16 * c + 8 * hf);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc += (float)a[e] * (float)b[e];
      }
      nlse2 = -p.lse_in[(int64_t)w.head * p.sumT + w.tok] * kLog2e;
    }
    acc = half_swap_sum(acc);
    if (!(two >> lane & 1)) dlt = acc;
    if (it.k_begin == 0) {  // the first part, if the keys are split
      if (w.live && hf == 0) {
        if (!((single | two) >> lane & 1)) p.ndelta[stat()] = -dlt;
        p.nlse2[stat()] = nlse2;
      }
    }
  }
  if constexpr (RANGES) {
    if (it.k_begin == 0 && g == 0) {
      const int lo = w.all_hi > w.all_lo ? w.all_lo : 0, hi = w.all_hi > w.all_lo ? w.all_hi : 0;
      const CrossRange rg = {wave_min_i(hi > lo ? lo : 0x7fffffff), wave_max_i(hi > lo ? hi : 0), wave_max_i(w.live ? lo : 0),
                             wave_min_i(w.live ? hi : 0x7fffffff)};
      if (lane == 0 && it.r0 + wave * 32 < it.live) p.ranges[it.blk0 + ((it.r0 + wave * 32) >> 5)] = rg;
    }
  }

  f32x16 acc[D / 32];
#pragma unroll
  for (int m = 0; m < D / 32; ++m) acc[m] = f32x16{};
  for (int t = 0; t < n_tiles; ++t) {
    const int k0 = key0 + t * BN;
    wait_tile<kStages, 2 * Dma::N>(t, n_tiles);
    __syncthreads();
    if (t + kStages - 1 < n_tiles) issue(k0 + (kStages - 1) * BN, t + kStages - 1);
    if (wk.none(k0, k0 + BN)) continue;
    const T* sK = sKV[t % kStages][0];
    const T* sV = sKV[t % kStages][1];
    f32x16 s[KB], dp[KB];
    products(sK, sV, s, dp);
    if (!wk.every(k0, k0 + BN)) mask_keys<KB>(s, k0, hf, w.lo, w.hi);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = fast_exp2(fmaf(s[kb][e], p.scale_log2, nlse2));
    if constexpr (sizeof(T) == 2) {
      const bool here = (single >> lane & 1) && w.hi > w.lo && (unsigned)(w.lo - k0) < (unsigned)BN;
      if (single && wave_any(here)) {
        const float sum = half_swap_sum(sum_products(s, dp));
        if (here) {
          dlt = sum;
          if (hf == 0) p.ndelta[stat()] = -sum;
        }
      }
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) dp[kb][e] = s[kb][e] * (dp[kb][e] - dlt);
    // dQ^T += K^T dS^T over 16-key chunks
#pragma unroll
    for (int ch = 0; ch < 2 * KB; ++ch) {
      const Frag db = O::from_acc(dp[ch >> 1], ch & 1);
#pragma unroll
      for (int m = 0; m < D / 32; ++m) acc[m] = O::mma(O::template tr8<D>(sK, 16 * ch, 32 * m, lane), db, acc[m]);
    }
  }

  if (!w.in_tile) return;
  if (it.slot >= 0) {
    if (!w.live) return;
    float* row = p.part + (((int64_t)it.slot * p.hkv + g) * kCrossRows + wave * 32 + ln) * D;
#pragma unroll
    for (int m = 0; m < D / 32; ++m)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<f32x4*>(row + 32 * m + 8 * r4 + 4 * hf) =
            f32x4{acc[m][4 * r4], acc[m][4 * r4 + 1], acc[m][4 * r4 + 2], acc[m][4 * r4 + 3]};
    return;
  }
  const bool seen = w.hi > w.lo;
#pragma unroll
  for (int m = 0; m < D / 32; ++m) store_block<T>(p.o + qrow + 32 * m, hf, acc[m], p.scale, seen);
}

// Adds the parts of dQ rows whose keys were split, in part order; block b of the splits'.
template <int D, typename T>
__device__ __forceinline__ void dq_sum_block(const CrossParams<T>& p, const CrossSplit* splits, int b) {
  constexpr int LPR = D / 4, RPB = 256 / LPR, YB = kCrossRows / RPB;
  const int y = b % YB;
  b /= YB;
  const int si = b / p.hkv, g = b - si * p.hkv;
  const CrossSplit sp = load_uniform(splits + si);
  const int lr = y * RPB + threadIdx.x / LPR, c = (threadIdx.x % LPR) * 4;
  const int r = sp.r0 + lr;
  if (r >= sp.rows) return;
  const int i = (int)((unsigned)r / (unsigned)p.G);
  f32x4 acc = f32x4{};
  if (r < sp.live) {
    constexpr int NP = 4;
    const int64_t stride = (int64_t)p.hkv * kCrossRows * D;
    const float* src = p.part + (((int64_t)sp.slot0 * p.hkv + g) * kCrossRows + lr) * D + c;
    for (int n0 = 0; n0 < sp.parts; n0 += NP, src += NP * stride) {
      f32x4 x[NP];
#pragma unroll
      for (int n = 0; n < NP; ++n)
        if (n0 + n < sp.parts) x[n] = *reinterpret_cast<const f32x4*>(src + n * stride);
#pragma unroll
      for (int n = 0; n < NP; ++n)
        if (n0 + n < sp.parts) acc += x[n];
    }
  }
  store4<T>(p.o + ((int64_t)(sp.tok0 + i) * p.hq + g * p.G + (r - i * p.G)) * D + c, acc * p.scale);
}

// ---------------------------------------------------------------------------
// dK, dV: key-major
// ---------------------------------------------------------------------------

// Head size 128, bf16: eight waves; waves w and w + 4 own keys 32 (w % 4) .. +31 and take
// the two 32-row halves of every 64-row step; K and V of the tile stay in LDS.
// Head size 64 or fp32: four waves and 32-row steps, K and V in registers; with bf16 three
// (fp32 of head size 64 two) workgroups share a compute unit, and one's barriers pass under the others' products (three
// for two: 162 -> 148 us on 24 rows of 14/2 heads, 280 -> 263 on long rows; a third stage of
// the ring instead was slower).  Two workgroups of fp32 at head size 64 leave 30 registers to
// memory, which the steps reload, and are faster all the same (810 -> 745 us on 6 rows of 16/4 heads).
template <int D, typename T>
struct KvShape {
  static constexpr bool HOLD = D * sizeof(T) != 256 || D == 64;
  static constexpr int QB = HOLD ? 1 : 2;  // row blocks a step
  static constexpr int STEP = kCrossStep(D, sizeof(T) == 4);
  static constexpr int WAVES = 4 * QB;
  static constexpr int PER_CU = HOLD && sizeof(T) == 2 ? 3 : D == 64 ? 2 : 1;
  static_assert(STEP == 32 * QB, "rows a step");
};

template <int D, typename T>
struct KvStage {
  T q[KvShape<D, T>::STEP * D];
  T dout[KvShape<D, T>::STEP * D];
  float nlse2[64];   // a DMA fills all 64
  float ndelta[64];
  int lo[64], hi[64];
};

template <int D, typename T, bool HOLD>
struct KvTiles {
  T k[kCrossKeys * D], v[kCrossKeys * D];
};
template <int D, typename T>
struct KvTiles<D, T, true> {};

template <int D, typename T>
struct KvSmem : KvTiles<D, T, KvShape<D, T>::HOLD> {
  union {
    KvStage<D, T> st[2];
    float red[4][32 * D];
  };
};

template <int D, typename T, bool RANGES>
__global__ __launch_bounds__((KvShape<D, T>::WAVES * 64), (KvShape<D, T>::PER_CU)) void cross_dkdv_kernel(CrossParams<T> p) {
  using O = Ops<T>;
  using Frag = typename O::Frag;
  using S = KvShape<D, T>;
  constexpr int STEP = S::STEP, RD = O::template kRowD<D>;
  constexpr int RPI = 1024 / (RD * 2), CPR = RD / 8;   // rows and 16-byte chunks of a DMA instruction
  constexpr int RPW = STEP / S::WAVES, NI = RPW / RPI;
  static_assert(RPW % RPI == 0, "whole DMA instructions");
  __shared__ __attribute__((aligned(1024))) KvSmem<D, T> sm;

  const int item_idx = blockIdx.x / p.hkv, g = blockIdx.x - item_idx * p.hkv;
  const CrossKvItem it = load_uniform(p.kv_items + item_idx);
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, ln = lane & 31, hf = lane >> 5;
  const int kb = wave & 3, qb = wave >> 2;
  const int wk0 = it.k0 + kb * 32, wk1 = min(it.elen, wk0 + 32);
  const bool wave_live = wk0 < wk1;
  const int j = wk0 + ln;
  const int k1 = min(it.elen, it.k0 + kCrossKeys);
  const int64_t kv_stride = (int64_t)p.hkv * D;

  // rows past the states repeat the last one
  using Held = typename O::Held;
  Held kf[S::HOLD ? D / 16 : 1], vf[S::HOLD ? D / 16 : 1];
  const bool any = it.n_begin < it.n_end;
  if constexpr (S::HOLD) {
    if (any) {
      const int64_t row = ((int64_t)(it.e0 + min(j, it.elen - 1)) * p.hkv + g) * D;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        kf[c] = *reinterpret_cast<const Held*>(p.k + row + 16 * c + 8 * hf);
        vf[c] = *reinterpret_cast<const Held*>(p.v + row + 16 * c + 8 * hf);
      }
    }
  } else {
    if (any) {
      TileDma<RD, kCrossKeys / S::WAVES> kd;
      kd.init(wave * (kCrossKeys / S::WAVES), kv_stride * (sizeof(T) / 2), lane);
      const int64_t row = ((int64_t)(it.e0 + it.k0) * p.hkv + g) * D;
      dma_rows(kd, sm.k, p.k + row, k1 - it.k0);
      dma_rows(kd, sm.v, p.v + row, k1 - it.k0);
    }
  }

  // RANGES: the next step from n on in which some row sees a key of the tile.  A lane
  // looks at a step, 64 of them at a time.
  const CrossRange* ranges = RANGES ? p.ranges + it.blk0 : nullptr;
  uint64_t hits = 0;
  int hits0 = 0, hits_end = 0;  // the steps that `hits` stands for
  auto next_step = [&](int n) {
    if constexpr (RANGES) {
      while (n < it.n_end) {
        if (n >= hits_end) {
          hits0 = n;
          hits_end = n + 64;
          bool hit = false;
#pragma unroll
          for (int b = 0; b < S::QB; ++b) {
            const int blk = (n + lane) * S::QB + b;
            if (n + lane < it.n_end && blk * 32 < it.live) hit |= ranges[blk].any_lo < k1 && ranges[blk].any_hi > it.k0;
          }
          hits = __ballot(hit);
        }
        const uint64_t rest = hits >> (n - hits0);
        if (rest) return n + __builtin_ctzll(rest);
        n = hits_end;
      }
    }
    return n;
  };
  // lane's row lr of the step from row r0 on, as the token past i0 and the head
  auto split_row = [&](int x, int& il, int& h) {
    il = p.G == 1 ? x : (int)__umulhi((unsigned)x, p.g_magic);
    h = x - il * p.G;
  };
  auto issue = [&](int n, int buf) {
    KvStage<D, T>& sg = sm.st[buf];
    const int r0 = n * STEP;
    const int rows = min(STEP, it.live - r0);
    const int i0 = (int)((unsigned)r0 / (unsigned)p.G), h0 = r0 - i0 * p.G;
    const int64_t t0 = (int64_t)it.tok0 + i0;
    const char* qbase = reinterpret_cast<const char*>(p.q + (t0 * p.hq + g * p.G) * D);
    const char* obase = reinterpret_cast<const char*>(p.dout + (t0 * p.hq + g * p.G) * D);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int first = wave * RPW + i * RPI, lr = first + lane / CPR;
      int il, h;
      split_row(h0 + min(lr, rows - 1), il, h);
      const uint32_t off = ((uint32_t)il * (uint32_t)p.hq + (uint32_t)h) * (uint32_t)(RD * 2) +
                           ((uint32_t)((lane % CPR) ^ swz<RD>(lr)) << 4);
      lds_dma16(qbase + off, sg.q + first * D);
      lds_dma16(obase + off, sg.dout + first * D);
    }
    const int lr = min(lane, rows - 1);
    const int64_t at = (int64_t)g * p.sumT * p.G + (int64_t)it.tok0 * p.G + r0 + lr;
    if (wave == 0) dma_dword(sg.nlse2, p.nlse2 + at);
    else if (wave == 1) dma_dword(sg.ndelta, p.ndelta + at);
    if constexpr (RANGES) {
      if (wave == 2 || wave == 3) {
        int il, h;
        split_row(h0 + lr, il, h);
        if (wave == 2) dma_dword(sg.lo, p.kbeg + t0 + il);
        else dma_dword(sg.hi, p.kend + t0 + il);
      }
    }
  };
  int n = next_step(it.n_begin), buf = 0;
  if (n < it.n_end) issue(n, 0);

  f32x16 acc_dk[D / 32], acc_dv[D / 32];
#pragma unroll
  for (int m = 0; m < D / 32; ++m) {
    acc_dk[m] = f32x16{};
    acc_dv[m] = f32x16{};
  }
  while (n < it.n_end) {
    const int nn = next_step(n + 1);
    wait_vmem<0>();
    __syncthreads();  // step n (and K, V) landed for every wave; the other stage is free
    if (nn < it.n_end) issue(nn, buf ^ 1);
    const KvStage<D, T>& sg = sm.st[buf];
    const int rb0 = n * STEP + qb * 32;
    n = nn;
    buf ^= 1;
    if (!wave_live || rb0 >= it.live) continue;
    bool masked = false;
    if constexpr (RANGES) {
      const CrossRange rg = load_uniform(ranges + (rb0 >> 5));
      if (rg.any_hi <= wk0 || rg.any_lo >= wk1) continue;
      masked = !(rg.all_lo <= wk0 && rg.all_hi >= wk1);
    }
    // S = Q K^T and dP = dO V^T: lane = key, registers = rows.  At head size 64 dP's
    // accumulator starts from -delta, which spares the subtractions.
    constexpr bool kAccDelta = D == 64 && sizeof(T) == 2;
    f32x16 s = f32x16{}, dp = f32x16{};
    if constexpr (kAccDelta) {
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 d4 = *reinterpret_cast<const f32x4*>(&sg.ndelta[qb * 32 + 8 * r4 + 4 * hf]);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * r4 + e] = d4[e];
      }
    }
    {
      constexpr int NC = D / 16;
      Held fq[2], fk[2], fo[2], fv[2];
      auto load = [&](int c, int b) {
        fq[b] = O::template row8<D>(sg.q, qb * 32 + ln, 2 * c + hf);
        if constexpr (!S::HOLD) fk[b] = O::template row8<D>(sm.k, kb * 32 + ln, 2 * c + hf);
        fo[b] = O::template row8<D>(sg.dout, qb * 32 + ln, 2 * c + hf);
        if constexpr (!S::HOLD) fv[b] = O::template row8<D>(sm.v, kb * 32 + ln, 2 * c + hf);
      };
      load(0, 0);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (c + 1 < NC) load(c + 1, (c + 1) & 1);
        if constexpr (S::HOLD) {
          // counts as rewritten, or the split parts of all of K and V would be kept across steps
          if constexpr (sizeof(T) == 4 && D == 128) asm volatile("" : "+v"(kf[c]), "+v"(vf[c]));
          s = O::mma(O::use(fq[c & 1]), O::use(kf[c]), s);
          dp = O::mma(O::use(fo[c & 1]), O::use(vf[c]), dp);
        } else {
          s = O::mma(O::use(fq[c & 1]), O::use(fk[c & 1]), s);
          dp = O::mma(O::use(fo[c & 1]), O::use(fv[c & 1]), dp);
        }
      }
      if constexpr (sizeof(T) == 2) {
        constexpr int R = S::HOLD ? 1 : 2;  // reads ahead of each MFMA
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, (kAccDelta ? 4 : 0) + 2 * R, 0);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if (c + 1 < NC) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, R, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
          if (c + 1 < NC) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, R, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
        }
      }
    }
    if (rb0 + 32 > it.live) {  // rows past the last repeat it: not to be counted again
      const uint32_t vis = bits_below32(it.live - rb0 - 4 * hf);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = keep_or_neginf(s[e], vis, 8 * (e >> 2) + (e & 3));
    }
    if constexpr (RANGES) {
      if (masked) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const int il = qb * 32 + 8 * r4 + 4 * hf;
          const i32x4 lo = *reinterpret_cast<const i32x4*>(&sg.lo[il]);
          const i32x4 hi = *reinterpret_cast<const i32x4*>(&sg.hi[il]);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * r4 + e] = j >= lo[e] && j < hi[e] ? s[4 * r4 + e] : kNegInf;
        }
      }
    }
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int il = qb * 32 + 8 * r4 + 4 * hf;
      const f32x4 l4 = *reinterpret_cast<const f32x4*>(&sg.nlse2[il]);
      f32x4 d4 = f32x4{};
      if constexpr (!kAccDelta) d4 = *reinterpret_cast<const f32x4*>(&sg.ndelta[il]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int x = 4 * r4 + e;
        const float pr = fast_exp2(fmaf(s[x], p.scale_log2, l4[e]));
        s[x] = pr;
        dp[x] = pr * (kAccDelta ? dp[x] : dp[x] + d4[e]);
      }
    }
    // dV^T += dO^T P and dK^T += Q^T dS over two 16-row chunks
    const Frag pb0 = O::from_acc(s, 0), pb1 = O::from_acc(s, 1);
    const Frag db0 = O::from_acc(dp, 0), db1 = O::from_acc(dp, 1);
#pragma unroll
    for (int m = 0; m < D / 32; ++m) {
      acc_dv[m] = O::mma(O::template tr8<D>(sg.dout, qb * 32, 32 * m, lane), pb0, acc_dv[m]);
      acc_dk[m] = O::mma(O::template tr8<D>(sg.q, qb * 32, 32 * m, lane), db0, acc_dk[m]);
      acc_dv[m] = O::mma(O::template tr8<D>(sg.dout, qb * 32 + 16, 32 * m, lane), pb1, acc_dv[m]);
      acc_dk[m] = O::mma(O::template tr8<D>(sg.q, qb * 32 + 16, 32 * m, lane), db1, acc_dk[m]);
    }
  }

  wait_vmem<0>();  // K and V of a tile that no row looks at are still on their way
  const int64_t krow = (((int64_t)it.e0 + j) * p.hkv + g) * D;
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    f32x16(&row)[D / 32] = pass == 0 ? acc_dk : acc_dv;
    if constexpr (S::QB == 2) {
      float* red = sm.red[kb];
      __syncthreads();  // the stages (pass 0) or the previous pass's buffer are free
      if (qb == 1) {
#pragma unroll
        for (int m = 0; m < D / 32; ++m)
#pragma unroll
          for (int r = 0; r < 16; ++r) red[(m * 16 + r) * 64 + lane] = row[m][r];
      }
      __syncthreads();
      if (qb == 0) {
#pragma unroll
        for (int m = 0; m < D / 32; ++m)
#pragma unroll
          for (int r = 0; r < 16; ++r) row[m][r] += red[(m * 16 + r) * 64 + lane];
      }
    }
    if (qb != 0) continue;
    if (it.slot >= 0) {
      float* part = p.part + ((((int64_t)it.slot * p.hkv + g) * 2 + pass) * 4 + kb) * (32 * D);
#pragma unroll
      for (int m = 0; m < D / 32; ++m)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          *reinterpret_cast<f32x4*>(part + ((m * 4 + r4) * 64 + lane) * 4) =
              f32x4{row[m][4 * r4], row[m][4 * r4 + 1], row[m][4 * r4 + 2], row[m][4 * r4 + 3]};
    } else if (j < it.ecap) {
      const float sc = pass == 0 ? p.scale : 1.f;
      T* dst = (pass == 0 ? p.dk : p.dv) + krow;
      const bool real = j < it.elen;
#pragma unroll
      for (int m = 0; m < D / 32; ++m)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          f32x4 v4 = f32x4{};
          if (real) v4 = f32x4{row[m][4 * r4] * sc, row[m][4 * r4 + 1] * sc, row[m][4 * r4 + 2] * sc, row[m][4 * r4 + 3] * sc};
          store4<T>(dst + 32 * m + 8 * r4 + 4 * hf, v4);
        }
    }
  }
}

// Adds the parts of key tiles whose rows were split, in part order.  A workgroup is one
// gradient of 32 keys: it reads the parts as they lie in the accumulators and turns the
// sums through LDS, so that a gradient's row is written by one workgroup and whole lines
// at a time (written 8 bytes a lane from 16 workgroups, 27 MB of parts took 17 us, now 5).
template <int D, typename T>
__device__ __forceinline__ void kv_sum_block(const CrossParams<T>& p, const float* kv_part, const CrossKvSplit* splits, int b) {
  constexpr int NQ = D / 8 / 4;  // groups of four registers a wave takes
  __shared__ T s_row[32][D + 16 / sizeof(T)];
  const int kb = b & 3;
  b >>= 2;
  const int g = b % p.hkv;
  b /= p.hkv;
  const int pass = b & 1;
  const CrossKvSplit sp = load_uniform(splits + (b >> 1));
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, hf = lane >> 5;
  const int j0 = sp.k0 + kb * 32;
  if (j0 >= sp.ecap) return;
  const int64_t stride = (int64_t)p.hkv * 2 * 4 * (32 * D);
  const float* part =
      kv_part + ((((int64_t)sp.slot0 * p.hkv + g) * 2 + pass) * 4 + kb) * (32 * D) + (wave * NQ * 64 + lane) * 4;
  f32x4 acc[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) acc[q] = f32x4{};
  constexpr int NP = 2;  // parts in flight
  for (int i = 0; i < sp.parts; i += NP, part += NP * stride) {
    f32x4 x[NP][NQ];
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int q = 0; q < NQ; ++q)
        if (i + n < sp.parts) x[n][q] = *reinterpret_cast<const f32x4*>(part + n * stride + q * 256);
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int q = 0; q < NQ; ++q)
        if (i + n < sp.parts) acc[q] += x[n][q];
  }
  const float sc = pass == 0 ? p.scale : 1.f;
  const bool real = j0 + (lane & 31) < sp.elen;
#pragma unroll
  for (int q = 0; q < NQ; ++q) store4<T>(&s_row[lane & 31][8 * (wave * NQ + q) + 4 * hf], real ? acc[q] * sc : f32x4{});
  __syncthreads();
  constexpr int CPR = D * (int)sizeof(T) / 16, V = 16 / (int)sizeof(T);
  T* dst = (pass == 0 ? p.dk : p.dv) + ((int64_t)(sp.e0 + j0) * p.hkv + g) * D;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  for (int i = threadIdx.x; i < 32 * CPR; i += 256) {
    const int r = i / CPR, c = (i % CPR) * V;
    if (j0 + r < sp.ecap)
      *reinterpret_cast<u32x4*>(dst + (int64_t)r * p.hkv * D + c) = *reinterpret_cast<const u32x4*>(&s_row[r][c]);
  }
}

// Both joins of a backward pass, in one launch: dQ's workgroups first.
template <int D, typename T>
__global__ __launch_bounds__(256) void cross_sum_kernel(CrossParams<T> p, const float* kv_part, const CrossSplit* splits,
                                                        const CrossKvSplit* kv_splits, int dq_blocks) {
  const int b = blockIdx.x;
  if (b < dq_blocks) dq_sum_block<D, T>(p, splits, b);
  else kv_sum_block<D, T>(p, kv_part, kv_splits, b - dq_blocks);
}

template <typename T>
CrossParams<T> params_of(const CrossLaunch& a) {
  CrossParams<T> p{};
  p.q = (const T*)a.q;
  p.k = (const T*)a.k;
  p.v = (const T*)a.v;
  p.dout = (const T*)a.dout;
  p.o_in = (const T*)a.o_in;
  p.o = (T*)a.out;
  p.dk = (T*)a.dk;
  p.dv = (T*)a.dv;
  p.lse = a.lse;
  p.lse_in = a.lse_in;
  p.items = a.items;
  p.kv_items = a.kv_items;
  p.kbeg = a.key_begin;
  p.kend = a.key_end;
  p.part = a.part;
  p.part_ml = a.part_ml;
  p.ndelta = a.ndelta;
  p.nlse2 = a.nlse2;
  p.ranges = a.ranges;
  p.hq = a.hq;
  p.hkv = a.hkv;
  p.G = a.hq / a.hkv;
  p.sumT = a.sumT;
  p.g_magic = (uint32_t)(0xffffffffu / (uint32_t)p.G) + 1u;
  p.scale = a.scale;
  p.scale_log2 = a.scale * kLog2e;
  return p;
}

// A launch with 3 KB of arguments takes the host 4.3 us, one with 500 bytes 3.5: few
// items, few splits or none of them have launches of their own.
template <int D, typename T, int N>
hipError_t launch_fwd_items(const CrossLaunch& a, const CrossParams<T>& p, hipStream_t s) {
  InlineItems<N> inl;
  for (int i = 0; i < N; ++i) inl.item[i] = !a.items && i < a.n_items ? a.host_items[i] : CrossItem{};
  const dim3 grid((unsigned)((int64_t)a.n_items * a.hkv));
  auto launch = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, grid, dim3(waves * 64), 0, s, p, inl); };
  if (a.tile_rows == kCrossFewRows) {
    if (a.key_begin) launch(cross_few_kernel<D, T, true, N>, kFewWaves<D, T>);
    else launch(cross_few_kernel<D, T, false, N>, kFewWaves<D, T>);
  } else {
    if (a.key_begin) launch(cross_fwd_kernel<D, T, true, N>, kWaves);
    else launch(cross_fwd_kernel<D, T, false, N>, kWaves);
  }
  return hipGetLastError();
}

template <int D, typename T, int N>
hipError_t launch_combine(const CrossLaunch& a, const CrossParams<T>& p, hipStream_t s) {
  CrossSplitList<N> sl;
  for (int i = 0; i < N; ++i) sl.split[i] = !a.splits && i < a.n_splits ? a.host_splits[i] : CrossSplit{};
  constexpr int RPB = 256 / (D / 4);
  const dim3 grid((unsigned)((int64_t)a.n_splits * a.hkv), (unsigned)((a.tile_rows + RPB - 1) / RPB));
  hipLaunchKernelGGL((cross_combine_kernel<D, T, N>), grid, dim3(256), 0, s, p, a.splits, sl, a.tile_rows);
  return hipGetLastError();
}

template <int D, typename T>
hipError_t launch_fwd_t(const CrossLaunch& a, hipStream_t s) {
  const CrossParams<T> p = params_of<T>(a);
  if (a.n_items > 0) {
    TimingScope t("pp_cross_attn_fwd", s);
    const hipError_t e = a.items ? launch_fwd_items<D, T, 1>(a, p, s)
                                 : a.n_items <= 16 ? launch_fwd_items<D, T, 16>(a, p, s)
                                                   : launch_fwd_items<D, T, kCrossInline>(a, p, s);
    if (e != hipSuccess) return e;
  }
  if (a.n_splits == 0) return hipSuccess;
  TimingScope t("pp_cross_attn_combine", s);
  if (a.splits || a.n_splits <= 8) return launch_combine<D, T, 8>(a, p, s);
  return launch_combine<D, T, kCrossInline / 2>(a, p, s);
}

template <int D, typename T>
hipError_t launch_bwd_t(const CrossLaunch& a, hipStream_t s) {
  const CrossParams<T> p = params_of<T>(a);
  hipError_t e = hipSuccess;
  if (a.n_items > 0) {
    TimingScope t("pp_cross_attn_dq", s);
    const dim3 grid((unsigned)((int64_t)a.n_items * a.hkv));
    if (a.key_begin) hipLaunchKernelGGL((cross_dq_kernel<D, T, true>), grid, dim3(kWaves * 64), 0, s, p);
    else hipLaunchKernelGGL((cross_dq_kernel<D, T, false>), grid, dim3(kWaves * 64), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.n_kv_items > 0) {
    TimingScope t("pp_cross_attn_dkdv", s);
    CrossParams<T> pk = p;
    pk.part = a.kv_part;
    const dim3 grid((unsigned)((int64_t)a.n_kv_items * a.hkv)), block(KvShape<D, T>::WAVES * 64);
    if (a.key_begin) hipLaunchKernelGGL((cross_dkdv_kernel<D, T, true>), grid, block, 0, s, pk);
    else hipLaunchKernelGGL((cross_dkdv_kernel<D, T, false>), grid, block, 0, s, pk);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  const int64_t dq_blocks = (int64_t)a.n_splits * a.hkv * (kCrossRows * (D / 4) / 256);
  const int64_t kv_blocks = (int64_t)a.n_kv_splits * 2 * a.hkv * 4;
  if (dq_blocks + kv_blocks > 0) {
    TimingScope t("pp_cross_attn_sum", s);
    hipLaunchKernelGGL((cross_sum_kernel<D, T>), dim3((unsigned)(dq_blocks + kv_blocks)), dim3(256), 0, s, p, a.kv_part, a.splits,
                       a.kv_splits, (int)dq_blocks);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_cross_fwd(const CrossLaunch& a, hipStream_t s) {
  if (a.dtype == kBF16) return a.head_dim == 128 ? launch_fwd_t<128, __bf16>(a, s) : launch_fwd_t<64, __bf16>(a, s);
  return a.head_dim == 128 ? launch_fwd_t<128, float>(a, s) : launch_fwd_t<64, float>(a, s);
}

hipError_t launch_cross_bwd(const CrossLaunch& a, hipStream_t s) {
  if (a.dtype == kBF16) return a.head_dim == 128 ? launch_bwd_t<128, __bf16>(a, s) : launch_bwd_t<64, __bf16>(a, s);
  return a.head_dim == 128 ? launch_bwd_t<128, float>(a, s) : launch_bwd_t<64, float>(a, s);
}

}  // namespace pp
