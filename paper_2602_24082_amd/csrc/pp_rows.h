// What the kernels of rows against keys share (cross attention, attention over the paged
// cache): fragments of bf16 and fp32 numbers for the bf16 MFMA, DMA of keys and values,
// and a row's running softmax.
#pragma once

#include "pp_device.h"

namespace pp {

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
  // elements col .. col + 3 of row r (col a multiple of 4)
  template <int D>
  static __device__ __forceinline__ f32x4 four(const __bf16* tile, int r, int col) {
    return __builtin_convertvector(*reinterpret_cast<const bf16x4*>(tile + r * D + (((col >> 3) ^ swz<D>(r)) << 3) + (col & 7)), f32x4);
  }
  // what the products take is below; in a word's magnitudes the rest carries into the sign's place
  static constexpr float kLimit = __builtin_inff();
  static constexpr uint32_t kMagnitude = 0x7fff7fffu, kCarry = 0x00800080u, kSign = 0x80008000u;
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
  template <int D>
  static __device__ __forceinline__ f32x4 four(const float* tile, int r, int col) {
    return *reinterpret_cast<const f32x4*>(tile + r * D + (((col >> 2) ^ swz<2 * D>(r)) << 2));
  }
  static constexpr float kLimit = 0x1.ffp127f;  // rounds to infinity as bf16
  static constexpr uint32_t kMagnitude = 0x7fffffffu, kCarry = 0x00808000u, kSign = 0x80000000u;
};

// Wave-cooperative DMA of NR rows of D elements of T (see TileDma).
template <typename T, int D, int NR>
using RowDma = TileDma<Ops<T>::template kRowD<D>, NR>;
template <bool ONCE = false, int RD, int NR, typename T>
__device__ __forceinline__ void dma_rows(const TileDma<RD, NR>& d, T* lds_tile, const T* src, int rows_valid) {
  d.template issue<ONCE>(reinterpret_cast<__bf16*>(lds_tile), reinterpret_cast<const __bf16*>(src), rows_valid);
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
      const float alpha = (m_ref == kNegInf) ? 1.f : fast_exp2(m_ref - m_new);  // nothing seen yet: l and O's finite elements are 0
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

}  // namespace pp
