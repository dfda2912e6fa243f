// Attention of new tokens over the paged cache, on gfx950: one token of each sequence, or a
// tree of drafted ones.
//
// Node i of sequence s sees the sequence's cached tokens and the nodes on its path to the
// root, itself included; the nodes' keys lie in the cache behind the cached ones:
//
//   S = Q K^T scale (visible keys),  P = softmax(S),  O = P V,  lse = ln sum exp(S)
//
// As in cross attention a row is one of the G query heads of a node, so that keys are read
// once for all of them.  The whole pages that a group's K sequences share are one more list
// of keys, seen by the rows of all K: they are read once a group, not once a response.  So
// there is an item for each group's shared keys and one for each sequence's own, and a unit
// is a block of 32 keys of an item, for one head and one tile of up to 64 rows (32 of fp32).
//
//   tree_plan     one workgroup: items, and their units dealt out evenly over all waves
//   tree_attn     a wave walks its run of units, through a ring of its own in LDS: no barrier
//                 anywhere.  Where an item ends or the run does, it leaves a partial result
//   tree_combine  joins a row's partial results, in order
//
// Bound by reading keys and values once.  A wave of RT x 32 rows reads each key fragment from
// LDS once and multiplies it RT times, so that only rows beyond a tile's read keys again.  No
// atomics on results: sums depend on lengths alone.  Products as in cross attention (pp_rows.h).

#include <hip/hip_runtime.h>

#include "pp_rows.h"
#include "pp_sample.h"

namespace pp {
namespace {

constexpr int kPlan = 1024;

__device__ __forceinline__ int64_t plan_scan64(int64_t x, int64_t* total) {
  __shared__ int64_t part[kPlan / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t s = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t y = __shfl_up(s, off, 64);
    if (lane >= off) s += y;
  }
  __syncthreads();
  if (lane == 63) part[wave] = s;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlan / 64; ++w) {
    before += w < wave ? part[w] : 0;
    all += part[w];
  }
  *total = all;
  return before + s - x;
}

// Items in the order of the groups: a group's shared keys, then its sequences' own.
__global__ __launch_bounds__(kPlan) void tree_plan_kernel(CacheView c, TreeShape t, const int32_t* slots, const int32_t* count,
                                                          const int32_t* shared, TreePlan out) {
  __shared__ int s_shared[kTreeSeqs], s_lead[kTreeSeqs], s_members[kTreeSeqs];
  __shared__ int64_t s_first[2 * kTreeSeqs];
  const int tid = threadIdx.x, items = t.n + t.groups;
  for (int g = tid; g < t.groups; g += kPlan) {
    s_shared[g] = s_lead[g] = 0x7fffffff;
    s_members[g] = 0;
  }
  __syncthreads();
  auto look = [&](int i, int& len, int& live) {  // nodes asked for of a sequence that is not sound
    const int slot = slots[i];
    len = live = 0;
    const int want = max(0, min(count ? count[i] : t.nodes, t.nodes));
    if (slot < 0 || want == 0) return 0;
    if (!c.has_slot(slot)) return want;
    const int64_t n = c.seq_len[slot], held = c.held[slot];
    if (!c.sound(n, held) || n + want > held << c.page_log2) return want;
    len = (int)n;
    live = want;
    return 0;
  };
  for (int i = tid; i < t.n; i += kPlan) {
    int len, live;
    look(i, len, live);
    out.live[i] = live;
    if (!live || !shared) continue;
    const int g = i / t.group;
    atomicMin(&s_shared[g], len);
    atomicMin(&s_lead[g], i);
    atomicAdd(&s_members[g], 1);
  }
  __syncthreads();
  for (int g = tid; g < t.groups; g += kPlan) {
    TreeItem it{};
    if (shared && s_members[g] > 1) {
      const int pages = max(0, min(shared[g], s_shared[g] >> c.page_log2));
      it.k1 = it.seen = pages << c.page_log2;
      it.blocks = (it.k1 + kTreeKeys - 1) / kTreeKeys;
      it.slot = slots[s_lead[g]];
    }
    it.seq = g * t.group;
    s_shared[g] = it.k1;
    out.items[g * (t.group + 1)] = it;
    s_first[g * (t.group + 1)] = (int64_t)it.blocks * t.tiles_shared * t.hkv;
  }
  __syncthreads();
  for (int i = tid; i < t.n; i += kPlan) {
    const int g = i / t.group, at = i + g + 1;
    int len, live;
    TreeItem it{};
    it.bad = look(i, len, live);
    it.seq = i;
    if (live) {
      it.slot = slots[i];
      it.k0 = s_shared[g];
      it.k1 = len + live;
      it.seen = len;
      it.blocks = (it.k1 - it.k0 + kTreeKeys - 1) / kTreeKeys;
    }
    out.items[at] = it;
    s_first[at] = (int64_t)it.blocks * t.tiles_own * t.hkv;
  }
  __syncthreads();
  constexpr int PER = 2 * kTreeSeqs / kPlan;
  int64_t w[PER], sum = 0, total;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int at = tid * PER + u;
    w[u] = at < items ? s_first[at] : 0;
    sum += w[u];
  }
  int64_t before = plan_scan64(sum, &total);
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int at = tid * PER + u;
    if (at < items) s_first[at] = out.first[at] = before;
    before += w[u];
  }
  __syncthreads();
  const int64_t run = max((int64_t)1, (total + t.waves - 1) / t.waves);
  if (tid == 0) {
    out.head[0] = total;
    out.head[1] = run;
  }
  for (int i = tid; i < t.waves; i += kPlan) {
    int lo = 0, hi = items - 1;  // the last item that starts at or before the wave's run (one with units)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_first[mid] <= i * run) lo = mid;
      else hi = mid - 1;
    }
    out.wave_item[i] = lo;
  }
}

// The number of tiles (of one head) ahead of an item's.
__device__ __forceinline__ int tiles_before(const TreeShape& t, int g, int member) {
  const int per = (t.tiles_shared + t.group * t.tiles_own) * t.hkv;
  return g * per + (member < 0 ? 0 : (t.tiles_shared + member * t.tiles_own) * t.hkv);
}

template <typename T>
struct TreeParams {
  const T* q;
  const T* k;
  const T* v;
  T* o;
  float* lse;
  const int32_t* parents;
  TreePlan plan;
  float* part;
  float* part_ml;
  float scale_log2;
};

// Of every node (lane) the nodes on its path to the root; false where a parent is none.
__device__ __forceinline__ uint64_t tree_paths(const int32_t* parents, int nodes, int lane, bool& fine) {
  fine = true;
  if (!parents) return lane == 63 ? ~0ull : (2ull << lane) - 1;
  int up = lane < nodes ? parents[lane] : -1;
  if (up >= lane || up < -1) {
    fine = false;
    up = -1;
  }
  uint64_t m = 1ull << lane;
  int ok = fine;
#pragma unroll
  for (int i = 0; i < 6; ++i) {  // the path's known part doubles
    const int from = up < 0 ? lane : up;
    const uint64_t m2 = __shfl(m, from, 64);
    const int up2 = __shfl(up, from, 64), ok2 = __shfl(ok, from, 64);
    if (up >= 0) {
      m |= m2;
      ok &= ok2;
      up = up2;
    }
  }
  fine = ok != 0;
  return m;
}

// One head's keys of a run of blocks.
struct TreeRun {
  int slot;    // whose table row
  int key, k1; // from key (16-key aligned) up to k1
  int blocks;
  int seen;    // all rows see the keys below
};

template <int D, typename T>
struct TreeRing {
  T kv[2][2][kTreeKeys * D];  // [stage][K / V]
};

// Walks a run with RT x 32 rows, row 32 t + ln of the tile in lanes ln and ln + 32, and leaves
// a partial result in rows `prow` and on.
template <int D, typename T, int RT>
__device__ __forceinline__ void tree_walk(const CacheView& c, const TreeShape& sh, const TreeParams<T>& p,
                                          __attribute__((address_space(3))) TreeRing<D, T>* ring,
                                          const TreeRun& run, int g, const int64_t* qrow, const uint64_t* tree, const bool* fine,
                                          int64_t prow) {
  using O = Ops<T>;
  using Frag = typename O::Frag;
  using Dma = RowDma<T, D, 16>;
  constexpr int NC = D / 16, HN = Dma::N, KN = 2 * HN;
  const int lane = threadIdx.x & 63, ln = lane & 31, hf = lane >> 5;
  const int lg = c.page_log2;
  Dma dma;
  dma.init(0, (int64_t)D * (sizeof(T) / 2), lane);

  // numbers of 64 pages at a time, a lane each
  const int last_page = (run.k1 - 1) >> lg;
  const int32_t* table = c.row(run.slot);
  bool bad = false;
  int pages = 0, page0 = run.key >> lg;
  auto refill = [&]() {
    const int at = page0 + lane;
    pages = at <= last_page ? table[at] : 0;
    if (!c.has_page(pages)) {
      bad = true;
      pages = 0;
    }
  };
  refill();
  auto page_of = [&](int key) {
    int at = (key >> lg) - page0;
    if (at >= 64) {
      page0 += at;
      at = 0;
      refill();
    }
    return __builtin_amdgcn_readlane(pages, at);
  };
  const int64_t page_rows = (int64_t)sh.hkv << lg;  // of a page, all heads
  struct Place {
    int64_t a, b;  // first row of the block's two halves of 16 keys
    int na, nb;    // keys of them
  };
  auto place = [&](int i) {
    const int key = run.key + kTreeKeys * i;
    Place x;
    x.a = page_of(key) * page_rows + ((int64_t)g << lg) + (key & (c.page_size - 1));
    x.na = min(16, run.k1 - key);
    x.nb = min(16, run.k1 - key - 16);
    x.b = x.a + 16;
    if (x.nb <= 0) {  // nothing there: what is read instead is not seen
      x.b = x.a;
      x.nb = x.na;
    } else if (c.page_size == 16) {
      x.b = page_of(key + 16) * page_rows + ((int64_t)g << lg);
    }
    return x;
  };
  auto issue = [&](int i, int kv, const T* pool, const Place& x) {
    T* tile = (T*)ring->kv[i & 1][kv];
    dma_rows<true>(dma, tile, pool + x.a * D, x.na);
    dma_rows<true>(dma, tile + 16 * D, pool + x.b * D, x.nb);
  };
  const int n = run.blocks;
  Place next = place(0);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (i < n) {
      if (i == 1) next = place(1);
      issue(i, 0, p.k, next);
      issue(i, 1, p.v, next);
    }
  }
  Frag qf[RT][NC];
  RowState<D> st[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    st[t].init();
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) qf[t][cc] = qrow[t] >= 0 ? O::load(p.q + qrow[t] + 16 * cc + 8 * hf) : Frag{};
  }
  for (int i = 0; i < n; ++i) {
    // in flight behind K(i): V(i), and K and V of block i + 1 if there is one
    if (i == 0) wait_vmem<0>();
    else if (i + 1 < n) wait_vmem<3 * KN>();
    else wait_vmem<KN>();
    asm volatile("" ::: "memory");
    const int k0 = run.key + kTreeKeys * i;
    const T* sK = (const T*)ring->kv[i & 1][0];
    const T* sV = (const T*)ring->kv[i & 1][1];
    f32x16 s[RT][1];
#pragma unroll
    for (int t = 0; t < RT; ++t) s[t][0] = f32x16{};
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) {
      const Frag kf = O::use(O::template row8<D>(sK, ln, 2 * cc + hf));
#pragma unroll
      for (int t = 0; t < RT; ++t) s[t][0] = O::mma(kf, qf[t][cc], s[t][0]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K's reads have returned
    if (i + 2 < n) {
      next = place(i + 2);
      issue(i + 2, 0, p.k, next);
    }
    if (k0 + kTreeKeys > run.seen) {
      const int d = run.seen - k0;  // keys of the block that all rows see
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        uint32_t word = bits_below32(d);
        if (d > -64) word |= d >= 0 ? (d < 32 ? (uint32_t)tree[t] << d : 0u) : (uint32_t)(tree[t] >> -d);
        word >>= 4 * hf;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][0][r] = keep_or_neginf(s[t][0][r], word, 8 * (r >> 2) + (r & 3));
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) st[t].probabilities(s[t], p.scale_log2);
    if (i + 2 < n) wait_vmem<3 * KN>();  // behind V(i): K and V of i + 1, K of i + 2
    else if (i + 1 < n) wait_vmem<2 * KN>();
    else wait_vmem<0>();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ch = 0; ch < 2; ++ch) {
      Frag pb[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) pb[t] = O::from_acc(s[t][0], ch);
#pragma unroll
      for (int m = 0; m < D / 32; ++m) {
        const Frag vf = O::template tr8<D>(sV, 16 * ch, 32 * m, lane);
#pragma unroll
        for (int t = 0; t < RT; ++t) st[t].o[m] = O::mma(vf, pb[t], st[t].o[m]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V's too
    if (i + 2 < n) issue(i + 2, 1, p.v, next);
  }
  bad = wave_any(bad);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const float l = half_swap_sum(st[t].l);
    if (qrow[t] < 0) continue;
    const int64_t row = prow + 32 * t + ln;
    float* o = p.part + row * D + 4 * hf;
#pragma unroll
    for (int m = 0; m < D / 32; ++m)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<f32x4*>(o + 32 * m + 8 * r4) =
            f32x4{st[t].o[m][4 * r4], st[t].o[m][4 * r4 + 1], st[t].o[m][4 * r4 + 2], st[t].o[m][4 * r4 + 3]};
    if (hf == 0) {
      p.part_ml[2 * row] = st[t].m_ref;
      p.part_ml[2 * row + 1] = bad || !fine[t] ? __builtin_nanf("") : l;
    }
  }
}

template <int D, typename T, int RT>
__global__ __launch_bounds__(64, 2) void tree_attn_kernel(CacheView c, TreeShape sh, TreeParams<T> p) {
  __shared__ __attribute__((aligned(1024))) TreeRing<D, T> ring;
  const int w = blockIdx.x, lane = threadIdx.x & 63, ln = lane & 31;
  const int64_t total = p.plan.head[0], run_len = p.plan.head[1];
  int64_t pos = w * run_len;
  const int64_t end = min(pos + run_len, total);
  if (pos >= end) return;
  int item = scalar_load(p.plan.wave_item + w);
  while (pos < end) {
    const TreeItem it = load_uniform(p.plan.items + item);
    const int64_t rel = pos - p.plan.first[item];
    const int grp = item / (sh.group + 1), member = item - grp * (sh.group + 1) - 1;
    const int tiles = member < 0 ? sh.tiles_shared : sh.tiles_own, rows = member < 0 ? sh.rows_shared : sh.rows_own;
    if (rel >= (int64_t)it.blocks * tiles * sh.hkv) {  // the next item (one without units, or this one's end)
      ++item;
      continue;
    }
    const int j = (int)(rel / it.blocks), b0 = (int)(rel - (int64_t)j * it.blocks);
    const int g = j / tiles, tile = j - g * tiles;
    TreeRun run;
    run.slot = it.slot;
    run.key = it.k0 + kTreeKeys * b0;
    run.k1 = it.k1;
    run.blocks = (int)min((int64_t)(it.blocks - b0), end - pos);
    run.seen = it.seen;
    bool path_fine = true;
    uint64_t path = 0;
    if (member >= 0) path = tree_paths(p.parents ? p.parents + (int64_t)it.seq * sh.nodes : nullptr, sh.nodes, lane, path_fine);
    int64_t qrow[RT];
    uint64_t tree[RT];
    bool fine[RT];
    const int in_tile = min(rows - tile * 32 * RT, 32 * RT);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = 32 * t + ln, row = tile * 32 * RT + r;
      const int node_at = row / sh.G, head = g * sh.G + (row - node_at * sh.G);
      const int m = member < 0 ? node_at / sh.nodes : 0, node = node_at - m * sh.nodes;
      const int seq = it.seq + m;
      const bool live = r < in_tile && node < p.plan.live[min(seq, sh.n - 1)];
      qrow[t] = live ? (((int64_t)seq * sh.nodes + node) * sh.hq + head) * D : -1;
      const int from = member < 0 ? 0 : min(node_at, 63);
      tree[t] = __shfl(path, from, 64);
      fine[t] = member < 0 || __shfl((int)path_fine, from, 64);
      if (member < 0) tree[t] = 0;
    }
    const int64_t prow = (int64_t)(tiles_before(sh, grp, member) + j + w) * sh.part_rows;
    tree_walk<D, T, RT>(c, sh, p, (__attribute__((address_space(3))) TreeRing<D, T>*)&ring, run, g, qrow, tree, fine, prow);
    pos += run.blocks;
  }
}

// A row is D / 4 lanes, four partial results' loads in flight: first those of its group's
// shared keys, then its own's.
template <int D, typename T>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeShape sh, TreeParams<T> p) {
  constexpr int LPR = D / 4, RPB = 256 / LPR, NP = 4;
  const int64_t out_row = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR;
  if (out_row >= (int64_t)sh.n * sh.nodes * sh.hq) return;
  const int col = (threadIdx.x % LPR) * 4;
  const int head = (int)(out_row % sh.hq);
  const int64_t tok = out_row / sh.hq;
  const int seq = (int)(tok / sh.nodes), node = (int)(tok - (int64_t)seq * sh.nodes);
  const int grp = seq / sh.group, member = seq - grp * sh.group;
  const int g = head / sh.G, h = head - g * sh.G;
  const int64_t run = p.plan.head[1];
  const int own = seq + grp + 1;
  f32x4 acc = f32x4{};
  float m = kNegInf, l = 0.f;
  if (node < p.plan.live[seq]) {
    auto join = [&](int item, int who, int tiles, int row) {
      const int blocks = p.plan.items[item].blocks;
      if (blocks == 0) return;
      const int j = g * tiles + row / sh.tile_rows;
      const int64_t from = p.plan.first[item] + (int64_t)j * blocks;
      const int64_t w0 = from / run, parts = (from + blocks - 1) / run - w0 + 1;
      int64_t prow = (tiles_before(sh, grp, who) + j + w0) * sh.part_rows + row % sh.tile_rows;
      for (int64_t n0 = 0; n0 < parts; n0 += NP, prow += (int64_t)NP * sh.part_rows) {
        f32x4 x[NP];
        float pm[NP], pl[NP];
#pragma unroll
        for (int n = 0; n < NP; ++n) {
          const bool on = n0 + n < parts;
          const int64_t r = prow + (on ? n : 0) * sh.part_rows;
          x[n] = *reinterpret_cast<const f32x4*>(p.part + r * D + col);
          pm[n] = p.part_ml[2 * r];
          pl[n] = on ? p.part_ml[2 * r + 1] : 0.f;
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
    };
    if (sh.tiles_shared) join(own - member - 1, -1, sh.tiles_shared, (member * sh.nodes + node) * sh.G + h);
    join(own, member, sh.tiles_own, node * sh.G + h);
  } else if (node < p.plan.items[own].bad) {
    l = __builtin_nanf("");
  }
  const bool some = l != 0.f;  // NaN: so is the row
  const float inv = some ? 1.f / l : 0.f;
  store4<T>(p.o + out_row * D + col, some ? acc * inv : f32x4{});
  if (col == 0) p.lse[(int64_t)head * sh.n * sh.nodes + tok] = some ? (m + __log2f(l)) * (1.0f / kLog2e) : 0.f;
}

template <int D, typename T>
hipError_t launch_tree_t(const CacheView& c, const TreeLaunch& a, hipStream_t s) {
  const TreeShape& sh = a.shape;
  TreeParams<T> p{};
  p.q = (const T*)a.q;
  p.k = (const T*)a.k;
  p.v = (const T*)a.v;
  p.o = (T*)a.o;
  p.lse = a.lse;
  p.parents = a.parents;
  p.plan = a.plan;
  p.part = a.part;
  p.part_ml = a.part_ml;
  p.scale_log2 = a.scale * kLog2e;
  {
    TimingScope t("pp_tree_attn_fwd", s);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(sh.waves), dim3(64), 0, s, c, sh, p); };
    if constexpr (kTreeTiles<T> > 1) {
      if (sh.tile_rows > 32) launch(tree_attn_kernel<D, T, kTreeTiles<T>>);
      else launch(tree_attn_kernel<D, T, 1>);
    } else {
      launch(tree_attn_kernel<D, T, 1>);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  TimingScope t("pp_tree_attn_combine", s);
  constexpr int RPB = 256 / (D / 4);
  const int64_t rows = (int64_t)sh.n * sh.nodes * sh.hq;
  hipLaunchKernelGGL((tree_combine_kernel<D, T>), dim3((unsigned)((rows + RPB - 1) / RPB)), dim3(256), 0, s, sh, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_attn(const CacheView& c, const TreeLaunch& a, hipStream_t s) {
  if (!a.planned) {
    TimingScope t("pp_tree_attn_plan", s);
    hipLaunchKernelGGL(tree_plan_kernel, dim3(1), dim3(kPlan), 0, s, c, a.shape, a.slots, a.count, a.shared, a.plan);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dtype == kBF16) return a.head_dim == 128 ? launch_tree_t<128, __bf16>(c, a, s) : launch_tree_t<64, __bf16>(c, a, s);
  return a.head_dim == 128 ? launch_tree_t<128, float>(c, a, s) : launch_tree_t<64, float>(c, a, s);
}

}  // namespace pp
