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
// is a block of keys of an item, for one head and one tile of its rows.
//
//   tree_plan     one workgroup: items, and their units dealt out evenly over all workers
//   tree_solo     up to 32 rows: a worker is a wave, which walks its run of units through a
//                 ring of its own in LDS, without a barrier anywhere
//   tree_team     more rows: a worker is four waves of 32 rows, which share a ring
//   tree_combine  joins a row's partial results, in order: a worker leaves one wherever an item
//                 ends or its run does
//
// Bound by reading keys and values once, and for teams by the matrix units as well.  No
// atomics: sums depend on lengths alone.  Products as in cross attention (pp_rows.h).

#include <hip/hip_runtime.h>

#include "pp_rows.h"
#include "pp_sample.h"

namespace pp {
namespace {

constexpr int kPlan = 1024;

// Exclusive sum of x over the workgroup's threads, and the whole; lanes by DPP (to the left by 1,
// 2, 4, 8 within rows of 16, then the rows' last lanes).
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t add_moved64(int64_t x) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
  return x + (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t plan_scan64(int64_t x, int64_t* total) {
  __shared__ int64_t part[kPlan / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t s = add_moved64<0x111, 0xf>(x);
  s = add_moved64<0x112, 0xf>(s);
  s = add_moved64<0x114, 0xf>(s);
  s = add_moved64<0x118, 0xf>(s);
  s = add_moved64<0x142, 0xa>(s);
  s = add_moved64<0x143, 0xc>(s);
  __syncthreads();
  if (lane == 63) part[wave] = s;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlan / 64; ++w) {
    const int64_t y = part[w];
    before += w < wave ? y : 0;
    all += y;
  }
  *total = all;
  return before + s - x;
}

// a / b for a >= 0, b > 0, short where both are
__device__ __forceinline__ int64_t div_floor(int64_t a, int64_t b) {
  if (((uint64_t)(a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
  return a / b;
}

// What a tile of an item counts as where units are dealt out: its blocks, and what its start
// costs (rows, pages and the first keys to fetch, a partial result to leave) in blocks.
__device__ __forceinline__ int units_of(int blocks) { return blocks ? blocks + kTreeStart : 0; }
__device__ __forceinline__ int rows_a_tile(const TreeKind& k) { return k.team ? kTeamRows : kSoloRows; }
__device__ __forceinline__ int tiles_of(int rows, const TreeKind& k) { return (rows + rows_a_tile(k) - 1) / rows_a_tile(k); }

// Items in the order of the groups: a group's shared keys, then its sequences' own.
__global__ __launch_bounds__(kPlan) void tree_plan_kernel(CacheView c, TreeShape t, const int32_t* slots, const int32_t* count,
                                                          const int32_t* shared, TreePlan out) {
  __shared__ int s_shared[kTreeSeqs], s_lead[kTreeSeqs], s_nodes[kTreeSeqs + 1], s_slot[kTreeSeqs];
  __shared__ int64_t s_units[2 * kTreeSeqs];
  __shared__ int64_t s_first[2 * kTreeSeqs];
  constexpr int PER = kTreeSeqs / kPlan;  // sequences a thread, next to each other
  const int tid = threadIdx.x, items = t.n + t.groups;
  const bool share = t.kind[0].tiles > 0;
  int slot_of[PER], len_of[PER], live_of[PER], bad_of[PER], lead = 0;
  int pages_of[PER];  // that groups tid, tid + kPlan .. share
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int g = tid + u * kPlan;
    if (!share || g >= t.groups) continue;
    s_shared[g] = s_lead[g] = 0x7fffffff;
    pages_of[u] = shared[g];
  }
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = tid * PER + u;
    slot_of[u] = i < t.n ? slots[i] : -1;
    bad_of[u] = slot_of[u] < 0 ? 0 : max(0, min(count ? count[i] : t.nodes, t.nodes));  // asked for
  }
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    len_of[u] = live_of[u] = 0;
    if (bad_of[u] == 0 || !c.has_slot(slot_of[u])) continue;
    const int64_t n = c.seq_len[slot_of[u]], held = c.held[slot_of[u]];
    if (!c.sound(n, held) || n + bad_of[u] > held << c.page_log2) continue;
    len_of[u] = (int)n;
    live_of[u] = bad_of[u];
    bad_of[u] = 0;
  }
  if (share) {
    // the nodes in use, group by group, are the rows of the shared keys
    int64_t sum = 0, total;
#pragma unroll
    for (int u = 0; u < PER; ++u) sum += live_of[u];
    lead = (int)plan_scan64(sum, &total);  // (its barriers cover s_shared's start as well)
    int at = lead;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int i = tid * PER + u;
      if (i <= t.n) s_nodes[i] = at;
      at += live_of[u];
      if (!live_of[u]) continue;
      s_slot[i] = slot_of[u];
      atomicMin(&s_shared[i / t.group], len_of[u]);
      atomicMin(&s_lead[i / t.group], i);
    }
    if (tid == 0) s_nodes[t.n] = (int)total;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int g = tid + u * kPlan;
      if (g >= t.groups) continue;
      TreeItem it{};
      const int nodes = s_nodes[min(t.n, (g + 1) * t.group)] - s_nodes[g * t.group];
      const int first = s_lead[g];
      // with one sequence in use there is nobody to share with
      if (nodes > 0 && first < t.n && s_nodes[first + 1] - s_nodes[first] < nodes) {
        const int pages = max(0, min(pages_of[u], s_shared[g] >> c.page_log2));
        it.k1 = it.seen = pages << c.page_log2;
        it.blocks = (it.k1 + t.kind[0].keys - 1) / t.kind[0].keys;
        it.slot = s_slot[first];
        it.rows = nodes * t.G;
      }
      it.seq = g * t.group;
      s_shared[g] = it.k1;
      out.items[g * (t.group + 1)] = it;
      s_units[g * (t.group + 1)] = (int64_t)tiles_of(it.rows, t.kind[0]) * units_of(it.blocks);
    }
    __syncthreads();
  } else {
    for (int g = tid; g < t.groups; g += kPlan) {
      TreeItem it{};
      it.seq = g * t.group;
      out.items[g * (t.group + 1)] = it;
      s_units[g * (t.group + 1)] = 0;
    }
  }
  int at = lead;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = tid * PER + u;
    if (i >= t.n) continue;
    const int g = i / t.group;
    TreeItem it{};
    it.bad = bad_of[u];
    it.seq = i;
    if (share) {
      const int base = s_nodes[g * t.group];
      it.row0 = at - base;
      for (int k = 0; k < live_of[u]; ++k) out.nodes[(int64_t)g * t.group * t.nodes + it.row0 + k] = i * t.nodes + k;
      at += live_of[u];
    }
    if (live_of[u]) {
      it.slot = slot_of[u];
      it.k0 = share ? s_shared[g] : 0;
      it.k1 = len_of[u] + live_of[u];
      it.seen = len_of[u];
      it.blocks = (it.k1 - it.k0 + t.kind[1].keys - 1) / t.kind[1].keys;
      it.rows = live_of[u] * t.G;
    }
    out.items[i + g + 1] = it;
    s_units[i + g + 1] = (int64_t)tiles_of(it.rows, t.kind[1]) * units_of(it.blocks);
  }
  for (int cls = 0; cls < 2; ++cls) {
    const bool takes[2] = {share && t.kind[0].team == cls, t.kind[1].team == cls};
    if (!takes[0] && !takes[1]) continue;
    __syncthreads();
    constexpr int PER_ITEM = 2 * kTreeSeqs / kPlan;
    int64_t w[PER_ITEM], sum = 0, total;
#pragma unroll
    for (int u = 0; u < PER_ITEM; ++u) {
      const int k = tid * PER_ITEM + u;
      w[u] = k < items && takes[k % (t.group + 1) != 0] ? s_units[k] * t.hkv : 0;
      sum += w[u];
    }
    int64_t before = plan_scan64(sum, &total);
#pragma unroll
    for (int u = 0; u < PER_ITEM; ++u) {
      const int k = tid * PER_ITEM + u;
      if (k < items) {
        s_first[k] = before;
        if (takes[k % (t.group + 1) != 0]) out.items[k].first = before;
      }
      before += w[u];
    }
    __syncthreads();
    const int64_t run = max((int64_t)1, (total + t.workers[cls] - 1) / t.workers[cls]);
    if (tid == 0) {
      out.head[4] = (int64_t)t.key;
      out.head[2 * cls] = total;
      out.head[2 * cls + 1] = run;
    }
    for (int i = tid; i < t.workers[cls]; i += kPlan) {
      int lo = 0, hi = items - 1;  // the last item that starts at or before the worker's run (one with units)
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_first[mid] <= i * run) lo = mid;
        else hi = mid - 1;
      }
      out.start_item[cls][i] = lo;
    }
  }
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

// Units in all that workers of a class take; none where ws holds no plan for this call.
__device__ __forceinline__ int64_t tree_units(const TreeShape& sh, const TreePlan& plan, int cls) {
  return (uint64_t)plan.head[4] == sh.key ? plan.head[2 * cls] : 0;
}

// A worker's run of units of one item, tile and head.
struct TreeRun {
  TreeItem it;
  int own;         // which kind of item
  int g, tile, tiles;  // kv-head, tile of rows, of how many
  int key, blocks; // from key on (a multiple of 16); blocks 0: the run ends ahead of the first
  int units;
  int64_t prow;    // row of its partial result
};

// The unit at `pos`, and the run from there to the item's end or `end`; `item` moves on to the
// one that has it.
__device__ __forceinline__ TreeRun tree_run(const TreeShape& sh, const TreePlan& plan, int cls, int worker, int64_t pos, int64_t end,
                                            int& item) {
  TreeRun r;
  for (;; ++item) {
    r.blocks = 0;
    if (item >= sh.n + sh.groups) return r;  // (never by a plan that is whole)
    const int grp = item / (sh.group + 1), member = item - grp * (sh.group + 1) - 1;
    r.own = member >= 0;
    const TreeKind& kind = sh.kind[r.own];
    if (kind.tiles == 0 || kind.team != cls) continue;
    r.it = load_uniform(plan.items + item);
    const int64_t rel = pos - r.it.first;
    const int units = units_of(r.it.blocks), tiles = tiles_of(r.it.rows, kind);
    r.tiles = tiles;
    if (rel >= (int64_t)units * tiles * sh.hkv) continue;  // none, or this one's end
    const int j = (int)div_floor(rel, units), u0 = (int)(rel - (int64_t)j * units);
    r.g = j / tiles;
    r.tile = j - r.g * tiles;
    r.units = (int)min((int64_t)(units - u0), end - pos);
    const int b0 = max(u0 - kTreeStart, 0);
    r.blocks = max(u0 + r.units - kTreeStart, 0) - b0;
    r.key = r.it.k0 + kind.keys * b0;
    const int64_t tile = (int64_t)((r.own ? r.it.seq : grp) * sh.hkv + r.g) * kind.tiles + r.tile;
    r.prow = kind.part0 + (tile + worker) * kind.part_rows;
    return r;
  }
}

// A lane's row of a tile: where its query lies (-1: no such row), and the nodes that it sees.
struct TreeRow {
  int64_t q;
  uint64_t tree;
  bool fine;
};
template <int D, typename T>
__device__ __forceinline__ TreeRow tree_row(const TreeShape& sh, const TreeParams<T>& p, const TreeRun& r, int row, uint64_t path,
                                            bool path_fine) {
  const int node_at = row / sh.G, head = r.g * sh.G + (row - node_at * sh.G);
  const bool live = row < r.it.rows;
  const int64_t tok = !live ? 0 : r.own ? (int64_t)r.it.seq * sh.nodes + node_at
                                       : p.plan.nodes[(int64_t)r.it.seq * sh.nodes + node_at];
  TreeRow x;
  x.q = live ? (tok * sh.hq + head) * D : -1;
  const uint64_t tree = __shfl(path, min(node_at, 63), 64);
  const int fine = __shfl((int)path_fine, min(node_at, 63), 64);
  x.tree = r.own ? tree : 0;
  x.fine = !r.own || fine;
  return x;
}

// Numbers of the pages that a wave reads, 64 at a time, a lane each.
struct TreePages {
  const int32_t* table;
  int last, page0, pages, lg, mask;
  int64_t page_rows, head_row;  // rows of a page (all heads), first of the head
  bool bad;

  __device__ __forceinline__ void init(const CacheView& c, const TreeShape& sh, const TreeRun& r) {
    table = c.row(r.it.slot);
    lg = c.page_log2;
    mask = c.page_size - 1;
    last = (r.it.k1 - 1) >> lg;
    page_rows = (int64_t)sh.hkv << lg;
    head_row = (int64_t)r.g << lg;
    bad = false;
    page0 = r.key >> lg;
    refill(c);
  }
  __device__ __forceinline__ void refill(const CacheView& c) {
    const int at = page0 + (threadIdx.x & 63);
    pages = at <= last ? table[at] : 0;
    if (!c.has_page(pages)) {
      bad = true;
      pages = 0;
    }
  }
  // the pool's row of a key (at most k1 - 1, and never behind an earlier one's page)
  __device__ __forceinline__ int64_t row(const CacheView& c, int key) {
    int at = (key >> lg) - page0;
    if (at >= 64) {
      page0 += at;
      at = 0;
      refill(c);
    }
    return __builtin_amdgcn_readlane(pages, at) * page_rows + head_row + (key & mask);
  }
};

// Scores of a block of 32 keys from k0 on: those that the row does not see become -inf.
__device__ __forceinline__ void tree_mask(f32x16& s, int k0, int seen, uint64_t tree, int hf) {
  const int d = seen - k0;  // keys of the block that all rows see
  uint32_t word = bits_below32(d);
  if (d > -64 && d < 32) word |= d >= 0 ? (uint32_t)tree << d : (uint32_t)(tree >> -d);
  word >>= 4 * hf;
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = keep_or_neginf(s[r], word, 8 * (r >> 2) + (r & 3));
}

// A probability of 0 keeps a number out of P V, but no infinity and no NaN.  So where a row does not see
// all keys of a block, values that are not finite (or not so as bf16) leave it ahead of the product, and
// a row that sees one adds infinity or NaN, whatever its probability.
//
// Whether N elements at `tile` have one, by a wave.
template <int N, typename T>
__device__ __forceinline__ bool not_finite(const T* tile, int lane) {
  typedef uint32_t Words __attribute__((ext_vector_type(4)));
  using O = Ops<T>;
  const Words* at = reinterpret_cast<const Words*>(tile) + lane;
  uint32_t carry = 0;
#pragma unroll
  for (int i = 0; i < (int)(N * sizeof(T) / 1024); ++i) {
    const Words w = at[64 * i];
#pragma unroll
    for (int e = 0; e < 4; ++e) carry |= (w[e] & O::kMagnitude) + O::kCarry;
  }
  return wave_any((carry & O::kSign) != 0);
}
// Adds what the row sees of them among KEYS keys from k0 on.
template <int D, int KEYS, typename T>
__device__ __forceinline__ void add_not_finite(RowState<D>& st, const T* sV, int k0, int seen, uint64_t tree, int hf) {
#pragma unroll 1
  for (int k = 0; k < KEYS; ++k) {
    const int node = k0 + k - seen;
    const bool sees = node < 0 || (node < 64 && (tree >> node & 1));
#pragma unroll
    for (int m = 0; m < D / 32; ++m)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 v = Ops<T>::template four<D>(sV, k, 32 * m + 8 * r4 + 4 * hf);
#pragma unroll
        for (int e = 0; e < 4; ++e) st.o[m][4 * r4 + e] += sees && !(fabsf(v[e]) < Ops<T>::kLimit) ? v[e] * __builtin_inff() : 0.f;
      }
  }
}
// Makes them 0.
template <int N, typename T>
__device__ __forceinline__ void drop_not_finite(T* tile, int lane) {
  for (int i = lane; i < N; i += 64)
    if (!(fabsf((float)tile[i]) < Ops<T>::kLimit)) tile[i] = (T)0.f;
}

template <int D, typename T>
__device__ __forceinline__ void leave_partial(const TreeParams<T>& p, const RowState<D>& st, const TreeRow& row, int64_t at, bool bad,
                                              int hf) {
  const float l = half_swap_sum(st.l);
  if (row.q < 0) return;
  float* o = p.part + at * D + 4 * hf;
#pragma unroll
  for (int m = 0; m < D / 32; ++m)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      *reinterpret_cast<f32x4*>(o + 32 * m + 8 * r4) =
          f32x4{st.o[m][4 * r4], st.o[m][4 * r4 + 1], st.o[m][4 * r4 + 2], st.o[m][4 * r4 + 3]};
  if (hf == 0) {
    p.part_ml[2 * at] = st.m_ref;
    p.part_ml[2 * at + 1] = bad || !row.fine ? __builtin_nanf("") : l;
  }
}

// Stages of keys and values.  The DMA goes by byte addresses in LDS: a generic pointer,
// carried round the kernels' outer loops, is checked for null where it is turned back, in a
// form that the compiler cannot encode.
template <typename T, int S, int N>
struct TreeRing {
  T kv[S][2][N];  // [stage][K / V]
};
template <typename X>
__device__ __forceinline__ __attribute__((address_space(3))) X* in_lds(X* x) {
  return (__attribute__((address_space(3))) X*)x;
}
// Rows of a tile at LDS byte `to` (the DMA's first row included), as dma_rows; ONCE: nobody reads
// them again.
template <bool ONCE, int RD, int NR, typename T>
__device__ __forceinline__ void dma_rows_at(const TileDma<RD, NR>& d, unsigned to, const T* src, int rows_valid) {
  using Dma = TileDma<RD, NR>;
  const char* base = reinterpret_cast<const char*>(src);
#pragma unroll
  for (int i = 0; i < Dma::N; ++i) {
    const uint32_t rs = (uint32_t)min(d.row_of(i), rows_valid - 1);
    lds_dma16_at<ONCE>(base + (rs * d.stride_b + d.chunk_b(i)), to + i * 1024);
  }
}

// Up to 32 rows, row ln in lanes ln and ln + 32.  BRANCH: sequences have several nodes, so that one
// row may see a key that another does not (the look at values takes single tokens from 22.4 to 23.1 us).
template <int D, typename T, bool BRANCH>
__global__ __launch_bounds__(64, 2) void tree_solo_kernel(CacheView c, TreeShape sh, TreeParams<T> p) {
  using O = Ops<T>;
  using Frag = typename O::Frag;
  using Dma = RowDma<T, D, 16>;
  constexpr int NC = D / 16, KN = 2 * Dma::N;
  __shared__ __attribute__((aligned(1024))) TreeRing<T, 2, kSoloKeys * D> smem;
  auto* ring = in_lds(&smem);
  const int worker = blockIdx.x, lane = threadIdx.x & 63, ln = lane & 31, hf = lane >> 5;
  const int64_t total = tree_units(sh, p.plan, 0), run_len = p.plan.head[1];
  if (total == 0) return;  // (without a plan the run's length is anything)
  int64_t pos = worker * run_len;
  const int64_t end = min(pos + run_len, total);
  if (pos >= end) return;
  int item = scalar_load(p.plan.start_item[0] + worker);
  Dma dma;
  dma.init(0, (int64_t)D * (sizeof(T) / 2), lane);
  while (pos < end) {
    const TreeRun r = tree_run(sh, p.plan, 0, worker, pos, end, item);
    if (r.blocks == 0) break;  // (the run's end)
    TreePages pages;
    pages.init(c, sh, r);
    struct Place {
      int64_t a, b;  // first row of the block's two halves of 16 keys
      int na, nb;    // keys of them
    };
    auto place = [&](int i) {
      const int key = r.key + kSoloKeys * i;
      Place x;
      x.a = pages.row(c, key);
      x.na = min(16, r.it.k1 - key);
      x.nb = min(16, r.it.k1 - key - 16);
      x.b = x.a + 16;
      if (x.nb <= 0) {  // nothing there: what is read instead is not seen
        x.b = x.a;
        x.nb = x.na;
      } else if (c.page_size == 16) {
        x.b = pages.row(c, key + 16);
      }
      return x;
    };
    auto issue = [&](int i, int kv, const T* pool, const Place& x) {
      const unsigned tile = (unsigned)(uintptr_t)&ring->kv[i & 1][kv][0];
      dma_rows_at<true>(dma, tile, pool + x.a * D, x.na);
      dma_rows_at<true>(dma, tile + 16 * D * sizeof(T), pool + x.b * D, x.nb);
    };
    const int n = r.blocks;
    Place next = place(0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (i < n) {
        if (i == 1) next = place(1);
        issue(i, 0, p.k, next);
        issue(i, 1, p.v, next);
      }
    }
    bool path_fine = true;
    uint64_t path = 0;
    if (r.own) path = tree_paths(p.parents ? p.parents + (int64_t)r.it.seq * sh.nodes : nullptr, sh.nodes, lane, path_fine);
    const TreeRow row = tree_row<D>(sh, p, r, ln, path, path_fine);
    Frag qf[NC];
    RowState<D> st;
    st.init();
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) qf[cc] = row.q >= 0 ? O::load(p.q + row.q + 16 * cc + 8 * hf) : Frag{};
    for (int i = 0; i < n; ++i) {
      // in flight behind K(i): V(i), and K and V of block i + 1 if there is one
      if (i == 0) wait_vmem<0>();
      else if (i + 1 < n) wait_vmem<3 * KN>();
      else wait_vmem<KN>();
      asm volatile("" ::: "memory");
      const int k0 = r.key + kSoloKeys * i;
      const T* sK = (const T*)ring->kv[i & 1][0];
      T* sV = (T*)ring->kv[i & 1][1];
      f32x16 s[1] = {f32x16{}};
#pragma unroll
      for (int cc = 0; cc < NC; ++cc) s[0] = O::mma(O::use(O::template row8<D>(sK, ln, 2 * cc + hf)), qf[cc], s[0]);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K's reads have returned
      if (i + 2 < n) {
        next = place(i + 2);
        issue(i + 2, 0, p.k, next);
      }
      const bool masked = k0 + kSoloKeys > r.it.seen;
      if (masked) tree_mask(s[0], k0, r.it.seen, row.tree, hf);
      st.probabilities(s, p.scale_log2);
      if (i + 2 < n) wait_vmem<3 * KN>();  // behind V(i): K and V of i + 1, K of i + 2
      else if (i + 1 < n) wait_vmem<2 * KN>();
      else wait_vmem<0>();
      asm volatile("" ::: "memory");
      if constexpr (BRANCH) {
        if (masked && r.own && not_finite<kSoloKeys * D>(sV, lane)) {
          add_not_finite<D, kSoloKeys>(st, sV, k0, r.it.seen, row.tree, hf);
          drop_not_finite<kSoloKeys * D>(sV, lane);
        }
      }
#pragma unroll
      for (int ch = 0; ch < 2; ++ch) {
        const Frag pb = O::from_acc(s[0], ch);
#pragma unroll
        for (int m = 0; m < D / 32; ++m) st.o[m] = O::mma(O::template tr8<D>(sV, 16 * ch, 32 * m, lane), pb, st.o[m]);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V's too
      if (i + 2 < n) issue(i + 2, 1, p.v, next);
    }
    leave_partial<D>(p, st, row, r.prow + ln, wave_any(pages.bad), hf);
    pos += r.units;
  }
}

// Waits until block t of n has landed, PER loads each, with S - 2 later ones in flight at most.
template <int S, int PER>
__device__ __forceinline__ void wait_block(int t, int n) {
  if constexpr (S > 2) {
    if (t + S - 2 < n) {
      wait_vmem<(S - 2) * PER>();
      return;
    }
    wait_block<S - 1, PER>(t, n);
  } else {
    wait_vmem<0>();
  }
}

// Tiles of 128 rows: four waves of 32, which fetch a quarter of every block each.
template <int D, typename T, bool BRANCH>
__global__ __launch_bounds__(kTeamWaves * 64, (kTreeTeam<D, T>)) void tree_team_kernel(CacheView c, TreeShape sh, TreeParams<T> p) {
  using O = Ops<T>;
  using Frag = typename O::Frag;
  constexpr int BN = kTeamKeys<D, T>, S = kTeamStages<D, T>, KB = BN / 32, RPW = BN / kTeamWaves, NC = D / 16, NI = KB * NC, PD = 3;
  using Dma = RowDma<T, D, RPW>;
  __shared__ __attribute__((aligned(1024))) TreeRing<T, S, BN * D> smem;
  auto* ring = in_lds(&smem);
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t total = tree_units(sh, p.plan, 1), run_len = p.plan.head[3];
  if (total == 0) return;
  // Workgroups go round the 8 XCDs: where an item may have several tiles an XCD takes a stretch of
  // workers, so that tiles, which walk the same keys at about the same time, meet in one L2 (groups of
  // eight sequences with eight nodes: 143 -> 141 us; alone, long trees would lose 1 us).
  const bool meet = max(sh.kind[0].team ? sh.kind[0].tiles : 0, sh.kind[1].team ? sh.kind[1].tiles : 0) > 1;
  const int stretch = (__builtin_amdgcn_readfirstlane((int)div_floor(total + run_len - 1, run_len)) + 7) >> 3;
  if (meet && (int)(blockIdx.x >> 3) >= stretch) return;
  const int worker = meet ? (int)(blockIdx.x & 7) * stretch + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
  int64_t pos = worker * run_len;
  const int64_t end = min(pos + run_len, total);
  if (pos >= end) return;
  int item = scalar_load(p.plan.start_item[1] + worker);
  Dma dma;
  dma.init(wave * RPW, (int64_t)D * (sizeof(T) / 2), lane);
  for (bool first = true; pos < end; first = false) {
    const TreeRun r = tree_run(sh, p.plan, 1, worker, pos, end, item);
    if (r.blocks == 0) break;  // (the run's end)
    TreePages pages;
    pages.init(c, sh, r);
    auto issue = [&](int t, int stage) {
      // this wave's rows of the block lie in one page; past the last key it fetches the block's first ones again
      const int key = r.key + BN * t, mine = key + wave * RPW;
      const int64_t at = pages.row(c, mine < r.it.k1 ? mine : key);
      const int rows = mine < r.it.k1 ? min(RPW, r.it.k1 - mine) : min(RPW, r.it.k1 - key);
      const int64_t base = (at - wave * RPW) * D;  // (the DMA adds the wave's first row)
      const unsigned tile = (unsigned)(uintptr_t)&ring->kv[stage][0][wave * RPW * D];
      if (r.tiles == 1) {  // nobody else reads them: past the L2 (long trees 139 -> 124 us, groups 141 -> 133)
        dma_rows_at<true>(dma, tile, p.k + base, wave * RPW + rows);
        dma_rows_at<true>(dma, tile + BN * D * sizeof(T), p.v + base, wave * RPW + rows);
      } else {
        dma_rows_at<false>(dma, tile, p.k + base, wave * RPW + rows);
        dma_rows_at<false>(dma, tile + BN * D * sizeof(T), p.v + base, wave * RPW + rows);
      }
    };
    if (!first) __syncthreads();  // the ring is free
    const int n = r.blocks;
#pragma unroll
    for (int t = 0; t < S - 1; ++t)
      if (t < n) issue(t, t);
    bool path_fine = true;
    uint64_t path = 0;
    if (r.own) path = tree_paths(p.parents ? p.parents + (int64_t)r.it.seq * sh.nodes : nullptr, sh.nodes, lane, path_fine);
    const TreeRow row = tree_row<D>(sh, p, r, r.tile * kTeamRows + wave * 32 + ln, path, path_fine);
    const bool some = wave_any(row.q >= 0);
    Frag qf[NC];
    RowState<D> st;
    st.init();
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) qf[cc] = row.q >= 0 ? O::load(p.q + row.q + 16 * cc + 8 * hf) : Frag{};
    int stage = 0;
    for (int t = 0; t < n; ++t) {
      if (t == 0) wait_vmem<0>();  // (Q's loads as well)
      else wait_block<S, 2 * Dma::N>(t, n);
      lds_barrier();  // block t has landed for every wave; the stage of block t - 1 is free
      if (t + S - 1 < n) issue(t + S - 1, stage == 0 ? S - 1 : stage - 1);
      const T* sK = (const T*)ring->kv[stage][0];
      T* sV = (T*)ring->kv[stage][1];
      stage = stage == S - 1 ? 0 : stage + 1;
      const int k0 = r.key + BN * t;
      const bool masked = k0 + BN > r.it.seen;
      if constexpr (BRANCH) {
        if (masked && r.own && __syncthreads_or(not_finite<RPW * D>(sV + wave * RPW * D, lane))) {
          if (some) add_not_finite<D, BN>(st, sV, k0, r.it.seen, row.tree, hf);
          __syncthreads();
          drop_not_finite<RPW * D>(sV + wave * RPW * D, lane);
          __syncthreads();
        }
      }
      if (!some) continue;
      f32x16 s[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] = f32x16{};
      Frag a[PD + 1];  // K's fragments, read ahead
#pragma unroll
      for (int x = 0; x < PD; ++x) a[x] = O::use(O::template row8<D>(sK, (x / NC) * 32 + ln, 2 * (x % NC) + hf));
#pragma unroll
      for (int x = 0; x < NI; ++x) {
        if (x + PD < NI) a[(x + PD) % (PD + 1)] = O::use(O::template row8<D>(sK, ((x + PD) / NC) * 32 + ln, 2 * ((x + PD) % NC) + hf));
        s[x / NC] = O::mma(a[x % (PD + 1)], qf[x % NC], s[x / NC]);
      }
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int x = 0; x < PD; ++x) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 1, 0);
#pragma unroll
        for (int x = 0; x < NI; ++x) {
          if (x + PD < NI) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 1, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
        }
      }
      if (masked) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) tree_mask(s[kb], k0 + 32 * kb, r.it.seen, row.tree, hf);
      }
      st.probabilities(s, p.scale_log2);
#pragma unroll
      for (int ch = 0; ch < 2 * KB; ++ch) {
        const Frag pb = O::from_acc(s[ch >> 1], ch & 1);
#pragma unroll
        for (int m = 0; m < D / 32; ++m) st.o[m] = O::mma(O::template tr8<D>(sV, 16 * ch, 32 * m, lane), pb, st.o[m]);
      }
    }
    // a page that is none may be another wave's
    const bool bad = __syncthreads_or(pages.bad);
    leave_partial<D>(p, st, row, r.prow + wave * 32 + ln, bad, hf);
    pos += r.units;
  }
}

// Where a row's partial results of one item lie.
struct TreeParts {
  int64_t row, n, stride;
};
__device__ __forceinline__ TreeParts tree_parts(const TreeShape& sh, int64_t run, int kind_of, const TreeItem& it, int who, int g,
                                                int row) {
  const TreeKind& kind = sh.kind[kind_of];
  const int per = rows_a_tile(kind), tile = row / per, j = g * tiles_of(it.rows, kind) + tile;
  const int64_t from = it.first + (int64_t)j * units_of(it.blocks) + kTreeStart, w0 = div_floor(from, run);
  TreeParts p;
  p.n = it.blocks ? div_floor(from + it.blocks - 1, run) - w0 + 1 : 0;
  p.stride = kind.part_rows;
  p.row = kind.part0 + ((int64_t)(who * sh.hkv + g) * kind.tiles + tile + w0) * kind.part_rows + row % per;
  return p;
}

// Where a row's partial results lie (its group's shared keys', then its own's) takes a few
// divisions, which one thread a row does ahead; then a row is D / 4 lanes, with four partial
// results' loads in flight.  Bound by reading them: 32 768 rows of head size 128 with four or five
// each, 80 MB, take 17 us.
template <int D, typename T>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeShape sh, TreeParams<T> p) {
  constexpr int LPR = D / 4, RPB = 256 / LPR, NP = 4;
  struct Row {
    int64_t lse;  // where its lse goes; < 0: no such row
    TreeParts a, b;
    float l;      // NaN: a node of a bad sequence
  };
  __shared__ Row s_row[RPB];
  const int64_t row0 = (int64_t)blockIdx.x * RPB, rows = (int64_t)sh.n * sh.nodes * sh.hq;
  if (threadIdx.x < RPB) {
    Row x;
    x.lse = -1;
    x.l = 0.f;
    x.a = x.b = TreeParts{0, 0, 0};
    const int64_t out_row = row0 + threadIdx.x;
    if (out_row < rows) {
      const int tok = (int)div_floor(out_row, sh.hq), head = (int)(out_row - (int64_t)tok * sh.hq);
      const int seq = tok / sh.nodes, node = tok - seq * sh.nodes, grp = seq / sh.group;
      const int g = head / sh.G, h = head - g * sh.G;
      const TreeItem mine = p.plan.items[seq + grp + 1], all = p.plan.items[grp * (sh.group + 1)];
      const int64_t run_all = p.plan.head[2 * sh.kind[0].team + 1], run_own = p.plan.head[2 * sh.kind[1].team + 1];
      x.lse = (int64_t)head * sh.n * sh.nodes + tok;
      if ((uint64_t)p.plan.head[4] != sh.key) {
        x.l = __builtin_nanf("");
      } else if (node * sh.G < mine.rows) {
        if (all.blocks) x.a = tree_parts(sh, run_all, 0, all, grp, g, (mine.row0 + node) * sh.G + h);
        x.b = tree_parts(sh, run_own, 1, mine, seq, g, node * sh.G + h);
      } else if (node < mine.bad) {
        x.l = __builtin_nanf("");
      }
    }
    s_row[threadIdx.x] = x;
  }
  __syncthreads();
  const int col = (threadIdx.x % LPR) * 4;
  const int at = threadIdx.x / LPR;
  const Row& x = s_row[at];
  if (x.lse < 0) return;
  const TreeParts a = x.a, b = x.b;
  f32x4 acc = f32x4{};
  float m = kNegInf, l = x.l;
  const int64_t parts = a.n + b.n;
  for (int64_t n0 = 0; n0 < parts; n0 += NP) {
    f32x4 y[NP];
    float pm[NP], pl[NP];
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const int64_t k = n0 + n < parts ? n0 + n : 0;
      const int64_t r = k < a.n ? a.row + k * a.stride : b.row + (k - a.n) * b.stride;
      y[n] = *reinterpret_cast<const f32x4*>(p.part + r * D + col);
      pm[n] = p.part_ml[2 * r];
      pl[n] = n0 + n < parts ? p.part_ml[2 * r + 1] : 0.f;
    }
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      if (pl[n] == 0.f) continue;  // a part without a visible key
      const float mn = fmaxf(m, pm[n]);
      const float c = m == kNegInf ? 0.f : fast_exp2(m - mn), d = fast_exp2(pm[n] - mn);
      l = l * c + pl[n] * d;
      acc = acc * c + y[n] * d;
      m = mn;
    }
  }
  const bool some = l != 0.f;  // NaN: so is the row
  const float inv = some ? 1.f / l : 0.f;
  store4<T>(p.o + (row0 + at) * D + col, some ? acc * inv : f32x4{});
  if (col == 0) p.lse[x.lse] = some ? (m + __log2f(l)) * (1.0f / kLog2e) : 0.f;
}

template <int D, typename T, bool BRANCH>
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
  bool takes[2] = {false, false};
  for (const TreeKind& k : sh.kind)
    if (k.tiles) takes[k.team] = true;
  if (takes[1]) {
    TimingScope t("pp_tree_attn_team", s);
    hipLaunchKernelGGL((tree_team_kernel<D, T, BRANCH>), dim3(sh.workers[1]), dim3(kTeamWaves * 64), 0, s, c, sh, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (takes[0]) {
    TimingScope t("pp_tree_attn_solo", s);
    hipLaunchKernelGGL((tree_solo_kernel<D, T, BRANCH>), dim3(sh.workers[0]), dim3(64), 0, s, c, sh, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  TimingScope t("pp_tree_attn_combine", s);
  constexpr int RPB = 256 / (D / 4);
  const int64_t rows = (int64_t)sh.n * sh.nodes * sh.hq;
  hipLaunchKernelGGL((tree_combine_kernel<D, T>), dim3((unsigned)((rows + RPB - 1) / RPB)), dim3(256), 0, s, sh, p);
  return hipGetLastError();
}

template <int D, typename T>
hipError_t launch_tree_d(const CacheView& c, const TreeLaunch& a, hipStream_t s) {
  return a.shape.nodes > 1 ? launch_tree_t<D, T, true>(c, a, s) : launch_tree_t<D, T, false>(c, a, s);
}

}  // namespace

hipError_t launch_tree_attn(const CacheView& c, const TreeLaunch& a, hipStream_t s) {
  if (!a.planned) {
    TimingScope t("pp_tree_attn_plan", s);
    hipLaunchKernelGGL(tree_plan_kernel, dim3(1), dim3(kPlan), 0, s, c, a.shape, a.slots, a.count, a.shared, a.plan);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dtype == kBF16) return a.head_dim == 128 ? launch_tree_d<128, __bf16>(c, a, s) : launch_tree_d<64, __bf16>(c, a, s);
  return a.head_dim == 128 ? launch_tree_d<128, float>(c, a, s) : launch_tree_d<64, float>(c, a, s);
}

}  // namespace pp
