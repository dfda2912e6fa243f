// Paged cache of keys and values: the pages of sampled sequences, on the device.
//
// A sequence (slot) s lists held_s pages in its row of the table; its token t lies in page
// table[s][t / page_size], row t % page_size.  A page may be listed by several sequences
// (the whole pages of a group's prompt): refs counts how often.  A page with no reference is
// free; whoever needs pages gets the lowest-numbered free ones, in the order of the call's
// entries and of their pages, so results do not depend on scheduling.
//
//   reserve   one workgroup: what every entry needs, a scan, the free pages, the table
//   fork      the same for the one page that an entry needs (its source's last, if partial),
//             then table rows, references and the partial pages' rows in every layer
//   free      a workgroup a slot
//   append    a wave a token: rotary embedding of its keys and queries, rows into the page
//   accept    the kept nodes of a drafted tree move together: lengths first (one workgroup),
//             then a workgroup a (slot, layer, head) reads all of its rows ahead of writing
//   compact   one workgroup numbers the moves, then pages are copied and table rows renumbered
//   shared    leading pages that the sequences of a group have in common
//
// Bound by the rows that they copy, and by launches where those are few.  What a device array
// says (slots, counts, lengths, page numbers) is checked here before it becomes an address.

#include <hip/hip_runtime.h>

#include "pp_device.h"
#include "pp_sample.h"

namespace pp {
namespace {

constexpr int kPlan = 1024;  // threads of the kernels that plan, one workgroup each
// Rows that the next kernel does not read, or hardly: they leave the L2 clean, which a kernel's
// end would else wait for (prompts of 102 MB: 45 -> 38 us a call).
template <typename T, typename Vec>
__device__ __forceinline__ void store_once(T* to, const Vec& x) {
  typedef uint32_t Words __attribute__((ext_vector_type(sizeof(Vec) / 4)));
  __builtin_nontemporal_store(__builtin_bit_cast(Words, x), reinterpret_cast<Words*>(to));
}

// 16-byte chunks by a workgroup of 256, four loads of a thread in flight.
template <bool ONCE>
__device__ __forceinline__ void copy_chunks(f32x4* to, const f32x4* from, int chunks) {
  constexpr int U = 4;
  for (int i0 = threadIdx.x; i0 < chunks; i0 += 256 * U) {
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + 256 * u < chunks) v[u] = from[i0 + 256 * u];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + 256 * u >= chunks) continue;
      if constexpr (ONCE) store_once(to + i0 + 256 * u, v[u]);
      else to[i0 + 256 * u] = v[u];
    }
  }
}

constexpr int kFreeRun = 8;  // pages a thread looks at in a row

// Exclusive sum of x over the workgroup's threads, and the whole; lanes by DPP (to the left by 1,
// 2, 4, 8 within rows of 16, then the rows' last lanes).
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_moved(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int plan_scan(int x, int* total) {
  __shared__ int part[kPlan / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = add_moved<0x111, 0xf>(x);
  s = add_moved<0x112, 0xf>(s);
  s = add_moved<0x114, 0xf>(s);
  s = add_moved<0x118, 0xf>(s);
  s = add_moved<0x142, 0xa>(s);
  s = add_moved<0x143, 0xc>(s);
  __syncthreads();  // the previous call's reads of `part`
  if (lane == 63) part[wave] = s;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlan / 64; ++w) {
    const int y = part[w];
    before += w < wave ? y : 0;
    all += y;
  }
  *total = all;
  return before + s - x;
}

// The refs of kFreeRun pages from p on that satisfy `want`, as bits.
template <typename Want>
__device__ __forceinline__ unsigned ref_bits(const CacheView& c, int64_t p, Want&& want) {
  int r[kFreeRun];
  unsigned m = 0;
  if (p + kFreeRun <= c.num_pages) {
    __builtin_memcpy(r, c.refs + p, sizeof(r));
#pragma unroll
    for (int u = 0; u < kFreeRun; ++u) m |= want(p + u, r[u]) ? 1u << u : 0u;
  } else {
    for (int u = 0; u < kFreeRun; ++u)
      if (p + u < c.num_pages && want(p + u, c.refs[p + u])) m |= 1u << u;
  }
  return m;
}

// Numbers of the pages that satisfy `want`, ascending, the first `most` of them to `list`;
// how many there are (once `most` are found it looks no further).
template <typename Want>
__device__ __forceinline__ int list_pages(const CacheView& c, int most, int32_t* list, Want&& want) {
  int found = 0;
  for (int64_t p0 = 0; p0 < c.num_pages && found < most; p0 += kPlan * kFreeRun) {
    const int64_t p = p0 + (int64_t)threadIdx.x * kFreeRun;
    unsigned m = p < c.num_pages ? ref_bits(c, p, want) : 0u;
    int total;
    int at = found + plan_scan(__popc(m), &total);
    for (; m; m &= m - 1, ++at)
      if (at < most) list[at] = (int32_t)(p + __ffs(m) - 1);
    found += total;
  }
  __syncthreads();
  return found;
}

// Which of the call's entries names a slot first (a slot named again is left out), in LDS for
// caches of up to kLdsSlots slots, else in the workspace.
constexpr int kLdsSlots = 8192;
struct Marks {
  int* lds;
  int32_t* ws;  // null: in LDS
  __device__ __forceinline__ void mark(const CacheView& c, int n, const int32_t* slots) const {
    for (int e = threadIdx.x; e < n; e += kPlan) {
      const int s = slots[e];
      if (!c.has_slot(s)) continue;
      if (ws) __hip_atomic_store(ws + s, 0x7fffffff, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      else lds[s] = 0x7fffffff;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < n; e += kPlan) {
      const int s = slots[e];
      if (!c.has_slot(s)) continue;
      if (ws) atomicMin(ws + s, e);
      else atomicMin(lds + s, e);
    }
    __syncthreads();
  }
  __device__ __forceinline__ bool first(int slot, int e) const {
    return (ws ? __hip_atomic_load(ws + slot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : lds[slot]) == e;
  }
};
__device__ __forceinline__ Marks marks_of(const CacheView& c, int32_t* ws) {
  __shared__ int s_mark[kLdsSlots];
  return Marks{s_mark, c.num_slots > kLdsSlots ? ws : nullptr};
}

// Adds a thread's refused entries up; valid in every thread.
__device__ __forceinline__ int plan_sum(int x) {
  int total;
  plan_scan(x, &total);
  return total;
}

// What an entry of reserve or fork gets.
struct Want {
  int need;  // pages, 0 if it is refused
  bool refused;
};

// Gives every entry the need_of(e) pages that it asks for.  `put(e, i, page)` stores an entry's
// i-th new page.  All or nothing: false if pages are missing.
template <typename NeedOf, typename Put>
__device__ __forceinline__ bool hand_out(const CacheView& c, int n, int32_t* first, int32_t* list, int32_t* status, int refused,
                                         NeedOf&& need_of, Put&& put) {
  int total = 0;
  for (int e0 = 0; e0 < n; e0 += kPlan) {
    const int e = e0 + threadIdx.x;
    int all;
    const int at = total + plan_scan(e < n ? need_of(e) : 0, &all);
    if (e < n) first[e] = at;
    total += all;
  }
  const int found = total == 0 ? 0 : list_pages(c, total, list, [](int64_t, int r) { return r <= 0; });
  const bool enough = found >= total;
  if (threadIdx.x == 0) {
    status[0] = enough ? 0 : total - found;
    status[1] = refused;
  }
  if (!enough) return false;
  __syncthreads();
  for (int j = threadIdx.x; j < total; j += kPlan) {
    int lo = 0, hi = n - 1;  // the last entry whose pages start at or before j (one that needs any)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= j) lo = mid;
      else hi = mid - 1;
    }
    const int32_t page = list[j];
    put(lo, j - first[lo], page);
    c.refs[page] = 1;
  }
  return true;
}

__global__ __launch_bounds__(kPlan) void cache_reserve_kernel(CacheView c, int n, const int32_t* slots, const int32_t* add,
                                                              int32_t* status, int32_t* mark, int32_t* first, int32_t* list) {
  const Marks marks = marks_of(c, mark);
  // what a thread's first entry says is looked up once: most calls have no more of them
  auto want = [&](int e) {
    const int s = slots[e];
    if (s < 0) return Want{0, false};
    if (!c.has_slot(s)) return Want{0, true};
    const int64_t len = c.seq_len[s], held = c.held[s], more = add[e];
    const int64_t pages = (len + more + c.page_size - 1) >> c.page_log2;
    if (more < 0 || !c.sound(len, held) || pages > c.max_pages) return Want{0, true};
    return Want{pages > held ? (int)(pages - held) : 0, false};
  };
  const int mine = threadIdx.x;
  Want my = mine < n ? want(mine) : Want{0, false};
  marks.mark(c, n, slots);
  auto settled = [&](int e) {
    Want w = e == mine ? my : want(e);
    if (c.has_slot(slots[e]) && !marks.first(slots[e], e)) w = Want{0, true};
    return w;
  };
  if (mine < n) my = settled(mine);
  int bad = 0;
  for (int e = mine; e < n; e += kPlan) bad += e == mine ? my.refused : settled(e).refused;
  bad = plan_sum(bad);
  const bool ok = hand_out(c, n, first, list, status, bad, [&](int e) { return e == mine ? my.need : settled(e).need; },
                           [&](int e, int i, int32_t page) { c.row(slots[e])[c.held[slots[e]] + i] = page; });
  __syncthreads();  // every read of held is done
  if (!ok) return;
  for (int e = mine; e < n; e += kPlan) {
    const int need = e == mine ? my.need : settled(e).need;
    if (need) c.held[slots[e]] += need;
  }
}

__global__ __launch_bounds__(kPlan) void cache_fork_plan_kernel(CacheView c, int n, const int32_t* src, const int32_t* dst,
                                                                int32_t* status, int32_t* mark, int32_t* first, int32_t* list,
                                                                ForkEntry* out) {
  const Marks marks = marks_of(c, mark);
  marks.mark(c, n, dst);
  int bad = 0;
  for (int e = threadIdx.x; e < n; e += kPlan) {
    const int a = src[e], b = dst[e];
    ForkEntry f{};
    f.src = f.dst = f.old_page = f.new_page = -1;
    if (a >= 0 || b >= 0) {
      bool fine = c.has_slot(a) && c.has_slot(b) && a != b && marks.first(b, e) && c.held[b] == 0 && c.seq_len[b] == 0;
      if (fine) {
        const int64_t len = c.seq_len[a];
        fine = c.sound(len, c.held[a]);
        f.whole = (int)(len >> c.page_log2);
        f.rest = (int)(len & (c.page_size - 1));
        if (fine && f.rest) {
          f.old_page = c.row(a)[f.whole];
          fine = c.has_page(f.old_page);
        }
      }
      if (fine) {
        f.src = a;
        f.dst = b;
      }
      bad += !fine;
    }
    out[e] = f;
  }
  bad = plan_sum(bad);  // (its barriers also publish the entries)
  const bool ok = hand_out(c, n, first, list, status, bad, [&](int e) { return out[e].dst >= 0 && out[e].rest ? 1 : 0; },
                           [&](int e, int, int32_t page) {
                             c.row(out[e].dst)[out[e].whole] = page;
                             out[e].new_page = page;
                           });
  __syncthreads();
  for (int e = threadIdx.x; e < n; e += kPlan) {
    if (out[e].dst < 0) continue;
    if (ok) {
      c.held[out[e].dst] = out[e].whole + (out[e].rest != 0);
      c.seq_len[out[e].dst] = (out[e].whole << c.page_log2) + out[e].rest;  // (src may be another entry's dst)
    } else {
      out[e].dst = -1;
    }
  }
}

// y = 0: an entry's table row and references; y > 0: the rows of its partial page in one
// layer's keys or values, head z.
__global__ __launch_bounds__(256) void cache_fork_kernel(CacheView c, CachePools p, const ForkEntry* entries) {
  const ForkEntry f = load_uniform(entries + blockIdx.x);
  if (f.dst < 0) return;
  if (blockIdx.y == 0) {
    if (blockIdx.z) return;
    const int32_t* from = c.row(f.src);
    int32_t* to = c.row(f.dst);
    for (int i = threadIdx.x; i < f.whole; i += 256) {
      const int32_t page = from[i];
      to[i] = page;
      if (c.has_page(page)) atomicAdd(c.refs + page, 1);
    }
    return;
  }
  if (f.new_page < 0) return;
  const int layer = (blockIdx.y - 1) >> 1;
  char* pool = ((blockIdx.y - 1) & 1 ? p.v : p.k) + layer * p.layer_bytes + blockIdx.z * p.head_bytes;
  const f32x4* from = reinterpret_cast<const f32x4*>(pool + f.old_page * p.page_bytes);
  f32x4* to = reinterpret_cast<f32x4*>(pool + f.new_page * p.page_bytes);
  const int chunks = f.rest * (p.row_bytes >> 4);
  copy_chunks<true>(to, from, chunks);
}

// Whoever takes a slot's count of pages to 0 releases them, so a slot named twice is freed once.
__global__ __launch_bounds__(256) void cache_free_kernel(CacheView c, int n, const int32_t* slots) {
  __shared__ int s_held;
  const int s = slots[blockIdx.x];
  if (!c.has_slot(s)) return;
  if (threadIdx.x == 0) {
    s_held = atomicExch(c.held + s, 0);
    c.seq_len[s] = 0;
  }
  __syncthreads();
  const int held = min(s_held, c.max_pages);
  for (int i = threadIdx.x; i < held; i += 256) {
    const int32_t page = c.row(s)[i];
    if (c.has_page(page)) atomicSub(c.refs + page, 1);
  }
}

// Numbers the moves: with L live pages, the i-th of those at L or above goes to the i-th free
// page below L.  from / to: the moves; renum: a moved page's new number, at its old one.
__global__ __launch_bounds__(kPlan) void cache_compact_plan_kernel(CacheView c, int32_t* live_out, int32_t* moves, int32_t* from,
                                                                   int32_t* to, int32_t* renum) {
  int mine = 0;
  for (int64_t p = (int64_t)threadIdx.x * kFreeRun; p < c.num_pages; p += kPlan * kFreeRun)
    mine += __popc(ref_bits(c, p, [](int64_t, int r) { return r > 0; }));
  const int live = plan_sum(mine);
  const int most = c.num_pages;
  const int n = list_pages(c, most, from, [=](int64_t p, int r) { return p >= live && r > 0; });
  if (n) list_pages(c, n, to, [=](int64_t p, int r) { return p < live && r <= 0; });
  for (int i = threadIdx.x; i < n; i += kPlan) {
    const int32_t a = from[i], b = to[i];
    c.refs[b] = c.refs[a];
    c.refs[a] = 0;
    renum[a] = b;
  }
  if (threadIdx.x == 0) {
    *live_out = live;
    moves[0] = n;
    moves[1] = live;
  }
}

constexpr int kMoveBytes = 16384;  // of a page, at a time

// The first `table_blocks` workgroups renumber the table's rows, the others copy pages.
__global__ __launch_bounds__(256) void cache_compact_kernel(CacheView c, CachePools p, const int32_t* moves, const int32_t* from,
                                                            const int32_t* to, const int32_t* renum, int table_blocks) {
  const int n = scalar_load(moves), live = scalar_load(moves + 1);
  if (n == 0) return;
  if ((int)blockIdx.x < table_blocks) {
    for (int s = blockIdx.x; s < c.num_slots; s += table_blocks) {
      const int held = min(c.held[s], c.max_pages);
      int32_t* row = c.row(s);
      for (int i = threadIdx.x; i < held; i += 256) {
        const int32_t page = row[i];
        if (page >= live && c.has_page(page) && c.refs[page] == 0) row[i] = renum[page];
      }
    }
    return;
  }
  const int per = (int)((p.page_bytes + kMoveBytes - 1) / kMoveBytes);
  const int64_t units = (int64_t)n * p.layers * 2 * per;
  for (int64_t u = blockIdx.x - table_blocks; u < units; u += gridDim.x - table_blocks) {
    const int part = (int)(u % per);
    const int64_t v = u / per;
    const int i = (int)(v / (2 * p.layers)), lk = (int)(v % (2 * p.layers));
    char* pool = (lk & 1 ? p.v : p.k) + (lk >> 1) * p.layer_bytes + (int64_t)part * kMoveBytes;
    const f32x4* a = reinterpret_cast<const f32x4*>(pool + from[i] * p.page_bytes);
    f32x4* b = reinterpret_cast<f32x4*>(pool + to[i] * p.page_bytes);
    const int chunks = (int)(min((int64_t)kMoveBytes, p.page_bytes - (int64_t)part * kMoveBytes) >> 4);
    copy_chunks<false>(b, a, chunks);
  }
}

// Which of the accepted nodes' lists are sound, and the new lengths.
__global__ __launch_bounds__(kPlan) void cache_accept_plan_kernel(CacheView c, int n, const int32_t* slots, int max_new,
                                                                  const int32_t* count, const int32_t* path, int32_t* status,
                                                                  int32_t* mark, AcceptEntry* out) {
  const Marks marks = marks_of(c, mark);
  marks.mark(c, n, slots);
  int bad = 0;
  // with a path an entry is a wave, a lane a node (64 at most)
  const int lane = threadIdx.x & 63, lanes = path ? 64 : 1;
  for (int e = threadIdx.x / lanes; e < n; e += kPlan / lanes) {
    const int s = slots[e], m = count[e];
    AcceptEntry a{-1, 0, 0, 0};
    bool fine = true;
    const bool any = s >= 0 && m != 0;
    if (any) {
      fine = c.has_slot(s) && marks.first(s, e) && m > 0 && m <= max_new;
      if (fine) {
        const int64_t len = c.seq_len[s], held = c.held[s];
        int last = m - 1;
        if (path) {
          const int at = lane < m ? path[(int64_t)e * max_new + lane] : 0;
          const int ahead = __shfl_up(at, 1, 64);
          fine = !__any(lane < m && (at <= (lane ? ahead : -1) || at >= max_new));
          a.moved = __any(lane < m && at != lane);
          last = __shfl(at, m - 1, 64);
        }
        fine = fine && c.sound(len, held) && len + last < held << c.page_log2;
        a.len = (int)len;
        a.count = m;
      }
      if (fine) a.slot = s;
    }
    if (threadIdx.x % lanes) continue;
    bad += !fine;
    out[e] = a;
    if (a.slot >= 0) c.seq_len[s] = a.len + m;
  }
  bad = plan_sum(bad);
  if (threadIdx.x == 0) {
    status[0] = 0;
    status[1] = bad;
  }
}

// Moves one head's rows of the kept nodes, in one layer's keys or values: all are read
// before the first is written.
__global__ __launch_bounds__(256) void cache_accept_kernel(CacheView c, CachePools p, const AcceptEntry* entries, int max_new,
                                                           const int32_t* path) {
  const AcceptEntry a = load_uniform(entries + blockIdx.x);
  if (a.slot < 0 || !a.moved) return;
  const int layer = blockIdx.z >> 1;
  char* pool = (blockIdx.z & 1 ? p.v : p.k) + layer * p.layer_bytes + blockIdx.y * p.head_bytes;
  const int32_t* row = c.row(a.slot);
  const int per = p.row_bytes >> 4;  // chunks of 16 bytes a row
  const int chunks = a.count * per;
  constexpr int U = kAcceptNodes * 32 / 256;
  f32x4 v[U];
  char* to[U];
  auto at = [&](int t, int chunk) -> char* {
    const int32_t page = row[t >> c.page_log2];
    return c.has_page(page) ? pool + page * p.page_bytes + (t & (c.page_size - 1)) * p.row_bytes + chunk * 16 : nullptr;
  };
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x + 256 * u;
    to[u] = nullptr;
    if (i >= chunks) continue;
    const int j = i / per, from = path[(int64_t)blockIdx.x * max_new + j];
    if (from == j) continue;
    const char* x = at(a.len + from, i - j * per);
    to[u] = x ? at(a.len + j, i - j * per) : nullptr;
    if (to[u]) v[u] = *reinterpret_cast<const f32x4*>(x);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (to[u]) *reinterpret_cast<f32x4*>(to[u]) = v[u];
}

// Leading pages that all sequences of a group list (slots below 0 left out), as whole pages
// that all of them have filled.
__global__ __launch_bounds__(256) void cache_shared_kernel(CacheView c, const int32_t* slots, int group, int32_t* shared) {
  __shared__ int s_limit;
  const int32_t* g = slots + (int64_t)blockIdx.x * group;
  if (threadIdx.x == 0) s_limit = 0x7fffffff;
  __syncthreads();
  int lead = -1, others = 0;
  for (int m = 0; m < group; ++m) {
    if (g[m] < 0) continue;
    if (lead < 0) lead = g[m];
    else ++others;
  }
  int limit = 0x7fffffff;
  for (int m = threadIdx.x; m < group; m += 256) {
    if (g[m] < 0) continue;
    const bool fine = c.has_slot(g[m]) && c.sound(c.seq_len[g[m]], c.held[g[m]]);
    limit = min(limit, fine ? c.seq_len[g[m]] >> c.page_log2 : 0);
  }
  atomicMin(&s_limit, limit);
  __syncthreads();
  limit = s_limit;
  if (lead < 0 || others == 0) limit = 0;
  __syncthreads();
  if (limit > 0) {
    for (int i = threadIdx.x; i < limit; i += 256) {
      const int32_t page = c.row(lead)[i];
      bool same = true;
      for (int m = 0; m < group; ++m)
        if (g[m] >= 0) same = same && c.row(g[m])[i] == page;
      if (!same) {
        atomicMin(&s_limit, i);
        break;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) shared[blockIdx.x] = limit > 0 ? min(limit, s_limit) : 0;
}

// A wave a token: D / 16 lanes a row, each with 8 elements of the row's first half and the 8
// that they are turned with; rows are the token's queries, keys and values.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheView c, AppendParams a) {
  typedef T Vec __attribute__((ext_vector_type(8)));
  constexpr int LPR = D / 16, RPW = 64 / LPR;
  const int lane = threadIdx.x & 63;
  const int j = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), i = blockIdx.y;
  if (j >= a.max_new) return;
  const int slot = a.slots[i];
  int n = a.count ? a.count[i] : a.max_new;
  n = min(n, a.max_new);
  const int64_t token = a.start ? (int64_t)a.start[i] + j : (int64_t)i * a.max_new + j;
  const int rl = lane / LPR, e = (lane % LPR) * 8;
  const bool live = slot >= 0 && j < n && token >= 0 && token < a.rows;
  if (!live) {
    if (!a.start && a.q_rot)  // a padded batch's row without a token
      for (int h = rl; h < a.hq; h += RPW) {
        T* y = (T*)a.q_rot + (token * a.hq + h) * D + e;
        *reinterpret_cast<Vec*>(y) = Vec{};
        *reinterpret_cast<Vec*>(y + D / 2) = Vec{};
      }
    return;
  }
  int64_t len = 0, page_base = -1;
  int off = 0;
  if (c.has_slot(slot)) {
    len = c.seq_len[slot];
    const int64_t held = c.held[slot], at = len + j;
    if (c.sound(len, held) && at < held << c.page_log2) {
      const int32_t page = c.row(slot)[at >> c.page_log2];
      if (c.has_page(page)) page_base = (int64_t)page * a.hkv;
      off = (int)(at & (c.page_size - 1));
    }
  }
  float cs[8], sn[8];
  if (a.turns) {
    int depth = j;
    if (a.parents) {  // at most 64 nodes: a lane holds one's parent
      const int par = lane <= j ? a.parents[(int64_t)i * a.max_new + lane] : -1;
      depth = 0;
      for (int at = j;;) {
        const int up = __builtin_amdgcn_readlane(par, at);
        if (up < 0 || up >= at) break;
        at = up;
        ++depth;
      }
    }
    const int64_t pos = len + depth;
#pragma unroll
    for (int u = 0; u < 8; ++u) rope_cos_sin((int)pos, a.inv_freq[e + u], cs[u], sn[u]);
  }
  auto turn = [&](Vec& lo, Vec& hi) {
    if (!a.turns) return;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float x = (float)lo[u], y = (float)hi[u];
      lo[u] = (T)(x * cs[u] - y * sn[u]);
      hi[u] = (T)(y * cs[u] + x * sn[u]);
    }
  };
  // queries, then keys, then values: one list of rows
  const int nq = a.q ? a.hq : 0, rows = nq + (page_base >= 0 ? 2 * a.hkv : 0);
  for (int r = rl; r < rows; r += RPW) {
    const int h = r - nq;
    const T* x;
    T* y;
    bool rotate = true;
    if (r < nq) {
      x = (const T*)a.q + (token * a.hq + r) * D + e;
      y = (T*)a.q_rot + (token * a.hq + r) * D + e;
    } else {
      const bool is_v = h >= a.hkv;
      const int g = is_v ? h - a.hkv : h;
      x = (const T*)(is_v ? a.v : a.k) + (token * a.hkv + g) * D + e;
      y = (T*)(is_v ? a.v_pages : a.k_pages) + (((page_base + g) << c.page_log2) + off) * D + e;
      rotate = !is_v;
    }
    Vec lo = *reinterpret_cast<const Vec*>(x), hi = *reinterpret_cast<const Vec*>(x + D / 2);
    if (rotate) turn(lo, hi);
    store_once(y, lo);
    store_once(y + D / 2, hi);
  }
}

}  // namespace

hipError_t launch_cache_reserve(const CacheView& c, int n, const int32_t* slots, const int32_t* add, int32_t* status,
                                const CacheScratch& w, hipStream_t s) {
  TimingScope t("pp_cache_reserve", s);
  hipLaunchKernelGGL(cache_reserve_kernel, dim3(1), dim3(kPlan), 0, s, c, n, slots, add, status, w.mark, w.first, w.list);
  return hipGetLastError();
}

hipError_t launch_cache_fork(const CacheView& c, const CachePools& p, int n, const int32_t* src, const int32_t* dst,
                             int32_t* status, const CacheScratch& w, hipStream_t s) {
  ForkEntry* entries = (ForkEntry*)w.entries;
  {
    TimingScope t("pp_cache_fork_plan", s);
    hipLaunchKernelGGL(cache_fork_plan_kernel, dim3(1), dim3(kPlan), 0, s, c, n, src, dst, status, w.mark, w.first, w.list, entries);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || n == 0) return e;
  }
  TimingScope t("pp_cache_fork", s);
  hipLaunchKernelGGL(cache_fork_kernel, dim3(n, 1 + 2 * p.layers, p.layers ? p.hkv : 1), dim3(256), 0, s, c, p, entries);
  return hipGetLastError();
}

hipError_t launch_cache_free(const CacheView& c, int n, const int32_t* slots, hipStream_t s) {
  TimingScope t("pp_cache_free", s);
  hipLaunchKernelGGL(cache_free_kernel, dim3(n), dim3(256), 0, s, c, n, slots);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheView& c, const CachePools& p, int32_t* live, const CacheScratch& w, hipStream_t s) {
  {
    TimingScope t("pp_cache_compact_plan", s);
    hipLaunchKernelGGL(cache_compact_plan_kernel, dim3(1), dim3(kPlan), 0, s, c, live, w.moves, w.list, w.list2, w.renum);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  TimingScope t("pp_cache_compact", s);
  const int table_blocks = c.num_slots < 256 ? c.num_slots : 256;
  hipLaunchKernelGGL(cache_compact_kernel, dim3(table_blocks + 2048), dim3(256), 0, s, c, p, w.moves, w.list, w.list2, w.renum,
                     table_blocks);
  return hipGetLastError();
}

hipError_t launch_cache_accept(const CacheView& c, const CachePools& p, int n, const int32_t* slots, int max_new,
                               const int32_t* count, const int32_t* path, int32_t* status, const CacheScratch& w, hipStream_t s) {
  AcceptEntry* entries = (AcceptEntry*)w.entries;
  {
    TimingScope t("pp_cache_accept_plan", s);
    hipLaunchKernelGGL(cache_accept_plan_kernel, dim3(1), dim3(kPlan), 0, s, c, n, slots, max_new, count, path, status, w.mark,
                       entries);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || n == 0 || !path || p.layers == 0) return e;
  }
  TimingScope t("pp_cache_accept", s);
  hipLaunchKernelGGL(cache_accept_kernel, dim3(n, p.hkv, 2 * p.layers), dim3(256), 0, s, c, p, entries, max_new, path);
  return hipGetLastError();
}

hipError_t launch_cache_shared(const CacheView& c, int groups, const int32_t* slots, int group, int32_t* shared, hipStream_t s) {
  TimingScope t("pp_cache_shared", s);
  hipLaunchKernelGGL(cache_shared_kernel, dim3(groups), dim3(256), 0, s, c, slots, group, shared);
  return hipGetLastError();
}

hipError_t launch_cache_append(const CacheView& c, const AppendParams& a, int n, int head_dim, int dtype, hipStream_t s) {
  TimingScope t("pp_cache_append", s);
  const dim3 grid((a.max_new + 3) / 4, n);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, c, a); };
  if (dtype == kBF16) {
    if (head_dim == 128) launch(cache_append_kernel<__bf16, 128>);
    else launch(cache_append_kernel<__bf16, 64>);
  } else {
    if (head_dim == 128) launch(cache_append_kernel<float, 128>);
    else launch(cache_append_kernel<float, 64>);
  }
  return hipGetLastError();
}

}  // namespace pp
