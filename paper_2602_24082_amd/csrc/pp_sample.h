// Internal interface of the sampling operators: the paged cache, attention of drafted trees
// over it, draft verification.  Host entry points in pp_sample_host.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pp_launch.h"

namespace pp {

// pp_cache as the kernels see it.
struct CacheView {
  int32_t* table;    // [num_slots, max_pages]
  int32_t* seq_len;  // [num_slots]
  int32_t* held;     // [num_slots]
  int32_t* refs;     // [num_pages]
  int num_slots, max_pages, num_pages, page_size, page_log2;
  __host__ __device__ bool has_slot(int s) const { return (unsigned)s < (unsigned)num_slots; }
  __host__ __device__ bool has_page(int p) const { return (unsigned)p < (unsigned)num_pages; }
  __host__ __device__ int32_t* row(int s) const { return table + (int64_t)s * max_pages; }
  // a sequence's length and pages belong together
  __host__ __device__ bool sound(int64_t len, int64_t n) const {
    return n >= 0 && n <= max_pages && len >= 0 && len <= n << page_log2;
  }
};

// Pools [layers, num_pages, hkv, page_size, head_dim] of keys and values, in bytes.
struct CachePools {
  char* k;
  char* v;
  int64_t layer_bytes, page_bytes;
  int head_bytes;  // a page's rows of one head
  int row_bytes;
  int layers, hkv;
};

struct ForkEntry {
  int32_t src, dst;  // dst < 0: none
  int32_t whole;     // pages that both list
  int32_t rest;      // rows of the partial page
  int32_t old_page, new_page;
};
struct AcceptEntry {
  int32_t slot;  // < 0: none
  int32_t len;   // ahead of the call
  int32_t count;
  int32_t moved;  // any node lies elsewhere
};
constexpr int kAcceptNodes = 64;  // nodes of a drafted tree

struct CacheScratch {
  int32_t* mark;   // [num_slots]
  int32_t* first;  // [n]
  int32_t* list;   // [num_pages]
  int32_t* list2;  // [num_pages]
  int32_t* renum;  // [num_pages]
  int32_t* moves;  // [2]
  void* entries;   // [n] ForkEntry or AcceptEntry
};

struct AppendParams {
  const int32_t* slots;    // [n]
  const int32_t* count;    // [n] or null: max_new
  const int32_t* start;    // [n] or null: i * max_new
  const int32_t* parents;  // [n, max_new] or null: a chain
  const void* q;           // null: none
  const void* k;
  const void* v;
  void* q_rot;
  void* k_pages;
  void* v_pages;
  int64_t rows;  // tokens that k, v and q have
  int max_new, hq, hkv;
  bool turns;           // rotate
  double inv_freq[64];  // base^(-2j / head_dim)
};

hipError_t launch_cache_reserve(const CacheView& c, int n, const int32_t* slots, const int32_t* add, int32_t* status,
                                const CacheScratch& w, hipStream_t s);
hipError_t launch_cache_fork(const CacheView& c, const CachePools& p, int n, const int32_t* src, const int32_t* dst,
                             int32_t* status, const CacheScratch& w, hipStream_t s);
hipError_t launch_cache_free(const CacheView& c, int n, const int32_t* slots, hipStream_t s);
hipError_t launch_cache_compact(const CacheView& c, const CachePools& p, int32_t* live, const CacheScratch& w, hipStream_t s);
hipError_t launch_cache_accept(const CacheView& c, const CachePools& p, int n, const int32_t* slots, int max_new,
                               const int32_t* count, const int32_t* path, int32_t* status, const CacheScratch& w, hipStream_t s);
hipError_t launch_cache_shared(const CacheView& c, int groups, const int32_t* slots, int group, int32_t* shared, hipStream_t s);
hipError_t launch_cache_append(const CacheView& c, const AppendParams& a, int n, int head_dim, int dtype, hipStream_t s);

// Attention of drafted trees over the cache (pp_tree.hip).
constexpr int kTreeSeqs = 2048;  // sequences a call
constexpr int kTreeNodes = 64;   // nodes a sequence
constexpr int kCus = 256;
// Workgroups a compute unit: of one wave, each with a ring of two blocks of 32 keys and values
// in LDS, and of a team of four waves, with a ring between them.  bf16 of head size 128, a team:
// 64 keys a block, two blocks, two teams a unit.  16 drafted nodes of each of four sequences of
// 36 000 tokens, 64 heads over 8, take 124 us so, 127 with four blocks of 32 keys, 143 with one
// team of four blocks of 64.
template <int D, typename T>
constexpr int kTreeSolo = D * sizeof(T) > 256 ? 2 : D * sizeof(T) > 128 ? 4 : 8;
template <int D, typename T>
constexpr int kTreeTeam = sizeof(T) == 4 ? (D == 64 ? 2 : 1) : D == 64 ? 3 : 2;
template <int D, typename T>
constexpr int kTeamKeys = sizeof(T) == 2 ? 64 : 32;
// Blocks that a team has room for: what a compute unit's LDS leaves each
template <int D, typename T>
constexpr int kTeamStages = sizeof(T) == 2 && D == 128 ? 2 : D * sizeof(T) > 128 ? 4 : 3;
// An item's start in blocks of keys, where work is dealt out: single tokens of 16 groups of 16 over
// 2048 shared and some 500 own tokens take 92 us with 0, 80 with 2, 79 with 4.
constexpr int kTreeStart = 4;
constexpr int kSoloKeys = 32, kSoloRows = 32, kTeamWaves = 4, kTeamRows = 128;

// An item: rows against a range of keys; its units: a block of keys, for a tile of rows of one
// kv-head.
struct TreeItem {
  int64_t first;   // units ahead of it, of those that solo waves / teams take
  int32_t blocks;  // of keys, for every tile of rows and head
  int32_t slot;    // whose pages
  int32_t k0, k1;  // keys [k0, k1)
  int32_t seen;    // all rows see the keys below
  int32_t seq;     // the (first) sequence of its rows
  int32_t bad;     // nodes asked for of a sequence that is not sound
  int32_t rows;    // for one kv-head: nodes in use x G
  int32_t row0;    // a sequence's first node among its group's
  int32_t pad[5];
};
// The two kinds of items: a group's shared keys, a sequence's own.
struct TreeKind {
  int rows;       // of an item, for one kv-head, at most
  int team;       // more than 32: taken by teams
  int keys;       // of a block
  int tiles;      // of rows, at most; 0: no such items
  int part_rows;  // of a partial result
  int64_t part0;  // row of the first one
};
struct TreeShape {
  int n, nodes, group, groups;  // sequences, nodes of each, sequences a group
  int hq, hkv, G;
  TreeKind kind[2];  // shared, own
  int workers[2];    // solo waves, teams
  uint64_t key;      // of calls that can go by one plan
};
struct TreePlan {
  TreeItem* items;         // [n + groups]
  int32_t* nodes;          // [n * max_new]: a group's nodes in use, the rows of its shared keys
  int64_t* head;           // [2][2]: units in all, units a worker; then the key
  int32_t* start_item[2];  // [workers]: where a worker starts
};
struct TreeLaunch {
  TreeShape shape;
  TreePlan plan;
  bool planned;  // the plan stands already
  const int32_t* slots;
  const int32_t* count;    // or null: all nodes
  const int32_t* shared;   // [groups] or null
  const int32_t* parents;  // [n, nodes] or null: chains
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;
  float* part;
  float* part_ml;
  float scale;
  int head_dim, dtype;
};
hipError_t launch_tree_attn(const CacheView& c, const TreeLaunch& a, hipStream_t s);

// Draft verification (pp_draft.hip).
constexpr int kOwnLine = 32;       // int32 counters of different sequences are a line of 128 bytes apart
constexpr int kDraftChunk = 2048;  // entries of a row that are looked at together
struct DraftShape {
  int n, nodes, vocab, chunks, max_children;
};
// What a row's entries in one chunk hold: their maximum (NaN: a NaN or +inf among them), the
// sum of e^((x - max) / T), and the first entry at the maximum.
struct DraftPart {
  double sum;
  float max;
  int32_t arg;
};
// A row's distribution, joined from its chunks.
struct DraftRow {
  double sum;
  float max;
  int32_t arg;  // < 0: the row cannot be used
};
// Of a drafted token: its probabilities, and whether what is left after its rejection may be
// asked for (first children).
struct DraftEdge {
  double p, q;
  int32_t need, pad;
};
struct DraftParams {
  DraftShape shape;
  const void* target;
  const void* draft;         // or null: given drafts
  const int32_t* tokens;
  const int32_t* parents;    // or null: chains
  const int32_t* count;      // or null
  const float* temperature;  // or null: 1
  const float* u;
  int32_t* out_count;
  int32_t* out_tokens;
  int32_t* out_path;
  float* out_logp;
  DraftPart* part;  // [2, n, nodes, chunks]: of the target's rows, of the draft's
  double* left;     // [n, nodes, chunks]: Z after a node is rejected
  DraftRow* row;    // [2, n, nodes]: the target's, the draft's (of nodes with children)
  DraftEdge* edge;  // [n, nodes]
  double* ends;     // [n, chunks]: Z where the walk ends
  int32_t* arrived; // [n * kOwnLine]: workgroups that have left theirs
};
hipError_t launch_verify_draft(const DraftParams& p, int dtype, hipStream_t s);

}  // namespace pp
