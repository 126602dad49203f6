// The key/value cache: device view and kernel launchers (cache.hip,
// cache_attn.hip), called from cache_api.hip.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <string>

#include "evisel.h"

namespace evisel {

// Records the message of a failing call (api.hip) and returns its status.
evisel_status set_error(evisel_status s, const char* msg);
evisel_status set_hip_error(hipError_t e, const char* what);

// Device view of a cache, strides in bytes.
struct CacheView {
  char* k;
  char* v;
  const int32_t* table;
  int32_t* length;
  int32_t* seen;
  float* weight;
  int32_t* pos;
  int64_t n_pages;
  int64_t page_bytes, head_bytes;
  int32_t token_bytes;
  int32_t n_seq, hkv, d;
  int32_t page_shift, max_pages;
  int64_t cap;          // max_pages << page_shift
  int32_t fp32;
};

// Slots of a sequence that a call looks at.
__device__ __forceinline__ int held(const CacheView& c, int seq,
                                    int most) {
  return min(max(c.length[seq], 0), most);
}

// Address of row `slot` (kv head 0) from the pool's base, or -1: no page.
__device__ __forceinline__ int64_t slot_offset(const CacheView& c, int seq,
                                               int slot) {
  const int id = c.table[(int64_t)seq * c.max_pages + (slot >> c.page_shift)];
  if (id < 0 || id >= c.n_pages) return -1;
  return id * c.page_bytes +
         (int64_t)(slot & ((1 << c.page_shift) - 1)) * c.token_bytes;
}

struct AppendCall {
  const char* k_new;
  const char* v_new;
  const int32_t* tok_ptr;
  const int32_t* accept;     // may be null
  const int32_t* n_accept;   // may be null
  const float* w_new;        // may be null
  int32_t n_tok, max_new;
};
hipError_t launch_cache_append(const CacheView& c, const AppendCall& a,
                               hipStream_t s);

struct EvictCall {
  int32_t budget, n_sink, n_recent, max_len;
  int32_t max_moves;   // min(budget, max_len - budget)
  int32_t* count;      // [n_seq][hkv] moves
  int32_t* from;       // [n_seq][hkv][max_moves] slots
  int32_t* to;
  // long caches (null otherwise): what a slot ranks by [n_seq][hkv][key_stride]
  // and histograms [n_seq][hkv][chunks][2048]
  uint32_t* keys;
  uint32_t* chunk_hist;
  int32_t chunks, key_stride;
};
// Sets max_moves and the workspace pointers from budget and max_len; the
// workspace's bytes.
size_t evict_layout(const CacheView& c, EvictCall& e, char* workspace);
hipError_t launch_cache_evict(const CacheView& c, const EvictCall& e,
                              hipStream_t s);

// A row's reference moves when a logit passes it by this (log2 units): the
// probabilities stay below 2^8, and fp32 sums and bf16 probabilities keep
// their relative precision at any such scale.
constexpr float kTreeSlack = 8.0f;

// How a tree attention call is split (host, from its bounds alone).
struct TreePlan {
  int32_t rows;        // most query rows of a kv head: group * max_tree
  int32_t row_tiles;   // 16-row tiles that a wave takes (1, 2 or 4)
  int32_t wide;        // many rows: the kernel that shares keys through LDS
  int32_t row_blocks;  // work-groups that the rows take
  int32_t padded;      // rows, to whole work-groups
  // Runs of keys: `groups` work-groups for each kv head and row block.
  int32_t groups;
  int32_t splits;      // runs of each sequence
  int32_t balanced;    // or by the lengths on the device (wide), with
  int32_t goal;        // runs to aim for,
  int32_t least;       // tiles of a run at least
  int32_t most_runs;   // and runs of a sequence at most
  int32_t joined;      // a sequence may have several
  int32_t stored;      // accumulate: the scores pass through the workspace
  int64_t len_pad;     // max_len rounded up, of the stored scores
  // workspace offsets and total, bytes
  size_t pO, pM, pL, share, row_m, row_inv, score, total;
};

struct TreeCall {
  const char* q;
  const char* k_new;         // may be null, with v_new
  const char* v_new;
  const int32_t* tree_ptr;
  const int32_t* parent;     // null: chains
  char* out;
  float* lse;                // may be null
  const float* vote;         // may be null
  float* w_new;              // may be null
  float scale_log2;          // of the logits, times log2(e)
  float decay;
  int32_t hq, n_tok, max_tree, max_len, accumulate;
  float* pO;                 // [part][kv head][row][d]
  float* pM;                 // [part][kv head][row] reference, log2 units
  float* pL;                 //                        and sum
  int32_t* share;            // [seq] first part, parts
  float* row_m;              // [seq][kv head][row] the same, over the splits:
  float* row_inv;            // reference and 1 / sum (accumulate)
  float* score;              // [seq][kv head][row][len_pad + 64] q.k

  // The token of a query row: r / group by a multiplication with 2^32 / group
  // rounded up, exact as r * group < 2^32 (0: a group of one).
  uint32_t group_inv;
  __device__ __forceinline__ int token_of(int r) const {
    return group_inv ? (int)__umulhi((uint32_t)r, group_inv) : r;
  }
  // exp2 of a logit (as q.k) over a reference (log2 units). One rounding, of
  // a value that is small where it matters; the reference's own cancels.
  __device__ __forceinline__ float exp_of(float x, float ref) const {
    return __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale_log2, -ref));
  }
  __device__ __forceinline__ float lse_of(float m, float sum) const {
    return sum == 0.f ? -__builtin_inff()
                      : (m + __builtin_amdgcn_logf(sum)) *
                            0.69314718055994530942f;
  }
};
TreePlan plan_tree(const CacheView& c, int32_t hq, int32_t max_tree,
                   int32_t max_len, int32_t accumulate);
hipError_t launch_tree_attention(const CacheView& c, const TreePlan& p,
                                 const TreeCall& t, hipStream_t s);

}  // namespace evisel
