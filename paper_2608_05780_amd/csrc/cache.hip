// The key/value cache's own upkeep: appending tokens and cutting a cache to a
// budget by accumulated attention weight. Both only move rows; what bounds
// them is memory traffic for long lists and launches for short ones.
#include <algorithm>

#include "cache.h"

namespace evisel {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// Append.

// What sequence `seq` appends: its first row, its rows, the tokens that fit.
struct Appended {
  int first, rows, n, len, seen;
};
__device__ __forceinline__ Appended appended(const CacheView& c,
                                             const AppendCall& a, int seq) {
  Appended r;
  r.first = min(max(a.tok_ptr[seq], 0), a.n_tok);
  r.rows = min(max(a.tok_ptr[seq + 1], r.first), a.n_tok) - r.first;
  r.len = held(c, seq, (int)c.cap);
  r.seen = c.seen[seq];
  r.n = a.n_accept ? min(max(a.n_accept[seq], 0), r.rows) : r.rows;
  r.n = min(min(r.n, a.max_new), (int)c.cap - r.len);
  return r;
}

// Tokens i0 .. i1 - 1 of a sequence, by THREADS threads: RC lanes copy a row
// of 16 RC bytes, so a wavefront takes whole rows; the rows of four heads are
// in flight at a time (K and V: eight loads).
template <int RC, int THREADS>
__device__ __forceinline__ void append_tokens(const CacheView& c,
                                              const AppendCall& a,
                                              const Appended& r, int seq,
                                              int i0, int i1) {
  constexpr int kRowBytes = 16 * RC;
  const int tid = threadIdx.x, ch = tid % RC;
  for (int i = i0 + tid / RC; i < i1; i += THREADS / RC) {
    int row = i;
    if (a.accept) row = min(max(a.accept[r.first + i], 0), r.rows - 1);
    const int64_t off = slot_offset(c, seq, r.len + i);
    const int64_t src =
        (int64_t)(r.first + row) * c.hkv * kRowBytes + 16 * ch;
    if (off < 0) continue;   // no page
    for (int h0 = 0; h0 < c.hkv; h0 += 4) {
      i32x4 k[4], v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (h0 + u < c.hkv) {
          k[u] = *(const i32x4*)(a.k_new + src + (int64_t)(h0 + u) * kRowBytes);
          v[u] = *(const i32x4*)(a.v_new + src + (int64_t)(h0 + u) * kRowBytes);
        }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (h0 + u < c.hkv) {
          const int64_t dst = off + (h0 + u) * c.head_bytes + 16 * ch;
          *(i32x4*)(c.k + dst) = k[u];
          *(i32x4*)(c.v + dst) = v[u];
        }
    }
  }
  if (!c.weight && !c.pos) return;
  // heads slowest: the slots of one head are neighbours
  const int n = i1 - i0;
  for (int64_t u = tid; u < (int64_t)n * c.hkv; u += THREADS) {
    const int h = (int)(u / n), i = i0 + (int)(u % n);
    const int64_t at = ((int64_t)seq * c.hkv + h) * c.cap + r.len + i;
    if (c.pos) c.pos[at] = r.seen + i;
    if (c.weight) {
      int row = i;
      if (a.accept) row = min(max(a.accept[r.first + i], 0), r.rows - 1);
      c.weight[at] =
          a.w_new ? a.w_new[(int64_t)(r.first + row) * c.hkv + h] : 0.f;
    }
  }
}

// Few tokens: a sequence's work-group copies them all and then counts them,
// one launch.
constexpr int kFewThreads = 512;
template <int RC>
__global__ __launch_bounds__(kFewThreads) void append_few_kernel(
    const CacheView c, const AppendCall a) {
  const int seq = blockIdx.x;
  const Appended r = appended(c, a, seq);
  __syncthreads();   // every thread has read the counts
  if (r.n <= 0) return;
  append_tokens<RC, kFewThreads>(c, a, r, seq, 0, r.n);
  if (threadIdx.x == 0) {
    c.length[seq] = r.len + r.n;
    c.seen[seq] = r.seen + r.n;
  }
}

// Many tokens: kAppendTokens per work-group, the counts in a second launch.
constexpr int kAppendThreads = 256;
constexpr int kAppendTokens = 64;
template <int RC>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(
    const CacheView c, const AppendCall a) {
  const int seq = blockIdx.y;
  const Appended r = appended(c, a, seq);
  const int i0 = blockIdx.x * kAppendTokens;
  if (i0 >= r.n) return;
  append_tokens<RC, kAppendThreads>(c, a, r, seq, i0,
                                    min(i0 + kAppendTokens, r.n));
}

__global__ __launch_bounds__(256) void append_count_kernel(
    const CacheView c, const AppendCall a) {
  const int seq = blockIdx.x * 256 + threadIdx.x;
  if (seq >= c.n_seq) return;
  const Appended r = appended(c, a, seq);
  if (r.n <= 0) return;
  c.length[seq] = r.len + r.n;
  c.seen[seq] = r.seen + r.n;
}

// Bytes of one sequence up to which its own work-group copies them.
constexpr int64_t kFewBytes = 128 << 10;

template <int RC>
hipError_t launch_append(const CacheView& c, const AppendCall& a,
                         hipStream_t s) {
  if ((int64_t)a.max_new * c.hkv * RC * 32 <= kFewBytes) {
    append_few_kernel<RC><<<dim3(c.n_seq), dim3(kFewThreads), 0, s>>>(c, a);
    return hipGetLastError();
  }
  // y holds 65,535 sequences at most
  for (int s0 = 0; s0 < c.n_seq; s0 += 65535) {
    CacheView v = c;
    AppendCall b = a;
    v.n_seq = std::min(65535, c.n_seq - s0);
    v.table += (int64_t)s0 * c.max_pages;
    v.length += s0;
    v.seen += s0;
    if (v.weight) v.weight += (int64_t)s0 * c.hkv * c.cap;
    if (v.pos) v.pos += (int64_t)s0 * c.hkv * c.cap;
    b.tok_ptr += s0;
    if (b.n_accept) b.n_accept += s0;
    append_kernel<RC><<<dim3((a.max_new + kAppendTokens - 1) / kAppendTokens,
                             v.n_seq),
                        dim3(kAppendThreads), 0, s>>>(v, b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  append_count_kernel<<<dim3((c.n_seq + 255) / 256), dim3(256), 0, s>>>(c, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Evict.

// Kept tokens rank by this: larger first. Tokens that are always kept lead,
// NaN ranks like -inf, and -0 like 0.
__device__ __forceinline__ uint32_t keep_key(float w, int pos, int n_sink,
                                             int64_t recent_from) {
  if (pos < n_sink || pos >= recent_from) return 0xFFFFFFFFu;
  uint32_t b = __float_as_uint(w);
  if (w != w) b = 0xFF800000u;
  if (b == 0x80000000u) b = 0u;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int kEvThreads = 1024;
constexpr int kEvWaves = kEvThreads / 64;
constexpr int kEvBins = 2048;
// keys that stay in LDS (the kernel's other arrays take 25 KB of the 160)
constexpr int kEvLdsKeys = 32 * 1024;

// keys of one digit's bin that stay in LDS as a list
constexpr int kEvList = 4096;

// One work-group per sequence and kv head: which slots it keeps, and from
// that the moves. The budget-th largest key comes digit by digit (11, 11 and
// 10 bits, a histogram each): the first digit from every key, the others, as a
// rule, from the short list of keys that share the digits before; equal keys
// are kept from the lowest slot on. Then every wavefront walks its own run of
// slots twice, 256 at a time: counting, and, with what the runs before it
// counted, writing the holes below the budget and the kept slots above it into
// the two lists. LDS: the keys stay in LDS between the passes; otherwise each
// pass makes them again from weight and pos.
template <bool LDS>
__global__ __launch_bounds__(kEvThreads) void evict_select_kernel(
    const CacheView c, const EvictCall e) {
  __shared__ uint32_t hist[kEvBins];
  __shared__ uint32_t list[kEvList];
  __shared__ uint32_t wave_tot[kEvWaves];
  __shared__ uint32_t found[2];          // the digit, and what is above it
  __shared__ uint32_t listed;
  __shared__ int runs[kEvWaves][4];      // above / equal, below / from budget
  extern __shared__ __attribute__((aligned(16))) uint32_t keys[];
  const int unit = blockIdx.x, seq = unit / c.hkv;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = held(c, seq, e.max_len);
  if (len <= e.budget) {
    if (tid == 0) e.count[unit] = 0;
    return;
  }
  const int64_t recent_from = (int64_t)c.seen[seq] - e.n_recent;
  const float* w = c.weight + (int64_t)unit * c.cap;
  const int32_t* pos = c.pos + (int64_t)unit * c.cap;
  // Keys i .. i + 3 (i a multiple of 4; the capacity is one of 16, so that
  // slots past the length can be read). Which of them are there: i + u < len.
  auto make = [&](int i) {
    const f32x4 x = *(const f32x4*)(w + i);
    const i32x4 p = *(const i32x4*)(pos + i);
    u32x4 k;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      k[u] = keep_key(x[u], p[u], e.n_sink, recent_from);
    return k;
  };
  auto four = [&](int i) {
    return LDS ? *(const u32x4*)(keys + i) : make(i);
  };
  // One key a lane into the histogram. The bin of the first lane that has one
  // is added at once, so that a run of equal weights is no chain of additions
  // to one place.
  auto count = [&](bool in, uint32_t bin) {
    const uint64_t active = __ballot(in);
    if (!active) return;
    const int lead = __builtin_ctzll(active);
    const uint32_t b0 = __builtin_amdgcn_readlane(bin, lead);
    const uint64_t same = __ballot(in && bin == b0);
    if (lane == lead) atomicAdd(&hist[b0], (uint32_t)__popcll(same));
    if (in && bin != b0) atomicAdd(&hist[bin], 1u);
  };
  auto clear = [&] {
    for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0;
    if (tid == 0) listed = 0;
    __syncthreads();
  };
  // The bin, from the largest down, in which the running count reaches
  // `need`: found[0], and the count above it: found[1]. Two bins a thread.
  auto locate = [&](uint32_t need) {
    __syncthreads();
    const uint32_t c0 = hist[kEvBins - 1 - 2 * tid];
    const uint32_t c1 = hist[kEvBins - 2 - 2 * tid];
    uint32_t run = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t up = __shfl_up(run, o);
      if (lane >= o) run += up;
    }
    if (lane == 63) wave_tot[wave] = run;
    __syncthreads();
    uint32_t before = run - c0 - c1;
    for (int i = 0; i < wave; ++i) before += wave_tot[i];
    if (before < need && before + c0 >= need) {
      found[0] = kEvBins - 1 - 2 * tid;
      found[1] = before;
    } else if (before + c0 < need && before + c0 + c1 >= need) {
      found[0] = kEvBins - 2 - 2 * tid;
      found[1] = before + c0;
    }
    __syncthreads();
  };
  constexpr int kStep = 4 * kEvThreads;

  // first digit
  clear();
#pragma unroll 2
  for (int i0 = 0; i0 < len; i0 += kStep) {
    const int i = i0 + 4 * tid;
    u32x4 k = {};
    if (i < len) {
      k = make(i);
      if (LDS) *(u32x4*)(keys + i) = k;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) count(i + u < len, k[u] >> 21);
  }
  uint32_t need = (uint32_t)e.budget;   // keys still wanted among the matching
  locate(need);
  uint32_t prefix = found[0] << 21;
  need -= found[1];
  // the keys that share it, into the list (or, if they are too many, again
  // from all keys), and their second digit
  clear();
#pragma unroll 2
  for (int i0 = 0; i0 < len; i0 += kStep) {
    const int i = i0 + 4 * tid;
    u32x4 k = {};
    if (i < len) k = four(i);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool in = i + u < len && (k[u] & 0xFFE00000u) == prefix;
      const uint64_t m = __ballot(in);
      if (!m) continue;
      const int lead = __builtin_ctzll(m);
      uint32_t at = 0;
      if (lane == lead) at = atomicAdd(&listed, (uint32_t)__popcll(m));
      at = __builtin_amdgcn_readlane(at, lead) +
           (uint32_t)__popcll(m & ((1ull << lane) - 1));
      if (in && at < kEvList) list[at] = k[u];
      count(in, (k[u] >> 10) & 2047u);
    }
  }
  locate(need);
  prefix |= found[0] << 10;
  need -= found[1];
  const uint32_t n_list = listed;
  __syncthreads();   // every thread has read `listed`
  clear();
  if (n_list <= kEvList) {
    for (uint32_t i0 = 0; i0 < n_list; i0 += kEvThreads) {
      const uint32_t i = i0 + tid, k = i < n_list ? list[i] : 0u;
      count(i < n_list && (k & 0xFFFFFC00u) == prefix, k & 1023u);
    }
  } else {
    for (int i0 = 0; i0 < len; i0 += kStep) {
      const int i = i0 + 4 * tid;
      u32x4 k = {};
      if (i < len) k = four(i);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        count(i + u < len && (k[u] & 0xFFFFFC00u) == prefix, k[u] & 1023u);
    }
  }
  locate(need);
  prefix |= found[0];
  need -= found[1];
  // kept: keys above `prefix`, and the first `need` that equal it

  const int per = ((len + 256 * kEvWaves - 1) / (256 * kEvWaves)) * 256;
  const int a = min(wave * per, len), b = min(a + per, len);
  int n_gt[2] = {0, 0}, n_eq[2] = {0, 0};
#pragma unroll 2
  for (int i0 = a; i0 < b; i0 += 256) {
    const int i = i0 + 4 * lane;
    u32x4 k = {};
    if (i < b) k = four(i);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool in = i + u < b, hi = i + u >= e.budget;
      const bool gt = in && k[u] > prefix, eq = in && k[u] == prefix;
      n_gt[0] += gt && !hi;
      n_gt[1] += gt && hi;
      n_eq[0] += eq && !hi;
      n_eq[1] += eq && hi;
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    n_gt[0] += __shfl_xor(n_gt[0], o);
    n_gt[1] += __shfl_xor(n_gt[1], o);
    n_eq[0] += __shfl_xor(n_eq[0], o);
    n_eq[1] += __shfl_xor(n_eq[1], o);
  }
  if (lane == 0) {
    runs[wave][0] = n_gt[0];
    runs[wave][1] = n_eq[0];
    runs[wave][2] = n_gt[1];
    runs[wave][3] = n_eq[1];
  }
  __syncthreads();
  // what the runs before this one hold: equal keys, holes, kept tail slots
  int eqs = 0, holes = 0, tails = 0;
  for (int u = 0; u < wave; ++u) {
    const int ua = min(u * per, len), ub = min(ua + per, len);
    const int below = max(0, min(ub, e.budget) - ua);
    const int k0 = min(max((int)need - eqs, 0), runs[u][1]);
    eqs += runs[u][1];
    const int k1 = min(max((int)need - eqs, 0), runs[u][3]);
    eqs += runs[u][3];
    holes += below - runs[u][0] - k0;
    tails += runs[u][2] + k1;
  }
  int32_t* to = e.to + (int64_t)unit * e.max_moves;
  int32_t* from = e.from + (int64_t)unit * e.max_moves;
  const uint64_t below_lane = (1ull << lane) - 1;
#pragma unroll 2
  for (int i0 = a; i0 < b; i0 += 256) {
    const int i = i0 + 4 * lane;
    u32x4 k = {};
    if (i < b) k = four(i);
    // slots in order: lane by lane, each its four
    int before = eqs;
    bool eq[4], kept[4], out[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      eq[u] = i + u < b && k[u] == prefix;
      const uint64_t m = __ballot(eq[u]);
      before += __popcll(m & below_lane);
      eqs += __popcll(m);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      kept[u] = i + u < b &&
                (k[u] > prefix || (eq[u] && before < (int)need));
      before += eq[u];
    }
    int hole = holes, tail = tails;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool hi = i + u >= e.budget;
      out[u] = i + u < b && !hi && !kept[u];
      kept[u] = kept[u] && hi;
      const uint64_t mh = __ballot(out[u]), mt = __ballot(kept[u]);
      hole += __popcll(mh & below_lane);
      tail += __popcll(mt & below_lane);
      holes += __popcll(mh);
      tails += __popcll(mt);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (out[u]) to[hole++] = i + u;
      if (kept[u]) from[tail++] = i + u;
    }
  }
  if (wave == kEvWaves - 1 && lane == 0) e.count[unit] = tails;
}

// The moves: RC lanes copy a row of K and of V. A slot from the budget on is
// never written, so no move waits for another. The first work-group of a
// sequence's first head sets its length: nothing here reads that.
constexpr int kMvThreads = 256;
template <int RC>
__global__ __launch_bounds__(kMvThreads) void evict_move_kernel(
    const CacheView c, const EvictCall e, int per_block, int blocks_per_unit) {
  const int unit = blockIdx.x / blocks_per_unit;
  const int part = blockIdx.x % blocks_per_unit;
  const int seq = unit / c.hkv, h = unit % c.hkv;
  if (part == 0 && h == 0 && threadIdx.x == 0 &&
      c.length[seq] > e.budget)
    c.length[seq] = e.budget;
  const int n = min(e.count[unit], (part + 1) * per_block);
  const int32_t* to = e.to + (int64_t)unit * e.max_moves;
  const int32_t* from = e.from + (int64_t)unit * e.max_moves;
  const int ch = threadIdx.x % RC;
  for (int i = part * per_block + (int)threadIdx.x / RC; i < n;
       i += kMvThreads / RC) {
    const int src = from[i], dst = to[i];
    const int64_t so = slot_offset(c, seq, src);
    const int64_t dp = slot_offset(c, seq, dst);
    const int64_t at = h * c.head_bytes + 16 * ch;
    if (so >= 0 && dp >= 0) {
      const i32x4 k = *(const i32x4*)(c.k + so + at);
      const i32x4 v = *(const i32x4*)(c.v + so + at);
      *(i32x4*)(c.k + dp + at) = k;
      *(i32x4*)(c.v + dp + at) = v;
    }
    if (ch == 0) {
      const int64_t row = (int64_t)unit * c.cap;
      c.weight[row + dst] = c.weight[row + src];
      c.pos[row + dst] = c.pos[row + src];
    }
  }
}

template <int RC>
hipError_t launch_move(const CacheView& c, const EvictCall& e, hipStream_t s) {
  const int units = c.n_seq * c.hkv;
  const int per = 4 * kMvThreads / RC;   // four rows per thread
  const int64_t parts = (e.max_moves + per - 1) / per;
  if (parts * units > 0x7FFFFFFF) return hipErrorInvalidValue;
  evict_move_kernel<RC><<<dim3((unsigned)(parts * units)), dim3(kMvThreads), 0,
                          s>>>(c, e, per, (int)parts);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheView& c, const AppendCall& a,
                               hipStream_t s) {
  const int rc = c.d * (c.fp32 ? 4 : 2) / 16;
  if (rc == 8) return launch_append<8>(c, a, s);
  if (rc == 16) return launch_append<16>(c, a, s);
  return launch_append<32>(c, a, s);
}

hipError_t launch_cache_evict(const CacheView& c, const EvictCall& e,
                              hipStream_t s) {
  const dim3 grid((unsigned)(c.n_seq * c.hkv)), block(kEvThreads);
  if ((int64_t)c.n_seq * c.hkv > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (e.max_len <= kEvLdsKeys) {
    const size_t lds = ((size_t)e.max_len * 4 + 15) & ~size_t(15);
    if (lds + 32 * 1024 > 64 * 1024) {
      const hipError_t r = hipFuncSetAttribute(
          (const void*)evict_select_kernel<true>,
          hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (r != hipSuccess) return r;
    }
    evict_select_kernel<true><<<grid, block, lds, s>>>(c, e);
  } else {
    evict_select_kernel<false><<<grid, block, 0, s>>>(c, e);
  }
  const hipError_t r = hipGetLastError();
  if (r != hipSuccess) return r;
  const int rc = c.d * (c.fp32 ? 4 : 2) / 16;
  if (rc == 8) return launch_move<8>(c, e, s);
  if (rc == 16) return launch_move<16>(c, e, s);
  return launch_move<32>(c, e, s);
}

}  // namespace evisel
