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
  for (int u = tid; u < n * c.hkv; u += THREADS) {
    const int h = u / n, i = i0 + u % n;
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
// one launch (4 us for 32 paths of up to 9 tokens).
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
// 579 MB of rows into pages: 205-235 us, 4.9-5.6 TB/s read and written.
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

// Kept tokens rank by this: larger first. Tokens that are always kept (those
// of positions outside n_sink .. n_sink + span - 1) lead, NaN ranks like -inf,
// and -0 like 0.
__device__ __forceinline__ uint32_t keep_key(float w, int pos, int n_sink,
                                             uint32_t span) {
  const int b = (int)__float_as_uint(w + 0.f);   // -0 + 0 = 0
  uint32_t k = (uint32_t)(b ^ ((b >> 31) | (int)0x80000000));
  if (w != w) k = 0x007FFFFFu;
  return (uint32_t)pos - (uint32_t)n_sink >= span ? 0xFFFFFFFFu : k;
}
// Which of slots i .. i + 3 lie below `end`, as bits.
__device__ __forceinline__ uint32_t below4(int i, int end) {
  return (1u << min(max(end - i, 0), 4)) - 1;
}

constexpr int kEvThreads = 1024;
constexpr int kEvWaves = kEvThreads / 64;
constexpr int kEvBins = 2048;
// Keys that stay in LDS (the select kernel's other arrays take 65 KB of 160).
constexpr int kEvLdsKeys = 23 * 1024;
// Histograms side by side, lane by lane: equal weights are 16 additions to one
// place and not 64, and the four neighbours lie in different banks.
constexpr int kEvCopies = 4;
// keys of one digit's bin that are kept as a list, with their slots
constexpr int kEvList = 4096;

// Sum over the lanes before this one, and over all (wave-uniform). Lanes add
// their neighbours 1, 2, 4 and 8 below within a row of 16, then the last lane of
// the rows below: six additions in registers, where shuffles through LDS took
// 0.3 us.
__device__ __forceinline__ uint32_t lanes_before(uint32_t x, uint32_t* all) {
  int s = (int)x;
  s += __builtin_amdgcn_update_dpp(0, s, 0x111, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x112, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x114, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x118, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x142, 0xA, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x143, 0xC, 0xF, false);
  *all = (uint32_t)__builtin_amdgcn_readlane(s, 63);
  return (uint32_t)s - x;
}

// Keys of a long cache, and the histogram of their first digit, kEvChunk slots
// a work-group: what one work-group does alone in 16 us for 65,664 slots, with
// the same again in both passes that follow (44 us in all, 35 so).
constexpr int kEvChunk = 4096;
constexpr int kKeyThreads = 256;
__global__ __launch_bounds__(kKeyThreads) void evict_keys_kernel(
    const CacheView c, const EvictCall e) {
  __shared__ uint32_t hist[kEvBins * kEvCopies];
  const int unit = blockIdx.x / e.chunks, chunk = blockIdx.x % e.chunks;
  const int seq = unit / c.hkv, tid = threadIdx.x;
  const int len = held(c, seq, e.max_len);
  const int i0 = chunk * kEvChunk, i1 = min(i0 + kEvChunk, len);
  if (len <= e.budget || i0 >= len) return;
  const uint32_t span = (uint32_t)max(
      (int64_t)0, (int64_t)c.seen[seq] - e.n_recent - e.n_sink);
  const float* w = c.weight + (int64_t)unit * c.cap;
  const int32_t* pos = c.pos + (int64_t)unit * c.cap;
  uint32_t* keys = e.keys + (int64_t)unit * e.key_stride;
  for (int i = 4 * tid; i < kEvBins * kEvCopies; i += 4 * kKeyThreads)
    *(u32x4*)(hist + i) = u32x4{};
  __syncthreads();
  constexpr int kSteps = kEvChunk / (4 * kKeyThreads);
  f32x4 x[kSteps];
  i32x4 p[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = i0 + 4 * (tid + s * kKeyThreads);
    if (i < i1) {   // (the capacity is a multiple of 16)
      x[s] = *(const f32x4*)(w + i);
      p[s] = *(const i32x4*)(pos + i);
    }
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = i0 + 4 * (tid + s * kKeyThreads);
    if (i >= i1) continue;
    u32x4 k;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      k[u] = keep_key(x[s][u], p[s][u], e.n_sink, span);
      if (i + u < i1)
        atomicAdd(&hist[(k[u] >> 21) * kEvCopies + tid % kEvCopies], 1u);
    }
    *(u32x4*)(keys + i) = k;
  }
  __syncthreads();
  uint32_t* out =
      e.chunk_hist + ((int64_t)unit * e.chunks + chunk) * kEvBins;
  for (int i = tid; i < kEvBins; i += kKeyThreads) {
    const u32x4 h = *(const u32x4*)(hist + 4 * i);
    out[i] = h[0] + h[1] + h[2] + h[3];
  }
}

// One work-group per sequence and kv head: which slots it keeps, and from
// that the moves. The budget-th largest key comes digit by digit, 11, 11 and
// 10 bits, a histogram each. The first takes every key; a second pass, in
// which every wavefront has a run of slots to itself, counts the run's keys
// above that digit and lists those that have it, and the rest works on that
// list (on all keys, if they are too many). Equal keys are kept from the
// lowest slot on. The third pass knows how many holes and kept tail slots the
// runs before hold and writes its own into the two lists, 256 slots at a time.
// LDS: the keys stay there between the passes. Otherwise evict_keys_kernel has
// left them in the workspace, with the first digit's histograms by chunk.
// 2,056 slots 8 us, 16,512 13 us, 65,664 30 us and 5 for the keys: a chain of
// passes and barriers, of which a long cache adds VALU and LDS time.
template <bool LDS>
__global__ __launch_bounds__(kEvThreads) void evict_select_kernel(
    const CacheView c, const EvictCall e) {
  __shared__ uint32_t hist[kEvBins * kEvCopies];
  __shared__ uint32_t list_key[kEvList];
  __shared__ int list_slot[kEvList];
  __shared__ uint32_t wave_tot[kEvWaves];
  __shared__ uint32_t found[2];          // the digit, and what is above it
  __shared__ uint32_t listed;
  // of a wavefront's run: keys above and equal, below the budget and from it
  __shared__ int runs[4][kEvWaves];
  extern __shared__ __attribute__((aligned(16))) uint32_t keys[];
  const int unit = blockIdx.x, seq = unit / c.hkv;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = held(c, seq, e.max_len);
  if (len <= e.budget) {
    if (tid == 0) e.count[unit] = 0;
    return;
  }
  const uint32_t span = (uint32_t)max(
      (int64_t)0, (int64_t)c.seen[seq] - e.n_recent - e.n_sink);
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
      k[u] = keep_key(x[u], p[u], e.n_sink, span);
    return k;
  };
  const uint32_t* made =
      LDS ? nullptr : e.keys + (int64_t)unit * e.key_stride;
  auto four = [&](int i) { return *(const u32x4*)((LDS ? keys : made) + i); };
  auto count = [&](uint32_t bin) {
    atomicAdd(&hist[bin * kEvCopies + lane % kEvCopies], 1u);
  };
  auto clear = [&] {
    for (int i = 4 * tid; i < kEvBins * kEvCopies; i += 4 * kEvThreads)
      *(u32x4*)(hist + i) = u32x4{};
    __syncthreads();
  };
  // The bin, from the largest down, in which the running count reaches
  // `need`: found[0], and the count above it: found[1]. Two bins a thread.
  auto locate = [&](uint32_t need) {
    __syncthreads();
    uint32_t n[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      static_assert(kEvCopies == 4, "one read a bin");
      const u32x4 h = *(const u32x4*)(hist + (kEvBins - 1 - 2 * tid - u) * 4);
      n[u] = h[0] + h[1] + h[2] + h[3];
    }
    uint32_t all;
    uint32_t before = lanes_before(n[0] + n[1], &all);
    if (lane == 0) wave_tot[wave] = all;
    __syncthreads();
    lanes_before(lane < wave ? wave_tot[lane] : 0u, &all);
    before += all;
    if (before < need && before + n[0] >= need) {
      found[0] = kEvBins - 1 - 2 * tid;
      found[1] = before;
    } else if (before + n[0] < need && before + n[0] + n[1] >= need) {
      found[0] = kEvBins - 2 - 2 * tid;
      found[1] = before + n[0];
    }
    __syncthreads();
  };
  constexpr int kStep = 4 * kEvThreads;

  // first digit
  if (tid == 0) listed = 0;
  if (tid < 4 * kEvWaves) runs[tid / kEvWaves][tid % kEvWaves] = 0;
  clear();
  if (LDS) {
#pragma unroll 2
    for (int i = 4 * tid; i < len; i += kStep) {
      const u32x4 k = make(i);
      *(u32x4*)(keys + i) = k;
      if (i + 4 <= len) {
#pragma unroll
        for (int u = 0; u < 4; ++u) count(k[u] >> 21);
      } else {
        for (int u = 0; u < (len & 3); ++u)
          count((u == 0 ? k[0] : u == 1 ? k[1] : k[2]) >> 21);
      }
    }
  } else {
    const uint32_t* part = e.chunk_hist + (int64_t)unit * e.chunks * kEvBins;
    const int n = (len + kEvChunk - 1) / kEvChunk;
    uint32_t s[2] = {};
#pragma unroll 8
    for (int i = 0; i < n; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        s[u] += part[(int64_t)i * kEvBins + tid + u * kEvThreads];
#pragma unroll
    for (int u = 0; u < 2; ++u)
      hist[(tid + u * kEvThreads) * kEvCopies] = s[u];
  }
  uint32_t need = (uint32_t)e.budget;   // keys still wanted among the matching
  locate(need);
  const uint32_t digit = found[0];
  uint32_t prefix = digit << 21;
  need -= found[1];

  // the keys that have it
  const int per = ((len + 256 * kEvWaves - 1) / (256 * kEvWaves)) * 256;
  const int a = min(wave * per, len), b = min(a + per, len);
  // f(keys i .. i + 3, i) over the wavefront's run, 256 slots at a time, all
  // lanes together (zeros past its end); kAhead of them are on their way
  auto run = [&](auto f) {
    constexpr int kAhead = LDS ? 2 : 8;
    for (int i0 = a; i0 < b; i0 += 256 * kAhead) {
      u32x4 k[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + 256 * u + 4 * lane;
        k[u] = u32x4{};
        if (i < b) k[u] = four(i);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i0 + 256 * u < b) f(k[u], i0 + 256 * u + 4 * lane);
    }
  };
  {
    int lo = 0, hi = 0;   // keys above, by side of the budget
    run([&](const u32x4& k, int i) {
      uint32_t gt = 0, eq = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t top = k[u] >> 21;
        gt |= (uint32_t)(top > digit) << u;
        eq |= (uint32_t)(top == digit) << u;
      }
      const uint32_t in = below4(i, b), low = below4(i, e.budget);
      gt &= in;
      lo += __popc(gt & low);
      hi += __popc(gt & ~low);
      // (one key at a time: the additions of a wavefront become one)
      for (eq &= in; eq; eq &= eq - 1) {
        const int u = __builtin_ctz(eq);
        const uint32_t at = atomicAdd(&listed, 1u);
        if (at < kEvList) {
          list_key[at] = u < 2 ? (u ? k[1] : k[0]) : (u == 3 ? k[3] : k[2]);
          list_slot[at] = i + u;
        }
      }
    });
    uint32_t all_lo, all_hi;
    lanes_before((uint32_t)lo, &all_lo);
    lanes_before((uint32_t)hi, &all_hi);
    if (lane == 0) {
      runs[0][wave] = (int)all_lo;
      runs[2][wave] = (int)all_hi;
    }
  }
  clear();
  const int n_list = (int)listed;
  const bool whole = n_list > kEvList;   // too many: all keys again
  // f(key, slot) for every key that may still matter
  auto each = [&](auto f) {
    if (!whole) {
      for (int i = tid; i < n_list; i += kEvThreads)
        f(list_key[i], list_slot[i]);
    } else {
      for (int i = 4 * tid; i < len; i += kStep) {
        const u32x4 k = four(i);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (i + u < len && k[u] >> 21 == digit)
            f(k[u], i + u);
      }
    }
  };
  each([&](uint32_t k, int) { count((k >> 10) & 2047u); });
  locate(need);
  prefix |= found[0] << 10;
  need -= found[1];
  clear();
  each([&](uint32_t k, int) {
    if ((k & 0xFFFFFC00u) == prefix) count(k & 1023u);
  });
  locate(need);
  prefix |= found[0];
  need -= found[1];
  // kept: keys above `prefix`, and the first `need` that equal it
  each([&](uint32_t k, int slot) {
    if (k >= prefix)
      atomicAdd(&runs[2 * (slot >= e.budget) + (k == prefix)][slot / per], 1);
  });
  __syncthreads();

  // what the runs before this one hold: equal keys, holes, kept tail slots; a
  // run a lane
  int eqs, holes, tails, all_eq;
  {
    const bool is = lane < kEvWaves;
    const int ua = min(lane * per, len), ub = min(ua + per, len);
    const int below = is ? max(0, min(ub, e.budget) - ua) : 0;
    const int g0 = is ? runs[0][lane] : 0, e0 = is ? runs[1][lane] : 0;
    const int g1 = is ? runs[2][lane] : 0, e1 = is ? runs[3][lane] : 0;
    uint32_t all;
    const int before = (int)lanes_before((uint32_t)(e0 + e1), &all);
    all_eq = (int)all;
    const int k0 = min(max((int)need - before, 0), e0);
    const int k1 = min(max((int)need - before - e0, 0), e1);
    const int h = (int)lanes_before((uint32_t)(below - g0 - k0), &all);
    const int s = (int)lanes_before((uint32_t)(g1 + k1), &all);
    eqs = __builtin_amdgcn_readlane(before, wave);
    holes = __builtin_amdgcn_readlane(h, wave);
    tails = __builtin_amdgcn_readlane(s, wave);
  }
  int32_t* to = e.to + (int64_t)unit * e.max_moves;
  int32_t* from = e.from + (int64_t)unit * e.max_moves;
  const bool ties = all_eq > (int)need;   // some equal keys go
  run([&](const u32x4& k, int i) {
    // slots in order: lane by lane, each its four
    uint32_t keep = 0, same = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      keep |= (uint32_t)(k[u] >= prefix) << u;
      same |= (uint32_t)(k[u] == prefix) << u;
    }
    const uint32_t in = below4(i, b), low = below4(i, e.budget);
    keep &= in;
    if (ties) {
      same &= in;
      uint32_t all;
      int left = (int)need - eqs -
                 (int)lanes_before((uint32_t)__popc(same), &all);
      eqs += (int)all;
      for (; same; same &= same - 1)
        if (left-- <= 0) keep &= ~(same & -same);
    }
    uint32_t out = in & low & ~keep, tail = keep & ~low;
    uint32_t all;
    const uint32_t at = lanes_before(
        (uint32_t)__popc(out) | (uint32_t)__popc(tail) << 16, &all);
    int h = holes + (int)(at & 0xFFFFu), s = tails + (int)(at >> 16);
    for (; out; out &= out - 1) to[h++] = i + __builtin_ctz(out);
    for (; tail; tail &= tail - 1) from[s++] = i + __builtin_ctz(tail);
    holes += (int)(all & 0xFFFFu);
    tails += (int)(all >> 16);
  });
  if (wave == kEvWaves - 1 && lane == 0) e.count[unit] = tails;
}

// The moves: RC lanes copy a row of K and of V, kMvRows rows each, all on
// their way at once (12.7 MB: 6.2 us, 7.2 one row after the other). A slot from the budget on is never written, so no move
// waits for another. The first work-group of a sequence's first head sets its
// length: nothing here reads that.
constexpr int kMvThreads = 256;
constexpr int kMvRows = 4;
template <int RC>
__global__ __launch_bounds__(kMvThreads) void evict_move_kernel(
    const CacheView c, const EvictCall e, int blocks_per_unit) {
  constexpr int kStep = kMvThreads / RC;
  const int unit = blockIdx.x / blocks_per_unit;
  const int part = blockIdx.x % blocks_per_unit;
  const int seq = unit / c.hkv, h = unit % c.hkv;
  if (part == 0 && h == 0 && threadIdx.x == 0 &&
      c.length[seq] > e.budget)
    c.length[seq] = e.budget;
  const int n = e.count[unit];
  const int ch = threadIdx.x % RC;
  const int i0 = part * kMvRows * kStep + (int)threadIdx.x / RC;
  if (i0 >= n) return;
  const int32_t* to = e.to + (int64_t)unit * e.max_moves;
  const int32_t* from = e.from + (int64_t)unit * e.max_moves;
  const int64_t at = h * c.head_bytes + 16 * ch, row = (int64_t)unit * c.cap;
  int src[kMvRows], dst[kMvRows];
  int64_t so[kMvRows], dp[kMvRows];
  i32x4 k[kMvRows], v[kMvRows];
#pragma unroll
  for (int u = 0; u < kMvRows; ++u) {   // (past the end: the first again)
    const int i = i0 + u * kStep < n ? i0 + u * kStep : i0;
    src[u] = from[i];
    dst[u] = to[i];
  }
#pragma unroll
  for (int u = 0; u < kMvRows; ++u) {
    so[u] = slot_offset(c, seq, src[u]);
    dp[u] = slot_offset(c, seq, dst[u]);
  }
#pragma unroll
  for (int u = 0; u < kMvRows; ++u)
    if (so[u] >= 0) {
      k[u] = *(const i32x4*)(c.k + so[u] + at);
      v[u] = *(const i32x4*)(c.v + so[u] + at);
    }
  float w[kMvRows];
  int32_t p[kMvRows];
  if (ch == 0)
#pragma unroll
    for (int u = 0; u < kMvRows; ++u) {
      w[u] = c.weight[row + src[u]];
      p[u] = c.pos[row + src[u]];
    }
#pragma unroll
  for (int u = 0; u < kMvRows; ++u) {
    if (u && i0 + u * kStep >= n) break;
    if (so[u] >= 0 && dp[u] >= 0) {
      *(i32x4*)(c.k + dp[u] + at) = k[u];
      *(i32x4*)(c.v + dp[u] + at) = v[u];
    }
    if (ch == 0) {
      c.weight[row + dst[u]] = w[u];
      c.pos[row + dst[u]] = p[u];
    }
  }
}

template <int RC>
hipError_t launch_move(const CacheView& c, const EvictCall& e, hipStream_t s) {
  const int units = c.n_seq * c.hkv;
  const int per = kMvRows * kMvThreads / RC;
  const int64_t parts = (e.max_moves + per - 1) / per;
  if (parts * units > 0x7FFFFFFF) return hipErrorInvalidValue;
  evict_move_kernel<RC><<<dim3((unsigned)(parts * units)), dim3(kMvThreads), 0,
                          s>>>(c, e, (int)parts);
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

size_t evict_layout(const CacheView& c, EvictCall& e, char* w) {
  const size_t n = (size_t)c.n_seq * c.hkv;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* const at = w + off;
    off += (bytes + 255) & ~size_t(255);
    return at;
  };
  e.max_moves = std::max(0, std::min(e.budget, e.max_len - e.budget));
  e.count = (int32_t*)take(n * 4);
  e.from = (int32_t*)take(n * e.max_moves * 4);
  e.to = (int32_t*)take(n * e.max_moves * 4);
  e.keys = e.chunk_hist = nullptr;
  if (e.max_len > kEvLdsKeys && e.max_moves) {
    e.chunks = (e.max_len + kEvChunk - 1) / kEvChunk;
    e.key_stride = (e.max_len + 3) & ~3;
    e.keys = (uint32_t*)take(n * e.key_stride * 4);
    e.chunk_hist = (uint32_t*)take(n * e.chunks * kEvBins * 4);
  }
  return off;
}

hipError_t launch_cache_evict(const CacheView& c, const EvictCall& e,
                              hipStream_t s) {
  const dim3 grid((unsigned)(c.n_seq * c.hkv)), block(kEvThreads);
  if ((int64_t)c.n_seq * c.hkv > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (!e.keys) {
    const size_t lds = ((size_t)e.max_len * 4 + 15) & ~size_t(15);
    if (lds > 0) {   // with the static arrays past 64 KB
      const hipError_t r = hipFuncSetAttribute(
          (const void*)evict_select_kernel<true>,
          hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (r != hipSuccess) return r;
    }
    evict_select_kernel<true><<<grid, block, lds, s>>>(c, e);
  } else {
    const int64_t n = (int64_t)c.n_seq * c.hkv * e.chunks;
    if (n > 0x7FFFFFFF) return hipErrorInvalidValue;
    evict_keys_kernel<<<dim3((unsigned)n), dim3(kKeyThreads), 0, s>>>(c, e);
    const hipError_t r = hipGetLastError();
    if (r != hipSuccess) return r;
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
