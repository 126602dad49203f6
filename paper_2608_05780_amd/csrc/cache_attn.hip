// Attention of drafted tokens over a paged cache, its join over the splits,
// and the accumulated attention weight.
#include <algorithm>

#include "attn_tiles.h"
#include "cache.h"

namespace evisel {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxTree = 64;
constexpr int kMaxSplits = 128;   // parts that a row is joined from
// Sequences up to which every work-group looks through all their lengths.
constexpr int kMaxBalanced = 256;
// Wavefronts of a work-group that takes 16 RT rows.
constexpr int waves_of(int row_tiles) { return row_tiles == 4 ? 4 : 8; }

// Over the four lanes that hold one query row (lane % 16).
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// The two operand paths. Both products keep the query row in the lane:
// S^T = K Q^T leaves lane (c = lane % 16, g = lane / 16) with the logits of
// row c for the keys 4g .. 4g + 3 of every 16, and O^T += V^T P^T takes P
// from exactly those registers. K's operand is 16 bytes of key c a step and
// comes from memory as it is. V's operand wants several keys at one column:
// a lane reads the columns of chunk c of the keys that it holds logits of,
// and turns the small square around in its registers. So nothing passes
// through LDS or waits at a barrier between the pages and the matrix cores.
template <int D>
struct TreeBf16 {
  static constexpr int ES = 2, KT = 32, NH = 2;
  static constexpr int KS = D * ES / 64;   // 64-byte steps of a row
  static constexpr int VC = D / 16;        // columns of a lane's V chunk
  static constexpr int NT = D / 16;        // 16-column tiles of O^T
  typedef uint32_t chunk __attribute__((ext_vector_type(VC / 2)));
  struct Row {
    bf16x8 x[KS];
  };
  struct Val {
    chunk x[NH][4];
  };
  // V's lane offset within a row, and O's column of (g, i, t)
  static constexpr int kLaneV = VC * ES;
  static __device__ int col(int g, int i, int t) {
    return VC * (4 * g + i) + t;
  }
  static __device__ void load_row(Row& r, const char* p) {
#pragma unroll
    for (int j = 0; j < KS; ++j) r.x[j] = *(const bf16x8*)(p + 64 * j);
  }
  static __device__ void load_val(chunk& v, const char* p) {
    v = *(const chunk*)p;
  }
  static __device__ void zero_val(chunk& v) { v = chunk{}; }
  static __device__ void zero_row(Row& r) {
#pragma unroll
    for (int j = 0; j < KS; ++j) r.x[j] = bf16x8{};
  }
  static __device__ f32x4 qk(const Row& k, const Row& q) {
    f32x4 s = {};
#pragma unroll
    for (int j = 0; j < KS; ++j)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.x[j], q.x[j], s, 0, 0, 0);
    return s;
  }
  // The A operands of V^T, for every column of the chunk its eight keys: 4g ..
  // 4g + 3 of the first 16, then of the second.
  struct ValT {
    bf16x8 x[NT];
  };
  static __device__ void turn(ValT& o, const Val& v) {
#pragma unroll
    for (int w = 0; w < VC / 2; ++w) {
      u32x4 lo, hi;
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const uint32_t a = v.x[p / 2][2 * (p % 2)][w];
        const uint32_t b = v.x[p / 2][2 * (p % 2) + 1][w];
        lo[p] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        hi[p] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      }
      o.x[2 * w] = __builtin_bit_cast(bf16x8, lo);
      o.x[2 * w + 1] = __builtin_bit_cast(bf16x8, hi);
    }
  }
  static __device__ void pv(f32x4 (&o)[NT], const ValT& v,
                            const f32x4 (&p)[NH]) {
    const f32x8 pf = __builtin_shufflevector(p[0], p[1], 0, 1, 2, 3, 4, 5, 6, 7);
    // rounded to bf16 for the matrix cores: half a step, 2^-9 of a
    // probability, and independent from key to key
    const bf16x8 pb = __builtin_convertvector(pf, bf16x8);
#pragma unroll
    for (int t = 0; t < NT; ++t)
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.x[t], pb, o[t], 0, 0, 0);
  }
  static __device__ bool finite(const chunk& v) {
    bool ok = true;
#pragma unroll
    for (int w = 0; w < VC / 2; ++w)
      ok = ok && (v[w] & 0x7F80u) != 0x7F80u &&
           (v[w] & 0x7F800000u) != 0x7F800000u;
    return ok;
  }
  static __device__ void drop_infinite(chunk& v) {
#pragma unroll
    for (int w = 0; w < VC / 2; ++w) {
      if ((v[w] & 0x7F80u) == 0x7F80u) v[w] &= 0xFFFF0000u;
      if ((v[w] & 0x7F800000u) == 0x7F800000u) v[w] &= 0xFFFFu;
    }
  }
  static __device__ float element(const char* row, int e) {
    return __uint_as_float((uint32_t)((const uint16_t*)row)[e] << 16);
  }
  template <int N>
  static __device__ void store(char* dst, const float (&x)[N]) {
    typedef __bf16 out_t __attribute__((ext_vector_type(N)));
    typedef float in_t __attribute__((ext_vector_type(N)));
    in_t v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = x[i];
    *(out_t*)dst = __builtin_convertvector(v, out_t);
  }
};

template <int D>
struct TreeF32 {
  static constexpr int ES = 4, KT = 16, NH = 1;
  static constexpr int KS = D * ES / 64;
  static constexpr int NT = D / 16;
  static constexpr int NC = D / 64;        // 16-byte chunks of V per lane
  struct chunk {
    f32x4 x[NC];
  };
  struct Row {
    f32x4 x[KS];
  };
  struct Val {
    chunk x[NH][4];
  };
  static constexpr int kLaneV = 16;
  static __device__ int col(int g, int i, int t) {
    return 64 * (t / 4) + 4 * (4 * g + i) + t % 4;
  }
  static __device__ void load_row(Row& r, const char* p) {
#pragma unroll
    for (int j = 0; j < KS; ++j) r.x[j] = *(const f32x4*)(p + 64 * j);
  }
  static __device__ void load_val(chunk& v, const char* p) {
#pragma unroll
    for (int j = 0; j < NC; ++j) v.x[j] = *(const f32x4*)(p + 256 * j);
  }
  static __device__ void zero_val(chunk& v) { v = chunk{}; }
  static __device__ void zero_row(Row& r) {
#pragma unroll
    for (int j = 0; j < KS; ++j) r.x[j] = f32x4{};
  }
  // Four sums, which are added at the end: a quarter of the roundings at the
  // size of the whole logit (one sum: 1.6e-6 of the output at d = 64, plain
  // fp32 4.5e-7).
  static __device__ f32x4 qk(const Row& k, const Row& q) {
    f32x4 s[4] = {};
#pragma unroll
    for (int j = 0; j < KS; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x[j][e], q.x[j][e], s[e],
                                                    0, 0, 0);
    return (s[0] + s[1]) + (s[2] + s[3]);
  }
  typedef Val ValT;   // one key a step: as it came
  static __device__ void turn(ValT& o, const Val& v) { o = v; }
  static __device__ void pv(f32x4 (&o)[NT], const ValT& v,
                            const f32x4 (&p)[NH]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.x[0][i].x[t / 4][t % 4],
                                                    p[0][i], o[t], 0, 0, 0);
  }
  static __device__ bool finite(const chunk& v) {
    bool ok = true;
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) ok = ok && __builtin_isfinite(v.x[j][e]);
    return ok;
  }
  static __device__ void drop_infinite(chunk& v) {
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (!__builtin_isfinite(v.x[j][e])) v.x[j][e] = 0.f;
  }
  static __device__ float element(const char* row, int e) {
    return ((const float*)row)[e];
  }
  template <int N>
  static __device__ void store(char* dst, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) ((float*)dst)[i] = x[i];
  }
};

struct Yes {
  static constexpr bool value = true;
};
struct No {
  static constexpr bool value = false;
};

// The page table is not written while a kernel reads it: scalar loads.
typedef const __attribute__((address_space(4))) int32_t* ScalarTable;

// A sequence's part of a call.
struct Tree {
  int first, n;   // its rows of q and their number
  int len;        // cached tokens
};
__device__ __forceinline__ Tree tree_of(const CacheView& c, const TreeCall& t,
                                        int seq) {
  Tree r;
  r.first = min(max(t.tree_ptr[seq], 0), t.n_tok);
  r.n = min(max(t.tree_ptr[seq + 1], r.first), t.n_tok) - r.first;
  r.n = min(r.n, t.max_tree);
  r.len = held(c, seq, t.max_len);
  return r;
}

// Tiles of kt keys: the cache's and the drafted tokens'; none without tokens.
__device__ __forceinline__ int cached_tiles(const Tree& r, int kt) {
  return (r.len + kt - 1) / kt;
}
__device__ __forceinline__ int tiles_of(const Tree& r, const TreeCall& t,
                                        int kt) {
  if (r.n == 0) return 0;
  return max(1, cached_tiles(r, kt) + (t.k_new ? (r.n + kt - 1) / kt : 0));
}

// A work-group's run of keys: run `run` of the `used` ones of `per` tiles that
// sequence `seq` has, whose parts start at index `slot`. seq is -1 if the
// work-group has nothing to do. The first run of a sequence leaves slot and
// used in the workspace for what joins the parts.
struct Share {
  int seq, run, per, used, slot;
};
// The same number of runs for each sequence, whatever its length.
__device__ __forceinline__ Share even_share(const CacheView& c,
                                            const TreePlan& pl,
                                            const TreeCall& t, int kt, int seq,
                                            int run) {
  Share r;
  r.seq = seq;
  r.run = run;
  r.slot = seq * pl.splits;
  const int n = tiles_of(tree_of(c, t, seq), t, kt);
  r.per = max(1, (n + pl.splits - 1) / pl.splits);
  r.used = (n + r.per - 1) / r.per;
  if (run >= r.used) r.seq = -1;
  return r;
}
// The tiles of all sequences over the work-groups that the card holds at
// once, so that long and short sequences make work-groups of one size: every
// wavefront finds its run for itself from the lengths on the device.
__device__ __forceinline__ Share fair_share(const CacheView& c,
                                            const TreePlan& pl,
                                            const TreeCall& t, int kt,
                                            int group) {
  if (!pl.balanced)
    return even_share(c, pl, t, kt, group / pl.splits, group % pl.splits);
  Share r;
  const int lane = threadIdx.x & 63;
  auto tiles = [&](int s0) {
    return s0 + lane < c.n_seq ? tiles_of(tree_of(c, t, s0 + lane), t, kt) : 0;
  };
  const int first = tiles(0), wide = min(c.n_seq, 64);
  int total = 0, active = 0, longest = 0;
  for (int s0 = 0; s0 < c.n_seq; s0 += 64) {
    const int n = s0 ? tiles(s0) : first;
    int sum = n, top = n;
    for (int o = 1; o < wide; o <<= 1) {
      sum += __shfl_xor(sum, o);
      top = max(top, __shfl_xor(top, o));
    }
    total += __builtin_amdgcn_readfirstlane(sum);
    longest = max(longest, __builtin_amdgcn_readfirstlane(top));
    active += __popcll(__ballot(n > 0));
  }
  // a run left over at the end of each sequence fits in, too
  const int room = max(pl.goal - active, (pl.goal + 1) / 2);
  int per = (total + room - 1) / room;
  per = max(max(per, pl.least), (longest + pl.most_runs - 1) / pl.most_runs);
  r.per = __builtin_amdgcn_readfirstlane(per);
  r.seq = -1;
  r.run = r.used = r.slot = 0;
  int before = 0;
  for (int s0 = 0; s0 < c.n_seq; s0 += 64) {
    const int n = s0 ? tiles(s0) : first, used = (n + r.per - 1) / r.per;
    int run = used;
    for (int o = 1; o < wide; o <<= 1) {
      const int up = __shfl_up(run, o);
      if (lane >= o) run += up;
    }
    run += before;   // of this sequence and all before it
    const uint64_t here = __ballot(lane < wide && group < run);
    if (here) {
      const int l = __builtin_ctzll(here);
      r.seq = s0 + l;
      r.used = __builtin_amdgcn_readlane(used, l);
      r.slot = __builtin_amdgcn_readlane(run, l) - r.used;
      r.run = group - r.slot;
      return r;
    }
    before = __builtin_amdgcn_readlane(run, wide - 1);
  }
  return r;
}

// Many rows (wide): a work-group takes 256 of them, kWideRows a wavefront,
// and where half of the wavefronts or fewer have rows, two share them, each
// with one half of the keys.
constexpr int kWideRt = 2, kWideRows = 16 * kWideRt;
constexpr int kWideWaves = 8;
constexpr int kWideBlock = kWideRows * kWideWaves;
constexpr int kWideKeys = 64;   // of a stage
__device__ __forceinline__ int key_halves(int n_rows, int row0) {
  return n_rows - row0 <= kWideBlock / 2 ? 2 : 1;
}
// Which drafted tokens token `lane` sees: itself and its ancestors. The lanes'
// parents are followed by doubling, six times for 64 tokens.
__device__ __forceinline__ uint64_t ancestors(const TreeCall& t, const Tree& r,
                                              int lane) {
  if (!t.parent) return ~0ull >> (63 - lane);
  int up = lane < r.n ? t.parent[r.first + lane] : -1;
  if (up < 0 || up >= lane) up = lane;   // a root sees itself
  uint64_t m = 1ull << lane;
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    m |= __shfl(m, up);
    up = __shfl(up, up);
  }
  return m;
}

// A tile's rows in memory: address of the first key of every 16 (K's pool and
// V's alike) and how many of the 16 are there.
template <int NH>
struct Where {
  int64_t off[NH];
  int n[NH];
};
// The page of slot `slot` (past the end: the last page, which is not used).
__device__ __forceinline__ int page_of(const CacheView& c, int seq, int len,
                                       int slot) {
  return ((ScalarTable)c.table)[(int64_t)seq * c.max_pages +
                                (max(min(slot, len - 1), 0) >> c.page_shift)];
}
// Rows slot .. slot + 15 of page `id`: their address and their number.
__device__ __forceinline__ int place(int64_t& off, const CacheView& c, int id,
                                     int64_t head, int len, int slot) {
  const bool ok = slot < len && (uint32_t)id < (uint32_t)c.n_pages;
  off = (ok ? id : 0) * c.page_bytes + head +
        (ok ? (int64_t)(slot & ((1 << c.page_shift) - 1)) : 0) * c.token_bytes;
  return ok ? min(16, len - slot) : 0;
}
template <int NH>
__device__ __forceinline__ void find(Where<NH>& w, const CacheView& c, int seq,
                                     int64_t head, int len, int slot0) {
#pragma unroll
  for (int h = 0; h < NH; ++h)
    w.n[h] = place(w.off[h], c, page_of(c, seq, len, slot0 + 16 * h), head, len,
                   slot0 + 16 * h);
}

template <class P>
__device__ __forceinline__ void fetch_k(typename P::Row (&k)[P::NH],
                                        const CacheView& c,
                                        const Where<P::NH>& at,
                                        uint32_t koff) {
#pragma unroll
  for (int h = 0; h < P::NH; ++h) P::load_row(k[h], c.k + at.off[h] + koff);
}
template <class P>
__device__ __forceinline__ void fetch_v(typename P::Val& v, const CacheView& c,
                                        const Where<P::NH>& at,
                                        uint32_t voff) {
#pragma unroll
  for (int h = 0; h < P::NH; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      P::load_val(v.x[h][i], c.v + at.off[h] + (voff + i * c.token_bytes));
}

// One wavefront's running softmax over RT tiles of 16 query rows.
template <class P, int D, int RT>
struct Rows {
  typename P::Row q[RT];
  f32x4 o[RT][P::NT];
  float m[RT], l[RT];   // reference (log2 units) and sum

  __device__ __forceinline__ void logits(f32x4 (&x)[RT][P::NH],
                                         const typename P::Row (&k)[P::NH]) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int h = 0; h < P::NH; ++h) x[rt][h] = P::qk(k[h], q[rt]);
  }
  // vis[rt]: bit 4h + i set if the row sees key 16h + 4g + i.
  __device__ __forceinline__ static void hide(f32x4 (&x)[RT][P::NH],
                                              const uint32_t (&vis)[RT]) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int h = 0; h < P::NH; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(vis[rt] >> (4 * h + i) & 1)) x[rt][h][i] = neg_inf();
  }
  // Moves the references of rows that a logit has passed.
  __device__ __forceinline__ void refer(const f32x4 (&x)[RT][P::NH],
                                        const TreeCall& t) {
    float top[RT];
    bool past = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      top[rt] = neg_inf();
#pragma unroll
      for (int h = 0; h < P::NH; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) top[rt] = fmaxf(top[rt], x[rt][h][i]);
      past = past || top[rt] * t.scale_log2 > m[rt] + kTreeSlack;
    }
    if (__any(past)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float next = fmaxf(m[rt], row_max(top[rt]) * t.scale_log2);
        const float a = m[rt] == neg_inf() ? 0.f : exp2_(m[rt] - next);
        m[rt] = next;
        l[rt] *= a;
#pragma unroll
        for (int u = 0; u < P::NT; ++u) o[rt][u] *= a;
      }
    }
  }
  // Logits to probabilities against the references, and their sums.
  __device__ __forceinline__ void weigh(f32x4 (&x)[RT][P::NH],
                                        const TreeCall& t) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float ref = m[rt] == neg_inf() ? 0.f : m[rt];
#pragma unroll
      for (int h = 0; h < P::NH; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[rt][h][i] = t.exp_of(x[rt][h][i], ref);
          l[rt] += x[rt][h][i];
        }
    }
  }
  __device__ __forceinline__ void softmax(f32x4 (&x)[RT][P::NH],
                                          const TreeCall& t) {
    refer(x, t);
    weigh(x, t);
  }
  __device__ __forceinline__ void add(const typename P::ValT& v,
                                      const f32x4 (&x)[RT][P::NH]) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) P::pv(o[rt], v, x[rt]);
  }
};

// A tile of drafted tokens j0 .. j0 + KT - 1: every row sees keys of its own.
// score: where a row's logits of the cache start, or null; probs: 16 RT KT
// floats of LDS of the wavefront's own.
template <class P, int D, int RT>
__device__ __forceinline__ void take_drafts(Rows<P, D, RT>& rows,
                                            const CacheView& c,
                                            const TreeCall& t, const Tree& tr,
                                            int kvh, int row0, int n_rows,
                                            int j0, float* score,
                                            int64_t len_pad, float* probs) {
  constexpr int KT = P::KT, NH = P::NH;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
  const int group = t.hq / c.hkv;
  const uint64_t anc = ancestors(t, tr, lane);
  const int64_t step = (int64_t)c.hkv * (D * P::ES);
  const int64_t base = (int64_t)tr.first * step + kvh * (D * P::ES);
  struct {
    typename P::Row k[NH];
    typename P::Val v;
  } x;
  bool fine = true;
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    const int j = min(j0 + 16 * h + c16, tr.n - 1);
    P::load_row(x.k[h], t.k_new + base + j * step + 16 * g);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int jv = j0 + 16 * h + 4 * g + i;
      if (jv < tr.n) {
        P::load_val(x.v.x[h][i], t.v_new + base + jv * step + c16 * P::kLaneV);
        fine = fine && P::finite(x.v.x[h][i]);
      } else {
        P::zero_val(x.v.x[h][i]);
      }
    }
  }
  uint32_t vis[RT];
  uint32_t sees[RT];   // by key of the tile
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + 16 * rt + c16;
    const uint64_t all = __shfl(anc, t.token_of(min(r, n_rows - 1)));
    sees[rt] = r < n_rows ? (uint32_t)(all >> j0) : 0u;
    vis[rt] = 0;
#pragma unroll
    for (int h = 0; h < NH; ++h)
      vis[rt] |= (sees[rt] >> (16 * h + 4 * g) & 15u) << (4 * h);
  }
  f32x4 p[RT][NH];
  rows.logits(p, x.k);
  rows.hide(p, vis);
  if (score)
#pragma unroll
    for (int h = 0; h < NH; ++h)
      *(f32x4*)(score + len_pad + j0 + 16 * h) = p[0][h];
  rows.softmax(p, t);
  // A value that is not finite reaches the rows that see its token and no
  // other: it is left out of the product, whose zeros it would spoil, and
  // added by itself.
  const bool plain = __all(fine);
  if (!plain) {
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) P::drop_infinite(x.v.x[h][i]);
  }
  typename P::ValT vt;
  P::turn(vt, x.v);
  rows.add(vt, p);
  if (plain) return;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int h = 0; h < NH; ++h)
      *(f32x4*)(probs + (16 * rt + c16) * KT + 16 * h + 4 * g) = p[rt][h];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int j = 0; j < KT && j0 + j < tr.n; ++j) {
    const char* v = t.v_new + base + (j0 + j) * step;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if (!(sees[rt] >> j & 1)) continue;
      const float pj = probs[(16 * rt + c16) * KT + j];
#pragma unroll
      for (int u = 0; u < P::NT; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = P::element(v, P::col(g, i, u));
          if (!__builtin_isfinite(e)) rows.o[rt][u][i] += pj * e;
        }
    }
  }
  __builtin_amdgcn_wave_barrier();
}

// One work-group: a sequence, a kv head, a run of its key tiles (a split) and
// 16 RT of its query rows. The wavefronts take the run's tiles in turn, each
// with the next tile's rows on their way while it works on one, and are
// joined in LDS at the end. Bound by memory: 64 sequences of up to 8,000 tokens
// (28 / 4 heads, d = 128, bf16, 536 MB) take 127-132 us with their logits stored,
// 4.4 TB/s of a copy's 4.9; a single one of 16,512 tokens 11 us, of which a run's
// start and end are 4 and its one round of tiles 2 to 3. What a run's rows come to is the output, if the
// sequence has one run, or a partial sum in the workspace.
template <class P, int D, int RT, bool SCORE>
__global__ __launch_bounds__(64 * waves_of(RT), RT == 4 ? 1 : 2) void tree_kernel(
    const CacheView c, const TreePlan pl, const TreeCall t) {
  constexpr int KT = P::KT, NH = P::NH, kWaves = waves_of(RT);
  constexpr int kPad = D + 4;
  // a wavefront's share of one row tile's O, or its probabilities of a tile
  constexpr int kOwn = RT * KT > kPad ? 16 * RT * KT : 16 * kPad;
  __shared__ __attribute__((aligned(16))) float so[kWaves][kOwn];
  __shared__ float sm[kWaves][16 * RT], sl[kWaves][16 * RT];
  // consecutive work-groups go to the 8 XCDs in turn; the row blocks of one
  // run stay on one of them, whose L2 then serves the run's keys again
  const int xcd = blockIdx.x % 8, y = blockIdx.x / 8;
  const int rb = y % pl.row_blocks;
  int unit = y / pl.row_blocks * 8 + xcd;
  if (unit >= pl.groups * c.hkv) return;
  const int split = unit % pl.splits;
  unit /= pl.splits;
  const int kvh = unit % c.hkv;
  const Share sh = even_share(c, pl, t, KT, unit / c.hkv, split);
  if (sh.seq < 0) return;
  const int seq = sh.seq;
  if (pl.joined && sh.run == 0 && kvh == 0 && rb == 0 && threadIdx.x == 0) {
    t.share[2 * seq] = sh.slot;
    t.share[2 * seq + 1] = sh.used;
  }
  unit = seq * c.hkv + kvh;
  const Tree tr = tree_of(c, t, seq);
  const int group = t.hq / c.hkv, n_rows = tr.n * group;
  const int row0 = rb * 16 * RT;
  if (row0 >= n_rows) return;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cached = cached_tiles(tr, KT);
  const int t0 = sh.run * sh.per;
  const int t1 = min(t0 + sh.per, tiles_of(tr, t, KT));
  const int64_t head = kvh * c.head_bytes;
  const uint32_t koff = (uint32_t)c16 * c.token_bytes + 16 * g;
  const uint32_t voff = (uint32_t)(4 * g) * c.token_bytes + c16 * P::kLaneV;

  Rows<P, D, RT> rows;
  float* score[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + 16 * rt + c16;
    rows.m[rt] = neg_inf();
    rows.l[rt] = 0.f;
#pragma unroll
    for (int i = 0; i < P::NT; ++i) rows.o[rt][i] = f32x4{};
    if (r < n_rows) {
      const int tok = t.token_of(r), qh = r - tok * group;
      P::load_row(rows.q[rt],
                  t.q + ((int64_t)(tr.first + tok) * t.hq + kvh * group + qh) *
                            (D * P::ES) + 16 * g);
    } else {
      P::zero_row(rows.q[rt]);
    }
    score[rt] = SCORE && r < n_rows
                    ? t.score + ((int64_t)unit * pl.rows + r) *
                                    (pl.len_pad + kMaxTree) + 4 * g
                    : nullptr;
  }

  const int c_end = min(t1, cached);
  int tile = t0 + wave;
  if (tile < c_end) {
    const int end = min(tr.len, c_end * KT);
    typename P::Row k[NH];
    typename P::Val v;
    Where<NH> at, next;
    find<NH>(at, c, seq, head, end, tile * KT);
    fetch_k<P>(k, c, at, koff);
    fetch_v<P>(v, c, at, voff);
    // K's and V's registers are refilled as soon as a product has read them
    auto take = [&](auto more) {
      constexpr bool kMore = decltype(more)::value;
      if (kMore) find<NH>(next, c, seq, head, end, (tile + kWaves) * KT);
      f32x4 x[RT][NH];
      rows.logits(x, k);
      if (kMore) fetch_k<P>(k, c, next, koff);
      bool full = true;
#pragma unroll
      for (int h = 0; h < NH; ++h) full = full && at.n[h] == 16;
      if (!full) {
        // keys past the end, or without a page: no row sees them, and their
        // values, whatever they are, must not meet a probability of zero
        uint32_t vis[RT] = {};
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (4 * g + i < at.n[h])
              vis[0] |= 1u << (4 * h + i);
            else
              P::zero_val(v.x[h][i]);
          }
#pragma unroll
        for (int rt = 1; rt < RT; ++rt) vis[rt] = vis[0];
        rows.hide(x, vis);
      }
      if (SCORE && score[0])
#pragma unroll
        for (int h = 0; h < NH; ++h)
          *(f32x4*)(score[0] + (int64_t)tile * KT + 16 * h) = x[0][h];
      rows.softmax(x, t);
      typename P::ValT vt;
      P::turn(vt, v);
      if (kMore) fetch_v<P>(v, c, next, voff);
      rows.add(vt, x);
      at = next;
    };
    for (; tile + kWaves < c_end; tile += kWaves) take(Yes{});
    take(No{});
  }
  for (tile = t0 + wave; tile < t1; tile += kWaves) {
    if (tile < cached || !t.k_new) continue;
    take_drafts<P, D, RT>(rows, c, t, tr, kvh, row0, n_rows,
                          (tile - cached) * KT,
                          SCORE ? score[0] : nullptr, pl.len_pad, so[wave]);
  }

  // the wavefronts' rows
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    rows.l[rt] = row_sum(rows.l[rt]);
    if (g == 0) {
      sm[wave][16 * rt + c16] = rows.m[rt];
      sl[wave][16 * rt + c16] = rows.l[rt];
    }
  }
  __syncthreads();
  constexpr int kCols = 16 * D / (64 * kWaves);   // of a thread
  const int er = threadIdx.x / (D / kCols), ec = threadIdx.x % (D / kCols);
  const int padded = pl.padded;
  const int64_t part = ((int64_t)(sh.slot + sh.run) * c.hkv + kvh) * padded;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = neg_inf();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm[w][16 * rt + c16]);
    const float f =
        rows.m[rt] == neg_inf() ? 0.f : exp2_(rows.m[rt] - top);
#pragma unroll
    for (int u = 0; u < P::NT; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        so[wave][c16 * kPad + P::col(g, i, u)] = rows.o[rt][u][i] * f;
    __syncthreads();
    const int r = row0 + 16 * rt + er;
    if (r < n_rows) {
      float big = neg_inf(), sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        big = fmaxf(big, sm[w][16 * rt + er]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float mw = sm[w][16 * rt + er];
        sum += (mw == neg_inf() ? 0.f : exp2_(mw - big)) *
               sl[w][16 * rt + er];
      }
      float x[kCols] = {};
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int i = 0; i < kCols; ++i)
          x[i] += so[w][er * kPad + ec * kCols + i];
      if (sh.used == 1) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < kCols; ++i) x[i] *= inv;
        const int tok = t.token_of(r), h = kvh * group + r - tok * group;
        P::template store<kCols>(
            t.out + ((int64_t)(tr.first + tok) * t.hq + h) * (D * P::ES) +
                ec * kCols * P::ES, x);
        if (ec == 0) {
          if (t.lse)
            t.lse[(int64_t)h * t.n_tok + tr.first + tok] = t.lse_of(big, sum);
          if (t.accumulate) {
            t.row_m[(int64_t)unit * padded + r] = big;
            t.row_inv[(int64_t)unit * padded + r] = inv;
          }
        }
      } else {
        float* dst = t.pO + (part + r) * D + ec * kCols;
#pragma unroll
        for (int i = 0; i < kCols; ++i) dst[i] = x[i];
        if (ec == 0) {
          t.pM[part + r] = big;
          t.pL[part + r] = sum;
        }
      }
    }
    __syncthreads();
  }
}

// Many query rows of bf16: here the matrix cores are the bound, and the
// wavefronts, 32 rows each, share every key. A stage of 64 keys passes from
// memory straight into one of three LDS buffers, two stages ahead of the one
// that is worked on; one barrier a stage.
// The products are those of tree_kernel, but V's operand comes from LDS by
// transposing reads: four lanes a key name the 16 columns, and lane c holds
// column c of four keys; the columns are chosen so that a lane's share of O is
// one run. Both buffers are swizzled in 16-byte chunks so that the lanes of
// one read touch every bank once.
// A tree of 64 tokens and 28 / 4 heads over 65,664 tokens (60 GFLOP): 95 us, MFMA
// busy 26 % of the time; with the keys' rows read by each wavefront from memory
// (tree_kernel, 64 rows a wavefront) 150.
template <class P, int D>
__global__ __launch_bounds__(64 * kWideWaves, kWideRt == 2 ? 2 : 1) void tree_wide_kernel(
    const CacheView c, const TreePlan pl, const TreeCall t) {
  constexpr int RT = kWideRt, KT = P::KT, NH = P::NH, NT = P::NT;
  constexpr int RC = D * P::ES / 16;             // 16-byte chunks of a row
  constexpr int kRuns = kWideKeys / 16;          // runs of 16 keys: one page
  constexpr int kBytes = kWideKeys * D * P::ES;
  __shared__ __attribute__((aligned(16))) char buf[3][2][kBytes];   // K, V
  __shared__ __attribute__((aligned(16))) float probs[kWideWaves][16 * RT * KT];
  __shared__ int odd;   // a drafted value that is not finite
  const int xcd = blockIdx.x % 8, y = blockIdx.x / 8;
  const int rb = y % pl.row_blocks;
  int unit = y / pl.row_blocks * 8 + xcd;
  if (unit >= pl.groups * c.hkv) return;
  const int kvh = unit % c.hkv;
  const Share sh = fair_share(c, pl, t, kWideKeys, unit / c.hkv);
  if (sh.seq < 0) return;
  const int seq = sh.seq;
  if (pl.joined && sh.run == 0 && kvh == 0 && rb == 0 && threadIdx.x == 0) {
    t.share[2 * seq] = sh.slot;
    t.share[2 * seq + 1] = sh.used;
  }
  unit = seq * c.hkv + kvh;
  const Tree tr = tree_of(c, t, seq);
  const int group = t.hq / c.hkv, n_rows = tr.n * group;
  const int block0 = rb * kWideBlock;
  if (block0 >= n_rows) return;
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int halves = key_halves(n_rows, block0);
  // the steps of a stage that this wavefront takes: from `half` on, every
  // halves-th
  const int half = halves == 2 ? wave / (kWideWaves / 2) : 0;
  const int row0 =
      block0 + (halves == 2 ? wave % (kWideWaves / 2) : wave) * kWideRows;
  const bool works = row0 < n_rows;
  const int64_t head = kvh * c.head_bytes;

  Rows<P, D, RT> rows;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + 16 * rt + c16;
    rows.m[rt] = neg_inf();
    rows.l[rt] = 0.f;
#pragma unroll
    for (int i = 0; i < NT; ++i) rows.o[rt][i] = f32x4{};
    if (r < n_rows) {
      const int tok = t.token_of(r), qh = r - tok * group;
      P::load_row(rows.q[rt],
                  t.q + ((int64_t)(tr.first + tok) * t.hq + kvh * group + qh) *
                            (D * P::ES) + 16 * g);
    } else {
      P::zero_row(rows.q[rt]);
    }
  }

  const int s0 = sh.run * sh.per;
  const int s1 = min(s0 + sh.per, cached_tiles(tr, kWideKeys));
  auto k_swizzle = [](int r) { return RC == 16 ? r & 15 : (r >> 1) & 7; };
  // a transposing read names four keys, and of each four chunks, every
  // fourth (D = 64: every second, of two keys in a line of 256 bytes)
  auto v_swizzle = [](int r) { return RC == 16 ? r & 3 : (r >> 1) & 1; };
  // A wavefront sends for K or V of one run of 16 keys, which is in one page:
  // 1 KB a load, its rows neighbours in LDS; the swizzle is in what a lane
  // fetches. The page is looked up a stage before.
  constexpr int kLoads = 16 * RC / 64;      // of a run
  constexpr int kLoadRows = 64 / RC;        // of a load
  static_assert(kWideWaves == 2 * kRuns, "one run of K or V a wavefront");
  const int my_run = wave / 2;
  const char* const pool = wave % 2 ? c.v : c.k;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(EV_LDS char*)&buf[0][0][0] +
                        (uint32_t)(wave % 2 * kBytes + my_run * 256 * RC);
  uint32_t from[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int r = j * kLoadRows + lane / RC;
    const int ch = lane % RC ^ (wave % 2 ? v_swizzle(r) : k_swizzle(r));
    from[j] = (uint32_t)r * c.token_bytes + 16 * ch;
  }
  int page = 0;
  auto look = [&](int stage) {
    page = page_of(c, seq, tr.len, stage * kWideKeys + 16 * my_run);
  };
  auto fetch = [&](int stage, int b) {
    int64_t at;
    place(at, c, page, head, tr.len, stage * kWideKeys + 16 * my_run);
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      lds_dma16(lds0 + (uint32_t)(2 * b * kBytes + j * 1024), pool + at,
                from[j]);
    look(stage + 1);
  };
  // Keys that are there of run i of a stage, where not all need be.
  auto there = [&](int stage, int i) {
    const int slot = stage * kWideKeys + 16 * i;
    int64_t at;
    return place(at, c, page_of(c, seq, tr.len, slot), head, tr.len, slot);
  };
  // Whether a page of this split is missing: then every stage is looked
  // through, otherwise only one that passes the end.
  int missing = 0;
  for (int i = s0 * kRuns + tid; i < s1 * kRuns; i += 64 * kWideWaves)
    missing |= 16 * i < tr.len &&
               (uint32_t)c.table[(int64_t)seq * c.max_pages +
                                 (16 * i >> c.page_shift)] >=
                   (uint32_t)c.n_pages;
  const bool holes = __syncthreads_or(missing);
  auto partial = [&](int stage) {
    return holes || (stage + 1) * kWideKeys > tr.len;
  };
  // Waits for a stage, not for the `later` one sent for after it. Keys past
  // the end or without a page: no row sees them, and their values must not
  // meet a probability of zero.
  auto arrive = [&](int stage, int b, bool later) {
    if (later)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (!partial(stage)) return;
    for (int u = tid; u < kWideKeys * RC; u += 64 * kWideWaves)
      if (u / RC % 16 >= there(stage, u / RC / 16))
        *(u32x4*)&buf[b][1][u * 16] = u32x4{};
    __syncthreads();
  };
  typename P::Row k[NH];
  auto read_k = [&](int b, int sub) {
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const int r = KT * sub + 16 * h + c16;
#pragma unroll
      for (int j = 0; j < P::KS; ++j)
        k[h].x[j] = *(const bf16x8*)&buf[b][0][(r * RC + ((g + 4 * j) ^
                                                          k_swizzle(r))) * 16];
    }
  };
  // V's operands of a step: tile u's column of lane c is D / 4 (c / 4) + 4u +
  // c % 4; lane j of 16 names the row 4g + j / 4 and the columns of j % 4
  auto read_v = [&](bf16x8 (&va)[NT], int b, int sub) {
    const int r = 4 * g + (c16 >> 2);   // and 16 below it
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      const int col = D / 4 * (c16 & 3) + 4 * u;
      const int at = ((KT * sub + r) * RC + ((col / 8) ^ v_swizzle(r))) * 16 +
                     (col % 8) * 2;
      const EV_LDS char* p = (const EV_LDS char*)buf[b][1] + at;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (EV_LDS i16x4*)p);
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (EV_LDS i16x4*)(p + 16 * RC * 16));
      const i16x4 both[2] = {lo, hi};
      va[u] = __builtin_bit_cast(bf16x8, both);
    }
  };
  auto add_v = [&](const bf16x8 (&va)[NT], const f32x4 (&x)[RT][NH]) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const f32x8 pf = __builtin_shufflevector(x[rt][0], x[rt][1], 0, 1, 2, 3,
                                               4, 5, 6, 7);
      const bf16x8 pb = __builtin_convertvector(pf, bf16x8);
#pragma unroll
      for (int u = 0; u < NT; ++u)
        rows.o[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            va[u], pb, rows.o[rt][u], 0, 0, 0);
    }
  };
  // The probabilities of the step before, and V's product with them, wait for
  // this step's logits: nothing then stands between the two products, and the
  // exponentials run beside the matrix cores. x: the logits of the step
  // before; va: its values.
  f32x4 x[RT][NH];
  bf16x8 va[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) va[u] = bf16x8{};
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[rt][h][i] = neg_inf();
  // 32 keys of a stage, whose K is in k; `next`: the step to read K of then
  auto step = [&](int stage, int b, int sub, int next) {
    f32x4 y[RT][NH];
    // (ahead of the other wavefront of its SIMD, which is at its softmax then)
    __builtin_amdgcn_s_setprio(2);
    rows.logits(y, k);
    rows.weigh(x, t);
    add_v(va, x);
    __builtin_amdgcn_s_setprio(0);
    read_v(va, b, sub);
    read_k(b, next);
    if (partial(stage)) {
      uint32_t vis[RT] = {};
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const int n = there(stage, NH * sub + h);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * g + i < n) vis[0] |= 1u << (4 * h + i);
      }
#pragma unroll
      for (int rt = 1; rt < RT; ++rt) vis[rt] = vis[0];
      rows.hide(y, vis);
    }
    rows.refer(y, t);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int h = 0; h < NH; ++h) x[rt][h] = y[rt][h];
  };
  static_assert(kWideKeys == 2 * KT, "two steps a stage");
  // The query rows are in registers before the first stage is sent for: the
  // compiler does not count those loads, and a wait of its own inside the loop
  // would be one for the next stage.
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int j = 0; j < P::KS; ++j) asm volatile("" : "+v"(rows.q[rt].x[j]));
  if (s0 < s1) {
    look(s0);
    fetch(s0, 0);
    if (s0 + 1 < s1) fetch(s0 + 1, 1);
    arrive(s0, 0, s0 + 1 < s1);
    for (int s = s0, b = 0; s < s1; ++s) {
      const int b1 = b == 2 ? 0 : b + 1, b2 = b1 == 2 ? 0 : b1 + 1;
      if (s + 2 < s1) fetch(s + 2, b2);
      if (works) {
        read_k(b, half);
        for (int sub = half; sub < 2; sub += halves) step(s, b, sub, sub | 1);
      }
      if (s + 1 < s1) arrive(s + 1, b1, s + 2 < s1);
      b = b1;
    }
  }
  rows.weigh(x, t);
  add_v(va, x);
  if (t.k_new && sh.run == sh.used - 1) {
    // the drafted tokens, one stage; every row has keys of its own
    const int64_t token = (int64_t)c.hkv * (D * P::ES);
    const int64_t base = (int64_t)tr.first * token + kvh * (D * P::ES);
    __syncthreads();   // the buffers are free
    if (tid == 0) odd = 0;
    __syncthreads();
    for (int u = tid; u < kWideKeys * RC; u += 64 * kWideWaves) {
      const int r = u / RC, ch = u % RC;
      const int64_t off = base + min(r, tr.n - 1) * token + 16 * ch;
      *(u32x4*)&buf[0][0][(r * RC + (ch ^ k_swizzle(r))) * 16] =
          *(const u32x4*)(t.k_new + off);
      u32x4 v = *(const u32x4*)(t.v_new + off);
      // A value that is not finite reaches the rows that see its token and no
      // other: it is left out of the product, whose zeros it would spoil, and
      // added by itself.
      bool fine = true;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if ((v[w] & 0x7F80u) == 0x7F80u) {
          v[w] &= 0xFFFF0000u;
          fine = false;
        }
        if ((v[w] & 0x7F800000u) == 0x7F800000u) {
          v[w] &= 0xFFFFu;
          fine = false;
        }
      }
      if (r >= tr.n) v = u32x4{};
      if (!fine && r < tr.n) odd = 1;
      *(u32x4*)&buf[0][1][(r * RC + (ch ^ v_swizzle(r))) * 16] = v;
    }
    __syncthreads();
    const bool plain = __builtin_amdgcn_readfirstlane(odd) == 0;
    if (works) {
      const uint64_t anc = ancestors(t, tr, lane);
      for (int sub = half; sub < 2 && KT * sub < tr.n; sub += halves) {
        uint32_t vis[RT], sees[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const int r = row0 + 16 * rt + c16;
          const uint64_t all = __shfl(anc, t.token_of(min(r, n_rows - 1)));
          sees[rt] = r < n_rows ? (uint32_t)(all >> (KT * sub)) : 0u;
          vis[rt] = 0;
#pragma unroll
          for (int h = 0; h < NH; ++h)
            vis[rt] |= (sees[rt] >> (16 * h + 4 * g) & 15u) << (4 * h);
        }
        read_k(0, sub);
        rows.logits(x, k);
        rows.hide(x, vis);
        rows.softmax(x, t);
        read_v(va, 0, sub);
        add_v(va, x);
        if (plain) continue;
        float* pr = probs[wave];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int h = 0; h < NH; ++h)
            *(f32x4*)(pr + (16 * rt + c16) * KT + 16 * h + 4 * g) = x[rt][h];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        for (int j = 0; j < KT && KT * sub + j < tr.n; ++j) {
          const char* v = t.v_new + base + (KT * sub + j) * token;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            if (!(sees[rt] >> j & 1)) continue;
            const float pj = pr[(16 * rt + c16) * KT + j];
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float e = P::element(v, D / 4 * g + 4 * u + i);
                if (!__builtin_isfinite(e)) rows.o[rt][u][i] += pj * e;
              }
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
  }
  if (!works) return;

  // every wavefront has its rows to itself: out, or its part of them
  const int used = sh.used * halves;
  const int64_t part =
      ((int64_t)(2 * (sh.slot + sh.run) + half) * c.hkv + kvh) * pl.padded;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float sum = row_sum(rows.l[rt]), big = rows.m[rt];
    const int r = row0 + 16 * rt + c16;
    if (r >= n_rows) continue;
    if (used > 1) {
      float* dst = t.pO + (part + r) * D + D / 4 * g;
#pragma unroll
      for (int u = 0; u < NT; ++u) *(f32x4*)(dst + 4 * u) = rows.o[rt][u];
      if (g == 0) {
        t.pM[part + r] = big;
        t.pL[part + r] = sum;
      }
      continue;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int tok = t.token_of(r), h = kvh * group + r - tok * group;
    char* dst = t.out + (((int64_t)(tr.first + tok) * t.hq + h) * D +
                         D / 4 * g) * P::ES;
#pragma unroll
    for (int u = 0; u < NT; u += 2) {
      const f32x8 y8 = __builtin_shufflevector(rows.o[rt][u] * inv,
                                               rows.o[rt][u + 1] * inv, 0, 1, 2,
                                               3, 4, 5, 6, 7);
      *(bf16x8*)(dst + 4 * u * P::ES) = __builtin_convertvector(y8, bf16x8);
    }
    if (g == 0) {
      if (t.lse)
        t.lse[(int64_t)h * t.n_tok + tr.first + tok] = t.lse_of(big, sum);
      if (t.accumulate) {
        t.row_m[(int64_t)unit * pl.padded + r] = big;
        t.row_inv[(int64_t)unit * pl.padded + r] = inv;
      }
    }
  }
}

// The join of row r over its sequence's splits, by a work-group: D / 4
// threads a split, the splits in turn over the groups of D / 4 threads (28 rows
// of 64 splits: 4.6 us, all of it latency; one wavefront a row 53 us).
template <class P, int D>
__device__ __forceinline__ void join_row(const CacheView& c,
                                         const TreePlan& pl, const TreeCall& t,
                                         int64_t row) {
  constexpr int kLanes = D / 4, kGroups = kThreads / kLanes;
  __shared__ __attribute__((aligned(16))) float part[kGroups][D];
  __shared__ float part_l[kGroups];
  const int padded = pl.padded;
  const int unit = (int)(row / pl.rows), r = (int)(row % pl.rows);
  const int kvh = unit % c.hkv, seq = unit / c.hkv;
  const Tree tr = tree_of(c, t, seq);
  const int group = t.hq / c.hkv;
  if (r >= tr.n * group) return;
  // A part of the row is `stride` behind the one before it. (wide: two a run,
  // of which the second is used where the keys are halved)
  const int halves =
      pl.wide ? key_halves(tr.n * group, r / kWideBlock * kWideBlock) : 1;
  const int slot = t.share[2 * seq], used = t.share[2 * seq + 1] * halves;
  if (used == 1) return;
  const int64_t stride = (int64_t)c.hkv * padded * (pl.wide ? 3 - halves : 1);
  const int64_t base =
      ((int64_t)slot * (pl.wide ? 2 : 1) * c.hkv + kvh) * padded + r;
  const int lane = threadIdx.x & 63;
  // every wavefront finds the largest reference for itself
  float big = neg_inf();
  static_assert(kMaxSplits <= 128, "two a lane");
#pragma unroll
  for (int u = 0; u < kMaxSplits / 64; ++u)
    if (lane + 64 * u < used)
      big = fmaxf(big, t.pM[base + (lane + 64 * u) * stride]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) big = fmaxf(big, __shfl_xor(big, o));
  const int e = 4 * (threadIdx.x % kLanes), gr = threadIdx.x / kLanes;
  float sum = 0.f;
  f32x4 x = {};
#pragma unroll 4
  for (int s = gr; s < used; s += kGroups) {
    const int64_t at = base + s * stride;
    const float m = t.pM[at], l = t.pL[at];
    const f32x4 o = *(const f32x4*)(t.pO + at * D + e);
    const float f = m == neg_inf() ? 0.f : exp2_(m - big);
    sum += f * l;
    x += f * o;
  }
  *(f32x4*)&part[gr][e] = x;
  if (e == 0) part_l[gr] = sum;
  __syncthreads();
  if (gr) return;
  x = f32x4{};
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    x += *(const f32x4*)&part[i][e];
    sum += part_l[i];
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  x *= inv;
  const int tok = t.token_of(r), h = kvh * group + r - tok * group;
  char* dst = t.out + (((int64_t)(tr.first + tok) * t.hq + h) * D + e) * P::ES;
  if constexpr (P::ES == 2)
    *(bf16x4*)dst = __builtin_convertvector(x, bf16x4);
  else
    *(f32x4*)dst = x;
  if (e) return;
  if (t.lse)
    t.lse[(int64_t)h * t.n_tok + tr.first + tok] = t.lse_of(big, sum);
  if (t.accumulate) {
    t.row_m[(int64_t)unit * padded + r] = big;
    t.row_inv[(int64_t)unit * padded + r] = inv;
  }
}

template <class P, int D>
__global__ __launch_bounds__(kThreads) void join_kernel(const CacheView c,
                                                        const TreePlan pl,
                                                        const TreeCall t) {
  join_row<P, D>(c, pl, t, blockIdx.x);
}

// Few rows (16 at most): their logits were stored, four keys a thread here.
// The same launch joins the rows; the weights' work-groups take the rows'
// sums from the splits themselves. 64 sequences of up to 8,000 tokens: 19 us for
// 29 MB of logits and 16 MB of weights.
constexpr int kStoredRows = 16;
template <class P, int D>
__global__ __launch_bounds__(kThreads) void mass_stored_kernel(
    const CacheView c, const TreePlan pl, const TreeCall t, int join_blocks,
    int key_blocks) {
  if ((int)blockIdx.x < join_blocks) {
    join_row<P, D>(c, pl, t, blockIdx.x);
    return;
  }
  __shared__ float row_m[kStoredRows], coef[kStoredRows];
  const int b = blockIdx.x - join_blocks;
  const int unit = b / key_blocks, kb = b % key_blocks;
  const int kvh = unit % c.hkv, seq = unit / c.hkv;
  const Tree tr = tree_of(c, t, seq);
  const int64_t key0 = (int64_t)kb * kThreads * 4;
  if (tr.n == 0 || (key0 >= tr.len && kb > 0)) return;
  const int group = t.hq / c.hkv, n_rows = tr.n * group;
  const int slot = pl.joined ? t.share[2 * seq] : 0;
  const int used = pl.joined ? t.share[2 * seq + 1] : 1;
  const int tid = threadIdx.x;
  const int64_t key = key0 + 4 * tid;
  const int padded = pl.padded;
  // sixteen threads a row
  {
    const int r = tid / 16, l16 = tid % 16;
    float m = neg_inf(), cf = 0.f;
    if (r < n_rows) {
      if (used == 1) {
        m = t.row_m[(int64_t)unit * padded + r];
        cf = t.row_inv[(int64_t)unit * padded + r];
      } else {
        const int64_t stride = (int64_t)c.hkv * padded;
        const int64_t base = ((int64_t)slot * c.hkv + kvh) * padded + r;
        float pm[kMaxSplits / 16], sum = 0.f;
#pragma unroll
        for (int u = 0; u < kMaxSplits / 16; ++u) {
          const int s = l16 + 16 * u;
          pm[u] = s < used ? t.pM[base + s * stride] : neg_inf();
          m = fmaxf(m, pm[u]);
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
#pragma unroll
        for (int u = 0; u < kMaxSplits / 16; ++u) {
          const int s = l16 + 16 * u;
          if (s < used)
            sum += (pm[u] == neg_inf() ? 0.f : exp2_(pm[u] - m)) *
                   t.pL[base + s * stride];
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) sum += __shfl_xor(sum, o);
        cf = sum == 0.f ? 0.f : 1.f / sum;
      }
      const float vote = t.vote ? t.vote[tr.first + t.token_of(r)] : 1.f;
      // (a vote of 0 keeps the row out, whatever it holds)
      cf = vote == 0.f ? 0.f : cf * vote;
    }
    if (l16 == 0) {
      row_m[r] = m;
      coef[r] = cf;
    }
  }
  __syncthreads();
  const float* score =
      t.score + (int64_t)unit * pl.rows * (pl.len_pad + kMaxTree);
  auto sum = [&](int64_t at) {
    f32x4 x[kStoredRows], acc = {};
#pragma unroll
    for (int r = 0; r < kStoredRows; ++r)
      if (r < n_rows)
        x[r] = *(const f32x4*)(score + r * (pl.len_pad + kMaxTree) + at);
#pragma unroll
    for (int r = 0; r < kStoredRows; ++r)
      if (r < n_rows && coef[r] != 0.f)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc[i] += coef[r] * t.exp_of(x[r][i], row_m[r]);
    return acc;
  };
  if (key < tr.len) {
    const f32x4 m = sum(key);
    float* w = c.weight + (int64_t)unit * c.cap + key;
    if (key + 4 <= tr.len) {
      *(f32x4*)w = t.decay * *(const f32x4*)w + m;
    } else {
      for (int i = 0; key + i < tr.len; ++i) w[i] = t.decay * w[i] + m[i];
    }
  }
  if (kb == 0 && t.w_new && 4 * tid < tr.n) {
    const f32x4 m = t.k_new ? sum(pl.len_pad + 4 * tid) : f32x4{};
    for (int i = 0; i < 4 && 4 * tid + i < tr.n; ++i)
      t.w_new[(int64_t)(tr.first + 4 * tid + i) * c.hkv + kvh] = m[i];
  }
}

// Many rows: the logits are formed again, 16 NK keys a wavefront, whose rows
// stay in registers while the query rows pass by in LDS, 128 at a time. Trees of
// up to 26 tokens over 8 x 16,512: 32 us (41 with 64 keys a wavefront, which
// leaves three wavefronts a SIMD and not four).
constexpr int kMassHalves = 2;
constexpr int kMassRows = 128;

template <class P, int D>
__global__ __launch_bounds__(kThreads, P::ES == 2 ? 4 : 2) void mass_kernel(
    const CacheView c, const TreePlan pl, const TreeCall t, int key_blocks) {
  constexpr int NK = kMassHalves, TK = 16 * NK;
  constexpr int RC = D * P::ES / 16;   // 16-byte chunks of a row
  __shared__ __attribute__((aligned(16))) char qs[kMassRows * D * P::ES];
  __shared__ float ref[kMassRows], coef[kMassRows];
  const int unit = blockIdx.x / key_blocks, kb = blockIdx.x % key_blocks;
  const int kvh = unit % c.hkv, seq = unit / c.hkv;
  const Tree tr = tree_of(c, t, seq);
  if (tr.n == 0) return;
  const int group = t.hq / c.hkv, n_rows = tr.n * group;
  constexpr int kWaves = kThreads / 64;
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cached = (tr.len + TK - 1) / TK;
  const int drafts = t.w_new ? (tr.n + TK - 1) / TK : 0;
  if (kb * kWaves >= cached + drafts) return;
  const int tile = kb * kWaves + wave;
  const bool draft = tile >= cached, works = tile < cached + drafts;
  const int j0 = (tile - cached) * TK;
  typename P::Row k[NK];
  int n[NK];
  uint64_t anc = 0;
  if (!draft) {
    Where<NK> at;
    find<NK>(at, c, seq, kvh * c.head_bytes, tr.len, tile * TK);
#pragma unroll
    for (int h = 0; h < NK; ++h) {
      P::load_row(k[h], c.k + at.off[h] + (uint32_t)c16 * c.token_bytes + 16 * g);
      n[h] = at.n[h];
    }
  } else {
    anc = ancestors(t, tr, lane);
    const int64_t step = (int64_t)c.hkv * (D * P::ES);
#pragma unroll
    for (int h = 0; h < NK; ++h) {
      n[h] = min(max(tr.n - j0 - 16 * h, 0), 16);
      const int j = min(j0 + 16 * h + c16, tr.n - 1);
      if (t.k_new)
        P::load_row(k[h], t.k_new + (tr.first + j) * step + kvh * (D * P::ES) +
                              16 * g);
      else {
        P::zero_row(k[h]);
        n[h] = 0;
      }
    }
  }
  // keys of the lane that are there: bit 4h + i
  uint32_t mine = 0;
#pragma unroll
  for (int h = 0; h < NK; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * g + i < n[h]) mine |= 1u << (4 * h + i);
  bool full = !draft;   // every row sees every key
#pragma unroll
  for (int h = 0; h < NK; ++h) full = full && n[h] == 16;
  f32x4 acc[NK] = {};
  // 16 query rows, from row r of the 128
  auto take = [&](int r0, int r, auto all) {
    typename P::Row q;
    const int row = r + c16;
#pragma unroll
    for (int j = 0; j < P::KS; ++j)
      __builtin_memcpy(&q.x[j],
                       &qs[(row * RC + ((g + 4 * j) ^ (row & (RC >= 16 ? 15 : 7)))) * 16],
                       16);
    const float m = ref[row], cf = coef[row];
    uint32_t see = mine;
    if (!decltype(all)::value && draft) {
      const uint64_t sees =
          __shfl(anc, t.token_of(min(r0 + row, n_rows - 1))) >> j0;
      see = 0;
#pragma unroll
      for (int h = 0; h < NK; ++h)
        see |= ((uint32_t)(sees >> (16 * h + 4 * g)) & 15u) << (4 * h);
      see &= mine;
    }
    // a row without weight: its logits may be anything
    const bool counts = cf != 0.f;
#pragma unroll
    for (int h = 0; h < NK; ++h) {
      const f32x4 s = P::qk(k[h], q);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = t.exp_of(s[i], m);
        const bool add =
            counts && (decltype(all)::value || (see >> (4 * h + i) & 1));
        acc[h][i] = __builtin_fmaf(cf, add ? p : 0.f, acc[h][i]);
      }
    }
  };
  for (int r0 = 0; r0 < n_rows; r0 += kMassRows) {
    const int rows = min(kMassRows, n_rows - r0), up = (rows + 15) & ~15;
    if (r0) __syncthreads();
    for (int u = tid; u < up * RC; u += kThreads) {
      const int row = u / RC, ch = u % RC;
      const int r = r0 + min(row, rows - 1), tok = t.token_of(r);
      *(u32x4*)&qs[(row * RC + (ch ^ (row & (RC >= 16 ? 15 : 7)))) * 16] =
          *(const u32x4*)(t.q + ((int64_t)(tr.first + tok) * t.hq +
                                 kvh * group + r - tok * group) *
                                    (D * P::ES) + 16 * ch);
    }
    if (tid < up) {
      const int r = r0 + min(tid, rows - 1);
      const float inv = t.row_inv[(int64_t)unit * pl.padded + r];
      const float vote = t.vote ? t.vote[tr.first + t.token_of(r)] : 1.f;
      ref[tid] = t.row_m[(int64_t)unit * pl.padded + r];
      // (a vote of 0 keeps the row out, whatever it holds)
      coef[tid] = vote == 0.f || tid >= rows ? 0.f : inv * vote;
    }
    __syncthreads();
    if (!works) continue;
    if (full)
      for (int r = 0; r < up; r += 16) take(r0, r, Yes{});
    else
      for (int r = 0; r < up; r += 16) take(r0, r, No{});
  }
  if (!works) return;
  // The sums over the 16 lanes of a key, each lane left with those of its own
  // keys: at every step it passes on the half that is not.
  constexpr int N = 4 * NK;
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = acc[i / 4][i % 4];
#pragma unroll
  for (int o = 8, m = N / 2; o >= 1; o /= 2, m /= 2) {
    const bool up = c16 & o;
    if (m >= 1) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        if (i >= m) continue;
        const float give = up ? v[i] : v[i + m];
        v[i] = (up ? v[i + m] : v[i]) + __shfl_xor(give, o);
      }
    } else {
      v[0] += __shfl_xor(v[0], o);
    }
  }
  constexpr int kShare = 16 / N;   // lanes that hold the same sum
  if (c16 % kShare) return;
  const int e = c16 / kShare;      // 4h + i
  const int at = 16 * (e / 4) + 4 * g + e % 4;
  if (!draft) {
    const int key = tile * TK + at;
    if (key >= tr.len) return;
    float* w = c.weight + (int64_t)unit * c.cap + key;
    *w = t.decay * *w + v[0];
  } else if (j0 + at < tr.n) {
    t.w_new[(int64_t)(tr.first + j0 + at) * c.hkv + kvh] = v[0];
  }
}

template <class P, int D>
hipError_t launch_tree(const CacheView& c, const TreePlan& pl,
                       const TreeCall& t, hipStream_t s) {
  const int64_t units = (int64_t)pl.groups * c.hkv;
  const int64_t blocks = (units + 7) / 8 * 8 * pl.row_blocks;
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kThreads);
  const dim3 waves(64 * waves_of(pl.row_tiles));
  if (pl.wide) {
    if constexpr (P::ES == 2)
      tree_wide_kernel<P, D><<<grid, dim3(64 * kWideWaves), 0, s>>>(c, pl, t);
  } else if (pl.stored)
    tree_kernel<P, D, 1, true><<<grid, waves, 0, s>>>(c, pl, t);
  else if (pl.row_tiles == 1)
    tree_kernel<P, D, 1, false><<<grid, waves, 0, s>>>(c, pl, t);
  else if (pl.row_tiles == 2)
    tree_kernel<P, D, 2, false><<<grid, waves, 0, s>>>(c, pl, t);
  else if constexpr (P::ES == 2)
    tree_kernel<P, D, 4, false><<<grid, waves, 0, s>>>(c, pl, t);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t join =
      pl.joined ? (int64_t)c.n_seq * c.hkv * pl.rows : 0;
  if (pl.stored) {
    const int kb = std::max(1, (t.max_len + 4 * kThreads - 1) / (4 * kThreads));
    const int64_t n = join + (int64_t)c.n_seq * c.hkv * kb;
    if (n > 0x7FFFFFFF) return hipErrorInvalidValue;
    mass_stored_kernel<P, D><<<dim3((unsigned)n), block, 0, s>>>(
        c, pl, t, (int)join, kb);
    return hipGetLastError();
  }
  if (join) {
    if (join > 0x7FFFFFFF) return hipErrorInvalidValue;
    join_kernel<P, D><<<dim3((unsigned)join), block, 0, s>>>(c, pl, t);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (t.accumulate) {
    constexpr int TK = 16 * kMassHalves;
    const int tiles = (t.max_len + TK - 1) / TK + (t.max_tree + TK - 1) / TK;
    const int kb = (tiles + kThreads / 64 - 1) / (kThreads / 64);
    const int64_t n = (int64_t)c.n_seq * c.hkv * kb;
    if (n > 0x7FFFFFFF) return hipErrorInvalidValue;
    mass_kernel<P, D><<<dim3((unsigned)n), block, 0, s>>>(c, pl, t, kb);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace

TreePlan plan_tree(const CacheView& c, int32_t hq, int32_t max_tree,
                   int32_t max_len, int32_t accumulate) {
  TreePlan p{};
  p.rows = hq / c.hkv * max_tree;
  p.row_tiles = p.rows <= 16 ? 1 : p.rows <= 32 || c.fp32 ? 2 : 4;
  p.wide = !c.fp32 && p.rows > 64;
  const int kt = p.wide ? kWideKeys : c.fp32 ? 16 : 32;
  const int block = p.wide ? kWideBlock : 16 * p.row_tiles;
  p.row_blocks = (p.rows + block - 1) / block;
  p.padded = p.row_blocks * block;
  const int64_t tiles =
      ((int64_t)max_len + kt - 1) / kt + (max_tree + kt - 1) / kt;
  const int64_t units = (int64_t)c.n_seq * c.hkv * p.row_blocks;
  int64_t splits = 1;
  p.groups = c.n_seq;
  if (p.wide) {
    // A work-group takes a CU, and four stages at least: one round of them
    // (the row blocks of a run are on one XCD, which has 32 CUs). Even runs
    // left CUs idle behind the longest of eight sequences of 1,100 to 16,512
    // tokens: 70 us, 56 with fair ones.
    p.least = 4;
    p.most_runs = kMaxSplits / 2;
    p.goal = (int32_t)std::max<int64_t>(
        1, std::max(1, 32 / p.row_blocks) * 8 / c.hkv);
    p.balanced = tiles > p.least && c.n_seq <= kMaxBalanced &&
                 tiles * c.n_seq < 1 << 30;
    if (p.balanced)
      p.groups = p.goal + c.n_seq;
    else
      splits = std::min<int64_t>({256 / units, tiles / p.least, p.most_runs});
  } else {
    // Work-groups for the 256 CUs, as far as every wavefront gets a tile; more
    // of them, up to eight for each CU so that sequences of unlike lengths
    // even out, while each keeps 32 tiles. Up to five rounds of tiles a
    // work-group takes less than it and the second launch (one token over 544:
    // 9.6 us, 10.2 with five splits; over 2,000: 22, 11.8 with eight). 28 / 4
    // heads: 64 sequences of up to 8,000 tokens take 131 us with 8 splits, 138
    // with 4, 163 with one; eight with trees of 8 25 us with 8 splits, 31 with
    // 16; 16 heads of their own, 16 sequences of up to 4,000: 61 us with 4
    // splits, 72 with 8, 73 with 1. Runs of one length for all sequences were
    // slower here (64 of up to 8,000: 140), as their work-groups start and end
    // together.
    const int w = waves_of(p.row_tiles);
    if (tiles > 5 * w) {
      splits = std::min<int64_t>(256 / units, (tiles + w - 1) / w);
      splits = std::max(splits,
                        std::min<int64_t>(2048 / units, (tiles + 31) / 32));
      splits = std::min<int64_t>(kMaxSplits, splits);
    }
  }
  p.splits = (int32_t)std::max<int64_t>(1, splits);
  if (!p.balanced) p.groups = c.n_seq * p.splits;
  p.joined = p.wide || p.groups > c.n_seq;
  // Few rows' logits pass through the workspace (one token of 28 / 4 heads: 56
  // bytes a key there and back, 256 for K again), unless a loose bound on the
  // lengths would make that more than 1 GiB.
  p.len_pad = ((int64_t)max_len + 31) / 32 * 32;
  const size_t scores = (size_t)c.n_seq * c.hkv * p.rows *
                        (p.len_pad + kMaxTree) * 4;
  p.stored = accumulate && p.rows <= kStoredRows && scores <= size_t(1) << 30;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 255) & ~size_t(255);
    return at;
  };
  const size_t all = (size_t)c.n_seq * c.hkv * p.padded;   // rows
  const size_t part =
      p.joined ? (size_t)p.groups * (p.wide ? 2 : 1) * c.hkv * p.padded : 0;
  p.pO = take(part * c.d * 4);
  p.pM = take(part * 4);
  p.pL = take(part * 4);
  p.share = take(p.joined ? (size_t)c.n_seq * 8 : 0);
  p.row_m = take(accumulate ? all * 4 : 0);
  p.row_inv = take(accumulate ? all * 4 : 0);
  p.score = take(p.stored ? scores : 0);
  p.total = off;
  return p;
}

hipError_t launch_tree_attention(const CacheView& c, const TreePlan& p,
                                 const TreeCall& t, hipStream_t s) {
  if (c.fp32)
    return c.d == 64 ? launch_tree<TreeF32<64>, 64>(c, p, t, s)
                     : launch_tree<TreeF32<128>, 128>(c, p, t, s);
  return c.d == 64 ? launch_tree<TreeBf16<64>, 64>(c, p, t, s)
                   : launch_tree<TreeBf16<128>, 128>(c, p, t, s);
}

}  // namespace evisel
