// Decode attention over the paged bf16 cache where a sequence's context is not read as a whole by itself: a window of the last
// positions and a few first ones, and groups of sequences that begin with the same pages.
//
// Both are streams of K and V at a few flops per byte, as the ragged decode attention is, over the same pages: runs of 32 tokens whose
// fragments a wavefront loads as whole KiB in operand order.  Scores are taken in fp32, with one running maximum and sum per wavefront
// and column; weights are rounded to bf16 for the second product (half a step of 2^-8 each, as V is held), sums and statistics are fp32.
#include "attn_math.h"
#include "attn_worklist.h"
#include "pl_common.h"

#include <algorithm>

namespace pl {
namespace {

typedef __attribute__((address_space(4))) int32_t scalar_i32;   // read by scalar loads
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int ITEM_INTS = 8;   // of a work item's record: {kind, row or first of the rows, chunk, context or shared runs, first run or rows, row whose pages are read, shared runs of a chunk}
                               // (with the ids of its first pages the list takes 1.7 us longer, and the items' first loads hide all of it: calls 2 us longer)
constexpr int HEAD_INTS = 64;
constexpr int64_t MOST_ITEMS = 1 << 30;   // a workgroup's next item stays below 2^31
enum { ITEM_OWN, ITEM_SHARED };

struct Parts {
  float *o, *ml;           // of row b, kv head g, chunk c: element ((b Hkv + g) max_chunks + c) of [G, HD] and of [ATTN_ML]
  int32_t max_chunks;
};
// How a group's shared runs are cut, by their number: into as many chunks as make 256 workgroups, 384 from from[0] runs on, 512 from from[1] on, but into fewer, of about own_runs, where
// rows' own parts keep the chip busy meanwhile.  Quotients by a reciprocal are put right, and no more than a step off: they are 512 at most.  (One workgroup does this while its
// first loads are under way; by four divisions it takes 0.8 us longer.)
struct SharedCut {
  Divisor by[3];
  int32_t from[2], own_runs;
  __device__ static int up4(int a) { return (a + 3) & ~3; }
  __device__ int chunk(int runs, int &chunks) const {
    // (the three read ahead of the choice: a choice between their places would be read behind it)
    const uint32_t m0 = __builtin_amdgcn_readfirstlane(by[0].m), m1 = __builtin_amdgcn_readfirstlane(by[1].m), m2 = __builtin_amdgcn_readfirstlane(by[2].m);
    const uint32_t s0 = __builtin_amdgcn_readfirstlane(by[0].shift), s1 = __builtin_amdgcn_readfirstlane(by[1].shift), s2 = __builtin_amdgcn_readfirstlane(by[2].shift);
    Divisor d;
    d.m = runs >= from[1] ? m2 : runs >= from[0] ? m1 : m0;
    d.shift = runs >= from[1] ? s2 : runs >= from[0] ? s1 : s0;
    const int even = d.of(runs - 1);   // (runs of an even cut, and one more)
    int c = max(up4(even + 1), up4((int)(__builtin_amdgcn_sqrtf(0.5f * (float)runs) + 0.99f)));   // (squared half of the runs at least, as for windows; 8 rollouts of one prompt of 16384, 7B shape, 33 -> 30 us)
    c = min(max(c, max(8, own_runs)), up4(runs));
    chunks = (int)((float)runs * __builtin_amdgcn_rcpf((float)c));
    chunks += chunks * (int64_t)c < runs ? 1 : (chunks - 1) * (int64_t)c >= runs ? -1 : 0;
    const int same = up4((int)((float)runs * __builtin_amdgcn_rcpf((float)chunks) + 0.99f));   // chunks of one length
    return same < c && (int64_t)same * chunks >= runs ? same : c;
  }
};
struct SharedWork {
  int32_t *head;                   // the number of items; behind it
  int32_t *items, *rows;           // records; rows that share, group by group
  int2 *start;                     // of every row: first run of its own part, shared parts before it
  Parts own, shared;
  int32_t own_runs;                // of a chunk
  SharedCut cut;
  int32_t tile_rows, cap;
};

template <int HD, int WAVES = 4>
struct Fold {   // wavefronts' results on their way into one
  float o[WAVES][16][HD + 4];   // (the columns of a store start at banks of their own)
  float m[WAVES][16], l[WAVES][16];
};
constexpr int RING = 4;   // runs that a workgroup's wavefronts share through LDS: one is computed with while three are on their way
template <int HD>
struct Pair {   // two wavefronts' results of 32 columns each on their way into two others'
  float o[2][32][HD + 4], ml[2][32][2];
};
template <int HD>
union Lds {               // (one object: with two, every read waits for the loads that are on their way to the other)
  Fold<HD> fold;
  Pair<HD> pair;
  bf16_t ring[RING][64 * HD];   // K, then V
};
typedef __attribute__((address_space(3))) void lds_void;

// Maxima are scores as the products leave them, and what is scaled is a difference of two of them, so that the largest weight is 1 whatever the scores are.  (Taken away from
// a score's power of two, a maximum's, which is rounded to 32 bits, leaves half a step of it: more than 1 from 2^24 on, more than a weight can hold from 2^31 on.)
// (m, l, o) <- (m, l, o) folded with a later part (mi, li, oi), the first part taken over as it is; a part without tokens has mi = -inf and changes nothing.
__device__ inline void score_factors(float m, float mi, float scale, float &M, float &e0, float &e1) {
  M = fmaxf(m, mi);
  e0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - M) * scale);
  e1 = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mi - M) * scale);
}
template <int HD>
__device__ inline float score_scale() { return 1.4426950408889634f / sqrtf((float)HD); }   // log2(e) / sqrt(hd)

// Which positions of its context a row sees: those below `first` and those from `from` on.  Runs are counted without the hidden ones between.
struct Sight {
  int ctx, first, from, head_runs, tail_run, runs;
  __device__ Sight(int ctx_, int window, int sinks) : ctx(ctx_) {
    first = min(sinks, ctx);
    from = ctx > window ? ctx - window : 0;
    head_runs = (first + 31) >> 5;
    tail_run = from >> 5;
    if (head_runs >= tail_run) head_runs = tail_run = 0;   // nothing, or less than a run, is hidden between
    runs = head_runs + ((ctx + 31) >> 5) - tail_run;
  }
  __device__ Sight(int ctx_, int start_run) : ctx(ctx_), first(0), from(start_run * 32), head_runs(0), tail_run(start_run), runs(((ctx_ + 31) >> 5) - start_run) {}
  __device__ int run(int v) const { return v < head_runs ? v : v - head_runs + tail_run; }
  __device__ bool whole(int run) const { return run * 32 + 32 <= ctx && (run * 32 >= from || run * 32 + 32 <= first); }
  __device__ bool sees(int t) const { return t < ctx && (t < first || t >= from); }
};

// Runs [v0, v1) of one row and kv head, dealt to WAVES wavefronts; the heads of the group are the columns of 16 x 16 x 32
// products.  put(i, head, quad of dims, m, l, o): the result, four elements of a head per thread.
template <int HD, int WAVES, typename F>
__device__ __forceinline__ void attend_runs(const RangeAttn &p, Fold<HD, WAVES> &sm, int b, int g, const scalar_i32 *pages, const Sight &see, int v0, int v1, F put) {
  constexpr int NS = HD == 128 ? 2 : 4, NJ = HD / 32, NV = HD / 16;   // register stages of K and V; products of a tile of scores, of a run
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, head = l & 15, qg = l >> 4, G = p.Hq / p.Hkv;
  const float scale = score_scale<HD>();
  const int64_t page_elems = (int64_t)2 * p.page_tokens * HD;
  const int n = v1 - v0, per_page = p.page_tokens >> 5;
  bf16x8 qf[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    qf[j] = bf16x8{};
    if (head < G) qf[j] = *(const bf16x8 *)(p.q + ((int64_t)b * p.Hq + g * G + head) * HD + j * 32 + qg * 8);
  }
  f32x4 o[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, lsum = 0.f;   // the largest score
  bf16x8 kf[NS][2][NJ], vf[NS][NV];
  auto run_base = [&](int run, int page) { return p.kv + ((int64_t)page * p.Hkv + g) * page_elems + (int64_t)(run % per_page) * 32 * HD + l * 8; };
  auto load_k = [&](int st, const bf16_t *kb) {
#pragma unroll
    for (int T = 0; T < 2; ++T)
#pragma unroll
      for (int j = 0; j < NJ; ++j) kf[st][T][j] = __builtin_nontemporal_load((const bf16x8 *)(kb + (T * NJ + j) * 512));
  };
  auto load_v = [&](int st, const bf16_t *kb) {
    const bf16_t *vb = kb + (int64_t)p.page_tokens * HD;
#pragma unroll
    for (int i = 0; i < NV; ++i) vf[st][i] = __builtin_nontemporal_load((const bf16x8 *)(vb + i * 512));
  };
  int page_next[NS];   // page of the run a stage takes after the one it holds
#pragma unroll
  for (int st = 0; st < NS; ++st) {
    const int v = wave + WAVES * st;
    if (v < n) {
      const int run = see.run(v0 + v);
      const bf16_t *kb = run_base(run, pages[run / per_page]);
      load_k(st, kb);
      load_v(st, kb);
    }
    page_next[st] = v + WAVES * NS < n ? pages[see.run(v0 + v + WAVES * NS) / per_page] : 0;
  }
  for (int base = wave; base < n; base += WAVES * NS) {
#pragma unroll
    for (int st = 0; st < NS; ++st) {
      const int v = base + WAVES * st;
      if (v >= n) continue;
      f32x4 s4[2];
#pragma unroll
      for (int T = 0; T < 2; ++T) {
        s4[T] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NJ; ++j) s4[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[st][T][j], qf[j], s4[T], 0, 0, 0);
      }
      const int run = see.run(v0 + v), nxt = v + WAVES * NS;
      const bf16_t *nb = nullptr;
      if (nxt < n) {
        nb = run_base(see.run(v0 + nxt), page_next[st]);
        load_k(st, nb);
        page_next[st] = nxt + WAVES * NS < n ? pages[see.run(v0 + nxt + WAVES * NS) / per_page] : 0;
      }
      float s[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = s4[e >> 2][e & 3];
      if (!see.whole(run)) {
        // hidden positions: no score, and zeros for V, whatever the page holds there
        uint32_t keep[4];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool in = see.sees(run * 32 + qg * 8 + e);
          s[e] = in ? s[e] : -INFINITY;
          keep[e / 2] = (e & 1 ? keep[e / 2] : 0) | (in ? 0xFFFFu << (e & 1) * 16 : 0);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) vf[st][i] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, vf[st][i]) & u32x4{keep[0], keep[1], keep[2], keep[3]});
      }
      const float top = fmaxf(m, run_max(s)), ref = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f((m - ref) * scale);
      float psum = 0.f;
      bf16x8 pf;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = __builtin_amdgcn_exp2f((s[e] - ref) * scale);
        psum += w;
        pf[e] = (__bf16)w;
      }
      lsum = __builtin_fmaf(lsum, alpha, psum);
      m = top;
      if (__builtin_amdgcn_ballot_w64(!(alpha == 1.f))) {   // a maximum has moved (a factor of 1 changes nothing)
#pragma unroll
        for (int i = 0; i < NV; ++i) o[i] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[st][i], pf, o[i], 0, 0, 0);
      if (nb) load_v(st, nb);
    }
  }
  lsum = column_sum(lsum);
#pragma unroll
  for (int i = 0; i < NV; ++i) *(f32x4 *)&sm.o[wave][head][i * 16 + qg * 4] = o[i];
  if (qg == 0) { sm.m[wave][head] = m; sm.l[wave][head] = lsum; }
  __syncthreads();
  for (int i = threadIdx.x; i < G * (HD / 4); i += WAVES * 64) {
    const int h = i / (HD / 4), d = i % (HD / 4) * 4;
    float M = sm.m[0][h];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sm.m[w][h]);
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f((sm.m[w][h] - ref) * scale);
      L = __builtin_fmaf(sm.l[w][h], f, L);
      O = fma4(*(const f32x4 *)&sm.o[w][h][d], f, O);
    }
    put(i, h, d, M, L, O);
  }
}

// An item's result: the row itself, or a part of it for the merge.
template <int HD, int WAVES>
__device__ __forceinline__ void attend_item(const RangeAttn &p, Fold<HD, WAVES> &sm, const Parts &parts, int b, int g, const scalar_i32 *pages, const Sight &see, int c,
                                            int chunk_runs, bool alone) {
  const int G = p.Hq / p.Hkv;
  const int64_t part = ((int64_t)b * p.Hkv + g) * parts.max_chunks + c;
  attend_runs<HD, WAVES>(p, sm, b, g, pages, see, c * chunk_runs, min(see.runs, (c + 1) * chunk_runs), [&](int i, int h, int d, float M, float L, f32x4 O) {
    if (alone) {
      *(bf16x4 *)(p.out + ((int64_t)b * p.Hq + g * G) * HD + i * 4) = finish(O, L);
    } else {
      *(f32x4 *)(parts.o + part * G * HD + i * 4) = O;
      if (d == 0) *(float2 *)(parts.ml + part * ATTN_ML + h * 2) = make_float2(M, L);
    }
  });
}

// Windowed attention: workgroup (row, chunk, kv head).  Windows are of one length, so no list balances them: a chunk is a share of
// the longest sight.  Bound by the bytes of the keys and values that rows see (256 rows, 7B shape, window 4096 and 4 sinks, 1866 MB: 285 to 302 us, 6.2 to 6.5 TB/s,
// where a stream that only reads reaches 7.0).
template <int HD, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void attn_window_kernel(RangeAttn p, Parts parts, int window, int sinks, int chunk_runs) {
  __shared__ __attribute__((aligned(16))) Fold<HD, WAVES> sm;
  // (first chunks first: later ones are empty in rows that see little, and all XCDs get some of both)
  const int g = blockIdx.x % p.Hkv, item = blockIdx.x / p.Hkv, c = item / p.n_seq, b = item - c * p.n_seq;
  const int ctx = min(p.ctx_len[b], p.max_ctx);
  if (ctx <= 0) return;
  const Sight see(ctx, window, sinks);
  if (c * chunk_runs >= see.runs) return;
  const scalar_i32 *pages = (const scalar_i32 *)(p.page_table + (int64_t)b * p.pages_per_seq);
  attend_item<HD, WAVES>(p, sm, parts, b, g, pages, see, c, chunk_runs, see.runs <= chunk_runs);
}

// A block of 32 columns of one wavefront over runs that all of them see whole: 32 x 32 x 16 products, no masks.  A lane has one column's 16 scores of a
// run, in the order in which the second product takes weights.
template <int HD>
struct Block {
  static constexpr int NJ = HD / 16, ND = HD / 32;
  bf16x8 qf[NJ];
  f32x16 o[ND];
  float m, off, lsum;   // the score that weights are relative to; its power of two, or 0 where scores have it taken away; the sum of the lane's weights
  bool far;             // whether they have: a power of two of the wavefront's is 2^10 at least

  __device__ __forceinline__ void begin(const bf16_t *q, bool mine) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      qf[j] = bf16x8{};
      if (mine) qf[j] = *(const bf16x8 *)(q + j * 16);
    }
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    m = -INFINITY;
    off = lsum = 0.f;
    far = false;
  }
  // where a lane's fragments of a run are, behind its K and its V block's beginning
  __device__ static int in_k(int l) { return ((l & 16) / 16 * (HD / 8) + l / 32) * 128 + (l & 15) * 8; }   // + j * 256
  __device__ static int in_v(int l) { return ((l & 16) / 16 * 4 + l / 32) * 128 + (l & 15) * 8; }           // + i * 1024 + half of the tokens * 256
  __device__ __forceinline__ f32x16 scores(const bf16x8 (&kf)[NJ]) const {
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j], qf[j], s, 0, 0, 0);
    return s;
  }
  // What the weights of a run are relative to, and the factor of the sum so far.  The reference stays while no score is more than 2^8 above it (weights of up to 256 lose
  // nothing, in bf16 as in the sums): a maximum of 32 columns moves in nearly every run of a chunk, and the results' way through the vector unit is a
  // quarter of its time (64 rows of 5 heads over 16384 positions, 8 kv heads, this kernel alone: 44 -> 41 us).
  // A weight is one fused operation and its power, relative to a power of two that was rounded by 2^-14 at most: next to nothing of a weight's own rounding.
  // Larger ones would be rounded by more, in the end by more than a weight holds: there the maximum is taken away from the scores first.
  __device__ __forceinline__ float peak(f32x16 &s, float scale) {
    float top = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
    top = with_xor32(top, OpMax{});
    float alpha = 1.f;
    const bool moves = top > m + 8.f / scale;   // (the first run's: from -infinity)
    if (__builtin_amdgcn_ballot_w64(moves)) {
      const float to = moves ? top : m;
      alpha = moves ? __builtin_amdgcn_exp2f((m - to) * scale) : 1.f;
      m = to;
      off = m == -INFINITY ? 0.f : m * scale;
      far = __builtin_amdgcn_ballot_w64(!(fabsf(off) < 1024.f));
      if (far) off = 0.f;
#pragma unroll
      for (int i = 0; i < ND; ++i) o[i] *= alpha;
    }
    if (far) {
      const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] -= from;
    }
    return alpha;
  }
  __device__ __forceinline__ void weigh(const f32x16 &s, float scale, float alpha, bf16x8 (&pf)[2]) {
    float psum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {   // element e: token 16 (e / 4 % 2) + 8 (lane / 32) + 4 (e / 8) + e % 4 of the run
      const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], scale, -off));
      psum += w;
      pf[e / 4 % 2][e / 8 * 4 + e % 4] = (__bf16)w;
    }
    lsum = __builtin_fmaf(lsum, alpha, psum);
  }
  __device__ __forceinline__ void add(const bf16x8 (&vf)[ND][2], const bf16x8 (&pf)[2]) {
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int q = 0; q < 2; ++q) o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i][q], pf[q], o[i], 0, 0, 0);
  }
  // four elements of the lane's column, from dim i * 32 + e * 2 + (lane / 32) * 4 on
  __device__ __forceinline__ f32x4 four(int i, int e) const { return f32x4{o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]}; }
};

// Runs [r0, r1) that `nrows` rows share, for one kv head: the heads of all rows are columns.
// More than 64 columns: every wavefront has a block of 32 and needs every run, so runs go through LDS, by direct loads three runs ahead, one barrier a run.
// Fewer: the wavefronts of a block take turns at the runs, which they load themselves.
template <int HD>
__device__ __forceinline__ void attend_shared(const RangeAttn &p, Lds<HD> &lds, const Parts &parts, const scalar_i32 *pages, const int32_t *rows, int nrows, int g, int c, int r0, int r1) {
  constexpr int NJ = HD / 16, ND = HD / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, half = l >> 5, G = p.Hq / p.Hkv;
  const int blocks = nrows * G > 64 ? 4 : nrows * G > 32 ? 2 : 1, turns = 4 / blocks, turn = wave / blocks;
  const int col = wave % blocks * 32 + (l & 31), r = col / G, head = col % G;
  const bool mine = r < nrows;
  const int b = rows[mine ? r : 0];
  const float scale = score_scale<HD>();
  const int64_t page_elems = (int64_t)2 * p.page_tokens * HD;
  const int per_page = p.page_tokens >> 5;
  Block<HD> x;
  auto run_at = [&](int run, int page) { return p.kv + ((int64_t)page * p.Hkv + g) * page_elems + (int64_t)(run % per_page) * 32 * HD; };
  const int in_k = Block<HD>::in_k(l), in_v = Block<HD>::in_v(l);
  if (blocks == 4) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int LOADS = HD / 32;   // of a wavefront per run: 1 KiB each, the first two wavefronts' of K, the others' of V
    const int n = r1 - r0;
    // Run i, or the last one again: three are always on their way, so every wait is for a number of them.
    // The page of the run that is loaded next.  Ids are held 64 at a time, one to a lane: a scalar load in the loop would make every read of LDS wait for all
    // that are under way.
    const int page0 = r0 / per_page, pages_most = (r1 - 1) / per_page - page0;
    int in_page = r0 - page0 * per_page, at_page = 0, ids;
    const bf16_t *base;
    auto take_ids = [&] {
      ids = pages[page0 + min(at_page + l, pages_most)];
      asm volatile("" : "+v"(ids));   // (the wait is here, not wherever they are used)
    };
    auto turn_page = [&] {
      base = p.kv + ((int64_t)__builtin_amdgcn_readlane(ids, at_page & 63) * p.Hkv + g) * page_elems + (wave >= 2 ? (int64_t)p.page_tokens * HD : 0);
    };
    take_ids();
    turn_page();
    auto load = [&](int i) {
      const bf16_t *from = base + (int64_t)in_page * (32 * HD);
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)from, 0, 32 * HD * 2, 0x00020000);
#pragma unroll
      for (int u = 0; u < LOADS; ++u)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void *)(lds.ring[i % RING] + (wave * LOADS + u) * 512), 16, l * 16, (wave % 2 * LOADS + u) * 1024, 0, 0);
      if (i + 1 < n && ++in_page == per_page) {
        in_page = 0;
        if ((++at_page & 63) == 0) take_ids();
        turn_page();
      }
    };
    x.begin(p.q + ((int64_t)b * p.Hq + g * G + head) * HD + half * 8, mine);
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) load(i);
    auto read_k = [&](int i, bf16x8 (&kf)[NJ]) {
      const bf16_t *kb = lds.ring[i % RING] + in_k;
#pragma unroll
      for (int j = 0; j < NJ; ++j) kf[j] = *(const bf16x8 *)(kb + j * 256);
    };
    // one run; the next one's scores are under way on the matrix cores while this one's are weighed
    auto step = [&](int i, f32x16 &s, f32x16 &s_next) {
      // run i + 1 has arrived, and every wavefront is done with run i - 1
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(LOADS) : "memory");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      load(i + RING - 1);
      // (behind the last run: whatever the ring holds, and nobody's scores)
      bf16x8 kf[NJ], vf[ND][2], pf[2];
      read_k(i + 1, kf);
      const bf16_t *vb = lds.ring[i % RING] + 32 * HD + in_v;
#pragma unroll
      for (int k = 0; k < ND; ++k)
#pragma unroll
        for (int q = 0; q < 2; ++q) vf[k][q] = *(const bf16x8 *)(vb + k * 1024 + q * 256);
      const float alpha = x.peak(s, scale);
      __builtin_amdgcn_s_setprio(1);   // before the other workgroup's reads and barriers (64 rows of 5 heads, 131072 shared positions, 8 kv heads, the call 234 -> 221 us)
      s_next = x.scores(kf);
      x.weigh(s, scale, alpha, pf);
      x.add(vf, pf);
      // weights between the products: a wavefront issues in order
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 6 * 8 / NJ, 0);
      }
#pragma unroll
      for (int j = 0; j < 2 * ND; ++j) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 2 * 4 / ND, 0);
      }
      __builtin_amdgcn_s_setprio(0);
    };
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(2 * LOADS) : "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(x.qf[j]));   // (the queries are here: in the loop their wait would be one for every load on its way)
    f32x16 s0, s1;
    {
      bf16x8 kf[NJ];
      read_k(0, kf);
      s0 = x.scores(kf);
    }
    for (int i = 0; i < n; i += 2) {
      step(i, s0, s1);
      if (i + 1 < n) step(i + 1, s1, s0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();   // the ring is free
#endif
  } else {
    bf16x8 kf[NJ], vf[ND][2];
    auto load_k = [&](const bf16_t *kb) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) kf[j] = *(const bf16x8 *)(kb + in_k + j * 256);
    };
    auto load_v = [&](const bf16_t *kb) {
      const bf16_t *vb = kb + (int64_t)p.page_tokens * HD + in_v;
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int q = 0; q < 2; ++q) vf[i][q] = *(const bf16x8 *)(vb + i * 1024 + q * 256);
    };
    x.begin(p.q + ((int64_t)b * p.Hq + g * G + head) * HD + half * 8, mine);
    const int first = r0 + turn;
    if (first < r1) {
      const bf16_t *kb = run_at(first, pages[first / per_page]);
      load_k(kb);
      load_v(kb);
    }
    int page = first + turns < r1 ? pages[(first + turns) / per_page] : 0;
    for (int run = first; run < r1; run += turns) {
      f32x16 s = x.scores(kf);
      const int nxt = run + turns;
      const bf16_t *nb = nullptr;
      if (nxt < r1) {
        nb = run_at(nxt, page);
        load_k(nb);
        page = nxt + turns < r1 ? pages[(nxt + turns) / per_page] : 0;
      }
      bf16x8 pf[2];
      const float alpha = x.peak(s, scale);
      x.weigh(s, scale, alpha, pf);
      x.add(vf, pf);
      if (nb) load_v(nb);
    }
  }
  x.lsum = with_xor32(x.lsum, OpSum{});
  // the wavefronts of a block of columns, half of those left at a time: the later runs' result through LDS into the earlier ones'
  auto &so = lds.pair.o;
  auto &sml = lds.pair.ml;
  for (int left = turns; left > 1; left /= 2) {
    const int at = (wave - left / 2 * blocks) & 1, cc = l & 31;   // (two blocks of one turn, or two turns of one block)
    if (turn >= left / 2 && turn < left) {
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) *(f32x4 *)&so[at][cc][i * 32 + e * 2 + half * 4] = x.four(i, e);
      if (half == 0) { sml[at][cc][0] = x.m; sml[at][cc][1] = x.lsum; }
    }
    __syncthreads();
    if (turn < left / 2) {
      const int from = wave & 1;
      float M, e0, e1;
      score_factors(x.m, sml[from][cc][0], scale, M, e0, e1);
      x.lsum = fold_value(x.lsum, e0, sml[from][cc][1], e1);
      x.m = M;
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const f32x4 v = *(const f32x4 *)&so[from][cc][i * 32 + e * 2 + half * 4];
#pragma unroll
          for (int k = 0; k < 4; ++k) x.o[i][e + k] = fold_value(x.o[i][e + k], e0, v[k], e1);
        }
    }
    __syncthreads();
  }
  if (turn || !mine) return;
  const int64_t part = ((int64_t)b * p.Hkv + g) * parts.max_chunks + c;
  float *to = parts.o + (part * G + head) * HD;
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int e = 0; e < 16; e += 4) *(f32x4 *)(to + i * 32 + e * 2 + half * 4) = x.four(i, e);
  if (half == 0) *(float2 *)(parts.ml + part * ATTN_ML + head * 2) = make_float2(x.m, x.lsum);
}

// A workgroup an item, and more where there are more than 4096 (workgroups without one cost nothing: 512 to 100000 the same time; 512 that draw items from a counter
// take 6 to 10 us longer).
// 16 prompts of 2048 with 16 rollouts of 1500 on average each, 7B shape, 779 MB and 11.5 GFLOP: 138 to 154 us, 5.1 to 5.7 TB/s.  64 rollouts of one prompt of up to 16384, 32B shape, 109 MB
// and 18.9 GFLOP: 42 us, bound by the matrix products and the vector operations on their results.
template <int HD>
__global__ __launch_bounds__(256, 2) void attn_shared_kernel(RangeAttn p, SharedWork w) {
  __shared__ __attribute__((aligned(16))) Lds<HD> sm;
  const scalar_i32 *head = (const scalar_i32 *)w.head;   // (the launch writes neither: scalar loads)
  const int total = head[0] * p.Hkv;
  for (int item = blockIdx.x; item < total; item += gridDim.x) {
    if (item != (int)blockIdx.x) __syncthreads();   // LDS is free
    const int g = item % p.Hkv;
    const scalar_i32 *rec = (const scalar_i32 *)(w.items + (int64_t)(item / p.Hkv) * ITEM_INTS);
    const int kind = rec[0], at = rec[1], c = rec[2], n = rec[3], last = rec[4], b = rec[5], chunk = rec[6];
    const scalar_i32 *pages = (const scalar_i32 *)(p.page_table + (int64_t)b * p.pages_per_seq);   // (the launch does not write it: scalar loads)
    if (kind == ITEM_OWN) {
      const Sight see(n, last);
      attend_item<HD, 4>(p, sm.fold, w.own, at, g, pages, see, c, w.own_runs, last == 0 && see.runs <= w.own_runs);
    } else {
      attend_shared<HD>(p, sm, w.shared, pages, w.rows + at, last, g, c, c * chunk, min(n, (c + 1) * chunk));
    }
  }
}

// Work items of a call, by one workgroup of a thread a row (256 threads where they do: 256 rows in 16 groups 7.0 -> 5.8 us): which rows take part in a group's
// shared runs (those whose context covers them), tiles of such rows times chunks of the runs, and chunks of what is left of every row.  Offsets that do not ascend
// inside [0, n_seq] make no groups; of a row that is listed twice the first place counts; every place out of range is passed over.
template <int NT>
__global__ __launch_bounds__(NT) void shared_items_kernel(RangeAttn p, SharedPrompts q, SharedWork w) {
  constexpr int LENGTHS = 64;
  __shared__ int count[LENGTHS], off[NT + 1], pre[NT + 1], claim[NT], s_ctx[NT], s_start[NT], first_item[NT], first_own[NT], cnt[NT], sh[NT], s_chunk[NT], s_chunks[NT], s_parts[NT], s_rows[NT];
  const int t = threadIdx.x;
  // (from places that are there for every thread: behind a condition each read would wait for the one before it)
  const int shared0 = q.shared[min(t, q.n_groups - 1)], ctx0 = p.ctx_len[min(t, p.n_seq - 1)], off0 = q.offsets[min(t, q.n_groups)];
  const int listed0 = q.offsets[0], listed1 = q.offsets[q.n_groups];
  const bool listed = listed0 >= 0 && t >= listed0 && listed1 <= p.n_seq && t < listed1;
  const int named = listed ? q.rows ? q.rows[t] : t : -1;   // (under way with everything else)
  int bad = 0;
  if (t < LENGTHS) count[t] = 0;
  for (int i = t; i <= q.n_groups; i += NT) {
    off[i] = i == t ? off0 : q.offsets[i];
    bad |= off[i] < 0 || off[i] > p.n_seq;
  }
  const int ctx = t < p.n_seq ? min(max(ctx0, 0), p.max_ctx) : 0;
  const int runs = t < q.n_groups ? min(max(shared0, 0), q.max_shared) >> 5 : 0;
  s_ctx[t] = ctx;
  claim[t] = NT;
  s_start[t] = s_parts[t] = 0;
  sh[t] = runs;
  int chunks = 0;
  s_chunk[t] = runs ? w.cut.chunk(runs, chunks) : 0;
  s_chunks[t] = chunks;
  __syncthreads();
  for (int i = t; i < q.n_groups; i += NT) bad |= off[i] > off[i + 1];
  bad = __syncthreads_or(bad);
  int row = -1, gr = 0;
  if (!bad && listed) {
    int hi = q.n_groups;
    while (hi - gr > 1) {
      const int mid = (gr + hi) >> 1;
      if (off[mid] <= t) gr = mid; else hi = mid;
    }
    row = named < 0 || named >= p.n_seq ? -1 : named;
    if (row >= 0) atomicMin(&claim[row], t);
  }
  __syncthreads();
  const bool shares = row >= 0 && claim[row] == t && sh[gr] > 0 && s_ctx[row] >= sh[gr] * 32;
  int2 total;
  const int place = block_scan<NT>(make_int2(shares, 0), &total).x - shares;
  pre[t] = place;
  if (t == 0) pre[NT] = total.x;
  if (shares) {
    w.rows[place] = s_rows[place] = row;
    s_start[row] = sh[gr];
    s_parts[row] = s_chunks[gr];
  }
  __syncthreads();
  const int own_runs = (ctx + 31) / 32 - s_start[t], own_chunks = (own_runs + w.own_runs - 1) / w.own_runs;
  const int mine = bad || t >= q.n_groups ? 0 : pre[off[t + 1]] - pre[off[t]];
  cnt[t] = mine;
  const int tiles = (mine + w.tile_rows - 1) / w.tile_rows;
  const int2 items = make_int2(tiles * chunks, max(0, own_chunks - 1));
  const int2 at = block_scan<NT>(items, &total);
  first_item[t] = at.x - items.x;
  first_own[t] = at.y - items.y;
  if (t < p.n_seq) w.start[t] = make_int2(s_start[t], s_parts[t]);
  // rows' last chunks, longest first (in no order among equals: who takes an item changes nothing in its result): places by counting
  const int last_runs = own_chunks > 0 ? own_runs - (own_chunks - 1) * w.own_runs : 0;   // 1 .. own_runs
  if (last_runs) atomicAdd(&count[LENGTHS - 1 - last_runs * (LENGTHS - 1) / w.own_runs], 1);
  __syncthreads();
  if (t < LENGTHS) {   // (one wavefront)
    const int up_to = wave_scan(count[t]);
    if (t == LENGTHS - 1) w.head[0] = min(w.cap, total.x + total.y + up_to);
    count[t] = up_to - count[t];
  }
  __syncthreads();
  const int last = last_runs ? atomicAdd(&count[LENGTHS - 1 - last_runs * (LENGTHS - 1) / w.own_runs], 1) : 0;
  auto find = [](const int *starts, int n, int i) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (starts[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
  };
  auto put = [&](int i, int kind, int a, int c, int n, int last, int b, int chunk) {
    if (i >= w.cap) return;
    int4 *rec = (int4 *)(w.items + (int64_t)i * ITEM_INTS);
    rec[0] = make_int4(kind, a, c, n);
    rec[1] = make_int4(last, b, chunk, 0);
  };
  auto put_own = [&](int i, int b, int c, int ctx, int start) { put(i, ITEM_OWN, b, c, ctx, start, b, 0); };
  for (int i = t; i < total.x; i += NT) {
    const int k = find(first_item, q.n_groups, i), j = i - first_item[k];
    const int n_tiles = (cnt[k] + w.tile_rows - 1) / w.tile_rows, per = (cnt[k] + n_tiles - 1) / n_tiles, tile = j % n_tiles, c = j / n_tiles;   // tiles of one chunk side by side
    const int rows = pre[off[k]] + tile * per;
    put(i, ITEM_SHARED, rows, c, sh[k], min(per, cnt[k] - tile * per), s_rows[rows], s_chunk[k]);
  }
  for (int i = t; i < total.y; i += NT) {
    const int b = find(first_own, p.n_seq, i);
    put_own(total.x + i, b, i - first_own[b], s_ctx[b], s_start[b]);
  }
  if (own_chunks > 0) put_own(total.x + total.y + last, t, own_chunks - 1, ctx, s_start[t]);
}

// Rows of several parts: a workgroup per (row, kv head), four elements of a head per thread, parts folded in order, eight loads under way (64 rows of 5 heads, 8 kv
// heads, 20 parts: 8.2 us; by four times as many threads, the parts cut in four, 11.9; by the workgroup that ends last in the main kernel, the call 58 -> 146).
struct MergeRows { Parts first, second; const int2 *start; int32_t second_runs, window, sinks; };
template <int HD>
__global__ __launch_bounds__(256) void attn_join_kernel(RangeAttn p, MergeRows q) {
  const int b = blockIdx.x / p.Hkv, g = blockIdx.x % p.Hkv, G = p.Hq / p.Hkv;
  const int ctx = min(p.ctx_len[b], p.max_ctx);
  if (ctx <= 0) return;
  const int64_t row = (int64_t)b * p.Hkv + g;
  const float scale = score_scale<HD>();
  int n1 = 0, n2;
  auto put = [&](int i, float L, f32x4 O) { *(bf16x4 *)(p.out + ((int64_t)b * p.Hq + g * G) * HD + i * 4) = finish(O, L); };
  auto load = [&](const Parts &from, int c, int i, float2 &ml, f32x4 &o) {
    const int64_t part = row * from.max_chunks + c;
    ml = *(const float2 *)(from.ml + part * ATTN_ML + i / (HD / 4) * 2);
    o = *(const f32x4 *)(from.o + part * G * HD + i * 4);
  };
  float2 ml[8];
  f32x4 o[8];
  const bool early = q.start && q.first.max_chunks >= 8;
  if (early)   // parts of what is shared: on their way before it is known how many there are (16 rollouts of one prompt of 16384, 32B shape, the call 34.8 -> 33.3 us)
#pragma unroll
    for (int u = 0; u < 8; ++u) load(q.first, u, min((int)threadIdx.x, G * (HD / 4) - 1), ml[u], o[u]);
  if (q.start) {
    const int2 at = q.start[b];
    n1 = at.y;
    n2 = ((ctx + 31) / 32 - at.x + q.second_runs - 1) / q.second_runs;
  } else {
    n2 = (Sight(ctx, q.window, q.sinks).runs + q.second_runs - 1) / q.second_runs;
  }
  if (n1 == 0 && n2 == 1) return;   // written already
  for (int i = threadIdx.x; i < G * (HD / 4); i += 256) {
    float M = -INFINITY, L = 0.f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
    auto fold = [&](float2 ml, f32x4 o) {
      float top, e0, e1;
      score_factors(M, ml.x, scale, top, e0, e1);
      O = fold_value(O, e0, o, e1);
      L = fold_value(L, e0, ml.y, e1);
      M = top;
    };
    int c0 = 0;
    if (early && i == (int)threadIdx.x) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (u < n1) fold(ml[u], o[u]);
      c0 = min(n1, 8);
    }
    for (; c0 < n1 + n2; c0 += 8) {
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int c = min(c0 + u, n1 + n2 - 1);
        load(c < n1 ? q.first : q.second, c < n1 ? c : c - n1, i, ml[u], o[u]);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c0 + u < n1 + n2) fold(ml[u], o[u]);
    }
    put(i, L, O);
  }
}

int ok() { return hipGetLastError() == hipSuccess ? 0 : -7; }
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <typename F>
void with_head(int hd, F f) {
  if (hd == 128) f(std::integral_constant<int, 128>{});
  else if (hd == 64) f(std::integral_constant<int, 64>{});
  else f(std::integral_constant<int, 32>{});
}

// Most runs a row sees through a window.
int64_t window_runs(int max_ctx, int window, int sinks) {
  return std::min<int64_t>(up(max_ctx, 32), up(sinks, 32) + ((int64_t)window + 30) / 32 + 1);
}

// How a windowed call is cut.  A workgroup of four wavefronts streams 45 to 57 bytes a nanosecond, the chip what 128 of them do: with fewer (row, kv head) pairs
// a row is cut into chunks, and the parts cost a launch and about 1.3 us for every eight of them (us, captured calls; c chunks: as many as squared stay
// below twice the runs).  Or all of a row goes to eight wavefronts, which saves the launch: where chunks hold next to nothing (runs * hd up to
// 2560; split / eight wavefronts: head dimension 128, 4 pairs, 16 runs 6.7 / 5.6, 32 runs 7.0 / 7.7; 64, 16 pairs, 32 runs 6.3 / 5.4, 64 runs 8.0 / 7.8; 32, 16 pairs, 64 runs
// 8.8 / 7.8, 128 runs 12.4 / 13.9), up to twice as much with 8 pairs or fewer, where the caller's second launch costs more than the cut saves (6 pairs of 128, 32 runs, captured
// 7.5 / 8.2, one by one 11.9 / 9.0, 40 runs 8.4 / 8.9 and 11.9 / 9.1; 4 pairs of 64, 80 runs 8.3 / 10.0 and 11.7 / 9.4), and where
// pairs are many but not four workgroups' worth (128 pairs, 128 runs 50 / 51; 200 pairs 74 / 66; 400 pairs 148 / 134).
// Of somewhat more pairs than units, some units would have two and most one: long rows are cut in four (260 pairs of 128, 64 runs 60.5 -> 52.0, 256 runs 231 -> 182; 320 pairs, 128 runs
// 129 -> 117; 352 pairs, 256 runs 264 -> 236; 384 pairs 150 / 149; 312 pairs, 40 runs 47 / 46).
// 256 workgroups are enough where rows see equally much (32 pairs, 128 runs: 128 workgroups 19.5, 256 17.0, 512 18.4, 1024 23.4).  A window over whole contexts, of which
// the longest may be several times the mean, has up to 1024, many of them with nothing to do (longest row / mean of lognormal lengths 4 to 5: 102 rows, one kv head of 32,
// mean 1150, 21.5 -> 11.1; 20 rows, two of 128, mean 2000, 25.7 -> 17.5; but 16 rows of 4300 each, two of 128, 14.1 -> 16.1).  So has any window of 512 runs or more over up to 256
// pairs, as rows may see little of it (lognormal lengths with a mean of 4000, window 32768, 7B shape: 16 rows 74 -> 44, 32 187 -> 88, 64 217 -> 171; rows of 33000 each 167 -> 173, 364 -> 333,
// 638 -> 648); more pairs lose more than they gain (200 of 200, equal rows 264 -> 285).
struct Split { int64_t parts; int chunk, chunks, waves; };
Split window_split(int n_seq, int Hkv, int hd, int max_ctx, int window, int sinks) {
  const int64_t runs = window_runs(max_ctx, window, sinks), pairs = (int64_t)n_seq * Hkv;
  int64_t chunks = 1;
  const bool whole = window >= max_ctx, unequal = whole || (runs >= 512 && pairs <= 256);
  const bool little = runs * hd <= 2560 || (pairs <= 8 && runs * std::max(hd, 64) <= 5120);
  if ((pairs < 128 || unequal) && !little) {
    chunks = std::max<int64_t>(1, (unequal ? 1024 : 256) / pairs);
    while (chunks > 1 && chunks * chunks > (whole ? 1 : 2) * runs) --chunks;
  } else if (pairs > 256 && pairs <= 352 && runs >= 48) {
    chunks = 4;
  }
  Split s;
  s.chunk = (int)(chunks > 1 ? up(up(runs, chunks), 4) * 4 : runs);
  s.chunks = (int)up(runs, s.chunk);
  s.waves = s.chunks == 1 && pairs < 512 ? 8 : 4;
  s.parts = s.chunks > 1 ? pairs * s.chunks : 0;
  return s;
}

// Most parts of any windowed call of as many pairs and runs or fewer, so that a workspace does for those too: fewer rows are cut into more chunks.  Chunks squared stay
// below twice the runs; a call of up to 256 pairs (a whole window: 1024) has as many parts at most, one of up to 352 pairs four a pair.
int64_t most_window_parts(int64_t pairs, int64_t runs) {
  int64_t chunks = 1;
  while (chunks < 1024 && (chunks + 1) * (chunks + 1) <= 2 * runs) ++chunks;
  return std::max(chunks > 1 ? std::min<int64_t>(1024, pairs * chunks) : 0, pairs > 256 && runs >= 48 ? 4 * std::min<int64_t>(pairs, 352) : 0);
}

// How a call with shared prompts is cut: by its shape, and a group's shared runs by their number, so that a row's result does not depend on what the other rows hold.  A row's own part
// goes in chunks of up to 64 runs (16 prompts of 2048 with 16 rollouts each, 7B shape: chunks of 16, 32, 64 and 128 runs 165, 158, 155 and 155 us) and
// at least 16 (32 rows of 4 prompts of 1000 and 300 on average, 7B shape: by 4, 8 and 16 runs 23.1, 21.6 and 20.8).  Shared runs are cut
// into as many chunks as make 256 workgroups, 384 where that leaves 24 runs each, 512 where that leaves 48: every chunk leaves a part of every row, and rows' own chunks wait for a place
// behind them (64 rollouts of one prompt, 32B shape, us by workgroups: 448 runs, 240 51.0, 336 47.7, 384 49.0, 456 52.6; 512 runs, 264 52.3, 360 51.2, 384 52.0, 456 54.7; 1640
// runs, 384 120, 512 115).  Longer ones do where the rows' own parts keep the chip busy meanwhile: half of their time, at a quarter of the most they could be and 0.9 us a run
// (16 prompts of 2048 with 16 rollouts of 1500 on average each, 7B shape, by 64, 256 and 512 workgroups 153, 169 and 179; 4 prompts of 4096 with 16 rollouts of 300 44, 36, 44).
// What own parts could be is a bound that may be far above what they are, in a captured step above all, so chunks are no longer than OWN_RUNS for it (the same 64 rollouts of up to 512 runs,
// max_ctx 17584 54 us, 131072 64, without this limit 295; the 4 prompts 31, 54 and 87; the 16 prompts 148, 148 and 148, with a limit of 48 or 32 153 and 156).
constexpr int64_t OWN_RUNS = 64;         // (by head dimension 128)
constexpr int64_t SHARED_GROUPS = 512;   // most workgroups of shared runs that are cut
struct SharedSplit { Split own; SharedCut cut; int chunks; int64_t shared_parts; int tile_rows; int64_t cap; };
SharedSplit shared_split(int n_seq, int n_groups, int Hq, int Hkv, int hd, int max_ctx, int max_shared) {
  SharedSplit s;
  s.tile_rows = 128 / (Hq / Hkv);
  s.own.chunk = std::clamp(attention_chunk_tokens(n_seq, Hkv, max_ctx) / 32, 16, 64);
  s.own.chunks = (int)up(up(max_ctx, 32), s.own.chunk);
  s.own.parts = (int64_t)n_seq * Hkv * s.own.chunks;
  const int64_t runs = std::max(1, max_shared / 32), units = n_groups * up(up(n_seq, n_groups), s.tile_rows) * Hkv;
  const int64_t own_bytes = (int64_t)n_seq * Hkv * (max_ctx - max_shared) * hd;   // (a quarter of four bytes per element and position)
  const int64_t own_runs = own_bytes / 5500000 * 128 / hd * 5 / 9;                // of 0.9 us (by head dimension) in half of their time at 5.5 TB/s
  int64_t most[3];
  for (int i = 0; i < 3; ++i) {
    most[i] = std::max<int64_t>(1, (i + 2) * SHARED_GROUPS / 4 / units);
    s.cut.by[i] = Divisor((uint32_t)most[i]);
  }
  s.cut.from[0] = (int32_t)up(24 * 384, units);
  s.cut.from[1] = (int32_t)up(48 * 512, units);
  s.cut.own_runs = (int32_t)std::min<int64_t>(up(own_runs, 4) * 4, OWN_RUNS * 128 / hd);
  s.chunks = (int)std::min(most[(runs >= s.cut.from[0]) + (runs >= s.cut.from[1])], up(runs, std::max(8, s.cut.own_runs)));   // the most of a group
  s.shared_parts = (int64_t)n_seq * Hkv * s.chunks;
  s.cap = (n_groups + n_seq / s.tile_rows) * (int64_t)s.chunks + (int64_t)n_seq * s.own.chunks;
  return s;
}

// The largest number of parts and items of any call of as many rows, groups and positions or fewer.  Own parts: chunks of less than 64 runs are taken where those of twice
// the length would be less than 2048.  Shared parts: chunks hold eight runs at least, and they are SHARED_GROUPS / units at most, or 1; units are a kv head's groups at least, and its tiles.
struct SharedMost { int64_t own_parts, shared_parts, cap; };
SharedMost most_shared(int n_seq, int n_groups, int Hq, int Hkv, int max_ctx, int max_shared) {
  const int64_t pairs = (int64_t)n_seq * Hkv, tile_rows = 128 / (Hq / Hkv), chunks = std::clamp<int64_t>(up(max_shared / 32, 8), 1, SHARED_GROUPS);
  SharedMost m;
  m.own_parts = std::max(pairs * up(max_ctx, 64 * 32), std::min<int64_t>(4096, pairs * up(max_ctx, 16 * 32)));
  m.shared_parts = std::min(pairs * chunks, std::max(pairs, SHARED_GROUPS * tile_rows));
  const int64_t tiles = n_groups + n_seq / tile_rows;
  m.cap = std::min(tiles * chunks, std::max<int64_t>(tiles, 2 * SHARED_GROUPS / Hkv)) + up(m.own_parts, Hkv);
  return m;
}

int64_t part_floats(int G, int hd) { return (int64_t)G * hd + ATTN_ML; }
Parts take_parts(float *&at, int64_t parts, int chunks, int G, int hd) {
  Parts r{at, at + parts * G * hd, chunks};
  at += parts * part_floats(G, hd);
  return r;
}

}  // namespace

bool shared_fits(int n_seq, int n_groups, int Hq, int Hkv, int hd, int max_ctx, int max_shared) {
  return shared_split(n_seq, n_groups, Hq, Hkv, hd, max_ctx, max_shared).cap * Hkv <= MOST_ITEMS;
}

int64_t window_workspace_bytes(int n_seq, int Hq, int Hkv, int hd, int max_ctx, int window, int sinks) {
  return most_window_parts((int64_t)n_seq * Hkv, window_runs(max_ctx, window, sinks)) * part_floats(Hq / Hkv, hd) * 4;
}

int launch_attention_window(const RangeAttn &p, int window, int sinks, void *workspace, hipStream_t s) {
  const Split sp = window_split(p.n_seq, p.Hkv, p.hd, p.max_ctx, window, sinks);
  float *at = (float *)workspace;
  const Parts parts = take_parts(at, sp.parts, sp.chunks, p.Hq / p.Hkv, p.hd);
  with_head(p.hd, [&](auto HD) {
    constexpr int hd = decltype(HD)::value;
    const dim3 grid((unsigned)((int64_t)p.n_seq * sp.chunks * p.Hkv));
    if (sp.waves == 8) hipLaunchKernelGGL((attn_window_kernel<hd, 8>), grid, dim3(512), 0, s, p, parts, window, sinks, sp.chunk);
    else hipLaunchKernelGGL((attn_window_kernel<hd, 4>), grid, dim3(256), 0, s, p, parts, window, sinks, sp.chunk);
    if (sp.chunks > 1) {
      const MergeRows q{parts, parts, nullptr, sp.chunk, window, sinks};
      hipLaunchKernelGGL((attn_join_kernel<hd>), dim3(p.n_seq * p.Hkv), dim3(256), 0, s, p, q);
    }
  });
  return ok();
}

static int64_t shared_ints(int n_seq, int64_t cap) { return (HEAD_INTS + cap * ITEM_INTS + 3 * n_seq + 63) / 64 * 64; }

// Calls in which every row reads all of its context by itself, in one or two launches instead of three.
// They hold at most 512 MiB, and sharing would read at most 128 MiB less, which is what the list and the join cost (us, by the list / every row by itself: 32 rows of 4 prompts
// of 700, 7B shape, 40 MB less, 19.6 / 15.3; 16 rows of one prompt of 8000, 1.5B shape, 123 MB, 24.0 / 20.5; 32 rows of 4 prompts of 2500, 7B shape, 143 MB, 22.5 / 25.7).
// Beyond, the list is worth its time even if nothing is shared, for the order in which rows of all lengths are taken (100 rows of 1500 on average, 7B shape, 64 / 98).
static bool shared_alone(int n_seq, int n_groups, int Hkv, int hd, int max_ctx, int max_shared) {
  const int64_t bytes = (int64_t)Hkv * hd * 4;   // of a position
  return n_seq * (max_ctx * bytes) <= (int64_t)512 << 20 && (n_seq - n_groups) * (max_shared * bytes) <= (int64_t)128 << 20;
}

int64_t shared_workspace_bytes(int n_seq, int n_groups, int Hq, int Hkv, int hd, int max_ctx, int max_shared) {
  const int64_t alone = window_workspace_bytes(n_seq, Hq, Hkv, hd, max_ctx, max_ctx, 0);
  if (shared_alone(n_seq, 1, Hkv, hd, max_ctx, max_shared)) return alone;   // (as are all smaller calls)
  const SharedMost m = most_shared(n_seq, n_groups, Hq, Hkv, max_ctx, max_shared);
  return std::max(alone, (shared_ints(n_seq, m.cap) + (m.own_parts + m.shared_parts) * part_floats(Hq / Hkv, hd)) * 4);
}

int launch_attention_shared(const RangeAttn &p, const SharedPrompts &q, void *workspace, hipStream_t s) {
  if (shared_alone(p.n_seq, q.n_groups, p.Hkv, p.hd, p.max_ctx, q.max_shared)) return launch_attention_window(p, p.max_ctx, 0, workspace, s);
  const int G = p.Hq / p.Hkv;
  const SharedSplit sp = shared_split(p.n_seq, q.n_groups, p.Hq, p.Hkv, p.hd, p.max_ctx, q.max_shared);
  SharedWork w;
  w.head = (int32_t *)workspace;
  w.items = w.head + HEAD_INTS;
  w.start = (int2 *)(w.items + sp.cap * ITEM_INTS);
  w.rows = (int32_t *)(w.start + p.n_seq);
  float *at = (float *)(w.head + shared_ints(p.n_seq, sp.cap));
  w.own = take_parts(at, sp.own.parts, sp.own.chunks, G, p.hd);
  w.shared = take_parts(at, sp.shared_parts, sp.chunks, G, p.hd);
  w.own_runs = sp.own.chunk;
  w.cut = sp.cut;
  w.tile_rows = sp.tile_rows;
  w.cap = (int32_t)sp.cap;
  if (p.n_seq <= 256) hipLaunchKernelGGL(shared_items_kernel<256>, dim3(1), dim3(256), 0, s, p, q, w);
  else hipLaunchKernelGGL(shared_items_kernel<1024>, dim3(1), dim3(1024), 0, s, p, q, w);
  with_head(p.hd, [&](auto HD) {
    constexpr int hd = decltype(HD)::value;
    hipLaunchKernelGGL((attn_shared_kernel<hd>), dim3((unsigned)std::min<int64_t>(sp.cap * p.Hkv, 4096)), dim3(256), 0, s, p, w);
    const MergeRows m{w.shared, w.own, w.start, w.own_runs, 0, 0};
    hipLaunchKernelGGL((attn_join_kernel<hd>), dim3(p.n_seq * p.Hkv), dim3(256), 0, s, p, m);
  });
  return ok();
}

}  // namespace pl
