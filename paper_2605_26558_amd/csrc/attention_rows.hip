// Attention for the query rows of several sequences over a prefix that they share, and attention that adds up what every
// cached position received.
//
// cas_attention decodes a page of the cache for the query rows of one sequence.  Where a batch of sequences begins with the
// same pages, the decode, which is most of the time (a step of a walk is some nine vector operations, and the walks of the exact
// form take 25 + 18 steps for 32 values at 60 % kept, those of the fullest of 64 lanes), is the same for all of them: here a workgroup decodes a page once for up to 256 query rows whichever sequence they belong to, and goes through a run
// of pages with running maxima and sums, so that a row has one partial result per run and not per page.  What follows the
// prefix goes through the same kernel, sequence by sequence, in the same launch.
//   grid: (runs of the prefix x blocks of all rows, then per sequence runs x blocks of its rows) x kv heads
// A second kernel joins the partial results of a row in the order of the runs, prefix first.
//
// Attention within a window: the same kernel over the pages that a column of the sequence sees, those of the first positions and those of
// the window, numbered one after the other; there is no prefix.  The rest of the page table is not looked at.  A run is as long as
// there are places for all of the call's runs.  0 times an infinity of V would reach columns that do not see it: committed positions that only some
// columns see (up to fifteen, in at most two groups of sixteen) are cleared of infinities and NaN in the tiles, and these are added where
// the partial results are joined, as for vectors in flight.
//
// Attention weights: the partial kernel also writes the exponents of its scores, and the second launch, beside joining the
// rows, forms the weights of all rows of a kv head from them and adds them up.  Exponents are 4 bytes per row and position,
// a vector of K 131 in the draft form: cheaper than decoding K again.
//
// Measured (8 kv heads, 60 % kept, t = 4; us, both launches; in brackets the bytes of the streams at the rate of a copy): 16 sequences
// of 4 query heads a kv head over a shared 8192 and 500 of their own, draft 30 (5.5), with shared exponents 34 (3.1); 8 of 5 columns,
// exact, 300 of their own 42 (8.9), with shared exponents 46 (7.0); 32 of 8 query heads over 32768, exact, shared exponents 119 (29).
// One sequence with weights: 8192 positions, exact 20.1 (7.7), draft 18 (3.7), with shared exponents 23 (6.1) and 20 (2.1); 30011 and 7
// columns, exact 53 (28), draft 42 (14).  Within a window: one sequence, window 1024, draft 10.0 (0.4); 4096 and 7 columns, exact 19.4 (3.6); 16
// sequences, 4096, draft 48 (28), exact 73; 16 of 5 columns and 8 query heads, 8192, exact, shared exponents 160 (91).
// Bound by the vector operations of the decode: 58 to 84 % of a SIMD's cycles, the matrix products and the LDS beside them (busy 21 and
// 41 % of the time with 256 rows); a short window of one sequence by the two launches and, in the first, four round trips that wait for each
// other (arguments, page table, bitmap, fields).
// Against the sequences' own decodes (cas_attention_multi), sharing / not: 2 sequences behind 703 positions 10.0 / 8.6, 4 behind 2000
// 14.1 / 13.6, 8 of 5 columns behind 500, exact, 25 / 27, 16 behind 256 15 / 34, behind 8192 29 / 107: it pays from
// some four sequences on, and for more whatever the prefix is.
#include <algorithm>
#include "attention_rows_kernel.inl"
#include "kv_value.hpp"

namespace cas {

extern template int launch_rows_partial<true, false, RowsArgs>(cas_ctx*, const RowsArgs&, int, int);
extern template int launch_rows_partial<true, false, RowsWindowArgs>(cas_ctx*, const RowsWindowArgs&, int, int);
extern template int launch_rows_partial<false, false, RowsArgs>(cas_ctx*, const RowsArgs&, int, int);
extern template int launch_rows_partial<false, false, RowsWindowArgs>(cas_ctx*, const RowsWindowArgs&, int, int);
extern template int launch_rows_partial<true, true, RowsArgs>(cas_ctx*, const RowsArgs&, int, int);
extern template int launch_rows_partial<true, true, RowsWindowArgs>(cas_ctx*, const RowsWindowArgs&, int, int);
extern template int launch_rows_partial<false, true, RowsArgs>(cas_ctx*, const RowsArgs&, int, int);
extern template int launch_rows_partial<false, true, RowsWindowArgs>(cas_ctx*, const RowsWindowArgs&, int, int);

// Joins the partial results of a row in kMergeSums sums, of every kMergeSums-th split each, in order; then these in order.  One
// wave forms all four or four waves one each (PARTS), a lane two channels: how many waves there are goes by the row with the most
// splits of the launch, so the order of a row's additions must not depend on it.  Bound by latency: the pairs and kMergeAhead outputs
// are requested at once, the outputs through buffer descriptors, of no length past the end of the part: what lies there reads as 0
// without a branch.
constexpr int kMergeAhead = 16, kMergeSums = 4;
template <int PARTS, class ARGS>
__device__ __forceinline__ void merge_row(const ARGS& a, int block, int head) {
  constexpr bool kWindow = std::is_same<ARGS, RowsWindowArgs>::value;
  static_assert(PARTS == 1 || PARTS == kMergeSums, "");
  constexpr int kOwn = kMergeSums / PARTS;  // sums of a wave
  __shared__ float2 joined[4][64];
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int rr = block * (4 / PARTS) + wv / PARTS, part = wv % PARTS;
  if (rr >= a.rows) return;  // with four parts no wave of the workgroup is left
  const SeqTable t_row0(a.row0), t_cols(a.ncols), t_splits(a.splits), t_len(a.len), t_new(a.n_new), t_part0(a.part0);
  const int si = t_row0.which(rr);
  const struct {
    int ncols, row0, splits, len, n_new;
    uint32_t part0;
  } me = {t_cols[si], t_row0[si], t_splits[si], t_len[si], t_new[si], (uint32_t)t_part0[si]};
  const int r = rr - me.row0, rows = me.ncols * a.grp, ps = a.prefix_splits, n = ps + me.splits;
  const float2* mlp = a.ml_prefix + ((size_t)head * a.rows + rr) * ps;
  const float2* mlt = a.ml_tail + me.part0 + ((size_t)head * rows + r) * me.splits;
  auto pair = [&](int i) { return i < ps ? mlp[i] : mlt[i - ps]; };
  const char* op = reinterpret_cast<const char*>(a.out_prefix + ((size_t)head * a.rows + rr) * 128);
  const char* ot = reinterpret_cast<const char*>(a.out_tail + (me.part0 + (size_t)head * rows + r) * 128);
  const size_t sp = (size_t)a.g.n_kv_heads * a.rows * 512, st = (size_t)a.g.n_kv_heads * rows * 512;
  const int cnt = (n - part + PARTS - 1) / PARTS;  // splits of this part: part, part + PARTS, ...
  float2 o[kMergeAhead];
  auto request = [&](int q0) {
#pragma unroll
    for (int q = 0; q < kMergeAhead; ++q) {
      const int s = __builtin_amdgcn_readfirstlane(part + PARTS * (q0 + q));
      const char* at = s < ps ? op + s * sp : ot + (s - ps) * st;
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0, q0 + q < cnt ? 512 : 0, kRawBufferFlags);
      const auto two = __builtin_amdgcn_raw_buffer_load_b64(rs, 8 * lane, 0, 0);
      o[q] = make_float2(__uint_as_float(two[0]), __uint_as_float(two[1]));
    }
  };
  // words of the in-flight V that hold infinities or NaN: of one or two pages
  const int page0 = me.len >> 6, flags = 4 * ((me.len + me.n_new + 63) / 64 - page0);
  uint64_t odd = 0;
  if (lane < flags) odd = a.odd[((size_t)si * a.g.n_kv_heads + head) * 8 + lane];
  float2 own = make_float2(kLowest, 0.f), all = make_float2(kLowest, 0.f);  // pairs of split `lane` of the part, of the row
  if (lane < cnt) own = pair(part + PARTS * lane);
  if (lane < n) all = pair(lane);
  request(0);
  float M = all.x;
  for (int i = lane + 64; i < n; i += 64) M = fmaxf(M, pair(i).x);
  M = wave_max(M);
  float den = __builtin_amdgcn_exp2f(all.x - M) * all.y;
  for (int i = lane + 64; i < n; i += 64) {
    const float2 p = pair(i);
    den += __builtin_amdgcn_exp2f(p.x - M) * p.y;
  }
  den = wave_sum(den);
  float2 sums[kOwn];
#pragma unroll
  for (int k = 0; k < kOwn; ++k) sums[k] = make_float2(0.f, 0.f);
  for (int q0 = 0; q0 < cnt; q0 += kMergeAhead) {
    if (q0 > 0) {
      if ((q0 & 63) == 0) own = q0 + lane < cnt ? pair(part + PARTS * (q0 + lane)) : make_float2(kLowest, 0.f);
      request(q0);
    }
    const int w = __float_as_int(__builtin_amdgcn_exp2f(own.x - M));
#pragma unroll
    for (int q = 0; q < kMergeAhead; ++q) {
      const float ws = __int_as_float(__builtin_amdgcn_readlane(w, (q0 & 63) + q));
      sums[q % kOwn].x += ws * o[q].x;
      sums[q % kOwn].y += ws * o[q].y;
    }
  }
  float2 num = sums[0];
  if constexpr (PARTS > 1) {
    joined[part][lane] = num;
    __syncthreads();
    if (part != 0) return;
  }
#pragma unroll
  for (int p = 1; p < kMergeSums; ++p) {
    const float2 add = PARTS > 1 ? joined[p][lane] : sums[p % kOwn];
    num.x += add.x;
    num.y += add.y;
  }
  const int c = r / a.grp, gi = r - c * a.grp;
  auto lo = [](uint32_t x) { return __uint_as_float(x << 16); };
  auto hi = [](uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); };
  int from = 0;  // the first position that the row sees in its window
  if constexpr (kWindow) from = me.len + me.n_new - me.ncols + c - a.window + 1;
  auto add = [&](uint32_t q, uint32_t k, uint32_t v) {  // channels 2 lane, 2 lane + 1: the infinities and NaN among the two of v
    const float w = __builtin_amdgcn_exp2f(wave_sum(lo(q) * lo(k) + hi(q) * hi(k)) * a.scale2 - M);
    if ((v & 0x7F80u) == 0x7F80u) num.x += w * lo(v);
    if ((v & 0x7F800000u) == 0x7F800000u) num.y += w * hi(v);
  };
  if (__builtin_amdgcn_ballot_w64(odd != 0)) {  // those that the row sees, which the partial results left out
    const uint32_t q = reinterpret_cast<const uint32_t*>(a.Q[si] + ((size_t)c * a.n_q_heads + head * a.grp + gi) * 128)[lane];
    for (int i = 0; i <= me.n_new - me.ncols + c; ++i) {
      const int t = me.len + i;
      if (!(__shfl(odd, (t >> 4) - 4 * page0) >> (4 * (t & 15)) & 0xF)) continue;
      if constexpr (kWindow)
        if (t < from && t >= a.n_first) continue;
      const uint32_t k = reinterpret_cast<const uint32_t*>(a.Knew[si] + ((size_t)i * a.g.n_kv_heads + head) * 128)[lane];
      const uint32_t v = reinterpret_cast<const uint32_t*>(a.Vnew[si] + ((size_t)i * a.g.n_kv_heads + head) * 128)[lane];
      add(q, k, v);
    }
  }
  if constexpr (kWindow) {  // and those among committed positions that only some columns see
    const WindowPages pages(a.n_first, a.window, me.len, me.len + me.n_new, me.ncols);
    if (pages.zone0 < pages.zone1) {
      const uint32_t* edge = a.edge + ((size_t)si * a.g.n_kv_heads + head) * 2;
      const int slab = pages.zone0 >> 4, slabs = ((pages.zone1 - 1) >> 4) - slab + 1;
      const uint32_t bits = edge[0] | (slabs > 1 ? edge[1] << 16 : 0u);
      if (bits) {
        const SeqTable t_seq(a.seq);
        const uint32_t q = reinterpret_cast<const uint32_t*>(a.Q[si] + ((size_t)c * a.n_q_heads + head * a.grp + gi) * 128)[lane];
        for (int t = max(pages.zone0, from); t < pages.zone1; ++t) {
          if (!(bits >> (t - 16 * slab) & 1)) continue;
          const int page = min(max(a.table[(size_t)t_seq[si] * a.g.max_pages_per_seq + (t >> 6)], 0), a.g.n_pages - 1);
          auto two = [&](int kv) {
            auto one = [&](int col) -> uint32_t { return cached_value(a.g, a.spec_pool, a.verif_pool, a.layer, page, kv, head, t & 63, col, a.full); };
            return one(2 * lane) | one(2 * lane + 1) << 16;
          };
          add(q, two(0), two(1));
        }
      }
    }
  }
  uint32_t* out = reinterpret_cast<uint32_t*>(a.O[si] + ((size_t)c * a.n_q_heads + head * a.grp + gi) * 128) + lane;
  *out = (uint32_t)f32_to_bf16(num.x / den) | ((uint32_t)f32_to_bf16(num.y / den) << 16);
}

template <int PARTS, class ARGS>
__global__ __launch_bounds__(256) void rows_merge_kernel(ARGS a) { merge_row<PARTS>(a, blockIdx.x, blockIdx.y); }

// Weights of 256 positions of a kv head.  Every row's maximum and sum first, 16 lanes to a row; then the waves take every
// fourth row each, four positions a lane and eight rows requested at once, and are added in order.
constexpr int kWeightsRows = 16 * 48;  // most query rows of a kv head
constexpr int kWeightsPos = 256;

__device__ __forceinline__ void add_weights(const RowsArgs& a, int block, int head, const float* in, float* out, int64_t ld) {
  __shared__ float2 row_ml[kWeightsRows];
  __shared__ rows_f32x4 joined[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), rows = a.rows;
  const int ps = a.prefix_splits, own = a.splits[0], n = ps + own, len = a.len[0], total = len + a.n_new[0];
  const int pos = block * kWeightsPos + 4 * lane;
  const float* x = a.score + (size_t)head * rows * a.score_ld + pos;  // rows are padded to whole pages
  const bool there = pos < total;
  rows_f32x4 before = {0.f, 0.f, 0.f, 0.f};
  const int64_t at = (int64_t)head * ld + pos;
  if (wv == 0 && in) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (pos + e < len) before[e] = in[at + e];
  }
  // four pairs of a lane at once: of one row, or of four where 16 lanes hold all splits of a row
  const bool wide = n > 16;
  for (int r0 = tid >> 4; r0 < rows; r0 += wide ? 16 : 64) {
    float M[4], L[4];
    float2 p[4];
    auto pair = [&](int r, int i) {  // split i of row r, those of the prefix first
      const size_t row = (size_t)head * rows + min(r, rows - 1);
      return i >= n ? make_float2(kLowest, 0.f) : i < ps ? a.ml_prefix[row * ps + i] : a.ml_tail[row * own + i - ps];
    };
    const int i0 = lane & 15;
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = wide ? pair(r0, i0 + 16 * k) : pair(r0 + 16 * k, i0);
#pragma unroll
    for (int k = 0; k < 4; ++k) M[k] = p[k].x;
    if (wide) {
      M[0] = fmaxf(fmaxf(M[0], M[1]), fmaxf(M[2], M[3]));
      for (int i = i0 + 64; i < n; i += 16) M[0] = fmaxf(M[0], pair(r0, i).x);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k == 0 || !wide) M[k] = row16_max(M[k]);
      L[k] = __builtin_amdgcn_exp2f(p[k].x - M[wide ? 0 : k]) * p[k].y;
    }
    if (wide) {
      L[0] = (L[0] + L[1]) + (L[2] + L[3]);
      for (int i = i0 + 64; i < n; i += 16) {
        const float2 q = pair(r0, i);
        L[0] += __builtin_amdgcn_exp2f(q.x - M[0]) * q.y;
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k > 0 && wide) break;
      L[k] = row16_sum(L[k]);
      if (i0 == 0 && r0 + 16 * k < rows) row_ml[r0 + 16 * k] = make_float2(M[k], 1.f / L[k]);
    }
  }
  __syncthreads();
  rows_f32x4 w = {0.f, 0.f, 0.f, 0.f};
  for (int r0 = wv; r0 < rows; r0 += 32) {
    rows_f32x4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] = rows_f32x4{0.f, 0.f, 0.f, 0.f};
      if (there && r0 + 4 * k < rows) v[k] = *reinterpret_cast<const rows_f32x4*>(x + (size_t)(r0 + 4 * k) * a.score_ld);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (r0 + 4 * k >= rows) break;
      const float2 ml = row_ml[r0 + 4 * k];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] += __builtin_amdgcn_exp2f(v[k][e] - ml.x) * ml.y;
    }
  }
  joined[wv][lane] = w;
  __syncthreads();
  if (wv != 0 || !there) return;
  w = ((w + joined[1][lane]) + joined[2][lane]) + joined[3][lane];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (pos + e < total) out[at + e] = before[e] + w[e];
}

// both in one launch: neither needs the other
template <int PARTS>
__global__ __launch_bounds__(256) void rows_merge_weights_kernel(RowsArgs a, int merge_blocks, const float* in, float* out, int64_t ld) {
  if ((int)blockIdx.x < merge_blocks) merge_row<PARTS>(a, blockIdx.x, blockIdx.y);
  else add_weights(a, (int)blockIdx.x - merge_blocks, blockIdx.y, in, out, ld);
}

// ---- host ---------------------------------------------------------------------------------------
// A prefix (or a sequence on its own) is cut into as many runs as there are workgroups at a time, two of eight waves or one of
// sixteen a CU (slots for 128 / 192 / 256 / 512 CUs: 32 sequences over 32768 positions 164 / 122 / 120 / 141 us, 8 over 8192
// 44.7 / 40.1 / 45.5 / 64); the length of the runs behind a prefix does not depend on the other sequences' lengths, so that a
// sequence's values do not either.
constexpr int kCus = 256;  // a constant: the calls that say how much workspace is needed have no context to ask

struct RowsPlan {
  RowsWindowArgs a;  // windowless calls pass the part that is theirs
  int tiles;   // of 16 query rows of a workgroup
  int items;
  size_t bytes;
};

// Pages of a run, whole steps of it, for `columns` workgroups side by side (kv heads x blocks of rows) and `others`
// workgroups behind them.  As many runs as there are workgroups at a time; or fewer, with room for one workgroup of each other,
// where that lengthens the runs by less than the others would take afterwards (some five steps: three before the first
// products and behind the last, two of their own).  Others that tail_run_of cuts more finely, or that have no room, take a second
// turn all the same: prefix / others / places of 16 sequences over 8192 positions 344 / 363 / 512, of 8 of 5 columns 176 / 135 / 256, of
// 32 of 64 query heads over 32768 256 / 256 / 256.  us with all / room for a workgroup a sequence and head: 16 sequences over
// 8192 positions, draft 33.1 / 30.0, 8 sequences of 5 columns 45.5 / 40.1; 32 sequences of 64 query heads over 32768 positions
// take the same run either way.
static int run_of(int64_t pages, int64_t columns, int64_t others, int tiles) {
  const int step = tiles == 16 ? 2 : 1;
  const int64_t slots = 2 / step * kCus;
  auto run = [&](int64_t places) {
    const int64_t runs = std::max<int64_t>(1, places / columns);
    return ((pages + runs - 1) / runs + step - 1) / step * step;
  };
  const int64_t all = run(slots);
  if (2 * others <= slots && all / step * others < 5 * (slots - others)) return (int)run(slots - others);
  return (int)all;
}

// Pages of a run of a sequence's own positions, behind the prefix; `columns` as above, of all sequences.  It depends on this
// sequence's length and on the numbers of the others.  A step where that leaves workgroups free, otherwise two, which share a start
// and an end; more where there are so many that all places are taken twice, up to four (or 32 runs); and no more than 64
// runs, a table of the merge's.  us, runs of two pages throughout / this: 2 sequences of 90 behind 703 positions 11.8 / 10.3; 32 of
// 1000 behind 2000 45.2 / 43.8; 8 of 16000 behind 1000 94 / 73; one of 9000 21.3 / 18.0, of 60000 98 / 65.
static int tail_run_of(int64_t pages, int64_t columns, int tiles) {
  const int step = tiles == 16 ? 2 : 1;
  const int64_t slots = 2 / step * kCus, steps = (pages + step - 1) / step;
  const int64_t least = std::max(steps, (int64_t)2) * columns >= slots ? 2 : 1, most = std::max<int64_t>(4, (steps + 31) / 32);
  return (int)std::max({least, std::min(most, steps * columns / (2 * slots)), (steps + 63) / 64}) * step;
}

static int64_t up256(int64_t b) { return (b + 255) / 256 * 256; }

// What a call will launch and need; Q, Knew, Vnew and O are left to the caller.
struct RowsWindow {
  int n_first, window;
};
static int plan_rows(const cas_kv* kv, int n_seqs, const int32_t* seqs, int prefix_len, const int32_t* ncols, int n_q_heads,
                     const int32_t* n_new, bool weights, RowsPlan* out, const RowsWindow* window = nullptr) {
  if (window && (window->n_first < 0 || window->window < 1)) return CAS_EINVAL;
  if (!kv || n_seqs < 1 || n_seqs > kRowsSeqs || !seqs || !ncols || !n_new || prefix_len < 0) return CAS_EINVAL;
  const KvGeom& g = kv->geom;
  if (n_q_heads < g.n_kv_heads || n_q_heads % g.n_kv_heads != 0) return CAS_EINVAL;
  RowsPlan p{};
  RowsWindowArgs& a = p.a;
  if (window) {
    a.n_first = std::min(window->n_first, 0x7FFFFFFF - 63);
    a.window = window->window;
  }
  a.g = g;
  a.n_q_heads = n_q_heads;
  a.grp = n_q_heads / g.n_kv_heads;
  if (a.grp > 48) return CAS_EINVAL;
  a.grp_inv = (65536u + (uint32_t)a.grp - 1u) / (uint32_t)a.grp;
  a.scale2 = (float)(1.4426950408889634 * 0.08838834764831845);
  a.n_seqs = n_seqs;
  a.prefix_pages = prefix_len / 64;
  int64_t rows = 0, parts = 0, items = 0;
  int most = 0, pages[kRowsSeqs];
  for (int i = 0; i < n_seqs; ++i) {
    if (seqs[i] < 0 || seqs[i] >= kv->desc.max_seqs) return CAS_EINVAL;
    for (int k = 0; k < i; ++k)
      if (seqs[k] == seqs[i]) return CAS_EINVAL;
    if (ncols[i] < 1 || ncols[i] > 16 || n_new[i] < ncols[i] || n_new[i] > 64) return CAS_EINVAL;
    a.seq[i] = seqs[i]; a.len[i] = kv->h_len[seqs[i]]; a.ncols[i] = ncols[i]; a.n_new[i] = n_new[i];
    if (prefix_len > a.len[i]) return CAS_EINVAL;
    if ((int64_t)a.len[i] + a.n_new[i] > kv_room(kv)) return CAS_ENOMEM;
    pages[i] = (a.len[i] + a.n_new[i] + 63) / 64;
    if (window) pages[i] -= WindowPages(a.n_first, a.window, a.len[i], a.len[i] + a.n_new[i], a.ncols[i]).skip;
    a.row0[i] = (int)rows;
    rows += ncols[i] * a.grp;
    most = std::max(most, ncols[i] * a.grp);
  }
  a.rows = (int)rows;
  if (a.prefix_pages > 0) most = a.rows;
  // Room for all rows of a decoded page, up to 256.  Smaller workgroups at the limits, us: 8 tiles above 128 rows 45 -> 62 (160
  // rows), 119 -> 147 (256); larger ones: 4 tiles above 16 rows 56 -> 62 (28 rows), 8 above 48 33 -> 36 (64).
  p.tiles = most <= 32 ? 2 : most <= 64 ? 4 : most <= 128 ? 8 : 16;
  const int block = 16 * p.tiles;
  if (a.prefix_pages > 0) {
    const int blocks = (a.rows + block - 1) / block;
    int64_t others = 0;
    for (int i = 0; i < n_seqs; ++i) others += (int64_t)g.n_kv_heads * ((ncols[i] * a.grp + block - 1) / block);
    a.prefix_run = run_of(a.prefix_pages, (int64_t)g.n_kv_heads * blocks, others, p.tiles);
    a.prefix_splits = (a.prefix_pages + a.prefix_run - 1) / a.prefix_run;
    a.prefix_items = a.prefix_splits * blocks;
  }
  for (int i = 0; i < n_seqs; ++i) {
    const int r = ncols[i] * a.grp;
    const int64_t tail = pages[i] - a.prefix_pages, blocks = (r + block - 1) / block;
    a.run[i] = weights || window ? run_of(tail, (int64_t)n_seqs * g.n_kv_heads * blocks, 0, p.tiles) : tail_run_of(tail, (int64_t)n_seqs * g.n_kv_heads * blocks, p.tiles);
    a.splits[i] = (int)((tail + a.run[i] - 1) / a.run[i]);
    a.item0[i] = (int)items;
    a.part0[i] = (uint32_t)parts;
    items += a.splits[i] * blocks;
    parts += (int64_t)a.splits[i] * g.n_kv_heads * r;
    if (items > 0x7FFFFFFF || parts > 0xFFFFFFFFll) return CAS_ENOTSUP;
  }
  for (int i = n_seqs; i < kRowsSeqs; ++i) a.row0[i] = a.item0[i] = 0x7FFFFFFF;
  const int64_t first = (int64_t)a.prefix_splits * g.n_kv_heads * a.rows;
  items += a.prefix_items;
  if (items * g.n_kv_heads > 0x3FFFFF) return CAS_ENOTSUP;  // a launch has fewer than 2^32 threads
  p.items = (int)items;
  // workspace: outputs, pairs, and the exponents of the rows
  int64_t off = up256((first + parts) * 512);
  const int64_t off_ml = off;
  off += up256((first + parts) * 8);
  const int64_t off_odd = off;
  off += up256((int64_t)n_seqs * g.n_kv_heads * 64);
  const int64_t off_score = off;
  if (weights) {
    a.score_ld = ((int64_t)a.len[0] + a.n_new[0] + 63) / 64 * 64;
    off += up256(a.score_ld * g.n_kv_heads * a.rows * 4);
  }
  if (window) {
    a.edge = (uint32_t*)(uintptr_t)off;
    off += up256((int64_t)n_seqs * g.n_kv_heads * 8);
  }
  p.bytes = (size_t)off;
  a.out_prefix = (float*)0;
  a.out_tail = (float*)(uintptr_t)(first * 512);
  a.ml_prefix = (float2*)(uintptr_t)off_ml;
  a.ml_tail = (float2*)(uintptr_t)(off_ml + first * 8);
  a.odd = (uint64_t*)(uintptr_t)off_odd;
  a.score = weights ? (float*)(uintptr_t)off_score : nullptr;
  *out = p;
  return CAS_OK;
}

static void place(RowsWindowArgs& a, void* ws) {  // offsets into the workspace become addresses
  char* b = (char*)ws;
  auto at = [&](auto*& p) { p = (std::remove_reference_t<decltype(p)>)(b + (uintptr_t)p); };
  at(a.out_prefix); at(a.out_tail); at(a.ml_prefix); at(a.ml_tail); at(a.odd);
  if (a.score) at(a.score);
  if (a.edge) at(a.edge);
}

template <class ARGS>
static int launch_partial_form(cas_ctx* ctx, const ARGS& a, int full, int tiles, int items) {
  return a.g.mx ? (full ? launch_rows_partial<true, true, ARGS>(ctx, a, tiles, items) : launch_rows_partial<false, true, ARGS>(ctx, a, tiles, items))
                : (full ? launch_rows_partial<true, false, ARGS>(ctx, a, tiles, items) : launch_rows_partial<false, false, ARGS>(ctx, a, tiles, items));
}

// weights: where the sums of a call for one sequence go
struct RowsWeights {
  const float* in;
  float* out;
  int64_t ld;
};
template <class ARGS = RowsArgs>
static int launch_rows(cas_ctx* ctx, cas_kv* kv, RowsPlan& p, int layer, int full, const RowsWeights* weights = nullptr) {
  if (!ctx->d_ws || !aligned256(ctx->d_ws) || p.bytes > ctx->ws_bytes) return ctx->d_ws && !aligned256(ctx->d_ws) ? CAS_EINVAL : CAS_ENOMEM;
  place(p.a, ctx->d_ws);
  p.a.full = full ? 1 : 0;
  ARGS& a = p.a;
  a.spec_pool = (const uint32_t*)kv->d_spec;
  a.verif_pool = (const uint32_t*)kv->d_verif;
  a.table = kv->d_page_table;
  a.layer = layer;
  const int rc = launch_partial_form<ARGS>(ctx, a, full, p.tiles, p.items);
  if (rc != CAS_OK) return rc;
  int most = 0;  // splits of a row: one wave can have 16 outputs in flight, so longer rows are shared by four
  for (int i = 0; i < a.n_seqs; ++i) most = std::max(most, a.prefix_splits + a.splits[i]);
  const int parts = most <= kMergeAhead ? 1 : 4, blocks = (a.rows * parts + 3) / 4;
  if (weights) {
    const dim3 grid(blocks + (a.len[0] + a.n_new[0] + kWeightsPos - 1) / kWeightsPos, a.g.n_kv_heads);
    hipLaunchKernelGGL(parts == 1 ? rows_merge_weights_kernel<1> : rows_merge_weights_kernel<4>, grid, dim3(256), 0, ctx->stream, a, blocks,
                       weights->in, weights->out, weights->ld);
  } else {
    hipLaunchKernelGGL((parts == 1 ? rows_merge_kernel<1, ARGS> : rows_merge_kernel<4, ARGS>), dim3(blocks, a.g.n_kv_heads), dim3(256), 0, ctx->stream, a);
  }
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

// The sequences' tensors; false if one is missing or not aligned
static bool take_tensors(RowsArgs& a, const uint16_t* const* Q, const uint16_t* const* Knew, const uint16_t* const* Vnew, uint16_t* const* O) {
  for (int i = 0; i < a.n_seqs; ++i) {
    a.Q[i] = Q[i]; a.Knew[i] = Knew[i]; a.Vnew[i] = Vnew[i]; a.O[i] = O[i];
    for (const void* d : {(const void*)Q[i], (const void*)Knew[i], (const void*)Vnew[i], (const void*)O[i]})
      if (!d || !aligned256(d)) return false;
  }
  return true;
}

}  // namespace cas

extern "C" {

int cas_attention_shared(cas_ctx* ctx, cas_kv* kv, int layer, int n_seqs, const int32_t* h_seqs, int prefix_len, int full,
                         const uint16_t* const* h_d_Q, const int32_t* h_ncols, int n_q_heads,
                         const uint16_t* const* h_d_Knew, const uint16_t* const* h_d_Vnew, const int32_t* h_n_new,
                         uint16_t* const* h_d_O) {
  if (!ctx || !kv || layer < 0 || layer >= kv->desc.n_layers || !h_d_Q || !h_d_Knew || !h_d_Vnew || !h_d_O) return CAS_EINVAL;
  cas::RowsPlan p;
  const int rc = cas::plan_rows(kv, n_seqs, h_seqs, prefix_len, h_ncols, n_q_heads, h_n_new, false, &p);
  if (rc != CAS_OK) return rc;
  if (!cas::take_tensors(p.a, h_d_Q, h_d_Knew, h_d_Vnew, h_d_O) || !cas::on_device(ctx)) return CAS_EINVAL;
  return cas::launch_rows(ctx, kv, p, layer, full);
}

size_t cas_attention_shared_bytes(const cas_kv* kv, int n_seqs, const int32_t* h_seqs, int prefix_len, const int32_t* h_ncols,
                                  int n_q_heads, const int32_t* h_n_new) {
  cas::RowsPlan p;
  return cas::plan_rows(kv, n_seqs, h_seqs, prefix_len, h_ncols, n_q_heads, h_n_new, false, &p) == CAS_OK ? p.bytes : 0;
}

int cas_attention_weights(cas_ctx* ctx, cas_kv* kv, int layer, int seq, int full, const uint16_t* d_Q, int ncols, int n_q_heads,
                          const uint16_t* d_Knew, const uint16_t* d_Vnew, int n_new, uint16_t* d_O, const float* d_score_in,
                          float* d_score_out, int64_t ld) {
  if (!ctx || !kv || layer < 0 || layer >= kv->desc.n_layers || !d_Q || !d_Knew || !d_Vnew || !d_O || !d_score_out) return CAS_EINVAL;
  cas::RowsPlan p;
  const int rc = cas::plan_rows(kv, 1, &seq, 0, &ncols, n_q_heads, &n_new, true, &p);
  if (rc != CAS_OK) return rc;
  const int total = p.a.len[0] + n_new;
  if (ld < total) return CAS_EINVAL;
  if (!cas::aligned256(d_Q) || !cas::aligned256(d_Knew) || !cas::aligned256(d_Vnew) || !cas::aligned256(d_O)) return CAS_EINVAL;
  if (!cas::on_device(ctx)) return CAS_EINVAL;
  p.a.Q[0] = d_Q; p.a.Knew[0] = d_Knew; p.a.Vnew[0] = d_Vnew; p.a.O[0] = d_O;
  const cas::RowsWeights w{d_score_in, d_score_out, ld};
  return cas::launch_rows(ctx, kv, p, layer, full, &w);
}

size_t cas_attention_weights_bytes(const cas_kv* kv, int seq, int ncols, int n_q_heads, int n_new) {
  cas::RowsPlan p;
  return cas::plan_rows(kv, 1, &seq, 0, &ncols, n_q_heads, &n_new, true, &p) == CAS_OK ? p.bytes : 0;
}

int cas_attention_window(cas_ctx* ctx, cas_kv* kv, int layer, int n_seqs, const int32_t* h_seqs, int n_first, int window, int full,
                         const uint16_t* const* h_d_Q, const int32_t* h_ncols, int n_q_heads, const uint16_t* const* h_d_Knew,
                         const uint16_t* const* h_d_Vnew, const int32_t* h_n_new, uint16_t* const* h_d_O) {
  if (!ctx || !kv || layer < 0 || layer >= kv->desc.n_layers || !h_d_Q || !h_d_Knew || !h_d_Vnew || !h_d_O) return CAS_EINVAL;
  cas::RowsPlan p;
  const cas::RowsWindow w{n_first, window};
  const int rc = cas::plan_rows(kv, n_seqs, h_seqs, 0, h_ncols, n_q_heads, h_n_new, false, &p, &w);
  if (rc != CAS_OK) return rc;
  if (!cas::take_tensors(p.a, h_d_Q, h_d_Knew, h_d_Vnew, h_d_O) || !cas::on_device(ctx)) return CAS_EINVAL;
  return cas::launch_rows<cas::RowsWindowArgs>(ctx, kv, p, layer, full);
}

size_t cas_attention_window_bytes(const cas_kv* kv, int n_seqs, const int32_t* h_seqs, int n_first, int window, const int32_t* h_ncols,
                                  int n_q_heads, const int32_t* h_n_new) {
  cas::RowsPlan p;
  const cas::RowsWindow w{n_first, window};
  return cas::plan_rows(kv, n_seqs, h_seqs, 0, h_ncols, n_q_heads, h_n_new, false, &p, &w) == CAS_OK ? p.bytes : 0;
}

}  // extern "C"
