// Partial attention over runs of pages for the query rows of one or several sequences, compiled in a translation unit per
// form of the cache; attention_rows.hip explains the algorithm.
#pragma once
#include "cas_device.hpp"
#include "cas_internal.hpp"

namespace cas {

typedef short rows_s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 rows_bf16x8 __attribute__((ext_vector_type(8)));
typedef float rows_f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int rows_u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRowsSeqs = 32;      // sequences of a launch
constexpr float kLowest = -3.402823466e38f;

// Kernel arguments lie in host memory: what a workgroup looks for in them is found by scalar loads at fixed places (which_of,
// query_of), since a loop of dependent loads, or a load per lane, crosses the bus every time (11 of the 27 us that 16
// sequences took over a prefix of 8192 positions).
struct RowsArgs {
  KvGeom g;
  const uint32_t* spec_pool;
  const uint32_t* verif_pool;
  const int32_t* table;
  int layer, n_q_heads, grp;
  uint32_t grp_inv;          // row / grp = row * grp_inv >> 16
  float scale2;              // log2(e) / sqrt(128): scores are kept as exponents of two
  int n_seqs, rows;          // rows: of all sequences
  int prefix_pages, prefix_run, prefix_splits, tail_run;
  // partial results: 128 outputs each, [split][kv head][row] of the prefix, then the same sequence by sequence; and the
  // pairs (maximum, sum) in the same two regions as [kv head][row][split]
  float* out_prefix;
  float* out_tail;
  float2* ml_prefix;
  float2* ml_tail;
  float* score;              // NULL or [kv head][row][score_ld]: exponents of every position behind the prefix
  int64_t score_ld;
  // the sequences
  int row0[kRowsSeqs];       // query rows (columns x group) of the sequences before; the largest number behind the last
  int item0[kRowsSeqs];      // work items behind the prefix, of the sequences before; as above
  const uint16_t* Q[kRowsSeqs];
  const uint16_t* Knew[kRowsSeqs];
  const uint16_t* Vnew[kRowsSeqs];
  uint16_t* O[kRowsSeqs];
  int seq[kRowsSeqs], len[kRowsSeqs], n_new[kRowsSeqs], ncols[kRowsSeqs];
  int splits[kRowsSeqs];     // runs of pages behind the prefix
  uint32_t part0[kRowsSeqs]; // partial results (row, run, kv head) behind the prefix, of the sequences before
};

// the sequence whose share of first[] holds n
__device__ __forceinline__ int which_of(const int (&first)[kRowsSeqs], int n) {
  int s = 0;
#pragma unroll
  for (int i = 1; i < kRowsSeqs; ++i) s += n >= first[i] ? 1 : 0;
  return s;
}

// K and V of a wave's 16 tokens in LDS as in attention_kernel.inl: [1 + 32 positions][64 values], for K the four words of a
// token at one position side by side, for V the tokens of a word; row 0 takes what lanes without a value left write.
constexpr int kRowsPos = 64;
constexpr int kRowsSlab = 33 * kRowsPos;

// Maximum / sum over the four lanes that hold one query row (lanes 16 apart)
__device__ __forceinline__ float over_groups_max(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float over_groups_sum(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Product kk of a page takes 8 positions of the four words; lane group mq takes two of them, two apart, so that the 32 lanes
// which the LDS serves at once read places that follow one another (its 64 banks hold two positions).
__device__ __forceinline__ int k_position(int kk, int mq) { return 8 * kk + (mq & 1) + 4 * (mq >> 1); }
__device__ __forceinline__ rows_bf16x8 k_fragment(const uint16_t* slab, int kk, int mi, int mq) {
  const uint16_t* src = slab + (1 + k_position(kk, mq)) * kRowsPos + 4 * mi;
  const uint2 k0 = *reinterpret_cast<const uint2*>(src), k1 = *reinterpret_cast<const uint2*>(src + 2 * kRowsPos);
  return __builtin_bit_cast(rows_bf16x8, rows_u32x4{k0.x, k0.y, k1.x, k1.y});
}
// The queries go through LDS, [row][position][word]: a load per lane of its own row takes an address unit some 20 ns, and a
// wave needs 16 of them (16 waves: 5 us).  Sixteen threads to a row, two positions of the four words each; rows that are
// not there are zeros.
constexpr int kQueryPitch = 136;
struct QueryPart {
  uint32_t w[4];
  __device__ __forceinline__ void load(const uint16_t* row, int i) {  // row = NULL: zeros
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = row ? *reinterpret_cast<const uint32_t*>(row + 32 * k + 2 * i) : 0u;
  }
  __device__ __forceinline__ void store(uint16_t* row, int i) const {
    auto low = [](uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x05040100u); };
    auto high = [](uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); };
    *reinterpret_cast<uint4*>(row + 8 * i) = make_uint4(low(w[0], w[1]), low(w[2], w[3]), high(w[0], w[1]), high(w[2], w[3]));
  }
};
// the values of a row that product kk takes
__device__ __forceinline__ rows_bf16x8 q_fragment(const uint16_t* row, int kk, int mq) {
  const uint16_t* src = row + 4 * k_position(kk, mq);
  const uint2 q0 = *reinterpret_cast<const uint2*>(src), q1 = *reinterpret_cast<const uint2*>(src + 8);
  return __builtin_bit_cast(rows_bf16x8, rows_u32x4{q0.x, q0.y, q1.x, q1.y});
}

// A workgroup: one kv head, one run of pages, up to 16 NT query rows.  Wave w owns tokens 16 w .. 16 w + 15 of every page,
// from their streams to its own running maxima, sums and outputs: the page loop has no barrier, and the four waves' results
// are joined at its end.  Products are formed as K Q^T and V^T P^T, so that a query row is a column of the result: the
// probabilities leave the first product where the second wants them (lane group q holds tokens 4 q .. 4 q + 3, which are
// its share of the second's inner index), and a row's factors are one value per lane.
template <int T, bool FULL, bool MX, int NT>
__global__ __launch_bounds__(256, NT > 1 ? 2 : FULL ? 3 : 4) void attn_rows_kernel(RowsArgs a) {
  __shared__ __align__(16) uint16_t tile[4 * kRowsSlab];
  __shared__ float red[2][4][NT * 16];
  const KvGeom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = (int)blockIdx.x % g.n_kv_heads;  // heads next to each other: workgroups that share pages share an XCD's L2
  int item = (int)blockIdx.x / g.n_kv_heads;
  const int r = tid >> 2, j = tid & 3;       // decode role: token r of the page, word j
  const int mi = lane & 15, mq = lane >> 4;  // role in the products: query row (token, channel) mi, group mq
  uint16_t* const slab = tile + wv * kRowsSlab;
  uint16_t* const kcol = slab + kRowsPos + (r & 15) * 4 + j;   // position 0 of the thread's token and word
  uint16_t* const vcol = slab + kRowsPos + j * 16 + (r & 15);

  // ---- what this workgroup works on (uniform)
  const int si = which_of(a.item0, item);
  struct {
    const uint16_t *Q, *Knew, *Vnew;
    int len, n_new, ncols, splits, item0;
    uint32_t part0;
  } const me = {a.Q[si], a.Knew[si], a.Vnew[si], a.len[si], a.n_new[si], a.ncols[si], a.splits[si], a.item0[si], a.part0[si]};
  item -= me.item0;
  const int rows = me.ncols * a.grp, blocks = (rows + 16 * NT - 1) / (16 * NT);
  const int split = item / blocks, row_base = (item - split * blocks) * 16 * NT;
  const int len = me.len, total = me.len + me.n_new;
  const int pg0 = a.prefix_pages + split * a.tail_run, pg1 = min(pg0 + a.tail_run, (total + 63) / 64);
  const int32_t* page_row = a.table + (size_t)a.seq[si] * g.max_pages_per_seq;

  // Pool pages two pages ahead, bitmap words one page ahead: a page's own round trip is that of its windows alone.  The pools
  // are touched only for pages that hold committed positions.
  auto page_of = [&](int pg) { return pg < pg1 && pg * 64 < len ? min(max(page_row[pg], 0), g.n_pages - 1) : 0; };
  auto tile_of = [&](int page) { return (((size_t)a.layer * g.n_pages + page) * 2) * g.n_kv_heads + head; };
  uint32_t next_k = 0, next_v = 0, next_ek = 0, next_ev = 0;
  auto request_masks = [&](int pg, int page) {
    next_k = next_v = next_ek = next_ev = 0;
    if (pg < pg1 && pg * 64 + r < len) {
      const uint32_t* ks = a.spec_pool + tile_of(page) * g.tile_spec_words;
      const uint32_t* vs = ks + (size_t)g.n_kv_heads * g.tile_spec_words;
      next_k = ks[r * 4 + j];
      next_v = vs[r * 4 + j];
      if constexpr (MX) {
        next_ek = ks[64 * 4 + r];
        next_ev = vs[64 * 4 + r];
      }
    }
  };
  int page_next = page_of(pg0), page_after = page_of(pg0 + 1);
  request_masks(pg0, page_next);

  // ---- queries
  rows_bf16x8 q[NT][4];
  int seen[NT];  // last position that the row sees
  static_assert(16 * NT * kQueryPitch <= 4 * kRowsSlab, "");
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int rr = row_base + nt * 16 + (tid >> 4), c = (int)((uint32_t)rr * a.grp_inv >> 16), gi = rr - c * a.grp;
    QueryPart part;
    part.load(rr < rows ? me.Q + ((size_t)c * a.n_q_heads + head * a.grp + gi) * 128 : nullptr, tid & 15);
    part.store(tile + (nt * 16 + (tid >> 4)) * kQueryPitch, tid & 15);
    seen[nt] = total - me.ncols + (int)((uint32_t)(row_base + nt * 16 + mi) * a.grp_inv >> 16);
  }
  __syncthreads();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) q[nt][kk] = q_fragment(tile + (nt * 16 + mi) * kQueryPitch, kk, mq);
  }
  __syncthreads();  // the tile is free

  rows_f32x4 o[NT][8];
  float m[NT], l[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = kLowest;
    l[nt] = 0.f;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) o[nt][ct] = rows_f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto word_prefix = [&](uint32_t mask) -> uint32_t {  // kept values of the token before word j
    const int cnt = __popc(mask);
    const int b0 = quad_dpp<0x00>(cnt), b1 = quad_dpp<0x55>(cnt), b2 = quad_dpp<0xAA>(cnt);
    return (uint32_t)((j > 0 ? b0 : 0) + (j > 1 ? b1 : 0) + (j > 2 ? b2 : 0));
  };
  // word j of an uncompressed vector, eight values at a time
  auto copy_fresh = [&](const uint16_t* v, int slot, uint16_t* to, auto&& value) {
    const uint4* src = reinterpret_cast<const uint4*>(v + ((size_t)slot * g.n_kv_heads + head) * 128 + 32 * j);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 x = src[i];
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int c = 0; c < 8; ++c) to[(8 * i + c) * kRowsPos] = value((uint16_t)(w[c >> 1] >> (16 * (c & 1))));
      asm volatile("" ::: "memory");
    }
  };
  auto ordered = [&]() {  // LDS writes of the wave before its reads, and the other way round
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };

  for (int pg = pg0; pg < pg1; ++pg) {
    const int tok0 = pg * 64, pos = tok0 + r;
    const bool has_live = tok0 < len, live = pos < len, fresh = !live && pos < total;
    // ---- streams of the thread's word of K and V
    const uint32_t mk = taken(next_k), mv = taken(next_v);
    int ek = 0, ev = 0;
    if constexpr (MX) {
      ek = (int)((taken(next_ek) >> (8 * j)) & 0xFFu);
      ev = (int)((taken(next_ev) >> (8 * j)) & 0xFFu);
    }
    const size_t tk = tile_of(page_next), tv = tk + g.n_kv_heads;
    page_next = page_after;
    page_after = page_of(pg + 2);
    WordWindows<T, FULL, MX> wk, wvw;
    auto load = [&](WordWindows<T, FULL, MX>& w, uint32_t mask, size_t t) {
      const uint32_t p = word_prefix(mask);
      const uint32_t* sp = a.spec_pool + t * g.tile_spec_words;
      const uint32_t* vf = a.verif_pool + t * g.tile_verif_words;
      if (has_live) w.load(p, 32u * j - p, sp + g.spec_off + r * g.sw, vf + r * g.lw, vf + 64 * g.lw + r * g.pw);
    };
    load(wk, mk, tk);
    if constexpr (!FULL) load(wvw, mv, tv);
    request_masks(pg + 1, page_next);
    // the exact form writes all channels of a page of committed tokens; otherwise what is not written has to read as 0
    const bool clear = !FULL || tok0 + 64 > len;
    auto clear_slab = [&]() {
#pragma unroll
      for (int k = 0; k < 4; ++k) reinterpret_cast<uint4*>(slab + kRowsPos)[lane + 64 * k] = make_uint4(0, 0, 0, 0);
    };
    if (clear) {
      clear_slab();
      ordered();
    }
    // ---- K: this thread's 32 channels of its token
    if (fresh) copy_fresh(me.Knew, pos - me.len, kcol, [](uint16_t v) { return v; });
    wk.k.decode(mk, [&](int bp, uint16_t v) { kcol[bp * kRowsPos] = v; }, ek);
    if constexpr (FULL) wk.pr.decode(live ? ~mk : 0u, [&](int bp, uint16_t v) { kcol[bp * kRowsPos] = v; });
    if constexpr (FULL) load(wvw, mv, tv);
    ordered();
    // ---- exponents of the wave's 16 tokens: lane (mi, mq) holds tokens 4 mq + e of row mi
    rows_f32x4 x[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) x[nt] = rows_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const rows_bf16x8 kf = k_fragment(slab, kk, mi, mq);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) x[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[nt][kk], x[nt], 0, 0, 0);
    }
    ordered();  // K has been read: its place may be written
    const int t0 = tok0 + 16 * wv + 4 * mq;
    rows_s16x4 p[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[nt][e] = t0 + e <= seen[nt] ? x[nt][e] * a.scale2 : -INFINITY;
      if (a.score != nullptr && row_base + nt * 16 + mi < rows)
        *reinterpret_cast<rows_f32x4*>(a.score + ((size_t)head * rows + row_base + nt * 16 + mi) * a.score_ld + t0) = x[nt];
      // at least the lowest finite number: where a row sees nothing of these tokens, the maximum is -inf as its scores are
      const float mx = over_groups_max(fmaxf(fmaxf(x[nt][0], x[nt][1]), fmaxf(x[nt][2], x[nt][3])));
      const float top = fmaxf(m[nt], mx);
      if (__builtin_amdgcn_ballot_w64(top > m[nt])) {  // a factor of 1 for all rows otherwise
        const float f = __builtin_amdgcn_exp2f(m[nt] - top);
        l[nt] *= f;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) o[nt][ct] *= f;
        m[nt] = top;
      }
      uint32_t h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // the sum takes the weight as it is (sums of weights per position are fp32 results), the product takes it rounded
        // to bf16: an output is off by at most 2^-8 of the weighted mean of |v|, some 2^-9 / sqrt(positions) of it in
        // fact, where the output's own rounding is 2^-8 of it
        const float w = __builtin_amdgcn_exp2f(x[nt][e] - top);
        l[nt] += w;
        h[e] = f32_to_bf16(w);
      }
      p[nt] = __builtin_bit_cast(rows_s16x4, make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16));
    }
    // ---- V over K
    if (clear) {
      clear_slab();
      ordered();
    }
    bool odd = false;  // an infinity or a NaN: times 0 it would reach rows that do not see the vector, so it is added below
    if (fresh) {
      copy_fresh(me.Vnew, pos - me.len, vcol, [&](uint16_t v) {
        const bool inf = (v & 0x7F80u) == 0x7F80u;
        odd |= inf;
        return inf ? (uint16_t)0 : v;
      });
    }
    const uint64_t odd_lanes = __builtin_amdgcn_ballot_w64(odd);
    wvw.k.decode(mv, [&](int bp, uint16_t v) { vcol[bp * kRowsPos] = v; }, ev);
    if constexpr (FULL) wvw.pr.decode(live ? ~mv : 0u, [&](int bp, uint16_t v) { vcol[bp * kRowsPos] = v; });
    ordered();
    // ---- outputs: lane (mi, mq) holds channels 32 mq + 4 ct + e of row mi
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      const rows_s16x4 vf = *reinterpret_cast<const rows_s16x4*>(slab + (1 + 4 * ct + (mi & 3)) * kRowsPos + (mi >> 2) * 16 + 4 * mq);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) o[nt][ct] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vf, p[nt], o[nt][ct], 0, 0, 0);
    }
    ordered();  // V has been read
    if (odd_lanes != 0) {  // tokens with infinities or NaN in flight, for the rows that see them; four channels at a time
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint2 pw = __builtin_bit_cast(uint2, p[nt]);
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) {
          for (uint64_t left = odd_lanes; left != 0;) {
            const int tt = __builtin_ctzll(left) >> 2, t = tok0 + 16 * wv + tt;
            left &= ~(0xFull << (4 * tt));
            const uint32_t half = tt & 2 ? pw.y : pw.x;
            const float pt = __shfl(__uint_as_float(tt & 1 ? half & 0xFFFF0000u : half << 16), mi + 16 * (tt >> 2));
            const uint2 two = *reinterpret_cast<const uint2*>(
                me.Vnew + ((size_t)(t - me.len) * g.n_kv_heads + head) * 128 + 32 * mq + 4 * ct);
            const uint32_t v[4] = {two.x << 16, two.x & 0xFFFF0000u, two.y << 16, two.y & 0xFFFF0000u};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if ((v[e] & 0x7F800000u) == 0x7F800000u && t <= seen[nt]) o[nt][ct][e] += pt * __uint_as_float(v[e]);
          }
        }
      }
    }
  }

  // ---- the four waves' results: to the maximum of all, then 2 + 0, 3 + 1, (3 + 1) + (2 + 0) through the tiles' place
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    l[nt] = over_groups_sum(l[nt]);
    if (mq == 0) {
      red[0][wv][nt * 16 + mi] = m[nt];
      red[1][wv][nt * 16 + mi] = l[nt];
    }
  }
  __syncthreads();
  float* const stage = reinterpret_cast<float*>(tile);  // two rows of waves: [2][16 rows][128] floats, 16 KB of 16.5
  float sum[NT], top[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int i = nt * 16 + mi;
    top[nt] = fmaxf(fmaxf(red[0][0][i], red[0][1][i]), fmaxf(red[0][2][i], red[0][3][i]));
    sum[nt] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) sum[nt] += red[1][w][i] * __builtin_amdgcn_exp2f(red[0][w][i] - top[nt]);
    const float f = __builtin_amdgcn_exp2f(m[nt] - top[nt]);
    rows_f32x4* const mine = reinterpret_cast<rows_f32x4*>(stage + (wv & 1) * 2048) + lane;  // [8][64 lanes] of four values
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) o[nt][ct] *= f;
    if (wv >= 2) {
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) mine[64 * ct] = o[nt][ct];
    }
    __syncthreads();
    if (wv < 2) {
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) o[nt][ct] += mine[64 * ct];
    }
    __syncthreads();
    if (wv == 1) {
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) mine[64 * ct] = o[nt][ct];
    }
    __syncthreads();
    if (wv == 0) {
      const rows_f32x4* const other = reinterpret_cast<const rows_f32x4*>(stage + 2048) + lane;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) o[nt][ct] += other[64 * ct];
    }
    __syncthreads();
  }
  if (wv != 0) return;
  float* const out = a.out_tail + ((size_t)me.part0 + ((size_t)split * g.n_kv_heads + head) * rows) * 128;
  float2* const ml = a.ml_tail + me.part0;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int rr = row_base + nt * 16 + mi;
    if (rr >= rows) continue;
    rows_f32x4* const dst = reinterpret_cast<rows_f32x4*>(out + (size_t)rr * 128 + 32 * mq);
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) dst[ct] = o[nt][ct];
    if (mq == 0) ml[((size_t)head * rows + rr) * me.splits + split] = make_float2(top[nt], sum[nt]);
  }
}

// LDS writes at base + i * pitch bytes with the address in one operation (the compiler's code takes two)
typedef __attribute__((address_space(3))) uint16_t lds_u16;
__device__ __forceinline__ uint32_t lds_address(uint16_t* p) { return (uint32_t)(uintptr_t)(lds_u16*)p; }
__device__ __forceinline__ void lds_write(uint32_t base, int i, int pitch, uint16_t v) {
  uint32_t at;
  asm("v_mad_i32_i24 %0, %1, %2, %3" : "=v"(at) : "v"(i), "s"(pitch), "v"(base));
  *(lds_u16*)(uintptr_t)at = v;
}

// The whole pages of a prefix, for up to 16 RT query rows of all sequences.  Sixteen waves, the most that a CU holds at 128
// registers, take two pages a step: each decodes 16 tokens of K or of V of one of them into a tile that all read, and forms
// the products of 16 rows with both pages (RT = 16), with one (8), or with half (4) or a quarter (2) of one.  There are two
// sets of tiles: a step's products, the decode of the next and the loads of the one after it are between the same two
// barriers.  The waves of a row are joined at the end.
//
// With many rows the reads of the tiles are what the LDS is busy with, and 16 lanes are served at once.  K: as above, with
// slabs 32 bytes off each other, so that a product's 16 tokens may be four of every eight of two slabs: lane group mq then
// holds the weights of eight tokens that follow one another.  V: eight tokens of a channel in one read; the 8 lanes served
// at once take two positions of the four words, and positions lie 144 bytes apart, so that these do not meet.  (128 apart, with
// reads of four tokens, four lanes met in every bank: 104 of the 286 thousand cycles that a CU was busy with 256 rows over
// 32768 positions.)  The walks' writes meet more often for it (some 4 lanes in place of 2), which is less.
constexpr int kPrefixWaves = 16;
constexpr int kVPos = 72;                                   // values from a position of V to the next
constexpr int kKSlab = 33 * kRowsPos + 16, kVSlab = 33 * kVPos;
constexpr int kPrefixPage = 4 * (kKSlab + kVSlab);          // [K, V][slab]
constexpr int kPrefixSet = 2 * kPrefixPage;
constexpr int kStageCt = 65;                                // values of four of a group of channels (64 lanes), padded
constexpr size_t kPrefixLds = sizeof(uint16_t) * 2 * kPrefixSet;    // 141 KB; the joining of 16 waves needs 130
static_assert(sizeof(float) * 4 * kStageCt * 8 * kPrefixWaves <= kPrefixLds, "");

template <int T, bool FULL, bool MX, int RT>
__global__ __launch_bounds__(64 * kPrefixWaves) void attn_prefix_kernel(RowsArgs a) {
  extern __shared__ __align__(16) uint16_t tiles[];
  __shared__ float red[2][kPrefixWaves][16];
  constexpr int NS = RT >= 8 ? 4 : RT / 2;  // slabs of 16 tokens that a wave's products take of a page
  const KvGeom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = (int)blockIdx.x % g.n_kv_heads, item = (int)blockIdx.x / g.n_kv_heads;
  const int slot = wv >> 3, u = wv & 7;                // page of the step, place among its waves
  const int kv = u >> 2, r = (u & 3) * 16 + (lane >> 2), j = lane & 3;  // decode role: K or V, token, word
  const int mi = lane & 15, mq = lane >> 4;
  const int tile = RT == 16 ? wv : u % RT, slab0 = RT >= 8 ? 0 : (u / RT) * NS;   // role in the products
  const int blocks = (a.rows + 16 * RT - 1) / (16 * RT), split = item / blocks, row_base = (item - split * blocks) * 16 * RT;
  const int pg0 = split * a.prefix_run, pg1 = min(pg0 + a.prefix_run, a.prefix_pages), steps = (pg1 - pg0 + 1) / 2;
  const int32_t* page_row = a.table + (size_t)a.seq[0] * g.max_pages_per_seq;
  // where the thread's word begins in a set, and what a position adds
  const int col = slot * kPrefixPage + (kv ? 4 * kKSlab + (u & 3) * kVSlab + kVPos + j * 16 + (lane >> 2)
                                           : (u & 3) * kKSlab + kRowsPos + (lane >> 2) * 4 + j);
  const int pitch = 2 * (kv ? kVPos : kRowsPos);  // bytes

  // ---- the wave's unit of a step: pool pages two steps ahead, bitmap words one, fields as soon as those are there
  auto page_of = [&](int step) {
    const int pg = pg0 + 2 * step + slot;
    return pg < pg1 ? min(max(page_row[pg], 0), g.n_pages - 1) : -1;
  };
  auto tile_of = [&](int page) { return (((size_t)a.layer * g.n_pages + page) * 2 + kv) * g.n_kv_heads + head; };
  uint32_t next_mask = 0, next_exp = 0;
  auto request_mask = [&](int page) {
    if (page < 0) return;
    const uint32_t* sp = a.spec_pool + tile_of(page) * g.tile_spec_words;
    next_mask = sp[r * 4 + j];
    if constexpr (MX) next_exp = sp[64 * 4 + r];
  };
  // the exact form with many rows has no registers for all fields during the products: those of the values that were not
  // kept are requested behind them, under the decode of the kept ones
  constexpr bool kLate = RT >= 4;
  WordWindows<T, FULL, MX> win;
  uint32_t mask = 0, pruned_at = 0;
  const uint32_t* pruned_row = nullptr;
  int shared_exp = 0;
  auto request_fields = [&](int page) {
    if (page < 0) return;
    mask = taken(next_mask);
    if constexpr (MX) shared_exp = (int)((taken(next_exp) >> (8 * j)) & 0xFFu);
    const int cnt = __popc(mask);
    const int b0 = quad_dpp<0x00>(cnt), b1 = quad_dpp<0x55>(cnt), b2 = quad_dpp<0xAA>(cnt);
    const uint32_t p = (uint32_t)((j > 0 ? b0 : 0) + (j > 1 ? b1 : 0) + (j > 2 ? b2 : 0));
    const size_t t = tile_of(page);
    const uint32_t* sp = a.spec_pool + t * g.tile_spec_words;
    const uint32_t* vf = a.verif_pool + t * g.tile_verif_words;
    win.k.load(p, sp + g.spec_off + r * g.sw, vf + r * g.lw);
    pruned_row = vf + 64 * g.lw + r * g.pw;
    pruned_at = 32u * j - p;
    if constexpr (FULL && !kLate) win.pr.load(pruned_at, pruned_row);
  };
  auto decode = [&](int set) {
    const uint32_t to = lds_address(tiles + set * kPrefixSet + col);
    if constexpr (!FULL) {  // what is not written has to read as 0: 512 or 576 groups of eight values
      uint16_t* const slab = tiles + set * kPrefixSet + slot * kPrefixPage + (kv ? 4 * kKSlab + (u & 3) * kVSlab + kVPos
                                                                                 : (u & 3) * kKSlab + kRowsPos);
#pragma unroll
      for (int k = 0; k < 4; ++k) reinterpret_cast<uint4*>(slab)[lane + 64 * k] = make_uint4(0, 0, 0, 0);
      if (kv && lane < 32) reinterpret_cast<uint4*>(slab)[lane + 256] = make_uint4(0, 0, 0, 0);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    if constexpr (FULL && kLate) win.pr.load(pruned_at, pruned_row);
    win.k.decode(mask, [&](int bp, uint16_t v) { lds_write(to, bp, pitch, v); }, shared_exp);
    if constexpr (FULL) win.pr.decode(~mask, [&](int bp, uint16_t v) { lds_write(to, bp, pitch, v); });
  };
  int page_a = page_of(0), page_b = page_of(1);
  request_mask(page_a);

  // ---- queries, through the second set of tiles, which the decode of the second step is the first to write
  rows_bf16x8 q[4];
  {
    static_assert(16 * RT * kQueryPitch <= kPrefixSet, "");
    constexpr int kParts = (RT * 256 + 64 * kPrefixWaves - 1) / (64 * kPrefixWaves);
    uint16_t* const stage = tiles + kPrefixSet;
    QueryPart part[kParts];
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const int i = tid + k * 64 * kPrefixWaves;
      int rr = row_base + (i >> 4), first = 0;
      const bool there = rr < a.rows && i < RT * 256;
      const uint16_t* src = a.Q[0];
#pragma unroll
      for (int s = 1; s < kRowsSeqs; ++s) {
        const bool in = rr >= a.row0[s];
        first = in ? a.row0[s] : first;
        src = in ? a.Q[s] : src;
      }
      rr -= first;
      const int c = (int)((uint32_t)rr * a.grp_inv >> 16), gi = rr - c * a.grp;
      part[k].load(there ? src + ((size_t)c * a.n_q_heads + head * a.grp + gi) * 128 : nullptr, i & 15);
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const int i = tid + k * 64 * kPrefixWaves;
      if (i < RT * 256) part[k].store(stage + (i >> 4) * kQueryPitch, i & 15);
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) q[kk] = q_fragment(stage + (tile * 16 + mi) * kQueryPitch, kk, mq);
  }
  rows_f32x4 o[8];
  float m = kLowest, l = 0.f;
#pragma unroll
  for (int ct = 0; ct < 8; ++ct) o[ct] = rows_f32x4{0.f, 0.f, 0.f, 0.f};

  // places of the lane's reads in a page: K, tokens of the two parities of a product; V, channels 32 w + f of the four words w,
  // f = 8 (mi / 4) + (ct ^ (mi / 4 & 1)), which lie in different halves of the banks
  const int kq = NS == 1 ? slab0 * kKSlab + 4 * mi : (2 * (slab0 >> 1) + (mi >> 3)) * kKSlab + ((mi >> 2) & 1) * 32 + (mi & 3) * 4;
  const int vq = 4 * kKSlab + (NS == 1 ? slab0 * kVSlab + 4 * mq : (2 * (slab0 >> 1) + (mq >> 1)) * kVSlab + 8 * (mq & 1)) +
                 (1 + 8 * (mi >> 2)) * kVPos + (mi & 3) * 16;
  const int odd = (mi >> 2) & 1 ? kVPos : 0;
  auto products = [&](int set, int page, int pg) {
    const uint16_t* const at = tiles + set * kPrefixSet + page * kPrefixPage;
    // exponents: lane (mi, mq) holds four tokens of row mi a product, tt: 4 mq + e of the slab (NS = 1), or
    // 32 (tt / 2) + 8 mq + 4 (tt & 1) + e
    rows_f32x4 x[NS];
#pragma unroll
    for (int tt = 0; tt < NS; ++tt) {
      x[tt] = rows_f32x4{0.f, 0.f, 0.f, 0.f};
      asm volatile("" ::: "memory");  // the reads of one product at a time: those of all do not fit the registers
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const uint16_t* src = at + kq + (tt >> 1) * 2 * kKSlab + (tt & 1) * 16 + (1 + k_position(kk, mq)) * kRowsPos;
        const uint2 k0 = *reinterpret_cast<const uint2*>(src), k1 = *reinterpret_cast<const uint2*>(src + 2 * kRowsPos);
        x[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(rows_bf16x8, rows_u32x4{k0.x, k0.y, k1.x, k1.y}), q[kk],
                                                        x[tt], 0, 0, 0);
      }
    }
    if (a.score != nullptr && row_base + tile * 16 + mi < a.rows) {
      float* const to = a.score + ((size_t)head * a.rows + row_base + tile * 16 + mi) * a.score_ld + pg * 64;
#pragma unroll
      for (int tt = 0; tt < NS; ++tt)
        *reinterpret_cast<rows_f32x4*>(to + (NS == 1 ? slab0 * 16 + 4 * mq : (slab0 >> 1) * 32 + (tt >> 1) * 32 + 8 * mq + 4 * (tt & 1))) =
            x[tt] * a.scale2;
    }
    float mx = x[0][0];
#pragma unroll
    for (int i = 1; i < 4 * NS; ++i) mx = fmaxf(mx, x[i >> 2][i & 3]);
    const float top = fmaxf(m, over_groups_max(mx) * a.scale2);
    if (__builtin_amdgcn_ballot_w64(top > m)) {  // a factor of 1 for all rows otherwise
      const float f = __builtin_amdgcn_exp2f(m - top);
      l *= f;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) o[ct] *= f;
      m = top;
    }
    uint32_t h[2 * NS];
#pragma unroll
    for (int tt = 0; tt < NS; ++tt) {
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = __builtin_amdgcn_exp2f(fmaf(x[tt][e], a.scale2, -top));
        l += w[e];
      }
      h[2 * tt] = (uint32_t)f32_to_bf16(w[0]) | ((uint32_t)f32_to_bf16(w[1]) << 16);
      h[2 * tt + 1] = (uint32_t)f32_to_bf16(w[2]) | ((uint32_t)f32_to_bf16(w[3]) << 16);
    }
    // outputs: value e of o[ct] is channel 32 e + 8 mq + (ct ^ (mq & 1))
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      const uint16_t* src = at + vq + ct * kVPos + (ct & 1 ? -odd : odd);
      if constexpr (NS == 1) {
        o[ct] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(*reinterpret_cast<const rows_s16x4*>(src),
                                                          __builtin_bit_cast(rows_s16x4, make_uint2(h[0], h[1])), o[ct], 0, 0, 0);
      } else {
#pragma unroll
        for (int kb = 0; kb < NS / 2; ++kb)
          o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              *reinterpret_cast<const rows_bf16x8*>(src + 2 * kb * kVSlab),
              __builtin_bit_cast(rows_bf16x8, rows_u32x4{h[4 * kb], h[4 * kb + 1], h[4 * kb + 2], h[4 * kb + 3]}), o[ct], 0, 0, 0);
      }
    }
  };

  request_fields(page_a);
  if (steps > 1) request_mask(page_b);
  if (page_a >= 0) decode(0);
  __syncthreads();
  for (int step = 0; step < steps; ++step) {
    const int set = step & 1;
    page_a = page_b;
    page_b = page_of(step + 2);
    if (step + 1 < steps) request_fields(page_a);
    if (step + 2 < steps) request_mask(page_b);
    if constexpr (RT == 16) {
      products(set, 0, pg0 + 2 * step);
      if (pg0 + 2 * step + 1 < pg1) products(set, 1, pg0 + 2 * step + 1);
    } else {
      if (pg0 + 2 * step + slot < pg1) products(set, slot, pg0 + 2 * step + slot);
    }
    if (step + 1 < steps && page_a >= 0) decode(set ^ 1);
    __syncthreads();
  }

  float* const out = a.out_prefix + (((size_t)split * g.n_kv_heads + head) * a.rows + row_base) * 128;
  float2* const ml = a.ml_prefix + ((size_t)head * a.rows + row_base) * a.prefix_splits + split;
  const int rows = a.rows - row_base;
  l = over_groups_sum(l);
  // eight channels that follow one another of each word: run[2 e], run[2 e + 1] are channels 32 e + 8 mq + 0 .. 3, 4 .. 7
  rows_f32x4 run[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int i = 0; i < 8; ++i) run[2 * e + (i >> 2)][i & 3] = mq & 1 ? o[i ^ 1][e] : o[i][e];
  }
  if constexpr (RT == 16) {
    const int rr = tile * 16 + mi;
    if (rr >= rows) return;
    rows_f32x4* const dst = reinterpret_cast<rows_f32x4*>(out + (size_t)rr * 128 + 8 * mq);
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[(i >> 1) * 8 + (i & 1)] = run[i];
    if (mq == 0) ml[(size_t)rr * a.prefix_splits] = make_float2(m, l);
  } else {
    // the waves of a tile of rows: RT apart, added in their order
    if (mq == 0) {
      red[0][wv][mi] = m;
      red[1][wv][mi] = l;
    }
    __syncthreads();
    float top = kLowest, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kPrefixWaves / RT; ++w) top = fmaxf(top, red[0][w * RT + tile][mi]);
#pragma unroll
    for (int w = 0; w < kPrefixWaves / RT; ++w) sum += red[1][w * RT + tile][mi] * __builtin_amdgcn_exp2f(red[0][w * RT + tile][mi] - top);
    const float f = __builtin_amdgcn_exp2f(m - top);
    rows_f32x4* const stage = reinterpret_cast<rows_f32x4*>(tiles);
#pragma unroll
    for (int i = 0; i < 8; ++i) stage[(wv * 8 + i) * kStageCt + lane] = run[i] * f;
    if (wv < RT && mq == 0 && tile * 16 + mi < rows) ml[(size_t)(tile * 16 + mi) * a.prefix_splits] = make_float2(top, sum);
    __syncthreads();
    for (int e = tid; e < RT * 16 * 32; e += 64 * kPrefixWaves) {  // four channels c4 of row rr
      const int rr = e >> 5, c4 = e & 31;
      if (rr >= rows) break;
      const rows_f32x4* const from = stage + ((rr >> 4) * 8 + (c4 >> 3) * 2 + (c4 & 1)) * kStageCt + ((c4 >> 1) & 3) * 16 + (rr & 15);
      rows_f32x4 sum4 = from[0];
#pragma unroll
      for (int w = 1; w < kPrefixWaves / RT; ++w) sum4 += from[w * RT * 8 * kStageCt];
      *reinterpret_cast<rows_f32x4*>(out + (size_t)rr * 128 + 4 * c4) = sum4;
    }
  }
}

// What follows the prefix
template <bool FULL, bool MX>
int launch_rows_partial(cas_ctx* ctx, const RowsArgs& a, int items) {
  const dim3 grid((unsigned)items * (unsigned)a.g.n_kv_heads);
#define CAS_LAUNCH(TV)                                                                                       \
  case TV:                                                                                                   \
    hipLaunchKernelGGL((attn_rows_kernel<TV, FULL, MX, 1>), grid, dim3(256), 0, ctx->stream, a);             \
    break;
  switch (a.g.t) {
    CAS_LAUNCH(0) CAS_LAUNCH(1) CAS_LAUNCH(2) CAS_LAUNCH(3) CAS_LAUNCH(4) CAS_LAUNCH(5) CAS_LAUNCH(6) CAS_LAUNCH(7)
    default: return CAS_EINVAL;
  }
#undef CAS_LAUNCH
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

template <int T, bool FULL, bool MX, int RT>
int launch_prefix_tiles(cas_ctx* ctx, const RowsArgs& a, dim3 grid) {
  static LdsLimit lim;
  const int rc = allow_lds(ctx, (const void*)attn_prefix_kernel<T, FULL, MX, RT>, kPrefixLds, lim);
  if (rc != CAS_OK) return rc;
  hipLaunchKernelGGL((attn_prefix_kernel<T, FULL, MX, RT>), grid, dim3(64 * kPrefixWaves), kPrefixLds, ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

// The prefix, for tiles (2, 4, 8 or 16) of 16 query rows a workgroup
template <bool FULL, bool MX>
int launch_prefix_partial(cas_ctx* ctx, const RowsArgs& a, int tiles, int items) {
  const dim3 grid((unsigned)items * (unsigned)a.g.n_kv_heads);
#define CAS_LAUNCH(TV)                                                             \
  case TV:                                                                         \
    return tiles == 2   ? launch_prefix_tiles<TV, FULL, MX, 2>(ctx, a, grid)       \
           : tiles == 4 ? launch_prefix_tiles<TV, FULL, MX, 4>(ctx, a, grid)       \
           : tiles == 8 ? launch_prefix_tiles<TV, FULL, MX, 8>(ctx, a, grid)       \
                        : launch_prefix_tiles<TV, FULL, MX, 16>(ctx, a, grid);
  switch (a.g.t) {
    CAS_LAUNCH(0) CAS_LAUNCH(1) CAS_LAUNCH(2) CAS_LAUNCH(3) CAS_LAUNCH(4) CAS_LAUNCH(5) CAS_LAUNCH(6) CAS_LAUNCH(7)
    default: return CAS_EINVAL;
  }
#undef CAS_LAUNCH
}

}  // namespace cas
