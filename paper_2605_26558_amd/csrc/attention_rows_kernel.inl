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

struct RowsSeq {
  const uint16_t* Q;
  const uint16_t* Knew;
  const uint16_t* Vnew;
  uint16_t* O;
  int seq, len, n_new, ncols;
  int row0;       // query rows (columns x group) of the sequences before
  int splits;     // runs of pages behind the prefix
  int item0;      // work items behind the prefix, of the sequences before
  uint32_t part0; // partial results (row, run, kv head) behind the prefix, of the sequences before
};
struct RowsArgs {
  KvGeom g;
  const uint32_t* spec_pool;
  const uint32_t* verif_pool;
  const int32_t* table;
  int layer, n_q_heads, grp;
  uint32_t grp_inv;          // row / grp = row * grp_inv >> 16
  float scale2;              // log2(e) / sqrt(128): scores are kept as exponents of two
  int n_seqs, rows;          // rows: of all sequences
  int prefix_pages, prefix_run, prefix_splits, prefix_items, tail_run;
  // partial results: 128 outputs each, [split][kv head][row] of the prefix, then the same sequence by sequence; and the
  // pairs (maximum, sum) in the same two regions as [kv head][row][split]
  float* out_prefix;
  float* out_tail;
  float2* ml_prefix;
  float2* ml_tail;
  float* score;              // NULL or [kv head][row][score_ld]: exponents of every position behind the prefix
  int64_t score_ld;
  RowsSeq s[kRowsSeqs];
};

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

__device__ __forceinline__ uint32_t rows_low(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x05040100u); }
__device__ __forceinline__ uint32_t rows_high(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); }

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
  const bool prefix = item < a.prefix_items;
  int si = 0, split, row_base, rows;
  if (prefix) {
    const int tiles = (a.rows + 16 * NT - 1) / (16 * NT);
    split = item / tiles;
    row_base = (item - split * tiles) * 16 * NT;
    rows = a.rows;
  } else {
    item -= a.prefix_items;
    while (si + 1 < a.n_seqs && item >= a.s[si + 1].item0) ++si;
    item -= a.s[si].item0;
    rows = a.s[si].ncols * a.grp;
    const int tiles = (rows + 16 * NT - 1) / (16 * NT);
    split = item / tiles;
    row_base = (item - split * tiles) * 16 * NT;
  }
  const RowsSeq& me = a.s[si];
  const int len = prefix ? a.prefix_pages * 64 : me.len, total = prefix ? len : me.len + me.n_new;
  const int pg0 = prefix ? split * a.prefix_run : a.prefix_pages + split * a.tail_run;
  const int pg1 = min(pg0 + (prefix ? a.prefix_run : a.tail_run), prefix ? a.prefix_pages : (total + 63) / 64);
  const int32_t* page_row = a.table + (size_t)me.seq * g.max_pages_per_seq;

  // ---- queries: fragment kk of a lane holds positions 8 kk + 2 mq, + 1 of the four words of its row
  rows_bf16x8 q[NT][4];
  int seen[NT];  // last position that the row sees
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    int rr = row_base + nt * 16 + mi;
    const bool there = rr < rows;
    int at = si;
    if (prefix) {  // a row of all sequences
      for (int s = 1; s < a.n_seqs; ++s) at = rr >= a.s[s].row0 ? s : at;
      rr -= a.s[at].row0;
    }
    const int c = (int)((uint32_t)rr * a.grp_inv >> 16), gi = rr - c * a.grp;
    seen[nt] = prefix ? 0x7FFFFFFF : total - me.ncols + c;
    const uint16_t* src = a.s[at].Q + ((size_t)c * a.n_q_heads + head * a.grp + gi) * 128 + 2 * mq;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      uint32_t w[4] = {0, 0, 0, 0};
      if (there) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint32_t*>(src + 32 * i + 8 * kk);
      }
      q[nt][kk] = __builtin_bit_cast(rows_bf16x8, rows_u32x4{rows_low(w[0], w[1]), rows_low(w[2], w[3]), rows_high(w[0], w[1]),
                                                              rows_high(w[2], w[3])});
    }
  }

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
    // ---- streams of the thread's word of K and V.  The pools are touched only for pages that hold committed positions
    uint32_t mk = 0, mv = 0;
    int ek = 0, ev = 0;
    WordWindows<T, FULL, MX> wk, wvw;
    const uint32_t *ks = nullptr, *vs = nullptr, *kvf = nullptr, *vvf = nullptr;
    auto load = [&](WordWindows<T, FULL, MX>& w, uint32_t mask, const uint32_t* sp, const uint32_t* vf) {
      const uint32_t p = word_prefix(mask);
      if (has_live) w.load(p, 32u * j - p, sp + g.spec_off + r * g.sw, vf + r * g.lw, vf + 64 * g.lw + r * g.pw);
    };
    if (has_live) {
      const int page = min(max(page_row[pg], 0), g.n_pages - 1);
      const size_t tk = (((size_t)a.layer * g.n_pages + page) * 2 + 0) * g.n_kv_heads + head, tv = tk + g.n_kv_heads;
      ks = a.spec_pool + tk * g.tile_spec_words;
      vs = a.spec_pool + tv * g.tile_spec_words;
      kvf = a.verif_pool + tk * g.tile_verif_words;
      vvf = a.verif_pool + tv * g.tile_verif_words;
      if (live) {
        mk = ks[r * 4 + j];
        mv = vs[r * 4 + j];
        if constexpr (MX) {
          ek = (int)((ks[64 * 4 + r] >> (8 * j)) & 0xFFu);
          ev = (int)((vs[64 * 4 + r] >> (8 * j)) & 0xFFu);
        }
      }
    }
    load(wk, mk, ks, kvf);
    if constexpr (!FULL) load(wvw, mv, vs, vvf);
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
    if constexpr (FULL) load(wvw, mv, vs, vvf);
    ordered();
    // ---- exponents of the wave's 16 tokens: lane (mi, mq) holds tokens 4 mq + e of row mi
    rows_f32x4 x[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) x[nt] = rows_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const uint16_t* src = slab + (1 + 8 * kk + 2 * mq) * kRowsPos + 4 * mi;
      const uint2 k0 = *reinterpret_cast<const uint2*>(src), k1 = *reinterpret_cast<const uint2*>(src + kRowsPos);
      const rows_bf16x8 kf = __builtin_bit_cast(rows_bf16x8, rows_u32x4{k0.x, k0.y, k1.x, k1.y});
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
  const size_t first = prefix ? 0 : me.part0;
  float* const out = (prefix ? a.out_prefix : a.out_tail) + (first + ((size_t)split * g.n_kv_heads + head) * rows) * 128;
  float2* const ml = (prefix ? a.ml_prefix : a.ml_tail) + first;
  const int splits = prefix ? a.prefix_splits : me.splits;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int rr = row_base + nt * 16 + mi;
    if (rr >= rows) continue;
    rows_f32x4* const dst = reinterpret_cast<rows_f32x4*>(out + (size_t)rr * 128 + 32 * mq);
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) dst[ct] = o[nt][ct];
    if (mq == 0) ml[((size_t)head * rows + rr) * splits + split] = make_float2(top[nt], sum[nt]);
  }
}

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

}  // namespace cas
