// The three encoders of the cache (Sec. 5.1), shared by the kernels that append vectors as they are (kv_cache.hip) and those
// that turn them on the way (kv_append_rope.hip).
#pragma once
#include "cas_device.hpp"
#include "cas_internal.hpp"

namespace cas {

// A wave formats four 128-value vectors, the tokens of four rows of a page that follow one another: 16 lanes per vector,
// eight columns per lane.  Four waves take sixteen rows of a tile, from a multiple of sixteen on, so that whole runs of
// lines are written.  The K-th largest magnitude is found bit by bit (15 of them); a lane counts its keys against a
// candidate two to a register (the upper bit of each half of a difference), the lanes of a vector add up through DPP.
// Equals of the K-th are kept in the order of the columns.  Kept values go to a list in LDS by rank, of which a lane packs
// 16 into the 16-T half words that their fields fill; the pruned ones to their place in the row.
// One wave per vector with ballots (kv_append_few_kernel) is bound on a full chip by the scalar unit, which the SIMDs of a CU
// share (298 scalar instructions per vector): 512 tokens of 8 heads would take 6.8 us, so 5.6, of which the search is a quarter (some 19 vector instructions
// a step and four vectors); the rest is launch, memory and packing.
constexpr int kAppendWaves = 4, kAppendRows = 16;
constexpr int kKeptPitch = 136;  // values of a list of kept ones: 16-byte steps, and vectors four banks apart

// over the 16 lanes of a DPP row: the sum in every lane, and the sum of the lanes before
__device__ __forceinline__ int row16_add(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x121, 0xf, 0xf, true);  // row_ror 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x122, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x124, 0xf, 0xf, true);
  return v + __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, true);
}
__device__ __forceinline__ int row16_before(int v) {
  int s = v;
  s += __builtin_amdgcn_update_dpp(0, s, DPP_ROW_SHR1, 0xf, 0xf, false);
  s += __builtin_amdgcn_update_dpp(0, s, DPP_ROW_SHR2, 0xf, 0xf, false);
  s += __builtin_amdgcn_update_dpp(0, s, DPP_ROW_SHR4, 0xf, 0xf, false);
  s += __builtin_amdgcn_update_dpp(0, s, DPP_ROW_SHR8, 0xf, 0xf, false);
  return s - v;
}

struct AppendStage {  // of a wave
  uint16_t kept[4][kKeptPitch];
  uint32_t bitmap[4][4], sexp[4];
  uint32_t spec[4 * 64], lo[4 * 32], pruned[4 * 64];  // rows side by side, as in the tile
};

// The wave's four vectors: columns 8 l .. 8 l + 7 of vector lane / 16 in w, two to a word, l = lane & 15.  They become rows row .. row + 3 of
// the tile of (layer, page, K or V, head) as far as keep(word of a stream of the four rows, words of a row) says.
template <int T, bool MX, class Keep>
__device__ __forceinline__ void format_four(const KvGeom& g, uint32_t* spec_pool, uint32_t* verif_pool, AppendStage& st, const uint32_t (&w)[4],
                                            int lane, int layer, int page, int kv, int head, int row, Keep&& keep) {
  constexpr int FW = MX ? 9 - T : 16 - T;
  const int q = lane >> 4, l = lane & 15;
  constexpr uint32_t kTop = 0x80008000u;
  uint32_t key[4];  // magnitudes under a set bit: a candidate of up to 0x8000 taken off either half leaves that bit if it is reached
#pragma unroll
  for (int i = 0; i < 4; ++i) key[i] = w[i] | kTop;
  uint32_t th = 0;  // the K-th largest magnitude, in both halves
#pragma unroll
  for (int bit = 14; bit >= 0; --bit) {
    const uint32_t cand = th | (0x00010001u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += __popc((key[i] - cand) & kTop);
    th = row16_add(n) >= g.K ? cand : th;
  }
  // columns of the lane, bit c = column 8 l + c: those that reach the candidate
  auto reach = [&](uint32_t cand) -> uint32_t {
    uint32_t x = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) x |= ((key[i] - cand) & kTop) >> (15 - 2 * i);
    return (x | (x >> 15)) & 0xFFu;
  };
  const uint32_t larger = reach(th + 0x00010001u);
  uint32_t equal = reach(th) & ~larger;
  // the larger ones, and as many of the equals as are needed, in the order of the columns
  const int n_equal = __popc(equal);
  const int need = g.K - row16_add(__popc(larger)) - row16_before(n_equal);  // of this lane's equals and those behind
  uint32_t kept = larger | (need >= n_equal ? equal : 0u);
  if (__builtin_amdgcn_ballot_w64(need > 0 && need < n_equal)) {  // the line falls among the equals of a lane
    int left = need < n_equal ? need : 0;
    for (; __builtin_amdgcn_ballot_w64(left > 0); --left) {
      const uint32_t low = left > 0 ? equal & (0u - equal) : 0u;
      kept |= low;
      equal ^= low;
    }
  }
  const int n_kept = __popc(kept);
  int rank = row16_before(n_kept);

  // shared-exponent form: the exponent of a 32-channel block, four lanes, is the largest among its kept values (0 for a
  // block without any)
  int E = 0;
  if constexpr (MX) {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint32_t v = (w[c >> 1] >> (16 * (c & 1))) & 0xFFFFu;
      if ((kept >> c) & 1u) E = max(E, eff_exponent(v));
    }
    E = max(E, quad_dpp<0xB1>(E));  // the lane beside, the other pair
    E = max(E, quad_dpp<0x4E>(E));
    if ((l & 3) == 0) reinterpret_cast<uint8_t*>(&st.sexp[q])[l >> 2] = (uint8_t)E;
  }
  reinterpret_cast<uint8_t*>(st.bitmap[q])[l] = (uint8_t)kept;
  uint16_t* const pr = reinterpret_cast<uint16_t*>(st.pruned + q * g.pw);
  uint16_t* const kp = st.kept[q];
  if (g.K + l < kKeptPitch) kp[g.K + l] = 0;  // up to a whole group of 16
  // the upper half of a row's last word may belong to no value
  if (l == 0 && (g.K & 1)) pr[128 - g.K] = 0;
  if (l == 1 && g.sw > 0) st.spec[q * g.sw + g.sw - 1] = 0;
  if (l == 2 && g.lw > 0) st.lo[q * g.lw + g.lw - 1] = 0;
  int gap = 8 * l - rank;  // pruned values before the column
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const uint32_t v = (w[c >> 1] >> (16 * (c & 1))) & 0xFFFFu;
    const bool k = (kept >> c) & 1u;
    uint32_t u = v;
    if constexpr (MX) {  // sign + magnitude: the significand shifted down to the block's exponent
      const int sh = E - eff_exponent(v);
      u = ((v >> 15) << 8) | (sh < 8 ? significand(v) >> sh : 0u);
    }
    *(k ? kp + rank : pr + gap) = (uint16_t)(MX ? (k ? u : v) : v);
    rank += k;
    gap += !k;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();

  if (16 * l < g.K) {  // values 16 l .. 16 l + 15 of the kept ones: FW half words of fields, T of dropped bits
    uint32_t v[8];
    *reinterpret_cast<uint4*>(v) = reinterpret_cast<const uint4*>(kp)[2 * l];
    *reinterpret_cast<uint4*>(v + 4) = reinterpret_cast<const uint4*>(kp)[2 * l + 1];
    auto pack = [&](auto W, auto DOWN, uint32_t* out, int words) {
      constexpr int width = decltype(W)::value, down = decltype(DOWN)::value, NW = (width + 1) / 2;
      uint32_t o[NW];
#pragma unroll
      for (int i = 0; i < NW; ++i) o[i] = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t f = __builtin_amdgcn_ubfe(v[i >> 1], 16 * (i & 1) + down, width);
        const int bit = i * width, k = bit >> 5, sh = bit & 31;
        o[k] |= f << sh;
        if (sh + width > 32) o[min(k + 1, NW - 1)] |= f >> (32 - sh);
      }
      if constexpr ((width & 1) == 0) {
#pragma unroll
        for (int i = 0; i < NW; ++i)
          if (l * NW + i < words) out[l * NW + i] = o[i];
      } else {
        uint16_t* const h = reinterpret_cast<uint16_t*>(out) + l * width;
#pragma unroll
        for (int i = 0; i < width; ++i)
          if (l * width + i < 2 * words) h[i] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
      }
    };
    pack(std::integral_constant<int, FW>{}, std::integral_constant<int, T>{}, st.spec + q * g.sw, g.sw);
    if constexpr (T > 0) pack(std::integral_constant<int, T>{}, std::integral_constant<int, 0>{}, st.lo + q * g.lw, g.lw);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();

  if (page < 0 || page >= g.n_pages) return;  // a page table entry outside the pool: nothing is written
  const size_t tile = (((size_t)layer * g.n_pages + page) * 2 + kv) * g.n_kv_heads + head;
  uint32_t* ts = spec_pool + tile * g.tile_spec_words;
  uint32_t* tv = verif_pool + tile * g.tile_verif_words;
  // the new rows of the wave, words of a stream each: read together, then written
  uint32_t vb, ve = 0, vs[4], vl[2], vp[4];
  vb = (&st.bitmap[0][0])[lane & 15];
  if constexpr (MX) ve = st.sexp[lane & 3];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (16 * k < g.sw) vs[k] = st.spec[64 * k + lane];
    if (k < 2 && 16 * k < g.lw) vl[k & 1] = st.lo[64 * k + lane];
    if (16 * k < g.pw) vp[k] = st.pruned[64 * k + lane];
  }
  auto flush = [&](uint32_t v, uint32_t* to, int words, int i) {
    if (keep(i, words)) to[i] = v;
  };
  uint32_t* const spec = ts + g.spec_off + row * g.sw;
  uint32_t* const lo = tv + row * g.lw;
  uint32_t* const pruned = tv + 64 * g.lw + row * g.pw;
  flush(vb, ts + row * 4, 4, lane);
  if constexpr (MX) flush(ve, ts + 256 + row, 1, lane);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (16 * k < g.sw) flush(vs[k], spec, g.sw, 64 * k + lane);
    if (k < 2 && 16 * k < g.lw) flush(vl[k & 1], lo, g.lw, 64 * k + lane);
    if (16 * k < g.pw) flush(vp[k], pruned, g.pw, 64 * k + lane);
  }
}

// A wave formats sixteen 128-value vectors, the tokens of sixteen rows of a page from a multiple of sixteen on, so that whole runs
// of lines are written: four lanes per vector, the 32 columns of a bitmap word per lane.
// The K-th largest magnitude is found bit by bit on bit planes: the lane's 32 magnitudes are turned into 15 words with a bit for
// each column (112 operations), and a step is then nine operations for all sixteen vectors: the columns that are as large as the
// candidate's bits so far and have the next one are counted, and either they or the others stay.  Equals of the K-th are kept in the order of
// the columns.  Kept values go to a list in LDS by rank, of which a lane packs 16 into the 16-T half words that their
// fields fill; the pruned ones to their place in the row.
// Of the 25 us that 8000 tokens of 8 heads take with the turn (kv_append_rope.hip) the search is 1.5, the way to the lists and the packing 4, the
// writes 6; some 1000 vector operations for sixteen vectors, a SIMD busy with them in 78 % of the cycles.

// Of a wave.  First the lists of kept values, each to a whole group of 16 and eight more (so that vectors lie in different
// banks), and behind them the pruned values, two to a word, row by row; then, once the lists are in registers, the fields and behind them the
// dropped bits of all rows in the lists' place.
struct RowsStage {
  uint32_t words[kAppendRows * 78];  // (128 + 15 + 8 kept, none pruned) or less: 76 words a vector
};

// A vector of 128 values in the stage, by which lanes exchange them: eights of values at places that lie in different banks for four
// lanes with neighbouring eights and for four that are four eights apart, of four rows
struct VectorRow {
  uint16_t* base;
  int turn;
  __device__ __forceinline__ VectorRow(RowsStage& st, int r) : base(reinterpret_cast<uint16_t*>(st.words) + 128 * r), turn(40 * (r & 3)) {}
  __device__ __forceinline__ void put(int c, const uint32_t (&w)[4]) const {
    *reinterpret_cast<uint4*>(base + (c ^ turn)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void eight(int c, uint32_t (&w)[4]) const {
    const uint4 v = *reinterpret_cast<const uint4*>(base + (c ^ turn));
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  }
  __device__ __forceinline__ uint32_t one(int c) const { return base[c ^ turn]; }
  // Four lanes j: channels 32 k + 8 j .. + 7 of x[k] -> 32 j + 8 k .. + 7
  __device__ __forceinline__ void swap(uint32_t (&x)[4][4], int j) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) put(32 * k + 8 * j, x[k]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 4; ++k) eight(32 * j + 8 * k, x[k]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
};

// columns (2 i, 2 i + 1) of the first and the last 16 of a word, two registers each -> (2 i, 16 + 2 i) and (2 i + 1, 17 + 2 i)
__device__ __forceinline__ uint32_t low_pair(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x05040100u); }
__device__ __forceinline__ uint32_t high_pair(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); }

// Two 16 x 16 matrices of bits, in the lower and the upper halves of 16 words, turned over
__device__ __forceinline__ void bit_planes(uint32_t (&p)[16]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = p[i], b = p[i + 8];
    p[i] = __builtin_amdgcn_perm(b, a, 0x06020400u);
    p[i + 8] = __builtin_amdgcn_perm(b, a, 0x07030501u);
  }
  auto stage = [&](auto K, uint32_t m) {
    constexpr int k = decltype(K)::value;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i & k) continue;
      const uint32_t a = p[i], b = p[i + k];
      p[i] = (a & m) | ((b << k) & ~m);
      p[i + k] = ((a >> k) & m) | (b & ~m);
    }
  };
  stage(std::integral_constant<int, 4>{}, 0x0F0F0F0Fu);
  stage(std::integral_constant<int, 2>{}, 0x33333333u);
  stage(std::integral_constant<int, 1>{}, 0x55555555u);
}

__device__ __forceinline__ int quad_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);  // the lane beside, the other pair
  return v + __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);
}
__device__ __forceinline__ int quad_before(int v, int j) {  // of the lanes before j
  const int b0 = quad_dpp<0x00>(v), b1 = quad_dpp<0x55>(v), b2 = quad_dpp<0xAA>(v);
  return (j > 0 ? b0 : 0) + (j > 1 ? b1 : 0) + (j > 2 ? b2 : 0);
}

// The wave's vectors: columns 32 j + i and 32 j + 16 + i of vector lane / 4 in the halves of w[i], j = lane & 3.  They become rows row0 ..
// row0 + 15 of the tile of (layer, page, K or V, head), those whose bit of `rows` is set.  quiet: NaN are made quiet.
template <int T, bool MX>
__device__ __forceinline__ void format_rows(const KvGeom& g, uint32_t* spec_pool, uint32_t* verif_pool, RowsStage& st, uint32_t (&w)[16],
                                            int lane, int layer, int page, int kv, int head, int row0, uint32_t rows, bool quiet = false) {
  constexpr int FW = MX ? 9 - T : 16 - T;
  const int r = lane >> 2, j = lane & 3;
  uint32_t plane[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) plane[i] = w[i];
  bit_planes(plane);
  if (quiet) {
    uint32_t nan = 0xFFFFFFFFu, low = 0u;
#pragma unroll
    for (int bit = 7; bit < 15; ++bit) nan &= plane[bit];
#pragma unroll
    for (int bit = 0; bit < 6; ++bit) low |= plane[bit];
    nan &= low;
    if (__builtin_amdgcn_ballot_w64(nan != 0u)) {
      plane[6] |= nan;
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] |= (nan >> i & 0x00010001u) << 6;
    }
  }
  // columns as large as the K-th in the bits so far, larger ones, and how many of the former are still to be taken
  uint32_t alive = 0xFFFFFFFFu, kept = 0;
  int spare = g.K - 1;  // to be taken but for one: below 0 where that is none
#pragma unroll
  for (int bit = 14; bit >= 0; --bit) {
    const uint32_t ones = alive & plane[bit];
    const int after = spare - quad_sum(__popc(ones));
    // stay: all bits where the larger ones are enough.  alive = stay ? ones : alive & ~ones; kept |= ones & ~stay.  Written out: the
    // compiler takes five operations for the latter two
    uint32_t stay;
    asm("v_ashrrev_i32 %0, 31, %1" : "=v"(stay) : "v"(after));
    asm("v_bitop3_b32 %0, %0, %1, %2 bitop3:0x98" : "+v"(alive) : "v"(ones), "v"(stay));
    asm("v_bitop3_b32 %0, %0, %1, %2 bitop3:0xf4" : "+v"(kept) : "v"(ones), "v"(stay));
    spare = (int)min((uint32_t)spare, (uint32_t)after);  // after, or spare where that is below 0
  }
  const int need = spare + 1, n_equal = __popc(alive), mine = need - quad_before(n_equal, j);  // of this lane's equals and those behind
  kept |= mine >= n_equal ? alive : 0u;
  if (__builtin_amdgcn_ballot_w64(mine > 0 && mine < n_equal)) {  // the line falls among the equals of a lane
    int left = mine < n_equal ? mine : 0;
    for (; __builtin_amdgcn_ballot_w64(left > 0); --left) {
      const uint32_t low = left > 0 ? alive & (0u - alive) : 0u;
      kept |= low;
      alive ^= low;
    }
  }
  const int before = quad_before(__popc(kept), j);

  // shared-exponent form: the exponent of the word's largest magnitude, which is kept if any of the word is (0 for a word
  // without kept values)
  int E = 0;
  if constexpr (MX) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    E = kept ? eff_exponent(top) : 0;
  }
  const int pitch = ((g.K + 15) & ~15) + 8;  // of a list
  uint16_t* const lists = reinterpret_cast<uint16_t*>(st.words);
  uint32_t* const spec = st.words;
  uint32_t* const lo = spec + kAppendRows * g.sw;
  uint32_t* const pruned = st.words + kAppendRows / 2 * pitch;
  uint16_t* kp = lists + r * pitch;
  uint16_t* pr = reinterpret_cast<uint16_t*>(pruned + r * g.pw);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (g.K + 4 * j + e < pitch) kp[g.K + 4 * j + e] = 0;  // up to a whole group of 16
  if (j == 0 && (g.K & 1)) pr[128 - g.K] = 0;  // the upper half of a row's last word belongs to no value
  // Where the next kept and the next pruned value go, both less 2 bytes for each column before: a column is then at either plus 2 i, and moves
  // the one that it does not take back by 2.  Five operations a value
  typedef __attribute__((address_space(3))) uint16_t lds_u16;
  auto address = [](uint16_t* p) { return (uint32_t)(uintptr_t)(lds_u16*)p; };
  uint32_t to_kept = address(kp + before), to_pruned = address(pr + 32 * j - before);
  const uint32_t others = ~kept;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint32_t v = i < 16 ? w[i & 15] & 0xFFFFu : w[i & 15] >> 16;
    uint32_t is, is_not;  // 0 or all bits.  Written out: the compiler makes comparisons and counts of these, eight operations and more
    asm("v_bfe_i32 %0, %1, %2, 1" : "=v"(is) : "v"(kept), "n"(i));
    asm("v_bfe_i32 %0, %1, %2, 1" : "=v"(is_not) : "v"(others), "n"(i));
    uint32_t u = v;
    if constexpr (MX) {  // sign + magnitude: the significand shifted down to the block's exponent
      const int sh = E - eff_exponent(v);
      u = is ? ((v >> 15) << 8) | (sh < 8 ? significand(v) >> sh : 0u) : v;
    }
    *(lds_u16*)(uintptr_t)(((to_kept & is) | (to_pruned & ~is)) + 2 * i) = (uint16_t)u;
    asm("v_lshl_add_u32 %0, %1, 1, %0" : "+v"(to_pruned) : "v"(is));
    asm("v_lshl_add_u32 %0, %1, 1, %0" : "+v"(to_kept) : "v"(is_not));
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();

  const int groups = (g.K + 15) >> 4;  // of 16 kept values of a vector: up to 128 of all, two to a lane
  const uint32_t groups_inv = groups ? 65536u / (uint32_t)groups + 1u : 0u;
  uint32_t v[2][8];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int t = lane + 64 * k, q = (int)((uint32_t)t * groups_inv >> 16), l = t - q * groups;
    if (t >= kAppendRows * groups) continue;
    const uint4* const src = reinterpret_cast<const uint4*>(lists + q * pitch) + 2 * l;
    *reinterpret_cast<uint4*>(v[k]) = src[0];
    *reinterpret_cast<uint4*>(v[k] + 4) = src[1];
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // the upper half of a row's last word may belong to no value
  if (j == 1 && g.sw > 0) spec[r * g.sw + g.sw - 1] = 0;
  if (j == 2 && g.lw > 0) lo[r * g.lw + g.lw - 1] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int k = 0; k < 2; ++k) {  // FW half words of fields, T of dropped bits
    const int t = lane + 64 * k, q = (int)((uint32_t)t * groups_inv >> 16), l = t - q * groups;
    if (t >= kAppendRows * groups) continue;
    const bool inner = l + 1 < groups;  // the last group of a row ends where its words do
    auto pack = [&](auto W, auto DOWN, uint32_t* out, int words) {
      constexpr int width = decltype(W)::value, down = decltype(DOWN)::value, NW = (width + 1) / 2;
      uint32_t o[NW];
#pragma unroll
      for (int i = 0; i < NW; ++i) o[i] = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t f = __builtin_amdgcn_ubfe(v[k][i >> 1], 16 * (i & 1) + down, width);
        const int bit = i * width, at = bit >> 5, sh = bit & 31;
        o[at] |= f << sh;
        if (sh + width > 32) o[min(at + 1, NW - 1)] |= f >> (32 - sh);
      }
      if constexpr ((width & 1) == 0) {
        const int last = words - (groups - 1) * NW;
#pragma unroll
        for (int i = 0; i < NW; ++i)
          if (i < last || inner) out[l * NW + i] = o[i];
      } else {
        uint16_t* const h = reinterpret_cast<uint16_t*>(out) + l * width;
        const int last = 2 * words - (groups - 1) * width;
#pragma unroll
        for (int i = 0; i < width; ++i)
          if (i < last || inner) h[i] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
      }
    };
    pack(std::integral_constant<int, FW>{}, std::integral_constant<int, T>{}, spec + q * g.sw, g.sw);
    if constexpr (T > 0) pack(std::integral_constant<int, T>{}, std::integral_constant<int, 0>{}, lo + q * g.lw, g.lw);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();

  if (page < 0 || page >= g.n_pages) return;  // a page table entry outside the pool: nothing is written
  const size_t tile = (((size_t)layer * g.n_pages + page) * 2 + kv) * g.n_kv_heads + head;
  uint32_t* ts = spec_pool + tile * g.tile_spec_words;
  uint32_t* tv = verif_pool + tile * g.tile_verif_words;
  const bool written = rows >> r & 1u;
  if (written) ts[row0 * 4 + lane] = kept;
  if constexpr (MX) {
    const int e01 = quad_dpp<0x00>(E) | quad_dpp<0x55>(E) << 8, e23 = quad_dpp<0xAA>(E) | quad_dpp<0xFF>(E) << 8;
    if (written && j == 0) ts[256 + row0 + r] = (uint32_t)(e01 | e23 << 16);
  }
  // rows of a stream lie side by side in the tile as they do here, sixteen of them from a multiple of 64 bytes on
  auto flush = [&](const uint32_t* from, uint32_t* to, int words) {
    if (rows == 0xFFFFu) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = lane + 64 * k;
        if (64 * k < 4 * words && i < 4 * words) reinterpret_cast<uint4*>(to)[i] = reinterpret_cast<const uint4*>(from)[i];
      }
    } else {
      const uint32_t inv = words ? 65536u / (uint32_t)words + 1u : 0u;  // rows of up to 64 words
      for (int i = lane; i < kAppendRows * words; i += 64)
        if (rows >> ((uint32_t)i * inv >> 16) & 1u) to[i] = from[i];
    }
  };
  flush(spec, ts + g.spec_off + row0 * g.sw, g.sw);
  flush(lo, tv + row0 * g.lw, g.lw);
  flush(pruned, tv + 64 * g.lw + row0 * g.pw, g.pw);
}

// One wave per vector, for launches that leave most of the chip idle (see the launch): what counts there is how long one
// wave takes from end to end, and a step of the search is a compare, a ballot and a scalar count here, a chain of some twelve
// dependent vector operations above.  All 15 bits are searched: ending when K values are left costs a branch per bit, as
// much as it saves.  Bound by dependent instructions between two memory round trips; 1.55 of the 2.65 us are the launch.
__device__ __forceinline__ void format_one(const KvGeom& g, uint32_t* spec_pool, uint32_t* verif_pool, uint32_t* stage, uint32_t v0, uint32_t v1,
                                           int lane, int layer, int page, int kv, int head, int row) {
  const uint32_t key0 = v0 & 0x7FFFu, key1 = v1 & 0x7FFFu;
  for (int i = lane; i < g.sw + g.lw + g.pw; i += 64) stage[i] = 0;
  uint32_t T = g.K > 0 ? 0u : 0xFFFFFFFFu;  // the K-th largest magnitude
  auto count = [](uint64_t m0, uint64_t m1) { return __popcll(m0) + __popcll(m1); };
#pragma unroll
  for (int bit = 14; bit >= 0; --bit) {
    const uint32_t cand = T | (1u << bit);
    if (count(__builtin_amdgcn_ballot_w64(key0 >= cand), __builtin_amdgcn_ballot_w64(key1 >= cand)) >= g.K) T = cand;
  }
  // the larger ones, and as many of its equals as are needed, in the order of the columns
  uint64_t m01 = __builtin_amdgcn_ballot_w64(key0 > T), m23 = __builtin_amdgcn_ballot_w64(key1 > T);
  const uint64_t eq0 = __builtin_amdgcn_ballot_w64(key0 == T), eq1 = __builtin_amdgcn_ballot_w64(key1 == T);
  const int need = g.K - count(m01, m23), need1 = need - __popcll(eq0);
  auto rank_in = [](uint64_t m) {
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
  };
  const int e0 = rank_in(eq0), e1 = rank_in(eq1);
  const bool k0 = (key0 > T) | ((key0 == T) & (e0 < need)), k1 = (key1 > T) | ((key1 == T) & (e1 < need1));
  m01 = __builtin_amdgcn_ballot_w64(k0);
  m23 = __builtin_amdgcn_ballot_w64(k1);
  const uint32_t r0 = (uint32_t)rank_in(m01), r1 = (uint32_t)(__popcll(m01) + rank_in(m23));

  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  uint32_t* st_spec = stage;
  uint32_t* st_lo = stage + g.sw;
  uint16_t* st_pr = reinterpret_cast<uint16_t*>(st_lo + g.lw);
  const int fw = g.mx ? 9 - g.t : 16 - g.t;
  const uint32_t lomask = (1u << g.t) - 1u;
  // shared-exponent form: the exponent of a 32-channel block is the largest among its kept values
  // (0 for a block without any); lanes 0..31 / 32..63 hold blocks 0 / 1 in v0 and blocks 2 / 3 in v1
  int E0 = 0, E1 = 0;
  if (g.mx) {
    E0 = k0 ? eff_exponent(v0) : 0;
    E1 = k1 ? eff_exponent(v1) : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      E0 = max(E0, __shfl_xor(E0, d));
      E1 = max(E1, __shfl_xor(E1, d));
    }
  }
  auto put = [&](uint32_t* s, uint32_t bit, uint32_t v, int width) {
    uint32_t w = bit >> 5, sh = bit & 31;
    atomicOr(&s[w], v << sh);
    if (sh + width > 32) atomicOr(&s[w + 1], v >> (32 - sh));
  };
  auto emit = [&](bool kept, uint32_t v, uint32_t rank, uint32_t col, int E) {
    if (kept) {
      if (g.mx) {  // sign + magnitude: the significand shifted down to the block's exponent
        const int sh = E - eff_exponent(v);
        const uint32_t mag = sh < 8 ? significand(v) >> sh : 0u;
        put(st_spec, rank * fw, ((v >> 15) << (8 - g.t)) | (mag >> g.t), fw);
        if (g.t) put(st_lo, rank * g.t, mag & lomask, g.t);
      } else {
        put(st_spec, rank * fw, v >> g.t, fw);
        if (g.t) put(st_lo, rank * g.t, v & lomask, g.t);
      }
    } else {
      st_pr[col - rank] = (uint16_t)v;
    }
  };
  emit(k0, v0, r0, (uint32_t)lane, E0);
  emit(k1, v1, r1, (uint32_t)lane + 64u, E1);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();

  if (page < 0 || page >= g.n_pages) return;  // a page table entry outside the pool: nothing is written
  const size_t tile = (((size_t)layer * g.n_pages + page) * 2 + kv) * g.n_kv_heads + head;
  uint32_t* ts = spec_pool + tile * g.tile_spec_words;
  uint32_t* tv = verif_pool + tile * g.tile_verif_words;
  if (lane < 4) {
    uint64_t m = lane < 2 ? m01 : m23;
    ts[row * 4 + lane] = (uint32_t)(m >> ((lane & 1) * 32));
  }
  if (g.mx) {  // the four block exponents of the vector, block j in byte j
    const int e01 = __shfl(E0, 0) | (__shfl(E0, 32) << 8), e23 = __shfl(E1, 0) | (__shfl(E1, 32) << 8);
    if (lane == 0) ts[g.page_tokens * 4 + row] = (uint32_t)(e01 | (e23 << 16));
  }
  uint32_t* dspec = ts + g.spec_off + row * g.sw;
  uint32_t* dlo = tv + row * g.lw - g.sw;
  uint32_t* dpr = tv + g.page_tokens * g.lw + row * g.pw - g.sw - g.lw;
  for (int i = lane; i < g.sw + g.lw + g.pw; i += 64) (i < g.sw ? dspec : i < g.sw + g.lw ? dlo : dpr)[i] = stage[i];
}

}  // namespace cas
