// Partial attention over runs of pages for the query rows of one or several sequences, compiled in a translation unit per
// form of the cache; attention_rows.hip explains the algorithm.
#pragma once
#include "cas_device.hpp"
#include "cas_internal.hpp"

namespace cas {

typedef short rows_s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 rows_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 rows_bf16x2 __attribute__((ext_vector_type(2)));
typedef float rows_f32x2 __attribute__((ext_vector_type(2)));
typedef float rows_f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int rows_u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRowsSeqs = 32;      // sequences of a launch
constexpr float kLowest = -3.402823466e38f;

// Kernel arguments lie in host memory: a loop of dependent loads from them, or a load whose place depends on another, crosses
// the bus every time (11 of the 27 us that 16 sequences took over a prefix of 8192 positions).
struct RowsArgs {
  KvGeom g;
  const uint32_t* spec_pool;
  const uint32_t* verif_pool;
  const int32_t* table;
  int layer, n_q_heads, grp;
  uint32_t grp_inv;          // row / grp = row * grp_inv >> 16
  float scale2;              // log2(e) / sqrt(128): scores are kept as exponents of two
  int n_seqs, rows;          // rows: of all sequences
  int prefix_pages, prefix_run, prefix_splits, prefix_items;
  // partial results: 128 outputs each, [split][kv head][row] of the prefix, then the same sequence by sequence; and the
  // pairs (maximum, sum) in the same two regions as [kv head][row][split]
  float* out_prefix;
  float* out_tail;
  float2* ml_prefix;
  float2* ml_tail;
  uint64_t* odd;             // [sequence][kv head][page of the two that hold in-flight vectors][slab]: a bit per word of 32 of
                             // their V, set if it holds an infinity or a NaN
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
  int run[kRowsSeqs];        // pages of a run behind the prefix
  int splits[kRowsSeqs];     // runs
  uint32_t part0[kRowsSeqs]; // partial results (row, run, kv head) behind the prefix, of the sequences before
};

// The form of attention within a window (attention_rows.hip): column c, at place P = total - columns + c, sees position i <= P where
// i < n_first or i > P - window.  Pages between the first positions and the window are left out: a run's pages are those that are left,
// numbered one after the other.
struct RowsWindowArgs : RowsArgs {
  int n_first, window, full;
  uint32_t* edge;  // [sequence][kv head][two slabs of 16 positions]: a bit per position that only some columns see and
                   // whose V holds an infinity or a NaN
};
struct WindowPages {
  int lowest;       // the first position that column 0 sees in its window; column c: c more.  May be below 0
  int first_pages;  // pages with first positions
  int skip;         // pages left out behind them
  int zone0, zone1; // committed positions that only some columns see
  __host__ __device__ __forceinline__ WindowPages(int n_first, int window, int len, int total, int ncols) {
    lowest = total - ncols + 1 - window;
    first_pages = (n_first + 63) >> 6;
    const int from = lowest > 0 ? lowest >> 6 : 0;
    skip = from > first_pages ? from - first_pages : 0;
    zone0 = lowest > n_first ? lowest : n_first;
    zone1 = lowest + ncols - 1 < len ? lowest + ncols - 1 : len;
  }
  __host__ __device__ __forceinline__ int page(int i) const { return i + (i >= first_pages ? skip : 0); }
};

// The tables of the sequences, an entry per lane: one load each, all at once; then the entry of the sequence whose share of a
// table (of the numbers before each) holds n, as a scalar.
struct SeqTable {
  int v;
  __device__ __forceinline__ explicit SeqTable(const int (&t)[kRowsSeqs]) : v(t[threadIdx.x & (kRowsSeqs - 1)]) {}
  __device__ __forceinline__ explicit SeqTable(const uint32_t (&t)[kRowsSeqs]) : v((int)t[threadIdx.x & (kRowsSeqs - 1)]) {}
  __device__ __forceinline__ int which(int n) const { return __popc((uint32_t)__builtin_amdgcn_ballot_w64(n >= v)) - 1; }
  __device__ __forceinline__ int operator[](int s) const { return __builtin_amdgcn_readlane(v, s); }
};

// Waves of a workgroup and pages of a step.  256 query rows need sixteen waves and both pages; with fewer, two workgroups of
// eight share a CU, and one decodes while the other waits for its streams.
template <int RT>
struct RowsShape {
  static constexpr int kWaves = RT == 16 ? 16 : 8, kPages = kWaves / 8;
};
// A page's K and V in LDS, slab by slab of 16 tokens: [1 + 32 positions][values], for K the four words of a token at one
// position side by side, for V the tokens of a word; row 0 takes what lanes without a value left write.
constexpr int kKPos = 64, kVPos = 72;                       // values from a position to the next
constexpr int kKSlab = 33 * kKPos + 16, kVSlab = 33 * kVPos;
constexpr int kRowsPage = 4 * (kKSlab + kVSlab);
constexpr int kStageRun = 65;                               // groups of four values of 64 lanes, padded
template <int RT>
struct RowsLds {  // two sets of tiles (72 KB a workgroup, 144 for sixteen waves), in which the waves' results are joined as well
  static constexpr int kSet = RowsShape<RT>::kPages * kRowsPage;
  static constexpr size_t kBytes = sizeof(uint16_t) * 2 * kSet;
  static_assert(sizeof(float) * 4 * kStageRun * 8 * RowsShape<RT>::kWaves <= kBytes && 16 * RT * 136 <= kSet, "");
};

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

// Product kk of a page takes 8 positions of the four words, lane group mq two of them, two apart
__device__ __forceinline__ int k_position(int kk, int mq) { return 8 * kk + (mq & 1) + 4 * (mq >> 1); }

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

// LDS writes at base + i * pitch bytes with the address in one operation (the compiler's code takes two)
typedef __attribute__((address_space(3))) uint16_t lds_u16;
__device__ __forceinline__ uint32_t lds_address(uint16_t* p) { return (uint32_t)(uintptr_t)(lds_u16*)p; }
__device__ __forceinline__ void lds_write(uint32_t base, int i, int pitch, uint16_t v) {
  uint32_t at;
  asm("v_mad_i32_i24 %0, %1, %2, %3" : "=v"(at) : "v"(i), "s"(pitch), "v"(base));
  *(lds_u16*)(uintptr_t)at = v;
}

// What the heads of two numbers leave of them, rounded to bf16: a product of two elements subtracts a head in one operation
// where it lies (its other element times 0), one conversion takes both.
__device__ __forceinline__ uint32_t bf16_rests(uint32_t heads, float lo, float hi) {
  uint32_t minus_lo = 0x0000BF80u, minus_hi = 0xBF800000u;
  asm("" : "+s"(minus_lo), "+s"(minus_hi));  // in registers: as constants of the instruction both came out as the upper one
  const rows_bf16x2 h = __builtin_bit_cast(rows_bf16x2, heads);
  const rows_f32x2 d = {__builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(rows_bf16x2, minus_lo), lo, false),
                        __builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(rows_bf16x2, minus_hi), hi, false)};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(d, rows_bf16x2));
}

// The N words of a window, the last ones only if a lane of the wave has fields there.  A scattered load takes a CU's address
// unit 8 to 12 ns whatever its width, and 16 waves have 11 such loads each for the windows of the exact form at t = 4; with
// 60 % kept, 7 nearly always hold all that is needed.
template <int N>
__device__ __forceinline__ void load_window(__amdgpu_buffer_rsrc_t rs, int off, uint32_t bits, uint32_t (&d)[N]) {
  constexpr int kSure = N > 12 ? 12 : (N - 1) / 4 * 4;
  if constexpr (kSure > 0) load_words<kSure>(rs, off, d);
  if (kSure == 0 || __builtin_amdgcn_ballot_w64(bits > 32u * kSure)) load_words<N - kSure>(rs, off + 4 * kSure, d + kSure);
}

// A workgroup: one kv head, one run of pages, up to 16 RT query rows: those of all sequences over the whole pages of the
// prefix, or of one sequence over pages behind it.  Sixteen waves, the most that a CU holds at 128 registers, take two pages
// a step: each decodes 16 tokens of K or of V of one of them into a tile that all read, and forms the products of 16 rows
// with both pages (RT = 16), with one (8), or with half (4) or a quarter (2) of one.  There are two sets of tiles: a step's
// products, the decode of the next and the loads of the one after it are between the same two barriers.  The waves of a
// row are joined at the end.
//
// Products are formed as K Q^T and V^T P^T, so that a query row is a column of the result: the probabilities leave the first
// product where the second wants them, and a row's factors are one value per lane.
//
// With many rows the reads of the tiles are what the LDS is busy with, and 16 lanes are served at once.  K: eight bytes of a
// lane, positions 128 bytes apart, slabs 32 bytes off each other, so that a product's 16 tokens may be four of every eight of two
// slabs: lane group mq then holds the weights of eight tokens that follow one another.  V: eight tokens of a channel in one
// read; the 8 lanes served at once take two positions of the four words, and positions lie 144 bytes apart, so that these do
// not meet.  (With V 128 bytes apart and reads of four tokens, four lanes met in every bank: 104 of the 286 thousand cycles
// that a CU was busy with 256 rows over 32768 positions, now 31 of 189.)  The walks' writes meet more often for it (some 4 lanes in
// place of 2), which is less.
//
// 128 registers a lane are what sixteen waves a CU leave.  The draft forms fit; the exact ones spill 1, 8, 8 and 1 of them at t = 4
// (RT = 2, 4, 8, 16; with shared exponents 20, 12, 12 and 2), 25 at the most (t = 5, RT = 4); within a window 0, 16, 16 and 0 (4, 12, 6
// and 2), 20 at the most.  They cost time: with what only some pages need (the mask, positions that some columns see) worked out ahead of the
// loop over pages 25 to 35 were spilled within a window, and 128 rows, exact, took 281 us for 196.
template <int T, bool FULL, bool MX, int RT, class ARGS>
__global__ __launch_bounds__(64 * RowsShape<RT>::kWaves, 4) void attn_rows_kernel(ARGS a) {
  constexpr bool kWindow = std::is_same<ARGS, RowsWindowArgs>::value;
  constexpr int kWaves = RowsShape<RT>::kWaves, kPages = RowsShape<RT>::kPages, kSet = RowsLds<RT>::kSet;
  extern __shared__ __align__(16) uint16_t tiles[];
  __shared__ float red[2][kWaves][16];
  constexpr int NS = RT >= 8 ? 4 : RT / 2;  // slabs of 16 tokens that a wave's products take of a page
  const KvGeom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = (int)blockIdx.x % g.n_kv_heads;  // heads next to each other: workgroups that share pages share an XCD's L2
  int item = (int)blockIdx.x / g.n_kv_heads;
  const int slot = kPages == 1 ? 0 : wv >> 3, u = wv & 7;  // page of the step, place among its waves
  const int kv = u >> 2, r = (u & 3) * 16 + (lane >> 2), j = lane & 3;  // decode role: K or V, token, word
  const int mi = lane & 15, mq = lane >> 4;            // role in the products: query row (token, channel) mi, group mq
  // and the wave's: tile of rows, first slab.  Waves of a workgroup go to the SIMDs in turn: where fewer rows leave tiles empty, the
  // waves that have products are spread over all four
  const int tile = RT == 16 ? wv : RT == 2 ? u >> 2 : RT == 4 ? (u + (u >> 2)) & 3 : u;
  const int slab0 = RT >= 8 ? 0 : RT == 2 ? u & 3 : (u >> 2) * NS;
  auto wave_of = [](int t, int w) { return RT == 2 ? 4 * t + w : RT == 4 ? 4 * w + ((t - w) & 3) : w * RT + t; };  // w-th wave of a tile

  // ---- what this workgroup works on (uniform)
  const SeqTable t_item0(a.item0), t_len(a.len), t_new(a.n_new), t_cols(a.ncols), t_seq(a.seq), t_splits(a.splits), t_part0(a.part0), t_run(a.run);
  const bool prefix = !kWindow && item < a.prefix_items;  // none within a window
  int si = 0;
  if (!prefix) {
    if (!kWindow) item -= a.prefix_items;
    si = t_item0.which(item);
    item -= t_item0[si];
  }
  const int rows = prefix ? a.rows : t_cols[si] * a.grp, blocks = (rows + 16 * RT - 1) / (16 * RT);
  const int split = item / blocks, row_base = (item - split * blocks) * 16 * RT;
  const int len = prefix ? a.prefix_pages * 64 : t_len[si], total = prefix ? len : len + t_new[si];
  const int run = prefix ? a.prefix_run : t_run[si];
  const int ncols = t_cols[si];
  auto pages_of = [&]() {
    if constexpr (kWindow) return WindowPages(a.n_first, a.window, len, total, ncols);
    else return 0;
  };
  const auto win_pages = pages_of();
  auto page_at = [&](int i) {  // which page of the sequence the i-th of a run is
    if constexpr (kWindow) return win_pages.page(i);
    else return i;
  };
  auto committed = [&](int pos) {  // a position of the cache that some row sees
    if constexpr (kWindow) return pos < len && (pos >= win_pages.lowest || pos < a.n_first);
    else return pos < len;
  };
  int left_out = 0;
  if constexpr (kWindow) left_out = win_pages.skip;
  const int pg0 = (prefix || kWindow ? 0 : a.prefix_pages) + split * run, pg1 = min(pg0 + run, (total + 63) / 64 - left_out), steps = (pg1 - pg0 + kPages - 1) / kPages;
  const int32_t* page_row = a.table + (size_t)t_seq[si] * g.max_pages_per_seq;
  const uint32_t first = prefix ? 0 : (uint32_t)t_part0[si];  // of the partial results
  const int splits = prefix ? a.prefix_splits : t_splits[si];
  const bool idle = row_base + tile * 16 >= rows;   // a wave without rows decodes only
  const int all_see = prefix ? 0x7FFFFFFF : total - ncols;  // the last position that every row sees

  // ---- the wave's unit of a step: pool pages two steps ahead, bitmap words one, fields as soon as those are there.  The pools
  // are touched only for pages that hold committed positions
  // where the thread's word begins in a set, and what a position adds
  const int col = slot * kRowsPage + (kv ? 4 * kKSlab + (u & 3) * kVSlab + kVPos + j * 16 + (lane >> 2)
                                         : (u & 3) * kKSlab + kKPos + (lane >> 2) * 4 + j);
  const int pitch = 2 * (kv ? kVPos : kKPos);  // bytes
  constexpr int kNone = -1, kFresh = -2;       // no page; one without committed positions
  auto page_of = [&](int step) {
    const int i = pg0 + kPages * step + slot, pg = page_at(i);
    return i >= pg1 ? kNone : pg * 64 >= len ? kFresh : min(max(page_row[pg], 0), g.n_pages - 1);
  };
  auto tile_of = [&](int page) { return (((size_t)a.layer * g.n_pages + page) * 2 + kv) * g.n_kv_heads + head; };
  uint32_t next_mask = 0, next_exp = 0;
  auto request_mask = [&](int step, int page) {
    next_mask = next_exp = 0;
    if (page < 0) return;
    const uint32_t* sp = a.spec_pool + tile_of(page) * g.tile_spec_words;
    if (committed(page_at(pg0 + kPages * step + slot) * 64 + r)) {
      next_mask = sp[r * 4 + j];
      if constexpr (MX) next_exp = sp[64 * 4 + r];
    }
  };
  // the exact form with many rows has no registers for all fields during the products: those of the values that were not
  // kept are requested behind them, under the decode of the kept ones
  constexpr bool kLate = RT >= 4;
  // Streams are read through buffer descriptors of a tile: a scalar base and 32-bit lane offsets, no 64-bit addresses.
  WordWindows<T, FULL, MX> win;
  uint32_t mask = 0, kept_before = 0;
  int shared_exp = 0;
  auto stream = [&](const uint32_t* pool, int page, int words) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t*>(pool + tile_of(page) * words), 0, words * 4, kRawBufferFlags);
  };
  auto request_pruned = [&](int page) {
    const uint32_t before = 32u * j - kept_before;
    win.pr.shp = (before & 1u) << 4;
    load_window(stream(a.verif_pool, page, g.tile_verif_words), (64 * g.lw + r * g.pw + (int)(before >> 1)) * 4,
                16u * (32u - (uint32_t)__popc(mask)) + win.pr.shp, win.pr.dp);
  };
  auto request_fields = [&](int page) {
    mask = taken(next_mask);
    if (page < 0) return;
    if constexpr (MX) shared_exp = (int)((taken(next_exp) >> (8 * j)) & 0xFFu);
    const int cnt = __popc(mask);
    const int b0 = quad_dpp<0x00>(cnt), b1 = quad_dpp<0x55>(cnt), b2 = quad_dpp<0xAA>(cnt);
    kept_before = (uint32_t)((j > 0 ? b0 : 0) + (j > 1 ? b1 : 0) + (j > 2 ? b2 : 0));
    constexpr int kField = MX ? 9 - T : 16 - T;
    uint32_t bit = kept_before * kField;
    win.k.shs = bit & 31u;
    load_window(stream(a.spec_pool, page, g.tile_spec_words), (g.spec_off + r * g.sw + (int)(bit >> 5)) * 4,
                (uint32_t)cnt * kField + win.k.shs, win.k.ds);
    if constexpr (FULL && T > 0) {
      bit = kept_before * T;
      win.k.shl = bit & 31u;
      load_window(stream(a.verif_pool, page, g.tile_verif_words), (r * g.lw + (int)(bit >> 5)) * 4, (uint32_t)cnt * T + win.k.shl, win.k.dl);
    }
    if constexpr (FULL && !kLate) request_pruned(page);
  };
  auto decode = [&](int step, int page) {
    if (page == kNone) return;
    const int set = step & 1, tok0 = page_at(pg0 + kPages * step + slot) * 64;
    bool whole = tok0 + 64 <= len;  // of committed positions
    if constexpr (kWindow) whole = whole && (tok0 >= win_pages.lowest || tok0 + 64 <= a.n_first);
    const uint32_t to = lds_address(tiles + set * kSet + col);
    if (!FULL || !whole) {  // what is not written has to read as 0: 256 or 288 groups of eight values
      uint16_t* const slab = tiles + set * kSet + slot * kRowsPage + (kv ? 4 * kKSlab + (u & 3) * kVSlab + kVPos : (u & 3) * kKSlab + kKPos);
      // The exact form does so for the last pages only.  With few rows its fields are all there by now: few registers, and nothing of it
      // ahead of the loop over pages.  16 sequences over 8192 positions, 4 / 20 rows, us: 144 / 150 -> 124 / 129; with 64 rows 152 -> 174
      if constexpr (FULL && !MX && RT == 2) {
        int k = lane;
        asm volatile("" : "+v"(k));
#pragma unroll 1
        for (; k < (kv ? 576 : 512); k += 64) reinterpret_cast<uint2*>(slab)[k] = make_uint2(0, 0);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) reinterpret_cast<uint4*>(slab)[lane + 64 * k] = make_uint4(0, 0, 0, 0);
        if (kv && lane < 32) reinterpret_cast<uint4*>(slab)[lane + 256] = make_uint4(0, 0, 0, 0);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    if (page >= 0) {
      if constexpr (FULL && kLate) request_pruned(page);
      if constexpr (MX) {
        win.k.decode_finite(mask, [&](int bp, uint32_t v) { lds_write(to, bp, pitch, (uint16_t)(v >> 16)); }, shared_exp);
        if (__builtin_amdgcn_ballot_w64(shared_exp == 255 && mask != 0u)) {  // words of infinities or NaN: value by value, from memory
          const uint32_t* const sp = a.spec_pool + tile_of(page) * g.tile_spec_words + g.spec_off + r * g.sw;
          const uint32_t* const lo = a.verif_pool + tile_of(page) * g.tile_verif_words + r * g.lw;
          uint32_t m = shared_exp == 255 ? mask : 0u, at = kept_before;
          while (m) {
            uint32_t v = read_field(sp, at * (9 - T), 9 - T), mag = v & ((1u << (8 - T)) - 1u);
            mag <<= T;
            if constexpr (FULL && T > 0) mag |= read_field(lo, at * T, T);
            lds_write(to, lowest_bit(m), pitch, (uint16_t)mx_word(v >> (8 - T), shared_exp, mag));
            m &= m - 1u;
            ++at;
          }
        }
      } else {
        win.k.decode(mask, [&](int bp, uint16_t v) { lds_write(to, bp, pitch, v); });
      }
      if constexpr (FULL) win.pr.decode(committed(tok0 + r) ? ~mask : 0u, [&](int bp, uint16_t v) { lds_write(to, bp, pitch, v); });
    }
    if (!whole) {  // in-flight vectors, eight values at a time
      const int pos = tok0 + r;
      bool odd = false;
      if (pos >= len && pos < total) {
        const uint4* src = reinterpret_cast<const uint4*>((kv ? a.Vnew[si] : a.Knew[si]) + ((size_t)(pos - len) * g.n_kv_heads + head) * 128 + 32 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 x = src[i];
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const uint16_t v = (uint16_t)(w[c >> 1] >> (16 * (c & 1)));
            // an infinity or a NaN of V, times 0, would reach rows that do not see the vector: 0 here, added where the
            // partial results are joined
            const bool inf = kv && (v & 0x7F80u) == 0x7F80u;
            odd |= inf;
            lds_write(to, 8 * i + c, pitch, inf ? (uint16_t)0 : v);
          }
          asm volatile("" ::: "memory");
        }
      }
      if (kv && (!kWindow || tok0 + 64 > len)) {
        const uint64_t lanes = __builtin_amdgcn_ballot_w64(odd);
        if (lane == 0) a.odd[(((size_t)si * g.n_kv_heads + head) * 2 + (tok0 - (len & ~63)) / 64) * 4 + (u & 3)] = lanes;
      }
    }
    if constexpr (kWindow) {
      // Committed positions that the later columns no longer see: an infinity or a NaN of their V, times 0, would reach these.  0 here,
      // added where the partial results are joined
      const int slab0 = tok0 + 16 * (u & 3);
      if (kv && win_pages.zone0 < win_pages.zone1 && slab0 < win_pages.zone1 && slab0 + 16 > win_pages.zone0) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        uint16_t* const slab = tiles + set * kSet + slot * kRowsPage + 4 * kKSlab + (u & 3) * kVSlab + kVPos;
        uint32_t odd = 0;
        int k = lane;
        asm volatile("" : "+v"(k));  // nothing of this ahead of the loop over pages, where it would take registers of it
#pragma unroll 1
        for (; k < 256; k += 64) {  // eight tokens of a position and word
          uint16_t* const at = slab + (k >> 3) * kVPos + (k & 7) * 8;
#pragma unroll 1
          for (int e = 0; e < 8; ++e) {
            const int token = (k & 1) * 8 + e, pos = slab0 + token;
            if (pos >= win_pages.zone0 && pos < win_pages.zone1 && (at[e] & 0x7F80u) == 0x7F80u) {
              odd |= 1u << token;
              at[e] = 0;
            }
          }
        }
        uint32_t any = 0;
#pragma unroll 1
        for (int t = 0; t < 16; ++t) any |= __builtin_amdgcn_ballot_w64(odd >> t & 1) ? 1u << t : 0u;
        if (lane == 0) a.edge[((size_t)si * g.n_kv_heads + head) * 2 + (slab0 >> 4) - (win_pages.zone0 >> 4)] = any;
      }
    }
  };
  int page_a = page_of(0), page_b = page_of(1);
  request_mask(0, page_a);

  // ---- queries, through the second set of tiles, which the decode of the second step is the first to write
  rows_bf16x8 q[4];
  {
    constexpr int kParts = (RT * 256 + 64 * kWaves - 1) / (64 * kWaves);
    uint16_t* const stage = tiles + kSet;
    QueryPart part[kParts];
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const int i = tid + k * 64 * kWaves;
      int rr = row_base + (i >> 4), first = 0;
      const bool there = rr < rows && i < RT * 256;
      const uint16_t* src = a.Q[si];
      if (prefix) {
#pragma unroll
        for (int s = 1; s < kRowsSeqs; ++s) {
          const bool in = rr >= a.row0[s];
          first = in ? a.row0[s] : first;
          src = in ? a.Q[s] : src;
        }
      }
      rr -= first;
      const int c = (int)((uint32_t)rr * a.grp_inv >> 16), gi = rr - c * a.grp;
      part[k].load(there ? src + ((size_t)c * a.n_q_heads + head * a.grp + gi) * 128 : nullptr, i & 15);
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const int i = tid + k * 64 * kWaves;
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
  const int swap = (mi >> 2) & 1 ? kVPos : 0;
  // token of a page that the lane holds as element e of product tt: four of the slab (NS = 1), or of every eight of two
  auto token = [&](int tt) { return NS == 1 ? slab0 * 16 + 4 * mq : slab0 * 16 + 32 * (tt >> 1) + 8 * mq + 4 * (tt & 1); };
  auto products = [&](int step, int page) {
    const int i = pg0 + kPages * step + page, set = step & 1, pg = page_at(i);
    if (idle || i >= pg1) return;
    const uint16_t* const at = tiles + set * kSet + page * kRowsPage;
    rows_f32x4 x[NS];
#pragma unroll
    for (int tt = 0; tt < NS; ++tt) {
      x[tt] = rows_f32x4{0.f, 0.f, 0.f, 0.f};
      asm volatile("" ::: "memory");  // the reads of one product at a time: those of all do not fit the registers
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const uint16_t* src = at + kq + (tt >> 1) * 2 * kKSlab + (tt & 1) * 16 + (1 + k_position(kk, mq)) * kKPos;
        const uint2 k0 = *reinterpret_cast<const uint2*>(src), k1 = *reinterpret_cast<const uint2*>(src + 2 * kKPos);
        x[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(rows_bf16x8, rows_u32x4{k0.x, k0.y, k1.x, k1.y}), q[kk],
                                                        x[tt], 0, 0, 0);
      }
    }
    const int row = row_base + tile * 16 + mi;
    bool all_in = pg * 64 + 63 <= all_see;  // for every row
    if constexpr (kWindow) all_in = all_in && (pg * 64 + 63 < a.n_first || pg * 64 >= win_pages.lowest + ncols - 1);
    if (!all_in) {
      const int seen = all_see + (int)((uint32_t)row * a.grp_inv >> 16);  // column c sees c positions more
      // from the lane's first token on: the last one that it sees, and within a window those between the first positions and it
      const int base = pg * 64 + token(0), last = seen - base;
      int hidden = 0;
      uint32_t n_hidden = 0;
      if constexpr (kWindow) {
        hidden = a.n_first - base;
        n_hidden = (uint32_t)max(max(seen - a.window, -1) - a.n_first + 1, 0);  // a sum of the two may pass 32 bits
      }
#pragma unroll
      for (int tt = 0; tt < NS; ++tt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = token(tt) - token(0) + e;
          bool sees = i <= last;
          if constexpr (kWindow) sees = sees && (uint32_t)(i - hidden) >= n_hidden;
          x[tt][e] = sees ? x[tt][e] : -INFINITY;
        }
      }
    }
    if (!kWindow && a.score != nullptr && row < rows) {
      float* const to = a.score + ((size_t)head * rows + row) * a.score_ld + pg * 64;
#pragma unroll
      for (int tt = 0; tt < NS; ++tt) *reinterpret_cast<rows_f32x4*>(to + token(tt)) = x[tt] * a.scale2;
    }
    float mx = x[0][0];
#pragma unroll
    for (int i = 1; i < 4 * NS; ++i) mx = fmaxf(mx, x[i >> 2][i & 3]);
    // at least the lowest finite number: where a row sees nothing of these tokens, the maximum is -inf as its scores are
    const float top = fmaxf(m, over_groups_max(mx) * a.scale2);
    if (__builtin_amdgcn_ballot_w64(top > m)) {  // a factor of 1 for all rows otherwise
      const float f = __builtin_amdgcn_exp2f(m - top);
      l *= f;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) o[ct] *= f;
      m = top;
    }
    // Weights for the second product: a bf16 head (cut off) and the bf16 rounding of what is left, 16 bits together.  With the
    // head alone, rounded, an output is off by 1.4e-3 of its size (mean square) beside the 1.7e-3 of its own rounding.
    uint32_t h[2 * NS], rest[2 * NS];
#pragma unroll
    for (int tt = 0; tt < NS; ++tt) {
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = __builtin_amdgcn_exp2f(fmaf(x[tt][e], a.scale2, -top));
        l += w[e];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        h[2 * tt + i] = __builtin_amdgcn_perm(__float_as_uint(w[2 * i + 1]), __float_as_uint(w[2 * i]), 0x07060302u);
        rest[2 * tt + i] = bf16_rests(h[2 * tt + i], w[2 * i], w[2 * i + 1]);
      }
    }
    // outputs: value e of o[ct] is channel 32 e + 8 mq + (ct ^ (mq & 1))
    auto part = [&](const uint32_t (&p)[2 * NS], int kb) {
      return __builtin_bit_cast(rows_bf16x8, rows_u32x4{p[4 * kb], p[4 * kb + 1], p[4 * kb + 2], p[4 * kb + 3]});
    };
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      const uint16_t* src = at + vq + ct * kVPos + (ct & 1 ? -swap : swap);
      if constexpr (NS == 1) {
        const rows_s16x4 v = *reinterpret_cast<const rows_s16x4*>(src);
        o[ct] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v, __builtin_bit_cast(rows_s16x4, make_uint2(h[0], h[1])), o[ct], 0, 0, 0);
        o[ct] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v, __builtin_bit_cast(rows_s16x4, make_uint2(rest[0], rest[1])), o[ct], 0, 0, 0);
      } else {
#pragma unroll
        for (int kb = 0; kb < NS / 2; ++kb) {
          const rows_bf16x8 v = *reinterpret_cast<const rows_bf16x8*>(src + 2 * kb * kVSlab);
          o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, part(h, kb), o[ct], 0, 0, 0);
          o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, part(rest, kb), o[ct], 0, 0, 0);
        }
      }
    }
  };

  request_fields(page_a);
  request_mask(1, page_b);
  decode(0, page_a);
  __syncthreads();
  for (int step = 0; step < steps; ++step) {
    page_a = page_b;
    page_b = page_of(step + 2);
    request_fields(page_a);
    request_mask(step + 2, page_b);
    if constexpr (RT == 16) {
      products(step, 0);
      products(step, 1);
    } else {
      products(step, slot);
    }
    // Before waves that are still at their products: the next step's loads go out the sooner.  16 sequences of 4096 visible positions, draft,
    // 52 -> 50 us, 40 rows of 8192 over shared exponents 190 -> 180; the products first instead 53 and 186.  Sixteen waves of one workgroup wait
    // for each other all the same: 8 sequences of 5 columns 42.2 -> 42.9
    if constexpr (RT < 16) __builtin_amdgcn_s_setprio(3);
    decode(step + 1, page_a);
    if constexpr (RT < 16) __builtin_amdgcn_s_setprio(0);
    __syncthreads();
  }

  // ---- partial results
  const int left = rows - row_base;
  float* const out = (prefix ? a.out_prefix : a.out_tail) + ((size_t)first + ((size_t)split * g.n_kv_heads + head) * rows + row_base) * 128;
  float2* const ml = (prefix ? a.ml_prefix : a.ml_tail) + first + ((size_t)head * rows + row_base) * splits + split;
  l = over_groups_sum(l);
  // eight channels that follow one another of each word: eight[2 e], eight[2 e + 1] are channels 32 e + 8 mq + 0 .. 3, 4 .. 7
  rows_f32x4 eight[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int i = 0; i < 8; ++i) eight[2 * e + (i >> 2)][i & 3] = mq & 1 ? o[i ^ 1][e] : o[i][e];
  }
  if constexpr (RT == kWaves) {  // each wave has rows of its own
    const int rr = tile * 16 + mi;
    if (rr >= left) return;
    rows_f32x4* const dst = reinterpret_cast<rows_f32x4*>(out + (size_t)rr * 128 + 8 * mq);
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[(i >> 1) * 8 + (i & 1)] = eight[i];
    if (mq == 0) ml[(size_t)rr * splits] = make_float2(m, l);
  } else {
    // the waves of a tile of rows: RT apart, added in their order
    if (mq == 0) {
      red[0][wv][mi] = m;
      red[1][wv][mi] = l;
    }
    __syncthreads();
    float top = kLowest, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves / RT; ++w) top = fmaxf(top, red[0][wave_of(tile, w)][mi]);
#pragma unroll
    for (int w = 0; w < kWaves / RT; ++w) sum += red[1][wave_of(tile, w)][mi] * __builtin_amdgcn_exp2f(red[0][wave_of(tile, w)][mi] - top);
    const float f = __builtin_amdgcn_exp2f(m - top);
    rows_f32x4* const stage = reinterpret_cast<rows_f32x4*>(tiles);
    if (!idle) {
#pragma unroll
      for (int i = 0; i < 8; ++i) stage[(wv * 8 + i) * kStageRun + lane] = eight[i] * f;
      if (slab0 == 0 && mq == 0 && tile * 16 + mi < left) ml[(size_t)(tile * 16 + mi) * splits] = make_float2(top, sum);
    }
    __syncthreads();
    for (int e = tid; e < RT * 16 * 32; e += 64 * kWaves) {  // four channels c4 of row rr
      const int rr = e >> 5, c4 = e & 31;
      if (rr >= left) break;
      const rows_f32x4* const from = stage + ((c4 >> 3) * 2 + (c4 & 1)) * kStageRun + ((c4 >> 1) & 3) * 16 + (rr & 15);
      rows_f32x4 sum4 = from[wave_of(rr >> 4, 0) * 8 * kStageRun];
#pragma unroll
      for (int w = 1; w < kWaves / RT; ++w) sum4 += from[wave_of(rr >> 4, w) * 8 * kStageRun];
      *reinterpret_cast<rows_f32x4*>(out + (size_t)rr * 128 + 4 * c4) = sum4;
    }
  }
}

template <int T, bool FULL, bool MX, int RT, class ARGS>
int launch_rows_tiles(cas_ctx* ctx, const ARGS& a, dim3 grid) {
  static LdsLimit lim;
  const int rc = allow_lds(ctx, (const void*)attn_rows_kernel<T, FULL, MX, RT, ARGS>, RowsLds<RT>::kBytes, lim);
  if (rc != CAS_OK) return rc;
  hipLaunchKernelGGL((attn_rows_kernel<T, FULL, MX, RT, ARGS>), grid, dim3(64 * RowsShape<RT>::kWaves), RowsLds<RT>::kBytes, ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

// tiles: of 16 query rows a workgroup, 2, 4, 8 or 16
template <bool FULL, bool MX, class ARGS>
int launch_rows_partial(cas_ctx* ctx, const ARGS& a, int tiles, int items) {
  const dim3 grid((unsigned)items * (unsigned)a.g.n_kv_heads);
#define CAS_LAUNCH(TV)                                                           \
  case TV:                                                                       \
    return tiles == 2   ? launch_rows_tiles<TV, FULL, MX, 2, ARGS>(ctx, a, grid)       \
           : tiles == 4 ? launch_rows_tiles<TV, FULL, MX, 4, ARGS>(ctx, a, grid)       \
           : tiles == 8 ? launch_rows_tiles<TV, FULL, MX, 8, ARGS>(ctx, a, grid)       \
                        : launch_rows_tiles<TV, FULL, MX, 16, ARGS>(ctx, a, grid);
  switch (a.g.t) {
    CAS_LAUNCH(0) CAS_LAUNCH(1) CAS_LAUNCH(2) CAS_LAUNCH(3) CAS_LAUNCH(4) CAS_LAUNCH(5) CAS_LAUNCH(6) CAS_LAUNCH(7)
    default: return CAS_EINVAL;
  }
#undef CAS_LAUNCH
}

}  // namespace cas
