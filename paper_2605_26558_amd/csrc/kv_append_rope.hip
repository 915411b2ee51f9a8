// Appending to the compressed cache with the position rotation on the way: q, k and v of the tokens of several sequences go from
// a projection to their places in one launch.  q is rounded, turned and written dense; k and v are rounded, turned
// and encoded into the pages (kv_append_kernel.inl has the encoders) without passing through memory as bf16.
//
//   y_a = x_a cos - x_b sin,  y_b = x_b cos + x_a sin      (fp32, an operation at a time, rounded to bf16 once)
//
// Every operation is the one that cas_rope does, so the bits are those of cas_rope followed by cas_kv_append, infinities and NaN
// included, unless both products of a sum are NaN: which of two an addition passes on goes by the order of its operands, the compiler's choice.
//
// What has to move: the projections once, the dense queries and the encoded vectors once.  Measured (60 % kept, t = 4; us; in brackets these bytes at the rate
// of a copy): 3 tokens of 48 heads 4.1 (0.02) and 101 of 80 heads in 32 sequences 6.6 (1.3), the launch and three round trips (arguments,
// position, angles); 4099 tokens of 48 fp32 heads 32.0 (30.3), memory; 8000 tokens of K and V of 8 heads 25.4 (13.9): all waves are on the chip at
// about the same time and read (7), turn (5), encode (6) and write (6) more or less together.  Four lanes read a vector's eights side by side and
// exchange them through LDS only after the turn: with 32 channels that follow one another for each lane from the start the two took 36.6 and 30.4,
// as a load of the angles then touches 64 lines.
#include <algorithm>
#include "kv_append_kernel.inl"

namespace cas {

constexpr int kRopeAppendSeqs = 32;  // sequences of a call

struct RopeAppendPart {
  uint64_t x, y;     // y: 0 for none
  int64_t ldx, ldy;  // bytes
  int fp32, turn;
};
struct RopeAppendArgs {
  KvGeom g;
  uint32_t* spec_pool;
  uint32_t* verif_pool;
  const int32_t* table;   // pages
  const float* angles;    // cos, sin
  const int32_t* pos;     // NULL: the place in the cache
  int n_pos, half, inter, layer, n_tok, n_q;
  int units, append_blocks, q_blocks;   // waves and workgroups that append; workgroups of a token's queries
  RopeAppendPart part[3];               // q, k, v
  int tok0[kRopeAppendSeqs];            // tokens of the sequences before; the largest number behind the last
  int group0[kRopeAppendSeqs];          // groups of sixteen rows of the sequences before; as above
  int seq[kRopeAppendSeqs], len[kRopeAppendSeqs], n[kRopeAppendSeqs];
};

// A table of the sequences, an entry per lane: the arguments lie in host memory, and loads from there whose place depends on
// another cost a trip each.
struct LaneTable {
  int v;
  __device__ __forceinline__ explicit LaneTable(const int (&t)[kRopeAppendSeqs]) : v(t[threadIdx.x & (kRopeAppendSeqs - 1)]) {}
  // of the numbers before each: the sequence whose share holds n
  __device__ __forceinline__ int which(int n) const { return __popc((uint32_t)__builtin_amdgcn_ballot_w64(n >= v)) - 1; }
  __device__ __forceinline__ int operator[](int s) const { return __builtin_amdgcn_readlane(v, s); }
};

__device__ __forceinline__ float value_at(uint64_t row, int c, bool fp32) {  // rounded to bf16
  return fp32 ? round_bf16(reinterpret_cast<const float*>(row)[c]) : bf16_to_f32(reinterpret_cast<const uint16_t*>(row)[c]);
}
// The channel that turns with c (c itself for none), their pair in the table, and whether c is the first of the two
struct Pairing {
  int other, pair;
  bool first, turns;
  __device__ __forceinline__ Pairing(int c, int half, bool inter) {
    turns = c < 2 * half;
    first = inter ? !(c & 1) : c < half;
    other = !turns ? c : inter ? c ^ 1 : first ? c + half : c - half;
    pair = !turns ? 0 : inter ? c >> 1 : first ? c : c - half;
  }
};

// x + p, or x - p for minus = the sign bit (the first of a pair).  The sign goes to the product, as a subtraction's does, and not to
// one of its factors: of a NaN the factor, or infinity times 0, it would come out otherwise.
__device__ __forceinline__ float plus(float x, float p, uint32_t minus) { return x + __uint_as_float(__float_as_uint(p) ^ minus); }
constexpr uint32_t kMinus = 0x80000000u;

// A wave per vector: lane l has channels l and l + 64.  For few tokens, where the time of one wave from end to end counts.
__global__ __launch_bounds__(64 * kAppendWaves) void rope_append_few_kernel(RopeAppendArgs a) {
  __shared__ uint32_t stages[kAppendWaves][3 * 64 + 8];  // as in kv_append_few_kernel
  const KvGeom& g = a.g;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tok = blockIdx.x * kAppendWaves + wv, unit = blockIdx.y;
  if (tok >= a.n_tok) return;  // the waves do not wait for each other
  const LaneTable t_tok0(a.tok0), t_seq(a.seq), t_len(a.len);
  const int which = unit < a.n_q ? 0 : unit < a.n_q + g.n_kv_heads ? 1 : 2;
  const int head = which == 0 ? unit : which == 1 ? unit - a.n_q : unit - a.n_q - g.n_kv_heads;
  const RopeAppendPart part = a.part[which];
  const uint64_t src = part.x + (uint64_t)(tok * part.ldx) + (uint32_t)head * (part.fp32 ? 512u : 256u);
  const bool fp32 = part.fp32, turn = part.turn;
  const Pairing p0(lane, a.half, a.inter), p1(lane + 64, a.half, a.inter);
  float x0 = value_at(src, lane, fp32), x1 = value_at(src, lane + 64, fp32), o0 = 0.f, o1 = 0.f;
  if (turn) {
    o0 = value_at(src, p0.other, fp32);
    o1 = value_at(src, p1.other, fp32);
  }
  const int s = t_tok0.which(tok), place = t_len[s] + tok - t_tok0[s];
  const int p = a.pos ? a.pos[tok] : place;
  int page = 0;
  if (which != 0) page = a.table[(size_t)t_seq[s] * g.max_pages_per_seq + place / 64];
  if (p < 0 || p >= a.n_pos) return;  // padding
  if (turn) {
    const float2* cs = reinterpret_cast<const float2*>(a.angles) + (size_t)p * a.half;
    const float2 c0 = cs[p0.pair], c1 = cs[p1.pair];
    const float y0 = plus(x0 * c0.x, o0 * c0.y, p0.first ? kMinus : 0u), y1 = plus(x1 * c1.x, o1 * c1.y, p1.first ? kMinus : 0u);
    x0 = p0.turns ? y0 : x0;
    x1 = p1.turns ? y1 : x1;
  }
  const uint32_t v0 = f32_to_bf16(x0), v1 = f32_to_bf16(x1);
  if (part.y) {
    uint16_t* const dst = reinterpret_cast<uint16_t*>(part.y + (uint64_t)(tok * part.ldy)) + head * 128;
    dst[lane] = (uint16_t)v0;
    dst[lane + 64] = (uint16_t)v1;
  }
  if (which == 0) return;
  format_one(g, a.spec_pool, a.verif_pool, stages[wv], v0, v1, lane, a.layer, page, which - 1, head, place & 63);
}

typedef float rope_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 rope_bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t two_bf16(float x, float y) {  // in one operation
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(rope_f32x2{x, y}, rope_bf16x2));
}
// N eights of channels of a vector, from c on and 32 apart, rounded, two to a word
template <int N>
__device__ __forceinline__ void request(uint64_t row, int c, bool fp32, uint32_t (&x)[N][4]) {
  if (fp32) {
    float raw[N][8];
#pragma unroll
    for (int k = 0; k < N; ++k) __builtin_memcpy(raw[k], reinterpret_cast<const float*>(row) + c + 32 * k, 32);
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[k][i] = two_bf16(raw[k][2 * i], raw[k][2 * i + 1]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) __builtin_memcpy(x[k], reinterpret_cast<const uint16_t*>(row) + c + 32 * k, 16);
  }
}
__device__ __forceinline__ float low_value(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_value(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// bf16 values that do not turn, as the conversion leaves them that turned and fp32 values go through: a NaN quiet
__device__ __forceinline__ void quiet(uint32_t (&w)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = two_bf16(low_value(w[i]), high_value(w[i]));
}

// How the partners of eight channels from a multiple of eight on are reached: half a vector away, in the same words, eight that follow one
// another, or one by one
enum Partners { kHalfAway, kNeighbours, kEights, kSingles };
__device__ __forceinline__ Partners partners_of(const RopeAppendArgs& a) {
  return a.inter ? kNeighbours : a.half == 64 ? kHalfAway : (a.half & 7) == 0 ? kEights : kSingles;
}
// Calls f with the kind as a constant: as branches inside, the kinds' registers add up (64 to 188 of them spilled)
template <class F>
__device__ __forceinline__ void with_partners(const RopeAppendArgs& a, F&& f) {
  switch (partners_of(a)) {
    case kHalfAway: f(std::integral_constant<int, kHalfAway>{}); break;
    case kNeighbours: f(std::integral_constant<int, kNeighbours>{}); break;
    case kEights: f(std::integral_constant<int, kEights>{}); break;
    default: f(std::integral_constant<int, kSingles>{});
  }
}

// cos and sin of channels c0 .. c0 + 7 at one position
template <int HOW>
struct EightAngles {
  float c[8], s[8];
  __device__ __forceinline__ void load(const RopeAppendArgs& a, int p, int c0) {
    const float2* cs = reinterpret_cast<const float2*>(a.angles) + (size_t)p * a.half;
    if constexpr (HOW == kHalfAway || HOW == kEights) {  // eight channels of one half
      float f[16];
      __builtin_memcpy(f, cs + Pairing(c0, a.half, false).pair, 64);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[i] = f[2 * i];
        s[i] = f[2 * i + 1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (HOW == kNeighbours && (i & 1)) {
          c[i] = c[i - 1];
          s[i] = s[i - 1];
        } else {
          const float2 v = cs[Pairing(c0 + i, a.half, HOW == kNeighbours).pair];
          c[i] = v.x;
          s[i] = v.y;
        }
      }
    }
  }
  // w: channels c0 .. c0 + 7, two to a word; o: their partners; first: whether they are the first of their pairs (HOW = kHalfAway)
  __device__ __forceinline__ void turn(const RopeAppendArgs& a, int c0, const uint32_t (&o)[4], uint32_t (&w)[4], bool first = false) const {
    const Pairing all(c0, a.half, false);  // eight channels that follow one another are alike but for kSingles
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t minus0, minus1;
      bool turns = true;
      if constexpr (HOW == kHalfAway) {
        minus0 = minus1 = first ? kMinus : 0u;
      } else if constexpr (HOW == kNeighbours) {
        minus0 = kMinus;
        minus1 = 0u;
        turns = c0 + 2 * i < 2 * a.half;  // an even number of channels turns
      } else if constexpr (HOW == kEights) {
        minus0 = minus1 = all.first ? kMinus : 0u;
        turns = all.turns;
      } else {
        const Pairing p0(c0 + 2 * i, a.half, false), p1(c0 + 2 * i + 1, a.half, false);
        minus0 = p0.first ? kMinus : 0u;
        minus1 = p1.first ? kMinus : 0u;
        turns = p0.turns;
      }
      const float x0 = low_value(w[i]), x1 = high_value(w[i]);
      const float y0 = plus(x0 * c[2 * i], low_value(o[i]) * s[2 * i], minus0), y1 = plus(x1 * c[2 * i + 1], high_value(o[i]) * s[2 * i + 1], minus1);
      w[i] = two_bf16(turns ? y0 : x0, turns ? y1 : x1);
    }
  }
};
// The partners of channels c0 .. c0 + 7 where they are not in words of the lane's own: of the words themselves, or out of the vector's values in LDS
template <int HOW>
__device__ __forceinline__ void partners(const RopeAppendArgs& a, int c0, const VectorRow& row, const uint32_t (&w)[4], uint32_t (&o)[4]) {
  if constexpr (HOW == kNeighbours) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_alignbit(w[i], w[i], 16);
  } else if constexpr (HOW == kEights) {
    row.eight(Pairing(c0, a.half, false).other, o);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      o[i] = row.one(Pairing(c0 + 2 * i, a.half, false).other) | row.one(Pairing(c0 + 2 * i + 1, a.half, false).other) << 16;
  }
}

// Sixteen vectors to a wave: the tokens of sixteen rows of a page (k, v; four lanes each), or four heads of a token at a time (q; 16
// lanes each).  A workgroup's waves do not wait for each other.
template <int T, bool MX>
__global__ __launch_bounds__(64 * kAppendWaves, 6) void rope_append_kernel(RopeAppendArgs a) {
  __shared__ __attribute__((aligned(16))) RowsStage stages[kAppendWaves];
  const KvGeom& g = a.g;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowsStage& st = stages[wv];
  const LaneTable t_tok0(a.tok0), t_seq(a.seq), t_len(a.len), t_n(a.n), t_group0(a.group0);
  auto share = [] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  if ((int)blockIdx.x >= a.append_blocks) {  // the queries of a token
    const int block = (int)blockIdx.x - a.append_blocks, q = lane >> 4, l = lane & 15;
    const int tok = block / a.q_blocks, first = (block - tok * a.q_blocks) * 4 * kAppendWaves + 4 * wv;
    const int s = t_tok0.which(tok), p = a.pos ? a.pos[tok] : t_len[s] + tok - t_tok0[s];
    if (p < 0 || p >= a.n_pos) return;
    const RopeAppendPart part = a.part[0];
    auto heads = [&](auto&& turn) {
      for (int h0 = first; h0 < a.n_q; h0 += a.q_blocks * 4 * kAppendWaves) {  // uniform in the wave
        const int head = min(h0 + q, a.n_q - 1);
        uint32_t x[1][4];
        uint32_t (&w)[4] = x[0];
        request(part.x + (uint64_t)(tok * part.ldx) + (uint32_t)head * (part.fp32 ? 512u : 256u), 8 * l, part.fp32, x);
        turn(w);
        if (h0 + q < a.n_q)
          __builtin_memcpy(reinterpret_cast<uint16_t*>(part.y + (uint64_t)(tok * part.ldy)) + head * 128 + 8 * l, w, 16);
      }
    };
    if (!part.turn) {
      heads([&](uint32_t (&w)[4]) {
        if (!part.fp32) quiet(w);
      });
      return;
    }
    with_partners(a, [&](auto H) {
      constexpr int how = decltype(H)::value;
      EightAngles<how> cs;
      cs.load(a, p, 8 * l);
      heads([&](uint32_t (&w)[4]) {
        uint32_t o[4];
        if constexpr (how == kHalfAway) {
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[i], 0x128, 0xf, 0xf, true);  // row_ror:8
        } else {
          const VectorRow row(st, q);
          if constexpr (how >= kEights) {
            row.put(8 * l, w);
            share();
          }
          partners<how>(a, 8 * l, row, w, o);
          if constexpr (how >= kEights) share();
        }
        cs.turn(a, 8 * l, o, w, l < 8);
      });
    });
    return;
  }
  const int unit = (int)blockIdx.x * kAppendWaves + wv;
  if (unit >= a.units) return;
  const int rest = unit / g.n_kv_heads, head = unit - rest * g.n_kv_heads, kv = rest & 1, group = rest >> 1;
  const int r = lane >> 2, c0 = 8 * (lane & 3);  // the lane's channels: c0 + 32 k .. c0 + 32 k + 7, as four lanes read side by side
  const int s = t_group0.which(group), pos0 = t_len[s];
  const int posw = (pos0 & -kAppendRows) + (group - t_group0[s]) * kAppendRows;     // place of the wave's first row
  const int ra = max(pos0 - posw, 0), rb = min(pos0 + t_n[s] - posw, kAppendRows);  // the wave's rows ra .. rb - 1 are new
  const RopeAppendPart part = a.part[1 + kv];
  const int place = posw + min(max(r, ra), rb - 1), tok = t_tok0[s] + place - pos0;  // rows that are not new repeat one that is
  const int p = a.pos ? a.pos[tok] : place;
  const int page = a.table[(size_t)t_seq[s] * g.max_pages_per_seq + posw / 64];
  asm volatile("" ::: "memory");
  uint32_t x[4][4];
  request(part.x + (uint64_t)(tok * part.ldx) + (uint32_t)head * (part.fp32 ? 512u : 256u), c0, part.fp32, x);
  const uint64_t lanes = __builtin_amdgcn_ballot_w64(p >= 0 && p < a.n_pos && r >= ra && r < rb);
  if (lanes == 0) return;
  uint32_t rows = 0;  // those that are written
#pragma unroll
  for (int i = 0; i < kAppendRows; ++i) rows |= (uint32_t)(lanes >> (4 * i) & 1) << i;
  const VectorRow row(st, r);
  if (part.turn) {
    const int at = min(max(p, 0), a.n_pos - 1);
    with_partners(a, [&](auto H) {
      constexpr int how = decltype(H)::value;
      if constexpr (how == kHalfAway) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          EightAngles<how> cs;
          uint32_t o[4];
          cs.load(a, at, c0 + 32 * k);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = x[k][i];
          cs.turn(a, c0 + 32 * k, x[k + 2], x[k], true);
          cs.turn(a, c0 + 32 * k, o, x[k + 2], false);
          asm volatile("" ::: "memory");  // the angles of all at once do not fit the registers
        }
      } else {
        if constexpr (how >= kEights) {
#pragma unroll
          for (int k = 0; k < 4; ++k) row.put(c0 + 32 * k, x[k]);
          share();
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          EightAngles<how> cs;
          uint32_t o[4];
          cs.load(a, at, c0 + 32 * k);
          partners<how>(a, c0 + 32 * k, row, x[k], o);
          cs.turn(a, c0 + 32 * k, o, x[k]);
          asm volatile("" ::: "memory");
        }
        if constexpr (how >= kEights) share();
      }
    });
  }
  const bool loud = !part.turn && !part.fp32;  // see quiet(); what the cache alone gets is looked through on bit planes, a third of the operations
  if (loud && part.y) {
#pragma unroll
    for (int k = 0; k < 4; ++k) quiet(x[k]);
  }
  if (part.y && (rows >> r & 1)) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      __builtin_memcpy(reinterpret_cast<uint16_t*>(part.y + (uint64_t)(tok * part.ldy)) + head * 128 + c0 + 32 * k, x[k], 16);
  }
  row.swap(x, lane & 3);
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    w[2 * i] = low_pair(x[i >> 2][i & 3], x[2 + (i >> 2)][i & 3]);
    w[2 * i + 1] = high_pair(x[i >> 2][i & 3], x[2 + (i >> 2)][i & 3]);
  }
  format_rows<T, MX>(g, a.spec_pool, a.verif_pool, st, w, lane, a.layer, page, kv, head, posw & 63, rows, loud && !part.y);
}

static int launch_rope_append(cas_ctx* ctx, RopeAppendArgs& a, int n_seqs) {
  const KvGeom& g = a.g;
  int64_t groups = 0;
  for (int i = 0; i < n_seqs; ++i) {
    a.group0[i] = (int)groups;
    if (a.n[i] > 0) groups += (a.len[i] + a.n[i] - 1) / kAppendRows - a.len[i] / kAppendRows + 1;
  }
  for (int i = n_seqs; i < kRopeAppendSeqs; ++i) a.group0[i] = 0x7FFFFFFF;
  const int64_t units = groups * g.n_kv_heads * 2, vectors = (int64_t)a.n_tok * (g.n_kv_heads * 2 + a.n_q / 4);
  // A wave a vector up to 20 vectors of K and V per CU (four of a token's queries count as one) and three more for each wave that the groups of
  // sixteen rows would make per CU, however few of their rows are new; 26 and 3.5 over shared exponents.  us, one / sixteen a wave: tokens of 8
  // heads bf16 without queries from a whole group on: 256 5.3 / 6.5, 384 6.5 / 6.5, 512 7.8 / 6.6, 1021 13.0 / 7.9; fp32 with 32 query heads: 192 6.7 / 6.9,
  // 256 7.6 / 7.2, 512 12.5 / 8.3; over shared exponents 384 7.0 / 8.3, 512 8.3 / 8.3, 640 9.6 / 8.3 and 320 9.2 / 9.0, 384 10.5 / 9.4.  32 sequences, fp32, tokens
  // each and heads of q, k and v: 12 of 32 + 8 + 8 10.4 / 9.3, 6 of 16 + 16 + 16 8.2 / 10.1, 12 12.5 / 11.1, 4 of 32 + 32 + 32 9.2 / 12.3, 8 16.0 / 13.7, 2 of 64
  // + 64 + 64 9.2 / 15.8, 4 15.7 / 16.9, 6 22.6 / 19.0; over shared exponents 10.8 / 10.7, 8.6 / 11.9, 13.1 / 12.8, 9.6 / 15.1, 16.7 / 16.2, 9.6 / 20.1, 16.3 /
  // 21.1, 23.7 / 23.7
  if (g.mx ? 2 * vectors <= 52 * ctx->num_cu + 7 * units : vectors <= 20 * ctx->num_cu + 3 * units) {
    const dim3 grid((a.n_tok + kAppendWaves - 1) / kAppendWaves, a.n_q + 2 * g.n_kv_heads);
    hipLaunchKernelGGL(rope_append_few_kernel, grid, dim3(64 * kAppendWaves), 0, ctx->stream, a);
    CAS_HIP(ctx, hipGetLastError());
    return CAS_OK;
  }
  a.q_blocks = a.n_q > 0 ? std::max(1, std::min((a.n_q + 4 * kAppendWaves - 1) / (4 * kAppendWaves), 1024 / a.n_tok)) : 0;
  if (units > 0x7FFFFFFF) return CAS_ENOTSUP;
  a.units = (int)units;
  a.append_blocks = (int)((units + kAppendWaves - 1) / kAppendWaves);
  const int64_t grid = a.append_blocks + (int64_t)a.n_tok * a.q_blocks;
  if (grid > 0xFFFFFF) return CAS_ENOTSUP;  // a launch has fewer than 2^32 threads
#define CAS_LAUNCH(TV)                                                                                                        \
  case TV:                                                                                                                    \
    hipLaunchKernelGGL(g.mx ? (rope_append_kernel<TV, true>) : (rope_append_kernel<TV, false>), dim3((unsigned)grid),         \
                       dim3(64 * kAppendWaves), 0, ctx->stream, a);                                                           \
    break;
  switch (g.t) {
    CAS_LAUNCH(0) CAS_LAUNCH(1) CAS_LAUNCH(2) CAS_LAUNCH(3) CAS_LAUNCH(4) CAS_LAUNCH(5) CAS_LAUNCH(6) CAS_LAUNCH(7)
    default: return CAS_EINVAL;
  }
#undef CAS_LAUNCH
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

}  // namespace cas

extern "C" int cas_kv_append_rope(cas_ctx* ctx, cas_kv* kv, int layer, int n_seqs, const int32_t* h_seqs, const int32_t* h_n_tok,
                                  const float* d_table, int n_pos, int rot, int layout, const int32_t* d_pos, const cas_rope_part* h_q,
                                  const cas_rope_part* h_k, const cas_rope_part* h_v) {
  if (!ctx || !kv || layer < 0 || layer >= kv->desc.n_layers || n_seqs < 0 || n_seqs > cas::kRopeAppendSeqs || n_pos < 0) return CAS_EINVAL;
  if (n_seqs > 0 && (!h_seqs || !h_n_tok)) return CAS_EINVAL;
  if (rot < 2 || rot > 128 || (rot & 1) || (layout != CAS_ROPE_HALF && layout != CAS_ROPE_INTERLEAVED) || !h_k || !h_v) return CAS_EINVAL;
  cas::RopeAppendArgs a{};
  a.g = kv->geom;
  int64_t n_tok = 0;
  for (int i = 0; i < n_seqs; ++i) {
    if (h_seqs[i] < 0 || h_seqs[i] >= kv->desc.max_seqs || h_n_tok[i] < 0) return CAS_EINVAL;
    for (int j = 0; j < i; ++j)
      if (h_seqs[j] == h_seqs[i]) return CAS_EINVAL;
    a.seq[i] = h_seqs[i]; a.len[i] = kv->h_len[h_seqs[i]]; a.n[i] = h_n_tok[i];
    if ((int64_t)a.len[i] + a.n[i] > cas::kv_room(kv)) return CAS_ENOMEM;
    a.tok0[i] = (int)n_tok;
    n_tok += h_n_tok[i];
    if (n_tok >= 1 << 24) return CAS_ENOTSUP;
  }
  for (int i = n_seqs; i < cas::kRopeAppendSeqs; ++i) a.tok0[i] = 0x7FFFFFFF;
  const cas_rope_part* parts[3] = {h_q, h_k, h_v};
  for (int i = 0; i < 3; ++i) {
    if (!parts[i]) continue;  // no queries
    const cas_rope_part& p = *parts[i];
    if (p.n_heads < 0 || (i > 0 && p.n_heads != a.g.n_kv_heads)) return CAS_EINVAL;
    const int64_t row = (int64_t)p.n_heads * 128;
    if (p.ldx < row || (p.d_y && p.ldy < row)) return CAS_EINVAL;
    if (i == 0) a.n_q = p.n_heads;
    a.part[i] = {(uint64_t)p.d_x, (uint64_t)p.d_y, p.ldx * (p.x_fp32 ? 4 : 2), p.ldy * 2, p.x_fp32 ? 1 : 0, p.turn ? 1 : 0};
    if (row == 0 || n_tok == 0) continue;
    const uintptr_t x = (uintptr_t)p.d_x, y = (uintptr_t)p.d_y;
    if (!x || (i == 0 && !y) || x % (p.x_fp32 ? 4 : 2) || y % 2) return CAS_EINVAL;
    if (x == y && (p.x_fp32 || p.ldx != p.ldy)) return CAS_EINVAL;
  }
  if ((int64_t)a.n_q + 2 * a.g.n_kv_heads > 65535) return CAS_ENOTSUP;
  if (n_tok == 0 || n_pos == 0) return CAS_OK;
  if (!d_table || !cas::aligned256(d_table) || (uintptr_t)d_pos % 4 || !cas::on_device(ctx)) return CAS_EINVAL;
  a.spec_pool = (uint32_t*)kv->d_spec;
  a.verif_pool = (uint32_t*)kv->d_verif;
  a.table = kv->d_page_table;
  a.angles = d_table; a.pos = d_pos; a.n_pos = n_pos; a.half = rot / 2; a.inter = layout == CAS_ROPE_INTERLEAVED;
  a.layer = layer; a.n_tok = (int)n_tok;
  return cas::launch_rope_append(ctx, a, n_seqs);
}
