// Appending to the compressed cache with the position rotation on the way: q, k and v of the tokens of several sequences go from
// a projection to their places in one launch.  q is rounded, turned and written dense; k and v are rounded, turned
// and encoded into the pages (kv_append_kernel.inl has the encoders) without passing through memory as bf16.
//
//   y_a = x_a cos - x_b sin,  y_b = x_b cos + x_a sin      (fp32, an operation at a time, rounded to bf16 once)
//
// Every operation is the one that cas_rope does, so the bits are those of cas_rope followed by cas_kv_append.
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
  int append_blocks, q_blocks;          // workgroups that append; workgroups of a token's queries
  RopeAppendPart part[3];               // q, k, v
  int tok0[kRopeAppendSeqs];            // tokens of the sequences before; the largest number behind the last
  int block0[kRopeAppendSeqs];          // groups of sixteen rows of the sequences before; as above
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
    const float y0 = x0 * c0.x + o0 * (p0.first ? -c0.y : c0.y), y1 = x1 * c1.x + o1 * (p1.first ? -c1.y : c1.y);
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

// Eight channels 8 l .. 8 l + 7 of a vector, two to a word
__device__ __forceinline__ void load_eight(uint64_t row, int l, bool fp32, uint32_t (&w)[4]) {
  if (fp32) {
    float f[8];
    __builtin_memcpy(f, reinterpret_cast<const void*>(row + 32u * (uint32_t)l), 32);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16(f[2 * i]) | (uint32_t)f32_to_bf16(f[2 * i + 1]) << 16;
  } else {
    __builtin_memcpy(w, reinterpret_cast<const void*>(row + 16u * (uint32_t)l), 16);
  }
}
__device__ __forceinline__ float low_value(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_value(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// cos and sin (with the sign that its channel takes it with) of a lane's eight channels at one position
struct EightAngles {
  float c[8], s[8];
  __device__ __forceinline__ void load(const RopeAppendArgs& a, int p, int l) {
    const float2* cs = reinterpret_cast<const float2*>(a.angles) + (size_t)p * a.half;
    if (!a.inter && (a.half & 7) == 0) {  // eight channels of one half
      const Pairing at(8 * l, a.half, false);
      float f[16];
      __builtin_memcpy(f, cs + at.pair, 64);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[i] = f[2 * i];
        s[i] = at.first ? -f[2 * i + 1] : f[2 * i + 1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Pairing at(8 * l + i, a.half, a.inter);
        const float2 v = cs[at.pair];
        c[i] = v.x;
        s[i] = at.first ? -v.y : v.y;
      }
    }
  }
};
// Turns the lane's eight channels; row: 128 values of LDS of the vector's 16 lanes.  All 64 lanes of the wave call it together.
__device__ __forceinline__ void turn_eight(const RopeAppendArgs& a, const EightAngles& cs, int l, uint16_t* row, uint32_t (&w)[4]) {
  float other[8];
  if (a.inter) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      other[2 * i] = high_value(w[i]);
      other[2 * i + 1] = low_value(w[i]);
    }
  } else {
    *reinterpret_cast<uint4*>(row + 8 * l) = make_uint4(w[0], w[1], w[2], w[3]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if ((a.half & 7) == 0) {
      const uint4 o = *reinterpret_cast<const uint4*>(row + Pairing(8 * l, a.half, false).other);
      const uint32_t ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        other[2 * i] = low_value(ow[i]);
        other[2 * i + 1] = high_value(ow[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) other[i] = bf16_to_f32(row[Pairing(8 * l + i, a.half, false).other]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = 8 * l + 2 * i;
    const float y0 = low_value(w[i]) * cs.c[2 * i] + other[2 * i] * cs.s[2 * i];
    const float y1 = high_value(w[i]) * cs.c[2 * i + 1] + other[2 * i + 1] * cs.s[2 * i + 1];
    if (c < 2 * a.half) w[i] = (uint32_t)f32_to_bf16(y0) | (uint32_t)f32_to_bf16(y1) << 16;  // an even number of channels turns
  }
}

// A wave for four vectors, 16 lanes each: the tokens of four rows of a page (k, v), or four heads of a token (q).
template <int T, bool MX>
__global__ __launch_bounds__(64 * kAppendWaves) void rope_append_kernel(RopeAppendArgs a) {
  __shared__ __attribute__((aligned(16))) AppendStage stages[kAppendWaves];
  const KvGeom& g = a.g;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q = lane >> 4, l = lane & 15;
  AppendStage& st = stages[wv];
  const LaneTable t_tok0(a.tok0), t_seq(a.seq), t_len(a.len), t_n(a.n), t_block0(a.block0);
  int block = blockIdx.x;
  EightAngles cs;
  uint32_t w[4];
  if (block >= a.append_blocks) {  // the queries of a token
    block -= a.append_blocks;
    const int tok = block / a.q_blocks, first = (block - tok * a.q_blocks) * 4 * kAppendWaves + 4 * wv;
    const int s = t_tok0.which(tok), p = a.pos ? a.pos[tok] : t_len[s] + tok - t_tok0[s];
    if (p < 0 || p >= a.n_pos) return;
    const RopeAppendPart part = a.part[0];
    if (part.turn) cs.load(a, p, l);
    for (int h0 = first; h0 < a.n_q; h0 += a.q_blocks * 4 * kAppendWaves) {  // uniform in the wave
      const int head = min(h0 + q, a.n_q - 1);
      load_eight(part.x + (uint64_t)(tok * part.ldx) + (uint32_t)head * (part.fp32 ? 512u : 256u), l, part.fp32, w);
      if (part.turn) turn_eight(a, cs, l, st.kept[q], w);
      if (h0 + q < a.n_q)
        __builtin_memcpy(reinterpret_cast<uint16_t*>(part.y + (uint64_t)(tok * part.ldy)) + head * 128 + 8 * l, w, 16);
    }
    return;
  }
  const int head = block % g.n_kv_heads, kv = block / g.n_kv_heads & 1;
  block = block / g.n_kv_heads >> 1;
  const int s = t_block0.which(block), pos0 = t_len[s];
  const int posw = (pos0 & -kAppendRows) + (block - t_block0[s]) * kAppendRows + 4 * wv;  // place of the wave's first row
  const int ra = max(pos0 - posw, 0), rb = min(pos0 + t_n[s] - posw, 4);                  // the wave's rows ra .. rb - 1 are new
  if (ra >= rb) return;  // the waves do not wait for each other
  const int page = a.table[(size_t)t_seq[s] * g.max_pages_per_seq + posw / 64];
  const RopeAppendPart part = a.part[1 + kv];
  const int place = posw + min(max(q, ra), rb - 1), tok = t_tok0[s] + place - pos0;  // rows that are not new repeat one that is
  const int p = a.pos ? a.pos[tok] : place;
  const bool there = p >= 0 && p < a.n_pos;
  const uint64_t rows = __builtin_amdgcn_ballot_w64(there && q >= ra && q < rb);  // bit 16 r: row r is written
  if (rows == 0) return;
  load_eight(part.x + (uint64_t)(tok * part.ldx) + (uint32_t)head * (part.fp32 ? 512u : 256u), l, part.fp32, w);
  if (part.turn) {
    cs.load(a, there ? p : 0, l);
    turn_eight(a, cs, l, st.kept[q], w);
  }
  if (part.y && (rows >> (16 * q) & 1))
    __builtin_memcpy(reinterpret_cast<uint16_t*>(part.y + (uint64_t)(tok * part.ldy)) + head * 128 + 8 * l, w, 16);
  const bool gaps = __popcll(rows) != 16 * (rb - ra);  // some of the rows are padding
  format_four<T, MX>(g, a.spec_pool, a.verif_pool, st, w, lane, a.layer, page, kv, head, posw & 63, [&](int i, int words) {
    bool in = i >= ra * words && i < rb * words;
    if (gaps) in = in && (rows >> (16 * ((i >= words) + (i >= 2 * words) + (i >= 3 * words))) & 1);
    return in;
  });
}

static int launch_rope_append(cas_ctx* ctx, RopeAppendArgs& a, int n_seqs) {
  const KvGeom& g = a.g;
  // as launch_kv_append_layers chooses
  if ((int64_t)a.n_tok * g.n_kv_heads * 2 <= (int64_t)(g.mx ? 10 : 12) * ctx->num_cu) {
    const dim3 grid((a.n_tok + kAppendWaves - 1) / kAppendWaves, a.n_q + 2 * g.n_kv_heads);
    hipLaunchKernelGGL(rope_append_few_kernel, grid, dim3(64 * kAppendWaves), 0, ctx->stream, a);
    CAS_HIP(ctx, hipGetLastError());
    return CAS_OK;
  }
  int64_t groups = 0;
  for (int i = 0; i < n_seqs; ++i) {
    a.block0[i] = (int)groups;
    if (a.n[i] > 0) groups += (a.len[i] + a.n[i] - 1) / kAppendRows - a.len[i] / kAppendRows + 1;
  }
  for (int i = n_seqs; i < kRopeAppendSeqs; ++i) a.block0[i] = 0x7FFFFFFF;
  a.q_blocks = a.n_q > 0 ? std::max(1, std::min((a.n_q + 4 * kAppendWaves - 1) / (4 * kAppendWaves), 1024 / a.n_tok)) : 0;
  const int64_t grid = groups * g.n_kv_heads * 2 + (int64_t)a.n_tok * a.q_blocks;
  if (grid > 0xFFFFFF) return CAS_ENOTSUP;  // a launch has fewer than 2^32 threads
  a.append_blocks = (int)(groups * g.n_kv_heads * 2);
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
    if ((int64_t)a.len[i] + a.n[i] > (int64_t)kv->desc.max_pages_per_seq * kv->desc.page_tokens) return CAS_ENOMEM;
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
