// Rotary positions for callers that drive the cache and the attention themselves: the table of cos and sin of a range of
// positions, with the frequencies scaled for long contexts, and the rotation of the heads of a projection at positions
// given one by one.  (The model passes rotate inside their own kernels, at the positions of the cache.)
#include <algorithm>
#include <cfloat>
#include <cmath>
#include "cas_device.hpp"
#include "cas_internal.hpp"

namespace cas {

constexpr int kRopePairs = 128;       // most pairs of a head
constexpr int kRopeTablePos = 16;     // positions of a thread

struct RopeFreqs {
  double quarter[kRopePairs];  // quarter turns per position of every pair
};

// sin and cos of a in [-pi/4, pi/4] (a little beyond for rounding) by their Taylor series: the first term left out is below
// 2e-9 and 2e-10.  Fused multiply-adds, so the error is that of the last two operations, about a unit in the last place.
__device__ __forceinline__ void sincos_eighth(float a, float& s, float& c) {
  const float z = a * a;
  s = fmaf(a * z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), a);
  c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
}

// Angles are formed and reduced to an eighth turn in 64 bits (four operations; position times frequency reaches 2^24 quarter
// turns of which 32 bits would leave nothing), the rest is fp32.  Bound by the writes: 67 MB for 131072 positions of 64 pairs
// in 13 us, 5.2 TB/s.
// A thread keeps its pair (PAIRS = 2: two, written as 16 bytes) over kRopeTablePos positions, so the frequency is read once.
template <int PAIRS>
__global__ __launch_bounds__(256) void rope_table_kernel(RopeFreqs f, int units, int rows, int pos0, int n_pos, float mag,
                                                         float* __restrict__ table) {
  const int row = (int)threadIdx.x / units, u = (int)threadIdx.x - row * units;
  if (row >= rows) return;  // units that do not divide the workgroup
  double fr[PAIRS];
#pragma unroll
  for (int k = 0; k < PAIRS; ++k) fr[k] = f.quarter[u * PAIRS + k];
  const int p0 = (int)blockIdx.x * rows * kRopeTablePos + row;
#pragma unroll 4
  for (int i = 0; i < kRopeTablePos; ++i) {
    const int p = p0 + i * rows;
    if (p >= n_pos) return;
    float v[2 * PAIRS];
#pragma unroll
    for (int k = 0; k < PAIRS; ++k) {
      const double t = (double)(pos0 + p) * fr[k], q = rint(t);
      const int quad = (int)(long long)q;
      float s, c;
      sincos_eighth((float)((t - q) * 1.5707963267948966), s, c);
      const float x = quad & 1 ? s : c, y = quad & 1 ? c : s;  // |cos|, |sin| change places every quarter turn
      v[2 * k] = mag * ((quad + 1) & 2 ? -x : x);
      v[2 * k + 1] = mag * (quad & 2 ? -y : y);
    }
    float* dst = table + ((size_t)p * units + u) * (2 * PAIRS);
    if constexpr (PAIRS == 2) *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<float2*>(dst) = make_float2(v[0], v[1]);
  }
}

constexpr int kRopeParts = 4;
struct RopePart {
  uint64_t x, y;      // where head 0 of the first token would be if all heads were the part's
  int64_t ldx, ldy;   // bytes
  int head0;          // heads of a token before the part; all heads for one that is not there
  int kind;           // bit 0: floats, bit 1: turns
};
struct RopeArgs {
  RopePart part[kRopeParts];
  const float* table;
  const int32_t* pos;
  int pos0, n_pos, n_tok, half, dim, heads, blocks;  // half: pairs of a head; heads: of all parts; blocks: workgroups of a token
  float sign;
};

// V consecutive values: requested as words (eight bf16 are four words, eight floats eight), and taken as floats: bf16 (exact) or floats
// rounded to bf16, as every tensor that passes from one operation to the next is
template <int V>
__device__ __forceinline__ void rope_request(uint64_t x, int at, bool fp32, uint32_t (&w)[V]) {
  const uint64_t src = x + (uint32_t)at * (fp32 ? 4u : 2u);
  if constexpr (V == 1) {
    if (fp32) w[0] = *reinterpret_cast<const uint32_t*>(src);
    else w[0] = *reinterpret_cast<const uint16_t*>(src);
  } else {
    const uint4 q = reinterpret_cast<const uint4*>(src)[0];
    w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
    if (fp32) {
      const uint4 r = reinterpret_cast<const uint4*>(src)[1];
      w[4] = r.x; w[5] = r.y; w[6] = r.z; w[7] = r.w;
    }
  }
}
template <int V>
__device__ __forceinline__ void rope_take(const uint32_t (&w)[V], bool fp32, float (&v)[V]) {
  if (fp32) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = round_bf16(__uint_as_float(w[i]));
  } else if constexpr (V == 1) {
    v[0] = bf16_to_f32((uint16_t)w[0]);
  } else {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}
template <int V>
__device__ __forceinline__ void rope_store(uint16_t* y, const float (&v)[V]) {
  if constexpr (V == 1) y[0] = f32_to_bf16(v[0]);
  else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16(v[2 * i]) | ((uint32_t)f32_to_bf16(v[2 * i + 1]) << 16);
    *reinterpret_cast<uint4*>(y) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The places of a head that one thread takes: with halves, V pairs (V values of either half) or V values behind the turning
// ones; interleaved, V/2 pairs (one for V = 1) or V values behind.
template <int V, bool INTER>
struct RopeUnits {
  static constexpr int kPairs = INTER && V > 1 ? V / 2 : V;
  static __host__ __device__ int turning(int half) { return half / kPairs; }
  static __host__ __device__ int of_head(int half, int dim) { return turning(half) + (dim - 2 * half) / V; }
};

// Bound by memory: every value is read and written once, a token's row of the table comes from a cache for all heads but
// the first.  A workgroup takes some heads of one token: `units` threads to a head, each with its part of the table's row in
// registers for all heads that it goes through.  4099 tokens of 40 heads of 256 values, 168 MB: 31 us, 5.4 TB/s (a
// copy of as much 33); 5 tokens of 48 heads of 128 values: 3.3 us, a launch.  Two, three or five heads of a thread requested at once: 30.6,
// 30.6, 31.0, and 512 tokens of fp32 heads 6.1 -> 6.4, 6.8, 8.7.  4096 tokens of 40 heads of 128, halves, 20 us; one value at a time
// (rows a value apart from the alignment) 42, 2.0 TB/s in accesses of 2 bytes a lane, of fp32 heads 30; heads of 80 of which 20 channels
// turn 41.
template <int V, bool INTER>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  using U = RopeUnits<V, INTER>;
  const int units = U::of_head(a.half, a.dim), turning = U::turning(a.half);
  const int slots = 256 / units, slot = (int)threadIdx.x / units, u = (int)threadIdx.x - slot * units;
  const int tok = __builtin_amdgcn_readfirstlane((int)blockIdx.x / a.blocks), block = (int)blockIdx.x - tok * a.blocks;
  const int p = a.pos ? a.pos[tok] : a.pos0 + tok;
  if (p < 0 || p >= a.n_pos || slot >= slots) return;  // padding, or a thread without a place
  const bool turns = u < turning;
  float c[U::kPairs], s[U::kPairs];
  if (turns) {
    const float2* row = reinterpret_cast<const float2*>(a.table) + (size_t)p * a.half + u * U::kPairs;
#pragma unroll
    for (int i = 0; i < U::kPairs; ++i) {
      const float2 cs = row[i];
      c[i] = cs.x;
      s[i] = a.sign * cs.y;
    }
  }
  // The parts in scalars: the arguments lie in host memory, and a load from there by
  // each lane, for its part, costs more than the head does: 44 us for the 4099 tokens from memory.
  RopePart part[kRopeParts];
#pragma unroll
  for (int i = 0; i < kRopeParts; ++i) {
    part[i] = a.part[i];
    part[i].x += (uint64_t)(tok * part[i].ldx);
    part[i].y += (uint64_t)(tok * part[i].ldy);
    asm("" : "+s"(part[i].x), "+s"(part[i].y), "+s"(part[i].head0), "+s"(part[i].kind));
  }
  // the thread's places in a head: V values, and as many in the other half
  const int e0 = !turns ? 2 * a.half + (u - turning) * V : INTER && V == 1 ? 2 * u : u * V;
  const int e1 = INTER ? 2 * u + 1 : a.half + u * V;
  const bool two = turns && !(INTER && V > 1);
  for (int h = block * slots + slot; h < a.heads; h += a.blocks * slots) {
    uint64_t x = part[0].x, y = part[0].y;
    int kind = part[0].kind;
#pragma unroll
    for (int i = 1; i < kRopeParts; ++i) {
      const bool in = h >= part[i].head0;
      x = in ? part[i].x : x;
      y = in ? part[i].y : y;
      kind = in ? part[i].kind : kind;
    }
    const bool fp32 = kind & 1, turn = turns && (kind & 2);
    uint16_t* const to = reinterpret_cast<uint16_t*>(y) + h * a.dim;
    uint32_t w0[V], w1[V];
    rope_request<V>(x, h * a.dim + e0, fp32, w0);
    if (two) rope_request<V>(x, h * a.dim + e1, fp32, w1);
    float v0[V];
    rope_take<V>(w0, fp32, v0);
    if constexpr (!INTER || V == 1) {
      if (two) {
        float v1[V];
        rope_take<V>(w1, fp32, v1);
        if (turn) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float p0 = v0[i], p1 = v1[i];
            v0[i] = p0 * c[i] - p1 * s[i];
            v1[i] = p1 * c[i] + p0 * s[i];
          }
        }
        rope_store<V>(to + e1, v1);
      }
    } else if (turn) {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const float p0 = v0[2 * i], p1 = v0[2 * i + 1];
        v0[2 * i] = p0 * c[i] - p1 * s[i];
        v0[2 * i + 1] = p1 * c[i] + p0 * s[i];
      }
    }
    rope_store<V>(to + e0, v0);
  }
}

template <int V, bool INTER>
static int launch_rope(cas_ctx* ctx, RopeArgs& a) {
  const int units = RopeUnits<V, INTER>::of_head(a.half, a.dim), slots = 256 / units;
  // few tokens: a workgroup for every 256/units heads; many: one for all heads of a token, whose table row is then read once
  const int most = (a.heads + slots - 1) / slots;
  a.blocks = std::max(1, std::min(most, 1024 / a.n_tok));
  const int64_t grid = (int64_t)a.n_tok * a.blocks;
  if (grid > 0xFFFFFF) return CAS_ENOTSUP;  // a launch has fewer than 2^32 threads
  hipLaunchKernelGGL((rope_kernel<V, INTER>), dim3((unsigned)grid), dim3(256), 0, ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

}  // namespace cas

static bool rope_cfg_ok(const cas_rope_cfg* c) {
  if (!c || c->rot < 2 || c->rot > 2 * cas::kRopePairs || (c->rot & 1)) return false;
  if (c->scaling < CAS_ROPE_PLAIN || c->scaling > CAS_ROPE_BANDS) return false;
  if (!(c->base >= 1.0) || !std::isfinite(c->base)) return false;
  if (!(c->magnitude >= (double)FLT_MIN) || !(c->magnitude <= (double)FLT_MAX)) return false;  // the table is fp32
  if (c->scaling != CAS_ROPE_PLAIN && (!(c->factor >= 1.0) || !std::isfinite(c->factor))) return false;
  if (c->scaling == CAS_ROPE_BASE && c->rot < 4) return false;
  if (c->scaling == CAS_ROPE_BANDS &&
      (c->trained < 1 || !(c->low >= 0.0) || !(c->high > c->low) || !std::isfinite(c->high)))
    return false;
  return true;
}

extern "C" {

int cas_rope_freqs(const cas_rope_cfg* cfg, double* h_freqs) {
  if (!rope_cfg_ok(cfg) || !h_freqs) return CAS_EINVAL;
  const double base = cfg->scaling == CAS_ROPE_BASE ? cfg->base * std::pow(cfg->factor, (double)cfg->rot / (cfg->rot - 2)) : cfg->base;
  for (int i = 0; i < cfg->rot / 2; ++i) {
    double f = std::pow(base, -2.0 * i / cfg->rot);
    if (cfg->scaling == CAS_ROPE_LINEAR) f /= cfg->factor;
    if (cfg->scaling == CAS_ROPE_BANDS) {
      const double turns = cfg->trained * f / 6.283185307179586;
      const double g = std::min(1.0, std::max(0.0, (turns - cfg->low) / (cfg->high - cfg->low)));
      f = g * f + (1.0 - g) * f / cfg->factor;
    }
    h_freqs[i] = f;
  }
  return CAS_OK;
}

int cas_rope_table(cas_ctx* ctx, const cas_rope_cfg* cfg, int pos0, int n_pos, float* d_table) {
  if (!ctx || !rope_cfg_ok(cfg) || pos0 < 0 || n_pos < 0 || (int64_t)pos0 + n_pos > (1 << 24)) return CAS_EINVAL;
  if (n_pos == 0) return CAS_OK;
  if (!d_table || !cas::aligned256(d_table) || !cas::on_device(ctx)) return CAS_EINVAL;
  cas::RopeFreqs f{};
  const int rc = cas_rope_freqs(cfg, f.quarter);
  if (rc != CAS_OK) return rc;
  for (int i = 0; i < cfg->rot / 2; ++i) f.quarter[i] *= 0.6366197723675814;  // 2 / pi
  const int half = cfg->rot / 2, pairs = half & 1 ? 1 : 2, units = half / pairs, rows = 256 / units;
  const dim3 grid((n_pos + rows * cas::kRopeTablePos - 1) / (rows * cas::kRopeTablePos));
  hipLaunchKernelGGL(pairs == 2 ? cas::rope_table_kernel<2> : cas::rope_table_kernel<1>, grid, dim3(256), 0, ctx->stream, f,
                     units, rows, pos0, n_pos, (float)cfg->magnitude, d_table);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

int cas_rope(cas_ctx* ctx, const float* d_table, int n_pos, int rot, int layout, int transposed, const int32_t* d_pos,
             int pos0, int n_tok, int head_dim, int n_parts, const cas_rope_part* h_parts) {
  if (!ctx || n_pos < 0 || n_tok < 0 || rot < 2 || (rot & 1) || head_dim < rot || n_parts < 1 || n_parts > cas::kRopeParts || !h_parts)
    return CAS_EINVAL;
  if (layout != CAS_ROPE_HALF && layout != CAS_ROPE_INTERLEAVED) return CAS_EINVAL;
  if (!d_pos && (int64_t)pos0 + n_tok > 0x7FFFFFFF) return CAS_EINVAL;
  if (head_dim > 2 * cas::kRopePairs) return CAS_ENOTSUP;
  cas::RopeArgs a{};
  const int half = rot / 2;
  // eight values at a time where every access then is 16 bytes on a multiple of 16; single pairs otherwise
  bool wide = head_dim % 8 == 0 && (layout == CAS_ROPE_HALF ? half % 8 == 0 : rot % 8 == 0);
  for (int i = 0; i < n_parts; ++i) {
    const cas_rope_part& p = h_parts[i];
    if (p.n_heads < 0 || p.n_heads > (1 << 16)) return CAS_EINVAL;
    const int64_t row = (int64_t)p.n_heads * head_dim;
    if (p.ldx < row || p.ldy < row) return CAS_EINVAL;
    const int64_t before = (int64_t)a.heads * head_dim, size = p.x_fp32 ? 4 : 2;
    a.part[i] = {(uint64_t)p.d_x - (uint64_t)(before * size), (uint64_t)p.d_y - (uint64_t)(before * 2), p.ldx * size, p.ldy * 2, a.heads,
                 (p.x_fp32 ? 1 : 0) | (p.turn ? 2 : 0)};
    a.heads += p.n_heads;
    if (row == 0 || n_tok == 0) continue;
    const uintptr_t x = (uintptr_t)p.d_x, y = (uintptr_t)p.d_y;
    if (!x || !y || x % (p.x_fp32 ? 4 : 2) || y % 2) return CAS_EINVAL;
    if (x == y && (p.x_fp32 || p.ldx != p.ldy)) return CAS_EINVAL;
    wide = wide && x % 16 == 0 && y % 16 == 0 && p.ldx % 8 == 0 && p.ldy % 8 == 0;
  }
  if (n_tok == 0 || n_pos == 0 || a.heads == 0) return CAS_OK;
  for (int i = n_parts; i < cas::kRopeParts; ++i) a.part[i].head0 = a.heads;
  if (!d_table || !cas::aligned256(d_table) || !cas::on_device(ctx)) return CAS_EINVAL;
  a.table = d_table; a.pos = d_pos; a.pos0 = pos0; a.n_pos = n_pos; a.n_tok = n_tok;
  a.half = half; a.dim = head_dim; a.sign = transposed ? -1.f : 1.f;
  if (layout == CAS_ROPE_HALF) return wide ? cas::launch_rope<8, false>(ctx, a) : cas::launch_rope<1, false>(ctx, a);
  return wide ? cas::launch_rope<8, true>(ctx, a) : cas::launch_rope<1, true>(ctx, a);
}

}  // extern "C"
