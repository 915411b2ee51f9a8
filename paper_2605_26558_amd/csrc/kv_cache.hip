// Compressed, paged KV cache: online formatting of new K/V vectors (Sec. 5.1 encoder,
// Sec. 4.2 per-token magnitude pruning) and a reference read-back.
//
// A tile holds the vectors of one (layer, page, K-or-V, kv head): page_tokens rows of
// head_dim = 128 values, K kept per row, in the same four-stream layout as a weight matrix
// (bitmap and spec in the speculation pool; lo and pruned in the verification pool).
#include "kv_append_kernel.inl"
#include "kv_value.hpp"

namespace cas {

template <int T, bool MX>
__global__ __launch_bounds__(64 * kAppendWaves) void kv_append_kernel(KvGeom g, uint32_t* spec_pool, uint32_t* verif_pool,
                                                                      const int32_t* __restrict__ page_row, int layer0,
                                                                      int pos0, int n_tok, const uint16_t* __restrict__ Kn,
                                                                      const uint16_t* __restrict__ Vn, size_t layer_stride) {
  __shared__ __attribute__((aligned(16))) AppendStage stages[kAppendWaves];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  AppendStage& st = stages[wv];
  // grid.z = 2 * (layers of this launch): the vectors of layer layer0 + i start i * layer_stride
  // values after those of layer0
  const int head = blockIdx.y, kv = blockIdx.z & 1, layer = layer0 + (blockIdx.z >> 1);
  const int posw = (pos0 & -kAppendRows) + blockIdx.x * kAppendRows + 4 * wv;  // position of the wave's first row
  const int ra = max(pos0 - posw, 0), rb = min(pos0 + n_tok - posw, 4);        // the wave's rows ra .. rb - 1 are new
  if (ra >= rb) return;  // the waves do not wait for each other
  const int page = page_row[posw / 64], row = posw % 64;
  const int q = lane >> 4, l = lane & 15;  // vector of the wave, columns 8 l .. 8 l + 7
  const int tok = posw + min(max(q, ra), rb - 1) - pos0;  // rows that are not new repeat one that is
  const uint16_t* src = (kv ? Vn : Kn) + (size_t)(blockIdx.z >> 1) * layer_stride +
                        ((size_t)tok * g.n_kv_heads + head) * 128 + 8 * l;
  uint32_t w[4];  // columns 2 i and 2 i + 1
  __builtin_memcpy(w, src, 16);

  format_four<T, MX>(g, spec_pool, verif_pool, st, w, lane, layer, page, kv, head, row,
                     [&](int i, int words) { return i >= ra * words && i < rb * words; });
}

// Sixteen vectors to a wave, for many
template <int T, bool MX>
__global__ __launch_bounds__(64 * kAppendWaves) void kv_append_rows_kernel(KvGeom g, uint32_t* spec_pool, uint32_t* verif_pool,
                                                                           const int32_t* __restrict__ page_row, int layer0,
                                                                           int pos0, int n_tok, const uint16_t* __restrict__ Kn,
                                                                           const uint16_t* __restrict__ Vn, size_t layer_stride) {
  __shared__ __attribute__((aligned(16))) RowsStage stages[kAppendWaves];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // grid.z = 2 * (layers of this launch), as above
  const int head = blockIdx.y, kv = blockIdx.z & 1, layer = layer0 + (blockIdx.z >> 1);
  const int posw = (pos0 & -kAppendRows) + (blockIdx.x * kAppendWaves + wv) * kAppendRows;  // position of the wave's first row
  const int ra = max(pos0 - posw, 0), rb = min(pos0 + n_tok - posw, kAppendRows);           // the wave's rows ra .. rb - 1 are new
  if (ra >= rb) return;  // the waves do not wait for each other
  const int page = page_row[posw / 64];
  const int tok = posw + min(max(lane >> 2, ra), rb - 1) - pos0;  // rows that are not new repeat one that is
  const uint16_t* src = (kv ? Vn : Kn) + (size_t)(blockIdx.z >> 1) * layer_stride +
                        ((size_t)tok * g.n_kv_heads + head) * 128 + 8 * (lane & 3);
  uint32_t x[4][4], w[16];
#pragma unroll
  for (int k = 0; k < 4; ++k) __builtin_memcpy(x[k], src + 32 * k, 16);
  VectorRow(stages[wv], lane >> 2).swap(x, lane & 3);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    w[2 * i] = low_pair(x[i >> 2][i & 3], x[2 + (i >> 2)][i & 3]);
    w[2 * i + 1] = high_pair(x[i >> 2][i & 3], x[2 + (i >> 2)][i & 3]);
  }
  format_rows<T, MX>(g, spec_pool, verif_pool, stages[wv], w, lane, layer, page, kv, head, posw & 63, (0xFFFFu << ra) & (0xFFFFu >> (kAppendRows - rb)));
}

__global__ __launch_bounds__(64 * kAppendWaves) void kv_append_few_kernel(KvGeom g, uint32_t* spec_pool, uint32_t* verif_pool,
                                                                          const int32_t* __restrict__ page_row, int layer0,
                                                                          int pos0, int n_tok, const uint16_t* __restrict__ Kn,
                                                                          const uint16_t* __restrict__ Vn, size_t layer_stride) {
  __shared__ uint32_t stages[kAppendWaves][3 * 64 + 8];  // sw + lw + pw <= 16*128/32 = 64 words (+ rounding)
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t* const stage = stages[wv];
  // grid.z = 2 * (layers of this launch): the vectors of layer layer0 + i start i * layer_stride
  // values after those of layer0
  const int tok = blockIdx.x * kAppendWaves + wv, head = blockIdx.y, kv = blockIdx.z & 1, layer = layer0 + (blockIdx.z >> 1);
  if (tok >= n_tok) return;  // the waves do not wait for each other
  const int pos = pos0 + tok, page_index = pos / g.page_tokens, row = pos - page_index * g.page_tokens;
  const int page = page_row[page_index];
  const uint16_t* src = (kv ? Vn : Kn) + (size_t)(blockIdx.z >> 1) * layer_stride +
                        ((size_t)tok * g.n_kv_heads + head) * 128;
  const uint32_t v0 = src[lane], v1 = src[lane + 64];
  format_one(g, spec_pool, verif_pool, stage, v0, v1, lane, layer, page, kv, head, row);
}

// Reference read-back of cached vectors to dense bf16 (full == 0: zero-padded draft view).
__global__ __launch_bounds__(128) void kv_read_kernel(KvGeom g, const uint32_t* spec_pool, const uint32_t* verif_pool,
                                                      const int32_t* __restrict__ page_row, int layer, int pos0,
                                                      int full, uint16_t* Ko, uint16_t* Vo) {
  const int col = threadIdx.x;
  const int tok = blockIdx.x, head = blockIdx.y, kv = blockIdx.z;
  const int pos = pos0 + tok;
  int page = page_row[pos / g.page_tokens];
  if (page < 0 || page >= g.n_pages) {  // a page table entry outside the pool reads as zeros
    (kv ? Vo : Ko)[((size_t)tok * g.n_kv_heads + head) * 128 + col] = 0;
    return;
  }
  const uint16_t v = cached_value(g, spec_pool, verif_pool, layer, page, kv, head, pos % g.page_tokens, col, full);
  uint16_t* dst = (kv ? Vo : Ko) + ((size_t)tok * g.n_kv_heads + head) * 128;
  dst[col] = v;
}

int launch_kv_append(cas_ctx* ctx, cas_kv* kv, int layer, int seq, const uint16_t* K, const uint16_t* V, int n_tok,
                     int pos0) {
  return launch_kv_append_layers(ctx, kv, layer, 1, 0, seq, K, V, n_tok, pos0);
}

int launch_kv_append_layers(cas_ctx* ctx, cas_kv* kv, int layer0, int n_layers, size_t layer_stride, int seq,
                            const uint16_t* K, const uint16_t* V, int n_tok, int pos0) {
  if (n_tok <= 0 || n_layers <= 0) return CAS_OK;
  const KvGeom& g = kv->geom;
  // Up to twelve vectors per CU (ten over shared exponents) a wave takes each, above four.  us, one wave a vector / a wave
  // for four, 600 per mille kept, t = 4: 1 token of 8 heads 2.65 / 3.63, 64 of 8 (1024 vectors) 2.98 / 3.92, 2048 vectors 3.33 /
  // 3.99, 3072 4.02 / 4.02, 4000 4.61 / 4.06, 8192 6.83 / 5.55; over shared exponents 2.94 / 3.79, 3.30 / 4.00, 3.72 / 4.11, 3072
  // 4.33 / 4.14, 4000 4.99 / 4.17.  A commit of 5 positions of 8 layers, event to event, 6.1 / 7.1, of 80 layers (6400) 11.1 / 9.0.
  if ((int64_t)n_tok * g.n_kv_heads * 2 * n_layers <= (int64_t)(g.mx ? 10 : 12) * ctx->num_cu) {
    const dim3 grid((n_tok + kAppendWaves - 1) / kAppendWaves, g.n_kv_heads, 2 * n_layers);
    hipLaunchKernelGGL(kv_append_few_kernel, grid, dim3(64 * kAppendWaves), 0, ctx->stream, g, (uint32_t*)kv->d_spec,
                       (uint32_t*)kv->d_verif, kv->d_page_table + (size_t)seq * g.max_pages_per_seq, layer0, pos0, n_tok,
                       K, V, layer_stride);
    CAS_HIP(ctx, hipGetLastError());
    return CAS_OK;
  }
  const int groups = (pos0 + n_tok - 1) / kAppendRows - pos0 / kAppendRows + 1, fours = (pos0 + n_tok - 1) / 4 - pos0 / 4 + 1;
  // Of sixteen from 48 vectors per CU on (80 over shared exponents), from 36 where the first row is the first of sixteen (others are written
  // row by row).  us, four / sixteen, 8 heads, from such a row and from others: 512 tokens 5.4 / 5.6 and 6.1 / 6.6, 576 6.2 / 5.6 and 6.2 / 6.6, 736
  // 6.3 / 5.8 and 6.3 / 6.7, 768 6.3 / 5.8 and 7.1 / 6.7, 1021 7.6 / 7.4 and 8.3 / 8.1, 4096 18.6 / 11.8 and 19.2 / 13.2; over shared exponents 1152 9.1 / 9.0
  // and 9.0 / 9.6, 1300 10.1 / 9.5 and 10.1 / 9.7, 4096 21.5 / 15.2 and 22.4 / 17.2.
  // And only where its waves are filled well enough: a commit is a few rows of many layers.  A wave of sixteen takes as long as some 1.7 of four (2 over
  // shared exponents), and a single group is one wave of its workgroup.  126 layers of 8 heads, waves of four / groups of sixteen that the
  // tokens touch: 1 / 1 5.8 / 8.3, 2 / 1 7.5 / 8.7, 2 / 2 9.1 / 11.2, 3 / 2 12.2 / 11.2, 5 / 2 18.0 / 12.0, whole groups 11.2 / 7.9; 48 layers of 32 heads
  // 8.0 / 13.1, 11.0 / 13.6, 12.0 / 17.5, 16.9 / 17.6, 24.9 / 18.6, 15.1 / 11.8, over shared exponents 8.6 / 16.8, 12.3 / 16.9, 13.2 / 23.6,
  // 19.9 / 23.7, 29.6 / 24.7, 17.3 / 15.8; three fours in one group 9.4 / 8.9, 13.1 / 14.0 and 14.9 / 17.3
  const bool filled = groups > 1 ? 2 * fours >= 5 * groups : n_tok == kAppendRows;
  const bool many = filled && (int64_t)n_tok * g.n_kv_heads * 2 * n_layers >= (int64_t)(g.mx ? 80 : pos0 % kAppendRows ? 48 : 36) * ctx->num_cu;
  const dim3 grid(many ? (groups + kAppendWaves - 1) / kAppendWaves : groups, g.n_kv_heads, 2 * n_layers);
#define CAS_LAUNCH(TV)                                                                                              \
  case TV:                                                                                                          \
    hipLaunchKernelGGL(many ? (g.mx ? (kv_append_rows_kernel<TV, true>) : (kv_append_rows_kernel<TV, false>))       \
                            : (g.mx ? (kv_append_kernel<TV, true>) : (kv_append_kernel<TV, false>)),                \
                       grid, dim3(64 * kAppendWaves), 0, ctx->stream, g, (uint32_t*)kv->d_spec, (uint32_t*)kv->d_verif, \
                       kv->d_page_table + (size_t)seq * g.max_pages_per_seq, layer0, pos0, n_tok, K, V, layer_stride); \
    break;
  switch (g.t) {
    CAS_LAUNCH(0) CAS_LAUNCH(1) CAS_LAUNCH(2) CAS_LAUNCH(3) CAS_LAUNCH(4) CAS_LAUNCH(5) CAS_LAUNCH(6) CAS_LAUNCH(7)
    default: return CAS_EINVAL;
  }
#undef CAS_LAUNCH
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

int launch_kv_read(cas_ctx* ctx, cas_kv* kv, int layer, int seq, int pos0, int n_tok, int full, uint16_t* K,
                   uint16_t* V) {
  if (n_tok <= 0) return CAS_OK;
  const KvGeom& g = kv->geom;
  dim3 grid(n_tok, g.n_kv_heads, 2);
  hipLaunchKernelGGL(kv_read_kernel, grid, dim3(128), 0, ctx->stream, g, (const uint32_t*)kv->d_spec,
                     (const uint32_t*)kv->d_verif, kv->d_page_table + (size_t)seq * g.max_pages_per_seq, layer, pos0,
                     full, K, V);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

}  // namespace cas
