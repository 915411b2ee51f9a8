// Attention for the query rows of several sequences over a prefix that they share, and attention that adds up what every
// cached position received.
//
// cas_attention decodes a page of the cache for the query rows of one sequence.  Where a batch of sequences begins with the
// same pages, the decode, which is most of the time (some nine vector operations per value), is the same for all of them:
// here a workgroup decodes a page once for 16, 32 or 64 query rows whichever sequence they belong to, and goes through a run
// of pages with running maxima and sums, so that a row has one partial result per run and not per page.  What follows the
// prefix goes through the same kernel, sequence by sequence, in the same launch.
//   grid: (runs of the prefix x tiles of all rows, then per sequence runs x tiles of its rows) x kv heads
// A second kernel joins the partial results of a row in the order of the runs, prefix first.
//
// Attention weights: the partial kernel also writes the exponents of its scores, and once the maximum and the sum of a row
// are known, a third kernel forms the weights of all rows of a kv head and adds them.  Exponents are 4 bytes per row and
// position, a vector of K 131 in the draft form: cheaper than decoding K again.
#include <algorithm>
#include "attention_rows_kernel.inl"

namespace cas {

extern template int launch_rows_partial<true, false>(cas_ctx*, const RowsArgs&, int);
extern template int launch_rows_partial<false, false>(cas_ctx*, const RowsArgs&, int);
extern template int launch_rows_partial<true, true>(cas_ctx*, const RowsArgs&, int);
extern template int launch_rows_partial<false, true>(cas_ctx*, const RowsArgs&, int);

// One wave per (query row, kv head); lane: two channels.  Splits in the order prefix, then the sequence's own; lane i keeps
// the pairs of splits i, i + 64, ... for maximum and sum.
__global__ __launch_bounds__(256) void rows_merge_kernel(RowsArgs a) {
  const int rr = 4 * (int)blockIdx.x + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), head = blockIdx.y, lane = threadIdx.x & 63;
  if (rr >= a.rows) return;
  int si = 0;
  while (si + 1 < a.n_seqs && rr >= a.s[si + 1].row0) ++si;
  const RowsSeq& me = a.s[si];
  const int r = rr - me.row0, rows = me.ncols * a.grp;
  const float2* mlp = a.ml_prefix + ((size_t)head * a.rows + rr) * a.prefix_splits;
  const float2* mlt = a.ml_tail + me.part0 + ((size_t)head * rows + r) * me.splits;
  const int n = a.prefix_splits + me.splits;
  auto pair = [&](int i) { return i < a.prefix_splits ? mlp[i] : mlt[i - a.prefix_splits]; };
  float M = kLowest;
  for (int i = lane; i < n; i += 64) M = fmaxf(M, pair(i).x);
  M = wave_max(M);
  float den = 0.f;
  float2 num = make_float2(0.f, 0.f);
  const float2* op = reinterpret_cast<const float2*>(a.out_prefix) + ((size_t)head * a.rows + rr) * 64 + lane;
  const float2* ot = reinterpret_cast<const float2*>(a.out_tail) + (me.part0 + (size_t)head * rows + r) * 64 + lane;
  const size_t sp = (size_t)a.g.n_kv_heads * a.rows * 64, st = (size_t)a.g.n_kv_heads * rows * 64;
  for (int i0 = 0; i0 < n; i0 += 64) {
    float w = 0.f;
    if (i0 + lane < n) {
      const float2 ml = pair(i0 + lane);
      w = __builtin_amdgcn_exp2f(ml.x - M);
      den += w * ml.y;
    }
    for (int i = 0; i < min(64, n - i0); ++i) {
      const int s = i0 + i;
      const float2 o = s < a.prefix_splits ? op[s * sp] : ot[(s - a.prefix_splits) * st];
      const float ws = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), i));
      num.x += ws * o.x;
      num.y += ws * o.y;
    }
  }
  den = wave_sum(den);
  const int c = r / a.grp, gi = r - c * a.grp;
  uint32_t* out = reinterpret_cast<uint32_t*>(me.O + ((size_t)c * a.n_q_heads + head * a.grp + gi) * 128) + lane;
  *out = (uint32_t)f32_to_bf16(num.x / den) | ((uint32_t)f32_to_bf16(num.y / den) << 16);
}

// Weights of 256 positions of a kv head: every row's maximum and sum first (a wave per row), then a thread per position.
__global__ __launch_bounds__(256) void rows_weights_kernel(RowsArgs a, const float* in, float* out, int64_t ld) {
  extern __shared__ float2 row_ml[];
  const RowsSeq& me = a.s[0];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, head = blockIdx.y, rows = a.rows, n = me.splits;
  for (int r = wv; r < rows; r += 4) {
    const float2* ml = a.ml_tail + ((size_t)head * rows + r) * n;
    float M = kLowest, L = 0.f;
    for (int i = lane; i < n; i += 64) M = fmaxf(M, ml[i].x);
    M = wave_max(M);
    for (int i = lane; i < n; i += 64) L += __builtin_amdgcn_exp2f(ml[i].x - M) * ml[i].y;
    L = wave_sum(L);
    if (lane == 0) row_ml[r] = make_float2(M, 1.f / L);
  }
  __syncthreads();
  const int pos = (int)blockIdx.x * 256 + tid;
  if (pos >= me.len + me.n_new) return;
  const float* x = a.score + (size_t)head * rows * a.score_ld + pos;
  float w = 0.f;
  for (int r = 0; r < rows; ++r) w += __builtin_amdgcn_exp2f(x[(size_t)r * a.score_ld] - row_ml[r].x) * row_ml[r].y;
  const int64_t at = (int64_t)head * ld + pos;
  out[at] = (in && pos < me.len ? in[at] : 0.f) + w;
}

// ---- host ---------------------------------------------------------------------------------------
constexpr int kTailRun = 2;  // pages of a run behind the prefix: fixed, so that a sequence's values do not depend on its length

struct RowsPlan {
  RowsArgs a;
  int nt, items;
  size_t bytes;
};

static int64_t up256(int64_t b) { return (b + 255) / 256 * 256; }

// What a call will launch and need; the pointers of a.s[] are left to the caller.
static int plan_rows(const cas_kv* kv, int n_seqs, const int32_t* seqs, int prefix_len, const int32_t* ncols, int n_q_heads,
                     const int32_t* n_new, bool weights, int num_cu, RowsPlan* out) {
  if (!kv || n_seqs < 1 || n_seqs > kRowsSeqs || !seqs || !ncols || !n_new || prefix_len < 0) return CAS_EINVAL;
  const KvGeom& g = kv->geom;
  if (n_q_heads < g.n_kv_heads || n_q_heads % g.n_kv_heads != 0) return CAS_EINVAL;
  RowsPlan p{};
  RowsArgs& a = p.a;
  a.g = g;
  a.n_q_heads = n_q_heads;
  a.grp = n_q_heads / g.n_kv_heads;
  if (a.grp > 48) return CAS_EINVAL;
  a.grp_inv = (65536u + (uint32_t)a.grp - 1u) / (uint32_t)a.grp;
  a.scale2 = (float)(1.4426950408889634 * 0.08838834764831845);
  a.n_seqs = n_seqs;
  a.prefix_pages = prefix_len / 64;
  a.tail_run = kTailRun;
  int64_t rows = 0, parts = 0, items = 0;
  for (int i = 0; i < n_seqs; ++i) {
    RowsSeq& s = a.s[i];
    if (seqs[i] < 0 || seqs[i] >= kv->desc.max_seqs) return CAS_EINVAL;
    for (int k = 0; k < i; ++k)
      if (seqs[k] == seqs[i]) return CAS_EINVAL;
    if (ncols[i] < 1 || ncols[i] > 16 || n_new[i] < ncols[i] || n_new[i] > 64) return CAS_EINVAL;
    s.seq = seqs[i]; s.len = kv->h_len[seqs[i]]; s.ncols = ncols[i]; s.n_new = n_new[i];
    if (prefix_len > s.len) return CAS_EINVAL;
    const int64_t pages = ((int64_t)s.len + s.n_new + 63) / 64;
    if (pages > g.max_pages_per_seq) return CAS_ENOMEM;
    s.splits = (int)(pages - a.prefix_pages + kTailRun - 1) / kTailRun;
    s.row0 = (int)rows;
    rows += s.ncols * a.grp;
  }
  a.rows = (int)rows;
  p.nt = 1;
  if (a.prefix_pages > 0) {
    a.prefix_run = 2;
    a.prefix_splits = (a.prefix_pages + a.prefix_run - 1) / a.prefix_run;
    a.prefix_items = a.prefix_splits * ((a.rows + 16 * p.nt - 1) / (16 * p.nt));
  }
  for (int i = 0; i < n_seqs; ++i) {
    RowsSeq& s = a.s[i];
    const int r = s.ncols * a.grp;
    s.item0 = (int)items;
    s.part0 = (uint32_t)parts;
    items += (int64_t)s.splits * ((r + 16 * p.nt - 1) / (16 * p.nt));
    parts += (int64_t)s.splits * g.n_kv_heads * r;
  }
  const int64_t first = (int64_t)a.prefix_splits * g.n_kv_heads * a.rows;
  if (parts > 0xFFFFFFFFll || (items + a.prefix_items) * g.n_kv_heads > 0x7FFFFFFF) return CAS_ENOTSUP;
  p.items = (int)items + a.prefix_items;
  // workspace: outputs, pairs, and the exponents of the rows
  int64_t off = up256((first + parts) * 512);
  const int64_t off_ml = off;
  off += up256((first + parts) * 8);
  const int64_t off_score = off;
  if (weights) {
    a.score_ld = ((int64_t)a.s[0].len + a.s[0].n_new + 63) / 64 * 64;
    off += up256(a.score_ld * g.n_kv_heads * a.rows * 4);
  }
  p.bytes = (size_t)off;
  a.out_prefix = (float*)0;
  a.out_tail = (float*)(uintptr_t)(first * 512);
  a.ml_prefix = (float2*)(uintptr_t)off_ml;
  a.ml_tail = (float2*)(uintptr_t)(off_ml + first * 8);
  a.score = weights ? (float*)(uintptr_t)off_score : nullptr;
  *out = p;
  return CAS_OK;
}

static void place(RowsArgs& a, void* ws) {  // offsets into the workspace become addresses
  char* b = (char*)ws;
  auto at = [&](auto*& p) { p = (std::remove_reference_t<decltype(p)>)(b + (uintptr_t)p); };
  at(a.out_prefix); at(a.out_tail); at(a.ml_prefix); at(a.ml_tail);
  if (a.score) at(a.score);
}

static int launch_rows(cas_ctx* ctx, cas_kv* kv, RowsPlan& p, int layer, int full) {
  if (!ctx->d_ws || !aligned256(ctx->d_ws) || p.bytes > ctx->ws_bytes) return ctx->d_ws && !aligned256(ctx->d_ws) ? CAS_EINVAL : CAS_ENOMEM;
  RowsArgs& a = p.a;
  place(a, ctx->d_ws);
  a.spec_pool = (const uint32_t*)kv->d_spec;
  a.verif_pool = (const uint32_t*)kv->d_verif;
  a.table = kv->d_page_table;
  a.layer = layer;
  const int rc = a.g.mx ? (full ? launch_rows_partial<true, true>(ctx, a, p.items) : launch_rows_partial<false, true>(ctx, a, p.items))
                        : (full ? launch_rows_partial<true, false>(ctx, a, p.items) : launch_rows_partial<false, false>(ctx, a, p.items));
  if (rc != CAS_OK) return rc;
  hipLaunchKernelGGL(rows_merge_kernel, dim3((a.rows + 3) / 4, a.g.n_kv_heads), dim3(256), 0, ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

}  // namespace cas

extern "C" {

int cas_attention_shared(cas_ctx* ctx, cas_kv* kv, int layer, int n_seqs, const int32_t* h_seqs, int prefix_len, int full,
                         const uint16_t* const* h_d_Q, const int32_t* h_ncols, int n_q_heads,
                         const uint16_t* const* h_d_Knew, const uint16_t* const* h_d_Vnew, const int32_t* h_n_new,
                         uint16_t* const* h_d_O) {
  if (!ctx || !kv || layer < 0 || layer >= kv->desc.n_layers || !h_d_Q || !h_d_Knew || !h_d_Vnew || !h_d_O) return CAS_EINVAL;
  cas::RowsPlan p;
  const int rc = cas::plan_rows(kv, n_seqs, h_seqs, prefix_len, h_ncols, n_q_heads, h_n_new, false, ctx->num_cu, &p);
  if (rc != CAS_OK) return rc;
  for (int i = 0; i < n_seqs; ++i) {
    cas::RowsSeq& s = p.a.s[i];
    s.Q = h_d_Q[i]; s.Knew = h_d_Knew[i]; s.Vnew = h_d_Vnew[i]; s.O = h_d_O[i];
    if (!s.Q || !s.Knew || !s.Vnew || !s.O || !cas::aligned256(s.Q) || !cas::aligned256(s.Knew) || !cas::aligned256(s.Vnew) || !cas::aligned256(s.O))
      return CAS_EINVAL;
  }
  if (!cas::on_device(ctx)) return CAS_EINVAL;
  return cas::launch_rows(ctx, kv, p, layer, full);
}

size_t cas_attention_shared_bytes(const cas_kv* kv, int n_seqs, const int32_t* h_seqs, int prefix_len, const int32_t* h_ncols,
                                  int n_q_heads, const int32_t* h_n_new) {
  cas::RowsPlan p;
  return cas::plan_rows(kv, n_seqs, h_seqs, prefix_len, h_ncols, n_q_heads, h_n_new, false, 256, &p) == CAS_OK ? p.bytes : 0;
}

int cas_attention_weights(cas_ctx* ctx, cas_kv* kv, int layer, int seq, int full, const uint16_t* d_Q, int ncols, int n_q_heads,
                          const uint16_t* d_Knew, const uint16_t* d_Vnew, int n_new, uint16_t* d_O, const float* d_score_in,
                          float* d_score_out, int64_t ld) {
  if (!ctx || !kv || layer < 0 || layer >= kv->desc.n_layers || !d_Q || !d_Knew || !d_Vnew || !d_O || !d_score_out) return CAS_EINVAL;
  cas::RowsPlan p;
  int rc = cas::plan_rows(kv, 1, &seq, 0, &ncols, n_q_heads, &n_new, true, ctx->num_cu, &p);
  if (rc != CAS_OK) return rc;
  cas::RowsSeq& s = p.a.s[0];
  const int total = s.len + n_new;
  if (ld < total) return CAS_EINVAL;
  if (!cas::aligned256(d_Q) || !cas::aligned256(d_Knew) || !cas::aligned256(d_Vnew) || !cas::aligned256(d_O)) return CAS_EINVAL;
  if (!cas::on_device(ctx)) return CAS_EINVAL;
  s.Q = d_Q; s.Knew = d_Knew; s.Vnew = d_Vnew; s.O = d_O;
  rc = cas::launch_rows(ctx, kv, p, layer, full);
  if (rc != CAS_OK) return rc;
  hipLaunchKernelGGL(cas::rows_weights_kernel, dim3((total + 255) / 256, p.a.g.n_kv_heads), dim3(256), sizeof(float2) * p.a.rows,
                     ctx->stream, p.a, d_score_in, d_score_out, ld);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

size_t cas_attention_weights_bytes(const cas_kv* kv, int seq, int ncols, int n_q_heads, int n_new) {
  cas::RowsPlan p;
  return cas::plan_rows(kv, 1, &seq, 0, &ncols, n_q_heads, &n_new, true, 256, &p) == CAS_OK ? p.bytes : 0;
}

}  // extern "C"
