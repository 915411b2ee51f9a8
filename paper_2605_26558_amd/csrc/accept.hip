// Verification of drafted tokens against the target's probabilities from given random numbers (Sec. 2.2, Eq. 1), and the token
// that follows them, for a batch of sequences, on the GPU.
//
// With p_i and q_i the softmax of the target's and the draft model's logits at temperature T after i drafts, draft x_i is kept
// while r_i <= p_i(x_i) / q_i(x_i); behind the first that is not, the token is drawn from max(0, p_i - q_i), behind the last
// from p_k, which leaves tokens distributed as the target's own.  A draw takes the lowest token whose sum of weights up to and
// with itself exceeds u times the sum of all.
//
// 64 bits throughout: tokens of a vocabulary of 10^5 are a 10^-5 th apart in that sum, and with weights and sums of 32 bits one
// draw in some thousands falls on a neighbour of the right one.
//   launch 1, a workgroup per chunk of a row: the chunk's maximum and its sum of exponentials under it
//   launch 2, a workgroup per chunk of a sequence: joins the chunks of the sequence's rows, judges the drafts, and where one is
//             not kept forms the chunk's sum of max(0, p - q); the last workgroup of a sequence to arrive looks up the chunk, then
//             the token.  Where all are kept the sums of launch 1 do and one workgroup is left.
#include <algorithm>
#include "cas_device.hpp"
#include "cas_internal.hpp"

namespace cas {

constexpr int kAcceptThreads = 256;
constexpr int kAcceptEach = 16;                          // values of a thread
constexpr int kAcceptChunk = kAcceptThreads * kAcceptEach;
constexpr int kAcceptSeqs = 256;                         // sequences of a call
constexpr int kAcceptDrafts = 64;                        // drafts of a sequence: a lane each
constexpr int kAcceptVocab = 1 << 22;

struct AcceptPart {  // of a chunk of a row
  double sum;        // of exp((z - max) / T); greedy: 1 if there is a token
  float max;
  int first;         // greedy: the first token of the largest
};

struct AcceptArgs {
  const float* target;
  const float* draft;  // NULL: drafts are certain
  int64_t ldt, ldd;
  const int32_t* tokens;
  const float* temp;   // NULL: 1
  const double* r;
  int32_t* n_accepted;
  int32_t* out;
  int64_t ld_out;
  float* p;
  float* q;
  AcceptPart* part;    // [rows of the target, then of the draft][chunk]
  double* rest;        // [sequence][chunk]
  uint32_t* arrived;   // [sequence]
  int vocab, chunks, rows;  // rows: of the target
  int before[kAcceptSeqs + 1];  // drafts of the sequences before
};

// e^x for x <= 0 (0 for NaN): x = n ln 2 + r, |r| <= ln 2 / 2, and the Taylor series of e^r up to r^13 / 13!, whose next term is below
// 5e-18.  ln 2 in two parts, the first (744261118 / 2^30) of 30 bits, so that n times it is exact.
__device__ __forceinline__ double exp64(double x) {
  x = fmax(x, -1000.0);  // 2^-1443 is 0
  const double n = rint(x * 1.4426950408889634);
  const double r = fma(n, 4.2009150726810846e-11, fma(n, -0.69314718060195446, x));
  double y = 1.0 / 6227020800.0;
  y = fma(y, r, 1.0 / 479001600.0);
  y = fma(y, r, 1.0 / 39916800.0);
  y = fma(y, r, 1.0 / 3628800.0);
  y = fma(y, r, 1.0 / 362880.0);
  y = fma(y, r, 1.0 / 40320.0);
  y = fma(y, r, 1.0 / 5040.0);
  y = fma(y, r, 1.0 / 720.0);
  y = fma(y, r, 1.0 / 120.0);
  y = fma(y, r, 1.0 / 24.0);
  y = fma(y, r, 1.0 / 6.0);
  y = fma(y, r, 0.5);
  y = fma(y, r, 1.0);
  y = fma(y, r, 1.0);
  return ldexp(y, (int)n);
}

// Over the wave, in a fixed order: the sum in every lane, the sum of the lanes up to and with each
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ double wave_upto64(double v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double before = __shfl_up(v, d);
    if (lane >= d) v += before;
  }
  return v;
}
__device__ __forceinline__ int wave_min_int(int v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = min(v, __shfl_xor(v, d));
  return v;
}

// Temperature of a sequence: 1 / T, or 0 for a greedy one (T of 0, below it, or no number)
struct Heat {
  double inv;
  bool greedy;
  __device__ __forceinline__ Heat(const AcceptArgs& a, int s) {
    const float t = a.temp ? a.temp[s] : 1.f;
    greedy = !(t > 0.f);
    inv = greedy ? 0.0 : 1.0 / (double)t;
  }
};

// exp((z - max) / T); the largest weigh 1 whatever they are, infinity included
__device__ __forceinline__ double weight(float z, float max, double inv) {
  const double e = exp64(((double)z - (double)max) * inv);
  return z == max ? 1.0 : z == -INFINITY ? 0.0 : e;
}

// What a row weighs: exp((z - max) / T) * scale, or all of it on one token
struct RowStat {
  double scale;  // 1 / sum; 0 for a row without a token
  float max;
  int first;
};
__device__ __forceinline__ double probability(const RowStat& row, const Heat& heat, float z, int token) {
  if (heat.greedy) return token == row.first ? row.scale : 0.0;
  return row.max == -INFINITY ? 0.0 : weight(z, row.max, heat.inv) * row.scale;
}

// Values of a row: 16 bytes at byte offset `at` of its chunk.  What lies behind the row is held back by the descriptor; NaN
// counts as -infinity.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t chunk_of(const float* row, int chunk, int vocab) {
  const int from = chunk * kAcceptChunk;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(row + from), 0, min(vocab - from, kAcceptChunk) * 4, kRawBufferFlags);
}
__device__ __forceinline__ void four_values(__amdgpu_buffer_rsrc_t rs, int at, int left, float (&z)[4]) {
  const auto v = __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = __uint_as_float(v[i]);
    z[i] = at / 4 + i < left && x == x ? x : -INFINITY;
  }
}

__global__ __launch_bounds__(kAcceptThreads) void accept_rows_kernel(AcceptArgs a) {
  __shared__ float top[kAcceptThreads / 64];
  __shared__ double sums[kAcceptThreads / 64];
  __shared__ int firsts[kAcceptThreads / 64];
  const int chunk = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, wv = tid >> 6;
  const int d0 = a.before[s], k = a.before[s + 1] - d0;
  int col = blockIdx.z;
  if (chunk == 0 && col == 0 && tid == 0) a.arrived[s] = 0;
  const bool of_target = col <= k;
  if (!of_target) {
    col -= k + 1;
    if (!a.draft || col >= k) return;
  }
  const float* row = of_target ? a.target + (d0 + s + col) * a.ldt : a.draft + (d0 + col) * a.ldd;
  const Heat heat(a, s);
  const __amdgpu_buffer_rsrc_t rs = chunk_of(row, chunk, a.vocab);
  const int left = a.vocab - chunk * kAcceptChunk;
  float z[kAcceptEach / 4][4];
#pragma unroll
  for (int j = 0; j < kAcceptEach / 4; ++j) four_values(rs, 16 * (tid + kAcceptThreads * j), left, z[j]);
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < kAcceptEach; ++j) m = fmaxf(m, z[j >> 2][j & 3]);
  m = wave_max(m);
  if ((tid & 63) == 0) top[wv] = m;
  __syncthreads();
  m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  double sum = 0.0;
  int first = 0x7FFFFFFF;
  if (m > -INFINITY) {
    if (heat.greedy) {
#pragma unroll
      for (int j = 0; j < kAcceptEach; ++j)
        if (z[j >> 2][j & 3] == m) first = min(first, chunk * kAcceptChunk + 4 * (tid + kAcceptThreads * (j >> 2)) + (j & 3));
      first = wave_min_int(first);
    } else {
#pragma unroll
      for (int j = 0; j < kAcceptEach; ++j) sum += weight(z[j >> 2][j & 3], m, heat.inv);
      sum = wave_sum64(sum);
    }
  }
  if ((tid & 63) == 0) {
    sums[wv] = sum;
    firsts[wv] = first;
  }
  __syncthreads();
  if (tid == 0) {
    AcceptPart part;
    part.max = m;
    part.first = min(min(firsts[0], firsts[1]), min(firsts[2], firsts[3]));
    part.sum = heat.greedy ? (m > -INFINITY ? 1.0 : 0.0) : (sums[0] + sums[1]) + (sums[2] + sums[3]);
    a.part[(size_t)(of_target ? d0 + s + col : a.rows + d0 + col) * a.chunks + chunk] = part;
  }
}

// Joins the chunks of a row: a wave, in a fixed order
__device__ __forceinline__ RowStat join_chunks(const AcceptArgs& a, const Heat& heat, size_t row, int lane) {
  const AcceptPart* part = a.part + row * a.chunks;
  float m = -INFINITY;
  for (int c = lane; c < a.chunks; c += 64) m = fmaxf(m, part[c].max);
  m = wave_max(m);
  double sum = 0.0;
  int first = 0x7FFFFFFF;
  if (m > -INFINITY) {
    for (int c = lane; c < a.chunks; c += 64) {
      const AcceptPart p = part[c];
      if (heat.greedy) {
        if (p.max == m) first = min(first, p.first);
      } else if (p.max > -INFINITY) {
        sum += p.sum * weight(p.max, m, heat.inv);
      }
    }
    first = wave_min_int(first);
    sum = wave_sum64(sum);
  }
  RowStat st;
  st.max = m;
  st.first = first;
  st.scale = m == -INFINITY ? 0.0 : heat.greedy ? 1.0 : 1.0 / sum;
  return st;
}

// What the token behind the drafts is drawn by: max(0, p - q) with q the draft's row or all of it on `x`, or p alone
struct Decision {
  RowStat t, d;
  const float* target;
  const float* draft;  // NULL: q is all on x
  int x;               // -1: p alone
};
__device__ __forceinline__ double rest_weight(const Decision& w, const Heat& heat, float zt, float zd, int token) {
  const double p = probability(w.t, heat, zt, token);
  if (w.x < 0) return p;
  const double q = w.draft ? probability(w.d, heat, zd, token) : token == w.x ? 1.0 : 0.0;
  return fmax(p - q, 0.0);
}

__global__ __launch_bounds__(kAcceptThreads) void accept_tokens_kernel(AcceptArgs a) {
  __shared__ RowStat stats[2 * kAcceptDrafts + 1];
  __shared__ double sums[kAcceptThreads / 64];
  __shared__ int found[kAcceptThreads / 64], lasts[kAcceptThreads / 64];
  __shared__ int s_kept, s_last, s_chunk, s_x;
  __shared__ double s_left;
  const int s = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int d0 = a.before[s], k = a.before[s + 1] - d0;
  const Heat heat(a, s);

  // ---- the rows' maxima and sums, the target's first
  const int n_rows = a.draft ? 2 * k + 1 : k + 1;
  for (int i = wv; i < n_rows; i += kAcceptThreads / 64) {
    const RowStat st = join_chunks(a, heat, i <= k ? d0 + s + i : a.rows + d0 + i - k - 1, lane);
    if (lane == 0) stats[i] = st;
  }
  __syncthreads();

  // ---- the drafts that are kept: a lane each
  if (wv == 0) {
    bool good = false;
    if (lane < k) {
      const int x = a.tokens[d0 + lane];
      double p = 0.0, q = 0.0;
      if (x >= 0 && x < a.vocab) {
        float zt = a.target[(d0 + s + lane) * a.ldt + x];
        zt = zt == zt ? zt : -INFINITY;
        p = probability(stats[lane], heat, zt, x);
        q = 1.0;
        if (a.draft) {
          float zd = a.draft[(d0 + lane) * a.ldd + x];
          zd = zd == zd ? zd : -INFINITY;
          q = probability(stats[k + 1 + lane], heat, zd, x);
        }
      }
      good = p > 0.0 && a.r[d0 + s + lane] <= p / q;
      if (blockIdx.x == 0) {
        if (a.p) a.p[d0 + lane] = (float)p;
        if (a.q) a.q[d0 + lane] = (float)q;
      }
    }
    const uint64_t bad = ~__builtin_amdgcn_ballot_w64(good);  // a lane without a draft is not kept either
    if (lane == 0) s_kept = bad ? __ffsll((unsigned long long)bad) - 1 : kAcceptDrafts;
  }
  __syncthreads();
  const int kept = __builtin_amdgcn_readfirstlane(s_kept);
  Decision w;
  w.t = stats[kept];
  w.target = a.target + (d0 + s + kept) * a.ldt;
  w.draft = nullptr;
  w.x = -1;
  if (kept < k) {
    w.x = a.tokens[d0 + kept];
    if (a.draft) {
      w.d = stats[k + 1 + kept];
      w.draft = a.draft + (d0 + kept) * a.ldd;
    }
    if (w.x < 0) w.x = 0x7FFFFFFF;  // no token of the vocabulary
  }

  // ---- sums of the chunks
  auto chunk_values = [&](int chunk, int at, float (&zt)[4], float (&zd)[4]) {
    const int left = a.vocab - chunk * kAcceptChunk;
    four_values(chunk_of(w.target, chunk, a.vocab), at, left, zt);
    if (w.draft) four_values(chunk_of(w.draft, chunk, a.vocab), at, left, zd);
  };
  if (kept == k) {
    if (blockIdx.x != 0) return;
  } else {
    const int chunk = blockIdx.x;
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < kAcceptEach / 4; ++j) {
      const int at = 16 * (tid + kAcceptThreads * j);
      float zt[4], zd[4] = {0.f, 0.f, 0.f, 0.f};
      chunk_values(chunk, at, zt, zd);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += rest_weight(w, heat, zt[i], zd[i], chunk * kAcceptChunk + at / 4 + i);
    }
    sum = wave_sum64(sum);
    if (lane == 0) sums[wv] = sum;
    __syncthreads();
    if (tid == 0) {
      __hip_atomic_store(&a.rest[(size_t)s * a.chunks + chunk], (sums[0] + sums[1]) + (sums[2] + sums[3]), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
      __threadfence();
      s_last = __hip_atomic_fetch_add(&a.arrived[s], 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.chunks - 1;
    }
    __syncthreads();
    if (!s_last) return;
  }

  // ---- the chunk of the token: the first whose sum up to and with itself exceeds the number's share
  const double u = a.r[d0 + s + k];
  if (wv == 0) {
    const AcceptPart* part = a.part + (size_t)(d0 + s + kept) * a.chunks;
    auto sum_of = [&](int c) -> double {
      if (w.x >= 0) return __hip_atomic_load(&a.rest[(size_t)s * a.chunks + c], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (w.t.max == -INFINITY) return 0.0;
      if (heat.greedy) return part[c].max == w.t.max && part[c].first == w.t.first ? 1.0 : 0.0;
      return part[c].max == -INFINITY ? 0.0 : part[c].sum * weight(part[c].max, w.t.max, heat.inv) * w.t.scale;
    };
    int chunk = -1;
    double left = 0.0;
    for (int turn = 0; turn < 2; ++turn) {
      double total = 0.0;
      for (int c = lane; c < a.chunks; c += 64) total += sum_of(c);
      total = wave_sum64(total);
      if (total > 0.0) {
        // 64 chunks at a time, each lane's sum up to and with its own
        double before = 0.0;
        int last = -1;
        const double t = u * total;
        for (int c0 = 0; c0 < a.chunks && chunk < 0; c0 += 64) {
          const double own = c0 + lane < a.chunks ? sum_of(c0 + lane) : 0.0;
          const double upto = wave_upto64(own, lane);
          const uint64_t some = __builtin_amdgcn_ballot_w64(own > 0.0);
          const uint64_t over = __builtin_amdgcn_ballot_w64(own > 0.0 && before + upto > t);
          if (some) last = c0 + 63 - __clzll((long long)some);
          if (over) {
            const int l = __ffsll((unsigned long long)over) - 1;
            chunk = c0 + l;
            left = t - (before + (__shfl(upto, l) - __shfl(own, l)));
          }
          before += __shfl(upto, 63);
        }
        if (chunk < 0) {  // a number of 1 or above, or a sum that rounding put below it: the last token
          chunk = last;
          left = INFINITY;
        }
        break;
      }
      if (w.x < 0) break;
      w.x = -1;  // nothing left of p - q, by rounding: p
    }
    if (lane == 0) {
      s_chunk = chunk;
      s_left = left;
      s_x = w.x;
    }
  }
  __syncthreads();
  const int chunk = __builtin_amdgcn_readfirstlane(s_chunk);
  const double left = s_left;
  w.x = s_x;

  // ---- the token: a thread's values follow one another here
  int token = -1;
  if (chunk >= 0) {
    double v[kAcceptEach], own = 0.0;
    const int base = chunk * kAcceptChunk + tid * kAcceptEach;
#pragma unroll
    for (int j = 0; j < kAcceptEach / 4; ++j) {
      float zt[4], zd[4] = {0.f, 0.f, 0.f, 0.f};
      chunk_values(chunk, 4 * (tid * kAcceptEach + 4 * j), zt, zd);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[4 * j + i] = rest_weight(w, heat, zt[i], zd[i], base + 4 * j + i);
        own += v[4 * j + i];
      }
    }
    const double upto = wave_upto64(own, lane);
    if (lane == 63) sums[wv] = upto;
    __syncthreads();
    double c = upto - own;
    for (int i = 0; i < wv; ++i) c += sums[i];
    int over = 0x7FFFFFFF, last = -1;
#pragma unroll
    for (int j = 0; j < kAcceptEach; ++j) {
      c += v[j];
      if (v[j] > 0.0) {
        last = base + j;
        if (c > left) over = min(over, base + j);
      }
    }
    over = wave_min_int(over);
    last = -wave_min_int(-last);
    if (lane == 0) {
      found[wv] = over;
      lasts[wv] = last;
    }
    __syncthreads();
    over = min(min(found[0], found[1]), min(found[2], found[3]));
    last = max(max(lasts[0], lasts[1]), max(lasts[2], lasts[3]));
    token = over != 0x7FFFFFFF ? over : last;
  }
  for (int64_t i = tid; i < a.ld_out; i += kAcceptThreads)
    a.out[s * a.ld_out + i] = i < kept ? a.tokens[d0 + i] : i == kept ? token : -1;
  if (tid == 0) a.n_accepted[s] = kept;
}

// Where the parts of the workspace lie; 0 bytes for arguments that are refused
struct AcceptPlan {
  int64_t drafts = 0, rest = 0, arrived = 0, bytes = 0;
  int most = 0, chunks = 0;
};
static int plan_accept(int n_seqs, const int32_t* h_k, int vocab, AcceptPlan* out) {
  if (n_seqs < 0 || vocab < 1 || (n_seqs > 0 && !h_k)) return CAS_EINVAL;
  AcceptPlan p;
  for (int i = 0; i < n_seqs; ++i) {
    if (h_k[i] < 0) return CAS_EINVAL;
    p.most = std::max(p.most, (int)h_k[i]);
    p.drafts += h_k[i];
  }
  if (n_seqs > kAcceptSeqs || p.most > kAcceptDrafts || vocab > kAcceptVocab) return CAS_ENOTSUP;
  p.chunks = (vocab + kAcceptChunk - 1) / kAcceptChunk;
  auto up256 = [](int64_t b) { return (b + 255) / 256 * 256; };
  p.rest = up256((2 * p.drafts + n_seqs) * p.chunks * (int64_t)sizeof(AcceptPart));
  p.arrived = p.rest + up256((int64_t)n_seqs * p.chunks * 8);
  p.bytes = p.arrived + up256((int64_t)n_seqs * 4);
  *out = p;
  return CAS_OK;
}

}  // namespace cas

extern "C" {

int cas_accept_tokens(cas_ctx* ctx, int n_seqs, const int32_t* h_k, int vocab, const float* d_target, int64_t ldt,
                      const float* d_draft, int64_t ldd, const int32_t* d_tokens, const float* d_temp, const double* d_r,
                      int32_t* d_n_accepted, int32_t* d_out, int64_t ld_out, float* d_p, float* d_q) {
  cas::AcceptPlan plan;
  const int rc = ctx ? cas::plan_accept(n_seqs, h_k, vocab, &plan) : CAS_EINVAL;
  if (rc != CAS_OK) return rc;
  if (n_seqs == 0) return CAS_OK;
  if (!d_target || ldt < vocab || !d_r || !d_n_accepted || !d_out || ld_out <= plan.most) return CAS_EINVAL;
  if (plan.drafts > 0 && (!d_tokens || (d_draft && ldd < vocab))) return CAS_EINVAL;
  for (const void* d : {(const void*)d_target, (const void*)d_draft, (const void*)d_tokens, (const void*)d_temp, (const void*)d_n_accepted,
                        (const void*)d_out, (const void*)d_p, (const void*)d_q})
    if ((uintptr_t)d % 4) return CAS_EINVAL;
  if ((uintptr_t)d_r % 8) return CAS_EINVAL;
  if (!cas::on_device(ctx)) return CAS_EINVAL;
  if (!ctx->d_ws) return CAS_ENOMEM;
  if (!cas::aligned256(ctx->d_ws)) return CAS_EINVAL;
  if ((size_t)plan.bytes > ctx->ws_bytes) return CAS_ENOMEM;
  cas::AcceptArgs a{};
  a.target = d_target; a.draft = plan.drafts > 0 ? d_draft : nullptr; a.ldt = ldt; a.ldd = ldd;
  a.tokens = d_tokens; a.temp = d_temp; a.r = d_r;
  a.n_accepted = d_n_accepted; a.out = d_out; a.ld_out = ld_out; a.p = d_p; a.q = d_q;
  char* ws = (char*)ctx->d_ws;
  a.part = (cas::AcceptPart*)ws;
  a.rest = (double*)(ws + plan.rest);
  a.arrived = (uint32_t*)(ws + plan.arrived);
  a.vocab = vocab; a.chunks = plan.chunks; a.rows = (int)plan.drafts + n_seqs;
  for (int i = 0; i < n_seqs; ++i) a.before[i + 1] = a.before[i] + h_k[i];
  const int cols = plan.most + 1 + (a.draft ? plan.most : 0);
  hipLaunchKernelGGL(cas::accept_rows_kernel, dim3(plan.chunks, n_seqs, cols), dim3(cas::kAcceptThreads), 0, ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  hipLaunchKernelGGL(cas::accept_tokens_kernel, dim3(plan.most > 0 ? plan.chunks : 1, n_seqs), dim3(cas::kAcceptThreads), 0, ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

size_t cas_accept_tokens_bytes(int n_seqs, const int32_t* h_k, int vocab) {
  cas::AcceptPlan plan;
  return cas::plan_accept(n_seqs, h_k, vocab, &plan) == CAS_OK ? (size_t)plan.bytes : 0;
}

}  // extern "C"
