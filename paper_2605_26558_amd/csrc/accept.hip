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
//   launch 2, workgroups per sequence: each joins the chunks of the sequence's rows and settles which drafts are kept, and where one is not kept forms
//             sums of max(0, p - q) over its pieces of the vocabulary.  Left out where there are no drafts
//   launch 3, a workgroup per sequence: looks up the piece (or the chunk of launch 1, where all drafts are kept), then the token
//
// Measured (us; in brackets the bytes of the logits at the rate of a copy): 32 sequences of up to 7 drafts over 128256 tokens 53 (32.2): launch 1 34, at the
// rate of memory, its vector issue, 22 operations a value, in 91 % of the cycles; launch 2 13.5 (row joins, then two exponentials a value of one row pair); launch 3
// 5.  64 draws over 128256 17 (6.4): 10.5 and 6.6.  One sequence of 4 drafts over 32000 13.4 (0.2): three launches of dependent round trips.
#include <algorithm>
#include "cas_device.hpp"
#include "cas_internal.hpp"

namespace cas {

constexpr int kAcceptThreads = 256, kAcceptWaves = kAcceptThreads / 64;
constexpr int kAcceptChunk = 16 * kAcceptThreads;        // values of a workgroup of the first launch
constexpr int kAcceptPiece = 8 * kAcceptThreads;         // of the second
constexpr int kAcceptSeqs = 256;                         // sequences of a call
constexpr int kAcceptDrafts = 64;                        // drafts of a sequence: a lane each
constexpr int kAcceptVocab = 1 << 22;

struct AcceptPart {  // of a chunk of a row
  double sum;        // of exp((z - max) / T); greedy: 1 if there is a token
  float max;
  int first;         // greedy: the first token of the largest
};

// What a row weighs: exp((z - max) / T) * scale, or all of it on one token
struct RowStat {
  double scale;  // 1 / sum; 0 for a row without a token
  float max;
  int first;
};
struct AcceptOutcome {
  RowStat t, d;  // of the rows behind the kept drafts
  int kept, x;   // x: the draft behind them, -1 if all are kept
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
  double* rest;        // [sequence][piece]
  AcceptOutcome* outcome;  // [sequence]
  int vocab, chunks, pieces, rows;  // rows: of the target
  int each;                         // pieces of a workgroup of the second launch
  int before[kAcceptSeqs + 1];      // drafts of the sequences before
};

// 2^y for y <= 0; 0 for y below -1100 and for NaN.  y = n + f, |f| <= 1/2, n by the addition of 1.5 * 2^52; 2^f = 1 + f g(f), g the polynomial of
// degree 8 through (2^f - 1) / f at the nine Chebyshev points of the interval: within 4e-14 of the result.  Which of 10^5
// neighbours a number falls on does not need more (the sums' own roundings are 1e-14 apart by their order).  N numbers side by side, so that
// no operation waits for the one before.
template <int N>
__device__ __forceinline__ void exp2_64(double (&y)[N]) {
  constexpr double kPoly[] = {1.0203121090457445e-07, 1.325522487884224e-06, 1.5252686846147753e-05, 0.00015403455852453318, 0.0013333558179043322,
                              0.009618129159402558,   0.055504108664760424,  0.2402265069581299,     0.6931471805599453,     1.0};
  double m[N], e[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    asm("v_max_f64 %0, %1, %2" : "=v"(y[i]) : "v"(y[i]), "s"(-1100.0));  // one operation; the compiler's own makes quiet numbers first
    m[i] = y[i] + 6755399441055744.0;
    y[i] -= m[i] - 6755399441055744.0;
    e[i] = kPoly[0];
  }
#pragma unroll
  for (int c = 1; c < 10; ++c) {
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = fma(e[i], y[i], kPoly[c]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = __builtin_amdgcn_ldexp(e[i], (int)(uint32_t)__builtin_bit_cast(uint64_t, m[i]));
}

// Sums over the lanes in a fixed order, up to and with each: the steps of wave_incl_scan on the halves of a number
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ double dpp_add64(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROW_MASK, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROW_MASK, 0xf, false);
  return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double row16_upto64(double v) {  // lanes of a row of 16; the last has the sum
  v = dpp_add64<DPP_ROW_SHR1, 0xf>(v);
  v = dpp_add64<DPP_ROW_SHR2, 0xf>(v);
  v = dpp_add64<DPP_ROW_SHR4, 0xf>(v);
  return dpp_add64<DPP_ROW_SHR8, 0xf>(v);
}
__device__ __forceinline__ double wave_upto64(double v) {
  v = row16_upto64(v);
  v = dpp_add64<DPP_ROW_BCAST15, 0xa>(v);
  return dpp_add64<DPP_ROW_BCAST31, 0xc>(v);
}
__device__ __forceinline__ double lane_of(double v, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int wave_min_int(int v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = min(v, __shfl_xor(v, d));
  return v;
}

// Temperature of a sequence: log2(e) / T, or 0 for a greedy one (T of 0, below it, or no number)
struct Heat {
  double inv;
  bool greedy;
  __device__ __forceinline__ Heat(const AcceptArgs& a, int s) {
    const float t = a.temp ? a.temp[s] : 1.f;
    greedy = !(t > 0.f);
    inv = greedy ? 0.0 : 1.4426950408889634 / (double)t;
  }
};

// exp((z - max) / T).  -infinity and NaN give 0 by themselves, the largest 1, unless it is infinite.
template <int N>
__device__ __forceinline__ void weights(const float (&z)[N], float max, double inv, double (&w)[N]) {
  if (max == INFINITY) {  // the same for all values of a row
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = z[i] == max ? 1.0 : 0.0;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = ((double)z[i] - (double)max) * inv;
    exp2_64(w);
  }
}
__device__ __forceinline__ double weight(float z, float max, double inv) {
  const float one[1] = {z};
  double w[1];
  weights(one, max, inv, w);
  return w[0];
}

template <int N>
__device__ __forceinline__ void probabilities(const RowStat& row, const Heat& heat, const float (&z)[N], int token, double (&p)[N]) {
  if (heat.greedy) {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = token + i == row.first ? row.scale : 0.0;
  } else if (row.max == -INFINITY) {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = 0.0;
  } else {
    weights(z, row.max, heat.inv, p);
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] *= row.scale;
  }
}
__device__ __forceinline__ double probability(const RowStat& row, const Heat& heat, float z, int token) {
  const float one[1] = {z};
  double p[1];
  probabilities(row, heat, one, token, p);
  return p[0];
}

// Values of a row from `from` on, through a descriptor that ends with the row or after `most` values; those behind it are none
struct RowPart {
  __amdgpu_buffer_rsrc_t rs;
  int left;
  __device__ __forceinline__ RowPart(const float* row, int from, int most, int vocab) : left(min(vocab - from, most)) {
    rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(row + from), 0, left * 4, kRawBufferFlags);
  }
  __device__ __forceinline__ void four(int i, float (&z)[4]) const {
    const auto v = __builtin_amdgcn_raw_buffer_load_b128(rs, 4 * i, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = __uint_as_float(v[e]);
  }
  __device__ __forceinline__ void cut(int i, float (&z)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = i + e < left ? z[e] : -INFINITY;
  }
};

__global__ __launch_bounds__(kAcceptThreads) void accept_rows_kernel(AcceptArgs a) {
  __shared__ float tops[kAcceptWaves];
  __shared__ double sums[kAcceptThreads];
  __shared__ int firsts[kAcceptWaves];
  const int chunk = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, wv = tid >> 6;
  const int d0 = a.before[s], k = a.before[s + 1] - d0;
  int col = blockIdx.z;
  const bool of_target = col <= k;
  if (!of_target) {
    col -= k + 1;
    if (!a.draft || col >= k) return;
  }
  const RowPart row(of_target ? a.target + (d0 + s + col) * a.ldt : a.draft + (d0 + col) * a.ldd, chunk * kAcceptChunk, kAcceptChunk, a.vocab);
  float z[4][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) row.four(4 * (tid + kAcceptThreads * j), z[j]);
  const Heat heat(a, s);
  if (row.left < kAcceptChunk) {
#pragma unroll
    for (int j = 0; j < 4; ++j) row.cut(4 * (tid + kAcceptThreads * j), z[j]);
  }
  // a wave's own maximum, and sums of its lanes under it; they are joined below
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < 16; ++j) m = fmaxf(m, z[j >> 2][j & 3]);
  m = wave_max(m);
  double sum = 0.0;
  int first = 0x7FFFFFFF;
  if (m > -INFINITY) {
    if (heat.greedy) {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (z[j >> 2][j & 3] == m) first = min(first, chunk * kAcceptChunk + 4 * (tid + kAcceptThreads * (j >> 2)) + (j & 3));
      first = wave_min_int(first);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        double w[4];
        weights(z[j], m, heat.inv, w);
        sum += (w[0] + w[1]) + (w[2] + w[3]);
      }
    }
  }
  sums[tid] = sum;
  if ((tid & 63) == 0) {
    tops[wv] = m;
    firsts[wv] = first;
  }
  __syncthreads();
  if (tid >= 64) return;
  const float top[kAcceptWaves] = {tops[0], tops[1], tops[2], tops[3]};
  AcceptPart part;
  part.max = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  part.first = 0x7FFFFFFF;
  part.sum = 0.0;
  if (part.max > -INFINITY) {
    if (heat.greedy) {
#pragma unroll
      for (int w = 0; w < kAcceptWaves; ++w)
        if (top[w] == part.max) part.first = min(part.first, firsts[w]);
      part.sum = 1.0;
    } else {  // one wave adds the lanes up for all four: 64-bit sums over lanes are as many operations as three values' exponentials
      double w[kAcceptWaves];
      weights(top, part.max, heat.inv, w);
      part.sum = lane_of(wave_upto64((sums[tid] * w[0] + sums[64 + tid] * w[1]) + (sums[128 + tid] * w[2] + sums[192 + tid] * w[3])), 63);
    }
  }
  if (tid == 0) a.part[(size_t)(of_target ? d0 + s + col : a.rows + d0 + col) * a.chunks + chunk] = part;
}

// Joins the chunks of a row: 16 lanes l, in a fixed order.  The last of them has the result.
__device__ __forceinline__ RowStat join_chunks(const AcceptArgs& a, const Heat& heat, size_t row, int l) {
  constexpr int kAhead = 4;  // parts of a lane that are requested at once: rows of up to 262144 values in one trip
  const AcceptPart* part = a.part + row * a.chunks;
  AcceptPart p[kAhead];
  const AcceptPart none = {0.0, -INFINITY, 0x7FFFFFFF};
#pragma unroll
  for (int i = 0; i < kAhead; ++i) p[i] = l + 16 * i < a.chunks ? part[l + 16 * i] : none;
  float m = fmaxf(fmaxf(p[0].max, p[1].max), fmaxf(p[2].max, p[3].max));
  for (int c = l + 16 * kAhead; c < a.chunks; c += 16) m = fmaxf(m, part[c].max);
  m = row16_max(m);
  double sum = 0.0;
  int first = 0x7FFFFFFF;
  auto add = [&](const AcceptPart& x) {
    if (heat.greedy) {
      if (x.max == m) first = min(first, x.first);
    } else if (x.max > -INFINITY) {
      sum += x.sum * weight(x.max, m, heat.inv);
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) add(p[i]);
  for (int c = l + 16 * kAhead; c < a.chunks; c += 16) add(part[c]);
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) first = min(first, __shfl_xor(first, d));
  RowStat st;
  st.max = m;
  st.first = first;
  sum = row16_upto64(sum);
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
// The weights of N values of a thread: those from `from` + 4 j * step + .. on, four at a time
template <int N>
__device__ __forceinline__ void rest_weights(const AcceptArgs& a, const Decision& w, const Heat& heat, int from, int first, int step, double (&v)[N]) {
  const RowPart t(w.target, from, N * kAcceptThreads, a.vocab), d(w.draft ? w.draft : w.target, from, N * kAcceptThreads, a.vocab);
  float zt[N / 4][4], zd[N / 4][4];
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    t.four(first + step * j, zt[j]);
    if (w.draft) d.four(first + step * j, zd[j]);
  }
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    t.cut(first + step * j, zt[j]);
    if (w.draft) d.cut(first + step * j, zd[j]);
    const int token = from + first + step * j;
    double p[4], q[4] = {0.0, 0.0, 0.0, 0.0};
    probabilities(w.t, heat, zt[j], token, p);
    if (w.draft) {
      probabilities(w.d, heat, zd[j], token, q);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e] = token + e == w.x ? 1.0 : 0.0;  // of no token if x is -1
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * j + e] = w.x < 0 ? p[e] : fmax(p[e] - q[e], 0.0);
  }
}

// Over the workgroup: the sum of the threads' values, and of those before
struct Found {
  double before, total;
};
__device__ __forceinline__ Found threads_before(double own, double* lds, int lane, int wv) {
  const double upto = wave_upto64(own);
  if (lane == 63) lds[wv] = upto;
  __syncthreads();
  Found f;
  f.total = 0.0;
  double waves = 0.0;
#pragma unroll
  for (int i = 0; i < kAcceptWaves; ++i) {
    if (i == wv) waves = f.total;
    f.total += lds[i];
  }
  f.before = waves + (upto - own);
  __syncthreads();
  return f;
}
// The lowest of the threads' numbers, and the highest of others
struct Ends {
  int low, high;
};
__device__ __forceinline__ Ends lowest_and_highest(int low, int high, int* lds, int lane, int wv) {
  // numbers ascend with the lanes: of the first and the last that has one
  const uint64_t lows = __builtin_amdgcn_ballot_w64(low != 0x7FFFFFFF), highs = __builtin_amdgcn_ballot_w64(high >= 0);
  low = lows ? __builtin_amdgcn_readlane(low, __ffsll((unsigned long long)lows) - 1) : 0x7FFFFFFF;
  high = highs ? __builtin_amdgcn_readlane(high, 63 - __clzll((long long)highs)) : -1;
  if (lane == 0) {
    lds[wv] = low;
    lds[kAcceptWaves + wv] = high;
  }
  __syncthreads();
  Ends e = {lds[0], lds[kAcceptWaves]};
#pragma unroll
  for (int i = 1; i < kAcceptWaves; ++i) {
    e.low = min(e.low, lds[i]);
    e.high = max(e.high, lds[kAcceptWaves + i]);
  }
  __syncthreads();
  return e;
}

// The token of N * kAcceptThreads values from `from` on at which the sum of the weights exceeds `share`, or the last with a weight
template <int N>
__device__ __forceinline__ int token_at(const AcceptArgs& a, const Decision& w, const Heat& heat, int from, double share, double* lds, int* ints,
                                        int tid) {
  const int lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  double v[N], own = 0.0;
  rest_weights<N>(a, w, heat, from, N * tid, 4, v);
#pragma unroll
  for (int j = 0; j < N; ++j) own += v[j];
  double c = threads_before(own, lds, lane, wv).before;
  int over = 0x7FFFFFFF, last = -1;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    c += v[j];
    if (v[j] > 0.0) {
      last = from + N * tid + j;
      if (c > share) over = min(over, last);
    }
  }
  const Ends e = lowest_and_highest(over, last, ints, lane, wv);
  return e.low != 0x7FFFFFFF ? e.low : e.high;
}

// The drafts that are kept, by a workgroup of the sequence each
__device__ __forceinline__ AcceptOutcome settle(const AcceptArgs& a, const Heat& heat, int s, int d0, int k, int tid, bool tell) {
  __shared__ RowStat stats[2 * kAcceptDrafts + 1];
  __shared__ int s_kept, s_x;
  const int lane = tid & 63, n_rows = a.draft ? 2 * k + 1 : k + 1;
  // a lane's draft: requested before the rows' parts, which its probabilities wait for
  int x = -1;
  double r = 0.0;
  float zt = -INFINITY, zd = -INFINITY;
  if (tid < k) {
    x = a.tokens[d0 + tid];
    r = a.r[d0 + s + tid];
  }
  if (x >= 0 && x < a.vocab) {
    zt = a.target[(d0 + s + lane) * a.ldt + x];
    if (a.draft) zd = a.draft[(d0 + lane) * a.ldd + x];
  }
  // the rows' maxima and sums, the target's first
  for (int i0 = 0; i0 < n_rows; i0 += kAcceptThreads / 16) {
    const int i = i0 + (tid >> 4), row = min(i, n_rows - 1);
    const RowStat st = join_chunks(a, heat, row <= k ? d0 + s + row : a.rows + d0 + row - k - 1, lane & 15);
    if ((lane & 15) == 15 && i < n_rows) stats[i] = st;
  }
  __syncthreads();
  if (tid < 64) {
    bool good = false;
    if (lane < k) {
      double p = 0.0, q = 0.0;
      if (x >= 0 && x < a.vocab) {
        p = probability(stats[lane], heat, zt, x);
        q = a.draft ? probability(stats[k + 1 + lane], heat, zd, x) : 1.0;
      }
      good = p > 0.0 && r <= p / q;
      if (tell) {
        if (a.p) a.p[d0 + lane] = (float)p;
        if (a.q) a.q[d0 + lane] = (float)q;
      }
    }
    const uint64_t bad = ~__builtin_amdgcn_ballot_w64(good);  // a lane without a draft is not kept either
    const int kept = bad ? __ffsll((unsigned long long)bad) - 1 : kAcceptDrafts;
    x = x < 0 ? 0x7FFFFFFF : x;  // no token of the vocabulary
    const int next = kept < k ? __builtin_amdgcn_readlane(x, kept & 63) : -1;
    if (lane == 0) {
      s_kept = kept;
      s_x = next;
    }
  }
  __syncthreads();
  AcceptOutcome v;
  v.kept = __builtin_amdgcn_readfirstlane(s_kept);
  v.x = __builtin_amdgcn_readfirstlane(s_x);
  v.t = stats[v.kept];
  v.d = stats[a.draft && v.kept < k ? k + 1 + v.kept : v.kept];
  return v;
}
__device__ __forceinline__ Decision decide(const AcceptArgs& a, const AcceptOutcome& v, int s, int d0, int k) {
  Decision w;
  w.t = v.t;
  w.d = v.d;
  w.target = a.target + (d0 + s + v.kept) * a.ldt;
  w.draft = nullptr;
  w.x = v.x;
  if (v.kept < k && a.draft) w.draft = a.draft + (d0 + v.kept) * a.ldd;
  return w;
}

__global__ __launch_bounds__(kAcceptThreads) void accept_drafts_kernel(AcceptArgs a) {
  __shared__ double sums[kAcceptWaves];
  const int s = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int d0 = a.before[s], k = a.before[s + 1] - d0;
  const Heat heat(a, s);
  const AcceptOutcome v = settle(a, heat, s, d0, k, tid, blockIdx.x == 0);
  if (blockIdx.x == 0 && tid == 0) a.outcome[s] = v;
  if (v.kept == k) return;  // the sums of the first launch do
  const Decision w = decide(a, v, s, d0, k);
  for (int piece = blockIdx.x * a.each, end = min(piece + a.each, a.pieces); piece < end; ++piece) {
    double x[kAcceptPiece / kAcceptThreads], sum = 0.0;
    rest_weights(a, w, heat, piece * kAcceptPiece, 4 * tid, 4 * kAcceptThreads, x);
#pragma unroll
    for (const double y : x) sum += y;
    const double total = threads_before(sum, sums, lane, wv).total;
    if (tid == 0) a.rest[(size_t)s * a.pieces + piece] = total;
  }
}

// ALONE: no sequence has drafts, and the second launch was left out
template <bool ALONE>
__global__ __launch_bounds__(kAcceptThreads) void accept_draw_kernel(AcceptArgs a) {
  __shared__ double sums[kAcceptWaves];
  __shared__ int ints[2 * kAcceptWaves];
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int d0 = a.before[s], k = a.before[s + 1] - d0;
  const double u = a.r[d0 + s + k];
  double early = 0.0;  // the sum of the thread's piece, if pieces it will be
  if (!ALONE && tid < a.pieces) early = a.rest[(size_t)s * a.pieces + tid];
  const Heat heat(a, s);
  AcceptOutcome v;
  if constexpr (ALONE) v = settle(a, heat, s, d0, k, tid, false);
  else v = a.outcome[s];
  const int kept = __builtin_amdgcn_readfirstlane(v.kept);
  v.kept = kept;
  v.x = __builtin_amdgcn_readfirstlane(v.x);
  Decision w = decide(a, v, s, d0, k);

  // the piece (chunk) of the token: the first whose sum up to and with itself exceeds the number's share
  int token = -1;
  for (int turn = 0; turn < 2; ++turn) {
    const bool pieces = w.x >= 0;
    const int n = pieces ? a.pieces : a.chunks;
    const AcceptPart* part = a.part + (size_t)(d0 + s + kept) * a.chunks;
    auto sum_of = [&](int c) -> double {
      if (c >= n) return 0.0;
      if (pieces) return a.rest[(size_t)s * a.pieces + c];
      const AcceptPart p = part[c];
      if (p.max == -INFINITY) return 0.0;
      if (heat.greedy) return p.max == w.t.max && p.first == w.t.first ? 1.0 : 0.0;
      // Drawn only where a token of it has a weight, as token_at forms it: thousands of tokens may add up to a smallest number that
      // each of them is below
      const double most = weight(p.max, w.t.max, heat.inv) * w.t.scale;
      return most > 0.0 ? p.sum * most : 0.0;
    };
    double own = pieces ? early : sum_of(tid);
    Found f = threads_before(own, sums, lane, wv);
    double total = f.total;
    for (int c0 = kAcceptThreads; c0 < n; c0 += kAcceptThreads) total += threads_before(sum_of(c0 + tid), sums, lane, wv).total;
    if (total > 0.0) {
      const double share = u * total;
      double before = 0.0, left = INFINITY;  // left: of the share, where the piece begins
      int at = -1, last = -1;
      for (int c0 = 0; c0 < n && at < 0; c0 += kAcceptThreads) {
        if (c0 > 0) {
          own = sum_of(c0 + tid);
          f = threads_before(own, sums, lane, wv);
        }
        const Ends e = lowest_and_highest(own > 0.0 && before + f.before + own > share ? c0 + tid : 0x7FFFFFFF, own > 0.0 ? c0 + tid : -1, ints, lane, wv);
        if (e.low != 0x7FFFFFFF) {
          at = e.low;
          if (c0 + tid == at) sums[0] = share - (before + f.before);
          __syncthreads();
          left = sums[0];
          __syncthreads();
        }
        last = max(last, e.high);
        before += f.total;
      }
      if (at < 0) at = last;  // a number of 1 or above, or a sum that rounding put below it: the last token
      at = __builtin_amdgcn_readfirstlane(at);
      token = pieces ? token_at<kAcceptPiece / kAcceptThreads>(a, w, heat, at * kAcceptPiece, left, sums, ints, tid)
                     : token_at<kAcceptChunk / kAcceptThreads>(a, w, heat, at * kAcceptChunk, left, sums, ints, tid);
      break;
    }
    if (w.x < 0) break;
    w.x = -1;  // nothing left of p - q, by rounding: p
  }
  for (int64_t i = tid; i < a.ld_out; i += kAcceptThreads)
    a.out[s * a.ld_out + i] = i < kept ? a.tokens[d0 + i] : i == kept ? token : -1;
  if (tid == 0) a.n_accepted[s] = kept;
}

// Where the parts of the workspace lie; 0 bytes for arguments that are refused
struct AcceptPlan {
  int64_t drafts = 0, rest = 0, outcome = 0, bytes = 0;
  int most = 0, chunks = 0, pieces = 0;
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
  p.pieces = (vocab + kAcceptPiece - 1) / kAcceptPiece;
  auto up256 = [](int64_t b) { return (b + 255) / 256 * 256; };
  p.rest = up256((2 * p.drafts + n_seqs) * p.chunks * (int64_t)sizeof(AcceptPart));
  p.outcome = p.rest + up256((int64_t)n_seqs * p.pieces * 8);
  p.bytes = p.outcome + up256((int64_t)n_seqs * (int64_t)sizeof(AcceptOutcome));
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
  a.outcome = (cas::AcceptOutcome*)(ws + plan.outcome);
  a.vocab = vocab; a.chunks = plan.chunks; a.pieces = plan.pieces; a.rows = (int)plan.drafts + n_seqs;
  for (int i = 0; i < n_seqs; ++i) a.before[i + 1] = a.before[i] + h_k[i];
  const int cols = plan.most + 1 + (a.draft ? plan.most : 0);
  hipLaunchKernelGGL(cas::accept_rows_kernel, dim3(plan.chunks, n_seqs, cols), dim3(cas::kAcceptThreads), 0, ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  if (plan.most > 0) {
    // a workgroup a piece, or more pieces where there are enough workgroups for every place: each joins the rows anew.  32 sequences
    // of up to 7 drafts over 128256 tokens, us of all launches, with 4 / 2 / 1 workgroups a CU: 59 / 54 / 55
    a.each = std::max(1, (int)((int64_t)n_seqs * plan.pieces / (2 * ctx->num_cu)));
    hipLaunchKernelGGL(cas::accept_drafts_kernel, dim3((plan.pieces + a.each - 1) / a.each, n_seqs), dim3(cas::kAcceptThreads), 0, ctx->stream, a);
    CAS_HIP(ctx, hipGetLastError());
  }
  hipLaunchKernelGGL(plan.most > 0 ? cas::accept_draw_kernel<false> : cas::accept_draw_kernel<true>, dim3(n_seqs), dim3(cas::kAcceptThreads), 0,
                     ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

size_t cas_accept_tokens_bytes(int n_seqs, const int32_t* h_k, int vocab) {
  cas::AcceptPlan plan;
  return cas::plan_accept(n_seqs, h_k, vocab, &plan) == CAS_OK ? (size_t)plan.bytes : 0;
}

}  // extern "C"
