// Eviction from the compressed cache: which positions of a row of scores stay, and the encoded vectors of these moved
// to the front of a sequence's pages as they are (no stream is decoded).
#include <algorithm>
#include "cas_device.hpp"
#include "cas_internal.hpp"

namespace cas {

// ---- selection ----------------------------------------------------------------------------------
// One workgroup per row.  The scores between the first and the last positions are mapped to integers of the same order;
// the threshold (the highest value that enough of them reach) is found kSelBits at a time: counts per digit in LDS, then the
// digit with which enough are reached by a sum over the counts; and of its equals the lower positions are taken.  Kept positions
// are dealt their places by counting those before them: ballots within a wave, one table of counts per wave and step for the workgroup.
// Bound by latency (three passes of four barriers), for long rows by vector issue of the one CU that a row has: the counts of a
// row meet in one LDS, so a layer's 8 rows use 8 of 256 CUs.  us, also where all scores are equal, and with two bits a turn by
// ballots instead of digits in LDS: 8 rows of 2049 6.8 / 8.5 / 9.9, of 8192 12.0 / 14.7 / 17, of 21647 27 / 32 / 42; 256 of 8192
// 14.6 / 15.6 / 19.7 (8 MB read and 4 written: 3 at the rate of a copy).
constexpr int kSelBits = 11, kSelBins = 1 << kSelBits;
constexpr int kGroup = 4;  // steps between two looks at the row's end
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;

__device__ __forceinline__ uint32_t score_key(float v) {  // NaN on top, -0 as +0; 0 is below every key
  if (v != v) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(v + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct SelectArgs {
  const float* score;
  int64_t ld, ld_kept;
  int len, n_keep, n_first, n_last;
  int32_t* index;
  float* kept;
};

// PER: scores of a thread kept in registers; 0: read again wherever they are needed, rows too long for registers.
template <int PER>
__global__ __launch_bounds__(kSelThreads) void select_kernel(SelectArgs a) {
  constexpr int N = PER > 0 ? PER : 1;
  constexpr int kAhead = 8;  // scores requested at once where they are read again
  __shared__ __align__(8) uint32_t bins[kSelBins];
  __shared__ uint32_t wave_total[kSelWaves], found[3];
  __shared__ uint32_t place[PER > 0 ? PER * kSelWaves : 2 * kSelWaves];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float* row = a.score + (int64_t)blockIdx.x * a.ld;
  int32_t* index = a.index + (int64_t)blockIdx.x * a.n_keep;
  float* kept = a.kept ? a.kept + (int64_t)blockIdx.x * a.ld_kept : nullptr;
  const int lo = a.n_first, hi = a.len - a.n_last;   // the middle: positions lo .. hi - 1
  const uint32_t want = (uint32_t)(a.n_keep - a.n_first - a.n_last);
  const int steps = (a.len + kSelThreads - 1) / kSelThreads;
  auto value = [&](int i) {
    const int p = i * kSelThreads + tid;
    return p < a.len ? row[p] : 0.f;
  };
  auto key_of = [&](int i, float x) {  // 0 outside the middle
    int p = tid;
    asm volatile("" : "+v"(p));  // worked out anew each time: the places and answers of all steps do not fit the registers
    p += i * kSelThreads;
    return p >= lo && p < hi ? score_key(x) : 0u;
  };
  float v[N];
  if constexpr (PER > 0) {  // 0 behind the row: the whole distance in the offset that is checked, the scalar one is not
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(row), 0, 4 * a.len, kRawBufferFlags);
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, 4 * (tid + i * kSelThreads), 0, 0));
  }
  // f(key) of every position, the workgroup's waves together
  auto each = [&](auto&& f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int i = 0; i < PER; i += kGroup) {
        if (i > 0 && i * kSelThreads >= a.len) break;
#pragma unroll
        for (int q = 0; q < kGroup; ++q) f(key_of(i + q, v[i + q]));
        asm volatile("" ::: "memory");
      }
    } else {
      for (int i = 0; i < steps; i += kAhead) {
        float x[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) x[q] = value(i + q);
#pragma unroll
        for (int q = 0; q < kAhead; ++q) f(key_of(i + q, x[q]));
      }
    }
  };
  // The largest T that at least `want` keys reach, some bits a pass; found early where exactly `want` keys reach it with the
  // bits behind as zeros.
  uint32_t T = 0, above = 0;
  if (want > 0) {
    bool exact = false;
    for (int left = 32; left > 0 && !exact;) {  // bits of T that are not known
      const int next = max(left - kSelBits, 0);
      const uint32_t mask = (1u << (left - next)) - 1u;
      for (int i = tid; i < kSelBins; i += kSelThreads) bins[i] = 0;
      __syncthreads();
      each([&](uint32_t k) {
        const bool in = k != 0 && (k ^ T) >> 1 >> (left - 1) == 0;
        const uint64_t all = __builtin_amdgcn_ballot_w64(in);
        if (all == 0) return;
        // those that agree with the first of them in one addition: many scores may be the same (all of 8192: 28.7 -> 14.7 us, none 10.2 -> 12.3)
        const int digit = kSelBins - 1 - (int)(k >> next & mask), first = __builtin_ctzll(all);
        const bool same = in && digit == __builtin_amdgcn_readlane(digit, first);
        const uint32_t agree = (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(same));
        if (in && (!same || lane == first)) atomicAdd(&bins[digit], same ? agree : 1u);
      });
      __syncthreads();
      const uint2 c = *reinterpret_cast<const uint2*>(bins + 2 * tid);  // the higher digits first
      const uint32_t sum = c.x + c.y, incl = (uint32_t)wave_incl_scan((int)sum);
      if (lane == 63) wave_total[wv] = incl;
      __syncthreads();
      uint32_t before = above + incl - sum;
#pragma unroll
      for (int w = 0; w < kSelWaves; ++w) before += w < wv ? wave_total[w] : 0u;
      if (before < want && before + sum >= want) {  // one thread
        const bool second = before + c.x < want;
        found[0] = T | (uint32_t)(kSelBins - 1 - (2 * tid + second)) << next;
        found[1] = second ? before + c.x : before;
        found[2] = second ? c.y : c.x;
      }
      __syncthreads();
      T = (uint32_t)__builtin_amdgcn_readfirstlane((int)found[0]);
      above = (uint32_t)__builtin_amdgcn_readfirstlane((int)found[1]);
      exact = above + (uint32_t)__builtin_amdgcn_readfirstlane((int)found[2]) == want;
      left = next;
    }
    if (exact) {  // those that reach T are those that stay: none is equal to one below it
      T -= 1u;
      above = want;
    }
  }
  const uint32_t ties = want - above;  // equals of the threshold that stay
  auto sure_of = [&](int i, uint32_t k) {
    int p = tid;
    asm volatile("" : "+v"(p));
    p += i * kSelThreads;
    return (p < a.len && (p < lo || p >= hi)) || (want > 0 && k > T);
  };
  auto tie_of = [&](uint32_t k) { return want > 0 && k == T; };
  // before: those kept for sure in the lower half, equals in the upper, of the positions in front of the wave's 64
  auto put = [&](int i, float x, bool sure, bool tie, uint64_t ms, uint64_t mt, uint32_t s_before, uint32_t t_before) {
    const uint64_t below = (1ull << lane) - 1ull;
    const uint32_t t_rank = t_before + (uint32_t)__popcll(mt & below);
    if (sure || (tie && t_rank < ties)) {
      const uint32_t at = s_before + (uint32_t)__popcll(ms & below) + min(t_rank, ties);
      if (at < (uint32_t)a.n_keep) {  // also where scores change meanwhile
        index[at] = i * kSelThreads + tid;
        if (kept) kept[at] = x;
      }
    }
  };
  if constexpr (PER > 0) {
    // one table of the counts of every 64 positions, summed up by one wave (at most 2^16 of either kind, those in front of the last 64 fewer)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (i * kSelThreads >= a.len) break;
      const uint32_t k = key_of(i, v[i]);
      const uint64_t ms = __builtin_amdgcn_ballot_w64(sure_of(i, k)), mt = __builtin_amdgcn_ballot_w64(tie_of(k));
      if (lane == 0) place[i * kSelWaves + wv] = (uint32_t)__popcll(ms) | (uint32_t)__popcll(mt) << 16;
      asm volatile("" ::: "memory");
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // all scores are here, over which kept ones may be written
    __syncthreads();
    if (wv == 0) {
      constexpr int kEach = PER * kSelWaves / 64;  // entries of a lane
      uint32_t c[kEach], sum = 0;
#pragma unroll
      for (int q = 0; q < kEach; ++q) {
        const int e = lane * kEach + q;
        c[q] = e < steps * kSelWaves ? place[e] : 0u;
        sum += c[q];
      }
      uint32_t before = (uint32_t)wave_incl_scan((int)sum) - sum;
#pragma unroll
      for (int q = 0; q < kEach; ++q) {
        place[lane * kEach + q] = before;
        before += c[q];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (i * kSelThreads >= a.len) break;
      const uint32_t k = key_of(i, v[i]), before = place[i * kSelWaves + wv];
      const bool sure = sure_of(i, k), tie = tie_of(k);
      put(i, v[i], sure, tie, __builtin_amdgcn_ballot_w64(sure), __builtin_amdgcn_ballot_w64(tie), before & 0xFFFFu, before >> 16);
      asm volatile("" ::: "memory");
    }
  } else {
    uint32_t s_base = 0, t_base = 0;
    for (int i = 0; i < steps; ++i) {
      const float x = value(i);
      const uint32_t k = key_of(i, x);
      const bool sure = sure_of(i, k), tie = tie_of(k);
      const uint64_t ms = __builtin_amdgcn_ballot_w64(sure), mt = __builtin_amdgcn_ballot_w64(tie);
      __syncthreads();  // the counts of the step before have been read
      if (lane == 0) {
        place[2 * wv] = (uint32_t)__popcll(ms);
        place[2 * wv + 1] = (uint32_t)__popcll(mt);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();  // and this step's scores are here, over which a kept one may be written
      uint32_t s_before = s_base, t_before = t_base;
#pragma unroll
      for (int w = 0; w < kSelWaves; ++w) {
        const uint32_t s = place[2 * w], t = place[2 * w + 1];
        s_before += w < wv ? s : 0u;
        t_before += w < wv ? t : 0u;
        s_base += s;
        t_base += t;
      }
      put(i, x, sure, tie, ms, mt, s_before, t_before);
    }
  }
}

// ---- moving ---------------------------------------------------------------------------------------
// A tile (64 vectors of one head) is two runs of words, its parts of the two pools, each made of streams of w words per
// vector in vector order.  A thread moves four words of a vector, the last four of a stream where fewer are left (two threads then
// write the same words): one load and one store of 16 bytes each, on multiples of 4 bytes, for every stream of four words
// or more.  Bound by latency and address units.  With 16 bytes of the destination to a thread, which may reach into the next
// vector, a quarter of the threads needs four loads, and their waves five: 175 us for 32 layers of 2048 of 8192 positions
// (549 MB read and written: 115 at the rate of a copy), now 141, or 160 in a row of such moves.
struct MoveStream {
  int begin, w;       // first word in the pool's part of a tile, words of a vector
  int first, groups;  // threads before, and to a vector
  uint32_t inv;       // ceil(2^18 / groups): place e < 2^14 of the stream takes vector e * inv >> 18
};
struct MoveArgs {
  KvGeom g;
  uint32_t* pool[2];
  int tile_words[2];
  int n_streams[2];
  MoveStream s[2][3];
  int threads[2];     // of a tile
  const int32_t* src_row;
  const int32_t* dst_row;
  const int32_t* index;
  int layer0, n_keep, len;
};

constexpr int kMoveThreads = 256;
constexpr int kMoveEach = 5;  // places of a thread: 64 vectors of at most 17 groups, 1088, in 5 x 256

typedef unsigned int words4 __attribute__((ext_vector_type(4), aligned(4)));
struct MovePlace {
  int row = 64, at = 0, w = 0, begin = 0;  // vector of the tile (of a step), first word of the four in it, the stream
  __device__ __forceinline__ MovePlace(const MoveStream& s, int e) : row((int)((uint32_t)e * s.inv >> 18)), w(s.w), begin(s.begin) {
    at = max(min(4 * (e - row * s.groups), s.w - 4), 0);
  }
  __device__ __forceinline__ MovePlace(const MoveStream (&t)[3], int n_streams, int threads, int e) {
    if (e >= threads) return;
    MoveStream s = t[0];
#pragma unroll
    for (int i = 1; i < 3; ++i)
      if (i < n_streams && e >= t[i].first) s = t[i];
    *this = MovePlace(s, e - s.first);
  }
  __device__ __forceinline__ void load(const uint32_t* from, words4& v) const {
    if (w >= 4) {
      v = __builtin_nontemporal_load(reinterpret_cast<const words4*>(from + at));  // read once: 148 -> 143 us for those
    } else {
      v.x = from[0];
      v.y = w > 1 ? from[1] : 0u;
      v.z = w > 2 ? from[2] : 0u;
    }
  }
  __device__ __forceinline__ void store(uint32_t* to, words4 v) const {
    if (w >= 4) {
      *reinterpret_cast<words4*>(to + at) = v;
    } else {
      to[0] = v.x;
      if (w > 1) to[1] = v.y;
      if (w > 2) to[2] = v.z;
    }
  }
};

// blockIdx.y: K heads, then V heads; blockIdx.z: 2 * layer + pool.
__global__ __launch_bounds__(kMoveThreads, 8) void move_kernel(MoveArgs a) {
  __shared__ const uint32_t* src[64];
  __shared__ int row[64];
  const KvGeom& g = a.g;
  const int pool = blockIdx.z & 1, layer = blockIdx.z >> 1, kvh = blockIdx.y, tid = threadIdx.x;
  const int head = kvh % g.n_kv_heads, kv = kvh / g.n_kv_heads;
  const int32_t* index = a.index + ((int64_t)layer * g.n_kv_heads + head) * a.n_keep;
  auto part = [&](int page) {
    const size_t tile = (((size_t)(a.layer0 + layer) * g.n_pages + page) * 2 + kv) * g.n_kv_heads + head;
    return a.pool[pool] + tile * a.tile_words[pool];
  };
  MoveStream streams[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {  // in scalar registers: a choice among them must not become a load per lane
    streams[i] = a.s[pool][i];
    asm("" : "+s"(streams[i].begin), "+s"(streams[i].w), "+s"(streams[i].first), "+s"(streams[i].groups), "+s"(streams[i].inv));
  }
  const int n_streams = a.n_streams[pool], threads = a.threads[pool], t = blockIdx.x;
  const int rows = min(64, a.n_keep - 64 * t);
  if (tid < 64) {
    const int p = min(max(index[64 * t + min(tid, rows - 1)], 0), a.len - 1);
    src[tid] = part(min(max(a.src_row[p >> 6], 0), g.n_pages - 1));
    row[tid] = p & 63;
  }
  __syncthreads();
  words4 v[kMoveEach];
#pragma unroll
  for (int i = 0; i < kMoveEach; ++i) {
    const MovePlace m(streams, n_streams, threads, tid + i * kMoveThreads);
    if (m.row < rows) m.load(src[m.row] + m.begin + row[m.row] * m.w, v[i]);
  }
  const int page = a.dst_row[t];
  if (page >= 0 && page < g.n_pages) {
    uint32_t* const dst = part(page);
#pragma unroll
    for (int i = 0; i < kMoveEach; ++i) {
      const MovePlace m(streams, n_streams, threads, tid + i * kMoveThreads);
      if (m.row < rows) m.store(dst + m.begin + m.row * m.w, v[i]);
    }
  }
}

// In place: a workgroup takes one stream (blockIdx.x) of a head (blockIdx.y: K heads, then V heads) of layer blockIdx.z, as many
// vectors a step as its places hold; all are read before one is written.  Position i moves to or before the place it comes from (the indices
// ascend), so that no step writes what a later one reads.  The places of the next step's vectors are looked up under the
// loads of this one.  Bound by the latency of a step (a stream of 7 or 8 groups has one per 585 or 512 vectors), and one
// after the other: what a step writes over may be what the step before reads, so that several workgroups to a stream would have
// to wait for one another.  us, with a tile of 64 vectors and all streams of a pool a step / this: one layer, 1024 of 2049 positions
// 35 / 8.9, 2048 of 8192 75 / 19, 16384 of 32768 663 / 124; 32 layers, 2048 of 8192 176 / 177.
constexpr int kInPlaceThreads = 1024, kInPlaceEach = 4;
__global__ __launch_bounds__(kInPlaceThreads, 8) void move_in_place_kernel(MoveArgs a) {
  const KvGeom& g = a.g;
  const int pool = (int)blockIdx.x >= a.n_streams[0], kvh = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x;
  const int head = kvh % g.n_kv_heads, kv = kvh / g.n_kv_heads;
  const MoveStream s = a.s[pool][blockIdx.x - (pool ? a.n_streams[0] : 0)];
  const int32_t* index = a.index + ((int64_t)layer * g.n_kv_heads + head) * a.n_keep;
  auto part = [&](int page) {
    const size_t tile = (((size_t)(a.layer0 + layer) * g.n_pages + page) * 2 + kv) * g.n_kv_heads + head;
    return a.pool[pool] + tile * a.tile_words[pool];
  };
  constexpr int kPlaces = kInPlaceEach * kInPlaceThreads;
  __shared__ const uint32_t* src[kPlaces];     // of a step's vectors
  __shared__ uint32_t* dst[2][kPlaces / 64 + 1];  // of its tiles; two sets in turn, the stores of a step use one while the next is written
  const int step = (int)((uint32_t)kPlaces * s.inv >> 18);  // vectors
  const uint32_t* from[kInPlaceEach];
  auto look_up = [&](int r0) {
#pragma unroll
    for (int i = 0; i < kInPlaceEach; ++i) {
      if (i * kInPlaceThreads >= step) break;
      const int p = min(max(index[min(r0 + tid + i * kInPlaceThreads, a.n_keep - 1)], 0), a.len - 1);
      from[i] = part(min(max(a.src_row[p >> 6], 0), g.n_pages - 1)) + s.begin + (p & 63) * s.w;
    }
  };
  look_up(0);
  int set = 0;
#pragma unroll 1
  for (int r0 = 0; r0 < a.n_keep; r0 += step, set ^= 1) {
    const int rows = min(step, a.n_keep - r0), tile0 = r0 >> 6;
#pragma unroll
    for (int i = 0; i < kInPlaceEach; ++i)
      if (tid + i * kInPlaceThreads < rows) src[tid + i * kInPlaceThreads] = from[i];
    if (tid <= (r0 + rows - 1) / 64 - tile0) {
      const int page = a.dst_row[tile0 + tid];
      dst[set][tid] = page >= 0 && page < g.n_pages ? part(page) + s.begin : nullptr;
    }
    __syncthreads();
    words4 v[kInPlaceEach];
#pragma unroll
    for (int i = 0; i < kInPlaceEach; ++i) {
      const MovePlace m(s, tid + i * kInPlaceThreads);
      m.load(src[min(m.row, rows - 1)], v[i]);
    }
    if (r0 + step < a.n_keep) look_up(r0 + step);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // all vectors of the step are in registers
#pragma unroll
    for (int i = 0; i < kInPlaceEach; ++i) {
      const MovePlace m(s, tid + i * kInPlaceThreads);
      if (m.row < rows) {
        uint32_t* const to = dst[set][((r0 + m.row) >> 6) - tile0];
        if (to) m.store(to + ((r0 + m.row) & 63) * s.w, v[i]);
      }
    }
  }
}

static int launch_select(cas_ctx* ctx, const SelectArgs& a, int n_rows) {
  const dim3 grid(n_rows), block(kSelThreads);
  if (a.len <= 8 * kSelThreads) hipLaunchKernelGGL(select_kernel<8>, grid, block, 0, ctx->stream, a);
  // longer rows from registers too, up to 64 scores a lane, where 66 of the 128 spill: 8 rows of 60000 85 us, 136 reading them again
  else if (a.len <= 32 * kSelThreads) hipLaunchKernelGGL(select_kernel<32>, grid, block, 0, ctx->stream, a);
  else if (a.len <= 64 * kSelThreads) hipLaunchKernelGGL(select_kernel<64>, grid, block, 0, ctx->stream, a);
  else hipLaunchKernelGGL(select_kernel<0>, grid, block, 0, ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

static void add_stream(MoveArgs& a, int pool, int begin, int w) {
  if (w == 0) return;
  const int groups = (w + 3) / 4;
  a.s[pool][a.n_streams[pool]++] = MoveStream{begin, w, a.threads[pool], groups, ((1u << 18) + (uint32_t)groups - 1u) / (uint32_t)groups};
  a.threads[pool] += 64 * groups;
}

static int launch_evict(cas_ctx* ctx, cas_kv* kv, int layer0, int n_layers, int seq, int dst_seq, const int32_t* d_index, int n_keep) {
  const KvGeom& g = kv->geom;
  MoveArgs a{};
  a.g = g;
  a.pool[0] = (uint32_t*)kv->d_spec; a.pool[1] = (uint32_t*)kv->d_verif;
  a.tile_words[0] = g.tile_spec_words; a.tile_words[1] = g.tile_verif_words;
  add_stream(a, 0, 0, 4);
  if (g.mx) add_stream(a, 0, 64 * 4, 1);
  add_stream(a, 0, g.spec_off, g.sw);
  add_stream(a, 1, 0, g.lw);
  add_stream(a, 1, 64 * g.lw, g.pw);
  a.src_row = kv->d_page_table + (size_t)seq * g.max_pages_per_seq;
  a.dst_row = kv->d_page_table + (size_t)dst_seq * g.max_pages_per_seq;
  a.index = d_index;
  a.layer0 = layer0; a.n_keep = n_keep; a.len = kv->h_len[seq];
  const int tiles = (n_keep + 63) / 64;
  if (seq == dst_seq) hipLaunchKernelGGL(move_in_place_kernel, dim3(a.n_streams[0] + a.n_streams[1], 2 * g.n_kv_heads, n_layers), dim3(kInPlaceThreads), 0, ctx->stream, a);
  else hipLaunchKernelGGL(move_kernel, dim3(tiles, 2 * g.n_kv_heads, 2 * n_layers), dim3(kMoveThreads), 0, ctx->stream, a);
  CAS_HIP(ctx, hipGetLastError());
  return CAS_OK;
}

}  // namespace cas

extern "C" {

int cas_kv_select(cas_ctx* ctx, const float* d_score, int64_t ld, int n_rows, int len, int n_keep, int n_first, int n_last,
                  int32_t* d_index, float* d_kept, int64_t ld_kept) {
  if (!ctx || n_rows < 0 || len < 0 || ld < len || n_first < 0 || n_last < 0 || n_keep < 0 || n_keep > len) return CAS_EINVAL;
  if ((int64_t)n_first + n_last > n_keep || (d_kept && ld_kept < n_keep)) return CAS_EINVAL;
  if (d_kept && d_kept == d_score && ld_kept != ld) return CAS_EINVAL;
  if (n_rows == 0 || n_keep == 0) return CAS_OK;
  if (len > 1 << 30 || n_rows > 0x3FFFFF) return CAS_ENOTSUP;  // a launch has fewer than 2^32 threads
  if (!d_score || !d_index || !cas::on_device(ctx)) return CAS_EINVAL;
  cas::SelectArgs a{d_score, ld, ld_kept, len, n_keep, n_first, n_last, d_index, d_kept};
  return cas::launch_select(ctx, a, n_rows);
}

int cas_kv_evict(cas_ctx* ctx, cas_kv* kv, int layer0, int n_layers, int seq, int dst_seq, const int32_t* d_index, int n_keep) {
  if (!ctx || !kv || seq < 0 || seq >= kv->desc.max_seqs || dst_seq < 0 || dst_seq >= kv->desc.max_seqs) return CAS_EINVAL;
  if (layer0 < 0 || n_layers < 0 || n_layers > kv->desc.n_layers - layer0 || n_keep < 0 || n_keep > kv->h_len[seq]) return CAS_EINVAL;
  if (n_layers == 0 || n_keep == 0) return CAS_OK;
  if (!d_index || !cas::on_device(ctx)) return CAS_EINVAL;
  return cas::launch_evict(ctx, kv, layer0, n_layers, seq, dst_seq, d_index, n_keep);
}

}  // extern "C"
