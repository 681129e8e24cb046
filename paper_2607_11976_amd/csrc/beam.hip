// Beam search's selection: of a request's beams w, each with a score c_w and a row
// of logits x_w, the `top` best continuations by
//
//   score(w, v) = c_w + scale x_wv - lse_w,   lse_w = log sum_v exp(scale x_wv),
//
// computed from the row's largest logit m as c_w + (scale (x_wv - m_w) - log s_w) with
// s_w = sum_v exp(scale (x_wv - m_w)): scale m_w may be so large (a mask of the type's
// lowest value) that log s_w is lost beside it.
//
// Order: larger score (float32) first; equal ones by beam, then by logit, then by
// token. Within a beam the score rises with the logit, so a beam's best `top` logits
// hold all that it can give, whatever its sum: one pass over the logits takes the
// sums and, per part of a row, the best `top` (logit, token) pairs; a second kernel
// joins a request's parts.
//
// Scores of different beams lie close together (a step of float32 at 20 is 2e-6), and
// their order is the result, so the sums are kept better than float32: a lane adds
// up 2^((x - m) scale log2 e) relative to its own largest logit m in short float32
// chains, those in float64; scale log2 e is two float32 numbers, and log s and score
// are float64 until the score's one rounding. What is float32, the distances, exponents
// and powers, makes log s wrong by (2 H + 2 j + 12) 2^-24 at most: 2 H for the first two,
// H the row's entropy (it bounds the mean distance to the largest logit), 2 for every
// power, of which there are 1 + j where a sum is brought j times to a larger m, 10 for
// the chains. Measured: 2e-7 at most over rows of 1000 to 260000, 1e-8 in the mean.
//
// Bound by reading the logits: 512 rows of 131072 in bfloat16 (134 MB), 16 of 8 beams:
// 27 us for the parts, 5.0 TB/s, and 5 for the join; 496 of 50001 in float32, 32 of 16
// beams: 22 and 6.5. Few rows are bound by two launches and a chain of loads each: 4
// rows of 32000 7 and 5 us.
#include <algorithm>

#include "internal.hpp"

namespace lt {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;  // of a part's block, where rows are long
constexpr int kLoads = 4;              // 16-byte loads of a lane in a tile
constexpr int kList = 256;             // candidates that a wave keeps, where there are very many
constexpr float kLowest = -3.402823466e38f;
constexpr uint32_t kNinfKey = 0x007FFFFFu;  // ord_key(-inf): values above it are candidates

__device__ __forceinline__ float ninf() { return -__builtin_inff(); }

template <class T>
struct Row;
template <>
struct Row<uint16_t> {
  static constexpr int N = 8;
  __device__ static __forceinline__ float one(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  __device__ static __forceinline__ void unpack(const uint4& a, float (&x)[8]) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};
template <>
struct Row<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ float one(const float* p) { return *p; }
  __device__ static __forceinline__ void unpack(const uint4& a, float (&x)[4]) {
    x[0] = __uint_as_float(a.x), x[1] = __uint_as_float(a.y);
    x[2] = __uint_as_float(a.z), x[3] = __uint_as_float(a.w);
  }
};

// First element of a lane's load k of the tile at `base`: the loads of a row's end are
// moved down to end there, and hold elements that other loads have too.
template <class T>
__device__ __forceinline__ int place_of(int base, int k, int e) {
  return min(base + (k * 64 + (int)(threadIdx.x & 63)) * Row<T>::N, e - Row<T>::N);
}
// A tile of a row of at least N elements (at the elements' alignment).
template <class T>
__device__ __forceinline__ void fetch_tile(const T* x, int base, int e, uint4 (&raw)[kLoads]) {
#pragma unroll
  for (int k = 0; k < kLoads; ++k) __builtin_memcpy(&raw[k], x + place_of<T>(base, k, e), 16);
}
// The tile's values; those that other loads have, or that lie past the end, as -inf.
template <class T>
__device__ __forceinline__ void unpack_tile(const uint4 (&raw)[kLoads], int base, int e, float (&v)[kLoads][Row<T>::N]) {
  constexpr int N = Row<T>::N;
#pragma unroll
  for (int k = 0; k < kLoads; ++k) Row<T>::unpack(raw[k], v[k]);
  if (base + 64 * N * kLoads <= e) return;
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    const int moved = base + (k * 64 + (int)(threadIdx.x & 63)) * N - place_of<T>(base, k, e);
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < moved) v[k][j] = ninf();
  }
}

// scale log2 e = hi + lo. hi is cut, lo > 0, so that -inf stays -inf.
struct Scale {
  float hi, lo;
};
__device__ __forceinline__ Scale scale_of(double scale) {
  const double s = scale * 1.44269504088896340736;
  const float near = (float)s, hi = (double)near > s ? __uint_as_float(__float_as_uint(near) - 1u) : near;
  return Scale{hi, fmaxf((float)(s - (double)hi), 1.17549435e-38f)};
}
__device__ __forceinline__ float power(float t, Scale c) {  // 2^(t scale log2 e), t <= 0
  return __builtin_amdgcn_exp2f(fmaf(t, c.hi, t * c.lo));
}

__device__ __forceinline__ float key_float(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

__device__ __forceinline__ uint64_t shfl64_xor(uint64_t v, int o) {
  return (uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), o) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)v, o);
}

// The parts of a request's rows: blocks are shared out among the beams that are alive
// (up to 64 beams; of more, every beam has its own).
struct Shares {
  uint64_t alive;
  int beams, splits;  // rows that are read, parts of each
  bool all;
};
__device__ __forceinline__ Shares shares_of(const BeamArgs& a, const float* cums) {
  Shares s{0, a.beams, a.splits, a.beams > 64};
  if (s.all) return s;
  const int lane = threadIdx.x & 63;
  s.alive = __ballot(lane < a.beams && cums[min(lane, a.beams - 1)] > ninf());
  s.beams = __popcll(s.alive);
  s.splits = s.beams ? min(a.beams * a.splits / s.beams, a.most) : 1;
  return s;
}
// The beam of row i.
__device__ __forceinline__ int beam_of(const Shares& s, int i) {
  if (s.all) return i;
  const int lane = threadIdx.x & 63;
  const uint64_t at = __ballot(((s.alive >> lane) & 1) && __popcll(s.alive & ((1ull << lane) - 1)) == i);
  return __ffsll((unsigned long long)at) - 1;
}
// Elements of a part but the last: whole tiles of each wave.
__device__ __forceinline__ int part_len(const BeamArgs& a, const Shares& s, int tile) {
  return (a.most + s.splits - 1) / s.splits * tile;
}

// What a wave leaves of its part of a row: sum of 2^((x - m) scale log2 e), and m.
struct Sum {
  double s;
  float m;
  float pad;
};
struct Part {
  Sum* sums;       // [rows * splits][waves]
  uint64_t* keys;  // [rows * splits][top], best first; 0: no candidate
};

// Of a block's values (VALUES in LDS; every wave looks at all of them) the n-th
// largest, cut to its upper 16 bits: at least n of them reach it.
template <int VALUES>
__device__ __forceinline__ uint32_t block_floor(const uint32_t* values, int n) {
  constexpr int kEach = VALUES / 64;
  uint32_t p[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) p[i] = values[i * 64 + (threadIdx.x & 63)];
  uint32_t t = 0;
#pragma unroll 4
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t c = t | 1u << bit;
    int reach = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) reach += __popcll(__ballot(p[i] >= c));
    if (reach >= n) t = c;
  }
  return t;
}

// Orders a wave's own LDS traffic across its lanes.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- parts where more values than usual reach the cut (equal ones, mostly; float32
// logits that lie far from 0 together, whose upper 16 bits tell them hardly apart: 256
// rows of 260000 take 64 us at a common offset of 1000, 59 without) ----
// A wave's candidates in LDS. Of values that come later, those above `strict` can still
// be among the best n (the list holds n that reach it and come before).
struct List {
  uint64_t* at;
  int count;  // uniform in the wave
  uint32_t strict;
};
// Leaves the best n.
__device__ __forceinline__ void cut(List& l, int n) {
  if (l.count <= n) return;
  const int lane = threadIdx.x & 63;
  wave_sync();
  uint64_t k[kList / 64];
#pragma unroll
  for (int i = 0; i < kList / 64; ++i) k[i] = i * 64 + lane < l.count ? l.at[i * 64 + lane] : 0;
  uint64_t t = 0;  // the n-th largest: keys differ, so n of them reach it
  for (int bit = 63; bit >= 0; --bit) {
    const uint64_t c = t | 1ull << bit;
    int reach = 0;
#pragma unroll
    for (int i = 0; i < kList / 64; ++i) reach += __popcll(__ballot(k[i] >= c));
    if (reach >= n) t = c;
    if (reach == n) break;
  }
  int at = 0;
#pragma unroll
  for (int i = 0; i < kList / 64; ++i) {
    const bool in = k[i] != 0 && k[i] >= t;
    const uint64_t who = __ballot(in);
    if (in) l.at[at + __popcll(who & ((1ull << lane) - 1))] = k[i];
    at += __popcll(who);
  }
  l.count = at;
  l.strict = max(l.strict, (uint32_t)(t >> 32));  // (t's upper half: a value that n reach)
  wave_sync();
}

// The best n of a wave's tiles among the values from `loose` on: register by register,
// cut where the list runs full.
template <class T, int WAVES>
__device__ __forceinline__ void take_all(List& list, const T* x, int base, int e, int n, uint32_t loose) {
  constexpr int N = Row<T>::N, kTile = 64 * N * kLoads;
  const int lane = threadIdx.x & 63;
  for (; base < e; base += WAVES * kTile) {
    uint32_t gate = max(list.strict + 1, loose);
    uint4 raw[kLoads];
    fetch_tile<T>(x, base, e, raw);
    float v[kLoads][N], top = ninf();
    unpack_tile<T>(raw, base, e, v);
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) top = fmaxf(top, v[k][j]);
    if (!__any(ord_key(top) >= gate)) continue;
#pragma unroll 1
    for (int q = 0; q < kLoads * N; ++q) {
      const int from = base + (q / N * 64 + lane) * N, i = min(from, e - N) + q % N;
      const float u = i >= from ? Row<T>::one(x + i) : ninf();
      uint64_t who = __ballot(u >= key_float(gate));
      if (list.count + __popcll(who) > kList) {
        cut(list, n);
        // equal values of this tile may come before those in the list
        gate = max(gate, list.strict);
        who = __ballot(u >= key_float(gate));
      }
      if ((who >> lane) & 1) list.at[list.count + __popcll(who & ((1ull << lane) - 1))] = comp_key(u, (uint32_t)i);
      list.count += __popcll(who);
    }
    cut(list, n);
  }
  cut(list, n);
}

// A part of a row: the block's four waves take its tiles in turn. A lane keeps the
// largest value of each of its chunks (kSlots of them, one tile each or more): the
// pass over the logits does nothing else for the selection. Then the n-th largest of
// the threads' own largest is a value that the best n reach, hardly more chunks than n
// hold one as large, and those are read again. (Keeping lists of candidates along the
// way took 37 to 42 us where this takes 27: 512 rows of 131072 in bfloat16.)
constexpr int kSlots = 8;
constexpr int kChunks = 256;   // chunks that are read again
template <class T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_beam_part(BeamArgs a, Part part) {
  constexpr int kThreads = 64 * WAVES, kFound = 256 * WAVES;  // values that are ranked
  constexpr int N = Row<T>::N, kTile = 64 * N * kLoads;
  // the lanes' largest values by chunk, or the lists of the waves
  __shared__ union {
    uint32_t best[kSlots][kThreads];
    uint64_t lists[WAVES][kList];
  } lds;
  __shared__ __align__(16) uint32_t tops[kThreads];
  __shared__ uint64_t found[kFound];
  __shared__ uint16_t chunks[kChunks];
  __shared__ int chunk_count, found_count, counts[WAVES];
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
  const int parts = a.beams * a.splits, req = blockIdx.x / parts, p = blockIdx.x - req * parts, n = a.top;
  const float* cums = a.cum + (int64_t)req * a.beams;
  const Shares share = shares_of(a, cums);
  const int i = p / share.splits, split = p - i * share.splits;
  if (i >= share.beams) return;
  const int w = beam_of(share, i), len = part_len(a, share, WAVES * kTile);
  if (share.all && !(cums[w] > ninf())) return;
  const T* x = reinterpret_cast<const T*>(a.logits) + ((int64_t)req * a.beams + w) * a.ld;
  const int b = min(split * len, a.vocab), e = min(a.vocab - b, len) + b;
  uint4 raw[kLoads] = {};
  if (b + wave * kTile < e && e >= N) fetch_tile<T>(x, b + wave * kTile, e, raw);
  const Scale c = scale_of(a.scale);
  const int per_chunk = (len / (WAVES * kTile) + kSlots - 1) / kSlots;  // tiles of a chunk
  if (t == 0) chunk_count = found_count = 0;
#pragma unroll
  for (int k = 0; k < kSlots; ++k) lds.best[k][t] = kNinfKey;
  float m = kLowest, chunk = ninf(), most = ninf();
  double s = 0.0;
  int slot = 0, left = per_chunk;
  for (int base = b + wave * kTile; base < e; base += WAVES * kTile) {
    float v[kLoads][N], top = ninf();
    unpack_tile<T>(raw, base, e, v);
    if (e < N) {  // a row shorter than a load: an element a lane
#pragma unroll
      for (int q = 0; q < kLoads * N; ++q) v[q / N][q % N] = ninf();
      if (lane < e) v[0][0] = Row<T>::one(x + lane);
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) top = fmaxf(top, v[k][j]);
    const int next = base + WAVES * kTile;
    if (next < e) fetch_tile<T>(x, next, e, raw);
    if (top > m) {
      s *= (double)power(m - top, c);
      m = top;
    }
    float ss[4] = {};
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) ss[j & 3] += power(v[k][j] - m, c);
    s += (double)((ss[0] + ss[1]) + (ss[2] + ss[3]));
    chunk = fmaxf(chunk, top);
    most = fmaxf(most, top);
    lds.best[slot][t] = ord_key(chunk);
    if (--left == 0) {
      ++slot;
      left = per_chunk;
      chunk = ninf();
    }
  }
  tops[t] = ord_key(most);
  // the wave's sums
  float wm = m;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) wm = fmaxf(wm, __shfl_xor(wm, o));
  s *= (double)power(m - wm, c);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
  if (lane == 0) part.sums[(int64_t)blockIdx.x * WAVES + wave] = Sum{s, wm, 0.0f};
  __syncthreads();
  const uint32_t floor = max(block_floor<kThreads>(tops, n), kNinfKey + 1);
#pragma unroll
  for (int k = 0; k < kSlots; ++k)
    if (lds.best[k][t] >= floor) {
      const int at = atomicAdd(&chunk_count, 1);
      if (at < kChunks) chunks[at] = (uint16_t)(k * kThreads + t);
    }
  __syncthreads();
  bool many = chunk_count > kChunks;
  if (!many) {
    // the chunks' loads, one a thread at a time
    const int per = per_chunk * kLoads, items = chunk_count * per;
    const float g = key_float(floor);
    for (int q = t; q < items; q += kThreads) {
      const int ch = q / per, load = q - ch * per, who = chunks[ch] % kThreads;
      const int tile = chunks[ch] / kThreads * per_chunk + load / kLoads, k = load % kLoads;
      const int base = b + (tile * WAVES + (who >> 6)) * kTile, from = base + (k * 64 + (who & 63)) * N;
      if (e < N) {
        const int at = who & 63;
        if (k == 0 && at < e && Row<T>::one(x + at) >= g)
          found[atomicAdd(&found_count, 1)] = comp_key(Row<T>::one(x + at), (uint32_t)at);
        continue;
      }
      if (from >= e) continue;
      const int place = min(from, e - N);
      uint4 r;
      __builtin_memcpy(&r, x + place, 16);
      float v[N];
      Row<T>::unpack(r, v);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (v[j] >= g && place + j >= from) {
          const int at = atomicAdd(&found_count, 1);
          if (at < kFound) found[at] = comp_key(v[j], (uint32_t)(place + j));
        }
    }
    __syncthreads();
    many = found_count > kFound;
  }
  uint64_t* out = part.keys + (int64_t)blockIdx.x * n;
  if (!many) {
    // each counts how many come before it
    const int total = found_count;
    for (int q = t; q < total; q += kThreads) {
      const uint64_t mine = found[q];
      int before = 0;
#pragma unroll 4
      for (int o = 0; o < total; ++o) before += found[o] > mine;
      if (before < n) out[before] = mine;
    }
    for (int q = total + t; q < n; q += kThreads) out[q] = 0;
    return;
  }
  __syncthreads();
  List list{lds.lists[wave], 0, kNinfKey};
  take_all<T, WAVES>(list, x, b + wave * kTile, e, n, floor);
  if (lane == 0) counts[wave] = list.count;
  __syncthreads();
  int total = 0, at = t, from = 0;
  for (int q = 0; q < WAVES; ++q) total += counts[q];
  while (from < WAVES - 1 && at >= counts[from]) at -= counts[from++];
  const uint64_t mine = t < total ? lds.lists[from][at] : 0;
  int before = 0;
  for (from = 0; from < WAVES; ++from)
    for (at = 0; at < counts[from]; ++at) before += lds.lists[from][at] > mine;
  if (mine && before < n) out[before] = mine;
  if (t >= total && t < n) out[t] = 0;
}

// ---- join: a block a request ----
struct Candidate {
  uint64_t rank;   // score (ord_key), then the lower row; 0: none
  uint64_t key;    // logit, then the lower token
};
__device__ __forceinline__ bool comes_before(const Candidate& a, const Candidate& b) {
  return a.rank != b.rank ? a.rank > b.rank : a.key > b.key;
}

constexpr int kMost = 512;     // candidates that are ranked together (more than any `top`)
constexpr int kHeld = 8;       // keys that a thread holds in registers

__global__ __launch_bounds__(kThreads) void k_beam_join(BeamArgs a, Part part, int lanes_log2) {
  extern __shared__ double logs[];            // [beams]: of the rows that were read log s,
  float* tip = reinterpret_cast<float*>(logs + a.beams);  // m,
  float* cum = tip + a.beams;                             // their beams' scores
  int* beam = reinterpret_cast<int*>(cum + a.beams);      // and the beams
  __shared__ Candidate found[kMost];
  __shared__ __align__(16) uint32_t tops[kThreads];
  __shared__ int count;
  __shared__ Candidate pick[kWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, n = a.top, req = blockIdx.x;
  const Scale c = scale_of(a.scale);
  const float* cums = a.cum + (int64_t)req * a.beams;
  const Shares share = shares_of(a, cums);
  const int per = share.splits * n, total = share.beams * per;  // keys of a row, of the request
  const uint64_t* keys = part.keys + (int64_t)req * a.beams * a.splits * n;
  // A thread's r-th key. The keys of a part are sorted: a thread that took every
  // kThreads-th one would have the same place in all parts, and few threads all that count.
  auto place_of_key = [&](int r) { return r * kThreads + ((t + 29 * r) & (kThreads - 1)); };
  const int rounds = (total + kThreads - 1) / kThreads;
  const bool held = rounds <= kHeld;
  uint64_t mine[kHeld];
  if (held) {
#pragma unroll
    for (int r = 0; r < kHeld; ++r) mine[r] = place_of_key(r) < total ? keys[place_of_key(r)] : 0;
  }
  if (t == 0) count = 0;
  if (share.all) {
    for (int i = t; i < a.beams; i += kThreads) beam[i] = i;
  } else if (wave == 0 && ((share.alive >> lane) & 1)) {
    beam[__popcll(share.alive & ((1ull << lane) - 1))] = lane;
  }
  __syncthreads();
  // log sums: 1 << lanes_log2 lanes a beam
  const int S = 1 << lanes_log2, sub = t & (S - 1);
  for (int w0 = 0; w0 < share.beams; w0 += kThreads >> lanes_log2) {
    const int w = w0 + (t >> lanes_log2);
    const Sum* sums = part.sums + ((int64_t)req * a.beams * a.splits + w * share.splits) * a.waves;
    float m = kLowest;
    double s = 0.0;
    if (w < share.beams) {
      for (int i = sub; i < share.splits * a.waves; i += S) {  // (of a beam that is not alive: anything)
        const Sum p = sums[i];
        const float hi = fmaxf(m, p.m);
        s = s * (double)power(m - hi, c) + p.s * (double)power(p.m - hi, c);
        m = hi;
      }
    }
    for (int o = 1; o < S; o <<= 1) {
      const float om = __shfl_xor(m, o), hi = fmaxf(m, om);
      const double os = __shfl_xor(s, o);
      s = s * (double)power(m - hi, c) + os * (double)power(om - hi, c);
      m = hi;
    }
    if (w < share.beams && sub == 0) {
      const float f = cums[beam[w]];
      logs[w] = f > ninf() ? log(s) : (double)__builtin_nanf("");
      tip[w] = m;
      cum[w] = f;
    }
  }
  __syncthreads();
  auto rank_of = [&](int i, uint64_t key) {
    if (!key) return 0ull;
    const int w = (uint32_t)i / (uint32_t)per;
    const double below = (double)key_float((uint32_t)(key >> 32)) - (double)tip[w];
    const float score = (float)((double)cum[w] + (below * a.scale - logs[w]));
    return score > ninf() ? (unsigned long long)ord_key(score) << 32 | (0xFFFFFFFFu - (uint32_t)w) : 0ull;
  };
  // f(rank, key) of each of the thread's keys
  auto each = [&](auto f) {
    for (int r = 0; r < rounds; ++r) {
      const int i = place_of_key(r);
      const uint64_t key = i < total ? keys[i] : 0;
      f(rank_of(i, key), key);
    }
  };
  // a score that n of the threads' own best reach (cut to its upper half)
  uint32_t best = 0;
  uint64_t rank[kHeld];
  if (held) {
#pragma unroll
    for (int r = 0; r < kHeld; ++r) {
      rank[r] = rank_of(place_of_key(r), mine[r]);
      best = max(best, (uint32_t)(rank[r] >> 32));
    }
  } else {
    each([&](uint64_t k, uint64_t) { best = max(best, (uint32_t)(k >> 32)); });
  }
  tops[t] = best;
  __syncthreads();
  const uint64_t floor = (uint64_t)max(block_floor<kThreads>(tops, n), 1u) << 32;
  auto keep = [&](uint64_t k, uint64_t key) {
    if (k < floor) return;
    const int at = atomicAdd(&count, 1);
    if (at < kMost) found[at] = Candidate{k, key};
  };
  if (held) {
#pragma unroll
    for (int r = 0; r < kHeld; ++r) keep(rank[r], mine[r]);
  } else {
    each(keep);
  }
  __syncthreads();
  const int have = count;
  auto put = [&](int place, const Candidate& k) {
    const int64_t o = (int64_t)req * n + place;
    a.out_score[o] = k.rank ? key_float((uint32_t)(k.rank >> 32)) : ninf();
    a.out_beam[o] = k.rank ? beam[0xFFFFFFFFu - (uint32_t)k.rank] : -1;
    a.out_token[o] = k.rank ? (int)comp_pos(k.key) : -1;
  };
  if (have <= kMost) {
    for (int i = t; i < have; i += kThreads) {
      const Candidate k = found[i];
      int before = 0;
#pragma unroll 4
      for (int j = 0; j < have; ++j) before += comes_before(found[j], k);
      if (before < n) put(before, k);
    }
    for (int i = have + t; i < n; i += kThreads) put(i, Candidate{0, 0});
    return;
  }
  // More than kMost reach the cut: equal scores, or different ones far from 0, where the
  // upper 16 bits of float32 are 4 apart from 512 on (1/8 at 20). One after the other, at
  // least n of them: 2 requests of 32 beams of 131072 logits, best 64, take 36 us with
  // scores from -20 to -300 and 269 from -600 on; one of 16 beams, best 32, 21 to 23 and 139.
  Candidate last{~0ull, ~0ull};
  for (int place = 0; place < n; ++place) {
    Candidate k{0, 0};
    each([&](uint64_t r, uint64_t key) {
      const Candidate v{r, key};
      if (r && comes_before(last, v) && comes_before(v, k)) k = v;
    });
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const Candidate v{shfl64_xor(k.rank, o), shfl64_xor(k.key, o)};
      if (comes_before(v, k)) k = v;
    }
    if (lane == 0) pick[wave] = k;
    __syncthreads();
    k = pick[0];
    for (int i = 1; i < kWaves; ++i)
      if (comes_before(pick[i], k)) k = pick[i];
    __syncthreads();
    if (t == 0) put(place, k);
    last = k;
  }
}

int wave_tile(const BeamArgs& a) { return 64 * kLoads * (a.bf16 ? 8 : 4); }

}  // namespace

// Parts of all rows, where they are long enough: two blocks a CU. More of them cost more
// in ends and in joins than they save: 176 rows of 75842 take 21 us with 512, 26 with
// 1024; 512 of 131072 34 and 36.
constexpr int64_t kParts = 512;
// Keys of a request's parts: what a join holds in registers. 16 rows of 260000, best 32 of
// 16 beams: 21 us; 25 with 8192 keys and blocks of 1024 threads that hold them.
constexpr int64_t kMostKeys = kHeld * kThreads;
constexpr int64_t kNarrowRows = 2048;

// Parts of a row: enough blocks to fill the GPU, none shorter than a tile for each wave,
// and no more keys of a request than its join's block holds. Rows of one tile take a
// wave, and so do short ones of which there are many: 8192 rows of 1000 take 26 us, 51 with
// four waves a row; 2048 of 4000 17 and 21; 512 of 4000 16 either way.
void beam_shape(BeamArgs& a) {
  const int64_t rows = (int64_t)a.batch * a.beams;
  const int64_t tiles = (a.vocab + (int64_t)wave_tile(a) - 1) / wave_tile(a);
  a.waves = a.top <= 32 && (tiles <= 1 || (tiles <= 4 && rows >= kNarrowRows)) ? 1 : kWaves;
  a.most = (int)std::max<int64_t>(1, (tiles + a.waves - 1) / a.waves);
  const int64_t keys = std::max<int64_t>(1, kMostKeys / ((int64_t)a.beams * a.top));
  a.splits = (int)std::min({(int64_t)a.most, std::max<int64_t>(1, kParts / std::max<int64_t>(rows, 1)), keys});
}

static size_t sums_bytes(int64_t parts) { return ((size_t)parts * kWaves * sizeof(Sum) + 255) / 256 * 256; }

// Splits follow from rows and vocabulary, but a call of fewer rows or entries may take
// more of them: sized for the most parts that any call within these sizes takes.
size_t beam_workspace_bytes(const BeamArgs& a) {
  const int64_t rows = (int64_t)a.batch * a.beams;
  const int64_t most = std::max<int64_t>(1, (a.vocab + (int64_t)wave_tile(a) - 1) / wave_tile(a));
  // rows * splits <= max(rows, kParts), and never more than rows * most
  const int64_t parts = std::max(rows, std::min<int64_t>(rows * most, kParts));
  return sums_bytes(parts) + (size_t)parts * a.top * sizeof(uint64_t) + 256;
}

hipError_t launch_beam_select(BeamArgs a, void* workspace, hipStream_t st) {
  beam_shape(a);
  const int64_t parts = (int64_t)a.batch * a.beams * a.splits;
  Part part;
  part.sums = static_cast<Sum*>(workspace);
  part.keys = reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(workspace) + sums_bytes(parts));
  const dim3 all((unsigned)parts);
  if (a.bf16 && a.waves == 1) k_beam_part<uint16_t, 1><<<all, 64, 0, st>>>(a, part);
  else if (a.bf16) k_beam_part<uint16_t, kWaves><<<all, kThreads, 0, st>>>(a, part);
  else if (a.waves == 1) k_beam_part<float, 1><<<all, 64, 0, st>>>(a, part);
  else k_beam_part<float, kWaves><<<all, kThreads, 0, st>>>(a, part);
  int lanes_log2 = 0;
  while (lanes_log2 < 6 && 1 << lanes_log2 < a.splits * a.waves) ++lanes_log2;
  k_beam_join<<<dim3((unsigned)a.batch), kThreads, (size_t)a.beams * 20, st>>>(a, part, lanes_log2);
  return hipGetLastError();
}

}  // namespace lt
