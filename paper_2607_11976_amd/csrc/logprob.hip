// Log probabilities of given tokens, entropy and best alternatives of rows of
// logits, and the logits' gradient.
//
//   y_i = scale * x_i,  lse = log sum exp(y_i),  lp = y_tok - lse,
//   H = lse - sum p_i y_i,  p_i = exp(y_i - lse)
//   dx_i = scale * (g_lp * (1[i = tok] - p_i) - g_H * p_i * (log p_i + H))
//
// Forward reads the logits once. With a running reference logit m, in powers of
// two (t = (x - m) scale log2 e), a thread sums s = sum 2^t and u = sum t 2^t in
// float32: lse = scale m + log2 s ln 2, lp = scale (x_tok - m) - log2 s ln 2 and
// H = (log2 s - u / s) ln 2, none with a large difference; logits at their type's
// lowest value are values like any other. The best `top` entries are kept by each
// wave, sorted over its lanes (one 64-bit key a lane: value, then the lower
// index), behind a threshold that the waves of a block share. Bound by reading the
// logits where few are asked for: 2039 rows of 128001 in bfloat16 (0.52 GB) take 126 us
// without, 134 with the best one, 4.2 and 3.9 TB/s, in float32 189 and 194, 5.5 and
// 5.4; more loads a thread or more blocks a CU lose. More of the best are inserted one
// by one before the threshold holds: with 5, 20 and 64 145, 194 and 351 us in bfloat16,
// 198, 230 and 341 in float32.
//
// The entropy is a difference of two sums of up to kSlack, and where one entry holds
// nearly all weight, of a sum near 1 and its rounding: its error, like the log
// probabilities', is absolute, up to 1e-6 in rows of every kind tried, not relative.
#include <algorithm>

#include "internal.hpp"

namespace lt {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kUnroll = 4;            // 16-byte loads a thread has in flight
constexpr float kSlack = 8.0f;        // log2 by which a value may pass the reference
constexpr float kStart = -3.402823466e38f;  // reference before the first value: the lowest there is
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float ninf() { return -__builtin_inff(); }

template <class T>
struct Vec;
template <>
struct Vec<uint16_t> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void unpack(const uint4& a, float (&x)[8]) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  __device__ static __forceinline__ float one(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static constexpr uint32_t kFill = 0xFF80FF80u;  // -inf
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void unpack(const uint4& a, float (&x)[4]) {
    x[0] = __uint_as_float(a.x), x[1] = __uint_as_float(a.y);
    x[2] = __uint_as_float(a.z), x[3] = __uint_as_float(a.w);
  }
  __device__ static __forceinline__ float one(const float* p) { return *p; }
  static constexpr uint32_t kFill = 0xFF800000u;
};

// 16 bytes of a row at its elements' alignment (rows need no other).
template <class T>
__device__ __forceinline__ uint4 load16(const T* p) {
  uint4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}

// The same of elements [i, i + N), those from e on as -inf.
template <class T>
__device__ __forceinline__ uint4 fetch16(const T* x, int i, int e) {
  constexpr int N = Vec<T>::N;
  if (i + N <= e) return load16(x + i);
  uint32_t w[4] = {Vec<T>::kFill, Vec<T>::kFill, Vec<T>::kFill, Vec<T>::kFill};
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (i + j >= e) continue;
    if constexpr (N == 8) {
      const uint32_t h = x[i + j];
      w[j >> 1] = j & 1 ? (w[j >> 1] & 0xFFFFu) | (h << 16) : (w[j >> 1] & 0xFFFF0000u) | h;
    } else {
      w[j] = __float_as_uint(x[i + j]);
    }
  }
  return uint4{w[0], w[1], w[2], w[3]};
}

// ---- sums ----
struct Sums {
  float m, s, u;
};
__device__ __forceinline__ void rebase(Sums& a, float m, float c) {
  const float d = (a.m - m) * c, f = __builtin_amdgcn_exp2f(d);
  a.u = f * fmaf(a.s, fmaxf(d, -1.0e4f), a.u);  // f is 0 long before that
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ Sums join(Sums a, Sums b, float c) {
  const float m = fmaxf(a.m, b.m);
  rebase(a, m, c);
  rebase(b, m, c);
  return Sums{m, a.s + b.s, a.u + b.u};
}
__device__ __forceinline__ Sums wave_join(Sums a, float c) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) a = join(a, Sums{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.u, o)}, c);
  return a;
}

// ---- the best entries ----
__device__ __forceinline__ uint64_t shfl64(uint64_t v, int lane) {
  return ((uint64_t)(uint32_t)__shfl((int)(v >> 32), lane) << 32) | (uint32_t)__shfl((int)(uint32_t)v, lane);
}
__device__ __forceinline__ uint64_t shfl64_xor(uint64_t v, int o) {
  return ((uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), o) << 32) | (uint32_t)__shfl_xor((int)(uint32_t)v, o);
}
// A list of 64 keys over the lanes, descending; 0 = no entry (below every key:
// a key's low word is never 0).
// Entry i of the union's best 64 of two such lists.
__device__ __forceinline__ uint64_t merge_lists(uint64_t a, uint64_t b) {
  const int lane = threadIdx.x & 63;
  const uint64_t r = shfl64(b, 63 - lane);
  uint64_t v = a > r ? a : r;  // bitonic: the best 64 of both
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    const uint64_t w = shfl64_xor(v, o);
    v = ((lane & o) == 0) == (v > w) ? v : w;
  }
  return v;
}
// 64 unordered keys, descending.
__device__ __forceinline__ uint64_t sort_list(uint64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
    for (int o = k >> 1; o; o >>= 1) {
      const uint64_t w = shfl64_xor(v, o);
      const bool first = ((lane & o) == 0) == ((lane & k) == 0);  // takes the larger
      v = first == (v > w) ? v : w;
    }
  return v;
}
__device__ __forceinline__ void insert(uint64_t& list, uint64_t key) {  // key is wave-uniform
  const int lane = threadIdx.x & 63;
  const int at = __popcll(__ballot(list > key));
  const uint64_t up = shfl64(list, lane - 1);
  list = lane < at ? list : lane == at ? key : up;
}
__device__ __forceinline__ uint64_t read_lane64(uint64_t v, int lane) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
// The score of a key's value part; keys of NaN and "no entry" give -inf.
__device__ __forceinline__ float key_floor(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return o ? __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o) : ninf();
}

struct Best {
  uint64_t list, thr;  // thr: a key that top keys of the row are known to reach
  float floor;
  __device__ __forceinline__ void raise(uint64_t key) {
    if (key > thr) {
      thr = key;
      floor = key_floor(key);
    }
  }
};

template <class T>
__device__ __forceinline__ void take(Best& b, const float (&x)[Vec<T>::N], int first, int count, int top) {
#pragma unroll
  for (int j = 0; j < Vec<T>::N; ++j) {
    const uint64_t key = j < count && !(x[j] < b.floor) ? comp_key(x[j], (uint32_t)(first + j)) : 0u;
    uint64_t who = __ballot(key > b.thr);
    while (who) {
      const int lane = __ffsll((unsigned long long)who) - 1;
      who &= who - 1;
      const uint64_t k = read_lane64(key, lane);
      if (k <= b.thr) continue;
      insert(b.list, k);
      b.raise(read_lane64(b.list, top - 1));
    }
  }
}

// A row's token's logit, asked for early: two loads, one after the other.
struct Token {
  bool in;  // inside the vocabulary
  float x;
};
template <class T>
__device__ __forceinline__ Token token_of(const LogprobArgs& a, int row) {
  const int64_t tok = a.tokens[row];
  const bool in = tok >= 0 && tok < a.vocab;
  return Token{in, in ? Vec<T>::one(reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.ld + tok) : 0.0f};
}

// What a row's sums say of its token; one thread.
__device__ __forceinline__ void finish_row(const LogprobArgs& a, int row, const Sums& s, const Token& k) {
  const bool none = s.s == 0.0f;  // no value above -inf
  const float l2 = __builtin_amdgcn_logf(s.s);
  float lp = 0.0f;
  if (k.in) lp = none ? ninf() : fmaf(k.x - s.m, a.scale, -l2 * kLn2);
  a.logprob[row] = lp;
  a.entropy[row] = none ? 0.0f : (l2 - s.u / s.s) * kLn2;
  a.lse[row] = none ? ninf() : fmaf(s.m, a.scale, l2 * kLn2);
}
// The row's best entry number `place`; key 0: there is none.
__device__ __forceinline__ void finish_top(const LogprobArgs& a, int row, const Sums& s, int place, uint64_t key) {
  float lp = ninf();
  if (key && s.s != 0.0f) {
    // a NaN among the logits makes the sums NaN, whatever the key's value
    lp = fmaf(key_floor(key) - s.m, a.scale, -__builtin_amdgcn_logf(s.s) * kLn2);
  }
  a.top_index[(int64_t)row * a.top + place] = key ? (int)comp_pos(key) : -1;
  a.top_logprob[(int64_t)row * a.top + place] = lp;
}

// What a split of a row leaves: its sums, and keys among which its best `top`
// are (0: no entry).
constexpr int kList = 128;
struct Partial {
  Sums* sums;      // [rows * splits]
  uint64_t* keys;  // [rows * splits][kList]
};
__device__ __forceinline__ void put_list(uint64_t* out, uint64_t list) {  // one wave
  const int lane = threadIdx.x & 63;
  out[lane] = list;
  out[64 + lane] = 0;
}

template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_logprobs(LogprobArgs a, Partial part) {
  constexpr int N = Vec<T>::N;
  __shared__ Sums wsum[kWaves];
  __shared__ uint64_t wlist[kWaves][64];
  __shared__ unsigned long long shared_thr;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits;
  const T* x = reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.ld;
  const int b = split * a.split_len, e = min(a.vocab - b, a.split_len) + b;  // elements [b, e)
  const float c = a.scale * kLog2e, slack = fminf(kSlack / c, 1.0e30f);
  if constexpr (TOP) {
    if (t == 0) shared_thr = 0;
    __syncthreads();
  }

  Sums s{kStart, 0.0f, 0.0f};
  Best best{0, 0, ninf()};
  bool primed = false;
  auto fetch = [&](int base, uint4 (&v)[kUnroll]) {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) v[k] = fetch16<T>(x, base + (k * kThreads + t) * N, e);
  };
  constexpr int kStep = kThreads * kUnroll * N;
  uint4 nxt[kUnroll];
  fetch(b, nxt);
  for (int base = b; base < e; base += kStep) {
    float v[kUnroll][N], vmax[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      Vec<T>::unpack(nxt[k], v[k]);
      vmax[k] = v[k][0];
#pragma unroll
      for (int j = 1; j < N; ++j) vmax[k] = fmaxf(vmax[k], v[k][j]);
    }
    if (base + kStep < e) fetch(base + kStep, nxt);
    float top = fmaxf(fmaxf(vmax[0], vmax[1]), fmaxf(vmax[2], vmax[3]));
    if (__any(top > s.m + slack)) rebase(s, fmaxf(s.m, top), c);
    // four chains of sums
    float ss[4] = {}, uu[4] = {};
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float d = (v[k][j] - s.m) * c, p = __builtin_amdgcn_exp2f(d);
        ss[j & 3] += p;
        // 2^d is 0 long before -200; -inf must not meet it
        uu[j & 3] = fmaf(p, fmaxf(d, -200.0f), uu[j & 3]);
      }
    s.s += (ss[0] + ss[1]) + (ss[2] + ss[3]);
    s.u += (uu[0] + uu[1]) + (uu[2] + uu[3]);
    if constexpr (TOP) {
      if (!primed) {
        // the top-th largest of 64 lanes' own largest values bounds the row's
        primed = true;
        const int i0 = base + t * N;
        uint64_t mine = 0;
        if (i0 + N <= e) mine = comp_key(vmax[0], 0xFFFFFFFEu);  // below every entry of that value
        const uint64_t bound = read_lane64(sort_list(mine), a.top - 1);
        if (bound) best.raise(bound - 1);
      }
      best.raise(*(volatile unsigned long long*)&shared_thr);
      const uint64_t was = best.thr;
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int i = base + (k * kThreads + t) * N;
        if (__any(i < e && !(vmax[k] < best.floor))) take<T>(best, v[k], i, e - i, a.top);
      }
      if (best.thr > was && lane == 0) atomicMax(&shared_thr, (unsigned long long)best.thr);
    }
  }

  s = wave_join(s, c);
  if (lane == 0) wsum[wave] = s;
  if constexpr (TOP) wlist[wave][lane] = best.list;
  __syncthreads();
  if (wave) return;
  for (int i = 1; i < kWaves; ++i) {
    s = join(s, wsum[i], c);
    if constexpr (TOP) best.list = merge_lists(best.list, wlist[i][lane]);
  }
  if (a.splits == 1) {
    if (lane == 0) finish_row(a, row, s, token_of<T>(a, row));
    if (TOP && lane < a.top) finish_top(a, row, s, lane, best.list);
  } else {
    if (lane == 0) part.sums[blockIdx.x] = s;
    if (TOP) put_list(part.keys + (int64_t)blockIdx.x * kList, lane < a.top ? best.list : 0);
  }
}

// ---- few rows: latency ----
// 8 rows of 131072 in bfloat16 and their best 20: 12.2 us in a captured graph,
// parts and join (a launch alone takes 3.8). Sorted lists of every wave took 24.7.
// The largest value, cut to its upper 16 bits, that at least n of a block's
// threads reach. One barrier; mine: LDS of a word a thread.
__device__ __forceinline__ uint32_t nth_floor(uint32_t v, int n, uint32_t* mine) {
  mine[threadIdx.x] = v;
  __syncthreads();
  const uint4 w = reinterpret_cast<const uint4*>(mine)[threadIdx.x & 63];  // each wave looks at all of them
  uint32_t t = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t c = t | 1u << bit;
    const int reach = __popcll(__ballot(w.x >= c)) + __popcll(__ballot(w.y >= c)) + __popcll(__ballot(w.z >= c)) +
                      __popcll(__ballot(w.w >= c));
    if (reach >= n) t = c;
  }
  return t;
}

// A part of a row in registers, kHeld loads a thread. The block's best lie at or
// above a value that the largest entries of `top` threads reach: hardly more
// entries than that (21 for 20, 73 for 64 of 4096 normal values), which go out in
// any order. (More than kList: sorted lists as above.)
constexpr int kHeld = 2;
constexpr int64_t kMostParts = 2048;  // of all rows
template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_logprobs_part(LogprobArgs a, Partial part) {
  constexpr int N = Vec<T>::N;
  __shared__ Sums wsum[kWaves];
  __shared__ __align__(16) uint32_t tops[kThreads];
  __shared__ int count;
  __shared__ uint64_t wlist[kWaves][64];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits;
  const T* x = reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.ld;
  const int b = split * a.split_len, e = min(a.vocab - b, a.split_len) + b;
  const float c = a.scale * kLog2e;
  if (t == 0) count = 0;
  uint4 raw[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) raw[k] = fetch16<T>(x, b + (k * kThreads + t) * N, e);
  float v[kHeld][N], top = ninf();
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    Vec<T>::unpack(raw[k], v[k]);
#pragma unroll
    for (int j = 0; j < N; ++j) top = fmaxf(top, v[k][j]);
  }
  uint32_t o[kHeld][N], mine = 0;
  if constexpr (TOP) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        o[k][j] = b + (k * kThreads + t) * N + j < e ? ord_key(v[k][j]) : 0u;
        mine = max(mine, o[k][j]);
      }
  }
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
  Sums s{fmaxf(top, kStart), 0.0f, 0.0f};
  float ss[4] = {}, uu[4] = {};
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float d = (v[k][j] - s.m) * c, p = __builtin_amdgcn_exp2f(d);
      ss[j & 3] += p;
      uu[j & 3] = fmaf(p, fmaxf(d, -200.0f), uu[j & 3]);
    }
  s.s = (ss[0] + ss[1]) + (ss[2] + ss[3]);
  s.u = (uu[0] + uu[1]) + (uu[2] + uu[3]);
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    s.s += __shfl_xor(s.s, i);
    s.u += __shfl_xor(s.u, i);
  }
  if (lane == 0) wsum[wave] = s;
  uint32_t f = 0;
  if constexpr (TOP) f = nth_floor(mine, a.top, tops);
  else __syncthreads();
  if (t == 0) {
    for (int i = 1; i < kWaves; ++i) s = join(s, wsum[i], c);
    part.sums[blockIdx.x] = s;
  }
  if constexpr (TOP) {
    int n = 0;
    uint64_t who[kHeld][N];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        who[k][j] = __ballot(o[k][j] >= f && b + (k * kThreads + t) * N + j < e);
        n += __popcll(who[k][j]);
      }
    int at = 0;
    if (lane == 0) at = atomicAdd(&count, n);
    at = __builtin_amdgcn_readfirstlane(at);
    const uint64_t below = (1ull << lane) - 1;
    uint64_t* list = wlist[0];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int p = at + __popcll(who[k][j] & below);
        if (((who[k][j] >> lane) & 1u) && p < kList)
          list[p] = comp_key(v[k][j], (uint32_t)(b + (k * kThreads + t) * N + j));
        at += __popcll(who[k][j]);
      }
    __syncthreads();
    const int total = count;
    uint64_t* out = part.keys + (int64_t)blockIdx.x * kList;
    if (total <= kList) {
      if (t < kList) out[t] = t < total ? list[t] : 0;
      return;
    }
    __syncthreads();  // (wlist is read by no one any more)
    Best best{0, 0, ninf()};
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      const int i = b + (k * kThreads + t) * N;
      take<T>(best, v[k], i, e - i, a.top);
    }
    wlist[wave][lane] = best.list;
    __syncthreads();
    if (wave) return;
    for (int i = 1; i < kWaves; ++i) best.list = merge_lists(best.list, wlist[i][lane]);
    put_list(out, lane < a.top ? best.list : 0);
  }
}

// Joins a row's splits: a block a row. The best entries lie at or above a value
// that `top` threads' own reach; of those, each counts how many come before it.
template <class T>
__global__ __launch_bounds__(kThreads) void k_logprobs_join(LogprobArgs a, Partial part) {
  constexpr int kMost = 512, kKept = 16;
  __shared__ Sums wsum[kWaves];
  __shared__ __align__(16) uint32_t tops[kThreads];
  __shared__ int count;
  __shared__ uint64_t wlist[kMost];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, row = blockIdx.x;
  const float c = a.scale * kLog2e;
  const uint64_t* keys = part.keys + (int64_t)row * a.splits * kList;
  const int slots = a.top > 0 ? a.splits * kList : 0;
  if (t == 0) count = 0;
  const Token token = token_of<T>(a, row);
  // the first keys stay in registers, loaded together; more are read twice
  uint64_t held[kKept];
#pragma unroll
  for (int u = 0; u < kKept; ++u) held[u] = u * kThreads + t < slots ? keys[u * kThreads + t] : 0;
  uint32_t mine = 0;
#pragma unroll 8
  for (int i = kKept * kThreads + t; i < slots; i += kThreads) mine = max(mine, (uint32_t)(keys[i] >> 32));
#pragma unroll
  for (int u = 0; u < kKept; ++u) mine = max(mine, (uint32_t)(held[u] >> 32));
  Sums s{kStart, 0.0f, 0.0f};
  for (int i = t; i < a.splits; i += kThreads) s = join(s, part.sums[(int64_t)row * a.splits + i], c);
  s = wave_join(s, c);
  if (lane == 0) wsum[wave] = s;
  const uint32_t f = nth_floor(mine, a.top, tops);
  s = wsum[0];
  for (int i = 1; i < kWaves; ++i) s = join(s, wsum[i], c);
  if (t == 0) finish_row(a, row, s, token);
  if (a.top == 0) return;

  auto list = [&](uint64_t k) {
    const uint64_t who = __ballot(k != 0 && (uint32_t)(k >> 32) >= f);
    if (!who) return;
    int at = 0;
    if (lane == 0) at = atomicAdd(&count, __popcll(who));
    at = __builtin_amdgcn_readfirstlane(at) + __popcll(who & ((1ull << lane) - 1));
    if (((who >> lane) & 1u) && at < kMost) wlist[at] = k;
  };
#pragma unroll
  for (int u = 0; u < kKept; ++u) list(held[u]);
  for (int i = kKept * kThreads + t; i < slots; i += kThreads) list(keys[i]);  // whole waves: a multiple of 64
  __syncthreads();
  const int total = count;
  if (total <= kMost) {
    for (int i = t; i < total; i += kThreads) {
      const uint64_t k = wlist[i];
      int before = 0;
      for (int j = 0; j < total; ++j) before += wlist[j] > k ? 1 : 0;
      if (before < a.top) finish_top(a, row, s, before, k);
    }
    if (t >= total && t < a.top) finish_top(a, row, s, t, 0);
    return;
  }
  // many equal values: sorted lists
  __syncthreads();
  uint64_t best = 0;
  for (int i = wave; i < slots / 64; i += kWaves) best = merge_lists(best, sort_list(keys[i * 64 + lane]));
  wlist[wave * 64 + lane] = best;
  __syncthreads();
  if (wave) return;
  for (int i = 1; i < kWaves; ++i) best = merge_lists(best, wlist[i * 64 + lane]);
  if (lane < a.top) finish_top(a, row, s, lane, best);
}

// ---- gradient: one pass, bound by reading and writing the logits once ----
// 2039 rows of 128001 in bfloat16 (1.04 GB) take 183 us on one card and 210 on another,
// 5.7 and 5.0 TB/s; on the latter rows of a large lse (below), which are read twice,
// take 294, and in float32 413 and 578.
// p = w 2^((x - from) scale log2 e - minus log2 e), with from = 0, minus = lse and w = 1
// where lse is near 0: half its last bit is then an error of at most 2^-21, common to
// the row's p, as large as the exponential's own. That doubles with every power of two
// of lse, though a softmax does not depend on a common offset. Rows of a larger lse
// (kFarLse and beyond; -inf too, which may be a finite sum below float32's range) are
// summed again, by one block that then writes the whole row: from = a logit near the
// largest, minus = 0, w = 1 / sum.
constexpr float kFarLse = 16.0f;

template <class T, int THREADS>
__global__ __launch_bounds__(THREADS, 2048 / THREADS) void k_logprobs_backward(
    const T* logits, int64_t ld, int vocab, const int64_t* tokens, float scale, const float* lse, const float* entropy,
    const float* g_lp, const float* g_ent, T* out, int64_t out_ld) {
  constexpr int N = Vec<T>::N, kSpan = THREADS * N;
  const int row = blockIdx.x, t = threadIdx.x;
  const T* x = logits + (int64_t)row * ld;
  T* o = out + (int64_t)row * out_ld;
  const int64_t tok = tokens[row];
  const bool counts = tok >= 0 && tok < vocab;
  const float z = lse[row];
  int first = blockIdx.y * kSpan + t * N, step = gridDim.y * kSpan;
  bool none = false;
  float from = 0.0f, minus = z, w = 1.0f;
  if (!(fabsf(z) < kFarLse)) {
    if (blockIdx.y) return;
    first = t * N;
    step = kSpan;
    __shared__ Sums wsum[THREADS / 64];
    const float c = scale * kLog2e, slack = fminf(kSlack / c, 1.0e30f);
    Sums s{kStart, 0.0f, 0.0f};
    // a wave stops at the row's end: its lanes' elements lie side by side
    for (int at = (t & ~63) * N; at < vocab; at += kUnroll * kSpan) {
      uint4 raw[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) raw[k] = fetch16<T>(x, at + k * kSpan + (t & 63) * N, vocab);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        if (at + k * kSpan >= vocab) break;
        float v[N], ss[2] = {};
        Vec<T>::unpack(raw[k], v);
        float top = v[0];
#pragma unroll
        for (int j = 1; j < N; ++j) top = fmaxf(top, v[j]);
        if (__any(top > s.m + slack)) rebase(s, fmaxf(s.m, top), c);
#pragma unroll
        for (int j = 0; j < N; ++j) ss[j & 1] += __builtin_amdgcn_exp2f((v[j] - s.m) * c);
        s.s += ss[0] + ss[1];
      }
    }
    s = wave_join(s, c);
    if ((t & 63) == 0) wsum[t >> 6] = s;
    __syncthreads();
    s = wsum[0];
    for (int i = 1; i < THREADS / 64; ++i) s = join(s, wsum[i], c);
    none = s.s == 0.0f;  // no value above -inf
    from = s.m;
    minus = 0.0f;
    w = none ? 0.0f : 1.0f / s.s;
  }
  const float gl = counts && g_lp ? g_lp[row] * scale : 0.0f, gh = g_ent ? g_ent[row] * scale : 0.0f;
  // -g_lp p - g_H p (log p + H) = 2^d (k0 - k1w d), d = log2 (p / w)
  const float k1 = gh * kLn2;
  const float k0 = w * (-gl - gh * entropy[row] - k1 * __builtin_amdgcn_logf(w)), k1w = k1 * w;
  for (int i = first; i < vocab; i += step) {
    const int n = min(N, vocab - i);
    float v[N];
    if (n == N) {
      Vec<T>::unpack(load16(x + i), v);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = j < n ? Vec<T>::one(x + i + j) : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      // log p first: it is small where p is large
      const float d = fmaf(v[j] - from, scale, -minus) * kLog2e, p = __builtin_amdgcn_exp2f(d);
      float g = p * fmaf(-k1w, fmaxf(d, -200.0f), k0);
      if (i + j == tok) g += gl;
      v[j] = none ? 0.0f : g;
    }
    if constexpr (N == 8) {
      typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
      const bf16x8_t r{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3],
                       (__bf16)v[4], (__bf16)v[5], (__bf16)v[6], (__bf16)v[7]};
      if (n == N) {
        __builtin_memcpy(o + i, &r, 16);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j < n) reinterpret_cast<__bf16*>(o)[i + j] = r[j];
      }
    } else {
      if (n == N) {
        __builtin_memcpy(o + i, v, 16);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j < n) o[i + j] = v[j];
      }
    }
  }
}

template <class T>
hipError_t run_forward(const LogprobArgs& a, const Partial& p, hipStream_t st) {
  const dim3 grid((unsigned)(a.rows * a.splits));
  if (a.parts) {
    if (a.top > 0) k_logprobs_part<T, true><<<grid, kThreads, 0, st>>>(a, p);
    else k_logprobs_part<T, false><<<grid, kThreads, 0, st>>>(a, p);
  } else if (a.top > 0) k_logprobs<T, true><<<grid, kThreads, 0, st>>>(a, p);
  else k_logprobs<T, false><<<grid, kThreads, 0, st>>>(a, p);
  if (a.splits > 1) k_logprobs_join<T><<<dim3((unsigned)a.rows), kThreads, 0, st>>>(a, p);
  return hipGetLastError();
}

}  // namespace

void logprob_shape(LogprobArgs& a) {
  // Few rows: parts that a block holds in registers, eight blocks a CU at most (kMostParts)
  // (8 rows of 131072: 32 parts each). More rows are split until there are four
  // blocks a CU, down to one load a thread.
  const int n = a.bf16 ? 8 : 4, unit = kThreads * n;
  const int64_t parts = ((int64_t)a.vocab + kHeld * unit - 1) / (kHeld * unit);
  a.parts = parts > 1 && parts * a.rows <= kMostParts;
  if (a.parts) {
    a.split_len = kHeld * unit;
    a.splits = (int)parts;
    return;
  }
  const int64_t most = ((int64_t)a.vocab + unit - 1) / unit;
  int64_t s = a.rows > 0 ? (1024 + a.rows - 1) / a.rows : 1;
  s = s > most ? most : s;
  s = s < 1 ? 1 : s;
  a.split_len = (int)((most + s - 1) / s) * unit;
  if ((int64_t)a.split_len > a.vocab) a.split_len = a.vocab > 0 ? a.vocab : 1;
  a.splits = a.vocab > 0 ? (int)(((int64_t)a.vocab + a.split_len - 1) / a.split_len) : 1;
}

// As many splits as a call of no more rows and entries may have, so that a larger
// call's workspace serves a smaller: up to kMostParts where parts are held in
// registers, fewer than that (two a row at least) where rows are split to fill the
// chip, none where one load a thread covers the row.
size_t logprob_workspace_bytes(const LogprobArgs& a) {
  const int64_t unit = kThreads * (a.bf16 ? 8 : 4), parts = ((int64_t)a.vocab + kHeld * unit - 1) / (kHeld * unit);
  if (a.vocab <= unit) return 256;
  const size_t n = (size_t)std::min(kMostParts, a.rows * std::max<int64_t>(parts, 2));
  return 256 + (n * sizeof(Sums) + 255) / 256 * 256 + (a.top > 0 ? n * kList * 8 : 0);
}

hipError_t launch_logprobs(LogprobArgs a, void* workspace, hipStream_t st) {
  logprob_shape(a);
  Partial p{};
  if (a.splits > 1) {
    const size_t n = (size_t)a.rows * a.splits;
    p.sums = static_cast<Sums*>(workspace);
    p.keys = reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(workspace) + (n * sizeof(Sums) + 255) / 256 * 256);
  }
  return a.bf16 ? run_forward<uint16_t>(a, p, st) : run_forward<float>(a, p, st);
}

template <class T, int THREADS>
static hipError_t run_backward(const void* logits, int64_t ld, int rows, int vocab, const int64_t* tokens, float scale,
                               const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy,
                               void* out, int64_t out_ld, hipStream_t st) {
  // up to 16384 waves, two rounds of the chip's
  const int64_t span = THREADS * Vec<T>::N, most = ((int64_t)vocab + span - 1) / span;
  const int64_t want = (4096 * 256 / THREADS + rows - 1) / rows;
  const dim3 grid((unsigned)rows, (unsigned)std::min(most, want));
  k_logprobs_backward<T, THREADS><<<grid, THREADS, 0, st>>>((const T*)logits, ld, vocab, tokens, scale, lse, entropy,
                                                            g_logprob, g_entropy, (T*)out, out_ld);
  return hipGetLastError();
}

hipError_t launch_logprobs_backward(const void* logits, int64_t ld, bool bf16, int rows, int vocab,
                                    const int64_t* tokens, float scale, const float* lse, const float* entropy,
                                    const float* g_logprob, const float* g_entropy, void* out, int64_t out_ld,
                                    hipStream_t st) {
  // Wide blocks for long rows: 4096 rows of 32000 in bfloat16 take 101 us, 110 with
  // narrow ones, of 18000 58 and 52; in float32 18000 take 113 and 121, 9000 57 and 50.
  const bool wide = (int64_t)vocab * (bf16 ? 2 : 4) >= 56 * 1024;
  auto run = bf16 ? wide ? run_backward<uint16_t, 1024> : run_backward<uint16_t, 256>
                  : wide ? run_backward<float, 1024> : run_backward<float, 256>;
  return run(logits, ld, rows, vocab, tokens, scale, lse, entropy, g_logprob, g_entropy, out, out_ld, st);
}

}  // namespace lt
