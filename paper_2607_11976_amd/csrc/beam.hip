// Beam search's selection: of a request's beams w, each with a score c_w and a row
// of logits x_w, the `top` best continuations by
//
//   score(w, v) = c_w + scale x_wv - lse_w,   lse_w = log sum_v exp(scale x_wv).
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
// chains, those in float64; scale log2 e is two float32 numbers, and lse and score
// are float64 until the score's one rounding.
//
// Bound by reading the logits.
#include <algorithm>

#include "internal.hpp"

namespace lt {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kLoads = 4;              // 16-byte loads of a lane in a tile
constexpr int kList = 256;             // candidates that a wave keeps before it cuts them to the best
constexpr float kLowest = -3.402823466e38f;
constexpr uint32_t kNinfKey = 0x007FFFFFu;  // ord_key(-inf): values above it are candidates

__device__ __forceinline__ float ninf() { return -__builtin_inff(); }

template <class T>
struct Row;
template <>
struct Row<uint16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t kFill = 0xFF80FF80u;  // -inf
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
  static constexpr uint32_t kFill = 0xFF800000u;
  __device__ static __forceinline__ void unpack(const uint4& a, float (&x)[4]) {
    x[0] = __uint_as_float(a.x), x[1] = __uint_as_float(a.y);
    x[2] = __uint_as_float(a.z), x[3] = __uint_as_float(a.w);
  }
};

// Elements [i, i + N) of a row (at the elements' alignment), those from e on as -inf.
template <class T>
__device__ __forceinline__ uint4 fetch(const T* x, int i, int e) {
  constexpr int N = Row<T>::N;
  uint4 v;
  if (i + N <= e) {
    __builtin_memcpy(&v, x + i, 16);
    return v;
  }
  uint32_t w[4] = {Row<T>::kFill, Row<T>::kFill, Row<T>::kFill, Row<T>::kFill};
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

// What a part of a row leaves: sum of 2^((x - m) scale log2 e), and m.
struct Sum {
  double s;
  float m;
  float pad;
};
struct Part {
  Sum* sums;       // [rows * splits]
  uint64_t* keys;  // [rows * splits][top], best first; 0: no candidate
};

// The n-th largest of the wave's 64 values, cut to its upper 16 bits: at least n
// lanes reach it.
__device__ __forceinline__ uint32_t lanes_floor(uint32_t v, int n) {
  uint32_t t = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t c = t | 1u << bit;
    if (__popcll(__ballot(v >= c)) >= n) t = c;
  }
  return t;
}

// Orders a wave's own LDS traffic across its lanes.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wave's candidates in LDS, cut to the best n when they run full.
struct List {
  uint64_t* at;
  int count;       // uniform in the wave
  uint32_t floor;  // the n-th best's value once there are n, else that of -inf
};
__device__ __forceinline__ void cut(List& l, int n) {
  wave_sync();
  if (l.count <= n) {
    if (l.count == n) {
      const int lane = threadIdx.x & 63;
      uint32_t low = lane < n ? (uint32_t)(l.at[lane] >> 32) : 0xFFFFFFFFu;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) low = min(low, (uint32_t)__shfl_xor((int)low, o));
      l.floor = max(l.floor, low);
    }
    return;
  }
  const int lane = threadIdx.x & 63;
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
  uint32_t low = 0xFFFFFFFFu;
#pragma unroll
  for (int i = 0; i < kList / 64; ++i) {
    const bool in = k[i] >= t && k[i] != 0;
    const uint64_t who = __ballot(in);
    if (in) {
      l.at[at + __popcll(who & ((1ull << lane) - 1))] = k[i];
      low = min(low, (uint32_t)(k[i] >> 32));
    }
    at += __popcll(who);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) low = min(low, (uint32_t)__shfl_xor((int)low, o));
  l.count = at;
  l.floor = max(l.floor, low);
  wave_sync();
}

// A part of a row: the block's four waves take its tiles in turn. A wave looks at a
// tile's values one by one only where a lane's largest passes the n-th best so far.
template <class T>
__global__ __launch_bounds__(kThreads) void k_beam_part(BeamArgs a, Part part) {
  constexpr int N = Row<T>::N, kTile = 64 * N * kLoads;
  __shared__ uint64_t lists[kWaves][kList];
  __shared__ Sum sums[kWaves];
  __shared__ int counts[kWaves];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits, n = a.top;
  const float cum = a.cum[row];
  if (!(cum > ninf())) return;  // a beam that is not alive: no candidate, whatever its logits
  const T* x = reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.ld;
  const int b = split * a.split_len, e = min(a.vocab - b, a.split_len) + b;
  const Scale c = scale_of(a.scale);
  float m = kLowest;
  double s = 0.0;
  List list{lists[wave], 0, kNinfKey};
  for (int base = b + wave * kTile; base < e; base += kWaves * kTile) {
    uint4 raw[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) raw[k] = fetch<T>(x, base + (k * 64 + lane) * N, e);
    float v[kLoads][N], top = ninf();
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      Row<T>::unpack(raw[k], v[k]);
#pragma unroll
      for (int j = 0; j < N; ++j) top = fmaxf(top, v[k][j]);
    }
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
    // candidates: values above the floor (later ones that equal it come after), and
    // where n lanes pass it, not below what n lanes reach
    const uint32_t best = ord_key(top);
    const uint64_t who = __ballot(best > list.floor);
    if (!who) continue;
    uint32_t gate = list.floor + 1;
    if (__popcll(who) > n) gate = max(gate, lanes_floor(best, n));
    float g = key_float(gate);
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        bool in = v[k][j] >= g;
        uint64_t mask = __ballot(in);
        if (!mask) continue;
        if (list.count + __popcll(mask) > kList) {
          cut(list, n);
          // equal values of this tile may come before those in the list
          if (list.floor > gate) gate = list.floor, g = key_float(gate);
          in = v[k][j] >= g;
          mask = __ballot(in);
        }
        if (in)
          list.at[list.count + __popcll(mask & ((1ull << lane) - 1))] =
              comp_key(v[k][j], (uint32_t)(base + (k * 64 + lane) * N + j));
        list.count += __popcll(mask);
      }
    cut(list, n);
  }
  // the wave's sums, then the block's
  float wm = m;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) wm = fmaxf(wm, __shfl_xor(wm, o));
  s *= (double)power(m - wm, c);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
  if (lane == 0) {
    sums[wave] = Sum{s, wm, 0.0f};
    counts[wave] = list.count;
  }
  __syncthreads();
  if (t == 0) {
    float bm = sums[0].m;
    for (int i = 1; i < kWaves; ++i) bm = fmaxf(bm, sums[i].m);
    double bs = 0.0;
    for (int i = 0; i < kWaves; ++i) bs += sums[i].s * (double)power(sums[i].m - bm, c);
    part.sums[blockIdx.x] = Sum{bs, bm, 0.0f};
  }
  // each of the waves' candidates (n a wave, 64 at most) counts how many come before it
  const uint64_t mine = lane < counts[wave] ? lists[wave][lane] : 0;
  int before = 0, total = 0;
  for (int w = 0; w < kWaves; ++w) {
    total += counts[w];
    for (int i = 0; i < counts[w]; ++i) before += lists[w][i] > mine;
  }
  uint64_t* out = part.keys + (int64_t)blockIdx.x * n;
  if (mine && before < n) out[before] = mine;
  if (t >= total && t < n) out[t] = 0;
}

// ---- join: a block a request ----
struct Candidate {
  uint32_t score;  // ord_key
  int beam;        // -1: none
  uint64_t key;    // logit and token
};
__device__ __forceinline__ bool comes_before(const Candidate& a, const Candidate& b) {
  if (a.score != b.score) return a.score > b.score;
  if (a.beam != b.beam) return a.beam < b.beam;
  return a.key > b.key;
}

constexpr int kMost = 512;     // candidates that are ranked together

__global__ __launch_bounds__(kThreads) void k_beam_join(BeamArgs a, Part part) {
  extern __shared__ double lse[];             // [beams]
  __shared__ Candidate found[kMost];
  __shared__ __align__(16) uint32_t tops[kThreads];
  __shared__ int count;
  __shared__ Candidate pick[kWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, n = a.top, req = blockIdx.x;
  const Scale c = scale_of(a.scale);
  if (t == 0) count = 0;
  for (int w = wave; w < a.beams; w += kWaves) {
    const Sum* sums = part.sums + ((int64_t)req * a.beams + w) * a.splits;
    const bool alive = a.cum[req * a.beams + w] > ninf();
    float m = kLowest;
    if (alive)
      for (int i = lane; i < a.splits; i += 64) m = fmaxf(m, sums[i].m);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    double s = 0.0;
    if (alive)
      for (int i = lane; i < a.splits; i += 64) s += sums[i].s * (double)power(sums[i].m - m, c);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
    if (lane == 0) lse[w] = (double)m * a.scale + log(s);
  }
  __syncthreads();
  const int per = a.splits * n, total = a.beams * per;  // keys of a beam, of the request
  const uint64_t* keys = part.keys + (int64_t)req * total;
  auto candidate = [&](int i) {
    const int w = i / per;
    const float cum = a.cum[req * a.beams + w];
    const uint64_t key = cum > ninf() ? keys[i] : 0;
    if (!key) return Candidate{0, -1, 0};
    const float score = (float)((double)cum + ((double)key_float((uint32_t)(key >> 32)) * a.scale - lse[w]));
    if (!(score > ninf())) return Candidate{0, -1, 0};
    return Candidate{ord_key(score), w, key};
  };
  // a score that n threads' own best reach (cut to its upper half)
  uint32_t best = 0;
  for (int i = t; i < total; i += kThreads) best = max(best, candidate(i).score);
  tops[t] = best;
  __syncthreads();
  const uint4 q = reinterpret_cast<const uint4*>(tops)[lane];
  uint32_t floor = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t v = floor | 1u << bit;
    const int reach = __popcll(__ballot(q.x >= v)) + __popcll(__ballot(q.y >= v)) + __popcll(__ballot(q.z >= v)) +
                      __popcll(__ballot(q.w >= v));
    if (reach >= n) floor = v;
  }
  for (int i = t; i < total; i += kThreads) {
    const Candidate k = candidate(i);
    if (k.beam >= 0 && k.score >= floor) {
      const int at = atomicAdd(&count, 1);
      if (at < kMost) found[at] = k;
    }
  }
  __syncthreads();
  const int have = count;
  auto put = [&](int place, const Candidate& k) {
    const int64_t o = (int64_t)req * n + place;
    a.out_score[o] = k.beam < 0 ? ninf() : key_float(k.score);
    a.out_beam[o] = k.beam;
    a.out_token[o] = k.beam < 0 ? -1 : (int)comp_pos(k.key);
  };
  if (have <= kMost) {
    for (int i = t; i < have; i += kThreads) {
      const Candidate k = found[i];
      int before = 0;
      for (int j = 0; j < have; ++j) before += comes_before(found[j], k);
      if (before < n) put(before, k);
    }
    for (int i = have + t; i < n; i += kThreads) put(i, Candidate{0, -1, 0});
    return;
  }
  // many equal scores: one after the other
  Candidate last{0xFFFFFFFFu, -1, ~0ull};  // before all
  for (int place = 0; place < n; ++place) {
    Candidate k{0, -1, 0};
    for (int i = t; i < total; i += kThreads) {
      const Candidate v = candidate(i);
      if (v.beam >= 0 && comes_before(last, v) && (k.beam < 0 || comes_before(v, k))) k = v;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const Candidate v{(uint32_t)__shfl_xor((int)k.score, o), __shfl_xor(k.beam, o),
                        ((uint64_t)(uint32_t)__shfl_xor((int)(k.key >> 32), o) << 32) |
                            (uint32_t)__shfl_xor((int)(uint32_t)k.key, o)};
      if (v.beam >= 0 && (k.beam < 0 || comes_before(v, k))) k = v;
    }
    if (lane == 0) pick[wave] = k;
    __syncthreads();
    k = pick[0];
    for (int i = 1; i < kWaves; ++i)
      if (pick[i].beam >= 0 && (k.beam < 0 || comes_before(pick[i], k))) k = pick[i];
    __syncthreads();
    if (t == 0) put(place, k);
    if (k.beam >= 0) last = k;
  }
}

}  // namespace

// Parts of a row: enough blocks to fill the GPU, none shorter than a tile for each wave.
void beam_shape(BeamArgs& a) {
  const int64_t rows = (int64_t)a.batch * a.beams;
  const int tile = kWaves * 64 * kLoads * (a.bf16 ? 8 : 4);
  const int64_t most = std::max<int64_t>(1, (a.vocab + tile - 1) / tile);
  a.splits = (int)std::min<int64_t>(most, std::max<int64_t>(1, 1024 / std::max<int64_t>(rows, 1)));
  a.split_len = (int)std::max<int64_t>(tile, ((a.vocab + (int64_t)a.splits - 1) / a.splits + tile - 1) / tile * tile);
  a.splits = (int)std::max<int64_t>(1, (a.vocab + (int64_t)a.split_len - 1) / a.split_len);
}

static size_t sums_bytes(int64_t parts) { return ((size_t)parts * sizeof(Sum) + 255) / 256 * 256; }

// Splits follow from rows and vocabulary, but a call of fewer rows or entries may take
// more of them: sized for the most parts that any call within these sizes takes.
size_t beam_workspace_bytes(const BeamArgs& a) {
  const int64_t rows = (int64_t)a.batch * a.beams;
  const int tile = kWaves * 64 * kLoads * (a.bf16 ? 8 : 4);
  const int64_t most = std::max<int64_t>(1, (a.vocab + tile - 1) / tile);
  // rows * splits <= max(rows, 1024), and never more than rows * most
  const int64_t parts = std::max(rows, std::min<int64_t>(rows * most, 1024));
  return sums_bytes(parts) + (size_t)parts * a.top * sizeof(uint64_t) + 256;
}

hipError_t launch_beam_select(BeamArgs a, void* workspace, hipStream_t st) {
  beam_shape(a);
  const int64_t parts = (int64_t)a.batch * a.beams * a.splits;
  Part part;
  part.sums = static_cast<Sum*>(workspace);
  part.keys = reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(workspace) + sums_bytes(parts));
  if (a.bf16) k_beam_part<uint16_t><<<dim3((unsigned)parts), kThreads, 0, st>>>(a, part);
  else k_beam_part<float><<<dim3((unsigned)parts), kThreads, 0, st>>>(a, part);
  k_beam_join<<<dim3((unsigned)a.batch), kThreads, (size_t)a.beams * sizeof(double), st>>>(a, part);
  return hipGetLastError();
}

}  // namespace lt
