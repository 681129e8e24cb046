// Rotary positions of queries and keys (rotary.hpp): rotated in their type or as
// fp8 codes with scales, and on the way into the 4-bit cache.
#include <algorithm>

#include "cache4.hpp"
#include "internal.hpp"
#include "rotary.hpp"

namespace lt {
namespace {

constexpr int kThreads = 256;
// Threads that fill the GPU; a thread takes more heads where there are more tokens than
// that. 16384 tokens of 40 heads of 128 in bfloat16 (335 MB): 67 us with 2^19, 71 with 2^18,
// 65 with 2^20, which costs 5003 tokens of 12 heads of 80 12 us where the others take 10.
constexpr int64_t kFill = 1 << 19;
// As fp8 (4096 tokens of 64 heads of 128, 101 MB): 22 us with 2^18, 25 with 2^19, 27 with 2^17.
constexpr int64_t kFillFp8 = 1 << 18;
// Into the cache: 25 us with 2^17 (below), 29 with 2^18.
constexpr int64_t kFillKv = 1 << 17;

// What a unit of a head covers: two vectors of V values. Halves: in the rotated part
// two vectors whose values are paired, elsewhere two that pass as they are. Interleaved,
// with pairs inside a vector (V > 1): neighbours, each of which is turned or passes.
// The values before, in and behind the part are covered each by vectors of their own;
// the last one of a length that V does not divide is moved down to end with it, so that
// some values are computed twice and written twice the same (never in place, where the
// second thread might read what the first has written). A part of 26 of 64 values in
// halves, 16384 tokens of 20 heads in bfloat16 (84 MB): 23 us, in place, value by value, 28.
struct Unit {
  int a, b;      // offsets of the vectors; b < 0: there is none
  int pa, pb;    // their first pairs, < 0: not rotated (halves: pb = pa)
};
template <int V>
__device__ __forceinline__ int piece(int i, int len) { return min(i * V, len - V); }
// Offset of a vector that passes.
template <int V>
__device__ __forceinline__ int beside(const RotaryArgs& r, int i) {
  const int behind = r.start + 2 * r.pairs;
  return i < r.front ? piece<V>(i, r.start) : behind + piece<V>(i - r.front, r.d - behind);
}
template <int V>
__device__ __forceinline__ Unit unit_of(const RotaryArgs& r, int u) {
  if (V > 1 && r.interleaved) {
    Unit w{0, -1, -1, -1};
    auto vector = [&](int i, int& at, int& pair) {
      const int j = i - r.front;
      if (j >= 0 && j < r.part) {
        const int k = piece<V>(j, 2 * r.pairs);
        at = r.start + k;
        pair = k / 2;
      } else {
        at = beside<V>(r, j < 0 ? i : i - r.part);
      }
    };
    vector(2 * u, w.a, w.pa);
    if (2 * u + 1 < r.front + r.part + r.back) vector(2 * u + 1, w.b, w.pb);
    return w;
  }
  if (u < r.part) {
    if (r.interleaved) return Unit{r.start + 2 * u, r.start + 2 * u + 1, u, u};
    const int k = piece<V>(u, r.pairs);
    return Unit{r.start + k, r.start + r.pairs + k, k, k};
  }
  const int i = 2 * (u - r.part);
  return Unit{beside<V>(r, i), i + 1 < r.front + r.back ? beside<V>(r, i + 1) : -1, -1, -1};
}

// Sines and cosines: of pairs pa ..., or interleaved of V / 2 pairs of either vector (of
// any pairs where one of the two passes).
template <int V>
__device__ __forceinline__ void turns_of(const RotaryArgs& r, const Unit& u, int pos, float (&c)[V], float (&s)[V]) {
  if (u.pa < 0 && u.pb < 0) return;
  const float *fa = r.freq + max(u.pa, 0), *fb = V > 1 && r.interleaved ? r.freq + max(u.pb, 0) : fa + V / 2;
  float f[V];
#pragma unroll
  for (int j = 0; j < V; ++j) f[j] = j < (V + 1) / 2 ? fa[j] : fb[j - (V + 1) / 2];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const Turn t = turn_of((double)pos * turns_per(f[j]), r.amplitude);
    c[j] = t.c;
    s[j] = r.inverse ? -t.s : t.s;
  }
}

// The unit's values x, y (of vectors a and b) turned in place.
template <int V>
__device__ __forceinline__ void turn_unit(const RotaryArgs& r, const Unit& w, float (&x)[V], float (&y)[V],
                                          const float (&c)[V], const float (&s)[V]) {
  if (V == 1 || !r.interleaved) {
    if (w.pa < 0) return;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float u = x[j], v = y[j];
      x[j] = turned(u, c[j], v, -s[j]);
      y[j] = turned(v, c[j], u, s[j]);
    }
    return;
  }
  constexpr int H = V > 1 ? V / 2 : 1;
  if (w.pa >= 0) {
#pragma unroll
    for (int j = 0; j + 1 < V; j += 2) {
      const float u = x[j], v = x[j + 1];
      x[j] = turned(u, c[j / 2], v, -s[j / 2]);
      x[j + 1] = turned(v, c[j / 2], u, s[j / 2]);
    }
  }
  if (w.pb >= 0) {
#pragma unroll
    for (int j = 0; j + 1 < V; j += 2) {
      const float u = y[j], v = y[j + 1];
      y[j] = turned(u, c[H + j / 2], v, -s[H + j / 2]);
      y[j + 1] = turned(v, c[H + j / 2], u, s[H + j / 2]);
    }
  }
}

// Lanes of a head, one unit each (in turn where there are more units); a group of
// them takes every head_lanes-th head of a token, kAhead heads' loads at a time, all
// with the same sines and cosines (two at a time: 71 us where four take 67).
constexpr int kAhead = 4;
template <class TI, class TO, int V>
__device__ __forceinline__ void rotate_rows(const RotaryArgs& r, uint32_t block) {
  const uint32_t at = block * kThreads + threadIdx.x, item = at / (uint32_t)r.lanes;
  const int lane = (int)(at - item * r.lanes);
  const uint32_t tok = item / (uint32_t)r.head_lanes;
  if (tok >= (uint32_t)r.T) return;
  const int h0 = (int)(item - tok * r.head_lanes), pos = r.positions[tok];
  const TI* in = reinterpret_cast<const TI*>(r.x) + (int64_t)tok * r.x_token;
  TO* out = reinterpret_cast<TO*>(r.out) + (int64_t)tok * r.out_token;
  for (int u = lane; u < r.units; u += r.lanes) {
    const Unit w = unit_of<V>(r, u);
    float c[V], s[V];
    for (int h = h0; h < r.H; h += kAhead * r.head_lanes) {
      Raw<TI, V> x[kAhead], y[kAhead];
      if (pos >= 0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int g = min(h + k * r.head_lanes, r.H - 1);
          x[k].load(in + g * r.x_head + w.a);
          if (w.b >= 0) y[k].load(in + g * r.x_head + w.b);
        }
      }
      if (h == h0) turns_of<V>(r, w, pos, c, s);  // while the first loads are on their way
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int g = h + k * r.head_lanes;
        if (g >= r.H) break;
        float a[V] = {}, b[V] = {};
        if (pos >= 0) {
          x[k].unpack(a);
          if (w.b >= 0) y[k].unpack(b);
          turn_unit<V>(r, w, a, b, c, s);
        }
        store_values<V>(out + g * r.out_head + w.a, a);
        if (w.b >= 0) store_values<V>(out + g * r.out_head + w.b, b);
      }
    }
  }
}

template <class TI, class TO, int V>
__global__ __launch_bounds__(kThreads) void k_rotary(RotaryArgs r) {
  rotate_rows<TI, TO, V>(r, blockIdx.x);
}

// ---- fp8 ----
// Exponent byte of the smallest power of two 2^e with top <= 448 * 2^e, from the
// bits of `top`: 448 = 1.75 * 2^8, so adding 0x1FFFFF carries where e has to be one
// larger. Not below 2^-126; 255 (a NaN for the scale) where top is not finite.
__device__ __forceinline__ uint32_t fp8_scale_byte(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;
  const uint32_t e = (top + 0x1FFFFFu) >> 23;
  return e > 9u ? e - 8u : 1u;
}
template <int V>
__device__ __forceinline__ void store_fp8(uint8_t* p, const float (&x)[V], float by) {
  if constexpr (V == 1) {
    *p = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[0] * by, 0.0f, 0, false);
  } else if constexpr (V == 2) {
    const uint16_t w = (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[0] * by, x[1] * by, 0, false);
    __builtin_memcpy(p, &w, 2);
  } else {
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * by, x[4 * i + 1] * by, 0, false);
      v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * by, x[4 * i + 3] * by, v, true);
      w[i] = (uint32_t)v;
    }
    __builtin_memcpy(p, w, V);
  }
}
template <int V>
__device__ __forceinline__ uint32_t top_of(uint32_t top, const float (&x)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
  return top;
}

// A head's scale is known once all its units are turned. ONCE: a lane has one unit and
// keeps it, and has kAhead heads' loads on their way; else the units are turned a second
// time (more than 64 of them).
template <class TI, int V, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_rotary_fp8(RotaryArgs r) {
  const int lanes = r.lanes, lane = threadIdx.x & (lanes - 1);  // a power of two
  const uint32_t item = (blockIdx.x * kThreads + threadIdx.x) / (uint32_t)lanes;
  const uint32_t tok = item / (uint32_t)r.head_lanes;
  if (tok >= (uint32_t)r.T) return;  // whole groups of lanes
  const int h0 = (int)(item - tok * r.head_lanes), pos = r.positions[tok];
  const TI* in = reinterpret_cast<const TI*>(r.x) + (int64_t)tok * r.x_token;
  uint8_t* out = reinterpret_cast<uint8_t*>(r.out) + (int64_t)tok * r.out_token;
  float c[V], s[V];
  // the head's scale from its lanes' largest magnitudes; what values are multiplied by
  auto scale_head = [&](int h, uint32_t top) {
    for (int o = 1; o < lanes; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    const uint32_t e = fp8_scale_byte(top);
    if (lane == 0) r.scale[(int64_t)tok * r.H + h] = e == 255u ? __builtin_nanf("") : __uint_as_float(e << 23);
    return e == 255u ? 0.0f : __uint_as_float((254u - e) << 23);
  };
  auto put = [&](const Unit& w, int h, float by, float (&x)[V], float (&y)[V]) {
    if (by == 0.0f) {  // not finite: codes of 0 (and no conversion of what is not finite)
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = y[j] = 0.0f;
    }
    store_fp8<V>(out + h * r.out_head + w.a, x, by);
    if (w.b >= 0) store_fp8<V>(out + h * r.out_head + w.b, y, by);
  };
  if constexpr (ONCE) {
    const bool mine = lane < r.units;
    const Unit w = unit_of<V>(r, mine ? lane : 0);
    for (int h = h0; h < r.H; h += kAhead * r.head_lanes) {
      Raw<TI, V> p[kAhead], q[kAhead];
      if (pos >= 0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int g = min(h + k * r.head_lanes, r.H - 1);
          p[k].load(in + g * r.x_head + w.a);
          if (w.b >= 0) q[k].load(in + g * r.x_head + w.b);
        }
      }
      if (h == h0) turns_of<V>(r, w, pos, c, s);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int g = h + k * r.head_lanes;
        if (g >= r.H) break;  // whole groups of lanes
        float x[V] = {}, y[V] = {};
        if (pos >= 0) {
          p[k].unpack(x);
          if (w.b >= 0) q[k].unpack(y);
          turn_unit<V>(r, w, x, y, c, s);
        }
        const float by = scale_head(g, mine ? top_of<V>(top_of<V>(0u, x), y) : 0u);
        if (mine) put(w, g, by, x, y);
      }
    }
  } else {
    auto values = [&](const Unit& w, int h, float (&x)[V], float (&y)[V]) {
      if (pos < 0) return;
      load_values<V>(in + h * r.x_head + w.a, x);
      if (w.b >= 0) load_values<V>(in + h * r.x_head + w.b, y);
      turns_of<V>(r, w, pos, c, s);
      turn_unit<V>(r, w, x, y, c, s);
    };
    for (int h = h0; h < r.H; h += r.head_lanes) {
      uint32_t top = 0;
      for (int u = lane; u < r.units; u += lanes) {
        float x[V] = {}, y[V] = {};
        values(unit_of<V>(r, u), h, x, y);
        top = top_of<V>(top_of<V>(top, x), y);
      }
      const float by = scale_head(h, top);
      for (int u = lane; u < r.units; u += lanes) {
        float x[V] = {}, y[V] = {};
        const Unit w = unit_of<V>(r, u);
        values(w, h, x, y);
        put(w, h, by, x, y);
      }
    }
  }
}

// ---- into the 4-bit cache ----
// As in k_cache4_append, four threads share a block of 32 values and its largest
// magnitude, 8 consecutive values each.
__device__ __forceinline__ void put_codes(const float (&x)[8], int64_t row, int d, int which, int ch, uint8_t* codes,
                                          uint8_t* scales) {
  uint32_t top = top_of<8>(0u, x);  // NaN and infinity lie above every finite value
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  const uint32_t e = scale_byte(top);
  const float s = __uint_as_float(e << 23);
  uint32_t w = 0;
  if (e != 255u) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  }
  *reinterpret_cast<uint32_t*>(codes + row * d + which * (d / 2) + ch * 4) = w;
  if ((ch & 3) == 0) scales[row * (d / 16) + which * (d / 32) + (ch >> 2)] = (uint8_t)e;
}

// A token's slot, or -1 where nothing is written.
__device__ __forceinline__ int64_t slot_of(const AppendRotaryArgs& a, const Cache4& c, uint32_t tok) {
  const int64_t slot = a.slots[tok];
  return a.positions[tok] < 0 || slot < 0 || slot >= c.num_pages << c.shift ? -1 : slot;
}

// Parts made of whole blocks of 32 (or of whole vectors, interleaved): a thread takes
// two vectors of 8 of a head, those that face each other where halves are paired, of the
// key and of the value, and every head_lanes-th head with the same sines and cosines. So
// a slot's key and value are written side by side, a line at a time. 16381 tokens of 8
// heads of 128 in bfloat16 (85 MB): 25 us, where k_cache4_append alone takes 27. (Loads of
// two heads ahead: 3 us more, of four 5.)
template <class T>
__device__ __forceinline__ void append_pairs(const AppendRotaryArgs& a, const Cache4& c, uint32_t block) {
  const int units = c.d / 16;  // lanes of a head: 4 or 8
  const uint32_t item = (block * kThreads + threadIdx.x) / units;
  const int u = threadIdx.x & (units - 1);
  const uint32_t tok = item / (uint32_t)a.head_lanes;
  if (tok >= a.rows) return;  // whole heads
  const int64_t slot = slot_of(a, c, tok);
  if (slot < 0) return;
  const int h0 = (int)(item - tok * a.head_lanes), pos = a.positions[tok];
  // the thread's vectors, and whether (and as which pairs) they are turned
  int va, vb, pair[2] = {-1, -1};
  if (a.interleaved) {
    va = u, vb = u + units;
    const int first = a.start / 8, last = first + a.pairs / 4;
    if (va >= first && va < last) pair[0] = (va - first) * 4;
    if (vb >= first && vb < last) pair[1] = (vb - first) * 4;
  } else {
    const int n = a.pairs / 8, first = a.start / 8;
    if (u < n) {
      va = first + u, vb = va + n;
      pair[0] = u * 8, pair[1] = pair[0] + 4;
    } else {  // blocks that pass, two at a time
      const int i = (u - n) / 4 * 8 + (u & 3);
      va = i < first ? i : i + 2 * n;
      vb = i + 4 < first ? i + 4 : i + 4 + 2 * n;
    }
  }
  const T* kin = reinterpret_cast<const T*>(a.k) + (int64_t)tok * a.k_stride;
  const T* vin = reinterpret_cast<const T*>(a.v) + (int64_t)tok * a.v_stride;
  float cs[8], sn[8];
  for (int h = h0; h < c.hkv; h += a.head_lanes) {
    Raw<T, 8> raw[4];
    raw[0].load(kin + h * c.d + va * 8);
    raw[1].load(kin + h * c.d + vb * 8);
    raw[2].load(vin + h * c.d + va * 8);
    raw[3].load(vin + h * c.d + vb * 8);
    if (h == h0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int p = pair[j / 4];
        if (p < 0) continue;
        const Turn t = turn_of((double)pos * turns_per(a.freq[p + j % 4]), a.amplitude);
        cs[j] = t.c, sn[j] = t.s;
      }
    }
    const int64_t row = c.row(slot, h);
    float x[8], y[8];
    raw[0].unpack(x);
    raw[1].unpack(y);
    if (!a.interleaved) {
      if (pair[0] >= 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = x[j], q = y[j];
          x[j] = turned(p, cs[j], q, -sn[j]);
          y[j] = turned(q, cs[j], p, sn[j]);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float p = x[2 * j], q = x[2 * j + 1];
        if (pair[0] >= 0) x[2 * j] = turned(p, cs[j], q, -sn[j]), x[2 * j + 1] = turned(q, cs[j], p, sn[j]);
        p = y[2 * j], q = y[2 * j + 1];
        if (pair[1] >= 0)
          y[2 * j] = turned(p, cs[4 + j], q, -sn[4 + j]), y[2 * j + 1] = turned(q, cs[4 + j], p, sn[4 + j]);
      }
    }
    put_codes(x, row, c.d, 0, va, a.codes, a.scales);
    put_codes(y, row, c.d, 0, vb, a.codes, a.scales);
    raw[2].unpack(x);
    raw[3].unpack(y);
    put_codes(x, row, c.d, 1, va, a.codes, a.scales);
    put_codes(y, row, c.d, 1, vb, a.codes, a.scales);
  }
}

// Any other part: a thread takes 8 consecutive values of a key and reads each one's
// partner by itself. The same rows with 32 of 128 values turned in halves: 33 us, 20 where
// whole blocks are.
template <class T>
__device__ __forceinline__ void append_keys(const AppendRotaryArgs& a, const Cache4& c, uint32_t block) {
  const int per_row = c.d / 8;  // lanes of a head: 8 or 16
  const uint32_t item = (block * kThreads + threadIdx.x) / per_row;
  const int ch = threadIdx.x & (per_row - 1);
  const uint32_t tok = item / (uint32_t)a.head_lanes;
  if (tok >= a.rows) return;  // whole heads
  const int64_t slot = slot_of(a, c, tok);
  if (slot < 0) return;
  const int h0 = (int)(item - tok * a.head_lanes), pos = a.positions[tok];
  // each value's partner (offset from its own), and its turn
  int partner[8];
  float cs[8], sn[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int i = ch * 8 + j - a.start;  // in the rotated part
    partner[j] = 0;
    cs[j] = 1.0f, sn[j] = 0.0f;
    if (i < 0 || i >= 2 * a.pairs) continue;
    const bool first = a.interleaved ? !(i & 1) : i < a.pairs;
    const int pair = a.interleaved ? i >> 1 : first ? i : i - a.pairs;
    partner[j] = a.interleaved ? (first ? 1 : -1) : first ? a.pairs : -a.pairs;
    const Turn t = turn_of((double)pos * turns_per(a.freq[pair]), a.amplitude);
    cs[j] = t.c;
    sn[j] = first ? -t.s : t.s;
  }
  const T* in = reinterpret_cast<const T*>(a.k) + (int64_t)tok * a.k_stride + ch * 8;
  for (int h = h0; h < c.hkv; h += a.head_lanes) {
    const T* p = in + (int64_t)h * c.d;
    float x[8], y[8];
    load_values<8>(p, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float z[1];
      load_values<1>(p + j + partner[j], z);
      y[j] = partner[j] ? turned(x[j], cs[j], z[0], sn[j]) : x[j];
    }
    put_codes(y, c.row(slot, h), c.d, 0, ch, a.codes, a.scales);
  }
}

template <class T>
__device__ __forceinline__ void append_values(const AppendRotaryArgs& a, const Cache4& c, uint32_t block) {
  const int per_row = c.d / 8, per_tok = c.hkv * per_row;
  const uint32_t at = block * kThreads + threadIdx.x, tok = at / (uint32_t)per_tok;
  if (tok >= a.rows) return;
  const int in = (int)(at - tok * per_tok), h = in / per_row, ch = in - h * per_row;
  const int64_t slot = slot_of(a, c, tok);
  if (slot < 0) return;
  float x[8];
  load_values<8>(reinterpret_cast<const T*>(a.v) + (int64_t)tok * a.v_stride + in * 8, x);
  put_codes(x, c.row(slot, h), c.d, 1, ch, a.codes, a.scales);
}

// One launch: blocks of keys and values and of queries, side by side (two kernels one after
// the other take 83 us where this takes 75: 32 query heads beside the above).
template <class T, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_append_rotary(AppendRotaryArgs a, Cache4 c) {
  const int64_t b = blockIdx.x;
  if (b < a.k_blocks) {
    if constexpr (WIDE) append_pairs<T>(a, c, (uint32_t)b);
    else append_keys<T>(a, c, (uint32_t)b);
  } else if (!WIDE && b < a.k_blocks + a.v_blocks) {
    append_values<T>(a, c, (uint32_t)(b - a.k_blocks));
  } else {
    const uint32_t q = (uint32_t)(b - a.k_blocks - a.v_blocks);
    if (WIDE || a.q.vec == 8) rotate_rows<T, uint16_t, 8>(a.q, q);
    else if (a.q.vec == 4) rotate_rows<T, uint16_t, 4>(a.q, q);
    else if (a.q.vec == 2) rotate_rows<T, uint16_t, 2>(a.q, q);
    else rotate_rows<T, uint16_t, 1>(a.q, q);
  }
}
// Whether vectors of n values cover a length (exactly, or the last one moved down).
bool covers(int len, int n, bool exact) { return len == 0 || (exact ? len % n == 0 : len >= n); }

// The widest vectors that cover the part and what lies before and behind it, in place
// without a value twice.
void choose_vec(RotaryArgs& a) {
  const int part = a.interleaved ? 2 * a.pairs : a.pairs, behind = a.d - a.start - 2 * a.pairs;
  const bool exact = a.x == a.out;
  for (a.vec = 8; a.vec > 1; a.vec /= 2)
    if (covers(a.start, a.vec, exact) && covers(part, a.vec, exact) && covers(behind, a.vec, exact)) break;
  const int V = a.vec;
  a.front = (a.start + V - 1) / V;
  a.back = (behind + V - 1) / V;
  a.part = V == 1 ? a.pairs : (part + V - 1) / V;
  a.units = V > 1 && a.interleaved ? (a.front + a.part + a.back + 1) / 2 : a.part + (a.front + a.back + 1) / 2;
}

// Lanes of a head: one a unit, 64 at most; where they exchange values a power of two.
void lanes_of(RotaryArgs& a, bool power) {
  a.lanes = std::min(std::max(a.units, 1), 64);
  if (power)
    while (a.lanes & (a.lanes - 1)) ++a.lanes;
}

// Groups of lanes of a token: as few as fill the GPU, so that each has several heads. (Few
// heads get a group each, which takes the sines and cosines again: 48887 tokens of 3 heads
// of 64 in bfloat16, 38 MB, 14 us, where the memory takes 7.6.)
int lanes_for(int64_t threads, int heads, int64_t fill) {  // threads with one group a token
  return (int)std::min<int64_t>(std::max(heads, 1), (fill + std::max<int64_t>(threads, 1) - 1) / std::max<int64_t>(threads, 1));
}

int64_t rotary_blocks(RotaryArgs& a, int64_t fill = kFill) {
  const int64_t threads = (int64_t)a.T * a.lanes;
  a.head_lanes = lanes_for(threads, a.H, fill);
  return (threads * a.head_lanes + kThreads - 1) / kThreads;
}

template <class TI, class TO>
void run_rotary(const RotaryArgs& a, dim3 grid, hipStream_t st) {
  switch (a.vec) {
    case 8: k_rotary<TI, TO, 8><<<grid, kThreads, 0, st>>>(a); break;
    case 4: k_rotary<TI, TO, 4><<<grid, kThreads, 0, st>>>(a); break;
    case 2: k_rotary<TI, TO, 2><<<grid, kThreads, 0, st>>>(a); break;
    default: k_rotary<TI, TO, 1><<<grid, kThreads, 0, st>>>(a); break;
  }
}
template <class TI, int V>
void run_fp8(const RotaryArgs& a, dim3 grid, hipStream_t st) {
  if (a.units <= a.lanes) k_rotary_fp8<TI, V, true><<<grid, kThreads, 0, st>>>(a);
  else k_rotary_fp8<TI, V, false><<<grid, kThreads, 0, st>>>(a);
}
template <class TI>
void run_rotary_fp8(const RotaryArgs& a, dim3 grid, hipStream_t st) {
  switch (a.vec) {
    case 8: run_fp8<TI, 8>(a, grid, st); break;
    case 4: run_fp8<TI, 4>(a, grid, st); break;
    case 2: run_fp8<TI, 2>(a, grid, st); break;
    default: run_fp8<TI, 1>(a, grid, st); break;
  }
}

}  // namespace

int64_t rotary_shape(RotaryArgs& a, bool fp8) {
  choose_vec(a);
  lanes_of(a, fp8);
  return rotary_blocks(a, fp8 ? kFillFp8 : kFill);
}

hipError_t launch_rotary(const RotaryArgs& r, hipStream_t st) {
  RotaryArgs a = r;
  const dim3 grid((unsigned)rotary_shape(a, a.scale != nullptr));
  if (a.scale) {
    if (a.in_f32) run_rotary_fp8<float>(a, grid, st);
    else run_rotary_fp8<uint16_t>(a, grid, st);
  } else if (a.in_f32 && a.out_f32) {
    run_rotary<float, float>(a, grid, st);
  } else if (a.in_f32) {
    run_rotary<float, uint16_t>(a, grid, st);
  } else {
    run_rotary<uint16_t, uint16_t>(a, grid, st);
  }
  return hipGetLastError();
}

int64_t append_rotary_shape(AppendRotaryArgs& a, const Cache4& c) {
  a.wide = a.interleaved ? a.start % 8 == 0 && a.pairs % 4 == 0 : a.start % 32 == 0 && a.pairs % 32 == 0;
  if (a.q.T > 0) {
    choose_vec(a.q);
    a.wide = a.wide && a.q.vec == 8;
  }
  const int lanes = c.d / (a.wide ? 16 : 8);
  a.head_lanes = lanes_for(a.rows * lanes, c.hkv, kFillKv);
  a.k_blocks = (a.rows * a.head_lanes * lanes + kThreads - 1) / kThreads;
  a.v_blocks = a.wide ? 0 : (a.rows * c.hkv * lanes + kThreads - 1) / kThreads;
  a.q_blocks = 0;
  if (a.q.T > 0) {
    lanes_of(a.q, false);
    a.q_blocks = rotary_blocks(a.q);
  }
  return a.q_blocks + a.k_blocks + a.v_blocks;
}

hipError_t launch_cache4_append_rotary(const AppendRotaryArgs& r, const Cache4& c, hipStream_t st) {
  AppendRotaryArgs a = r;
  const int64_t blocks = append_rotary_shape(a, c);
  const dim3 grid((unsigned)blocks);
  if (a.in_f32 && a.wide) k_append_rotary<float, true><<<grid, kThreads, 0, st>>>(a, c);
  else if (a.in_f32) k_append_rotary<float, false><<<grid, kThreads, 0, st>>>(a, c);
  else if (a.wide) k_append_rotary<uint16_t, true><<<grid, kThreads, 0, st>>>(a, c);
  else k_append_rotary<uint16_t, false><<<grid, kThreads, 0, st>>>(a, c);
  return hipGetLastError();
}

}  // namespace lt
