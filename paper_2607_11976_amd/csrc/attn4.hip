// Attention over the 4-bit paged cache: the new tokens of each request attend
// to the request's cached keys, all visible ones or the ones on a token's list.
//
//   s_j = scale * q . k_j,   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
//
// One pass over the keys with the running maximum m and sum (per row, float32;
// powers of two, so scale carries log2 e). Keys and values are decoded in
// registers (exact in bfloat16) and multiplied on the matrix cores with
// float32 accumulators; the probabilities are rounded to bfloat16 for the
// second product, as its operands have to be, which is of the size of the
// output's own rounding.
//
// Rows are (token, head of the group) pairs that share a KV head. A tile is up
// to 16 (k_attn4_few), 64 or 128 (k_attn4_many) rows of one request; the keys
// of all tiles are shared out evenly over the blocks, and the parts of a tile
// that falls to several are joined by a second kernel.
#include <algorithm>

#include "cache4.hpp"
#include "internal.hpp"

namespace lt {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;

constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kInlineRequests = 64;  // requests that a wave schedules by itself

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }
__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ uint32_t lane_bcast(uint32_t v, int lane) {
  return (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// ---------------------------------------------------------------------------
// Schedule. All tiles, laid end to end by the keys they see, are one line of
// work, cut into equal shares for the blocks: whatever the lengths of the
// requests, every block has as much to do, and only tiles that a cut falls into
// are joined afterwards (at most two parts a block).
//
// A tile's length on that line is an estimate: request r has n row tiles a KV
// head, the j-th from the end sees about u_j = top - j * slope keys, the line
// between its last and its first token's ranges (exact for a causal mask and for
// a window), and its start costs as much time as kStart keys. The estimate only
// balances: the last part of a tile takes the keys that are left. A cut falls on
// a multiple of 64 keys of the tile.
//
// One share for each block that is resident at once, two a CU: a decode step of
// 48 requests of 1K to 128K keys (1.31 GB) takes 246 us, 256 with two shares a
// block and 302 with eight (each pays its start again), and with three blocks a
// CU (fewer registers for loads in flight) 293.
// ---------------------------------------------------------------------------
constexpr int kShares = 512;
template <int ROWS>
constexpr int kStart = ROWS == 16 ? 384 : 128;
constexpr int kMinShare = 128;
constexpr int kCut = 64;

// Keys of a request; positions and steps past them stay within 31 bits.
__device__ __forceinline__ int key_count(int n) { return min(max(n, 0), LT_CACHE4_MAX_KEYS); }

struct Req {
  int t0, nt, len, tiles;  // first token, tokens, cached keys, row tiles
  uint32_t top, slope;
  // keys of the tiles before the j-th, one head
  __device__ __forceinline__ uint64_t before(uint32_t j) const {
    return (uint64_t)j * top - (uint64_t)j * (j - 1) / 2 * slope;
  }
  __device__ __forceinline__ uint32_t keys(uint32_t j) const { return top - j * slope; }
};

template <int ROWS>
__device__ __forceinline__ Req load_req(const Attn4Args& a, int r) {
  Req q;
  const int t0 = min(max(a.cu[r], 0), a.T), t1 = min(max(a.cu[r + 1], t0), a.T);
  q.t0 = t0;
  q.nt = t1 - t0;
  q.len = key_count(a.seq[r]);
  q.tiles = (int)(((int64_t)q.nt * a.group + ROWS - 1) / ROWS);
  int e0 = q.len - q.nt + 1, e1 = q.len, s0 = 0, s1 = 0;
  if (q.nt > 0 && a.end) e0 = a.end[t0], e1 = a.end[t1 - 1];
  if (q.nt > 0 && a.start) s0 = a.start[t0], s1 = a.start[t1 - 1];
  e0 = min(max(e0, 0), q.len), e1 = min(max(e1, 0), q.len);
  const int first = max(e0 - max(s0, 0), 0), last = max(e1 - max(s1, 0), 0);
  q.slope = q.tiles > 1 && last > first ? (uint32_t)(last - first) / (uint32_t)(q.tiles - 1) : 0u;
  q.top = (uint32_t)max(first, last) + kStart<ROWS>;
  return q;
}

__device__ __forceinline__ uint64_t shfl64_up(uint64_t v, int o) {
  return ((uint64_t)(uint32_t)__shfl_up((int)(v >> 32), o) << 32) | (uint32_t)__shfl_up((int)(uint32_t)v, o);
}
__device__ __forceinline__ uint64_t wave_prefix64(uint64_t v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t u = shfl64_up(v, o);
    if (lane >= o) v += u;
  }
  return v;
}
__device__ __forceinline__ uint64_t lane_bcast64(uint64_t v, int lane) {
  return ((uint64_t)lane_bcast((uint32_t)(v >> 32), lane) << 32) | lane_bcast((uint32_t)v, lane);
}
__device__ __forceinline__ uint64_t uniform64(uint64_t v) { return lane_bcast64(v, 0); }

// The lines' beginnings of more than kInlineRequests requests, and their end.
template <int ROWS>
__global__ __launch_bounds__(1024) void k_attn4_schedule(Attn4Args a) {
  __shared__ uint64_t part[16];
  const int t = threadIdx.x, w = t >> 6, lane = t & 63;
  uint64_t base = 0;
  for (int r0 = 0; r0 < a.R; r0 += 1024) {
    const int r = r0 + t;
    uint64_t n = 0;
    if (r < a.R) {
      const Req q = load_req<ROWS>(a, r);
      n = a.hkv * q.before(q.tiles);
    }
    const uint64_t in = wave_prefix64(n);
    __syncthreads();
    if (lane == 63) part[w] = in;
    __syncthreads();
    uint64_t before = base;
    for (int i = 0; i < 16; ++i) {
      if (i < w) before += part[i];
      base += part[i];
    }
    if (r < a.R) a.sched[r] = before + in - n;
  }
  if (t == 0) a.sched[a.R] = base;
}

// The last of n >= 1 ascending entries (the first is taken to be <= x) that is <= x; wave-uniform.
template <class T>
__device__ __forceinline__ int last_le(const T* v, int n, T x) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64, o = lane * step;
    const uint64_t le = __ballot(o == 0 || (o < n && v[lo + o] <= x));
    const int at = (63 - __clzll((long long)le)) * step;
    lo += at;
    n = step > 1 ? min(step, n - at) : 1;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// A tile (or a part of one): its request, KV head and rows, and its place on the line.
struct Tile {
  int r, t0, nt, len;    // request, its first token, tokens and keys
  int head, row0, rows;  // KV head; the tile's rows [row0, rows) within the request, at most ROWS
  uint32_t keys;         // its length
  uint64_t at;           // where it begins
  int k0, k1;            // the part: keys [k0, k1) of the tile, k1 < 0: to its end
  int slot;              // where the part's sums go, -1: it is the whole tile
};

// Length of the line and of a share.
struct Line {
  uint64_t end, share;
};
__device__ __forceinline__ Line line_of(uint64_t end) {
  const uint64_t s = ((end + kShares - 1) / kShares + kCut - 1) / kCut * kCut;
  return Line{end, max(s, (uint64_t)kMinShare)};
}

template <int ROWS, bool LIST>
__device__ __forceinline__ Line measure(const Attn4Args& a) {
  if constexpr (LIST) {
    return Line{a.R > 0 ? (uint64_t)a.T * a.hkv * a.row_tiles * a.list_parts * a.list_share : 0,
                (uint64_t)a.list_share};
  } else if (a.R > kInlineRequests) {
    return line_of(uniform64(a.sched[a.R]));
  } else {
    const int lane = threadIdx.x & 63;
    uint64_t n = 0;
    if (lane < a.R) {
      const Req q = load_req<ROWS>(a, lane);
      n = a.hkv * q.before(q.tiles);
    }
    return line_of(lane_bcast64(wave_prefix64(n), 63));
  }
}

// The tile that holds the place x < end of the line; wave-uniform.
template <int ROWS>
__device__ __forceinline__ Tile tile_at(const Attn4Args& a, uint64_t x) {
  Tile it;
  Req q{};
  uint64_t base;
  if (a.R <= kInlineRequests) {
    const int lane = threadIdx.x & 63;
    uint64_t n = 0;
    if (lane < a.R) {
      q = load_req<ROWS>(a, lane);
      n = a.hkv * q.before(q.tiles);
    }
    const uint64_t in = wave_prefix64(n);
    it.r = __ffsll((unsigned long long)__ballot(in > x)) - 1;
    base = lane_bcast64(in - n, it.r);
    q.t0 = lane_bcast(q.t0, it.r);
    q.nt = lane_bcast(q.nt, it.r);
    q.len = lane_bcast(q.len, it.r);
    q.tiles = lane_bcast(q.tiles, it.r);
    q.top = lane_bcast(q.top, it.r);
    q.slope = lane_bcast(q.slope, it.r);
  } else {
    it.r = last_le<uint64_t>(a.sched, a.R, x);
    base = uniform64(a.sched[it.r]);
    q = load_req<ROWS>(a, it.r);
    q.t0 = __builtin_amdgcn_readfirstlane(q.t0);
    q.nt = __builtin_amdgcn_readfirstlane(q.nt);
    q.len = __builtin_amdgcn_readfirstlane(q.len);
    q.tiles = __builtin_amdgcn_readfirstlane(q.tiles);
    q.top = __builtin_amdgcn_readfirstlane(q.top);
    q.slope = __builtin_amdgcn_readfirstlane(q.slope);
  }
  x -= base;
  // row tiles from the end of the request, each with all its heads
  uint32_t j = 0, n = (uint32_t)q.tiles;
  while (n > 1) {  // the last j with heads * before(j) <= x
    const uint32_t half = n / 2;
    if (a.hkv * q.before(j + half) <= x) {
      j += half;
      n -= half;
    } else {
      n = half;
    }
  }
  it.keys = q.keys(j);
  x -= a.hkv * q.before(j);
  it.head = (int)((uint32_t)(x / it.keys));
  it.at = base + a.hkv * q.before(j) + (uint64_t)it.head * it.keys;
  it.t0 = q.t0;
  it.nt = q.nt;
  it.len = q.len;
  it.row0 = (q.tiles - 1 - (int)j) * ROWS;
  it.rows = q.nt * a.group;
  return it;
}

// The same for list attention: every token, KV head and row tile has list_parts
// shares of its own. rows = 0: the token belongs to no request.
template <int ROWS>
__device__ __forceinline__ Tile list_tile_at(const Attn4Args& a, uint64_t x) {
  Tile it;
  it.keys = (uint32_t)(a.list_parts * a.list_share);
  const uint32_t tile = (uint32_t)(x / it.keys), per_tok = (uint32_t)(a.hkv * a.row_tiles);
  const int t = (int)(tile / per_tok), in = (int)(tile - t * per_tok);
  it.at = (uint64_t)tile * it.keys;
  it.r = last_le<int32_t>(a.cu, a.R, t);
  const int c0 = __builtin_amdgcn_readfirstlane(a.cu[it.r]), c1 = __builtin_amdgcn_readfirstlane(a.cu[it.r + 1]);
  it.t0 = c0;
  it.nt = min(c1, a.T) - c0;
  it.len = key_count(__builtin_amdgcn_readfirstlane(a.seq[it.r]));
  it.head = in / a.row_tiles;
  it.row0 = (t - c0) * a.group + (in - it.head * a.row_tiles) * ROWS;
  it.rows = t < c0 || t >= c1 ? 0 : (t - c0 + 1) * a.group;  // of this token
  return it;
}

template <int ROWS, bool LIST>
__device__ __forceinline__ Tile find(const Attn4Args& a, uint64_t x) {
  if constexpr (LIST) return list_tile_at<ROWS>(a, x);
  else return tile_at<ROWS>(a, x);
}

// The keys of a tile before a cut at the place x of the line.
template <int ROWS, bool LIST>
__device__ __forceinline__ int cut_in(const Tile& it, uint64_t x) {
  const uint64_t from = it.at + (LIST ? 0 : kStart<ROWS>);
  return x <= from ? 0 : (int)((uint32_t)(x - from) / kCut * kCut);
}

// The part of a tile that a share beginning at `begin` has from x on; returns
// where the next one begins. A part without keys is left out (false in `any`).
template <int ROWS, bool LIST>
__device__ __forceinline__ uint64_t take_part(Tile& it, uint64_t begin, uint64_t end, uint64_t x, int block,
                                              bool& any) {
  const uint64_t tile_end = it.at + it.keys, stop = min(end, tile_end);
  it.k0 = cut_in<ROWS, LIST>(it, x);
  it.k1 = stop == tile_end ? -1 : cut_in<ROWS, LIST>(it, stop);
  it.slot = it.k0 == 0 && it.k1 < 0 ? -1 : 2 * block + (x == begin ? 0 : 1);
  any = it.k1 < 0 || it.k0 < it.k1;
  return stop;
}

// Visible keys of the i-th token of a tile's request.
__device__ __forceinline__ RowRange token_range(const Attn4Args& a, const Tile& it, int i) {
  int e = a.end ? a.end[it.t0 + i] : it.len - it.nt + i + 1;
  e = min(max(e, 0), it.len);
  int s = a.start ? a.start[it.t0 + i] : 0;
  s = min(max(s, 0), e);
  return RowRange{s, e};
}

// What the rows of a tile see together: [lo, hi) holds every visible key,
// [smax, emin) the keys that all of them see.
struct Reach {
  int lo, hi, smax, emin;
};
template <int ROWS>
__device__ __forceinline__ Reach tile_reach(const Attn4Args& a, const Tile& it) {
  Reach r{0x7FFFFFFF, 0, 0, 0x7FFFFFFF};
  for (int x = it.row0 + (threadIdx.x & 63); x < min(it.row0 + ROWS, it.rows); x += 64) {
    const RowRange rr = token_range(a, it, x / a.group);
    if (rr.s < rr.e) {
      r.lo = min(r.lo, rr.s);
      r.hi = max(r.hi, rr.e);
    }
    r.smax = max(r.smax, rr.s);
    r.emin = min(r.emin, rr.e);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    r.lo = min(r.lo, __shfl_xor(r.lo, o));
    r.hi = max(r.hi, __shfl_xor(r.hi, o));
    r.smax = max(r.smax, __shfl_xor(r.smax, o));
    r.emin = min(r.emin, __shfl_xor(r.emin, o));
  }
  r.lo = __builtin_amdgcn_readfirstlane(min(r.lo, r.hi));
  r.hi = __builtin_amdgcn_readfirstlane(r.hi);
  r.smax = __builtin_amdgcn_readfirstlane(r.smax);
  r.emin = __builtin_amdgcn_readfirstlane(r.emin);
  return r;
}

// The places of a part, positions or entries of the token's list, and the keys
// that they name.
template <bool LIST>
struct Keys {
  const int32_t *list, *table;
  int base, lo, hi, k0, k1, head;
  __device__ __forceinline__ void init(const Attn4Args& a, const Tile& it, const Reach& r) {
    table = a.table + (int64_t)it.r * a.table_ld;
    head = it.head;
    lo = r.lo;
    hi = r.hi;
    list = nullptr;
    base = 0;
    if constexpr (LIST) {
      const int t = it.t0 + it.row0 / a.group;
      list = a.list + (int64_t)t * a.list_ld;
      base = a.list_base ? a.list_base[t] : 0;
      k0 = min(it.k0, a.list_k);
      k1 = lo == hi ? k0 : it.k1 < 0 ? a.list_k : min(it.k1, a.list_k);
    } else {
      k0 = min(lo + min(it.k0, hi - lo), hi);
      k1 = it.k1 < 0 ? hi : lo + min(it.k1, hi - lo);
    }
  }
  // Each lookup in two halves, so that a loop can keep its load in flight: the
  // load, at some entry that there is, and what its result says.
  __device__ __forceinline__ int fetch(const Attn4Args& a, int j) const {
    if constexpr (LIST) return list[min(j, a.list_k - 1)];
    else return 0;
  }
  // the position of place j, or -1
  __device__ __forceinline__ int position(int j, int raw) const {
    if constexpr (LIST) {
      const int64_t p = (int64_t)raw - base;
      return ((j < k1) & (p >= lo) & (p < hi)) ? (int)p : -1;
    } else {
      return j < k1 ? j : -1;
    }
  }
  __device__ __forceinline__ int look(const Attn4Args& a, int pos) const {
    return table[min(max(pos, 0) >> a.shift, max(a.table_width - 1, 0))];
  }
  // its page, or -1
  __device__ __forceinline__ int page(const Attn4Args& a, int pos, int raw) const {
    return ((pos >= 0) & ((pos >> a.shift) < a.table_width) & (raw < a.num_pages)) ? max(raw, -1) : -1;
  }
};

__device__ __forceinline__ float max_groups(float x) {  // over the four lanes of a column
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// A quarter (`part`) of one key's codes and of its value's, and the scales of both rows.
template <int D>
struct KeyRegs {
  uint32_t k[D / 32], v[D / 32];
  uint32_t ks, vs;  // scale bytes (D = 64: the key's and the value's in ks)
};

template <int D>
__device__ __forceinline__ void load_key(const Attn4Args& a, int page, int pos, int head, int part, KeyRegs<D>& x) {
  const int64_t row =
      page >= 0 ? (((int64_t)page * a.hkv + head) << a.shift) + (pos & ((1 << a.shift) - 1)) : 0;  // any row serves
  const uint8_t* c = a.codes + row * D + part * (D / 8);
  const uint8_t* s = a.scales + row * (D / 16);
  if constexpr (D == 128) {
    const uint4 k = *reinterpret_cast<const uint4*>(c), v = *reinterpret_cast<const uint4*>(c + D / 2);
    x.k[0] = k.x, x.k[1] = k.y, x.k[2] = k.z, x.k[3] = k.w;
    x.v[0] = v.x, x.v[1] = v.y, x.v[2] = v.z, x.v[3] = v.w;
    const uint2 w = *reinterpret_cast<const uint2*>(s);
    x.ks = w.x, x.vs = w.y;
  } else {
    const uint2 k = *reinterpret_cast<const uint2*>(c), v = *reinterpret_cast<const uint2*>(c + D / 2);
    x.k[0] = k.x, x.k[1] = k.y;
    x.v[0] = v.x, x.v[1] = v.y;
    x.ks = *reinterpret_cast<const uint32_t*>(s);
  }
}

// The exponents of a quarter of a key and of its value; 0 for a key that does
// not count, whose codes are then finite whatever they are.
template <int D>
__device__ __forceinline__ uint32_t key_byte(const KeyRegs<D>& x, int part, bool ok) {
  const uint32_t b = D == 128 ? x.ks >> (8 * part) : x.ks >> (8 * (part >> 1));
  return ok ? b & 255u : 0u;
}
template <int D>
__device__ __forceinline__ uint32_t value_byte(const KeyRegs<D>& x, int part, bool ok) {
  const uint32_t b = D == 128 ? x.vs >> (8 * part) : x.ks >> (16 + 8 * (part >> 1));
  return ok ? b & 255u : 0u;
}

// Rows of decoded keys (k_attn4_many) and values (k_attn4_few) in LDS, in bytes.
// The padding spreads 16 lanes that read 16 bytes of 16 key rows, and 32 that read 8
// bytes of 8 value rows in fours, over all banks. Conflicts are left, mostly by groups
// of lanes other than these: 39% of LDS's busy cycles in a decode batch.
template <int D>
constexpr int kKRow = 2 * D + 16;
template <int D>
constexpr int kVRow = 2 * D + 32;

// ---------------------------------------------------------------------------
// A column of rows: lane (c = lane % 16, g = lane / 16) holds row c's maximum
// m (and mc = m * scale), its share of the sum l and, as O^T tiles, the outputs
// 16 n + 4 g .. + 3. The products are taken as S^T = K Q^T and O^T = V^T P^T, so
// a lane's probabilities are already the operand of the second product.
// ---------------------------------------------------------------------------
template <int D>
struct Column {
  f32x4_t acc[D / 16];
  float m, mc, l;
  int s, e;  // the row's visible range; empty for no row
  bool row;

  __device__ __forceinline__ void init(const Attn4Args& a, const Tile& it, int x, bf16x8_t (&q)[D / 32], int stride,
                                       int step) {
    m = neg_inf();
    mc = l = 0.0f;
#pragma unroll
    for (int n = 0; n < D / 16; ++n) acc[n] = f32x4_t{};
    s = e = 0;
    row = x < it.rows;
    if (row) {
      const int i = x / a.group, h = it.head * a.group + (x - i * a.group), g = (threadIdx.x & 63) >> 4;
      const uint16_t* p = a.q + (int64_t)(it.t0 + i) * a.q_stride + (int64_t)h * D + g * stride;
#pragma unroll
      for (int n = 0; n < D / 32; ++n) q[n] = *reinterpret_cast<const bf16x8_t*>(p + n * step);
      const RowRange rr = token_range(a, it, i);
      s = rr.s;
      e = rr.e;
    } else {
#pragma unroll
      for (int n = 0; n < D / 32; ++n) q[n] = bf16x8_t{};
    }
  }

  // Scores of KT tiles of 16 keys, place j0 on, to probabilities. valid: a bit
  // a key, looked at (with the row's range) unless every row sees all of them.
  template <int KT, bool LIST>
  __device__ __forceinline__ void weigh(f32x4_t (&x)[KT], bool whole, uint64_t valid, int j0, float sc, float slack,
                                        bf16x8_t (&p)[KT / 2]) {
    const int g = (threadIdx.x & 63) >> 4;
    if (!whole) {
#pragma unroll
      for (int u = 0; u < KT; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int kk = 16 * u + 4 * g + i;
          bool v = (valid >> kk) & 1u;
          if constexpr (!LIST) v = v && j0 + kk >= s && j0 + kk < e;
          x[u][i] = v ? x[u][i] : neg_inf();
        }
    }
    float top = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3]));
#pragma unroll
    for (int u = 1; u < KT; ++u) top = fmaxf(top, fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3])));
    // the maximum is renewed only where it would grow by more than 2^8: the
    // sums keep their precision at any power of two
    if (__any(top > m + slack)) {
      const float mn = fmaxf(m, max_groups(top));
      const float nc = mn == neg_inf() ? 0.0f : mn * sc;
      const float f = m == neg_inf() ? 0.0f : exp2_fast(mc - nc);
      m = mn;
      mc = nc;
      l *= f;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) acc[n] *= f;
    }
#pragma unroll
    for (int u = 0; u < KT; ++u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[u][i] = exp2_fast(fmaf(x[u][i], sc, -mc));
      l += (x[u][0] + x[u][1]) + (x[u][2] + x[u][3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) p[u >> 1][4 * (u & 1) + i] = (__bf16)x[u][i];
    }
  }

  // Values that are not finite, into the rows that see them: bad has a bit for
  // each (quarter, key of 16) of the tile of keys at place j0.
  template <bool LIST>
  __device__ __forceinline__ void spoil(uint64_t bad, int j0) {
    while (bad) {
      const int from = __ffsll((unsigned long long)bad) - 1;
      bad &= bad - 1;
      const int j = j0 + (from & 15);
      if (row && (LIST || (j >= s && j < e))) {
#pragma unroll
        for (int n = 0; n < D / 16; ++n)
          if (n / (D / 64) == from >> 4) acc[n] += __builtin_nanf("");
      }
    }
  }

  // One row's result, or its part of it. M, L: the row's maximum (times scale) and sum.
  __device__ __forceinline__ void store(const Attn4Args& a, const Tile& it, int x, int rows_per_tile, float M,
                                        float L) const {
    if (!row) return;
    const int g = (threadIdx.x & 63) >> 4;
    if (it.slot < 0) {
      const int i = x / a.group, h = it.head * a.group + (x - i * a.group);
      const int64_t at = (int64_t)(it.t0 + i) * a.hkv * a.group + h;
      const float inv = L == 0.0f ? 0.0f : 1.0f / L;
      __bf16* o = reinterpret_cast<__bf16*>(a.out) + at * D + 4 * g;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        const f32x4_t y = acc[n] * inv;
        *reinterpret_cast<bf16x4_t*>(o + n * 16) = bf16x4_t{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
      }
      if (a.lse && g == 0) a.lse[at] = L == 0.0f ? neg_inf() : (M + __builtin_amdgcn_logf(L)) * kLn2;
    } else {
      const int64_t at = (int64_t)it.slot * rows_per_tile + (x - it.row0);
      f32x4_t* o = reinterpret_cast<f32x4_t*>(a.part_o + at * D) + g;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) o[n * 4] = acc[n];
      if (g == 0) a.part_ml[at] = float2{M, L};
    }
  }
};

// O^T += V^T P^T for 32 keys whose decoded values are in LDS rows at v.
template <int D, int RW>
__device__ __forceinline__ void add_values(const uint8_t* v, const bf16x8_t (&p)[RW], Column<D> (&col)[RW]) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const uint8_t* vr = v + (4 * g + (c >> 2)) * kVRow<D> + (c & 3) * 8;
#pragma unroll
  for (int n = 0; n < D / 16; ++n) {
    const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(vr + n * 32));
    const s16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(vr + 16 * kVRow<D> + n * 32));
    const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
    for (int w = 0; w < RW; ++w)
      col[w].acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[w], col[w].acc[n], 0, 0, 0);
  }
}

// Rows of tokens that belong to no request, those before cu[0] and from cu[R] on:
// zero, by all blocks of a launch.
template <int D>
__device__ __forceinline__ void clear_padding(const Attn4Args& a) {
  const int first = a.R > 0 ? min(max(a.cu[0], 0), a.T) : 0, used = a.R > 0 ? min(max(a.cu[a.R], first), a.T) : 0;
  const int heads = a.hkv * a.group, per = heads * D / 2, n = first + a.T - used;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int64_t t = i < first ? i : used + (i - first);
    uint32_t* o = reinterpret_cast<uint32_t*>(a.out) + t * per;
    for (int j = threadIdx.x; j < per; j += blockDim.x) o[j] = 0u;
    if (a.lse)
      for (int j = threadIdx.x; j < heads; j += blockDim.x) a.lse[t * heads + j] = neg_inf();
  }
}

// ---------------------------------------------------------------------------
// Up to 16 rows a tile: the four waves of a block share the chunk's keys, 32 at
// a time in turn, and join their sums at the end. Keys are decoded straight
// into the matrix operand; values pass through the wave's own LDS rows, whose
// transposing reads give the other operand. No barrier inside the loop.
//
// Bound by the cache's bytes where there are many (1.31 GB in 246 us, 5.3 TB/s) and
// by a chain of dependent loads (places, pages, codes) and two launches where there
// are few: one request of 4001 keys takes 15 us and 32 tokens with lists of 2048
// keys (10.2 MB) 20 us, the joins' 6 and 4 included.
// ---------------------------------------------------------------------------
template <int D, bool LIST>
__global__ __launch_bounds__(256, 2) void k_attn4_few(Attn4Args a) {
  constexpr int ROWS = 16, NI = D / 32, NT = D / 16;
  __shared__ __align__(16) uint8_t lds[4 * 32 * kVRow<D>];
  __shared__ float ml[4][2][ROWS];
  const int lane = threadIdx.x & 63, wave = wave_id(), c = lane & 15, g = lane >> 4;
  clear_padding<D>(a);
  const Line line = measure<ROWS, LIST>(a);
  const uint64_t begin = blockIdx.x * line.share, end = min(begin + line.share, line.end);
  for (uint64_t at = begin; at < end;) {
    Tile it = find<ROWS, LIST>(a, at);
    bool any;
    at = take_part<ROWS, LIST>(it, begin, end, at, blockIdx.x, any);
    if (!any || it.rows == 0) continue;
    const Reach reach = tile_reach<ROWS>(a, it);
    Keys<LIST> keys;
    keys.init(a, it, reach);

    // lane group g takes the dims [g D/4, (g + 1) D/4) of every key, 8 at a time
    bf16x8_t q[NI];
    Column<D> col[1];
    col[0].init(a, it, it.row0 + c, q, D / 4, 8);
    uint8_t* vrows = lds + wave * 32 * kVRow<D>;
    const int steps = (keys.k1 - keys.k0 + 31) / 32;

    // in flight: the codes of the next step, the pages of the one after, the places of a third
    KeyRegs<D> kv[2];
    int page0[2], pos1[2], raw1[2], raw2[2];
    auto at_step = [&](int s, int u) { return keys.k0 + s * 32 + u * 16 + c; };
    {
      int p0[2], r0[2], r1[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        r0[u] = keys.fetch(a, at_step(wave, u));
        r1[u] = keys.fetch(a, at_step(wave + 4, u));
        raw2[u] = keys.fetch(a, at_step(wave + 8, u));
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        p0[u] = keys.position(at_step(wave, u), r0[u]);
        pos1[u] = keys.position(at_step(wave + 4, u), r1[u]);
        r0[u] = keys.look(a, p0[u]);
        raw1[u] = keys.look(a, pos1[u]);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        page0[u] = keys.page(a, p0[u], r0[u]);
        load_key<D>(a, page0[u], p0[u], it.head, g, kv[u]);
      }
    }
    for (int s = wave; s < steps; s += 4) {
      const uint64_t valid = (__ballot(page0[0] >= 0) & 0xFFFFu) | (__ballot(page0[1] >= 0) & 0xFFFFu) << 16;
      const int j0 = keys.k0 + s * 32;
      bool whole = valid == 0xFFFFFFFFu;
      if constexpr (!LIST) whole = whole && j0 >= reach.smax && j0 + 32 <= reach.emin;
      uint64_t bad[2] = {0, 0};
      f32x4_t x[2] = {};
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float ks = __uint_as_float(key_byte<D>(kv[u], g, page0[u] >= 0) << 23);
        uint32_t vb = value_byte<D>(kv[u], g, page0[u] >= 0);
        // a value that is not finite must not reach rows that do not see it
        if (!whole) {
          bad[u] = __ballot(vb == 255u);
          if (vb == 255u) vb = 0u;
        }
        const float vs = __uint_as_float(vb << 23);
        uint8_t* w = vrows + (u * 16 + c) * kVRow<D> + g * (D / 2);
#pragma unroll
        for (int n = 0; n < NI; ++n) {
          x[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8(kv[u].k[n], ks), q[n], x[u], 0, 0, 0);
          *reinterpret_cast<bf16x8_t*>(w + 16 * n) = decode8(kv[u].v[n], vs);
        }
      }
      // loads come back in order: pages and places first, codes last
      int at[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        page0[u] = keys.page(a, pos1[u], raw1[u]);
        at[u] = pos1[u];
        pos1[u] = keys.position(at_step(s + 8, u), raw2[u]);
        raw1[u] = keys.look(a, pos1[u]);
        raw2[u] = keys.fetch(a, at_step(s + 12, u));
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) load_key<D>(a, page0[u], at[u], it.head, g, kv[u]);
      bf16x8_t p[1];
      col[0].template weigh<2, LIST>(x, whole, valid, j0, a.scale_log2, a.slack, p);
      __builtin_amdgcn_wave_barrier();
      add_values<D, 1>(vrows, p, col);
      __builtin_amdgcn_wave_barrier();
      col[0].template spoil<LIST>(bad[0], j0);
      col[0].template spoil<LIST>(bad[1], j0 + 16);
    }

    // join the four waves: maxima and sums first, then the outputs by halves
    __syncthreads();
    col[0].l = sum_groups(col[0].l);
    if (g == 0) {
      ml[wave][0][c] = col[0].m == neg_inf() ? neg_inf() : col[0].mc;
      ml[wave][1][c] = col[0].l;
    }
    __syncthreads();
    float M = neg_inf(), L = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) M = fmaxf(M, ml[i][0][c]);
    const float ref = M == neg_inf() ? 0.0f : M;
#pragma unroll
    for (int i = 0; i < 4; ++i) L += exp2_fast(ml[i][0][c] - ref) * ml[i][1][c];
    const float w = col[0].m == neg_inf() ? 0.0f : exp2_fast(col[0].mc - ref);
#pragma unroll
    for (int n = 0; n < NT; ++n) col[0].acc[n] *= w;
    f32x4_t* box = reinterpret_cast<f32x4_t*>(lds);  // [2][NT][64]
#pragma unroll
    for (int half = 2; half >= 1; half >>= 1) {
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int n = 0; n < NT; ++n) box[((wave - half) * NT + n) * 64 + lane] = col[0].acc[n];
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int n = 0; n < NT; ++n) col[0].acc[n] += box[(wave * NT + n) * 64 + lane];
      }
      __syncthreads();
    }
    if (wave == 0) col[0].store(a, it, it.row0 + c, ROWS, M, L);
  }
}

// ---------------------------------------------------------------------------
// Many rows a tile: WR waves hold 32 rows each, and with WK = 2 two waves share
// their rows and take half of a step's keys each. The block decodes a step's keys,
// 16 a wave, once into LDS (two buffers, one barrier a step): the decoding and the
// cache's bytes are spent once for all rows, and what is left is bound by the
// matrix products and the exponentials.
//
// Prefill of 4047 tokens of two requests at 9K to 20K keys (928 GFLOP) takes 925
// to 965 us, 1.0 PFLOP/s: a step of 64 keys keeps the matrix pipe, the vector ALU
// and LDS busy for 1.0 to 1.3K cycles each of about 2.4K, with two waves a SIMD to
// overlap them. Tiles of 256 rows would halve the decoding, but their registers
// spill (1978 us); one LDS buffer and more blocks a CU spill too (3.4 ms). 1000
// tokens with lists of 2048 keys and 64 heads (67 GFLOP) take 96 us with two waves
// a tile, 106 with four; the scattered reads do not bind there.
//
// 32 x 32 products: one occupies the matrix pipe for 32 cycles and the issue
// port for few, so up to six other instructions run beside it (16 x 16 ones
// leave room for two); measured with both in a loop of its own.
// ---------------------------------------------------------------------------

// 32 rows: lane (r = lane % 32, h = lane / 32) holds row r's maximum and sum as
// a Column does and the outputs 32 n + 8 (i / 4) + 4 h + i % 4.
template <int D>
struct Wide {
  f32x16_t acc[D / 32];
  float m, mc, l;
  int s, e;
  bool row;

  __device__ __forceinline__ void init(const Attn4Args& a, const Tile& it, int x, bf16x8_t (&q)[D / 16]) {
    m = neg_inf();
    mc = l = 0.0f;
#pragma unroll
    for (int n = 0; n < D / 32; ++n) acc[n] = f32x16_t{};
    s = e = 0;
    row = x < it.rows;
    if (row) {
      const int i = x / a.group, head = it.head * a.group + (x - i * a.group), h = (threadIdx.x & 63) >> 5;
      const uint16_t* p = a.q + (int64_t)(it.t0 + i) * a.q_stride + (int64_t)head * D + h * 8;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) q[n] = *reinterpret_cast<const bf16x8_t*>(p + n * 16);
      const RowRange rr = token_range(a, it, i);
      s = rr.s;
      e = rr.e;
    } else {
#pragma unroll
      for (int n = 0; n < D / 16; ++n) q[n] = bf16x8_t{};
    }
  }

  // The scores of 32 * KT keys from place j0 on become weights; see Column::weigh.
  template <int KT, bool LIST>
  __device__ __forceinline__ void mask(f32x16_t (&x)[KT], uint64_t valid, int j0) const {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int u = 0; u < KT; ++u) {
      const uint32_t bits = (uint32_t)(valid >> (32 * u)) >> (4 * h);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int kk = 8 * (i / 4) + i % 4, j = j0 + 32 * u + kk + 4 * h;
        bool v = (bits >> kk) & 1u;
        if constexpr (!LIST) v = v && j >= s && j < e;
        x[u][i] = v ? x[u][i] : neg_inf();
      }
    }
  }
  template <int KT>
  __device__ __forceinline__ void renew(const f32x16_t (&x)[KT], float sc, float slack) {
    float top = x[0][0];
#pragma unroll
    for (int u = 0; u < KT; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x[u][i]);
    if (__any(top > m + slack)) {
      const float mn = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
      const float nc = mn == neg_inf() ? 0.0f : mn * sc;
      const float f = m == neg_inf() ? 0.0f : exp2_fast(mc - nc);
      m = mn;
      mc = nc;
      l *= f;
#pragma unroll
      for (int n = 0; n < D / 32; ++n) acc[n] *= f;
    }
  }
  // weights of half a tile (16 keys): values 8 u .. 8 u + 7 of x
  __device__ __forceinline__ bf16x8_t weights(const f32x16_t& x, int u, float sc) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = exp2_fast(fmaf(x[8 * u + i], sc, -mc));
    l += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
    return bf16x8_t{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3],
                    (__bf16)y[4], (__bf16)y[5], (__bf16)y[6], (__bf16)y[7]};
  }

  // Values that are not finite, into the rows that see them: bad has the bit 4 k + quarter for each of 16 keys.
  template <bool LIST>
  __device__ __forceinline__ void spoil(uint64_t bad, int j0) {
    while (bad) {
      const int from = __ffsll((unsigned long long)bad) - 1;
      bad &= bad - 1;
      const int j = j0 + (from >> 2);
      if (row && (LIST || (j >= s && j < e))) {
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if ((D == 128 ? n : 2 * n + i / 8) == (from & 3)) acc[n][i] += __builtin_nanf("");
      }
    }
  }

  __device__ __forceinline__ void store(const Attn4Args& a, const Tile& it, int x, int rows_per_tile, float M,
                                        float L) const {
    if (!row) return;
    const int h = (threadIdx.x & 63) >> 5;
    if (it.slot < 0) {
      const int i = x / a.group, head = it.head * a.group + (x - i * a.group);
      const int64_t at = (int64_t)(it.t0 + i) * a.hkv * a.group + head;
      const float inv = L == 0.0f ? 0.0f : 1.0f / L;
      __bf16* o = reinterpret_cast<__bf16*>(a.out) + at * D + 4 * h;
#pragma unroll
      for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          *reinterpret_cast<bf16x4_t*>(o + n * 32 + b * 8) =
              bf16x4_t{(__bf16)(acc[n][4 * b] * inv), (__bf16)(acc[n][4 * b + 1] * inv),
                       (__bf16)(acc[n][4 * b + 2] * inv), (__bf16)(acc[n][4 * b + 3] * inv)};
      if (a.lse && h == 0) a.lse[at] = L == 0.0f ? neg_inf() : (M + __builtin_amdgcn_logf(L)) * kLn2;
    } else {
      const int64_t at = (int64_t)it.slot * rows_per_tile + (x - it.row0);
      float* o = a.part_o + at * D + 4 * h;
#pragma unroll
      for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          *reinterpret_cast<f32x4_t*>(o + n * 32 + b * 8) =
              f32x4_t{acc[n][4 * b], acc[n][4 * b + 1], acc[n][4 * b + 2], acc[n][4 * b + 3]};
      if (h == 0) a.part_ml[at] = float2{M, L};
    }
  }
};

// Decoded values in LDS: rows of 2 D bytes whose 16-byte chunks are permuted by
// the key, chunk ^ swizzle(key). It spreads sixteen lanes that write a chunk of four
// keys' quarters, and 32 that read 64 bytes of four keys, over all banks; conflicts
// still are 24% of LDS's busy cycles in a prefill and 32% with lists.
template <int D>
__device__ __forceinline__ int swizzle(int key) {
  return D == 128 ? 5 * (key & 3) : 5 * ((key >> 1) & 1);
}

template <int N>
struct Int {
  static constexpr int value = N;
};

template <int D, int WR, int WK, bool LIST>
__global__ __launch_bounds__(64 * WR * WK, 2) void k_attn4_many(Attn4Args a) {
  constexpr int ROWS = 32 * WR, NK = D / 16, NV = D / 32, WAVES = WR * WK, KEYS = 16 * WAVES, KT = WR / 2;
  constexpr int kBuf = KEYS * (kKRow<D> + 2 * D);
  extern __shared__ __align__(16) uint8_t lds[];  // two buffers of decoded keys, then values
  __shared__ uint64_t bad_of[2][WAVES];           // per 16 keys: quarters of values that are not finite
  __shared__ uint32_t valid_of[2][WAVES];         // per 16 keys: those that count; bit 16: bad_of is not 0
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id(), r = lane & 31, h = lane >> 5;
  const int wr = wave / WK, wk = wave % WK;  // the wave's rows, its keys of a step
  clear_padding<D>(a);
  const Line line = measure<ROWS, LIST>(a);
  const uint64_t begin = blockIdx.x * line.share, end = min(begin + line.share, line.end);
  for (uint64_t at = begin; at < end;) {
    Tile it = find<ROWS, LIST>(a, at);
    bool any;
    at = take_part<ROWS, LIST>(it, begin, end, at, blockIdx.x, any);
    if (!any || it.rows == 0) continue;
    const Reach reach = tile_reach<ROWS>(a, it);
    Keys<LIST> keys;
    keys.init(a, it, reach);

    bf16x8_t q[NK];
    Wide<D> col;
    col.init(a, it, it.row0 + wr * 32 + r, q);
    // what all of this wave's rows see
    int smax = col.row ? col.s : 0, emin = col.row ? col.e : 0x7FFFFFFF;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      smax = max(smax, __shfl_xor(smax, o));
      emin = min(emin, __shfl_xor(emin, o));
    }
    smax = __builtin_amdgcn_readfirstlane(smax);
    emin = __builtin_amdgcn_readfirstlane(emin);

    // the loading side: four threads a key
    const int part = tid & 3, mine = tid >> 2;
    const int steps = (keys.k1 - keys.k0 + KEYS - 1) / KEYS;
    const int kw = mine * kKRow<D> + part * (D / 2);
    const int vw = KEYS * kKRow<D> + mine * 2 * D + ((part * (D / 32)) ^ swizzle<D>(mine)) * 16;
    // in flight: the codes of kAhead steps, the pages of one more, the places of a
    // second. Listed keys lie anywhere: two steps ahead.
    constexpr int kAhead = LIST ? 2 : 1;
    KeyRegs<D> kvs[kAhead];
    int page[kAhead], pos1, raw1, raw2;
    auto at_step = [&](int s) { return keys.k0 + s * KEYS + mine; };
    {
      int p[kAhead + 1], raw[kAhead + 1];
#pragma unroll
      for (int i = 0; i <= kAhead; ++i) raw[i] = keys.fetch(a, at_step(i));
      raw2 = keys.fetch(a, at_step(kAhead + 1));
#pragma unroll
      for (int i = 0; i <= kAhead; ++i) {
        p[i] = keys.position(at_step(i), raw[i]);
        raw[i] = keys.look(a, p[i]);
      }
      pos1 = p[kAhead];
      raw1 = raw[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        page[i] = keys.page(a, p[i], raw[i]);
        load_key<D>(a, page[i], p[i], it.head, part, kvs[i]);
      }
    }
    auto stage = [&](int s, auto bc) {  // decode step s into buffer b, start loading step s + kAhead
      constexpr int b = decltype(bc)::value, c = b % kAhead;
      KeyRegs<D>& kv = kvs[c];
      // loads come back in order: the next page and place are asked for before
      // the codes, so that waiting for them does not wait for those
      const int now = keys.page(a, pos1, raw1), at = pos1;
      pos1 = keys.position(at_step(s + kAhead + 1), raw2);
      raw1 = keys.look(a, pos1);
      raw2 = keys.fetch(a, at_step(s + kAhead + 2));
      const bool ok = page[c] >= 0;
      const float ks = __uint_as_float(key_byte<D>(kv, part, ok) << 23);
      uint32_t vb = value_byte<D>(kv, part, ok);
      const int j0 = keys.k0 + s * KEYS;
      const uint64_t oks = __ballot(ok);
      bool whole = oks == ~0ull;
      if constexpr (!LIST) whole = whole & (j0 >= reach.smax) & (j0 + KEYS <= reach.emin);
      // a value that is not finite must not reach rows that do not see it
      const bool drop = !whole & (vb == 255u);
      const uint64_t bad = __ballot(drop);
      vb = drop ? 0u : vb;
      bad_of[b][wave] = bad;  // wave-uniform, no branch
      uint64_t v = oks & 0x1111111111111111ull;  // a key's four threads agree
      v = (v | v >> 3) & 0x0303030303030303ull;
      v = (v | v >> 6) & 0x000F000F000F000Full;
      v = (v | v >> 12) & 0x000000FF000000FFull;
      valid_of[b][wave] = ((uint32_t)(v | v >> 24) & 0xFFFFu) | (bad ? 0x10000u : 0u);
      const float vs = __uint_as_float(vb << 23);
      uint8_t* buf = lds + b * kBuf;
#pragma unroll
      for (int n = 0; n < D / 32; ++n) {
        *reinterpret_cast<bf16x8_t*>(buf + kw + 16 * n) = decode8(kv.k[n], ks);
        *reinterpret_cast<bf16x8_t*>(buf + (vw ^ (16 * n))) = decode8(kv.v[n], vs);
      }
      page[c] = now;
      load_key<D>(a, now, at, it.head, part, kv);
    };

    // the reading side: a key's row of 16 dims, and 8 bytes of a value's chunk
    const int kr = (wk * 32 + r) * kKRow<D> + h * 16;
    const int vk = 4 * h + ((lane & 15) >> 2);  // key of a lane's transposing read
    int vr[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n)
      vr[n] = KEYS * kKRow<D> + (wk * 32 + vk) * 2 * D +
              ((4 * n + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ swizzle<D>(vk)) * 16 + (lane & 1) * 8;

    auto work = [&](int s, auto bc) {
      constexpr int b = decltype(bc)::value;
      const int j0 = keys.k0 + s * KEYS + wk * 32;
      // The decoding of the next step runs beside the first products, the weights
      // of each 16 keys beside the second products of the 16 before. A wave in its
      // first products goes before one that weighs (prefill 975 -> 950 us).
      // (Rows or keys that there are not take part like any other: a branch around
      // them would make every path wait for all loads in flight.)
      const uint8_t* buf = lds + b * kBuf;
      __builtin_amdgcn_s_setprio(1);
      f32x16_t x[KT];
#pragma unroll
      for (int u = 0; u < KT; ++u) x[u] = f32x16_t{};
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int u = 0; u < KT; ++u) {
          const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(buf + kr + u * 32 * kKRow<D> + n * 32);
          x[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[n], x[u], 0, 0, 0);
        }
      stage(s + 1, Int<b ^ 1>{});  // past the last step: keys that do not count
      uint64_t valid = 0;
      uint32_t any_bad = 0;
#pragma unroll
      for (int u = 0; u < 2 * KT; ++u) {
        const uint32_t v = valid_of[b][2 * wk + u];
        valid |= (uint64_t)(v & 0xFFFFu) << (16 * u);
        any_bad |= v >> 16;
      }
      bool whole = valid == (KT == 1 ? 0xFFFFFFFFull : ~0ull);
      if constexpr (!LIST) whole = whole & (j0 >= smax) & (j0 + 32 * KT <= emin);
      if (!whole) {
        asm volatile("");  // a branch, not selects: most steps need no mask
        col.template mask<KT, LIST>(x, valid, j0);
      }
      __builtin_amdgcn_s_setprio(0);
      col.template renew<KT>(x, a.scale_log2, a.slack);
      bf16x8_t p = col.weights(x[0], 0, a.scale_log2);
#pragma unroll
      for (int u = 0; u < 2 * KT; ++u) {
        bf16x8_t next;
        if (u + 1 < 2 * KT) next = col.weights(x[(u + 1) >> 1], (u + 1) & 1, a.scale_log2);
#pragma unroll
        for (int n = 0; n < NV; ++n) {
          const uint8_t* v = buf + vr[n] + u * 16 * 2 * D;
          const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)v);
          const s16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(v + 8 * 2 * D));
          const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
          col.acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p, col.acc[n], 0, 0, 0);
        }
        p = next;
      }
      if (any_bad) {
#pragma unroll 1
        for (int u = 0; u < 2 * KT; ++u) {
          const uint64_t bad = bad_of[b][2 * wk + u];
          col.template spoil<LIST>(bad, j0 + 16 * u);
        }
      }
      __syncthreads();
    };
    stage(0, Int<0>{});
    __syncthreads();
    int s = 0;
    for (; s + 1 < steps; s += 2) {
      work(s, Int<0>{});
      work(s + 1, Int<1>{});
    }
    if (s < steps) work(s, Int<0>{});
    float L = col.l + __shfl_xor(col.l, 32), M = col.m == neg_inf() ? neg_inf() : col.mc;
    if constexpr (WK == 2) {
      // the two waves of the same rows
      f32x4_t* box = reinterpret_cast<f32x4_t*>(lds) + wr * (4 * NV * 64 + 32);
      float2* ml = reinterpret_cast<float2*>(box + 4 * NV * 64);
      if (wk == 1) {
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            box[(4 * n + i) * 64 + lane] =
                f32x4_t{col.acc[n][4 * i], col.acc[n][4 * i + 1], col.acc[n][4 * i + 2], col.acc[n][4 * i + 3]};
        if (h == 0) ml[r] = float2{M, L};
      }
      __syncthreads();
      if (wk == 0) {
        const float2 o = ml[r];
        const float top = fmaxf(M, o.x), ref = top == neg_inf() ? 0.0f : top;
        const float f0 = exp2_fast(M - ref), f1 = exp2_fast(o.x - ref);
        M = top;
        L = L * f0 + o.y * f1;
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            col.acc[n][i] = col.acc[n][i] * f0 + box[(4 * n + i / 4) * 64 + lane][i % 4] * f1;
      }
    }
    if (wk == 0) col.store(a, it, it.row0 + wr * 32 + r, ROWS, M, L);
    __syncthreads();  // the buffers are free again
  }
}

// Joins the parts of a tile, by the block of the first cut inside it: parts c =
// b - 1, b, ... of the shares that reach into it. A thread takes four outputs of
// a row, a block 1024 / D rows at a time. Its time is that of waiting for loads:
// sixteen parts' in flight, and eight for lists and wide tiles, which mostly have few
// parts (one request of 4001 keys, 35 parts a tile: both kernels 15.2 us, with eight
// 16.4; 128K keys, 64 parts: 38.9 and 41.4; 32 lists of 4 parts: 21.6 and 20.0; the
// join of a prefill of two requests 44 and 25).
template <int D, int ROWS, bool LIST>
__global__ __launch_bounds__(256) void k_attn4_join(Attn4Args a) {
  constexpr int kRowThreads = D / 4, kAtOnce = 256 / kRowThreads, kParts = !LIST && ROWS == 16 ? 16 : 8;
  const Line line = measure<ROWS, LIST>(a);
  const int b = blockIdx.x + 1;
  const uint64_t cut = b * line.share, before = cut - line.share;
  if (cut >= line.end) return;
  const Tile it = find<ROWS, LIST>(a, cut);
  if (it.rows == 0 || cut_in<ROWS, LIST>(it, cut) == 0 || cut_in<ROWS, LIST>(it, before) > 0) return;
  const int parts = 1 + (int)((it.at + it.keys - cut + line.share - 1) / line.share);
  const int slot0 = 2 * (b - 1) + (it.at > before ? 1 : 0);
  const int c = threadIdx.x % kRowThreads;
  const int n = min(ROWS, it.rows - it.row0);
  for (int in = blockIdx.y * kAtOnce + threadIdx.x / kRowThreads; in < n; in += gridDim.y * kAtOnce) {
    float M = neg_inf(), L = 0.0f;
    f32x4_t o = {};
    for (int i0 = 0; i0 < parts; i0 += kParts) {
      float2 w[kParts];
      f32x4_t v[kParts];
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        const int i = min(i0 + u, parts - 1);
        const int64_t row = (int64_t)(i == 0 ? slot0 : 2 * (b - 1 + i)) * ROWS + in;
        w[u] = a.part_ml[row];
        v[u] = reinterpret_cast<const f32x4_t*>(a.part_o)[row * kRowThreads + c];
      }
      float top = M;
#pragma unroll
      for (int u = 0; u < kParts; ++u) top = fmaxf(top, w[u].x);
      const float ref = top == neg_inf() ? 0.0f : top, f = exp2_fast(M - ref);
      M = top;
      L *= f;
      o *= f;
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        const float g = exp2_fast(w[u].x - ref);
        if (i0 + u < parts) {
          L = fmaf(g, w[u].y, L);
          o += g * v[u];
        }
      }
    }
    const int x = it.row0 + in, i = x / a.group, h = it.head * a.group + (x - i * a.group);
    const int64_t row = (int64_t)(it.t0 + i) * a.hkv * a.group + h;
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    o *= inv;
    reinterpret_cast<bf16x4_t*>(reinterpret_cast<__bf16*>(a.out) + row * D)[c] =
        bf16x4_t{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
    if (a.lse && c == 0) a.lse[row] = L == 0.0f ? neg_inf() : (M + __builtin_amdgcn_logf(L)) * kLn2;
  }
}

template <int D, int WR, int WK, bool LIST>
hipError_t run_many(const Attn4Args& a, dim3 grid, hipStream_t st) {
  constexpr size_t lds = 2 * 16 * WR * WK * (kKRow<D> + 2 * D);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_attn4_many<D, WR, WK, LIST>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  k_attn4_many<D, WR, WK, LIST><<<grid, 64 * WR * WK, lds, st>>>(a);
  return hipSuccess;
}

// Blocks of the first launch: a share of the line each.
int64_t blocks_of(const Attn4Args& a) {
  return a.list_k > 0 ? (int64_t)a.T * a.hkv * a.row_tiles * a.list_parts : kShares;
}

template <int D, int ROWS, bool LIST>
hipError_t run(const Attn4Args& a, hipStream_t st) {
  if (!LIST && a.R > kInlineRequests) k_attn4_schedule<ROWS><<<1, 1024, 0, st>>>(a);
  const unsigned shares = (unsigned)blocks_of(a);
  const dim3 grid(shares);
  if constexpr (ROWS == 16) {
    k_attn4_few<D, LIST><<<grid, 256, 0, st>>>(a);
  } else {
    hipError_t e;
    if constexpr (ROWS == 128) {
      e = run_many<D, 4, 1, LIST>(a, grid, st);
    } else if constexpr (LIST) {
      // Four waves a tile, 512 tiles at once, or two, 1024 at once, which has fewer
      // starts: the rounds of lists of 2048 keys take 9 and 5. Two and four waves, us:
      // 2048 keys, 512 tokens 78 and 57, 1000 98 and 105, 1500 164 and 156, 2000 189
      // and 203; 1000 keys, the same tokens 45 and 34, 54 and 63, 93 and 91, 108 and
      // 117; 256 keys 19 and 18, 26 and 33, 40 and 45, 56 and 58. So shorter lists lose
      // up to 20% where the rule takes four waves for a third half-filled round.
      const int64_t tiles = grid.x;
      e = 9 * ((tiles + 1023) / 1024) <= 5 * ((tiles + 511) / 512) ? run_many<D, 2, 1, LIST>(a, grid, st)
                                                                   : run_many<D, 2, 2, LIST>(a, grid, st);
    } else {
      e = run_many<D, 2, 2, LIST>(a, grid, st);
    }
    if (e != hipSuccess) return e;
  }
  if constexpr (!LIST || ROWS == 16) {  // wide list tiles have one part
    if (!LIST || a.list_parts > 1)
      k_attn4_join<D, ROWS, LIST><<<dim3(shares - 1, ROWS == 16 ? 2 : ROWS / 32), 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

template <int D, bool LIST>
hipError_t run_rows(const Attn4Args& a, hipStream_t st) {
  if (a.rows_per_tile == 16) return run<D, 16, LIST>(a, st);
  if (a.rows_per_tile == 64) return run<D, 64, LIST>(a, st);
  return run<D, 128, LIST>(a, st);
}

// Rows of a dense tile, for a request's mean of rows.
int tile_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 64 ? 64 : 128; }

// What depends on host values alone: the rows of a tile, and for lists, which are
// all as long, the parts of a tile: none but where there are too few tiles.
void shape_of(Attn4Args& a) {
  const int64_t rows = a.list_k > 0 ? a.group : ((int64_t)a.T * a.group + a.R - 1) / (a.R > 0 ? a.R : 1);
  a.rows_per_tile = tile_rows(rows);
  if (a.list_k == 0) return;
  // Few tokens: more, narrower tiles. Narrow and wide (of one part), lists of 2048 keys,
  // us: 64 heads, 64 tokens 25 and 42, 128 33 and 43, 192 50 and 44, 256 61 and 45, 512
  // 108 and 55; 32 heads, 128 25 and 42, 256 31 and 42, 320 48 and 51, 512 58 and 52. Of
  // 256 keys, 64 heads: 64 tokens 9 and 12, 128 12 and 13, 192 18 and 13, 256 20 and 13.
  // The line fits neither group exactly: 64 heads lose up to 15 us from 160 tokens on,
  // 32 heads up to 11 from 256 to 320.
  if ((int64_t)a.T * a.hkv < 256) a.rows_per_tile = 16;
  a.row_tiles = (a.group + a.rows_per_tile - 1) / a.rows_per_tile;
  const int64_t tiles = (int64_t)a.T * a.hkv * a.row_tiles, most = ((int64_t)a.list_k + kMinShare - 1) / kMinShare;
  const int64_t parts = tiles >= 256 || tiles == 0 ? 1 : std::min(512 / tiles, most);
  a.list_share = (int)((((int64_t)a.list_k + parts - 1) / parts + kCut - 1) / kCut * kCut);
  a.list_parts = (int)(((int64_t)a.list_k + a.list_share - 1) / a.list_share);
}

// Rows of parts that may have to be kept, as many as a call of no more tokens and
// requests may need, so that a larger call's workspace serves a smaller. Dense: the
// same tokens in one request have the widest tiles. Lists: only narrow tiles have
// parts, 512 at most.
size_t kept_rows(const Attn4Args& a) {
  return 2 * (size_t)kShares * (a.list_k > 0 ? 16 : tile_rows((int64_t)a.T * a.group));
}

}  // namespace

int64_t attn4_blocks(const Attn4Args& args) {
  Attn4Args a = args;
  shape_of(a);
  return blocks_of(a);
}

size_t attn4_workspace_bytes(const Attn4Args& a) {
  return 256 + (((size_t)a.R + 1) * 8 + 255) / 256 * 256 +
         kept_rows(a) * ((size_t)a.d * 4 + 8);
}

hipError_t launch_attn4(Attn4Args a, void* workspace, hipStream_t st) {
  shape_of(a);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.sched = reinterpret_cast<uint64_t*>(ws);
  ws += (((size_t)a.R + 1) * 8 + 255) / 256 * 256;
  a.part_o = reinterpret_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(ws + kept_rows(a) * a.d * 4);
  a.slack = 8.0f / a.scale_log2;
  if (!(a.slack < 1e30f)) a.slack = 1e30f;
  if (a.list_k > 0) return a.d == 128 ? run_rows<128, true>(a, st) : run_rows<64, true>(a, st);
  return a.d == 128 ? run_rows<128, false>(a, st) : run_rows<64, false>(a, st);
}

}  // namespace lt
