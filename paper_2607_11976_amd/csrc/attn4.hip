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
// to 16 * RT rows of one request; its key range is cut into chunks so that the
// work of all tiles, long and short, fills the GPU evenly; chunks of a tile
// are joined by a second kernel.
#include "cache4.hpp"
#include "internal.hpp"

namespace lt {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;

constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kInlineRequests = 64;  // requests that a wave schedules by itself
constexpr int kMinChunk = 128;       // shortest chunk: one step of 32 keys for each wave

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ uint32_t lane_bcast(uint32_t v, int lane) {
  return (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// ---------------------------------------------------------------------------
// Schedule. Request r has tiles_r = heads * ceil(rows_r / ROWS) tiles over
// about span_r keys; with a chunk length C it makes tiles_r * ceil(span_r / C)
// items, and C = sum tiles_r * span_r / target keeps the items within
// target + tiles. span_r only balances: a tile's last chunk takes what is left.
// ---------------------------------------------------------------------------
struct Req {
  int t0, nt, len, tiles;  // first token, tokens, cached keys, tiles
  uint32_t span;
};

template <int ROWS>
__device__ __forceinline__ Req load_req(const Attn4Args& a, int r) {
  Req q;
  const int t0 = min(max(a.cu[r], 0), a.T), t1 = min(max(a.cu[r + 1], t0), a.T);
  q.t0 = t0;
  q.nt = t1 - t0;
  q.len = max(a.seq[r], 0);
  q.tiles = q.nt > 0 ? a.hkv * (int)(((int64_t)q.nt * a.group + ROWS - 1) / ROWS) : 0;
  int lo = 0, hi = q.len;
  if (q.nt > 0 && a.end) hi = min(max(a.end[t1 - 1], 0), hi);
  if (q.nt > 0 && a.start) lo = min(max(a.start[t0], 0), hi);
  q.span = (uint32_t)max(hi - lo, 1);
  return q;
}

__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)v, o), hi = (uint32_t)__shfl_xor((int)(v >> 32), o);
    v += ((uint64_t)hi << 32) | lo;
  }
  return v;
}
__device__ __forceinline__ uint32_t wave_prefix(uint32_t v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = (uint32_t)__shfl_up((int)v, o);
    if (lane >= o) v += u;
  }
  return v;
}

__device__ __forceinline__ uint32_t chunk_len(uint64_t work, int target) {
  const uint64_t c = (work + target - 1) / target;
  const uint64_t r = (c + kMinChunk - 1) / kMinChunk * kMinChunk;
  return r < kMinChunk ? kMinChunk : r > 0x40000000u ? 0x40000000u : (uint32_t)r;
}

struct Item {
  int r, t0, nt, len;       // request, its first token, tokens and keys
  int head, row0;           // KV head; first row of the tile within the request
  int chunk, chunks;
  uint32_t C;
  bool any;
};

// The schedule of more than kInlineRequests requests: the items' prefix sums
// sched[0..R] and the chunk length sched[R + 1].
template <int ROWS>
__global__ __launch_bounds__(1024) void k_attn4_schedule(Attn4Args a) {
  __shared__ uint64_t sum[16];
  __shared__ uint32_t part[16];
  const int t = threadIdx.x, w = t >> 6, lane = t & 63;
  uint64_t work = 0;
  for (int r = t; r < a.R; r += 1024) {
    const Req q = load_req<ROWS>(a, r);
    work += (uint64_t)q.tiles * q.span;
  }
  work = wave_sum64(work);
  if (lane == 0) sum[w] = work;
  __syncthreads();
  work = 0;
  for (int i = 0; i < 16; ++i) work += sum[i];
  const uint32_t C = a.target > 0 ? chunk_len(work, a.target) : 0x80000000u;
  uint32_t base = 0;
  for (int r0 = 0; r0 < a.R; r0 += 1024) {
    const int r = r0 + t;
    uint32_t n = 0;
    if (r < a.R) {
      const Req q = load_req<ROWS>(a, r);
      n = (uint32_t)q.tiles * ((q.span + C - 1) / C);
    }
    const uint32_t in = wave_prefix(n);
    __syncthreads();
    if (lane == 63) part[w] = in;
    __syncthreads();
    uint32_t before = base, all = base;
    for (int i = 0; i < 16; ++i) {
      if (i < w) before += part[i];
      all += part[i];
    }
    if (r < a.R) a.sched[r] = before + in - n;
    base = all;
  }
  if (t == 0) {
    a.sched[a.R] = base;
    a.sched[a.R + 1] = C;
  }
}

// The item a block works on; wave-uniform.
template <int ROWS>
__device__ __forceinline__ Item find_item(const Attn4Args& a, uint32_t item) {
  const int lane = threadIdx.x & 63;
  Item it{};
  Req q{};
  uint32_t first = 0;
  if (a.R <= kInlineRequests) {
    if (lane < a.R) q = load_req<ROWS>(a, lane);
    it.C = a.target > 0 ? chunk_len(wave_sum64((uint64_t)q.tiles * q.span), a.target) : 0x80000000u;
    const uint32_t n = lane < a.R ? (uint32_t)q.tiles * ((q.span + it.C - 1) / it.C) : 0u;
    const uint32_t in = wave_prefix(n);
    const uint64_t hit = __ballot(in > item);
    if (!hit) return it;
    it.r = __ffsll((unsigned long long)hit) - 1;
    first = lane_bcast(in - n, it.r);
    q.t0 = lane_bcast(q.t0, it.r);
    q.nt = lane_bcast(q.nt, it.r);
    q.len = lane_bcast(q.len, it.r);
    q.tiles = lane_bcast(q.tiles, it.r);
    q.span = lane_bcast(q.span, it.r);
  } else {
    if (item >= a.sched[a.R]) return it;
    it.C = a.sched[a.R + 1];
    // last r with sched[r] <= item, 64 at a time (sched[0] = 0)
    int lo = 0, n = a.R;
    while (n > 0) {
      const int step = (n + 63) / 64, r = lo + lane * step;
      const uint64_t le = __ballot(lane * step < n && a.sched[min(r, a.R)] <= item);
      lo += (63 - __clzll((long long)le)) * step;
      n = step > 1 ? min(step, a.R - lo) : 0;
    }
    it.r = __builtin_amdgcn_readfirstlane(lo);
    first = a.sched[it.r];
    q = load_req<ROWS>(a, it.r);
  }
  it.any = true;
  it.t0 = __builtin_amdgcn_readfirstlane(q.t0);
  it.nt = __builtin_amdgcn_readfirstlane(q.nt);
  it.len = __builtin_amdgcn_readfirstlane(q.len);
  it.chunks = (int)((q.span + it.C - 1) / it.C);
  const uint32_t at = item - first, tile = at / (uint32_t)it.chunks;
  it.chunk = (int)(at - tile * it.chunks);
  const int per_head = q.tiles / a.hkv;
  it.head = (int)tile / per_head;
  it.row0 = ((int)tile - it.head * per_head) * ROWS;
  return it;
}

// Items of list attention: every token of the batch, KV head and row tile over
// a.chunks chunks of the list.
template <int ROWS>
__device__ __forceinline__ Item find_list_item(const Attn4Args& a, uint32_t item) {
  const int lane = threadIdx.x & 63;
  Item it{};
  if (a.R == 0) return it;
  const uint32_t per_tok = (uint32_t)(a.hkv * a.row_tiles * a.chunks);
  const int t = (int)(item / per_tok);
  const uint32_t in = item - t * per_tok;
  // the request whose tokens hold t: the last r with cu[r] <= t
  int lo = 0, n = a.R;
  while (n > 0) {
    const int step = (n + 63) / 64, r = lo + lane * step;
    const uint64_t le = __ballot(lane * step < n && (r == 0 || a.cu[min(r, a.R)] <= t));
    lo += (63 - __clzll((long long)le)) * step;
    n = step > 1 ? min(step, a.R - lo) : 0;
  }
  it.r = __builtin_amdgcn_readfirstlane(lo);
  const int c0 = a.cu[it.r], c1 = a.cu[it.r + 1];
  if (t < c0 || t >= c1) return it;
  it.any = true;
  it.t0 = c0;
  it.nt = min(c1, a.T) - c0;
  it.len = max(a.seq[it.r], 0);
  it.chunks = a.chunks;
  it.chunk = (int)(in % (uint32_t)a.chunks);
  const uint32_t tile = in / (uint32_t)a.chunks;
  it.head = (int)tile / a.row_tiles;
  it.row0 = (t - c0) * a.group + ((int)tile - it.head * a.row_tiles) * ROWS;
  it.C = (uint32_t)a.chunk_keys;
  return it;
}

// Visible keys of token t (the i-th of its request).
__device__ __forceinline__ RowRange token_range(const Attn4Args& a, const Item& it, int i) {
  int e = a.end ? a.end[it.t0 + i] : it.len - it.nt + i + 1;
  e = min(max(e, 0), it.len);
  int s = a.start ? a.start[it.t0 + i] : 0;
  s = min(max(s, 0), e);
  return RowRange{s, e};
}

__device__ __forceinline__ float max_groups(float x) {  // over the four lanes of a column
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// The codes and scales of a lane's part of one key and its value.
template <int D>
struct KeyRegs {
  uint32_t k[D / 32], v[D / 32];
  uint32_t ks, vs;  // the row's scale bytes (D = 64: the key's and the value's in ks)
};

// Lane (c = lane % 16, g = lane / 16) takes dims [g D/4, (g + 1) D/4) of key c.
template <int D>
__device__ __forceinline__ void load_key(const Attn4Args& a, int page, int pos, int head, bool ok, KeyRegs<D>& x) {
  const int g = (threadIdx.x & 63) >> 4;
  const int64_t row =
      ok ? (((int64_t)page * a.hkv + head) << a.shift) + (pos & ((1 << a.shift) - 1)) : 0;  // any row serves
  const uint8_t* c = a.codes + row * D + g * (D / 8);
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

// The exponents of a lane's part of a key and of its value; 0 for a key that
// does not count, whose codes are then finite whatever they are.
template <int D>
__device__ __forceinline__ uint32_t key_byte(const KeyRegs<D>& x, int g, bool ok) {
  const uint32_t b = D == 128 ? x.ks >> (8 * g) : x.ks >> (8 * (g >> 1));
  return ok ? b & 255u : 0u;
}
template <int D>
__device__ __forceinline__ uint32_t value_byte(const KeyRegs<D>& x, int g, bool ok) {
  const uint32_t b = D == 128 ? x.vs >> (8 * g) : x.ks >> (16 + 8 * (g >> 1));
  return ok ? b & 255u : 0u;
}

template <int D>
constexpr int kVRow = 2 * D + 32;  // bytes of a decoded value row in LDS: 8 rows cover all banks once

// ---------------------------------------------------------------------------
// Few rows a tile: the four waves of a block share the chunk's keys, 32 at a
// time in turn, and join their sums at the end. Keys are decoded straight into
// the matrix operand; values pass through the wave's own LDS rows, whose
// transposing reads give the other operand. The products are taken as
// S^T = K Q^T and O^T = V^T P^T, so that a lane's probabilities are already
// the operand of the second product.
// ---------------------------------------------------------------------------
template <int D, int RT, bool LIST>
__global__ __launch_bounds__(256) void k_attn4_few(Attn4Args a) {
  constexpr int ROWS = 16 * RT, NI = D / 32, NT = D / 16;
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  const Item it = LIST ? find_list_item<ROWS>(a, blockIdx.x) : find_item<ROWS>(a, blockIdx.x);

  // rows of tokens that belong to no request
  {
    const int used = a.R > 0 ? min(max(a.cu[a.R], 0), a.T) : 0;
    const int per = a.hkv * a.group * D / 2;
    for (int t = used + blockIdx.x; t < a.T; t += gridDim.x) {
      uint32_t* o = reinterpret_cast<uint32_t*>(a.out + (int64_t)t * per * 2);
      for (int i = threadIdx.x; i < per; i += 256) o[i] = 0u;
      if (a.lse)
        for (int i = threadIdx.x; i < a.hkv * a.group; i += 256) a.lse[(int64_t)t * a.hkv * a.group + i] = neg_inf();
    }
  }
  if (!it.any) return;

  // this lane's rows (column c of every row tile) and their ranges
  const int rows = LIST ? min((it.row0 / a.group + 1) * a.group, it.nt * a.group) : it.nt * a.group;
  bf16x8_t q[RT][NI];
  int rs[RT], re[RT];
  int lo = 0x7FFFFFFF, hi = 0, smax = 0, emin = 0x7FFFFFFF;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int x = it.row0 + rt * 16 + c;
    rs[rt] = re[rt] = 0;
    if (x < rows) {
      const int i = x / a.group, h = it.head * a.group + (x - i * a.group);
      const uint16_t* p = a.q + (int64_t)(it.t0 + i) * a.q_stride + (int64_t)h * D + g * (D / 4);
#pragma unroll
      for (int n = 0; n < NI; ++n) q[rt][n] = *reinterpret_cast<const bf16x8_t*>(p + 8 * n);
      const RowRange rr = token_range(a, it, i);
      rs[rt] = rr.s;
      re[rt] = rr.e;
      if (rr.s < rr.e) {
        lo = min(lo, rr.s);
        hi = max(hi, rr.e);
      }
      smax = max(smax, rr.s);
      emin = min(emin, rr.e);
    } else {
#pragma unroll
      for (int n = 0; n < NI; ++n) q[rt][n] = bf16x8_t{};
    }
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    lo = min(lo, __shfl_xor(lo, o));
    hi = max(hi, __shfl_xor(hi, o));
    smax = max(smax, __shfl_xor(smax, o));
    emin = min(emin, __shfl_xor(emin, o));
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  smax = __builtin_amdgcn_readfirstlane(smax);
  emin = __builtin_amdgcn_readfirstlane(emin);
  if (lo > hi) lo = hi;

  // the chunk's keys: positions, or places on the token's list
  int64_t k0, k1;
  const int32_t* list = nullptr;
  int base = 0;
  if constexpr (LIST) {
    const int t = it.t0 + it.row0 / a.group;
    list = a.list + (int64_t)t * a.list_ld;
    base = a.list_base ? a.list_base[t] : 0;
    k0 = (int64_t)it.chunk * it.C;
    k1 = min(k0 + (int64_t)it.C, (int64_t)a.list_k);
    if (lo == hi) k1 = k0;
  } else {
    k0 = lo + (int64_t)it.chunk * it.C;
    k1 = it.chunk == it.chunks - 1 ? hi : min(k0 + (int64_t)it.C, (int64_t)hi);
  }
  const int32_t* table = a.table + (int64_t)it.r * a.table_ld;

  f32x4_t acc[RT][NT];
  float m[RT], mc[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = neg_inf();
    mc[rt] = 0.0f;
    l[rt] = 0.0f;
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[rt][n] = f32x4_t{};
  }
  uint8_t* vrows = lds + wave * 32 * kVRow<D>;
  const float sc = a.scale_log2;

  const int steps = k1 > k0 ? (int)((k1 - k0 + 31) / 32) : 0;

  // position of place j, or -1
  auto place = [&](int64_t j) -> int {
    if (j >= k1) return -1;
    if constexpr (LIST) {
      const int p = list[j] - base;
      return p >= lo && p < hi ? p : -1;
    } else {
      return (int)j;
    }
  };
  auto page_of = [&](int pos) -> int {
    const int b = pos >> a.shift;
    return pos >= 0 && b < a.table_width ? table[b] : -1;
  };

  // software pipeline: codes one step ahead, pages two, list entries three
  KeyRegs<D> kv[2];
  int pos[2] = {-1, -1}, pos1[2] = {-1, -1}, page1[2] = {-1, -1}, pos2[2] = {-1, -1};
  bool ok[2] = {false, false};
  auto place_of_step = [&](int s, int (&p)[2]) {
    const int64_t j = k0 + (int64_t)s * 32 + c;
    p[0] = s < steps ? place(j) : -1;
    p[1] = s < steps ? place(j + 16) : -1;
  };
  {
    int p0[2];
    place_of_step(wave, p0);
    place_of_step(wave + 4, pos1);
    place_of_step(wave + 8, pos2);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int pg = page_of(p0[u]);
      page1[u] = page_of(pos1[u]);
      pos[u] = p0[u];
      ok[u] = pg >= 0 && pg < a.num_pages;
      load_key<D>(a, pg, p0[u], it.head, ok[u], kv[u]);
    }
  }

  for (int s = wave; s < steps; s += 4) {
    // decode this step
    bf16x8_t kf[2][NI];
    const uint32_t valid0 = (uint32_t)__ballot(ok[0]) & 0xFFFFu, valid1 = (uint32_t)__ballot(ok[1]) & 0xFFFFu;
    const int64_t j0 = k0 + (int64_t)s * 32;
    bool whole = (valid0 & valid1) == 0xFFFFu;
    if constexpr (!LIST) whole = whole && j0 >= smax && j0 + 32 <= emin;
    uint64_t bad[2] = {0, 0};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float ks = __uint_as_float(key_byte<D>(kv[u], g, ok[u]) << 23);
      uint32_t vb = value_byte<D>(kv[u], g, ok[u]);
      // a value that is not finite must not reach rows that do not see it
      if (!whole) {
        bad[u] = __ballot(vb == 255u);
        if (vb == 255u) vb = 0u;
      }
      const float vs = __uint_as_float(vb << 23);
      uint8_t* w = vrows + (u * 16 + c) * kVRow<D> + g * (D / 2);
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        kf[u][n] = decode8(kv[u].k[n], ks);
        *reinterpret_cast<bf16x8_t*>(w + 16 * n) = decode8(kv[u].v[n], vs);
      }
    }
    // start the next one
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      pos[u] = pos1[u];
      const int pg = page1[u];
      ok[u] = pg >= 0 && pg < a.num_pages;
      load_key<D>(a, pg, pos[u], it.head, ok[u], kv[u]);
      pos1[u] = pos2[u];
      page1[u] = page_of(pos1[u]);
    }
    place_of_step(s + 12, pos2);

    // S^T, then probabilities
    bf16x8_t p[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      f32x4_t s0 = {}, s1 = {};
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[0][n], q[rt][n], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[1][n], q[rt][n], s1, 0, 0, 0);
      }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int kk = 4 * g + i;
          bool v0 = (valid0 >> kk) & 1u, v1 = (valid1 >> kk) & 1u;
          if constexpr (!LIST) {
            const int64_t j = j0 + kk;
            v0 = v0 && j >= rs[rt] && j < re[rt];
            v1 = v1 && j + 16 >= rs[rt] && j + 16 < re[rt];
          }
          s0[i] = v0 ? s0[i] : neg_inf();
          s1[i] = v1 ? s1[i] : neg_inf();
        }
      }
      const float top = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])),
                              fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
      // the maximum is renewed only where it would grow by more than 2^8: the
      // sums keep their precision at any power of two
      if (__any(top > m[rt] + a.slack)) {
        const float mn = fmaxf(m[rt], max_groups(top));
        const float nc = mn == neg_inf() ? 0.0f : mn * sc;
        const float f = m[rt] == neg_inf() ? 0.0f : exp2_fast(mc[rt] - nc);
        m[rt] = mn;
        mc[rt] = nc;
        l[rt] *= f;
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[rt][n] *= f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s0[i] = exp2_fast(fmaf(s0[i], sc, -mc[rt]));
        s1[i] = exp2_fast(fmaf(s1[i], sc, -mc[rt]));
      }
      l[rt] += (s0[0] + s0[1]) + (s0[2] + s0[3]) + ((s1[0] + s1[1]) + (s1[2] + s1[3]));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[rt][i] = (__bf16)s0[i];
        p[rt][4 + i] = (__bf16)s1[i];
      }
    }
    // O^T += V^T P^T
    __builtin_amdgcn_wave_barrier();
    const uint8_t* vr = vrows + (4 * g + (c >> 2)) * kVRow<D> + (c & 3) * 8;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(vr + n * 32));
      const s16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(vr + 16 * kVRow<D> + n * 32));
      const bf16x8_t vf = __builtin_bit_cast(
          bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) acc[rt][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[rt], acc[rt][n], 0, 0, 0);
    }
    __builtin_amdgcn_wave_barrier();
    // values that are not finite, into the rows that see them
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint64_t b = bad[u];
      while (b) {
        const int from = __ffsll((unsigned long long)b) - 1;
        b &= b - 1;
        const int kk = from & 15, gg = from >> 4;  // key, quarter of the dims
        const int64_t j = j0 + u * 16 + kk;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          bool sees = it.row0 + rt * 16 + c < rows;
          if constexpr (!LIST) sees = sees && j >= rs[rt] && j < re[rt];
          if (sees) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
              if (n / (NT / 4) == gg) acc[rt][n] += __builtin_nanf("");
          }
        }
      }
    }
  }

  // join the four waves: maxima and sums first, then the outputs by halves
  float* ml = reinterpret_cast<float*>(lds + a.lds_join);  // [4][2][ROWS]
  float w[RT];
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] = sum_groups(l[rt]);
    if (g == 0) {
      ml[(wave * 2) * ROWS + rt * 16 + c] = m[rt] == neg_inf() ? neg_inf() : mc[rt];
      ml[(wave * 2 + 1) * ROWS + rt * 16 + c] = l[rt];
    }
  }
  __syncthreads();
  float M[RT], L[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    M[rt] = neg_inf();
#pragma unroll
    for (int i = 0; i < 4; ++i) M[rt] = fmaxf(M[rt], ml[(i * 2) * ROWS + rt * 16 + c]);
    const float ref = M[rt] == neg_inf() ? 0.0f : M[rt];
    L[rt] = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      L[rt] += exp2_fast(ml[(i * 2) * ROWS + rt * 16 + c] - ref) * ml[(i * 2 + 1) * ROWS + rt * 16 + c];
    w[rt] = m[rt] == neg_inf() ? 0.0f : exp2_fast(mc[rt] - ref);
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[rt][n] *= w[rt];
  }
  f32x4_t* box = reinterpret_cast<f32x4_t*>(lds);  // [2][RT * NT][64]
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int n = 0; n < NT; ++n) box[((wave - half) * RT * NT + rt * NT + n) * 64 + lane] = acc[rt][n];
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[rt][n] += box[(wave * RT * NT + rt * NT + n) * 64 + lane];
    }
    __syncthreads();
  }
  if (wave) return;

#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int x = it.row0 + rt * 16 + c;
    if (x >= rows) continue;
    if (it.chunks == 1) {
      const int i = x / a.group, h = it.head * a.group + (x - i * a.group);
      const int64_t row = (int64_t)(it.t0 + i) * a.hkv * a.group + h;
      const float inv = L[rt] == 0.0f ? 0.0f : 1.0f / L[rt];
      __bf16* o = reinterpret_cast<__bf16*>(a.out) + row * D + 4 * g;
      typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const f32x4_t y = acc[rt][n] * inv;
        *reinterpret_cast<bf16x4_t*>(o + n * 16) = bf16x4_t{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
      }
      if (a.lse && g == 0)
        a.lse[row] = L[rt] == 0.0f ? neg_inf() : (M[rt] + __builtin_amdgcn_logf(L[rt])) * kLn2;
    } else {
      const int64_t at = (int64_t)blockIdx.x * ROWS + rt * 16 + c;
      f32x4_t* o = reinterpret_cast<f32x4_t*>(a.part_o + at * D) + g;
#pragma unroll
      for (int n = 0; n < NT; ++n) o[n * 4] = acc[rt][n];
      if (g == 0) a.part_ml[at] = float2{M[rt], L[rt]};
    }
  }
}

// Joins the chunks of a tile: one block for each item and 4 of its rows (only
// the items that are a tile's first chunk of several do anything), a wave a
// row.
template <int D, int ROWS, bool LIST>
__global__ __launch_bounds__(256) void k_attn4_join(Attn4Args a) {
  const Item it = LIST ? find_list_item<ROWS>(a, blockIdx.x) : find_item<ROWS>(a, blockIdx.x);
  if (!it.any || it.chunks == 1 || it.chunk != 0) return;
  const int lane = threadIdx.x & 63, in = blockIdx.y * 4 + (threadIdx.x >> 6), x = it.row0 + in;
  const int rows = LIST ? min((it.row0 / a.group + 1) * a.group, it.nt * a.group) : it.nt * a.group;
  if (x >= rows) return;
  const int64_t at = (int64_t)blockIdx.x * ROWS + in;
  float M = neg_inf();
  for (int i = lane; i < it.chunks; i += 64) M = fmaxf(M, a.part_ml[at + (int64_t)i * ROWS].x);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
  const float ref = M == neg_inf() ? 0.0f : M;
  float L = 0.0f, o0 = 0.0f, o1 = 0.0f;
  for (int i = 0; i < it.chunks; ++i) {
    const float2 ml = a.part_ml[at + (int64_t)i * ROWS];
    const float w = exp2_fast(ml.x - ref);
    L = fmaf(w, ml.y, L);
    const float* o = a.part_o + (at + (int64_t)i * ROWS) * D;
    if (ml.x != neg_inf()) {
      if constexpr (D == 128) {
        const float2 v = reinterpret_cast<const float2*>(o)[lane];
        o0 = fmaf(w, v.x, o0);
        o1 = fmaf(w, v.y, o1);
      } else {
        o0 = fmaf(w, o[lane], o0);
      }
    }
  }
  const int i = x / a.group, h = it.head * a.group + (x - i * a.group);
  const int64_t row = (int64_t)(it.t0 + i) * a.hkv * a.group + h;
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  __bf16* out = reinterpret_cast<__bf16*>(a.out) + row * D;
  if constexpr (D == 128) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    reinterpret_cast<pair*>(out)[lane] = pair{(__bf16)(o0 * inv), (__bf16)(o1 * inv)};
  } else {
    out[lane] = (__bf16)(o0 * inv);
  }
  if (a.lse && lane == 0) a.lse[row] = L == 0.0f ? neg_inf() : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

template <int D, int RT, bool LIST>
hipError_t run_few(Attn4Args a, hipStream_t st) {
  constexpr int ROWS = 16 * RT;
  constexpr int stage = 4 * 32 * kVRow<D>, box = 2 * RT * (D / 16) * 64 * 16;
  a.lds_join = stage > box ? stage : box;
  const size_t lds = (size_t)a.lds_join + 4 * 2 * ROWS * 4;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_attn4_few<D, RT, LIST>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  if (!LIST && a.R > kInlineRequests) k_attn4_schedule<ROWS><<<1, 1024, 0, st>>>(a);
  k_attn4_few<D, RT, LIST><<<dim3((unsigned)a.items), 256, lds, st>>>(a);
  if (a.split) k_attn4_join<D, ROWS, LIST><<<dim3((unsigned)a.items, ROWS / 4), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <int D, bool LIST>
hipError_t run_rt(const Attn4Args& a, hipStream_t st) {
  if (a.rt == 1) return run_few<D, 1, LIST>(a, st);
  if (a.rt == 2) return run_few<D, 2, LIST>(a, st);
  return run_few<D, 4, LIST>(a, st);
}

constexpr int kTargetItems = 1024;

// Shape of the launch: everything that depends on host values alone.
bool shape_of(Attn4Args& a) {
  const int64_t rows = a.list_k > 0 ? a.group : ((int64_t)a.T * a.group + a.R - 1) / (a.R > 0 ? a.R : 1);
  a.rt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const int ROWS = 16 * a.rt;
  int64_t items;
  if (a.list_k > 0) {
    a.row_tiles = (a.group + ROWS - 1) / ROWS;
    const int64_t tiles = (int64_t)a.T * a.hkv * a.row_tiles;
    const int64_t most = (a.list_k + kMinChunk - 1) / kMinChunk;
    int64_t n = (kTargetItems + tiles - 1) / tiles;
    n = n < 1 ? 1 : n > most ? most : n;
    a.chunk_keys = (int)(((a.list_k + n - 1) / n + 31) / 32 * 32);
    a.chunks = (a.list_k + a.chunk_keys - 1) / a.chunk_keys;
    a.split = a.chunks > 1;
    a.target = 0;
    items = tiles * a.chunks;
  } else {
    const int64_t tiles = (int64_t)a.hkv * (((int64_t)a.T * a.group + ROWS - 1) / ROWS + a.R);
    a.split = (int64_t)a.T * a.group * a.hkv <= 131072;
    a.target = a.split ? kTargetItems : 0;
    items = tiles + a.target;
  }
  a.items = items;
  return items <= 0x3FFFFFFF;
}

}  // namespace

size_t attn4_workspace_bytes(Attn4Args a) {
  if (!shape_of(a)) return 0;
  size_t n = 256 + (((size_t)a.R + 2) * 4 + 255) / 256 * 256;
  if (a.split) n += (size_t)a.items * 16 * a.rt * ((size_t)a.d * 4 + 8);
  return n;
}

hipError_t launch_attn4(Attn4Args a, void* workspace, hipStream_t st) {
  if (!shape_of(a)) return hipErrorInvalidValue;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.sched = reinterpret_cast<uint32_t*>(ws);
  ws += (((size_t)a.R + 2) * 4 + 255) / 256 * 256;
  a.part_o = reinterpret_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(ws + (a.split ? (size_t)a.items * 16 * a.rt * a.d * 4 : 0));
  a.slack = 8.0f / a.scale_log2;
  if (!(a.slack < 1e30f)) a.slack = 1e30f;
  if (a.list_k > 0) return a.d == 128 ? run_rt<128, true>(a, st) : run_rt<64, true>(a, st);
  return a.d == 128 ? run_rt<128, false>(a, st) : run_rt<64, false>(a, st);
}

}  // namespace lt
