// Paged serving cache: the plan of a step (block tables and slot maps from the
// requests' lengths) and the 4-bit key/value pages (writing and reading rows).
#include <algorithm>

#include "cache4.hpp"
#include "internal.hpp"

namespace lt {
namespace {

// ---------------------------------------------------------------------------
// Plan. Request r holds c_r tokens and adds n_r; it needs
// g_r = ceil((c_r + n_r) / P) - ceil(c_r / P) pages more. With the prefix sums
// N_r of n_r and G_r of g_r, token N_r + i lies at position c_r + i, and the
// request's i-th new page is free[used + G_r + i].
//
// One launch: every block repeats the two prefix sums in LDS (8 bytes a
// request) and then takes its slice of the tokens, of the new pages and of the
// requests; a search in the sums tells whose they are. Blocks share nothing, so
// there is no second launch, no flag between blocks and no atomic. The first
// blocks do the tokens, the others the pages and requests, side by side. With
// TOKENS = 4 a thread takes four consecutive tokens, which then mostly share their
// request and page: one search and one dependent load for all. The call is bound
// by its latency: the loads of the lengths, the sums and the load of the page.
// ---------------------------------------------------------------------------
constexpr uint32_t kPlanTop = 0x7FFFFFFFu;

// Both operands are at most kPlanTop; sums stop there (associative, monotone).
__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, kPlanTop); }

// First index i in (lo, hi] with s[i] > x, given s[lo] <= x; hi if there is none below it.
__device__ __forceinline__ int upper(const uint32_t* s, int lo, int hi, uint32_t x) {
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s[mid] <= x) lo = mid;
    else hi = mid;
  }
  return hi;
}

struct Need {
  uint32_t ctx, add, held, pages;
  bool longer;  // the block table has no room for the request's pages
};
__device__ __forceinline__ Need need_of(const PlanArgs& a, int r) {
  Need n;
  n.ctx = (uint32_t)max(a.context[r], 0);
  n.add = (uint32_t)max(a.added[r], 0);
  const uint32_t total = sat_add(n.ctx, n.add), low = (1u << a.shift) - 1u;
  n.held = (n.ctx >> a.shift) + ((n.ctx & low) ? 1u : 0u);
  const uint32_t all = (total >> a.shift) + ((total & low) ? 1u : 0u);
  n.longer = n.add > 0 && all > (uint32_t)a.width;
  n.pages = n.add > 0 && !n.longer ? all - n.held : 0u;
  return n;
}

// In-place exclusive prefix sums of two arrays of n entries, the totals at [n].
template <int THREADS>
__device__ __forceinline__ void plan_sums(uint32_t* x, uint32_t* y, int n, uint32_t* part) {
  constexpr int kWaves = THREADS / 64;
  const int t = threadIdx.x, per = (n + THREADS - 1) / THREADS;
  const int b = min(t * per, n), e = min(b + per, n);
  uint32_t sx = 0, sy = 0;
  for (int i = b; i < e; ++i) {
    sx = sat_add(sx, x[i]);
    sy = sat_add(sy, y[i]);
  }
  const int lane = t & 63, w = t >> 6;
  uint32_t ix = sx, iy = sy;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t ux = __shfl_up(ix, o), uy = __shfl_up(iy, o);
    if (lane >= o) {
      ix = sat_add(ix, ux);
      iy = sat_add(iy, uy);
    }
  }
  if (lane == 63) {
    part[w] = ix;
    part[kWaves + w] = iy;
  }
  // exclusive inside the wave
  uint32_t bx = __shfl_up(ix, 1), by = __shfl_up(iy, 1);
  if (lane == 0) bx = by = 0;
  __syncthreads();
  for (int i = 0; i < w; ++i) {
    bx = sat_add(bx, part[i]);
    by = sat_add(by, part[kWaves + i]);
  }
  for (int i = b; i < e; ++i) {
    const uint32_t vx = x[i], vy = y[i];
    x[i] = bx;
    y[i] = by;
    bx = sat_add(bx, vx);
    by = sat_add(by, vy);
  }
  if (t == THREADS - 1) {
    x[n] = bx;
    y[n] = by;
  }
  __syncthreads();
}

template <int THREADS, int TOKENS>
__global__ __launch_bounds__(THREADS) void k_paged_plan(PlanArgs a, int token_blocks) {
  extern __shared__ uint32_t lds[];
  __shared__ uint32_t part[2 * THREADS / 64];
  uint32_t* tok = lds;                  // [R + 1] prefix sums of the new tokens
  uint32_t* pag = lds + a.R + 1;        // [R + 1] prefix sums of the new pages
  const int t = threadIdx.x;
#pragma unroll 4
  for (int r = t; r < a.R; r += THREADS) {
    const Need n = need_of(a, r);
    tok[r] = n.add;
    pag[r] = n.pages;
  }
  const int used = min(max(*a.free_used, 0), a.free_count);
  __syncthreads();
  plan_sums<THREADS>(tok, pag, a.R, part);

  // Pages are handed out in request order until one request's do not fit: the
  // sums pass the number of free pages there for good, so the pages taken are
  // the largest sum within it.
  const uint32_t avail = (uint32_t)(a.free_count - used);
  const uint32_t taken = pag[upper(pag, 0, a.R + 1, avail) - 1];
  if ((int)blockIdx.x >= token_blocks) {
    const int stride = ((int)gridDim.x - token_blocks) * THREADS, at = ((int)blockIdx.x - token_blocks) * THREADS + t;
    if (at == 0) *a.free_out = used + (int)taken;
    for (int r = at; r <= a.R; r += stride) {
      a.cu[r] = (int)tok[r];
      if (r == a.R) break;
      const Need n = need_of(a, r);
      const bool out = n.pages > 0 && pag[r + 1] > avail;
      a.status[r] = n.longer ? 1 : out ? 2 : 0;
      a.seq[r] = (int)(n.longer || out ? n.ctx : sat_add(n.ctx, n.add));
    }
    for (uint32_t i = at; i < taken; i += stride) {
      const int r = upper(pag, 0, a.R, i) - 1;
      const Need n = need_of(a, r);
      a.table[(int64_t)r * a.table_ld + n.held + (i - pag[r])] = a.free_list[used + i];
    }
    return;
  }
  const uint32_t tokens = tok[a.R];
  const int64_t stride = (int64_t)token_blocks * THREADS * TOKENS;
  for (int64_t i0 = ((int64_t)blockIdx.x * THREADS + t) * TOKENS; i0 < a.capacity; i0 += stride) {
    int64_t slot[TOKENS];
    int pos[TOKENS];
    uint32_t first = 0, end = 0, block = 0;  // the request's tokens, and the page looked up
    int r = 0, page = -1;
    Need n{};
    bool served = false;
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
      const uint32_t i = (uint32_t)i0 + j;
      slot[j] = -1;
      pos[j] = -1;
      if (i >= tokens) continue;
      const bool next = i >= end;
      if (next) {
        r = upper(tok, 0, a.R, i) - 1;
        n = need_of(a, r);
        first = tok[r];
        end = tok[r + 1];
        served = !n.longer && (n.pages == 0 || pag[r + 1] <= avail);
      }
      const uint32_t p = sat_add(n.ctx, i - first), b = p >> a.shift;
      pos[j] = (int)p;
      if (!served) continue;
      if (next || b != block) {
        block = b;
        page = b < n.held ? a.table[(int64_t)r * a.table_ld + b] : a.free_list[used + pag[r] + (b - n.held)];
      }
      if (page >= 0) slot[j] = ((int64_t)page << a.shift) + (p & ((1u << a.shift) - 1u));
    }
    if (i0 + TOKENS <= a.capacity) {
      __builtin_memcpy(a.slots + i0, slot, sizeof(slot));
      __builtin_memcpy(a.positions + i0, pos, sizeof(pos));
    } else {
#pragma unroll
      for (int j = 0; j < TOKENS; ++j)
        if (i0 + j < a.capacity) a.slots[i0 + j] = slot[j], a.positions[i0 + j] = pos[j];
    }
  }
}

// ---------------------------------------------------------------------------
// Writing rows. A thread takes 8 consecutive values, the four threads of a
// block of 32 share its largest magnitude (two exchanges inside the quad), so
// a wave reads and writes whole lines. Bound by its memory traffic: 16381
// tokens of 8 heads of 128 values in float32 (134 MB read, 18 MB written) take
// 24 us, 6.3 TB/s.
// ---------------------------------------------------------------------------
template <class T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float (&x)[8]) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

template <class T>
__global__ __launch_bounds__(256) void k_cache4_append(const T* k, const T* v, int64_t k_stride, int64_t v_stride,
                                                       int64_t rows, Cache4 c, uint8_t* codes, uint8_t* scales,
                                                       const int64_t* slots) {
  const int per_row = c.d / 8, per_tok = c.hkv * per_row;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int which = blockIdx.y;
  const int64_t tok = at / per_tok;
  if (tok >= rows) return;  // whole quads: per_tok is a multiple of 8
  const int in = (int)(at - tok * per_tok), h = in / per_row, ch = in - h * per_row;
  const int64_t slot = slots[tok];
  if (slot < 0 || slot >= c.num_pages << c.shift) return;
  float x[8];
  load8((which ? v + tok * v_stride : k + tok * k_stride) + (int64_t)h * c.d + ch * 8, x);
  // largest magnitude as bits: NaN and infinity lie above every finite value
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
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
  const int64_t row = c.row(slot, h);
  *reinterpret_cast<uint32_t*>(codes + row * c.d + which * (c.d / 2) + ch * 4) = w;
  if ((ch & 3) == 0) scales[row * (c.d / 16) + which * (c.d / 32) + (ch >> 2)] = (uint8_t)e;
}

// Reading rows back: 8 values a thread. The same 16381 tokens (18 MB read, 67 MB
// written) take 20 us, 4.3 TB/s.
__global__ __launch_bounds__(256) void k_cache4_read(Cache4 c, const uint8_t* codes, const uint8_t* scales,
                                                     const int64_t* slots, int64_t rows, uint16_t* k, uint16_t* v) {
  const int per_row = c.d / 8, per_tok = c.hkv * per_row;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int which = blockIdx.y;
  const int64_t tok = at / per_tok;
  if (tok >= rows) return;
  const int in = (int)(at - tok * per_tok), h = in / per_row, ch = in - h * per_row;
  const int64_t slot = slots[tok];
  uint4 o = {0, 0, 0, 0};
  if (slot >= 0 && slot < c.num_pages << c.shift) {
    const int64_t row = c.row(slot, h);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + row * c.d + which * (c.d / 2) + ch * 4);
    const uint32_t e = scales[row * (c.d / 16) + which * (c.d / 32) + (ch >> 2)];
    o = __builtin_bit_cast(uint4, decode8(w, __uint_as_float(e << 23)));
  }
  *reinterpret_cast<uint4*>((which ? v : k) + tok * per_tok * 8 + (int64_t)in * 8) = o;
}

}  // namespace

template <int THREADS, int TOKENS>
static hipError_t run_plan(const PlanArgs& a, hipStream_t st) {
  constexpr int64_t per = THREADS * TOKENS;
  const int64_t tokens = std::min(((int64_t)a.capacity + per - 1) / per, (int64_t)512);
  const int64_t others = std::min(((int64_t)a.R + THREADS) / THREADS, (int64_t)32);
  const size_t lds = 8 * ((size_t)a.R + 1);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_paged_plan<THREADS, TOKENS>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  k_paged_plan<THREADS, TOKENS><<<dim3((unsigned)(tokens + others)), THREADS, lds, st>>>(a, (int)tokens);
  return hipGetLastError();
}

hipError_t launch_paged_plan(const PlanArgs& a, hipStream_t st) {
  // Every block sums all requests: wide blocks where there are many, narrow
  // ones for few, whose barriers cost less. Several tokens a thread only where
  // requests have several (64 decoding requests: 6.5 us with four, 4.2 with one;
  // 4096 requests and 540K tokens: 24 us with one and narrow blocks, 14 as here,
  // where writing the 6.5 MB would take 1.3).
  const bool several = a.capacity > 4 * (int64_t)a.R;
  if (a.R > 512) return several ? run_plan<1024, 4>(a, st) : run_plan<1024, 1>(a, st);
  return several ? run_plan<256, 4>(a, st) : run_plan<256, 1>(a, st);
}

hipError_t launch_cache4_append(const void* k, const void* v, bool f32, int64_t k_stride, int64_t v_stride,
                                int64_t rows, const Cache4& c, uint8_t* codes, uint8_t* scales, const int64_t* slots,
                                hipStream_t st) {
  const int64_t blocks = (rows * c.hkv * (c.d / 8) + 255) / 256;
  const dim3 grid((unsigned)blocks, 2);
  if (f32)
    k_cache4_append<float><<<grid, 256, 0, st>>>((const float*)k, (const float*)v, k_stride, v_stride, rows, c, codes,
                                                 scales, slots);
  else
    k_cache4_append<uint16_t><<<grid, 256, 0, st>>>((const uint16_t*)k, (const uint16_t*)v, k_stride, v_stride, rows,
                                                    c, codes, scales, slots);
  return hipGetLastError();
}

hipError_t launch_cache4_read(const Cache4& c, const uint8_t* codes, const uint8_t* scales, const int64_t* slots,
                              int64_t rows, void* k, void* v, hipStream_t st) {
  const int64_t blocks = (rows * c.hkv * (c.d / 8) + 255) / 256;
  k_cache4_read<<<dim3((unsigned)blocks, 2), 256, 0, st>>>(c, codes, scales, slots, rows, (uint16_t*)k, (uint16_t*)v);
  return hipGetLastError();
}

}  // namespace lt
