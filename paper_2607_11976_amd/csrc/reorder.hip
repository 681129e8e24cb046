// Rows of a paged cache go on as their parents (beam search): block tables, lengths,
// the pages to copy, and the free list.
//
// A child shares its parent's full pages. A partial page goes to the parent's first
// child (lowest row); the others get a page of the free list and a copy. What a row
// without children held is given back, unless another row has it: rows of a group share
// their pages from the first on up to where they parted, so of row r the pages from
//   d_r = max over the rows q that have children, or lie before r, of the length of the
//         tables' common start
// on are nobody else's. Pages given back go onto the list from its mark downwards, in
// row order, and are the first that copies take.
//
// Two launches, both bound by chains of dependent loads. First a wave per row: which
// rows have children (parents of the group in its lanes), and d_r by a search in which
// the lanes share the columns (64 / group of them per other row). Then every block
// repeats the sums over the rows in LDS, as the page plan does, and its waves take the
// rows in turn: no block waits for another, and no atomic.
#include <algorithm>

#include "cache4.hpp"
#include "internal.hpp"

namespace lt {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// What the first launch leaves of a row.
struct RowInfo {
  int parent;     // row that it goes on from, -1: it ends
  int take;       // 1: its partial page is a copy
  int from, give; // columns [from, held) hold `give` pages that go back
};

__device__ __forceinline__ int pages_held(const ReorderArgs& a, int len) {
  if (len <= 0) return 0;
  return min((int)(((int64_t)len + (1 << a.shift) - 1) >> a.shift), a.width);
}

__device__ __forceinline__ uint64_t or_lanes(uint64_t v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t hi = (uint32_t)__shfl_xor((int)(v >> 32), o), lo = (uint32_t)__shfl_xor((int)(uint32_t)v, o);
    v |= (uint64_t)hi << 32 | lo;
  }
  return v;
}

// Row r's, by a whole wave.
__device__ __forceinline__ RowInfo find_row(const ReorderArgs& a, int r, int lanes_log2) {
  const int lane = threadIdx.x & 63;
  const int g = r / a.group * a.group, w = r - g;
  int par = -1, length = 0;  // of the group's rows
  if (lane < a.group) {
    par = a.parents[g + lane];
    length = a.lens[g + lane];
    if (par >= a.group) par = -1;
  }
  const uint64_t alive = or_lanes(par >= 0 ? 1ull << par : 0);  // rows of the group that go on
  const int mine = __shfl(par, w);
  const int parent = mine < 0 ? -1 : g + mine;
  const bool first = mine >= 0 && __ffsll((unsigned long long)__ballot(par == mine)) - 1 == w;
  int take = 0;
  if (parent >= 0 && !first) {
    const int len = __shfl(length, mine), at = len >> a.shift;
    if (len > 0 && (len & ((1 << a.shift) - 1)) && at < a.width)
      take = a.table[(int64_t)parent * a.table_ld + at] >= 0;
  }
  int from = 0, give = 0;
  if (!((alive >> w) & 1)) {
    const int held = pages_held(a, __shfl(length, w));
    const int32_t* row = a.table + (int64_t)r * a.table_ld;
    // 1 << lanes_log2 lanes search the common start with row q
    const int S = 1 << lanes_log2, q = lane >> lanes_log2, sub = lane & (S - 1);
    const uint64_t others = (alive | ((1ull << w) - 1)) & ~(1ull << w);
    int lo = 0, hi = 0;
    const int other_len = __shfl(length, min(q, a.group - 1));
    if (q < a.group && ((others >> q) & 1)) hi = min(held, pages_held(a, other_len));
    const int32_t* other = a.table + (int64_t)(g + min(q, a.group - 1)) * a.table_ld;
    const uint64_t mask = S == 64 ? ~0ull : (1ull << S) - 1;
    while (__any(lo < hi)) {  // columns before lo are alike; column hi is not, or past the end
      const int64_t n = hi - lo;
      const int p = lo + (int)(n * (sub + 1) / (S + 1));  // < hi where lo < hi
      const bool same = lo < hi && row[p] == other[p];
      const uint64_t differ = ~(__ballot(same) >> (q << lanes_log2)) & mask;
      const int f = differ ? __ffsll((unsigned long long)differ) - 1 : S;  // first probe that differs
      if (lo < hi) {
        const int l = f > 0 ? lo + (int)(n * f / (S + 1)) + 1 : lo;
        if (f < S) hi = lo + (int)(n * (f + 1) / (S + 1));
        lo = l;
      }
    }
    from = lo;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) from = max(from, __shfl_xor(from, o));
    if (a.keep) from = max(from, a.keep[r]);
    from = min(from, held);
    for (int c = from; c < held; c += 64) give += __popcll(__ballot(c + lane < held && row[min(c + lane, held - 1)] >= 0));
  }
  return RowInfo{parent, take, from, give};
}

__global__ __launch_bounds__(kThreads) void k_reorder_find(ReorderArgs a, RowInfo* info, int lanes_log2) {
  const int r = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (r >= a.R) return;
  const RowInfo me = find_row(a, r, lanes_log2);
  if ((threadIdx.x & 63) == 0) info[r] = me;
}

// In-place exclusive prefix sums of two arrays of n entries, the totals at [n].
template <int THREADS>
__device__ __forceinline__ void sums_of(uint32_t* x, uint32_t* y, int n, uint32_t* part) {
  constexpr int kParts = THREADS / 64;
  const int t = threadIdx.x, per = (n + THREADS - 1) / THREADS, lane = t & 63, w = t >> 6;
  const int b = min(t * per, n), e = min(b + per, n);
  uint32_t sx = 0, sy = 0;
  for (int i = b; i < e; ++i) sx += x[i], sy += y[i];
  uint32_t ix = sx, iy = sy;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t ux = __shfl_up(ix, o), uy = __shfl_up(iy, o);
    if (lane >= o) ix += ux, iy += uy;
  }
  if (lane == 63) part[w] = ix, part[kParts + w] = iy;
  __syncthreads();
  uint32_t bx = ix - sx, by = iy - sy;
  for (int i = 0; i < w; ++i) bx += part[i], by += part[kParts + i];
  for (int i = b; i < e; ++i) {
    const uint32_t vx = x[i], vy = y[i];
    x[i] = bx, y[i] = by;
    bx += vx, by += vy;
  }
  if (t == THREADS - 1) x[n] = bx, y[n] = by;
  __syncthreads();
}

// Column of the j-th page (from 0) among entries [c, held) of a row; a whole wave.
__device__ __forceinline__ int nth_page(const int32_t* row, int c, int held, int j) {
  const int lane = threadIdx.x & 63;
  for (; c < held; c += 64) {
    const uint64_t in = __ballot(c + lane < held && row[min(c + lane, held - 1)] >= 0);
    const int n = __popcll(in);
    if (j < n) {
      const uint64_t at = __ballot(((in >> lane) & 1) && __popcll(in & ((1ull << lane) - 1)) == j);
      return c + __ffsll((unsigned long long)at) - 1;
    }
    j -= n;
  }
  return -1;
}

// What the sums over the rows say of the list.
struct Marks {
  int used, mark;   // the list's mark before, and with the pages given back
  uint32_t room;    // pages behind it
};
__device__ __forceinline__ Marks marks_of(const ReorderArgs& a, int used, const uint32_t* taken, const uint32_t* given) {
  const uint32_t back = given[a.R];
  const int mark = back < (uint32_t)used ? used - (int)back : 0;  // pages past the list's start are not kept
  const Marks m{used, mark, (uint32_t)(a.free_count - mark)};
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.free_out = mark + (int)min(taken[a.R], m.room);
  return m;
}

// Row r's results and the pages that it gives back, by a whole wave; the sums over the
// rows before each row (R + 1 entries) and all rows' infos.
__device__ __forceinline__ void write_row(const ReorderArgs& a, int r, const RowInfo* info, const uint32_t* taken,
                                          const uint32_t* given, const Marks& m) {
  const int lane = threadIdx.x & 63;
  const RowInfo me = info[r];
  if (me.give > 0) {
    const int32_t* row = a.table + (int64_t)r * a.table_ld;
    const int held = pages_held(a, a.lens[r]);
    int64_t at = (int64_t)m.used - 1 - given[r];
    for (int c = me.from; c < held; c += 64) {
      const int page = c + lane < held ? row[c + lane] : -1;
      const uint64_t in = __ballot(page >= 0);
      const int64_t place = at - __popcll(in & ((1ull << lane) - 1));
      if (page >= 0 && place >= 0) a.free_list[place] = page;
      at -= __popcll(in);
    }
  }
  // the page of a copy: the list from its mark on, where the pages given back come first
  int source = -1, target = -1, status = me.parent < 0 ? 1 : 0;
  const int len = me.parent < 0 ? 0 : a.lens[me.parent];
  const int32_t* from = a.table + (int64_t)max(me.parent, 0) * a.table_ld;
  const int cut = len > 0 ? len >> a.shift : 0;  // column of the partial page
  if (me.take) {
    const uint32_t n = taken[r];
    if (n >= m.room) {
      status = 2;
    } else {
      const int at = m.mark + (int)n;
      source = from[cut];
      if (at >= m.used) {
        target = a.free_list[at];
      } else {
        const uint32_t j = (uint32_t)(m.used - 1 - at);  // of the pages given back
        int lo = 0, hi = a.R;                            // given[lo] <= j < given[hi]
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (given[mid] <= j) lo = mid;
          else hi = mid;
        }
        const int32_t* row = a.table + (int64_t)lo * a.table_ld;
        const int c = nth_page(row, info[lo].from, pages_held(a, a.lens[lo]), (int)(j - given[lo]));
        if (c >= 0) target = row[c];
      }
    }
  }
  const int held = status ? 0 : pages_held(a, len);
  int32_t* out = a.out_table + (int64_t)r * a.out_ld;
  for (int c = lane; c < a.width; c += 64) {
    int page = c < held ? from[c] : -1;
    if (me.take && c == cut && c < held) page = target;
    out[c] = page;
  }
  if (lane == 0) {
    a.out_lens[r] = status ? 0 : len;
    a.status[r] = status;
    a.copies[2 * (int64_t)r] = source;
    a.copies[2 * (int64_t)r + 1] = target;
  }
}

__global__ __launch_bounds__(kThreads) void k_reorder_write(ReorderArgs a, const RowInfo* info) {
  extern __shared__ uint32_t lds[];
  __shared__ uint32_t part[2 * kWaves];
  uint32_t* taken = lds;                // [R + 1] prefix sums of the copies
  uint32_t* given = lds + a.R + 1;      // [R + 1] and of the pages given back
  const int t = threadIdx.x;
  for (int r = t; r < a.R; r += kThreads) taken[r] = (uint32_t)info[r].take, given[r] = (uint32_t)info[r].give;
  const int used = min(max(*a.free_used, 0), a.free_count);
  __syncthreads();
  sums_of<kThreads>(taken, given, a.R, part);
  const Marks m = marks_of(a, used, taken, given);
  const int waves = gridDim.x * kWaves;
  for (int r = blockIdx.x * kWaves + (t >> 6); r < a.R; r += waves) write_row(a, r, info, taken, given, m);
}

// Few rows: all in one block, one launch, which saves the host's 4 us for another: with
// cache4_copy from a program's loop a step takes 19.3 us where two launches take 23.5, with
// tables 63 to 512 pages wide; with 2048 pages 32 rows take 25.1 and 23.3. On the GPU alone
// (us in a graph, tables 63, 512, 2048 and 8192 wide): 4 rows 6.3, 7.6, 10.9, 24.8, by two
// kernels 6.9, 8.1, 11.4, 25.0; 16 rows 9.0, 10.1, 14.6, 30.7 and 8.8, 10.1, 13.9, 28.2; 32
// rows, two a wave, 11.7, 14.0, 22.4, 54 and 8.3, 9.8, 13.7, 28: the rule costs where tables
// are long or the calls are in a graph; 64 rows take 20 and 8.5.
constexpr int kFewRows = 32, kFewThreads = 1024;
__global__ __launch_bounds__(kFewThreads) void k_reorder_few(ReorderArgs a, int lanes_log2) {
  __shared__ uint32_t part[2 * kFewThreads / 64], taken[kFewRows + 1], given[kFewRows + 1];
  __shared__ RowInfo info[kFewRows];
  const int wave = threadIdx.x >> 6, waves = kFewThreads / 64;
  const int used = min(max(*a.free_used, 0), a.free_count);
  for (int r = wave; r < a.R; r += waves) {
    const RowInfo me = find_row(a, r, lanes_log2);
    if ((threadIdx.x & 63) == 0) {
      info[r] = me;
      taken[r] = (uint32_t)me.take;
      given[r] = (uint32_t)me.give;
    }
  }
  __syncthreads();
  sums_of<kFewThreads>(taken, given, a.R, part);
  const Marks m = marks_of(a, used, taken, given);
  for (int r = wave; r < a.R; r += waves) write_row(a, r, info, taken, given, m);
}

// ---- copies of whole pages ----
// A block copies 16 KB, so that a page of 64 slots, 8 heads and 128 values is the work of
// five: two such pages take 2.8 us, 405 of a quarter of that (14 MB moved) 4.5.
constexpr int kCopyBytes = 16 * 1024;  // of a block

__global__ __launch_bounds__(kThreads) void k_cache4_copy(Cache4 c, uint8_t* codes, uint8_t* scales,
                                                          const int32_t* copies, int code_blocks) {
  const int pair = blockIdx.x, part = blockIdx.y;
  const int64_t from = copies[2 * (int64_t)pair], to = copies[2 * (int64_t)pair + 1];
  if (from < 0 || to < 0 || from >= c.num_pages || to >= c.num_pages || from == to) return;
  const int64_t rows = (int64_t)c.hkv << c.shift;
  if (part < code_blocks) {
    const int64_t bytes = rows * c.d, end = min((int64_t)(part + 1) * kCopyBytes, bytes);
    const uint8_t* in = codes + from * bytes;
    uint8_t* out = codes + to * bytes;
#pragma unroll 4
    for (int64_t i = (int64_t)part * kCopyBytes + threadIdx.x * 16; i < end; i += kThreads * 16)
      *reinterpret_cast<uint4*>(out + i) = *reinterpret_cast<const uint4*>(in + i);
  } else {
    // a row's scales are 4 or 8 bytes
    const int64_t bytes = rows * (c.d / 16), first = (int64_t)(part - code_blocks) * kCopyBytes,
                  end = min(first + kCopyBytes, bytes);
    const uint8_t* in = scales + from * bytes;
    uint8_t* out = scales + to * bytes;
#pragma unroll 4
    for (int64_t i = first + threadIdx.x * 4; i < end; i += kThreads * 4)
      *reinterpret_cast<uint32_t*>(out + i) = *reinterpret_cast<const uint32_t*>(in + i);
  }
}

int copy_blocks(int64_t bytes) { return (int)((bytes + kCopyBytes - 1) / kCopyBytes); }

}  // namespace

size_t reorder_workspace_bytes(int rows) { return ((size_t)std::max(rows, 1) * sizeof(RowInfo) + 255) / 256 * 256; }

hipError_t launch_paged_reorder(const ReorderArgs& a, void* workspace, hipStream_t st) {
  RowInfo* info = static_cast<RowInfo*>(workspace);
  int lanes_log2 = 6;
  while (a.group << lanes_log2 > 64) --lanes_log2;
  if (a.R <= kFewRows) {
    k_reorder_few<<<1, kFewThreads, 0, st>>>(a, lanes_log2);
    return hipGetLastError();
  }
  k_reorder_find<<<dim3((unsigned)((a.R + kWaves - 1) / kWaves)), kThreads, 0, st>>>(a, info, lanes_log2);
  const hipError_t found = hipGetLastError();
  if (found != hipSuccess) return found;
  const size_t lds = 8 * ((size_t)a.R + 1);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_reorder_write),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  // every block sums all rows: no more blocks than fill the GPU
  const int blocks = std::min((a.R + kWaves - 1) / kWaves, 512);
  k_reorder_write<<<dim3((unsigned)blocks), kThreads, lds, st>>>(a, info);
  return hipGetLastError();
}

int64_t cache4_copy_blocks(const Cache4& c, int n) {
  const int64_t rows = (int64_t)c.hkv << c.shift;
  return (int64_t)n * (copy_blocks(rows * c.d) + copy_blocks(rows * (c.d / 16)));
}

hipError_t launch_cache4_copy(const Cache4& c, uint8_t* codes, uint8_t* scales, const int32_t* copies, int n,
                              hipStream_t st) {
  const int64_t rows = (int64_t)c.hkv << c.shift;
  const int cb = copy_blocks(rows * c.d), sb = copy_blocks(rows * (c.d / 16));
  k_cache4_copy<<<dim3((unsigned)n, (unsigned)(cb + sb)), kThreads, 0, st>>>(c, codes, scales, copies, cb);
  return hipGetLastError();
}

}  // namespace lt
