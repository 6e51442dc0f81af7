// The paged K/V cache: tables, reference counts and the copies they ask for.
//
// The bookkeeping is a few thousand integers, so each call does it in one
// workgroup (one thread per sequence, block-wide prefix sums), without atomics
// whose order could change a result: free pages go to the sequences lowest id
// first. References are counted with atomic adds, which commute. What moves
// bytes (rows into pages, whole pages) runs over the GPU and is bound by HBM.
//
// Measured, Qwen3-8B heads, five layers, pages of 64: reserve 6 us, keep 2, fork 5 (64
// sequences); rows of 64 x 17 tokens 16 us (45 MB in and out, 2.8 TB/s), of 16 x 17 7 us;
// copies of 64 pages 26 us (84 MB written, 3.2 TB/s, the source in cache); compaction of half
// the pages of 32 x 4096 rows 6 + 258 us (1.2 GB, 4.7 TB/s).
#include "ldr_internal.h"

namespace ldr {
namespace {

constexpr int kThreads = 256;
constexpr int kBook = 1024;        // threads of a bookkeeping workgroup
constexpr int kPiece = 16384;      // bytes of a page that a workgroup copies at a time
static_assert(kBook >= kMaxSeqs, "one thread per sequence");

__device__ inline int clamp_rows(const PagesShape& s, int r) {
  return min(max(r, 0), s.max_pages * s.page);
}
__device__ inline int clamp_page(const PagesShape& s, int id) {
  return min(max(id, 0), s.n_pages - 1);
}
__device__ inline int pages_of(const PagesShape& s, int rows) { return (rows + s.page - 1) / s.page; }

// Exclusive prefix sum of one value per thread of a bookkeeping workgroup, and
// the total. `sums`: kBook / 64 words of LDS.
template <typename T> __device__ inline T block_scan(T v, T* sums, T* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T inc = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const T o = __shfl_up(inc, off);
    if (lane >= off) inc += o;
  }
  __syncthreads();   // the last call's readers are done
  if (lane == 63) sums[wave] = inc;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kBook / 64; ++w) {
    const T x = sums[w];
    before += w < wave ? x : 0;
    all += x;
  }
  *total = all;
  return before + inc - v;
}

// The counter of changes goes on from what the memory holds: a plan of the cache that
// was there before is no plan of the empty one.
__global__ void __launch_bounds__(kBook) pages_reset_kernel(PagesShape s, PagesPtrs p) {
  for (size_t i = blockIdx.x * (size_t)kBook + threadIdx.x; i < s.words;
       i += (size_t)gridDim.x * kBook) {
    if (i == kPagesVersion) p.state[i] = (int32_t)((uint32_t)p.state[i] + 1u);
    else p.state[i] = i >= s.table && i < s.refs ? -1 : 0;
  }
}

__global__ void pages_clear_flags_kernel(PagesPtrs p) { p.state[kPagesFlags] = 0; }

// Room for n_new rows a sequence. The free list is taken in id order until it
// covers the pages wanted; the wanted pages' prefix sum over the sequences says
// which of them a sequence gets, its copy of a shared partial page first.
__global__ void __launch_bounds__(kBook)
pages_reserve_kernel(PagesShape s, PagesPtrs p, const int32_t* n_new, int max_new) {
  __shared__ long needs[kBook / 64];
  __shared__ int sums[kBook / 64], start[kBook], first_slot[kBook];
  __shared__ uint8_t granted[kBook];
  const int b = threadIdx.x;
  int32_t* table = p.state + s.table;
  int32_t* refs = p.state + s.refs;
  int32_t* list = p.state + s.list;
  int32_t* pairs = p.state + s.pairs;
  int flags = 0, rows = 0, n = 0, need = 0, first = 0, old = -1;
  if (b < s.batch) {
    rows = clamp_rows(s, p.state[s.rows + b]);
    n = n_new[b];
    if (n < 0 || n > max_new) {
      flags = kFlagRange;
      n = 0;
    } else if (n > s.max_pages * s.page - rows) {
      flags = kFlagPages;
      n = 0;
    }
    if (n > 0) {
      first = rows / s.page;
      if (rows % s.page) {
        const int id = clamp_page(s, table[(size_t)b * s.max_pages + first]);
        if (refs[id] > 1) old = id; else ++first;
      }
      need = pages_of(s, rows + n) - first;
    }
  }
  long all = 0;     // of all sequences: may be more than an int holds
  const long before = block_scan((long)need, needs, &all);
  const int want = (int)min(all, (long)s.n_pages);
  const int at = (int)min(before, (long)s.n_pages);
  start[b] = at;
  first_slot[b] = first;
  // the first `want` free pages (fewer if there are not as many)
  int found = 0;
  for (int base = 0; base < s.n_pages && found < want; base += 4 * kBook) {
    const int i = base + 4 * b;
    int r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = i + k < s.n_pages ? refs[i + k] : 1;
    const int mine = (r[0] <= 0) + (r[1] <= 0) + (r[2] <= 0) + (r[3] <= 0);
    int sum = 0;
    int k0 = found + block_scan(mine, sums, &sum);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (r[k] <= 0) {
        if (k0 < want) list[k0] = i + k;
        ++k0;
      }
    found += sum;
  }
  __syncthreads();
  const bool ok = need == 0 || need <= found - at;
  granted[b] = ok;
  if (b < s.batch) {
    if (!ok) {
      flags |= kFlagPages;
      n = 0;
      old = -1;
    }
    p.state[s.rows + b] = rows + n;
    p.state[s.open + b] = n;
    // the copy of the partial page; its old place has one holder less
    pairs[2 * b] = old;
    pairs[2 * b + 1] = old >= 0 ? list[at] : -1;
    if (old >= 0) atomicSub(refs + old, 1);
    if (flags) atomicOr(p.state + kPagesFlags, flags);
  }
  __syncthreads();
  const int last = min(want, found);
  for (int t = b; t < last; t += kBook) {
    int lo = 0, hi = s.batch - 1;    // the sequence whose pages hold t: the last start <= t
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (start[mid] <= t) lo = mid; else hi = mid - 1;
    }
    if (granted[lo]) {
      const int id = list[t];
      table[(size_t)lo * s.max_pages + first_slot[lo] + t - start[lo]] = id;
      refs[id] = 1;
    }
  }
  if (b == 0) p.state[kPagesVersion] += 1;
}

// One piece of a page of one plane (a layer's K or V) from page `from` to `to`.
__device__ inline void copy_piece(const PagesShape& s, const PagesPtrs& p, int plane, int piece,
                                  int from, int to) {
  constexpr int U = kPiece / 16 / kThreads;
  const size_t base = (size_t)plane * s.n_pages * s.page_bytes + (size_t)piece * kPiece;
  const size_t n = min((size_t)kPiece, s.page_bytes - (size_t)piece * kPiece) / 16;
  const uint4* in = reinterpret_cast<const uint4*>(p.pool + base + (size_t)from * s.page_bytes);
  uint4* out = reinterpret_cast<uint4*>(p.pool + base + (size_t)to * s.page_bytes);
  uint4 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const size_t i = (size_t)u * kThreads + threadIdx.x;
    x[u] = in[i < n ? i : 0];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const size_t i = (size_t)u * kThreads + threadIdx.x;
    if (i < n) out[i] = x[u];
  }
}

// The copies that a reserve asked for, at most one page a sequence: whole pages, so
// that the copy holds what its original does behind the rows too.
__global__ void __launch_bounds__(kThreads) pages_part_kernel(PagesShape s, PagesPtrs p) {
  const int b = blockIdx.z;
  const int from = p.state[s.pairs + 2 * b], to = p.state[s.pairs + 2 * b + 1];
  if (from < 0 || from >= s.n_pages || to < 0 || to >= s.n_pages) return;
  copy_piece(s, p, blockIdx.y, blockIdx.x, from, to);
}

// Open rows into their pages: one workgroup per (32 positions, layer and head,
// sequence), on two pages at most. K rows are copied; V is transposed through LDS
// and stored by runs of 16 bytes of one dimension. Tiles begin at multiples of such
// a run, so that no two workgroups write to one; the first and the last run keep
// their other rows, which nobody else writes (the page is the sequence's own). Stores
// of single values, dimension by dimension, took 10 and 26 us instead of 7 and 16.
template <typename T>
__global__ void __launch_bounds__(kThreads)
pages_write_kernel(PagesShape s, PagesPtrs p, int layer0, int n_layers, const T* K, const T* V,
                   int max_new) {
  constexpr int RT = 32, E = 16 / (int)sizeof(T), LD = 128 + E, RUNS = RT / E;
  __shared__ alignas(16) T tile[RT * LD];
  const int b = blockIdx.z, h = blockIdx.y % s.hkv, l = blockIdx.y / s.hkv;
  const int rows = clamp_rows(s, p.state[s.rows + b]);
  const int open = min(max(p.state[s.open + b], 0), rows);
  const int start = rows - open, end = start + min(open, max_new);
  const int first = start / E * E + (int)blockIdx.x * RT;
  if (first >= end) return;
  const int lo = max(first, start), hi = min(first + RT, end), cnt = hi - lo;
  const int32_t* table = p.state + s.table + (size_t)b * s.max_pages;
  const int j0 = lo / s.page;
  const int id0 = clamp_page(s, table[j0]), id1 = clamp_page(s, table[(hi - 1) / s.page]);
  const size_t plane = (size_t)2 * (layer0 + l) * s.n_pages;
  const size_t head = (size_t)h * s.page * s.d;
  uint8_t* kpool = p.pool + plane * s.page_bytes;
  uint8_t* vpool = kpool + (size_t)s.n_pages * s.page_bytes;
  auto page = [&](uint8_t* pool, int pos) {     // of a position of the tile
    return reinterpret_cast<T*>(pool + (size_t)(pos / s.page == j0 ? id0 : id1) * s.page_bytes) + head;
  };
  const size_t row = (size_t)n_layers * s.hkv * s.d;
  const size_t in0 = ((size_t)b * max_new + (lo - start)) * row + ((size_t)l * s.hkv + h) * s.d;
  const int c = s.d / E;                        // 16-byte pieces of a row
  for (int i = threadIdx.x; i < cnt * c; i += kThreads) {
    const int r = i / c, e = (i - r * c) * E;
    *reinterpret_cast<uint4*>(page(kpool, lo + r) + (size_t)(lo + r) % s.page * s.d + e) =
        *reinterpret_cast<const uint4*>(K + in0 + r * row + e);
    *reinterpret_cast<uint4*>(tile + r * LD + e) =
        *reinterpret_cast<const uint4*>(V + in0 + r * row + e);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < s.d * RUNS; i += kThreads) {
    const int dim = i / RUNS, pos = first + (i - dim * RUNS) * E;
    if (pos >= hi) continue;
    uint4* out = reinterpret_cast<uint4*>(page(vpool, max(pos, lo)) + (size_t)dim * s.page +
                                          pos % s.page);
    alignas(16) T x[E];
    if (pos < lo || pos + E > hi) *reinterpret_cast<uint4*>(x) = *out;
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (pos + k >= lo && pos + k < hi) x[k] = tile[(pos + k - lo) * LD + dim];
    *out = *reinterpret_cast<const uint4*>(x);
  }
}

__global__ void __launch_bounds__(kBook)
pages_keep_kernel(PagesShape s, PagesPtrs p, const int32_t* kept) {
  const int b = threadIdx.x;
  if (b == 0) p.state[kPagesVersion] += 1;
  if (b >= s.batch) return;
  const int rows = clamp_rows(s, p.state[s.rows + b]);
  const int open = min(max(p.state[s.open + b], 0), rows);
  const int k = kept[b];
  if (k < 0 || k > open) {
    atomicOr(p.state + kPagesFlags, kFlagRange);
    return;
  }
  const int left = rows - open + k;
  p.state[s.rows + b] = left;
  p.state[s.open + b] = k;
  int32_t* t = p.state + s.table + (size_t)b * s.max_pages;
  for (int j = pages_of(s, left); j < pages_of(s, rows); ++j) {
    const int id = t[j];
    t[j] = -1;
    if (id >= 0 && id < s.n_pages) atomicSub(p.state + s.refs + id, 1);
  }
}

// One workgroup per sequence. A source keeps its pages in the same launch, so
// its table and length are only read.
__global__ void __launch_bounds__(kThreads)
pages_fork_kernel(PagesShape s, PagesPtrs p, const int32_t* src) {
  const int b = blockIdx.x, from = src[b];
  if (b == 0 && threadIdx.x == 0) p.state[kPagesVersion] += 1;
  if (from == b) return;
  if (from < -1 || from >= s.batch || (from >= 0 && src[from] != from)) {
    if (threadIdx.x == 0) atomicOr(p.state + kPagesFlags, kFlagRange);
    return;
  }
  int32_t* t = p.state + s.table + (size_t)b * s.max_pages;
  const int32_t* f = p.state + s.table + (size_t)max(from, 0) * s.max_pages;
  int32_t* refs = p.state + s.refs;
  const int mine = pages_of(s, clamp_rows(s, p.state[s.rows + b]));
  const int theirs = from >= 0 ? pages_of(s, clamp_rows(s, p.state[s.rows + from])) : 0;
  for (int j = threadIdx.x; j < max(mine, theirs); j += kThreads) {
    const int old = t[j], id = j < theirs ? f[j] : -1;
    if (j < mine && old >= 0 && old < s.n_pages) atomicSub(refs + old, 1);
    if (id >= 0 && id < s.n_pages) atomicAdd(refs + id, 1);
    t[j] = id;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    p.state[s.rows + b] = from >= 0 ? clamp_rows(s, p.state[s.rows + from]) : 0;
    p.state[s.open + b] = 0;
    if (from >= 0) p.state[s.open + from] = 0;   // every copy of a source stores the same 0
  }
}

// Compaction, its list: with n live pages, the k-th live page at or above n goes
// to the k-th free id below n. `list` maps a moved page to its new id (-1:
// stays), `pairs` holds the moves.
__global__ void __launch_bounds__(kBook) pages_moves_kernel(PagesShape s, PagesPtrs p) {
  __shared__ int sums[kBook / 64];
  int32_t* refs = p.state + s.refs;
  int32_t* list = p.state + s.list;
  int32_t* pairs = p.state + s.pairs;
  int live = 0;
  for (int i = threadIdx.x; i < s.n_pages; i += kBook) live += refs[i] > 0;
  int n = 0;
  block_scan(live, sums, &n);
  int holes = 0, moved = 0;
  for (int base = 0; base < s.n_pages; base += 4 * kBook) {
    const int i = base + 4 * (int)threadIdx.x;
    bool hole[4], mover[4];
    int nh = 0, nm = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool in = i + k < s.n_pages, used = in && refs[i + k] > 0;
      hole[k] = in && !used && i + k < n;
      mover[k] = used && i + k >= n;
      nh += hole[k];
      nm += mover[k];
    }
    int th = 0, tm = 0;
    int h = holes + block_scan(nh, sums, &th), m = moved + block_scan(nm, sums, &tm);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (hole[k]) pairs[2 * h++ + 1] = i + k;
      if (mover[k]) pairs[2 * m++] = i + k;
      if (i + k < s.n_pages) list[i + k] = -1;
    }
    holes += th;
    moved += tm;
  }
  __syncthreads();
  for (int k = threadIdx.x; k < moved; k += kBook) {
    const int from = pairs[2 * k], to = pairs[2 * k + 1];
    list[from] = to;
    refs[to] = refs[from];
    refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    p.state[kPagesPairs] = moved;
    p.state[kPagesVersion] += 1;
  }
}

// Compaction, its moves: the workgroups take pieces of the moved pages in turn;
// each also maps a part of the tables.
__global__ void __launch_bounds__(kThreads)
pages_move_kernel(PagesShape s, PagesPtrs p, int pieces) {
  const int moved = min(max(p.state[kPagesPairs], 0), s.n_pages / 2);
  if (moved == 0) return;
  const int32_t* list = p.state + s.list;
  const int32_t* pairs = p.state + s.pairs;
  const size_t entries = (size_t)s.batch * s.max_pages;
  for (size_t i = blockIdx.x * (size_t)kThreads + threadIdx.x; i < entries;
       i += (size_t)gridDim.x * kThreads) {
    const int id = p.state[s.table + i];
    if (id < 0 || id >= s.n_pages) continue;
    const int to = list[id];
    if (to >= 0) p.state[s.table + i] = to;
  }
  const int planes = 2 * s.layers;
  const size_t work = (size_t)moved * planes * pieces;
  for (size_t i = blockIdx.x; i < work; i += gridDim.x) {
    const size_t m = i / pieces;
    const int piece = (int)(i - m * pieces), plane = (int)(m / moved);
    const int k = (int)(m - (size_t)plane * moved);
    copy_piece(s, p, plane, piece, clamp_page(s, pairs[2 * k]), clamp_page(s, pairs[2 * k + 1]));
  }
}

int pieces_of(const PagesShape& s) { return (int)((s.page_bytes + kPiece - 1) / kPiece); }

}  // namespace

hipError_t launch_pages_reset(const PagesShape& s, const PagesPtrs& p, hipStream_t st) {
  // a launch holds fewer than 2^32 threads, the largest state 2^35 words
  const size_t wgs = (s.words + kBook - 1) / kBook;
  hipLaunchKernelGGL(pages_reset_kernel, dim3((unsigned)(wgs < 65536 ? wgs : 65536)), dim3(kBook), 0,
                     st, s, p);
  return hipGetLastError();
}

hipError_t launch_pages_clear_flags(const PagesPtrs& p, hipStream_t st) {
  hipLaunchKernelGGL(pages_clear_flags_kernel, dim3(1), dim3(1), 0, st, p);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const PagesShape& s, const PagesPtrs& p, const int32_t* n_new,
                                int max_new, hipStream_t st) {
  hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(kBook), 0, st, s, p, n_new, max_new);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_part_kernel, dim3(pieces_of(s), 2 * s.layers, s.batch), dim3(kThreads),
                     0, st, s, p);
  return hipGetLastError();
}

hipError_t launch_pages_write(const PagesShape& s, const PagesPtrs& p, int layer, int n_layers,
                              const void* K, const void* V, int max_new, hipStream_t st) {
  // tiles begin at a multiple of 16 bytes, up to a run less one before the rows
  const dim3 grid((max_new + 16 / (int)s.el + 30) / 32, n_layers * s.hkv, s.batch);
  if (s.dtype == LDR_BF16)
    hipLaunchKernelGGL(pages_write_kernel<uint16_t>, grid, dim3(kThreads), 0, st, s, p, layer,
                       n_layers, static_cast<const uint16_t*>(K),
                       static_cast<const uint16_t*>(V), max_new);
  else
    hipLaunchKernelGGL(pages_write_kernel<float>, grid, dim3(kThreads), 0, st, s, p, layer,
                       n_layers, static_cast<const float*>(K), static_cast<const float*>(V),
                       max_new);
  return hipGetLastError();
}

hipError_t launch_pages_keep(const PagesShape& s, const PagesPtrs& p, const int32_t* kept,
                             hipStream_t st) {
  hipLaunchKernelGGL(pages_keep_kernel, dim3(1), dim3(kBook), 0, st, s, p, kept);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesShape& s, const PagesPtrs& p, const int32_t* src,
                             hipStream_t st) {
  hipLaunchKernelGGL(pages_fork_kernel, dim3(s.batch), dim3(kThreads), 0, st, s, p, src);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesShape& s, const PagesPtrs& p, hipStream_t st) {
  hipLaunchKernelGGL(pages_moves_kernel, dim3(1), dim3(kBook), 0, st, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_move_kernel, dim3(2048), dim3(kThreads), 0, st, s, p, pieces_of(s));
  return hipGetLastError();
}

}  // namespace ldr
