// Rows into a coded cache and rows out of any cache.
//
// One workgroup per (32 positions, layer and head, sequence), on two pages at most, as
// for rows of bf16 and fp32. Tiles begin at multiples of 16 positions: V's pairs and
// scales are stored by runs of 16 bytes along the positions, and no two workgroups write
// to one run. Four lanes have the 32 dimensions of a block; V's codes, a quarter of its
// rows' bytes or a half, are what goes through LDS.
//
// Bound by HBM. Measured, Qwen3-8B heads, five layers, pages of 64: 1536 rows of each of two
// sequences into 8 bits 22 us (95 MB in and out, 4.3 TB/s) and back 20 us; 16 x 13 rows into 4
// bits 7 us and back 5; 49700 rows of 4 bits out 283 us (1.3 GB, 4.6 TB/s), of 8 bits 305 (1.5 GB,
// 5.1 TB/s), of bf16 376 (2.0 GB, 5.4 TB/s), of fp32 795 (4.1 GB, 5.1 TB/s).
#include "mx.h"

namespace ldr {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 32;        // positions of a workgroup
constexpr int kRun = 16;         // positions a tile's start is a multiple of

__device__ inline int clamp_rows(const PagesShape& s, int r) {
  return min(max(r, 0), s.max_pages * s.page);
}
__device__ inline int clamp_page(const PagesShape& s, int id) {
  return min(max(id, 0), s.n_pages - 1);
}

// A tile of positions lo .. hi - 1 of a sequence, in one layer's K and V of one head.
struct Place {
  uint8_t *k, *v;          // the planes, at the head
  size_t page_bytes;
  int page, j0, id0, id1;
  __device__ Place(const PagesShape& s, const PagesPtrs& p, int b, int layer, int h, int lo, int hi)
      : page_bytes(s.page_bytes), page(s.page), j0(lo / s.page) {
    const int32_t* table = p.state + s.table + (size_t)b * s.max_pages;
    id0 = clamp_page(s, table[j0]);
    id1 = clamp_page(s, table[(hi - 1) / s.page]);
    k = p.pool + (size_t)2 * layer * s.n_pages * s.page_bytes + h * s.head_bytes;
    v = k + (size_t)s.n_pages * s.page_bytes;
  }
  __device__ uint8_t* of(uint8_t* plane, int pos) const {     // the page of a position
    return plane + (size_t)(pos / page == j0 ? id0 : id1) * page_bytes;
  }
};

// The largest of a quad of lanes.
__device__ inline uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, false));
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, false));
}

// Eight dimensions of a row, a quarter of a block that a quad of lanes has: their codes,
// and the block's scale.
template <int BITS> __device__ inline uint32_t encode8(uint4 in, uint32_t* out) {
  const uint32_t w[4] = {in.x, in.y, in.z, in.w};
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max(w[i] >> 16 & 0x7fffu, w[i] & 0x7fffu));
  top = quad_max(top);
  const float t = Mx<BITS>::kTop;
  const int e = mx_exponent<BITS>(fminf(bf16_to_f32((uint16_t)top), t));
  const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_amdgcn_fmed3f(__uint_as_float(w[i] << 16), -t, t);
    x[2 * i + 1] = __builtin_amdgcn_fmed3f(__uint_as_float(w[i] & 0xffff0000u), -t, t);
  }
  const bool bad = top >= 0x7f80u;
  if constexpr (BITS == 4) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
    out[0] = bad ? 0u : c;
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      i16x2 c = {};
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, x[4 * i], x[4 * i + 1], scale, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, x[4 * i + 2], x[4 * i + 3], scale, true);
      out[i] = bad ? 0u : __builtin_bit_cast(uint32_t, c);
    }
  }
  return bad ? 255u : (uint32_t)(e + 127);
}

// The bytes of a run of 16 along the positions from pos on: those of positions lo .. hi - 1
// from LDS, UNIT bytes a position `ld` apart; the others stay.
template <int UNIT>
__device__ inline void store_run(uint8_t* out, const uint8_t* lds, int ld, int pos, int lo, int hi) {
  constexpr int N = 16 / UNIT;
  alignas(16) uint8_t x[16];
  if (pos < lo || pos + N > hi) *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(out);
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (pos + k >= lo && pos + k < hi)
#pragma unroll
      for (int u = 0; u < UNIT; ++u) x[k * UNIT + u] = lds[(pos + k - lo) * ld + u];
  *reinterpret_cast<uint4*>(out) = *reinterpret_cast<const uint4*>(x);
}

template <int BITS>
__global__ void __launch_bounds__(kThreads)
pages_write_mx_kernel(PagesShape s, PagesPtrs p, int layer0, int n_layers, const uint16_t* K,
                      const uint16_t* V, int max_new) {
  constexpr int UNIT = BITS / 4, LD = 128 * BITS / 8 + 4, LS = 4 + 1, N = 16 / UNIT;
  __shared__ alignas(16) uint8_t codes[kTile * LD], scales[kTile * LS];
  const int b = blockIdx.z, h = blockIdx.y % s.hkv, l = blockIdx.y / s.hkv;
  const int rows = clamp_rows(s, p.state[s.rows + b]);
  const int open = min(max(p.state[s.open + b], 0), rows);
  const int start = rows - open, end = start + min(open, max_new);
  const int first = start / kRun * kRun + (int)blockIdx.x * kTile;
  if (first >= end) return;
  const int lo = max(first, start), hi = min(first + kTile, end), cnt = hi - lo;
  const Place at(s, p, b, layer0 + l, h, lo, hi);
  const int rowb = s.d * BITS / 8, blocks = s.d / kMxBlock;
  const size_t row = (size_t)n_layers * s.hkv * s.d;
  const size_t in0 = ((size_t)b * max_new + (lo - start)) * row + ((size_t)l * s.hkv + h) * s.d;
  const int c = s.d / 8;                      // pieces of 8 dimensions: whole quads a row
  for (int i = threadIdx.x; i < cnt * c; i += kThreads) {
    const int r = i / c, e = i - r * c, off = (lo + r) % s.page;
    const uint4 kx = *reinterpret_cast<const uint4*>(K + in0 + r * row + e * 8);
    const uint4 vx = *reinterpret_cast<const uint4*>(V + in0 + r * row + e * 8);
    uint32_t kc[2], vc[2];
    const uint32_t ks = encode8<BITS>(kx, kc), vs = encode8<BITS>(vx, vc);
    uint8_t* kp = at.of(at.k, lo + r);
    uint8_t* kr = kp + (size_t)off * rowb + e * BITS;
    uint8_t* vr = codes + r * LD + e * BITS;
    *reinterpret_cast<uint32_t*>(vr) = vc[0];
    if constexpr (BITS == 4) {
      *reinterpret_cast<uint32_t*>(kr) = kc[0];
    } else {
      *reinterpret_cast<uint2*>(kr) = uint2{kc[0], kc[1]};
      *reinterpret_cast<uint32_t*>(vr + 4) = vc[1];
    }
    if (e % 4 == 0) {
      kp[(size_t)s.page * rowb + off * blocks + e / 4] = (uint8_t)ks;
      scales[r * LS + e / 4] = (uint8_t)vs;
    }
  }
  __syncthreads();
  const int runs = kTile / N;
  for (int i = threadIdx.x; i < s.d / 2 * runs; i += kThreads) {
    const int pair = i / runs, pos = first + (i - pair * runs) * N;
    if (pos + N <= lo || pos >= hi) continue;
    store_run<UNIT>(at.of(at.v, max(pos, lo)) + ((size_t)pair * s.page + pos % s.page) * UNIT,
                    codes + pair * UNIT, LD, pos, lo, hi);
  }
  for (int i = threadIdx.x; i < blocks * (kTile / kRun); i += kThreads) {
    const int block = i / (kTile / kRun), pos = first + i % (kTile / kRun) * kRun;
    if (pos + kRun <= lo || pos >= hi) continue;
    store_run<1>(at.of(at.v, max(pos, lo)) + (size_t)s.page * rowb + block * s.page + pos % s.page,
                 scales + block, LS, pos, lo, hi);
  }
}

// Whether a read's range is within the sequence; else the first workgroup of the sequence
// says so.
__device__ inline bool read_range(const PagesShape& s, const PagesPtrs& p, const int32_t* first,
                                  const int32_t* n, int max_rows, int b, int* start, int* count) {
  const int rows = clamp_rows(s, p.state[s.rows + b]);
  *start = first[b];
  *count = n[b];
  const bool ok = *count >= 0 && *count <= max_rows && *count <= rows && *start >= 0 &&
                  *start <= rows - *count;
  if (!ok && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0)
    atomicOr(p.state + kPagesFlags, kFlagRange);
  return ok;
}

// BITS: 4 or 8, or 0 for rows of T as they are.
template <typename T, int BITS>
__global__ void __launch_bounds__(kThreads)
pages_read_kernel(PagesShape s, PagesPtrs p, int layer0, int n_layers, const int32_t* firsts,
                  const int32_t* counts, T* K, T* V, int max_rows) {
  constexpr int E = 16 / (int)sizeof(T), LD = 128 + E;
  constexpr int N = BITS ? 8 : E, RUNS = kTile / N;     // positions a load of V
  __shared__ alignas(16) T tile[kTile * LD];
  const int b = blockIdx.z, h = blockIdx.y % s.hkv, l = blockIdx.y / s.hkv;
  int start, count;
  if (!read_range(s, p, firsts, counts, max_rows, b, &start, &count)) return;
  const int end = start + count, first = start / kRun * kRun + (int)blockIdx.x * kTile;
  if (first >= end) return;
  const int lo = max(first, start), hi = min(first + kTile, end), cnt = hi - lo;
  const Place at(s, p, b, layer0 + l, h, lo, hi);
  const size_t row = (size_t)n_layers * s.hkv * s.d;
  const size_t out0 = ((size_t)b * max_rows + (lo - start)) * row + ((size_t)l * s.hkv + h) * s.d;
  const int c = s.d / E;                      // 16-byte pieces of a row
  if constexpr (BITS == 0) {
    for (int i = threadIdx.x; i < s.d * RUNS; i += kThreads) {
      const int dim = i / RUNS, pos = first + (i - dim * RUNS) * N;
      if (pos + N <= lo || pos >= hi) continue;
      alignas(16) T x[E];
      *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(
          reinterpret_cast<const T*>(at.of(at.v, max(pos, lo))) + (size_t)dim * s.page + pos % s.page);
#pragma unroll
      for (int k = 0; k < E; ++k) tile[(pos + k - first) * LD + dim] = x[k];
    }
  } else {
    const int rowb = s.d * BITS / 8;
    for (int i = threadIdx.x; i < s.d / 2 * RUNS; i += kThreads) {
      const int pair = i / RUNS, pos = first + (i - pair * RUNS) * N;
      if (pos + N <= lo || pos >= hi) continue;
      const uint8_t* vp = at.of(at.v, max(pos, lo));
      const int in = pos % s.page;
      uint32_t w[BITS / 2], x[8];
      if constexpr (BITS == 4) {
        const uint2 t = *reinterpret_cast<const uint2*>(vp + (size_t)pair * s.page + in);
        w[0] = t.x; w[1] = t.y;
      } else {
        const uint4 t = *reinterpret_cast<const uint4*>(vp + 2 * ((size_t)pair * s.page + in));
        w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w;
      }
      const uint2 sc = *reinterpret_cast<const uint2*>(vp + (size_t)s.page * rowb +
                                                       pair / (kMxBlock / 2) * s.page + in);
      mx_rows8<BITS>(w, sc.x, sc.y, x);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        *reinterpret_cast<uint32_t*>(tile + (pos + k - first) * LD + 2 * pair) = x[k];
    }
  }
  for (int i = threadIdx.x; i < cnt * c; i += kThreads) {
    const int r = i / c, e = (i - r * c) * E, off = (lo + r) % s.page;
    const uint8_t* kp = at.of(at.k, lo + r);
    uint4 x;
    if constexpr (BITS == 0) {
      x = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(kp) + (size_t)off * s.d + e);
    } else {
      const int rowb = s.d * BITS / 8;
      const uint8_t* kc = kp + (size_t)off * rowb + e * BITS / 8;
      const float scale =
          mx_scale<0>(kp[(size_t)s.page * rowb + off * (s.d / kMxBlock) + e / kMxBlock]);
      uint32_t w[2] = {*reinterpret_cast<const uint32_t*>(kc), 0}, o[4];
      if constexpr (BITS == 8) w[1] = *reinterpret_cast<const uint32_t*>(kc + 4);
      mx_eight<BITS>(w, scale, o);
      x = uint4{o[0], o[1], o[2], o[3]};
    }
    *reinterpret_cast<uint4*>(K + out0 + r * row + e) = x;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < cnt * c; i += kThreads) {
    const int r = i / c, e = (i - r * c) * E;
    *reinterpret_cast<uint4*>(V + out0 + r * row + e) =
        *reinterpret_cast<const uint4*>(tile + (lo - first + r) * LD + e);
  }
}

// tiles begin at a multiple of kRun, up to kRun - 1 before the rows
dim3 grid_of(const PagesShape& s, int n_layers, int rows) {
  return dim3((rows + kRun - 1 + kTile - 1) / kTile, n_layers * s.hkv, s.batch);
}

}  // namespace

hipError_t launch_pages_write_mx(const PagesShape& s, const PagesPtrs& p, int layer, int n_layers,
                                 const void* K, const void* V, int max_new, hipStream_t st) {
  const uint16_t *k = static_cast<const uint16_t*>(K), *v = static_cast<const uint16_t*>(V);
  const dim3 grid = grid_of(s, n_layers, max_new);
  if (s.bits == 4)
    hipLaunchKernelGGL(pages_write_mx_kernel<4>, grid, dim3(kThreads), 0, st, s, p, layer, n_layers,
                       k, v, max_new);
  else
    hipLaunchKernelGGL(pages_write_mx_kernel<8>, grid, dim3(kThreads), 0, st, s, p, layer, n_layers,
                       k, v, max_new);
  return hipGetLastError();
}

hipError_t launch_pages_read(const PagesShape& s, const PagesPtrs& p, int layer, int n_layers,
                             const int32_t* first, const int32_t* n, void* K, void* V,
                             int max_rows, hipStream_t st) {
  const dim3 grid = grid_of(s, n_layers, max_rows), threads(kThreads);
  uint16_t *k = static_cast<uint16_t*>(K), *v = static_cast<uint16_t*>(V);
  if (s.dtype == LDR_F32)
    hipLaunchKernelGGL((pages_read_kernel<float, 0>), grid, threads, 0, st, s, p, layer, n_layers,
                       first, n, static_cast<float*>(K), static_cast<float*>(V), max_rows);
  else if (s.bits == 0)
    hipLaunchKernelGGL((pages_read_kernel<uint16_t, 0>), grid, threads, 0, st, s, p, layer, n_layers,
                       first, n, k, v, max_rows);
  else if (s.bits == 4)
    hipLaunchKernelGGL((pages_read_kernel<uint16_t, 4>), grid, threads, 0, st, s, p, layer, n_layers,
                       first, n, k, v, max_rows);
  else
    hipLaunchKernelGGL((pages_read_kernel<uint16_t, 8>), grid, threads, 0, st, s, p, layer, n_layers,
                       first, n, k, v, max_rows);
  return hipGetLastError();
}

}  // namespace ldr
