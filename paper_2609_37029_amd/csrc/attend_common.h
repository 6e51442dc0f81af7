// What the attention kernels over the paged cache share: the plan's items and
// layout (attend.hip writes them), matrix products, and the joining of partial
// results. Included by one source file a kind of cache, hence the unnamed namespace.
#ifndef LDR_ATTEND_COMMON_H
#define LDR_ATTEND_COMMON_H

#include <type_traits>

#include "serve_internal.h"

namespace ldr {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWideThreads = 512;
constexpr int kBook = 1024;          // threads of the plan's workgroup
constexpr int kStep = 32;            // keys of a step; a page holds whole steps
constexpr int kStage = 64;           // keys of a stage of the bf16 main kernel
// Keys in common that are worth a segment of their own. 64 sequences with one row, 300
// keys of their own and as many in common, two layers: 77 us with the segment and 88
// without at 256 keys, 76 and 97 at 512.
constexpr int kMinShared = 256;
// Keys of a sequence's own that are worth items; fewer are left to the last kernel. 64
// sequences as above with 32768 keys in common: 167 us, 181 if their 256 keys become
// items; with 700 keys of their own 139 us, 154 if they do not. Fresh prompts, all rows
// open, a layer: one of 300 14.7 us, 20.2 if its 256 keys become items; one of 512 20.2 and
// 26.0, eight of 300 55 and 59, but four of 512 61 and 54.
constexpr int kMinMain = 512;
constexpr int kBlock = 32;           // rows of a block of partial results

// Tiles of a dtype's main kernel: rows of an item, the keys that an item's are a
// multiple of (four stages: the bf16 kernel's loop has no branch), workgroups that
// the plan cuts the work for, and the keys whose work an item costs on top of its own
// (its start, and writing and joining its part). 256 bf16 workgroups run at once (by their
// LDS with head_dim 128, by the registers that the kernel asks for with 64); 768 of fp32 run
// with head_dim 64 and 256 with 128, and are cut for as 512.
struct Tile { int rows, unit, slots, cost; };
__host__ __device__ constexpr Tile tile_of(bool bf16) {
  return bf16 ? Tile{256, 4 * kStage, 256, 384} : Tile{32, 128, 512, 192};
}
__host__ __device__ inline Tile tile_of(const PagesShape& s) { return tile_of(s.dtype != LDR_F32); }
// Whether 65 to 96 rows are two tiles, of 64 rows and of the rest. With 4 bits and head_dim 128
// 16 sequences with 68 rows a K/V head over 8192 keys, five layers, take 408 us so and 419 as
// one tile; one with 68 over 16384, two layers, 61 and 66; 16 with 96 over 8192 171 and 175. (8
// with 68 over 4096 76 and 70, 64 over 2000 189 and 179: short ones are slower.) With 8 bits
// two tiles load and decode twice the bytes: the first 501 and 437, 32 with 72 over 4096 241
// and 192, none slower as one. With head_dim 64 16 with 80 over 4096, 4 bits, 61 and 60.
__host__ __device__ inline bool two_tiles(const PagesShape& s) { return s.bits == 4 && s.d == 128; }
// Rows of the tiles of a segment of R rows.
__host__ __device__ inline int tile_rows(const Tile& t, bool two, int R) {
  return two && R > 64 && R <= 96 ? 64 : t.rows;
}
// Rounds of items over those workgroups, at most (4 took 2% longer: the
// grid is sized for as many, and most of it ends at once).
constexpr int kMaxRounds = 2;

__device__ inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// One unit of work: rows r0 .. r0 + nr of a segment over keys k0 .. k1 of
// sequence seq. Row r belongs to the segment's query r / rep, entry q0 + r / rep
// of the row map, head r % rep of the group. Partial results go to blocks of 32
// rows from `part` on.
struct Item { int q0, r0, nr, seq, k0, k1, part, pad; };

// A sequence: its first entry in the row map, open rows, keys, and the keys it
// leaves to its group; its own chunks of `step` keys (0: none), chunk c of its
// row r in block own_part + c own_blocks + r / 32; the same for its group's chunks
// and its row grp_off + r there.
struct SeqInfo {
  int qoff, open, rows, share, step, own_part, own_chunks, own_blocks;
  int grp_part, grp_chunks, grp_blocks, grp_off, pad[4];
};
static_assert(sizeof(Item) == 32 && sizeof(SeqInfo) == 64, "read as words");

// Keys, from `share` on, that every row of the tile from row t on sees and items
// can take: whole units.
__device__ inline int tile_keys(int rows, int open, int share, int t, int rep, int unit) {
  return max(0, rows - open + t / rep + 1 - share) / unit * unit;
}

struct Header { int version, hq, max_new, items, id, pad[59]; };

struct AttendWs {          // byte offsets in the workspace
  size_t map, info, items, ml, o, bytes;
  int max_items;
  int tiles;               // of 32 rows of a sequence
  long blocks;             // of partial results, per K/V head
};

// Items of one K/V head that the chunks add to a cut by tiles alone.
__host__ __device__ inline int added_items(const PagesShape& s) {
  return kMaxRounds * tile_of(s).slots / s.hkv + 1;
}

AttendWs plan_ws(const PagesShape& s, int hq, int max_new) {
  AttendWs w;
  const int rep = hq / s.hkv, tile = tile_of(s).rows;
  const long rows = (long)s.batch * max_new * rep;
  // every tile of the own and of the shared segments once, and the added ones
  const long tiles = ((long)max_new * rep + tile - 1) / tile;
  w.max_items = (int)(s.batch * tiles + rows / tile + s.batch / 2 + added_items(s));
  if (two_tiles(s)) w.max_items += s.batch + s.batch / 2;   // the second of 65 to 96 rows
  w.tiles = (int)(((long)max_new * rep + kBlock - 1) / kBlock);
  w.blocks = (long)s.batch * w.tiles + rows / kBlock + s.batch / 2 +
             (long)(tile / kBlock) * added_items(s);
  size_t off = sizeof(Header);
  w.map = off; off = align_up(off + (size_t)s.batch * max_new * 4);
  w.info = off; off = align_up(off + (size_t)s.batch * sizeof(SeqInfo));
  w.items = off; off = align_up(off + (size_t)w.max_items * sizeof(Item));
  w.ml = off; off = align_up(off + (size_t)s.hkv * w.blocks * kBlock * 8);
  w.o = off; off = align_up(off + (size_t)s.hkv * w.blocks * kBlock * s.d * 4);
  w.bytes = off;
  return w;
}

__device__ inline int clamp_rows(const PagesShape& s, int r) {
  return min(max(r, 0), s.max_pages * s.page);
}
__device__ inline int clamp_page(const PagesShape& s, int id) {
  return min(max(id, 0), s.n_pages - 1);
}

// Matrix products of 32 x 32 tiles. A fragment is 16 bytes a lane: E elements
// of row (or column) lane % 32, the E that half lane / 32 holds of 2 E
// consecutive ones. The accumulator of lane l holds column l % 32; entry i is row
// 8 (i / 4) + 4 (l / 32) + i % 4.
//
// Probabilities of a bf16 cache are rounded to bf16 where they meet V, half a step (2^-8) of
// each at most; their sum takes them unrounded, so that lse is not touched. With a second
// product for what the rounding leaves, o differs from its definition by 0.0017 (root mean
// square, relative: its own rounding to bf16) instead of 0.0023, but it is half as much matrix
// work again: five layers of the sequences above take 436 instead of 393 us, 1110 instead of
// 893, 572 instead of 553 and 989 instead of 787. fp32 caches keep fp32.
template <typename T> struct Mma;
template <> struct Mma<uint16_t> {
  static constexpr int E = 8;
  __device__ static f32x16 run(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  __device__ static u32x4 pack(const float* x) {   // probabilities, rounded to bf16
    bf16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (__bf16)x[j];
    return __builtin_bit_cast(u32x4, v);
  }
  __device__ static void store4(uint16_t* o, const float* x) {
    uint2 v{f32_to_bf16(x[0]) | (uint32_t)f32_to_bf16(x[1]) << 16,
            f32_to_bf16(x[2]) | (uint32_t)f32_to_bf16(x[3]) << 16};
    *reinterpret_cast<uint2*>(o) = v;
  }
  __device__ static float get(u32x4 v, int j) {
    return __uint_as_float(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16);
  }
};
template <> struct Mma<float> {
  static constexpr int E = 4;
  __device__ static f32x16 run(u32x4 a, u32x4 b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0,
                                               0, 0);
    return c;
  }
  __device__ static u32x4 pack(const float* x) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                 __float_as_uint(x[3])};
  }
  __device__ static void store4(float* o, const float* x) {
    *reinterpret_cast<float4*>(o) = float4{x[0], x[1], x[2], x[3]};
  }
  __device__ static float get(u32x4 v, int j) { return __uint_as_float(v[j]); }
};

struct AttendArgs {
  PagesShape s;
  PagesPtrs p;
  const void* q; long q_stride;
  void* o; float* lse;
  int layer, hq, rep, max_new;
  float scale;
  uint8_t* ws;
  AttendWs w;
};

// A word that an earlier launch wrote and this one only reads, at an address that
// a wave's lanes share: a scalar load into a scalar register.
__device__ inline int32_t scalar_word(const void* p, size_t i) {
  return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)p)[i];
}
__device__ inline Item scalar_item(const void* items, size_t i) {
  Item it;
  it.q0 = scalar_word(items, 8 * i); it.r0 = scalar_word(items, 8 * i + 1);
  it.nr = scalar_word(items, 8 * i + 2); it.seq = scalar_word(items, 8 * i + 3);
  it.k0 = scalar_word(items, 8 * i + 4); it.k1 = scalar_word(items, 8 * i + 5);
  it.part = scalar_word(items, 8 * i + 6); it.pad = 0;
  return it;
}

__device__ inline SeqInfo scalar_info(const void* infos, size_t i) {
  SeqInfo f;
  f.qoff = scalar_word(infos, 16 * i); f.open = scalar_word(infos, 16 * i + 1);
  f.rows = scalar_word(infos, 16 * i + 2); f.share = scalar_word(infos, 16 * i + 3);
  f.step = scalar_word(infos, 16 * i + 4); f.own_part = scalar_word(infos, 16 * i + 5);
  f.own_chunks = scalar_word(infos, 16 * i + 6); f.own_blocks = scalar_word(infos, 16 * i + 7);
  f.grp_part = scalar_word(infos, 16 * i + 8); f.grp_chunks = scalar_word(infos, 16 * i + 9);
  f.grp_blocks = scalar_word(infos, 16 * i + 10); f.grp_off = scalar_word(infos, 16 * i + 11);
  return f;
}

// Whether the workspace holds this handle's plan of the cache's present state for
// these sizes; a workgroup that finds none records it and leaves, before it follows a
// word of the plan. The handle's number stands for the layout of the workspace and of
// the cache: another cache may have counted as many changes.
__device__ inline bool plan_ok(const AttendArgs& a, int items) {
  const bool ok = scalar_word(a.ws, 0) == scalar_word(a.p.state, kPagesVersion) &&
                  scalar_word(a.ws, 1) == a.hq && scalar_word(a.ws, 2) == a.max_new &&
                  scalar_word(a.ws, 4) == a.p.id &&
                  items >= 0 && items <= a.w.max_items;
  if (!ok && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.p.state + kPagesFlags, kFlagPlan);
  return ok;
}

// The larger (the sum) of a lane's value and that of the lane 32 away.
__device__ inline float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
__device__ inline float half_max(float x) { return fmaxf(x, other_half(x)); }
__device__ inline float half_sum(float x) { return x + other_half(x); }

// What scales the results so far from their maximum m to another, mu = max c2. The
// product is rounded as mu was: fused with the difference it would leave mu's rounding
// error where the maximum stays, and every step would scale by it (fp32, 512 rows, each
// over 16384 keys of the score 7055: their mean off by 3.6e-3 instead of 1.7e-6).
__device__ inline float rescale(float m, float c2, float mu) {
#pragma clang fp contract(off)
  return __builtin_amdgcn_exp2f(m * c2 - mu);
}

// The value of the column 16, 8, 4, 2 or 1 to the side, of the same half. By turns
// for 8 and 4: of columns that agree at twice the distance, that is the same.
template <int OFF> __device__ inline float aside(float x) {
  const int v = __float_as_int(x);
  if constexpr (OFF == 16) return __int_as_float(__builtin_amdgcn_ds_swizzle(v, 0x401f));
  else return __int_as_float(__builtin_amdgcn_update_dpp(
      0, v, OFF == 8 ? 0x128 : OFF == 4 ? 0x124 : OFF == 2 ? 0x4e : 0xb1, 0xf, 0xf, true));
}

// V where a mask crosses a step: keys from k1 on hold anything and count as 0. A
// value that is not finite but masked for some rows only would reach them as
// 0 x inf: it is taken out here (true: there was one), to be added to the rows
// that see it when they are written. `k`: the key of the fragment's first element.
template <typename T> __device__ inline bool clean_values(u32x4& v, int k, int k1) {
  constexpr int E = Mma<T>::E;
#pragma unroll
  for (int j = 0; j < E; ++j)
    if (k + j >= k1) {
      if constexpr (E == 8) v[j >> 1] &= j & 1 ? 0x0000ffffu : 0xffff0000u;
      else v[j] = 0u;
    }
  bool bad = false;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    const bool inf = !(fabsf(Mma<T>::get(v, j)) < INFINITY);
    bad = bad || inf;
    if constexpr (E == 8) v[j >> 1] &= !inf ? 0xffffffffu : j & 1 ? 0x0000ffffu : 0xffff0000u;
    else v[j] = inf ? 0u : v[j];
  }
  return bad;
}

// A block's partial results: O^T as the matrix products leave it, 16 bytes a lane
// behind one another, and (m, l) of its rows. m is in units of the scores.
template <int D> __device__ inline float* part_o(const AttendArgs& a, int head, long block) {
  return reinterpret_cast<float*>(a.ws + a.w.o) + (head * a.w.blocks + block) * kBlock * D;
}
__device__ inline float2* part_ml(const AttendArgs& a, int head, long block) {
  return reinterpret_cast<float2*>(a.ws + a.w.ml) + (head * a.w.blocks + block) * kBlock;
}

// The maximum that is taken out of a row's exponents follows the scores only when they
// pass it by 2^kLazy, and is a whole power of two in the base of the exponential.
constexpr float kLazy = 8.f;

// The chunk of row r lies at its own number with these bits flipped, rows of C
// chunks: 16 rows then have 16 places mod 256 bytes.
template <int C> __device__ inline int turn(int r) {
  static_assert(C == 16 || C == 8, "rows of 256 or 128 bytes");
  return C == 16 ? r & 15 : (r >> 1) & 7;
}
}  // namespace
}  // namespace ldr
#endif
