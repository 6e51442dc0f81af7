// Causal attention of the open rows over the paged K/V cache, with the pages
// that sequences have in common at the front read once for all of them.
//
// softmax(q K^T) V over a row's keys is the join of its parts over disjoint key
// ranges: a part gives its maximum m, l = sum e^{s - m} and O = sum e^{s - m} v,
// and parts add up after scaling by e^{m_part - m}. So the work is cut into
// segments (rows x keys): the rows of a group of sequences over the keys they
// share, and the rows of each sequence over its own keys. A segment is cut into
// tiles of rows and chunks of keys, enough items to fill the GPU. A plan kernel
// writes the list of items (the lengths are on the device), one workgroup takes
// an item of one K/V head, and a last kernel joins the parts of each row.
#include "ldr_internal.h"

namespace ldr {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kBook = 1024;          // threads of the plan's workgroup: one per sequence
constexpr int kRows = 32;            // query rows (x heads of a group) of an item
constexpr int kKeys = 32;            // keys of a step; a page holds whole steps
constexpr int kTarget = 1024;        // items x K/V heads aimed at
constexpr int kWideRows = 256;       // rows of an item of the wide kernel
constexpr int kWideFrom = 97;        // rows of a segment that go to it (bf16)
constexpr int kWideTarget = 256;     // its items x K/V heads: one a CU
constexpr int kMinChunk = 256;       // keys of an item, at least (but for a segment's end)
constexpr int kMinShared = 128;      // keys in common that are worth a segment of their own
constexpr int kNoMask = 1 << 30;

// One unit of work: rows r0 .. r0 + nr of a segment over keys k0 .. k1 of
// sequence seq. Row r belongs to the segment's query r / rep, entry q0 + r / rep
// of the row map, head r % rep of the group; it sees keys up to cbase + r / rep.
// Its partial results go to rows part + (r - r0); part < 0: the row has no other
// part and is finished at once.
struct Item { int q0, r0, nr, seq, k0, k1, cbase, part; };

// Parts of a sequence's rows: entries [own_part + c own_rows + own row] for its
// own chunks c, the same for its group's. qoff: its first entry in the row map.
struct SeqInfo { int own_part, own_chunks, own_rows, qoff; int grp_part, grp_chunks, grp_rows, grp_qoff; };

// The wide kernel's items come first in the list.
struct Header { int version, hq, max_new, items, wide, rows, pad[58]; };

struct AttendWs {          // byte offsets in the workspace
  size_t map, info, items, ml, o, bytes;
  int max_items, max_wide;
  long part_rows;          // rows of partial results, per K/V head
};

// Whether a segment of `rows` rows goes to the wide kernel.
__host__ __device__ inline bool is_wide(const PagesShape& s, long rows) {
  return s.dtype == LDR_BF16 && rows >= kWideFrom;
}

AttendWs plan_ws(const PagesShape& s, int hq, int max_new) {
  AttendWs w;
  const int rep = hq / s.hkv;
  const long rows = (long)s.batch * max_new * rep;
  // every tile once, and the chunks that the cut into about the targets' items adds
  const long tiles = (long)s.batch * (((long)max_new * rep + kRows - 1) / kRows) + rows / kRows +
                     s.batch / 2;
  w.max_items = (int)(tiles + kTarget / s.hkv + 1 + kWideTarget / s.hkv + 1);
  const long wide = 2 * (rows / kWideRows + s.batch) + kWideTarget / s.hkv + 1;
  w.max_wide = is_wide(s, rows) ? (int)(wide < w.max_items ? wide : w.max_items) : 0;
  w.part_rows = 2 * rows + (long)kRows * (kTarget / s.hkv + 1) +
                (long)kWideRows * (kWideTarget / s.hkv + 1);
  size_t off = sizeof(Header);
  w.map = off; off = align_up(off + (size_t)s.batch * max_new * 4);
  w.info = off; off = align_up(off + (size_t)s.batch * sizeof(SeqInfo));
  w.items = off; off = align_up(off + (size_t)w.max_items * sizeof(Item));
  w.ml = off; off = align_up(off + (size_t)s.hkv * w.part_rows * 8);
  w.o = off; off = align_up(off + (size_t)s.hkv * w.part_rows * s.d * 4);
  w.bytes = off;
  return w;
}

__device__ inline int clamp_rows(const PagesShape& s, int r) {
  return min(max(r, 0), s.max_pages * s.page);
}
__device__ inline int clamp_page(const PagesShape& s, int id) {
  return min(max(id, 0), s.n_pages - 1);
}

// Sum over the workgroup before this thread, and the total.
__device__ inline long block_scan(long v, long* sums, long* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long inc = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const long o = __shfl_up(inc, off);
    if (lane >= off) inc += o;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = inc;
  __syncthreads();
  long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kBook / 64; ++w) {
    before += w < wave ? sums[w] : 0;
    all += sums[w];
  }
  *total = all;
  return before + inc - v;
}

__device__ inline long ceil_div(long a, long b) { return (a + b - 1) / b; }

__global__ void __launch_bounds__(kBook)
attend_plan_kernel(PagesShape s, PagesPtrs p, int hq, int max_new, const int32_t* groups,
                   uint8_t* ws, AttendWs w) {
  __shared__ long sums[kBook / 64];
  __shared__ int label[kBook], lead[kBook], opens[kBook], fulls[kBook], common[kBook],
      qoffs[kBook], members[kBook];
  __shared__ int w_off[kBook], kinds[kBook], i_off[kBook], o_tiles[kBook], o_chunks[kBook], g_tiles[kBook], g_chunks[kBook],
      o_part[kBook], g_part[kBook], ends[kBook], shares[kBook];
  const int b = threadIdx.x, rep = hq / s.hkv;
  const bool in = b < s.batch;
  const int32_t* table = p.state + s.table;
  Header* hd = reinterpret_cast<Header*>(ws);
  int32_t* map = reinterpret_cast<int32_t*>(ws + w.map);
  SeqInfo* info = reinterpret_cast<SeqInfo*>(ws + w.info);
  Item* items = reinterpret_cast<Item*>(ws + w.items);

  const int all = in ? clamp_rows(s, p.state[s.rows + b]) : 0;
  const int held = in ? min(max(p.state[s.open + b], 0), all) : 0;
  const int open = min(held, max_new);
  const int rows = all - held + open;        // the keys that a query of the plan can see
  const int full = (all - held) / s.page;    // whole pages before the open rows
  // a sequence that has nothing to share stands alone
  const int own = -1 - b;
  int lb = own;
  if (open > 0 && full > 0) {
    if (groups) lb = groups[b] >= 0 ? groups[b] : own;
    else lb = clamp_page(s, table[(size_t)b * s.max_pages]);
  }
  label[b] = lb;
  opens[b] = open;
  fulls[b] = full;
  common[b] = full;
  members[b] = 0;
  __syncthreads();
  int ld = b;
  if (in && lb >= 0)
    for (int i = 0; i < b; ++i)
      if (label[i] == lb) { ld = i; break; }
  lead[b] = ld;
  if (in && open > 0) atomicAdd(&members[ld], 1);
  __syncthreads();
  // pages in common with the first of the group, one wave per sequence
  for (int c = threadIdx.x >> 6; c < s.batch; c += kBook / 64) {
    const int l = lead[c];
    if (l == c) continue;
    const int lim = min(fulls[c], fulls[l]);
    const int32_t* tc = table + (size_t)c * s.max_pages;
    const int32_t* tl = table + (size_t)l * s.max_pages;
    int same = lim;
    for (int j = 0; j < lim; j += 64) {
      const int k = j + (threadIdx.x & 63);
      const uint64_t diff = __ballot(k < lim && tc[k] != tl[k]);
      if (diff) { same = j + __builtin_ctzll(diff); break; }
    }
    if ((threadIdx.x & 63) == 0) atomicMin(&common[l], same);
  }
  __syncthreads();
  const int share_rows = common[ld] * s.page;
  const int share = members[ld] > 1 && share_rows >= kMinShared ? share_rows : 0;
  // row map: the sequences of a group behind one another
  int qoff = 0, gopen = 0;
  for (int i = 0; i < s.batch; ++i) {
    const int l = lead[i], o = opens[i];
    qoff += l < ld || (l == ld && i < b) ? o : 0;
    gopen += l == ld ? o : 0;
  }
  qoffs[b] = qoff;
  // segments: own rows over own keys; the group's rows over the shared ones
  const long R = (long)open * rep, Rg = share && ld == b ? (long)gopen * rep : 0;
  const int len = rows - share;
  const bool ow = is_wide(s, R), gw = is_wide(s, Rg);
  const int ot = (int)ceil_div(R, ow ? kWideRows : kRows),
            gt = (int)ceil_div(Rg, gw ? kWideRows : kRows);
  const long own_work = (long)ot * len, grp_work = (long)gt * share;
  long work = 0, wide_work = 0;
  long before = block_scan((ow ? 0 : own_work) + (gw ? 0 : grp_work), sums, &work);
  block_scan((ow ? own_work : 0) + (gw ? grp_work : 0), sums, &wide_work);
  const long per = max(1, kTarget / s.hkv), wide_per = max(1, kWideTarget / s.hkv);
  const long narrow_chunk = max((long)kMinChunk, ceil_div(ceil_div(work, per), 64) * 64L);
  const long wide_chunk = max((long)kMinChunk, ceil_div(ceil_div(wide_work, wide_per), 64) * 64L);
  const int oc = open ? (int)ceil_div(len, ow ? wide_chunk : narrow_chunk) : 0;
  const int gc = Rg ? (int)ceil_div(share, gw ? wide_chunk : narrow_chunk) : 0;
  // the list: wide items, then the others, each in the order of the sequences,
  // a sequence's own before its group's
  const long oi = (long)ot * oc, gi = (long)gt * gc;
  long n_items = 0, n_wide = 0;
  const long woff = block_scan((ow ? oi : 0) + (gw ? gi : 0), sums, &n_wide);
  const long noff = n_wide + block_scan((ow ? 0 : oi) + (gw ? 0 : gi), sums, &n_items);
  n_items += n_wide;
  const bool direct = !share && oc == 1;
  long n_part = 0;
  before = block_scan((direct ? 0 : oc * R) + gc * Rg, sums, &n_part);
  w_off[b] = (int)woff;
  i_off[b] = (int)noff;
  kinds[b] = (ow ? 1 : 0) | (gw ? 2 : 0);
  o_tiles[b] = ot; o_chunks[b] = oc; g_tiles[b] = gt; g_chunks[b] = gc;
  o_part[b] = direct ? -1 : (int)before;
  g_part[b] = (int)(before + (direct ? 0 : oc * R));
  ends[b] = rows;
  shares[b] = share;
  __syncthreads();
  if (in) {
    const int leader = share ? ld : b;
    info[b] = SeqInfo{o_part[b], oc, (int)R, qoff, g_part[leader], share ? g_chunks[leader] : 0,
                      share ? gopen * rep : 0, qoffs[leader]};
  }
  // holds by the bounds of plan_ws; a list that would not fit is left empty
  if (n_items > w.max_items || n_wide > w.max_wide || n_part > w.part_rows) n_items = n_wide = 0;
  long total = 0;
  block_scan(open, sums, &total);
  if (b == 0) {
    hd->version = p.state[kPagesVersion];
    hd->hq = hq;
    hd->max_new = max_new;
    hd->items = (int)n_items;
    hd->wide = (int)n_wide;
    hd->rows = (int)total;
  }
  for (int c = threadIdx.x >> 6; c < s.batch; c += kBook / 64)
    for (int i = threadIdx.x & 63; i < opens[c]; i += 64) map[qoffs[c] + i] = c * max_new + i;
  for (int t = b; t < (int)n_items; t += kBook) {
    const bool wide = t < (int)n_wide;
    const int* offs = wide ? w_off : i_off;
    int lo = 0, hi = s.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (offs[mid] <= t) lo = mid; else hi = mid - 1;
    }
    int k = t - offs[lo];
    const int mine = ((kinds[lo] & 1) != 0) == wide ? o_tiles[lo] * o_chunks[lo] : 0;
    const bool g = k >= mine;
    if (g) k -= mine;
    const int tiles = g ? g_tiles[lo] : o_tiles[lo], chunks = g ? g_chunks[lo] : o_chunks[lo];
    const int c = k / tiles, tile = k - c * tiles;
    const int from = g ? 0 : shares[lo], to = g ? shares[lo] : ends[lo];
    const int seg = info[lo].own_rows;
    const int R2 = g ? info[lo].grp_rows : seg;
    const int step = (int)(ceil_div(ceil_div(to - from, chunks), 64) * 64);   // even chunks
    const int height = wide ? kWideRows : kRows;
    Item it;
    it.q0 = qoffs[lo];
    it.r0 = tile * height;
    it.nr = min(height, R2 - it.r0);
    it.seq = lo;
    it.k0 = from + c * step;
    it.k1 = min(to, it.k0 + step);
    it.cbase = g ? kNoMask : ends[lo] - opens[lo];
    // keys behind the last row's own are no work
    it.k1 = min(it.k1, it.cbase + (it.r0 + it.nr - 1) / rep + 1);
    const int pb = g ? g_part[lo] : o_part[lo];
    it.part = pb < 0 ? -1 : pb + c * R2 + it.r0;
    items[t] = it;
  }
}

// Matrix products of 32 x 32 tiles. A fragment is 16 bytes a lane: E elements
// of row (or column) lane % 32, the E that half lane / 32 holds of 2 E
// consecutive ones. The accumulator of lane l holds column l % 32; entry i is row
// 8 (i / 4) + 4 (l / 32) + i % 4.
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

// Whether the workspace holds a plan of the cache's present state for these
// sizes; a workgroup that finds none records it and leaves.
__device__ inline bool plan_ok(const AttendArgs& a) {
  const Header* h = reinterpret_cast<const Header*>(a.ws);
  const bool ok = h->version == a.p.state[kPagesVersion] && h->hq == a.hq &&
                  h->max_new == a.max_new && h->items >= 0 && h->items <= a.w.max_items;
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

// V where a mask crosses a step: keys from k1 on hold anything and count as 0. A
// value that is not finite but masked for some rows only would reach them as
// 0 x inf: it is taken out here (true: there was one), and add_non_finite adds
// it to the rows that see it. `k`: the key of the fragment's first element.
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
// vt: the V^T rows of a head, at the first of n keys, the first of which is k.
template <typename T, int ND>
__device__ inline void add_non_finite(f32x16 (&o)[ND], const T* vt, int page, int n, int k, int last,
                                      int half) {
  for (int j = 0; j < n && k + j <= last; ++j)
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int dim = dt * 32 + i / 4 * 8 + half * 4 + i % 4;
        const float v = Elem<T>::load(vt + (size_t)dim * page + j);
        if (!(fabsf(v) < INFINITY)) o[dt][i] += v;
      }
}

// One item of one K/V head: four waves take its key steps in turn, each for all
// of its (up to 32) rows, and join at the end. A wave holds its queries as the
// column operand, so that S^T = K Q^T leaves each lane one query's scores: the
// softmax is lane-local but for one exchange between the halves, and the scores
// become the column operand of O^T = V^T P^T where they are. The key that an
// entry of S^T stands for is set by the row order in which K is loaded: the one
// that makes each lane's entries the E consecutive keys of a V^T fragment.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) attend_kernel(AttendArgs a) {
  using M = Mma<T>;
  constexpr int E = M::E, NF = D / (2 * E), ND = D / 32, NP = 16 / E, W = kThreads / 64;
  if (!plan_ok(a)) return;
  const Header* hd = reinterpret_cast<const Header*>(a.ws);
  const int item = hd->wide + (int)(blockIdx.x / a.s.hkv), head = (int)(blockIdx.x % a.s.hkv);
  if (item >= hd->items) return;
  const Item it = reinterpret_cast<const Item*>(a.ws + a.w.items)[item];
  const int32_t* map = reinterpret_cast<const int32_t*>(a.ws + a.w.map);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int32_t* table = a.p.state + a.s.table + (size_t)it.seq * a.s.max_pages;
  const size_t plane = (size_t)2 * a.layer * a.s.n_pages * a.s.page_bytes;
  const size_t hoff = (size_t)head * a.s.page * D;
  const uint8_t* kpool = a.p.pool + plane;
  const uint8_t* vpool = kpool + (size_t)a.s.n_pages * a.s.page_bytes;

  // the lane's query; columns behind the last row repeat it and are not stored
  const int r = it.r0 + min(col, it.nr - 1), qi = r / a.rep, hr = r - qi * a.rep;
  const size_t qrow = map[it.q0 + qi];
  const T* qp = static_cast<const T*>(a.q) + qrow * a.q_stride + (head * a.rep + hr) * D;
  const int last = it.cbase + qi;                      // the last key it sees
  const int first_last = it.cbase + it.r0 / a.rep;     // the least of them in the item
  u32x4 qf[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) qf[f] = *reinterpret_cast<const u32x4*>(qp + (2 * f + half) * E);

  // the key of a step whose K row this lane loads
  const int mi = ((col >> 3) << 2) | (col & 3), mh = (col >> 2) & 1;
  const int krow = mi / E * 2 * E + mh * E + mi % E;
  const float c2 = a.scale * 1.44269504088896341f;
  f32x16 o[ND] = {};
  float m = -INFINITY, l = 0.f;

  const int steps = (it.k1 - it.k0 + kKeys - 1) / kKeys;
  int ids = 0;    // the pages of this wave's next 64 steps, one a lane
  u32x4 kf[NF];
  const T* vbase = nullptr;
  auto fetch = [&](int t) {   // K of the wave's step t; where its V is
    const int st = t * W + wave;
    if ((t & 63) == 0) {
      const int sl = min((t + lane) * W + wave, steps - 1);
      ids = clamp_page(a.s, table[(it.k0 + sl * kKeys) / a.s.page]);
    }
    const int k = it.k0 + st * kKeys;
    const size_t off = (size_t)__builtin_amdgcn_readlane(ids, t & 63) * a.s.page_bytes;
    const int in = k & (a.s.page - 1);
    const T* kp = reinterpret_cast<const T*>(kpool + off) + hoff + (size_t)(in + krow) * D;
#pragma unroll
    for (int f = 0; f < NF; ++f) kf[f] = *reinterpret_cast<const u32x4*>(kp + (2 * f + half) * E);
    vbase = reinterpret_cast<const T*>(vpool + off) + hoff + in + half * E;
  };
  if (wave < steps) fetch(0);
  for (int t = 0; t * W + wave < steps; ++t) {
    const int kb = it.k0 + (t * W + wave) * kKeys;
    u32x4 vf[ND][NP];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int f = 0; f < NP; ++f)
        vf[dt][f] = *reinterpret_cast<const u32x4*>(vbase + (size_t)(dt * 32 + col) * a.s.page +
                                                    f * 2 * E);
    f32x16 sc = {};
#pragma unroll
    for (int f = 0; f < NF; ++f) sc = M::run(kf[f], qf[f], sc);
    if ((t + 1) * W + wave < steps) fetch(t + 1);
    const bool masked = kb + kKeys > min(it.k1, first_last + 1);
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = sc[i];
    if (masked) {
      const int lim = min(it.k1 - 1, last);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (kb + i / E * 2 * E + half * E + i % E > lim) x[i] = -INFINITY;
    }
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
    mx = half_max(mx);
    const float mn = fmaxf(m, mx), mu = mn == -INFINITY ? 0.f : mn * c2;
    const float alpha = __builtin_amdgcn_exp2f(m * c2 - mu);
    m = mn;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c2, -mu));
      sum += x[i];
    }
    l = l * alpha + sum;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] *= alpha;
    u32x4 pf[NP];
#pragma unroll
    for (int f = 0; f < NP; ++f) pf[f] = M::pack(x + f * E);
    if (masked) {
      bool bad = false;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int f = 0; f < NP; ++f)
          bad = clean_values<T>(vf[dt][f], kb + f * 2 * E + half * E, it.k1) || bad;
      if (__any(bad)) {
        const size_t off = (size_t)clamp_page(a.s, table[kb / a.s.page]) * a.s.page_bytes;
        add_non_finite<T, ND>(o, reinterpret_cast<const T*>(vpool + off) + hoff +
                                     (kb & (a.s.page - 1)),
                              a.s.page, min(kKeys, it.k1 - kb), kb, last, half);
      }
    }
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int f = 0; f < NP; ++f) o[dt] = M::run(vf[dt][f], pf[f], o[dt]);
  }
  l = half_sum(l);

  // join the waves: each one's (m, l) of the 32 rows, then O scaled to the common
  // maximum and added up, D / 4 floats a thread row
  __shared__ float sm[W][32], sl[W][32];
  constexpr int LD = D + 4;
  __shared__ alignas(16) float so[W][32 * LD];
  if (half == 0) { sm[wave][col] = m; sl[wave][col] = l; }
  __syncthreads();
  float mt = sm[0][col];
#pragma unroll
  for (int k = 1; k < W; ++k) mt = fmaxf(mt, sm[k][col]);
  const float mu = mt == -INFINITY ? 0.f : mt;
  const float own = __builtin_amdgcn_exp2f((m - mu) * c2);
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(&so[wave][col * LD + dt * 32 + g * 8 + half * 4]) =
          float4{o[dt][4 * g] * own, o[dt][4 * g + 1] * own, o[dt][4 * g + 2] * own,
                 o[dt][4 * g + 3] * own};
  __syncthreads();
  const int nh = a.hq;
  for (int i = threadIdx.x; i < it.nr * (D / 4); i += kThreads) {
    const int row = i / (D / 4), e = (i - row * (D / 4)) * 4;
    float mm = sm[0][row];
#pragma unroll
    for (int k = 1; k < W; ++k) mm = fmaxf(mm, sm[k][row]);
    const float mz = mm == -INFINITY ? 0.f : mm;
    float ll = 0.f, acc[4] = {};
#pragma unroll
    for (int k = 0; k < W; ++k) {
      ll += sl[k][row] * __builtin_amdgcn_exp2f((sm[k][row] - mz) * c2);
      const float4 v = *reinterpret_cast<const float4*>(&so[k][row * LD + e]);
      acc[0] += v.x; acc[1] += v.y; acc[2] += v.z; acc[3] += v.w;
    }
    if (it.part >= 0) {
      const size_t pr = (size_t)head * a.w.part_rows + it.part + row;
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.ws + a.w.o) + pr * D + e) =
          float4{acc[0], acc[1], acc[2], acc[3]};
      if (e == 0) reinterpret_cast<float2*>(a.ws + a.w.ml)[pr] = float2{mm * a.scale, ll};
    } else {
      const int rr = it.r0 + row, q = rr / a.rep;
      const size_t at = (size_t)map[it.q0 + q] * nh + head * a.rep + (rr - q * a.rep);
      const float inv = ll == 0.f ? 0.f : 1.f / ll;
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[k] *= inv;
      M::store4(static_cast<T*>(a.o) + at * D + e, acc);
      if (e == 0 && a.lse) a.lse[at] = ll == 0.f ? -INFINITY : mm * a.scale + logf(ll);
    }
  }
}

// The same for many rows: a workgroup takes 256 of them, 32 a wave, over stages
// of 64 keys that reach all waves through LDS.
//
// The maximum that is taken out of a row's exponents follows the scores only
// when they pass it by 2^kLazy, and is a whole power of two in the base of the
// exponential: O and l then change by an exact factor, in a branch that is
// rarely taken, and nothing is scaled stage by stage.
//
// A stage's K and V^T travel global memory -> registers -> LDS: loaded during
// stage j - 2, written during j - 1 into the buffer that stage j - 2 has left,
// read in stage j; one barrier a stage. A 16-byte chunk c of row r lies at chunk
// c ^ (r mod chunks a row), so that reads of 32 rows and writes of whole rows
// both spread over the banks.
constexpr float kLazy = 8.f;
constexpr int kWideThreads = 512;

template <int D>
__global__ void __launch_bounds__(kWideThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
attend_wide_kernel(AttendArgs a) {
  using M = Mma<uint16_t>;
  constexpr int NF = D / 16, ND = D / 32, NT = kWideThreads;
  constexpr int KC = D / 8, VC = 8;                  // 16-byte chunks of a K row, a V^T row
  constexpr int LU = 64 * KC / NT;                   // chunks a thread loads of each a stage
  constexpr int STAGE = 64 * D * 2;                  // bytes of a stage of K (or V)
  __shared__ alignas(1024) uint8_t sk[2 * STAGE];
  __shared__ alignas(1024) uint8_t sv[2 * STAGE];
  __shared__ int odd_values;
  if (!plan_ok(a)) return;
  const Header* hd = reinterpret_cast<const Header*>(a.ws);
  const int item = (int)(blockIdx.x / a.s.hkv), head = (int)(blockIdx.x % a.s.hkv);
  if (item >= hd->wide) return;
  const Item it = reinterpret_cast<const Item*>(a.ws + a.w.items)[item];
  const int32_t* map = reinterpret_cast<const int32_t*>(a.ws + a.w.map);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int32_t* table = a.p.state + a.s.table + (size_t)it.seq * a.s.max_pages;
  const size_t plane = (size_t)2 * a.layer * a.s.n_pages * a.s.page_bytes;
  const uint16_t* kpool = reinterpret_cast<const uint16_t*>(a.p.pool + plane) +
                          (size_t)head * a.s.page * D;
  const uint16_t* vpool = kpool + (size_t)a.s.n_pages * a.s.page_bytes / 2;
  const size_t page_el = a.s.page_bytes / 2;

  // the lane's query; columns behind the last row repeat it
  const bool active = wave * 32 < it.nr;
  if (tid == 0) odd_values = 0;
  __syncthreads();
  int last;
  u32x4 qf[NF];
  {
    const int r = it.r0 + min(wave * 32 + col, it.nr - 1), qi = r / a.rep;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) +
                         (size_t)map[it.q0 + qi] * a.q_stride + (head * a.rep + r - qi * a.rep) * D;
    last = it.cbase + qi;
#pragma unroll
    for (int f = 0; f < NF; ++f) qf[f] = *reinterpret_cast<const u32x4*>(qp + (2 * f + half) * 8);
  }
  const int first_last = it.cbase + it.r0 / a.rep;
  const int stages = (max(it.k1 - it.k0, 0) + 63) / 64;
  const int full = max(0, min(it.k1, first_last + 1) - it.k0) / 64;   // stages without a mask

  // the loads of a stage: K rows tid / KC + .., V^T rows tid / VC + ..
  const int kr = tid / KC, kc = tid % KC, vr = tid / VC, vc = tid % VC;
  int ids = 0;    // pages of 32 stages, a half stage a lane
  auto page_of = [&](int j, int h) {
    return (size_t)__builtin_amdgcn_readlane(ids, ((j & 31) << 1) | h) * page_el;
  };
  u32x4 gk[LU], gv[LU];
  auto load = [&](int j) {
    if ((j & 31) == 0) {
      const int k = min(it.k0 + j * 64 + lane * 32, it.k1 - 1);
      ids = clamp_page(a.s, table[k / a.s.page]);
    }
    const size_t p0 = page_of(j, 0), p1 = page_of(j, 1);
    const int k = it.k0 + j * 64;
#pragma unroll
    for (int u = 0; u < LU; ++u) {
      const int row = kr + u * (NT / KC);
      gk[u] = *reinterpret_cast<const u32x4*>(kpool + (row < 32 ? p0 : p1) +
                                              (size_t)((k + row) & (a.s.page - 1)) * D + kc * 8);
    }
    const uint16_t* vb = vpool + (vc < 4 ? p0 : p1) + ((k + vc * 8) & (a.s.page - 1));
#pragma unroll
    for (int u = 0; u < LU; ++u)
      gv[u] = *reinterpret_cast<const u32x4*>(vb + (size_t)(vr + u * (NT / VC)) * a.s.page);
  };
  auto store = [&](int j) {
    const int at = (j & 1) * STAGE;
    if (j >= full) {
      bool bad = false;
#pragma unroll
      for (int u = 0; u < LU; ++u)
        bad = clean_values<uint16_t>(gv[u], it.k0 + j * 64 + vc * 8, it.k1) || bad;
      if (bad) odd_values = 1;
    }
#pragma unroll
    for (int u = 0; u < LU; ++u) {
      const int row = kr + u * (NT / KC), vrow = vr + u * (NT / VC);
      *reinterpret_cast<u32x4*>(sk + at + row * (2 * D) + ((kc ^ (row & (KC - 1))) << 4)) = gk[u];
      *reinterpret_cast<u32x4*>(sv + at + vrow * 128 + ((vc ^ (vrow & (VC - 1))) << 4)) = gv[u];
    }
  };
  // fragments: K rows in the order that leaves a lane 8 consecutive keys. The
  // swizzle makes a fragment's offset that of the first with bits flipped.
  const int mi = ((col >> 3) << 2) | (col & 3), mh = (col >> 2) & 1;
  const int krow = mi / 8 * 16 + mh * 8 + mi % 8;
  const uint32_t klane = krow * (2 * D) + ((half ^ (krow & (KC - 1))) << 4);
  const uint32_t vlane = col * 128 + ((half ^ (col & (VC - 1))) << 4);
  auto kfrag = [&](uint32_t at, int sub, int f) {
    return *reinterpret_cast<const u32x4*>(sk + (klane ^ (at + (f << 5))) + sub * (64 * D));
  };
  auto vfrag = [&](uint32_t at, int dt, int f) {
    return *reinterpret_cast<const u32x4*>(sv + (vlane ^ (at + (f << 5))) + dt * 4096);
  };

  const float c2 = a.scale * 1.44269504088896341f;
  f32x16 o[ND] = {};
  float mu = -INFINITY, l = 0.f;
  if (stages > 0) {
    load(0);
    store(0);
    if (stages > 1) load(1);
  }
  for (int j = 0; j < stages; ++j) {
    lds_barrier();   // stage j is whole, and stage j - 1 has been read
    if (j + 1 < stages) store(j + 1);
    if (j + 2 < stages) load(j + 2);
    if (!active) continue;
    const uint32_t at = (j & 1) * STAGE;
    f32x16 sc[2] = {};
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int f = 0; f < NF; ++f) sc[sub] = M::run(kfrag(at, sub, f), qf[f], sc[sub]);
    if (j >= full) {
      const int lim = min(it.k1 - 1, last) - (it.k0 + j * 64);
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (sub * 32 + i / 8 * 16 + half * 8 + i % 8 > lim) sc[sub][i] = -INFINITY;
    }
    float mx = fmaxf(sc[0][0], sc[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, fmaxf(sc[0][i], sc[1][i]));
    mx = half_max(mx) * c2;
    const bool up = mx > mu + kLazy;
    if (__any(up)) {
      const float mn = up ? ceilf(mx) : mu;
      const float alpha = up ? __builtin_amdgcn_exp2f(mu - mn) : 1.f;
      mu = mn;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[dt] *= alpha;
    }
    const float z = mu == -INFINITY ? 0.f : mu;
    u32x4 pf[4];
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[i] = __builtin_amdgcn_exp2f(fmaf(sc[sub][i], c2, -z));
        sum[sub] += x[i];
      }
#pragma unroll
      for (int f = 0; f < 2; ++f) pf[sub * 2 + f] = M::pack(x + 8 * f);
    }
    l += sum[0] + sum[1];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int f = 0; f < 4; ++f) o[dt] = M::run(vfrag(at, dt, f), pf[f], o[dt]);
  }
  if (full < stages) {
    lds_barrier();
    if (odd_values)
      for (int k = it.k0 + full * 64; k < it.k1; k += kKeys)
        add_non_finite<uint16_t, ND>(o, vpool + clamp_page(a.s, table[k / a.s.page]) * page_el +
                                            (k & (a.s.page - 1)),
                                     a.s.page, min(kKeys, it.k1 - k), k, last, half);
  }

  // parts or results, straight from the registers
  l = half_sum(l);
  const int row = wave * 32 + col;
  if (row >= it.nr) return;
  const float m = mu * 0.693147180559945309f;
  if (it.part >= 0) {
    const size_t pr = (size_t)head * a.w.part_rows + it.part + row;
    float* out = reinterpret_cast<float*>(a.ws + a.w.o) + pr * D + half * 4;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(out + dt * 32 + g * 8) =
            float4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]};
    if (half == 0) reinterpret_cast<float2*>(a.ws + a.w.ml)[pr] = float2{m, l};
  } else {
    const int rr = it.r0 + row, q = rr / a.rep;
    const size_t at = (size_t)map[it.q0 + q] * a.hq + head * a.rep + (rr - q * a.rep);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* out = static_cast<uint16_t*>(a.o) + at * D + half * 4;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = o[dt][4 * g + k] * inv;
        M::store4(out + dt * 32 + g * 8, x);
      }
    if (half == 0 && a.lse) a.lse[at] = l == 0.f ? -INFINITY : m + logf(l);
  }
}

// Joins the parts of each row: one wave per (row, query head).
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) attend_join_kernel(AttendArgs a) {
  if (!plan_ok(a)) return;
  const Header* hd = reinterpret_cast<const Header*>(a.ws);
  const long id = (long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int k = (int)(id / a.hq), h = (int)(id - (long)k * a.hq);
  if (k >= hd->rows) return;
  const int row = reinterpret_cast<const int32_t*>(a.ws + a.w.map)[k];
  const SeqInfo f = reinterpret_cast<const SeqInfo*>(a.ws + a.w.info)[row / a.max_new];
  if (f.own_part < 0) return;                 // finished by its only item
  const int lane = threadIdx.x & 63, g = h / a.rep, hr = h - g * a.rep;
  const int n = f.grp_chunks + f.own_chunks;
  const long grp = f.grp_part + (long)(k - f.grp_qoff) * a.rep + hr;
  const long own = f.own_part + (long)(k - f.qoff) * a.rep + hr;
  const size_t base = (size_t)g * a.w.part_rows;
  const float2* ml = reinterpret_cast<const float2*>(a.ws + a.w.ml) + base;
  const float* po = reinterpret_cast<const float*>(a.ws + a.w.o) + base * D;
  auto at = [&](int c) {
    return c < f.grp_chunks ? grp + (long)c * f.grp_rows
                            : own + (long)(c - f.grp_chunks) * f.own_rows;
  };
  float m = -INFINITY;
  for (int c = lane; c < n; c += 64) m = fmaxf(m, ml[at(c)].x);
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  const float mu = m == -INFINITY ? 0.f : m;
  constexpr int V = D / 64;
  float acc[V] = {}, l = 0.f;
  for (int c = 0; c < n; ++c) {
    const long pr = at(c);
    const float2 x = ml[pr];
    const float wgt = __builtin_amdgcn_exp2f((x.x - mu) * 1.44269504088896341f);
    l += x.y * wgt;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] += wgt * po[pr * D + lane * V + v];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const size_t out = (size_t)row * a.hq + h;
#pragma unroll
  for (int v = 0; v < V; ++v)
    Elem<T>::store(static_cast<T*>(a.o) + out * D + lane * V + v, acc[v] * inv);
  if (lane == 0 && a.lse) a.lse[out] = l == 0.f ? -INFINITY : m + logf(l);
}

template <typename T, int D>
hipError_t launch(const AttendArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((attend_kernel<T, D>), dim3((unsigned)a.w.max_items * a.s.hkv),
                     dim3(kThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if constexpr (sizeof(T) == 2) {
    if (a.w.max_wide > 0) {
      hipLaunchKernelGGL(attend_wide_kernel<D>, dim3((unsigned)a.w.max_wide * a.s.hkv),
                         dim3(kWideThreads), 0, st, a);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  const long rows = (long)a.s.batch * a.max_new * a.hq;
  hipLaunchKernelGGL((attend_join_kernel<T, D>), dim3((unsigned)((rows + 3) / 4)), dim3(kThreads),
                     0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t attend_workspace_bytes(const PagesShape& s, int hq, int max_new) {
  return plan_ws(s, hq, max_new).bytes;
}

hipError_t launch_attend_plan(const PagesShape& s, const PagesPtrs& p, int hq, int max_new,
                              const int32_t* groups, void* ws, hipStream_t st) {
  hipLaunchKernelGGL(attend_plan_kernel, dim3(1), dim3(kBook), 0, st, s, p, hq, max_new, groups,
                     static_cast<uint8_t*>(ws), plan_ws(s, hq, max_new));
  return hipGetLastError();
}

hipError_t launch_attend(const PagesShape& s, const PagesPtrs& p, int layer, const void* q,
                         long q_stride, int hq, int max_new, float scale, void* o, float* lse,
                         void* ws, hipStream_t st) {
  AttendArgs a{s, p, q, q_stride, o, lse, layer, hq, hq / s.hkv, max_new, scale,
               static_cast<uint8_t*>(ws), plan_ws(s, hq, max_new)};
  if (s.dtype == LDR_BF16)
    return s.d == 128 ? launch<uint16_t, 128>(a, st) : launch<uint16_t, 64>(a, st);
  return s.d == 128 ? launch<float, 128>(a, st) : launch<float, 64>(a, st);
}

}  // namespace ldr
