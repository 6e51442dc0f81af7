// Causal attention of the open rows over the paged K/V cache, with the pages
// that sequences have in common at the front read once for all of them.
//
// softmax(q K^T) V over a row's keys is the join of its parts over disjoint key
// ranges: a part gives its maximum m, l = sum e^{s - m} and O = sum e^{s - m} v,
// and parts add up after scaling by e^{m_part - m}. So the work is cut into
// segments (rows x keys): the rows of a group of sequences over the keys they
// share, and the rows of each sequence over its own keys. A segment is cut into
// tiles of rows and chunks of keys, enough items to fill the GPU. A plan kernel
// writes the list of items (the lengths are on the device), one workgroup of the
// main kernel takes an item of one K/V head. Items hold whole units of 256 keys
// (128 of fp32) that all rows of their tile see; the keys behind them, where the
// mask runs (or all of a sequence's own where they are few), go to the last kernel,
// which also joins the parts of its rows.
//
// Measured with 32 query and 8 K/V heads of 128, bf16, a layer, passes in a loop: 64
// sequences with one row, 32768 keys in common and 300 of their own 48 us + 27 us in the
// last kernel (the shared keys alone are 28 us of a large matrix product); 16 with 17 rows
// and 512 keys of their own 152 + 25 (115); 16 with 17 rows and up to 8192 keys of their
// own, none in common, 94 + 15 (4.8 TB/s); 2 with 512 rows over 8192 keys 129 + 28 (109).
#include <type_traits>

#include "attend_common.h"

namespace ldr {
namespace {

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
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    before += w < wave ? sums[w] : 0;
    all += sums[w];
  }
  *total = all;
  return before + inc - v;
}

template <typename T> __device__ inline T wave_sum(T v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// Keys of each of n even chunks of len: whole units.
__device__ inline int even_step(int len, int n, int unit) {
  return ((len + n - 1) / n + unit - 1) / unit * unit;
}

// The time of an item of a coded cache, in sixteenths of a whole tile's, and the smallest
// chunk (of the lightest items, tile.unit keys). Measured, eight K/V heads, all compute units
// at it, us for 1024 keys of up to 32 rows, 64, 128, 256: 4 bits, head_dim 128 7, 10, 19, 30
// (and 65 to 96 rows as two tiles 16, 4 sixteenths each), head_dim 64 3.3, 5.1, 10.7, 21; 8 bits,
// head_dim 64 5.2, 6.8, 12, 22. With 8 bits and head_dim 128, 14.6, 14.8, 21, 33, the first two
// are HBM's time with all compute units at it, not a workgroup's: alone they take less.
constexpr int kMxLeast = 48;
__device__ inline int mx_weighted(int len, int rows, bool two) {
  const int w = rows <= 32 ? 3 : rows <= 64 ? 5 : two && rows <= 96 ? 4 : rows <= 128 ? 9 : 16;
  return (int)(((long)len * w + 15) / 16);
}

// The plan, in one workgroup: thread b has sequence b; what looks at all
// sequences for each goes by waves, a sequence at a time. 5.7 us for one sequence, 23 for
// 64 with 512 pages in common (their tables, 128 KB, through one compute unit): once
// for all layers.
// MX: a coded cache, whose items take as long as their rows ask for (mx_weighted): a chunk is
// as many sixteenths of a whole tile's keys.
template <bool BF16, bool MX = false>
__global__ void __launch_bounds__(kBook)
attend_plan_kernel(PagesShape s, PagesPtrs p, int hq, int max_new, const int32_t* groups,
                   uint8_t* ws, AttendWs w) {
  constexpr int kMost = kBook / 64;
  __shared__ long sums[kMost];
  __shared__ int label[kBook], lead[kBook], opens[kBook], fulls[kBook], common[kBook];
  __shared__ int qoffs[kBook], members[kBook], gopens[kBook];
  __shared__ int i_off[kBook], o_chunks[kBook], g_chunks[kBook], o_part[kBook], g_part[kBook];
  __shared__ int o_len[kBook], shares[kBook], ends[kBook];
  __shared__ float4 cuts[kBook];           // tiles and keys, own and shared
  __shared__ float works[kMost], counts[kMost][64];
  const int b = threadIdx.x, lane = b & 63, wave = b >> 6, rep = hq / s.hkv;
  const int NW = blockDim.x / 64;
  const bool in = b < s.batch;
  const int32_t* table = p.state + s.table;
  Header* hd = reinterpret_cast<Header*>(ws);
  int32_t* map = reinterpret_cast<int32_t*>(ws + w.map);
  SeqInfo* info = reinterpret_cast<SeqInfo*>(ws + w.info);
  Item* items = reinterpret_cast<Item*>(ws + w.items);
  constexpr Tile tile = tile_of(BF16);   // divisions by its entries are shifts
  constexpr int least_chunk = MX ? kMxLeast : tile.unit, quantum = MX ? 16 : tile.unit;
  const bool two = MX && two_tiles(s);

  const int all = in ? clamp_rows(s, p.state[s.rows + b]) : 0;
  const int held = in ? min(max(p.state[s.open + b], 0), all) : 0;
  const int page0 = in ? clamp_page(s, table[(size_t)b * s.max_pages]) : 0;
  const int grp = in && groups ? groups[b] : page0;
  const int open = min(held, max_new);
  const int rows = all - held + open;        // the keys that a query of the plan can see
  const int full = (all - held) / s.page;    // whole pages before the open rows
  // a sequence that has nothing to share stands alone
  label[b] = open > 0 && full > 0 && grp >= 0 ? grp : -1 - b;
  opens[b] = open;
  fulls[b] = full;
  __syncthreads();
  // the first sequence of each one's group, and the size of the group
  for (int c = wave; c < s.batch; c += NW) {
    const int lb = label[c];
    int first = -1, n = 0;
    for (int i = 0; i < s.batch; i += 64) {
      const uint64_t eq = __ballot(i + lane < s.batch && label[i + lane] == lb);
      if (eq && first < 0) first = i + __builtin_ctzll(eq);
      n += __builtin_popcountll(eq);
    }
    if (lane == 0) {
      lead[c] = first;
      members[c] = n;
      common[c] = fulls[c];
    }
  }
  __syncthreads();
  // row map: the sequences of a group behind one another; pages in common with
  // the first of the group, many loads at a time, those of the first once
  constexpr int U = 8;
  int y[U], y_of = -1, y_at = 0;
  for (int c = wave; c < s.batch; c += NW) {
    const int ld = lead[c];
    int before = 0, sum = 0;
    for (int i = lane; i < s.batch; i += 64) {
      const int l = lead[i], o = opens[i];
      before += l < ld || (l == ld && i < c) ? o : 0;
      sum += l == ld ? o : 0;
    }
    before = wave_sum(before);
    sum = wave_sum(sum);
    if (lane == 0) {
      qoffs[c] = before;
      gopens[c] = sum;
    }
    if (ld == c) continue;
    const int lim = min(fulls[c], fulls[ld]);
    const int32_t* tc = table + (size_t)c * s.max_pages;
    const int32_t* tl = table + (size_t)ld * s.max_pages;
    int same = lim;
    for (int j = 0; j < lim; j += 64 * U) {
      int x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = tc[min(j + u * 64 + lane, lim - 1)];
      if (y_of != ld || y_at != j) {
        y_of = ld;
        y_at = j;
#pragma unroll
        for (int u = 0; u < U; ++u) y[u] = tl[min(j + u * 64 + lane, fulls[ld] - 1)];
      }
      int at = lim;
#pragma unroll
      for (int u = U - 1; u >= 0; --u) {
        const int k = j + u * 64 + lane;
        const uint64_t diff = __ballot(k < lim && x[u] != y[u]);
        if (diff) at = j + u * 64 + (int)__builtin_ctzll(diff);
      }
      if (at < lim) { same = at; break; }
    }
    if (lane == 0) atomicMin(&common[ld], same);
  }
  __syncthreads();
  // segments: a sequence's own rows over its own keys; a group's rows, kept with
  // its first sequence, over the shared ones
  const int ld = in ? lead[b] : b;
  const int common_rows = in ? common[ld] * s.page / tile.unit * tile.unit : 0;
  const int share = in && members[b] > 1 && common_rows >= kMinShared ? common_rows : 0;
  const int gopen = in ? gopens[b] : 0;
  const int R = open * rep, Rg = share && ld == b ? gopen * rep : 0;    // below 2^28
  const int otr = tile_rows(tile, two, R), ot = ceil_div(R, otr);
  const int gt = ceil_div(Rg, tile_rows(tile, two, Rg));
  int len = open ? tile_keys(rows, open, share, (ot - 1) * otr, rep, tile.unit) : 0;
  if (len < kMinMain) len = 0;
  const int glen = Rg ? share : 0;
  o_len[b] = len;
  shares[b] = share;
  ends[b] = rows;
  // what the chunks are cut by
  const int wlen = MX ? mx_weighted(len, R, two) : len;
  const int wglen = MX ? mx_weighted(glen, Rg, two) : glen;
  cuts[b] = float4{(float)ot, (float)wlen, (float)gt, (float)wglen};
  const float mine = wave_sum((float)ot * wlen + (float)gt * wglen);
  if (lane == 0) works[wave] = mine;
  __syncthreads();
  // The chunk: a lane has a length, a wave some of the sequences. With slots for all
  // items the time is a chunk's; else it is near an even spread, and half a chunk at the
  // end.
  float work = 0.f;
  for (int w = 0; w < NW; ++w) work += works[w];
  const float even = work * s.hkv / tile.slots;
  const int least = max((int)min(even / kMaxRounds + 1.f, 1e8f), least_chunk);
  // from `least` to 4.5 x kMaxRounds of it, in even ratios
  const float x = least * __builtin_amdgcn_exp2f(lane * (3.2f / 64));
  int chunk = ceil_div((int)x, quantum) * quantum;
  {
    const float per = __builtin_amdgcn_rcpf((float)chunk);
    float n = 0.f;           // of chunks, nearly: for an estimate
    for (int i = wave; i < s.batch; i += NW) {
      const float4 c = cuts[i];
      n += c.x * ceilf(c.y * per) + c.z * ceilf(c.w * per);
    }
    counts[wave][lane] = n;
    __syncthreads();
    n = 0.f;
    for (int w = 0; w < NW; ++w) n += counts[w][lane];
    const float wgs = n * s.hkv;
    float cost = wgs <= tile.slots ? (float)chunk + tile.cost
                                   : (even * tile.slots + wgs * tile.cost) / tile.slots +
                                         0.5f * (chunk + tile.cost);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      const float oc = __shfl_xor(cost, off);
      const int ch = __shfl_xor(chunk, off);
      if (oc < cost || (oc == cost && ch < chunk)) { cost = oc; chunk = ch; }
    }
  }
  int oc = (wlen + chunk - 1) / chunk, gc = (wglen + chunk - 1) / chunk;
  if (MX) {     // of whole units there may be fewer: none of the chunks is empty
    if (oc) oc = ceil_div(len, even_step(len, oc, tile.unit));
    if (gc) gc = ceil_div(glen, even_step(glen, gc, tile.unit));
  }
  const int ob = ceil_div(R, kBlock), gb = ceil_div(Rg, kBlock);
  // the list: each sequence's own items, then its group's; and the blocks of parts
  // both counts in one scan: below 2^31 each, by the bound on the chunk
  long both = 0;
  const long at = block_scan((long)(ot * oc + gt * gc) << 32 | (long)(oc * ob + gc * gb), sums, &both);
  long n_items = both >> 32, n_part = both & 0xffffffff;
  const long off = at >> 32, part = at & 0xffffffff;
  i_off[b] = (int)off;
  o_chunks[b] = oc; g_chunks[b] = gc;
  o_part[b] = (int)part;
  g_part[b] = (int)(part + (long)oc * ob);
  __syncthreads();
  if (in) {
    SeqInfo f{};
    f.qoff = qoffs[b];
    f.open = open;
    f.rows = rows;
    f.share = share;
    f.step = oc ? even_step(len, oc, tile.unit) : tile.unit;
    f.own_part = o_part[b];
    f.own_chunks = oc;
    f.own_blocks = ob;
    if (share) {
      f.grp_part = g_part[ld];
      f.grp_chunks = g_chunks[ld];
      f.grp_blocks = ceil_div(gopen * rep, kBlock);
      f.grp_off = (qoffs[b] - qoffs[ld]) * rep;
    }
    info[b] = f;
  }
  // fits by the bounds of plan_ws; a list that did not would be no plan
  if (n_items > w.max_items || n_part > w.blocks) n_items = -1;
  if (b == 0) {
    hd->version = p.state[kPagesVersion];
    hd->hq = hq;
    hd->max_new = max_new;
    hd->items = (int)n_items;
    hd->id = p.id;
  }
  for (int c = wave; c < s.batch; c += NW)
    for (int i = lane; i < opens[c]; i += 64) map[qoffs[c] + i] = c * max_new + i;
  for (int t = b; t < (int)n_items; t += blockDim.x) {
    int lo = 0, hi = s.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (i_off[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const int own_rows = opens[lo] * rep;
    const int own_tiles = ceil_div(own_rows, tile_rows(tile, two, own_rows));
    int k = t - i_off[lo];
    const bool g = k >= own_tiles * o_chunks[lo];
    if (g) k -= own_tiles * o_chunks[lo];
    const int n = g ? gopens[lo] * rep : own_rows;
    const int tr = tile_rows(tile, two, n), tiles = ceil_div(n, tr);
    const int c = k / tiles, r0 = (k - c * tiles) * tr;
    const int from = g ? 0 : shares[lo];
    const int keys = g ? shares[lo] : tile_keys(ends[lo], opens[lo], from, r0, rep, tile.unit);
    const int step = even_step(g ? shares[lo] : o_len[lo], g ? g_chunks[lo] : o_chunks[lo],
                               tile.unit);
    Item it;
    it.q0 = qoffs[lo];
    it.r0 = r0;
    it.nr = min(tr, n - r0);
    it.seq = lo;
    it.k0 = from + c * step;
    it.k1 = from + min(keys, (c + 1) * step);   // not above k0: the tile has no such chunk
    it.part = (g ? g_part[lo] : o_part[lo]) + c * ((n + kBlock - 1) / kBlock) + r0 / kBlock;
    it.pad = 0;
    items[t] = it;
  }
}

// 32 rows of one K/V head: four waves take the steps of 32 keys in turn, each for
// all of the rows, and join at the end. A wave holds its queries as the column
// operand, so that S^T = K Q^T leaves each lane one query's scores: the softmax is
// lane-local but for one exchange between the halves, and the scores become the
// column operand of O^T = V^T P^T where they are. The key that an entry of S^T
// stands for is set by the row order in which K is loaded: the one that makes each
// lane's entries the E consecutive keys of a V^T fragment.
//
// FINISH: the rows' parts, which the waves take in turn, and their last keys, where the
// mask runs; then the results are written. Bound by bytes where parts and keys are many (64
// sequences with one row: 34 MB of parts and 78 MB of keys in 27 us), else by the chain
// of loads (plan, table, keys, V; 8 us for one sequence). Else: an item of the f32 main
// kernel, its results a part (7 us for 2048 keys of 4 heads of 64).
template <typename T, int D, bool FINISH>
__global__ void __launch_bounds__(kThreads, sizeof(T) * D <= 256 ? 2 : 1)
attend_rows_kernel(AttendArgs a) {
  using M = Mma<T>;
  constexpr int E = M::E, NF = D / (2 * E), ND = D / 32, NP = 16 / E, W = kThreads / 64;
  const int unit = (int)(blockIdx.x / a.s.hkv), head = (int)(blockIdx.x % a.s.hkv);
  const int items = scalar_word(a.ws, 3);
  Item it{};
  SeqInfo f{};
  int cbase = 0;      // row r sees keys up to cbase + r / rep
  if constexpr (FINISH) {
    it.seq = unit / a.w.tiles;
    it.r0 = (unit - it.seq * a.w.tiles) * kBlock;
    f = scalar_info(a.ws + a.w.info, it.seq);
    if (!plan_ok(a, items) || it.r0 >= f.open * a.rep) return;
    it.nr = min(kBlock, f.open * a.rep - it.r0);
    it.q0 = f.qoff;
    cbase = f.rows - f.open;
    const int t = it.r0 / tile_of(a.s).rows * tile_of(a.s).rows;
    it.k0 = f.share + (f.own_chunks ? tile_keys(f.rows, f.open, f.share, t, a.rep, tile_of(a.s).unit) : 0);
    it.k1 = cbase + (it.r0 + it.nr - 1) / a.rep + 1;
  } else {
    it = scalar_item(a.ws + a.w.items, unit);
    if (!plan_ok(a, items) || unit >= items || it.k1 <= it.k0) return;
  }
  const int32_t* map = reinterpret_cast<const int32_t*>(a.ws + a.w.map);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int32_t* table = a.p.state + a.s.table + (size_t)it.seq * a.s.max_pages;
  const size_t plane = (size_t)2 * a.layer * a.s.n_pages * a.s.page_bytes;
  const size_t hoff = (size_t)head * a.s.page * D;
  const uint8_t* kpool = a.p.pool + plane;
  const uint8_t* vpool = kpool + (size_t)a.s.n_pages * a.s.page_bytes;

  // the lane's query; columns behind the last row repeat it and are not stored
  const int r = it.r0 + min(col, it.nr - 1), qi = r / a.rep, hr = r - qi * a.rep;
  const size_t qrow = FINISH ? (size_t)it.seq * a.max_new + qi : (size_t)map[it.q0 + qi];
  const T* qp = static_cast<const T*>(a.q) + qrow * a.q_stride + (head * a.rep + hr) * D;
  u32x4 qf[NF];
#pragma unroll
  for (int i = 0; i < NF; ++i) qf[i] = *reinterpret_cast<const u32x4*>(qp + (2 * i + half) * E);

  // the key of a step whose K row this lane loads
  const int mi = ((col >> 3) << 2) | (col & 3), mh = (col >> 2) & 1;
  const int krow = mi / E * 2 * E + mh * E + mi % E;
  const float c2 = a.scale * kLog2e;
  f32x16 o[ND] = {};
  float m = -INFINITY, l = 0.f;
  bool bad = false;   // V held a value that is not finite where a mask is

  const int steps = (max(it.k1 - it.k0, 0) + kStep - 1) / kStep;
  const int shift = 31 - __builtin_clz(a.s.page);
  auto id_of = [&](int t) {   // the page of the wave's step t, on its way until it is looked at
    return scalar_word(table, (it.k0 + min(t * W + wave, max(steps - 1, 0)) * kStep) >> shift);
  };
  u32x4 kf[NF];
  const T* vbase = nullptr;
  int id = wave < steps ? id_of(0) : 0;
  auto fetch = [&](int t) {   // K of the wave's step t; where its V is
    const size_t off = (size_t)clamp_page(a.s, id) * a.s.page_bytes;
    const int in = (it.k0 + (t * W + wave) * kStep) & (a.s.page - 1);
    const T* kp = reinterpret_cast<const T*>(kpool + off) + hoff + (size_t)(in + krow) * D;
#pragma unroll
    for (int i = 0; i < NF; ++i) kf[i] = *reinterpret_cast<const u32x4*>(kp + (2 * i + half) * E);
    vbase = reinterpret_cast<const T*>(vpool + off) + hoff + in + half * E;
    id = id_of(t + 1);
  };
  if (wave < steps) fetch(0);
  if constexpr (FINISH) {
    // parts: the group's chunks, then the tile's own. Of few rows there are columns
    // to spare: R a part, and 32 / R parts at a time (4 rows of 32 parts, as 64
    // sequences with one token each have, took 8 loads behind one another, 11 us).
    // join_parts (attend_mx.hip) does the same for coded caches.
    const int t = it.r0 / tile_of(a.s).rows * tile_of(a.s).rows;
    const int own = f.own_chunks
                        ? (tile_keys(f.rows, f.open, f.share, t, a.rep, tile_of(a.s).unit) + f.step - 1) / f.step : 0;
    const int parts = f.grp_chunks + own;
    int R = 32;
    while (R > 1 && 2 * it.nr <= R && W * 32 < parts * R) R >>= 1;
    const int rp = it.r0 + min(col & (R - 1), it.nr - 1), gr = f.grp_off + rp;
    for (int c = wave + W * (col / R); c < parts; c += W * (32 / R)) {
      const bool g = c < f.grp_chunks;
      const long block = g ? f.grp_part + (long)c * f.grp_blocks + gr / kBlock
                           : f.own_part + (long)(c - f.grp_chunks) * f.own_blocks + it.r0 / kBlock;
      const int at = g ? gr % kBlock : rp % kBlock;
      const float2 ml = part_ml(a, head, block)[at];
      const float4* po = reinterpret_cast<const float4*>(part_o<D>(a, head, block)) + half * 32 + at;
      float4 v[D / 8];
#pragma unroll
      for (int i = 0; i < D / 8; ++i) v[i] = po[i * 64];
      const float mn = fmaxf(m, ml.x), mu = mn == -INFINITY ? 0.f : mn;
      const float wo = __builtin_amdgcn_exp2f((m - mu) * c2);
      const float wp = __builtin_amdgcn_exp2f((ml.x - mu) * c2);
      m = mn;
      l = l * wo + ml.y * wp;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const int dt = i / 4, q = i % 4 * 4;
        o[dt][q] = o[dt][q] * wo + v[i].x * wp;
        o[dt][q + 1] = o[dt][q + 1] * wo + v[i].y * wp;
        o[dt][q + 2] = o[dt][q + 2] * wo + v[i].z * wp;
        o[dt][q + 3] = o[dt][q + 3] * wo + v[i].w * wp;
      }
    }
    if (R < 32) {            // the columns of a row, to their common maximum and added up
      float mn = fmaxf(m, aside<16>(m));
      if (R < 16) mn = fmaxf(mn, aside<8>(mn));
      if (R < 8) mn = fmaxf(mn, aside<4>(mn));
      if (R < 4) mn = fmaxf(mn, aside<2>(mn));
      if (R < 2) mn = fmaxf(mn, aside<1>(mn));
      const float w = __builtin_amdgcn_exp2f((m - (mn == -INFINITY ? 0.f : mn)) * c2);
      m = mn;
      l *= w;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[dt] *= w;
      auto add = [&](auto off) {
        constexpr int OFF = decltype(off)::value;
        l += aside<OFF>(l);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[dt][i] += aside<OFF>(o[dt][i]);
      };
      add(std::integral_constant<int, 16>{});
      if (R < 16) add(std::integral_constant<int, 8>{});
      if (R < 8) add(std::integral_constant<int, 4>{});
      if (R < 4) add(std::integral_constant<int, 2>{});
      if (R < 2) add(std::integral_constant<int, 1>{});
    }
    l = half ? 0.f : l;      // of both halves; the steps' sums are of one each
  }
  for (int t = 0; t * W + wave < steps; ++t) {
    const int kb = it.k0 + (t * W + wave) * kStep;
    u32x4 vf[ND][NP];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i = 0; i < NP; ++i)
        vf[dt][i] = *reinterpret_cast<const u32x4*>(vbase + (size_t)(dt * 32 + col) * a.s.page +
                                                    i * 2 * E);
    f32x16 sc = {};
#pragma unroll
    for (int i = 0; i < NF; ++i) sc = M::run(kf[i], qf[i], sc);
    if ((t + 1) * W + wave < steps) fetch(t + 1);
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = sc[i];
    if constexpr (FINISH) {
      const int lim = cbase + qi - kb;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i / E * 2 * E + half * E + i % E > lim) x[i] = -INFINITY;
    }
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
    mx = half_max(mx);
    const float mn = fmaxf(m, mx), mu = mn == -INFINITY ? 0.f : mn * c2;
    const float alpha = rescale(m, c2, mu);
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
    for (int i = 0; i < NP; ++i) pf[i] = M::pack(x + i * E);
    if (FINISH && kb + kStep > cbase + it.r0 / a.rep + 1)
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < NP; ++i)
          bad = clean_values<T>(vf[dt][i], kb + i * 2 * E + half * E, it.k1) || bad;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i = 0; i < NP; ++i) o[dt] = M::run(vf[dt][i], pf[i], o[dt]);
  }
  l = half_sum(l);

  // join the waves: each one's (m, l) of the 32 rows, then O scaled to the common
  // maximum and added up, four values a thread
  __shared__ float sm[W][32], sl[W][32];
  __shared__ int odd[W];
  const bool any_bad = __any(bad);
  if (lane == 0) odd[wave] = any_bad;
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
  // thread i: values e .. e + 3 of a row; rows fastest for a part's order
  constexpr int NI = 32 * (D / 4) / kThreads;
  auto row_of = [](int i) { return FINISH ? i / (D / 4) : i % 32; };
  auto el_of = [](int i) { return FINISH ? i % (D / 4) * 4 : i / 32 * 4; };
  float acc[NI][4], ll[NI], mm[NI];
#pragma unroll
  for (int u = 0; u < NI; ++u) {
    const int i = u * kThreads + threadIdx.x, row = row_of(i), e = el_of(i);
    mm[u] = sm[0][row];
#pragma unroll
    for (int k = 1; k < W; ++k) mm[u] = fmaxf(mm[u], sm[k][row]);
    const float mz = mm[u] == -INFINITY ? 0.f : mm[u];
    ll[u] = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[u][k] = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      ll[u] += sl[k][row] * __builtin_amdgcn_exp2f((sm[k][row] - mz) * c2);
      const float4 v = *reinterpret_cast<const float4*>(&so[k][row * LD + e]);
      acc[u][0] += v.x; acc[u][1] += v.y; acc[u][2] += v.z; acc[u][3] += v.w;
    }
    if constexpr (FINISH) {
      const float inv = ll[u] == 0.f ? 0.f : 1.f / ll[u];
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[u][k] *= inv;
    }
  }
  if constexpr (FINISH) {
    if (odd[0] | odd[1] | odd[2] | odd[3]) {   // what clean_values took out
      const int s0 = max(0, cbase + it.r0 / a.rep + 1 - it.k0) / kStep;
#pragma unroll
      for (int u = 0; u < NI; ++u) {
        const int i = u * kThreads + threadIdx.x, row = row_of(i), e = el_of(i);
        const int last = row < it.nr ? cbase + (it.r0 + row) / a.rep : -1;
        for (int k = it.k0 + s0 * kStep; k <= last; ++k) {
          const size_t off = (size_t)clamp_page(a.s, table[k >> shift]) * a.s.page_bytes;
          const int in = k & (a.s.page - 1);
          const T* vt = reinterpret_cast<const T*>(vpool + off) + hoff + in;
          float v[4];
          bool any = false;
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            v[d] = Elem<T>::load(vt + (size_t)(e + d) * a.s.page);
            any = any || !(fabsf(v[d]) < INFINITY);
          }
          if (!any) continue;
          // a key without weight gives 0 x inf, as in the main kernel
          const int rr = it.r0 + row, i = rr / a.rep;
          const T* qr = static_cast<const T*>(a.q) +
                        ((size_t)it.seq * a.max_new + i) * a.q_stride + (head * a.rep + rr - i * a.rep) * D;
          const T* kr = reinterpret_cast<const T*>(kpool + off) + hoff + (size_t)in * D;
          float sc = 0.f;
#pragma unroll 1
          for (int j = 0; j < D; ++j) sc += Elem<T>::load(qr + j) * Elem<T>::load(kr + j);
          const float w = sc * c2 == -INFINITY ? 0.f : 1.f;
#pragma unroll
          for (int d = 0; d < 4; ++d)
            if (!(fabsf(v[d]) < INFINITY)) acc[u][d] += w * v[d];
        }
      }
      __syncthreads();      // q has been read: it may be o
    }
    // a row without weight is 0, whatever values 0 was multiplied with
#pragma unroll
    for (int u = 0; u < NI; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[u][k] = ll[u] == 0.f ? 0.f : acc[u][k];
  }
#pragma unroll
  for (int u = 0; u < NI; ++u) {
    const int i = u * kThreads + threadIdx.x, row = row_of(i), e = el_of(i);
    if constexpr (FINISH) {
      if (row >= it.nr) continue;
      const int rr = it.r0 + row, q = rr / a.rep;
      const size_t at = ((size_t)it.seq * a.max_new + q) * a.hq + head * a.rep + (rr - q * a.rep);
      M::store4(static_cast<T*>(a.o) + at * D + e, acc[u]);
      if (e == 0 && a.lse) a.lse[at] = ll[u] == 0.f ? -INFINITY : mm[u] * a.scale + logf(ll[u]);
    } else {
      // e = 32 dt + 8 g + 4 half
      reinterpret_cast<float4*>(part_o<D>(a, head, it.part))[(e / 8) * 64 + (e / 4 % 2) * 32 + row] =
          float4{acc[u][0], acc[u][1], acc[u][2], acc[u][3]};
      if (e == 0) part_ml(a, head, it.part)[row] = float2{mm[u], ll[u]};
    }
  }
}

// The bf16 kernel: a workgroup takes an item of up to 256 rows, 32 a wave, over
// stages of 64 keys that reach all waves through LDS.
//
// O and l change by an exact factor when a row's maximum does (kLazy), in a branch
// that is rarely taken, and nothing is scaled stage by stage.
//
// A stage is the products of a wave (V^T P^T of the stage before, then K Q^T:
// 1024 cycles of the matrix unit at D = 128) and the softmax of its scores. The
// two waves of a SIMD belong to two groups, half a stage apart: a stage has one
// barrier, which the first group meets before its products and the second
// before its softmax, so that one makes probabilities while the other has its
// products.
//
// K and V^T go to LDS by DMA, three stages ahead, in a ring of four buffers: the
// one of stage j has K of j and V of j - 1, which its products read between
// barriers j and j + 1. What was read before barrier j (the buffer of j - 1) is
// filled again among those products, for stage j + 3; a wave waits for its share
// of buffer j in front of barrier j. Separate arrays let the compiler see that a
// read does not depend on the DMA in flight. Rows are turned (below), so that the
// reads of 16 of them spread over the banks.

template <int N> __device__ inline void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}
#define LDR_LP(p) ((__attribute__((address_space(3))) void*)(p))

// SMALL: pages of 32 rows, half a stage.
template <int D, bool SMALL>
__global__ void __launch_bounds__(kWideThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
attend_wide_kernel(AttendArgs a) {
  using M = Mma<uint16_t>;
  constexpr int NF = D / 16, ND = D / 32, NW = kWideThreads / 64;
  constexpr int KC = D / 8, VC = 8;                  // 16-byte chunks of a K row, a V^T row
  constexpr int STAGE = kStage * D * 2;              // bytes of a stage of K (or V)
  constexpr int LU = STAGE / 1024 / NW;              // DMA instructions a wave, of each a stage
  __shared__ alignas(1024) uint8_t S0[2 * STAGE], S1[2 * STAGE], S2[2 * STAGE], S3[2 * STAGE];
  const int item = (int)(blockIdx.x / a.s.hkv), head = (int)(blockIdx.x % a.s.hkv);
  const int items = scalar_word(a.ws, 3);
  const Item it = scalar_item(a.ws + a.w.items, item);
  if (!plan_ok(a, items) || item >= items || it.k1 <= it.k0) return;
  const int32_t* map = reinterpret_cast<const int32_t*>(a.ws + a.w.map);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int32_t* table = a.p.state + a.s.table + (size_t)it.seq * a.s.max_pages;
  const size_t plane = (size_t)2 * a.layer * a.s.n_pages * a.s.page_bytes;
  const uint16_t* kpool = reinterpret_cast<const uint16_t*>(a.p.pool + plane) +
                          (size_t)head * a.s.page * D;
  const uint16_t* vpool = kpool + (size_t)a.s.n_pages * a.s.page_bytes / 2;
  const size_t page_el = a.s.page_bytes / 2;

  // Up to 128 rows: both groups take the same rows, each 32 of a stage's keys, and join
  // at the end (16 sequences with 68 rows over 8192 keys of their own, two layers: 232
  // us; 239 if half of the waves are idle). The lane's query; columns behind the last
  // row repeat it.
  const bool split = it.nr <= NW / 2 * kBlock;
  const int block = split ? wave % (NW / 2) : wave;
  const bool active = block * kBlock < it.nr;
  u32x4 qf[NF];
  {
    const int r = it.r0 + min(block * kBlock + col, it.nr - 1), qi = r / a.rep;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) +
                         (size_t)map[it.q0 + qi] * a.q_stride + (head * a.rep + r - qi * a.rep) * D;
#pragma unroll
    for (int f = 0; f < NF; ++f) qf[f] = *reinterpret_cast<const u32x4*>(qp + (2 * f + half) * 8);
  }
  const int stages = (it.k1 - it.k0) / kStage;

  // DMA. A half stage starts a page of 32, a stage lies at a multiple of 64 of a
  // larger one: the lanes' offsets in it stay.
  const int shift = 31 - __builtin_clz(a.s.page);
  uint32_t koff[LU], voff[LU];
  bool second[LU];     // the lane's V is of keys 32 ..
#pragma unroll
  for (int u = 0; u < LU; ++u) {
    const int n = wave * LU + u;
    const int kr = n * (64 / KC) + lane / KC, vr = n * (64 / VC) + lane / VC;
    const int kc = (lane % KC) ^ turn<KC>(kr), vc = (lane % VC) ^ turn<VC>(vr);
    koff[u] = ((SMALL ? kr & 31 : kr) * D + kc * 8) * 2;
    voff[u] = (vr * a.s.page + (SMALL ? (vc & 3) * 8 : vc * 8)) * 2;
    second[u] = vc >= 4;
  }
  // where a stage's keys are: elements from the pool's start to its page (and, of
  // pages of 32, that of its second half), keys into it
  struct Place { size_t a, b; int in; };
  struct Ids { int a, b; };
  auto ids_of = [&](int j) {     // on their way until they are looked at
    const int k = it.k0 + j * kStage;
    return Ids{scalar_word(table, k >> shift), SMALL ? scalar_word(table, (k + 32) >> shift) : 0};
  };
  auto place = [&](Ids ids, int j) {
    Place p;
    p.a = (size_t)clamp_page(a.s, ids.a) * page_el;
    p.b = SMALL ? (size_t)clamp_page(a.s, ids.b) * page_el : p.a;
    p.in = SMALL ? 0 : (it.k0 + j * kStage) & (a.s.page - 1);
    return p;
  };
  auto dma = [&](uint8_t* to, const uint16_t* base, uint32_t off) {
    const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base), 0, 0x7fffffff,
                                                        0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, LDR_LP(to), 16, off, 0, 0, 0);
  };
  auto dma_k = [&](uint8_t* to, const Place& p, int u) {
    const int n = wave * LU + u;
    dma(to + n * 1024, kpool + (n * (64 / KC) < 32 ? p.a : p.b) + p.in * D, koff[u]);
  };
  auto dma_v = [&](uint8_t* to, const Place& p, int u) {
    to += (wave * LU + u) * 1024;
    if (SMALL && second[u]) dma(to, vpool + p.b + p.in, voff[u]);
    else dma(to, vpool + p.a + p.in, voff[u]);
  };
  auto buffer = [&](auto i) -> uint8_t* {
    constexpr int I = decltype(i)::value & 3;
    if constexpr (I == 0) return S0; else if constexpr (I == 1) return S1;
    else if constexpr (I == 2) return S2; else return S3;
  };
  Ids next;       // pages of the next K to start
  Place kp, vp;   // where the K and V to start behind the last barrier are
  // barrier j, J = j mod 4
  auto meet = [&](int j) {
    wait_vmcnt<4 * LU>();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    vp = kp;
    kp = place(next, min(j + 3, stages - 1));
    next = ids_of(min(j + 4, stages - 1));
  };
  // the DMA behind barrier j, one instruction of 2 LU
  auto start = [&](auto J, int q) {
    uint8_t* to = buffer(std::integral_constant<int, decltype(J)::value + 3>{});
    if (q < LU) dma_k(to, kp, q);
    else dma_v(to + STAGE, vp, q - LU);
  };

  // fragments: K rows in the order that leaves a lane 8 consecutive keys. The
  // swizzle makes a fragment's offset that of the first with bits flipped.
  const int mi = ((col >> 3) << 2) | (col & 3), mh = (col >> 2) & 1;
  const int krow = mi / 8 * 16 + mh * 8 + mi % 8;
  const uint32_t klane = krow * (2 * D) + ((half ^ turn<KC>(krow)) << 4);
  const uint32_t vlane = col * 128 + ((half ^ turn<VC>(col)) << 4);

  const float c2 = a.scale * kLog2e;
  f32x16 o[ND] = {};
  float mu = -INFINITY, l = 0.f;
  f32x16 sc[2];
  u32x4 pf[4] = {};      // none before the first stage, and its V is 0
  // The products of stage j, J = j mod 4: V^T P^T of j - 1, then (unless j is the
  // end) K Q^T of j, two at a time, with the LDS reads kAhead fragments in front of
  // them. The order is pinned: left to itself the compiler reads each fragment
  // right before its product and waits for it. Half: 0 or 1, or both (2).
  auto products = [&](auto scores, auto Half, auto J) {
    constexpr int H = decltype(Half)::value, NS = H == 2 ? 2 : 1, F0 = H == 1 ? 2 : 0;
    constexpr int G = 2, kAhead = 4, R = kAhead + G;
    constexpr int NV = 2 * NS * ND, N = NV + (decltype(scores)::value ? NS * NF : 0);
    static_assert(N % G == 0 && kAhead % G == 0, "whole groups");
    const uint8_t* kb = buffer(J) + (H == 1 ? 64 * D : 0);
    const uint8_t* vb = buffer(J) + STAGE;
    u32x4 fr[R];
    auto read = [&](int i) {
      const int f = i < NV ? F0 + i / ND : (i - NV) / NS;
      fr[i % R] = i < NV ? *reinterpret_cast<const u32x4*>(vb + (vlane ^ (f << 5)) + i % ND * 4096)
                         : *reinterpret_cast<const u32x4*>(kb + (klane ^ (f << 5)) +
                                                           (i - NV) % NS * (64 * D));
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
    for (int i0 = 0; i0 < N; i0 += G) {
      __builtin_amdgcn_sched_barrier(0x6);
      // the DMA in between, one at a time: 4 of each wave at once stall them all
      if (decltype(scores)::value && i0 % (N / (2 * LU)) == 0) start(J, i0 / (N / (2 * LU)));
#pragma unroll
      for (int i = i0 + kAhead; i < i0 + kAhead + G; ++i)
        if (i < N) read(i);
      __builtin_amdgcn_sched_barrier(0x6);
#pragma unroll
      for (int i = i0; i < i0 + G; ++i) {
        if (i < NV) {
          o[i % ND] = M::run(fr[i % R], pf[i / ND], o[i % ND]);
        } else {
          const int f = (i - NV) / NS, sub = (i - NV) % NS;
          sc[sub] = M::run(fr[i % R], qf[f], f ? sc[sub] : f32x16{});
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0x6);
  };
  auto softmax = [&](auto Half) {
    constexpr int NS = decltype(Half)::value == 2 ? 2 : 1;
    float mx = sc[0][0];
#pragma unroll
    for (int i = NS == 2 ? 0 : 1; i < 16; ++i)
      mx = fmaxf(mx, NS == 2 ? fmaxf(sc[0][i], sc[1][i]) : sc[0][i]);
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
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int sub = 0; sub < NS; ++sub) {
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
  };

  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  std::integral_constant<int, 0> i0;
  std::integral_constant<int, 1> i1;
  std::integral_constant<int, 2> i2;
  std::integral_constant<int, 3> i3;
  // K of stages 0 .. 2, V of 0 and 1, in the order in which the barriers wait
  {
    const int j1 = min(1, stages - 1), j2 = min(2, stages - 1);
    const Ids n0 = ids_of(0), n1 = ids_of(j1), n2 = ids_of(j2);
    next = ids_of(min(3, stages - 1));
    const Place p0 = place(n0, 0), p1 = place(n1, j1);
    kp = place(n2, j2);
#pragma unroll
    for (int u = 0; u < LU; ++u)
      reinterpret_cast<u32x4*>(S0 + STAGE + (wave * LU + u) * 1024)[lane] = u32x4{};
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));   // in LDS before barrier 0
#pragma unroll
    for (int u = 0; u < LU; ++u) dma_k(S0, p0, u);
#pragma unroll
    for (int u = 0; u < LU; ++u) { dma_k(S1, p1, u); dma_v(S1 + STAGE, p0, u); }
#pragma unroll
    for (int u = 0; u < LU; ++u) { dma_k(S2, kp, u); dma_v(S2 + STAGE, p1, u); }
  }
  // the stages of a wave without rows (its share of the loads, and the barriers),
  // of the first group, or of the second
  auto run = [&](auto works, auto late, auto Half) {
    constexpr bool WORKS = decltype(works)::value, LATE = decltype(late)::value;
    auto stage = [&](auto J, int j) {
      if constexpr (!LATE) meet(j);
      if constexpr (WORKS) {
        __builtin_amdgcn_s_setprio(1);
        products(yes, Half, J);
        __builtin_amdgcn_s_setprio(0);
      } else {
#pragma unroll
        for (int q = 0; q < 2 * LU; ++q) start(J, q);
      }
      if constexpr (LATE) meet(j + 1);
      if constexpr (WORKS) softmax(Half);
    };
    if constexpr (LATE) meet(0);
    for (int j = 0; j < stages; j += 4) {   // whole fours
      stage(i0, j);
      stage(i1, j + 1);
      stage(i2, j + 2);
      stage(i3, j + 3);
    }
    if constexpr (!LATE) meet(stages);      // as many barriers as the other group's
    if constexpr (WORKS) products(no, Half, i0);
  };
  if (!active) run(no, no, i2);
  else if (wave < NW / 2) { if (split) run(yes, no, i0); else run(yes, no, i2); }
  else { if (split) run(yes, yes, i1); else run(yes, yes, i2); }
  wait_vmcnt<0>();   // no DMA outlives the workgroup
  l = half_sum(l);

  if (split) {       // the second group's results reach the first through LDS
    __syncthreads();
    uint8_t* at = (block < 2 ? S0 : S1) + block % 2 * STAGE;
    float4* po = reinterpret_cast<float4*>(at) + lane;
    float2* ml = reinterpret_cast<float2*>(S2) + block * kBlock;
    if (wave >= NW / 2) {
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          po[(dt * 4 + g) * 64] = float4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2],
                                         o[dt][4 * g + 3]};
      if (half == 0) ml[col] = float2{mu, l};
    }
    __syncthreads();
    if (wave >= NW / 2 || !active) return;
    const float2 x = ml[col];
    const float mn = fmaxf(mu, x.x), z = mn == -INFINITY ? 0.f : mn;
    const float wo = __builtin_amdgcn_exp2f(mu - z), wx = __builtin_amdgcn_exp2f(x.x - z);
    mu = mn;
    l = l * wo + x.y * wx;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 v = po[(dt * 4 + g) * 64];
        o[dt][4 * g] = o[dt][4 * g] * wo + v.x * wx;
        o[dt][4 * g + 1] = o[dt][4 * g + 1] * wo + v.y * wx;
        o[dt][4 * g + 2] = o[dt][4 * g + 2] * wo + v.z * wx;
        o[dt][4 * g + 3] = o[dt][4 * g + 3] * wo + v.w * wx;
      }
  }
  if (!active) return;

  // the wave's block of partial results, straight from the registers
  float4* out = reinterpret_cast<float4*>(part_o<D>(a, head, it.part + block)) + lane;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      out[(dt * 4 + g) * 64] = float4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2],
                                      o[dt][4 * g + 3]};
  if (half == 0) part_ml(a, head, it.part + block)[col] = float2{mu / c2, l};
}

template <typename T, int D>
hipError_t launch(const AttendArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.w.max_items * a.s.hkv);
  if constexpr (sizeof(T) == 2)
    if (a.s.page < kStage)
      hipLaunchKernelGGL((attend_wide_kernel<D, true>), grid, dim3(kWideThreads), 0, st, a);
    else
      hipLaunchKernelGGL((attend_wide_kernel<D, false>), grid, dim3(kWideThreads), 0, st, a);
  else
    hipLaunchKernelGGL((attend_rows_kernel<T, D, false>), grid, dim3(kThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attend_rows_kernel<T, D, true>),
                     dim3((unsigned)((long)a.s.batch * a.w.tiles * a.s.hkv)), dim3(kThreads), 0,
                     st, a);
  return hipGetLastError();
}

}  // namespace

size_t attend_workspace_bytes(const PagesShape& s, int hq, int max_new) {
  return plan_ws(s, hq, max_new).bytes;
}

hipError_t launch_attend_plan(const PagesShape& s, const PagesPtrs& p, int hq, int max_new,
                              const int32_t* groups, void* ws, hipStream_t st) {
  // a wave a sequence: four waves share a SIMD, so that 16 make every step four times as
  // long (one sequence over 2048 keys, all launches: 20.9 us, 22.5 with 16)
  const int waves = min(max(s.batch, 4), kBook / 64);
  const auto kernel = s.bits ? attend_plan_kernel<true, true>
                      : s.dtype == LDR_BF16 ? attend_plan_kernel<true, false>
                                            : attend_plan_kernel<false, false>;
  hipLaunchKernelGGL(kernel, dim3(1), dim3(64 * waves), 0, st, s, p, hq, max_new, groups,
                     static_cast<uint8_t*>(ws), plan_ws(s, hq, max_new));
  return hipGetLastError();
}

hipError_t launch_attend(const PagesShape& s, const PagesPtrs& p, int layer, const void* q,
                         long q_stride, int hq, int max_new, float scale, void* o, float* lse,
                         void* ws, hipStream_t st) {
  if (s.bits) return launch_attend_mx(s, p, layer, q, q_stride, hq, max_new, scale, o, lse, ws, st);
  AttendArgs a{s, p, q, q_stride, o, lse, layer, hq, hq / s.hkv, max_new, scale,
               static_cast<uint8_t*>(ws), plan_ws(s, hq, max_new)};
  if (s.dtype == LDR_BF16)
    return s.d == 128 ? launch<uint16_t, 128>(a, st) : launch<uint16_t, 64>(a, st);
  return s.d == 128 ? launch<float, 128>(a, st) : launch<float, 64>(a, st);
}

}  // namespace ldr
