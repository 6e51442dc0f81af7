// Attention over a cache of coded rows: the plan, the items and the partial results are
// those of attend.hip, the rows are decoded on their way to the matrix products.
//
// The decoded values are bf16 numbers, so products, sums, probabilities and their rounding
// are those of the attention over a bf16 cache. A pair of dimensions is decoded by one
// conversion, at the rate of an ordinary vector instruction, in the ways that suit the work:
//
// Items of up to 32 rows (a token a sequence): every wave takes steps of 32 keys of its
// own and decodes them into the operands of its products; nothing waits for another
// wave until the end. Bound by HBM: 16 sequences with one row over 16384 keys, 32 query and 8
// K/V heads of 128, 4 bits, 60 us a layer (280 MB, 4.7 TB/s), 48 with all keys in cache; 8 bits
// 103 (540 MB, 5.3 TB/s).
//
// Up to 64 rows: the same with two tiles of rows a wave.
//
// More: the workgroup decodes a stage of 64 keys into LDS once for all of its waves, in the
// layout, and between the products, of the bf16 kernel. 64 sequences with one row over 32768
// keys in common, 8 bits, 41 us a layer; 2 with 512 rows over 8192, 4 bits, 124 us, 8 bits 131
// (28 and 108 us of a large matrix product).
//
// What bounds the last two: a wave's matrix products and its vector instructions (the
// exponentials and their neighbours, 110 a tile and step of 32 keys, and 130 of decoding) take
// turns more than they overlap: a step takes nearly the sum of both, whatever the order in
// which they are issued, the priorities of the two waves of a SIMD, or the distance between
// them; one wave a SIMD, with 512 registers and nothing waiting in LDS, was slower still (a
// lone wave issues a vector instruction every 5 to 9 cycles, two one every 4.3).
//
// Two waves a SIMD have 256 registers each. With head_dim 128 the 8-bit kernel spills 6 of
// them, 11 with pages of 32 rows (4 bits 0 and 4), its last kernel 8 with eight waves and 3
// with four (4 bits none; with half of the dimensions a workgroup none); head_dim 64 none. What
// these cost was not measured.
//
// K and q may be taken along head_dim in any order that is the same for both, keys in any
// order that is the same for P and V, and the dimensions of O in any order that all parts
// share: tile t of O^T has the dimensions 64 (t / 2) + 2 r + t % 2 in its rows r, so that
// a lane's pair of dimensions gives the operands of two tiles.
#include "attend_common.h"
#include "mx.h"

namespace ldr {
namespace {

using M16 = Mma<uint16_t>;

// What a lane has of a step of 32 keys, as it is in the cache: half of a K row, and 16 keys
// of a pair of dimensions for each two tiles of O^T (NPL of them).
template <int BITS, int D, int NPL = D / 64> struct RawStep {
  static constexpr int KW = D * BITS / 256, VW = BITS / 4, NP = NPL;
  u32x4 k[KW], v[NP][VW], vs[NP];
  uint32_t ks;
};

// Where a head's rows of a page are.
template <int BITS, int D> struct MxPage {
  static constexpr int kRow = D * BITS / 8, kBlocks = D / kMxBlock, kUnit = BITS / 4;
  const uint8_t* base;
  int page;
  __device__ const uint8_t* k(int row) const { return base + row * kRow; }
  __device__ const uint8_t* kscale(int row) const { return base + page * kRow + row * kBlocks; }
  __device__ const uint8_t* v(int pair, int row) const {
    return base + (pair * page + row) * kUnit;
  }
  __device__ const uint8_t* vscale(int block, int row) const {
    return base + page * kRow + block * page + row;
  }
};

// One value of a V page, where few are needed.
template <int BITS, int D>
__device__ inline float value_of_v(const MxPage<BITS, D>& p, int row, int dim) {
  const uint8_t* pair = p.v(dim / 2, row);
  const uint32_t code = BITS == 4 ? *pair >> (4 * (dim & 1)) & 15 : pair[dim & 1];
  return mx_value<BITS>(code, *p.vscale(dim / kMxBlock, row));
}

// attend_rows_kernel (attend.hip) joins the parts of uncoded caches by the same steps and the
// same places, written out there since as a function it rounds otherwise: a change of where
// parts lie, or of how few rows share the columns, is one to both.
// Into a wave's o, m and l (column col: row it.r0 + col of sequence it.seq): the parts of
// its rows, which W waves take in turn; l in the first half alone. Of O^T the 2 NPL tiles
// from pair p0 of them on, U parts on their way at a time.
template <int D, int W, int NPL, int U>
__device__ inline void join_parts(const AttendArgs& a, const Item& it, const SeqInfo& f, int head,
                                  int wave, int p0, float c2, f32x16 (&o)[2 * NPL], float& m,
                                  float& l) {
  constexpr int ND = 2 * NPL, NV = 8 * NPL;
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  // parts: the group's chunks, then the tile's own. Of few rows there are columns
  // to spare: R a part, and 32 / R parts at a time (4 rows of 32 parts, as 64
  // sequences with one token each have, took 8 loads behind one another, 11 us).
  const int tr = tile_rows(tile_of(a.s), two_tiles(a.s), f.open * a.rep), t = it.r0 / tr * tr;
  const int own = f.own_chunks ? ceil_div(tile_keys(f.rows, f.open, f.share, t, a.rep,
                                                    tile_of(a.s).unit), f.step) : 0;
  const int parts = f.grp_chunks + own;
  int R = 32;
  while (R > 1 && 2 * it.nr <= R && W * 32 < parts * R) R >>= 1;
  const int rp = it.r0 + min(col & (R - 1), it.nr - 1), gr = f.grp_off + rp, each = W * (32 / R);
  for (int c0 = wave + W * (col / R); c0 < parts; c0 += U * each) {
    float2 ml[U];
    float4 v[U][NV];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = min(c0 + u * each, parts - 1);
      const bool g = c < f.grp_chunks;
      const long block = g ? f.grp_part + (long)c * f.grp_blocks + gr / kBlock
                           : f.own_part + (long)(c - f.grp_chunks) * f.own_blocks + it.r0 / kBlock;
      const int at = g ? gr % kBlock : rp % kBlock;
      ml[u] = part_ml(a, head, block)[at];
      const float4* po = reinterpret_cast<const float4*>(part_o<D>(a, head, block)) + half * 32 + at +
                         p0 * 512;
#pragma unroll
      for (int i = 0; i < NV; ++i) v[u][i] = po[i * 64];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u && c0 + u * each >= parts) continue;
      const float mn = fmaxf(m, ml[u].x), mu = mn == -INFINITY ? 0.f : mn;
      const float wo = __builtin_amdgcn_exp2f((m - mu) * c2);
      const float wp = __builtin_amdgcn_exp2f((ml[u].x - mu) * c2);
      m = mn;
      l = l * wo + ml[u].y * wp;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int dt = i / 4, q = i % 4 * 4;
        o[dt][q] = o[dt][q] * wo + v[u][i].x * wp;
        o[dt][q + 1] = o[dt][q + 1] * wo + v[u][i].y * wp;
        o[dt][q + 2] = o[dt][q + 2] * wo + v[u][i].z * wp;
        o[dt][q + 3] = o[dt][q + 3] * wo + v[u][i].w * wp;
      }
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

// Rows it.r0 .. + it.nr (32 at most) over the keys it.k0 .. it.k1, by W waves; `lds`: room
// for W 32 (64 NPL + 4) + 68 W words. FINISH: also the rows' parts; the keys may end anywhere,
// row r sees those up to cbase + r / rep, and the results are written. Of O the NPL pairs of
// tiles from p0 on: dimensions 64 p0 .. 64 (p0 + NPL) - 1.
template <int BITS, int D, bool FINISH, int W, int NPL>
__device__ inline void mx_rows(const AttendArgs& a, const Item& it, const SeqInfo& f, int cbase,
                               int head, int p0, int tid, float* lds) {
  using Raw = RawStep<BITS, D, NPL>;
  using Page = MxPage<BITS, D>;
  constexpr int NF = D / 16, ND = 2 * NPL, DL = 64 * NPL, NT = W * 64;
  const int32_t* map = reinterpret_cast<const int32_t*>(a.ws + a.w.map);
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int32_t* table = a.p.state + a.s.table + (size_t)it.seq * a.s.max_pages;
  const uint8_t* kpool = a.p.pool + (size_t)2 * a.layer * a.s.n_pages * a.s.page_bytes +
                         head * a.s.head_bytes;
  const size_t vplane = (size_t)a.s.n_pages * a.s.page_bytes;

  // the lane's query, half of its dimensions; columns behind the last row repeat it and
  // are not stored
  const int r = it.r0 + min(col, it.nr - 1), qi = r / a.rep, hr = r - qi * a.rep;
  const size_t qrow = FINISH ? (size_t)it.seq * a.max_new + qi : (size_t)map[it.q0 + qi];
  const uint16_t* qp = static_cast<const uint16_t*>(a.q) + qrow * a.q_stride +
                       (head * a.rep + hr) * D + half * (D / 2);
  u32x4 qf[NF];
#pragma unroll
  for (int i = 0; i < NF; ++i) qf[i] = reinterpret_cast<const u32x4*>(qp)[i];

  // the key of a step whose K row this lane loads: entry i of a lane's scores is that of
  // key 16 half + i
  const int krow = (col >> 2 & 1) * 16 + (col >> 3) * 4 + (col & 3);
  const float c2 = a.scale * kLog2e;
  f32x16 o[ND] = {};
  float m = -INFINITY, l = 0.f;
  bool bad = false;   // V held a value that is not finite where a mask is

  const int steps = (max(it.k1 - it.k0, 0) + kStep - 1) / kStep;
  const int shift = 31 - __builtin_clz(a.s.page);
  auto id_of = [&](int t) {   // the page of the wave's step t, on its way until it is looked at
    return scalar_word(table, (it.k0 + min(t * W + wave, max(steps - 1, 0)) * kStep) >> shift);
  };
  // What the rounding of P to bf16 leaves gets a product too (P then has 16 bits) in the last
  // kernel, which is bound by the chain of its loads, and where the waves have few steps, for
  // the same reason: o is then 0.0017 from its definition (root mean square, relative), its
  // own rounding to bf16, instead of 0.0023. Without it in any item 8 sequences with 8 rows
  // over 4096 keys, 4 bits, two layers, take 53 instead of 55 us, the small ones as long. With
  // it in all of these items 16 sequences with one row over 16384 keys, five layers, take 390
  // instead of 340, and with it in the others too 16 with 17 rows over 8192 519 instead of 413,
  // two with 512 over 8192 382 instead of 299: those keep the 8 bits of a bf16 cache. The steps
  // are those of the plan's cut, so that a row's roundings follow from its batch.
  const bool fine = FINISH || steps <= 4 * W;
  int id = wave < steps ? id_of(0) : 0;
  auto fetch = [&](Raw& x, int t) {
    const uint8_t* at = kpool + (size_t)clamp_page(a.s, id) * a.s.page_bytes;
    const int in = (it.k0 + (t * W + wave) * kStep) & (a.s.page - 1);
    const Page kp{at, a.s.page}, vp{at + vplane, a.s.page};
    const u32x4* ka = reinterpret_cast<const u32x4*>(kp.k(in + krow) + half * (Page::kRow / 2));
#pragma unroll
    for (int i = 0; i < Raw::KW; ++i) x.k[i] = ka[i];
    if constexpr (D == 128) x.ks = reinterpret_cast<const uint16_t*>(kp.kscale(in + krow))[half];
    else x.ks = kp.kscale(in + krow)[half];
#pragma unroll
    for (int p = 0; p < Raw::NP; ++p) {
      const u32x4* va = reinterpret_cast<const u32x4*>(vp.v((p0 + p) * 32 + col, in + half * 16));
#pragma unroll
      for (int i = 0; i < Raw::VW; ++i) x.v[p][i] = va[i];
      x.vs[p] = *reinterpret_cast<const u32x4*>(vp.vscale(2 * (p0 + p) + (col >> 4), in + half * 16));
    }
    id = id_of(t + 1);
  };
  Raw ra, rb;
  if (wave < steps) fetch(ra, 0);
  if constexpr (FINISH)
    join_parts<D, W, NPL, NPL * 64 < D ? 2 : 1>(a, it, f, head, wave, p0, c2, o, m, l);
  float mu = m == -INFINITY ? -INFINITY : m * c2;

  auto step = [&](const Raw& now, Raw& next, int t) {
    const int kb = it.k0 + (t * W + wave) * kStep;
    if ((t + 1) * W + wave < steps) fetch(next, t + 1);
    f32x16 sc = {};
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      uint32_t w[BITS / 4];
#pragma unroll
      for (int j = 0; j < BITS / 4; ++j) {
        const int at = i * (BITS / 4) + j;
        w[j] = now.k[at / 4][at % 4];
      }
      u32x4 kf;
      uint32_t x[4];
      mx_eight<BITS>(w, i < 4 ? mx_scale<0>(now.ks) : mx_scale<1>(now.ks), x);
      kf = u32x4{x[0], x[1], x[2], x[3]};
      sc = M16::run(kf, qf[i], sc);
    }
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = sc[i];
    if constexpr (FINISH) {
      const int lim = cbase + qi - kb;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (half * 16 + i > lim) x[i] = -INFINITY;
    }
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
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
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c2, -z));
      sum += x[i];
    }
    l += sum;
    u32x4 pf[2], rest[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) pf[i] = M16::pack(x + i * 8);
    if (fine)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i * 8 + j] -= M16::get(pf[i], j);
        rest[i] = M16::pack(x + i * 8);
      }
#pragma unroll
    for (int p = 0; p < Raw::NP; ++p)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t w[BITS / 2], even[4], odd[4];
#pragma unroll
        for (int j = 0; j < BITS / 2; ++j) {
          const int at = i * (BITS / 2) + j;
          w[j] = now.v[p][at / 4][at % 4];
        }
        mx_turned8<BITS>(w, now.vs[p][2 * i], now.vs[p][2 * i + 1], even, odd);
        u32x4 v0{even[0], even[1], even[2], even[3]}, v1{odd[0], odd[1], odd[2], odd[3]};
        if (FINISH && kb + kStep > cbase + it.r0 / a.rep + 1) {
          bad = clean_values<uint16_t>(v0, kb + half * 16 + i * 8, it.k1) || bad;
          bad = clean_values<uint16_t>(v1, kb + half * 16 + i * 8, it.k1) || bad;
        }
        o[2 * p] = M16::run(v0, pf[i], o[2 * p]);
        o[2 * p + 1] = M16::run(v1, pf[i], o[2 * p + 1]);
        if (fine) {
          o[2 * p] = M16::run(v0, rest[i], o[2 * p]);
          o[2 * p + 1] = M16::run(v1, rest[i], o[2 * p + 1]);
        }
      }
  };
  for (int t = 0; t * W + wave < steps; t += 2) {
    step(ra, rb, t);
    if ((t + 1) * W + wave < steps) step(rb, ra, t + 1);
  }
  l = half_sum(l);
  m = mu == -INFINITY ? mu : mu / c2;

  // join the waves: each one's (m, l) of the 32 rows, then O scaled to the common
  // maximum and added up, four values a thread. O in its dimensions' order for the
  // results, as the products leave it for a part.
  constexpr int LD = DL + 4;
  float* sm = lds + W * 32 * LD;
  float* sl = sm + W * 32;
  int* odds = reinterpret_cast<int*>(sl + W * 32);
  const bool any_bad = __any(bad);
  if (lane == 0) odds[wave] = any_bad;
  if (half == 0) { sm[wave * 32 + col] = m; sl[wave * 32 + col] = l; }
  __syncthreads();
  float mt = sm[col];
#pragma unroll
  for (int k = 1; k < W; ++k) mt = fmaxf(mt, sm[k * 32 + col]);
  const float own = __builtin_amdgcn_exp2f((m - (mt == -INFINITY ? 0.f : mt)) * c2);
  float* so = lds + (wave * 32 + col) * LD;
#pragma unroll
  for (int p = 0; p < ND / 2; ++p)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float e[4], d[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        e[k] = o[2 * p][4 * g + k] * own;
        d[k] = o[2 * p + 1][4 * g + k] * own;
      }
      if constexpr (FINISH) {
        float4* to = reinterpret_cast<float4*>(so + p * 64 + g * 16 + half * 8);
        to[0] = float4{e[0], d[0], e[1], d[1]};
        to[1] = float4{e[2], d[2], e[3], d[3]};
      } else {
        *reinterpret_cast<float4*>(so + p * 64 + g * 8 + half * 4) = float4{e[0], e[1], e[2], e[3]};
        *reinterpret_cast<float4*>(so + p * 64 + 32 + g * 8 + half * 4) =
            float4{d[0], d[1], d[2], d[3]};
      }
    }
  __syncthreads();
  // thread i: values e .. e + 3 of a row; rows fastest for a part's order
  constexpr int NI = 32 * (DL / 4) / NT;
  auto row_of = [](int i) { return FINISH ? i / (DL / 4) : i % 32; };
  auto el_of = [](int i) { return FINISH ? i % (DL / 4) * 4 : i / 32 * 4; };
  float acc[NI][4], ll[NI], mm[NI];
#pragma unroll
  for (int u = 0; u < NI; ++u) {
    const int i = u * NT + tid, row = row_of(i), e = el_of(i);
    mm[u] = sm[row];
#pragma unroll
    for (int k = 1; k < W; ++k) mm[u] = fmaxf(mm[u], sm[k * 32 + row]);
    const float mz = mm[u] == -INFINITY ? 0.f : mm[u];
    ll[u] = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[u][k] = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      ll[u] += sl[k * 32 + row] * __builtin_amdgcn_exp2f((sm[k * 32 + row] - mz) * c2);
      const float4 v = *reinterpret_cast<const float4*>(lds + (k * 32 + row) * LD + e);
      acc[u][0] += v.x; acc[u][1] += v.y; acc[u][2] += v.z; acc[u][3] += v.w;
    }
    if constexpr (FINISH) {
      const float inv = ll[u] == 0.f ? 0.f : 1.f / ll[u];
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[u][k] *= inv;
    }
  }
  if constexpr (FINISH) {
    int any = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) any |= odds[k];
    if (any) {     // the NaN that clean_values took out, to the rows that see them
      const int s0 = max(0, cbase + it.r0 / a.rep + 1 - it.k0) / kStep;
#pragma unroll
      for (int u = 0; u < NI; ++u) {
        const int i = u * NT + tid, row = row_of(i), e = el_of(i);
        const int last = row < it.nr ? cbase + (it.r0 + row) / a.rep : -1;
        for (int k = it.k0 + s0 * kStep; k <= last; ++k) {
          const uint8_t* at = kpool + (size_t)clamp_page(a.s, table[k >> shift]) * a.s.page_bytes;
          const Page vp{at + vplane, a.s.page};
          const int in = k & (a.s.page - 1);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const float v = value_of_v(vp, in, p0 * 64 + e + d);
            if (!(fabsf(v) < INFINITY)) acc[u][d] += v;
          }
        }
      }
    }
    // a row without weight is 0, whatever values 0 was multiplied with
#pragma unroll
    for (int u = 0; u < NI; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[u][k] = ll[u] == 0.f ? 0.f : acc[u][k];
  }
#pragma unroll
  for (int u = 0; u < NI; ++u) {
    const int i = u * NT + tid, row = row_of(i), e = el_of(i);
    if constexpr (FINISH) {
      if (row >= it.nr) continue;
      const int rr = it.r0 + row, q = rr / a.rep;
      const size_t at = ((size_t)it.seq * a.max_new + q) * a.hq + head * a.rep + (rr - q * a.rep);
      M16::store4(static_cast<uint16_t*>(a.o) + at * D + p0 * 64 + e, acc[u]);
      if (e == 0 && p0 == 0 && a.lse) a.lse[at] = ll[u] == 0.f ? -INFINITY : mm[u] * a.scale + logf(ll[u]);
    } else {
      reinterpret_cast<float4*>(part_o<D>(a, head, it.part))[(e / 8) * 64 + (e / 4 % 2) * 32 + row] =
          float4{acc[u][0], acc[u][1], acc[u][2], acc[u][3]};
      if (e == 0) part_ml(a, head, it.part)[row] = float2{mm[u], ll[u]};
    }
  }
}

// The last kernel: the parts of 32 rows, the keys behind them, and the results.
// W waves: 4, two workgroups a compute unit; 8 where no more workgroups than compute units
// are there. NPL: of the dimensions, all or half, two workgroups for them.
template <int BITS, int D, int W, int NPL>
__global__ void __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
attend_mx_last_kernel(AttendArgs a) {
  __shared__ alignas(16) float lds[W * 32 * (64 * NPL + 4) + 68 * W];
  constexpr int SPLIT = D / 64 / NPL;
  const int unit = (int)(blockIdx.x / SPLIT / a.s.hkv), head = (int)(blockIdx.x / SPLIT % a.s.hkv);
  const int items = scalar_word(a.ws, 3);
  Item it{};
  it.seq = unit / a.w.tiles;
  it.r0 = (unit - it.seq * a.w.tiles) * kBlock;
  const SeqInfo f = scalar_info(a.ws + a.w.info, it.seq);
  if (!plan_ok(a, items) || it.r0 >= f.open * a.rep) return;
  it.nr = min(kBlock, f.open * a.rep - it.r0);
  it.q0 = f.qoff;
  const int cbase = f.rows - f.open;
  const Tile tile = tile_of(a.s);
  const int tr = tile_rows(tile, two_tiles(a.s), f.open * a.rep), t = it.r0 / tr * tr;
  it.k0 = f.share + (f.own_chunks ? tile_keys(f.rows, f.open, f.share, t, a.rep, tile.unit) : 0);
  it.k1 = cbase + (it.r0 + it.nr - 1) / a.rep + 1;
  mx_rows<BITS, D, true, W, NPL>(a, it, f, cbase, head, (int)blockIdx.x % SPLIT * NPL,
                                 (int)threadIdx.x, lds);
}

// An item of 33 to 64 rows: as mx_rows, but a wave has both tiles of 32 rows, so that a key
// is decoded once for them. The queries are in LDS. Rows of a step are loaded where those of
// the last one have been taken: the two waves of a SIMD have the time of the other one's
// instructions too.
template <int BITS, int D>
__device__ inline void mx_pair(const AttendArgs& a, const Item& it, int head, int tid, float* lds) {
  using Raw = RawStep<BITS, D>;
  using Page = MxPage<BITS, D>;
  constexpr int NF = D / 16, ND = D / 32, W = kWideThreads / 64, NT = kWideThreads;
  const int32_t* map = reinterpret_cast<const int32_t*>(a.ws + a.w.map);
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int32_t* table = a.p.state + a.s.table + (size_t)it.seq * a.s.max_pages;
  const uint8_t* kpool = a.p.pool + (size_t)2 * a.layer * a.s.n_pages * a.s.page_bytes +
                         head * a.s.head_bytes;
  const size_t vplane = (size_t)a.s.n_pages * a.s.page_bytes;
  constexpr int N = 2;                    // tiles

  u32x4* qs = reinterpret_cast<u32x4*>(lds);
  for (int f = wave; f < N * NF; f += W) {
    const int r = it.r0 + min(f / NF * kBlock + col, it.nr - 1), qi = r / a.rep;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) +
                         (size_t)map[it.q0 + qi] * a.q_stride +
                         (head * a.rep + r - qi * a.rep) * D + half * (D / 2) + f % NF * 8;
    qs[f * 64 + lane] = *reinterpret_cast<const u32x4*>(qp);
  }
  const int krow = (col >> 2 & 1) * 16 + (col >> 3) * 4 + (col & 3);
  const float c2 = a.scale * kLog2e;
  f32x16 o[2][ND] = {};
  float mu[2] = {-INFINITY, -INFINITY}, l[2] = {};
  const int steps = (it.k1 - it.k0) / kStep;
  const int shift = 31 - __builtin_clz(a.s.page);
  auto id_of = [&](int t) {
    return scalar_word(table, (it.k0 + min(t * W + wave, steps - 1) * kStep) >> shift);
  };
  Raw x;
  int id = id_of(0);
  const uint8_t* page = nullptr;
  int in = 0;
  auto go_to = [&](int t) {
    page = kpool + (size_t)clamp_page(a.s, id) * a.s.page_bytes;
    in = (it.k0 + min(t * W + wave, steps - 1) * kStep) & (a.s.page - 1);
    id = id_of(t + 1);
  };
  auto load_k = [&]() {
    const Page kp{page, a.s.page};
    const u32x4* ka = reinterpret_cast<const u32x4*>(kp.k(in + krow) + half * (Page::kRow / 2));
#pragma unroll
    for (int i = 0; i < Raw::KW; ++i) x.k[i] = ka[i];
    if constexpr (D == 128) x.ks = reinterpret_cast<const uint16_t*>(kp.kscale(in + krow))[half];
    else x.ks = kp.kscale(in + krow)[half];
  };
  auto load_v = [&]() {
    const Page vp{page + vplane, a.s.page};
#pragma unroll
    for (int p = 0; p < Raw::NP; ++p) {
      const u32x4* va = reinterpret_cast<const u32x4*>(vp.v(p * 32 + col, in + half * 16));
#pragma unroll
      for (int i = 0; i < Raw::VW; ++i) x.v[p][i] = va[i];
      x.vs[p] = *reinterpret_cast<const u32x4*>(vp.vscale(2 * p + (col >> 4), in + half * 16));
    }
  };
  go_to(0);
  load_k();
  __syncthreads();
  const u32x4* qw = qs + lane;
  {
    for (int t = 0; t * W + wave < steps; ++t) {
      __builtin_amdgcn_s_setprio(1);      // before the other wave's vector instructions
      f32x16 sc[N] = {};
      // query fragments kAhead products in front; held there, or all of them are in registers
      constexpr int kAhead = BITS == 4 ? 6 : 4, R = kAhead + N;
      u32x4 fr[R];
      auto read = [&](int n) { fr[n % R] = qw[(n % N * NF + n / N) * 64]; };
#pragma unroll
      for (int n = 0; n < kAhead; ++n) read(n);
#pragma unroll
      for (int i = 0; i < NF; ++i) {
        __builtin_amdgcn_sched_barrier(0x6);
#pragma unroll
        for (int n = i * N + kAhead; n < (i + 1) * N + kAhead; ++n)
          if (n < N * NF) read(n);
        __builtin_amdgcn_sched_barrier(0x6);
        uint32_t w[BITS / 4], k[4];
#pragma unroll
        for (int j = 0; j < BITS / 4; ++j) {
          const int at = i * (BITS / 4) + j;
          w[j] = x.k[at / 4][at % 4];
        }
        mx_eight<BITS>(w, i < 4 ? mx_scale<0>(x.ks) : mx_scale<1>(x.ks), k);
#pragma unroll
        for (int u = 0; u < N; ++u)
          sc[u] = M16::run(u32x4{k[0], k[1], k[2], k[3]}, fr[(i * N + u) % R], sc[u]);
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
      // V's rows of this step, not before K's products: with both there the accumulators
      // leave no room for the queries on their way from LDS
      load_v();
      go_to(t + 1);
      load_k();
      u32x4 pf[N][2];
#pragma unroll
      for (int u = 0; u < N; ++u) {
        float mx = sc[u][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[u][i]);
        mx = half_max(mx) * c2;
        const bool up = mx > mu[u] + kLazy;
        if (__any(up)) {
          const float mn = up ? ceilf(mx) : mu[u];
          const float alpha = up ? __builtin_amdgcn_exp2f(mu[u] - mn) : 1.f;
          mu[u] = mn;
          l[u] *= alpha;
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) o[u][dt] *= alpha;
        }
        const float z = mu[u] == -INFINITY ? 0.f : mu[u];
        float e[16], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          e[i] = __builtin_amdgcn_exp2f(fmaf(sc[u][i], c2, -z));
          sum += e[i];
        }
        l[u] += sum;
#pragma unroll
        for (int i = 0; i < 2; ++i) pf[u][i] = M16::pack(e + i * 8);
      }
      // the values, eight keys of two tiles of O^T at a time: the next ones are decoded
      // between the products
      constexpr int G = 2 * Raw::NP;
      u32x4 vf[2][2];
      auto decode = [&](int g) {
        uint32_t w[BITS / 2], even[4], odd[4];
        const int p = g / 2, i = g % 2;
#pragma unroll
        for (int j = 0; j < BITS / 2; ++j) {
          const int at = i * (BITS / 2) + j;
          w[j] = x.v[p][at / 4][at % 4];
        }
        mx_turned8<BITS>(w, x.vs[p][2 * i], x.vs[p][2 * i + 1], even, odd);
        vf[g % 2][0] = u32x4{even[0], even[1], even[2], even[3]};
        vf[g % 2][1] = u32x4{odd[0], odd[1], odd[2], odd[3]};
      };
      __builtin_amdgcn_sched_barrier(0);
      decode(0);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        __builtin_amdgcn_sched_barrier(0);
        if (g + 1 < G) decode(g + 1);
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int u = 0; u < N; ++u)
            o[u][g / 2 * 2 + q] = M16::run(vf[g % 2][q], pf[u][g % 2], o[u][g / 2 * 2 + q]);
        if (g + 1 < G)
#pragma unroll
          for (int q = 0; q < 2 * N; ++q) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);             // a product
            __builtin_amdgcn_sched_group_barrier(0x2, 24 / (2 * N), 0);  // and decoding
          }
      }
      __builtin_amdgcn_sched_barrier(0);
        }
  }

  // join the waves, a tile after the other
  constexpr int LD = D + 4;
  float* sm = lds + W * 32 * LD;
  float* sl = sm + W * 32;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const float lu = half_sum(l[u]);
    __syncthreads();       // the queries, or the last tile, have been read
    if (half == 0) { sm[wave * 32 + col] = mu[u]; sl[wave * 32 + col] = lu; }
    __syncthreads();
    float mt = sm[col];
#pragma unroll
    for (int k = 1; k < W; ++k) mt = fmaxf(mt, sm[k * 32 + col]);
    const float own = __builtin_amdgcn_exp2f(mu[u] - (mt == -INFINITY ? 0.f : mt));
    float* so = lds + (wave * 32 + col) * LD;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(so + dt * 32 + g * 8 + half * 4) =
            float4{o[u][dt][4 * g] * own, o[u][dt][4 * g + 1] * own, o[u][dt][4 * g + 2] * own,
                   o[u][dt][4 * g + 3] * own};
    __syncthreads();
    constexpr int NI = 32 * (D / 4) / NT;
#pragma unroll
    for (int v = 0; v < NI; ++v) {
      const int i = v * NT + tid, row = i % 32, e = i / 32 * 4;
      float mm = sm[row], ll = 0.f;
      float4 acc{};
#pragma unroll
      for (int k = 1; k < W; ++k) mm = fmaxf(mm, sm[k * 32 + row]);
      const float mz = mm == -INFINITY ? 0.f : mm;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        ll += sl[k * 32 + row] * __builtin_amdgcn_exp2f(sm[k * 32 + row] - mz);
        const float4 y = *reinterpret_cast<const float4*>(lds + (k * 32 + row) * LD + e);
        acc.x += y.x; acc.y += y.y; acc.z += y.z; acc.w += y.w;
      }
      const long at = it.part + u;
      reinterpret_cast<float4*>(part_o<D>(a, head, at))[(e / 8) * 64 + (e / 4 % 2) * 32 + row] = acc;
      if (e == 0) part_ml(a, head, at)[row] = float2{mm == -INFINITY ? mm : mm / c2, ll};
    }
  }
}

// An item of more than 64 rows: 32 a wave, over stages of 64 keys that the workgroup decodes
// into LDS. As in the bf16 kernel the two waves of a SIMD belong to two groups half a stage
// apart, one in the matrix unit while the other makes probabilities, and a stage has one
// barrier. Buffer j mod 2 has K of stage j and V of j - 1, which the products of stage j read
// between barriers j and j + 1; in the same interval every wave decodes its share of the next
// buffer, K of j + 1 and V of j, from registers and loads what is two stages on.
// Measured and left out: a ring of coded stages in LDS, filled by DMA (memory is not what is
// waited for: with all keys in cache 68 rows take as long), stages of 128 keys for up to 128
// rows, and those rows as pairs of tiles, each with waves of its own, in registers (16 sequences
// with 60 to 68 rows over 8192 keys 70 to 77 us a layer whichever it is; of 8 bits, one with
// 68 rows over 65536 keys 42 us so, 57 in registers).
// Of 65 to 96 rows as one tile two waves have no rows, and decode their share like the others (8
// bits, 16 sequences with 68 rows over 8192 keys, two layers: 183 us; all of V left to those two
// 200, K and V 217).
template <int BITS, int D, bool SMALL>
__device__ inline void mx_wide(const AttendArgs& a, const Item& it, int head, int tid, uint8_t* lds) {
  using Page = MxPage<BITS, D>;
  constexpr int NF = D / 16, ND = D / 32, NW = kWideThreads / 64;
  constexpr int KC = D / 8;                          // 16-byte chunks of a K row in LDS
  constexpr int STAGE = kStage * D * 2;              // bytes of a stage of K (or V) there
  constexpr int KE = D / 64;                         // chunks of K that a thread decodes
  constexpr int KB = KE * BITS / 4, VB = BITS / 2;   // words of K and V that it loads
  const int32_t* map = reinterpret_cast<const int32_t*>(a.ws + a.w.map);
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int32_t* table = a.p.state + a.s.table + (size_t)it.seq * a.s.max_pages;
  const uint8_t* kpool = a.p.pool + (size_t)2 * a.layer * a.s.n_pages * a.s.page_bytes +
                         head * a.s.head_bytes;
  const size_t vplane = (size_t)a.s.n_pages * a.s.page_bytes;

  // up to 128 rows: both groups take the same rows, each 32 of a stage's keys, and join
  // at the end. The lane's query; columns behind the last row repeat it.
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

  // the thread's share of a stage: 8 KE dimensions of one K row, eight keys of one pair
  // of V's (of 64 dimensions half of the waves have none)
  const int shift = 31 - __builtin_clz(a.s.page);
  const int kr = wave * 8 + lane / 8, kc = lane % 8;        // row, piece of it
  const int vp = (wave * 8 + lane / 8) % (D / 2), oct = lane % 8;
  const bool has_v = wave * 8 < D / 2;
  struct Place { const uint8_t *a, *b; int in; };           // pages of the stage's halves
  struct Ids { int a, b; };
  auto ids_of = [&](int j) {     // on their way until they are looked at
    const int k = it.k0 + j * kStage;
    return Ids{scalar_word(table, k >> shift), SMALL ? scalar_word(table, (k + 32) >> shift) : 0};
  };
  auto place = [&](Ids ids, int j) {
    Place p;
    p.a = kpool + (size_t)clamp_page(a.s, ids.a) * a.s.page_bytes;
    p.b = SMALL ? kpool + (size_t)clamp_page(a.s, ids.b) * a.s.page_bytes : p.a;
    p.in = SMALL ? 0 : (it.k0 + j * kStage) & (a.s.page - 1);
    return p;
  };
  struct Raw { uint32_t k[KB], v[VB], ks; uint2 vs; };
  auto load = [&](auto& to, const uint32_t* from, auto n) {
    constexpr int N = decltype(n)::value;
    if constexpr (N == 1) to[0] = from[0];
    else if constexpr (N == 2) {
      const uint2 t = *reinterpret_cast<const uint2*>(from);
      to[0] = t.x; to[1] = t.y;
    } else {
      const u32x4 t = *reinterpret_cast<const u32x4*>(from);
      to[0] = t[0]; to[1] = t[1]; to[2] = t[2]; to[3] = t[3];
    }
  };
  auto load_k = [&](Raw& x, const Place& p) {
    const Page pg{SMALL && wave >= 4 ? p.b : p.a, a.s.page};
    const int row = p.in + (SMALL ? kr & 31 : kr);
    load(x.k, reinterpret_cast<const uint32_t*>(pg.k(row) + kc * (KB * 4)),
         std::integral_constant<int, KB>{});
    x.ks = pg.kscale(row)[kc * KE * 8 / kMxBlock];
  };
  auto load_v = [&](Raw& x, const Place& p) {
    if (!has_v) return;
    const Page pg{(SMALL && oct >= 4 ? p.b : p.a) + vplane, a.s.page};
    const int row = p.in + (SMALL ? oct % 4 : oct) * 8;
    load(x.v, reinterpret_cast<const uint32_t*>(pg.v(vp, row)), std::integral_constant<int, VB>{});
    x.vs = *reinterpret_cast<const uint2*>(pg.vscale(vp / (kMxBlock / 2), row));
  };
  auto put_k = [&](uint8_t* to, const Raw& x, int c) {     // chunk c of the thread's
    uint32_t o[4];
    mx_eight<BITS>(x.k + c * (BITS / 4), mx_scale<0>(x.ks), o);
    *reinterpret_cast<u32x4*>(to + kr * (2 * D) + (((kc * KE + c) ^ turn<KC>(kr)) << 4)) =
        u32x4{o[0], o[1], o[2], o[3]};
  };
  const int vrow = (vp >> 5) * 64 + (vp & 31);             // of the even dimension in LDS
  auto put_v = [&](uint8_t* to, const Raw& x) {
    if (!has_v) return;
    uint32_t even[4], odd[4];
    mx_turned8<BITS>(x.v, x.vs.x, x.vs.y, even, odd);
    uint8_t* at = to + vrow * 128 + ((oct ^ turn<8>(vrow)) << 4);   // 32 rows on, the same
    *reinterpret_cast<u32x4*>(at) = u32x4{even[0], even[1], even[2], even[3]};
    *reinterpret_cast<u32x4*>(at + 32 * 128) = u32x4{odd[0], odd[1], odd[2], odd[3]};
  };

  // the set of stage j + 1 (its K, and V of j) is ra or rb by j + 1's parity
  Raw ra, rb;
  Ids next;       // pages of the next K to load
  Place kp, vpl;  // where the K and V of the next set to load are
  auto advance = [&](int j) {    // to the set of stage j
    vpl = kp;
    kp = place(next, min(j, stages - 1));
    next = ids_of(min(j + 1, stages - 1));
  };
  constexpr int kTasks = KE + 2;
  // task q of stage j, its parity odd or not: of the next buffer's decoding, and the loads
  auto task = [&](auto Odd, int j, int q) {
    constexpr bool ODD = decltype(Odd)::value;
    uint8_t* to = lds + (ODD ? 0 : 2 * STAGE);
    Raw& x = ODD ? ra : rb;
    if (q < KE) put_k(to, x, q);
    else if (q == KE) put_v(to + STAGE, x);
    else { advance(j + 3); load_k(x, kp); load_v(x, vpl); }
  };

  // fragments: K rows in the order that leaves a lane 8 consecutive keys. The
  // swizzle makes a fragment's offset that of the first with bits flipped.
  const int mi = ((col >> 3) << 2) | (col & 3), mh = (col >> 2) & 1;
  const int krow = mi / 8 * 16 + mh * 8 + mi % 8;
  const uint32_t klane = krow * (2 * D) + ((half ^ turn<KC>(krow)) << 4);
  const uint32_t vlane = col * 128 + ((half ^ turn<8>(col)) << 4);

  const float c2 = a.scale * kLog2e;
  f32x16 o[ND] = {};
  float mu = -INFINITY, l = 0.f;
  f32x16 sc[2];
  u32x4 pf[4] = {};      // none before the first stage, and its V is 0
  // The products of stage j: V^T P^T of j - 1, then (unless j is the end) K Q^T of j, two
  // at a time, with the LDS reads kAhead fragments in front of them and the tasks between
  // them. Half: 0 or 1, or both (2).
  auto products = [&](auto scores, auto Half, auto Odd, int j) {
    constexpr int H = decltype(Half)::value, NS = H == 2 ? 2 : 1, F0 = H == 1 ? 2 : 0;
    constexpr int G = 2, kAhead = 4, R = kAhead + G;
    constexpr int NV = 2 * NS * ND, N = NV + (decltype(scores)::value ? NS * NF : 0);
    constexpr int EACH = N / kTasks < G ? G : N / kTasks / G * G;     // products a task
    static_assert(N % G == 0 && kAhead % G == 0, "whole groups");
    static_assert(!decltype(scores)::value || EACH * kTasks <= N, "room for every task");
    const uint8_t* kb = lds + (decltype(Odd)::value ? 2 * STAGE : 0) + (H == 1 ? 64 * D : 0);
    const uint8_t* vb = lds + (decltype(Odd)::value ? 3 * STAGE : STAGE);
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
      if (decltype(scores)::value && i0 % EACH == 0 && i0 / EACH < kTasks) task(Odd, j, i0 / EACH);
#pragma unroll
      for (int i = i0 + kAhead; i < i0 + kAhead + G; ++i)
        if (i < N) read(i);
      __builtin_amdgcn_sched_barrier(0x6);
#pragma unroll
      for (int i = i0; i < i0 + G; ++i) {
        if (i < NV) {
          o[i % ND] = M16::run(fr[i % R], pf[i / ND], o[i % ND]);
        } else {
          const int f = (i - NV) / NS, sub = (i - NV) % NS;
          sc[sub] = M16::run(fr[i % R], qf[f], f ? sc[sub] : f32x16{});
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
      for (int f = 0; f < 2; ++f) pf[sub * 2 + f] = M16::pack(x + 8 * f);
    }
    l += sum[0] + sum[1];
  };

  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  std::integral_constant<int, 0> i0;
  std::integral_constant<int, 1> i1;
  std::integral_constant<int, 2> i2;
  // what is in LDS is there before the barrier; loads in flight go on
  auto meet = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  // buffer 0: K of stage 0, no V yet; the sets of stages 1 and 2. Each kind of wave on its own:
  // loaded before they part, the sets take more registers than there are (64 sequences with one
  // row over 32768 keys in common, 8 bits, two layers: 148 us so, 153 before).
  auto begin = [&]() {
    kp = place(ids_of(0), 0);
    next = ids_of(min(1, stages - 1));
    load_k(ra, kp);
    u32x4* zero = reinterpret_cast<u32x4*>(lds + STAGE);
    for (int i = tid; i < STAGE / 16; i += kWideThreads) zero[i] = u32x4{};
    advance(1);
    load_k(rb, kp);
    load_v(rb, vpl);
#pragma unroll
    for (int c = 0; c < KE; ++c) put_k(lds, ra, c);
    advance(2);
    load_k(ra, kp);
    load_v(ra, vpl);
  };
  // the stages of a wave without rows (its share of the decoding, and the barriers),
  // of the first group, or of the second
  auto run = [&](auto works, auto late, auto Half) {
    constexpr bool WORKS = decltype(works)::value, LATE = decltype(late)::value;
    auto stage = [&](auto Odd, int j) {
      if constexpr (!LATE) meet();
      if constexpr (WORKS) {
        __builtin_amdgcn_s_setprio(1);
        products(yes, Half, Odd, j);
        __builtin_amdgcn_s_setprio(0);
      } else {
#pragma unroll
        for (int q = 0; q < kTasks; ++q) task(Odd, j, q);
      }
      if constexpr (LATE) meet();
      if constexpr (WORKS) softmax(Half);
    };
    begin();
    if constexpr (LATE) meet();
    for (int j = 0; j < stages; j += 2) {   // whole twos
      stage(no, j);
      stage(yes, j + 1);
    }
    if constexpr (!LATE) meet();            // as many barriers as the other group's
    if constexpr (WORKS) products(no, Half, no, stages);
  };
  if (!active) run(no, no, i2);
  else if (wave < NW / 2) { if (split) run(yes, no, i0); else run(yes, no, i2); }
  else { if (split) run(yes, yes, i1); else run(yes, yes, i2); }
  l = half_sum(l);

  if (split) {       // the second group's results reach the first through LDS
    __syncthreads();
    float4* po = reinterpret_cast<float4*>(lds + block * STAGE) + lane;
    float2* ml = reinterpret_cast<float2*>(lds + 4 * STAGE) + block * kBlock;
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
    if (wave >= NW / 2 || !active) return;      // from the item
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
  if (!active) return;      // from the item

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

// SMALL: pages of 32 rows, half a stage.
template <int BITS, int D, bool SMALL>
__global__ void __launch_bounds__(kWideThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
attend_mx_kernel(AttendArgs a) {
  constexpr int W = kWideThreads / 64;
  constexpr int kRows = (W * 32 * (D + 4) + 68 * W) * 4;
  constexpr int kWide = 4 * kStage * D * 2 + W / 2 * kBlock * 8;
  __shared__ alignas(1024) uint8_t lds[kRows > kWide ? kRows : kWide];
  const int items = scalar_word(a.ws, 3);
  if (!plan_ok(a, items)) return;
  // the items in turn: a workgroup that found none would wait for the LDS of one that did
  for (int i = blockIdx.x; i < items * a.s.hkv; i += gridDim.x) {
    const int item = i / a.s.hkv, head = i - item * a.s.hkv;
    const Item it = scalar_item(a.ws + a.w.items, item);
    if (it.k1 <= it.k0) continue;
    // not the same to the compiler in every round: what it would keep of a lane's places for
    // all kinds of items are 60 registers more than there are
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    if (it.nr <= kBlock)
      mx_rows<BITS, D, false, W, D / 64>(a, it, SeqInfo{}, 0, head, 0, tid,
                                         reinterpret_cast<float*>(lds));
    else if (it.nr <= 2 * kBlock)
      mx_pair<BITS, D>(a, it, head, tid, reinterpret_cast<float*>(lds));
    else
      mx_wide<BITS, D, SMALL>(a, it, head, tid, lds);
    __syncthreads();
  }
}

// Workgroups that run at once: one a compute unit, by their registers and LDS.
constexpr int kSlots = 256;

template <int BITS, int D> hipError_t launch(const AttendArgs& a, hipStream_t st) {
  const int64_t most = (int64_t)a.w.max_items * a.s.hkv;
  const dim3 grid((unsigned)(most < kSlots ? most : kSlots));
  if (a.s.page < kStage)
    hipLaunchKernelGGL((attend_mx_kernel<BITS, D, true>), grid, dim3(kWideThreads), 0, st, a);
  else
    hipLaunchKernelGGL((attend_mx_kernel<BITS, D, false>), grid, dim3(kWideThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t last = (int64_t)a.s.batch * a.w.tiles * a.s.hkv;
  // Few workgroups are bound by their chain of loads: two for the dimensions of 32 rows, unless
  // one would write over queries that the other reads. 32 query and 8 K/V heads, two layers: one
  // sequence with 17 rows over 65536 keys, 8 bits, 115 us instead of 124, 4 with 17 over 16384, 4
  // bits, 92 instead of 98, 16 with one over 16384, 8 bits, 234 instead of 244. Two rounds of
  // workgroups are slower: 4 bits, 8 with 17 over 4096 84 instead of 77, 20 with one over 5000 95
  // instead of 88 (but 6 with 17 over 4096, 8 bits, 68 instead of 75).
  const char *q = static_cast<const char*>(a.q), *o = static_cast<const char*>(a.o);
  const int64_t rows = (int64_t)a.s.batch * a.max_new;
  const bool apart = o + rows * a.hq * D * 2 <= q || q + rows * a.q_stride * 2 <= o;
  if (D == 128 && 2 * last <= kSlots && apart)
    hipLaunchKernelGGL((attend_mx_last_kernel<BITS, D, 8, 1>), dim3((unsigned)last * 2), dim3(512), 0,
                       st, a);
  else if (last <= kSlots)
    hipLaunchKernelGGL((attend_mx_last_kernel<BITS, D, 8, D / 64>), dim3((unsigned)last), dim3(512),
                       0, st, a);
  else
    hipLaunchKernelGGL((attend_mx_last_kernel<BITS, D, 4, D / 64>), dim3((unsigned)last), dim3(256),
                       0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_mx(const PagesShape& s, const PagesPtrs& p, int layer, const void* q,
                            long q_stride, int hq, int max_new, float scale, void* o, float* lse,
                            void* ws, hipStream_t st) {
  AttendArgs a{s, p, q, q_stride, o, lse, layer, hq, hq / s.hkv, max_new, scale,
               static_cast<uint8_t*>(ws), plan_ws(s, hq, max_new)};
  if (s.bits == 4) return s.d == 128 ? launch<4, 128>(a, st) : launch<4, 64>(a, st);
  return s.d == 128 ? launch<8, 128>(a, st) : launch<8, 64>(a, st);
}

}  // namespace ldr
