// Log probabilities of given tokens, the entropy of their rows, the tokens' ranks, and
// the rows' largest entries.
//
// With m the largest logit of a row, x_v = (z_v - m) / T and S = sum e^{x_v}, which is the
// number of entries equal to m plus the rest R:
//   log p(v) = x_v - log S,  entropy = log S - sum e^{x_v} x_v / S,  log S = log1p(S - 1),
// so that a nearly certain token keeps its digits. One pass over the logits cuts a row
// into pieces; a piece stays in registers while its m, and then its sums, are taken, and it
// counts the entries that rank before the token. A second launch joins the pieces of a row.
//
// The n largest entries are among the n groups of 64 neighbours with the largest maxima (in
// the order by value, then by index: a group that is not has n entries before any of its
// own). The first pass writes the maxima; the second picks the groups, then the entries in
// them (select).
//
// Bound by the one read of the logits: 1024 rows of 151936, the largest entry of each, 137 to 142
// us a pass in a loop, 123 to 125 without (622 MB, 5.0 TB/s); launches that stand apart 138 to
// 154 and 14, 126 to 130 and 5. 16 sequences with up to 17 rows, 20 entries, 24 and 14 us: 2700
// workgroups, of which 1280 run at once by their registers. One row 3.6 and 8 us, chains of loads.
#include "serve_internal.h"

namespace ldr {
namespace {

constexpr int kThreads = 256;
constexpr int kGroup = 64;        // neighbours that share a maximum
constexpr int kPicked = 4096;     // keys that a workgroup which picks entries holds
constexpr int kMostTop = 64;

// An exponent whose power is 0: -inf times that is to be 0 too.
constexpr float kFar = -1e4f;
struct __attribute__((packed, aligned(4))) Four { float x[4]; };   // rows may start anywhere

// A piece of a row: its maximum, how many entries equal it, the others' sum of e^x and the
// sum of e^x x (x of base 2), and the entries that rank before the token.
struct Piece { float m, rest, ex; int ones, before; };

struct LogprobsArgs {
  const float* z; long stride;
  const int32_t* tokens; const int32_t* n_rows;
  int rows, vocab, pieces, groups, top;
  float temperature, c;           // c: log2(e) / T
  float *logp, *entropy; int32_t* rank; int32_t* top_tokens; float* top_logp;
  Piece* parts; uint32_t* maxima;
};

// Larger entries have larger keys; a NaN's is the lowest.
__device__ inline uint32_t key_of(float z) { return z == z ? order_key(z) : 0u; }

// Over a wave, in every lane: rows of 16 by lane swaps, then the four rows.
__device__ inline float lane_of(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ inline float wave_max(float v) {
  v = max16(v);
  return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
__device__ inline float wave_sum(float v) {
  v = sum16(v);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
__device__ inline int wave_sum(int v) {
  v += __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, false);
  v += __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, false);
  v += __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, false);
  v += __builtin_amdgcn_mov_dpp(v, 0x140, 0xF, 0xF, false);
  return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) +
         __builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48);
}

// One piece of 1024 U entries: thread t has four of every 1024.
template <int U, bool TOP>
__global__ void __launch_bounds__(kThreads) logprobs_pieces_kernel(LogprobsArgs a) {
  constexpr int W = kThreads / 64;
  __shared__ float sm[W], srest[W], sex[W];
  __shared__ int sones[W], sbefore[W];
  const int b = blockIdx.z, i = blockIdx.y, piece = blockIdx.x;
  if (a.n_rows && i >= a.n_rows[b]) return;
  const size_t row = (size_t)b * a.rows + i;
  const float* z = a.z + row * a.stride;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int first = piece * (1024 * U) + (int)threadIdx.x * 4;
  const int y = a.tokens[row];
  const bool given = y >= 0 && y < a.vocab;
  const float zy = given ? z[y] : NAN;
  float v[U][4];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = first + u * 1024;
    if (at + 4 <= a.vocab) {
      const Four f = *reinterpret_cast<const Four*>(z + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[u][k] = f.x[k];
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[u][k] = at + k < a.vocab ? z[at + k] : -INFINITY;
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = first + u * 1024;
    float g = NAN;            // stays where all are NaN
#pragma unroll
    for (int k = 0; k < 4; ++k) g = fmaxf(g, at + k < a.vocab ? v[u][k] : NAN);
    m = fmaxf(m, g);
    if constexpr (TOP) {      // a group is the entries of 16 lanes
      const float most = max16(g);
      if (lane % 16 == 0 && at < a.vocab) a.maxima[row * a.groups + at / kGroup] = key_of(most);
    }
  }
  m = wave_max(m);
  if (lane == 0) sm[wave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) m = fmaxf(m, sm[w]);
  const float base = m == -INFINITY ? 0.f : m;
  float rest = 0.f, ex = 0.f;
  int ones = 0, before = 0;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float w = v[u][k], x = (w - base) * a.c, e = __builtin_amdgcn_exp2f(x);
      ones += __builtin_popcountll(__ballot(w == m));
      rest += w == m ? 0.f : e;
      ex = fmaf(e, fmaxf(x, kFar), ex);       // of -inf: 0
      before += w > zy || (w == zy && first + u * 1024 + k < y);
    }
  if (zy != zy && given) {                      // behind every number
    before = 0;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int at = first + u * 1024 + k;
        before += at < a.vocab && (v[u][k] == v[u][k] || at < y);
      }
  }
  rest = wave_sum(rest);
  ex = wave_sum(ex);
  before = wave_sum(before);
  if (lane == 0) { srest[wave] = rest; sex[wave] = ex; sones[wave] = ones; sbefore[wave] = before; }
  __syncthreads();
  if (threadIdx.x == 0) {
    Piece p{m, 0.f, 0.f, 0, 0};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      p.rest += srest[w]; p.ex += sex[w]; p.ones += sones[w]; p.before += sbefore[w];
    }
    a.parts[row * a.pieces + piece] = p;
  }
}

// An entry's place in the order: its value's key above the complement of its index, so that
// no two are equal; 0: none.
typedef uint64_t Key;
__device__ inline Key place_of(uint32_t key, int index) { return (Key)key << 32 | (uint32_t)~index; }
__device__ inline int index_of(Key k) { return (int)~(uint32_t)k; }

template <int CTRL> __device__ inline Key key_dpp(Key k) {
  const uint32_t lo = __builtin_amdgcn_mov_dpp((int)(uint32_t)k, CTRL, 0xF, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_mov_dpp((int)(uint32_t)(k >> 32), CTRL, 0xF, 0xF, false);
  return (Key)hi << 32 | lo;
}
__device__ inline Key key_lane(Key k, int lane) {
  return (Key)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(k >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, lane);
}
// The largest of a wave, in every lane.
__device__ inline Key wave_max(Key k) {
  k = max(k, key_dpp<0xB1>(k));     // quads
  k = max(k, key_dpp<0x4E>(k));
  k = max(k, key_dpp<0x141>(k));    // half rows, rows of 16
  k = max(k, key_dpp<0x140>(k));
  return max(max(key_lane(k, 0), key_lane(k, 16)), max(key_lane(k, 32), key_lane(k, 48)));
}
__device__ inline Key key_xor(Key k, int mask) {
  return (Key)(uint32_t)__shfl_xor((int)(uint32_t)(k >> 32), mask) << 32 |
         (uint32_t)__shfl_xor((int)(uint32_t)k, mask);
}
// The larger (or the smaller) of a lane's key and that of the lane `mask` away.
__device__ inline void exchange(Key& k, int mask, bool larger) {
  const Key o = key_xor(k, mask);
  if ((o > k) == larger) k = o;
}
// The 64 largest of a wave's sorted list (lane 0 first) and of 64 keys more.
__device__ inline void add64(Key& list, Key k, bool sorted) {
  const int lane = threadIdx.x & 63;
  if (!sorted) {
#pragma unroll
    for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
      for (int off = size >> 1; off >= 1; off >>= 1)
        exchange(k, off, ((lane & off) == 0) == ((lane & size) == 0));
  }
  list = max(list, key_xor(k, 63));
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) exchange(list, off, (lane & off) == 0);
}

template <int W> struct SelectLds { Key keys[W * 64], least[W], picked[kMostTop]; int count; };

// A workgroup's W waves take the n largest of `m` keys, in order, to lds.picked (0 behind
// them); get(i): key i. Each wave's k-th largest of its threads' maxima, k W >= n, leaves n
// keys at or above the least of them; keys above that are few, unless one wave has nothing
// but small ones, and each counts those before it. Neighbours belong to different waves, so
// that keys in order do not do that. Where there are too many, the waves keep sorted lists and
// join them (20 of a row's 2374 maxima, then of their groups: 15 us so, 8 by counting).
template <int W, typename F> struct Select {
  static constexpr int NT = W * 64, R = kPicked / NT;
  SelectLds<W>& lds;
  int n, m;
  F get;
  Key held[R];       // the first kPicked keys, R a thread; those behind them are taken again

  __device__ static int first() { return (threadIdx.x & 63) * W + (threadIdx.x >> 6); }
  __device__ Select(SelectLds<W>& l, int n, int m, F f) : lds(l), n(n), m(m), get(f) {
#pragma unroll
    for (int t = 0; t < R; ++t) held[t] = t * NT + first() < m ? get(t * NT + first()) : 0;
  }
  // f(key) for the thread's keys, all threads at once
  template <typename G> __device__ void each(G f) {
#pragma unroll
    for (int t = 0; t < R; ++t)
      if (t * NT < m) f(held[t]);
    for (int i0 = kPicked; i0 < m; i0 += NT) f(i0 + first() < m ? get(i0 + first()) : 0);
  }
  __device__ void run() {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Key best = 0;
    each([&](Key k) { best = max(best, k); });
    Key kth = 0;
    for (int k = 0; k < n; k += W) {
      kth = wave_max(best);
      if (best == kth) best = 0;
    }
    if (lane == 0) lds.least[wave] = kth;
    if (tid == 0) lds.count = 0;
    if (tid < kMostTop) lds.picked[tid] = 0;
    __syncthreads();
    Key least = lds.least[0];
#pragma unroll
    for (int w = 1; w < W; ++w) least = min(least, lds.least[w]);
    each([&](Key k) {
      const uint64_t in = __ballot(k != 0 && k >= least);
      if (in == 0) return;
      int at = 0;
      if (lane == 0) at = atomicAdd(&lds.count, __builtin_popcountll(in));
      at = __builtin_amdgcn_readfirstlane(at) + __builtin_popcountll(in & ((1ull << lane) - 1));
      if (in >> lane & 1 && at < NT) lds.keys[at] = k;
    });
    __syncthreads();
    const int count = lds.count;
    if (count <= NT) {
      if (tid < count) {
        const Key mine = lds.keys[tid];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < count; ++j) rank += lds.keys[j] > mine;
        if (rank < n) lds.picked[rank] = mine;
      }
      __syncthreads();
      return;
    }
    Key list = 0;
    each([&](Key k) {
      if (__any(k > key_lane(list, n - 1))) add64(list, k, false);
    });
    lds.keys[tid] = list;
#pragma unroll
    for (int w = W / 2; w >= 1; w >>= 1) {
      __syncthreads();
      if (wave < w) {
        add64(list, lds.keys[tid + w * 64], true);
        lds.keys[tid] = list;
      }
    }
    if (tid < n) lds.picked[tid] = list;
    __syncthreads();
  }
};
template <int W, typename F>
__device__ inline Select<W, F> select(SelectLds<W>& lds, int n, int m, F f) {
  return Select<W, F>(lds, n, m, f);
}

// The pieces of a row, and what is left of each row's answer, by W waves; W = 1: without the
// largest entries. With them: 8 waves (one row of 151936, 20 entries, both launches: 13.3 us;
// 16.7 with 16, 14.3 with 4), or 4 where there are many rows (1024 rows, the largest entry of
// each, this launch: 42 us with 16 and 14 with 4).
template <int W>
__global__ void __launch_bounds__(W * 64) logprobs_rows_kernel(LogprobsArgs a) {
  constexpr bool TOP = W > 1;
  const int b = blockIdx.y, i = blockIdx.x;
  if (a.n_rows && i >= a.n_rows[b]) return;
  const size_t row = (size_t)b * a.rows + i;
  __shared__ SelectLds<W> lds;
  __shared__ int groups[kMostTop];
  const uint32_t* maxima = a.maxima + row * a.groups;
  // on their way while the pieces are joined
  auto by_group = select(lds, a.top, TOP ? a.groups : 0, [&](int g) { return place_of(maxima[g], g); });
  const float* z = a.z + row * a.stride;
  const int lane = threadIdx.x & 63;
  const Piece* parts = a.parts + row * a.pieces;
  const int y = a.tokens[row];
  const bool given = y >= 0 && y < a.vocab;
  const float zy = given ? z[y] : -INFINITY;
  float m = -INFINITY;
  for (int p = lane; p < a.pieces; p += 64) m = fmaxf(m, parts[p].m);
  m = wave_max(m);
  const float base = m == -INFINITY ? 0.f : m;
  float rest = 0.f, ex = 0.f;
  int ones = 0, before = 0;
  for (int p = lane; p < a.pieces; p += 64) {
    const Piece q = parts[p];
    const float x = (q.m - base) * a.c, w = __builtin_amdgcn_exp2f(x);
    if (q.m == m) ones += q.ones;
    else rest += w * q.ones;
    rest += w * q.rest;
    ex += w * fmaf(q.rest + q.ones, fmaxf(x, kFar), q.ex);
    before += q.before;
  }
  rest = wave_sum(rest);
  ex = wave_sum(ex);
  ones = wave_sum(ones);
  before = wave_sum(before);
  if (m == INFINITY) rest = NAN;
  const bool empty = m == -INFINITY && rest == 0.f;       // every entry is -inf
  const float more = (float)(ones - 1) + rest, ls = log1pf(more);
  auto logp = [&](float v) {
    return empty || v == -INFINITY ? (rest == rest ? -INFINITY : rest) : (v - base) / a.temperature - ls;
  };
  if (threadIdx.x == 0) {
    a.logp[row] = given ? logp(zy) : rest == rest ? -INFINITY : rest;
    a.entropy[row] = empty ? 0.f : ls - ex / (more + 1.f) * 0.693147180559945309f;
    a.rank[row] = given ? before : a.vocab;
  }
  if constexpr (TOP) {
    by_group.run();
    const int n = min(a.top, a.groups);
    if (threadIdx.x < n) groups[threadIdx.x] = index_of(lds.picked[threadIdx.x]);
    __syncthreads();
    select(lds, a.top, n * kGroup, [&](int i) {
      const int v = groups[i / kGroup] * kGroup + i % kGroup;
      return v < a.vocab ? place_of(key_of(z[v]), v) : 0;
    }).run();
    if (threadIdx.x < a.top) {
      const int v = index_of(lds.picked[threadIdx.x]);
      a.top_tokens[row * a.top + threadIdx.x] = v;
      a.top_logp[row * a.top + threadIdx.x] = logp(z[v]);
    }
  }
}

// Entries of a piece: enough pieces to fill the GPU, or as many loads in flight.
int units_of(int64_t rows, int vocab) {
  return rows * ((vocab + 8191) / 8192) >= 512 ? 8 : 2;
}
int pieces_of(int64_t rows, int vocab) {
  const int n = 1024 * units_of(rows, vocab);
  return (vocab + n - 1) / n;
}

template <int U> void launch_pieces(const LogprobsArgs& a, int batch, hipStream_t st) {
  const dim3 grid(a.pieces, a.rows, batch);
  if (a.top)
    hipLaunchKernelGGL((logprobs_pieces_kernel<U, true>), grid, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((logprobs_pieces_kernel<U, false>), grid, dim3(kThreads), 0, st, a);
}

}  // namespace

size_t logprobs_workspace_bytes(int batch, int rows, int vocab, int top) {
  const int64_t n = (int64_t)batch * rows;
  return align_up(n * pieces_of(n, vocab) * sizeof(Piece)) +
         (top ? align_up(n * ((vocab + kGroup - 1) / kGroup) * 4) : 0);
}

hipError_t launch_logprobs(const float* logits, int64_t stride, const int32_t* tokens,
                           const int32_t* n_rows, int batch, int rows, int vocab,
                           float temperature, int top, float* logp, float* entropy, int32_t* rank,
                           int32_t* top_tokens, float* top_logp, void* ws, hipStream_t st) {
  const int64_t n = (int64_t)batch * rows;
  LogprobsArgs a{logits, (long)stride, tokens, n_rows, rows, vocab, pieces_of(n, vocab),
                 (vocab + kGroup - 1) / kGroup, top, temperature, kLog2e / temperature,
                 logp, entropy, rank, top_tokens, top_logp, static_cast<Piece*>(ws), nullptr};
  a.maxima = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(ws) +
                                         align_up(n * a.pieces * sizeof(Piece)));
  if (units_of(n, vocab) == 8) launch_pieces<8>(a, batch, st);
  else launch_pieces<2>(a, batch, st);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(rows, batch);
  if (top == 0)
    hipLaunchKernelGGL(logprobs_rows_kernel<1>, grid, dim3(64), 0, st, a);
  else if (n <= 512)
    hipLaunchKernelGGL(logprobs_rows_kernel<8>, grid, dim3(512), 0, st, a);
  else
    hipLaunchKernelGGL(logprobs_rows_kernel<4>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace ldr
