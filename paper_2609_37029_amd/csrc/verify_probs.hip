// Speculative verification from given probabilities and uniforms (Eq. 1-2).
//
// Two launches. The first has one workgroup per (run of parts of 1024 tokens, a
// wave a part; sequence): each takes the in-order acceptance test itself (block gathered pairs
// of probabilities), then sums its parts of the target row where the round stops,
// and of the residual, in fp64. The second, one workgroup per sequence, finds the
// part in which the cumulative sum passes u C and the token inside it.
//
// fp64: differences of fp32 numbers and sums of 150 thousand of them lose nothing
// that a draw could see: how the sum is cut up matters within their rounding of a border only.
// The test u q < p compares a 48-bit product exactly.
//
// Bound by reading one target and one draft row a sequence, once, and at small
// batches by the latency of the chain: tokens, gathers, rows, sums, second launch,
// part. 64 sequences of 151936 tokens: sums 18 us (78 MB, 4.3 TB/s), draw 4 us; one: 6
// and 4. With a workgroup a part of 4096, and without the next part's loads under way,
// 64 took 56 and 41 us.
#include "ldr_internal.h"

namespace ldr {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kPart = 1024;            // tokens of a part
constexpr int kEach = kPart / kThreads;    // tokens of a part a thread draws from
constexpr int kLane = kPart / 64;          // and a lane sums

struct Part { double res, tgt; };      // sums of [p - q]_+ and p over a part

struct ProbsArgs {
  const float* P;        // [batch][B + 1][V]
  const float* Q;        // [batch][B][V] or null
  const int32_t* y;      // [batch][B]
  const int32_t* n;      // [batch] or null
  const float* u;        // [batch][B + 1]
  int batch, B, V, parts;
  int run;               // parts of a wave of the first launch
  Part* part;            // [batch][parts]
  int32_t* accepted; int32_t* token; int32_t* n_new;
};

__device__ inline double positive(double w) {
  return w > 0.0 && w < (double)INFINITY ? w : 0.0;
}

// What a round stopped on: its accepted candidates, and whether a rejection
// ended it.
struct Stop { int r; bool rejected; };

__device__ Stop find_stop(const ProbsArgs& a, int b) {
  __shared__ int firsts[kWaves];
  int first = a.B;
  const int n = a.n ? min(max(a.n[b], 0), a.B) : a.B;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int y = a.y[(size_t)b * a.B + i];
    bool ok = y >= 0 && y < a.V;
    if (ok) {
      const float p = a.P[((size_t)b * (a.B + 1) + i) * a.V + y];
      const float q = a.Q ? a.Q[((size_t)b * a.B + i) * a.V + y] : 1.f;
      ok = (double)a.u[(size_t)b * (a.B + 1) + i] * (double)q < (double)p;
    }
    if (!ok) {
      first = i;
      break;
    }
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) first = min(first, __shfl_xor(first, off));
  if ((threadIdx.x & 63) == 0) firsts[threadIdx.x >> 6] = first;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWaves; ++k) first = min(first, firsts[k]);
  const int r = min(first, n);
  return Stop{r, r < n};
}

struct Row {
  const float* p; const float* q;   // q null: none, or 1 at y
  int y;
};
__device__ inline Row row_of(const ProbsArgs& a, int b, const Stop& s) {
  Row w{a.P + ((size_t)b * (a.B + 1) + s.r) * a.V, nullptr, -1};
  if (s.rejected) {
    if (a.Q) w.q = a.Q + ((size_t)b * a.B + s.r) * a.V;
    else w.y = a.y[(size_t)b * a.B + s.r];
  }
  return w;
}
// w_v of the residual from p and q at v, and of p alone.
__device__ inline double residual(const Row& w, float p, float q, int v) {
  return positive((double)p - (w.q ? (double)q : v == w.y ? 1.0 : 0.0));
}

__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}
// The sum over the threads up to this one, and over all.
__device__ inline double block_scan(double v, double* sums, double* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double inc = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double o = __shfl_up(inc, off);
    if (lane >= off) inc += o;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = inc;
  __syncthreads();
  double before = 0.0, all = 0.0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    before += k < wave ? sums[k] : 0.0;
    all += sums[k];
  }
  *total = all;
  return before + inc;
}

// A place that a thread found (-1: none), with what came before it.
struct Found { int at; double before; };
// The first of the threads that found one, or the last. By ballots: minima and maxima in
// LDS, lane by lane, took 8 of the 11 us of the draw.
template <bool LAST> __device__ inline Found pick(Found f, Found* found) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t have = __ballot(f.at >= 0);
  if (have ? lane == (LAST ? 63 - __builtin_clzll(have) : __builtin_ctzll(have)) : lane == 0)
    found[wave] = f;
  __syncthreads();
  Found r = found[LAST ? kWaves - 1 : 0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) {
    const Found o = found[LAST ? kWaves - 1 - i : i];
    if (r.at < 0) r = o;
  }
  return r;
}

// VEC: rows start on 16 bytes and V is a multiple of 4.
template <bool VEC>
__global__ void __launch_bounds__(kThreads) probs_sum_kernel(ProbsArgs a) {
  const int b = blockIdx.y, lane = threadIdx.x & 63;
  const Stop s = find_stop(a, b);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.accepted[b] = s.r;
    a.n_new[b] = s.r + 1;
  }
  const Row w = row_of(a, b, s);
  const int first = (blockIdx.x * kWaves + (threadIdx.x >> 6)) * a.run;
  const int last = min(first + a.run, a.parts);
  constexpr int W = VEC ? 4 : 1;
  struct Chunk { float p[kLane], q[kLane]; };
  auto load = [&](Chunk& x, int c) {
#pragma unroll
    for (int k = 0; k < kLane; k += W) {
      const int v = c * kPart + lane * W + k * 64;
      const bool in = v < a.V;
      if constexpr (VEC) {
        const float4 z{0.f, 0.f, 0.f, 0.f};
        *reinterpret_cast<float4*>(x.p + k) = in ? *reinterpret_cast<const float4*>(w.p + v) : z;
        *reinterpret_cast<float4*>(x.q + k) =
            in && w.q ? *reinterpret_cast<const float4*>(w.q + v) : z;
      } else {
        x.p[k] = in ? w.p[v] : 0.f;
        x.q[k] = in && w.q ? w.q[v] : 0.f;
      }
    }
  };
  auto add = [&](const Chunk& x, int c) {
    double res = 0.0, tgt = 0.0;
#pragma unroll
    for (int k = 0; k < kLane; ++k) {
      tgt += positive(x.p[k]);
      if (s.rejected)
        res += residual(w, x.p[k], x.q[k], c * kPart + lane * W + k / W * W * 64 + k % W);
    }
    res = wave_sum(res);
    tgt = wave_sum(tgt);
    if (lane == 0) a.part[(size_t)b * a.parts + c] = Part{res, tgt};
  };
  if (first >= last) return;
  Chunk x, y;                      // the next part on its way while one is added up
  load(x, first);
  for (int c = first; c < last; c += 2) {
    if (c + 1 < last) load(y, c + 1);
    add(x, c);
    if (c + 1 >= last) break;
    if (c + 2 < last) load(x, c + 2);
    add(y, c + 1);
  }
}

template <bool VEC>
__global__ void __launch_bounds__(kThreads) probs_draw_kernel(ProbsArgs a) {
  __shared__ double sums[kWaves];
  __shared__ Found hits[kWaves], lasts[kWaves], hit_tokens[kWaves], last_tokens[kWaves];
  const int b = blockIdx.x, tid = threadIdx.x;
  const int r = a.accepted[b];
  const int n = a.n ? min(max(a.n[b], 0), a.B) : a.B;
  const double u = a.u[(size_t)b * (a.B + 1) + a.B];
  const Stop s{r, r < n};
  const Row w = row_of(a, b, s);
  const Part* pt = a.part + (size_t)b * a.parts;
  // a run of consecutive parts a thread
  const int each = (a.parts + kThreads - 1) / kThreads;
  const int c0 = min(tid * each, a.parts), c1 = min(c0 + each, a.parts);
  double res = 0.0, tgt = 0.0;
  for (int c = c0; c < c1; ++c) { res += pt[c].res; tgt += pt[c].tgt; }
  const bool use = __syncthreads_or(res > 0.0);
  double total = 0.0;
  double cum = block_scan(use ? res : tgt, sums, &total) - (use ? res : tgt);
  const double t = u * total;
  Found at{-1, 0.0}, final{-1, 0.0};
  for (int c = c0; c < c1; ++c) {
    const double x = use ? pt[c].res : pt[c].tgt;
    if (x > 0.0) {
      if (at.at < 0 && cum + x > t) at = Found{c, cum};
      final = Found{c, cum};
    }
    cum += x;
  }
  const Found hit_part = pick<false>(at, hits), last_part = pick<true>(final, lasts);
  const Found in = hit_part.at >= 0 ? hit_part : last_part;
  const int c = in.at;
  if (c < 0) {   // no entry above 0
    if (tid == 0) a.token[b] = 0;
    return;
  }
  // kEach consecutive tokens a thread
  const int v0 = c * kPart + tid * kEach;
  static_assert(kEach == 4, "16 bytes");
  float p[kEach] = {}, q[kEach] = {};
  if constexpr (VEC) {
    if (v0 < a.V) {
      *reinterpret_cast<float4*>(p) = *reinterpret_cast<const float4*>(w.p + v0);
      if (w.q) *reinterpret_cast<float4*>(q) = *reinterpret_cast<const float4*>(w.q + v0);
    }
  } else {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (v0 + k < a.V) {
        p[k] = w.p[v0 + k];
        if (w.q) q[k] = w.q[v0 + k];
      }
    }
  }
  double x[kEach], sum = 0.0;
  Found end{-1, 0.0}, hit{-1, 0.0};
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    x[k] = use ? residual(w, p[k], q[k], v0 + k) : positive(p[k]);   // 0 behind the row
    if (x[k] > 0.0) end.at = v0 + k;
    sum += x[k];
  }
  double all = 0.0;
  double run = in.before + block_scan(sum, sums, &all) - sum;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    run += x[k];
    if (hit.at < 0 && x[k] > 0.0 && run > t) hit.at = v0 + k;
  }
  hit = pick<false>(hit, hit_tokens);
  end = pick<true>(end, last_tokens);
  if (tid == 0) a.token[b] = hit.at >= 0 ? hit.at : end.at;
}

}  // namespace

size_t verify_probs_workspace_bytes(int batch, int B, int V) {
  return align_up((size_t)batch * ((V + kPart - 1) / kPart) * sizeof(Part));
}

hipError_t launch_verify_probs(const float* P, const float* Q, const int32_t* y,
                               const int32_t* n_draft, const float* u, int batch, int B, int V,
                               int32_t* accepted, int32_t* token, int32_t* n_new, void* ws,
                               hipStream_t st) {
  const int parts = (V + kPart - 1) / kPart;
  // A wave's parts: its workgroup tests the candidates first, and its next part's
  // loads need one before them; but 4096 waves, 4 a SIMD, come first. 64 sequences of
  // 151936 tokens, both launches: 24.4 us with 1 part a wave, 23.5 with 2, 24.9 with 3, 26.2
  // with 4, 30.0 with 8.
  const int run = max(1, min(8, (int)((long)parts * batch / 4096)));
  ProbsArgs a{P, Q, y, n_draft, u, batch, B, V, parts, run, static_cast<Part*>(ws), accepted, token,
              n_new};
  const bool vec = V % 4 == 0 && reinterpret_cast<uintptr_t>(P) % 16 == 0 &&
                   reinterpret_cast<uintptr_t>(Q) % 16 == 0;
  const int wg = run * kWaves;    // parts of a workgroup
  const dim3 grid((parts + wg - 1) / wg, batch);
  if (vec) hipLaunchKernelGGL(probs_sum_kernel<true>, grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(probs_sum_kernel<false>, grid, dim3(kThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (vec) hipLaunchKernelGGL(probs_draw_kernel<true>, dim3(batch), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(probs_draw_kernel<false>, dim3(batch), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace ldr
