// Speculative verification from given probabilities and uniforms (Eq. 1-2).
//
// Two launches. The first has one workgroup per (part of the vocabulary,
// sequence): each takes the in-order acceptance test itself (block gathered
// pairs of probabilities), then sums its part of the target row where the round
// stops, and of the residual, in fp64. The second, one workgroup per sequence,
// finds the part in which the cumulative sum passes u C and the token inside it.
//
// fp64: differences of fp32 numbers and sums of 150 thousand of them lose nothing
// that a draw could see, so the token does not depend on how the sum is cut up.
// The test u q < p compares a 48-bit product exactly.
//
// Bound by reading one target and one draft row a sequence, once, and at small
// batches by the latency of the chain: gathers, rows, sums, second launch.
#include "ldr_internal.h"

namespace ldr {
namespace {

constexpr int kThreads = 256;
constexpr int kPart = 4096;            // tokens of a part
constexpr int kEach = kPart / kThreads;

struct Part { double res, tgt; };      // sums of [p - q]_+ and p over a part

struct ProbsArgs {
  const float* P;        // [batch][B + 1][V]
  const float* Q;        // [batch][B][V] or null
  const int32_t* y;      // [batch][B]
  const int32_t* n;      // [batch] or null
  const float* u;        // [batch][B + 1]
  int batch, B, V, parts;
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
  __shared__ int first;
  if (threadIdx.x == 0) first = a.B;
  __syncthreads();
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
      atomicMin(&first, i);
      break;
    }
  }
  __syncthreads();
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
__device__ inline double residual(const Row& w, double p, int v) {
  return positive(p - (w.q ? (double)w.q[v] : v == w.y ? 1.0 : 0.0));
}

__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

__global__ void __launch_bounds__(kThreads) probs_sum_kernel(ProbsArgs a) {
  const int b = blockIdx.y, v0 = blockIdx.x * kPart;
  const Stop s = find_stop(a, b);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.accepted[b] = s.r;
    a.n_new[b] = s.r + 1;
  }
  const Row w = row_of(a, b, s);
  double res = 0.0, tgt = 0.0;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int v = v0 + k * kThreads + threadIdx.x;
    if (v < a.V) {
      const double p = w.p[v];
      tgt += positive(p);
      if (s.rejected) res += residual(w, p, v);
    }
  }
  res = wave_sum(res);
  tgt = wave_sum(tgt);
  __shared__ Part red[kThreads / 64];
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = Part{res, tgt};
  __syncthreads();
  if (threadIdx.x == 0) {
    Part t{0.0, 0.0};
    for (int k = 0; k < kThreads / 64; ++k) { t.res += red[k].res; t.tgt += red[k].tgt; }
    a.part[(size_t)b * a.parts + blockIdx.x] = t;
  }
}

__global__ void __launch_bounds__(kThreads) probs_draw_kernel(ProbsArgs a) {
  __shared__ double sums[kThreads];
  __shared__ double before;
  __shared__ int part, found, last;
  const int b = blockIdx.x, tid = threadIdx.x;
  const int r = a.accepted[b];
  const int n = a.n ? min(max(a.n[b], 0), a.B) : a.B;
  const Stop s{r, r < n};
  const Row w = row_of(a, b, s);
  const Part* pt = a.part + (size_t)b * a.parts;
  if (tid == 0) {
    bool use = false;
    for (int c = 0; c < a.parts; ++c) use = use || pt[c].res > 0.0;
    double total = 0.0;
    for (int c = 0; c < a.parts; ++c) total += use ? pt[c].res : pt[c].tgt;
    const double t = (double)a.u[(size_t)b * (a.B + 1) + a.B] * total;
    double sum = 0.0;
    int at = -1, final = -1;
    double at_before = 0.0, final_before = 0.0;
    for (int c = 0; c < a.parts; ++c) {
      const double x = use ? pt[c].res : pt[c].tgt;
      if (x > 0.0) {
        if (at < 0 && sum + x > t) { at = c; at_before = sum; }
        final = c;
        final_before = sum;
      }
      sum += x;
    }
    part = at >= 0 ? at : final;
    before = at >= 0 ? at_before : final_before;
    sums[0] = t;
    found = a.V;
    last = use ? 1 : 0;
  }
  __syncthreads();
  const double t = sums[0];
  const bool use = last;
  const int c = part;
  __syncthreads();
  if (c < 0) {   // no entry above 0
    if (tid == 0) a.token[b] = 0;
    return;
  }
  // kEach consecutive tokens a thread
  const int v0 = c * kPart + tid * kEach;
  double x[kEach], sum = 0.0;
  int end = -1;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int v = v0 + k;
    const double p = v < a.V ? (double)w.p[v] : 0.0;
    x[k] = v < a.V ? (use ? residual(w, p, v) : positive(p)) : 0.0;
    if (x[k] > 0.0) end = v;
    sum += x[k];
  }
  sums[tid] = sum;
  if (tid == 0) last = -1;
  __syncthreads();
  double cum = before;
  for (int k = 0; k < tid; ++k) cum += sums[k];
  int hit = a.V;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    cum += x[k];
    if (hit == a.V && x[k] > 0.0 && cum > t) hit = v0 + k;
  }
  if (hit < a.V) atomicMin(&found, hit);
  if (end >= 0) atomicMax(&last, end);
  __syncthreads();
  if (tid == 0) a.token[b] = found < a.V ? found : last;
}

}  // namespace

size_t verify_probs_workspace_bytes(int batch, int B, int V) {
  return align_up((size_t)batch * ((V + kPart - 1) / kPart) * sizeof(Part));
}

hipError_t launch_verify_probs(const float* P, const float* Q, const int32_t* y,
                               const int32_t* n_draft, const float* u, int batch, int B, int V,
                               int32_t* accepted, int32_t* token, int32_t* n_new, void* ws,
                               hipStream_t st) {
  ProbsArgs a{P, Q, y, n_draft, u, batch, B, V, (V + kPart - 1) / kPart,
              static_cast<Part*>(ws), accepted, token, n_new};
  hipLaunchKernelGGL(probs_sum_kernel, dim3(a.parts, batch), dim3(kThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(probs_draw_kernel, dim3(batch), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace ldr
