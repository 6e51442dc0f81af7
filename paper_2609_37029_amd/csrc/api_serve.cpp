// Host side of the operators on rows of probabilities and logits beside the drafting
// step: sizes, argument validation and launches. The kernels are in verify_probs.hip and
// logprobs.hip.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "serve_internal.h"

using namespace ldr;

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

extern "C" {

size_t ldr_verify_probs_workspace_bytes(int32_t batch, int32_t block, int32_t vocab) {
  if (batch <= 0 || batch > 65535 || block <= 0 || block > (1 << 30) || vocab <= 0 ||
      vocab > (1 << 30))
    return 0;
  return verify_probs_workspace_bytes(batch, block, vocab);
}

int ldr_verify_probs(const float* target_probs, const float* draft_probs,
                     const int32_t* draft_tokens, const int32_t* n_draft, const float* uniforms,
                     int32_t batch, int32_t block, int32_t vocab, int32_t* accepted,
                     int32_t* next_token, int32_t* n_new, void* workspace,
                     size_t workspace_bytes, void* stream) {
  if (!target_probs || !draft_tokens || !uniforms || !accepted || !next_token || !n_new ||
      !workspace)
    return LDR_EINVAL;
  const size_t need = ldr_verify_probs_workspace_bytes(batch, block, vocab);
  if (!need || workspace_bytes < need || !aligned(workspace, 16)) return LDR_EINVAL;
  // every workgroup of a sequence reads the inputs while one writes its counts, and the
  // second launch reads the first one's
  const size_t rows = (size_t)batch * block, all = rows + batch;
  const Range out[] = {{accepted, batch * 4ul}, {next_token, batch * 4ul}, {n_new, batch * 4ul},
                       {workspace, need}};
  const Range in[] = {{target_probs, all * vocab * 4}, {draft_probs, rows * vocab * 4},
                      {draft_tokens, rows * 4}, {n_draft, batch * 4ul}, {uniforms, all * 4}};
  for (const Range& o : out) {
    for (const Range& i : in)
      if (overlap(o, i)) return LDR_EINVAL;
    for (const Range& x : out)
      if (&x != &o && overlap(o, x)) return LDR_EINVAL;
  }
  return launch_verify_probs(target_probs, draft_probs, draft_tokens, n_draft, uniforms, batch,
                             block, vocab, accepted, next_token, n_new, workspace,
                             static_cast<hipStream_t>(stream)) == hipSuccess
             ? LDR_OK : LDR_EHIP;
}

size_t ldr_logprobs_workspace_bytes(int32_t batch, int32_t rows, int32_t vocab, int32_t top_n) {
  if (batch <= 0 || batch > 65535 || rows <= 0 || rows > 65535 || vocab <= 0 ||
      vocab > (1 << 30) || top_n < 0 || top_n > 64 || top_n > vocab)
    return 0;
  return logprobs_workspace_bytes(batch, rows, vocab, top_n);
}

int ldr_logprobs(const float* logits, int64_t row_stride, const int32_t* tokens,
                 const int32_t* n_rows, int32_t batch, int32_t rows, int32_t vocab,
                 float temperature, int32_t top_n, float* logp, float* entropy, int32_t* rank,
                 int32_t* top_tokens, float* top_logp, void* workspace, size_t workspace_bytes,
                 void* stream) {
  const size_t need = ldr_logprobs_workspace_bytes(batch, rows, vocab, top_n);
  if (!need || !logits || !tokens || !logp || !entropy || !rank || !workspace) return LDR_EINVAL;
  if (top_n && (!top_tokens || !top_logp)) return LDR_EINVAL;
  const size_t n = (size_t)batch * rows;
  if (row_stride < vocab || row_stride > (int64_t)1 << 40) return LDR_EINVAL;
  // the kernels' exponents are of base 2, of a factor that has all its digits
  if (!std::isnormal(temperature) || temperature < 0.f || !std::isnormal(kLog2e / temperature))
    return LDR_EINVAL;
  if (workspace_bytes < need || !aligned(workspace, kAlign) || !aligned(logits, 4) ||
      !aligned(tokens, 4) || !aligned(n_rows, 4) || !aligned(logp, 4) || !aligned(entropy, 4) ||
      !aligned(rank, 4) || !aligned(top_tokens, 4) || !aligned(top_logp, 4))
    return LDR_EINVAL;
  // the second launch reads the inputs again while it writes
  const size_t top = top_n ? n * top_n * 4 : 0;
  const Range out[] = {{logp, n * 4}, {entropy, n * 4}, {rank, n * 4}, {top_tokens, top},
                       {top_logp, top}, {workspace, need}};
  const Range in[] = {{logits, ((n - 1) * (size_t)row_stride + vocab) * 4}, {tokens, n * 4},
                      {n_rows, n_rows ? batch * 4ul : 0}};
  for (const Range& o : out) {
    for (const Range& i : in)
      if (overlap(o, i)) return LDR_EINVAL;
    for (const Range& x : out)
      if (&x != &o && overlap(o, x)) return LDR_EINVAL;
  }
  return launch_logprobs(logits, row_stride, tokens, n_rows, batch, rows, vocab, temperature,
                         top_n, logp, entropy, rank, top_tokens, top_logp, workspace,
                         static_cast<hipStream_t>(stream)) == hipSuccess ? LDR_OK : LDR_EHIP;
}

}  // extern "C"
