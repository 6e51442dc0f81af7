// Internal declarations of the operators beside the drafting step: the paged cache, the
// attention over it, verification from given probabilities, log probabilities. Apart from
// the step's, so that a change here is none of the step's sources.
#pragma once

#include "ldr_internal.h"

namespace ldr {

// Memory of a call, and whether two have a byte in common.
struct Range { const void* p; size_t bytes; };   // p null: none
inline bool overlap(const Range& a, const Range& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
}

// Paged K/V cache (pages.hip). The state is int32 words: a header, rows, open,
// table, refs, then scratch of the calls (lists of pages).
struct PagesShape {
  int layers, hkv, d, page, n_pages, batch, max_pages, dtype;
  int bits;                          // of a code; 0: rows of the dtype
  size_t el;                         // bytes of an element of the rows outside the pool
  size_t head_bytes;                 // one head's rows in a page of one layer's K (or V)
  size_t page_bytes;                 // all heads' of them
  size_t rows, open, table, refs;    // word offsets in the state
  size_t list;                       // scratch: n_pages words (free pages; compaction map)
  size_t pairs;                      // scratch: 2 max(batch, n_pages / 2 + 1) words (from, to)
  size_t words;
};
constexpr int kMxBlock = 32;      // dimensions that share a scale in a coded cache
// Header words of the state.
constexpr int kPagesFlags = 0;    // sticky flags
constexpr int kPagesVersion = 1;  // counts the calls that change the tables, resets too
constexpr int kPagesPairs = 2;    // pairs in the scratch list (compaction)
constexpr int kPagesHeader = 64;
constexpr int kFlagPages = 4;     // no room in the pool or a table
constexpr int kFlagPlan = 8;      // an attention ran on a plan of another state or handle
constexpr int kMaxSeqs = 1024;    // sequences of a cache: one thread each in the bookkeeping
// id: the handle's number, no other handle's of the process
struct PagesPtrs { uint8_t* pool; int32_t* state; int32_t id; };
hipError_t launch_pages_reset(const PagesShape& s, const PagesPtrs& p, hipStream_t st);
hipError_t launch_pages_reserve(const PagesShape& s, const PagesPtrs& p, const int32_t* n_new,
                                int max_new, hipStream_t st);
hipError_t launch_pages_write(const PagesShape& s, const PagesPtrs& p, int layer, int n_layers,
                              const void* K, const void* V, int max_new, hipStream_t st);
hipError_t launch_pages_write_mx(const PagesShape& s, const PagesPtrs& p, int layer, int n_layers,
                                 const void* K, const void* V, int max_new, hipStream_t st);
hipError_t launch_pages_read(const PagesShape& s, const PagesPtrs& p, int layer, int n_layers,
                             const int32_t* first, const int32_t* n, void* K, void* V,
                             int max_rows, hipStream_t st);
hipError_t launch_pages_keep(const PagesShape& s, const PagesPtrs& p, const int32_t* kept,
                             hipStream_t st);
hipError_t launch_pages_fork(const PagesShape& s, const PagesPtrs& p, const int32_t* src,
                             hipStream_t st);
hipError_t launch_pages_compact(const PagesShape& s, const PagesPtrs& p, hipStream_t st);
hipError_t launch_pages_clear_flags(const PagesPtrs& p, hipStream_t st);

// Attention over the paged cache (attend.hip); exponents are of base 2.
constexpr float kLog2e = 1.44269504088896341f;
size_t attend_workspace_bytes(const PagesShape& s, int hq, int max_new);
hipError_t launch_attend_plan(const PagesShape& s, const PagesPtrs& p, int hq, int max_new,
                              const int32_t* groups, void* ws, hipStream_t st);
hipError_t launch_attend(const PagesShape& s, const PagesPtrs& p, int layer, const void* q,
                         long q_stride, int hq, int max_new, float scale, void* o, float* lse,
                         void* ws, hipStream_t st);
// over coded rows (attend_mx.hip)
hipError_t launch_attend_mx(const PagesShape& s, const PagesPtrs& p, int layer, const void* q,
                            long q_stride, int hq, int max_new, float scale, void* o, float* lse,
                            void* ws, hipStream_t st);

// Verification from given probabilities and uniforms (verify_probs.hip).
size_t verify_probs_workspace_bytes(int batch, int B, int V);
hipError_t launch_verify_probs(const float* P, const float* Q, const int32_t* y,
                               const int32_t* n_draft, const float* u, int batch, int B, int V,
                               int32_t* accepted, int32_t* token, int32_t* n_new, void* ws,
                               hipStream_t st);

// Log probabilities of given tokens (logprobs.hip).
size_t logprobs_workspace_bytes(int batch, int rows, int vocab, int top);
hipError_t launch_logprobs(const float* logits, int64_t stride, const int32_t* tokens,
                           const int32_t* n_rows, int batch, int rows, int vocab,
                           float temperature, int top, float* logp, float* entropy, int32_t* rank,
                           int32_t* top_tokens, float* top_logp, void* ws, hipStream_t st);

}  // namespace ldr
