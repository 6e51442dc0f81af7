// Drives the host side of coded caches, reads and log probabilities without a device:
// configurations, sizes and argument checks.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "ldr.h"

#define EXPECT(c)                                                  \
  do {                                                             \
    if (!(c)) {                                                    \
      std::fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #c); \
      std::exit(1);                                                \
    }                                                              \
  } while (0)

int main() {
  // aligned, never dereferenced: a call is refused first, or finds no device
  void* fake = reinterpret_cast<void*>(uintptr_t(1) << 20);
  int32_t* n = static_cast<int32_t*>(fake);
  const ldr_pages_config good{5, 8, 128, 64, 2048, 16, 600, LDR_MXFP4};
  for (int32_t dtype : {INT32_MIN, -1, 2, 3, 5, 6, 7, 9, INT32_MAX}) {
    ldr_pages_config c = good;
    c.dtype = dtype;
    EXPECT(ldr_pages_pool_bytes(&c) == 0 && ldr_attend_workspace_bytes(&c, 32, 17) == 0);
  }
  // the largest of each configuration: sizes in 64 bits
  for (int32_t dtype : {LDR_MXFP4, LDR_MXFP8})
    for (const ldr_pages_config& c :
         {ldr_pages_config{1024, 63, 128, 256, 1 << 28, 1024, (1 << 22) - 1, dtype},
          ldr_pages_config{1, 1, 64, 32, 1, 1024, (1 << 25) - 1, dtype},
          ldr_pages_config{63, 1024, 128, 256, 1, 1, 1, dtype}}) {
      EXPECT(ldr_pages_pool_bytes(&c) == size_t(2) * c.n_layers * c.n_kv_heads * c.n_pages * c.page *
                                             (c.head_dim * dtype / 8 + c.head_dim / 32));
      size_t off[4] = {};
      EXPECT(ldr_pages_layout(&c, off) == LDR_OK && ldr_pages_state_bytes(&c) > off[3]);
      EXPECT(ldr_attend_workspace_bytes(&c, c.n_kv_heads, 1) > 0);
      EXPECT(ldr_attend_workspace_bytes(&c, c.n_kv_heads, (1 << 27) / c.n_kv_heads) == 0);
    }
  ldr_pages* h = nullptr;
  EXPECT(ldr_pages_init(&h, &good, fake, fake, nullptr) != LDR_OK && !h);   // no device
  EXPECT(ldr_pages_read(nullptr, 0, 1, n, n, fake, fake, 17, nullptr) == LDR_EINVAL);

  EXPECT(ldr_logprobs_workspace_bytes(1, 1, 1, 0) > 0);
  EXPECT(ldr_logprobs_workspace_bytes(65535, 65535, 1 << 30, 64) >
         size_t(65535) * 65535 * (1 << 30) / 64 * 4);
  for (int32_t bad : {INT32_MIN, -1, 0, INT32_MAX}) {
    EXPECT(ldr_logprobs_workspace_bytes(bad, 2, 64, 3) == 0);
    EXPECT(ldr_logprobs_workspace_bytes(2, bad, 64, 3) == 0);
    EXPECT(ldr_logprobs_workspace_bytes(2, 2, bad, 3) == 0);
    if (bad) EXPECT(ldr_logprobs_workspace_bytes(2, 2, 64, bad) == 0);
  }
  EXPECT(ldr_logprobs_workspace_bytes(2, 2, 63, 64) == 0);
  auto at = [](int i) { return reinterpret_cast<void*>((uintptr_t(1) << 24) + (uintptr_t(i) << 16)); };
  auto f = [&](int i) { return static_cast<float*>(at(i)); };
  auto w = [&](int i) { return static_cast<int32_t*>(at(i)); };
  const size_t ws = ldr_logprobs_workspace_bytes(2, 2, 64, 3);
  for (float t : {0.f, -1.f, NAN, INFINITY, 1e-40f})
    EXPECT(ldr_logprobs(f(0), 64, w(1), nullptr, 2, 2, 64, t, 3, f(2), f(3), w(4), w(5), f(6), at(7),
                        ws, nullptr) == LDR_EINVAL);
  for (int64_t stride : {INT64_MIN, int64_t(0), int64_t(63), INT64_MAX})
    EXPECT(ldr_logprobs(f(0), stride, w(1), nullptr, 2, 2, 64, 1.f, 3, f(2), f(3), w(4), w(5), f(6),
                        at(7), ws, nullptr) == LDR_EINVAL);
  EXPECT(ldr_logprobs(f(0), 64, w(1), nullptr, 2, 2, 64, 1.f, 3, f(2), f(2), w(4), w(5), f(6), at(7),
                      ws, nullptr) == LDR_EINVAL);
  // top_n = 0 needs no outputs for them; without a device the launch fails
  EXPECT(ldr_logprobs(f(0), 64, w(1), nullptr, 2, 2, 64, 1.f, 0, f(2), f(3), w(4), nullptr, nullptr,
                      at(7), ws, nullptr) == LDR_EHIP);
  std::puts("mx checks ok");
  return 0;
}
