// Drives the host side of the paged cache, its attention and the verification from
// probabilities without a device: configurations, layouts, workspace sizes, argument
// checks, and the error path of a handle that cannot be reset.
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
  void* odd = reinterpret_cast<void*>((uintptr_t(1) << 20) + 16);
  int32_t* n = static_cast<int32_t*>(fake);
  float* f = static_cast<float*>(fake);
  const ldr_pages_config good{5, 8, 128, 64, 2048, 16, 600, LDR_BF16};

  size_t off[4] = {};
  ldr_pages* h = nullptr;
  for (int field = 0; field < 8; ++field)
    for (int32_t bad : {INT32_MIN, -1, INT32_MAX}) {
      ldr_pages_config c = good;
      reinterpret_cast<int32_t*>(&c)[field] = bad;
      EXPECT(ldr_pages_pool_bytes(&c) == 0 && ldr_pages_state_bytes(&c) == 0);
      EXPECT(ldr_pages_layout(&c, off) == LDR_EINVAL);
      EXPECT(ldr_attend_workspace_bytes(&c, 32, 17) == 0);
      EXPECT(ldr_pages_init(&h, &c, fake, fake, nullptr) == LDR_EINVAL && !h);
    }
  EXPECT(ldr_pages_pool_bytes(nullptr) == 0 && ldr_pages_state_bytes(nullptr) == 0);
  EXPECT(ldr_pages_layout(nullptr, off) == LDR_EINVAL);
  EXPECT(ldr_pages_layout(&good, nullptr) == LDR_EINVAL);
  EXPECT(ldr_attend_workspace_bytes(nullptr, 32, 17) == 0);

  // the largest of each configuration: sizes in 64 bits, regions behind one another
  const ldr_pages_config large[] = {
      {1024, 63, 128, 256, 1 << 28, 1024, (1 << 22) - 1, LDR_F32},
      {1, 1, 64, 32, 1, 1024, (1 << 25) - 1, LDR_BF16},
      {63, 1024, 128, 256, 1, 1, 1, LDR_F32},
  };
  for (const ldr_pages_config& c : large) {
    EXPECT(ldr_pages_pool_bytes(&c) ==
           size_t(2) * c.n_layers * c.n_kv_heads * c.n_pages * c.page * c.head_dim *
               (c.dtype == LDR_BF16 ? 2 : 4));
    EXPECT(ldr_pages_layout(&c, off) == LDR_OK);
    EXPECT(off[0] < off[1] && off[1] < off[2] && off[2] < off[3]);
    EXPECT(off[3] - off[2] >= size_t(c.batch) * c.max_pages * 4);
    EXPECT(ldr_pages_state_bytes(&c) >= off[3] + size_t(c.n_pages) * 4);
    EXPECT(ldr_attend_workspace_bytes(&c, c.n_kv_heads, 1) > 0);
  }
  for (int32_t hq : {INT32_MIN, -8, 0, 31, INT32_MAX})
    EXPECT(ldr_attend_workspace_bytes(&good, hq, 17) == 0);
  for (int32_t rows : {INT32_MIN, -1, 0, 1 << 18, INT32_MAX})
    EXPECT(ldr_attend_workspace_bytes(&good, 32, rows) == 0);
  EXPECT(ldr_attend_workspace_bytes(&good, 32, (1 << 18) - 1) > 0);

  EXPECT(ldr_pages_init(nullptr, &good, fake, fake, nullptr) == LDR_EINVAL);
  EXPECT(ldr_pages_init(&h, &good, nullptr, fake, nullptr) == LDR_EINVAL && !h);
  EXPECT(ldr_pages_init(&h, &good, fake, nullptr, nullptr) == LDR_EINVAL && !h);
  EXPECT(ldr_pages_init(&h, &good, odd, fake, nullptr) == LDR_EINVAL && !h);
  EXPECT(ldr_pages_init(&h, &good, fake, odd, nullptr) == LDR_EINVAL && !h);
  // no device: the reset does not start, and the handle is not kept
  for (int i = 0; i < 3; ++i)
    EXPECT(ldr_pages_init(&h, &good, fake, fake, nullptr) == LDR_EHIP && !h);

  EXPECT(ldr_pages_reserve(nullptr, n, 17, nullptr) == LDR_EINVAL);
  EXPECT(ldr_pages_write(nullptr, 0, 5, fake, fake, 17, nullptr) == LDR_EINVAL);
  EXPECT(ldr_pages_keep(nullptr, n, nullptr) == LDR_EINVAL);
  EXPECT(ldr_pages_fork(nullptr, n, nullptr) == LDR_EINVAL);
  EXPECT(ldr_pages_compact(nullptr, nullptr) == LDR_EINVAL);
  EXPECT(ldr_pages_status(nullptr, 1, nullptr) == LDR_EINVAL);
  EXPECT(ldr_attend_plan(nullptr, 32, 17, nullptr, fake, 1 << 30, nullptr) == LDR_EINVAL);
  EXPECT(ldr_attend(nullptr, 0, fake, 4096, 32, 17, 1.f, fake, f, fake, 1 << 30, nullptr) ==
         LDR_EINVAL);
  EXPECT(ldr_views_fork(nullptr, n, nullptr) == LDR_EINVAL);
  ldr_pages_destroy(nullptr);

  // the verification: regions of one allocation's addresses, apart or over one another
  const int32_t batch = 3, block = 4, vocab = 1000;
  const size_t need = ldr_verify_probs_workspace_bytes(batch, block, vocab);
  EXPECT(need > 0 && ldr_verify_probs_workspace_bytes(65535, 1 << 30, 1 << 30) > 0);
  EXPECT(ldr_verify_probs_workspace_bytes(65536, 1, 1) == 0);
  EXPECT(ldr_verify_probs_workspace_bytes(1, INT32_MAX, 1) == 0);
  EXPECT(ldr_verify_probs_workspace_bytes(1, 1, INT32_MIN) == 0);
  auto at = [](int i) { return reinterpret_cast<void*>(uintptr_t(1 + i) << 20); };
  auto verify = [&](void* accepted, void* n_draft, void* draft, size_t bytes) {
    return ldr_verify_probs(static_cast<float*>(at(0)), static_cast<float*>(draft),
                            static_cast<int32_t*>(at(2)), static_cast<int32_t*>(n_draft),
                            static_cast<float*>(at(4)), batch, block, vocab,
                            static_cast<int32_t*>(accepted), static_cast<int32_t*>(at(6)),
                            static_cast<int32_t*>(at(7)), at(8), bytes, nullptr);
  };
  EXPECT(verify(at(5), at(3), at(1), need - 1) == LDR_EINVAL);
  EXPECT(verify(at(3), at(3), at(1), need) == LDR_EINVAL);
  EXPECT(verify(at(6), at(3), at(1), need) == LDR_EINVAL);
  EXPECT(verify(at(5), nullptr, at(5), need) == LDR_EINVAL);
  EXPECT(verify(at(5), at(3), at(1), need) == LDR_EHIP);       // no device
  EXPECT(verify(at(5), nullptr, nullptr, need) == LDR_EHIP);
  std::puts("pages checks ok");
  return 0;
}
