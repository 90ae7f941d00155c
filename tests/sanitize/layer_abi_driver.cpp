// Drives the host code of the gated-delta layer's entry points
// (csrc/layer_abi.cpp) for a build with AddressSanitizer and
// UndefinedBehaviorSanitizer: every refusal, every call with nothing to do, and
// descriptors of extreme numbers, where a sum or product of sizes could
// overflow.  No call gets as far as a launch.  Test infrastructure only.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <limits>
#include <vector>

#include "precog.h"

static int failures = 0;
#define CHECK(c)                                                            \
  do {                                                                      \
    if (!(c)) {                                                             \
      std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c);  \
      ++failures;                                                           \
    }                                                                       \
  } while (0)

static void* at(uintptr_t v) { return reinterpret_cast<void*>(v); }

// A call that gets past its argument checks ends at the device check: there is
// no GPU in this build's runs, or it is not asked (see the stubs).
static bool refused(precog_status s) { return s != PRECOG_OK; }

int main() {
  const int64_t big = std::numeric_limits<int64_t>::max(), low = std::numeric_limits<int64_t>::min();
  const std::vector<int64_t> odd = {low, -1, 0, 1, 7, 8, 128, 136, 65535, 65536, 1LL << 24, 1LL << 31, 1LL << 40, big};
  float* f = static_cast<float*>(at(0x10004));
  precog_delta_desc good{};
  good.batch = 2;
  good.seqlen = 16;
  good.k_heads = 2;
  good.v_heads = 4;
  good.k_dim = good.v_dim = 64;
  good.in_dtype = PRECOG_BF16;
  good.out_dtype = good.state_dtype = PRECOG_F32;
  int64_t precog_delta_desc::*const sizes[] = {
      &precog_delta_desc::batch,    &precog_delta_desc::seqlen,   &precog_delta_desc::k_heads,
      &precog_delta_desc::v_heads,  &precog_delta_desc::k_dim,    &precog_delta_desc::v_dim,
      &precog_delta_desc::q_stride, &precog_delta_desc::k_stride, &precog_delta_desc::v_stride,
      &precog_delta_desc::h0_batch_stride, &precog_delta_desc::hT_batch_stride};
  // q is misaligned, so that no call that the descriptor allows gets further
  void* q = at(0x10008);
  for (auto a : sizes)
    for (auto b : sizes)
      for (int64_t x : odd)
        for (int64_t y : odd) {
          precog_delta_desc d = good;
          d.*a = x;
          d.*b = y;
          const precog_status s = precog_delta_encode(&d, q, at(0x20000), at(0x30000), f, f, nullptr, at(0x40000),
                                                      x, nullptr, at(0x50000), at(0x60000), nullptr, 0, nullptr);
          precog_delta_workspace_bytes(&d, static_cast<int>(x & 1));
          CHECK(refused(s) || d.batch == 0);
          const precog_status t = precog_delta_step(&d, q, at(0x20000), at(0x30000), f, f, at(0x40000), 4,
                                                    static_cast<int32_t*>(at(0x1000)), at(0x50000), nullptr);
          CHECK(refused(t) || d.batch == 0);
        }
  // overlaps of the states, up to the end of the address space
  for (uintptr_t h0 : {uintptr_t{0x100000}, ~uintptr_t{0xfffff}})
    for (uintptr_t hT : {uintptr_t{0x100010}, ~uintptr_t{0xfffef}, uintptr_t{0x110000}})
      precog_delta_encode(&good, q, at(0x20000), at(0x30000), f, f, nullptr, at(h0), 2, nullptr, at(0x50000), at(hT),
                          nullptr, 0, nullptr);
  CHECK(precog_delta_encode(nullptr, q, q, q, f, f, nullptr, q, 0, nullptr, q, q, nullptr, 0, nullptr) == PRECOG_ERR_NULL);
  for (float v : {-1.f, std::nanf(""), INFINITY}) {
    precog_delta_desc d = good;
    d.eps = v;
    CHECK(refused(precog_delta_encode(&d, q, q, q, f, f, nullptr, q, 0, nullptr, q, q, nullptr, 0, nullptr)));
  }

  precog_conv_desc conv{2, 16, 64, 4, 0, PRECOG_BF16, PRECOG_F32, 1};
  int64_t precog_conv_desc::*const conv_sizes[] = {&precog_conv_desc::batch, &precog_conv_desc::seqlen,
                                                   &precog_conv_desc::dim, &precog_conv_desc::width,
                                                   &precog_conv_desc::x_stride};
  for (auto a : conv_sizes)
    for (auto b : conv_sizes)
      for (int64_t x : odd)
        for (int64_t y : odd) {
          precog_conv_desc d = conv;
          d.*a = x;
          d.*b = y;
          const precog_status s = precog_conv_encode(&d, q, f, f, nullptr, at(0x40000), x, nullptr, at(0x50000),
                                                     at(0x60000), nullptr);
          CHECK(refused(s) || d.batch == 0 || d.dim == 0);
          const precog_status t = precog_conv_step(&d, q, f, f, at(0x40000), 4, static_cast<int32_t*>(at(0x1000)),
                                                   at(0x50000), nullptr);
          CHECK(refused(t) || d.batch == 0 || d.dim == 0);
        }
  for (int64_t T : odd)
    for (int64_t V : odd)
      for (int64_t top : odd) {
        precog_score_workspace_bytes(T, V, top);
        const precog_status s = precog_score_tokens(at(0x10001), PRECOG_BF16, T, V, 0, nullptr, top, f, f,
                                                    static_cast<int32_t*>(at(0x1000)), f, nullptr, 0, nullptr);
        CHECK(refused(s) || T == 0);
      }
  if (failures) return 1;
  std::puts("all checks passed");
  return 0;
}
