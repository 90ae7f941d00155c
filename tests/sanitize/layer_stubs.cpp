// Host-only stand-ins for the launchers of the gated-delta layer's kernels (see
// launch_stubs.cpp): a stub that is reached fails the run.
#include <cstdio>
#include <cstdlib>

#include "layer_kernels.h"

namespace {
hipError_t reached(const char* fn) {
  std::fprintf(stderr, "launcher %s reached in a host-only build\n", fn);
  std::abort();
}
}  // namespace

namespace precog {
hipError_t launch_delta(const DeltaParams&, int, int, int, int, hipStream_t) { return reached("delta"); }
hipError_t launch_delta_step(const DeltaParams&, int, int, int, int, hipStream_t) {
  return reached("delta_step");
}
hipError_t launch_conv(const ConvParams&, int, int, int, hipStream_t) { return reached("conv"); }
hipError_t launch_conv_step(const ConvParams&, int, int, hipStream_t) { return reached("conv_step"); }
hipError_t launch_score(const ScoreParams&, int, hipStream_t) { return reached("score"); }
}  // namespace precog
