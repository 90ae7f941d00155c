// The short causal depthwise convolution: every lane owns eight channels and
// slides the last W - 1 inputs of them over a run of tokens in registers, so
// each input is read once (and the W - 1 before a run once more).  Memory
// bounds it: W multiply-adds and one exponential an element.  The four waves of
// a workgroup take neighbouring channels of the same tokens, 4 KB of a bf16 row
// (48 packed documents of 4,096 channels: 305 us with four runs of tokens side
// by side, 270 us so with streamed stores), and four of them share a SIMD: with
// four tokens on their way in each, instead of eight, nothing spills at 128
// registers (262 us, 4.2 TB/s).
#include "layer_ops.h"

namespace precog {
namespace {

constexpr int kLaneCh = 8;                // channels of a lane: 16 bytes of bf16
constexpr int kWaveCh = 64 * kLaneCh;
constexpr int kConvWaves = 4;             // waves of a workgroup, beside one another in the channels
constexpr int kAhead = 4;                 // tokens loaded at a time
constexpr int kRunMost = 32, kRunLeast = 8;  // tokens of a run
constexpr int64_t kL2Bytes = 32LL << 20;  // of the 8 XCDs

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Input j (0 = oldest) of the W - 1 before the first token of sequence b.
template <typename TIn>
__device__ __forceinline__ void tail_input(const ConvParams& p, int64_t b, int j, int64_t d,
                                           float (&out)[kLaneCh]) {
  const TIn* tails = static_cast<const TIn*>(p.tail0);
  int64_t row = b;
  bool known = true;
  if (p.idx != nullptr) {
    row = p.idx[b];
    known = row >= 0 && row < p.tail_rows;
  }
  if (tails == nullptr || !known) {
#pragma unroll
    for (int c = 0; c < kLaneCh; ++c) out[c] = known ? 0.f : __builtin_nanf("");
    return;
  }
  const Pack<TIn, kLaneCh> v = load_pack<kLaneCh>(tails + (row * (p.W - 1) + j) * p.D + d);
#pragma unroll
  for (int c = 0; c < kLaneCh; ++c) out[c] = widen(v.v[c]);
}

template <int W>
__device__ __forceinline__ void load_taps(const ConvParams& p, int64_t d, float (&w)[W][kLaneCh],
                                          float (&bias)[kLaneCh]) {
#pragma unroll
  for (int c = 0; c < kLaneCh; ++c) {
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][c] = p.w[(d + c) * W + j];
    bias[c] = p.bias != nullptr ? p.bias[d + c] : 0.f;
  }
}

// One token: the sum over the window and the new input, then the window moves on.
// Stores eight results; streamed past the cache if the call's do not fit there.
template <bool STREAM, typename TOut>
__device__ __forceinline__ void store_out(TOut* y, const float (&f)[kLaneCh]) {
  if constexpr (!STREAM) {
    store_pack<kLaneCh>(y, f);
    return;
  }
  typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
  Pack<TOut, kLaneCh> r;
#pragma unroll
  for (int i = 0; i < kLaneCh; ++i) r.v[i] = narrow<TOut>(f[i]);
  struct Words {
    uint4v w[sizeof(r) / 16];
  };
  const Words words = __builtin_bit_cast(Words, r);
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(r) / 16); ++i)
    __builtin_nontemporal_store(words.w[i], reinterpret_cast<uint4v*>(y) + i);
}

template <bool STREAM, typename TOut, int W>
__device__ __forceinline__ void conv_token(const float (&w)[W][kLaneCh], const float (&bias)[kLaneCh],
                                           float (&win)[W - 1][kLaneCh], const float (&x)[kLaneCh],
                                           int silu, TOut* y) {
  float out[kLaneCh];
#pragma unroll
  for (int c = 0; c < kLaneCh; ++c) {
    float s = w[0][c] * win[0][c];
#pragma unroll
    for (int j = 1; j < W - 1; ++j) s += w[j][c] * win[j][c];
    s += w[W - 1][c] * x[c];
    s += bias[c];
    out[c] = silu ? s / (1.f + __expf(-s)) : s;
#pragma unroll
    for (int j = 0; j + 2 < W; ++j) win[j][c] = win[j + 1][c];
    win[W - 2][c] = x[c];
  }
  store_out<STREAM>(y, out);
}

// The tail behind sequence b: the last W - 1 of its tail and its tokens.
template <typename TIn>
__device__ __forceinline__ void capture_tail(const ConvParams& p, int64_t b, int64_t d) {
  const Span span = sequence(p.starts, b, p.L, p.T);
  const int64_t n = span.end - span.begin;
  float keep[3][kLaneCh];
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    if (j >= p.W - 1) break;
    const int64_t back = n - (p.W - 1) + j;  // position in the sequence, negative: in the tail
    if (back < 0) {
      tail_input<TIn>(p, b, static_cast<int>(back + p.W - 1), d, keep[j]);
    } else {
      const Pack<TIn, kLaneCh> v =
          load_pack<kLaneCh>(static_cast<const TIn*>(p.x) + (span.begin + back) * p.x_stride + d);
#pragma unroll
      for (int c = 0; c < kLaneCh; ++c) keep[j][c] = widen(v.v[c]);
    }
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < p.W - 1) store_pack<kLaneCh>(static_cast<TIn*>(p.tailT) + (b * (p.W - 1) + j) * p.D + d, keep[j]);
}

// Workgroups [0, run_blocks): a run of `run` tokens.  Those behind: a sequence's
// tail.
template <typename TIn, typename TOut, int W, bool STREAM>
__global__ void __launch_bounds__(64 * kConvWaves) __attribute__((amdgpu_waves_per_eu(4))) conv_kernel(ConvParams p, int64_t run_blocks, int run) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t d = (static_cast<int64_t>(blockIdx.y) * (blockDim.x / 64) + wave) * kWaveCh + (threadIdx.x % 64) * kLaneCh;
  if (d >= p.D) return;
  if (static_cast<int64_t>(blockIdx.x) >= run_blocks) {
    capture_tail<TIn>(p, blockIdx.x - run_blocks, d);
    return;
  }
  const int64_t first = static_cast<int64_t>(blockIdx.x) * run;
  const int64_t last = first + run < p.T ? first + run : p.T;

  // the last sequence that begins at or before the run's first token (if starts
  // ascend: any one if not)
  int64_t b = 0;
  if (p.starts == nullptr) {
    b = first / p.L;
  } else {
    int64_t lo = 0, hi = p.B - 1;
    while (lo < hi) {
      const int64_t mid = (lo + hi + 1) / 2;
      if (clamp_token(p.starts[mid], p.T) <= first) lo = mid; else hi = mid - 1;
    }
    b = lo;
  }
  float w[W][kLaneCh], bias[kLaneCh];
  load_taps<W>(p, d, w, bias);
  const TIn* x = static_cast<const TIn*>(p.x) + d;
  TOut* y = static_cast<TOut*>(p.y) + d;

  // The sequences in their order, while each begins where the one before has ended.
  // What is left of the run then, tokens of no sequence or of one that descending
  // starts have put elsewhere, is sought in all of them, one a lane.
  const int lane = threadIdx.x % 64;
  const int64_t rest = (p.D - d) / kLaneCh + lane;  // lanes of the wave that are on: those below it
  const int lanes = uniform(rest < 64 ? static_cast<int>(rest) : 64);
  bool in_order = true;
  int64_t reached = first;
  int sought = 0, base = 0;
  uint64_t found = 0;
  for (;;) {
    Span span = {0, 0};
    int64_t seq = b;
    if (in_order) {
      if (reached >= last) break;
      if (b < p.B) span = sequence(p.starts, b, p.L, p.T);
      const bool holds = span.begin <= reached && reached < span.end;
      in_order = holds || (b < p.B && span.begin == reached);  // (an empty one)
      ++b;
      if (!holds) continue;
    } else {
      while (found == 0 && sought < p.B) {
        Span any = {0, 0};
        if (sought + lane < p.B) any = sequence(p.starts, sought + lane, p.L, p.T);
        found = __ballot(any.begin < any.end && any.begin < last && any.end > reached);
        base = sought;
        sought += lanes;
      }
      if (found == 0) break;
      seq = base + __builtin_ctzll(found);
      found &= found - 1;
      span = sequence(p.starts, seq, p.L, p.T);
    }
    int64_t t = span.begin > reached ? span.begin : reached;
    const int64_t stop = span.end < last ? span.end : last;
    if (in_order) reached = stop;
    float win[W - 1][kLaneCh];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int64_t back = t - (W - 1) + j;
      if (back < span.begin) {
        tail_input<TIn>(p, seq, static_cast<int>(back - span.begin + W - 1), d, win[j]);
      } else {
        const Pack<TIn, kLaneCh> v = load_pack<kLaneCh>(x + back * p.x_stride);
#pragma unroll
        for (int c = 0; c < kLaneCh; ++c) win[j][c] = widen(v.v[c]);
      }
    }
    for (; t < stop; t += kAhead) {
      Pack<TIn, kLaneCh> in[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (t + i < stop) in[i] = load_pack<kLaneCh>(x + (t + i) * p.x_stride);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (t + i < stop) {
          float v[kLaneCh];
#pragma unroll
          for (int c = 0; c < kLaneCh; ++c) v[c] = widen(in[i].v[c]);
          conv_token<STREAM, TOut, W>(w, bias, win, v, p.silu, y + (t + i) * p.D);
        }
      }
    }
  }
}

// One token of session i: the workgroup is one wave of 512 channels.
template <typename TIn, typename TOut, int W>
__global__ void __launch_bounds__(64) conv_step_kernel(ConvParams p) {
  __shared__ int next_row;
  const int tid = threadIdx.x;
  const int64_t b = blockIdx.x;
  const int64_t d = static_cast<int64_t>(blockIdx.y) * kWaveCh + tid * kLaneCh;
  const int64_t slot = p.idx[b];
  if (slot < 0 || slot >= p.tail_rows) return;
  if (!leads_slot(p.idx, b, static_cast<int32_t>(slot), tid, 64)) return;
  const bool on = d < p.D;
  TIn* tail = static_cast<TIn*>(p.tailT) + slot * (W - 1) * p.D + d;
  float w[W][kLaneCh], bias[kLaneCh], win[W - 1][kLaneCh];
  if (on) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const Pack<TIn, kLaneCh> v = load_pack<kLaneCh>(tail + j * p.D);
#pragma unroll
      for (int c = 0; c < kLaneCh; ++c) win[j][c] = widen(v.v[c]);
    }
    if (p.y != nullptr) load_taps<W>(p, d, w, bias);
  }
  for (int64_t row = b; row >= 0;
       row = next_of_slot(p.idx, p.B, row, static_cast<int32_t>(slot), tid, 64, &next_row)) {
    if (!on) continue;
    const Pack<TIn, kLaneCh> in = load_pack<kLaneCh>(static_cast<const TIn*>(p.x) + row * p.x_stride + d);
    float v[kLaneCh];
#pragma unroll
    for (int c = 0; c < kLaneCh; ++c) v[c] = widen(in.v[c]);
    if (p.y != nullptr) {
      conv_token<false, TOut, W>(w, bias, win, v, p.silu, static_cast<TOut*>(p.y) + row * p.D + d);
    } else {
#pragma unroll
      for (int c = 0; c < kLaneCh; ++c) {
#pragma unroll
        for (int j = 0; j + 2 < W; ++j) win[j][c] = win[j + 1][c];
        win[W - 2][c] = v[c];
      }
    }
  }
  if (on) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) store_pack<kLaneCh>(tail + j * p.D, win[j]);
  }
}

template <typename Fn>
hipError_t by_types(int W, int in_dtype, int out_dtype, Fn fn) {
  const auto width = [&](auto in, auto out) {
    if (W == 2) return fn(in, out, std::integral_constant<int, 2>{});
    if (W == 3) return fn(in, out, std::integral_constant<int, 3>{});
    return fn(in, out, std::integral_constant<int, 4>{});
  };
  if (in_dtype == PRECOG_F32)
    return out_dtype == PRECOG_F32 ? width(float{}, float{}) : width(float{}, bf16_t{});
  return out_dtype == PRECOG_F32 ? width(bf16_t{}, float{}) : width(bf16_t{}, bf16_t{});
}

}  // namespace

hipError_t launch_conv(const ConvParams& p, int in_dtype, int out_dtype, int cus, hipStream_t s) {
  return by_types(p.W, in_dtype, out_dtype, [&](auto in, auto out, auto width) {
    using TIn = decltype(in);
    using TOut = decltype(out);
    constexpr int W = decltype(width)::value;
    const int64_t wave_cols = (p.D + kWaveCh - 1) / kWaveCh;
    const int waves = static_cast<int>(wave_cols < kConvWaves ? wave_cols : kConvWaves);
    const uint32_t cols = static_cast<uint32_t>((wave_cols + waves - 1) / waves);
    // runs of 32 tokens where eight waves a CU remain, else down to 8 (3 x 1,001
    // tokens of 1,000 fp32 channels: 23 us a call with 32, 15 us with 8)
    int run = kRunMost;
    while (run > kRunLeast && (p.T + run - 1) / run * wave_cols < 8LL * cus) run /= 2;
    const int64_t runs = p.y != nullptr ? (p.T + run - 1) / run : 0;
    const int64_t tails = p.tailT != nullptr ? p.B : 0;
    const bool streamed = p.T * p.D * static_cast<int64_t>(sizeof(TOut)) > kL2Bytes;
    // in place, the runs read tails that the capture replaces: then it goes
    // behind them, in a launch of its own
    const bool apart = p.tail0 != nullptr && p.tail0 == p.tailT && runs > 0;
    const dim3 grid(static_cast<uint32_t>(runs + (apart ? 0 : tails)), cols);
    if (streamed)
      conv_kernel<TIn, TOut, W, true><<<grid, 64 * waves, 0, s>>>(p, runs, run);
    else
      conv_kernel<TIn, TOut, W, false><<<grid, 64 * waves, 0, s>>>(p, runs, run);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !apart || tails == 0) return e;
    conv_kernel<TIn, TOut, W, false><<<dim3(static_cast<uint32_t>(tails), cols), 64 * waves, 0, s>>>(p, 0, run);
    return hipGetLastError();
  });
}

hipError_t launch_conv_step(const ConvParams& p, int in_dtype, int out_dtype, hipStream_t s) {
  return by_types(p.W, in_dtype, out_dtype, [&](auto in, auto out, auto width) {
    const dim3 grid(static_cast<uint32_t>(p.B), static_cast<uint32_t>((p.D + kWaveCh - 1) / kWaveCh));
    conv_step_kernel<decltype(in), decltype(out), decltype(width)::value><<<grid, 64, 0, s>>>(p);
    return hipGetLastError();
  });
}

}  // namespace precog
