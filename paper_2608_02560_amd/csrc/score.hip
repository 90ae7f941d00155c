// Log probabilities, entropy and top alternatives of rows of logits in one
// pass over them:
//
//   m = max x, s = sum exp(x - m), t = sum exp(x - m) (x - m)
//   log p_v = x_v - m - ln s,   entropy = ln s - t / s
//
// Every lane keeps (m, s, t) of the logits it has seen, rescaled when its
// maximum grows; the lanes' triples are joined by the same rule.
//
// Every wave keeps the best `top` logits it has seen, sorted, one per lane.
// Logits larger than the last of them go to a list in LDS and are sorted and
// merged 64 at a time, so that what a wave does for them is a comparison a
// tile and some hundred instructions for 64 that pass it.  Before the first
// ones, the top-th largest of the lanes' first maxima bounds them: at least
// `top` logits reach it.  A wave's tiles come in ascending order of token ids,
// and entries are compared by (logit, lower id), so equal logits keep the
// order of their ids.
#include "layer_ops.h"
#include "wave_ops.h"

#include <type_traits>

namespace precog {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kLane = 8;                    // logits of a lane in a tile
constexpr int kWaveTile = 64 * kLane;
constexpr int kTiles = 4;                   // tiles of a wave that are on their way together
constexpr int kWaiting = 64 + kWaveTile;    // candidates of a wave in LDS
constexpr float kLog2e = 1.44269504088896341f;
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
constexpr float kNone = -__builtin_inff();
static_assert(kScoreTile == kWaves * kWaveTile, "a tile of every wave");

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

struct Sums {
  float m, s, t;
};

// Sums with maximum `to` >= a.m (or both -infinity).
__device__ __forceinline__ void rescale(Sums& a, float to) {
  const float delta = a.m == kNone ? 0.f : to - a.m;
  const float f = a.m == kNone ? 0.f : exp_of(-delta);
  a.t = f > 0.f ? f * (a.t - delta * a.s) : 0.f * a.t;
  a.s = f * a.s;
  a.m = to;
}

__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  rescale(a, m);
  rescale(b, m);
  return {m, a.s + b.s, a.t + b.t};
}

// (value, id) a is better than b: larger, or equal and lower; id -1 is worse
// than any.
__device__ __forceinline__ bool better(float av, int ai, float bv, int bi) {
  // as unsigned numbers, -1 is the highest id: only -infinity stands beside it
  return av > bv || (av == bv && static_cast<uint32_t>(ai) < static_cast<uint32_t>(bi));
}

struct Entry {
  float val;
  int id;
};

// The value of lane l ^ kMask, without a trip through LDS.
template <int kMask>
__device__ __forceinline__ int other_lane(int v) {
  constexpr int kHalfMirror = 0x141, kQuadMirror = 0x1B;  // l ^ 7, l ^ 3
  if constexpr (kMask == 1) return dpp<kQuadSwap1>(v);
  if constexpr (kMask == 2) return dpp<kQuadSwap2>(v);
  if constexpr (kMask == 4) return dpp<kQuadMirror>(dpp<kHalfMirror>(v));
  if constexpr (kMask == 8) return dpp<kRowRor8>(v);
  const bool upper = threadIdx.x % 64 & kMask;
  if constexpr (kMask == 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return upper ? s[0] : s[1];
  }
  const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return upper ? s[0] : s[1];
}
template <int kMask>
__device__ __forceinline__ Entry other_lane(const Entry& e) {
  return {__int_as_float(other_lane<kMask>(__float_as_int(e.val))), other_lane<kMask>(e.id)};
}

// One stage of a bitonic network: lanes l and l ^ kMask keep the better or the
// worse of their entries.
template <int kMask>
__device__ __forceinline__ void exchange(Entry& e, bool keep_better) {
  const Entry o = other_lane<kMask>(e);
  if (better(o.val, o.id, e.val, e.id) == keep_better) e = o;
}

// Sorts the entries of a wave, the best first.
__device__ __forceinline__ void sort64(Entry& e) {
  const int lane = threadIdx.x % 64;
  const auto stage = [&](auto mask, int block) {
    constexpr int kMask = decltype(mask)::value;
    exchange<kMask>(e, ((lane & kMask) == 0) == ((lane & block) == 0));
  };
  using std::integral_constant;
#pragma unroll
  for (int block = 2; block <= 64; block <<= 1) {
    if (block >= 64) stage(integral_constant<int, 32>{}, block);
    if (block >= 32) stage(integral_constant<int, 16>{}, block);
    if (block >= 16) stage(integral_constant<int, 8>{}, block);
    if (block >= 8) stage(integral_constant<int, 4>{}, block);
    if (block >= 4) stage(integral_constant<int, 2>{}, block);
    stage(integral_constant<int, 1>{}, block);
  }
}

// The best 64 of two sorted lists, sorted.
__device__ __forceinline__ void merge64(Entry& list, const Entry& other) {
  const int lane = threadIdx.x % 64;
  constexpr int kRowMirror = 0x140;  // l ^ 15
  Entry o{dpp<kRowMirror>(other.val), dpp<kRowMirror>(other.id)};
  o = other_lane<32>(other_lane<16>(o));
  if (better(o.val, o.id, list.val, list.id)) list = o;
  const auto stage = [&](auto mask) {
    exchange<decltype(mask)::value>(list, (lane & decltype(mask)::value) == 0);
  };
  using std::integral_constant;
  stage(integral_constant<int, 32>{});
  stage(integral_constant<int, 16>{});
  stage(integral_constant<int, 8>{});
  stage(integral_constant<int, 4>{});
  stage(integral_constant<int, 2>{});
  stage(integral_constant<int, 1>{});
}

// The largest number that at least n lanes' v reach, as far as the upper 16
// bits of the order-preserving whole numbers tell (lower bits as zeros).
__device__ __forceinline__ float reached_by(float v, int n) {
  const int bits = __float_as_int(v);
  const uint32_t key = static_cast<uint32_t>(bits < 0 ? ~bits : bits | 0x80000000) >> 16;
  uint32_t at = 0;
#pragma unroll
  for (int b = 15; b >= 0; --b) {
    const uint32_t next = at | 1u << b;
    if (__popcll(__ballot(key >= next)) >= n) at = next;
  }
  at <<= 16;
  return __uint_as_float(at & 0x80000000 ? at & 0x7fffffff : ~at);
}

// Writes a row's numbers from its joined sums; its alternatives' ids and
// logits come from lane i of the calling wave.
template <typename T>
__device__ __forceinline__ void write_row(const ScoreParams& p, int64_t row, const Sums& a, float val, int id) {
  const int lane = threadIdx.x % 64;
  const float nan = __builtin_nanf("");
  const bool broken = !(a.s == a.s) || a.m == __builtin_inff();  // a NaN or an infinity
  const float lse = logf(a.s);
  if (lane == 0) {
    if (p.token != nullptr) {
      const int64_t tok = p.token[row];
      float lp;
      if (broken)
        lp = nan;
      else if (tok < 0)
        lp = 0.f;
      else if (tok >= p.V || a.m == kNone)
        lp = kNone;
      else
        lp = (widen(static_cast<const T*>(p.logits)[row * p.row_stride + tok]) - a.m) - lse;
      p.logprob[row] = lp;
    }
    if (p.entropy != nullptr) p.entropy[row] = broken ? nan : a.m == kNone ? 0.f : lse - a.t / a.s;
  }
  if (lane < p.top) {
    p.top_id[row * p.top + lane] = broken ? -1 : id;
    p.top_logprob[row * p.top + lane] = broken ? nan : id < 0 ? kNone : (val - a.m) - lse;
  }
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) score_kernel(ScoreParams p) {
  __shared__ Sums wave_sums[kWaves];
  __shared__ Entry waiting[TOP ? kWaves : 1][TOP ? kWaiting : 1];
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int64_t row = blockIdx.x / p.splits;
  const int part = static_cast<int>(blockIdx.x % p.splits);
  // 16-byte aligned address at or below the row; its logits begin `skip` on
  const uintptr_t at = reinterpret_cast<uintptr_t>(p.logits) + row * p.row_stride * sizeof(T);
  const int skip = static_cast<int>((at & 15) / sizeof(T));

  Sums a{kNone, 0.f, 0.f};
  Entry best{kNone, -1};
  float last = kNone;  // what a logit has to be larger than
  int count = 0;       // candidates in `waiting`
  bool first_group = true;
  const auto settle = [&] {  // takes up to 64 candidates into the list
    wave_fence();
    const int n = count < 64 ? count : 64;
    Entry e{kNone, -1};
    if (lane < n) e = waiting[TOP ? wave : 0][TOP ? count - n + lane : 0];
    wave_fence();
    count -= n;
    sort64(e);
    merge64(best, e);
    last = fmaxf(last, readlane(best.val, p.top - 1));
  };
  // Position j of the aligned axis holds token j - skip; this workgroup's
  // positions are [low, high), the last part's up to the row's end.
  const int vocab = static_cast<int>(p.V), span = static_cast<int>(p.span);
  const int begin = part * span;
  const int low = part == 0 ? skip : begin;
  const int high = begin >= vocab ? low : begin + span >= vocab ? vocab + skip : begin + span;
  // loads past the last position read nothing
  const __amdgpu_buffer_rsrc_t base =
      make_rsrc(reinterpret_cast<const void*>(at & ~static_cast<uintptr_t>(15)),
                (static_cast<uint32_t>(high) * sizeof(T) + 3) & ~3u);
  struct Group {
    uint4v raw[kTiles][sizeof(T) * kLane / 16];
  };
  const auto fetch = [&](int j0, Group& g) {
#pragma unroll
    for (int u = 0; u < kTiles; ++u)
#pragma unroll
      for (int w = 0; w < static_cast<int>(sizeof(T) * kLane / 16); ++w)
        g.raw[u][w] = __builtin_bit_cast(
            uint4v, __builtin_amdgcn_raw_buffer_load_b128(
                        base, static_cast<uint32_t>((j0 + u * kScoreTile + lane * kLane) * sizeof(T)) + 16 * w, 0, 0));
  };
  const auto take = [&](int j0, const Group& g) {
    float x[kTiles][kLane];
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
      const Pack<T, kLane> v = __builtin_bit_cast(Pack<T, kLane>, g.raw[u]);
#pragma unroll
      for (int i = 0; i < kLane; ++i) x[u][i] = widen(v.v[i]);
    }
    if (j0 < low || j0 + (kTiles - 1) * kScoreTile + kWaveTile > high) {  // part of the group is another's
#pragma unroll
      for (int u = 0; u < kTiles; ++u)
#pragma unroll
        for (int i = 0; i < kLane; ++i) {
          const int j = j0 + u * kScoreTile + lane * kLane + i;
          x[u][i] = j >= low && j < high ? x[u][i] : kNone;
        }
    }
    float tile_max[kTiles];
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
      float m = x[u][0];
#pragma unroll
      for (int i = 1; i < kLane; ++i) m = fmaxf(m, x[u][i]);
      tile_max[u] = m;
    }
    float m = tile_max[0];
#pragma unroll
    for (int u = 1; u < kTiles; ++u) m = fmaxf(m, tile_max[u]);
    if (m > a.m) rescale(a, m);
    const float ref = a.m == kNone ? 0.f : a.m;
#pragma unroll
    for (int u = 0; u < kTiles; ++u)
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        const float d = x[u][i] - ref, e = exp_of(d);
        a.s += e;
        a.t += e * fmaxf(d, -1e30f);
      }
    if (!TOP) return;
    if (first_group) {
      first_group = false;
      const float bound = reached_by(m, p.top);
      // larger than the next number below it: at least as large as it
      last = bound > kNone ? __uint_as_float(__float_as_uint(bound) + (bound > 0.f ? -1 : 1)) : kNone;
      if (bound == 0.f) last = -1e-45f;
    }
    if (__ballot(m > last) == 0) return;
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
      if (__ballot(tile_max[u] > last) == 0) continue;
      const int first = j0 + u * kScoreTile + lane * kLane - skip;
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        const float v = x[u][i] + 0.f;  // one zero
        const uint64_t mask = __ballot(v > last);
        if (mask == 0) continue;
        if (v > last)
          waiting[TOP ? wave : 0][TOP ? count + __builtin_amdgcn_mbcnt_hi(
                                                    static_cast<uint32_t>(mask >> 32),
                                                    __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0))
                                      : 0] = Entry{v, first + i};
        count += __popcll(mask);
      }
      while (count >= 64) settle();
    }
  };
  Group even, odd;
  constexpr int kStep = kTiles * kScoreTile;
  int j0 = begin + wave * kWaveTile;
  if (j0 < high) fetch(j0, even);
  while (j0 < high) {
    fetch(j0 + kStep, odd);  // past the row: zeros that no one takes
    take(j0, even);
    j0 += kStep;
    if (j0 >= high) break;
    fetch(j0 + kStep, even);
    take(j0, odd);
    j0 += kStep;
  }
  if (TOP)
    while (count > 0) settle();
#pragma unroll
  for (int mask = 1; mask < 64; mask <<= 1) {
    const Sums b{__shfl_xor(a.m, mask), __shfl_xor(a.s, mask), __shfl_xor(a.t, mask)};
    a = join(a, b);
  }
  if (lane == 0) wave_sums[wave] = a;
  if (TOP) waiting[TOP ? wave : 0][TOP ? lane : 0] = best;
  __syncthreads();
  if (wave != 0) return;
  a = join(join(wave_sums[0], wave_sums[1]), join(wave_sums[2], wave_sums[3]));
  if (TOP)
#pragma unroll
    for (int w = 1; w < kWaves; ++w) merge64(best, waiting[TOP ? w : 0][TOP ? lane : 0]);
  const float val = best.val;
  const int id = best.id;
  if (p.splits == 1) {
    write_row<T>(p, row, a, val, id);
    return;
  }
  const int64_t piece = row * p.splits + part;
  if (lane == 0) p.part[piece] = ScorePart{a.m, a.s, a.t, 0};
  if (lane < p.top) {
    p.cand_val[piece * p.top + lane] = val;
    p.cand_id[piece * p.top + lane] = id;
  }
}

// Joins the parts of a row.  Wave w merges the lists of the parts w, w + 4, ..
// (two on their way at a time), then the first wave the four that remain.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) score_join_kernel(ScoreParams p) {
  __shared__ Entry lists[kWaves][64];
  const int lane = threadIdx.x % 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t row = blockIdx.x;
  Entry best{kNone, -1};
  if (TOP) {
    const auto load = [&](int part) {
      Entry e{kNone, -1};
      if (part < p.splits && lane < p.top) {
        const int64_t at = (row * p.splits + part) * p.top + lane;
        e = {p.cand_val[at], p.cand_id[at]};
      }
      return e;
    };
    best = load(wave);
    Entry next = load(wave + kWaves);
    for (int part = wave + kWaves; part < p.splits; part += kWaves) {
      const Entry now = next;
      next = load(part + kWaves);
      merge64(best, now);
    }
    lists[wave][lane] = best;
    __syncthreads();
  }
  if (wave != 0) return;
  Sums a{kNone, 0.f, 0.f};
  if (lane < p.splits) {
    const ScorePart b = p.part[row * p.splits + lane];
    a = {b.m, b.s, b.t};
  }
#pragma unroll
  for (int mask = 1; mask < 64; mask <<= 1) {
    const Sums b{__shfl_xor(a.m, mask), __shfl_xor(a.s, mask), __shfl_xor(a.t, mask)};
    a = join(a, b);
  }
  if (TOP)
#pragma unroll
    for (int w = 1; w < kWaves; ++w) merge64(best, lists[w][lane]);
  write_row<T>(p, row, a, best.val, best.id);
}

template <typename T>
hipError_t launch_typed(const ScoreParams& p, hipStream_t s) {
  const uint32_t blocks = static_cast<uint32_t>(p.T * p.splits);
  if (p.top > 0)
    score_kernel<T, true><<<dim3(blocks), kThreads, 0, s>>>(p);
  else
    score_kernel<T, false><<<dim3(blocks), kThreads, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  if (p.top > 0)
    score_join_kernel<T, true><<<dim3(static_cast<uint32_t>(p.T)), kThreads, 0, s>>>(p);
  else
    score_join_kernel<T, false><<<dim3(static_cast<uint32_t>(p.T)), 64, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_score(const ScoreParams& p, int dtype, hipStream_t s) {
  if (dtype == PRECOG_F32) return launch_typed<float>(p, s);
  return dtype == PRECOG_BF16 ? launch_typed<bf16_t>(p, s) : launch_typed<f16_t>(p, s);
}

}  // namespace precog
