// Log probabilities, entropy and top alternatives of rows of logits in one
// pass over them:
//
//   m = max x, s = sum exp(x - m), t = sum exp(x - m) (x - m)
//   log p_v = x_v - m - ln s,   entropy = ln s - t / s
//
// Every lane keeps (m, s, t) of the logits it has seen, rescaled when its
// maximum grows; the lanes' triples are joined by the same rule.  Every wave
// keeps the `top` best logits it has seen, sorted, one per lane, and its
// tiles come in ascending order of token ids, so a logit enters the list only
// if it is larger than the last entry, and behind its equals.
#include "layer_ops.h"
#include "wave_ops.h"

namespace precog {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kLane = 8;                    // logits of a lane in a tile
constexpr int kWaveTile = 64 * kLane;
constexpr float kLog2e = 1.44269504088896341f;
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

// The list of a wave: entry i (i < top) in lane i, best first.
struct Best {
  float val;
  int id;
  float last;  // entry top - 1: what a logit has to be larger than
};

__device__ __forceinline__ void insert(Best& best, float v, int id, int top) {
  const int lane = threadIdx.x % 64;
  const int at = __popcll(__ballot(best.val >= v && best.id >= 0));
  const float up = __shfl_up(best.val, 1);
  const int up_id = __shfl_up(best.id, 1);
  if (lane == at) {
    best.val = v;
    best.id = id;
  } else if (lane > at && lane < top) {
    best.val = up;
    best.id = up_id;
  }
  best.last = readlane(best.val, top - 1);
}

// (value, id) a is better than b: larger, or equal and lower; id -1 is worse
// than any.
__device__ __forceinline__ bool better(float av, int ai, float bv, int bi) {
  if (ai < 0 || bi < 0) return ai >= 0;
  return av > bv || (av == bv && ai < bi);
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
  __shared__ float vals[kWaves * kScoreMaxTop];
  __shared__ int ids[kWaves * kScoreMaxTop];
  __shared__ float out_val[kScoreMaxTop];
  __shared__ int out_id[kScoreMaxTop];
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int64_t row = blockIdx.x / p.splits;
  const int part = static_cast<int>(blockIdx.x % p.splits);
  // 16-byte aligned address at or below the row; its logits begin `skip` on
  const uintptr_t at = reinterpret_cast<uintptr_t>(p.logits) + row * p.row_stride * sizeof(T);
  const int skip = static_cast<int>((at & 15) / sizeof(T));
  const T* base = reinterpret_cast<const T*>(at & ~static_cast<uintptr_t>(15));

  Sums a{kNone, 0.f, 0.f};
  Best best{kNone, -1, kNone};
  // Position j of the aligned axis holds token j - skip; this workgroup's
  // positions are [low, high), the last part's up to the row's end.
  const int64_t begin = part * p.span;
  const int64_t low = part == 0 ? skip : begin;
  const int64_t high = begin >= p.V ? low : begin + p.span >= p.V ? p.V + skip : begin + p.span;
  for (int64_t j0 = begin + wave * kWaveTile; j0 < high; j0 += kScoreTile) {
    const int64_t j = j0 + lane * kLane;
    float x[kLane];
    if (j >= low && j + kLane <= high) {
      const Pack<T, kLane> v = load_pack<kLane>(base + j);
#pragma unroll
      for (int i = 0; i < kLane; ++i) x[i] = widen(v.v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kLane; ++i) x[i] = j + i >= low && j + i < high ? widen(base[j + i]) : kNone;
    }
    float m = x[0];
#pragma unroll
    for (int i = 1; i < kLane; ++i) m = fmaxf(m, x[i]);
    if (m > a.m) rescale(a, m);
    const float ref = a.m == kNone ? 0.f : a.m;
#pragma unroll
    for (int i = 0; i < kLane; ++i) {
      const float d = x[i] - ref, e = exp_of(d);
      a.s += e;
      a.t += e * fmaxf(d, -1e30f);
    }
    if (TOP) {
      uint64_t more = __ballot(m > best.last);
      while (more) {
        const int from = __builtin_ctzll(more);
#pragma unroll
        for (int i = 0; i < kLane; ++i) {
          const float v = readlane(x[i], from);
          if (v > best.last) insert(best, v, static_cast<int>(j0 + from * kLane + i - skip), p.top);
        }
        more = __ballot(m > best.last) & ~((2ull << from) - 1);
      }
    }
  }
#pragma unroll
  for (int mask = 1; mask < 64; mask <<= 1) {
    const Sums b{__shfl_xor(a.m, mask), __shfl_xor(a.s, mask), __shfl_xor(a.t, mask)};
    a = join(a, b);
  }
  if (lane == 0) wave_sums[wave] = a;
  if (TOP && lane < p.top) {
    vals[wave * p.top + lane] = best.val;
    ids[wave * p.top + lane] = best.id;
  }
  __syncthreads();
  a = join(join(wave_sums[0], wave_sums[1]), join(wave_sums[2], wave_sums[3]));
  if (TOP) {
    // every candidate counts the better ones; entries without a token are
    // ranked among themselves by their place
    const int n = kWaves * p.top;
    if (tid < n) {
      const float v = vals[tid];
      const int id = ids[tid];
      int rank = 0;
      for (int i = 0; i < n; ++i)
        rank += better(vals[i], ids[i], v, id) || (id < 0 && ids[i] < 0 && i < tid);
      if (rank < p.top) {
        out_val[rank] = v;
        out_id[rank] = id;
      }
    }
    __syncthreads();
  }
  if (wave != 0) return;
  const float val = TOP && lane < p.top ? out_val[lane] : kNone;
  const int id = TOP && lane < p.top ? out_id[lane] : -1;
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

// Joins the parts of a row: one wave, one part a lane.  Each round takes the
// best head of the parts' sorted lists.
template <typename T>
__global__ void __launch_bounds__(64) score_join_kernel(ScoreParams p) {
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x, piece = row * p.splits + lane;
  Sums a{kNone, 0.f, 0.f};
  if (lane < p.splits) {
    const ScorePart b = p.part[piece];
    a = {b.m, b.s, b.t};
  }
#pragma unroll
  for (int mask = 1; mask < 64; mask <<= 1) {
    const Sums b{__shfl_xor(a.m, mask), __shfl_xor(a.s, mask), __shfl_xor(a.t, mask)};
    a = join(a, b);
  }
  float val = kNone;
  int id = -1, head = 0;
  float hv = kNone;
  int hi = -1;
  if (p.top > 0 && lane < p.splits) {
    hv = p.cand_val[piece * p.top];
    hi = p.cand_id[piece * p.top];
  }
  for (int k = 0; k < p.top; ++k) {
    float bv = hv;
    int bi = hi;
#pragma unroll
    for (int mask = 1; mask < 64; mask <<= 1) {
      const float ov = __shfl_xor(bv, mask);
      const int oi = __shfl_xor(bi, mask);
      if (better(ov, oi, bv, bi)) {
        bv = ov;
        bi = oi;
      }
    }
    if (lane == k) {
      val = bv;
      id = bi;
    }
    if (bi >= 0 && hi == bi) {  // ids are unique in a row: this lane's head was taken
      ++head;
      hv = kNone;
      hi = -1;
      if (head < p.top) {
        hv = p.cand_val[piece * p.top + head];
        hi = p.cand_id[piece * p.top + head];
      }
    }
  }
  write_row<T>(p, row, a, val, id);
}

template <typename T>
hipError_t launch_typed(const ScoreParams& p, hipStream_t s) {
  const uint32_t blocks = static_cast<uint32_t>(p.T * p.splits);
  if (p.top > 0)
    score_kernel<T, true><<<dim3(blocks), kThreads, 0, s>>>(p);
  else
    score_kernel<T, false><<<dim3(blocks), kThreads, 0, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  score_join_kernel<T><<<dim3(static_cast<uint32_t>(p.T)), 64, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_score(const ScoreParams& p, int dtype, hipStream_t s) {
  if (dtype == PRECOG_F32) return launch_typed<float>(p, s);
  return dtype == PRECOG_BF16 ? launch_typed<bf16_t>(p, s) : launch_typed<f16_t>(p, s);
}

}  // namespace precog
