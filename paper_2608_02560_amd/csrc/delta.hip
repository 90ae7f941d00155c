// The gated delta rule over whole sequences, a block of 32 tokens at a time.
//
// With b_i the sum of the log decays of a block's tokens up to i, G_ij =
// exp(b_i - b_j) for i >= j, S the state before the block and u_i the values
// that the tokens write:
//
//   A_ij = beta_i G_ij k_i.k_j  (i > j),   T = (I + A)^-1
//   X = diag(beta) (V - diag(e^b) K S),   U = T X
//   O = scale (diag(e^b) Q S + (G . Q K^T) U)
//   S <- e^{b_end} S + K^T diag(e^{b_end - b}) U
//
// so a block is a handful of small matrix products, and only those with S
// depend on the block before.  One workgroup owns one head of one sequence (or
// some of its columns: the columns of S and V do not meet).  Two kinds of
// waves share it:
//
//   prepare  one wave takes a block from the queries, keys and gates to the
//            matrix operands K, K^T, Q, T, G . QK^T and the row factors, in
//            LDS, some blocks ahead of their use;
//   chain    each wave keeps its columns of S in registers and runs the
//            dependent products; no operand of it that changes leaves the
//            wave, since a product's result lies in the registers as the next
//            product wants its operand.
//
// Keys have any length: with |k| the power of two next to it (over what qk_norm
// divides by), k^ = k / |k| and u' = |k| u in place of u, A_ij = beta_i |k_i|^2 G_ij
// k^_i.k^_j and X = diag(beta |k|) V - diag(beta |k|^2 e^b) K^ S.
// What a closed gate or a key of zeros keeps out, however large, is a zero of X.
//
// Operands.  v_mfma_f32_16x16x32_f16 takes rows (columns) l % 16 and the eight
// depths 8 (l / 16) + j of its operands from lane l, and gives lane l the rows
// 4 (l / 16) + r of column l % 16.  Two results of 16 rows are therefore one
// operand of depth 32 whose depth 8 q + j is row 4 q + j of the first (j < 4)
// or row 4 q + j - 4 of the second, and the other operand is laid out to match.
//
// Numbers.  The states, all sums, decays and norms are fp32 (b is summed in
// fp64, where the differences of two positions are taken), and so are T, X, U and
// G . Q K^T with their products: the tokens of a block differ by what decays, gates,
// values and key lengths make of them, and a token's small numbers are not to
// depend on its neighbours' large ones.  The products with S and K have operands of
// fp16: keys and queries under the power of two that brings the row's norm to
// [2^-1/2, 2^1/2) (exact for bf16 down to 2^-16 of the norm, good to 2^-24 of it;
// fp32 inputs as two halves of 11 bits), S and the U that goes into it as two halves
// (22 bits) under a power of two of their column's, below 2^16 and 2^8.  Products of
// two low halves are left out (2^-22).  A bf16 o is computed as an fp32 one and
// rounded at the end: its two terms may cancel, as they do where a value is replaced.
// Errors against 64 bits over 40,001 tokens: states 1.8e-7, o 2.2e-7 (a plain
// evaluation of blocks in 32 bits: 2.3e-7 and 3.1e-7).
//
// What bounds it: vector instructions take 55 % of the SIMDs' cycles and matrix
// ones 45 %, half of these the fp32 ones (32 sequences of 3,000 tokens and 16 heads of
// 128 x 128: 650 us at 2.06 GHz, 1.9 TB/s).
//
// Long sequences of few heads.  A head's blocks follow one another, so a call of up
// to 64 heads (blocks of 128 columns of them) whose sequences have 64 blocks or more
// on average is cut into segments of each sequence: the end state of a
// segment is Phi S + F, where F is its end state from zeros and the columns of
// Phi are those from unit vectors with values of zero, both computed by the same
// blocks.  Three launches: Phi and F of every segment but the last; the states
// between them, one after the other (join_kernel, in fp32); all segments again,
// from those, with their outputs.  Three times the work, on all CUs.
#include "layer_ops.h"
#include "wave_ops.h"

#include <type_traits>

namespace precog {
namespace {

constexpr int kBlockTokens = 32;
constexpr int kChainMax = kDeltaChainMax;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// Row factors of a block's tokens, and what belongs to the block.
struct Factors {
  float v[kBlockTokens];   // beta |k| of V
  float x[kBlockTokens];   // beta |k|^2 e^b of X's subtrahend
  float u[kBlockTokens];   // e^{b_end - b} of a row of U before K^T
  float q[kBlockTokens];   // scale |q| e^b of Q S
  float o[kBlockTokens];   // scale |q| of Q K^T U
  float decay;             // e^{b_end}
  float pad[3];
};

// What a call computes beside the states.
constexpr int kNoOutput = 0, kOut16 = 1, kOut32 = 2;

// A lower triangle of 32 x 32 numbers as operands of v_mfma_f32_16x16x4_f32: the tiles
// (0, 0), (1, 0) and (1, 1); lane l has the columns 4 (l / 16) .. + 3 of row l % 16.
// Step r multiplies those of register r, as a result's register r holds its rows.
using Lower = float4v[3][64];

// A block's operands in LDS, in 1 KB fragments of one matrix instruction.
template <int KP, bool IN32, int OUT>
struct Buffer {
  static constexpr int kHalves = IN32 ? 2 : 1;
  static constexpr int kSteps = KP / 32;
  half8 k[kHalves][2][kSteps][64];    // token tile, depth step
  half8 q[OUT ? kHalves : 0][2][kSteps][64];
  half8 kt[kHalves][KP / 16][64];     // state row tile; depth: the block's tokens
  Lower t;
  Lower p[OUT ? 1 : 0];
  Factors f;
};

// A prepare wave's own LDS.  b log2(e) is the sum of two floats, so that
// differences of it are good to 2^-24 of themselves.
struct Scratch {
  float b[kBlockTokens], b_low[kBlockTokens];
  float rk[kBlockTokens];
  float rq[kBlockTokens];
  float beta[kBlockTokens];   // beta |k|^2
};

// A and its inverse take the place of T's operands until these are made, tile by
// tile.  Groups of four columns are permuted within a row, so that 16 lanes that read
// a column of groups meet different banks, and neighbouring rows of the last tile
// change places, so that a row of it and the same one of the first do.
__device__ __forceinline__ uint32_t a_at(uint32_t tile, uint32_t r, uint32_t c) {
  return 256 * tile + 16 * (r ^ tile / 2) + (4 * (c / 4 ^ r / 4) | c % 4);
}

template <int KP, bool IN32, int OUT>
struct Shared {
  // as many as fit into the 160 KB of a CU, up to five; each prepare wave works on a
  // buffer of its own
  static constexpr int kPrepare = delta_prepare_waves(IN32, KP == 128);
  static constexpr int kBuffers = kPrepare + 1;
  Buffer<KP, IN32, OUT> buf[kBuffers];
  Scratch scratch[kPrepare];
  int ready[kBuffers];       // block held by the buffer, counted from 1
  int done[kChainMax];       // blocks that the chain wave has read
};

__device__ __forceinline__ float4v mfma(half8 a, half8 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float4v mfma(float a, float b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ half2 to_half2(float a, float b) {
  return __builtin_convertvector((float2v{a, b}), half2);  // nearest even
}

// The lane's number as a value of its own: what is computed from it is not kept
// in registers from one part of a long function to the next.
__device__ __forceinline__ int fresh_lane() {
  int lane = threadIdx.x % 64;
  asm volatile("" : "+v"(lane));
  return lane;
}

__device__ __forceinline__ float max_abs(float m, float v) { return fmaxf(m, fabsf(v)); }

// The largest of lanes l, l ^ 16, l ^ 32 and l ^ 48.
__device__ __forceinline__ float max_of_rows(float v) {
  const uint32_t b = __float_as_uint(v);
  const auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  const float m = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
  const uint32_t c = __float_as_uint(m);
  const auto t = __builtin_amdgcn_permlane16_swap(c, c, false, false);
  return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}

// 2^e and 2^-e with 2^e m in [2^14, 2^15), e bounded where one of them would
// leave fp32.
struct Scale {
  float up, down;
};
__device__ __forceinline__ Scale scale_of(float m) {
  int e = static_cast<int>(__float_as_uint(m) >> 23 & 255);
  e = e < 15 ? 15 : e;
  return {__uint_as_float(static_cast<uint32_t>(268 - e) << 23), __uint_as_float(static_cast<uint32_t>(e - 14) << 23)};
}

// x - h[i], in one instruction.  x may come straight from a matrix instruction:
// the conversion that made h has read it before, and has waited for it.
template <int I>
__device__ __forceinline__ float less_half(float x, half2 h) {
  float d;
  if constexpr (I == 0)
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(d) : "v"(h), "v"(x));
  else
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d) : "v"(h), "v"(x));
  return d;
}

// Eight fp32 values as halves of 11 bits each.
__device__ __forceinline__ void split(const float4v& a, const float4v& b, half8& hi, half8& lo) {
  half2 h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = i < 2 ? a[2 * i] : b[2 * i - 4], y = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
    h[i] = to_half2(x, y);
    l[i] = to_half2(less_half<0>(x, h[i]), less_half<1>(y, h[i]));
  }
  hi = half8{h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
  lo = half8{l[0][0], l[0][1], l[1][0], l[1][1], l[2][0], l[2][1], l[3][0], l[3][1]};
}
// 2^x.  The integer part by itself: in fp32 2^-90 would be good to 2^-18.
__device__ __forceinline__ float exp2_of(double x) {
  const double whole = rint(x);
  return __builtin_ldexpf(__builtin_amdgcn_exp2f(static_cast<float>(x - whole)), static_cast<int>(whole));
}

__device__ __forceinline__ int exponent(float v) { return static_cast<int>(__float_as_uint(v) >> 23 & 255); }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ void wait_for(const int* flag, int at_least) {
  while (__hip_atomic_load(flag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) < at_least)
    __builtin_amdgcn_s_sleep(1);
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}
__device__ __forceinline__ void publish(int* flag, int value) {
  __hip_atomic_store(flag, value, __ATOMIC_RELEASE, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// ------------------------------------------------------------------ prepare

// Sum over the KP / 8 lanes of a token's row (8 or 16 neighbours).
template <int KP>
__device__ __forceinline__ float row_sum(float v) {
  v += dpp<kQuadSwap1>(v);
  v += dpp<kQuadSwap2>(v);
  v += dpp<0x141>(v);                    // mirrored within 8 lanes
  if (KP == 128) v += dpp<0x140>(v);     // mirrored within 16 lanes
  return v;
}

// Swaps the 4 x 4 matrix that four registers of the lanes l, l + 16, l + 32
// and l + 48 hold with its transpose.
__device__ __forceinline__ void transpose4(uint32_t (&r)[4]) {
  const auto a = __builtin_amdgcn_permlane32_swap(r[0], r[2], false, false);
  const auto b = __builtin_amdgcn_permlane32_swap(r[1], r[3], false, false);
  const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  r[0] = c[0];
  r[1] = c[1];
  r[2] = d[0];
  r[3] = d[1];
}

// The 32 rows of k or q of a block: a lane loads eight elements (depths 8 c ..)
// of the tokens 4 lp + l / 16, where c = l % (KP / 8) and lp = kPer i + (l % 16)
// / (KP / 8) in load i, so that the lanes l, l + 16, l + 32, l + 48 hold four
// consecutive tokens.
template <int KP, typename TIn>
struct Rows {
  static constexpr int kLanes = KP / 8;
  static constexpr int kPer = 16 / kLanes;
  static constexpr int kLoads = 8 / kPer;
  static constexpr int kWords = sizeof(TIn) == 4 ? 2 : 1;
  uint4v raw[kLoads][kWords];

  // `first`: the lane's offset in load 0, kDropOffset for lanes beyond K; rows
  // past `rows` lie past the buffer's end and read as zeros
  __device__ __forceinline__ void load(const TIn* base, uint32_t first, uint32_t row_bytes, int K, int rows) {
    const __amdgpu_buffer_rsrc_t r =
        make_rsrc(base, (rows - 1) * row_bytes + K * static_cast<uint32_t>(sizeof(TIn)));
    // the loads' offsets are cheaper made than kept
    asm volatile("" : "+v"(first));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
#pragma unroll
      for (int w = 0; w < kWords; ++w)
        raw[i][w] = __builtin_bit_cast(
            uint4v, __builtin_amdgcn_raw_buffer_load_b128(r, first + 4 * kPer * i * row_bytes + 16 * w, 0, 0));
    }
  }
  static __device__ __forceinline__ uint32_t lane_offset(uint32_t row_bytes, int K) {
    const int lane = threadIdx.x % 64, c = lane % kLanes;
    if (8 * c >= K) return kDropOffset;
    return (4 * (lane % 16 / kLanes) + lane / 16) * row_bytes + 8 * c * static_cast<uint32_t>(sizeof(TIn));
  }
  __device__ __forceinline__ void values(int i, float (&v)[8]) const {
    if constexpr (sizeof(TIn) == 4) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(raw[i][j / 4][j % 4]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(raw[i][0][j] << 16);
        v[2 * j + 1] = __uint_as_float(raw[i][0][j] & 0xffff0000u);
      }
    }
  }
  // sum of the squares of the lane's eight elements of load i
  __device__ __forceinline__ float squares(int i, const float (&v)[8]) const {
    float sq = 0.f;
    if constexpr (sizeof(TIn) == 4) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sq += v[j] * v[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x2 pair = __builtin_bit_cast(bf16x2, static_cast<uint32_t>(raw[i][0][j]));
        sq = __builtin_amdgcn_fdot2_f32_bf16(pair, pair, sq, false);
      }
    }
    return sq;
  }
};

// A row's power of two: its norm times `up` is in [2^-1/2, 2^1/2).
__device__ __forceinline__ Scale row_scale(float sq) {
  int half_e = static_cast<int>(__float_as_uint(sq) >> 24 & 127);
  half_e = half_e < 1 ? 1 : half_e;
  return {__uint_as_float(static_cast<uint32_t>(127 + 63 - half_e) << 23),
          __uint_as_float(static_cast<uint32_t>(127 - 63 + half_e) << 23)};
}
// What a row's operand lacks: that power of two, over the norm where the row is
// to be normalised.
__device__ __forceinline__ float row_factor(float sq, int norm, float eps) {
  const float down = row_scale(sq).down;
  return norm ? down * __builtin_amdgcn_rsqf(sq + eps) : down;
}

// Rows as operands in LDS (and, for keys, transposed ones), and every token's
// sum of squares.
template <int KP, bool IN32, bool TRANSPOSE, typename TIn, typename Frags, typename FragsT>
__device__ __forceinline__ void make_operand(const Rows<KP, TIn>& rows, Frags& frags, FragsT& turned, float* squares) {
  using R = Rows<KP, TIn>;
  const int lane = fresh_lane(), c = lane % R::kLanes, row = lane / 16;
#pragma unroll
  for (int i = 0; i < R::kLoads; ++i) {
    const int lp = R::kPer * i + lane % 16 / R::kLanes;
    float v[8];
    rows.values(i, v);
    const float sq = row_sum<KP>(rows.squares(i, v));
    const float up = row_scale(sq).up;
    if (c == 0) squares[4 * lp + row] = sq;
    uint32_t word[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = v[2 * j] * up, y = v[2 * j + 1] * up;
      const half2 h = to_half2(x, y);
      word[0][j] = __builtin_bit_cast(uint32_t, h);
      if (IN32)
        word[1][j] = __builtin_bit_cast(
            uint32_t, to_half2(less_half<0>(x, h), less_half<1>(y, h)));
    }
    const int tile = lp / 4, m = 4 * (lp % 4) + row, q = c % 4;
#pragma unroll
    for (int s = 0; s < (IN32 ? 2 : 1); ++s) {
      // the fragment's 16-byte slots are permuted by q: the 16 lanes of a row
      // of keys, a quarter of a kilobyte apart, write to different banks
      frags[s][tile][c / 4][q * 16 + (m ^ 4 * q)] =
          __builtin_bit_cast(half8, uint4v{word[s][0], word[s][1], word[s][2], word[s][3]});
      if (TRANSPOSE) {
        transpose4(word[s]);
        // now tokens 4 lp .. + 3 of the depths 8 c + 2 row and the next one
        const uint2v even = {__builtin_amdgcn_perm(word[s][1], word[s][0], 0x05040100),
                             __builtin_amdgcn_perm(word[s][3], word[s][2], 0x05040100)};
        const uint2v odd = {__builtin_amdgcn_perm(word[s][1], word[s][0], 0x07060302),
                            __builtin_amdgcn_perm(word[s][3], word[s][2], 0x07060302)};
        // state row 32 p + 8 n + 4 h + r is row 4 n + r of row tile 2 p + h
        const int rt = 2 * (c / 4) + row / 2, rm = 4 * (c % 4) + row % 2 * 2;
        uint2v* at = reinterpret_cast<uint2v*>(&turned[s][rt][lp % 4 * 16 + rm]) + lp / 4;
        at[0] = even;
        at[2] = odd;
      }
    }
  }
}

// What a prepare wave reads of a block, on its way.
template <int KP, int OUT, typename TIn>
struct Inputs {
  Rows<KP, TIn> k, q;
  float g, beta;
  int rows;

  // Block c of the sequence.
  __device__ __forceinline__ void load(const DeltaParams& p, Span span, int c, int hk, int h, uint32_t k_off,
                                       uint32_t q_off) {
    const int64_t first = span.begin + static_cast<int64_t>(c) * kBlockTokens, left = span.end - first;
    rows = left < kBlockTokens ? static_cast<int>(left) : kBlockTokens;
    const int64_t head = static_cast<int64_t>(hk) * p.K;
    k.load(static_cast<const TIn*>(p.k) + first * p.k_stride + head, k_off,
           static_cast<uint32_t>(p.k_stride * sizeof(TIn)), p.K, rows);
    if (OUT)
      q.load(static_cast<const TIn*>(p.q) + first * p.q_stride + head, q_off,
             static_cast<uint32_t>(p.q_stride * sizeof(TIn)), p.K, rows);
    g = beta = 0.f;
    const int lane = threadIdx.x % 64;
    if (lane < rows) {
      const int64_t th = (first + lane) * p.Hv + h;
      if (p.g != nullptr) g = p.g[th];
      beta = p.beta != nullptr ? p.beta[th] : 1.f;
    }
  }
};

// A block's operands from its inputs, once the buffer is free; `next` is called
// when the inputs' registers are.
template <int KP, bool IN32, int OUT, typename TIn, typename Next>
__device__ __forceinline__ void prepare_block(const DeltaParams& p, Inputs<KP, OUT, TIn>& in, Scratch& s,
                                              Buffer<KP, IN32, OUT>& buf, const int* done, int waves, int free_at,
                                              Next next) {
  constexpr int kSteps = KP / 32;
  int lane = fresh_lane();
  constexpr bool outputs = OUT != kNoOutput;
  for (int w = 0; w < waves; ++w) wait_for(&done[w], free_at);

  double b = static_cast<double>(in.g < kDeltaErase ? kDeltaErase : in.g);
#pragma unroll
  for (int d = 1; d < kBlockTokens; d <<= 1) {
    const double up = __shfl_up(b, d, kBlockTokens);
    if (lane % kBlockTokens >= d) b += up;
  }
  make_operand<KP, IN32, true, TIn>(in.k, buf.k, buf.kt, s.rk);
  if constexpr (outputs) make_operand<KP, IN32, false, TIn>(in.q, buf.q, buf.kt, s.rq);
  wave_fence();
  // lane l has token l % 32 (a token behind the last one has no key and no query;
  // a key of zeros has no length either, so its value does not reach X, unless it is
  // to be divided by a zero)
  const bool live = lane % kBlockTokens < in.rows;
  const float sq = s.rk[lane % kBlockTokens];
  const float length = row_factor(sq, p.norm, p.eps);
  const float rk = live && (sq != 0.f || length == __builtin_inff()) ? length : 0.f;
  const float rq = live && outputs ? row_factor(s.rq[lane % kBlockTokens], p.norm, p.eps) : 0.f;
  const double b2 = b * 1.4426950408889634;
  const float gate = in.beta * rk;
  if (lane < kBlockTokens) {
    s.b[lane] = static_cast<float>(b2);
    s.b_low[lane] = static_cast<float>(b2 - static_cast<double>(s.b[lane]));
    s.beta[lane] = in.beta * rk * rk;
  }
  next();
  wave_fence();

  lane = fresh_lane();
  int m = lane % 16, q = lane / 16;
  // k_i.k_j and q_i.k_j with i in the lanes and j = 4 q + r in the registers
  float4v kk[3] = {}, qk[3] = {};  // tiles (0, 0), (1, 0), (1, 1)
#pragma unroll
  for (int st = 0; st < kSteps; ++st) {
    const int at = q * 16 + (m ^ 4 * q);
    half8 kf[2], qf[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      kf[t] = buf.k[0][t][st][at];
      if (outputs) qf[t] = buf.q[0][t][st][at];
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) kk[i] = mfma(kf[i / 2], kf[i > 0], kk[i]);
    if (outputs) {
#pragma unroll
      for (int i = 0; i < 3; ++i) qk[i] = mfma(kf[i / 2], qf[i > 0], qk[i]);
    }
    if (IN32) {
      half8 kl[2], ql[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        kl[t] = buf.k[Buffer<KP, IN32, OUT>::kHalves - 1][t][st][at];
        if (outputs) ql[t] = buf.q[Buffer<KP, IN32, OUT>::kHalves - 1][t][st][at];
      }
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        kk[i] = mfma(kl[i / 2], kf[i > 0], kk[i]);
        kk[i] = mfma(kf[i / 2], kl[i > 0], kk[i]);
        if (outputs) {
          qk[i] = mfma(kl[i / 2], qf[i > 0], qk[i]);
          qk[i] = mfma(kf[i / 2], ql[i > 0], qk[i]);
        }
      }
    }
  }
  float* const A = reinterpret_cast<float*>(&buf.t);
  float4v pm[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int ti = i > 0, tj = i / 2, row = 16 * ti + m, cols = 16 * tj + 4 * q;
    const float bi = s.b[row], bi_low = s.b_low[row], ri = s.beta[row];
    const float4v bj = *reinterpret_cast<const float4v*>(&s.b[cols]);
    const float4v bj_low = *reinterpret_cast<const float4v*>(&s.b_low[cols]);
    float4v a;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float d = (bi - bj[r]) + (bi_low - bj_low[r]);
      const float decay = __builtin_amdgcn_exp2f(ti > tj || row >= cols + r ? d : -__builtin_inff());
      const float v = ri * (decay * kk[i][r]);
      a[r] = ti > tj || row > cols + r ? v : 0.f;
      pm[i][r] = decay * qk[i][r];
    }
    *reinterpret_cast<float4v*>(&A[a_at(i, m, 4 * q)]) = a;
  }
  if constexpr (outputs) {
#pragma unroll
    for (int i = 0; i < 3; ++i) buf.p[0][i][lane] = pm[i];
  }
  wave_fence();

  lane = fresh_lane();
  m = lane % 16;
  q = lane / 16;
  // (I + A)^-1 of the two diagonal 16 x 16 blocks: lane l has column l % 16 of
  // block l / 16 (the upper lanes repeat the lower ones)
  const uint32_t diagonal = 2 * (q & 1);
  float col[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float sum = i == m ? 1.f : 0.f;
#pragma unroll
    for (int j4 = 0; j4 < (i + 3) / 4; ++j4) {
      const float4v a = *reinterpret_cast<const float4v*>(&A[a_at(diagonal, i, 4 * j4)]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (4 * j4 + j < i) sum -= a[j] * col[4 * j4 + j];
    }
    col[i] = sum;
    // rows' loads are not drawn further ahead than this: they would fill the
    // registers that the next block's inputs arrive in
    if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
  }
  wave_fence();
  if (lane < 32) {
#pragma unroll
    for (int i = 0; i < 16; ++i) A[a_at(diagonal, i, m)] = col[i];
  }
  wave_fence();
  lane = fresh_lane();
  m = lane % 16;
  q = lane / 16;
  // the lower left one: -T22 A21 T11, in fp32
  float4v y = {}, z = {};
#pragma unroll
  for (int st = 0; st < 4; ++st)
    y = mfma(A[a_at(1, m, 4 * st + q)], A[a_at(0, 4 * st + q, m)], y);
  const float4v t22 = *reinterpret_cast<const float4v*>(&A[a_at(2, m, 4 * q)]);
#pragma unroll
  for (int st = 0; st < 4; ++st) z = mfma(t22[st], y[st], z);
  wave_fence();
#pragma unroll
  for (int r = 0; r < 4; ++r) A[a_at(1, 4 * q + r, m)] = -z[r];
  wave_fence();
  {
    const float4v t11 = *reinterpret_cast<const float4v*>(&A[a_at(0, m, 4 * q)]);
    const float4v t21 = *reinterpret_cast<const float4v*>(&A[a_at(1, m, 4 * q)]);
    wave_fence();  // A has been read
    buf.t[0][lane] = t11;
    buf.t[1][lane] = t21;
    buf.t[2][lane] = t22;
    const float fo = p.scale * rq;
    const float eb = exp2_of(b2);
    const float fu = exp2_of(readlane_d(b2, kBlockTokens - 1) - b2);
    if (lane < kBlockTokens) {
      buf.f.v[lane] = gate;
      buf.f.x[lane] = gate * rk * eb;
      buf.f.u[lane] = fu;
      buf.f.q[lane] = fo * eb;
      buf.f.o[lane] = fo;
      if (lane == kBlockTokens - 1) buf.f.decay = eb;
    }
  }
  wave_fence();
}

// -------------------------------------------------------------------- chain

// NV neighbouring elements at a byte offset of a buffer, and NV results to one.
template <typename T, int NV>
__device__ __forceinline__ void load_cols(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t (&raw)[2]) {
  constexpr int kBytes = static_cast<int>(sizeof(T)) * NV;
  if constexpr (kBytes == 2) {
    raw[0] = static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0));
  } else if constexpr (kBytes == 4) {
    raw[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0));
  } else {
    const uint2v v = __builtin_bit_cast(uint2v, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0));
    raw[0] = v[0];
    raw[1] = v[1];
  }
}
template <typename T>
__device__ __forceinline__ float col_value(const uint32_t (&raw)[2], int n) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(raw[n]);
  if constexpr (std::is_same_v<T, f16_t>) return widen(f16_t{static_cast<uint16_t>(raw[0] >> 16 * n)});
  return __uint_as_float(n ? raw[0] & 0xffff0000u : raw[0] << 16);
}
template <typename T, int NV>
__device__ __forceinline__ void store_cols(__amdgpu_buffer_rsrc_t r, uint32_t off, const float (&v)[NV]) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (NV == 1)
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[0]), r, off, 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b64(uint2v{__float_as_uint(v[0]), __float_as_uint(v[1])}, r, off, 0, 0);
  } else {
    if constexpr (NV == 1)
      __builtin_amdgcn_raw_buffer_store_b16(narrow<T>(v[0]).bits, r, off, 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b32(
          narrow<T>(v[0]).bits | static_cast<uint32_t>(narrow<T>(v[1]).bits) << 16, r, off, 0, 0);
  }
}

// A lower triangle times 32 tokens of 16 NV columns.
template <int NV>
__device__ __forceinline__ void by_lower(const Lower& a, int lane, const float4v (&x)[2][NV], float4v (&out)[2][NV]) {
  const float4v t00 = a[0][lane], t10 = a[1][lane], t11 = a[2][lane];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      out[0][n] = mfma(t00[r], x[0][n][r], out[0][n]);
      out[1][n] = mfma(t10[r], x[0][n][r], out[1][n]);
    }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int n = 0; n < NV; ++n) out[1][n] = mfma(t11[r], x[1][n][r], out[1][n]);
}

// The states of a wave's columns: row r of tile t is the state row 32 (t / 2) +
// 8 q + 4 (t % 2) + r, columns col .. col + NV - 1.  Rows from K on lie past the
// buffer's end: read as zeros, not written.
template <int KP, int NV, typename TSt>
__device__ __forceinline__ void load_state(const TSt* base, int V, int K, int col, float4v (&S)[NV][KP / 16]) {
  constexpr uint32_t kSize = sizeof(TSt);
  const __amdgpu_buffer_rsrc_t buf = make_rsrc(base, static_cast<uint32_t>(K * V) * kSize);
  const uint32_t at = col < V ? static_cast<uint32_t>(threadIdx.x % 64 / 16 * 8 * V + col) * kSize : kDropOffset;
#pragma unroll
  for (int t = 0; t < KP / 16; ++t) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      uint32_t raw[2];
      load_cols<TSt, NV>(buf, at + static_cast<uint32_t>((32 * (t / 2) + 4 * (t % 2) + r) * V) * kSize, raw);
#pragma unroll
      for (int n = 0; n < NV; ++n) S[n][t][r] = col_value<TSt>(raw, n);
    }
  }
}
template <int KP, int NV, typename TSt>
__device__ __forceinline__ void store_state(TSt* base, int V, int K, int col, const float4v (&S)[NV][KP / 16]) {
  constexpr uint32_t kSize = sizeof(TSt);
  const __amdgpu_buffer_rsrc_t buf = make_rsrc(base, static_cast<uint32_t>(K * V) * kSize);
  const uint32_t at = col < V ? static_cast<uint32_t>(threadIdx.x % 64 / 16 * 8 * V + col) * kSize : kDropOffset;
#pragma unroll
  for (int t = 0; t < KP / 16; ++t) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float v[NV];
#pragma unroll
      for (int n = 0; n < NV; ++n) v[n] = S[n][t][r];
      store_cols<TSt, NV>(buf, at + static_cast<uint32_t>((32 * (t / 2) + 4 * (t % 2) + r) * V) * kSize, v);
    }
  }
}

template <int KP, bool IN32, int OUT, int NV>
__global__ void __launch_bounds__(64 * (kChainMax + Shared<KP, IN32, OUT>::kPrepare))
    delta_kernel(DeltaParams p, int chain_waves, int state16) {
  using TIn = std::conditional_t<IN32, float, bf16_t>;
  using TOut = std::conditional_t<OUT == kOut32, float, bf16_t>;
  using Sh = Shared<KP, IN32, OUT>;
  using Buf = Buffer<KP, IN32, OUT>;
  constexpr int kSteps = KP / 32, kTiles = KP / 16, kLow = Buf::kHalves - 1;
  static_assert(sizeof(Sh) <= 160 * 1024, "LDS of a CU");
  __shared__ __align__(16) unsigned char lds[sizeof(Sh)];
  Sh& sh = *reinterpret_cast<Sh*>(lds);

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lane = threadIdx.x % 64, m = lane % 16, q = lane / 16;
  const int width = 16 * NV * chain_waves;
  const int vblocks = (p.V + width - 1) / width;
  // the heads that share keys follow one another, on one XCD
  const int at_block = xcd_remap(blockIdx.x, gridDim.x);
  const int column_blocks = vblocks + (p.phase == kSegmentEnds);
  const int segments = p.phase == kSegmentEnds ? p.segments - 1 : p.segments;
  const int vb = at_block % column_blocks;
  const int h = uniform(at_block / column_blocks % p.Hv);
  const int seg = uniform(at_block / column_blocks / p.Hv % segments);
  const int64_t b = uniform(at_block / column_blocks / p.Hv / segments);
  const bool phi = vb == vblocks;  // the columns of Phi, values of zero
  if (phi && seg == 0) return;     // the first segment starts from the given state
  Span span = sequence(p.starts, b, p.L, p.T);
  if (p.segments > 1) {
    const int first = static_cast<int>(span.begin), last = static_cast<int>(span.end);
    const int each = ((last - first + kBlockTokens - 1) / kBlockTokens + p.segments - 1) / p.segments;  // blocks
    const int64_t begin = first + static_cast<int64_t>(seg) * each * kBlockTokens, end = begin + each * kBlockTokens;
    span = {begin < last ? begin : last, end < last ? end : last};
  }
  span = {uniform(static_cast<int>(span.begin)), uniform(static_cast<int>(span.end))};
  const int blocks = static_cast<int>((span.end - span.begin + kBlockTokens - 1) / kBlockTokens);

  if (threadIdx.x < Sh::kBuffers) sh.ready[threadIdx.x] = 0;
  if (threadIdx.x < kChainMax) sh.done[threadIdx.x] = 0;
  __syncthreads();

  if (wave >= chain_waves) {
    const int hk = h / (p.Hv / p.Hk);
    const int self = wave - chain_waves;
    const uint32_t k_off = Rows<KP, TIn>::lane_offset(static_cast<uint32_t>(p.k_stride * sizeof(TIn)), p.K);
    const uint32_t q_off = Rows<KP, TIn>::lane_offset(static_cast<uint32_t>(p.q_stride * sizeof(TIn)), p.K);
    // a block's inputs are on their way while the one before is worked on, unless
    // they take 128 registers
    constexpr bool kAhead = !(IN32 && KP == 128);
    Inputs<KP, OUT, TIn> in;
    if (kAhead && self < blocks) in.load(p, span, self, hk, h, k_off, q_off);
    for (int c = self; c < blocks; c += Sh::kPrepare) {
      if (!kAhead) in.load(p, span, c, hk, h, k_off, q_off);
      prepare_block<KP, IN32, OUT, TIn>(p, in, sh.scratch[self], sh.buf[c % Sh::kBuffers], sh.done, chain_waves,
                                        c - Sh::kBuffers + 1, [&] {
                                          if (kAhead && c + Sh::kPrepare < blocks)
                                            in.load(p, span, c + Sh::kPrepare, hk, h, k_off, q_off);
                                        });
      publish(&sh.ready[c % Sh::kBuffers], c + 1);
    }
    return;
  }

  const int wave_col = (phi ? 0 : vb * width) + wave * 16 * NV, col = wave_col + m * NV;
  const int columns = phi ? p.K : p.V;
  if (wave_col >= columns) {  // no columns: the prepare waves need not wait
    publish(&sh.done[wave], 0x7fffffff);
    return;
  }
  const int64_t state_at = static_cast<int64_t>(h) * p.K * p.V;
  // state of slot `s` between the segments
  const auto between = [&](int s) {
    return p.between + ((b * p.segments + s) * p.Hv + h) * static_cast<int64_t>(p.K) * p.V;
  };
  float4v S[NV][kTiles] = {};
  if (p.phase == kSegments) {
    load_state<KP, NV>(between((seg + p.segments - 1) % p.segments), p.V, p.K, col, S);
  } else if (phi) {
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[n][t][r] = 32 * (t / 2) + 8 * q + 4 * (t % 2) + r == col + n ? 1.f : 0.f;
  } else if (seg == 0) {
    int64_t row = b;
    bool known = true;
    if (p.idx != nullptr) {
      row = p.idx[b];
      known = row >= 0 && row < p.state_rows;
    }
    if (!known) {
      const float nan = __builtin_nanf("");
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int t = 0; t < kTiles; ++t) S[n][t] = float4v{nan, nan, nan, nan};
    } else if (p.h0 != nullptr) {
      if (state16)
        load_state<KP, NV>(static_cast<const f16_t*>(p.h0) + row * p.h0_stride + state_at, p.V, p.K, col, S);
      else
        load_state<KP, NV>(static_cast<const float*>(p.h0) + row * p.h0_stride + state_at, p.V, p.K, col, S);
    }
  }

  const uint32_t v_step = static_cast<uint32_t>(p.v_stride * sizeof(TIn));
  const uint32_t o_step = static_cast<uint32_t>(static_cast<int64_t>(p.Hv) * p.V * sizeof(TOut));
  const uint32_t v_off = col < p.V && !phi ? static_cast<uint32_t>(col * sizeof(TIn)) + 4 * q * v_step : kDropOffset;
  const uint32_t o_off = col < p.V ? static_cast<uint32_t>(col * sizeof(TOut)) + 4 * q * o_step : kDropOffset;
  uint32_t raw[2][4][2];  // the block's values: tokens 16 t + 4 q + r
  const int tokens = static_cast<int>(span.end - span.begin);
  const TIn* v_at = static_cast<const TIn*>(p.v) + span.begin * p.v_stride + static_cast<int64_t>(h) * p.V;
  TOut* o_at = static_cast<TOut*>(p.o) + (span.begin * p.Hv + h) * p.V;
  // rows of block c
  const auto rows_of = [&](int c) {
    return static_cast<uint32_t>(min(tokens - c * kBlockTokens, kBlockTokens));
  };
  const auto fetch = [&](int c) {
    const __amdgpu_buffer_rsrc_t r =
        make_rsrc(v_at, (rows_of(c) - 1) * v_step + p.V * static_cast<uint32_t>(sizeof(TIn)));
    v_at += kBlockTokens * p.v_stride;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) load_cols<TIn, NV>(r, v_off + (16 * t + i) * v_step, raw[t][i]);
  };
  if (blocks > 0) fetch(0);

  // A column of S is held as S~ = S / sigma, sigma a power of two such that
  // |S~| < 2^16: its halves are fp16 numbers as they are.  `bound` >= |S~|.
  // A block multiplies S~ by decay sigma / sigma' and adds K^T (U / sigma'),
  // where 32 keys' elements below 2^1/2 meet |U / sigma'| < 2^8: sigma' is
  // chosen so that both terms stay below 2^14, from the largest element that U
  // has under its decays to the block's end (what a block wrote and has forgotten
  // by then sets no scale) and from S~'s bound.  The halves' floor of 2^-24 leaves
  // them 22 bits of the column's largest while that is above 2^-2; the bound of
  // S~, which can grow by 2^6 times U a block, is taken anew from S~ every eighth
  // block.  (Bounds of U that are known before it is, 32 |T| |X|, would take 2 %
  // of the time away and lost all of a state that a block's last tokens shrink by
  // 2^24.)
  float sigma[NV], bound[NV];
  const auto largest = [&](int n) {
    float most = 0.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) most = max_abs(most, S[n][t][r]);
    return max_of_rows(most);
  };
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const float most = largest(n);
    // (a sequence without tokens hands its state on bit for bit)
    const Scale sc = blocks > 0 ? scale_of(most) : Scale{1.f, 1.f};
    sigma[n] = sc.down;
    bound[n] = most * sc.up;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) S[n][t] *= sc.up;
  }

  for (int c = 0; c < blocks; ++c) {
    // the state as an operand
    half8 s_hi[NV][kSteps], s_lo[NV][kSteps];
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int st = 0; st < kSteps; ++st) split(S[n][2 * st], S[n][2 * st + 1], s_hi[n][st], s_lo[n][st]);
    const Buf& buf = sh.buf[c % Sh::kBuffers];
    wait_for(&sh.ready[c % Sh::kBuffers], c + 1);

    // K S, which the rest waits for, then Q S
    const int at = q * 16 + (m ^ 4 * q);
    float4v ks[2][NV] = {}, qs[2][NV] = {};
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const half8 kf = buf.k[0][t][st][at];
#pragma unroll
        for (int n = 0; n < NV; ++n) {
          ks[t][n] = mfma(kf, s_hi[n][st], ks[t][n]);
          ks[t][n] = mfma(kf, s_lo[n][st], ks[t][n]);
        }
        if (IN32) {
          const half8 kl = buf.k[kLow][t][st][at];
#pragma unroll
          for (int n = 0; n < NV; ++n) ks[t][n] = mfma(kl, s_hi[n][st], ks[t][n]);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (OUT) {
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const half8 qf = buf.q[0][t][st][at];
#pragma unroll
          for (int n = 0; n < NV; ++n) {
            qs[t][n] = mfma(qf, s_hi[n][st], qs[t][n]);
            qs[t][n] = mfma(qf, s_lo[n][st], qs[t][n]);
          }
          if (IN32) {
            const half8 ql = buf.q[kLow][t][st][at];
#pragma unroll
            for (int n = 0; n < NV; ++n) qs[t][n] = mfma(ql, s_hi[n][st], qs[t][n]);
          }
        }
      }
    }
    // X, then U = T X
    float4v u[2][NV] = {};
    {
      float4v x[2][NV];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float4v fx = *reinterpret_cast<const float4v*>(&buf.f.x[16 * t + 4 * q]);
        const float4v fv = *reinterpret_cast<const float4v*>(&buf.f.v[16 * t + 4 * q]);
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[t][n][r] = fv[r] * col_value<TIn>(raw[t][r], n) - fx[r] * sigma[n] * ks[t][n][r];
      }
      if (c + 1 < blocks) fetch(c + 1);
      by_lower<NV>(buf.t, lane, x, u);
    }
    // U / sigma' under its decays, for K^T
    half8 u_hi[NV], u_lo[NV];
    float next[NV], keep[NV];  // sigma', and the factor of S~
    {
      float4v fu[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) fu[t] = *reinterpret_cast<const float4v*>(&buf.f.u[16 * t + 4 * q]);
      const float decay = buf.f.decay;
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const float4v end[2] = {u[0][n] * fu[0], u[1][n] * fu[1]};
        float most = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) most = max_abs(most, end[t][r]);
        most = max_of_rows(most);
        // exponents of sigma' for U, for S~, and the least, where both vanish
        const int unit = exponent(sigma[n]);
        int e = exponent(most) - 7;
        e = max(e, exponent(bound[n] * decay) + unit - 127 - 13);
        e = max(e, exponent(decay) + unit - 127 - 64);
        e = min(max(e, 2), 252);
        next[n] = __uint_as_float(static_cast<uint32_t>(e) << 23);
        const float up = __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
        keep[n] = __builtin_ldexpf(decay, unit - e);
        bound[n] = bound[n] * keep[n] + 64.f * (most * up);
        split(end[0] * up, end[1] * up, u_hi[n], u_lo[n]);
      }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const half8 kf = buf.kt[0][t][lane];
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        S[n][t] *= keep[n];
        S[n][t] = mfma(kf, u_hi[n], S[n][t]);
        S[n][t] = mfma(kf, u_lo[n], S[n][t]);
        if (IN32) S[n][t] = mfma(buf.kt[kLow][t][lane], u_hi[n], S[n][t]);
      }
    }
    if (OUT) {
      const __amdgpu_buffer_rsrc_t ro =
          make_rsrc(o_at, (rows_of(c) - 1) * o_step + p.V * static_cast<uint32_t>(sizeof(TOut)));
      o_at += static_cast<int64_t>(kBlockTokens) * p.Hv * p.V;
      float4v pu[2][NV] = {};
      // not among the products that the next block waits for
      __builtin_amdgcn_sched_barrier(0);
      by_lower<NV>(buf.p[0], lane, u, pu);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float4v fq = *reinterpret_cast<const float4v*>(&buf.f.q[16 * t + 4 * q]);
        const float4v fo = *reinterpret_cast<const float4v*>(&buf.f.o[16 * t + 4 * q]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v[NV];
#pragma unroll
          for (int n = 0; n < NV; ++n)
            v[n] = fq[r] * (sigma[n] * qs[t][n][r]) + fo[r] * pu[t][n][r];
          store_cols<TOut, NV>(ro, o_off + (16 * t + r) * o_step, v);
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) sigma[n] = next[n];
    if (c % 8 == 7) {
#pragma unroll
      for (int n = 0; n < NV; ++n) bound[n] = largest(n);
    }
    publish(&sh.done[wave], c + 1);
  }

#pragma unroll
  for (int n = 0; n < NV; ++n)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) S[n][t] *= sigma[n];
  if (p.phase == kSegmentEnds) {
    if (phi)
      store_state<KP, NV>(p.phi + ((b * p.segments + seg) * p.Hv + h) * static_cast<int64_t>(p.K) * p.K, p.K, p.K, col, S);
    else
      store_state<KP, NV>(between(seg), p.V, p.K, col, S);
  } else if (p.hT != nullptr && seg == p.segments - 1) {
    if (state16)
      store_state<KP, NV>(static_cast<f16_t*>(p.hT) + b * p.hT_stride + state_at, p.V, p.K, col, S);
    else
      store_state<KP, NV>(static_cast<float*>(p.hT) + b * p.hT_stride + state_at, p.V, p.K, col, S);
  }
}

// The states between the segments of a sequence: slot j holds F_j (slot 0: the
// first segment's end from the given state) and gets the end of segment j,
// Phi_j S + F_j; the last slot gets the given state, which a state written in
// place may replace before the first segment has read it again.  A workgroup
// has 16 columns of one head, a wave 16 rows of them.
template <int KP>
__global__ void __launch_bounds__(4 * KP) join_kernel(DeltaParams p, int state16) {
  constexpr int kGroups = KP / 16;
  __shared__ float state[KP][17];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lane = threadIdx.x % 64, m = lane % 16, q = lane / 16;
  const int vblocks = (p.V + 15) / 16;
  const int at_block = xcd_remap(blockIdx.x, gridDim.x);  // a head's columns read one Phi
  const int head = at_block / vblocks;
  const int h = head % p.Hv;
  const int64_t b = head / p.Hv;
  const int col = at_block % vblocks * 16 + m;
  const int row = 16 * wave + 4 * q;  // the lane's rows of a result: row .. row + 3
  const int64_t size = static_cast<int64_t>(p.K) * p.V;
  const auto between = [&](int s) { return p.between + ((b * p.segments + s) * p.Hv + h) * size; };
  // rows from K on and columns from V on lie past a buffer's end: read as zeros,
  // not written
  const uint32_t f_off = col < p.V ? static_cast<uint32_t>(row * p.V + col) * 4 : kDropOffset;
  const auto rows_of = [&](const float* at) {
    const __amdgpu_buffer_rsrc_t buf = make_rsrc(at, static_cast<uint32_t>(size) * 4);
    float4v v;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      v[r] = __uint_as_float(
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_raw_buffer_load_b32(buf, f_off + 4 * r * p.V, 0, 0)));
    return v;
  };
  // row 16 wave + m of Phi_j, columns 16 g + 4 q ..
  const auto phi_of = [&](int j, float4v (&a)[kGroups]) {
    const __amdgpu_buffer_rsrc_t buf =
        make_rsrc(p.phi + ((b * p.segments + j) * p.Hv + h) * static_cast<int64_t>(p.K) * p.K,
                  static_cast<uint32_t>(p.K * p.K) * 4);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int c = 16 * g + 4 * q;
      const uint32_t off = c < p.K ? static_cast<uint32_t>((16 * wave + m) * p.K + c) * 4 : kDropOffset;
      a[g] = __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(buf, off, 0, 0));
    }
  };
  const auto put = [&](float* at, const float4v& v) {
    const __amdgpu_buffer_rsrc_t buf = make_rsrc(at, static_cast<uint32_t>(size) * 4);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[r]), buf, f_off + 4 * r * p.V, 0, 0);
  };
  {  // the given state
    int64_t from = b;
    bool known = true;
    if (p.idx != nullptr) {
      from = p.idx[b];
      known = from >= 0 && from < p.state_rows;
    }
    float4v v = {};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t at = from * p.h0_stride + h * size + static_cast<int64_t>(row + r) * p.V + col;
      if (!known)
        v[r] = __builtin_nanf("");
      else if (p.h0 != nullptr && row + r < p.K && col < p.V)
        v[r] = state16 ? widen(static_cast<const f16_t*>(p.h0)[at]) : static_cast<const float*>(p.h0)[at];
    }
    put(between(p.segments - 1), v);
  }
  // Phi and F are asked for two segments ahead
  struct Segment {
    float4v f, a[kGroups];
  } even = {}, odd = {};
  const auto load = [&](int j, Segment& to) {
    if (j + 1 >= p.segments) return;
    to.f = rows_of(between(j));
    phi_of(j, to.a);
  };
  float4v S = rows_of(between(0));
  const auto step = [&](int j, Segment& seg) {
#pragma unroll
    for (int r = 0; r < 4; ++r) state[row + r][m] = S[r];
    __syncthreads();
    S = seg.f;
    float4v more = {};  // two sums, so that a product does not wait for the one before
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        float4v& to = g % 2 ? more : S;
        to = mfma(seg.a[g][st], state[16 * g + 4 * q + st][m], to);
      }
    S += more;
    put(between(j), S);
    load(j + 2, seg);
    __syncthreads();
  };
  load(1, odd);
  load(2, even);
  for (int j = 1; j + 1 < p.segments; j += 2) {
    step(j, odd);
    if (j + 2 < p.segments) step(j + 1, even);
  }
}

template <int KP, bool IN32, int OUT, int NV>
hipError_t launch_typed(const DeltaParams& p, int chain_waves, int state16, hipStream_t s) {
  using Sh = Shared<KP, IN32, OUT>;
  const int width = 16 * NV * chain_waves;
  int64_t grid = p.B * p.Hv * ((p.V + width - 1) / width) * p.segments;
  if (p.phase == kSegmentEnds) grid = p.B * p.Hv * ((p.V + width - 1) / width + 1) * (p.segments - 1);
  delta_kernel<KP, IN32, OUT, NV>
      <<<dim3(static_cast<uint32_t>(grid)), 64 * (chain_waves + Sh::kPrepare), 0, s>>>(p, chain_waves, state16);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta(const DeltaParams& given, int in_dtype, int out_dtype, int state_dtype, int cus, hipStream_t s) {
  DeltaParams p = given;
  const int state16 = state_dtype == PRECOG_F16;
  // Columns of a workgroup: all of a head's, up to 128, or as few as leave every
  // workgroup a CU of its own (a block takes 3.7 us with 128 columns, 3.0 us with
  // 32, 2.0 us with 16; two rounds of narrower ones take longer than one).
  int nv = 2, waves = (p.V + 31) / 32;
  if (waves > kChainMax) waves = kChainMax;
  if (p.segments == 1) {
    const auto fits = [&](int width) { return p.B * p.Hv * ((p.V + width - 1) / width) <= cus; };
    while (waves > 1 && fits(32 * (waves / 2))) waves /= 2;
    if (waves == 1 && fits(16)) nv = 1;
  }
  const auto go = [&](auto kp, auto in32, auto out) {
    constexpr int KP = decltype(kp)::value, OUT = decltype(out)::value;
    constexpr bool IN32 = decltype(in32)::value;
    if (p.segments == 1) {
      p.phase = kWhole;
      return nv == 2 ? launch_typed<KP, IN32, OUT, 2>(p, waves, state16, s)
                     : launch_typed<KP, IN32, OUT, 1>(p, waves, state16, s);
    }
    p.phase = kSegmentEnds;
    const int phi_waves = (p.K + 31) / 32;
    hipError_t e = launch_typed<KP, IN32, kNoOutput, 2>(p, waves > phi_waves ? waves : phi_waves, state16, s);
    if (e != hipSuccess) return e;
    join_kernel<KP><<<dim3(static_cast<uint32_t>(p.B * p.Hv * ((p.V + 15) / 16))), 4 * KP, 0, s>>>(p, state16);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    p.phase = kSegments;
    return launch_typed<KP, IN32, OUT, 2>(p, waves, state16, s);
  };
  const auto sized = [&](auto in32, auto out) {
    return p.K <= 64 ? go(std::integral_constant<int, 64>{}, in32, out)
                     : go(std::integral_constant<int, 128>{}, in32, out);
  };
  const auto typed = [&](auto in32) {
    if (p.o == nullptr) return sized(in32, std::integral_constant<int, kNoOutput>{});
    return out_dtype == PRECOG_F32 ? sized(in32, std::integral_constant<int, kOut32>{})
                                   : sized(in32, std::integral_constant<int, kOut16>{});
  };
  return in_dtype == PRECOG_F32 ? typed(std::true_type{}) : typed(std::false_type{});
}

}  // namespace precog
