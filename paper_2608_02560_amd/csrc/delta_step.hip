// The gated delta rule token by token: one workgroup keeps CT columns of one
// head's [K, V] state in registers and applies its tokens in order.
//
//   u = beta (v - a S^T k),  S <- a S + k u^T,  o = scale (a S^T q + (k.q) u)
//
// with S the state before the token: S^T k and S^T q come out of one pass over
// the state and one reduction, and the state is read and written once.
#include "layer_ops.h"

namespace precog {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

template <typename TIn, typename TOut, typename TSt, int CT, bool STEP>
__global__ void __launch_bounds__(kThreads) delta_rows_kernel(DeltaParams p) {
  constexpr int kLanes = CT / 4;            // threads across the columns, four each
  constexpr int kGroups = kThreads / kLanes;  // row groups
  constexpr int kRows = kDeltaMaxK / kGroups;
  __shared__ float qk[2][kDeltaMaxK];
  __shared__ float red[kWaves][CT][2];
  __shared__ float red_kq[kWaves], red_sq[kWaves];
  __shared__ int next_row;

  const int tid = threadIdx.x, wave = tid / 64;
  const int blocks = (p.V + CT - 1) / CT;
  const int64_t bid = blockIdx.x;
  const int cb = static_cast<int>(bid % blocks);
  const int h = static_cast<int>(bid / blocks % p.Hv);
  const int64_t b = bid / blocks / p.Hv;
  const int hk = h / (p.Hv / p.Hk);
  const int cl = tid % kLanes, rg = tid / kLanes;
  const int col = cb * CT + 4 * cl;
  const bool on = col < p.V;

  int64_t row = b;
  bool known = true;
  if (p.idx != nullptr) {
    row = p.idx[b];
    known = row >= 0 && row < p.state_rows;
  }
  if (STEP) {
    if (!known) return;
    if (!leads_slot(p.idx, p.B, b, static_cast<int32_t>(row), tid, kThreads)) return;
  }
  const int64_t at = (static_cast<int64_t>(h) * p.K) * p.V + col;
  float S[kRows][4];
  const TSt* h0 = static_cast<const TSt*>(p.h0);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = rg + kGroups * i;
    const bool in = on && r < p.K;
    if (in && h0 != nullptr && known) {
      const Pack<TSt, 4> s = load_pack<4>(h0 + row * p.h0_stride + at + static_cast<int64_t>(r) * p.V);
#pragma unroll
      for (int c = 0; c < 4; ++c) S[i][c] = widen(s.v[c]);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) S[i][c] = known ? 0.f : __builtin_nanf("");
    }
  }

  const Span span = STEP ? Span{b, b + 1} : sequence(p.starts, b, p.L, p.T);
  int64_t t = span.begin;
  while (STEP ? t >= 0 : t < span.end) {
    __syncthreads();
    {  // waves 0 and 1 prepare k, waves 2 and 3 q
      const int which = tid / 128, i = tid % 128;
      float x = 0.f;
      if (i < p.K) {
        if (which == 0)
          x = widen(static_cast<const TIn*>(p.k)[t * p.k_stride + static_cast<int64_t>(hk) * p.K + i]);
        else if (p.o != nullptr)
          x = widen(static_cast<const TIn*>(p.q)[t * p.q_stride + static_cast<int64_t>(hk) * p.K + i]);
      }
      if (p.norm) {
        float sq = x * x;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sq += __shfl_xor(sq, m);
        if (tid % 64 == 0) red_sq[wave] = sq;
        __syncthreads();
        x /= sqrtf(red_sq[which * 2] + red_sq[which * 2 + 1] + p.eps);
      }
      qk[which][i] = x;
    }
    __syncthreads();
    float sk[4] = {}, sq[4] = {}, kq = 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const float kr = qk[0][rg + kGroups * i], qr = qk[1][rg + kGroups * i];
      kq += kr * qr;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        sk[c] += S[i][c] * kr;
        sq[c] += S[i][c] * qr;
      }
    }
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1) {
      kq += __shfl_xor(kq, m);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        sk[c] += __shfl_xor(sk[c], m);
        sq[c] += __shfl_xor(sq[c], m);
      }
    }
    if (tid % 64 < kLanes) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        red[wave][4 * cl + c][0] = sk[c];
        red[wave][4 * cl + c][1] = sq[c];
      }
      if (cl == 0) red_kq[wave] = kq;
    }
    __syncthreads();
    kq = (red_kq[0] + red_kq[1]) + (red_kq[2] + red_kq[3]);
    const int64_t th = t * p.Hv + h;
    float gt = p.g != nullptr ? p.g[th] : 0.f;
    gt = gt < kDeltaErase ? kDeltaErase : gt;
    const float a = __expf(gt), beta = p.beta != nullptr ? p.beta[th] : 1.f;
    float u[4], o[4];
    if (on) {
      const Pack<TIn, 4> v =
          load_pack<4>(static_cast<const TIn*>(p.v) + t * p.v_stride + static_cast<int64_t>(h) * p.V + col);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = 4 * cl + c;
        const float dk = (red[0][j][0] + red[1][j][0]) + (red[2][j][0] + red[3][j][0]);
        const float dq = (red[0][j][1] + red[1][j][1]) + (red[2][j][1] + red[3][j][1]);
        u[c] = beta * (widen(v.v[c]) - a * dk);
        o[c] = p.scale * (a * dq + kq * u[c]);
      }
      if (p.o != nullptr && rg == 0) store_pack<4>(static_cast<TOut*>(p.o) + th * p.V + col, o);
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const float kr = qk[0][rg + kGroups * i];
#pragma unroll
        for (int c = 0; c < 4; ++c) S[i][c] = a * S[i][c] + kr * u[c];
      }
    }
    if (STEP) {
      t = next_of_slot(p.idx, p.B, t, static_cast<int32_t>(row), tid, kThreads, &next_row);
      if (t >= 0)  // as a call of its own would store and load the state
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) S[i][c] = widen(narrow<TSt>(S[i][c]));
    } else {
      ++t;
    }
  }
  if (p.hT != nullptr && on) {
    TSt* hT = static_cast<TSt*>(p.hT) + (STEP ? row : b) * p.hT_stride + at;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = rg + kGroups * i;
      if (r < p.K) store_pack<4>(hT + static_cast<int64_t>(r) * p.V, S[i]);
    }
  }
}

template <typename TIn, typename TOut, typename TSt, bool STEP>
hipError_t launch_rows(const DeltaParams& p, int cus, hipStream_t s) {
  const auto blocks = [&](int ct) { return p.B * p.Hv * ((p.V + ct - 1) / ct); };
  if (blocks(128) >= 4LL * cus)
    delta_rows_kernel<TIn, TOut, TSt, 128, STEP><<<dim3(static_cast<uint32_t>(blocks(128))), kThreads, 0, s>>>(p);
  else
    delta_rows_kernel<TIn, TOut, TSt, 32, STEP><<<dim3(static_cast<uint32_t>(blocks(32))), kThreads, 0, s>>>(p);
  return hipGetLastError();
}

template <bool STEP>
hipError_t by_types(const DeltaParams& p, int in_dtype, int out_dtype, int state_dtype, int cus,
                    hipStream_t s) {
  const auto st = [&](auto in, auto out) {
    using TIn = decltype(in);
    using TOut = decltype(out);
    return state_dtype == PRECOG_F32 ? launch_rows<TIn, TOut, float, STEP>(p, cus, s)
                                     : launch_rows<TIn, TOut, f16_t, STEP>(p, cus, s);
  };
  if (in_dtype == PRECOG_F32)
    return out_dtype == PRECOG_F32 ? st(float{}, float{}) : st(float{}, bf16_t{});
  return out_dtype == PRECOG_F32 ? st(bf16_t{}, float{}) : st(bf16_t{}, bf16_t{});
}

}  // namespace

hipError_t launch_delta_step(const DeltaParams& p, int in_dtype, int out_dtype, int state_dtype,
                             int cus, hipStream_t s) {
  return by_types<true>(p, in_dtype, out_dtype, state_dtype, cus, s);
}

}  // namespace precog
