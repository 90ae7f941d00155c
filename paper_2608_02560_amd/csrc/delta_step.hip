// One token of each of many sessions through the gated delta rule: a workgroup
// keeps CT columns of one head's [K, V] state in registers for it.
//
//   u = beta (v - a S^T k),  S <- a S + k u^T,  o = scale (a S^T q + (k.q) u)
//
// with S the state before the token: S^T k and S^T q come out of one pass over
// the state and one reduction, and the state is read and written once, which is
// what bounds it: 96 sessions of 16 heads of 128 x 128 fp32 states, 201 MB, take
// 43 us, 4.7 TB/s, the rate of a large copy (35 us where they are in the cache).
#include "layer_ops.h"

namespace precog {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ void load_four(__amdgpu_buffer_rsrc_t r, uint32_t off, float (&f)[4]) {
  if constexpr (sizeof(T) == 4) {
    const uint4v v = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
#pragma unroll
    for (int c = 0; c < 4; ++c) f[c] = __uint_as_float(v[c]);
  } else {
    const uint2v v = __builtin_bit_cast(uint2v, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0));
#pragma unroll
    for (int c = 0; c < 4; ++c) f[c] = widen(T{static_cast<uint16_t>(v[c / 2] >> 16 * (c % 2))});
  }
}
template <typename T>
__device__ __forceinline__ void store_four(__amdgpu_buffer_rsrc_t r, uint32_t off, const float (&f)[4]) {
  if constexpr (sizeof(T) == 4) {
    __builtin_amdgcn_raw_buffer_store_b128(
        uint4v{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])}, r, off, 0, 0);
  } else {
    uint2v v;
#pragma unroll
    for (int c = 0; c < 2; ++c)
      v[c] = narrow<T>(f[2 * c]).bits | static_cast<uint32_t>(narrow<T>(f[2 * c + 1]).bits) << 16;
    __builtin_amdgcn_raw_buffer_store_b64(v, r, off, 0, 0);
  }
}

template <typename TIn, typename TOut, typename TSt, int CT>
__global__ void __launch_bounds__(kThreads) delta_step_kernel(DeltaParams p) {
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

  const int32_t slot = p.idx[b];
  if (slot < 0 || slot >= p.state_rows) return;
  if (!leads_slot(p.idx, b, slot, tid, kThreads)) return;
  // the head's state as a buffer: rows from K on lie past its end, read as zeros
  // and are not written
  constexpr uint32_t kSize = sizeof(TSt);
  const __amdgpu_buffer_rsrc_t state =
      make_rsrc(static_cast<TSt*>(p.hT) + slot * p.h0_stride + static_cast<int64_t>(h) * p.K * p.V,
                static_cast<uint32_t>(p.K * p.V) * kSize);
  const uint32_t at = on ? static_cast<uint32_t>(rg * p.V + col) * kSize : kDropOffset;
  const uint32_t step = static_cast<uint32_t>(kGroups * p.V) * kSize;
  float S[kRows][4];
#pragma unroll
  for (int i = 0; i < kRows; ++i) load_four<TSt>(state, at + i * step, S[i]);

  for (int64_t t = b;;) {  // this row, then the others of the slot
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
    // (expf, not 2^(g log2 e), whose rounded exponent is good to 2^-18 near -60)
    const float a = expf(gt), beta = p.beta != nullptr ? p.beta[th] : 1.f;
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
    t = next_of_slot(p.idx, p.B, t, slot, tid, kThreads, &next_row);
    if (t < 0) break;
    // as a call of its own would store and load the state
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) S[i][c] = widen(narrow<TSt>(S[i][c]));
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) store_four<TSt>(state, at + i * step, S[i]);
}

template <typename TIn, typename TOut, typename TSt>
hipError_t launch_typed(const DeltaParams& p, int cus, hipStream_t s) {
  // all 128 columns a workgroup where that leaves four of them a CU, else 32:
  // a single session's eight heads are 16 workgroups rather than 8
  const auto blocks = [&](int ct) { return static_cast<uint32_t>(p.B * p.Hv * ((p.V + ct - 1) / ct)); };
  if (blocks(128) >= 4u * cus)
    delta_step_kernel<TIn, TOut, TSt, 128><<<dim3(blocks(128)), kThreads, 0, s>>>(p);
  else
    delta_step_kernel<TIn, TOut, TSt, 32><<<dim3(blocks(32)), kThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_step(const DeltaParams& p, int in_dtype, int out_dtype, int state_dtype,
                             int cus, hipStream_t s) {
  const auto typed = [&](auto in, auto out) {
    using TIn = decltype(in);
    using TOut = decltype(out);
    return state_dtype == PRECOG_F32 ? launch_typed<TIn, TOut, float>(p, cus, s)
                                     : launch_typed<TIn, TOut, f16_t>(p, cus, s);
  };
  if (in_dtype == PRECOG_F32)
    return out_dtype == PRECOG_F32 ? typed(float{}, float{}) : typed(float{}, bf16_t{});
  return out_dtype == PRECOG_F32 ? typed(bf16_t{}, float{}) : typed(bf16_t{}, bf16_t{});
}

}  // namespace precog
