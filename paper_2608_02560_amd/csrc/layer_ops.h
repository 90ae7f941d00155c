// Conversions and vector accesses shared by the gated-delta layer's kernels.
// Internal to the library.
#pragma once

#include <hip/hip_runtime.h>

#include "layer_kernels.h"

namespace precog {
namespace {

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return __uint_as_float(static_cast<uint32_t>(v.bits) << 16); }
__device__ __forceinline__ float widen(f16_t v) { return static_cast<float>(__builtin_bit_cast(_Float16, v.bits)); }

// Round to nearest even.
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t narrow<bf16_t>(float v) {
  return bf16_t{__builtin_bit_cast(uint16_t, static_cast<__bf16>(v))};
}
template <> __device__ __forceinline__ f16_t narrow<f16_t>(float v) {
  return f16_t{__builtin_bit_cast(uint16_t, static_cast<_Float16>(v))};
}

// N consecutive elements as they lie in memory, loaded and stored with
// accesses of up to 16 bytes.  The address is a multiple of the smaller of 16
// bytes and the group.
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack {
  T v[N];
};
template <int N, typename T>
__device__ __forceinline__ Pack<T, N> load_pack(const T* at) {
  return *reinterpret_cast<const Pack<T, N>*>(at);
}
template <int N, typename T>
__device__ __forceinline__ void store_pack(T* at, const float (&f)[N]) {
  Pack<T, N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = narrow<T>(f[i]);
  *reinterpret_cast<Pack<T, N>*>(at) = r;
}

// Orders a wave's LDS accesses before and after it (other lanes' among them).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Begin and end of sequence b among T tokens: [b * L, (b + 1) * L), or the
// clamped [starts[b], starts[b + 1]); an end before its begin is empty.
struct Span {
  int64_t begin, end;
};
__device__ __forceinline__ int64_t clamp_token(int64_t t, int64_t T) { return t < 0 ? 0 : t > T ? T : t; }
__device__ __forceinline__ Span sequence(const int32_t* starts, int64_t b, int64_t L, int64_t T) {
  if (starts == nullptr) return {b * L, b * L + L};
  const int64_t begin = clamp_token(starts[b], T), end = clamp_token(starts[b + 1], T);
  return {begin, end < begin ? begin : end};
}

// The row of a step (precog_delta_step, precog_conv_step): whether a call's
// row b leads its slot's rows, and the next row of the same slot after `row`.
// Every thread of the workgroup calls these; `shared` is one int of LDS.
__device__ __forceinline__ bool leads_slot(const int32_t* slots, int64_t b, int32_t slot, int tid, int threads) {
  int earlier = 0;
  for (int64_t j = tid; j < b; j += threads) earlier |= slots[j] == slot;
  return __syncthreads_or(earlier) == 0;
}
__device__ __forceinline__ int64_t next_of_slot(const int32_t* slots, int64_t n, int64_t row, int32_t slot,
                                                int tid, int threads, int* shared) {
  int next = 0x7fffffff;
  for (int64_t j = row + 1 + tid; j < n; j += threads)
    if (slots[j] == slot) {
      next = static_cast<int>(j);
      break;
    }
  if (__syncthreads_or(next != 0x7fffffff) == 0) return -1;
  if (tid == 0) *shared = 0x7fffffff;
  __syncthreads();
  if (next != 0x7fffffff) atomicMin(shared, next);
  __syncthreads();
  next = *shared;
  __syncthreads();
  return next;
}

}  // namespace
}  // namespace precog
