// zo_logits.cuh -- what the losses over rows of logits share: a row's maximum
// and sum of exponentials in one pass, their joins, and launches with an
// attribute.
#pragma once

#include "zo_forward.cuh"

namespace zo {

constexpr int kRowVectors = 4;  // 16-byte loads in flight per thread

struct Tail {  // max and sum of exp(x - max)
  float top;
  double sum;
};

// The first kLanes lanes' tails as one, on each of them: the maxima first, so that a sum is scaled once; sums in fp64.
template <int kLanes>
__device__ __forceinline__ Tail lanes_join(Tail t) {
  float top = t.top;
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  double sum = t.sum * exp2_approx((t.top - top) * kLog2e);
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  return {top, sum};
}
constexpr Tail kNone = {-3.402823466e38f, 0.0};

// x joins a thread's running maximum and sum; n values at once. x - top, then
// times log2(e): the difference is formed before its rounding, so logits far
// from 0 (or all at the type's lowest value) lose nothing.
template <int N>
__device__ __forceinline__ void take(const float* x, float& top, float& sum) {
  float most = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) most = fmaxf(most, x[i]);
  if (most > top) {
    sum *= exp2_approx((top - most) * kLog2e);
    top = most;
  }
  if constexpr (N == 1) {
    sum += exp2_approx((x[0] - top) * kLog2e);
  } else {
    const uint64_t away = pack2(-top, -top), unit = pack2(kLog2e, kLog2e);
    uint64_t s = 0;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const uint64_t d = mul2(add2(pack2(x[i], x[i + 1]), away), unit);
      s = add2(s, pack2(exp2_approx(low2(d)), exp2_approx(high2(d))));
    }
    sum += low2(s) + high2(s);
  }
}

// n logits from x on by kThreads threads: 16-byte vectors between the boundaries, the ends one by one.
template <typename T, int kThreads>
__device__ __forceinline__ void row_tail(const T* x, int n, int tid, float& top, float& sum) {
  constexpr int E = Vec<T>::kN;
  const int off = static_cast<int>(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T));
  const int head = min(off ? E - off : 0, n), vectors = (n - head) / E, tail = head + vectors * E;
  if (tid < head) {
    const float one = widen(x[tid]);
    take<1>(&one, top, sum);
  }
  if (tid < n - tail) {
    const float one = widen(x[tail + tid]);
    take<1>(&one, top, sum);
  }
  const uint4* v = reinterpret_cast<const uint4*>(x + head);
  const uint32_t none = sizeof(T) == 4 ? 0xFF800000u : __is_same(T, __nv_bfloat16) ? 0xFF80FF80u : 0xFC00FC00u;  // -inf
  for (int i = tid; i < vectors; i += kRowVectors * kThreads) {
    uint4 raw[kRowVectors];
#pragma unroll
    for (int k = 0; k < kRowVectors; ++k) {
      raw[k] = make_uint4(none, none, none, none);
      if (i + k * kThreads < vectors) raw[k] = __ldcs(v + i + k * kThreads);
    }
    float f[kRowVectors * E];
#pragma unroll
    for (int k = 0; k < kRowVectors; ++k) Vec<T>::widen_all(raw[k], f + k * E);
    take<kRowVectors * E>(f, top, sum);
  }
}

// The loss to where the caller wants it (flags: 2 added to what is there, 4 fp32).
__device__ __forceinline__ void put_loss(void* loss, int flags, double sum) {
  if (flags & 4) {
    float* out = static_cast<float*>(loss);
    *out = static_cast<float>(flags & 2 ? *out + sum : sum);
  } else {
    double* out = static_cast<double*>(loss);
    *out = flags & 2 ? *out + sum : sum;
  }
}

template <typename F, typename... A>
cudaError_t launch_with(F f, unsigned grid, unsigned threads, cudaLaunchAttribute attr, cudaStream_t stream, A... a) {
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(grid);
  c.blockDim = dim3(threads);
  c.stream = stream;
  c.attrs = &attr;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, f, a...);
}

}  // namespace zo
