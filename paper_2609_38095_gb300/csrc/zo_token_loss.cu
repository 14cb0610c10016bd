// zo_token_loss.cu -- a token's -log p of its target from its logits, and the
// sum over the tokens (zo_token_loss).
#include "zo_forward.cuh"

namespace zo {

namespace {

constexpr int kLossThreads = 256;
constexpr int kLossCtas = 5;     // per SM, by registers: with kLossVectors 80 KB in flight
constexpr int kLossVectors = 4;  // 16-byte loads in flight per thread
constexpr int kMaxParts = 8;     // CTAs of a cluster, where tokens are few
constexpr int kSumThreads = 1024;

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
  for (int i = tid; i < vectors; i += kLossVectors * kThreads) {
    uint4 raw[kLossVectors];
#pragma unroll
    for (int k = 0; k < kLossVectors; ++k) {
      raw[k] = make_uint4(none, none, none, none);
      if (i + k * kThreads < vectors) raw[k] = __ldcs(v + i + k * kThreads);
    }
    float f[kLossVectors * E];
#pragma unroll
    for (int k = 0; k < kLossVectors; ++k) Vec<T>::widen_all(raw[k], f + k * E);
    take<kLossVectors * E>(f, top, sum);
  }
}

// A token per CTA, or per cluster of CTAs that split the vocabulary where there
// are fewer tokens than the SMs hold CTAs. One pass with the running maximum
// and sum in registers; bound by HBM: each counted row is read once (3068 rows of
// 151936, bf16: 154 us = 6.05 TB/s).
template <typename T>
__global__ void __launch_bounds__(kLossThreads, kLossCtas)
    token_loss_kernel(const __grid_constant__ TokenLossParams p, int parts) {
  __shared__ float tops[kLossThreads / 32];
  __shared__ double sums[kLossThreads / 32];
  __shared__ float part_top;
  __shared__ float part_sum[2];  // high and low part
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the sum's CTA may come once every CTA here has begun
  const int64_t t = blockIdx.x / parts;
  const int rank = blockIdx.x % parts, tid = threadIdx.x;
  const int64_t target = load_index(p.targets, t, p.target64);
  if (target < 0 || target >= p.vocab) {
    if (rank == 0 && tid == 0) {
      p.rows[t] = target < 0 ? 0.0 : NAN;
      if (p.nll != nullptr) p.nll[t] = target < 0 ? 0.0f : NAN;
    }
    return;
  }
  const T* x = static_cast<const T*>(p.logits) + t * p.row;
  const int64_t from = p.vocab * rank / parts, to = p.vocab * (rank + 1) / parts;
  float top = kNone.top, sum = 0.0f;
  row_tail<T, kLossThreads>(x + from, static_cast<int>(to - from), tid, top, sum);
  Tail mine = lanes_join<32>({top, sum});
  if ((tid & 31) == 0) {
    tops[tid >> 5] = mine.top;
    sums[tid >> 5] = mine.sum;
  }
  __syncthreads();
  if (tid < 32) {
    constexpr int kWarps = kLossThreads / 32;
    mine = lanes_join<kWarps>(tid < kWarps ? Tail{tops[tid], sums[tid]} : kNone);
    if (tid == 0 && parts > 1) {
      part_top = mine.top;
      part_sum[0] = static_cast<float>(mine.sum);
      part_sum[1] = static_cast<float>(mine.sum - part_sum[0]);
    }
  }
  if (parts > 1) {
    cluster_sync();
    if (rank == 0 && tid < 32) {
      mine = kNone;
      if (tid < parts)
        mine = {peer_load(peer_address(&part_top, tid)),
                static_cast<double>(peer_load(peer_address(&part_sum[0], tid))) +
                    peer_load(peer_address(&part_sum[1], tid))};
      mine = lanes_join<kMaxParts>(mine);
    }
    cluster_sync();  // no CTA leaves before its part is read
  }
  if (rank == 0 && tid == 0) {
    const double nll = log(mine.sum) + (static_cast<double>(mine.top) - widen(x[target]));
    p.rows[t] = nll;
    if (p.nll != nullptr) p.nll[t] = static_cast<float>(nll);
  }
}

// A token per warp, for vocabularies of at most 4096: a CTA per token would come and go in more time than its row takes (4000
// rows of 2001, fp16: 21 us, with a CTA per token 41; the bytes alone 2.4).
template <typename T>
__global__ void __launch_bounds__(kLossThreads) token_loss_warp_kernel(const __grid_constant__ TokenLossParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kLossThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= p.tokens) return;
  const int64_t target = load_index(p.targets, t, p.target64);
  if (target < 0 || target >= p.vocab) {
    if (lane == 0) {
      p.rows[t] = target < 0 ? 0.0 : NAN;
      if (p.nll != nullptr) p.nll[t] = target < 0 ? 0.0f : NAN;
    }
    return;
  }
  const T* x = static_cast<const T*>(p.logits) + t * p.row;
  float top = kNone.top, sum = 0.0f;
  row_tail<T, 32>(x, static_cast<int>(p.vocab), lane, top, sum);
  const Tail all = lanes_join<32>({top, sum});
  if (lane == 0) {
    const double nll = log(all.sum) + (static_cast<double>(all.top) - widen(x[target]));
    p.rows[t] = nll;
    if (p.nll != nullptr) p.nll[t] = static_cast<float>(nll);
  }
}

// The tokens' sum in one CTA, in an order of their number alone. Launched so
// that it may be resident before the tokens' kernel has ended.
__global__ void __launch_bounds__(kSumThreads) token_loss_sum_kernel(const __grid_constant__ TokenLossParams p) {
  __shared__ double sums[kSumThreads / 32];
  __shared__ double counts[kSumThreads / 32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  double sum = 0.0, count = 0.0;
  for (int64_t t = threadIdx.x; t < p.tokens; t += blockDim.x) {
    sum += p.rows[t];
    if (p.flags & 1) count += load_index(p.targets, t, p.target64) >= 0 ? 1.0 : 0.0;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    count += __shfl_xor_sync(0xFFFFFFFFu, count, o);
  }
  if ((threadIdx.x & 31) == 0) {
    sums[threadIdx.x >> 5] = sum;
    counts[threadIdx.x >> 5] = count;
  }
  __syncthreads();
  if (threadIdx.x >= 32) return;
  sum = threadIdx.x < blockDim.x / 32 ? sums[threadIdx.x] : 0.0;
  count = threadIdx.x < blockDim.x / 32 ? counts[threadIdx.x] : 0.0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    count += __shfl_xor_sync(0xFFFFFFFFu, count, o);
  }
  if (threadIdx.x != 0) return;
  if (p.flags & 1) sum = count > 0.0 ? sum / count : NAN;
  if (p.flags & 4) {
    float* out = static_cast<float*>(p.loss);
    *out = static_cast<float>(p.flags & 2 ? *out + sum : sum);
  } else {
    double* out = static_cast<double*>(p.loss);
    *out = p.flags & 2 ? *out + sum : sum;
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

template <typename T>
cudaError_t launch_rows(const TokenLossParams& p, int sms, cudaStream_t stream) {
  if (p.vocab <= 4096) {
    constexpr int kRows = kLossThreads / 32;
    token_loss_warp_kernel<T><<<static_cast<unsigned>((p.tokens + kRows - 1) / kRows), kLossThreads, 0, stream>>>(p);
    return cudaGetLastError();
  }
  // as many parts as the SMs hold at once (100 rows of 151936, bf16: in 4 parts 12.8 us, in 8, two rounds, 17.5; 800 rows,
  // fp32: in one part 77 us, in two 89), none with less than 4096 logits
  int parts = 1;
  while (parts < kMaxParts && p.tokens * parts * 2 <= kLossCtas * sms && p.vocab / (parts * 2) >= 4096) parts *= 2;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = parts;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  return launch_with(token_loss_kernel<T>, static_cast<unsigned>(p.tokens * parts), kLossThreads, attr, stream, p,
                     parts);
}

}  // namespace

cudaError_t launch_token_loss(const TokenLossParams& p, int dtype, int sms, cudaStream_t stream) {
  if (p.tokens > 0) {
    const cudaError_t e = dtype == 0   ? launch_rows<float>(p, sms, stream)
                          : dtype == 1 ? launch_rows<__nv_bfloat16>(p, sms, stream)
                                       : launch_rows<__half>(p, sms, stream);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  const int64_t threads = p.tokens < kSumThreads ? (p.tokens + 31) / 32 * 32 : kSumThreads;
  return launch_with(token_loss_sum_kernel, 1, static_cast<unsigned>(threads > 0 ? threads : 32), attr, stream, p);
}

}  // namespace zo
