// zo_answer_losses.cu -- losses over a model's own answers: the clipped policy
// loss and the loss of preferred and rejected answers, with their gradients in
// the logits (zo_policy_loss, zo_preference_loss).
//
// Both are functions of the targets' log-probabilities alone, so the gradient
// of a row of logits is one number, the loss's slope by its log-probability,
// times 1[v = target] - p_v.
#include <algorithm>

#include "zo_logits.cuh"

namespace zo {

namespace {

constexpr int kSumThreads = 1024;
constexpr int kGradThreads = 256;

struct Term {
  float value, slope;
};

// expm1(d) - d: by its series where the difference would lose what is left of it.
__device__ __forceinline__ float expm1_less(float d) {
  if (fabsf(d) >= 0.25f) return expm1f(d) - d;
  const float c = fmaf(fmaf(fmaf(fmaf(1.0f / 5040.0f, d, 1.0f / 720.0f), d, 1.0f / 120.0f), d, 1.0f / 24.0f), d, 1.0f / 6.0f);
  return d * d * fmaf(c, d, 0.5f);
}

// A token's loss and its slope by its log-probability. With r = exp(logp - old):
// -min(r A, clip(r) A) + kl (exp(d) - 1 - d), d = ref - logp. A NaN stays one:
// each comparison is written so that it picks the side that is NaN.
__device__ __forceinline__ Term policy_term(const PolicyLossParams& p, int64_t t, double logp) {
  const float a = p.advantages[t], r = expf(static_cast<float>(logp - p.old_logp[t]));
  const float lo = 1.0f - p.clip_low, hi = 1.0f + p.clip_high;
  const float whole = r * a, cut = (r < lo ? lo : r > hi ? hi : r) * a;
  Term term = {whole > cut ? -cut : -whole, whole > cut ? 0.0f : -whole};
  if (p.ref_logp != nullptr) {
    const float d = static_cast<float>(p.ref_logp[t] - logp);
    term.value += p.kl * expm1_less(d);
    term.slope -= p.kl * expm1f(d);
  }
  return term;
}

// The tokens' terms and their sum, in one CTA and an order of their number alone.
__global__ void __launch_bounds__(kSumThreads) policy_sum_kernel(const __grid_constant__ PolicyLossParams p) {
  __shared__ double over;
  const TokenLossParams& r = p.rows;
  double weight = 0.0;
  if (r.flags & 1) {
    for (int64_t t = threadIdx.x; t < r.tokens; t += blockDim.x)
      if (load_index(r.targets, t, r.target64) >= 0) weight += p.weights != nullptr ? p.weights[t] : 1.0;
    const Sums all = cta_sums({weight, 0.0});
    if (threadIdx.x == 0) over = all.a != 0.0 ? 1.0 / all.a : NAN;
    __syncthreads();
  }
  const double unit = r.flags & 1 ? over : 1.0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  double sum = 0.0;
  for (int64_t t = threadIdx.x; t < r.tokens; t += blockDim.x) {
    const bool counts = load_index(r.targets, t, r.target64) >= 0;
    const double logp = -r.rows[t];
    Term term = {0.0f, 0.0f};
    if (counts) term = policy_term(p, t, logp);
    const double w = !counts ? 0.0 : p.weights != nullptr ? p.weights[t] : 1.0;
    if (counts) sum += w * term.value;
    if (p.logp != nullptr) p.logp[t] = counts ? static_cast<float>(logp) : 0.0f;
    if (p.slopes != nullptr) p.slopes[t] = counts ? static_cast<float>(w * unit * term.slope) : 0.0f;
  }
  const Sums all = cta_sums({sum, 0.0});
  if (threadIdx.x == 0) put_loss(r.loss, r.flags, r.flags & 1 ? all.a * unit : all.a);
}

// The sequences' sums, the pairs' losses and their sum, and each token's slope,
// in one CTA; a warp has a sequence.
__global__ void __launch_bounds__(kSumThreads) preference_sum_kernel(const __grid_constant__ PreferenceLossParams p) {
  __shared__ int unsorted;
  const TokenLossParams& r = p.rows;
  const int warps = blockDim.x / 32, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t sequences = 2 * p.pairs;
  if (threadIdx.x == 0) unsorted = 0;
  __syncthreads();
  for (int64_t j = threadIdx.x; j <= sequences; j += blockDim.x) {
    const int64_t at = p.starts[j];
    if (at < 0 || at > r.tokens || (j > 0 && p.starts[j - 1] > at)) unsorted = 1;
  }
  __syncthreads();
  const bool bad = unsorted != 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int64_t j = warp; j < sequences && !bad; j += warps) {
    double sum = 0.0, count = 0.0;
    for (int64_t t = p.starts[j] + lane; t < p.starts[j + 1]; t += 32)
      if (load_index(r.targets, t, r.target64) >= 0) {
        sum -= r.rows[t];
        count += 1.0;
      }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      count += __shfl_xor_sync(0xFFFFFFFFu, count, o);
    }
    if (lane == 0) p.sums[j] = p.by_length ? sum / fmax(count, 1.0) : sum;
  }
  __syncthreads();
  double loss = 0.0;
  const double over = r.flags & 1 ? 1.0 / p.pairs : 1.0;
  for (int64_t i = threadIdx.x; i < p.pairs; i += blockDim.x) {
    const double chosen = bad ? NAN : p.sums[2 * i], rejected = bad ? NAN : p.sums[2 * i + 1];
    double away = chosen - rejected;
    if (p.ref_logp != nullptr) away -= static_cast<double>(p.ref_logp[2 * i]) - p.ref_logp[2 * i + 1];
    const float m = static_cast<float>(p.beta * away - p.margin);
    // softplus(x) = max(x, 0) + log1p(exp(-|x|)), and its derivative
    const float e = expf(-fabsf(m)), tail = log1pf(e), small = e / (1.0f + e), large = 1.0f / (1.0f + e);
    const float up = m > 0.0f ? large : m <= 0.0f ? small : NAN, down = m > 0.0f ? small : m <= 0.0f ? large : NAN;
    loss += (1.0 - p.smoothing) * (fmaxf(-m, 0.0f) + tail) + p.smoothing * (fmaxf(m, 0.0f) + tail);
    if (p.logp != nullptr) {
      p.logp[2 * i] = static_cast<float>(chosen);
      p.logp[2 * i + 1] = static_cast<float>(rejected);
    }
    if (p.slopes != nullptr) {
      const double slope = over * p.beta * (p.smoothing * up - (1.0 - p.smoothing) * down);
      p.sums[2 * i] = slope;
      p.sums[2 * i + 1] = -slope;
    }
  }
  const Sums all = cta_sums({loss, 0.0});
  if (threadIdx.x == 0) put_loss(r.loss, r.flags, all.a * over);
  if (p.slopes == nullptr) return;
  __syncthreads();  // the slopes are in p.sums
  const int64_t first = bad ? 0 : p.starts[0], end = bad ? r.tokens : p.starts[sequences];
  for (int64_t t = threadIdx.x; t < r.tokens; t += blockDim.x)
    if (bad || t < first || t >= end)
      p.slopes[t] = load_index(r.targets, t, r.target64) >= 0 && bad ? NAN : 0.0f;
  for (int64_t j = warp; j < sequences && !bad; j += warps) {
    const int64_t from = p.starts[j], to = p.starts[j + 1];
    double count = 1.0;
    if (p.by_length) {
      count = 0.0;
      for (int64_t t = from + lane; t < to; t += 32) count += load_index(r.targets, t, r.target64) >= 0 ? 1.0 : 0.0;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) count += __shfl_xor_sync(0xFFFFFFFFu, count, o);
    }
    const float slope = static_cast<float>(p.sums[j] / fmax(count, 1.0));
    for (int64_t t = from + lane; t < to; t += 32) p.slopes[t] = load_index(r.targets, t, r.target64) >= 0 ? slope : 0.0f;
  }
}

// grad_v = slope scale (1[v = target] - exp(x_v - lse)). A CTA has kPerRow threads per row's part of kPart vectors. x - lse is
// formed from the row's maximum first, then from the rest in the product's rounding. Rows of slope 0 are not read. The target's own
// element is -expm1(x - lse), which 1 - p would lose where p is near 1.
template <typename T, int kPerRow>
__global__ void __launch_bounds__(kGradThreads) logits_grad_kernel(const __grid_constant__ LogitsGradParams p, int parts) {
  constexpr int E = Vec<T>::kN, kLoads = 4, kRows = kGradThreads / kPerRow;
  const int tid = threadIdx.x % kPerRow;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kPerRow;
  const int64_t t = item / parts, part = item - t * parts;
  if (t >= p.tokens) return;
  const T* x = static_cast<const T*>(p.logits) + t * p.row;
  T* g = static_cast<T*>(p.grad) + t * p.grad_row;
  const float slope = p.slopes[t];
  const int64_t target = load_index(p.targets, t, p.target64);
  const bool reads = slope != 0.0f;
  float2 lse = make_float2(0.0f, 0.0f);
  if (reads) lse = p.lse[t];
  const float times = slope * p.scale, low = -lse.y * kLog2e;
  const auto one = [&](float v, int64_t at) {
    if (!reads) return 0.0f;
    const float away = v - lse.x;
    return at == target ? times * -expm1f(away - lse.y) : -times * exp2_approx(fmaf(away, kLog2e, low));
  };
  const int64_t chunk = static_cast<int64_t>(kLoads) * kPerRow;
  const int off = static_cast<int>(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T));
  if (reinterpret_cast<uintptr_t>(g) % 16 / sizeof(T) != off) {  // no vector of one is a vector of the other
    const int64_t from = part * chunk * E, to = min(p.vocab, from + chunk * E);
    for (int64_t i = from + tid; i < to; i += kPerRow) g[i] = narrow<T>(one(reads ? widen(x[i]) : 0.0f, i));
    return;
  }
  const int64_t head = min(static_cast<int64_t>(off ? E - off : 0), p.vocab), vectors = (p.vocab - head) / E;
  const int64_t tail = head + vectors * E;
  if (part == 0) {
    if (tid < head) g[tid] = narrow<T>(one(reads ? widen(x[tid]) : 0.0f, tid));
    if (tid < p.vocab - tail) g[tail + tid] = narrow<T>(one(reads ? widen(x[tail + tid]) : 0.0f, tail + tid));
  }
  const uint4* xv = reinterpret_cast<const uint4*>(x + head);
  uint4* gv = reinterpret_cast<uint4*>(g + head);
  const int64_t from = part * chunk + tid;
  uint4 raw[kLoads];
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    raw[k] = make_uint4(0, 0, 0, 0);
    if (reads && from + k * kPerRow < vectors) raw[k] = __ldcs(xv + from + k * kPerRow);
  }
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    const int64_t i = from + k * kPerRow, first = head + i * E;
    if (i >= vectors) continue;
    float f[E];
    Vec<T>::widen_all(raw[k], f);
    const bool here = target >= first && target < first + E;
    float own = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (here && first + e == target) own = f[e];
      f[e] = reads ? -times * exp2_approx(fmaf(f[e] - lse.x, kLog2e, low)) : 0.0f;
    }
    if (here) {
      own = one(own, target);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (first + e == target) f[e] = own;
    }
    __stcs(gv + i, Vec<T>::narrow_all(f));
  }
}

template <typename T>
cudaError_t launch_grad(const LogitsGradParams& p, cudaStream_t stream) {
  constexpr int E = Vec<T>::kN;
  if (p.vocab <= 4096) {
    constexpr int kRows = kGradThreads / 32;
    const int parts = static_cast<int>((p.vocab + 128 * E - 1) / (128 * E));
    const int64_t grid = (p.tokens * parts + kRows - 1) / kRows;
    logits_grad_kernel<T, 32><<<static_cast<unsigned>(grid), kGradThreads, 0, stream>>>(p, parts);
  } else {
    constexpr int kPart = 4 * kGradThreads * E;
    const int parts = static_cast<int>((p.vocab + kPart - 1) / kPart);
    logits_grad_kernel<T, kGradThreads><<<static_cast<unsigned>(p.tokens * parts), kGradThreads, 0, stream>>>(p, parts);
  }
  return cudaGetLastError();
}

cudaError_t launch_logits_grad(const LogitsGradParams& p, int dtype, cudaStream_t stream) {
  if (p.tokens == 0) return cudaSuccess;
  return dtype == 0   ? launch_grad<float>(p, stream)
         : dtype == 1 ? launch_grad<__nv_bfloat16>(p, stream)
                      : launch_grad<__half>(p, stream);
}

template <typename F, typename P>
cudaError_t launch_sum(F kernel, const P& p, int64_t items, cudaStream_t stream) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = p.rows.tokens > 0;  // behind the rows' kernel; else behind the caller's
  const int64_t threads = items < kSumThreads ? (items + 31) / 32 * 32 : kSumThreads;
  return launch_with(kernel, 1, static_cast<unsigned>(threads > 0 ? threads : 32), attr, stream, p);
}

}  // namespace

cudaError_t launch_policy_loss(const PolicyLossParams& p, const LogitsGradParams* g, int dtype, int sms, cudaStream_t stream) {
  cudaError_t e = launch_token_rows(p.rows, dtype, sms, stream);
  if (e == cudaSuccess) e = launch_sum(policy_sum_kernel, p, p.rows.tokens, stream);
  if (e == cudaSuccess && g != nullptr) e = launch_logits_grad(*g, dtype, stream);
  return e;
}

cudaError_t launch_preference_loss(const PreferenceLossParams& p, const LogitsGradParams* g, int dtype, int sms,
                                   cudaStream_t stream) {
  cudaError_t e = launch_token_rows(p.rows, dtype, sms, stream);
  if (e == cudaSuccess) e = launch_sum(preference_sum_kernel, p, std::max(p.rows.tokens, 64 * p.pairs), stream);
  if (e == cudaSuccess && g != nullptr) e = launch_logits_grad(*g, dtype, stream);
  return e;
}

}  // namespace zo
