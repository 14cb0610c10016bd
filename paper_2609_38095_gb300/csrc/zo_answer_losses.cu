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
constexpr int kMaxParts = 8;      // CTAs of a cluster
constexpr int kWarpVocab = 4096;  // vocabularies up to which a warp has a row

// Sums here are pairs of fp32, the second what the first has lost: the fp64 units take 16 cycles for a warp's addition, and a
// CTA's joins of fp64 took more time than the rows they joined.
struct Pair {
  float high, low;
};
// a + b and the rounding error of that (Knuth, The Art of Computer Programming 2, 4.2.2).
__device__ __forceinline__ Pair two_sum(float a, float b) {
  const float s = __fadd_rn(a, b), bb = __fadd_rn(s, -a);
  const float error = __fadd_rn(__fadd_rn(a, -__fadd_rn(s, -bb)), __fadd_rn(b, -bb));
  return {s, fabsf(s) < kInf ? error : 0.0f};
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
  const Pair s = two_sum(a.high, b.high);
  return two_sum(s.high, __fadd_rn(s.low, __fadd_rn(a.low, b.low)));
}
__device__ __forceinline__ Pair operator-(Pair a) { return {-a.high, -a.low}; }
__device__ __forceinline__ Pair over(Pair a, float n) {
  const float q = __fdiv_rn(a.high, n);
  if (!(fabsf(q) < kInf)) return {q, 0.0f};
  return two_sum(q, __fdiv_rn(__fadd_rn(fmaf(-q, n, a.high), a.low), n));
}
__device__ __forceinline__ double wide(Pair a) { return static_cast<double>(a.high) + a.low; }
__device__ __forceinline__ Pair pair_of(float2 v) { return {v.x, v.y}; }

__device__ __forceinline__ Pair warp_sum(Pair s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    s = s + Pair{__shfl_xor_sync(0xFFFFFFFFu, s.high, o), __shfl_xor_sync(0xFFFFFFFFu, s.low, o)};
  return s;
}
// Over the CTA's threads, in an order of their number alone; on warp 0. The CTA comes to a barrier before it is called again.
__device__ __forceinline__ Pair cta_sum(Pair s) {
  __shared__ float2 warps[kSumThreads / 32];
  s = warp_sum(s);
  if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = make_float2(s.high, s.low);
  __syncthreads();
  if (threadIdx.x < 32) s = warp_sum(threadIdx.x < blockDim.x / 32 ? pair_of(warps[threadIdx.x]) : Pair{0.0f, 0.0f});
  return s;
}

// log of a sum: the mantissa's, at most 0.35, and the exponent's times log 2 = 355 / 512 - 2.1219444e-4, the first exactly (Cody
// and Waite, Software Manual for the Elementary Functions, 1980: the logarithm's argument reduction). The sum is fp32, and so is
// its logarithm's accuracy; the second part is there so that sums of many rows lose no more.
__device__ __forceinline__ Pair log_pair(float sum) {
  int e;
  float m = frexpf(sum, &e);
  if (!(sum > 0.0f && sum < kInf)) return {logf(sum), 0.0f};
  if (m < 0.70710678f) m *= 2.0f, --e;
  return two_sum(e * 0.693359375f, fmaf(static_cast<float>(e), -2.12194440e-4f, logf(m)));
}
// x - (top + rest)
__device__ __forceinline__ Pair logp_of(float x, float top, Pair rest) { return two_sum(x, -top) + -rest; }

struct Term {
  float value, slope;
};

// What a factor is multiplied with: where it is 0 and that is infinite, or beyond fp32, nothing (0 times it is NaN). A NaN stays one.
__device__ __forceinline__ float with_factor(float factor, float x) { return factor == 0.0f && fabsf(x) == kInf ? 0.0f : x; }

// expm1(d) - d: by its series where the difference would lose what is left of it.
__device__ __forceinline__ float expm1_less(float d) {
  if (fabsf(d) >= 0.25f) return expm1f(d) - d;
  const float c = fmaf(fmaf(fmaf(fmaf(1.0f / 5040.0f, d, 1.0f / 720.0f), d, 1.0f / 120.0f), d, 1.0f / 24.0f), d, 1.0f / 6.0f);
  return d * d * fmaf(c, d, 0.5f);
}

struct Token {  // what stands beside its logits
  float old_logp, advantage, ref_logp, weight;
  __device__ __forceinline__ Token(const PolicyLossParams& p, int64_t t)
      : old_logp(p.old_logp[t]),
        advantage(p.advantages[t]),
        ref_logp(p.ref_logp != nullptr ? p.ref_logp[t] : 0.0f),
        weight(p.weights != nullptr ? p.weights[t] : 1.0f) {}
  __device__ __forceinline__ Token() {}
};

// A token's loss and its slope by its log-probability. With r = exp(logp - old):
// -min(r A, clip(r) A) + kl (exp(d) - 1 - d), d = ref - logp. A NaN stays one:
// each comparison is written so that it picks the side that is NaN.
__device__ __forceinline__ Term policy_term(const PolicyLossParams& p, const Token& t, Pair logp) {
  const float a = t.advantage, r = expf((logp.high - t.old_logp) + logp.low);
  const float lo = 1.0f - p.clip_low, hi = 1.0f + p.clip_high;
  const float whole = with_factor(a, r) * a, cut = (r < lo ? lo : r > hi ? hi : r) * a;
  Term term = {whole > cut ? -cut : -whole, whole > cut ? 0.0f : -whole};
  if (p.ref_logp != nullptr) {
    const float d = (t.ref_logp - logp.high) - logp.low;
    term.value += p.kl * expm1_less(d);
    term.slope -= p.kl * expm1f(d);
  }
  return term;
}

__device__ __forceinline__ float token_slope(const Token& t, float unit, const Term& term) {
  return t.weight * unit * with_factor(t.weight, term.slope);
}

// 1 over the counted tokens' weights, on thread 0.
__device__ __forceinline__ float mean_unit(const PolicyLossParams& p) {
  const AnswerRows& r = p.rows;
  Pair weight = {0.0f, 0.0f};
#pragma unroll 4
  for (int64_t t = threadIdx.x; t < r.tokens; t += blockDim.x) {
    const float w = p.weights != nullptr ? p.weights[t] : 1.0f;
    if (load_index(r.targets, t, r.target64) >= 0) weight = weight + Pair{w, 0.0f};
  }
  weight = cta_sum(weight);
  return weight.high != 0.0f ? static_cast<float>(1.0 / wide(weight)) : NAN;
}

// The tokens' terms and their sum, in one CTA and an order of their number alone. What it costs is latency: what stands beside
// the logits is read ahead of the rows' sums, whether a token counts or not, and four tokens of a thread at once.
__global__ void __launch_bounds__(kSumThreads) policy_sum_kernel(const __grid_constant__ PolicyLossParams p) {
  __shared__ float shared_unit;
  constexpr int kAtOnce = 4;
  const AnswerRows& r = p.rows;
  Token token[kAtOnce];
  bool counts[kAtOnce];
  const auto read = [&](int64_t first) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int64_t t = first + k * static_cast<int64_t>(blockDim.x);
      counts[k] = false;
      if (t < r.tokens) {
        token[k] = Token(p, t);
        counts[k] = load_index(r.targets, t, r.target64) >= 0;
      }
    }
  };
  read(threadIdx.x);
  float unit = 1.0f;
  if (p.unit != nullptr) {
    unit = mean_unit(p);
    if (threadIdx.x == 0) shared_unit = unit;
    __syncthreads();
    unit = shared_unit;
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the gradient's kernel: the rows' CTAs are gone
  Pair sum = {0.0f, 0.0f};
  for (int64_t first = threadIdx.x; first < r.tokens; first += kAtOnce * static_cast<int64_t>(blockDim.x)) {
    if (first != threadIdx.x) read(first);
    Pair logp[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int64_t t = first + k * static_cast<int64_t>(blockDim.x);
      logp[k] = t < r.tokens ? pair_of(r.logp[t]) : Pair{0.0f, 0.0f};
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int64_t t = first + k * static_cast<int64_t>(blockDim.x);
      if (t >= r.tokens) continue;
      Term term = {0.0f, 0.0f};
      if (counts[k]) {
        term = policy_term(p, token[k], logp[k]);
        const float w = token[k].weight, value = with_factor(w, term.value), part = w * value;
        sum = sum + Pair{part, fabsf(part) < kInf ? fmaf(w, value, -part) : 0.0f};
      }
      if (p.logp != nullptr) p.logp[t] = logp[k].high;
      if (p.slopes != nullptr) p.slopes[t] = counts[k] ? token_slope(token[k], unit, term) : 0.0f;
    }
  }
  sum = cta_sum(sum);
  if (threadIdx.x == 0) put_loss(r.loss, r.flags, p.unit != nullptr ? wide(sum) * unit : wide(sum));
}

// The sequences' sums, the pairs' losses and their sum, and each token's slope, in one CTA. A sequence has one warp, or where
// there are few as many as it takes for all to have some; a token that does not count has a log-probability of 0 already.
__global__ void __launch_bounds__(kSumThreads) preference_sum_kernel(const __grid_constant__ PreferenceLossParams p) {
  __shared__ int unsorted;
  __shared__ float2 part_sum[kSumThreads / 32];
  __shared__ int part_count[kSumThreads / 32];
  const AnswerRows& r = p.rows;
  const int warps = blockDim.x / 32, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t sequences = 2 * p.pairs;
  int per = 1;  // warps of a sequence
  while (sequences > 0 && 2 * per * sequences <= warps) per *= 2;
  const int at_once = warps / per, mine = warp / per, share = warp - mine * per;  // sequences at once; the warp's, its place
  if (threadIdx.x == 0) unsorted = 0;
  __syncthreads();
  for (int64_t j = threadIdx.x; j <= sequences; j += blockDim.x) {
    const int64_t at = p.starts[j];
    if (at < 0 || at > r.tokens || (j > 0 && p.starts[j - 1] > at)) unsorted = 1;
  }
  __syncthreads();
  const bool bad = unsorted != 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the gradient's kernel: the rows' CTAs are gone
  for (int64_t first = 0; first < sequences && !bad; first += at_once) {
    const int64_t j = first + mine;
    Pair sum = {0.0f, 0.0f};
    int count = 0;
    if (j < sequences && mine < at_once) {
      const int64_t from = p.starts[j] + share * 32 + lane, to = p.starts[j + 1];
#pragma unroll 4
      for (int64_t t = from; t < to; t += per * 32) sum = sum + pair_of(r.logp[t]);
      if (p.by_length) {
#pragma unroll 4
        for (int64_t t = from; t < to; t += per * 32) count += load_index(r.targets, t, r.target64) >= 0;
      }
    }
    sum = warp_sum(sum);
    count = __reduce_add_sync(0xFFFFFFFFu, count);
    if (lane == 0) part_sum[warp] = make_float2(sum.high, sum.low), part_count[warp] = count;
    __syncthreads();
    if (j < sequences && mine < at_once && share == 0 && lane == 0) {
      for (int i = 1; i < per; ++i) sum = sum + pair_of(part_sum[warp + i]), count += part_count[warp + i];
      const float by = p.by_length && count > 1 ? static_cast<float>(count) : 1.0f;
      if (by > 1.0f) sum = over(sum, by);
      p.sums[j] = make_float2(sum.high, sum.low);
      p.counts[j] = by;
    }
    __syncthreads();
  }
  Pair loss = {0.0f, 0.0f};
  const float per_pair = r.flags & 1 ? 1.0f / static_cast<float>(p.pairs) : 1.0f;
  for (int64_t i = threadIdx.x; i < p.pairs; i += blockDim.x) {
    const Pair chosen = bad ? Pair{NAN, 0.0f} : pair_of(p.sums[2 * i]), rejected = bad ? Pair{NAN, 0.0f} : pair_of(p.sums[2 * i + 1]);
    Pair away = chosen + -rejected;
    if (p.ref_logp != nullptr) away = away + two_sum(p.ref_logp[2 * i + 1], -p.ref_logp[2 * i]);
    const float m = p.beta * with_factor(p.beta, away.high) - p.margin;
    // softplus(x) = max(x, 0) + log1p(exp(-|x|)), and its derivative
    const float e = expf(-fabsf(m)), tail = log1pf(e), small = e / (1.0f + e), large = 1.0f / (1.0f + e);
    const float up = m > 0.0f ? large : m <= 0.0f ? small : NAN, down = m > 0.0f ? small : m <= 0.0f ? large : NAN;
    // an answer that cannot be given makes one of the two infinite, which without smoothing has the factor 0
    const float right = 1.0f - p.smoothing, turned = p.smoothing;
    loss = loss + Pair{right * with_factor(right, fmaxf(-m, 0.0f) + tail), turned * with_factor(turned, fmaxf(m, 0.0f) + tail)};
    if (p.logp != nullptr) {
      p.logp[2 * i] = chosen.high;
      p.logp[2 * i + 1] = rejected.high;
    }
    if (p.slopes != nullptr) {
      const float slope = per_pair * p.beta * (turned * up - right * down);
      p.sums[2 * i] = make_float2(slope, 0.0f);
      p.sums[2 * i + 1] = make_float2(-slope, 0.0f);
    }
  }
  loss = cta_sum(loss);
  if (threadIdx.x == 0) put_loss(r.loss, r.flags, r.flags & 1 ? wide(loss) / static_cast<double>(p.pairs) : wide(loss));
  if (p.slopes == nullptr) return;
  __syncthreads();  // the slopes are in p.sums
  if (bad) {
    for (int64_t t = threadIdx.x; t < r.tokens; t += blockDim.x) p.slopes[t] = NAN;
    return;
  }
  // rows in no sequence, and the sequences' (whether they count: the gradient's kernel goes by that too)
  const int64_t begin = p.starts[0], end = p.starts[sequences];
  for (int64_t t = threadIdx.x; t < begin; t += blockDim.x) p.slopes[t] = 0.0f;
  for (int64_t t = end + threadIdx.x; t < r.tokens; t += blockDim.x) p.slopes[t] = 0.0f;
  for (int64_t j = mine; j < sequences && mine < at_once; j += at_once) {
    const float slope = p.sums[j].x / p.counts[j];
    for (int64_t t = p.starts[j] + share * 32 + lane; t < p.starts[j + 1]; t += per * 32) p.slopes[t] = slope;
  }
}

// The gradient of a row's logits in place of the logits: grad_v = slope scale (1[v = target] - exp(x_v - lse)). x - lse is formed
// from the row's maximum first, then from the rest in the product's rounding. The target's own element is -expm1(x - lse), 1 - p
// without the rounding of p. (Where all other logits together weigh less than 2^-24 of it the row's sum is 1 in fp32, and it is 0.)
struct Slope {
  float times, top, rest, low;  // slope scale; of lse; -rest log2(e)
  __device__ __forceinline__ Slope(float slope, float scale, float2 lse)
      : times(slope * scale), top(lse.x), rest(lse.y), low(-lse.y * kLog2e) {}
  __device__ __forceinline__ float other(float x) const { return -times * exp2_approx(fmaf(x - top, kLog2e, low)); }
  __device__ __forceinline__ uint64_t other2(float a, float b) const {
    const uint64_t y = fma2(add2(pack2(a, b), pack2(-top, -top)), pack2(kLog2e, kLog2e), pack2(low, low));
    return mul2(pack2(exp2_approx(low2(y)), exp2_approx(high2(y))), pack2(-times, -times));
  }
  __device__ __forceinline__ float target(float x) const { return times * -expm1f(x - top - rest); }
};

// Which elements of a row a CTA has: the vectors of 16 bytes between its boundaries in `parts` equal parts, the elements in
// front of them with the first part, those behind with the last.
template <typename T>
struct Part {
  static constexpr int E = Vec<T>::kN;
  int first;  // element of the first vector
  int vectors;
  int edge;  // this thread's element in front or behind, -1: none
  __device__ __forceinline__ Part(const T* x, int64_t n, int rank, int parts) {
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T));
    const int head = min(off ? E - off : 0, static_cast<int>(n)), all = (static_cast<int>(n) - head) / E, tail = head + all * E;
    const int each = (all + parts - 1) / parts, from = min(rank * each, all);
    first = head + from * E;
    vectors = min(each, all - from);
    edge = -1;
    if (rank == 0 && threadIdx.x < head) edge = threadIdx.x;
    if (rank == parts - 1 && threadIdx.x >= 32 && threadIdx.x - 32 < n - tail) edge = tail + threadIdx.x - 32;
  }
};

constexpr int kPartThreads = 256;

template <typename T>
__device__ __forceinline__ void fetch_part(const T* x, const Part<T>& part, uint4* to) {
  const uint4* from = reinterpret_cast<const uint4*>(x + part.first);
  for (int i = threadIdx.x; i < part.vectors; i += kPartThreads)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(to + i))),
                 "l"(from + i)
                 : "memory");
}

// Writes a part's gradient from its logits in shared memory (each thread reads what it has put there itself), or zeros.
template <typename T>
__device__ __forceinline__ void put_part(T* g, const Part<T>& part, const uint4* x, float edge, bool zero, const Slope& s,
                                         int64_t target) {
  constexpr int E = Vec<T>::kN;
  const int tid = threadIdx.x;
  if (part.edge >= 0) g[part.edge] = narrow<T>(zero ? 0.0f : part.edge == target ? s.target(edge) : s.other(edge));
  const int64_t at = target - part.first;  // the target's element among the part's, and its vector
  const int64_t here = at >= 0 ? at / E : -1;
  T* to = g + part.first;
  const bool vector = reinterpret_cast<uintptr_t>(to) % 16 == 0;
#pragma unroll 2
  for (int i = tid; i < part.vectors; i += kPartThreads) {
    float f[E] = {};
    if (!zero) {
      float w[E];
      Vec<T>::widen_all(x[i], w);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const uint64_t y = s.other2(w[e], w[e + 1]);
        f[e] = low2(y), f[e + 1] = high2(y);
      }
      if (here == i) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (at % E == e) f[e] = s.target(w[e]);
      }
    }
    if (vector) {
      __stcs(reinterpret_cast<uint4*>(to) + i, Vec<T>::narrow_all(f));
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) to[static_cast<int64_t>(i) * E + e] = narrow<T>(f[e]);
    }
  }
}

// A row's gradient from its slope and log-sum: parts of a row of up to 24 KB, eight CTAs per SM, so that one's loads cover
// another's arithmetic. Bound by HBM: rows read and written once (2598 rows of 151936, 1950 of them counted, bf16: 197 us =
// 7.0 TB/s). The rows go from the last to the first, since the last ones read for their sums may still be in L2 (310 us for
// the whole call, 308 since; from the first on 312; with the last 80 MB kept there by hints 305, but the sums' pass 2 % slower).
// Launched while the sums' kernel runs: what its first CTAs read of the logits is on its way before the slopes are there.
template <typename T>
__global__ void __launch_bounds__(kPartThreads) logits_grad_kernel(const __grid_constant__ LogitsGradParams p, int parts) {
  extern __shared__ __align__(16) uint4 tile[];
  const int64_t t = p.tokens - 1 - blockIdx.x / parts;
  const T* x = static_cast<const T*>(p.logits) + t * p.row;
  const Part<T> part(x, p.vocab, blockIdx.x % parts, parts);
  const int64_t target = load_index(p.targets, t, p.target64);
  float edge = 0.0f;
  if (target >= 0) {
    fetch_part(x, part, tile);
    if (part.edge >= 0) edge = widen(x[part.edge]);
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float slope = p.slopes[t];
  const float2 lse = p.lse[t];
  const bool zero = slope == 0.0f || target < 0;
  asm volatile("cp.async.wait_all;" ::: "memory");
  put_part(static_cast<T*>(p.grad) + t * p.grad_row, part, tile, edge, zero, Slope(slope, p.scale, lse), target);
}

// The same for vocabularies of at most 4096: a warp per row.
template <typename T>
__global__ void __launch_bounds__(kPartThreads) logits_grad_warp_kernel(const __grid_constant__ LogitsGradParams p) {
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kPartThreads / 32) + (threadIdx.x >> 5);
  if (t >= p.tokens) return;
  const T* x = static_cast<const T*>(p.logits) + t * p.row;
  T* g = static_cast<T*>(p.grad) + t * p.grad_row;
  const int64_t target = load_index(p.targets, t, p.target64);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float slope = p.slopes[t];
  const bool zero = slope == 0.0f || target < 0;
  const Slope s(slope, p.scale, p.lse[t]);
  for (int64_t i = threadIdx.x & 31; i < p.vocab; i += 32) {
    const float v = zero ? 0.0f : widen(x[i]);
    g[i] = narrow<T>(zero ? 0.0f : i == target ? s.target(v) : s.other(v));
  }
}

template <typename T>
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (__is_same(T, __nv_bfloat16)) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// take() of vectors; 16-bit values are compared as they are, two at a time. (Where both are NaN the larger is one, and so the sum.)
template <typename T, int N>
__device__ __forceinline__ void take_raw(const uint4 (&raw)[N], float& top, float& sum) {
  constexpr int E = Vec<T>::kN;
  float most;
  if constexpr (sizeof(T) == 4) {
    most = __uint_as_float(raw[0].x);
#pragma unroll
    for (int k = 0; k < N; ++k)
      most = fmaxf(fmaxf(fmaxf(most, __uint_as_float(raw[k].x)), __uint_as_float(raw[k].y)),
                   fmaxf(__uint_as_float(raw[k].z), __uint_as_float(raw[k].w)));
  } else {
    uint32_t m = raw[0].x;
#pragma unroll
    for (int k = 0; k < N; ++k) m = max2<T>(max2<T>(max2<T>(m, raw[k].x), raw[k].y), max2<T>(raw[k].z, raw[k].w));
    const T* two = reinterpret_cast<const T*>(&m);
    most = fmaxf(widen(two[0]), widen(two[1]));
  }
  if (most > top) {
    sum *= exp2_approx((top - most) * kLog2e);
    top = most;
  }
  const uint64_t away = pack2(-top, -top), unit = pack2(kLog2e, kLog2e);
  uint64_t s[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float f[E];
    Vec<T>::widen_all(raw[k], f);
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const uint64_t d = mul2(add2(pack2(f[i], f[i + 1]), away), unit);
      s[i / 2 & 1] = add2(s[i / 2 & 1], pack2(exp2_approx(low2(d)), exp2_approx(high2(d))));
    }
  }
  const uint64_t all = add2(s[0], s[1]);
  sum += low2(all) + high2(all);
}

// lanes_join in fp32, for sums of some hundred values: the fp64 units would take as long for the joins of a part as the fp32
// units for the part.
template <int kLanes>
__device__ __forceinline__ void lanes_join_f32(float& top, float& sum) {
  float all = top;
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xFFFFFFFFu, all, o));
  sum *= exp2_approx((top - all) * kLog2e);
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  top = all;
}

// A row's maximum and sum over the CTA's threads and its cluster's CTAs, on warp 0. The caller waits for the cluster's barrier
// before it leaves: its part may be read until then.
__device__ __forceinline__ void join_rows(float& top, float& sum, int parts) {
  constexpr int kWarps = kPartThreads / 32;
  __shared__ float tops[kWarps];
  __shared__ float sums[kWarps];
  __shared__ float part_top, part_sum;
  const int tid = threadIdx.x;
  lanes_join_f32<32>(top, sum);
  if ((tid & 31) == 0) {
    tops[tid >> 5] = top;
    sums[tid >> 5] = sum;
  }
  __syncthreads();
  if (tid < 32) {
    top = tid < kWarps ? tops[tid] : kNone.top;
    sum = tid < kWarps ? sums[tid] : 0.0f;
    lanes_join_f32<kWarps>(top, sum);
    if (tid == 0) part_top = top, part_sum = sum;
    __syncwarp();
  }
  if (parts > 1) {
    if (tid < 32) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    else asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (tid < 32) {
      top = tid < parts ? peer_load(peer_address(&part_top, tid)) : kNone.top;
      sum = tid < parts ? peer_load(peer_address(&part_sum, tid)) : 0.0f;
      lanes_join_f32<kMaxParts>(top, sum);
      __syncwarp();
    }
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // its peers' parts are read
  }
}

// The rows' log-probabilities and log-sums: a CTA per counted row, or a cluster that splits the vocabulary where rows are few.
// Bound by HBM: each counted row is read once (3069 rows of 151936, bf16: 147 us a call = 6.3 TB/s; six loads a thread in flight and
// four CTAs per SM instead of four and five: the same, and 16 rows in 11.3 us instead of 10.5).
template <typename T>
__global__ void __launch_bounds__(kPartThreads, 5) row_sums_kernel(const __grid_constant__ AnswerRows r, int parts) {
  constexpr int kLoads = 4;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, rank = static_cast<int>(cluster_rank());
  const int64_t t = blockIdx.x / static_cast<unsigned>(parts), target = load_index(r.targets, t, r.target64);
  if (target < 0 || target >= r.vocab) {  // the same for the whole cluster
    if (rank == 0 && tid == 0) r.logp[t] = make_float2(target < 0 ? 0.0f : NAN, 0.0f), r.lse[t] = make_float2(0.0f, 0.0f);
    return;
  }
  const T* x = static_cast<const T*>(r.logits) + t * r.row;
  const Part<T> part(x, r.vocab, rank, parts);
  float own = 0.0f, edge = 0.0f, top = kNone.top, sum = 0.0f;
  if (rank == 0 && tid == 0) own = widen(x[target]);
  if (part.edge >= 0) edge = widen(x[part.edge]);
  const uint4* v = reinterpret_cast<const uint4*>(x + part.first);
  constexpr uint32_t kNothing = sizeof(T) == 4 ? 0xFF800000u : __is_same(T, __nv_bfloat16) ? 0xFF80FF80u : 0xFC00FC00u;  // -inf
  for (int i = tid; i < part.vectors; i += kLoads * kPartThreads) {
    uint4 raw[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      raw[k] = make_uint4(kNothing, kNothing, kNothing, kNothing);
      if (i + k * kPartThreads < part.vectors) raw[k] = __ldg(v + i + k * kPartThreads);
    }
    take_raw<T>(raw, top, sum);
  }
  if (part.edge >= 0) take<1>(&edge, top, sum);
  join_rows(top, sum, parts);
  if (rank == 0 && tid == 0) {
    const Pair rest = log_pair(sum), logp = logp_of(own, top, rest);
    r.logp[t] = make_float2(logp.high, logp.low);
    r.lse[t] = make_float2(top, rest.high);
  }
  if (parts > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}

// The same for vocabularies of at most 4096: a warp per row.
template <typename T>
__global__ void __launch_bounds__(kPartThreads) row_sums_warp_kernel(const __grid_constant__ AnswerRows r) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kPartThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= r.tokens) return;
  const int64_t target = load_index(r.targets, t, r.target64);
  if (target < 0 || target >= r.vocab) {
    if (lane == 0) r.logp[t] = make_float2(target < 0 ? 0.0f : NAN, 0.0f), r.lse[t] = make_float2(0.0f, 0.0f);
    return;
  }
  const T* x = static_cast<const T*>(r.logits) + t * r.row;
  float top = kNone.top, sum = 0.0f;
  row_tail<T, 32>(x, static_cast<int>(r.vocab), lane, top, sum);
  lanes_join_f32<32>(top, sum);
  if (lane == 0) {
    const Pair rest = log_pair(sum), logp = logp_of(widen(x[target]), top, rest);
    r.logp[t] = make_float2(logp.high, logp.low);
    r.lse[t] = make_float2(top, rest.high);
  }
}

// A row's sum, its token's term and its gradient with the row read once: a cluster of CTAs holds it in shared memory, up to 52
// KB each, four or five per SM, as long as eight of them hold it (rows of up to 416 KB); beyond, up to 200 KB each and fewer per
// SM (151936 logits in fp32: 76 KB, two). A thread fetches by cp.async what it alone reads, so that a part has no barrier but the joins';
// the slope's chain (joins, logarithm, exponential, a mean's weight) is on one thread of each CTA while the others' loads are on
// their way. Bound by HBM, with the instructions at 64 % of their slots (4091 tokens of 151936, 3069 of them counted, bf16: 357
// us = 6.1 TB/s of the 2.18 GB that have to move; the rows' sums and then the gradient 466; CTAs that take several rows and fetch
// the next row into places as they come free 430, by the instructions that this takes).
template <typename T>
__global__ void __launch_bounds__(kPartThreads, 5) policy_rows_kernel(const __grid_constant__ PolicyLossParams p,
                                                                      const __grid_constant__ LogitsGradParams g, int parts) {
  extern __shared__ __align__(16) uint4 tile[];
  __shared__ float shared_slope;
  __shared__ float2 shared_lse;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const AnswerRows& r = p.rows;
  const int tid = threadIdx.x, rank = static_cast<int>(cluster_rank());
  const int64_t t = blockIdx.x / static_cast<unsigned>(parts), target = load_index(r.targets, t, r.target64);
  const T* x = static_cast<const T*>(r.logits) + t * r.row;
  T* grad = static_cast<T*>(g.grad) + t * g.grad_row;
  const Part<T> part(x, r.vocab, rank, parts);
  const bool counts = target >= 0;
  if (!counts || target >= r.vocab) {  // the same for the whole cluster
    const float nan = NAN;
    if (rank == 0 && tid == 0) r.logp[t] = make_float2(counts ? NAN : 0.0f, 0.0f);
    put_part(grad, part, tile, nan, !counts, Slope(nan, 1.0f, make_float2(0.0f, 0.0f)), -1);
    if (p.unit != nullptr) asm volatile("griddepcontrol.wait;" ::: "memory");  // what follows may count on the kernel before
    return;
  }
  fetch_part(x, part, tile);
  float edge = 0.0f, own = 0.0f;
  if (part.edge >= 0) edge = widen(x[part.edge]);
  Token token;
  if (tid == 0) {
    own = widen(x[target]);
    token = Token(p, t);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  float top = kNone.top, sum = 0.0f;
  if (part.edge >= 0) take<1>(&edge, top, sum);
  int i = tid;
  for (; i + 3 * kPartThreads < part.vectors; i += 4 * kPartThreads) {
    uint4 raw[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) raw[k] = tile[i + k * kPartThreads];
    take_raw<T>(raw, top, sum);
  }
  for (; i < part.vectors; i += kPartThreads) {
    const uint4 raw[1] = {tile[i]};
    take_raw<T>(raw, top, sum);
  }
  join_rows(top, sum, parts);
  if (tid == 0) {
    const Pair rest = log_pair(sum), logp = logp_of(own, top, rest);
    if (rank == 0) r.logp[t] = make_float2(logp.high, logp.low);
    const Term term = policy_term(p, token, logp);
    float unit = 1.0f;
    if (p.unit != nullptr) {
      asm volatile("griddepcontrol.wait;" ::: "memory");
      unit = __ldcg(p.unit);
    }
    shared_slope = token_slope(token, unit, term);
    shared_lse = make_float2(top, rest.high);
  }
  __syncthreads();
  const float slope = shared_slope;
  put_part(grad, part, tile, edge, slope == 0.0f, Slope(slope, g.scale, shared_lse), target);
  if (parts > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}

// What a mean's weights are multiplied by.
__global__ void __launch_bounds__(kSumThreads) policy_unit_kernel(const __grid_constant__ PolicyLossParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const float unit = mean_unit(p);
  if (threadIdx.x == 0) *p.unit = unit;
}

template <typename T>
cudaError_t launch_grad(const LogitsGradParams& p, cudaStream_t stream) {
  constexpr int kRows = kPartThreads / 32, kMost = 24 * 1024;
  const int64_t bytes = p.vocab * static_cast<int64_t>(sizeof(T));
  const int parts = static_cast<int>((bytes + kMost - 1) / kMost);
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.blockDim = dim3(kPartThreads);
  c.stream = stream;
  c.attrs = &attr;
  c.numAttrs = 1;
  if (p.vocab <= kWarpVocab) {
    c.gridDim = dim3(static_cast<unsigned>((p.tokens + kRows - 1) / kRows));
    return cudaLaunchKernelEx(&c, logits_grad_warp_kernel<T>, p);
  }
  c.gridDim = dim3(static_cast<unsigned>(p.tokens * parts));
  c.dynamicSmemBytes = static_cast<size_t>((bytes / parts + 31) / 16 * 16);
  return cudaLaunchKernelEx(&c, logits_grad_kernel<T>, p, parts);
}

cudaError_t launch_logits_grad(const LogitsGradParams& p, int dtype, cudaStream_t stream) {
  if (p.tokens == 0) return cudaSuccess;
  return dtype == 0   ? launch_grad<float>(p, stream)
         : dtype == 1 ? launch_grad<__nv_bfloat16>(p, stream)
                      : launch_grad<__half>(p, stream);
}

cudaLaunchAttribute clusters_of(int parts) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = parts;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  return attr;
}

template <typename T>
cudaError_t launch_sums(const AnswerRows& r, int sms, cudaStream_t stream) {
  if (r.vocab <= kWarpVocab) {
    constexpr int kRows = kPartThreads / 32;
    row_sums_warp_kernel<T><<<static_cast<unsigned>((r.tokens + kRows - 1) / kRows), kPartThreads, 0, stream>>>(r);
    return cudaGetLastError();
  }
  // as many parts as the SMs hold at once, none with less than 4096 logits
  int parts = 1;
  while (parts < kMaxParts && r.tokens * parts * 2 <= 5 * sms && r.vocab / (parts * 2) >= 4096) parts *= 2;
  return launch_with(row_sums_kernel<T>, static_cast<unsigned>(r.tokens * parts), kPartThreads, clusters_of(parts), stream, r, parts);
}

cudaError_t launch_row_sums(const AnswerRows& r, int dtype, int sms, cudaStream_t stream) {
  if (r.tokens == 0) return cudaSuccess;
  return dtype == 0   ? launch_sums<float>(r, sms, stream)
         : dtype == 1 ? launch_sums<__nv_bfloat16>(r, sms, stream)
                      : launch_sums<__half>(r, sms, stream);
}

constexpr int64_t kMostPart = 200 * 1024;

// Whether rows of that many bytes are taken at once: beyond the vocabularies that a warp takes, up to what a cluster holds.
bool rows_at_once(int64_t vocab, int64_t bytes) { return vocab > kWarpVocab && bytes <= kMaxParts * (kMostPart - 16); }

template <typename T>
cudaError_t launch_rows(const PolicyLossParams& p, const LogitsGradParams& g, int sms, cudaStream_t stream) {
  const int64_t bytes = g.vocab * static_cast<int64_t>(sizeof(T));
  int parts = 1;
  while (parts < kMaxParts &&
         (bytes / parts > 52 * 1024 || (g.tokens * parts * 2 <= 5 * sms && g.vocab / (parts * 2) >= 4096)))
    parts *= 2;
  const int tile = static_cast<int>((bytes / parts + 31) / 16 * 16);
  // the most that a call takes, not this one's: host threads share what is set here
  cudaError_t e = cudaFuncSetAttribute(policy_rows_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMostPart));
  if (e != cudaSuccess) return e;
  if (p.unit != nullptr) {
    policy_unit_kernel<<<1, kSumThreads, 0, stream>>>(p);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  cudaLaunchAttribute attr[2] = {};
  attr[0] = clusters_of(parts);
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(static_cast<unsigned>(g.tokens * parts));
  c.blockDim = dim3(kPartThreads);
  c.dynamicSmemBytes = tile;
  c.stream = stream;
  c.attrs = attr;
  c.numAttrs = p.unit != nullptr ? 2 : 1;
  return cudaLaunchKernelEx(&c, policy_rows_kernel<T>, p, g, parts);
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
  if (g != nullptr && g->tokens > 0 && rows_at_once(g->vocab, g->vocab * (dtype == 0 ? 4 : 2))) {
    PolicyLossParams at_once = p;
    at_once.slopes = nullptr;
    cudaError_t e = dtype == 0   ? launch_rows<float>(at_once, *g, sms, stream)
                    : dtype == 1 ? launch_rows<__nv_bfloat16>(at_once, *g, sms, stream)
                                 : launch_rows<__half>(at_once, *g, sms, stream);
    return e != cudaSuccess ? e : launch_sum(policy_sum_kernel, at_once, p.rows.tokens, stream);
  }
  cudaError_t e = launch_row_sums(p.rows, dtype, sms, stream);
  if (e == cudaSuccess) e = launch_sum(policy_sum_kernel, p, p.rows.tokens, stream);
  if (e == cudaSuccess && g != nullptr) e = launch_logits_grad(*g, dtype, stream);
  return e;
}

cudaError_t launch_preference_loss(const PreferenceLossParams& p, const LogitsGradParams* g, int dtype, int sms,
                                   cudaStream_t stream) {
  cudaError_t e = launch_row_sums(p.rows, dtype, sms, stream);
  if (e == cudaSuccess) e = launch_sum(preference_sum_kernel, p, std::max(p.rows.tokens, 64 * p.pairs), stream);
  if (e == cudaSuccess && g != nullptr) e = launch_logits_grad(*g, dtype, stream);
  return e;
}

}  // namespace zo
