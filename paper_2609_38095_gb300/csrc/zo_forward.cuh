// zo_forward.cuh -- parameter blocks, launch wrappers and small device helpers
// of the forward point's operators (include/zo_forward.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace zo {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();

struct RotatePart {
  const void* in;
  void* out;
  const void* weight;
  int64_t in_token, in_head, out_page, out_token, out_head;
  int32_t weight_dtype, heads, rotate, slotted;
  int32_t slice;  // first of its slices of a token's heads
};

struct RotateParams {
  RotatePart part[3];
  int32_t n_parts, dim, rotary, interleaved, index64;
  int64_t tokens;
  const float* table;
  int64_t table_rows;
  const void* positions;
  const void* slots;
  int64_t n_slots, page_size;
  float eps;
};

struct AttentionParams {
  const void *q, *k, *v;
  void* out;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;
  int64_t q_tokens, k_tokens;
  int32_t heads, group, dim;  // group: query heads per key-value head
  const int32_t* spans;       // [3][q_tokens]
  float scale, softcap;
  const float* slopes;
  float* lse;
};

struct DecodeParams {
  const void *q, *k, *v;
  void* out;
  int64_t q_token, q_head, out_token, out_head;
  int64_t k_page, k_token, k_head, v_page, v_token, v_head;
  int64_t pages_stride, max_pages, n_pages;
  const int32_t *pages, *lengths;
  int32_t heads, kv_heads, group, dim, page_size;
  int32_t page_shift;   // log2 of page_size, -1 where it is no power of two
  int32_t head_blocks;  // CTAs (or clusters) per key-value head, by blocks of query heads
  float scale, softcap;
  const float* slopes;
  float* lse;
};

// Several rows per sequence, the nodes of a tree: row r of a key-value head is node r / group, query head r % group of its own.
// A sequence's stride is q_token and out_token, head_blocks is of blocks of rows, and the tree's keys are behind `lengths`.
struct DraftParams : DecodeParams {
  int64_t q_node, out_node;
  const int64_t* masks;
  int32_t drafts;
};

struct TokenLossParams {
  const void* logits;
  int64_t row, tokens, vocab;
  const void* targets;
  int32_t target64, flags;
  void* loss;
  float* nll;
  double* rows;  // a token's nll before its rounding
};

// Losses over answers: a row's statistics, from them its slope, from it the row's gradient.
struct AnswerRows {
  const void* logits;
  int64_t row, tokens, vocab;
  const void* targets;
  int32_t target64, flags;
  void* loss;
  float2* logp;  // a target's log-probability, high and low part; 0 for tokens that do not count
  float2* lse;   // a row's maximum, and what its log sum exp is above it
};

struct PolicyLossParams {
  AnswerRows rows;
  const float *old_logp, *advantages, *ref_logp, *weights;
  float clip_low, clip_high, kl;
  float* logp;
  float* unit;    // place for what a mean's weights are multiplied by; NULL: they are not
  float* slopes;  // of the loss by a token's log-probability; NULL without a gradient
};

struct PreferenceLossParams {
  AnswerRows rows;
  const int32_t* starts;
  int64_t pairs;
  const float* ref_logp;
  float beta, margin, smoothing;
  int32_t by_length;
  float* logp;
  float2* sums;   // [2 pairs] of the sequences' tokens, high and low part; then the loss's slopes by them
  float* counts;  // [2 pairs] what a sequence's sum is divided by
  float* slopes;  // of the loss by a token's log-probability, per token; NULL without a gradient
};

struct LogitsGradParams {
  const void* logits;
  void* grad;
  int64_t row, grad_row, tokens, vocab;
  const void* targets;
  int32_t target64;
  const float* slopes;
  const float2* lse;
  float scale;
};

cudaError_t launch_rotary_table(float* table, int64_t rows, int rotary, double base, double scale, int64_t original,
                                double low, double high, double magnitude, cudaStream_t stream);
cudaError_t launch_document_spans(const int32_t* q_starts, const int32_t* k_starts, const int32_t* prefix, int docs,
                                  int32_t* spans, int64_t tokens, cudaStream_t stream);
cudaError_t launch_rotate_heads(const RotateParams& p, int dtype, cudaStream_t stream);
cudaError_t launch_attention_tiles(const AttentionParams& p, int dtype, int sms, cudaStream_t stream);
// The same on the tensor cores, where type, head size, strides and alignment
// admit it (false: nothing was launched).
bool launch_attention_mma(const AttentionParams& p, int dtype, cudaStream_t stream, cudaError_t* e);
cudaError_t launch_decode_scalar(const DecodeParams& p, int64_t batch, int dtype, int sms, cudaStream_t stream);
bool launch_decode_mma(const DecodeParams& p, int64_t batch, int dtype, int sms, cudaStream_t stream, cudaError_t* e);
cudaError_t launch_draft_masks(const int32_t* parents, int64_t batch, int drafts, int64_t* masks, cudaStream_t stream);
cudaError_t launch_draft_scalar(const DraftParams& p, int64_t batch, int dtype, int sms, cudaStream_t stream);
// For many rows; work: draft_wide_work's bytes on 16 of them (0: not for these).
int64_t draft_wide_work(int64_t batch, int64_t rows, int dim, int dtype);
bool launch_draft_wide(const DraftParams& p, int64_t batch, int dtype, int sms, void* work, cudaStream_t stream, cudaError_t* e);
bool launch_draft_mma(const DraftParams& p, int64_t batch, int dtype, int sms, cudaStream_t stream, cudaError_t* e);
cudaError_t launch_token_loss(const TokenLossParams& p, int dtype, int sms, cudaStream_t stream);
cudaError_t launch_policy_loss(const PolicyLossParams& p, const LogitsGradParams* g, int dtype, int sms, cudaStream_t stream);
cudaError_t launch_preference_loss(const PreferenceLossParams& p, const LogitsGradParams* g, int dtype, int sms,
                                   cudaStream_t stream);

#ifdef __CUDACC__
__host__ __device__
#endif
inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

#ifdef __CUDACC__

template <typename T>
__device__ __forceinline__ float widen(T v);
template <>
__device__ __forceinline__ float widen(float v) { return v; }
template <>
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }

template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half narrow(float v) { return __float2half_rn(v); }

// The elements of a 16-byte vector, widened.
template <typename T>
struct Vec {
  static constexpr int kN = 16 / sizeof(T);
  static __device__ __forceinline__ void widen_all(const uint4& u, float* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        f[i] = __uint_as_float(w[i]);
      } else if constexpr (__is_same(T, __nv_bfloat16)) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      } else {
        const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        f[2 * i] = g.x;
        f[2 * i + 1] = g.y;
      }
    }
  }
  static __device__ __forceinline__ uint4 narrow_all(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        w[i] = __float_as_uint(f[i]);
      } else if constexpr (__is_same(T, __nv_bfloat16)) {
        const __nv_bfloat162 g = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&g);
      } else {
        const __half2 g = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&g);
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two fp32 values in one register pair.
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  return static_cast<uint64_t>(__float_as_uint(b)) << 32 | __float_as_uint(a);
}
__device__ __forceinline__ float low2(uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v)); }
__device__ __forceinline__ float high2(uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }

// Two values rounded to 16 bits, the first in the lower half.
template <typename T>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
  uint32_t r;
  if constexpr (__is_same(T, __nv_bfloat16)) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// Softmax weights in 16 bits are 2^kLift for a score at the reference, and up to kSlack (log2) more before the reference and
// the output move. fp16 has 2^15 above 1 to spare and needs it below, where a weight under 2^-14 loses bits and one under
// 2^-25 is lost while the sum counts it: thousands of keys that weigh little beside one of their row's.
constexpr float kSlack = 8.0f;
template <typename T>
constexpr float kLift = __is_same(T, __half) ? 7.0f : 0.0f;

__device__ __forceinline__ int64_t load_index(const void* p, int64_t i, int is64) {
  return is64 ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A float (or two) at `p` in the shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t peer_address(const void* p, uint32_t rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;"
      : "=r"(a)
      : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
  return a;
}
__device__ __forceinline__ float peer_load(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

constexpr float kNearCap = 0.3f;

// cap2 tanh(s over_cap), a capped score in units of log2 (cap2 = cap log2(e),
// over_cap = scale / cap). tanh(x) = 1 - 2 / (1 + e^{2x}) is off by about 1e-7
// whatever x is, which for scores far below the cap would be more than their own
// rounding: there, |x| < kNearCap, by its series up to x^9 (5e-8 of x beyond).
__device__ __forceinline__ float capped(float s, float over_cap, float cap2) {
  const float x = s * over_cap, y = x * x;
  const float e = exp2_approx(x * (2.0f * kLog2e));
  const float far = cap2 - __fdividef(2.0f * cap2, 1.0f + (e > 1e30f ? 1e30f : e));  // (fminf would make a NaN a number)
  const float series = fmaf(fmaf(fmaf(62.0f / 2835.0f, y, -17.0f / 315.0f), y, 2.0f / 15.0f), y, -1.0f / 3.0f);
  return fabsf(x) < kNearCap ? cap2 * fmaf(x * y, series, x) : far;
}

// The same of two scores that are known to be below kNearCap of the cap.
__device__ __forceinline__ uint64_t capped_near(uint64_t s, uint64_t over_cap, uint64_t cap2) {
  const uint64_t x = mul2(s, over_cap), y = mul2(x, x);
  uint64_t series = fma2(pack2(62.0f / 2835.0f, 62.0f / 2835.0f), y, pack2(-17.0f / 315.0f, -17.0f / 315.0f));
  series = fma2(series, y, pack2(2.0f / 15.0f, 2.0f / 15.0f));
  series = fma2(series, y, pack2(-1.0f / 3.0f, -1.0f / 3.0f));
  return mul2(fma2(mul2(x, y), series, x), cap2);
}

// A value that another thread of the CTA may have stored by TMA: from L2, since L1 may hold the line as it was before.
template <typename T>
__device__ __forceinline__ float widen_stored(const T* p) {
  if constexpr (sizeof(T) == 4) {
    return __ldcg(reinterpret_cast<const float*>(p));
  } else {
    const unsigned short u = __ldcg(reinterpret_cast<const unsigned short*>(p));
    return widen(*reinterpret_cast<const T*>(&u));
  }
}

// kPer elements in one load and their arithmetic: one, or two of 16 bits as a pair of fp32 values.
template <typename T, int kPer>
struct Elements {
  using Wide = float;
  T raw;
  static __device__ __forceinline__ Elements load(const T* p) { return {*p}; }
  __device__ __forceinline__ Wide wide() const { return widen(raw); }
  __device__ __forceinline__ void clear(int) { raw = narrow<T>(0.0f); }
  static __device__ __forceinline__ Wide twice(float a) { return a; }
  static __device__ __forceinline__ Wide times_plus(Wide a, Wide b, Wide c) { return fmaf(a, b, c); }
  static __device__ __forceinline__ float at(Wide a, int) { return a; }
};
template <typename T>
struct Elements<T, 2> {
  using Wide = uint64_t;
  uint32_t raw;
  static __device__ __forceinline__ Elements load(const T* p) { return {*reinterpret_cast<const uint32_t*>(p)}; }
  __device__ __forceinline__ Wide wide() const {
    if constexpr (__is_same(T, __nv_bfloat16)) {
      return static_cast<uint64_t>(raw & 0xFFFF0000u) << 32 | raw << 16;
    } else {
      const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&raw));
      return pack2(g.x, g.y);
    }
  }
  __device__ __forceinline__ void clear(int e) { raw &= e ? 0xFFFFu : 0xFFFF0000u; }
  static __device__ __forceinline__ Wide twice(float a) { return pack2(a, a); }
  static __device__ __forceinline__ Wide times_plus(Wide a, Wide b, Wide c) { return fma2(a, b, c); }
  static __device__ __forceinline__ float at(Wide a, int e) { return e ? high2(a) : low2(a); }
};

// Rows of a tile, from row0 of head h on, whose weights' sum is finite and whose output is not: a bit in `left` and their
// log-sum in `lse` (shared memory, `words` of 32 rows). Their tile may hold keys that a row does not see, whose weight is
// 0, and 0 times NaN or infinity is NaN. By warp `part` of `parts`, two rows at a time and the pairs in turn. A column in
// which a key that the row sees has such a value stays as it is; the others are formed again from the seen keys alone,
// kBatch at a time, with the weights exp(s - lse). The last key found for a column is the first looked at for the rows that
// follow, so that a warp walks to a late one once and not once per row. kPer = 2: pairs of elements are aligned. (4096
// tokens, 8 heads of 128: bf16 clean 50 us, an infinity or NaN in the first key's values 140, in key 3000's 1.19 ms, most
// of it the 56 rows before that key in its tile; fp32 1.12, 1.31 and 2.66 ms.)
template <typename T, int kDim, int kPer>
__device__ __noinline__ void attention_rows(const AttentionParams& p, int64_t row0, int h, const uint32_t* left,
                                            const float* lse, int words, int part, int parts, int lane) {
  constexpr int kRows = 2, kLoads = kDim / 32 / kPer, kBatch = kLoads <= 3 ? 8 : 4;  // keys; loads of a lane and key
  using Load = Elements<T, kPer>;
  using Wide = typename Load::Wide;
  const int g = h / p.group, column0 = lane * kPer;
  const T* k = static_cast<const T*>(p.k) + g * p.k_head + column0;
  const T* v = static_cast<const T*>(p.v) + g * p.v_head + column0;
  const float slope = p.slopes != nullptr ? p.slopes[h] : 0.0f;
  const auto in = [&](int c) { return column0 + 32 * kPer * c < p.dim; };  // load c is of the head's elements
  int witness[kLoads][kPer];  // a key whose value in the column is not finite
#pragma unroll
  for (int c = 0; c < kLoads; ++c)
#pragma unroll
    for (int e = 0; e < kPer; ++e) witness[c][e] = -1;
  int found = 0, turn = 0, rows[kRows] = {};
  for (int r = 0; r < words * 32; ++r) {
    if (left[r / 32] >> r % 32 & 1) {
      if (found++ == 0) rows[0] = r;
      rows[1] = r;
    }
    if (found == 0 || (found < kRows && r < words * 32 - 1)) continue;
    found = 0;
    if (turn++ % parts != part) continue;
    uint32_t first[kRows], end[kRows], open[kRows];  // open: a bit per column that is formed again
    T* out[kRows];
    Wide qr[kRows][kLoads], acc[kRows][kLoads];
#pragma unroll
    for (int m = 0; m < kRows; ++m) {  // (a row alone is both)
      const int64_t i = row0 + rows[m];
      first[m] = max(p.spans[i], 0);
      end[m] = static_cast<uint32_t>(min(static_cast<int64_t>(p.spans[p.q_tokens + i]), p.k_tokens));
      const T* q = static_cast<const T*>(p.q) + i * p.q_token + h * p.q_head + column0;
      out[m] = static_cast<T*>(p.out) + i * p.out_token + h * p.out_head + column0;
      open[m] = 0;
#pragma unroll
      for (int c = 0; c < kLoads; ++c) {
        qr[m][c] = acc[m][c] = Load::twice(0.0f);
        if (!in(c)) continue;
        qr[m][c] = Load::load(q + 32 * kPer * c).wide();
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          if (!(fabsf(widen_stored(out[m] + 32 * kPer * c + e)) < kInf)) open[m] |= 1u << (c * kPer + e);
      }
    }
#pragma unroll
    for (int c = 0; c < kLoads; ++c)
#pragma unroll
      for (int e = 0; e < kPer; ++e)
#pragma unroll
        for (int m = 0; m < kRows; ++m)
          if (witness[c][e] >= static_cast<int>(first[m]) && witness[c][e] < static_cast<int>(end[m]))
            open[m] &= ~(1u << (c * kPer + e));
    const int mine = lane / kBatch % kRows;  // of a batch the lane has key lane mod kBatch, and this row
    const int64_t my_row = row0 + (mine ? rows[1] : rows[0]);
    const float my_lse = lse[mine ? rows[1] : rows[0]];
    const uint32_t my_first = mine ? first[1] : first[0], my_end = mine ? end[1] : end[0];
    const int64_t self = p.slopes != nullptr ? p.spans[2 * p.q_tokens + my_row] : 0;
    float total = 0.0f;
    // The rows' last kTail batches of keys first, then from the first on: a late key is found soon by the rows of its tile.
    constexpr uint32_t kTail = 128 / kBatch;
    const uint32_t from = min(first[0], first[1]), last = max(end[0], end[1]) - 1, batches = (last - from) / kBatch + 1;
    for (uint32_t b = 0; b < batches && __any_sync(0xFFFFFFFFu, (open[0] | open[1]) != 0); ++b) {
      const uint32_t j0 = from + (b < kTail && batches > kTail ? batches - kTail + b : batches > kTail ? b - kTail : b) * kBatch;
      Load kk[kBatch][kLoads], vv[kBatch][kLoads];
#pragma unroll
      for (int n = 0; n < kBatch; ++n) {
        const int64_t j = min(j0 + n, last);
        const T *kj = k + j * p.k_token, *vj = v + j * p.v_token;
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
          kk[n][c] = vv[n][c] = {};
          if (in(c)) {
            kk[n][c] = Load::load(kj + 32 * kPer * c);
            vv[n][c] = Load::load(vj + 32 * kPer * c);
          }
        }
      }
      float s[kRows * kBatch];
#pragma unroll
      for (int n = 0; n < kBatch; ++n) {
        Wide dots[kRows];
#pragma unroll
        for (int m = 0; m < kRows; ++m) dots[m] = Load::twice(0.0f);
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
          const Wide f = kk[n][c].wide();
#pragma unroll
          for (int m = 0; m < kRows; ++m) dots[m] = Load::times_plus(qr[m][c], f, dots[m]);
        }
#pragma unroll
        for (int m = 0; m < kRows; ++m) s[m * kBatch + n] = Load::at(dots[m], 0) + (kPer == 2 ? Load::at(dots[m], 1) : 0.0f);
      }
      // the lanes' sums, each lane left with that of its key and row
#pragma unroll
      for (int o = kRows * kBatch / 2; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < o; ++n) {
          const float there = lane & o ? s[n] : s[n + o], here = lane & o ? s[n + o] : s[n];
          s[n] = here + __shfl_xor_sync(0xFFFFFFFFu, there, o);
        }
      float x = s[0];
#pragma unroll
      for (int o = kRows * kBatch; o < 32; o <<= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
      x *= p.scale;
      if (p.softcap > 0.0f) x = p.softcap * tanhf(x / p.softcap);
      const uint32_t j = j0 + lane % kBatch;
      if (p.slopes != nullptr) x -= slope * fabsf(static_cast<float>(self - static_cast<int64_t>(j)));
      const float w = j >= my_first && j < my_end ? __expf(x - my_lse) : 0.0f;
      total += w;
      Wide sums[kRows][kLoads];  // the batch's
      const auto weigh = [&] {
#pragma unroll
        for (int m = 0; m < kRows; ++m)
#pragma unroll
          for (int c = 0; c < kLoads; ++c) sums[m][c] = Load::twice(0.0f);
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
          Wide wn[kRows];
#pragma unroll
          for (int m = 0; m < kRows; ++m) wn[m] = Load::twice(__shfl_sync(0xFFFFFFFFu, w, m * kBatch + n));
#pragma unroll
          for (int c = 0; c < kLoads; ++c) {
            const Wide f = vv[n][c].wide();
#pragma unroll
            for (int m = 0; m < kRows; ++m) sums[m][c] = Load::times_plus(wn[m], f, sums[m][c]);
          }
        }
      };
      weigh();
      Wide zeros = Load::twice(0.0f);  // 0 times the sums: NaN where a value is not finite
#pragma unroll
      for (int c = 0; c < kLoads; ++c)
#pragma unroll
        for (int m = 0; m < kRows; ++m) zeros = Load::times_plus(sums[m][c], Load::twice(0.0f), zeros);
      if (__any_sync(0xFFFFFFFFu, Load::at(zeros, 0) != 0.0f || Load::at(zeros, kPer - 1) != 0.0f)) {
#pragma unroll
        for (int n = 0; n < kBatch; ++n)
#pragma unroll
          for (int c = 0; c < kLoads; ++c)
#pragma unroll
            for (int e = 0; e < kPer; ++e)
              if (!(fabsf(Load::at(vv[n][c].wide(), e)) < kInf)) {
                const uint32_t at = min(j0 + n, last);
                witness[c][e] = static_cast<int>(at);
                vv[n][c].clear(e);  // for the other row, which may not see it
#pragma unroll
                for (int m = 0; m < kRows; ++m)
                  if (at >= first[m] && at < end[m]) open[m] &= ~(1u << (c * kPer + e));
              }
        weigh();
      }
#pragma unroll
      for (int c = 0; c < kLoads; ++c)
#pragma unroll
        for (int m = 0; m < kRows; ++m) acc[m][c] = Load::times_plus(sums[m][c], Load::twice(1.0f), acc[m][c]);
    }
#pragma unroll
    for (int m = 0; m < kRows; ++m) {
      float sum = mine == m && lane < kRows * kBatch ? total : 0.0f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      const float over = 1.0f / sum;
#pragma unroll
      for (int c = 0; c < kLoads; ++c)
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          if (open[m] >> (c * kPer + e) & 1) out[m][32 * kPer * c + e] = narrow<T>(Load::at(acc[m][c], e) * over);
    }
  }
}

#endif  // __CUDACC__

}  // namespace zo
