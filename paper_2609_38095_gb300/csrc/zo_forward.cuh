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

struct TokenLossParams {
  const void* logits;
  int64_t row, tokens, vocab;
  const void* targets;
  int32_t target64, flags;
  void* loss;
  float* nll;
  double* rows;  // a token's nll before its rounding
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
cudaError_t launch_token_loss(const TokenLossParams& p, int dtype, int sms, cudaStream_t stream);

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

// Row i of head h alone, by one warp, a key at a time: for rows whose tile gave
// a value that is not finite, so that NaN or infinities of keys that the row
// does not see (their weight is 0, and 0 times NaN is NaN) stay out of it.
template <typename T>
__device__ __noinline__ void attention_row(const AttentionParams& p, int64_t i, int h, int lane) {
  const T* q = static_cast<const T*>(p.q) + i * p.q_token + h * p.q_head;
  const int g = h / p.group;
  const T* k = static_cast<const T*>(p.k) + g * p.k_head;
  const T* v = static_cast<const T*>(p.v) + g * p.v_head;
  const int64_t first = max(p.spans[i], 0), end = min(static_cast<int64_t>(p.spans[p.q_tokens + i]), p.k_tokens);
  const int64_t self = p.slopes != nullptr ? p.spans[2 * p.q_tokens + i] : 0;
  const float slope = p.slopes != nullptr ? p.slopes[h] : 0.0f;
  float qr[8], acc[8];
  bool nan = false;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    qr[c] = lane + 32 * c < p.dim ? widen(q[lane + 32 * c]) : 0.0f;
    acc[c] = 0.0f;
    nan = nan || qr[c] != qr[c];
  }
  nan = __any_sync(0xFFFFFFFFu, nan) && end > first;  // then every score is NaN (a forward that has diverged: all rows)
  float top = -kInf, total = nan ? NAN : 0.0f;
  for (int64_t j = first; j < end && total == total; ++j) {  // from the first NaN score on nothing changes
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (lane + 32 * c < p.dim) s = fmaf(qr[c], widen(k[j * p.k_token + lane + 32 * c]), s);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    s *= p.scale;
    if (p.softcap > 0.0f) s = p.softcap * tanhf(s / p.softcap);
    if (p.slopes != nullptr) s -= slope * fabsf(static_cast<float>(self - j));
    const float next = s > top ? s : top;  // a NaN score makes w NaN, not the maximum
    const float back = next == -kInf ? 1.0f : __expf(top - next);
    const float w = s == -kInf ? 0.0f : __expf(s - next);
    total = total * back + w;
    top = next;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (lane + 32 * c < p.dim) acc[c] = acc[c] * back + w * widen(v[j * p.v_token + lane + 32 * c]);
  }
  const float over = total == 0.0f ? 0.0f : 1.0f / total;
  T* out = static_cast<T*>(p.out) + i * p.out_token + h * p.out_head;
#pragma unroll
  for (int c = 0; c < 8; ++c)
    if (lane + 32 * c < p.dim) out[lane + 32 * c] = narrow<T>(acc[c] * over);
  if (p.lse != nullptr && lane == 0) p.lse[h * p.q_tokens + i] = total == 0.0f ? -kInf : top + logf(total);
}

#endif  // __CUDACC__

}  // namespace zo
