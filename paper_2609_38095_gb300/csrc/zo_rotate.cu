// zo_rotate.cu -- a head's norm and its rotation by position in one pass
// (zo_rotate_heads), the table of angles, and the spans of packed documents.
#include "zo_forward.cuh"

namespace zo {

namespace {

constexpr int kRotateThreads = 256;
constexpr int kRotateCtas = 4;  // per SM, by registers

// Position t's row of the table; a position outside it: NULL.
__device__ __forceinline__ const float* table_row(const RotateParams& p, int64_t t) {
  const int64_t pos = load_index(p.positions, t, p.index64);
  return pos < 0 || pos >= p.table_rows ? nullptr : p.table + pos * p.rotary;
}

// Where token t's row of a part starts; NULL for a slot that is none.
template <typename T>
__device__ __forceinline__ T* out_row(const RotateParams& p, const RotatePart& part, int64_t t) {
  if (!part.slotted) return static_cast<T*>(part.out) + t * part.out_token;
  const int64_t slot = load_index(p.slots, t, p.index64);
  if (slot < 0 || slot >= p.n_slots) return nullptr;
  const int64_t page = p.page_size == 1 ? slot : slot / p.page_size;
  return static_cast<T*>(part.out) + page * part.out_page + (slot - page * p.page_size) * part.out_token;
}

__device__ __forceinline__ const RotatePart& part_of(const RotateParams& p, int slice) {
  const int i = (p.n_parts > 1 && slice >= p.part[1].slice) + (p.n_parts > 2 && slice >= p.part[2].slice);
  return p.part[i];
}

__device__ __forceinline__ float weight_at(const RotatePart& part, int i) {
  if (part.weight_dtype == 0) return static_cast<const float*>(part.weight)[i];
  if (part.weight_dtype == 1) return widen(static_cast<const __nv_bfloat16*>(part.weight)[i]);
  return widen(static_cast<const __half*>(part.weight)[i]);
}

template <typename T>
constexpr int kCode = sizeof(T) == 4 ? 0 : __is_same(T, __nv_bfloat16) ? 1 : 2;  // zo_dtype

// Two values: in one register pair for 16-bit types, whose instructions on two values at once halve what bounds them, and
// as two for fp32, where the pairs' aligned registers would spill (130 against 161 us, 20000 tokens of 40 heads of 128).
template <typename T>
struct PairOf {
  using type = uint64_t;
};
template <>
struct PairOf<float> {
  using type = float2;
};
__device__ __forceinline__ void set(uint64_t& p, float a, float b) { p = pack2(a, b); }
__device__ __forceinline__ void set(float2& p, float a, float b) { p = make_float2(a, b); }
__device__ __forceinline__ float lower(uint64_t p) { return low2(p); }
__device__ __forceinline__ float lower(float2 p) { return p.x; }
__device__ __forceinline__ float upper(uint64_t p) { return high2(p); }
__device__ __forceinline__ float upper(float2 p) { return p.y; }
__device__ __forceinline__ uint64_t times(uint64_t a, uint64_t b) { return mul2(a, b); }
__device__ __forceinline__ float2 times(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
__device__ __forceinline__ uint64_t times_plus(uint64_t a, uint64_t b, uint64_t c) { return fma2(a, b, c); }
__device__ __forceinline__ float2 times_plus(float2 a, float2 b, float2 c) {
  return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y));
}

// W words of 4 bytes in one load, W = 4 or 2.
template <int W>
struct Words {
  uint32_t w[W];
  __device__ __forceinline__ void load(const void* p) {
    if constexpr (W == 4) {
      const uint4 u = *static_cast<const uint4*>(p);
      w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    } else {
      const uint2 u = *static_cast<const uint2*>(p);
      w[0] = u.x, w[1] = u.y;
    }
  }
  __device__ __forceinline__ void store(void* p) const {
    if constexpr (W == 4) *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *static_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  }
  template <typename T>
  __device__ __forceinline__ void widen_all(typename PairOf<T>::type* f) const {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if constexpr (sizeof(T) == 4) {
        if (i % 2 == 0) set(f[i / 2], __uint_as_float(w[i]), __uint_as_float(w[i + 1]));
      } else if constexpr (__is_same(T, __nv_bfloat16)) {
        f[i] = static_cast<uint64_t>(w[i] & 0xFFFF0000u) << 32 | w[i] << 16;
      } else {
        const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        set(f[i], g.x, g.y);
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void narrow_all(const typename PairOf<T>::type* f) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(i % 2 ? upper(f[i / 2]) : lower(f[i / 2]));
      else w[i] = narrow2<T>(lower(f[i]), upper(f[i]));
    }
  }
};

// A lane's E angles as pairs.
template <int E, typename P>
__device__ __forceinline__ void load_angles(const float* at, P* f) {
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    if constexpr (E >= 8) {
      if (e % 4 != 0) continue;
      const float4 v = *reinterpret_cast<const float4*>(at + e);
      set(f[e / 2], v.x, v.y);
      set(f[e / 2 + 1], v.z, v.w);
    } else {
      const float2 v = *reinterpret_cast<const float2*>(at + e);
      set(f[e / 2], v.x, v.y);
    }
  }
}

// A head lies on kLanes lanes, each with a unit of two vectors of W words: the
// two halves of its pairs (layout half), or neighbours (interleaved, and what is
// not rotated), so that a lane has both elements of a pair and reads E cosines
// and sines at E times its number in both layouts. W is 4, or 2 where the size or
// the rotated part leaves a half vector. A warp takes kHeads heads of each of its
// groups of lanes; angles and weight are loaded once for them. Bound by HBM: 2
// bytes in and 2 out per 16-bit element, and by its instructions (50001 tokens of
// 80 heads of 128, fp16: 350 us = 5.9 TB/s; before the arithmetic by pairs of fp32
// values 361, with four heads per group of lanes on fewer CTAs 365, with one 521).
template <typename T, int W, int kLanes>
__global__ void __launch_bounds__(kRotateThreads, kRotateCtas) rotate_heads_kernel(const __grid_constant__ RotateParams p) {
  constexpr int E = W * 4 / sizeof(T);
  constexpr int kGroups = 32 / kLanes, kHeads = 8 / W;
  const int lane = threadIdx.x & 31;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kRotateThreads / 32) + (threadIdx.x >> 5);
  if (t >= p.tokens) return;
  const RotatePart& part = part_of(p, blockIdx.y);
  T* row = out_row<T>(p, part, t);
  if (row == nullptr) return;
  const int unit = lane % kLanes, head0 = (blockIdx.y - part.slice) * kHeads * kGroups + lane / kLanes;
  const bool here = unit * 2 * E < p.dim;
  const bool turned = part.rotate && unit * 2 * E < p.rotary;
  int a = unit * 2 * E, b = a + E;
  if (turned && !p.interleaved) {
    a = unit * E;
    b = p.rotary / 2 + a;
  }
  const T* in = static_cast<const T*>(part.in) + t * part.in_token;
  Words<W> raw[kHeads][2];
#pragma unroll
  for (int n = 0; n < kHeads; ++n) {
    const int h = head0 + n * kGroups;
#pragma unroll
    for (int i = 0; i < W; ++i) raw[n][0].w[i] = raw[n][1].w[i] = 0;
    if (here && h < part.heads) {
      raw[n][0].load(in + h * part.in_head + a);
      raw[n][1].load(in + h * part.in_head + b);
    }
  }
  using P = typename PairOf<T>::type;
  P cs[E / 2], sn[E / 2];
  if (turned) {
    const float* angles = table_row(p, t);
    if (angles == nullptr) {
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        set(cs[e], NAN, NAN);
        set(sn[e], NAN, NAN);
      }
    } else {
      load_angles<E>(angles + unit * E, cs);
      load_angles<E>(angles + p.rotary / 2 + unit * E, sn);
    }
  }
  const bool norm = part.weight != nullptr;
  Words<W> w[2];  // packed: as floats, a quarter of the registers would be weights
  if (norm && here) {
    w[0].load(static_cast<const T*>(part.weight) + a);
    w[1].load(static_cast<const T*>(part.weight) + b);
  }
#pragma unroll
  for (int n = 0; n < kHeads; ++n) {
    const int h = head0 + n * kGroups;
    if (head0 - lane / kLanes + n * kGroups >= part.heads) break;  // the same for the whole warp
    P x[E];
    raw[n][0].template widen_all<T>(x);
    raw[n][1].template widen_all<T>(x + E / 2);
    if (norm) {
      P sums = times(x[0], x[0]);
#pragma unroll
      for (int e = 1; e < E; ++e) sums = times_plus(x[e], x[e], sums);
      float sum = lower(sums) + upper(sums);
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      const float r = rsqrtf(sum / p.dim + p.eps);
      P both, f[E];
      set(both, r, r);
      w[0].template widen_all<T>(f);
      w[1].template widen_all<T>(f + E / 2);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = times(x[e], times(both, f[e]));
    }
    if (turned) {
      P flip;  // a sine's signs for a pair's two elements, or for two pairs' first ones
      set(flip, -1.0f, p.interleaved ? 1.0f : -1.0f);
      if (p.interleaved) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float c = e % 2 ? upper(cs[e / 2]) : lower(cs[e / 2]), s = e % 2 ? upper(sn[e / 2]) : lower(sn[e / 2]);
          P cc, ss, other;
          set(cc, c, c);
          set(ss, s, s);
          set(other, upper(x[e]), lower(x[e]));
          x[e] = times_plus(x[e], cc, times(other, times(ss, flip)));
        }
      } else {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const P u = x[e], v = x[E / 2 + e];
          x[e] = times_plus(u, cs[e], times(v, times(sn[e], flip)));
          x[E / 2 + e] = times_plus(v, cs[e], times(u, sn[e]));
        }
      }
    }
    if (here && h < part.heads) {
      Words<W> out;
      out.template narrow_all<T>(x);
      out.store(row + h * part.out_head + a);
      out.template narrow_all<T>(x + E / 2);
      out.store(row + h * part.out_head + b);
    }
  }
}

// Any head size, stride and alignment: a warp per token and head, pairs of
// elements by lane.
template <typename T>
__global__ void __launch_bounds__(kRotateThreads) rotate_heads_any_kernel(const __grid_constant__ RotateParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kRotateThreads / 32) + (threadIdx.x >> 5);
  if (t >= p.tokens) return;
  const RotatePart& part = part_of(p, blockIdx.y);
  T* row = out_row<T>(p, part, t);
  if (row == nullptr) return;
  const int h = blockIdx.y - part.slice;
  const T* in = static_cast<const T*>(part.in) + t * part.in_token + h * part.in_head;
  row += h * part.out_head;
  const int half = p.rotary / 2;
  float x[4][2];
  int at[4][2];
  float sum = 0.0f;
#pragma unroll
  for (int c = 0; c < 4; ++c) {  // pair by pair: at most 128 of them
    const int i = lane + 32 * c;
    const bool split = part.rotate && !p.interleaved && i < half;
    at[c][0] = split ? i : 2 * i;
    at[c][1] = split ? i + half : 2 * i + 1;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      x[c][s] = at[c][s] < p.dim ? widen(in[at[c][s]]) : 0.0f;
      sum = fmaf(x[c][s], x[c][s], sum);
    }
  }
  if (part.weight != nullptr) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    const float r = rsqrtf(sum / p.dim + p.eps);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (at[c][s] < p.dim) {
          const float w = weight_at(part, at[c][s]);
          x[c][s] = x[c][s] * r * w;
        }
  }
  const float* angles = part.rotate ? table_row(p, t) : nullptr;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int i = lane + 32 * c;
    if (part.rotate && i < half) {
      const float cs = angles != nullptr ? angles[i] : NAN, sn = angles != nullptr ? angles[half + i] : NAN;
      const float u = x[c][0], v = x[c][1];
      x[c][0] = u * cs - v * sn;
      x[c][1] = v * cs + u * sn;
    }
  }
  __syncwarp();  // in place, a pair's elements may lie on other lanes' places: all are read by now
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int s = 0; s < 2; ++s)
      if (at[c][s] < p.dim) row[at[c][s]] = narrow<T>(x[c][s]);
}

__global__ void rotary_table_kernel(float* table, int64_t rows, int half, double base, double scale, double original,
                                    double low, double high, double magnitude) {
  const int64_t n = rows * half;
  for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i < n;
       i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    const int64_t pos = i / half;
    const int c = static_cast<int>(i - pos * half);
    double w = pow(base, -static_cast<double>(c) / half);
    if (scale != 1.0) {
      double g = 0.0;
      if (original > 0.0) {
        const double turns = original * w / 6.283185307179586477;
        g = high > low ? fmin(1.0, fmax(0.0, (turns - low) / (high - low))) : (turns >= low ? 1.0 : 0.0);
      }
      w *= (1.0 - g) / scale + g;
    }
    double s, cs;
    sincos(static_cast<double>(pos) * w, &s, &cs);
    table[pos * 2 * half + c] = static_cast<float>(cs * magnitude);
    table[pos * 2 * half + half + c] = static_cast<float>(s * magnitude);
  }
}

__global__ void document_spans_kernel(const int32_t* q_starts, const int32_t* k_starts, const int32_t* prefix, int docs,
                                      int32_t* spans, int64_t tokens) {
  for (int64_t t = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; t < tokens;
       t += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    int lo = 0, hi = docs;  // the last document that starts at or before t
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (q_starts[mid] <= t) lo = mid;
      else hi = mid;
    }
    int64_t first = 0, end = 0, self = 0;
    if (docs > 0 && t >= q_starts[lo] && t < q_starts[lo + 1]) {
      const int64_t start = k_starts[lo], stop = k_starts[lo + 1];
      self = stop - (q_starts[lo + 1] - t);
      first = start;
      end = self + 1;
      if (prefix != nullptr) end = max(end, min(start + prefix[lo], stop));
      if (end <= first) first = end = 0;
    }
    spans[t] = static_cast<int32_t>(first);
    spans[tokens + t] = static_cast<int32_t>(end);
    spans[2 * tokens + t] = static_cast<int32_t>(self);
  }
}

// Whether every vector of a part, its weight's among them, starts on `bytes` bytes and is of the data's type. (A weight of
// another type alone leaves aligned heads to rotate_heads_any_kernel: 4091 tokens of 40 heads of 128, bf16, with fp32 weights
// 82 us against 16.7.)
template <typename T>
bool part_aligned(const RotatePart& r, int64_t bytes) {
  const int64_t n = bytes / static_cast<int64_t>(sizeof(T));
  return (r.weight == nullptr || (r.weight_dtype == kCode<T> && aligned_to(r.weight, bytes))) && aligned_to(r.in, bytes) &&
         aligned_to(r.out, bytes) && r.in_token % n == 0 && r.in_head % n == 0 && r.out_token % n == 0 &&
         r.out_head % n == 0 && (!r.slotted || r.out_page % n == 0);
}

template <typename T, int W, int kLanes>
void launch_lanes(RotateParams& p, unsigned blocks, cudaStream_t stream) {
  constexpr int kHeads = 8 / W * 32 / kLanes;
  int slices = 0;
  for (int i = 0; i < p.n_parts; ++i) {
    p.part[i].slice = slices;
    slices += (p.part[i].heads + kHeads - 1) / kHeads;
  }
  rotate_heads_kernel<T, W, kLanes><<<dim3(blocks, slices), kRotateThreads, 0, stream>>>(p);
}

// By vectors of W words; false where sizes or addresses do not admit them.
template <typename T, int W>
bool launch_vectors(RotateParams& p, unsigned blocks, cudaStream_t stream) {
  constexpr int kUnit = 2 * W * 4 / sizeof(T);  // elements
  const int units = p.dim / kUnit;
  bool fits = p.dim % kUnit == 0 && p.rotary % kUnit == 0 && units <= 32 && aligned_to(p.table, kUnit >= 16 ? 16 : 8);
  for (int i = 0; i < p.n_parts; ++i) fits = fits && part_aligned<T>(p.part[i], W * 4);
  if (!fits) return false;
  if (units <= 4) launch_lanes<T, W, 4>(p, blocks, stream);
  else if (units <= 8) launch_lanes<T, W, 8>(p, blocks, stream);
  else if (units <= 16) launch_lanes<T, W, 16>(p, blocks, stream);
  else launch_lanes<T, W, 32>(p, blocks, stream);
  return true;
}

template <typename T>
cudaError_t launch_rotate(RotateParams p, cudaStream_t stream) {
  const unsigned blocks = static_cast<unsigned>((p.tokens + kRotateThreads / 32 - 1) / (kRotateThreads / 32));
  if (!launch_vectors<T, 4>(p, blocks, stream) && !launch_vectors<T, 2>(p, blocks, stream)) {
    int heads = 0;
    for (int i = 0; i < p.n_parts; ++i) {
      p.part[i].slice = heads;
      heads += p.part[i].heads;
    }
    rotate_heads_any_kernel<T><<<dim3(blocks, heads), kRotateThreads, 0, stream>>>(p);
  }
  return cudaGetLastError();
}

unsigned blocks_for(int64_t n, int threads) {
  const int64_t b = (n + threads - 1) / threads;
  return static_cast<unsigned>(b < 65536 ? b : 65536);
}

}  // namespace

cudaError_t launch_rotate_heads(const RotateParams& p, int dtype, cudaStream_t stream) {
  if (dtype == 0) return launch_rotate<float>(p, stream);
  if (dtype == 1) return launch_rotate<__nv_bfloat16>(p, stream);
  return launch_rotate<__half>(p, stream);
}

cudaError_t launch_rotary_table(float* table, int64_t rows, int rotary, double base, double scale, int64_t original,
                                double low, double high, double magnitude, cudaStream_t stream) {
  rotary_table_kernel<<<blocks_for(rows * (rotary / 2), 256), 256, 0, stream>>>(
      table, rows, rotary / 2, base, scale, static_cast<double>(original), low, high, magnitude);
  return cudaGetLastError();
}

cudaError_t launch_document_spans(const int32_t* q_starts, const int32_t* k_starts, const int32_t* prefix, int docs,
                                  int32_t* spans, int64_t tokens, cudaStream_t stream) {
  document_spans_kernel<<<blocks_for(tokens, 256), 256, 0, stream>>>(q_starts, k_starts, prefix, docs, spans, tokens);
  return cudaGetLastError();
}

}  // namespace zo
