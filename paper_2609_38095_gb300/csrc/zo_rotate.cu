// zo_rotate.cu -- a head's norm and its rotation by position in one pass
// (zo_rotate_heads), the table of angles, and the spans of packed documents.
#include "zo_forward.cuh"

namespace zo {

namespace {

constexpr int kRotateThreads = 256;
constexpr int kHeadsPerGroup = 2;  // heads that a group of lanes takes, their loads issued together
constexpr int kRotateCtas = 4;     // per SM, by registers: with two heads per group 64 KB in flight

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

// A head lies on kLanes lanes, each with a unit of two 16-byte vectors: the two
// halves of its pairs (layout half), or neighbours (interleaved, and what is not
// rotated), so that a lane has both elements of a pair and reads E cosines and
// sines at E times its number in both layouts. A warp takes one token's
// kHeadsPerGroup * 32 / kLanes heads; angles and weight are loaded once for them.
// Bound by HBM: 2 bytes in and 2 out per 16-bit element.
template <typename T, int kLanes>
__global__ void __launch_bounds__(kRotateThreads, kRotateCtas) rotate_heads_kernel(const __grid_constant__ RotateParams p) {
  constexpr int E = Vec<T>::kN;
  constexpr int kGroups = 32 / kLanes;
  const int lane = threadIdx.x & 31;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kRotateThreads / 32) + (threadIdx.x >> 5);
  if (t >= p.tokens) return;
  const RotatePart& part = part_of(p, blockIdx.y);
  T* row = out_row<T>(p, part, t);
  if (row == nullptr) return;
  const int unit = lane % kLanes, head0 = (blockIdx.y - part.slice) * kHeadsPerGroup * kGroups + lane / kLanes;
  const bool here = unit * 2 * E < p.dim;
  const bool turned = part.rotate && unit * 2 * E < p.rotary;
  int a = unit * 2 * E, b = a + E;
  if (turned && !p.interleaved) {
    a = unit * E;
    b = p.rotary / 2 + a;
  }
  const T* in = static_cast<const T*>(part.in) + t * part.in_token;
  uint4 raw[kHeadsPerGroup][2];
#pragma unroll
  for (int n = 0; n < kHeadsPerGroup; ++n) {
    const int h = head0 + n * kGroups;
    raw[n][0] = raw[n][1] = make_uint4(0, 0, 0, 0);
    if (here && h < part.heads) {
      raw[n][0] = *reinterpret_cast<const uint4*>(in + h * part.in_head + a);
      raw[n][1] = *reinterpret_cast<const uint4*>(in + h * part.in_head + b);
    }
  }
  float cs[E], sn[E];
  if (turned) {
    const float* angles = table_row(p, t);
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const float4 c = angles != nullptr ? *reinterpret_cast<const float4*>(angles + unit * E + e)
                                         : make_float4(NAN, NAN, NAN, NAN);
      const float4 s = angles != nullptr ? *reinterpret_cast<const float4*>(angles + p.rotary / 2 + unit * E + e)
                                         : make_float4(NAN, NAN, NAN, NAN);
      cs[e] = c.x, cs[e + 1] = c.y, cs[e + 2] = c.z, cs[e + 3] = c.w;
      sn[e] = s.x, sn[e + 1] = s.y, sn[e + 2] = s.z, sn[e + 3] = s.w;
    }
  }
  const bool norm = part.weight != nullptr;
  uint4 w[2];  // packed: as floats, a quarter of the registers would be weights
  if (norm && here) {
    w[0] = *reinterpret_cast<const uint4*>(static_cast<const T*>(part.weight) + a);
    w[1] = *reinterpret_cast<const uint4*>(static_cast<const T*>(part.weight) + b);
  }
#pragma unroll
  for (int n = 0; n < kHeadsPerGroup; ++n) {
    const int h = head0 + n * kGroups;
    if (head0 - lane / kLanes + n * kGroups >= part.heads) break;  // the same for the whole warp
    float x[2 * E];
    Vec<T>::widen_all(raw[n][0], x);
    Vec<T>::widen_all(raw[n][1], x + E);
    if (norm) {
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 2 * E; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      const float r = rsqrtf(sum / p.dim + p.eps);
      float f[E];
      Vec<T>::widen_all(w[0], f);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = x[e] * r * f[e];
      Vec<T>::widen_all(w[1], f);
#pragma unroll
      for (int e = 0; e < E; ++e) x[E + e] = x[E + e] * r * f[e];
    }
    if (turned) {
      if (p.interleaved) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float u = x[2 * e], v = x[2 * e + 1];
          x[2 * e] = u * cs[e] - v * sn[e];
          x[2 * e + 1] = v * cs[e] + u * sn[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float u = x[e], v = x[E + e];
          x[e] = u * cs[e] - v * sn[e];
          x[E + e] = v * cs[e] + u * sn[e];
        }
      }
    }
    if (here && h < part.heads) {
      *reinterpret_cast<uint4*>(row + h * part.out_head + a) = Vec<T>::narrow_all(x);
      *reinterpret_cast<uint4*>(row + h * part.out_head + b) = Vec<T>::narrow_all(x + E);
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

// Whether every vector of a part, its weight's among them, starts on 16 bytes and is of the data's type.
template <typename T>
bool part_aligned(const RotatePart& r) {
  constexpr int64_t E = Vec<T>::kN;
  return (r.weight == nullptr || (r.weight_dtype == kCode<T> && aligned_to(r.weight, 16))) && aligned_to(r.in, 16) &&
         aligned_to(r.out, 16) && r.in_token % E == 0 && r.in_head % E == 0 &&
         r.out_token % E == 0 && r.out_head % E == 0 && (!r.slotted || r.out_page % E == 0);
}

template <typename T, int kLanes>
void launch_vectors(RotateParams& p, unsigned blocks, cudaStream_t stream) {
  constexpr int kHeads = kHeadsPerGroup * 32 / kLanes;
  int slices = 0;
  for (int i = 0; i < p.n_parts; ++i) {
    p.part[i].slice = slices;
    slices += (p.part[i].heads + kHeads - 1) / kHeads;
  }
  rotate_heads_kernel<T, kLanes><<<dim3(blocks, slices), kRotateThreads, 0, stream>>>(p);
}

template <typename T>
cudaError_t launch_rotate(RotateParams p, cudaStream_t stream) {
  constexpr int E = Vec<T>::kN;
  const unsigned blocks = static_cast<unsigned>((p.tokens + kRotateThreads / 32 - 1) / (kRotateThreads / 32));
  bool vectors = p.dim % (2 * E) == 0 && p.rotary % (2 * E) == 0 && aligned_to(p.table, 16);
  for (int i = 0; i < p.n_parts; ++i) vectors = vectors && part_aligned<T>(p.part[i]);
  if (vectors) {
    const int units = p.dim / (2 * E);
    if (units <= 4) launch_vectors<T, 4>(p, blocks, stream);
    else if (units <= 8) launch_vectors<T, 8>(p, blocks, stream);
    else if (units <= 16) launch_vectors<T, 16>(p, blocks, stream);
    else launch_vectors<T, 32>(p, blocks, stream);
  } else {
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
