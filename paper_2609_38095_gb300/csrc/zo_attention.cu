// zo_attention.cu -- attention of packed documents on the fp32 units: every
// type, head size, stride and alignment (zo_attention).
#include "zo_forward.cuh"

namespace zo {

namespace {

constexpr int kTile = 64;      // query rows and keys of a tile
constexpr int kThreads256 = 256;

// rows [from, from + kTile) of a head as fp32, either transposed ([d][row]) or
// as they are ([row][d]); zero outside [lo, hi) and beyond the head's size.
template <typename T, int DP, bool kTransposed, bool kVec>
__device__ __forceinline__ void load_tile(float* dst, const T* src, int64_t stride, int64_t from, int64_t lo, int64_t hi,
                                          int dim) {
  constexpr int E = kVec ? Vec<T>::kN : 1;
  constexpr int kChunks = DP / E;
  if constexpr (kTransposed) {  // lanes on rows: stores without bank conflicts, a row's sectors from L1
    const int r = threadIdx.x % kTile;
    const int64_t row = from + r;
    const bool in = row >= lo && row < hi;
    for (int c = threadIdx.x / kTile; c < kChunks; c += kThreads256 / kTile) {
      float f[E];
      if constexpr (kVec) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (in && c * E < dim) u = *reinterpret_cast<const uint4*>(src + row * stride + c * E);
        Vec<T>::widen_all(u, f);
      } else {
        f[0] = in && c < dim ? widen(src[row * stride + c]) : 0.0f;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) dst[(c * E + e) * kTile + r] = f[e];
    }
  } else {
    for (int i = threadIdx.x; i < kTile * kChunks; i += kThreads256) {
      const int r = i / kChunks, c = i % kChunks;
      const int64_t row = from + r;
      const bool in = row >= lo && row < hi;
      if constexpr (kVec) {
        float f[E];
        uint4 u = make_uint4(0, 0, 0, 0);
        if (in && c * E < dim) u = *reinterpret_cast<const uint4*>(src + row * stride + c * E);
        Vec<T>::widen_all(u, f);
#pragma unroll
        for (int e = 0; e < E; e += 4)
          *reinterpret_cast<float4*>(dst + r * DP + c * E + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
      } else {
        dst[r * DP + c] = in && c < dim ? widen(src[row * stride + c]) : 0.0f;
      }
    }
  }
}

// 64 query rows of one head; keys in tiles of 64, scores and products by fp32
// multiply-adds, 4 x 4 scores and 4 x DP/16 output elements per thread. Row
// statistics run along; a row's 16 threads share them by shuffles.
template <typename T, int DP, bool kVec>
__global__ void __launch_bounds__(kThreads256, DP <= 128 ? 2 : 1)
    attention_tiles_kernel(const __grid_constant__ AttentionParams p) {
  extern __shared__ __align__(16) float smem[];
  float* qs = smem;                 // [DP][64]
  float* ks = qs + DP * kTile;      // [DP][64]
  float* vs = ks + DP * kTile;      // [64][DP]
  float* ps = vs + DP * kTile;      // [64 rows][64 keys]
  __shared__ int64_t range[2];
  __shared__ int bad[kTile];
  const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16, h = blockIdx.y, g = h / p.group;
  const int64_t row0 = (static_cast<int64_t>(gridDim.x) - 1 - blockIdx.x) * kTile;  // the longest causal rows first
  int64_t lo[4], hi[4], self[4];
  int64_t least = INT64_MAX, most = 0;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t i = row0 + ty * 4 + r;
    lo[r] = hi[r] = self[r] = 0;
    if (i < p.q_tokens) {
      lo[r] = max(p.spans[i], 0);
      hi[r] = min(static_cast<int64_t>(p.spans[p.q_tokens + i]), p.k_tokens);
      if (p.slopes != nullptr) self[r] = p.spans[2 * p.q_tokens + i];
    }
    if (lo[r] < hi[r]) {
      least = min(least, lo[r]);
      most = max(most, hi[r]);
    }
  }
  if (tid == 0) {
    range[0] = INT64_MAX;
    range[1] = 0;
  }
  if (tid < kTile) bad[tid] = 0;
  __syncthreads();
  if (tx == 0 && most > 0) {
    atomicMin(reinterpret_cast<long long*>(&range[0]), static_cast<long long>(least));
    atomicMax(reinterpret_cast<long long*>(&range[1]), static_cast<long long>(most));
  }
  const T* q = static_cast<const T*>(p.q) + h * p.q_head;
  const T* k = static_cast<const T*>(p.k) + g * p.k_head;
  const T* v = static_cast<const T*>(p.v) + g * p.v_head;
  load_tile<T, DP, true, kVec>(qs, q, p.q_token, row0, 0, p.q_tokens, p.dim);
  __syncthreads();
  const int64_t begin = range[0], stop = range[1];

  const float slope2 = p.slopes != nullptr ? p.slopes[h] * kLog2e : 0.0f;
  const float scale2 = p.softcap > 0.0f ? p.scale / p.softcap : p.scale * kLog2e;
  const float cap2 = p.softcap * kLog2e;
  float acc[4][DP / 16], top[4], total[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    top[r] = -kInf;
    total[r] = 0.0f;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) acc[r][c] = 0.0f;
  }
  for (int64_t j0 = begin; j0 < stop; j0 += kTile) {
    if (j0 != begin) __syncthreads();
    load_tile<T, DP, true, kVec>(ks, k, p.k_token, j0, begin, stop, p.dim);
    load_tile<T, DP, false, kVec>(vs, v, p.v_token, j0, begin, stop, p.dim);
    __syncthreads();
    float s[4][4] = {};
#pragma unroll 8
    for (int d = 0; d < DP; ++d) {
      const float4 a = *reinterpret_cast<const float4*>(qs + d * kTile + ty * 4);
      const float4 b = *reinterpret_cast<const float4*>(ks + d * kTile + tx * 4);
      const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[r][c] = fmaf(av[r], bv[c], s[r][c]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float most_here = -kInf;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int64_t j = j0 + tx * 4 + c;
        float x = p.softcap > 0.0f ? cap2 * tanhf(s[r][c] * scale2) : s[r][c] * scale2;
        if (p.slopes != nullptr) x -= slope2 * fabsf(static_cast<float>(self[r] - j));
        s[r][c] = j >= lo[r] && j < hi[r] ? x : -kInf;
        most_here = fmaxf(most_here, s[r][c]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) most_here = fmaxf(most_here, __shfl_xor_sync(0xFFFFFFFFu, most_here, o));
      const float next = fmaxf(top[r], most_here), base = next == -kInf ? 0.0f : next;
      const float back = exp2_approx(top[r] - base);
      float sum = 0.0f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[r][c] = exp2_approx(s[r][c] - base);
        sum += s[r][c];
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      total[r] = total[r] * back + sum;
      top[r] = next;
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) acc[r][c] *= back;
      *reinterpret_cast<float4*>(ps + (ty * 4 + r) * kTile + tx * 4) = make_float4(s[r][0], s[r][1], s[r][2], s[r][3]);
    }
    __syncwarp();  // a row's 16 threads are of one warp
#pragma unroll 2
    for (int j = 0; j < kTile; j += 4) {
      float4 w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) w[r] = *reinterpret_cast<const float4*>(ps + (ty * 4 + r) * kTile + j);
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
#pragma unroll
        for (int c = 0; c < DP / 64; ++c) {
          const float4 x = *reinterpret_cast<const float4*>(vs + (j + jj) * DP + c * 64 + tx * 4);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float wr = jj == 0 ? w[r].x : jj == 1 ? w[r].y : jj == 2 ? w[r].z : w[r].w;
            acc[r][c * 4] = fmaf(wr, x.x, acc[r][c * 4]);
            acc[r][c * 4 + 1] = fmaf(wr, x.y, acc[r][c * 4 + 1]);
            acc[r][c * 4 + 2] = fmaf(wr, x.z, acc[r][c * 4 + 2]);
            acc[r][c * 4 + 3] = fmaf(wr, x.w, acc[r][c * 4 + 3]);
          }
        }
      }
    }
    __syncwarp();
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t i = row0 + ty * 4 + r;
    if (i >= p.q_tokens) continue;
    const float over = total[r] == 0.0f ? 0.0f : 1.0f / total[r];
    T* out = static_cast<T*>(p.out) + i * p.out_token + h * p.out_head;
    bool finite = true;
#pragma unroll
    for (int c = 0; c < DP / 64; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = c * 64 + tx * 4 + e;
        const float x = acc[r][c * 4 + e] * over;
        finite = finite && fabsf(acc[r][c * 4 + e]) < kInf;
        if (d < p.dim) out[d] = narrow<T>(total[r] == 0.0f ? 0.0f : x);
      }
    if (!finite || !(total[r] < kInf)) bad[ty * 4 + r] = 1;
    if (p.lse != nullptr && tx == 0)
      p.lse[h * p.q_tokens + i] = total[r] == 0.0f ? -kInf : (top[r] + log2f(total[r])) * kLn2;
  }
  __syncthreads();
  for (int r = tid / 32; r < kTile; r += kThreads256 / 32)
    if (bad[r]) attention_row<T>(p, row0 + r, h, tid % 32);
}

template <typename T, int DP, bool kVec>
cudaError_t launch_tiles(const AttentionParams& p, cudaStream_t stream) {
  constexpr int kBytes = (3 * DP + kTile) * kTile * 4;
  const cudaError_t e = cudaFuncSetAttribute(attention_tiles_kernel<T, DP, kVec>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>((p.q_tokens + kTile - 1) / kTile), p.heads);
  attention_tiles_kernel<T, DP, kVec><<<grid, kThreads256, kBytes, stream>>>(p);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const AttentionParams& p, cudaStream_t stream) {
  constexpr int64_t E = Vec<T>::kN;
  const bool vec = p.dim % E == 0 && p.q_token % E == 0 && p.q_head % E == 0 && p.k_token % E == 0 && p.k_head % E == 0 &&
                   p.v_token % E == 0 && p.v_head % E == 0 && aligned_to(p.q, 16) && aligned_to(p.k, 16) &&
                   aligned_to(p.v, 16);
  if (p.dim <= 64) return vec ? launch_tiles<T, 64, true>(p, stream) : launch_tiles<T, 64, false>(p, stream);
  if (p.dim <= 128) return vec ? launch_tiles<T, 128, true>(p, stream) : launch_tiles<T, 128, false>(p, stream);
  return vec ? launch_tiles<T, 256, true>(p, stream) : launch_tiles<T, 256, false>(p, stream);
}

}  // namespace

cudaError_t launch_attention_tiles(const AttentionParams& p, int dtype, cudaStream_t stream) {
  if (dtype == 0) return launch_type<float>(p, stream);
  if (dtype == 1) return launch_type<__nv_bfloat16>(p, stream);
  return launch_type<__half>(p, stream);
}

}  // namespace zo
