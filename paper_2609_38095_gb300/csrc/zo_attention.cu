// zo_attention.cu -- attention of packed documents on the fp32 units: every
// type, head size, stride and alignment (zo_attention).
#include "zo_forward.cuh"

namespace zo {

namespace {

constexpr int kTile = 64;        // query rows and keys of a tile
constexpr int kThreads256 = 256;
constexpr int kMaxParts = 2;     // CTAs of a cluster, which share a tile's keys

// rows [from, from + kTile) of a head as fp32, either transposed ([d][row]) or
// as they are ([row][d]); zero outside [lo, hi) and beyond the head's size.
template <typename T, int DP, bool kTransposed, bool kVec>
__device__ __forceinline__ void load_tile(float* dst, const T* src, int64_t stride, int64_t from, int64_t lo, int64_t hi,
                                          int dim) {
  constexpr int E = kVec ? Vec<T>::kN : 1;
  constexpr int kChunks = DP / E, kEach = kChunks * kTile / kThreads256;  // loads of a thread
  constexpr int kBatch = kEach % 8 == 0 ? 8 : kEach % 6 == 0 ? 6 : kEach;  // of them on their way together
  for (int n0 = 0; n0 < kEach; n0 += kBatch) {
    uint4 raw[kBatch];
    float one[kBatch];
    int row[kBatch], chunk[kBatch];
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      const int i = threadIdx.x + (n0 + n) * kThreads256;
      // transposed, lanes on rows: stores without bank conflicts, a row's sectors from L1
      row[n] = kTransposed ? i % kTile : i / kChunks;
      chunk[n] = kTransposed ? i / kTile : i % kChunks;
      const int64_t r = from + row[n];
      const bool in = r >= lo && r < hi && chunk[n] * E < dim;
      if constexpr (kVec) {
        raw[n] = make_uint4(0, 0, 0, 0);
        if (in) raw[n] = *reinterpret_cast<const uint4*>(src + r * stride + chunk[n] * E);
      } else {
        one[n] = in ? widen(src[r * stride + chunk[n]]) : 0.0f;
      }
    }
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      float f[E];
      if constexpr (kVec) Vec<T>::widen_all(raw[n], f);
      else f[0] = one[n];
      if constexpr (kTransposed) {
#pragma unroll
        for (int e = 0; e < E; ++e) dst[(chunk[n] * E + e) * kTile + row[n]] = f[e];
      } else if constexpr (kVec) {
#pragma unroll
        for (int e = 0; e < E; e += 4)
          *reinterpret_cast<float4*>(dst + row[n] * DP + chunk[n] * E + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
      } else {
        dst[row[n] * DP + chunk[n]] = f[0];
      }
    }
  }
}

// 64 query rows of one head; keys in tiles of 64, scores and products by fp32
// multiply-adds, 4 x 4 scores and 4 x DP/16 output elements per thread. Row
// statistics run along; a row's 16 threads share them by shuffles. Where the
// SMs would have few CTAs, a cluster takes a row's tiles of keys in turn and
// joins its outputs over distributed shared memory, each CTA a part of the rows.
// Bound by the multiply-adds and the shared-memory loads that feed them: 3000
// causal tokens of 32 heads of 128 in fp32 2.29 ms = 32 TFLOP/s, 5 documents of at
// most 333 over 100 cached keys (16 heads of 80, capped and biased) 88 to 99 us. Eight
// rows per thread on half the threads: 2.90 ms and 102 us, for want of warps.
template <typename T, int DP, bool kVec>
__global__ void __launch_bounds__(kThreads256, DP <= 128 ? 2 : 1)
    attention_tiles_kernel(const __grid_constant__ AttentionParams p) {
  constexpr int V = DP % 64 == 0 ? 4 : 2;  // output elements of a thread that lie together
  extern __shared__ __align__(16) float smem[];
  float* qs = smem;                 // [DP][64]
  float* ks = qs + DP * kTile;      // [DP][64]
  float* vs = ks + DP * kTile;      // [64][DP]
  float* ps = vs + DP * kTile;      // [64 rows][64 keys]
  __shared__ int64_t range[2];
  __shared__ float tops[kTile], totals[kTile];  // of this CTA's keys
  __shared__ float lses[kTile];
  __shared__ uint32_t left[kTile / 32];  // rows for attention_rows
  const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16, h = blockIdx.y, g = h / p.group;
  const int ranks = static_cast<int>(cluster_size()), rank = static_cast<int>(cluster_rank());
  const int64_t row0 = (static_cast<int64_t>(gridDim.x - 1 - blockIdx.x) / ranks) * kTile;  // the longest causal rows first
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
    for (int i = 0; i < kTile / 32; ++i) left[i] = 0;
  }
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
  const int64_t stop = range[1], begin = stop > 0 ? range[0] : 0;

  // scores in their own units here, not in log2: with fp32 results their rounding would show
  const float slope = p.slopes != nullptr ? p.slopes[h] : 0.0f, over_cap = p.softcap > 0.0f ? 1.0f / p.softcap : 0.0f;
  float acc[4][DP / 16], top[4], total[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    top[r] = -kInf;
    total[r] = 0.0f;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) acc[r][c] = 0.0f;
  }
  const int dims = (p.dim + 7) / 8 * 8;
  for (int64_t j0 = begin + rank * kTile; j0 < stop; j0 += ranks * kTile) {
    __syncthreads();  // the tile before is done with
    load_tile<T, DP, true, kVec>(ks, k, p.k_token, j0, begin, stop, p.dim);
    load_tile<T, DP, false, kVec>(vs, v, p.v_token, j0, begin, stop, p.dim);
    __syncthreads();
    int low[4], high[4], own[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      low[r] = static_cast<int>(min(max(lo[r] - j0, INT64_C(0)), INT64_C(64)));
      high[r] = static_cast<int>(min(max(hi[r] - j0, INT64_C(0)), INT64_C(64)));
      own[r] = static_cast<int>(self[r] - j0);
    }
    float s[4][4] = {};
#pragma unroll 8
    for (int d = 0; d < dims; ++d) {
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
        const int j = tx * 4 + c;  // from the tile's first key, as the bounds
        float x = s[r][c] * p.scale;
        if (p.softcap > 0.0f) x = p.softcap * tanhf(x * over_cap);
        if (p.slopes != nullptr) x -= slope * fabsf(static_cast<float>(own[r] - j));
        s[r][c] = j >= low[r] && j < high[r] ? x : -kInf;
        most_here = fmaxf(most_here, s[r][c]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) most_here = fmaxf(most_here, __shfl_xor_sync(0xFFFFFFFFu, most_here, o));
      const float next = fmaxf(top[r], most_here), base = next == -kInf ? 0.0f : next;
      const float back = exp2_approx((top[r] - base) * kLog2e);
      float sum = 0.0f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[r][c] = exp2_approx((s[r][c] - base) * kLog2e);
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
        for (int c = 0; c < DP / 16; c += V) {
          float x[V];
          const float* at = vs + (j + jj) * DP + c * 16 + tx * V;
          if constexpr (V == 4) {
            const float4 y = *reinterpret_cast<const float4*>(at);
            x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
          } else {
            const float2 y = *reinterpret_cast<const float2*>(at);
            x[0] = y.x, x[1] = y.y;
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float wr = jj == 0 ? w[r].x : jj == 1 ? w[r].y : jj == 2 ? w[r].z : w[r].w;
#pragma unroll
            for (int e = 0; e < V; ++e) acc[r][c + e] = fmaf(wr, x[e], acc[r][c + e]);
          }
        }
      }
    }
    __syncwarp();
  }
  // this CTA's outputs and statistics, where its peers find them: in the place of the tiles
  __syncthreads();
  float* outs = ks;  // [64][DP]
#pragma unroll
  for (int r = 0; r < 4; ++r) {
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) outs[(ty * 4 + r) * DP + c / V * V * 16 + tx * V + c % V] = acc[r][c];
    if (tx == 0) {
      tops[ty * 4 + r] = top[r];
      totals[ty * 4 + r] = total[r];
    }
  }
  if (ranks > 1) cluster_sync();
  else __syncthreads();
  const int lane = tid % 32;
  for (int r = rank + tid / 32 * ranks; r < kTile; r += kThreads256 / 32 * ranks) {  // a warp per row
    const int64_t i = row0 + r;
    if (i >= p.q_tokens) break;
    float most = -kInf, sum = 0.0f, scale[kMaxParts];
#pragma unroll
    for (int n = 0; n < kMaxParts; ++n) {
      scale[n] = n < ranks ? peer_load(peer_address(&tops[r], n)) : -kInf;
      most = fmaxf(most, scale[n]);
    }
#pragma unroll
    for (int n = 0; n < kMaxParts; ++n) {
      scale[n] = most == -kInf ? 1.0f : exp2_approx((scale[n] - most) * kLog2e);  // without a maximum sums are 0, or NaN
      if (n < ranks) sum += peer_load(peer_address(&totals[r], n)) * scale[n];
    }
    const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
    bool finite = true;
    T* out = static_cast<T*>(p.out) + i * p.out_token + h * p.out_head;
#pragma unroll
    for (int d = lane; d < DP; d += 32) {
      float x = 0.0f;
#pragma unroll
      for (int n = 0; n < kMaxParts; ++n)
        if (n < ranks) x += peer_load(peer_address(&outs[r * DP + d], n)) * scale[n];
      finite = finite && (sum == 0.0f || fabsf(x) < kInf);
      if (d < p.dim) out[d] = narrow<T>(sum == 0.0f ? 0.0f : x * over);
    }
    const float lse = sum == 0.0f ? -kInf : most + logf(sum);
    if (p.lse != nullptr && lane == 0) p.lse[h * p.q_tokens + i] = lse;
    if (!__all_sync(0xFFFFFFFFu, finite) && sum < kInf && lane == 0) {  // (a sum that is NaN is that of seen scores)
      lses[r] = lse;
      atomicOr(&left[r / 32], 1u << r % 32);
    }
  }
  if (ranks > 1) cluster_sync();  // no CTA leaves before its part is read
  else __syncthreads();
  if ((left[0] | left[1]) != 0)
    attention_rows<T, DP, 1>(p, row0, h, left, lses, kTile / 32, tid / 32, kThreads256 / 32, lane);
}

template <typename T, int DP, bool kVec>
cudaError_t launch_tiles(const AttentionParams& p, int sms, cudaStream_t stream) {
  constexpr int kBytes = (3 * DP + kTile) * kTile * 4;
  const cudaError_t e = cudaFuncSetAttribute(attention_tiles_kernel<T, DP, kVec>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
  if (e != cudaSuccess) return e;
  const int64_t tiles = (p.q_tokens + kTile - 1) / kTile;
  // CTAs for two rounds of the SMs, none with less than two tiles of the keys there are (5 documents of at most 333, 16 heads
  // of 80: 109 us without, 97 with two CTAs, 99 with four)
  int parts = 1;
  while (parts < kMaxParts && tiles * p.heads * parts < 4 * sms && p.k_tokens >= parts * 4 * kTile) parts *= 2;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = parts;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(static_cast<unsigned>(tiles * parts), p.heads);
  c.blockDim = dim3(kThreads256);
  c.dynamicSmemBytes = kBytes;
  c.stream = stream;
  c.attrs = &attr;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, attention_tiles_kernel<T, DP, kVec>, p);
}

template <typename T>
cudaError_t launch_type(const AttentionParams& p, int sms, cudaStream_t stream) {
  constexpr int64_t E = Vec<T>::kN;
  const bool vec = p.dim % E == 0 && p.q_token % E == 0 && p.q_head % E == 0 && p.k_token % E == 0 && p.k_head % E == 0 &&
                   p.v_token % E == 0 && p.v_head % E == 0 && aligned_to(p.q, 16) && aligned_to(p.k, 16) &&
                   aligned_to(p.v, 16);
  if (p.dim <= 64) return vec ? launch_tiles<T, 64, true>(p, sms, stream) : launch_tiles<T, 64, false>(p, sms, stream);
  if (p.dim <= 96) return vec ? launch_tiles<T, 96, true>(p, sms, stream) : launch_tiles<T, 96, false>(p, sms, stream);
  if (p.dim <= 128) return vec ? launch_tiles<T, 128, true>(p, sms, stream) : launch_tiles<T, 128, false>(p, sms, stream);
  return vec ? launch_tiles<T, 256, true>(p, sms, stream) : launch_tiles<T, 256, false>(p, sms, stream);
}

}  // namespace

cudaError_t launch_attention_tiles(const AttentionParams& p, int dtype, int sms, cudaStream_t stream) {
  if (dtype == 0) return launch_type<float>(p, sms, stream);
  if (dtype == 1) return launch_type<__nv_bfloat16>(p, sms, stream);
  return launch_type<__half>(p, sms, stream);
}

}  // namespace zo
