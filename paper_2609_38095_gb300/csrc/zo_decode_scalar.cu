// zo_decode_scalar.cu -- one-token attention over a paged cache on the fp32
// units: every type, head size, stride and alignment (zo_attention_decode).
#include "zo_decode.cuh"

namespace zo {

namespace {

constexpr int kDecodeKeys = 16;  // keys of a warp's tile

template <int DP, int HB>
struct Scalar {
  static constexpr int kWarps = DP == 256 ? 2 : 4;
  static constexpr int kStages = 2;
  static constexpr int kPitch = DP + 4;  // floats from one key to the next: 16 keys' vectors on distinct banks
  static constexpr int kStage = kDecodeKeys * (kPitch + DP);
  static constexpr int kWarp = kStages * kStage + kDecodeKeys * HB;  // and the keys' weights
  static constexpr int kBytes = 4 * (kWarps * kWarp + HB * DP + 2 * kWarps * HB);
  static_assert(HB * DP * kWarps <= kWarps * kWarp, "a warp's output takes its tiles' place");
};

// A warp's tile of 16 keys lies in its own shared memory as fp32, the next one
// on its way (fp32 caches by cp.async; others are widened on the way and stored
// before the products start). Scores: a lane has half of a key's dot product
// with every head; outputs: a lane has DP / 32 elements of every head. Bound by
// shared memory and instructions before HBM (134 KB of tiles and queries leave one
// CTA of 4 warps per SM at heads of 128): 16 sequences of up to 4001 keys, fp32, 32 / 8
// heads of 128 in 112 us = 2.5 TB/s, 40 / 40 heads (2000 keys) 194 us = 3.6.
template <typename T, int DP, int HB, bool kAsync>
__global__ void __launch_bounds__(Scalar<DP, HB>::kWarps * 32)
    decode_scalar_kernel(const __grid_constant__ DecodeParams p) {
  using S = Scalar<DP, HB>;
  extern __shared__ __align__(16) float smem[];
  __shared__ DecodeJoin<HB> join;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* qs = smem;  // [HB][DP]
  float* tops = qs + HB * DP;
  float* totals = tops + S::kWarps * HB;
  float* tiles = totals + S::kWarps * HB;
  float* mine = tiles + warp * S::kWarp;
  float* weights = mine + S::kStages * S::kStage;  // [16][HB]
  const uint32_t ranks = cluster_size();
  const DecodePlace w = decode_place<HB>(p, blockIdx.x / ranks);
  if (threadIdx.x == 0) join.bad = w.bad;
  const T* q = static_cast<const T*>(p.q) + w.b * p.q_token;
  for (int i = threadIdx.x; i < HB * DP; i += S::kWarps * 32) {
    const int h = i / DP, d = i - h * DP;
    qs[i] = h < w.heads && d < p.dim ? widen(q[(w.head0 + h) * p.q_head + d]) : 0.0f;
  }
  __syncthreads();

  const T* kc = static_cast<const T*>(p.k) + w.g * p.k_head;
  const T* vc = static_cast<const T*>(p.v) + w.g * p.v_head;
  const int64_t tiles_in = (w.len + kDecodeKeys - 1) / kDecodeKeys;
  const int64_t step = static_cast<int64_t>(ranks) * S::kWarps;
  int bad = 0;

  // a page is looked up a tile before its number is used, which would wait for the load
  const auto look = [&](int64_t tile) {
    const int64_t j = tile * kDecodeKeys + (lane & 15);
    return j < w.len ? p.pages[w.b * p.pages_stride + decode_page(p, j)] : 0;
  };
  const auto fetch = [&](int64_t tile, int id, int stage) {
    float* ks = mine + stage * S::kStage;
    float* vs = ks + kDecodeKeys * S::kPitch;
    const int2 key = decode_key(p, w, tile * kDecodeKeys + (lane & 15), id, bad);
    const int64_t k_at = key.x >= 0 ? key.x * p.k_page + key.y * p.k_token : -1;
    const int64_t v_at = key.x >= 0 ? key.x * p.v_page + key.y * p.v_token : 0;
    for (int r = 0; r < kDecodeKeys; ++r) {
      const int64_t at = __shfl_sync(0xFFFFFFFFu, k_at, r);
      const T* k = kc + at;
      const T* v = vc + __shfl_sync(0xFFFFFFFFu, v_at, r);
      if constexpr (kAsync) {
#pragma unroll
        for (int c = lane; c < DP / 4; c += 32) {
          const int n = at >= 0 && c * 4 < p.dim ? 16 : 0;  // the rest is filled with zeros
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                           static_cast<uint32_t>(__cvta_generic_to_shared(ks + r * S::kPitch + c * 4))),
                       "l"(n ? static_cast<const void*>(k + c * 4) : p.k), "r"(n)
                       : "memory");
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                           static_cast<uint32_t>(__cvta_generic_to_shared(vs + r * DP + c * 4))),
                       "l"(n ? static_cast<const void*>(v + c * 4) : p.v), "r"(n)
                       : "memory");
        }
      } else {
#pragma unroll
        for (int d = lane; d < DP; d += 32) {
          const bool in = at >= 0 && d < p.dim;
          ks[r * S::kPitch + d] = in ? widen(k[d]) : 0.0f;
          vs[r * DP + d] = in ? widen(v[d]) : 0.0f;
        }
      }
    }
    if constexpr (kAsync) asm volatile("cp.async.commit_group;" ::: "memory");
  };

  // scores in their own units here, not in log2: with fp32 results their rounding would show
  const float over_cap = p.softcap > 0.0f ? 1.0f / p.softcap : 0.0f;
  float slope[HB], top[HB], total[HB], acc[HB][DP / 32];
#pragma unroll
  for (int h = 0; h < HB; ++h) {
    slope[h] = p.slopes != nullptr && h < w.heads ? p.slopes[w.head0 + h] : 0.0f;
    top[h] = -kInf;
    total[h] = 0.0f;
#pragma unroll
    for (int c = 0; c < DP / 32; ++c) acc[h][c] = 0.0f;
  }
  int64_t tile = static_cast<int64_t>(cluster_rank()) * S::kWarps + warp;
  int stage = 0;
  int id = look(tile);
  if (tile < tiles_in) fetch(tile, id, 0);
  id = look(tile + step);
  for (; tile < tiles_in; tile += step, stage ^= 1) {
    const int here = id;
    id = look(tile + 2 * step);
    if (tile + step < tiles_in) {
      fetch(tile + step, here, stage ^ 1);
      if constexpr (kAsync) asm volatile("cp.async.wait_group 1;" ::: "memory");
    } else {
      if constexpr (kAsync) asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    const float* ks = mine + stage * S::kStage;
    const float* vs = ks + kDecodeKeys * S::kPitch;
    const int key = lane & 15, half = lane >> 4;
    const int64_t j = tile * kDecodeKeys + key;
    float s[HB] = {};
#pragma unroll 4
    for (int c = half * (DP / 8); c < (half + 1) * (DP / 8); ++c) {
      const float4 x = *reinterpret_cast<const float4*>(ks + key * S::kPitch + c * 4);
#pragma unroll
      for (int h = 0; h < HB; ++h) {
        const float4 y = *reinterpret_cast<const float4*>(qs + h * DP + c * 4);
        s[h] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s[h]))));
      }
    }
    const float away = static_cast<float>(w.len - 1 - j);
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      float x = s[h] + __shfl_xor_sync(0xFFFFFFFFu, s[h], 16);
      x *= p.scale;
      if (p.softcap > 0.0f) x = p.softcap * tanhf(x * over_cap);
      x = j < w.len ? x - slope[h] * away : -kInf;
      float most = x;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
      const float next = fmaxf(top[h], most), base = next == -kInf ? 0.0f : next;
      if (next > top[h]) {  // the same for the whole warp
        const float back = exp2_approx((top[h] - base) * kLog2e);
        total[h] *= back;
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) acc[h][c] *= back;
        top[h] = next;
      }
      s[h] = exp2_approx((x - base) * kLog2e);
      total[h] += half == 0 ? s[h] : 0.0f;
    }
    if (half == 0) {
#pragma unroll
      for (int h = 0; h < HB; ++h) weights[key * HB + h] = s[h];
    }
    __syncwarp();
#pragma unroll 4
    for (int r = 0; r < kDecodeKeys; ++r) {
      float wr[HB];
#pragma unroll
      for (int h = 0; h < HB; ++h) wr[h] = weights[r * HB + h];
#pragma unroll
      for (int c = 0; c < DP / 32; ++c) {
        const float x = vs[r * DP + c * 32 + lane];
#pragma unroll
        for (int h = 0; h < HB; ++h) acc[h][c] = fmaf(wr[h], x, acc[h][c]);
      }
    }
    __syncwarp();  // the tile and the weights may be overwritten
  }
#pragma unroll
  for (int h = 0; h < HB; ++h) {
    float sum = total[h];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) {
      tops[warp * HB + h] = top[h];
      totals[warp * HB + h] = sum;
    }
  }
  if (bad) join.bad = 1;
  __syncthreads();  // every warp is done with its tiles: the outputs take their place
#pragma unroll
  for (int h = 0; h < HB; ++h)
#pragma unroll
    for (int c = 0; c < DP / 32; ++c) tiles[(warp * HB + h) * DP + c * 32 + lane] = acc[h][c];
  decode_join<T, HB, DP, S::kWarps, false>(p, w, tiles, tops, totals, join);
}

template <typename T, int DP, int HB, bool kAsync>
cudaError_t launch_heads(DecodeParams p, int64_t batch, int sms, cudaStream_t stream) {
  using S = Scalar<DP, HB>;
  p.head_blocks = (p.group + HB - 1) / HB;
  const int64_t items = batch * p.kv_heads * p.head_blocks;
  const int c = decode_cluster(items, p.max_pages * p.page_size, sms, 6);
  return launch_decode(decode_scalar_kernel<T, DP, HB, kAsync>, p, items, c, S::kWarps * 32, S::kBytes, stream);
}

// A cluster's query heads: no more than the group has, whose products would be of zeros.
template <typename T, int DP, bool kAsync>
cudaError_t launch_size(const DecodeParams& p, int64_t batch, int sms, cudaStream_t stream) {
  if (p.group == 1) return launch_heads<T, DP, 1, kAsync>(p, batch, sms, stream);
  return p.group <= 4 ? launch_heads<T, DP, 4, kAsync>(p, batch, sms, stream)
                      : launch_heads<T, DP, 8, kAsync>(p, batch, sms, stream);
}

template <typename T>
cudaError_t launch_type(const DecodeParams& p, int64_t batch, int sms, cudaStream_t stream) {
  if constexpr (sizeof(T) == 4) {
    if (p.dim % 4 == 0 && p.k_page % 4 == 0 && p.k_token % 4 == 0 && p.k_head % 4 == 0 && p.v_page % 4 == 0 &&
        p.v_token % 4 == 0 && p.v_head % 4 == 0 && aligned_to(p.k, 16) && aligned_to(p.v, 16)) {
      if (p.dim <= 64) return launch_size<T, 64, true>(p, batch, sms, stream);
      if (p.dim <= 128) return launch_size<T, 128, true>(p, batch, sms, stream);
      return launch_size<T, 256, true>(p, batch, sms, stream);
    }
  }
  if (p.dim <= 64) return launch_size<T, 64, false>(p, batch, sms, stream);
  if (p.dim <= 128) return launch_size<T, 128, false>(p, batch, sms, stream);
  return launch_size<T, 256, false>(p, batch, sms, stream);
}

}  // namespace

cudaError_t launch_decode_scalar(const DecodeParams& p, int64_t batch, int dtype, int sms, cudaStream_t stream) {
  if (dtype == 0) return launch_type<float>(p, batch, sms, stream);
  if (dtype == 1) return launch_type<__nv_bfloat16>(p, batch, sms, stream);
  return launch_type<__half>(p, batch, sms, stream);
}

}  // namespace zo
