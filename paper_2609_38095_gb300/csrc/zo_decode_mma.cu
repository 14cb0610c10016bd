// zo_decode_mma.cu -- one-token attention over a paged cache on the tensor
// cores: 16-bit types, vectors aligned to 16 bytes (zo_attention_decode).
#include "zo_decode.cuh"

namespace zo {

namespace {

constexpr int kWarps = 4;
constexpr float kSlack = 8.0f;  // log2: how far scores may pass the reference before the output is rescaled

template <int DP, int HB>
struct Tiles {
  static constexpr int kStages = 3;
  static constexpr int kRow = DP * 2;                      // bytes of a key
  static constexpr int kStage = 2 * kDecodeKeys * kRow;    // keys, then values
  static constexpr int kWarp = kStages * kStage;
  static constexpr int kBytes = kWarps * kWarp + 2 * kWarps * HB * 4;
  static_assert(HB * DP * 4 <= kWarp, "a warp's output takes its tiles' place");
};

__device__ __forceinline__ void load4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void load4_transposed(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}

template <typename T>
__device__ __forceinline__ void mma16816(float& c0, float& c1, float& c2, float& c3, uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (__is_same(T, __nv_bfloat16))
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c0), "+f"(c1), "+f"(c2), "+f"(c3)
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c0), "+f"(c1), "+f"(c2), "+f"(c3)
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A warp's tiles of 16 keys come by cp.async, two ahead of the one in use, into
// its own shared memory, 16-byte vectors swizzled by row. Scores: m16n8k16 with
// the query heads as the 16 rows (8 of them zeros where HB is 8, and their
// halves of the accumulators are not kept), which leaves the weights in the
// layout of the next product's left operand. The 16 x 16 products are far from
// what bounds this: the cache is read once, from HBM. (A 128-row tcgen05 tile
// would be empty but for `group` rows.)
template <typename T, int DP, int HB>
__global__ void __launch_bounds__(kWarps * 32) decode_mma_kernel(const __grid_constant__ DecodeParams p) {
  using L = Tiles<DP, HB>;
  constexpr int kVectors = DP / 8, kHalves = HB / 8;  // 16-byte vectors of a key; rows of a thread
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ DecodeJoin<HB> join;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t tiles = static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + warp * L::kWarp;
  float* tops = reinterpret_cast<float*>(smem + kWarps * L::kWarp);
  float* totals = tops + kWarps * HB;
  const uint32_t ranks = cluster_size();
  const DecodePlace w = decode_place<HB>(p, blockIdx.x / ranks);
  if (threadIdx.x == 0) join.bad = w.bad;

  const T* kc = static_cast<const T*>(p.k) + w.g * p.k_head;
  const T* vc = static_cast<const T*>(p.v) + w.g * p.v_head;
  const int64_t tiles_in = (w.len + kDecodeKeys - 1) / kDecodeKeys;
  const int64_t step = static_cast<int64_t>(ranks) * kWarps;
  const int64_t first = static_cast<int64_t>(cluster_rank()) * kWarps + warp;
  int bad = 0;
  const auto find = [&](int64_t tile) { return decode_key(p, w, tile * kDecodeKeys + (lane & 15), bad); };
  const auto fetch = [&](int2 key, int stage) {
    constexpr int kRowsAtOnce = 32 / kVectors > 0 ? 32 / kVectors : 1;
    const uint32_t ks = tiles + stage * L::kStage, vs = ks + kDecodeKeys * L::kRow;
    const int c = lane % kVectors;
#pragma unroll
    for (int i = 0; i < kDecodeKeys / kRowsAtOnce; ++i) {
      const int r = i * kRowsAtOnce + lane / kVectors;
      const int page = __shfl_sync(0xFFFFFFFFu, key.x, r), row = __shfl_sync(0xFFFFFFFFu, key.y, r);
      const int n = page >= 0 && c * 8 < p.dim ? 16 : 0;  // the rest is filled with zeros
      const uint32_t at = r * L::kRow + ((c ^ (r & 7)) << 4);
      const void* k = n ? static_cast<const void*>(kc + page * p.k_page + row * p.k_token + c * 8) : p.k;
      const void* v = n ? static_cast<const void*>(vc + page * p.v_page + row * p.v_token + c * 8) : p.v;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ks + at), "l"(k), "r"(n) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(vs + at), "l"(v), "r"(n) : "memory");
    }
  };

  int2 ahead = find(first);
#pragma unroll
  for (int s = 0; s < L::kStages - 1; ++s) {
    const int2 key = ahead;
    ahead = find(first + (s + 1) * step);
    if (first + s * step < tiles_in) fetch(key, s);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // the queries as left operands: rows lane / 4 and lane / 4 + 8, columns 2 (lane mod 4) and 8 more
  uint32_t qa[DP / 16][2 * kHalves];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s)
#pragma unroll
    for (int r = 0; r < kHalves; ++r)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int h = lane / 4 + 8 * r, d = s * 16 + c * 8 + lane % 4 * 2;
        qa[s][c * kHalves + r] = 0;
        if (h < w.heads && d < p.dim) {
          const T* q = static_cast<const T*>(p.q) + w.b * p.q_token + (w.head0 + h) * p.q_head + d;
          uint16_t e[2];
          e[0] = *reinterpret_cast<const uint16_t*>(q);
          e[1] = *reinterpret_cast<const uint16_t*>(q + 1);
          qa[s][c * kHalves + r] = e[0] | static_cast<uint32_t>(e[1]) << 16;
        }
      }
  const float scale2 = p.softcap > 0.0f ? p.scale / p.softcap : p.scale * kLog2e, cap2 = p.softcap * kLog2e;
  float slope2[kHalves], base[kHalves], total[kHalves], acc[DP / 8][2 * kHalves];
#pragma unroll
  for (int r = 0; r < kHalves; ++r) {
    const int h = lane / 4 + 8 * r;
    slope2[r] = p.slopes != nullptr && h < w.heads ? p.slopes[w.head0 + h] * kLog2e : 0.0f;
    base[r] = -kInf;
    total[r] = 0.0f;
  }
#pragma unroll
  for (int n = 0; n < DP / 8; ++n)
#pragma unroll
    for (int c = 0; c < 2 * kHalves; ++c) acc[n][c] = 0.0f;

  int stage = 0;
  for (int64_t tile = first; tile < tiles_in; tile += step) {
    {
      const int2 key = ahead;
      const int64_t next = tile + (L::kStages - 1) * step;
      ahead = find(next + step);
      if (next < tiles_in) fetch(key, stage == 0 ? L::kStages - 1 : stage - 1);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 1) : "memory");
    __syncwarp();
    const uint32_t ks = tiles + stage * L::kStage, vs = ks + kDecodeKeys * L::kRow;
    float s[2][4] = {};  // keys 0-7 and 8-15; a thread's two of each row
    {
      const int row = (lane & 7) + (lane >> 4 << 3);
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        uint32_t b[4];
        load4(b, ks + row * L::kRow + (((2 * d + (lane >> 3 & 1)) ^ (row & 7)) << 4));
#pragma unroll
        for (int n = 0; n < 2; ++n)
          mma16816<T>(s[n][0], s[n][1], s[n][2], s[n][3], qa[d][0], kHalves == 2 ? qa[d][1] : 0u, qa[d][kHalves],
                      kHalves == 2 ? qa[d][3] : 0u, b[2 * n], b[2 * n + 1]);
      }
    }
    const int64_t j0 = tile * kDecodeKeys + lane % 4 * 2;
    float back[kHalves];
    bool moved = false;
#pragma unroll
    for (int r = 0; r < kHalves; ++r) {
      float most = -kInf;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int64_t j = j0 + n * 8 + c;
          float x = s[n][2 * r + c];
          x = p.softcap > 0.0f ? capped(x, scale2, cap2) : x * scale2;
          x = j < w.len ? x - slope2[r] * static_cast<float>(w.len - 1 - j) : -kInf;
          s[n][2 * r + c] = x;
          most = fmaxf(most, x);
        }
      most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
      most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
      back[r] = 1.0f;
      if (most > base[r] + kSlack || (base[r] == -kInf && most > -kInf)) {
        back[r] = exp2_approx(base[r] - most);
        base[r] = most;
        moved = true;
      }
      total[r] *= back[r];
    }
    if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
      for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int r = 0; r < kHalves; ++r) {
          acc[n][2 * r] *= back[r];
          acc[n][2 * r + 1] *= back[r];
        }
    }
    uint32_t weight[2][kHalves];
#pragma unroll
    for (int r = 0; r < kHalves; ++r) {
      const float shift = base[r] == -kInf ? 0.0f : base[r];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float a = exp2_approx(s[n][2 * r] - shift), b = exp2_approx(s[n][2 * r + 1] - shift);
        total[r] += a + b;
        weight[n][r] = narrow2<T>(a, b);
      }
    }
    {
      const int row = (lane & 7) + (lane >> 3 & 1) * 8;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        uint32_t b[4];
        load4_transposed(b, vs + row * L::kRow + (((2 * d + (lane >> 4)) ^ (row & 7)) << 4));
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          float none0 = 0.0f, none1 = 0.0f;
          float* a = acc[2 * d + n];
          mma16816<T>(a[0], a[1], kHalves == 2 ? a[2 * (kHalves - 1)] : none0, kHalves == 2 ? a[2 * kHalves - 1] : none1,
                      weight[0][0], kHalves == 2 ? weight[0][kHalves - 1] : 0u, weight[1][0],
                      kHalves == 2 ? weight[1][kHalves - 1] : 0u, b[2 * n], b[2 * n + 1]);
        }
      }
    }
    __syncwarp();  // the stage may be filled again
    stage = stage + 1 == L::kStages ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int r = 0; r < kHalves; ++r) {
    float sum = total[r];
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
    if (lane % 4 == 0) {
      tops[warp * HB + lane / 4 + 8 * r] = base[r];
      totals[warp * HB + lane / 4 + 8 * r] = sum;
    }
  }
  __syncthreads();  // join.bad is set, and every warp is done with its tiles: the outputs take their place
  if (bad) join.bad = 1;
  float* outs = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int n = 0; n < DP / 8; ++n)
#pragma unroll
    for (int r = 0; r < kHalves; ++r)
      *reinterpret_cast<float2*>(outs + (warp * HB + lane / 4 + 8 * r) * DP + n * 8 + lane % 4 * 2) =
          make_float2(acc[n][2 * r], acc[n][2 * r + 1]);
  decode_join<T, HB, DP, kWarps>(p, w, outs, tops, totals, join);
}

template <typename T, int DP, int HB>
cudaError_t launch_size(DecodeParams p, int64_t batch, int sms, cudaStream_t stream) {
  p.head_blocks = (p.group + HB - 1) / HB;
  const int64_t items = batch * p.kv_heads * p.head_blocks;
  const int c = decode_cluster(items, p.max_pages * p.page_size, sms, 4, 128);
  return launch_decode(decode_mma_kernel<T, DP, HB>, p, items, c, kWarps * 32, Tiles<DP, HB>::kBytes, stream);
}

template <typename T>
cudaError_t launch_type(const DecodeParams& p, int64_t batch, int sms, cudaStream_t stream) {
  if (p.dim <= 64)
    return p.group <= 8 ? launch_size<T, 64, 8>(p, batch, sms, stream) : launch_size<T, 64, 16>(p, batch, sms, stream);
  if (p.dim <= 128)
    return p.group <= 8 ? launch_size<T, 128, 8>(p, batch, sms, stream) : launch_size<T, 128, 16>(p, batch, sms, stream);
  return launch_size<T, 256, 8>(p, batch, sms, stream);
}

}  // namespace

bool launch_decode_mma(const DecodeParams& p, int64_t batch, int dtype, int sms, cudaStream_t stream, cudaError_t* e) {
  if (dtype == 0 || p.dim % 8 != 0 || p.k_page % 8 != 0 || p.k_token % 8 != 0 || p.k_head % 8 != 0 || p.v_page % 8 != 0 ||
      p.v_token % 8 != 0 || p.v_head % 8 != 0 || !aligned_to(p.k, 16) || !aligned_to(p.v, 16))
    return false;
  *e = dtype == 1 ? launch_type<__nv_bfloat16>(p, batch, sms, stream) : launch_type<__half>(p, batch, sms, stream);
  return true;
}

}  // namespace zo
