// zo_decode_mma.cu -- one-token attention over a paged cache on the tensor
// cores: 16-bit types, vectors aligned to 16 bytes (zo_attention_decode).
#include "zo_decode.cuh"

namespace zo {

namespace {

constexpr int kWarps = 4;

template <int DP, int HB>
struct Tiles {
  static constexpr int kBlocksOfKeys = DP == 64 ? 2 : 1;  // of 16, in a tile
  static constexpr int kKeys = 16 * kBlocksOfKeys;
  static constexpr int kStages = 2;
  static constexpr int kRow = DP * 2;                      // bytes of a key
  static constexpr int kStage = 2 * kKeys * kRow;      // keys, then values
  static constexpr int kWarp = kStages * kStage;
  static constexpr int kBytes = kWarps * kWarp + 2 * kWarps * HB * 4;
  static_assert(HB * DP * 4 <= kWarp, "a warp's output takes its tiles' place");
};

// An 8 x 8 matrix of 16-bit values, a row's pair per thread, transposed within the warp.
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// A warp's tiles of 16 keys come by cp.async into its own shared memory, the
// next one on its way, 16-byte vectors swizzled by row. The keys are the 16 rows
// of m16n8k16 and 8 query heads its columns (with the heads as rows, half the
// products would be of zeros for groups of up to 8): S^T = K Q^T, then
// O^T += V^T P^T, for which the weights are transposed by movmatrix. (A 128-row
// tcgen05 tile would be empty but for the group's columns.) Bound by HBM's
// latency and the chain of a tile, so many warps: three CTAs per SM (48 sequences
// of up to 16384 keys, 32 / 8 heads of 128, bf16: 244 us = 6.0 TB/s; 16 of up to
// 4001, 32 heads of 64, fp16, capped and biased: 55 us = 5.1). A third tile on its
// way leaves room for two CTAs: 274 us.
template <typename T, int DP, int HB>
__global__ void __launch_bounds__(kWarps * 32, HB == 8 && DP <= 128 ? 3 : 1) decode_mma_kernel(const __grid_constant__ DecodeParams p) {
  using L = Tiles<DP, HB>;
  constexpr int kVectors = DP / 8, kBlocks = HB / 8, kDeep = L::kBlocksOfKeys;  // a key's 16-byte vectors; blocks of 8 heads
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
  const int64_t tiles_in = (w.len + L::kKeys - 1) / L::kKeys;
  const int64_t step = static_cast<int64_t>(ranks) * kWarps;
  const int64_t first = static_cast<int64_t>(cluster_rank()) * kWarps + warp;
  const int len = static_cast<int>(w.len);
  int bad = 0;
  // A lane looks up the page of one of a tile's keys a whole tile before it needs it (a use any earlier would wait for the
  // load), and then finds where the key's vectors start, in bytes (-1: no key). The caches mostly have the same strides.
  const bool same = p.k_page == p.v_page && p.k_token == p.v_token;
  struct Place {
    int64_t k, v;
  };
  const auto look = [&](int64_t tile) {
    const int64_t j = tile * L::kKeys + lane % L::kKeys;
    return j < w.len ? p.pages[w.b * p.pages_stride + decode_page(p, j)] : 0;
  };
  const auto find = [&](int64_t tile, int id) {
    const int2 key = decode_key(p, w, tile * L::kKeys + lane % L::kKeys, id, bad);
    Place at = {-1, -1};
    if (key.x >= 0) {
      at.k = (key.x * p.k_page + key.y * p.k_token) * 2;
      at.v = same ? at.k : (key.x * p.v_page + key.y * p.v_token) * 2;
    }
    return at;
  };
  const int vector = lane % kVectors;
  const char* kl = reinterpret_cast<const char*>(kc + (vector * 8 < p.dim ? vector * 8 : 0));
  const char* vl = reinterpret_cast<const char*>(vc + (vector * 8 < p.dim ? vector * 8 : 0));
  const int bytes = vector * 8 < p.dim ? 16 : 0;  // of a vector; the rest is filled with zeros
  const auto fetch = [&](const Place& place, int stage) {
    constexpr int kRowsAtOnce = 32 / kVectors > 0 ? 32 / kVectors : 1;
    const uint32_t ks = tiles + stage * L::kStage, vs = ks + L::kKeys * L::kRow;
#pragma unroll
    for (int i = 0; i < L::kKeys / kRowsAtOnce; ++i) {
      const int r = i * kRowsAtOnce + lane / kVectors;
      const int64_t k = __shfl_sync(0xFFFFFFFFu, place.k, r);
      const int64_t v = same ? k : __shfl_sync(0xFFFFFFFFu, place.v, r);
      const uint32_t at = r * L::kRow + ((vector ^ (r & 7)) << 4);
      const int n = k >= 0 ? bytes : 0;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ks + at), "l"(kl + (k >= 0 ? k : 0)), "r"(n)
                   : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(vs + at), "l"(vl + (k >= 0 ? v : 0)), "r"(n)
                   : "memory");
    }
  };

  int id = look(first);
#pragma unroll
  for (int s = 0; s < L::kStages - 1; ++s) {
    const int64_t tile = first + s * step;
    const int here = id;
    id = look(tile + step);
    if (tile < tiles_in) fetch(find(tile, here), s);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // the queries as right operands: head lane / 4 (and 8 more), elements 2 (lane mod 4) and 8 more
  uint32_t qb[kBlocks][DP / 16][2];
#pragma unroll
  for (int m = 0; m < kBlocks; ++m)
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int h = lane / 4 + 8 * m, d = s * 16 + c * 8 + lane % 4 * 2;
        qb[m][s][c] = 0;
        if (h < w.heads && d < p.dim) {
          const uint16_t* q = reinterpret_cast<const uint16_t*>(static_cast<const T*>(p.q) + w.b * p.q_token +
                                                                (w.head0 + h) * p.q_head + d);
          qb[m][s][c] = q[0] | static_cast<uint32_t>(q[1]) << 16;
        }
      }
  const float scale2 = p.softcap > 0.0f ? p.scale / p.softcap : p.scale * kLog2e, cap2 = p.softcap * kLog2e;
  // a thread's two heads of each block of 8: 2 (lane mod 4) and the next
  float slope2[kBlocks][2], base[kBlocks][2], total[kBlocks][2], acc[kBlocks][DP / 16][4];
#pragma unroll
  for (int m = 0; m < kBlocks; ++m)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int h = lane % 4 * 2 + c + 8 * m;
      slope2[m][c] = p.slopes != nullptr && h < w.heads ? p.slopes[w.head0 + h] * kLog2e : 0.0f;
      base[m][c] = -kInf;
      total[m][c] = 0.0f;
#pragma unroll
      for (int n = 0; n < DP / 16; ++n) acc[m][n][2 * c] = acc[m][n][2 * c + 1] = 0.0f;
    }

  int stage = 0;
  for (int64_t tile = first; tile < tiles_in; tile += step) {
    {
      const int64_t next = tile + (L::kStages - 1) * step;
      const int here = id;
      id = look(next + step);
      if (next < tiles_in) fetch(find(next, here), stage == 0 ? L::kStages - 1 : stage - 1);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 1) : "memory");
    __syncwarp();
    const uint32_t ks = tiles + stage * L::kStage, vs = ks + L::kKeys * L::kRow;
    // scores: keys lane / 4 and 8 more of each block of 16, the thread's heads; even and odd steps apart
    float s[kBlocks][kDeep][2][4] = {};
#pragma unroll
    for (int b = 0; b < kDeep; ++b) {
      const int row = b * 16 + (lane & 7) + (lane >> 3 & 1) * 8;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        uint32_t a[4];
        load4(a, ks + row * L::kRow + (((2 * d + (lane >> 4)) ^ (row & 7)) << 4));
#pragma unroll
        for (int m = 0; m < kBlocks; ++m) mma16816<T>(s[m][b][d & 1], a, qb[m][d][0], qb[m][d][1]);
      }
    }
    const int j = static_cast<int>(tile) * L::kKeys + lane / 4;
    const float away = static_cast<float>(len - 1 - j);
    const bool part = tile == tiles_in - 1;  // a tile that may pass the length
    float back[kBlocks][2];
    bool moved = false;
    uint32_t weight[kBlocks][kDeep][2];
#pragma unroll
    for (int m = 0; m < kBlocks; ++m) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x[kDeep][2];
        float most = -kInf;
#pragma unroll
        for (int b = 0; b < kDeep; ++b)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int key = j + b * 16 + r * 8;
            float y = s[m][b][0][2 * r + c] + s[m][b][1][2 * r + c];
            y = p.softcap > 0.0f ? capped(y, scale2, cap2) : y * scale2;
            if (p.slopes != nullptr) y -= slope2[m][c] * (away - (b * 16 + r * 8));
            if (part && key >= len) y = -kInf;
            x[b][r] = y;
            most = fmaxf(most, y);
          }
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 4));
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 8));
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 16));
        most -= kLift<T>;
        back[m][c] = 1.0f;
        if (most > base[m][c] + kSlack || (base[m][c] == -kInf && most > -kInf)) {
          back[m][c] = exp2_approx(base[m][c] - most);
          base[m][c] = most;
          moved = true;
        }
        const float shift = base[m][c] == -kInf ? 0.0f : base[m][c];
        total[m][c] *= back[m][c];
#pragma unroll
        for (int b = 0; b < kDeep; ++b)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            s[m][b][r][c] = exp2_approx(x[b][r] - shift);
            total[m][c] += s[m][b][r][c];
          }
      }
#pragma unroll
      for (int b = 0; b < kDeep; ++b)
#pragma unroll
        for (int r = 0; r < 2; ++r) weight[m][b][r] = transposed(narrow2<T>(s[m][b][r][0], s[m][b][r][1]));
    }
    if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
      for (int m = 0; m < kBlocks; ++m)
#pragma unroll
        for (int n = 0; n < DP / 16; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[m][n][c] *= back[m][c & 1];
    }
#pragma unroll
    for (int b = 0; b < kDeep; ++b) {
      const int row = b * 16 + (lane & 7) + (lane >> 4) * 8;
#pragma unroll
      for (int n = 0; n < DP / 16; ++n) {
        uint32_t a[4];
        load4_transposed(a, vs + row * L::kRow + (((2 * n + (lane >> 3 & 1)) ^ (row & 7)) << 4));
#pragma unroll
        for (int m = 0; m < kBlocks; ++m) mma16816<T>(acc[m][n], a, weight[m][b][0], weight[m][b][1]);
      }
    }
    __syncwarp();  // the stage may be filled again
    stage = stage + 1 == L::kStages ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int m = 0; m < kBlocks; ++m)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float sum = total[m][c];
      sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 4);
      sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 8);
      sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 16);
      if (lane < 4) {
        tops[warp * HB + lane * 2 + c + 8 * m] = base[m][c];
        totals[warp * HB + lane * 2 + c + 8 * m] = sum;
      }
    }
  __syncthreads();  // join.bad is set, and every warp is done with its tiles: the outputs take their place
  if (bad) join.bad = 1;
  float* outs = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int m = 0; m < kBlocks; ++m)
#pragma unroll
    for (int n = 0; n < DP / 16; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        outs[(warp * HB + lane % 4 * 2 + (c & 1) + 8 * m) * DP + n * 16 + lane / 4 + c / 2 * 8] = acc[m][n][c];
  decode_join<T, HB, DP, kWarps, true>(p, w, DecodeRows<T>(p, w), outs, tops, totals, join);
}

template <typename T, int DP, int HB>
cudaError_t launch_size(DecodeParams p, int64_t batch, int sms, cudaStream_t stream) {
  p.head_blocks = (p.group + HB - 1) / HB;
  const int64_t items = batch * p.kv_heads * p.head_blocks;
  // CTAs per SM: 4 leave long sequences in too few (48 of up to 16384 keys 293 us, with 6 or 8 248); 8 split short ones
  // for their joins' sake (16 of up to 4001 keys, 32 heads: 67 us, with 4 or 6 57)
  const int c = decode_cluster(items, p.max_pages * p.page_size, sms, 6);
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
  if (dtype == 0 || !paged_vectors(p)) return false;
  *e = dtype == 1 ? launch_type<__nv_bfloat16>(p, batch, sms, stream) : launch_type<__half>(p, batch, sms, stream);
  return true;
}

}  // namespace zo
