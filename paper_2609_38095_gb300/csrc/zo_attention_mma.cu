// zo_attention_mma.cu -- attention of packed documents on the tensor cores:
// 16-bit types, heads of up to 128 elements, vectors aligned to 16 bytes
// (zo_attention).
#include "zo_forward.cuh"
#include "zo_tcgen05.cuh"

namespace zo {

namespace {

bool encode_map(CUtensorMap* map, bool bf16, const void* p, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
                const cuuint32_t* box) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<Encode>(f);
  }();
  const cuuint32_t steps[4] = {1, 1, 1, 1};
  return encode != nullptr &&
         encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, const_cast<void*>(p), dims,
                strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// a dimension of one element has no stride of its own
cuuint64_t stride_of(int64_t n, int64_t stride) { return static_cast<cuuint64_t>(n > 1 ? stride * 2 : 16); }

}  // namespace

bool make_head_map(CUtensorMap* map, bool bf16, const void* p, int dim, int heads, int64_t tokens, int64_t head_stride,
                   int64_t token_stride, int rows) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(tokens)};
  const cuuint64_t strides[2] = {stride_of(heads, head_stride), stride_of(tokens, token_stride)};
  const cuuint32_t box[3] = {64, 1, static_cast<cuuint32_t>(rows)};
  return encode_map(map, bf16, p, 3, dims, strides, box);
}

bool make_page_map(CUtensorMap* map, bool bf16, const void* p, int dim, int heads, int64_t page_rows, int64_t pages, int64_t head_stride,
                   int64_t row_stride, int64_t page_stride, int rows) {
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(page_rows),
                              static_cast<cuuint64_t>(pages)};
  const cuuint64_t strides[3] = {stride_of(heads, head_stride), stride_of(page_rows, row_stride), stride_of(pages, page_stride)};
  const cuuint32_t box[4] = {64, 1, static_cast<cuuint32_t>(rows), 1};
  return encode_map(map, bf16, p, 4, dims, strides, box);
}

namespace {

constexpr int kRows = 128;           // query rows of a slot
constexpr int kKeys = 64;            // keys of a step
constexpr int kChunk = kRows * 128;  // bytes of 64 elements of a slot's queries

// A CTA of two slots, one per SM, with keys and values by 128; or of one slot, two per SM, with keys and values by 64.
template <int D, int kSlots>
struct Plan {
  static constexpr int kSteps = kSlots;                          // of a tile of keys and values
  static constexpr int kQueries = D / 64 * kChunk;               // bytes of a slot's queries
  static constexpr int kTileChunk = kSteps * kKeys * 128;        // bytes of 64 elements of a tile
  static constexpr int kTile = D / 64 * kTileChunk;
  static constexpr int kStages = kSlots == 1 ? 4 : D == 128 ? 5 : 8;  // tiles of keys and values in turn
  static constexpr int kBytes = kSlots * kQueries + kStages * kTile + 1024;
  static constexpr int kSoftmaxWarps = 4 * kSlots;
  static constexpr int kThreads = kSlots == 1 ? 256 : 384;
  static constexpr int kColumns = 256 * kSlots;                  // of tensor memory
  static constexpr int kOutputs = 128 * kSlots;                  // the first column of the outputs
};

// Barriers of steps come in pairs, for even and odd steps. A wait by parity is sound while the barrier can be at most one
// phase past the one waited for, and each of these cannot reach its next phase before the waiter has done its part: scores
// c + 2 follow the weights c, weights c + 2 the scores c + 2, outputs c + 2 the weights c + 2, and a stage's next load
// follows both slots' use of it. (One barrier for a slot's outputs could be two phases ahead of the last wait.)
struct MmaShared {
  uint64_t q_full, kv_full[8], kv_empty[8], s_full[2][2], p_full[2][2], o_done[2][2], drain[2];
  int lo[2], hi[2];
  uint32_t tmem;
  int dead;
  uint32_t left[2][kRows / 32];  // rows for attention_rows
  float lse[2][kRows];
};

// Bits 0 to n - 1.
__device__ __forceinline__ uint32_t bits_below(int n) { return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u; }

// A slot is 128 query rows of a head. A CTA of two slots has two heads that share
// their keys (the same rows, the same spans) where a group has an even number of
// them, else two tiles of rows of one head; a CTA of one slot has one. Keys and
// values come in tiles of 128 (one slot: 64) and go through the products in steps
// of 64.
//
//   two slots        one slot
//   warps 0-3, 4-7   0-3       softmax of slot 0, 1: a thread has a row
//   warps 8, 9       4         the matrix products of slot 0, 1, one thread each: a warp alone issues a step's for both in
//                              more time than they take
//   warp 10          5         TMA loads, one thread (11 and 6 set up the barriers)
//
// Tensor memory (512 columns, or 256): a slot's scores of two steps, 64 columns
// each, the weights of a step in 16 bits over the first half of its scores; outputs
// from column 256 (128) on. S = Q K^T has both operands in shared memory; O += P V
// takes P from tensor memory and V as TMA left it, along N. Behind step i's output
// go step i + 2's scores, into the place of the weights that it has read: a slot's
// softmax always has its next scores, and its tensor-core warp one wait per step.
//
// What bounds it, two slots and heads of 128: a product with 64 columns reads 6 KB
// of shared memory in the 32 cycles that it would take; 16 of them and 8 with 128
// columns, a slot's for 128 keys, were measured alone at 1262 cycles (1024 by the
// columns), so 2524 for both slots, where the kernel takes some 2880. 8192 tokens,
// 32 / 8 heads of 128, bf16: 334 to 339 us = 1.63 PFLOP/s for the first tens of
// launches after a pause, 360 us = 1.53 once the GPU's clock has settled under the
// load. With steps of 128 keys the products would take 2048 cycles, but there is no
// tensor memory for a second step's scores then, and a slot's softmax, 1600 cycles
// and two waits of 400, is in series with its own products (460 us).
//
// The output is rescaled only when a row's maximum has passed the reference that
// its weights are relative to by 2^8, which seldom happens after the first steps:
// weights up to 2^8 (fp16: 2^15, kLift) lose nothing in 16 bits and their sum is fp32.
template <typename T, int D, int kSlots, bool kCap, bool kBias>
__global__ void __launch_bounds__(Plan<D, kSlots>::kThreads, 3 - kSlots)
    attention_mma_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                         const __grid_constant__ CUtensorMap v_map, const __grid_constant__ CUtensorMap o_map,
                         const __grid_constant__ AttentionParams p, int by_heads) {
  using L = Plan<D, kSlots>;
  constexpr int kSoftmaxWarps = L::kSoftmaxWarps;
  constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
  extern __shared__ uint8_t raw[];
  __shared__ MmaShared sh;
  uint8_t* tiles = raw + (1024 - smem_address(raw) % 1024) % 1024;  // the slots' queries, then the stages
  uint8_t* stages = tiles + kSlots * L::kQueries;
  const int tid = threadIdx.x, warp = static_cast<int>(uniform(tid >> 5)), lane = tid & 31;
  const int heads_here = kSlots == 2 && by_heads ? 2 : 1, tiles_here = kSlots / heads_here;  // heads, tiles of rows
  const int per = p.heads / heads_here;  // CTAs per tile of rows; the longest causal rows come first
  const int item = blockIdx.x % per, block = (gridDim.x / per - 1 - blockIdx.x / per) * tiles_here;
  const int head0 = item * heads_here, kv_head = head0 / p.group;
  const auto head_of = [&](int s) { return heads_here == 2 ? head0 + s : head0; };
  const auto block_of = [&](int s) { return tiles_here == 2 ? block + s : block; };
  volatile int* dead = &sh.dead;

  int64_t row = 0;
  int lo = 0, hi = 0, self = 0;
  const int slot = warp >> 2;
  if (warp < kSoftmaxWarps) {
    row = static_cast<int64_t>(block_of(slot)) * kRows + (tid & 127);
    if (row < p.q_tokens) {
      lo = max(p.spans[row], 0);
      hi = min(p.spans[p.q_tokens + row], static_cast<int>(p.k_tokens));
      if (kBias) self = p.spans[2 * p.q_tokens + row];
    }
    if (hi <= lo) lo = hi = 0;
  }
  if (tid == (kSoftmaxWarps + kSlots + 1) * 32) {
    mbar_init(&sh.q_full, 1);
    for (int i = 0; i < L::kStages; ++i) {
      mbar_init(&sh.kv_full[i], 1);
      mbar_init(&sh.kv_empty[i], kSlots);
    }
    for (int s = 0; s < 2; ++s) {
      for (int b = 0; b < 2; ++b) {
        mbar_init(&sh.s_full[s][b], 1);
        mbar_init(&sh.p_full[s][b], 4);
        mbar_init(&sh.o_done[s][b], 1);
      }
      mbar_init(&sh.drain[s], 1);
      for (int w = 0; w < kRows / 32; ++w) sh.left[s][w] = 0;
      sh.lo[s] = 0x7FFFFFFF;
      sh.hi[s] = 0;
    }
    sh.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kSoftmaxWarps) tmem_alloc(&sh.tmem, L::kColumns);
  if (tid == (kSoftmaxWarps + kSlots) * 32) {
    prefetch_map(&q_map);
    prefetch_map(&k_map);
    prefetch_map(&v_map);
    prefetch_map(&o_map);
  }
  __syncthreads();
  if (tid == (kSoftmaxWarps + kSlots) * 32) {  // the queries, before the spans are known
    mbar_expect(&sh.q_full, kSlots * L::kQueries);
    for (int s = 0; s < kSlots; ++s)
      for (int c = 0; c < D / 64; ++c)
        tma_load_3d(tiles + s * L::kQueries + c * kChunk, &q_map, c * 64, head_of(s), block_of(s) * kRows, &sh.q_full);
  }
  if (warp < kSoftmaxWarps) {
    const int least = __reduce_min_sync(0xFFFFFFFFu, hi > lo ? lo : 0x7FFFFFFF);
    const int most = __reduce_max_sync(0xFFFFFFFFu, hi);
    if (lane == 0 && most > 0) {
      atomicMin(&sh.lo[slot], least);
      atomicMax(&sh.hi[slot], most);
    }
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = uniform(sh.tmem);
  const int begin = static_cast<int>(uniform(min(sh.lo[0], sh.lo[kSlots - 1])));
  const int stop = static_cast<int>(uniform(max(sh.hi[0], sh.hi[kSlots - 1])));
  const int n = stop > begin ? (stop - begin + kKeys - 1) / kKeys : 0;  // steps
  int from[kSlots], to[kSlots];                                         // those that a slot sees
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    from[s] = to[s] = 0;
    if (sh.hi[s] > sh.lo[s]) {
      from[s] = static_cast<int>(uniform((sh.lo[s] - begin) / kKeys));
      to[s] = static_cast<int>(uniform((sh.hi[s] - begin + kKeys - 1) / kKeys));
    }
  }

  int again = 0;  // whether rows are left for attention_rows
  if (warp == kSoftmaxWarps + kSlots) {
    if (lane == 0) {
      int issued = 0;
      for (int i = 0; i < (n + L::kSteps - 1) / L::kSteps * 2; ++i) {  // keys 0, values 0, keys 1, ...
        const int stage = i % L::kStages;
        if (i >= L::kStages && !mbar_wait(&sh.kv_empty[stage], (i / L::kStages - 1) & 1, dead)) break;
        mbar_expect(&sh.kv_full[stage], L::kTile);
        for (int c = 0; c < D / 64; ++c)
          tma_load_3d(stages + stage * L::kTile + c * L::kTileChunk, i % 2 == 0 ? &k_map : &v_map, c * 64, kv_head,
                      begin + (i / 2) * L::kSteps * kKeys, &sh.kv_full[stage]);
        ++issued;
      }
      if (*dead) {  // nothing may land in shared memory after the CTA is gone
        const long long start = clock64();
        for (int i = max(0, issued - L::kStages); i < issued; ++i)
          while (!mbar_try(&sh.kv_full[i % L::kStages], (i / L::kStages) & 1) && clock64() - start < kWaitCycles) {}
        while (!mbar_try(&sh.q_full, 0) && clock64() - start < kWaitCycles) {}
      }
    }
  } else if (warp >= kSoftmaxWarps && warp < kSoftmaxWarps + kSlots) {
    const int s = warp - kSoftmaxWarps;
    const int first = s ? from[kSlots - 1] : from[0], last = s ? to[kSlots - 1] : to[0];
    const uint32_t at = uniform(smem_address(stages));
    const uint64_t queries = operand_desc(uniform(smem_address(tiles)) + s * L::kQueries, 16, 1024);
    const uint64_t keys = operand_desc(at, 16, 1024), values = operand_desc(at, L::kTileChunk, 1024);
    constexpr uint32_t kScores = mma_desc(kBf16, kKeys, false), kOutput = mma_desc(kBf16, D, true);
    constexpr uint32_t kHalf = kKeys * 128;  // bytes from a tile's first step to its second
    const uint32_t scores = tmem + s * 128, out = tmem + L::kOutputs + s * D;
    const auto scores_of = [&](int j, uint64_t k) {  // of step j, its keys at k
      const int b = (j - first) & 1;
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
        mma_ss(scores + b * kKeys, queries + (d / 4 * kChunk + d % 4 * 32) / 16,
               k + (d / 4 * L::kTileChunk + d % 4 * 32) / 16, kScores, d > 0);
      mma_commit(&sh.s_full[s][b]);
    };
    // Tile t's keys are the loads' 2 t, its values 2 t + 1. The stages and parities of tile t's values and tile t + 1's keys:
    int v_stage = 1, k_stage = 2;
    uint32_t v_parity = 0, k_parity = 0;
    const auto advance = [](int& stage, uint32_t& parity) {
      if ((stage += 2) >= L::kStages) {
        stage -= L::kStages;
        parity ^= 1;
      }
    };
    bool alive = n == 0 || mbar_wait_warp(&sh.q_full, 0, dead);
    if (n > 0 && alive) alive = mbar_wait_warp(&sh.kv_full[0], 0, dead);
    // The first two steps' scores: both of the first tile, or with a step per tile the first here and the second in front of
    // the loop, which then has the stages of step i's values and of step i + 2's keys.
    if (n > 0 && alive && elect_one()) {
      if (first == 0 && last > 0) scores_of(0, keys);
      if (L::kSteps == 2 && first <= 1 && last > 1) scores_of(1, keys + kHalf / 16);
      mma_commit(&sh.kv_empty[0]);
    }
    if (L::kSteps == 1 && n > 1 && alive) {
      alive = mbar_wait_warp(&sh.kv_full[k_stage], k_parity, dead);
      if (alive && elect_one()) {
        if (first <= 1 && last > 1) scores_of(1, keys + static_cast<uint32_t>(k_stage) * L::kTile / 16);
        mma_commit(&sh.kv_empty[k_stage]);
      }
      advance(k_stage, k_parity);
    }
    for (int i = 0; i < n && alive; ++i) {  // step i's output, and step i + 2's scores in the place of step i's
      const bool more = i / L::kSteps * L::kSteps + 2 < n;  // there is a tile of step i + 2
      if (i % L::kSteps == 0) {
        if (i > 0) {
          advance(v_stage, v_parity);
          advance(k_stage, k_parity);
        }
        alive = mbar_wait_warp(&sh.kv_full[v_stage], v_parity, dead);
        if (L::kSteps == 2 && alive && more) alive = mbar_wait_warp(&sh.kv_full[k_stage], k_parity, dead);
        if (!alive) break;
        const int rest = stop - (begin + i * kKeys), used = min(L::kSteps, n - i) * kKeys;
        if (rest < used && stop < p.k_tokens) {
          // keys that no row sees (TMA gives zeros only beyond the last of all): their weight is 0, and 0 times what is
          // there has to be 0. A row's 16-byte vectors are swizzled among themselves.
          uint8_t* v = stages + v_stage * L::kTile + lane % 8 * 16;
          for (int r = rest + lane / 8; r < used; r += 4)
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
              *reinterpret_cast<uint4*>(v + c * L::kTileChunk + r * 128) = make_uint4(0, 0, 0, 0);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
      }
      const int c = i - first, b = c & 1;
      const bool mine = i >= first && i < last;
      if (mine) {
        alive = mbar_wait_warp(&sh.p_full[s][b], c >> 1 & 1, dead);
        if (!alive) break;
      }
      tmem_fence_after();
      const uint64_t v = values + (static_cast<uint32_t>(v_stage) * L::kTile + i % L::kSteps * kHalf) / 16;
      const uint64_t k = keys + (static_cast<uint32_t>(k_stage) * L::kTile + i % L::kSteps * kHalf) / 16;
      if (elect_one()) {
        if (mine) {
          mma_ts(out, scores + b * kKeys, v, kOutput, c > 0);
#pragma unroll
          for (int d = 1; d < kKeys / 16; ++d) mma_ts(out, scores + b * kKeys + d * 8, v + d * (2048 / 16), kOutput, true);
          mma_commit(&sh.o_done[s][b]);
        }
      }
      // with four short tiles, step i + 2's keys may still be on their way
      if (L::kSteps == 1 && more) alive = mbar_wait_warp(&sh.kv_full[k_stage], k_parity, dead);
      if (!alive) break;
      if (elect_one()) {
        if (i + 2 >= first && i + 2 < last) scores_of(i + 2, k);
        if (i % L::kSteps == L::kSteps - 1 || i == n - 1) {
          mma_commit(&sh.kv_empty[v_stage]);
          if (more) mma_commit(&sh.kv_empty[k_stage]);
        }
      }
    }
    __syncwarp();
    if (__any_sync(0xFFFFFFFFu, *dead != 0) && elect_one()) {  // the products that are on their way end first
      mma_commit(&sh.drain[s]);
      const long long start = clock64();
      while (!mbar_try(&sh.drain[s], 0) && clock64() - start < kWaitCycles) {}
    }
    __syncwarp();
  } else if (warp < kSoftmaxWarps) {
    const int h = head_of(slot);
    const uint32_t at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16), out = at + L::kOutputs + slot * D;
    const float scale2 = kCap ? p.scale / p.softcap : p.scale * kLog2e;
    const float cap2 = p.softcap * kLog2e, slope2 = kBias ? p.slopes[h] * kLog2e : 0.0f;
    const int steps = to[slot] - from[slot];
    float base = -kInf, total = 0.0f;  // log2 of what the weights are relative to, and their sum
    bool alive = true;
    for (int c = 0; c < steps; ++c) {
      const int b = c & 1;
      const uint32_t scores = at + slot * 128 + b * kKeys;
      alive = mbar_wait_warp(&sh.s_full[slot][b], c >> 1 & 1, dead);
      if (!alive) break;
      tmem_fence_after();
      uint32_t x[2][32];
      tmem_load32(x[0], scores);
      tmem_load32(x[1], scores + 32);
      tmem_wait_ld(x[0]);
      tie32(x[1]);
      const int key0 = begin + (from[slot] + c) * kKeys;
      if (kCap) {
        float far = 0.0f;
#pragma unroll
        for (int e = 0; e < 64; ++e) far = fmaxf(far, fabsf(__uint_as_float(x[e / 32][e % 32])));
        if (__all_sync(0xFFFFFFFFu, far * scale2 < kNearCap)) {  // mostly: caps are there for the rare large score
          const uint64_t over2 = pack2(scale2, scale2), caps = pack2(cap2, cap2);
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            uint32_t* at = &x[e / 32][e % 32];
            const uint64_t s = capped_near(static_cast<uint64_t>(at[1]) << 32 | at[0], over2, caps);
            at[0] = static_cast<uint32_t>(s), at[1] = static_cast<uint32_t>(s >> 32);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 64; ++e)
            x[e / 32][e % 32] = __float_as_uint(capped(__uint_as_float(x[e / 32][e % 32]), scale2, cap2));
        }
      }
      if (kBias) {
        const float away = static_cast<float>(self - key0);  // exact, and its differences, below 2^24
        const float times = kCap ? 1.0f : scale2;
#pragma unroll
        for (int e = 0; e < 64; ++e)
          x[e / 32][e % 32] = __float_as_uint(__uint_as_float(x[e / 32][e % 32]) * times - slope2 * fabsf(away - e));
      }
      if (!__all_sync(0xFFFFFFFFu, lo <= key0 && hi >= key0 + kKeys)) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint32_t seen = bits_below(hi - key0 - 32 * c) & ~bits_below(lo - key0 - 32 * c);
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (!(seen >> e & 1)) x[c][e] = __float_as_uint(-kInf);
        }
      }
      float most[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        most[e] = __uint_as_float(x[e / 2][e % 2 * 16]);
#pragma unroll
        for (int i = 1; i < 16; ++i) most[e] = fmaxf(most[e], __uint_as_float(x[e / 2][e % 2 * 16 + i]));
      }
      float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
      if (!kCap && !kBias) top *= scale2;
      top -= kLift<T>;
      // A row's first score sets its reference: its output so far is a sum of zeros (or of 0 times NaN, which shows at the
      // end), so there is nothing to rescale.
      const bool moved = base > -kInf && top > base + kSlack;
      if (__any_sync(0xFFFFFFFFu, moved)) {
        const float back = moved ? exp2_approx(base - top) : 1.0f;
        total *= back;
        // the step before is in the output
        alive = mbar_wait_warp(&sh.o_done[slot][b ^ 1], (c - 1) >> 1 & 1, dead);
        if (!alive) break;
        tmem_fence_after();
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          uint32_t o[16];
          tmem_load16_wait(o, out + d * 16);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * back);
          tmem_store16(out + d * 16, o);
        }
      }
      if (moved || base == -kInf) base = top;
      const float shift = base == -kInf ? 0.0f : -base;
      const float times = kCap || kBias ? 1.0f : scale2;
      const uint64_t times2 = pack2(times, times), shift2 = pack2(shift, shift);
      uint64_t sums[2] = {0, 0};
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint64_t t =
              fma2(pack2(__uint_as_float(x[half][2 * i]), __uint_as_float(x[half][2 * i + 1])), times2, shift2);
          const float u = exp2_approx(low2(t)), v = exp2_approx(high2(t));
          sums[i & 1] = add2(sums[i & 1], pack2(u, v));
          w[i] = narrow2<T>(u, v);
        }
        tmem_store16(scores + half * 16, w);
      }
      const uint64_t sum = add2(sums[0], sums[1]);
      total += low2(sum) + high2(sum);
      tmem_wait_st();
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_full[slot][b]);
    }
    const bool any = steps > 0;
    if (!any) alive = mbar_wait_warp(&sh.q_full, 0, dead);  // the queries' place is written below
    if (alive && any) alive = mbar_wait_warp(&sh.o_done[slot][(steps - 1) & 1], (steps - 1) >> 1 & 1, dead);
    tmem_fence_after();
    const bool seen = alive && any && total != 0.0f;
    const float over = seen ? 1.0f / total : 0.0f;
    const float lse = !alive ? NAN : seen ? (base + log2f(total)) * kLn2 : -kInf;
    bool finite = true;
    // Through shared memory, in the place of the slot's queries: a warp's rows of 64 elements as TMA stores them (rows
    // apart in memory, a thread's own stores took 3 us).
    const uint32_t mine = smem_address(tiles + slot * L::kQueries) + (warp & 3) * 32 * 128;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[32];
      if (alive && any) {
        tmem_load32(o, out + c * 32);
        tmem_wait_ld(o);
      }
#pragma unroll
      for (int e = 0; e < 32; e += 8) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f[i] = !alive ? NAN : seen ? __uint_as_float(o[e + i]) * over : 0.0f;
          finite = finite && fabsf(f[i]) < kInf;
        }
        const uint4 w = Vec<T>::narrow_all(f);
        const int vector = c % 2 * 4 + e / 8;
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(mine + c / 2 * kChunk + lane * 128 +
                                                                      ((vector ^ (lane & 7)) << 4)),
                     "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w)
                     : "memory");
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0 && row < p.q_tokens) {
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        if (c * 64 < p.dim) tma_store_3d(&o_map, c * 64, h, static_cast<int>(row), mine + c * kChunk);
      tma_store_commit();
    }
    if (row < p.q_tokens && p.lse != nullptr) p.lse[h * p.q_tokens + row] = lse;
    // (a sum that is NaN is that of seen scores, and the outputs' too)
    const uint32_t left = __ballot_sync(0xFFFFFFFFu, alive && row < p.q_tokens && !finite && total < kInf);
    if (left != 0) {
      sh.lse[slot][tid & 127] = lse;
      if (lane == 0) sh.left[slot][warp & 3] = left;
      again = 1;
    }
    if (lane == 0) {
      if (left != 0) tma_stored<false>();  // those rows are read again
      else tma_stored<true>();
    }
    __syncwarp();
  }
  tmem_fence_before();
  again = __syncthreads_or(again);
  if (warp == kSoftmaxWarps) {
    tmem_fence_after();
    tmem_free(tmem, L::kColumns);
  }
  if (again == 0) return;
  for (int s = 0; s < kSlots; ++s)
    attention_rows<T, D, 2>(p, static_cast<int64_t>(block_of(s)) * kRows, head_of(s), sh.left[s], sh.lse[s], kRows / 32,
                            warp, L::kThreads / 32, lane);
}

template <typename T, int D, int kSlots, bool kCap, bool kBias>
cudaError_t launch_kind(const CUtensorMap (&m)[4], const AttentionParams& p, cudaStream_t stream) {
  using L = Plan<D, kSlots>;
  const auto kernel = attention_mma_kernel<T, D, kSlots, kCap, kBias>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes);
  if (e != cudaSuccess) return e;
  const int by_heads = p.group % 2 == 0;
  const int heads_here = kSlots == 2 && by_heads ? 2 : 1;
  const int64_t rows = kRows * (kSlots / heads_here);
  const int64_t grid = (p.q_tokens + rows - 1) / rows * (p.heads / heads_here);
  kernel<<<static_cast<unsigned>(grid), L::kThreads, L::kBytes, stream>>>(m[0], m[1], m[2], m[3], p, by_heads);
  return cudaGetLastError();
}

template <typename T, int D, int kSlots>
cudaError_t launch_slots(const CUtensorMap (&m)[4], const AttentionParams& p, cudaStream_t stream) {
  if (p.softcap > 0.0f)
    return p.slopes != nullptr ? launch_kind<T, D, kSlots, true, true>(m, p, stream)
                               : launch_kind<T, D, kSlots, true, false>(m, p, stream);
  return p.slopes != nullptr ? launch_kind<T, D, kSlots, false, true>(m, p, stream)
                             : launch_kind<T, D, kSlots, false, false>(m, p, stream);
}

template <typename T>
cudaError_t launch_head(const CUtensorMap (&m)[4], const AttentionParams& p, bool two, cudaStream_t stream) {
  if (p.dim <= 64) return two ? launch_slots<T, 64, 2>(m, p, stream) : launch_slots<T, 64, 1>(m, p, stream);
  return two ? launch_slots<T, 128, 2>(m, p, stream) : launch_slots<T, 128, 1>(m, p, stream);
}

// Whether a CTA takes two slots: two CTAs of one slot per SM hide each other's starts and ends (one document of 512 tokens
// 10.1 us with one slot, 11.8 with two; of 1024 18.8 / 17.2), two slots share their keys' tiles and issue ahead (of 2048 tokens
// 40 / 32, of 8192 476 / 335). The spans are on the device, so this goes by all the keys of a call, as if they were one
// document's: a packed batch beyond 768 keys takes two slots though its documents are short (24 of at most 256 24.9 / 28.7),
// since two slots lose less there than one slot does on a long document.
bool two_slots(const AttentionParams& p) { return p.k_tokens > 768; }

}  // namespace

bool launch_attention_mma(const AttentionParams& p, int dtype, cudaStream_t stream, cudaError_t* e) {
  const auto vectors = [](const void* x, int64_t token, int64_t head, int64_t tokens, int64_t heads) {
    return aligned_to(x, 16) && token % 8 == 0 && head % 8 == 0 && (token > 0 || tokens <= 1) && (head > 0 || heads <= 1);
  };
  const int kv_heads = p.heads / p.group;
  constexpr int64_t kMost = 0x7FFFFFFF - 4 * kRows;  // rows, keys and CTAs, a last tile's end among them, in 32 bits
  // The scores' maximum is taken before the scale, and -inf times it has to stay -inf: it is positive
  if (dtype == 0 || p.dim > 128 || p.dim % 8 != 0 || p.k_tokens == 0 || !(p.scale > 0.0f)) return false;
  if (p.q_tokens > kMost || p.k_tokens > kMost || (p.q_tokens / kRows + 1) * p.heads > kMost) return false;
  if (!vectors(p.q, p.q_token, p.q_head, p.q_tokens, p.heads) || !vectors(p.k, p.k_token, p.k_head, p.k_tokens, kv_heads) ||
      !vectors(p.v, p.v_token, p.v_head, p.k_tokens, kv_heads) ||
      !vectors(p.out, p.out_token, p.out_head, p.q_tokens, p.heads))
    return false;
  CUtensorMap m[4];
  const bool bf16 = dtype == 1, two = two_slots(p);
  const int keys = two ? 2 * kKeys : kKeys;
  if (!make_head_map(&m[0], bf16, p.q, p.dim, p.heads, p.q_tokens, p.q_head, p.q_token, kRows) ||
      !make_head_map(&m[1], bf16, p.k, p.dim, kv_heads, p.k_tokens, p.k_head, p.k_token, keys) ||
      !make_head_map(&m[2], bf16, p.v, p.dim, kv_heads, p.k_tokens, p.v_head, p.v_token, keys) ||
      !make_head_map(&m[3], bf16, p.out, p.dim, p.heads, p.q_tokens, p.out_head, p.out_token, 32))
    return false;
  *e = bf16 ? launch_head<__nv_bfloat16>(m, p, two, stream) : launch_head<__half>(m, p, two, stream);
  return true;
}

}  // namespace zo
