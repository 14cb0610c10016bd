// zo_draft_wide.cu -- attention of trees of drafted tokens over a paged cache
// where many rows share a key (zo_attention_draft): tcgen05, 16-bit types, heads
// of up to 128 elements, vectors aligned to 16 bytes.
#include "zo_decode.cuh"
#include "zo_tcgen05.cuh"

namespace zo {

namespace {

constexpr int kRows = 128;           // rows of a slot
constexpr int kKeys = 64;            // keys of a step
constexpr int kChunk = kRows * 128;  // bytes of 64 elements of a slot's queries
constexpr int kLoaders = 2;          // warps that fetch

template <int D, int kSlots>
struct Plan {
  static constexpr int kBlock = kSlots * kRows;
  static constexpr int kQueries = D / 64 * kChunk;      // bytes of a slot's queries
  static constexpr int kTileChunk = kKeys * 128;        // bytes of 64 elements of a step's keys or values
  static constexpr int kTile = D / 64 * kTileChunk;
  static constexpr int kStages = kSlots == 2 ? (D == 128 ? 8 : 12) : (D == 128 ? 4 : 8);  // tiles, of keys and values in turn
  // Tiles on their way before the oldest is waited for. A tile of values is fetched into the place of one that the products
  // are done with only when the next step's scores are, whose keys have to be known to be there by then: at most kStages - 2.
  static constexpr int kAhead = kSlots == 2 ? (D == 128 ? 5 : 9) : (D == 128 ? 2 : 6);
  static constexpr int kPitch = D + 4;                  // floats of a row of outputs: rows' vectors on distinct banks
  static constexpr int kOuts = kBlock * kPitch * 4;
  static constexpr int kUsed = kSlots * kQueries + kStages * kTile;
  static constexpr int kBytes = (kUsed > kOuts ? kUsed : kOuts) + 1024;
  static constexpr int kSoftmaxWarps = 4 * kSlots;
  static constexpr int kThreads = 32 * (kSoftmaxWarps + kSlots + kLoaders);
  static constexpr int kColumns = 256 * kSlots;         // of tensor memory
  static constexpr int kOutputs = 128 * kSlots;         // the first column of the outputs
  static_assert(kAhead <= kStages - 2, "");
};

// As in zo_attention_mma.cu: barriers of steps in pairs, for even and odd ones; none can be two phases ahead of a waiter.
template <int kSlots>
struct Shared {
  uint64_t full[12], empty[12], s_full[2][2], p_full[2][2], o_done[2][2], drain[2];
  DraftShared<kSlots * kRows> rows;
  uint32_t odd[64][4];  // a node's columns whose value is not finite
  float top[kSlots * kRows], total[kSlots * kRows];
  uint32_t tmem;
  int dead, bad, any_odd;
};

template <typename T>
__device__ __forceinline__ bool odd16(uint32_t v) {  // infinite or NaN
  constexpr uint32_t kExponent = __is_same(T, __nv_bfloat16) ? 0x7F80u : 0x7C00u;
  return (v & kExponent) == kExponent;
}

// A CTA has up to 128 kSlots rows of a sequence and key-value head, and its
// cluster splits the keys: rows are what they are in zo_draft.cu, products and
// barriers as in zo_attention_mma.cu (a slot's scores of two steps and their
// weights in tensor memory, a step's scores issued behind the output of the one
// two before it).
//
//   warps 0-3 (4-7)   softmax of slot 0 (1): a thread has a row; those without a row that sees anything stay out
//   the next (two)    the products of slot 0 (1)
//   the last two      keys and values by cp.async, a lane per key's page: any size of page
template <typename T, int D, int kSlots, bool kCap, bool kBias>
__global__ void __launch_bounds__(Plan<D, kSlots>::kThreads, 3 - kSlots)
    draft_wide_kernel(const __grid_constant__ DraftParams p) {
  using L = Plan<D, kSlots>;
  constexpr int kSoftmaxWarps = L::kSoftmaxWarps, kVectors = D / 8;
  constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
  extern __shared__ uint8_t raw[];
  __shared__ Shared<kSlots> sh;
  uint8_t* tiles = raw + (1024 - smem_address(raw) % 1024) % 1024;  // the slots' queries, then the stages
  uint8_t* stages = tiles + kSlots * L::kQueries;
  const int tid = threadIdx.x, warp = static_cast<int>(uniform(tid >> 5)), lane = tid & 31;
  const uint32_t ranks = cluster_size(), rank = cluster_rank();
  const DraftPlace w = draft_place<L::kBlock>(p, blockIdx.x / ranks, sh.rows);
  const DraftRows<T, L::kBlock> rows = {p, w, sh.rows};
  volatile int* dead = &sh.dead;

  // steps here, and rows up to the last that sees anything
  const int all = static_cast<int>((w.len + kKeys - 1) / kKeys);
  const int begin = static_cast<int>(static_cast<int64_t>(all) * rank / ranks);
  const int n = static_cast<int>(static_cast<int64_t>(all) * (rank + 1) / ranks) - begin;
  const int live = n == 0 ? 0 : w.live;
  const auto warps_of = [&](int s) { return max(0, min(4, (live - s * kRows + 31) / 32)); };

  if (tid == L::kThreads - 32) {
    const int slots = (live + kRows - 1) / kRows;
    for (int i = 0; i < L::kStages; ++i) {
      mbar_init(&sh.full[i], kLoaders);
      mbar_init(&sh.empty[i], slots > 0 ? slots : 1);
    }
    for (int s = 0; s < kSlots; ++s) {
      for (int b = 0; b < 2; ++b) {
        mbar_init(&sh.s_full[s][b], 1);
        mbar_init(&sh.p_full[s][b], warps_of(s) > 0 ? warps_of(s) : 1);
        mbar_init(&sh.o_done[s][b], 1);
      }
      mbar_init(&sh.drain[s], 1);
    }
    sh.dead = sh.any_odd = 0;
    sh.bad = w.bad;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = tid; i < 64 * 4; i += L::kThreads) (&sh.odd[0][0])[i] = 0;
  if (warp == kSoftmaxWarps) tmem_alloc(&sh.tmem, L::kColumns);
  if (warp < kSoftmaxWarps && live > 0) {
    // The queries, swizzled as a product's operand is: 16-byte vector v of a row goes to place v ^ (row mod 8) of its 64
    // elements. Rows that are none are zeros.
    const bool whole = aligned_to(p.q, 16) && p.q_token % 8 == 0 && p.q_node % 8 == 0 && p.q_head % 8 == 0;
    for (int i = tid; i < L::kBlock * kVectors; i += kSoftmaxWarps * 32) {
      const int r = i / kVectors, v = i % kVectors;
      uint8_t* to = tiles + r / kRows * L::kQueries + v / 8 * kChunk + r % kRows * 128 + ((v % 8 ^ (r & 7)) << 4);
      uint4 x = make_uint4(0, 0, 0, 0);
      if (r < live && v * 8 < p.dim) {
        const T* q = rows.query(r) + v * 8;
        if (whole) {
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_address(to)), "l"(q) : "memory");
          continue;
        } else {
          const uint16_t* u = reinterpret_cast<const uint16_t*>(q);
          const auto two = [&](int e) { return u[e] | static_cast<uint32_t>(u[e + 1]) << 16; };
          x = make_uint4(two(0), two(2), two(4), two(6));
        }
      }
      *reinterpret_cast<uint4*>(to) = x;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = uniform(sh.tmem);

  if (warp >= kSoftmaxWarps + kSlots) {
    // Tile l is step l / 2's keys (even) or values. Each of the two warps has 32 of its keys, a lane one of their places.
    const int half = warp - kSoftmaxWarps - kSlots;
    const T* kc = static_cast<const T*>(p.k) + w.g * p.k_head;
    const T* vc = static_cast<const T*>(p.v) + w.g * p.v_head;
    const int vector = lane % kVectors;
    const int bytes = vector * 8 < p.dim ? 16 : 0;  // of a vector; the rest is filled with zeros
    const char* kl = reinterpret_cast<const char*>(kc + (bytes ? vector * 8 : 0));
    const char* vl = reinterpret_cast<const char*>(vc + (bytes ? vector * 8 : 0));
    constexpr int kAtOnce = 32 / kVectors;  // keys of a warp's copy
    const auto place_of = [&](int l, int i) {  // in a stage: the lane's vector of copy i
      const int r = half * 32 + i * kAtOnce + lane / kVectors;
      return stages + l % L::kStages * L::kTile + vector / 8 * L::kTileChunk + r * 128 + ((vector % 8 ^ (r & 7)) << 4);
    };
    int bad = 0;
    const auto key_of = [&](int step) { return static_cast<int64_t>(begin + step) * kKeys + half * 32 + lane; };
    const auto look = [&](int step) {
      const int64_t j = key_of(step);
      return draft_sees(w, j) ? p.pages[w.b * p.pages_stride + decode_page(p, j)] : 0;
    };
    const auto arrived = [&](int l) {  // tile l's copies are done
      if (l & 1) {
        const int64_t key0 = static_cast<int64_t>(begin + l / 2) * kKeys;
        if (key0 + kKeys > w.n) {
          // Values of the tree's keys that are not finite are noted and taken out: a row that does not see one has the
          // weight 0 there, and 0 times it is NaN.
          for (int i = 0; i < 32 / kAtOnce; ++i) {
            const int64_t node = key0 + half * 32 + i * kAtOnce + lane / kVectors - w.n;
            uint16_t* x = reinterpret_cast<uint16_t*>(place_of(l, i));
            if (node < 0 || node >= 64) continue;
            for (int e = 0; e < 8; ++e)
              if (odd16<T>(x[e])) {
                const int column = vector * 8 + e;
                atomicOr(&sh.odd[node][column / 32], 1u << column % 32);
                sh.any_odd = 1;
                x[e] = 0;
              }
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.full[l % L::kStages]);
    };
    int id = look(0);
    int64_t k_at = -1, v_at = -1;
    bool alive = true;
    int issued = 0;
    for (int l = 0; l < (live > 0 ? 2 * n : 0) && alive; ++l) {
      if (l >= L::kStages) alive = mbar_wait_warp(&sh.empty[l % L::kStages], (l / L::kStages - 1) & 1, dead);
      if (!alive) break;
      if (l % 2 == 0) {
        const int64_t j = key_of(l / 2);
        const int2 key = decode_key(p, w, draft_sees(w, j) ? j : w.len, id, bad);
        k_at = key.x >= 0 ? (key.x * p.k_page + key.y * p.k_token) * 2 : -1;
        v_at = key.x >= 0 ? (key.x * p.v_page + key.y * p.v_token) * 2 : -1;
        id = look(l / 2 + 1);
      }
#pragma unroll
      for (int i = 0; i < 32 / kAtOnce; ++i) {
        const int64_t at = __shfl_sync(0xFFFFFFFFu, l % 2 == 0 ? k_at : v_at, i * kAtOnce + lane / kVectors);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_address(place_of(l, i))),
                     "l"((l % 2 == 0 ? kl : vl) + (at >= 0 ? at : 0)), "r"(at >= 0 ? bytes : 0)
                     : "memory");
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      ++issued;
      if (l >= L::kAhead) {
        asm volatile("cp.async.wait_group %0;" ::"n"(L::kAhead) : "memory");
        arrived(l - L::kAhead);
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (alive)
      for (int l = max(0, issued - L::kAhead); l < issued; ++l) arrived(l);
    if (bad) sh.bad = 1;
  } else if (warp >= kSoftmaxWarps) {
    const int s = warp - kSoftmaxWarps;
    const uint32_t at = uniform(smem_address(stages));
    const uint64_t queries = operand_desc(uniform(smem_address(tiles)) + s * L::kQueries, 16, 1024);
    const uint64_t keys = operand_desc(at, 16, 1024), values = operand_desc(at, L::kTileChunk, 1024);
    constexpr uint32_t kScores = mma_desc(kBf16, kKeys, false), kOutput = mma_desc(kBf16, D, true);
    const uint32_t scores = tmem + s * 128, out = tmem + L::kOutputs + s * D;
    const int mine = warps_of(s) > 0 ? n : 0;
    const auto scores_of = [&](int i) {  // one thread; step i's keys are there
      const int stage = 2 * i % L::kStages;
      const uint64_t k = keys + static_cast<uint32_t>(stage) * L::kTile / 16;
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
        mma_ss(scores + (i & 1) * kKeys, queries + (d / 4 * kChunk + d % 4 * 32) / 16,
               k + (d / 4 * L::kTileChunk + d % 4 * 32) / 16, kScores, d > 0);
      mma_commit(&sh.s_full[s][i & 1]);
      mma_commit(&sh.empty[stage]);
    };
    const auto there = [&](int l) { return mbar_wait_warp(&sh.full[l % L::kStages], l / L::kStages & 1, dead); };
    bool alive = true;
    for (int i = 0; i < min(2, mine) && alive; ++i) {
      alive = there(2 * i);
      if (alive && elect_one()) scores_of(i);
      __syncwarp();
    }
    for (int i = 0; i < mine && alive; ++i) {  // step i's output, and step i + 2's scores in the place of its weights
      alive = there(2 * i + 1) && mbar_wait_warp(&sh.p_full[s][i & 1], i >> 1 & 1, dead);
      if (!alive) break;
      tmem_fence_after();
      const int stage = (2 * i + 1) % L::kStages;
      const uint64_t v = values + static_cast<uint32_t>(stage) * L::kTile / 16;
      if (elect_one()) {
#pragma unroll
        for (int d = 0; d < kKeys / 16; ++d)
          mma_ts(out, scores + (i & 1) * kKeys + d * 8, v + d * (2048 / 16), kOutput, d > 0 || i > 0);
        mma_commit(&sh.o_done[s][i & 1]);
        mma_commit(&sh.empty[stage]);
      }
      __syncwarp();
      if (i + 2 < mine) {
        alive = there(2 * (i + 2));
        if (alive && elect_one()) scores_of(i + 2);
        __syncwarp();
      }
    }
    if (__any_sync(0xFFFFFFFFu, *dead != 0) && elect_one()) {  // the products that are on their way end first
      mma_commit(&sh.drain[s]);
      const long long start = clock64();
      while (!mbar_try(&sh.drain[s], 0) && clock64() - start < kWaitCycles) {}
    }
    __syncwarp();
  } else {
    const int slot = warp >> 2, r = tid;  // the thread's row
    const bool in = r < live;
    const uint64_t mask = in ? rows.mask(r) : 0;
    const int depth = __popcll(mask) - 1;
    const uint32_t at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16), out = at + L::kOutputs + slot * D;
    const float scale2 = kCap ? p.scale / p.softcap : p.scale * kLog2e;
    const float cap2 = p.softcap * kLog2e, slope2 = kBias && in ? p.slopes[rows.head(r)] * kLog2e : 0.0f;
    const int steps = warp * 32 < live ? n : 0;
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
      const int64_t key0 = static_cast<int64_t>(begin + c) * kKeys;
      const bool nodes = key0 + kKeys > w.n;  // keys of the tree, or beyond the last
      if (kCap) {
        float far = 0.0f;
#pragma unroll
        for (int e = 0; e < 64; ++e) far = fmaxf(far, fabsf(__uint_as_float(x[e / 32][e % 32])));
        if (__all_sync(0xFFFFFFFFu, far * fabsf(scale2) < kNearCap)) {
          const uint64_t over2 = pack2(scale2, scale2), caps = pack2(cap2, cap2);
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            uint32_t* two = &x[e / 32][e % 32];
            const uint64_t y = capped_near(static_cast<uint64_t>(two[1]) << 32 | two[0], over2, caps);
            two[0] = static_cast<uint32_t>(y), two[1] = static_cast<uint32_t>(y >> 32);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 64; ++e)
            x[e / 32][e % 32] = __float_as_uint(capped(__uint_as_float(x[e / 32][e % 32]), scale2, cap2));
        }
      }
      if (kBias) {
        const float times = kCap ? 1.0f : scale2;
        const float away = static_cast<float>(w.n + depth - key0);  // exact, and its differences, below 2^24
        if (!nodes) {
#pragma unroll
          for (int e = 0; e < 64; ++e)
            x[e / 32][e % 32] = __float_as_uint(__uint_as_float(x[e / 32][e % 32]) * times - slope2 * (away - e));
        } else {
#pragma unroll
          for (int e = 0; e < 64; ++e) {
            const int64_t node = key0 + e - w.n;
            const float far = node < 0 ? away - e : node < 64 ? fabsf(static_cast<float>(depth + 1 - __popcll(sh.rows.masks[node]))) : 0.0f;
            x[e / 32][e % 32] = __float_as_uint(__uint_as_float(x[e / 32][e % 32]) * times - slope2 * far);
          }
        }
      }
      if (nodes || __any_sync(0xFFFFFFFFu, mask == 0)) {
        const int64_t ahead = w.n - key0;  // the step's first keys that are not the tree's
        uint64_t seen = mask == 0 || ahead <= 0 ? 0 : ahead >= 64 ? ~UINT64_C(0) : (UINT64_C(1) << ahead) - 1;
        if (ahead < 64 && ahead > -64) seen |= ahead >= 0 ? mask << ahead : mask >> -ahead;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t bits = static_cast<uint32_t>(seen >> 32 * h);
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (!(bits >> e & 1)) x[h][e] = __float_as_uint(-kInf);
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
      const bool moved = base > -kInf && top > base + kSlack;
      if (__any_sync(0xFFFFFFFFu, moved)) {
        const float back = moved ? exp2_approx(base - top) : 1.0f;
        total *= back;
        alive = mbar_wait_warp(&sh.o_done[slot][b ^ 1], (c - 1) >> 1 & 1, dead);  // the step before is in the output
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
        uint32_t weights[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint64_t t =
              fma2(pack2(__uint_as_float(x[half][2 * i]), __uint_as_float(x[half][2 * i + 1])), times2, shift2);
          const float u = exp2_approx(low2(t)), v = exp2_approx(high2(t));
          sums[i & 1] = add2(sums[i & 1], pack2(u, v));
          weights[i] = narrow2<T>(u, v);
        }
        tmem_store16(scores + half * 16, weights);
      }
      const uint64_t sum = add2(sums[0], sums[1]);
      total += low2(sum) + high2(sum);
      tmem_wait_st();
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_full[slot][b]);
    }
    if (steps > 0 && alive) alive = mbar_wait_warp(&sh.o_done[slot][(steps - 1) & 1], (steps - 1) >> 1 & 1, dead);
    sh.top[r] = steps > 0 ? base : -kInf;
    sh.total[r] = steps > 0 ? total : 0.0f;
    tmem_fence_after();
  }
  __syncthreads();  // the products are done: the outputs take the place of what they read
  float* outs = reinterpret_cast<float*>(tiles);
  if (warp < kSoftmaxWarps && warp * 32 < live && sh.dead == 0) {
    const uint32_t at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + L::kOutputs + (warp >> 2) * D;
    const uint64_t mask = tid < live ? rows.mask(tid) : 0;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[32];
      tmem_load32(o, at + c * 32);
      tmem_wait_ld(o);
      if (sh.any_odd) {
        uint32_t odd = 0;
        for (int j = 0; j < 64; ++j)
          if (mask >> j & 1) odd |= sh.odd[j][c];
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if (odd >> e & 1) o[e] = 0x7FC00000u;
      }
#pragma unroll
      for (int e = 0; e < 32; e += 4)
        *reinterpret_cast<uint4*>(outs + tid * L::kPitch + c * 32 + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
    }
  }
  if (tid == 0 && sh.dead != 0) sh.bad = 1;
  tmem_fence_before();
  __syncthreads();
  if (warp == kSoftmaxWarps) {
    tmem_fence_after();
    tmem_free(tmem, L::kColumns);
  }
  __syncwarp();
  rows_join<T, D, L::kPitch, L::kThreads>(p, w, rows, outs, sh.top, sh.total, &sh.bad);
}

template <typename T, int D, int kSlots, bool kCap, bool kBias>
cudaError_t launch_kind(DraftParams p, int64_t batch, int sms, cudaStream_t stream) {
  using L = Plan<D, kSlots>;
  p.head_blocks = (p.drafts * p.group + L::kBlock - 1) / L::kBlock;
  const int64_t items = batch * p.kv_heads * p.head_blocks;
  const int c = decode_cluster(items, p.max_pages * p.page_size, sms, 6);
  return launch_decode(draft_wide_kernel<T, D, kSlots, kCap, kBias>, p, items, c, L::kThreads, L::kBytes, stream);
}

template <typename T, int D, int kSlots>
cudaError_t launch_slots(const DraftParams& p, int64_t batch, int sms, cudaStream_t stream) {
  if (p.softcap > 0.0f)
    return p.slopes != nullptr ? launch_kind<T, D, kSlots, true, true>(p, batch, sms, stream)
                               : launch_kind<T, D, kSlots, true, false>(p, batch, sms, stream);
  return p.slopes != nullptr ? launch_kind<T, D, kSlots, false, true>(p, batch, sms, stream)
                             : launch_kind<T, D, kSlots, false, false>(p, batch, sms, stream);
}

template <typename T>
cudaError_t launch_head(const DraftParams& p, int64_t batch, int sms, cudaStream_t stream) {
  const bool two = p.drafts * p.group > kRows;
  if (p.dim <= 64) return two ? launch_slots<T, 64, 2>(p, batch, sms, stream) : launch_slots<T, 64, 1>(p, batch, sms, stream);
  return two ? launch_slots<T, 128, 2>(p, batch, sms, stream) : launch_slots<T, 128, 1>(p, batch, sms, stream);
}

}  // namespace

bool launch_draft_wide(const DraftParams& p, int64_t batch, int dtype, int sms, cudaStream_t stream, cudaError_t* e) {
  // The scores' maximum is taken before the scale, and -inf times it has to stay -inf: it is positive
  if (dtype == 0 || p.dim > 128 || !paged_vectors(p) || !(p.scale > 0.0f) || p.drafts * p.group <= 32) return false;
  *e = dtype == 1 ? launch_head<__nv_bfloat16>(p, batch, sms, stream) : launch_head<__half>(p, batch, sms, stream);
  return true;
}

}  // namespace zo
