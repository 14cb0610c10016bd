// zo_draft_wide.cu -- attention of trees of drafted tokens over a paged cache
// where many rows share a key (zo_attention_draft): tcgen05, 16-bit types, heads
// of up to 128 elements, vectors aligned to 16 bytes.
#include <algorithm>

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
  static constexpr int kBytes = kSlots * kQueries + kStages * kTile + 1024;
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
  float2 part[kRows];   // the copies' statistics
  uint32_t tmem;
  int dead, any_odd;
};

// A copy's output in the joint one's units; one that has seen nothing has none.
__device__ __forceinline__ float times_scale(uint32_t o, float scale) { return scale == 0.0f ? 0.0f : __uint_as_float(o) * scale; }

template <typename T>
__device__ __forceinline__ bool odd16(uint32_t v) {  // infinite or NaN
  constexpr uint32_t kExponent = __is_same(T, __nv_bfloat16) ? 0x7F80u : 0x7C00u;
  return (v & kExponent) == kExponent;
}

template <typename T>
__device__ __forceinline__ bool odd32(uint32_t v) {  // either of two values
  return odd16<T>(v) || odd16<T>(v >> 16);
}

// The work of all sequences, heads and blocks of rows in a line of steps, cut into as many equal runs as there are CTAs: with
// runs, unlike clusters, every SM has a CTA and each as many steps (+- 1), whatever the lengths. A CTA takes its run piece by
// piece, a piece being the steps of one block of rows; one that is not the whole block leaves its unscaled outputs and
// statistics in the workspace (the first in place 2 i of CTA i, the last in 2 i + 1), and draft_wide_join_kernel puts the
// pieces together.
constexpr int kMaxCtas = 304;  // of one slot; of two, half as many
constexpr int kFewest = 110;   // units of a CTA
constexpr int kStart = 120;    // units that a piece's start and end cost (10 us); a block of rows counts as that many more
// Units of a step, measured at 0.08 us each: up to 64 rows are bound by HBM, more by their softmax.
__device__ __forceinline__ int units_of_step(int rows) { return rows > 128 ? 11 : rows > 64 ? 10 : 8; }

// Steps that lie wholly in front of a unit of a block of rows.
__device__ __forceinline__ int steps_before(int64_t unit, int per_step) {
  return unit <= kStart ? 0 : static_cast<int>(static_cast<uint32_t>(unit - kStart) / static_cast<uint32_t>(per_step));
}

struct WideParams : DraftParams {
  int64_t batch;
  int64_t* prefix;   // [batch + 1] units in front of a sequence
  int4* shape;       // [batch] units of a block of rows (kStart and its steps'), steps, units of a step, blocks that see anything
  int32_t* bad;      // [batch]
  float2* stats;     // [2 CTAs][rows of a block] log2 of what the weights are relative to, their sum
  float4* outs;      // [2 CTAs][D / 4][rows of a block]: neighbouring rows' columns together, as threads have them
  int32_t ctas, block;
  int32_t rows_at_once;  // of a page by TMA, 0: none
};

// The first unit of CTA i (or of none, i = ctas), and the CTA of a unit.
struct Runs {
  int64_t each, more;  // units of a CTA; CTAs with one more
  int ctas;
  __device__ __forceinline__ Runs(int64_t units, int most) {
    ctas = static_cast<int>(min(static_cast<int64_t>(most), (units + kFewest - 1) / kFewest));
    each = ctas > 0 ? units / ctas : 0;
    more = units - each * ctas;
  }
  __device__ __forceinline__ int64_t first(int64_t i) const { return i * each + min(i, more); }
  __device__ __forceinline__ int64_t cta(int64_t unit) const {
    return unit < more * (each + 1) ? unit / (each + 1) : more + (unit - more * (each + 1)) / each;
  }
};

// The sequences' shapes and the sums of their steps, in one CTA; a warp has a sequence.
__global__ void __launch_bounds__(1024) draft_wide_plan_kernel(const __grid_constant__ WideParams p) {
  __shared__ int64_t steps[1024];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int64_t before = 0;
  for (int64_t first = 0; first < p.batch; first += 1024) {
    const int64_t here = min(static_cast<int64_t>(1024), p.batch - first);
    for (int64_t i = warp; i < here; i += 32) {
      const int n = p.lengths[first + i];
      const auto mask = [&](int node) {
        return node < p.drafts ? p.masks[(first + i) * p.drafts + node] & (~UINT64_C(0) >> (64 - p.drafts)) : UINT64_C(0);
      };
      const uint64_t a = mask(lane), b = mask(lane + 32);
      const DraftKeys k = draft_keys(p, max(n, 0), n >= 0 ? a : 0, n >= 0 ? b : 0);
      const int count = k.bad ? 0 : static_cast<int>((k.len + kKeys - 1) / kKeys);
      const int per_step = units_of_step(min(k.nodes * p.group, p.block));
      const int64_t each = count == 0 ? 0 : kStart + count * static_cast<int64_t>(per_step);
      const int blocks = (k.nodes * p.group + p.block - 1) / p.block;
      if (lane == 0) {
        p.shape[first + i] = make_int4(static_cast<int>(each), count, per_step, blocks);
        p.bad[first + i] = k.bad;
        steps[i] = each * blocks * p.kv_heads;
      }
    }
    __syncthreads();
    int64_t mine = tid < here ? steps[tid] : 0, all = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xFFFFFFFFu, all, o);
      if (lane >= o) all += x;
    }
    __syncthreads();
    if (lane == 31) steps[warp] = all;
    __syncthreads();
    int64_t sum = before;
    for (int i = 0; i < 32; ++i) {
      if (i < warp) all += steps[i];
      sum += steps[i];
    }
    if (tid < here) p.prefix[first + tid] = before + all - mine;
    before = sum;
    __syncthreads();
  }
  if (tid == 0) p.prefix[p.batch] = before;
}

// With up to 32 or 64 rows, which would leave three warps or two of a slot's four without any, the rows are there four times
// or twice, in lanes of their own, and each copy takes its part of every step's keys: its weights for the others are zero.
//
// A block of up to 128 kSlots rows at a time: rows are what they are in zo_draft.cu,
// products and barriers as in zo_attention_mma.cu (a slot's scores of two steps
// and their weights in tensor memory, a step's scores issued behind the output
// of the one two before it).
//
//   warps 0-3 (4-7)   softmax of slot 0 (1): a thread has a row; those without a row that sees anything stay out
//   the next (two)    the products of slot 0 (1)
//   the last two      keys and values: by TMA, a lane per page, where a step has no key of the tree and pages and steps begin
//                     together; else by cp.async, a lane per key
//
// 16 sequences of up to 16384 keys, trees of up to 64 nodes, 32 / 8 heads of 128, bf16 (646 MB, 97 us by HBM): 138 us, of which
// 5 plan and launch, 115 to 120 are the steps and 11 the join. A step takes 0.65 us with up to 64 rows, which is HBM's rate
// (152 x 32 KB), 0.84 with 256, whose softmax and products take turns as in zo_attention_mma.cu; a piece's start and end cost
// some 8. On the way: clusters per block of rows joined over distributed shared memory 356 us (an SM had work for two thirds
// of the time: a cluster of 8 waits for 8 SMs of a GPC, and lengths are unequal); equal runs of steps 281; pages by TMA instead of cp.async 183
// (two warps cannot issue 32 KB of 16-byte copies and their addresses per 0.7 us); pieces by columns 160 (by rows a warp's store
// touches 32 lines); shares by what a step and a start were measured at, loads ahead of the queries 149; pages looked up in
// groups 145. 16 of up to 4001 keys, trees of 26, 32 heads of 64, fp16, capped and biased (49 us by HBM): 92 us, with one copy of
// the rows 180, two 119; a step is held by the softmax's latency (1000 cycles) and the issue of TMA for pages of 16 rows.
template <typename T, int D, int kSlots, int kCopies, bool kPlain>
__global__ void __launch_bounds__(Plan<D, kSlots>::kThreads, 3 - kSlots)
    draft_wide_kernel(const __grid_constant__ WideParams p, const __grid_constant__ CUtensorMap k_map,
                      const __grid_constant__ CUtensorMap v_map) {
  using L = Plan<D, kSlots>;
  constexpr int kSoftmaxWarps = L::kSoftmaxWarps, kVectors = D / 8;
  constexpr int kSpan = L::kBlock / kCopies, kColumns = kKeys / kCopies;  // rows of a copy, a step's keys that are its own
  static_assert(kSlots == 1 || kCopies == 1, "");
  constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
  extern __shared__ uint8_t raw[];
  __shared__ Shared<kSlots> sh;
  uint8_t* tiles = raw + (1024 - smem_address(raw) % 1024) % 1024;  // the slots' queries, then the stages
  uint8_t* stages = tiles + kSlots * L::kQueries;
  const int tid = threadIdx.x, warp = static_cast<int>(uniform(tid >> 5)), lane = tid & 31;
  volatile int* dead = &sh.dead;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (warp == kSoftmaxWarps) tmem_alloc(&sh.tmem, L::kColumns);
  if (tid == 0) sh.dead = 0;
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = uniform(sh.tmem);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Runs runs(p.prefix[p.batch], p.ctas);
  const int64_t start = blockIdx.x < runs.ctas ? runs.first(blockIdx.x) : 0;
  const int64_t stop = blockIdx.x < runs.ctas ? runs.first(blockIdx.x + 1) : 0;
  bool again = false;
  for (int64_t at_unit = start; at_unit < stop;) {
    // the last sequence whose steps begin here or before: by 32 places at a time
    int64_t b = 0;
    for (int64_t end = p.batch; end - b > 1;) {
      const int64_t stride = (end - b + 31) / 32, mine = b + lane * stride;
      const uint32_t before = __ballot_sync(0xFFFFFFFFu, mine < end && p.prefix[mine] <= at_unit);
      b += (31 - __clz(before)) * stride;
      end = min(end, b + stride);
    }
    const int4 shape = p.shape[b];
    const int64_t inside = at_unit - p.prefix[b];
    const int item = static_cast<int>(inside / shape.x), from = static_cast<int>(inside - static_cast<int64_t>(item) * shape.x);
    const int units = static_cast<int>(min(static_cast<int64_t>(shape.x - from), stop - at_unit));
    const int begin = steps_before(from, shape.z), n = steps_before(from + static_cast<int64_t>(units), shape.z) - begin;
    if (n == 0) {
      at_unit += units;
      continue;
    }
    const int g = item / shape.w;
    const DraftPlace w = draft_place<L::kBlock>(p, static_cast<int>(b), g, item - g * shape.w, sh.rows);
    const DraftRows<T, L::kBlock> rows = {p, w, sh.rows};
    const int live = w.live;
    const auto warps_of = [&](int s) {
      return kCopies > 1 ? kCopies * ((live + 31) / 32) : max(0, min(4, (live - s * kRows + 31) / 32));
    };

    if (tid == L::kThreads - 32) {
      const int slots = (live + kRows - 1) / kRows;
      const auto barrier = [&](uint64_t* x, int count) {
        if (again) mbar_inval(x);
        mbar_init(x, count > 0 ? count : 1);
      };
      for (int i = 0; i < L::kStages; ++i) {
        barrier(&sh.full[i], kLoaders);
        barrier(&sh.empty[i], slots);
      }
      for (int s = 0; s < kSlots; ++s) {
        for (int b = 0; b < 2; ++b) {
          barrier(&sh.s_full[s][b], 1);
          barrier(&sh.p_full[s][b], warps_of(s));
          barrier(&sh.o_done[s][b], 1);
        }
        barrier(&sh.drain[s], 1);
      }
      sh.any_odd = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    again = true;
    // With a bias by distance from the last step to the first: a row's largest scores come first then, and its output is not
    // rescaled at every step (26 rows of 32 heads of 64: 100 -> 96 us).
    constexpr bool kBackward = !kPlain;
    const auto step_of = [&](int l) { return kBackward ? n - 1 - l / 2 : l / 2; };  // of tile l
    // the warps of the softmax and the products; the loads need not wait for the queries
    const auto softmax_warps = [] { asm volatile("bar.sync 2, %0;" ::"n"(kSoftmaxWarps * 32) : "memory"); };
    const auto queries_there = [] { asm volatile("bar.sync 1, %0;" ::"n"((kSoftmaxWarps + kSlots) * 32) : "memory"); };
    for (int i = tid; i < 64 * 4; i += L::kThreads) (&sh.odd[0][0])[i] = 0;
    __syncthreads();

    if (warp >= kSoftmaxWarps + kSlots) {
      // Tile l is a step's keys (even) or values. Each of the two warps has 32 of its keys, a lane one of their places.
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
          const int64_t key0 = static_cast<int64_t>(begin + step_of(l)) * kKeys;
          if (key0 + kKeys > w.n) {
            // Values of the tree's keys that are not finite are noted and taken out: a row that does not see one has the
            // weight 0 there, and 0 times it is NaN.
#pragma unroll 4
            for (int i = 0; i < 32 / kAtOnce; ++i) {
              const int64_t node = key0 + half * 32 + i * kAtOnce + lane / kVectors - w.n;
              uint16_t* x = reinterpret_cast<uint16_t*>(place_of(l, i));
              const uint4 u = *reinterpret_cast<const uint4*>(x);
              if (node < 0 || node >= 64 || !(odd32<T>(u.x) || odd32<T>(u.y) || odd32<T>(u.z) || odd32<T>(u.w))) continue;
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
      // by TMA: a box of rows_at_once keys of a page; lanes hold the pages of as many steps as there is room for, and of as many
      // behind them (a page looked up a step ahead would be waited for: 1.0 us of a step of 64 x 64 elements, which takes 0.7)
      const int boxes = p.rows_at_once > 0 ? kKeys / p.rows_at_once : 0, held = boxes > 0 ? 32 / boxes : 1;
      const auto whole = [&](int step) { return boxes > 0 && static_cast<int64_t>(begin + step + 1) * kKeys <= w.n; };
      const auto look_pages = [&](int l) {  // of the steps from tile l on
        const int step = boxes == 0 ? -1 : kBackward ? step_of(l) - lane / boxes : step_of(l) + lane / boxes;
        const int64_t j = static_cast<int64_t>(begin + step) * kKeys + lane % (boxes > 0 ? boxes : 1) * p.rows_at_once;
        return step >= 0 && step < n && j < w.n ? p.pages[w.b * p.pages_stride + decode_page(p, j)] : 0;
      };
      int first_tiled = 0;  // backward, the first step may hold the tree's keys, and the second
      while (kBackward && boxes > 0 && first_tiled < 2 * n && !whole(step_of(first_tiled))) first_tiled += 2;
      int ids = look_pages(first_tiled), next_ids = look_pages(first_tiled + 2 * held), at_id = 0;
      int id = whole(step_of(0)) ? 0 : look(step_of(0)), box_page = 0, box_row = 0;
      int64_t k_at = -1, v_at = -1;
      bool alive = true;
      int issued = 0;
      for (int l = 0; l < 2 * n && alive; ++l) {
        const bool tiled = whole(step_of(l)), mine = !tiled || half == l % 2;  // by TMA one warp has the keys, the other the values
        if (mine && l >= L::kStages) alive = mbar_wait_warp(&sh.empty[l % L::kStages], (l / L::kStages - 1) & 1, dead);
        if (!alive) break;
        if (l % 2 == 0) {
          if (tiled) {
            const uint32_t j = static_cast<uint32_t>(begin + step_of(l)) * kKeys + lane * p.rows_at_once;
            box_page = __shfl_sync(0xFFFFFFFFu, ids, (at_id * boxes + lane) & 31);
            box_row = static_cast<int>(j - decode_page(p, j) * static_cast<uint32_t>(p.page_size));
            if (lane < boxes && (box_page < 0 || box_page >= p.n_pages)) bad = 1;  // (and zeros come)
            if (++at_id == held) {
              at_id = 0;
              ids = next_ids;
              next_ids = look_pages(l + 2 + 2 * held);
            }
          } else {
            const int64_t j = key_of(step_of(l));
            const int2 key = decode_key(p, w, draft_sees(w, j) ? j : w.len, id, bad);
            k_at = key.x >= 0 ? (key.x * p.k_page + key.y * p.k_token) * 2 : -1;
            v_at = key.x >= 0 ? (key.x * p.v_page + key.y * p.v_token) * 2 : -1;
          }
          if (l + 2 < 2 * n && !whole(step_of(l + 2))) id = look(step_of(l + 2));
        }
        if (tiled) {
          uint64_t* const full = &sh.full[l % L::kStages];
          if (mine && lane == 0) {
            mbar_expect(full, L::kTile);
            mbar_arrive(full);  // for the other
          }
          __syncwarp();
          if (mine && lane < boxes) {
            uint8_t* const to = stages + l % L::kStages * L::kTile + lane * p.rows_at_once * 128;
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
              tma_load_4d(to + c * L::kTileChunk, l % 2 == 0 ? &k_map : &v_map, c * 64, w.g, box_row, box_page, full);
          }
          __syncwarp();
        } else {
#pragma unroll
          for (int i = 0; i < 32 / kAtOnce; ++i) {
            const int64_t at = __shfl_sync(0xFFFFFFFFu, l % 2 == 0 ? k_at : v_at, i * kAtOnce + lane / kVectors);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_address(place_of(l, i))),
                         "l"((l % 2 == 0 ? kl : vl) + (at >= 0 ? at : 0)), "r"(at >= 0 ? bytes : 0)
                         : "memory");
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        ++issued;
        if (l >= L::kAhead) {
          asm volatile("cp.async.wait_group %0;" ::"n"(L::kAhead) : "memory");
          if (!whole(step_of(l - L::kAhead))) arrived(l - L::kAhead);
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (alive)
        for (int l = max(0, issued - L::kAhead); l < issued; ++l)
          if (!whole(step_of(l))) arrived(l);
      if (lane == 0 && *dead) {  // nothing may land in shared memory after the CTA is gone
        const long long start = clock64();
        for (int l = max(0, issued - L::kStages); l < issued; ++l)
          while (whole(step_of(l)) && !mbar_try(&sh.full[l % L::kStages], l / L::kStages & 1) && clock64() - start < kWaitCycles) {}
      }
      __syncwarp();
      // the barriers are made anew for the next block: every arrival has come before that
      for (int l = max(0, 2 * n - L::kStages); l < 2 * n && alive; ++l)
        alive = mbar_wait_warp(&sh.empty[l % L::kStages], l / L::kStages & 1, dead);
      if (bad) p.bad[w.b] = 1;
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
      queries_there();
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
      // The queries, swizzled as a product's operand is: 16-byte vector v of a row goes to place v ^ (row mod 8) of its 64
      // elements, a copy behind another. Rows that are none are zeros.
      const bool whole = aligned_to(p.q, 16) && p.q_token % 8 == 0 && p.q_node % 8 == 0 && p.q_head % 8 == 0;
      for (int i = tid; i < L::kBlock * kVectors; i += kSoftmaxWarps * 32) {
        const int r = i / kVectors, v = i % kVectors;
        uint8_t* to = tiles + r / kRows * L::kQueries + v / 8 * kChunk + r % kRows * 128 + ((v % 8 ^ (r & 7)) << 4);
        uint4 x = make_uint4(0, 0, 0, 0);
        if (r % kSpan < live && v * 8 < p.dim) {
          const T* q = rows.query(r % kSpan) + v * 8;
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
      __syncwarp();
      queries_there();
      const int slot = warp >> 2, r = tid % kSpan, copy = kCopies > 1 ? warp / (4 / kCopies) : 0;  // the thread's row
      const bool in = r < live, cap = !kPlain && p.softcap > 0.0f, bias = !kPlain && p.slopes != nullptr;
      const uint64_t mask = in ? rows.mask(r) : 0;
      const int depth = __popcll(mask) - 1;
      const uint32_t at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16), out = at + L::kOutputs + slot * D;
      const float scale2 = cap ? p.scale / p.softcap : p.scale * kLog2e;
      const float cap2 = p.softcap * kLog2e, slope2 = bias && in ? p.slopes[rows.head(r)] * kLog2e : 0.0f;
      const int steps = warp * 32 % kSpan < live ? n : 0;
      float base = -kInf, total = 0.0f;  // log2 of what the weights are relative to, and their sum
      bool alive = true;
      for (int c = 0; c < steps; ++c) {
        const int b = c & 1;
        const uint32_t scores = at + slot * 128 + b * kKeys;
        alive = mbar_wait_warp(&sh.s_full[slot][b], c >> 1 & 1, dead);
        if (!alive) break;
        tmem_fence_after();
        constexpr int kWidth = kColumns < 32 ? kColumns : 32;
        uint32_t x[kColumns / kWidth][kWidth];
        if constexpr (kWidth == 16) {
          tmem_load16_wait(x[0], scores + copy * kColumns);
        } else {
          tmem_load32(x[0], scores + copy * kColumns);
          if constexpr (kColumns == 64) tmem_load32(x[1], scores + 32);
          tmem_wait_ld(x[0]);
          if constexpr (kColumns == 64) tie32(x[1]);
        }
        const auto score = [&](int e) -> uint32_t& { return x[e / kWidth][e % kWidth]; };
        const auto two = [&](int e) { return static_cast<uint64_t>(score(e + 1)) << 32 | score(e); };
        const auto put_two = [&](int e, uint64_t y) {
          score(e) = static_cast<uint32_t>(y), score(e + 1) = static_cast<uint32_t>(y >> 32);
        };
        const int key0 = (begin + step_of(2 * c)) * kKeys + copy * kColumns;  // (the last step's end is below 2^31)
        const bool nodes = key0 + kColumns > w.n;  // keys of the tree, or beyond the last
        if (cap) {
          float fars[4] = {};
#pragma unroll
          for (int e = 0; e < kColumns; ++e) fars[e % 4] = fmaxf(fars[e % 4], fabsf(__uint_as_float(score(e))));
          const float far = fmaxf(fmaxf(fars[0], fars[1]), fmaxf(fars[2], fars[3]));
          if (__builtin_expect(__all_sync(0xFFFFFFFFu, far * fabsf(scale2) < kNearCap), 1)) {
            const uint64_t over2 = pack2(scale2, scale2), caps = pack2(cap2, cap2);
#pragma unroll
            for (int e = 0; e < kColumns; e += 2) put_two(e, capped_near(two(e), over2, caps));
          } else {
#pragma unroll
            for (int e = 0; e < kColumns; ++e) score(e) = __float_as_uint(capped(__uint_as_float(score(e)), scale2, cap2));
          }
        } else if (!kPlain) {
#pragma unroll
          for (int e = 0; e < kColumns; e += 2) put_two(e, mul2(two(e), pack2(scale2, scale2)));
        }
        if (bias) {
          const float away = static_cast<float>(w.n - key0 + depth);  // exact, and its differences, below 2^24
          if (__builtin_expect(!nodes, 1)) {
#pragma unroll
            for (int e = 0; e < kColumns; e += 2)
              put_two(e, fma2(pack2(-slope2, -slope2),
                              add2(pack2(away, away), pack2(-static_cast<float>(e), -static_cast<float>(e + 1))), two(e)));
          } else {
#pragma unroll
            for (int e = 0; e < kColumns; ++e) {
              const int node = key0 - w.n + e;
              const int place = node >= 0 && node < 64 ? __popcll(sh.rows.masks[node]) - 1 : depth;
              const float far = node < 0 ? away - e : fabsf(static_cast<float>(depth - place));
              score(e) = __float_as_uint(fmaf(-slope2, far, __uint_as_float(score(e))));
            }
          }
        }
        if (__builtin_expect(nodes || __any_sync(0xFFFFFFFFu, mask == 0), 0)) {
          const int ahead = w.n - key0;  // the columns' first keys that are not the tree's
          uint64_t seen = mask == 0 || ahead <= 0 ? 0 : ahead >= 64 ? ~UINT64_C(0) : (UINT64_C(1) << ahead) - 1;
          if (ahead < 64 && ahead > -64) seen |= ahead >= 0 ? mask << ahead : mask >> -ahead;
#pragma unroll
          for (int h = 0; h < kColumns / kWidth; ++h) {
            const uint32_t bits = static_cast<uint32_t>(seen >> 32 * h);
#pragma unroll
            for (int e = 0; e < kWidth; ++e)
              if (!(bits >> e & 1)) x[h][e] = __float_as_uint(-kInf);
          }
        }
        float most[4];
#pragma unroll
        for (int e = 0; e < kColumns; ++e) {
          const float y = __uint_as_float(score(e));
          most[e % 4] = e < 4 ? y : fmaxf(most[e % 4], y);
        }
        float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
        if (kPlain) top *= scale2;
        top -= kLift<T>;
        const bool moved = base > -kInf && top > base + kSlack;
        if (__builtin_expect(__any_sync(0xFFFFFFFFu, moved), 0)) {
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
        const float times = kPlain ? scale2 : 1.0f;
        const uint64_t times2 = pack2(times, times), shift2 = pack2(shift, shift);
        uint64_t sums[2] = {0, 0};
        uint32_t weights[kColumns / 2];  // rounded to 16 bits for the tensor cores, as in zo_draft.cu
#pragma unroll
        for (int i = 0; i < kColumns / 2; ++i) {
          const uint64_t t = fma2(two(2 * i), times2, shift2);
          const float u = exp2_approx(low2(t)), v = exp2_approx(high2(t));
          sums[i & 1] = add2(sums[i & 1], pack2(u, v));
          weights[i] = narrow2<T>(u, v);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // the other copies' keys weigh nothing here
          uint32_t all[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            constexpr int kMine = kColumns / 2;
            all[i] = kCopies == 1 || (half * 16 + i) / kMine == copy ? weights[(half * 16 + i) % kMine] : 0;
          }
          tmem_store16(scores + half * 16, all);
        }
        const uint64_t sum = add2(sums[0], sums[1]);
        total += low2(sum) + high2(sum);
        tmem_wait_st();
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[slot][b]);
      }
      for (int c = max(0, steps - 2); c < steps && alive; ++c) alive = mbar_wait_warp(&sh.o_done[slot][c & 1], c >> 1 & 1, dead);
      tmem_fence_after();
      float scale = 1.0f;  // of a copy's outputs
      float* const gathered = reinterpret_cast<float*>(stages);  // the copies' behind the first, in place of keys and values
      constexpr int kPitch = D + 4;
      if constexpr (kCopies > 1) {  // the copies' statistics, then their outputs, as one
        sh.part[tid] = make_float2(base, total);
        softmax_warps();
        float most = -kInf, all = 0.0f;
#pragma unroll
        for (int k = 0; k < kCopies; ++k) most = fmaxf(most, sh.part[k * kSpan + r].x);
#pragma unroll
        for (int k = 0; k < kCopies; ++k) {
          const float2 part = sh.part[k * kSpan + r];
          all += part.y != part.y ? part.y : part.x == -kInf ? 0.0f : part.y * exp2_approx(part.x - most);
        }
        scale = base == -kInf ? 0.0f : exp2_approx(base - most);
        base = most, total = all;
        if (copy > 0 && steps > 0 && alive) {
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_load32(o, out + c * 32);
            tmem_wait_ld(o);
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(gathered + ((copy - 1) * kSpan + r) * kPitch + c * 32 + e) =
                  make_float4(times_scale(o[e], scale), times_scale(o[e + 1], scale), times_scale(o[e + 2], scale),
                              times_scale(o[e + 3], scale));
          }
          tmem_fence_before();
        }
        softmax_warps();
      }
      if (steps > 0 && alive && copy == 0) {
        const bool whole = n == shape.y, seen = total != 0.0f;
        const float over = seen ? 1.0f / total : 0.0f;
        const int64_t place_of_cta = 2 * static_cast<int64_t>(blockIdx.x) + (at_unit > start);
        T* const to = rows.row(r);
        const bool vectors = reinterpret_cast<uintptr_t>(to) % 16 == 0;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          __syncwarp();  // the load is the whole warp's; the stores of the columns before split it by rows and alignment
          tmem_load32(o, out + c * 32);
          tmem_wait_ld(o);
          if constexpr (kCopies > 1) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              float y[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) y[i] = times_scale(o[e + i], scale);
#pragma unroll
              for (int k = 0; k < kCopies - 1; ++k) {
                const float4 z = *reinterpret_cast<const float4*>(gathered + (k * kSpan + r) * kPitch + c * 32 + e);
                y[0] += z.x, y[1] += z.y, y[2] += z.z, y[3] += z.w;
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) o[e + i] = __float_as_uint(y[i]);
            }
          }
          if (sh.any_odd) {
            uint32_t odd = 0;
            for (int j = 0; j < 64; ++j)
              if (mask >> j & 1) odd |= sh.odd[j][c];
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (odd >> e & 1) o[e] = 0x7FC00000u;
          }
          if (in && whole) {
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
              float f[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) f[i] = seen ? __uint_as_float(o[e + i]) * over : 0.0f;
              const uint4 u = Vec<T>::narrow_all(f);
              if (c * 32 + e >= p.dim) continue;
              if (vectors) {
                *reinterpret_cast<uint4*>(to + c * 32 + e) = u;
              } else {
                const uint32_t two[4] = {u.x, u.y, u.z, u.w};
                uint16_t* one = reinterpret_cast<uint16_t*>(to + c * 32 + e);
#pragma unroll
                for (int i = 0; i < 8; ++i) one[i] = static_cast<uint16_t>(two[i / 2] >> 16 * (i & 1));
              }
            }
          } else if (in) {
            float4* part = p.outs + (place_of_cta * (D / 4) + c * 8) * L::kBlock + tid;
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              part[e / 4 * L::kBlock] = make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]), __uint_as_float(o[e + 2]),
                                                    __uint_as_float(o[e + 3]));
          }
        }
        if (in && whole) {
          if (p.lse != nullptr) *rows.sum(r) = seen ? (base + log2f(total)) * kLn2 : -kInf;
        } else if (in) {
          p.stats[place_of_cta * L::kBlock + tid] = make_float2(base, total);
        }
        __syncwarp();
        tmem_fence_before();
      }
      if constexpr (kCopies > 1) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // TMA's turn
    }
    __syncthreads();
    tmem_fence_after();
    if (sh.dead != 0) {  // what is left of the run is not formed
      if (tid == 0) p.bad[w.b] = 1;
      at_unit += units;
      for (b += 1; b < p.batch && p.prefix[b] < stop; ++b)
        if (tid == 0) p.bad[b] = 1;
      break;
    }
    at_unit += units;
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == kSoftmaxWarps) {
    tmem_fence_after();
    tmem_free(tmem, L::kColumns);
  }
}

// 32 rows of a block, a lane per row: the pieces of their block, if there is more than one; rows that see nothing, and those of
// sequences whose pages are none. Warps share the columns, and the rows leave through shared memory.
template <typename T, int D>
__global__ void __launch_bounds__(256, 4) draft_wide_join_kernel(const __grid_constant__ WideParams p) {
  constexpr int kWarps = 8, kMine = D / 4 / kWarps;  // a warp's vectors of 4 columns
  constexpr int kPitch = D + 8;                      // 16-bit elements of a row
  __shared__ __align__(16) T tile[32 * kPitch];
  __shared__ int64_t to_row[32];  // where its elements go, -1: nowhere
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t chunks = p.block / 32, rows = p.drafts * p.group, blocks = (rows + p.block - 1) / p.block;
  const uint32_t item = blockIdx.x / chunks, chunk = blockIdx.x - item * chunks;
  const uint32_t head_block = item / blocks, block = item - head_block * blocks;
  const uint32_t b = head_block / p.kv_heads, g = head_block - b * p.kv_heads;
  const uint32_t in_block = chunk * 32 + lane, r = block * p.block + in_block;
  if (block * p.block + chunk * 32 >= rows) return;
  const bool in = r < rows;
  const uint32_t node = (in ? r : rows - 1) / p.group, head = g * p.group + (in ? r : rows - 1) - node * p.group;
  const uint64_t mask = p.masks[static_cast<int64_t>(b) * p.drafts + node] & (~UINT64_C(0) >> (64 - p.drafts));
  const bool sees = p.lengths[b] >= 0 && mask != 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int4 shape = p.shape[b];
  const int64_t before = p.prefix[b], all = p.prefix[p.batch];
  const bool bad = p.bad[b] != 0;
  float top = -kInf, total = 0.0f;
  float4 x[kMine];
#pragma unroll
  for (int k = 0; k < kMine; ++k) x[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  bool whole = false;
  if (shape.x > 0 && static_cast<int>(block) < shape.w && !bad) {
    const Runs runs(all, p.ctas);
    const int64_t first = before + (static_cast<int64_t>(g) * shape.w + block) * shape.x;
    int64_t from = runs.cta(first);
    const int64_t last = runs.cta(first + shape.x - 1);
    const auto end_of = [&](int64_t i) { return min(runs.first(i + 1) - first, static_cast<int64_t>(shape.x)); };
    const bool split = from < last && runs.first(from) < first;  // the first CTA's is not its first piece
    const int64_t from_first = from;
    while (from < last && steps_before(end_of(from), shape.z) == 0) ++from;  // CTAs with units of the block but no step
    whole = from == last;
    if (!whole) {
      const auto place = [&](int64_t i) { return 2 * i + (split && i == from_first); };
      constexpr int kAtOnce = 2;
      for (int64_t i0 = from; i0 <= last; i0 += kAtOnce) {
        float2 part[kAtOnce];
        float4 y[kAtOnce][kMine];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const int64_t at = place(min(i0 + k, last));
          part[k] = p.stats[at * p.block + in_block];
          const float4* outs = p.outs + (at * (D / 4) + warp) * p.block + in_block;
#pragma unroll
          for (int m = 0; m < kMine; ++m) y[k][m] = outs[m * kWarps * p.block];
          if (i0 + k > last) part[k] = make_float2(-kInf, 0.0f);
        }
        float most = top;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) most = fmaxf(most, part[k].x);
        const float back = top == -kInf ? 0.0f : exp2_approx(top - most);
        top = most;
        total *= back;  // (a NaN stays one)
#pragma unroll
        for (int m = 0; m < kMine; ++m) x[m].x *= back, x[m].y *= back, x[m].z *= back, x[m].w *= back;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const float scale = part[k].x == -kInf ? 0.0f : exp2_approx(part[k].x - top);
          total += part[k].y != part[k].y ? part[k].y : part[k].y * scale;
          if (part[k].x > -kInf) {
#pragma unroll
            for (int m = 0; m < kMine; ++m) {
              x[m].x = fmaf(y[k][m].x, scale, x[m].x), x[m].y = fmaf(y[k][m].y, scale, x[m].y);
              x[m].z = fmaf(y[k][m].z, scale, x[m].z), x[m].w = fmaf(y[k][m].w, scale, x[m].w);
            }
          }
        }
      }
    }
  }
  if (!sees) total = 0.0f;
  const float over = sees && bad ? NAN : total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const float f[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
    uint2 two;
    two.x = narrow2<T>(over == 0.0f ? 0.0f : f[0] * over, over == 0.0f ? 0.0f : f[1] * over);
    two.y = narrow2<T>(over == 0.0f ? 0.0f : f[2] * over, over == 0.0f ? 0.0f : f[3] * over);
    *reinterpret_cast<uint2*>(tile + lane * kPitch + (warp + k * kWarps) * 4) = two;
  }
  if (warp == 0) {
    const bool writes = in && !(whole && sees);  // a whole block's rows are written
    to_row[lane] = writes ? b * p.out_token + node * p.out_node + head * p.out_head : -1;
    if (writes && p.lse != nullptr)
      p.lse[(static_cast<int64_t>(b) * p.drafts + node) * p.heads + head] =
          sees && bad ? NAN : total == 0.0f ? -kInf : (top + log2f(total)) * kLn2;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * (D / 8); i += 256) {
    const int row = i / (D / 8), d = i % (D / 8) * 8;
    if (to_row[row] < 0 || d >= p.dim) continue;
    T* to = static_cast<T*>(p.out) + to_row[row] + d;
    const T* from = tile + row * kPitch + d;
    if (reinterpret_cast<uintptr_t>(to) % 16 == 0) {
      *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) to[e] = from[e];
    }
  }
}

template <typename F, typename... A>
cudaError_t launch_behind(F kernel, int64_t grid, int threads, int bytes, cudaStream_t stream, const A&... a) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(static_cast<unsigned>(grid));
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = bytes;
  c.stream = stream;
  c.attrs = &attr;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, a...);
}

template <typename T, int D, int kSlots, int kCopies, bool kPlain>
cudaError_t launch_kind(WideParams p, cudaStream_t stream) {
  using L = Plan<D, kSlots>;
  const auto kernel = draft_wide_kernel<T, D, kSlots, kCopies, kPlain>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes);
  if (e != cudaSuccess) return e;
  // pages that hold whole steps, or of which a step holds whole ones, by 8 rows (the swizzle's) at least
  CUtensorMap k_map = {}, v_map = {};
  constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
  const bool fits = p.page_size % kKeys == 0 || (p.page_size >= 8 && kKeys % p.page_size == 0);
  const int rows = std::min(p.page_size, kKeys);
  if (fits && make_page_map(&k_map, kBf16, p.k, p.dim, p.kv_heads, p.page_size, p.n_pages, p.k_head, p.k_token, p.k_page, rows) &&
      make_page_map(&v_map, kBf16, p.v, p.dim, p.kv_heads, p.page_size, p.n_pages, p.v_head, p.v_token, p.v_page, rows))
    p.rows_at_once = rows;
  draft_wide_plan_kernel<<<1, 1024, 0, stream>>>(p);
  e = cudaGetLastError();
  if (e == cudaSuccess) e = launch_behind(kernel, p.ctas, L::kThreads, L::kBytes, stream, p, k_map, v_map);
  const int64_t blocks = (static_cast<int64_t>(p.drafts) * p.group + p.block - 1) / p.block;
  const int64_t chunks = p.batch * p.kv_heads * blocks * (p.block / 32);
  return e != cudaSuccess ? e : launch_behind(draft_wide_join_kernel<T, D>, chunks, 256, 0, stream, p);
}

template <typename T, int D, int kSlots, int kCopies>
cudaError_t launch_rows(const WideParams& p, cudaStream_t stream) {
  return p.softcap > 0.0f || p.slopes != nullptr ? launch_kind<T, D, kSlots, kCopies, false>(p, stream)
                                                 : launch_kind<T, D, kSlots, kCopies, true>(p, stream);
}

template <typename T, int D>
cudaError_t launch_size(const WideParams& p, cudaStream_t stream) {
  const int64_t rows = static_cast<int64_t>(p.drafts) * p.group;
  if (rows > kRows) return launch_rows<T, D, 2, 1>(p, stream);
  if (rows > 64) return launch_rows<T, D, 1, 1>(p, stream);
  return rows > 32 ? launch_rows<T, D, 1, 2>(p, stream) : launch_rows<T, D, 1, 4>(p, stream);
}

template <typename T>
cudaError_t launch_head(const WideParams& p, cudaStream_t stream) {
  return p.dim <= 64 ? launch_size<T, 64>(p, stream) : launch_size<T, 128>(p, stream);
}

// What can be taken here, if strides, alignment and scale admit it: more than 16 rows, 16-bit types.
bool wide(int64_t rows, int dim, int dtype) { return dtype != 0 && dim <= 128 && rows > 16; }

// Whether it is: three launches and the pieces' way through memory take 27 us at least, where draft_mma_kernel begins at 13 but
// reads every key once per 32 rows. By the most keys that the page table holds, times blocks of 32 rows and the head size, 20e6
// (32 / 8 heads of 128; rows, sequences of up to so many keys, this kernel / that one, us: 32, 8 x 1000, 33 / 23; 32, 8 x 4000,
// 40 / 45; 96, 8 x 1000, 33 / 36; 256, 1 x 1000, 31 / 25; 256, 1 x 8000, 36 / 85; 256, 8 x 4000, 48 / 149).
bool worth(const DraftParams& p, int64_t batch, int64_t rows) {
  return static_cast<double>(batch) * p.kv_heads * p.max_pages * p.page_size * ((rows + 31) / 32) * (p.dim <= 64 ? 64 : 128) > 20e6;
}

constexpr int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

}  // namespace

int64_t draft_wide_work(int64_t batch, int64_t rows, int dim, int dtype) {
  if (!wide(rows, dim, dtype)) return 0;
  const int64_t places = static_cast<int64_t>(2 * kMaxCtas) * kRows;  // two slots: half as many CTAs, twice the rows
  return up16(8 * (batch + 1)) + 16 * batch + up16(4 * batch) + places * (8 + 4 * (dim <= 64 ? 64 : 128));
}

bool launch_draft_wide(const DraftParams& p, int64_t batch, int dtype, int sms, void* work, cudaStream_t stream, cudaError_t* e) {
  // The scores' maximum is taken before the scale, and -inf times it has to stay -inf: it is positive
  const int64_t rows = static_cast<int64_t>(p.drafts) * p.group;
  if (!wide(rows, p.dim, dtype) || !worth(p, batch, rows) || !paged_vectors(p) || !(p.scale > 0.0f)) return false;
  WideParams q = {};
  static_cast<DraftParams&>(q) = p;
  q.batch = batch;
  q.block = rows > kRows ? 2 * kRows : kRows;
  q.ctas = std::min(sms * (rows > kRows ? 1 : 2), kMaxCtas / (rows > kRows ? 2 : 1));
  char* at = static_cast<char*>(work);
  q.prefix = reinterpret_cast<int64_t*>(at), at += up16(8 * (batch + 1));
  q.shape = reinterpret_cast<int4*>(at), at += 16 * batch;
  q.bad = reinterpret_cast<int32_t*>(at), at += up16(4 * batch);
  q.stats = reinterpret_cast<float2*>(at), at += static_cast<int64_t>(2 * kMaxCtas) * kRows * 8;
  q.outs = reinterpret_cast<float4*>(at);
  *e = dtype == 1 ? launch_head<__nv_bfloat16>(q, stream) : launch_head<__half>(q, stream);
  return true;
}

}  // namespace zo
