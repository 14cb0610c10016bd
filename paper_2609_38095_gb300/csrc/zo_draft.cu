// zo_draft.cu -- masks of trees of drafted tokens (zo_draft_masks), and their
// attention over a paged cache on the tensor cores: 16-bit types, vectors
// aligned to 16 bytes (zo_attention_draft).
#include "zo_decode.cuh"

namespace zo {

namespace {

constexpr int kWarps = 4;

// A warp per sequence; a lane walks up from two of its nodes.
__global__ void draft_masks_kernel(const int32_t* parents, int64_t batch, int drafts, int64_t* masks) {
  const int64_t b = static_cast<int64_t>(blockIdx.x) * (blockDim.x / 32) + (threadIdx.x >> 5);
  if (b >= batch) return;
  const int32_t* up = parents + b * drafts;
  for (int i = threadIdx.x & 31; i < drafts; i += 32) {
    uint64_t m = 0;
    int at = i;
    while (at >= 0) {
      m |= UINT64_C(1) << at;
      const int next = up[at];
      at = next >= -1 && next < at ? next : -2;
    }
    masks[b * drafts + i] = at == -1 ? static_cast<int64_t>(m) : 0;
  }
}

template <int DP, int MB>
struct Tiles {
  static constexpr int kRows = 16 * MB;
  static constexpr int kBlocksOfKeys = DP == 64 ? 2 : 1;  // of 16, in a tile
  static constexpr int kKeys = 16 * kBlocksOfKeys;
  static constexpr int kStages = 2;
  static constexpr int kRow = DP * 2;                  // bytes of a key
  static constexpr int kStage = 2 * kKeys * kRow;      // keys, then values
  static constexpr int kWarp = kStages * kStage;
  static constexpr int kBytes = kWarps * kWarp;
  static_assert(kRows * DP * 4 <= kWarp, "a warp's output takes its tiles' place");
};

// Two 16-bit values of which one is infinite or NaN.
template <typename T>
__device__ __forceinline__ bool not_finite2(uint32_t v) {
  constexpr uint32_t kExponent = __is_same(T, __nv_bfloat16) ? 0x7F80u : 0x7C00u;
  return (v & kExponent) == kExponent || (v >> 16 & kExponent) == kExponent;
}

// A cluster takes 16 MB rows of a sequence and key-value head: a node's query
// heads that share it, node by node. As in one-token attention a warp has its own
// tiles of 16 or 32 keys, by cp.async into its own shared memory, and shares
// nothing until its last; but the rows are the products' rows, S = Q K^T and
// O += P V, so that a step's scores are the next product's left operand as they
// are. What a row sees of the tree's own keys is a bit of its node's mask. For few
// rows or short sequences, and heads beyond 128: bound by latency, the chain
// length and masks -> pages -> keys -> products -> joins and the code's own way into
// the instruction caches (one sequence of 2039 keys, 8 nodes, 32 / 8 heads of 128,
// bf16: 16.4 us a call, where its bytes take 1.3). Every 32
// rows read the keys again: zo_draft_wide.cu takes over where that costs more.
template <typename T, int DP, int MB, bool kPlain>
__global__ void __launch_bounds__(kWarps * 32, DP > 128 ? 1 : MB == 1 || DP == 64 ? 3 : 2)
    draft_mma_kernel(const __grid_constant__ DraftParams p) {
  using L = Tiles<DP, MB>;
  constexpr int kVectors = DP / 8, kDeep = L::kBlocksOfKeys, kRows = L::kRows;  // a key's 16-byte vectors
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ DraftShared<kRows> sh;
  __shared__ float tops[kWarps][kRows], totals[kWarps][kRows];  // then the first the warps' scales
  __shared__ float top[kRows], sum[kRows];
  __shared__ int bad_here;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t tiles = static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + warp * L::kWarp;
  const uint32_t ranks = cluster_size();
  if (threadIdx.x == 0) bad_here = 0;
  const DraftPlace w = draft_place<kRows>(p, blockIdx.x / ranks, sh);
  const DraftRows<T, kRows> rows = {p, w, sh};

  const T* kc = static_cast<const T*>(p.k) + w.g * p.k_head;
  const T* vc = static_cast<const T*>(p.v) + w.g * p.v_head;
  const int64_t tiles_in = (w.len + L::kKeys - 1) / L::kKeys;
  const int64_t step = static_cast<int64_t>(ranks) * kWarps;
  const int64_t first = static_cast<int64_t>(cluster_rank()) * kWarps + warp;
  int bad = 0;
  // A lane looks up the page of one of a tile's keys a whole tile before it needs it, as in one-token attention.
  const bool same = p.k_page == p.v_page && p.k_token == p.v_token;
  struct Place {
    int64_t k, v;
  };
  // With a bias by distance the tiles in turn from the last to the first: a row's largest scores come first then, and its output
  // is not rescaled at every tile.
  const bool cap = !kPlain && p.softcap > 0.0f, bias = !kPlain && p.slopes != nullptr, backward = bias;
  const auto key_of = [&](int64_t tile) { return (backward ? tiles_in - 1 - tile : tile) * L::kKeys; };
  const auto look = [&](int64_t tile) {
    const int64_t j = key_of(tile) + lane % L::kKeys;
    return j >= 0 && draft_sees(w, j) ? p.pages[w.b * p.pages_stride + decode_page(p, j)] : 0;
  };
  const auto find = [&](int64_t tile, int id) {
    const int64_t j = key_of(tile) + lane % L::kKeys;
    const int2 key = decode_key(p, w, draft_sees(w, j) ? j : w.len, id, bad);
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
    constexpr int kRowsAtOnce = 32 / kVectors;
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
  // the queries as left operands: rows lane / 4 and 8 more of each block of 16, elements 2 (lane mod 4) and 8 more
  const bool pairs = aligned_to(p.q, 4) && (p.q_token | p.q_node | p.q_head) % 2 == 0;
  uint32_t qa[MB][DP / 16][4];
  float slope2[MB][2], depth[MB][2];  // depth: a row's place from the tree's first
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int h = 16 * m + 8 * r + lane / 4;
      const T* q = rows.query(h);
      slope2[m][r] = bias ? p.slopes[rows.head(h)] * kLog2e : 0.0f;
      depth[m][r] = static_cast<float>(__popcll(rows.mask(h)) - 1);
#pragma unroll
      for (int s = 0; s < DP / 16; ++s)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int d = s * 16 + c * 8 + lane % 4 * 2;
          qa[m][s][r + 2 * c] = 0;
          if (d < p.dim) {
            if (pairs) {
              qa[m][s][r + 2 * c] = *reinterpret_cast<const uint32_t*>(q + d);
            } else {
              const uint16_t* x = reinterpret_cast<const uint16_t*>(q + d);
              qa[m][s][r + 2 * c] = x[0] | static_cast<uint32_t>(x[1]) << 16;
            }
          }
        }
    }
  const float scale2 = cap ? p.scale / p.softcap : p.scale * kLog2e, cap2 = p.softcap * kLog2e;
  float base[MB][2], total[MB][2], acc[MB][DP / 8][4];
#pragma unroll
  for (int m = 0; m < MB; ++m) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      base[m][r] = -kInf;
      total[m][r] = 0.0f;
    }
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[m][n][c] = 0.0f;
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
    // scores: keys 2 (lane mod 4) and the next of each block of 8
    float s[MB][2 * kDeep][4] = {};
#pragma unroll
    for (int b = 0; b < kDeep; ++b) {
      const int row = b * 16 + (lane & 7) + (lane >> 4) * 8;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        uint32_t k[4];
        load4(k, ks + row * L::kRow + (((2 * d + (lane >> 3 & 1)) ^ (row & 7)) << 4));
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          mma16816<T>(s[m][2 * b], qa[m][d], k[0], k[1]);
          mma16816<T>(s[m][2 * b + 1], qa[m][d], k[2], k[3]);
        }
      }
    }
    const int64_t key0 = key_of(tile);
    const bool nodes = key0 + L::kKeys > w.n;  // keys of the tree, or beyond the last
    float times = scale2;  // what the scores are in, times
    if (cap) {
      times = 1.0f;
      float far = 0.0f;
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < 2 * kDeep; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) far = fmaxf(far, fabsf(s[m][n][c]));
      const bool near = __all_sync(0xFFFFFFFFu, far * fabsf(scale2) < kNearCap);  // mostly: caps are there for the rare large score
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < 2 * kDeep; ++n)
#pragma unroll
          for (int c = 0; c < 4; c += 2) {
            float* const y = &s[m][n][c];
            if (__builtin_expect(near, 1)) {
              const uint64_t two = capped_near(pack2(y[0], y[1]), pack2(scale2, scale2), pack2(cap2, cap2));
              y[0] = low2(two), y[1] = high2(two);
            } else {
              y[0] = capped(y[0], scale2, cap2), y[1] = capped(y[1], scale2, cap2);
            }
          }
    } else if (bias || nodes || p.scale <= 0.0f) {
      times = 1.0f;
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < 2 * kDeep; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[m][n][c] *= scale2;
    }
    if (__builtin_expect(nodes, 0)) {
      const int from = static_cast<int>(key0 - w.n) + lane % 4 * 2;  // the thread's first key, from the tree's first
#pragma unroll
      for (int n = 0; n < 2 * kDeep; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int node = from + n * 8 + c;
          const bool tree = node >= 0 && node < 64;
          const float place = static_cast<float>(node < 0 ? node : tree ? __popcll(sh.masks[node]) - 1 : 0);
#pragma unroll
          for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              float& y = s[m][n][2 * r + c];
              if (bias) y -= slope2[m][r] * fabsf(depth[m][r] - place);
              if (node >= 0 && !(tree && (rows.mask(16 * m + 8 * r + lane / 4) >> node & 1))) y = -kInf;
            }
        }
    } else if (bias) {
      const float from = static_cast<float>(static_cast<int>(w.n - key0) - lane % 4 * 2);  // exact, and its sums, below 2^24
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float away = depth[m][r] + from;
#pragma unroll
          for (int n = 0; n < 2 * kDeep; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c)
              s[m][n][2 * r + c] = fmaf(-slope2[m][r], away - static_cast<float>(n * 8 + c), s[m][n][2 * r + c]);
        }
    }
    bool moved = false;
    float back[MB][2];
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float most = fmaxf(s[m][0][2 * r], s[m][0][2 * r + 1]);
#pragma unroll
        for (int n = 1; n < 2 * kDeep; ++n) most = fmaxf(fmaxf(most, s[m][n][2 * r]), s[m][n][2 * r + 1]);
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
        most = most * times - kLift<T>;
        back[m][r] = 1.0f;
        if (most > base[m][r] + kSlack || (base[m][r] == -kInf && most > -kInf)) {
          back[m][r] = exp2_approx(base[m][r] - most);
          base[m][r] = most;
          moved = true;
        }
        const float shift = base[m][r] == -kInf ? 0.0f : -base[m][r];
        uint64_t sums = 0;
#pragma unroll
        for (int n = 0; n < 2 * kDeep; ++n) {
          const uint64_t t = fma2(pack2(s[m][n][2 * r], s[m][n][2 * r + 1]), pack2(times, times), pack2(shift, shift));
          const uint64_t e = pack2(exp2_approx(low2(t)), exp2_approx(high2(t)));
          s[m][n][2 * r] = low2(e), s[m][n][2 * r + 1] = high2(e);
          sums = add2(sums, e);
        }
        total[m][r] = fmaf(total[m][r], back[m][r], low2(sums) + high2(sums));
      }
    if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[m][n][c] *= back[m][c >> 1];
    }
    if (__builtin_expect(nodes, 0)) {
      // Values of the tree's keys that are not finite: a row that sees one has NaN in its column, for the others (whose
      // weight is 0, and 0 times it is NaN) it is taken out.
      uint4* const v = reinterpret_cast<uint4*>(smem + warp * L::kWarp + stage * L::kStage + L::kKeys * L::kRow);
      bool odd = false;
      for (int i = lane; i < L::kKeys * kVectors; i += 32) {
        const uint4 u = v[i];
        odd = odd || not_finite2<T>(u.x) || not_finite2<T>(u.y) || not_finite2<T>(u.z) || not_finite2<T>(u.w);
      }
      if (__any_sync(0xFFFFFFFFu, odd)) {
        const uint16_t* const one = reinterpret_cast<const uint16_t*>(v);
        for (int k = 0; k < L::kKeys; ++k) {
          const int64_t node = key0 + k - w.n;
          if (node < 0 || node >= 64) continue;
#pragma unroll
          for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int h = 16 * m + 8 * r + lane / 4;
              if (!(rows.mask(h) >> node & 1)) continue;
#pragma unroll
              for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                  if (not_finite2<T>(one[k * DP + ((n ^ (k & 7)) << 3) + lane % 4 * 2 + c])) acc[m][n][2 * r + c] = NAN;
            }
        }
        __syncwarp();
        for (int i = lane; i < L::kKeys * kVectors; i += 32) {
          if (key0 + i / kVectors < w.n) continue;
          uint4 u = v[i];
          const auto clean = [](uint32_t x) {
            return (not_finite2<T>(x & 0xFFFFu) ? 0u : x & 0xFFFFu) | (not_finite2<T>(x >> 16) ? 0u : x & 0xFFFF0000u);
          };
          v[i] = make_uint4(clean(u.x), clean(u.y), clean(u.z), clean(u.w));
        }
        __syncwarp();
      }
    }
#pragma unroll
    for (int b = 0; b < kDeep; ++b) {
      const int row = b * 16 + (lane & 15);
      uint32_t weight[MB][4];  // rounded to 16 bits for the tensor cores: off by half a step of each, their sum is of the fp32 ones
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int r = 0; r < 2; ++r)
            weight[m][2 * n + r] = narrow2<T>(s[m][2 * b + n][2 * r], s[m][2 * b + n][2 * r + 1]);
#pragma unroll
      for (int n = 0; n < DP / 16; ++n) {
        uint32_t x[4];
        load4_transposed(x, vs + row * L::kRow + (((2 * n + (lane >> 4)) ^ (row & 7)) << 4));
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          mma16816<T>(acc[m][2 * n], weight[m], x[0], x[1]);
          mma16816<T>(acc[m][2 * n + 1], weight[m], x[2], x[3]);
        }
      }
    }
    __syncwarp();  // the stage may be filled again
    stage = stage + 1 == L::kStages ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float all = total[m][r];
      all += __shfl_xor_sync(0xFFFFFFFFu, all, 1);
      all += __shfl_xor_sync(0xFFFFFFFFu, all, 2);
      if (lane % 4 == 0) {
        tops[warp][16 * m + 8 * r + lane / 4] = base[m][r];
        totals[warp][16 * m + 8 * r + lane / 4] = all;
      }
    }
  if (bad || w.bad) bad_here = 1;
  __syncthreads();  // every warp is done with its tiles: the outputs take their place
  float* outs = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
      for (int r = 0; r < 2; ++r)
        *reinterpret_cast<float2*>(outs + (warp * kRows + 16 * m + 8 * r + lane / 4) * DP + n * 8 + lane % 4 * 2) =
            make_float2(acc[m][n][2 * r], acc[m][n][2 * r + 1]);
  if (threadIdx.x < kRows) {  // the warps' scales
    const int h = threadIdx.x;
    float most = -kInf, all = 0.0f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) most = fmaxf(most, tops[i][h]);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const float scale = tops[i][h] == -kInf ? 0.0f : exp2_approx(tops[i][h] - most);
      all += totals[i][h] != totals[i][h] ? totals[i][h] : totals[i][h] * scale;
      tops[i][h] = scale;
    }
    top[h] = most, sum[h] = all;
  }
  __syncthreads();
  for (int i = threadIdx.x * 4; i < w.live * DP; i += kWarps * 32 * 4) {
    const int h = i / DP;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int n = 0; n < kWarps; ++n) {
      const float scale = tops[n][h];
      const float4 y = *reinterpret_cast<const float4*>(outs + n * kRows * DP + i);
      x.x = fmaf(y.x, scale, x.x), x.y = fmaf(y.y, scale, x.y), x.z = fmaf(y.z, scale, x.z), x.w = fmaf(y.w, scale, x.w);
    }
    *reinterpret_cast<float4*>(outs + i) = x;
  }
  rows_join<T, DP, DP, kWarps * 32>(p, w, rows, outs, top, sum, &bad_here);
}

template <typename T, int DP, int MB, bool kPlain>
cudaError_t launch_kind(DraftParams p, int64_t batch, int sms, cudaStream_t stream) {
  using L = Tiles<DP, MB>;
  p.head_blocks = (p.drafts * p.group + L::kRows - 1) / L::kRows;
  const int64_t items = batch * p.kv_heads * p.head_blocks;
  const int c = decode_cluster(items, p.max_pages * p.page_size, sms, MB == 1 ? 6 : 4);
  return launch_decode(draft_mma_kernel<T, DP, MB, kPlain>, p, items, c, kWarps * 32, L::kBytes, stream);
}

// Without caps and biases in a kernel of its own: less code to come to the SMs (one sequence of 2000
// keys, 8 nodes, 32 / 8 heads of 128: 20.0 -> 19.0 us with cold caches; 8 of up to 1000, 32 heads: 34.4 -> 32.3).
template <typename T, int DP, int MB>
cudaError_t launch_size(const DraftParams& p, int64_t batch, int sms, cudaStream_t stream) {
  return p.softcap > 0.0f || p.slopes != nullptr ? launch_kind<T, DP, MB, false>(p, batch, sms, stream)
                                                 : launch_kind<T, DP, MB, true>(p, batch, sms, stream);
}

template <typename T>
cudaError_t launch_type(const DraftParams& p, int64_t batch, int sms, cudaStream_t stream) {
  const bool few = p.drafts * p.group <= 16;
  if (p.dim <= 64) return few ? launch_size<T, 64, 1>(p, batch, sms, stream) : launch_size<T, 64, 2>(p, batch, sms, stream);
  if (p.dim <= 128) return few ? launch_size<T, 128, 1>(p, batch, sms, stream) : launch_size<T, 128, 2>(p, batch, sms, stream);
  return launch_size<T, 256, 1>(p, batch, sms, stream);
}

}  // namespace

cudaError_t launch_draft_masks(const int32_t* parents, int64_t batch, int drafts, int64_t* masks, cudaStream_t stream) {
  draft_masks_kernel<<<static_cast<unsigned>((batch + 7) / 8), 256, 0, stream>>>(parents, batch, drafts, masks);
  return cudaGetLastError();
}

bool launch_draft_mma(const DraftParams& p, int64_t batch, int dtype, int sms, cudaStream_t stream, cudaError_t* e) {
  if (dtype == 0 || !paged_vectors(p)) return false;
  *e = dtype == 1 ? launch_type<__nv_bfloat16>(p, batch, sms, stream) : launch_type<__half>(p, batch, sms, stream);
  return true;
}

}  // namespace zo
