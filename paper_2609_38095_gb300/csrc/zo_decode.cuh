// zo_decode.cuh -- what the kernels of attention over a paged cache share, of
// one token per sequence or a tree of them: how a cluster's CTAs and their warps
// split a sequence, and how they join.
//
// A cluster of CTAs takes one sequence and key-value head. The keys go in tiles
// of 16 or 32 to the cluster's warps in turn, so that warps differ by one tile at
// most; a warp keeps a running maximum, sum and output for each of its query
// heads and shares nothing with the others until its last key. Then a CTA joins
// its warps in shared memory and the cluster its CTAs over distributed shared
// memory, each CTA a part of the output: one launch, no workspace, and an order
// of additions that depends on the launch's shape alone.
#pragma once

#include "zo_forward.cuh"

namespace zo {

constexpr int kMaxCluster = 16;

template <int HB>
struct DecodeJoin {  // a CTA's statistics, read by its peers; and what it makes of theirs
  float top[HB], total[HB];
  int bad;
  float scale[kMaxCluster][HB], over[HB], lse[HB];
};

struct DecodePlace {
  int b, g, head0, heads;  // sequence, key-value head, first query head, query heads here
  int64_t len;
  int bad;  // a length beyond the page table, or no cache
};

template <int HB>
__device__ __forceinline__ DecodePlace decode_place(const DecodeParams& p, uint32_t cluster) {
  const int blocks = p.head_blocks;
  DecodePlace w;
  w.b = cluster / (p.kv_heads * blocks);
  const int rest = cluster - w.b * (p.kv_heads * blocks);
  w.g = rest / blocks;
  const int first = (rest - w.g * blocks) * HB;
  w.head0 = w.g * p.group + first;
  w.heads = min(HB, p.group - first);
  w.len = max(p.lengths[w.b], 0);
  // (keys, a last tile's end among them, are counted in 32 bits)
  w.bad = w.len > p.max_pages * p.page_size || (w.len > 0 && p.n_pages == 0) || w.len > 0x7FFFFFFF - 64;
  if (w.bad) w.len = 0;
  return w;
}

// The place of key j's page in a sequence's row of the page table.
__device__ __forceinline__ uint32_t decode_page(const DecodeParams& p, int64_t j) {
  const uint32_t at = static_cast<uint32_t>(j);
  return p.page_shift >= 0 ? at >> p.page_shift : at / static_cast<uint32_t>(p.page_size);
}

// Key j's row in its page `id`; page -1 where j is beyond the length, and where
// the table names no page of the cache (bad).
__device__ __forceinline__ int2 decode_key(const DecodeParams& p, const DecodePlace& w, int64_t j, int id, int& bad) {
  if (j >= w.len) return make_int2(-1, 0);
  if (id < 0 || id >= p.n_pages) {
    bad = 1;
    return make_int2(-1, 0);
  }
  return make_int2(id, static_cast<int>(static_cast<uint32_t>(j) - decode_page(p, j) * static_cast<uint32_t>(p.page_size)));
}

// Where a row of the cluster goes, a query head of the sequence's token: for decode_join.
template <typename T>
struct DecodeRows {
  T* out;
  float* lse;  // or NULL
  int64_t out_head;
  __device__ __forceinline__ DecodeRows(const DecodeParams& p, const DecodePlace& w)
      : out(static_cast<T*>(p.out) + w.b * p.out_token + w.head0 * p.out_head),
        lse(p.lse != nullptr ? p.lse + static_cast<int64_t>(w.b) * p.heads + w.head0 : nullptr),
        out_head(p.out_head) {}
  __device__ __forceinline__ bool sees(int) const { return true; }
  __device__ __forceinline__ T* row(int h) const { return out + h * out_head; }
  __device__ __forceinline__ float* sum(int h) const { return lse + h; }
};

struct DraftPlace : DecodePlace {  // heads: rows here, head0: the first
  int n;                           // keys ahead of the tree's
  int live;                        // rows here up to the last that sees anything
  uint64_t any;                    // nodes that are seen
};

template <int HB>
struct DraftShared {
  uint64_t masks[64];  // the nodes', without bits of no node; 0 in a sequence of negative length
  uint16_t node[HB], head[HB];  // of the rows here
};

// Which keys a tree has: `last` nodes up to the last that is seen, `nodes` up to the last that sees anything; and whether there
// are more than the page table or 32 bits hold, a last tile's end among them.
struct DraftKeys {
  uint64_t any;
  int64_t len;
  int nodes, bad;
};
__host__ __device__ __forceinline__ DraftKeys draft_reach(const DecodeParams& p, int n, uint64_t any, int last, int nodes) {
  DraftKeys k;
  k.any = any;
  k.nodes = nodes;
  k.len = last == 0 ? 0 : static_cast<int64_t>(n) + last;
  k.bad = k.len > p.max_pages * p.page_size || (k.len > 0 && p.n_pages == 0) || k.len > 0x7FFFFFFF - 64;
  return k;
}
// A warp with each lane's two masks of a sequence, 0 where there is no node.
__device__ __forceinline__ DraftKeys draft_keys(const DraftParams& p, int n, uint64_t a, uint64_t b) {
  const uint64_t both = a | b;
  const uint64_t any = static_cast<uint64_t>(__reduce_or_sync(0xFFFFFFFFu, static_cast<uint32_t>(both >> 32))) << 32 |
                       __reduce_or_sync(0xFFFFFFFFu, static_cast<uint32_t>(both));
  const uint32_t high = __ballot_sync(0xFFFFFFFFu, b != 0), low = __ballot_sync(0xFFFFFFFFu, a != 0);
  return draft_reach(p, n, any, 64 - __clzll(any), 64 - __clzll(static_cast<uint64_t>(high) << 32 | low));
}

// What a block of rows has of them. One behind the last row that sees anything, or of a sequence whose keys are more than
// the page table holds, has none: draft_sees() is what pages are looked up by, so that neither length is left.
__host__ __device__ __forceinline__ void draft_take(DraftPlace& w, const DecodeParams& p, const DraftKeys& k, int n) {
  const int live = k.nodes * p.group - w.head0;
  w.live = live < 0 ? 0 : live < w.heads ? live : w.heads;
  w.n = n;
  w.any = k.any;
  w.len = k.len;
  w.bad = k.bad;
  if (w.bad || w.live == 0) w.n = 0, w.len = 0, w.live = 0;
}

// Whether key j is one that the tree sees.
__host__ __device__ __forceinline__ bool draft_sees(const DraftPlace& w, int64_t j) {
  return j < w.n || (j < w.len && (w.any >> (j - w.n) & 1) != 0);
}

// Every thread of the CTA: sequence b, key-value head g and the block'th HB rows.
template <int HB>
__device__ __forceinline__ DraftPlace draft_place(const DraftParams& p, int b, int g, int block, DraftShared<HB>& sh) {
  const uint32_t lane = threadIdx.x & 31;
  DraftPlace w;
  w.b = b, w.g = g, w.head0 = block * HB;
  w.heads = min(HB, p.drafts * p.group - w.head0);
  const int n = p.lengths[w.b];
  if (threadIdx.x < 64) {
    uint64_t m = 0;  // (both loads on their way at once)
    if (threadIdx.x < p.drafts) m = p.masks[static_cast<int64_t>(w.b) * p.drafts + threadIdx.x] & (~UINT64_C(0) >> (64 - p.drafts));
    sh.masks[threadIdx.x] = n >= 0 ? m : 0;
  }
  for (uint32_t h = threadIdx.x; h < HB; h += blockDim.x) {
    const uint32_t r = w.head0 + min(h, static_cast<uint32_t>(w.heads) - 1), node = r / static_cast<uint32_t>(p.group);
    sh.node[h] = static_cast<uint16_t>(node);
    sh.head[h] = static_cast<uint16_t>(w.g * p.group + r - node * p.group);
  }
  __syncthreads();
  draft_take(w, p, draft_keys(p, max(n, 0), sh.masks[lane], sh.masks[lane + 32]), max(n, 0));
  return w;
}
template <int HB>
__device__ __forceinline__ DraftPlace draft_place(const DraftParams& p, uint32_t cluster, DraftShared<HB>& sh) {
  const uint32_t blocks = p.head_blocks, b = cluster / (p.kv_heads * blocks), rest = cluster - b * (p.kv_heads * blocks);
  const uint32_t g = rest / blocks;
  return draft_place<HB>(p, b, g, rest - g * blocks, sh);
}

// The tree's rows: see DecodeRows. (A row that is none is the last.)
template <typename T, int HB>
struct DraftRows {
  const DraftParams& p;
  const DraftPlace& w;
  const DraftShared<HB>& sh;
  __device__ __forceinline__ int node(int h) const { return sh.node[h]; }
  __device__ __forceinline__ int head(int h) const { return sh.head[h]; }
  __device__ __forceinline__ uint64_t mask(int h) const { return sh.masks[sh.node[h]]; }
  __device__ __forceinline__ bool sees(int h) const { return mask(h) != 0; }
  __device__ __forceinline__ T* row(int h) const {
    return static_cast<T*>(p.out) + w.b * p.out_token + node(h) * p.out_node + head(h) * p.out_head;
  }
  __device__ __forceinline__ float* sum(int h) const {
    return p.lse + (static_cast<int64_t>(w.b) * p.drafts + node(h)) * p.heads + head(h);
  }
  __device__ __forceinline__ const T* query(int h) const {
    return static_cast<const T*>(p.q) + w.b * p.q_token + node(h) * p.q_node + head(h) * p.q_head;
  }
};

// Every thread of the cluster. outs: [kWarps][HB][DP] unscaled outputs, tops and
// totals: [kWarps][HB], all in shared memory; tops in units of log2 (kLog2), or
// of the scores.
template <typename T, int HB, int DP, int kWarps, bool kLog2, typename R>
__device__ __forceinline__ void decode_join(const DecodeParams& p, const DecodePlace& w, const R& rows, float* outs,
                                            const float* tops, const float* totals, DecodeJoin<HB>& join) {
  const int tid = threadIdx.x;
  const auto less = [](float a, float b) { return exp2_approx(kLog2 ? a - b : (a - b) * kLog2e); };
  __syncthreads();
  if (tid < HB) {
    float top = -kInf, total = 0.0f;
    for (int i = 0; i < kWarps; ++i) top = fmaxf(top, tops[i * HB + tid]);
    for (int i = 0; i < kWarps; ++i)
      if (top > -kInf || totals[i * HB + tid] != 0.0f) total += totals[i * HB + tid] * less(tops[i * HB + tid], top);
    join.top[tid] = top;
    join.total[tid] = total;
  }
  for (int i = tid; i < w.heads * DP; i += kWarps * 32) {
    const int h = i / DP;
    float top = -kInf, x = 0.0f;
    for (int n = 0; n < kWarps; ++n) top = fmaxf(top, tops[n * HB + h]);
    if (top > -kInf)
      for (int n = 0; n < kWarps; ++n) x = fmaf(outs[n * HB * DP + i], less(tops[n * HB + h], top), x);
    outs[i] = x;
  }
  const uint32_t ranks = cluster_size(), rank = cluster_rank();
  cluster_sync();
  // a thread per head and CTA of the cluster: 16 lanes hold a head's CTAs (every lane of a warp takes part, with heads or
  // without)
  for (int first = 0; first < HB * kMaxCluster; first += kWarps * 32) {
    const int i = first + tid, h = min(i / kMaxCluster, HB - 1), r = i % kMaxCluster;
    const bool in = i < HB * kMaxCluster && r < static_cast<int>(ranks);
    const float mine = in ? peer_load(peer_address(&join.top[h], r)) : -kInf;
    const float part = in ? peer_load(peer_address(&join.total[h], r)) : 0.0f;
    bool bad = in && __float_as_int(peer_load(peer_address(&join.bad, r))) != 0;
    float top = mine;
#pragma unroll
    for (int o = kMaxCluster / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float scale = top == -kInf ? 0.0f : less(mine, top);
    float total = part * scale;
    if (part != part) total = part;  // a NaN where every score is one
#pragma unroll
    for (int o = kMaxCluster / 2; o > 0; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
    const uint32_t bads = __ballot_sync(0xFFFFFFFFu, bad);
    bad = (bads >> (tid & 16) & 0xFFFFu) != 0;
    if (i >= HB * kMaxCluster) continue;
    join.scale[r][h] = scale;
    if (r == 0) {
      if (h < w.heads && !rows.sees(h)) bad = false, total = 0.0f;
      join.over[h] = bad ? NAN : total == 0.0f ? 0.0f : 1.0f / total;
      join.lse[h] = bad ? NAN : total == 0.0f ? -kInf : kLog2 ? (top + log2f(total)) * kLn2 : top + logf(total);
    }
  }
  __syncthreads();
  for (int i = rank * (kWarps * 32) + tid; i < w.heads * DP; i += ranks * (kWarps * 32)) {
    const int h = i / DP, d = i - h * DP;
    float x = 0.0f;
#pragma unroll 4
    for (uint32_t r = 0; r < ranks; ++r) x = fmaf(peer_load(peer_address(outs + i, r)), join.scale[r][h], x);
    const float over = join.over[h];
    if (d < p.dim) rows.row(h)[d] = narrow<T>(over == 0.0f ? 0.0f : x * over);
    if (d == 0 && p.lse != nullptr) *rows.sum(h) = join.lse[h];
  }
  cluster_sync();  // no CTA leaves before its part is read
}

// Every thread of the cluster: the join of its CTAs alone, each with tops and totals of its HB rows (tops in units of log2) and
// unscaled outputs, kPitch floats from one row to the next, on 16 bytes. A warp has a row at a time: its lanes the CTAs'
// statistics, then four columns each. Returns when the peers are done with this CTA's part.
template <typename T, int DP, int kPitch, int kThreads, typename R>
__device__ __forceinline__ void rows_join(const DecodeParams& p, const DecodePlace& w, const R& rows, const float* outs,
                                          const float* tops, const float* totals, const int* bad_here) {
  constexpr int kLanes = DP / 4 < 32 ? DP / 4 : 32, kVectors = DP / 4 / kLanes;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ranks = static_cast<int>(cluster_size());
  cluster_sync();
  const bool peer = lane < ranks;
  const bool bad_any =
      __any_sync(0xFFFFFFFFu, peer && __float_as_int(peer_load(peer_address(bad_here, peer ? lane : 0))) != 0);
  for (int r = static_cast<int>(cluster_rank()) * (kThreads / 32) + warp; r < w.heads; r += ranks * (kThreads / 32)) {
    const float mine = peer ? peer_load(peer_address(tops + r, lane)) : -kInf;
    const float part = peer ? peer_load(peer_address(totals + r, lane)) : 0.0f;
    float top = mine;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float scale = mine == -kInf ? 0.0f : exp2_approx(mine - top);
    float total = part * scale;
    if (part != part) total = part;  // a NaN where every score is one
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
    top = __shfl_sync(0xFFFFFFFFu, top, 0);
    total = __shfl_sync(0xFFFFFFFFu, total, 0);
    const bool sees = rows.sees(r), bad = bad_any && sees;
    if (!sees) total = 0.0f;
    const uint32_t has = __ballot_sync(0xFFFFFFFFu, mine > -kInf);  // CTAs in which the row saw something
    float4 x[kVectors];
#pragma unroll
    for (int v = 0; v < kVectors; ++v) x[v] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (total != 0.0f && !bad) {
      constexpr int kBatch = kVectors == 1 ? 8 : 4;
      for (int first = 0; first < ranks; first += kBatch) {
        float4 y[kBatch][kVectors];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const bool in = first + i < ranks && (has >> (first + i) & 1) != 0 && lane < kLanes;
#pragma unroll
          for (int v = 0; v < kVectors; ++v) {
            y[i][v] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (in)
              asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                           : "=f"(y[i][v].x), "=f"(y[i][v].y), "=f"(y[i][v].z), "=f"(y[i][v].w)
                           : "r"(peer_address(outs + r * kPitch + v * 128 + lane * 4, first + i)));
          }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const float s = __shfl_sync(0xFFFFFFFFu, scale, (first + i) & 31);
#pragma unroll
          for (int v = 0; v < kVectors; ++v) {
            x[v].x = fmaf(y[i][v].x, s, x[v].x), x[v].y = fmaf(y[i][v].y, s, x[v].y);
            x[v].z = fmaf(y[i][v].z, s, x[v].z), x[v].w = fmaf(y[i][v].w, s, x[v].w);
          }
        }
      }
    }
    const float over = bad ? NAN : total == 0.0f ? 0.0f : 1.0f / total;
    const auto value = [&](float f) { return narrow<T>(over == 0.0f ? 0.0f : f * over); };
#pragma unroll
    for (int v = 0; v < kVectors; ++v) {
      const int d = v * 128 + lane * 4;
      T* to = rows.row(r) + d;
      if (d < p.dim) to[0] = value(x[v].x);
      if (d + 1 < p.dim) to[1] = value(x[v].y);
      if (d + 2 < p.dim) to[2] = value(x[v].z);
      if (d + 3 < p.dim) to[3] = value(x[v].w);
    }
    if (lane == 0 && p.lse != nullptr) *rows.sum(r) = bad ? NAN : total == 0.0f ? -kInf : (top + log2f(total)) * kLn2;
  }
  cluster_sync();
}

// Fragments of tiles of 16-bit values in shared memory, and their products.
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
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (__is_same(T, __nv_bfloat16))
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Whether every key's and value's elements are whole 16-byte vectors of a 16-bit type.
inline bool paged_vectors(const DecodeParams& p) {
  return p.dim % 8 == 0 && p.k_page % 8 == 0 && p.k_token % 8 == 0 && p.k_head % 8 == 0 && p.v_page % 8 == 0 &&
         p.v_token % 8 == 0 && p.v_head % 8 == 0 && aligned_to(p.k, 16) && aligned_to(p.v, 16);
}

// CTAs of a cluster: a CTA per SM, none with less than 128 keys of the longest
// sequence that the page table can hold; up to `per_sm` where each keeps 512,
// because a CTA's start and its part in the join cost as much as some 200 keys
// (128 sequences and heads of up to 4001 keys: 4 CTAs 33 us, 8 40 us).
inline int decode_cluster(int64_t items, int64_t longest, int sms, int per_sm) {
  int c = 1;
  while (c < kMaxCluster && ((items * c < sms && longest >= 2 * c * 128) ||
                             (items * c < static_cast<int64_t>(sms) * per_sm && longest >= 2 * c * 512)))
    c *= 2;
  return c;
}

template <typename K, typename P>
cudaError_t launch_decode(K kernel, const P& p, int64_t items, int cluster, int threads, int bytes,
                          cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && cluster > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(static_cast<unsigned>(items * cluster));
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = bytes;
  c.stream = stream;
  c.attrs = &attr;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, p);
}

}  // namespace zo
