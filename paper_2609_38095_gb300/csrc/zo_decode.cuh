// zo_decode.cuh -- what the kernels of one-token attention share: how a
// cluster's CTAs and their warps split a sequence, and how they join.
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

// Every thread of the cluster. outs: [kWarps][HB][DP] unscaled outputs, tops and
// totals: [kWarps][HB], all in shared memory; tops in units of log2 (kLog2), or
// of the scores.
template <typename T, int HB, int DP, int kWarps, bool kLog2>
__device__ __forceinline__ void decode_join(const DecodeParams& p, const DecodePlace& w, float* outs, const float* tops,
                                            const float* totals, DecodeJoin<HB>& join) {
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
      join.over[h] = bad ? NAN : total == 0.0f ? 0.0f : 1.0f / total;
      join.lse[h] = bad ? NAN : total == 0.0f ? -kInf : kLog2 ? (top + log2f(total)) * kLn2 : top + logf(total);
    }
  }
  __syncthreads();
  T* out = static_cast<T*>(p.out) + w.b * p.out_token;
  for (int i = rank * (kWarps * 32) + tid; i < w.heads * DP; i += ranks * (kWarps * 32)) {
    const int h = i / DP, d = i - h * DP;
    float x = 0.0f;
#pragma unroll 4
    for (uint32_t r = 0; r < ranks; ++r) x = fmaf(peer_load(peer_address(outs + i, r)), join.scale[r][h], x);
    const int head = w.head0 + h;
    const float over = join.over[h];
    if (d < p.dim) out[head * p.out_head + d] = narrow<T>(over == 0.0f ? 0.0f : x * over);
    if (d == 0 && p.lse != nullptr) p.lse[static_cast<int64_t>(w.b) * p.heads + head] = join.lse[h];
  }
  cluster_sync();  // no CTA leaves before its part is read
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

template <typename K>
cudaError_t launch_decode(K kernel, const DecodeParams& p, int64_t items, int cluster, int threads, int bytes,
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
