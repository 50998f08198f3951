// hs_draft_tree: the M - 1 best of the D x K nodes that a query's steps have grown, as a breadth-first
// tree with parents, ancestor bits and kept children. One wave per query: lane j is slot j of a step,
// then node j of the tree.
//   1. ranks e = min(score, e of the parent), step after step through LDS, as keys (e, then the lower
//      step and slot), which are distinct;
//   2. the (M - 1)-th largest key by a bitwise search; kept nodes numbered in step and slot order by
//      ballots;
//   3. lane n is node n: its parent's number from LDS, its path by D rounds over the depths, its place
//      among its siblings by counting the earlier nodes with its parent.
// Bound by latency (a few KB per query): D dependent LDS rounds, the search, then the stores.
#include "hs_beam.h"

namespace hs {

namespace {

constexpr int kNodes = HS_MAX_DEPTH * HS_MAX_BEAMS;

__global__ __launch_bounds__(64) void hs_tree_kernel(hs_tree_args A) {
  __shared__ uint64_t s_key[kNodes];          // 0: no node
  __shared__ uint8_t s_num[kNodes];           // a kept node's number
  __shared__ int16_t s_grown[HS_MAX_POSITIONS];  // step * K + slot of every kept node
  __shared__ int32_t s_cand[HS_MAX_POSITIONS * HS_MAX_BEAMS];
  const int lane = threadIdx.x, b = blockIdx.x;
  const int D = A.D, K = A.K, M = A.M, N = D * K;
  const int64_t step = (int64_t)A.B * K, at = (int64_t)b * K;

  for (int d = 0; d < D; ++d) {
    if (lane < K) {
      const float v = A.score[d * step + at + lane];
      const int p = A.parent[d * step + at + lane];
      uint64_t k = 0;
      if (p >= 0 && isfinite(v)) {
        uint32_t e = ordered_of(v);
        if (d > 0) {
          const uint32_t up = p < K ? (uint32_t)(s_key[(d - 1) * K + p] >> 32) : 0;
          e = min(e, up);  // 0 where the parent is empty
        }
        if (e != 0) k = ((uint64_t)e << 32) | (0xFFFFFFFFu - (uint32_t)(d * K + lane));
      }
      s_key[d * K + lane] = k;
    }
    lds_wave_fence();
  }

  uint64_t u[kNodes / 64];
  const int nu = (N + 63) / 64;
#pragma unroll
  for (int j = 0; j < kNodes / 64; ++j) u[j] = j * 64 + lane < N ? s_key[j * 64 + lane] : 0;
  const uint64_t x = nth_largest(u, nu, M - 1);
  int n = 1;
#pragma unroll
  for (int j = 0; j < kNodes / 64; ++j) {
    const bool keep = u[j] != 0 && u[j] >= x;
    const uint64_t m = __ballot(keep);
    if (keep) {
      const int num = n + lanes_below(m);
      s_num[j * 64 + lane] = (uint8_t)num;
      s_grown[num] = (int16_t)(j * 64 + lane);
    }
    n += __builtin_popcountll(m);
  }
  for (int i = lane; i < M * K; i += 64) s_cand[i] = -1;
  lds_wave_fence();

  // lane = node
  int token = -1, parent = -1, depth = -1, slot = -1;
  float score = -INFINITY;
  uint64_t mask = 0;
  if (lane == 0) {
    depth = 0;
    score = 0.0f;
    mask = 1;
  } else if (lane < n) {
    const int g = s_grown[lane], d = g / K;
    slot = g - d * K;
    depth = d + 1;
    const int64_t i = d * step + at + slot;
    token = A.token[i];
    score = A.score[i];
    parent = d == 0 ? 0 : s_num[(d - 1) * K + A.parent[i]];
  }
  for (int d = 1; d <= D; ++d) {
    const uint64_t up = __shfl(mask, parent < 0 ? 0 : parent, 64);
    if (depth == d) mask = up | (1ull << lane);
  }
  int place = 0;
  for (int i = 1; i < n; ++i) {
    const int p = __builtin_amdgcn_readlane(parent, i);
    if (i < lane && p == parent) ++place;
  }
  if (lane > 0 && lane < n) s_cand[parent * K + place] = token;
  lds_wave_fence();

  const int64_t o = (int64_t)b * M;
  if (lane < M) {
    if (A.node_token) A.node_token[o + lane] = token;
    if (A.node_parent) A.node_parent[o + lane] = parent;
    if (A.node_depth) A.node_depth[o + lane] = depth;
    if (A.node_slot) A.node_slot[o + lane] = slot;
    if (A.node_score) A.node_score[o + lane] = score;
    if (A.node_mask) A.node_mask[o + lane] = mask;
  }
  if (A.cand)
    for (int i = lane; i < M * K; i += 64) A.cand[o * K + i] = s_cand[i];
  if (A.count && lane == 0) A.count[b] = n;
}

}  // namespace

int launch_draft_tree(const hs_tree_args& a, hipStream_t stream) {
  hs_tree_kernel<<<a.B, 64, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? HS_OK : HS_ERR_HIP;
}

}  // namespace hs
