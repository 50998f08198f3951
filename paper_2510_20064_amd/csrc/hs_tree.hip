// hs_draft_tree: the M - 1 best of the D x K nodes that a query's steps have grown, as a breadth-first
// tree with parents, ancestor bits and kept children. One workgroup of four waves per query:
//   1. every node's score, parent and token to LDS, all loads at once;
//   2. a node's rank e = min of the scores on its path: each thread walks its nodes' paths in LDS;
//   3. one wave finds the (M - 1)-th largest e by a bitwise search that ends as soon as a threshold
//      splits off M - 1 nodes (equal ranks: the first in step and slot order), and numbers the kept
//      nodes in that order by ballots;
//   4. lane n of it is node n: its parent's number from LDS, its path's bits by doubling (after r
//      rounds a lane holds 2^r nodes of its path), its place among its siblings from the lanes with
//      the same parent, six ballots;
//      The children's slots are filled with -1 while the loads of 1. fly, and the kept children then
//      written over them.
// Bound by latency: a few KB per query, and five short steps that depend on each other.
// One query of 7 steps x 10 slots: kernel 3.5 us (one wave, its loads step by step, 19.5); 256 queries
// of 8 x 64: 8.3 us (27).
#include "hs_beam.h"

namespace hs {

namespace {

constexpr int kNodes = HS_MAX_DEPTH * HS_MAX_BEAMS;

// NU: 64 NU nodes at most.
template <int NU>
__global__ __launch_bounds__(kThreads) void hs_tree_kernel(hs_tree_args A) {
  constexpr int kMine = (NU * 64 + kThreads - 1) / kThreads;  // nodes of a thread
  __shared__ uint2 s_node[NU * 64];      // a node's score as an ordered integer (0: none), its parent's slot
  __shared__ uint32_t s_rank[NU * 64];   // its rank
  __shared__ int32_t s_token[NU * 64];
  __shared__ uint8_t s_num[NU * 64];     // a kept node's number
  __shared__ int16_t s_grown[HS_MAX_POSITIONS];  // step * K + slot of every kept node
  const int t = threadIdx.x, lane = t & 63, b = blockIdx.x;
  const int D = A.D, K = A.K, M = A.M, N = D * K;

  float v[kMine];
  int p[kMine], token[kMine];
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int i = min(j * kThreads + t, N - 1), d = i / K;
    const int64_t at = ((int64_t)d * A.B + b) * K + (i - d * K);
    v[j] = A.score[at];
    p[j] = A.parent[at];
    token[j] = A.token[at];
  }
  int32_t* cand = A.cand ? A.cand + (int64_t)b * M * K : nullptr;
  if (cand) {
    int i = t;
    if ((M * K & 3) == 0 && ((uintptr_t)cand & 15) == 0) {
      for (; i < M * K / 4; i += kThreads) reinterpret_cast<int4*>(cand)[i] = make_int4(-1, -1, -1, -1);
    } else {
      for (; i < M * K; i += kThreads) cand[i] = -1;
    }
  }
  uint32_t e[kMine], up[kMine];
  int step_at[kMine];  // the first node of the step that the path has come to
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int i = j * kThreads + t;
    const bool node = i < N && isfinite(v[j]) && p[j] >= 0 && (i < K || p[j] < K);
    e[j] = node ? ordered_of(v[j]) : 0;
    up[j] = node ? (uint32_t)p[j] : 0;  // (of the first step: not used)
    step_at[j] = i / K * K;
    if (i < N) {
      s_node[i] = make_uint2(e[j], up[j]);
      s_token[i] = token[j];
    }
  }
  __syncthreads();
  for (int d = 1; d < D; ++d) {  // a thread's nodes side by side: their reads do not wait for each other
#pragma unroll
    for (int j = 0; j < kMine; ++j)
      if (step_at[j] > 0 && e[j] != 0) {
        step_at[j] -= K;
        const uint2 above = s_node[step_at[j] + (int)up[j]];
        e[j] = min(e[j], above.x);  // 0 where the parent is none
        up[j] = above.y;
      }
  }
#pragma unroll
  for (int j = 0; j < kMine; ++j)
    if (j * kThreads + t < N) s_rank[j * kThreads + t] = e[j];
  __syncthreads();

  if (t < 64) {
    uint32_t u[NU];
    int have = 0;
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      u[j] = j * 64 + lane < N ? s_rank[j * 64 + lane] : 0;
      have += __builtin_popcountll(__ballot(u[j] != 0));
    }
    uint32_t least = 1;  // kept: ranks >= least, and the first `ties` of rank least - 1
    int ties = 0;
    if (have > M - 1) {
      // the bits that all ranks share first
      uint32_t some = 0, lack = 0;
#pragma unroll
      for (int j = 0; j < NU; ++j) {
        some |= u[j];
        lack |= u[j] != 0 ? ~u[j] : 0;
      }
      const uint32_t vary = wave_or_bits(some) & wave_or_bits(lack);
      const int top = vary ? 31 - __builtin_clz(vary) : -1;
      uint32_t x = top < 31 ? wave_or_bits(some) >> (top + 1) << (top + 1) : 0;
      int above = 0;  // ranks > the largest value that starts with x's bits
      bool exact = false;
      for (int bit = top; bit >= 0 && !exact; --bit) {
        const uint32_t y = x | (1u << bit);
        int c = 0;
#pragma unroll
        for (int j = 0; j < NU; ++j) c += __builtin_popcountll(__ballot(u[j] >= y));
        if (c >= M - 1) x = y;
        else above = c;
        exact = c == M - 1;
      }
      least = exact ? x : x + 1;
      ties = exact ? 0 : M - 1 - above;
    }
    int n = 1;
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const uint64_t tied = ties ? __ballot(u[j] != 0 && u[j] == least - 1) : 0;
      const bool keep = (u[j] != 0 && u[j] >= least) ||
                        (((tied >> lane) & 1) != 0 && lanes_below(tied) < ties);
      const uint64_t m = __ballot(keep);
      if (keep) {
        const int num = n + lanes_below(m);
        s_num[j * 64 + lane] = (uint8_t)num;
        s_grown[num] = (int16_t)(j * 64 + lane);
      }
      n += __builtin_popcountll(m);
      ties -= min(ties, (int)__builtin_popcountll(tied));
    }
    lds_wave_fence();

    // lane = node
    int tok = -1, parent = -1, depth = -1, slot = -1;
    float score = -INFINITY;
    if (lane == 0) {
      depth = 0;
      score = 0.0f;
    } else if (lane < n) {
      const int g = s_grown[lane], d = g / K;
      slot = g - d * K;
      depth = d + 1;
      tok = s_token[g];
      const uint2 node = s_node[g];
      score = value_of(node.x);
      parent = d == 0 ? 0 : s_num[(d - 1) * K + (int)node.y];
    }
    uint64_t mask = lane < n ? 1ull << lane : 0;
    int far = parent < 0 ? 0 : parent;  // r steps above; the root is its own parent
    for (int r = 1; r <= D; r *= 2) {
      const uint64_t above = __shfl(mask, far, 64);
      const int further = __shfl(far, far, 64);
      if (lane < n) mask |= above;
      far = further;
    }
    uint64_t same = ~0ull;
#pragma unroll
    for (int bit = 0; bit < 6; ++bit) {
      const uint64_t m = __ballot((parent >> bit) & 1);
      same &= (parent >> bit) & 1 ? m : ~m;
    }
    same &= n < 64 ? (1ull << n) - 1 : ~0ull;
    // (the two barriers order these stores after the -1 of every wave)
    if (cand && lane > 0 && lane < n)  // (the root has its own like, lane 0)
      cand[parent * K + lanes_below(same & ~1ull)] = tok;

    const int64_t o = (int64_t)b * M;
    if (lane < M) {
      if (A.node_token) A.node_token[o + lane] = tok;
      if (A.node_parent) A.node_parent[o + lane] = parent;
      if (A.node_depth) A.node_depth[o + lane] = depth;
      if (A.node_slot) A.node_slot[o + lane] = slot;
      if (A.node_score) A.node_score[o + lane] = score;
      if (A.node_mask) A.node_mask[o + lane] = mask;
    }
    if (A.count && lane == 0) A.count[b] = n;
  }
}

}  // namespace

int launch_draft_tree(const hs_tree_args& a, hipStream_t stream) {
  // the search is over registers: as many as the nodes need (132 queries of 135 nodes with 4 a lane 5.1 us, with
  // 8 7.2; 64 of 640 with 16 11.8, with 32 20.0)
  const int N = a.D * a.K;
  if (N <= 128) hs_tree_kernel<2><<<a.B, kThreads, 0, stream>>>(a);
  else if (N <= 256) hs_tree_kernel<4><<<a.B, kThreads, 0, stream>>>(a);
  else if (N <= 512) hs_tree_kernel<8><<<a.B, kThreads, 0, stream>>>(a);
  else if (N <= 1024) hs_tree_kernel<16><<<a.B, kThreads, 0, stream>>>(a);
  else hs_tree_kernel<kNodes / 64><<<a.B, kThreads, 0, stream>>>(a);
  return hipPeekAtLastError() == hipSuccess ? HS_OK : HS_ERR_HIP;
}

}  // namespace hs
