// hs_verify: of a drafted chain or tree the nodes that the target accepts, from given random numbers, and the
// token that the target draws behind the last of them.
//
// With w_v = 2^((z_v - m) c) of node n's target row, c = log2(e) / T, m its largest logit, and children
// c_1 .. c_k of n in the order of their numbers, tokens x_1 .. x_k: what is left of the mass before child j is
//   S_j = rest + w(x_j) + .. + w(x_k),   rest = the sum of w over the tokens of no child,
// and child j is accepted where u[c_j] S_j < w(x_j). S_j is summed from its own terms, not as the total less
// those before it, so that where only children have mass the last one is accepted, whatever the rounding. The
// next token is the first whose running sum over the tokens of no child exceeds u[root] rest. Of a chain with its
// drafter's rows q, the child is accepted where u q(x) < p(x), and the next token is drawn from max(0, p - q).
//
// Launches:
//   1. hs_verify_rows_kernel, a wave per slice of a row: of its weights the sum, relative to its largest logit,
//      without the tokens of the row's children;
//   2. hs_verify_walk_kernel, a workgroup per query: every node's normaliser and accepted child, a wave a node;
//      the path; of its last row the slice in which the running sum passes, read again for the token;
//   3. with a drafter hs_verify_rest_kernel, a wave per slice of the two rows where the path ended at a rejection:
//      the sum of max(0, p - q); and hs_verify_draw_kernel, a workgroup per query: the token.
//
// Precision. Tokens are part of the result and a border between two of 150 thousand is as narrow as their
// probability, so weights and sums are fp64 and an exponential good to 1.1e-12 of itself: a draw from a flat row of
// 152 thousand tokens differs from exact arithmetic once in 6 million (with fp32 exponentials, whose errors leave
// 3.5e-9 in a slice's sum, about once in 2000).
#include <algorithm>
#include <cfloat>

#include "hs_draft.h"

namespace hs {

namespace {

constexpr int kLoads = kVerifySlice / 64;  // of 16 bytes per lane
constexpr int kWalkThreads = 1024;
constexpr int kWalkWaves = kWalkThreads / 64;
constexpr int kHeldParts = kMaxTeamSlices / 64;  // a row's parts per lane

struct Part {
  double sum;  // of the slice's weights relative to m (not finite: a NaN or +inf logit)
  float m;     // its largest logit; -inf: none above
  int at;      // greedy: the lowest token that has it
};

// Where a query's walk ended, for the launches behind it.
struct End {
  double zp, zq;  // 1 / the sums of the target's and the drafter's weights
  double rest;    // of the target's parts
  float mp, mq;   // the largest logits
  int node;       // the last accepted node
  int length;     // nodes on the path; 0: no draft
  int residual;   // the next token comes from max(0, p - q)
  int pad;
};

struct VerifyArgs {
  const char* x;
  const char* y;  // the drafter's rows, or NULL
  int64_t sb, sn, tb, tn;  // bytes between queries and between nodes, of both
  int B, M, S, depth;
  int64_t V, nvec;
  uint32_t units;    // target rows * S
  uint32_t groups0;  // the launch's first workgroup
  FastDiv divS, divM;
  double c;
  const int32_t* token;
  const int32_t* parent;
  const int32_t* count;
  const double* u;
  int32_t* path;
  int32_t* emitted;
  int32_t* length;
  Part* part;       // [2][B * M][S]
  Part* rest_part;  // [B][S]
  End* end;         // [B]
};

// 2^d for d <= 0 (NaN stays) to 1.1e-12 of itself, 0 below 2^-1074: 2^n 2^f, |f| <= 1/2, by the polynomial of degree 8
// that meets 2^f at the nine Chebyshev points of that interval.
__device__ inline double weight_of(double d) {
  const double x = d < -1100.0 ? -1100.0 : d, n = rint(x), f = x - n;
  double p = 1.32552248847991267e-06;
  p = fma(p, f, 1.53100794023831035e-05);
  p = fma(p, f, 1.54034558524190164e-04);
  p = fma(p, f, 1.33334505680000079e-03);
  p = fma(p, f, 9.61812915940261914e-03);
  p = fma(p, f, 5.55041094120593409e-02);
  p = fma(p, f, 2.40226506958129887e-01);
  p = fma(p, f, 6.93147180545933494e-01);
  p = fma(p, f, 1.0);
  return ldexp(p, (int)n);
}
__device__ inline double weight_of(float z, float m, double c) {
  return weight_of(((double)z - (double)m) * c);
}
// What a part's sum counts for relative to M >= m; a part of no logits counts what it holds, 0 or NaN.
__device__ inline double part_value(const Part& p, float M, double c) {
  return p.m == -INFINITY ? p.sum : p.sum * weight_of(p.m, M, c);
}

__device__ inline double shfl_d(double v, int lane) { return __shfl(v, lane, 64); }

// The sum of v over the lanes up to and with this one, in lane order.
__device__ inline double wave_scan_d(double v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double o = __shfl_up(v, d, 64);
    if (lane >= d) v = o + v;
  }
  return v;
}

template <int DT>
__device__ inline float logit_at(const char* row, int64_t t) {
  if constexpr (DT == HS_F32) return reinterpret_cast<const float*>(row)[t];
  else return Vec<DT>::lo(reinterpret_cast<const uint16_t*>(row)[t]);
}

template <int DT>
__device__ inline void load_slice(const char* row, int slice, int lane, const VerifyArgs& A,
                                  float (&z)[kLoads][Vec<DT>::kElems]) {
  using Vt = Vec<DT>;
  typename Vt::Raw raw[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int64_t v = (int64_t)slice * kVerifySlice + i * 64 + lane;
    raw[i] = v < A.nvec ? Vt::load_raw(row, v, A.V) : Vt::neg_raw();
  }
#pragma unroll
  for (int i = 0; i < kLoads; ++i) Vt::unpack(raw[i], z[i]);
}

// The nodes of the draft that are node n's children, as the bit of each lane = node.
__device__ inline bool is_child(const VerifyArgs& A, int b, int n, int count, int lane, int* token) {
  bool child = lane > 0 && lane < count;
  const int64_t o = (int64_t)b * A.M + lane;
  if (child) child = (A.parent ? A.parent[o] : lane - 1) == n;
  *token = -1;
  if (child) {
    const int t = A.token[o];
    child = t >= 0 && t < A.V;
    *token = t;
  }
  return child;
}
__device__ inline int count_of(const VerifyArgs& A, int b) {
  return A.count ? min(max(A.count[b], 0), A.M) : A.M;
}

template <int DT, bool GREEDY>
__global__ void __launch_bounds__(kThreads) hs_verify_rows_kernel(const VerifyArgs A) {
  using Vt = Vec<DT>;
  constexpr int E = Vt::kElems;
  const int lane = threadIdx.x & 63;
  uint32_t unit = uniform((A.groups0 + blockIdx.x) * kWaves + (threadIdx.x >> 6));
  if (unit >= A.units) return;
  const bool q = blockIdx.y != 0;  // the drafter's row
  const uint32_t row = fdiv(unit, A.divS);
  const int slice = (int)(unit - row * (uint32_t)A.S);
  const int b = (int)fdiv(row, A.divM), n = (int)row - b * A.M;
  const int count = count_of(A, b);
  if (n + (q ? 1 : 0) >= count) return;
  const char* x = q ? A.y + b * A.tb + n * A.tn : A.x + b * A.sb + n * A.sn;
  float z[kLoads][E];
  load_slice<DT>(x, slice, lane, A, z);
  const int first = slice * kVerifySlice * E;
  if (!GREEDY && !A.y) {  // the children's tokens have no weight
    int t;
    const bool child = is_child(A, b, n, count, lane, &t);
    uint64_t here = __ballot(child && t >= first && t - first < kVerifySlice * E);
    while (here) {
      const int k = __builtin_ctzll(here);
      here &= here - 1;
      const int mine = __builtin_amdgcn_readlane(t, k) - first - lane * E;
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (mine == i * 64 * E + e) z[i][e] = -INFINITY;
    }
  }
  float m = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      m = fmaxf(m, z[i][e]);
      if (GREEDY) bad |= !(z[i][e] < INFINITY);
    }
  m = fkey_inv(wave_max_i(fkey(m)));
  Part* const out = A.part + ((int64_t)(q ? A.B * A.M : 0) + row) * A.S + slice;
  if (GREEDY) {
    int at = INT_MAX;
#pragma unroll
    for (int i = kLoads - 1; i >= 0; --i)
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (z[i][e] == m) at = first + (i * 64 + lane) * E + e;
    at = -wave_max_i(-at);
    const bool any = __ballot(bad) != 0;
    if (lane == 0) *out = Part{any ? (double)NAN : 0.0, m, at};
    return;
  }
  const float ref = m == -INFINITY ? 0.0f : m;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) s[e & 3] += weight_of(z[i][e], ref, A.c);
  const double sum = wave_sum_d((s[0] + s[1]) + (s[2] + s[3]));
  if (lane == 0) *out = Part{sum, m, 0};
}

// The parts of a row of S, lane l's being those from l * kHeldParts on, so that lanes and parts have one order.
struct RowParts {
  Part p[kHeldParts];
  int held;  // parts a lane
  __device__ RowParts(const Part* part, int S, int lane) {
    held = (S + 63) / 64;
#pragma unroll
    for (int i = 0; i < kHeldParts; ++i) {
      const int k = lane * held + i;
      p[i] = i < held && k < S ? part[k] : Part{0.0, -INFINITY, INT_MAX};
    }
  }
  __device__ float largest() const {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kHeldParts; ++i) m = fmaxf(m, p[i].m);
    return fkey_inv(wave_max_i(fkey(m)));
  }
  __device__ double sum(float M, double c) const {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kHeldParts; ++i)
      if (i < held) s += part_value(p[i], M, c);
    return wave_sum_d(s);
  }
};

// The first of this wave's ordered values whose running sum exceeds `goal`, or the last above 0 where rounding leaves
// none: its lane (-1: none is above 0), and the running sum before that lane. mine: the lane's value.
__device__ inline int passing_lane(double mine, double goal, int lane, double* before) {
  const double upto = wave_scan_d(mine, lane);
  const uint64_t over = __ballot(upto > goal && mine > 0.0), some = __ballot(mine > 0.0);
  if (!some) return -1;
  const int l = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);
  *before = shfl_d(upto, l) - shfl_d(mine, l);
  return l;
}

// One wave: the token of a row at which the running sum of weight(z, w) over the slices' values passes goal.
// value(i): the lane's i-th part's value; weights(slice, w): the slice's weights, in vectors by lane.
template <int E, typename Value, typename Weights>
__device__ inline int draw_token(int held, double goal, int lane, Value value, Weights weights) {
  double v[kHeldParts], mine = 0.0;
#pragma unroll
  for (int i = 0; i < kHeldParts; ++i) {
    v[i] = i < held ? value(i) : 0.0;
    mine += v[i];
  }
  double before = 0.0;
  const int l = passing_lane(mine, goal, lane, &before);
  if (l < 0) return -1;
  // of that lane's parts: the first that passes, or the last above 0
  double run = before;
  int slice = -1;
  double base = before;
#pragma unroll
  for (int i = 0; i < kHeldParts; ++i) {
    const double x = shfl_d(v[i], l);
    if (x > 0.0 && (slice < 0 || !(run > goal))) {
      slice = l * held + i;
      base = run;
      run += x;
    }
  }
  double w[kLoads][E];
  weights(slice, w);
  int token = -1;
  bool done = false;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) sum += w[i][e];
    double start = 0.0;
    const double upto = base + wave_scan_d(sum, lane);
    const uint64_t over = __ballot(upto > goal && sum > 0.0), some = __ballot(sum > 0.0);
    if (done || !some) continue;
    const int k = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);
    start = shfl_d(upto, k) - shfl_d(sum, k);
    int at = -1;
    bool passed = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (!passed && w[i][e] > 0.0) {
        at = e;
        start += w[i][e];
        passed = start > goal;
      }
    }
    at = __shfl(at, k, 64);
    token = (slice * kVerifySlice + i * 64 + k) * E + at;
    done = over != 0;
    base = shfl_d(upto, 63);
  }
  return token;
}

template <int DT>
__device__ inline void weights_of_slice(const char* row, int slice, float M, int lane, const VerifyArgs& A,
                                        double (&w)[kLoads][Vec<DT>::kElems]) {
  float z[kLoads][Vec<DT>::kElems];
  load_slice<DT>(row, slice, lane, A, z);
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
#pragma unroll
    for (int e = 0; e < Vec<DT>::kElems; ++e) w[i][e] = weight_of(z[i][e], M, A.c);
}

// A token drawn from a target row: its parts hold the weights without the children's tokens; `with`: those count
// too (the draft goes no deeper).
template <int DT>
__device__ inline int draw_row(const VerifyArgs& A, int b, int n, int count, bool with, float M, double total, double u,
                               int lane) {
  constexpr int E = Vec<DT>::kElems;
  const char* row = A.x + b * A.sb + n * A.sn;
  const RowParts parts(A.part + ((int64_t)b * A.M + n) * A.S, A.S, lane);
  int t = -1;
  uint64_t children = 0;
  if (!A.y) {
    const bool child = is_child(A, b, n, count, lane, &t);
    children = __ballot(child);
  }
  double extra[kHeldParts];
#pragma unroll
  for (int i = 0; i < kHeldParts; ++i) extra[i] = 0.0;
  if (with) {
    const double mine = (children >> lane) & 1 ? weight_of(logit_at<DT>(row, t), M, A.c) : 0.0;
    for (uint64_t left = children; left; left &= left - 1) {
      const int k = __builtin_ctzll(left), x = __builtin_amdgcn_readlane(t, k);
      // a token that a child before had counts once
      if (__ballot(((children >> lane) & 1) != 0 && lane < k && t == x)) continue;
      const int slice = x / (kVerifySlice * E);
      const double wx = lane_d(mine, k);
#pragma unroll
      for (int i = 0; i < kHeldParts; ++i)
        if (i < parts.held && lane * parts.held + i == slice) extra[i] += wx;
    }
  }
  return draw_token<E>(
      parts.held, u * total, lane, [&](int i) { return part_value(parts.p[i], M, A.c) + extra[i]; },
      [&](int slice, double (&w)[kLoads][E]) {
        weights_of_slice<DT>(row, slice, M, lane, A, w);
        if (with) return;
        for (uint64_t left = children; left; left &= left - 1) {
          const int mine = __builtin_amdgcn_readlane(t, __builtin_ctzll(left)) - (slice * kVerifySlice + lane) * E;
#pragma unroll
          for (int i = 0; i < kLoads; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e)
              if (mine == i * 64 * E + e) w[i][e] = 0.0;
        }
      });
}

// What a node of the draft comes to.
struct Node {
  double total, rest, zq;  // the row's weights with and without its children's; 1 / the drafter's
  float m, mq;
  int next;     // the accepted child; -1: none
  int kind;     // 0: no distribution; 1: draw from the rest; 2: a child of a drafter was rejected
  int arg;      // greedy: the largest logit's token
};

template <int DT, bool GREEDY>
__device__ inline Node fold_node(const VerifyArgs& A, int b, int n, int count, int lane) {
  Node o{};
  o.next = -1;
  const int64_t row = (int64_t)b * A.M + n;
  const RowParts parts(A.part + row * A.S, A.S, lane);
  int t;
  const bool child = is_child(A, b, n, count, lane, &t);
  const uint64_t children = __ballot(child);
  if constexpr (GREEDY) {
    o.m = parts.largest();
    int at = INT_MAX;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kHeldParts; ++i) {
      if (parts.p[i].m == o.m) at = min(at, parts.p[i].at);
      bad |= !(parts.p[i].sum == 0.0);
    }
    at = -wave_max_i(-at);
    o.kind = __ballot(bad) == 0 && o.m > -INFINITY ? 1 : 0;
    o.arg = at;
    const uint64_t hit = __ballot(child && t == at);
    if (o.kind && hit) o.next = __builtin_ctzll(hit);
    return o;
  }
  const char* x = A.x + b * A.sb + n * A.sn;
  const float z = child ? logit_at<DT>(x, t) : -INFINITY;
  const double u = child ? A.u[(int64_t)b * A.M + lane] : 0.0;
  o.m = fmaxf(parts.largest(), fkey_inv(wave_max_i(fkey(fmaxf(z, -INFINITY)))));
  const float ref = o.m == -INFINITY ? 0.0f : o.m;
  o.rest = parts.sum(ref, A.c);
  double w = child ? weight_of(z, ref, A.c) : 0.0;
  if (!A.y) {
    // a token that a child before had is not left
    for (uint64_t k = children; k; k &= k - 1) {
      const int j = __builtin_ctzll(k);
      if (child && j < lane && __builtin_amdgcn_readlane(t, j) == t) w = 0.0;
    }
    double left = o.rest, mine = 0.0;
    for (uint64_t k = children; k;) {
      const int j = 63 - __builtin_clzll(k);
      k &= ~(1ull << j);
      left += lane_d(w, j);
      if (lane == j) mine = left;
    }
    o.total = left;
    o.kind = o.m > -INFINITY && o.total < INFINITY && o.m < INFINITY ? 1 : 0;  // (a NaN total is not below)
    const uint64_t takes = __ballot(child && u * mine < w);
    if (o.kind && takes) o.next = __builtin_ctzll(takes);
    return o;
  }
  o.total = o.rest;
  o.kind = o.m > -INFINITY && o.total < INFINITY && o.m < INFINITY ? 1 : 0;
  if (!o.kind || !children) return o;
  const RowParts drafted(A.part + ((int64_t)A.B * A.M + row) * A.S, A.S, lane);
  o.mq = drafted.largest();
  const double f = drafted.sum(o.mq == -INFINITY ? 0.0f : o.mq, A.c);
  const bool fine = o.mq > -INFINITY && o.mq < INFINITY && f < INFINITY;
  if (!fine) return o;  // nothing can have been drawn from it: the child is rejected, the token drawn from p
  o.zq = 1.0 / f;
  const float zy = child ? logit_at<DT>(A.y + b * A.tb + n * A.tn, t) : -INFINITY;
  const double p = w / o.total, q = child ? weight_of(zy, o.mq, A.c) / f : 0.0;
  const uint64_t takes = __ballot(child && u * q < p);
  if (takes) o.next = __builtin_ctzll(takes);
  else o.kind = 2;
  return o;
}

template <int DT, bool GREEDY>
__global__ void __launch_bounds__(kWalkThreads) hs_verify_walk_kernel(const VerifyArgs A) {
  __shared__ Node s_node[HS_MAX_POSITIONS];
  __shared__ int s_path[HS_MAX_POSITIONS];
  __shared__ int s_len, s_with;
  const int b = blockIdx.x, lane = threadIdx.x & 63, wv = (int)uniform(threadIdx.x >> 6);
  const int count = count_of(A, b);
  for (int n = wv; n < count; n += kWalkWaves) {
    const Node o = fold_node<DT, GREEDY>(A, b, n, count, lane);
    if (lane == 0) s_node[n] = o;
  }
  __syncthreads();
  if (wv != 0) return;
  if (lane == 0) {
    int len = 0, n = 0;
    bool cut = false;
    while (count > 0) {
      s_path[len++] = n;
      const int next = s_node[n].next;
      if (next < 0) break;
      if (len > A.depth) {
        cut = true;
        break;
      }
      n = next;
    }
    s_len = len;
    s_with = len > A.depth;  // the draft ends here, whatever the children
  }
  lds_wave_fence();
  const int len = s_len;
  const int64_t o = (int64_t)b * A.M;
  const int last = len > 0 ? s_path[len - 1] : 0;
  int token = -1;
  bool residual = false;
  Node end{};
  if (len > 0) {
    end = s_node[last];
    const bool with = s_with != 0;
    if (with && end.kind == 2) end.kind = 1;
    residual = end.kind == 2;
    if (GREEDY) token = end.kind ? end.arg : -1;
    else if (end.kind == 1)
      token = draw_row<DT>(A, b, last, count, with, end.m, with ? end.total : end.rest, A.u[o], lane);
  }
  if (lane < A.M) {
    const int next = lane + 1 < len ? s_path[lane + 1] : -1;
    A.path[o + lane] = lane < len ? s_path[lane] : -1;
    A.emitted[o + lane] = next >= 0 ? A.token[o + next] : lane + 1 == len ? token : -1;
  }
  if (lane == 0) {
    A.length[b] = len;
    if (!GREEDY && A.y)
      A.end[b] = End{1.0 / end.total, end.zq, end.rest, end.m, end.mq, last, len, residual ? 1 : 0, 0};
  }
}

// max(0, p - q) of the slice's tokens
template <int DT>
__device__ inline void residual_of_slice(const VerifyArgs& A, int b, const End& e, int slice, int lane,
                                         double (&w)[kLoads][Vec<DT>::kElems]) {
  constexpr int E = Vec<DT>::kElems;
  float z[kLoads][E], y[kLoads][E];
  load_slice<DT>(A.x + b * A.sb + e.node * A.sn, slice, lane, A, z);
  load_slice<DT>(A.y + b * A.tb + e.node * A.tn, slice, lane, A, y);
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
#pragma unroll
    for (int k = 0; k < E; ++k)
      w[i][k] = fmax(0.0, weight_of(z[i][k], e.mp, A.c) * e.zp - weight_of(y[i][k], e.mq, A.c) * e.zq);
}

template <int DT>
__global__ void __launch_bounds__(kThreads) hs_verify_rest_kernel(const VerifyArgs A) {
  constexpr int E = Vec<DT>::kElems;
  const int lane = threadIdx.x & 63;
  const uint32_t unit = uniform(blockIdx.x * kWaves + (threadIdx.x >> 6));
  if (unit >= (uint32_t)A.B * (uint32_t)A.S) return;
  const int b = (int)fdiv(unit, A.divS), slice = (int)unit - b * A.S;
  const End e = A.end[b];
  if (!e.residual) return;
  double w[kLoads][E];
  residual_of_slice<DT>(A, b, e, slice, lane, w);
  double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
#pragma unroll
    for (int k = 0; k < E; ++k) s[k & 3] += w[i][k];
  const double sum = wave_sum_d((s[0] + s[1]) + (s[2] + s[3]));
  if (lane == 0) A.rest_part[(int64_t)b * A.S + slice] = Part{sum, 0.0f, 0};
}

template <int DT>
__global__ void __launch_bounds__(64) hs_verify_draw_kernel(const VerifyArgs A) {
  constexpr int E = Vec<DT>::kElems;
  const int b = blockIdx.x, lane = threadIdx.x;
  const End e = A.end[b];
  if (!e.residual) return;
  const RowParts parts(A.rest_part + (int64_t)b * A.S, A.S, lane);
  double mine = 0.0;
#pragma unroll
  for (int i = 0; i < kHeldParts; ++i) mine += parts.p[i].sum;
  const double total = wave_sum_d(mine), u = A.u[(int64_t)b * A.M];
  int token;
  if (total > 0.0)
    token = draw_token<E>(
        parts.held, u * total, lane, [&](int i) { return parts.p[i].sum; },
        [&](int slice, double (&w)[kLoads][E]) { residual_of_slice<DT>(A, b, e, slice, lane, w); });
  else  // p and q are the same but for rounding
    token = draw_row<DT>(A, b, e.node, 0, false, e.mp, e.rest, u, lane);
  if (lane == 0) A.emitted[(int64_t)b * A.M + e.length - 1] = token;
}

template <int DT, bool GREEDY>
void launch_of(VerifyArgs A, hipStream_t st) {
  const uint32_t groups = (A.units + kWaves - 1) / kWaves;
  for (A.groups0 = 0; A.groups0 < groups; A.groups0 += kMostGroups) {
    const dim3 grid(std::min(groups - A.groups0, kMostGroups), !GREEDY && A.y ? 2 : 1);
    hs_verify_rows_kernel<DT, GREEDY><<<grid, kThreads, 0, st>>>(A);
    if (hipPeekAtLastError() != hipSuccess) return;
  }
  hs_verify_walk_kernel<DT, GREEDY><<<A.B, kWalkThreads, 0, st>>>(A);
  if (GREEDY || !A.y || hipPeekAtLastError() != hipSuccess) return;
  hs_verify_rest_kernel<DT><<<(int)(((int64_t)A.B * A.S + kWaves - 1) / kWaves), kThreads, 0, st>>>(A);
  if (hipPeekAtLastError() != hipSuccess) return;
  hs_verify_draw_kernel<DT><<<A.B, 64, 0, st>>>(A);
}

}  // namespace

bool verify_geom(int B, int M, int64_t V, int dtype, bool drafter, VerifyGeom* g) {
  if (B < 1 || M < 1 || V < 1) return false;
  if (B > HS_MAX_QUERIES || M > HS_MAX_POSITIONS || V > INT32_MAX) return false;
  if (dtype != HS_F32 && dtype != HS_BF16 && dtype != HS_F16) return false;
  const int E = dtype == HS_F32 ? 4 : 8;
  g->B = B;
  g->M = M;
  g->V = V;
  g->nvec = (V + E - 1) / E;
  g->dtype = dtype;
  g->drafter = drafter;
  if (g->nvec > (int64_t)kMaxTeamSlices * kVerifySlice) return false;
  g->S = (int)((g->nvec + kVerifySlice - 1) / kVerifySlice);
  return true;
}

size_t verify_ws_bytes(const VerifyGeom& g) {
  const size_t rows = (size_t)g.B * g.M * (g.drafter ? 2 : 1);
  const size_t more = g.drafter ? align256((size_t)g.B * g.S * sizeof(Part)) + align256((size_t)g.B * sizeof(End)) : 0;
  return align256(rows * g.S * sizeof(Part)) + more;
}

int launch_verify(const VerifyGeom& g, const hs_verify_args& a, hipStream_t stream) {
  VerifyArgs A;
  const int64_t es = g.dtype == HS_F32 ? 4 : 2;
  A.x = reinterpret_cast<const char*>(a.target.ptr);
  A.sb = a.target.stride_b * es;
  A.sn = a.target.stride_k * es;
  A.y = g.drafter ? reinterpret_cast<const char*>(a.drafter.ptr) : nullptr;
  A.tb = a.drafter.stride_b * es;
  A.tn = a.drafter.stride_k * es;
  A.B = g.B;
  A.M = g.M;
  A.S = g.S;
  A.depth = a.depth;
  A.V = g.V;
  A.nvec = g.nvec;
  A.units = (uint32_t)((int64_t)g.B * g.M * g.S);
  A.divS = make_fastdiv((uint32_t)g.S);
  A.divM = make_fastdiv((uint32_t)g.M);
  A.c = 1.4426950408889634074 / a.temperature;
  A.token = a.token;
  A.parent = a.parent;
  A.count = a.count;
  A.u = a.u;
  A.path = a.out_path;
  A.emitted = a.out_token;
  A.length = a.out_length;
  char* ws = reinterpret_cast<char*>(a.workspace);
  A.part = reinterpret_cast<Part*>(ws);
  ws += align256((size_t)A.units * (g.drafter ? 2 : 1) * sizeof(Part));
  A.rest_part = reinterpret_cast<Part*>(ws);
  A.end = reinterpret_cast<End*>(ws + align256((size_t)g.B * g.S * sizeof(Part)));
  const bool greedy = a.mode == HS_GREEDY;
  if (greedy) A.c = 0.0;
  if (g.dtype == HS_F32) greedy ? launch_of<HS_F32, true>(A, stream) : launch_of<HS_F32, false>(A, stream);
  else if (g.dtype == HS_F16) greedy ? launch_of<HS_F16, true>(A, stream) : launch_of<HS_F16, false>(A, stream);
  else greedy ? launch_of<HS_BF16, true>(A, stream) : launch_of<HS_BF16, false>(A, stream);
  return hipPeekAtLastError() == hipSuccess ? HS_OK : HS_ERR_HIP;
}

}  // namespace hs
