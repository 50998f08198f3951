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
//      without the tokens of the row's children. Every node's row in one launch, or, of a large tree (by_levels), a
//      launch per level for the nodes that the level before accepted: no row off the paths is read;
//   2. hs_verify_walk_kernel, a workgroup per query: the normaliser and accepted child of every node that has children,
//      a wave a node; the path; of its last row the slice in which the running sum passes, read again for the token.
//      Behind levels the path is known, and a wave a query does the rest;
//   3. with a drafter hs_verify_rest_kernel, a wave per slice of the two rows where the path ended at a rejection:
//      the sum of max(0, p - q); and hs_verify_draw_kernel, a workgroup per query: the token.
//
// Precision. Tokens are part of the result and a border between two of 150 thousand is as narrow as their
// probability, so weights and sums are fp64 and an exponential good to 1.1e-12 of itself: a draw from a flat row of
// 152 thousand tokens differs from exact arithmetic once in 6 million (with fp32 exponentials, whose errors leave
// 3.5e-9 in a slice's sum, about once in 2000).
//
// What bounds it. Few rows: the launches and the latencies of a row read twice (a chain of 4 tokens over 32 thousand fp32
// 14 us in four launches; 61 nodes over 152 thousand bf16 9 in the rows and 11 in the walk). Many: the vector units in
// the rows kernel, which are never idle, at 19 instructions a logit, ten of them fp64, all at one rate (64 chains of 8
// tokens and their drafter, 151936 bf16: 165 million logits in 96 to 105 us, 3.4 TB/s; with 21, 106 to 125; with seventeen
// in fp64, 123 to 140), then 9 for the walk and 21 for what a rejection leaves. 32 trees of 61 nodes by levels: 55 to 58,
// launches of 2.1 to 7 that wait for cur, parts, token and logit one behind the other before their row's first load.
#include <algorithm>
#include <cfloat>

#include "hs_draft.h"

namespace hs {

namespace {

constexpr int kLoads = kVerifySlice / 64;  // of 16 bytes per lane
constexpr int kWalkThreads = 1024;
constexpr int kWalkWaves = kWalkThreads / 64;
constexpr int kMostHeld = kMaxTeamSlices / 64;  // a row's parts per lane

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
  int level;         // of the launch, where a launch is a level
  int32_t* cur;      // [depth + 1][B]: the nodes on the paths, then -1
  FastDiv divS, divM;
  double c;
  float reach;       // 120 / c
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
// 2^(i / 128): by the series of the exponential, from its least term on.
struct Powers {
  double at[128];
};
constexpr Powers powers_of_two() {
  Powers t{};
  for (int i = 0; i < 128; ++i) {
    const double x = i * (0.6931471805599453094 / 128);
    double p = 1.0;
    for (int k = 24; k >= 1; --k) p = 1.0 + x / k * p;
    t.at[i] = p;
  }
  return t;
}
__device__ const Powers kPowers = powers_of_two();

// weight_of(z, m) added to `sum`, for a row's largest logit m, by ten instructions in fp64 instead of seventeen:
// d = (z - m) c is rounded to a multiple k of 1/128 by adding 1.5 * 2^45, whose last bits are then 128 k; the rest
// r = d - k, |r| <= 2^-8, is exact, 2^r by the polynomial of degree 3 that has 2^r's value and slope at 0 and meets it at
// +-0.91 2^-8 (3.9e-13 of itself, and 1 at 0: a flat row's weights are 1), and 2^k a power from LDS and an exponent.
// Below `low`, 120 under the largest, weights are 2^-120: they do not reach a sum that holds 1. NaN stays.
struct Sums {
  const double* powers;
  double c, m;
  float low;
  __device__ void add(float z, double& sum) const {
    const double x = (double)__builtin_elementwise_maximum(z, low) - m, s = fma(x, c, 0x1.8p45), r = fma(x, c, 0x1.8p45 - s);
    const int k = (int)(uint32_t)(uint64_t)__double_as_longlong(s);
    const double power = ldexp(powers[k & 127], k >> 7);
    double p = 5.55041255195012004e-02;
    p = fma(p, r, 2.40226628539921244e-01);
    p = fma(p, r, 6.93147180559945286e-01);
    p = fma(p, r, 1.0);
    sum = fma(power, p, sum);
  }
};
__device__ inline double weight_of(float z, float m, double c) {
  return weight_of(((double)z - (double)m) * c);
}
// What a part's sum counts for relative to M >= m; a part of no logits counts what it holds, 0 or NaN.
__device__ inline double part_value(const Part& p, float M, double c) {
  return p.m == -INFINITY ? p.sum : p.sum * weight_of(p.m, M, c);
}

// v of the lane that CTRL names, 0 where there is none or the row of 16 lanes is not in ROWS.
template <int CTRL, int ROWS>
__device__ inline double dpp_or_0(double v) {
  const uint64_t x = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xF, false);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
// The sum of v over the lanes up to and with this one.
__device__ inline double wave_scan_d(double v) {
  v += dpp_or_0<0x111, 0xF>(v);  // row_shr by 1, 2, 4 and 8
  v += dpp_or_0<0x112, 0xF>(v);
  v += dpp_or_0<0x114, 0xF>(v);
  v += dpp_or_0<0x118, 0xF>(v);
  v += dpp_or_0<0x142, 0xA>(v);  // row_bcast15: the last of a row to the next one
  v += dpp_or_0<0x143, 0xC>(v);  // row_bcast31: that of the lower half to the upper
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

// The i-th of a lane's vectors of a slice.
template <int DT>
__device__ inline void load_vector(const char* row, int slice, int i, int lane, const VerifyArgs& A,
                                   float (&z)[Vec<DT>::kElems]) {
  using Vt = Vec<DT>;
  const int64_t v = (int64_t)slice * kVerifySlice + i * 64 + lane;
  Vt::unpack(v < A.nvec ? Vt::load_raw(row, v, A.V) : Vt::neg_raw(), z);
}

// A query's draft: lane = node.
struct Draft {
  int parent, token;  // parent: -2 where the lane is no node that may be accepted
  __device__ Draft(const VerifyArgs& A, int b, int count, int lane) {
    parent = -2;
    token = -1;
    if (lane > 0 && lane < count) {
      const int64_t o = (int64_t)b * A.M + lane;
      token = A.token[o];
      parent = A.parent ? A.parent[o] : lane - 1;
      if (token < 0 || token >= A.V) parent = -2;
    }
  }
  __device__ bool child_of(int n) const { return parent == n; }
};
__device__ inline int count_of(const VerifyArgs& A, int b) {
  return A.count ? min(max(A.count[b], 0), A.M) : A.M;
}

// The parts of a row of S <= 64 HELD, a lane's one behind the other, so that lanes and parts have one order.
template <int HELD>
struct RowParts {
  Part p[HELD];
  int held;  // parts a lane
  __device__ void load(const Part* part, int S, int lane) {
    held = (S + 63) / 64;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int k = lane * held + i;
      p[i] = i < held && k < S ? part[k] : Part{0.0, -INFINITY, INT_MAX};
    }
  }
  __device__ float largest() const {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < HELD; ++i) m = fmaxf(m, p[i].m);
    return fkey_inv(wave_max_i(fkey(m)));
  }
  __device__ double sum(float M, double c) const {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (i < held) s += part_value(p[i], M, c);
    return wave_sum_d(s);
  }
};

// The first of this wave's ordered values whose running sum exceeds `goal`, or the last above 0 where rounding leaves
// none: its lane (-1: none is above 0), and the running sum before that lane. mine: the lane's value.
__device__ inline int passing_lane(double mine, double goal, double* before) {
  const double upto = wave_scan_d(mine);
  const uint64_t over = __ballot(upto > goal && mine > 0.0), some = __ballot(mine > 0.0);
  if (!some) return -1;
  const int l = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);
  *before = lane_d(upto, l) - lane_d(mine, l);
  return l;
}

// What the waves of a draw tell each other.
struct Draw {
  double total[kLoads];
  int some[kLoads], over[kLoads], token;
};
// kLoads waves: the token of a row at which the running sum over the slices' values passes goal. value(i): the lane's i-th
// part's value; weights(slice, i, w): the weights of the i-th of the lane's vectors of a slice, the wv-th wave's. (One wave
// for all of a slice: a draw from the residual 6.6 to 8.0 us and so 4.6 to 5.1, the walk of 61 nodes 12.0 and 10.9.)
template <int E, int HELD, typename Value, typename Weights>
__device__ inline int draw_token(int held, double goal, int lane, int wv, Draw* s, Value value, Weights weights) {
  double v[HELD], mine = 0.0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    v[i] = i < held ? value(i) : 0.0;
    mine += v[i];
  }
  double before = 0.0;
  const int l = passing_lane(mine, goal, &before);
  if (l < 0) return -1;
  // of that lane's parts: the first that passes, or the last above 0
  double run = before;
  int slice = -1;
  double base = before;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const double x = lane_d(v[i], l);
    if (x > 0.0 && (slice < 0 || !(run > goal))) {
      slice = l * held + i;
      base = run;
      run += x;
    }
  }
  double w[E], sum = 0.0;
  weights(slice, wv, w);
#pragma unroll
  for (int e = 0; e < E; ++e) sum += w[e];
  const double upto = wave_scan_d(sum);
  const uint64_t some = __ballot(sum > 0.0);
  if (lane == 63) {
    s->total[wv] = upto;
    s->some[wv] = some != 0;
  }
  __syncthreads();
  for (int i = 0; i < wv; ++i) base += s->total[i];
  // the lane of the wave's first vector that passes, or of the last above 0; so of the waves
  const uint64_t over = __ballot(base + upto > goal) & some;
  if (lane == 63) s->over[wv] = over != 0;
  __syncthreads();
  int which = -1;
  for (int i = 0; i < kLoads; ++i)
    if (s->some[i] && (which < 0 || !s->over[which])) which = i;
  if (which < 0) return -1;
  if (wv == which) {
    const int k = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);
    before = base + (lane_d(upto, k) - lane_d(sum, k));
    int at = -1;
    bool passed = false;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (!passed && w[e] > 0.0) {
        at = e;
        before += w[e];
        passed = before > goal;
      }
    if (lane == k) s->token = (slice * kVerifySlice + which * 64 + k) * E + at;
  }
  __syncthreads();
  return s->token;
}

// A token drawn from a target row: its parts hold the weights without the children's tokens; `with`: those count
// too (the draft goes no deeper).
template <int DT, int HELD>
__device__ inline int draw_row(const VerifyArgs& A, int b, int n, int count, bool with, float M, double total, double u,
                               int lane, int wv, Draw* s) {
  constexpr int E = Vec<DT>::kElems;
  const char* row = A.x + b * A.sb + n * A.sn;
  RowParts<HELD> parts;
  parts.load(A.part + ((int64_t)b * A.M + n) * A.S, A.S, lane);
  const Draft draft(A, b, count, lane);
  const int t = draft.token;
  const uint64_t children = A.y ? 0 : __ballot(draft.child_of(n));
  double extra[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) extra[i] = 0.0;
  if (with) {
    const double mine = (children >> lane) & 1 ? weight_of(logit_at<DT>(row, t), M, A.c) : 0.0;
    for (uint64_t left = children; left; left &= left - 1) {
      const int k = __builtin_ctzll(left), x = __builtin_amdgcn_readlane(t, k);
      // a token that a child before had counts once
      if (__ballot(((children >> lane) & 1) != 0 && lane < k && t == x)) continue;
      const int slice = x / (kVerifySlice * E);
      const double wx = lane_d(mine, k);
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (i < parts.held && lane * parts.held + i == slice) extra[i] += wx;
    }
  }
  return draw_token<E, HELD>(
      parts.held, u * total, lane, wv, s, [&](int i) { return part_value(parts.p[i], M, A.c) + extra[i]; },
      [&](int slice, int i, double (&w)[E]) {
        float z[E];
        load_vector<DT>(row, slice, i, lane, A, z);
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = weight_of(z[e], M, A.c);
        if (with) return;
        for (uint64_t left = children; left; left &= left - 1) {
          const int mine = __builtin_amdgcn_readlane(t, __builtin_ctzll(left)) - (slice * kVerifySlice + i * 64 + lane) * E;
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (mine == e) w[e] = 0.0;
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

// What a node is folded from.
template <int HELD>
struct NodeIn {
  RowParts<HELD> parts, drafted;
  float z, zy;  // the logits of the lane's token, where it is a child's
  template <int DT, bool GREEDY>
  __device__ void load(const VerifyArgs& A, const Draft& draft, int b, int n, int lane) {
    const int64_t row = (int64_t)b * A.M + n;
    parts.load(A.part + row * A.S, A.S, lane);
    if (GREEDY) return;
    const bool child = draft.child_of(n);
    z = child ? logit_at<DT>(A.x + b * A.sb + n * A.sn, draft.token) : -INFINITY;
    if (!A.y || !__ballot(child)) return;
    drafted.load(A.part + ((int64_t)A.B * A.M + row) * A.S, A.S, lane);
    zy = child ? logit_at<DT>(A.y + b * A.tb + n * A.tn, draft.token) : -INFINITY;
  }
};

// u: the lane's random number.
template <bool GREEDY, int HELD>
__device__ inline Node fold_node(const VerifyArgs& A, const Draft& draft, const NodeIn<HELD>& in, double u, int n,
                                 int lane) {
  Node o{};
  o.next = -1;
  const int t = draft.token;
  const bool child = draft.child_of(n);
  const uint64_t children = __ballot(child);
  if constexpr (GREEDY) {
    o.m = in.parts.largest();
    int at = INT_MAX;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      if (in.parts.p[i].m == o.m) at = min(at, in.parts.p[i].at);
      bad |= !(in.parts.p[i].sum == 0.0);
    }
    at = -wave_max_i(-at);
    o.kind = __ballot(bad) == 0 && o.m > -INFINITY ? 1 : 0;
    o.arg = at;
    const uint64_t hit = __ballot(child && t == at);
    if (o.kind && hit) o.next = __builtin_ctzll(hit);
    return o;
  }
  o.m = fmaxf(in.parts.largest(), fkey_inv(wave_max_i(fkey(fmaxf(in.z, -INFINITY)))));
  const float ref = o.m == -INFINITY ? 0.0f : o.m;
  o.rest = in.parts.sum(ref, A.c);
  double w = child ? weight_of(in.z, ref, A.c) : 0.0;
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
  o.mq = in.drafted.largest();
  const double f = in.drafted.sum(o.mq == -INFINITY ? 0.0f : o.mq, A.c);
  const bool fine = o.mq > -INFINITY && o.mq < INFINITY && f < INFINITY;
  if (!fine) return o;  // nothing can have been drawn from it: the child is rejected, the token drawn from p
  o.zq = 1.0 / f;
  const double p = w / o.total, q = child ? weight_of(in.zy, o.mq, A.c) / f : 0.0;
  const uint64_t takes = __ballot(child && u * q < p);
  if (takes) o.next = __builtin_ctzll(takes);
  else o.kind = 2;
  return o;
}
template <int DT, bool GREEDY, int HELD>
__device__ inline Node node_of(const VerifyArgs& A, const Draft& draft, int b, int n, int lane) {
  NodeIn<HELD> in;
  in.template load<DT, GREEDY>(A, draft, b, n, lane);
  const double u = !GREEDY && lane < A.M ? A.u[(int64_t)b * A.M + lane] : 0.0;
  return fold_node<GREEDY, HELD>(A, draft, in, u, n, lane);
}

// HELD 0: every node's row. Otherwise the rows of one level: of the nodes that follow the ones of the level before,
// which every wave of a query finds by itself.
template <int DT, bool GREEDY, int HELD>
__global__ void __launch_bounds__(kThreads) hs_verify_rows_kernel(const VerifyArgs A) {
  using Vt = Vec<DT>;
  constexpr int E = Vt::kElems;
  const int lane = threadIdx.x & 63;
  uint32_t unit = uniform((A.groups0 + blockIdx.x) * kWaves + (threadIdx.x >> 6));
  if (unit >= A.units) return;
  const bool q = blockIdx.y != 0;  // the drafter's row
  uint32_t row = fdiv(unit, A.divS);
  const int slice = (int)(unit - row * (uint32_t)A.S);
  int b, n, count;
  if constexpr (HELD == 0) {
    b = (int)fdiv(row, A.divM);
    n = (int)row - b * A.M;
    count = count_of(A, b);
  } else {
    b = (int)row;
    count = count_of(A, b);
    n = count > 0 ? 0 : -1;
    if (A.level > 0) {
      n = A.cur[(int64_t)(A.level - 1) * A.B + b];
      if (n >= 0) n = node_of<DT, GREEDY, HELD>(A, Draft(A, b, count, lane), b, n, lane).next;
    }
    if (slice == 0 && !q && lane == 0) A.cur[(int64_t)A.level * A.B + b] = n;
    if (n < 0) return;
    row = (uint32_t)(b * A.M + n);
  }
  if (n + (q ? 1 : 0) >= count) return;
  const char* x = q ? A.y + b * A.tb + n * A.tn : A.x + b * A.sb + n * A.sn;
  __shared__ double2 s_powers[GREEDY ? 1 : kWaves][64];  // a wave's own: the table arrives with its logits
  const int wv = (int)uniform(threadIdx.x >> 6);
  double2 power;
  if (!GREEDY) power = reinterpret_cast<const double2*>(kPowers.at)[lane];
  float z[kLoads][E];
  load_slice<DT>(x, slice, lane, A, z);
  if (!GREEDY) s_powers[wv][lane] = power;
  const int first = slice * kVerifySlice * E;
  if (!GREEDY && !A.y) {  // the children's tokens have no weight
    const Draft draft(A, b, count, lane);
    const int t = draft.token;
    uint64_t here = __ballot(draft.child_of(n) && t >= first && t - first < kVerifySlice * E);
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
  // (beyond 2^16 the last bit of m is not far below 120 / c)
  if (uniform((uint32_t)(m > -INFINITY && fabs((double)m * A.c) <= 65536.0))) {
    lds_wave_fence();
    const Sums by{reinterpret_cast<const double*>(s_powers[wv]), A.c, (double)m, m - A.reach};
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) by.add(z[i][e], s[e & 3]);
  } else {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) s[e & 3] += weight_of(z[i][e], ref, A.c);
  }
  const double sum = wave_sum_d((s[0] + s[1]) + (s[2] + s[3]));
  if (lane == 0) *out = Part{sum, m, 0};
}

// LEVELS: the path is known but for whether its last node is the end. The draw is its first kLoads waves', of which each
// finds the path's end for itself.
template <int DT, bool GREEDY, int HELD, bool LEVELS>
__global__ void __launch_bounds__(LEVELS ? 64 * kLoads : kWalkThreads) hs_verify_walk_kernel(const VerifyArgs A) {
  __shared__ Node s_node[LEVELS ? 1 : HS_MAX_POSITIONS];
  __shared__ int s_path[HS_MAX_POSITIONS];
  __shared__ int s_len, s_with;
  __shared__ Draw s_draw;
  const int b = blockIdx.x, lane = threadIdx.x & 63, wv = (int)uniform(threadIdx.x >> 6);
  const int count = count_of(A, b);
  const Draft draft(A, b, count, lane);
  Node end{};
  if constexpr (LEVELS) {
    const int at = lane <= A.depth ? A.cur[(int64_t)lane * A.B + b] : -1;
    const int len = __builtin_popcountll(__ballot(at >= 0));
    if (len > 0) end = node_of<DT, GREEDY, HELD>(A, draft, b, __builtin_amdgcn_readlane(at, max(len, 1) - 1), lane);
    if (wv == 0) s_path[lane] = at;
    if (threadIdx.x == 0) {
      s_len = len;
      s_with = len > A.depth;
    }
  } else {
    // (a node without children is folded only where the path ends with it: most of a tree are such, 61 nodes 14.6 -> 12.1 us)
    for (int n = wv; n < count; n += kWalkWaves) {
      if (!__ballot(draft.child_of(n))) {
        if (lane == 0) s_node[n].next = -1;
        continue;
      }
      const Node o = node_of<DT, GREEDY, HELD>(A, draft, b, n, lane);
      if (lane == 0) s_node[n] = o;
    }
    __syncthreads();
    if (wv >= kLoads) return;
  }
  if (!LEVELS && threadIdx.x == 0) {
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
  __syncthreads();
  const int len = s_len;
  const int64_t o = (int64_t)b * A.M;
  const int last = len > 0 ? s_path[len - 1] : 0;
  int token = -1;
  bool residual = false;
  if (len > 0) {
    if constexpr (!LEVELS)
      end = __ballot(draft.child_of(last)) ? s_node[last] : node_of<DT, GREEDY, HELD>(A, draft, b, last, lane);
    const bool with = s_with != 0;
    if (with && end.kind == 2) end.kind = 1;
    residual = end.kind == 2;
    if (GREEDY) token = end.kind ? end.arg : -1;
    else if (end.kind == 1)
      token = draw_row<DT, HELD>(A, b, last, count, with, end.m, with ? end.total : end.rest, A.u[o], lane, wv, &s_draw);
  }
  if (wv != 0) return;
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

// max(0, p - q) of a token
__device__ inline double residual(float z, float y, const End& e, const VerifyArgs& A) {
  return fmax(0.0, weight_of(z, e.mp, A.c) * e.zp - weight_of(y, e.mq, A.c) * e.zq);
}
// and of the slice's
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
      w[i][k] = residual(z[i][k], y[i][k], e, A);
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

template <int DT, int HELD>
__global__ void __launch_bounds__(64 * kLoads) hs_verify_draw_kernel(const VerifyArgs A) {
  constexpr int E = Vec<DT>::kElems;
  __shared__ Draw s_draw;
  const int b = blockIdx.x, lane = threadIdx.x & 63, wv = (int)uniform(threadIdx.x >> 6);
  const End e = A.end[b];
  if (!e.residual) return;
  RowParts<HELD> parts;
  parts.load(A.rest_part + (int64_t)b * A.S, A.S, lane);
  double mine = 0.0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) mine += parts.p[i].sum;
  const double total = wave_sum_d(mine), u = A.u[(int64_t)b * A.M];
  int token;
  if (total > 0.0)
    token = draw_token<E, HELD>(
        parts.held, u * total, lane, wv, &s_draw, [&](int i) { return parts.p[i].sum; },
        [&](int slice, int i, double (&w)[E]) {
          float z[E], y[E];
          load_vector<DT>(A.x + b * A.sb + e.node * A.sn, slice, i, lane, A, z);
          load_vector<DT>(A.y + b * A.tb + e.node * A.tn, slice, i, lane, A, y);
#pragma unroll
          for (int k = 0; k < E; ++k) w[k] = residual(z[k], y[k], e, A);
        });
  else  // p and q are the same but for rounding
    token = draw_row<DT, HELD>(A, b, e.node, 0, false, e.mp, e.rest, u, lane, wv, &s_draw);
  if (threadIdx.x == 0) A.emitted[(int64_t)b * A.M + e.length - 1] = token;
}

template <int DT, bool GREEDY, int HELD>
void launch_held(VerifyArgs A, bool levels, hipStream_t st) {
  const bool drafter = !GREEDY && A.y;
  const uint32_t groups = (A.units + kWaves - 1) / kWaves;
  for (A.level = 0; A.level <= (levels ? A.depth : 0); ++A.level)
    for (A.groups0 = 0; A.groups0 < groups; A.groups0 += kMostGroups) {
      const dim3 grid(std::min(groups - A.groups0, kMostGroups), drafter ? 2 : 1);
      if (levels) hs_verify_rows_kernel<DT, GREEDY, HELD><<<grid, kThreads, 0, st>>>(A);
      else hs_verify_rows_kernel<DT, GREEDY, 0><<<grid, kThreads, 0, st>>>(A);
      if (hipPeekAtLastError() != hipSuccess) return;
    }
  if (levels) hs_verify_walk_kernel<DT, GREEDY, HELD, true><<<A.B, 64 * kLoads, 0, st>>>(A);
  else hs_verify_walk_kernel<DT, GREEDY, HELD, false><<<A.B, kWalkThreads, 0, st>>>(A);
  if (!drafter || hipPeekAtLastError() != hipSuccess) return;
  hs_verify_rest_kernel<DT><<<(int)(((int64_t)A.B * A.S + kWaves - 1) / kWaves), kThreads, 0, st>>>(A);
  if (hipPeekAtLastError() != hipSuccess) return;
  hs_verify_draw_kernel<DT, HELD><<<A.B, 64 * kLoads, 0, st>>>(A);
}

template <int DT, bool GREEDY>
void launch_of(const VerifyArgs& A, bool levels, hipStream_t st) {
  if (A.S <= 128) launch_held<DT, GREEDY, 2>(A, levels, st);
  else launch_held<DT, GREEDY, kMostHeld>(A, levels, st);
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
  const size_t cur = align256((size_t)g.B * g.M * sizeof(int32_t));
  const size_t rows = (size_t)g.B * g.M * (g.drafter ? 2 : 1);
  const size_t more = g.drafter ? align256((size_t)g.B * g.S * sizeof(Part)) + align256((size_t)g.B * sizeof(End)) : 0;
  return align256(rows * g.S * sizeof(Part)) + more + cur;
}

// Whether a tree's rows are read level by level, those on the paths alone, in depth + 1 launches: where the rows off the
// paths surely take longer than the launches, by a rate of rows and 8 us a level that are on the safe side. us all at once and
// by levels, trees of 61 nodes, 7 deep, of 128256 bf16, paths of 2 to 3 nodes: 4 trees 35 and 42, 8 50 and 43, 13 (the rule's
// border) 68 to 70 and 46, 32 164 and 53; greedy 8 25 and 33, 13 36 and 34, 24 (the border) 69 and 36, 32 89 and 38.
// 64 chains of 8 tokens of 151936 with their drafter, all on the path, 102 and 167, of fixed tokens 55 and 71, greedy 29 and
// 60. With depth M - 1, which a call that does not know better gives, no row counts as off the paths.
static bool by_levels(const VerifyGeom& g, int depth, bool greedy) {
  const double row = (double)g.B * g.V * (g.dtype == HS_F32 ? 4 : 2);
  return !g.drafter && row * (g.M - (depth + 1)) / (greedy ? 5e6 : 2.8e6) > 8.0 * (depth + 1);
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
  const bool greedy = a.mode == HS_GREEDY, levels = by_levels(g, a.depth, greedy);
  A.units = (uint32_t)((int64_t)g.B * (levels ? 1 : g.M) * g.S);
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
  ws += align256((size_t)g.B * g.M * g.S * (g.drafter ? 2 : 1) * sizeof(Part));
  A.cur = reinterpret_cast<int32_t*>(ws);
  ws += align256((size_t)g.B * g.M * sizeof(int32_t));
  A.rest_part = reinterpret_cast<Part*>(ws);
  A.end = reinterpret_cast<End*>(ws + align256((size_t)g.B * g.S * sizeof(Part)));
  A.reach = (float)(120.0 / A.c);
  if (greedy) A.c = 0.0;
  if (g.dtype == HS_F32) greedy ? launch_of<HS_F32, true>(A, levels, stream) : launch_of<HS_F32, false>(A, levels, stream);
  else if (g.dtype == HS_F16) greedy ? launch_of<HS_F16, true>(A, levels, stream) : launch_of<HS_F16, false>(A, levels, stream);
  else greedy ? launch_of<HS_BF16, true>(A, levels, stream) : launch_of<HS_BF16, false>(A, levels, stream);
  return hipPeekAtLastError() == hipSuccess ? HS_OK : HS_ERR_HIP;
}

}  // namespace hs
