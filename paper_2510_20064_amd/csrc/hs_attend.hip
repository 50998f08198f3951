// hs_tree_attention: the queries of a draft's nodes over a cache held in 8 bits and over the nodes on their paths.
//
// A query's rows r are its nodes' query heads that share a cached head; with s_rt = scale log2(e) ks_t (q_r . k_t),
// ks and vs the scales of t's page,
//   o_r = sum_t p_rt vs_t v_t / sum_t p_rt,   p_rt = 2^(s_rt - m_r).
// The values' scales go into the weights: with x_rt = s_rt + log2 vs_t, w_rt = 2^(x_rt - m_r) and m_r following the
// largest x, o_r = sum w v / sum w / vs: a weight is rounded relative to what it adds, whatever its page's scale.
//
// Layout. Products are S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16 tiles, so that a row's scores, weights,
// maximum and sum all stay in the two lanes (r, r + 32) that hold its column, and the weights are the second
// product's operand as they stand: the scores' registers of lane half h are tokens 16 h .. 16 h + 15 of a tile of
// 32 if the tile's K rows are taken in the order pi below. A page holds its values by dimension, so those 16 tokens
// of one dimension are one 16-byte load. No operand goes through LDS.
// Codes of 8 bits become bf16 or fp16 without error (3 bits of mantissa, 2^-9 to 448), one instruction for two.
// Weights are rounded to fp16 (relative 2^-12, half of a bf16 query's own rounding), as 2^12 w, so that what lies
// below 2^-36 of the largest is lost and not what lies below 2^-24; m follows only in steps above 2^3 (w stays
// below 2^16), which spares most tiles the multiplication of O. Sums and O are fp32.
#include <algorithm>
#include <cfloat>

#include "hs_draft.h"

namespace hs {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kHeadroom = 12.0f;  // weights are held as 2^12 w
constexpr float kSlack = 3.0f;      // m follows a maximum more than this above it
constexpr float kLowest = -1.7e38f; // m before the first token

struct AttendArgs {
  const char* q;
  const char* k;
  const char* v;
  char* out;
  int64_t qb, qn, qh, kb, kn, kh, vb, vn, vh, ob, on, oh;  // bytes
  int B, M, heads, kv, group;  // query heads, cached heads, query heads a cached one
  const uint8_t* ck;
  const uint8_t* cv;
  const float* ks;
  const float* vs;
  int64_t pages;
  int page, shift;  // tokens of a page, their log2
  const int32_t* table;
  int64_t table_stride;
  int slots;  // pages of a table's row
  const int32_t* length;
  const uint64_t* mask;
  const int32_t* count;
  float scale2;  // scale log2(e)
  int tiles, splits;  // of 32 rows, of a cached head; parts of the cached tokens at most
  uint32_t items, group0;  // B * kv * splits
  FastDiv div_splits, div_kv, div_tiles, div_group;
  float* part;     // [B * kv * tiles][splits][32][D]
  float2* part_ml; // [B * kv * tiles][splits][32]
};

// How a query's cached tokens are parted: `used` splits of `per` tiles of 32 tokens.
struct Parts {
  int tokens, used, per;
};
__device__ inline Parts parts_of(const AttendArgs& A, int b) {
  Parts p;
  const int most = (int)min((int64_t)A.slots << A.shift, (int64_t)INT_MAX - 31);
  p.tokens = min(max(A.length[b], 0), most);
  const int tiles = (p.tokens + 31) / 32;
  const int n = min(max((tiles + kAttendLeast - 1) / kAttendLeast, 1), A.splits);
  p.per = max((tiles + n - 1) / n, 1);
  p.used = max((tiles + p.per - 1) / p.per, 1);
  return p;
}
__device__ inline int nodes_of(const AttendArgs& A, int b) {
  return A.count ? min(max(A.count[b], 0), A.M) : A.M;
}

template <bool F16>
struct Type {
  using V8 = bf16x8;
  using V2 = bf16x2;
};
template <>
struct Type<true> {
  using V8 = f16x8;
  using V2 = f16x2;
};
template <bool F16>
using V8 = typename Type<F16>::V8;

__device__ inline f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mfma(f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Eight codes as bf16 or fp16.
template <bool F16>
__device__ inline V8<F16> widen(uint32_t lo, uint32_t hi) {
  typename Type<F16>::V2 x[4];
  if constexpr (F16) {
    x[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
    x[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    x[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
    x[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  } else {
    x[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    x[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    x[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    x[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  }
  V8<F16> r;
  __builtin_memcpy(&r, x, 16);
  return r;
}

// Eight weights as fp16.
__device__ inline f16x8 narrow(const float* w) {
  f16x2 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __builtin_convertvector((f32x2{w[2 * i], w[2 * i + 1]}), f16x2);
  f16x8 r;
  __builtin_memcpy(&r, x, 16);
  return r;
}

// The token of a tile whose key is row rho of the first product: register i of lane half h is then token 16 h + i.
__device__ inline int pi_of(int rho) {
  return ((rho >> 2) & 1) * 16 + (rho >> 4) * 8 + ((rho >> 3) & 1) * 4 + (rho & 3);
}

__device__ inline float other_half(float x) { return __shfl_xor(x, 32, 64); }

// A tile of 32 cached tokens, as one wave holds it: lane (rho, h) dims 32 j + 16 h .. + 15 of the key of token
// pi(rho), and tokens 16 h .. 16 h + 15 of the dims 32 j + rho of the values.
template <int DB>
struct Tile {
  uint4 k[DB], v[DB];
  float ks, vs;
  int valid;
};

template <int DB>
__device__ inline void load_tile(const AttendArgs& A, int b, int h, int t, int tokens, int lane, Tile<DB>& T) {
  constexpr int D = 32 * DB;
  const int token = t * 32;
  int id = A.table[b * A.table_stride + (token >> A.shift)];
  T.valid = min(32, tokens - token);
  if (id < 0 || id >= A.pages) {  // no page: its tokens are not there
    T.valid = 0;
    id = 0;
  }
  const int64_t at = (int64_t)id * A.kv + h;
  const int off = token & (A.page - 1);
  T.ks = A.ks[at];
  T.vs = A.vs[at];
  const int rho = lane & 31, half = lane >> 5;
  const uint8_t* kp = A.ck + (at * A.page + off) * D;
  const uint8_t* vp = A.cv + at * A.page * D + off;
  const int ko = pi_of(rho) * D + 16 * half, vo = rho * A.page + 16 * half;
#pragma unroll
  for (int j = 0; j < DB; ++j) T.k[j] = *reinterpret_cast<const uint4*>(kp + (ko + 32 * j));
#pragma unroll
  for (int j = 0; j < DB; ++j) T.v[j] = *reinterpret_cast<const uint4*>(vp + (vo + 32 * j * A.page));
}

// A wave's running state of 32 rows: lane (r, h) has row r.
template <int DB>
struct State {
  f32x16 o[DB];  // o[j][i]: dim 32 j + 8 (i / 4) + 4 h + i % 4
  float m, l;    // l: this half's share
};

// x: scores plus the log2 of the values' scale. Leaves 2^12 weights in x, and O and l relative to the new m.
template <int DB>
__device__ inline void weigh(State<DB>& S, float (&x)[16]) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
  top = fmaxf(top, other_half(top));
  if (__ballot(top > S.m + kSlack)) {
    const float m = fmaxf(S.m, top), f = __builtin_amdgcn_exp2f(S.m - m);
    S.m = m;
    S.l *= f;
#pragma unroll
    for (int j = 0; j < DB; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) S.o[j][i] *= f;
  }
  const float from = S.m - kHeadroom;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(x[i] - from);
}

__device__ inline float sum16_of(const float (&w)[16]) {
  float a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = w[2 * i] + w[2 * i + 1];
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = a[2 * i] + a[2 * i + 1];
  return (a[0] + a[1]) + (a[2] + a[3]);
}

template <bool F16, int DB>
__device__ inline void attend_tile(const AttendArgs& A, const V8<F16> (&q)[2 * DB], Tile<DB>& T, int lane,
                                   State<DB>& S) {
  const int half = lane >> 5;
  f32x16 s = {};
#pragma unroll
  for (int j = 0; j < DB; ++j) {
    s = mfma(widen<F16>(T.k[j].x, T.k[j].y), q[2 * j], s);
    s = mfma(widen<F16>(T.k[j].z, T.k[j].w), q[2 * j + 1], s);
  }
  const float vs = fminf(fmaxf(T.vs, 0x1p-40f), 0x1p40f);
  const float f = A.scale2 * T.ks, bias = __builtin_amdgcn_logf(vs);
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = fmaf(s[i], f, bias);
  if (T.valid < 32) {  // what lies behind the last token has no weight, and its codes may be any
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (16 * half + i >= T.valid) x[i] = -INFINITY;
    uint32_t keep[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = min(max(T.valid - 16 * half - 4 * i, 0), 4);
      keep[i] = n == 4 ? ~0u : (1u << (8 * n)) - 1;
    }
#pragma unroll
    for (int j = 0; j < DB; ++j) {
      T.v[j].x &= keep[0];
      T.v[j].y &= keep[1];
      T.v[j].z &= keep[2];
      T.v[j].w &= keep[3];
    }
  }
  weigh<DB>(S, x);
  S.l = fmaf(sum16_of(x), 1.0f / vs, S.l);
  const f16x8 p0 = narrow(x), p1 = narrow(x + 8);
#pragma unroll
  for (int j = 0; j < DB; ++j) {
    S.o[j] = mfma(widen<true>(T.v[j].x, T.v[j].y), p0, S.o[j]);
    S.o[j] = mfma(widen<true>(T.v[j].z, T.v[j].w), p1, S.o[j]);
  }
}

__device__ inline bool not_finite16(uint32_t x, bool f16) {
  return f16 ? (x & 0x7C00u) == 0x7C00u : (x & 0x7F80u) == 0x7F80u;
}

// 32 nodes from `first` on, in their own type. bits: the nodes that the lane's row sees.
template <bool F16, int DB>
__device__ inline void attend_nodes(const AttendArgs& A, const V8<F16> (&q)[2 * DB], int b, int h, int first, int nodes,
                                    uint64_t bits, int lane, State<DB>& S) {
  const int rho = lane & 31, half = lane >> 5;
  const int mine = first + pi_of(rho);
  const char* kp = A.k + b * A.kb + h * A.kh + (mine < nodes ? mine : 0) * A.kn + 32 * half;
  f32x16 s = {};
#pragma unroll
  for (int j = 0; j < DB; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      s = mfma(*reinterpret_cast<const V8<F16>*>(kp + 64 * j + 16 * e), q[2 * j + e], s);
  float x[16];
  const uint32_t sees = (uint32_t)(bits >> (first + 16 * half)) & 0xFFFFu;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = (sees >> i) & 1 ? s[i] * A.scale2 : -INFINITY;
  weigh<DB>(S, x);
  S.l += sum16_of(x);
  // The nodes' values are fp16, or bf16, whose range fp16 lacks: the weights are then two bf16 (16 bits).
  V8<F16> p[2], rest[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if constexpr (F16) p[e] = narrow(x + 8 * e);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[e][i] = (__bf16)x[8 * e + i];
        rest[e][i] = (__bf16)(x[8 * e + i] - (float)p[e][i]);
      }
  }
  bool bad = false;
  const char* vp = A.v + b * A.vb + h * A.vh;
#pragma unroll
  for (int j = 0; j < DB; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint16_t y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int n = first + 16 * half + 8 * e + i;
        y[i] = 0;
        if (n < nodes) y[i] = *reinterpret_cast<const uint16_t*>(vp + n * A.vn + 2 * (32 * j + rho));
        if (not_finite16(y[i], F16)) {  // 0 times it is no 0: it is added below to the rows that see it
          bad = true;
          y[i] = 0;
        }
      }
      V8<F16> a;
      __builtin_memcpy(&a, y, 16);
      S.o[j] = mfma(a, p[e], S.o[j]);
      if constexpr (!F16) S.o[j] = mfma(a, rest[e], S.o[j]);
    }
  if (__ballot(bad)) {
    for (int n = first; n < min(first + 32, nodes); ++n) {
      const bool on = (bits >> n) & 1;
#pragma unroll
      for (int j = 0; j < DB; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int d = 32 * j + 8 * (i >> 2) + 4 * half + (i & 3);
          const uint16_t y = *reinterpret_cast<const uint16_t*>(vp + n * A.vn + 2 * d);
          if (on && not_finite16(y, F16))
            S.o[j][i] += F16 ? (float)__builtin_bit_cast(_Float16, y) : __uint_as_float((uint32_t)y << 16);
        }
    }
  }
}

template <bool F16>
__device__ inline void store4(char* p, f32x4 v) {
  typename Type<F16>::V2 x[2];
  x[0] = __builtin_convertvector((f32x2{v[0], v[1]}), typename Type<F16>::V2);
  x[1] = __builtin_convertvector((f32x2{v[2], v[3]}), typename Type<F16>::V2);
  *reinterpret_cast<uint2*>(p) = make_uint2(__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]));
}

template <bool F16, int DB>
__global__ void __launch_bounds__(kThreads) hs_attend_kernel(const AttendArgs A) {
  constexpr int D = 32 * DB, kPitch = D + 4;
  __shared__ __attribute__((aligned(16))) float s_o[2][32 * kPitch];
  __shared__ float s_m[kWaves][32], s_l[kWaves][32];
  const int lane = threadIdx.x & 63, wv = (int)uniform(threadIdx.x >> 6);
  const int rho = lane & 31, half = lane >> 5;
  // eight items, then the next row tile of the same eight: an XCD reads an item's pages once
  const uint32_t g = A.group0 + blockIdx.x, eight = g >> 3, lot = fdiv(eight, A.div_tiles);
  const int tile = (int)(eight - lot * (uint32_t)A.tiles);
  const uint32_t item = lot * 8 + (g & 7);
  if (item >= A.items) return;
  const uint32_t bh = fdiv(item, A.div_splits);
  const int split = (int)(item - bh * (uint32_t)A.splits);
  const int b = (int)fdiv(bh, A.div_kv), h = (int)bh - b * A.kv;
  const int nodes = nodes_of(A, b), rows = nodes * A.group;
  if (tile * 32 >= rows) return;
  const Parts P = parts_of(A, b);
  if (split >= P.used) return;

  const int row = tile * 32 + rho;
  const bool live = row < rows;
  const int node = live ? (int)fdiv((uint32_t)row, A.div_group) : 0, head = h * A.group + (live ? row - node * A.group : 0);
  V8<F16> q[2 * DB];
  const char* qp = A.q + b * A.qb + node * A.qn + head * A.qh + 32 * half;
#pragma unroll
  for (int j = 0; j < DB; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint4 x = *reinterpret_cast<const uint4*>(qp + 64 * j + 16 * e);
      if (!live) x = make_uint4(0, 0, 0, 0);
      __builtin_memcpy(&q[2 * j + e], &x, 16);
    }
  State<DB> S;
#pragma unroll
  for (int j = 0; j < DB; ++j) S.o[j] = f32x16{};
  S.m = kLowest;
  S.l = 0.0f;

  const int last = min((P.tokens + 31) / 32, (split + 1) * P.per);
  int t = split * P.per + wv;
  Tile<DB> one, two;
  if (t < last) load_tile<DB>(A, b, h, t, P.tokens, lane, one);
  while (t < last) {
    if (t + kWaves < last) load_tile<DB>(A, b, h, t + kWaves, P.tokens, lane, two);
    attend_tile<F16, DB>(A, q, one, lane, S);
    t += kWaves;
    if (t >= last) break;
    if (t + kWaves < last) load_tile<DB>(A, b, h, t + kWaves, P.tokens, lane, one);
    attend_tile<F16, DB>(A, q, two, lane, S);
    t += kWaves;
  }
  if (split == P.used - 1 && wv < 2 && wv * 32 < nodes) {  // the last split has the nodes too
    uint64_t bits = 0;
    if (live) {
      bits = A.mask ? A.mask[(int64_t)b * A.M + node] : (2ull << node) - 1;
      if (nodes < 64) bits &= (1ull << nodes) - 1;
    }
    attend_nodes<F16, DB>(A, q, b, h, wv * 32, nodes, bits, lane, S);
  }
  S.l += other_half(S.l);

  // the waves' states, joined
  if (half == 0) {
    s_m[wv][rho] = S.m;
    s_l[wv][rho] = S.l;
  }
  __syncthreads();
  float m = s_m[0][rho], l = 0.0f;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m = fmaxf(m, s_m[w][rho]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) l = fmaf(s_l[w][rho], __builtin_amdgcn_exp2f(s_m[w][rho] - m), l);
  const float f = __builtin_amdgcn_exp2f(S.m - m);
#pragma unroll
  for (int j = 0; j < DB; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) S.o[j][i] *= f;
#pragma unroll
  for (int step = 0; step < 2; ++step) {  // waves 2 and 3 to 0 and 1, then 1 to 0
    const int from = step == 0 ? 2 : 1;
    if (wv >= from && wv < 2 * from) {
      float* to = &s_o[wv - from][rho * kPitch + 4 * half];
#pragma unroll
      for (int j = 0; j < DB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(to + 32 * j + 8 * i) =
              f32x4{S.o[j][4 * i], S.o[j][4 * i + 1], S.o[j][4 * i + 2], S.o[j][4 * i + 3]};
    }
    __syncthreads();
    if (wv < from) {
      const float* at = &s_o[wv][rho * kPitch + 4 * half];
#pragma unroll
      for (int j = 0; j < DB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 y = *reinterpret_cast<const f32x4*>(at + 32 * j + 8 * i);
#pragma unroll
          for (int k = 0; k < 4; ++k) S.o[j][4 * i + k] += y[k];
        }
    }
    __syncthreads();
  }
  if (wv != 0) return;
  const int64_t slot = ((int64_t)bh * A.tiles + tile) * A.splits + split;
  if (P.used == 1) {
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;  // (a NaN stays)
    if (live) {
      char* op = A.out + b * A.ob + node * A.on + head * A.oh + 8 * half;
#pragma unroll
      for (int j = 0; j < DB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          store4<F16>(op + 64 * j + 16 * i, f32x4{S.o[j][4 * i] * inv, S.o[j][4 * i + 1] * inv,
                                                  S.o[j][4 * i + 2] * inv, S.o[j][4 * i + 3] * inv});
    }
    return;
  }
  if (!live) return;
  float* op = A.part + (slot * 32 + rho) * D + 4 * half;
#pragma unroll
  for (int j = 0; j < DB; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(op + 32 * j + 8 * i) =
          f32x4{S.o[j][4 * i], S.o[j][4 * i + 1], S.o[j][4 * i + 2], S.o[j][4 * i + 3]};
  if (half == 0) A.part_ml[slot * 32 + rho] = make_float2(m, l);
}

// A wave a row: its splits, joined.
template <bool F16, int DB>
__global__ void __launch_bounds__(kThreads) hs_attend_join_kernel(const AttendArgs A) {
  constexpr int D = 32 * DB;
  const int lane = threadIdx.x & 63;
  const uint32_t u = uniform((A.group0 + blockIdx.x) * kWaves + (threadIdx.x >> 6));
  const uint32_t bt = u >> 5;  // (query, cached head, tile)
  if (bt >= (uint32_t)A.B * (uint32_t)A.kv * (uint32_t)A.tiles) return;
  const uint32_t bh = fdiv(bt, A.div_tiles);
  const int tile = (int)(bt - bh * (uint32_t)A.tiles);
  const int b = (int)fdiv(bh, A.div_kv), h = (int)bh - b * A.kv;
  const int row = tile * 32 + (int)(u & 31);
  if (row >= nodes_of(A, b) * A.group) return;
  const int used = parts_of(A, b).used;
  if (used == 1) return;
  const int64_t slot = (int64_t)bt * A.splits;
  const float2* ml = A.part_ml + slot * 32 + (u & 31);
  float m = kLowest;
  for (int s = 0; s < used; ++s) m = fmaxf(m, ml[s * 32].x);
  float l = 0.0f, o[(D + 63) / 64] = {};
  for (int s = 0; s < used; ++s) {
    const float2 y = ml[s * 32];
    const float f = __builtin_amdgcn_exp2f(y.x - m);
    l = fmaf(y.y, f, l);
    const float* p = A.part + ((slot + s) * 32 + (u & 31)) * D;
#pragma unroll
    for (int i = 0; i < (D + 63) / 64; ++i)
      if (i * 64 + lane < D) o[i] = fmaf(p[i * 64 + lane], f, o[i]);
  }
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  const int node = (int)fdiv((uint32_t)row, A.div_group), head = h * A.group + row - node * A.group;
  char* op = A.out + b * A.ob + node * A.on + head * A.oh;
#pragma unroll
  for (int i = 0; i < (D + 63) / 64; ++i)
    if (i * 64 + lane < D) {
      const float y = o[i] * inv;
      if constexpr (F16) reinterpret_cast<_Float16*>(op)[i * 64 + lane] = (_Float16)y;
      else reinterpret_cast<__bf16*>(op)[i * 64 + lane] = (__bf16)y;
    }
}

template <bool F16, int DB>
void launch_dim(AttendArgs A, hipStream_t st) {
  const uint64_t groups = ((uint64_t)A.items + 7) / 8 * 8 * A.tiles;
  for (uint64_t at = 0; at < groups; at += kMostGroups) {
    A.group0 = (uint32_t)at;
    hs_attend_kernel<F16, DB><<<(uint32_t)std::min<uint64_t>(groups - at, kMostGroups), kThreads, 0, st>>>(A);
    if (hipPeekAtLastError() != hipSuccess) return;
  }
  if (A.splits == 1) return;
  const uint64_t joins = (uint64_t)A.B * A.kv * A.tiles * 32 / kWaves;
  for (uint64_t at = 0; at < joins; at += kMostGroups) {
    A.group0 = (uint32_t)at;
    hs_attend_join_kernel<F16, DB><<<(uint32_t)std::min<uint64_t>(joins - at, kMostGroups), kThreads, 0, st>>>(A);
    if (hipPeekAtLastError() != hipSuccess) return;
  }
}

template <bool F16>
void launch_type(const AttendArgs& A, int dim, hipStream_t st) {
  switch (dim / 32) {
    case 1: return launch_dim<F16, 1>(A, st);
    case 2: return launch_dim<F16, 2>(A, st);
    case 3: return launch_dim<F16, 3>(A, st);
    case 4: return launch_dim<F16, 4>(A, st);
    case 5: return launch_dim<F16, 5>(A, st);
    case 6: return launch_dim<F16, 6>(A, st);
    case 7: return launch_dim<F16, 7>(A, st);
    default: return launch_dim<F16, 8>(A, st);
  }
}

}  // namespace

bool attend_geom(int B, int M, int heads, int kv, int dim, int page, int slots, AttendGeom* g) {
  if (B < 1 || M < 1 || heads < 1 || kv < 1 || slots < 1) return false;
  if (B > HS_MAX_QUERIES || M > HS_MAX_POSITIONS || heads > HS_MAX_HEADS || heads % kv != 0) return false;
  if (dim < 32 || dim > HS_MAX_HEAD_DIM || dim % 32 != 0) return false;
  if (page < 32 || page > HS_MAX_PAGE || (page & (page - 1)) != 0) return false;
  g->B = B;
  g->M = M;
  g->heads = heads;
  g->kv = kv;
  g->dim = dim;
  g->tiles = (M * (heads / kv) + 31) / 32;
  const int64_t groups = (int64_t)B * kv * g->tiles, most = ((int64_t)slots * page + 31) / 32;
  const int64_t want = (1024 + groups - 1) / groups, can = (most + kAttendLeast - 1) / kAttendLeast;
  g->splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, can), 128));
  return groups * g->splits < ((int64_t)1 << 31);
}

size_t attend_ws_bytes(const AttendGeom& g) {
  if (g.splits == 1) return 0;
  const size_t slots = (size_t)g.B * g.kv * g.tiles * g.splits * 32;
  return align256(slots * g.dim * sizeof(float)) + align256(slots * sizeof(float2));
}

int launch_attend(const AttendGeom& g, const hs_tree_attention_args& a, hipStream_t stream) {
  AttendArgs A;
  A.q = reinterpret_cast<const char*>(a.q.ptr);
  A.k = reinterpret_cast<const char*>(a.k.ptr);
  A.v = reinterpret_cast<const char*>(a.v.ptr);
  A.out = reinterpret_cast<char*>(a.out.ptr);
  A.qb = 2 * a.q.stride_b, A.qn = 2 * a.q.stride_n, A.qh = 2 * a.q.stride_h;
  A.kb = 2 * a.k.stride_b, A.kn = 2 * a.k.stride_n, A.kh = 2 * a.k.stride_h;
  A.vb = 2 * a.v.stride_b, A.vn = 2 * a.v.stride_n, A.vh = 2 * a.v.stride_h;
  A.ob = 2 * a.out.stride_b, A.on = 2 * a.out.stride_n, A.oh = 2 * a.out.stride_h;
  A.B = g.B;
  A.M = g.M;
  A.heads = g.heads;
  A.kv = g.kv;
  A.group = g.heads / g.kv;
  A.ck = reinterpret_cast<const uint8_t*>(a.cache.k);
  A.cv = reinterpret_cast<const uint8_t*>(a.cache.v);
  A.ks = a.cache.k_scale;
  A.vs = a.cache.v_scale;
  A.pages = a.cache.pages;
  A.page = a.cache.page;
  A.shift = __builtin_ctz((unsigned)a.cache.page);
  A.table = a.table;
  A.table_stride = a.table_stride;
  A.slots = a.slots;
  A.length = a.length;
  A.mask = a.mask;
  A.count = a.count;
  A.scale2 = (float)(a.scale * 1.4426950408889634074);
  A.tiles = g.tiles;
  A.splits = g.splits;
  A.items = (uint32_t)((int64_t)g.B * g.kv * g.splits);
  A.div_splits = make_fastdiv((uint32_t)g.splits);
  A.div_kv = make_fastdiv((uint32_t)g.kv);
  A.div_tiles = make_fastdiv((uint32_t)g.tiles);
  A.div_group = make_fastdiv((uint32_t)A.group);
  const size_t slots = (size_t)g.B * g.kv * g.tiles * g.splits * 32;
  A.part = reinterpret_cast<float*>(a.workspace);
  A.part_ml = reinterpret_cast<float2*>(reinterpret_cast<char*>(a.workspace) +
                                        align256(slots * g.dim * sizeof(float)));
  if (a.dtype == HS_F16) launch_type<true>(A, g.dim, stream);
  else launch_type<false>(A, g.dim, stream);
  return hipPeekAtLastError() == hipSuccess ? HS_OK : HS_ERR_HIP;
}

}  // namespace hs
