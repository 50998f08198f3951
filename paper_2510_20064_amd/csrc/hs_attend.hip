// hs_tree_attention: the queries of a draft's nodes over a cache held in 8 bits and over the nodes on their paths.
//
// A query's rows r are its nodes' query heads that share a cached head; with s_rt = scale log2(e) ks_t (q_r . k_t),
// ks and vs the scales of t's page,
//   o_r = sum_t p_rt vs_t v_t / sum_t p_rt,   p_rt = 2^(s_rt - m_r).
// The values' scales go into the weights: with x_rt = s_rt + log2 vs_t, w_rt = 2^(x_rt - m_r) and m_r following the
// largest x, o_r = sum w v / sum w / vs.
//
// Layout. Products are S^T = K Q^T and O^T = V^T P^T, so that a row's scores, weights, maximum and sum all stay in the
// lanes that hold its column, and the weights are the second product's operand as they stand: the scores' registers of a
// lane are consecutive tokens of a tile of 32 if the tile's K rows are taken in the order of row_of. A page holds its
// values by dimension, so those tokens of one dimension are 16 (8) bytes in a row. Tiles are 32 x 32 x 16 with 32 rows a
// wave, or 16 x 16 x 32 with 16 for up to 16 rows: a third less registers and half the exponentials, three waves a SIMD
// where there are two (32 single tokens over 16 thousand: 128 us and 118 to 120; four waves spill, 187; two, 118, lose on
// short caches).
// A workgroup brings stages of four tiles to LDS, the next one on its way to registers: its waves share a stage's rows of
// queries or its tiles. From memory to registers without LDS, each wave its own tiles, a load of keys took 32 bytes of 32
// lines (61 nodes over 16 thousand tokens 101 us and 46, 32 such over 8 thousand 509 and 230).
// Codes of 8 bits become bf16 or fp16 without error (3 bits of mantissa, 2^-9 to 448), one instruction for two.
// Weights are rounded to fp16 (relative 2^-11, an eighth of a bf16 output's own rounding), as 2^12 w, so that what is lost lies
// below 2^-36 of the largest x and not below 2^-24; m follows only in steps above 2^3 (w stays
// below 2^16), which spares most tiles the multiplication of O. Sums and O are fp32.
// m follows x whatever a page's codes are, so a page whose scale an outlier set would take fp16's range from pages of finer
// scales. While a tile whose scale is more than 2^kSpread below the largest met is added, O and its weights are held larger,
// and also while one of scores beyond 2^22 is, whose products are rounded first (see lifted). Nodes' values have no scale: m
// follows them as if it were 2^kNodes, so that pages down to 2^-21 are no finer ones, and their weights, which that makes
// larger than fp16, are two bf16 each. That costs tiles that need none of it 3 to 6% (one query's tree 41.4 us and 42.6, 32
// trees 198 and 207 to 210, fp16 nodes of short drafts 15.0 and 15.9, a token 13.2 and 13.6) and trees whose tiles all do
// up to twice the time (64.8, 371; a token 14.1). Weights as two bf16 for all, whose range is fp32's: 47.3, 249, 15.9 and
// 13.3. kSpread trades what fp16 loses, 2^(kSpread - 37) of the largest weight, for pages that take the longer way: values
// of one distribution have scales 4 times apart, and pages of 8 times the values 32; with 4 for it those made 258 us of 201.
//
// Split. The stages of all queries' cached tokens are cut into as many equal ranges as the device holds workgroups, so that
// lengths that differ, and one query alone, load it alike; what a range holds of a query that others share goes to the
// workspace, and hs_attend_join_kernel adds the parts in their order. See attend_geom for when a query is a workgroup's
// instead. Nodes do not count: the range with a query's end has up to 64 of them too, and with few stages a range (one tree
// over 16 thousand: four) sets the time.
//
// What bounds it, heads of 128, eight cached for 32. One token over 512: two launches and four dependent reads (length,
// table, scales, codes), 13.6 us. 32 tokens over up to 16 thousand, 537 MB: the memory, 115 to 118 us with the join's 5.4,
// 4.6 TB/s, where a large copy reaches 4.8. 32 trees of 61 nodes over up to 8 thousand, 131 GFLOP: 200 to 210 us with the
// join's 16 in a run of calls (245 from an idle card), 0.64 PFLOP/s, where a large product reaches 1.4: the matrix units are
// busy 29% of the time, the vector units 42% (161 instructions a wave and tile), LDS 25%, and a wave waits 50% of its time,
// which the second wave that the registers leave a SIMD fills half. No part took more than an eighth when it was left out. No
// gain: the next
// tile's scores before this one's weights, a product's operands read under the softmax before it, two buffers and one
// barrier a stage, other wave priorities, the values' loads before the softmax;
// 64 rows a wave spill.
#include <algorithm>
#include <cfloat>

#include "hs_draft.h"

namespace hs {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kHeadroom = 12.0f;  // weights are held as 2^12 w
constexpr float kSlack = 3.0f;      // m follows a maximum more than this above it
constexpr float kLowest = -FLT_MAX; // m before the first token
constexpr float kSpread = 5.0f;     // log2 of how far a page's scale may be below others'
constexpr float kNodes = -16.0f;    // log2 of the scale that m takes nodes' values to have
constexpr float kHugeNodes = 24.0f; // and where some are 2^90 or more: 64 of the largest at weights of 2^(15 - 24) are fp32
constexpr int kStage = 4;           // tiles of 32 tokens that a workgroup brings to LDS at once

// Waves of a SIMD, by the registers that they take.
constexpr int waves_of(int rw, int dim) { return dim > 128 ? rw == 16 ? 2 : 1 : rw == 16 ? 3 : 2; }

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
  int tiles;   // workgroups that share a cached head's rows
  int chunks;  // ranges that all queries' cached tokens are cut into; 0: a query is one
  uint32_t items, group0;  // (ranges, or queries) * kv
  uint32_t row_tiles;      // 32 (16) rows of a query's cached head
  FastDiv div_kv, div_tiles, div_group, div_rows;
  float* part;      // [kv * tiles][2 * chunks][WR][groups of a State][64 lanes][4]
  float2* part_ml;  // [kv * tiles][2 * chunks][WR][32 or 16 rows]
};

__device__ inline int same(int x) { return (int)uniform((uint32_t)x); }  // (what every lane has, in a scalar register)
__device__ inline int tokens_of(const AttendArgs& A, int b) {
  return min(max(A.length[b], 0), (int)min((int64_t)A.slots << A.shift, (int64_t)INT_MAX));
}
// Stages of a query's cached tokens; one without tokens counts for one. (Up to 2^31 - 1 tokens: rounded up without sign,
// here and where tokens are counted in tiles.)
__device__ inline int stages_of(const AttendArgs& A, int b) {
  return max((int)(((uint32_t)tokens_of(A, b) + 32 * kStage - 1) / (32 * kStage)), 1);
}
// The stages of all queries, one behind the other, are cut into ranges of `per`: a workgroup does a range, and a query
// may lie in several, whose parts the join adds. Range i has up to two parts of such queries: place 2 i is that of the
// query with which the range starts, 2 i + 1 that of one that starts inside it.
// One wave; a lane has the queries from lane * held on.
struct Plan {
  int per, held, upto, mine;  // upto: stages of the lanes up to and with this one, mine: this one's
  __device__ Plan(const AttendArgs& A, int lane) {
    held = (A.B + 63) / 64;
    mine = 0;
    for (int i = lane * held; i < min((lane + 1) * held, A.B); ++i) mine += stages_of(A, i);
    upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(upto, d, 64);
      if (lane >= d) upto += o;
    }
    const int all = __builtin_amdgcn_readlane(upto, 63);
    per = same((all + A.chunks - 1) / A.chunks);
  }
  // The query that stage `at` of all lies in, and the stages before it; -1: none.
  __device__ int query(const AttendArgs& A, int at, int* before) const {
    const uint64_t over = __ballot(upto > at);
    if (!over) return -1;
    const int l = __builtin_ctzll(over);
    int n = __builtin_amdgcn_readlane(upto - mine, l), b = l * held;
    for (;; ++b) {
      const int w = same(stages_of(A, b));
      if (at < n + w) break;
      n += w;
    }
    *before = n;
    return b;
  }
  __device__ int before(const AttendArgs& A, int b) const {
    const int l = b / held;
    int n = __builtin_amdgcn_readlane(upto - mine, l);
    for (int i = l * held; i < b; ++i) n += same(stages_of(A, i));
    return n;
  }
};
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

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
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

// Eight weights as two bf16 each, whose sum is good to 2^-16 of the weight: its upper 16 bits, and what they leave out,
// rounded.
struct Weights {
  bf16x8 hi, lo;
  __device__ explicit Weights(const float* w) {
    uint32_t u[4];
    bf16x2 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = __float_as_uint(w[2 * i]), b = __float_as_uint(w[2 * i + 1]);
      u[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      const f32x2 rest = {w[2 * i] - __uint_as_float(a & 0xFFFF0000u), w[2 * i + 1] - __uint_as_float(b & 0xFFFF0000u)};
      x[i] = __builtin_convertvector(rest, bf16x2);
    }
    __builtin_memcpy(&hi, u, 16);
    __builtin_memcpy(&lo, x, 16);
  }
};

// Eight fp16 values as sums of two bf16, exactly: of their 11 bits the upper 8, and the rest.
struct Parts {
  bf16x8 hi, lo;
  __device__ explicit Parts(u32x4 y) {
    uint32_t u[4], r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = y[i];  // (a bit cast of a vector's element itself takes the first)
      const f16x2 h = __builtin_bit_cast(f16x2, w);
      const float a = (float)h[0], b = (float)h[1];
      const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
      u[i] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
      r[i] = __builtin_amdgcn_perm(__float_as_uint(b - __uint_as_float(ub & 0xFFFF0000u)),
                                   __float_as_uint(a - __uint_as_float(ua & 0xFFFF0000u)), 0x07060302u);
    }
    __builtin_memcpy(&hi, u, 16);
    __builtin_memcpy(&lo, r, 16);
  }
};

// The row of a token's key in its tile, so that a lane's scores are consecutive tokens: of 32 rows register i of lane half
// h is token 16 h + i, of 16 rows register i of product a and lane quarter g token 8 g + 4 a + i.
template <int RW>
__device__ inline int row_of(int token) {
  if constexpr (RW == 32)
    return ((token >> 4) & 1) * 4 + ((token >> 3) & 1) * 16 + ((token >> 2) & 1) * 8 + (token & 3);
  else return ((token >> 2) & 1) * 16 + (token >> 3) * 4 + (token & 3);
}

// The largest value, and the sum, of the lanes that have a row: l and l + 32, or of 16 rows also l + 16 and l + 48.
struct Pair {
  float a, b;
};
__device__ inline Pair halves(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return Pair{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ inline Pair quarters(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return Pair{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
template <int RW>
__device__ inline float row_max(float x) {
  const Pair p = halves(x);
  x = fmaxf(p.a, p.b);
  if constexpr (RW == 16) {
    const Pair q = quarters(x);
    x = fmaxf(q.a, q.b);
  }
  return x;
}
template <int RW>
__device__ inline float row_sum(float x) {
  const Pair p = halves(x);
  x = p.a + p.b;
  if constexpr (RW == 16) {
    const Pair q = quarters(x);
    x = q.a + q.b;
  }
  return x;
}

// The pages of the tiles of stage t, lane i that of tile i, or -1. (By a vector load like the scales below: a scalar
// one would be in the count that the wait for each read of LDS brings to 0.)
__device__ inline int pages_of(const AttendArgs& A, int b, int t, int last, int lane) {
  const int id = lane < kStage && t + lane < last ? A.table[b * A.table_stride + (((t + lane) * 32) >> A.shift)] : -1;
  return id < A.pages ? id : -1;
}
// The scales of the tiles of a stage: lane i the keys' of tile i, lane kStage + i the values'; 1 where there is no tile,
// whose products are computed like the others'. (Its codes are read from the first page, below, and not used.)
__device__ inline float scales_of(const AttendArgs& A, int h, int pages, int lane) {
  const int id = __shfl(pages, lane & (kStage - 1), 64);
  return lane < 2 * kStage && id >= 0 ? (lane < kStage ? A.ks : A.vs)[(int64_t)id * A.kv + h] : 1.0f;
}
// And with the keys' times the products' own, finite: infinite times a product of 0 is no 0. (Apart, for it waits.)
__device__ inline float factors_of(const AttendArgs& A, float scales, int lane) {
  const float f = scales * A.scale2;
  return lane < kStage ? fabsf(f) == INFINITY ? copysignf(FLT_MAX, f) : f : scales;
}
// Tokens of a stage's tile that there are.
__device__ inline int valid_of(int pages, int t, int sub, int tokens) {
  return __builtin_amdgcn_readlane(pages, sub) < 0 ? 0 : min(32, max(tokens - (t + sub) * 32, 0));
}

// A stage on its way to LDS. A tile's keys are 32 * D bytes one behind the other, its values D rows of 32 bytes; a wave
// brings pieces of 1 KB of both. In LDS a row is 16 bytes longer than what it holds: an odd number of 16 bytes, so that 16
// lanes that read 16 bytes of consecutive rows each use all banks once. WIDE, where each of eight waves reads every tile:
// the codes are widened on the way to LDS, once instead of by each wave (32 trees of 61 nodes 230 us and 219, at twice
// the bytes; with four waves no gain).
template <int DB, bool WIDE>
struct Staged {
  static constexpr int kCode = WIDE ? 2 : 1;  // bytes
  static constexpr int kKeyPitch = 32 * DB * kCode + 16, kValuePitch = 32 * kStage * kCode + 16;
  static constexpr int kKeys = 32 * kStage * kKeyPitch, kBytes = kKeys + 32 * DB * kValuePitch;
};
template <int DB, int NW>
struct Loads {
  static constexpr int kAll = kStage * DB, kN = (kAll + NW - 1) / NW;  // pieces of a stage's keys; of a wave
  u32x4 k[kN], v[kN];
};
template <int DB, int NW>
__device__ __forceinline__ void load_stage(const AttendArgs& A, int h, int t, int pages, int wv, int lane,
                                           Loads<DB, NW>& L) {
  constexpr int D = 32 * DB;
  const uint32_t ko = 16 * lane, vo = (lane >> 1) * A.page + 16 * (lane & 1);
#pragma unroll
  for (int i = 0; i < L.kN; ++i) {
    const int piece = min(wv + NW * i, L.kAll - 1), sub = piece / DB, part = piece - sub * DB;
    const int id = max(__builtin_amdgcn_readlane(pages, sub), 0), off = (int)(((uint32_t)(t + sub) * 32) & (uint32_t)(A.page - 1));
    const int64_t at = ((int64_t)id * A.kv + h) * A.page;
    L.k[i] = *reinterpret_cast<const u32x4*>(A.ck + (at + off) * D + part * 1024 + ko);
    L.v[i] = *reinterpret_cast<const u32x4*>(A.cv + at * D + off + part * 32 * A.page + vo);
  }
}
__device__ inline bool is_zero(float x) { return __float_as_uint(x) << 1 == 0; }  // (+-0, by scalar instructions)
// Of 16 codes those that are NaN, 0 for others.
__device__ inline u32x4 nans_of(u32x4 x) {
  asm volatile("");  // (a branch, not selects for every tile)
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] &= (((x[e] & 0x7F7F7F7Fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xFFu;
  return x;
}
// pages, t, tokens, scales: of the stage. What lies behind the last token may be any code: its values are held as 0. So are
// codes of a page whose scale is 0, but for NaN: a page's weights count as if its values' were 2^-40, and products as if its
// keys' were 1 (infinite ones, which get no weight, stay so).
template <bool F16, int RW, int DB, int NW, bool WIDE>
__device__ __forceinline__ void store_stage(uint8_t* lds, int t, int pages, int tokens, float scales, int wv, int lane,
                                            Loads<DB, NW>& L) {
  using St = Staged<DB, WIDE>;
#pragma unroll
  for (int i = 0; i < L.kN; ++i) {
    const int piece = wv + NW * i, sub = piece / DB, part = piece - sub * DB;
    if (L.kAll % NW != 0 && piece >= L.kAll) continue;
    const int valid = valid_of(pages, t, sub, tokens);
    if (valid < 32) {
      asm volatile("");  // (a branch, not selects for every tile)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = min(max(valid - 16 * (lane & 1) - 4 * e, 0), 4);
        L.v[i][e] &= c == 4 ? ~0u : (1u << (8 * c)) - 1;
      }
    }
    if (is_zero(lane_f(scales, kStage + sub))) L.v[i] = nans_of(L.v[i]);
    if (is_zero(lane_f(scales, sub))) L.k[i] = nans_of(L.k[i]);
    const int q = part * 64 + lane, token = q / (2 * DB), c = q - token * (2 * DB);
    uint8_t* kp = lds + (32 * sub + row_of<RW>(token)) * St::kKeyPitch + 16 * c * St::kCode;
    uint8_t* vp = lds + St::kKeys + (32 * part + (lane >> 1)) * St::kValuePitch + (32 * sub + 16 * (lane & 1)) * St::kCode;
    if constexpr (WIDE) {
      reinterpret_cast<V8<F16>*>(kp)[0] = widen<F16>(L.k[i].x, L.k[i].y);
      reinterpret_cast<V8<F16>*>(kp)[1] = widen<F16>(L.k[i].z, L.k[i].w);
      reinterpret_cast<f16x8*>(vp)[0] = widen<true>(L.v[i].x, L.v[i].y);
      reinterpret_cast<f16x8*>(vp)[1] = widen<true>(L.v[i].z, L.v[i].w);
    } else {
      *reinterpret_cast<u32x4*>(kp) = L.k[i];
      *reinterpret_cast<u32x4*>(vp) = L.v[i];
    }
  }
}
// Sixteen staged codes, as two operands.
template <bool F16, bool WIDE>
__device__ __forceinline__ void operands(const uint8_t* at, V8<F16> (&x)[2]) {
  if constexpr (WIDE) {
    x[0] = reinterpret_cast<const V8<F16>*>(at)[0];
    x[1] = reinterpret_cast<const V8<F16>*>(at)[1];
  } else {
    const u32x4 c = *reinterpret_cast<const u32x4*>(at);
    x[0] = widen<F16>(c.x, c.y);
    x[1] = widen<F16>(c.z, c.w);
  }
}

// A wave's running state of RW = 32 or 16 rows: lane (r, c), l = RW c + r, has row r; O in groups of four dims, group n
// those from kDims n + 4 c on.
template <int DB, int RW>
struct State {
  static constexpr int kGroups = DB * RW / 8, kDims = 256 / RW;
  f32x16 o32[RW == 32 ? DB : 1];
  f32x4 o16[RW == 16 ? 2 * DB : 1];
  float m, l;  // l: this lane's share
  float base;  // log2 of the largest scale of values met
  __device__ f32x4 get(int n) const {
    if constexpr (RW == 16) return o16[n];
    else return f32x4{o32[n / 4][n % 4 * 4], o32[n / 4][n % 4 * 4 + 1], o32[n / 4][n % 4 * 4 + 2], o32[n / 4][n % 4 * 4 + 3]};
  }
  __device__ void set(int n, f32x4 v) {
    if constexpr (RW == 16) o16[n] = v;
    else
#pragma unroll
      for (int k = 0; k < 4; ++k) o32[n / 4][n % 4 * 4 + k] = v[k];
  }
  __device__ void clear() {
#pragma unroll
    for (int n = 0; n < kGroups; ++n) set(n, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
    m = kLowest;
    l = 0.0f;
    base = -INFINITY;
  }
  __device__ void scale(float f) {
#pragma unroll
    for (int n = 0; n < kGroups; ++n) set(n, get(n) * f);
  }
};

// m, and O and l with it, after scores (plus the log2 of the values' scale) of which the lane's largest is `top`. What
// weights are relative to: 2^12 w = 2^(x - that).
template <int DB, int RW>
__device__ inline float follow(State<DB, RW>& S, float top) {
  top = row_max<RW>(top);
  if (__ballot(top > S.m + kSlack)) {
    const float m = fmaxf(S.m, top), f = __builtin_amdgcn_exp2f(S.m - m);
    S.m = m;
    S.l *= f;
    S.scale(f);
  }
  return S.m - kHeadroom;
}
template <int N>
__device__ inline float max_of(const float (&x)[N]) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
  return top;
}
template <int N>
__device__ inline float sum_of(const float (&w)[N]) {
  float a[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) a[i] = w[2 * i] + w[2 * i + 1];
  if constexpr (N > 2) return sum_of(a);
  else return a[0];
}

// A lane's products of a tile: those of its row with RW / 2 tokens, the first of which is RW / 2 times its part of the wave.
template <int RW>
struct Scores {
  f32x16 a{};
  __device__ float at(int i) const { return a[i]; }
  __device__ void set(int i, float x) { a[i] = x; }
};
template <>
struct Scores<16> {
  f32x4 a[2]{};
  __device__ float at(int i) const { return a[i / 4][i % 4]; }
  __device__ void set(int i, float x) { a[i / 4][i % 4] = x; }
};
// A tile of the stage in LDS: its tokens, the factor of its products, log2 of its values' scale and what a weight counts for in
// the sum; the largest score's product, and that score with the scale.
struct Tile {
  int valid;
  float f, bias, inv, best, top;
};
// The products of N tiles from the `sub`-th on, which do not wait for each other.
template <bool F16, int DB, int RW, bool WIDE, int N, int NQ>
__device__ __forceinline__ void multiply(const V8<F16> (&q)[NQ], const uint8_t* lds, int sub, const int (&valid)[N],
                                         float scales, int lane, Scores<RW> (&s)[N], Tile (&t)[N]) {
  using St = Staged<DB, WIDE>;
  const int rho = lane % RW, c = lane / RW;
  const uint8_t* kp = lds + (32 * sub + rho) * St::kKeyPitch + RW / 2 * c * St::kCode;
#pragma unroll
  for (int j = 0; j < DB; ++j)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if constexpr (RW == 32) {
        V8<F16> k[2];
        operands<F16, WIDE>(kp + 32 * n * St::kKeyPitch + 32 * j * St::kCode, k);
        s[n].a = mfma(k[0], q[2 * j], s[n].a);
        s[n].a = mfma(k[1], q[2 * j + 1], s[n].a);
      } else {
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const u32x2 k = *reinterpret_cast<const u32x2*>(kp + (32 * n + 16 * a) * St::kKeyPitch + 32 * j);
          s[n].a[a] = mfma(widen<F16>(k.x, k.y), q[j], s[n].a[a]);
        }
      }
    }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const float vs = fminf(fmaxf(lane_f(scales, kStage + sub + n), 0x1p-40f), 0x1p40f);
    t[n].valid = valid[n];
    t[n].f = lane_f(scales, sub + n);
    t[n].bias = __builtin_amdgcn_logf(vs);
    t[n].inv = __builtin_amdgcn_rcpf(vs);
    if (valid[n] < 32) {  // what lies behind the last token has no weight
      asm volatile("");   // (a branch, not selects for every tile)
      const float none = t[n].f < 0.0f ? INFINITY : -INFINITY;
#pragma unroll
      for (int i = 0; i < RW / 2; ++i) s[n].set(i, RW / 2 * c + i < valid[n] ? s[n].at(i) : none);
    }
    float hi = s[n].at(0), lo = hi;  // the largest score is that of the largest product, or of the least
#pragma unroll
    for (int i = 1; i < RW / 2; ++i) {
      hi = fmaxf(hi, s[n].at(i));
      lo = fminf(lo, s[n].at(i));
    }
    t[n].best = t[n].f < 0.0f ? lo : hi;
    t[n].top = fmaf(t[n].best, t[n].f, t[n].bias);
  }
}
// The largest scale of values met with a tile's, which counts if it has tokens, and whether that is far below the largest
// (as log2).
__device__ inline float met(float base, const Tile& t) { return t.valid > 0 ? fmaxf(base, t.bias) : base; }
__device__ inline bool is_far(float base, const Tile& t) { return t.valid > 0 && t.bias < base - kSpread; }
// Whether scores are so large that fp32 holds them in steps of 1/2 or more: a weight's exponent is no longer their difference
// if what is added to a product is rounded before.
__device__ inline bool is_big(float top) { return fabsf(top) > 0x1p22f && fabsf(top) < INFINITY; }
// O and the `sub`-th tile's values with weights p.
template <int DB, int RW, bool WIDE>
__device__ __forceinline__ void add_values(const uint8_t* lds, int sub, const f16x8 (&p)[RW / 16], int lane, State<DB, RW>& S) {
  using St = Staged<DB, WIDE>;
  const int rho = lane % RW, c = lane / RW;
  const uint8_t* vp = lds + St::kKeys + rho * St::kValuePitch + (32 * sub + RW / 2 * c) * St::kCode;
  if constexpr (RW == 32) {
#pragma unroll
    for (int j = 0; j < DB; ++j) {
      f16x8 v[2];
      operands<true, WIDE>(vp + 32 * j * St::kValuePitch, v);
      S.o32[j] = mfma(v[0], p[0], S.o32[j]);
      S.o32[j] = mfma(v[1], p[1], S.o32[j]);
    }
  } else {
#pragma unroll
    for (int n = 0; n < 2 * DB; ++n) {
      const u32x2 v = *reinterpret_cast<const u32x2*>(vp + 16 * n * St::kValuePitch);
      S.o16[n] = mfma(widen<true>(v.x, v.y), p[0], S.o16[n]);
    }
  }
}
template <int N>
__device__ inline void narrow_all(const float (&x)[N], f16x8 (&p)[N / 8]) {
#pragma unroll
  for (int i = 0; i < N / 8; ++i) p[i] = narrow(x + 8 * i);
}

// What comes before the weights of a tile of a scale far below the largest met, or of big scores, m having followed top. While
// it is added, O is held 2^lift times as large, lift per row, and its weights are: as much as brings the row's largest of the
// tile to 2^12, unless O would overflow. Of big scores products are rounded first, m follows them alone, and weights are
// 2^(s - m): lift is what O needs for that. To be undone by S.scale(2^-lift).
template <int DB, int RW>
__device__ inline float lifted(State<DB, RW>& S, float top, bool big, Tile& t, float& off) {
  float most = 0.0f;
#pragma unroll
  for (int n = 0; n < S.kGroups; ++n) {
    const f32x4 o = S.get(n);
#pragma unroll
    for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(o[i]) <= FLT_MAX ? fabsf(o[i]) : 0.0f);
    __builtin_amdgcn_sched_barrier(0);  // (a rare path that takes no registers from the others)
  }
  const int e = __builtin_amdgcn_frexp_expf(row_max<RW>(most));
  float lift = rintf(fmaxf(fminf(S.m - row_max<RW>(top), (float)(124 - max(e, 0))), 0.0f));
  if (big) lift = -(t.bias + kHeadroom);
  off = big ? -S.m : off + lift;
  t.inv *= __builtin_amdgcn_exp2f(-lift);
  S.scale(__builtin_amdgcn_exp2f(lift));
  return lift;
}

// The `sub`-th tile of the stage in LDS, of `valid` tokens: products, one step of the softmax, products.
template <bool F16, int DB, int RW, bool WIDE, int NQ>
__device__ __forceinline__ void attend_tile(const V8<F16> (&q)[NQ], const uint8_t* lds, int sub, int valid, float scales,
                                            int lane, State<DB, RW>& S) {
  Scores<RW> s[1];
  Tile t[1];
  multiply<F16, DB, RW, WIDE>(q, lds, sub, {valid}, scales, lane, s, t);
  S.base = met(S.base, t[0]);
  float top = t[0].top;
  const bool rare = __ballot(is_far(S.base, t[0]) || is_big(top)) != 0;
  bool big = false;
  if (rare && __ballot(is_big(top))) {
    big = true;
    top = t[0].best * t[0].f;
  }
  float off = t[0].bias - follow(S, top), lift = 0.0f;
  if (rare) lift = lifted(S, top, big, t[0], off);
  float x[RW / 2];
#pragma unroll
  for (int i = 0; i < RW / 2; ++i) x[i] = fmaf(s[0].at(i), t[0].f, off);
  if (big) {
    asm volatile("");
#pragma unroll
    for (int i = 0; i < RW / 2; ++i) x[i] = s[0].at(i) * t[0].f + off;
  }
#pragma unroll
  for (int i = 0; i < RW / 2; ++i) x[i] = __builtin_amdgcn_exp2f(x[i]);
  S.l = fmaf(sum_of(x), t[0].inv, S.l);
  f16x8 p[RW / 16];
  narrow_all(x, p);
  add_values<DB, RW, WIDE>(lds, sub, p, lane, S);
  if (rare) S.scale(__builtin_amdgcn_exp2f(-lift));
}
// Two tiles at once, whose products do not wait for each other. False, with nothing added, if they are not plain ones.
template <bool F16, int DB, bool WIDE, int NQ>
__device__ __forceinline__ bool attend_two(const V8<F16> (&q)[NQ], const uint8_t* lds, int sub, const int (&valid)[2],
                                           float scales, int lane, State<DB, 32>& S) {
  Scores<32> s[2];
  Tile t[2];
  multiply<F16, DB, 32, WIDE>(q, lds, sub, valid, scales, lane, s, t);
  const float base = met(met(S.base, t[0]), t[1]), top = fmaxf(t[0].top, t[1].top);
  if (__ballot(is_far(base, t[0]) || is_far(base, t[1]) || is_big(t[0].top) || is_big(t[1].top))) return false;
  S.base = base;
  const float from = follow(S, top);
  f16x8 p[2][2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const float off = t[n].bias - from;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(s[n].at(i), t[n].f, off));
    S.l = fmaf(sum_of(x), t[n].inv, S.l);
    narrow_all(x, p[n]);
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) add_values<DB, 32, WIDE>(lds, sub + n, p[n], lane, S);
  return true;
}

// 32 nodes in LDS, in their own type: keys like a tile's, values by dimension.
template <int DB>
struct Nodes {
  static constexpr int kKeyPitch = 64 * DB + 16, kValuePitch = 64 + 16;
  static constexpr int kKeys = 32 * kKeyPitch, kBytes = kKeys + 32 * DB * kValuePitch;
  static constexpr int kPieces = 32 * 4 * DB;  // of 16 bytes, of keys and of values
};
template <int DB, int T>
struct NodeLoads {
  static constexpr int kN = (Nodes<DB>::kPieces + T - 1) / T;
  u32x4 k[kN], v[kN];
};
template <int DB, int T>
__device__ __forceinline__ void load_nodes(const AttendArgs& A, int b, int h, int first, int nodes, int t,
                                           NodeLoads<DB, T>& L) {
  const char* kp = A.k + b * A.kb + h * A.kh;
  const char* vp = A.v + b * A.vb + h * A.vh;
#pragma unroll
  for (int i = 0; i < L.kN; ++i) {
    const int u = t + T * i, n = u / (4 * DB), c = u - n * (4 * DB);
    L.k[i] = L.v[i] = u32x4{0, 0, 0, 0};
    if (u < Nodes<DB>::kPieces && first + n < nodes) {
      L.k[i] = *reinterpret_cast<const u32x4*>(kp + (first + n) * A.kn + 16 * c);
      L.v[i] = *reinterpret_cast<const u32x4*>(vp + (first + n) * A.vn + 16 * c);
    }
  }
}
__device__ inline bool not_finite16(uint32_t x, bool f16) {
  return f16 ? (x & 0x7C00u) == 0x7C00u : (x & 0x7F80u) == 0x7F80u;
}
// Whether a value is not finite or, of bf16, 2^90 or more. (One that is not finite is held as 0, for 0 times it is no 0, and
// added to the rows that see it.)
template <bool F16, int RW, int DB, int T>
__device__ __forceinline__ bool store_nodes(uint8_t* lds, int t, const NodeLoads<DB, T>& L) {
  using Nd = Nodes<DB>;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < L.kN; ++i) {
    const int u = t + T * i, n = u / (4 * DB), c = u - n * (4 * DB);
    if (u >= Nd::kPieces) continue;
    *reinterpret_cast<u32x4*>(lds + row_of<RW>(n) * Nd::kKeyPitch + 16 * c) = L.k[i];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint16_t y = (uint16_t)(L.v[i][e / 2] >> (16 * (e & 1)));
      if ((y & 0x7FFFu) >= (F16 ? 0x7C00u : 0x6C80u)) {
        bad = true;
        if (not_finite16(y, F16)) y = 0;
      }
      *reinterpret_cast<uint16_t*>(lds + Nd::kKeys + (8 * c + e) * Nd::kValuePitch + 2 * n) = y;
    }
  }
  return bad;
}

// The 32 nodes in LDS, `first` the first of them. bits: the nodes that the lane's row sees; bad: there are values that
// are not finite, or huge.
template <bool F16, int DB, int RW, int NQ>
__device__ inline void attend_nodes(const AttendArgs& A, const V8<F16> (&q)[NQ], const uint8_t* lds, int b, int h,
                                    int first, int nodes, uint64_t bits, bool bad, int lane, State<DB, RW>& S) {
  using Nd = Nodes<DB>;
  constexpr int NX = RW / 2;  // a lane's nodes
  const int rho = lane % RW, c = lane / RW;
  float x[NX];
  const uint8_t* kp = lds + rho * Nd::kKeyPitch + (RW == 32 ? 32 : 16) * c;
  const uint32_t sees = (uint32_t)(bits >> (first + NX * c)) & ((1u << NX) - 1);
  if constexpr (RW == 32) {
    f32x16 s = {};
#pragma unroll
    for (int j = 0; j < DB; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) s = mfma(*reinterpret_cast<const V8<F16>*>(kp + 64 * j + 16 * e), q[2 * j + e], s);
#pragma unroll
    for (int i = 0; i < NX; ++i) x[i] = (sees >> i) & 1 ? s[i] * A.scale2 : -INFINITY;
  } else {
    f32x4 s[2] = {};
#pragma unroll
    for (int j = 0; j < DB; ++j)
#pragma unroll
      for (int a = 0; a < 2; ++a)
        s[a] = mfma(*reinterpret_cast<const V8<F16>*>(kp + 16 * a * Nd::kKeyPitch + 64 * j), q[j], s[a]);
#pragma unroll
    for (int i = 0; i < NX; ++i) x[i] = (sees >> i) & 1 ? s[i / 4][i % 4] * A.scale2 : -INFINITY;
  }
  const float scale = bad && !F16 ? kHugeNodes : kNodes, from = follow(S, max_of(x) + scale);
  S.base = fmaxf(S.base, scale);
#pragma unroll
  for (int i = 0; i < NX; ++i) x[i] = __builtin_amdgcn_exp2f(x[i] - from);
  S.l += sum_of(x);
  const uint8_t* vp = lds + Nd::kKeys + rho * Nd::kValuePitch + 2 * NX * c;
#pragma unroll
  for (int e = 0; e < NX / 8; ++e) {
    const Weights p(x + 8 * e);
#pragma unroll
    for (int n = 0; n < 32 * DB / RW; ++n) {
      const u32x4 y = *reinterpret_cast<const u32x4*>(vp + RW * n * Nd::kValuePitch + 16 * e);
      auto product = [&](bf16x8 v, bf16x8 w) {
        if constexpr (RW == 32) S.o32[n] = mfma(v, w, S.o32[n]);
        else S.o16[n] = mfma(v, w, S.o16[n]);
      };
      if constexpr (F16) {  // (both rests: below 2^-15 of the product)
        const Parts v(y);
        product(v.hi, p.hi);
        product(v.hi, p.lo);
        product(v.lo, p.hi);
      } else {
        product(__builtin_bit_cast(bf16x8, y), p.hi);
        product(__builtin_bit_cast(bf16x8, y), p.lo);
      }
    }
  }
  if (!bad) return;
  const char* gp = A.v + b * A.vb + h * A.vh;
#pragma unroll 1
  for (int n = first; n < min(first + 32, nodes); ++n) {
    const bool on = (bits >> n) & 1;
#pragma unroll
    for (int k = 0; k < S.kGroups; ++k) {
      f32x4 o = S.get(k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint16_t y = *reinterpret_cast<const uint16_t*>(gp + n * A.vn + 2 * (S.kDims * k + 4 * c + i));
        if (on && not_finite16(y, F16))
          o[i] += F16 ? (float)__builtin_bit_cast(_Float16, y) : __uint_as_float((uint32_t)y << 16);
      }
      S.set(k, o);
      __builtin_amdgcn_sched_barrier(0);  // (a rare path that takes no registers from the others)
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

// A query's stages that lie in the range [from, to) of all, `before` of which come before the query's.
template <bool F16, int DB, int RW, int WR, int NW>
__device__ __forceinline__ void attend_range(const AttendArgs& A, int b, int h, int tile, int wv, int nth, int per, int from,
                                             int to, int before, uint8_t* s_stage, float (*s_m)[32],
                                             float (*s_l)[32]) {
  constexpr int D = 32 * DB, kPitch = D + 4, WT = NW / WR, kRows = RW * WR, T = 64 * NW;
  float(*s_o)[RW * kPitch] = reinterpret_cast<float(*)[RW * kPitch]>(s_stage);
  int thread = threadIdx.x;
  asm volatile("" : "+v"(thread));  // no address is formed before the loop over queries and kept through it
  const int lane = thread & 63, rho = lane % RW, c = lane / RW, wr = wv % WR, wt = wv / WR;
  const int nodes = nodes_of(A, b), rows = nodes * A.group;
  if (tile * kRows >= rows) return;
  const int tokens = same(tokens_of(A, b)), stages = same(stages_of(A, b));
  const bool starts = before >= from, ends = before + stages <= to;  // the query's first, its last stage is in the range
  const int first = starts ? 0 : (from - before) * kStage;
  const int last = min(ends ? INT_MAX : (to - before) * kStage, (int)(((uint32_t)tokens + 31) / 32));

  const int row = tile * kRows + wr * RW + rho;
  const bool live = row < rows, busy = tile * kRows + wr * RW < rows;  // busy: the wave has rows
  const int node = live ? (int)fdiv((uint32_t)row, A.div_group) : 0;
  const int head = h * A.group + (live ? row - node * A.group : 0);
  // What comes first is asked for first: a draft's nodes (their keys and values go through LDS before the stages), the
  // queries, the first stage.
  NodeLoads<DB, T> nl;
  if (ends) load_nodes<DB, T>(A, b, h, 0, nodes, thread, nl);
  constexpr int NQ = DB * RW / 16;
  V8<F16> q[NQ];
  const char* qp = A.q + b * A.qb + node * A.qn + head * A.qh + (RW == 32 ? 32 : 16) * c;
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    u32x4 x = *reinterpret_cast<const u32x4*>(qp + (RW == 32 ? 64 * (j / 2) + 16 * (j % 2) : 64 * j));
    if (!live) x = u32x4{0, 0, 0, 0};
    __builtin_memcpy(&q[j], &x, 16);
  }
  State<DB, RW> S;
  S.clear();

  Loads<DB, NW> L;
  int pages = pages_of(A, b, first, last, lane), next = -1;  // of the stage that is on its way, of the one behind it
  float coming = 0.0f;                                       // its scales
  if (first < last) {
    coming = scales_of(A, h, pages, lane);
    next = pages_of(A, b, first + kStage, last, lane);
    load_stage<DB, NW>(A, h, first, pages, wv, lane, L);
  }
  if (ends) {  // the query's last part has the nodes too
    uint64_t bits = 0;
    if (live) {
      bits = A.mask ? A.mask[(int64_t)b * A.M + node] : (2ull << node) - 1;
      if (nodes < 64) bits &= (1ull << nodes) - 1;
    }
#pragma unroll 1
    for (int n = 0; n < nodes; n += 32) {
      if (n > 0) {
        load_nodes<DB, T>(A, b, h, n, nodes, thread, nl);
        __syncthreads();  // the 32 before are read
      }
      const bool bad = __syncthreads_or(store_nodes<F16, RW, DB, T>(s_stage, thread, nl));
      if (busy && (n >> 5) % WT == wt) attend_nodes<F16, DB, RW>(A, q, s_stage, b, h, n, nodes, bits, bad, lane, S);
    }
    __syncthreads();
  }

  for (int t = first; t < last; t += kStage) {
    if (t > first) __syncthreads();  // the stage before is read
    const float factors = factors_of(A, coming, lane);
    store_stage<F16, RW, DB, NW, WR == 8>(s_stage, t, pages, tokens, factors, wv, lane, L);
    const int here = pages;
    const float scales = lane < kStage && factors == 0.0f ? 1.0f : factors;
    pages = next;
    __syncthreads();
    if (t + kStage < last) {
      coming = scales_of(A, h, pages, lane);
      next = pages_of(A, b, t + 2 * kStage, last, lane);
      load_stage<DB, NW>(A, h, t + kStage, pages, wv, lane, L);
    }
    if (!busy) continue;
    if constexpr (WR == 8) {  // (two tiles at once: 32 trees of 61 nodes 210 us, one at a time 214; with four waves no gain)
#pragma unroll
      for (int i = 0; i < kStage; i += 2) {
        const int valid[2] = {valid_of(here, t, i, tokens), valid_of(here, t, i + 1, tokens)};
        if (!attend_two<F16, DB, true>(q, s_stage, i, valid, scales, lane, S))
#pragma unroll 1
          for (int n = i; n < i + 2; ++n)
            attend_tile<F16, DB, RW, true>(q, s_stage, n, valid_of(here, t, n, tokens), scales, lane, S);
      }
    } else {
#pragma unroll
      for (int i = wt; i < kStage + wt; i += WT)
        attend_tile<F16, DB, RW, false>(q, s_stage, i, valid_of(here, t, i, tokens), scales, lane, S);
    }
  }

  float m = S.m, l = row_sum<RW>(S.l);
  if constexpr (WT > 1) {  // the states of the waves of a group, joined
    if (c == 0) {
      s_m[wv][rho] = m;
      s_l[wv][rho] = l;
    }
    __syncthreads();  // (and the last stage is read)
    m = s_m[wr][rho];
#pragma unroll
    for (int w = 1; w < WT; ++w) m = fmaxf(m, s_m[w * WR + wr][rho]);
    l = 0.0f;
#pragma unroll
    for (int w = 0; w < WT; ++w)
      l = fmaf(s_l[w * WR + wr][rho], __builtin_amdgcn_exp2f(s_m[w * WR + wr][rho] - m), l);
    S.scale(__builtin_amdgcn_exp2f(S.m - m));
#pragma unroll
    for (int half = WT / 2; half >= 1; half /= 2) {  // the upper half of the waves to the lower
      if (wt >= half && wt < 2 * half) {
        float* at = &s_o[(wt - half) * WR + wr][rho * kPitch + 4 * c];
#pragma unroll
        for (int n = 0; n < S.kGroups; ++n) *reinterpret_cast<f32x4*>(at + S.kDims * n) = S.get(n);
      }
      __syncthreads();
      if (wt < half) {
        const float* at = &s_o[wt * WR + wr][rho * kPitch + 4 * c];
#pragma unroll
        for (int n = 0; n < S.kGroups; ++n) S.set(n, S.get(n) + *reinterpret_cast<const f32x4*>(at + S.kDims * n));
      }
      if (half > 1) __syncthreads();
    }
    if (wt != 0) return;
  }
  if (starts && ends) {
    if (!live) return;
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;  // (a NaN stays)
    char* op = A.out + b * A.ob + node * A.on + head * A.oh + 8 * c;
#pragma unroll
    for (int n = 0; n < S.kGroups; ++n) store4<F16>(op + 2 * S.kDims * n, S.get(n) * inv);
    return;
  }
  const int64_t at = (((int64_t)(h * A.tiles + tile) * (2 * A.chunks) + 2 * nth + (before > from ? 1 : 0)) * WR + wr) * RW;
  float* op = A.part + at * D + 4 * lane;  // (as the registers are: a wave writes 1 KB at a time)
#pragma unroll
  for (int n = 0; n < S.kGroups; ++n) *reinterpret_cast<f32x4*>(op + n * 256) = S.get(n);
  if (c == 0) A.part_ml[at + rho] = make_float2(m, l);
}

// A workgroup of NW waves has RW rows for each of WR groups of its waves. It brings kStage tiles at a time to LDS, of
// which the WT = NW / WR waves of a group take every WT-th each; their states are joined at the end. The next stage is on
// its way to registers meanwhile.
template <bool F16, int DB, int RW, int WR, int NW>
__global__ void __launch_bounds__(64 * NW, waves_of(RW, 32 * DB)) hs_attend_kernel(const AttendArgs A) {
  constexpr int kPitch = 32 * DB + 4, WT = NW / WR;
  using St = Staged<DB, WR == 8>;
  constexpr int kBytes = St::kBytes > Nodes<DB>::kBytes ? St::kBytes : Nodes<DB>::kBytes;
  __shared__ __attribute__((aligned(16))) uint8_t s_stage[kBytes];
  static_assert(WT == 1 || kBytes >= WT / 2 * WR * RW * kPitch * 4, "the join shares the stage's memory");
  static_assert(WT <= kStage, "a wave has a tile of every stage");
  __shared__ float s_m[NW][32], s_l[NW][32];
  const int lane = threadIdx.x & 63, wv = (int)uniform(threadIdx.x >> 6);
  // eight items, then the next rows of the same eight: an XCD reads an item's pages once
  const uint32_t g = A.group0 + blockIdx.x, eight = g >> 3, lot = fdiv(eight, A.div_tiles);
  const int tile = (int)(eight - lot * (uint32_t)A.tiles);
  const uint32_t item = lot * 8 + (g & 7);
  if (item >= A.items) return;
  const int nth = (int)fdiv(item, A.div_kv), h = (int)item - nth * A.kv;
  // the range's stages, of all queries'; of a query that is its own range they are its own
  int per = 0, from = 0, to = INT_MAX, b = nth, before = 0;
  if (A.chunks) {
    const Plan plan(A, lane);
    per = plan.per;
    from = nth * per;
    to = from + per;
    b = plan.query(A, from, &before);
    if (b < 0) return;
  }
  for (bool again = false;; again = true) {  // the queries of the range
    if (again) {
      before += same(stages_of(A, b));
      if (!A.chunks || ++b >= A.B || before >= to) return;
      __syncthreads();  // (the last query's join is read)
    }
    attend_range<F16, DB, RW, WR, NW>(A, b, h, tile, wv, nth, per, from, to, before, s_stage, s_m, s_l);
  }
}
// The parts of a query's rows, joined: a wave a group of dims of RW rows at a time, as they were in the registers. A
// workgroup does four groups, those from 4 blockIdx.y on, 4 (blockIdx.y + gridDim.y), .. With W > 1 it does one group,
// blockIdx.y, its W waves every W-th part each, joined through LDS: a wave alone reads eight parts at a time (one query's
// call, eight heads: one token over 4096, 32 parts, 16.5 us and by four waves 14.2; over 32768, 96 parts, 32.8 and by
// sixteen, of whose registers 15 to 17 spill, 25.6; a tree of 61 nodes, whose 33 MB of parts are the bound, 45.2 and 45.3).
template <bool F16, int DB, int RW, int WR, int W>
__global__ void __launch_bounds__(W > 1 ? 64 * W : kThreads) hs_attend_join_kernel(const AttendArgs A) {
  constexpr int D = 32 * DB, kAhead = 8;
  __shared__ f32x4 s_o[W > 1 ? W : 1][64];
  __shared__ float2 s_ml[W > 1 ? W : 1][64];
  using St = State<DB, RW>;
  const int lane = threadIdx.x & 63, rho = lane % RW, c = lane / RW;
  const uint32_t bh = fdiv(blockIdx.x, A.div_rows);
  const int rt = (int)(blockIdx.x - bh * A.row_tiles);
  const int b = (int)fdiv(bh, A.div_kv), h = (int)bh - b * A.kv;
  const int rows = nodes_of(A, b) * A.group;
  if (rt * RW >= rows) return;
  const Plan plan(A, lane);
  const int before = plan.before(A, b), r0 = before / plan.per, r1 = (before + same(stages_of(A, b)) - 1) / plan.per;
  if (r0 == r1) return;  // one part
  const int tile = rt / WR, row = rt * RW + rho;
  const int64_t base = (int64_t)(h * A.tiles + tile) * (2 * A.chunks);
  auto place = [&](int r) -> int64_t {  // the first of the RW rows of part r
    return ((base + 2 * r + (before > r * plan.per ? 1 : 0)) * WR + (rt - tile * WR)) * RW;
  };
  const int node = (int)fdiv((uint32_t)min(row, rows - 1), A.div_group), head = h * A.group + row - node * A.group;
  const int wv = (int)uniform(threadIdx.x >> 6), r00 = W > 1 ? r0 + wv : r0;
  for (int n = W > 1 ? blockIdx.y : 4 * blockIdx.y + wv; n < St::kGroups; n += W > 1 ? St::kGroups : 4 * gridDim.y) {
    float m = kLowest, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int r = r00; r <= r1; r += W * kAhead) {
      f32x4 y[kAhead];
      float2 ml[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a)
        if (r + W * a <= r1) {
          const int64_t at = place(r + W * a);
          ml[a] = A.part_ml[at + rho];
          y[a] = *reinterpret_cast<const f32x4*>(A.part + at * D + n * 256 + 4 * lane);
        }
      const float old = m;
#pragma unroll
      for (int a = 0; a < kAhead; ++a)
        if (r + W * a <= r1) m = fmaxf(m, ml[a].x);
      const float less = __builtin_amdgcn_exp2f(old - m);
      l *= less;
      o *= less;
#pragma unroll
      for (int a = 0; a < kAhead; ++a)
        if (r + W * a <= r1) {
          const float f = __builtin_amdgcn_exp2f(ml[a].x - m);
          l = fmaf(ml[a].y, f, l);
#pragma unroll
          for (int k = 0; k < 4; ++k) o[k] = fmaf(y[a][k], f, o[k]);
        }
    }
    if constexpr (W > 1) {
      s_o[wv][lane] = o;
      s_ml[wv][lane] = make_float2(m, l);
      __syncthreads();
      if (wv != 0) return;
#pragma unroll
      for (int w = 1; w < W; ++w) m = fmaxf(m, s_ml[w][lane].x);
      l = 0.0f;
      o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_ml[w][lane].x - m);
        l = fmaf(s_ml[w][lane].y, f, l);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = fmaf(s_o[w][lane][k], f, o[k]);
      }
    }
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    if (row < rows)
      store4<F16>(A.out + b * A.ob + node * A.on + head * A.oh + 2 * (St::kDims * n + 4 * c), o * inv);
  }
}

template <bool F16, int DB, int RW, int WR, int NW>
void launch_rows(AttendArgs A, hipStream_t st) {
  const uint64_t groups = ((uint64_t)A.items + 7) / 8 * 8 * A.tiles;
  constexpr uint64_t kMost = kMostGroups / (NW / kWaves);
  for (uint64_t at = 0; at < groups; at += kMost) {
    A.group0 = (uint32_t)at;
    hs_attend_kernel<F16, DB, RW, WR, NW><<<(uint32_t)std::min<uint64_t>(groups - at, kMost), 64 * NW, 0, st>>>(A);
    if (hipPeekAtLastError() != hipSuccess) return;
  }
  if (!A.chunks) return;
  const uint32_t joins = (uint32_t)A.B * A.kv * A.row_tiles;  // (few: ranges are for few queries and heads)
  constexpr int kGroups = State<DB, RW>::kGroups;
  const int parts = A.chunks / A.B;  // of a query, where lengths are alike
  if (parts > 32) hs_attend_join_kernel<F16, DB, RW, WR, 16><<<dim3(joins, kGroups), 1024, 0, st>>>(A);
  else if (parts > 8) hs_attend_join_kernel<F16, DB, RW, WR, 4><<<dim3(joins, kGroups), 256, 0, st>>>(A);
  else hs_attend_join_kernel<F16, DB, RW, WR, 1><<<dim3(joins, joins < 512 ? (kGroups + 3) / 4 : 1), kThreads, 0, st>>>(A);
}

template <bool F16, int DB>
void launch_dim(const AttendArgs& A, const AttendGeom& g, hipStream_t st) {
  if constexpr (DB <= 4)
    if (g.wr == 8) return launch_rows<F16, DB, 32, 8, 8>(A, st);
  if constexpr (DB <= 7)
    if (g.wr == 4) return launch_rows<F16, DB, 32, 4, 4>(A, st);
  if (g.wr == 2) return launch_rows<F16, DB, 32, 2, 4>(A, st);
  if (g.rw == 32) return launch_rows<F16, DB, 32, 1, 4>(A, st);
  launch_rows<F16, DB, 16, 1, 4>(A, st);
}

template <bool F16>
void launch_type(const AttendArgs& A, const AttendGeom& g, hipStream_t st) {
  switch (g.dim / 32) {
    case 1: return launch_dim<F16, 1>(A, g, st);
    case 2: return launch_dim<F16, 2>(A, g, st);
    case 3: return launch_dim<F16, 3>(A, g, st);
    case 4: return launch_dim<F16, 4>(A, g, st);
    case 5: return launch_dim<F16, 5>(A, g, st);
    case 6: return launch_dim<F16, 6>(A, g, st);
    case 7: return launch_dim<F16, 7>(A, g, st);
    default: return launch_dim<F16, 8>(A, g, st);
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
  const int rows = M * (heads / kv);
  g->rw = rows > 16 ? 32 : 16;
  // (Four groups of rows of 256 dimensions spill: 16 trees of 61 nodes 200 us, in groups of two 164; one of 45 95 and 66. Those
  // of 160 to 224 by four and by two, 16 trees over 1024 tokens, 32 heads of 8: 61 nodes 64 and 84, 68 and 92, 91 and 109 us;
  // 20 nodes, whose 80 rows leave four groups a third idle, 42 and 38, 48 and 43, 60 and 50. At 224 dimensions 33 registers
  // spill, at 256 15 with 64 rows, 26 with 16 rows and up to 2 with 32.)
  g->wr = rows > 128 && dim <= 128 ? 8 : rows > 64 && dim <= 224 ? 4 : rows > 32 ? 2 : 1;
  g->tiles = (rows + g->rw * g->wr - 1) / (g->rw * g->wr);
  // Ranges for the workgroups that the device holds at once; a workgroup a query and head, and no join, where there are
  // four times as many of those, or where caches are so short that the join costs more than cutting them saves. us cut and
  // whole at 8 heads of 128, one token: one query of 128 tokens 12.3 and 8.9, of 256 13.2 and 10.5, of 512 13.2 and 13.5;
  // 32 queries of 512 18.6 and 14.2, of 1024 27.5 and 21.8. Trees of 61 nodes: one query of 128 tokens 20.8 and 17.3, of 512
  // 22.1 and 30.9; 32 queries of 512 44.5 and 41.2. Longer caches are cut whatever their number: their lengths differ, and
  // the longest alone would set the time (32 trees over up to 8192 tokens: 220 cut, 318 whole).
  const int64_t groups = (int64_t)B * kv * g->tiles, hold = 256 * waves_of(g->rw, dim) / (g->wr == 8 ? 2 : 1);
  const int64_t each = ((int64_t)slots * page + 32 * kStage - 1) / (32 * kStage);  // stages of a query
  const bool whole = groups >= 4 * hold || each * B >= 1 << 30 ||  // (the stages of all are counted in 32 bits)
                     each <= std::min<int64_t>(std::max<int64_t>(groups / 32, 2), 8);
  g->chunks = whole ? 0 : (int)std::min(std::max<int64_t>(hold / ((int64_t)kv * g->tiles), 1), each * B);
  return groups < ((int64_t)1 << 30);
}

size_t attend_ws_bytes(const AttendGeom& g) {
  if (!g.chunks) return 0;
  const size_t slots = (size_t)g.kv * g.tiles * (2 * g.chunks) * (g.rw * g.wr);
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
  A.chunks = g.chunks;
  A.items = (uint32_t)((int64_t)(g.chunks ? g.chunks : g.B) * g.kv);
  A.div_kv = make_fastdiv((uint32_t)g.kv);
  A.div_tiles = make_fastdiv((uint32_t)g.tiles);
  A.div_group = make_fastdiv((uint32_t)A.group);
  A.row_tiles = (uint32_t)((g.M * A.group + g.rw - 1) / g.rw);
  A.div_rows = make_fastdiv(A.row_tiles);
  const size_t slots = (size_t)g.kv * g.tiles * (2 * g.chunks) * (g.rw * g.wr);
  A.part = reinterpret_cast<float*>(a.workspace);
  A.part_ml = reinterpret_cast<float2*>(reinterpret_cast<char*>(a.workspace) +
                                        align256(slots * g.dim * sizeof(float)));
  if (a.dtype == HS_F16) launch_type<true>(A, g, stream);
  else launch_type<false>(A, g, stream);
  return hipPeekAtLastError() == hipSuccess ? HS_OK : HS_ERR_HIP;
}

}  // namespace hs
