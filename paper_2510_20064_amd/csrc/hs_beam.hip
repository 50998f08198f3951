// hs_beam_step: the K best continuations of a query's W beams by
//   s(w, v) = score_w + log softmax(z_w / T)_v = score_w + (z_wv c - lse2_w) ln 2,
// c = log2(e) / T, lse2_w = log2 sum_v 2^(z_wv c). Within a beam the order of s is the order of the
// logits. Two launches:
//   1. hs_beam_rows_kernel reads every logit once and keeps, of each slice (one wave's chunks of 256
//      16-byte vectors), its exp2 sum, and of each quarter of a chunk (a unit: what 16 lanes hold) its
//      largest logit. No candidates: what a unit must hold to matter is not known before the rows'
//      normalisers are;
//   2. hs_beam_merge_kernel, one workgroup per query: the normalisers, then a bound from the scores of
//      the units' maxima: the K-th largest of them is reached by K entries at least, so only the units
//      whose maximum reaches it (about K of all the query's units) can hold any of the K best: these
//      are read again, and what reaches the bound is ranked by (s, lower beam, larger logit, lower
//      token).
//
// Precision. Two beams' candidates are often closer than fp32 tells apart and the order is part of
// the result, so s is formed in fp64 and the normalisers are made good to 1e-7 (measured: 3.5e-9 rms on
// flat rows, 1.5e-8 on a model's, 3e-10 at most where one logit has the mass, 1.4e-7 at most of all): z c is
// taken as z ca + z cb with ca = c rounded to 12 bits (for 16-bit logits z ca - offset is exact), the fp32
// exponentials of a vector are added in pairs and the vectors in fp64, and the exponentials of the units'
// largest logits, most of the sum where the distribution is peaked, are replaced by fp64 ones.
// Sums are relative to an offset near the slice's maximum, and a slice whose maximum is large
// (|z c| > 4096) takes z - maximum first, so that logits of any size do, the lowest finite value
// in every place included.
//
// Bound. The rows kernel reads 311 MB (32 x 32 rows of 151936 bf16) in 50.2 us, 6.2 TB/s, each byte once (its
// 552 vector instructions per two chunks and wave take about as long as the memory does), 110 MB in
// 22.6 us, and a call too short for that in 4.0 us. The merge is bound by latency, by six steps that wait
// for each other: 5.0 us for 4 rows of 128 units and 4 slots, 16.4 us for 32 workgroups of 32 rows of 300
// units and 64 slots (an instruction that all of its 16 waves make costs 16 cycles). Two launches: in
// one, with a query's last workgroup merging, the fences between the XCDs' caches cost what the second
// launch does (10 rows of bf16 13.3 us, or 11.4 with device-scope words instead of fences; two 10.8). That was
// measured on calls of few rows only, where there is nothing to merge behind.
#include <algorithm>
#include <cfloat>

#include "hs_beam.h"

namespace hs {

namespace {

constexpr int kMergeThreads = 1024;  // (256, 512, 1024: 10 rows of bf16 14.7, 11.8, 10.7 us, 32 x 32 rows 89, 72, 65)
constexpr int kMergeWaves = kMergeThreads / 64;
constexpr int kAtOnce = 4;       // units that a wave reads at once
constexpr int kPairs = 2048;     // entries of one query held in LDS, twice what a round can add
constexpr int kTokenBits = 26;
constexpr uint32_t kTokenMask = (1u << kTokenBits) - 1;

constexpr int kUnits = 4;        // of a chunk

struct SliceRec {
  double sum;  // of 2^(z c - offset) over the slice (not finite: a NaN or +inf logit)
  float ref;   // the logit that the offset came from; -inf: no logit above -inf
  int off;     // the offset of a small one
};

struct StepArgs {
  const char* x;
  int64_t sb, sw;  // bytes between queries and between beams
  int W, K, S, chunks, nc;  // slices per row, chunks per slice and per row
  int nu;                   // units per row
  int64_t V, nvec, score_stride;
  uint32_t units;  // B * W * S
  uint32_t group0;  // the launch's first workgroup of the rows kernel's
  FastDiv divS, divW, divU;  // by S, W and nu
  float ca, cb;
  double c, inv_c;  // c and 1 / c
  const float* score;
  const uint8_t* done;
  int eos;
  float* out_score;
  int32_t* out_parent;
  int32_t* out_token;
  uint8_t* out_done;
  SliceRec* rec;   // [B * W][S]
  float* top;      // [B * W][nu]: the units' largest logits
};

// The offset of exponents z c - off, from a logit at or near the largest.
struct Offset {
  float o;     // of small logits: an integer at or above ref c
  float ref;   // of large ones: subtracted from the logit first
  bool large;
  __device__ Offset(float m, float c) : ref(m) {
    large = !(fabsf(m * c) <= 4096.0f);
    o = large ? 0.0f : ceilf(m * c);
  }
  // in log2 units
  __device__ double value(double c) const { return large ? (double)ref * c : (double)o; }
  __device__ float exponent(float z, float ca, float cb) const {
    if (large) {
      const float d = z - ref;
      return fmaf(d, cb, d * ca);
    }
    return fmaf(z, cb, fmaf(z, ca, -o));
  }
};

// 2^d for d < 1024 to 2.8e-10 of itself: 2^n e^(f ln 2), |f| <= 1/2, by the series of degree 8. (A wave
// computes it once or twice for a slice of 4096 logits: a quarter of the instructions of exp2().)
__device__ inline double exp2_of(double d) {
  const double x = fmax(d, -2000.0), n = rint(x), f = (x - n) * 0.69314718055994530942;
  double p = 1.0 / 40320.0;
  p = fma(p, f, 1.0 / 5040.0);
  p = fma(p, f, 1.0 / 720.0);
  p = fma(p, f, 1.0 / 120.0);
  p = fma(p, f, 1.0 / 24.0);
  p = fma(p, f, 1.0 / 6.0);
  p = fma(p, f, 0.5);
  p = fma(p, f, 1.0);
  p = fma(p, f, 1.0);
  return ldexp(p, (int)n);
}

// log2 of a positive finite x to 1e-11: x = m 2^e with m near 1, log m = 2 artanh t, t = (m - 1) / (m + 1)
// and |t| < 0.172. (A whole wave computes it for its row: a third of the instructions of log2().)
__device__ inline double log2_of(double x) {
  double m = __builtin_amdgcn_frexp_mant(x);
  int e = __builtin_amdgcn_frexp_exp(x);
  if (m < 0.70710678118654752440) {
    m += m;
    --e;
  }
  const double t = (m - 1.0) / (m + 1.0), q = t * t;
  double p = 1.0 / 13.0;
  p = fma(p, q, 1.0 / 11.0);
  p = fma(p, q, 1.0 / 9.0);
  p = fma(p, q, 1.0 / 7.0);
  p = fma(p, q, 1.0 / 5.0);
  p = fma(p, q, 1.0 / 3.0);
  p = fma(p, q, 1.0);
  return fma(2.0 * 1.4426950408889634074 * t, p, (double)e);
}

// A beam that continues by its logits: a finite score, and not finished.
__device__ inline bool beam_grows(const StepArgs& A, int b, int w) {
  const int64_t i = (int64_t)b * A.score_stride + w;
  return isfinite(A.score[i]) && !(A.done && A.done[i]);
}

template <int DT>
__device__ inline void load_chunk(const char* row, int64_t v0, int64_t nvec, int64_t V, int lane,
                                  typename Vec<DT>::Raw (&x)[4]) {
  if ((v0 + kBeamChunk) * Vec<DT>::kElems <= V) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      typedef unsigned int u4 __attribute__((ext_vector_type(4)));
      typedef const __attribute__((address_space(1))) u4* gp4;
      // (every logit is read once: nontemporal, 8% faster on 311 MB of bf16)
      const u4 y = __builtin_nontemporal_load((gp4)(row + (v0 + i * 64 + lane) * 16));
      __builtin_memcpy(&x[i], &y, 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t vi = v0 + i * 64 + lane;
      x[i] = vi < nvec ? Vec<DT>::load_raw(row, vi, V) : Vec<DT>::neg_raw();
    }
  }
}

// ---- launch 1: sums of slices, maxima of units -------------------------------------------------------

template <int DT>
__global__ __launch_bounds__(kThreads) void hs_beam_rows_kernel(StepArgs A) {
  using Vt = Vec<DT>;
  using Raw = typename Vt::Raw;
  constexpr int E = Vt::kElems;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t u = (A.group0 + blockIdx.x) * kWaves + wv;
  if (u >= A.units) return;  // wave-uniform; the waves share nothing
  const uint32_t row = fdiv(u, A.divS);
  const int s = (int)(u - row * (uint32_t)A.S);
  const int b = (int)fdiv(row, A.divW), w = (int)row - b * A.W;
  if (!beam_grows(A, b, w)) return;
  const char* rowp = A.x + (int64_t)b * A.sb + (int64_t)w * A.sw;
  const int c0 = s * A.chunks, c1 = min(A.nc, c0 + A.chunks);
  const float c = (float)A.c;

  Offset off(-INFINITY, c);
  bool any = false;   // an offset is set
  double sum = 0.0;   // the lane's
  float mine = -INFINITY, mine_ref = -INFINITY;  // lane 16 r + i: unit r of the slice's i-th chunk
  Raw cur[4], nxt[4];
  load_chunk<DT>(rowp, (int64_t)c0 * kBeamChunk, A.nvec, A.V, lane, cur);
  for (int k = c0; k < c1; ++k) {
    if (k + 1 < c1) load_chunk<DT>(rowp, (int64_t)(k + 1) * kBeamChunk, A.nvec, A.V, lane, nxt);
    float z[4][E], lmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      Vt::unpack(cur[i], z[i]);
#pragma unroll
      for (int e = 0; e < E; ++e) lmax = fmaxf(lmax, z[i][e]);
    }
    const int key = row16_max(fkey(lmax));
    const float m = fkey_inv(key);
    // the offset stays while no exponent exceeds 4, so that a slice rarely changes it and the
    // rounding of z c - off stays that of small numbers
    if (!any || __ballot(off.exponent(m, A.ca, A.cb) > 4.0f)) {
      const float most = fkey_inv(
          max(max(__builtin_amdgcn_readlane(key, 0), __builtin_amdgcn_readlane(key, 16)),
              max(__builtin_amdgcn_readlane(key, 32), __builtin_amdgcn_readlane(key, 48))));
      if (most != -INFINITY) {
        const Offset now(most, c);
        if (any) sum *= exp2_of(off.value(A.c) - now.value(A.c));
        off = now;
        any = true;
      }
    }
    // a vector's exponentials are added in pairs and then in fp64: a term that is most of the row's sum
    // is rounded three times at most
    auto add_terms = [&](auto exponent) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float e[E];
#pragma unroll
        for (int j = 0; j < E; ++j) e[j] = __builtin_amdgcn_exp2f(exponent(z[i][j]));
#pragma unroll
        for (int n = E / 2; n > 0; n /= 2)
#pragma unroll
          for (int j = 0; j < n; ++j) e[j] += e[j + n];
        sum += (double)e[0];
      }
    };
    if (!any)
      add_terms([](float y) { return y; });  // 0, or NaN
    else if (off.large)
      add_terms([&](float y) { return fmaf(y - off.ref, A.cb, (y - off.ref) * A.ca); });
    else
      add_terms([&](float y) { return fmaf(y, A.cb, fmaf(y, A.ca, -off.o)); });
    if ((lane & 15) == k - c0) {
      mine = m;
      mine_ref = off.ref;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) cur[i] = nxt[i];
  }
  if (any && mine > -INFINITY) {  // the units' largest terms, from fp32 to fp64
    const Offset at(mine_ref, c);
    sum += (exp2_of((double)mine * A.c - at.value(A.c)) -
            (double)__builtin_amdgcn_exp2f(at.exponent(mine, A.ca, A.cb))) *
           (mine_ref == off.ref ? 1.0 : exp2_of(at.value(A.c) - off.value(A.c)));
  }
  sum = wave_sum_d(sum);
  const int k = c0 + (lane & 15);
  if (k < c1) A.top[(int64_t)row * A.nu + k * kUnits + (lane >> 4)] = mine;
  if (lane == 0) A.rec[u] = SliceRec{sum, off.ref, (int)off.o};
}

// ---- launch 2: the rows' normalisers and the K best ------------------------------------------------------

// The largest x that n of the C words in LDS reach, `of` mapping a place to its key (0: none): the n-th
// largest key, where there are n.
template <typename F>
__device__ inline uint64_t nth_of(F of, int C, int n, int lane) {
  uint64_t x = 0;
  for (int bit = 63; bit >= 0; --bit) {
    const uint64_t y = x | (1ull << bit);
    int c = 0;
    for (int i = 0; i < C; i += 64) c += __builtin_popcountll(__ballot(i + lane < C && of(i + lane) >= y));
    if (c >= n) x = y;
  }
  return x;
}

// The K best of C pairs, ordered by h, then l, to the front in no order; *kth: the least h among them,
// where there are K. One wave; rare (many equal scores).
__device__ __noinline__ int keep_best(uint64_t* h, uint64_t* l, int C, int K, int lane, uint64_t* kth) {
  lds_wave_fence();
  if (C < K) return C;
  const uint64_t x = nth_of([=](int i) { return h[i]; }, C, K, lane);
  if (lane == 0) *kth = x;
  int above = 0;
  for (int i = 0; i < C; i += 64) above += __builtin_popcountll(__ballot(i + lane < C && h[i + lane] > x));
  // ties at the K-th: the second words decide
  const uint64_t y = nth_of([=](int i) { return h[i] == x ? l[i] : 0; }, C, K - above, lane);
  int kept = 0;
  for (int i = 0; i < C; i += 64) {
    const uint64_t a = i + lane < C ? h[i + lane] : 0, c = i + lane < C ? l[i + lane] : 0;
    const bool win = a > x || (a != 0 && a == x && c >= y);
    const uint64_t m = __ballot(win);
    lds_wave_fence();
    if (win) {  // never past what has been read
      h[kept + lanes_below(m)] = a;
      l[kept + lanes_below(m)] = c;
    }
    lds_wave_fence();
    kept += __builtin_popcountll(m);
  }
  return kept;
}

// Pairs of one workgroup in LDS, ordered by hi, then lo.
struct PairList {
  uint64_t* hi;
  uint64_t* lo;
  int* n;  // above kPairs: some found no room

  // A wave's lanes with `pass` add their pairs.
  __device__ void add(bool pass, uint64_t h, uint64_t l, int lane) {
    const uint64_t m = __ballot(pass);
    if (m == 0) return;
    const int first = __builtin_ctzll(m);
    int at = 0;
    if (lane == first) at = atomicAdd(n, __builtin_popcountll(m));
    at = __builtin_amdgcn_readlane(at, first) + lanes_below(m);
    if (pass && at < kPairs) {
      hi[at] = h;
      lo[at] = l;
    }
  }
  // Keeps the K best if there are more than `most`, and raises *bound to the K-th's hi. All threads of
  // the workgroup together.
  __device__ void shrink(int most, int K, int wv, int lane, uint64_t* bound) {
    __syncthreads();
    const int have = *n;
    __syncthreads();  // every wave has read it: the branch is the same for all
    if (have > most) {
      if (wv == 0) {
        const int C = keep_best(hi, lo, have, K, lane, bound);
        if (lane == 0) *n = C;
      }
      __syncthreads();
    }
  }
};

// kRows: rows of a wave, at least W / 16. kHeld: units' maxima of a row that a lane holds: all (kAll), or the
// others are read again. kPerCu: workgroups that a CU's registers hold.
template <int DT, int kRows, int kHeld, bool kAll, int kPerCu>
__global__ __launch_bounds__(kMergeThreads, 4 * kPerCu) void hs_beam_merge_kernel(StepArgs A) {
  using Vt = Vec<DT>;
  using Raw = typename Vt::Raw;
  constexpr int E = Vt::kElems;
  constexpr int kMost = kAll ? kHeld * 64 / kUnits : 1 << 30;  // slices of a row
  __shared__ double s_off[HS_MAX_BEAMS], s_lse[HS_MAX_BEAMS];  // a row's log2 normaliser: their sum
  __shared__ float s_score[HS_MAX_BEAMS];
  __shared__ float s_least[HS_MAX_BEAMS];    // a row's logits below it do not reach the bound
  __shared__ uint8_t s_kind[HS_MAX_BEAMS];   // 0: gives nothing, 1: by its logits, 2: finished
  __shared__ uint32_t s_group[128];
  __shared__ __align__(16) uint64_t s_uhi[kPairs];
  __shared__ uint64_t s_ulo[kPairs], s_hi[kPairs], s_lo[kPairs];
  // (where s_uhi was, which is done with by then: 70 KB in all, so that a CU holds two workgroups)
  static_assert(sizeof(s_uhi) >= kMergeWaves * 64 * sizeof(Raw), "s_vec lies in s_uhi");
  Raw(*const s_vec)[64] = reinterpret_cast<Raw(*)[64]>(s_uhi);
  __shared__ uint8_t s_from[kMergeWaves][64], s_unit[kMergeWaves][64];
  __shared__ int s_units, s_count;
  __shared__ uint64_t s_bound;
  const int t = threadIdx.x, lane = t & 63;
  const int wv = __builtin_amdgcn_readfirstlane(t >> 6);
  const int b = blockIdx.x, W = A.W, S = A.S, K = A.K, nu = A.nu;
  const float* top = A.top + (int64_t)b * W * nu;
  const float c32 = (float)A.c;

  // a wave's rows are w = wv + 16 r; every load first (a row that gives nothing has records of
  // another call, which are not used)
  SliceRec r0[kRows], r1[kRows];
  float m[kRows][kHeld], sc[kRows];
  bool over[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int w = wv + kMergeWaves * r;
    if (w >= W) break;
    const SliceRec* rec = A.rec + ((int64_t)b * W + w) * S;
    r0[r] = rec[min(lane, S - 1)];
    if (kMost > 64) r1[r] = rec[min(lane + 64, S - 1)];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) m[r][i] = top[w * nu + min(lane + 64 * i, nu - 1)];
    sc[r] = A.score[(int64_t)b * A.score_stride + w];
    over[r] = A.done && A.done[(int64_t)b * A.score_stride + w];
  }
  if (t < 128) s_group[t] = 0;
  if (t == 0) {
    s_units = s_count = 0;
    s_bound = ~0ull;
  }
  __syncthreads();

  auto score_of = [&](int w, float z) -> uint64_t {
    return ordered_of((double)s_score[w] +
                      (((double)z * A.c - s_off[w]) - s_lse[w]) * 0.69314718055994530942);
  };
  // Entries fall into groups (a lane's of some rows), each with its largest score's upper half: the
  // K-th largest of them is a bound that K entries reach. Of random scores 18 reach the 16th of 64
  // groups, and 89 the 64th of 128.
  const int groups = K <= 16 ? 64 : 128;
  auto group_of = [&](int w) { return groups > 64 ? ((w / kMergeWaves + w) & 1) * 64 : 0; };

  // the rows' normalisers, and the groups' largest entries
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int w = wv + kMergeWaves * r;
    if (w >= W) break;
    const int kind = !isfinite(sc[r]) ? 0 : over[r] ? 2 : 1;
    if (kind != 1) {
      if (lane == 0) {
        s_score[w] = sc[r];
        s_kind[w] = (uint8_t)kind;
        if (kind == 2)
          atomicMax(&s_group[group_of(w)], (uint32_t)(ordered_of((double)sc[r]) >> 32));
      }
      continue;
    }
    const SliceRec* rec = A.rec + ((int64_t)b * W + w) * S;
    int best = fkey(r0[r].ref);
    if (kMost > 64) best = max(best, fkey(r1[r].ref));
    if (kMost > 128)
      for (int s = lane + 128; s < S; s += 64) best = max(best, fkey(rec[s].ref));
    const Offset to(fkey_inv(wave_max_i(best)), c32);  // the row's: from its largest reference
    double sum = 0.0;
    auto part = [&](const SliceRec& q, bool mine) {
      const Offset from(q.ref, c32);
      if (!__ballot(mine && (to.large || (from.large && q.ref != -INFINITY)))) {  // small offsets
        if (mine) sum += ldexp(q.sum, q.off - (int)to.o);
      } else if (mine) {
        sum += q.ref == -INFINITY ? q.sum : q.sum * exp2_of(from.value(A.c) - to.value(A.c));
      }
    };
    part(r0[r], lane < S);
    if (kMost > 64 && S > 64) part(r1[r], lane + 64 < S);
    if (kMost > 128)
      for (int s0 = 128; s0 < S; s0 += 64) part(rec[min(s0 + lane, S - 1)], s0 + lane < S);
    sum = wave_sum_d(sum);
    const bool live = isfinite(sum) && sum > 0.0;
    const double lg = log2_of(sum);
    if (lane == 0) {
      s_score[w] = sc[r];
      s_off[w] = to.value(A.c);
      s_lse[w] = lg;
      s_kind[w] = live ? 1 : 0;
    }
    lds_wave_fence();
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (lane + 64 * i < nu) most = fmaxf(most, m[r][i]);
    if (!kAll)
      for (int k = lane + 64 * kHeld; k < nu; k += 64) most = fmaxf(most, top[w * nu + k]);
    if (live && most > -INFINITY)
      atomicMax(&s_group[group_of(w) + lane], (uint32_t)(score_of(w, most) >> 32));
  }
  __syncthreads();
  // the smallest group that fewer than K exceed; 0 (no bound) with fewer than K groups. Each wave
  // looks at its share of them
  {
    const uint32_t g0 = s_group[lane], g1 = groups > 64 ? s_group[64 + lane] : 0;
    uint32_t least = 0xFFFFFFFFu;
    for (int j = wv; j < groups; j += kMergeWaves) {
      const uint32_t g = (uint32_t)__builtin_amdgcn_readlane((int)(j < 64 ? g0 : g1), j & 63);
      const int above = __builtin_popcountll(__ballot(g0 > g)) + __builtin_popcountll(__ballot(g1 > g));
      if (above < K) least = min(least, g);
    }
    if (lane == 0) atomicMin((unsigned long long*)&s_bound, (unsigned long long)least << 32);
  }
  __syncthreads();
  uint64_t bound = s_bound;

  // the units that reach it
  PairList units{s_uhi, s_ulo, &s_units};
  // a unit of a list, with its largest logit where lists are cut; larger: lower beam, larger logit, lower unit
  auto place = [](int w, uint32_t most, int k) {
    return ((uint64_t)(63 - w) << 58) | ((uint64_t)most << kTokenBits) | (uint64_t)(kTokenMask - (uint32_t)k);
  };
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int w = wv + kMergeWaves * r;
    if (w >= W) break;
    if (s_kind[w] != 1) continue;
    const double base = (double)s_score[w] * 1.4426950408889634074;
    const double at = (value_of(bound) * 1.4426950408889634074 - base + s_lse[w] + s_off[w]) * A.inv_c;
    const double slack = 1e-6 * (fabs(at) + (fabs(base) + fabs(s_off[w])) * A.inv_c);
    const float least = bound == 0 ? -FLT_MAX : fmaxf((float)(at - slack), -FLT_MAX);
    if (lane == 0) s_least[w] = least;
    uint64_t who[kHeld];  // lanes whose unit reaches it; one count for all of them
    int found = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      who[i] = __ballot(lane + 64 * i < nu && m[r][i] >= least);
      found += __builtin_popcountll(who[i]);
    }
    if (found) {
      int at = 0;
      if (lane == 0) at = atomicAdd(&s_units, found);
      at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        const int to = at + lanes_below(who[i]);
        if (((who[i] >> lane) & 1) && to < kPairs) s_ulo[to] = place(w, 0, lane + 64 * i);
        at += __builtin_popcountll(who[i]);
      }
    }
    for (int k0 = 64 * kHeld; !kAll && k0 < nu; k0 += 64) {
      const int k = k0 + lane;
      const bool pass = k < nu && top[w * nu + min(k, nu - 1)] >= least;
      units.add(pass, 0, place(w, 0, k), lane);
    }
  }
  __syncthreads();
  int n = s_units;
  // If they are too many (maxima of equal score), the 4 K first by (s, lower beam, larger maximum, lower unit) do,
  // which is the entries' order: all but three of them (units of its chunk, whose tokens lie between its
  // own) have an entry before any of a later unit. The logits decide where fp64 scores them the same
  // (large T, large scores)
  if (n > 4 * K + 64) {  // the same for all: nobody adds any more
    __syncthreads();
    if (t == 0) s_units = 0;
    __syncthreads();
    for (int i0 = 0; i0 < W * nu; i0 += kMergeThreads) {
      units.shrink(kPairs - kMergeThreads, 4 * K, wv, lane, &s_bound);
      bound = s_bound;
      const int i = i0 + t;
      uint64_t h = 0;
      const int w = i < W * nu ? (int)fdiv((uint32_t)i, A.divU) : 0;
      if (i < W * nu && s_kind[w] == 1 && top[i] > -INFINITY) h = score_of(w, top[i]);
      units.add(h != 0 && h >= bound, h, place(w, h ? ordered_of(top[i]) : 0, i - w * nu), lane);
    }
    units.shrink(4 * K, 4 * K, wv, lane, &s_bound);
    n = s_units;
    bound = s_bound;
  }

  // their entries, and the finished beams; a second time, keeping only the K best on the way, if they
  // are too many
  PairList best{s_hi, s_lo, &s_count};
  auto add_finished = [&]() {
    if (wv != 0) return;
    const bool ended = lane < W && s_kind[lane] == 2;
    const uint64_t h = ended ? ordered_of((double)s_score[lane]) : 0;
    best.add(ended && h >= bound, h, ((uint64_t)(63 - lane) << 58) | kTokenMask, lane);
  };
  auto row_of = [](uint64_t lo) { return 63 - (int)(lo >> 58); };
  auto first_vector = [](uint64_t lo, int l) {  // of lane l in a unit
    const int k = (int)(kTokenMask - ((uint32_t)lo & kTokenMask));
    return (k / kUnits) * kBeamChunk + (l >> 4) * 64 + (k % kUnits) * 16 + (l & 15);
  };
  auto fetch = [&](uint64_t lo) {
    const char* row = A.x + (int64_t)b * A.sb + (int64_t)row_of(lo) * A.sw;
    const int64_t vi = first_vector(lo, lane);
    return vi < A.nvec ? Vt::load_raw(row, vi, A.V) : Vt::neg_raw();
  };
  auto add_logit = [&](bool has, float y, uint64_t lo, int l, int e) {
    const int w = has ? row_of(lo) : 0;
    const uint64_t h = has ? score_of(w, y) : 0;
    best.add(has && h >= bound, h,
             ((uint64_t)(63 - w) << 58) | ((uint64_t)ordered_of(y) << kTokenBits) |
                 (uint64_t)(kTokenMask - ((uint32_t)first_vector(lo, l) * E + e)), lane);
  };
  add_finished();
  // four units of a wave at once, so that their loads are in flight together. The few lanes with a logit
  // that reaches the bound leave their vectors in LDS, and then every lane looks at one logit
  for (int i0 = wv; i0 < n; i0 += kMergeWaves * kAtOnce) {
    Raw x[kAtOnce];
    uint64_t of[kAtOnce];
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      if (i0 + q * kMergeWaves >= n) break;
      of[q] = uniform(s_ulo[i0 + q * kMergeWaves]);
      x[q] = fetch(of[q]);
    }
    int hits = 0;
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      if (i0 + q * kMergeWaves >= n) break;
      float z[E], most = -INFINITY;
      Vt::unpack(x[q], z);
#pragma unroll
      for (int e = 0; e < E; ++e) most = fmaxf(most, z[e]);
      const uint64_t who = __ballot(most >= s_least[row_of(of[q])]);
      const int at = hits + lanes_below(who);
      if (((who >> lane) & 1) && at < 64) {
        s_vec[wv][at] = x[q];
        s_from[wv][at] = (uint8_t)lane;
        s_unit[wv][at] = (uint8_t)q;
      }
      hits += __builtin_popcountll(who);
    }
    lds_wave_fence();
    if (hits > 64) {
      if (lane == 0) atomicAdd(&s_count, kPairs + 1);  // no room: the second way
      break;
    }
    for (int p = 0; p < hits; p += 64 / E) {
      const int at = p + lane / E, e = lane % E;
      const bool in = at < hits;
      uint64_t lo = of[0];
#pragma unroll
      for (int q = 1; q < kAtOnce; ++q) lo = in && s_unit[wv][at & 63] == q ? of[q] : lo;
      float y;
      if constexpr (DT == HS_F32) y = reinterpret_cast<const float*>(&s_vec[wv][at & 63])[e];
      else y = Vt::lo(reinterpret_cast<const uint16_t*>(&s_vec[wv][at & 63])[e]);
      add_logit(in && y >= s_least[row_of(lo)], y, lo, s_from[wv][at & 63], e);
    }
    lds_wave_fence();
  }
  __syncthreads();
  if (s_count > kPairs) {  // the same for all: nobody adds any more
    __syncthreads();
    if (t == 0) s_count = 0;
    __syncthreads();
    add_finished();
    for (int i0 = 0; i0 < n; i0 += kMergeWaves) {
      best.shrink(kPairs - kMergeWaves * 64, K, wv, lane, &s_bound);
      bound = s_bound;
      const int i = i0 + wv;
      if (i >= n) continue;
      const uint64_t lo = uniform(s_ulo[i]);
      const float least = s_least[row_of(lo)];
      const uint32_t token = (uint32_t)first_vector(lo, lane) * E;
      float z[E];
      Vt::unpack(fetch(lo), z);
      uint32_t pass = 0;  // of the lane's logits
#pragma unroll
      for (int e = 0; e < E; ++e) pass |= z[e] >= least ? 1u << e : 0u;
      if (wave_sum_i(__builtin_popcount(pass)) > 64) {  // the unit's K best: by logit, by token
        auto count = [&](auto reaches) {
          int c = 0;
#pragma unroll
          for (int e = 0; e < E; ++e)
            c += __builtin_popcountll(__ballot(((pass >> e) & 1) != 0 && reaches(e)));
          return c;
        };
        uint32_t cut = 0, last = 0;
        for (int bit = 31; bit >= 0; --bit) {
          const uint32_t y = cut | (1u << bit);
          if (count([&](int e) { return ordered_of(z[e]) >= y; }) >= K) cut = y;
        }
        const int left = K - count([&](int e) { return ordered_of(z[e]) > cut; });
        for (int bit = kTokenBits - 1; bit >= 0; --bit) {
          const uint32_t y = last | (1u << bit);
          if (count([&](int e) { return ordered_of(z[e]) == cut && kTokenMask - (token + e) >= y; }) >= left)
            last = y;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint32_t u = ordered_of(z[e]);
          if (u < cut || (u == cut && kTokenMask - (token + e) < last)) pass &= ~(1u << e);
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (__ballot((pass >> e) & 1)) add_logit((pass >> e) & 1, z[e], lo, lane, e);
    }
    __syncthreads();
  }
  int C = s_count;
  if (C > 256) {  // what a wave can rank
    best.shrink(256, K, wv, lane, &s_bound);
    C = s_count;
  }
  // every entry's rank: a wave takes every 16th, one a lane, and compares them one after the other with all
  uint64_t h[4], l[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    h[j] = j * 64 + lane < C ? s_hi[j * 64 + lane] : 0;
    l[j] = j * 64 + lane < C ? s_lo[j * 64 + lane] : 0;
  }
  const int i = wv + kMergeWaves * lane;
  const uint64_t hi = i < C ? s_hi[i] : 0, lo = i < C ? s_lo[i] : 0;
  int at = i;  // past the last entry: an empty slot
  for (int q = 0; wv + kMergeWaves * q < C; ++q) {
    const uint64_t qh = lane_u(hi, q), ql = lane_u(lo, q);
    int above = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j * 64 < C)
        above += __builtin_popcountll(__ballot(h[j] > qh || (h[j] == qh && l[j] > ql)));
    at = lane == q ? above : at;
  }
  if (at < K) {  // (lanes past the entries and slots have i >= K)
    const int parent = i < C ? 63 - (int)(lo >> 58) : -1;
    const bool was = i < C && s_kind[max(parent, 0)] == 2;
    const int token = i >= C ? -1 : was ? A.eos : (int)(kTokenMask - ((uint32_t)lo & kTokenMask));
    const int64_t o = (int64_t)b * K + at;
    A.out_score[o] = i < C ? (float)value_of(hi) : -INFINITY;
    A.out_parent[o] = parent;
    A.out_token[o] = token;
    if (A.out_done) A.out_done[o] = was || (i < C && A.eos >= 0 && token == A.eos) ? 1 : 0;
  }
}

// The smallest kernel that does. us with one kernel for all (4 rows, 5 maxima), with 5 and 10 maxima for the rows there
// are, and with this rule: 10 rows of 300 units 10.8, 10.4, 10.9 and 10.3; 15 of 536 15.6, 15.3, 14.0 and 14.0; 4 of
// 128 9.6, 9.2, 9.6 and 9.0; 64 of 64 27.7, 27.6, 27.6 and 25.9.
// Two workgroups per CU where there are more than CUs: 4000 x 1 rows of 4000 bf16 82 -> 54 us, 1024 x 2 of 8000 29 -> 23;
// 13 x 5 of 50257 10.4 -> 10.7.
template <int DT, int ROWS, int HELD, bool ALL>
void launch_merge_of(const StepArgs& A, int B, hipStream_t st) {
  constexpr int kMany = ROWS * HELD <= 10 ? 2 : 1;
  if (B > 256) hs_beam_merge_kernel<DT, ROWS, HELD, ALL, kMany><<<B, kMergeThreads, 0, st>>>(A);
  else hs_beam_merge_kernel<DT, ROWS, HELD, ALL, 1><<<B, kMergeThreads, 0, st>>>(A);
}
template <int DT, int ROWS>
void launch_merge(const StepArgs& A, int B, hipStream_t st) {
  if (A.nu <= 128) launch_merge_of<DT, ROWS, 2, true>(A, B, st);
  else if (A.nu <= 320) launch_merge_of<DT, ROWS, 5, true>(A, B, st);
  else launch_merge_of<DT, ROWS, (ROWS > 2 ? 5 : 10), false>(A, B, st);
}

template <int DT>
void launch_step(StepArgs A, int B, hipStream_t st) {
  const uint32_t groups = (A.units + kWaves - 1) / kWaves;
  for (A.group0 = 0; A.group0 < groups; A.group0 += kMostGroups) {
    hs_beam_rows_kernel<DT><<<std::min(groups - A.group0, kMostGroups), kThreads, 0, st>>>(A);
    if (hipPeekAtLastError() != hipSuccess) return;
  }
  if (A.W <= kMergeWaves) launch_merge<DT, 1>(A, B, st);
  else if (A.W <= 2 * kMergeWaves) launch_merge<DT, 2>(A, B, st);
  else launch_merge<DT, HS_MAX_BEAMS / kMergeWaves>(A, B, st);
}

}  // namespace

// One wave per slice, of two chunks (the second one's loads fly while the first is summed), or of one where
// that leaves the device's 8192 waves unfilled. us with one, two, three and four chunks: 10 x 75 chunks 11.0,
// 11.6, 12.0, 12.8; 8064 of 128 rows 16.1, 15.8, 16.1, 15.8; 16128 22.5, 21.3, 22.5, 22.3; 32256 32.7, 30.8,
// 30.4, 31.6; 76800 78.8, 67.4, 66.9, 69.3; 64 x 8 fp32 rows of 126 53.1, 49.0, 50.1, 52.1.
bool beam_geom(int B, int W, int K, int64_t V, int dtype, BeamGeom* g) {
  if (B < 1 || W < 1 || K < 1 || V < 1) return false;
  if (B > HS_MAX_QUERIES || W > HS_MAX_BEAMS || K > HS_MAX_BEAMS || V > INT32_MAX) return false;
  if (dtype != HS_F32 && dtype != HS_BF16 && dtype != HS_F16) return false;
  const int E = dtype == HS_F32 ? 4 : 8;
  g->B = B;
  g->W = W;
  g->K = K;
  g->V = V;
  g->nvec = (V + E - 1) / E;
  g->dtype = dtype;
  if (g->nvec > (int64_t)kMaxTeamSlices * kThreads) return false;
  g->nc = (int)((g->nvec + kBeamChunk - 1) / kBeamChunk);
  g->chunks = g->nc > 1 && (int64_t)g->nc * B * W >= 8000 ? 2 : 1;
  g->S = (g->nc + g->chunks - 1) / g->chunks;
  return true;
}

size_t beam_ws_bytes(const BeamGeom& g) {
  const size_t rows = (size_t)g.B * g.W;
  return align256(rows * g.S * sizeof(SliceRec)) + align256(rows * g.nc * kUnits * sizeof(float));
}

int launch_beam_step(const BeamGeom& g, const hs_beam_args& a, hipStream_t stream) {
  StepArgs A;
  const int64_t es = g.dtype == HS_F32 ? 4 : 2;
  A.x = reinterpret_cast<const char*>(a.logits.ptr);
  A.sb = a.logits.stride_b * es;
  A.sw = a.logits.stride_k * es;
  A.W = g.W;
  A.K = g.K;
  A.S = g.S;
  A.chunks = g.chunks;
  A.nc = g.nc;
  A.nu = g.nc * kUnits;
  A.V = g.V;
  A.nvec = g.nvec;
  A.score_stride = a.score_stride;
  A.units = (uint32_t)((int64_t)g.B * g.W * g.S);
  A.divS = make_fastdiv((uint32_t)g.S);
  A.divW = make_fastdiv((uint32_t)g.W);
  A.divU = make_fastdiv((uint32_t)A.nu);
  A.c = 1.4426950408889634074 / a.temperature;
  A.inv_c = 1.0 / A.c;
  // ca: the top 12 bits of c; cb: the rest, above 0 so that -inf stays -inf in z cb + (z ca - offset)
  uint64_t bits;
  __builtin_memcpy(&bits, &A.c, 8);
  bits &= ~((1ull << 41) - 1);
  double ca;
  __builtin_memcpy(&ca, &bits, 8);
  A.ca = (float)ca;
  A.cb = fmaxf((float)(A.c - ca), 1e-37f);
  A.score = a.score;
  A.done = a.done;
  A.eos = a.eos;
  A.out_score = a.out_score;
  A.out_parent = a.out_parent;
  A.out_token = a.out_token;
  A.out_done = a.out_done;
  char* ws = reinterpret_cast<char*>(a.workspace);
  A.rec = reinterpret_cast<SliceRec*>(ws);
  A.top = reinterpret_cast<float*>(ws + align256((size_t)A.units * sizeof(SliceRec)));
  if (g.dtype == HS_F32) launch_step<HS_F32>(A, g.B, stream);
  else if (g.dtype == HS_F16) launch_step<HS_F16>(A, g.B, stream);
  else launch_step<HS_BF16>(A, g.B, stream);
  return hipPeekAtLastError() == hipSuccess ? HS_OK : HS_ERR_HIP;
}

}  // namespace hs
