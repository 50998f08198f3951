// hs_beam_step: the K best continuations of a query's W beams by
//   s(w, v) = score_w + log softmax(z_w / T)_v = score_w + (z_wv c - lse2_w) ln 2,
// c = log2(e) / T, lse2_w = log2 sum_v 2^(z_wv c). Within a beam the order of s is the order of the
// logits, so a beam's row needs one pass that keeps a sum and the K largest logits; only the rows'
// normalisers decide between beams. Two launches:
//   1. hs_beam_slice_kernel: a wave reads one slice of a row once and leaves its exp2 sum and
//      its K largest logits as keys (value, then lower token), largest first;
//   2. hs_beam_merge_kernel, one workgroup per query: the rows' normalisers from the slices' sums,
//      then the K best of the slices' lists by (s, lower beam, larger logit, lower token). A slice
//      whose first key lies below the K-th largest of some others' cannot hold any of them, so that
//      only about K lists are read.
//
// Precision. Two beams' candidates are often closer than fp32 tells apart and the order is part of
// the result, so s is formed in fp64 and the normalisers are made good to about 1e-8: z c is taken
// as z ca + z cb with ca = c rounded to 12 bits (for 16-bit logits z ca - offset is exact), each
// lane adds its fp32 exponentials per chunk and the chunks in fp64, and the exponentials of a slice's
// K largest logits, most of the sum where the distribution is peaked, are replaced by fp64 ones.
// Sums are relative to an offset near the slice's maximum, and a slice whose maximum is large
// (|z c| > 4096) takes z - maximum first, so that logits of any size do, the lowest finite value
// in every place included.
#include "hs_beam.h"

namespace hs {

namespace {

constexpr int kCap = 512;        // keys of one slice held in LDS
constexpr int kMergeCap = 1024;  // candidates of one query held in LDS
constexpr int kTokenBits = 26;
constexpr int64_t kTokenMask = (1 << kTokenBits) - 1;

struct SliceRec {
  double sum;  // of 2^(z c - off) over the slice (not finite: a NaN or +inf logit)
  double off;  // -inf: no logit above -inf
  int count;   // keys in the slice's list
};

// The offset of a slice's exponents, from the largest logit m of its first chunk that has any.
struct Offset {
  double off;  // in log2 units; -inf: none yet
  float o;     // the same for small ones (an integer at or above m c)
  float ref;   // m, which large ones subtract first
  bool large;
  __device__ void set(float m, float c, double c64) {
    ref = m;
    large = !(fabsf(m * c) <= 4096.0f);
    o = large ? 0.0f : ceilf(m * c);
    off = large ? (double)m * c64 : (double)o;
  }
  // the exponent of a logit
  __device__ float exponent(float z, float ca, float cb) const {
    if (large) {
      const float d = z - ref;
      return fmaf(d, cb, d * ca);
    }
    return fmaf(z, cb, fmaf(z, ca, -o));
  }
};

struct StepArgs {
  const char* x;
  int64_t sb, sw;  // bytes between queries and between beams
  int W, K, S, chunks;
  int64_t V, nvec, score_stride;
  uint32_t units;  // B * W * S
  FastDiv divS, divW, divK;
  float ca, cb;
  double c;
  const float* score;
  const uint8_t* done;
  int eos;
  float* out_score;
  int32_t* out_parent;
  int32_t* out_token;
  uint8_t* out_done;
  uint64_t* key;   // [B * W][S][K]
  SliceRec* rec;   // [B * W][S]
};

// A beam that continues by its logits: a finite score, and not finished.
__device__ inline bool beam_grows(const StepArgs& A, int b, int w) {
  const int64_t i = (int64_t)b * A.score_stride + w;
  return isfinite(A.score[i]) && !(A.done && A.done[i]);
}

__device__ inline uint64_t logit_key(float z, int64_t token) {
  return ((uint64_t)ordered_of(z) << 32) | (0xFFFFFFFFu - (uint32_t)token);
}

template <int DT>
__device__ inline float logit_at(const char* row, int64_t v) {
  if constexpr (DT == HS_F32) return reinterpret_cast<const float*>(row)[v];
  else return Vec<DT>::lo(reinterpret_cast<const uint16_t*>(row)[v]);
}

template <int DT>
__device__ inline void load_chunk(const char* row, int64_t v0, int64_t nvec, int64_t V, int lane,
                                  typename Vec<DT>::Raw (&x)[4]) {
  if ((v0 + kBeamChunk) * Vec<DT>::kElems <= V) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      typedef unsigned int u4 __attribute__((ext_vector_type(4)));
      typedef const __attribute__((address_space(1))) u4* gp4;
      const u4 y = *(gp4)(row + (v0 + i * 64 + lane) * 16);
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

// The K largest of the wave's C <= kCap keys to the front of buf, largest first; how many there are.
__device__ inline int keep_best(uint64_t* buf, int C, int K, int lane) {
  lds_wave_fence();
  if (C > 64) {
    uint64_t u[kCap / 64];
    const int nu = (C + 63) / 64;
#pragma unroll
    for (int j = 0; j < kCap / 64; ++j) u[j] = j * 64 + lane < C ? buf[j * 64 + lane] : 0;
    const uint64_t x = nth_largest(u, nu, K);
    lds_wave_fence();
    C = 0;
#pragma unroll
    for (int j = 0; j < kCap / 64; ++j) {
      const bool win = u[j] != 0 && u[j] >= x;
      const uint64_t m = __ballot(win);
      if (win) buf[C + lanes_below(m)] = u[j];
      C += __builtin_popcountll(m);
    }
    lds_wave_fence();
  }
  if (lane < 16) buf[C + lane] = 0;
  lds_wave_fence();
  const uint64_t mine = lane < C ? buf[lane] : 0;
  const int rank = count_above(buf, C, mine);
  lds_wave_fence();
  if (lane < C && rank < K) buf[rank] = mine;
  lds_wave_fence();
  return min(C, K);
}

// A value that at least K of the wave's logits reach: the K-th largest lane maximum (its last 6 bits
// rounded down to make room for the lane number, which makes the keys distinct), as the largest
// value below it, so that `z > bound` passes them. -inf where fewer than K lanes have a logit.
__device__ inline float lane_bound(float lmax, int K, int lane, int* s_lane) {
  const int key = (fkey(lmax) & ~63) | (63 - lane);
  s_lane[lane] = key;
  lds_wave_fence();
  typedef int i4 __attribute__((ext_vector_type(4)));
  int r = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const i4 v = reinterpret_cast<const i4*>(s_lane)[i];
    r += (v[0] > key ? 1 : 0) + (v[1] > key ? 1 : 0) + (v[2] > key ? 1 : 0) + (v[3] > key ? 1 : 0);
  }
  const uint64_t who = __ballot(r == K - 1);  // one lane
  const int k = __builtin_amdgcn_readlane(key, __builtin_ctzll(who)) & ~63;
  lds_wave_fence();
  if (k <= (fkey(-INFINITY) | 63)) return -INFINITY;
  const float v = fkey_inv(k);
  return v == 0.0f ? -__int_as_float(1) : fkey_inv(k - 1);
}

template <int DT>
__global__ __launch_bounds__(kThreads) void hs_beam_slice_kernel(StepArgs A) {
  using Vt = Vec<DT>;
  using Raw = typename Vt::Raw;
  constexpr int E = Vt::kElems;
  __shared__ __attribute__((aligned(16))) uint64_t s_key[kWaves][kCap + 16];
  __shared__ __attribute__((aligned(16))) int s_lane[kWaves][64];
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t u = blockIdx.x * kWaves + wv;
  if (u >= A.units) return;  // wave-uniform; the waves share no barrier
  const uint32_t row = fdiv(u, A.divS);
  const int s = (int)(u - row * (uint32_t)A.S);
  const int b = (int)fdiv(row, A.divW), w = (int)row - b * A.W;
  SliceRec* rec = A.rec + u;
  if (!beam_grows(A, b, w)) {
    if (lane == 0) *rec = SliceRec{0.0, -(double)INFINITY, 0};
    return;
  }
  const char* rowp = A.x + (int64_t)b * A.sb + (int64_t)w * A.sw;
  const int64_t v0 = (int64_t)s * A.chunks * kBeamChunk;
  const int64_t vend = min(A.nvec, v0 + (int64_t)A.chunks * kBeamChunk);
  uint64_t* buf = s_key[wv];
  const float c = (float)A.c;

  Offset off;
  off.off = -INFINITY;
  off.o = off.ref = 0.0f;
  off.large = false;
  double sum = 0.0;         // the lane's
  int C = 0;                // keys in buf
  bool sorted = true;
  uint64_t kth = 0;         // the K-th best key, once there are K
  Raw cur[4], nxt[4];
  load_chunk<DT>(rowp, v0, A.nvec, A.V, lane, cur);
  for (int64_t v = v0; v < vend; v += kBeamChunk) {
    if (v + kBeamChunk < vend) load_chunk<DT>(rowp, v + kBeamChunk, A.nvec, A.V, lane, nxt);
    float z[4][E], vmax[4], lmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      Vt::unpack(cur[i], z[i]);
      vmax[i] = -INFINITY;
#pragma unroll
      for (int e = 0; e < E; ++e) vmax[i] = fmaxf(vmax[i], z[i][e]);
      lmax = fmaxf(lmax, vmax[i]);
    }
    // the offset stays while no exponent exceeds 4, so that a slice rarely changes it and the
    // rounding of z c - off stays that of small numbers
    if (off.off == -INFINITY || __ballot(off.exponent(lmax, A.ca, A.cb) > 4.0f)) {
      float m = lmax;
      int none = 0;
      wave_max<false>(m, none);
      if (m != -INFINITY) {
        const double before = off.off;
        off.set(m, c, A.c);
        if (before != -INFINITY) sum *= exp2(before - off.off);
      }
    }
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    if (off.large) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float d = z[i][e] - off.ref;
          acc[e & 3] += __builtin_amdgcn_exp2f(fmaf(d, A.cb, d * A.ca));
        }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e)
          acc[e & 3] += __builtin_amdgcn_exp2f(fmaf(z[i][e], A.cb, fmaf(z[i][e], A.ca, -off.o)));
    }
    sum += (double)((acc[0] + acc[1]) + (acc[2] + acc[3]));

    // candidates. Tokens of later chunks are higher, so an equal logit no longer counts there
    const bool first = C < A.K;
    const float bound = first ? lane_bound(lmax, A.K, lane, s_lane[wv])
                              : value_of((uint32_t)(kth >> 32));
    const int C0 = C;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!__ballot(vmax[i] > bound)) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const bool p = z[i][e] > bound;
        const uint64_t m = __ballot(p);
        if (m) {
          const int at = C + lanes_below(m);
          if (p && at < kCap) buf[at] = logit_key(z[i][e], (v + i * 64 + lane) * E + e);
          C += __builtin_popcountll(m);
        }
      }
    }
    if (C > kCap) {
      // more than the list holds (long runs of rising or equal logits): the chunk again, one element
      // of every lane at a time, with room made before each
      C = C0;
      for (int j = 0; j < 4 * E; ++j) {
        const int64_t t = (v + (j / E) * 64 + lane) * E + j % E;
        const float y = t < A.V ? logit_at<DT>(rowp, t) : -INFINITY;
        const uint64_t k = y > -INFINITY ? logit_key(y, t) : 0;
        if (C + 64 > kCap) {
          C = keep_best(buf, C, A.K, lane);
          kth = C == A.K ? uniform(buf[A.K - 1]) : 0;
        }
        const uint64_t m = __ballot(k > kth);
        if (k > kth) buf[C + lanes_below(m)] = k;
        C += __builtin_popcountll(m);
      }
      sorted = false;
    }
    if (C != C0) sorted = false;
    if (!sorted && (first || C > 64)) {
      C = keep_best(buf, C, A.K, lane);
      kth = C == A.K ? uniform(buf[A.K - 1]) : 0;
      sorted = true;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) cur[i] = nxt[i];
  }
  if (!sorted) C = keep_best(buf, C, A.K, lane);
  lds_wave_fence();
  const uint64_t mine = lane < C ? buf[lane] : 0;
  uint64_t* out = A.key + (int64_t)u * A.K;
  if (lane < A.K) out[lane] = mine;
  double fix = 0.0;
  if (lane < C) {
    const float zk = value_of((uint32_t)(mine >> 32));
    fix = exp2((double)zk * A.c - off.off) -
          (double)__builtin_amdgcn_exp2f(off.exponent(zk, A.ca, A.cb));
  }
  double tot = sum;
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) {
    tot += __shfl_xor(tot, i, 64);
    fix += __shfl_xor(fix, i, 64);
  }
  if (lane == 0) *rec = SliceRec{tot + fix, off.off, C};
}

// The K best of C <= kMergeCap pairs to the front of (hi, lo), best first; how many there are. One wave.
__device__ inline int keep_best_pairs(uint64_t* hi, uint64_t* lo, int C, int K, int lane) {
  constexpr int NU = kMergeCap / 64;
  lds_wave_fence();
  if (C > 64) {
    uint64_t h[NU], l[NU];
    const int nu = (C + 63) / 64;
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const int i = j * 64 + lane;
      h[j] = i < C ? hi[i] : 0;
      l[j] = i < C ? lo[i] : 0;
    }
    const uint64_t x = nth_largest(h, nu, K);
    int above = 0, equal = 0;
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      above += __builtin_popcountll(__ballot(h[j] > x));
      equal += __builtin_popcountll(__ballot(h[j] != 0 && h[j] == x));
    }
    uint64_t y = 0;
    if (above + equal > K) {  // ties at the K-th: the second words decide
      uint64_t t[NU];
#pragma unroll
      for (int j = 0; j < NU; ++j) t[j] = h[j] != 0 && h[j] == x ? l[j] : 0;
      y = nth_largest(t, nu, K - above);
    }
    lds_wave_fence();
    C = 0;
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const bool win = h[j] > x || (h[j] != 0 && h[j] == x && l[j] >= y);
      const uint64_t m = __ballot(win);
      const int at = C + lanes_below(m);
      if (win) {
        hi[at] = h[j];
        lo[at] = l[j];
      }
      C += __builtin_popcountll(m);
    }
    lds_wave_fence();
  }
  const uint64_t mh = lane < C ? hi[lane] : 0, ml = lane < C ? lo[lane] : 0;
  int rank = 0;
  for (int i = 0; i < C; ++i) {
    const uint64_t oh = hi[i], ol = lo[i];
    rank += oh > mh || (oh == mh && ol > ml) ? 1 : 0;
  }
  lds_wave_fence();
  if (lane < C && rank < K) {
    hi[rank] = mh;
    lo[rank] = ml;
  }
  lds_wave_fence();
  return min(C, K);
}

__global__ __launch_bounds__(kThreads) void hs_beam_merge_kernel(StepArgs A) {
  __shared__ double s_off[HS_MAX_BEAMS], s_lse[HS_MAX_BEAMS];  // a row's log2 normaliser: their sum
  __shared__ double s_score[HS_MAX_BEAMS];
  __shared__ uint8_t s_kind[HS_MAX_BEAMS];   // 0: gives nothing, 1: by its logits, 2: finished
  __shared__ uint64_t s_head[kThreads];
  __shared__ uint16_t s_list[HS_MAX_BEAMS * kBeamMaxSlices];
  __shared__ uint64_t s_hi[kMergeCap], s_lo[kMergeCap];
  __shared__ int s_lists, s_count;
  __shared__ uint64_t s_bound;
  const int t = threadIdx.x, lane = t & 63, wv = t >> 6;
  const int b = blockIdx.x, W = A.W, S = A.S, K = A.K;
  const SliceRec* rec = A.rec + (int64_t)b * W * S;
  const uint64_t* key = A.key + (int64_t)b * W * S * K;
  if (t == 0) s_lists = s_count = 0;

  // the rows' normalisers
  for (int w = wv; w < W; w += kWaves) {
    const float sc = A.score[(int64_t)b * A.score_stride + w];
    const bool over = A.done && A.done[(int64_t)b * A.score_stride + w];
    double o = -INFINITY;
    for (int s = lane; s < S; s += 64) o = fmax(o, rec[w * S + s].off);
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) o = fmax(o, __shfl_xor(o, i, 64));
    double sum = 0.0;
    for (int s = lane; s < S; s += 64) {
      const SliceRec r = rec[w * S + s];
      sum += r.off == -INFINITY ? r.sum : r.sum * exp2(r.off - o);
    }
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) sum += __shfl_xor(sum, i, 64);
    if (lane == 0) {
      s_score[w] = (double)sc;
      s_off[w] = o;
      s_lse[w] = log2(sum);
      s_kind[w] = !isfinite(sc) ? 0 : over ? 2 : isfinite(sum) && sum > 0.0 ? 1 : 0;
    }
  }
  __syncthreads();
  // the score of a slice's key (0 for none); a finished beam has one entry, in its first slice
  auto score_of = [&](int w, int s, int j, uint64_t k) -> uint64_t {
    if (s_kind[w] == 1 && k != 0)
      return ordered_of(s_score[w] +
                        (((double)value_of((uint32_t)(k >> 32)) * A.c - s_off[w]) - s_lse[w]) *
                            0.69314718055994530942);
    if (s_kind[w] == 2 && s == 0 && j == 0) return ordered_of(s_score[w]);
    return 0;
  };
  auto head_of = [&](int i) -> uint64_t {
    const int w = i / S, s = i - w * S;
    const uint64_t k = s_kind[w] == 1 && rec[i].count > 0 ? key[(int64_t)i * K] : 0;
    return score_of(w, s, 0, k);
  };

  // a bound that K entries reach: the K-th largest of 64 groups' largest first entries
  uint64_t best = 0;
  for (int i = t; i < W * S; i += kThreads) best = max(best, head_of(i));
  s_head[t] = best;
  __syncthreads();
  if (wv == 0) {
    uint64_t u[1] = {max(max(s_head[lane], s_head[lane + 64]),
                         max(s_head[lane + 128], s_head[lane + 192]))};
    const int have = __builtin_popcountll(__ballot(u[0] != 0));
    const uint64_t x = have >= K ? nth_largest(u, 1, K) : 1;
    if (lane == 0) s_bound = x;
  }
  __syncthreads();
  for (int i = t; i < W * S; i += kThreads) {
    const uint64_t h = head_of(i);
    if (h != 0 && h >= s_bound) s_list[atomicAdd(&s_lists, 1)] = (uint16_t)i;
  }
  __syncthreads();
  const int items = s_lists * K;
  for (int i0 = 0; i0 < items; i0 += kThreads) {
    const int i = i0 + t;
    if (i < items) {
      const int n = (int)fdiv((uint32_t)i, A.divK), j = i - n * K;
      const int q = s_list[n], w = q / S, s = q - w * S;
      const uint64_t k = s_kind[w] == 1 && j < rec[q].count ? key[(int64_t)q * K + j] : 0;
      const uint64_t h = score_of(w, s, j, k);
      if (h != 0 && h >= s_bound) {
        const int at = atomicAdd(&s_count, 1);
        s_hi[at] = h;
        // among equal scores the lower beam, the larger logit, the lower token
        const uint64_t token = k != 0 ? 0xFFFFFFFFu - (uint32_t)k : 0;
        s_lo[at] = ((uint64_t)(63 - w) << 58) | ((k >> 32) << kTokenBits) |
                   (uint64_t)(kTokenMask - (int64_t)token);
      }
    }
    if (items <= kMergeCap) continue;  // nothing can overflow
    __syncthreads();
    const int have = s_count;
    __syncthreads();  // every wave has read it: the branch is the same for all
    if (have > kMergeCap - kThreads) {
      if (wv == 0) {
        const int C = keep_best_pairs(s_hi, s_lo, s_count, K, lane);
        if (lane == 0) {
          s_count = C;
          if (C == K) s_bound = s_hi[K - 1];
        }
      }
      __syncthreads();
    }
  }
  __syncthreads();
  if (wv != 0) return;
  const int C = keep_best_pairs(s_hi, s_lo, s_count, K, lane);
  if (lane < K) {
    const int64_t o = (int64_t)b * K + lane;
    float sc = -INFINITY;
    int parent = -1, token = -1;
    uint8_t over = 0;
    if (lane < C) {
      sc = (float)value_of(s_hi[lane]);
      parent = 63 - (int)(s_lo[lane] >> 58);
      const bool was = s_kind[parent] == 2;
      token = was ? A.eos : (int)(kTokenMask - (int64_t)(s_lo[lane] & kTokenMask));
      over = was || (A.eos >= 0 && token == A.eos) ? 1 : 0;
    }
    A.out_score[o] = sc;
    A.out_parent[o] = parent;
    A.out_token[o] = token;
    if (A.out_done) A.out_done[o] = over;
  }
}

template <int DT>
void launch_step(const StepArgs& A, int B, hipStream_t st) {
  hs_beam_slice_kernel<DT><<<(A.units + kWaves - 1) / kWaves, kThreads, 0, st>>>(A);
  if (hipGetLastError() != hipSuccess) return;
  hs_beam_merge_kernel<<<B, kThreads, 0, st>>>(A);
}

}  // namespace

// One wave per slice: as many slices as give the device its 8192 resident waves, of one chunk at least.
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
  const int64_t all = (g->nvec + kBeamChunk - 1) / kBeamChunk;  // chunks of a row
  int64_t n = all * B * W / 8192;
  n = n < 1 ? 1 : n;
  const int64_t least = (all + kBeamMaxSlices - 1) / kBeamMaxSlices;
  n = n < least ? least : n > all ? all : n;
  g->chunks = (int)n;
  g->S = (int)((all + n - 1) / n);
  return true;
}

size_t beam_ws_bytes(const BeamGeom& g) {
  const size_t slices = (size_t)g.B * g.W * g.S;
  return align256(slices * g.K * 8) + align256(slices * sizeof(SliceRec));
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
  A.V = g.V;
  A.nvec = g.nvec;
  A.score_stride = a.score_stride;
  A.units = (uint32_t)((int64_t)g.B * g.W * g.S);
  A.divS = make_fastdiv((uint32_t)g.S);
  A.divW = make_fastdiv((uint32_t)g.W);
  A.divK = make_fastdiv((uint32_t)g.K);
  A.c = 1.4426950408889634074 / a.temperature;
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
  A.key = reinterpret_cast<uint64_t*>(ws);
  A.rec = reinterpret_cast<SliceRec*>(ws + align256((size_t)A.units * g.K * 8));
  if (g.dtype == HS_F32) launch_step<HS_F32>(A, g.B, stream);
  else if (g.dtype == HS_F16) launch_step<HS_F16>(A, g.B, stream);
  else launch_step<HS_BF16>(A, g.B, stream);
  return hipGetLastError() == hipSuccess ? HS_OK : HS_ERR_HIP;
}

}  // namespace hs
