// hs_cache_append: keys and values of new tokens to a paged cache in 8 bits.
//
// For each page that gets tokens, each head, keys and values by themselves: the largest |x| of the new rows, the
// least power of two that brings it to 448 or below, and the codes. Where the page's scale grows, the codes that are
// there follow. One workgroup does a page and head, so that nothing is shared between workgroups.
#include <algorithm>

#include "hs_draft.h"

namespace hs {

namespace {

struct AppendArgs {
  const char* x[2];  // keys, values
  int64_t xb[2], xn[2], xh[2];  // bytes
  uint8_t* cache[2];
  float* scale[2];
  int B, rows, taken, kv, page, shift, dim, span, slots;
  int64_t pages;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* length;
  const int32_t* path;
  int64_t path_stride;
  const int32_t* count;
  uint32_t units, group0;  // B * kv * span
  FastDiv div_span, div_kv, div_vec;
};

constexpr float kTop = 448.0f;
constexpr int kHold = 2;                     // squares of a thread
constexpr int kSlab = 64;                  // dims of a page's values that are in LDS at once
constexpr int kPitch = HS_MAX_PAGE / 4 + 1;  // words of a dim
constexpr uint32_t kNan8 = 0x7F;

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

__device__ inline bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// Four values as codes, the first in the low byte.
__device__ inline uint32_t codes_of(const float (&y)[4]) {
  float z[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = fminf(fmaxf(y[i], -kTop), kTop);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], r, true);
  uint32_t u = (uint32_t)r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (!finite(y[i])) u = (u & ~(0xFFu << (8 * i))) | (kNan8 << (8 * i));
  return u;
}
__device__ inline uint32_t rescaled(uint32_t u, float f) {
  const float y[4] = {__builtin_amdgcn_cvt_f32_fp8(u, 0) * f, __builtin_amdgcn_cvt_f32_fp8(u, 1) * f,
                      __builtin_amdgcn_cvt_f32_fp8(u, 2) * f, __builtin_amdgcn_cvt_f32_fp8(u, 3) * f};
  return codes_of(y);
}

// Eight values as codes of x / now, now a power of two, |x| <= 448 now.
template <bool F16>
__device__ inline uint2 plain_codes(const uint4& r, float now) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  i16x2 y[2] = {};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (F16) {
      y[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(y[i], __builtin_bit_cast(f16x2, w[2 * i]), now, false);
      y[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(y[i], __builtin_bit_cast(f16x2, w[2 * i + 1]), now, true);
    } else {
      y[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(y[i], __builtin_bit_cast(bf16x2, w[2 * i]), now, false);
      y[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(y[i], __builtin_bit_cast(bf16x2, w[2 * i + 1]), now, true);
    }
  }
  return make_uint2(__builtin_bit_cast(uint32_t, y[0]), __builtin_bit_cast(uint32_t, y[1]));
}

// Four words of four bytes, bytes and words exchanged.
__device__ inline void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t* u) {
  const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x05010400u), cd = __builtin_amdgcn_perm(d, c, 0x05010400u);
  const uint32_t AB = __builtin_amdgcn_perm(b, a, 0x07030602u), CD = __builtin_amdgcn_perm(d, c, 0x07030602u);
  u[0] = __builtin_amdgcn_perm(cd, ab, 0x05040100u);
  u[1] = __builtin_amdgcn_perm(cd, ab, 0x07060302u);
  u[2] = __builtin_amdgcn_perm(CD, AB, 0x05040100u);
  u[3] = __builtin_amdgcn_perm(CD, AB, 0x07060302u);
}

// The largest x >= 0 of the workgroup.
template <int NT>
__device__ inline uint32_t largest(int x, int* s_most) {
  x = wave_max_i(x);
  __syncthreads();  // (the one before is read)
  if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = x;
  __syncthreads();
  x = s_most[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) x = max(x, s_most[w]);
  return (uint32_t)x;
}

// The least power of two s with most <= 448 s, from 2^-40 to 2^40: most = a 2^e with 1/2 <= a < 1, 448 = 7/8 2^9.
__device__ inline float scale_of(float most) {
  if (!(most > 0.0f)) return 0x1p-40f;
  const int e = __builtin_amdgcn_frexp_expf(most) - (__builtin_amdgcn_frexp_mantf(most) <= 0.875f ? 9 : 8);
  return ldexpf(1.0f, min(max(e, -40), 40));
}

// The work is cut in squares of four tokens and eight dims, a thread a square, so that consecutive lanes read consecutive
// bytes of a row. A workgroup has 256, 512 or 1024 threads, as many as hold a page's squares two a thread (1024: a page of
// 256 tokens of 256 dims) in registers between the pass for the largest and the pass that writes. A square's values by
// dimension are words of four tokens: through LDS, so that consecutive lanes write consecutive words of a dimension.
// Bound: 8 prompts of 8192 tokens of 8 heads of 128 (302 MB read and written) 77 to 85 us, 3.6 to 3.9 TB/s; waiting for the
// chain count, length, table, rows (73% of the waves' time) with the five workgroups a CU holds. Steps, when it took 87: values
// written from the squares, 4 bytes a row, 127; every value tested for infinities and clamped, 145; both of the writing loops in one, with 168
// registers, 122; one square a thread of twice the threads 112. Pages of 256 tokens of 256 dims by 256 threads, which read
// twice what they do not hold, 63 us for two prompts of 7420 tokens and four heads, by 1024 27.
template <bool F16, int NT>
__global__ void __launch_bounds__(NT) hs_append_kernel(const AppendArgs A) {
  __shared__ int s_most[NT / 64];
  __shared__ uint32_t s_words[kSlab * kPitch];
  const uint32_t unit = A.group0 + blockIdx.x;
  if (unit >= A.units) return;
  const int kind = blockIdx.y, t = threadIdx.x;
  const uint32_t bh = fdiv(unit, A.div_span);
  const int nth = (int)(unit - bh * (uint32_t)A.span);
  const int b = (int)fdiv(bh, A.div_kv), h = (int)bh - b * A.kv;
  const int n = A.count ? min(max(A.count[b], 0), A.taken) : A.taken;
  const int64_t length = A.length[b];
  if (length < 0) return;
  const int64_t slot = (length >> A.shift) + nth;
  if (slot >= A.slots) return;
  const int first = nth == 0 ? (int)(length & (A.page - 1)) : 0;  // the page's first new token
  const int64_t from = (slot << A.shift) + first - length;         // of the new tokens
  if (from >= n) return;
  const int num = min(A.page - first, n - (int)from);
  const int id = A.table[b * A.table_stride + slot];
  if (id < 0 || id >= A.pages) return;
  const int64_t at = (int64_t)id * A.kv + h;
  const char* x = A.x[kind] + b * A.xb[kind] + h * A.xh[kind];
  const int32_t* path = A.path ? A.path + b * A.path_stride + from : nullptr;
  const int vecs = A.dim / 8, lo4 = first / 4, squares = ((first + num + 3) / 4 - lo4) * vecs;

  // square v's four rows from the page's token 4 (lo4 + v / vecs) on; 0 where there is no new one
  auto load = [&](int v, uint4 (&r)[4]) {
    const int g = (int)fdiv((uint32_t)v, A.div_vec), c = v - g * vecs;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = 4 * (lo4 + g) + k - first;
      r[k] = make_uint4(0, 0, 0, 0);
      if (i < 0 || i >= num) continue;
      const int row = path ? path[i] : (int)from + i;
      if (row >= 0 && row < A.rows) r[k] = *reinterpret_cast<const uint4*>(x + row * A.xn[kind] + 16 * c);
    }
  };
  // the largest |x| by its 16 bits, which order like it, two at a time; with an infinity or NaN among them, of the rest
  constexpr uint32_t kInf = F16 ? 0x7C00u : 0x7F80u;
  u16x2 top = {0, 0};
  const float was = A.scale[kind][at];
  auto grow = [&](const uint4 (&r)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t w[4] = {r[k].x, r[k].y, r[k].z, r[k].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w[e] & 0x7FFF7FFFu));
    }
  };
  uint4 held[kHold][4];
#pragma unroll
  for (int i = 0; i < kHold; ++i) {
    held[i][0] = held[i][1] = held[i][2] = held[i][3] = make_uint4(0, 0, 0, 0);
    if (t + NT * i < squares) load(t + NT * i, held[i]);
  }
#pragma unroll
  for (int i = 0; i < kHold; ++i) grow(held[i]);
  uint32_t bits = largest<NT>(max((int)top[0], (int)top[1]), s_most);
  const bool all_finite = bits < kInf;
  if (!all_finite) {
    int rest = 0;
    for (int v = t; v < squares; v += NT) {
      uint4 r[4];
      load(v, r);
      for (int k = 0; k < 4; ++k) {
        const uint32_t w[4] = {r[k].x, r[k].y, r[k].z, r[k].w};
        for (int e = 0; e < 8; ++e) {
          const uint32_t y = (w[e / 2] >> (16 * (e & 1))) & 0x7FFFu;
          rest = max(rest, y < kInf ? (int)y : 0);
        }
      }
    }
    bits = largest<NT>(rest, s_most);
  }
  const float most = Vec16<F16>::lo(bits);
  const float need = scale_of(most), now = first > 0 ? fmaxf(need, was) : need;
  const bool grows = first > 0 && now != was;
  const float ratio = was / now;
  if (t == 0) A.scale[kind][at] = now;
  // Where every quotient is in the range and the scale a power of two, one instruction converts two values.
  const bool plain = all_finite && __builtin_amdgcn_frexp_mantf(now) == 0.5f && most <= kTop * now;
  uint8_t* const page = A.cache[kind] + at * A.page * A.dim;
  const int shift = A.shift - 2, words = squares / vecs;  // log2 of a dim's words; its words that have new tokens
  if (grows) {  // the codes that are there, but those of a word with new tokens
    if (kind == 0) {
      for (int v = t; v < first * vecs; v += NT) {
        uint2* const to = reinterpret_cast<uint2*>(page + 8 * v);
        const uint2 old = *to;
        *to = make_uint2(rescaled(old.x, ratio), rescaled(old.y, ratio));
      }
    } else {
      for (int v = t; v < A.dim << shift; v += NT) {
        uint32_t* const to = reinterpret_cast<uint32_t*>(page + 4 * v);
        if ((v & ((1 << shift) - 1)) < lo4) *to = rescaled(*to, ratio);
      }
    }
  }
  auto keys = [&](int v, const uint2 (&y)[4]) {  // [token][dim]
    const int g = (int)fdiv((uint32_t)v, A.div_vec), c = v - g * vecs, tok = 4 * (lo4 + g);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (tok + k >= first && tok + k < first + num) *reinterpret_cast<uint2*>(page + (tok + k) * A.dim + 8 * c) = y[k];
  };
  auto values = [&](int v, int d0, const uint2 (&y)[4]) {  // [dim][token]: to LDS
    const int g = (int)fdiv((uint32_t)v, A.div_vec), d = 8 * (v - g * vecs) - d0;
    if (d < 0 || d >= kSlab) return;
    uint32_t u[8];
    transpose4(y[0].x, y[1].x, y[2].x, y[3].x, u);
    transpose4(y[0].y, y[1].y, y[2].y, y[3].y, u + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) s_words[(d + e) * kPitch + g] = u[e];
  };
  auto write = [&](int d0) {  // and from there
    __syncthreads();
    const int g = t & ((1 << shift) - 1), tok = 4 * (lo4 + g);
    const bool edge = tok < first || tok + 4 > first + num;  // codes of other tokens are in the word
    if (g < words)
      for (int d = t >> shift; d < min(kSlab, A.dim - d0); d += NT >> shift) {
        uint32_t* const to = reinterpret_cast<uint32_t*>(page + (d0 + d) * A.page + tok);
        uint32_t u = s_words[d * kPitch + g];
        if (edge) {
          const uint32_t old = *to, kept = grows ? rescaled(old, ratio) : old;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t byte = 0xFFu << (8 * k);
            if (tok + k < first) u = (u & ~byte) | (kept & byte);
            else if (tok + k >= first + num) u = (u & ~byte) | (old & byte);
          }
        }
        *to = u;
      }
    __syncthreads();
  };
  auto all = [&](auto codes, bool again) {
    for (int d0 = 0; d0 < (kind == 0 ? 1 : A.dim); d0 += kSlab) {
      auto square = [&](int v, const uint4 (&r)[4]) {
        const uint2 y[4] = {codes(r[0]), codes(r[1]), codes(r[2]), codes(r[3])};
        if (kind == 0) keys(v, y);
        else values(v, d0, y);
      };
      if (!again) {
#pragma unroll
        for (int i = 0; i < kHold; ++i)
          if (t + NT * i < squares) square(t + NT * i, held[i]);
      } else {
#pragma unroll 1
        for (int v = t; v < squares; v += NT) {
          uint4 r[4];
          load(v, r);
          square(v, r);
        }
      }
      if (kind != 0) write(d0);
    }
  };
  if (plain) all([&](const uint4& r) { return plain_codes<F16>(r, now); }, false);
  else
    all([&](const uint4& r) {
      float z[8];
      Vec16<F16>::unpack(r, z);
#pragma unroll
      for (int k = 0; k < 8; ++k) z[k] /= now;
      const float lo[4] = {z[0], z[1], z[2], z[3]}, hi[4] = {z[4], z[5], z[6], z[7]};
      return make_uint2(codes_of(lo), codes_of(hi));
    }, true);
}

template <bool F16>
void launch_threads(const AppendArgs& A, dim3 grid, int nt, hipStream_t st) {
  if (nt == 1024) hs_append_kernel<F16, 1024><<<grid, 1024, 0, st>>>(A);
  else if (nt == 512) hs_append_kernel<F16, 512><<<grid, 512, 0, st>>>(A);
  else hs_append_kernel<F16, kThreads><<<grid, kThreads, 0, st>>>(A);
}

}  // namespace

int launch_append(const hs_cache_append_args& a, hipStream_t stream) {
  AppendArgs A;
  const hs_heads x[2] = {a.k, a.v};
  for (int i = 0; i < 2; ++i) {
    A.x[i] = reinterpret_cast<const char*>(x[i].ptr);
    A.xb[i] = 2 * x[i].stride_b;
    A.xn[i] = 2 * x[i].stride_n;
    A.xh[i] = 2 * x[i].stride_h;
  }
  A.cache[0] = reinterpret_cast<uint8_t*>(a.cache.k);
  A.cache[1] = reinterpret_cast<uint8_t*>(a.cache.v);
  A.scale[0] = a.cache.k_scale;
  A.scale[1] = a.cache.v_scale;
  A.B = a.B;
  A.rows = a.rows;
  A.taken = a.taken;
  A.kv = a.cache.heads;
  A.page = a.cache.page;
  A.shift = __builtin_ctz((unsigned)a.cache.page);
  A.dim = a.cache.dim;
  // pages that `taken` tokens touch at most, wherever the first one lies
  A.span = (int)std::min<int64_t>(((int64_t)a.taken + a.cache.page - 2) / a.cache.page + 1, a.slots);
  A.slots = a.slots;
  A.pages = a.cache.pages;
  A.table = a.table;
  A.table_stride = a.table_stride;
  A.length = a.length;
  A.path = a.path;
  A.path_stride = a.path_stride;
  A.count = a.count;
  A.div_span = make_fastdiv((uint32_t)A.span);
  A.div_kv = make_fastdiv((uint32_t)A.kv);
  A.div_vec = make_fastdiv((uint32_t)(A.dim / 8));
  const uint64_t units = (uint64_t)A.B * A.kv * A.span;
  A.units = (uint32_t)units;
  // as many threads as keep a page's new tokens in registers: all of it, or what `taken` leaves of it
  const int64_t squares = (int64_t)std::min((a.taken + 6) / 4, A.page / 4) * (A.dim / 8);
  const int nt = squares > 2 * 512 ? 1024 : squares > 2 * kThreads ? 512 : kThreads;
  for (uint64_t at = 0; at < units; at += kMostGroups / (nt / kThreads)) {
    A.group0 = (uint32_t)at;
    const dim3 grid((uint32_t)std::min<uint64_t>(units - at, kMostGroups / (nt / kThreads)), 2);
    if (a.dtype == HS_F16) launch_threads<true>(A, grid, nt, stream);
    else launch_threads<false>(A, grid, nt, stream);
    if (hipPeekAtLastError() != hipSuccess) return HS_ERR_HIP;
  }
  return HS_OK;
}

}  // namespace hs
