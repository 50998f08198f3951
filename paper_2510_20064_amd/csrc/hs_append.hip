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
constexpr uint32_t kNan8 = 0x7F;

template <bool F16>
__device__ inline void unpack8(const uint4& r, float (&z)[8]) {
  Vec16<F16>::unpack(r, z);
}
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

// The least power of two s with most <= 448 s, from 2^-40 to 2^40: most = a 2^e with 1/2 <= a < 1, 448 = 7/8 2^9.
__device__ inline float scale_of(float most) {
  if (!(most > 0.0f)) return 0x1p-40f;
  const int e = __builtin_amdgcn_frexp_expf(most) - (__builtin_amdgcn_frexp_mantf(most) <= 0.875f ? 9 : 8);
  return ldexpf(1.0f, min(max(e, -40), 40));
}

template <bool F16>
__global__ void __launch_bounds__(kThreads) hs_append_kernel(const AppendArgs A) {
  __shared__ float s_most[kWaves];
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
  const int vecs = A.dim / 8;

  auto row_of = [&](int i) -> int { return path ? path[i] : (int)from + i; };
  auto load = [&](int row, int c, float (&z)[8]) {
    uint4 r = make_uint4(0, 0, 0, 0);
    if (row >= 0 && row < A.rows) r = *reinterpret_cast<const uint4*>(x + row * A.xn[kind] + 16 * c);
    unpack8<F16>(r, z);
  };

  float most = 0.0f;
  for (int v = t; v < num * vecs; v += kThreads) {
    const int i = (int)fdiv((uint32_t)v, A.div_vec), c = v - i * vecs;
    float z[8];
    load(row_of(i), c, z);
#pragma unroll
    for (int k = 0; k < 8; ++k) most = fmaxf(most, finite(z[k]) ? fabsf(z[k]) : 0.0f);
  }
  most = __int_as_float(wave_max_i(__float_as_int(most)));  // not negative: ordered like its bits
  if ((t & 63) == 0) s_most[t >> 6] = most;
  const float was = A.scale[kind][at];
  __syncthreads();
  most = fmaxf(fmaxf(s_most[0], s_most[1]), fmaxf(s_most[2], s_most[3]));
  const float need = scale_of(most), now = first > 0 ? fmaxf(need, was) : need;
  const bool grows = first > 0 && now != was;
  const float ratio = was / now;
  if (t == 0) A.scale[kind][at] = now;

  uint8_t* const page = A.cache[kind] + at * A.page * A.dim;
  if (kind == 0) {  // [token][dim]
    for (int v = t + (grows ? 0 : first * vecs); v < (first + num) * vecs; v += kThreads) {
      const int i = (int)fdiv((uint32_t)v, A.div_vec), c = v - i * vecs;
      uint2* const to = reinterpret_cast<uint2*>(page + i * A.dim + 8 * c);
      if (i < first) {
        const uint2 old = *to;
        *to = make_uint2(rescaled(old.x, ratio), rescaled(old.y, ratio));
        continue;
      }
      float z[8];
      load(row_of(i - first), c, z);
      const float lo[4] = {z[0] / now, z[1] / now, z[2] / now, z[3] / now};
      const float hi[4] = {z[4] / now, z[5] / now, z[6] / now, z[7] / now};
      *to = make_uint2(codes_of(lo), codes_of(hi));
    }
    return;
  }
  // [dim][token]: a thread does four tokens of eight dims
  const int lo4 = grows ? 0 : first / 4, hi4 = (first + num + 3) / 4;
  for (int v = t; v < (hi4 - lo4) * vecs; v += kThreads) {
    const int g = (int)fdiv((uint32_t)v, A.div_vec), c = v - g * vecs, tok = 4 * (lo4 + g);
    float z[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = tok + k - first;
      load(i >= 0 && i < num ? row_of(i) : -1, c, z[k]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t* const to = reinterpret_cast<uint32_t*>(page + (8 * c + e) * A.page + tok);
      const float y[4] = {z[0][e] / now, z[1][e] / now, z[2][e] / now, z[3][e] / now};
      uint32_t u = codes_of(y);
      if (tok < first || tok + 4 > first + num) {
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
  }
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
  for (uint64_t at = 0; at < units; at += kMostGroups) {
    A.group0 = (uint32_t)at;
    const dim3 grid((uint32_t)std::min<uint64_t>(units - at, kMostGroups), 2);
    if (a.dtype == HS_F16) hs_append_kernel<true><<<grid, kThreads, 0, stream>>>(A);
    else hs_append_kernel<false><<<grid, kThreads, 0, stream>>>(A);
    if (hipPeekAtLastError() != hipSuccess) return HS_ERR_HIP;
  }
  return HS_OK;
}

}  // namespace hs
