// Declarations shared by the kernels that grow a draft tree or run a beam search (hs_beam.hip,
// hs_reorder.hip, hs_tree.hip) and their host entries, with the wave-wide selection they use.
#pragma once

#include "hs_wave.h"

namespace hs {

// ---- launches (host side, defined next to their kernels) ----------------------------------------
// Workgroups of 256 threads of one launch: the runtime takes fewer than 2^32 threads. (A multiple of the 8 XCDs.)
constexpr uint32_t kMostGroups = (1u << 24) - 8;
// A launch that fails leaves its error to the entry, which clears it and says what it was.

// How a step's rows are cut: nc chunks of kBeamChunk vectors, in S slices of `chunks`, one wave each.
constexpr int kBeamChunk = 256;  // 16-byte vectors of a chunk, four per lane
struct BeamGeom {
  int B, W, K, S, chunks, nc;
  int64_t V, nvec;
  int dtype;
};
bool beam_geom(int B, int W, int K, int64_t V, int dtype, BeamGeom* g);
size_t beam_ws_bytes(const BeamGeom& g);
int launch_beam_step(const BeamGeom& g, const hs_beam_args& a, hipStream_t stream);
bool reorder_fits(const hs_state& s, int B, bool counted);  // its workgroups, of all launches, are numbered with 31 bits
// Whether the rows of a state's dst (B queries, K slots, `row` bytes a row) are apart from each other.
bool state_apart(const hs_state& s, int B, int K, int64_t row);
// The bytes that `beams` beams of every query span from a state's pointer; false where they do not fit
// 62 bits.
bool state_span(const hs_state& s, int B, int beams, int64_t sb, int64_t sw, int64_t sr, uint64_t* n);
// Whether no dst of a call shares a byte with another tensor of it, or with parent or count (but its own src
// in place). Every state is sound by itself. *bad: a state whose dst does.
bool states_apart(const hs_state* states, int n, int B, int W, int K, const int32_t* parent,
                  int64_t parent_stride, const int32_t* count, int* bad);
int launch_reorder(const hs_state* states, int n, int B, int W, int K, const int32_t* parent,
                   int64_t parent_stride, const int32_t* count, hipStream_t stream);
int launch_draft_tree(const hs_tree_args& a, hipStream_t stream);

// ---- wave-wide selection -------------------------------------------------------------------------

// Lanes below this one whose bit is set in m.
__device__ inline int lanes_below(uint64_t m) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                        __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
}
// LDS written by some lanes of a wave, then read by others of the same wave.
__device__ inline void lds_wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ inline uint32_t uniform(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ inline uint64_t uniform(uint64_t x) {
  return ((uint64_t)uniform((uint32_t)(x >> 32)) << 32) | uniform((uint32_t)x);
}
__device__ inline uint32_t wave_or_bits(uint32_t x) {
  x |= (uint32_t)dpp_i<0xB1>((int)x);
  x |= (uint32_t)dpp_i<0x4E>((int)x);
  x |= (uint32_t)dpp_i<0x141>((int)x);
  x |= (uint32_t)dpp_i<0x140>((int)x);
  return (uint32_t)(__builtin_amdgcn_readlane((int)x, 0) | __builtin_amdgcn_readlane((int)x, 16) |
                    __builtin_amdgcn_readlane((int)x, 32) | __builtin_amdgcn_readlane((int)x, 48));
}

__device__ inline int wave_sum_i(int x) {
  x += dpp_i<0xB1>(x);
  x += dpp_i<0x4E>(x);
  x += dpp_i<0x141>(x);
  x += dpp_i<0x140>(x);
  return __builtin_amdgcn_readlane(x, 0) + __builtin_amdgcn_readlane(x, 16) +
         __builtin_amdgcn_readlane(x, 32) + __builtin_amdgcn_readlane(x, 48);
}

// The sum of one fp64 value per lane, the same in every lane.
template <int CTRL>
__device__ inline double dpp_d(double v) {
  const uint64_t x = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)dpp_i<CTRL>((int)(uint32_t)x);
  const uint32_t hi = (uint32_t)dpp_i<CTRL>((int)(uint32_t)(x >> 32));
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
__device__ inline uint64_t lane_u(uint64_t x, int l) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, l);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), l);
  return ((uint64_t)hi << 32) | lo;
}
__device__ inline double lane_d(double v, int l) {
  return __longlong_as_double((long long)lane_u((uint64_t)__double_as_longlong(v), l));
}
__device__ inline double wave_sum_d(double v) {
  v += dpp_d<0xB1>(v);
  v += dpp_d<0x4E>(v);
  v += dpp_d<0x141>(v);
  v += dpp_d<0x140>(v);
  return (lane_d(v, 0) + lane_d(v, 16)) + (lane_d(v, 32) + lane_d(v, 48));
}
// An fp32 value (no NaN) as an unsigned integer that orders like it, -0 as +0, and back (0 as +0).
__device__ inline uint32_t ordered_of(float f) {
  const int32_t x = __float_as_int(f), m = x >> 31;
  return (uint32_t)((x ^ (m & 0x7FFFFFFF)) - m) ^ 0x80000000u;
}
__device__ inline float value_of(uint32_t u) {
  const int32_t k = (int32_t)(u ^ 0x80000000u);
  return __int_as_float(k >= 0 ? k : (int32_t)(0x80000000u | (uint32_t)(-k)));
}
// The same for fp64 (0 is below every value's image).
__device__ inline uint64_t ordered_of(double d) {
  const int64_t x = __double_as_longlong(d), m = x >> 63;
  return (uint64_t)((x ^ (m & 0x7FFFFFFFFFFFFFFFll)) - m) ^ 0x8000000000000000ull;
}
__device__ inline double value_of(uint64_t u) {
  const int64_t k = (int64_t)(u ^ 0x8000000000000000ull);
  return __longlong_as_double(k >= 0 ? k
                                     : (int64_t)(0x8000000000000000ull | (uint64_t)(-k)));
}

}  // namespace hs
