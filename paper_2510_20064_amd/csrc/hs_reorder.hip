// hs_beam_reorder: dst[b][j] = src[b][parent[b][j]] for many tensors in one launch. A thread owns one
// vector (16, 4 or 1 bytes) of a row position and moves it for every slot of the query: all of its
// loads come before its first store and no other thread touches those bytes, so a tensor can be
// reordered in place whatever the parents are (cycles, one beam continued by many), with no second
// buffer. Bound by HBM: every byte that changes hands is read once and written once.
#include <utility>

#include "hs_beam.h"

namespace hs {

namespace {

constexpr int kStates = 32;  // tensors of one launch (its arguments stay below 4 KB)

struct MoveState {
  const char* src;
  char* dst;
  int64_t ssb, ssw, ssr, dsb, dsw, dsr;
  int64_t units, unit;
  FastDiv div_chunks, div_rows;
  int chunks, rows;  // workgroups per row, rows per query
};
struct MoveArgs {
  int n, B, W, K;
  int64_t parent_stride;
  const int32_t* parent;
  const int32_t* count;
  uint32_t first[kStates];  // first workgroup of each tensor (past the last one: none)
  MoveState st[kStates];
};

// A thread's word of up to BYTES bytes at `at` of a buffer of `bytes` bytes: what lies outside is not
// read (0) and not written, by the bounds of the buffer's descriptor.
template <int BYTES>
struct Word;
template <>
struct Word<16> {
  typedef unsigned int T __attribute__((ext_vector_type(4)));
  static __device__ T load(__amdgpu_buffer_rsrc_t r, int at) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
  }
  static __device__ void store(T x, __amdgpu_buffer_rsrc_t r, int at) {
    __builtin_amdgcn_raw_buffer_store_b128(x, r, at, 0, 0);
  }
};
template <>
struct Word<4> {
  typedef uint32_t T;
  static __device__ T load(__amdgpu_buffer_rsrc_t r, int at) {
    return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
  }
  static __device__ void store(T x, __amdgpu_buffer_rsrc_t r, int at) {
    __builtin_amdgcn_raw_buffer_store_b32(x, r, at, 0, 0);
  }
};
template <>
struct Word<1> {
  typedef uint8_t T;
  static __device__ T load(__amdgpu_buffer_rsrc_t r, int at) {
    return __builtin_amdgcn_raw_buffer_load_b8(r, at, 0, 0);
  }
  static __device__ void store(T x, __amdgpu_buffer_rsrc_t r, int at) {
    __builtin_amdgcn_raw_buffer_store_b8(x, r, at, 0, 0);
  }
};
constexpr int kRawBuffer = 0x00020000;  // a descriptor's last word: plain 32-bit data

// KMAX: at least K; every slot's word is in a register between the loads and the stores. A slot that
// moves nothing has a descriptor of no bytes instead of a branch, so all loads go out together.
template <int BYTES, int KMAX>
__global__ __launch_bounds__(kThreads) void hs_reorder_kernel(MoveArgs A) {
  using Wd = Word<BYTES>;
  int i = 0;
#pragma unroll
  for (int j = 1; j < kStates; ++j) i += blockIdx.x >= A.first[j] ? 1 : 0;
  const MoveState S = A.st[i];
  const uint32_t u = blockIdx.x - A.first[i];
  const uint32_t br = fdiv(u, S.div_chunks);
  const int64_t chunk = u - br * (uint32_t)S.chunks;
  const int b = (int)fdiv(br, S.div_rows);
  const int64_t r = br - (uint32_t)b * (uint32_t)S.rows;
  int64_t units = S.units;
  if (A.count) {
    const int64_t c = A.count[b];
    units = c < 0 ? 0 : c < units ? c : units;
  }
  const int64_t begin = chunk * kThreads * BYTES, left = units * S.unit - begin;
  if (left <= 0) return;  // the whole workgroup
  const int bytes = (int)(left < kThreads * BYTES ? left : kThreads * BYTES);
  const bool inplace = S.src == S.dst;
  // lane j: slot j's parent, -1 where nothing moves
  const int lane = threadIdx.x & 63;
  int mine = lane < A.K ? A.parent[b * A.parent_stride + lane] : -1;
  if (mine >= A.W || (inplace && mine == lane)) mine = -1;
  // (the same in every lane, told to the compiler: descriptors live in scalar registers)
  const uint64_t src = uniform((uint64_t)(S.src + b * S.ssb + r * S.ssr + begin));
  const uint64_t dst = uniform((uint64_t)(S.dst + b * S.dsb + r * S.dsr + begin));
  const uint64_t ssw = uniform((uint64_t)S.ssw), dsw = uniform((uint64_t)S.dsw);
  auto buffer = [&](uint64_t base, uint64_t stride, int w, bool some) {
    return __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>(uniform(base + (uint64_t)(uint32_t)w * stride)), 0,
        (int)uniform(some ? (uint32_t)bytes : 0u), kRawBuffer);
  };
  const int at = (int)threadIdx.x * BYTES;
  typename Wd::T x[KMAX];
#pragma unroll
  for (int j = 0; j < KMAX; ++j) {
    const int p = __builtin_amdgcn_readlane(mine, j);
    x[j] = Wd::load(buffer(src, ssw, max(p, 0), p >= 0), at);
  }
#pragma unroll
  for (int j = 0; j < KMAX; ++j)
    Wd::store(x[j], buffer(dst, dsw, j, __builtin_amdgcn_readlane(mine, j) >= 0), at);
}

template <int BYTES>
void launch_words(const MoveArgs& A, uint32_t grid, hipStream_t st) {
  if (A.K <= 8) hs_reorder_kernel<BYTES, 8><<<grid, kThreads, 0, st>>>(A);
  else if (A.K <= 16) hs_reorder_kernel<BYTES, 16><<<grid, kThreads, 0, st>>>(A);
  else if (A.K <= 32) hs_reorder_kernel<BYTES, 32><<<grid, kThreads, 0, st>>>(A);
  else hs_reorder_kernel<BYTES, 64><<<grid, kThreads, 0, st>>>(A);
}

// The widest word that every pointer, stride and unit of a tensor is a multiple of.
int word_of(const hs_state& s) {
  const uint64_t all = (uint64_t)(uintptr_t)s.src | (uint64_t)(uintptr_t)s.dst |
                       (uint64_t)s.src_stride_b | (uint64_t)s.src_stride_w |
                       (uint64_t)s.src_stride_row | (uint64_t)s.dst_stride_b |
                       (uint64_t)s.dst_stride_w | (uint64_t)s.dst_stride_row | (uint64_t)s.unit;
  return (all & 15) == 0 ? 16 : (all & 3) == 0 ? 4 : 1;
}

uint64_t chunks_of(const hs_state& s, int word) {
  const uint64_t bytes = (uint64_t)s.units * (uint64_t)s.unit, per = (uint64_t)kThreads * word;
  return bytes / per + (bytes % per != 0);
}

}  // namespace

bool reorder_fits(const hs_state& s, int B) {
  const unsigned __int128 wgs = (unsigned __int128)chunks_of(s, word_of(s)) *
                                (unsigned __int128)s.rows * (unsigned __int128)B;
  return wgs < ((unsigned __int128)1 << 31);
}

// Three nested strides over rows: sorted, each must step over everything inside it.
bool state_apart(const hs_state& s, int B, int K, int64_t row) {
  struct {
    int64_t stride, n;
  } d[3] = {{s.dst_stride_b, B}, {s.dst_stride_w, K}, {s.dst_stride_row, s.rows}};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (d[j].stride < d[i].stride) std::swap(d[i], d[j]);
  __int128 inner = row;
  for (int i = 0; i < 3; ++i) {
    if (d[i].n == 1) continue;
    if (d[i].stride < inner) return false;
    inner += (__int128)d[i].stride * (d[i].n - 1);
  }
  return true;
}

int launch_reorder(const hs_state* states, int n, int B, int W, int K, const int32_t* parent,
                   int64_t parent_stride, const int32_t* count, hipStream_t stream) {
  for (int word = 16; word >= 1; word /= 4) {  // the tensors of one word width together
    int i = 0;
    while (i < n) {
      MoveArgs A;
      A.n = 0;
      A.B = B;
      A.W = W;
      A.K = K;
      A.parent = parent;
      A.parent_stride = parent_stride;
      A.count = count;
      uint64_t grid = 0;
      for (; i < n && A.n < kStates; ++i) {
        const hs_state& s = states[i];
        if (word_of(s) != word) continue;
        const uint64_t chunks = chunks_of(s, word);
        const uint64_t wgs = chunks * (uint64_t)s.rows * (uint64_t)B;
        if (grid + wgs >= (1ull << 31)) break;
        A.first[A.n] = (uint32_t)grid;
        MoveState& m = A.st[A.n++];
        m.src = reinterpret_cast<const char*>(s.src);
        m.dst = reinterpret_cast<char*>(s.dst);
        m.ssb = s.src_stride_b;
        m.ssw = s.src_stride_w;
        m.ssr = s.src_stride_row;
        m.dsb = s.dst_stride_b;
        m.dsw = s.dst_stride_w;
        m.dsr = s.dst_stride_row;
        m.units = s.units;
        m.unit = s.unit;
        m.chunks = (int)chunks;
        m.rows = (int)s.rows;
        m.div_chunks = make_fastdiv((uint32_t)chunks);
        m.div_rows = make_fastdiv((uint32_t)s.rows);
        grid += wgs;
      }
      if (A.n == 0) break;
      for (int j = A.n; j < kStates; ++j) A.first[j] = 0xFFFFFFFFu;
      if (word == 16) launch_words<16>(A, (uint32_t)grid, stream);
      else if (word == 4) launch_words<4>(A, (uint32_t)grid, stream);
      else launch_words<1>(A, (uint32_t)grid, stream);
      if (hipGetLastError() != hipSuccess) return HS_ERR_HIP;
    }
  }
  return HS_OK;
}

}  // namespace hs
