// hs_beam_reorder: dst[b][j] = src[b][parent[b][j]] for many tensors in one launch. A thread owns one
// word (16 bytes, or 1) of a row position and moves it for every slot of the query: all of its
// loads come before its first store and no other thread touches those bytes, so a tensor can be
// reordered in place whatever the parents are (cycles, one beam continued by many), with no second
// buffer. Bound by HBM: every byte that changes hands is read once and written once.
#include <utility>

#include "hs_beam.h"

namespace hs {

namespace {

constexpr int kStates = 32;  // tensors of one launch (its arguments stay below 4 KB)
constexpr int kFew = 4;      // ... where they are few: 3 KB less of arguments, 1 us of the host's time

struct MoveState {
  const char* src;
  char* dst;
  int64_t ssb, ssw, ssr, dsb, dsw, dsr;
  int64_t units, unit;
  FastDiv div_chunks, div_rows;
  int chunks, rows;  // workgroups per row, rows per query
};
template <int STATES>
struct MoveArgs {
  int n, W, K;
  int64_t parent_stride;
  const int32_t* parent;
  const int32_t* count;
  uint32_t first[STATES];  // first workgroup of each tensor (past the last one: none)
  MoveState st[STATES];
};

// A thread's word of up to BYTES bytes at `at` of a buffer of `bytes` bytes: what lies outside is not
// read (0) and not written, by the bounds of the buffer's descriptor.
// STREAM: nontemporal.
template <int BYTES, bool STREAM>
struct Word;
template <bool STREAM>
struct Word<16, STREAM> {
  typedef unsigned int T __attribute__((ext_vector_type(4)));
  static constexpr int kHow = STREAM ? 2 : 0;  // the instructions' nt bit
  static __device__ T load(__amdgpu_buffer_rsrc_t r, int at) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, kHow);
  }
  static __device__ void store(T x, __amdgpu_buffer_rsrc_t r, int at) {
    __builtin_amdgcn_raw_buffer_store_b128(x, r, at, 0, kHow);
  }
};
template <>
struct Word<4, false> {
  typedef uint32_t T;
  static __device__ T load(__amdgpu_buffer_rsrc_t r, int at) {
    return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
  }
  static __device__ void store(T x, __amdgpu_buffer_rsrc_t r, int at) {
    __builtin_amdgcn_raw_buffer_store_b32(x, r, at, 0, 0);
  }
};
template <>
struct Word<1, false> {
  typedef uint8_t T;
  static __device__ T load(__amdgpu_buffer_rsrc_t r, int at) {
    return __builtin_amdgcn_raw_buffer_load_b8(r, at, 0, 0);
  }
  static __device__ void store(T x, __amdgpu_buffer_rsrc_t r, int at) {
    __builtin_amdgcn_raw_buffer_store_b8(x, r, at, 0, 0);
  }
};
constexpr int kRawBuffer = 0x00020000;  // a descriptor's last word: plain 32-bit data

// Moves the word at byte `at` < bytes of every slot, KMAX of them at most: every slot's word is in a
// register between the loads and the stores. A slot that moves nothing (mine of its lane < 0) has a
// descriptor of no bytes instead of a branch, so all loads go out together.
template <typename Wd, int KMAX>
__device__ __forceinline__ void move_words(int mine, uint64_t src, uint64_t ssw, uint64_t dst,
                                           uint64_t dsw, int bytes, int at) {
  auto buffer = [&](uint64_t base, uint64_t stride, int w, bool some) {
    return __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>(uniform(base + (uint64_t)(uint32_t)w * stride)), 0,
        (int)uniform(some ? (uint32_t)bytes : 0u), kRawBuffer);
  };
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

// KMAX: at least K.
template <int BYTES, int KMAX, bool STREAM, int STATES>
__global__ __launch_bounds__(kThreads) void hs_reorder_kernel(MoveArgs<STATES> A) {
  using Wd = Word<BYTES, STREAM>;
  int i = 0;
#pragma unroll
  for (int j = 1; j < STATES; ++j) i += blockIdx.x >= A.first[j] ? 1 : 0;
  MoveState S = A.st[STATES > kFew ? i : 0];
  uint32_t first = A.first[STATES > kFew ? i : 0];
  if (STATES <= kFew) {  // loads that wait for none: the arguments are far away (host memory)
#pragma unroll
    for (int j = 1; j < STATES; ++j)
      if (i == j) {
        S = A.st[j];
        first = A.first[j];
      }
  }
  const uint32_t u = blockIdx.x - first;
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
  move_words<Wd, KMAX>(mine, src, ssw, dst, dsw, bytes / BYTES * BYTES,
                       (int)threadIdx.x * BYTES);
  if (BYTES == 16 && (bytes & 15) != 0)  // a row's last one to three dwords
    move_words<Word<4, false>, KMAX>(mine, src, ssw, dst, dsw, bytes,
                                     bytes / 16 * 16 + (int)threadIdx.x * 4);
}

template <int BYTES, bool STREAM, int STATES>
void launch_slots(const MoveArgs<STATES>& A, uint32_t grid, hipStream_t st) {
  if (A.K <= 8) hs_reorder_kernel<BYTES, 8, STREAM, STATES><<<grid, kThreads, 0, st>>>(A);
  else if (A.K <= 16) hs_reorder_kernel<BYTES, 16, STREAM, STATES><<<grid, kThreads, 0, st>>>(A);
  else if (A.K <= 32) hs_reorder_kernel<BYTES, 32, STREAM, STATES><<<grid, kThreads, 0, st>>>(A);
  else hs_reorder_kernel<BYTES, 64, STREAM, STATES><<<grid, kThreads, 0, st>>>(A);
}

template <int BYTES, bool STREAM>
void launch_words(const MoveArgs<kStates>& A, uint32_t grid, hipStream_t st) {
  if (A.n > kFew) {
    launch_slots<BYTES, STREAM, kStates>(A, grid, st);
    return;
  }
  MoveArgs<kFew> few{A.n, A.W, A.K, A.parent_stride, A.parent, A.count, {}, {}};
  for (int j = 0; j < kFew; ++j) few.first[j] = A.first[j];
  for (int j = 0; j < A.n; ++j) few.st[j] = A.st[j];
  launch_slots<BYTES, STREAM, kFew>(few, grid, st);
}

// Slots' bytes of a call from which on its words are nontemporal. Four caches of 8 slots x 8 heads x 1024
// tokens x 256 bytes a query, half of them moved, in us without and with: 67 MB 12.8 and 13.2, 134 MB
// 23.3 and 23.0, 268 MB 51 and 46, 1.07 GB 183 and 166; 2.1 GB of 64 slots 404 and 379.
constexpr __int128 kStreamBytes = (__int128)100 << 20;

// The word a tensor moves by: 16 bytes where every pointer, stride and unit is a multiple of 4 (what the
// loads and stores need), else 1.
int word_of(const hs_state& s) {
  const uint64_t all = (uint64_t)(uintptr_t)s.src | (uint64_t)(uintptr_t)s.dst |
                       (uint64_t)s.src_stride_b | (uint64_t)s.src_stride_w |
                       (uint64_t)s.src_stride_row | (uint64_t)s.dst_stride_b |
                       (uint64_t)s.dst_stride_w | (uint64_t)s.dst_stride_row | (uint64_t)s.unit;
  return (all & 3) == 0 ? 16 : 1;
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
  __int128 all = 0;
  for (int i = 0; i < n; ++i) all += (__int128)B * K * states[i].rows * states[i].units * states[i].unit;
  const bool stream_past = all >= kStreamBytes;
  for (int word = 16; word >= 1; word /= 16) {  // the tensors of one word width together
    int i = 0;
    while (i < n) {
      MoveArgs<kStates> A;
      A.n = 0;
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
      if (word == 16 && stream_past) launch_words<16, true>(A, (uint32_t)grid, stream);
      else if (word == 16) launch_words<16, false>(A, (uint32_t)grid, stream);
      else launch_words<1, false>(A, (uint32_t)grid, stream);
      if (hipGetLastError() != hipSuccess) return HS_ERR_HIP;
    }
  }
  return HS_OK;
}

}  // namespace hs
