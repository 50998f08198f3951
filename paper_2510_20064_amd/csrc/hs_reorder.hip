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
  uint32_t first;   // first workgroup of this tensor
  FastDiv div_chunks, div_rows;
  int chunks, rows;  // workgroups per row, rows per query
};
struct MoveArgs {
  int n, B, W, K;
  int64_t parent_stride;
  const int32_t* parent;
  const int32_t* count;
  MoveState st[kStates];
};

template <int BYTES>
struct Word;
template <>
struct Word<16> {
  typedef unsigned int T __attribute__((ext_vector_type(4)));
};
template <>
struct Word<4> {
  typedef uint32_t T;
};
template <>
struct Word<1> {
  typedef uint8_t T;
};

// KMAX: slots handled at once, at least K in place (all loads come before the stores).
template <int BYTES, int KMAX>
__global__ __launch_bounds__(kThreads) void hs_reorder_kernel(MoveArgs A) {
  typedef typename Word<BYTES>::T T;
  int i = 0;
  while (i + 1 < A.n && blockIdx.x >= A.st[i + 1].first) ++i;
  const MoveState& S = A.st[i];
  const uint32_t u = blockIdx.x - S.first;
  const uint32_t br = fdiv(u, S.div_chunks);
  const int64_t chunk = u - br * (uint32_t)S.chunks;
  const int b = (int)fdiv(br, S.div_rows);
  const int64_t r = br - (uint32_t)b * (uint32_t)S.rows;
  int64_t units = S.units;
  if (A.count) {
    const int64_t c = A.count[b];
    units = c < 0 ? 0 : c < units ? c : units;
  }
  const int64_t at = (chunk * kThreads + threadIdx.x) * BYTES;
  if (at >= units * S.unit) return;
  const char* src = S.src + b * S.ssb + r * S.ssr + at;
  char* dst = S.dst + b * S.dsb + r * S.dsr + at;
  const bool inplace = S.src == S.dst;
  const int32_t* parent = A.parent + b * A.parent_stride;
  for (int j0 = 0; j0 < A.K; j0 += KMAX) {
    T x[KMAX];
    bool moves[KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
      const int p = j0 + j < A.K ? parent[j0 + j] : -1;
      moves[j] = p >= 0 && p < A.W && !(inplace && p == j0 + j);
      if (moves[j]) x[j] = *reinterpret_cast<const T*>(src + p * S.ssw);
    }
#pragma unroll
    for (int j = 0; j < KMAX; ++j)
      if (moves[j]) *reinterpret_cast<T*>(dst + (j0 + j) * S.dsw) = x[j];
  }
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
        m.first = (uint32_t)grid;
        m.chunks = (int)chunks;
        m.rows = (int)s.rows;
        m.div_chunks = make_fastdiv((uint32_t)chunks);
        m.div_rows = make_fastdiv((uint32_t)s.rows);
        grid += wgs;
      }
      if (A.n == 0) break;
      if (word == 16) launch_words<16>(A, (uint32_t)grid, stream);
      else if (word == 4) launch_words<4>(A, (uint32_t)grid, stream);
      else launch_words<1>(A, (uint32_t)grid, stream);
      if (hipGetLastError() != hipSuccess) return HS_ERR_HIP;
    }
  }
  return HS_OK;
}

}  // namespace hs
