// hs_beam_reorder: dst[b][j] = src[b][parent[b][j]] for many tensors in one launch. A lane owns words (16 bytes; at
// a row's end 1) of a row and moves each for every slot of the query: all of a word's loads come before its
// first store and no other lane touches those bytes, so a tensor can be reordered in place whatever the
// parents are (cycles, one beam continued by many), with no second buffer. (Where nothing is in place, waves
// may share the slots.) Bound by HBM: every byte that changes hands is read once and written once; 1.07 GB in
// 187 us, 5.7 TB/s.
#include <algorithm>
#include <type_traits>

#include "hs_beam.h"

namespace hs {

namespace {

constexpr int kStates = 32;  // tensors of one launch (its arguments stay below 4 KB)
constexpr int kFew = 4;      // ... where they are few and differ: 3 KB less of arguments, 1 us of the host's time
constexpr int kChunk = 1024;             // a wave's bytes of a row: 16 a lane
constexpr int kPiece = kWaves * kChunk;  // a workgroup's
constexpr int kSpan = 4;                 // pieces of a workgroup where few slots may move,
constexpr int kWideSlots = 8;            // in calls of at most so many slots

struct MoveState {
  const char* src;
  char* dst;
  int64_t ssb, ssw, ssr, dsb, dsw, dsr;
  int64_t units, unit;
  FastDiv div_parts, div_rows;
  int parts, rows;  // workgroups per row (where rows share them: waves), rows per query
  int queries;
  int span;  // pieces of a workgroup: 1 or kSpan; 0: rows share workgroups
};
struct MoveCall {
  int n, W, K;
  int split;  // log2 of the waves that share a position's slots, KMAX each (not in place)
  int64_t parent_stride;
  const int32_t* parent;
  const int32_t* count;
};
template <int STATES>
struct MoveArgs : MoveCall {
  uint32_t first[STATES];  // first workgroup of each tensor (past the last one: none)
  MoveState st[STATES];
};
// Tensors that differ in their pointers only: the caches of a model's layers.
struct AlikeArgs : MoveCall {
  uint32_t group0;  // the launch's first workgroup of each tensor's
  MoveState st;
  const char* src[kStates];
  char* dst[kStates];
};

// The workgroup's tensor and its number in it.
template <int STATES>
__device__ __forceinline__ uint32_t pick(const MoveArgs<STATES>& A, MoveState& S) {
  int i = 0;
#pragma unroll
  for (int j = 1; j < STATES; ++j) i += blockIdx.x >= A.first[j] ? 1 : 0;
  S = A.st[STATES > kFew ? i : 0];
  uint32_t first = A.first[STATES > kFew ? i : 0];
  if (STATES <= kFew) {  // loads that wait for none: the arguments are far away (host memory)
#pragma unroll
    for (int j = 1; j < STATES; ++j)
      if (i == j) {
        S = A.st[j];
        first = A.first[j];
      }
  }
  return blockIdx.x - first;
}
__device__ __forceinline__ uint32_t pick(const AlikeArgs& A, MoveState& S) {
  S = A.st;
  S.src = A.src[blockIdx.y];
  S.dst = A.dst[blockIdx.y];
  return A.group0 + blockIdx.x;
}

typedef unsigned int Vec16 __attribute__((ext_vector_type(4)));

// A thread's 16 bytes, or one, at byte `at` of `bytes` bytes from an address on that is the same in all lanes:
// what lies outside is not read and not written. STREAM: nontemporal.
// By the bounds of a buffer's descriptor; 16 bytes must then be at a multiple of 4.
constexpr int kRawBuffer = 0x00020000;  // a descriptor's last word: plain 32-bit data
struct Buffer {
  __amdgpu_buffer_rsrc_t r;
  __device__ Buffer(uint64_t base, int bytes)
      : r(__builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(uniform(base)), 0,
                                            (int)uniform((uint32_t)bytes), kRawBuffer)) {}
};
template <bool STREAM>
struct Aligned : Buffer {
  typedef Vec16 T;
  static constexpr int kBytes = 16, kHow = STREAM ? 2 : 0;  // the instructions' nt bit
  __device__ Aligned(uint64_t base, int bytes) : Buffer(base, bytes) {}
  __device__ T load(int at) const { return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, kHow); }
  __device__ void store(T x, int at) const { __builtin_amdgcn_raw_buffer_store_b128(x, r, at, 0, kHow); }
};
struct Byte : Buffer {
  typedef uint8_t T;
  static constexpr int kBytes = 1;
  __device__ Byte(uint64_t base, int bytes) : Buffer(base, bytes) {}
  __device__ T load(int at) const { return __builtin_amdgcn_raw_buffer_load_b8(r, at, 0, 0); }
  __device__ void store(T x, int at) const { __builtin_amdgcn_raw_buffer_store_b8(x, r, at, 0, 0); }
};
// At any address, without a descriptor; 16 bytes there can be read also where bytes is 0. For aligned rows the
// descriptors read less: 1 GB 205 us, so 241.
template <bool STREAM>
struct Anywhere {
  typedef Vec16 T;
  typedef Vec16 Any __attribute__((aligned(1)));
  typedef __attribute__((address_space(1))) Any* Ptr;
  static constexpr int kBytes = 16;
  uint64_t base;
  int bytes;
  __device__ Anywhere(uint64_t base, int bytes) : base(base), bytes(bytes) {}
  __device__ T load(int at) const {
    const Ptr q = (Ptr)(base + (uint64_t)max(min(at, bytes - 16), 0));
    if constexpr (STREAM) return __builtin_nontemporal_load(q);
    else return *q;
  }
  __device__ void store(T x, int at) const {
    if (at >= bytes) return;
    const Ptr q = (Ptr)(base + (uint64_t)at);
    if constexpr (STREAM) __builtin_nontemporal_store((Any)x, q);
    else *q = x;
  }
};

struct Slots {
  uint64_t src, dst, ssw, dsw;
  int mine;        // lane j: slot j's parent, -1 where nothing moves
  int first;       // the wave's first slot
  uint64_t moves;  // the slots that move
};

// A lane's words at `at`, `at` + step, ... (COUNT of them) before byte `bytes`, of M slots: from the wave's first one on,
// or, PICK, the M first that move. A slot that moves nothing has no bytes instead of a branch, so that all loads
// go out together.
template <typename Wd, int M, int COUNT, bool PICK>
struct Tile {
  typename Wd::T x[M][COUNT];

  template <bool LOAD>
  __device__ __forceinline__ void pass(const Slots& s, int at, int step, int bytes) {
    uint64_t rest = s.moves;
#pragma unroll
    for (int q = 0; q < M; ++q) {
      const int j = PICK ? __builtin_ctzll(rest | 1ull << 63) : s.first + q, p = __builtin_amdgcn_readlane(s.mine, j);
      const bool on = PICK ? rest != 0 : p >= 0;
      const Wd w(LOAD ? s.src + (uint64_t)(uint32_t)(on ? p : 0) * s.ssw : s.dst + (uint64_t)j * s.dsw,
                 on ? bytes : 0);
#pragma unroll
      for (int c = 0; c < COUNT; ++c) {
        if constexpr (LOAD) x[q][c] = w.load(at + c * step);
        else w.store(x[q][c], at + c * step);
      }
      rest &= rest - 1;
    }
  }
  __device__ __forceinline__ void load(const Slots& s, int at, int step, int bytes) {
    pass<true>(s, at, step, bytes);
  }
  __device__ __forceinline__ void store(const Slots& s, int at, int step, int bytes) {
    pass<false>(s, at, step, bytes);
  }
  // The loads all come before the stores.
  __device__ __forceinline__ void move(const Slots& s, int at, int step, int bytes) {
    load(s, at, step, bytes);
    store(s, at, step, bytes);
  }
};

// A lane's n words of each slot that moves: several at once where few do.
template <typename Wd, int KMAX, bool WIDE>
__device__ __forceinline__ void move_words(const Slots& s, int at, int n, int step, int bytes) {
  if constexpr (WIDE) {
    const int m = __builtin_popcountll(s.moves);
    if (n > 2 && m <= KMAX / 4) {
      Tile<Wd, KMAX / 4, kSpan, true>().move(s, at, step, bytes);
    } else if (n > 1 && m <= KMAX / 2) {
      for (int c = 0; c < n; c += 2) Tile<Wd, KMAX / 2, 2, true>().move(s, at + c * step, step, bytes);
    } else {
      for (int c = 0; c < n; ++c) Tile<Wd, KMAX, 1, false>().move(s, at + c * step, step, bytes);
    }
  } else {
    Tile<Wd, KMAX, 1, false>().move(s, at, step, bytes);
  }
}

// KMAX: at least K, or its share of a wave. WIDE: some tensor has a span above 1. ALIGNED: every row of the tensors starts at a multiple of 4 bytes.
template <bool ALIGNED, int KMAX, bool WIDE, bool STREAM, typename Args>
__global__ __launch_bounds__(kThreads) void hs_reorder_kernel(Args A) {
  MoveState S;
  const uint32_t wg = pick(A, S);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // a row of less than a workgroup's bytes has a wave for each of its chunks; a longer one has workgroups that
  // move `span` pieces of kPiece bytes each, `parts` pieces apart
  const int sub = WIDE ? wave : wave >> A.split;  // the wave's chunk of the workgroup's
  const uint32_t u = S.span == 0 ? wg * (kWaves >> A.split) + sub : wg;
  const uint32_t br = fdiv(u, S.div_parts);
  const int64_t part = u - br * (uint32_t)S.parts;
  const int b = (int)fdiv(br, S.div_rows);
  if (b >= S.queries) return;  // past the tensor's end
  const int64_t r = br - (uint32_t)b * (uint32_t)S.rows;
  int64_t units = S.units;
  if (A.count) {
    const int64_t c = A.count[b];
    units = c < 0 ? 0 : c < units ? c : units;
  }
  const int64_t all = units * S.unit, begin = S.span == 0 ? part * kChunk : part * (kPiece >> A.split) + sub * kChunk;
  if (all <= begin) return;  // all of the wave
  // the wave's words end at `left` (that is below 2^31 where there is more than one), but for a row's last bytes
  const int64_t left = (all & ~15ll) - begin;
  const int span = WIDE && S.span > 1 ? S.span : 1, step = span > 1 ? S.parts * kPiece : kChunk;
  const int n = span == 1 ? 1 : 1 + (left > step) + (left > 2ll * step) + (left > 3ll * step);
  const int bytes = (int)(span > 1 || left < kChunk ? left : kChunk);
  const bool inplace = S.src == S.dst;
  Slots s;
  s.mine = lane < A.K ? A.parent[b * A.parent_stride + lane] : -1;
  if (s.mine >= A.W || (inplace && s.mine == lane)) s.mine = -1;
  s.moves = __ballot(s.mine >= 0);
  s.first = WIDE ? 0 : (wave & ((1 << A.split) - 1)) * KMAX;
  // (the same in every lane, told to the compiler: descriptors live in scalar registers)
  s.src = uniform((uint64_t)(S.src + b * S.ssb + r * S.ssr + begin));
  s.dst = uniform((uint64_t)(S.dst + b * S.dsb + r * S.dsr + begin));
  s.ssw = uniform((uint64_t)S.ssw);
  s.dsw = uniform((uint64_t)S.dsw);
  using Wd = typename std::conditional<ALIGNED, Aligned<STREAM>, Anywhere<STREAM>>::type;
  if (left > 0) move_words<Wd, KMAX, WIDE>(s, lane * 16, n, step, bytes);
  if ((all & 15) != 0) {  // a row's last bytes
    int last = -1;
    for (int c = 0; c < span; ++c)
      if (left >= (int64_t)c * step && left < (int64_t)c * step + kChunk) last = (int)left;
    if (last >= 0)
      Tile<Byte, KMAX, 1, false>().move(s, last + lane, 0, last + (int)(all & 15));
  }
}

template <bool ALIGNED, bool STREAM, typename Args>
void launch_slots(const Args& A, bool wide, dim3 grid, hipStream_t st) {
  if (wide) hs_reorder_kernel<ALIGNED, kWideSlots, true, STREAM><<<grid, kThreads, 0, st>>>(A);
  else if (A.K <= 8 << A.split) hs_reorder_kernel<ALIGNED, 8, false, STREAM><<<grid, kThreads, 0, st>>>(A);
  else if (A.K <= 16 << A.split) hs_reorder_kernel<ALIGNED, 16, false, STREAM><<<grid, kThreads, 0, st>>>(A);
  else if (A.K <= 32) hs_reorder_kernel<ALIGNED, 32, false, STREAM><<<grid, kThreads, 0, st>>>(A);
  else hs_reorder_kernel<ALIGNED, 64, false, STREAM><<<grid, kThreads, 0, st>>>(A);
}

bool alike(const MoveState& a, const MoveState& b) {
  return a.ssb == b.ssb && a.ssw == b.ssw && a.ssr == b.ssr && a.dsb == b.dsb && a.dsw == b.dsw &&
         a.dsr == b.dsr && a.units == b.units && a.unit == b.unit && a.rows == b.rows &&
         a.parts == b.parts && a.span == b.span;
}

// Short arguments where they do: seven tensors of 3 x 2 rows of 172 KB 6.7 us alike, 8.1 with arguments for 32, eight of 8
// queries of 64 rows of 15 KB 8.5 and 9.7.
template <bool ALIGNED, bool STREAM>
void launch_words(const MoveArgs<kStates>& A, uint32_t grid, hipStream_t st) {
  bool wide = false, same = true;
  for (int j = 0; j < A.n; ++j) {
    wide = wide || A.st[j].span > 1;
    same = same && alike(A.st[j], A.st[0]);
  }
  if (same) {
    AlikeArgs like;
    static_cast<MoveCall&>(like) = A;
    like.st = A.st[0];
    for (int j = 0; j < A.n; ++j) {
      like.src[j] = A.st[j].src;
      like.dst[j] = A.st[j].dst;
    }
    const uint32_t groups = grid / A.n;
    for (like.group0 = 0; like.group0 < groups; like.group0 += kMostGroups) {
      launch_slots<ALIGNED, STREAM>(like, wide, dim3(std::min(groups - like.group0, kMostGroups), A.n), st);
      if (hipPeekAtLastError() != hipSuccess) return;
    }
  } else if (A.n <= kFew) {
    MoveArgs<kFew> few;
    static_cast<MoveCall&>(few) = A;
    for (int j = 0; j < kFew; ++j) few.first[j] = A.first[j];
    for (int j = 0; j < A.n; ++j) few.st[j] = A.st[j];
    launch_slots<ALIGNED, STREAM>(few, wide, dim3(grid), st);
  } else {
    launch_slots<ALIGNED, STREAM>(A, wide, dim3(grid), st);
  }
}

// Slots' bytes of a call from which on its words are nontemporal. Four caches of 8 slots x 8 heads x 1024
// tokens x 256 bytes a query, half of them moved, in us without and with: 67 MB 12.8 and 13.2, 134 MB
// 23.3 and 23.0, 268 MB 51 and 46, 1.07 GB 183 and 166; 2.1 GB of 64 slots 404 and 379.
constexpr __int128 kStreamBytes = (__int128)100 << 20;

// Whether every row of a tensor starts at a multiple of 4 bytes.
bool aligned(const hs_state& s) {
  const uint64_t all = (uint64_t)(uintptr_t)s.src | (uint64_t)(uintptr_t)s.dst |
                       (uint64_t)s.src_stride_b | (uint64_t)s.src_stride_w |
                       (uint64_t)s.src_stride_row | (uint64_t)s.dst_stride_b |
                       (uint64_t)s.dst_stride_w | (uint64_t)s.dst_stride_row;
  return (all & 3) == 0;
}

// Rows one behind the other, all of their units moved, are one row (8 tensors of 128 queries x 8 slots x 8
// rows of 66 bytes: 34.8 us as 8 rows, 5.8 as one).
hs_state in_one_row(const hs_state& s, bool counted) {
  hs_state one = s;
  if (!counted && s.src_stride_row == s.units * s.unit && s.dst_stride_row == s.src_stride_row) {
    one.units *= s.rows;
    one.rows = 1;
    one.src_stride_row = one.dst_stride_row = 0;
  }
  return one;
}

// Bytes of a slot, over all tensors, queries and rows, from which on a workgroup may have several pieces.
constexpr __int128 kWideBytes = (__int128)16 << 20;

// How a row is cut (MoveState's span). Rows that share workgroups are those of less than a workgroup's bytes (64
// queries x 64 rows of 512 bytes, counted: 11.8 us with a workgroup for each, 5.9; but rows of 34 chunks
// 12.9 shared, 11.2). A wave with one piece and one moving slot has one load in flight, hence up to four
// pieces for it where few slots may move. In us, with one piece and four: 1 of 4 slots of 1.0 GB 88 and 50; 4
// of 8 slots of 2.1 GB 205 and 187; all of 8 of 1.1 GB 310 and 322. Of more slots half of the calls lose: 3 of 15 30
// and 18, but 7 of 16 151 and 164, 11 of 12 219 and 250, 16 of 16 333 and 415. (The host does not see how many of
// a call's slots move: the rule bets on some of up to 8 in place, or 4, staying, and loses 4% where none does.) The pieces lie a multiple of 8
// apart where there are enough, so that each XCD stays with its eighth of the memory's 4 KB pages (the 205
// are 238 with pieces side by side).
uint64_t row_bytes(const hs_state& s) { return (uint64_t)s.units * (uint64_t)s.unit; }
int span_of(const hs_state& s, int K, bool wide, int split) {
  if (row_bytes(s) <= (kPiece >> split) - kChunk) return 0;
  const bool few = K <= kWideSlots / 2 || (K <= kWideSlots && s.src == s.dst);
  return wide && few && row_bytes(s) > kPiece && row_bytes(s) < (1u << 30) ? kSpan : 1;
}
uint64_t parts_of(const hs_state& s, int span, int split) {
  const uint64_t per = span == 0 ? kChunk : kPiece >> split;
  const uint64_t n = row_bytes(s) / per + (row_bytes(s) % per != 0);
  if (span <= 1) return n;
  const uint64_t parts = (n + span - 1) / span;
  return n >= 32 ? (parts + 7) / 8 * 8 : parts;
}

// The waves (as a power of two) that share a position's slots where nothing is in place: fewer registers each, more
// waves per CU. us with one wave and with this rule: 13 queries of 30 slots of 0.27 MB at odd addresses 41 and
// 26, 7 of 31 of 1.2 MB 48 and 42, 4 of 64 of 2.5 MB 140 and 132, 9 of 32 of 0.1 MB 10.0 and 6.8, 15 of 28 of
// 2.6 MB 372 and 385 (what the rule loses: large aligned slots, 4%; K alone does not tell them from the others); 7 of 9
// slots (two waves) 4.7 and 4.4, but 8 of 16 of 8 MB 327 and 346.
int split_of(int K, bool past) { return K <= 8 ? 0 : K > 16 ? 2 : past ? 0 : 1; }

}  // namespace

bool reorder_fits(const hs_state& state, int B, bool counted) {
  const hs_state s = in_one_row(state, counted);
  const unsigned __int128 parts = (unsigned __int128)parts_of(s, 1, 2) *
                                  (unsigned __int128)s.rows * (unsigned __int128)B;
  return parts < ((unsigned __int128)1 << 31);
}

namespace {

// What a call reads or writes of one tensor: rows of `row` bytes, along up to three strides.
struct Region {
  uint64_t at, end;  // its bytes lie in [at, end)
  int state;         // -1: parent, count
  bool writes;
  int nd;
  int64_t stride[3], n[3], row;  // ascending; none of a single row

  Region() {}
  Region(const void* p, int state, bool writes, int64_t row, int64_t sb, int64_t nb, int64_t sw,
         int64_t nw, int64_t sr, int64_t nr)
      : at((uint64_t)(uintptr_t)p), state(state), writes(writes), nd(0), row(row) {
    const int64_t all[3][2] = {{sb, nb}, {sw, nw}, {sr, nr}};
    for (const auto& d : all) {
      if (d[1] == 1) continue;
      int i = nd++;
      for (; i > 0 && stride[i - 1] > d[0]; --i) {
        stride[i] = stride[i - 1];
        n[i] = n[i - 1];
      }
      stride[i] = d[0];
      n[i] = d[1];
    }
    end = at + (uint64_t)extent(nd);
  }
  // The bytes that the first l strides span.
  __int128 extent(int l) const {
    __int128 e = row;
    for (int i = 0; i < l; ++i) e += (__int128)stride[i] * (n[i] - 1);
    return e;
  }
  // Each stride steps over everything inside it: no two rows share a byte.
  bool nested() const {
    for (int i = 0; i < nd; ++i)
      if (stride[i] < extent(i)) return false;
    return true;
  }
  bool same_strides(const Region& o) const {
    return nd == o.nd && std::equal(stride, stride + nd, o.stride);
  }
};

// Whether a row of a and one of b, which starts p bytes further on, share a byte. Both nested, with the same
// strides: only the two steps of the largest stride that leave less than itself between the two can
// bring them together, and so on inside.
bool meet(const Region& a, const Region& b, int l, __int128 p) {
  if (l == 0) return p < a.row && -p < b.row;
  const int64_t s = a.stride[l - 1];
  const __int128 down = p >= 0 ? p / s : -((-p + s - 1) / s);  // rounded down
  for (__int128 i = down; i <= down + 1; ++i)  // steps of a less steps of b
    if (i < a.n[l - 1] && -i < b.n[l - 1] && meet(a, b, l - 1, p - i * s)) return true;
  return false;
}

// Regions in the order of `at`, each taken as the bytes that its first l strides span (all: its span):
// the state of a written one that shares some with another, or -1.
int first_shared(const Region* r, int m, bool all, int l) {
  __int128 any = 0, written = 0;  // ends so far
  int writer = -1;
  for (int i = 0; i < m; ++i) {
    const __int128 at = r[i].at, end = all ? (__int128)r[i].end : at + r[i].extent(l);
    if (at < written) return r[writer].state;
    if (r[i].writes && at < any) return r[i].state;
    any = std::max(any, end);
    if (r[i].writes && end > written) {
      written = end;
      writer = i;
    }
  }
  return -1;
}

// The same for regions whose spans overlap, exactly: tensors that lie between each other's rows, as slices
// of one buffer do, are apart.
int shared_bytes(const Region* r, int m) {
  for (int i = 0; i < m; ++i)
    if (!r[i].nested() || !r[i].same_strides(r[0])) return first_shared(r, m, true, 0);
  const int nd = r[0].nd;
  for (int l = 0; l < nd; ++l) {  // all of them side by side inside one step of every stride from l on
    __int128 most = 0;  // the bytes of a step
    for (int i = 0; i < m; ++i)
      most = std::max(most, (__int128)r[i].at - (__int128)r[0].at + r[i].extent(l));
    bool fits = true;
    for (int q = l; q < nd; ++q) {
      int64_t n = 1;
      for (int i = 0; i < m; ++i) n = std::max(n, r[i].n[q]);
      fits = fits && r[0].stride[q] >= most;
      most += (__int128)r[0].stride[q] * (n - 1);
    }
    if (fits && first_shared(r, m, false, l) < 0) return -1;
  }
  for (int i = 0; i < m; ++i)
    for (int j = i + 1; j < m; ++j)
      if ((r[i].writes || r[j].writes) &&
          meet(r[i], r[j], nd, (__int128)r[j].at - (__int128)r[i].at))
        return r[i].writes ? r[i].state : r[j].state;
  return -1;
}

}  // namespace

bool state_apart(const hs_state& s, int B, int K, int64_t row) {
  return Region(s.dst, 0, true, row, s.dst_stride_b, B, s.dst_stride_w, K, s.dst_stride_row, s.rows)
      .nested();
}

bool state_span(const hs_state& s, int B, int beams, int64_t sb, int64_t sw, int64_t sr, uint64_t* n) {
  const __int128 row = (__int128)s.units * s.unit;
  const __int128 all = row + (__int128)(B - 1) * sb + (__int128)(beams - 1) * sw +
                       (__int128)(s.rows - 1) * sr;
  if (all >= ((__int128)1 << 62)) return false;
  *n = (uint64_t)all;
  return true;
}

bool states_apart(const hs_state* states, int n, int B, int W, int K, const int32_t* parent,
                  int64_t parent_stride, const int32_t* count, int* bad) {
  Region r[2 * HS_MAX_STATES + 2];
  int m = 0;
  for (int i = 0; i < n; ++i) {
    const hs_state& s = states[i];
    const int64_t row = s.units * s.unit;
    const bool inplace = s.src == s.dst;
    if (!inplace)
      r[m++] = Region(s.src, i, false, row, s.src_stride_b, B, s.src_stride_w, W, s.src_stride_row, s.rows);
    r[m++] = Region(s.dst, i, true, row, s.dst_stride_b, B, s.dst_stride_w, inplace ? std::max(W, K) : K,
                    s.dst_stride_row, s.rows);
  }
  r[m++] = Region(parent, -1, false, 4 * (int64_t)K, 4 * parent_stride, B, 0, 1, 0, 1);
  if (count) r[m++] = Region(count, -1, false, 4 * (int64_t)B, 0, 1, 0, 1, 0, 1);
  std::sort(r, r + m, [](const Region& a, const Region& b) { return a.at < b.at; });
  if (first_shared(r, m, true, 0) < 0) return true;
  for (int i = 0; i < m;) {  // regions whose spans hang together
    uint64_t end = r[i].end;
    int j = i + 1;
    for (; j < m && r[j].at < end; ++j) end = std::max(end, r[j].end);
    *bad = first_shared(r + i, j - i, true, 0) < 0 ? -1 : shared_bytes(r + i, j - i);
    if (*bad >= 0) return false;
    i = j;
  }
  return true;
}

int launch_reorder(const hs_state* states, int n, int B, int W, int K, const int32_t* parent,
                   int64_t parent_stride, const int32_t* count, hipStream_t stream) {
  __int128 all = 0;
  for (int i = 0; i < n; ++i) all += (__int128)B * K * states[i].rows * states[i].units * states[i].unit;
  const bool stream_past = all >= kStreamBytes;
  const bool wide = all >= kWideBytes * K;
  bool inplace = false;
  for (int i = 0; i < n; ++i) inplace = inplace || states[i].src == states[i].dst;
  const int split = inplace ? 0 : split_of(K, stream_past);
  for (int odd = 0; odd < 2; ++odd) {  // the aligned tensors together, then the others
    int i = 0;
    while (i < n) {
      MoveArgs<kStates> A;
      A.n = 0;
      A.W = W;
      A.K = K;
      A.split = split;
      A.parent = parent;
      A.parent_stride = parent_stride;
      A.count = count;
      uint64_t grid = 0;
      for (; i < n && A.n < kStates; ++i) {
        const hs_state s = in_one_row(states[i], count != nullptr);
        if (aligned(s) == (odd != 0)) continue;
        const int span = span_of(s, K, wide, split);
        const uint64_t parts = parts_of(s, span, split), of = span == 0 ? kWaves >> split : 1;
        const uint64_t wgs = (parts * (uint64_t)s.rows * (uint64_t)B + of - 1) / of;
        // (a tensor of more than a launch's workgroups is by itself, in several launches)
        if (A.n > 0 && grid + wgs > kMostGroups) break;
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
        m.parts = (int)parts;
        m.span = span;
        m.rows = (int)s.rows;
        m.queries = B;
        m.div_parts = make_fastdiv((uint32_t)parts);
        m.div_rows = make_fastdiv((uint32_t)s.rows);
        grid += wgs;
      }
      if (A.n == 0) break;
      for (int j = A.n; j < kStates; ++j) A.first[j] = 0xFFFFFFFFu;
      if (!odd && stream_past) launch_words<true, true>(A, (uint32_t)grid, stream);
      else if (!odd) launch_words<true, false>(A, (uint32_t)grid, stream);
      else if (stream_past) launch_words<false, true>(A, (uint32_t)grid, stream);
      else launch_words<false, false>(A, (uint32_t)grid, stream);
      if (hipPeekAtLastError() != hipSuccess) return HS_ERR_HIP;
    }
  }
  return HS_OK;
}

}  // namespace hs
