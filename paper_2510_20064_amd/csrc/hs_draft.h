// Declarations shared by the kernels that verify a draft (hs_verify.hip, hs_attend.hip, hs_append.hip) and
// their host entries.
#pragma once

#include "hs_beam.h"

namespace hs {

// How a verification's rows are cut: S slices of kVerifySlice 16-byte vectors, one wave each.
constexpr int kVerifySlice = 256;
struct VerifyGeom {
  int B, M, S;
  int64_t V, nvec;
  int dtype;
  bool drafter;
};
bool verify_geom(int B, int M, int64_t V, int dtype, bool drafter, VerifyGeom* g);
size_t verify_ws_bytes(const VerifyGeom& g);
int launch_verify(const VerifyGeom& g, const hs_verify_args& a, hipStream_t stream);

// How an attention is cut: `tiles` workgroups of rw * wr rows of a cached head, and all queries' cached tokens into
// `chunks` ranges (0: a query is one).
struct AttendGeom {
  int B, M, heads, kv, dim, rw, wr, tiles, chunks;
};
bool attend_geom(int B, int M, int heads, int kv, int dim, int page, int slots, AttendGeom* g);
size_t attend_ws_bytes(const AttendGeom& g);  // 0: none
int launch_attend(const AttendGeom& g, const hs_tree_attention_args& a, hipStream_t stream);

int launch_append(const hs_cache_append_args& a, hipStream_t stream);

}  // namespace hs
