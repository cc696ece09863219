// The record that a workgroup of an attention launch works for (attention_step.hip, attention_step_tiles.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "flp_internal.h"

// The last of n records whose first unit is not behind `at` (the same for the whole wave): up to 64 records in one trip to memory, up to
// 4096 in two.  first(i): the first unit of record i
template <typename F>
__device__ __forceinline__ int flp_step_search(int n, int at, F first) {
  const int lane = threadIdx.x & 63, stride = (n + 63) >> 6;
  int lo = 0;
  if (stride > 1) {
    const unsigned long long le = __builtin_amdgcn_ballot_w64(lane * stride < n && first(lane * stride) <= at);
    lo = (__builtin_popcountll(le) - 1) * stride;
  }
  for (;; lo += 64) {
    const unsigned long long le = __builtin_amdgcn_ballot_w64(lo + lane < n && first(lo + lane) <= at);
    if (le != ~0ull) return __builtin_amdgcn_readfirstlane(lo + __builtin_popcountll(le) - 1);
  }
}

__device__ __forceinline__ FlpStepSeq flp_step_scalar(const FlpStepSeq& r) {
  int32_t w[sizeof(FlpStepSeq) / 4];
  __builtin_memcpy(w, &r, sizeof(r));
#pragma unroll
  for (int i = 0; i < (int)(sizeof(FlpStepSeq) / 4); ++i) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
  FlpStepSeq out;
  __builtin_memcpy(&out, w, sizeof(out));
  return out;
}

// The record of unit (MERGE: merge row) `at`, in scalar registers.  Where every record has as many units as every other, no search is needed;
// a single record in the arguments comes together with them.
template <bool MERGE = false, int N>
__device__ __forceinline__ FlpStepSeq flp_step_record(const FlpStepArgs& a, const FlpStepList<N>& list, int at) {
  if (a.recs) {
    if (!MERGE && a.units_each) return flp_step_scalar(a.recs[at / a.units_each]);
    return flp_step_scalar(a.recs[flp_step_search(a.n_recs, at, [&](int i) { return MERGE ? a.recs[i].merge0 : a.recs[i].unit0; })]);
  }
  if (a.n_recs == 1) return list.seq[0];
  if (!MERGE && a.units_each) return flp_step_scalar(list.seq[at / a.units_each]);
  return flp_step_scalar(list.seq[flp_step_search(a.n_recs, at, [&](int i) { return MERGE ? list.seq[i].merge0 : list.seq[i].unit0; })]);
}
template <bool MERGE = false>
__device__ __forceinline__ FlpStepSeq flp_step_record(const FlpStepArgs& a, const FlpStepPacked& list, int at) {
  const int i = a.units_each ? at / a.units_each : flp_step_search(a.n_recs, at, [&](int x) { return list.seq[x].unit0; });
  const uint32_t seq_n = __builtin_amdgcn_readfirstlane(list.seq[i].seq_n);
  const int t0 = __builtin_amdgcn_readfirstlane(list.seq[i].t0), prefix = __builtin_amdgcn_readfirstlane(list.seq[i].prefix),
            unit0 = __builtin_amdgcn_readfirstlane(list.seq[i].unit0);
  return FlpStepSeq{(int32_t)(seq_n & 0xffff), t0, (int32_t)(seq_n >> 16), prefix, unit0, 1, 0, 0};
}

// launch(list): the kernel with its records in a list as short as they allow
template <typename F>
void flp_with_records(const FlpStepArgs& a, const FlpStepSeq* inline_recs, F launch) {
  const int n = a.recs ? 0 : a.n_recs;
  if (n <= kShortList) {
    FlpStepList<kShortList> list;
    for (int i = 0; i < n; ++i) list.seq[i] = inline_recs[i];
    launch(list);
  } else if (a.merge_rows) {
    FlpStepList<kStepInline> list;
    for (int i = 0; i < n; ++i) list.seq[i] = inline_recs[i];
    launch(list);
  } else {
    FlpStepPacked list;
    for (int i = 0; i < n; ++i) {
      const FlpStepSeq& r = inline_recs[i];
      list.seq[i] = {(uint32_t)r.seq | (uint32_t)r.n << 16, r.t0, r.prefix, r.unit0};
    }
    launch(list);
  }
}
