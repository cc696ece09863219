// The record that a workgroup of an attention launch works for (attention_step.hip, attention_step_tiles.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "flp_internal.h"

// The last record whose `first` (unit0, or merge0) is not behind `at`, in scalar registers; `at` is the same for the whole wave.  Records in the
// launch's arguments are read there, a single one together with the other arguments.
template <int N>
__device__ __forceinline__ FlpStepSeq flp_step_record(const FlpStepArgs& a, const FlpStepList<N>& list, int at, int32_t FlpStepSeq::*first) {
  if (a.n_recs == 1) return list.seq[0];
  const auto search = [&](auto recs) {
    int found = -1;
    for (int base = 0; base < a.n_recs; base += 64) {
      const int i = base + (threadIdx.x & 63);
      const unsigned long long le = __builtin_amdgcn_ballot_w64(i < a.n_recs && recs(i).*first <= at);
      found += __builtin_popcountll(le);
      if (le != ~0ull) break;
    }
    const FlpStepSeq r = recs(__builtin_amdgcn_readfirstlane(found));
    int32_t w[sizeof(FlpStepSeq) / 4];
    __builtin_memcpy(w, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(FlpStepSeq) / 4); ++i) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
    FlpStepSeq out;
    __builtin_memcpy(&out, w, sizeof(out));
    return out;
  };
  if (a.recs) return search([&](int i) -> const FlpStepSeq& { return a.recs[i]; });
  return search([&](int i) -> const FlpStepSeq& { return list.seq[i]; });
}

// launch(list): the kernel with its records in a list as short as they allow
template <typename F>
void flp_with_records(const FlpStepArgs& a, const FlpStepSeq* inline_recs, F launch) {
  const int n = a.recs ? 0 : a.n_recs;
  if (n <= kShortList) {
    FlpStepList<kShortList> list;
    for (int i = 0; i < n; ++i) list.seq[i] = inline_recs[i];
    launch(list);
  } else {
    FlpStepList<kStepInline> list;
    for (int i = 0; i < n; ++i) list.seq[i] = inline_recs[i];
    launch(list);
  }
}
