// What an attention call over an 8-bit cache or of drafted trees enqueues, in which order, and what it waits for, built and run by
// tests/test_step_order.py on the CPU: the library's own host code with its launches and the runtime's calls replaced by records.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <string>
#include <vector>

#include "flp_internal.h"

#define REQUIRE(cond)                                                                   \
  do {                                                                                  \
    if (!(cond)) {                                                                      \
      std::fprintf(stderr, "step_order: line %d: %s\n", __LINE__, #cond);               \
      for (const Did& d : did) std::fprintf(stderr, "  %s on %p\n", d.what.c_str(), (void*)d.stream); \
      std::exit(1);                                                                     \
    }                                                                                   \
  } while (0)

namespace {
struct Did {
  std::string what;
  hipStream_t stream;
  const void* of;
};
std::vector<Did> did;
bool capturing = false, device_full = false;
flp_status note(const char* what, hipStream_t s, const void* of = nullptr) {
  did.push_back(Did{what, s, of});
  return FLP_OK;
}
const char* step_name(const FlpStepArgs& a, const char* cut, const char* whole) { return a.merge_rows ? cut : whole; }
}  // namespace

flp_status flp_static_scratch_setup(int, void**) { return FLP_EHIP; }
flp_status flp_launch_stage_copy(const void*, void* dst, size_t, hipStream_t s) { return note("upload", s, dst); }
flp_status flp_launch_kv_append(int, int, const FlpAttnArgs&, const FlpAppendUnit*, int32_t, const void*, void*, size_t, hipStream_t s) {
  return note("append", s);
}
flp_status flp_launch_kv_append8(int, int, const FlpStepArgs&, const FlpSeqList<kListSeqs>&, int32_t, hipStream_t s) {
  return note("append8", s);
}
flp_status flp_launch_attn_step(int, int, const FlpStepArgs& a, const FlpStepSeq*, int32_t, int64_t, hipStream_t s) {
  return note(step_name(a, "pieces", "rows"), s, a.merge_rows ? (const void*)a.partials : a.recs);
}
flp_status flp_launch_attn_step_tiles(int, const FlpStepArgs& a, const FlpStepSeq*, int64_t, hipStream_t s) {
  return note(step_name(a, "tile pieces", "tiles"), s, a.merge_rows ? (const void*)a.partials : a.recs);
}
flp_status flp_launch_attn_step_merge(int, int, const FlpStepArgs& a, const FlpStepSeq*, hipStream_t s) {
  return a.merge_rows ? note("merge", s, a.partials) : FLP_OK;
}

extern "C" {
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) {
  *e = reinterpret_cast<hipEvent_t>(new int(0));
  return hipSuccess;
}
hipError_t hipEventDestroy(hipEvent_t e) {
  delete reinterpret_cast<int*>(e);
  return hipSuccess;
}
hipError_t hipEventRecord(hipEvent_t e, hipStream_t s) {
  note("record", s, e);
  return hipSuccess;
}
hipError_t hipEventQuery(hipEvent_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t s, hipEvent_t e, unsigned) {
  note("wait", s, e);
  return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* st) {
  *st = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
hipError_t hipMalloc(void** p, size_t n) {
  if (device_full) return hipErrorOutOfMemory;
  *p = std::malloc(n);
  return hipSuccess;
}
hipError_t hipHostMalloc(void** p, size_t n, unsigned) {
  *p = std::malloc(n);
  return hipSuccess;
}
hipError_t hipFree(void* p) {
  std::free(p);
  return hipSuccess;
}
hipError_t hipHostFree(void* p) { return hipFree(p); }
hipError_t hipGetDevice(int* d) {
  *d = 0;
  return hipSuccess;
}
}

namespace {
const hipStream_t s1 = reinterpret_cast<hipStream_t>(16), s2 = reinterpret_cast<hipStream_t>(32);
void* const at = reinterpret_cast<void*>(1 << 20);     // an address that no check reads

flp_status tree(flp_pool* p, const std::vector<std::pair<int, int>>& seqs, bool append, bool kv8, hipStream_t s) {
  std::vector<int32_t> cu{0}, prefix;
  for (const auto& x : seqs) {
    prefix.push_back(x.first);
    cu.push_back(cu.back() + x.second);
  }
  flp_attn_batch b{};
  b.n_seqs = (int32_t)seqs.size();
  b.n_q_heads = 8;
  b.max_blocks_per_seq = 1000;
  b.q = b.out = at;
  b.k_new = b.v_new = append ? at : nullptr;
  b.cu_new = cu.data();
  b.prefix_len = prefix.data();
  b.block_tables = (const int32_t*)at;
  const flp_kv8_scales sc{(const float*)at, (const float*)at};
  did.clear();
  return flp_paged_tree_attention(p, &b, (const uint64_t*)at, kv8 ? &sc : nullptr, s);
}

flp_pool* make_pool() {
  flp_pool_config cfg{};
  cfg.dtype = FLP_F16;
  cfg.block_tokens = 16;
  cfg.n_kv_heads = 2;
  cfg.head_dim = 128;
  flp_pool* p = nullptr;
  REQUIRE(flp_pool_create(&cfg, &p) == FLP_OK);
  return p;
}

// the calls' names in order, without what is only counted
std::string order() {
  std::string s;
  for (const Did& d : did) s += (s.empty() ? "" : " ") + d.what;
  return s;
}
}  // namespace

int main() {
  const std::vector<std::pair<int, int>> small{{100, 3}, {0, 1}}, cut{{4000, 2}, {3000, 3}}, other{{3900, 1}, {2500, 4}, {50, 2}};
  std::vector<std::pair<int, int>> many(240, {20, 1}), cut_many = many;
  cut_many.push_back({4000, 3});

  {                                                    // one launch, nothing handed from call to call: also under capture
    flp_pool* p = make_pool();
    for (int i = 0; i < 2; ++i) {
      capturing = i == 1;
      REQUIRE(tree(p, small, false, false, s1) == FLP_OK && order() == "rows");
      REQUIRE(tree(p, small, false, true, s1) == FLP_OK && order() == "rows");
      REQUIRE(tree(p, small, true, true, s1) == FLP_OK && order() == "append8 rows");
      if (i == 0) REQUIRE(tree(p, small, true, false, s1) == FLP_OK && order().substr(0, 6) == "append" && order().find(" rows") != order().npos);
    }
    for (bool kv8 : {false, true}) {                   // what needs a slot, the workspace or the pool's own append is refused there
      REQUIRE(tree(p, cut, false, kv8, s1) == FLP_ENOTSUP && did.empty());
      REQUIRE(tree(p, many, true, kv8, s1) == FLP_ENOTSUP && did.empty());
    }
    REQUIRE(tree(p, small, true, false, s1) == FLP_ENOTSUP && did.empty());
    capturing = false;
    flp_pool_destroy(p);
  }
  for (bool kv8 : {false, true}) {                     // the workspace goes from stream to stream behind an event of its last user
    flp_pool* p = make_pool();
    REQUIRE(tree(p, cut, false, kv8, s1) == FLP_OK && order() == "pieces merge record");
    REQUIRE(did[0].of && did[0].of == did[1].of);
    const void* ws = did[0].of;
    const void* first = did[2].of;
    REQUIRE(tree(p, other, false, kv8, s2) == FLP_OK && order() == "wait pieces merge record");
    REQUIRE(did[0].stream == s2 && did[0].of == first && did[1].of == ws && did[3].stream == s2);
    const void* second = did[3].of;
    REQUIRE(second != first);
    REQUIRE(tree(p, cut, false, kv8, s2) == FLP_OK && order() == "pieces merge record");
    const void* third = did[2].of;
    REQUIRE(tree(p, small, false, kv8, s1) == FLP_OK && order() == "rows");
    REQUIRE(tree(p, cut_many, false, kv8, s1) == FLP_OK && order() == "wait upload pieces merge record" && did[0].of == third);
    // staged records: uploaded before they are read, on the call's stream, into a slot that is its own until the event behind the call
    REQUIRE(tree(p, many, false, kv8, s2) == FLP_OK && order() == "upload rows record" && did[0].of == did[1].of);
    const void* slot = did[0].of;
    for (int i = 0; i < kStageSlots - 1; ++i) {
      REQUIRE(tree(p, many, false, kv8, s1) == FLP_OK && did[0].of == did[1].of && did[0].of != slot);
    }
    flp_pool_destroy(p);
  }
  // no room for the workspace: refused with nothing enqueued, the append of K and V among it
  for (bool kv8 : {false, true}) {
    flp_pool* p = make_pool();
    for (int i = 0; i < kStageSlots; ++i) REQUIRE(tree(p, small, true, kv8, s1) == FLP_OK);      // every slot has its memory
    device_full = true;
    REQUIRE(tree(p, cut, true, kv8, s1) == FLP_EHIP && did.empty());
    device_full = false;
    REQUIRE(tree(p, cut, true, kv8, s1) == FLP_OK);
    flp_pool_destroy(p);
  }
  std::printf("in order\n");
  return 0;
}
