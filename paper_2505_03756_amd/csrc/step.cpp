// Host side of the calls over an 8-bit cache, of drafted trees and of accepted paths: argument checks, the records of the
// sequences, and the launches.  C ABI in flpool.h, kernels in attention_step.hip, attention_step_tiles.hip and kv8.hip.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "flp_internal.h"

namespace {

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// e4m3 positions in a block's bytes
int kv8_tokens(const flp_pool* p) { return p->elem_bytes == 2 ? 2 * p->cfg.block_tokens : 0; }

flp_status check_device(const flp_pool* p, const char* who) {
  int cur = -1;
  FLP_TRY_HIP(hipGetDevice(&cur));
  if (cur != p->device) {
    flp_set_error("%s: device %d is current, the pool lives on device %d", who, cur, p->device);
    return FLP_EINVAL;
  }
  return FLP_OK;
}

struct Call {
  const char* who;
  bool kv8, need_qo, need_kv;
  int32_t most_new;            // new tokens that a sequence may have; 0: any number
};

flp_status check_heads(const flp_pool* p, const flp_attn_batch* b, const char* who) {
  if (b->n_q_heads <= 0 || b->n_q_heads % p->cfg.n_kv_heads) {
    flp_set_error("%s: n_q_heads %d is not a multiple of n_kv_heads %d", who, b->n_q_heads, p->cfg.n_kv_heads);
    return FLP_EINVAL;
  }
  return FLP_OK;
}

// The checks of a batch; `recs`: the sequences with new tokens, unit0 and what follows still to be filled in
flp_status check_batch(const flp_pool* p, const flp_attn_batch* b, const flp_kv8_scales* sc, const Call& c, std::vector<FlpStepSeq>* recs) {
  if (!p || !b) {
    flp_set_error("%s: null pool or batch", c.who);
    return FLP_EINVAL;
  }
  if (b->n_seqs < 0 || b->max_blocks_per_seq < 0 || (b->n_seqs > 0 && (!b->cu_new || !b->prefix_len || !b->block_tables)) ||
      !aligned(b->block_tables, 4)) {
    flp_set_error("%s: bad sequence arrays", c.who);
    return FLP_EINVAL;
  }
  if ((p->cfg.block_tokens != 16 && p->cfg.block_tokens != 32) || (p->cfg.head_dim != 64 && p->cfg.head_dim != 128)) {
    flp_set_error("%s: kernels support block_tokens 16 or 32 and head_dim 64/128 (pool has %d / %d)", c.who, p->cfg.block_tokens,
                  p->cfg.head_dim);
    return FLP_ENOTSUP;
  }
  if (c.kv8 && !kv8_tokens(p)) {
    flp_set_error("%s: an fp32 pool holds no 8-bit cache", c.who);
    return FLP_ENOTSUP;
  }
  if (sc && (!sc->k_scale || !sc->v_scale || !aligned(sc->k_scale, 4) || !aligned(sc->v_scale, 4))) {
    flp_set_error("%s: null or misaligned scales", c.who);
    return FLP_EINVAL;
  }
  if (c.need_qo) FLP_TRY(check_heads(p, b, c.who));
  if (b->n_seqs > 0 && b->cu_new[0] != 0) {
    flp_set_error("%s: cu_new[0] must be 0", c.who);
    return FLP_EINVAL;
  }
  const int64_t cap = (int64_t)b->max_blocks_per_seq * (c.kv8 ? kv8_tokens(p) : p->cfg.block_tokens);
  for (int32_t i = 0; i < b->n_seqs; ++i) {
    const int64_t n = (int64_t)b->cu_new[i + 1] - b->cu_new[i];
    if (n < 0 || b->prefix_len[i] < 0) {
      flp_set_error("%s: sequence %d has negative length", c.who, i);
      return FLP_EINVAL;
    }
    if (b->prefix_len[i] + n > cap || b->prefix_len[i] + n > INT32_MAX - 4096) {
      flp_set_error("%s: sequence %d needs %lld positions, its block table covers %lld", c.who, i,
                    (long long)(b->prefix_len[i] + n), (long long)cap);
      return FLP_ERANGE;
    }
    if (c.most_new && n > c.most_new) {
      flp_set_error("%s: sequence %d has %lld new tokens, at most %d supported", c.who, i, (long long)n, c.most_new);
      return FLP_ERANGE;
    }
    if (n > 0) recs->push_back(FlpStepSeq{i, b->cu_new[i], (int32_t)n, b->prefix_len[i], 0, 1, 0, 0});
  }
  if (recs->empty()) return FLP_OK;
  if (c.need_qo && (!b->q || !b->out || !aligned(b->q, 16) || !aligned(b->out, 16))) {
    flp_set_error("%s: q/out must be non-null and 16-byte aligned", c.who);
    return FLP_EINVAL;
  }
  if (c.need_kv && (!b->k_new || !b->v_new || !aligned(b->k_new, 16) || !aligned(b->v_new, 16))) {
    flp_set_error("%s: k_new/v_new must be non-null and 16-byte aligned", c.who);
    return FLP_EINVAL;
  }
  return FLP_OK;
}

FlpStepArgs make_args(const flp_pool* p, const flp_attn_batch* b, const flp_kv8_scales* sc, bool kv8) {
  FlpStepArgs a{};
  a.pool = p->dev_base;
  a.block_bytes = p->block_bytes;
  a.tables = b->block_tables;
  a.max_blocks = b->max_blocks_per_seq;
  a.n_h = b->n_q_heads;
  a.n_kv = p->cfg.n_kv_heads;
  a.pb = kv8 ? kv8_tokens(p) : p->cfg.block_tokens;
  a.head_waves = a.row_waves = 1;
  a.q = b->q;
  a.out = b->out;
  a.k_new = b->k_new;
  a.v_new = b->v_new;
  if (sc) {
    a.k_scale = sc->k_scale;
    a.v_scale = sc->v_scale;
  }
  a.scale_log2e = (b->sm_scale > 0.f ? b->sm_scale : 1.0f / std::sqrt((float)p->cfg.head_dim)) * 1.4426950408889634f;
  return a;
}

// Staging slots and the workspace are handed from call to call by events, which a replayed graph would not see
flp_status refuse_capture(hipStream_t stream, const char* who) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  FLP_TRY_HIP(hipStreamIsCapturing(stream, &st));
  if (st != hipStreamCaptureStatusNone) {
    flp_set_error("%s: this batch needs a staging slot or the pool's workspace and cannot be captured", who);
    return FLP_ENOTSUP;
  }
  return FLP_OK;
}

// The sequences of one append or accept launch, from sequence `first` of the batch on; returns the units of its append, the runs of
// kAppend8Slots positions that get new slots
int64_t seq_list(const flp_attn_batch* b, int32_t first, FlpSeqList<kListSeqs>* l) {
  l->seq0 = first;
  l->n = std::min(kListSeqs, b->n_seqs - first);
  int64_t units = 0;
  for (int32_t i = 0; i < l->n; ++i) {
    const int32_t prefix = b->prefix_len[first + i], n = b->cu_new[first + i + 1] - b->cu_new[first + i];
    l->t0[i] = b->cu_new[first + i];
    l->prefix[i] = prefix;
    l->unit0[i] = (int32_t)units;
    if (n > 0) units += (prefix + n - 1) / kAppend8Slots - prefix / kAppend8Slots + 1;
  }
  l->t0[l->n] = b->cu_new[first + l->n];
  return units;
}

// before anything of the call is enqueued: every launch of its append takes its units, four waves each
flp_status check_append8(const flp_attn_batch* b, const char* who) {
  if (b->cu_new[b->n_seqs] / kAppend8Slots + 2 * kListSeqs <= kMaxWaves / 4) return FLP_OK;
  FlpSeqList<kListSeqs> list;
  for (int32_t first = 0; first < b->n_seqs; first += kListSeqs)
    if (4 * seq_list(b, first, &list) > kMaxWaves) {
      flp_set_error("%s: more new tokens than one launch takes", who);
      return FLP_ERANGE;
    }
  return FLP_OK;
}

flp_status append8(const flp_pool* p, const flp_attn_batch* b, const flp_kv8_scales* sc, hipStream_t stream) {
  const FlpStepArgs a = make_args(p, b, sc, true);
  FlpSeqList<kListSeqs> list;
  for (int32_t first = 0; first < b->n_seqs; first += kListSeqs) {
    const int64_t units = seq_list(b, first, &list);
    FLP_TRY(flp_launch_kv_append8(p->cfg.dtype, p->cfg.head_dim, a, list, (int32_t)units, stream));
  }
  return FLP_OK;
}

// One launch of an attention kernel
struct AttnLaunch {
  std::vector<FlpStepSeq> recs;
  bool tiles;                  // attention_step_tiles.hip
  int32_t head_waves, row_waves, waves, merge_rows;
  int64_t units, units_each;   // units_each: of every record, 0 where they differ
};

bool inline_records(const AttnLaunch& l) {
  if (l.merge_rows || l.recs.size() <= (size_t)kShortList) return l.recs.size() <= (size_t)kStepInline;
  return l.recs.size() <= (size_t)kStepPacked &&
         std::all_of(l.recs.begin(), l.recs.end(), [](const FlpStepSeq& r) { return r.seq < 65536 && r.n < 65536; });
}

constexpr int kMaxPieces = 64;
constexpr int kWaveSlots = 512, kTileSlots = 256;      // workgroups of four waves, and of the tiled kernel, that the chip holds at once

// The pieces of a launch's contexts, `piece` tiles at most, and the places that follow from them; tiles, groups: of each record, tiles
// of its context and workgroups that its rows take
void cut(AttnLaunch& l, int64_t piece, int n_kv, const int64_t* tiles, const int64_t* groups, int64_t* parts) {
  l.units = l.units_each = 0;
  l.merge_rows = 0;
  for (size_t i = 0; i < l.recs.size(); ++i) {
    FlpStepSeq& r = l.recs[i];
    r.pieces = (int32_t)std::min<int64_t>(kMaxPieces, (tiles[i] + piece - 1) / piece);
    r.unit0 = (int32_t)l.units;
    const int64_t units = groups[i] * r.pieces;
    l.units_each = i == 0 || l.units_each == units ? units : 0;
    l.units += units;
    r.part0 = (int32_t)*parts;
    r.merge0 = l.merge_rows;
    if (r.pieces > 1) {
      *parts += (int64_t)r.n * r.pieces;
      l.merge_rows += r.n;
    }
  }
}

// Which kernel takes which sequences, how a workgroup's waves divide the work, and where contexts are cut.  Times below: whole calls, us.
//
// Tiled kernel or few rows.  The first reads K and V once for 256 rows, the second once for 16 (from L2 after the first time).  Few rows / tiled,
// 64 / 8 heads, bf16 trees: 48 sequences of 2000 positions, 48 tokens 674 / 187; 14 of 280, 5 to 15 tokens 17.3 / 13.0; one of 700, 16
// tokens 12.4 / 20; in 8 bits 48 of 1000, 16 tokens 72 / 55, one of 2000, 32 tokens 17 / 26, and with 40 heads of their own, 56 of 600, 6 to 11
// tokens 58 / 152.  So: from 17 rows on (8 bits, where the second kernel reads half as much: 65), where there is enough of it, and not for
// short contexts of few rows (169 of 60, 3 to 9 tokens 36 / 49; 124 of 19 to 191, 3 to 22 tokens 60 / 46).  One launch where either kind
// of sequence is few: 15 of 192 to 1992, 8 to 27 tokens, 32 heads: few rows 55, tiled 57, both kernels 88.
//
// Few rows: waves of a workgroup on slices of a context / on heads / on row tiles.  248 single tokens over 28 positions, 40 heads 111 / 50 / 123; 70
// over 490, 32 heads 52 / 58 / -; 256 over 600, 64 / 8 heads 72 / 69 / 93; 17 sequences of 62 tokens over 210, 40 heads 43 / 43 / 36; 49 of 1
// to 34 tokens over 2300, 32 heads 187 / - / 247 (most of them fill one row tile).  Eight waves: one token over 2000 positions in 8 bits 15.5,
// four 16.5.
//
// Pieces.  A workgroup alone on its CU fetches 64 bytes a nanosecond; pieces cost the launch that merges them, 6 us.  Whole / pieces of 8 tiles / of
// 32, one token, 64 / 8 heads, bf16: 600 positions 10.6 / 13.2 / 10.5; 2000 23 / 13.5 / 21; 8000 75 / 15.3 / 22; eight of 8000 87 / 52 / 48.  48 of
// 1000 fill the chip: 33.5 / 42 / 33.5.  Tiled kernel: a step of a workgroup takes about 1.8 us, what is not in steps about 4; with pieces 5
// for the launch and the partials' way out and back (520 bytes a row).  Trees of 32 to 64 tokens over 8 to 16 k positions, 64 / 8 heads: pieces
// of 90 tiles 283, 40 244, 24 265; 16 prompts of 40 heads whole 213, of 32 tiles 255.
std::vector<AttnLaunch> attn_plan(const flp_pool* p, int G, int elem_bytes, const std::vector<FlpStepSeq>& all, size_t* part_rows) {
  std::vector<AttnLaunch> launches;
  const int n_kv = p->cfg.n_kv_heads, pb = p->cfg.block_tokens * (p->elem_bytes / elem_bytes), run = 64 / elem_bytes;
  const bool tiles_ok = p->elem_bytes == 2 && p->cfg.head_dim == 128;
  const auto length = [](const FlpStepSeq& r) { return (int64_t)r.prefix + r.n; };
  const auto over = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
  const auto fits = [&](const FlpStepSeq& r) { return over(length(r), pb) <= kMfmaMaxBlocks; };
  // 16-row tiles of the queries times tiles of the context, over all kv heads, of the sequences with more than `rows` query rows (w[1]) and
  // of the others; area: of the former, rows times positions of a sequence and kv head, the mean
  int64_t w[2], area = 0;
  const auto work = [&](int rows) {
    int64_t seqs = 0;
    w[0] = w[1] = area = 0;
    for (const FlpStepSeq& r : all) {
      const int64_t R = (int64_t)r.n * G;
      const bool is = tiles_ok && fits(r) && R > rows;
      w[is] += over(R, 16) * over(length(r), run) * n_kv;
      if (!is) continue;
      area += R * length(r);
      ++seqs;
    }
    if (seqs) area /= seqs;
  };
  int from = 16;                                       // sequences with more query rows than that go to the tiled kernel
  work(from);
  if (elem_bytes == 1 || w[1] < 8 * w[0]) work(from = 64);
  if (w[1] <= (elem_bytes == 1 ? 12000 : 6000) || area < 8000)
    from = INT32_MAX;
  else if (w[1] > 8 * w[0])
    from = 0;                                          // what little is left comes along
  const auto tiled = [&](const FlpStepSeq& r) { return tiles_ok && fits(r) && (int64_t)r.n * G > from; };
  int64_t parts = 0;
  std::vector<int64_t> tiles, groups;
  for (int t = 1; t >= 0; --t) {
    AttnLaunch l{};
    l.tiles = t == 1;
    for (const FlpStepSeq& r : all)
      if (tiled(r) == l.tiles) l.recs.push_back(r);
    if (l.recs.empty()) continue;
    std::stable_sort(l.recs.begin(), l.recs.end(), [&](const FlpStepSeq& x, const FlpStepSeq& y) { return length(x) > length(y); });
    l.head_waves = l.row_waves = 1;
    const int tile = l.tiles ? 64 : run;
    if (!l.tiles) {
      int64_t waves = 0, steps = 0;                    // were every row tile of every head one
      for (const FlpStepSeq& r : l.recs) {
        const int64_t x = over((int64_t)r.n * G, 16) * n_kv;
        waves += x;
        steps += x * over(length(r), tile);
      }
      const bool few_steps = waves >= 768 && steps <= 4 * waves;
      if (waves >= 3 * n_kv * (int64_t)l.recs.size() && (waves >= 4 * kWaveSlots || few_steps))
        l.row_waves = 4;
      else if (few_steps || (waves >= 6 * kWaveSlots && steps <= 16 * waves))
        l.head_waves = 4;
    }
    const int per_group = l.tiles ? kMfmaRowsPerItem : 16 * l.row_waves;
    tiles.clear();
    groups.clear();
    int64_t total = 0, units = 0;
    for (const FlpStepSeq& r : l.recs) {
      tiles.push_back(over(length(r), tile));
      groups.push_back(over((int64_t)r.n * G, per_group));
      units += groups.back() * n_kv;
      total += groups.back() * tiles.back() * n_kv;
    }
    const int64_t longest = tiles[0];
    int64_t piece = longest;
    if (l.tiles) {
      double best = 0;
      for (int k = 1; k <= 16 && (k == 1 || over(longest, k) >= 4); ++k) {
        const int64_t cand = over(longest, k);
        int64_t n = 0, kept = 0;
        double sum = 0;
        for (size_t i = 0; i < tiles.size(); ++i) {
          const int64_t pieces = over(tiles[i], cand);
          const double us = 1.8 * tiles[i] / pieces + 4;
          n += groups[i] * pieces * n_kv;
          sum += us * groups[i] * pieces * n_kv;
          if (pieces > 1) kept += pieces * l.recs[i].n;
        }
        const double idle = n % kTileSlots ? 1 - (double)(n % kTileSlots) / kTileSlots : 0;
        const double us = sum / kTileSlots + idle * (sum / n) + (k > 1 ? 5 : 0) + kept * G * n_kv * 1040 / 4e6;
        if (k == 1 || us < best) {
          best = us;
          piece = cand;
        }
      }
      l.waves = 8;
    } else {
      l.waves = 4;
      if (l.row_waves == 1 && l.head_waves == 1) {
        if (units <= kWaveSlots / 2 && longest <= 28)
          l.waves = 8;
        else if (units <= kWaveSlots / 2)
          piece = std::max<int64_t>(8, over(total, kWaveSlots));
        else
          piece = std::max<int64_t>(32, over(2 * total, kWaveSlots));
      }
    }
    cut(l, piece, n_kv, tiles.data(), groups.data(), &parts);
    launches.push_back(std::move(l));
  }
  *part_rows = (size_t)parts;
  return launches;
}

// The attention of a batch that has passed the checks; with_append: K and V of the new tokens are stored before it
flp_status attend(flp_pool* p, const flp_attn_batch* b, const flp_kv8_scales* sc, const uint64_t* mask, bool with_append,
                  const std::vector<FlpStepSeq>& recs, hipStream_t stream, const char* who) {
  std::lock_guard<std::mutex> lk(p->mu);
  size_t part_rows = 0;
  const std::vector<AttnLaunch> launches = attn_plan(p, b->n_q_heads / p->cfg.n_kv_heads, sc ? 1 : p->elem_bytes, recs, &part_rows);
  size_t staged = 0;
  for (const AttnLaunch& l : launches) {
    if (l.units * p->cfg.n_kv_heads * l.waves > kMaxWaves || (int64_t)l.merge_rows * b->n_q_heads > kMaxWaves) {
      flp_set_error("%s: more rows than one launch takes", who);
      return FLP_ERANGE;
    }
    staged += inline_records(l) ? 0 : l.recs.size();
  }
  FlpStageSlot* slot = nullptr;
  FlpStepArgs a = make_args(p, b, sc, sc != nullptr);
  a.mask = mask;
  const bool append16 = with_append && !sc;            // the pool's own append, whose units are staged
  if (staged || part_rows || append16) FLP_TRY(refuse_capture(stream, who));
  if (staged || part_rows) {                           // what may find no memory, before anything is enqueued
    if (part_rows) {
      void* w = nullptr;
      FLP_TRY(flp_attn_workspace(p, part_rows * b->n_q_heads * (p->cfg.head_dim + 2) * sizeof(float), stream, &w));
      a.partials = (float*)w;
    }
    FLP_TRY(flp_stage_acquire(p, staged * sizeof(FlpStepSeq), &slot));
    FlpStepSeq* to = (FlpStepSeq*)slot->host;
    for (const AttnLaunch& l : launches)
      if (!inline_records(l)) to = std::copy(l.recs.begin(), l.recs.end(), to);
  }
  if (append16) FLP_TRY(flp_enqueue_append(p, b, stream));
  flp_status s = staged ? flp_stage_upload(slot, staged * sizeof(FlpStepSeq), stream) : FLP_OK;
  if (s == FLP_OK && with_append && sc) s = append8(p, b, sc, stream);
  const FlpStepSeq* at = slot ? (const FlpStepSeq*)slot->dev : nullptr;
  for (size_t i = 0; i < launches.size() && s == FLP_OK; ++i) {
    const AttnLaunch& l = launches[i];
    a.n_recs = (int32_t)l.recs.size();
    a.merge_rows = l.merge_rows;
    a.units_each = (int32_t)l.units_each;
    a.head_waves = l.head_waves;
    a.row_waves = l.row_waves;
    a.recs = nullptr;
    if (!inline_records(l)) {
      a.recs = at;
      at += l.recs.size();
    }
    s = l.tiles ? flp_launch_attn_step_tiles(p->cfg.dtype, a, l.recs.data(), l.units, stream)
                : flp_launch_attn_step(p->cfg.dtype, p->cfg.head_dim, a, l.recs.data(), l.waves, l.units, stream);
    if (s == FLP_OK) s = flp_launch_attn_step_merge(p->cfg.dtype, p->cfg.head_dim, a, l.recs.data(), stream);
  }
  if (!slot) return s;
  const flp_status released = flp_stage_release(slot, stream);
  if (part_rows && released == FLP_OK) {
    p->attn_slot = slot;
    p->attn_stream = stream;
  }
  return s != FLP_OK ? s : released;
}

// no exception leaves the C ABI: the lists are the only allocations
template <typename F>
flp_status guarded(const char* who, F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    flp_set_error("%s: out of host memory", who);
    return FLP_ENOSPC;
  }
}

}  // namespace

extern "C" int32_t flp_step_attention_route(const flp_pool* p, const flp_attn_batch* b, int32_t kv8) {
  static const char who[] = "flp_step_attention_route";
  int32_t route = 0;
  const flp_status s = guarded(who, [&]() -> flp_status {
    std::vector<FlpStepSeq> recs;
    FLP_TRY(check_batch(p, b, nullptr, Call{who, kv8 != 0, false, false, 0}, &recs));
    FLP_TRY(check_heads(p, b, who));
    size_t part_rows = 0;
    for (const AttnLaunch& l : attn_plan(p, b->n_q_heads / p->cfg.n_kv_heads, kv8 ? 1 : p->elem_bytes, recs, &part_rows)) {
      const int place = !inline_records(l) ? 3 : l.recs.size() <= (size_t)kShortList ? 0 : l.merge_rows ? 1 : 2;
      const int split = l.tiles ? 0 : l.head_waves > 1 ? 1 : l.row_waves > 1 ? 2 : l.waves == 8 ? 3 : 0;
      route |= (1 | (l.merge_rows ? 2 : 0) | 4 * place | 16 * split) << (l.tiles ? 8 : 0);
    }
    return FLP_OK;
  });
  return s == FLP_OK ? route : -1;
}

extern "C" int64_t flp_pool_kv8_block_tokens(const flp_pool* p) { return p ? kv8_tokens(p) : 0; }

extern "C" flp_status flp_kv_append8(flp_pool* p, const flp_attn_batch* b, const flp_kv8_scales* sc, void* hip_stream) {
  static const char who[] = "flp_kv_append8";
  return guarded(who, [&]() -> flp_status {
    std::vector<FlpStepSeq> recs;
    if (!sc) {
      flp_set_error("%s: null scales", who);
      return FLP_EINVAL;
    }
    FLP_TRY(check_batch(p, b, sc, Call{who, true, false, true, 0}, &recs));
    if (recs.empty()) return FLP_OK;
    FLP_TRY(check_append8(b, who));
    FLP_TRY(check_device(p, who));
    return append8(p, b, sc, (hipStream_t)hip_stream);
  });
}

extern "C" flp_status flp_paged_prefix_attention8(flp_pool* p, const flp_attn_batch* b, const flp_kv8_scales* sc, void* hip_stream) {
  static const char who[] = "flp_paged_prefix_attention8";
  return guarded(who, [&]() -> flp_status {
    std::vector<FlpStepSeq> recs;
    if (!sc) {
      flp_set_error("%s: null scales", who);
      return FLP_EINVAL;
    }
    const bool append = b && (b->k_new || b->v_new);
    FLP_TRY(check_batch(p, b, sc, Call{who, true, true, append, 0}, &recs));
    if (recs.empty()) return FLP_OK;
    if (append) FLP_TRY(check_append8(b, who));
    FLP_TRY(check_device(p, who));
    return attend(p, b, sc, nullptr, append, recs, (hipStream_t)hip_stream, who);
  });
}

extern "C" flp_status flp_paged_tree_attention(flp_pool* p, const flp_attn_batch* b, const uint64_t* tree_mask,
                                               const flp_kv8_scales* sc, void* hip_stream) {
  static const char who[] = "flp_paged_tree_attention";
  return guarded(who, [&]() -> flp_status {
    std::vector<FlpStepSeq> recs;
    const bool append = b && (b->k_new || b->v_new);
    FLP_TRY(check_batch(p, b, sc, Call{who, sc != nullptr, true, append, 64}, &recs));
    if (recs.empty()) return FLP_OK;
    if (!tree_mask || !aligned(tree_mask, 8)) {
      flp_set_error("%s: null or misaligned tree_mask", who);
      return FLP_EINVAL;
    }
    FLP_TRY(check_device(p, who));
    return attend(p, b, sc, tree_mask, append, recs, (hipStream_t)hip_stream, who);
  });
}

extern "C" flp_status flp_kv_accept(flp_pool* p, const flp_attn_batch* b, const int32_t* n_accept, const int32_t* path, int32_t kv8,
                                    void* hip_stream) {
  static const char who[] = "flp_kv_accept";
  return guarded(who, [&]() -> flp_status {
    std::vector<FlpStepSeq> recs;
    if (kv8 != 0 && kv8 != 1) {
      flp_set_error("%s: kv8 must be 0 or 1", who);
      return FLP_EINVAL;
    }
    FLP_TRY(check_batch(p, b, nullptr, Call{who, kv8 == 1, false, false, 0}, &recs));
    if (recs.empty()) return FLP_OK;
    if (!n_accept || !path || !aligned(n_accept, 4) || !aligned(path, 4)) {
      flp_set_error("%s: null or misaligned n_accept / path", who);
      return FLP_EINVAL;
    }
    FLP_TRY(check_device(p, who));
    hipStream_t stream = (hipStream_t)hip_stream;
    const FlpStepArgs a = make_args(p, b, nullptr, kv8 == 1);
    FlpSeqList<kListSeqs> list;
    for (int32_t first = 0; first < b->n_seqs; first += kListSeqs) {
      seq_list(b, first, &list);
      FLP_TRY(flp_launch_kv_accept(kv8 ? 1 : p->elem_bytes, p->cfg.head_dim, a, list, n_accept, path, stream));
    }
    return FLP_OK;
  });
}
