// Prompts over an 8-bit cache and large drafted trees on the matrix cores, head_dim 128: the kernel for calls of attention_step.hip
// with many query rows per kv head.
//
// The walk is attn_mfma_kernel's (attention_mfma.hip describes rows, operands and the LDS layout): a workgroup of eight waves owns up to
// 256 query rows of one (sequence, kv head) and takes K and V through LDS 64 positions at a time, so that they are read once for all
// of them.  What differs:
//
//   8 bit    A thread takes 16 bytes of K and 16 of V of the next tile to registers, a step ahead, and widens them on their way to LDS
//            (K to the type of q, V to fp16, both exact), once for the eight waves.  Two stages, one barrier per tile.
//   masks    A tile in which some row does not see every position is masked by what each row sees: positions up to its own, or its tree's bits.
//            There, values of V that are not finite are taken out (8 bit: on their way to LDS; 16 bit: in LDS) and noted per channel, by
//            position or by bit of the tree, and put into the rows that see them at the end.  16-bit V of the prefix stays as it is in the
//            products; where a result is not finite, the prefix is searched for the channels' infinities, which are the result's however
//            small their weights (in the products a weight rounded to zero would make them NaN).
//   pieces   Contexts of small launches are cut over workgroups as in attention_step.hip and merged by its merge kernel.
//
// Weights are rounded to 16 bits once, and their sum is taken as rounded: an error of half a step of each weight, about as large as that of
// rounding the result, which the few rows of attention_step.hip, bound by memory, avoid with a second piece at no cost (here it would cost
// prompts 222 -> 277 us, long trees over 8 bits 253 -> 345, trees over fp16 277 -> 293).  fp16 weights are lifted as there against the end
// of fp16's range: one is off by 2^-11 of itself or 2^-35 of the largest, whichever is more.
//
// Measured: 16 prompts of 128 to 512 tokens over prefixes of up to 2048, 40 heads, fp16 over 8 bits, 120 GFLOP 217 us; 8 trees of 32 to 64
// tokens over 8 to 16 k positions, 64 / 8 heads, bf16 over 8 bits, 158 GFLOP 233 us and 18 for the merge; a step of a workgroup (256 rows, 64
// positions) takes 1.8 us, of which the matrix instructions are 0.9: their issue and the vector work between the products bound it.  32
// trees of 8 to 64 tokens over 256 to 4096 positions, 40 heads, fp16, 1.47 GB: 276 us, 5.3 TB/s.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "attention_step_record.h"
#include "attention_tile.h"
#include "flp_internal.h"
#include "flp_types.h"

namespace {

using namespace flp_tile;

constexpr int kScheduleAlu = 6;        // __builtin_amdgcn_sched_barrier: vector and scalar arithmetic may cross
constexpr int kWaitVm0 = 0 | (7 << 4) | (15 << 8);

// 8 bytes of e4m3 -> 8 numbers of 16 bits
template <typename M>
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi) {
  u32x4 w;
  if constexpr (std::is_same<M, MF16>::value) {
    const h16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true)};
    __builtin_memcpy(&w, p, 16);
  } else {
    const b16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true),
                        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)};
    __builtin_memcpy(&w, p, 16);
  }
  return w;
}

template <typename M, bool KV8, typename List>
__global__ __launch_bounds__(512, 2) void attn_step_tiles_kernel(FlpStepArgs a, List list) {
  typedef typename M::vec vec;                                       // scores
  typedef typename std::conditional<KV8, MF16, M>::type MV;          // second product
  typedef typename MV::vec wvec;
  constexpr int ES = KV8 ? 1 : 2, kStages = KV8 ? 2 : 3;
  constexpr int kWaitTile = 4 | (7 << 4) | (15 << 8);                // direct loads: all but the newest tile's four have landed
  __shared__ __attribute__((aligned(16))) uint8_t smem[kStages * kStage];
  __shared__ int32_t tab_lds[kMfmaMaxBlocks];                        // the piece's part of the block table
  __shared__ uint64_t odd[2][D];                                     // V not finite: tree bits by sign (NaN both); causal: first NaN's position
  __shared__ uint32_t prefix_odd[KV8 ? 1 : D];                       // V of the prefix, as far as the piece has it: an infinity 1, its negative 2, NaN 3
  __shared__ int32_t any_odd, broken;

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lh = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int u = blockIdx.x / a.n_kv, g = blockIdx.x - u * a.n_kv;
  const FlpStepSeq rec = flp_step_record(a, list, u);
  const int G = a.n_h / a.n_kv, R = rec.n * G, P = rec.prefix, L = P + rec.n;
  const int groups = (R + kMfmaRowsPerItem - 1) / kMfmaRowsPerItem;
  const int local = u - rec.unit0, piece = local / groups;
  const int r0 = (groups - 1 - (local - piece * groups)) * kMfmaRowsPerItem;      // the last rows, which see most, first
  const int row_end = r0 + kMfmaRowsPerItem < R ? r0 + kMfmaRowsPerItem : R;
  const bool tree = a.mask != nullptr;
  const float c = a.scale_log2e * (KV8 ? a.k_scale[g] : 1.f);

  // ---- tiles of the piece
  const int all_tiles = (L + BN - 1) / BN;
  const int lo = (int)((int64_t)all_tiles * piece / rec.pieces);
  int hi = (int)((int64_t)all_tiles * (piece + 1) / rec.pieces);
  const int item_sees = tree ? L : P + (row_end - 1) / G + 1;
  if (hi > (item_sees + BN - 1) / BN) hi = (item_sees + BN - 1) / BN;
  const int all_see = tree ? P : P + r0 / G + 1;                     // positions that every row of the item sees

  // ---- this wave's 32 query rows: rows wrow0 + 16 j + lr, j = 0, 1, of a lane
  const int wrow0 = r0 + wave * 32;
  const bool wave_active = wrow0 < row_end;
  const int wrow_last = wrow0 + 31 < row_end - 1 ? wrow0 + 31 : row_end - 1;
  const int wave_sees = tree ? L : P + wrow_last / G + 1, wave_all_see = tree ? P : P + wrow0 / G + 1;
  int wave_hi = wave_active ? (wave_sees + BN - 1) / BN : 0;
  if (wave_hi > hi) wave_hi = hi;
  int prow[2];                                                       // positions of this lane's rows
  uint64_t bits[2];
  int64_t rowoff[2];
  vec qf[2][4];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = wrow0 + 16 * j + lr, rc = row < row_end ? row : row_end - 1;
    prow[j] = P + rc / G;
    bits[j] = tree ? a.mask[rec.t0 + rc / G] & (~0ull >> (64 - rec.n)) : 0;
    rowoff[j] = ((int64_t)(rec.t0 + rc / G) * a.n_h + (g * G + rc % G)) * D;
    const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q) + rowoff[j] + 8 * lh;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) qf[j][kk] = as_vec<vec>(*reinterpret_cast<const u32x4*>(qp + 32 * kk));
  }
  constexpr bool FP16_W = std::is_same<MV, MF16>::value;
  constexpr float LIFT = FP16_W ? 10.f : 0.f, LAG = FP16_W ? 5.f : 8.f, UNLIFT = FP16_W ? 0x1p-10f : 1.f;      // as in attention_step.hip
  // Scores are differences from the running maximum, as there: its negative is what the first product adds to (subtracted
  // from every score instead: the prompts below 229, the long trees 262 us)
  const float lag = LAG / c;
  f32x4 O[8][2], base[2];
  float mrow[2] = {-INFINITY, -INFINITY}, lsum[2] = {0.f, 0.f};
  base[0] = base[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int ct = 0; ct < 8; ++ct)
#pragma unroll
    for (int j = 0; j < 2; ++j) O[ct][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // ---- staging.  LDS chunk ci (16 bytes) of a 16-position group's K part holds key ci / 16, logical chunk (ci % 16) ^ swizzle(key); chunk
  //      ci of its V part channel ci / 2, positions 8 ((ci % 2) ^ swizzle(channel)) ..  Groups past the piece read its last one again.
  const int pb = a.pb, psh = __builtin_ctz(pb);
  const int last_grp = (L - 1) / BT < 4 * hi - 1 ? (L - 1) / BT : 4 * hi - 1;
  const int blk_lo = lo * BN >> psh;
  if (lo < hi) {
    const int32_t* const table = a.tables + (int64_t)rec.seq * a.max_blocks;
    for (int i = blk_lo + tid; i <= (last_grp * BT >> psh); i += 512) tab_lds[i - blk_lo] = table[i];
  }
  if (tid < D) {
    odd[0][tid] = tree ? 0 : ~0ull >> 1;
    odd[1][tid] = 0;
    if (!KV8) prefix_odd[tid] = 0;
  }
  if (tid == 0) any_odd = broken = 0;
  const auto clamped = [&](int grp) { return grp < last_grp ? grp : last_grp; };
  const auto block_of = [&](int grp) { return tab_lds[(clamped(grp) * BT >> psh) - blk_lo]; };

  // 16 bit: wave w moves group w / 2 of every tile, quarters 2 (w % 2) and the next of its K rows and of its V runs
  const int sblk = wave >> 1;
  const int64_t k_region = (int64_t)g * pb * D * ES, v_region = (int64_t)(a.n_kv + g) * pb * D * ES;
  uint32_t kg[2], vg[2], lds_wave = 0;
  // 8 bit: a thread's 16 channels of key 8 w + lane / 8, and 16 positions of channel 32 (w % 4) + lane % 32 (so that what 16 lanes
  // write to LDS lies in different banks)
  u32x4 rawk, rawv;
  int32_t next_k = 0, next_v = 0;                                    // blocks of the tile that is requested next
  if constexpr (!KV8) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int ci = (2 * (wave & 1) + j) * 64 + lane, key = ci >> 4, vd = ci >> 1;
      kg[j] = (uint32_t)(2 * (key * D + 8 * ((ci & 15) ^ k_swz(16 * (sblk & 1) + key))));
      vg[j] = (uint32_t)(2 * (vd * pb + 8 * ((ci & 1) ^ v_swz(vd))));
    }
    lds_wave = (uint32_t)(uintptr_t)(lds_u8*)smem + sblk * 4096 + 2 * (wave & 1) * 1024;
  }
  const int vch = 32 * (wave & 3) + (lane & 31), vgrp = 2 * (wave >> 2) + (lane >> 5);
  __builtin_amdgcn_s_waitcnt(kWaitVm0);                              // from here on only tile loads are in flight
  __syncthreads();

  const auto request16 = [&](int t, int32_t id) {                    // 4 direct loads: tile t -> its stage
    const int slot = clamped(4 * t + sblk) * BT & (pb - 1);
    const uint8_t* blk = a.pool + (int64_t)__builtin_amdgcn_readfirstlane(id) * a.block_bytes;
    const uint32_t dst = lds_wave + (uint32_t)((t - lo) % kStages) * kStage;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      load_to_lds16(blk + k_region + slot * D * 2, kg[j], dst + j * 1024);
      load_to_lds16(blk + v_region + slot * 2, vg[j], dst + kTile + j * 1024);
    }
  };
  const auto request8 = [&](int t, int32_t idk, int32_t idv) {
    const int kslot = (clamped(4 * t + sblk) * BT & (pb - 1)) + 8 * (wave & 1) + (lane >> 3);
    const int vslot = clamped(4 * t + vgrp) * BT & (pb - 1);
    const uint8_t* const kb = a.pool + (int64_t)__builtin_amdgcn_readfirstlane(idk) * a.block_bytes + k_region;
    const uint8_t* const vb = a.pool + (int64_t)__builtin_amdgcn_readfirstlane(idv) * a.block_bytes + v_region;
    rawk = *reinterpret_cast<const u32x4*>(kb + kslot * D + 16 * (lane & 7));
    rawv = *reinterpret_cast<const u32x4*>(vb + vch * pb + vslot);
  };
  const auto store8 = [&](int t) {                                   // what request8 fetched for tile t -> its stage
    uint8_t* const buf = smem + ((t - lo) % kStages) * kStage;
    const int key16 = 8 * (wave & 1) + (lane >> 3), kx = k_swz(16 * (sblk & 1) + key16);
    uint8_t* const kd = buf + sblk * 4096 + key16 * 256;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<u32x4*>(kd + (((2 * (lane & 7) + h) ^ kx) << 4)) = widen<M>(rawk[2 * h], rawk[2 * h + 1]);
    const int pos0 = BN * t + BT * vgrp;
    if (BN * t + BN > all_see) {                                     // slots past the end are zeroed, NaN that some row does not see noted
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t x = rawv[w];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int pos = pos0 + 4 * w + e;
          const bool nan = ((x >> (8 * e)) & 0x7f) == 0x7f;
          if (pos < L && !(nan && pos >= all_see)) continue;
          if (pos < L) {
            if (tree)
              atomicOr((unsigned long long*)&odd[0][vch], 1ull << (pos - P));
            else
              atomicMin((unsigned long long*)&odd[0][vch], (unsigned long long)pos);
            any_odd = 1;
          }
          x &= ~(0xffu << (8 * e));
        }
        rawv[w] = x;
      }
    }
    uint8_t* const vd = buf + kTile + vgrp * 4096 + vch * 32;
#pragma unroll
    for (int h = 0; h < 2; ++h) *reinterpret_cast<u32x4*>(vd + ((h ^ v_swz(vch)) << 4)) = widen<MF16>(rawv[2 * h], rawv[2 * h + 1]);
  };
  const auto look_up = [&](int t) {
    next_k = block_of(4 * t + sblk);
    if (KV8) next_v = block_of(4 * t + vgrp);                        // both groups of a wave's V lie in one block: it holds 32 positions or more
  };
  if (lo < hi) {
    look_up(lo);
    if constexpr (KV8) {
      request8(lo, next_k, next_v);
      look_up(lo + 1);
      store8(lo);
      request8(lo + 1, next_k, next_v);
      look_up(lo + 2);
    } else {
      request16(lo, next_k);
      look_up(lo + 1);
      request16(lo + 1, next_k);
      look_up(lo + 2);
    }
  }
  const auto request = [&](int kt) {                                 // in step kt: the tile that takes the stage of tile kt - 1
    if constexpr (KV8) {
      if (kt + 1 < hi) store8(kt + 1);                               // past the piece the last group was read again
      request8(kt + 2, next_k, next_v);
      look_up(kt + 3);
    } else {
      request16(kt + 2, next_k);
      look_up(kt + 3);
    }
  };

  // ---- operand fragments, as in attn_mfma_kernel
  const uint32_t kbase = (uint32_t)((8 * (lr >> 2) + (lr & 3)) * 256 + ((lh ^ lr) << 4));
  const uint32_t vbase = (uint32_t)(kTile + (lh >> 1) * 4096 + lr * 32 + (((lh & 1) ^ v_swz(lr)) << 4));
  f32x4 S[4][2];
  wvec Pw[2][2];
  const auto load_k = [&](vec(&kf)[2], const uint8_t* buf, int q) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      kf[i] = *reinterpret_cast<const vec*>(buf + (kbase ^ (uint32_t)((q & 3) << 6)) + (q >> 2) * 8192 + i * 1024);
  };
  const auto load_v = [&](wvec(&vf)[2], const uint8_t* buf, int q) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      vf[i] = *reinterpret_cast<const wvec*>(buf + vbase + (q >> 2) * 8192 + (2 * (q & 3) + i) * 512);
  };
  const auto score = [&](const vec(&kf)[2], int q) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        S[2 * (q >> 2) + i][j] = M::mfma(kf[i], qf[j][q & 3], q & 3 ? S[2 * (q >> 2) + i][j] : base[j]);
  };
  const auto mask = [&](int t) {
    if (BN * t + BN <= wave_all_see) return;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int b = 0; b < 2; ++b) {                                  // positions p0 .. p0 + 7 of the lane
        const int p0 = BN * t + 32 * b + 8 * lh;
        uint32_t vis;
        if (tree) {
          const int before = P - p0 < 0 ? 0 : P - p0 > 8 ? 8 : P - p0, ahead = p0 - P;
          const uint64_t x = ahead >= 64 || ahead <= -8 ? 0 : ahead >= 0 ? bits[j] >> ahead : bits[j] << -ahead;
          vis = ((1u << before) - 1) | (uint32_t)x;
        } else {
          const int n = prow[j] + 1 - p0;
          vis = (1u << (n < 0 ? 0 : n > 8 ? 8 : n)) - 1;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) S[2 * b + (e >> 2)][j][e & 3] = (vis >> e) & 1 ? S[2 * b + (e >> 2)][j][e & 3] : -INFINITY;
      }
  };
  const auto raise = [&]() {                                         // only where a row has outgrown its maximum by 2^LAG
    float tm[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      tm[j] = S[0][j][0];
#pragma unroll
      for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
        for (int i = 0; i < 4; ++i) tm[j] = fmaxf(tm[j], S[k4][j][i]);
    }
    // a maximum of minus infinity: nothing seen yet
    if (__builtin_amdgcn_ballot_w64(tm[0] > (mrow[0] == -INFINITY ? -INFINITY : lag) || tm[1] > (mrow[1] == -INFINITY ? -INFINITY : lag))) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        tm[j] = fmaxf(tm[j], __shfl_xor(tm[j], 16));
        tm[j] = fmaxf(tm[j], __shfl_xor(tm[j], 32));
        const bool first = mrow[j] == -INFINITY;
        const float up = !first ? fmaxf(tm[j], 0.f) : tm[j] == -INFINITY ? 0.f : tm[j];
        const float alpha = first ? 1.f : __builtin_amdgcn_exp2f(-up * c);
        mrow[j] = first ? tm[j] : mrow[j] + up;
        const float from = first && tm[j] == -INFINITY ? 0.f : -mrow[j];
        base[j] = f32x4{from, from, from, from};
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
          for (int i = 0; i < 4; ++i) S[k4][j][i] -= up;
        lsum[j] *= alpha;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct)
#pragma unroll
          for (int i = 0; i < 4; ++i) O[ct][j][i] *= alpha;
      }
    }
  };
  const auto weights = [&](int j, int b) {
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(S[2 * b + (e >> 2)][j][e & 3], c, LIFT));
    Pw[j][b] = MV::pack(p, lsum[j]);
  };
  const auto step = [&](int kt) {
    const uint8_t* buf = smem + ((kt - lo) % kStages) * kStage;
    vec kf[3][2];
    load_k(kf[0], buf, 0);
    load_k(kf[1], buf, 1);
    __builtin_amdgcn_sched_barrier(kScheduleAlu);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      if (q < 6) load_k(kf[(q + 2) % 3], buf, q + 2);
      score(kf[q % 3], q);
      if (q == 3) request(kt);
      __builtin_amdgcn_sched_barrier(kScheduleAlu);
    }
    __builtin_amdgcn_sched_barrier(0);
    wvec vf[3][2];
    load_v(vf[0], buf, 0);
    load_v(vf[1], buf, 1);
    __builtin_amdgcn_sched_barrier(0);
    mask(kt);
    raise();
#pragma unroll
    for (int q = 0; q < 4; ++q) weights(q & 1, q >> 1);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      if (q < 6) load_v(vf[(q + 2) % 3], buf, q + 2);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          O[2 * (q & 3) + i][j] = MV::mfma(vf[q % 3][i], Pw[j][q >> 2], O[2 * (q & 3) + i][j]);
    }
    __builtin_amdgcn_sched_group_barrier(0x002, 40, 0);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      if (q < 6) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
      }
    }
  };
  // 16 bit: the same care as in store8, once the tile has landed
  const auto take_out = [&](int kt) {
    if (KV8 || BN * kt + BN <= all_see) return;
    uint8_t* buf = smem + ((kt - lo) % kStages) * kStage;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int ci = tid + 512 * j;
      const int grp = ci >> 8, vd = (ci & 255) >> 1, vh = (ci & 1) ^ v_swz(vd);
      const int pos0 = BN * kt + BT * grp + 8 * vh;
      u32x4* slot = reinterpret_cast<u32x4*>(buf + kTile + ci * 16);
      u32x4 v = *slot;
      uint16_t e[8];
      __builtin_memcpy(e, &v, 16);
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        constexpr uint16_t kInf = std::is_same<M, MF16>::value ? 0x7c00 : 0x7f80;
        const int pos = pos0 + s;
        const uint16_t size = e[s] & 0x7fff;
        if (pos < all_see || (pos < L && size < kInf)) continue;
        if (pos < L) {                                               // trees only: a prompt over a 16-bit cache is not this kernel's
          if (size > kInf || !(e[s] & 0x8000)) atomicOr((unsigned long long*)&odd[0][vd], 1ull << (pos - P));
          if (size > kInf || (e[s] & 0x8000)) atomicOr((unsigned long long*)&odd[1][vd], 1ull << (pos - P));
          any_odd = 1;
        }
        e[s] = 0;
      }
      __builtin_memcpy(&v, e, 16);
      *slot = v;
    }
    __syncthreads();
  };
  const auto enter = [&](int kt) {                                   // tile kt is in LDS, and nobody reads the stage that is filled next
    if (!KV8) __builtin_amdgcn_s_waitcnt(kWaitTile);
    __syncthreads();
    take_out(kt);
  };
  int kt = lo;
  for (; kt < wave_hi; ++kt) {
    enter(kt);
    step(kt);
  }
  for (; kt < hi; ++kt) {                                            // tiles that only the other waves have keys in
    enter(kt);
    request(kt);
  }
  if constexpr (!KV8) {
    float x = 0.f;                                                   // NaN where one of the sums is not finite
#pragma unroll
    for (int ct = 0; ct < 8; ++ct)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) x = fmaf(O[ct][j][i], 0.f, x);
    if (__builtin_amdgcn_ballot_w64(x != x)) broken = 1;
  }
  __builtin_amdgcn_s_waitcnt(kWaitVm0);                              // the look-ahead loads must land before the LDS is released
  __syncthreads();                                                   // and everybody's notes be there
  if constexpr (!KV8) {
    if (broken) {                                                    // a thread: a channel, every fourth run of 8 positions
      constexpr uint16_t kInf = std::is_same<M, MF16>::value ? 0x7c00 : 0x7f80;
      const int ch = tid & (D - 1), end = all_see < hi * BN ? all_see : hi * BN;
      uint32_t found = 0;
      for (int pos = lo * BN + 8 * (tid >> 7); pos < end; pos += 32) {
        const uint8_t* const blk = a.pool + (int64_t)tab_lds[(pos >> psh) - blk_lo] * a.block_bytes + v_region;
        const u32x4 v = *reinterpret_cast<const u32x4*>(blk + (ch * pb + (pos & (pb - 1))) * 2);
        uint16_t e[8];
        __builtin_memcpy(e, &v, 16);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          const uint16_t size = e[s] & 0x7fff;
          if (pos + s < end && size >= kInf) found |= size > kInf ? 3 : e[s] & 0x8000 ? 2 : 1;
        }
      }
      if (found) atomicOr(&prefix_odd[ch], found);
      __syncthreads();
    }
  }

  // ---- lane (row lr of tile j, quarter lh) holds channels 16 ct + 4 lh + (0..3)
  if (!wave_active) return;
  if (any_odd || (!KV8 && broken)) {
#pragma unroll
    for (int ct = 0; ct < 8; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 16 * ct + 4 * lh + i;
        const uint64_t up = odd[0][ch], down = odd[1][ch];
        const uint32_t before = KV8 ? 0 : prefix_odd[KV8 ? 0 : ch];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (KV8) {                                                 // NaN alone
            if (tree ? (bits[j] & up) != 0 : (uint64_t)prow[j] >= up) O[ct][j][i] = NAN;
          } else {
            const bool plus = (bits[j] & up) || (before & 1), minus = (bits[j] & down) || (before & 2);
            if (plus || minus) O[ct][j][i] = plus && minus ? NAN : plus ? INFINITY : -INFINITY;
          }
        }
      }
  }
  const float vs = KV8 ? a.v_scale[g] : 1.f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float l = lsum[j];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (wrow0 + 16 * j + lr >= row_end) continue;
    const int64_t tok = prow[j] - P;
    if (rec.pieces > 1) {
      const int64_t head = rowoff[j] / D - (rec.t0 + tok) * a.n_h;
      float* const pp = a.partials + ((rec.part0 + tok * rec.pieces + piece) * a.n_h + head) * (D + 2);
      if (lh == 0) *reinterpret_cast<float2*>(pp) = make_float2(mrow[j] * c, l * UNLIFT);
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        float2* const d2 = reinterpret_cast<float2*>(pp + 2 + 16 * ct + 4 * lh);
        d2[0] = make_float2(O[ct][j][0] * (vs * UNLIFT), O[ct][j][1] * (vs * UNLIFT));
        d2[1] = make_float2(O[ct][j][2] * (vs * UNLIFT), O[ct][j][3] * (vs * UNLIFT));
      }
      continue;
    }
    const bool nothing = tree && P == 0 && bits[j] == 0;
    const float inv = 1.f / l;
    uint16_t* op = reinterpret_cast<uint16_t*>(a.out) + rowoff[j] + 4 * lh;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      uint16_t o4[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o4[i] = nothing ? 0 : M::out(O[ct][j][i] * inv * vs);
      uint2 w;
      __builtin_memcpy(&w, o4, 8);
      *reinterpret_cast<uint2*>(op + 16 * ct) = w;
    }
  }
}

}  // namespace

flp_status flp_launch_attn_step_tiles(int dtype, const FlpStepArgs& a, const FlpStepSeq* inline_recs, int64_t n_units, hipStream_t stream) {
  if (n_units <= 0) return FLP_OK;
  flp_with_records(a, inline_recs, [&](const auto& list) {
    typedef typename std::decay<decltype(list)>::type L;
    const auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)(n_units * a.n_kv)), dim3(512), 0, stream, a, list);
    };
    if (dtype == FLP_F16)
      a.k_scale ? launch(attn_step_tiles_kernel<MF16, true, L>) : launch(attn_step_tiles_kernel<MF16, false, L>);
    else
      a.k_scale ? launch(attn_step_tiles_kernel<MBF16, true, L>) : launch(attn_step_tiles_kernel<MBF16, false, L>);
  });
  FLP_TRY_HIP(hipGetLastError());
  return FLP_OK;
}
