// Paged attention of the calls that add to flp_paged_prefix_attention: new tokens over a cache held in e4m3, and trees of up to 64
// drafted tokens over a cache of any type.
//
// For query row r = (new token, query head of kv head g):  out_r = v_scale sum_k w_rk V_k,  w_r = softmax over the k that r sees of
// (sm_scale k_scale) q_r . K_k.  A token sees every position of the prefix; of its sequence's new tokens those up to itself, or
// those whose bit is set in its mask.  A row that sees nothing is zero.
//
// One wave owns 16 rows of one (sequence, kv head) and walks tiles of the context with a running maximum and sum.  K and V go from
// memory to registers 16 bytes per lane and are used there for all rows; nothing is staged.  S^T = K Q^T and O^T = V^T W^T with
// 16x16 instructions: a lane holds one query row (column l % 16) and the RUN = 16 bytes / element size consecutive
// positions from RUN (l / 16) on, because row m of key tile t is key RUN (m / 4) + 4 t + m % 4; these positions are also its 16-byte
// run of the transposed V.  Which channels a step of the scores takes is free as long as K and Q agree, so that a lane's 16 bytes of
// K are one step in 16 bits, two in 8, four (16x16x4) in fp32.
//
//   fp32     fp32 instructions throughout.
//   16 bit   weights in two pieces of the pool's type, the value and its remainder, where one piece would add an error as large as the
//            rounding of the result.  An infinite V would meet a negative remainder, so V is multiplied by zero first, and what is
//            not finite goes another way (below).
//   8 bit    e4m3 is exact in fp16 and in bf16: K is widened to the type of q, V and the weights to fp16, two pieces as well.
//
// In bf16 the pieces hold 16 bits of a weight whatever its size.  In fp16 they hold 22, but nothing below 2^-24, which a long context under one
// dominant key is full of.  So the weight at the running maximum is 2^10 there (LIFT), and the maximum is raised when a row outgrows it
// by 2^5 (LAG), so that no weight exceeds 2^15; a weight is off by 2^-22 of itself or 2^-35 of the largest, whichever is more.  The lift is the
// weights' sum's as well.  More of it leaves less room above the maximum: 2^13 and 2^2 made the tiled kernel's long trees 271 us
// instead of 253 (2^7 and 2^8: 251), for raising the maximum in so many steps.
//
// Exponents are differences from the maximum before they are scaled: the product of a large maximum and the scale has more bits than a float,
// and what its rounding leaves would be the exponent of the largest weight (scores of 2^34: infinite or all zero).
//
// A workgroup is four waves, eight in small launches.  Where the launch has enough of them they are independent, side by side on row tiles
// of a (sequence, kv head), which then read the same K and V at about the same time, or on kv heads; otherwise they take slices of the
// context, merged in LDS.  Contexts of the smallest launches are cut into pieces over workgroups as well, because one CU
// fetches no more than 64 bytes a nanosecond; a second launch merges them in piece order.  For the same reason launches of up to
// half a workgroup per CU whose contexts are whole give each workgroup a part of V's channels and all of K (launch_kind).
//
// Bound by memory: 128 single tokens over 512 to 4096 positions, 32 heads, 8 bits, 2.48 GB: 424 us, 5.8 TB/s; small calls by the trips to
// memory one after the other (arguments, block table, K and V) and by what a CU fetches: one token over 300 positions of 32 heads,
// 8 bits, 7.6 us; a tree of 16 tokens over 700, 64 / 8 heads, bf16, 12.4 us.
//
// Infinities and NaN in V reach the rows that see them and no others: in the tiles where some row does not see everything, and in
// all tiles of 16-bit V, values that are not finite are replaced by zero, and whether a row sees one is counted with products of
// indicators.  They are put in where the slices have been added up: an infinity is the result's however small its weight, which may have
// become zero on the way.  Slots past the end of a sequence hold arbitrary bits and are replaced, never multiplied.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "attention_step_record.h"
#include "flp_internal.h"
#include "flp_types.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(h16x8 a, h16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(b16x8 a, b16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

template <typename V>
__device__ __forceinline__ V bits_as(u32x4 r) {
  V v;
  __builtin_memcpy(&v, &r, 16);
  return v;
}
__device__ __forceinline__ h16x8 widen(uint32_t lo, uint32_t hi, h16x8*) {
  h16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true),
                __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true)};
  h16x8 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
__device__ __forceinline__ b16x8 widen(uint32_t lo, uint32_t hi, b16x8*) {
  b16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true),
                __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)};
  b16x8 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}

template <typename S, bool KV8>
struct Kind {                                          // 16-bit cache
  typedef typename std::conditional<std::is_same<S, F16>::value, h16x8, b16x8>::type kvec;
  typedef kvec vvec;
  static constexpr int ES = 2, STEPS = 1, PIECES = 2;
  static __device__ __forceinline__ kvec k(u32x4 raw, int) { return bits_as<kvec>(raw); }
  static __device__ __forceinline__ vvec v(u32x4 raw, int) { return bits_as<vvec>(raw); }
  static __device__ __forceinline__ uint32_t odd(uint32_t w) {       // high bits set where a value is not finite
    return std::is_same<S, F16>::value ? ((w & 0x7fff7fffu) + 0x04000400u) & 0x80008000u : ((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
  }
};
template <typename S>
struct Kind<S, true> {                                 // e4m3 cache
  typedef typename std::conditional<std::is_same<S, F16>::value, h16x8, b16x8>::type kvec;
  typedef h16x8 vvec;
  static constexpr int ES = 1, STEPS = 2, PIECES = 2;
  static __device__ __forceinline__ kvec k(u32x4 raw, int s) { return widen(raw[2 * s], raw[2 * s + 1], (kvec*)nullptr); }
  static __device__ __forceinline__ vvec v(u32x4 raw, int s) { return widen(raw[2 * s], raw[2 * s + 1], (vvec*)nullptr); }
  static __device__ __forceinline__ uint32_t odd(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
};
template <>
struct Kind<F32, false> {
  typedef float kvec;
  typedef float vvec;
  static constexpr int ES = 4, STEPS = 4, PIECES = 1;
  static __device__ __forceinline__ float k(u32x4 raw, int s) { return __uint_as_float(raw[s]); }
  static __device__ __forceinline__ float v(u32x4 raw, int s) { return __uint_as_float(raw[s]); }
  static __device__ __forceinline__ uint32_t odd(uint32_t w) { return ((w & 0x7fffffffu) + 0x00800000u) & 0x80000000u; }
};

// element e of a step's operand
__device__ __forceinline__ void put(float& v, int, float x) { v = x; }
__device__ __forceinline__ void put(h16x8& v, int e, float x) { v[e] = (_Float16)x; }
__device__ __forceinline__ void put(b16x8& v, int e, float x) { v[e] = (__bf16)x; }
__device__ __forceinline__ float got(float v, int) { return v; }
__device__ __forceinline__ float got(h16x8 v, int e) { return (float)v[e]; }
__device__ __forceinline__ float got(b16x8 v, int e) { return (float)v[e]; }

// W waves per workgroup; VS workgroups side by side on channels of V; List: the records in the arguments
template <typename S, int D, bool KV8, int W, int VS, typename List>
__global__ __launch_bounds__(64 * W, 2) void attn_step_kernel(FlpStepArgs a, List list) {
  typedef Kind<S, KV8> C;
  typedef typename C::kvec kvec;
  typedef typename C::vvec vvec;
  typedef typename S::storage ST;
  constexpr int RUN = 16 / C::ES, TP = 4 * RUN, NT = RUN / 4, KC = D * C::ES / 64, CT = D / 16 / VS, STEPS = C::STEPS;
  constexpr int VE = RUN / STEPS;                      // positions of a lane's run that one step of the second product takes
  constexpr uint32_t ALL = (1u << RUN) - 1;
  __shared__ f32x4 merge_o[W][CT][64];
  __shared__ float2 merge_ml[W][16];
  __shared__ uint8_t flags[W][CT][64];
  __shared__ __attribute__((aligned(8))) uint8_t any_flags[8];

  const int lane = threadIdx.x & 63, lr = lane & 15, lh = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // waves side by side on kv heads, within a head on row tiles, and within those on slices of the context
  const int hw = a.head_waves, rw = a.row_waves, per_head = W / hw, kw = per_head / rw;
  const int head_groups = (a.n_kv + hw - 1) / hw, ub = blockIdx.x / head_groups, u = ub / VS;
  const int ch0 = (ub - u * VS) * (D / VS);            // the workgroup's first channel
  const int own_head = (blockIdx.x - ub * head_groups) * hw + wave / per_head, in_head = wave % per_head;
  const int g = own_head < a.n_kv ? own_head : a.n_kv - 1;
  const FlpStepSeq rec = flp_step_record(a, list, u);
  const int G = a.n_h / a.n_kv, R = rec.n * G, P = rec.prefix, L = P + rec.n;
  const int groups = (R + 16 * rw - 1) / (16 * rw);    // workgroups that the rows take
  const int local = u - rec.unit0, piece = local / groups, rgroup = local - piece * groups;
  const int row0 = (rgroup * rw + in_head % rw) * 16, slice = in_head / rw;
  const bool active = row0 < R && own_head < a.n_kv;
  const int row_last = row0 + 16 < R ? row0 + 15 : R - 1;

  // ---- this lane's place in a tile: its K rows are keys RUN (lr / 4) + 4 t + lr % 4, its run of V starts at position RUN lh
  const int pb = a.pb, psh = __builtin_ctz(pb), last = (L - 1) / RUN;      // the last run that holds a position of the sequence
  const int32_t* __restrict__ table = a.tables + (int64_t)rec.seq * a.max_blocks;
  const auto run_of = [&](int tile, int sel) {         // past the end: the last run again
    const int r = 4 * tile + sel;
    return (r < last ? r : last) * RUN;
  };
  const auto id = [&](int tile, int sel) { return table[run_of(tile, sel) >> psh]; };

  // ---- tiles of the piece, and those of them that this wave's rows see something of
  const int n_tiles = (L + TP - 1) / TP;
  const int lo = (int)((int64_t)n_tiles * piece / rec.pieces);
  int hi = (int)((int64_t)n_tiles * (piece + 1) / rec.pieces);
  const int sees = a.mask ? L : P + row_last / G + 1;  // positions that the wave's rows see together
  if (hi > (sees + TP - 1) / TP) hi = (sees + TP - 1) / TP;
  const int all_see = a.mask ? P : P + row0 / G + 1;   // positions that each of them sees

  u32x4 kr[NT][KC], vr[CT];
  const auto load_k = [&](int tile, int32_t blk) {
    const int slot = (run_of(tile, lr >> 2) & (pb - 1)) + (lr & 3);
    const uint8_t* p = a.pool + (int64_t)blk * a.block_bytes + ((int64_t)(g * pb + slot) * D) * C::ES + 16 * lh;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int cc = 0; cc < KC; ++cc) kr[t][cc] = *reinterpret_cast<const u32x4*>(p + 4 * t * D * C::ES + 64 * cc);
  };
  const auto load_v = [&](int tile, int32_t blk) {
    const int slot = run_of(tile, lh) & (pb - 1);
    const uint8_t* p = a.pool + (int64_t)blk * a.block_bytes + ((int64_t)a.n_kv * pb * D + (int64_t)(g * D + ch0 + lr) * pb + slot) * C::ES;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) vr[ct] = *reinterpret_cast<const u32x4*>(p + (int64_t)16 * ct * pb * C::ES);
  };
  const int tile0 = lo + slice;
  const bool works = active && tile0 < hi;
  int32_t idk = 0, idv = 0;                            // blocks of the tile that is requested next
  if (works) {
    const int32_t k0 = id(tile0, lr >> 2), v0 = id(tile0, lh);
    idk = id(tile0 + kw, lr >> 2);
    idv = id(tile0 + kw, lh);
    load_k(tile0, k0);
    load_v(tile0, v0);
  }

  // ---- the rows: token and head, the queries, what of the new tokens they see
  const int r = row0 + lr, rc = r < R ? r : R - 1, tok = rc / G;
  const int64_t rowoff = ((int64_t)(rec.t0 + tok) * a.n_h + (g * G + rc - tok * G)) * D;
  const uint64_t bits = a.mask ? a.mask[rec.t0 + tok] & (~0ull >> (64 - rec.n)) : 0;
  const float c = a.scale_log2e * (KV8 ? a.k_scale[g] : 1.f);
  kvec qf[KC * STEPS];
#pragma unroll
  for (int cc = 0; cc < KC; ++cc) {
    constexpr int PER = 16 / C::ES;                    // channels of a lane's 16 bytes of K
    const ST* p = reinterpret_cast<const ST*>(a.q) + rowoff + cc * 4 * PER + lh * PER;
    if constexpr (std::is_same<S, F32>::value) {
      const u32x4 raw = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int s = 0; s < STEPS; ++s) qf[cc * STEPS + s] = __uint_as_float(raw[s]);
    } else {
#pragma unroll
      for (int s = 0; s < STEPS; ++s) qf[cc * STEPS + s] = bits_as<kvec>(*reinterpret_cast<const u32x4*>(p + 8 * s));
    }
  }

  constexpr bool FP16_W = std::is_same<vvec, h16x8>::value;
  constexpr float LIFT = FP16_W ? 10.f : 0.f, LAG = FP16_W ? 5.f : 8.f, UNLIFT = FP16_W ? 0x1p-10f : 1.f;
  f32x4 O[CT];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) O[ct] = f32x4{0.f, 0.f, 0.f, 0.f};

  // V with values that are not finite: they are replaced by zero, and which sums they would have gone into is kept, a byte per four
  // channels of a row (bit e of vis: position e of the lane's run); NaN counts as both infinities.  By way of LDS, in a loop that is not
  // unrolled: what is hardly ever run should cost neither registers nor code.
  bool flagged = false;
  const auto not_finite = [&](uint32_t vis) __attribute__((always_inline)) {
    u32x4* const hold = reinterpret_cast<u32x4*>(&merge_o[wave][0][0]) + lane;
    uint8_t* const flag = &flags[wave][0][lane];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) hold[64 * ct] = vr[ct];
#pragma unroll 1
    for (int ct = 0; ct < CT; ++ct) {
      u32x4 v = hold[64 * ct];
      uint32_t f = flagged ? flag[64 * ct] : 0u;
#pragma unroll
      for (int sign = 0; sign < (KV8 ? 1 : 2); ++sign) {             // e4m3 has no infinities
        f32x4 n = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const vvec x = C::v(v, s);
          vvec is, seen;
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float y = got(x, e);
            put(is, e, y != y || y == (sign ? -INFINITY : INFINITY) ? 1.f : 0.f);
            put(seen, e, (vis >> (VE * s + e)) & 1 ? 1.f : 0.f);
          }
          n = mma(is, seen, n);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) f |= n[i] > 0.f ? (KV8 ? 0x11u : sign ? 0x10u : 1u) << i : 0u;
      }
      flag[64 * ct] = (uint8_t)f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {                    // the high bit of each such value, spread over it
        const uint32_t o = C::odd(v[w]);
        v[w] &= ~(C::ES == 4 ? 0u - (o >> 31) : C::ES == 2 ? (o >> 15) * 0xffffu : (o >> 7) * 0xffu);
      }
      hold[64 * ct] = v;
    }
    flagged = true;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) vr[ct] = hold[64 * ct];
  };

  // one tile; the registers of K and V are filled with the wave's next tile as soon as they are used up
  const auto step = [&](int tile) __attribute__((always_inline)) {
    const int next = tile + kw;
    const bool more = next < hi;
    const int32_t next_k = idk, next_v = idv;
    if (more) {
      idk = id(next + kw, lr >> 2);
      idv = id(next + kw, lh);
    }
    f32x4 s[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int cc = 0; cc < KC; ++cc)
#pragma unroll
        for (int st = 0; st < STEPS; ++st) s[t] = mma(C::k(kr[t][cc], st), qf[cc * STEPS + st], s[t]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_k(next, next_k);                 // on their way during the rest of the step
    __builtin_amdgcn_sched_barrier(0);

    const int p0 = TP * tile + RUN * lh;
    const bool careful = TP * tile + TP > all_see;     // some row does not see the whole tile
    uint32_t vis = ALL;
    if (careful) {
      const auto low = [&](int n) { return n <= 0 ? 0u : n >= RUN ? ALL : (1u << n) - 1; };
      if (a.mask) {
        const int ahead = p0 - P;                      // which new token the run's first position holds
        const uint64_t x = ahead >= 64 || ahead <= -64 ? 0 : ahead >= 0 ? bits >> ahead : bits << -ahead;
        vis = low(P - p0) | ((uint32_t)x & ALL);
      } else {
        vis = low(P + tok + 1 - p0);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[t][i] = (vis >> (4 * t + i)) & 1 ? s[t][i] : -INFINITY;
      const uint32_t there = low(L - p0);              // slots past the end hold arbitrary bits
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t keep = 0;
#pragma unroll
        for (int e = 0; e < RUN / 4; ++e)
          if ((there >> (RUN / 4 * w + e)) & 1) keep |= (C::ES == 4 ? 0xffffffffu : C::ES == 2 ? 0xffffu : 0xffu) << (8 * C::ES * e % 32);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) vr[ct][w] &= keep;
      }
    }

    // The running maximum is raised only when a row has outgrown it by 2^LAG: until then weights are relative to the old one
    float tm = s[0][0];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) tm = fmaxf(tm, s[t][i]);
    if (__builtin_amdgcn_ballot_w64((tm - m) * c > LAG)) {
      tm = fmaxf(tm, __shfl_xor(tm, 16));
      tm = fmaxf(tm, __shfl_xor(tm, 32));
      const float mn = fmaxf(m, tm);
      const float alpha = mn == m ? 1.f : __builtin_amdgcn_exp2f((m - mn) * c);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) O[ct][i] *= alpha;
    }
    vvec w[STEPS][C::PIECES];
    const float base = m == -INFINITY ? 0.f : m;       // nothing seen yet: weights 0
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[t][i] - base, c, LIFT));
        sum += x;
        const int e = 4 * t + i;
        put(w[e / VE][0], e % VE, x);
        if constexpr (C::PIECES == 2) put(w[e / VE][1], e % VE, x - got(w[e / VE][0], e % VE));
      }
    l += sum;
    __builtin_amdgcn_sched_barrier(0);
    if (careful || !KV8) {
      bool any = false;
      if constexpr (C::ES == 2) {                      // zero times V: the matrix cores have the time, the vector units have not
        f32x4 z[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
        vvec zero = {};
        asm volatile("" : "+v"(zero));                 // or the products are folded away
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) z[ct & 1] = mma(C::v(vr[ct], 0), zero, z[ct & 1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) any = any || z[0][i] != z[0][i] || z[1][i] != z[1][i];
      } else {
        uint32_t odd = 0;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int x = 0; x < 4; ++x) odd |= C::odd(vr[ct][x]);
        any = odd != 0;
      }
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(any) != 0, 0)) not_finite(vis);
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const vvec v = C::v(vr[ct], st);
#pragma unroll
        for (int pc = C::PIECES - 1; pc >= 0; --pc) O[ct] = mma(v, w[st][pc], O[ct]);
      }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_v(next, next_v);
    __builtin_amdgcn_sched_barrier(0);
  };

  if (works)
    for (int tile = tile0; tile < hi; tile += kw) step(tile);
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // ---- slices of the context, then the result or the piece's share of it.  Lane (row lr, quarter lh): channels 16 ct + 4 lh ..; a wave
  //      takes every kw-th channel tile of its rows.  In a loop that is not unrolled: small calls wait for the code as well
  const float vs = KV8 ? a.v_scale[g] : 1.f;
  if (lh == 0) merge_ml[wave][lr] = make_float2(m, l);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) merge_o[wave][ct][lane] = O[ct];
  if (lane == 0) any_flags[wave] = flagged;
  if (W < 8 && lane == 1) any_flags[W + wave] = 0;
  __syncthreads();
  if (!active) return;
  const int first = wave - slice * rw;
  float M = -INFINITY, total = 0.f, factor[W];
  const bool any = *reinterpret_cast<const uint64_t*>(any_flags) != 0;
  float2 ml[W];
#pragma unroll
  for (int x = 0; x < W; ++x) {
    ml[x] = merge_ml[(first + x * rw) & (W - 1)][lr];
    if (x >= kw) ml[x] = make_float2(-INFINITY, 0.f);
    M = fmaxf(M, ml[x].x);
  }
#pragma unroll
  for (int x = 0; x < W; ++x) {
    factor[x] = ml[x].x == -INFINITY ? 0.f : ml[x].x == M ? 1.f : __builtin_amdgcn_exp2f((ml[x].x - M) * c);
    total = fmaf(ml[x].y, factor[x], total);
  }
  const bool nothing = a.mask && P == 0 && bits == 0;
  const float inv = 1.f / total;                       // apart from the scale, which may be as small as 2^-100
  const int64_t prow = (int64_t)rec.part0 + (int64_t)tok * rec.pieces + piece;
  float* const pp = a.partials + (prow * a.n_h + (g * G + (rc - tok * G))) * (D + 2);
  if (r < R && rec.pieces > 1 && lh == 0 && slice == 0 && ch0 == 0) *reinterpret_cast<float2*>(pp) = make_float2(M * c, total * UNLIFT);
#pragma unroll 1
  for (int ct = slice; ct < CT; ct += kw) {
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < W; ++x) {
      const f32x4 v = merge_o[(first + x * rw) & (W - 1)][ct][lane];
      if (x < kw)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(v[i], factor[x], o[i]);
    }
    if (__builtin_expect(any, 0)) {
      uint32_t f = 0;
      for (int x = 0; x < kw; ++x) {
        const int y = (first + x * rw) & (W - 1);
        if (any_flags[y]) f |= flags[y][ct][lane];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((f >> i) & 1) o[i] += INFINITY;
        if ((f >> (4 + i)) & 1) o[i] -= INFINITY;
      }
    }
    if (r >= R) continue;
    if (rec.pieces > 1) {
      float2* const d2 = reinterpret_cast<float2*>(pp + 2 + ch0 + 16 * ct + 4 * lh);
      const float f = vs * UNLIFT;                     // or a scale of 2^100 would have no room for the sum
      d2[0] = make_float2(o[0] * f, o[1] * f);
      d2[1] = make_float2(o[2] * f, o[3] * f);
      continue;
    }
    ST* const op = reinterpret_cast<ST*>(a.out) + rowoff + ch0 + 16 * ct + 4 * lh;
    ST e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = S::from_float(nothing ? 0.f : o[i] * inv * vs);
    __builtin_memcpy(__builtin_assume_aligned(op, 4 * sizeof(ST)), e, sizeof(e));
  }
}

// The pieces of a (token, head) row, at most 64, in piece order: a wave per row, lane i piece i's maximum and sum, every lane its channels
template <typename S, int D, typename List>
__global__ __launch_bounds__(256) void attn_step_merge_kernel(FlpStepArgs a, List list) {
  typedef typename S::storage ST;
  constexpr int CPL = D / 64;
  typedef float chan __attribute__((ext_vector_type(CPL)));
  const int lane = threadIdx.x & 63;
  const int64_t wid = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(wid / a.n_h), h = (int)(wid - (int64_t)row * a.n_h);
  if (row >= a.merge_rows) return;
  const FlpStepSeq rec = flp_step_record<true>(a, list, row);
  const int tok = row - rec.merge0, ns = rec.pieces;
  const int64_t stride = (int64_t)a.n_h * (D + 2);
  const float* __restrict__ pp = a.partials + ((int64_t)rec.part0 + (int64_t)tok * ns) * stride + (int64_t)h * (D + 2);
  const float* mine = pp + (lane < ns ? lane : 0) * stride;
  const float mi = mine[0], li = mine[1];
  constexpr int B = 16;
  chan q[B];
  const auto request = [&](int i0) {
#pragma unroll
    for (int i = 0; i < B; ++i) q[i] = *reinterpret_cast<const chan*>(pp + (int64_t)(i0 + i < ns ? i0 + i : ns - 1) * stride + 2 + CPL * lane);
  };
  request(0);
  float M = lane < ns ? mi : -INFINITY;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
  // a piece that the row sees nothing of has m = -inf, l = 0 and zeros; any other a weight, 2^-149 (which is as near as its rounding) rather
  // than zero, for the sake of its infinities
  const float wi = lane < ns && mi != -INFINITY ? (mi == M ? 1.f : fmaxf(exp2f(mi - M), 0x1p-149f)) : 0.f;
  float l = lane < ns ? li * wi : 0.f;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) l += __shfl_xor(l, off);
  float acc[CPL];
#pragma unroll
  for (int x = 0; x < CPL; ++x) acc[x] = 0.f;
  for (int i0 = 0; i0 < ns; i0 += B) {
    if (i0) request(i0);
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const float w = __shfl(wi, (i0 + i) & 63);
      if (i0 + i < ns)
#pragma unroll
        for (int x = 0; x < CPL; ++x) acc[x] = fmaf(q[i][x], w, acc[x]);
    }
  }
  const bool nothing = a.mask && rec.prefix == 0 && (a.mask[rec.t0 + tok] & (~0ull >> (64 - rec.n))) == 0;
  const float inv = 1.f / l;
  ST* op = reinterpret_cast<ST*>(a.out) + ((int64_t)(rec.t0 + tok) * a.n_h + h) * D + CPL * lane;
#pragma unroll
  for (int x = 0; x < CPL; ++x) op[x] = S::from_float(nothing ? 0.f : acc[x] * inv);
}

template <typename S, int D>
void launch_kind(const FlpStepArgs& a, const FlpStepSeq* recs, int waves, unsigned groups, hipStream_t stream) {
  flp_with_records(a, recs, [&](const auto& list) {
    typedef typename std::decay<decltype(list)>::type L;
    const auto launch = [&](auto kernel, int parts = 1) {
      hipLaunchKernelGGL(kernel, dim3(groups * parts), dim3(64 * waves), 0, stream, a, list);
    };
    const auto by_waves = [&](auto kv8) {
      constexpr bool KV8 = decltype(kv8)::value;
      if (waves == 4) return launch(attn_step_kernel<S, D, KV8, 4, 1, L>);
      // Workgroups on parts of V's channels, as many as leave one for each CU.  Whole / 2 / 4 parts, us: one token over 300 positions, 32 heads,
      // bf16 9.0 / - / 8.0; 16 over 700, 64 / 8 heads 13.3 / - / 12.1; 16 over 300, fp32 15.7 / - / 12.8; 128 workgroups: four tokens over
      // 700, 32 heads 16.6 / 15.0 / 18.5; 200: three times 16 over 700, 64 / 8 heads 14.9 / 23.8 / 25.
      if constexpr (std::is_same<L, FlpStepList<kShortList>>::value) {
        if (groups <= 64) return launch(attn_step_kernel<S, D, KV8, 8, 4, L>, 4);
        if (groups <= 128) return launch(attn_step_kernel<S, D, KV8, 8, 2, L>, 2);
      }
      launch(attn_step_kernel<S, D, KV8, 8, 1, L>);
    };
    if constexpr (!std::is_same<S, F32>::value)
      if (a.k_scale) return by_waves(std::true_type());
    by_waves(std::false_type());
  });
}

}  // namespace

flp_status flp_launch_attn_step(int dtype, int head_dim, const FlpStepArgs& a, const FlpStepSeq* inline_recs, int32_t waves, int64_t n_units,
                                hipStream_t stream) {
  if (n_units <= 0) return FLP_OK;
  const unsigned grid = (unsigned)(n_units * ((a.n_kv + a.head_waves - 1) / a.head_waves));
  const auto launch = [&](auto kind64, auto kind128) {
    head_dim == 64 ? kind64(a, inline_recs, waves, grid, stream) : kind128(a, inline_recs, waves, grid, stream);
  };
  if (dtype == FLP_F32)
    launch(launch_kind<F32, 64>, launch_kind<F32, 128>);
  else if (dtype == FLP_F16)
    launch(launch_kind<F16, 64>, launch_kind<F16, 128>);
  else
    launch(launch_kind<BF16, 64>, launch_kind<BF16, 128>);
  FLP_TRY_HIP(hipGetLastError());
  return FLP_OK;
}

flp_status flp_launch_attn_step_merge(int dtype, int head_dim, const FlpStepArgs& a, const FlpStepSeq* inline_recs, hipStream_t stream) {
  if (a.merge_rows <= 0) return FLP_OK;
  const dim3 grid((unsigned)(((int64_t)a.merge_rows * a.n_h + 3) / 4));
  flp_with_records(a, inline_recs, [&](const auto& list) {
    typedef typename std::decay<decltype(list)>::type L;
    const bool d64 = head_dim == 64;
    const auto merge = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, list); };
    if (dtype == FLP_F32)
      d64 ? merge(attn_step_merge_kernel<F32, 64, L>) : merge(attn_step_merge_kernel<F32, 128, L>);
    else if (dtype == FLP_F16)
      d64 ? merge(attn_step_merge_kernel<F16, 64, L>) : merge(attn_step_merge_kernel<F16, 128, L>);
    else
      d64 ? merge(attn_step_merge_kernel<BF16, 64, L>) : merge(attn_step_merge_kernel<BF16, 128, L>);
  });
  FLP_TRY_HIP(hipGetLastError());
  return FLP_OK;
}
