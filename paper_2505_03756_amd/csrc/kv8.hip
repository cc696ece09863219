// The 8-bit KV cache's append, and the move of an accepted path's K and V (any element size).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "flp_internal.h"
#include "flp_types.h"

namespace {

// x / scale as fp32 division rounds it, limited to what e4m3 holds; a NaN stays one.  With r the rounded reciprocal, q = x r is
// corrected once by its remainder (exact in an fma), which rounds as the division does but for rare last bits; a quotient that lies on
// the border between two e4m3 values is exact.  Limited before the correction as well, so that an infinite x leaves no inf - inf; the
// correction of a zero loses its sign.
__device__ __forceinline__ float quotient(float x, float s, float r) {
  float q = __builtin_amdgcn_fmed3f(x * r, -448.f, 448.f);
  q = fmaf(fmaf(-q, s, x), r, q);
  q = __builtin_amdgcn_fmed3f(q, -448.f, 448.f);
  return x != x ? x : copysignf(q, x);
}

// One workgroup per (run of 32 slots, 1024 elements of a token's row) unit; a thread owns 4 channels of one head.  K: the threads'
// words of a token are contiguous.  V: a thread turns its channels' 32 slots into their 32-byte runs of the transposed V, whole
// sectors; with runs of 16 slots per unit every sector would be written by two workgroups.  A unit that covers part of its run (the ends
// of a sequence's new tokens, single tokens) writes whole words where all four slots are new and single bytes elsewhere.
template <typename S, int D>
__global__ __launch_bounds__(256) void kv_append8_kernel(FlpStepArgs a, FlpStepList list) {
  typedef typename S::storage ST;
  constexpr int SL = kAppend8Slots, C = 4;
  const int row = a.n_kv * D;
  const int e0 = (blockIdx.y * 256 + threadIdx.x) * C;
  const int u = blockIdx.x;
  const FlpStepSeq* __restrict__ recs = a.recs ? a.recs : list.seq;
  int at = -1;
  for (int base = 0; base < a.n_recs; base += 64) {
    const int i = base + (threadIdx.x & 63);
    const unsigned long long le = __builtin_amdgcn_ballot_w64(i < a.n_recs && recs[i].unit0 <= u);
    at += __builtin_popcountll(le);
    if (le != ~0ull) break;
  }
  const FlpStepSeq rec = recs[__builtin_amdgcn_readfirstlane(at)];
  if (e0 >= row) return;
  const int run = rec.prefix / SL + (u - rec.unit0);               // run of the sequence's positions
  const int s0 = rec.prefix > run * SL ? rec.prefix - run * SL : 0;
  const int end = rec.prefix + rec.n - run * SL, s1 = end < SL ? end : SL;
  const int t0 = rec.t0 + run * SL + s0 - rec.prefix;              // token of slot s0
  const int slot0 = run * SL & (a.pb - 1);
  const int64_t blk = a.tables[(int64_t)rec.seq * a.max_blocks + run * SL / a.pb];
  uint8_t* const base = a.pool + blk * a.block_bytes;
  const int g = e0 / D, c0 = e0 - g * D;
  const float ks = a.k_scale[g], vs = a.v_scale[g], kr = 1.f / ks, vr = 1.f / vs;
  uint8_t* const kdst = base + ((int64_t)g * a.pb + slot0) * D + c0;
  uint8_t* const vdst = base + (int64_t)row * a.pb + (int64_t)e0 * a.pb + slot0;
  const ST* const kn = reinterpret_cast<const ST*>(a.k_new) + (int64_t)t0 * row + e0;
  const ST* const vn = reinterpret_cast<const ST*>(a.v_new) + (int64_t)t0 * row + e0;
  const auto word = [&](const ST* p, float s, float r) {
    ST e[C];
    __builtin_memcpy(e, __builtin_assume_aligned(p, 8), sizeof(e));
    float f[C];
#pragma unroll
    for (int i = 0; i < C; ++i) f[i] = quotient(S::to_float(e[i]), s, r);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
    return w;
  };
  if (s0 == 0 && s1 == SL) {
#pragma unroll 8
    for (int s = 0; s < SL; ++s) *reinterpret_cast<uint32_t*>(kdst + s * D) = word(kn + (int64_t)s * row, ks, kr);
#pragma unroll
    for (int h = 0; h < SL / 16; ++h) {
      uint32_t by_slot[16], by_chan[C][4];
#pragma unroll
      for (int s = 0; s < 16; ++s) by_slot[s] = word(vn + (int64_t)(16 * h + s) * row, vs, vr);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          uint32_t w = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) w |= ((by_slot[4 * q + i] >> (8 * c)) & 0xffu) << (8 * i);
          by_chan[c][q] = w;
        }
#pragma unroll
      for (int c = 0; c < C; ++c)
        *reinterpret_cast<u32x4*>(vdst + (int64_t)c * a.pb + 16 * h) = u32x4{by_chan[c][0], by_chan[c][1], by_chan[c][2], by_chan[c][3]};
    }
    return;
  }
  for (int s = s0; s < s1; ++s) {
    *reinterpret_cast<uint32_t*>(kdst + s * D) = word(kn + (int64_t)(s - s0) * row, ks, kr);
    const uint32_t w = word(vn + (int64_t)(s - s0) * row, vs, vr);
#pragma unroll
    for (int c = 0; c < C; ++c) vdst[(int64_t)c * a.pb + s] = (uint8_t)(w >> (8 * c));
  }
}

// One workgroup per (sequence, 256 threads' share of a token's row); a thread owns 16 bytes of K and the channels of these in V and
// walks the path.  Places are taken in increasing order and a place is never behind the token that comes to it, so nothing is
// overwritten before it is read; four moves are read together and then stored, which keeps that.
template <int ES, int D>
__global__ __launch_bounds__(256) void kv_accept_kernel(FlpStepArgs a, FlpStepList list, const int32_t* __restrict__ n_accept,
                                                        const int32_t* __restrict__ path) {
  typedef typename std::conditional<ES == 4, uint32_t, typename std::conditional<ES == 2, uint16_t, uint8_t>::type>::type E;
  constexpr int C = 16 / ES;
  const FlpStepSeq* __restrict__ recs = a.recs ? a.recs : list.seq;
  const FlpStepSeq rec = recs[blockIdx.x];
  const int row = a.n_kv * D, e0 = (blockIdx.y * 256 + threadIdx.x) * C;
  if (e0 >= row) return;
  const int taken = n_accept[rec.seq], m = taken < rec.n ? taken : rec.n;
  const int32_t* const p = path + rec.t0;
  const int32_t* const table = a.tables + (int64_t)rec.seq * a.max_blocks;
  const int g = e0 / D, c0 = e0 - g * D, psh = __builtin_ctz(a.pb);
  const int64_t koff = ((int64_t)g * a.pb * D + c0) * ES, voff = ((int64_t)row * a.pb + (int64_t)e0 * a.pb) * ES;
  constexpr int B = 4;
  bool on = true;
  for (int j0 = 0; j0 < m && on; j0 += B) {
    u32x4 k[B];
    E v[B][C];
    bool move[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int j = j0 + b, src = j < m ? p[j] : -1;
      on = on && src >= 0 && src < rec.n;
      move[b] = on && src != j;
      if (!move[b]) continue;
      const int pos = rec.prefix + src, slot = pos & (a.pb - 1);
      const uint8_t* const blk = a.pool + (int64_t)table[pos >> psh] * a.block_bytes;
      k[b] = *reinterpret_cast<const u32x4*>(blk + koff + (int64_t)slot * D * ES);
#pragma unroll
      for (int c = 0; c < C; ++c) v[b][c] = *reinterpret_cast<const E*>(blk + voff + ((int64_t)c * a.pb + slot) * ES);
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (!move[b]) continue;
      const int pos = rec.prefix + j0 + b, slot = pos & (a.pb - 1);
      uint8_t* const blk = a.pool + (int64_t)table[pos >> psh] * a.block_bytes;
      *reinterpret_cast<u32x4*>(blk + koff + (int64_t)slot * D * ES) = k[b];
#pragma unroll
      for (int c = 0; c < C; ++c) *reinterpret_cast<E*>(blk + voff + ((int64_t)c * a.pb + slot) * ES) = v[b][c];
    }
  }
}

}  // namespace

flp_status flp_launch_kv_append8(int dtype, int head_dim, const FlpStepArgs& a, const FlpStepList& list, int64_t n_units,
                                 hipStream_t stream) {
  if (n_units <= 0) return FLP_OK;
  const dim3 grid((unsigned)n_units, (unsigned)((a.n_kv * head_dim + 1023) / 1024));
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, list); };
  if (dtype == FLP_F16)
    head_dim == 64 ? launch(kv_append8_kernel<F16, 64>) : launch(kv_append8_kernel<F16, 128>);
  else
    head_dim == 64 ? launch(kv_append8_kernel<BF16, 64>) : launch(kv_append8_kernel<BF16, 128>);
  FLP_TRY_HIP(hipGetLastError());
  return FLP_OK;
}

flp_status flp_launch_kv_accept(int elem_bytes, int head_dim, const FlpStepArgs& a, const FlpStepList& list, const int32_t* n_accept,
                                const int32_t* path, hipStream_t stream) {
  if (a.n_recs <= 0) return FLP_OK;
  const int per = 256 * 16 / elem_bytes;
  const dim3 grid((unsigned)a.n_recs, (unsigned)((a.n_kv * head_dim + per - 1) / per));
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, list, n_accept, path); };
  if (elem_bytes == 1)
    head_dim == 64 ? launch(kv_accept_kernel<1, 64>) : launch(kv_accept_kernel<1, 128>);
  else if (elem_bytes == 2)
    head_dim == 64 ? launch(kv_accept_kernel<2, 64>) : launch(kv_accept_kernel<2, 128>);
  else
    head_dim == 64 ? launch(kv_accept_kernel<4, 64>) : launch(kv_accept_kernel<4, 128>);
  FLP_TRY_HIP(hipGetLastError());
  return FLP_OK;
}
