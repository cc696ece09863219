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

// Workgroups of K and workgroups of V per unit of 32 slots and 64 Q elements of a token's row; a thread owns 8 channels of Q slots, and all
// its reads are on their way together.  V is turned in registers into Q bytes of each channel's run of the transposed layout; whole runs
// leave by way of LDS, neighbouring lanes side by side in memory.  A unit that covers part of its run (the ends of a sequence's new tokens)
// merges its slots into the words already there, which belong to this sequence alone; units of one or two slots (a decode batch)
// store single bytes of V, neighbouring lanes on neighbouring channels.
//
// Q = 16: bound by memory; 32 prompts of 300 tokens, 40 heads, 295 MB 61 us, 4.8 TB/s (each thread storing its own runs 66 us; 500 drafts of 40
// tokens, 4 heads, whose runs are cut, 33 and 31).  Where runs follow one another and exceed the caches they are stored past these: 20
// prompts of 2000 tokens 264 -> 219 us (32 of 300 the same; blocks of 64 positions 73 -> 80).  256 single tokens of 32 heads 11.5 us, a million
// sectors of 32 bytes written in part (with eight channels per thread 12.6).
// Q = 4: four times as many threads, where a workgroup's 16 x 8 conversions are what a launch waits for: 16 tokens of 8 heads 7.5 -> 4.0
// us, 24 x 64 tokens 8.8 -> 6.8, 512 of 40 heads 8.9 -> 6.7; 2 x 512 (340 workgroups of the other kind) 11.5 either way; and for rows that
// fill a quarter of the other kind's: 100 x 300 tokens of 4 x 64 elements 22.5 -> 16.9, 32 prompts of 300 tokens, 40 heads 61 -> 88.
template <typename S, int D, int Q, int N>
__global__ __launch_bounds__(256) void kv_append8_kernel(FlpStepArgs a, FlpSeqList<N> list) {
  typedef typename S::storage ST;
  typedef uint32_t words __attribute__((ext_vector_type(Q / 4)));
  constexpr int SL = kAppend8Slots, COLS = 64 * Q;     // elements of a token's row that a workgroup takes
  __shared__ u32x4 turn[Q == 16 ? 2048 : 1];
  const int row = a.n_kv * D, u = blockIdx.x;
  const bool is_v = blockIdx.y & 1;
  int rec = -1;                                        // the last sequence whose first unit is not behind u
  for (int base = 0; base < list.n; base += 64) {
    const int i = base + (threadIdx.x & 63);
    const unsigned long long le = __builtin_amdgcn_ballot_w64(i < list.n && list.unit0[i] <= u);
    rec += __builtin_popcountll(le);
    if (le != ~0ull) break;
  }
  rec = __builtin_amdgcn_readfirstlane(rec);
  const int prefix = list.prefix[rec], n = list.t0[rec + 1] - list.t0[rec];
  const int run = prefix / SL + (u - list.unit0[rec]);             // run of the sequence's positions
  const int s0 = prefix > run * SL ? prefix - run * SL : 0;
  const int end = prefix + n - run * SL, s1 = end < SL ? end : SL;
  const int64_t t0 = (int64_t)list.t0[rec] + run * SL - prefix;    // token of slot 0, were it new
  const int slot0 = run * SL & (a.pb - 1);
  const int64_t blk = a.tables[(int64_t)(list.seq0 + rec) * a.max_blocks + run * SL / a.pb];
  uint8_t* const base = a.pool + blk * a.block_bytes;
  const int c0 = (blockIdx.y >> 1) * COLS;
  if (is_v && s1 - s0 <= 2) {
    for (int s = s0; s < s1; ++s) {
      const ST* const src = reinterpret_cast<const ST*>(a.v_new) + (t0 + s) * row;
      ST x[COLS / 256];
#pragma unroll
      for (int j = 0; j < COLS / 256; ++j) x[j] = src[min(c0 + 256 * j + (int)threadIdx.x, row - 1)];
#pragma unroll
      for (int j = 0; j < COLS / 256; ++j) {
        const int e = c0 + 256 * j + threadIdx.x;
        if (e >= row) break;
        const float scale = a.v_scale[e / D], q = quotient(S::to_float(x[j]), scale, 1.f / scale);
        base[(int64_t)(row + e) * a.pb + slot0 + s] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(q, q, 0, false);
      }
    }
    return;
  }
  const int e0 = c0 + (threadIdx.x % (8 * Q)) * 8, h = threadIdx.x / (8 * Q);
  const bool turned = Q == 16 && is_v && s1 - s0 == SL;               // a whole run: by way of LDS, whole lines to memory
  if (!turned && (e0 >= row || s1 <= Q * h || s0 >= Q * h + Q)) return;
  if (e0 < row) {
    const int g = e0 / D;
    const float scale = is_v ? a.v_scale[g] : a.k_scale[g], r = 1.f / scale;
    const ST* const src = reinterpret_cast<const ST*>(is_v ? a.v_new : a.k_new) + t0 * row + e0;
    uint8_t* const dst = base + (is_v ? (int64_t)row * a.pb + (int64_t)e0 * a.pb + slot0 : ((int64_t)g * a.pb + slot0) * D + (e0 - g * D));
    const auto bytes8 = [&](u32x4 x) {
      ST e[8];
      __builtin_memcpy(e, &x, 16);
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = quotient(S::to_float(e[i]), scale, r);
      uint2 w = make_uint2(0, 0);
      w.x = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], w.x, false);
      w.x = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w.x, true);
      w.y = __builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], w.y, false);
      w.y = __builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], w.y, true);
      return w;
    };
    if (s1 - s0 <= 2) {                                // K
      for (int s = s0 > Q * h ? s0 : Q * h; s < s1 && s < Q * h + Q; ++s)
        *reinterpret_cast<uint2*>(dst + (int64_t)s * D) = bytes8(*reinterpret_cast<const u32x4*>(src + (int64_t)s * row));
      return;
    }
    u32x4 x[Q];
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      const int s = Q * h + i;
      if (s >= s0 && s < s1) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (int64_t)s * row));
    }
    uint2 by_slot[Q];
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      const int s = Q * h + i;
      by_slot[i] = bytes8(x[i]);
      if (!is_v && s >= s0 && s < s1) *reinterpret_cast<uint2*>(dst + (int64_t)s * D) = by_slot[i];
    }
    if (!is_v) return;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      words* const at = reinterpret_cast<words*>(dst + (int64_t)c * a.pb + Q * h);
      words w;
#pragma unroll
      for (int q = 0; q < Q / 4; ++q) {
        uint32_t b = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) b |= (((c < 4 ? by_slot[4 * q + i].x : by_slot[4 * q + i].y) >> (8 * (c & 3))) & 0xffu) << (8 * i);
        w[q] = b;
      }
      if constexpr (Q == 16) {
        if (turned) {                                  // channel 8 i + c's half h: place 16 i + 2 c + h, the low four bits turned by i for the banks
          const int i = threadIdx.x & 127;
          turn[16 * i + ((2 * c + h) ^ (i & 15))] = w;
          continue;
        }
      }
      if (s0 > Q * h || s1 < Q * h + Q) {
        const words old = *at;
#pragma unroll
        for (int q = 0; q < Q / 4; ++q) {
          uint32_t mask = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) mask |= Q * h + 4 * q + i >= s0 && Q * h + 4 * q + i < s1 ? 0xffu << (8 * i) : 0u;
          w[q] = (w[q] & mask) | (old[q] & ~mask);
        }
      }
      *at = w;
    }
  }
  if constexpr (Q == 16) {
    if (!turned) return;
    __syncthreads();
    const bool stream = a.pb == SL &&                  // whole lines, and more bytes than the last cache holds
                         (int64_t)gridDim.x * (2 * SL) * row > (int64_t)256 << 20;
    const auto move = [&](auto past) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = 256 * j + threadIdx.x, ch = at >> 1;
        if (c0 + ch >= row) break;
        u32x4* const to = reinterpret_cast<u32x4*>(base + ((int64_t)row + c0 + ch) * a.pb + slot0 + 16 * (at & 1));
        const u32x4 w = turn[(at & ~15) | ((at & 15) ^ ((at >> 4) & 15))];
        if constexpr (decltype(past)::value)
          __builtin_nontemporal_store(w, to);
        else
          *to = w;
      }
    };
    if (stream) {
      asm volatile("");                                // or the compiler makes one of the two
      move(std::true_type());
      asm volatile("");
    } else {
      move(std::false_type());
    }
  }
}

// One workgroup per (sequence, kv head).  Bound by latency (one path of 16 tokens, 8 heads 4.7 us) and, in large batches, by the lines of V
// that the paths' elements lie in, nearly all of the new tokens' blocks (128 paths, 40 heads 24 us).  The path, its length and the blocks
// that the new tokens lie in are requested together, then 32 places of the path at a time are read, K 16 bytes and V an element per
// access with neighbouring threads on neighbouring places of a channel, and stored behind a barrier.  A place is never behind the
// token that comes to it, so what is stored for these places is not read for later ones.
template <int ES, int D, int N>
__global__ __launch_bounds__(256) void kv_accept_kernel(FlpStepArgs a, FlpSeqList<N> list, const int32_t* __restrict__ n_accept,
                                                        const int32_t* __restrict__ path) {
  typedef typename std::conditional<ES == 4, uint32_t, typename std::conditional<ES == 2, uint16_t, uint8_t>::type>::type E;
  constexpr int B = 32, KV = D * ES / 16;              // places at a time; 16-byte pieces of a K row
  constexpr int NK = B * KV / 256 ? B * KV / 256 : 1, NV = B * D / 256;
  const int g = blockIdx.x % a.n_kv, i = blockIdx.x / a.n_kv, seq = list.seq0 + i;
  const int prefix = list.prefix[i], t0 = list.t0[i], n = list.t0[i + 1] - t0;
  if (n == 0) return;
  const int32_t* const p = path + t0;
  const int32_t* const table = a.tables + (int64_t)seq * a.max_blocks;
  const int psh = __builtin_ctz(a.pb), tid = threadIdx.x, lane = tid & 63;
  const int first = prefix >> psh, blocks = ((prefix + n - 1) >> psh) - first + 1;
  int src = lane < n ? p[lane] : -1;                   // lane j: the token of place j
  const int id = lane < blocks ? table[first + lane] : 0;
  const int taken = n_accept[seq], m = taken < n ? taken : n;
  const int64_t k0 = (int64_t)g * a.pb * D * ES, v0 = (int64_t)(a.n_kv + g) * a.pb * D * ES;
  const auto block = [&](int pos) {
    const int b = (pos >> psh) - first;
    const int held = __shfl(id, b & 63);
    return a.pool + (int64_t)(b < 64 ? held : table[first + b]) * a.block_bytes;
  };
  for (int j0 = 0; j0 < m; j0 += B) {
    // the path's next places: lane j holds that of place j0 + j; an entry that is none ends it
    if (j0) src = lane < B && j0 + lane < m ? p[j0 + lane] : -1;
    const unsigned long long bad = __builtin_amdgcn_ballot_w64(lane >= B || j0 + lane >= m || src < 0 || src >= n);
    const int cnt = __builtin_ctzll(bad);              // at most B
    if (cnt == 0) return;                              // the same for all waves
    const int wsh = cnt <= 4 ? 2 : cnt <= 8 ? 3 : cnt <= 16 ? 4 : 5;     // 4, 8, 16 or 32 threads side by side on places
    u32x4 k[NK];
    E v[NV];
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      const int at = x * 256 + tid, j = at / KV, pos = prefix + __shfl(src, j & 63);
      if (x * 256 / KV >= cnt) break;
      const uint8_t* const blk = block(j < cnt ? pos : prefix);
      if (j < cnt) k[x] = *reinterpret_cast<const u32x4*>(blk + k0 + (int64_t)(pos & (a.pb - 1)) * D * ES + at % KV * 16);
    }
#pragma unroll
    for (int x = 0; x < NV; ++x) {
      const int at = x * 256 + tid, j = at & ((1 << wsh) - 1), ch = at >> wsh, pos = prefix + __shfl(src, j);
      if (x * 256 >> wsh >= D) break;
      const bool on = j < cnt && ch < D;
      const uint8_t* const blk = block(on ? pos : prefix);
      if (on) v[x] = *reinterpret_cast<const E*>(blk + v0 + ((int64_t)ch * a.pb + (pos & (a.pb - 1))) * ES);
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      const int at = x * 256 + tid, j = at / KV, pos = prefix + j0 + j;
      if (x * 256 / KV >= cnt) break;
      uint8_t* const blk = block(j < cnt ? pos : prefix);
      if (j < cnt) *reinterpret_cast<u32x4*>(blk + k0 + (int64_t)(pos & (a.pb - 1)) * D * ES + at % KV * 16) = k[x];
    }
#pragma unroll
    for (int x = 0; x < NV; ++x) {
      const int at = x * 256 + tid, j = at & ((1 << wsh) - 1), ch = at >> wsh, pos = prefix + j0 + j;
      if (x * 256 >> wsh >= D) break;
      const bool on = j < cnt && ch < D;
      uint8_t* const blk = block(on ? pos : prefix);
      if (on) *reinterpret_cast<E*>(blk + v0 + ((int64_t)ch * a.pb + (pos & (a.pb - 1))) * ES) = v[x];
    }
    if (cnt < B) return;
  }
}

// launch(list): the kernel with its sequences in a list as short as they allow
template <typename F>
void with_list(const FlpSeqList<kListSeqs>& list, F launch) {
  if (list.n > kShortList) return launch(list);
  FlpSeqList<kShortList> few;
  few.seq0 = list.seq0;
  few.n = list.n;
  for (int i = 0; i < list.n; ++i) {
    few.t0[i] = list.t0[i];
    few.prefix[i] = list.prefix[i];
    few.unit0[i] = list.unit0[i];
  }
  few.t0[list.n] = list.t0[list.n];
  launch(few);
}

}  // namespace

flp_status flp_launch_kv_append8(int dtype, int head_dim, const FlpStepArgs& a, const FlpSeqList<kListSeqs>& list, int32_t n_units,
                                 hipStream_t stream) {
  if (n_units <= 0) return FLP_OK;
  const int row = a.n_kv * head_dim, wide = 2 * ((row + 1023) / 1024);
  const bool few = row <= 256 || (int64_t)n_units * wide < 256;      // fewer workgroups than CUs
  const dim3 grid((unsigned)n_units, few ? 2 * (unsigned)((row + 255) / 256) : (unsigned)wide);
  with_list(list, [&](const auto& l) {
    constexpr int N = sizeof(l.prefix) / sizeof(int32_t);
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, l); };
    const auto by_size = [&](auto q) {
      constexpr int Q = decltype(q)::value;
      if (dtype == FLP_F16)
        head_dim == 64 ? launch(kv_append8_kernel<F16, 64, Q, N>) : launch(kv_append8_kernel<F16, 128, Q, N>);
      else
        head_dim == 64 ? launch(kv_append8_kernel<BF16, 64, Q, N>) : launch(kv_append8_kernel<BF16, 128, Q, N>);
    };
    few ? by_size(std::integral_constant<int, 4>{}) : by_size(std::integral_constant<int, 16>{});
  });
  FLP_TRY_HIP(hipGetLastError());
  return FLP_OK;
}

flp_status flp_launch_kv_accept(int elem_bytes, int head_dim, const FlpStepArgs& a, const FlpSeqList<kListSeqs>& list,
                                const int32_t* n_accept, const int32_t* path, hipStream_t stream) {
  if (list.n <= 0) return FLP_OK;
  const dim3 grid((unsigned)(list.n * a.n_kv));
  with_list(list, [&](const auto& l) {
    constexpr int N = sizeof(l.prefix) / sizeof(int32_t);
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, l, n_accept, path); };
    if (elem_bytes == 1)
      head_dim == 64 ? launch(kv_accept_kernel<1, 64, N>) : launch(kv_accept_kernel<1, 128, N>);
    else if (elem_bytes == 2)
      head_dim == 64 ? launch(kv_accept_kernel<2, 64, N>) : launch(kv_accept_kernel<2, 128, N>);
    else
      head_dim == 64 ? launch(kv_accept_kernel<4, 64, N>) : launch(kv_accept_kernel<4, 128, N>);
  });
  FLP_TRY_HIP(hipGetLastError());
  return FLP_OK;
}
