// What the tiled attention kernels share: their types, the swizzles of their LDS layouts and the direct global-to-LDS load
// (attention_mfma.hip, where the layout is described, and attention_step_tiles.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "flp_internal.h"
#include "flp_types.h"

namespace flp_tile {

constexpr int D = 128;
constexpr int BT = 16;
constexpr int BN = 64;                 // keys per tile
constexpr int kTile = BN * D * 2;      // bytes of one K (or V) tile: 16 KiB
constexpr int kStage = 2 * kTile;      // K tile followed by V tile

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));

struct MF16 {
  typedef h16x8 vec;
  static __device__ __forceinline__ f32x4 mfma(vec a, vec b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  // 8 weights -> 16 bit; adds their sum as seen after rounding
  static __device__ __forceinline__ vec pack(const float* p, float& sum) {
    vec v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (_Float16)p[j];
    const h16x2 one = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = __builtin_amdgcn_fdot2(h16x2{v[2 * j], v[2 * j + 1]}, one, sum, false);
    return v;
  }
  static __device__ __forceinline__ uint16_t out(float f) { return F16::from_float(f); }
};
struct MBF16 {
  typedef b16x8 vec;
  static __device__ __forceinline__ f32x4 mfma(vec a, vec b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ vec pack(const float* p, float& sum) {
    vec v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (__bf16)p[j];
    const b16x2 one = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = __builtin_amdgcn_fdot2_f32_bf16(b16x2{v[2 * j], v[2 * j + 1]}, one, sum, false);
    return v;
  }
  static __device__ __forceinline__ uint16_t out(float f) { return BF16::from_float(f); }
};

template <typename V>
__device__ __forceinline__ V as_vec(u32x4 r) {
  V v;
  __builtin_memcpy(&v, &r, 16);
  return v;
}

// XOR term of the K row swizzle: the key's row of its A operand
__device__ __forceinline__ int k_swz(int key32) { return ((key32 >> 3) << 2) | (key32 & 3); }
__device__ __forceinline__ int v_swz(int d) { return ((d >> 2) & 1) ^ ((d >> 3) & 1); }

// One direct global-to-LDS load: every lane fetches 16 bytes from base + voff and the wave's 64
// pieces land at LDS byte address lds .. lds + 1023 in lane order (base and lds wave-uniform).
// Written as inline assembly on purpose: the compiler does not see these loads, so it neither
// counts them in its own memory-counter waits nor makes every later LDS read wait for all of
// them; the kernel orders them against the LDS reads itself (s_waitcnt vmcnt + barrier).
// M0 is named as clobbered so that no pass keeps a value of its own alive in it across the statement; the
// compiler notes that it reserves the register, which is the point.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds16(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(lds)
               : "memory", "m0");
}
#pragma clang diagnostic pop
typedef __attribute__((address_space(3))) uint8_t lds_u8;

}  // namespace flp_tile
