// Helpers and geometry of the prefill tile (prefill_tile.inc).
#pragma once

#include "device.hpp"
#include "prefill_common.hpp"

#include <type_traits>

namespace cpattn {

namespace prefill_impl {

typedef __attribute__((address_space(3))) void* lds_ptr_t;

// Compile-time loop: f(std::integral_constant<int, I>) for I in [I0, N).  Every
// index into a register array stays a constant, so the arrays never spill to
// scratch however large the unrolled body gets.
template <int I0, int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I0 < N) {
    f(std::integral_constant<int, I0>());
    static_for<I0 + 1, N>(f);
  }
}

// Marks x as used here (no instruction), so the optimiser cannot sink its
// computation past this point into a later phase.
// (The "v" register constraint exists only for the device pass.)
__device__ __forceinline__ void keep(uint32_t x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" ::"v"(x));
#endif
}
__device__ __forceinline__ void keep(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" ::"v"(x));
#endif
}

// hides the known bits of x from the optimiser (no instruction)
__device__ __forceinline__ uint32_t opaque(uint32_t x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(x));
#endif
  return x;
}

__device__ __forceinline__ void set_word(uint4& v, int e, uint32_t w) {
  if (e == 0) v.x = w;
  else if (e == 1) v.y = w;
  else if (e == 2) v.z = w;
  else v.w = w;
}
__device__ __forceinline__ uint32_t get_word(const uint4& v, int e) {
  return e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w;
}

// 16 bytes per lane from global memory (uniform base + this lane's byte
// offset) straight into LDS at lds + 16 * lane (`lds` wave-uniform, in M0),
// written as the instruction itself.  Built from the compiler's intrinsic,
// the copies were tracked by its wait insertion, which cannot tell which of
// the four LDS tiles a copy in flight fills: it waited for every copy,
// including the K tile issued 1.5 iterations ahead, before the V operand
// reads of every other iteration.  Untracked, the copies are awaited only by
// the explicit vmcnt waits below (no other vector-memory loads run in the
// loop, so the counts are exact; the compiler's own waits for the Q loads
// issued before them only ever wait longer).  The s_nop is the wait state a
// copy needs after M0 is written, which the compiler inserts only for its own.
__device__ __forceinline__ void copy16_to_lds(const uint16_t* base, uint32_t byte_off,
                                              uint8_t* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t dst = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(byte_off), "s"(base),
               "{m0}"(dst)
               : "memory");
#endif
}

// s_waitcnt with vmcnt <= N, the other counters unconstrained (gfx9 encoding)
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 15) | (0x7 << 4) | (0xF << 8) | ((N >> 4) << 14));
}

// until this wave's LDS accesses are done
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xc07f); }

__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

// max and sum of a value over the two 32-lane halves (v_permlane32_swap)
__device__ __forceinline__ float halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int D, int B, int NW>
struct PrefillGeom {
  static constexpr int NKS = D / 16;               // k-steps of S^T (MFMAs per 32-key half)
  static constexpr int NDT = D / 32;               // 32-feature tiles of O^T
  static constexpr int NQK = 2 * NKS;              // K operand reads per step
  static constexpr int NPV = 4 * NDT;              // V operand reads per step
  static constexpr int KCH = D / 8;                // 16-byte chunks per K row
  static constexpr int TILE_BYTES = BN * D * 2;    // one step of K (or of V)
  static constexpr int PIECES = TILE_BYTES / 1024; // 1 KiB copies per step and tensor
  static constexpr int PW = PIECES / NW;           // ... per wave
  static constexpr int KPP = 1024 / (2 * D);       // keys per K piece
  static constexpr int PPB = D * B * 2 / 1024;     // pieces per block (K or V)
  static constexpr int NBW = PW > PPB ? PW / PPB : 1;  // blocks a wave copies per step
  static constexpr int V_ROWS = 1024 / (B * 2);    // V feature rows per piece
  static constexpr int V_LPR = B / 8;              // lanes per V feature row
  static constexpr int LOG2B = B == 16 ? 4 : 5;
  static constexpr int kRing = 3;                  // operand reads ahead of their MFMAs
  static_assert(PW >= 1 && PIECES % NW == 0, "gather geometry");
  static_assert(PW % NBW == 0 && (PW <= PPB ? PPB % PW == 0 : PW % PPB == 0), "piece split");
};

}  // namespace prefill_impl

// What a row of the tile sees: keys up to its own position (a chunk of a prompt).
struct CausalVis {
  static constexpr bool kTree = false;
  // of a tree only
  __device__ int start() const;
  __device__ uint64_t seen(int node, int k0) const;
  template <int D, int B, int NW>
  __device__ void clean(uint8_t* vb, int k0, int tid) const;
};

}  // namespace cpattn
