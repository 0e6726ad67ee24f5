// da_device.hpp -- device code shared by the gfx950 kernels: vector types, the
// matrix instruction, LDS DMA and the transposing LDS reads.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <math.h>

#include <hip/hip_runtime.h>

#include "da_internal.hpp"

namespace da {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The lanes of a wavefront exchange data through LDS here and there (each
// writes its own part, then reads what other lanes wrote).  The hardware runs
// a wave's LDS instructions in order, but the compiler knows nothing of the
// other lanes: without a fence it may move a read above another lane's write
// (into the branch that made that write conditional, say).  This orders every
// LDS access before it against every one after it, with all lanes present.
__device__ __forceinline__ void wave_lds_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Sums and maxima over a wavefront by DPP moves, which cost a few clocks each where an
// exchange through LDS takes about a hundred.  An inclusive scan: shifts by 1, 2, 4 and 8
// inside rows of 16 lanes, then lane 15 of each row to the next one and lane 31 to the
// upper half; lanes without a source take the identity.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_move(int identity, int x) {
  return __builtin_amdgcn_update_dpp(identity, x, CTRL, ROWS, 0xf, false);
}
template <typename Op>
__device__ __forceinline__ int wave_scan(int x, int identity, Op op) {
  x = op(x, dpp_move<0x111, 0xf>(identity, x));
  x = op(x, dpp_move<0x112, 0xf>(identity, x));
  x = op(x, dpp_move<0x114, 0xf>(identity, x));
  x = op(x, dpp_move<0x118, 0xf>(identity, x));
  x = op(x, dpp_move<0x142, 0xa>(identity, x));
  x = op(x, dpp_move<0x143, 0xc>(identity, x));
  return x;
}
__device__ __forceinline__ int wave_scan_add(int x) {
  return wave_scan(x, 0, [](int a, int b) { return a + b; });
}
// (the whole wavefront's, in every lane)
template <typename Op>
__device__ __forceinline__ int wave_reduce(int x, int identity, Op op) {
  return __builtin_amdgcn_readlane(wave_scan(x, identity, op), 63);
}
__device__ __forceinline__ int wave_add(int x) { return __builtin_amdgcn_readlane(wave_scan_add(x), 63); }
// of floats, none of them NaN
__device__ __forceinline__ float wave_fmax(float x) {
  return __int_as_float(wave_reduce(__float_as_int(x), __float_as_int(-INFINITY), [](int a, int b) {
    return __float_as_int(fmaxf(__int_as_float(a), __int_as_float(b)));
  }));
}

// of doubles that are not negative
__device__ __forceinline__ double wave_dmax(double x) {
  auto step = [&](auto move) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint64_t v = (uint64_t)(uint32_t)move((int)(uint32_t)u) | (uint64_t)(uint32_t)move((int)(u >> 32)) << 32;
    x = fmax(x, __builtin_bit_cast(double, v));
  };
  step([](int a) { return dpp_move<0x111, 0xf>(0, a); });
  step([](int a) { return dpp_move<0x112, 0xf>(0, a); });
  step([](int a) { return dpp_move<0x114, 0xf>(0, a); });
  step([](int a) { return dpp_move<0x118, 0xf>(0, a); });
  step([](int a) { return dpp_move<0x142, 0xa>(0, a); });
  step([](int a) { return dpp_move<0x143, 0xc>(0, a); });
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 63) |
                                        (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), 63) << 32);
}

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16 bytes per lane from a buffer into LDS at byte address lds + 16*lane (LDS
// DMA; rsrc and lds are wave-uniform scalars).  Written as asm so that the
// compiler does not track the transfer: its wait-count pass would otherwise
// wait for every DMA in flight before any LDS read it cannot prove disjoint
// from the DMA's target (the V^T reads of the current tile, while the next
// tile's DMA is in flight).  The main loop waits for each tile's DMA itself
// (vmcnt) before the barrier that publishes the tile.  The host pass of the
// kernel templates sees empty bodies.
//
// The compiler inserts no wait states for an instruction inside asm, and the
// hardware does not interlock two of the operands here: a VMEM instruction
// that reads an SGPR written by a VALU instruction (v_readfirstlane, which
// builds the descriptors) needs 5 wait states, and an LDS DMA needs 1 after M0
// is written.  With fewer it can read the SGPR's previous value: a stale
// record count makes the fetch return zeros past it.  So the descriptors and
// the LDS base of a group of DMAs first pass through settle_sgprs (s_nop 4,
// which hands them back as its own outputs: every use comes after it, and
// only scalar arithmetic lies between), and each DMA then waits the one state
// M0 needs.

// A descriptor as read from the first lane (wave-uniform values in scalar
// registers: the compiler cannot hand an "s" asm operand a vector copy).
__device__ __forceinline__ i32x4 first_lane(i32x4 r) {
  return {__builtin_amdgcn_readfirstlane(r[0]), __builtin_amdgcn_readfirstlane(r[1]),
          __builtin_amdgcn_readfirstlane(r[2]), __builtin_amdgcn_readfirstlane(r[3])};
}
__device__ __forceinline__ void settle_sgprs(i32x4& r0, i32x4& r1, uint32_t& m) {
#if defined(__HIP_DEVICE_COMPILE__)
  r0 = first_lane(r0);
  r1 = first_lane(r1);
  m = (uint32_t)__builtin_amdgcn_readfirstlane((int)m);
  asm volatile("s_nop 4" : "+s"(r0), "+s"(r1), "+s"(m));
#endif
}
__device__ __forceinline__ void settle_sgprs(i32x4& r0, uint32_t& m) {
#if defined(__HIP_DEVICE_COMPILE__)
  r0 = first_lane(r0);
  m = (uint32_t)__builtin_amdgcn_readfirstlane((int)m);
  asm volatile("s_nop 4" : "+s"(r0), "+s"(m));
#endif
}
__device__ __forceinline__ void dma16(const i32x4& rsrc, uint32_t lds, int voff) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :: "v"(voff), "s"(rsrc), "{m0}"(lds) : "memory");
#endif
}

// ds_read_b64_tr_b16: inside each group of 16 lanes, lane i receives element
// k (k = 0..3) of the 8-byte row read by lane 4k + i/4, at position i%4.
__device__ __forceinline__ i16x4 lds_read_tr(const uint16_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (i16x4 __attribute__((address_space(3)))*)(p));
}

// Raw scores of NB blocks of 32 keys, capped, in base-2 units of the logits, and base added (see Cap).
// Every instruction per score counts in the prefill kernels, whose vector instructions hide little behind
// the matrix ones.  Delta, 32K tokens, 32 heads on 8, window 2048: 1156 us plain, 1358 capped with unit normal
// queries and keys, 1532 where every score is wide.  (A degree of 9 throughout was 5 % slower than the two
// polynomials; the first block's polynomial between the products of the second gained nothing.)
// Where the wavefront has none past a limit, four or five at the full rate each, and half of one for the
// test.  Else tanh y = 1 - 2 / (1 + e^2y), each score by itself: past the range of e^2y that is -1 or 1, and a
// NaN stays one, as it does in the polynomials, without reaching the scores of other keys.  (One reciprocal
// for four scores needs e^2y held below 2^31 and 13 to 27 registers more, and took longer: the call above with
// wide scores 1585 us against 1539, dense rows of 8192 tokens 633 against 614.)
template <int NB>
__device__ __forceinline__ void cap_scores(f32x16 (&s)[NB], const Cap& cap, float base) {
  float top = 0.f;
#pragma unroll
  for (int q = 0; q < 16; ++q)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) top = fmaxf(top, fabsf(s[nb][q]));
  if (!__any(!(top <= cap.limit[0]))) {
    const float p2 = cap.p[0][2];
#pragma unroll
    for (int q = 0; q < 16; ++q)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float x = s[nb][q], y = x * x;
        s[nb][q] = __builtin_fmaf(x, __builtin_fmaf(y, __builtin_fmaf(y, p2, cap.p[0][1]), cap.p[0][0]), base);
      }
    return;
  }
  if (!__any(!(top <= cap.limit[1]))) {
    const float p3 = cap.p[1][3];
#pragma unroll
    for (int q = 0; q < 16; ++q)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float x = s[nb][q], y = x * x;
        const float p = __builtin_fmaf(y, __builtin_fmaf(y, p3, cap.p[1][2]), cap.p[1][1]);
        s[nb][q] = __builtin_fmaf(x, __builtin_fmaf(y, p, cap.p[1][0]), base);
      }
    return;
  }
  const float c = cap.in, m = -2.f * cap.cap2, one = cap.cap2 + base;
#pragma unroll
  for (int q = 0; q < 16; ++q)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      s[nb][q] = __builtin_fmaf(m, __builtin_amdgcn_rcpf(1.f + fast_exp2(c * s[nb][q])), one);
}

}  // namespace
}  // namespace da
