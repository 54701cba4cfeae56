// Wavefront helpers shared by the kernels: types, cross-lane reductions, LDS
// ordering and the conversions of 8-bit codes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "art_internal.h"

namespace art {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int v2i32 __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_inff();

// The kernel's parameters, read where they are used from the kernel argument
// segment through the scalar cache.  fresh() hides the pointer's origin from
// the compiler: it then loads a phase's fields in that phase, instead of
// holding all of them (about 60 registers' worth, with what it derives from
// them) in scalar registers across the whole kernel.  Held so, 140 of them
// were spilled to lanes of vector registers, and 1170 of the kernel's 3600
// instructions (g = 4) were v_readlane to fetch them back.
typedef const __attribute__((address_space(4))) KernelParams Params;
__device__ __forceinline__ Params* fresh(Params* p) {
  __asm__ __volatile__("" : "+s"(p));
  return p;
}

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// two floats to two bf16 (round to nearest even), one v_cvt_pk_bf16_f32
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

__device__ __forceinline__ uint32_t f32_to_bf16_bits(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7fc0u;  // NaN
  u += 0x7fffu + ((u >> 16) & 1u);                       // round to nearest even
  return u >> 16;
}

// ---- wavefront reductions over the 16 lanes of a DPP row -------------------
template <int CTRL>
__device__ __forceinline__ float dpp_f(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false));
}
constexpr int kQuadXor1 = 0xB1;       // quad_perm [1,0,3,2]
constexpr int kQuadXor2 = 0x4E;       // quad_perm [2,3,0,1]
constexpr int kRowHalfMirror = 0x141; // lane i <- lane 7-i within each 8
constexpr int kRowMirror = 0x140;     // lane i <- lane 15-i within each 16
constexpr int kRowRor4 = 0x124;       // lane i <- lane i-4 of its row of 16 (= i+12)
constexpr int kRowRor8 = 0x128;       // lane i <- lane i-8 (= i+8)

// Every lane of the row ends with the same bits (each step adds the same two
// partial sums, only in swapped operand order).
__device__ __forceinline__ float row_sum(float x) {
  x = x + dpp_f<kQuadXor1>(x);
  x = x + dpp_f<kQuadXor2>(x);
  x = x + dpp_f<kRowHalfMirror>(x);
  x = x + dpp_f<kRowMirror>(x);
  return x;
}
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, dpp_f<kQuadXor1>(x));
  x = fmaxf(x, dpp_f<kQuadXor2>(x));
  x = fmaxf(x, dpp_f<kRowHalfMirror>(x));
  x = fmaxf(x, dpp_f<kRowMirror>(x));
  return x;
}

__device__ __forceinline__ float read_lane(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
// Maximum and sum over the four rows of 16 lanes (lanes l, l ^ 16, l ^ 32,
// l ^ 48), by gfx950's half swaps: each swap hands every lane both operands
// in the same order, so all four lanes end with the same bits.
__device__ __forceinline__ void swap_rows16(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
  a = __int_as_float(r[0]);
  b = __int_as_float(r[1]);
}
__device__ __forceinline__ void swap_rows32(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
  a = __int_as_float(r[0]);
  b = __int_as_float(r[1]);
}
__device__ __forceinline__ float rows_max(float x) {
  float a, b;
  swap_rows16(x, a, b);
  swap_rows32(fmaxf(a, b), a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float rows_sum(float x) {
  float a, b;
  swap_rows16(x, a, b);
  swap_rows32(a + b, a, b);
  return a + b;
}

// LDS written by some lanes of this wave, read by others.  LDS operations of
// one wavefront complete in order; this waits for them and keeps the
// compiler from moving memory operations across.
__device__ __forceinline__ void wave_lds_sync() {
  __asm__ __volatile__("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __builtin_amdgcn_wave_barrier();
  __asm__ __volatile__("" ::: "memory");
}

// The same ordering without the wait, where only this wave touches the
// memory: the LDS unit executes one wavefront's operations in the order they
// were issued, so a read issued after a write of any lane of the wave sees
// it, and a write issued after a read cannot overtake it.  Only the compiler
// has to be kept from reordering them.
__device__ __forceinline__ void wave_lds_order() {
  __asm__ __volatile__("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
  __asm__ __volatile__("" ::: "memory");
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
// single hardware instructions (about 1 ulp): the same bits wherever used
__device__ __forceinline__ float fast_rcp(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ float fast_sqrt(float x) { return __builtin_amdgcn_sqrtf(x); }

// ---- 8-bit codes (FMT: an art_quant_format) --------------------------------
// Eight codes of a lane's sixteen (the lower or the upper half), and eight
// codes in two words, as bf16: exact, as e4m3 holds 4 significant bits and
// int8 at most 8.
template <int FMT>
__device__ __forceinline__ u32x4 codes_bf16(uint32_t x0, uint32_t x1) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t x = i ? x1 : x0;
    if constexpr (FMT == ART_QUANT_E4M3) {
      r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false));
      r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true));
    } else {
      r[2 * i] = pack_bf16((float)(int8_t)x, (float)(int8_t)(x >> 8));
      r[2 * i + 1] = pack_bf16((float)(int8_t)(x >> 16), (float)((int32_t)x >> 24));
    }
  }
  return r;
}
template <int FMT>
__device__ __forceinline__ u32x4 codes_bf16(const u32x4& w, int half) {
  return codes_bf16<FMT>(w[2 * half], w[2 * half + 1]);
}

// V's codes in LDS, 128 bytes a token: token r's 16-byte piece j sits at piece
// j ^ swizzle(r), so that the eight rows that a transposing read touches
// (tokens 4g .. 4g + 3 and 16 more of each, for two lane groups at once) fall
// on distinct banks.  Half a tile takes kCodeStage bytes.
constexpr int kCodeStage = 32 * 128;
__device__ __forceinline__ int code_stage_off(int r, int j) {
  return r * 128 + ((j ^ (((r >> 1) & 1) | ((r >> 4) & 1) << 1 | ((r >> 2) & 1) << 2)) << 4);
}
// The B operand of a P.V product (32 tokens x dims 16d .. 16d + 15): source
// lane 2k + h of each 16 points the transposing read at bytes 8h .. +7 of the
// 16 that row k has there, and lane i receives byte i of all eight rows.
template <int FMT>
__device__ __forceinline__ bf16x8 codes_tr(uint8_t* stage, int row, int d, int lo) {
  const v2i32 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
      (__attribute__((address_space(3))) v2i32*)(stage + code_stage_off(row, d) + 8 * (lo & 1)));
  return __builtin_bit_cast(bf16x8, codes_bf16<FMT>((uint32_t)w[0], (uint32_t)w[1]));
}

// Scores are computed in REP copies over the 16 columns of the matrix
// instruction, and copy u keeps those of the 16-token groups REP i + u: the
// scale of such a group out of those of the tile's four.
template <int REP>
__device__ __forceinline__ float own_scale(float s0, float s1, float s2, float s3, int i, int u) {
  if constexpr (REP == 1) return i == 0 ? s0 : i == 1 ? s1 : i == 2 ? s2 : s3;
  if constexpr (REP == 2) return i == 0 ? (u ? s1 : s0) : (u ? s3 : s2);
  const float a = (u & 1) ? s1 : s0, b = (u & 1) ? s3 : s2;
  return (u & 2) ? b : a;
}

}  // namespace
}  // namespace art
