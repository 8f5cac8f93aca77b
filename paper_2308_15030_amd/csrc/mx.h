// 8-bit values with scales, as SMOE_MXFP8 layers hold them: blocks of 32 numbers along the reduction, each an e4m3 value
// (4 significant bits, largest magnitude 448) times one power of two for the block, kept as exponent + 127 in a byte.  The matrix cores
// multiply such operands with the scales inside the instruction (v_mfma_scale_f32_32x32x64_f8f6f4), so nothing is
// widened on the way.
//
// The scale of a block is the smallest power of two with which its largest magnitude does not exceed 448: nothing saturates, and a
// value of the block that is at least 2^-6 in units of the scale is off by at most 2^-4 of itself (half a step of e4m3), a smaller one by
// at most 2^-10 units.
//
// Sums.  The accumulators are fp32, but inside an instruction the matrix core adds 8 consecutive products at a time with what lies
// below 2^-13 of the largest of them rounded off (seen with single products beside larger ones; groups of 8 are added to one another and
// to the accumulator with 24 bits).  Beside the 2^-4 of the operands that is little: the products of 2426 rows of 416 x 1696 are 1.9e-3 off
// 64-bit sums of the same 8-bit values, of which rounding the result to bf16 is 1.7e-3.
//
// Operand order.  One instruction takes 32 rows (features or tokens) x 64 reduction elements of each operand, 32 bytes a lane:
// lane l holds of row l % 32 the elements 16 h .. 16 h + 15 and 32 + 16 h .. 32 + 16 h + 15, h = l / 32, and its scale register the scale of the
// row's elements 32 h .. 32 h + 31.  A matrix [rows][reduction] in operand order is
//     elements  [rows / 32][step of 64][half 2][lane 64][16 bytes]
//     scales    [rows / 32][group of 4 steps][lane 64][4 bytes, one a step]
// so that an operand is two contiguous 1-KiB loads, and the scales of four steps one of 256 bytes.  A reduction that ends in the middle of a
// step is filled with zeros up to the step's end.
#pragma once

#include "smoe_internal.h"

typedef int smoe_i32x8 __attribute__((ext_vector_type(8)));
typedef float smoe_mx_acc __attribute__((ext_vector_type(16)));

// Exponent + 127 of a block's scale from its largest magnitude (448 = 1.75 * 2^8), kept to [1, 254]: a block of zeros has the smallest.
__device__ __forceinline__ uint32_t smoe_mx_scale(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u);
    return (uint32_t)max(e, 1);
}
// 2^-e of a scale: exact, and so are its products with numbers that e4m3 does not round to zero.
__device__ __forceinline__ float smoe_mx_inverse(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }

// Four values, in units of the scale already, as e4m3 (to nearest, ties to even): the conversion instruction.
__device__ __forceinline__ uint32_t smoe_mx_pack(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// acc += A . B of one step; S: the byte of the scale registers that belongs to the step.
template <int S>
__device__ __forceinline__ void smoe_mx_mfma(smoe_mx_acc& acc, const uint4 (&a)[2], const uint4 (&b)[2], uint32_t sa, uint32_t sb) {
    const smoe_i32x8 av = {(int)a[0].x, (int)a[0].y, (int)a[0].z, (int)a[0].w, (int)a[1].x, (int)a[1].y, (int)a[1].z, (int)a[1].w};
    const smoe_i32x8 bv = {(int)b[0].x, (int)b[0].y, (int)b[0].z, (int)b[0].w, (int)b[1].x, (int)b[1].y, (int)b[1].z, (int)b[1].w};
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(av, bv, acc, 0, 0, S, (int)sa, S, (int)sb);
}

// The lanes' lower halves of a and b in a, the upper halves in b: a = {a.lo, b.lo}, b = {a.hi, b.hi}.
__device__ __forceinline__ void smoe_swap_halves(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
