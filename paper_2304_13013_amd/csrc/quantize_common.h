// Device helpers shared by the quantizers (quantize.hip, which describes the arithmetic, and quantize_block.hip).
#pragma once
#include "sb_common.h"

namespace sb {
namespace {

constexpr float kRoundMagic = 12582912.0f;  // 1.5 * 2^23

enum { CODE_INT8 = 0, CODE_E4M3 = 1, CODE_E5M2 = 2 };

__device__ __forceinline__ unsigned int pk_absmax_u16(unsigned int running, unsigned int two_bf16) {
    v2us a = __builtin_bit_cast(v2us, running);
    v2us b = __builtin_bit_cast(v2us, two_bf16 & 0x7fff7fffu);
    return __builtin_bit_cast(unsigned int, __builtin_elementwise_max(a, b));
}

__device__ __forceinline__ unsigned int absmax_of_chunk(unsigned int running, v4u c) {
    running = pk_absmax_u16(running, c.x);
    running = pk_absmax_u16(running, c.y);
    running = pk_absmax_u16(running, c.z);
    return pk_absmax_u16(running, c.w);
}

__device__ __forceinline__ unsigned int wave_max_u32(unsigned int v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        unsigned int o = (unsigned int)__shfl_xor((int)v, off, 64);
        v = o > v ? o : v;
    }
    return v;
}

// absmax bit pattern (15 bits) -> (scale t, stored state).  Zero rows and rows whose scale would overflow
// binary32 quantize to zeros and store state 0.
template <int CODE = CODE_INT8>
__device__ __forceinline__ float scale_from_absmax_bits(unsigned int bits15, float *stored_state) {
    float s = bf16_bits_to_float(bits15);
    float t = (CODE == CODE_INT8 ? 127.0f : 1.0f) / s;
    if (bits15 == 0u || __builtin_isinf(t)) {
        t = 0.0f;
        s = 0.0f;
    }
    *stored_state = s;
    return t;
}

__device__ __forceinline__ unsigned int code_bits(float x, float t) {
    float p = x * t;            // one rounding
    float r = p + kRoundMagic;  // second rounding: nearest-even integer lands in the low mantissa bits
    return __float_as_uint(r);
}

// 8 bf16 (4 dwords, element 2d in the low half of dword d) -> 8 one-byte codes (2 dwords).
template <int CODE = CODE_INT8>
__device__ __forceinline__ v2u quantize_chunk(v4u c, float t) {
    if (CODE != CODE_INT8) {
        const unsigned int d[4] = {c.x, c.y, c.z, c.w};
        float p[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            p[2 * j] = __uint_as_float(d[j] << 16) * t;  // one rounding each
            p[2 * j + 1] = __uint_as_float(d[j] & 0xffff0000u) * t;
        }
        int lo = 0, hi = 0;  // the conversion writes one 16-bit half of its destination and keeps the other
        if (CODE == CODE_E4M3) {
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(p[0], p[1], lo, false);
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(p[2], p[3], lo, true);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(p[4], p[5], hi, false);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(p[6], p[7], hi, true);
        } else {
            lo = __builtin_amdgcn_cvt_pk_bf8_f32(p[0], p[1], lo, false);
            lo = __builtin_amdgcn_cvt_pk_bf8_f32(p[2], p[3], lo, true);
            hi = __builtin_amdgcn_cvt_pk_bf8_f32(p[4], p[5], hi, false);
            hi = __builtin_amdgcn_cvt_pk_bf8_f32(p[6], p[7], hi, true);
        }
        return v2u{(unsigned int)lo, (unsigned int)hi};
    }
    unsigned int r[8];
    r[0] = code_bits(__uint_as_float(c.x << 16), t);
    r[1] = code_bits(__uint_as_float(c.x & 0xffff0000u), t);
    r[2] = code_bits(__uint_as_float(c.y << 16), t);
    r[3] = code_bits(__uint_as_float(c.y & 0xffff0000u), t);
    r[4] = code_bits(__uint_as_float(c.z << 16), t);
    r[5] = code_bits(__uint_as_float(c.z & 0xffff0000u), t);
    r[6] = code_bits(__uint_as_float(c.w << 16), t);
    r[7] = code_bits(__uint_as_float(c.w & 0xffff0000u), t);
    // v_perm_b32: selector bytes 0-3 pick from the second operand, 4-7 from the first, 0x0c gives zero.
    unsigned int p01 = __builtin_amdgcn_perm(r[1], r[0], 0x0c0c0400u);
    unsigned int p23 = __builtin_amdgcn_perm(r[3], r[2], 0x0c0c0400u);
    unsigned int p45 = __builtin_amdgcn_perm(r[5], r[4], 0x0c0c0400u);
    unsigned int p67 = __builtin_amdgcn_perm(r[7], r[6], 0x0c0c0400u);
    v2u out;
    out.x = __builtin_amdgcn_perm(p23, p01, 0x05040100u);
    out.y = __builtin_amdgcn_perm(p67, p45, 0x05040100u);
    return out;
}

constexpr int kTile = 128;
// The tile's codes sit in LDS row-major as dwords (4 codes each), 33 dwords per row and the lower half of the rows
// shifted by another 8, which makes the transposing read-out below free of bank conflicts.
constexpr int kTileRowDwords = kTile / 4 + 1;
constexpr int kTileDwords = kTile * kTileRowDwords + 8;
__device__ __forceinline__ int tile_dword(int row, int dcol) { return row * kTileRowDwords + ((row >> 6) << 3) + dcol; }

// Writes the transposed tile: q_t[c0 + c, r0 + r] = tile[r, c].  Thread t takes the four columns 4*(t/8).. and the
// sixteen rows 16*(t%8)..: sixteen dword reads, 4x4 byte transposes with v_perm_b32, four 16-byte stores; eight
// consecutive lanes cover 128 contiguous bytes of one transposed row.
__device__ __forceinline__ void store_tile_transposed(const unsigned int *tile, int8_t *__restrict__ q_t, int rows,
                                                      int cols, int r0, int c0) {
    const int rb = threadIdx.x & 7, cg = threadIdx.x >> 3;
    unsigned int piece[4][4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const unsigned int a0 = tile[tile_dword(16 * rb + 4 * g + 0, cg)], a1 = tile[tile_dword(16 * rb + 4 * g + 1, cg)];
        const unsigned int a2 = tile[tile_dword(16 * rb + 4 * g + 2, cg)], a3 = tile[tile_dword(16 * rb + 4 * g + 3, cg)];
        // v_perm_b32: selector bytes 0-3 pick from the second operand, 4-7 from the first.
        const unsigned int lo01 = __builtin_amdgcn_perm(a1, a0, 0x05010400u), hi01 = __builtin_amdgcn_perm(a1, a0, 0x07030602u);
        const unsigned int lo23 = __builtin_amdgcn_perm(a3, a2, 0x05010400u), hi23 = __builtin_amdgcn_perm(a3, a2, 0x07030602u);
        piece[0][g] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
        piece[1][g] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
        piece[2][g] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
        piece[3][g] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
    }
    const int r = r0 + 16 * rb;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = c0 + 4 * cg + k;
        if (c < cols && r < rows)
            *reinterpret_cast<v4u *>(q_t + (int64_t)c * rows + r) = v4u{piece[k][0], piece[k][1], piece[k][2], piece[k][3]};
    }
}

}  // namespace
}  // namespace sb
