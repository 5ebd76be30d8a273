// code8.hpp -- rows in 8 bits: an exponent for each 32 channels of a row, codes of -127 .. 127 in steps of 2^E.
#pragma once

#include "conv_common.hpp"
#include "lanes.hpp"

namespace spv {

constexpr int kCodeBlock = SPV_CHECKPOINT8_BLOCK;
__host__ __device__ inline int code_blocks(int C) { return (C + kCodeBlock - 1) / kCodeBlock; }

// |x| where x is finite, else 0, as bits (which order as the values do)
__device__ inline uint32_t finite_bits(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}
// the exponent byte of a block whose largest finite |x| has these bits: a subnormal maximum counts as 2^-127
template <int DT>
__device__ inline int code_exp(uint32_t top) {
    const int e = (int)(top >> 23) - 6, lowest = DT == SPV_F16 ? 127 - 24 : 1;
    return e < lowest ? lowest : e;
}
// 2^(byte - 127) and its inverse, for bytes 1 .. 248
__device__ inline float code_step(int byte) { return __uint_as_float((uint32_t)byte << 23); }
__device__ inline float code_rate(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }
// the code of x: products by a power of two are exact
__device__ inline int code_of(float x, float rate) {
    const float q = fminf(fmaxf(rintf(x * rate), -127.f), 127.f);
    return finite_bits(x) == 0u && x != 0.f ? -128 : (int)q;
}
__device__ inline float code_value(int code, float step) {
    return code == -128 ? __uint_as_float(0x7FC00000u) : (float)code * step;
}

// What 4 N codes stand for: a byte counted from -128 takes a conversion and two exact steps.  A code of -128 (a zero
// byte then) is looked for in all of them at once.
template <int N>
__device__ inline void code_values(const uint32_t (&w)[N], float step, float (&x)[4 * N]) {
    uint32_t u[N], none = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        u[j] = w[j] ^ 0x80808080u;
        none |= (u[j] - 0x01010101u) & ~u[j] & 0x80808080u;  // not 0 where there is a zero byte
        x[4 * j] = ((float)(u[j] & 0xFFu) - 128.f) * step;
        x[4 * j + 1] = ((float)((u[j] >> 8) & 0xFFu) - 128.f) * step;
        x[4 * j + 2] = ((float)((u[j] >> 16) & 0xFFu) - 128.f) * step;
        x[4 * j + 3] = ((float)(u[j] >> 24) - 128.f) * step;
    }
    if (none) {
#pragma unroll
        for (int e = 0; e < 4 * N; ++e)
            if (((u[e / 4] >> (8 * (e % 4))) & 0xFFu) == 0u) x[e] = __uint_as_float(0x7FC00000u);
    }
}

// The codes of a lane's VEC channels of a block that LANES lanes hold (a power of two of them, next to each other);
// returns the block's exponent byte.  All lanes of a block call it.  Where all values are finite a code is the low
// byte of x 2^-E plus 1.5 2^23, whose addition rounds to a whole number, ties to even.
template <int DT, int VEC, int LANES>
__device__ inline int code_block(const float (&x)[VEC], uint32_t (&w)[VEC / 4]) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    top = lanes_max<LANES>(top);
    if (top < 0x7F800000u) {
        const int byte = code_exp<DT>(top);
        const float rate = code_rate(byte);
#pragma unroll
        for (int j = 0; j < VEC / 4; ++j) {
            uint32_t q[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                q[e] = __float_as_uint(__builtin_amdgcn_fmed3f(x[4 * j + e] * rate, -127.f, 127.f) + 12582912.f);
            w[j] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0C0C0400u),
                                         __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u), 0x05040100u);
        }
        return byte;
    }
    top = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) top = max(top, finite_bits(x[e]));
    const int byte = code_exp<DT>(lanes_max<LANES>(top));
    const float rate = code_rate(byte);
#pragma unroll
    for (int j = 0; j < VEC / 4; ++j) {
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = (uint32_t)code_of(x[4 * j + e], rate) & 0xFFu;
        w[j] = (q[0] | (q[1] << 8)) | ((q[2] << 16) | (q[3] << 24));
    }
    return byte;
}

}  // namespace spv
