// lanes.hpp -- exchanges between the lanes of a wave in vector registers (a lane's partner through DPP and the swaps of
// rows of 16 and of 32 lanes), without the trip through LDS that a shuffle takes; and the 16 bytes a lane moves.
#pragma once

#include "spv_common.hpp"

namespace spv {

// A launch's axis has room for 2^32 threads: workgroups of 256 are laid out in lines of 2^23.  Those past the last find
// nothing to do.  (The length of a line read from the launch instead cost 300,007 x 96 into 8 bits and back 1.7 us of 29.)
constexpr int kGridLine = 23;
inline dim3 grid_of(int64_t groups) {
    const int64_t line = (int64_t)1 << kGridLine;
    return groups <= line ? dim3((unsigned)(groups < 1 ? 1 : groups)) : dim3((unsigned)line, (unsigned)((groups + line - 1) >> kGridLine));
}
__device__ inline int64_t group_of_grid() { return ((int64_t)blockIdx.y << kGridLine) + blockIdx.x; }

template <int CTRL>
__device__ inline int dpp(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true);
}
// f(own, partner's) over groups of N lanes (a power of two), the same result in each lane of a group: lanes 1 and 2
// apart, then, of equal quads and eights, the mirrored one; then rows of 16 and halves of the wave
template <int N, class F>
__device__ inline int lanes_join(int v, F&& f) {
    if constexpr (N >= 2) v = f(v, dpp<0xB1>(v));
    if constexpr (N >= 4) v = f(v, dpp<0x4E>(v));
    if constexpr (N >= 8) v = f(v, dpp<0x141>(v));
    if constexpr (N >= 16) v = f(v, dpp<0x140>(v));
    if constexpr (N >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = f((int)p[0], (int)p[1]);
    }
    if constexpr (N >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = f((int)p[0], (int)p[1]);
    }
    return v;
}
template <int N>
__device__ inline float lanes_sum(float v) {
    return __int_as_float(
        lanes_join<N>(__float_as_int(v), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}
template <int N>
__device__ inline uint32_t lanes_max(uint32_t v) {
    return (uint32_t)lanes_join<N>((int)v, [](int a, int b) { return (int)max((uint32_t)a, (uint32_t)b); });
}
// of the four lanes 16 apart, in 64 bits
__device__ inline double rows_sum(double v) {
    auto pair = [](int lo, int hi) { return __hiloint2double(hi, lo); };
    {
        const auto l = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
        const auto h = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
        v = pair((int)l[0], (int)h[0]) + pair((int)l[1], (int)h[1]);
    }
    const auto l = __builtin_amdgcn_permlane32_swap(__double2loint(v), __double2loint(v), false, false);
    const auto h = __builtin_amdgcn_permlane32_swap(__double2hiint(v), __double2hiint(v), false, false);
    return pair((int)l[0], (int)h[0]) + pair((int)l[1], (int)h[1]);
}
// over groups of 8 lanes or (wide) the whole wave, in 64 bits
__device__ inline double lanes_sum(double v, bool wide) {
    auto pair = [](int lo, int hi) { return __hiloint2double(hi, lo); };
    v += pair(dpp<0xB1>(__double2loint(v)), dpp<0xB1>(__double2hiint(v)));
    v += pair(dpp<0x4E>(__double2loint(v)), dpp<0x4E>(__double2hiint(v)));
    v += pair(dpp<0x141>(__double2loint(v)), dpp<0x141>(__double2hiint(v)));
    if (!wide) return v;
    v += pair(dpp<0x140>(__double2loint(v)), dpp<0x140>(__double2hiint(v)));
    return rows_sum(v);
}

// 16 bytes of channels in float32, and back with one rounding
template <int DT, int V>
__device__ inline void unpack16(const uint4& r, float (&x)[V]) {
    static_assert(V == (DT == SPV_F32 ? 4 : 8), "16 bytes");
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (DT == SPV_F32) {
            x[j] = __uint_as_float(w[j]);
        } else {
            x[2 * j] = from16<DT>(w[j] & 0xFFFF);
            x[2 * j + 1] = from16<DT>(w[j] >> 16);
        }
    }
}
template <int DT, int V>
__device__ inline uint4 pack16(const float (&x)[V]) {
    static_assert(V == (DT == SPV_F32 ? 4 : 8), "16 bytes");
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (DT == SPV_F32) w[j] = __float_as_uint(x[j]);
        else w[j] = pack2<DT>(x[2 * j], x[2 * j + 1]);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace spv
