// rope.hip -- rotary positions over three axes: pair p of a head's channels turns by
//   theta = c_a freqs[p],  (u, w) -> (u cos theta - w sin theta, u sin theta + w cos theta),
// c_a the row's coordinate on the axis whose section holds p.  The inverse turns by -theta.
#include "conv_common.hpp"

namespace spv {

// (cos, sin) of c f.  The product of 16 bits and 24 is exact in float64; a turn is taken off there, which leaves an
// eighth of one at most, whose sine and cosine are their Taylor sums: the terms left out are below 2^-28.
__device__ inline float2 cos_sin(int c, float f) {
    double t = (double)c * (double)f * 0.15915494309189535;  // turns
    t -= rint(t);
    const double q = rint(4.0 * t);
    const float r = (float)((t - 0.25 * q) * 6.283185307179586), z = r * r;
    const float s = fmaf(fmaf(fmaf(fmaf(2.7557319e-6f, z, -1.9841270e-4f), z, 8.3333333e-3f), z, -0.16666667f) * z, r, r);
    const float k = fmaf(fmaf(fmaf(fmaf(-2.7557319e-7f, z, 2.4801587e-5f), z, -1.3888889e-3f), z, 4.1666667e-2f), z * z,
                         fmaf(z, -0.5f, 1.f));
    const int n = (int)q & 3;
    const float a = n & 1 ? s : k, b = n & 1 ? k : s;
    return make_float2(n == 1 || n == 2 ? -a : a, n & 2 ? -b : b);
}

__device__ inline int voxel_axis(const int32_t* c) {
    const int v = *c;
    return v < kCoordMin ? kCoordMin : (v > kCoordMax ? kCoordMax : v);
}

// a thread takes one pair of one head of one row, or two of the channels that stay
template <int DT>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a) {
    const int half = a.D / 2, heads = a.q.heads + a.k.heads;
    const int64_t m = clamp_rows(a.m_dev, a.n), all = m * heads * half;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < all; t += (int64_t)gridDim.x * 256) {
        const int p = (int)(t % half), hh = (int)(t / half % heads);
        const int64_t i = t / half / heads;
        const bool of_q = hh < a.q.heads;
        const RopeSide& s = of_q ? a.q : a.k;
        const int h = of_q ? hh : hh - a.q.heads;
        const bool turned = p < a.P;
        const int c0 = !turned || !a.halves ? 2 * p : p, c1 = !turned || !a.halves ? 2 * p + 1 : p + a.P;
        const int64_t src = i * s.ld + (int64_t)h * a.D, dst = i * s.ldo + (int64_t)h * a.D;
        float u = ld_feat<DT>(s.in, src + c0), w = ld_feat<DT>(s.in, src + c1);
        if (turned) {
            const int axis = p < a.sx ? 1 : p < a.sx + a.sy ? 2 : 3;
            float2 cs = cos_sin(voxel_axis(a.coords + 4 * i + axis), a.freqs[p]);
            if (a.inverse) cs.y = -cs.y;
            const float v = u * cs.x - w * cs.y;
            w = u * cs.y + w * cs.x;
            u = v;
        }
        st_feat<DT>(s.out, dst + c0, u);
        st_feat<DT>(s.out, dst + c1, w);
    }
}

void launch_rope(hipStream_t s, const RopeArgs& a) {
    const int64_t threads = a.n * (a.q.heads + a.k.heads) * (a.D / 2);
    const unsigned g = (unsigned)(threads / 256 + 1 < 65536 ? threads / 256 + 1 : 65536);
    if (a.dt == SPV_F32) k_rope<SPV_F32><<<g, 256, 0, s>>>(a);
    else if (a.dt == SPV_BF16) k_rope<SPV_BF16><<<g, 256, 0, s>>>(a);
    else k_rope<SPV_F16><<<g, 256, 0, s>>>(a);
}

}  // namespace spv
