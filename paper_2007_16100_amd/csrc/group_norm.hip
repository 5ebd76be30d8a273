// group_norm.hip -- group norm of packed scans with an activation, and its backward:
//   xh = (x - mu) r,  z = xh gamma + beta,  y = act(z),
//   mu, r from the rows of a scan and the channels of a group together;
//   gz = dy act'(z),  h = gz gamma,  dx = r (h - mean h - xh mean(h xh)) (+ dres),
//   dgamma = sum gz xh,  dbeta = sum gz.
#include <type_traits>

#include "attn_common.hpp"
#include "code8.hpp"

namespace spv {

template <int ACT>
__device__ inline float act_of(float z) {
    if constexpr (ACT == SPV_ACT_RELU) return z <= 0.f ? 0.f : z;
    else if constexpr (ACT == SPV_ACT_SILU) return z / (1.f + expf(-z));
    else return z;
}
template <int ACT>
__device__ inline float act_slope(float z) {
    if constexpr (ACT == SPV_ACT_RELU) {
        return z <= 0.f ? 0.f : 1.f;
    } else if constexpr (ACT == SPV_ACT_SILU) {
        const float s = 1.f / (1.f + expf(-z));
        return s * fmaf(z, 1.f - s, 1.f);
    } else {
        return 1.f;
    }
}

__device__ inline double block_sum(double v, double* red) {
    __syncthreads();
    red[threadIdx.x] = v;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
        if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
        __syncthreads();
    }
    return red[0];
}

// what a backward reads of x
template <int DT>
__device__ inline float saved_x(const GnArgs& a, int64_t i, int c) {
    if (a.x) return ld_feat<DT>(a.x, i * a.C + c);
    return code_value(a.saved.codes[i * a.C + c], code_step(a.saved.exps[i * code_blocks(a.C) + c / kCodeBlock]));
}

// a workgroup takes a group of a scan
template <int DT>
__global__ __launch_bounds__(256) void k_gn_stat(GnArgs a) {
    __shared__ double red[256];
    const int b = blockIdx.x / a.G, g = blockIdx.x % a.G, w = a.C / a.G;
    const int64_t r0 = clamp_off(a.off[b], a.m), r1 = clamp_off(a.off[b + 1], a.m);
    const int64_t n = r1 > r0 ? (r1 - r0) * w : 0;
    double s = 0.0;
    for (int64_t t = threadIdx.x; t < n; t += 256) s += (double)ld_feat<DT>(a.x, (r0 + t / w) * a.C + g * w + t % w);
    const double mu = n ? block_sum(s, red) / (double)n : 0.0;
    s = 0.0;
    for (int64_t t = threadIdx.x; t < n; t += 256) {
        const double d = (double)ld_feat<DT>(a.x, (r0 + t / w) * a.C + g * w + t % w) - mu;
        s += d * d;
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) {
        a.part[2 * blockIdx.x] = (float)mu;
        a.part[2 * blockIdx.x + 1] = n ? (float)(1.0 / sqrt(s / (double)n + (double)a.eps)) : 0.f;
        if (a.stat) {
            a.stat[2 * blockIdx.x] = a.part[2 * blockIdx.x];
            a.stat[2 * blockIdx.x + 1] = a.part[2 * blockIdx.x + 1];
        }
    }
}

// the scan of row i, or -1
__device__ inline int scan_of(const GnArgs& a, int64_t i) {
    int lo = 0, hi = a.B;  // off[lo] <= i < off[hi] where there is such
    if (i < clamp_off(a.off[0], a.m) || i >= clamp_off(a.off[a.B], a.m)) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((int64_t)a.off[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <int DT, int ACT>
__global__ __launch_bounds__(256) void k_gn_apply(GnArgs a) {
    for (int64_t i = blockIdx.x; i < a.m; i += gridDim.x) {
        const int b = scan_of(a, i);
        if (b < 0) continue;
        for (int c = threadIdx.x; c < a.C; c += 256) {
            const float* st = a.part + 2 * ((int64_t)b * a.G + c / (a.C / a.G));
            const float xh = (ld_feat<DT>(a.x, i * a.C + c) - st[0]) * st[1];
            st_feat<DT>(a.out, i * a.C + c,
                        act_of<ACT>(fmaf(xh, a.gamma ? a.gamma[c] : 1.f, a.beta ? a.beta[c] : 0.f)));
        }
    }
}

// a workgroup takes a channel of a scan: sum gz and sum gz xh
template <int DT, int ACT>
__global__ __launch_bounds__(256) void k_gn_sums(GnArgs a) {
    __shared__ double red[256];
    const int b = blockIdx.x / a.C, c = blockIdx.x % a.C;
    const int64_t r0 = clamp_off(a.off[b], a.m), r1 = clamp_off(a.off[b + 1], a.m);
    const float* st = a.stat + 2 * ((int64_t)b * a.G + c / (a.C / a.G));
    const float g = a.gamma ? a.gamma[c] : 1.f, be = a.beta ? a.beta[c] : 0.f;
    double s1 = 0.0, s2 = 0.0;
    for (int64_t i = r0 + threadIdx.x; i < r1; i += 256) {
        const float xh = (saved_x<DT>(a, i, c) - st[0]) * st[1];
        const float gz = ld_feat<DT>(a.dy, i * a.C + c) * act_slope<ACT>(fmaf(xh, g, be));
        s1 += (double)gz;
        s2 += (double)gz * xh;
    }
    s1 = block_sum(s1, red);
    s2 = block_sum(s2, red);
    if (threadIdx.x == 0) {
        a.part[2 * (int64_t)blockIdx.x] = (float)s1;
        a.part[2 * (int64_t)blockIdx.x + 1] = (float)s2;
    }
}

template <int DT, int ACT>
__global__ __launch_bounds__(256) void k_gn_dx(GnArgs a) {
    const int w = a.C / a.G;
    for (int64_t i = blockIdx.x; i < a.m; i += gridDim.x) {
        const int b = scan_of(a, i);
        if (b < 0) continue;
        const float n = (float)(clamp_off(a.off[b + 1], a.m) - clamp_off(a.off[b], a.m)) * (float)w;
        for (int c = threadIdx.x; c < a.C; c += 256) {
            const int g0 = c / w * w;
            float m1 = 0.f, m2 = 0.f;
            for (int j = g0; j < g0 + w; ++j) {
                const float gj = a.gamma ? a.gamma[j] : 1.f;
                m1 = fmaf(gj, a.part[2 * ((int64_t)b * a.C + j)], m1);
                m2 = fmaf(gj, a.part[2 * ((int64_t)b * a.C + j) + 1], m2);
            }
            const float* st = a.stat + 2 * ((int64_t)b * a.G + c / w);
            const float g = a.gamma ? a.gamma[c] : 1.f, xh = (saved_x<DT>(a, i, c) - st[0]) * st[1];
            const float h = ld_feat<DT>(a.dy, i * a.C + c) * act_slope<ACT>(fmaf(xh, g, a.beta ? a.beta[c] : 0.f)) * g;
            float d = st[1] * (h - m1 / n - xh * (m2 / n));
            if (a.dres) d += ld_feat<DT>(a.dres, i * a.C + c);
            st_feat<DT>(a.dx, i * a.C + c, d);
        }
    }
}

__global__ __launch_bounds__(256) void k_gn_params(GnArgs a) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.C) return;
    double s1 = 0.0, s2 = 0.0;
    for (int b = 0; b < a.B; ++b) {
        s1 += (double)a.part[2 * ((int64_t)b * a.C + c)];
        s2 += (double)a.part[2 * ((int64_t)b * a.C + c) + 1];
    }
    if (a.dbeta) a.dbeta[c] = (float)s1;
    if (a.dgamma) a.dgamma[c] = (float)s2;
}

void plan_group_norm_ws(Arena& a, GnArgs& t) { t.part = a.take<float>((size_t)2 * t.B * t.G); }
void plan_group_norm_backward_ws(Arena& a, GnArgs& t) { t.part = a.take<float>((size_t)2 * t.B * t.C); }

// f(type, activation) for those of a
template <class F>
static void gn_kinds(const GnArgs& a, F&& f) {
    auto act = [&](auto dt) {
        if (a.act == SPV_ACT_RELU) f(dt, std::integral_constant<int, SPV_ACT_RELU>{});
        else if (a.act == SPV_ACT_SILU) f(dt, std::integral_constant<int, SPV_ACT_SILU>{});
        else f(dt, std::integral_constant<int, SPV_ACT_NONE>{});
    };
    if (a.dt == SPV_F32) act(std::integral_constant<int, SPV_F32>{});
    else if (a.dt == SPV_BF16) act(std::integral_constant<int, SPV_BF16>{});
    else act(std::integral_constant<int, SPV_F16>{});
}

void launch_group_norm(hipStream_t s, const GnArgs& a) {
    const unsigned rows = (unsigned)(a.m < 1 ? 1 : a.m > 65536 ? 65536 : a.m);
    // before out, which may be x
    if (a.saved.codes && a.m) launch_checkpoint8(s, a.x, a.saved, RowRange{a.m, nullptr, a.off, a.B}, a.C, a.dt);
    gn_kinds(a, [&](auto dt, auto act) {
        k_gn_stat<decltype(dt)::value><<<(unsigned)(a.B * a.G), 256, 0, s>>>(a);
        if (a.m) k_gn_apply<decltype(dt)::value, decltype(act)::value><<<rows, 256, 0, s>>>(a);
    });
}
void launch_group_norm_backward(hipStream_t s, const GnArgs& a) {
    const unsigned rows = (unsigned)(a.m < 1 ? 1 : a.m > 65536 ? 65536 : a.m);
    gn_kinds(a, [&](auto dt, auto act) {
        if (a.B) k_gn_sums<decltype(dt)::value, decltype(act)::value><<<(unsigned)(a.B * a.C), 256, 0, s>>>(a);
        if (a.dgamma || a.dbeta) k_gn_params<<<(unsigned)((a.C + 255) / 256), 256, 0, s>>>(a);
        if (a.dx && a.m && a.B) k_gn_dx<decltype(dt)::value, decltype(act)::value><<<rows, 256, 0, s>>>(a);
    });
}

}  // namespace spv
