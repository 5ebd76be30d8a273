// norm.hip -- layer norm over the channels of feature rows and its backward:
//   y = (x - mu) r gamma + beta,  mu = mean x,  r = 1 / sqrt(mean (x - mu)^2 + eps)
//   dx = r (h - mean h - xh mean(h xh)) (+ dres),  h = dy gamma,  xh = (x - mu) r
//   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
// The variance is the mean square of the deviations, taken after the mean: no
// cancellation where a row sits far from zero.
#include "conv_common.hpp"

namespace spv {

constexpr int kNormWaves = 4;
constexpr unsigned kNormGrid = 1024;  // workgroups at most (four per CU): their column sums are joined

__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// mean and 1 / deviation of row x[0 .. C), the whole wave
template <int DT>
__device__ inline void row_stats(const void* x, int64_t base, int C, float eps, int lane, float& mu, float& r) {
    float s = 0.f;
    for (int c = lane; c < C; c += 64) s += ld_feat<DT>(x, base + c);
    mu = wave_sum(s) / (float)C;
    float ss = 0.f;
    for (int c = lane; c < C; c += 64) {
        const float d = ld_feat<DT>(x, base + c) - mu;
        ss = fmaf(d, d, ss);
    }
    r = 1.f / sqrtf(wave_sum(ss) / (float)C + eps);
}

// a wave per row, any width and alignment
template <int DT>
__global__ __launch_bounds__(64 * kNormWaves) void k_norm_any(NormArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m = clamp_rows(a.m_dev, a.m_cap);
    for (int64_t i = (int64_t)blockIdx.x * kNormWaves + wave; i < m; i += (int64_t)gridDim.x * kNormWaves) {
        float mu, r;
        row_stats<DT>(a.x, i * a.C, a.C, a.eps, lane, mu, r);
        for (int c = lane; c < a.C; c += 64) {
            const float xh = (ld_feat<DT>(a.x, i * a.C + c) - mu) * r;
            st_feat<DT>(a.out, i * a.C + c, fmaf(xh, a.gamma ? a.gamma[c] : 1.f, a.beta ? a.beta[c] : 0.f));
        }
    }
}

// dx, and each row's statistics for the column sums
template <int DT>
__global__ __launch_bounds__(64 * kNormWaves) void k_norm_bwd_any(NormBwdArgs a, float* stat) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m = clamp_rows(a.m_dev, a.m_cap);
    for (int64_t i = (int64_t)blockIdx.x * kNormWaves + wave; i < m; i += (int64_t)gridDim.x * kNormWaves) {
        float mu, r;
        row_stats<DT>(a.x, i * a.C, a.C, a.eps, lane, mu, r);
        if (stat && lane == 0) {
            stat[2 * i] = mu;
            stat[2 * i + 1] = r;
        }
        if (!a.dx) continue;
        float s1 = 0.f, s2 = 0.f;
        for (int c = lane; c < a.C; c += 64) {
            const float h = ld_feat<DT>(a.dy, i * a.C + c) * (a.gamma ? a.gamma[c] : 1.f);
            s1 += h;
            s2 = fmaf(h, (ld_feat<DT>(a.x, i * a.C + c) - mu) * r, s2);
        }
        s1 = wave_sum(s1) / (float)a.C;
        s2 = wave_sum(s2) / (float)a.C;
        for (int c = lane; c < a.C; c += 64) {
            const int64_t t = i * a.C + c;
            const float h = ld_feat<DT>(a.dy, t) * (a.gamma ? a.gamma[c] : 1.f);
            const float xh = (ld_feat<DT>(a.x, t) - mu) * r;
            float d = r * (h - s1 - xh * s2);
            if (a.dres) d += ld_feat<DT>(a.dres, t);
            st_feat<DT>(a.dx, t, d);
        }
    }
}

// the column sums of 64 channels over a run of rows: part[blockIdx.x][2][C].  dx may
// be dy itself, so this runs before k_norm_bwd_any overwrites it and forms xh from x.
template <int DT>
__global__ __launch_bounds__(64 * kNormWaves) void k_norm_cols_any(NormBwdArgs a, const float* stat, float* part) {
    __shared__ float red[kNormWaves][2][64];
    const int cl = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.y * 64 + cl;
    const int64_t m = clamp_rows(a.m_dev, a.m_cap);
    float sg = 0.f, sb = 0.f;
    if (c < a.C)
        for (int64_t i = (int64_t)blockIdx.x * kNormWaves + wave; i < m; i += (int64_t)gridDim.x * kNormWaves) {
            const float dy = ld_feat<DT>(a.dy, i * a.C + c);
            sg = fmaf(dy, (ld_feat<DT>(a.x, i * a.C + c) - stat[2 * i]) * stat[2 * i + 1], sg);
            sb += dy;
        }
    red[wave][0][cl] = sg;
    red[wave][1][cl] = sb;
    __syncthreads();
    if (wave == 0 && c < a.C) {
        for (int w = 1; w < kNormWaves; ++w) {
            sg += red[w][0][cl];
            sb += red[w][1][cl];
        }
        part[((int64_t)blockIdx.x * 2) * a.C + c] = sg;
        part[((int64_t)blockIdx.x * 2 + 1) * a.C + c] = sb;
    }
}

// a thread per channel and half adds the workgroups' sums in order
__global__ __launch_bounds__(64) void k_norm_join(const float* __restrict__ part, int nblk, int C,
                                                  float* __restrict__ dgamma, float* __restrict__ dbeta) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    float* out = blockIdx.y ? dbeta : dgamma;
    if (c >= C || !out) return;
    double s = 0.0;
    for (int b = 0; b < nblk; ++b) s += (double)part[((int64_t)b * 2 + blockIdx.y) * C + c];
    out[c] = (float)s;
}

static unsigned norm_grid(int64_t m_cap) {
    const int64_t g = (m_cap + kNormWaves - 1) / kNormWaves;
    return (unsigned)(g < 1 ? 1 : g > kNormGrid ? kNormGrid : g);
}

NormWs plan_norm_ws(Arena& a, int64_t m_cap, int C) {
    NormWs w;
    w.part = a.take<float>((size_t)norm_grid(m_cap) * 2 * (size_t)C);
    w.stat = a.take<float>((size_t)2 * (size_t)m_cap);
    return w;
}

template <int DT>
static void norm_dt(hipStream_t s, const NormArgs& a) {
    k_norm_any<DT><<<norm_grid(a.m_cap), 64 * kNormWaves, 0, s>>>(a);
}
void launch_layer_norm(hipStream_t s, const NormArgs& a) {
    if (a.dt == SPV_F32) norm_dt<SPV_F32>(s, a);
    else if (a.dt == SPV_BF16) norm_dt<SPV_BF16>(s, a);
    else norm_dt<SPV_F16>(s, a);
}

template <int DT>
static void norm_bwd_dt(hipStream_t s, const NormBwdArgs& a, const NormWs& w) {
    const unsigned g = norm_grid(a.m_cap);
    const bool sums = a.dgamma || a.dbeta;
    if (sums) {
        // the statistics alone, then the column sums, then dx (which may overwrite dy)
        NormBwdArgs st = a;
        st.dx = nullptr;
        k_norm_bwd_any<DT><<<g, 64 * kNormWaves, 0, s>>>(st, w.stat);
        k_norm_cols_any<DT><<<dim3(g, (unsigned)((a.C + 63) / 64)), 64 * kNormWaves, 0, s>>>(a, w.stat, w.part);
        k_norm_join<<<dim3((unsigned)((a.C + 63) / 64), 2), 64, 0, s>>>(w.part, (int)g, a.C, a.dgamma, a.dbeta);
    }
    if (a.dx) k_norm_bwd_any<DT><<<g, 64 * kNormWaves, 0, s>>>(a, nullptr);
}
void launch_layer_norm_backward(hipStream_t s, const NormBwdArgs& a, const NormWs& w) {
    if (a.dt == SPV_F32) norm_bwd_dt<SPV_F32>(s, a, w);
    else if (a.dt == SPV_BF16) norm_bwd_dt<SPV_BF16>(s, a, w);
    else norm_bwd_dt<SPV_F16>(s, a, w);
}

}  // namespace spv
