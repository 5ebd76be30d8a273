// norm.hip -- layer norm over the channels of feature rows and its backward:
//   y = (x - mu) r gamma + beta,  mu = mean x,  r = 1 / sqrt(mean (x - mu)^2 + eps)
//   dx = r (h - mean h - xh mean(h xh)) (+ dres),  h = dy gamma,  xh = (x - mu) r
//   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
// The variance is the mean square of the deviations, taken after the mean: no
// cancellation where a row sits far from zero.
#include <type_traits>

#include "conv_common.hpp"

namespace spv {

constexpr int kNormWaves = 4;
constexpr unsigned kNormGrid = 2048;    // workgroups of the forward at most
// of the backward: two per CU, whose column sums are joined.  Forward and backward of 300,007 x 96 in bf16 with the
// residual's gradient take 65 us with 512, 77 with 768, 73 with 1024.
constexpr unsigned kNormBwdGrid = 512;

// sum over the L lanes of a row
template <int L>
__device__ inline float row_sum(float v) {
#pragma unroll
    for (int o = 1; o < L; o <<= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// mean and 1 / deviation of row x[0 .. C) (on: there is one), from the L lanes that hold it
template <int DT, int L>
__device__ inline void row_stats(const void* x, int64_t base, int C, float eps, int l, bool on, float& mu, float& r) {
    float s = 0.f;
    for (int c = l; on && c < C; c += L) s += ld_feat<DT>(x, base + c);
    mu = row_sum<L>(s) / (float)C;
    float ss = 0.f;
    for (int c = l; on && c < C; c += L) {
        const float d = ld_feat<DT>(x, base + c) - mu;
        ss = fmaf(d, d, ss);
    }
    r = 1.f / sqrtf(row_sum<L>(ss) / (float)C + eps);
}

// any width and alignment: L lanes a row, 64 / L rows a wave, which leave the loop together
template <int DT, int L>
__global__ __launch_bounds__(64 * kNormWaves) void k_norm_any(NormArgs a) {
    constexpr int R = 64 / L;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & (L - 1);
    const int64_t m = clamp_rows(a.m_dev, a.m_cap), step = (int64_t)gridDim.x * kNormWaves * R;
    for (int64_t i0 = ((int64_t)blockIdx.x * kNormWaves + wave) * R; i0 < m; i0 += step) {
        const int64_t i = i0 + lane / L;
        const bool on = i < m;
        float mu, r;
        row_stats<DT, L>(a.x, i * a.C, a.C, a.eps, l, on, mu, r);
        for (int c = l; on && c < a.C; c += L) {
            const float xh = (ld_feat<DT>(a.x, i * a.C + c) - mu) * r;
            st_feat<DT>(a.out, i * a.C + c, fmaf(xh, a.gamma ? a.gamma[c] : 1.f, a.beta ? a.beta[c] : 0.f));
        }
    }
}

// dx, and each row's statistics for the column sums
template <int DT, int L>
__global__ __launch_bounds__(64 * kNormWaves) void k_norm_bwd_any(NormBwdArgs a, float* stat) {
    constexpr int R = 64 / L;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & (L - 1);
    const int64_t m = clamp_rows(a.m_dev, a.m_cap), step = (int64_t)gridDim.x * kNormWaves * R;
    for (int64_t i0 = ((int64_t)blockIdx.x * kNormWaves + wave) * R; i0 < m; i0 += step) {
        const int64_t i = i0 + lane / L;
        const bool on = i < m;
        float mu, r;
        row_stats<DT, L>(a.x, i * a.C, a.C, a.eps, l, on, mu, r);
        if (stat && on && l == 0) {
            stat[2 * i] = mu;
            stat[2 * i + 1] = r;
        }
        if (!a.dx) continue;
        float s1 = 0.f, s2 = 0.f;
        for (int c = l; on && c < a.C; c += L) {
            const float h = ld_feat<DT>(a.dy, i * a.C + c) * (a.gamma ? a.gamma[c] : 1.f);
            s1 += h;
            s2 = fmaf(h, (ld_feat<DT>(a.x, i * a.C + c) - mu) * r, s2);
        }
        s1 = row_sum<L>(s1) / (float)a.C;
        s2 = row_sum<L>(s2) / (float)a.C;
        for (int c = l; on && c < a.C; c += L) {
            const int64_t t = i * a.C + c;
            const float h = ld_feat<DT>(a.dy, t) * (a.gamma ? a.gamma[c] : 1.f);
            const float xh = (ld_feat<DT>(a.x, t) - mu) * r;
            float d = r * (h - s1 - xh * s2);
            if (a.dres) d += ld_feat<DT>(a.dres, t);
            st_feat<DT>(a.dx, t, d);
        }
    }
}

// the column sums of 64 channels over a run of rows: part[blockIdx.x][2][C].  It reads
// dy, so it runs before k_norm_bwd_any writes dx, which may be dy.
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

// ---------------------------------------------------------------------------
// 16 bytes at a time: L lanes hold a row, NV vectors of VEC channels each (vector v of lane l is number
// v * L + l of the row), 64 / L rows a wave.  A row is read once: the mean, the deviations and, in the
// backward, both of its means are formed in registers.  What bounds it is memory, so each wave's next rows
// are loaded before the present ones are reduced, and gamma, beta and the column sums stay in registers
// over a workgroup's rows.  Three vectors a lane hold rows of 96, 192, 384 .. without idle lanes.
// 300,007 x 96 in bf16: 23.8 us, 4.8 TB/s (a copy of 1 GiB reaches 5.1).  Forward and backward of 88,119 x 96
// in bf16 with the residual's gradient: 29 us, of which the join of the column sums 4; of 26,881 x 256 in
// f16: 25 us.  701 x 96 in float32: 3.4 us on the GPU, 7.4 a call.
// ---------------------------------------------------------------------------
template <int DT>
constexpr int kVec = DT == SPV_F32 ? 4 : 8;

template <int DT>
__device__ inline void unpack(const uint4& u, float (&x)[kVec<DT>]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
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
template <int DT>
__device__ inline uint4 pack(const float (&x)[kVec<DT>]) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (DT == SPV_F32) w[j] = __float_as_uint(x[j]);
        else w[j] = pack2<DT>(x[2 * j], x[2 * j + 1]);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int DT, int L, int NV>
struct Rows {
    static constexpr int V = kVec<DT>;
    int l, nvec, C;
    float inv;  // 1 / C
    bool live[NV];
    __device__ Rows(int lane, int C) : l(lane & (L - 1)), nvec(C / V), C(C), inv(1.f / (float)C) {
#pragma unroll
        for (int v = 0; v < NV; ++v) live[v] = v * L + l < nvec;
    }
    __device__ int chan(int v) const { return (v * L + l) * V; }
    __device__ void load(const void* p, int64_t row, bool on, uint4 (&u)[NV]) const {
#pragma unroll
        for (int v = 0; v < NV; ++v)
            u[v] = on && live[v] ? *(const uint4*)((const char*)p + (row * C + chan(v)) * (16 / V))
                                 : make_uint4(0, 0, 0, 0);
    }
    __device__ void channels(const float* p, float other, float (&g)[NV][V]) const {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int e = 0; e < V; ++e) g[v][e] = other;
            if (p && live[v]) __builtin_memcpy(g[v], p + chan(v), sizeof(g[v]));
        }
    }
    // x -> (x - mean) / deviation in place (0 in idle vectors); returns 1 / deviation
    __device__ float normalize(float (&x)[NV][V], float eps) const {
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < V; ++e) s += x[v][e];
        const float mu = row_sum<L>(s) / (float)C;  // exact where the sum is
        float ss = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[v][e] = live[v] ? x[v][e] - mu : 0.f;
                ss = fmaf(x[v][e], x[v][e], ss);
            }
        const float r = 1.f / sqrtf(row_sum<L>(ss) * inv + eps);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < V; ++e) x[v][e] *= r;
        return r;
    }
};

template <int DT, int L, int NV>
__global__ __launch_bounds__(64 * kNormWaves) void k_norm(NormArgs a) {
    constexpr int V = kVec<DT>, R = 64 / L;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Rows<DT, L, NV> t(lane, a.C);
    const int64_t m = clamp_rows(a.m_dev, a.m_cap), step = (int64_t)gridDim.x * kNormWaves * R;
    int64_t i = ((int64_t)blockIdx.x * kNormWaves + wave) * R + lane / L;
    uint4 u[NV], nu[NV];
    t.load(a.x, i, i < m, u);
    float g[NV][V], b[NV][V];
    t.channels(a.gamma, 1.f, g);
    t.channels(a.beta, 0.f, b);
    // the row groups of a wave leave the loop together: the row sums take the whole wave
    for (int64_t i0 = i - lane / L; i0 < m; i0 += step, i += step) {
        t.load(a.x, i + step, i + step < m, nu);
        float x[NV][V];
#pragma unroll
        for (int v = 0; v < NV; ++v) unpack<DT>(u[v], x[v]);
        t.normalize(x, a.eps);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int e = 0; e < V; ++e) x[v][e] = fmaf(x[v][e], g[v][e], b[v][e]);
            if (i < m && t.live[v]) *(uint4*)((char*)a.out + (i * a.C + t.chan(v)) * (16 / V)) = pack<DT>(x[v]);
            u[v] = nu[v];
        }
    }
}

// dx, and (part given) the workgroup's column sums: each lane's over its rows in float32, then the lanes of a channel in
// a fixed order.  A single workgroup's are the result.
template <int DT, int L, int NV>
__global__ __launch_bounds__(64 * kNormWaves) void k_norm_bwd(NormBwdArgs a, float* part) {
    constexpr int V = kVec<DT>, R = 64 / L;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Rows<DT, L, NV> t(lane, a.C);
    float g[NV][V], sg[NV][V], sb[NV][V];
    t.channels(a.gamma, 1.f, g);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < V; ++e) sg[v][e] = sb[v][e] = 0.f;
    const int64_t m = clamp_rows(a.m_dev, a.m_cap), step = (int64_t)gridDim.x * kNormWaves * R;
    int64_t i = ((int64_t)blockIdx.x * kNormWaves + wave) * R + lane / L;
    uint4 ux[NV], ud[NV], ur[NV];
    t.load(a.x, i, i < m, ux);
    t.load(a.dy, i, i < m, ud);
    for (int64_t i0 = i - lane / L; i0 < m; i0 += step, i += step) {
        float x[NV][V], h[NV][V];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            unpack<DT>(ux[v], x[v]);
            unpack<DT>(ud[v], h[v]);
        }
        if (a.dres) t.load(a.dres, i, i < m, ur);
        t.load(a.x, i + step, i + step < m, ux);
        t.load(a.dy, i + step, i + step < m, ud);
        const float r = t.normalize(x, a.eps);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sg[v][e] = fmaf(h[v][e], x[v][e], sg[v][e]);  // a row past the end adds 0 * 0
                sb[v][e] += h[v][e];
                h[v][e] *= g[v][e];
                s1 += h[v][e];
                s2 = fmaf(h[v][e], x[v][e], s2);
            }
        if (!a.dx) continue;
        s1 = row_sum<L>(s1) * t.inv;
        s2 = row_sum<L>(s2) * t.inv;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float q[V] = {};
            if (a.dres) unpack<DT>(ur[v], q);
#pragma unroll
            for (int e = 0; e < V; ++e) h[v][e] = fmaf(r, h[v][e] - s1 - x[v][e] * s2, q[e]);
            if (i < m && t.live[v]) *(uint4*)((char*)a.dx + (i * a.C + t.chan(v)) * (16 / V)) = pack<DT>(h[v]);
        }
    }
    if (!part) return;  // the whole workgroup
    __shared__ float red[kNormWaves][2][L * NV * V];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < V; ++e) {
#pragma unroll
            for (int o = L; o < 64; o <<= 1) {
                sg[v][e] += __shfl_xor(sg[v][e], o, 64);
                sb[v][e] += __shfl_xor(sb[v][e], o, 64);
            }
            if (lane < L) {
                red[wave][0][t.chan(v) + e] = sg[v][e];
                red[wave][1][t.chan(v) + e] = sb[v][e];
            }
        }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.C; c += 64 * kNormWaves) {
        const int half = c >= a.C, cc = half ? c - a.C : c;
        float s = red[0][half][cc];
        for (int w = 1; w < kNormWaves; ++w) s += red[w][half][cc];
        if (gridDim.x > 1) part[(int64_t)blockIdx.x * 2 * a.C + c] = s;
        else if (half ? a.dbeta : a.dgamma) (half ? a.dbeta : a.dgamma)[cc] = s;
    }
}

// adds the workgroups' column sums in 64 bits in a fixed order: 16 columns of part [nblk][cols] a workgroup,
// each in 64 runs of consecutive workgroups, eight of a run's loads in flight
__global__ __launch_bounds__(1024) void k_norm_join(const float* __restrict__ part, int nblk, int C,
                                                    float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ double red[64][17];
    const int col = threadIdx.x & 15, run = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    const int len = (nblk + 63) / 64, b0 = run * len, b1 = b0 + len < nblk ? b0 + len : nblk;
    double s = 0.0;
    if (c < 2 * C)
        for (int b = b0; b < b1; b += 8) {
            float f[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) f[q] = b + q < b1 ? part[(int64_t)(b + q) * 2 * C + c] : 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) s += (double)f[q];
        }
    red[run][col] = s;
    __syncthreads();
    // eight runs of eight, then one of those
    if (run < 8) {
        s = red[run * 8][col];
        for (int q = 1; q < 8; ++q) s += red[run * 8 + q][col];
        red[run * 8][col] = s;
    }
    __syncthreads();
    if (run || c >= 2 * C) return;
    for (int q = 1; q < 8; ++q) s += red[q * 8][col];
    if (c < C) {
        if (dgamma) dgamma[c] = (float)s;
    } else if (dbeta) {
        dbeta[c - C] = (float)s;
    }
}

// workgroups, each with rows_wg rows at a time
static unsigned norm_grid(int64_t m_cap, int rows_wg, unsigned most) {
    const int64_t tiles = (m_cap + rows_wg - 1) / rows_wg;
    if (tiles <= (int64_t)most) return (unsigned)(tiles < 1 ? 1 : tiles);
    const int64_t rounds = (tiles + most - 1) / most;  // as many rounds with the fewest workgroups: none runs one more
    return (unsigned)((tiles + rounds - 1) / rounds);
}

NormWs plan_norm_ws(Arena& a, int64_t m_cap, int C) {
    NormWs w;
    const int64_t wgs = (m_cap + kNormWaves - 1) / kNormWaves;  // no kernel takes fewer rows a workgroup
    w.part = a.take<float>((size_t)(wgs < 1 ? 1 : wgs > kNormBwdGrid ? kNormBwdGrid : wgs) * 2 * (size_t)C);
    w.stat = a.take<float>((size_t)2 * (size_t)m_cap);
    return w;
}

// Calls f(L, NV) for the first shape of the list that holds the row's C / VEC vectors (the fewest idle ones), or
// returns false where the vector kernel has none: unaligned rows, odd widths, over 256 vectors.
template <int L, int NV>
struct NormShape {
    static constexpr int lanes = L, vectors = NV;
};
template <class F>
static bool norm_pick(int, F&&) {
    return false;
}
template <class S, class... More, class F>
static bool norm_pick(int n, F&& f) {
    if (n > S::lanes * S::vectors) return norm_pick<More...>(n, f);
    f(std::integral_constant<int, S::lanes>{}, std::integral_constant<int, S::vectors>{});
    return true;
}
template <int DT, class F>
static bool norm_shape(int C, bool aligned, F&& f) {
    if (!aligned || C % kVec<DT>) return false;
    return norm_pick<NormShape<1, 1>, NormShape<2, 1>, NormShape<1, 3>, NormShape<4, 1>, NormShape<2, 3>,
                     NormShape<8, 1>, NormShape<4, 3>, NormShape<16, 1>, NormShape<8, 3>, NormShape<32, 1>,
                     NormShape<16, 3>, NormShape<64, 1>, NormShape<32, 3>, NormShape<64, 2>, NormShape<64, 3>,
                     NormShape<64, 4>>(C / kVec<DT>, f);
}
static bool norm_aligned(const void* p, const void* q, const void* r = nullptr, const void* t = nullptr) {
    return (((uintptr_t)p | (uintptr_t)q | (uintptr_t)r | (uintptr_t)t) & 15u) == 0;
}

// Channels up to which the plain kernels give a row 8 lanes, not 64.  Forward and backward of 88,119 x 19 in float32 take
// 42 us with 8, 145 with 64; of 20,011 x 131 54 and 74; of 5003 x 511 in f16 86 and 50.
constexpr int kNarrow = 256;

template <int DT>
static void norm_dt(hipStream_t s, const NormArgs& a) {
    const bool vec = norm_shape<DT>(a.C, norm_aligned(a.x, a.out), [&](auto l, auto nv) {
        constexpr int L = decltype(l)::value, NV = decltype(nv)::value;
        k_norm<DT, L, NV><<<norm_grid(a.m_cap, kNormWaves * (64 / L), kNormGrid), 64 * kNormWaves, 0, s>>>(a);
    });
    if (vec) return;
    if (a.C <= kNarrow) k_norm_any<DT, 8><<<norm_grid(a.m_cap, kNormWaves * 8, kNormGrid), 64 * kNormWaves, 0, s>>>(a);
    else k_norm_any<DT, 64><<<norm_grid(a.m_cap, kNormWaves, kNormGrid), 64 * kNormWaves, 0, s>>>(a);
}
void launch_layer_norm(hipStream_t s, const NormArgs& a) {
    if (a.dt == SPV_F32) norm_dt<SPV_F32>(s, a);
    else if (a.dt == SPV_BF16) norm_dt<SPV_BF16>(s, a);
    else norm_dt<SPV_F16>(s, a);
}

template <int DT>
static void norm_bwd_dt(hipStream_t s, const NormBwdArgs& a, const NormWs& w) {
    const bool sums = a.dgamma || a.dbeta;
    unsigned g = 0;
    const bool vec = norm_shape<DT>(a.C, norm_aligned(a.x, a.dy, a.dres, a.dx), [&](auto l, auto nv) {
        constexpr int L = decltype(l)::value, NV = decltype(nv)::value;
        g = norm_grid(a.m_cap, kNormWaves * (64 / L), kNormBwdGrid);
        k_norm_bwd<DT, L, NV><<<g, 64 * kNormWaves, 0, s>>>(a, sums ? w.part : nullptr);
    });
    if (!vec) {
        const bool narrow = a.C <= kNarrow;
        const unsigned g8 = norm_grid(a.m_cap, kNormWaves * 8, kNormGrid);
        g = norm_grid(a.m_cap, kNormWaves, kNormBwdGrid);
        if (sums) {
            // the statistics alone, then the column sums, then dx (which may overwrite dy)
            NormBwdArgs st = a;
            st.dx = nullptr;
            if (narrow) k_norm_bwd_any<DT, 8><<<g8, 64 * kNormWaves, 0, s>>>(st, w.stat);
            else k_norm_bwd_any<DT, 64><<<g, 64 * kNormWaves, 0, s>>>(st, w.stat);
            k_norm_cols_any<DT><<<dim3(g, (unsigned)((a.C + 63) / 64)), 64 * kNormWaves, 0, s>>>(a, w.stat, w.part);
        }
        if (a.dx && narrow) k_norm_bwd_any<DT, 8><<<g8, 64 * kNormWaves, 0, s>>>(a, nullptr);
        else if (a.dx) k_norm_bwd_any<DT, 64><<<g, 64 * kNormWaves, 0, s>>>(a, nullptr);
    }
    if (sums && !(vec && g == 1))
        k_norm_join<<<(unsigned)((2 * a.C + 15) / 16), 1024, 0, s>>>(w.part, (int)g, a.C, a.dgamma, a.dbeta);
}
void launch_layer_norm_backward(hipStream_t s, const NormBwdArgs& a, const NormWs& w) {
    if (a.dt == SPV_F32) norm_bwd_dt<SPV_F32>(s, a, w);
    else if (a.dt == SPV_BF16) norm_bwd_dt<SPV_BF16>(s, a, w);
    else norm_bwd_dt<SPV_F16>(s, a, w);
}

}  // namespace spv
