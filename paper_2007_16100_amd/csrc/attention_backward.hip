// attention_backward.hip -- the backward of attention over packed scans:
//   s_ij = cap(scale q_i . k_j) - slope_h |c_i - c_j|_1,  j over the keys of i's scan,
//   out_i = sum_j p_ij v_j,  p_ij = exp(s_ij - lse_i)
// One wave per (row, head): a first version that is right for every shape.
#include "conv_common.hpp"

namespace spv {

constexpr int kAttnWaves = 4;

static __device__ inline int clamp_off(int32_t o, int64_t n) { return o < 0 ? 0 : (o > n ? (int)n : o); }

// the scan of a row of `off`'s side: the last b with off[b] <= row, or -1 when the row is in none
__device__ inline int scan_of(const int32_t* off, int B, int64_t row) {
    int lo = 0, hi = B;  // off[lo] <= row < off[hi]
    if (row < off[0] || row >= off[B]) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ inline int voxel_coord(int c) { return c < kCoordMin ? kCoordMin : (c > kCoordMax ? kCoordMax : c); }
__device__ inline float voxel_dist(const int32_t* a, const int32_t* b) {
    int d = 0;
#pragma unroll
    for (int e = 1; e < 4; ++e) d += abs(voxel_coord(a[e]) - voxel_coord(b[e]));
    return (float)d;
}

template <int DT>
__device__ inline float head_dot(const void* a, int64_t i, const void* b, int64_t j, int D) {
    float s = 0.f;
    for (int d = 0; d < D; ++d) s = fmaf(ld_feat<DT>(a, i + d), ld_feat<DT>(b, j + d), s);
    return s;
}

// the score of query row i (head h) and key row j; *slope receives d score / d product
template <int DT>
__device__ inline float score(const AttnArgs& a, int64_t i, int64_t j, int h, float* slope) {
    const int g = h / (a.H / a.K);
    float z = a.scale * head_dot<DT>(a.q, i * a.ldq + (int64_t)h * a.D, a.k, j * a.ldk + (int64_t)g * a.D, a.D);
    *slope = a.scale;
    if (a.cap > 0.f) {
        const float t = tanhf(z / a.cap);
        z = a.cap * t;
        *slope = a.scale * (1.f - t * t);
    }
    if (a.slopes) z -= a.slopes[h] * voxel_dist(a.q_coords + 4 * i, a.k_coords + 4 * j);
    return z;
}

__device__ inline float wave_add(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ inline float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

template <int DT>
__global__ __launch_bounds__(64 * kAttnWaves) void k_attn_dq(AttnArgs a) {
    const int lane = threadIdx.x & 63, h = blockIdx.y, g = h / (a.H / a.K);
    for (int64_t i = (int64_t)blockIdx.x * kAttnWaves + (threadIdx.x >> 6); i < a.nq;
         i += (int64_t)gridDim.x * kAttnWaves) {
        const int b = scan_of(a.q_off, a.B, i);
        if (b < 0) continue;
        const int64_t j0 = clamp_off(a.k_off[b], a.nk), j1 = clamp_off(a.k_off[b + 1], a.nk);
        const int64_t to = i * a.ldo + (int64_t)h * a.D;
        const int64_t td = i * a.lddo + (int64_t)h * a.D;
        const float delta = head_dot<DT>(a.dout, td, a.out, to, a.D), lse = a.lse[i * a.H + h];
        if (lane == 0) a.delta[i * a.H + h] = delta;
        float o0 = 0.f, o1 = 0.f;
        for (int64_t j = j0; j < j1; j += 64) {
            float dz = 0.f;
            if (j + lane < j1) {
                float sl;
                const float s = score<DT>(a, i, j + lane, h, &sl);
                const float dp = head_dot<DT>(a.dout, td, a.v, (j + lane) * a.ldv + (int64_t)g * a.D, a.D);
                dz = expf(s - lse) * (dp - delta) * sl;
            }
            const int n = (int)(j1 - j < 64 ? j1 - j : 64);
            for (int u = 0; u < n; ++u) {
                const float du = __shfl(dz, u, 64);
                const int64_t t = (j + u) * a.ldk + (int64_t)g * a.D;
                if (lane < a.D) o0 = fmaf(du, ld_feat<DT>(a.k, t + lane), o0);
                if (lane + 64 < a.D) o1 = fmaf(du, ld_feat<DT>(a.k, t + lane + 64), o1);
            }
        }
        const int64_t t = i * a.lddq + (int64_t)h * a.D;
        if (lane < a.D) st_feat<DT>(a.dq, t + lane, o0);
        if (lane + 64 < a.D) st_feat<DT>(a.dq, t + lane + 64, o1);
    }
}

template <int DT>
__global__ __launch_bounds__(64 * kAttnWaves) void k_attn_dkv(AttnArgs a) {
    const int lane = threadIdx.x & 63, g = blockIdx.y, G = a.H / a.K;
    for (int64_t j = (int64_t)blockIdx.x * kAttnWaves + (threadIdx.x >> 6); j < a.nk;
         j += (int64_t)gridDim.x * kAttnWaves) {
        const int b = scan_of(a.k_off, a.B, j);
        if (b < 0) continue;
        const int64_t i0 = clamp_off(a.q_off[b], a.nq), i1 = clamp_off(a.q_off[b + 1], a.nq);
        const int64_t tv = j * a.ldv + (int64_t)g * a.D, tk = j * a.ldk + (int64_t)g * a.D;
        float k0 = 0.f, k1 = 0.f, v0 = 0.f, v1 = 0.f;
        for (int h = g * G; h < (g + 1) * G; ++h)
            for (int64_t i = i0; i < i1; i += 64) {
                float p = 0.f, dz = 0.f;
                if (i + lane < i1) {
                    float sl;
                    const int64_t r = i + lane;
                    p = expf(score<DT>(a, r, j, h, &sl) - a.lse[r * a.H + h]);
                    dz = p * (head_dot<DT>(a.dout, r * a.lddo + (int64_t)h * a.D, a.v, tv, a.D) - a.delta[r * a.H + h]) *
                         sl;
                }
                const int n = (int)(i1 - i < 64 ? i1 - i : 64);
                for (int u = 0; u < n; ++u) {
                    const float pu = __shfl(p, u, 64), du = __shfl(dz, u, 64);
                    const int64_t to = (i + u) * a.lddo + (int64_t)h * a.D, tq = (i + u) * a.ldq + (int64_t)h * a.D;
                    if (lane < a.D) {
                        v0 = fmaf(pu, ld_feat<DT>(a.dout, to + lane), v0);
                        k0 = fmaf(du, ld_feat<DT>(a.q, tq + lane), k0);
                    }
                    if (lane + 64 < a.D) {
                        v1 = fmaf(pu, ld_feat<DT>(a.dout, to + lane + 64), v1);
                        k1 = fmaf(du, ld_feat<DT>(a.q, tq + lane + 64), k1);
                    }
                }
            }
        const int64_t ok = j * a.lddk + (int64_t)g * a.D, ov = j * a.lddv + (int64_t)g * a.D;
        if (lane < a.D) {
            st_feat<DT>(a.dk, ok + lane, k0);
            st_feat<DT>(a.dv, ov + lane, v0);
        }
        if (lane + 64 < a.D) {
            st_feat<DT>(a.dk, ok + lane + 64, k1);
            st_feat<DT>(a.dv, ov + lane + 64, v1);
        }
    }
}

void plan_attention_backward_ws(Arena& a, AttnArgs& t) { t.delta = a.take<float>((size_t)t.nq * (size_t)t.H); }

static unsigned attn_grid(int64_t n) {
    const int64_t g = (n + kAttnWaves - 1) / kAttnWaves;
    return (unsigned)(g > 65536 ? 65536 : g);
}

template <int DT>
static void attn_bwd_dt(hipStream_t s, const AttnArgs& a) {
    if (a.nq > 0) k_attn_dq<DT><<<dim3(attn_grid(a.nq), (unsigned)a.H), 64 * kAttnWaves, 0, s>>>(a);
    if (a.nk > 0) k_attn_dkv<DT><<<dim3(attn_grid(a.nk), (unsigned)a.K), 64 * kAttnWaves, 0, s>>>(a);
}
void launch_attention_backward(hipStream_t s, const AttnArgs& a) {
    if (a.dt == SPV_F32) attn_bwd_dt<SPV_F32>(s, a);
    else if (a.dt == SPV_BF16) attn_bwd_dt<SPV_BF16>(s, a);
    else attn_bwd_dt<SPV_F16>(s, a);
}

}  // namespace spv
