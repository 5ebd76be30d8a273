// checkpoint8.hip -- activation checkpoints in 8 bits: rows into codes and back, and the weight gradient of a linear
// layer from codes, dW = in^T da.
#include "attn_common.hpp"
#include "code8.hpp"

namespace spv {

__device__ inline int64_t RowRange::begin() const { return off ? clamp_off(off[0], cap) : 0; }
__device__ inline int64_t RowRange::end() const { return off ? clamp_off(off[B], cap) : clamp_rows(m_dev, cap); }

// a thread takes a block of 32 channels
template <int DT>
__global__ __launch_bounds__(256) void k_code8(const void* x, Saved8 to, RowRange rows, int C) {
    const int nb = code_blocks(C);
    const int64_t end = rows.end() * nb;
    for (int64_t t = rows.begin() * nb + (int64_t)blockIdx.x * 256 + threadIdx.x; t < end; t += (int64_t)gridDim.x * 256) {
        const int64_t i = t / nb;
        const int c0 = (int)(t % nb) * kCodeBlock, c1 = c0 + kCodeBlock < C ? c0 + kCodeBlock : C;
        uint32_t top = 0;
        for (int c = c0; c < c1; ++c) top = max(top, finite_bits(ld_feat<DT>(x, i * C + c)));
        const int e = code_exp<DT>(top);
        const float rate = code_rate(e);
        to.exps[t] = (uint8_t)e;
        for (int c = c0; c < c1; ++c) to.codes[i * C + c] = (int8_t)code_of(ld_feat<DT>(x, i * C + c), rate);
    }
}

template <int DT>
__global__ __launch_bounds__(256) void k_code8_read(Saved8 from, void* out, const int64_t* m_dev, int64_t m_cap, int C) {
    const int64_t all = clamp_rows(m_dev, m_cap) * C;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < all; t += (int64_t)gridDim.x * 256) {
        const int64_t i = t / C;
        const int c = (int)(t % C);
        st_feat<DT>(out, t, code_value(from.codes[t], code_step(from.exps[i * code_blocks(C) + c / kCodeBlock])));
    }
}

static unsigned grid_for(int64_t threads) {
    const int64_t g = (threads + 255) / 256;
    return (unsigned)(g < 1 ? 1 : g > 65536 ? 65536 : g);
}
void launch_checkpoint8(hipStream_t s, const void* x, Saved8 to, const RowRange& rows, int C, int dt) {
    const unsigned g = grid_for(rows.cap * code_blocks(C));
    if (dt == SPV_F32) k_code8<SPV_F32><<<g, 256, 0, s>>>(x, to, rows, C);
    else if (dt == SPV_BF16) k_code8<SPV_BF16><<<g, 256, 0, s>>>(x, to, rows, C);
    else k_code8<SPV_F16><<<g, 256, 0, s>>>(x, to, rows, C);
}
void launch_checkpoint8_read(hipStream_t s, Saved8 from, void* out, const int64_t* m_dev, int64_t m_cap, int C, int dt) {
    const unsigned g = grid_for(m_cap * C);
    if (dt == SPV_F32) k_code8_read<SPV_F32><<<g, 256, 0, s>>>(from, out, m_dev, m_cap, C);
    else if (dt == SPV_BF16) k_code8_read<SPV_BF16><<<g, 256, 0, s>>>(from, out, m_dev, m_cap, C);
    else k_code8_read<SPV_F16><<<g, 256, 0, s>>>(from, out, m_dev, m_cap, C);
}

// ---------------------------------------------------------------------------
// dW = in^T da: a workgroup takes 32 x 32 of dW over every S-th chunk of 32 rows
// ---------------------------------------------------------------------------
constexpr int kWg8Rows = 32;
static int wgrad8_parts(int64_t m_cap, int Cin, int Cout) {
    const int64_t tiles = (int64_t)((Cin + 31) / 32) * ((Cout + 31) / 32), chunks = (m_cap + kWg8Rows - 1) / kWg8Rows;
    int64_t s = (1024 + tiles - 1) / tiles;
    if (s > chunks) s = chunks;
    return (int)(s < 1 ? 1 : s);
}
float* plan_wgrad8_ws(Arena& a, int64_t m_cap, int Cin, int Cout) {
    return a.take<float>((size_t)wgrad8_parts(m_cap, Cin, Cout) * Cin * Cout);
}

template <int DT>
__global__ __launch_bounds__(256) void k_wgrad8(Wgrad8Args a) {
    __shared__ float xs[kWg8Rows][33], ds[kWg8Rows][33];
    const int ci = blockIdx.y * 32, co = blockIdx.z * 32, tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int64_t m = clamp_rows(a.m_dev, a.m_cap);
    float acc[4] = {};
    for (int64_t r0 = (int64_t)blockIdx.x * kWg8Rows; r0 < m; r0 += (int64_t)gridDim.x * kWg8Rows) {
        __syncthreads();
        for (int r = ty; r < kWg8Rows; r += 8) {
            const int64_t i = r0 + r;
            xs[r][tx] = i < m && ci + tx < a.Cin ? code_value(a.in.codes[i * a.Cin + ci + tx],
                                                              code_step(a.in.exps[i * code_blocks(a.Cin) + blockIdx.y]))
                                                 : 0.f;
            ds[r][tx] = i < m && co + tx < a.Cout ? ld_feat<DT>(a.da, i * a.Cout + co + tx) : 0.f;
        }
        __syncthreads();
        for (int r = 0; r < kWg8Rows; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = fmaf(xs[r][ty + 8 * j], ds[r][tx], acc[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (ci + ty + 8 * j < a.Cin && co + tx < a.Cout)
            a.part[((int64_t)blockIdx.x * a.Cin + ci + ty + 8 * j) * a.Cout + co + tx] = acc[j];
}

__global__ __launch_bounds__(256) void k_wgrad8_join(const float* part, int parts, int64_t n, float* dW) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= n) return;
    double s = 0.0;
    for (int p = 0; p < parts; ++p) s += (double)part[p * n + t];
    dW[t] = (float)s;
}

void launch_wgrad8(hipStream_t s, const Wgrad8Args& a) {
    const int parts = wgrad8_parts(a.m_cap, a.Cin, a.Cout);
    const dim3 g((unsigned)parts, (unsigned)((a.Cin + 31) / 32), (unsigned)((a.Cout + 31) / 32));
    if (a.dt == SPV_F32) k_wgrad8<SPV_F32><<<g, 256, 0, s>>>(a);
    else if (a.dt == SPV_BF16) k_wgrad8<SPV_BF16><<<g, 256, 0, s>>>(a);
    else k_wgrad8<SPV_F16><<<g, 256, 0, s>>>(a);
    const int64_t n = (int64_t)a.Cin * a.Cout;
    k_wgrad8_join<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(a.part, parts, n, a.dW);
}

}  // namespace spv
