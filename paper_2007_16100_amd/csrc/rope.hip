// rope.hip -- rotary positions over three axes: pair p of a head's channels turns by
//   theta = c_a freqs[p],  (u, w) -> (u cos theta - w sin theta, u sin theta + w cos theta),
// c_a the row's coordinate on the axis whose section holds p.  The inverse turns by -theta.
#include "conv_common.hpp"
#include "lanes.hpp"

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

// What a row is made of: vectors of 16 bytes (pairs of halves: of two, P channels apart), those of q's heads first.
struct RopeUnits {
    int head;       // units of a head
    int turned;     // of those, pairs of vectors of halves (0: pairs are in a vector)
    int row;        // units of a row
    int rows;       // rows of a workgroup
    uint32_t by_row, by_head;  // 2^32 over the numbers of units, rounded up; 0 for one unit
};
__device__ inline int over(int i, uint32_t by) { return by ? (int)__umulhi((uint32_t)i, by) : i; }
constexpr int kRopeAhead = 4;  // units a thread asks for before it waits
constexpr int kRopeRows = 64;  // of a workgroup at most

// A workgroup takes some rows: its threads form the sines and cosines of all their pairs once for all heads, in LDS, while
// their first vectors are on the way.  Bound by memory: 88,119 rows of 16 heads of 32 in bf16.
template <int DT, bool HALVES>
__global__ __launch_bounds__(256) void k_rope_rows(RopeArgs a, RopeUnits un) {
    constexpr int V = DT == SPV_F32 ? 4 : 8, NV = HALVES ? 2 : 1;
    extern __shared__ float2 table[];  // [rows][P]
    const int64_t m = clamp_rows(a.m_dev, a.n), row0 = (int64_t)blockIdx.x * un.rows;
    if (row0 >= m) return;
    const int rows = (int)(m - row0 < un.rows ? m - row0 : un.rows), all = rows * un.row;
    struct Unit {
        uint4 v[NV];
        char* out;
        int r, c;   // row, first channel of the head
        bool two;   // halves: both vectors
    };
    auto ask = [&](int idx, Unit& t) {
        const int i = idx < all ? idx : 0;
        t.r = over(i, un.by_row);
        const int u = i - t.r * un.row;
        const int h = over(u, un.by_head), x = u - h * un.head;
        const bool of_q = h < a.q.heads;
        const RopeSide& s = of_q ? a.q : a.k;
        t.two = HALVES && x < un.turned;
        t.c = !HALVES || t.two ? x * V : (x + un.turned) * V;
        const int64_t e = (int64_t)(of_q ? h : h - a.q.heads) * a.D + t.c;
        const char* in = (const char*)s.in + ((row0 + t.r) * s.ld + e) * (16 / V);
        t.out = (char*)s.out + ((row0 + t.r) * s.ldo + e) * (16 / V);
        t.v[0] = *(const uint4*)in;
        if constexpr (HALVES)
            if (t.two) t.v[1] = *(const uint4*)(in + (int64_t)a.P * (16 / V));
    };
    Unit now[kRopeAhead];
#pragma unroll
    for (int k = 0; k < kRopeAhead; ++k) ask((int)threadIdx.x + k * 256, now[k]);
    for (int j = threadIdx.x; j < rows * a.P; j += 256) {
        const int r = j / a.P, p = j - r * a.P, axis = p < a.sx ? 1 : p < a.sx + a.sy ? 2 : 3;
        float2 cs = cos_sin(voxel_axis(a.coords + 4 * (row0 + r) + axis), a.freqs[p]);
        if (a.inverse) cs.y = -cs.y;
        table[j] = cs;
    }
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < all; i0 += kRopeAhead * 256) {
#pragma unroll
        for (int k = 0; k < kRopeAhead; ++k) {
            if (i0 + k * 256 >= all) break;
            Unit& t = now[k];
            const float2* cs = table + t.r * a.P;
            if constexpr (HALVES) {
                if (t.two) {
                    float x[V], y[V];
                    unpack16<DT>(t.v[0], x);
                    unpack16<DT>(t.v[1], y);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float2 q = cs[t.c + e];
                        const float u = x[e], w = y[e];
                        x[e] = u * q.x - w * q.y;
                        y[e] = u * q.y + w * q.x;
                    }
                    *(uint4*)(t.out + (int64_t)a.P * (16 / V)) = pack16<DT>(y);
                    t.v[0] = pack16<DT>(x);
                }
            } else if (t.c < 2 * a.P) {
                float x[V];
                unpack16<DT>(t.v[0], x);
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const int p = (t.c + e) / 2;
                    if (p >= a.P) break;  // channels that stay
                    const float2 q = cs[p];
                    const float u = x[e], w = x[e + 1];
                    x[e] = u * q.x - w * q.y;
                    x[e + 1] = u * q.y + w * q.x;
                }
                t.v[0] = pack16<DT>(x);
            }
            *(uint4*)t.out = t.v[0];
        }
        if (i0 + kRopeAhead * 256 < all)
#pragma unroll
            for (int k = 0; k < kRopeAhead; ++k) ask(i0 + (kRopeAhead + k) * 256, now[k]);
    }
}

// Pairs of halves that vectors do not hold whole (P no multiple of theirs), and rows of millions of channels:
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

template <int DT>
static bool rope_rows(hipStream_t s, const RopeArgs& a) {
    constexpr int V = DT == SPV_F32 ? 4 : 8;
    if (a.halves && a.P % V) return false;
    RopeUnits u;
    u.turned = a.halves ? a.P / V : 0;
    u.head = a.halves ? a.D / V - u.turned : a.D / V;
    const int64_t row = (int64_t)(a.q.heads + a.k.heads) * u.head;
    // kRopeAhead units a thread
    int64_t rows = (256 * kRopeAhead + row - 1) / row;
    if (rows > kRopeRows) rows = kRopeRows;
    if (rows * row * row >= ((int64_t)1 << 32)) return false;  // quotients by a product are exact below
    u.row = (int)row;
    u.rows = (int)rows;
    auto by = [](int64_t n) { return n > 1 ? (uint32_t)((((uint64_t)1 << 32) + (uint64_t)n - 1) / (uint64_t)n) : 0u; };
    u.by_row = by(row);
    u.by_head = by(u.head);
    const unsigned g = (unsigned)((a.n + rows - 1) / rows);
    const size_t lds = (size_t)rows * a.P * sizeof(float2);  // 32 KiB at most
    if (a.halves) k_rope_rows<DT, true><<<g, 256, lds, s>>>(a, u);
    else k_rope_rows<DT, false><<<g, 256, lds, s>>>(a, u);
    return true;
}
void launch_rope(hipStream_t s, const RopeArgs& a) {
    if (a.dt == SPV_F32 ? rope_rows<SPV_F32>(s, a) : a.dt == SPV_BF16 ? rope_rows<SPV_BF16>(s, a) : rope_rows<SPV_F16>(s, a))
        return;
    const int64_t threads = a.n * (a.q.heads + a.k.heads) * (a.D / 2);
    const unsigned g = (unsigned)(threads / 256 + 1 < 65536 ? threads / 256 + 1 : 65536);
    if (a.dt == SPV_F32) k_rope<SPV_F32><<<g, 256, 0, s>>>(a);
    else if (a.dt == SPV_BF16) k_rope<SPV_BF16><<<g, 256, 0, s>>>(a);
    else k_rope<SPV_F16><<<g, 256, 0, s>>>(a);
}

}  // namespace spv
