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

// cosines and sines of all pairs of some rows, by a workgroup
__device__ inline void rope_table(const RopeArgs& a, int64_t row0, int rows, float2* table) {
    for (int j = threadIdx.x; j < rows * a.P; j += 256) {
        const int r = j / a.P, p = j - r * a.P, axis = p < a.sx ? 1 : p < a.sx + a.sy ? 2 : 3;
        float2 cs = cos_sin(voxel_axis(a.coords + 4 * (row0 + r) + axis), a.freqs[p]);
        if (a.inverse) cs.y = -cs.y;
        table[j] = cs;
    }
}

// What a row is made of: vectors of 16 bytes (pairs of halves: of two, P channels apart), those of q's heads first.
struct RopeUnits {
    int head;       // units of a head
    int turned;     // of those, pairs of vectors of halves (0: pairs are in a vector)
    int row;        // units of a row
    int rows;       // rows of a workgroup
    uint32_t by_row, by_head;  // 2^32 over the numbers of units, rounded up; 0 where that is not exact
};
__device__ inline int over(int i, uint32_t by, int n) { return by ? (int)__umulhi((uint32_t)i, by) : i / n; }
constexpr int kRopeAhead = 4;  // units a thread asks for before it waits
constexpr int kRopeRows = 64;  // of a workgroup at most

// A workgroup takes some rows: its threads form the sines and cosines of all their pairs once for all heads, in LDS,
// while their first vectors are on the way.  Bound by memory: 88,119 rows of 16 heads of 32 in bf16, 180 MB, take 34
// us.
template <int DT, bool HALVES>
__global__ __launch_bounds__(256) void k_rope_rows(RopeArgs a, RopeUnits un) {
    constexpr int V = DT == SPV_F32 ? 4 : 8, NV = HALVES ? 2 : 1;
    extern __shared__ float2 table[];  // [rows][P]
    const int64_t m = clamp_rows(a.m_dev, a.n), row0 = group_of_grid() * un.rows;
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
        t.r = over(i, un.by_row, un.row);
        const int u = i - t.r * un.row;
        const int h = over(u, un.by_head, un.head), x = u - h * un.head;
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
    rope_table(a, row0, rows, table);
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

// Pairs of halves that vectors do not hold whole (P no multiple of theirs), and rows of millions of channels: a
// thread takes pairs of single channels, those that stay two by two.
template <int DT>
__global__ __launch_bounds__(256) void k_rope_pairs(RopeArgs a, RopeUnits un) {
    extern __shared__ float2 table[];  // [rows][P]
    const int64_t m = clamp_rows(a.m_dev, a.n), row0 = group_of_grid() * un.rows;
    if (row0 >= m) return;
    const int rows = (int)(m - row0 < un.rows ? m - row0 : un.rows), all = rows * un.row;
    rope_table(a, row0, rows, table);
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < all; i0 += kRopeAhead * 256) {
        float u[kRopeAhead], w[kRopeAhead];
        int64_t to[kRopeAhead];
        int r[kRopeAhead], p[kRopeAhead], step[kRopeAhead];
        void* out[kRopeAhead];
#pragma unroll
        for (int k = 0; k < kRopeAhead; ++k) {
            const int i = i0 + k * 256 < all ? i0 + k * 256 : 0;
            r[k] = over(i, un.by_row, un.row);
            const int v = i - r[k] * un.row, hh = over(v, un.by_head, un.head);
            p[k] = v - hh * un.head;
            const bool of_q = hh < a.q.heads, turned = p[k] < a.P;
            const RopeSide& s = of_q ? a.q : a.k;
            const int64_t e = (int64_t)(of_q ? hh : hh - a.q.heads) * a.D + (turned && a.halves ? p[k] : 2 * p[k]);
            step[k] = turned && a.halves ? a.P : 1;
            out[k] = s.out;
            to[k] = (row0 + r[k]) * s.ldo + e;
            u[k] = ld_feat<DT>(s.in, (row0 + r[k]) * s.ld + e);
            w[k] = ld_feat<DT>(s.in, (row0 + r[k]) * s.ld + e + step[k]);
        }
#pragma unroll
        for (int k = 0; k < kRopeAhead; ++k) {
            if (i0 + k * 256 >= all) break;
            if (p[k] < a.P) {
                const float2 q = table[r[k] * a.P + p[k]];
                const float x = u[k] * q.x - w[k] * q.y;
                w[k] = u[k] * q.y + w[k] * q.x;
                u[k] = x;
            }
            st_feat<DT>(out[k], to[k], u[k]);
            st_feat<DT>(out[k], to[k] + step[k], w[k]);
        }
    }
}

template <int DT>
static void rope(hipStream_t s, const RopeArgs& a) {
    constexpr int V = DT == SPV_F32 ? 4 : 8;
    const bool wide = !(a.halves && a.P % V) && (int64_t)(a.q.heads + a.k.heads) * a.D < (1 << 20);
    RopeUnits u;
    u.turned = a.halves ? a.P / V : 0;
    u.head = !wide ? a.D / 2 : a.halves ? a.D / V - u.turned : a.D / V;
    u.row = (a.q.heads + a.k.heads) * u.head;  // 131,070 heads of 64 pairs at most
    u.rows = (256 * kRopeAhead + u.row - 1) / u.row;  // kRopeAhead units a thread
    if (u.rows > kRopeRows) u.rows = kRopeRows;
    // a quotient by a product is exact while units * units of a row stay below 2^32
    auto by = [&](int n, int64_t most) {
        return n > 1 && most * n < ((int64_t)1 << 32) ? (uint32_t)((((uint64_t)1 << 32) + (uint64_t)n - 1) / (uint64_t)n) : 0u;
    };
    u.by_row = by(u.row, (int64_t)u.rows * u.row);
    u.by_head = by(u.head, u.row);
    const dim3 g = grid_of((a.n + u.rows - 1) / u.rows);
    const size_t lds = (size_t)u.rows * a.P * sizeof(float2);  // 32 KiB at most
    if (!wide) k_rope_pairs<DT><<<g, 256, lds, s>>>(a, u);
    else if (a.halves) k_rope_rows<DT, true><<<g, 256, lds, s>>>(a, u);
    else k_rope_rows<DT, false><<<g, 256, lds, s>>>(a, u);
}
void launch_rope(hipStream_t s, const RopeArgs& a) {
    if (a.dt == SPV_F32) rope<SPV_F32>(s, a);
    else if (a.dt == SPV_BF16) rope<SPV_BF16>(s, a);
    else rope<SPV_F16>(s, a);
}

}  // namespace spv
