// group_norm.hip -- group norm of packed scans with an activation, and its backward:
//   xh = (x - mu) r,  z = xh gamma + beta,  y = act(z),
//   mu, r from the rows of a scan and the channels of a group together;
//   gz = dy act'(z),  h = gz gamma,  dx = r (h - mean h - xh mean(h xh)) (+ dres),
//   dgamma = sum gz xh,  dbeta = sum gz.
//
// A scan's statistics take all of its rows, so each direction reads its rows twice.  Rows are cut into tiles of one
// scan each, one to a workgroup: a first kernel leaves a tile's sums of each group, a second joins those of the
// tile's scan (each workgroup again: a few thousand numbers, and a launch less) and writes the rows.  (One kernel
// that keeps its rows over a barrier of all workgroups would read them once, but two such kernels on two streams
// could each wait for room that the other holds.)
//
// Bound by memory, where rows are many: 300,007 x 96 in bf16 takes 35 us, 173 MB at 4.9 TB/s (a copy reaches 5.1): 13
// for the statistics, 20 for the rows.  A training step of 88,119 x 96 with the residual's gradient, 152 MB, 41 us:
// 8, 10, 11 and 14 in a kernel trace (which adds some), of which 4 each are the launch, the search for the tile, the
// join and the last waves.
#include <type_traits>

#include "attn_common.hpp"
#include "code8.hpp"

namespace spv {

// exp and the reciprocal are the hardware's, each off by 2^-23 of itself at most, and the exponent's rounding adds
// |z| 2^-24
__device__ inline float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -kLog2e));
}
template <int ACT>
__device__ inline float act_of(float z) {
    if constexpr (ACT == SPV_ACT_RELU) return z <= 0.f ? 0.f : z;
    else if constexpr (ACT == SPV_ACT_SILU) return z * sigmoid(z);
    else return z;
}
// d act'(z); ReLU's is d or 0, also where d is not finite
template <int ACT>
__device__ inline float act_grad(float d, float z) {
    if constexpr (ACT == SPV_ACT_RELU) {
        return z <= 0.f ? 0.f : d;
    } else if constexpr (ACT == SPV_ACT_SILU) {
        const float s = sigmoid(z);
        return d * fmaf(s, fmaf(-z, s, z), s);  // s (1 + z (1 - s))
    } else {
        return d;
    }
}

// ---------------------------------------------------------------------------
// Tiles.  A thread holds VEC channels (16 bytes, or one where rows are odd or unaligned) of every R-th row of its
// workgroup's tile, so what belongs to a channel stays in registers over the rows; R = kGnThreads / (C / VEC).
// ---------------------------------------------------------------------------
constexpr int kGnThreads = 512, kGnWaves = kGnThreads / 64;
// Tiles of one long scan: with the scans' first ones and the workgroups that join the channels, about one a CU.  What
// a workgroup does besides its rows (some 4 us, at the start and the end) is not hidden by a second one that does the
// same: 240, 384 and 512 tiles take 35.4, 35.7 and 37.9 us for 300,007 x 96 in bf16 (512 being more than fit at once) and
// 41.0, 44.4 and 44.9 for the training step of 88,119 x 96.
constexpr int kGnTiles = 240;

template <int DT>
constexpr int kGnVec = DT == SPV_F32 ? 4 : 8;

// VEC channels as they are loaded, in float32 and stored
template <int DT, int VEC>
struct Chans {
    using Raw = std::conditional_t<VEC == 1, float, uint4>;
    static __device__ Raw load(const void* p, int64_t e) {
        if constexpr (VEC == 1) return ld_feat<DT>(p, e);
        else return *(const uint4*)((const char*)p + e * (16 / VEC));
    }
    static __device__ void unpack(const Raw& r, float (&x)[VEC]) {
        if constexpr (VEC == 1) x[0] = r;
        else unpack16<DT>(r, x);
    }
    static __device__ void store(void* p, int64_t e, const float (&x)[VEC]) {
        if constexpr (VEC == 1) st_feat<DT>(p, e, x[0]);
        else *(uint4*)((char*)p + e * (16 / VEC)) = pack16<DT>(x);
    }
};

// VEC channels of a row in 8 bits: VEC codes and their exponent
template <int VEC>
struct Codes {
    struct Raw {
        uint32_t w[VEC == 8 ? 2 : 1];
        int e;
    };
    // at element e, whose block is number block
    static __device__ Raw load(const Saved8& s, int64_t e, int64_t block) {
        Raw r;
        const int8_t* p = s.codes + e;
        if constexpr (VEC == 8) {
            const uint2 u = *(const uint2*)p;
            r.w[0] = u.x, r.w[1] = u.y;
        } else if constexpr (VEC == 4) {
            r.w[0] = *(const uint32_t*)p;
        } else {
            r.w[0] = (uint8_t)*p;
        }
        r.e = s.exps[block];
        return r;
    }
    static __device__ void unpack(const Raw& r, float (&x)[VEC]) {
        if constexpr (VEC == 1) x[0] = code_value((int8_t)r.w[0], code_step(r.e));
        else code_values(r.w, code_step(r.e), x);
    }
};

__device__ inline int over(int i, uint32_t by) { return by ? (int)__umulhi((uint32_t)i, by) : i; }

// a thread's row of R and its first channel (row R: it has none)
template <int VEC>
struct GnThread {
    int row, c;
    __device__ explicit GnThread(const GnShape& s)
        : row(over((int)threadIdx.x, s.by_nv)), c(((int)threadIdx.x - row * s.nv) * VEC) {}
};

// the two numbers of a thread's channels' groups
template <int VEC, class F>
__device__ inline void gn_of_groups(const GnShape& s, const float2* groups, int c, F&& f) {
    if (VEC == 1 || s.whole) {
        const float2 v = groups[over(c, s.by_w)];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f(e, v);
    } else {
        float2 v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = groups[over(c + e, s.by_w)];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f(e, v[e]);
    }
}

// a thread's channels of a vector, or `other` of each
template <int VEC>
__device__ inline void gn_channels(const float* p, int c, float other, float (&v)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = other;
    if (p) __builtin_memcpy(v, p + c, sizeof(v));
}

struct GnTile {
    int b;            // scan
    int64_t row0;     // first row
    int rows;         // of the tile
    uint32_t n;       // rows of the scan
    int64_t tile0;    // number of the scan's first tile
    bool first;       // this is it
};
// Scan b's first tile is number off[b] / tile_rows + b: known without a pass over the scans, with room for every
// scan's tiles.  Tile t's scan is found with 63 intervals a step.
__device__ inline GnTile gn_tile(const GnArgs& a, uint32_t tile_rows, uint32_t t) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = a.B, step, k;
    uint32_t o, tile;
    do {
        step = (hi - lo + 62) / 63;
        const int at = lo + step * lane;
        o = at <= hi ? (uint32_t)clamp_off(a.off[at], a.m) : 0u;
        tile = o / tile_rows + (uint32_t)at;
        k = __popcll(__ballot(at < hi && tile <= t));
        k = uniform(k > 0 ? k - 1 : 0);
        lo += step * k;
        hi = lo + step < hi ? lo + step : hi;
    } while (step > 1);
    GnTile g;
    g.b = uniform(lo);
    const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)o, k), end = (uint32_t)__builtin_amdgcn_readlane((int)o, k + 1);
    g.tile0 = (uint32_t)__builtin_amdgcn_readlane((int)tile, k);
    g.n = end > first ? end - first : 0u;
    const uint32_t done = (t - (uint32_t)g.tile0) * tile_rows;  // t is at least tile0, or past all of the scans
    g.row0 = first + done;
    g.rows = t >= (uint32_t)g.tile0 && done < g.n ? (int)(g.n - done < tile_rows ? g.n - done : tile_rows) : 0;
    g.first = t == (uint32_t)g.tile0;
    return g;
}

// The tiles of a group of a scan, taken by a wave, or where scans have few tiles by 8 lanes: four a lane are asked
// for by the constructor, before whatever else the workgroup has to wait for, the others in turn.
struct GnGroup {
    const float2* part;
    int64_t stride, tiles;
    int lanes;
    float first;  // the mean of the first tile
    float2 p[4];
    // group g of a thread that has none (past G): as group 0
    __device__ GnGroup(const GnArgs& a, int g, int64_t tile0, uint32_t n, uint32_t tile_rows)
        : part(a.tiles + tile0 * a.G + (g < a.G ? g : 0)), stride(a.G), tiles((n + tile_rows - 1) / tile_rows),
          lanes(a.few_tiles ? 8 : 64) {
        first = tiles > 0 ? part[0].x : 0.f;
        ask(0);
    }
    __device__ int64_t tile(int64_t t0, int k) const { return t0 + k * lanes + (threadIdx.x & (lanes - 1)); }
    __device__ void ask(int64_t t0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = tile(t0, k) < tiles ? part[tile(t0, k) * stride] : make_float2(0.f, 0.f);
    }
    // f(tile, its numbers) for the lane's tiles, zeros past the last
    template <class F>
    __device__ void each(F&& f) {
        for (int64_t t0 = 0;;) {
#pragma unroll
            for (int k = 0; k < 4; ++k) f(tile(t0, k), p[k]);
            t0 += 4 * lanes;
            if (t0 >= tiles) break;
            ask(t0);
        }
    }
    __device__ double sum(double v) const { return lanes_sum(v, lanes == 64); }
};
// Mean and r of a group of a scan of n rows from its tiles' means and sums of squares.  Deviations are from
// the first tile's mean, whose distance from the mean of all, squared, is at most (tiles) times the variance: what
// cancels in 64 bits is a few thousand of their units.
__device__ inline float2 gn_join_stat(GnGroup& t, uint32_t n, uint32_t tile_rows, int w, float eps) {
    if (n == 0) return make_float2(0.f, 0.f);
    const double first = (double)t.first, per = 1.0 / (double)n;
    double s = 0.0, q = 0.0;
    t.each([&](int64_t i, const float2& p) {
        const int64_t left = (int64_t)n - i * tile_rows;
        const double rows = (double)(left < 0 ? 0 : left < tile_rows ? left : tile_rows), d = (double)p.x - first;
        s = fma(rows, d, s);
        q += fma(rows * w * d, d, (double)p.y);
    });
    s = t.sum(s) * per;
    q = t.sum(q) * per / (double)w - s * s;
    return make_float2((float)(first + s), 1.f / sqrtf((float)(q > 0.0 ? q : q == q ? 0.0 : q) + eps));
}
// the sums of a group of a scan from its tiles', over the count
__device__ inline float2 gn_join_sums(GnGroup& t, uint32_t n, int w) {
    const double per = n > 0 ? 1.0 / ((double)n * (double)w) : 0.0;
    double s1 = 0.0, s2 = 0.0;
    t.each([&](int64_t, const float2& p) {
        s1 += (double)p.x;
        s2 += (double)p.y;
    });
    return make_float2((float)(t.sum(s1) * per), (float)(t.sum(s2) * per));
}
// All groups of a tile's scan into LDS, the thread's first one asked for already: f(group's tiles) is what is stored.
template <class F>
__device__ inline void gn_join_all(const GnArgs& a, const GnTile& t, uint32_t tile_rows, GnGroup& first, float2* out, F&& f) {
    if (a.joined) {
        for (int g = threadIdx.x; g < a.G; g += kGnThreads) out[g] = a.joined[(int64_t)t.b * a.G + g];
        return;
    }
    const int lanes = first.lanes, own = (int)threadIdx.x / lanes;
    for (int g0 = 0; g0 < a.G; g0 += kGnThreads / lanes) {  // all lanes take part in the sums
        if (g0) first = GnGroup(a, g0 + own, t.tile0, t.n, tile_rows);
        const float2 v = f(first);
        if ((threadIdx.x & (lanes - 1)) == 0 && g0 + own < a.G) out[g0 + own] = v;
    }
}

// rows a thread asks for at a time: more of single channels, which are 2 or 4 bytes each
// (300,007 x 19 in 19 groups 23 -> 21 us)
constexpr int gn_ahead(int vec, int rows) { return vec == 1 ? 4 * rows : rows; }

// A thread's rows of a tile (row, row + R, ..), U at a time, the next U asked for before the present ones are used.
// ask() comes before whatever the first rows can be waited for during.  A row past the end is asked for as row 0.
template <int U, class Raw>
struct GnRows {
    int row, R, rows;
    Raw u[U];
    template <class L>
    __device__ void ask(int i0, Raw (&to)[U], L&& load) const {
#pragma unroll
        for (int k = 0; k < U; ++k) to[k] = load(i0 + k * R < rows ? i0 + k * R : 0);
    }
    // use(first row, rows asked for); rows from `rows` on are not the thread's
    template <class L, class F>
    __device__ void run(L&& load, F&& use) {
        for (int i0 = row; i0 < rows; i0 += U * R) {
            Raw next[U];
            if (i0 + U * R < rows) ask(i0 + U * R, next, load);
            use(i0, u);
#pragma unroll
            for (int k = 0; k < U; ++k) u[k] = next[k];
        }
    }
};

// a wave takes a group of a scan
template <bool STAT>
__global__ __launch_bounds__(256) void k_gn_join(GnArgs a, uint32_t tile_rows) {
    const int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (u >= (int64_t)a.B * a.G) return;
    const int b = (int)(u / a.G), g = (int)(u % a.G);
    const uint32_t r0 = (uint32_t)clamp_off(a.off[b], a.m), r1 = (uint32_t)clamp_off(a.off[b + 1], a.m);
    const uint32_t n = r1 > r0 ? r1 - r0 : 0u;
    GnGroup t(a, g, (int64_t)(r0 / tile_rows) + b, n, tile_rows);
    const float2 v = STAT ? gn_join_stat(t, n, tile_rows, a.C / a.G, a.eps) : gn_join_sums(t, n, a.C / a.G);
    if ((threadIdx.x & 63) == 0) a.joined[u] = v;
}

// The groups of a tile of `rows` rows, joined from the units' means and squares: val[R][C / unit], L lanes a group.
// A thread's row holds every R-th one.
template <int L>
__device__ inline void gn_units(const GnArgs& a, int rows, const float2* val) {
    const GnShape& sh = a.sh;
    const int l = threadIdx.x & (L - 1), R = sh.R, per = sh.per, units = sh.units, all = R * per;
    const int least = rows / R, more = rows - least * R;  // a thread's row has least rows, the first ones one more
    const float inv = 1.f / ((float)rows * (float)per);
    for (int g0 = 0; g0 < a.G; g0 += kGnThreads / L) {  // all lanes take part in the sums
        const int g = g0 + (int)threadIdx.x / L;
        const float2* v = val + (g < a.G ? g : 0) * per;
        const float first = v[0].x;  // equal values give their mean exactly
        float s = 0.f, q = 0.f;
        for (int j = l; j < all; j += L) {
            const int r = over(j, sh.by_per);
            s = fmaf((float)(least + (r < more)), v[r * units + (j - r * per)].x - first, s);
        }
        const float mu = fmaf(lanes_sum<L>(s), inv, first);
        for (int j = l; j < all; j += L) {
            const int r = over(j, sh.by_per), n = least + (r < more);
            const float2 p = v[r * units + (j - r * per)];
            const float d = n ? p.x - mu : 0.f;  // a unit of no rows: mu's square may be infinite
            q += fmaf(d * d, (float)(n * sh.unit), p.y);
        }
        q = lanes_sum<L>(q);
        if (l == 0 && g < a.G) a.tiles[(int64_t)blockIdx.x * a.G + g] = make_float2(mu, q);
    }
}

// A tile's mean and sum of squared deviations of each group.  A thread keeps the running mean of each of its channels
// and the squares of the deviations from it, four rows at a time: no cancellation however far from zero the rows sit.
template <int DT, int VEC>
__global__ __launch_bounds__(kGnThreads) void k_gn_tile_stat(GnArgs a, int tile_rows) {
    using V = Chans<DT, VEC>;
    __shared__ float2 s_val[kGnThreads * VEC];
    const GnTile t = gn_tile(a, tile_rows, blockIdx.x);
    if (t.rows == 0) return;
    const GnThread<VEC> th(a.sh);
    const int R = a.sh.R, row = th.row, c = th.c, unit = a.sh.unit;
    if (row < R) {
        float mean[VEC], sq[VEC], n = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) mean[e] = sq[e] = 0.f;
        const int64_t base = t.row0 * a.C + c;
        auto load = [&](int i) { return V::load(a.x, base + (int64_t)i * a.C); };
        constexpr int U = gn_ahead(VEC, 4);
        GnRows<U, typename V::Raw> rows{row, R, t.rows};
        rows.ask(row, rows.u, load);
        auto four = [&](int i0, const typename V::Raw* u) {
            float x[4][VEC];
#pragma unroll
            for (int k = 0; k < 4; ++k) V::unpack(u[k], x[k]);
            if (i0 + 3 * R < t.rows) {
                const float f = 4.f * __builtin_amdgcn_rcpf(n + 4.f), g = n * f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    // distances to the first: equal values give their mean exactly, the type's largest and smallest too;
                    // the squares about the mean are what is left of those about the first, a quarter at least
                    const float d1 = x[1][e] - x[0][e], d2 = x[2][e] - x[0][e], d3 = x[3][e] - x[0][e], s = (d1 + d2) + d3;
                    const float m = s * 0.25f, d = (x[0][e] - mean[e]) + m;
                    sq[e] = fmaf(d3, d3, fmaf(d2, d2, fmaf(d1, d1, sq[e])));
                    sq[e] = fmaf(-s, m, sq[e]);
                    mean[e] = fmaf(d, f, mean[e]);
                    sq[e] = fmaf(d * g, d, sq[e]);
                }
                n += 4.f;
                return;
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                if (i0 + k * R >= t.rows) break;
                n += 1.f;
                const float f = __builtin_amdgcn_rcpf(n);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float d = x[k][e] - mean[e];
                    mean[e] = fmaf(d, f, mean[e]);
                    sq[e] = fmaf(d, x[k][e] - mean[e], sq[e]);
                }
            }
        };
        rows.run(load, [&](int i0, const typename V::Raw(&u)[U]) {
#pragma unroll
            for (int k = 0; k < U; k += 4) four(i0 + k * R, u + k);
        });
        // equal counts: units of two, four and eight channels, while a group is made of those
#pragma unroll
        for (int h = 1; h < VEC; h *= 2) {
            if (unit < 2 * h) break;
#pragma unroll
            for (int e = 0; e + h < VEC; e += 2 * h) {
                const float d = mean[e + h] - mean[e];
                mean[e] = fmaf(d, 0.5f, mean[e]);
                sq[e] += fmaf(d * d, 0.5f * n * (float)h, sq[e + h]);
            }
        }
        const int shift = unit >> 1 ? unit >> 2 ? unit >> 3 ? 3 : 2 : 1 : 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if ((e & (unit - 1)) == 0) s_val[row * a.sh.units + ((c + e) >> shift)] = make_float2(mean[e], sq[e]);
    }
    __syncthreads();
    // a group's units of all the threads' rows, by 64 lanes or by 8
    if (R * a.sh.per > 32) gn_units<64>(a, t.rows, s_val);
    else gn_units<8>(a, t.rows, s_val);
}

// the rows' second pass: y, and x in 8 bits (CODE: whole blocks of 32 channels)
template <int DT, int VEC, int ACT, bool CODE>
__global__ __launch_bounds__(kGnThreads) void k_gn_tile_apply(GnArgs a, int tile_rows) {
    using V = Chans<DT, VEC>;
    __shared__ float2 s_stat[kGnThreads * VEC];  // at most as many groups as channels
    const GnThread<VEC> th(a.sh);
    const int R = a.sh.R, row = th.row, c = th.c, w = a.sh.w;
    const GnTile t = gn_tile(a, tile_rows, blockIdx.x);
    if (t.rows == 0 && !(t.first && a.stat)) return;
    GnGroup first(a, (int)threadIdx.x / (a.few_tiles ? 8 : 64), t.tile0, a.joined ? 0u : t.n, tile_rows);
    float ga[VEC], be[VEC];
    gn_channels<VEC>(a.gamma, c, 1.f, ga);
    gn_channels<VEC>(a.beta, c, 0.f, be);
    const int64_t base = t.row0 * a.C + c;
    auto load = [&](int i) { return V::load(a.x, base + (int64_t)i * a.C); };
    constexpr int U = gn_ahead(VEC, 4);
    GnRows<U, typename V::Raw> rows{row, R, row < R ? t.rows : 0};
    if (rows.rows) rows.ask(row, rows.u, load);
    gn_join_all(a, t, tile_rows, first, s_stat, [&](GnGroup& g) { return gn_join_stat(g, t.n, tile_rows, w, a.eps); });
    __syncthreads();
    if (t.first && a.stat)
        for (int g = threadIdx.x; g < a.G; g += kGnThreads) ((float2*)a.stat)[(int64_t)t.b * a.G + g] = s_stat[g];
    if (row >= R) return;  // whole blocks of 32 channels
    float mu[VEC];
    gn_of_groups<VEC>(a.sh, s_stat, c, [&](int e, const float2& st) { mu[e] = st.x, ga[e] *= st.y; });
    rows.run(load, [&](int i0, const typename V::Raw(&u)[U]) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (i0 + k * R >= t.rows) break;
            const int64_t e = base + (int64_t)(i0 + k * R) * a.C;
            float x[VEC], y[VEC];
            V::unpack(u[k], x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) y[j] = act_of<ACT>(fmaf(x[j] - mu[j], ga[j], be[j]));
            V::store(a.out, e, y);
            if constexpr (CODE) {
                uint32_t w8[VEC / 4];
                const int byte = code_block<DT, VEC, kCodeBlock / VEC>(x, w8);
                int8_t* q = a.saved.codes + e;
                if constexpr (VEC == 8) *(uint2*)q = make_uint2(w8[0], w8[1]);
                else *(uint32_t*)q = w8[0];
                if (c % kCodeBlock == 0) a.saved.exps[e / kCodeBlock] = (uint8_t)byte;
            }
        }
    });
}

// what a thread's channels of the backward need of a row's dy and x (or its codes)
template <int DT, int VEC, bool X8>
struct GnSource {
    using V = Chans<DT, VEC>;
    using RawX = std::conditional_t<X8, typename Codes<VEC>::Raw, typename V::Raw>;
    struct Raw {
        typename V::Raw dy;
        RawX x;
    };
    struct RawRes : Raw {
        typename V::Raw res;
    };
    // row i of a tile, from the elements and blocks of its first row
    static __device__ Raw load(const GnArgs& a, int64_t base, int64_t block, int i) {
        const int64_t e = base + (int64_t)i * a.C;
        Raw r;
        r.dy = V::load(a.dy, e);
        if constexpr (X8) r.x = Codes<VEC>::load(a.saved, e, block + (int64_t)i * code_blocks(a.C));
        else r.x = V::load(a.x, e);
        return r;
    }
    static __device__ void unpack(const RawX& r, float (&x)[VEC]) {
        if constexpr (X8) Codes<VEC>::unpack(r, x);
        else V::unpack(r, x);
    }
};

// Mean and r of a thread's channels.  Both kernels form x - mean first, as the forward does: it is 0 where a group's values
// are equal, and z is beta there.  (x r - mean r in one step leaves the rounding of mean r instead, of either sign, and
// ReLU then lets half of such groups' gradients through.)
template <int VEC>
__device__ inline void gn_stat(const GnArgs& a, int b, int c, float (&mu)[VEC], float (&r)[VEC]) {
    gn_of_groups<VEC>(a.sh, (const float2*)a.stat + (int64_t)b * a.G, c,
                      [&](int e, const float2& st) { mu[e] = st.x, r[e] = st.y; });
}

// a tile's sums of gz and gz xh, of each channel and (times gamma) of each group
template <int DT, int VEC, int ACT, bool X8>
__global__ __launch_bounds__(kGnThreads) void k_gn_tile_sums(GnArgs a, int tile_rows) {
    using V = Chans<DT, VEC>;
    using S = GnSource<DT, VEC, X8>;
    constexpr int N = kGnThreads * VEC;
    __shared__ float s_sum[2 * N];  // [gz, gz xh][R][C]
    const GnThread<VEC> th(a.sh);
    const int R = a.sh.R, row = th.row, c = th.c, w = a.sh.w;
    const GnTile t = gn_tile(a, tile_rows, blockIdx.x);
    float* cols = a.part + (int64_t)blockIdx.x * 2 * a.C;
    if (t.rows == 0) {  // the join of the channels takes every tile
        for (int c = threadIdx.x; c < 2 * a.C; c += kGnThreads) cols[c] = 0.f;
        return;
    }
    if (row < R) {
        float mu[VEC], r[VEC], gr[VEC], be[VEC], s1[VEC], s2[VEC];
        const int64_t base = t.row0 * a.C + c, block = t.row0 * code_blocks(a.C) + c / kCodeBlock;
        auto load = [&](int i) { return S::load(a, base, block, i); };
        constexpr int U = gn_ahead(VEC, 2);
        GnRows<U, typename S::Raw> rows{row, R, t.rows};
        rows.ask(row, rows.u, load);
        gn_channels<VEC>(a.gamma, c, 1.f, gr);
        gn_channels<VEC>(a.beta, c, 0.f, be);
        gn_stat<VEC>(a, t.b, c, mu, r);
#pragma unroll
        for (int e = 0; e < VEC; ++e) gr[e] *= r[e], s1[e] = s2[e] = 0.f;
        rows.run(load, [&](int i0, const typename S::Raw(&u)[U]) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (i0 + k * R >= t.rows) break;
                float x[VEC], d[VEC];
                V::unpack(u[k].dy, d);
                S::unpack(u[k].x, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float dev = x[e] - mu[e], gz = act_grad<ACT>(d[e], fmaf(dev, gr[e], be[e]));
                    s1[e] += gz;
                    s2[e] = fmaf(gz, dev, s2[e]);
                }
            }
        });
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            s_sum[row * a.C + c + e] = s1[e];
            s_sum[N + row * a.C + c + e] = s2[e] * r[e];  // r once a channel
        }
    }
    __syncthreads();
    // a column of R numbers by as many threads as there are, each every so many rows; a thread writes to a row of its own
    const int parts = a.sh.parts;
    for (int j = threadIdx.x; j < 2 * a.C * parts; j += kGnThreads) {
        const int p = over(j, a.sh.by_cols), k = j - p * 2 * a.C;
        float* v = s_sum + (k < a.C ? k : N + k - a.C);
        float u = 0.f;
        for (int i = p; i < R; i += parts) u += v[i * a.C];
        v[p * a.C] = u;
        if (parts == 1) cols[k] = u;
    }
    __syncthreads();
    if (parts > 1) {
        for (int k = threadIdx.x; k < 2 * a.C; k += kGnThreads) {
            float* v = s_sum + (k < a.C ? k : N + k - a.C);
            float u = v[0];
            for (int i = 1; i < parts; ++i) u += v[i * a.C];
            v[0] = u;
            cols[k] = u;
        }
        __syncthreads();
    }
    const int lane = threadIdx.x & 63;
    for (int g = threadIdx.x >> 6; g < a.G; g += kGnWaves) {
        float p = 0.f, q = 0.f;
        for (int j = g * w + lane; j < (g + 1) * w; j += 64) {
            const float gj = a.gamma ? a.gamma[j] : 1.f;
            p = fmaf(gj, s_sum[j], p);
            q = fmaf(gj, s_sum[N + j], q);
        }
        p = lanes_sum<64>(p);
        q = lanes_sum<64>(q);
        if (lane == 0) a.tiles[(int64_t)blockIdx.x * a.G + g] = make_float2(p, q);
    }
}

// dbeta and dgamma: 16 of the 2 C columns of the tiles' sums a workgroup, in runs of consecutive tiles, in 64 bits
__device__ inline void gn_join_channels(const GnArgs& a, int64_t tiles, int which) {
    constexpr int RUNS = kGnThreads / 16;
    __shared__ double red[RUNS][17];
    const int col = threadIdx.x & 15, run = threadIdx.x >> 4, j = which * 16 + col;
    const int64_t len = (tiles + RUNS - 1) / RUNS, t0 = run * len, t1 = t0 + len < tiles ? t0 + len : tiles;
    double s = 0.0;
    if (j < 2 * a.C)
        for (int64_t t = t0; t < t1; t += 8) {
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = t + k < t1 ? a.part[(t + k) * 2 * a.C + j] : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) s += (double)f[k];
        }
    red[run][col] = s;
    __syncthreads();
    if (run || j >= 2 * a.C) return;
    for (int k = 1; k < RUNS; ++k) s += red[k][col];
    float* out = j < a.C ? a.dbeta : a.dgamma;
    if (out) out[j < a.C ? j : j - a.C] = (float)s;
}

__global__ __launch_bounds__(kGnThreads) void k_gn_channels(GnArgs a, int64_t tiles) {
    gn_join_channels(a, tiles, (int)blockIdx.x);
}

// the rows' second pass: dx; the first workgroups join the channels
// (128 registers: room for the joins' workgroups beside those of the tiles)
template <int DT, int VEC, int ACT, bool X8>
__global__ __launch_bounds__(kGnThreads, 4) void k_gn_tile_dx(GnArgs a, int tile_rows, int64_t tiles, unsigned join) {
    using V = Chans<DT, VEC>;
    using S = GnSource<DT, VEC, X8>;
    if (blockIdx.x < join) {
        gn_join_channels(a, tiles, (int)blockIdx.x);
        return;
    }
    __shared__ float2 s_mean[kGnThreads * VEC];
    const GnThread<VEC> th(a.sh);
    const int R = a.sh.R, row = th.row, c = th.c, w = a.sh.w;
    const GnTile t = gn_tile(a, tile_rows, blockIdx.x - join);
    if (t.rows == 0) return;
    GnGroup first(a, (int)threadIdx.x / (a.few_tiles ? 8 : 64), t.tile0, a.joined ? 0u : t.n, tile_rows);
    const int64_t base = t.row0 * a.C + c, block = t.row0 * code_blocks(a.C) + c / kCodeBlock;
    auto load = [&](int i) {
        typename S::RawRes r;
        (typename S::Raw&)r = S::load(a, base, block, i);
        if (a.dres) r.res = V::load(a.dres, base + (int64_t)i * a.C);
        return r;
    };
    constexpr int U = gn_ahead(VEC, 2);
    GnRows<U, typename S::RawRes> rows{row, R, row < R ? t.rows : 0};
    float mu[VEC], r[VEC], ga[VEC], be[VEC], m1[VEC], m2[VEC];
    if (row < R) rows.ask(row, rows.u, load);
    gn_channels<VEC>(a.gamma, c, 1.f, ga);
    gn_channels<VEC>(a.beta, c, 0.f, be);
    gn_stat<VEC>(a, t.b, c, mu, r);
    gn_join_all(a, t, tile_rows, first, s_mean, [&](GnGroup& g) { return gn_join_sums(g, t.n, w); });
    __syncthreads();
    if (row >= R) return;
    gn_of_groups<VEC>(a.sh, s_mean, c, [&](int e, const float2& me) { m1[e] = me.x, m2[e] = me.y; });
    rows.run(load, [&](int i0, const typename S::RawRes(&u)[U]) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (i0 + k * R >= t.rows) break;
            float x[VEC], d[VEC], q[VEC] = {};
            V::unpack(u[k].dy, d);
            S::unpack(u[k].x, x);
            if (a.dres) V::unpack(u[k].res, q);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float xh = (x[e] - mu[e]) * r[e];
                const float h = act_grad<ACT>(d[e], fmaf(xh, ga[e], be[e])) * ga[e];
                d[e] = fmaf(r[e], fmaf(-xh, m2[e], h - m1[e]), q[e]);
            }
            V::store(a.dx, base + (int64_t)(i0 + k * R) * a.C, d);
        }
    });
}

// ---------------------------------------------------------------------------
// Few rows: a workgroup takes a group of a scan, all of it in its threads' registers: the mean, the deviations from
// it and the output in one launch.
// ---------------------------------------------------------------------------
constexpr int kGnFewThreads = 512;
constexpr int kGnHeld = 24;  // values a thread holds
// values in all up to which that is done: 701 x 96 in a graph takes 6.9 us in float32 with 8 groups (7.5 in tiles), in bf16
// with 8 groups 9.2 (8.0: a thread's 17 loads of 2 bytes wait for each other) and with 96 groups 4.5 (13.6); 8000 x 32
// with 32 groups, whose rows are then read 4 bytes at a time, 14.4 (10.0)
constexpr int64_t kGnFew = 1 << 17;

__device__ inline float block_sum(float v, float* red) {
    v = lanes_sum<64>(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = red[0];
#pragma unroll
    for (int w = 1; w < kGnFewThreads / 64; ++w) s += red[w];
    return s;
}

template <int DT, int ACT>
__global__ __launch_bounds__(kGnFewThreads) void k_gn_few(GnArgs a, uint32_t by_w) {
    __shared__ float red[2][kGnFewThreads / 64];
    const int b = (int)(blockIdx.x / (unsigned)a.G), g = (int)(blockIdx.x % (unsigned)a.G), w = a.C / a.G;
    const int64_t r0 = clamp_off(a.off[b], a.m), r1 = clamp_off(a.off[b + 1], a.m);
    const int n = r1 > r0 ? (int)(r1 - r0) * w : 0;
    if (n == 0) {
        if (threadIdx.x == 0 && a.stat) ((float2*)a.stat)[blockIdx.x] = make_float2(0.f, 0.f);
        return;
    }
    const int64_t base = r0 * a.C + g * w;
    const float first = ld_feat<DT>(a.x, base);  // equal values give their mean exactly
    float x[kGnHeld];
    int at[kGnHeld], c[kGnHeld];  // from the group's first value: rows * C is at most kGnHeld kGnFewThreads G
    float s = 0.f, q = 0.f;
#pragma unroll
    for (int k = 0; k < kGnHeld; ++k) {
        if (k * kGnFewThreads >= n) break;
        const int t = (int)threadIdx.x + k * kGnFewThreads, i = t < n ? t : 0, r = by_w ? (int)__umulhi((uint32_t)i, by_w) : i;
        c[k] = i - r * w;
        at[k] = r * a.C + c[k];
        x[k] = ld_feat<DT>(a.x, base + at[k]);
    }
#pragma unroll
    for (int k = 0; k < kGnHeld; ++k)
        if ((int)threadIdx.x + k * kGnFewThreads < n) s += x[k] - first;
    const float mu = first + block_sum(s, red[0]) / (float)n;
#pragma unroll
    for (int k = 0; k < kGnHeld; ++k) {
        if ((int)threadIdx.x + k * kGnFewThreads >= n) break;
        x[k] -= mu;
        q = fmaf(x[k], x[k], q);
    }
    const float rd = 1.f / sqrtf(block_sum(q, red[1]) / (float)n + a.eps);
    if (threadIdx.x == 0 && a.stat) ((float2*)a.stat)[blockIdx.x] = make_float2(mu, rd);
#pragma unroll
    for (int k = 0; k < kGnHeld; ++k)
        if ((int)threadIdx.x + k * kGnFewThreads < n)
            st_feat<DT>(a.out, base + at[k],
                        act_of<ACT>(fmaf(x[k] * rd, a.gamma ? a.gamma[g * w + c[k]] : 1.f, a.beta ? a.beta[g * w + c[k]] : 0.f)));
}

// ---------------------------------------------------------------------------
// Rows too wide for a workgroup's threads, by elements: a workgroup takes a group or a channel of a scan, all of its
// rows.  Right, and not meant for many rows: 11,263 x 1028 in bf16 takes 5.3 ms with 4 groups and 21 with one (rows of 1024,
// aligned, 0.02), the backward 0.14.
// ---------------------------------------------------------------------------
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

template <int DT>
__global__ __launch_bounds__(256) void k_gn_stat(GnArgs a) {
    __shared__ double red[256];
    const int w = a.C / a.G;
    for (int64_t u = blockIdx.x; u < (int64_t)a.B * a.G; u += gridDim.x) {
        const int b = (int)(u / a.G), g = (int)(u % a.G);
        const int64_t r0 = clamp_off(a.off[b], a.m), r1 = clamp_off(a.off[b + 1], a.m);
        const int64_t n = r1 > r0 ? (r1 - r0) * w : 0;
        double s = 0.0, q = 0.0;
        for (int64_t t = threadIdx.x; t < n; t += 256) s += (double)ld_feat<DT>(a.x, (r0 + t / w) * a.C + g * w + t % w);
        const double mu = block_sum(s, red) / (double)(n ? n : 1);
        for (int64_t t = threadIdx.x; t < n; t += 256) {
            const double d = (double)ld_feat<DT>(a.x, (r0 + t / w) * a.C + g * w + t % w) - mu;
            q += d * d;
        }
        q = block_sum(q, red);
        if (threadIdx.x) continue;
        const float2 v = n ? make_float2((float)mu, (float)(1.0 / sqrt(q / (double)n + (double)a.eps)))
                           : make_float2(0.f, 0.f);
        a.joined[u] = v;
        if (a.stat) ((float2*)a.stat)[u] = v;
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
            const float2 st = a.joined[(int64_t)b * a.G + c / (a.C / a.G)];
            const float xh = (ld_feat<DT>(a.x, i * a.C + c) - st.x) * st.y;
            st_feat<DT>(a.out, i * a.C + c,
                        act_of<ACT>(fmaf(xh, a.gamma ? a.gamma[c] : 1.f, a.beta ? a.beta[c] : 0.f)));
        }
    }
}

// sum gz and sum gz xh of a channel of a scan: part[b][C][2]
template <int DT, int ACT>
__global__ __launch_bounds__(256) void k_gn_sums(GnArgs a) {
    __shared__ double red[256];
    for (int64_t u = blockIdx.x; u < (int64_t)a.B * a.C; u += gridDim.x) {
        const int b = (int)(u / a.C), c = (int)(u % a.C);
        const int64_t r0 = clamp_off(a.off[b], a.m), r1 = clamp_off(a.off[b + 1], a.m);
        const float2 st = ((const float2*)a.stat)[(int64_t)b * a.G + c / (a.C / a.G)];
        const float g = a.gamma ? a.gamma[c] : 1.f, be = a.beta ? a.beta[c] : 0.f;
        double s1 = 0.0, s2 = 0.0;
        for (int64_t i = r0 + threadIdx.x; i < r1; i += 256) {
            const float xh = (saved_x<DT>(a, i, c) - st.x) * st.y;
            const float gz = act_grad<ACT>(ld_feat<DT>(a.dy, i * a.C + c), fmaf(xh, g, be));
            s1 += (double)gz;
            s2 += (double)gz * xh;
        }
        s1 = block_sum(s1, red);
        s2 = block_sum(s2, red);
        if (threadIdx.x == 0) ((float2*)a.part)[u] = make_float2((float)s1, (float)s2);
    }
}

// a wave takes a group of a scan: the means of h and h xh
__global__ __launch_bounds__(256) void k_gn_groups(GnArgs a) {
    const int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (u >= (int64_t)a.B * a.G) return;
    const int b = (int)(u / a.G), w = a.C / a.G, c0 = (int)(u % a.G) * w;
    const int64_t n = clamp_off(a.off[b + 1], a.m) - clamp_off(a.off[b], a.m);
    double m1 = 0.0, m2 = 0.0;
    for (int c = c0 + (threadIdx.x & 63); c < c0 + w; c += 64) {
        const float2 p = ((const float2*)a.part)[(int64_t)b * a.C + c];
        const float g = a.gamma ? a.gamma[c] : 1.f;
        m1 += (double)g * p.x;
        m2 += (double)g * p.y;
    }
    m1 = lanes_sum(m1, true);
    m2 = lanes_sum(m2, true);
    const double count = n > 0 ? (double)n * (double)w : 1.0;
    if ((threadIdx.x & 63) == 0) a.joined[u] = make_float2((float)(m1 / count), (float)(m2 / count));
}

template <int DT, int ACT>
__global__ __launch_bounds__(256) void k_gn_dx(GnArgs a) {
    const int w = a.C / a.G;
    for (int64_t i = blockIdx.x; i < a.m; i += gridDim.x) {
        const int b = scan_of(a, i);
        if (b < 0) continue;
        for (int c = threadIdx.x; c < a.C; c += 256) {
            const int64_t u = (int64_t)b * a.G + c / w;
            const float2 st = ((const float2*)a.stat)[u], me = a.joined[u];
            const float g = a.gamma ? a.gamma[c] : 1.f, xh = (saved_x<DT>(a, i, c) - st.x) * st.y;
            const float h = act_grad<ACT>(ld_feat<DT>(a.dy, i * a.C + c), fmaf(xh, g, a.beta ? a.beta[c] : 0.f)) * g;
            float d = st.y * (h - me.x - xh * me.y);
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
        const float2 p = ((const float2*)a.part)[(int64_t)b * a.C + c];
        s1 += (double)p.x;
        s2 += (double)p.y;
    }
    if (a.dbeta) a.dbeta[c] = (float)s1;
    if (a.dgamma) a.dgamma[c] = (float)s2;
}

// ---------------------------------------------------------------------------

// Rows of a tile: kGnTiles tiles for a long scan, and 8192 values at least, a few rows a thread.
static int64_t gn_least_rows(int C) { return (8191 + C) / C; }
static int gn_tile_rows(int64_t m, int C) {
    const int64_t few = gn_least_rows(C), many = (m + kGnTiles - 1) / kGnTiles;
    return (int)(few > many ? few : many);
}
static int64_t gn_tiles(int64_t m, int C, int B) { return m / gn_tile_rows(m, C) + B; }
// Room in the workspace: no fewer, and never less for more rows (gn_tiles falls where a tile gets a row more), so that a
// workspace for the largest batch serves every smaller one.
static size_t gn_room(int64_t m, int C, int B) {
    const int64_t t = m / gn_least_rows(C);
    return (size_t)((t < kGnTiles ? t : kGnTiles) + B);
}
// A workgroup joins its scan's tiles itself: up to 32 of them by 8 lanes a group, 64 groups at a time (2000 x 96 in
// 96 groups takes 14.2 us, 23.5 by a wave a group and 15.3 by a launch of its own), more by a wave, up to twice over.
// Beyond, a launch of its own is shorter: 100,000 x 96 in bf16 14.9 against 16.7 us with 8 groups, 18.0 and 17.7 with
// 24, 37.2 and 21.6 with 96.
static bool gn_few_tiles(const GnArgs& a) { return gn_tiles(a.m, a.C, 1) <= 32; }
static bool gn_join_apart(const GnArgs& a) { return !gn_few_tiles(a) && a.G > 2 * kGnWaves; }

// All groups of all scans fit a workgroup's registers each (no scan has more than m rows), and there are few values:
// rows are read a group's channels at a time.  (Whether codes are asked for makes no difference to the other
// outputs.)
static bool gn_few(const GnArgs& a) {
    return a.m * (a.C / a.G) <= (int64_t)kGnHeld * kGnFewThreads && a.m * a.C <= kGnFew && (int64_t)a.B * a.G <= 4096;
}

static uint32_t gn_by(int64_t n) { return n > 1 ? (uint32_t)((((uint64_t)1 << 32) + (uint64_t)n - 1) / (uint64_t)n) : 0u; }
static GnShape gn_shape(int C, int G, int vec) {
    GnShape s{};
    s.nv = C / vec, s.R = kGnThreads / s.nv, s.w = C / G, s.whole = s.w % vec == 0;
    s.unit = 1;
    while (2 * s.unit <= vec && s.w % (2 * s.unit) == 0) s.unit *= 2;
    s.per = s.w / s.unit, s.units = C / s.unit;
    s.parts = kGnThreads / (2 * C);
    s.parts = s.parts < 1 ? 1 : s.parts > s.R ? s.R : s.parts;
    s.by_nv = gn_by(s.nv), s.by_w = gn_by(s.w), s.by_per = gn_by(s.per), s.by_cols = gn_by(2 * C);
    return s;
}

static void gn_ws(Arena& a, GnArgs& t) {
    t.tiles = a.take<float2>(gn_room(t.m, t.C, t.B) * t.G);
    t.joined = a.take<float2>((size_t)t.B * t.G);
}
void plan_group_norm_ws(Arena& a, GnArgs& t) { gn_ws(a, t); }
void plan_group_norm_backward_ws(Arena& a, GnArgs& t) {
    gn_ws(a, t);
    t.part = a.take<float>(gn_room(t.m, t.C, t.B) * 2 * t.C);
}

template <int V>
using Num = std::integral_constant<int, V>;
// f(type, channels a thread, activation); 0 channels: rows too wide for the tiles
template <class F>
static void gn_kinds(const GnArgs& a, F&& f) {
    const bool aligned = (((uintptr_t)a.x | (uintptr_t)a.out | (uintptr_t)a.dy | (uintptr_t)a.dres | (uintptr_t)a.dx) & 15u) == 0;
    auto act = [&](auto dt, auto vec) {
        if (a.act == SPV_ACT_RELU) f(dt, vec, Num<SPV_ACT_RELU>{});
        else if (a.act == SPV_ACT_SILU) f(dt, vec, Num<SPV_ACT_SILU>{});
        else f(dt, vec, Num<SPV_ACT_NONE>{});
    };
    auto wide = [&](auto dt) {
        constexpr int V = kGnVec<decltype(dt)::value>;
        if (aligned && ((uintptr_t)a.saved.codes % V) == 0 && a.C % V == 0 && a.C / V <= kGnThreads) act(dt, Num<V>{});
        else if (a.C <= kGnThreads) act(dt, Num<1>{});
        else act(dt, Num<0>{});
    };
    if (a.dt == SPV_F32) wide(Num<SPV_F32>{});
    else if (a.dt == SPV_BF16) wide(Num<SPV_BF16>{});
    else wide(Num<SPV_F16>{});
}
static unsigned gn_grid(int64_t n) { return (unsigned)(n < 1 ? 1 : n > 65536 ? 65536 : n); }

void launch_group_norm(hipStream_t s, const GnArgs& given) {
    gn_kinds(given, [&](auto dt, auto vec, auto act) {
        constexpr int DT = decltype(dt)::value, VEC = decltype(vec)::value, ACT = decltype(act)::value;
        GnArgs a = given;
        const bool code = VEC > 1 && a.C % kCodeBlock == 0 && a.saved.codes && !gn_few(a);
        // before out, which may be x
        if (a.saved.codes && !code && a.m)
            launch_checkpoint8(s, a.x, a.saved, RowRange{a.m, nullptr, a.off, a.B}, a.C, a.dt);
        if (gn_few(a)) {
            const int w = a.C / a.G;
            k_gn_few<DT, ACT><<<(unsigned)(a.B * a.G), kGnFewThreads, 0, s>>>(a, gn_by(w));
            return;
        }
        if constexpr (VEC == 0) {
            k_gn_stat<DT><<<gn_grid((int64_t)a.B * a.G), 256, 0, s>>>(a);
            if (a.m) k_gn_apply<DT, ACT><<<gn_grid(a.m), 256, 0, s>>>(a);
        } else {
            a.sh = gn_shape(a.C, a.G, VEC);
            const int rows = gn_tile_rows(a.m, a.C);
            const unsigned tiles = (unsigned)gn_tiles(a.m, a.C, a.B);
            a.few_tiles = gn_few_tiles(a);
            k_gn_tile_stat<DT, VEC><<<tiles, kGnThreads, 0, s>>>(a, rows);
            if (gn_join_apart(a)) k_gn_join<true><<<(unsigned)(((int64_t)a.B * a.G + 3) / 4), 256, 0, s>>>(a, rows);
            else a.joined = nullptr;
            if constexpr (VEC > 1) {
                if (code) {
                    k_gn_tile_apply<DT, VEC, ACT, true><<<tiles, kGnThreads, 0, s>>>(a, rows);
                    return;
                }
            }
            k_gn_tile_apply<DT, VEC, ACT, false><<<tiles, kGnThreads, 0, s>>>(a, rows);
        }
    });
}

template <int DT, int VEC, int ACT, bool X8>
static void gn_backward_tiles(hipStream_t s, GnArgs a) {
    const int rows = gn_tile_rows(a.m, a.C);
    const int64_t tiles = gn_tiles(a.m, a.C, a.B);
    a.few_tiles = gn_few_tiles(a);
    a.sh = gn_shape(a.C, a.G, VEC);
    const unsigned join = a.dgamma || a.dbeta ? (unsigned)((2 * a.C + 15) / 16) : 0;
    k_gn_tile_sums<DT, VEC, ACT, X8><<<(unsigned)tiles, kGnThreads, 0, s>>>(a, rows);
    if (a.dx && gn_join_apart(a)) k_gn_join<false><<<(unsigned)(((int64_t)a.B * a.G + 3) / 4), 256, 0, s>>>(a, rows);
    else a.joined = nullptr;
    if (a.dx) k_gn_tile_dx<DT, VEC, ACT, X8><<<(unsigned)tiles + join, kGnThreads, 0, s>>>(a, rows, tiles, join);
    else k_gn_channels<<<join, kGnThreads, 0, s>>>(a, tiles);
}
void launch_group_norm_backward(hipStream_t s, const GnArgs& a) {
    if (a.B == 0) {
        if (a.dgamma || a.dbeta) k_gn_params<<<(unsigned)((a.C + 255) / 256), 256, 0, s>>>(a);
        return;
    }
    gn_kinds(a, [&](auto dt, auto vec, auto act) {
        constexpr int DT = decltype(dt)::value, VEC = decltype(vec)::value, ACT = decltype(act)::value;
        if constexpr (VEC == 0) {
            k_gn_sums<DT, ACT><<<gn_grid((int64_t)a.B * a.C), 256, 0, s>>>(a);
            if (a.dgamma || a.dbeta) k_gn_params<<<(unsigned)((a.C + 255) / 256), 256, 0, s>>>(a);
            if (!a.dx || !a.m) return;
            k_gn_groups<<<(unsigned)(((int64_t)a.B * a.G + 3) / 4), 256, 0, s>>>(a);
            k_gn_dx<DT, ACT><<<gn_grid(a.m), 256, 0, s>>>(a);
        } else if (a.x || !a.saved.codes) {
            gn_backward_tiles<DT, VEC, ACT, false>(s, a);
        } else {
            gn_backward_tiles<DT, VEC, ACT, true>(s, a);
        }
    });
}

}  // namespace spv
