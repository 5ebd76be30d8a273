// attn_common.hpp -- what the attention kernels share: matrix-core tiles of 32 rows by 32 columns, the staging of
// rows in LDS, the scans' ranges and the scores.
//
// A wave owns 32 columns, one to each pair of lanes (c, c + 32), and takes 32 rows at a time from LDS as the A
// operand.  The accumulator of a tile holds, in lane (c, h), rows 8 (i / 4) + 4 h + i % 4 of column c (i = 0 .. 15):
// sums and maxima down a column stay in a lane and one exchange between the halves.  Those same registers are the
// B operand of the product that follows (weights times values): the k index of a product may be numbered in any
// order as long as both operands agree, so k slot (h, j) is given the row that lane half h already holds, and the A
// operand is gathered to match by transposing LDS reads (16-bit types: ds_read_b64_tr_b16 hands each lane four
// rows of one channel) or plain ones (float32).  Weights never move between lanes.
#pragma once

#include "conv_common.hpp"

namespace spv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ inline int64_t clamp_off(int32_t o, int64_t n) { return o < 0 ? 0 : ((int64_t)o > n ? n : (int64_t)o); }

// a uniform value in a vector register: float32 arithmetic on vector registers alone runs at 2.7 cycles a wave, with a
// scalar operand at 4
__device__ inline float in_vgpr(float v) {
    asm("" : "+v"(v));
    return v;
}
// wave-uniform values, in scalar registers
__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ inline int64_t uniform(int64_t v) {
    return (int64_t)(((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32) | (uint32_t)uniform((int)v));
}

// The tiles of a side: scan b's rows * per columns are cut into tiles of BM from its own start, and its first tile
// is number floor(off[b] * per / BM) + b: ascending in b, with room for every scan's tiles and known without a
// pass over the scans.  attn_tiles bounds their number.
__device__ inline int64_t scan_tile(int32_t off, int b, int64_t n, int per, int BM) {
    return clamp_off(off, n) * per / BM + b;
}
inline int64_t attn_tiles(int64_t n, int B, int per, int BM) { return n * per / BM + B; }

// What a workgroup takes: a key head, a tile of columns and one of `parts` shares of the rows.  In one part the heads
// come first in the grid, so that the eight dies (which take workgroups in turn) each keep to few heads' rows in
// their L2.  In parts those come first: the heads of one part, which share its cache lines, then run on one die.
struct Share {
    int kh, part, parts;
    int64_t tile;
};
__device__ inline Share attn_share(const AttnArgs& a) {
    if (a.part) return Share{(int)blockIdx.y, (int)blockIdx.x, (int)gridDim.x, (int64_t)blockIdx.z};
    return Share{(int)(blockIdx.x % (unsigned)a.K), 0, 1, (int64_t)(blockIdx.x / (unsigned)a.K)};
}

struct ScanTile {
    int b;           // scan
    int64_t first;   // its first row
    int64_t cols;    // its columns (rows * per)
    int64_t col0;    // the tile's first column; at least cols: nothing to do
    int64_t r0, r1;  // the scan's rows of the other side
};
// The scan of tile t, by a search with 63 intervals a step.  Both sides' offsets are read in the same step and handed
// over between lanes: one wait for memory (up to 63 scans) before the rows themselves can be asked for.
__device__ inline ScanTile find_tile(const int32_t* off, int64_t n, const int32_t* other, int64_t n_other, int B, int per,
                                     int BM, int64_t t) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = B, step, k, o, r;
    do {
        step = (hi - lo + 62) / 63;
        const int at = lo + step * lane;
        o = r = 0;
        if (at <= hi) o = off[at], r = other[at];
        k = __popcll(__ballot(at < hi && scan_tile(o, at, n, per, BM) <= t));
        k = uniform(k > 0 ? k - 1 : 0);
        lo += step * k;
        hi = lo + step < hi ? lo + step : hi;
    } while (step > 1);
    ScanTile s;
    s.b = uniform(lo);
    const int32_t first = __builtin_amdgcn_readlane(o, k);
    s.first = clamp_off(first, n);
    const int64_t end = clamp_off(__builtin_amdgcn_readlane(o, k + 1), n), mine = t - scan_tile(first, s.b, n, per, BM);
    s.cols = end > s.first ? (end - s.first) * per : 0;
    s.col0 = mine >= 0 ? mine * BM : s.cols;
    s.r0 = clamp_off(__builtin_amdgcn_readlane(r, k), n_other);
    s.r1 = clamp_off(__builtin_amdgcn_readlane(r, k + 1), n_other);
    return s;
}

// The voxels' L1 distance.  Coordinates are 16 bits each: two words, and a distance is two sums of absolute differences
// onto the bits of 2^23, which read as a float are 2^23 + distance.  Where a workgroup's columns and 32 rows lie in one
// cube of 256 voxels a side (most do: a scan at a coarse stride is hardly wider), three bytes of one word hold a
// voxel's place in it, and one sum does.
constexpr uint32_t kDistBits = 0x4B000000u;  // 2^23
__device__ inline int voxel_coord(int c) { return c < kCoordMin ? kCoordMin : (c > kCoordMax ? kCoordMax : c); }
struct Cube {
    int x, y, z;  // lowest corner
    bool any;     // the columns fit in it
    // the word of a place in the cube (coordinates in the voxel range); false: it is outside
    __device__ bool place(const int4& c, uint32_t& w) const {
        const uint32_t dx = c.y - x, dy = c.z - y, dz = c.w - z;
        w = dx | (dy << 8) | (dz << 16);
        return any && (dx | dy | dz) < 256u;
    }
};
struct Words {
    uint32_t a, b;  // x | y << 16 and z, from 2^15 below zero; or the place in the cube
};
__device__ inline int4 voxel_clamp(const int4& c) {
    return make_int4(c.x, voxel_coord(c.y), voxel_coord(c.z), voxel_coord(c.w));
}
__device__ inline Words voxel_words(const int4& c) {
    return Words{(uint32_t)(c.y + 32768) | ((uint32_t)(c.z + 32768) << 16), (uint32_t)(c.w + 32768)};
}
// The cube around a workgroup's columns (one to each lane; both halves of a wave hold the same), with equal margins:
// every thread of its NW waves calls it.
template <int NW>
__device__ inline Cube columns_cube(const int4& c, bool live, uint32_t (&lds)[NW][3]) {
    // the lowest of x, y, z, -x, -y, -z, two to a word
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    auto two = [&](int a, int b) { return live ? i16x2{(short)a, (short)b} : i16x2{32767, 32767}; };
    i16x2 v[3] = {two(c.y, c.z), two(c.w, -c.y), two(-c.z, -c.w)};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        i16x2 w[3];
#pragma unroll
        for (int e = 0; e < 3; ++e) w[e] = __builtin_bit_cast(i16x2, __shfl_xor(__builtin_bit_cast(int, v[e]), o, 64));
#pragma unroll
        for (int e = 0; e < 3; ++e) v[e] = __builtin_elementwise_min(v[e], w[e]);
    }
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int e = 0; e < 3; ++e) lds[threadIdx.x >> 6][e] = __builtin_bit_cast(uint32_t, v[e]);
    __syncthreads();
    int m[6];
#pragma unroll
    for (int e = 0; e < 3; ++e) {
        i16x2 t = __builtin_bit_cast(i16x2, lds[0][e]);
#pragma unroll
        for (int w = 1; w < NW; ++w) t = __builtin_elementwise_min(t, __builtin_bit_cast(i16x2, lds[w][e]));
        m[2 * e] = uniform((int)t.x);
        m[2 * e + 1] = uniform((int)t.y);
    }
    Cube q;
    int lo[3];
    q.any = true;
#pragma unroll
    for (int e = 0; e < 3; ++e) {
        const int span = -m[3 + e] - m[e];
        q.any = q.any && span < 256;
        lo[e] = m[e] - (255 - span) / 2;
    }
    q.x = lo[0], q.y = lo[1], q.z = lo[2];
    return q;
}
// The words of KT rows in LDS, one row a thread (tid < KT): those of the cube where all rows of its 32 lie in it.
template <int KT>
struct Places {
    uint32_t w[2][2][KT];
    uint32_t near[2][KT / 32];  // of each 32 rows
    __device__ inline void put(int s, int tid, const int4& raw, bool in, const Cube& cube) {
        const int4 c = voxel_clamp(raw);
        uint32_t p;
        const bool ok = cube.place(c, p) || !in;
        const uint64_t all = __ballot(ok);
        const bool near = (uint32_t)(all >> (tid & 32)) == 0xFFFFFFFFu;
        const Words f = voxel_words(c);
        w[s][0][tid] = near ? p : f.a;
        w[s][1][tid] = f.b;
        if ((tid & 31) == 0) this->near[s][tid >> 5] = near;
    }
    // f(r, -slope * distance) for the lane's 16 of the 32 rows from row0, from the column's words; lift is what the 2^23
    // of a distance brings too much: slope 2^23, so that the sum is rounded once
    template <class F>
    __device__ inline void bias(int s, int row0, int h, const Words& far, uint32_t place, float slope, float lift,
                                F&& f) const {
        const uint32_t *wa = &w[s][0][row0 + 4 * h], *wb = &w[s][1][row0 + 4 * h];
        if (uniform((int)near[s][row0 >> 5])) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 v = *(const uint4*)(wa + 8 * q);
                const uint32_t a[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    f(4 * q + e, fmaf(__uint_as_float(__builtin_amdgcn_sad_u8(a[e], place, kDistBits)), -slope, lift));
            }
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 v = *(const uint4*)(wa + 8 * q), y = *(const uint4*)(wb + 8 * q);
                const uint32_t a[4] = {v.x, v.y, v.z, v.w}, z[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    f(4 * q + e, fmaf(__uint_as_float(__builtin_amdgcn_sad_u16(
                                          z[e], far.b, __builtin_amdgcn_sad_u16(a[e], far.a, kDistBits))),
                                      -slope, lift));
            }
        }
    }
};

// the other half's value of a column: (max, sum) over both
__device__ inline f32x2 both_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ inline float half_sum(float v) {
    const f32x2 r = both_halves(v);
    return r.x + r.y;
}
__device__ inline float half_max(float v) {
    const f32x2 r = both_halves(v);
    return fmaxf(r.x, r.y);
}

template <int DT>
__device__ inline f32x16 mfma32x32x16(uint4 a, uint4 b, f32x16 c) {
    if constexpr (DT == SPV_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
}

// Rows of up to DP channels (a multiple of 32; D <= DP of them real, the rest zero) in LDS, and products with them.
template <int DT, int DP>
struct Tile {
    static constexpr bool W = DT == SPV_F32;
    static constexpr int SZ = W ? 4 : 2;       // bytes of an element
    static constexpr int E = 16 / SZ;          // elements of 16 bytes
    static constexpr int LD = DP * SZ + 16;    // bytes from row to row: 16 of padding spread the rows over the banks
    static constexpr int NF = DP / (2 * E);    // 16-byte fragments of a row that a lane holds
    static constexpr int CH = DP / E;          // 16-byte chunks of a row
    static constexpr int NB = DP / 32;         // blocks of 32 channels

    // B operand: a lane's fragments of its column's row (channels 2 E s + E h ..), zeros past D
    static __device__ inline void load_cols(const void* p, int64_t at, bool live, int D, int h, uint4 (&f)[NF]) {
#pragma unroll
        for (int s = 0; s < NF; ++s) {
            const int d = 2 * E * s + E * h;
            f[s] = live && d < D ? *(const uint4*)((const char*)p + (at + d) * SZ) : make_uint4(0, 0, 0, 0);
        }
    }

    // c + rows (32 of them, at lds) . columns
    static __device__ inline f32x16 rows_dot(const char* lds, int lane, const uint4 (&f)[NF], f32x16 c) {
        const char* a = lds + (lane & 31) * LD + (lane >> 5) * 16;
#pragma unroll
        for (int s = 0; s < NF; ++s) {
            const uint4 x = *(const uint4*)(a + 32 * s), y = f[s];
            if constexpr (W) {
                c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x.x), __uint_as_float(y.x), c, 0, 0, 0);
                c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x.y), __uint_as_float(y.y), c, 0, 0, 0);
                c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x.z), __uint_as_float(y.z), c, 0, 0, 0);
                c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x.w), __uint_as_float(y.w), c, 0, 0, 0);
            } else {
                c = mfma32x32x16<DT>(x, y, c);
            }
        }
        return c;
    }

    // the weights of 32 rows (accumulator registers) as B operands
    struct Weights {
        uint4 f[W ? 4 : 2];
    };
    // the dot product of two fragments' channels, added to s
    static __device__ inline float frag_dot(const uint4& a, const uint4& b, float s) {
        const uint32_t u[4] = {a.x, a.y, a.z, a.w}, v[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (W) {
                s = fmaf(__uint_as_float(u[e]), __uint_as_float(v[e]), s);
            } else {
                s = fmaf(from16<DT>(u[e] & 0xFFFF), from16<DT>(v[e] & 0xFFFF), s);
                s = fmaf(from16<DT>(u[e] >> 16), from16<DT>(v[e] >> 16), s);
            }
        }
        return s;
    }
    static __device__ inline Weights weights(const f32x16& p) {
        Weights w;
        if constexpr (W) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
                w.f[t] = make_uint4(__float_as_uint(p[4 * t]), __float_as_uint(p[4 * t + 1]),
                                    __float_as_uint(p[4 * t + 2]), __float_as_uint(p[4 * t + 3]));
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
                w.f[t] = make_uint4(pack2<DT>(p[8 * t], p[8 * t + 1]), pack2<DT>(p[8 * t + 2], p[8 * t + 3]),
                                    pack2<DT>(p[8 * t + 4], p[8 * t + 5]), pack2<DT>(p[8 * t + 6], p[8 * t + 7]));
        }
        return w;
    }
    // s + the sum of the lane's 16 weights as they are multiplied
    static __device__ inline float sum(const Weights& w, float s) {
#pragma unroll
        for (int t = 0; t < (W ? 4 : 2); ++t) {
            const uint32_t u[4] = {w.f[t].x, w.f[t].y, w.f[t].z, w.f[t].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (W)
                    s += __uint_as_float(u[e]);
                else if constexpr (DT == SPV_BF16)
                    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, u[e]),
                                                        __builtin_bit_cast(bf16x2, 0x3F803F80u), s, false);
                else
                    s = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, u[e]), __builtin_bit_cast(f16x2, 0x3C003C00u),
                                               s, false);
            }
        }
        return s;
    }

    // o[b] + (channels 32 b .. 32 b + 31 of the 32 rows at lds, transposed) . weights: lane (c, h) of o[b] holds
    // channels 32 b + 8 (i / 4) + 4 h + i % 4 of column c
    // (16-bit types: o2 the same with weights w2, of the same reads)
    static __device__ inline void add_weighted(const char* lds, int lane, const Weights& w, f32x16 (&o)[NB],
                                               const Weights* w2 = nullptr, f32x16* o2 = nullptr) {
        if constexpr (W) {
            const char* a = lds + (lane >> 5) * 4 * LD + (lane & 31) * 4;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t u[4] = {w.f[i / 4].x, w.f[i / 4].y, w.f[i / 4].z, w.f[i / 4].w};
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(*(const float*)(a + (8 * (i / 4) + i % 4) * LD + 128 * b),
                                                                __uint_as_float(u[i % 4]), o[b], 0, 0, 0);
            }
        } else {
            typedef short i16x8 __attribute__((ext_vector_type(8)));
            typedef __attribute__((address_space(3))) i16x4 lds4;
            // lanes 16 g .. 16 g + 15 read four rows of 16 channels, and each gets its channel of the four
            const int t = lane & 15, g = lane >> 4;
            const uint32_t a = lds_addr(lds) + (4 * (g >> 1) + (t >> 2)) * LD + (16 * (g & 1) + 4 * (t & 3)) * 2;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(a + 16 * k * LD + 64 * b));
                    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(a + (16 * k + 8) * LD + 64 * b));
                    const i16x8 x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    o[b] = mfma32x32x16<DT>(__builtin_bit_cast(uint4, x), w.f[k], o[b]);
                    if (w2) o2[b] = mfma32x32x16<DT>(__builtin_bit_cast(uint4, x), w2->f[k], o2[b]);
                }
        }
    }

    // a lane's sums of its column, times f, to channels of row `at` (elements) of dst
    static __device__ inline void store_cols(void* dst, int64_t at, int D, int h, const f32x16 (&o)[NB], float f) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int d = 32 * b + 8 * q + 4 * h;
                if (d >= D) continue;
                char* p = (char*)dst + (at + d) * SZ;
                if constexpr (W)
                    *(float4*)p = make_float4(o[b][4 * q] * f, o[b][4 * q + 1] * f, o[b][4 * q + 2] * f,
                                              o[b][4 * q + 3] * f);
                else
                    *(uint2*)p = make_uint2(pack2<DT>(o[b][4 * q] * f, o[b][4 * q + 1] * f),
                                            pack2<DT>(o[b][4 * q + 2] * f, o[b][4 * q + 3] * f));
            }
    }
};

// Scores under a cap, cap tanh(w) with w = scale z / cap, and 4 / kBend of their slope 1 - tanh(w)^2.
// kCapQuick: tanh(w) = 1 - 2 r, r = 1 / (exp(2 w) + 1), slope 4 (r - r^2).  Near zero it cancels: a score is off by 2^-22
// cap whatever its size.  In 16-bit types that is 1.5e-5 at a cap of 64, a thirtieth of float16's half step; in float32
// 2e-6 at 8, as much as the other roundings of a score (cap 5, [1457, 1544] x 3 heads: out is off by 4.5e-7, as by 4.7e-7
// with the exact form, and a training step takes 175 us, 208 with that).
// kCapExact, for larger caps: with e = exp(-2 |w|), |tanh(w)| = (1 - e) / (1 + e) and slope 4 e / (1 + e)^2; below a
// quarter, where 1 - e cancels, an odd polynomial (through three nodes of Chebyshev's in w^2; 1e-8).  Off by 5 2^-24
// of itself at most, for eleven more instructions a score.
constexpr int kNoCap = 0, kCapQuick = 1, kCapExact = 2;
constexpr float quick_cap(int dt) { return dt == SPV_F32 ? 8.f : 64.f; }
inline int attn_cap(const AttnArgs& a) {
    return !(a.cap > 0.f) ? kNoCap : a.cap <= quick_cap(a.dt) ? kCapQuick : kCapExact;
}
// the bias is added after the product and what a cap makes of it, not what the product is added to
__host__ __device__ constexpr bool attn_after(int dt, bool bias, bool cap) { return cap || (dt == SPV_F32 && bias); }
template <int CAP>
constexpr float kBend = CAP ? 4.f : 1.f;
template <int CAP>
struct Capped {
    float cz, cw, cap2, fall, lift;  // lift: what a score is added to beside its bias
    __device__ explicit Capped(const AttnArgs& a) {
        cw = a.scale / a.cap;
        cz = in_vgpr((CAP == kCapQuick ? 2.f : -2.f) * kLog2e * cw);
        cap2 = a.cap * kLog2e;
        fall = in_vgpr(-2.f * cap2);
        lift = CAP == kCapQuick ? cap2 : 0.f;
    }
    // the score of product z in units of log 2, added to rest (which has lift in it)
    __device__ float operator()(float z, float rest, float* bend = nullptr) const {
        if constexpr (CAP == kCapQuick) {
            const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z * cz) + 1.f);
            if (bend) *bend = fmaf(-r, r, r);
            return fmaf(fall, r, rest);
        } else {
            const float w = z * cw, v = w * w, e = __builtin_amdgcn_exp2f(fabsf(z) * cz);
            const float r = __builtin_amdgcn_rcpf(e + 1.f);
            const float low = fmaf(w * v, fmaf(v, fmaf(v, -0.05197494f, 0.13328699f), -0.33333317f), w);
            const float t = fabsf(w) < 0.25f ? low : copysignf((1.f - e) * r, w);
            if (bend) *bend = e * r * r;
            return fmaf(t, cap2, rest);
        }
    }
};

// the values of the lane's 16 of 32 rows, from LDS.  A product of the values with ones gives the same without the reads,
// but two of those are a third of a tile's matrix cycles: dk and dv of [3451, 3654, 1963, 2195] x 8 heads of 32, 185 us
// that way, 174 so.
__device__ inline f32x16 row_values(const float* p, int h) {
    f32x16 z;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float4 v = *(const float4*)(p + 8 * q + 4 * h);
        z[4 * q] = v.x, z[4 * q + 1] = v.y, z[4 * q + 2] = v.z, z[4 * q + 3] = v.w;
    }
    return z;
}

// Rows of a scan, KT at a time, as buffers: what lies outside reads as zero.  Scalar state: the next rows' address and
// the bytes of a whole tile.
template <int KT>
struct RowTiles {
    const char* at;
    int64_t step;
    int ld, row;
    __device__ RowTiles() {}
    // of p from row `first` on, ld_bytes apart, row_bytes of each
    __device__ RowTiles(const void* p, int64_t first, int64_t ld_bytes, int row_bytes)
        : at((const char*)p + first * ld_bytes), step(KT * ld_bytes), ld((int)ld_bytes), row(row_bytes) {}
    // the next 1 .. KT of them
    __device__ inline __amdgpu_buffer_rsrc_t next(int rows) {
        const __amdgpu_buffer_rsrc_t r = make_rsrc(at, (uint32_t)(rows - 1) * (uint32_t)ld + (uint32_t)row);
        at += step;
        return r;
    }
};

// KT rows of DP channels on their way from memory to LDS by TH threads: 16 bytes at a time, loaded to registers a tile
// ahead; zeros for rows past the buffer's and channels past D.  The offsets within a tile stay the same.
template <int DT, int DP, int KT, int TH>
struct Stage {
    using T = Tile<DT, DP>;
    static constexpr int RP = TH / T::CH, N = (KT + RP - 1) / RP;  // rows a pass, passes
    uint32_t off[N];
    uint4 u[N];
    __device__ Stage(int tid, int64_t ld, int D) {
        const int r = tid / T::CH, ch = tid % T::CH;
#pragma unroll
        for (int i = 0; i < N; ++i)
            off[i] = r < RP && r + i * RP < KT && ch * T::E < D ? (uint32_t)((r + i * RP) * ld + ch * T::E) * T::SZ
                                                                 : kOutOfRange;
    }
    __device__ inline void load(__amdgpu_buffer_rsrc_t rows) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            u[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rows, off[i], 0, 0));
    }
    __device__ inline void store(char* lds, int tid) const {
        const int r = tid / T::CH, ch = tid % T::CH;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((TH % T::CH == 0 || r < RP) && (KT % RP == 0 || r + i * RP < KT))
                *(uint4*)(lds + (r + i * RP) * T::LD + ch * 16) = u[i];
    }
};

// registers of a wave in LDS, 256 bytes each
template <int N>
__device__ inline void lds_put(float* p, int lane, const f32x16 (&o)[N]) {
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) p[(16 * b + r) * 64 + lane] = o[b][r];
}
template <int N>
__device__ inline void lds_add(const float* p, int lane, float f, f32x16 (&o)[N]) {
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] = fmaf(f, p[(16 * b + r) * 64 + lane], o[b][r]);
}

// The four waves of a workgroup: CW blocks of 32 columns, and KW waves on each that take every KW'th 32 rows of what is
// staged and join at the end.  More waves on fewer columns read the rows more often but leave more workgroups.
// The waves of `mode` 0, 1, 2 on a block of columns; a head too wide for LDS takes the last mode that fits.
constexpr int attn_kw(int dt, int DP, int mode) {
    const int most = (dt == SPV_F32 ? 2 : 1) * DP <= 64 ? 4 : (dt == SPV_F32 ? 2 : 1) * DP <= 128 ? 2 : 1;
    return (1 << mode) < most ? 1 << mode : most;
}
// rows that a wave takes between two barriers
constexpr int attn_rows(int dt, int DP, int KW) { return dt == SPV_F32 || DP > 32 || KW > 1 ? 32 : 64; }

// channels a head's rows are padded to
constexpr int attn_dp(int D) { return (D + 31) / 32 * 32; }

// a launch: mode (above), parts that the rows of a scan are taken in, tiles of columns
struct AttnShape {
    int mode, parts;
    int64_t tiles;
};
inline dim3 attn_grid(const AttnShape& s, int K) {
    return s.parts > 1 ? dim3((unsigned)s.parts, (unsigned)K, (unsigned)s.tiles) : dim3((unsigned)(s.tiles * K));
}
// The fewest waves on a block of columns that leave two waves to each SIMD (kAttnFull).  Where even the most leave a
// compute unit without a workgroup, the rows are also taken in parts, two workgroups to a compute unit, of at least 256
// rows of the average scan.  More parts cost more in joining them than they bring: at [1457, 1544] x 3 heads, float32,
// 51 us in one part, 59 in six; at [2000] x 8 heads, bf16, 26 and 42.
constexpr int64_t kAttnFull = 2048;
inline AttnShape attn_shape(int dt, int DP, int64_t n, int per, int B, int K, int64_t rows) {
    AttnShape s{0, 1, 0};
    for (;; ++s.mode) {
        s.tiles = attn_tiles(n, B, per, 128 / attn_kw(dt, DP, s.mode));
        if (s.mode == 2 || s.tiles * K * 4 >= kAttnFull) break;
    }
    const int64_t wgs = s.tiles * K;
    if (wgs < 256) {
        int64_t p = 512 / (wgs < 1 ? 1 : wgs);
        if (p > rows / 256) p = rows / 256;
        if (p > 256) p = 256;
        if (p > 8) p &= ~(int64_t)7;  // a part's heads on one die
        s.parts = p < 2 ? 1 : (int)p;
    }
    return s;
}
// of a launch, in tiles of 32 columns; a scan's tiles of rows, each once for a key head's query heads, are no more, so
// 32 bits count them
constexpr int64_t kMaxWorkgroups = (int64_t)1 << 22;

}  // namespace spv
