// checkpoint8.hip -- activation checkpoints in 8 bits: rows into codes and back, and the weight gradient of a linear
// layer from codes, dW = in^T da.
#include "attn_common.hpp"
#include "code8.hpp"

namespace spv {

__device__ inline int64_t RowRange::begin() const { return off ? clamp_off(off[0], cap) : 0; }
__device__ inline int64_t RowRange::end() const { return off ? clamp_off(off[B], cap) : clamp_rows(m_dev, cap); }

// Vectors that a thread asks for before it uses the first; of single channels, rows it takes at a time.
constexpr int kCodeAhead = 4;

// Half a wave takes a block of 32 channels of kCodeAhead rows, a lane a channel: any width and alignment.  As compiled, a
// 16-bit value is waited for before the next row's is asked for, and so is a row's exponent on the way back (300,007 x 19
// in bf16 into codes and back 35 us; 17 MB each way, which a copy moves in 3.4).
template <int DT>
__global__ __launch_bounds__(256) void k_code8_any(const void* x, Saved8 to, RowRange rows, int C) {
    const int nb = code_blocks(C), l = threadIdx.x & 31;
    const int64_t end = rows.end(), step = (int64_t)gridDim.x * 8;
    for (int64_t i0 = rows.begin() + (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i0 < end; i0 += kCodeAhead * step)
        for (int b = 0; b < nb; ++b) {
            const int c = b * kCodeBlock + l;
            float v[kCodeAhead];
#pragma unroll
            for (int k = 0; k < kCodeAhead; ++k) {
                const int64_t i = i0 + k * step;
                v[k] = c < C && i < end ? ld_feat<DT>(x, i * C + c) : 0.f;
            }
#pragma unroll
            for (int k = 0; k < kCodeAhead; ++k) {
                const int64_t i = i0 + k * step;
                const int byte = code_exp<DT>(lanes_max<32>(finite_bits(v[k])));
                if (i >= end) break;
                if (c < C) to.codes[i * C + c] = (int8_t)code_of(v[k], code_rate(byte));
                if (l == 0) to.exps[i * nb + b] = (uint8_t)byte;
            }
        }
}
template <int DT>
__global__ __launch_bounds__(256) void k_code8_read_any(Saved8 from, void* out, RowRange rows, int C) {
    const int nb = code_blocks(C), l = threadIdx.x & 31;
    const int64_t end = rows.end(), step = (int64_t)gridDim.x * 8;
    for (int64_t i0 = rows.begin() + (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i0 < end; i0 += kCodeAhead * step)
        for (int b = 0; b < nb; ++b) {
            const int c = b * kCodeBlock + l;
            int q[kCodeAhead], e[kCodeAhead];
#pragma unroll
            for (int k = 0; k < kCodeAhead; ++k) {
                const int64_t i = i0 + k * step;
                const bool on = c < C && i < end;
                q[k] = on ? from.codes[i * C + c] : 0;
                e[k] = on ? from.exps[i * nb + b] : 1;
            }
#pragma unroll
            for (int k = 0; k < kCodeAhead; ++k)
                if (c < C && i0 + k * step < end) st_feat<DT>(out, (i0 + k * step) * C + c, code_value(q[k], code_step(e[k])));
        }
}

// Rows of whole blocks: the blocks of all rows are one after the other.  A thread takes 16 bytes of x, four times
// over.  Bound by memory: 300,007 x 96 in bf16, 57.6 MB and 29.7, take 14.8 us into codes and 14.1 back.
template <int DT>
constexpr int kCodeVec = DT == SPV_F32 ? 4 : 8;

template <int DT>
__global__ __launch_bounds__(256) void k_code8(const void* x, Saved8 to, RowRange rows, int C) {
    constexpr int V = kCodeVec<DT>, LANES = kCodeBlock / V;
    const int64_t per = C / V, end = rows.end() * per;  // vectors
    const int64_t t0 = rows.begin() * per + group_of_grid() * (256 * kCodeAhead) + threadIdx.x;
    uint4 u[kCodeAhead];
#pragma unroll
    for (int k = 0; k < kCodeAhead; ++k) {
        const int64_t t = t0 + k * 256;
        u[k] = t < end ? ((const uint4*)x)[t] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kCodeAhead; ++k) {
        const int64_t t = t0 + k * 256;
        float f[V];
        uint32_t w[V / 4];
        unpack16<DT>(u[k], f);
        const int byte = code_block<DT, V, LANES>(f, w);
        if (t >= end) break;  // whole blocks
        if constexpr (V == 8) ((uint2*)to.codes)[t] = make_uint2(w[0], w[1]);
        else ((uint32_t*)to.codes)[t] = w[0];
        if (t % LANES == 0) to.exps[t / LANES] = (uint8_t)byte;
    }
}
template <int DT>
__global__ __launch_bounds__(256) void k_code8_read(Saved8 from, void* out, RowRange rows, int C) {
    constexpr int V = kCodeVec<DT>, LANES = kCodeBlock / V;
    const int64_t end = rows.end() * (C / V), t0 = group_of_grid() * (256 * kCodeAhead) + threadIdx.x;
    uint32_t w[kCodeAhead][V / 4];
    int e[kCodeAhead];
#pragma unroll
    for (int k = 0; k < kCodeAhead; ++k) {
        const int64_t t = t0 + k * 256;
        if (t >= end) continue;
        __builtin_memcpy(w[k], (const char*)__builtin_assume_aligned(from.codes, V) + t * V, V);
        e[k] = from.exps[t / LANES];
    }
#pragma unroll
    for (int k = 0; k < kCodeAhead; ++k) {
        const int64_t t = t0 + k * 256;
        if (t >= end) break;
        float f[V];
        code_values(w[k], code_step(e[k]), f);
        ((uint4*)out)[t] = pack16<DT>(f);
    }
}

// Rows of whole vectors whose last block is shorter: a row is nb blocks of LANES threads, those past its end idle,
// and a workgroup takes 256 / (nb LANES) rows at a time, kCodeAhead times over.
template <int DT>
__global__ __launch_bounds__(256) void k_code8_short(const void* x, Saved8 to, RowRange rows, int C) {
    constexpr int V = kCodeVec<DT>, LANES = kCodeBlock / V;
    const int nb = code_blocks(C), per = nb * LANES, R = 256 / per, row = (int)threadIdx.x / per, v = (int)threadIdx.x - row * per;
    if (row >= R) return;  // whole blocks
    const int64_t end = rows.end(), i0 = rows.begin() + group_of_grid() * (R * kCodeAhead) + row;
    const bool on = v * V < C;
    uint4 u[kCodeAhead];
#pragma unroll
    for (int k = 0; k < kCodeAhead; ++k) {
        const int64_t i = i0 + k * R;
        u[k] = on && i < end ? *(const uint4*)((const char*)x + (i * C + v * V) * (16 / V)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kCodeAhead; ++k) {
        const int64_t i = i0 + k * R;
        float f[V];
        uint32_t w[V / 4];
        unpack16<DT>(u[k], f);
        const int byte = code_block<DT, V, LANES>(f, w);
        if (i >= end) break;
        if (on) __builtin_memcpy(__builtin_assume_aligned(to.codes + i * C + v * V, V), w, V);
        if (v % LANES == 0) to.exps[i * nb + v / LANES] = (uint8_t)byte;
    }
}
template <int DT>
__global__ __launch_bounds__(256) void k_code8_read_short(Saved8 from, void* out, RowRange rows, int C) {
    constexpr int V = kCodeVec<DT>, LANES = kCodeBlock / V;
    const int nb = code_blocks(C), per = C / V, R = 256 / per, row = (int)threadIdx.x / per, v = (int)threadIdx.x - row * per;
    const int64_t end = rows.end(), i0 = group_of_grid() * (R * kCodeAhead) + row;
    uint32_t w[kCodeAhead][V / 4];
    int e[kCodeAhead];
#pragma unroll
    for (int k = 0; k < kCodeAhead; ++k) {
        const int64_t i = i0 + k * R;
        if (row >= R || i >= end) continue;
        __builtin_memcpy(w[k], __builtin_assume_aligned(from.codes + i * C + v * V, V), V);
        e[k] = from.exps[i * nb + v / LANES];
    }
#pragma unroll
    for (int k = 0; k < kCodeAhead; ++k) {
        const int64_t i = i0 + k * R;
        if (row >= R || i >= end) break;
        float f[V];
        code_values(w[k], code_step(e[k]), f);
        *(uint4*)((char*)out + (i * C + v * V) * (16 / V)) = pack16<DT>(f);
    }
}

// vectors of rows that are aligned and hold whole ones: 2 where blocks are whole too, 1 where a row's threads fit a
// workgroup
template <int DT>
static int code8_vectors(const void* x, const Saved8& s, const RowRange& rows, int C) {
    constexpr int V = kCodeVec<DT>;
    if (C % V || (uintptr_t)x % 16 || (uintptr_t)s.codes % V || rows.cap * C >= ((int64_t)1 << 40)) return 0;
    return C % kCodeBlock == 0 ? 2 : code_blocks(C) * (kCodeBlock / V) <= 256 ? 1 : 0;
}
static unsigned grid_rows(int64_t m) {
    const int64_t g = (m + 8 * kCodeAhead - 1) / (8 * kCodeAhead);
    return (unsigned)(g < 1 ? 1 : g > 16384 ? 16384 : g);
}
template <int DT>
static dim3 grid_vecs(int64_t m, int C) {
    const int64_t per = 256 * kCodeAhead;
    return grid_of((m * (C / kCodeVec<DT>) + per - 1) / per);
}
static dim3 grid_short(int64_t m, int threads) {
    const int64_t rows = 256 / threads * kCodeAhead;
    return grid_of((m + rows - 1) / rows);
}
template <int DT>
static void code8(hipStream_t s, const void* x, const Saved8& to, const RowRange& rows, int C) {
    const int v = code8_vectors<DT>(x, to, rows, C);
    if (v == 2) k_code8<DT><<<grid_vecs<DT>(rows.cap, C), 256, 0, s>>>(x, to, rows, C);
    else if (v == 1)
        k_code8_short<DT><<<grid_short(rows.cap, code_blocks(C) * (kCodeBlock / kCodeVec<DT>)), 256, 0, s>>>(x, to, rows, C);
    else k_code8_any<DT><<<grid_rows(rows.cap), 256, 0, s>>>(x, to, rows, C);
}
template <int DT>
static void code8_read(hipStream_t s, const Saved8& from, void* out, const RowRange& rows, int C) {
    const int v = code8_vectors<DT>(out, from, rows, C);
    if (v == 2) k_code8_read<DT><<<grid_vecs<DT>(rows.cap, C), 256, 0, s>>>(from, out, rows, C);
    else if (v == 1) k_code8_read_short<DT><<<grid_short(rows.cap, C / kCodeVec<DT>), 256, 0, s>>>(from, out, rows, C);
    else k_code8_read_any<DT><<<grid_rows(rows.cap), 256, 0, s>>>(from, out, rows, C);
}
void launch_checkpoint8(hipStream_t s, const void* x, Saved8 to, const RowRange& rows, int C, int dt) {
    if (dt == SPV_F32) code8<SPV_F32>(s, x, to, rows, C);
    else if (dt == SPV_BF16) code8<SPV_BF16>(s, x, to, rows, C);
    else code8<SPV_F16>(s, x, to, rows, C);
}
void launch_checkpoint8_read(hipStream_t s, Saved8 from, void* out, const RowRange& rows, int C, int dt) {
    if (dt == SPV_F32) code8_read<SPV_F32>(s, from, out, rows, C);
    else if (dt == SPV_BF16) code8_read<SPV_BF16>(s, from, out, rows, C);
    else code8_read<SPV_F16>(s, from, out, rows, C);
}

// ---------------------------------------------------------------------------
// dW = in^T da.  A workgroup takes TM x TN tiles of 32 x 32 of dW and a share of the rows, its waves some of those
// each, with nothing between them but the sum at the end.  The shares' sums go to the workspace and are joined in 64
// bits. 88,119 x 96 -> 96 in bf16: 12.9 us and 4.9 for the join; 26,881 x 256 -> 256 in f16: 15.1 and 4.2 (matrix
// cores busy 12% of the time, vector units 43%: a code takes four steps to become a value, in each of the four
// columns of blocks that read it).
// ---------------------------------------------------------------------------
constexpr int kWg8Step = 32;     // rows of a wave's step
constexpr int kWg8Most = 3;      // tiles of a side of a workgroup's block
// Workgroups, as far as the rows go: one a CU.  Each leaves a share of dW (88,119 x 96 -> 96 with the codes' making
// takes 24.3 us with 128 shares, 23.0 with 256, 30.4 with 512; 26,881 x 256 -> 256 30.6, 24.2, 29.5).
constexpr int kWg8Groups = 256;
// waves of a workgroup: eight where a wave's sums leave room for two on a SIMD (26,881 x 256 -> 256 32 -> 28 us with
// four tiles; nine tiles, 144 registers of sums, 23.8 -> 28.4)
constexpr int wg8_waves(int dt, int tm, int tn) { return tm * tn <= 4 && !(dt == SPV_F32 && tn == 3) ? 8 : 4; }

// tiles of a side: the fewest padded, then the most
static int wgrad8_side(int C) {
    const int t = (C + 31) / 32;
    int best = 1;
    for (int k = 2; k <= kWg8Most; ++k)
        if ((t + k - 1) / k * k <= (t + best - 1) / best * best) best = k;
    return best;
}
static int wgrad8_blocks(int C) { return ((C + 31) / 32 + wgrad8_side(C) - 1) / wgrad8_side(C); }
static int wgrad8_parts(int64_t m_cap, int Cin, int Cout) {
    const int64_t blocks = (int64_t)wgrad8_blocks(Cin) * wgrad8_blocks(Cout);
    int64_t s = kWg8Groups / blocks;
    if (s >= 8) s = s / 8 * 8;  // shares of the same rows on one die
    const int64_t steps = (m_cap + kWg8Step - 1) / kWg8Step;
    if (s > steps) s = steps;
    return (int)(s < 1 ? 1 : s);
}
// numbers of a share: whole tiles
static int64_t wgrad8_numbers(int Cin, int Cout) {
    return (int64_t)wgrad8_blocks(Cin) * wgrad8_side(Cin) * wgrad8_blocks(Cout) * wgrad8_side(Cout) * 1024;
}
float* plan_wgrad8_ws(Arena& a, int64_t m_cap, int Cin, int Cout) {
    return a.take<float>((size_t)wgrad8_parts(m_cap, Cin, Cout) * wgrad8_numbers(Cin, Cout));
}

struct Wg8Block {
    int part, block;    // share of the rows, block of dW
    int ci, co;         // its first channels
    int64_t r0, r1;     // the wave's rows
};
// the shares come first in the grid, so that the blocks of one share, which read the same rows, run on one die; a wave has
// its share's part of the steps, the first waves of all one more where they do not come out even
template <int TM, int TN, int NW, int STEP>
__device__ inline Wg8Block wg8_block(const Wgrad8Args& a) {
    Wg8Block b;
    b.part = (int)blockIdx.x;
    b.block = (int)(blockIdx.z * gridDim.y + blockIdx.y);
    b.ci = (int)blockIdx.y * (32 * TM);
    b.co = (int)blockIdx.z * (32 * TN);
    const int64_t m = clamp_rows(a.m_dev, a.m_cap);
    const uint32_t steps = (uint32_t)((m + STEP - 1) / STEP), waves = gridDim.x * NW;
    const uint32_t w = blockIdx.x * NW + (uint32_t)uniform((int)(threadIdx.x >> 6)), each = steps / waves, more = steps - each * waves;
    b.r0 = (int64_t)(w * each + (w < more ? w : more)) * STEP;
    b.r1 = b.r0 + (int64_t)(each + (w < more)) * STEP;
    if (b.r1 > m) b.r1 = m;
    return b;
}

// A tile of 32 x 32 as it lies in LDS and in the workspace: column c's 32 rows one after the other, four rows (q of
// eight) at place q ^ (c / 2) % 8, so that the lanes of a wave, a column each, meet in no bank.
__device__ inline int wg8_place(int c, int q) { return c * 32 + 4 * (q ^ ((c >> 1) & 7)); }

// The waves' sums of a block, added up in LDS, and then to the share's part of the workspace.  Four waves share an
// image of the block; in each of four rounds a wave adds every fourth tile, another wave's next: the order of a
// tile's sum is the same on every call.
template <int NW, int TM, int TN>
__device__ inline void wg8_store(const Wgrad8Args& a, const Wg8Block& b, const f32x16 (&acc)[TM][TN], float* lds) {
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), c = lane & 31, h = lane >> 5;
    float* image = lds + (wave >> 2) * (TM * TN * 1024);
    for (int w = 0; w < 4; ++w) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                if (((i * TN + j - wave - w) & 3) != 0) continue;
                float* p = image + (i * TN + j) * 1024;
                float4 v[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    v[q] = w ? *(const float4*)(p + wg8_place(c, 2 * q + h)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(float4*)(p + wg8_place(c, 2 * q + h)) =
                        make_float4(v[q].x + acc[i][j][4 * q], v[q].y + acc[i][j][4 * q + 1],
                                    v[q].z + acc[i][j][4 * q + 2], v[q].w + acc[i][j][4 * q + 3]);
            }
    }
    __syncthreads();
    const int64_t n = (int64_t)gridDim.y * gridDim.z * (TM * TN * 1024);
    float4* out = (float4*)(a.part + b.part * n + (int64_t)b.block * (TM * TN * 1024));
    for (int t = threadIdx.x; t < TM * TN * 256; t += 64 * NW) {
        float4 v = ((const float4*)lds)[t];
        if constexpr (NW == 8) {
            const float4 u = ((const float4*)lds)[t + TM * TN * 256];
            v = make_float4(v.x + u.x, v.y + u.y, v.z + u.z, v.w + u.w);
        }
        out[t] = v;
    }
}

// A float32 number as three of bf16 (8 bits each, cut off, the last one what is left): their sum is the number, down to
// 2^-126 or so.  One that is not finite is the first of the three.
__device__ inline void three_parts(float d, uint32_t (&p)[3]) {
    const bool finite = (__float_as_uint(d) & 0x7F800000u) != 0x7F800000u;
    const uint32_t top = __float_as_uint(d) & 0xFFFF0000u;
    const float r = d - __uint_as_float(top);
    const uint32_t mid = __float_as_uint(r) & 0xFFFF0000u;
    p[0] = finite || d == d ? top : 0x7FC00000u;
    p[1] = finite ? mid : 0u;
    p[2] = finite ? __float_as_uint(r - __uint_as_float(mid)) : 0u;
}

// 16 channels of codes and 16 bytes of da at a time: a wave brings 32 rows of codes, as values of the type, and of da into
// its own part of LDS (the next 32 are on the way) and reads both back transposed: the matrix cores sum over rows.  With
// float32 the values are multiplied as bf16, which holds them (7 bits), by da in three parts of bf16: every product is
// exact, and three of them take a third of the time of one of float32's own.
template <int DT, int TM, int TN>
__global__ __launch_bounds__(64 * wg8_waves(DT, TM, TN), TM * TN > 6 ? 1 : 2) void k_wgrad8(Wgrad8Args a) {
    constexpr bool W = DT == SPV_F32;
    constexpr int MT = W ? SPV_BF16 : DT, PARTS = W ? 3 : 1, SZ = W ? 4 : 2, E = 16 / SZ;  // type of the products
    constexpr int BM = 32 * TM, BN = 32 * TN, LM = 2 * BM + 16, LN = 2 * BN + 16;  // bytes from row to row in LDS
    constexpr int QM = BM / 16, QN = BN / E;                         // 16-byte chunks of a row
    constexpr int KM = kWg8Step * QM / 64, KN = kWg8Step * QN / 64;  // of a lane
    constexpr int PART = kWg8Step * LN, SIZE = kWg8Step * LM + PARTS * PART;
    constexpr int NW = wg8_waves(DT, TM, TN), SUMS = NW / 4 * BM * BN * 4, LDS = NW * SIZE > SUMS ? NW * SIZE : SUMS;
    typedef short i16x8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) i16x4 lds4;
    __shared__ __align__(16) char lds[LDS];
    const Wg8Block b = wg8_block<TM, TN, NW, kWg8Step>(a);
    const int lane = threadIdx.x & 63, nb = code_blocks(a.Cin);
    char *lx = lds + (threadIdx.x >> 6) * SIZE, *ld = lx + kWg8Step * LM;
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    // what a lane brings of a step, from its first row: channels past the ends are read as the last ones and not stored
    uint4 ux[KM], ud[KN];
    int ue[KM];
    uint32_t atx[KM], ate[KM], atd[KN];
#pragma unroll
    for (int k = 0; k < KM; ++k) {
        const int t = lane + 64 * k, c = b.ci + t % QM * 16 < a.Cin ? b.ci + t % QM * 16 : a.Cin - 16;
        atx[k] = (uint32_t)(t / QM * a.Cin + c);
        ate[k] = (uint32_t)(t / QM * nb + c / kCodeBlock);
    }
#pragma unroll
    for (int k = 0; k < KN; ++k) {
        const int t = lane + 64 * k, c = b.co + t % QN * E < a.Cout ? b.co + t % QN * E : a.Cout - E;
        atd[k] = (uint32_t)(t / QN * a.Cout + c) * SZ;
    }
    auto ask = [&](int64_t r0) {
        const int8_t* px = a.in.codes + r0 * a.Cin;
        const uint8_t* pe = a.in.exps + r0 * nb;
        const char* pd = (const char*)a.da + r0 * a.Cout * SZ;
        if (r0 + kWg8Step <= b.r1) {
#pragma unroll
            for (int k = 0; k < KM; ++k) {
                ux[k] = *(const uint4*)(px + atx[k]);
                ue[k] = pe[ate[k]];
            }
#pragma unroll
            for (int k = 0; k < KN; ++k) ud[k] = *(const uint4*)(pd + atd[k]);
        } else {  // rows past the end count as 0
            const int rows = (int)(b.r1 - r0);
#pragma unroll
            for (int k = 0; k < KM; ++k) {
                const bool on = (lane + 64 * k) / QM < rows;
                ux[k] = on ? *(const uint4*)(px + atx[k]) : make_uint4(0, 0, 0, 0);
                ue[k] = on ? pe[ate[k]] : 1;
            }
#pragma unroll
            for (int k = 0; k < KN; ++k)
                ud[k] = (lane + 64 * k) / QN < rows ? *(const uint4*)(pd + atd[k]) : make_uint4(0, 0, 0, 0);
        }
    };
    // lanes 16 g .. 16 g + 15 read four rows of 16 channels, and each gets its channel of the four
    const int tl = lane & 15, tg = lane >> 4, row = 4 * (tg >> 1) + (tl >> 2), at = (16 * (tg & 1) + 4 * (tl & 3)) * 2;
    auto transposed = [&](const char* p, int LD) {
        const uint32_t q = lds_addr(p) + row * LD + at;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)q);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(q + 8 * LD));
        return __builtin_bit_cast(uint4, (i16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    if (b.r0 < b.r1) ask(b.r0);
    for (int64_t r0 = b.r0; r0 < b.r1; r0 += kWg8Step) {
#pragma unroll
        for (int k = 0; k < KM; ++k) {
            const int t = lane + 64 * k;
            const uint32_t w[4] = {ux[k].x, ux[k].y, ux[k].z, ux[k].w};
            float f[16];
            code_values(w, code_step(ue[k]), f);
            uint32_t v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = pack2<MT>(f[2 * e], f[2 * e + 1]);
            uint4* p = (uint4*)(lx + t / QM * LM + t % QM * 32);
            p[0] = make_uint4(v[0], v[1], v[2], v[3]);
            p[1] = make_uint4(v[4], v[5], v[6], v[7]);
        }
#pragma unroll
        for (int k = 0; k < KN; ++k) {
            const int t = lane + 64 * k;
            char* p = ld + t / QN * LN + t % QN * (2 * E);
            if constexpr (W) {
                const uint32_t w[4] = {ud[k].x, ud[k].y, ud[k].z, ud[k].w};
                uint32_t q[4][3];
#pragma unroll
                for (int e = 0; e < 4; ++e) three_parts(__uint_as_float(w[e]), q[e]);
#pragma unroll
                for (int h = 0; h < 3; ++h)  // the upper halves of two words
                    *(uint2*)(p + h * PART) = make_uint2(__builtin_amdgcn_perm(q[1][h], q[0][h], 0x07060302u),
                                                         __builtin_amdgcn_perm(q[3][h], q[2][h], 0x07060302u));
            } else {
                *(uint4*)p = ud[k];
            }
        }
        if (r0 + kWg8Step < b.r1) ask(r0 + kWg8Step);
        lds_wait();
#pragma unroll
        for (int k = 0; k < kWg8Step / 16; ++k) {
            uint4 x[TM], d[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) x[i] = transposed(lx + 16 * k * LM + 64 * i, LM);
#pragma unroll
            for (int h = PARTS - 1; h >= 0; --h) {  // the smallest first
#pragma unroll
                for (int j = 0; j < TN; ++j) d[j] = transposed(ld + h * PART + 16 * k * LN + 64 * j, LN);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = mfma32x32x16<MT>(x[i], d[j], acc[i][j]);
            }
        }
        lds_wait();
    }
    wg8_store<NW>(a, b, acc, (float*)lds);
}

// Other widths and alignments, and few rows of float32, in products of float32: a lane's operands are a channel
// of a row each, as memory has them.  Rows and channels past the ends are read as the last ones, and count as 0.
template <int DT, int TM, int TN>
__global__ __launch_bounds__(64 * wg8_waves(DT, TM, TN), TM * TN > 6 ? 1 : 2) void k_wgrad8_any(Wgrad8Args a) {
    constexpr int U = 4, STEP = 2 * U, NW = wg8_waves(DT, TM, TN);
    __shared__ __align__(16) float lds[NW / 4 * TM * TN * 1024];
    const Wg8Block b = wg8_block<TM, TN, NW, STEP>(a);
    const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5, nb = code_blocks(a.Cin);
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    int q[U][TM], x[U][TM];
    float d[U][TN];
    auto ask = [&](int64_t r0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = r0 + 2 * u + h, r = at < b.r1 ? at : b.r1 - 1;
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int k = b.ci + 32 * i + c < a.Cin ? b.ci + 32 * i + c : a.Cin - 1;
                q[u][i] = a.in.codes[r * a.Cin + k];
                x[u][i] = a.in.exps[r * nb + k / kCodeBlock];
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int k = b.co + 32 * j + c < a.Cout ? b.co + 32 * j + c : a.Cout - 1;
                d[u][j] = ld_feat<DT>(a.da, r * a.Cout + k);
            }
        }
    };
    if (b.r0 < b.r1) ask(b.r0);
    for (int64_t r0 = b.r0; r0 < b.r1; r0 += STEP) {
        float f[U][TM], g[U][TN];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool on = r0 + 2 * u + h < b.r1;
#pragma unroll
            for (int i = 0; i < TM; ++i) f[u][i] = on ? code_value(q[u][i], code_step(x[u][i])) : 0.f;
#pragma unroll
            for (int j = 0; j < TN; ++j) g[u][j] = on ? d[u][j] : 0.f;
        }
        if (r0 + STEP < b.r1) ask(r0 + STEP);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(f[u][i], g[u][j], acc[i][j], 0, 0, 0);
    }
    wg8_store<NW>(a, b, acc, lds);
}

// adds the shares of the n numbers in 64 bits, 64 of them a workgroup, in 32 runs of consecutive shares; each is then
// put where it belongs in dW (blocks of TM x TN tiles, those of a column of blocks one after the other)
__global__ __launch_bounds__(512) void k_wgrad8_join(const float* __restrict__ part, int parts, int64_t n, int TM, int TN, int Cin,
                                                     int Cout, float* __restrict__ dW) {
    __shared__ double red[8][65];
    const int col = threadIdx.x & 15, run = threadIdx.x >> 4, len = (parts + 31) / 32;
    const int p0 = run * len, p1 = p0 + len < parts ? p0 + len : parts;
    const float4* from = (const float4*)(part + (int64_t)blockIdx.x * 64) + col;
    double s[4] = {};
    for (int p = p0; p < p1; p += 8) {
        float4 f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            f[k] = p + k < p1 ? from[(int64_t)(p + k) * (n / 4)] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            s[0] += (double)f[k].x;
            s[1] += (double)f[k].y;
            s[2] += (double)f[k].z;
            s[3] += (double)f[k].w;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // a wave's four runs, then the waves'
        s[e] = rows_sum(s[e]);
        if ((threadIdx.x & 63) < 16) red[threadIdx.x >> 6][4 * col + e] = s[e];
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    double sum = red[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < 8; ++w) sum += red[w][threadIdx.x];
    const int64_t t = (int64_t)blockIdx.x * 64 + threadIdx.x;
    const int tile = (int)(t / 1024), c = (int)(t % 1024) / 32, q = (int)(t % 32) / 4 ^ ((c >> 1) & 7);
    const int block = tile / (TM * TN), in = tile % (TM * TN), nm = (Cin + 32 * TM - 1) / (32 * TM);
    const int i = (block % nm * TM + in / TN) * 32 + 4 * q + (int)(t % 4), j = (block / nm * TN + in % TN) * 32 + c;
    if (i < Cin && j < Cout) dW[(int64_t)i * Cout + j] = (float)sum;
}

template <int DT, int TM, int TN>
static void wgrad8(hipStream_t s, const Wgrad8Args& a, int parts) {
    const dim3 g((unsigned)parts, (unsigned)wgrad8_blocks(a.Cin), (unsigned)wgrad8_blocks(a.Cout));
    // float32: rows enough for a wave's steps of 32 (96 -> 96, 1024 waves: 701 rows take 12.1 us in three parts, 10.0 in
    // float32's products; 12,000 18.0 and 17.6; 256 -> 256, 128 waves: 701 12.8 and 12.2, 12,000 19.3 and 35.3)
    const bool rows = DT != SPV_F32 || a.m_cap >= (int64_t)12 * parts * wg8_waves(DT, TM, TN);
    if (rows && a.Cin % 16 == 0 && a.Cout % (DT == SPV_F32 ? 4 : 8) == 0 &&
        (((uintptr_t)a.in.codes | (uintptr_t)a.da) & 15u) == 0)
        k_wgrad8<DT, TM, TN><<<g, 64 * wg8_waves(DT, TM, TN), 0, s>>>(a);
    else
        k_wgrad8_any<DT, TM, TN><<<g, 64 * wg8_waves(DT, TM, TN), 0, s>>>(a);
}
template <int DT, int TM>
static void wgrad8_n(hipStream_t s, const Wgrad8Args& a, int parts) {
    const int n = wgrad8_side(a.Cout);
    if (n == 1) wgrad8<DT, TM, 1>(s, a, parts);
    else if (n == 2) wgrad8<DT, TM, 2>(s, a, parts);
    else wgrad8<DT, TM, 3>(s, a, parts);
}
template <int DT>
static void wgrad8_m(hipStream_t s, const Wgrad8Args& a, int parts) {
    const int n = wgrad8_side(a.Cin);
    if (n == 1) wgrad8_n<DT, 1>(s, a, parts);
    else if (n == 2) wgrad8_n<DT, 2>(s, a, parts);
    else wgrad8_n<DT, 3>(s, a, parts);
}
void launch_wgrad8(hipStream_t s, const Wgrad8Args& a) {
    const int parts = wgrad8_parts(a.m_cap, a.Cin, a.Cout);
    if (a.dt == SPV_F32) wgrad8_m<SPV_F32>(s, a, parts);
    else if (a.dt == SPV_BF16) wgrad8_m<SPV_BF16>(s, a, parts);
    else wgrad8_m<SPV_F16>(s, a, parts);
    const int64_t n = wgrad8_numbers(a.Cin, a.Cout);
    k_wgrad8_join<<<(unsigned)(n / 64), 512, 0, s>>>(a.part, parts, n, wgrad8_side(a.Cin), wgrad8_side(a.Cout), a.Cin, a.Cout,
                                                     a.dW);
}

}  // namespace spv
