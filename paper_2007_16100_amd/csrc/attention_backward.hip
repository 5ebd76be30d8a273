// attention_backward.hip -- the backward of attention over packed scans:
//   p_ij = exp(s_ij - lse_i),  delta_i = dout_i . out_i,  dz_ij = p_ij (dout_i . v_j - delta_i) ds_ij/dz_ij
//   dq_i = scale sum_j dz_ij k_j,   dk_j = scale sum_i dz_ij q_i,   dv_j = sum_i p_ij dout_i
// Two kernels, each of which forms the weights anew: dq with the queries in the columns, as the forward has them (it
// also forms delta), and dk, dv with the keys in the columns.  One kernel for all three would save two products of
// seven, but either add dq in the order that workgroups happen to run in, or hold it for every part of the keys.
// -delta is what the products dout . v are added to; the bias, over scale, or (keys in the columns) the rows' -lse are
// what the products q . k are added to, unless a cap's tanh stands between or (float32) the roundings at their size of each
// step of the product would show (dv of 300 x 300 heads of 128: 1.7e-6 that way, 5.7e-7 so).
//
// In 16 bits p and dz are rounded to the type before their products: dq of bf16 is off by 2.3e-3 (root of the mean square
// against 64 bits), dk and dv by 2.4e-3, their own last rounding alone by 1.7e-3.  Two halves of dz would bring dq and dk
// to 1.7e-3, for 21 us more in each kernel at the size below.  Out, which delta is formed of, comes in rounded too: see
// DqSums.
//
// [3451, 3654, 1963, 2195] x 8 heads of 32, bf16, bias: a training step takes 328 us; in a kernel trace of a cold start the
// forward takes 105 of it, dq 131, dk and dv 140.  The vector units are busy 67% of the time in dq, 55% in dk and dv, the
// matrix units 27 and 25%.  Dk and dv have two accumulators of a column, so 2.5 waves a SIMD, which wait for LDS (its
// index unit active 45%) and the matrix unit in turn, with a barrier every 32 rows.
// [1457, 1544] x 3 heads in float32, cap and bias: dq 60 us, dk and dv 76; 285 workgroups, one wave to a SIMD, whose
// products (44 and 47% of the cycles), vector instructions (21 and 18%) and waits follow one another.
#include "attn_common.hpp"

namespace spv {

// A row's lse in units of log 2, as the weights are formed from it.  A float32 holds it to 2^-24 of itself, and a weight
// exp2(s - lse) is off by as much: past kMaxLse by a factor, up to overflow.  Such a row, and one whose scores are all
// minus infinity, has no gradient.
constexpr float kMaxLse = 4194304.f;  // 2^22
__device__ inline float row_lse(float lse) {
    const float e = lse * kLog2e;
    return fabsf(e) > kMaxLse ? INFINITY : e;
}

// Waves per SIMD that the registers have to leave room for, each the faster of two.  Some forms spill all the same: up to
// 96 channels dozens of registers with a bias and a cap, at 128 in float32 with a bias over a hundred.  Backward of [8192]
// in bf16: 4 heads of 128, one wave in dq 806 us, two 1103; 8 heads of 96 two 754, one 984, but under a cap one 1211, two
// 1325; 8 heads of 32 under a cap two 596, three 1720.  [9000] x 8 heads of 96, forward and backward, with two in dk, dv
// 1908 us, with one 2319 (before dq had its fourth product); [4096] x 4 heads of 64 in float32 with two everywhere 1026
// us, with one 773.
constexpr int dq_waves(int dt, int DP, int cap) {
    return dt == SPV_F32 ? (DP > 64 ? 1 : 2) : DP > 96 || (DP > 64 && cap) ? 1 : DP > 32 || cap ? 2 : 3;
}
constexpr int dkv_waves(int dt, int DP, int KW) {
    return dt == SPV_F32 ? (DP > 32 ? 1 : 2) : DP > 96 || (DP > 64 && KW > 1) ? 1 : DP > 32 ? 2 : 3;
}

// The weights are at most 1 and, over long scans, far below float16's smallest normal number (6e-5): in that type they
// are multiplied as 2^12 p (and may be some times 1 where scores of millions round).
template <int DT>
constexpr float kUp = DT == SPV_F16 ? 12.f : 0.f;

// In 16 bits delta, formed of the rounded out, is off by an error e, every dz of a row by p e ds/dz, and dq by e times the
// sum of p ds/dz k.  That is more than dq itself where keys and values lie around a mean: with both around 4 dq of bf16 was
// off by 0.6, now by 2.3e-3.  The row shows e: the sum over its keys of p (dout . v - delta) is -e where it would be zero.
// So one more product gives the sum of p ds/dz k, and e times it is taken off; dk takes the corrected delta.  What
// rounding dz to the type adds to the sum of dz k for the mean key is taken off the same way: without a cap the sum
// of dz as they are multiplied has both in it, under one (where the sum of dz need not be zero) they are counted apart.
// A training step of [3451, 3654, 1963, 2195] x 8 heads of 32, bf16: 303 -> 327 us.
struct DqSums {
    float s[3] = {0.f, 0.f, 0.f};  // of dz as multiplied; of dz; under a cap of p (dout . v - delta)
    float p = 0.f;                 // of p ds/dz
    __device__ inline void halves() {
#pragma unroll
        for (int i = 0; i < 3; ++i) s[i] = half_sum(s[i]);
        p = half_sum(p);
    }
    __device__ inline void scale(float f, float fp) { s[0] *= f, s[1] *= f, s[2] *= f, p *= fp; }
    // -e, for delta
    __device__ inline float error(bool cap) const { return cap ? s[2] : s[1]; }
    // what the sum of p ds/dz k is taken off times
    __device__ inline float off(bool cap) const { return cap ? s[2] + (p > 0.f ? (s[0] - s[1]) / p : 0.f) : s[0]; }
    // a wave's, 64 floats apart
    __device__ inline void put(float* l) const { l[0] = s[0], l[64] = s[1], l[128] = s[2], l[192] = p; }
    __device__ inline void add(const float* l) { s[0] += l[0], s[1] += l[64], s[2] += l[128], p += l[192]; }
};

// Float16 holds dz neither where weights are small (below 6e-5 in fewer than eleven bits, below 3e-8 not at all) nor where
// dout . v passes 65,504.  So a column's dz are multiplied as 2^up dz, and its sums scaled back at the end: up is lowered,
// and the sums so far with it, whenever one passes 2^15, to leave the largest at 2^8.  It starts where the first rows
// lower it, unless all of them are below 2^-45.  Finding the largest takes a tenth of a training step: 310 -> 341 us at
// [3451, 3654, 1963, 2195] x 8 heads of 32, and dq of 60 queries over 6720 keys at dout of 1e-4 was off by 8e-2
// without it, where rounding the exact result gives 8e-3, as now.
constexpr int kUpMost = 60;
// true: up of some column of the wave was lowered
template <int N, int M>
__device__ inline bool lower(f32x16& z, f32x16 (&o)[N], int& up, float (&sums)[M]) {
    float top = fabsf(z[0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, fabsf(z[r]));
    if (!__any(top > 32768.f)) return false;
    top = half_max(top);
    int by = top > 32768.f ? (int)(__float_as_uint(top) >> 23) - 127 - 8 : 0;
    if (by > up + 200) by = up + 200;  // infinities stay what they are
    const float f = __builtin_amdgcn_ldexpf(1.f, -by);
    up -= by;
#pragma unroll
    for (int i = 0; i < M; ++i) sums[i] *= f;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] *= f;
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] *= f;
    return true;
}
template <int N>
__device__ inline void scale_back(f32x16 (&o)[N], int up) {
    const float f = __builtin_amdgcn_ldexpf(1.f, -up);
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] *= f;
}

template <int DT, int DP, int KW, bool BIAS, int CAP>
__global__ __launch_bounds__(256, dq_waves(DT, DP, CAP)) void k_attn_dq(AttnArgs a) {
    using T = Tile<DT, DP>;
    constexpr int RT = attn_rows(DT, DP, KW), KT = RT * KW, KS = RT / 32, CW = 4 / KW, BM = 32 * CW;
    constexpr bool AFTER = attn_after(DT, BIAS, CAP), LOW = DT != SPV_F32;
    constexpr bool WIDE = LOW && DP > 64;  // -delta is added after the product: 16 registers less
    __shared__ __align__(16) char lk[2][KT * T::LD], lv[2][KT * T::LD];
    __shared__ __align__(16) Places<BIAS ? KT : 32> lc;
    __shared__ uint32_t box[4][3];
    __shared__ float ls[LOW && KW > 1 ? 4 * CW * (KW - 1) : 1][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), cw = wave / KW, kw = wave % KW;
    const int c = lane & 31, h = lane >> 5;
    const Share sh = attn_share(a);
    const int G = a.H / a.K, kh = sh.kh;
    const ScanTile t = find_tile(a.q_off, a.nq, a.k_off, a.nk, a.B, G, BM, sh.tile);
    if (t.col0 >= t.cols) return;  // the whole workgroup
    const int64_t k0 = t.r0, k1 = t.r1;
    const int keys = (int)(k1 > k0 ? k1 - k0 : 0), tiles = keys / KT + (keys % KT != 0);
    const int per = (tiles + sh.parts - 1) / sh.parts, t0 = sh.part * per, t1 = t0 + per < tiles ? t0 + per : tiles;

    const bool busy = t.col0 + 32 * cw < t.cols, live = t.col0 + 32 * cw + c < t.cols;
    const int64_t q0 = t.col0 / G;
    const int y0 = (int)(t.col0 - q0 * G) + 32 * cw + c, head = kh * G + y0 % G;
    const int64_t qi = t.first + q0 + y0 / G;
    uint4 qf[T::NF], df[T::NF];
    T::load_cols(a.q, qi * a.ldq + (int64_t)head * a.D, live, a.D, h, qf);
    T::load_cols(a.dout, qi * a.lddo + (int64_t)head * a.D, live, a.D, h, df);
    float lse = 0.f, delta = 0.f;
    uint4 of[T::NF];
    T::load_cols(a.out, qi * a.ldo + (int64_t)head * a.D, live, a.D, h, of);
    int4 qc{0, 0, 0, 0};
    float slope = 0.f;  // of the scores where the bias is added after, else of the products
    if (live) {
        lse = a.lse[qi * a.H + head];
        if constexpr (BIAS) {
            qc = *(const int4*)(a.q_coords + 4 * qi);
            slope = a.slopes[head];
        }
    }

    Stage<DT, DP, KT, 256> sk(tid, a.ldk, a.D), sv(tid, a.ldv, a.D);
    const int64_t first = k0 + (int64_t)t0 * KT;
    RowTiles<KT> rk((const char*)a.k + kh * a.D * T::SZ, first, a.ldk * T::SZ, a.D * T::SZ);
    RowTiles<KT> rv((const char*)a.v + kh * a.D * T::SZ, first, a.ldv * T::SZ, a.D * T::SZ);
    RowTiles<KT> rc(a.k_coords, first, 16, 16);
    int4 ck{0, 0, 0, 0};
    int ahead = keys - t0 * KT, got = 0;  // keys to load, and how many of them the tile loaded last has
    auto load = [&]() __attribute__((always_inline)) {
        got = ahead < KT ? ahead : KT;
        ahead -= KT;
        sk.load(rk.next(got));
        sv.load(rv.next(got));
        if constexpr (BIAS) {
            const __amdgpu_buffer_rsrc_t r = rc.next(got);
            if (tid < KT) ck = __builtin_bit_cast(int4, __builtin_amdgcn_raw_buffer_load_b128(r, tid * 16, 0, 0));
        }
    };
    // the first rows are asked for before anything waits for the columns'
    if (t0 < t1) load();

    lse = row_lse(lse);
#pragma unroll
    for (int s = 0; s < T::NF; ++s) delta = T::frag_dot(df[s], of[s], delta);
    delta = half_sum(delta);
    Words far{0, 0};
    uint32_t place = 0;
    Cube cube{};
    if constexpr (BIAS) {
        qc = voxel_clamp(qc);
        slope = AFTER ? slope * kLog2e : slope / a.scale;
        cube = columns_cube(qc, live, box);
        cube.place(qc, place);
        far = voxel_words(qc);
    }
    const float lift = slope * 8388608.f;
    const float cs = in_vgpr(a.scale * kLog2e);
    const Capped<CAP> capped(a);
    int up = DT == SPV_F16 ? kUpMost : 0;
    float lift_p = __builtin_amdgcn_ldexpf(1.f, (int)kUp<DT> - up);
    float rest = (float)up - lse;  // what a weight's exponent is beside the score
    f32x16 dref;
#pragma unroll
    for (int r = 0; r < 16; ++r) dref[r] = WIDE ? 0.f : -delta;

    auto store = [&](int s) __attribute__((always_inline)) {
        sk.store(lk[s], tid);
        sv.store(lv[s], tid);
        if constexpr (BIAS)
            if (tid < KT) lc.put(s, tid, ck, tid < got, cube);
    };
    f32x16 o[T::NB], mean[T::NB];  // sums of dz k and (16 bits) of the weights of its error, p ds/dz, times k
#pragma unroll
    for (int b = 0; b < T::NB; ++b) o[b] = mean[b] = f32x16{};
    DqSums sums;
    if (t0 < t1) {
        store(0);
        if (t0 + 1 < t1) load();
    }
    __syncthreads();
    for (int i = t0; i < t1; ++i) {
        const int s = (i - t0) & 1;
        const int row0 = RT * kw, left = keys - i * KT - row0;  // the wave's rows of the tile, keys from there on
        if (busy && left > 0) {
            f32x16 z[KS], d[KS];
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                d[u] = T::rows_dot(lv[s] + (row0 + 32 * u) * T::LD, lane, df, dref);
                f32x16 b{};
                if constexpr (BIAS && !AFTER)
                    lc.bias(s, row0 + 32 * u, h, far, place, slope, lift,
                            [&](int r, float x) __attribute__((always_inline)) { b[r] = x; });
                z[u] = T::rows_dot(lk[s] + (row0 + 32 * u) * T::LD, lane, qf, b);
            }
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                f32x16 p, free;  // weights times ds/dz, p (dout . v - delta) free of it
                const int end = left - 32 * u;
                auto grad = [&](int r, float b) __attribute__((always_inline)) {
                    if constexpr (CAP) {
                        float bend;
                        const float x = capped(z[u][r], b + (capped.lift + rest), &bend), w = __builtin_amdgcn_exp2f(x);
                        p[r] = w * bend;
                        free[r] = w * (WIDE ? d[u][r] - delta : d[u][r]);
                        z[u][r] = free[r] * bend;
                    } else {
                        p[r] = __builtin_amdgcn_exp2f(fmaf(z[u][r], cs, AFTER ? b + rest : rest));
                    }
                    if constexpr (!CAP) z[u][r] = p[r] * (WIDE ? d[u][r] - delta : d[u][r]);
                    if constexpr (DT == SPV_F16) p[r] *= lift_p;
                };
                if constexpr (AFTER && BIAS)
                    lc.bias(s, row0 + 32 * u, h, far, place, slope, lift, grad);
                else
#pragma unroll
                    for (int r = 0; r < 16; ++r) grad(r, 0.f);
                // keys past the scan's end: their rows are zero, but not their weights, which may pass any bound
                if (end < 32) {
                    asm volatile("");  // a branch, not selects on every tile
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r / 4) + 4 * h + r % 4 >= end) z[u][r] = p[r] = free[r] = 0.f;
                }
                if constexpr (LOW && CAP)
#pragma unroll
                    for (int r = 0; r < 16; ++r) sums.s[2] += free[r];
                if constexpr (DT == SPV_F16)
                    if (lower(z[u], o, up, sums.s)) {
                        rest = (float)up - lse;
                        lift_p = __builtin_amdgcn_ldexpf(1.f, (int)kUp<DT> - up);
                    }
                const typename T::Weights w = T::weights(z[u]);
                if constexpr (LOW) {
                    const typename T::Weights wp = T::weights(p);
                    sums.s[0] = T::sum(w, sums.s[0]);
#pragma unroll
                    for (int r = 0; r < 16; ++r) sums.s[1] += z[u][r];
                    if constexpr (CAP) sums.p = T::sum(wp, sums.p);
                    T::add_weighted(lk[s] + (row0 + 32 * u) * T::LD, lane, w, o, &wp, mean);
                } else {
                    T::add_weighted(lk[s] + (row0 + 32 * u) * T::LD, lane, w, o);
                }
            }
        }
        if (i + 1 < t1) {
            store(s ^ 1);
            if (i + 2 < t1) load();
        }
        __syncthreads();
    }
    if constexpr (DT == SPV_F16) {
        scale_back(o, up);
        scale_back(mean, (int)kUp<DT>);
        sums.scale(__builtin_amdgcn_ldexpf(1.f, -up), __builtin_amdgcn_ldexpf(1.f, -(int)kUp<DT>));
    }
    if constexpr (LOW) sums.halves();
    if constexpr (KW > 1) {
        // the waves of a block of columns add up (the tiles' LDS is free by now)
        static_assert(2 * KT * T::LD >= CW * (KW - 1) * T::NB * 16 * 256, "a wave's sums have room");
        constexpr int N = T::NB * 16 * 64;
        float *p = (float*)&lk[0][0] + cw * (KW - 1) * N, *pm = (float*)&lv[0][0] + cw * (KW - 1) * N;
        if (kw) {
            lds_put(p + (kw - 1) * N, lane, o);
            if constexpr (LOW) {
                lds_put(pm + (kw - 1) * N, lane, mean);
                sums.put(&ls[4 * (cw * (KW - 1) + kw - 1)][lane]);
            }
        }
        __syncthreads();
        if (kw) return;
#pragma unroll
        for (int w = 1; w < KW; ++w) {
            lds_add(p + (w - 1) * N, lane, 1.f, o);
            if constexpr (LOW) {
                lds_add(pm + (w - 1) * N, lane, 1.f, mean);
                sums.add(&ls[4 * (cw * (KW - 1) + w - 1)][lane]);
            }
        }
    }
    if (!live) return;
    const float f = a.scale * kBend<CAP>;
    const int64_t row = qi * a.H + head;
    if (a.part) {
        const int64_t at = (int64_t)sh.part * a.nq * a.H + row;
        if (h == 0 && sh.part == 0) a.delta[row] = delta;
        if constexpr (LOW) {
            if (h == 0) *(float4*)(a.part_ml + 4 * at) = make_float4(sums.s[0], sums.s[1], sums.s[2], sums.p);
            Tile<SPV_F32, DP>::store_cols(a.part, (2 * at + 1) * a.D, a.D, h, mean, f);
            Tile<SPV_F32, DP>::store_cols(a.part, 2 * at * a.D, a.D, h, o, f);
        } else {
            Tile<SPV_F32, DP>::store_cols(a.part, at * a.D, a.D, h, o, f);
        }
        return;
    }
    if constexpr (LOW) {
        const float off = sums.off(CAP);
#pragma unroll
        for (int b = 0; b < T::NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[b][r] = fmaf(-off, mean[b][r], o[b][r]);
        delta += sums.error(CAP);
    }
    if (h == 0) a.delta[row] = delta;
    T::store_cols(a.dq, qi * a.lddq + (int64_t)head * a.D, a.D, h, o, f);
}

// dq from the parts of its sums (16-bit types), and the rows' delta; four channels a thread
template <int DT>
__global__ __launch_bounds__(256) void k_attn_dq_join(AttnArgs a, int parts) {
    const int w = a.D / 4;
    const int64_t id = blockIdx.x * (int64_t)256 + threadIdx.x, row = id / w, rows = a.nq * a.H, qi = row / a.H;
    if (qi >= a.nq || qi < a.q_off[0] || qi >= a.q_off[a.B]) return;  // past the end, or a row of no scan
    const int d = (int)(id - row * w) * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f), m = s;
    DqSums sums;
    for (int q = 0; q < parts; ++q) {
        const int64_t at = q * rows + row;
        const float4 x = *(const float4*)(a.part + 2 * at * a.D + d), y = *(const float4*)(a.part + (2 * at + 1) * a.D + d);
        const float4 z = *(const float4*)(a.part_ml + 4 * at);
        s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
        m.x += y.x, m.y += y.y, m.z += y.z, m.w += y.w;
        sums.s[0] += z.x, sums.s[1] += z.y, sums.s[2] += z.z, sums.p += z.w;
    }
    const bool cap = a.cap > 0.f;
    const float off = -sums.off(cap);
    *(uint2*)((uint16_t*)a.dq + qi * a.lddq + (row - qi * a.H) * a.D + d) =
        make_uint2(pack2<DT>(fmaf(off, m.x, s.x), fmaf(off, m.y, s.y)),
                   pack2<DT>(fmaf(off, m.z, s.z), fmaf(off, m.w, s.w)));
    if (d == 0) a.delta[row] += sums.error(cap);
}

// Columns are keys; the rows are the scan's queries, once for each head of the key head's group, in that order.
template <int DT, int DP, int KW, bool BIAS, int CAP>
__global__ __launch_bounds__(256, dkv_waves(DT, DP, KW)) void k_attn_dkv(AttnArgs a) {
    using T = Tile<DT, DP>;
    constexpr int RT = 32, KT = RT * KW, KS = RT / 32, CW = 4 / KW, BM = 32 * CW;
    constexpr bool AFTER = CAP || DT == SPV_F32;  // the row's -lse is added after the product
    __shared__ __align__(16) char lq[2][KT * T::LD], ld[2][KT * T::LD];
    __shared__ __align__(16) Places<BIAS ? KT : 32> lc;
    __shared__ uint32_t box[4][3];
    __shared__ __align__(16) float lr[2][2][KT];  // the rows' -lse (see below) and -delta
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), cw = wave / KW, kw = wave % KW;
    const int c = lane & 31, h = lane >> 5;
    const Share sh = attn_share(a);
    const int G = a.H / a.K, kh = sh.kh;
    const ScanTile t = find_tile(a.k_off, a.nk, a.q_off, a.nq, a.B, 1, BM, sh.tile);
    if (t.col0 >= t.cols) return;  // the whole workgroup
    const int64_t q0 = t.r0, q1 = t.r1;
    const int rows = (int)(q1 > q0 ? q1 - q0 : 0), tiles = rows / KT + (rows % KT != 0), all = tiles * G;
    const int per = (all + sh.parts - 1) / sh.parts, t0 = sh.part * per, t1 = t0 + per < all ? t0 + per : all;

    const bool busy = t.col0 + 32 * cw < t.cols, live = t.col0 + 32 * cw + c < t.cols;
    const int64_t kj = t.first + t.col0 + 32 * cw + c;
    uint4 kf[T::NF], vf[T::NF];
    T::load_cols(a.k, kj * a.ldk + (int64_t)kh * a.D, live, a.D, h, kf);
    T::load_cols(a.v, kj * a.ldv + (int64_t)kh * a.D, live, a.D, h, vf);
    int4 kc{0, 0, 0, 0};
    if constexpr (BIAS)
        if (live) kc = *(const int4*)(a.k_coords + 4 * kj);

    Stage<DT, DP, KT, 256> sq(tid, a.ldq, a.D), sd(tid, a.lddo, a.D);
    int4 cq{0, 0, 0, 0};
    float rl = 0.f, rd = 0.f;
    int got = 0;  // rows of the tile loaded last
    // the tile to load and the one at work, as head of the group and tile of its rows
    int next = t0, g_next = tiles ? t0 / tiles : 0, i_next = t0 - g_next * tiles;
    RowTiles<KT> rq, ro, re, rt, rc;
    auto start = [&]() __attribute__((always_inline)) {
        const int64_t r = q0 + (int64_t)i_next * KT, head = (int64_t)kh * G + g_next;
        rq = RowTiles<KT>((const char*)a.q + head * a.D * T::SZ, r, a.ldq * T::SZ, a.D * T::SZ);
        ro = RowTiles<KT>((const char*)a.dout + head * a.D * T::SZ, r, a.lddo * T::SZ, a.D * T::SZ);
        re = RowTiles<KT>(a.lse + head, r, 4 * a.H, 4);
        rt = RowTiles<KT>(a.delta + head, r, 4 * a.H, 4);
        rc = RowTiles<KT>(a.q_coords, r, 16, 16);
    };
    start();
    auto load = [&]() __attribute__((always_inline)) {
        got = rows - i_next * KT < KT ? rows - i_next * KT : KT;
        sq.load(rq.next(got));
        sd.load(ro.next(got));
        const __amdgpu_buffer_rsrc_t be = re.next(got), bt = rt.next(got);
        if (tid < KT) {
            rl = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(be, tid * 4 * a.H, 0, 0));
            rd = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(bt, tid * 4 * a.H, 0, 0));
        }
        if constexpr (BIAS) {
            const __amdgpu_buffer_rsrc_t bc = rc.next(got);
            if (tid < KT) cq = __builtin_bit_cast(int4, __builtin_amdgcn_raw_buffer_load_b128(bc, tid * 16, 0, 0));
        }
        ++next;
        if (++i_next == tiles) {
            i_next = 0, ++g_next;
            if (next < t1) start();
        }
    };
    int i_now = i_next, g_now = g_next;
    // the first rows are asked for before anything waits for the columns'
    if (t0 < t1) load();

    const float cs = in_vgpr(a.scale * kLog2e), inv_cs = 1.f / cs;
    const Capped<CAP> capped(a);
    Words far{0, 0};
    uint32_t place = 0;
    Cube cube{};
    if constexpr (BIAS) {
        kc = voxel_clamp(kc);
        cube = columns_cube(kc, live, box);
        cube.place(kc, place);
        far = voxel_words(kc);
    }
    auto store = [&](int s) __attribute__((always_inline)) {
        sq.store(lq[s], tid);
        sd.store(ld[s], tid);
        if (tid < KT) {
            // a row past the end has no weight: its lse counts as infinite
            const bool in = tid < got;
            const float e = in ? kUp<DT> - row_lse(rl) : -INFINITY;
            lr[s][0][tid] = CAP ? e + capped.lift : AFTER ? e : e * inv_cs;
            lr[s][1][tid] = -rd;
            if constexpr (BIAS) lc.put(s, tid, cq, in, cube);
        }
    };
    constexpr float down = DT == SPV_F16 ? 1.f / 4096.f : 1.f;  // 2^-kUp
    int up = DT == SPV_F16 ? kUpMost : 0;
    float lift_z = __builtin_amdgcn_ldexpf(down, up), none[1] = {0.f};  // 2^up, less the weights' kUp
    f32x16 ok[T::NB], ov[T::NB];
#pragma unroll
    for (int b = 0; b < T::NB; ++b) ok[b] = ov[b] = f32x16{};
    if (t0 < t1) {
        store(0);
        if (t0 + 1 < t1) load();
    }
    __syncthreads();
    for (int i = t0; i < t1; ++i) {
        const int s = (i - t0) & 1;
        const int row0 = RT * kw;  // the wave's rows of the tile
        if (busy && i_now * KT + row0 < rows) {
            float slope = 0.f, lift = 0.f;
            if constexpr (BIAS) {
                slope = in_vgpr(a.slopes[kh * G + g_now] * kLog2e);
                lift = slope * 8388608.f;
            }
            f32x16 z[KS], d[KS], rest[AFTER ? KS : 1];
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                z[u] = row_values(&lr[s][0][row0 + 32 * u], h);
                d[u] = row_values(&lr[s][1][row0 + 32 * u], h);
                if constexpr (AFTER) {
                    rest[u] = z[u];
                    z[u] = f32x16{};
                }
                z[u] = T::rows_dot(lq[s] + (row0 + 32 * u) * T::LD, lane, kf, z[u]);
                d[u] = T::rows_dot(ld[s] + (row0 + 32 * u) * T::LD, lane, vf, d[u]);
            }
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                f32x16 p;
                auto grad = [&](int r, float b) __attribute__((always_inline)) {
                    if constexpr (CAP) {
                        float bend;
                        const float x = capped(z[u][r], b + rest[AFTER ? u : 0][r], &bend);
                        p[r] = __builtin_amdgcn_exp2f(x);
                        z[u][r] = p[r] * d[u][r] * bend;
                    } else {
                        const float y = AFTER ? (BIAS ? b + rest[u][r] : rest[u][r]) : b;
                        p[r] = __builtin_amdgcn_exp2f(AFTER || BIAS ? fmaf(z[u][r], cs, y) : z[u][r] * cs);
                        z[u][r] = p[r] * d[u][r];
                    }
                    if constexpr (DT == SPV_F16) z[u][r] *= lift_z;
                };
                if constexpr (BIAS)
                    lc.bias(s, row0 + 32 * u, h, far, place, slope, lift, grad);
                else
#pragma unroll
                    for (int r = 0; r < 16; ++r) grad(r, 0.f);
                T::add_weighted(ld[s] + (row0 + 32 * u) * T::LD, lane, T::weights(p), ov);
                if constexpr (DT == SPV_F16)
                    if (lower(z[u], ok, up, none)) lift_z = __builtin_amdgcn_ldexpf(down, up);
                T::add_weighted(lq[s] + (row0 + 32 * u) * T::LD, lane, T::weights(z[u]), ok);
            }
        }
        if (++i_now == tiles) i_now = 0, ++g_now;
        if (i + 1 < t1) {
            store(s ^ 1);
            if (next < t1) load();
        }
        __syncthreads();
    }
    if constexpr (DT == SPV_F16) scale_back(ok, up);
    if constexpr (KW > 1) {
        // the waves of a block of columns add up (the tiles' LDS is free by now)
        static_assert(2 * KT * T::LD >= CW * (KW - 1) * T::NB * 16 * 256, "a wave's sums have room");
        constexpr int N = T::NB * 16 * 64;
        float* pk = (float*)&lq[0][0] + cw * (KW - 1) * N;
        float* pv = (float*)&ld[0][0] + cw * (KW - 1) * N;
        if (kw) {
            lds_put(pk + (kw - 1) * N, lane, ok);
            lds_put(pv + (kw - 1) * N, lane, ov);
        }
        __syncthreads();
        if (kw) return;
#pragma unroll
        for (int w = 1; w < KW; ++w) {
            lds_add(pk + (w - 1) * N, lane, 1.f, ok);
            lds_add(pv + (w - 1) * N, lane, 1.f, ov);
        }
    }
    if (!live) return;
    const float f = a.scale * kBend<CAP>;
    if (a.part) {
        const int64_t at = (((int64_t)sh.part * a.nk + kj) * a.K + kh) * a.D;
        const int64_t half = (int64_t)sh.parts * a.nk * a.K * a.D;
        Tile<SPV_F32, DP>::store_cols(a.part, at, a.D, h, ok, f);
        Tile<SPV_F32, DP>::store_cols(a.part, half + at, a.D, h, ov, down);
    } else {
        T::store_cols(a.dk, kj * a.lddk + (int64_t)kh * a.D, a.D, h, ok, f);
        T::store_cols(a.dv, kj * a.lddv + (int64_t)kh * a.D, a.D, h, ov, down);
    }
}

// the parts of rows [n][heads][D], added in their order, to dst; four channels a thread
template <int DT>
__global__ __launch_bounds__(256) void k_attn_add_parts(const float* __restrict__ part, int parts, int64_t n, int heads,
                                                        int D, const int32_t* __restrict__ off, int B,
                                                        void* __restrict__ dst, int64_t ld) {
    const int w = heads * D / 4;
    const int64_t id = blockIdx.x * (int64_t)256 + threadIdx.x, i = id / w;
    if (i >= n || i < off[0] || i >= off[B]) return;  // past the end, or a row of no scan
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int q = 0; q < parts; ++q) {
        const float4 p = *(const float4*)(part + ((int64_t)q * n * w + id) * 4);
        s.x += p.x, s.y += p.y, s.z += p.z, s.w += p.w;
    }
    const int64_t at = i * ld + (id - i * w) * 4;
    if constexpr (DT == SPV_F32) *(float4*)((float*)dst + at) = s;
    else *(uint2*)((uint16_t*)dst + at) = make_uint2(pack2<DT>(s.x, s.y), pack2<DT>(s.z, s.w));
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static AttnShape dq_shape(const AttnArgs& a) {
    return attn_shape(a.dt, attn_dp(a.D), a.nq, a.H / a.K, a.B, a.K, a.nk / (a.B < 1 ? 1 : a.B));
}
static AttnShape dkv_shape(const AttnArgs& a) {
    return attn_shape(a.dt, attn_dp(a.D), a.nk, 1, a.B, a.K, a.nq / (a.B < 1 ? 1 : a.B) * (a.H / a.K));
}

void plan_attention_backward_ws(Arena& a, AttnArgs& t) {
    t.delta = a.take<float>((size_t)t.nq * (size_t)t.H);
    const AttnShape q = dq_shape(t), k = dkv_shape(t);
    // the two kernels use the parts one after the other
    const size_t rows = q.parts > 1 ? (size_t)q.parts * (size_t)t.nq * (size_t)t.H : 0;
    const size_t pq = rows * (size_t)t.D * (t.dt == SPV_F32 ? 1 : 2);
    const size_t pk = k.parts > 1 ? (size_t)k.parts * (size_t)t.nk * (size_t)t.K * (size_t)t.D * 2 : 0;
    if (pq || pk) t.part = a.take<float>(pq > pk ? pq : pk);
    if (rows && t.dt != SPV_F32) t.part_ml = a.take<float>(4 * rows);
}

template <int DT, int DP, int KW, bool BIAS, int CAP>
static void launch_side(hipStream_t s, const AttnArgs& a, const AttnShape& sh, bool keys) {
    const dim3 g = attn_grid(sh, a.K);
    if (keys) k_attn_dkv<DT, DP, KW, BIAS, CAP><<<g, 256, 0, s>>>(a);
    else k_attn_dq<DT, DP, KW, BIAS, CAP><<<g, 256, 0, s>>>(a);
}
template <int DT, int DP, int KW>
static void launch_kw(hipStream_t s, const AttnArgs& a, const AttnShape& sh, bool keys) {
    const int cap = attn_cap(a);
    if (a.slopes && cap == kCapQuick) launch_side<DT, DP, KW, true, kCapQuick>(s, a, sh, keys);
    else if (a.slopes && cap) launch_side<DT, DP, KW, true, kCapExact>(s, a, sh, keys);
    else if (a.slopes) launch_side<DT, DP, KW, true, kNoCap>(s, a, sh, keys);
    else if (cap == kCapQuick) launch_side<DT, DP, KW, false, kCapQuick>(s, a, sh, keys);
    else if (cap) launch_side<DT, DP, KW, false, kCapExact>(s, a, sh, keys);
    else launch_side<DT, DP, KW, false, kNoCap>(s, a, sh, keys);
}
template <int DT, int DP>
static void launch_dp(hipStream_t s, const AttnArgs& a, const AttnShape& sh, bool keys) {
    constexpr int K1 = attn_kw(DT, DP, 1), K2 = attn_kw(DT, DP, 2);
    if (K2 > 1 && sh.mode == 2) launch_kw<DT, DP, K2>(s, a, sh, keys);
    else if (K1 > 1 && sh.mode == 1) launch_kw<DT, DP, K1>(s, a, sh, keys);
    else launch_kw<DT, DP, 1>(s, a, sh, keys);
}
template <int DT>
static void backward_dt(hipStream_t s, const AttnArgs& a, bool keys) {
    const AttnShape sh = keys ? dkv_shape(a) : dq_shape(a);
    AttnArgs t = a;
    if (sh.parts < 2) t.part = nullptr;
    switch (attn_dp(a.D)) {
        case 32: launch_dp<DT, 32>(s, t, sh, keys); break;
        case 64: launch_dp<DT, 64>(s, t, sh, keys); break;
        case 96: launch_dp<DT, 96>(s, t, sh, keys); break;
        case 128: launch_dp<DT, 128>(s, t, sh, keys); break;
    }
    if (sh.parts < 2) return;
    if (!keys && DT != SPV_F32) {
        if constexpr (DT != SPV_F32) k_attn_dq_join<DT><<<blocks_for(a.nq * a.H * a.D / 4, 256), 256, 0, s>>>(a, sh.parts);
        return;
    }
    if (!keys) {
        k_attn_add_parts<DT><<<blocks_for(a.nq * a.H * a.D / 4, 256), 256, 0, s>>>(a.part, sh.parts, a.nq, a.H, a.D,
                                                                                   a.q_off, a.B, a.dq, a.lddq);
        return;
    }
    const unsigned g = blocks_for(a.nk * a.K * a.D / 4, 256);
    const float* pv = a.part + (int64_t)sh.parts * a.nk * a.K * a.D;
    k_attn_add_parts<DT><<<g, 256, 0, s>>>(a.part, sh.parts, a.nk, a.K, a.D, a.k_off, a.B, a.dk, a.lddk);
    k_attn_add_parts<DT><<<g, 256, 0, s>>>(pv, sh.parts, a.nk, a.K, a.D, a.k_off, a.B, a.dv, a.lddv);
}

void launch_attention_backward(hipStream_t s, const AttnArgs& a) {
    for (int keys = 0; keys < 2; ++keys) {  // delta comes from the first
        if ((keys ? a.nk : a.nq) == 0) continue;
        if (a.dt == SPV_F32) backward_dt<SPV_F32>(s, a, keys);
        else if (a.dt == SPV_BF16) backward_dt<SPV_BF16>(s, a, keys);
        else backward_dt<SPV_F16>(s, a, keys);
    }
}

}  // namespace spv
