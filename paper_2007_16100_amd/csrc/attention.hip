// attention.hip -- attention over packed scans, forward:
//   s_ij = cap(scale q_i . k_j) - slope_h |c_i - c_j|_1,  j over the keys of i's scan,
//   out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(s_ij - m_i)
// in one pass over the keys with a running reference m and a running sum.
#include "attn_common.hpp"

namespace spv {

// Columns are (query, head of a key head's group) pairs, so shared key heads are staged once for all of their query
// heads; a workgroup takes the columns of one scan and one key head.  Scores are kept in units of log 2.  A column's
// reference m moves (and the sums are scaled) only when a score passes it by more than kLead: weights of up to
// 2^kLead lose nothing in float32 sums or 16-bit weights, and after the first tiles m hardly ever moves.  It moves to kLift
// below the score: in float16 the largest weights are 2^7 to 2^15, and those of 2^-21 of the largest still normal numbers.
// The bias, over scale, is what the products are added to, unless a cap's tanh stands between them or (float32) D roundings
// at the bias's size would show: 400 voxels from every key, at a slope of a half, out was off by up to 7e-5 so, by 6e-6
// with the bias added after the product.
//
// In 16 bits the weights are rounded to the type before they multiply the values, and the sum they are divided by is of
// the rounded ones: out of bf16 is off by 2.1e-3 (one query over 88,119 keys 2.4e-3) in the root of the mean square against
// 64 bits, its own last rounding alone by 1.7e-3.  Two halves of a weight would leave that alone, for half of the products
// again and two more instructions a score.
//
// In 16 bits at 32 channels a score costs two matrix products of 32 channels but seven vector instructions (distance,
// bias, reference, exponential, maximum, sum, rounding), of which the exponential counts double.
// [3451, 3654, 1963, 2195] x 8 heads of 32, bf16, bias: 92 us, of which the scores' instructions take 50 - 60 and the
// products, beside them, 29.  The vector units are busy 70% of the time, the matrix units 17%; 720 workgroups leave 2.5
// waves a SIMD, of scans of unequal length, which wait at barriers and for each other's products.  (At [16384] x 8 heads
// the vector units were busy 82%.)
// Four scans of 26,881 in all x 4 heads of 64 on 2, f16, cap and bias: 475 us; a cap adds an exponential, a reciprocal
// and three more instructions.  One query over 88,119 keys x 8 heads of 32: 18 us in 64 parts, 3.8 TB/s with the join.
// 211 x 3 heads in float32: 9.5 us a call.  [1457, 1544] x 3 heads in float32, cap and bias: 48 us, where 285 workgroups
// lie on 256 units, one wave to a SIMD: its products (36% of the cycles), its vector instructions (23%) and the waits for
// LDS and memory follow one another.
template <int DT>
constexpr float kLead = DT == SPV_F16 ? 15.f : 8.f;
template <int DT>
constexpr float kLift = DT == SPV_F16 ? 7.f : 0.f;
// A reference is base + m: base in the units that the products come in (of the scores, where the bias is added after), m in
// units of log 2.  One of up to kNear is all in m, and weights are exp2(z cs - m) in one step.  A larger one is a base, the
// largest z itself, and is taken off z first: rounded to a float, m = base cs would be off by more than the weights'
// range, the same for every key but enough to overflow or lose them all.
constexpr float kNear = 1024.f;
// the base of a column without a finite score so far: one of minus infinity has no weight under it, and any finite one
// passes it
constexpr float kNoScore = -3.402823466e38f;
// what sums under several references are joined under, from the largest (in units of log 2) and the largest base
struct Reference {
    float base, m;
    __device__ Reference(float top, float top_base) {
        base = far(top) ? top_base : 0.f;
        m = far(top) ? 0.f : top;
    }
    // no reference without a base is as large, lifted or not
    static __device__ bool far(float top) { return !(fabsf(top) <= 2.f * kNear); }
    __device__ float factor(float b, float mm, float unit) const {
        return __builtin_amdgcn_exp2f(fmaf(b - base, unit, mm - m));
    }
};
// units of log 2 in one of the base's
__device__ inline float attn_unit(const AttnArgs& a) {
    return attn_after(a.dt, a.slopes, a.cap > 0.f) ? 1.f : a.scale * kLog2e;
}

// Waves per SIMD that the registers have to leave room for.  [8192] x 4 heads of 128 with two 217 us, with one 350;
// [16384] x 8 heads of 32 with four 621 us, with three 685.
constexpr int attn_waves(int dt, int DP) { return dt == SPV_F32 || DP > 64 ? 2 : 4; }

template <int DT, int DP, int KW, bool BIAS, int CAP>
__global__ __launch_bounds__(256, attn_waves(DT, DP)) void k_attn(AttnArgs a) {
    using T = Tile<DT, DP>;
    constexpr int RT = attn_rows(DT, DP, KW), KT = RT * KW, KS = RT / 32, CW = 4 / KW, BM = 32 * CW;
    constexpr bool AFTER = attn_after(DT, BIAS, CAP);  // z becomes the score, in units of log 2
    __shared__ __align__(16) char lk[2][KT * T::LD], lv[2][KT * T::LD];
    __shared__ __align__(16) Places<BIAS ? KT : 32> lc;
    __shared__ uint32_t box[4][3];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), cw = wave / KW, kw = wave % KW;
    const int c = lane & 31, h = lane >> 5;
    const Share sh = attn_share(a);
    const int G = a.H / a.K, kh = sh.kh;
    const ScanTile t = find_tile(a.q_off, a.nq, a.k_off, a.nk, a.B, G, BM, sh.tile);
    if (t.col0 >= t.cols) return;  // the whole workgroup
    const int64_t k0 = t.r0, k1 = t.r1;
    const int keys = (int)(k1 > k0 ? k1 - k0 : 0), tiles = keys / KT + (keys % KT != 0);
    const int per = (tiles + sh.parts - 1) / sh.parts, t0 = sh.part * per, t1 = t0 + per < tiles ? t0 + per : tiles;

    // the lane's column
    const bool busy = t.col0 + 32 * cw < t.cols, live = t.col0 + 32 * cw + c < t.cols;
    const int64_t q0 = t.col0 / G;
    const int x = (int)(t.col0 - q0 * G) + 32 * cw + c, head = kh * G + x % G;
    const int64_t qi = t.first + q0 + x / G;
    uint4 qf[T::NF];
    T::load_cols(a.q, qi * a.ldq + (int64_t)head * a.D, live, a.D, h, qf);
    const float cs = in_vgpr(a.scale * kLog2e);
    const Capped<CAP> capped(a);
    int4 qc{0, 0, 0, 0};
    float slope = 0.f;  // of the scores where the bias is added after, else of the products
    if constexpr (BIAS)
        if (live) {
            qc = *(const int4*)(a.q_coords + 4 * qi);
            slope = a.slopes[head];
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

    auto store = [&](int s) __attribute__((always_inline)) {
        sk.store(lk[s], tid);
        sv.store(lv[s], tid);
        if constexpr (BIAS)
            if (tid < KT) lc.put(s, tid, ck, tid < got, cube);
    };

    // weights of scores (relative to m already where they are AFTER) over their base
    auto weights = [](const f32x16& z, float cs, float m) __attribute__((always_inline)) {
        f32x16 p;
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(AFTER ? z[r] : fmaf(z[r], cs, -m));
        return T::weights(p);
    };
    f32x16 o[T::NB];
#pragma unroll
    for (int b = 0; b < T::NB; ++b) o[b] = f32x16{};
    float m = 0.f, base = kNoScore, l = 0.f;
    bool based = true;  // a column of the wave has a base
    if (t0 < t1) {
        store(0);
        if (t0 + 1 < t1) load();
    }
    __syncthreads();
    for (int i = t0; i < t1; ++i) {
        const int s = (i - t0) & 1;
        const int row0 = RT * kw, left = keys - i * KT - row0;  // the wave's rows of the tile, keys from there on
        if (busy && left > 0) {
            f32x16 z[KS];
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                f32x16 b{};
                if constexpr (BIAS && !AFTER)
                    lc.bias(s, row0 + 32 * u, h, far, place, slope, lift,
                            [&](int r, float x) __attribute__((always_inline)) { b[r] = x; });
                z[u] = T::rows_dot(lk[s] + (row0 + 32 * u) * T::LD, lane, qf, b);
            }
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                auto bend = [&](int r, float b) __attribute__((always_inline)) {
                    z[u][r] = CAP ? capped(z[u][r], b + (capped.lift - m)) : fmaf(z[u][r], cs, b - m);
                };
                if constexpr (AFTER && BIAS)
                    lc.bias(s, row0 + 32 * u, h, far, place, slope, lift, bend);
                else if constexpr (CAP)
#pragma unroll
                    for (int r = 0; r < 16; ++r) bend(r, 0.f);
                const int end = left - 32 * u;
                if (end < 32) {  // keys past the scan's end
                    asm volatile("");  // a branch: selects on every tile cost two instructions a score
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r / 4) + 4 * h + r % 4 >= end) z[u][r] = -INFINITY;
                }
                float top = z[u][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) top = fmaxf(top, z[u][r]);
                if (__any((AFTER ? top - base : fmaf(top - base, cs, -m)) > kLead<DT>)) {
                    top = half_max(top);
                    const float past = AFTER ? top - base : fmaf(top - base, cs, -m), old_m = m, old_base = base;
                    if (past > kLead<DT>) {
                        const float to = AFTER ? top + m : top * cs;
                        const bool near = fabsf(to) <= kNear;
                        m = near ? to - kLift<DT> : 0.f;
                        base = near ? 0.f : AFTER ? to : top;
                    }
                    const float f = __builtin_amdgcn_exp2f(fmaf(old_base - base, AFTER ? 1.f : cs, old_m - m));
                    based = __any(base != 0.f);
                    l *= f;
#pragma unroll
                    for (int b = 0; b < T::NB; ++b)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[b][r] *= f;
                    if constexpr (AFTER)
#pragma unroll
                        for (int r = 0; r < 16; ++r) z[u][r] += old_m - m;
                }
                if (based) {
                    asm volatile("");  // a branch: it is hardly ever taken after the first rows
#pragma unroll
                    for (int r = 0; r < 16; ++r) z[u][r] -= base;
                }
                const typename T::Weights w = weights(z[u], cs, m);
                l = T::sum(w, l);
                T::add_weighted(lv[s] + (row0 + 32 * u) * T::LD, lane, w, o);
            }
        }
        if (i + 1 < t1) {
            store(s ^ 1);
            if (i + 2 < t1) load();
        }
        __syncthreads();
    }
    l = half_sum(l);
    if constexpr (KW > 1) {
        // the waves of a block of columns join under their largest reference (the tiles' LDS is free by now)
        static_assert(2 * KT * T::LD >= CW * (KW - 1) * (T::NB * 16 + 3) * 256, "a wave's sums have room");
        constexpr int N = (T::NB * 16 + 3) * 64;
        float* p = (float*)&lk[0][0] + (cw * (KW - 1) + kw - 1) * N;
        if (kw) {
            lds_put(p + 192, lane, o);
            p[lane] = m;
            p[64 + lane] = l;
            p[128 + lane] = base;
        }
        __syncthreads();
        if (kw) return;
        p += N;
        const float unit = AFTER ? 1.f : cs;
        float top = -INFINITY, top_base = kNoScore;
        auto count = [&](float m, float l, float base) __attribute__((always_inline)) {
            if (l != 0.f) top = fmaxf(top, fmaf(base, unit, m)), top_base = fmaxf(top_base, base);
        };
        count(m, l, base);
#pragma unroll
        for (int w = 0; w < KW - 1; ++w) count(p[w * N + lane], p[w * N + 64 + lane], p[w * N + 128 + lane]);
        const Reference to(top, top_base);
        const float f = l != 0.f ? to.factor(base, m, unit) : 0.f;
        l *= f;
#pragma unroll
        for (int b = 0; b < T::NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[b][r] *= f;
#pragma unroll
        for (int w = 0; w < KW - 1; ++w) {
            const float* pw = p + w * N;
            const float lw = pw[64 + lane];
            if (lw == 0.f) continue;  // both lanes of a column: no key among the wave's
            const float fw = to.factor(pw[128 + lane], pw[lane], unit);
            l = fmaf(fw, lw, l);
            lds_add(pw + 192, lane, fw, o);
        }
        m = to.m, base = to.base;
    }
    if (!live) return;
    const int64_t row = qi * a.H + head;
    if (a.part) {
        // one of the parts: sums as they are, in float32
        const int64_t at = (int64_t)sh.part * a.nq * a.H + row;
        if (h == 0) *(float4*)(a.part_ml + 4 * at) = make_float4(m, l, base, 0.f);
        if (l != 0.f) Tile<SPV_F32, DP>::store_cols(a.part, at * a.D, a.D, h, o, 1.f);  // else they are not read
        return;
    }
    T::store_cols(a.out, qi * a.ldo + (int64_t)head * a.D, a.D, h, o, l != 0.f ? 1.f / l : 0.f);
    if (a.lse && h == 0)
        a.lse[row] = l != 0.f ? fmaf(base, AFTER ? 1.f : cs, m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// The parts of a row joined under their largest reference: WR waves a row, a lane for each four channels of one of
// every NP parts, added in a fixed order.  Latency bounds it: 8 rows of 64 parts take 4.4 us, 320 rows of 16 4.8.
template <int DT, int WR>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a, int parts) {
    constexpr int RW = 4 / WR;  // rows a workgroup
    __shared__ float so[4][64][4], sl[4][64], sm[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rw = wave / WR, w = wave % WR;
    const int P4 = a.D <= 32 ? 8 : a.D <= 64 ? 16 : 32, NP = 64 / P4 * WR;
    const int64_t rows = a.nq * a.H, row = (int64_t)blockIdx.x * RW + rw, qi = row / a.H;
    // a row of no scan has no parts
    const bool on = row < rows && qi >= a.q_off[0] && qi < a.q_off[a.B];
    const float4* ml = (const float4*)a.part_ml + row;  // m, sum of weights, base
    const float unit = attn_unit(a);
    float m = -INFINITY, base = kNoScore;
    if (on)
        for (int s = lane + 64 * w; s < parts; s += 64 * WR) {
            const float4 v = ml[s * rows];
            if (v.y != 0.f) m = fmaxf(m, fmaf(v.z, unit, v.x)), base = fmaxf(base, v.z);
        }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
    if constexpr (WR > 1) {
        if (lane == 0) sm[wave] = m;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < WR; ++x) m = fmaxf(m, sm[rw * WR + x]);
    }
    if (Reference::far(m)) {  // the same in all of a row's waves
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) base = fmaxf(base, __shfl_xor(base, x, 64));
        if constexpr (WR > 1) {
            __syncthreads();
            if (lane == 0) sm[wave] = base;
            __syncthreads();
#pragma unroll
            for (int x = 0; x < WR; ++x) base = fmaxf(base, sm[rw * WR + x]);
        }
    }
    const Reference to(m, base);
    const int d = lane % P4 * 4;
    float l = 0.f;
    float o[4] = {};
    if (on && d < a.D) {
        constexpr int U = 4;  // parts in flight
        for (int s0 = lane / P4 + 64 / P4 * w; s0 < parts; s0 += U * NP) {
            float4 v[U];
            float4 p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int s = s0 + u * NP;
                v[u] = s < parts ? ml[s * rows] : make_float4(0.f, 0.f, 0.f, 0.f);
                // sums of no key are not written
                p[u] = v[u].y != 0.f ? *(const float4*)(a.part + (s * rows + row) * a.D + d)
                                     : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v[u].y == 0.f) continue;
                const float f = to.factor(v[u].z, v[u].x, unit);
                l = fmaf(f, v[u].y, l);
                o[0] = fmaf(f, p[u].x, o[0]);
                o[1] = fmaf(f, p[u].y, o[1]);
                o[2] = fmaf(f, p[u].z, o[2]);
                o[3] = fmaf(f, p[u].w, o[3]);
            }
        }
    }
    for (int x = P4; x < 64; x <<= 1) {
        l += __shfl_xor(l, x, 64);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], x, 64);
    }
    if constexpr (WR > 1) {
        sl[wave][lane] = l;
#pragma unroll
        for (int e = 0; e < 4; ++e) so[wave][lane][e] = o[e];
        __syncthreads();
        if (w) return;
        for (int x = 1; x < WR; ++x) {
            l += sl[rw * WR + x][lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += so[rw * WR + x][lane][e];
        }
    }
    if (!on || lane >= P4 || d >= a.D) return;
    const float f = l != 0.f ? 1.f / l : 0.f;
    const int64_t at = qi * a.ldo + (row - qi * a.H) * a.D + d;
    if constexpr (DT == SPV_F32)
        *(float4*)((float*)a.out + at) = make_float4(o[0] * f, o[1] * f, o[2] * f, o[3] * f);
    else
        *(uint2*)((uint16_t*)a.out + at) = make_uint2(pack2<DT>(o[0] * f, o[1] * f), pack2<DT>(o[2] * f, o[3] * f));
    if (a.lse && lane == 0)
        a.lse[row] = l != 0.f ? fmaf(to.base, unit, to.m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static AttnShape forward_shape(const AttnArgs& a) {
    return attn_shape(a.dt, attn_dp(a.D), a.nq, a.H / a.K, a.B, a.K, a.nk / (a.B < 1 ? 1 : a.B));
}

bool attention_supported(const AttnArgs& a) {
    const int G = a.H / a.K;
    return attn_tiles(a.nq, a.B, G, 32) * a.K <= kMaxWorkgroups && attn_tiles(a.nk, a.B, 1, 32) * a.K <= kMaxWorkgroups;
}

void plan_attention_ws(Arena& a, AttnArgs& t) {
    const AttnShape s = forward_shape(t);
    if (s.parts < 2) return;
    const size_t rows = (size_t)s.parts * (size_t)t.nq * (size_t)t.H;
    t.part_ml = a.take<float>(4 * rows);
    t.part = a.take<float>(rows * (size_t)t.D);
}

template <int DT, int DP, int KW>
static void attn_launch(hipStream_t s, const AttnArgs& a, const AttnShape& sh) {
    const dim3 g = attn_grid(sh, a.K);
    const int cap = attn_cap(a);
    if (a.slopes && cap == kCapQuick) k_attn<DT, DP, KW, true, kCapQuick><<<g, 256, 0, s>>>(a);
    else if (a.slopes && cap) k_attn<DT, DP, KW, true, kCapExact><<<g, 256, 0, s>>>(a);
    else if (a.slopes) k_attn<DT, DP, KW, true, kNoCap><<<g, 256, 0, s>>>(a);
    else if (cap == kCapQuick) k_attn<DT, DP, KW, false, kCapQuick><<<g, 256, 0, s>>>(a);
    else if (cap) k_attn<DT, DP, KW, false, kCapExact><<<g, 256, 0, s>>>(a);
    else k_attn<DT, DP, KW, false, kNoCap><<<g, 256, 0, s>>>(a);
}
template <int DT, int DP>
static void attn_dp_launch(hipStream_t s, const AttnArgs& a, const AttnShape& sh) {
    constexpr int K1 = attn_kw(DT, DP, 1), K2 = attn_kw(DT, DP, 2);
    if (K2 > 1 && sh.mode == 2) attn_launch<DT, DP, K2>(s, a, sh);
    else if (K1 > 1 && sh.mode == 1) attn_launch<DT, DP, K1>(s, a, sh);
    else attn_launch<DT, DP, 1>(s, a, sh);
}
template <int DT>
static void attn_dt(hipStream_t s, const AttnArgs& a) {
    const AttnShape sh = forward_shape(a);
    switch (attn_dp(a.D)) {
        case 32: attn_dp_launch<DT, 32>(s, a, sh); break;
        case 64: attn_dp_launch<DT, 64>(s, a, sh); break;
        case 96: attn_dp_launch<DT, 96>(s, a, sh); break;
        case 128: attn_dp_launch<DT, 128>(s, a, sh); break;
    }
    if (sh.parts > 16) k_attn_join<DT, 4><<<blocks_for(a.nq * a.H, 1), 256, 0, s>>>(a, sh.parts);
    else if (sh.parts > 1) k_attn_join<DT, 1><<<blocks_for(a.nq * a.H, 4), 256, 0, s>>>(a, sh.parts);
}

void launch_attention(hipStream_t s, const AttnArgs& a) {
    if (a.dt == SPV_F32) attn_dt<SPV_F32>(s, a);
    else if (a.dt == SPV_BF16) attn_dt<SPV_BF16>(s, a);
    else attn_dt<SPV_F16>(s, a);
}

}  // namespace spv
