// attention.hip -- attention over packed scans, forward:
//   s_ij = cap(scale q_i . k_j) - slope_h |c_i - c_j|_1,  j over the keys of i's scan,
//   out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(s_ij - m_i)
// in one pass over the keys with a running reference m and a running sum.
#include "attn_common.hpp"

namespace spv {

// Columns are (query, head of a key head's group) pairs, so shared key heads are staged once for all of their query
// heads; a workgroup takes 32 NW columns of one scan and one key head.  Scores are kept in units of log 2 and
// relative to the column's reference; the reference moves (and the sums are scaled) only when a score passes it by
// more than kLead: weights of up to 2^kLead lose nothing in float32 sums or 16-bit weights, and after the first
// tiles the reference hardly ever moves.
constexpr float kLead = 8.f;


// waves per SIMD that the registers have to leave room for
constexpr int attn_waves(int dt, int DP, int nw) { return nw == 1 || dt == SPV_F32 || DP > 64 ? 1 : DP > 32 ? 4 : 3; }

template <int DT, int DP, int NW, bool BIAS, bool CAP>
__global__ __launch_bounds__(64 * NW, attn_waves(DT, DP, NW)) void k_attn(AttnArgs a) {
    using T = Tile<DT, DP>;
    constexpr int KT = attn_rows(DT, DP), KS = KT / 32, TH = 64 * NW, CB = 1, WC = 32 * CB, BM = WC * NW;
    // the reference goes into the products' accumulator, where no tanh stands between them
    constexpr bool FOLD = DT != SPV_F32 && !CAP;
    __shared__ __align__(16) char lk[2][KT * T::LD], lv[2][KT * T::LD];
    __shared__ __align__(16) uint32_t lc[2][2][BIAS ? KT : 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), c = lane & 31, h = lane >> 5;
    const int G = a.H / a.K, kh = (int)(blockIdx.x % (unsigned)a.K);
    const ScanTile t = find_tile(a.q_off, a.B, a.nq, G, BM, blockIdx.x / (unsigned)a.K);
    if (t.col0 >= t.cols) return;  // the whole workgroup
    const int64_t k0 = uniform(clamp_off(a.k_off[t.b], a.nk)), k1 = uniform(clamp_off(a.k_off[t.b + 1], a.nk));
    const int64_t tiles = k1 > k0 ? (k1 - k0 + KT - 1) / KT : 0, per = (tiles + gridDim.y - 1) / gridDim.y;
    const int64_t t0 = blockIdx.y * per, t1 = t0 + per < tiles ? t0 + per : tiles;

    // the lane's columns
    const float cs = a.scale * kLog2e, inv_cs = 1.f / cs;
    const float cz = CAP ? 2.f * kLog2e * a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;
    const bool busy = t.col0 + WC * wave < t.cols;
    const int64_t q0 = t.col0 / G;
    int64_t qi[CB];
    int head[CB];
    bool live[CB];
    uint4 qf[CB][T::NF];
    Voxel qc[CB];
    float slope[CB], lift[CB];  // lift: what the 2^23 of a distance brings too much
#pragma unroll
    for (int n = 0; n < CB; ++n) {
        const int x = WC * wave + 32 * n + c, y = (int)(t.col0 - q0 * G) + x;
        live[n] = t.col0 + x < t.cols;
        qi[n] = t.first + q0 + y / G;
        head[n] = kh * G + y % G;
        T::load_cols(a.q, qi[n] * a.ldq + (int64_t)head[n] * a.D, live[n], a.D, h, qf[n]);
        qc[n] = Voxel{0, 0};
        slope[n] = lift[n] = 0.f;
        if (BIAS && live[n]) {
            qc[n] = voxel_of(*(const int4*)(a.q_coords + 4 * qi[n]));
            slope[n] = a.slopes[head[n]] * kLog2e;
            lift[n] = slope[n] * 8388608.f;
        }
    }

    Stage<DT, DP, KT, TH> sk, sv;
    int4 ck{0, 0, 0, 0};
    auto load = [&](int64_t i) __attribute__((always_inline)) {
        const int64_t r = k0 + i * KT;
        sk.load(a.k, a.ldk, (int64_t)kh * a.D, r, k1, a.D, tid);
        sv.load(a.v, a.ldv, (int64_t)kh * a.D, r, k1, a.D, tid);
        if constexpr (BIAS)
            if (tid < KT && r + tid < k1) ck = *(const int4*)(a.k_coords + 4 * (r + tid));
    };
    auto store = [&](int s) __attribute__((always_inline)) {
        sk.store(lk[s], tid);
        sv.store(lv[s], tid);
        if constexpr (BIAS)
            if (tid < KT) {
                const Voxel v = voxel_of(ck);
                lc[s][0][tid] = v.xy;
                lc[s][1][tid] = v.z;
            }
    };

    f32x16 o[CB][T::NB], ref[CB];  // ref: -reference / cs in every register (FOLD)
    float m[CB], l[CB];
#pragma unroll
    for (int n = 0; n < CB; ++n) {
#pragma unroll
        for (int b = 0; b < T::NB; ++b) o[n][b] = f32x16{};
        ref[n] = f32x16{};
        m[n] = l[n] = 0.f;
    }
    if (t0 < t1) {
        load(t0);
        store(0);
        if (t0 + 1 < t1) load(t0 + 1);
    }
    __syncthreads();
    for (int64_t i = t0; i < t1; ++i) {
        const int s = (int)(i - t0) & 1;
        if (busy) {
            f32x16 z[KS][CB];
            float d[CB];
#pragma unroll
            for (int u = 0; u < KS; ++u) {
#pragma unroll
                for (int n = 0; n < CB; ++n) z[u][n] = FOLD ? ref[n] : f32x16{};
                T::rows_dot(lk[s] + 32 * u * T::LD, lane, qf, z[u]);
            }
#pragma unroll
            for (int u = 0; u < KS; ++u)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t xy[4] = {}, zz[4] = {};
                    if constexpr (BIAS) {
                        lds_words(&lc[s][0][32 * u + 8 * q + 4 * h], xy);
                        lds_words(&lc[s][1][32 * u + 8 * q + 4 * h], zz);
                    }
#pragma unroll
                    for (int n = 0; n < CB; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float b = 0.f;
                            if constexpr (BIAS)
                                b = fmaf(voxel_dist(xy[e], zz[e], qc[n].xy, qc[n].z), -slope[n], lift[n]);
                            float y = z[u][n][4 * q + e];
                            if constexpr (CAP && DT == SPV_F32) {
                                y = fmaf(cap2, tanhf(y * (a.scale / a.cap)), b - m[n]);
                            } else if constexpr (CAP) {
                                // cap tanh(w) = cap - 2 cap / (exp(2 w) + 1)
                                const float ex = __builtin_amdgcn_exp2f(y * cz);
                                y = fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(ex + 1.f), b + (cap2 - m[n]));
                            } else if constexpr (FOLD) {
                                y = BIAS ? fmaf(y, cs, b) : y * cs;
                            } else {
                                y = fmaf(y, cs, b) - m[n];
                            }
                            z[u][n][4 * q + e] = y;
                        }
                }
            if (k0 + (i + 1) * KT > k1) {  // keys past the scan's end
                const int end = (int)(k1 - k0 - i * KT);
                asm volatile("");  // a branch: selects on every tile cost two instructions a score
#pragma unroll
                for (int u = 0; u < KS; ++u)
#pragma unroll
                    for (int n = 0; n < CB; ++n)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (32 * u + 8 * (r / 4) + 4 * h + r % 4 >= end) z[u][n][r] = -INFINITY;
            }
            bool ahead = i == t0;
#pragma unroll
            for (int n = 0; n < CB; ++n) {
                d[n] = -INFINITY;
#pragma unroll
                for (int u = 0; u < KS; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) d[n] = fmaxf(d[n], z[u][n][r]);
                ahead = ahead || d[n] > kLead;
            }
            if (__any(ahead)) {
#pragma unroll
                for (int n = 0; n < CB; ++n) {
                    const bool first = i == t0;
                    const float dn = half_max(d[n]), up = first || dn > kLead ? dn : 0.f;
                    const float f = first ? 1.f : __builtin_amdgcn_exp2f(-up);
                    m[n] += up;
                    l[n] *= f;
#pragma unroll
                    for (int b = 0; b < T::NB; ++b)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[n][b][r] *= f;
#pragma unroll
                    for (int u = 0; u < KS; ++u)
#pragma unroll
                        for (int r = 0; r < 16; ++r) z[u][n][r] -= up;
                    if constexpr (FOLD)
#pragma unroll
                        for (int r = 0; r < 16; ++r) ref[n][r] = -m[n] * inv_cs;
                }
            }
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                typename T::Weights w[CB];
#pragma unroll
                for (int n = 0; n < CB; ++n) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) z[u][n][r] = __builtin_amdgcn_exp2f(z[u][n][r]);
                    w[n] = T::weights(z[u][n]);
                    l[n] = T::sum(w[n], l[n]);
                }
                T::add_weighted(lv[s] + 32 * u * T::LD, lane, w, o);
            }
        }
        if (i + 1 < t1) {
            store(s ^ 1);
            if (i + 2 < t1) load(i + 2);
        }
        __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < CB; ++n) {
        const float ln = half_sum(l[n]);
        if (!live[n]) continue;
        const int64_t row = qi[n] * a.H + head[n];
        if (a.part) {
            // one of gridDim.y parts: sums as they are, in float32
            const int64_t at = (int64_t)blockIdx.y * a.nq * a.H + row;
            if (h == 0) *(float2*)(a.part_ml + 2 * at) = make_float2(m[n], ln);
            // without a key they are not read
            if (ln != 0.f) Tile<SPV_F32, DP>::store_cols(a.part, at * a.D, a.D, h, o[n], 1.f);
            continue;
        }
        T::store_cols(a.out, qi[n] * a.ldo + (int64_t)head[n] * a.D, a.D, h, o[n], tiles ? 1.f / ln : 0.f);
        if (a.lse && h == 0) a.lse[row] = tiles ? (m[n] + __builtin_amdgcn_logf(ln)) * kLn2 : -INFINITY;
    }
}

// the parts of a row, added in their order under the largest reference; four channels a thread
template <int DT>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a, int parts) {
    const int D4 = a.D / 4;
    const int64_t id = blockIdx.x * (int64_t)256 + threadIdx.x, rows = a.nq * a.H, row = id / D4;
    if (row >= rows) return;
    const int d = (int)(id - row * D4) * 4;
    const int64_t qi = row / a.H;
    if (qi < a.q_off[0] || qi >= a.q_off[a.B]) return;  // a row of no scan
    float m = -INFINITY;
    for (int s = 0; s < parts; ++s) {
        const float2 ml = *(const float2*)(a.part_ml + 2 * (s * rows + row));
        if (ml.y != 0.f) m = fmaxf(m, ml.x);
    }
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < parts; ++s) {
        const float2 ml = *(const float2*)(a.part_ml + 2 * (s * rows + row));
        if (ml.y == 0.f) continue;
        const float f = __builtin_amdgcn_exp2f(ml.x - m);
        const float4 p = *(const float4*)(a.part + (s * rows + row) * a.D + d);
        l = fmaf(f, ml.y, l);
        o.x = fmaf(f, p.x, o.x);
        o.y = fmaf(f, p.y, o.y);
        o.z = fmaf(f, p.z, o.z);
        o.w = fmaf(f, p.w, o.w);
    }
    const float f = l != 0.f ? 1.f / l : 0.f;
    const int64_t at = qi * a.ldo + (row - qi * a.H) * a.D + d;
    if constexpr (DT == SPV_F32)
        *(float4*)((float*)a.out + at) = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
    else
        *(uint2*)((uint16_t*)a.out + at) = make_uint2(pack2<DT>(o.x * f, o.y * f), pack2<DT>(o.z * f, o.w * f));
    if (a.lse && d == 0) a.lse[row] = l != 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// ---------------------------------------------------------------------------
// host: the shape of a launch
// ---------------------------------------------------------------------------
static AttnShape attn_shape(const AttnArgs& a) {
    const int G = a.H / a.K, B = a.B < 1 ? 1 : a.B;
    AttnShape s{4, 1, attn_tiles(a.nq, a.B, G, 128)};
    // 128 columns a workgroup while that gives every CU one and the scans fill them
    if (s.tiles * a.K < 256 || a.nq * G / B < 64) s = AttnShape{1, 1, attn_tiles(a.nq, a.B, G, 32)};
    // keys in parts of at least four tiles (of the average scan) while there are under four waves a CU
    const int KT = attn_rows(a.dt, attn_dp(a.D));
    const int64_t wgs = s.tiles * a.K * s.nw, key_tiles = a.nk / B / KT;
    if (s.nw == 1 && wgs < 1024) {
        int64_t p = (2048 + wgs - 1) / (wgs < 1 ? 1 : wgs);
        if (p > key_tiles / 4) p = key_tiles / 4;
        if (p > 256) p = 256;
        s.parts = p < 2 ? 1 : (int)p;
    }
    return s;
}

bool attention_supported(const AttnArgs& a) {
    const int G = a.H / a.K;
    return attn_tiles(a.nq, a.B, G, 32) * a.K <= kMaxWorkgroups && attn_tiles(a.nk, a.B, G, 32) * a.K <= kMaxWorkgroups;
}

void plan_attention_ws(Arena& a, AttnArgs& t) {
    const AttnShape s = attn_shape(t);
    if (s.parts < 2) return;
    const size_t rows = (size_t)s.parts * (size_t)t.nq * (size_t)t.H;
    t.part_ml = a.take<float>(2 * rows);
    t.part = a.take<float>(rows * (size_t)t.D);
}

template <int DT, int DP, int NW>
static void attn_launch(hipStream_t s, const AttnArgs& a, const AttnShape& sh) {
    const dim3 g((unsigned)(sh.tiles * a.K), (unsigned)sh.parts);
    if (a.slopes && a.cap > 0.f) k_attn<DT, DP, NW, true, true><<<g, 64 * NW, 0, s>>>(a);
    else if (a.slopes) k_attn<DT, DP, NW, true, false><<<g, 64 * NW, 0, s>>>(a);
    else if (a.cap > 0.f) k_attn<DT, DP, NW, false, true><<<g, 64 * NW, 0, s>>>(a);
    else k_attn<DT, DP, NW, false, false><<<g, 64 * NW, 0, s>>>(a);
}
template <int DT, int DP>
static void attn_dp_launch(hipStream_t s, const AttnArgs& a, const AttnShape& sh) {
    if (sh.nw == 4) attn_launch<DT, DP, 4>(s, a, sh);
    else attn_launch<DT, DP, 1>(s, a, sh);
}
template <int DT>
static void attn_dt(hipStream_t s, const AttnArgs& a) {
    const AttnShape sh = attn_shape(a);
    switch (attn_dp(a.D)) {
        case 32: attn_dp_launch<DT, 32>(s, a, sh); break;
        case 64: attn_dp_launch<DT, 64>(s, a, sh); break;
        case 96: attn_dp_launch<DT, 96>(s, a, sh); break;
        case 128: attn_dp_launch<DT, 128>(s, a, sh); break;
    }
    if (sh.parts > 1) k_attn_join<DT><<<blocks_for(a.nq * a.H * (a.D / 4), 256), 256, 0, s>>>(a, sh.parts);
}

void launch_attention(hipStream_t s, const AttnArgs& a) {
    if (a.dt == SPV_F32) attn_dt<SPV_F32>(s, a);
    else if (a.dt == SPV_BF16) attn_dt<SPV_BF16>(s, a);
    else attn_dt<SPV_F16>(s, a);
}

}  // namespace spv
