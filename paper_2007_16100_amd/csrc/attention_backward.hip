// attention_backward.hip -- the backward of attention over packed scans:
//   p_ij = exp(s_ij - lse_i),  delta_i = dout_i . out_i,  dz_ij = p_ij (dout_i . v_j - delta_i) ds_ij/dz_ij
//   dq_i = scale sum_j dz_ij k_j,   dk_j = scale sum_i dz_ij q_i,   dv_j = sum_i p_ij dout_i
// Two kernels, each of which forms the weights anew: dq with the queries in the columns, as the forward has them (it
// also forms delta), and dk, dv with the keys in the columns.  One kernel for all three would save two products of
// seven, but either add dq in the order that workgroups happen to run in, or hold it for every part of the keys.
// lse and delta enter as the products' accumulators (dout . v - delta and, where no tanh stands between,
// q . k - lse / scale come out of the matrix cores).
#include "attn_common.hpp"

namespace spv {

// score (log 2 units, less the row's lse) and its slope by the product, from a product y
template <int DT, bool CAP>
struct Score {
    float cs, cz, cap2;
    __device__ explicit Score(const AttnArgs& a)
        : cs(a.scale * kLog2e), cz(CAP ? 2.f * kLog2e * a.scale / a.cap : 0.f), cap2(a.cap * kLog2e) {}
    static constexpr bool kFold = DT != SPV_F32 && !CAP;  // the products already hold -lse / cs
    // x: the score; the return value times kBend is d score / d (scale * product)
    __device__ float operator()(float y, float bias, float lse, float& x) const {
        if constexpr (CAP) {
            // t = 1 - 2 r with r = 1 / (exp(2 w) + 1): 1 - t^2 = 4 (r - r^2)
            const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * cz) + 1.f);
            x = fmaf(-2.f * cap2, r, bias + (cap2 - lse));
            return fmaf(-r, r, r);
        } else {
            x = kFold ? fmaf(y, cs, bias) : fmaf(y, cs, bias - lse);
            return 1.f;
        }
    }
    static constexpr float kBend = CAP ? 4.f : 1.f;
};

// waves per SIMD that the registers have to leave room for
constexpr int dq_waves(int dt, int DP, int nw) { return nw == 1 || dt == SPV_F32 || DP > 64 ? 1 : 2; }
constexpr int dkv_waves(int dt, int DP, int nw) { return nw == 1 || dt == SPV_F32 || DP > 64 ? 1 : 2; }

template <int DT, int DP, int NW, bool BIAS, bool CAP>
__global__ __launch_bounds__(64 * NW, dq_waves(DT, DP, NW)) void k_attn_dq(AttnArgs a) {
    using T = Tile<DT, DP>;
    using S = Score<DT, CAP>;
    constexpr int KT = 32, TH = 64 * NW, BM = 32 * NW;
    __shared__ __align__(16) char lk[2][KT * T::LD], lv[2][KT * T::LD];
    __shared__ __align__(16) uint32_t lc[2][2][BIAS ? KT : 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), c = lane & 31, h = lane >> 5;
    const Share sh = attn_share(a);
    const int G = a.H / a.K, kh = sh.kh;
    const ScanTile t = find_tile(a.q_off, a.B, a.nq, G, BM, sh.tile);
    if (t.col0 >= t.cols) return;  // the whole workgroup
    const int64_t k0 = uniform(clamp_off(a.k_off[t.b], a.nk)), k1 = uniform(clamp_off(a.k_off[t.b + 1], a.nk));
    const int64_t tiles = k1 > k0 ? (k1 - k0 + KT - 1) / KT : 0, per = (tiles + sh.parts - 1) / sh.parts;
    const int64_t t0 = sh.part * per, t1 = t0 + per < tiles ? t0 + per : tiles;

    const S score(a);
    const bool busy = t.col0 + 32 * wave < t.cols;
    const int64_t q0 = t.col0 / G;
    const int col = 32 * wave + c, y0 = (int)(t.col0 - q0 * G) + col;
    const bool live = t.col0 + col < t.cols;
    const int64_t qi = t.first + q0 + y0 / G;
    const int head = kh * G + y0 % G;
    uint4 qf[1][T::NF], df[1][T::NF];
    T::load_cols(a.q, qi * a.ldq + (int64_t)head * a.D, live, a.D, h, qf[0]);
    T::load_cols(a.dout, qi * a.lddo + (int64_t)head * a.D, live, a.D, h, df[0]);
    float lse = 0.f, delta = 0.f;
    {
        uint4 of[T::NF];
        T::load_cols(a.out, qi * a.ldo + (int64_t)head * a.D, live, a.D, h, of);
#pragma unroll
        for (int s = 0; s < T::NF; ++s) delta = T::frag_dot(df[0][s], of[s], delta);
        delta = half_sum(delta);
    }
    if (live) {
        lse = a.lse[qi * a.H + head] * kLog2e;
        if (h == 0 && sh.part == 0) a.delta[qi * a.H + head] = delta;
    }
    Voxel qc{0, 0};
    float slope = 0.f, lift = 0.f;
    if (BIAS && live) {
        qc = voxel_of(*(const int4*)(a.q_coords + 4 * qi));
        slope = a.slopes[head] * kLog2e;
        lift = slope * 8388608.f;
    }
    f32x16 zref, dref;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        zref[r] = S::kFold ? -lse / score.cs : 0.f;
        dref[r] = -delta;
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
    f32x16 o[1][T::NB];
#pragma unroll
    for (int b = 0; b < T::NB; ++b) o[0][b] = f32x16{};
    if (t0 < t1) {
        load(t0);
        store(0);
        if (t0 + 1 < t1) load(t0 + 1);
    }
    __syncthreads();
    for (int64_t i = t0; i < t1; ++i) {
        const int s = (int)(i - t0) & 1;
        if (busy) {
            f32x16 z[1] = {zref}, d[1] = {dref};
            T::rows_dot(lk[s], lane, qf, z);
            T::rows_dot(lv[s], lane, df, d);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t xy[4] = {}, zz[4] = {};
                if constexpr (BIAS) {
                    lds_words(&lc[s][0][8 * q + 4 * h], xy);
                    lds_words(&lc[s][1][8 * q + 4 * h], zz);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float b = 0.f, x;
                    if constexpr (BIAS) b = fmaf(voxel_dist(xy[e], zz[e], qc.xy, qc.z), -slope, lift);
                    const float bend = score(z[0][4 * q + e], b, lse, x);
                    float g = __builtin_amdgcn_exp2f(x) * d[0][4 * q + e];
                    if constexpr (CAP) g *= bend;
                    z[0][4 * q + e] = g;
                }
            }
            if (k0 + (i + 1) * KT > k1) {  // keys past the scan's end: their rows are zero, but not their weights
                const int end = (int)(k1 - k0 - i * KT);
                asm volatile("");  // a branch, not selects on every tile
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (8 * (r / 4) + 4 * h + r % 4 >= end) z[0][r] = 0.f;
            }
            const typename T::Weights w[1] = {T::weights(z[0])};
            T::add_weighted(lk[s], lane, w, o);
        }
        if (i + 1 < t1) {
            store(s ^ 1);
            if (i + 2 < t1) load(i + 2);
        }
        __syncthreads();
    }
    if (!live) return;
    const float f = a.scale * S::kBend;
    if (a.part)
        Tile<SPV_F32, DP>::store_cols(a.part, (((int64_t)sh.part * a.nq + qi) * a.H + head) * a.D, a.D, h, o[0], f);
    else
        T::store_cols(a.dq, qi * a.lddq + (int64_t)head * a.D, a.D, h, o[0], f);
}

// Columns are keys; the rows are the scan's queries, once for each head of the key head's group, in that order.
// The weights are at most 1 and, over long scans, far below float16's smallest normal number (6e-5): in that type they
// are multiplied as 2^12 p (and may be some times 1 where scores of millions round).  dz is not scaled: its size is that of dout, which a caller may have scaled up.
template <int DT>
constexpr float kUp = DT == SPV_F16 ? 12.f : 0.f;

template <int DT, int DP, int NW, bool BIAS, bool CAP>
__global__ __launch_bounds__(64 * NW, dkv_waves(DT, DP, NW)) void k_attn_dkv(AttnArgs a) {
    using T = Tile<DT, DP>;
    using S = Score<DT, CAP>;
    constexpr int KT = 32, TH = 64 * NW, BM = 32 * NW;
    __shared__ __align__(16) char lq[2][KT * T::LD], ld[2][KT * T::LD];
    __shared__ __align__(16) uint32_t lc[2][2][BIAS ? KT : 4];
    __shared__ __align__(16) float lr[2][2][KT];  // the rows' lse (as the score wants it) and -delta
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), c = lane & 31, h = lane >> 5;
    const Share sh = attn_share(a);
    const int G = a.H / a.K, kh = sh.kh;
    const ScanTile t = find_tile(a.k_off, a.B, a.nk, 1, BM, sh.tile);
    if (t.col0 >= t.cols) return;  // the whole workgroup
    const int64_t q0 = uniform(clamp_off(a.q_off[t.b], a.nq)), q1 = uniform(clamp_off(a.q_off[t.b + 1], a.nq));
    const int64_t tiles = q1 > q0 ? (q1 - q0 + KT - 1) / KT : 0, all = tiles * G;
    const int64_t per = (all + sh.parts - 1) / sh.parts;
    const int64_t t0 = sh.part * per, t1 = t0 + per < all ? t0 + per : all;

    const S score(a);
    const bool busy = t.col0 + 32 * wave < t.cols, live = t.col0 + 32 * wave + c < t.cols;
    const int64_t kj = t.first + t.col0 + 32 * wave + c;
    uint4 kf[1][T::NF], vf[1][T::NF];
    T::load_cols(a.k, kj * a.ldk + (int64_t)kh * a.D, live, a.D, h, kf[0]);
    T::load_cols(a.v, kj * a.ldv + (int64_t)kh * a.D, live, a.D, h, vf[0]);
    Voxel kc{0, 0};
    if (BIAS && live) kc = voxel_of(*(const int4*)(a.k_coords + 4 * kj));

    Stage<DT, DP, KT, TH> sq, sd;
    int4 cq{0, 0, 0, 0};
    float rl = 0.f, rd = 0.f;
    // tile i is number i % tiles of head i / tiles of the group
    auto load = [&](int64_t i) __attribute__((always_inline)) {
        const int64_t g = i / tiles, r = q0 + (i - g * tiles) * KT;
        const int64_t head = (int64_t)kh * G + g;
        sq.load(a.q, a.ldq, head * a.D, r, q1, a.D, tid);
        sd.load(a.dout, a.lddo, head * a.D, r, q1, a.D, tid);
        if (tid < KT) {
            const bool in = r + tid < q1;
            // a row past the end has no weight: its lse is infinite
            rl = in ? a.lse[(r + tid) * a.H + head] * kLog2e - kUp<DT> : INFINITY;
            rd = in ? -a.delta[(r + tid) * a.H + head] : 0.f;
            if constexpr (BIAS)
                if (in) cq = *(const int4*)(a.q_coords + 4 * (r + tid));
        }
    };
    auto store = [&](int s) __attribute__((always_inline)) {
        sq.store(lq[s], tid);
        sd.store(ld[s], tid);
        if (tid < KT) {
            lr[s][0][tid] = S::kFold ? -rl / score.cs : rl;
            lr[s][1][tid] = rd;
            if constexpr (BIAS) {
                const Voxel v = voxel_of(cq);
                lc[s][0][tid] = v.xy;
                lc[s][1][tid] = v.z;
            }
        }
    };
    constexpr float down = DT == SPV_F16 ? 1.f / 4096.f : 1.f;  // 2^-kUp
    f32x16 ok[1][T::NB], ov[1][T::NB];
#pragma unroll
    for (int b = 0; b < T::NB; ++b) ok[0][b] = ov[0][b] = f32x16{};
    if (t0 < t1) {
        load(t0);
        store(0);
        if (t0 + 1 < t1) load(t0 + 1);
    }
    __syncthreads();
    for (int64_t i = t0; i < t1; ++i) {
        const int s = (int)(i - t0) & 1;
        if (busy) {
            float slope = 0.f, lift = 0.f;
            if constexpr (BIAS) {
                slope = a.slopes[(int64_t)kh * G + i / tiles] * kLog2e;
                lift = slope * 8388608.f;
            }
            f32x16 z[1], d[1];
            float lse[16];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 x = *(const float4*)&lr[s][0][8 * q + 4 * h], y = *(const float4*)&lr[s][1][8 * q + 4 * h];
                lse[4 * q] = x.x, lse[4 * q + 1] = x.y, lse[4 * q + 2] = x.z, lse[4 * q + 3] = x.w;
                d[0][4 * q] = y.x, d[0][4 * q + 1] = y.y, d[0][4 * q + 2] = y.z, d[0][4 * q + 3] = y.w;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) z[0][r] = S::kFold ? lse[r] : 0.f;
            T::rows_dot(lq[s], lane, kf, z);
            T::rows_dot(ld[s], lane, vf, d);
            f32x16 p;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t xy[4] = {}, zz[4] = {};
                if constexpr (BIAS) {
                    lds_words(&lc[s][0][8 * q + 4 * h], xy);
                    lds_words(&lc[s][1][8 * q + 4 * h], zz);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 4 * q + e;
                    float b = 0.f, x;
                    if constexpr (BIAS) b = fmaf(voxel_dist(xy[e], zz[e], kc.xy, kc.z), -slope, lift);
                    const float bend = score(z[0][r], b, lse[r], x);
                    p[r] = __builtin_amdgcn_exp2f(x);
                    z[0][r] = p[r] * d[0][r];
                    if constexpr (CAP) z[0][r] *= bend;
                    if constexpr (DT == SPV_F16) z[0][r] *= down;
                }
            }
            const typename T::Weights wp[1] = {T::weights(p)}, wz[1] = {T::weights(z[0])};
            T::add_weighted(ld[s], lane, wp, ov);
            T::add_weighted(lq[s], lane, wz, ok);
        }
        if (i + 1 < t1) {
            store(s ^ 1);
            if (i + 2 < t1) load(i + 2);
        }
        __syncthreads();
    }
    if (!live) return;
    const float f = a.scale * S::kBend;
    if (a.part) {
        const int64_t at = (((int64_t)sh.part * a.nk + kj) * a.K + kh) * a.D;
        const int64_t half = (int64_t)sh.parts * a.nk * a.K * a.D;
        Tile<SPV_F32, DP>::store_cols(a.part, at, a.D, h, ok[0], f);
        Tile<SPV_F32, DP>::store_cols(a.part, half + at, a.D, h, ov[0], down);
    } else {
        T::store_cols(a.dk, kj * a.lddk + (int64_t)kh * a.D, a.D, h, ok[0], f);
        T::store_cols(a.dv, kj * a.lddv + (int64_t)kh * a.D, a.D, h, ov[0], down);
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
    const int G = a.H / a.K;
    return attn_shape(a.nq, G, a.B, a.K, a.nk / (a.B < 1 ? 1 : a.B) / 32);
}
static AttnShape dkv_shape(const AttnArgs& a) {
    const int G = a.H / a.K;
    return attn_shape(a.nk, 1, a.B, a.K, a.nq / (a.B < 1 ? 1 : a.B) / 32 * G);
}

void plan_attention_backward_ws(Arena& a, AttnArgs& t) {
    t.delta = a.take<float>((size_t)t.nq * (size_t)t.H);
    const AttnShape q = dq_shape(t), k = dkv_shape(t);
    // the two kernels use the parts one after the other
    const size_t pq = q.parts > 1 ? (size_t)q.parts * (size_t)t.nq * (size_t)t.H * (size_t)t.D : 0;
    const size_t pk = k.parts > 1 ? (size_t)k.parts * (size_t)t.nk * (size_t)t.K * (size_t)t.D * 2 : 0;
    if (pq || pk) t.part = a.take<float>(pq > pk ? pq : pk);
}

template <int DT, int DP, int NW, bool BIAS, bool CAP>
static void launch_side(hipStream_t s, const AttnArgs& a, const AttnShape& sh, bool keys) {
    const dim3 g = attn_grid(sh, a.K);
    if (keys) k_attn_dkv<DT, DP, NW, BIAS, CAP><<<g, 64 * NW, 0, s>>>(a);
    else k_attn_dq<DT, DP, NW, BIAS, CAP><<<g, 64 * NW, 0, s>>>(a);
}
template <int DT, int DP, int NW>
static void launch_nw(hipStream_t s, const AttnArgs& a, const AttnShape& sh, bool keys) {
    if (a.slopes && a.cap > 0.f) launch_side<DT, DP, NW, true, true>(s, a, sh, keys);
    else if (a.slopes) launch_side<DT, DP, NW, true, false>(s, a, sh, keys);
    else if (a.cap > 0.f) launch_side<DT, DP, NW, false, true>(s, a, sh, keys);
    else launch_side<DT, DP, NW, false, false>(s, a, sh, keys);
}
template <int DT, int DP>
static void launch_dp(hipStream_t s, const AttnArgs& a, const AttnShape& sh, bool keys) {
    if (sh.nw == 4) launch_nw<DT, DP, 4>(s, a, sh, keys);
    else launch_nw<DT, DP, 1>(s, a, sh, keys);
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
