// attention_backward.hip -- the backward of attention over packed scans:
//   p_ij = exp(s_ij - lse_i),  delta_i = dout_i . out_i,  dz_ij = p_ij (dout_i . v_j - delta_i) ds_ij/dz_ij
//   dq_i = scale sum_j dz_ij k_j,   dk_j = scale sum_i dz_ij q_i,   dv_j = sum_i p_ij dout_i
// Two kernels, each of which forms the weights anew: dq with the queries in the columns, as the forward has them (it
// also forms delta), and dk, dv with the keys in the columns.  One kernel for all three would save two products of
// seven, but either add dq in the order that workgroups happen to run in, or hold it for every part of the keys.
// -delta is what the products dout . v are added to; the bias, over scale, or (keys in the columns) the rows' -lse are
// what the products q . k are added to, unless a cap's tanh stands between.
#include "attn_common.hpp"

namespace spv {

// d score / d product, over scale and kBend, and the score itself from a product under a cap
struct Capped {
    float cz, cap2;
    __device__ explicit Capped(const AttnArgs& a) : cz(2.f * kLog2e * a.scale / a.cap), cap2(a.cap * kLog2e) {}
    // t = tanh(w) = 1 - 2 r with r = 1 / (exp(2 w) + 1): 1 - t^2 = 4 (r - r^2)
    __device__ float operator()(float y, float rest, float& x) const {
        const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * cz) + 1.f);
        x = fmaf(-2.f * cap2, r, rest);
        return fmaf(-r, r, r);
    }
};
template <bool CAP>
constexpr float kBend = CAP ? 4.f : 1.f;

// waves per SIMD that the registers have to leave room for
#ifndef OCQ
#define OCQ 2
#endif
#ifndef OCK
#define OCK 2
#endif
constexpr int dq_waves(int dt, int DP, int nw) { return nw == 1 || dt == SPV_F32 || DP > 64 ? 1 : OCQ; }
constexpr int dkv_waves(int dt, int DP, int nw) { return nw == 1 || dt == SPV_F32 || DP > 64 ? 1 : OCK; }

template <int DT, int DP, int NW, bool BIAS, bool CAP>
__global__ __launch_bounds__(64 * NW, dq_waves(DT, DP, NW)) void k_attn_dq(AttnArgs a) {
    using T = Tile<DT, DP>;
    constexpr int KT = 32, TH = 64 * NW, BM = 32 * NW;
    __shared__ __align__(16) char lk[2][KT * T::LD], lv[2][KT * T::LD];
    __shared__ __align__(16) uint32_t lc[2][2][BIAS ? KT : 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), c = lane & 31, h = lane >> 5;
    const Share sh = attn_share(a);
    const int G = a.H / a.K, kh = sh.kh;
    const ScanTile t = find_tile(a.q_off, a.B, a.nq, G, BM, sh.tile);
    if (t.col0 >= t.cols) return;  // the whole workgroup
    const int64_t k0 = uniform(clamp_off(a.k_off[t.b], a.nk)), k1 = uniform(clamp_off(a.k_off[t.b + 1], a.nk));
    const int keys = (int)(k1 > k0 ? k1 - k0 : 0), tiles = keys / KT + (keys % KT != 0);
    const int per = (tiles + sh.parts - 1) / sh.parts, t0 = sh.part * per, t1 = t0 + per < tiles ? t0 + per : tiles;

    const bool busy = t.col0 + 32 * wave < t.cols, live = t.col0 + 32 * wave + c < t.cols;
    const int64_t q0 = t.col0 / G;
    const int y0 = (int)(t.col0 - q0 * G) + 32 * wave + c, head = kh * G + y0 % G;
    const int64_t qi = t.first + q0 + y0 / G;
    uint4 qf[T::NF], df[T::NF];
    T::load_cols(a.q, qi * a.ldq + (int64_t)head * a.D, live, a.D, h, qf);
    T::load_cols(a.dout, qi * a.lddo + (int64_t)head * a.D, live, a.D, h, df);
    float lse = 0.f, delta = 0.f;
    {
        uint4 of[T::NF];
        T::load_cols(a.out, qi * a.ldo + (int64_t)head * a.D, live, a.D, h, of);
#pragma unroll
        for (int s = 0; s < T::NF; ++s) delta = T::frag_dot(df[s], of[s], delta);
        delta = half_sum(delta);
    }
    Voxel qc{0, 0};
    float slope = 0.f;  // of the scores where there is a cap, else of the products
    if (live) {
        lse = a.lse[qi * a.H + head] * kLog2e;
        if (h == 0 && sh.part == 0) a.delta[qi * a.H + head] = delta;
        if constexpr (BIAS) {
            qc = voxel_of(*(const int4*)(a.q_coords + 4 * qi));
            slope = CAP ? a.slopes[head] * kLog2e : a.slopes[head] / a.scale;
        }
    }
    const float lift = slope * 8388608.f;  // what the 2^23 of a distance brings too much
    const float cs = a.scale * kLog2e;
    const Capped capped(a);
    f32x16 dref;
#pragma unroll
    for (int r = 0; r < 16; ++r) dref[r] = -delta;

    Stage<DT, DP, KT, TH> sk(tid, a.ldk, a.D), sv(tid, a.ldv, a.D);
    int4 ck{0, 0, 0, 0};
    auto load = [&](int i) __attribute__((always_inline)) {
        const int64_t r = k0 + (int64_t)i * KT, n = k1 - r;
        sk.load(rows_buffer((const char*)a.k + (r * a.ldk + kh * a.D) * T::SZ, a.ldk * T::SZ, n, KT, a.D * T::SZ));
        sv.load(rows_buffer((const char*)a.v + (r * a.ldv + kh * a.D) * T::SZ, a.ldv * T::SZ, n, KT, a.D * T::SZ));
        if constexpr (BIAS)
            if (tid < KT)
                ck = __builtin_bit_cast(int4, __builtin_amdgcn_raw_buffer_load_b128(
                                                  rows_buffer(a.k_coords + 4 * r, 16, n, KT, 16), tid * 16, 0, 0));
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
    f32x16 o[T::NB];
#pragma unroll
    for (int b = 0; b < T::NB; ++b) o[b] = f32x16{};
    if (t0 < t1) {
        load(t0);
        store(0);
        if (t0 + 1 < t1) load(t0 + 1);
    }
    __syncthreads();
    for (int i = t0; i < t1; ++i) {
        const int s = (i - t0) & 1;
        if (busy) {
            f32x16 b{};
            const f32x16 d = T::rows_dot(lv[s], lane, df, dref);
            if constexpr (BIAS)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t xy[4], zz[4];
                    lds_words(&lc[s][0][8 * q + 4 * h], xy);
                    lds_words(&lc[s][1][8 * q + 4 * h], zz);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        b[4 * q + e] = fmaf(voxel_dist(xy[e], zz[e], qc.xy, qc.z), -slope, lift);
                }
            f32x16 z = T::rows_dot(lk[s], lane, qf, CAP ? f32x16{} : b);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if constexpr (CAP) {
                    float x;
                    const float bend = capped(z[r], BIAS ? b[r] + (capped.cap2 - lse) : capped.cap2 - lse, x);
                    z[r] = __builtin_amdgcn_exp2f(x) * d[r] * bend;
                } else {
                    z[r] = __builtin_amdgcn_exp2f(fmaf(z[r], cs, -lse)) * d[r];
                }
            }
            const int end = keys - i * KT;
            if (end < KT) {  // keys past the scan's end: their rows are zero, but not their weights
                asm volatile("");  // a branch, not selects on every tile
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (8 * (r / 4) + 4 * h + r % 4 >= end) z[r] = 0.f;
            }
            T::add_weighted(lk[s], lane, T::weights(z), o);
        }
        if (i + 1 < t1) {
            store(s ^ 1);
            if (i + 2 < t1) load(i + 2);
        }
        __syncthreads();
    }
    if (!live) return;
    const float f = a.scale * kBend<CAP>;
    if (a.part)
        Tile<SPV_F32, DP>::store_cols(a.part, (((int64_t)sh.part * a.nq + qi) * a.H + head) * a.D, a.D, h, o, f);
    else
        T::store_cols(a.dq, qi * a.lddq + (int64_t)head * a.D, a.D, h, o, f);
}

// The weights are at most 1 and, over long scans, far below float16's smallest normal number (6e-5): in that type they
// are multiplied as 2^12 p (and may be some times 1 where scores of millions round).  dz is not scaled: its size is
// that of dout, which a caller may have scaled up.
template <int DT>
constexpr float kUp = DT == SPV_F16 ? 12.f : 0.f;

// Columns are keys; the rows are the scan's queries, once for each head of the key head's group, in that order.
template <int DT, int DP, int NW, bool BIAS, bool CAP>
__global__ __launch_bounds__(64 * NW, dkv_waves(DT, DP, NW)) void k_attn_dkv(AttnArgs a) {
    using T = Tile<DT, DP>;
    constexpr int KT = 32, TH = 64 * NW, BM = 32 * NW;
    __shared__ __align__(16) char lq[2][KT * T::LD], ld[2][KT * T::LD];
    __shared__ __align__(16) uint32_t lc[2][2][BIAS ? KT : 4];
    __shared__ float lr[2][2][64];  // the rows' -lse (see below) and -delta, then zeros
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), c = lane & 31, h = lane >> 5;
    const Share sh = attn_share(a);
    const int G = a.H / a.K, kh = sh.kh;
    const ScanTile t = find_tile(a.k_off, a.B, a.nk, 1, BM, sh.tile);
    if (t.col0 >= t.cols) return;  // the whole workgroup
    const int64_t q0 = uniform(clamp_off(a.q_off[t.b], a.nq)), q1 = uniform(clamp_off(a.q_off[t.b + 1], a.nq));
    const int64_t tiles = q1 > q0 ? (q1 - q0 + KT - 1) / KT : 0, all = tiles * G;
    const int64_t per = (all + sh.parts - 1) / sh.parts;
    const int64_t t0 = sh.part * per, t1 = t0 + per < all ? t0 + per : all;

    const bool busy = t.col0 + 32 * wave < t.cols, live = t.col0 + 32 * wave + c < t.cols;
    const int64_t kj = t.first + t.col0 + 32 * wave + c;
    uint4 kf[T::NF], vf[T::NF];
    T::load_cols(a.k, kj * a.ldk + (int64_t)kh * a.D, live, a.D, h, kf);
    T::load_cols(a.v, kj * a.ldv + (int64_t)kh * a.D, live, a.D, h, vf);
    Voxel kc{0, 0};
    if (BIAS && live) kc = voxel_of(*(const int4*)(a.k_coords + 4 * kj));
    const float cs = a.scale * kLog2e, inv_cs = 1.f / cs;
    const Capped capped(a);
    if (tid < 128) lr[tid >> 6][0][tid & 63] = lr[tid >> 6][1][tid & 63] = 0.f;
    if (NW == 1) lr[1][0][lane] = lr[1][1][lane] = 0.f;

    Stage<DT, DP, KT, TH> sq(tid, a.ldq, a.D), sd(tid, a.lddo, a.D);
    int4 cq{0, 0, 0, 0};
    float rl = 0.f, rd = 0.f;
    int64_t next = t0, g_next = tiles ? t0 / tiles : 0, i_next = t0 - g_next * tiles;  // the tile to load: head, tile of its rows
    auto load = [&]() __attribute__((always_inline)) {
        const int64_t r = q0 + i_next * KT, n = q1 - r, head = (int64_t)kh * G + g_next;
        sq.load(rows_buffer((const char*)a.q + (r * a.ldq + head * a.D) * T::SZ, a.ldq * T::SZ, n, KT, a.D * T::SZ));
        sd.load(rows_buffer((const char*)a.dout + (r * a.lddo + head * a.D) * T::SZ, a.lddo * T::SZ, n, KT, a.D * T::SZ));
        if (tid < KT) {
            const bool in = tid < n;
            // a row past the end has no weight: its lse is infinite
            rl = in ? kUp<DT> - a.lse[(r + tid) * a.H + head] * kLog2e : -INFINITY;
            rd = in ? -a.delta[(r + tid) * a.H + head] : 0.f;
            if constexpr (BIAS)
                if (in) cq = *(const int4*)(a.q_coords + 4 * (r + tid));
        }
        ++next;
        if (++i_next == tiles) i_next = 0, ++g_next;
    };
    auto store = [&](int s) __attribute__((always_inline)) {
        sq.store(lq[s], tid);
        sd.store(ld[s], tid);
        if (tid < KT) {
            lr[s][0][tid] = CAP ? rl + capped.cap2 : rl * inv_cs;
            lr[s][1][tid] = rd;
            if constexpr (BIAS) {
                const Voxel v = voxel_of(cq);
                lc[s][0][tid] = v.xy;
                lc[s][1][tid] = v.z;
            }
        }
    };
    constexpr float down = DT == SPV_F16 ? 1.f / 4096.f : 1.f;  // 2^-kUp
    f32x16 ok[T::NB], ov[T::NB];
#pragma unroll
    for (int b = 0; b < T::NB; ++b) ok[b] = ov[b] = f32x16{};
    int64_t i_now = i_next, g_now = g_next;
    __syncthreads();
    if (t0 < t1) {
        load();
        store(0);
        if (t0 + 1 < t1) load();
    }
    __syncthreads();
    for (int64_t i = t0; i < t1; ++i) {
        const int s = (int)(i - t0) & 1;
        if (busy) {
            float slope = 0.f, lift = 0.f;
            if constexpr (BIAS) {
                slope = a.slopes[(int64_t)kh * G + g_now] * kLog2e;
                lift = slope * 8388608.f;
            }
            f32x16 z = spread_rows(lr[s][0][lane]), rest = z;
            f32x16 d = T::rows_dot(ld[s], lane, vf, spread_rows(lr[s][1][lane]));
            z = T::rows_dot(lq[s], lane, kf, CAP ? f32x16{} : z);
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
                    float b = 0.f;
                    if constexpr (BIAS) b = fmaf(voxel_dist(xy[e], zz[e], kc.xy, kc.z), -slope, lift);
                    if constexpr (CAP) {
                        float x;
                        const float bend = capped(z[r], BIAS ? b + rest[r] : rest[r], x);
                        p[r] = __builtin_amdgcn_exp2f(x);
                        z[r] = p[r] * d[r] * bend;
                    } else {
                        p[r] = __builtin_amdgcn_exp2f(BIAS ? fmaf(z[r], cs, b) : z[r] * cs);
                        z[r] = p[r] * d[r];
                    }
                    if constexpr (DT == SPV_F16) z[r] *= down;
                }
            }
            T::add_weighted(ld[s], lane, T::weights(p), ov);
            T::add_weighted(lq[s], lane, T::weights(z), ok);
        }
        if (++i_now == tiles) i_now = 0, ++g_now;
        if (i + 1 < t1) {
            store(s ^ 1);
            if (next < t1) load();
        }
        __syncthreads();
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
