// Gated delta rule, chunk form: backward.
//
// The forward's walk is repeated first; it leaves u, r, the state S0 before each chunk, and dO.o per token.
// With D the adjoint of the state after a chunk, P as in the forward, T the inverse triangle:
//   dU = P^T dO + e^{G_C - G} (K D^T),   rb = T^T (beta dU),   dV = rb
//   D <- e^{G_C} D + (scale e^G dO)^T Q - (e^G rb)^T K
// is the reverse walk (delta_reverse_kernel: laid out like the forward's).  The rest of dQ and dK is local to a chunk (delta_grads_kernel):
//   dP_ij = scale Gam_ij dO_i.u_j (i >= j),   E_ij = -Gam_ij rb_i.u_j (i > j)
//   dQ = scale e^G dO S0 + dP K
//   dK = dP^T Q + e^{G_C - G} u D - e^G rb S0 + (E + E^T) K
// The gradients of beta and g are dots of float accumulators of the two walks.  rb is beta times the adjoint
// of u, so dbeta_t = rb_t.r_t / beta_t.  For g: in terms of e^{-G} S the decays appear in o_t as a factor e^{G_t}
// and in v_t as a factor e^{-G_t} only, so with G over the whole sequence
//   dL/dG_t = dO_t.o_t - dV_t.v_t,   dg_t = sum_{s >= t} dL/dG_s,
// taken chunk by chunk: what lies behind the chunk's end is <state, D> there.  Sums of 64 terms, nothing
// accumulates along the sequence.
#include "cawn_delta_chunk.cuh"

#include <type_traits>

namespace cawn {
namespace {

// ------------------------------------------------------------------------------ reverse walk

template <int DK, int NP> struct RevStage {
    static constexpr int NT = NP == 1 ? 2 : 3, VLD = 16 * kRowGroups<NP> + kPad;
    // r and the state come with the tiles, except where that would leave room for one stage only: asked for by the
    // walk itself they cost it a trip to L2 each.
    static constexpr bool FLOATS = DK == 64 || NP == 3;
    bf16 k[NP][kC * (DK + kPad)], q[NP][kC * (DK + kPad)], tri[NT][kC * kLd], p[NT][kC * kLd], go[NP][kC * VLD], v[NP][kC * VLD];
    float coef[kCoef][kC];
    float4 rf[FLOATS ? kRowGroups<NP> * 8 * 32 : 0], sf[FLOATS ? kRowGroups<NP> * (DK / 8) * 32 : 0];
};
// No side warps: measured with dO^T P and (scale e^G dO)^T Q made ahead on the side, 160 us instead of 149.
template <int DK, int NP> struct RevPlan {
    static constexpr int RG = kRowGroups<NP>, threads = 32 * (RG + kFetch<NP>);        // walking and fetching warps
    static constexpr int stages = fit_stages(sizeof(RevStage<DK, NP>), 0, 0).chain;
    static constexpr size_t smem = sizeof(RevStage<DK, NP>) * stages;
    static_assert(smem <= 227 * 1024, "fits an SM");
};

template <int DK, int NP>
__device__ __forceinline__ void rev_load(const ChunkParams &P, RevStage<DK, NP> &st, int bh, int c, int v0, int vcols, bool floats)
{
    constexpr int NT = NP == 1 ? 2 : 3, TH = 32 * kFetch<NP>, VW = 16 * kRowGroups<NP>;
    const long long t0 = (long long)c * kC, nc = (long long)bh * P.chunks + c;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
#pragma unroll
    for (int i = 0; i < NP; i++) {
        load_tile<kC, DK, TH>(st.k[i], P.k.at + i * P.k.plane + q_base(P, P.k, bh, t0), P.k.stride_t, rows, P.Dk);
        load_tile<kC, VW, TH>(st.go[i], P.go.at + i * P.go.plane + v_base(P, P.go, bh, t0) + v0, P.go.stride_t, rows, vcols);
        load_tile<kC, DK, TH>(st.q[i], P.q.at + i * P.q.plane + q_base(P, P.q, bh, t0), P.q.stride_t, rows, P.Dk);
        load_tile<kC, VW, TH>(st.v[i], P.v.at + i * P.v.plane + v_base(P, P.v, bh, t0) + v0, P.v.stride_t, rows, vcols);
    }
#pragma unroll
    for (int i = 0; i < NT; i++) {
        load_dense<TH>(st.tri[i], P.tri + (nc * NT + i) * kTile);
        load_dense<TH>(st.p[i], P.p + (nc * NT + i) * kTile);
    }
    for (int i = threadIdx.x % TH; i < kCoef * kC / 4; i += TH) cp16(smem_addr(&st.coef[0][0]) + i * 16, P.coef + nc * (kCoef * kC) + i * 4, true);
    if constexpr (RevStage<DK, NP>::FLOATS) {
        if (floats) {           // this block's row groups lie one after the other
            const long long after = c + 1 < P.chunks ? nc + 1 : (long long)P.B * P.Hv * P.chunks + bh, g = v0 / 16 % 4;
            const float4 *rf = P.rf + ((nc * P.vblocks + v0 / kC) * 4 + g) * (8 * 32), *sf = P.sf + ((after * P.vblocks + v0 / kC) * 4 + g) * (DK / 8 * 32);
            for (int i = threadIdx.x % TH; i < kRowGroups<NP> * 8 * 32; i += TH) cp16(smem_addr(st.rf) + i * 16, rf + i, true);
            for (int i = threadIdx.x % TH; i < kRowGroups<NP> * (DK / 8) * 32; i += TH) cp16(smem_addr(st.sf) + i * 16, sf + i, true);
        }
    }
    cp_commit();
}

// SUMMARY: only the adjoint that a segment's own outputs send to its start.
template <int DK, int NP, bool SUMMARY, class T>
__global__ void __launch_bounds__((RevPlan<DK, NP>::threads), 1) delta_reverse_kernel(const ChunkParams P)
{
    using Plan = RevPlan<DK, NP>;
    constexpr int ld = DK + kPad, NT = NP == 1 ? 2 : 3, RG = Plan::RG, VW = 16 * RG, VLD = VW + kPad, CS = Plan::stages, PAIR = Plan::threads;
    extern __shared__ __align__(16) unsigned char raw[];
    auto *stages = reinterpret_cast<RevStage<DK, NP> *>(raw);
    const int bh = blockIdx.x, seg = blockIdx.z;
    const int r0 = blockIdx.y * VW, vcols = P.Dv - r0 < VW ? P.Dv - r0 : VW;
    const int c0 = seg * P.seg_chunks, c1 = c0 + P.seg_chunks < P.chunks ? c0 + P.seg_chunks : P.chunks, count = c1 - c0;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, w = warp % RG, gr = lane / 4, tc = lane % 4 * 2;
    const int w4 = (r0 / 16 + w) % 4;

    if (warp >= RG) {           // fetch only
        for (int i = 0; i < count; i++) {
            const int s = i % CS;
            if (i >= CS) bar_sync(BAR_EMPTY + s, PAIR);
            rev_load<DK, NP>(P, stages[s], bh, c1 - 1 - i, r0, vcols, !SUMMARY);
            cp_wait<0>();
            bar_arrive(BAR_FULL + s, PAIR);
        }
        return;
    }

    const int row[2] = {r0 + 16 * w + gr, r0 + 16 * w + gr + 8};
    float D[DK / 8][4];
    const float *from = SUMMARY ? nullptr
                        : P.segs > 1 ? P.seg_start + ((long long)bh * P.segs + seg) * P.Dv * P.Dk
                                     : (P.state_in != nullptr ? P.state_in + (long long)bh * P.Dv * P.Dk : nullptr);
#pragma unroll
    for (int n = 0; n < DK / 8; n++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            float2 x = make_float2(0.f, 0.f);
            const int col = 8 * n + tc;
            if (from != nullptr && row[h] < P.Dv && col < P.Dk) x = *reinterpret_cast<const float2 *>(from + (long long)row[h] * P.Dk + col);
            D[n][2 * h] = x.x;
            D[n][2 * h + 1] = x.y;
        }

    for (int i = 0; i < count; i++) {
        const int c = c1 - 1 - i, s = i % CS;
        auto &st = stages[s];
        const long long t0 = (long long)c * kC, nc = (long long)bh * P.chunks + c, nv = nc * P.vblocks + r0 / kC;
        const unsigned ks = smem_addr(st.k[0]), qs = smem_addr(st.q[0]), ts = smem_addr(st.tri[0]), ps = smem_addr(st.p[0]);
        const unsigned gs = smem_addr(st.go[0]), vs = smem_addr(st.v[0]);

        // D for the chunk's own gradients
        if constexpr (!SUMMARY) {
            bf16 *dst = P.ds + nv * (NP * kC * DK) + (16 * w4 + gr) * DK + tc;
#pragma unroll
            for (int n = 0; n < DK / 8; n++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    unsigned y[NP];
                    split(D[n][2 * h], D[n][2 * h + 1], y);
#pragma unroll
                    for (int j = 0; j < NP; j++) *reinterpret_cast<unsigned *>(dst + j * (kC * DK) + 8 * h * DK + 8 * n) = y[j];
                }
        }
        bar_sync(BAR_FULL + s, PAIR);
        // <state after the chunk, D>
        if constexpr (!SUMMARY) {
            const long long after = c + 1 < P.chunks ? nc + 1 : (long long)P.B * P.Hv * P.chunks + bh;
            const float4 *sf = RevStage<DK, NP>::FLOATS ? st.sf + w * (DK / 8 * 32) + lane
                                                        : P.sf + ((after * P.vblocks + r0 / kC) * 4 + w4) * (DK / 8 * 32) + lane;
            float dot = 0.f;
#pragma unroll
            for (int n = 0; n < DK / 8; n++) {
                const float4 x = sf[n * 32];
                dot = fmaf(D[n][0], x.x, fmaf(D[n][1], x.y, fmaf(D[n][2], x.z, fmaf(D[n][3], x.w, dot))));
            }
#pragma unroll
            for (int o = 16; o > 0; o /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, o);
            if (lane == 0) P.sd[nv * 4 + w4] = dot;
        }
        // X = beta (e^{G_C - G} (D K^T) + dO^T P)
        float X[8][4] = {};
#pragma unroll
        for (int d = 0; d < DK / 16; d++) {
            unsigned a[3][4], b[4][NP][4];
#pragma unroll
            for (int j = 0; j < 4; j++) load_right<NP, false>(b[j], at_nk(ks, ld, 16 * j, 16 * d), kC * ld);
            as_left(D[2 * d], D[2 * d + 1], a);
            multiply<3, NP, 4>(X, a, b);
        }
#pragma unroll
        for (int n = 0; n < 8; n++) {
            const f32x2 lf = pair(*reinterpret_cast<const float2 *>(&st.coef[COEF_LEFT][8 * n + tc]));
            scale_row(X[n], 0, lf);
            scale_row(X[n], 1, lf);
        }
        triangle<NP, NT, true, true>(X, [&](unsigned (&a)[NP][4], int ib) { load_left<NP, true>(a, at_nk(gs, VLD, 16 * ib, 16 * w), kC * VLD); },
                                     [&](int ib, int nb) { return at_kn(ps, kLd, 16 * ib, 16 * nb); }, kC * kLd);
        float rb[8][4];
#pragma unroll
        for (int n = 0; n < 8; n++) {
            const f32x2 bt = pair(*reinterpret_cast<const float2 *>(&st.coef[COEF_BETA][8 * n + tc]));
            scale_row(X[n], 0, bt);
            scale_row(X[n], 1, bt);
#pragma unroll
            for (int e = 0; e < 4; e++) rb[n][e] = X[n][e];
        }
        // rb = X + (T - I)^T X
        triangle<3, NT, false, true>(rb, [&](unsigned (&a)[3][4], int ib) { as_left(X[2 * ib], X[2 * ib + 1], a); },
                                     [&](int ib, int nb) { return at_nk(ts, kLd, 16 * nb, 16 * ib); }, kC * kLd);
        if constexpr (!SUMMARY) {
            // rb.r and rb.v over this row group's 16 values
            float dots[8][4];
#pragma unroll
            for (int nb = 0; nb < 4; nb++) {
                unsigned x[NP][4];
                load_left<NP, true>(x, at_nk(vs, VLD, 16 * nb, 16 * w), kC * VLD);
#pragma unroll
                for (int m = 0; m < 2; m++) {
                    const int n = 2 * nb + m;
                    const float4 r = RevStage<DK, NP>::FLOATS ? st.rf[(w * 8 + n) * 32 + lane] : P.rf[((nv * 4 + w4) * 8 + n) * 32 + lane];
                    const float2 a = sum_terms(x, 2 * m), b = sum_terms(x, 2 * m + 1);
                    dots[n][0] = fmaf(rb[n][0], r.x, rb[n][2] * r.z);
                    dots[n][1] = fmaf(rb[n][1], r.y, rb[n][3] * r.w);
                    dots[n][2] = fmaf(rb[n][0], a.x, rb[n][2] * b.x);
                    dots[n][3] = fmaf(rb[n][1], a.y, rb[n][3] * b.y);
                }
            }
            column_sums(dots);
            float *to = P.rd + (nv * 4 + w4) * (2 * kC) + 8 * gr + tc;
            *reinterpret_cast<float2 *>(to) = make_float2(dots[0][0], dots[0][1]);
            *reinterpret_cast<float2 *>(to + kC) = make_float2(dots[0][2], dots[0][3]);
            // rb as token rows, through this warp's own part of the V tile: dV (bfloat16: the first term is the
            // rounded value), or its terms for the chunk's gradients
            const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
#pragma unroll
            for (int term = 0; term < NP; term++) {
                bf16 *dst = NP == 1 ? static_cast<bf16 *>(P.o) : P.rbt + term * P.rb.plane;
                dst += v_base(P, P.rb, bh, t0) + r0;
                __syncwarp();
#pragma unroll
                for (int nb = 0; nb < 4; nb++) {
                    unsigned x[NP][4];
                    as_left(rb[2 * nb], rb[2 * nb + 1], x);
                    stsm_t(at_nk(vs, VLD, 16 * nb, 16 * w), x[term][0], x[term][1], x[term][2], x[term][3]);
                }
                __syncwarp();
#pragma unroll
                for (int j = lane; j < 128; j += 32) {
                    const int t = j / 2, v = 16 * w + j % 2 * 8;
                    if (t < rows && v < vcols)
                        *reinterpret_cast<uint4 *>(dst + t * P.rb.stride_t + v) = *reinterpret_cast<const uint4 *>(&st.v[0][t * VLD + v]);
                }
            }
            if constexpr (sizeof(T) == 4) {
                T *gv = static_cast<T *>(P.o) + v_base(P, P.rb, bh, t0) + r0;
#pragma unroll
                for (int n = 0; n < 8; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int t = 8 * n + tc + (e & 1), v = 16 * w + gr + (e >> 1) * 8;
                        if (t < rows && v < vcols) gv[t * P.rb.stride_t + v] = narrow<T>(rb[n][e]);
                    }
            }
        }
        // D <- e^{G_C} D + (scale e^G dO)^T Q - (e^G rb)^T K, the update summed from zero as in the forward
        const float eC = st.coef[COEF_EG][kC - 1];
        unsigned a[4][3][4], f[4][3][4];
#pragma unroll
        for (int tb = 0; tb < 4; tb++) {
            unsigned x[NP][4];
            load_left<NP, true>(x, at_nk(gs, VLD, 16 * tb, 16 * w), kC * VLD);
            float y[2][4];
#pragma unroll
            for (int m = 0; m < 2; m++) {
                const float2 e = *reinterpret_cast<const float2 *>(&st.coef[COEF_EG][16 * tb + 8 * m + tc]);
                const f32x2 plus = pair(P.scale * e.x, P.scale * e.y), minus = pair(-e.x, -e.y);
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const float2 z = halves(mul2(plus, pair(sum_terms(x, 2 * m + h))));
                    y[m][2 * h] = z.x;
                    y[m][2 * h + 1] = z.y;
                    scale_row(rb[2 * tb + m], h, minus);
                }
            }
            as_left(y[0], y[1], a[tb]);
            as_left(rb[2 * tb], rb[2 * tb + 1], f[tb]);
        }
#pragma unroll
        for (int nb = 0; nb < DK / 16; nb += 2) {
            float x[4][4] = {};
#pragma unroll
            for (int tb = 0; tb < 4; tb++) {
                unsigned b[2][NP][4];
#pragma unroll
                for (int k = 0; k < 2; k++) load_right<NP, true>(b[k], at_kn(qs, ld, 16 * tb, 16 * (nb + k)), kC * ld);
                multiply<3, NP, 2>(x, a[tb], b);
#pragma unroll
                for (int k = 0; k < 2; k++) load_right<NP, true>(b[k], at_kn(ks, ld, 16 * tb, 16 * (nb + k)), kC * ld);
                multiply<3, NP, 2>(x, f[tb], b);
            }
#pragma unroll
            for (int m = 0; m < 4; m++)
#pragma unroll
                for (int h = 0; h < 2; h++) fma_row(D[2 * nb + m], h, pair(eC, eC), pair(x[m][2 * h], x[m][2 * h + 1]));
        }
        if (i + CS < count) bar_arrive(BAR_EMPTY + s, PAIR);
    }
    float *to = SUMMARY ? P.seg_end + ((long long)bh * P.segs + seg) * P.Dv * P.Dk
                : P.state_out != nullptr && seg == 0 ? P.state_out + (long long)bh * P.Dv * P.Dk : nullptr;
    if (to != nullptr) {
#pragma unroll
        for (int n = 0; n < DK / 8; n++)
#pragma unroll
            for (int h = 0; h < 2; h++)
                if (row[h] < P.Dv && 8 * n + tc < P.Dk)
                    *reinterpret_cast<float2 *>(to + (long long)row[h] * P.Dk + 8 * n + tc) = make_float2(D[n][2 * h], D[n][2 * h + 1]);
    }
}

// ------------------------------------------------------------------------------ gradients of a chunk

// Eight warps: the first four own 16 query rows each (dP, dQ), the others 16 key rows (E, dK).  Values pass in
// blocks of VW: 64, or 32 where three terms of 128 keys leave room for no more.  All factors take the terms
// of the inputs: what is computed here is rounded to the inputs' type anyway.
template <int DK, int NP> constexpr int kGradVW = NP == 3 && DK == 128 ? 32 : 64;

template <int DK, int NP> struct GradSmem {
    static constexpr int VW = kGradVW<DK, NP>;
    bf16 q[NP][kC * (DK + kPad)], k[NP][kC * (DK + kPad)];
    union {
        struct {
            bf16 go[NP][kC * (VW + kPad)], u[NP][kC * (VW + kPad)], rb[NP][kC * (VW + kPad)];
            bf16 s0[NP][VW * (DK + kPad)], ds[NP][VW * (DK + kPad)];
        } v;
        struct {
            bf16 dp[NP][kC * kLd], e[NP][kC * kLd];
        } m;
    };
    float coef[kCoef][kC];
    float dots[8][3][kC];                   // per 16 values: dO.o, rb.r, rb.v (up to 128 values)
};

template <int DK, int NP, class T>
__global__ void __launch_bounds__(256, (DK == 64 && NP == 1 ? 2 : 1)) delta_grads_kernel(const ChunkParams P)
{
    constexpr int ld = DK + kPad, ND = DK / 16, VW = kGradVW<DK, NP>, ldv = VW + kPad;
    extern __shared__ __align__(16) unsigned char raw[];
    auto &sm = *reinterpret_cast<GradSmem<DK, NP> *>(raw);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, w = warp % 4, gr = lane / 4, tc = lane % 4 * 2;
    const bool qside = warp < 4;
    const int c = (int)(blockIdx.x % P.chunks), bk = (int)(blockIdx.x / P.chunks), b = bk / P.Hk, hk = bk % P.Hk, rep = P.Hv / P.Hk;
    const long long t0 = (long long)c * kC;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
    const unsigned qs = smem_addr(sm.q[0]), ks = smem_addr(sm.k[0]);
    const unsigned us = smem_addr(sm.v.u[0]), s0s = smem_addr(sm.v.s0[0]), dss = smem_addr(sm.v.ds[0]);
    const unsigned mine = qside ? smem_addr(sm.v.go[0]) : smem_addr(sm.v.rb[0]);
    const unsigned dps = smem_addr(sm.m.dp[0]), es = smem_addr(sm.m.e[0]);

#pragma unroll
    for (int i = 0; i < NP; i++) {
        load_tile<kC, DK, 256>(sm.q[i], P.q.at + i * P.q.plane + q_base(P, P.q, b * P.Hv + hk * rep, t0), P.q.stride_t, rows, P.Dk);
        load_tile<kC, DK, 256>(sm.k[i], P.k.at + i * P.k.plane + q_base(P, P.k, b * P.Hv + hk * rep, t0), P.k.stride_t, rows, P.Dk);
    }
    cp_commit();

    float acc[2 * ND][4] = {};              // dQ or dK rows of this warp, over the heads that share them
    const int i0 = 16 * w + gr;             // rows i0 and i0 + 8

    for (int hv = 0; hv < rep; hv++) {
        const int bh = b * P.Hv + hk * rep + hv;
        const long long nc = (long long)bh * P.chunks + c;
        if (threadIdx.x < kCoef * 16)
            cp16(smem_addr(&sm.coef[0][0]) + threadIdx.x * 16, P.coef + nc * (kCoef * kC) + threadIdx.x * 4, true);
        const int groups = (P.Dv + 15) / 16;                // row groups of the walks
        const long long g0 = nc * P.vblocks * 4;
        for (int i = threadIdx.x; i < groups * 48; i += 256) {
            const int g = i / 48, x = i % 48 * 4;
            cp16(smem_addr(&sm.dots[g][0][0]) + x * 4, x < kC ? P.od + (g0 + g) * kC + x : P.rd + (g0 + g) * (2 * kC) + x - kC, true);
        }
        float X[8][4] = {};                 // dO.u or rb.u, then dP or E
        for (int v0 = 0; v0 < P.Dv; v0 += VW) {
            const int vcols = P.Dv - v0 < VW ? P.Dv - v0 : VW, in = v0 % kC;
            const long long nv = nc * P.vblocks + v0 / kC;
#pragma unroll
            for (int i = 0; i < NP; i++) {
                load_tile<kC, VW, 256>(sm.v.go[i], P.go.at + i * P.go.plane + v_base(P, P.go, bh, t0) + v0, P.go.stride_t, rows, vcols);
                load_tile<kC, VW, 256>(sm.v.rb[i], P.rb.at + i * P.rb.plane + v_base(P, P.rb, bh, t0) + v0, P.rb.stride_t, rows, vcols);
                load_tile<kC, VW, 256>(sm.v.u[i], P.u + (nv * NP + i) * kTile + in, kC, kC, vcols);
                load_tile<VW, DK, 256>(sm.v.s0[i], P.s0 + (nv * NP + i) * (kC * DK) + in * DK, DK, vcols, DK);
                load_tile<VW, DK, 256>(sm.v.ds[i], P.ds + (nv * NP + i) * (kC * DK) + in * DK, DK, vcols, DK);
            }
            cp_commit();
            cp_wait<0>();
            __syncthreads();

            unsigned a[VW / 16][NP][4];     // rows of dO or rb
#pragma unroll
            for (int d = 0; d < VW / 16; d++) {
                load_left<NP, false>(a[d], at_kn(mine, ldv, 16 * w, 16 * d), kC * ldv);
#pragma unroll
                for (int nb = 0; nb < 4; nb++)
                    if (nb <= w) product<NP, NP, false>(X[2 * nb], X[2 * nb + 1], a[d], at_nk(us, ldv, 16 * nb, 16 * d), kC * ldv);
            }
            // times S0: the state's part of dQ, or minus the read-out's part of dK
            const float sign = qside ? P.scale : -1.f;
            const float f[2] = {sign * sm.coef[COEF_EG][i0], sign * sm.coef[COEF_EG][i0 + 8]};
#pragma unroll
            for (int nb = 0; nb < ND; nb++) {
                float x[2][4] = {};
#pragma unroll
                for (int d = 0; d < VW / 16; d++) product<NP, NP, true>(x[0], x[1], a[d], at_kn(s0s, ld, 16 * d, 16 * nb), VW * ld);
#pragma unroll
                for (int m = 0; m < 2; m++)
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[2 * nb + m][e] = fmaf(f[e >> 1], x[m][e], acc[2 * nb + m][e]);
            }
            if (!qside) {                   // e^{G_C - G} u D
                const float g[2] = {sm.coef[COEF_LEFT][i0], sm.coef[COEF_LEFT][i0 + 8]};
#pragma unroll
                for (int d = 0; d < VW / 16; d++) load_left<NP, false>(a[d], at_kn(us, ldv, 16 * w, 16 * d), kC * ldv);
#pragma unroll
                for (int nb = 0; nb < ND; nb++) {
                    float x[2][4] = {};
#pragma unroll
                    for (int d = 0; d < VW / 16; d++) product<NP, NP, true>(x[0], x[1], a[d], at_kn(dss, ld, 16 * d, 16 * nb), VW * ld);
#pragma unroll
                    for (int m = 0; m < 2; m++)
#pragma unroll
                        for (int e = 0; e < 4; e++) acc[2 * nb + m][e] = fmaf(g[e >> 1], x[m][e], acc[2 * nb + m][e]);
                }
            }
            __syncthreads();        // the value tiles are free
        }

        // dP or E, and as tiles (they feed dK transposed)
        bf16 *tile = qside ? sm.m.dp[0] : sm.m.e[0];
        const float sign = qside ? P.scale : -1.f;
#pragma unroll
        for (int n = 0; n < 8; n++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int i = i0 + 8 * h, j = 8 * n + tc;
                float x[2];
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const bool on = n / 2 <= w && (qside ? i >= j + e : i > j + e);
                    x[e] = on ? sign * X[n][2 * h + e] * exp2_fast((sm.coef[COEF_GHI][i] - sm.coef[COEF_GHI][j + e]) +
                                                                   (sm.coef[COEF_GLO][i] - sm.coef[COEF_GLO][j + e])) : 0.f;
                    X[n][2 * h + e] = x[e];
                }
                unsigned y[NP];
                split(x[0], x[1], y);
#pragma unroll
                for (int m = 0; m < NP; m++) *reinterpret_cast<unsigned *>(tile + m * (kC * kLd) + i * kLd + j) = y[m];
            }
        __syncthreads();

        // dQ += dP K;  dK += E K + E^T K + dP^T Q, each head's sum from zero
#pragma unroll
        for (int nb = 0; nb < ND; nb++) {
            float x[2][4] = {};
#pragma unroll
            for (int jb = 0; jb < 4; jb++) {
                unsigned a[NP][4];
                if (jb <= w) {
                    as_left(X[2 * jb], X[2 * jb + 1], a);
                    product<NP, NP, true>(x[0], x[1], a, at_kn(ks, ld, 16 * jb, 16 * nb), kC * ld);
                }
                if (!qside && jb >= w) {
                    load_left<NP, true>(a, at_nk(es, kLd, 16 * jb, 16 * w), kC * kLd);
                    product<NP, NP, true>(x[0], x[1], a, at_kn(ks, ld, 16 * jb, 16 * nb), kC * ld);
                    load_left<NP, true>(a, at_nk(dps, kLd, 16 * jb, 16 * w), kC * kLd);
                    product<NP, NP, true>(x[0], x[1], a, at_kn(qs, ld, 16 * jb, 16 * nb), kC * ld);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                acc[2 * nb][e] += x[0][e];
                acc[2 * nb + 1][e] += x[1][e];
            }
        }
        // decays and betas: one warp, two tokens a lane
        if (warp == 0) {
            float dG[2], end = 0.f;
            const long long at = ((long long)b * P.L + t0) * P.Hv + bh % P.Hv;
            for (int i = lane; i < groups; i += 32) end += P.sd[g0 + i];
#pragma unroll
            for (int o = 16; o > 0; o /= 2) end += __shfl_xor_sync(0xffffffffu, end, o);
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int t = 2 * lane + e;
                float od = 0.f, rr = 0.f, rv = 0.f;
                for (int i = 0; i < groups; i++) {
                    od += sm.dots[i][0][t];
                    rr += sm.dots[i][1][t];
                    rv += sm.dots[i][2][t];
                }
                dG[e] = od - rv;
                if (t < rows) P.gbeta[at + (long long)t * P.Hv] = rr / sm.coef[COEF_BETA][t];
            }
            float run = dG[0] + dG[1];      // suffix sums
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const float other = __shfl_down_sync(0xffffffffu, run, o);
                if (lane + o < 32) run += other;
            }
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int t = 2 * lane + e;
                if (t < rows) {
                    const long long to = at + (long long)t * P.Hv;
                    // a decay that is zero in float passes nothing on, and its derivative is zero
                    P.gg[to] = P.g[to] < -104.f ? 0.f : run - (e == 1 ? dG[0] : 0.f) + end;
                }
            }
        }
        if (hv + 1 < rep) __syncthreads();      // tiles and coefficients are free for the next head
    }

    T *dst = static_cast<T *>(qside ? P.gq : P.gk) + ((long long)b * P.L + t0) * P.Hk * P.Dk + (long long)hk * P.Dk;
#pragma unroll
    for (int n = 0; n < 2 * ND; n++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int t = i0 + 8 * h, col = 8 * n + tc;
            if (t < rows && col < P.Dk) {
                T *to = dst + (long long)t * P.Hk * P.Dk + col;
                if constexpr (sizeof(T) == 2) *reinterpret_cast<unsigned *>(to) = pack_bf16(acc[n][2 * h], acc[n][2 * h + 1]);
                else *reinterpret_cast<float2 *>(to) = make_float2(acc[n][2 * h], acc[n][2 * h + 1]);
            }
        }
}

template <int DK, int NP, bool SUMMARY> cudaError_t walk(const ChunkParams &P, cudaStream_t st)
{
    using T = typename std::conditional<NP == 1, bf16, float>::type;
    using Plan = RevPlan<DK, NP>;
    auto *kernel = delta_reverse_kernel<DK, NP, SUMMARY, T>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Plan::smem);
    if (e != cudaSuccess) return e;
    constexpr int VW = 16 * Plan::RG;
    return launch(kernel, dim3((unsigned)(P.B * P.Hv), (P.Dv + VW - 1) / VW, P.segs), dim3(Plan::threads), Plan::smem, st, P);
}

template <int DK, int NP> cudaError_t reverse(const ChunkParams &P, cudaStream_t st)
{
    if (P.segs > 1) {           // the forward's transitions are still in the workspace
        cudaError_t e = walk<DK, NP, true>(P, st);
        if (e == cudaSuccess) e = launch_delta_join(P, DK, true, st);
        if (e != cudaSuccess) return e;
    }
    return walk<DK, NP, false>(P, st);
}

template <int DK, int NP> cudaError_t grads(const ChunkParams &P, cudaStream_t st)
{
    using T = typename std::conditional<NP == 1, bf16, float>::type;
    const size_t smem = sizeof(GradSmem<DK, NP>);
    static_assert(sizeof(GradSmem<DK, NP>) <= 227 * 1024, "fits an SM");
    auto *kernel = delta_grads_kernel<DK, NP, T>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch(kernel, dim3((unsigned)(P.B * P.Hk * (long long)P.chunks)), dim3(256), smem, st, P);
}

}  // namespace

cudaError_t launch_delta_reverse(const ChunkParams &P, int dk, int terms, cudaStream_t st)
{
    if (dk == 64) return terms == 1 ? reverse<64, 1>(P, st) : reverse<64, 3>(P, st);
    return terms == 1 ? reverse<128, 1>(P, st) : reverse<128, 3>(P, st);
}

cudaError_t launch_delta_grads(const ChunkParams &P, int dk, int terms, cudaStream_t st)
{
    if (dk == 64) return terms == 1 ? grads<64, 1>(P, st) : grads<64, 3>(P, st);
    return terms == 1 ? grads<128, 1>(P, st) : grads<128, 3>(P, st);
}

}  // namespace cawn
