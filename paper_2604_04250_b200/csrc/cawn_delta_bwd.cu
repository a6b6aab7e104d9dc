// Gated delta rule, chunk form: backward.
//
// The forward's walk is repeated first (states S0 before each chunk and corrections r are kept in the
// workspace).  With D the adjoint of the state after a chunk, P as in the forward, T the inverse triangle:
//   dU = P^T dO + e^{G_C - G} (K D^T),   rb = T^T (beta dU),   dV = rb
//   D <- e^{G_C} D + (scale e^G dO)^T Q - (e^G rb)^T K
// is the reverse walk (delta_reverse_kernel: transposed like the forward's, a warp owns 16 value rows,
// products chained in registers).  Everything else is local to a chunk (delta_grads_kernel):
//   D1 = dO r^T,  M = rb r^T,  dP_ij = Gam_ij scale beta_j D1_ij,  E_ij = -Gam_ij beta_j M_ij (i > j)
//   dQ = scale e^G dO S0 + dP K
//   dK = dP^T Q + beta e^{G_C - G} (r D) - e^G rb S0 + (E + E^T) K
//   dbeta_t = r_t.dU_t - sum_i At_it M_it
// and for the decays, with Z = dP . (Q K^T) + E . (K K^T) below the diagonal and z_t = beta_t r_t.(e^{G_C - G}
// K D)_t,  dG_t = sum_j Z_tj - sum_i Z_it + q_t.(scale e^G dO S0)_t - k_t.(e^G rb S0)_t - z_t,
//   dg_t = sum_{s >= t} dG_s + sum z + e^{G_C} <S0, D>:  every term carries its own decay, so nothing large
// cancels.  The dots with r are taken in the reverse walk, where dU is at hand in float.
#include "cawn_delta_chunk.cuh"

#include <type_traits>

namespace cawn {
namespace {

// ------------------------------------------------------------------------------ reverse walk

template <int DK, int NP> struct RevStage {
    static constexpr int NT = NP == 1 ? 2 : 3;
    bf16 k[NP][kC * (DK + kPad)], q[NP][kC * (DK + kPad)];
    bf16 tri[NT][kC * kLd], p[NT][kC * kLd], r[3][kC * kLd];
    bf16 go[NP][kC * kLd];
    float coef[3][kC];
};
template <int DK, int NP> constexpr int kRevStages = sizeof(RevStage<DK, NP>) * 2 <= 227 * 1024 ? 2 : 1;

template <int DK, int NP>
__device__ __forceinline__ void rev_load(const ChunkParams &P, RevStage<DK, NP> &st, int bh, int c, int vb, int vcols)
{
    constexpr int NT = NP == 1 ? 2 : 3;
    const long long t0 = (long long)c * kC, nc = (long long)bh * P.chunks + c;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
#pragma unroll
    for (int i = 0; i < NP; i++) {
        load_tile<kC, DK, 128>(st.k[i], P.k.at + i * P.k.plane + q_base(P, P.k, bh, t0), P.k.stride_t, rows, P.Dk);
        load_tile<kC, DK, 128>(st.q[i], P.q.at + i * P.q.plane + q_base(P, P.q, bh, t0), P.q.stride_t, rows, P.Dk);
        load_tile<kC, kC, 128>(st.go[i], P.go.at + i * P.go.plane + v_base(P, P.go, bh, t0) + vb * kC, P.go.stride_t, rows, vcols);
    }
#pragma unroll
    for (int i = 0; i < NT; i++) {
        load_tile<kC, kC, 128>(st.tri[i], P.tri + (nc * NT + i) * kTile, kC, kC, kC);
        load_tile<kC, kC, 128>(st.p[i], P.p + (nc * NT + i) * kTile, kC, kC, kC);
    }
#pragma unroll
    for (int i = 0; i < 3; i++) load_tile<kC, kC, 128>(st.r[i], P.r + ((nc * P.vblocks + vb) * 3 + i) * kTile, kC, kC, kC);
    if (threadIdx.x < 48)
        cp16(smem_addr(&st.coef[0][0]) + threadIdx.x * 16, P.coef + nc * (kCoef * kC) + threadIdx.x * 4, true);
    cp_commit();
}

template <int DK, int NP, class T>
__global__ void __launch_bounds__(128) delta_reverse_kernel(const ChunkParams P)
{
    constexpr int STAGES = kRevStages<DK, NP>, ld = DK + kPad, NT = NP == 1 ? 2 : 3;
    extern __shared__ __align__(16) unsigned char raw[];
    auto *stages = reinterpret_cast<RevStage<DK, NP> *>(raw);
    const int bh = blockIdx.x, vb = blockIdx.y, seg = blockIdx.z;
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32, gr = lane / 4, tc = lane % 4 * 2;
    const int r0 = vb * kC, vcols = P.Dv - r0 < kC ? P.Dv - r0 : kC;
    const int row[2] = {r0 + 16 * w + gr, r0 + 16 * w + gr + 8};
    const int c0 = seg * P.seg_chunks, c1 = c0 + P.seg_chunks < P.chunks ? c0 + P.seg_chunks : P.chunks;

    rev_load<DK, NP>(P, stages[0], bh, c1 - 1, vb, vcols);

    float D[DK / 8][4];
    const float *from = P.segs > 1 ? P.seg_start + ((long long)bh * P.segs + seg) * P.Dv * P.Dk
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

    for (int c = c1 - 1; c >= c0; c--) {
        auto &st = stages[(c1 - 1 - c) % STAGES];
        if (STAGES == 2 && c > c0) {
            rev_load<DK, NP>(P, stages[(c1 - c) % STAGES], bh, c - 1, vb, vcols);
            cp_wait<1>();
        } else {
            cp_wait<0>();
        }
        __syncthreads();
        const long long t0 = (long long)c * kC, nc = (long long)bh * P.chunks + c;
        const unsigned ks = smem_addr(st.k[0]), qs = smem_addr(st.q[0]), ts = smem_addr(st.tri[0]), ps = smem_addr(st.p[0]), gs = smem_addr(st.go[0]), rs = smem_addr(st.r[0]);

        // D of this chunk, kept for the chunk's own gradients
        {
            bf16 *dst = P.ds + (nc * P.vblocks + vb) * (NT * kC * DK);
#pragma unroll
            for (int n = 0; n < DK / 8; n++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    unsigned x[NT];
                    split(D[n][2 * h], D[n][2 * h + 1], x);
#pragma unroll
                    for (int i = 0; i < NT; i++)
                        *reinterpret_cast<unsigned *>(dst + i * (kC * DK) + (row[h] - r0) * DK + 8 * n + tc) = x[i];
                }
        }
        // X = e^{G_C - G} (D K^T) + dO^T P
        float X[8][4] = {};
#pragma unroll
        for (int d = 0; d < DK / 16; d++) {
            unsigned x[NT][4];
            as_left(D[2 * d], D[2 * d + 1], x);
#pragma unroll
            for (int nb = 0; nb < 4; nb++) product<NT, NP, false>(X[2 * nb], X[2 * nb + 1], x, at_nk(ks, ld, 16 * nb, 16 * d), kC * ld);
        }
        float dots[8][4];           // columns t = 8 n + tc, +1: r.(e^{G_C - G} K D^T), then r.dU, over this thread's rows
#pragma unroll
        for (int nb = 0; nb < 4; nb++) {
            unsigned x[3][4];
            load_left<3, true>(x, at_nk(rs, kLd, 16 * nb, 16 * w), kC * kLd);
#pragma unroll
            for (int m = 0; m < 2; m++) {
                const int n = 2 * nb + m;
                const float2 lf = *reinterpret_cast<const float2 *>(&st.coef[COEF_LEFT][8 * n + tc]);
                X[n][0] *= lf.x; X[n][1] *= lf.y; X[n][2] *= lf.x; X[n][3] *= lf.y;
                const float2 r0v = sum_terms(x, 2 * m), r1v = sum_terms(x, 2 * m + 1);
                dots[n][0] = fmaf(X[n][0], r0v.x, X[n][2] * r1v.x);
                dots[n][1] = fmaf(X[n][1], r0v.y, X[n][3] * r1v.y);
            }
        }
#pragma unroll
        for (int ib = 0; ib < 4; ib++) {
            unsigned x[NP][4];
            load_left<NP, true>(x, at_nk(gs, kLd, 16 * ib, 16 * w), kC * kLd);
#pragma unroll
            for (int nb = 0; nb <= ib; nb++) product<NP, NT, true>(X[2 * nb], X[2 * nb + 1], x, at_kn(ps, kLd, 16 * ib, 16 * nb), kC * kLd);
        }
#pragma unroll
        for (int nb = 0; nb < 4; nb++) {
            unsigned x[3][4];
            load_left<3, true>(x, at_nk(rs, kLd, 16 * nb, 16 * w), kC * kLd);
#pragma unroll
            for (int m = 0; m < 2; m++) {
                const int n = 2 * nb + m;
                const float2 r0v = sum_terms(x, 2 * m), r1v = sum_terms(x, 2 * m + 1);
                dots[n][2] = fmaf(X[n][0], r0v.x, X[n][2] * r1v.x);
                dots[n][3] = fmaf(X[n][1], r0v.y, X[n][3] * r1v.y);
            }
        }
        // over the eight lanes of a column; each lane keeps one of the eight tiles, tile gr
#pragma unroll
        for (int bit = 4; bit > 0; bit /= 2)
#pragma unroll
            for (int n = 0; n < bit; n++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const bool up = (gr & bit) != 0;
                    const float keep = up ? dots[n + bit][e] : dots[n][e], send = up ? dots[n][e] : dots[n + bit][e];
                    dots[n][e] = keep + __shfl_xor_sync(0xffffffffu, send, bit * 4);
                }
        {
            float *to = P.dots + ((nc * P.vblocks + vb) * 4 + w) * (2 * kC) + 8 * gr + tc;
            *reinterpret_cast<float2 *>(to) = make_float2(dots[0][0], dots[0][1]);
            *reinterpret_cast<float2 *>(to + kC) = make_float2(dots[0][2], dots[0][3]);
        }
        // rb = T^T (beta dU)
        float rb[8][4];
#pragma unroll
        for (int n = 0; n < 8; n++) {
            const float2 bt = *reinterpret_cast<const float2 *>(&st.coef[COEF_BETA][8 * n + tc]);
            X[n][0] *= bt.x; X[n][1] *= bt.y; X[n][2] *= bt.x; X[n][3] *= bt.y;
#pragma unroll
            for (int e = 0; e < 4; e++) rb[n][e] = X[n][e];
        }
#pragma unroll
        for (int ib = 0; ib < 4; ib++) {
            unsigned x[NT][4];
            as_left(X[2 * ib], X[2 * ib + 1], x);
#pragma unroll
            for (int nb = 0; nb <= ib; nb++) product<NT, NT, false>(rb[2 * nb], rb[2 * nb + 1], x, at_nk(ts, kLd, 16 * nb, 16 * ib), kC * kLd);
        }
        // D <- e^{G_C} D + (scale e^G dO)^T Q - (e^G rb)^T K, the update summed from zero as in the forward
        const float eC = st.coef[COEF_EG][kC - 1];
        unsigned a[4][NT][4], f[4][NT][4];
#pragma unroll
        for (int tb = 0; tb < 4; tb++) {
            unsigned x[NP][4];
            load_left<NP, true>(x, at_nk(gs, kLd, 16 * tb, 16 * w), kC * kLd);
            float s[2][4], y[2][4];
#pragma unroll
            for (int m = 0; m < 2; m++) {
                const float2 eg = *reinterpret_cast<const float2 *>(&st.coef[COEF_EG][16 * tb + 8 * m + tc]);
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const float2 z = sum_terms(x, 2 * m + h);
                    s[m][2 * h] = P.scale * eg.x * z.x;
                    s[m][2 * h + 1] = P.scale * eg.y * z.y;
                    y[m][2 * h] = -eg.x * rb[2 * tb + m][2 * h];
                    y[m][2 * h + 1] = -eg.y * rb[2 * tb + m][2 * h + 1];
                }
            }
            as_left(s[0], s[1], a[tb]);
            as_left(y[0], y[1], f[tb]);
        }
#pragma unroll
        for (int nb = 0; nb < DK / 16; nb++) {
            float x[2][4] = {};
#pragma unroll
            for (int tb = 0; tb < 4; tb++) {
                product<NT, NP, true>(x[0], x[1], a[tb], at_kn(qs, ld, 16 * tb, 16 * nb), kC * ld);
                product<NT, NP, true>(x[0], x[1], f[tb], at_kn(ks, ld, 16 * tb, 16 * nb), kC * ld);
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                D[2 * nb][e] = fmaf(eC, D[2 * nb][e], x[0][e]);
                D[2 * nb + 1][e] = fmaf(eC, D[2 * nb + 1][e], x[1][e]);
            }
        }
        // rb as token rows, through this warp's own columns of the dO tile: for the chunk's gradients,
        // and as dV
        bf16 *dst = P.rb + (nc * P.vblocks + vb) * (NT * kTile);
        T *gv = static_cast<T *>(P.o) + (bh / P.Hv) * P.o_stride_b + t0 * P.o_stride_t + (long long)(bh % P.Hv) * P.Dv + r0;
        const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
#pragma unroll
        for (int term = 0; term < NT; term++) {
            __syncwarp();
#pragma unroll
            for (int nb = 0; nb < 4; nb++) {
                unsigned x[NT][4];
                as_left(rb[2 * nb], rb[2 * nb + 1], x);
                stsm_t(at_nk(gs, kLd, 16 * nb, 16 * w), x[term][0], x[term][1], x[term][2], x[term][3]);
            }
            __syncwarp();
#pragma unroll
            for (int i = lane; i < 128; i += 32) {
                const int t = i / 2, v = 16 * w + i % 2 * 8;
                const uint4 word = *reinterpret_cast<const uint4 *>(&st.go[0][t * kLd + v]);
                *reinterpret_cast<uint4 *>(dst + term * kTile + t * kC + v) = word;
                // the first term is the value rounded to bfloat16
                if (sizeof(T) == 2 && term == 0 && t < rows && v < vcols) *reinterpret_cast<uint4 *>(gv + t * P.o_stride_t + v) = word;
            }
        }
        if (sizeof(T) == 4) {
#pragma unroll
            for (int n = 0; n < 8; n++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int t = 8 * n + tc + (e & 1), v = 16 * w + gr + (e >> 1) * 8;
                    if (t < rows && v < vcols) gv[t * P.o_stride_t + v] = narrow<T>(rb[n][e]);
                }
        }
        __syncthreads();
        if (STAGES == 1 && c > c0) rev_load<DK, NP>(P, stages[0], bh, c - 1, vb, vcols);
    }
    if (P.state_out != nullptr && seg == 0) {
        float *to = P.state_out + (long long)bh * P.Dv * P.Dk;
#pragma unroll
        for (int n = 0; n < DK / 8; n++)
#pragma unroll
            for (int h = 0; h < 2; h++)
                if (row[h] < P.Dv && 8 * n + tc < P.Dk)
                    *reinterpret_cast<float2 *>(to + (long long)row[h] * P.Dk + 8 * n + tc) = make_float2(D[n][2 * h], D[n][2 * h + 1]);
    }
}

// ------------------------------------------------------------------------------ gradients of a chunk

// Eight warps: the first four own 16 query rows each (D1, dQ, the dP side), the others 16 key rows
// (M, r D, rb S0, dK).  Values pass in blocks of VW: 64, or 32 where three terms of 128 keys leave room
// for no more.
template <int DK, int NP> constexpr int kGradVW = NP == 3 && DK == 128 ? 32 : 64;

template <int DK, int NP> struct GradSmem {
    static constexpr int NT = NP == 1 ? 2 : 3, VW = kGradVW<DK, NP>;
    bf16 q[NP][kC * (DK + kPad)], k[NP][kC * (DK + kPad)];
    union {
        struct {
            bf16 go[NP][kC * (VW + kPad)], r[NT][kC * (VW + kPad)], rb[NT][kC * (VW + kPad)];
            bf16 s0[NT][VW * (DK + kPad)], ds[NT][VW * (DK + kPad)];
        } v;
        struct {
            bf16 dp[NP][kC * kLd], e[NP][kC * kLd];     // NP terms: what feeds dK only
        } m;
    };
    float coef[kCoef][kC];
    float row_q[kC], row_k[kC];             // row sums of Z plus the row's own terms, query and key side
    float col[8][2][kC];                    // per warp: column sums of Z, of -At.M (key side)
    float dot[8];                           // <S0, D>, per warp
};

__device__ __forceinline__ float quad_sum(float v)      // over the four lanes of a row
{
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}
__device__ __forceinline__ float rows_sum(float v)      // over the eight lanes of a column
{
    v += __shfl_xor_sync(0xffffffffu, v, 4);
    v += __shfl_xor_sync(0xffffffffu, v, 8);
    return v + __shfl_xor_sync(0xffffffffu, v, 16);
}

template <int NP> __device__ __forceinline__ float2 from_terms(const bf16 *at, int plane)
{
    float2 x = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = NP - 1; i >= 0; i--) {
        const float2 y = unpack(*reinterpret_cast<const unsigned *>(at + i * plane));
        x.x += y.x;
        x.y += y.y;
    }
    return x;
}

template <int DK, int NP, class T>
__global__ void __launch_bounds__(256) delta_grads_kernel(const ChunkParams P)
{
    constexpr int ld = DK + kPad, NT = NP == 1 ? 2 : 3, ND = DK / 16, VW = kGradVW<DK, NP>, ldv = VW + kPad;
    extern __shared__ __align__(16) unsigned char raw[];
    auto &sm = *reinterpret_cast<GradSmem<DK, NP> *>(raw);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, w = warp % 4, gr = lane / 4, tc = lane % 4 * 2;
    const bool qside = warp < 4;
    const int c = (int)(blockIdx.x % P.chunks), bk = (int)(blockIdx.x / P.chunks), b = bk / P.Hk, hk = bk % P.Hk, rep = P.Hv / P.Hk;
    const long long t0 = (long long)c * kC;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
    const unsigned qs = smem_addr(sm.q[0]), ks = smem_addr(sm.k[0]);
    const unsigned gos = smem_addr(sm.v.go[0]), rs = smem_addr(sm.v.r[0]), rbs = smem_addr(sm.v.rb[0]), s0s = smem_addr(sm.v.s0[0]), dss = smem_addr(sm.v.ds[0]);
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
        float X[8][4] = {};                 // D1 or M
        float self[2] = {};                 // query side: q.(scale e^G dO S0); key side: -k.(e^G rb S0) - z
        float dot = 0.f;
        for (int v0 = 0; v0 < P.Dv; v0 += VW) {
            const int vcols = P.Dv - v0 < VW ? P.Dv - v0 : VW, in = v0 % kC;
            const long long nv = nc * P.vblocks + v0 / kC;
#pragma unroll
            for (int i = 0; i < NP; i++)
                load_tile<kC, VW, 256>(sm.v.go[i], P.go.at + i * P.go.plane + v_base(P, P.go, bh, t0) + v0, P.go.stride_t, rows, vcols);
#pragma unroll
            for (int i = 0; i < NT; i++) {
                load_tile<kC, VW, 256>(sm.v.r[i], P.r + (nv * 3 + i) * kTile + in, kC, kC, VW);
                load_tile<kC, VW, 256>(sm.v.rb[i], P.rb + (nv * NT + i) * kTile + in, kC, kC, VW);
                load_tile<VW, DK, 256>(sm.v.s0[i], P.s0 + (nv * NT + i) * (kC * DK) + in * DK, DK, VW, DK);
                load_tile<VW, DK, 256>(sm.v.ds[i], P.ds + (nv * NT + i) * (kC * DK) + in * DK, DK, VW, DK);
            }
            cp_commit();
            cp_wait<0>();
            __syncthreads();

            // <S0, D>: the block's rows dealt to the warps
#pragma unroll
            for (int i = lane; i < VW / 8 * DK / 2; i += 32) {
                const int at = (warp * (VW / 8) + i / (DK / 2)) * ld + i % (DK / 2) * 2;
                const float2 x = from_terms<NT>(&sm.v.s0[0][at], VW * ld), y = from_terms<NT>(&sm.v.ds[0][at], VW * ld);
                dot = fmaf(x.x, y.x, fmaf(x.y, y.y, dot));
            }
            if (qside) {
                // D1 = dO r^T (blocks j <= i), and the state's part of dQ
#pragma unroll
                for (int d = 0; d < VW / 16; d++) {
                    unsigned a[NP][4];
                    load_left<NP, false>(a, at_kn(gos, ldv, 16 * w, 16 * d), kC * ldv);
#pragma unroll
                    for (int nb = 0; nb < 4; nb++)
                        if (nb <= w) product<NP, NT, false>(X[2 * nb], X[2 * nb + 1], a, at_nk(rs, ldv, 16 * nb, 16 * d), kC * ldv);
                }
                unsigned a[VW / 16][NP][4];
#pragma unroll
                for (int d = 0; d < VW / 16; d++) load_left<NP, false>(a[d], at_kn(gos, ldv, 16 * w, 16 * d), kC * ldv);
                const float f[2] = {P.scale * sm.coef[COEF_EG][i0], P.scale * sm.coef[COEF_EG][i0 + 8]};
#pragma unroll
                for (int nb = 0; nb < ND; nb++) {
                    float x[2][4] = {};
#pragma unroll
                    for (int d = 0; d < VW / 16; d++) product<NP, NT, true>(x[0], x[1], a[d], at_kn(s0s, ld, 16 * d, 16 * nb), VW * ld);
#pragma unroll
                    for (int m = 0; m < 2; m++)
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            const float2 q = from_terms<NP>(&sm.q[0][(i0 + 8 * h) * ld + 16 * nb + 8 * m + tc], kC * ld);
                            const float y0 = f[h] * x[m][2 * h], y1 = f[h] * x[m][2 * h + 1];
                            self[h] = fmaf(q.x, y0, fmaf(q.y, y1, self[h]));
                            acc[2 * nb + m][2 * h] += y0;
                            acc[2 * nb + m][2 * h + 1] += y1;
                        }
                }
            } else {
#pragma unroll
                for (int d = 0; d < VW / 16; d++) {
                    unsigned a[NT][4];
                    load_left<NT, false>(a, at_kn(rbs, ldv, 16 * w, 16 * d), kC * ldv);
#pragma unroll
                    for (int nb = 0; nb < 4; nb++)
                        if (nb <= w) product<NT, NT, false>(X[2 * nb], X[2 * nb + 1], a, at_nk(rs, ldv, 16 * nb, 16 * d), kC * ldv);
                }
                const float fl[2] = {sm.coef[COEF_LEFT][i0], sm.coef[COEF_LEFT][i0 + 8]};
                const float fb[2] = {sm.coef[COEF_BETA][i0], sm.coef[COEF_BETA][i0 + 8]};
                const float fe[2] = {sm.coef[COEF_EG][i0], sm.coef[COEF_EG][i0 + 8]};
#pragma unroll
                for (int nb = 0; nb < ND; nb++) {
                    float x[2][4] = {}, y[2][4] = {};
#pragma unroll
                    for (int d = 0; d < VW / 16; d++) {
                        unsigned a[NT][4];
                        load_left<NT, false>(a, at_kn(rs, ldv, 16 * w, 16 * d), kC * ldv);
                        product<NP, NP, true>(x[0], x[1], leading<NP>(a), at_kn(dss, ld, 16 * d, 16 * nb), VW * ld);   // feeds dK only
                        load_left<NT, false>(a, at_kn(rbs, ldv, 16 * w, 16 * d), kC * ldv);
                        product<NT, NT, true>(y[0], y[1], a, at_kn(s0s, ld, 16 * d, 16 * nb), VW * ld);
                    }
#pragma unroll
                    for (int m = 0; m < 2; m++)
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            const float2 k = from_terms<NP>(&sm.k[0][(i0 + 8 * h) * ld + 16 * nb + 8 * m + tc], kC * ld);
                            const float x0 = fl[h] * fb[h] * x[m][2 * h], x1 = fl[h] * fb[h] * x[m][2 * h + 1];
                            const float y0 = -fe[h] * y[m][2 * h], y1 = -fe[h] * y[m][2 * h + 1];
                            self[h] = fmaf(k.x, y0, fmaf(k.y, y1, self[h]));
                            acc[2 * nb + m][2 * h] += x0 + y0;
                            acc[2 * nb + m][2 * h + 1] += x1 + y1;
                        }
                }
            }
            __syncthreads();        // the value tiles are free
        }

        // scores of this warp's rows: q.k or k.k, blocks j <= i
        float Y[8][4] = {};
        const unsigned left = qside ? qs : ks;
#pragma unroll
        for (int d = 0; d < ND; d++) {
            unsigned a[NP][4];
            load_left<NP, false>(a, at_kn(left, ld, 16 * w, 16 * d), kC * ld);
#pragma unroll
            for (int nb = 0; nb < 4; nb++)
                if (nb <= w) product<NP, NP, false>(Y[2 * nb], Y[2 * nb + 1], a, at_nk(ks, ld, 16 * nb, 16 * d), kC * ld);
        }
        // X becomes dP or E; sums over rows and columns
        float zrow[2] = {};
#pragma unroll
        for (int n = 0; n < 8; n++) {
            float zc[2] = {}, bc[2] = {};
            if (n / 2 <= w) {
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const int i = i0 + 8 * h, j = 8 * n + tc + e;
                        const bool in = qside ? i >= j : i > j;
                        const float gam = in ? expf((sm.coef[COEF_GHI][i] - sm.coef[COEF_GHI][j]) + (sm.coef[COEF_GLO][i] - sm.coef[COEF_GLO][j])) : 0.f;
                        const float f = (qside ? P.scale : -1.f) * gam, x = in ? f * X[n][2 * h + e] : 0.f;
                        bc[e] += x * Y[n][2 * h + e];               // key side: -At . M
                        const float d = x * sm.coef[COEF_BETA][j], z = i > j ? d * Y[n][2 * h + e] : 0.f;
                        X[n][2 * h + e] = d;
                        zrow[h] += z;
                        zc[e] += z;
                    }
            }
            zc[0] = rows_sum(zc[0]); zc[1] = rows_sum(zc[1]);
            bc[0] = rows_sum(bc[0]); bc[1] = rows_sum(bc[1]);
            if (gr == 0) {
                *reinterpret_cast<float2 *>(&sm.col[warp][0][8 * n + tc]) = make_float2(zc[0], zc[1]);
                *reinterpret_cast<float2 *>(&sm.col[warp][1][8 * n + tc]) = make_float2(bc[0], bc[1]);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const float s = quad_sum(zrow[h] + self[h]);
            if (lane % 4 == 0) (qside ? sm.row_q : sm.row_k)[i0 + 8 * h] = s;
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, o);
        if (lane == 0) sm.dot[warp] = dot;
        // dP and E as tiles (they feed dK transposed)
        bf16 *tile = qside ? sm.m.dp[0] : sm.m.e[0];
#pragma unroll
        for (int n = 0; n < 8; n++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                unsigned x[NP];
                split(X[n][2 * h], X[n][2 * h + 1], x);
#pragma unroll
                for (int i = 0; i < NP; i++) *reinterpret_cast<unsigned *>(tile + i * (kC * kLd) + (i0 + 8 * h) * kLd + 8 * n + tc) = x[i];
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
            float dG[2], z[2], total = 0.f;
            const long long at = ((long long)b * P.L + t0) * P.Hv + bh % P.Hv;
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int t = 2 * lane + e;
                float cz = 0.f, cb = 0.f, rd = 0.f, ru = 0.f;
#pragma unroll
                for (int i = 0; i < 8; i++) cz += sm.col[i][0][t];
#pragma unroll
                for (int i = 4; i < 8; i++) cb += sm.col[i][1][t];
                for (int i = 0; i < 4 * P.vblocks; i++) {
                    const float *from = P.dots + (nc * P.vblocks * 4 + i) * (2 * kC) + t;
                    rd += from[0];
                    ru += from[kC];
                }
                z[e] = sm.coef[COEF_BETA][t] * rd;
                dG[e] = sm.row_q[t] + sm.row_k[t] - cz - z[e];
                total += z[e];
                if (t < rows) P.gbeta[at + (long long)t * P.Hv] = cb + ru;
            }
            // suffix sums inside the chunk, plus what every decay of the chunk touches
            float run = dG[0] + dG[1];
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const float other = __shfl_down_sync(0xffffffffu, run, o);
                if (lane + o < 32) run += other;
                total += __shfl_xor_sync(0xffffffffu, total, o);
            }
            float all = 0.f;
#pragma unroll
            for (int i = 0; i < 8; i++) all += sm.dot[i];
            total = fmaf(sm.coef[COEF_EG][kC - 1], all, total);
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int t = 2 * lane + e;
                if (t < rows) {
                    const long long to = at + (long long)t * P.Hv;
                    // a decay that is zero in float passes nothing on, and its derivative is zero
                    P.gg[to] = P.g[to] < -104.f ? 0.f : run - (e == 1 ? dG[0] : 0.f) + total;
                }
            }
        }
        __syncthreads();        // tiles and sums are free for the next head
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

template <int DK, int NP> cudaError_t reverse(const ChunkParams &P, cudaStream_t st)
{
    using T = typename std::conditional<NP == 1, bf16, float>::type;
    const size_t smem = sizeof(RevStage<DK, NP>) * kRevStages<DK, NP>;
    auto *kernel = delta_reverse_kernel<DK, NP, T>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch(kernel, dim3((unsigned)(P.B * P.Hv), P.vblocks, P.segs), dim3(128), smem, st, P);
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
