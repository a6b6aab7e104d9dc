// Gated delta rule, chunk form: the gradients that are local to a chunk, from what the two walks left.
//
//   dP_ij = scale Gam_ij dO_i.u_j (i >= j),   E_ij = -Gam_ij rb_i.u_j (i > j)
//   dQ = scale e^G dO S0 + dP K
//   dK = dP^T Q + e^{G_C - G} u D - e^G rb S0 + (E + E^T) K
// The gradients of beta and g are dots of the walks' float accumulators.  rb is beta times the adjoint of u, so
// dbeta_t = rb_t.r_t / beta_t.  For g: in terms of e^{-G} S the decays appear in o_t as a factor e^{G_t} and in v_t
// as a factor e^{-G_t} only, so with G over the whole sequence
//   dL/dG_t = dO_t.o_t - dV_t.v_t,   dg_t = sum_{s >= t} dL/dG_s,
// taken chunk by chunk: what lies behind the chunk's end is <state, D> there.  Sums of 64 terms, nothing
// accumulates along the sequence.
//
// Bound: instructions and the trip to memory at the start of a block; all chunks of all key heads at once, two
// blocks per SM (3072 chunks of 64 keys and values, bfloat16: 112 us; the scheduler issues in 34% of the cycles,
// 128 registers x 256 threads leave no room for a third block).
#include "cawn_delta_chunk.cuh"

#include <type_traits>

namespace cawn {
namespace {

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
    float dots[8][3][kC];                   // per 16 values: dO.o, rb.v, rb.r (up to 128 values)
    float sd[8];                            // per 16 values: <state after the chunk, D>
};

template <int DK, int NP, class T>
__global__ void __launch_bounds__(256, (DK == 64 && NP == 1 ? 2 : 1)) delta_grads_kernel(const ChunkParams P)
{
    follow_previous();
    constexpr int ld = DK + kPad, ND = DK / 16, VW = kGradVW<DK, NP>, ldv = VW + kPad;
    extern __shared__ __align__(16) unsigned char raw[];
    auto &sm = *reinterpret_cast<GradSmem<DK, NP> *>(raw);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, w = warp % 4, gr = lane / 4, tc = lane % 4 * 2;
    const bool qside = warp < 4;
    const int c = (int)(blockIdx.x % P.chunks), bk = P.key_first + (int)(blockIdx.x / P.chunks), b = bk / P.Hk, hk = bk % P.Hk, rep = P.Hv / P.Hk;
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

    // rb.r per token (first four warps) and <state after the chunk, D> (the others), per row group of the walks.
    auto dots_of_walks = [&](int bh, long long nc, int groups) {
        for (int at = w; at < groups; at += 4) {
            const long long g = nc * P.vblocks * 4 + at;
            if (qside) {
                float dots[8][2];
#pragma unroll
                for (int n = 0; n < 8; n++) {
                    const float4 r = P.rf[(g * 8 + n) * 32 + lane], rb = P.rbf[(g * 8 + n) * 32 + lane];
                    dots[n][0] = fmaf(r.x, rb.x, r.z * rb.z);
                    dots[n][1] = fmaf(r.y, rb.y, r.w * rb.w);
                }
                column_sums(dots);
                *reinterpret_cast<float2 *>(&sm.dots[at][2][8 * gr + tc]) = make_float2(dots[0][0], dots[0][1]);
            } else {
                const long long next = c + 1 < P.chunks ? g + P.vblocks * 4 : ((long long)P.B * P.Hv * P.chunks + bh) * P.vblocks * 4 + at;
                float dot = 0.f;
#pragma unroll
                for (int n = 0; n < DK / 8; n++) {
                    const float4 s = P.sf[(next * (DK / 8) + n) * 32 + lane], d = P.df[(g * (DK / 8) + n) * 32 + lane];
                    dot = fmaf(s.x, d.x, fmaf(s.y, d.y, fmaf(s.z, d.z, fmaf(s.w, d.w, dot))));
                }
#pragma unroll
                for (int o = 16; o > 0; o /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, o);
                if (lane == 0) sm.sd[at] = dot;
            }
        }
    };

    float acc[2 * ND][4] = {};              // dQ or dK rows of this warp, over the heads that share them
    const int i0 = 16 * w + gr;             // rows i0 and i0 + 8

    for (int hv = 0; hv < rep; hv++) {
        const int bh = b * P.Hv + hk * rep + hv;
        const long long nc = (long long)bh * P.chunks + c;
        if (threadIdx.x < kCoef * 16)
            cp16(smem_addr(&sm.coef[0][0]) + threadIdx.x * 16, P.coef + nc * (kCoef * kC) + threadIdx.x * 4, true);
        const int groups = (P.Dv + 15) / 16;                // row groups of the walks
        const long long g0 = nc * P.vblocks * 4;
        for (int i = threadIdx.x; i < groups * (P.together ? 32 : 48); i += 256) {
            const int at = i / 16 % groups, what = i / 16 / groups, x = i % 16 * 4;
            cp16(smem_addr(&sm.dots[at][what][x]), (what == 0 ? P.od : what == 1 ? P.rv : P.rr) + (g0 + at) * kC + x, true);
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
            if (v0 == 0 && P.together) dots_of_walks(bh, nc, groups);       // while the tiles are on their way
            else if (v0 == 0 && threadIdx.x < groups) sm.sd[threadIdx.x] = P.sd[g0 + threadIdx.x];
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
            for (int i = 0; i < groups; i++) end += sm.sd[i];
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int t = 2 * lane + e;
                float od = 0.f, rr = 0.f, rv = 0.f;
                for (int i = 0; i < groups; i++) {
                    od += sm.dots[i][0][t];
                    rv += sm.dots[i][1][t];
                    rr += sm.dots[i][2][t];
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

template <int DK, int NP> cudaError_t grads(const ChunkParams &P, cudaStream_t st)
{
    using T = typename std::conditional<NP == 1, bf16, float>::type;
    const size_t smem = sizeof(GradSmem<DK, NP>);
    static_assert(sizeof(GradSmem<DK, NP>) <= 227 * 1024, "fits an SM");
    auto *kernel = delta_grads_kernel<DK, NP, T>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch(kernel, dim3((unsigned)(P.key_heads * (long long)P.chunks)), dim3(256), smem, st, P);
}

}  // namespace

cudaError_t launch_delta_grads(const ChunkParams &P, int dk, int terms, cudaStream_t st)
{
    if (dk == 64) return terms == 1 ? grads<64, 1>(P, st) : grads<64, 3>(P, st);
    return terms == 1 ? grads<128, 1>(P, st) : grads<128, 3>(P, st);
}

}  // namespace cawn
