// Gated delta rule, chunk form: the gradients that are local to a chunk, from what the two walks left.
//
//   dP_ij = scale Gam_ij beta_j dO_i.r_j (i >= j),   E_ij = -Gam_ij beta_j rb_i.r_j (i > j)
//   dQ = scale e^G dO S0 + dP K
//   dK = dP^T Q + e^{G_C - G} u D - e^G rb S0 + (E + E^T) K,   u = beta r
// rb is beta times the adjoint of u, so dbeta_t = rb_t.r_t / beta_t.  For g: the decay of token t is a factor of what
// passes from a token j < t (or from S0) to a token i >= t (or to the chunk's end), so with
//   W_ij = dP_ij q_i.k_j + E_ij k_i.k_j,   a_i = e^G_i (scale q_i.(dO_i S0) - k_i.(rb_i S0)),   z_j = e^{G_C - G_j} k_j.(u_j D)
//   dg_t = sum_{j < t <= i} W_ij + sum_{i >= t} a_i + sum_{j < t} z_j + e^{G_C} <S0, D>,
// in which every term carries the decay: no two large ones cancel, and a token's gradient is as small as its decay is
// strong.  (As a suffix sum of dO.o - dV.v, which is cheaper, terms of order one cancelled: heads with g = -8 were off by
// 7e-3 of their gradient, with g = -12 by half of it.)
//
// Precision: with bfloat16 storage r, rb and both states enter products in two terms and pairs of those take all four
// products; z and <S0, D> are float.
//
// Bound: the chains of products within a warp, the barriers between them and the trip to memory at the start of a
// block; all chunks of all key heads at once, two blocks per SM of 64 keys and values in bfloat16, at the 128 registers a
// thread that these leave (3072 chunks: 188 us; an earlier form took 12% longer with one block and 255 registers).
#include "cawn_delta_chunk.cuh"

#include <type_traits>

namespace cawn {
namespace {

// Eight warps: the first four own 16 query rows each (dP, dQ), the others 16 key rows (E, dK).  Values pass in
// blocks of VW: 64, or 32 where three terms of 128 keys leave room for no more.
template <int DK, int NP> constexpr int kGradVW = NP == 3 && DK == 128 ? 32 : 64;

template <int DK, int NP> struct GradSmem {
    static constexpr int NT = NP == 1 ? 2 : 3, VW = kGradVW<DK, NP>, LDV = VW + kPad;
    bf16 q[NP][kC * (DK + kPad)], k[NP][kC * (DK + kPad)];
    union {
        struct {
            bf16 go[NP][kC * LDV], rb[NT][kC * LDV], r[NT][VW * kLd];      // r as value rows
            bf16 s0[NT][VW * (DK + kPad)], ds[NT][VW * (DK + kPad)];
        } v;
        struct {
            bf16 dp[NT][kC * kLd], e[NT][kC * kLd];
        } m;
    };
    float coef[kCoef][kC];
    float pairs[8][kC];                     // per warp: its rows' part of the sum over pairs
    float dots[2][kC];                      // a of the query rows, a of the key rows
    float ends[8];                          // per warp: its part of <S0, D>
    union {
        float4 handed[4][4][32];            // from a query warp to its key warp: accumulators of two column blocks
        float z[8][kC];                     // then, per warp, its part of z
    };
};
enum { DOTS_Q = 0, DOTS_K = 1 };

// Sum over the four lanes that share a row
__device__ __forceinline__ float row_sum(float v)
{
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}
// N words of four floats of a thread's share of two arrays with rows of COLS, zero from row `rows` on.
template <int COLS, int N> __device__ __forceinline__ void fetch_rows(float4 (&x)[N], float4 (&y)[N], const float *from_x, const float *from_y, int rows)
{
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int at = i * 256 + threadIdx.x;
        x[i] = y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at / (COLS / 4) < rows) {
            x[i] = reinterpret_cast<const float4 *>(from_x)[at];
            y[i] = reinterpret_cast<const float4 *>(from_y)[at];
        }
    }
}
// a word as terms into a tile, planes `plane` elements apart
template <int NT> __device__ __forceinline__ void put_terms(bf16 *to, int plane, float4 x)
{
    unsigned a[NT], b[NT];
    split(x.x, x.y, a);
    split(x.z, x.w, b);
#pragma unroll
    for (int n = 0; n < NT; n++) *reinterpret_cast<uint2 *>(to + n * plane) = make_uint2(a[n], b[n]);
}
// What the walks left of a block of values, from floats to terms in the tiles; <S0, D> and r.(D K^T) in float on the way.
// (Those dots make the gradients of g where decays are weak, and are often small differences: from products of two
// terms the gradients of short sequences were off by up to 2e-5.)
template <int DK, int NP>
__device__ __forceinline__ void load_floats(GradSmem<DK, NP> &sm, const ChunkParams &P, long long nv, int in, int rows, float &dot, float4 &z)
{
    constexpr int NT = GradSmem<DK, NP>::NT, VW = GradSmem<DK, NP>::VW, ld = DK + kPad;
    float4 s[VW * DK / 1024], d[VW * DK / 1024], x[VW * kC / 1024], y[VW * kC / 1024];
    fetch_rows<DK>(s, d, P.s0 + nv * (kC * DK) + in * DK, P.ds + nv * (kC * DK) + in * DK, rows);
    fetch_rows<kC>(x, y, P.r + nv * kTile + in * kC, P.dk + nv * kTile + in * kC, rows);
#pragma unroll
    for (int i = 0; i < VW * DK / 1024; i++) {
        const int at = i * 256 + threadIdx.x, to = at / (DK / 4) * ld + at % (DK / 4) * 4;
        dot = fmaf(s[i].x, d[i].x, fmaf(s[i].y, d[i].y, fmaf(s[i].z, d[i].z, fmaf(s[i].w, d[i].w, dot))));
        put_terms<NT>(sm.v.s0[0] + to, VW * ld, s[i]);
        put_terms<NT>(sm.v.ds[0] + to, VW * ld, d[i]);
    }
#pragma unroll
    for (int i = 0; i < VW * kC / 1024; i++) {
        const int at = i * 256 + threadIdx.x, to = at / (kC / 4) * kLd + at % (kC / 4) * 4;
        z.x = fmaf(x[i].x, y[i].x, z.x);
        z.y = fmaf(x[i].y, y[i].y, z.y);
        z.z = fmaf(x[i].z, y[i].z, z.z);
        z.w = fmaf(x[i].w, y[i].w, z.w);
        put_terms<NT>(sm.v.r[0] + to, VW * kLd, x[i]);
    }
}

// x (column blocks nb, nb + 1 of a side's rows) = f (by row half) rows (NA terms, at `left`) x state; dots += x times this
// thread's places of a tile (NP planes, its row i0 at `own`).  Two column blocks at a time: the left factors are read
// again for each two, which leaves the registers to the sums.  OF_R: the rows are r's, stored transposed; no dots.
template <int DK, int NP, int NA, bool OF_R>
__device__ __forceinline__ void times_state(float (&x)[4][4], int nb, unsigned left, unsigned state, const f32x2 (&f)[2], f32x2 (&dots)[2], const bf16 *own)
{
    using Smem = GradSmem<DK, NP>;
    constexpr int NT = Smem::NT, MORE = NA == 2 ? 1 : 0, VW = Smem::VW, ldv = Smem::LDV, ld = DK + kPad;
    const int w = threadIdx.x / 32 % 4;
#pragma unroll
    for (int n = 0; n < 4; n++)
#pragma unroll
        for (int e = 0; e < 4; e++) x[n][e] = 0.f;
#pragma unroll
    for (int d = 0; d < VW / 16; d++) {
        unsigned a[NA][4], b[2][NT][4];
        if (OF_R) load_left<NA, true>(a, at_nk(left, kLd, 16 * d, 16 * w), VW * kLd);
        else load_left<NA, false>(a, at_kn(left, ldv, 16 * w, 16 * d), kC * ldv);
#pragma unroll
        for (int i = 0; i < 2; i++) load_right<NT, true>(b[i], at_kn(state, ld, 16 * d, 16 * (nb + i)), VW * ld);
        multiply<NA, NT, 2, MORE>(x, a, b);
    }
#pragma unroll
    for (int n = 0; n < 4; n++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const f32x2 y = mul2(f[h], pair(x[n][2 * h], x[n][2 * h + 1]));
            x[n][2 * h] = halves(y).x;
            x[n][2 * h + 1] = halves(y).y;
            if (OF_R) continue;
            const bf16 *at = own + 8 * h * ld + 16 * nb + 8 * n;
            f32x2 k = pair(unpack(*reinterpret_cast<const unsigned *>(at)));
#pragma unroll
            for (int i = 1; i < NP; i++) k = add2(k, pair(unpack(*reinterpret_cast<const unsigned *>(at + i * (kC * ld)))));
            dots[h] = fma2(y, k, dots[h]);
        }
}
template <int N> __device__ __forceinline__ void add_tiles(float (*acc)[4], const float (&x)[N][4])
{
#pragma unroll
    for (int n = 0; n < N; n++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const float2 y = halves(add2(pair(acc[n][2 * h], acc[n][2 * h + 1]), pair(x[n][2 * h], x[n][2 * h + 1])));
            acc[n][2 * h] = y.x;
            acc[n][2 * h + 1] = y.y;
        }
}

// A side's products with a block of values: X += rows r^T; acc += f rows S0; a.  The query side, which has less to do,
// also makes the key side's e^{G_C - G} u D and hands it over, two column blocks at a time (all of it on the key side: 3072
// chunks 209 us where they now took 180, before r and the states came as floats).
enum { BAR_HANDED = 1, BAR_TAKEN = 2 };
template <int DK, int NP, bool QSIDE>
__device__ __forceinline__ void with_values(GradSmem<DK, NP> &sm, float (&X)[8][4], float (&acc)[DK / 8][4], f32x2 (&dots)[2], float scale)
{
    using Smem = GradSmem<DK, NP>;
    constexpr int NT = Smem::NT, NA = QSIDE ? NP : NT, MORE = NA == 2 ? 1 : 0, ldv = Smem::LDV, ld = DK + kPad;
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32 % 4, gr = lane / 4, tc = lane % 4 * 2, i0 = 16 * w + gr;
    const unsigned mine = QSIDE ? smem_addr(sm.v.go[0]) : smem_addr(sm.v.rb[0]), rs = smem_addr(sm.v.r[0]);
    const unsigned s0s = smem_addr(sm.v.s0[0]), dss = smem_addr(sm.v.ds[0]);
    const bf16 *own = (QSIDE ? sm.q[0] : sm.k[0]) + i0 * ld + tc;
#pragma unroll
    for (int d = 0; d < Smem::VW / 16; d++) {
        unsigned a[NA][4];
        load_left<NA, false>(a, at_kn(mine, ldv, 16 * w, 16 * d), kC * ldv);
#pragma unroll
        for (int nb = 0; nb < 4; nb += 2) {
            if (nb + 1 <= w) {
                unsigned b[2][NT][4];
                load_right<NT, true>(b[0], at_kn(rs, kLd, 16 * d, 16 * nb), Smem::VW * kLd);
                load_right<NT, true>(b[1], at_kn(rs, kLd, 16 * d, 16 * nb + 16), Smem::VW * kLd);
                multiply<NA, NT, 2, MORE>(reinterpret_cast<float (&)[4][4]>(X[2 * nb]), a, b);
            } else if (nb == w) {
                product<NA, NT, true, MORE>(X[2 * nb], X[2 * nb + 1], a, at_kn(rs, kLd, 16 * d, 16 * nb), Smem::VW * kLd);
            }
        }
    }
    auto twice = [](float v) { return pair(v, v); };
    const float sign = QSIDE ? scale : -1.f;
    const f32x2 f[2] = {twice(sign * sm.coef[COEF_EG][i0]), twice(sign * sm.coef[COEF_EG][i0 + 8])};
    const f32x2 g[2] = {twice(sm.coef[COEF_LEFT][i0] * sm.coef[COEF_BETA][i0]), twice(sm.coef[COEF_LEFT][i0 + 8] * sm.coef[COEF_BETA][i0 + 8])};
#pragma unroll
    for (int nb = 0; nb < DK / 16; nb += 2) {
        float x[4][4];
        if constexpr (QSIDE) {
            times_state<DK, NP, NT, true>(x, nb, rs, dss, g, dots, nullptr);
            if (nb > 0) bar_sync(BAR_TAKEN, 256);
#pragma unroll
            for (int n = 0; n < 4; n++) sm.handed[w][n][lane] = make_float4(x[n][0], x[n][1], x[n][2], x[n][3]);
            bar_arrive(BAR_HANDED, 256);
        }
        times_state<DK, NP, NA, false>(x, nb, mine, s0s, f, dots, own);
        add_tiles<4>(acc + 2 * nb, x);
        if constexpr (!QSIDE) {
            bar_sync(BAR_HANDED, 256);
#pragma unroll
            for (int n = 0; n < 4; n++) {
                const float4 y = sm.handed[w][n][lane];
                x[n][0] = y.x; x[n][1] = y.y; x[n][2] = y.z; x[n][3] = y.w;
            }
            if (nb + 2 < DK / 16) bar_arrive(BAR_TAKEN, 256);
            add_tiles<4>(acc + 2 * nb, x);
        }
    }
}

// dP or E from X, as left factors (xa) and as a tile (for dK, transposed), and for every token t the sum over this warp's
// rows i >= t and all j < t of it times the rows' scores with the keys.  A row's sum over j < t is a running sum without
// what lies at t (which may be larger than all of it).  Key side: the gradients of beta, which are X's diagonal.
template <int DK, int NP, bool QSIDE>
__device__ __forceinline__ void weights(GradSmem<DK, NP> &sm, float (&X)[8][4], unsigned (&xa)[4][GradSmem<DK, NP>::NT][4], float scale, float *gbeta, long long step, int valid)
{
    constexpr int ld = DK + kPad, NT = GradSmem<DK, NP>::NT;
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32 % 4, gr = lane / 4, tc = lane % 4 * 2, i0 = 16 * w + gr;
    const unsigned keys = smem_addr(sm.k[0]), rows = QSIDE ? smem_addr(sm.q[0]) : keys;
    bf16 *tile = QSIDE ? sm.m.dp[0] : sm.m.e[0];
    const f32x2 sign = QSIDE ? pair(scale, scale) : pair(-1.f, -1.f);
    const float hi0 = sm.coef[COEF_GHI][i0], lo0 = sm.coef[COEF_GLO][i0], hi8 = sm.coef[COEF_GHI][i0 + 8], lo8 = sm.coef[COEF_GLO][i0 + 8];
    const f32x2 hi[2] = {pair(hi0, hi0), pair(hi8, hi8)}, lo[2] = {pair(lo0, lo0), pair(lo8, lo8)}, minus = pair(-1.f, -1.f);
    float run[2] = {0.f, 0.f}, sums[8][2];
#pragma unroll
    for (int nb = 0; nb < 4; nb++) {
        sums[2 * nb][0] = sums[2 * nb][1] = sums[2 * nb + 1][0] = sums[2 * nb + 1][1] = 0.f;
        if (nb > w) continue;
        float s[2][4] = {};
#pragma unroll
        for (int d = 0; d < DK / 16; d++) {
            unsigned a[NP][4];
            load_left<NP, false>(a, at_kn(rows, ld, 16 * w, 16 * d), kC * ld);
            product<NP, NP, false>(s[0], s[1], a, at_nk(keys, ld, 16 * nb, 16 * d), kC * ld);
        }
#pragma unroll
        for (int m = 0; m < 2; m++) {
            const int n = 2 * nb + m, j = 8 * n + tc;
            auto two = [&](int which) { return *reinterpret_cast<const f32x2 *>(&sm.coef[which][j]); };
            const f32x2 factor = mul2(sign, two(COEF_BETA)), jhi = two(COEF_GHI), jlo = two(COEF_GLO);
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int i = i0 + 8 * h;
                float2 x = make_float2(X[n][2 * h], X[n][2 * h + 1]);
                if (!QSIDE && nb == w && i < valid && (i == j || i == j + 1)) gbeta[i * step] = (i == j ? x.x : x.y) / sm.coef[COEF_BETA][i];
                const float2 g = halves(add2(fma2(jhi, minus, hi[h]), fma2(jlo, minus, lo[h])));
                x = halves(mul2(mul2(factor, pair(exp2_fast(g.x), exp2_fast(g.y))), pair(x)));
                if (nb == w) {
                    if (QSIDE ? i < j : i <= j) x.x = 0.f;
                    if (QSIDE ? i < j + 1 : i <= j + 1) x.y = 0.f;
                }
                X[n][2 * h] = x.x;
                X[n][2 * h + 1] = x.y;
                const float w0 = x.x * s[m][2 * h], w1 = x.y * s[m][2 * h + 1];
                float upto = w0 + w1;
#pragma unroll
                for (int o = 1; o < 4; o *= 2) {
                    const float other = __shfl_up_sync(0xffffffffu, upto, o, 4);
                    if (lane % 4 >= o) upto += other;
                }
                const float left = __shfl_up_sync(0xffffffffu, upto, 1, 4), before = run[h] + (lane % 4 > 0 ? left : 0.f);
                if (nb < w || j <= i) sums[n][0] += before;
                if (nb < w || j + 1 <= i) sums[n][1] += before + w0;
                run[h] += __shfl_sync(0xffffffffu, upto, 3, 4);
            }
        }
        as_left(X[2 * nb], X[2 * nb + 1], xa[nb]);
#pragma unroll
        for (int m = 0; m < NT; m++)
#pragma unroll
            for (int e = 0; e < 4; e++)
                *reinterpret_cast<unsigned *>(tile + m * (kC * kLd) + (i0 + e % 2 * 8) * kLd + 16 * nb + e / 2 * 8 + tc) = xa[nb][m][e];
    }
    column_sums(sums);
    *reinterpret_cast<float2 *>(&sm.pairs[threadIdx.x / 32][8 * gr + tc]) = make_float2(sums[0][0], sums[0][1]);
}

// ONE: one block of values and one value head per key head, so that all sums begin in the block and the registers are free
// for what is fetched first (3072 chunks: 188 us, in the general form, which spills 456 bytes, 215).
template <int DK, int NP, bool ONE, class T>
__global__ void __launch_bounds__(256, (DK == 64 && NP == 1 ? 2 : 1)) delta_grads_kernel(const ChunkParams P)
{
    follow_previous();
    using Smem = GradSmem<DK, NP>;
    constexpr int ld = DK + kPad, ND = DK / 16, VW = Smem::VW, NT = Smem::NT;
    extern __shared__ __align__(16) unsigned char raw[];
    auto &sm = *reinterpret_cast<Smem *>(raw);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, w = warp % 4, gr = lane / 4, tc = lane % 4 * 2;
    const bool qside = warp < 4;
    const int c = (int)(blockIdx.x % P.chunks), bk = (int)(blockIdx.x / P.chunks), b = bk / P.Hk, hk = bk % P.Hk, rep = ONE ? 1 : P.Hv / P.Hk;
    const long long t0 = (long long)c * kC;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
    const unsigned qs = smem_addr(sm.q[0]), ks = smem_addr(sm.k[0]);
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
        const long long nc = (long long)bh * P.chunks + c, at = ((long long)b * P.L + t0) * P.Hv + bh % P.Hv;
        if (threadIdx.x < kCoef * 16)
            cp16(smem_addr(&sm.coef[0][0]) + threadIdx.x * 16, P.coef + nc * (kCoef * kC) + threadIdx.x * 4, true);
        float X[8][4] = {};                 // dO.r or rb.r, then dP or E
        f32x2 a_dots[2] = {};
        float end = 0.f;
        float4 z4 = make_float4(0.f, 0.f, 0.f, 0.f);       // of tokens 4 (lane % 16) ..
        for (int v0 = 0; v0 < (ONE ? VW : P.Dv); v0 += VW) {
            const int vcols = P.Dv - v0 < VW ? P.Dv - v0 : VW, in = v0 % kC;
            const long long nv = nc * P.vblocks + v0 / kC, here = v_base(P, P.rb, bh, t0) + v0;
#pragma unroll
            for (int i = 0; i < NP; i++) load_tile<kC, VW, 256>(sm.v.go[i], P.go.at + i * P.go.plane + v_base(P, P.go, bh, t0) + v0, P.go.stride_t, rows, vcols);
#pragma unroll
            for (int i = 0; i < NT; i++) {
                const bf16 *rb = NP == 1 && i == 0 ? static_cast<const bf16 *>(P.o) : P.rbt + (i - (NP == 1 ? 1 : 0)) * P.rb.plane;
                load_tile<kC, VW, 256>(sm.v.rb[i], rb + here, P.rb.stride_t, rows, vcols);
            }
            cp_commit();
            load_floats<DK, NP>(sm, P, nv, in, vcols, end, z4);
            cp_wait<0>();
            __syncthreads();
            if (qside) with_values<DK, NP, true>(sm, X, acc, a_dots, P.scale);
            else with_values<DK, NP, false>(sm, X, acc, a_dots, P.scale);
            __syncthreads();        // the value tiles are free
        }

        unsigned xa[4][NT][4];              // dP or E as left factors
        if (qside) weights<DK, NP, true>(sm, X, xa, P.scale, nullptr, 0, 0);
        else weights<DK, NP, false>(sm, X, xa, P.scale, P.gbeta + at, P.Hv, rows);
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const float2 ah = halves(a_dots[h]);
            const float a = row_sum(ah.x + ah.y);
            if (tc == 0) sm.dots[qside ? DOTS_Q : DOTS_K][i0 + 8 * h] = a;
        }
        z4.x += __shfl_xor_sync(0xffffffffu, z4.x, 16);
        z4.y += __shfl_xor_sync(0xffffffffu, z4.y, 16);
        z4.z += __shfl_xor_sync(0xffffffffu, z4.z, 16);
        z4.w += __shfl_xor_sync(0xffffffffu, z4.w, 16);
        if (lane < 16) *reinterpret_cast<float4 *>(&sm.z[warp][4 * lane]) = z4;
#pragma unroll
        for (int o = 16; o > 0; o /= 2) end += __shfl_xor_sync(0xffffffffu, end, o);
        if (lane == 0) sm.ends[warp] = end;
        __syncthreads();

        // dQ += dP K;  dK += E K + E^T K + dP^T Q, each head's sum from zero
#pragma unroll
        for (int nb = 0; nb < ND; nb++) {
            float x[2][4] = {};
#pragma unroll
            for (int jb = 0; jb < 4; jb++) {
                unsigned a[NT][4];
                if (jb <= w) {
                    product<NT, NP, true>(x[0], x[1], xa[jb], at_kn(ks, ld, 16 * jb, 16 * nb), kC * ld);
                }
                if (!qside && jb >= w) {
                    load_left<NT, true>(a, at_nk(es, kLd, 16 * jb, 16 * w), kC * kLd);
                    product<NT, NP, true>(x[0], x[1], a, at_kn(ks, ld, 16 * jb, 16 * nb), kC * ld);
                    load_left<NT, true>(a, at_nk(dps, kLd, 16 * jb, 16 * w), kC * kLd);
                    product<NT, NP, true>(x[0], x[1], a, at_kn(qs, ld, 16 * jb, 16 * nb), kC * ld);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                acc[2 * nb][e] += x[0][e];
                acc[2 * nb + 1][e] += x[1][e];
            }
        }
        // decays: one warp, two tokens a lane; sums over later tokens (a) and earlier ones (z) without subtractions
        if (warp == 0) {
            float pairs[2] = {0.f, 0.f}, a[2], z[2], state = 0.f;
            for (int i = 0; i < 8; i++) state += sm.ends[i];
            state *= sm.coef[COEF_EG][kC - 1];
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int t = 2 * lane + e;
                for (int i = 0; i < 8; i++) pairs[e] += sm.pairs[i][t];
                a[e] = sm.dots[DOTS_Q][t] + sm.dots[DOTS_K][t];
                z[e] = 0.f;
                for (int i = 0; i < 8; i++) z[e] += sm.z[i][t];
                z[e] *= sm.coef[COEF_LEFT][t] * sm.coef[COEF_BETA][t];
            }
            float after = a[0] + a[1], before = z[0] + z[1];
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const float x = __shfl_down_sync(0xffffffffu, after, o), y = __shfl_up_sync(0xffffffffu, before, o);
                if (lane + o < 32) after += x;
                if (lane >= o) before += y;
            }
            after = __shfl_down_sync(0xffffffffu, after, 1);
            before = __shfl_up_sync(0xffffffffu, before, 1);
            if (lane == 31) after = 0.f;
            if (lane == 0) before = 0.f;
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int t = 2 * lane + e;
                const float late = e == 0 ? a[0] + (a[1] + after) : a[1] + after, early = e == 0 ? before : before + z[0];
                if (t < rows) P.gg[at + (long long)t * P.Hv] = pairs[e] + (late + early) + state;
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

template <int DK, int NP, bool ONE> cudaError_t grads(const ChunkParams &P, cudaStream_t st)
{
    using T = typename std::conditional<NP == 1, bf16, float>::type;
    const size_t smem = sizeof(GradSmem<DK, NP>);
    static_assert(sizeof(GradSmem<DK, NP>) <= 227 * 1024, "fits an SM");
    auto *kernel = delta_grads_kernel<DK, NP, ONE, T>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch(kernel, dim3((unsigned)(P.B * P.Hk * (long long)P.chunks)), dim3(256), smem, st, P);
}

}  // namespace

cudaError_t launch_delta_grads(const ChunkParams &P, int dk, int terms, cudaStream_t st)
{
    if (dk == 64 && terms == 1) return P.Hk == P.Hv && P.Dv <= kGradVW<64, 1> ? grads<64, 1, true>(P, st) : grads<64, 1, false>(P, st);
    if (dk == 64) return grads<64, 3, false>(P, st);
    return terms == 1 ? grads<128, 1, false>(P, st) : grads<128, 3, false>(P, st);
}

}  // namespace cawn
