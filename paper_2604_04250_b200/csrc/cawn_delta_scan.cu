// Gated delta rule, chunk form: the walk over a head's chunks.
//
// Per chunk and warp (16 value rows, transposed products; see cawn_delta_chunk.cuh):
//   X = S K^T,  R = V^T - e^G X,  r = R T^T,  u = beta r,  O = scale e^G S Q^T + u P^T,
//   S <- e^{G_C} S + (e^{G_C - G} u) K
// Bound: the chain of these products, chunk after chunk, on the tensor pipes of the SMs that have a head.  The
// chain's warps do nothing else; side warps make the outputs from the state and the corrections handed to them.
//
// Few heads leave SMs idle while the chain is long, so the time axis is cut into segments: a chunk acts on
// a state row s as s <- s M + l, so a first pass computes each segment's M (the same walk over the rows
// of the identity with V = 0) and l (from a zero state); a small kernel chains them to every segment's
// start state, and the output pass runs all segments side by side.
#include "cawn_delta_chunk.cuh"

#include <type_traits>

namespace cawn {
namespace {

// OUT: outputs.  SAVE: what the backward needs, dO.o among it (o more exact than bfloat16 stores it).
// SUMMARY: end states and transitions of segments only.
enum { MODE_OUT, MODE_SAVE, MODE_SUMMARY };

// Tiles of the chain; SAVE: and those of dO.o, which its chain takes along.
template <int DK, int NP, int MODE> struct ScanStage {
    static constexpr int NT = NP == 1 ? 2 : 3, VLD = 16 * kRowGroups<NP> + kPad;
    static constexpr bool SAVE = MODE == MODE_SAVE;
    bf16 k[NP][kC * (DK + kPad)], tri[NT][kC * kLd], v[NP][kC * VLD];
    bf16 q[SAVE ? NP : 0][kC * (DK + kPad)], p[SAVE ? NT : 0][kC * kLd], go[SAVE ? NP : 0][kC * VLD];
    float coef[kCoef][kC];
};
// Tiles of the outputs.
template <int DK, int NP> struct ScanSide {
    bf16 q[NP][kC * (DK + kPad)], p[NP][kC * kLd];
    bf16 t[kC * (16 * kRowGroups<NP> + kPad)];          // the way out for token rows
    float coef[kCoef][kC];
};
// From chain to side warp: terms of the state and of u.
template <int DK, int NP> struct ScanSwap {
    uint4 s[NP * DK / 16 * 32], u[NP * 4 * 32];
};

template <int DK, int NP, int MODE> struct ScanPlan {
    static constexpr int RG = kRowGroups<NP>;
    // Measured for the backward's walk too: with dO.o on the side it took 152 us instead of 126, because three
    // terms of everything keep the tensor pipe busy enough, and splitting them twice costs more than it fills.
    static constexpr bool SIDE = MODE == MODE_OUT;
    static constexpr size_t chain = sizeof(ScanStage<DK, NP, MODE>), side = SIDE ? sizeof(ScanSide<DK, NP>) : 0;
    static constexpr size_t swap = SIDE ? sizeof(ScanSwap<DK, NP>) * RG : 0;
    static constexpr Stages n = fit_stages(chain, side, swap);
    static constexpr size_t smem = chain * n.chain + side * n.side + swap * n.swap;
    static constexpr int fetch = SIDE ? RG : kFetch<NP>, threads = 32 * (RG + fetch);       // chain warps, then side or fetching warps
    static_assert(smem <= 227 * 1024, "fits an SM");
};

template <int DK, int NP, int MODE>
__device__ __forceinline__ void scan_load(const ChunkParams &P, ScanStage<DK, NP, MODE> &st, int bh, int c, int v0, int vcols)
{
    constexpr int NT = NP == 1 ? 2 : 3, TH = 32 * ScanPlan<DK, NP, MODE>::fetch, VW = 16 * kRowGroups<NP>;
    const long long t0 = (long long)c * kC, nc = (long long)bh * P.chunks + c;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
#pragma unroll
    for (int i = 0; i < NP; i++) {
        load_tile<kC, DK, TH>(st.k[i], P.k.at + i * P.k.plane + q_base(P, P.k, bh, t0), P.k.stride_t, rows, P.Dk);
        if (vcols > 0) load_tile<kC, VW, TH>(st.v[i], P.v.at + i * P.v.plane + v_base(P, P.v, bh, t0) + v0, P.v.stride_t, rows, vcols);
        if constexpr (MODE == MODE_SAVE) {
            load_tile<kC, DK, TH>(st.q[i], P.q.at + i * P.q.plane + q_base(P, P.q, bh, t0), P.q.stride_t, rows, P.Dk);
            load_tile<kC, VW, TH>(st.go[i], P.go.at + i * P.go.plane + v_base(P, P.go, bh, t0) + v0, P.go.stride_t, rows, vcols);
        }
    }
#pragma unroll
    for (int i = 0; i < NT; i++) {
        load_dense<TH>(st.tri[i], P.tri + (nc * NT + i) * kTile);
        if constexpr (MODE == MODE_SAVE) load_dense<TH>(st.p[i], P.p + (nc * NT + i) * kTile);
    }
    for (int i = threadIdx.x % TH; i < kCoef * kC / 4; i += TH) cp16(smem_addr(&st.coef[0][0]) + i * 16, P.coef + nc * (kCoef * kC) + i * 4, true);
    cp_commit();
}

template <int DK, int NP>
__device__ __forceinline__ void side_load(const ChunkParams &P, ScanSide<DK, NP> &st, int bh, int c)
{
    constexpr int NT = NP == 1 ? 2 : 3, TH = 32 * kRowGroups<NP>;
    const long long t0 = (long long)c * kC, nc = (long long)bh * P.chunks + c;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
#pragma unroll
    for (int i = 0; i < NP; i++) {
        load_tile<kC, DK, TH>(st.q[i], P.q.at + i * P.q.plane + q_base(P, P.q, bh, t0), P.q.stride_t, rows, P.Dk);
        load_dense<TH>(st.p[i], P.p + (nc * NT + i) * kTile);
    }
    for (int i = threadIdx.x % TH; i < kCoef * kC / 4; i += TH) cp16(smem_addr(&st.coef[0][0]) + i * 16, P.coef + nc * (kCoef * kC) + i * 4, true);
    cp_commit();
}

template <int DK, int NP, int MODE, class T>
__global__ void __launch_bounds__((ScanPlan<DK, NP, MODE>::threads), 1) delta_scan_kernel(const ChunkParams P)
{
    using Plan = ScanPlan<DK, NP, MODE>;
    using Side = ScanSide<DK, NP>;
    using Swap = ScanSwap<DK, NP>;
    constexpr int ld = DK + kPad, NT = NP == 1 ? 2 : 3, RG = Plan::RG, VW = 16 * RG, VLD = VW + kPad, CS = Plan::n.chain, SS = Plan::n.side, WS = Plan::n.swap;
    constexpr int PAIR = Plan::threads, ONE = 32 * RG;
    extern __shared__ __align__(16) unsigned char raw[];
    auto *stages = reinterpret_cast<ScanStage<DK, NP, MODE> *>(raw);
    const int bh = blockIdx.x, seg = blockIdx.z;
    const int vblks = (P.Dv + VW - 1) / VW;
    const bool ident = MODE == MODE_SUMMARY && (int)blockIdx.y >= vblks;        // rows of the identity instead of values
    const int r0 = ((int)blockIdx.y - (ident ? vblks : 0)) * VW;                // first value (or identity) row of the block
    const int vcols = ident ? 0 : (P.Dv - r0 < VW ? P.Dv - r0 : VW);
    const int c0 = seg * P.seg_chunks, c1 = c0 + P.seg_chunks < P.chunks ? c0 + P.seg_chunks : P.chunks;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, w = warp % RG, gr = lane / 4, tc = lane % 4 * 2;
    const int w4 = (r0 / 16 + w) % 4;                                           // row group inside its block of 64 values

    if (!Plan::SIDE && warp >= RG) {            // fetch only
        for (int c = c0; c < c1; c++) {
            const int s = (c - c0) % CS;
            if (c - c0 >= CS) bar_sync(BAR_EMPTY + s, PAIR);
            scan_load<DK, NP, MODE>(P, stages[s], bh, c, r0, vcols);
            cp_wait<0>();
            bar_arrive(BAR_FULL + s, PAIR);
        }
        return;
    }
    if constexpr (Plan::SIDE) if (warp >= RG) { // ---------------------------- side warps: tiles and outputs
        auto *tiles = reinterpret_cast<Side *>(raw + Plan::chain * CS);
        scan_load<DK, NP, MODE>(P, stages[0], bh, c0, r0, vcols);
        cp_wait<0>();
        bar_arrive(BAR_FULL, PAIR);
        side_load<DK, NP>(P, tiles[0], bh, c0);
        if (CS == 2 && c0 + 1 < c1) scan_load<DK, NP, MODE>(P, stages[1], bh, c0 + 1, r0, vcols);
        else cp_commit();
        for (int c = c0; c < c1; c++) {
            const int cs = (c - c0) % CS, par = (c - c0) % WS;
            auto &st = tiles[(c - c0) % SS];
            const Swap &sw = reinterpret_cast<const Swap *>(raw + Plan::chain * CS + Plan::side * SS)[par * RG + w];
            const long long t0 = (long long)c * kC;
            const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
            const unsigned qs = smem_addr(st.q[0]), ps = smem_addr(st.p[0]), os = smem_addr(st.t);
            // The side's tiles of this chunk were asked for before the chain's next ones, which may still be on
            // their way until the chain is about to need them.
            if (SS == 2 && CS == 2) cp_wait<1>(); else cp_wait<0>();
            bar_sync(BAR_SIDE, ONE);            // the tiles are here, and the previous chunk's are done with
            if (SS == 2) {
                if (c + 1 < c1) side_load<DK, NP>(P, tiles[(c + 1 - c0) % SS], bh, c + 1);
                else cp_commit();               // an empty group keeps the count
            }
            bar_sync(BAR_READY + par, PAIR);
            // Y = scale e^G S Q^T + u P^T; factors in the output's terms
            float Y[8][4] = {};
#pragma unroll
            for (int d = 0; d < DK / 16; d++) {
                unsigned a[NP][4], b[4][NP][4];
                get_left(a, sw.s, d);
#pragma unroll
                for (int i = 0; i < 4; i++) load_right<NP, false>(b[i], at_nk(qs, ld, 16 * i, 16 * d), kC * ld);
                multiply<NP, NP, 4>(Y, a, b);
            }
#pragma unroll
            for (int n = 0; n < 8; n++) {
                const float2 e = *reinterpret_cast<const float2 *>(&st.coef[COEF_EG][8 * n + tc]);
                const f32x2 f = pair(P.scale * e.x, P.scale * e.y);
                scale_row(Y[n], 0, f);
                scale_row(Y[n], 1, f);
            }
            if (CS == 2 && c + 1 < c1) {        // the chain's next tiles
                if (SS == 2) cp_wait<1>(); else cp_wait<0>();
                bar_arrive(BAR_FULL + (cs ^ 1), PAIR);
            }
            triangle<NP, NP, false, false>(Y, [&](unsigned (&a)[NP][4], int tb) { get_left(a, sw.u, tb); },
                                           [&](int tb, int nb) { return at_nk(ps, kLd, 16 * nb, 16 * tb); }, kC * kLd);
            if (c + WS < c1) bar_arrive(BAR_FREE + par, PAIR);
            if (c + CS >= c1) {
                cp_commit();
            } else {                            // the chain's next tiles but CS - 1
                bar_sync(BAR_EMPTY + cs, PAIR);
                scan_load<DK, NP, MODE>(P, stages[cs], bh, c + CS, r0, vcols);
                if (CS == 1) {
                    cp_wait<0>();
                    bar_arrive(BAR_FULL, PAIR);
                }
            }
            T *o = static_cast<T *>(P.o) + (bh / P.Hv) * P.o_stride_b + t0 * P.o_stride_t + (long long)(bh % P.Hv) * P.Dv + r0;
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int nb = 0; nb < 4; nb++)
                    stsm_t(at_nk(os, VLD, 16 * nb, 16 * w), pack_bf16(Y[2 * nb][0], Y[2 * nb][1]), pack_bf16(Y[2 * nb][2], Y[2 * nb][3]),
                           pack_bf16(Y[2 * nb + 1][0], Y[2 * nb + 1][1]), pack_bf16(Y[2 * nb + 1][2], Y[2 * nb + 1][3]));
                __syncwarp();
#pragma unroll
                for (int i = lane; i < 128; i += 32) {
                    const int t = i / 2, v = 16 * w + i % 2 * 8;
                    if (t < rows && v < vcols)
                        *reinterpret_cast<uint4 *>(o + t * P.o_stride_t + v) = *reinterpret_cast<const uint4 *>(&st.t[t * VLD + v]);
                }
            } else {
#pragma unroll
                for (int n = 0; n < 8; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int t = 8 * n + tc + (e & 1), v = 16 * w + gr + (e >> 1) * 8;
                        if (t < rows && v < vcols) o[t * P.o_stride_t + v] = narrow<T>(Y[n][e]);
                    }
            }
            if (SS == 1 && c + 1 < c1) {
                bar_sync(BAR_SIDE, ONE);
                side_load<DK, NP>(P, tiles[0], bh, c + 1);
            }
        }
        return;
    }

    // -------------------------------------------------------------------------- chain warps
    constexpr int NR = MODE == MODE_SAVE ? 3 : NT;          // terms of R: three where the backward's dots need them
    const int rlim = ident ? P.Dk : P.Dv;                   // rows that exist
    const int row[2] = {r0 + 16 * w + gr, r0 + 16 * w + gr + 8};
    // state rows row[0], row[1]; columns 8 n + tc, +1 of tile n
    float S[DK / 8][4];
    const float *from = nullptr;
    if (MODE != MODE_SUMMARY)
        from = P.segs > 1 ? P.seg_start + ((long long)bh * P.segs + seg) * P.Dv * P.Dk
                          : (P.state_in != nullptr ? P.state_in + (long long)bh * P.Dv * P.Dk : nullptr);
#pragma unroll
    for (int n = 0; n < DK / 8; n++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            float2 x = make_float2(0.f, 0.f);
            const int col = 8 * n + tc;
            if (ident) x = make_float2(row[h] == col ? 1.f : 0.f, row[h] == col + 1 ? 1.f : 0.f);
            else if (from != nullptr && row[h] < P.Dv && col < P.Dk) x = *reinterpret_cast<const float2 *>(from + (long long)row[h] * P.Dk + col);
            S[n][2 * h] = x.x;
            S[n][2 * h + 1] = x.y;
        }

    for (int c = c0; c < c1; c++) {
        const int s = (c - c0) % CS, par = (c - c0) % WS;
        auto &st = stages[s];
        Swap &sw = reinterpret_cast<Swap *>(raw + Plan::chain * CS + Plan::side * SS)[par * RG + w];
        const unsigned ks = smem_addr(st.k[0]), ts = smem_addr(st.tri[0]), vs = smem_addr(st.v[0]);

        const long long nv = ((long long)bh * P.chunks + c) * P.vblocks + r0 / kC;
        if (Plan::SIDE && c - c0 >= WS) bar_sync(BAR_FREE + par, PAIR);
        if constexpr (MODE == MODE_SAVE) {      // the state before the chunk, in float and in the inputs' terms
            bf16 *dst = P.s0 + nv * (NP * kC * DK) + (16 * w4 + gr) * DK + tc;
#pragma unroll
            for (int n = 0; n < DK / 8; n++) {
                P.sf[((nv * 4 + w4) * (DK / 8) + n) * 32 + lane] = make_float4(S[n][0], S[n][1], S[n][2], S[n][3]);
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    unsigned x[NP];
                    split(S[n][2 * h], S[n][2 * h + 1], x);
#pragma unroll
                    for (int i = 0; i < NP; i++) *reinterpret_cast<unsigned *>(dst + i * (kC * DK) + 8 * h * DK + 8 * n) = x[i];
                }
            }
        }
        bar_sync(BAR_FULL + s, PAIR);
        // X = S K^T; SAVE: Y = S Q^T
        float X[8][4] = {}, Y[MODE == MODE_SAVE ? 8 : 1][4] = {};
#pragma unroll
        for (int d = 0; d < DK / 16; d++) {
            constexpr int NS = MODE == MODE_SAVE || NP == 3 ? 3 : 2;
            unsigned a[NS][4], b[4][NP][4];
#pragma unroll
            for (int i = 0; i < 4; i++) load_right<NP, false>(b[i], at_nk(ks, ld, 16 * i, 16 * d), kC * ld);
            as_left(S[2 * d], S[2 * d + 1], a);
            if constexpr (MODE == MODE_OUT) put_left(sw.s, d, leading<NP>(a));
            multiply<NS, NP, 4>(X, a, b);
            if constexpr (MODE == MODE_SAVE) {
#pragma unroll
                for (int i = 0; i < 4; i++) load_right<NP, false>(b[i], at_nk(smem_addr(st.q[0]), ld, 16 * i, 16 * d), kC * ld);
                multiply<NS, NP, 4>(Y, a, b);
            }
        }
        // R = V^T - e^G X (in X, and the start of r)
        float r[8][4];
#pragma unroll
        for (int nb = 0; nb < 4; nb++) {
            unsigned vf[NP][4] = {};
            if (vcols > 0) load_left<NP, true>(vf, at_nk(vs, VLD, 16 * nb, 16 * w), kC * VLD);
#pragma unroll
            for (int m = 0; m < 2; m++) {
                const int n = 2 * nb + m;
                const float2 e = *reinterpret_cast<const float2 *>(&st.coef[COEF_EG][8 * n + tc]);
                const f32x2 minus = pair(-e.x, -e.y);
#pragma unroll
                for (int h = 0; h < 2; h++) fma_row(X[n], h, minus, pair(sum_terms(vf, 2 * m + h)));
#pragma unroll
                for (int i = 0; i < 4; i++) r[n][i] = X[n][i];
                if constexpr (MODE == MODE_SAVE) {
                    const f32x2 f = pair(P.scale * e.x, P.scale * e.y);
                    scale_row(Y[n], 0, f);
                    scale_row(Y[n], 1, f);
                }
            }
        }
        // r = R + R (T - I)^T: tokens t of the result from block t' on
        triangle<NR, NT, true, false>(r, [&](unsigned (&a)[NR][4], int tb) { as_left(X[2 * tb], X[2 * tb + 1], a); },
                                      [&](int tb, int nb) { return at_kn(ts, kLd, 16 * tb, 16 * nb); }, kC * kLd);
        if constexpr (MODE == MODE_SAVE) {
#pragma unroll
            for (int n = 0; n < 8; n++) P.rf[((nv * 4 + w4) * 8 + n) * 32 + lane] = make_float4(r[n][0], r[n][1], r[n][2], r[n][3]);
        }
        // u = beta r, handed over
#pragma unroll
        for (int tb = 0; tb < 4; tb++) {
#pragma unroll
            for (int m = 0; m < 2; m++) {
                const f32x2 bt = pair(*reinterpret_cast<const float2 *>(&st.coef[COEF_BETA][16 * tb + 8 * m + tc]));
                scale_row(r[2 * tb + m], 0, bt);
                scale_row(r[2 * tb + m], 1, bt);
            }
            if constexpr (MODE == MODE_OUT) {
                unsigned a[NP][4];
                as_left(r[2 * tb], r[2 * tb + 1], a);
                put_left(sw.u, tb, a);
            }
        }
        if (Plan::SIDE) bar_arrive(BAR_READY + par, PAIR);
        if constexpr (MODE == MODE_SAVE) {
            const unsigned ps = smem_addr(st.p[0]);
            triangle<3, NT, false, false>(Y, [&](unsigned (&a)[3][4], int tb) { as_left(r[2 * tb], r[2 * tb + 1], a); },
                                          [&](int tb, int nb) { return at_nk(ps, kLd, 16 * nb, 16 * tb); }, kC * kLd);
            // dO.o over this row group's 16 values
            float dots[8][2];
#pragma unroll
            for (int nb = 0; nb < 4; nb++) {
                unsigned g[NP][4];
                load_left<NP, true>(g, at_nk(smem_addr(st.go[0]), VLD, 16 * nb, 16 * w), kC * VLD);
#pragma unroll
                for (int m = 0; m < 2; m++) {
                    const int n = 2 * nb + m;
                    const float2 a = sum_terms(g, 2 * m), b = sum_terms(g, 2 * m + 1);
                    dots[n][0] = fmaf(Y[n][0], a.x, Y[n][2] * b.x);
                    dots[n][1] = fmaf(Y[n][1], a.y, Y[n][3] * b.y);
                }
            }
            column_sums(dots);
            *reinterpret_cast<float2 *>(P.od + (nv * 4 + w4) * kC + 8 * gr + tc) = make_float2(dots[0][0], dots[0][1]);
            // u as token rows in the inputs' terms, through this warp's own part of the V tile
#pragma unroll
            for (int term = 0; term < NP; term++) {
                __syncwarp();
#pragma unroll
                for (int nb = 0; nb < 4; nb++) {
                    unsigned x[NP][4];
                    as_left(r[2 * nb], r[2 * nb + 1], x);
                    stsm_t(at_nk(vs, VLD, 16 * nb, 16 * w), x[term][0], x[term][1], x[term][2], x[term][3]);
                }
                __syncwarp();
#pragma unroll
                for (int i = lane; i < 128; i += 32)
                    *reinterpret_cast<uint4 *>(P.u + (nv * NP + term) * kTile + i / 2 * kC + 16 * w4 + i % 2 * 8) =
                        *reinterpret_cast<const uint4 *>(&st.v[0][i / 2 * VLD + 16 * w + i % 2 * 8]);
            }
        }
        // S <- e^{G_C} S + (e^{G_C - G} u) K.  The update is summed from zero and added once: the tensor
        // core's running sum drops low bits at every step, always towards zero, which on a state that lives
        // for many chunks would add up.
        const float eC = st.coef[COEF_EG][kC - 1];
        unsigned a[4][3][4];
#pragma unroll
        for (int tb = 0; tb < 4; tb++) {
#pragma unroll
            for (int m = 0; m < 2; m++) {
                const f32x2 lf = pair(*reinterpret_cast<const float2 *>(&st.coef[COEF_LEFT][16 * tb + 8 * m + tc]));
                scale_row(r[2 * tb + m], 0, lf);
                scale_row(r[2 * tb + m], 1, lf);
            }
            as_left(r[2 * tb], r[2 * tb + 1], a[tb]);
        }
#pragma unroll
        for (int nb = 0; nb < DK / 16; nb += 2) {
            float x[4][4] = {};
#pragma unroll
            for (int tb = 0; tb < 4; tb++) {
                unsigned b[2][NP][4];
#pragma unroll
                for (int i = 0; i < 2; i++) load_right<NP, true>(b[i], at_kn(ks, ld, 16 * tb, 16 * (nb + i)), kC * ld);
                multiply<3, NP, 2>(x, a[tb], b);
            }
#pragma unroll
            for (int m = 0; m < 4; m++)
#pragma unroll
                for (int h = 0; h < 2; h++) fma_row(S[2 * nb + m], h, pair(eC, eC), pair(x[m][2 * h], x[m][2 * h + 1]));
        }
        if (c + CS < c1) bar_arrive(BAR_EMPTY + s, PAIR);
    }

    float *to = nullptr;
    if (MODE == MODE_SUMMARY)
        to = ident ? P.seg_map + ((long long)bh * P.segs + seg) * P.Dk * P.Dk : P.seg_end + ((long long)bh * P.segs + seg) * P.Dv * P.Dk;
    else if (P.state_out != nullptr && seg == P.segs - 1)
        to = P.state_out + (long long)bh * P.Dv * P.Dk;
    if (to != nullptr) {
#pragma unroll
        for (int n = 0; n < DK / 8; n++)
#pragma unroll
            for (int h = 0; h < 2; h++)
                if (row[h] < rlim && 8 * n + tc < P.Dk)
                    *reinterpret_cast<float2 *>(to + (long long)row[h] * P.Dk + 8 * n + tc) = make_float2(S[n][2 * h], S[n][2 * h + 1]);
    }
    if constexpr (MODE == MODE_SAVE) {
        // the state after the last chunk, for the reverse walk's <state, adjoint>
        const long long nv = ((long long)P.B * P.Hv * P.chunks + bh) * P.vblocks + r0 / kC;
        if (seg == P.segs - 1)
#pragma unroll
            for (int n = 0; n < DK / 8; n++) P.sf[((nv * 4 + w4) * (DK / 8) + n) * 32 + lane] = make_float4(S[n][0], S[n][1], S[n][2], S[n][3]);
    }
}

template <int DK, int NP, int MODE> cudaError_t scan(const ChunkParams &P, cudaStream_t st)
{
    using T = typename std::conditional<NP == 1, bf16, float>::type;
    using Plan = ScanPlan<DK, NP, MODE>;
    auto *kernel = delta_scan_kernel<DK, NP, MODE, T>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Plan::smem);
    if (e != cudaSuccess) return e;
    constexpr int VW = 16 * Plan::RG;
    const int blocks = (P.Dv + VW - 1) / VW + (MODE == MODE_SUMMARY ? (P.Dk + VW - 1) / VW : 0);
    return launch(kernel, dim3((unsigned)(P.B * P.Hv), blocks, P.segs), dim3(Plan::threads), Plan::smem, st, P);
}

// Start states of the segments from their end states and transitions, one segment after the other.  A block has 16
// rows of one head's state, a thread four rows of one column; the next transition is on its way (in registers)
// while the current one is multiplied from shared memory.  Float arithmetic: a few products per segment, once, are
// not worth the tensor cores.  REVERSE: adjoints, last segment first, with the transposed transitions.
template <int DK, bool REVERSE>
__global__ void __launch_bounds__(4 * DK) delta_join_kernel(const ChunkParams P)
{
    extern __shared__ __align__(16) float map[];            // [DK][DK + 1], row k: what state column k sends on
    __shared__ __align__(16) float S[16][DK];
    constexpr int EACH = DK / 4, LD = DK + 1;               // transition elements per thread
    const int col = threadIdx.x % DK, part = threadIdx.x / DK, bh = blockIdx.x, r0 = blockIdx.y * 16 + 4 * part;
    const long long rows = (long long)P.Dv * P.Dk;
    const bool in = col < P.Dk;
    float s[4], end[4], m[EACH];
    auto fetch = [&](int n) {
        const long long seg = (long long)bh * P.segs + (REVERSE ? P.segs - 1 - n : n);
        const float *from = P.seg_map + seg * P.Dk * P.Dk;
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            const int k = 4 * i + part;
            m[i] = in && k < P.Dk ? from[(long long)k * P.Dk + col] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; i++) end[i] = in && r0 + i < P.Dv ? P.seg_end[seg * rows + (long long)(r0 + i) * P.Dk + col] : 0.f;
    };
#pragma unroll
    for (int i = 0; i < 4; i++) s[i] = in && r0 + i < P.Dv && P.state_in != nullptr ? P.state_in[bh * rows + (long long)(r0 + i) * P.Dk + col] : 0.f;
    fetch(0);
    for (int n = 0; n < P.segs; n++) {
        const long long seg = (long long)bh * P.segs + (REVERSE ? P.segs - 1 - n : n);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (in && r0 + i < P.Dv) P.seg_start[seg * rows + (long long)(r0 + i) * P.Dk + col] = s[i];
            S[4 * part + i][col] = s[i];
            s[i] = end[i];
        }
        if (n + 1 == P.segs) break;
#pragma unroll
        for (int i = 0; i < EACH; i++) map[REVERSE ? col * LD + 4 * i + part : (4 * i + part) * LD + col] = m[i];
        __syncthreads();
        fetch(n + 1);
#pragma unroll 4
        for (int k = 0; k < DK; k += 4) {
            const float a = map[k * LD + col], b = map[(k + 1) * LD + col], c = map[(k + 2) * LD + col], d = map[(k + 3) * LD + col];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float4 x = *reinterpret_cast<const float4 *>(&S[4 * part + i][k]);
                s[i] = fmaf(x.x, a, fmaf(x.y, b, fmaf(x.z, c, fmaf(x.w, d, s[i]))));
            }
        }
        __syncthreads();
    }
}

template <int DK, bool REVERSE> cudaError_t join1(const ChunkParams &P, cudaStream_t st)
{
    const size_t smem = DK * (DK + 1) * sizeof(float);
    const cudaError_t e = cudaFuncSetAttribute(delta_join_kernel<DK, REVERSE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch(delta_join_kernel<DK, REVERSE>, dim3((unsigned)(P.B * P.Hv), (P.Dv + 15) / 16), dim3(4 * DK), smem, st, P);
}
template <int DK> cudaError_t join(const ChunkParams &P, bool reverse, cudaStream_t st) { return reverse ? join1<DK, true>(P, st) : join1<DK, false>(P, st); }

template <int DK, int NP> cudaError_t run(const ChunkParams &P, bool save, cudaStream_t st)
{
    if (P.segs > 1) {
        cudaError_t e = scan<DK, NP, MODE_SUMMARY>(P, st);
        if (e == cudaSuccess) e = join<DK>(P, false, st);
        if (e != cudaSuccess) return e;
    }
    return save ? scan<DK, NP, MODE_SAVE>(P, st) : scan<DK, NP, MODE_OUT>(P, st);
}

}  // namespace

cudaError_t launch_delta_join(const ChunkParams &P, int dk, bool reverse, cudaStream_t st)
{
    return dk == 64 ? join<64>(P, reverse, st) : join<128>(P, reverse, st);
}

cudaError_t launch_delta_scan(const ChunkParams &P, int dk, int terms, bool save, cudaStream_t st)
{
    if (dk == 64) return terms == 1 ? run<64, 1>(P, save, st) : run<64, 3>(P, save, st);
    return terms == 1 ? run<128, 1>(P, save, st) : run<128, 3>(P, save, st);
}

}  // namespace cawn
