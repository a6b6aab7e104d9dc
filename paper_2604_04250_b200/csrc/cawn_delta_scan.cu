// Gated delta rule, chunk form: the walk over a head's chunks.
//
// Per chunk and warp (16 value rows, transposed products; see cawn_delta_chunk.cuh):
//   X = S K^T,  R = V^T - e^G X,  r = R T^T,  u = beta r,  O = scale e^G S Q^T + u P^T,
//   S <- e^{G_C} S + (e^{G_C - G} u) K
// Bound: the chain of these products, chunk after chunk, on the tensor pipes of the SMs that have a head.  The
// chain's warps do nothing else; side warps make the outputs from the state and the corrections handed to them.
// Measured: 96 heads of 64 x 64, 2048 tokens, bfloat16: 87 us, 2.7 us a chunk; the tensor pipes of the 96 SMs are busy 59%
// of the time with the chain's 220 products and the outputs' 124 a chunk and row group (with 52 for the outputs, whose
// factors then had 8 bits, 75 us).  64 blocks of 128 x 64, 4096 tokens: 237 us, pipes busy 69%.
//
// Few heads leave SMs idle while the chain is long, so the time axis is cut into segments: a chunk acts on
// a state row s as s <- s M + l, so a first pass computes each segment's M (the same walk over the rows
// of the identity with V = 0) and l (from a zero state); a small kernel chains them to every segment's
// start state, and the output pass runs all segments side by side.  12 heads x 32768 tokens in 12 segments: 137 us for
// the first pass, 18 for the chaining, 127 for the outputs; in one segment the walk took 1.5 ms.
#include "cawn_delta_chunk.cuh"

#include <type_traits>

namespace cawn {
namespace {

// OUT: outputs.  SUMMARY: end states and transitions of segments only.
enum { MODE_OUT, MODE_SUMMARY };

// Tiles of the chain.
template <int DK, int NP> struct ScanStage {
    static constexpr int NT = NP == 1 ? 2 : 3, VLD = 16 * kRowGroups<NP> + kPad;
    bf16 k[NP][kC * (DK + kPad)], tri[NT][kTri], v[NP][kC * VLD];
    float coef[kCoef][kC];
};
// Tiles of the outputs.
template <int DK, int NP> struct ScanSide {
    static constexpr int NT = NP == 1 ? 2 : 3;
    bf16 q[NP][kC * (DK + kPad)], p[NT][kTri];
    bf16 t[kC * (16 * kRowGroups<NP> + kPad)];          // the way out for token rows
    float coef[kCoef][kC];
};
// From chain to side warp: terms of the state and of u.
template <int DK, int NP> struct ScanSwap {
    static constexpr int NT = NP == 1 ? 2 : 3;
    uint4 s[NT * DK / 16 * 32], u[NT * 4 * 32];
};

template <int DK, int NP, int MODE> struct ScanPlan {
    static constexpr int RG = kRowGroups<NP>;
    static constexpr bool SIDE = MODE == MODE_OUT;
    static constexpr size_t chain = sizeof(ScanStage<DK, NP>), side = SIDE ? sizeof(ScanSide<DK, NP>) : 0;
    static constexpr size_t swap = SIDE ? sizeof(ScanSwap<DK, NP>) * RG : 0;
    static constexpr Stages n = fit_stages(chain, side, swap);
    static constexpr size_t smem = chain * n.chain + side * n.side + swap * n.swap;
    static constexpr int fetch = SIDE ? RG : NP == 1 ? 1 : 4, threads = 32 * (RG + fetch);       // chain warps, then side or fetching warps
    static_assert(smem <= 227 * 1024, "fits an SM");
};

template <int DK, int NP, int MODE>
__device__ __forceinline__ void scan_load(const ChunkParams &P, ScanStage<DK, NP> &st, int bh, int c, int v0, int vcols)
{
    constexpr int NT = NP == 1 ? 2 : 3, TH = 32 * ScanPlan<DK, NP, MODE>::fetch, VW = 16 * kRowGroups<NP>;
    const long long t0 = (long long)c * kC, nc = (long long)bh * P.chunks + c;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
#pragma unroll
    for (int i = 0; i < NP; i++) {
        load_tile<kC, DK, TH>(st.k[i], P.k.at + i * P.k.plane + q_base(P, P.k, bh, t0), P.k.stride_t, rows, P.Dk);
        if (vcols > 0) load_tile<kC, VW, TH>(st.v[i], P.v.at + i * P.v.plane + v_base(P, P.v, bh, t0) + v0, P.v.stride_t, rows, vcols);
    }
#pragma unroll
    for (int i = 0; i < NT; i++) load_triangle<TH>(st.tri[i], P.tri + (nc * NT + i) * kTri);
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
    for (int i = 0; i < NP; i++) load_tile<kC, DK, TH>(st.q[i], P.q.at + i * P.q.plane + q_base(P, P.q, bh, t0), P.q.stride_t, rows, P.Dk);
#pragma unroll
    for (int i = 0; i < NT; i++) load_triangle<TH>(st.p[i], P.p + (nc * NT + i) * kTri);
    for (int i = threadIdx.x % TH; i < kCoef * kC / 4; i += TH) cp16(smem_addr(&st.coef[0][0]) + i * 16, P.coef + nc * (kCoef * kC) + i * 4, true);
    cp_commit();
}

template <int DK, int NP, int MODE, class T>
__global__ void __launch_bounds__((ScanPlan<DK, NP, MODE>::threads), 1) delta_scan_kernel(const ChunkParams P)
{
    follow_previous();
    using Plan = ScanPlan<DK, NP, MODE>;
    using Side = ScanSide<DK, NP>;
    using Swap = ScanSwap<DK, NP>;
    constexpr int ld = DK + kPad, NT = NP == 1 ? 2 : 3, RG = Plan::RG, VW = 16 * RG, VLD = VW + kPad, CS = Plan::n.chain, SS = Plan::n.side, WS = Plan::n.swap;
    constexpr int PAIR = Plan::threads, ONE = 32 * RG;
    extern __shared__ __align__(16) unsigned char raw[];
    auto *stages = reinterpret_cast<ScanStage<DK, NP> *>(raw);
    const int bh = blockIdx.x, seg = blockIdx.z;
    const int vblks = (P.Dv + VW - 1) / VW;
    const bool ident = MODE == MODE_SUMMARY && (int)blockIdx.y >= vblks;        // rows of the identity instead of values
    const int r0 = ((int)blockIdx.y - (ident ? vblks : 0)) * VW;                // first value (or identity) row of the block
    const int vcols = ident ? 0 : (P.Dv - r0 < VW ? P.Dv - r0 : VW);
    const int c0 = seg * P.seg_chunks, c1 = c0 + P.seg_chunks < P.chunks ? c0 + P.seg_chunks : P.chunks;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, w = warp % RG, gr = lane / 4, tc = lane % 4 * 2;

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
            // Y = scale e^G S Q^T + u P^T
            float Y[8][4] = {};
#pragma unroll
            for (int d = 0; d < DK / 16; d++) {
                unsigned a[NT][4], b[4][NP][4];
                get_left(a, sw.s, d);
#pragma unroll
                for (int i = 0; i < 4; i++) load_right<NP, false>(b[i], at_nk(qs, ld, 16 * i, 16 * d), kC * ld);
                multiply<NT, NP, 4>(Y, a, b);
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
            triangle<NT, NT, false, false>(Y, [&](unsigned (&a)[NT][4], int tb) { get_left(a, sw.u, tb); },
                                           [&](int tb, int nb) { return triangle_nk(ps, nb, tb); });
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
    // Two terms of the state are enough for what is read from it; its update takes three.
    const int row = r0 + 16 * w + gr;                       // state rows row, row + 8; columns 8 n + tc, +1 of tile n
    float S[DK / 8][4];
    if (ident) {
#pragma unroll
        for (int n = 0; n < DK / 8; n++)
#pragma unroll
            for (int e = 0; e < 4; e++) S[n][e] = row + e / 2 * 8 == 8 * n + tc + e % 2 ? 1.f : 0.f;
    } else {
        const float *from = MODE == MODE_SUMMARY ? nullptr
                            : P.segs > 1 ? P.seg_start + ((long long)bh * P.segs + seg) * P.Dv * P.Dk
                                         : (P.state_in != nullptr ? P.state_in + (long long)bh * P.Dv * P.Dk : nullptr);
        load_state<DK>(S, from, row, P.Dv, P.Dk);
    }

    for (int c = c0; c < c1; c++) {
        const int s = (c - c0) % CS, par = (c - c0) % WS;
        auto &st = stages[s];
        Swap &sw = reinterpret_cast<Swap *>(raw + Plan::chain * CS + Plan::side * SS)[par * RG + w];
        const unsigned ks = smem_addr(st.k[0]), ts = smem_addr(st.tri[0]);

        if (Plan::SIDE && c - c0 >= WS) bar_sync(BAR_FREE + par, PAIR);
        bar_sync(BAR_FULL + s, PAIR);
        // X = S K^T
        float X[8][4] = {};
#pragma unroll
        for (int d = 0; d < DK / 16; d++) {
            unsigned a[NT][4], b[4][NP][4];
#pragma unroll
            for (int i = 0; i < 4; i++) load_right<NP, false>(b[i], at_nk(ks, ld, 16 * i, 16 * d), kC * ld);
            as_left(S[2 * d], S[2 * d + 1], a);
            if constexpr (MODE == MODE_OUT) put_left(sw.s, d, a);
            multiply<NT, NP, 4>(X, a, b);
        }
        // R (in X), r = R + R (T - I)^T: tokens t of the result from block t' on
        residual<NP>(X, st.coef, smem_addr(st.v[0]), VLD, 16 * w, vcols > 0);
        float r[8][4];
#pragma unroll
        for (int n = 0; n < 8; n++)
#pragma unroll
            for (int i = 0; i < 4; i++) r[n][i] = X[n][i];
        triangle<NT, NT, true, false>(r, [&](unsigned (&a)[NT][4], int tb) { as_left(X[2 * tb], X[2 * tb + 1], a); },
                                      [&](int tb, int nb) { return triangle_kn(ts, nb, tb); });
        // u = beta r, handed over
        scale_tokens(r, st.coef, COEF_BETA);
        if constexpr (MODE == MODE_OUT) {
#pragma unroll
            for (int tb = 0; tb < 4; tb++) {
                unsigned a[NT][4];
                as_left(r[2 * tb], r[2 * tb + 1], a);
                put_left(sw.u, tb, a);
            }
        }
        if (Plan::SIDE) bar_arrive(BAR_READY + par, PAIR);
        // S <- e^{G_C} S + (e^{G_C - G} u) K.  The update is summed from zero and added once: the tensor
        // core's running sum drops low bits at every step, always towards zero, which on a state that lives
        // for many chunks would add up.
        const float eC = st.coef[COEF_EG][kC - 1];
        scale_tokens(r, st.coef, COEF_LEFT);
        unsigned a[4][3][4];
#pragma unroll
        for (int tb = 0; tb < 4; tb++) as_left(r[2 * tb], r[2 * tb + 1], a[tb]);
#pragma unroll
        for (int nb = 0; nb < DK / 16; nb += 2) {
            float x[4][4] = {};
            columns_times<NP, DK>(x, a, ks, nb);
#pragma unroll
            for (int m = 0; m < 4; m++)
#pragma unroll
                for (int h = 0; h < 2; h++) fma_row(S[2 * nb + m], h, pair(eC, eC), pair(x[m][2 * h], x[m][2 * h + 1]));
        }
        if (c + CS < c1) bar_arrive(BAR_EMPTY + s, PAIR);
    }

    if (MODE == MODE_SUMMARY) {
        if (ident) store_state<DK>(P.seg_map + ((long long)bh * P.segs + seg) * P.Dk * P.Dk, S, row, P.Dk, P.Dk);
        else store_state<DK>(P.seg_end + ((long long)bh * P.segs + seg) * P.Dv * P.Dk, S, row, P.Dv, P.Dk);
    } else if (P.state_out != nullptr && seg == P.segs - 1) {
        store_state<DK>(P.state_out + (long long)bh * P.Dv * P.Dk, S, row, P.Dv, P.Dk);
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
    return launch<true>(kernel, dim3((unsigned)(P.B * P.Hv), blocks, P.segs), dim3(Plan::threads), Plan::smem, st, P);
}

// Start states of the segments from their end states and transitions, one segment after the other.  A block has 16
// rows of one head's state, a thread four rows of one column; the next two transitions are on their way to shared memory
// while one is multiplied (in registers on the way, and one ahead: 22 us for 12 heads x 12 segments, now 18).  Float
// arithmetic: a few products per segment, once, are not worth the tensor cores.  Adjoints (second grid layer): last
// segment first, with the transposed transitions.
constexpr int kMaps = 3;
template <int DK> constexpr int kMapLd = DK + 4;         // rows of whole 16-byte words that eight lanes read without conflicts

template <int DK>
__global__ void __launch_bounds__(4 * DK) delta_join_kernel(const ChunkParams P)
{
    follow_previous();
    extern __shared__ __align__(16) float maps[];           // [kMaps][DK][kMapLd], row k: what state column k sends on
    __shared__ __align__(16) float S[2][16][DK];
    constexpr int LD = kMapLd<DK>, WORDS = DK / 4;
    const bool adjoint = blockIdx.z == 1;
    const float *first = adjoint ? P.adj_in : P.state_in, *ends = adjoint ? P.adj_end : P.seg_end;
    float *starts = adjoint ? P.adj_start : P.seg_start;
    const int col = threadIdx.x % DK, part = threadIdx.x / DK, bh = blockIdx.x, r0 = blockIdx.y * 16 + 4 * part;
    const long long rows = (long long)P.Dv * P.Dk;
    const bool in = col < P.Dk;
    float s[4], end[4];
    auto place = [&](int n) { return (long long)bh * P.segs + (adjoint ? P.segs - 1 - n : n); };
    auto fetch_map = [&](int n) {
        if (n + 1 < P.segs) {
            const float *from = P.seg_map + place(n) * P.Dk * P.Dk;
            const unsigned to = smem_addr(maps + n % kMaps * (DK * LD));
#pragma unroll
            for (int i = threadIdx.x; i < DK * WORDS; i += 4 * DK) {
                const int k = i / WORDS, c = i % WORDS * 4;
                const bool ok = k < P.Dk && c < P.Dk;
                cp16(to + (k * LD + c) * 4, ok ? from + (long long)k * P.Dk + c : from, ok);
            }
        }
        cp_commit();                    // possibly empty, which keeps the count
    };
    auto fetch_end = [&](int n) {
#pragma unroll
        for (int i = 0; i < 4; i++) end[i] = in && r0 + i < P.Dv ? ends[place(n) * rows + (long long)(r0 + i) * P.Dk + col] : 0.f;
    };
    fetch_map(0);
    fetch_map(1);
#pragma unroll
    for (int i = 0; i < 4; i++) s[i] = in && r0 + i < P.Dv && first != nullptr ? first[bh * rows + (long long)(r0 + i) * P.Dk + col] : 0.f;
    fetch_end(0);
    for (int n = 0; n < P.segs; n++) {
        float(&now)[16][DK] = S[n % 2];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (in && r0 + i < P.Dv) starts[place(n) * rows + (long long)(r0 + i) * P.Dk + col] = s[i];
            now[4 * part + i][col] = s[i];
            s[i] = end[i];
        }
        if (n + 1 == P.segs) break;
        cp_wait<1>();
        __syncthreads();                // this transition and the rows are here, everyone is done with the one before
        fetch_map(n + 2);
        fetch_end(n + 1);
        const float *map = maps + n % kMaps * (DK * LD);
#pragma unroll 4
        for (int k = 0; k < DK; k += 4) {
            float4 m;
            if (adjoint) m = *reinterpret_cast<const float4 *>(&map[col * LD + k]);
            else m = make_float4(map[k * LD + col], map[(k + 1) * LD + col], map[(k + 2) * LD + col], map[(k + 3) * LD + col]);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float4 x = *reinterpret_cast<const float4 *>(&now[4 * part + i][k]);
                s[i] = fmaf(x.x, m.x, fmaf(x.y, m.y, fmaf(x.z, m.z, fmaf(x.w, m.w, s[i]))));
            }
        }
    }
}

template <int DK> cudaError_t join(const ChunkParams &P, bool adjoint, cudaStream_t st)
{
    const size_t smem = kMaps * DK * kMapLd<DK> * sizeof(float);
    const cudaError_t e = cudaFuncSetAttribute(delta_join_kernel<DK>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch(delta_join_kernel<DK>, dim3((unsigned)(P.B * P.Hv), (P.Dv + 15) / 16, adjoint ? 2 : 1), dim3(4 * DK), smem, st, P);
}

template <int DK, int NP> cudaError_t run(const ChunkParams &P, cudaStream_t st)
{
    if (P.segs > 1) {
        cudaError_t e = scan<DK, NP, MODE_SUMMARY>(P, st);
        if (e == cudaSuccess) e = join<DK>(P, false, st);
        if (e != cudaSuccess) return e;
    }
    return scan<DK, NP, MODE_OUT>(P, st);
}

}  // namespace

cudaError_t launch_delta_join(const ChunkParams &P, int dk, bool adjoint, cudaStream_t st)
{
    return dk == 64 ? join<64>(P, adjoint, st) : join<128>(P, adjoint, st);
}

cudaError_t launch_delta_scan(const ChunkParams &P, int dk, int terms, cudaStream_t st)
{
    if (dk == 64) return terms == 1 ? run<64, 1>(P, st) : run<64, 3>(P, st);
    return terms == 1 ? run<128, 1>(P, st) : run<128, 3>(P, st);
}

}  // namespace cawn
