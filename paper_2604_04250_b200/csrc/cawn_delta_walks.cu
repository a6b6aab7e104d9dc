// Gated delta rule, chunk form: the backward's two walks, side by side.
//
// The forward's walk again, for what the gradients need of it,
//   X = S K^T,  R = V^T - e^G X,  r = R T^T,  u = beta r,  S <- e^{G_C} S + (e^{G_C - G} u) K,
// and the reverse walk, with D the adjoint of the state after a chunk,
//   dU = P^T dO + e^{G_C - G} (K D^T),   rb = T^T (beta dU),   D <- e^{G_C} D + (scale e^G dO)^T Q - (e^G rb)^T K.
// Neither needs the other, and all sums over both are left to the chunk-local kernel.  They leave r, D K^T and both
// states as floats, and rb.  Bound: each walk is a chain of products and of the instructions between them, on the SMs that
// have a head.  One launch runs both, the reverse ones, which take longer, first: with few heads each walk has an SM of
// its own, with many the forward walks fill the SMs that the reverse ones leave or come free first (96 heads of 64 x 64,
// 2048 tokens, bfloat16: 151 us; with r and the states converted to bfloat16 terms here 177).
// A block is 16 * row groups of values of one head and one direction.  Warps of their own fetch the tiles (with the
// chain warps fetching, either walk of 96 heads took 153 us instead of 127), a chunk ahead where shared memory holds
// two sets; else the tiles that a chunk starts with come a chunk ahead and the others when it starts.
#include "cawn_delta_chunk.cuh"

#include <type_traits>

namespace cawn {
namespace {

template <int DK, int NP> struct WalkTiles {
    static constexpr int NT = NP == 1 ? 2 : 3, VLD = 16 * kRowGroups<NP> + kPad;
    using Keys = bf16[NP][kC * (DK + kPad)];
    using Values = bf16[NP][kC * VLD];
    using Triangle = bf16[NT][kTri];
    struct FwdEarly { Keys k; Values v; float coef[kCoef][kC]; };
    struct FwdLate { Triangle tri; };
    struct RevEarly { Keys k; Values go; Triangle p; float coef[kCoef][kC]; };
    struct RevLate { Keys q; Triangle tri; bf16 way[kC * VLD]; };       // way: on which rb leaves as token rows
};
template <int DK, int NP> struct WalkPlan {
    using Tiles = WalkTiles<DK, NP>;
    static constexpr int RG = kRowGroups<NP>, VW = 16 * RG;
    static constexpr int fetch = NP == 1 ? 32 : 128, threads = 32 * RG + fetch;
    static constexpr size_t need(int early, int late)
    {
        const size_t fwd = early * sizeof(typename Tiles::FwdEarly) + late * sizeof(typename Tiles::FwdLate);
        const size_t rev = early * sizeof(typename Tiles::RevEarly) + late * sizeof(typename Tiles::RevLate);
        return fwd > rev ? fwd : rev;
    }
    static constexpr size_t room = 227 * 1024;
    static constexpr int early = need(2, 1) <= room ? 2 : 1, late = need(2, 2) <= room ? 2 : 1;      // sets of each
    static constexpr size_t smem = need(early, late);
    static_assert(smem <= room, "fits an SM");
};

template <int DK, int NP> struct Fetch {
    using Plan = WalkPlan<DK, NP>;
    static constexpr int TH = Plan::fetch, NT = Plan::Tiles::NT, VW = Plan::VW;
    const ChunkParams &P;
    int bh, v0, vcols;
    __device__ __forceinline__ int rows(int c) const { return P.L - (long long)c * kC < kC ? (int)(P.L - (long long)c * kC) : kC; }
    __device__ __forceinline__ void keys(typename Plan::Tiles::Keys &to, const Terms &t, int c) const
    {
#pragma unroll
        for (int i = 0; i < NP; i++) load_tile<kC, DK, TH>(to[i], t.at + i * t.plane + q_base(P, t, bh, (long long)c * kC), t.stride_t, rows(c), P.Dk);
    }
    __device__ __forceinline__ void values(typename Plan::Tiles::Values &to, const Terms &t, int c) const
    {
#pragma unroll
        for (int i = 0; i < NP; i++) load_tile<kC, VW, TH>(to[i], t.at + i * t.plane + v_base(P, t, bh, (long long)c * kC) + v0, t.stride_t, rows(c), vcols);
    }
    __device__ __forceinline__ void triangle(typename Plan::Tiles::Triangle &to, const bf16 *from, int c) const
    {
#pragma unroll
        for (int i = 0; i < NT; i++) load_triangle<TH>(to[i], from + (((long long)bh * P.chunks + c) * NT + i) * kTri);
    }
    __device__ __forceinline__ void coef(float (&to)[kCoef][kC], int c) const
    {
        for (int i = threadIdx.x % TH; i < kCoef * kC / 4; i += TH)
            cp16(smem_addr(&to[0][0]) + i * 16, P.coef + ((long long)bh * P.chunks + c) * (kCoef * kC) + i * 4, true);
    }
};

// Two sets of everything: the fetching warps run ahead on their own, and the chain warps do not wait for one another.
// Returns true for the former, which are done.
template <class Plan, class Early, class Late> __device__ __forceinline__ bool fetch_ahead(bool walks, int count, Early load_early, Late load_late)
{
    if constexpr (Plan::late == 1) return false;
    if (walks) return false;
    for (int i = 0; i < count; i++) {
        if (i >= 2) bar_sync(BAR_EMPTY + i % 2, Plan::threads);
        load_early(i);
        load_late(i);
        cp_commit();
        cp_wait<0>();
        bar_arrive(BAR_FULL + i % 2, Plan::threads);
    }
    return true;
}
// A walk's chunk: wait for the early tiles; with one late set the fetching warps ask for what the buffers have room
// for.  `load_early(i)`, `load_late(i)`: tiles of the i-th chunk of the walk.
template <class Plan, class Early, class Late> __device__ __forceinline__ void begin_chunk(bool walks, int i, int count, Early load_early, Late load_late)
{
    if (Plan::late == 2) {
        bar_sync(BAR_FULL + i % 2, Plan::threads);
        return;
    }
    if (Plan::early == 1 && i > 0) __syncthreads();     // everyone is done with the one set there is
    if (!walks) {
        if (Plan::early == 1 || i == 0) {
            load_early(i);
            cp_commit();
        }
        cp_wait<0>();
    }
    __syncthreads();            // the tiles are here, and everyone is done with the chunk before
    if (walks) return;
    load_late(i);
    cp_commit();
    if (Plan::early == 2) {
        if (i + 1 < count) load_early(i + 1);
        cp_commit();            // possibly empty, which keeps the count
    }
}
template <class Plan> __device__ __forceinline__ void end_chunk(int i, int count)
{
    if (Plan::late == 2 && i + 2 < count) bar_arrive(BAR_EMPTY + i % 2, Plan::threads);
}
template <class Plan> __device__ __forceinline__ void late_tiles(bool walks)
{
    if (Plan::late == 2) return;                        // they came with the early ones
    if (!walks) {
        if (Plan::early == 2) cp_wait<1>(); else cp_wait<0>();
    }
    __syncthreads();
}

// A thread's accumulators as token rows of 16 values per warp, in N terms, through shared memory (`way`, this warp's own
// columns); `put(term, t, v, x)`: eight values of token t, from value v of the warp's on.
template <int N, class Put> __device__ __forceinline__ void token_rows(const float (&x)[8][4], bf16 *way, int ld, int col, Put put)
{
    const int lane = threadIdx.x % 32;
    const unsigned to = smem_addr(way);
#pragma unroll
    for (int term = 0; term < N; term++) {
        __syncwarp();
#pragma unroll
        for (int nb = 0; nb < 4; nb++) {
            unsigned w[N][4];
            as_left(x[2 * nb], x[2 * nb + 1], w);
            stsm_t(at_nk(to, ld, 16 * nb, col), w[term][0], w[term][1], w[term][2], w[term][3]);
        }
        __syncwarp();
#pragma unroll
        for (int j = lane; j < 128; j += 32) put(term, j / 2, j % 2 * 8, *reinterpret_cast<const uint4 *>(&way[j / 2 * ld + col + j % 2 * 8]));
    }
}

// SUMMARY: what a segment's own tokens leave at its end (forward; with the transitions, which are the walk of the
// identity's rows with V = 0) or send to its start (reverse).
template <int DK, int NP, bool SUMMARY>
__device__ __forceinline__ void forward_walk(const ChunkParams &P, unsigned char *raw, int bh, int block)
{
    using Plan = WalkPlan<DK, NP>;
    using Early = typename Plan::Tiles::FwdEarly;
    using Late = typename Plan::Tiles::FwdLate;
    constexpr int NT = Plan::Tiles::NT, VW = Plan::VW, VLD = Plan::Tiles::VLD;
    auto stage = [&](int i) -> Early & { return reinterpret_cast<Early *>(raw)[i % Plan::early]; };
    auto stage_late = [&](int i) -> Late & { return reinterpret_cast<Late *>(raw + Plan::early * sizeof(Early))[i % Plan::late]; };
    const int seg = blockIdx.z, vblks = (P.Dv + VW - 1) / VW;
    const bool ident = SUMMARY && block >= vblks;
    const int r0 = (block - (ident ? vblks : 0)) * VW, vcols = ident ? 0 : (P.Dv - r0 < VW ? P.Dv - r0 : VW);
    const int c0 = seg * P.seg_chunks, c1 = c0 + P.seg_chunks < P.chunks ? c0 + P.seg_chunks : P.chunks, count = c1 - c0;
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32, gr = lane / 4, tc = lane % 4 * 2, w4 = (r0 / 16 + w) % 4;
    const bool walks = w < Plan::RG;
    const int row = r0 + 16 * w + gr;
    const Fetch<DK, NP> fetch = {P, bh, r0, vcols};
    auto load_early = [&](int i) {
        Early &e = stage(i);
        fetch.keys(e.k, P.k, c0 + i);
        if (vcols > 0) fetch.values(e.v, P.v, c0 + i);
        fetch.coef(e.coef, c0 + i);
    };
    auto load_late = [&](int i) { fetch.triangle(stage_late(i).tri, P.tri, c0 + i); };
    float S[DK / 8][4];
    if (ident) {
#pragma unroll
        for (int n = 0; n < DK / 8; n++)
#pragma unroll
            for (int e = 0; e < 4; e++) S[n][e] = row + e / 2 * 8 == 8 * n + tc + e % 2 ? 1.f : 0.f;
    } else {
        const float *from = SUMMARY ? nullptr
                            : P.segs > 1 ? P.seg_start + ((long long)bh * P.segs + seg) * P.Dv * P.Dk
                                         : (P.state_in != nullptr ? P.state_in + (long long)bh * P.Dv * P.Dk : nullptr);
        load_state<DK>(S, from, walks ? row : P.Dv, P.Dv, P.Dk);
    }
    if (fetch_ahead<Plan>(walks, count, load_early, load_late)) return;
    for (int i = 0; i < count; i++) {
        begin_chunk<Plan>(walks, i, count, load_early, load_late);
        const long long nv = ((long long)bh * P.chunks + c0 + i) * P.vblocks + r0 / kC;
        Early &e = stage(i);
        Late &late = stage_late(i);
        const unsigned ks = smem_addr(e.k[0]);
        float X[8][4] = {};
        if (walks) {
            rows_times<3, NP, DK>(X, S, ks);
            if constexpr (!SUMMARY) store_rows(P.s0 + nv * (kC * DK) + 16 * w4 * DK, S);
            residual<NP>(X, e.coef, smem_addr(e.v[0]), VLD, 16 * w, vcols > 0);
        }
        late_tiles<Plan>(walks);
        if (!walks) continue;
        float r[8][4];
#pragma unroll
        for (int n = 0; n < 8; n++)
#pragma unroll
            for (int j = 0; j < 4; j++) r[n][j] = X[n][j];
        triangle<3, NT, true, false>(r, [&](unsigned (&a)[3][4], int tb) { as_left(X[2 * tb], X[2 * tb + 1], a); },
                                     [&](int tb, int nb) { return triangle_kn(smem_addr(late.tri[0]), nb, tb); });
        if constexpr (!SUMMARY) store_rows(P.r + nv * kTile + 16 * w4 * kC, r);
        scale_tokens(r, e.coef, COEF_BETA);
        // the update is summed from zero and added once, as in the forward
        const float eC = e.coef[COEF_EG][kC - 1];
        scale_tokens(r, e.coef, COEF_LEFT);
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
        end_chunk<Plan>(i, count);
    }
    if (!SUMMARY || !walks) return;
    if (ident) store_state<DK>(P.seg_map + ((long long)bh * P.segs + seg) * P.Dk * P.Dk, S, row, P.Dk, P.Dk);
    else store_state<DK>(P.seg_end + ((long long)bh * P.segs + seg) * P.Dv * P.Dk, S, row, P.Dv, P.Dk);
}

template <int DK, int NP, bool SUMMARY, class T>
__device__ __forceinline__ void reverse_walk(const ChunkParams &P, unsigned char *raw, int bh, int block)
{
    using Plan = WalkPlan<DK, NP>;
    using Early = typename Plan::Tiles::RevEarly;
    using Late = typename Plan::Tiles::RevLate;
    constexpr int NT = Plan::Tiles::NT, VW = Plan::VW, VLD = Plan::Tiles::VLD;
    auto stage = [&](int i) -> Early & { return reinterpret_cast<Early *>(raw)[i % Plan::early]; };
    auto stage_late = [&](int i) -> Late & { return reinterpret_cast<Late *>(raw + Plan::early * sizeof(Early))[i % Plan::late]; };
    const int seg = blockIdx.z, r0 = block * VW, vcols = P.Dv - r0 < VW ? P.Dv - r0 : VW;
    const int c0 = seg * P.seg_chunks, c1 = c0 + P.seg_chunks < P.chunks ? c0 + P.seg_chunks : P.chunks, count = c1 - c0;
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32, gr = lane / 4, tc = lane % 4 * 2, w4 = (r0 / 16 + w) % 4;
    const bool walks = w < Plan::RG;
    const int row = r0 + 16 * w + gr;
    const Fetch<DK, NP> fetch = {P, bh, r0, vcols};
    auto load_early = [&](int i) {
        Early &e = stage(i);
        fetch.keys(e.k, P.k, c1 - 1 - i);
        fetch.values(e.go, P.go, c1 - 1 - i);
        fetch.triangle(e.p, P.p, c1 - 1 - i);
        fetch.coef(e.coef, c1 - 1 - i);
    };
    auto load_late = [&](int i) {
        Late &late = stage_late(i);
        fetch.triangle(late.tri, P.tri, c1 - 1 - i);
        fetch.keys(late.q, P.q, c1 - 1 - i);
    };
    float D[DK / 8][4];
    const float *from = SUMMARY ? nullptr
                        : P.segs > 1 ? P.adj_start + ((long long)bh * P.segs + seg) * P.Dv * P.Dk
                                     : (P.adj_in != nullptr ? P.adj_in + (long long)bh * P.Dv * P.Dk : nullptr);
    load_state<DK>(D, from, walks ? row : P.Dv, P.Dv, P.Dk);

    if (fetch_ahead<Plan>(walks, count, load_early, load_late)) return;
    for (int i = 0; i < count; i++) {
        begin_chunk<Plan>(walks, i, count, load_early, load_late);
        const int c = c1 - 1 - i;
        const long long t0 = (long long)c * kC, nv = ((long long)bh * P.chunks + c) * P.vblocks + r0 / kC;
        Early &e = stage(i);
        Late &late = stage_late(i);
        const unsigned ks = smem_addr(e.k[0]), gs = smem_addr(e.go[0]);
        // X = beta (e^{G_C - G} (D K^T) + dO^T P)
        float X[8][4] = {};
        if (walks) {
            rows_times<3, NP, DK>(X, D, ks);
            if constexpr (!SUMMARY) {
                store_rows(P.ds + nv * (kC * DK) + 16 * w4 * DK, D);
                store_rows(P.dk + nv * kTile + 16 * w4 * kC, X);
            }
            scale_tokens(X, e.coef, COEF_LEFT);
            triangle<NP, NT, true, true>(X, [&](unsigned (&a)[NP][4], int ib) { load_left<NP, true>(a, at_nk(gs, VLD, 16 * ib, 16 * w), kC * VLD); },
                                         [&](int ib, int nb) { return triangle_kn(smem_addr(e.p[0]), ib, nb); });
            scale_tokens(X, e.coef, COEF_BETA);
        }
        late_tiles<Plan>(walks);
        if (!walks) continue;
        const unsigned qs = smem_addr(late.q[0]);
        // rb = X + (T - I)^T X
        float rb[8][4];
#pragma unroll
        for (int n = 0; n < 8; n++)
#pragma unroll
            for (int j = 0; j < 4; j++) rb[n][j] = X[n][j];
        triangle<3, NT, false, true>(rb, [&](unsigned (&a)[3][4], int ib) { as_left(X[2 * ib], X[2 * ib + 1], a); },
                                     [&](int ib, int nb) { return triangle_nk(smem_addr(late.tri[0]), ib, nb); });
        if constexpr (!SUMMARY) {
            // dV (bfloat16: its first term, the rounded value), and the terms that the chunk's gradients take
            const int rows = fetch.rows(c);
            const long long here = v_base(P, P.rb, bh, t0) + r0;
            token_rows<NT>(rb, late.way, VLD, 16 * w, [&](int term, int t, int v, uint4 x) {
                bf16 *to = (NP == 1 && term == 0 ? static_cast<bf16 *>(P.o) : P.rbt + (term - (NP == 1 ? 1 : 0)) * P.rb.plane) + here;
                if (t < rows && 16 * w + v < vcols) *reinterpret_cast<uint4 *>(to + t * P.rb.stride_t + 16 * w + v) = x;
            });
            if constexpr (sizeof(T) == 4) {
                T *gv = static_cast<T *>(P.o) + here;
#pragma unroll
                for (int n = 0; n < 8; n++)
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const int t = 8 * n + tc + (j & 1), v = 16 * w + gr + (j >> 1) * 8;
                        if (t < rows && v < vcols) gv[t * P.rb.stride_t + v] = narrow<T>(rb[n][j]);
                    }
            }
        }
        // D <- e^{G_C} D + (scale e^G dO)^T Q - (e^G rb)^T K, the update summed from zero
        const float eC = e.coef[COEF_EG][kC - 1];
        scale_tokens(rb, e.coef, COEF_EG, -1.f);
        unsigned a[4][3][4], f[4][3][4];
#pragma unroll
        for (int tb = 0; tb < 4; tb++) {
            unsigned x[NP][4];
            load_left<NP, true>(x, at_nk(gs, VLD, 16 * tb, 16 * w), kC * VLD);
            float y[2][4];
#pragma unroll
            for (int m = 0; m < 2; m++) {
                const float2 eg = *reinterpret_cast<const float2 *>(&e.coef[COEF_EG][16 * tb + 8 * m + tc]);
                const f32x2 plus = pair(P.scale * eg.x, P.scale * eg.y);
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const float2 z = halves(mul2(plus, pair(sum_terms(x, 2 * m + h))));
                    y[m][2 * h] = z.x;
                    y[m][2 * h + 1] = z.y;
                }
            }
            as_left(y[0], y[1], a[tb]);
            as_left(rb[2 * tb], rb[2 * tb + 1], f[tb]);
        }
#pragma unroll
        for (int nb = 0; nb < DK / 16; nb += 2) {
            float x[4][4] = {};
            columns_times<NP, DK>(x, a, qs, nb);
            columns_times<NP, DK>(x, f, ks, nb);
#pragma unroll
            for (int m = 0; m < 4; m++)
#pragma unroll
                for (int h = 0; h < 2; h++) fma_row(D[2 * nb + m], h, pair(eC, eC), pair(x[m][2 * h], x[m][2 * h + 1]));
        }
        end_chunk<Plan>(i, count);
    }
    if (!walks) return;
    float *to = SUMMARY ? P.adj_end + ((long long)bh * P.segs + seg) * P.Dv * P.Dk
                : P.adj_out != nullptr && seg == 0 ? P.adj_out + (long long)bh * P.Dv * P.Dk : nullptr;
    if (to != nullptr) store_state<DK>(to, D, row, P.Dv, P.Dk);
}

template <int DK, int NP, bool SUMMARY, class T>
__global__ void __launch_bounds__((WalkPlan<DK, NP>::threads), 1) delta_walks_kernel(const ChunkParams P)
{
    follow_previous();
    extern __shared__ __align__(16) unsigned char raw[];
    constexpr int VW = WalkPlan<DK, NP>::VW;
    const int heads = P.B * P.Hv, back = heads * ((P.Dv + VW - 1) / VW), at = (int)blockIdx.x - back;       // reverse walks come first
    if (at < 0) reverse_walk<DK, NP, SUMMARY, T>(P, raw, (int)blockIdx.x % heads, (int)blockIdx.x / heads);
    else forward_walk<DK, NP, SUMMARY>(P, raw, at % heads, at / heads);
}

template <int DK, int NP, bool SUMMARY> cudaError_t walks(const ChunkParams &P, cudaStream_t st)
{
    using T = typename std::conditional<NP == 1, bf16, float>::type;
    using Plan = WalkPlan<DK, NP>;
    auto *kernel = delta_walks_kernel<DK, NP, SUMMARY, T>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Plan::smem);
    if (e != cudaSuccess) return e;
    const int vblks = (P.Dv + Plan::VW - 1) / Plan::VW, ident = SUMMARY ? (P.Dk + Plan::VW - 1) / Plan::VW : 0;
    const unsigned blocks = (unsigned)(P.B * P.Hv) * (2 * vblks + ident);
    return launch(kernel, dim3(blocks, 1, P.segs), dim3(Plan::threads), Plan::smem, st, P);
}

}  // namespace

cudaError_t launch_delta_walks(const ChunkParams &P, int dk, int terms, bool summary, cudaStream_t st)
{
    if (dk == 64) return terms == 1 ? (summary ? walks<64, 1, true>(P, st) : walks<64, 1, false>(P, st))
                                    : (summary ? walks<64, 3, true>(P, st) : walks<64, 3, false>(P, st));
    return terms == 1 ? (summary ? walks<128, 1, true>(P, st) : walks<128, 1, false>(P, st))
                      : (summary ? walks<128, 3, true>(P, st) : walks<128, 3, false>(P, st));
}

}  // namespace cawn
