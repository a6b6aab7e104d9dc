// Gated delta rule, chunk form: the walk over a head's chunks.
//
// Per chunk and warp (16 value rows, transposed products; see cawn_delta_chunk.cuh):
//   X = S K^T,  R = V^T - e^G X,  r = R T^T,  u = beta r,  O = scale e^G S Q^T + u P^T,
//   S <- e^{G_C} S + (e^{G_C - G} u) K
// Bound: the chain of these products, chunk after chunk, and the instructions between them (with one
// warp per scheduler, every one costs).  So the four warps that compute do nothing else: a fifth fetches the
// next chunk's tiles with cp.async while the current one is computed, and hands them over with a barrier;
// arithmetic between the products runs on pairs of floats.
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

template <int DK, int NP, int MODE> struct ScanStage {
    static constexpr int NT = NP == 1 ? 2 : 3;
    bf16 k[NP][kC * (DK + kPad)];
    bf16 q[MODE == MODE_SUMMARY ? 0 : NP][kC * (DK + kPad)];
    bf16 tri[NT][kC * kLd];
    bf16 p[MODE == MODE_OUT ? NP : MODE == MODE_SAVE ? NT : 0][kC * kLd];
    bf16 v[NP][kC * kLd];
    bf16 go[MODE == MODE_SAVE ? NP : 0][kC * kLd];
    float coef[kCoef][kC];
};
// two where they fit, so that the next chunk's tiles arrive during the current one
template <int DK, int NP, int MODE> constexpr int kScanStages = sizeof(ScanStage<DK, NP, MODE>) * 2 <= 227 * 1024 ? 2 : 1;
template <int DK, int NP, int MODE> constexpr int kScanBlocks = DK == 64 && NP == 1 && MODE != MODE_SAVE ? 2 : 1;   // per SM

template <int DK, int NP, int MODE>
__device__ __forceinline__ void scan_load(const ChunkParams &P, ScanStage<DK, NP, MODE> &st, int bh, int c, int vb, int vcols)
{
    constexpr int NT = NP == 1 ? 2 : 3;
    const long long t0 = (long long)c * kC, nc = (long long)bh * P.chunks + c;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC, lane = threadIdx.x % 32;
#pragma unroll
    for (int i = 0; i < NP; i++) {
        load_tile<kC, DK, 32>(st.k[i], P.k.at + i * P.k.plane + q_base(P, P.k, bh, t0), P.k.stride_t, rows, P.Dk);
        if (vcols > 0) load_tile<kC, kC, 32>(st.v[i], P.v.at + i * P.v.plane + v_base(P, P.v, bh, t0) + vb * kC, P.v.stride_t, rows, vcols);
        if constexpr (MODE != MODE_SUMMARY)
            load_tile<kC, DK, 32>(st.q[i], P.q.at + i * P.q.plane + q_base(P, P.q, bh, t0), P.q.stride_t, rows, P.Dk);
        if constexpr (MODE == MODE_SAVE)
            load_tile<kC, kC, 32>(st.go[i], P.go.at + i * P.go.plane + v_base(P, P.go, bh, t0) + vb * kC, P.go.stride_t, rows, vcols);
        if constexpr (MODE == MODE_OUT) load_dense<32>(st.p[i], P.p + (nc * NT + i) * kTile);
    }
#pragma unroll
    for (int i = 0; i < NT; i++) {
        load_dense<32>(st.tri[i], P.tri + (nc * NT + i) * kTile);
        if constexpr (MODE == MODE_SAVE) load_dense<32>(st.p[i], P.p + (nc * NT + i) * kTile);
    }
#pragma unroll
    for (int i = 0; i < 3; i++)
        if (i * 32 + lane < kCoef * kC / 4) cp16(smem_addr(&st.coef[0][0]) + (i * 32 + lane) * 16, P.coef + nc * (kCoef * kC) + (i * 32 + lane) * 4, true);
    cp_commit();
}

template <int DK, int NP, int MODE, class T>
__global__ void __launch_bounds__(kWalkThreads, (kScanBlocks<DK, NP, MODE>)) delta_scan_kernel(const ChunkParams P)
{
    constexpr int STAGES = kScanStages<DK, NP, MODE>, ld = DK + kPad, NT = NP == 1 ? 2 : 3;
    // Terms of the walk's own factors: three for the state and its update, three for R and in the output's
    // sum where the backward's dots need them, else NT and the terms of the output's type.
    constexpr int NR = MODE == MODE_SAVE ? 3 : NT, NO = MODE == MODE_SAVE ? 3 : NP, NB = MODE == MODE_SAVE ? NT : NP;
    extern __shared__ __align__(16) unsigned char raw[];
    auto *stages = reinterpret_cast<ScanStage<DK, NP, MODE> *>(raw);
    const int bh = blockIdx.x, vb = blockIdx.y, seg = blockIdx.z;
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32, gr = lane / 4, tc = lane % 4 * 2;
    const bool ident = MODE == MODE_SUMMARY && vb >= P.vblocks;     // rows of the identity instead of values
    const int r0 = (ident ? vb - P.vblocks : vb) * kC;              // first value (or identity) row of the block
    const int vcols = ident ? 0 : (P.Dv - r0 < kC ? P.Dv - r0 : kC);
    const int c0 = seg * P.seg_chunks, c1 = c0 + P.seg_chunks < P.chunks ? c0 + P.seg_chunks : P.chunks;

    if (w == 4) {               // producer: barrier 1 + s: stage s is full, 3 + s: stage s is free again
        for (int c = c0; c < c1; c++) {
            const int s = (c - c0) % STAGES;
            if (c - c0 >= STAGES) bar_sync(3 + s);
            scan_load<DK, NP, MODE>(P, stages[s], bh, c, vb, vcols);
            cp_wait<0>();
            bar_arrive(1 + s);
        }
        return;
    }

    const int rlim = ident ? P.Dk : P.Dv;                           // rows that exist
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
        const int s = (c - c0) % STAGES;
        auto &st = stages[s];
        const long long t0 = (long long)c * kC, nv = ((long long)bh * P.chunks + c) * P.vblocks + vb;
        const unsigned ks = smem_addr(st.k[0]), ts = smem_addr(st.tri[0]), vs = smem_addr(st.v[0]);

        if constexpr (MODE == MODE_SAVE) {
            bf16 *dst = P.s0 + nv * (NP * kC * DK) + (16 * w + gr) * DK + tc;
            float4 *df = P.sf + (nv * 4 + w) * (DK / 8 * 32) + lane;
#pragma unroll
            for (int n = 0; n < DK / 8; n++) {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    unsigned x[NP];
                    split(S[n][2 * h], S[n][2 * h + 1], x);
#pragma unroll
                    for (int i = 0; i < NP; i++) *reinterpret_cast<unsigned *>(dst + i * (kC * DK) + 8 * h * DK + 8 * n) = x[i];
                }
                df[n * 32] = make_float4(S[n][0], S[n][1], S[n][2], S[n][3]);
            }
        }
        bar_sync(1 + s);
        // X = S K^T, Y = S Q^T
        float X[8][4] = {}, Y[MODE == MODE_SUMMARY ? 1 : 8][4] = {};
#pragma unroll
        for (int d = 0; d < DK / 16; d++) {
            unsigned a[3][4];
            as_left(S[2 * d], S[2 * d + 1], a);
#pragma unroll
            for (int nb = 0; nb < 4; nb++) {
                product<3, NP, false>(X[2 * nb], X[2 * nb + 1], a, at_nk(ks, ld, 16 * nb, 16 * d), kC * ld);
                if constexpr (MODE != MODE_SUMMARY)     // bfloat16 results: one term of the state is enough
                    product<NO, NP, false>(Y[2 * nb], Y[2 * nb + 1], leading<NO>(a), at_nk(smem_addr(st.q[0]), ld, 16 * nb, 16 * d), kC * ld);
            }
        }
        // R = V^T - e^G X (into X and as the start of r); the read-out's first part gets its factor
        float r[8][4];
#pragma unroll
        for (int nb = 0; nb < 4; nb++) {
            unsigned vf[NP][4] = {};
            if (vcols > 0) load_left<NP, true>(vf, at_nk(vs, kLd, 16 * nb, 16 * w), kC * kLd);
#pragma unroll
            for (int m = 0; m < 2; m++) {
                const int n = 2 * nb + m;
                const float2 e = *reinterpret_cast<const float2 *>(&st.coef[COEF_EG][8 * n + tc]);
                const f32x2 minus = pair(-e.x, -e.y);
#pragma unroll
                for (int h = 0; h < 2; h++) fma_row(X[n], h, minus, pair(sum_terms(vf, 2 * m + h)));
                if constexpr (MODE != MODE_SUMMARY) {
                    const f32x2 f = pair(P.scale * e.x, P.scale * e.y);
                    scale_row(Y[n], 0, f);
                    scale_row(Y[n], 1, f);
                }
#pragma unroll
                for (int i = 0; i < 4; i++) r[n][i] = X[n][i];
            }
        }
        // r = R + R (T - I)^T: tokens t of the result from block t' on
#pragma unroll
        for (int tb = 0; tb < 4; tb++) {
            unsigned a[NR][4];
            as_left(X[2 * tb], X[2 * tb + 1], a);
#pragma unroll
            for (int nb = tb; nb < 4; nb++)
                product<NR, NT, true>(r[2 * nb], r[2 * nb + 1], a, at_kn(ts, kLd, 16 * tb, 16 * nb), kC * kLd);
        }
        if constexpr (MODE == MODE_SAVE) {
            float4 *df = P.rf + (nv * 4 + w) * (8 * 32) + lane;
#pragma unroll
            for (int n = 0; n < 8; n++) df[n * 32] = make_float4(r[n][0], r[n][1], r[n][2], r[n][3]);
        }
        // u = beta r
#pragma unroll
        for (int n = 0; n < 8; n++) {
            const f32x2 bt = pair(*reinterpret_cast<const float2 *>(&st.coef[COEF_BETA][8 * n + tc]));
            scale_row(r[n], 0, bt);
            scale_row(r[n], 1, bt);
        }
        if constexpr (MODE != MODE_SUMMARY) {
            const unsigned ps = smem_addr(st.p[0]);
#pragma unroll
            for (int tb = 0; tb < 4; tb++) {
                unsigned a[NO][4];
                as_left(r[2 * tb], r[2 * tb + 1], a);
#pragma unroll
                for (int nb = tb; nb < 4; nb++)
                    product<NO, NB, false>(Y[2 * nb], Y[2 * nb + 1], a, at_nk(ps, kLd, 16 * nb, 16 * tb), kC * kLd);
            }
        }
        if constexpr (MODE == MODE_SAVE) {
            // dO.o over this warp's 16 values
            float dots[8][2];
#pragma unroll
            for (int nb = 0; nb < 4; nb++) {
                unsigned g[NP][4];
                load_left<NP, true>(g, at_nk(smem_addr(st.go[0]), kLd, 16 * nb, 16 * w), kC * kLd);
#pragma unroll
                for (int m = 0; m < 2; m++) {
                    const int n = 2 * nb + m;
                    const float2 a = sum_terms(g, 2 * m), b = sum_terms(g, 2 * m + 1);
                    dots[n][0] = fmaf(Y[n][0], a.x, Y[n][2] * b.x);
                    dots[n][1] = fmaf(Y[n][1], a.y, Y[n][3] * b.y);
                }
            }
            column_sums(dots);
            *reinterpret_cast<float2 *>(P.od + (nv * 4 + w) * kC + 8 * gr + tc) = make_float2(dots[0][0], dots[0][1]);
            // u as token rows, through this warp's own columns of the V tile
            bf16 *dst = P.u + nv * (NP * kTile);
#pragma unroll
            for (int term = 0; term < NP; term++) {
                __syncwarp();
#pragma unroll
                for (int nb = 0; nb < 4; nb++) {
                    unsigned x[NP][4];
                    as_left(r[2 * nb], r[2 * nb + 1], x);
                    stsm_t(at_nk(vs, kLd, 16 * nb, 16 * w), x[term][0], x[term][1], x[term][2], x[term][3]);
                }
                __syncwarp();
#pragma unroll
                for (int i = lane; i < 128; i += 32)
                    *reinterpret_cast<uint4 *>(dst + term * kTile + i / 2 * kC + 16 * w + i % 2 * 8) =
                        *reinterpret_cast<const uint4 *>(&st.v[0][i / 2 * kLd + 16 * w + i % 2 * 8]);
            }
        }
        if constexpr (MODE == MODE_OUT) {
            T *o = static_cast<T *>(P.o) + (bh / P.Hv) * P.o_stride_b + t0 * P.o_stride_t + (long long)(bh % P.Hv) * P.Dv + r0;
            const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
            if constexpr (sizeof(T) == 2) {
                __syncwarp();
#pragma unroll
                for (int nb = 0; nb < 4; nb++)
                    stsm_t(at_nk(vs, kLd, 16 * nb, 16 * w), pack_bf16(Y[2 * nb][0], Y[2 * nb][1]), pack_bf16(Y[2 * nb][2], Y[2 * nb][3]),
                           pack_bf16(Y[2 * nb + 1][0], Y[2 * nb + 1][1]), pack_bf16(Y[2 * nb + 1][2], Y[2 * nb + 1][3]));
                __syncwarp();
#pragma unroll
                for (int i = lane; i < 128; i += 32) {
                    const int t = i / 2, v = 16 * w + i % 2 * 8;
                    if (t < rows && v < vcols)
                        *reinterpret_cast<uint4 *>(o + t * P.o_stride_t + v) = *reinterpret_cast<const uint4 *>(&st.v[0][t * kLd + v]);
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
        for (int nb = 0; nb < DK / 16; nb++) {
            float x[2][4] = {};
#pragma unroll
            for (int tb = 0; tb < 4; tb++) product<3, NP, true>(x[0], x[1], a[tb], at_kn(ks, ld, 16 * tb, 16 * nb), kC * ld);
#pragma unroll
            for (int m = 0; m < 2; m++)
#pragma unroll
                for (int h = 0; h < 2; h++) fma_row(S[2 * nb + m], h, pair(eC, eC), pair(x[m][2 * h], x[m][2 * h + 1]));
        }
        if (c + STAGES < c1) bar_arrive(3 + s);
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
        float4 *df = P.sf + ((((long long)P.B * P.Hv * P.chunks + bh) * P.vblocks + vb) * 4 + w) * (DK / 8 * 32) + lane;
        if (seg == P.segs - 1)
#pragma unroll
            for (int n = 0; n < DK / 8; n++) df[n * 32] = make_float4(S[n][0], S[n][1], S[n][2], S[n][3]);
    }
}

template <int DK, int NP, int MODE> cudaError_t scan(const ChunkParams &P, int row_blocks, cudaStream_t st)
{
    using T = typename std::conditional<NP == 1, bf16, float>::type;
    const size_t smem = sizeof(ScanStage<DK, NP, MODE>) * kScanStages<DK, NP, MODE>;
    static_assert(sizeof(ScanStage<DK, NP, MODE>) <= 227 * 1024, "fits an SM");
    auto *kernel = delta_scan_kernel<DK, NP, MODE, T>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch(kernel, dim3((unsigned)(P.B * P.Hv), row_blocks, P.segs), dim3(kWalkThreads), smem, st, P);
}

// Start states of the segments from their end states and transitions, one segment after the other.  A block has 16
// rows of one head's state, a thread eight rows of one column; the next transition is on its way (in registers)
// while the current one is multiplied from shared memory.  Float arithmetic: a few products per segment, once, are
// not worth the tensor cores.  REVERSE: adjoints, last segment first, with the transposed transitions.
template <int DK, bool REVERSE>
__global__ void __launch_bounds__(2 * DK) delta_join_kernel(const ChunkParams P)
{
    extern __shared__ __align__(16) float map[];            // [DK][DK + 1], row k: what state column k sends on
    __shared__ __align__(16) float S[16][DK];
    constexpr int EACH = DK / 2, LD = DK + 1;               // transition elements per thread
    const int col = threadIdx.x % DK, half = threadIdx.x / DK, bh = blockIdx.x, r0 = blockIdx.y * 16 + 8 * half;
    const long long rows = (long long)P.Dv * P.Dk;
    const bool in = col < P.Dk;
    float s[8], end[8], m[EACH];
    auto fetch = [&](int n) {
        const long long seg = (long long)bh * P.segs + (REVERSE ? P.segs - 1 - n : n);
        const float *from = P.seg_map + seg * P.Dk * P.Dk;
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            const int k = 2 * i + half;
            m[i] = in && k < P.Dk ? from[(long long)k * P.Dk + col] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) end[i] = in && r0 + i < P.Dv ? P.seg_end[seg * rows + (long long)(r0 + i) * P.Dk + col] : 0.f;
    };
#pragma unroll
    for (int i = 0; i < 8; i++) s[i] = in && r0 + i < P.Dv && P.state_in != nullptr ? P.state_in[bh * rows + (long long)(r0 + i) * P.Dk + col] : 0.f;
    fetch(0);
    for (int n = 0; n < P.segs; n++) {
        const long long seg = (long long)bh * P.segs + (REVERSE ? P.segs - 1 - n : n);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (in && r0 + i < P.Dv) P.seg_start[seg * rows + (long long)(r0 + i) * P.Dk + col] = s[i];
            S[8 * half + i][col] = s[i];
            s[i] = end[i];
        }
        if (n + 1 == P.segs) break;
#pragma unroll
        for (int i = 0; i < EACH; i++) map[REVERSE ? col * LD + 2 * i + half : (2 * i + half) * LD + col] = m[i];
        __syncthreads();
        fetch(n + 1);
#pragma unroll 4
        for (int k = 0; k < DK; k += 4) {
            const float a = map[k * LD + col], b = map[(k + 1) * LD + col], c = map[(k + 2) * LD + col], d = map[(k + 3) * LD + col];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float4 x = *reinterpret_cast<const float4 *>(&S[8 * half + i][k]);
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
    return launch(delta_join_kernel<DK, REVERSE>, dim3((unsigned)(P.B * P.Hv), (P.Dv + 15) / 16), dim3(2 * DK), smem, st, P);
}
template <int DK> cudaError_t join(const ChunkParams &P, bool reverse, cudaStream_t st) { return reverse ? join1<DK, true>(P, st) : join1<DK, false>(P, st); }

template <int DK, int NP> cudaError_t run(const ChunkParams &P, bool save, cudaStream_t st)
{
    if (P.segs > 1) {
        cudaError_t e = scan<DK, NP, MODE_SUMMARY>(P, P.vblocks + (P.Dk + kC - 1) / kC, st);
        if (e == cudaSuccess) e = join<DK>(P, false, st);
        if (e != cudaSuccess) return e;
    }
    return save ? scan<DK, NP, MODE_SAVE>(P, P.vblocks, st) : scan<DK, NP, MODE_OUT>(P, P.vblocks, st);
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
