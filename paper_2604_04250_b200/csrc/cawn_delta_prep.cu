// Gated delta rule, chunk form: what a chunk needs that does not depend on the state.  All chunks of all
// heads at once: decays, the scores P, and the inverse T of the chunk's triangle.
//
// Bound: instructions and their latency (exponentials, splitting, substitution) and the shared memory pipe, so many
// small blocks per SM, which is why A reuses the tiles' shared memory: five, at 96 registers (3072 chunks of 64 keys:
// 35 us; with six, which spill, 39, with four 39).
// The inverse: 16 x 16 blocks on the diagonal by substitution in float (a lane per column), the blocks
// below from T_IJ = -T_II sum_K A_IK T_KJ on the tensor cores, a block column per warp with the
// intermediate blocks in registers.  Substitution is stable for every triangle whose inverse is moderate;
// a power series of A is not (equal keys give binomial coefficients).
#include "cawn_delta_chunk.cuh"

namespace cawn {
namespace {

template <int DK, int NP> struct PrepSmem {
    static constexpr int NT = NP == 1 ? 2 : 3;
    union {
        struct { bf16 q[NP][kC * (DK + kPad)], k[NP][kC * (DK + kPad)]; };
        bf16 a[NT][kC * kLd];           // A = At diag(beta), terms: takes the tiles' place once the scores are made
    };
    bf16 d[NT][4][16 * 24];             // inverses of the diagonal blocks, transposed, terms
    float diag[4][16][20];              // diagonal blocks of A
    float nhi[kC], nlo[kC], beta[kC];   // -G in two parts
};

// Each of the four warps owns the 8-row blocks w and 7 - w: below the diagonal that is nine 8 x 8 blocks for
// everyone.  (With 16 adjacent rows the last warp had four times the first one's exponentials.)
template <int DK, int NP>
__global__ void __launch_bounds__(128, (DK == 64 && NP == 1 ? 5 : 1)) delta_prep_kernel(const ChunkParams P)
{
    follow_previous();
    extern __shared__ __align__(16) unsigned char raw[];
    auto &sm = *reinterpret_cast<PrepSmem<DK, NP> *>(raw);
    constexpr int ld = DK + kPad, NT = NP == 1 ? 2 : 3;
    const long long nc = blockIdx.x;
    const int bh = (int)(nc / P.chunks), c = (int)(nc % P.chunks);
    const long long t0 = (long long)c * kC;
    const int rows = P.L - t0 < kC ? (int)(P.L - t0) : kC;
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32, gr = lane / 4, tc = lane % 4 * 2;

#pragma unroll
    for (int i = 0; i < NP; i++) {
        load_tile<kC, DK, 128>(sm.k[i], P.k.at + i * P.k.plane + q_base(P, P.k, bh, t0), P.k.stride_t, rows, P.Dk);
        load_tile<kC, DK, 128>(sm.q[i], P.q.at + i * P.q.plane + q_base(P, P.q, bh, t0), P.q.stride_t, rows, P.Dk);
    }
    cp_commit();

    if (w == 0) {
        // Running sum in double, in units of log 2: differences G_i - G_j of strong decays keep their
        // accuracy, and one instruction turns them into decays.  Below
        // -200 every decay is zero in float, and so is every product with one: the clamp changes no
        // result and keeps -infinity out of the differences.
        const long long at = ((long long)(bh / P.Hv) * P.L + t0) * P.Hv + bh % P.Hv;
        double sum[2];
        float bt[2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int t = lane * 2 + e;
            const float g = t < rows ? P.g[at + (long long)t * P.Hv] : 0.f;
            const float x = t < rows ? P.beta[at + (long long)t * P.Hv] : 1.f;
            // the backward divides by beta; 2^-100 in place of 0 changes nothing that float could show
            bt[e] = fabsf(x) < 0x1p-100f ? copysignf(0x1p-100f, x) : x;
            sum[e] = (g < -200.f ? -200.0 : (double)g) * 1.4426950408889634;
        }
        sum[1] += sum[0];
        double run = sum[1];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const double other = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += other;
        }
        const double before = run - sum[1];
        sum[0] += before;
        sum[1] += before;
        const double last = __shfl_sync(0xffffffffu, sum[1], 31);
        float *coef = P.coef + nc * (kCoef * kC);
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int t = lane * 2 + e;
            const float hi = (float)sum[e], lo = (float)(sum[e] - (double)hi);
            sm.nhi[t] = -hi; sm.nlo[t] = -lo; sm.beta[t] = bt[e];
            coef[COEF_EG * kC + t] = exp2_fast(hi) * fmaf(lo, 0.69314718f, 1.f);
            coef[COEF_LEFT * kC + t] = exp2_fast((float)(last - sum[e]));
            coef[COEF_BETA * kC + t] = bt[e];
            coef[COEF_GHI * kC + t] = hi;
            coef[COEF_GLO * kC + t] = lo;
        }
    }
    cp_wait<0>();
    __syncthreads();

    // rows 8 w + gr and 8 (7 - w) + gr against column blocks 0 .. 7 - w
    float kk[8][4] = {}, qk[8][4] = {};
    const unsigned ks = smem_addr(sm.k[0]), qs = smem_addr(sm.q[0]);
    const int left = (lane / 8 % 2 == 0 ? 8 * w : 8 * (7 - w)) + lane % 8;      // this lane's row address of a left operand
#pragma unroll
    for (int d = 0; d < DK; d += 16) {
        unsigned ka[NP][4], qa[NP][4];
        load_left<NP, false>(ka, ks + (left * ld + d + lane / 16 * 8) * 2, kC * ld);
        load_left<NP, false>(qa, qs + (left * ld + d + lane / 16 * 8) * 2, kC * ld);
#pragma unroll
        for (int nb = 0; nb < 4; nb++)
            if (2 * nb <= 7 - w) {
                unsigned r[1][NP][4];
                load_right<NP, false>(r[0], at_nk(ks, ld, 16 * nb, d), kC * ld);
                multiply<NP, NP, 1>(reinterpret_cast<float (&)[2][4]>(kk[2 * nb]), ka, r);
                multiply<NP, NP, 1>(reinterpret_cast<float (&)[2][4]>(qk[2 * nb]), qa, r);
            }
    }
    __syncthreads();                    // A takes the place of the tiles
    bf16 *pt = P.p + nc * NT * kTri;
    const f32x2 scale = pair(P.scale, P.scale);
    f32x2 hi[2], lo[2];
#pragma unroll
    for (int half = 0; half < 2; half++) {
        const int i = 8 * (half == 0 ? w : 7 - w) + gr;
        hi[half] = pair(-sm.nhi[i], -sm.nhi[i]);
        lo[half] = pair(-sm.nlo[i], -sm.nlo[i]);
    }
#pragma unroll
    for (int n = 0; n < 8; n++) {
        if (n / 2 > (7 - w) / 2) continue;
        const int j = 8 * n + tc;
        const f32x2 jhi = *reinterpret_cast<const f32x2 *>(&sm.nhi[j]), jlo = *reinterpret_cast<const f32x2 *>(&sm.nlo[j]);
        const f32x2 bt = *reinterpret_cast<const f32x2 *>(&sm.beta[j]);
#pragma unroll
        for (int half = 0; half < 2; half++) {
            const int block = half == 0 ? w : 7 - w, i = 8 * block + gr;
            // whole 16 x 16 blocks on and below the diagonal are read later: the block's upper half as zeros
            if (n / 2 > block / 2) continue;
            const float2 x = halves(add2(add2(hi[half], jhi), add2(lo[half], jlo)));
            const f32x2 decay = pair(exp2_fast(x.x), exp2_fast(x.y));
            float2 p = halves(mul2(mul2(scale, decay), pair(qk[n][2 * half], qk[n][2 * half + 1])));
            float2 a = halves(mul2(mul2(decay, pair(kk[n][2 * half], kk[n][2 * half + 1])), bt));
            if (n >= block) {
                p.x = i >= j ? p.x : 0.f; p.y = i >= j + 1 ? p.y : 0.f;
                a.x = i > j ? a.x : 0.f; a.y = i > j + 1 ? a.y : 0.f;
            }
            unsigned pw[NT], aw[NT];
            split(p.x, p.y, pw);
            split(a.x, a.y, aw);
            const int to = in_triangle(block / 2, n / 2) + (block % 2 * 2 + n % 2) * 64 + lane * 2;
#pragma unroll
            for (int m = 0; m < NT; m++) {
                *reinterpret_cast<unsigned *>(pt + m * kTri + to) = pw[m];
                *reinterpret_cast<unsigned *>(&sm.a[m][i * kLd + j]) = aw[m];
            }
            if (n / 2 == block / 2) *reinterpret_cast<float2 *>(&sm.diag[block / 2][i % 16][j % 16]) = a;
        }
    }
    __syncthreads();
    // inverse of diagonal block w, lane = column; two sums, so that the chain of products is half as long
    if (lane < 16) {
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; i++) {
            float s = i == lane ? 1.f : 0.f, s1 = 0.f;
#pragma unroll
            for (int l = 0; l < i; l += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(&sm.diag[w][i][l]);
                s = fmaf(-v.x, x[l], s);
                if (l + 1 < i) s1 = fmaf(-v.y, x[l + 1], s1);
                if (l + 2 < i) s = fmaf(-v.z, x[l + 2], s);
                if (l + 3 < i) s1 = fmaf(-v.w, x[l + 3], s1);
            }
            x[i] = s + s1;
        }
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            unsigned t[4][NT];
#pragma unroll
            for (int e = 0; e < 4; e++) split(x[i + 2 * e], x[i + 2 * e + 1], t[e]);
#pragma unroll
            for (int m = 0; m < NT; m++) *reinterpret_cast<uint4 *>(&sm.d[m][w][lane * 24 + i]) = make_uint4(t[0][m], t[1][m], t[2][m], t[3][m]);
        }
    }
    __syncthreads();

    // block column J = w: left operands hold T_KJ transposed
    bf16 *tri = P.tri + nc * NT * kTri;
    const unsigned as = smem_addr(sm.a[0]), dsm = smem_addr(sm.d[0][0]);
    unsigned tw[4][NT][4];
    load_left<NT, false>(tw[0], at_kn(dsm + w * 16 * 24 * 2, 24, 0, 0), 4 * 16 * 24);
#pragma unroll
    for (int step = 0; step < 4; step++) {
        const int I = w + step;
        if (I >= 4) break;
        if (step > 0) {
            float y[2][4] = {}, z[2][4] = {};
#pragma unroll
            for (int m = 0; m < step; m++)
                product<NT, NT, false>(y[0], y[1], tw[m], at_nk(as, kLd, 16 * I, 16 * (w + m)), kC * kLd);
            unsigned yw[NT][4];
            as_left(y[0], y[1], yw);
            product<NT, NT, true>(z[0], z[1], yw, at_kn(dsm + I * 16 * 24 * 2, 24, 0, 0), 4 * 16 * 24);
#pragma unroll
            for (int e = 0; e < 4; e++) { z[0][e] = -z[0][e]; z[1][e] = -z[1][e]; }
            as_left(z[0], z[1], tw[step]);
        }
        // rows j = 16 w + (gr, gr + 8), columns i = 16 I + tc (+8); the identity is left out: who uses T adds its
        // factor in float, which keeps that part of the product exact
        unsigned out[NT][4];
#pragma unroll
        for (int m = 0; m < NT; m++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                out[m][e] = tw[step][m][e];
                // words 0 and 3 of a diagonal block hold the diagonal: element tc == gr low half, tc + 1 == gr high
                if (step == 0 && (e == 0 || e == 3)) {
                    if (tc == gr) out[m][e] &= 0xffff0000u;
                    if (tc + 1 == gr) out[m][e] &= 0x0000ffffu;
                }
            }
        bf16 *dst = tri + in_triangle(I, w) + lane * 2;
#pragma unroll
        for (int m = 0; m < NT; m++)
#pragma unroll
            for (int e = 0; e < 4; e++) *reinterpret_cast<unsigned *>(dst + m * kTri + ((e & 1) * 2 + (e >> 1)) * 64) = out[m][e];
    }
}

// Float arrays -> three bfloat16 terms each, dense rows: one launch for all arrays of a call, an array per grid row.
__global__ void __launch_bounds__(256) delta_split_kernel(const SplitJobs jobs)
{
    follow_previous();
    const SplitJob &j = jobs.job[blockIdx.y];
    const int width8 = j.width / 8;
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x, words = jobs.rows * width8;
    if (i >= words) return;
    const long long row = i / width8;
    const int col = (int)(i - row * width8) * 8;
    float f[8];
    load_vec(f, j.src + row * j.stride + col);
    unsigned w[4][3];
#pragma unroll
    for (int e = 0; e < 4; e++) split(f[2 * e], f[2 * e + 1], w[e]);
#pragma unroll
    for (int m = 0; m < 3; m++) *reinterpret_cast<uint4 *>(j.dst + m * (words * 8) + i * 8) = make_uint4(w[0][m], w[1][m], w[2][m], w[3][m]);
}

template <int DK, int NP> cudaError_t prep(const ChunkParams &P, cudaStream_t st)
{
    const size_t smem = sizeof(PrepSmem<DK, NP>);
    const cudaError_t e = cudaFuncSetAttribute(delta_prep_kernel<DK, NP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch<true>(delta_prep_kernel<DK, NP>, dim3((unsigned)(P.B * P.Hv * (long long)P.chunks)), dim3(128), smem, st, P);
}

}  // namespace

cudaError_t launch_delta_prep(const ChunkParams &P, int dk, int terms, cudaStream_t st)
{
    if (terms == 3) return dk == 64 ? prep<64, 3>(P, st) : prep<128, 3>(P, st);
    return dk == 64 ? prep<64, 1>(P, st) : prep<128, 1>(P, st);
}

cudaError_t launch_delta_split(const SplitJobs &jobs, cudaStream_t st)
{
    int width = 0;
    for (int i = 0; i < jobs.count; i++) width = jobs.job[i].width > width ? jobs.job[i].width : width;
    const long long words = jobs.rows * (width / 8);
    return launch<true>(delta_split_kernel, dim3((unsigned)((words + 255) / 256), jobs.count), dim3(256), 0, st, jobs);
}

}  // namespace cawn
