// Root-mean-square norm of a stream that a branch is added to, with an output of the branch's type or in 8 bits.
//
// Mathematics: s = x + residual, rounded to the stream's type; r = rsqrt(mean(s^2) + eps), y = s r w.  8 bits: of each
// stretch of channels (or the row) scale = max|y| / 448 and q = y / scale rounded to e4m3, whose largest value is 448.
// Backward with d = w dL/dy, sh = s r:  ds = r (d - sh mean(d sh)) + dL/ds from past the norm;  dw = sum of dL/dy sh.
// Bound: memory.  A row is held in the registers of a team (a warp up to 1024 channels, a block of eight above), eight
// neighbours a lane and word, and read once.
// Measured, 32768 x 768 bfloat16: a float stream with its sum, to 8 bits with a scale per 128 channels, 54 us (5.1 TB/s); the
// backward with a bfloat16 stream 39 us (5.2 TB/s).
#include "cawn_seq.cuh"

#include <cuda_fp8.h>

namespace cawn {
namespace {

struct ResidualNormParams {
    const void *x, *residual, *sum, *gy, *gsum;
    void *y, *sum_out, *gresidual, *gx;
    const float *w;
    float *scales, *part;
    long long N, x_stride;
    int M, words, block_words, scale_cols;      // words of eight channels; of a scale (0: the row)
    float eps, inv_m;
    int x_whole, m_whole;
};

constexpr int kWarps = 8, kNormBlock = 32 * kWarps;

template <class T> __device__ __forceinline__ void pairs_of(f32x2 (&r)[4], const Eight<T> &e)
{
    float f[8];
    e.widen_to(f);
#pragma unroll
    for (int i = 0; i < 4; i++) r[i] = pair(f[2 * i], f[2 * i + 1]);
}
template <bool WHOLE, class T> __device__ __forceinline__ void put_eight(T *p, const float (&f)[8], int n, bool whole)
{
    if constexpr (!WHOLE) store_eight(p, f, n, whole);
    else if (n > 0) store_vec(p, f);
}

// Sum (or maximum) over a team: a warp, or the block's eight.  `turn` tells one use of the block's exchange from the next.
template <int TEAM, bool MAX> __device__ __forceinline__ float over_team(float v, float (*red)[kWarps], int turn)
{
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? (u > v || u != u ? u : v) : v + u;            // a NaN stays
    }
    if constexpr (TEAM > 32) {
        if (threadIdx.x % 32 == 0) red[turn][threadIdx.x / 32] = v;
        __syncthreads();
        v = red[turn][0];
#pragma unroll
        for (int i = 1; i < kWarps; i++) {
            const float u = red[turn][i];
            v = MAX ? (u > v || u != u ? u : v) : v + u;
        }
    }
    return v;
}

__device__ __forceinline__ uint2 to_e4m3(const float (&f)[8])
{
    unsigned u[4];
#pragma unroll
    for (int i = 0; i < 4; i++) u[i] = __nv_cvt_float2_to_fp8x2(make_float2(f[2 * i], f[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
    return make_uint2(u[0] | u[1] << 16, u[2] | u[3] << 16);
}

template <class T, class S, int TEAM, int NV, bool E4M3, bool WHOLE>
__global__ void __launch_bounds__(kNormBlock) residual_norm_fwd_kernel(const ResidualNormParams P)
{
    follow_previous();
    __shared__ float red[2][kWarps];
    const int lane = threadIdx.x % TEAM;
    const long long r = (long long)blockIdx.x * (kNormBlock / TEAM) + threadIdx.x / TEAM;
    if (r >= P.N) return;                                       // whole teams
    const T *x = static_cast<const T *>(P.x) + r * P.x_stride;
    const S *res = P.residual != nullptr ? static_cast<const S *>(P.residual) + r * P.M : nullptr;
    S *sum = P.sum_out != nullptr ? static_cast<S *>(P.sum_out) + r * P.M : nullptr;
    float v[NV][8], q = 0.f;
    Eight<T> xs[NV];
    Eight<S> rs[NV];
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * TEAM + lane) * 8;
        xs[j] = eight_of<WHOLE>(x + c, P.M - c, P.x_whole);
        rs[j] = eight_of<WHOLE>(res + c, res != nullptr ? P.M - c : 0, P.m_whole);
    }
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * TEAM + lane) * 8;
        float b[8];
        xs[j].widen_to(v[j]);
        rs[j].widen_to(b);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            v[j][i] = widen(narrow<S>(v[j][i] + b[i]));         // the stream's own value is what is normed
            q = fmaf(v[j][i], v[j][i], q);
        }
        if (sum != nullptr) put_eight<WHOLE>(sum + c, v[j], P.M - c, P.m_whole);
    }
    const float rstd = __frsqrt_rn(over_team<TEAM, false>(q, red, 0) * P.inv_m + P.eps);
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * TEAM + lane) * 8;
        const Eight<float> wt = eight_of<WHOLE>(P.w + c, P.w != nullptr ? P.M - c : 0, P.M % 4 == 0);
        float w[8];
        wt.widen_to(w);
#pragma unroll
        for (int i = 0; i < 8; i++) v[j][i] = P.w != nullptr ? v[j][i] * rstd * w[i] : v[j][i] * rstd;
        if constexpr (E4M3) {
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float u = fabsf(v[j][i]);
                if (c + i < P.M) m = u > m || u != u ? u : m;
            }
            if (P.block_words > 0) {
                for (int o = P.block_words / 2; o > 0; o /= 2) {
                    const float u = __shfl_xor_sync(0xffffffffu, m, o);
                    m = u > m || u != u ? u : m;
                }
                const float scale = (m < 1e-30f ? 1e-30f : m) / 448.f;
                const int word = j * TEAM + lane;
                if (word < P.words && word % P.block_words == 0) P.scales[r * P.scale_cols + word / P.block_words] = scale;
#pragma unroll
                for (int i = 0; i < 8; i++) v[j][i] /= scale;
            } else {
                top = m > top || m != m ? m : top;
            }
        } else {
            put_eight<WHOLE>(static_cast<T *>(P.y) + r * P.M + c, v[j], P.M - c, P.m_whole);
        }
    }
    if constexpr (E4M3) {
        if (P.block_words == 0) {
            top = over_team<TEAM, true>(top, red, 1);
            const float scale = (top < 1e-30f ? 1e-30f : top) / 448.f;
            if (lane == 0) P.scales[r] = scale;
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int i = 0; i < 8; i++) v[j][i] /= scale;
        }
        unsigned char *y = static_cast<unsigned char *>(P.y) + r * P.M;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TEAM + lane) * 8;
            const uint2 u = to_e4m3(v[j]);
            if (P.M % 8 == 0 && c < P.M) {
                *reinterpret_cast<uint2 *>(y + c) = u;
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (c + i < P.M) y[c + i] = (unsigned char)((i < 4 ? u.x : u.y) >> (8 * (i % 4)));
            }
        }
    }
}

// Two blocks a multiprocessor up to three words a lane, chosen at 768 channels (32768 x 768: 56 us with one, 37 with two, although three words
// do not fit in 128 registers: 64 to 144 bytes a thread are spilled); one or two words do fit, four take 211 to 242.
template <class T, class S, int TEAM, int NV, bool WHOLE>
__global__ void __launch_bounds__(kNormBlock, NV <= 3 ? 2 : 1) residual_norm_bwd_kernel(const ResidualNormParams P)
{
    follow_previous();
    __shared__ float red[2][kWarps];
    __shared__ float fold[TEAM == 32 ? kNormBlock * 8 : 1];
    const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    constexpr int kTeams = kNormBlock / TEAM;
    f32x2 w[NV][4], gw[NV][4] = {};
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * TEAM + lane) * 8;
        if (P.w != nullptr) {
            pairs_of(w[j], eight_of<WHOLE>(P.w + c, P.M - c, P.M % 4 == 0));
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) w[j][i] = twice(1.f);
        }
    }
    for (long long r = (long long)blockIdx.x * kTeams + team; r < P.N; r += (long long)gridDim.x * kTeams) {
        Eight<S> ss[NV], gs[NV];
        Eight<T> gy[NV];
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TEAM + lane) * 8;
            ss[j] = eight_of<WHOLE>(static_cast<const S *>(P.sum) + r * P.M + c, P.M - c, P.m_whole);
            gy[j] = eight_of<WHOLE>(static_cast<const T *>(P.gy) + r * P.M + c, P.M - c, P.m_whole);
            gs[j] = eight_of<WHOLE>(static_cast<const S *>(P.gsum) + r * P.M + c, P.gsum != nullptr ? P.M - c : 0, P.m_whole);
        }
        f32x2 qq = 0ull, pp = 0ull;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            f32x2 s[4], g[4];
            pairs_of(s, ss[j]);
            pairs_of(g, gy[j]);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                qq = fma2(s[i], s[i], qq);
                pp = fma2(mul2(g[i], w[j][i]), s[i], pp);
            }
        }
        const float2 qh = halves(qq), ph = halves(pp);
        const float q = over_team<TEAM, false>(qh.x + qh.y, red, 0), p = over_team<TEAM, false>(ph.x + ph.y, red, 1);
        // r (d - s k) with k = mean(d s) / (mean(s^2) + eps): the two terms may cancel, so k is rounded as few times as it can be
        const float var = q * P.inv_m + P.eps, rstd = __frsqrt_rn(var), k = p * P.inv_m / var;
        const f32x2 r2 = twice(rstd), k2 = twice(-k);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TEAM + lane) * 8;
            f32x2 s[4], g[4], past[4];
            float d[8];
            pairs_of(s, ss[j]);
            pairs_of(g, gy[j]);
            pairs_of(past, gs[j]);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                gw[j][i] = fma2(g[i], mul2(s[i], r2), gw[j][i]);
                const float2 o = halves(fma2(r2, fma2(s[i], k2, mul2(g[i], w[j][i])), past[i]));
                d[2 * i] = o.x;
                d[2 * i + 1] = o.y;
            }
            if (P.gresidual != nullptr) put_eight<WHOLE>(static_cast<S *>(P.gresidual) + r * P.M + c, d, P.M - c, P.m_whole);
            if (P.gx != nullptr) put_eight<WHOLE>(static_cast<T *>(P.gx) + r * P.M + c, d, P.M - c, P.m_whole);
        }
        if constexpr (TEAM > 32) __syncthreads();               // red is written again in the next row
    }
    if (P.part == nullptr) return;
    float *part = P.part + (long long)blockIdx.x * P.M;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        if constexpr (TEAM > 32) {
            const int c = (j * TEAM + lane) * 8;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 v = halves(gw[j][i]);
                if (c + 2 * i < P.M) part[c + 2 * i] = v.x;
                if (c + 2 * i + 1 < P.M) part[c + 2 * i + 1] = v.y;
            }
        } else {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 v = halves(gw[j][i]);
                fold[(team * 8 + 2 * i) * 32 + lane] = v.x;
                fold[(team * 8 + 2 * i + 1) * 32 + lane] = v.y;
            }
            __syncthreads();
            // one channel a thread: 256 of the word row j
            float v = 0.f;
            const int c = threadIdx.x, of = c % 8 * 32 + c / 8;
#pragma unroll
            for (int t = 0; t < kTeams; t++) v += fold[t * 256 + of];
            if (j * 256 + c < P.M) part[j * 256 + c] = v;
        }
    }
}

int check(const cawn_residual_norm_params *p)
{
    if (p == nullptr) return CAWN_ERR_NULL_POINTER;
    if (p->struct_size != sizeof(cawn_residual_norm_params)) return CAWN_ERR_INVALID_ARG;
    if (p->N < 0 || p->M < 1 || !(p->eps >= 0.f) || !storage_flags_ok(p->flags) || (p->stream_float != 0 && p->stream_float != 1) || p->reserved != 0 ||
        (p->out != CAWN_NORM_OUT_SAME && p->out != CAWN_NORM_OUT_E4M3) || (p->x_stride != 0 && p->x_stride < p->M) ||
        (p->out == CAWN_NORM_OUT_SAME ? p->scale_block != 0 : p->scale_block != 0 && p->scale_block != 32 && p->scale_block != 64 && p->scale_block != 128))
        return CAWN_ERR_INVALID_ARG;
    if (p->M > 8192 || p->N > ((int64_t)1 << 31) - 8) return CAWN_ERR_UNSUPPORTED;
    if ((double)p->N * (double)(p->x_stride > p->M ? p->x_stride : p->M) > 1.0e17) return CAWN_ERR_UNSUPPORTED;
    return CAWN_OK;
}

// A team holds up to four words a lane.
struct Team { int size, nv; };
Team team_of(int M)
{
    const int words = (int)ceil_div(M, 8);
    const int size = words <= 128 ? 32 : kNormBlock, need = (int)ceil_div(words, size);
    return {size, need <= 1 ? 1 : need <= 2 ? 2 : need <= 3 ? 3 : 4};
}

// Blocks of the backward: as many as run at once, each with a partial row of sums.  Never fewer for more rows.
int64_t workers(const cawn_residual_norm_params *p)
{
    const Team t = team_of(p->M);
    const int64_t blocks = ceil_div(p->N, kNormBlock / t.size), want = (int64_t)sm_count() * (t.nv <= 3 ? 2 : 1);
    return blocks < want ? blocks : want;
}

ResidualNormParams fill(const cawn_residual_norm_params *p)
{
    ResidualNormParams P = {};
    const int per = p->flags != 0 ? 8 : 4;
    P.N = p->N; P.M = p->M; P.words = (int)ceil_div(p->M, 8);
    P.x_stride = p->x_stride != 0 ? p->x_stride : p->M;
    P.block_words = p->scale_block / 8;
    P.scale_cols = p->scale_block > 0 ? (int)ceil_div(p->M, p->scale_block) : 1;
    P.eps = p->eps; P.inv_m = 1.f / (float)p->M;
    P.x_whole = P.x_stride % per == 0;
    P.m_whole = p->M % per == 0;
    return P;
}

using Kernel = void (*)(ResidualNormParams);
// KIND: 0 forward, 1 forward to e4m3, 2 backward.  WHOLE: all rows are whole 16-byte words of eight channels.
template <class T, class S, int KIND, bool WHOLE> Kernel pick(const Team &t)
{
#define CAWN_PICK(TEAM, NV)                                                                                           \
    if (t.size == TEAM && t.nv == NV) {                                                                               \
        if constexpr (KIND == 2) return residual_norm_bwd_kernel<T, S, TEAM, NV, WHOLE>;                              \
        else return residual_norm_fwd_kernel<T, S, TEAM, NV, KIND == 1, WHOLE>;                                       \
    }
    CAWN_PICK(32, 1) CAWN_PICK(32, 2) CAWN_PICK(32, 3) CAWN_PICK(32, 4)
    CAWN_PICK(kNormBlock, 1) CAWN_PICK(kNormBlock, 2) CAWN_PICK(kNormBlock, 3) CAWN_PICK(kNormBlock, 4)
#undef CAWN_PICK
    return nullptr;
}
template <int KIND, bool WHOLE> Kernel pick(const cawn_residual_norm_params *p, const Team &t)
{
    if (p->flags == 0) return pick<float, float, KIND, WHOLE>(t);
    return p->stream_float ? pick<bf16, float, KIND, WHOLE>(t) : pick<bf16, bf16, KIND, WHOLE>(t);
}
template <int KIND> Kernel pick(const cawn_residual_norm_params *p, const ResidualNormParams &P, const Team &t)
{
    const bool whole = P.m_whole && (KIND == 2 || P.x_whole) && p->M % 8 == 0;
    return whole ? pick<KIND, true>(p, t) : pick<KIND, false>(p, t);
}

}  // namespace
}  // namespace cawn

extern "C" int cawn_residual_norm_fwd(const cawn_residual_norm_params *params, const void *x, const void *residual, const float *weight,
                                      void *sum_out, void *y, float *scales, void *cuda_stream)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    const bool e4m3 = params->out == CAWN_NORM_OUT_E4M3;
    if (!e4m3 && scales != nullptr) return CAWN_ERR_INVALID_ARG;
    if (params->N == 0) return CAWN_OK;
    if (x == nullptr || y == nullptr || (e4m3 && scales == nullptr)) return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(residual, weight, sum_out, y, scales) || !elements_aligned(params->flags, x)) return CAWN_ERR_MISALIGNED;
    ResidualNormParams P = fill(params);
    P.x = x; P.x_whole = P.x_whole && begins_on(x, 16); P.residual = residual; P.w = weight; P.sum_out = sum_out; P.y = y; P.scales = scales;
    const Team t = team_of(params->M);
    return status_of(launch<true>(e4m3 ? pick<1>(params, P, t) : pick<0>(params, P, t), dim3((unsigned)ceil_div(P.N, kNormBlock / t.size)), dim3(kNormBlock), 0,
                                  static_cast<cudaStream_t>(cuda_stream), P));
}

extern "C" int cawn_residual_norm_workspace_bytes(const cawn_residual_norm_params *params, size_t *bytes)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (bytes == nullptr) return CAWN_ERR_NULL_POINTER;
    *bytes = (size_t)workers(params) * params->M * sizeof(float);
    return CAWN_OK;
}

extern "C" int cawn_residual_norm_bwd(const cawn_residual_norm_params *params, const void *sum, const float *weight, const void *grad_y,
                                      const void *grad_sum, void *grad_residual, void *grad_x, float *grad_weight,
                                      void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (params->N > 0 && (sum == nullptr || grad_y == nullptr || (grad_residual == nullptr && grad_x == nullptr))) return CAWN_ERR_NULL_POINTER;
    if (grad_weight != nullptr && workspace == nullptr && params->N > 0) return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(sum, weight, grad_y, grad_sum, grad_residual, grad_x, grad_weight, workspace)) return CAWN_ERR_MISALIGNED;
    const int64_t blocks = workers(params);
    if (grad_weight != nullptr && workspace_bytes < (size_t)blocks * params->M * sizeof(float)) return CAWN_ERR_WORKSPACE_TOO_SMALL;
    if (params->N == 0)
        return grad_weight != nullptr ? status_of(cudaMemsetAsync(grad_weight, 0, (size_t)params->M * sizeof(float), st)) : CAWN_OK;
    ResidualNormParams P = fill(params);
    P.sum = sum; P.w = weight; P.gy = grad_y; P.gsum = grad_sum; P.gresidual = grad_residual; P.gx = grad_x;
    P.part = grad_weight != nullptr ? static_cast<float *>(workspace) : nullptr;
    const int first = status_of(launch<true>(pick<2>(params, P, team_of(params->M)), dim3((unsigned)blocks), dim3(kNormBlock), 0, st, P));
    if (first != CAWN_OK || grad_weight == nullptr) return first;
    PartialSums S = {P.part, blocks, params->M, {grad_weight, nullptr, nullptr}, {params->M, 0, 0}};
    return sum_partials(S, st);
}
