// Short causal convolution, channel by channel, with its history and an optional SiLU.
//
// Mathematics: with e the sequence behind its history of K - 1 rows, z_t = bias + sum_k w_k e_{t+k}, y_t = z_t or z_t sigmoid(z_t);
// the new history is e's last K - 1 rows.  Backward: dz = dy act'(z), de_i = sum_k w_k dz_{i-k} (and the new history's
// gradient on the last K - 1), dw_k = sum_t dz_t e_{t+k}, dbias = sum_t dz_t.
// Bound: memory; an element costs K products.  A thread keeps eight channels (a 16-byte word of bfloat16) and walks
// kRows rows with the last K - 1 of them in registers, so that a row is fetched once but for the K - 1 in front of
// a walk, which the neighbour's fetch has brought to L1 or L2.
#include "cawn_seq.cuh"

namespace cawn {
namespace {

constexpr int kRows = 16, kLanes = 32, kWalks = 4, kTile = kRows * kWalks;     // a block: 32 words of channels, 4 walks
constexpr int kConvThreads = kLanes * kWalks;

struct ConvParams {
    Sequences seq;
    const void *x, *gy;
    void *y, *gx;
    const float *w, *b, *state_in, *gstate_out;
    float *state_out, *gstate_in, *part;
    long long x_stride, tiles, all_tiles;       // tiles of a sequence of L rows, of all sequences
    int C, words, silu, x_whole, c_whole;
};

template <class T> __device__ __forceinline__ void row_of(float (&f)[8], const T *p, int n, bool whole) { fetch_eight(p, n, whole).widen_to(f); }

// Row `i` of the sequence behind its history (i < 0: history, zero without one), as the arrays hold it.
template <class T, int K>
__device__ __forceinline__ void extended(float (&f)[8], const ConvParams &P, const T *x, const float *history, long long i, int n)
{
    if (i >= 0) row_of(f, x + i * P.x_stride, n, P.x_whole);
    else if (history != nullptr) row_of(f, history + (i + K - 1) * P.C, n, P.c_whole);
    else {
#pragma unroll
        for (int c = 0; c < 8; c++) f[c] = 0.f;
    }
}

template <int K> __device__ __forceinline__ void taps_of(float (&w)[K][8], float (&b)[8], const ConvParams &P, int c0, int n)
{
#pragma unroll
    for (int c = 0; c < 8; c++) {
#pragma unroll
        for (int k = 0; k < K; k++) w[k][c] = c < n ? P.w[(long long)(c0 + c) * K + k] : 0.f;
        b[c] = c < n && P.b != nullptr ? P.b[c0 + c] : 0.f;
    }
}

template <class T, int K>
__global__ void __launch_bounds__(kConvThreads) conv_fwd_kernel(const ConvParams P)
{
    follow_previous();
    const int word = (blockIdx.y * kLanes + threadIdx.x % kLanes), c0 = word * 8;
    if (word >= P.words) return;
    const int n = P.C - c0 < 8 ? P.C - c0 : 8;
    const int b = (int)(blockIdx.x / P.tiles);
    const long long t0 = (blockIdx.x % P.tiles) * kTile + threadIdx.x / kLanes * kRows;
    const Span s = span_of(P.seq, b);
    const T *x = static_cast<const T *>(P.x) + s.begin * P.x_stride + c0;
    const float *history = P.state_in != nullptr && K > 1 ? P.state_in + (long long)b * (K - 1) * P.C + c0 : nullptr;

    // The new history, by the walk at the sequence's start: it alone reads the old one, which may be the same array.
    float old[K][8];            // row j of the window's past; K - 1 are used
    if (t0 < s.len || t0 == 0) {
#pragma unroll
        for (int j = 0; j < K - 1; j++) extended<T, K>(old[j], P, x, history, t0 + j - (K - 1), n);
    }
    if (K > 1 && t0 == 0 && P.state_out != nullptr) {
        float *out = P.state_out + (long long)b * (K - 1) * P.C + c0;
#pragma unroll
        for (int j = 0; j < K - 1; j++) {
            float f[8];
            extended<T, K>(f, P, x, history, s.len + j - (K - 1), n);       // never a row of the history that is overwritten already
            store_eight(out + (long long)j * P.C, f, n, P.c_whole);
        }
    }
    if (t0 >= s.len) return;
    float w[K][8], bias[8];
    taps_of<K>(w, bias, P, c0, n);
    T *y = static_cast<T *>(P.y) + (s.begin + t0) * P.C + c0;
    x += t0 * P.x_stride;
    const int rows = s.len - t0 < kRows ? (int)(s.len - t0) : kRows;
#pragma unroll
    for (int r0 = 0; r0 < kRows; r0 += 8) {
        Eight<T> next[8];       // eight rows in flight
#pragma unroll
        for (int r = 0; r < 8; r++) next[r] = fetch_eight(x + (r0 + r) * P.x_stride, r0 + r < rows ? n : 0, P.x_whole);
#pragma unroll
        for (int r = 0; r < 8; r++) {
            float f[8], z[8];
            next[r].widen_to(f);
#pragma unroll
            for (int c = 0; c < 8; c++) {
                float v = bias[c];
#pragma unroll
                for (int k = 0; k < K - 1; k++) v = fmaf(w[k][c], old[k][c], v);
                v = fmaf(w[K - 1][c], f[c], v);
                z[c] = P.silu ? v * sigmoid_of(v) : v;
#pragma unroll
                for (int k = 0; k + 2 < K; k++) old[k][c] = old[k + 1][c];
                if (K > 1) old[K > 1 ? K - 2 : 0][c] = f[c];
            }
            if (r0 + r < rows) store_eight(y + (long long)(r0 + r) * P.C, z, n, P.c_whole);
        }
    }
}

// A block takes tile after tile, so that few partial sums of the parameters' gradients are left.
template <class T, int K>
__global__ void __launch_bounds__(kConvThreads) conv_bwd_kernel(const ConvParams P)
{
    follow_previous();
    __shared__ float fold[kWalks][kLanes][8];
    const int lane = threadIdx.x % kLanes, walk = threadIdx.x / kLanes, word = blockIdx.y * kLanes + lane, c0 = word * 8;
    const int n = word < P.words ? (P.C - c0 < 8 ? P.C - c0 : 8) : 0;
    float w[K][8], bias[8], gw[K][8] = {}, gb[8] = {};
    taps_of<K>(w, bias, P, n > 0 ? c0 : 0, n);
    for (long long tile = blockIdx.x; tile < P.all_tiles; tile += gridDim.x) {
        const int b = (int)(tile / P.tiles);
        const long long t0 = (tile % P.tiles) * kTile + walk * kRows;
        const Span s = span_of(P.seq, b);
        if (n == 0 || (t0 >= s.len && t0 != 0)) continue;
        const T *x = static_cast<const T *>(P.x) + s.begin * P.x_stride + c0;
        const T *gy = static_cast<const T *>(P.gy) + s.begin * P.C + c0;
        T *gx = static_cast<T *>(P.gx) + s.begin * P.C + c0;
        const float *history = P.state_in != nullptr && K > 1 ? P.state_in + (long long)b * (K - 1) * P.C + c0 : nullptr;
        const float *gso = P.gstate_out != nullptr && K > 1 ? P.gstate_out + (long long)b * (K - 1) * P.C + c0 : nullptr;
        float old[K][8], dz[K][8] = {};         // rows t-K+1 .. t-1 of e; dz of rows t-K+1 .. t (0 before this walk)
#pragma unroll
        for (int j = 0; j < K - 1; j++) extended<T, K>(old[j], P, x, history, t0 + j - (K - 1), n);
        const long long end = t0 + kRows < s.len ? t0 + kRows : s.len;      // this walk's own rows end here
        // row t gives dz_t; what then is complete is the gradient of row t - (K - 1), whose last term dz_t is
#pragma unroll 4
        for (int r = 0; r < kRows + K - 1; r++) {
            const long long t = t0 + r;
            if (t - (K - 1) >= end && t0 != 0) break;
            float f[8], g[8];
            row_of(f, x + t * P.x_stride, t < s.len ? n : 0, P.x_whole);
            row_of(g, gy + t * P.C, t < s.len ? n : 0, P.c_whole);
            const bool own = t < end;
#pragma unroll
            for (int c = 0; c < 8; c++) {
                float d = g[c];
                if (P.silu) {
                    float v = bias[c];
#pragma unroll
                    for (int k = 0; k < K - 1; k++) v = fmaf(w[k][c], old[k][c], v);
                    v = fmaf(w[K - 1][c], f[c], v);
                    d *= silu_slope(v, sigmoid_of(v));
                }
                if (t >= s.len) d = 0.f;
#pragma unroll
                for (int k = 0; k + 1 < K; k++) dz[k][c] = dz[k + 1][c];
                dz[K - 1][c] = d;
                if (own) {
#pragma unroll
                    for (int k = 0; k < K - 1; k++) gw[k][c] = fmaf(d, old[k][c], gw[k][c]);
                    gw[K - 1][c] = fmaf(d, f[c], gw[K - 1][c]);
                    gb[c] += d;
                }
#pragma unroll
                for (int k = 0; k + 2 < K; k++) old[k][c] = old[k + 1][c];
                if (K > 1) old[K > 1 ? K - 2 : 0][c] = f[c];
            }
            const long long i = t - (K - 1);                // the row of x that is complete, or below 0 one of the history
            if (i >= end || (i < t0 && (t0 != 0 || P.gstate_in == nullptr || K == 1))) continue;
            float de[8];
#pragma unroll
            for (int c = 0; c < 8; c++) {
                de[c] = 0.f;
#pragma unroll
                for (int k = 0; k < K; k++) de[c] = fmaf(w[k][c], dz[K - 1 - k][c], de[c]);
            }
            const long long j = i + (K - 1) - s.len;        // its place in the new history
            if (j >= 0 && gso != nullptr) {
                float g2[8];
                row_of(g2, gso + j * P.C, n, P.c_whole);
#pragma unroll
                for (int c = 0; c < 8; c++) de[c] += g2[c];
            }
            if (i >= 0) store_eight(gx + i * P.C, de, n, P.c_whole);
            else store_eight(P.gstate_in + ((long long)b * (K - 1) + i + K - 1) * P.C + c0, de, n, P.c_whole);
        }
    }
    if (P.part == nullptr) return;
    float *part = P.part + (long long)blockIdx.x * P.C * (K + 1);
#pragma unroll
    for (int k = 0; k <= K; k++) {
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 8; c++) fold[walk][lane][c] = k < K ? gw[k < K ? k : 0][c] : gb[c];
        __syncthreads();
        for (int i = threadIdx.x; i < kLanes * 8; i += kConvThreads) {
            const int c = blockIdx.y * kLanes * 8 + i;
            float v = 0.f;
#pragma unroll
            for (int q = 0; q < kWalks; q++) v += fold[q][i / 8][i % 8];
            if (c < P.C) part[k < K ? (long long)c * K + k : (long long)P.C * K + c] = v;
        }
    }
}

int check(const cawn_conv_params *p)
{
    if (p == nullptr) return CAWN_ERR_NULL_POINTER;
    if (p->struct_size != sizeof(cawn_conv_params)) return CAWN_ERR_INVALID_ARG;
    if (p->B < 1 || p->L < 0 || p->C < 1 || p->K < 1 || !storage_flags_ok(p->flags) || p->rows < 0 || p->reserved[0] != 0 || p->reserved[1] != 0 ||
        (p->act != CAWN_CONV_ACT_NONE && p->act != CAWN_CONV_ACT_SILU) || (p->x_stride != 0 && p->x_stride < p->C))
        return CAWN_ERR_INVALID_ARG;
    if (p->K > 4 || p->C > (1 << 22)) return CAWN_ERR_UNSUPPORTED;
    const double rows = p->rows > 0 ? (double)p->rows : (double)p->B * (double)p->L;
    if (rows * (double)(p->x_stride > p->C ? p->x_stride : p->C) > 1.0e17) return CAWN_ERR_UNSUPPORTED;
    if ((double)p->B * (double)(p->L / kTile + 1) > 2.0e9) return CAWN_ERR_UNSUPPORTED;
    return CAWN_OK;
}

ConvParams fill(const cawn_conv_params *p, const int64_t *offsets)
{
    ConvParams P = {};
    const int per = p->flags != 0 ? 8 : 4;
    P.seq = {reinterpret_cast<const long long *>(offsets), p->L, offsets != nullptr ? p->rows : (int64_t)p->B * p->L, p->B};
    P.C = p->C;
    P.x_stride = p->x_stride != 0 ? p->x_stride : p->C;
    P.words = (int)ceil_div(p->C, 8);
    P.tiles = most(ceil_div(p->L, kTile), 1);
    P.all_tiles = P.tiles * p->B;
    P.silu = p->act == CAWN_CONV_ACT_SILU;
    P.x_whole = P.x_stride % per == 0;
    P.c_whole = p->C % per == 0 && p->C % 4 == 0;
    return P;
}

// Blocks along the tiles in the backward: about eight a SM, each with a partial row of sums.  Never fewer for more tiles.
int64_t workers(const cawn_conv_params *p)
{
    const int64_t across = ceil_div(ceil_div(p->C, 8), kLanes), tiles = most(ceil_div(p->L, kTile), 1) * p->B;
    const int64_t want = most((int64_t)sm_count() * 8 / across, 1);
    return tiles < want ? tiles : want;
}

using ConvKernel = void (*)(ConvParams);
template <class T> ConvKernel pick(int K, bool bwd)
{
    switch (K) {
    case 1: return bwd ? conv_bwd_kernel<T, 1> : conv_fwd_kernel<T, 1>;
    case 2: return bwd ? conv_bwd_kernel<T, 2> : conv_fwd_kernel<T, 2>;
    case 3: return bwd ? conv_bwd_kernel<T, 3> : conv_fwd_kernel<T, 3>;
    default: return bwd ? conv_bwd_kernel<T, 4> : conv_fwd_kernel<T, 4>;
    }
}

}  // namespace
}  // namespace cawn

extern "C" int cawn_short_conv_fwd(const cawn_conv_params *params, const void *x, const float *weight, const float *bias,
                                   const float *state_in, const int64_t *offsets, void *y, float *state_out, void *cuda_stream)
{
    using namespace cawn;
    int rc = check(params);
    if (rc == CAWN_OK) rc = check_offsets(offsets, params->B, params->L, params->rows);
    if (rc != CAWN_OK) return rc;
    if (weight == nullptr || (params->L > 0 && (x == nullptr || y == nullptr))) return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(x, weight, bias, state_in, y, state_out)) return CAWN_ERR_MISALIGNED;
    ConvParams P = fill(params, offsets);
    P.x = x; P.w = weight; P.b = bias; P.state_in = state_in; P.y = y; P.state_out = state_out;
    const ConvKernel k = params->flags != 0 ? pick<bf16>(params->K, false) : pick<float>(params->K, false);
    return status_of(launch<true>(k, dim3((unsigned)P.all_tiles, (unsigned)ceil_div(P.words, kLanes)), dim3(kConvThreads), 0,
                                  static_cast<cudaStream_t>(cuda_stream), P));
}

extern "C" int cawn_short_conv_workspace_bytes(const cawn_conv_params *params, size_t *bytes)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (bytes == nullptr) return CAWN_ERR_NULL_POINTER;
    *bytes = (size_t)workers(params) * params->C * (params->K + 1) * sizeof(float);
    return CAWN_OK;
}

extern "C" int cawn_short_conv_bwd(const cawn_conv_params *params, const void *x, const float *weight, const float *bias,
                                   const float *state_in, const int64_t *offsets, const void *grad_y, const float *grad_state_out,
                                   void *grad_x, float *grad_weight, float *grad_bias, float *grad_state_in,
                                   void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    using namespace cawn;
    int rc = check(params);
    if (rc == CAWN_OK) rc = check_offsets(offsets, params->B, params->L, params->rows);
    if (rc != CAWN_OK) return rc;
    const bool sums = grad_weight != nullptr || grad_bias != nullptr;
    if (weight == nullptr || (params->L > 0 && (x == nullptr || grad_y == nullptr || grad_x == nullptr)) || (sums && workspace == nullptr))
        return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(x, weight, bias, state_in, grad_y, grad_state_out, grad_x, grad_weight, grad_bias, grad_state_in, workspace))
        return CAWN_ERR_MISALIGNED;
    const int64_t blocks = workers(params), cols = (int64_t)params->C * (params->K + 1);
    if (sums && workspace_bytes < (size_t)blocks * cols * sizeof(float)) return CAWN_ERR_WORKSPACE_TOO_SMALL;
    ConvParams P = fill(params, offsets);
    P.x = x; P.w = weight; P.b = bias; P.state_in = state_in; P.gy = grad_y; P.gstate_out = grad_state_out;
    P.gx = grad_x; P.gstate_in = grad_state_in; P.part = sums ? static_cast<float *>(workspace) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const ConvKernel k = params->flags != 0 ? pick<bf16>(params->K, true) : pick<float>(params->K, true);
    rc = status_of(launch<true>(k, dim3((unsigned)blocks, (unsigned)ceil_div(P.words, kLanes)), dim3(kConvThreads), 0, st, P));
    if (rc != CAWN_OK || !sums) return rc;
    PartialSums S = {P.part, blocks, cols, {grad_weight, grad_bias, nullptr}, {(long long)params->C * params->K, params->C, 0}};
    return sum_partials(S, st);
}
