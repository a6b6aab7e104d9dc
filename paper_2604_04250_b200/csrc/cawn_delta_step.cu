// Gated delta rule, token by token.
//
// Mathematics, per value row (a Dk-vector s of the state): s <- a s, u = beta (v - s.k), s <- s + u k,
// o = scale s.q.  With both dot products taken on the old row, s.k and s.q, the new row's read-out is
// a s.q + u k.q, so one reduction round serves both.
// Bound: the state is read and written once (8 bytes a cell), everything else is Dk + Dv numbers; a call is HBM-bound
// for a batch (1536 states of 128 x 128, one token: 33.5 us, 6.1 TB/s) and latency-bound for one stream (12 states of
// 64 x 64: 3.5 us).  A row is dealt to LPR lanes, 8 floats each as two float4 (coalesced, no shared memory); a thread
// holds R rows so that a batch keeps R * 32 bytes per thread in flight, while few rows take R = 1 and spread over
// more SMs.
// The 2R dot products are summed over the lanes by halving: each exchange sends half of a lane's partial sums away and
// keeps the other half, so that 2R - 1 exchanges (and a full one per bit that is left) do what 2R log2(LPR) would, and
// each lane ends up with one dot product, its row's u or o to compute, and only that row's v to read.  The next token's
// rows are fetched while this one's are summed (1024 heads of 128 x 128, 16 tokens: 155 -> 102 us for both).
#include "cawn_delta.cuh"

namespace cawn {
namespace {

constexpr int kStepThreads = 128;
constexpr unsigned kAll = 0xffffffffu;

// Four elements as they are stored, and as two pairs of floats.
template <class T> struct Four;
template <> struct Four<float> {
    float4 w;
    __device__ f32x2 low() const { return pair(w.x, w.y); }
    __device__ f32x2 high() const { return pair(w.z, w.w); }
};
template <> struct Four<bf16> {
    uint2 w;
    __device__ f32x2 low() const { return pair(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u)); }
    __device__ f32x2 high() const { return pair(__uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)); }
};
template <class T> __device__ __forceinline__ Four<T> four(const T *p, bool in)
{
    Four<T> r = {};
    if (in) r = *reinterpret_cast<const Four<T> *>(p);
    return r;
}

// One token as a lane needs it: its columns of key and query, its row's value, decay and step.
template <class T> struct Token {
    Four<T> k[2], q[2];
    float v, g, beta;
};

template <class T, int LPR, int R>
__global__ void __launch_bounds__(kStepThreads) delta_step_kernel(const DeltaParams P)
{
    follow_previous();
    constexpr int kRowsWarp = 32 / LPR, kRowsPass = kStepThreads / LPR, kSums = 2 * R, kHolds = LPR / kSums;
    static_assert(kHolds >= 1, "a dot product per lane");
    const int lane = threadIdx.x % LPR, row0 = blockIdx.y * (kRowsPass * R) + (threadIdx.x / 32) * kRowsWarp + (threadIdx.x % 32) / LPR;
    const int bh = blockIdx.x, b = bh / P.Hv, h = bh % P.Hv, hk = h / (P.Hv / P.Hk);
    const int c0 = lane * 4, c1 = (LPR + lane) * 4;              // this lane's columns: c0..c0+3 and c1..c1+3
    const bool in0 = c0 < P.Dk, in1 = c1 < P.Dk;
    // after the exchanges this lane holds s.k (lower half of the lanes) or s.q (upper half) of row `mine`
    const int mine = row0 + (lane / kHolds % R) * kRowsPass;
    const long long srow = (long long)bh * P.Dv * P.Dk;
    const T *q = static_cast<const T *>(P.q) + (long long)b * P.L * P.q_stride + (long long)hk * P.Dk;
    const T *k = static_cast<const T *>(P.k) + (long long)b * P.L * P.k_stride + (long long)hk * P.Dk;
    const T *v = static_cast<const T *>(P.v) + (long long)b * P.L * P.v_stride + (long long)h * P.Dv;
    T *o = static_cast<T *>(P.o) + (long long)b * P.L * P.o_stride + (long long)h * P.Dv;
    const float *g = P.g + (long long)b * P.L * P.Hv + h, *beta = P.beta + (long long)b * P.L * P.Hv + h;

    f32x2 s[R][4];
#pragma unroll
    for (int i = 0; i < R; i++) {
        const int row = row0 + i * kRowsPass;
        float4 lo = make_float4(0.f, 0.f, 0.f, 0.f), hi = lo;
        if (P.state_in != nullptr && row < P.Dv) {
            const float *src = P.state_in + srow + (long long)row * P.Dk;
            if (in0) lo = *reinterpret_cast<const float4 *>(src + c0);
            if (in1) hi = *reinterpret_cast<const float4 *>(src + c1);
        }
        s[i][0] = pair(lo.x, lo.y); s[i][1] = pair(lo.z, lo.w);
        s[i][2] = pair(hi.x, hi.y); s[i][3] = pair(hi.z, hi.w);
    }
    auto fetch = [&](long long t) {
        Token<T> x;
        x.k[0] = four(k + t * P.k_stride + c0, in0); x.k[1] = four(k + t * P.k_stride + c1, in1);
        x.q[0] = four(q + t * P.q_stride + c0, in0); x.q[1] = four(q + t * P.q_stride + c1, in1);
        x.v = mine < P.Dv ? widen(v[t * P.v_stride + mine]) : 0.f;
        x.g = g[t * P.Hv]; x.beta = beta[t * P.Hv];
        return x;
    };
    Token<T> next = fetch(0);
    for (long long t = 0; t < P.L; t++) {
        const Token<T> now = next;
        if (t + 1 < P.L) next = fetch(t + 1);
        const f32x2 kv[4] = {now.k[0].low(), now.k[0].high(), now.k[1].low(), now.k[1].high()};
        const f32x2 qv[4] = {now.q[0].low(), now.q[0].high(), now.q[1].low(), now.q[1].high()};
        const float a = decay_of(now.g);
        float sums[kSums];                                       // s.k of the R rows, then s.q
#pragma unroll
        for (int i = 0; i < R; i++) {
            f32x2 sk = mul2(s[i][0], kv[0]), sq = mul2(s[i][0], qv[0]);
#pragma unroll
            for (int e = 1; e < 4; e++) { sk = fma2(s[i][e], kv[e], sk); sq = fma2(s[i][e], qv[e], sq); }
            const float2 x = halves(sk), y = halves(sq);
            sums[i] = x.x + x.y; sums[R + i] = y.x + y.y;
        }
        f32x2 both = mul2(kv[0], qv[0]);
#pragma unroll
        for (int e = 1; e < 4; e++) both = fma2(kv[e], qv[e], both);
        float kq = halves(both).x + halves(both).y;
#pragma unroll
        for (int m = LPR / 2, n = R; m > 0; m /= 2, n /= 2) {
            kq += __shfl_xor_sync(kAll, kq, m);
            if (n == 0) sums[0] += __shfl_xor_sync(kAll, sums[0], m);
            const bool upper = lane & m;
#pragma unroll
            for (int i = 0; i < n; i++) {
                const float sent = upper ? sums[i] : sums[n + i], kept = upper ? sums[n + i] : sums[i];
                sums[i] = kept + __shfl_xor_sync(kAll, sent, m);
            }
        }
        const float u = now.beta * (now.v - a * sums[0]), u_of_mine = __shfl_xor_sync(kAll, u, LPR / 2);   // u: lower half
        if (lane >= LPR / 2 && lane % kHolds == 0 && mine < P.Dv)
            o[t * P.o_stride + mine] = narrow<T>(P.scale * fmaf(u_of_mine, kq, a * sums[0]));
        const f32x2 aa = pair(a, a);
#pragma unroll
        for (int i = 0; i < R; i++) {
            const float ui = __shfl_sync(kAll, u, i * kHolds, LPR);
            const f32x2 uu = pair(ui, ui);
#pragma unroll
            for (int e = 0; e < 4; e++) s[i][e] = fma2(uu, kv[e], mul2(aa, s[i][e]));
        }
    }
    if (P.state_out == nullptr) return;
#pragma unroll
    for (int i = 0; i < R; i++) {
        const int row = row0 + i * kRowsPass;
        if (row >= P.Dv) continue;
        float *dst = P.state_out + srow + (long long)row * P.Dk;
        const float2 w0 = halves(s[i][0]), w1 = halves(s[i][1]), w2 = halves(s[i][2]), w3 = halves(s[i][3]);
        if (in0) *reinterpret_cast<float4 *>(dst + c0) = make_float4(w0.x, w0.y, w1.x, w1.y);
        if (in1) *reinterpret_cast<float4 *>(dst + c1) = make_float4(w2.x, w2.y, w3.x, w3.y);
    }
}

template <class T, int LPR> cudaError_t go(const DeltaParams &P, cudaStream_t st)
{
    constexpr int pass = kStepThreads / LPR;
    const long long heads = (long long)P.B * P.Hv;
    const int blocks1 = (P.Dv + pass - 1) / pass, blocks4 = (P.Dv + 4 * pass - 1) / (4 * pass);
    // four rows a thread when that still gives every SM several blocks
    if (heads * blocks4 >= 4ll * sm_count())
        return launch<true>(delta_step_kernel<T, LPR, 4>, dim3((unsigned)heads, blocks4), dim3(kStepThreads), 0, st, P);
    return launch<true>(delta_step_kernel<T, LPR, 1>, dim3((unsigned)heads, blocks1), dim3(kStepThreads), 0, st, P);
}

}  // namespace

cudaError_t launch_delta_step(const DeltaParams &P, bool half, cudaStream_t st)
{
    // 8 lanes cover 64 columns, 16 lanes 128
    if (P.Dk <= 64) return half ? go<bf16, 8>(P, st) : go<float, 8>(P, st);
    return half ? go<bf16, 16>(P, st) : go<float, 16>(P, st);
}

}  // namespace cawn
