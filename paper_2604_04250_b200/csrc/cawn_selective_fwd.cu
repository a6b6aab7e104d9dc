// Selective scan, forward: walks over tiles of tokens.
#include "cawn_selective.cuh"

namespace cawn {
namespace {

template <class T, int NL, int NS, bool SUMMARY>
__global__ void __launch_bounds__(32 * NL) selective_fwd_kernel(const SelectiveParams P)
{
    follow_previous();
    using At = Place<NL, NS>;
    constexpr int TT = At::kTile, kThreads = At::kThreads, NP = At::kPad, NK = At::kPairs;
    constexpr int kWords = (TT * 4 + kThreads - 1) / kThreads, kQuads = TT * 2 * NP / 4 / kThreads, kRow = 40;
    __shared__ __align__(16) float2 dd[TT][kScanChannels];
    __shared__ __align__(16) float bc[2][TT][NP];
    __shared__ __align__(16) float ys[SUMMARY ? 1 : TT][kRow];
    __shared__ float bias[kScanChannels], skip[kScanChannels];

    const At at;
    const int tid = threadIdx.x, cb = blockIdx.x % (P.G * P.blocks), b = blockIdx.x / (P.G * P.blocks), g = cb / P.blocks;
    const int c0 = g * P.Dg + cb % P.blocks * kScanChannels;
    const int nch = min(kScanChannels, (g + 1) * P.Dg - c0), seg = blockIdx.y;
    const Span s = span_of(P.seq, b);
    const long long begin = seg * P.per, end = s.len < begin + P.per ? s.len : begin + P.per;
    const bool in = at.ch < nch;
    const int c = c0 + (in ? at.ch : 0), n0 = at.nl * NS;
    const long long state = (long long)b * P.D + c;

    f32x2 A2[NK], h[NK];
    load_states<NS>(A2, P.A + (long long)c * P.N, n0, P.N, in);
#pragma unroll
    for (int k = 0; k < NK; k++) A2[k] = mul2(A2[k], twice(kLog2e));
    if constexpr (SUMMARY) {
#pragma unroll
        for (int k = 0; k < NK; k++) h[k] = 0ull;
        if (seg == 0 && P.state_in != nullptr) {        // the walk may overwrite state_in while others still need it
            load_states<NS>(h, P.state_in + state * P.N, n0, P.N, in);
            store_states<NS>(P.first + state * P.N, h, n0, P.N, in);
        }
        if (end >= s.len) return;                       // nobody comes behind this segment
    } else {
        if (seg > 0 && begin >= s.len) return;
        if (seg == 0) {
            const float *from = P.S > 1 ? P.first : P.state_in;
            load_states<NS>(h, from + state * P.N, n0, P.N, in && P.state_in != nullptr);
        } else {
            const long long segment = (long long)b * (P.S - 1) * P.D + c;
            load_states<NS>(h, P.seg_state + segment * P.N, n0, P.N, in);
            for (int i = 1; i < seg; i++) fold_segment<NS>(h, P, A2, segment + (long long)i * P.D, n0, in);
        }
    }
    for (int i = tid; i < kScanChannels; i += kThreads) {
        bias[i] = i < nch && P.dt_bias != nullptr ? P.dt_bias[c0 + i] : 0.f;
        skip[i] = i < nch && P.skip != nullptr ? P.skip[c0 + i] : 0.f;
    }

    const T *x = static_cast<const T *>(P.x) + s.begin * P.xs + c0, *dt = static_cast<const T *>(P.dt) + s.begin * P.dts + c0;
    const T *z = P.z != nullptr && !SUMMARY && P.y != nullptr ? static_cast<const T *>(P.z) + s.begin * P.zs + c0 : nullptr;
    const T *bm = static_cast<const T *>(P.bm) + s.begin * P.bs + g * P.N, *cm = static_cast<const T *>(P.cm) + s.begin * P.cs + g * P.N;
    T *y = !SUMMARY && P.y != nullptr ? static_cast<T *>(P.y) + s.begin * P.D + c0 : nullptr;
    const int word = tid % 4 * 8;                       // this thread's eight channels of a row, at staging and output
    Eight<T> nx[kWords], ndt[kWords], nz[kWords], cx[kWords], cz[kWords];
    Quad<T> nbc[kQuads];
    auto fetch = [&](long long t0) {
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const int r = tid / 4 + i * (kThreads / 4);
            const int n = r < TT && t0 + r < end ? nch - word : 0;
            nx[i] = fetch_eight(x + (t0 + r) * P.xs + word, n, P.whole_x);
            ndt[i] = fetch_eight(dt + (t0 + r) * P.dts + word, n, P.whole_dt);
            if (z != nullptr) nz[i] = fetch_eight(z + (t0 + r) * P.zs + word, n, P.whole_z);
        }
#pragma unroll
        for (int i = 0; i < kQuads; i++) {
            const int q = tid + i * kThreads, m = q / (TT * NP / 4), r = q / (NP / 4) % TT, n = q % (NP / 4) * 4;
            if (SUMMARY && m == 1) continue;
            const int left = t0 + r < end ? P.N - n : 0;
            nbc[i] = m == 0 ? fetch_quad(bm + (t0 + r) * P.bs + n, left, P.whole_b) : fetch_quad(cm + (t0 + r) * P.cs + n, left, P.whole_c);
        }
    };
    fetch(begin);
    float time = 0.f;
    long long mark = !SUMMARY && P.checkpoints != nullptr ? (checkpoint_of(s, b) + begin / kCheckpoint) * P.D + c : 0;
    for (long long t0 = begin; t0 < end; t0 += TT) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const int r = tid / 4 + i * (kThreads / 4);
            if (kWords * kThreads > TT * 4 && r >= TT) break;
            float xf[8], df[8];
            cx[i] = nx[i];
            cz[i] = nz[i];
            nx[i].widen_to(xf);
            ndt[i].widen_to(df);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const float raw = df[j] + bias[word + j], d = P.softplus ? softplus_of(raw) : raw;
                dd[r][word + j] = t0 + r < end ? make_float2(d, d * xf[j]) : make_float2(0.f, 0.f);       // past the end nothing moves
            }
        }
#pragma unroll
        for (int i = 0; i < kQuads; i++) {
            const int q = tid + i * kThreads, m = q / (TT * NP / 4);
            if (SUMMARY && m == 1) continue;
            *reinterpret_cast<float4 *>(&bc[0][0][0] + q * 4) = nbc[i].get();
        }
        __syncthreads();
        if (t0 + TT < end) fetch(t0 + TT);
#pragma unroll 2
        for (int t = 0; t < TT; t += 4) {
            if (!SUMMARY && P.checkpoints != nullptr && t % kCheckpoint == 0 && t0 + t < end) {
                store_states<NS>(P.checkpoints + mark * P.N, h, n0, P.N, in);
                mark += P.D;
            }
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 d = dd[t + i][at.ch];
                f32x2 B[NK], C[NK];
                row_pairs<NS>(B, &bc[0][t + i][n0]);
                if constexpr (!SUMMARY) row_pairs<NS>(C, &bc[1][t + i][n0]);
                f32x2 acc = 0ull;
                const f32x2 dl = twice(d.x), dx = twice(d.y);
#pragma unroll
                for (int k = 0; k < NK; k++) {
                    h[k] = fma2(exp2_pair(mul2(dl, A2[k])), h[k], mul2(dx, B[k]));
                    if constexpr (!SUMMARY) acc = k == 0 ? mul2(h[k], C[k]) : fma2(h[k], C[k], acc);
                }
                if constexpr (SUMMARY) time += d.x;
                else v[i] = sum_of(acc);
            }
            if constexpr (!SUMMARY) sum_four<NL>(v, at.nl, &ys[t][at.ch], kRow);
        }
        if constexpr (!SUMMARY) {
            __syncthreads();
            if (y != nullptr) {
#pragma unroll
                for (int i = 0; i < kWords; i++) {
                    const int r = tid / 4 + i * (kThreads / 4);
                    if (r >= TT || t0 + r >= end) break;
                    float xf[8], f[8];
                    cx[i].widen_to(xf);
#pragma unroll
                    for (int j = 0; j < 8; j += 4) *reinterpret_cast<float4 *>(f + j) = *reinterpret_cast<const float4 *>(&ys[r][word + j]);
#pragma unroll
                    for (int j = 0; j < 8; j++) f[j] = fmaf(skip[word + j], xf[j], f[j]);
                    if (z != nullptr) {
                        float zf[8];
                        cz[i].widen_to(zf);
#pragma unroll
                        for (int j = 0; j < 8; j++) f[j] *= zf[j] * sigmoid_of(zf[j]);
                    }
                    store_eight(y + (t0 + r) * P.D + word, f, nch - word, P.whole_d);
                }
            }
        }
    }
    if constexpr (SUMMARY) {
        const long long segment = ((long long)b * (P.S - 1) + seg) * P.D + c;
        store_states<NS>(P.seg_state + segment * P.N, h, n0, P.N, in);
        if (in && at.nl == 0) P.seg_time[segment] = time;
    } else {
        if (end == s.len && P.state_out != nullptr) store_states<NS>(P.state_out + state * P.N, h, n0, P.N, in);
    }
}

template <class T, bool SUMMARY> SelectiveKernel pick(const Shape &s)
{
    return s.ns == 8 ? selective_fwd_kernel<T, 8, 8, SUMMARY> : s.nl == 8 ? selective_fwd_kernel<T, 8, 4, SUMMARY>
           : s.nl == 4 ? selective_fwd_kernel<T, 4, 4, SUMMARY> : s.nl == 2 ? selective_fwd_kernel<T, 2, 4, SUMMARY> : selective_fwd_kernel<T, 1, 4, SUMMARY>;
}

}  // namespace

int launch_selective_fwd(const SelectiveParams &P, const Shape &s, bool half, bool summary, cudaStream_t st)
{
    const SelectiveKernel k = half ? (summary ? pick<bf16, true>(s) : pick<bf16, false>(s)) : (summary ? pick<float, true>(s) : pick<float, false>(s));
    return status_of(launch<true>(k, dim3((unsigned)(P.G * P.blocks * P.seq.B), (unsigned)(summary ? P.S - 1 : P.S)), dim3(32 * s.nl), 0, st, P));
}

}  // namespace cawn
