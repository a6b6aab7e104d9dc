// Selective scan, forward: walks over tiles of tokens.
#include "cawn_selective.cuh"

namespace cawn {
namespace {

template <class T, int NL, int NS, int CD, bool SUMMARY, bool WHOLE>
__global__ void __launch_bounds__(32 * NL / CD) selective_fwd_kernel(const SelectiveParams P)
{
    follow_previous();
    using At = Place<NL, NS, CD>;
    constexpr int kThreads = At::kThreads, NP = At::kPad, NK = At::kPairs, kWords = At::kWords, kStagers = At::kStagers;
    __shared__ __align__(16) float2 dd[2][kTile][kScanChannels];                  // d, d x
    __shared__ __align__(16) float2 gates[SUMMARY ? 1 : 2][kTile][kScanChannels]; // skip x, silu(z)
    __shared__ __align__(16) float bc[2][2][kTile][NP];
    __shared__ __align__(16) float bias[kScanChannels], skip[kScanChannels];

    const At at;
    const int tid = threadIdx.x, cb = blockIdx.x % (P.G * P.blocks), b = blockIdx.x / (P.G * P.blocks), g = cb / P.blocks;
    const int c0 = g * P.Dg + cb % P.blocks * kScanChannels;
    const int nch = min(kScanChannels, (g + 1) * P.Dg - c0), seg = blockIdx.y;
    const Span s = span_of(P.seq, b);
    const long long begin = seg * P.per, end = s.len < begin + P.per ? s.len : begin + P.per;
    const int n0 = at.nl * NS;

    f32x2 A2[CD][NK], h[CD][NK];
    if constexpr (SUMMARY) {
        const bool first = seg == 0 && P.state_in != nullptr;
#pragma unroll
        for (int j = 0; j < CD; j++) {
            const bool in = at.ch + j < nch;
            const long long state = (long long)b * P.D + c0 + at.ch + j;
            load_states<NS>(h[j], P.state_in + state * P.N, n0, P.N, in && first);
            if (first) store_states<NS>(P.first + state * P.N, h[j], n0, P.N, in);      // the walk may overwrite state_in while others need it
        }
        if (end >= s.len) return;                       // nobody comes behind this segment
    } else {
        if (seg > 0 && begin >= s.len) return;
    }
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const int c = c0 + at.ch + j;
        load_states<NS>(A2[j], P.A + (long long)c * P.N, n0, P.N, in);
#pragma unroll
        for (int k = 0; k < NK; k++) A2[j][k] = mul2(A2[j][k], twice(kLog2e));
        if constexpr (!SUMMARY) {
            if (seg == 0) {
                const float *from = P.S > 1 ? P.first : P.state_in;
                load_states<NS>(h[j], from + ((long long)b * P.D + c) * P.N, n0, P.N, in && P.state_in != nullptr);
            } else {
                const long long segment = (long long)b * (P.S - 1) * P.D + c;
                load_states<NS>(h[j], P.seg_state + segment * P.N, n0, P.N, in);
                for (int i = 1; i < seg; i++) fold_segment<NS>(h[j], P, A2[j], segment + (long long)i * P.D, n0, in);
            }
        }
    }
    for (int i = tid; i < kScanChannels; i += kThreads) {
        bias[i] = i < nch && P.dt_bias != nullptr ? P.dt_bias[c0 + i] : 0.f;
        skip[i] = i < nch && P.skip != nullptr ? P.skip[c0 + i] : 0.f;
    }

    const T *x = static_cast<const T *>(P.x) + s.begin * P.xs + c0, *dt = static_cast<const T *>(P.dt) + s.begin * P.dts + c0;
    const T *z = P.z != nullptr && !SUMMARY && P.y != nullptr ? static_cast<const T *>(P.z) + s.begin * P.zs + c0 : nullptr;
    T *y = !SUMMARY && P.y != nullptr ? static_cast<T *>(P.y) + s.begin * P.D + c0 : nullptr;
    const int word = tid % 4 * 8;                       // this thread's eight channels of a row, at staging
    const int quad_row = tid / (NP / 4), quad = tid % (NP / 4) * 4;     // and its four states of a row of B and C
    const T *bm = static_cast<const T *>(P.bm) + (s.begin + quad_row) * P.bs + g * P.N + quad, *cm = static_cast<const T *>(P.cm) + (s.begin + quad_row) * P.cs + g * P.N + quad;
    Eight<T> nx[kWords], ndt[kWords], nz[kWords];
    Quad<T> nb, nc;
    auto fetch = [&](long long t0) {
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const long long r = t0 + tid / 4 + i * (kStagers / 4);
            const int n = tid < kStagers && r < end ? nch - word : 0;
            nx[i] = eight_of<WHOLE>(x + r * P.xs + word, n, P.whole_x);
            ndt[i] = eight_of<WHOLE>(dt + r * P.dts + word, n, P.whole_dt);
            if (!SUMMARY) nz[i] = eight_of<WHOLE>(z + r * P.zs + word, z != nullptr ? n : 0, P.whole_z);
        }
        const int left = t0 + quad_row < end ? P.N - quad : 0;
        nb = quad_of<WHOLE>(bm + t0 * P.bs, left, P.whole_b);
        if (!SUMMARY) nc = quad_of<WHOLE>(cm + t0 * P.cs, left, P.whole_c);
    };
    auto stage = [&](long long t0, int to) {
        if (kStagers == kThreads || tid < kStagers) {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const int r = tid / 4 + i * (kStagers / 4);
                float xf[8], df[8], zf[8];
                nx[i].widen_to(xf);
                ndt[i].widen_to(df);
                if (!SUMMARY) nz[i].widen_to(zf);
                const f32x2 there = twice(t0 + r < end ? 1.f : 0.f);        // past the end nothing moves
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const f32x2 xx = pair(xf[j], xf[j + 1]), raw = add2(pair(df[j], df[j + 1]), *reinterpret_cast<const f32x2 *>(&bias[word + j]));
                    const f32x2 d = mul2(chosen(P.softplus, softplus_of(raw), raw), there);
                    const float2 e = halves(d), f = halves(mul2(d, xx));
                    *reinterpret_cast<float4 *>(&dd[to][r][word + j]) = make_float4(e.x, f.x, e.y, f.y);
                    if constexpr (!SUMMARY) {
                        const f32x2 zz = pair(zf[j], zf[j + 1]);
                        const float2 v = halves(mul2(*reinterpret_cast<const f32x2 *>(&skip[word + j]), xx));
                        const float2 w = halves(chosen(z != nullptr, mul2(zz, sigmoid_of(zz)), twice(1.f)));
                        *reinterpret_cast<float4 *>(&gates[to][r][word + j]) = make_float4(v.x, w.x, v.y, w.y);
                    }
                }
            }
        }
        *reinterpret_cast<float4 *>(&bc[to][0][quad_row][quad]) = nb.get();
        if (!SUMMARY) *reinterpret_cast<float4 *>(&bc[to][1][quad_row][quad]) = nc.get();
    };
    fetch(begin);
    __syncthreads();            // bias, skip
    stage(begin, 0);
    fetch(begin + kTile);
    float time[CD] = {};
    float *mark = P.checkpoints + ((checkpoint_of(s, b) + begin / kTile) * P.D + c0 + at.ch) * P.N;
    int buf = 0;
    for (long long t0 = begin; t0 < end; t0 += kTile, mark += (long long)P.D * P.N, buf ^= 1) {
        __syncthreads();        // this tile is staged, and the one before has been read
        if (!SUMMARY && P.checkpoints != nullptr) {
#pragma unroll
            for (int j = 0; j < CD; j++) store_states<NS>(mark + j * P.N, h[j], n0, P.N, at.ch + j < nch);
        }
        // straight on from here: the next tile is staged, the one after it sets out, this one is computed; two tokens' decays
        // are found while the two before them move the states
        stage(t0 + kTile, buf ^ 1);
        fetch(t0 + 2 * kTile);
        f32x2 a[2][2][CD][NK], in[2][2][CD][NK];
        auto decays = [&](int u) {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                f32x2 B[NK];
                float2 d[CD];
                row_pairs<NS>(B, &bc[buf][0][2 * u + i][n0]);
                two_of<CD>(d, &dd[buf][2 * u + i][at.ch]);
#pragma unroll
                for (int j = 0; j < CD; j++) {
#pragma unroll
                    for (int k = 0; k < NK; k++) {
                        a[u % 2][i][j][k] = exp2_pair(mul2(twice(d[j].x), A2[j][k]));
                        in[u % 2][i][j][k] = mul2(twice(d[j].y), B[k]);
                    }
                    if constexpr (SUMMARY) time[j] += d[j].x;
                }
            }
        };
        decays(0);
        float v[CD][4];
#pragma unroll
        for (int u = 0; u < kTile / 2; u++) {
            if (u + 1 < kTile / 2) decays(u + 1);
#pragma unroll
            for (int i = 0; i < 2; i++) {
                f32x2 C[NK];
                if constexpr (!SUMMARY) row_pairs<NS>(C, &bc[buf][1][2 * u + i][n0]);
#pragma unroll
                for (int j = 0; j < CD; j++) {
                    f32x2 acc = 0ull;
#pragma unroll
                    for (int k = 0; k < NK; k++) {
                        h[j][k] = fma2(a[u % 2][i][j][k], h[j][k], in[u % 2][i][j][k]);
                        if constexpr (!SUMMARY) acc = k == 0 ? mul2(h[j][k], C[k]) : fma2(h[j][k], C[k], acc);
                    }
                    if constexpr (!SUMMARY) v[j][u % 2 * 2 + i] = sum_of(acc);
                }
            }
            if constexpr (!SUMMARY) {
                if (u % 2 == 1) {
#pragma unroll
                    for (int j = 0; j < CD; j++) sum_four<NL>(v[j], at.nl);
#pragma unroll
                    for (int q = 0; q < Four<NL>::kSums; q++) {
                        const int t = 2 * u - 2 + at.nl % 4 + 2 * q;
                        float2 gate[CD];
                        float o[CD];
                        two_of<CD>(gate, &gates[buf][t][at.ch]);
#pragma unroll
                        for (int j = 0; j < CD; j++) o[j] = (v[j][q] + gate[j].x) * gate[j].y;
                        if (y != nullptr && t0 + t < end && at.nl < 4)
                            store_channels<T, CD>(y + (t0 + t) * P.D + at.ch, o, nch - at.ch, WHOLE || P.whole_d);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const int c = c0 + at.ch + j;
        if constexpr (SUMMARY) {
            const long long segment = ((long long)b * (P.S - 1) + seg) * P.D + c;
            store_states<NS>(P.seg_state + segment * P.N, h[j], n0, P.N, in);
            if (in && at.nl == 0) P.seg_time[segment] = time[j];
        } else {
            if (end == s.len && P.state_out != nullptr) store_states<NS>(P.state_out + ((long long)b * P.D + c) * P.N, h[j], n0, P.N, in);
        }
    }
}

template <class T, bool SUMMARY, bool WHOLE> SelectiveKernel pick(const Shape &s)
{
#define CAWN_CALL(NL, NS, CD) selective_fwd_kernel<T, NL, NS, CD, SUMMARY, WHOLE>
    return CAWN_BY_SHAPE(s, CAWN_CALL);
#undef CAWN_CALL
}

}  // namespace

int launch_selective_fwd(const SelectiveParams &P, const Shape &s, bool half, bool summary, cudaStream_t st)
{
    const SelectiveKernel k = half ? (summary ? (P.whole ? pick<bf16, true, true>(s) : pick<bf16, true, false>(s)) : (P.whole ? pick<bf16, false, true>(s) : pick<bf16, false, false>(s)))
                                   : (summary ? (P.whole ? pick<float, true, true>(s) : pick<float, true, false>(s)) : (P.whole ? pick<float, false, true>(s) : pick<float, false, false>(s)));
    return status_of(launch<true>(k, dim3((unsigned)(P.G * P.blocks * P.seq.B), (unsigned)(summary ? P.S - 1 : P.S)), dim3(32 * s.warps()), 0, st, P));
}

}  // namespace cawn
