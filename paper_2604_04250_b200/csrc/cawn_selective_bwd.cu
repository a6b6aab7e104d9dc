// Selective scan, backward.
//
// Mathematics, with w_t = e^{d_t A} h_{t-1} and dy' = dy silu(z): going back in time
//   lam_t = C_t dy'_t + e^{d_{t+1} A} lam_{t+1},   dB_t = sum_c lam d x,  dC_t = sum_c dy' h_t,  flow = sum_n lam B,
//   dx = d flow + skip dy',   dd = sum_n lam w A + x flow,   ddt = dd sigmoid(dt + bias),   dA = sum_t lam w d,
//   dz = dy (sum_n C h + skip x) silu'(z).
// A walk takes tiles of 32 tokens from the last to the first.  States are found again from the checkpoints, 16 tokens
// apart: w and the decays of 32 / NS tokens stay in registers while the walk turns round.  So a decay's exponential is
// taken 1.5 times, which hides behind the arithmetic.
// Sums over states go by shuffles.  Sums over channels (dB, dC) go through the tensor cores: the left factor is a selection,
// ones in row t (and 8 + t) and zeros elsewhere, so that one m16n8k8 adds four channels' lam d x to row t and their
// dy' h to row 8 + t for eight lanes' states at once.  Its operands have 11 bits of mantissa, so a term goes in as two
// (with one, gradients of bfloat16 rows that a few channels cancel in were off by twice their rounding).
#include "cawn_selective.cuh"

namespace cawn {
namespace {

__device__ __forceinline__ void select_add(float (&d)[4], unsigned one, unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%5,%4}, {%6,%7}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(one), "r"(0u), "r"(b0), "r"(b1));
}
// The leading 11 bits of a float's mantissa, and the next 11 of what is left.
__device__ __forceinline__ unsigned leading(float v) { return __float_as_uint(v) & 0xffffe000u; }
__device__ __forceinline__ void sum_channels(float (&d)[4], unsigned one, float u, float v)
{
    const unsigned a = leading(u), b = leading(v);
    select_add(d, one, a, b);
    select_add(d, one, leading(u - __uint_as_float(a)), leading(v - __uint_as_float(b)));
}

template <int NL, int NS> struct BwdShared {
    using At = Place<NL, NS>;
    static constexpr int TT = At::kTile, kRow = 40, kStagers = At::kThreads < TT * 4 ? At::kThreads : TT * 4;
    float2 dd[TT][kScanChannels];
    float dy[TT][kScanChannels];
    float bc[2][TT][At::kPad];
    float sums[3][TT][kRow];            // flow, drift (sum of lam w A log2 e), read-out
    float red[2][NL][512];              // [state of a lane][dB, dC][token][lane group]
    float param[2][kStagers][8];        // grad_skip, grad_dt_bias of a stager's channels
    float bias[kScanChannels], skip[kScanChannels];
};

template <class T, int NL, int NS, bool GATE>
__global__ void __launch_bounds__(32 * NL, NL == 4 ? 3 : 1) selective_bwd_kernel(const SelectiveParams P)
{
    follow_previous();
    using At = Place<NL, NS>;
    using Shared = BwdShared<NL, NS>;
    constexpr int TT = At::kTile, kThreads = At::kThreads, NP = At::kPad, NK = At::kPairs, kRow = Shared::kRow;
    constexpr int kWords = (TT * 4 + kThreads - 1) / kThreads, kQuads = TT * 2 * NP / 4 / kThreads;
    constexpr int TS = 32 / NS, kSubs = kCheckpoint / TS, kChunks = TT / kCheckpoint;
    extern __shared__ __align__(16) unsigned char raw_shared[];
    Shared &sh = *reinterpret_cast<Shared *>(raw_shared);

    const At at;
    const int tid = threadIdx.x, lane = tid % 32, cb = blockIdx.x % (P.G * P.blocks), b = blockIdx.x / (P.G * P.blocks), g = cb / P.blocks;
    const int c0 = g * P.Dg + cb % P.blocks * kScanChannels;
    const int nch = min(kScanChannels, (g + 1) * P.Dg - c0), seg = blockIdx.y;
    const Span s = span_of(P.seq, b);
    const long long begin = seg * P.per, end = s.len < begin + P.per ? s.len : begin + P.per;
    const bool in = at.ch < nch;
    const int c = c0 + (in ? at.ch : 0), n0 = at.nl * NS;
    const long long state = (long long)b * P.D + c;
    float *param = P.part_param + ((long long)b * P.S + seg) * P.param_cols;

    f32x2 A2[NK], carry[NK], dA[NK];
    load_states<NS>(A2, P.A + (long long)c * P.N, n0, P.N, in);
#pragma unroll
    for (int k = 0; k < NK; k++) {
        A2[k] = mul2(A2[k], twice(kLog2e));
        dA[k] = 0ull;
    }
    for (int i = tid; i < kScanChannels; i += kThreads) {
        sh.bias[i] = i < nch && P.dt_bias != nullptr ? P.dt_bias[c0 + i] : 0.f;
        sh.skip[i] = i < nch && P.skip != nullptr ? P.skip[c0 + i] : 0.f;
    }
    for (int i = tid; i < Shared::kStagers; i += kThreads)
#pragma unroll
        for (int j = 0; j < 8; j++) sh.param[0][i][j] = sh.param[1][i][j] = 0.f;
    load_states<NS>(carry, P.gstate_out + state * P.N, n0, P.N, in && P.gstate_out != nullptr);
    for (long long i = (s.len - 1) / P.per; i > seg; i--)
        fold_segment<NS>(carry, P, A2, ((long long)b * (P.S - 1) + i - 1) * P.D + c, n0, in);

    const T *x = static_cast<const T *>(P.x) + s.begin * P.xs + c0, *dt = static_cast<const T *>(P.dt) + s.begin * P.dts + c0;
    const T *z = GATE ? static_cast<const T *>(P.z) + s.begin * P.zs + c0 : nullptr, *gy = static_cast<const T *>(P.gy) + s.begin * P.D + c0;
    const T *bm = static_cast<const T *>(P.bm) + s.begin * P.bs + g * P.N, *cm = static_cast<const T *>(P.cm) + s.begin * P.cs + g * P.N;
    const float *marks = P.checkpoints + (checkpoint_of(s, b) * P.D + c) * P.N;
    T *gx = static_cast<T *>(P.gx) + s.begin * P.D + c0, *gdt = static_cast<T *>(P.gdt) + s.begin * P.D + c0;
    T *gz = GATE ? static_cast<T *>(P.gz) + s.begin * P.D + c0 : nullptr;
    float *bc_out = P.part_bc + ((long long)cb * P.seq.rows + s.begin) * 2 * P.N;
    const int word = tid % 4 * 8;
    struct Words { Eight<T> x, dt, z, gy; };
    auto fetch_word = [&](Words &w, long long t0, int r) {
        const int n = r < TT && t0 + r < end ? nch - word : 0;
        w.x = fetch_eight(x + (t0 + r) * P.xs + word, n, P.whole_x);
        w.dt = fetch_eight(dt + (t0 + r) * P.dts + word, n, P.whole_dt);
        if (GATE) w.z = fetch_eight(z + (t0 + r) * P.zs + word, n, P.whole_z);
        w.gy = fetch_eight(gy + (t0 + r) * P.D + word, n, P.whole_d);
    };
    Words next[kWords];
    Quad<T> nbc[kQuads];
    f32x2 nh[kChunks][NK];
    auto fetch = [&](long long t0) {
#pragma unroll
        for (int i = 0; i < kWords; i++) fetch_word(next[i], t0, tid / 4 + i * (kThreads / 4));
#pragma unroll
        for (int i = 0; i < kQuads; i++) {
            const int q = tid + i * kThreads, m = q / (TT * NP / 4), r = q / (NP / 4) % TT, n = q % (NP / 4) * 4;
            const int left = t0 + r < end ? P.N - n : 0;
            nbc[i] = m == 0 ? fetch_quad(bm + (t0 + r) * P.bs + n, left, P.whole_b) : fetch_quad(cm + (t0 + r) * P.cs + n, left, P.whole_c);
        }
#pragma unroll
        for (int q = 0; q < kChunks; q++) {
            const long long t = t0 + q * kCheckpoint;
            load_states<NS>(nh[q], marks + (t < end ? t / kCheckpoint : 0) * P.D * P.N, n0, P.N, in && t < end);
        }
    };
    const long long last = begin + (end - 1 - begin) / TT * TT;
    if (end > begin) fetch(last);
    int buf = 0;
    for (long long t0 = last; t0 >= begin && end > begin; t0 -= TT) {
        __syncthreads();
        f32x2 hq[kChunks][NK];
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const int r = tid / 4 + i * (kThreads / 4);
            if (kWords * kThreads > TT * 4 && r >= TT) break;
            float xf[8], df[8], gf[8], zf[8];
            next[i].x.widen_to(xf);
            next[i].dt.widen_to(df);
            next[i].gy.widen_to(gf);
            if (GATE) next[i].z.widen_to(zf);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const float raw = df[j] + sh.bias[word + j], d = P.softplus ? softplus_of(raw) : raw;
                sh.dd[r][word + j] = t0 + r < end ? make_float2(d, d * xf[j]) : make_float2(0.f, 0.f);
                sh.dy[r][word + j] = GATE ? gf[j] * zf[j] * sigmoid_of(zf[j]) : gf[j];
            }
        }
#pragma unroll
        for (int i = 0; i < kQuads; i++) *reinterpret_cast<float4 *>(&sh.bc[0][0][0] + (tid + i * kThreads) * 4) = nbc[i].get();
#pragma unroll
        for (int q = 0; q < kChunks; q++)
#pragma unroll
            for (int k = 0; k < NK; k++) hq[q][k] = nh[q][k];
        __syncthreads();
        if (t0 > begin) fetch(t0 - TT);
#pragma unroll 1
        for (int q = kChunks - 1; q >= 0; q--) {
            if (t0 + q * kCheckpoint >= end) continue;          // for the whole block
            f32x2 hs[kSubs][NK];                                // the states in front of each stretch of TS tokens
#pragma unroll
            for (int k = 0; k < NK; k++) hs[0][k] = kChunks > 1 && q > 0 ? hq[kChunks - 1][k] : hq[0][k];
#pragma unroll
            for (int u = 0; u + 1 < kSubs; u++) {
#pragma unroll
                for (int k = 0; k < NK; k++) hs[u + 1][k] = hs[u][k];
#pragma unroll
                for (int i = 0; i < TS; i++) {
                    const int t = q * kCheckpoint + u * TS + i;
                    const float2 d = sh.dd[t][at.ch];
                    f32x2 B[NK];
                    row_pairs<NS>(B, &sh.bc[0][t][n0]);
#pragma unroll
                    for (int k = 0; k < NK; k++) hs[u + 1][k] = fma2(exp2_pair(mul2(twice(d.x), A2[k])), hs[u + 1][k], mul2(twice(d.y), B[k]));
                }
            }
#pragma unroll
            for (int u = kSubs - 1; u >= 0; u--) {
                const int t1 = q * kCheckpoint + u * TS;
                f32x2 a[TS][NK], w[TS][NK], h[NK];
                float v[4];
#pragma unroll
                for (int k = 0; k < NK; k++) h[k] = hs[u][k];
#pragma unroll
                for (int i = 0; i < TS; i++) {
                    const float2 d = sh.dd[t1 + i][at.ch];
                    f32x2 B[NK], C[NK], acc = 0ull;
                    row_pairs<NS>(B, &sh.bc[0][t1 + i][n0]);
                    if constexpr (GATE) row_pairs<NS>(C, &sh.bc[1][t1 + i][n0]);
#pragma unroll
                    for (int k = 0; k < NK; k++) {
                        a[i][k] = exp2_pair(mul2(twice(d.x), A2[k]));
                        w[i][k] = mul2(a[i][k], h[k]);
                        h[k] = fma2(twice(d.y), B[k], w[i][k]);
                        if constexpr (GATE) acc = k == 0 ? mul2(h[k], C[k]) : fma2(h[k], C[k], acc);
                    }
                    if constexpr (GATE) {
                        v[i % 4] = sum_of(acc);
                        if (i % 4 == 3) sum_four<NL>(v, at.nl, &sh.sums[2][t1 + i - 3][at.ch], kRow);
                    }
                }
                float sums[NS][4] = {}, flow[4], drift[4];
#pragma unroll
                for (int i = TS - 1; i >= 0; i--) {
                    const int t = t1 + i;
                    const float2 d = sh.dd[t][at.ch];
                    const f32x2 dl = twice(d.x), dx = twice(d.y), dy = twice(sh.dy[t][at.ch]);
                    f32x2 B[NK], C[NK], fl = 0ull, dr = 0ull;
                    row_pairs<NS>(B, &sh.bc[0][t][n0]);
                    row_pairs<NS>(C, &sh.bc[1][t][n0]);
                    const unsigned one = lane >> 2 == i ? 0x3f800000u : 0u;
#pragma unroll
                    for (int k = 0; k < NK; k++) {
                        const f32x2 now = fma2(dx, B[k], w[i][k]), lam = fma2(C[k], dy, carry[k]), m = mul2(lam, w[i][k]);
                        fl = k == 0 ? mul2(lam, B[k]) : fma2(lam, B[k], fl);
                        dr = k == 0 ? mul2(m, A2[k]) : fma2(m, A2[k], dr);
                        dA[k] = fma2(m, dl, dA[k]);
                        carry[k] = mul2(a[i][k], lam);
                        const float2 gb = halves(mul2(lam, dx)), gc = halves(mul2(now, dy));
                        sum_channels(sums[2 * k], one, gb.x, gc.x);
                        sum_channels(sums[2 * k + 1], one, gb.y, gc.y);
                    }
                    flow[i % 4] = sum_of(fl);
                    drift[i % 4] = sum_of(dr);
                    if (i % 4 == 0) {
                        sum_four<NL>(flow, at.nl, &sh.sums[0][t][at.ch], kRow);
                        sum_four<NL>(drift, at.nl, &sh.sums[1][t][at.ch], kRow);
                    }
                }
                // rows of a selection's result: tokens; columns: the groups of lanes that a lane / 4 names
                float *red = sh.red[buf][tid / 32];
                if (lane / 4 < TS) {
#pragma unroll
                    for (int k = 0; k < NS; k++) {
                        *reinterpret_cast<float2 *>(red + (k * 2 * TS + lane / 4) * 8 + lane % 4 * 2) = make_float2(sums[k][0], sums[k][1]);
                        *reinterpret_cast<float2 *>(red + ((k * 2 + 1) * TS + lane / 4) * 8 + lane % 4 * 2) = make_float2(sums[k][2], sums[k][3]);
                    }
                }
                __syncthreads();
                for (int o = tid; o < 2 * TS * NP; o += kThreads) {
                    const int n = o % NP, m = o / NP % 2, i = o / NP / 2;
                    float sum = 0.f;
#pragma unroll
                    for (int r = 0; r < 8; r++)         // warps, and groups of channels in a warp
                        sum += sh.red[buf][r % NL][((n % NS * 2 + m) * TS + i) * 8 + r / NL * NL + n / NS];
                    if (n < P.N && t0 + t1 + i < end) bc_out[((t0 + t1 + i) * 2 + m) * P.N + n] = sum;
                }
                buf ^= 1;
            }
        }
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const int r = tid / 4 + i * (kThreads / 4);
            if (r >= TT || t0 + r >= end) break;
            Words own;
            fetch_word(own, t0, r);
            float xf[8], df[8], gf[8], zf[8], ox[8], od[8], oz[8];
            own.x.widen_to(xf);
            own.dt.widen_to(df);
            own.gy.widen_to(gf);
            if (GATE) own.z.widen_to(zf);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const int ch = word + j;
                const float fl = sh.sums[0][r][ch], raw = df[j] + sh.bias[ch], skip = sh.skip[ch], dy = sh.dy[r][ch];
                ox[j] = fmaf(sh.dd[r][ch].x, fl, skip * dy);
                od[j] = fmaf(sh.sums[1][r][ch], kLn2, xf[j] * fl);
                if (P.softplus) od[j] *= sigmoid_of(raw);
                if (GATE) oz[j] = gf[j] * fmaf(skip, xf[j], sh.sums[2][r][ch]) * silu_slope(zf[j], sigmoid_of(zf[j]));
                if (ch < nch) {
                    sh.param[0][tid][j] = fmaf(dy, xf[j], sh.param[0][tid][j]);
                    sh.param[1][tid][j] += od[j];
                }
            }
            store_eight(gx + (t0 + r) * P.D + word, ox, nch - word, P.whole_d);
            store_eight(gdt + (t0 + r) * P.D + word, od, nch - word, P.whole_d);
            if (GATE) store_eight(gz + (t0 + r) * P.D + word, oz, nch - word, P.whole_d);
        }
    }
    if (seg == 0 && P.gstate_in != nullptr) store_states<NS>(P.gstate_in + state * P.N, carry, n0, P.N, in);
    store_states<NS>(param + (long long)c * P.N, dA, n0, P.N, in);
    __syncthreads();
    for (int i = tid; i < 2 * nch; i += kThreads) {
        const int m = i / nch, ch = i % nch;
        float sum = 0.f;
        for (int r = ch / 8; r < Shared::kStagers; r += 4) sum += sh.param[m][r][ch % 8];
        param[(long long)P.D * (P.N + m) + c0 + ch] = sum;
    }
}

// A segment's own gradient at its start, and its sum of d: for the segments in front of it.
template <class T, int NL, int NS>
__global__ void __launch_bounds__(32 * NL) selective_bwd_summary_kernel(const SelectiveParams P)
{
    follow_previous();
    using At = Place<NL, NS>;
    constexpr int TT = At::kTile, kThreads = At::kThreads, NP = At::kPad, NK = At::kPairs;
    constexpr int kWords = (TT * 4 + kThreads - 1) / kThreads, kQuads = (TT * NP / 4 + kThreads - 1) / kThreads;
    __shared__ __align__(16) float2 dd[TT][kScanChannels];
    __shared__ __align__(16) float cs[TT][NP];
    const At at;
    const int tid = threadIdx.x, cb = blockIdx.x % (P.G * P.blocks), b = blockIdx.x / (P.G * P.blocks), g = cb / P.blocks;
    const int c0 = g * P.Dg + cb % P.blocks * kScanChannels;
    const int nch = min(kScanChannels, (g + 1) * P.Dg - c0), seg = blockIdx.y + 1;
    const Span s = span_of(P.seq, b);
    const long long begin = seg * P.per, end = s.len < begin + P.per ? s.len : begin + P.per;
    if (begin >= s.len) return;
    const bool in = at.ch < nch;
    const int c = c0 + (in ? at.ch : 0), n0 = at.nl * NS;
    f32x2 A2[NK], own[NK], past[NK];
    load_states<NS>(A2, P.A + (long long)c * P.N, n0, P.N, in);
#pragma unroll
    for (int k = 0; k < NK; k++) {
        A2[k] = mul2(A2[k], twice(kLog2e));
        own[k] = 0ull;
        past[k] = twice(1.f);
    }
    const T *dt = static_cast<const T *>(P.dt) + s.begin * P.dts + c0, *gy = static_cast<const T *>(P.gy) + s.begin * P.D + c0;
    const T *z = P.z != nullptr ? static_cast<const T *>(P.z) + s.begin * P.zs + c0 : nullptr;
    const T *cm = static_cast<const T *>(P.cm) + s.begin * P.cs + g * P.N;
    const int word = tid % 4 * 8;
    Eight<T> ndt[kWords], ngy[kWords], nz[kWords];
    Quad<T> nc[kQuads];
    auto fetch = [&](long long t0) {
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const int r = tid / 4 + i * (kThreads / 4), n = r < TT && t0 + r < end ? nch - word : 0;
            ndt[i] = fetch_eight(dt + (t0 + r) * P.dts + word, n, P.whole_dt);
            ngy[i] = fetch_eight(gy + (t0 + r) * P.D + word, n, P.whole_d);
            if (z != nullptr) nz[i] = fetch_eight(z + (t0 + r) * P.zs + word, n, P.whole_z);
        }
#pragma unroll
        for (int i = 0; i < kQuads; i++) {
            const int q = tid + i * kThreads, r = q / (NP / 4), n = q % (NP / 4) * 4;
            nc[i] = fetch_quad(cm + (t0 + r) * P.cs + n, r < TT && t0 + r < end ? P.N - n : 0, P.whole_c);
        }
    };
    fetch(begin);
    float time = 0.f;
    for (long long t0 = begin; t0 < end; t0 += TT) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const int r = tid / 4 + i * (kThreads / 4);
            if (kWords * kThreads > TT * 4 && r >= TT) break;
            float df[8], gf[8], zf[8];
            ndt[i].widen_to(df);
            ngy[i].widen_to(gf);
            if (z != nullptr) nz[i].widen_to(zf);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const float raw = df[j] + (P.dt_bias != nullptr && word + j < nch ? P.dt_bias[c0 + word + j] : 0.f);
                const float d = P.softplus ? softplus_of(raw) : raw, dy = z != nullptr ? gf[j] * zf[j] * sigmoid_of(zf[j]) : gf[j];
                dd[r][word + j] = t0 + r < end ? make_float2(d, dy) : make_float2(0.f, 0.f);
            }
        }
#pragma unroll
        for (int i = 0; i < kQuads; i++) {
            const int q = tid + i * kThreads;
            if (q < TT * NP / 4) *reinterpret_cast<float4 *>(&cs[0][0] + q * 4) = nc[i].get();
        }
        __syncthreads();
        if (t0 + TT < end) fetch(t0 + TT);
#pragma unroll 4
        for (int t = 0; t < TT; t++) {
            const float2 d = dd[t][at.ch];
            f32x2 C[NK];
            row_pairs<NS>(C, &cs[t][n0]);
            time += d.x;
#pragma unroll
            for (int k = 0; k < NK; k++) {
                past[k] = mul2(past[k], exp2_pair(mul2(twice(d.x), A2[k])));
                own[k] = fma2(past[k], mul2(C[k], twice(d.y)), own[k]);
            }
        }
    }
    const long long segment = ((long long)b * (P.S - 1) + seg - 1) * P.D + c;
    store_states<NS>(P.seg_state + segment * P.N, own, n0, P.N, in);
    if (in && at.nl == 0) P.seg_time[segment] = time;
}

// Gradients of B and C: the sums over a group's blocks of channels, in their order.
template <class T>
__global__ void __launch_bounds__(256) selective_bc_kernel(const SelectiveParams P, T *gb, T *gc, long long tiles)
{
    follow_previous();
    const int b = (int)(blockIdx.x / tiles), g = blockIdx.y, cols = 2 * P.N;
    const Span s = span_of(P.seq, b);
    const long long t0 = blockIdx.x % tiles * 32, rows = s.len - t0 < 32 ? s.len - t0 : 32, step = P.seq.rows * cols;
    const float *part = P.part_bc + (long long)g * P.blocks * step + (s.begin + t0) * cols;
    for (long long i = threadIdx.x; i < rows * cols; i += blockDim.x) {
        float sum = 0.f;
        for (int k = 0; k < P.blocks; k++) sum += part[k * step + i];
        const long long row = s.begin + t0 + i / cols;
        const int n = (int)(i % cols);
        T *out = n < P.N ? gb + row * P.G * P.N + g * P.N + n : gc + row * P.G * P.N + g * P.N + n - P.N;
        *out = narrow<T>(sum);
    }
}

template <class T, bool GATE, int NL, int NS> int run(const SelectiveParams &P, dim3 grid, cudaStream_t st)
{
    constexpr size_t bytes = sizeof(BwdShared<NL, NS>);
    auto k = selective_bwd_kernel<T, NL, NS, GATE>;
    if (bytes > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != cudaSuccess) return status_of(e);
    }
    return status_of(launch<true>(k, grid, dim3(32 * NL), bytes, st, P));
}
template <class T, bool GATE> int run(const SelectiveParams &P, const Shape &s, dim3 grid, cudaStream_t st)
{
    return s.ns == 8 ? run<T, GATE, 8, 8>(P, grid, st) : s.nl == 8 ? run<T, GATE, 8, 4>(P, grid, st) : s.nl == 4 ? run<T, GATE, 4, 4>(P, grid, st)
           : s.nl == 2 ? run<T, GATE, 2, 4>(P, grid, st) : run<T, GATE, 1, 4>(P, grid, st);
}
template <class T> SelectiveKernel pick_summary(const Shape &s)
{
    return s.ns == 8 ? selective_bwd_summary_kernel<T, 8, 8> : s.nl == 8 ? selective_bwd_summary_kernel<T, 8, 4>
           : s.nl == 4 ? selective_bwd_summary_kernel<T, 4, 4> : s.nl == 2 ? selective_bwd_summary_kernel<T, 2, 4> : selective_bwd_summary_kernel<T, 1, 4>;
}

}  // namespace

int launch_selective_bwd(const SelectiveParams &P, const Shape &s, bool half, bool summary, cudaStream_t st)
{
    const dim3 grid((unsigned)(P.G * P.blocks * P.seq.B), (unsigned)(summary ? P.S - 1 : P.S));
    if (summary) return status_of(launch<true>(half ? pick_summary<bf16>(s) : pick_summary<float>(s), grid, dim3(32 * s.nl), 0, st, P));
    return half ? (P.z != nullptr ? run<bf16, true>(P, s, grid, st) : run<bf16, false>(P, s, grid, st))
                : (P.z != nullptr ? run<float, true>(P, s, grid, st) : run<float, false>(P, s, grid, st));
}

int launch_selective_bc(const SelectiveParams &P, bool half, void *grad_b, void *grad_c, cudaStream_t st)
{
    const long long tiles = ceil_div(P.seq.L, 32);
    const dim3 grid((unsigned)(tiles * P.seq.B), (unsigned)P.G);
    return half ? status_of(launch<true>(selective_bc_kernel<bf16>, grid, dim3(256), 0, st, P, static_cast<bf16 *>(grad_b), static_cast<bf16 *>(grad_c), tiles))
                : status_of(launch<true>(selective_bc_kernel<float>, grid, dim3(256), 0, st, P, static_cast<float *>(grad_b), static_cast<float *>(grad_c), tiles));
}

}  // namespace cawn
