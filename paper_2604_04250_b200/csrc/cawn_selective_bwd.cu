// Selective scan, backward.
//
// Mathematics, with w_t = e^{d_t A} h_{t-1} and dy' = dy silu(z): going back in time
//   lam_t = C_t dy'_t + e^{d_{t+1} A} lam_{t+1},   dB_t = sum_c lam d x,  dC_t = sum_c dy' h_t,  flow = sum_n lam B,
//   dx = d flow + skip dy',   dd = sum_n lam w A + x flow,   ddt = dd sigmoid(dt + bias),   dA = sum_t lam w d,
//   dz = dy (sum_n C h + skip x) silu'(z).
// A walk takes tiles of 16 tokens from the last to the first.  A tile's first state is a checkpoint; the states in front of
// each four tokens are found from it, and then w and the decays of four tokens stay in registers while the walk turns
// round.  So a decay's exponential is taken 1.75 times; the bound is what shared memory and the issue slots give.
// Sums over states go by shuffles.  Sums over channels (dB, dC) go through the tensor cores: the left factor is a selection,
// ones in row t (and 8 + t) and zeros elsewhere, so that one product adds four lanes' lam d x to row t and their dy' h to
// row 8 + t, for eight groups of lanes at once.  Operands: with bfloat16 storage the leading 8 and the next 8 bits of a term
// side by side (m16n8k16; the rest, 2^-16 of a term, is an eighth of a percent of the result's own rounding; with one operand of 11
// bits, gradients of rows that a few channels cancel in were off by twice their rounding); with float storage 11 and 11 bits in two
// products (m16n8k8).
#include "cawn_selective.cuh"

namespace cawn {
namespace {

// d: rows t and 8 + t gain u and v of four lanes; `one`: what a lane holds of the selection of t.
template <class T> __device__ __forceinline__ void sum_channels(float (&d)[4], unsigned one, float u, float v);
template <> __device__ __forceinline__ void sum_channels<bf16>(float (&d)[4], unsigned one, float u, float v)
{
    // upper half of a register: the leading bits; lower half: those of what is left
    const unsigned a = __float_as_uint(u) & 0xffff0000u, b = __float_as_uint(v) & 0xffff0000u;
    const unsigned x = __byte_perm(__float_as_uint(u - __uint_as_float(a)), a, 0x7632), y = __byte_perm(__float_as_uint(v - __uint_as_float(b)), b, 0x7632);
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%5,%4}, {%6,%7}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(one), "r"(0u), "r"(x), "r"(y));
}
template <> __device__ __forceinline__ void sum_channels<float>(float (&d)[4], unsigned one, float u, float v)
{
    const unsigned a = __float_as_uint(u) & 0xffffe000u, b = __float_as_uint(v) & 0xffffe000u;
    const unsigned x = __float_as_uint(u - __uint_as_float(a)) & 0xffffe000u, y = __float_as_uint(v - __uint_as_float(b)) & 0xffffe000u;
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%5,%4}, {%6,%7}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(one), "r"(0u), "r"(a), "r"(b));
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%5,%4}, {%6,%7}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(one), "r"(0u), "r"(x), "r"(y));
}

template <class T, int NL, int NS, int CD> struct BwdShared {
    using At = Place<NL, NS, CD>;
    static constexpr int kRow = 40, kWarps = At::kThreads / 32;
    float2 dd[kTile][kScanChannels];
    float bc[2][kTile][At::kPad];
    float dy[kTile][kRow];
    float sums[3][kTile][kRow];             // flow, drift (sum of lam w A log2 e), read-out
    float red[2][kWarps][NS * 2 * 64];      // [state of a lane][dB, dC][token of eight][group of lanes]
    float param[2][At::kStagers][8];        // grad_skip, grad_dt_bias of a stager's channels
    float bias[kScanChannels], skip[kScanChannels];
    struct { Eight<T> x, dt, z, gy; } words[At::kWords][At::kStagers];      // a stager's own, from staging to output
};

template <class T, int NL, int NS, int CD, bool GATE>
__global__ void __launch_bounds__(32 * NL / CD) selective_bwd_kernel(const SelectiveParams P)
{
    follow_previous();
    using At = Place<NL, NS, CD>;
    using Shared = BwdShared<T, NL, NS, CD>;
    constexpr int kThreads = At::kThreads, NP = At::kPad, NK = At::kPairs, kRow = Shared::kRow, kWords = At::kWords, kStagers = At::kStagers;
    constexpr int TS = 4, kSubs = kTile / TS;       // tokens whose decays stay in registers
    extern __shared__ __align__(16) unsigned char raw_shared[];
    Shared &sh = *reinterpret_cast<Shared *>(raw_shared);

    const At at;
    const int tid = threadIdx.x, lane = tid % 32, cb = blockIdx.x % (P.G * P.blocks), b = blockIdx.x / (P.G * P.blocks), g = cb / P.blocks;
    const int c0 = g * P.Dg + cb % P.blocks * kScanChannels;
    const int nch = min(kScanChannels, (g + 1) * P.Dg - c0), seg = blockIdx.y;
    const Span s = span_of(P.seq, b);
    const long long begin = seg * P.per, end = s.len < begin + P.per ? s.len : begin + P.per;
    const int n0 = at.nl * NS;
    float *param = P.part_param + ((long long)b * P.S + seg) * P.param_cols;

    f32x2 A2[CD][NK], carry[CD][NK], dA[CD][NK];
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const int c = c0 + at.ch + j;
        load_states<NS>(A2[j], P.A + (long long)c * P.N, n0, P.N, in);
        load_states<NS>(carry[j], P.gstate_out + ((long long)b * P.D + c) * P.N, n0, P.N, in && P.gstate_out != nullptr);
#pragma unroll
        for (int k = 0; k < NK; k++) {
            A2[j][k] = mul2(A2[j][k], twice(kLog2e));
            dA[j][k] = 0ull;
        }
        for (long long i = (s.len - 1) / P.per; i > seg; i--) fold_segment<NS>(carry[j], P, A2[j], ((long long)b * (P.S - 1) + i - 1) * P.D + c, n0, in);
    }
    for (int i = tid; i < kScanChannels; i += kThreads) {
        sh.bias[i] = i < nch && P.dt_bias != nullptr ? P.dt_bias[c0 + i] : 0.f;
        sh.skip[i] = i < nch && P.skip != nullptr ? P.skip[c0 + i] : 0.f;
    }
    for (int i = tid; i < 2 * kStagers * 8; i += kThreads) (&sh.param[0][0][0])[i] = 0.f;

    const T *x = static_cast<const T *>(P.x) + s.begin * P.xs + c0, *dt = static_cast<const T *>(P.dt) + s.begin * P.dts + c0;
    const T *z = GATE ? static_cast<const T *>(P.z) + s.begin * P.zs + c0 : nullptr, *gy = static_cast<const T *>(P.gy) + s.begin * P.D + c0;
    const int word = tid % 4 * 8, quad_row = tid / (NP / 4), quad = tid % (NP / 4) * 4;
    const T *bm = static_cast<const T *>(P.bm) + (s.begin + quad_row) * P.bs + g * P.N + quad, *cm = static_cast<const T *>(P.cm) + (s.begin + quad_row) * P.cs + g * P.N + quad;
    const float *marks = P.checkpoints + (checkpoint_of(s, b) * P.D + c0 + at.ch) * P.N;
    T *gx = static_cast<T *>(P.gx) + s.begin * P.D + c0, *gdt = static_cast<T *>(P.gdt) + s.begin * P.D + c0;
    T *gz = GATE ? static_cast<T *>(P.gz) + s.begin * P.D + c0 : nullptr;
    float *bc_out = P.part_bc + ((long long)cb * P.seq.rows + s.begin) * 2 * P.N;
    Eight<T> nx[kWords], ndt[kWords], nz[kWords], ngy[kWords];
    Quad<T> nb, nc;
    f32x2 nh[CD][NK];
    auto fetch = [&](long long t0) {
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const long long r = t0 + tid / 4 + i * (kStagers / 4);
            const int n = tid < kStagers && r < end ? nch - word : 0;
            nx[i] = fetch_eight(x + r * P.xs + word, n, P.whole_x);
            ndt[i] = fetch_eight(dt + r * P.dts + word, n, P.whole_dt);
            if (GATE) nz[i] = fetch_eight(z + r * P.zs + word, n, P.whole_z);
            ngy[i] = fetch_eight(gy + r * P.D + word, n, P.whole_d);
        }
        const int left = t0 + quad_row < end ? P.N - quad : 0;
        nb = fetch_quad(bm + t0 * P.bs, left, P.whole_b);
        nc = fetch_quad(cm + t0 * P.cs, left, P.whole_c);
#pragma unroll
        for (int j = 0; j < CD; j++) load_states<NS>(nh[j], marks + (t0 / kTile * P.D + j) * P.N, n0, P.N, at.ch + j < nch);
    };
    const long long last = begin + (end - 1 - begin) / kTile * kTile;
    if (end > begin) fetch(last);
    int buf = 0;
    for (long long t0 = last; t0 >= begin && end > begin; t0 -= kTile) {
        __syncthreads();
        if (tid < kStagers) {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const int r = tid / 4 + i * (kStagers / 4);
                float xf[8], df[8], gf[8], zf[8];
                nx[i].widen_to(xf);
                ndt[i].widen_to(df);
                ngy[i].widen_to(gf);
                auto &own = sh.words[i][tid];
                own.x = nx[i];
                own.dt = ndt[i];
                own.gy = ngy[i];
                if (GATE) {
                    nz[i].widen_to(zf);
                    own.z = nz[i];
                }
                const bool there = t0 + r < end;
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const f32x2 raw = add2(pair(df[j], df[j + 1]), *reinterpret_cast<const f32x2 *>(&sh.bias[word + j]));
                    const float2 d = halves(P.softplus ? softplus_of(raw) : raw);
                    *reinterpret_cast<float4 *>(&sh.dd[r][word + j]) = there ? make_float4(d.x, d.x * xf[j], d.y, d.y * xf[j + 1]) : make_float4(0.f, 0.f, 0.f, 0.f);
                    f32x2 dy = pair(gf[j], gf[j + 1]);
                    if (GATE) dy = mul2(dy, mul2(pair(zf[j], zf[j + 1]), sigmoid_of(pair(zf[j], zf[j + 1]))));
                    *reinterpret_cast<f32x2 *>(&sh.dy[r][word + j]) = dy;
                }
            }
        }
        *reinterpret_cast<float4 *>(&sh.bc[0][quad_row][quad]) = nb.get();
        *reinterpret_cast<float4 *>(&sh.bc[1][quad_row][quad]) = nc.get();
        f32x2 hs[kSubs][CD][NK];                        // the states in front of each four tokens
#pragma unroll
        for (int j = 0; j < CD; j++)
#pragma unroll
            for (int k = 0; k < NK; k++) hs[0][j][k] = nh[j][k];
        __syncthreads();
        if (t0 > begin) fetch(t0 - kTile);
        auto token = [&](float2 (&d)[CD], int t) {
            if constexpr (CD == 2) {
                const float4 v = *reinterpret_cast<const float4 *>(&sh.dd[t][at.ch]);
                d[0] = make_float2(v.x, v.y);
                d[CD - 1] = make_float2(v.z, v.w);
            } else {
                d[0] = sh.dd[t][at.ch];
            }
        };
#pragma unroll
        for (int u = 0; u + 1 < kSubs; u++) {
#pragma unroll
            for (int j = 0; j < CD; j++)
#pragma unroll
                for (int k = 0; k < NK; k++) hs[u + 1][j][k] = hs[u][j][k];
#pragma unroll
            for (int i = 0; i < TS; i++) {
                float2 d[CD];
                f32x2 B[NK];
                token(d, u * TS + i);
                row_pairs<NS>(B, &sh.bc[0][u * TS + i][n0]);
#pragma unroll
                for (int j = 0; j < CD; j++)
#pragma unroll
                    for (int k = 0; k < NK; k++)
                        hs[u + 1][j][k] = fma2(exp2_pair(mul2(twice(d[j].x), A2[j][k])), hs[u + 1][j][k], mul2(twice(d[j].y), B[k]));
            }
        }
        float sums[NS][4];
#pragma unroll
        for (int u = kSubs - 1; u >= 0; u--) {
            const int t1 = u * TS;
            f32x2 a[TS][CD][NK], w[TS][CD][NK], h[CD][NK];
#pragma unroll
            for (int j = 0; j < CD; j++)
#pragma unroll
                for (int k = 0; k < NK; k++) h[j][k] = hs[u][j][k];
            float v[CD][TS];
#pragma unroll
            for (int i = 0; i < TS; i++) {
                float2 d[CD];
                f32x2 B[NK], C[NK];
                token(d, t1 + i);
                row_pairs<NS>(B, &sh.bc[0][t1 + i][n0]);
                if constexpr (GATE) row_pairs<NS>(C, &sh.bc[1][t1 + i][n0]);
#pragma unroll
                for (int j = 0; j < CD; j++) {
                    f32x2 acc = 0ull;
#pragma unroll
                    for (int k = 0; k < NK; k++) {
                        a[i][j][k] = exp2_pair(mul2(twice(d[j].x), A2[j][k]));
                        w[i][j][k] = mul2(a[i][j][k], h[j][k]);
                        h[j][k] = fma2(twice(d[j].y), B[k], w[i][j][k]);
                        if constexpr (GATE) acc = k == 0 ? mul2(h[j][k], C[k]) : fma2(h[j][k], C[k], acc);
                    }
                    if constexpr (GATE) v[j][i] = sum_of(acc);
                }
            }
            if constexpr (GATE) {
#pragma unroll
                for (int j = 0; j < CD; j++) sum_four<NL>(v[j], at.nl, &sh.sums[2][t1][at.ch + j], kRow);
            }
            if (u % 2 == 1) {
#pragma unroll
                for (int k = 0; k < NS; k++) sums[k][0] = sums[k][1] = sums[k][2] = sums[k][3] = 0.f;
            }
            float flow[CD][TS], drift[CD][TS];
#pragma unroll
            for (int i = TS - 1; i >= 0; i--) {
                const int t = t1 + i;
                float2 d[CD];
                f32x2 B[NK], C[NK], gb[NK], gc[NK];
                token(d, t);
                row_pairs<NS>(B, &sh.bc[0][t][n0]);
                row_pairs<NS>(C, &sh.bc[1][t][n0]);
#pragma unroll
                for (int j = 0; j < CD; j++) {
                    const f32x2 dl = twice(d[j].x), dx = twice(d[j].y), dy = twice(sh.dy[t][at.ch + j]);
                    f32x2 fl = 0ull, dr = 0ull;
#pragma unroll
                    for (int k = 0; k < NK; k++) {
                        const f32x2 now = fma2(dx, B[k], w[i][j][k]), lam = fma2(C[k], dy, carry[j][k]), m = mul2(lam, w[i][j][k]);
                        fl = k == 0 ? mul2(lam, B[k]) : fma2(lam, B[k], fl);
                        dr = k == 0 ? mul2(m, A2[j][k]) : fma2(m, A2[j][k], dr);
                        dA[j][k] = fma2(m, dl, dA[j][k]);
                        carry[j][k] = mul2(a[i][j][k], lam);
                        gb[k] = j == 0 ? mul2(lam, dx) : fma2(lam, dx, gb[k]);
                        gc[k] = j == 0 ? mul2(now, dy) : fma2(now, dy, gc[k]);
                    }
                    flow[j][i] = sum_of(fl);
                    drift[j][i] = sum_of(dr);
                }
                const unsigned one = lane >> 2 == t % 8 ? (sizeof(T) == 2 ? 0x3f803f80u : 0x3f800000u) : 0u;
#pragma unroll
                for (int k = 0; k < NK; k++) {
                    const float2 p = halves(gb[k]), q = halves(gc[k]);
                    sum_channels<T>(sums[2 * k], one, p.x, q.x);
                    sum_channels<T>(sums[2 * k + 1], one, p.y, q.y);
                }
            }
#pragma unroll
            for (int j = 0; j < CD; j++) {
                sum_four<NL>(flow[j], at.nl, &sh.sums[0][t1][at.ch + j], kRow);
                sum_four<NL>(drift[j], at.nl, &sh.sums[1][t1][at.ch + j], kRow);
            }
            if (u % 2 == 0) {
                // rows of a selection's result: eight tokens; columns: the groups of lanes that a lane / 4 names
                float *red = sh.red[buf][tid / 32] + lane * 2;
#pragma unroll
                for (int k = 0; k < NS; k++) {
                    *reinterpret_cast<float2 *>(red + k * 128) = make_float2(sums[k][0], sums[k][1]);
                    *reinterpret_cast<float2 *>(red + k * 128 + 64) = make_float2(sums[k][2], sums[k][3]);
                }
                __syncthreads();
                // warps, and groups of channels in a warp, in their order; neighbours take neighbouring lane groups
                for (int o = tid; o < 16 * NP; o += kThreads) {
                    const int nl = o % NL, i = o / NL % 8, m = o / (NL * 8) % 2, k = o / (NL * 16), n = nl * NS + k;
                    float sum = 0.f;
#pragma unroll
                    for (int r = 0; r < Shared::kWarps; r++)
#pragma unroll
                        for (int q = 0; q < 8; q += NL) sum += sh.red[buf][r][((k * 2 + m) * 8 + i) * 8 + q + nl];
                    if (n < P.N && t0 + t1 + i < end) bc_out[((t0 + t1 + i) * 2 + m) * P.N + n] = sum;
                }
                buf ^= 1;
            }
        }
        if (tid < kStagers) {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const int r = tid / 4 + i * (kStagers / 4);
                if (t0 + r >= end) break;
                const auto &own = sh.words[i][tid];
                float xf[8], df[8], gf[8], zf[8], ox[8], od[8], oz[8];
                own.x.widen_to(xf);
                own.dt.widen_to(df);
                own.gy.widen_to(gf);
                if (GATE) own.z.widen_to(zf);
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    auto two = [&](const float *p) { return *reinterpret_cast<const f32x2 *>(p + word + j); };
                    const float4 d = *reinterpret_cast<const float4 *>(&sh.dd[r][word + j]);
                    const f32x2 xx = pair(xf[j], xf[j + 1]), fl = two(sh.sums[0][r]), skip = two(sh.skip), dy = two(sh.dy[r]);
                    const f32x2 raw = add2(pair(df[j], df[j + 1]), two(sh.bias));
                    f32x2 o = fma2(pair(d.x, d.z), fl, mul2(skip, dy));
                    float2 v = halves(o);
                    ox[j] = v.x; ox[j + 1] = v.y;
                    o = fma2(two(sh.sums[1][r]), twice(kLn2), mul2(xx, fl));
                    if (P.softplus) o = mul2(o, sigmoid_of(raw));
                    v = halves(o);
                    od[j] = v.x; od[j + 1] = v.y;
                    if (GATE) {
                        const f32x2 zz = pair(zf[j], zf[j + 1]), sg = sigmoid_of(zz), one = twice(1.f);
                        const f32x2 slope = mul2(sg, fma2(zz, fma2(sg, twice(-1.f), one), one));
                        v = halves(mul2(mul2(pair(gf[j], gf[j + 1]), slope), fma2(skip, xx, two(sh.sums[2][r]))));
                        oz[j] = v.x; oz[j + 1] = v.y;
                    }
                    f32x2 *acc = reinterpret_cast<f32x2 *>(&sh.param[0][tid][j]);
                    *acc = fma2(dy, xx, *acc);
                    acc = reinterpret_cast<f32x2 *>(&sh.param[1][tid][j]);
                    *acc = add2(o, *acc);
                }
                store_eight(gx + (t0 + r) * P.D + word, ox, nch - word, P.whole_d);
                store_eight(gdt + (t0 + r) * P.D + word, od, nch - word, P.whole_d);
                if (GATE) store_eight(gz + (t0 + r) * P.D + word, oz, nch - word, P.whole_d);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const int c = c0 + at.ch + j;
        if (seg == 0 && P.gstate_in != nullptr) store_states<NS>(P.gstate_in + ((long long)b * P.D + c) * P.N, carry[j], n0, P.N, in);
        store_states<NS>(param + (long long)c * P.N, dA[j], n0, P.N, in);
    }
    __syncthreads();
    for (int i = tid; i < 2 * nch; i += kThreads) {
        const int m = i / nch, ch = i % nch;
        float sum = 0.f;
        for (int r = ch / 8; r < kStagers; r += 4) sum += sh.param[m][r][ch % 8];
        param[(long long)P.D * (P.N + m) + c0 + ch] = sum;
    }
}

// A segment's own gradient at its start, and its sum of d: for the segments in front of it.
template <class T, int NL, int NS, int CD>
__global__ void __launch_bounds__(32 * NL / CD) selective_bwd_summary_kernel(const SelectiveParams P)
{
    follow_previous();
    using At = Place<NL, NS, CD>;
    constexpr int kThreads = At::kThreads, NP = At::kPad, NK = At::kPairs, kWords = At::kWords, kStagers = At::kStagers;
    __shared__ __align__(16) float2 dd[kTile][kScanChannels];           // d, dy'
    __shared__ __align__(16) float cs[kTile][NP];
    __shared__ __align__(16) float bias[kScanChannels];
    const At at;
    const int tid = threadIdx.x, cb = blockIdx.x % (P.G * P.blocks), b = blockIdx.x / (P.G * P.blocks), g = cb / P.blocks;
    const int c0 = g * P.Dg + cb % P.blocks * kScanChannels;
    const int nch = min(kScanChannels, (g + 1) * P.Dg - c0), seg = blockIdx.y + 1;
    const Span s = span_of(P.seq, b);
    const long long begin = seg * P.per, end = s.len < begin + P.per ? s.len : begin + P.per;
    if (begin >= s.len) return;
    const int n0 = at.nl * NS;
    f32x2 A2[CD][NK], own[CD][NK], past[CD][NK];
#pragma unroll
    for (int j = 0; j < CD; j++) {
        load_states<NS>(A2[j], P.A + (long long)(c0 + at.ch + j) * P.N, n0, P.N, at.ch + j < nch);
#pragma unroll
        for (int k = 0; k < NK; k++) {
            A2[j][k] = mul2(A2[j][k], twice(kLog2e));
            own[j][k] = 0ull;
            past[j][k] = twice(1.f);
        }
    }
    for (int i = tid; i < kScanChannels; i += kThreads) bias[i] = i < nch && P.dt_bias != nullptr ? P.dt_bias[c0 + i] : 0.f;
    const T *dt = static_cast<const T *>(P.dt) + s.begin * P.dts + c0, *gy = static_cast<const T *>(P.gy) + s.begin * P.D + c0;
    const T *z = P.z != nullptr ? static_cast<const T *>(P.z) + s.begin * P.zs + c0 : nullptr;
    const int word = tid % 4 * 8, quad_row = tid / (NP / 4), quad = tid % (NP / 4) * 4;
    const T *cm = static_cast<const T *>(P.cm) + (s.begin + quad_row) * P.cs + g * P.N + quad;
    Eight<T> ndt[kWords], ngy[kWords], nz[kWords];
    Quad<T> nc;
    auto fetch = [&](long long t0) {
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const long long r = t0 + tid / 4 + i * (kStagers / 4);
            const int n = tid < kStagers && r < end ? nch - word : 0;
            ndt[i] = fetch_eight(dt + r * P.dts + word, n, P.whole_dt);
            ngy[i] = fetch_eight(gy + r * P.D + word, n, P.whole_d);
            if (z != nullptr) nz[i] = fetch_eight(z + r * P.zs + word, n, P.whole_z);
        }
        nc = fetch_quad(cm + t0 * P.cs, t0 + quad_row < end ? P.N - quad : 0, P.whole_c);
    };
    fetch(begin);
    float time[CD] = {};
    for (long long t0 = begin; t0 < end; t0 += kTile) {
        __syncthreads();
        if (tid < kStagers) {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const int r = tid / 4 + i * (kStagers / 4);
                float df[8], gf[8], zf[8];
                ndt[i].widen_to(df);
                ngy[i].widen_to(gf);
                if (z != nullptr) nz[i].widen_to(zf);
                const bool there = t0 + r < end;
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const f32x2 raw = add2(pair(df[j], df[j + 1]), *reinterpret_cast<const f32x2 *>(&bias[word + j]));
                    const float2 d = halves(P.softplus ? softplus_of(raw) : raw);
                    f32x2 dy = pair(gf[j], gf[j + 1]);
                    if (z != nullptr) dy = mul2(dy, mul2(pair(zf[j], zf[j + 1]), sigmoid_of(pair(zf[j], zf[j + 1]))));
                    const float2 e = halves(dy);
                    *reinterpret_cast<float4 *>(&dd[r][word + j]) = there ? make_float4(d.x, e.x, d.y, e.y) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            }
        }
        *reinterpret_cast<float4 *>(&cs[quad_row][quad]) = nc.get();
        __syncthreads();
        if (t0 + kTile < end) fetch(t0 + kTile);
#pragma unroll 4
        for (int t = 0; t < kTile; t++) {
            f32x2 C[NK];
            row_pairs<NS>(C, &cs[t][n0]);
#pragma unroll
            for (int j = 0; j < CD; j++) {
                const float2 d = dd[t][at.ch + j];
                time[j] += d.x;
#pragma unroll
                for (int k = 0; k < NK; k++) {
                    past[j][k] = mul2(past[j][k], exp2_pair(mul2(twice(d.x), A2[j][k])));
                    own[j][k] = fma2(past[j][k], mul2(C[k], twice(d.y)), own[j][k]);
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const long long segment = ((long long)b * (P.S - 1) + seg - 1) * P.D + c0 + at.ch + j;
        store_states<NS>(P.seg_state + segment * P.N, own[j], n0, P.N, in);
        if (in && at.nl == 0) P.seg_time[segment] = time[j];
    }
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

template <class T, bool GATE, int NL, int NS, int CD> int run(const SelectiveParams &P, dim3 grid, cudaStream_t st)
{
    constexpr size_t bytes = sizeof(BwdShared<T, NL, NS, CD>);
    auto k = selective_bwd_kernel<T, NL, NS, CD, GATE>;
    if (bytes > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != cudaSuccess) return status_of(e);
    }
    return status_of(launch<true>(k, grid, dim3(32 * NL / CD), bytes, st, P));
}
template <class T, bool GATE> int run(const SelectiveParams &P, const Shape &s, dim3 grid, cudaStream_t st)
{
#define CAWN_CALL(NL, NS, CD) run<T, GATE, NL, NS, CD>(P, grid, st)
    return CAWN_BY_SHAPE(s, CAWN_CALL);
#undef CAWN_CALL
}
template <class T> SelectiveKernel pick_summary(const Shape &s)
{
#define CAWN_CALL(NL, NS, CD) selective_bwd_summary_kernel<T, NL, NS, CD>
    return CAWN_BY_SHAPE(s, CAWN_CALL);
#undef CAWN_CALL
}

}  // namespace

int launch_selective_bwd(const SelectiveParams &P, const Shape &s, bool half, bool summary, cudaStream_t st)
{
    const dim3 grid((unsigned)(P.G * P.blocks * P.seq.B), (unsigned)(summary ? P.S - 1 : P.S));
    if (summary) return status_of(launch<true>(half ? pick_summary<bf16>(s) : pick_summary<float>(s), grid, dim3(32 * s.warps()), 0, st, P));
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
