// Selective scan, backward.
//
// Mathematics, with w_t = e^{d_t A} h_{t-1} and dy' = dy silu(z): going back in time
//   lam_t = C_t dy'_t + e^{d_{t+1} A} lam_{t+1},   dB_t = sum_c lam d x,  dC_t = sum_c dy' h_t,  flow = sum_n lam B,
//   dx = d flow + skip dy',   dd = sum_n lam w A + x flow,   ddt = dd sigmoid(dt + bias),   dA = sum_t lam w d,
//   dz = dy (sum_n C h + skip x) silu'(z).
// A walk takes tiles of 16 tokens from the last to the first, a tile as two halves.  A tile's first state is a checkpoint; the
// states in front of each four tokens are found from it, and then w and the decays of four tokens stay in registers while
// the walk turns round.  So a decay's exponential is taken 1.75 times.  Those registers (some 250 a thread) are why every warp here
// does all of the work, two a scheduler, where the forward has warps of two kinds: lanes leave sums over their own states in
// shared memory, and when half a tile is done all threads add them up, finish and store.
// Sums over channels (dB, dC) go through the tensor cores: the left factor is a selection, ones in row t (and 8 + t) and
// zeros elsewhere, so that one product adds four lanes' lam d x to row t and their dy' h to row 8 + t, for eight groups of
// lanes at once.  Operands: a term in three bfloat16 parts of eight bits, which hold all of a float's 24; two of them in one product
// (m16n8k16), the third in another (m16n8k8).  (With two parts, 16 bits, results in bfloat16 were off by 2e-4 of their norm.)
// Bound: the latency of those chains with eight warps a multiprocessor.  8 x 2048 x 1024 x 16 bfloat16 with the gate: walk 581 us
// (issue 39%, shared memory 45%, exponentials 24%, tensor cores 11%; with two parts a term 545), the pass before its two segments 63, the
// sums of dB and dC 18.  In float, six warps a multiprocessor by shared memory: walk 862.
#include "cawn_selective.cuh"

namespace cawn {
namespace {

// Rows t and 8 + t of d0 gain u.x and v.x of four lanes, those of d1 u.y and v.y; `here`: this lane's row of the selection is t.
__device__ __forceinline__ void sum_channels(float (&d0)[4], float (&d1)[4], bool here, f32x2 u, f32x2 v)
{
    // What a term is beyond its first eight bits, and beyond those the next eight: what is left then has no more than eight.
    auto lead = [](f32x2 a) { return a & 0xffff0000ffff0000ull; };
    auto rest = [&](f32x2 a) { return fma2(lead(a), twice(-1.f), a); };
    const f32x2 ur = rest(u), vr = rest(v), ul = rest(ur), vl = rest(vr);
    const unsigned both = here ? 0x3f803f80u : 0u, low = both & 0xffffu, high = both & 0xffff0000u;
    auto add = [&](float (&d)[4], float u0, float v0, float u1, float v1, float u2, float v2) {
        // upper half of a register: the leading bits; lower half: the next ones
        const unsigned x = __byte_perm(__float_as_uint(u1), __float_as_uint(u0), 0x7632), y = __byte_perm(__float_as_uint(v1), __float_as_uint(v0), 0x7632);
        const unsigned z = __byte_perm(__float_as_uint(u2), __float_as_uint(v2), 0x7632);           // the last bits: u's, and v's above
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%5,%4}, {%6,%7}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(both), "r"(0u), "r"(x), "r"(y));
        asm("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(low), "r"(high), "r"(z));
    };
    const float2 a = halves(u), b = halves(v), ar = halves(ur), br = halves(vr), al = halves(ul), bl = halves(vl);
    add(d0, a.x, b.x, ar.x, br.x, al.x, bl.x);
    add(d1, a.y, b.y, ar.y, br.y, al.y, bl.y);
}

// Where a thread is: as in the forward's computing warps, and for staging and finishing.
template <int NL, int NS, int CD> struct Walker : Place<NL, NS, CD> {
    using At = Place<NL, NS, CD>;
    static constexpr int kThreads = At::kCompute, kWarps = kThreads / 32;
    static constexpr int kStagers = kThreads < 64 ? kThreads : 64, kWords = 64 / kStagers;     // words of eight channels of a tile
    static constexpr int kFinishers = kThreads < 64 ? kThreads : 64, kTurns = 64 / kFinishers;  // quads of channels of half a tile
    static_assert(kTile * At::kPad / 4 == kThreads, "a quad of B and one of C for each thread");
};

template <class T, int NL, int NS, int CD> struct BwdShared {
    using At = Walker<NL, NS, CD>;
    float2 dd[2][kTile][kRowPairs];         // d, d x
    float dy[2][kTile][kRowFloats];         // dy'
    float bc[2][2][kTile][At::kPad];
    float parts[3][8][NL * kRowFloats + 8]; // flow, drift (sum of lam w A log2 e) and read-out, by lane of a channel
    float red[At::kWarps][NS * 2 * 64];     // [state of a lane][dB, dC][token of eight][group of lanes]
    float4 states[kTile / 4][CD * NS / 4][At::kThreads];    // a thread's own, in front of each four tokens
    Eight<T> words[2][4][kTile][4];         // x, dt, z, dy as they were fetched
    float bias[kScanChannels], skip[kScanChannels];
};

// Tokens of a segment's first half, whole tiles.
__device__ __forceinline__ long long half_of(long long per) { return (per / kTile + 1) / 2 * kTile; }

template <class T, int NL, int NS, int CD, bool GATE>
__global__ void __launch_bounds__(32 * NL / CD) selective_bwd_kernel(const SelectiveParams P)
{
    follow_previous();
    using At = Walker<NL, NS, CD>;
    using Shared = BwdShared<T, NL, NS, CD>;
    constexpr int NP = At::kPad, NK = At::kPairs, kThreads = At::kThreads;
    constexpr int TS = 4;       // tokens whose decays stay in registers
    extern __shared__ __align__(16) unsigned char raw_shared[];
    Shared &sh = *reinterpret_cast<Shared *>(raw_shared);

    const At at;
    const int tid = threadIdx.x, lane = tid % 32, cb = blockIdx.x % (P.G * P.blocks), b = blockIdx.x / (P.G * P.blocks), g = cb / P.blocks;
    const int c0 = g * P.Dg + cb % P.blocks * kScanChannels;
    const int nch = min(kScanChannels, (g + 1) * P.Dg - c0), seg = blockIdx.y;
    const Span s = span_of(P.seq, b);
    const long long begin = seg * P.per, end = s.len < begin + P.per ? s.len : begin + P.per;
    const int n0 = at.nl * NS;

    f32x2 A2[CD][NK], carry[CD][NK], dA[CD][NK];
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const int c = c0 + at.ch + j;
        load_states<NS>(A2[j], P.A + (long long)c * P.N, n0, P.N, in);
        load_states<NS>(carry[j], P.gstate_out + ((long long)b * P.D + c) * P.N, n0, P.N, in && P.gstate_out != nullptr);
#pragma unroll
        for (int k = 0; k < NK; k++) {
            A2[j][k] = rate_of(A2[j][k]);
            dA[j][k] = 0ull;
        }
        const long long behind = (s.len - 1) / P.per;           // the sequence's last segment
        const int end_of_all = (int)(behind - 1) * P.halves + (P.halves == 2 && s.len - 1 - behind * P.per >= half_of(P.per));
        fold_segments<NS>(carry[j], P, A2[j], (first_end(P, s, b) * P.halves + end_of_all) * P.D + c, -P.D, end_of_all - seg * P.halves + 1, n0, in);
    }
    for (int i = tid; i < kScanChannels; i += kThreads) {
        sh.bias[i] = i < nch && P.dt_bias != nullptr ? P.dt_bias[c0 + i] : 0.f;
        sh.skip[i] = i < nch && P.skip != nullptr ? P.skip[c0 + i] : 0.f;
    }

    const T *x = static_cast<const T *>(P.x) + s.begin * P.xs + c0, *dt = static_cast<const T *>(P.dt) + s.begin * P.dts + c0;
    const T *z = GATE ? static_cast<const T *>(P.z) + s.begin * P.zs + c0 : nullptr, *gy = static_cast<const T *>(P.gy) + s.begin * P.D + c0;
    const int word = tid % 4 * 8, quad_row = tid / (NP / 4), quad = tid % (NP / 4) * 4;
    const T *bm = static_cast<const T *>(P.bm) + (s.begin + quad_row) * P.bs + g * P.N + quad, *cm = static_cast<const T *>(P.cm) + (s.begin + quad_row) * P.cs + g * P.N + quad;
    const float *marks = P.checkpoints + (checkpoint_of(s, b) * P.D + c0 + at.ch) * P.N;
    Eight<T> nx[At::kWords], ndt[At::kWords], nz[At::kWords], ngy[At::kWords];
    Quad<T> nb, nc;
    f32x2 nh[CD][NK];
    auto fetch = [&](long long t0) {
#pragma unroll
        for (int i = 0; i < At::kWords; i++) {
            const long long r = t0 + tid / 4 + i * (At::kStagers / 4);
            const int n = tid < At::kStagers && r < end ? nch - word : 0;
            nx[i] = fetch_eight(x + r * P.xs + word, n, P.whole_x);
            ndt[i] = fetch_eight(dt + r * P.dts + word, n, P.whole_dt);
            if (GATE) nz[i] = fetch_eight(z + r * P.zs + word, n, P.whole_z);
            ngy[i] = fetch_eight(gy + r * P.D + word, n, P.whole_d);
        }
        const int left = t0 + quad_row < end ? P.N - quad : 0;
        nb = fetch_quad(bm + t0 * P.bs, left, P.whole_b);
        nc = fetch_quad(cm + t0 * P.cs, left, P.whole_c);
    };
    auto fetch_states = [&](long long t0) {
#pragma unroll
        for (int j = 0; j < CD; j++) load_states<NS>(nh[j], marks + (t0 / kTile * P.D + j) * P.N, n0, P.N, at.ch + j < nch);
    };
    auto stage = [&](long long t0, int to) {
        if (At::kStagers == kThreads || tid < At::kStagers) {
#pragma unroll
            for (int i = 0; i < At::kWords; i++) {
                const int r = tid / 4 + i * (At::kStagers / 4);
                float xf[8], df[8], gf[8], zf[8];
                nx[i].widen_to(xf);
                ndt[i].widen_to(df);
                ngy[i].widen_to(gf);
                sh.words[to][0][r][tid % 4] = nx[i];
                sh.words[to][1][r][tid % 4] = ndt[i];
                sh.words[to][3][r][tid % 4] = ngy[i];
                if constexpr (GATE) {
                    nz[i].widen_to(zf);
                    sh.words[to][2][r][tid % 4] = nz[i];
                }
                const bool there = t0 + r < end;
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const f32x2 xx = pair(xf[j], xf[j + 1]), raw = add2(pair(df[j], df[j + 1]), *reinterpret_cast<const f32x2 *>(&sh.bias[word + j]));
                    const f32x2 d = chosen(there, chosen(P.softplus, softplus_of(raw), raw), 0ull);
                    const float2 u = halves(d), v = halves(mul2(d, xx));
                    *reinterpret_cast<float4 *>(&sh.dd[to][r][slot_of(word) + j]) = make_float4(u.x, v.x, u.y, v.y);
                    f32x2 dy = pair(gf[j], gf[j + 1]);
                    if constexpr (GATE) dy = mul2(dy, mul2(pair(zf[j], zf[j + 1]), sigmoid_of(pair(zf[j], zf[j + 1]))));
                    *reinterpret_cast<f32x2 *>(&sh.dy[to][r][word + j]) = dy;
                }
            }
        }
        *reinterpret_cast<float4 *>(&sh.bc[to][0][quad_row][quad]) = nb.get();
        *reinterpret_cast<float4 *>(&sh.bc[to][1][quad_row][quad]) = nc.get();
    };
    // Half a tile: a thread has four channels of one row (or two rows).
    const int four = tid % 8 * 4;
    f32x2 gskip[2] = {}, gbias[2] = {};
    T *gx = static_cast<T *>(P.gx) + s.begin * P.D + c0 + four, *gdt = static_cast<T *>(P.gdt) + s.begin * P.D + c0 + four;
    T *gz = GATE ? static_cast<T *>(P.gz) + s.begin * P.D + c0 + four : nullptr;
    float *bc_out = P.part_bc + ((long long)cb * P.seq.rows + s.begin) * 2 * P.N;
    auto finish = [&](long long t0, int from, int half) {
        if (At::kFinishers == kThreads || tid < At::kFinishers) {
#pragma unroll
            for (int i = 0; i < At::kTurns; i++) {
                const int r8 = tid / 8 + i * (At::kFinishers / 8), r = half * 8 + r8;
                f32x2 sum[3][2];
#pragma unroll
                for (int m = 0; m < (GATE ? 3 : 2); m++)
#pragma unroll
                    for (int q = 0; q < NL; q++) {
                        const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(&sh.parts[m][r8][q * kRowFloats + four]);
                        sum[m][0] = q == 0 ? v.x : add2(sum[m][0], v.x);
                        sum[m][1] = q == 0 ? v.y : add2(sum[m][1], v.y);
                    }
                auto row = [&](int m) { return reinterpret_cast<const Quad<T> *>(&sh.words[from][m][r][0])[tid % 8].get(); };
                const float4 xf = row(0), df = row(1), gf = row(3), zf = GATE ? row(2) : xf;
                float ox[4], od[4], oz[4];
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const f32x2 xx = j == 0 ? pair(xf.x, xf.y) : pair(xf.z, xf.w), raw = add2(j == 0 ? pair(df.x, df.y) : pair(df.z, df.w), *reinterpret_cast<const f32x2 *>(&sh.bias[four + 2 * j]));
                    const f32x2 skip = *reinterpret_cast<const f32x2 *>(&sh.skip[four + 2 * j]), dy = *reinterpret_cast<const f32x2 *>(&sh.dy[from][r][four + 2 * j]);
                    const float4 d = *reinterpret_cast<const float4 *>(&sh.dd[from][r][slot_of(four) + 2 * j]);
                    float2 v = halves(fma2(pair(d.x, d.z), sum[0][j], mul2(skip, dy)));
                    ox[2 * j] = v.x;
                    ox[2 * j + 1] = v.y;
                    f32x2 o = fma2(sum[1][j], twice(kLn2), mul2(xx, sum[0][j]));
                    o = chosen(P.softplus, mul2(o, sigmoid_of(raw)), o);
                    v = halves(o);
                    od[2 * j] = v.x;
                    od[2 * j + 1] = v.y;
                    if (t0 + r < end) {
                        gskip[j] = fma2(dy, xx, gskip[j]);
                        gbias[j] = add2(gbias[j], o);
                    }
                    if constexpr (GATE) {
                        const f32x2 zz = j == 0 ? pair(zf.x, zf.y) : pair(zf.z, zf.w), gg = j == 0 ? pair(gf.x, gf.y) : pair(gf.z, gf.w), sg = sigmoid_of(zz), one = twice(1.f);
                        const f32x2 slope = mul2(sg, fma2(zz, fma2(sg, twice(-1.f), one), one));
                        v = halves(mul2(mul2(gg, slope), fma2(skip, xx, sum[2][j])));
                        oz[2 * j] = v.x;
                        oz[2 * j + 1] = v.y;
                    }
                }
                if (t0 + r < end) {
                    store_quad(gx + (t0 + r) * P.D, make_float4(ox[0], ox[1], ox[2], ox[3]), nch - four, P.whole_d);
                    store_quad(gdt + (t0 + r) * P.D, make_float4(od[0], od[1], od[2], od[3]), nch - four, P.whole_d);
                    if (GATE) store_quad(gz + (t0 + r) * P.D, make_float4(oz[0], oz[1], oz[2], oz[3]), nch - four, P.whole_d);
                }
            }
        }
        // dB, dC: warps, and groups of channels in a warp, in their order; neighbours take neighbouring groups of lanes
#pragma unroll
        for (int o = tid; o < 16 * NP; o += kThreads) {
            const int nl = o % NL, i = o / NL % 8, m = o / (NL * 8) % 2, k = o / (NL * 16), n = nl * NS + k;
            const long long t = t0 + half * 8 + i;
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < At::kWarps; r++)
#pragma unroll
                for (int q = 0; q < 8; q += NL) sum += sh.red[r][((k * 2 + m) * 8 + i) * 8 + q + nl];
            if (n < P.N && t < end) bc_out[(t * 2 + m) * P.N + n] = sum;
        }
    };
    const long long last = begin + (end - 1 - begin) / kTile * kTile;
    __syncthreads();            // bias, skip
    if (end > begin) {
        fetch(last);
        fetch_states(last);
        stage(last, 0);
        if (last > begin) fetch(last - kTile);
    }
    const int slot = slot_of(at.ch);
    int buf = 0;
    for (long long t0 = last; t0 >= begin && end > begin; t0 -= kTile, buf ^= 1) {
        __syncthreads();        // this tile is staged, and the one behind it is finished
        f32x2 h[CD][NK];
#pragma unroll
        for (int j = 0; j < CD; j++)
#pragma unroll
            for (int k = 0; k < NK; k++) h[j][k] = nh[j][k];
        if (t0 > begin) {
            fetch_states(t0 - kTile);
            stage(t0 - kTile, buf ^ 1);
            if (t0 - kTile > begin) fetch(t0 - 2 * kTile);
        }
#pragma unroll 1
        for (int u = 0; u < kTile / TS; u++) {
#pragma unroll
            for (int j = 0; j < CD; j++)
#pragma unroll
                for (int k = 0; k < NK; k += 2) {
                    const float2 p = halves(h[j][k]), q = halves(h[j][k + 1]);
                    sh.states[u][(j * NK + k) / 2][tid] = make_float4(p.x, p.y, q.x, q.y);
                }
            if (u == kTile / TS - 1) break;
#pragma unroll
            for (int i = 0; i < TS; i++) {
                float2 d[CD];
                f32x2 B[NK];
                two_of<CD>(d, &sh.dd[buf][u * TS + i][slot]);
                row_pairs<NS>(B, &sh.bc[buf][0][u * TS + i][n0]);
#pragma unroll
                for (int j = 0; j < CD; j++)
#pragma unroll
                    for (int k = 0; k < NK; k++) h[j][k] = fma2(exp2_pair(mul2(twice(d[j].x), A2[j][k])), h[j][k], mul2(twice(d[j].y), B[k]));
            }
        }
        // Eight tokens, then the eight before them, four at a time.
#pragma unroll 1
        for (int half = 1; half >= 0; half--) {
            float sums[NS][4] = {};
#pragma unroll 1
            for (int u = 1; u >= 0; u--) {
                const int t1 = half * 8 + u * TS;
                f32x2 a[TS][CD][NK], w[TS][CD][NK];
#pragma unroll
                for (int j = 0; j < CD; j++)
#pragma unroll
                    for (int k = 0; k < NK; k += 2) {
                        const float4 f = sh.states[t1 / TS][(j * NK + k) / 2][tid];
                        h[j][k] = pair(f.x, f.y);
                        h[j][k + 1] = pair(f.z, f.w);
                    }
#pragma unroll
                for (int i = 0; i < TS; i++) {
                    float out[CD];
                    float2 d[CD];
                    f32x2 B[NK], C[NK];
                    two_of<CD>(d, &sh.dd[buf][t1 + i][slot]);
                    row_pairs<NS>(B, &sh.bc[buf][0][t1 + i][n0]);
                    if constexpr (GATE) row_pairs<NS>(C, &sh.bc[buf][1][t1 + i][n0]);
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
                        if constexpr (GATE) out[j] = sum_of(acc);
                    }
                    if constexpr (GATE) put_channels<CD>(&sh.parts[2][u * TS + i][at.nl * kRowFloats + at.ch], out);
                }
#pragma unroll
                for (int i = TS - 1; i >= 0; i--) {
                    const int t = t1 + i;
                    float2 d[CD];
                    float e[CD], flow[CD], drift[CD];
                    f32x2 B[NK], C[NK], gb[NK], gc[NK];
                    two_of<CD>(d, &sh.dd[buf][t][slot]);
                    get_channels<CD>(e, &sh.dy[buf][t][at.ch]);
                    row_pairs<NS>(B, &sh.bc[buf][0][t][n0]);
                    row_pairs<NS>(C, &sh.bc[buf][1][t][n0]);
#pragma unroll
                    for (int j = 0; j < CD; j++) {
                        const f32x2 dl = twice(d[j].x), dx = twice(d[j].y), dy = twice(e[j]);
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
                        flow[j] = sum_of(fl);
                        drift[j] = sum_of(dr);
                    }
                    put_channels<CD>(&sh.parts[0][u * TS + i][at.nl * kRowFloats + at.ch], flow);
                    put_channels<CD>(&sh.parts[1][u * TS + i][at.nl * kRowFloats + at.ch], drift);
                    const bool here = lane >> 2 == u * TS + i;
#pragma unroll
                    for (int k = 0; k < NK; k++) sum_channels(sums[2 * k], sums[2 * k + 1], here, gb[k], gc[k]);
                }
            }
            // rows of a selection's result: eight tokens; columns: the groups of lanes that a lane / 4 names
            float *red = sh.red[tid / 32] + lane * 2;
#pragma unroll
            for (int k = 0; k < NS; k++) {
                *reinterpret_cast<float2 *>(red + k * 128) = make_float2(sums[k][0], sums[k][1]);
                *reinterpret_cast<float2 *>(red + k * 128 + 64) = make_float2(sums[k][2], sums[k][3]);
            }
            __syncthreads();
            finish(t0, buf, half);
            if (half == 1) __syncthreads();
        }
    }
    // found again, so that nothing of it is kept while the walk needs every register (float, 8 x 2048 x 1024 x 16: 1155 -> 1097 us)
    const int sequence = blockIdx.x / (P.G * P.blocks);
    const Span own = span_of(P.seq, sequence);
    if (P.by_rows && blockIdx.y > 0 && blockIdx.y * P.per >= own.len) return;       // no row is theirs
    float *param = P.part_param + param_row(P, own, sequence, blockIdx.y) * P.param_cols;
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const int c = c0 + at.ch + j;
        if (seg == 0 && P.gstate_in != nullptr) store_states<NS>(P.gstate_in + ((long long)b * P.D + c) * P.N, carry[j], n0, P.N, in);
        store_states<NS>(param + (long long)c * P.N, dA[j], n0, P.N, in);
    }
    // a channel's sums: over the rows of a warp (lanes of the same four), then over the warps
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int o = 8; o < 32; o *= 2) {
            gskip[j] = add2(gskip[j], __shfl_xor_sync(0xffffffffu, gskip[j], o));
            gbias[j] = add2(gbias[j], __shfl_xor_sync(0xffffffffu, gbias[j], o));
        }
    __syncthreads();
    float (*sums)[2][kScanChannels] = reinterpret_cast<float (*)[2][kScanChannels]>(&sh.dd[0][0][0]);
    if (lane < 8) {
#pragma unroll
        for (int j = 0; j < 2; j++) {
            *reinterpret_cast<f32x2 *>(&sums[tid / 32][0][four + 2 * j]) = gskip[j];
            *reinterpret_cast<f32x2 *>(&sums[tid / 32][1][four + 2 * j]) = gbias[j];
        }
    }
    __syncthreads();
    for (int i = tid; i < 2 * nch; i += kThreads) {
        const int m = i / nch, ch = i % nch;
        float sum = 0.f;
        for (int w = 0; w < At::kWarps; w++) sum += sums[w][m][ch];
        param[(long long)P.D * (P.N + m) + c0 + ch] = sum;
    }
}

// A segment's own gradient at its start, and its sum of d: for the segments in front of it.  In halves where there is room for as many
// blocks at once, since there is one segment less than in the walk (8 x 2048 x 1024 x 16: 90 us whole, 63 in halves).
template <class T, int NL, int NS, int CD>
__global__ void __launch_bounds__(Place<NL, NS, CD>::kThreads, resident_blocks(NL, NS)) selective_bwd_summary_kernel(const SelectiveParams P)
{
    follow_previous();
    using At = Place<NL, NS, CD>;
    constexpr int NP = At::kPad, NK = At::kPairs, kWords = At::kWords, kQuads = At::kQuads;
    __shared__ __align__(16) float2 dd[2][kTile][kRowPairs];            // d, dy'
    __shared__ __align__(16) float cs[2][kTile][NP];
    __shared__ long long own_end;           // its place; a stager finds it, since the walk needs every register
    if (P.by_rows) {            // rows of part_param that no segment has
        const long long all = P.param_rows * P.param_cols, step = (long long)gridDim.x * gridDim.y * blockDim.x;
        for (long long i = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * blockDim.x + threadIdx.x; i < all; i += step) P.part_param[i] = 0.f;
    }
    const int cb = blockIdx.x % (P.G * P.blocks), b = blockIdx.x / (P.G * P.blocks), g = cb / P.blocks;
    const int c0 = g * P.Dg + cb % P.blocks * kScanChannels;
    const int nch = min(kScanChannels, (g + 1) * P.Dg - c0), seg = blockIdx.y / P.halves + 1, half = blockIdx.y % P.halves;
    const Span s = span_of(P.seq, b);
    const long long begin = seg * P.per + half * half_of(P.per), behind = half + 1 < P.halves ? begin + half_of(P.per) : (seg + 1) * P.per;
    const long long end = s.len < behind ? s.len : behind;
    if (begin >= end) return;
    if (threadIdx.x >= At::kCompute) {
        if (threadIdx.x == At::kCompute) own_end = (first_end(P, s, b) + seg - 1) * P.halves + half;
        const int lane = threadIdx.x - At::kCompute, word = lane % 4 * 8;
        const T *dt = static_cast<const T *>(P.dt) + s.begin * P.dts + c0 + word, *gy = static_cast<const T *>(P.gy) + s.begin * P.D + c0 + word;
        const T *z = P.z != nullptr ? static_cast<const T *>(P.z) + s.begin * P.zs + c0 + word : nullptr;
        const T *cm = static_cast<const T *>(P.cm) + s.begin * P.cs + g * P.N;
        f32x2 bias[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int c = word + 2 * j;
            bias[j] = pair(P.dt_bias != nullptr && c < nch ? P.dt_bias[c0 + c] : 0.f, P.dt_bias != nullptr && c + 1 < nch ? P.dt_bias[c0 + c + 1] : 0.f);
        }
        struct Raw { Eight<T> dt[kWords], z[kWords], gy[kWords]; Quad<T> c[kQuads]; };
        auto fetch = [&](Raw &to, long long t0) {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const long long r = t0 + lane / 4 + i * (At::kStagers / 4);
                const int n = r < end ? nch - word : 0;
                to.dt[i] = fetch_eight(dt + r * P.dts, n, P.whole_dt);
                to.gy[i] = fetch_eight(gy + r * P.D, n, P.whole_d);
                to.z[i] = fetch_eight(z + r * P.zs, z != nullptr ? n : 0, P.whole_z);
            }
#pragma unroll
            for (int i = 0; i < kQuads; i++) {
                const int q = lane + i * At::kStagers, n = q % (NP / 4) * 4;
                const long long r = t0 + q / (NP / 4);
                to.c[i] = fetch_quad(cm + r * P.cs + n, r < end ? P.N - n : 0, P.whole_c);
            }
        };
        Raw next;
        fetch(next, begin);
        int to = 0;
        for (long long t0 = begin; t0 < end; t0 += kTile, to ^= 1) {
            const Raw now = next;
            fetch(next, t0 + kTile);
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const int r = lane / 4 + i * (At::kStagers / 4);
                float df[8], gf[8], zf[8];
                now.dt[i].widen_to(df);
                now.gy[i].widen_to(gf);
                now.z[i].widen_to(zf);
                const bool there = t0 + r < end;
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const f32x2 raw = add2(pair(df[j], df[j + 1]), bias[j / 2]), zz = pair(zf[j], zf[j + 1]);
                    const float2 d = halves(chosen(there, chosen(P.softplus, softplus_of(raw), raw), 0ull));
                    const float2 e = halves(mul2(pair(gf[j], gf[j + 1]), chosen(z != nullptr, mul2(zz, sigmoid_of(zz)), twice(1.f))));
                    *reinterpret_cast<float4 *>(&dd[to][r][slot_of(word) + j]) = make_float4(d.x, e.x, d.y, e.y);
                }
            }
#pragma unroll
            for (int i = 0; i < kQuads; i++) *reinterpret_cast<float4 *>(&cs[to][0][0] + (lane + i * At::kStagers) * 4) = now.c[i].get();
            meet();
        }
        return;
    }
    const At at;
    const int n0 = at.nl * NS, slot = slot_of(at.ch);
    f32x2 A2[CD][NK], own[CD][NK], past[CD][NK];
#pragma unroll
    for (int j = 0; j < CD; j++) {
        load_states<NS>(A2[j], P.A + (long long)(c0 + at.ch + j) * P.N, n0, P.N, at.ch + j < nch);
#pragma unroll
        for (int k = 0; k < NK; k++) {
            A2[j][k] = rate_of(A2[j][k]);
            own[j][k] = 0ull;
            past[j][k] = twice(1.f);
        }
    }
    float time[CD] = {};
    int buf = 0;
    for (long long t0 = begin; t0 < end; t0 += kTile, buf ^= 1) {
        meet();
#pragma unroll
        for (int t = 0; t < kTile; t++) {
            f32x2 C[NK];
            float2 d[CD];
            row_pairs<NS>(C, &cs[buf][t][n0]);
            two_of<CD>(d, &dd[buf][t][slot]);
#pragma unroll
            for (int j = 0; j < CD; j++) {
                time[j] += d[j].x;
#pragma unroll
                for (int k = 0; k < NK; k++) {
                    past[j][k] = mul2(past[j][k], exp2_pair(mul2(twice(d[j].x), A2[j][k])));
                    own[j][k] = fma2(past[j][k], mul2(C[k], twice(d[j].y)), own[j][k]);
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const long long segment = own_end * P.D + c0 + at.ch + j;
        store_states<NS>(P.seg_state + segment * P.N, own[j], n0, P.N, in);
        if (in && at.nl == 0) P.seg_time[segment] = time[j];
    }
}

// Gradients of B and C: the sums over a group's blocks of channels, in their order; four neighbours a thread, eight blocks' on their way.
template <class T>
__global__ void __launch_bounds__(128) selective_bc_kernel(const SelectiveParams P, T *gb, T *gc, long long tiles)
{
    follow_previous();
    const int b = (int)(blockIdx.x / tiles), g = blockIdx.y, cols = 2 * P.N;
    const Span s = span_of(P.seq, b);
    const long long t0 = blockIdx.x % tiles * kTile, rows = s.len - t0 < kTile ? s.len - t0 : kTile, step = P.seq.rows * cols;
    const float *part = P.part_bc + (long long)g * P.blocks * step + (s.begin + t0) * cols;
    auto put = [&](long long i, float sum) {
        const long long row = s.begin + t0 + i / cols;
        const int n = (int)(i % cols);
        T *out = n < P.N ? gb + row * P.G * P.N + g * P.N + n : gc + row * P.G * P.N + g * P.N + n - P.N;
        *out = narrow<T>(sum);
    };
    if (P.N % 2 == 0) {         // rows of whole 16-byte words
        for (long long i = threadIdx.x * 4; i < rows * cols; i += 4 * blockDim.x) {
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
            for (int k = 0; k < P.blocks; k++) {
                const float4 v = *reinterpret_cast<const float4 *>(part + k * step + i);
                sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
            }
            put(i, sum.x);
            put(i + 1, sum.y);
            put(i + 2, sum.z);
            put(i + 3, sum.w);
        }
    } else {
        for (long long i = threadIdx.x; i < rows * cols; i += blockDim.x) {
            float sum = 0.f;
            for (int k = 0; k < P.blocks; k++) sum += part[k * step + i];
            put(i, sum);
        }
    }
}

template <class T, bool GATE, int NL, int NS, int CD> int run(const SelectiveParams &P, dim3 grid, cudaStream_t st)
{
    // 228 KB of shared memory, of which a block takes 1 KB more than it asks for, and 65,536 registers, 256 a thread
    constexpr int shared = 228 * 1024 / (int)(sizeof(BwdShared<T, NL, NS, CD>) + 1024), registers = 65536 / (256 * Walker<NL, NS, CD>::kThreads);
    static_assert(resident_walks(NL, NS, sizeof(T) == 2) == (shared < registers ? shared : registers), "the time axis is cut for this many blocks");
    return launch_shared(selective_bwd_kernel<T, NL, NS, CD, GATE>, grid, Walker<NL, NS, CD>::kThreads, sizeof(BwdShared<T, NL, NS, CD>), P, st);
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
    const dim3 grid((unsigned)(P.G * P.blocks * P.seq.B), (unsigned)(summary ? P.halves * (P.S - 1) : P.S));
    if (summary) return status_of(launch<true>(half ? pick_summary<bf16>(s) : pick_summary<float>(s), grid, dim3(s.threads()), 0, st, P));
    return half ? (P.z != nullptr ? run<bf16, true>(P, s, grid, st) : run<bf16, false>(P, s, grid, st))
                : (P.z != nullptr ? run<float, true>(P, s, grid, st) : run<float, false>(P, s, grid, st));
}

int launch_selective_bc(const SelectiveParams &P, bool half, void *grad_b, void *grad_c, cudaStream_t st)
{
    const long long tiles = ceil_div(P.seq.L, kTile);
    const dim3 grid((unsigned)(tiles * P.seq.B), (unsigned)P.G);
    return half ? status_of(launch<true>(selective_bc_kernel<bf16>, grid, dim3(128), 0, st, P, static_cast<bf16 *>(grad_b), static_cast<bf16 *>(grad_c), tiles))
                : status_of(launch<true>(selective_bc_kernel<float>, grid, dim3(128), 0, st, P, static_cast<float *>(grad_b), static_cast<float *>(grad_c), tiles));
}

}  // namespace cawn
