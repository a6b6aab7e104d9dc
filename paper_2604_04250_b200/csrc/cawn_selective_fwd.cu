// Selective scan, forward: walks over tiles of tokens.
//
// Two kinds of warps.  The computing ones hold the states and leave, for each token and channel, what each lane's states give to
// the read-out.  The stagers bring tile k + 1 into shared memory, and finish tile k - 1: they sum over the lanes, add skip x, gate and
// store.  (With the sums by shuffles and the stores in the computing warps these waited for them in order: 82 of 278 us of
// 8 x 2048 x 2368 x 16.)
// Measured, bfloat16 with the gate: 8 x 2048 x 2048 x 16 in 224 us, 1.9 times the decays' exponentials: their unit is busy 68% of
// the time (the step's and the gate's are a quarter more), issue 48%, and 80 of 148 multiprocessors have three blocks where the
// others have four.  1 x 32768 x 768 x 16, 24 segments behind a pass: 283 us (exponentials 176, each taken twice).
#include "cawn_selective.cuh"

namespace cawn {
namespace {

template <class T, int NL, int NS, int CD, bool SUMMARY> struct FwdShared {
    using At = Place<NL, NS, CD>;
    float2 dd[2][kTile][kRowPairs];                             // d, d x
    float bc[2][2][kTile][At::kPad];
    float out[SUMMARY ? 1 : 2][kTile][NL * kRowFloats + 4];     // read-out by lane of a channel (and 16 bytes, for the stagers' two rows at a time)
    long long own_end;                                          // of a summary: its place.  A stager finds it, since the walk needs every register
    Eight<T> words[SUMMARY ? 1 : 3][2][At::kWords][At::kStagers];       // x and z as a stager fetched them, until their tile is finished
};

// SPLIT: the finishing has warps of its own and the computing warps look four tokens ahead, not two.  For calls of so few blocks that
// half of a multiprocessor's places are enough, and with them half of the registers: 8 x 2048 x 1024 x 16 in 131 instead of 166 us.
template <class T, int NL, int NS, int CD, bool SUMMARY, bool WHOLE, bool SPLIT>
__global__ void __launch_bounds__(Place<NL, NS, CD>::kThreads + (SPLIT ? Place<NL, NS, CD>::kStagers : 0), resident_blocks(NL, NS) / (SPLIT ? 2 : 1)) selective_fwd_kernel(const SelectiveParams P)
{
    follow_previous();
    using At = Place<NL, NS, CD>;
    constexpr int NP = At::kPad, NK = At::kPairs, kWords = At::kWords, kQuads = At::kQuads;
    using Shared = FwdShared<T, NL, NS, CD, SUMMARY>;
    extern __shared__ __align__(16) unsigned char raw_shared[];
    Shared &sh = *reinterpret_cast<Shared *>(raw_shared);

    const int cb = blockIdx.x % (P.G * P.blocks), b = blockIdx.x / (P.G * P.blocks), g = cb / P.blocks;
    const int c0 = g * P.Dg + cb % P.blocks * kScanChannels;
    const int nch = min(kScanChannels, (g + 1) * P.Dg - c0), seg = blockIdx.y;
    const Span s = span_of(P.seq, b);
    const long long begin = seg * P.per, end = s.len < begin + P.per ? s.len : begin + P.per;
    const bool walks = SUMMARY ? end < s.len : begin < end;             // a summary: somebody comes behind this segment

    if (threadIdx.x >= At::kCompute) {
        if (!walks) return;
        if (SUMMARY && threadIdx.x == At::kCompute) sh.own_end = first_end(P, s, b) + seg;
        const int lane = (threadIdx.x - At::kCompute) % At::kStagers, word = lane % 4 * 8;
        const T *x = static_cast<const T *>(P.x) + s.begin * P.xs + c0 + word, *dt = static_cast<const T *>(P.dt) + s.begin * P.dts + c0 + word;
        const T *z = P.z != nullptr && !SUMMARY && P.y != nullptr ? static_cast<const T *>(P.z) + s.begin * P.zs + c0 + word : nullptr;
        const T *bm = static_cast<const T *>(P.bm) + s.begin * P.bs + g * P.N, *cm = static_cast<const T *>(P.cm) + s.begin * P.cs + g * P.N;
        f32x2 bias[4], skip[4];         // of this lane's eight channels
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int c = word + 2 * j;
            auto two = [&](const float *p) { return pair(p != nullptr && c < nch ? p[c0 + c] : 0.f, p != nullptr && c + 1 < nch ? p[c0 + c + 1] : 0.f); };
            bias[j] = two(P.dt_bias);
            skip[j] = two(P.skip);
        }
        struct Raw { Eight<T> x[kWords], dt[kWords], z[kWords]; Quad<T> b[kQuads], c[kQuads]; };
        auto fetch = [&](Raw &to, long long t0) {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const long long r = t0 + lane / 4 + i * (At::kStagers / 4);
                const int n = r < end ? nch - word : 0;
                to.x[i] = eight_of<WHOLE>(x + r * P.xs, n, P.whole_x);
                to.dt[i] = eight_of<WHOLE>(dt + r * P.dts, n, P.whole_dt);
                if (!SUMMARY) to.z[i] = eight_of<WHOLE>(z + r * P.zs, z != nullptr ? n : 0, P.whole_z);
            }
#pragma unroll
            for (int i = 0; i < kQuads; i++) {
                const int q = lane + i * At::kStagers, n = q % (NP / 4) * 4;
                const long long r = t0 + q / (NP / 4);
                const int left = r < end ? P.N - n : 0;
                to.b[i] = quad_of<WHOLE>(bm + r * P.bs + n, left, P.whole_b);
                if (!SUMMARY) to.c[i] = quad_of<WHOLE>(cm + r * P.cs + n, left, P.whole_c);
            }
        };
        T *y = !SUMMARY && P.y != nullptr ? static_cast<T *>(P.y) + s.begin * P.D + c0 + word : nullptr;
        auto finish = [&](long long t0, int from, int kept, bool there) {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const int r = lane / 4 + i * (At::kStagers / 4);
                float xf[8], zf[8], f[8];
                sh.words[kept][0][i][lane].widen_to(xf);
                sh.words[kept][1][i][lane].widen_to(zf);
                f32x2 sum[4] = {};
#pragma unroll
                for (int q = 0; q < NL; q++) {
                    f32x2 part[4];
                    row_pairs<8>(part, &sh.out[from][r][q * kRowFloats + word]);
#pragma unroll
                    for (int j = 0; j < 4; j++) sum[j] = q == 0 ? part[j] : add2(sum[j], part[j]);
                }
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const f32x2 zz = pair(zf[2 * j], zf[2 * j + 1]), v = fma2(skip[j], pair(xf[2 * j], xf[2 * j + 1]), sum[j]);
                    const float2 o = halves(chosen(z != nullptr, mul2(v, mul2(zz, sigmoid_of(zz))), v));
                    f[2 * j] = o.x;
                    f[2 * j + 1] = o.y;
                }
                if (there && y != nullptr && t0 + r < end) store_eight(y + (t0 + r) * P.D, f, nch - word, WHOLE || P.whole_d);
            }
        };
        int to = 0, kept = 0;           // buffers of the tile that is staged
        auto finish_last_two = [&] {
            const long long tiles = (end - begin + kTile - 1) / kTile;
            if (tiles > 1) finish(begin + (tiles - 2) * kTile, to, kept == 2 ? 0 : kept + 1, true);
            meet();
            finish(begin + (tiles - 1) * kTile, to ^ 1, kept == 0 ? 2 : kept - 1, true);
        };
        if (SPLIT && threadIdx.x >= At::kCompute + At::kStagers) {
            for (long long t0 = begin; t0 < end; t0 += kTile, to ^= 1, kept = kept == 2 ? 0 : kept + 1) {
                finish(t0 - 2 * kTile, to, kept == 2 ? 0 : kept + 1, t0 >= begin + 2 * kTile);
                meet();
            }
            finish_last_two();
            return;
        }
        // Finished among the staging, or behind it: floats have no registers left for the first (8 x 2048 x 2368 x 8: 276 us, 205).
        constexpr bool kEarly = sizeof(T) == 2;
        Raw next;
        fetch(next, begin);
        for (long long t0 = begin; t0 < end; t0 += kTile, to ^= 1, kept = kept == 2 ? 0 : kept + 1) {
            const Raw now = next;
            fetch(next, t0 + kTile);        // on its way while this tile is staged and the one before is computed
            if constexpr (!SUMMARY && !SPLIT && kEarly) finish(t0 - 2 * kTile, to, kept == 2 ? 0 : kept + 1, t0 >= begin + 2 * kTile);
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const int r = lane / 4 + i * (At::kStagers / 4);
                float xf[8], df[8];
                now.x[i].widen_to(xf);
                now.dt[i].widen_to(df);
                if constexpr (!SUMMARY) {
                    sh.words[kept][0][i][lane] = now.x[i];
                    sh.words[kept][1][i][lane] = now.z[i];
                }
                const bool there = t0 + r < end;        // past the end nothing moves
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const f32x2 xx = pair(xf[j], xf[j + 1]), raw = add2(pair(df[j], df[j + 1]), bias[j / 2]);
                    const f32x2 d = chosen(there, chosen(P.softplus, softplus_of(raw), raw), 0ull);
                    const float2 e = halves(d), f = halves(mul2(d, xx));
                    *reinterpret_cast<float4 *>(&sh.dd[to][r][slot_of(word) + j]) = make_float4(e.x, f.x, e.y, f.y);
                }
            }
#pragma unroll
            for (int i = 0; i < kQuads; i++) {
                *reinterpret_cast<float4 *>(&sh.bc[to][0][0][0] + (lane + i * At::kStagers) * 4) = now.b[i].get();
                if (!SUMMARY) *reinterpret_cast<float4 *>(&sh.bc[to][1][0][0] + (lane + i * At::kStagers) * 4) = now.c[i].get();
            }
            if constexpr (!SUMMARY && !SPLIT && !kEarly) finish(t0 - 2 * kTile, to, kept == 2 ? 0 : kept + 1, t0 >= begin + 2 * kTile);
            meet();             // the tile is there; the one before it is computed
        }
        if constexpr (SPLIT) meet();
        else if constexpr (!SUMMARY) finish_last_two();
        return;
    }

    const At at;
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
        if (!walks) return;
    } else {
        if (seg > 0 && !walks) return;
    }
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const int c = c0 + at.ch + j;
        load_states<NS>(A2[j], P.A + (long long)c * P.N, n0, P.N, in);
#pragma unroll
        for (int k = 0; k < NK; k++) A2[j][k] = rate_of(A2[j][k]);
        if constexpr (!SUMMARY) {
            if (seg == 0) {
                const float *from = P.S > 1 ? P.first : P.state_in;
                load_states<NS>(h[j], from + ((long long)b * P.D + c) * P.N, n0, P.N, in && P.state_in != nullptr);
            } else {
                const long long segment = first_end(P, s, b) * P.D + c;
                load_states<NS>(h[j], P.seg_state + segment * P.N, n0, P.N, in);
                fold_segments<NS>(h[j], P, A2[j], segment + P.D, P.D, seg - 1, n0, in);
            }
        }
    }
    float time[CD] = {};
    float *mark = P.checkpoints + ((checkpoint_of(s, b) + begin / kTile) * P.D + c0 + at.ch) * P.N;
    const int slot = slot_of(at.ch);
    int buf = 0;
    for (long long t0 = begin; t0 < end; t0 += kTile, mark += (long long)P.D * P.N, buf ^= 1) {
        meet();
        if (!SUMMARY && P.checkpoints != nullptr) {
#pragma unroll
            for (int j = 0; j < CD; j++) store_states<NS>(mark + j * P.N, h[j], n0, P.N, at.ch + j < nch);
        }
        // some tokens' decays are found while those before them move the states
        constexpr int kSome = SPLIT ? 4 : 2;
        f32x2 a[2][kSome][CD][NK], in[2][kSome][CD][NK];
        auto decays = [&](int u) {
#pragma unroll
            for (int i = 0; i < kSome; i++) {
                f32x2 B[NK];
                float2 d[CD];
                row_pairs<NS>(B, &sh.bc[buf][0][kSome * u + i][n0]);
                two_of<CD>(d, &sh.dd[buf][kSome * u + i][slot]);
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
#pragma unroll
        for (int u = 0; u < kTile / kSome; u++) {
            if (u + 1 < kTile / kSome) decays(u + 1);
#pragma unroll
            for (int i = 0; i < kSome; i++) {
                f32x2 C[NK];
                float v[CD];
                if constexpr (!SUMMARY) row_pairs<NS>(C, &sh.bc[buf][1][kSome * u + i][n0]);
#pragma unroll
                for (int j = 0; j < CD; j++) {
                    f32x2 acc = 0ull;
#pragma unroll
                    for (int k = 0; k < NK; k++) {
                        h[j][k] = fma2(a[u % 2][i][j][k], h[j][k], in[u % 2][i][j][k]);
                        if constexpr (!SUMMARY) acc = k == 0 ? mul2(h[j][k], C[k]) : fma2(h[j][k], C[k], acc);
                    }
                    v[j] = sum_of(acc);
                }
                if constexpr (!SUMMARY) put_channels<CD>(&sh.out[buf][kSome * u + i][at.nl * kRowFloats + at.ch], v);
            }
        }
    }
    if (!SUMMARY && walks) meet();      // for the stagers, which finish the last tile
#pragma unroll
    for (int j = 0; j < CD; j++) {
        const bool in = at.ch + j < nch;
        const int c = c0 + at.ch + j;
        if constexpr (SUMMARY) {
            const long long segment = sh.own_end * P.D + c;
            store_states<NS>(P.seg_state + segment * P.N, h[j], n0, P.N, in);
            if (in && at.nl == 0) P.seg_time[segment] = time[j];
        } else {
            if (end == s.len && P.state_out != nullptr) store_states<NS>(P.state_out + ((long long)b * P.D + c) * P.N, h[j], n0, P.N, in);
        }
    }
}

template <class T, bool SUMMARY, bool WHOLE, bool SPLIT, int NL, int NS, int CD> int run(const SelectiveParams &P, dim3 grid, cudaStream_t st)
{
    using At = Place<NL, NS, CD>;
    return launch_shared(selective_fwd_kernel<T, NL, NS, CD, SUMMARY, WHOLE, SPLIT>, grid, At::kThreads + (SPLIT ? At::kStagers : 0), sizeof(FwdShared<T, NL, NS, CD, SUMMARY>), P, st);
}
template <class T, bool SUMMARY, bool SPLIT> int run(const SelectiveParams &P, const Shape &s, dim3 grid, cudaStream_t st)
{
#define CAWN_CALL(NL, NS, CD)                                                                                  \
    (P.whole ? run<T, SUMMARY, true, SPLIT && NS == 4, NL, NS, CD>(P, grid, st)                                \
             : run<T, SUMMARY, false, SPLIT && NS == 4, NL, NS, CD>(P, grid, st))
    return CAWN_BY_SHAPE(s, CAWN_CALL);
#undef CAWN_CALL
}
template <class T, bool SUMMARY> int run(const SelectiveParams &P, const Shape &s, cudaStream_t st)
{
    const dim3 grid((unsigned)(P.G * P.blocks * P.seq.B), (unsigned)(SUMMARY ? P.S - 1 : P.S));
    const bool few = s.ns == 4 && (int64_t)grid.x * grid.y <= (int64_t)sm_count() * (s.resident() / 2);
    if constexpr (!SUMMARY) return few ? run<T, false, true>(P, s, grid, st) : run<T, false, false>(P, s, grid, st);
    else return run<T, true, false>(P, s, grid, st);
}

}  // namespace

int launch_selective_fwd(const SelectiveParams &P, const Shape &s, bool half, bool summary, cudaStream_t st)
{
    return half ? (summary ? run<bf16, true>(P, s, st) : run<bf16, false>(P, s, st)) : (summary ? run<float, true>(P, s, st) : run<float, false>(P, s, st));
}

}  // namespace cawn
