// Short causal convolution, channel by channel, with its history and an optional SiLU.
//
// Mathematics: with e the sequence behind its history of K - 1 rows, z_t = bias + sum_k w_k e_{t+k}, y_t = z_t or z_t sigmoid(z_t);
// the new history is e's last K - 1 rows.  Backward: dz = dy act'(z), de_i = sum_k w_k dz_{i-k} (and the new history's
// gradient on the last K - 1), dw_k = sum_t dz_t e_{t+k}, dbias = sum_t dz_t.
// Bound: memory; an element costs K products.  A thread keeps four channels and walks rows with the last K - 1 of them in
// registers, so that a row is fetched once but for the K - 1 in front of a walk, which the neighbour's fetch has brought to L1 or L2.
// Measured with SiLU, K = 4: 8 x 2048 x 2048 bfloat16 forward 30 us (4.4 TB/s; memory's time 21, the exponentials and reciprocals of
// the sigmoid 15), backward 71 (2.9 TB/s; memory's time 31: issue 51% with 12 warps a multiprocessor of 152 registers, which wait for
// their own arithmetic), float 52 (5.2 TB/s) and 80 (5.1 TB/s).
#include "cawn_seq.cuh"

namespace cawn {
namespace {

constexpr int kLanes = 32, kWalks = 4, kStep = 8;        // a block: 32 words of four channels, 4 walks of a multiple of 8 rows
constexpr int kConvThreads = kLanes * kWalks;
constexpr int kBatch = 4;       // rows that are computed at a time
// Blocks that a multiprocessor holds.
constexpr int fwd_blocks(size_t element) { return element == 2 ? 8 : 5; }
constexpr int kBwdBlocks = 3;

struct ConvParams {
    Sequences seq;
    const void *x, *gy;
    void *y, *gx;
    const float *w, *b, *state_in, *gstate_out;
    float *state_out, *gstate_in, *part;
    int rows;                                   // of a walk
    long long x_stride, tiles, all_tiles;       // tiles (kWalks walks) of a sequence of L rows, of all sequences
    int C, words, silu, x_whole, c_whole;
};

constexpr int kWord = 4, kPairs = kWord / 2;
using Row = f32x2[kPairs];      // a thread's channels as pairs

// A row's four channels.  WHOLE: every row of every array begins on a word and C is a multiple of four, so that an access is
// one instruction (8 x 2048 x 2048, forward: 18 instructions an element without, 10 with).
template <bool WHOLE, class T> __device__ __forceinline__ Quad<T> word_of(const T *p, bool in, int n, bool whole)
{
    if constexpr (!WHOLE) return fetch_quad(p, in ? n : 0, whole);
    Quad<T> r;
    r.set(make_float4(0.f, 0.f, 0.f, 0.f));
    if (in) r.load(p);
    return r;
}
template <class T> __device__ __forceinline__ void pairs_of(Row &r, const Quad<T> &e)
{
    const float4 f = e.get();
    r[0] = pair(f.x, f.y);
    r[1] = pair(f.z, f.w);
}
template <bool WHOLE, class T> __device__ __forceinline__ void store_row(T *p, const Row &r, int n, bool whole)
{
    const float2 a = halves(r[0]), b = halves(r[1]);
    store_quad(p, make_float4(a.x, a.y, b.x, b.y), WHOLE ? kWord : n, WHOLE || whole);
}

// A thread's rows on their way: DEPTH batches in shared memory, each thread's own words, so that no one waits for another
// and none of them takes registers (with eight rows in registers the forward of 8 x 2048 x 2048 took 36 us, the backward 91).
template <class T, int DEPTH, bool WHOLE> struct Ring {
    Quad<T> words[DEPTH][kBatch][kConvThreads];
    // Four rows set out, `left` of them there; as one group even where there is none.
    __device__ __forceinline__ void fetch(int slot, const T *p, long long stride, int left, int n, bool whole)
    {
#pragma unroll
        for (int r = 0; r < kBatch; r++) {
            Quad<T> *to = &words[slot][r][threadIdx.x];
            if constexpr (WHOLE) {
                const unsigned at = (unsigned)__cvta_generic_to_shared(to);
                const int bytes = r < left ? (int)sizeof(Quad<T>) : 0;
                asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" :: "r"(at), "l"(p + r * stride), "n"(sizeof(Quad<T>)), "r"(bytes) : "memory");
            } else {
                *to = fetch_quad(p + r * stride, r < left ? n : 0, whole);
            }
        }
    }
    __device__ __forceinline__ void row(Row &r, int slot, int i) const { pairs_of(r, words[slot][i][threadIdx.x]); }
};
__device__ __forceinline__ void close_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int NEWER> __device__ __forceinline__ void wait_group() { asm volatile("cp.async.wait_group %0;" :: "n"(NEWER) : "memory"); }

// Row `i` of the sequence behind its history (i < 0: history, zero without one), as the arrays hold it.
template <class T, int K, bool WHOLE>
__device__ __forceinline__ void extended(Row &r, const ConvParams &P, const T *x, const float *history, long long i, int n)
{
    if (i >= 0) {
        pairs_of(r, word_of<WHOLE>(x + i * P.x_stride, true, n, P.x_whole));
    } else if (history != nullptr) {
        pairs_of(r, word_of<WHOLE>(history + (i + K - 1) * P.C, true, n, P.c_whole));
    } else {
#pragma unroll
        for (int c = 0; c < kPairs; c++) r[c] = 0ull;
    }
}

// The block's weights and biases, fetched as they lie, turned over in shared memory, and a thread's own of them.
constexpr int kChannels = kLanes * kWord;
template <int K> __device__ __forceinline__ void taps_of(Row (&w)[K], Row &b, const ConvParams &P)
{
    __shared__ __align__(16) float turned[K + 1][kChannels + 8];
    const int first = blockIdx.y * kChannels, here = P.C - first < kChannels ? P.C - first : kChannels;
    for (int i = threadIdx.x; i < kChannels * K; i += kConvThreads) turned[i % K][i / K] = i < here * K ? P.w[(long long)first * K + i] : 0.f;
    for (int i = threadIdx.x; i < kChannels; i += kConvThreads) turned[K][i] = i < here && P.b != nullptr ? P.b[first + i] : 0.f;
    __syncthreads();
    const int at = threadIdx.x % kLanes * kWord;
#pragma unroll
    for (int k = 0; k <= K; k++) {
        const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(&turned[k][at]);
        (k < K ? w[k < K ? k : 0] : b)[0] = v.x;
        (k < K ? w[k < K ? k : 0] : b)[1] = v.y;
    }
}

template <class T, int K, bool WHOLE>
__global__ void __launch_bounds__(kConvThreads, fwd_blocks(sizeof(T))) conv_fwd_kernel(const ConvParams P)
{
    follow_previous();
    const int word = (blockIdx.y * kLanes + threadIdx.x % kLanes), c0 = word * kWord;
    const int n = P.C - c0 < kWord ? P.C - c0 : kWord;
    const int b = (int)(blockIdx.x / P.tiles);
    const long long t0 = (blockIdx.x % P.tiles * kWalks + threadIdx.x / kLanes) * (long long)P.rows;
    const Span s = span_of(P.seq, b);
    const bool here = word < P.words && (t0 < s.len || t0 == 0);
    const T *x = static_cast<const T *>(P.x) + s.begin * P.x_stride + c0;
    const float *history = P.state_in != nullptr && K > 1 ? P.state_in + (long long)b * (K - 1) * P.C + c0 : nullptr;
    const int rows = !here ? 0 : s.len - t0 < P.rows ? (int)(s.len - t0) : P.rows;
    // The first batches, and the K - 1 rows in front, set out before the weights do.
    constexpr int kDepth = 4;
    __shared__ __align__(16) Ring<T, kDepth, WHOLE> ring;
    const T *ahead = x + t0 * P.x_stride;
    int left = rows;            // of what is still to set out
    auto fetch = [&](int slot) {
        ring.fetch(slot, ahead, P.x_stride, left, n, P.x_whole);
        close_group();
        ahead += kBatch * P.x_stride;
        left -= kBatch;
    };
    Row old[K];                 // the K - 1 rows in front of the next one
#pragma unroll
    for (int q = 0; q < kDepth; q++) fetch(q);
    if (here) {
#pragma unroll
        for (int j = 0; j < K - 1; j++) extended<T, K, WHOLE>(old[j], P, x, history, t0 + j - (K - 1), n);
    }
    Row w[K], bias;
    taps_of<K>(w, bias, P);
    if (!here) return;
    // The new history, by the walk at the sequence's start: it alone reads the old one, which may be the same array.
    if (K > 1 && t0 == 0 && P.state_out != nullptr) {
        float *out = P.state_out + (long long)b * (K - 1) * P.C + c0;
#pragma unroll
        for (int j = 0; j < K - 1; j++) {
            Row r;
            extended<T, K, WHOLE>(r, P, x, history, s.len + j - (K - 1), n);       // never a row of the history that is overwritten already
            store_row<WHOLE>(out + (long long)j * P.C, r, n, P.c_whole);
        }
    }
    T *y = static_cast<T *>(P.y) + (s.begin + t0) * P.C + c0;
    int slot = 0;
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += kBatch, slot = slot + 1 == kDepth ? 0 : slot + 1) {
        wait_group<kDepth - 1>();
#pragma unroll
        for (int r = 0; r < kBatch; r++) {
            Row now, z;
            ring.row(now, slot, r);
#pragma unroll
            for (int c = 0; c < kPairs; c++) {
                z[c] = fma2(w[K - 1][c], now[c], bias[c]);
#pragma unroll
                for (int k = 0; k < K - 1; k++) z[c] = fma2(w[k][c], old[k][c], z[c]);
                if (P.silu) z[c] = mul2(z[c], sigmoid_of(z[c]));
#pragma unroll
                for (int k = 0; k + 2 < K; k++) old[k][c] = old[k + 1][c];
                if (K > 1) old[K > 1 ? K - 2 : 0][c] = now[c];
            }
            if (r0 + r < rows) store_row<WHOLE>(y + r * (long long)P.C, z, n, P.c_whole);
        }
        y += (long long)kBatch * P.C;
        fetch(slot);
    }
}

// Single tokens: a thread has four channels of kTokens sequences, which share their weights.
constexpr int kTokens = 4;
template <class T, int K>
__global__ void __launch_bounds__(kConvThreads) conv_step_kernel(const ConvParams P)
{
    follow_previous();
    const int word = blockIdx.x * kConvThreads + threadIdx.x, c0 = word * kWord;
    if (word >= P.words) return;
    const int n = P.C - c0 < kWord ? P.C - c0 : kWord;
    const long long b0 = (long long)blockIdx.y * kTokens;
    Quad<T> x[kTokens];
    Quad<float> old[kTokens][K], w[K];          // rows of the history; the four channels' K weights as they lie
#pragma unroll
    for (int r = 0; r < kTokens; r++) {
        const bool in = b0 + r < P.seq.B;
        x[r] = fetch_quad(static_cast<const T *>(P.x) + (b0 + r) * P.x_stride + c0, in ? n : 0, P.x_whole);
#pragma unroll
        for (int k = 0; k < K - 1; k++)
            old[r][k] = fetch_quad(P.state_in + ((b0 + r) * (K - 1) + k) * P.C + c0, in && P.state_in != nullptr ? n : 0, P.c_whole);
    }
#pragma unroll
    for (int i = 0; i < K; i++) w[i] = fetch_quad(P.w + (long long)c0 * K + i * 4, n * K - i * 4, true);
    const Quad<float> bias = fetch_quad(P.b + c0, P.b != nullptr ? n : 0, true);
    float ws[K * 4];
#pragma unroll
    for (int i = 0; i < K; i++) {
        const float4 v = w[i].get();
        ws[4 * i] = v.x; ws[4 * i + 1] = v.y; ws[4 * i + 2] = v.z; ws[4 * i + 3] = v.w;
    }
#pragma unroll
    for (int r = 0; r < kTokens; r++) {
        if (b0 + r >= P.seq.B) break;
        const float4 now = x[r].get(), bv = bias.get();
        float xs[4] = {now.x, now.y, now.z, now.w}, z[4] = {bv.x, bv.y, bv.z, bv.w};
#pragma unroll
        for (int c = 0; c < 4; c++) z[c] = fmaf(ws[c * K + K - 1], xs[c], z[c]);
#pragma unroll
        for (int k = 0; k < K - 1; k++) {
            const float4 o = old[r][k].get();
            const float os[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int c = 0; c < 4; c++) z[c] = fmaf(ws[c * K + k], os[c], z[c]);
        }
        if (P.silu) {
#pragma unroll
            for (int c = 0; c < 4; c++) z[c] *= sigmoid_of(z[c]);
        }
        store_quad(static_cast<T *>(P.y) + (b0 + r) * P.C + c0, make_float4(z[0], z[1], z[2], z[3]), n, P.c_whole);
        if (K > 1 && P.state_out != nullptr) {
            float *out = P.state_out + (b0 + r) * (K - 1) * P.C + c0;
#pragma unroll
            for (int k = 0; k < K - 1; k++) store_quad(out + (long long)k * P.C, k + 2 < K ? old[r][k + 2 < K ? k + 1 : 0].get() : now, n, P.c_whole);
        }
    }
}

// A block takes tile after tile, so that few partial sums of the parameters' gradients are left.
template <class T, int K, bool WHOLE>
__global__ void __launch_bounds__(kConvThreads, kBwdBlocks) conv_bwd_kernel(const ConvParams P)
{
    follow_previous();
    constexpr int kDepth = sizeof(T) == 2 ? 4 : 2;
    __shared__ __align__(16) Ring<T, kDepth, WHOLE> ring, ringg;        // x; grad_y
    const int lane = threadIdx.x % kLanes, walk = threadIdx.x / kLanes, word = blockIdx.y * kLanes + lane, c0 = word * kWord;
    const int n = word < P.words ? (P.C - c0 < kWord ? P.C - c0 : kWord) : 0;
    Row w[K], bias, gw[K] = {}, gb = {};
    taps_of<K>(w, bias, P);
    for (long long tile = blockIdx.x; tile < P.all_tiles; tile += gridDim.x) {
        const int b = (int)(tile / P.tiles);
        const long long t0 = (tile % P.tiles * kWalks + walk) * P.rows;
        const Span s = span_of(P.seq, b);
        if (n == 0 || (t0 >= s.len && t0 != 0)) continue;
        const T *x = static_cast<const T *>(P.x) + s.begin * P.x_stride + c0;
        const T *gy = static_cast<const T *>(P.gy) + s.begin * P.C + c0;
        T *gx = static_cast<T *>(P.gx) + s.begin * P.C + c0;
        const float *history = P.state_in != nullptr && K > 1 ? P.state_in + (long long)b * (K - 1) * P.C + c0 : nullptr;
        const float *gso = P.gstate_out != nullptr && K > 1 ? P.gstate_out + (long long)b * (K - 1) * P.C + c0 : nullptr;
        Row old[K], dz[K] = {};                 // rows t-K+1 .. t-1 of e; dz of rows t-K+1 .. t (0 before this walk)
        const int own = (int)(s.len - t0 < P.rows ? s.len - t0 : P.rows);            // rows of this walk
        const int all = own + K - 1, have = (int)(s.len - t0 < all ? s.len - t0 : all);  // those gone through, and of them in the sequence
        const T *ax = x + t0 * P.x_stride, *ag = gy + t0 * P.C;
        int left = have;            // of what is still to set out
        auto fetch = [&](int slot) {
            ring.fetch(slot, ax, P.x_stride, left, n, P.x_whole);
            ringg.fetch(slot, ag, P.C, left, n, P.c_whole);
            close_group();
            ax += kBatch * P.x_stride;
            ag += (long long)kBatch * P.C;
            left -= kBatch;
        };
        wait_group<0>();            // nothing of the tile before is on its way
#pragma unroll
        for (int q = 0; q < kDepth; q++) fetch(q);
#pragma unroll
        for (int j = 0; j < K - 1; j++) extended<T, K, WHOLE>(old[j], P, x, history, t0 + j - (K - 1), n);
        T *out = gx + (t0 - (K - 1)) * P.C;         // of the row that the next one completes
        // row r gives dz_r; what then is complete is the gradient of row r - (K - 1), whose last term dz_r is (in front of the
        // first walk of a sequence: of the history)
        int slot = 0;
#pragma unroll 1
        for (int r0 = 0; r0 < all; r0 += kBatch, slot = slot + 1 == kDepth ? 0 : slot + 1) {
            wait_group<kDepth - 1>();
#pragma unroll
            for (int k0 = 0; k0 < kBatch; k0++) {
                    const int r = r0 + k0;
                    Row now, d;
                    ring.row(now, slot, k0);
                    ringg.row(d, slot, k0);         // past the end: zero
#pragma unroll
                    for (int c = 0; c < kPairs; c++) {
                        if (P.silu) {
                            f32x2 z = fma2(w[K - 1][c], now[c], bias[c]);
#pragma unroll
                            for (int k = 0; k < K - 1; k++) z = fma2(w[k][c], old[k][c], z);
                            const f32x2 sg = sigmoid_of(z), one = twice(1.f);
                            const f32x2 slope = mul2(sg, fma2(z, fma2(sg, twice(-1.f), one), one));
                            d[c] = r < have ? mul2(d[c], slope) : 0ull;     // a select: the slope there may be anything
                        }
#pragma unroll
                        for (int k = 0; k + 1 < K; k++) dz[k][c] = dz[k + 1][c];
                        dz[K - 1][c] = d[c];
                    }
                    if (r < own) {
#pragma unroll
                        for (int c = 0; c < kPairs; c++) {
#pragma unroll
                            for (int k = 0; k < K - 1; k++) gw[k][c] = fma2(d[c], old[k][c], gw[k][c]);
                            gw[K - 1][c] = fma2(d[c], now[c], gw[K - 1][c]);
                            gb[c] = add2(gb[c], d[c]);
                        }
                    }
                    Row de;
#pragma unroll
                    for (int c = 0; c < kPairs; c++) {
#pragma unroll
                        for (int k = 0; k + 2 < K; k++) old[k][c] = old[k + 1][c];
                        if (K > 1) old[K > 1 ? K - 2 : 0][c] = now[c];
                        de[c] = mul2(w[0][c], dz[K - 1][c]);
#pragma unroll
                        for (int k = 1; k < K; k++) de[c] = fma2(w[k][c], dz[K - 1 - k][c], de[c]);
                    }
                    if (gso != nullptr && t0 + r >= s.len && r < all) {     // in the new history as well
                        Row g2;
                        pairs_of(g2, word_of<WHOLE>(gso + (t0 + r - s.len) * P.C, true, n, P.c_whole));
#pragma unroll
                        for (int c = 0; c < kPairs; c++) de[c] = add2(de[c], g2[c]);
                    }
                    if (r >= K - 1 && r < all) store_row<WHOLE>(out, de, n, P.c_whole);
                    if (K > 1 && r < K - 1 && r < all && t0 == 0 && P.gstate_in != nullptr)
                        store_row<WHOLE>(P.gstate_in + ((long long)b * (K - 1) + r) * P.C + c0, de, n, P.c_whole);
                    out += P.C;
            }
            fetch(slot);
        }
    }
    if (P.part == nullptr) return;
    // sums of the block's walks, in their order
    float (*fold)[K + 1][kChannels] = reinterpret_cast<float (*)[K + 1][kChannels]>(&ring);
    static_assert(sizeof(ring) >= sizeof(float) * kWalks * (K + 1) * kChannels, "the rows' words serve again");
    wait_group<0>();
    __syncthreads();
#pragma unroll
    for (int k = 0; k <= K; k++)
#pragma unroll
        for (int c = 0; c < kPairs; c++) *reinterpret_cast<f32x2 *>(&fold[walk][k][lane * kWord + 2 * c]) = k < K ? gw[k < K ? k : 0][c] : gb[c];
    __syncthreads();
    float *part = P.part + (long long)blockIdx.x * P.C * (K + 1);
    const int first = blockIdx.y * kChannels, here = P.C - first < kChannels ? P.C - first : kChannels;
    for (int i = threadIdx.x; i < here * (K + 1); i += kConvThreads) {
        const int k = i < here * K ? i % K : K, c = i < here * K ? i / K : i - here * K;
        float v = 0.f;
#pragma unroll
        for (int q = 0; q < kWalks; q++) v += fold[q][k][c];
        part[k < K ? (long long)first * K + i : (long long)P.C * K + first + c] = v;
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
    if ((double)p->B * (double)(p->L / (kWalks * kStep) + 1) > 2.0e9) return CAWN_ERR_UNSUPPORTED;
    return CAWN_OK;
}

// Tiles that run at once by the kernels' registers, for each of the blocks across the channels.
int64_t room(const cawn_conv_params *p, bool bwd)
{
    return most((int64_t)sm_count() * (bwd ? kBwdBlocks : fwd_blocks(p->flags != 0 ? 2 : 4)) / ceil_div(p->C, kChannels), 1);
}

ConvParams fill(const cawn_conv_params *p, const void *x, const int64_t *offsets, bool bwd)
{
    ConvParams P = {};
    P.seq = {reinterpret_cast<const long long *>(offsets), p->L, offsets != nullptr ? p->rows : (int64_t)p->B * p->L, p->B};
    P.C = p->C;
    P.x_stride = p->x_stride != 0 ? p->x_stride : p->C;
    P.words = (int)ceil_div(p->C, kWord);
    // as many tiles as there is room for at once
    const int64_t rows = offsets != nullptr ? ceil_div(p->rows, room(p, bwd)) : ceil_div(p->L, most(room(p, bwd) / p->B, 1));
    const int64_t steps = most(ceil_div(rows, kWalks * kStep), 1);
    P.rows = (int)(steps < 1 << 16 ? steps : 1 << 16) * kStep;
    P.tiles = most(ceil_div(p->L, P.rows * kWalks), 1);
    P.all_tiles = P.tiles * p->B;
    P.silu = p->act == CAWN_CONV_ACT_SILU;
    P.x = x;
    P.x_whole = P.x_stride % kWord == 0 && begins_on(x, p->flags != 0 ? 8 : 16);
    P.c_whole = p->C % kWord == 0;
    return P;
}

// Blocks along the tiles in the backward, each with a partial row of sums; what a workspace is sized for never falls as a call grows.
int64_t most_workers(const cawn_conv_params *p)
{
    const int64_t tiles = most(ceil_div(p->L, kWalks * kStep), 1) * p->B, want = room(p, true);
    return tiles < want ? tiles : want;
}

using ConvKernel = void (*)(ConvParams);
template <class T, bool WHOLE> ConvKernel pick(int K, bool bwd)
{
    switch (K) {
    case 1: return bwd ? conv_bwd_kernel<T, 1, WHOLE> : conv_fwd_kernel<T, 1, WHOLE>;
    case 2: return bwd ? conv_bwd_kernel<T, 2, WHOLE> : conv_fwd_kernel<T, 2, WHOLE>;
    case 3: return bwd ? conv_bwd_kernel<T, 3, WHOLE> : conv_fwd_kernel<T, 3, WHOLE>;
    default: return bwd ? conv_bwd_kernel<T, 4, WHOLE> : conv_fwd_kernel<T, 4, WHOLE>;
    }
}
template <class T> ConvKernel pick_step(int K)
{
    return K == 1 ? conv_step_kernel<T, 1> : K == 2 ? conv_step_kernel<T, 2> : K == 3 ? conv_step_kernel<T, 3> : conv_step_kernel<T, 4>;
}
ConvKernel pick(const cawn_conv_params *p, const ConvParams &P, bool bwd)
{
    const bool whole = P.x_whole && P.c_whole;
    return p->flags != 0 ? (whole ? pick<bf16, true>(p->K, bwd) : pick<bf16, false>(p->K, bwd)) : (whole ? pick<float, true>(p->K, bwd) : pick<float, false>(p->K, bwd));
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
    if (!all_aligned16(weight, bias, state_in, y, state_out) || !elements_aligned(params->flags, x)) return CAWN_ERR_MISALIGNED;
    ConvParams P = fill(params, x, offsets, false);
    P.w = weight; P.b = bias; P.state_in = state_in; P.y = y; P.state_out = state_out;
    if (params->L == 1 && offsets == nullptr && ceil_div(params->B, kTokens) <= 65535)
        return status_of(launch<true>(params->flags != 0 ? pick_step<bf16>(params->K) : pick_step<float>(params->K),
                                      dim3((unsigned)ceil_div(P.words, kConvThreads), (unsigned)ceil_div(params->B, kTokens)), dim3(kConvThreads), 0,
                                      static_cast<cudaStream_t>(cuda_stream), P));
    return status_of(launch<true>(pick(params, P, false), dim3((unsigned)P.all_tiles, (unsigned)ceil_div(P.words, kLanes)), dim3(kConvThreads), 0,
                                  static_cast<cudaStream_t>(cuda_stream), P));
}

extern "C" int cawn_short_conv_workspace_bytes(const cawn_conv_params *params, size_t *bytes)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (bytes == nullptr) return CAWN_ERR_NULL_POINTER;
    *bytes = (size_t)most_workers(params) * params->C * (params->K + 1) * sizeof(float);
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
    if (!all_aligned16(weight, bias, state_in, grad_y, grad_state_out, grad_x, grad_weight, grad_bias, grad_state_in, workspace) || !elements_aligned(params->flags, x))
        return CAWN_ERR_MISALIGNED;
    ConvParams P = fill(params, x, offsets, true);
    const int64_t want = room(params, true), blocks = P.all_tiles < want ? P.all_tiles : want, cols = (int64_t)params->C * (params->K + 1);
    if (sums && workspace_bytes < (size_t)blocks * cols * sizeof(float)) return CAWN_ERR_WORKSPACE_TOO_SMALL;
    P.w = weight; P.b = bias; P.state_in = state_in; P.gy = grad_y; P.gstate_out = grad_state_out;
    P.gx = grad_x; P.gstate_in = grad_state_in; P.part = sums ? static_cast<float *>(workspace) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    rc = status_of(launch<true>(pick(params, P, true), dim3((unsigned)blocks, (unsigned)ceil_div(P.words, kLanes)), dim3(kConvThreads), 0, st, P));
    if (rc != CAWN_OK || !sums) return rc;
    PartialSums S = {P.part, blocks, cols, {grad_weight, grad_bias, nullptr}, {(long long)params->C * params->K, params->C, 0}};
    return sum_partials(S, st);
}
