// Selective scan: what its translation units share.
//
// Mathematics, per channel c with N states:  d = softplus(dt + bias),  h_n <- e^{d A_n} h_n + d x B_n,
// y = (sum_n C_n h_n + skip x) silu(z).  B and C belong to a token and a group of channels.
//
// Layout of the work.  A block has 32 channels of one group and one sequence (or a segment of it) and walks its tokens in
// tiles of 16 (blocks of 16 channels would spread more evenly over the multiprocessors, but 8 x 2048 x 2048 x 16 then took 311 us
// instead of 235: each stages B and C for itself).  A thread has CD neighbouring channels and NS states of each; NL lanes share a channel (N up to NL * NS).  In a
// warp lane bits 0-1 are channels, the next log2 NL bits the lane's states, the rest channels again.  A tile's (d, d x) and
// rows of B and C are made floats once, in shared memory; the next tile is fetched while one is computed.  What a
// thread reads there for a token is 8 bytes a channel and 8 a state, so two channels by four states (6 bytes a cell) and not one by
// four (10): shared memory fills 128 bytes of registers a clock, and that was the bound.
// Bound: a decay is an exponential a cell, and a multiprocessor takes 16 a clock: 119 us for 8 x 2048 x 2048 x 16, whose
// arrays take 42 us of memory's time.
// Few channels: the time axis is cut into segments that run side by side, behind a pass that finds each segment's own end
// state and its sum of d (the decay over a segment is e^{A sum d}), so that every exponential is taken twice.
#pragma once
#include "cawn_seq.cuh"

namespace cawn {

constexpr int kScanChannels = 32, kTile = 16;           // a tile is also what lies between two states that the forward leaves for the backward

struct SelectiveParams {
    Sequences seq;
    const void *x, *dt, *z, *bm, *cm, *gy;
    const float *A, *skip, *dt_bias, *state_in, *gstate_out;
    void *y, *gx, *gdt, *gz;
    float *state_out, *gstate_in, *checkpoints;
    float *seg_state, *seg_time, *first;        // segments' own ends and sums of d; a copy of state_in
    float *part_bc, *part_param;                // backward: partial sums of a block's channels, of a block's tokens
    long long xs, dts, zs, bs, cs;              // elements between rows
    long long param_cols;                       // floats of a row of part_param, a multiple of 4
    long long per;                              // tokens of a segment, a multiple of kTile
    double per_inverse;
    long long param_rows;                       // rows of part_param
    int D, N, G, Dg, blocks;                    // channels of a group, blocks of channels per group
    int S;                                      // segments
    int by_rows;                                // segments' ends, and rows of part_param, are numbered by rows and not by sequences
    int halves;                                 // 2: the backward's first pass takes segments in halves
    int softplus, whole_x, whole_dt, whole_z, whole_d, whole_b, whole_c, whole;     // whole: all of them
};

// log(1 + e^v) = v^+ + log1p(u), u = e^{-|v|} in [0, 1], without loss where it is small: log1p(u) / u by the polynomial of degree
// 8 that fits it best in relative error (found by weighted least squares on Chebyshev points; with its coefficients as floats 6.4e-8, computed in
// floats 1.3e-7).
__device__ __forceinline__ f32x2 softplus_of(f32x2 v)
{
    const float2 f = halves(v);
    const float2 e = halves(mul2(pair(fabsf(f.x), fabsf(f.y)), twice(-kLog2e)));
    const f32x2 u = pair(exp2_fast(e.x), exp2_fast(e.y));
    f32x2 p = twice(5.232693627e-03f);
    p = fma2(p, u, twice(-2.950523980e-02f));
    p = fma2(p, u, twice(7.822596282e-02f));
    p = fma2(p, u, twice(-1.366324723e-01f));
    p = fma2(p, u, twice(1.910600811e-01f));
    p = fma2(p, u, twice(-2.484298199e-01f));
    p = fma2(p, u, twice(3.331909776e-01f));
    p = fma2(p, u, twice(-4.999949336e-01f));
    p = fma2(p, u, twice(9.999999404e-01f));
    return fma2(p, u, pair(fmaxf(f.x, 0.f), fmaxf(f.y, 0.f)));       // a NaN comes through u
}
__device__ __forceinline__ float softplus_of(float v) { return halves(softplus_of(twice(v))).x; }
__device__ __forceinline__ f32x2 chosen(bool c, f32x2 a, f32x2 b) { return c ? a : b; }

// Where a thread of the computing warps is, and what its states are.  The last one or two warps stage the tiles: a thread of
// theirs has kWords words of eight channels and kQuads quads of B (and of C).
constexpr int stage_warps(int states) { return states >= 16 ? 2 : 1; }
template <int NL, int NS, int CD> struct Place {
    static constexpr int kStageWarps = stage_warps(NL * NS), kStagers = 32 * kStageWarps;
    static constexpr int kCompute = 32 * NL / CD, kThreads = kCompute + kStagers, kPad = NL * NS, kPairs = NS / 2, kShift = NL == 2 ? 1 : NL == 4 ? 2 : 3;
    static constexpr int kWords = kTile * 4 / kStagers, kQuads = kTile * kPad / 4 / kStagers;
    static_assert(kQuads * kStagers == kTile * kPad / 4, "whole quads");
    int nl, ch;                 // lane among a channel's, first channel of the block
    __device__ __forceinline__ Place()
    {
        const int lane = threadIdx.x % 32;
        nl = (lane >> 2) & (NL - 1);
        ch = (threadIdx.x / 32 * (32 / NL) + (lane & 3) + 4 * (lane >> (2 + kShift))) * CD;
    }
};
// Two floats of each channel of a row, in shared memory: eight channels and a gap of 16 bytes, so that the stagers' words (four a
// row, two rows at a time) and the lanes' reads of four rows go to different banks.
constexpr int kRowPairs = 40;
__device__ __forceinline__ int slot_of(int ch) { return ch + ch / 8 * 2; }
// One float of each channel of a row.
constexpr int kRowFloats = kScanChannels + 8;
template <int CD> __device__ __forceinline__ void put_channels(float *p, const float (&f)[CD])
{
    if constexpr (CD == 2) *reinterpret_cast<float2 *>(p) = make_float2(f[0], f[1]);
    else *p = f[0];
}
template <int CD> __device__ __forceinline__ void get_channels(float (&f)[CD], const float *p)
{
    if constexpr (CD == 2) {
        const float2 v = *reinterpret_cast<const float2 *>(p);
        f[0] = v.x;
        f[CD - 1] = v.y;
    } else {
        f[0] = *p;
    }
}
// All threads of a block, from whatever place of the code each warp is at.
__device__ __forceinline__ void meet() { asm volatile("barrier.sync 0;" ::: "memory"); }

// This lane's NS of a channel's N floats at p; those past N are zero.
template <int NS> __device__ __forceinline__ void load_states(f32x2 (&h)[NS / 2], const float *p, int n0, int N, bool in)
{
    float f[NS];
    if (in && N % 4 == 0) {
#pragma unroll
        for (int k = 0; k < NS; k += 4) {
            const float4 v = n0 + k < N ? *reinterpret_cast<const float4 *>(p + n0 + k) : make_float4(0.f, 0.f, 0.f, 0.f);
            f[k] = v.x; f[k + 1] = v.y; f[k + 2] = v.z; f[k + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < NS; k++) f[k] = in && n0 + k < N ? p[n0 + k] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < NS / 2; k++) h[k] = pair(f[2 * k], f[2 * k + 1]);
}
template <int NS> __device__ __forceinline__ void store_states(float *p, const f32x2 (&h)[NS / 2], int n0, int N, bool in)
{
    float f[NS];
#pragma unroll
    for (int k = 0; k < NS / 2; k++) {
        const float2 v = halves(h[k]);
        f[2 * k] = v.x;
        f[2 * k + 1] = v.y;
    }
    if (!in) return;
    if (N % 4 == 0) {
#pragma unroll
        for (int k = 0; k < NS; k += 4)
            if (n0 + k < N) *reinterpret_cast<float4 *>(p + n0 + k) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
    } else {
#pragma unroll
        for (int k = 0; k < NS; k++)
            if (n0 + k < N) p[n0 + k] = f[k];
    }
}

// Rates for exponentials of base two.  They are finite (a NaN stays), so that a step of zero, as tokens past the end have, leaves a
// state as it is whatever its rate.
__device__ __forceinline__ float rate_of(float a)
{
    constexpr float most = 3.402823466e38f;
    const float v = a * kLog2e;
    return v < -most ? -most : v > most ? most : v;
}
__device__ __forceinline__ f32x2 rate_of(f32x2 a)
{
    const float2 f = halves(a);
    return pair(rate_of(f.x), rate_of(f.y));
}

__device__ __forceinline__ f32x2 exp2_pair(f32x2 v)
{
    const float2 f = halves(v);
    return pair(exp2_fast(f.x), exp2_fast(f.y));
}
__device__ __forceinline__ float sum_of(f32x2 v)
{
    const float2 f = halves(v);
    return f.x + f.y;
}
template <int NS> __device__ __forceinline__ void row_pairs(f32x2 (&r)[NS / 2], const float *p)
{
#pragma unroll
    for (int k = 0; k < NS / 2; k += 2) {
        const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(p + 2 * k);
        r[k] = v.x;
        r[k + 1] = v.y;
    }
}

// CD neighbouring pairs of floats in shared memory.
template <int CD> __device__ __forceinline__ void two_of(float2 (&d)[CD], const float2 *p)
{
    if constexpr (CD == 2) {
        const float4 v = *reinterpret_cast<const float4 *>(p);
        d[0] = make_float2(v.x, v.y);
        d[CD - 1] = make_float2(v.z, v.w);
    } else {
        d[0] = *p;
    }
}

// The state (or gradient) that comes into a segment: `count` segments' own ends, from `at` by `step`, folded in order.  Four are on their
// way at a time: one after the other they take 0.9 us each, up to 62 of them (in halves, as the backward may have them, 126).
template <int NS> __device__ __forceinline__ void fold_segments(f32x2 (&h)[NS / 2], const SelectiveParams &P, const f32x2 (&A2)[NS / 2], long long at, long long step, int count, int n0, bool in)
{
    constexpr int kAhead = 4;
#pragma unroll 1
    for (int i = 0; i < count; i += kAhead) {
        f32x2 own[kAhead][NS / 2];
        float time[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; q++) {
            const bool there = in && i + q < count;
            const long long segment = at + (i + q) * step;
            load_states<NS>(own[q], P.seg_state + segment * P.N, n0, P.N, there);
            time[q] = there ? P.seg_time[segment] : 0.f;
        }
#pragma unroll
        for (int q = 0; q < kAhead; q++) {
            if (i + q >= count) break;
#pragma unroll
            for (int k = 0; k < NS / 2; k++) h[k] = fma2(exp2_pair(mul2(twice(time[q]), A2[k])), h[k], own[q][k]);
        }
    }
}

// floor(row / per).  The product is off by less than one; a division of long integers is a call, whose registers cost the walk of
// 1 x 32768 x 768 x 16 2% (294 -> 300 us) though it does not come here.
__device__ __forceinline__ long long over_per(const SelectiveParams &P, long long row)
{
    long long q = (long long)((double)row * P.per_inverse);
    q -= q * P.per > row;
    return q + ((q + 1) * P.per <= row);
}
// A sequence's first segment among those that keep an end, and its segments' rows of part_param.
__device__ __forceinline__ long long first_end(const SelectiveParams &P, const Span &s, int b) { return P.by_rows ? over_per(P, s.begin) : (long long)b * (P.S - 1); }
__device__ __forceinline__ long long param_row(const SelectiveParams &P, const Span &s, int b, int seg) { return (P.by_rows ? over_per(P, s.begin) + b : (long long)b * P.S) + seg; }

// First checkpoint of a sequence: those of two sequences never meet, whatever the lengths.
__device__ __forceinline__ long long checkpoint_of(const Span &s, int b) { return s.begin / kTile + b; }

// Blocks that a multiprocessor holds at once: the forward's by the registers it is given, the backward's (of the walk, of which the
// type of the arrays decides too) by shared memory and 255 registers, as is asserted there.
constexpr int resident_blocks(int nl, int ns) { return nl == 2 ? 6 : nl == 4 ? 4 : ns == 4 ? 2 : 1; }
constexpr int resident_walks(int nl, int ns, bool half) { return nl == 2 ? (half ? 5 : 4) : nl == 4 ? (half ? 4 : 3) : ns == 4 ? 2 : 1; }

using SelectiveKernel = void (*)(SelectiveParams);
struct Shape {
    int nl, ns, cd;
    int threads() const { return 32 * (nl / cd + stage_warps(nl * ns)); }
    int resident() const { return resident_blocks(nl, ns); }
    int resident_bwd(bool half) const { return resident_walks(nl, ns, half); }
};
inline Shape shape_of(int N) { return N <= 8 ? Shape{2, 4, 2} : N <= 16 ? Shape{4, 4, 2} : N <= 32 ? Shape{8, 4, 2} : Shape{8, 8, 1}; }
// A launch for the shape: CALL(NL, NS, CD).
#define CAWN_BY_SHAPE(S, CALL) ((S).ns == 8 ? CALL(8, 8, 1) : (S).nl == 8 ? CALL(8, 4, 2) : (S).nl == 4 ? CALL(4, 4, 2) : CALL(2, 4, 2))

// More than 48 KB of shared memory are asked for.
inline int launch_shared(SelectiveKernel k, dim3 grid, int threads, size_t bytes, const SelectiveParams &P, cudaStream_t st)
{
    if (bytes > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != cudaSuccess) return status_of(e);
    }
    return status_of(launch<true>(k, grid, dim3(threads), bytes, st, P));
}

// One call of each kernel family; the grid is (blocks of channels x sequences, segments).
int launch_selective_fwd(const SelectiveParams &P, const Shape &s, bool half, bool summary, cudaStream_t st);
int launch_selective_step(const SelectiveParams &P, bool half, cudaStream_t st);
int launch_selective_bwd(const SelectiveParams &P, const Shape &s, bool half, bool summary, cudaStream_t st);
int launch_selective_bc(const SelectiveParams &P, bool half, void *grad_b, void *grad_c, cudaStream_t st);

}  // namespace cawn
