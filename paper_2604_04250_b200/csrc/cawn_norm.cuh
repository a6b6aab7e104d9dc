// Group norm with an activation, channels last: what its translation units share.
//
// Mathematics (per position and group of M channels): xh = (x - mean) rstd, z = xh w + b, y = act(z).
// Backward with d = w * dL/dz:  dx = rstd (d - mean(d) - xh mean(d xh));  rms form: no mean(d) term.
//
// Each element is read once: a power-of-two team of lanes inside a warp holds a group in registers (NV 16-byte
// words per lane), statistics are two-pass over those registers (mean first, then squares of the differences) and
// meet by shuffles.  A thread keeps its channels and walks over rows.  Both directions should be bound by
// memory, but at 8 elements per thread they run into instructions first: arithmetic is on pairs of floats, and the
// activation is a template argument (with neither, the backward took 54 instructions an element and 73 us for
// 32768 x 768 in bfloat16, twice the memory's time; now 53, and 7 for the sums of the parameters' gradients, which start
// while it drains: 56 together, 4.5 TB/s).
#pragma once
#include "cawn_ops.cuh"

namespace cawn {

struct NormParams {
    const void *x, *gate, *gy;
    void *y, *gx, *ggate;
    const float *w, *b;
    float *part;                 // backward: [row blocks][2][C] partial sums, NULL if not wanted
    long long N, x_stride, gate_stride;
    int G, M, C, act;
    int TX, TY;                  // column slots (LPG lanes per group) and row lanes of a block; TX a multiple of LPG.
                                 // Threads past TX * TY fill up the last warp and stay idle.
    long long rows_per_block;    // rows of the walk of one block
    float eps, inv_m;
    bool rms;
};

// How a call is cut: a team of `lpg` lanes with `nv` words of V elements per lane for each group
// (lpg = 0: the wide kernel), TX column slots x TY row lanes per block, `bx` blocks along the rows.
struct Cut {
    int v, lpg, nv, TX, TY, bx, by;
    int most;                    // bx at most, for this or any smaller N: what a workspace is sized for
    long long rows;
};

inline int threads_of(const Cut &c) { return (c.TX * c.TY + 31) / 32 * 32; }

inline Cut cut_of(const cawn_norm_params *p, bool backward)
{
    Cut c = {};
    const int per = p->flags != 0 ? 8 : 4;
    const int64_t xs = p->x_stride, gs = p->gate_stride;
    // 16-byte words need every row and every group to start on one
    c.v = p->M % per == 0 && xs % per == 0 && gs % per == 0 ? per : 1;
    const int words = (p->M + c.v - 1) / c.v;
    c.lpg = 4;
    while (c.lpg < 32 && c.lpg < words) c.lpg *= 2;
    const int need = (words + c.lpg - 1) / c.lpg;
    c.nv = need <= 1 ? 1 : need <= 2 ? 2 : need <= 4 ? 4 : 8;
    const int limit = c.v == 8 ? 4 : 8;          // registers: at most 32 elements per thread
    if (need > limit) { c.lpg = 0; c.nv = 0; }
    const int sms = sm_count();
    if (c.lpg == 0) {
        c.by = p->G;
        const int64_t want = backward ? (int64_t)sms * 4 / p->G + 1 : p->N;
        c.bx = (int)(p->N < want ? p->N : want < 65535 * 16 ? want : 65535 * 16);
        if (c.bx < 1) c.bx = 1;
        c.most = c.bx;
        c.rows = (p->N + c.bx - 1) / c.bx;
        return c;
    }
    const int64_t slots = (int64_t)p->G * c.lpg;
    c.TX = slots < 256 ? (int)slots : 256;
    c.by = (int)((slots + c.TX - 1) / c.TX);
    c.TY = c.TX >= 256 ? 1 : 256 / c.TX;
    // forward: four rows a thread once there are enough rows to fill the GPU with that; backward: as many blocks
    // as are resident at once by the registers a thread takes (by elements held), so that no second, mostly
    // empty wave follows and few partial rows are left to sum
    int64_t bx;
    if (backward) {
        const int held = c.nv * c.v, regs = held <= 1 ? 32 : held <= 4 ? 64 : held <= 8 ? 96 : held <= 16 ? 176 : 255;
        int64_t each = 4 * (16384 / (32 * regs)) / (threads_of(c) / 32);       // a scheduler has 16384 registers
        if (each > 8) each = 8;
        if (each < 1) each = 1;
        bx = sms * each / c.by;
    } else {
        const int64_t each = p->N * c.by >= (int64_t)sms * c.TY * 32 ? 4 : 1;
        bx = (p->N + c.TY * each - 1) / (c.TY * each);
    }
    const int64_t most = (p->N + c.TY - 1) / c.TY;
    if (bx > most) bx = most;
    if (bx < 1) bx = 1;
    c.most = (int)bx;            // whole turns of the row lanes below can take fewer blocks for more rows
    c.rows = (p->N + bx - 1) / bx;
    c.rows = (c.rows + c.TY - 1) / c.TY * c.TY;
    c.bx = (int)((p->N + c.rows - 1) / (c.rows > 0 ? c.rows : 1));
    if (c.bx < 1) c.bx = 1;
    return c;
}


using NormKernel = void (*)(NormParams);
// The kernel of a cut, for the storage type and activation of the call.
NormKernel norm_fwd_pick(const Cut &c, bool half, int act);
NormKernel norm_bwd_pick(const Cut &c, bool half, int act);

#ifdef __CUDACC__
constexpr int kNormThreads = 256;

template <int LPG> __device__ __forceinline__ float team_sum(float v)
{
#pragma unroll
    for (int o = LPG / 2; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ float sigmoidf(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }

// The unit of arithmetic: a pair of floats, or one float where a word is one element.
template <int V> struct UnitOf { using type = f32x2; static constexpr int N = V / 2; };
template <> struct UnitOf<1> { using type = float; static constexpr int N = 1; };
__device__ __forceinline__ float add2(float a, float b) { return a + b; }
__device__ __forceinline__ float mul2(float a, float b) { return a * b; }
__device__ __forceinline__ float fma2(float a, float b, float c) { return fmaf(a, b, c); }
template <class U> __device__ __forceinline__ U both(float v);
template <> __device__ __forceinline__ float both<float>(float v) { return v; }
template <> __device__ __forceinline__ f32x2 both<f32x2>(float v) { return pair(v, v); }
__device__ __forceinline__ float total(float v) { return v; }
__device__ __forceinline__ float total(f32x2 v) { const float2 h = halves(v); return h.x + h.y; }
__device__ __forceinline__ float sigmoid2(float v) { return sigmoidf(v); }
__device__ __forceinline__ f32x2 sigmoid2(f32x2 v)
{
    const float2 e = halves(mul2(v, pair(-1.44269504f, -1.44269504f)));
    const float2 d = halves(add2(pair(exp2_fast(e.x), exp2_fast(e.y)), pair(1.f, 1.f)));
    return pair(__fdividef(1.f, d.x), __fdividef(1.f, d.y));
}

// One word per lane and position, as stored and as units.
template <class T, int V> struct Word {
    using U = typename UnitOf<V>::type;
    static constexpr int N = UnitOf<V>::N, W = V * (int)sizeof(T) / 16;
    uint4 w[W];
    __device__ __forceinline__ void get(const T *p)
    {
#pragma unroll
        for (int i = 0; i < W; i++) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void put(T *p) const
    {
#pragma unroll
        for (int i = 0; i < W; i++) reinterpret_cast<uint4 *>(p)[i] = w[i];
    }
    __device__ __forceinline__ void to(U (&f)[N]) const
    {
        const unsigned *u = &w[0].x;
#pragma unroll
        for (int i = 0; i < N; i++)
            f[i] = sizeof(T) == 4 ? pair(__uint_as_float(u[2 * i % (4 * W)]), __uint_as_float(u[(2 * i + 1) % (4 * W)]))
                                  : pair(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
    }
    __device__ __forceinline__ void from(const U (&f)[N])
    {
        unsigned *u = &w[0].x;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float2 v = halves(f[i]);
            if (sizeof(T) == 4) {
                u[2 * i % (4 * W)] = __float_as_uint(v.x);
                u[(2 * i + 1) % (4 * W)] = __float_as_uint(v.y);
            } else {
                u[i] = pack_bf16(v.x, v.y);
            }
        }
    }
};
template <class T> struct Word<T, 1> {
    using U = float;
    static constexpr int N = 1;
    T w;
    __device__ __forceinline__ void get(const T *p) { w = *p; }
    __device__ __forceinline__ void put(T *p) const { *p = w; }
    __device__ __forceinline__ void to(float (&f)[1]) const { f[0] = widen(w); }
    __device__ __forceinline__ void from(const float (&f)[1]) { w = narrow<T>(f[0]); }
};
// V weights (or biases) of a word
template <int V> __device__ __forceinline__ void load_units(typename UnitOf<V>::type (&f)[UnitOf<V>::N], const float *p, float missing)
{
    using U = typename UnitOf<V>::type;
#pragma unroll
    for (int i = 0; i < UnitOf<V>::N; i++) {
        if (p == nullptr) f[i] = both<U>(missing);
        else f[i] = *reinterpret_cast<const U *>(p + i * (V == 1 ? 1 : 2));
    }
}

// A thread's place: block-local row lane, and its words' channels (a group's words are dealt to the team round
// robin, so that a team's accesses are contiguous); ch[j] < 0 marks words past the group's end.
template <int LPG, int V, int NV>
__device__ __forceinline__ int my_place(const NormParams &P, int (&ch)[NV])
{
    const int slot = blockIdx.y * P.TX + threadIdx.x % P.TX, group = slot / LPG, lane = slot % LPG;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int in_group = (j * LPG + lane) * V;
        ch[j] = group < P.G && in_group < P.M ? group * P.M + in_group : -1;
    }
    return threadIdx.x / P.TX;
}

// Normalised values in place of x (zero where there is no channel); returns rstd.
template <int LPG, class U, int N, int NV>
__device__ __forceinline__ float normalise(U (&f)[NV][N], const int (&ch)[NV], const NormParams &P)
{
    if (!P.rms) {
        U s = both<U>(0.f);
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int i = 0; i < N; i++) s = add2(s, f[j][i]);
        const U minus = both<U>(-team_sum<LPG>(total(s)) * P.inv_m);
#pragma unroll
        for (int j = 0; j < NV; j++)
            if (ch[j] >= 0)
#pragma unroll
                for (int i = 0; i < N; i++) f[j][i] = add2(f[j][i], minus);
    }
    U q = both<U>(0.f);
#pragma unroll
    for (int j = 0; j < NV; j++)
#pragma unroll
        for (int i = 0; i < N; i++) q = fma2(f[j][i], f[j][i], q);
    const float rstd = rsqrtf(team_sum<LPG>(total(q)) * P.inv_m + P.eps);
    const U r = both<U>(rstd);
#pragma unroll
    for (int j = 0; j < NV; j++)
#pragma unroll
        for (int i = 0; i < N; i++) f[j][i] = mul2(f[j][i], r);
    return rstd;
}

// dL/dz from dL/dy; for the gate form also dL/dgate (in g).
template <int ACT, class U> __device__ __forceinline__ U act_backward(U dy, U z, U &g)
{
    const U one = both<U>(1.f), minus = both<U>(-1.f);
    if (ACT == CAWN_NORM_ACT_SILU) {            // s (1 + z (1 - s))
        const U s = sigmoid2(z);
        return mul2(dy, fma2(mul2(z, s), fma2(s, minus, one), s));
    }
    if (ACT == CAWN_NORM_ACT_GATE) {
        const U s = sigmoid2(g), gs = mul2(g, s);
        g = mul2(mul2(dy, z), fma2(gs, fma2(s, minus, one), s));
        return mul2(dy, gs);
    }
    return dy;
}

#endif

}  // namespace cawn
