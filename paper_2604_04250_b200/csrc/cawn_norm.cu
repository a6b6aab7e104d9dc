// Group norm with an activation, channels last: forward and backward.
//
// Mathematics (per position and group of M channels): xh = (x - mean) rstd, z = xh w + b, y = act(z).
// Backward with d = w * dL/dz:  dx = rstd (d - mean(d) - xh mean(d xh));  rms form: no mean(d) term.
// Both are bound by memory, so each element is read once: a power-of-two team of lanes inside a warp
// holds a group in registers (NV 16-byte words per lane), statistics are two-pass over those
// registers (mean first, then squares of the differences) and meet by shuffles.
// A thread keeps its channels and walks over rows, so weights are loaded once per thread and the
// parameter gradients are register sums; they are folded per block in shared memory, written as one
// partial row per block, and summed in double in a fixed order by a second launch.
#include "cawn_ops.cuh"

namespace cawn {
namespace {

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

template <int LPG> __device__ __forceinline__ float team_sum(float v)
{
#pragma unroll
    for (int o = LPG / 2; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ float sigmoidf(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }

// A row's words as they are stored, so that the next row can be on its way without taking a float register per
// element; V = 1 keeps the element itself.
template <class T, int V> struct Word {
    static constexpr int N = V * (int)sizeof(T) / 16;
    uint4 w[N];
    __device__ __forceinline__ void get(const T *p) { for (int i = 0; i < N; i++) w[i] = reinterpret_cast<const uint4 *>(p)[i]; }
    __device__ __forceinline__ void to(float (&f)[V]) const
    {
        const unsigned *u = &w[0].x;
#pragma unroll
        for (int i = 0; i < V; i++)
            f[i] = sizeof(T) == 4 ? __uint_as_float(u[i]) : __uint_as_float(i % 2 == 0 ? u[i / 2] << 16 : u[i / 2] & 0xffff0000u);
    }
};
template <class T> struct Word<T, 1> {
    T w;
    __device__ __forceinline__ void get(const T *p) { w = *p; }
    __device__ __forceinline__ void to(float (&f)[1]) const { f[0] = widen(w); }
};
template <class T, int V, int NV>
__device__ __forceinline__ void fetch_row(Word<T, V> (&r)[NV], const T *row, const int (&ch)[NV], bool live)
{
#pragma unroll
    for (int j = 0; j < NV; j++)
        if (live && ch[j] >= 0) r[j].get(row + ch[j]);
}
template <class T, int V, int NV>
__device__ __forceinline__ void unpack_row(float (&f)[NV][V], const Word<T, V> (&r)[NV], const int (&ch)[NV], bool live)
{
#pragma unroll
    for (int j = 0; j < NV; j++) {
        if (live && ch[j] >= 0) {
            r[j].to(f[j]);
        } else {
#pragma unroll
            for (int e = 0; e < V; e++) f[j][e] = 0.f;
        }
    }
}

template <class T, int V, int NV>
__device__ __forceinline__ void load_row(float (&f)[NV][V], const T *row, const int (&ch)[NV], bool live)
{
#pragma unroll
    for (int j = 0; j < NV; j++) {
        if (live && ch[j] >= 0) {
            load_vec(f[j], row + ch[j]);
        } else {
#pragma unroll
            for (int e = 0; e < V; e++) f[j][e] = 0.f;
        }
    }
}

// Normalised values in place of x; returns rstd.  ch[j] < 0 marks words past the group's end.
template <int LPG, int V, int NV>
__device__ __forceinline__ float normalise(float (&f)[NV][V], const int (&ch)[NV], const NormParams &P)
{
    float mean = 0.f;
    if (!P.rms) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < V; e++) s += f[j][e];
        mean = team_sum<LPG>(s) * P.inv_m;
    }
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < NV; j++)
#pragma unroll
        for (int e = 0; e < V; e++) {
            f[j][e] -= mean;
            q += ch[j] >= 0 ? f[j][e] * f[j][e] : 0.f;
        }
    const float rstd = rsqrtf(team_sum<LPG>(q) * P.inv_m + P.eps);
#pragma unroll
    for (int j = 0; j < NV; j++)
#pragma unroll
        for (int e = 0; e < V; e++) f[j][e] *= rstd;
    return rstd;
}

// A thread's place: block-local row, and its words' channels (a group's words are dealt to the team
// round robin, so that a team's accesses are contiguous).
template <int LPG, int V, int NV>
__device__ __forceinline__ void my_place(const NormParams &P, int &ty, int (&ch)[NV], float (&w)[NV][V], float (&b)[NV][V])
{
    const int tx = threadIdx.x % P.TX, slot = blockIdx.y * P.TX + tx, group = slot / LPG, lane = slot % LPG;
    ty = threadIdx.x / P.TX;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int in_group = (j * LPG + lane) * V;
        ch[j] = group < P.G && in_group < P.M ? group * P.M + in_group : -1;
#pragma unroll
        for (int e = 0; e < V; e++) { w[j][e] = 1.f; b[j][e] = 0.f; }
        if (ch[j] >= 0 && P.w != nullptr) load_vec(w[j], P.w + ch[j]);
        if (ch[j] >= 0 && P.b != nullptr) load_vec(b[j], P.b + ch[j]);
    }
}

template <class T, int LPG, int V, int NV>
__global__ void __launch_bounds__(256) norm_fwd_kernel(const NormParams P)
{
    int ty, ch[NV];
    float w[NV][V], b[NV][V];
    my_place<LPG>(P, ty, ch, w, b);
    const int TY = P.TY;
    const long long r0 = (long long)blockIdx.x * P.rows_per_block;
    const long long r1 = r0 + P.rows_per_block < P.N ? r0 + P.rows_per_block : P.N;
    // the bound is the block's, not the row's: whole warps stay in the loop for the shuffles
    for (long long base = r0; base < r1; base += TY) {
        const long long r = base + ty;
        const bool live = r < r1 && ty < TY;
        float f[NV][V], g[NV][V];
        load_row(f, static_cast<const T *>(P.x) + r * P.x_stride, ch, live);
        if (P.act == CAWN_NORM_ACT_GATE) load_row(g, static_cast<const T *>(P.gate) + r * P.gate_stride, ch, live);
        normalise<LPG>(f, ch, P);
#pragma unroll
        for (int j = 0; j < NV; j++) {
#pragma unroll
            for (int e = 0; e < V; e++) {
                float z = fmaf(f[j][e], w[j][e], b[j][e]);
                if (P.act == CAWN_NORM_ACT_SILU) z *= sigmoidf(z);
                if (P.act == CAWN_NORM_ACT_GATE) z *= g[j][e] * sigmoidf(g[j][e]);
                f[j][e] = z;
            }
            if (live && ch[j] >= 0) store_vec(static_cast<T *>(P.y) + r * P.C + ch[j], f[j]);
        }
    }
}

// dL/dz from dL/dy; for the gate form also dL/dgate (in g).
__device__ __forceinline__ float act_backward(int act, float dy, float z, float &g)
{
    if (act == CAWN_NORM_ACT_SILU) {
        const float s = sigmoidf(z);
        return dy * s * (1.f + z * (1.f - s));
    }
    if (act == CAWN_NORM_ACT_GATE) {
        const float s = sigmoidf(g), gv = g;
        g = dy * z * s * (1.f + gv * (1.f - s));
        return dy * gv * s;
    }
    return dy;
}

template <class T, int LPG, int V, int NV>
__global__ void __launch_bounds__(256) norm_bwd_kernel(const NormParams P)
{
    constexpr int AHEAD = NV * V <= 8 ? 2 : 1;      // rows on their way: what registers allow
    extern __shared__ float fold[];                 // [2][TX * NV * V]
    int ty, ch[NV];
    float w[NV][V], b[NV][V], sw[NV][V] = {}, sb[NV][V] = {};
    my_place<LPG>(P, ty, ch, w, b);
    const int TY = P.TY, tx = threadIdx.x % P.TX;
    const long long r0 = (long long)blockIdx.x * P.rows_per_block;
    const long long r1 = r0 + P.rows_per_block < P.N ? r0 + P.rows_per_block : P.N;
    const bool gated = P.act == CAWN_NORM_ACT_GATE;
    struct Row { Word<T, V> f[NV], d[NV], g[NV]; };
    auto fetch = [&](Row &w, long long r) {
        const bool live = r < r1 && ty < TY;
        fetch_row(w.f, static_cast<const T *>(P.x) + r * P.x_stride, ch, live);
        fetch_row(w.d, static_cast<const T *>(P.gy) + r * P.C, ch, live);
        if (gated) fetch_row(w.g, static_cast<const T *>(P.gate) + r * P.gate_stride, ch, live);
    };
    auto work = [&](Row &row, long long r) {
        const bool live = r < r1 && ty < TY;
        float f[NV][V], g[NV][V], d[NV][V];
        unpack_row(f, row.f, ch, live);
        unpack_row(d, row.d, ch, live);
        if (gated) unpack_row(g, row.g, ch, live);
        fetch(row, r + AHEAD * TY);     // a later row, while this one is worked on
        const float rstd = normalise<LPG>(f, ch, P);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; j++) {
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float z = fmaf(f[j][e], w[j][e], b[j][e]);
                const float dz = act_backward(P.act, d[j][e], z, g[j][e]);
                if (live) {
                    sw[j][e] = fmaf(dz, f[j][e], sw[j][e]);
                    sb[j][e] += dz;
                }
                d[j][e] = ch[j] >= 0 ? dz * w[j][e] : 0.f;
                s1 += d[j][e];
                s2 = fmaf(d[j][e], f[j][e], s2);
            }
        }
        s2 = team_sum<LPG>(s2) * P.inv_m;
        s1 = P.rms ? 0.f : team_sum<LPG>(s1) * P.inv_m;
#pragma unroll
        for (int j = 0; j < NV; j++) {
#pragma unroll
            for (int e = 0; e < V; e++) d[j][e] = rstd * (d[j][e] - s1 - f[j][e] * s2);
            if (live && ch[j] >= 0) {
                store_vec(static_cast<T *>(P.gx) + r * P.C + ch[j], d[j]);
                if (P.act == CAWN_NORM_ACT_GATE) store_vec(static_cast<T *>(P.ggate) + r * P.C + ch[j], g[j]);
            }
        }
    };
    Row row[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; i++) fetch(row[i], r0 + ty + i * TY);
    // the bound is the block's, not the row's: whole warps stay in the loop for the shuffles
    for (long long base = r0; base < r1; base += AHEAD * TY)
#pragma unroll
        for (int i = 0; i < AHEAD; i++) work(row[i], base + ty + i * TY);
    if (P.part == nullptr) return;
    // row lanes fold their sums one after the other in a fixed order: shared memory holds one row
    for (int turn = 0; turn < TY; turn++) {
        if (ty == turn) {
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const int at = (j * V + e) * P.TX + tx, half = NV * V * P.TX;
                    fold[at] = turn == 0 ? sw[j][e] : fold[at] + sw[j][e];
                    fold[half + at] = turn == 0 ? sb[j][e] : fold[half + at] + sb[j][e];
                }
        }
        __syncthreads();
    }
    if (ty == 0) {
        float *pw = P.part + (size_t)blockIdx.x * 2 * P.C;
#pragma unroll
        for (int j = 0; j < NV; j++)
            if (ch[j] >= 0)
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const int at = (j * V + e) * P.TX + tx, half = NV * V * P.TX;
                    pw[ch[j] + e] = fold[at];
                    pw[P.C + ch[j] + e] = fold[half + at];
                }
    }
}

// Groups that a team cannot hold in registers: a block per group and stretch of rows, re-reading the
// row from cache for each pass.  Column sums live in shared memory (2 M floats, M <= 4096).
constexpr int kWideThreads = 256;

__device__ __forceinline__ float block_sum(float v, float *red)
{
    v = team_sum<32>(v);
    __syncthreads();
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    float s = 0.f;
    for (int i = 0; i < kWideThreads / 32; i++) s += red[i];
    return s;
}

template <class T, bool BWD>
__global__ void __launch_bounds__(kWideThreads) norm_wide_kernel(const NormParams P)
{
    __shared__ float red[kWideThreads / 32];
    extern __shared__ float fold[];
    const int c0 = blockIdx.y * P.M;
    const long long r0 = (long long)blockIdx.x * P.rows_per_block;
    const long long r1 = r0 + P.rows_per_block < P.N ? r0 + P.rows_per_block : P.N;
    if (BWD && P.part != nullptr)
        for (int i = threadIdx.x; i < 2 * P.M; i += kWideThreads) fold[i] = 0.f;   // each thread its own columns
    for (long long r = r0; r < r1; r++) {
        const T *x = static_cast<const T *>(P.x) + r * P.x_stride + c0;
        const T *gate = P.act == CAWN_NORM_ACT_GATE ? static_cast<const T *>(P.gate) + r * P.gate_stride + c0 : nullptr;
        float s = 0.f, q = 0.f;
        if (!P.rms)
            for (int i = threadIdx.x; i < P.M; i += kWideThreads) s += widen(x[i]);
        const float mean = P.rms ? 0.f : block_sum(s, red) * P.inv_m;
        for (int i = threadIdx.x; i < P.M; i += kWideThreads) {
            const float v = widen(x[i]) - mean;
            q += v * v;
        }
        const float rstd = rsqrtf(block_sum(q, red) * P.inv_m + P.eps);
        float s1 = 0.f, s2 = 0.f;
        for (int pass = 0; pass < (BWD ? 2 : 1); pass++) {
            for (int i = threadIdx.x; i < P.M; i += kWideThreads) {
                const float xh = (widen(x[i]) - mean) * rstd;
                const float wt = P.w != nullptr ? P.w[c0 + i] : 1.f, z = fmaf(xh, wt, P.b != nullptr ? P.b[c0 + i] : 0.f);
                float g = gate != nullptr ? widen(gate[i]) : 0.f;
                if constexpr (!BWD) {
                    float y = z;
                    if (P.act == CAWN_NORM_ACT_SILU) y *= sigmoidf(z);
                    if (P.act == CAWN_NORM_ACT_GATE) y *= g * sigmoidf(g);
                    static_cast<T *>(P.y)[r * P.C + c0 + i] = narrow<T>(y);
                } else {
                    const float dz = act_backward(P.act, widen(static_cast<const T *>(P.gy)[r * P.C + c0 + i]), z, g);
                    if (pass == 0) {
                        s1 += dz * wt;
                        s2 += dz * wt * xh;
                    } else {
                        if (P.part != nullptr) {
                            fold[i] += dz * xh;
                            fold[P.M + i] += dz;
                        }
                        static_cast<T *>(P.gx)[r * P.C + c0 + i] = narrow<T>(rstd * (dz * wt - s1 - xh * s2));
                        if (gate != nullptr) static_cast<T *>(P.ggate)[r * P.C + c0 + i] = narrow<T>(g);
                    }
                }
            }
            if (BWD && pass == 0) {
                s2 = block_sum(s2, red) * P.inv_m;
                s1 = P.rms ? 0.f : block_sum(s1, red) * P.inv_m;
            }
        }
    }
    if (BWD && P.part != nullptr) {
        float *pw = P.part + (size_t)blockIdx.x * 2 * P.C + c0;
        for (int i = threadIdx.x; i < P.M; i += kWideThreads) {
            pw[i] = fold[i];
            pw[P.C + i] = fold[P.M + i];
        }
    }
}

// Parameter gradients: 32 columns a block, 32 row lanes with two sums each, doubles, fixed order.
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float *part, int blocks, int C, float *gw, float *gb)
{
    __shared__ double sums[32][33];
    const int x = threadIdx.x % 32, lane = threadIdx.x / 32, col = blockIdx.x * 32 + x;
    double s = 0.0, t = 0.0;
    if (col < 2 * C) {
        int i = lane;
        for (; i + 32 < blocks; i += 64) {
            s += (double)part[(size_t)i * 2 * C + col];
            t += (double)part[(size_t)(i + 32) * 2 * C + col];
        }
        if (i < blocks) s += (double)part[(size_t)i * 2 * C + col];
    }
    sums[lane][x] = s + t;
    __syncthreads();
    // a warp per column: lane x holds row lane x of column `lane`
    s = sums[x][lane];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int mine = blockIdx.x * 32 + lane;
    if (x == 0 && mine < 2 * C) {
        if (mine < C) {
            if (gw != nullptr) gw[mine] = (float)s;
        } else if (gb != nullptr) {
            gb[mine - C] = (float)s;
        }
    }
}

// How a call is cut: a team of `lpg` lanes with `nv` words of V elements per lane for each group
// (lpg = 0: the wide kernel), TX column slots x TY row lanes per block, `bx` blocks along the rows.
struct Cut {
    int v, lpg, nv, TX, TY, bx, by;
    long long rows;
};

inline int threads_of(const Cut &c) { return (c.TX * c.TY + 31) / 32 * 32; }

Cut cut_of(const cawn_norm_params *p, bool backward)
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
        const int held = c.nv * c.v, regs = held <= 1 ? 40 : held <= 4 ? 72 : held <= 8 ? 112 : held <= 16 ? 168 : 255;
        int64_t each = 65536 / (regs * (int64_t)threads_of(c));
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
    c.rows = (p->N + bx - 1) / bx;
    c.rows = (c.rows + c.TY - 1) / c.TY * c.TY;
    c.bx = (int)((p->N + c.rows - 1) / (c.rows > 0 ? c.rows : 1));
    if (c.bx < 1) c.bx = 1;
    return c;
}

int check(const cawn_norm_params *p)
{
    if (p == nullptr) return CAWN_ERR_NULL_POINTER;
    if (p->struct_size != sizeof(cawn_norm_params)) return CAWN_ERR_INVALID_ARG;
    if (p->N < 0 || p->G < 1 || p->M < 1 || !(p->eps >= 0.f) || p->reserved != 0 || !storage_flags_ok(p->flags) ||
        p->act < CAWN_NORM_ACT_NONE || p->act > CAWN_NORM_ACT_GATE || (p->rms != 0 && p->rms != 1))
        return CAWN_ERR_INVALID_ARG;
    const int64_t C = (int64_t)p->G * p->M;
    if ((p->x_stride != 0 && p->x_stride < C) || (p->gate_stride != 0 && p->gate_stride < C)) return CAWN_ERR_INVALID_ARG;
    if (p->M > 4096 || C > (1 << 24) || p->G > 65535) return CAWN_ERR_UNSUPPORTED;
    const int64_t wide = p->x_stride > p->gate_stride ? p->x_stride : p->gate_stride;
    if ((double)p->N * (double)(wide > C ? wide : C) > 1.0e17 || p->N > ((int64_t)1 << 32)) return CAWN_ERR_UNSUPPORTED;
    return CAWN_OK;
}

NormParams fill(const cawn_norm_params *p, const Cut &c)
{
    NormParams P = {};
    P.N = p->N; P.G = p->G; P.M = p->M; P.C = p->G * p->M; P.act = p->act;
    P.x_stride = p->x_stride != 0 ? p->x_stride : P.C;
    P.gate_stride = p->gate_stride != 0 ? p->gate_stride : P.C;
    P.TX = c.TX; P.TY = c.TY; P.rows_per_block = c.rows;
    P.eps = p->eps; P.inv_m = 1.f / (float)p->M; P.rms = p->rms != 0;
    return P;
}

template <class T, int V> using Kernel = void (*)(NormParams);

template <class T, int V, int LPG, int NV> Kernel<T, V> pick2(bool bwd)
{
    return bwd ? norm_bwd_kernel<T, LPG, V, NV> : norm_fwd_kernel<T, LPG, V, NV>;
}
template <class T, int V> Kernel<T, V> pick(const Cut &c, bool bwd)
{
    if (c.lpg == 4) return pick2<T, V, 4, 1>(bwd);
    if (c.lpg == 8) return pick2<T, V, 8, 1>(bwd);
    if (c.lpg == 16) return pick2<T, V, 16, 1>(bwd);
    if (c.nv == 1) return pick2<T, V, 32, 1>(bwd);
    if (c.nv == 2) return pick2<T, V, 32, 2>(bwd);
    if constexpr (V == 8) return pick2<T, V, 32, 4>(bwd);
    else return c.nv == 4 ? pick2<T, V, 32, 4>(bwd) : pick2<T, V, 32, 8>(bwd);
}

int run(const cawn_norm_params *p, const Cut &c, const NormParams &P, bool bwd, cudaStream_t st)
{
    const bool half = p->flags != 0;
    if (c.lpg == 0) {
        const size_t smem = bwd && P.part != nullptr ? (size_t)2 * P.M * sizeof(float) : 0;
        Kernel<float, 1> k = half ? (bwd ? norm_wide_kernel<bf16, true> : norm_wide_kernel<bf16, false>)
                                  : (bwd ? norm_wide_kernel<float, true> : norm_wide_kernel<float, false>);
        return status_of(launch(k, dim3(c.bx, c.by), dim3(kWideThreads), smem, st, P));
    }
    Kernel<float, 1> k = half ? (c.v == 1 ? pick<bf16, 1>(c, bwd) : pick<bf16, 8>(c, bwd))
                              : (c.v == 1 ? pick<float, 1>(c, bwd) : pick<float, 4>(c, bwd));
    const int threads = threads_of(c);
    const size_t smem = bwd && P.part != nullptr ? (size_t)2 * c.TX * c.nv * c.v * sizeof(float) : 0;
    return status_of(launch(k, dim3(c.bx, c.by), dim3(threads), smem, st, P));
}

}  // namespace
}  // namespace cawn

extern "C" int cawn_group_norm_fwd(const cawn_norm_params *params, const void *x, const float *weight, const float *bias,
                                   const void *gate, void *y, void *cuda_stream)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (params->N == 0) return CAWN_OK;
    if (x == nullptr || y == nullptr || (params->act == CAWN_NORM_ACT_GATE && gate == nullptr)) return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(x, weight, bias, gate, y)) return CAWN_ERR_MISALIGNED;
    const Cut c = cut_of(params, false);
    NormParams P = fill(params, c);
    P.x = x; P.w = weight; P.b = bias; P.gate = gate; P.y = y;
    return run(params, c, P, false, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int cawn_group_norm_workspace_bytes(const cawn_norm_params *params, size_t *bytes)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (bytes == nullptr) return CAWN_ERR_NULL_POINTER;
    *bytes = (size_t)cut_of(params, true).bx * 2 * params->G * params->M * sizeof(float);
    return CAWN_OK;
}

extern "C" int cawn_group_norm_bwd(const cawn_norm_params *params, const void *x, const float *weight, const float *bias,
                                   const void *gate, const void *grad_y, void *grad_x, void *grad_gate, float *grad_weight,
                                   float *grad_bias, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    const bool gated = params->act == CAWN_NORM_ACT_GATE, sums = grad_weight != nullptr || grad_bias != nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const Cut c = cut_of(params, true);
    const int C = params->G * params->M;
    if (params->N > 0 && (x == nullptr || grad_y == nullptr || grad_x == nullptr || (gated && (gate == nullptr || grad_gate == nullptr))))
        return CAWN_ERR_NULL_POINTER;
    if (!gated && grad_gate != nullptr) return CAWN_ERR_INVALID_ARG;
    if (sums && workspace == nullptr) return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(x, weight, bias, gate, grad_y, grad_x, grad_gate, grad_weight, grad_bias, workspace)) return CAWN_ERR_MISALIGNED;
    if (sums && workspace_bytes < (size_t)c.bx * 2 * C * sizeof(float)) return CAWN_ERR_WORKSPACE_TOO_SMALL;
    if (params->N == 0) {
        if (grad_weight != nullptr && cudaMemsetAsync(grad_weight, 0, (size_t)C * sizeof(float), st) != cudaSuccess) return CAWN_ERR_CUDA;
        if (grad_bias != nullptr && cudaMemsetAsync(grad_bias, 0, (size_t)C * sizeof(float), st) != cudaSuccess) return CAWN_ERR_CUDA;
        return CAWN_OK;
    }
    NormParams P = fill(params, c);
    P.x = x; P.w = weight; P.b = bias; P.gate = gate; P.gy = grad_y; P.gx = grad_x; P.ggate = grad_gate;
    P.part = sums ? static_cast<float *>(workspace) : nullptr;
    const int first = run(params, c, P, true, st);
    if (first != CAWN_OK || !sums) return first;
    return status_of(launch(norm_sum_kernel, dim3((2 * C + 31) / 32), dim3(1024), 0, st, (const float *)P.part, c.bx, C, grad_weight, grad_bias));
}
