// Gated delta rule, chunk form: matrix fragments, tiles and the workspace shared by its kernels.
//
// Mathematics of a chunk of 64 tokens (G = running sum of g inside the chunk, Gam_ij = e^{G_i - G_j},
// S0 the state before it, states written [value, key]):
//   At_ij = Gam_ij k_i.k_j (i > j)           T = (I + At diag(beta))^{-1}, unit lower triangular
//   r = T (V - e^G K S0^T),  u = beta r       P_ij = scale Gam_ij q_i.k_j (i >= j)
//   O = scale e^G Q S0^T + P u               S = e^{G_C} S0 + sum_j e^{G_C - G_j} u_j k_j^T
//
// Precision.  Products run on the tensor cores with bfloat16 factors and float sums; a float factor enters
// as a sum of bfloat16 terms (8 mantissa bits each).  NP: terms of inputs, NT: terms of T and P.
// bfloat16 storage: inputs are exact as one term (NP 1), T and P take two (NT 2), the state and R as factors of the
// chain two in the forward and three in the backward, the state's update three.  The factors of o (state, u, P) and of
// dq, dk and the gradients of g and beta (r, rb, both states, the products' weights) take two, in the backward with all
// four products of a pair: o, dq and dk are rounded to 8 bits once, at the end, the gradients of g and beta off by
// 1e-6 .. 8e-6 of their norm.  Sixteen bits and not eight for these, because their sums may be differences: where keys
// overwrite a state 50 times the values, one term each left o off by 6e-2 and dq, dk by more.
// Float storage: three terms everywhere (NP = NT = 3), inputs by a pass of their own: 1e-6 .. 3e-6.
// (With two terms throughout the state was off by 5e-6 and the gradient of g by up to 2e-5.)
//
// Layout of the walks.  They work on transposed chunks: a row group is 16 rows of values against all keys and
// tokens, so that every product of the chain (state x keys, triangle, update) has the previous result as its left
// factor.  The accumulator layout of mma.m16n8k16 is the layout of that operand: the chain stays in one warp's
// registers.  The right factors (K, Q, T, P tiles) come from shared memory.  Chain warps do what the next
// chunk waits for, one per scheduler of the SM.  Other warps fetch all tiles (cp.async); in the forward they also make
// the outputs, which hang off the chain (8 x 2048 x 12 heads, with outputs of one term: 91 -> 72 us).  (Two warps sharing a
// row group's chain were slower, 101 us: handing fragments over doubled the shared-memory traffic.)
#pragma once
#include "cawn_delta.cuh"

namespace cawn {

constexpr int kC = 64;                  // tokens of a chunk
constexpr int kPad = 8;                 // bfloat16 of padding per shared row: ldmatrix reads 8 rows without conflicts
constexpr int kTile = kC * kC;          // elements of a 64 x 64 tile in the workspace
constexpr int kTri = 10 * 256;          // of a triangle there: its ten 16 x 16 blocks on and below the diagonal
constexpr int kLd = kC + kPad;
constexpr int kCoef = 5;                // floats per token: e^G, e^{G_C - G}, beta, log2(e) G (high, low part)
enum { COEF_EG = 0, COEF_LEFT = 1, COEF_BETA = 2, COEF_GHI = 3, COEF_GLO = 4 };

// One input array as NP bfloat16 terms, `plane` elements apart; strides in elements.
struct Terms {
    const bf16 *at;
    long long plane, stride_t, stride_b;
};

// Everything the chunk kernels share.  nc = bh * chunks + c numbers chunks of value heads, nv = nc * vblocks +
// vb their blocks of 64 values; tiles and coefficients of the workspace are dense over these.
struct ChunkParams {
    Terms q, k, v, go;
    const float *g, *beta;
    float *coef;                        // [nc][kCoef][64]
    bf16 *tri, *p;                      // [nc][NT][kTri]: T - I, transposed, and P, see in_triangle
    // What the backward's walks leave for the chunk-local products, value rows: the state before the chunk, the adjoint D
    // of the one after it, r and D K^T
    float *s0, *ds;                     // [nv][64 v][DK]
    float *r, *dk;                      // [nv][64 v][64 t]
    bf16 *rbt;                          // and rb, laid out like v; with bfloat16 storage the first term is dV itself (o)
    Terms rb;                           // its plane and strides
    const float *state_in;              // [bh][Dv][Dk], may be NULL
    float *state_out;
    const float *adj_in;                // gradient of state_out, may be NULL
    float *adj_out;                     // gradient of state_in, may be NULL
    void *o;                            // forward output; backward: grad_v
    void *gq, *gk;
    float *gg, *gbeta;
    long long L, o_stride_t, o_stride_b;
    // time segments: start states per segment, local end states, transitions; adjoints likewise, from the end
    float *seg_start, *seg_end, *seg_map;   // [bh][segs][Dv][Dk], same, [bh][segs][Dk][Dk]
    float *adj_start, *adj_end;
    int segs, seg_chunks;
    int B, Hk, Hv, Dk, Dv, chunks, vblocks;
    float scale;
};

__device__ __forceinline__ unsigned smem_addr(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void cp16(unsigned dst, const void *src, bool ok)
{
    const int n = ok ? 16 : 0;          // 0 bytes read: the 16 bytes in shared memory become zero
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

// ROWS x COLS tile into shared rows of COLS + kPad; rows and columns past the valid ones become zero.
template <int ROWS, int COLS, int THREADS>
__device__ __forceinline__ void load_tile(bf16 *dst, const bf16 *src, long long stride, int rows, int cols)
{
    static_assert(THREADS % (COLS / 8) == 0 && ROWS % (THREADS / (COLS / 8)) == 0, "whole passes");
    constexpr int STEP = THREADS / (COLS / 8);
    const int tid = threadIdx.x % THREADS, r = tid / (COLS / 8), c = tid % (COLS / 8) * 8;
    unsigned to = smem_addr(dst) + (r * (COLS + kPad) + c) * 2;
    const bf16 *from = src + r * stride + c;
#pragma unroll
    for (int i = 0; i < ROWS / STEP; i++) {
        const bool ok = r + i * STEP < rows && c < cols;
        cp16(to, ok ? from : src, ok);
        to += STEP * (COLS + kPad) * 2;
        from += STEP * stride;
    }
}
// Where block (I, J), I >= J, of a triangle starts, in the workspace and in shared memory: four blocks of 8 x 8 (half of
// the row, half of the column), 128 bytes each, which is what a warp holds of an accumulator tile and writes at once,
// and what one phase of ldmatrix reads.  (As 64 x 64 tiles a warp's words fell on eight rows: those stores took a
// third of the shared memory pipe's time in the kernel that makes T and P.)
__host__ __device__ constexpr int in_triangle(int I, int J) { return (I * (I + 1) / 2 + J) * 256; }
template <int THREADS> __device__ __forceinline__ void load_triangle(bf16 *dst, const bf16 *src)
{
    const int tid = threadIdx.x % THREADS;
    const unsigned to = smem_addr(dst) + tid * 16;
#pragma unroll
    for (int i = 0; i < kTri / 8; i += THREADS)
        if ((kTri / 8) % THREADS == 0 || i + tid < kTri / 8) cp16(to + i * 16, src + (i + tid) * 8, true);
}

__device__ __forceinline__ void ldsm(unsigned (&r)[4], unsigned addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_t(unsigned (&r)[4], unsigned addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void stsm_t(unsigned addr, unsigned a, unsigned b, unsigned c, unsigned d)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};"
                 :: "r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// This lane's row address inside a 16 x 16 block at (row, col) of a tile with rows of `ld` elements.
// NK: rows are the n index of a right factor (or the k index of a transposed left one), KN: rows are the
// k index of a right factor read transposed, or the m index of a left factor.
__device__ __forceinline__ unsigned at_nk(unsigned base, int ld, int row, int col)
{
    const int l = threadIdx.x % 32;
    return base + ((row + l % 8 + l / 16 * 8) * ld + col + l / 8 % 2 * 8) * 2;
}
__device__ __forceinline__ unsigned at_kn(unsigned base, int ld, int row, int col)
{
    const int l = threadIdx.x % 32;
    return base + ((row + l % 8 + l / 8 % 2 * 8) * ld + col + l / 16 * 8) * 2;
}

// the same for block (I, J) of a triangle
__device__ __forceinline__ unsigned triangle_nk(unsigned base, int I, int J) { return base + in_triangle(I, J) * 2 + threadIdx.x % 32 * 16; }
__device__ __forceinline__ unsigned triangle_kn(unsigned base, int I, int J)
{
    const int l = threadIdx.x % 32;
    return base + in_triangle(I, J) * 2 + (l / 8 % 2 * 16 + l / 16 * 8 + l % 8) * 16;
}

// rows h = 0, 1 of an accumulator tile, times / plus pairs
__device__ __forceinline__ void scale_row(float (&c)[4], int h, f32x2 f)
{
    const float2 v = halves(mul2(pair(c[2 * h], c[2 * h + 1]), f));
    c[2 * h] = v.x;
    c[2 * h + 1] = v.y;
}
// c row h <- a * (c row h) + b
__device__ __forceinline__ void fma_row(float (&c)[4], int h, f32x2 a, f32x2 b)
{
    const float2 v = halves(fma2(a, pair(c[2 * h], c[2 * h + 1]), b));
    c[2 * h] = v.x;
    c[2 * h + 1] = v.y;
}

// Barriers of the walks, `threads` of both sides together: chain tiles are here / free again, what passes between chain
// and side is here / free again, and one among the side warps.
enum { BAR_FULL = 1, BAR_EMPTY = 3, BAR_READY = 5, BAR_FREE = 7, BAR_SIDE = 9 };    // the first four: + stage or parity
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" :: "r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" :: "r"(id), "r"(threads) : "memory"); }

// Row groups of a block: float storage has three times the tiles, so half the row groups fit.
template <int NP> constexpr int kRowGroups = NP == 1 ? 4 : 2;

// Stages of the chain's and the side's tiles and of what they exchange: as many as fit.
struct Stages { int chain, side, swap; };
constexpr Stages fit_stages(size_t chain, size_t side, size_t swap)
{
    const size_t room = 227 * 1024;
    if (2 * (chain + side + swap) <= room) return {2, 2, 2};
    if (2 * chain + side + 2 * swap <= room) return {2, 1, 2};
    if (2 * chain + side + swap <= room) return {2, 1, 1};
    return {1, 1, 1};
}

// Fragments handed from warp to warp: N terms of left operand number i.
template <int N> __device__ __forceinline__ void put_left(uint4 *buf, int i, const unsigned (&a)[N][4])
{
#pragma unroll
    for (int t = 0; t < N; t++) buf[(i * N + t) * 32 + threadIdx.x % 32] = make_uint4(a[t][0], a[t][1], a[t][2], a[t][3]);
}
template <int N> __device__ __forceinline__ void get_left(unsigned (&a)[N][4], const uint4 *buf, int i)
{
#pragma unroll
    for (int t = 0; t < N; t++) {
        const uint4 v = buf[(i * N + t) * 32 + threadIdx.x % 32];
        a[t][0] = v.x; a[t][1] = v.y; a[t][2] = v.z; a[t][3] = v.w;
    }
}

// Sums over the eight lanes that share a column pair, for N values of each of eight tiles; lane row gr ends with the
// sums of tile gr in v[0].
template <int N> __device__ __forceinline__ void column_sums(float (&v)[8][N])
{
    const int gr = threadIdx.x % 32 / 4;
#pragma unroll
    for (int bit = 4; bit > 0; bit /= 2)
#pragma unroll
        for (int n = 0; n < bit; n++)
#pragma unroll
            for (int e = 0; e < N; e++) {
                const bool up = (gr & bit) != 0;
                const float keep = up ? v[n + bit][e] : v[n][e], send = up ? v[n][e] : v[n + bit][e];
                v[n][e] = keep + __shfl_xor_sync(0xffffffffu, send, bit * 4);
            }
}

// x, y as N bfloat16 terms of falling size, packed; N = 1 rounds
template <int N> __device__ __forceinline__ void split(float x, float y, unsigned (&w)[N])
{
    f32x2 rest = pair(x, y);
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float2 v = halves(rest);
        w[i] = pack_bf16(v.x, v.y);
        if (i + 1 < N)
            rest = fma2(pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), pair(-1.f, -1.f), rest);
    }
}
__device__ __forceinline__ float2 unpack(unsigned w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

// The value pair that the terms of word e of a fragment stand for
template <int N> __device__ __forceinline__ float2 sum_terms(const unsigned (&a)[N][4], int e)
{
    float2 x = unpack(a[N - 1][e]);
#pragma unroll
    for (int i = N - 2; i >= 0; i--) {
        const float2 y = unpack(a[i][e]);
        x.x += y.x;
        x.y += y.y;
    }
    return x;
}

// Accumulators of two neighbouring 16 x 8 tiles as N terms of the left operand of the next product.
template <int N> __device__ __forceinline__ void as_left(const float (&c0)[4], const float (&c1)[4], unsigned (&a)[N][4])
{
#pragma unroll
    for (int e = 0; e < 4; e++) {
        unsigned w[N];
        split(e < 2 ? c0[2 * e] : c1[2 * e - 4], e < 2 ? c0[2 * e + 1] : c1[2 * e - 3], w);
#pragma unroll
        for (int i = 0; i < N; i++) a[i][e] = w[i];
    }
}

// Left operand of AP terms from shared planes `plane` elements apart (TRANS: stored [k][m], at_nk; else at_kn).
template <int AP, bool TRANS> __device__ __forceinline__ void load_left(unsigned (&a)[AP][4], unsigned addr, int plane)
{
#pragma unroll
    for (int i = 0; i < AP; i++)
        if (TRANS) ldsm_t(a[i], addr + i * plane * 2); else ldsm(a[i], addr + i * plane * 2);
}

// Right operand of a 16 x 16 block, BP terms in shared planes `plane` elements apart; TRANS as ldsm_t.
template <int BP, bool TRANS> __device__ __forceinline__ void load_right(unsigned (&b)[BP][4], unsigned addr, int plane)
{
#pragma unroll
    for (int j = 0; j < BP; j++)
        if (TRANS) ldsm_t(b[j], addr + j * plane * 2); else ldsm(b[j], addr + j * plane * 2);
}

// Tiles 2 i, 2 i + 1 += left (AP terms) x right block i (BP terms), N blocks.  Pairs of terms
// beyond the precision of the longer operand are left out: 2 x 2 terms take three products, 3 x 3 six (MORE: pairs of
// so many further orders are taken).  Blocks are the inner loop: a product waits 21 cycles for the sum before it but
// issues every 8.
template <int AP, int BP, int N, int MORE = 0>
__device__ __forceinline__ void multiply(float (&c)[2 * N][4], const unsigned (&a)[AP][4], const unsigned (&b)[N][BP][4])
{
    constexpr int ORDER = (AP > BP ? AP : BP) + MORE;
#pragma unroll
    for (int j = 0; j < BP; j++)
#pragma unroll
        for (int i = 0; i < AP; i++)
            if (i + j < ORDER)
#pragma unroll
                for (int n = 0; n < N; n++) {
                    mma(c[2 * n], a[i], b[n][j][0], b[n][j][1]);
                    mma(c[2 * n + 1], a[i], b[n][j][2], b[n][j][3]);
                }
}

// One block at a time
template <int AP, int BP, bool TRANS, int MORE = 0>
__device__ __forceinline__ void product(float (&c0)[4], float (&c1)[4], const unsigned (&a)[AP][4], unsigned addr, int plane)
{
    constexpr int ORDER = (AP > BP ? AP : BP) + MORE;
    unsigned b[BP][4];
    load_right<BP, TRANS>(b, addr, plane);
#pragma unroll
    for (int j = 0; j < BP; j++)
#pragma unroll
        for (int i = 0; i < AP; i++)
            if (i + j < ORDER) {
                mma(c0, a[i], b[j][0], b[j][1]);
                mma(c1, a[i], b[j][2], b[j][3]);
            }
}

// C (token tiles of 8, in 16-row blocks) += chain of 16-token blocks A_b x right blocks, on and below the triangle's
// diagonal: C block n takes A blocks b <= n (UPPER: b >= n).  `left(a, b)` loads or makes A_b, `at(b, n)` is the
// address of the right block.  Two C blocks at a time, so that four sums are under way.
template <int AP, int BP, bool TRANS, bool UPPER, class Left, class At>
__device__ __forceinline__ void triangle(float (&c)[8][4], Left left, At at)
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int b = UPPER ? 3 - i : i;
        unsigned a[AP][4];
        left(a, b);
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            // the pair of C blocks j, j + 1
            const bool first = UPPER ? j <= b : j >= b, second = UPPER ? j + 1 <= b : j + 1 >= b;
            if (first && second) {
                unsigned r[2][BP][4];
                load_right<BP, TRANS>(r[0], at(b, j), kTri);
                load_right<BP, TRANS>(r[1], at(b, j + 1), kTri);
                multiply<AP, BP, 2>(reinterpret_cast<float (&)[4][4]>(c[2 * j]), a, r);
            } else if (first) {
                product<AP, BP, TRANS>(c[2 * j], c[2 * j + 1], a, at(b, j), kTri);
            } else if (second) {
                product<AP, BP, TRANS>(c[2 * j + 2], c[2 * j + 3], a, at(b, j + 1), kTri);
            }
        }
    }
}

// ------------------------------------------------------------------------------------ steps shared by the walks
// X (8 token tiles) += rows of a state (NS terms) x K^T or Q^T (tile with rows of tokens)
template <int NS, int NP, int DK> __device__ __forceinline__ void rows_times(float (&X)[8][4], const float (&S)[DK / 8][4], unsigned tile)
{
#pragma unroll
    for (int d = 0; d < DK / 16; d++) {
        unsigned a[NS][4], b[4][NP][4];
#pragma unroll
        for (int i = 0; i < 4; i++) load_right<NP, false>(b[i], at_nk(tile, DK + kPad, 16 * i, 16 * d), kC * (DK + kPad));
        as_left(S[2 * d], S[2 * d + 1], a);
        multiply<NS, NP, 4>(X, a, b);
    }
}
// x (tiles 2 nb .. 2 nb + 3 of a state's columns) += left x K or Q, token block by token block
template <int NP, int DK> __device__ __forceinline__ void columns_times(float (&x)[4][4], const unsigned (&a)[4][3][4], unsigned tile, int nb)
{
#pragma unroll
    for (int tb = 0; tb < 4; tb++) {
        unsigned b[2][NP][4];
#pragma unroll
        for (int i = 0; i < 2; i++) load_right<NP, true>(b[i], at_kn(tile, DK + kPad, 16 * tb, 16 * (nb + i)), kC * (DK + kPad));
        multiply<3, NP, 2>(x, a[tb], b);
    }
}
// every token's column of tiles times its coefficient (row `which` of coef)
__device__ __forceinline__ void scale_tokens(float (&x)[8][4], const float (*coef)[kC], int which, float sign = 1.f)
{
    const int tc = threadIdx.x % 4 * 2;
#pragma unroll
    for (int n = 0; n < 8; n++) {
        const float2 f = *reinterpret_cast<const float2 *>(&coef[which][8 * n + tc]);
        const f32x2 g = sign == 1.f ? pair(f) : pair(sign * f.x, sign * f.y);
        scale_row(x[n], 0, g);
        scale_row(x[n], 1, g);
    }
}
// R = V^T - e^G X, V a tile with rows of tokens, `addr` this row group's block of it
template <int NP> __device__ __forceinline__ void residual(float (&X)[8][4], const float (*coef)[kC], unsigned tile, int vld, int col, bool values)
{
    const int tc = threadIdx.x % 4 * 2;
#pragma unroll
    for (int nb = 0; nb < 4; nb++) {
        unsigned v[NP][4] = {};
        if (values) load_left<NP, true>(v, at_nk(tile, vld, 16 * nb, col), kC * vld);
#pragma unroll
        for (int m = 0; m < 2; m++) {
            const float2 e = *reinterpret_cast<const float2 *>(&coef[COEF_EG][16 * nb + 8 * m + tc]);
#pragma unroll
            for (int h = 0; h < 2; h++) fma_row(X[2 * nb + m], h, pair(-e.x, -e.y), pair(sum_terms(v, 2 * m + h)));
        }
    }
}
// state rows r, r + 8 (r = this thread's) from / to [Dv][Dk] floats
template <int DK> __device__ __forceinline__ void load_state(float (&S)[DK / 8][4], const float *from, int r, int rows, int Dk)
{
    const int tc = threadIdx.x % 4 * 2;
#pragma unroll
    for (int n = 0; n < DK / 8; n++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            float2 x = make_float2(0.f, 0.f);
            if (from != nullptr && r + 8 * h < rows && 8 * n + tc < Dk) x = *reinterpret_cast<const float2 *>(from + (long long)(r + 8 * h) * Dk + 8 * n + tc);
            S[n][2 * h] = x.x;
            S[n][2 * h + 1] = x.y;
        }
}
template <int DK> __device__ __forceinline__ void store_state(float *to, const float (&S)[DK / 8][4], int r, int rows, int Dk)
{
    const int tc = threadIdx.x % 4 * 2;
#pragma unroll
    for (int n = 0; n < DK / 8; n++)
#pragma unroll
        for (int h = 0; h < 2; h++)
            if (r + 8 * h < rows && 8 * n + tc < Dk)
                *reinterpret_cast<float2 *>(to + (long long)(r + 8 * h) * Dk + 8 * n + tc) = make_float2(S[n][2 * h], S[n][2 * h + 1]);
}
// a row group's value rows, 8 N floats each
template <int N> __device__ __forceinline__ void store_rows(float *to, const float (&x)[N][4])
{
    to += threadIdx.x % 32 / 4 * (8 * N) + threadIdx.x % 4 * 2;
#pragma unroll
    for (int n = 0; n < N; n++)
#pragma unroll
        for (int h = 0; h < 2; h++) *reinterpret_cast<float2 *>(to + 8 * h * (8 * N) + 8 * n) = make_float2(x[n][2 * h], x[n][2 * h + 1]);
}
// Value head's place
__device__ __forceinline__ long long q_base(const ChunkParams &P, const Terms &t, int bh, long long t0)
{
    return (bh / P.Hv) * t.stride_b + t0 * t.stride_t + (long long)(bh % P.Hv / (P.Hv / P.Hk)) * P.Dk;
}
__device__ __forceinline__ long long v_base(const ChunkParams &P, const Terms &t, int bh, long long t0)
{
    return (bh / P.Hv) * t.stride_b + t0 * t.stride_t + (long long)(bh % P.Hv) * P.Dv;
}

// Float arrays of `rows` rows to split, `stride` elements from row to row; terms go one after the other into dst.
struct SplitJob {
    const float *src;
    bf16 *dst;
    long long stride;
    int width;
};
struct SplitJobs {
    SplitJob job[4];
    long long rows;
    int count;
};

// terms: NP
cudaError_t launch_delta_split(const SplitJobs &jobs, cudaStream_t st);
cudaError_t launch_delta_prep(const ChunkParams &P, int dk, int terms, cudaStream_t st);
// forward over the chunks: outputs and end state
cudaError_t launch_delta_scan(const ChunkParams &P, int dk, int terms, cudaStream_t st);
// start states of time segments (and of the adjoint's) from what the summaries left
cudaError_t launch_delta_join(const ChunkParams &P, int dk, bool adjoint, cudaStream_t st);
// backward: the forward's walk and the reverse one, then what is local to a chunk
// the backward's walks, in both directions; `summary`: of segments
cudaError_t launch_delta_walks(const ChunkParams &P, int dk, int terms, bool summary, cudaStream_t st);
cudaError_t launch_delta_grads(const ChunkParams &P, int dk, int terms, cudaStream_t st);

}  // namespace cawn
