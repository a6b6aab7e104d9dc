// What the short convolution and the selective scan share: rows that belong to sequences, words of eight
// channels, and parameter gradients summed over blocks.
#pragma once
#include "cawn_ops.cuh"

namespace cawn {

// Sequences of rows.  Dense: L rows each.  Packed: sequence b has rows offsets[b] .. offsets[b + 1] - 1, clamped on the
// device to the arrays' rows and to L tokens, so that no content of the offsets leads out of an array.
struct Sequences {
    const long long *offsets;
    long long L, rows;
    int B;
};

struct Span { long long begin, len; };

__device__ __forceinline__ Span span_of(const Sequences &s, int b)
{
    if (s.offsets == nullptr) return {(long long)b * s.L, s.L};
    long long a = s.offsets[b], e = s.offsets[b + 1];
    a = a < 0 ? 0 : a > s.rows ? s.rows : a;
    e = e < a ? a : e > s.rows ? s.rows : e;
    return {a, e - a < s.L ? e - a : s.L};
}

// Eight elements as they are stored.
template <class T> struct Eight;
template <> struct Eight<bf16> {
    uint4 w;
    __device__ __forceinline__ void widen_to(float (&f)[8]) const
    {
        const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            f[2 * j] = __uint_as_float(u[j] << 16);
            f[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void load(const bf16 *p) { w = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void load_part(const bf16 *p, int n)
    {
        const unsigned short *s = reinterpret_cast<const unsigned short *>(p);
        unsigned u[4] = {};
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) u[i / 2] |= (unsigned)s[i] << (16 * (i % 2));
        w = make_uint4(u[0], u[1], u[2], u[3]);
    }
    __device__ __forceinline__ void clear() { w = make_uint4(0, 0, 0, 0); }
};
template <> struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void widen_to(float (&f)[8]) const
    {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void load(const float *p)
    {
        a = *reinterpret_cast<const float4 *>(p);
        b = *reinterpret_cast<const float4 *>(p + 4);
    }
    __device__ __forceinline__ void load_part(const float *p, int n)
    {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = i < n ? p[i] : 0.f;
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
    __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
};

// `n` of eight elements at p; `whole`: p may be read in 16-byte words when all eight are there.
template <class T> __device__ __forceinline__ Eight<T> fetch_eight(const T *p, int n, bool whole)
{
    Eight<T> r;
    if (whole && n >= 8) r.load(p);
    else if (n > 0) r.load_part(p, n);
    else r.clear();
    return r;
}
template <class T> __device__ __forceinline__ void store_eight(T *p, const float (&f)[8], int n, bool whole)
{
    if (whole && n >= 8) {
        store_vec(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) p[i] = narrow<T>(f[i]);
    }
}

// Four elements as they are stored.
template <class T> struct Quad;
template <> struct __align__(8) Quad<bf16> {
    uint2 w;
    __device__ __forceinline__ float4 get() const
    {
        return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
    }
    __device__ __forceinline__ void set(float4 v) { w = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)); }
    __device__ __forceinline__ void load(const bf16 *p) { w = *reinterpret_cast<const uint2 *>(p); }
};
template <> struct __align__(16) Quad<float> {
    float4 w;
    __device__ __forceinline__ float4 get() const { return w; }
    __device__ __forceinline__ void set(float4 v) { w = v; }
    __device__ __forceinline__ void load(const float *p) { w = *reinterpret_cast<const float4 *>(p); }
};
template <class T> __device__ __forceinline__ Quad<T> fetch_quad(const T *p, int n, bool whole)
{
    Quad<T> r;
    if (whole && n >= 4) r.load(p);
    else r.set(make_float4(n > 0 ? widen(p[0]) : 0.f, n > 1 ? widen(p[1]) : 0.f, n > 2 ? widen(p[2]) : 0.f, n > 3 ? widen(p[3]) : 0.f));
    return r;
}
template <class T> __device__ __forceinline__ void store_quad(T *p, float4 v, int n, bool whole)
{
    if (whole && n >= 4) {
        Quad<T> r;
        r.set(v);
        *reinterpret_cast<Quad<T> *>(p) = r;
    } else {
        if (n > 0) p[0] = narrow<T>(v.x);
        if (n > 1) p[1] = narrow<T>(v.y);
        if (n > 2) p[2] = narrow<T>(v.z);
        if (n > 3) p[3] = narrow<T>(v.w);
    }
}

// Rows all of whose words are whole are fetched without a branch.
template <bool WHOLE, class T> __device__ __forceinline__ Eight<T> eight_of(const T *p, int n, bool whole)
{
    if constexpr (!WHOLE) return fetch_eight(p, n, whole);
    Eight<T> r;
    r.clear();
    if (n > 0) r.load(p);
    return r;
}
template <bool WHOLE, class T> __device__ __forceinline__ Quad<T> quad_of(const T *p, int n, bool whole)
{
    if constexpr (!WHOLE) return fetch_quad(p, n, whole);
    Quad<T> r;
    r.set(make_float4(0.f, 0.f, 0.f, 0.f));
    if (n > 0) r.load(p);
    return r;
}

__device__ __forceinline__ float reciprocal_fast(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float sigmoid_of(float v) { return reciprocal_fast(1.f + exp2_fast(-kLog2e * v)); }
__device__ __forceinline__ f32x2 twice(float v) { return pair(v, v); }
__device__ __forceinline__ f32x2 sigmoid_of(f32x2 v)
{
    const float2 e = halves(mul2(v, twice(-kLog2e)));
    const float2 d = halves(add2(pair(exp2_fast(e.x), exp2_fast(e.y)), twice(1.f)));
    return pair(reciprocal_fast(d.x), reciprocal_fast(d.y));
}

// Sums of `rows` partial rows of `cols` floats each, in double and in a fixed order, into up to three arrays that the
// columns belong to one after the other (NULL: not wanted).
struct PartialSums {
    const float *part;
    long long rows, cols;
    float *out[3];
    long long count[3];
};
int sum_partials(const PartialSums &p, cudaStream_t st);

// Packed calls say how many rows there are (none only where there are no tokens), dense ones have B * L.
inline int check_offsets(const int64_t *offsets, int64_t B, int64_t L, int64_t rows)
{
    if (offsets == nullptr ? rows != 0 && rows != B * L : rows == 0 && L > 0) return CAWN_ERR_INVALID_ARG;
    return (reinterpret_cast<uintptr_t>(offsets) & 7) != 0 ? CAWN_ERR_MISALIGNED : CAWN_OK;
}

// Slices may begin at any element; whole words are read where rows begin on `bytes`.
template <class... P> inline bool elements_aligned(uint32_t flags, P... p)
{
    const uintptr_t mask = flags != 0 ? 1 : 3;
    return (((reinterpret_cast<uintptr_t>(p) & mask) == 0) && ...);
}
inline bool begins_on(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

inline int64_t most(int64_t a, int64_t b) { return a > b ? a : b; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace cawn
