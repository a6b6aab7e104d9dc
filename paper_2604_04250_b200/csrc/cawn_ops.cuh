// What the operators next to the scan share: storage types, 16-byte vectors, argument checks and
// the launch helper.
#pragma once
#include "../../include/cawn.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace cawn {

using bf16 = __nv_bfloat16;

constexpr uint32_t kFlagsBf16 = CAWN_FLAG_INPUT_BF16 | CAWN_FLAG_OUTPUT_BF16;

inline bool storage_flags_ok(uint32_t flags) { return flags == 0 || flags == kFlagsBf16; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }   // NULL passes
template <class... P> inline bool all_aligned16(P... p) { return (aligned16(p) && ...); }

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 narrow<bf16>(float v) { return __float2bfloat16_rn(v); }

// V consecutive elements of storage type T as floats: one 16-byte access (two where V floats need
// them) when V > 1, an ordinary one for V = 1.
template <class T, int V> __device__ __forceinline__ void load_vec(float (&f)[V], const T *p)
{
    if constexpr (V == 1) {
        f[0] = widen(*p);
    } else if constexpr (sizeof(T) == 4) {
        static_assert(V % 4 == 0, "whole 16-byte words");
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 w = *reinterpret_cast<const float4 *>(p + i);
            f[i] = w.x; f[i + 1] = w.y; f[i + 2] = w.z; f[i + 3] = w.w;
        }
    } else {
        static_assert(V % 8 == 0, "whole 16-byte words");
#pragma unroll
        for (int i = 0; i < V; i += 8) {
            const uint4 w = *reinterpret_cast<const uint4 *>(p + i);
            const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; j++) {
                f[i + 2 * j] = __uint_as_float(u[j] << 16);
                f[i + 2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
            }
        }
    }
}

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned *>(&v);
}

template <class T, int V> __device__ __forceinline__ void store_vec(T *p, const float (&f)[V])
{
    if constexpr (V == 1) {
        *p = narrow<T>(f[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V; i += 4)
            *reinterpret_cast<float4 *>(p + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 8)
            *reinterpret_cast<uint4 *>(p + i) = make_uint4(pack_bf16(f[i], f[i + 1]), pack_bf16(f[i + 2], f[i + 3]),
                                                           pack_bf16(f[i + 4], f[i + 5]), pack_bf16(f[i + 6], f[i + 7]));
    }
}

// A pair of floats in one 64-bit register: sm_100 adds and multiplies two at a time.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float x, float y)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ f32x2 pair(float2 v) { return pair(v.x, v.y); }
__device__ __forceinline__ float2 halves(f32x2 v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Launch with the runtime's own error code (a launch error of somebody else's earlier call is not ours to report).
// EARLY: as a programmatic dependent.  Blocks may come to the SMs while the kernel before drains and wait there in
// follow_previous(), with which every kernel here begins, until all that was before is done and visible.  That hides
// the launch (norm backward of 32768 x 768: 59 -> 56 us; 12 heads x 32768 tokens forward: 314 -> 310), but takes the
// walks, the join and the chunk-local gradients longer than it hides (backward of 8 x 2048 x 12 heads: 409 -> 420 us;
// the join before the 12 heads' output walk: 314 -> 333), so those are launched plainly.
template <bool EARLY = false, class... A, class... B>
inline cudaError_t launch(void (*kernel)(A...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, B... args)
{
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st; cfg.attrs = &attr; cfg.numAttrs = EARLY ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, A(args)...);
}
// The wait comes first: a launch behind this one may read before its own wait what the caller says this one does not
// write (CAWN_FLAG_INPUT_INDEPENDENT), and that has to be complete by then, whoever wrote it.
__device__ __forceinline__ void follow_previous()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// SMs of the current device, read once per device.
inline int sm_count()
{
    static int sms[64] = {};
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    if (sms[dev] == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 148;
        sms[dev] = n;
    }
    return sms[dev];
}

inline int status_of(cudaError_t e) { return e == cudaSuccess ? CAWN_OK : CAWN_ERR_CUDA; }

}  // namespace cawn
