// Sums of parameter gradients over the blocks that made parts of them.
#include "cawn_seq.cuh"

namespace cawn {
namespace {

// The sum of a column to its place.
__device__ __forceinline__ void put(const PartialSums &P, long long col, double sum)
{
#pragma unroll
    for (int k = 0; k < 3; k++) {
        if (col < P.count[k]) {
            if (P.out[k] != nullptr) P.out[k][col] = (float)sum;
            return;
        }
        col -= P.count[k];
    }
}

__global__ void __launch_bounds__(1024) sum_partials_kernel(const PartialSums P)
{
    follow_previous();
    __shared__ double sums[32][33];
    const int x = threadIdx.x % 32, lane = threadIdx.x / 32;
    const long long col = (long long)blockIdx.x * 32 + x;
    double s = 0.0, t = 0.0;
    if (col < P.cols) {
        long long i = lane;
        for (; i + 32 < P.rows; i += 64) {
            s += (double)P.part[i * P.cols + col];
            t += (double)P.part[(i + 32) * P.cols + col];
        }
        if (i < P.rows) s += (double)P.part[i * P.cols + col];
    }
    sums[lane][x] = s + t;
    __syncthreads();
    // a warp per column: lane x holds row lane x of column `lane`
    s = sums[x][lane];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    const long long mine = (long long)blockIdx.x * 32 + lane;
    if (x == 0) put(P, mine, s);
}

// Few rows: a thread a column (16 rows of 18432 columns: 14 us by the kernel above, 5 here).
constexpr int kFewRows = 32;
__global__ void __launch_bounds__(128) sum_few_kernel(const PartialSums P)
{
    follow_previous();
    const long long col = (long long)blockIdx.x * 128 + threadIdx.x;
    if (col >= P.cols) return;
    double s = 0.0;
#pragma unroll 16
    for (long long i = 0; i < P.rows; i++) s += (double)P.part[i * P.cols + col];
    put(P, col, s);
}

}  // namespace

int sum_partials(const PartialSums &p, cudaStream_t st)
{
    if (p.rows <= kFewRows) return status_of(launch<true>(sum_few_kernel, dim3((unsigned)ceil_div(p.cols, 128)), dim3(128), 0, st, p));
    return status_of(launch<true>(sum_partials_kernel, dim3((unsigned)ceil_div(p.cols, 32)), dim3(1024), 0, st, p));
}

}  // namespace cawn
