// Sums of partial rows, in a fixed order: the last step of gradients that are sums over tokens.
#include "hla_internal.h"

namespace hla {
namespace {

constexpr int kCols = 32, kGroups = 32;  // columns of a block, and the rows it reads side by side

// (bound by latency: each thread's loads are independent, a few dozen at most; 304 rows of 6144 columns take
// 3 us)
__global__ void __launch_bounds__(kCols *kGroups) column_sum_kernel(ColumnSum p) {
    __shared__ float red[kGroups][kCols + 1];
    let_next_begin();
    after_previous();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.header = WsHeader{};  // no device-side waits before: never an error
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const long long cols = (long long)p.C * p.parts, at = (long long)blockIdx.x * kCols;
    float sum = 0.f;
    if (at + lane < cols) {
        const float *from = p.partial + at + lane;
#pragma unroll 8
        for (long long r = group; r < p.rows; r += kGroups) sum += from[r * cols];
    }
    red[group][lane] = sum;
    __syncthreads();
    // warp w: column w
    sum = red[lane][group];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const long long c = at + group;
    if (lane == 0 && c < cols) {
        const int part = (int)(c / p.C), i = (int)(c - (long long)part * p.C);
#pragma unroll
        for (int o = 0; o < 3; ++o) {
            const ColumnSum::Out &out = p.out[o];
            if (!out.to || out.part != part) continue;
            const float by = !out.factor           ? 1.f
                             : p.dt == HLA_BF16 ? to_f32(static_cast<const __nv_bfloat16 *>(out.factor)[i])
                                                : static_cast<const float *>(out.factor)[i];
            out.to[i] = sum * by;
        }
    }
}

}  // namespace

cudaError_t column_sum_launch(const ColumnSum &p, cudaStream_t s) {
    const long long cols = (long long)p.C * p.parts;
    return launch_after(column_sum_kernel, (unsigned)((cols + kCols - 1) / kCols), kCols * kGroups, 0, s, p);
}

}  // namespace hla
