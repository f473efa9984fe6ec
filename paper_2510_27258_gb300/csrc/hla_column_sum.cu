// Sums of partial rows, in a fixed order: the last step of gradients that are sums over tokens.
#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kCols = 32, kThreads = 1024;  // columns of a block

// Bound by latency: with four columns a thread (kV 4) all the rows of a block are on their way at once (304 rows of 4096
// columns, not in cache: 9 us with one column a thread)
template <int kV>
__global__ void __launch_bounds__(kThreads) column_sum_kernel(ColumnSum p) {
    constexpr int kLanes = kCols / kV, kGroups = kThreads / kLanes;  // lanes of a row, rows side by side
    __shared__ float red[kCols][kGroups + 1];
    let_next_begin();
    after_previous();
    // (of calls without device-side waits: never an error)
    if (p.header && blockIdx.x == 0 && threadIdx.x == 0) *p.header = WsHeader{};
    const int place = threadIdx.x % kLanes * kV, group = threadIdx.x / kLanes;
    const long long cols = (long long)p.C * p.parts, at = (long long)blockIdx.x * kCols;
    float sum[kV] = {};
    if (at + place < cols) {
        const float *from = p.partial + at + place;
#pragma unroll 8
        for (long long r = group; r < p.rows; r += kGroups) {
            float v[kV];
            VecIo<float, kV>::load(from + r * cols, v);
#pragma unroll
            for (int i = 0; i < kV; ++i) sum[i] += v[i];
        }
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) red[place + i][group] = sum[i];
    __syncthreads();
    // warp w: column w
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    float all = 0.f;
#pragma unroll
    for (int k = 0; k < kGroups; k += 32) all += red[w][k + lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    const long long c = at + w;
    if (lane == 0 && c < cols) {
        const int part = (int)(c / p.C), i = (int)(c - (long long)part * p.C);
#pragma unroll
        for (int o = 0; o < 3; ++o) {
            const ColumnSum::Out &out = p.out[o];
            if (out.to && out.part == ColumnSum::kNoSum && part == 0) out.to[i] = 0.f;
            if (!out.to || out.part != part) continue;
            const float by = !out.factor           ? 1.f
                             : p.dt == HLA_BF16 ? to_f32(static_cast<const __nv_bfloat16 *>(out.factor)[i])
                                                : static_cast<const float *>(out.factor)[i];
            out.to[i] = all * by;
        }
    }
}

}  // namespace

cudaError_t column_sum_launch(const ColumnSum &p, cudaStream_t s) {
    const long long cols = (long long)p.C * p.parts;
    const unsigned blocks = (unsigned)((cols + kCols - 1) / kCols);
    return cols % 4 == 0 ? launch_after(column_sum_kernel<4>, blocks, kThreads, 0, s, p)
                         : launch_after(column_sum_kernel<1>, blocks, kThreads, 0, s, p);
}

}  // namespace hla
