// Gated feed-forward projections and their gradients in fp32, on the CUDA cores (bf16: hla_ffn_sm103.cu).
//
//   Z = x [Wg; Wu]^T (two products of one tile),  out = act(Zg) Zu
//   dZg = dout Zu act'(Zg),  dZu = dout act(Zg),  dx = [dZg dZu] [Wg; Wu],  d[Wg; Wu] = [dZg dZu]^T x
//
// One tiled product serves all four: a block of 256 threads forms 128 x 128 outputs (64 x 64 where those would leave
// SMs without a tile) from panels of 16 in shared memory, the next panel in registers meanwhile; a thread holds 8 x 8 (4 x 4)
// sums and adds two neighbours an instruction.  The forward's tile is half gate and half up columns of the same
// features, so that the activation and product happen in registers.  The gradient keeps [dZg dZu] in the workspace; its dx,
// whose sum is over 2 F and whose tiles may be few, is cut along the sum, and the parts are added in their order.
#include "hla_ffn.h"
#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kThreads = 256, kDepth = 16;

enum Mode { kProduct, kParts, kOut, kGrad };

// a matrix by its rows' and columns' strides; a column is an index of the sum
struct Mat {
    const float *p;
    long long row, col;
};

struct Product {
    Mat a, b;
    int M, N, K, act;  // outputs M x N (kOut, kGrad: N features, whose up rows of b are N rows behind)
    int per;           // indices of the sum for each blockIdx.y
    int across;        // tiles along N (blockIdx.x counts all tiles)
    float *out;        // kParts: [y][M][N]
    long long out_row;
    const float *dout;  // kGrad: out is fp32 [M][2 N]
    long long dout_row;
    WsHeader *header;  // cleared (kOut, kGrad: the call's first product)
};

__device__ __forceinline__ float act_of(int act, float v, float &slope) {
    if (act == HLA_LINEAR) {
        slope = 1.f;
        return v;
    }
    const float s = __fdividef(1.f, 1.f + __expf(-v));
    slope = act == HLA_SIGMOID ? s * (1.f - s) : s * (1.f + v * (1.f - s));
    return act == HLA_SIGMOID ? s : v * s;
}

// A panel's elements of one thread: kRows x kDepth over 256 threads, neighbours along the contiguous direction
template <int kRows, bool kAlong>
struct Panel {
    static constexpr int kEach = kRows * kDepth / kThreads;
    float v[kEach];
    static __device__ __forceinline__ int row(int i) {
        return kAlong ? (threadIdx.x >> 4) + 16 * i : threadIdx.x % kRows;
    }
    static __device__ __forceinline__ int depth(int i) {
        return kAlong ? threadIdx.x & 15 : threadIdx.x / kRows + kThreads / kRows * i;
    }
    // rows from `at` on (of `rows`), the second half of the panel `pair` rows on where pair > 0
    __device__ __forceinline__ void load(const Mat &m, int at, int rows, int k0, int k1, int pair) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            int r = row(i);
            const int k = k0 + depth(i);
            const bool second = pair > 0 && r >= kRows / 2;
            if (second) r -= kRows / 2;
            const long long from = (long long)(at + r) + (second ? pair : 0);
            v[i] = at + r < rows && k < k1 ? m.p[from * m.row + k * m.col] : 0.f;
        }
    }
    __device__ __forceinline__ void store(float (&to)[kDepth][kRows + 4]) const {
#pragma unroll
        for (int i = 0; i < kEach; ++i) to[depth(i)][row(i)] = v[i];
    }
};

// kTile 128 or 64; kA, kB: whether the sum's index is the contiguous one
template <int kTile, bool kA, bool kB, Mode kMode>
__global__ void __launch_bounds__(kThreads) ffn_product_kernel(Product p) {
    constexpr int kE = kTile / 16, kH = kE / 2;  // a thread's rows and columns, in two runs of kH
    constexpr bool kPair = kMode == kOut || kMode == kGrad;
    constexpr int kCols = kPair ? kTile / 2 : kTile;
    __shared__ __align__(16) float as[2][kDepth][kTile + 4], bs[2][kDepth][kTile + 4];
    let_next_begin();
    after_previous();
    if (kPair && blockIdx.x == 0 && threadIdx.x == 0) *p.header = WsHeader{};  // no device-side waits here: never an error
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int down = blockIdx.x / p.across, m0 = down * kTile, n0 = (blockIdx.x - down * p.across) * kCols;
    const int k_lo = blockIdx.y * p.per, k_hi = (int)min((long long)p.K, (long long)k_lo + p.per), pair_rows = kPair ? p.N : 0;
    Panel<kTile, kA> pa;
    Panel<kTile, kB> pb;
    uint64_t acc[kE][kH];
#pragma unroll
    for (int i = 0; i < kE; ++i)
#pragma unroll
        for (int j = 0; j < kH; ++j) acc[i][j] = 0;
    pa.load(p.a, m0, p.M, k_lo, k_hi, 0);
    pb.load(p.b, n0, p.N, k_lo, k_hi, pair_rows);
    int buf = 0;
    for (int k0 = k_lo; k0 < k_hi; k0 += kDepth, buf ^= 1) {
        pa.store(as[buf]);
        pb.store(bs[buf]);
        __syncthreads();  // (the other buffer was read before it)
        if (k0 + kDepth < k_hi) {
            pa.load(p.a, m0, p.M, k0 + kDepth, k_hi, 0);
            pb.load(p.b, n0, p.N, k0 + kDepth, k_hi, pair_rows);
        }
#pragma unroll
        for (int k = 0; k < kDepth; ++k) {
            float a[kE];
            uint64_t b[kH];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float f[kH];
                VecIo<float, kH>::load(&as[buf][k][h * kTile / 2 + ty * kH], f);
#pragma unroll
                for (int i = 0; i < kH; ++i) a[h * kH + i] = f[i];
                VecIo<float, kH>::load(&bs[buf][k][h * kTile / 2 + tx * kH], f);
#pragma unroll
                for (int i = 0; i < kH; i += 2) b[(h * kH + i) / 2] = pair(f[i], f[i + 1]);
            }
#pragma unroll
            for (int i = 0; i < kE; ++i) {
                const uint64_t a2 = pair(a[i], a[i]);
#pragma unroll
                for (int j = 0; j < kH; ++j) acc[i][j] = fma2(a2, b[j], acc[i][j]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kE; ++i) {
        const int m = m0 + (i / kH) * kTile / 2 + ty * kH + i % kH;
        if (m >= p.M) continue;
        float v[kE];
#pragma unroll
        for (int j = 0; j < kH; ++j) unpair(acc[i][j], v[2 * j], v[2 * j + 1]);
        if (kPair) {
#pragma unroll
            for (int j = 0; j < kH; ++j) {
                const int n = n0 + tx * kH + j;
                if (n >= p.N) continue;
                float slope;
                const float a = act_of(p.act, v[j], slope), up = v[kH + j];
                if (kMode == kOut) {
                    p.out[m * p.out_row + n] = a * up;
                } else {
                    const float d = p.dout[m * p.dout_row + n];
                    float *to = p.out + m * p.out_row + n;
                    to[0] = d * up * slope;
                    to[p.N] = d * a;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < kE; ++j) {
                const int n = n0 + (j / kH) * kTile / 2 + tx * kH + j % kH;
                if (n < p.N) p.out[((kMode == kParts ? (long long)blockIdx.y * p.M : 0) + m) * p.out_row + n] = v[j];
            }
        }
    }
}

// out = the sum of `parts` runs of M x N
__global__ void __launch_bounds__(kThreads) ffn_parts_kernel(const float *from, int parts, int M, int N, float *out,
                                                            long long out_row) {
    let_next_begin();
    after_previous();
    const long long all = (long long)M * N;
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < all; i += (long long)gridDim.x * kThreads) {
        float sum = 0.f;
        for (int z = 0; z < parts; ++z) sum += from[z * all + i];
        const long long m = i / N;
        out[m * out_row + (i - m * N)] = sum;
    }
}

constexpr int kSMs = 152;

long long tiles(long long M, long long N, int tile, bool paired) {
    return ((M + tile - 1) / tile) * ((N + (paired ? tile / 2 : tile) - 1) / (paired ? tile / 2 : tile));
}
bool small_tiles(long long M, long long N, bool paired) { return tiles(M, N, 128, paired) < kSMs; }

// how many parts the sum of dx is cut into: as many as bring two blocks an SM, each of 128 indices or more
int parts_of(int M, int K, int F) {
    const long long t = tiles(M, K, small_tiles(M, K, false) ? 64 : 128, false);
    const long long by_blocks = 2 * kSMs / t, by_sum = 2LL * F / 128;
    const long long parts = by_blocks < by_sum ? by_blocks : by_sum;
    return parts < 1 ? 1 : parts > 64 ? 64 : (int)parts;
}

template <bool kA, bool kB, Mode kMode>
cudaError_t product(Product p, int parts, cudaStream_t s) {
    constexpr bool paired = kMode == kOut || kMode == kGrad;
    const int tile = small_tiles(p.M, p.N, paired) ? 64 : 128, cols = paired ? tile / 2 : tile;
    p.across = (p.N + cols - 1) / cols;
    const dim3 grid((unsigned)p.across * ((p.M + tile - 1) / tile), parts);
    return tile == 64 ? launch_after(ffn_product_kernel<64, kA, kB, kMode>, grid, kThreads, 0, s, p)
                      : launch_after(ffn_product_kernel<128, kA, kB, kMode>, grid, kThreads, 0, s, p);
}

const float *floats(const void *p) { return static_cast<const float *>(p); }

cudaError_t forward_f32(const Ffn &p, cudaStream_t s) {
    const Product q{{floats(p.x), p.x_stride, 1}, {floats(p.w), p.K, 1}, p.M, p.F, p.K, p.act, p.K, 0,
                    static_cast<float *>(p.out), p.out_stride, nullptr, 0, reinterpret_cast<WsHeader *>(p.ws)};
    return product<true, true, kOut>(q, 1, s);
}

cudaError_t backward_f32(const FfnBwd &p, cudaStream_t s) {
    const Ffn &f = p.f;
    float *dz = reinterpret_cast<float *>(f.ws + kWsHeaderBytes);
    const int F2 = 2 * f.F, parts = parts_of(f.M, f.K, f.F);
    const Product q{{floats(f.x), f.x_stride, 1}, {floats(f.w), f.K, 1}, f.M, f.F, f.K, f.act, f.K, 0, dz, F2,
                    floats(p.dout), p.dout_stride, reinterpret_cast<WsHeader *>(f.ws)};
    cudaError_t e = product<true, true, kGrad>(q, 1, s);
    if (e) return e;
    const Product dw{{dz, 1, F2}, {floats(f.x), 1, f.x_stride}, F2, f.K, f.M, 0, f.M, 0, static_cast<float *>(p.dw), f.K,
                     nullptr, 0, nullptr};
    e = product<false, false, kProduct>(dw, 1, s);
    if (e) return e;
    Product dx{{dz, F2, 1}, {floats(f.w), 1, f.K}, f.M, f.K, F2, 0, F2, 0, static_cast<float *>(p.dx), p.dx_stride,
               nullptr, 0, nullptr};
    if (parts == 1) return product<true, false, kProduct>(dx, 1, s);
    dx.per = ((F2 + parts - 1) / parts + kDepth - 1) / kDepth * kDepth;
    float *sums = dz + (size_t)f.M * F2;
    dx.out = sums;
    dx.out_row = f.K;
    e = product<true, false, kParts>(dx, parts, s);
    if (e) return e;
    const long long all = (long long)f.M * f.K, blocks = (all + kThreads - 1) / kThreads;
    return launch_after(ffn_parts_kernel, (unsigned)(blocks < 8 * kSMs ? blocks : 8 * kSMs), kThreads, 0, s, sums, parts, f.M,
                        f.K, static_cast<float *>(p.dx), p.dx_stride);
}

}  // namespace

size_t ffn_forward_scratch_bytes(int M, int K, int F, hla_dtype dt) {
    return dt == HLA_BF16 ? ffn_tc_forward_scratch_bytes(M, K, F) : 0;
}
size_t ffn_backward_scratch_bytes(int M, int K, int F, hla_dtype dt) {
    if (dt == HLA_BF16) return ffn_tc_backward_scratch_bytes(M, K, F);
    const int parts = M ? parts_of(M, K, F) : 1;
    return sizeof(float) * ((size_t)M * 2 * F + (parts > 1 ? (size_t)parts * M * K : 0));
}
cudaError_t ffn_forward_launch(const Ffn &p, cudaStream_t s) {
    return p.dt == HLA_BF16 ? ffn_tc_forward(p, s) : forward_f32(p, s);
}
cudaError_t ffn_backward_launch(const FfnBwd &p, cudaStream_t s) {
    return p.f.dt == HLA_BF16 ? ffn_tc_backward(p, s) : backward_f32(p, s);
}

}  // namespace hla
