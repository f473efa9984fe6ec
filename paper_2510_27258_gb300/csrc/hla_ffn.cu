// Gated feed-forward projections and their gradients in fp32, on the CUDA cores (bf16: hla_ffn_sm103.cu).
//
//   Z = x [Wg; Wu]^T (two products of one tile),  out = act(Zg) Zu
//   dZg = dout Zu act'(Zg),  dZu = dout act(Zg),  dx = [dZg dZu] [Wg; Wu],  d[Wg; Wu] = [dZg dZu]^T x
//
// One tiled product serves all four: a block of 256 threads forms 128 x 128 outputs (or 64 x 64, with two groups of
// threads that share each panel's indices, so that SMs have twice the warps), a thread 8 x 8 (4 x 4) of them, from panels
// of 32 (16) in a ring of shared memory, all but the one in use in flight.  A panel lies as its matrix does: where the
// sum's index is the contiguous one a thread reads two (four) of its indices of a row at a time, else four rows of an
// index, so that either way a wide access feeds many products.  The forward's tile is half
// gate and half up columns of the same features, so that the activation and product happen in registers.  The gradient
// keeps [dZg dZu] in the workspace; its last two products, whose sums are over 2 F and over tokens, are cut along the sum
// where that fills the SMs better, and the parts are added in their order.  Few tokens have kernels of their own, below.
//
// Bound by the CUDA cores (80 TFLOP/s at the highest clock): 4096 x 2048 x 1408 44.8 TFLOP/s, its gradient 49; tiles of
// 128 with panels of 32 and products in pairs instead of 16 and single ones: 43.1 and 42.3.  Gradient of 333 x 260 x 1031
// 72 us (one group of threads a small tile 85, four 106), where 1.3 blocks an SM are all there is.
#include <type_traits>

#include "hla_ffn.h"
#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kThreads = 256;
// of a tile of 128 or 64: indices of a panel, panels of the ring, groups of threads that share a panel's indices
constexpr int depth_of(int tile) { return tile == 128 ? 32 : 16; }
constexpr int stages_of(int tile) { return tile == 128 ? 3 : 4; }
constexpr int groups_of(int tile) { return tile == 128 ? 1 : 2; }

enum Mode { kProduct, kParts, kOut, kGrad };

// A matrix of the product, its rows those of A or B and its columns the sum's indices: `step` elements from one row to
// the next where columns are neighbours (kAlong), else from one column to the next.  wide: such runs begin at 16 bytes.
struct Mat {
    const float *p;
    long long step;
    int wide;
};
Mat mat(const float *p, long long step) { return {p, step, rows_aligned(p, step, 4, 16)}; }

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
    const float s = __fdividef(1.f, 1.f + exp_minus<float>(v));
    slope = act == HLA_SIGMOID ? s * (1.f - s) : s * (1.f + v * (1.f - s));
    return act == HLA_SIGMOID ? s : v * s;
}

// A panel of kRows rows and kDepth indices of the sum: rows from `at` on (of `rows`), the second half of them `pair` rows
// behind the first's where pair > 0
template <int kRows, bool kAlong>
struct Panel {
    static constexpr int kDepth = depth_of(kRows);
    static constexpr int kPitch = (kAlong ? kDepth : kRows) + 4, kFloats = (kAlong ? kRows : kDepth) * kPitch;
    static constexpr int kRun = (kAlong ? kDepth : kRows) / 4, kChunks = kRows * kDepth / 4;
    // (by a block of kBlock threads)
    template <int kBlock>
    static __device__ __forceinline__ void send(const Mat &m, float *to, int at, int rows, int pair, int k0, int k1) {
#pragma unroll
        for (int i = 0; i < (kChunks + kBlock - 1) / kBlock; ++i) {
            const int c = threadIdx.x + i * kBlock;
            if (kChunks % kBlock && c >= kChunks) break;
            const int line = c / kRun, four = c % kRun * 4;
            int r = kAlong ? line : four;
            const int k = k0 + (kAlong ? four : line);
            const bool second = pair > 0 && r >= kRows / 2;
            if (second) r -= kRows / 2;
            const long long row = (long long)(at + r) + (second ? pair : 0);
            const int left = kAlong ? (at + r < rows ? k1 - k : 0) : (k < k1 ? rows - at - r : 0);  // of the four
            const float *from = m.p + (kAlong ? row * m.step + k : k * m.step + row);
            const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(to + line * kPitch + four));
            if (m.wide) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(from),
                             "r"(min(max(left, 0), 4) * 4)
                             : "memory");
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 4 * j), "l"(from + j),
                                 "r"(j < left ? 4 : 0)
                                 : "memory");
            }
        }
    }
    // row i of thread t (of 16 along this side)
    static __device__ __forceinline__ int row(int t, int i) { return kAlong ? t + 16 * i : i / 4 * 64 + t * 4 + i % 4; }
    // kK indices from k on of its kE rows
    template <int kE, int kK>
    static __device__ __forceinline__ void get(const float *from, int t, int k, float (&v)[kK][kE]) {
        if constexpr (kAlong) {
#pragma unroll
            for (int i = 0; i < kE; ++i) {
                float f[kK];
                VecIo<float, kK>::load(from + row(t, i) * kPitch + k, f);
#pragma unroll
                for (int q = 0; q < kK; ++q) v[q][i] = f[q];
            }
        } else {
#pragma unroll
            for (int q = 0; q < kK; ++q)
#pragma unroll
                for (int i = 0; i < kE; i += 4) {
                    float f[4];
                    VecIo<float, 4>::load(from + (k + q) * kPitch + row(t, i), f);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[q][i + j] = f[j];
                }
        }
    }
};

// kTile 128 or 64; kA, kB: whether the sum's index is the contiguous one
template <int kTile, bool kA, bool kB, Mode kMode>
__global__ void __launch_bounds__(kThreads *groups_of(kTile)) ffn_product_kernel(Product p) {
    constexpr int kG = groups_of(kTile), kDepth = depth_of(kTile), kStages = stages_of(kTile);
    constexpr int kE = kTile / 16, kK = kTile == 64 ? 4 : 2;  // a thread's rows and columns; indices read at a time
    constexpr bool kPair = kMode == kOut || kMode == kGrad;
    constexpr int kCols = kPair ? kTile / 2 : kTile;
    static_assert(!kPair || kB, "a thread's gate and up columns are of the same features");
    using A = Panel<kTile, kA>;
    using B = Panel<kTile, kB>;
    constexpr int kFloats = A::kFloats + B::kFloats;
    extern __shared__ __align__(16) float ring[];  // [stage][a, b]
    let_next_begin();
    after_previous();
    if (kPair && blockIdx.x == 0 && threadIdx.x == 0) *p.header = WsHeader{};  // no device-side waits here: never an error
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4 & 15, group = threadIdx.x / kThreads;
    const int down = blockIdx.x / p.across, m0 = down * kTile, n0 = (blockIdx.x - down * p.across) * kCols;
    const int k_lo = blockIdx.y * p.per, k_hi = (int)min((long long)p.K, (long long)k_lo + p.per);
    auto send = [&](int stage, int k0) {
        A::template send<kThreads * kG>(p.a, ring + stage * kFloats, m0, p.M, 0, k0, k_hi);
        B::template send<kThreads * kG>(p.b, ring + stage * kFloats + A::kFloats, n0, p.N, kPair ? p.N : 0, k0, k_hi);
        ring_commit();
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) send(i, k_lo + i * kDepth);
    // pairs of products at a time (tiles of 128): of neighbouring indices of the sum where both panels have them side by
    // side, else of neighbouring columns
    constexpr bool kTwo = kTile == 128, kAlong = kA && kB;
    constexpr int kPairs = kAlong ? kE : kE / 2;
    float acc[kE][kE] = {};
    uint64_t pairs[kTwo ? kE : 1][kPairs] = {};
    int stage = 0;
    for (int k0 = k_lo; k0 < k_hi; k0 += kDepth, stage = stage + 1 < kStages ? stage + 1 : 0) {
        ring_wait<kStages - 2>();
        __syncthreads();  // (and the stage of the last step has been read)
        send(stage ? stage - 1 : kStages - 1, k0 + (kStages - 1) * kDepth);
        const float *as = ring + stage * kFloats, *bs = as + A::kFloats;
#pragma unroll
        for (int step = 0; step < kDepth / kG; step += kK) {
            const int k = group * (kDepth / kG) + step;
            float a[kK][kE], b[kK][kE];
            A::template get<kE, kK>(as, ty, k, a);
            B::template get<kE, kK>(bs, tx, k, b);
            if constexpr (kTwo) {
#pragma unroll
                for (int q = 0; q < kK; q += kAlong ? 2 : 1) {
                    uint64_t ap[kE], bp[kPairs];
#pragma unroll
                    for (int i = 0; i < kE; ++i) ap[i] = pair(a[q][i], a[kAlong ? q + 1 : q][i]);
#pragma unroll
                    for (int j = 0; j < kPairs; ++j) {
                        if constexpr (kAlong) bp[j] = pair(b[q][j], b[q + 1][j]);
                        else bp[j] = pair(b[q][2 * j], b[q][2 * j + 1]);
                    }
#pragma unroll
                    for (int i = 0; i < kE; ++i)
#pragma unroll
                        for (int j = 0; j < kPairs; ++j) pairs[i][j] = fma2(ap[i], bp[j], pairs[i][j]);
                }
            } else {
#pragma unroll
                for (int q = 0; q < kK; ++q)
#pragma unroll
                    for (int i = 0; i < kE; ++i)
#pragma unroll
                        for (int j = 0; j < kE; ++j) acc[i][j] = fmaf(a[q][i], b[q][j], acc[i][j]);
            }
        }
    }
    ring_wait<0>();
    if constexpr (kTwo) {
#pragma unroll
        for (int i = 0; i < kE; ++i)
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                float x, y;
                unpair(pairs[i][j], x, y);
                if constexpr (kAlong) {
                    acc[i][j] = x + y;
                } else {
                    acc[i][2 * j] = x;
                    acc[i][2 * j + 1] = y;
                }
            }
    }
    if constexpr (kG > 1) {  // the groups' sums, in their order
        __syncthreads();
#pragma unroll 1
        for (int g = 1; g < kG; ++g) {
#pragma unroll
            for (int i = 0; i < kE * kE; ++i) {
                float *at = ring + i * kThreads + threadIdx.x % kThreads;
                if (group == g) *at = acc[i / kE][i % kE];
            }
            __syncthreads();
            if (group == 0)
#pragma unroll
                for (int i = 0; i < kE * kE; ++i) acc[i / kE][i % kE] += ring[i * kThreads + threadIdx.x];
            __syncthreads();
        }
        if (group > 0) return;
    }
#pragma unroll
    for (int i = 0; i < kE; ++i) {
        const int m = m0 + A::row(ty, i);
        if (m >= p.M) continue;
        if constexpr (kPair) {
#pragma unroll
            for (int j = 0; j < kE / 2; ++j) {
                const int n = n0 + B::row(tx, j);
                if (n >= p.N) continue;
                float slope;
                const float a = act_of(p.act, acc[i][j], slope), up = acc[i][j + kE / 2];
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
                const int n = n0 + B::row(tx, j);
                if (n < p.N) p.out[((kMode == kParts ? (long long)blockIdx.y * p.M : 0) + m) * p.out_row + n] = acc[i][j];
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// few rows: up to 32 tokens, whose tiles of 64 would be half empty while the weights' bytes are what counts.  The sum is
// cut over a block's eight warps and over the blocks of a cluster, whose parts meet in shared memory and are added in
// order; each block finishes some of the tokens.  2048 x 5632: one token 29 us, 16 40, 32 65 (by tiles 140; 33 tokens
// 139), gradient of one 80, of 16 125 instead of 293, of 32 193; the weights' bytes take 14 us (42 in the gradient), the
// rest goes with the tokens (issue slots 63 % in use).  Not kept: panels of 64 indices (no change), four or eight rows
// by eight tokens a lane (gradient of 16 202), two blocks an SM (forward of 16 53).
// ------------------------------------------------------------------------------------------------

constexpr int kFewMost = 32, kWarps = kThreads / 32, kFewDepth = 4 * kWarps, kFewPitch = kFewDepth + 4, kFewStages = 4;
constexpr int few_blocks(int tok) { return tok == 32 ? 2 : 3; }  // of an SM, at 128 or 80 registers a thread

__device__ __forceinline__ unsigned cluster_rank() {
    unsigned r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// one value of every block's, added in the blocks' order
__device__ __forceinline__ float of_blocks(const float *mine, int S) {
    if (S == 1) return *mine;
    float sum = 0.f;
#pragma unroll 2
    for (int b = 0; b < S; ++b) {
        uint32_t at;
        float v;
        asm("mapa.shared::cluster.u32 %0, %1, %2;"
            : "=r"(at)
            : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(mine))), "r"(b));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
        sum += v;
    }
    return sum;
}
// the warps' values ([warp][kValues] in shared memory), added in the warps' order in place of the first's; the cluster's
// blocks have done so when this returns
template <int kValues>
__device__ __forceinline__ void add_warps(float *values, int S) {
    __syncthreads();
    for (int i = threadIdx.x; i < kValues; i += kThreads) {
        float sum = values[i];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) sum += values[w * kValues + i];
        values[i] = sum;
    }
    __syncthreads();
    if (S > 1) cluster_meet();
}

// kOut and kGrad.  A lane has one feature's gate and up row for all tokens, a warp four of a panel's 32 indices.
template <int kTok>
constexpr int kFewFloats = (64 + kTok) * kFewPitch;  // of a panel
template <int kTok, Mode kMode>
__global__ void __launch_bounds__(kThreads, few_blocks(kTok)) ffn_few_kernel(Product p, int S) {
    extern __shared__ __align__(16) float ring[];  // [stage][32 gate rows, 32 up rows, tokens]
    let_next_begin();
    after_previous();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.header = WsHeader{};  // no device-side waits here: never an error
    const int rank = S > 1 ? (int)cluster_rank() : 0, f0 = blockIdx.x / S * 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int k_lo = (int)min((long long)p.K, (long long)rank * p.per), k_hi = (int)min((long long)p.K, (long long)k_lo + p.per);
    auto send = [&](int stage, int k0) {
#pragma unroll
        for (int c = threadIdx.x; c < (64 + kTok) * 8; c += kThreads) {
            const int line = c / 8, four = c % 8 * 4;
            const bool weight = line < 64;
            const Mat &m = weight ? p.b : p.a;
            const int row = weight ? f0 + line % 32 : line - 64, left = row < (weight ? p.N : p.M) ? k_hi - k0 - four : 0;
            const float *from = m.p + ((long long)row + (weight && line >= 32 ? p.N : 0)) * m.step + k0 + four;
            const uint32_t dst =
                static_cast<uint32_t>(__cvta_generic_to_shared(ring + stage * kFewFloats<kTok> + line * kFewPitch + four));
            if (m.wide) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(from),
                             "r"(min(max(left, 0), 4) * 4)
                             : "memory");
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 4 * j), "l"(from + j),
                                 "r"(j < left ? 4 : 0)
                                 : "memory");
            }
        }
        ring_commit();
    };
#pragma unroll
    for (int i = 0; i < kFewStages - 1; ++i) send(i, k_lo + i * kFewDepth);
    float acc[2][kTok] = {};
    int stage = 0;
    for (int k0 = k_lo; k0 < k_hi; k0 += kFewDepth, stage = stage + 1 < kFewStages ? stage + 1 : 0) {
        ring_wait<kFewStages - 2>();
        __syncthreads();  // (and the stage of the last step has been read)
        send(stage ? stage - 1 : kFewStages - 1, k0 + (kFewStages - 1) * kFewDepth);
        const float *at = ring + stage * kFewFloats<kTok> + warp * 4;
        float g[4], u[4];
        VecIo<float, 4>::load(at + lane * kFewPitch, g);
        VecIo<float, 4>::load(at + (32 + lane) * kFewPitch, u);
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            float x[4];
            VecIo<float, 4>::load(at + (64 + t) * kFewPitch, x);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                acc[0][t] = fmaf(g[q], x[q], acc[0][t]);
                acc[1][t] = fmaf(u[q], x[q], acc[1][t]);
            }
        }
    }
    ring_wait<0>();
    __syncthreads();
    constexpr int kValues = 2 * kTok * 32;
#pragma unroll
    for (int t = 0; t < 2 * kTok; ++t) ring[warp * kValues + t * 32 + lane] = acc[t / kTok][t % kTok];
    add_warps<kValues>(ring, S);
    const int each = (p.M + S - 1) / S, lo = rank * each, hi = min(lo + each, p.M);
    for (int t = lo + warp; t < hi; t += kWarps) {
        const int n = f0 + lane;
        const float g = of_blocks(ring + t * 32 + lane, S), up = of_blocks(ring + (kTok + t) * 32 + lane, S);
        if (n >= p.N) continue;
        float slope;
        const float a = act_of(p.act, g, slope);
        float *to = p.out + t * p.out_row + n;
        if (kMode == kOut) {
            *to = a * up;
        } else {
            const float d = p.dout[t * p.dout_row + n];
            to[0] = d * up * slope;
            to[p.N] = d * a;
        }
    }
    if (S > 1) cluster_meet();  // the others have read this block's sums
}

// dx.  A lane has two of 64 columns for all tokens, a warp every eighth row of the weights.
constexpr int kBackCols = 64;
constexpr int back_rows(int tok) { return tok == 32 ? 64 : 128; }  // of a panel
template <int kTok>
constexpr int kBackFloats = kWarps * kTok * kBackCols;  // the warps' sums (and room for a panel of dZ)
template <int kTok>
__global__ void __launch_bounds__(kThreads, 2) ffn_few_back_kernel(Product p, int S) {
    extern __shared__ __align__(16) float panel[];  // [row][token]
    constexpr int kBackRows = back_rows(kTok), kPitch = kTok + 4, kOfWarp = kBackRows / kWarps;
    static_assert(kBackRows * kPitch <= kBackFloats<kTok>, "a panel's room");
    let_next_begin();
    after_previous();
    const int rank = S > 1 ? (int)cluster_rank() : 0, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c0 = blockIdx.x / S * kBackCols + lane;
    const int r_lo = (int)min((long long)p.K, (long long)rank * p.per), r_hi = (int)min((long long)p.K, (long long)r_lo + p.per);
    float acc[2][kTok] = {};
    float next[kOfWarp][2];  // of the weights' next panel
    auto fetch = [&](int r0) {
#pragma unroll
        for (int i = 0; i < kOfWarp; ++i) {
            const int r = r0 + warp + kWarps * i;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                next[i][j] = r < r_hi && c0 + 32 * j < p.N ? p.b.p[r * p.b.step + c0 + 32 * j] : 0.f;
        }
    };
    fetch(r_lo);
    for (int r0 = r_lo; r0 < r_hi; r0 += kBackRows) {
        __syncthreads();  // the last panel has been read
        const int row = threadIdx.x % kBackRows;
#pragma unroll
        for (int t = threadIdx.x / kBackRows; t < kTok; t += kThreads / kBackRows)
            panel[row * kPitch + t] = t < p.M && r0 + row < r_hi ? p.a.p[t * p.a.step + r0 + row] : 0.f;
        float w[kOfWarp][2];
#pragma unroll
        for (int i = 0; i < kOfWarp; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) w[i][j] = next[i][j];
        fetch(r0 + kBackRows);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kOfWarp; ++i)
#pragma unroll
            for (int t = 0; t < kTok; t += 4) {
                float d[4];
                VecIo<float, 4>::load(panel + (warp + kWarps * i) * kPitch + t, d);
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[j][t + q] = fmaf(w[i][j], d[q], acc[j][t + q]);
            }
    }
    __syncthreads();
    constexpr int kValues = kTok * kBackCols;
#pragma unroll
    for (int t = 0; t < 2 * kTok; ++t) panel[warp * kValues + t / 2 * kBackCols + t % 2 * 32 + lane] = acc[t % 2][t / 2];
    add_warps<kValues>(panel, S);
    const int each = (p.M + S - 1) / S, lo = rank * each, hi = min(lo + each, p.M);
    for (int i = threadIdx.x; i < (hi - lo) * kBackCols; i += kThreads) {
        const int t = lo + i / kBackCols, c = i % kBackCols, n = blockIdx.x / S * kBackCols + c;
        const float sum = of_blocks(panel + t * kBackCols + c, S);
        if (n < p.N) p.out[t * p.out_row + n] = sum;
    }
    if (S > 1) cluster_meet();  // the others have read this block's sums
}

// dw of up to 16 tokens (above, a tile's panel is full enough: 32 of them 196 us instead of 212 in all).  A lane has four of
// 128 columns of x for all tokens, a warp every eighth of a panel's rows of dZ.
constexpr int kFewWeights = 16;
template <int kTok>
__global__ void __launch_bounds__(kThreads) ffn_few_weights_kernel(Product p) {
    constexpr int kCols = 4, kRows = 128, kPitch = kTok + 4;
    __shared__ __align__(16) float panel[kRows * kPitch];  // [row][token]
    let_next_begin();
    after_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int down = blockIdx.x / p.across, r0 = down * kRows, c0 = (blockIdx.x - down * p.across) * 32 * kCols + lane;
    float x[kCols][kTok];
#pragma unroll
    for (int t = 0; t < kTok; ++t)
#pragma unroll
        for (int j = 0; j < kCols; ++j) x[j][t] = t < p.K && c0 + 32 * j < p.N ? p.b.p[t * p.b.step + c0 + 32 * j] : 0.f;
    const int row = threadIdx.x % kRows;
#pragma unroll
    for (int t = threadIdx.x / kRows; t < kTok; t += kThreads / kRows)
        panel[row * kPitch + t] = t < p.K && r0 + row < p.M ? p.a.p[t * p.a.step + r0 + row] : 0.f;
    __syncthreads();
#pragma unroll 2
    for (int i = warp; i < kRows; i += kWarps) {
        if (r0 + i >= p.M) break;
        float sum[kCols] = {};
#pragma unroll
        for (int t = 0; t < kTok; t += 4) {
            float d[4];
            VecIo<float, 4>::load(panel + i * kPitch + t, d);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < kCols; ++j) sum[j] = fmaf(x[j][t + q], d[q], sum[j]);
        }
        float *to = p.out + (r0 + i) * p.out_row + c0;
#pragma unroll
        for (int j = 0; j < kCols; ++j)
            if (c0 + 32 * j < p.N) to[32 * j] = sum[j];
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
#pragma unroll 8
        for (int z = 0; z < parts; ++z) sum += from[z * all + i];
        const long long m = i / N;
        out[m * out_row + (i - m * N)] = sum;
    }
}

constexpr int kSMs = 152;

long long tiles(long long M, long long N, int tile, bool paired) {
    return ((M + tile - 1) / tile) * ((N + (paired ? tile / 2 : tile) - 1) / (paired ? tile / 2 : tile));
}

// Tiles of 128 or 64, and how many parts the sum is cut into
struct Plan {
    int tile, parts;
};
// What takes least by this count, in us: the blocks that an SM works through, each with its share of the sum, at the rates
// that full SMs reach (48 and 36 TFLOP/s over all of them; blocks of 64 that have an SM each take 1.7 times as long),
// and the parts' way through memory.  A part has 128 indices or more.  Against tiles of 128 wherever there are 152 and
// as many parts as bring two blocks an SM: gradient of 2048 x 1024 x 2816 1522 us instead of 1849, of 1000 x 512 x 1500 268
// instead of 343.
Plan plan(long long M, long long N, long long sum, bool paired, int most) {
    Plan best{128, 1};
    double least = 0;
    for (int tile = 128; tile >= 64; tile /= 2)
        for (int parts = 1; parts == 1 || (parts <= most && sum / parts >= 128); ++parts) {
            const long long rounds = (tiles(M, N, tile, paired) * parts + kSMs - 1) / kSMs;
            const double each = 2. * tile * tile * (double)((sum + parts - 1) / parts) / ((tile == 128 ? 48e6 : 36e6) / kSMs);
            const double start = tile == 128 ? 2 : rounds == 1 ? 0.7 * each : 0;
            const double us = rounds * each + start + (parts > 1 ? 5 + parts * 8e-6 * (double)(M * N) / 6 : 0);
            if ((tile == 128 && parts == 1) || us < least) {
                least = us;
                best = {tile, parts};
            }
        }
    return best;
}
constexpr int kMostParts = 64;
Plan plan_dx(int M, int K, int F) { return plan(M, K, 2LL * F, false, kMostParts); }
Plan plan_dw(int M, int K, int F) { return plan(2LL * F, K, M, false, kMostParts); }

template <bool kA, bool kB, Mode kMode>
cudaError_t product(Product p, const Plan &by, cudaStream_t s) {
    constexpr bool paired = kMode == kOut || kMode == kGrad;
    const int tile = by.tile, cols = paired ? tile / 2 : tile;
    p.across = (p.N + cols - 1) / cols;
    const dim3 grid((unsigned)p.across * ((p.M + tile - 1) / tile), by.parts);
    auto as = [&](auto kernel, int floats) -> cudaError_t {
        const int smem = stages_of(tile) * floats * (int)sizeof(float);
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        return e ? e : launch_after(kernel, grid, kThreads * groups_of(tile), smem, s, p);
    };
    return tile == 64 ? as(ffn_product_kernel<64, kA, kB, kMode>, Panel<64, kA>::kFloats + Panel<64, kB>::kFloats)
                      : as(ffn_product_kernel<128, kA, kB, kMode>, Panel<128, kA>::kFloats + Panel<128, kB>::kFloats);
}

// Few rows: blocks of a cluster as many as fill `blocks` an SM, each with `least` indices of the sum or more
template <typename K>
cudaError_t few(K kernel, Product p, long long tiles, int blocks, int least, int step, int floats, cudaStream_t s) {
    int S = 1;
    while (S < 8 && tiles * S * 2 <= blocks * kSMs && p.K >= S * 2 * least) S *= 2;
    p.per = ((p.K + S - 1) / S + step - 1) / step * step;
    const int smem = floats * (int)sizeof(float);
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    return e ? e : launch_cluster_after(kernel, (unsigned)(tiles * S), kThreads, S, smem, s, p, S);
}
template <Mode kMode>
cudaError_t few_forward(const Product &p, cudaStream_t s) {
    auto as = [&](auto Tok) {
        constexpr int kTok = Tok(), kSums = kWarps * 2 * kTok * 32, kRing = kFewStages * kFewFloats<kTok>;
        return few(ffn_few_kernel<kTok, kMode>, p, (p.N + 31) / 32, 3, 4 * kFewDepth, kFewDepth,
                   kRing > kSums ? kRing : kSums, s);
    };
    return p.M <= 8    ? as(std::integral_constant<int, 8>())
           : p.M <= 16 ? as(std::integral_constant<int, 16>())
                       : as(std::integral_constant<int, 32>());
}
cudaError_t few_back(const Product &p, cudaStream_t s) {
    auto as = [&](auto Tok) {
        constexpr int kTok = Tok();
        return few(ffn_few_back_kernel<kTok>, p, (p.N + kBackCols - 1) / kBackCols, 2, 128, back_rows(kTok),
                   kBackFloats<kTok>, s);
    };
    return p.M <= 8    ? as(std::integral_constant<int, 8>())
           : p.M <= 16 ? as(std::integral_constant<int, 16>())
                       : as(std::integral_constant<int, 32>());
}

cudaError_t few_weights(Product p, cudaStream_t s) {
    p.across = (p.N + 127) / 128;
    const unsigned blocks = (unsigned)p.across * ((p.M + 127) / 128);
    return p.K <= 8 ? launch_after(ffn_few_weights_kernel<8>, blocks, kThreads, 0, s, p)
                    : launch_after(ffn_few_weights_kernel<16>, blocks, kThreads, 0, s, p);
}

const float *floats(const void *p) { return static_cast<const float *>(p); }

size_t parts_floats(int parts, long long M, long long N) { return parts > 1 ? (size_t)parts * M * N : 0; }

// a product whose sum is cut into parts, which lie in `sums` until they are added
template <bool kA>
cudaError_t cut_product(Product p, const Plan &by, float *sums, cudaStream_t s) {
    const int parts = by.parts, depth = depth_of(by.tile);
    if (parts == 1) return product<kA, false, kProduct>(p, by, s);
    float *out = p.out;
    const long long out_row = p.out_row, all = (long long)p.M * p.N, blocks = (all + kThreads - 1) / kThreads;
    p.per = ((p.K + parts - 1) / parts + depth - 1) / depth * depth;
    p.out = sums;
    p.out_row = p.N;
    const cudaError_t e = product<kA, false, kParts>(p, by, s);
    if (e) return e;
    return launch_after(ffn_parts_kernel, (unsigned)(blocks < 8 * kSMs ? blocks : 8 * kSMs), kThreads, 0, s, sums, parts,
                        p.M, p.N, out, out_row);
}

// [dZg dZu] in rows of whole 16 bytes
long long dz_row(int F) { return (2LL * F + 3) / 4 * 4; }

cudaError_t forward_f32(const Ffn &p, cudaStream_t s) {
    const Product q{mat(floats(p.x), p.x_stride), mat(floats(p.w), p.K), p.M, p.F, p.K, p.act, p.K, 0,
                    static_cast<float *>(p.out), p.out_stride, nullptr, 0, reinterpret_cast<WsHeader *>(p.ws)};
    return p.M <= kFewMost ? few_forward<kOut>(q, s) : product<true, true, kOut>(q, plan(p.M, p.F, p.K, true, 1), s);
}

cudaError_t backward_f32(const FfnBwd &p, cudaStream_t s) {
    const Ffn &f = p.f;
    float *dz = reinterpret_cast<float *>(f.ws + kWsHeaderBytes);
    const int F2 = 2 * f.F;
    const long long row = dz_row(f.F);
    const Product q{mat(floats(f.x), f.x_stride), mat(floats(f.w), f.K), f.M, f.F, f.K, f.act, f.K, 0, dz, row,
                    floats(p.dout), p.dout_stride, reinterpret_cast<WsHeader *>(f.ws)};
    cudaError_t e = f.M <= kFewMost ? few_forward<kGrad>(q, s) : product<true, true, kGrad>(q, plan(f.M, f.F, f.K, true, 1), s);
    if (e) return e;
    float *sums = dz + (size_t)f.M * row;
    const Product dw{mat(dz, row), mat(floats(f.x), f.x_stride), F2, f.K, f.M, 0, f.M, 0, static_cast<float *>(p.dw), f.K,
                     nullptr, 0, nullptr};
    if (f.M <= kFewWeights) {
        e = few_weights(dw, s);
        if (e) return e;
    } else {
        const Plan by_dw = plan_dw(f.M, f.K, f.F);
        e = cut_product<false>(dw, by_dw, sums, s);
        if (e) return e;
        sums += parts_floats(by_dw.parts, F2, f.K);
    }
    const Product dx{mat(dz, row), mat(floats(f.w), f.K), f.M, f.K, F2, 0, F2, 0, static_cast<float *>(p.dx), p.dx_stride,
                     nullptr, 0, nullptr};
    return f.M <= kFewMost ? few_back(dx, s) : cut_product<true>(dx, plan_dx(f.M, f.K, f.F), sums, s);
}

}  // namespace

size_t ffn_forward_scratch_bytes(int M, int K, int F, hla_dtype dt) {
    return dt == HLA_BF16 ? ffn_tc_forward_scratch_bytes(M, K, F) : 0;
}
size_t ffn_backward_scratch_bytes(int M, int K, int F, hla_dtype dt) {
    if (dt == HLA_BF16) return ffn_tc_backward_scratch_bytes(M, K, F);
    if (M == 0) return 0;
    if (M <= kFewMost) return sizeof(float) * (size_t)M * dz_row(F);  // (a sum of so few is not cut)
    const Plan dx = plan_dx(M, K, F), dw = plan_dw(M, K, F);
    return sizeof(float) * ((size_t)M * dz_row(F) + parts_floats(dx.parts, M, K) + parts_floats(dw.parts, 2LL * F, K));
}
cudaError_t ffn_forward_launch(const Ffn &p, cudaStream_t s) {
    return p.dt == HLA_BF16 ? ffn_tc_forward(p, s) : forward_f32(p, s);
}
cudaError_t ffn_backward_launch(const FfnBwd &p, cudaStream_t s) {
    return p.f.dt == HLA_BF16 ? ffn_tc_backward(p, s) : backward_f32(p, s);
}

}  // namespace hla
