// Short causal depthwise convolution: forward over a prompt, one-token step, gradients.
//
//   pre_t = bias + sum_j w[c, j] x_{t - (W-1) + j},   out_t = pre_t or silu(pre_t)
//   g_t = dout_t (silu'(pre_t)),  dx_t = sum_j w[c, j] g_{t + (W-1) - j},
//   dw[c, j] = sum_t g_t x_{t - (W-1) + j},  dbias = sum_t g_t
//
// Rows x_t with t < 0 come from the state (the last W - 1 rows before the call) or are zero; rows at
// and after a sequence's length give zero outputs and are not read.
//
// About 2 W flops a value: bound by memory traffic.  A thread owns V neighbouring channels (one
// 16-byte access a row, neighbouring lanes on neighbouring channels) and walks a strip of
// consecutive tokens with the W - 1 previous rows in registers, so each x row is loaded once a strip
// and W - 1 rows a strip are read twice (from L2).  A ring of kAhead rows is in flight (asynchronous
// copies: a ring in registers took 43 us where this took 29).
//
// Measured on a GB300: forward, B2 n8192 C2304 bf16, 28.3 us a pass (5.3 TB/s), gradient, B8 n2048
// C1280 bf16, 31.6 us (4.0 TB/s: latency, with 122 registers and so at most 16 warps an SM; issue slots are 49 %
// and DRAM 40 % busy), step of 64 sequences 2.3 us.
#include <type_traits>

#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kThreads = 128, kStrips = kThreads / 32;
constexpr int kAhead = 8;  // rows a thread has in flight
constexpr int kAheadBwd = 4;
constexpr int kStrip = 4;  // strip lengths are multiples of this

struct Geom {
    int B, n, C, L;          // L: tokens a strip
    int cblocks, tblocks;    // blocks along the channels (32 V each) and the tokens (kStrips L each)
};

struct Place {
    int b, c0, t0;
    bool lead;  // this warp holds a sequence's first strip
};

template <int V>
__device__ __forceinline__ Place place(const Geom &g) {
    const int cb = blockIdx.x % g.cblocks, rest = blockIdx.x / g.cblocks;
    const int tb = rest % g.tblocks, warp = threadIdx.x >> 5;
    return {rest / g.tblocks, (cb * 32 + (int)(threadIdx.x & 31)) * V, (tb * kStrips + warp) * g.L,
            tb == 0 && warp == 0};
}

__device__ __forceinline__ int length_of(const int *lengths, int b, int n) {
    if (!lengths) return n;
    const int m = lengths[b];
    return m < 0 ? 0 : m > n ? n : m;
}

__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// sigmoids of a pair, 1 / (1 + 2^(-v log2 e)).  (exp(-v) may overflow: the reciprocal is then 0.)
__device__ __forceinline__ uint64_t sigmoids(uint64_t v) {
    float e0, e1, s0, s1;
    unpair(mul2(v, pair(-1.4426950408889634f, -1.4426950408889634f)), e0, e1);
    unpair(add2(pair(fast_exp2(e0), fast_exp2(e1)), pair(1.f, 1.f)), e0, e1);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s0) : "f"(e0));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s1) : "f"(e1));
    return pair(s0, s1);
}

// w[c0 .. c0 + V - 1][W] and bias[c0 ..] as pairs of channels
template <typename T, int W, int V>
__device__ __forceinline__ void load_taps(const T *w, const T *bias, int c0, uint64_t (&wr)[W][(V + 1) / 2],
                                          uint64_t (&br)[(V + 1) / 2]) {
    float flat[W][V];  // V W consecutive elements
#pragma unroll
    for (int i = 0; i < W; ++i) VecIo<T, V>::load(w + (size_t)c0 * W + i * V, flat[i]);
#pragma unroll
    for (int v = 0; v < V; v += 2)
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const int a = v * W + j, b = a + W;
            wr[j][v / 2] = pair(flat[a / V][a % V], v + 1 < V ? flat[(b / V) % W][b % V] : 0.f);
        }
#pragma unroll
    for (int v = 0; v < (V + 1) / 2; ++v) br[v] = pair(0.f, 0.f);
    if (bias) to_pairs(raw_load<T, V>(bias + c0), br);
}

// row t of x (t >= 0), of the state (-(W-1) <= t < 0), or zero
template <typename T, int W, int V>
__device__ __forceinline__ Raw<T, V> load_row(const T *x, size_t stride, const T *state, int C, int c0, int t) {
    if (t >= 0) return raw_load<T, V>(x + (size_t)t * stride + c0);
    if (state) return raw_load<T, V>(state + (size_t)(t + W - 1) * C + c0);
    return raw_zero<T, V>();
}

template <typename T, int W, int V, bool kSilu>
__global__ void __launch_bounds__(kThreads)
conv_forward_kernel(Geom g, const T *x, const T *w, const T *bias,
                    T *out, size_t xs, size_t os, const int *lengths, const T *state_in,
                    T *state_out) {
    __shared__ Raw<T, V> ring[kAhead][kThreads];
    let_next_begin();
    after_previous();
    const Place at = place<V>(g);
    if (at.c0 >= g.C) return;
    const int len = length_of(lengths, at.b, g.n);
    x += (size_t)at.b * g.n * xs;
    out += (size_t)at.b * g.n * os + at.c0;
    const T *st = state_in ? state_in + (size_t)at.b * (W - 1) * g.C : nullptr;
    const int end = min(at.t0 + g.L, g.n), live = min(end, len);
    if (at.t0 < live) {
        constexpr int kP = (V + 1) / 2;
        uint64_t wr[W][kP], br[kP], win[W][kP];  // row t of x in win[t % W] (counted from the strip's start)
        const T *src = x + (size_t)at.t0 * xs + at.c0;
        const int count = live - at.t0;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            ring_copy<T, V>(&ring[u][threadIdx.x], src + (size_t)u * xs, u < count);
            ring_commit();
        }
        load_taps<T, W, V>(w, bias, at.c0, wr, br);
#pragma unroll
        for (int i = 1; i < W; ++i) to_pairs(load_row<T, W, V>(x, xs, st, g.C, at.c0, at.t0 - W + i), win[i]);
        // unrolled over a common multiple of the window's and the ring's turns
        constexpr int kTurn = W == 3 ? 3 * kAhead : kAhead;
        T *dst = out + (size_t)at.t0 * os;
        src += (size_t)kAhead * xs;
        for (int t = 0; t < count; t += kTurn) {
#pragma unroll
            for (int u = 0; u < kTurn; ++u) {
                if (t + u < count) {
                    ring_wait<kAhead - 1>();
                    Raw<T, V> &slot = ring[u % kAhead][threadIdx.x];
                    to_pairs(slot, win[u % W]);
                    ring_copy<T, V>(&slot, src, t + u + kAhead < count);
                    ring_commit();
                    src += xs;
                    uint64_t y[kP];
#pragma unroll
                    for (int v = 0; v < kP; ++v) {
                        y[v] = br[v];
#pragma unroll
                        for (int j = 0; j < W; ++j) y[v] = fma2(wr[j][v], win[(u + 1 + j) % W][v], y[v]);
                        if (kSilu) y[v] = mul2(y[v], sigmoids(y[v]));
                    }
                    store_pairs<T, V>(dst, y);
                    dst += os;
                }
            }
        }
    }
    const float zero[V] = {};
    for (int t = max(at.t0, live); t < end; ++t) VecIo<T, V>::store(out + (size_t)t * os, zero);
    // the state after the sequence's last token; the thread that read these channels' state_in
    // writes it, so the two may be the same buffer
    if (state_out && at.lead) {
        Raw<T, V> r[W - 1];
#pragma unroll
        for (int i = 0; i < W - 1; ++i) r[i] = load_row<T, W, V>(x, xs, st, g.C, at.c0, len - (W - 1) + i);
#pragma unroll
        for (int i = 0; i < W - 1; ++i)
            *reinterpret_cast<Raw<T, V> *>(state_out + ((size_t)at.b * (W - 1) + i) * g.C + at.c0) = r[i];
    }
}

// one token a sequence: out = act(bias + taps . [state, x]), the state shifted by one row in place
template <typename T, int W, int V, bool kSilu>
__global__ void __launch_bounds__(kThreads)
conv_step_kernel(long long units, int C, const T *x, const T *w, const T *bias, T *out,
                 size_t xs, size_t os, T *state) {
    let_next_begin();
    after_previous();
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (i >= units) return;
    const int per = C / V, c0 = (int)(i % per) * V;
    const size_t b = i / per;
    constexpr int kP = (V + 1) / 2;
    Raw<T, V> row[W];
    T *st = state + b * (W - 1) * C + c0;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) row[j] = raw_load<T, V>(st + (size_t)j * C);
    row[W - 1] = raw_load<T, V>(x + b * xs + c0);
    uint64_t wr[W][kP], y[kP];
    load_taps<T, W, V>(w, bias, c0, wr, y);
#pragma unroll
    for (int j = 0; j < W; ++j) {
        uint64_t f[kP];
        to_pairs(row[j], f);
#pragma unroll
        for (int v = 0; v < kP; ++v) y[v] = fma2(wr[j][v], f[v], y[v]);
    }
    if (kSilu) {
#pragma unroll
        for (int v = 0; v < kP; ++v) y[v] = mul2(y[v], sigmoids(y[v]));
    }
    store_pairs<T, V>(out + b * os + c0, y);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) *reinterpret_cast<Raw<T, V> *>(st + (size_t)j * C) = row[j + 1];
}

// Gradients.  A strip computes g for its tokens and the W - 1 that follow (which its dx needs), sums
// dw and dbias over its own tokens in registers, then over the block's strips in shared memory, and
// writes one partial [W + 1][C] a token block; conv_sum_kernel adds the partials in a fixed order, so
// equal inputs give equal bits.
template <typename T, int W, int V, bool kSilu>
__global__ void __launch_bounds__(kThreads)
conv_backward_kernel(Geom g, const T *x, const T *w, const T *bias,
                     const T *dout, T *dx, size_t xs, size_t gs, size_t ds,
                     const int *lengths, float *partial) {
    union Scratch {
        Raw<T, V> ring[2][kAheadBwd][kThreads];
        float red[kStrips][W + 1][V][32];
    };
    __shared__ Scratch sm;
    auto &red = sm.red;
    let_next_begin();
    after_previous();
    const Place at = place<V>(g);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kP = (V + 1) / 2;
    uint64_t dw[W + 1][kP] = {};  // row W: dbias
    if (at.c0 < g.C) {
        const int len = length_of(lengths, at.b, g.n);
        x += (size_t)at.b * g.n * xs + at.c0;
        dout += (size_t)at.b * g.n * gs + at.c0;
        dx += (size_t)at.b * g.n * ds + at.c0;
        const int end = min(at.t0 + g.L, g.n), live = min(end, len);
        if (at.t0 < live) {
            // rows t of x and g in xw[t % W], gw[t % W] (counted from the strip's start)
            uint64_t wr[W][kP], br[kP], xw[W][kP], gw[W][kP];
            const int last = min(live + W - 1, len);  // tokens from here on have g = 0
            const T *xp = x + (size_t)at.t0 * xs, *gp = dout + (size_t)at.t0 * gs;
#pragma unroll
            for (int u = 0; u < kAheadBwd; ++u) {
                ring_copy<T, V>(&sm.ring[0][u][threadIdx.x], xp, at.t0 + u < last);
                ring_copy<T, V>(&sm.ring[1][u][threadIdx.x], gp, at.t0 + u < last);
                ring_commit();
                xp += xs;
                gp += gs;
            }
            load_taps<T, W, V>(w, bias, at.c0, wr, br);
#pragma unroll
            for (int i = 0; i < W; ++i) {
#pragma unroll
                for (int v = 0; v < kP; ++v) xw[i][v] = gw[i][v] = pair(0.f, 0.f);
                if (i > 0 && at.t0 - W + i >= 0) to_pairs(raw_load<T, V>(x + (size_t)(at.t0 - W + i) * xs), xw[i]);
            }
            constexpr int kTurn = W == 3 ? 3 * kAheadBwd : kAheadBwd;
            T *to = dx + (size_t)at.t0 * ds;  // of token t + u - (W - 1), once its g and the next W - 1 are there
            auto turn = [&](int t, auto edge) {
                constexpr bool kEdge = edge();
#pragma unroll
                for (int u = 0; u < kTurn; ++u) {
                    const int tt = t + u;
                    if (!kEdge || tt < live + W - 1) {
                        uint64_t(&gc)[kP] = gw[u % W];
                        ring_wait<kAheadBwd - 1>();
                        Raw<T, V> &xr = sm.ring[0][u % kAheadBwd][threadIdx.x], &gr = sm.ring[1][u % kAheadBwd][threadIdx.x];
                        to_pairs(!kEdge || tt < last ? xr : raw_zero<T, V>(), xw[u % W]);
                        to_pairs(!kEdge || tt < last ? gr : raw_zero<T, V>(), gc);
                        ring_copy<T, V>(&xr, xp, !kEdge || tt + kAheadBwd < last);
                        ring_copy<T, V>(&gr, gp, !kEdge || tt + kAheadBwd < last);
                        ring_commit();
                        xp += xs;
                        gp += gs;
                        if (kSilu) {
#pragma unroll
                            for (int v = 0; v < kP; ++v) {
                                uint64_t a = br[v];
#pragma unroll
                                for (int j = 0; j < W; ++j) a = fma2(wr[j][v], xw[(u + 1 + j) % W][v], a);
                                const uint64_t s = sigmoids(a), one = pair(1.f, 1.f);
                                gc[v] = mul2(mul2(gc[v], s), fma2(a, fma2(s, pair(-1.f, -1.f), one), one));
                            }
                        }
                        if (kEdge && tt >= last) {  // (silu' of a row that was not read may be anything)
#pragma unroll
                            for (int v = 0; v < kP; ++v) gc[v] = pair(0.f, 0.f);
                        }
                        if (!kEdge || tt < live) {
#pragma unroll
                            for (int v = 0; v < kP; ++v) {
#pragma unroll
                                for (int j = 0; j < W; ++j) dw[j][v] = fma2(gc[v], xw[(u + 1 + j) % W][v], dw[j][v]);
                                dw[W][v] = add2(dw[W][v], gc[v]);
                            }
                        }
                        if (!kEdge || tt - (W - 1) >= at.t0) {
                            uint64_t d[kP];
#pragma unroll
                            for (int v = 0; v < kP; ++v) {
                                d[v] = mul2(wr[0][v], gw[u % W][v]);
#pragma unroll
                                for (int j = 1; j < W; ++j) d[v] = fma2(wr[j][v], gw[(u + W - j) % W][v], d[v]);
                            }
                            store_pairs<T, V>(to, d);
                            to += ds;
                        }
                    }
                }
            };
            // (a turn with neither end of the strip in it needs no conditions: 37 -> 34 us)
            for (int t = at.t0; t < live + W - 1; t += kTurn) {
                if (t > at.t0 && t + kTurn + kAheadBwd <= last && t + kTurn <= live)
                    turn(t, std::false_type());
                else
                    turn(t, std::true_type());
            }
        }
        const float zero[V] = {};
        for (int t = max(at.t0, live); t < end; ++t) VecIo<T, V>::store(dx + (size_t)t * ds, zero);
    }
    __syncthreads();  // every thread has done with its ring
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int v = 0; v < kP; ++v) {
            float d0, d1;
            unpair(dw[j][v], d0, d1);
            red[warp][j][2 * v][lane] = d0;
            if (2 * v + 1 < V) red[warp][j][2 * v + 1][lane] = d1;
        }
    __syncthreads();
    const int cb = blockIdx.x % g.cblocks;
    float *to = partial + (size_t)(blockIdx.x / g.cblocks) * (W + 1) * g.C;
    for (int i = threadIdx.x; i < (W + 1) * V * 32; i += kThreads) {
        const int j = i / (V * 32), c = i % (V * 32);  // channel c of the block: lane c / V, element c % V
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kStrips; ++k) s += red[k][j][c % V][c / V];
        if (cb * 32 * V + c < g.C) to[(size_t)j * g.C + cb * 32 * V + c] = s;
    }
}

// dw[c][j] and dbias[c] from `rows` partials [W + 1][C]: 32 entries a block, a warp for every 16th row.  (The entries
// of 430 million channels and more pass 32 bits.)
constexpr int kSumGroups = 16;
template <int W>
__global__ void __launch_bounds__(kSumGroups * 32)
conv_sum_kernel(const float *partial, int rows, int C, float *dw, float *dbias,
                WsHeader *header) {
    __shared__ float red[kSumGroups][32];
    let_next_begin();
    after_previous();
    if (blockIdx.x == 0 && threadIdx.x == 0) *header = WsHeader{};  // no device-side waits here: never an error
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const size_t width = (size_t)(W + 1) * C, i = (size_t)blockIdx.x * 32 + lane;
    float s = 0.f;
    if (i < width)
#pragma unroll 8
        for (int r = group; r < rows; r += kSumGroups) s += partial[(size_t)r * width + i];
    red[group][lane] = s;
    __syncthreads();
    if (group || i >= width) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < kSumGroups; ++k) s += red[k][lane];
    size_t c = i;
    int j = 0;
    for (; c >= (size_t)C; c -= C) ++j;  // (at most W)
    if (j < W)
        dw[c * W + j] = s;
    else if (dbias)
        dbias[c] = s;
}

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// Strip length: the one that ends first, by the blocks of the fullest SM (at least kFull, below which
// they gain nothing from one another's absence), each costing its strip and about eight tokens more
// (the rows read twice, the taps, the first loads)
Geom geometry(int B, int n, int C, int V) {
    constexpr long long kFull = 4;
    Geom g{B, n, C, kStrip, ceil_div(C, 32 * V), 1};
    long long best = 0;
    for (int L = kStrip; L <= 128; L += kStrip) {
        const long long tb = n > 0 ? ceil_div(n, (long long)L * kStrips) : 1;
        long long blocks = ((long long)B * g.cblocks * tb + 151) / 152;
        if (blocks < kFull) blocks = kFull;
        if (L == kStrip || blocks * (L + 8) <= best) {
            best = blocks * (L + 8);
            g.L = L;
            g.tblocks = (int)tb;
        }
    }
    return g;
}

template <typename F>
cudaError_t by_width(int width, F f) {
    switch (width) {
        case 2: return f(std::integral_constant<int, 2>());
        case 3: return f(std::integral_constant<int, 3>());
        default: return f(std::integral_constant<int, 4>());
    }
}

template <typename T, int V, bool kSilu>
cudaError_t forward_as(const Conv &p, cudaStream_t s) {
    return by_width(p.width, [&](auto W) -> cudaError_t {
        const Geom g = geometry(p.B, p.n, p.C, V);
        const unsigned blocks = (unsigned)g.cblocks * g.tblocks * p.B;
        return launch_after(conv_forward_kernel<T, W(), V, kSilu>, blocks, kThreads, 0, s,
            g, (const T *)p.x, (const T *)p.w, (const T *)p.bias, (T *)p.out, p.x_stride, p.out_stride, p.lengths,
            (const T *)p.state_in, (T *)p.state_out);
    });
}

template <typename T, int V, bool kSilu>
cudaError_t step_as(const Conv &p, cudaStream_t s) {
    return by_width(p.width, [&](auto W) -> cudaError_t {
        const long long units = (long long)p.B * (p.C / V);
        return launch_after(conv_step_kernel<T, W(), V, kSilu>, ceil_div(units, kThreads), kThreads, 0, s,
            units, p.C, (const T *)p.x, (const T *)p.w, (const T *)p.bias, (T *)p.out, p.x_stride, p.out_stride,
            (T *)p.state_out);
    });
}

template <typename T, int V, bool kSilu>
cudaError_t backward_as(const ConvBwd &p, cudaStream_t s) {
    return by_width(p.width, [&](auto W) -> cudaError_t {
        const Geom g = geometry(p.B, p.n, p.C, V);
        const int rows = g.tblocks * p.B;
        cudaError_t e = launch_after(conv_backward_kernel<T, W(), V, kSilu>, (unsigned)g.cblocks * rows, kThreads, 0, s,
            g, (const T *)p.x, (const T *)p.w, (const T *)p.bias, (const T *)p.dout, (T *)p.dx, p.x_stride,
            p.dout_stride, p.dx_stride, p.lengths, p.partial);
        if (e) return e;
        return launch_after(conv_sum_kernel<W()>, ceil_div((long long)(W() + 1) * p.C, 32), kSumGroups * 32, 0, s,
                            p.partial, rows, p.C, p.dw, p.dbias, p.header);
    });
}

// the widest access that the channel count, the pointers and the strides allow
bool wide(const Conv &p, size_t eb, int V) {
    const size_t by = V * eb;
    return p.C % V == 0 && rows_aligned(p.x, p.x_stride, eb, by) && rows_aligned(p.out, p.out_stride, eb, by) &&
           rows_aligned(p.w, 0, eb, by) && rows_aligned(p.bias, 0, eb, by) && rows_aligned(p.state_in, p.C, eb, by) &&
           rows_aligned(p.state_out, p.C, eb, by);
}

bool wide(const ConvBwd &p, size_t eb, int V) {
    const size_t by = V * eb;
    return p.C % V == 0 && rows_aligned(p.x, p.x_stride, eb, by) && rows_aligned(p.dout, p.dout_stride, eb, by) &&
           rows_aligned(p.dx, p.dx_stride, eb, by) && rows_aligned(p.w, 0, eb, by) && rows_aligned(p.bias, 0, eb, by);
}

}  // namespace

// the largest of what the variants write
size_t conv_backward_partial_floats(int B, int n, int C, int width) {
    size_t rows = 0;
    for (int V : {1, 2, 4}) {
        const Geom g = geometry(B, n, C, V);
        const size_t r = (size_t)g.tblocks * B;
        if (r > rows) rows = r;
    }
    return rows * (width + 1) * C;
}

// the widest access of V16 (bf16) or 4 (fp32) channels, 2 or 1
#define HLA_CONV_WIDTH(FN, T, V, P) ((P).silu ? FN<T, V, true>(P, s) : FN<T, V, false>(P, s))
#define HLA_CONV_DISPATCH(FN, P, V16)                                  \
    if ((P).dt == HLA_BF16) {                                          \
        if (wide(P, 2, V16)) return HLA_CONV_WIDTH(FN, __nv_bfloat16, V16, P); \
        if (wide(P, 2, 2)) return HLA_CONV_WIDTH(FN, __nv_bfloat16, 2, P);     \
        return HLA_CONV_WIDTH(FN, __nv_bfloat16, 1, P);                \
    }                                                                  \
    if (wide(P, 4, 4)) return HLA_CONV_WIDTH(FN, float, 4, P);         \
    if (wide(P, 4, 2)) return HLA_CONV_WIDTH(FN, float, 2, P);         \
    return HLA_CONV_WIDTH(FN, float, 1, P);

cudaError_t conv_forward_launch(const Conv &p, cudaStream_t s) { HLA_CONV_DISPATCH(forward_as, p, 8) }
cudaError_t conv_step_launch(const Conv &p, cudaStream_t s) { HLA_CONV_DISPATCH(step_as, p, 8) }
cudaError_t conv_backward_launch(const ConvBwd &p, cudaStream_t s) { HLA_CONV_DISPATCH(backward_as, p, 4) }

}  // namespace hla
