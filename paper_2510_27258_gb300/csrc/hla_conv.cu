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
// and W - 1 rows a strip are read twice (from L2).  A ring of kAhead rows is in flight.
#include <type_traits>

#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kThreads = 256, kStrips = kThreads / 32;
constexpr int kAhead = 4;  // rows a thread has in flight; strip lengths are multiples of it

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

// sigmoid(v[i]) for V values: exp(-v) is kept below 2^63 (v above -43.6, where v sigmoid(v) has come
// down to 5e-18), so that two values can share one reciprocal (the multi-function unit is what they
// wait for).  v itself is replaced by the kept value; NaN stays NaN.
template <int V>
__device__ __forceinline__ void sigmoids(float (&v)[V], float (&s)[V]) {
    float a[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(v[i]) : "f"(v[i]), "f"(-43.6f));
        a[i] = 1.f + __expf(-v[i]);
    }
#pragma unroll
    for (int i = 0; i + 1 < V; i += 2) {
        const float r = __fdividef(1.f, a[i] * a[i + 1]);
        s[i] = r * a[i + 1];
        s[i + 1] = r * a[i];
    }
    if (V % 2) s[V - 1] = __fdividef(1.f, a[V - 1]);
}

// w[c0 .. c0 + V - 1][W] and bias[c0 ..] as fp32
template <typename T, int W, int V>
__device__ __forceinline__ void load_taps(const T *w, const T *bias, int c0, float (&wr)[V][W], float (&br)[V]) {
    float flat[W][V];  // V W consecutive elements
#pragma unroll
    for (int i = 0; i < W; ++i) VecIo<T, V>::load(w + (size_t)c0 * W + i * V, flat[i]);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) wr[v][j] = flat[(v * W + j) / V][(v * W + j) % V];
#pragma unroll
    for (int v = 0; v < V; ++v) br[v] = 0.f;
    if (bias) VecIo<T, V>::load(bias + c0, br);
}

// row t of x (t >= 0), of the state (-(W-1) <= t < 0), or zero
template <typename T, int W, int V>
__device__ __forceinline__ void load_row(const T *x, size_t stride, const T *state, int C, int c0, int t, float (&r)[V]) {
    if (t >= 0) {
        VecIo<T, V>::load(x + (size_t)t * stride + c0, r);
    } else if (state) {
        VecIo<T, V>::load(state + (size_t)(t + W - 1) * C + c0, r);
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) r[v] = 0.f;
    }
}

template <typename T, int W, int V, bool kSilu>
__global__ void __launch_bounds__(kThreads)
conv_forward_kernel(Geom g, const T *__restrict__ x, const T *__restrict__ w, const T *__restrict__ bias,
                    T *__restrict__ out, size_t xs, size_t os, const int *__restrict__ lengths, const T *state_in,
                    T *state_out) {
    const Place at = place<V>(g);
    if (at.c0 >= g.C) return;
    const int len = length_of(lengths, at.b, g.n);
    x += (size_t)at.b * g.n * xs;
    out += (size_t)at.b * g.n * os + at.c0;
    const T *st = state_in ? state_in + (size_t)at.b * (W - 1) * g.C : nullptr;
    const int end = min(at.t0 + g.L, g.n), live = min(end, len);
    if (at.t0 < live) {
        float wr[V][W], br[V], win[W][V];  // row t of x in win[t % W] (counted from the strip's start)
        const T *src = x + (size_t)at.t0 * xs + at.c0;
        Raw<T, V> ring[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            ring[u] = at.t0 + u < live ? raw_load<T, V>(src + (size_t)u * xs) : raw_zero<T, V>();
        load_taps<T, W, V>(w, bias, at.c0, wr, br);
#pragma unroll
        for (int i = 1; i < W; ++i) load_row<T, W, V>(x, xs, st, g.C, at.c0, at.t0 - W + i, win[i]);
        // unrolled over a common multiple of the window's and the ring's turns
        constexpr int kTurn = W == 3 ? 3 * kAhead : kAhead;
        T *dst = out + (size_t)at.t0 * os;
        for (int t = at.t0; t < live; t += kTurn) {
#pragma unroll
            for (int u = 0; u < kTurn; ++u) {
                if (t + u < live) {
                    raw_floats(ring[u % kAhead], win[u % W]);
                    if (t + u + kAhead < live) ring[u % kAhead] = raw_load<T, V>(src + (size_t)kAhead * xs);
                    src += xs;
                    float y[V], s[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float a = br[v];
#pragma unroll
                        for (int j = 0; j < W; ++j) a = fmaf(wr[v][j], win[(u + 1 + j) % W][v], a);
                        y[v] = a;
                    }
                    if (kSilu) {
                        sigmoids<V>(y, s);
#pragma unroll
                        for (int v = 0; v < V; ++v) y[v] *= s[v];
                    }
                    VecIo<T, V>::store(dst, y);
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
        float r[W - 1][V];
#pragma unroll
        for (int i = 0; i < W - 1; ++i) load_row<T, W, V>(x, xs, st, g.C, at.c0, len - (W - 1) + i, r[i]);
#pragma unroll
        for (int i = 0; i < W - 1; ++i)
            VecIo<T, V>::store(state_out + ((size_t)at.b * (W - 1) + i) * g.C + at.c0, r[i]);
    }
}

// one token a sequence: out = act(bias + taps . [state, x]), the state shifted by one row in place
template <typename T, int W, int V, bool kSilu>
__global__ void __launch_bounds__(kThreads)
conv_step_kernel(long long units, int C, const T *x, const T *__restrict__ w, const T *__restrict__ bias, T *out,
                 size_t xs, size_t os, T *__restrict__ state) {
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (i >= units) return;
    const int per = C / V, c0 = (int)(i % per) * V;
    const size_t b = i / per;
    float wr[V][W], br[V], win[W][V], y[V];
    T *st = state + b * (W - 1) * C + c0;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) VecIo<T, V>::load(st + (size_t)j * C, win[j]);
    VecIo<T, V>::load(x + b * xs + c0, win[W - 1]);
    load_taps<T, W, V>(w, bias, c0, wr, br);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float a = br[v];
#pragma unroll
        for (int j = 0; j < W; ++j) a = fmaf(wr[v][j], win[j][v], a);
        y[v] = a;
    }
    if (kSilu) {
        float s[V];
        sigmoids<V>(y, s);
#pragma unroll
        for (int v = 0; v < V; ++v) y[v] *= s[v];
    }
    VecIo<T, V>::store(out + b * os + c0, y);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) VecIo<T, V>::store(st + (size_t)j * C, win[j + 1]);
}

// Gradients.  A strip computes g for its tokens and the W - 1 that follow (which its dx needs), sums
// dw and dbias over its own tokens in registers, then over the block's strips in shared memory, and
// writes one partial [W + 1][C] a token block; conv_sum_kernel adds the partials in a fixed order, so
// equal inputs give equal bits.
template <typename T, int W, int V, bool kSilu>
__global__ void __launch_bounds__(kThreads)
conv_backward_kernel(Geom g, const T *__restrict__ x, const T *__restrict__ w, const T *__restrict__ bias,
                     const T *__restrict__ dout, T *__restrict__ dx, size_t xs, size_t gs, size_t ds,
                     const int *__restrict__ lengths, float *__restrict__ partial) {
    __shared__ float red[kStrips][W + 1][V][32];
    const Place at = place<V>(g);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float dw[W + 1][V] = {};  // row W: dbias
    if (at.c0 < g.C) {
        const int len = length_of(lengths, at.b, g.n);
        x += (size_t)at.b * g.n * xs + at.c0;
        dout += (size_t)at.b * g.n * gs + at.c0;
        dx += (size_t)at.b * g.n * ds + at.c0;
        const int end = min(at.t0 + g.L, g.n), live = min(end, len);
        if (at.t0 < live) {
            // rows t of x and g in xw[t % W], gw[t % W] (counted from the strip's start)
            float wr[V][W], br[V], xw[W][V], gw[W][V];
            const int last = min(live + W - 1, len);  // tokens from here on have g = 0
            Raw<T, V> xr[kAhead], gr[kAhead];
            const T *xp = x + (size_t)at.t0 * xs, *gp = dout + (size_t)at.t0 * gs;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                xr[u] = at.t0 + u < last ? raw_load<T, V>(xp + (size_t)u * xs) : raw_zero<T, V>();
                gr[u] = at.t0 + u < last ? raw_load<T, V>(gp + (size_t)u * gs) : raw_zero<T, V>();
            }
            load_taps<T, W, V>(w, bias, at.c0, wr, br);
#pragma unroll
            for (int i = 0; i < W; ++i) {
#pragma unroll
                for (int v = 0; v < V; ++v) xw[i][v] = gw[i][v] = 0.f;
                if (i > 0 && at.t0 - W + i >= 0) VecIo<T, V>::load(x + (ptrdiff_t)(at.t0 - W + i) * (ptrdiff_t)xs, xw[i]);
            }
            constexpr int kTurn = W == 3 ? 3 * kAhead : kAhead;
            T *to = dx + (size_t)at.t0 * ds;  // of token t + u - (W - 1), once its g and the next W - 1 are there
            for (int t = at.t0; t < live + W - 1; t += kTurn) {
#pragma unroll
                for (int u = 0; u < kTurn; ++u) {
                    const int tt = t + u;
                    if (tt < live + W - 1) {
                        float(&xc)[V] = xw[u % W];
                        float(&gc)[V] = gw[u % W];
                        raw_floats(xr[u % kAhead], xc);
                        raw_floats(gr[u % kAhead], gc);
                        if (tt + kAhead < last) {
                            xr[u % kAhead] = raw_load<T, V>(xp + (size_t)kAhead * xs);
                            gr[u % kAhead] = raw_load<T, V>(gp + (size_t)kAhead * gs);
                        } else {
                            xr[u % kAhead] = gr[u % kAhead] = raw_zero<T, V>();
                        }
                        xp += xs;
                        gp += gs;
                        if (kSilu) {
                            float a[V], s[V];
#pragma unroll
                            for (int v = 0; v < V; ++v) {
                                a[v] = br[v];
#pragma unroll
                                for (int j = 0; j < W; ++j) a[v] = fmaf(wr[v][j], xw[(u + 1 + j) % W][v], a[v]);
                            }
                            sigmoids<V>(a, s);
#pragma unroll
                            for (int v = 0; v < V; ++v) gc[v] *= s[v] * fmaf(a[v], 1.f - s[v], 1.f);
                        }
                        if (tt >= len) {  // (silu' of a row that was not read may be anything)
#pragma unroll
                            for (int v = 0; v < V; ++v) gc[v] = 0.f;
                        }
                        if (tt < live) {
#pragma unroll
                            for (int v = 0; v < V; ++v) {
#pragma unroll
                                for (int j = 0; j < W; ++j) dw[j][v] = fmaf(gc[v], xw[(u + 1 + j) % W][v], dw[j][v]);
                                dw[W][v] += gc[v];
                            }
                        }
                        if (tt - (W - 1) >= at.t0) {
                            float d[V];
#pragma unroll
                            for (int v = 0; v < V; ++v) {
                                float a = 0.f;
#pragma unroll
                                for (int j = 0; j < W; ++j) a = fmaf(wr[v][j], gw[(u + W - j) % W][v], a);
                                d[v] = a;
                            }
                            VecIo<T, V>::store(to, d);
                            to += ds;
                        }
                    }
                }
            }
        }
        const float zero[V] = {};
        for (int t = max(at.t0, live); t < end; ++t) VecIo<T, V>::store(dx + (size_t)t * ds, zero);
    }
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) red[warp][j][v][lane] = dw[j][v];
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

// dw[c][j] and dbias[c] from `rows` partials [W + 1][C]: 32 entries a block, 8 groups of rows
template <int W>
__global__ void __launch_bounds__(kThreads)
conv_sum_kernel(const float *__restrict__ partial, int rows, int C, float *__restrict__ dw, float *__restrict__ dbias,
                WsHeader *header) {
    __shared__ float red[kStrips][32];
    if (blockIdx.x == 0 && threadIdx.x == 0) *header = WsHeader{};  // no device-side waits here: never an error
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    const size_t width = (size_t)(W + 1) * C;
    float s = 0.f;
    if (i < (int)width)
#pragma unroll 8
        for (int r = group; r < rows; r += kStrips) s += partial[(size_t)r * width + i];
    red[group][lane] = s;
    __syncthreads();
    if (group || i >= (int)width) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < kStrips; ++k) s += red[k][lane];
    const int j = i / C, c = i % C;
    if (j < W)
        dw[(size_t)c * W + j] = s;
    else if (dbias)
        dbias[c] = s;
}

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// Strip length: 32 tokens where that still gives every SM eight blocks, else shorter (a strip
// re-reads W - 1 rows, 9 % of a 32-token strip, and shorter strips give more threads).
Geom geometry(int B, int n, int C, int V) {
    Geom g{B, n, C, 32, ceil_div(C, 32 * V), 1};
    while (g.L > kAhead && (long long)B * g.cblocks * ceil_div(n, g.L * kStrips) < 152 * 8) g.L /= 2;
    g.tblocks = n > 0 ? ceil_div(n, g.L * kStrips) : 1;
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
        conv_forward_kernel<T, W(), V, kSilu><<<blocks, kThreads, 0, s>>>(
            g, (const T *)p.x, (const T *)p.w, (const T *)p.bias, (T *)p.out, p.x_stride, p.out_stride, p.lengths,
            (const T *)p.state_in, (T *)p.state_out);
        return cudaGetLastError();
    });
}

template <typename T, int V, bool kSilu>
cudaError_t step_as(const Conv &p, cudaStream_t s) {
    return by_width(p.width, [&](auto W) -> cudaError_t {
        const long long units = (long long)p.B * (p.C / V);
        conv_step_kernel<T, W(), V, kSilu><<<ceil_div(units, kThreads), kThreads, 0, s>>>(
            units, p.C, (const T *)p.x, (const T *)p.w, (const T *)p.bias, (T *)p.out, p.x_stride, p.out_stride,
            (T *)p.state_out);
        return cudaGetLastError();
    });
}

template <typename T, int V, bool kSilu>
cudaError_t backward_as(const ConvBwd &p, cudaStream_t s) {
    return by_width(p.width, [&](auto W) -> cudaError_t {
        const Geom g = geometry(p.B, p.n, p.C, V);
        const int rows = g.tblocks * p.B;
        conv_backward_kernel<T, W(), V, kSilu><<<(unsigned)g.cblocks * rows, kThreads, 0, s>>>(
            g, (const T *)p.x, (const T *)p.w, (const T *)p.bias, (const T *)p.dout, (T *)p.dx, p.x_stride,
            p.dout_stride, p.dx_stride, p.lengths, p.partial);
        cudaError_t e = cudaGetLastError();
        if (e) return e;
        conv_sum_kernel<W()><<<ceil_div((long long)(W() + 1) * p.C, 32), kThreads, 0, s>>>(p.partial, rows, p.C, p.dw,
                                                                                        p.dbias, p.header);
        return cudaGetLastError();
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

// fewer token blocks than this for any V: the scalar variant has the most channel blocks, hence
// the longest strips; the shortest strips (kAhead tokens) bound the number of partial rows
size_t conv_backward_partial_floats(int B, int n, int C, int width) {
    size_t rows = 0;
    for (int V : {1, 4}) {
        const Geom g = geometry(B, n, C, V);
        const size_t r = (size_t)g.tblocks * B;
        if (r > rows) rows = r;
    }
    return rows * (width + 1) * C;
}

#define HLA_CONV_DISPATCH(FN, P, V16)                                                      \
    if ((P).dt == HLA_BF16) {                                                              \
        if (wide(P, 2, V16))                                                               \
            return (P).silu ? FN<__nv_bfloat16, V16, true>(P, s) : FN<__nv_bfloat16, V16, false>(P, s); \
        return (P).silu ? FN<__nv_bfloat16, 1, true>(P, s) : FN<__nv_bfloat16, 1, false>(P, s); \
    }                                                                                      \
    if (wide(P, 4, 4)) return (P).silu ? FN<float, 4, true>(P, s) : FN<float, 4, false>(P, s); \
    return (P).silu ? FN<float, 1, true>(P, s) : FN<float, 1, false>(P, s);

cudaError_t conv_forward_launch(const Conv &p, cudaStream_t s) { HLA_CONV_DISPATCH(forward_as, p, 8) }
cudaError_t conv_step_launch(const Conv &p, cudaStream_t s) { HLA_CONV_DISPATCH(step_as, p, 8) }
cudaError_t conv_backward_launch(const ConvBwd &p, cudaStream_t s) { HLA_CONV_DISPATCH(backward_as, p, 4) }

}  // namespace hla
