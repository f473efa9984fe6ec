// Norm of queries and keys for each head with the position rotation, from projection rows
// [B, n, heads, d] to the [B, H, n, d] the HLA kernels read, and its gradients.
//
//   u = x rsqrt(mean(x^2) + eps),  y = u w,  out_i = y_i c_i + y_p(i) s_i
// where p(i) is the partner of component i in the rotated pair (i + rot/2 or i - rot/2, or i ^ 1
// interleaved), c_i its cosine, s_i minus the sine for a pair's first component and plus the sine
// for its second; components at and after rot have c = 1, s = 0.  A key head is written to each of
// the H / Hk query heads that share it.  Backwards, with g the output's gradient (summed over the
// sharing heads):
//   dy_i = g_i c_i - g_p(i) s_i,  dw = sum dy u,  dx = r (dy w - u mean(dy w u)).
//
// A few operations a value: bound by memory traffic.  A row of d components belongs to d / V
// neighbouring lanes (one 16- or 8-byte access each), which hold the token's cosines and sines and
// the weights in registers and walk through the heads, so tables and weights are read once a token
// and block, not once a head.  Statistics and products are fp32; each output is rounded once.
#include <type_traits>

#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4, kAheadBwd = 2;  // heads whose rows a thread has in flight

// V elements at p: one access, or element by element where rows are not aligned to it
template <typename T, int V, bool kVec>
__device__ __forceinline__ void load_row(const T *p, float (&v)[V]) {
    if (kVec) {
        VecIo<T, V>::load(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = to_f32(p[i]);
    }
}

template <typename T, int V, bool kVec>
__device__ __forceinline__ Raw<T, V> load_raw(const T *p) {
    if (kVec) return raw_load<T, V>(p);
    Raw<T, V> r;
    T *e = reinterpret_cast<T *>(&r);
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = p[i];
    return r;
}

// the row another lane holds
template <typename R>
__device__ __forceinline__ R raw_from(const R &r, int lane) {
    R got;
    const uint32_t *from = reinterpret_cast<const uint32_t *>(&r);
    uint32_t *to = reinterpret_cast<uint32_t *>(&got);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(R) / 4); ++i) to[i] = __shfl_sync(0xffffffffu, from[i], lane);
    return got;
}

template <typename T, int V, bool kVec>
__device__ __forceinline__ void store_row(T *p, const float (&v)[V]) {
    if (kVec) {
        VecIo<T, V>::store(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) from_f32(p + i, v[i]);
    }
}

template <int W>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// this thread's cosines and signed sines: components i0 .. i0 + V - 1 at table row `pos`
template <int V>
__device__ __forceinline__ void load_turn(const QkNorm &p, int i0, long long pos, float (&c)[V], float (&s)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = 1.f;
        s[v] = 0.f;
    }
    if (i0 >= p.rot) return;
    if (pos < 0 || pos >= p.table_rows) {  // no such row: the rotated part becomes NaN
#pragma unroll
        for (int v = 0; v < V; ++v) c[v] = s[v] = __int_as_float(0x7fffffff);
        return;
    }
    const int half = p.rot / 2;
    const float *ct = p.cos + pos * half, *st = p.sin + pos * half;
    if (p.interleaved) {
#pragma unroll
        for (int v = 0; v < V; v += 2) {
            c[v] = c[v + 1] = ct[(i0 + v) / 2];
            s[v + 1] = st[(i0 + v) / 2];
            s[v] = -s[v + 1];
        }
    } else {
        const bool first = i0 < half;
        const int j = first ? i0 : i0 - half;
#pragma unroll
        for (int v = 0; v < V; v += 4) {
            const float4 cu = *reinterpret_cast<const float4 *>(ct + j + v);
            const float4 su = *reinterpret_cast<const float4 *>(st + j + v);
            c[v] = cu.x; c[v + 1] = cu.y; c[v + 2] = cu.z; c[v + 3] = cu.w;
            s[v] = first ? -su.x : su.x;
            s[v + 1] = first ? -su.y : su.y;
            s[v + 2] = first ? -su.z : su.z;
            s[v + 3] = first ? -su.w : su.w;
        }
    }
}

template <typename T, int V>
__device__ __forceinline__ void load_weight(const void *w, int i0, float (&r)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) r[v] = w ? to_f32(static_cast<const T *>(w)[i0 + v]) : 1.f;
}

struct Split {
    int hpb;  // input heads a block walks through (blockIdx.y picks them)
};

template <typename T, int D, int V, bool kVec>
__global__ void __launch_bounds__(kThreads) qk_norm_forward_kernel(QkNorm p, Split sp) {
    constexpr int kLanes = D / V, kRows = kThreads / kLanes;
    const int sub = threadIdx.x % kLanes, i0 = sub * V;
    const long long row = (long long)blockIdx.x * kRows + threadIdx.x / kLanes, rows = (long long)p.B * p.n;
    // rows past the end repeat the last one without storing: every lane joins the shuffles
    const long long r0 = row < rows ? row : rows - 1;
    const int b = (int)(r0 / p.n), t = (int)(r0 % p.n);
    float c[V], s[V];
    load_turn<V>(p, i0, p.positions ? (long long)p.positions[r0] : (long long)p.pos0 + t, c, s);
    const int half = p.rot / 2;
    const bool turned = i0 < p.rot, paired = turned && !p.interleaved;
    const int partner = paired ? (i0 < half ? half : -half) : 0;
    const int mate_lane = (int)(threadIdx.x & 31) + partner / V;
    const int h_lo = blockIdx.y * sp.hpb, h_hi = min(h_lo + sp.hpb, p.H + p.Hk);

    auto walk = [&](const T *x, T *out, const void *weight, int lo, int hi, int per) {
        if (lo >= hi) return;
        // the rotation with the weights in it: out_i = r (v_i wc_i + v_p(i) ws_i)
        float wc[V], ws[V];
        load_weight<T, V>(weight, i0, wc);
        load_weight<T, V>(weight, i0 + partner, ws);
        if (turned && p.interleaved) {
#pragma unroll
            for (int e = 0; e < V; ++e) ws[e] = wc[e ^ 1] * s[e];
#pragma unroll
            for (int e = 0; e < V; ++e) wc[e] *= c[e];
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                wc[e] *= c[e];
                ws[e] *= s[e];
            }
        }
        T *to = out + (((size_t)b * p.H + (size_t)lo * per) * p.n + t) * D + i0;
        const size_t step = (size_t)p.n * D;
        Raw<T, V> ring[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            ring[u] = lo + u < hi ? load_raw<T, V, kVec>(x + (size_t)(lo + u) * D + i0) : raw_zero<T, V>();
        for (int h = lo; h < hi; h += kAhead) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (h + u >= hi) break;
                const Raw<T, V> raw = ring[u];
                if (h + u + kAhead < hi) ring[u] = load_raw<T, V, kVec>(x + (size_t)(h + u + kAhead) * D + i0);
                float v[V], m[V];
                raw_floats(raw, v);
                if (p.interleaved) {
#pragma unroll
                    for (int e = 0; e < V; ++e) m[e] = v[e ^ 1];
                } else {
                    raw_floats(raw_from(raw, mate_lane), m);
                }
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) ss = fmaf(v[e], v[e], ss);
                const float r = rsqrtf(row_sum<kLanes>(ss) * (1.f / D) + p.eps);
                float y[V];
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] = r * fmaf(v[e], wc[e], turned ? m[e] * ws[e] : 0.f);
                for (int k = 0; k < per; ++k) {
                    if (row < rows) VecIo<T, V>::store(to, y);
                    to += step;
                }
            }
        }
    };
    walk(static_cast<const T *>(p.q) + (size_t)r0 * p.q_stride, static_cast<T *>(p.q_out), p.wq, h_lo,
         min(h_hi, p.H), 1);
    walk(static_cast<const T *>(p.k) + (size_t)r0 * p.k_stride, static_cast<T *>(p.k_out), p.wk, max(h_lo - p.H, 0),
         h_hi - p.H, p.H / p.Hk);
}

// Gradients.  Weight gradients are summed over a thread's heads in registers, over the block's
// rows in shared memory, and over blocks by qk_norm_sum_kernel in a fixed order.
template <typename T, int D, int V, bool kVec>
__global__ void __launch_bounds__(kThreads) qk_norm_backward_kernel(QkNormBwd p, Split sp) {
    constexpr int kLanes = D / V, kRows = kThreads / kLanes;
    __shared__ float red[kRows][D];
    const QkNorm &f = p.f;
    const int sub = threadIdx.x % kLanes, i0 = sub * V;
    const long long row = (long long)blockIdx.x * kRows + threadIdx.x / kLanes, rows = (long long)f.B * f.n;
    const long long r0 = row < rows ? row : rows - 1;
    const bool real = row < rows;
    const int b = (int)(r0 / f.n), t = (int)(r0 % f.n);
    float c[V], s[V];
    load_turn<V>(f, i0, f.positions ? (long long)f.positions[r0] : (long long)f.pos0 + t, c, s);
    const int half = f.rot / 2;
    const bool turned = i0 < f.rot, paired = turned && !f.interleaved;
    const int mate_lane = (threadIdx.x & 31) + (paired ? (i0 < half ? half : -half) / V : 0);
    const int h_lo = blockIdx.y * sp.hpb, h_hi = min(h_lo + sp.hpb, f.H + f.Hk);

    auto walk = [&](const T *x, const T *dout, T *dx, const void *weight, int lo, int hi, int per, float (&dw)[V]) {
        float w[V];
        load_weight<T, V>(weight, i0, w);
        const size_t step = (size_t)f.n * D;
        const T *src = dout + (((size_t)b * f.H + (size_t)lo * per) * f.n + t) * D + i0;
        Raw<T, V> xr[kAheadBwd], gr[kAheadBwd];
#pragma unroll
        for (int u = 0; u < kAheadBwd; ++u) {
            const bool on = lo + u < hi;
            xr[u] = on ? load_raw<T, V, kVec>(x + (size_t)(lo + u) * D + i0) : raw_zero<T, V>();
            gr[u] = on ? raw_load<T, V>(src + (size_t)u * per * step) : raw_zero<T, V>();
        }
        for (int h0 = lo; h0 < hi; h0 += kAheadBwd) {
#pragma unroll
            for (int u = 0; u < kAheadBwd; ++u) {
                const int h = h0 + u;
                if (h >= hi) break;
                float v[V], g[V];
                raw_floats(xr[u], v);
                raw_floats(gr[u], g);
                for (int m = 1; m < per; ++m) {
                    float more[V];
                    VecIo<T, V>::load(src + (size_t)m * step, more);
#pragma unroll
                    for (int e = 0; e < V; ++e) g[e] += more[e];
                }
                if (h + kAheadBwd < hi) {
                    xr[u] = load_raw<T, V, kVec>(x + (size_t)(h + kAheadBwd) * D + i0);
                    gr[u] = raw_load<T, V>(src + (size_t)kAheadBwd * per * step);
                }
                src += (size_t)per * step;
                float dy[V], ss = 0.f, dot = 0.f;
                float gp[V];
#pragma unroll
                for (int e = 0; e < V; ++e) gp[e] = f.interleaved ? g[e ^ 1] : __shfl_sync(0xffffffffu, g[e], mate_lane);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    dy[e] = fmaf(g[e], c[e], turned ? -gp[e] * s[e] : 0.f);
                    ss = fmaf(v[e], v[e], ss);
                    dot = fmaf(dy[e] * w[e], v[e], dot);
                }
                ss = row_sum<kLanes>(ss);
                dot = row_sum<kLanes>(dot);
                const float r = rsqrtf(ss * (1.f / D) + f.eps);
                const float m = dot * r * (1.f / D);
                float d[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float unit = v[e] * r;
                    d[e] = r * fmaf(dy[e], w[e], -unit * m);
                    if (real) dw[e] = fmaf(dy[e], unit, dw[e]);
                }
                if (real) store_row<T, V, kVec>(dx + (size_t)h * D + i0, d);
            }
        }
    };
    float dwq[V] = {}, dwk[V] = {};
    walk(static_cast<const T *>(f.q) + (size_t)r0 * f.q_stride, static_cast<const T *>(p.dq_out),
         static_cast<T *>(p.dq) + (size_t)r0 * p.dq_stride, f.wq, h_lo, min(h_hi, f.H), 1, dwq);
    walk(static_cast<const T *>(f.k) + (size_t)r0 * f.k_stride, static_cast<const T *>(p.dk_out),
         static_cast<T *>(p.dk) + (size_t)r0 * p.dk_stride, f.wk, max(h_lo - f.H, 0), h_hi - f.H, f.H / f.Hk, dwk);
    float *to = p.partial + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * D;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) red[threadIdx.x / kLanes][i0 + e] = which ? dwk[e] : dwq[e];
        __syncthreads();
        for (int i = threadIdx.x; i < D; i += kThreads) {
            float sum = 0.f;
#pragma unroll 8
            for (int k = 0; k < kRows; ++k) sum += red[k][i];
            to[which * D + i] = sum;
        }
    }
}

// dwq and dwk from `rows` partials [2][d]: one warp an entry
__global__ void __launch_bounds__(kThreads)
qk_norm_sum_kernel(const float *__restrict__ partial, int rows, int d, float *dwq, float *dwk, WsHeader *header) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *header = WsHeader{};  // no device-side waits here: never an error
    const int i = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (i >= 2 * d) return;
    float s = 0.f;
#pragma unroll 8
    for (int r = lane; r < rows; r += 32) s += partial[(size_t)r * 2 * d + i];
    s = row_sum<32>(s);
    float *to = i < d ? dwq : dwk;
    if (lane == 0 && to) to[i < d ? i : i - d] = s;
}

struct Plan {
    unsigned gx, gy;
    Split sp;
};

// All heads in one block where the rows alone give every SM eight blocks (tables and weights are
// then read once a token), else as many head groups as that takes
Plan plan(long long rows, int heads, int per_block) {
    Plan g;
    g.gx = (unsigned)((rows + per_block - 1) / per_block);
    long long groups = (152 * 8 + (long long)g.gx - 1) / g.gx;
    if (groups > heads) groups = heads;
    g.sp.hpb = (int)((heads + groups - 1) / groups);
    g.gy = (unsigned)((heads + g.sp.hpb - 1) / g.sp.hpb);
    return g;
}

template <typename F>
cudaError_t by_size(int d, F f) {
    switch (d) {
        case 16: return f(std::integral_constant<int, 16>());
        case 32: return f(std::integral_constant<int, 32>());
        case 64: return f(std::integral_constant<int, 64>());
        default: return f(std::integral_constant<int, 128>());
    }
}

template <typename T, int V, bool kVec>
cudaError_t forward_as(const QkNorm &p, cudaStream_t s) {
    return by_size(p.d, [&](auto D) -> cudaError_t {
        const Plan g = plan((long long)p.B * p.n, p.H + p.Hk, kThreads / (D() / V));
        qk_norm_forward_kernel<T, D(), V, kVec><<<dim3(g.gx, g.gy), kThreads, 0, s>>>(p, g.sp);
        return cudaGetLastError();
    });
}

template <typename T, int V, bool kVec>
cudaError_t backward_as(const QkNormBwd &p, cudaStream_t s) {
    return by_size(p.f.d, [&](auto D) -> cudaError_t {
        const Plan g = plan((long long)p.f.B * p.f.n, p.f.H + p.f.Hk, kThreads / (D() / V));
        qk_norm_backward_kernel<T, D(), V, kVec><<<dim3(g.gx, g.gy), kThreads, 0, s>>>(p, g.sp);
        cudaError_t e = cudaGetLastError();
        if (e) return e;
        qk_norm_sum_kernel<<<(2 * p.f.d * 32 + kThreads - 1) / kThreads, kThreads, 0, s>>>(
            p.partial, (int)(g.gx * g.gy), p.f.d, p.dwq, p.dwk, p.header);
        return cudaGetLastError();
    });
}

// components a lane holds: 8 bf16 or 4 fp32 (16 bytes); 4 bf16 where the pairs of a half-split
// rotation would not lie whole in other lanes
int lane_width(const QkNorm &p) { return p.dt == HLA_BF16 && (p.interleaved || p.rot % 16 == 0) ? 8 : 4; }

}  // namespace

size_t qk_norm_partial_floats(int B, int n, int H, int Hk, int d) {
    size_t most = 0;
    for (int V : {4, 8}) {
        const Plan g = plan((long long)B * n, H + Hk, kThreads / (d / V));
        const size_t f = (size_t)g.gx * g.gy * 2 * d;
        if (f > most) most = f;
    }
    return most;
}

cudaError_t qk_norm_forward_launch(const QkNorm &p, cudaStream_t s) {
    const int V = lane_width(p);
    const size_t eb = p.dt == HLA_BF16 ? 2 : 4, by = V * eb;
    const bool vec = rows_aligned(p.q, p.q_stride, eb, by) && rows_aligned(p.k, p.k_stride, eb, by);
    if (p.dt == HLA_F32) return vec ? forward_as<float, 4, true>(p, s) : forward_as<float, 4, false>(p, s);
    if (V == 8)
        return vec ? forward_as<__nv_bfloat16, 8, true>(p, s) : forward_as<__nv_bfloat16, 8, false>(p, s);
    return vec ? forward_as<__nv_bfloat16, 4, true>(p, s) : forward_as<__nv_bfloat16, 4, false>(p, s);
}

cudaError_t qk_norm_backward_launch(const QkNormBwd &p, cudaStream_t s) {
    const int V = lane_width(p.f);
    const size_t eb = p.f.dt == HLA_BF16 ? 2 : 4, by = V * eb;
    const bool vec = rows_aligned(p.f.q, p.f.q_stride, eb, by) && rows_aligned(p.f.k, p.f.k_stride, eb, by) &&
                     rows_aligned(p.dq, p.dq_stride, eb, by) && rows_aligned(p.dk, p.dk_stride, eb, by);
    if (p.f.dt == HLA_F32) return vec ? backward_as<float, 4, true>(p, s) : backward_as<float, 4, false>(p, s);
    if (V == 8)
        return vec ? backward_as<__nv_bfloat16, 8, true>(p, s) : backward_as<__nv_bfloat16, 8, false>(p, s);
    return vec ? backward_as<__nv_bfloat16, 4, true>(p, s) : backward_as<__nv_bfloat16, 4, false>(p, s);
}

}  // namespace hla
