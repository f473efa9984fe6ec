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
// A few operations a value: bound by memory traffic (the gradient by latency: its 92 registers let 20 warps
// reside on an SM, with issue slots 54 % and DRAM 51 % busy).  A row of d
// components belongs to d / 8 neighbouring lanes.  A lane holds both members of its four pairs (two
// runs of four components, half a rotation apart; eight consecutive ones if interleaved), so the
// rotation needs no other lane, keeps its products of cosines, sines and weights in registers, and
// walks through the heads of its token with the next heads' rows in flight.  Statistics and products
// are fp32; each output is rounded once.
//
// Measured on a GB300: forward, B8 n2048 H16 Hk16 d64 bf16, 24.4 us a pass (5.5 TB/s), gradient with
// Hk4, 33.5 us (4.5 TB/s).
#include <type_traits>

#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kThreads = 128;
constexpr int kAhead = 4, kAheadBwd = 4;       // rows a thread has in flight
// blocks of an SM at a time (forward with 8, whose 64 registers spill more for fp32: 29.9 instead of 25.6 us for
// B4 n2048 H16 d64 fp32; with 6 29.6 instead of 24.2 us for the bf16 case above)
constexpr int kBlocksFwd = 7, kBlocksBwd = 5;

// four elements at p: one access, or element by element where rows are not aligned to it
template <typename T, bool kVec>
__device__ __forceinline__ Raw<T, 4> load4(const T *p) {
    if (kVec) return raw_load<T, 4>(p);
    Raw<T, 4> r;
    T *e = reinterpret_cast<T *>(&r);
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = p[i];
    return r;
}

template <typename T, bool kVec>
__device__ __forceinline__ void store4(T *p, uint64_t a, uint64_t b) {
    if (kVec) {
        const uint64_t f[2] = {a, b};
        store_pairs<T, 4>(p, f);
    } else {
        float v[4];
        unpair(a, v[0], v[1]);
        unpair(b, v[2], v[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) from_f32(p + i, v[i]);
    }
}

template <int W>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// a lane's eight components: runs of four from at[0] and at[1]
struct Runs {
    int at[2];
};

template <int D, bool kInter>
__device__ __forceinline__ Runs runs_of(int sub, int rot) {
    if (kInter) return {{8 * sub, 8 * sub + 4}};
    // pairs i < rot / 2 turn with i + rot / 2; what is not rotated is paired alike
    const int half = rot / 2, i = 4 * sub;
    if (i < half) return {{i, i + half}};
    return {{half + i, half + i + (D - rot) / 2}};
}

// the pairs of two runs
template <typename T>
__device__ __forceinline__ void pairs_of(const Raw<T, 4> (&r)[2], uint64_t (&v)[4]) {
    uint64_t f[2];
    to_pairs(r[0], f);
    v[0] = f[0]; v[1] = f[1];
    to_pairs(r[1], f);
    v[2] = f[0]; v[3] = f[1];
}

template <typename T, bool kVec>
struct Row {
    Raw<T, 4> r[2];
    __device__ __forceinline__ void load(const T *p, const Runs &at) {
        r[0] = load4<T, kVec>(p + at.at[0]);
        r[1] = load4<T, kVec>(p + at.at[1]);
    }
    __device__ __forceinline__ void pairs(uint64_t (&v)[4]) const { pairs_of<T>(r, v); }
};

// the other members of the pairs a lane holds
template <bool kInter>
__device__ __forceinline__ void mates(const uint64_t (&v)[4], uint64_t (&m)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (kInter) {
            float a, b;
            unpair(v[e], a, b);
            m[e] = pair(b, a);
        } else {
            m[e] = v[e ^ 2];
        }
    }
}

// this lane's cosines and signed sines at table row `pos`: minus the sine for a pair's first member
template <bool kInter>
__device__ __forceinline__ void load_turn(const QkNorm &p, const Runs &at, long long pos, float (&c)[8], float (&s)[8]) {
#pragma unroll
    for (int v = 0; v < 8; ++v) {
        c[v] = 1.f;
        s[v] = 0.f;
    }
    if (at.at[0] >= p.rot) return;
    if (pos < 0 || pos >= p.table_rows) {  // no such row: the rotated part becomes NaN
#pragma unroll
        for (int v = 0; v < 8; ++v) c[v] = s[v] = __int_as_float(0x7fffffff);
        return;
    }
    const size_t from = (size_t)pos * (p.rot / 2) + (kInter ? at.at[0] / 2 : at.at[0]);
    const float4 cu = *reinterpret_cast<const float4 *>(p.cos + from);
    const float4 su = *reinterpret_cast<const float4 *>(p.sin + from);
    const float cv[4] = {cu.x, cu.y, cu.z, cu.w}, sv[4] = {su.x, su.y, su.z, su.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int first = kInter ? 2 * i : i, second = kInter ? 2 * i + 1 : i + 4;
        c[first] = c[second] = cv[i];
        s[first] = -sv[i];
        s[second] = sv[i];
    }
}

template <typename T>
__device__ __forceinline__ void load_weight(const void *w, const Runs &at, float (&r)[8]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const T *p = static_cast<const T *>(w) + at.at[k];
        float f[4] = {1.f, 1.f, 1.f, 1.f};
        if (w && reinterpret_cast<uintptr_t>(w) % sizeof(Raw<T, 4>) == 0) {
            VecIo<T, 4>::load(p, f);
        } else if (w) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = to_f32(p[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) r[4 * k + i] = f[i];
    }
}

struct Split {
    int hpb;  // input heads a block walks through (blockIdx.y picks them)
};

template <typename T, int D, bool kInter, bool kVec>
__global__ void __launch_bounds__(kThreads, kBlocksFwd) qk_norm_forward_kernel(QkNorm p, Split sp) {
    constexpr int kLanes = D / 8, kRows = kThreads / kLanes;
    let_next_begin();
    after_previous();
    const Runs at = runs_of<D, kInter>(threadIdx.x % kLanes, p.rot);
    const unsigned row = blockIdx.x * kRows + threadIdx.x / kLanes, rows = (unsigned)p.B * p.n;  // below 2^31
    // rows past the end repeat the last one without storing: every lane joins the shuffles
    const unsigned r0 = row < rows ? row : rows - 1;
    const unsigned b = r0 / p.n, t = r0 - b * p.n;
    const int h_lo = blockIdx.y * sp.hpb, h_hi = min(h_lo + sp.hpb, p.H + p.Hk);
    float c[8], s[8];
    load_turn<kInter>(p, at, p.positions ? (long long)p.positions[r0] : (long long)p.pos0 + t, c, s);

    auto walk = [&](const T *x, T *out, const void *weight, int lo, int hi, int per) {
        if (lo >= hi) return;
        x += (size_t)lo * D;
        Row<T, kVec> ring[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) ring[u].load(x + (lo + u < hi ? u : 0) * D, at);
        // the rotation with the weights in it: out_i = r (v_i wc_i + v_p(i) ws_i)
        uint64_t wc[4], ws[4];
        {
            float w[8];
            load_weight<T>(weight, at, w);
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const int m0 = kInter ? e + 1 : e ^ 4, m1 = kInter ? e : (e + 1) ^ 4;
                wc[e / 2] = pair(w[e] * c[e], w[e + 1] * c[e + 1]);
                ws[e / 2] = pair(w[m0] * s[e], w[m1] * s[e + 1]);
            }
        }
        const bool turned = at.at[0] < p.rot;
        const size_t step = (size_t)p.n * D;
        T *to = out + (((size_t)b * p.H + (size_t)lo * per) * p.n + t) * D;
        int left = hi - lo;
        while (left > 0) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (left <= 0) break;
                uint64_t v[4], m[4];
                ring[u].pairs(v);
                if (left > kAhead) ring[u].load(x + (u + kAhead) * D, at);
                mates<kInter>(v, m);
                uint64_t sum = mul2(v[0], v[0]);
#pragma unroll
                for (int e = 1; e < 4; ++e) sum = fma2(v[e], v[e], sum);
                float s0, s1;
                unpair(sum, s0, s1);
                const float r = rsqrtf(row_sum<kLanes>(s0 + s1) * (1.f / D) + p.eps);
                const uint64_t r2 = pair(r, r);
                uint64_t y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = mul2(v[e], wc[e]);
                    if (turned) y[e] = fma2(m[e], ws[e], y[e]);
                    y[e] = mul2(y[e], r2);
                }
                for (int k = 0; k < per; ++k) {
                    if (row < rows) {
                        store4<T, true>(to + at.at[0], y[0], y[1]);
                        store4<T, true>(to + at.at[1], y[2], y[3]);
                    }
                    to += step;
                }
                --left;
            }
            x += kAhead * D;
        }
    };
    walk(static_cast<const T *>(p.q) + (size_t)r0 * p.q_stride, static_cast<T *>(p.q_out), p.wq, h_lo,
         min(h_hi, p.H), 1);
    walk(static_cast<const T *>(p.k) + (size_t)r0 * p.k_stride, static_cast<T *>(p.k_out), p.wk, max(h_lo - p.H, 0),
         h_hi - p.H, p.H / p.Hk);
}

// Gradients.  Weight gradients are summed over a thread's heads in registers, over the block's
// rows in shared memory, and over blocks by qk_norm_sum_kernel in a fixed order.
template <typename T, int D, bool kInter, bool kVec>
__global__ void __launch_bounds__(kThreads, kBlocksBwd) qk_norm_backward_kernel(QkNormBwd p, Split sp) {
    constexpr int kLanes = D / 8, kRows = kThreads / kLanes;
    union Scratch {
        Raw<T, 4> ring[2][kAheadBwd][kThreads][2];  // rows of dout, rows of x
        float red[kRows][D];
    };
    __shared__ Scratch sm;
    let_next_begin();
    after_previous();
    auto &ring = sm.ring;
    auto &red = sm.red;
    const QkNorm &f = p.f;
    const Runs at = runs_of<D, kInter>(threadIdx.x % kLanes, f.rot);
    const unsigned row = blockIdx.x * kRows + threadIdx.x / kLanes, rows = (unsigned)f.B * f.n;  // below 2^31
    const unsigned r0 = row < rows ? row : rows - 1;
    const bool real = row < rows;
    const unsigned b = r0 / f.n, t = r0 - b * f.n;
    const int h_lo = blockIdx.y * sp.hpb, h_hi = min(h_lo + sp.hpb, f.H + f.Hk);
    uint64_t c2[4], s2[4];  // cosines, and the negated signed sines
    {
        float c[8], s[8];
        load_turn<kInter>(f, at, f.positions ? (long long)f.positions[r0] : (long long)f.pos0 + t, c, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c2[e] = pair(c[2 * e], c[2 * e + 1]);
            s2[e] = pair(-s[2 * e], -s[2 * e + 1]);
        }
    }
    const bool turned = at.at[0] < f.rot;

    auto walk = [&](const T *x, const T *dout, T *dx, const void *weight, int lo, int hi, int per, uint64_t (&dw)[4]) {
        if (lo >= hi) return;
        uint64_t w2[4];
        {
            float w[8];
            load_weight<T>(weight, at, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) w2[e] = pair(w[2 * e], w[2 * e + 1]);
        }
        const size_t step = (size_t)f.n * D;
        x += (size_t)lo * D;
        dx += (size_t)lo * D;
        const T *src = dout + (((size_t)b * f.H + (size_t)lo * per) * f.n + t) * D;
        // the rows of dout in their order (a head's `per` rows are neighbours), and a head's row of x with
        // its first one
        const int count = (hi - lo) * per;
        int sent = 0, h_sent = 0, k_sent = 0;  // rows of dout sent for; the next one's head and place in it
        const T *x_next = x, *g_next = src;
        auto send = [&]() {
            if (sent < count) {
                Raw<T, 4> *slot = ring[0][sent % kAheadBwd][threadIdx.x];
                ring_copy<T, 4>(slot, g_next + at.at[0], true);
                ring_copy<T, 4>(slot + 1, g_next + at.at[1], true);
                g_next += step;
                if (k_sent == 0) {
                    slot = ring[1][h_sent % kAheadBwd][threadIdx.x];
                    if (kVec) {
                        ring_copy<T, 4>(slot, x_next + at.at[0], true);
                        ring_copy<T, 4>(slot + 1, x_next + at.at[1], true);
                    } else {
                        slot[0] = load4<T, false>(x_next + at.at[0]);
                        slot[1] = load4<T, false>(x_next + at.at[1]);
                    }
                    x_next += D;
                }
                if (++k_sent == per) {
                    k_sent = 0;
                    ++h_sent;
                }
                ++sent;
            }
            ring_commit();
        };
#pragma unroll
        for (int u = 0; u < kAheadBwd; ++u) send();
        for (int h = 0, i = 0; h < hi - lo; ++h) {
            {
                uint64_t v[4], g[4], m[4];
                for (int k = 0; k < per; ++k, ++i) {
                    ring_wait<kAheadBwd - 1>();
                    if (k == 0) pairs_of<T>(ring[1][h % kAheadBwd][threadIdx.x], v);
                    if (k == 0) {
                        pairs_of<T>(ring[0][i % kAheadBwd][threadIdx.x], g);
                    } else {
                        uint64_t more[4];
                        pairs_of<T>(ring[0][i % kAheadBwd][threadIdx.x], more);
#pragma unroll
                        for (int e = 0; e < 4; ++e) g[e] = add2(g[e], more[e]);
                    }
                    send();
                }
                mates<kInter>(g, m);
                uint64_t ss2 = pair(0.f, 0.f), dot2 = ss2;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint64_t dy = mul2(g[e], c2[e]);
                    if (turned) dy = fma2(m[e], s2[e], dy);
                    ss2 = fma2(v[e], v[e], ss2);
                    dot2 = fma2(mul2(dy, w2[e]), v[e], dot2);
                    g[e] = dy;
                }
                float ss, dot, more;
                unpair(ss2, ss, more);
                ss = row_sum<kLanes>(ss + more);
                unpair(dot2, dot, more);
                dot = row_sum<kLanes>(dot + more);
                const float r = rsqrtf(ss * (1.f / D) + f.eps);
                const float q = -dot * r * r * (1.f / D);  // dx = r (dy w + v q)
                const uint64_t r2 = pair(r, r), q2 = pair(q, q);
                uint64_t d[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    d[e] = mul2(r2, fma2(v[e], q2, mul2(g[e], w2[e])));
                    if (real) dw[e] = fma2(g[e], mul2(v[e], r2), dw[e]);
                }
                if (real) {
                    store4<T, kVec>(dx + at.at[0], d[0], d[1]);
                    store4<T, kVec>(dx + at.at[1], d[2], d[3]);
                }
                dx += D;
            }
        }
    };
    uint64_t dwq[4] = {}, dwk[4] = {};
    walk(static_cast<const T *>(f.q) + (size_t)r0 * f.q_stride, static_cast<const T *>(p.dq_out),
         static_cast<T *>(p.dq) + (size_t)r0 * p.dq_stride, f.wq, h_lo, min(h_hi, f.H), 1, dwq);
    walk(static_cast<const T *>(f.k) + (size_t)r0 * f.k_stride, static_cast<const T *>(p.dk_out),
         static_cast<T *>(p.dk) + (size_t)r0 * p.dk_stride, f.wk, max(h_lo - f.H, 0), h_hi - f.H, f.H / f.Hk, dwk);
    float *to = p.partial + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * D;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        float *mine = red[threadIdx.x / kLanes];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = at.at[e / 2] + 2 * (e % 2);
            unpair(which ? dwk[e] : dwq[e], mine[i], mine[i + 1]);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < D; i += kThreads) {
            float sum = 0.f;
#pragma unroll 8
            for (int k = 0; k < kRows; ++k) sum += red[k][i];
            to[which * D + i] = sum;
        }
    }
}

// dwq and dwk from `rows` partials [2][d]: 32 entries a block, four a thread, every 128th row
constexpr int kSumThreads = 1024, kSumGroups = kSumThreads / 8;

__global__ void __launch_bounds__(kSumThreads)
qk_norm_sum_kernel(const float *partial, int rows, int d, float *dwq, float *dwk, WsHeader *header) {
    __shared__ float red[32][kSumGroups + 1];
    let_next_begin();
    after_previous();
    if (blockIdx.x == 0 && threadIdx.x == 0) *header = WsHeader{};  // no device-side waits here: never an error
    const int quad = threadIdx.x & 7, group = threadIdx.x >> 3;  // (2 d is a multiple of 32)
    const float *from = partial + blockIdx.x * 32 + quad * 4;
    float s[4] = {};
#pragma unroll 8
    for (int r = group; r < rows; r += kSumGroups) {
        const float4 v = *reinterpret_cast<const float4 *>(from + (size_t)r * 2 * d);
        s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) red[quad * 4 + i][group] = s[i];
    __syncthreads();
    // warp w: entry w of the block
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, e = blockIdx.x * 32 + w;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kSumGroups; k += 32) sum += red[w][k + lane];
    sum = row_sum<32>(sum);
    float *to = e < d ? dwq : dwk;
    if (lane == 0 && to) to[e < d ? e : e - d] = sum;
}

struct Plan {
    unsigned gx, gy;
    Split sp;
};

// The split of the heads over blocks that ends first: the blocks of the fullest SM (at least half of
// what is resident, below which they gain nothing from one another's absence), each costing its heads
// and about four heads' time more (tables, weights, first loads)
Plan plan(long long rows, int heads, int per_block, int resident) {
    Plan best{};
    long long least = 0;
    const unsigned gx = (unsigned)((rows + per_block - 1) / per_block);
    for (int groups = 1; groups <= heads && groups <= 64; ++groups) {
        const int hpb = (heads + groups - 1) / groups, gy = (heads + hpb - 1) / hpb;
        long long blocks = ((long long)gx * gy + 151) / 152;
        if (blocks < resident / 2) blocks = resident / 2;
        if (groups == 1 || blocks * (hpb + 4) < least) {
            least = blocks * (hpb + 4);
            best = {gx, (unsigned)gy, {hpb}};
        }
    }
    return best;
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

template <typename T, bool kInter, bool kVec>
cudaError_t forward_as(const QkNorm &p, cudaStream_t s) {
    return by_size(p.d, [&](auto D) -> cudaError_t {
        const Plan g = plan((long long)p.B * p.n, p.H + p.Hk, kThreads / (D() / 8), kBlocksFwd);
        return launch_after(qk_norm_forward_kernel<T, D(), kInter, kVec>, dim3(g.gx, g.gy), kThreads, 0, s, p, g.sp);
    });
}

template <typename T, bool kInter, bool kVec>
cudaError_t backward_as(const QkNormBwd &p, cudaStream_t s) {
    return by_size(p.f.d, [&](auto D) -> cudaError_t {
        const Plan g = plan((long long)p.f.B * p.f.n, p.f.H + p.f.Hk, kThreads / (D() / 8), kBlocksBwd);
        cudaError_t e = launch_after(qk_norm_backward_kernel<T, D(), kInter, kVec>, dim3(g.gx, g.gy), kThreads, 0, s, p, g.sp);
        if (e) return e;
        return launch_after(qk_norm_sum_kernel, 2 * p.f.d / 32, kSumThreads, 0, s, p.partial, (int)(g.gx * g.gy), p.f.d,
                            p.dwq, p.dwk, p.header);
    });
}

}  // namespace

size_t qk_norm_partial_floats(int B, int n, int H, int Hk, int d) {
    const Plan g = plan((long long)B * n, H + Hk, kThreads / (d / 8), kBlocksBwd);
    return (size_t)g.gx * g.gy * 2 * d;
}

#define HLA_QK_DISPATCH(FN, VEC, INTER, DT)                                                              \
    if ((DT) == HLA_BF16) {                                                                              \
        if (INTER) return (VEC) ? FN<__nv_bfloat16, true, true>(p, s) : FN<__nv_bfloat16, true, false>(p, s); \
        return (VEC) ? FN<__nv_bfloat16, false, true>(p, s) : FN<__nv_bfloat16, false, false>(p, s);     \
    }                                                                                                    \
    if (INTER) return (VEC) ? FN<float, true, true>(p, s) : FN<float, true, false>(p, s);                \
    return (VEC) ? FN<float, false, true>(p, s) : FN<float, false, false>(p, s);

cudaError_t qk_norm_forward_launch(const QkNorm &p, cudaStream_t s) {
    const size_t eb = p.dt == HLA_BF16 ? 2 : 4, by = 4 * eb;
    const bool vec = rows_aligned(p.q, p.q_stride, eb, by) && rows_aligned(p.k, p.k_stride, eb, by);
    HLA_QK_DISPATCH(forward_as, vec, p.interleaved, p.dt)
}

cudaError_t qk_norm_backward_launch(const QkNormBwd &p, cudaStream_t s) {
    const size_t eb = p.f.dt == HLA_BF16 ? 2 : 4, by = 4 * eb;
    const bool vec = rows_aligned(p.f.q, p.f.q_stride, eb, by) && rows_aligned(p.f.k, p.f.k_stride, eb, by) &&
                     rows_aligned(p.dq, p.dq_stride, eb, by) && rows_aligned(p.dk, p.dk_stride, eb, by);
    HLA_QK_DISPATCH(backward_as, vec, p.f.interleaved, p.f.dt)
}

}  // namespace hla
