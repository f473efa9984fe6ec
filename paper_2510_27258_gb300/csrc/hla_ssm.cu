// Selective state space scan: single tokens, and prompts in fp32 on the CUDA cores.
//
//   delta_t = softplus(raw_t + bias_h) (or raw_t + bias_h),  h_t = exp(a_h delta_t) h_{t-1} + delta_t b_t x_t^T
//   y_t = h_t^T c_t + D_h x_t
// with h an N x P state a head, and b, c shared by the H / G heads of a group.  The recurrence is
// separate for every column of h, so a head's columns can be split over blocks.
//
// Prompts: the serial recurrence itself, 16 columns a block, a column's N states spread over 8
// lanes' registers.  A column costs 3 N multiply-adds a token, so it is bound by issue slots (about
// 70 instructions a warp and token at N = 128) and, with few heads, by the length of the chain; then
// the sequence is cut into segments: every segment but the last is scanned from a zero state first
// (state only), the segments' states are chained, and the scan proper starts each segment from its
// state.  All of it is fp32, with no rounding between the tokens and the outputs.
//
// Measured on a GB300: step, B64 H32 P64 N128, 21.7 us a pass (6.2 TB/s); B3 n517 H6 P32 N16 fp32,
// 14.1 us on the device (two scans of 48 tokens' latency and the chain of 11 segments between them);
// B8 n2048 H32 P64 N128 fp32, 1290 us (3 % of the HBM roofline).
#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kCols = 16, kScanThreads = 128, kLanes = 8, kTok = 16;

__device__ __forceinline__ float softplus(float v) { return fmaxf(v, 0.f) + log1pf(expf(-fabsf(v))); }

__device__ __forceinline__ float step_size(float raw, float bias, int on) {
    const float v = raw + bias;
    return on ? softplus(v) : v;
}

__device__ __forceinline__ int length_of(const Ssm &p, int b) {
    if (!p.lengths) return p.n;
    const int m = p.lengths[b];
    return m < 0 ? 0 : m > p.n ? p.n : m;
}

// State n of a lane's NS states: groups of up to 4 consecutive ones, the lanes side by side
template <int NS>
__device__ __forceinline__ int state_index(int lane8, int i) {
    constexpr int kGroup = NS < 4 ? NS : 4;
    return (i / kGroup) * (kLanes * kGroup) + lane8 * kGroup + i % kGroup;
}

template <typename T, int N, bool kStateOnly>
__global__ void __launch_bounds__(kScanThreads)
scan_kernel(Ssm p, int segments, int seg_len, float *seg_state, float *seg_decay) {
    constexpr int NS = N / kLanes;
    if (kStateOnly || segments == 1) after_previous();
    let_next_begin();
    __shared__ __align__(16) float bs[kTok][N], cs[kTok][N];
    __shared__ float xs[kTok][kCols], ys[kTok][kCols], decay[kTok], dl[kTok], la_sum;
    const int slices = p.P / kCols;
    const int slice = blockIdx.x % slices, head = (blockIdx.x / slices) % (p.B * p.H), seg = blockIdx.x / slices / (p.B * p.H);
    const int b = head / p.H, h = head % p.H, g = h / (p.H / p.G);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, lane8 = lane & 7;
    const int col = warp * 4 + (lane >> 3), pc = slice * kCols + col;
    const int len = length_of(p, b);
    const int t_lo = seg * seg_len, t_hi = min(t_lo + seg_len, p.n);
    const int live = min(t_hi, len);
    // (a row may hold more than 2^31 elements)
    const T *x = static_cast<const T *>(p.x) + (size_t)b * p.n * p.x_stride + (size_t)h * p.P + slice * kCols;
    const T *raw = static_cast<const T *>(p.delta) + (size_t)b * p.n * p.delta_stride + h;
    const T *bm = static_cast<const T *>(p.b) + (size_t)b * p.n * p.b_stride + (size_t)g * N;
    const T *cm = static_cast<const T *>(p.c) + (size_t)b * p.n * p.c_stride + (size_t)g * N;
    T *y = static_cast<T *>(p.y) + (size_t)b * p.n * p.y_stride + (size_t)h * p.P + slice * kCols;
    const float a = p.a[h], bias = p.delta_bias ? p.delta_bias[h] : 0.f, skip = p.skip ? p.skip[h] : 0.f;

    if (!kStateOnly && segments > 1) after_previous();
    float st[NS];
    const float *from = kStateOnly ? nullptr
                        : segments > 1 ? seg_state + ((size_t)head * segments + seg) * N * p.P
                        : p.state_in   ? p.state_in + (size_t)head * N * p.P
                                       : nullptr;
#pragma unroll
    for (int i = 0; i < NS; ++i) st[i] = from ? from[(size_t)state_index<NS>(lane8, i) * p.P + pc] : 0.f;
    if (tid == 0) la_sum = 0.f;
    if (!kStateOnly && blockIdx.x == 0 && tid == 0)  // no device-side waits here: never an error
        *reinterpret_cast<WsHeader *>(p.ws) = WsHeader{};

    // a block of tokens is loaded into registers while the one before it is computed
    constexpr int kPer = kTok * N / kScanThreads, kPerX = kTok * kCols / kScanThreads;
    float br[kPer], cr[kPer], xr[kPerX], dr = 0.f;
    auto fetch = [&](int t0) {
        const int left = live - t0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = tid + i * kScanThreads, t = e / N, k = e % N;
            br[i] = t < left ? to_f32(bm[(size_t)(t0 + t) * p.b_stride + k]) : 0.f;
            if (!kStateOnly) cr[i] = t < left ? to_f32(cm[(size_t)(t0 + t) * p.c_stride + k]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kPerX; ++i) {
            const int e = tid + i * kScanThreads, t = e / kCols;
            xr[i] = t < left ? to_f32(x[(size_t)(t0 + t) * p.x_stride + e % kCols]) : 0.f;
        }
        if (tid < kTok) dr = tid < left ? to_f32(raw[(size_t)(t0 + tid) * p.delta_stride]) : 0.f;
    };
    if (t_lo < live) fetch(t_lo);
    for (int t0 = t_lo; t0 < live; t0 += kTok) {
        const int count = min(kTok, live - t0);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = tid + i * kScanThreads;
            bs[e / N][e % N] = br[i];
            if (!kStateOnly) cs[e / N][e % N] = cr[i];
        }
#pragma unroll
        for (int i = 0; i < kPerX; ++i) {
            const int e = tid + i * kScanThreads;
            xs[e / kCols][e % kCols] = xr[i];
        }
        if (tid < count) {
            const float d = step_size(dr, bias, p.softplus);
            dl[tid] = d;
            decay[tid] = expf(a * d);
            if (kStateOnly) {
                float sum = a * d;
                const unsigned mask = (1u << count) - 1u;
                for (int o = 1; o < kTok; o <<= 1) {
                    const float other = __shfl_down_sync(mask, sum, o);
                    if (tid + o < count) sum += other;
                }
                if (tid == 0) la_sum += sum;
            }
        }
        if (t0 + kTok < live) fetch(t0 + kTok);
        __syncthreads();
        for (int t8 = 0; t8 < count; t8 += 8) {
            float part[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                part[u] = 0.f;
                if (t8 + u < count) {
                    const int t = t8 + u;
                    const float e = decay[t], w = dl[t] * xs[t][col];
                    float acc = 0.f;
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        const int k = state_index<NS>(lane8, i);
                        st[i] = fmaf(st[i], e, bs[t][k] * w);
                        if (!kStateOnly) acc = fmaf(st[i], cs[t][k], acc);
                    }
                    part[u] = acc;
                }
            }
            if (!kStateOnly) {
                // sums over the 8 lanes of a column, lane l keeping token t8 + l
#pragma unroll
                for (int w = 4; w > 0; w >>= 1) {
                    const bool up = (lane8 & w) != 0;
#pragma unroll
                    for (int i = 0; i < w; ++i) {
                        const float send = up ? part[i] : part[i + w], keep = up ? part[i + w] : part[i];
                        part[i] = keep + __shfl_xor_sync(0xffffffffu, send, w);
                    }
                }
                if (t8 + lane8 < kTok) ys[t8 + lane8][col] = part[0];
            }
        }
        if (!kStateOnly) {
            __syncthreads();
            for (int i = tid; i < count * kCols; i += kScanThreads) {
                const int t = i / kCols, k = i % kCols;
                from_f32(y + (size_t)(t0 + t) * p.y_stride + k, fmaf(skip, xs[t][k], ys[t][k]));
            }
        }
    }
    if constexpr (kStateOnly) {
        float *to = seg_state + ((size_t)head * segments + seg) * N * p.P;
#pragma unroll
        for (int i = 0; i < NS; ++i) to[(size_t)state_index<NS>(lane8, i) * p.P + pc] = st[i];
        if (tid == 0 && slice == 0) seg_decay[(size_t)head * segments + seg] = la_sum;
    } else {
        for (int i = tid; i < (t_hi - max(t_lo, live)) * kCols; i += kScanThreads)
            from_f32(y + (size_t)(max(t_lo, live) + i / kCols) * p.y_stride + i % kCols, 0.f);
        if (p.state_out && seg == segments - 1) {
            float *to = p.state_out + (size_t)head * N * p.P;
#pragma unroll
            for (int i = 0; i < NS; ++i) to[(size_t)state_index<NS>(lane8, i) * p.P + pc] = st[i];
        }
    }
}

// replaces each segment's own state (from zero) by the state before the segment
__global__ void __launch_bounds__(256)
chain_kernel(const float *state_in, float *seg_state, const float *seg_decay, long long units, int NP, int segments) {
    let_next_begin();
    after_previous();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= units) return;
    const size_t head = i / NP, e = i % NP;
    float h = state_in ? state_in[head * NP + e] : 0.f;
    float *s = seg_state + head * segments * NP + e;
    const float *la = seg_decay + head * segments;
    constexpr int kBatch = 16;  // segments loaded at once
    for (int k0 = 0; k0 < segments; k0 += kBatch) {
        float own[kBatch], decay[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {  // (the last segment has no state of its own)
            const bool on = k0 + u + 1 < segments;
            own[u] = on ? s[(size_t)(k0 + u) * NP] : 0.f;
            decay[u] = on ? la[k0 + u] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (k0 + u < segments) s[(size_t)(k0 + u) * NP] = h;
            h = fmaf(h, expf(decay[u]), own[u]);
        }
    }
}

// One token: the state is read and written once (fp32), HBM-bound.  A block holds `kC` columns of one
// head, four a thread, and all N rows; column sums go through shared memory.
constexpr int kStepThreads = 256;

template <typename T, int kC>
__global__ void __launch_bounds__(kStepThreads) ssm_step_kernel(Ssm p) {
    constexpr int kQuads = kC / 4, kRows = kStepThreads / kQuads;
    __shared__ float4 red[kRows][kQuads];
    __shared__ float bs[128], cs[128];
    let_next_begin();
    after_previous();
    const int slices = p.P / kC, head = blockIdx.x / slices, c0 = (blockIdx.x % slices) * kC;
    const int b = head / p.H, h = head % p.H, g = h / (p.H / p.G), tid = threadIdx.x;
    const int quad = tid % kQuads, row = tid / kQuads;
    float *st = p.state_out + (size_t)head * p.N * p.P + c0 + quad * 4;
    float4 v[128 / kRows > 0 ? 128 / kRows : 1];
    constexpr int kMost = 128 / kRows > 0 ? 128 / kRows : 1;
#pragma unroll
    for (int i = 0; i < kMost; ++i)
        if (row + i * kRows < p.N) v[i] = *reinterpret_cast<const float4 *>(st + (size_t)(row + i * kRows) * p.P);
    if (tid < p.N) {
        bs[tid] = to_f32(static_cast<const T *>(p.b)[(size_t)b * p.b_stride + (size_t)g * p.N + tid]);
        cs[tid] = to_f32(static_cast<const T *>(p.c)[(size_t)b * p.c_stride + (size_t)g * p.N + tid]);
    }
    const float d = step_size(to_f32(static_cast<const T *>(p.delta)[(size_t)b * p.delta_stride + h]),
                              p.delta_bias ? p.delta_bias[h] : 0.f, p.softplus);
    const float e = expf(p.a[h] * d);
    const T *xp = static_cast<const T *>(p.x) + (size_t)b * p.x_stride + (size_t)h * p.P + c0 + quad * 4;
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = to_f32(xp[i]);
    __syncthreads();
    float acc[4] = {};
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int k = row + i * kRows;
        if (k < p.N) {
            const float w = d * bs[k], c = cs[k];
            v[i].x = fmaf(v[i].x, e, w * x[0]);
            v[i].y = fmaf(v[i].y, e, w * x[1]);
            v[i].z = fmaf(v[i].z, e, w * x[2]);
            v[i].w = fmaf(v[i].w, e, w * x[3]);
            *reinterpret_cast<float4 *>(st + (size_t)k * p.P) = v[i];
            acc[0] = fmaf(v[i].x, c, acc[0]);
            acc[1] = fmaf(v[i].y, c, acc[1]);
            acc[2] = fmaf(v[i].z, c, acc[2]);
            acc[3] = fmaf(v[i].w, c, acc[3]);
        }
    }
    red[row][quad] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    __syncthreads();
    if (tid < kC) {
        const float *r = reinterpret_cast<const float *>(&red[0][0]);
        float s = 0.f;
        for (int k = 0; k < kRows && k < p.N; ++k) s += r[k * kC + tid];
        const float xv = to_f32(static_cast<const T *>(p.x)[(size_t)b * p.x_stride + (size_t)h * p.P + c0 + tid]);
        from_f32(static_cast<T *>(p.y) + (size_t)b * p.y_stride + (size_t)h * p.P + c0 + tid,
                 fmaf(p.skip ? p.skip[h] : 0.f, xv, s));
    }
}

// Segments of a prompt: none where the heads alone give every SM two blocks; else as many as that
// takes, of 32 tokens or more (a segment costs a second pass over its tokens)
int segments_of(const Ssm &p) {
    const long long blocks = (long long)p.B * p.H * (p.P / kCols);
    if (blocks >= 152 * 2 || blocks == 0) return 1;
    long long s = (152 * 4 + blocks - 1) / blocks;
    const long long most = p.n / 32;
    if (s > most) s = most;
    return s < 1 ? 1 : (int)s;
}

template <typename T, int N>
cudaError_t scan_as(const Ssm &p, cudaStream_t s) {
    int segments = segments_of(p);
    int seg_len = p.n;
    if (segments > 1) {
        seg_len = ((p.n + segments - 1) / segments + kTok - 1) / kTok * kTok;
        segments = (p.n + seg_len - 1) / seg_len;
    }
    float *state = reinterpret_cast<float *>(p.ws + kWsHeaderBytes);
    const long long BH = (long long)p.B * p.H, NP = (long long)p.N * p.P;
    float *decay = state + BH * segments * NP;
    const unsigned per = (unsigned)(BH * (p.P / kCols));
    if (segments > 1) {
        cudaError_t e = launch_after(scan_kernel<T, N, true>, per * (segments - 1), kScanThreads, 0, s, p, segments,
                                     seg_len, state, decay);
        if (e) return e;
        e = ssm_chain_launch(p.state_in, state, decay, BH, (int)NP, segments, s);
        if (e) return e;
        return launch_after(scan_kernel<T, N, false>, per * segments, kScanThreads, 0, s, p, segments, seg_len, state,
                            decay);
    }
    return launch_after(scan_kernel<T, N, false>, per, kScanThreads, 0, s, p, 1, seg_len, state, decay);
}

template <typename T>
cudaError_t scan_of(const Ssm &p, cudaStream_t s) {
    switch (p.N) {
        case 16: return scan_as<T, 16>(p, s);
        case 32: return scan_as<T, 32>(p, s);
        case 64: return scan_as<T, 64>(p, s);
        default: return scan_as<T, 128>(p, s);
    }
}

template <typename T>
cudaError_t step_of(const Ssm &p, cudaStream_t s) {
    // 16 columns a block (64-byte rows of the state) where whole heads would leave SMs without work
    const long long BH = (long long)p.B * p.H;
    if (p.P == 16 || p.P == 32 || BH < 152 * 2)
        return launch_after(ssm_step_kernel<T, 16>, (unsigned)(BH * (p.P / 16)), kStepThreads, 0, s, p);
    return launch_after(ssm_step_kernel<T, 64>, (unsigned)(BH * (p.P / 64)), kStepThreads, 0, s, p);
}

}  // namespace

cudaError_t ssm_chain_launch(const float *state_in, float *seg_state, const float *seg_decay, long long heads, int NP,
                             int segments, cudaStream_t s) {
    const long long units = heads * NP;
    return launch_after(chain_kernel, (unsigned)((units + 255) / 256), 256, 0, s, state_in, seg_state, seg_decay, units,
                        NP, segments);
}

size_t ssm_scan_workspace_floats(const Ssm &p) {
    const long long s = segments_of(p), BH = (long long)p.B * p.H;
    return s > 1 ? (size_t)(BH * s * ((long long)p.N * p.P + 1)) : 0;
}

int ssm_scan_launches(const Ssm &p) { return segments_of(p) > 1 ? 3 : 1; }

cudaError_t ssm_scan_launch(const Ssm &p, cudaStream_t s) {
    return p.dt == HLA_BF16 ? scan_of<__nv_bfloat16>(p, s) : scan_of<float>(p, s);
}

cudaError_t ssm_step_launch(const Ssm &p, cudaStream_t s) {
    return p.dt == HLA_BF16 ? step_of<__nv_bfloat16>(p, s) : step_of<float>(p, s);
}

}  // namespace hla
