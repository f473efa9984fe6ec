// Gated linear recurrence: prompts, single tokens and gradients.
//
//   s = sigmoid(r), i = sigmoid(g), a = e^(decay s), m = sqrt(1 - a^2), b = m i x,  h_t = a_t h_{t-1} + b_t
// and backwards, with D_t = a_t (dy_t + D_{t+1}) the gradient of h_{t-1} and G_t = dy_t + D_{t+1} that of h_t,
//   dx = G m i,  dg = dx x (1 - i),  e = G (a h_{t-1} - i x (1/m - m)),  dr = e decay s (1 - s),  ddecay = sum e s
// (a^2 / m = 1/m - m).  1 - a^2 is u - u^2/2 + ... where u = -2 decay s is below 1/2: the difference would
// lose what a slow decay is about.
//
// The recurrence composes: a run of tokens takes h to P h + l, so the sequence is walked in tiles whose warps
// scan their own tokens side by side and join by P and l in shared memory; one pass over the data.  A block holds 64
// channels (two a lane, 128 bytes of bf16 a row).  Where there are few channels a cluster of blocks walks
// one sequence together: every block hands its tile's P and l to the others' shared memory, one cluster barrier a
// round, and all form the same state in the same order, so equal inputs give equal bits and no kernel waits on
// another.  The gradient walks the tiles backwards and takes h before each tile from the marks that the forward
// leaves, so it reads every token once too.
#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kChannels = 64;                 // channels of a block
constexpr int kTile = kGlrTile;               // tokens of a block's tile, a mark each
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.44269504f;
constexpr float kTiny = 1e-37f;               // below any 1 - a^2 of a decay that matters: keeps 1/m finite

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rsqrt_of(float x) {
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <typename F>
__device__ __forceinline__ uint64_t each(uint64_t v, F f) {
    float x, y;
    unpair(v, x, y);
    return pair(f(x), f(y));
}
__device__ __forceinline__ uint64_t twice(float x) { return pair(x, x); }

// 1 + e^-v, whose reciprocal is the sigmoid
__device__ __forceinline__ uint64_t one_plus_exp(uint64_t v) {
    return add2(each(mul2(v, twice(-kLog2e)), ex2), twice(1.f));
}

// a lane's decays: log2 and, doubled and negated, natural
struct Decay {
    uint64_t log2a, u;
    __device__ __forceinline__ explicit Decay(uint64_t d) : log2a(mul2(d, twice(kLog2e))), u(mul2(d, twice(-2.f))) {}
};

// a and w = 1 - a^2 from s
__device__ __forceinline__ void decay_of(const Decay &d, uint64_t s, uint64_t &a, uint64_t &w) {
    a = each(mul2(d.log2a, s), ex2);
    const uint64_t u = mul2(d.u, s);
    uint64_t p = fma2(u, twice(1.f / 5040.f), twice(-1.f / 720.f));
    p = fma2(p, u, twice(1.f / 120.f));
    p = fma2(p, u, twice(-1.f / 24.f));
    p = fma2(p, u, twice(1.f / 6.f));
    p = fma2(p, u, twice(-0.5f));
    p = fma2(p, u, twice(1.f));
    p = mul2(p, u);
    const uint64_t far = fma2(mul2(a, twice(-1.f)), a, twice(1.f));
    float u0, u1, p0, p1, f0, f1;
    unpair(u, u0, u1);
    unpair(p, p0, p1);
    unpair(far, f0, f1);
    // (a NaN in r is in both)
    w = pair(u0 < 0.5f ? fmaxf(p0, kTiny) : f0, u1 < 0.5f ? fmaxf(p1, kTiny) : f1);
}

// two channels of one lane: neighbours, or 32 apart where rows are not aligned to pairs
template <bool kVec>
struct Lane {
    int c0, c1;
    bool on0, on1;
    __device__ __forceinline__ Lane(int slab, int C) {
        const int lane = threadIdx.x & 31;
        c0 = slab * kChannels + (kVec ? 2 * lane : lane);
        c1 = kVec ? c0 + 1 : c0 + 32;
        on0 = c0 < C;
        on1 = c1 < C;
    }
    template <typename T>
    __device__ __forceinline__ Raw<T, 2> load(const T *row, bool on) const {
        Raw<T, 2> r = raw_zero<T, 2>();
        if (kVec) {
            if (on && on0) r = raw_load<T, 2>(row + c0);
        } else {
            T *e = reinterpret_cast<T *>(&r);
            if (on && on0) e[0] = row[c0];
            if (on && on1) e[1] = row[c1];
        }
        return r;
    }
    template <typename T>
    __device__ __forceinline__ uint64_t get(const T *row) const {
        uint64_t f[1];
        to_pairs(load(row, true), f);
        return f[0];
    }
    template <typename T>
    __device__ __forceinline__ void put(T *row, uint64_t v) const {
        float x, y;
        unpair(v, x, y);
        if (kVec) {
            const float f[2] = {x, y};
            if (on0) VecIo<T, 2>::store(row + c0, f);
        } else {
            if (on0) from_f32(row + c0, x);
            if (on1) from_f32(row + c1, y);
        }
    }
};

template <typename T>
__device__ __forceinline__ uint64_t as_pair(const Raw<T, 2> &r) {
    uint64_t f[1];
    to_pairs(r, f);
    return f[0];
}

__device__ __forceinline__ unsigned cluster_rank() {
    unsigned r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a value into the same place of another block's shared memory
__device__ __forceinline__ void put_remote(void *mine, unsigned rank, uint64_t a, uint64_t b) {
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(to)
                 : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(mine))), "r"(rank));
    asm volatile("st.shared::cluster.v2.b64 [%0], {%1, %2};" ::"r"(to), "l"(a), "l"(b) : "memory");
}

// what a run of tokens does to a state: h -> p h + l
struct __align__(16) Run {
    uint64_t p, l;
};
__device__ __forceinline__ uint64_t after(const Run &r, uint64_t h) { return fma2(r.p, h, r.l); }

// The state before this warp's tokens and, in `state`, behind the cluster's round, from the runs of every
// warp (in their order, `first` to `last` by `step`) and block.  kOrder 1: tokens forwards, -1: backwards.
template <int kWarps, int kOrder>
__device__ __forceinline__ uint64_t join(const Run (&runs)[kWarps][32], Run (&blocks)[kMaxCluster][32], int S,
                                         unsigned rank, uint64_t &state, uint64_t &tile_in) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint64_t one = twice(1.f);
    __syncthreads();
    if (S == 1) {
        uint64_t mine = 0, h = state;
        tile_in = h;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
            const int w = kOrder > 0 ? k : kWarps - 1 - k;
            if (w == warp) mine = h;
            h = after(runs[w][lane], h);
        }
        state = h;
        return mine;
    }
    Run all{one, 0}, before{one, 0};
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
        const int w = kOrder > 0 ? k : kWarps - 1 - k;
        if (w == warp) before = all;
        const Run r = runs[w][lane];
        all = {mul2(r.p, all.p), after(r, all.l)};
    }
    for (int to = warp; to < S; to += kWarps) put_remote(&blocks[rank][lane], to, all.p, all.l);
    cluster_meet();
    uint64_t h = state;
    for (int k = 0; k < S; ++k) {
        const int b = kOrder > 0 ? k : S - 1 - k;
        if (b == (int)rank) tile_in = h;
        h = after(blocks[b][lane], h);
    }
    state = h;
    return after(before, tile_in);
}

// ------------------------------------------------------------------------------------------------
// forward
// ------------------------------------------------------------------------------------------------

template <typename T>
struct Fwd {
    static constexpr int kTokens = sizeof(T) == 2 ? 8 : 4;  // of a warp: 24 registers of loads in flight
    static constexpr int kWarps = 8, kSpan = kWarps * kTokens;
    static_assert(kSpan % kTile == 0, "a mark is before a warp's tokens");
};

template <typename T, bool kVec>
__global__ void __launch_bounds__(256) glr_forward_kernel(Glr p, int slabs, int S) {
    constexpr int kTok = Fwd<T>::kTokens, kWarps = Fwd<T>::kWarps, kSpan = Fwd<T>::kSpan;
    __shared__ Run runs[2][kWarps][32];
    __shared__ Run blocks[2][kMaxCluster][32];
    let_next_begin();
    after_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = S > 1 ? cluster_rank() : 0, unit = blockIdx.x / S;
    const int b = unit / slabs, slab = unit - b * slabs;
    const Lane<kVec> at(slab, p.C);
    const int len = p.lengths ? min(max(p.lengths[b], 0), p.n) : p.n;
    const Decay decay(at.get(p.decay));
    uint64_t state = p.state_in ? at.get(p.state_in + (size_t)b * p.C) : 0;
    const size_t row0 = (size_t)b * p.n;
    const T *x = static_cast<const T *>(p.x) + row0 * p.x_stride, *r = static_cast<const T *>(p.r) + row0 * p.r_stride,
            *g = static_cast<const T *>(p.g) + row0 * p.g_stride;
    T *y = static_cast<T *>(p.y) + row0 * p.y_stride;

    Raw<T, 2> rx[kTok], rr[kTok], rg[kTok];
    auto load = [&](int t0) {
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            const bool on = t0 + u < len;
            rx[u] = at.load(x + (size_t)(t0 + u) * p.x_stride, on);
            rr[u] = at.load(r + (size_t)(t0 + u) * p.r_stride, on);
            rg[u] = at.load(g + (size_t)(t0 + u) * p.g_stride, on);
        }
    };
    int t0 = rank * kSpan + warp * kTok;
    load(t0);
    if (S > 1) cluster_meet();  // every block is there before its shared memory is written
    const int rounds = (int)(((long long)p.n + (long long)S * kSpan - 1) / ((long long)S * kSpan));
    for (int round = 0; round < rounds; ++round, t0 += S * kSpan) {
        uint64_t h[kTok], pr[kTok];  // this warp's states from 0, and the products of decays
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            uint64_t a, w;
            const uint64_t s = each(one_plus_exp(as_pair(rr[u])), rcp);
            decay_of(decay, s, a, w);
            const uint64_t d = one_plus_exp(as_pair(rg[u]));
            // sqrt(w) / d = w rsqrt(w d^2)  (0 where d^2 leaves the range: i is below 1e-19 there)
            const uint64_t in = mul2(mul2(w, each(mul2(mul2(d, d), w), rsqrt_of)), as_pair(rx[u]));
            const bool on = t0 + u < len;
            if (!on) a = twice(1.f);
            h[u] = u ? fma2(a, h[u - 1], on ? in : 0) : on ? in : 0;
            pr[u] = u ? mul2(a, pr[u - 1]) : a;
        }
        if (round + 1 < rounds) load(t0 + S * kSpan);
        const int buf = round & 1;
        runs[buf][warp][lane] = {pr[kTok - 1], h[kTok - 1]};
        uint64_t tile_in;
        const uint64_t before = join<kWarps, 1>(runs[buf], blocks[buf], S, rank, state, tile_in);
        if (p.marks && t0 % kTile == 0 && t0 < p.n)
            at.put(p.marks + ((size_t)b * glr_marks(p.n) + t0 / kTile) * p.C, before);
#pragma unroll
        for (int u = 0; u < kTok; ++u)
            if (t0 + u < p.n)
                at.put(y + (size_t)(t0 + u) * p.y_stride, t0 + u < len ? fma2(pr[u], before, h[u]) : 0);
    }
    if (p.state_out && rank == 0 && warp == 0) at.put(p.state_out + (size_t)b * p.C, state);
}

// ------------------------------------------------------------------------------------------------
// one token
// ------------------------------------------------------------------------------------------------

template <typename T, bool kVec>
__global__ void __launch_bounds__(128) glr_step_kernel(Glr p, int slabs) {
    let_next_begin();
    after_previous();
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (unit >= (long long)p.B * slabs) return;
    const int b = (int)(unit / slabs);
    const Lane<kVec> at((int)(unit - (long long)b * slabs), p.C);
    const uint64_t x = at.get(static_cast<const T *>(p.x) + (size_t)b * p.x_stride),
                   r = at.get(static_cast<const T *>(p.r) + (size_t)b * p.r_stride),
                   g = at.get(static_cast<const T *>(p.g) + (size_t)b * p.g_stride),
                   h = at.get(p.state_in + (size_t)b * p.C);
    const Decay decay(at.get(p.decay));
    uint64_t a, w;
    decay_of(decay, each(one_plus_exp(r), rcp), a, w);
    const uint64_t d = one_plus_exp(g);
    const uint64_t in = mul2(mul2(w, each(mul2(mul2(d, d), w), rsqrt_of)), x), y = fma2(a, h, in);
    at.put(p.state_out + (size_t)b * p.C, y);
    at.put(static_cast<T *>(p.y) + (size_t)b * p.y_stride, y);
}

// ------------------------------------------------------------------------------------------------
// gradient
// ------------------------------------------------------------------------------------------------

constexpr int kTokBwd = 4, kWarpsBwd = 8;
static_assert(kTokBwd * kWarpsBwd == kTile, "a block's tile of the gradient begins at a mark");

template <typename T, bool kVec>
__global__ void __launch_bounds__(256) glr_backward_kernel(GlrBwd p, int slabs, int S) {
    constexpr int kTok = kTokBwd, kWarps = kWarpsBwd;
    __shared__ Run fwd[2][kWarps][32], bwd[2][kWarps][32];
    __shared__ Run blocks[2][kMaxCluster][32];
    let_next_begin();
    after_previous();
    const Glr &f = p.f;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = S > 1 ? cluster_rank() : 0, unit = blockIdx.x / S;
    const int b = unit / slabs, slab = unit - b * slabs;
    const Lane<kVec> at(slab, f.C);
    const int len = f.lengths ? min(max(f.lengths[b], 0), f.n) : f.n;
    const uint64_t dec = at.get(f.decay);
    const Decay decay(dec);
    uint64_t D = p.dstate_out ? at.get(p.dstate_out + (size_t)b * f.C) : 0;  // the gradient of the state behind the round
    const size_t row0 = (size_t)b * f.n;
    const T *x = static_cast<const T *>(f.x) + row0 * f.x_stride, *r = static_cast<const T *>(f.r) + row0 * f.r_stride,
            *g = static_cast<const T *>(f.g) + row0 * f.g_stride,
            *dy = static_cast<const T *>(p.dy) + row0 * p.dy_stride;
    T *dx = static_cast<T *>(p.dx) + row0 * p.dx_stride, *dr = static_cast<T *>(p.dr) + row0 * p.dr_stride,
      *dg = static_cast<T *>(p.dg) + row0 * p.dg_stride;
    const int marks = glr_marks(f.n);
    const float *mark = f.marks + (size_t)b * marks * f.C;

    Raw<T, 2> rx[kTok], rr[kTok], rg[kTok], rd[kTok];
    uint64_t first = 0;  // the state before the tile
    auto load = [&](int t0) {
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            const bool on = t0 + u < len;
            rx[u] = at.load(x + (size_t)(t0 + u) * f.x_stride, on);
            rr[u] = at.load(r + (size_t)(t0 + u) * f.r_stride, on);
            rg[u] = at.load(g + (size_t)(t0 + u) * f.g_stride, on);
            rd[u] = at.load(dy + (size_t)(t0 + u) * p.dy_stride, on);
        }
        if (t0 / kTile < marks) first = at.get(mark + (size_t)(t0 / kTile) * f.C);
    };
    const int rounds = (marks + S - 1) / S;
    int t0 = ((rounds - 1) * S + rank) * kTile + warp * kTok;
    load(t0);
    if (S > 1) cluster_meet();  // every block is there before its shared memory is written
    uint64_t dsum = 0;
    for (int round = rounds - 1; round >= 0; --round, t0 -= S * kTile) {
        uint64_t a[kTok], s[kTok], m[kTok], in[kTok], vx[kTok], vd[kTok];
        Run forward{twice(1.f), 0};
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            uint64_t w;
            s[u] = each(one_plus_exp(as_pair(rr[u])), rcp);
            decay_of(decay, s[u], a[u], w);
            m[u] = mul2(w, each(w, rsqrt_of));
            in[u] = each(one_plus_exp(as_pair(rg[u])), rcp);
            vx[u] = as_pair(rx[u]);
            vd[u] = as_pair(rd[u]);
            if (t0 + u >= len) a[u] = twice(1.f);  // (x and dy are 0 there)
            forward = {mul2(a[u], forward.p), fma2(a[u], forward.l, mul2(mul2(m[u], in[u]), vx[u]))};
        }
        Run backward{forward.p, 0};
#pragma unroll
        for (int u = kTok - 1; u >= 0; --u) backward.l = mul2(a[u], add2(vd[u], backward.l));
        const int buf = round & 1;
        fwd[buf][warp][lane] = forward;
        bwd[buf][warp][lane] = backward;
        uint64_t h = first, tile_in;
        if (round > 0) load(t0 - S * kTile);
        uint64_t later = join<kWarps, -1>(bwd[buf], blocks[buf], S, rank, D, tile_in);
#pragma unroll
        for (int k = 0; k < kWarps - 1; ++k)
            if (k < warp) h = after(fwd[buf][k][lane], h);
        uint64_t hb[kTok];  // the states before each token
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            hb[u] = h;
            h = fma2(a[u], h, mul2(mul2(m[u], in[u]), vx[u]));
        }
#pragma unroll
        for (int u = kTok - 1; u >= 0; --u) {
            const uint64_t G = add2(vd[u], later);
            later = mul2(a[u], G);
            if (t0 + u < f.n) {
                const bool on = t0 + u < len;
                const uint64_t minus = twice(-1.f);
                const uint64_t vdx = mul2(G, mul2(m[u], in[u]));
                const uint64_t vdg = mul2(mul2(vdx, vx[u]), fma2(in[u], minus, twice(1.f)));
                const uint64_t inv = fma2(m[u], minus, each(m[u], rcp));
                const uint64_t e = mul2(G, fma2(mul2(mul2(in[u], vx[u]), minus), inv, mul2(a[u], hb[u])));
                const uint64_t es = mul2(e, s[u]);
                const uint64_t vdr = mul2(mul2(es, dec), fma2(s[u], minus, twice(1.f)));
                if (on) dsum = add2(dsum, es);
                at.put(dx + (size_t)(t0 + u) * p.dx_stride, on ? vdx : 0);
                at.put(dr + (size_t)(t0 + u) * p.dr_stride, on ? vdr : 0);
                at.put(dg + (size_t)(t0 + u) * p.dg_stride, on ? vdg : 0);
            }
        }
    }
    if (p.dstate_in && rank == 0 && warp == 0) at.put(p.dstate_in + (size_t)b * f.C, D);
    // decay's gradient: the block's warps in order, then (another kernel) its blocks
    __syncthreads();
    fwd[0][warp][lane].p = dsum;
    __syncthreads();
    if (warp == 0) {
#pragma unroll
        for (int k = 1; k < kWarps; ++k) dsum = add2(dsum, fwd[0][k][lane].p);
        at.put(p.partial + ((size_t)b * S + rank) * f.C, dsum);
    }
}

// blocks of one sequence: as many as fill the GPU, each with a tile to work on
int cluster_of(long long units, int n, int span, int want) {
    int S = 1;
    while (S < kMaxCluster && units * S * 2 <= want && (long long)S * span < n) S *= 2;
    return S;
}
int bwd_cluster(int B, int n, int C) { return cluster_of((long long)B * ((C + kChannels - 1) / kChannels), n, kTile, 608); }

template <typename T>
bool pairs_ok(const void *p, long long stride, int C) {
    return C % 2 == 0 && rows_aligned(p, stride, sizeof(T), 2 * sizeof(T));
}

template <typename T, bool kVec>
cudaError_t forward_as(const Glr &p, cudaStream_t s) {
    const int slabs = (p.C + kChannels - 1) / kChannels;
    const int S = cluster_of((long long)p.B * slabs, p.n, Fwd<T>::kSpan, 608);
    return launch_cluster_after(glr_forward_kernel<T, kVec>, (unsigned)((long long)p.B * slabs * S), 256, S, 0, s, p, slabs, S);
}
template <typename T>
cudaError_t forward_of(const Glr &p, cudaStream_t s) {
    return pairs_ok<T>(p.x, p.x_stride, p.C) && pairs_ok<T>(p.r, p.r_stride, p.C) && pairs_ok<T>(p.g, p.g_stride, p.C) &&
                   pairs_ok<T>(p.y, p.y_stride, p.C)
               ? forward_as<T, true>(p, s)
               : forward_as<T, false>(p, s);
}

template <typename T, bool kVec>
cudaError_t step_as(const Glr &p, cudaStream_t s) {
    const int slabs = (p.C + kChannels - 1) / kChannels;
    return launch_after(glr_step_kernel<T, kVec>, (unsigned)(((long long)p.B * slabs + 3) / 4), 128, 0, s, p, slabs);
}
template <typename T>
cudaError_t step_of(const Glr &p, cudaStream_t s) {
    return pairs_ok<T>(p.x, p.x_stride, p.C) && pairs_ok<T>(p.r, p.r_stride, p.C) && pairs_ok<T>(p.g, p.g_stride, p.C) &&
                   pairs_ok<T>(p.y, p.y_stride, p.C)
               ? step_as<T, true>(p, s)
               : step_as<T, false>(p, s);
}

template <typename T, bool kVec>
cudaError_t backward_as(const GlrBwd &p, cudaStream_t s) {
    const Glr &f = p.f;
    const int slabs = (f.C + kChannels - 1) / kChannels, S = bwd_cluster(f.B, f.n, f.C);
    cudaError_t e = launch_cluster_after(glr_backward_kernel<T, kVec>, (unsigned)((long long)f.B * slabs * S), 256, S, 0, s, p,
                                         slabs, S);
    if (e) return e;
    return column_sum_launch({p.partial, (long long)f.B * S, f.C, 1, {p.ddecay}, p.header}, s);
}
template <typename T>
cudaError_t backward_of(const GlrBwd &p, cudaStream_t s) {
    const Glr &f = p.f;
    const bool vec = pairs_ok<T>(f.x, f.x_stride, f.C) && pairs_ok<T>(f.r, f.r_stride, f.C) &&
                     pairs_ok<T>(f.g, f.g_stride, f.C) && pairs_ok<T>(p.dy, p.dy_stride, f.C) &&
                     pairs_ok<T>(p.dx, p.dx_stride, f.C) && pairs_ok<T>(p.dr, p.dr_stride, f.C) &&
                     pairs_ok<T>(p.dg, p.dg_stride, f.C);
    return vec ? backward_as<T, true>(p, s) : backward_as<T, false>(p, s);
}

}  // namespace

bool glr_fits(int B, int C) { return (long long)B * ((C + kChannels - 1) / kChannels) <= (1LL << 27); }
cudaError_t glr_forward_launch(const Glr &p, cudaStream_t s) {
    return p.dt == HLA_BF16 ? forward_of<__nv_bfloat16>(p, s) : forward_of<float>(p, s);
}
cudaError_t glr_step_launch(const Glr &p, cudaStream_t s) {
    return p.dt == HLA_BF16 ? step_of<__nv_bfloat16>(p, s) : step_of<float>(p, s);
}
size_t glr_backward_partial_floats(int B, int n, int C) { return (size_t)B * bwd_cluster(B, n, C) * C; }
cudaError_t glr_backward_launch(const GlrBwd &p, cudaStream_t s) {
    return p.f.dt == HLA_BF16 ? backward_of<__nv_bfloat16>(p, s) : backward_of<float>(p, s);
}

}  // namespace hla
