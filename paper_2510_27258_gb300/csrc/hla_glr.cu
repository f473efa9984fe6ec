// Gated linear recurrence: prompts, single tokens and gradients.
//
//   s = sigmoid(r), i = sigmoid(g), a = e^(decay s), m = sqrt(1 - a^2), b = m i x,  h_t = a_t h_{t-1} + b_t
// and backwards, with D_t = a_t (dy_t + D_{t+1}) the gradient of h_{t-1} and G_t = dy_t + D_{t+1} that of h_t,
//   dx = G m i,  dg = G b (1 - i),  e = G (h_t - i x / m),  dr = e decay s (1 - s),  ddecay = sum e s
// (the derivative of h_t by log a is a h_{t-1} - i x a^2 / m, and a h_{t-1} = h_t - m i x).  Where v = -decay s is at
// most 1, q = 1 - e^-v is a polynomial, and a = 1 - q, m^2 = 1 - a^2 = q (2 - q): a slow decay, which a long memory
// multiplies up, is off by no more than its rounding, and m keeps what 1 - a^2 would lose.  Slabs whose decays are all
// -1 or above take that alone.
//
// The recurrence composes: a run of tokens takes h to P h + l, so the sequence is walked in tiles whose warps scan
// their own tokens side by side and join by P and l in shared memory; one pass over the data.  A block holds 64
// channels (two a lane, 128 bytes of bf16 a row).  Where there are few channels a cluster of blocks walks one sequence
// together: every block hands its tiles' P and l to the others' shared memory, where their bytes count at a barrier, and
// all form the same state in the same order, so equal inputs give equal bits.  The gradient walks the tiles backwards
// and takes h before each tile from the marks that the forward leaves, so it reads every token once too.
//
// Least traffic: four (gradient: seven) values a token and channel.  bf16, B8 n2048 C2048: 53 us, 5.0 TB/s, 76 % of what
// a copy reaches; the gradient 113 us, 4.2 TB/s, 63 %.  Both are bound by issue slots (60 % of them in use, 256 blocks
// of 304 places, 16 warps an SM, which their 128 registers a thread allow), not by DRAM.  B1 n32768 C1024, clusters of
// eight: 86 us, 47 %, of which the exchanges take 10 us and the joins of the tiles 12.  One token of 64 x 2048: 2.6 us on
// the device, 3.5 from memory.  fp32, B4 n2048 C2048: 57 us (71 %), gradient 87 (82 %).  Marks cost the forward 0.3 us.
#include <cstdlib>
#include <type_traits>

#include "hla_vec.cuh"
#include "sm103_prims.cuh"

namespace hla {
namespace {

using namespace sm103;

constexpr int kThreads = 256;
template <int kLanes>
constexpr int kMostBlocks = kLanes == 32 ? 8 : 16;  // of a cluster
// a round in use, the next in flight (with three, on B8 n2048 C2048 bf16: forward 57.3 us instead of 56.3, gradient 124.9
// instead of 124.5)
constexpr int kSlots = 2;
constexpr int kSMs = 152;
constexpr long long kWaitCycles = 4000000000ll, kLandCycles = 200000000ll;  // about 2 and 0.1 s
constexpr uint64_t kLost = 0x7fffffff7fffffffull;  // two NaN, for states behind a wait that ran out
constexpr float kTiny = 1e-37f;               // beside 1 - a^2: keeps 1/m finite where a is 1

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
template <typename T>
__device__ __forceinline__ uint64_t one_plus_exp(uint64_t v) {
    return add2(exp_minus2<T>(v), twice(1.f));
}

// a lane's decays, negated
struct Decay {
    uint64_t d;
    bool near;  // all of the warp's at most 1
    __device__ __forceinline__ explicit Decay(uint64_t decay) : d(mul2(decay, twice(-1.f))) {
        float x, y;
        unpair(d, x, y);
        near = __all_sync(0xffffffffu, x <= 1.f && y <= 1.f);
    }
};

// a and w = 1 - a^2 from s
template <typename T, bool kNear>
__device__ __forceinline__ void decay_of(const Decay &d, uint64_t s, uint64_t &a, uint64_t &w) {
    // (1 - e^-v) / v on 0..1 to 1.3e-8: interpolated at the Chebyshev nodes with the value 1 at 0
    constexpr float kPoly[7] = {1.f, -0.5f, 0.166666031f, -0.0416592546f, 0.00830117054f, -0.001324818f, 0.000137424184f};
    const uint64_t v = mul2(d.d, s), minus = twice(-1.f);
    uint64_t q = fma2(v, twice(kPoly[6]), twice(kPoly[5]));
#pragma unroll
    for (int i = 4; i >= 0; --i) q = fma2(q, v, twice(kPoly[i]));
    q = mul2(q, v);
    a = fma2(q, minus, twice(1.f));
    w = mul2(q, fma2(q, minus, twice(2.f)));
    if (kNear) return;
    const uint64_t far_a = exp_minus2<T>(v), far_w = fma2(mul2(far_a, minus), far_a, twice(1.f));
    float v0, v1, a0, a1, w0, w1, f0, f1, g0, g1;
    unpair(v, v0, v1);
    unpair(a, a0, a1);
    unpair(w, w0, w1);
    unpair(far_a, f0, f1);
    unpair(far_w, g0, g1);
    a = pair(v0 <= 1.f ? a0 : f0, v1 <= 1.f ? a1 : f1);  // (a NaN in r is in both)
    w = pair(v0 <= 1.f ? w0 : g0, v1 <= 1.f ? w1 : g1);
}

// sqrt(w) / d, d = 1 + e^-g being 1 / i: w rsqrt((w + tiny) d^2), whose argument is above 0 whatever w is.  0 where w is 0
// (a shut r) or d^2 leaves the range (i below 1e-19), and where both are so, as where both gates mask a token.  B8 n2048
// C2048 bf16: 53.4 us; with the tiny value behind the product with d^2, which is infinity times 0 there, 52.4; as the
// root of w times the reciprocal of d 55.0.
__device__ __forceinline__ uint64_t input_of(uint64_t w, uint64_t d) {
    return mul2(w, each(mul2(mul2(d, d), add2(w, twice(kTiny))), rsqrt_of));
}

// A block's shape: kLanes lanes walk a token's 2 kLanes channels, so a block of 256 threads has kGroups runs of kTok
// tokens side by side
template <int kLanes_, int kTok_>
struct Shape {
    static constexpr int kLanes = kLanes_, kTok = kTok_, kChannels = 2 * kLanes, kGroups = kThreads / kLanes;
    static constexpr int kOfWarp = 32 / kLanes, kSpan = kGroups * kTok;
    static_assert(kSpan % kGlrTile == 0, "a block's tile begins at a mark");
    static __device__ __forceinline__ int lane() { return threadIdx.x % kLanes; }
    static __device__ __forceinline__ int group() {
        // (the same for a warp where a warp is a group: rows are uniform registers then)
        return kLanes == 32 ? __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0) : threadIdx.x / kLanes;
    }
};

// Two neighbouring channels of one lane
struct Lane {
    uint32_t c0;
    bool on0, on1;
    __device__ __forceinline__ Lane(uint32_t first, int lane, int C) {
        c0 = first + 2 * lane;  // (C is below 2^31 - 256: no wrap)
        on0 = c0 < (uint32_t)C;
        on1 = c0 + 1 < (uint32_t)C;
    }
    // pairs: rows are aligned to two elements, and C is even
    template <typename T>
    __device__ __forceinline__ Raw<T, 2> load(const T *row, bool pairs) const {
        Raw<T, 2> r = raw_zero<T, 2>();
        if (pairs) {
            if (on0) r = raw_load<T, 2>(row + c0);
        } else {
            T *e = reinterpret_cast<T *>(&r);
            if (on0) e[0] = row[c0];
            if (on1) e[1] = row[c0 + 1];
        }
        return r;
    }
    template <typename T>
    __device__ __forceinline__ uint64_t get(const T *row, bool pairs) const {
        uint64_t f[1];
        to_pairs(load(row, pairs), f);
        return f[0];
    }
    template <typename T>
    __device__ __forceinline__ void put(T *row, uint64_t v, bool pairs) const {
        float x, y;
        unpair(v, x, y);
        if (pairs) {
            const float f[2] = {x, y};
            if (on0) VecIo<T, 2>::store(row + c0, f);
        } else {
            if (on0) from_f32(row + c0, x);
            if (on1) from_f32(row + c0 + 1, y);
        }
    }
};

// A lane's next tokens of kTensors tensors, through a ring of kSlots rounds in shared memory by asynchronous copies of a
// warp for itself, all but the round in use in flight.  kWide: rows begin at 16 bytes and are copied in chunks of that.
// Else a lane copies the one or two 4-byte words that hold its two channels, wherever they begin.
template <typename T, typename S, int kTensors, bool kWide>
struct Tokens {
    static constexpr int kTok = S::kTok, kRow = kWide ? S::kChannels * (int)sizeof(T) : S::kLanes * 8, kChunks = kRow / 16;
    static constexpr int kRows = kTok * S::kOfWarp, kSlotBytes = kTensors * kRows * kRow;
    static constexpr int kSmem = kThreads / 32 * kSlots * kSlotBytes;
    const T *from[kTensors];  // the lane's first element of the next round to be sent for
    long long stride[kTensors], ahead_by[kTensors];
    char *ring;      // this warp's
    int len, bytes;  // of the sequence; of this lane's chunk
    unsigned odd;    // a bit for each tensor: this lane's channels of token 0 begin in the middle of a word

    // t0: the group's first token, step: from a round's to the next one's
    __device__ __forceinline__ void set(int i, const void *p, long long row_stride, size_t row0, uint32_t channel, int t0,
                                        int step) {
        const int lane = threadIdx.x & 31;
        const T *at = static_cast<const T *>(p) + row0 * row_stride + channel;
        stride[i] = row_stride;
        ahead_by[i] = step * row_stride;
        if constexpr (kWide) {
            at += (t0 - (S::kOfWarp > 1 ? lane / S::kLanes * kTok : 0) + lane / kChunks) * row_stride +
                  lane % kChunks * (16 / (int)sizeof(T));
        } else {
            if (i == 0) odd = 0;
            odd |= (unsigned)(reinterpret_cast<uintptr_t>(at) >> 1 & 1) << i;
            at += t0 * row_stride + 2 * S::lane();
        }
        from[i] = at;
    }
    __device__ __forceinline__ void open(char *smem, uint32_t channel, int C, int length) {
        ring = smem + (threadIdx.x >> 5) * (kSlots * kSlotBytes);
        len = length;
        const int left = min((int)(C - channel), S::kChannels) * (int)sizeof(T) - (int)(threadIdx.x % kChunks) * 16;
        bytes = min(max(left, 0), 16);
    }
    // whether a lane's channels of token t begin in the middle of a word
    __device__ __forceinline__ bool split(int i, int t) const { return (odd >> i ^ (unsigned)(t & stride[i])) & 1; }
    __device__ __forceinline__ void send(int slot, int t0, const Lane &at) {
        const int lane = threadIdx.x & 31;
        if constexpr (kWide) {
            const int first = t0 - (S::kOfWarp > 1 ? lane / S::kLanes * kTok : 0);  // the warp's
            char *to = ring + slot * kSlotBytes + lane % kChunks * 16;
            const bool all = first >= 0 && first + kRows <= len;
#pragma unroll
            for (int i = 0; i < kTensors; ++i) {
                const T *p = from[i];
                from[i] += ahead_by[i];
#pragma unroll
                for (int u = 0; u < kRows; u += 32 / kChunks, p += 32 / kChunks * stride[i]) {
                    const int t = u + lane / kChunks, row = t % kTok * S::kOfWarp + t / kTok;  // (groups' rows by turns)
                    const int n = all || (unsigned)(first + t) < (unsigned)len ? bytes : 0;  // (0 reads nothing)
                    const uint32_t dst = smem_u32(to + (i * kRows + row) * kRow);
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(p), "r"(n) : "memory");
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kTensors; ++i) {
                const T *p = from[i];
                from[i] += ahead_by[i];
#pragma unroll
                for (int u = 0; u < kTok; ++u, p += stride[i]) {
                    const bool live = (unsigned)(t0 + u) < (unsigned)len;
                    const uint32_t to = smem_u32(ring + slot * kSlotBytes + (i * kTok + u) * 256 + lane * 8);
                    const char *word = reinterpret_cast<const char *>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(3));
                    // (a word that holds one element of the row is memory of the tensor)
                    const bool second = sizeof(T) == 4 || split(i, t0 + u);
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(word),
                                 "r"(live && at.on0 ? 4 : 0)
                                 : "memory");
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 4), "l"(word + 4),
                                 "r"(live && second && at.on1 ? 4 : 0)
                                 : "memory");
                }
            }
        }
        ring_commit();
    }
    // before the first round: the rounds behind it `step` tokens apart
    __device__ __forceinline__ void begin(int t0, int step, const Lane &at) {
#pragma unroll
        for (int k = 0; k < kSlots - 1; ++k) send(k, t0 + k * step, at);
    }
    // at the start of a round: its tokens are there, and the slot of the last round is filled again
    __device__ __forceinline__ void next(int slot, int t0, int step, const Lane &at) {
        ring_wait<kSlots - 2>();
        __syncwarp();
        send(slot ? slot - 1 : kSlots - 1, t0 + (kSlots - 1) * step, at);
    }
    // token t0 + u of the slot
    __device__ __forceinline__ Raw<T, 2> get(int slot, int i, int t0, int u) const {
        if constexpr (kWide) {
            return raw_load<T, 2>(
                reinterpret_cast<const T *>(ring + slot * kSlotBytes + (i * kRows + u * S::kOfWarp) * kRow) +
                2 * (threadIdx.x & 31));
        } else {
            const char *at = ring + slot * kSlotBytes + (i * kTok + u) * 256 + (threadIdx.x & 31) * 8;
            const uint2 w = *reinterpret_cast<const uint2 *>(at);
            Raw<T, 2> r;
            if constexpr (sizeof(T) == 4) r.v = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
            else r.v = split(i, t0 + u) ? __byte_perm(w.x, w.y, 0x5432) : w.x;
            return r;
        }
    }
};

// r of tokens behind a length: minus infinity, whose decay is 1
__device__ __forceinline__ void shut(Raw<__nv_bfloat16, 2> &r) { r.v = 0xff80ff80u; }
__device__ __forceinline__ void shut(Raw<float, 2> &r) { r.v.x = r.v.y = __int_as_float(0xff800000); }

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

// what a run of tokens does to a state: h -> p h + l
struct __align__(16) Run {
    uint64_t p, l;
};
__device__ __forceinline__ uint64_t after(const Run &r, uint64_t h) { return fma2(r.p, h, r.l); }

// What the blocks of a cluster tell one another, in two buffers by turns: a block writes a round's run over the one
// of two rounds before, which every warp of the receiver has read before it sent its run of the last round, which the
// writer has waited for.
template <int kLanes, int kTiles>
struct Exchange {
    Run runs[2][kMostBlocks<kLanes>][kTiles][kLanes], mine[2][kTiles][kLanes];
    uint64_t bar[2];
    int lost;          // a wait of this block's ran out (at the end, in the first block: one of the cluster's did)
    uint32_t missing;  // bytes to wait for that do not come (a test's, in the second block)
};
__device__ __forceinline__ uint32_t in_block(const void *mine, unsigned rank) {
    uint32_t to;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(mine)), "r"(rank));
    return to;
}
// every block is there, its barriers ready
template <int kLanes, int kTiles>
__device__ __forceinline__ void open_exchange(Exchange<kLanes, kTiles> &x, int S, uint32_t missing) {
    if (S == 1) return;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) mbar_init(&x.bar[i], 1);
        x.lost = 0;
        x.missing = cluster_rank() == 1 ? missing : 0;
        fence_mbar_init();
    }
    __syncthreads();
    cluster_meet();
}

template <int kLanes, int kTiles>
__device__ __forceinline__ bool is_lost(const Exchange<kLanes, kTiles> &x) {
    return *reinterpret_cast<const volatile int *>(&x.lost);
}
// Whether the runs of one of the buffers came in time (where a wait of the block's has run out, no other takes longer).
// A lane's own verdict, which decides no more than what the lane's channels are; what a warp or the block does goes by
// x.lost behind a barrier.  (A vote of the warp here took the registers that the gradient's next mark is loaded into: B4
// n2048 C2048 in fp32 97 us instead of 81.)
template <int kLanes, int kTiles>
__device__ __forceinline__ bool wait(Exchange<kLanes, kTiles> &x, int buf, uint32_t parity) {
    if (mbar_try_wait(&x.bar[buf], parity)) return true;
    const long long t0 = clock64();
    while (!mbar_try_wait(&x.bar[buf], parity))
        if (is_lost(x) || clock64() - t0 > kWaitCycles) {
            *reinterpret_cast<volatile int *>(&x.lost) = 1;
            return false;
        }
    return true;
}

// At the end: what was sent to a block has arrived before its shared memory goes.  Where a wait ran out there is no sign
// of a copy but its time: one that was sent lands within microseconds.  The first block, which hands the state on, learns
// whether a wait of any block ran out.
template <int kLanes, int kTiles>
__device__ __forceinline__ void close_exchange(Exchange<kLanes, kTiles> &x) {
    __syncthreads();
    const bool lost = is_lost(x);
    if (lost && threadIdx.x == 0)
        asm volatile("st.shared::cluster.u32 [%0], 1;" ::"r"(in_block(&x.lost, 0)) : "memory");
    __syncwarp();
    cluster_meet();
    const long long t0 = clock64();
    while (lost && clock64() - t0 < kLandCycles) {
    }
}

// A warp's groups as one run: returns it, and in `before` what comes before the lane's group within the warp
template <typename Sh, int kOrder>
__device__ __forceinline__ Run of_warp(const Run &mine, Run &before) {
    before = {twice(1.f), 0};
    if constexpr (Sh::kOfWarp == 1) return mine;
    const Run other{__shfl_xor_sync(0xffffffffu, mine.p, 16), __shfl_xor_sync(0xffffffffu, mine.l, 16)};
    const bool second = ((threadIdx.x & 16) != 0) == (kOrder > 0);
    if (second) before = other;
    const Run &first = second ? other : mine, &then = second ? mine : other;
    return {mul2(then.p, first.p), after(then, first.l)};
}

constexpr int kWarps = kThreads / 32;
template <int kLanes>
using Runs = Run[kWarps][kLanes];

// Joining a tile's runs (kOrder 1: in the warps' order, -1: against it).  Every warp takes those before its own; the last
// one has the tile's, and hands the state behind it to the next tile's warps (`carry`, two places by turns).
template <typename Sh, int kOrder>
struct Joint {
    int warp, place, lane;  // place: in the joining order
    __device__ __forceinline__ Joint() : lane(Sh::lane()) {
        warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
        place = kOrder > 0 ? warp : kWarps - 1 - warp;
    }
    __device__ __forceinline__ bool last() const { return place == kWarps - 1; }
    __device__ __forceinline__ bool speaks() const { return (threadIdx.x & 31) < Sh::kLanes; }
    __device__ __forceinline__ const Run &run(const Runs<Sh::kLanes> &runs, int k) const {
        return runs[kOrder > 0 ? k : kWarps - 1 - k][lane];
    }
    __device__ __forceinline__ void tell(Runs<Sh::kLanes> &runs, const Run &mine) const {
        if (speaks()) runs[warp][lane] = mine;
    }
    // The state before the lane's group; in the last warp `end` is the one behind the tile
    __device__ __forceinline__ uint64_t alone(const Runs<Sh::kLanes> &runs, uint64_t (&carry)[2][Sh::kLanes], int turn,
                                              const Run &mine, const Run &before, uint64_t &end) const {
        __syncthreads();
        uint64_t h = carry[(turn + 1) & 1][lane];
        for (int k = 0; k < place; ++k) h = after(run(runs, k), h);
        if (last()) {
            end = after(mine, h);
            if (speaks()) carry[turn & 1][lane] = end;
        }
        return Sh::kOfWarp == 1 ? h : after(before, h);
    }
    // The same for a cluster's S blocks, each with kTiles tiles of its own between two exchanges: the cluster's first
    // tiles (one a block) come before its second ones.  `state`: behind the round, in every warp.  The wait for the
    // others' runs has a limit, after which (`lost`) the states are NaN from there on, and so is what follows from them.
    // From the next turn on the block sends no more, so no block has all runs of that turn, and every wait for them runs out.
    template <int kTiles>
    __device__ __forceinline__ void among(const Runs<Sh::kLanes> (&runs)[kTiles], Exchange<Sh::kLanes, kTiles> &x,
                                          int turn, int S, unsigned rank, const Run (&mine)[kTiles],
                                          const Run (&before)[kTiles], bool &lost, uint64_t &state,
                                          uint64_t (&got)[kTiles]) const {
        const int buf = turn & 1;
        Run ahead[kTiles];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            ahead[i] = {twice(1.f), 0};
            for (int k = 0; k < place; ++k) {
                const Run r = run(runs[i], k);
                ahead[i] = {mul2(r.p, ahead[i].p), after(r, ahead[i].l)};
            }
            if (last() && speaks()) x.mine[buf][i][lane] = {mul2(mine[i].p, ahead[i].p), after(mine[i], ahead[i].l)};
        }
        if (last() && __all_sync(0xffffffffu, !is_lost(x))) {
            fence_async_smem();
            const int to = threadIdx.x & 31;
            if (to == 0) mbar_arrive_expect_tx(&x.bar[buf], S * (uint32_t)sizeof(x.mine[buf]) + x.missing);
            __syncwarp();
            if (to < S)
                asm volatile(
                    "cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                        in_block(x.runs[buf][rank], to)),
                    "r"(smem_u32(x.mine[buf])), "r"((uint32_t)sizeof(x.mine[buf])), "r"(in_block(&x.bar[buf], to))
                    : "memory");
        }
        if (!lost) lost = !wait(x, buf, (turn >> 1) & 1);
        uint64_t h = lost ? kLost : state;
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            uint64_t tile_in = 0;
            for (int k0 = 0; k0 < S; k0 += 2) {  // (S is even)
                Run r[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) r[k] = x.runs[buf][kOrder > 0 ? k0 + k : S - 1 - k0 - k][i][lane];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if ((kOrder > 0 ? k0 + k : S - 1 - k0 - k) == (int)rank) tile_in = h;
                    h = after(r[k], h);
                }
            }
            got[i] = after(ahead[i], tile_in);
            if (Sh::kOfWarp > 1) got[i] = after(before[i], got[i]);
            if (lost) got[i] = kLost;
        }
        state = h;
    }
};

// ------------------------------------------------------------------------------------------------
// forward
// ------------------------------------------------------------------------------------------------

template <typename T, int kLanes>
using FwdShape = Shape<kLanes, sizeof(T) == 2 ? 8 : 4>;

// kTiles: tiles of a block between two exchanges with its cluster's others (1: a block alone).  The states of all but the
// last one wait in shared memory.  Two: half as many exchanges (B1 n32768 C1024 with three tiles, which leave room for one
// block an SM: 177 us instead of 85).
template <typename T, int kLanes, bool kWide, int kTiles>
struct FwdSmem {
    using In = Tokens<T, FwdShape<T, kLanes>, 3, kWide>;
    static constexpr int kKept = (kTiles - 1) * FwdShape<T, kLanes>::kTok * kThreads * (int)sizeof(Run);
    static constexpr int kBytes = In::kSmem + kKept;
};

template <typename T, int kLanes, bool kWide, int kTiles>
__global__ void __launch_bounds__(kThreads, 2) glr_forward_kernel(Glr p, int slabs, int S, bool y_pairs) {
    using Sh = FwdShape<T, kLanes>;
    constexpr int kTok = Sh::kTok;
    extern __shared__ __align__(128) char smem[];
    // (a cluster's turns take one place, behind a barrier more: two blocks an SM have to fit)
    __shared__ Runs<kLanes> runs[kTiles == 1 ? 2 : 1][kTiles];
    __shared__ uint64_t carry[2][kLanes];        // (kTiles 1)
    __shared__ Exchange<kLanes, kTiles> others;  // (kTiles > 1)
    let_next_begin();
    after_previous();
    const int group = Sh::group(), lane = Sh::lane();
    const unsigned rank = S > 1 ? cluster_rank() : 0, unit = blockIdx.x / S;
    const int b = unit / slabs;
    const uint32_t channel = (unit - b * slabs) * Sh::kChannels;
    const Lane at(channel, lane, p.C);
    const bool pairs = p.C % 2 == 0;
    const int len = p.lengths ? min(max(p.lengths[b], 0), p.n) : p.n;
    const size_t row0 = (size_t)b * p.n;
    const int step = S * Sh::kSpan;
    Tokens<T, Sh, 3, kWide> in;
    int t0 = rank * Sh::kSpan + group * kTok;
    in.set(0, p.x, p.x_stride, row0, channel, t0, step);
    in.set(1, p.r, p.r_stride, row0, channel, t0, step);
    in.set(2, p.g, p.g_stride, row0, channel, t0, step);
    in.open(smem, channel, p.C, len);
    in.begin(t0, step, at);
    Run *kept = reinterpret_cast<Run *>(smem + FwdSmem<T, kLanes, kWide, kTiles>::In::kSmem) + threadIdx.x;
    const Decay decay(at.get(p.decay, pairs));
    uint64_t state = p.state_in ? at.get(p.state_in + (size_t)b * p.C, pairs) : 0;
    T *y = static_cast<T *>(p.y) + (row0 + t0) * p.y_stride;
    const long long y_step = step * p.y_stride;
    const Joint<Sh, 1> joint;
    if (kTiles > 1) open_exchange(others, S, p.missing);
    else if (joint.last() && joint.speaks()) carry[1][lane] = state;
    const int turns = (int)(((long long)p.n + kTiles * step - 1) / (kTiles * step));
    bool lost = false;
    auto walk = [&](auto near) {
        int slot = 0;
        for (int turn = 0; turn < turns; ++turn) {
            uint64_t h[kTok], pr[kTok];  // this group's states from 0, and the products of decays
            Run mine[kTiles], ahead[kTiles];
            const int buf = kTiles == 1 ? turn & 1 : 0;
#pragma unroll
            for (int i = 0; i < kTiles; ++i, t0 += step) {
                in.next(slot, t0, step, at);
                // (a block's second tile may lie behind the sequence as a whole)
                const bool some = kTiles == 1 || i == 0 || t0 - group * kTok < len;
                if (some) {
#pragma unroll
                    for (int u = 0; u < kTok; ++u) {
                        uint64_t a, w;
                        Raw<T, 2> rr = in.get(slot, 1, t0, u);
                        if (t0 + u >= len) shut(rr);  // (x is 0 there)
                        decay_of<T, near()>(decay, each(one_plus_exp<T>(as_pair(rr)), rcp), a, w);
                        const uint64_t d = one_plus_exp<T>(as_pair(in.get(slot, 2, t0, u)));
                        const uint64_t x = as_pair(in.get(slot, 0, t0, u)), add = mul2(input_of(w, d), x);
                        h[u] = u ? fma2(a, h[u - 1], add) : add;
                        pr[u] = u ? mul2(a, pr[u - 1]) : a;
                        if (i + 1 < kTiles) kept[(i * kTok + u) * kThreads] = {pr[u], h[u]};
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < kTok; ++u) {
                        h[u] = 0;
                        pr[u] = twice(1.f);
                        if (i + 1 < kTiles) kept[(i * kTok + u) * kThreads] = {pr[u], 0};
                    }
                }
                if (++slot == kSlots) slot = 0;
                mine[i] = of_warp<Sh, 1>({pr[kTok - 1], h[kTok - 1]}, ahead[i]);
                joint.tell(runs[buf][i], mine[i]);
            }
            uint64_t before[kTiles];
            if constexpr (kTiles == 1) before[0] = joint.alone(runs[buf][0], carry, turn, mine[0], ahead[0], state);
            else joint.among(runs[buf], others, turn, S, rank, mine, ahead, lost, state, before);
            if (kTiles > 1) __syncthreads();  // every warp has read this turn's runs
            int t = t0 - kTiles * step;
#pragma unroll
            for (int i = 0; i < kTiles; ++i, t += step, y += y_step) {
                if (p.marks && t % kGlrTile == 0 && t < p.n)
                    at.put(p.marks + ((size_t)b * glr_marks(p.n) + t / kGlrTile) * p.C, before[i], pairs);
                auto put = [&](T *to, int u, bool on, bool as_pairs) {
                    const Run r = i + 1 < kTiles ? kept[(i * kTok + u) * kThreads] : Run{pr[u], h[u]};
                    at.put(to, on ? after(r, before[i]) : 0, as_pairs);
                };
                T *to = y;
                if (t + kTok <= len && y_pairs) {
#pragma unroll
                    for (int u = 0; u < kTok; ++u, to += p.y_stride) put(to, u, true, true);
                } else {
#pragma unroll
                    for (int u = 0; u < kTok; ++u, to += p.y_stride)
                        if (t + u < p.n) put(to, u, t + u < len, y_pairs);
                }
            }
        }
    };
    if (decay.near) walk(std::true_type());
    else walk(std::false_type());
    auto put_state = [&](uint64_t v) {  // (a block alone: the last warp has it)
        if (p.state_out && rank == 0 && joint.last() && joint.speaks()) at.put(p.state_out + (size_t)b * p.C, v, pairs);
    };
    put_state(state);
    ring_wait<0>();
    if (kTiles > 1) {
        close_exchange(others);
        if (is_lost(others)) put_state(kLost);
    }
}

// ------------------------------------------------------------------------------------------------
// one token
// ------------------------------------------------------------------------------------------------

template <typename T>
__global__ void __launch_bounds__(128) glr_step_kernel(Glr p, int slabs, bool rows_pairs) {
    let_next_begin();
    after_previous();
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (unit >= (long long)p.B * slabs) return;
    const int b = (int)(unit / slabs);
    const Lane at((uint32_t)(unit - (long long)b * slabs) * 64, threadIdx.x & 31, p.C);
    const bool pairs = p.C % 2 == 0;
    const uint64_t x = at.get(static_cast<const T *>(p.x) + (size_t)b * p.x_stride, rows_pairs),
                   r = at.get(static_cast<const T *>(p.r) + (size_t)b * p.r_stride, rows_pairs),
                   g = at.get(static_cast<const T *>(p.g) + (size_t)b * p.g_stride, rows_pairs),
                   h = at.get(p.state_in + (size_t)b * p.C, pairs);
    const Decay decay(at.get(p.decay, pairs));
    uint64_t a, w;
    decay_of<T, false>(decay, each(one_plus_exp<T>(r), rcp), a, w);
    const uint64_t d = one_plus_exp<T>(g);
    const uint64_t add = mul2(input_of(w, d), x), y = fma2(a, h, add);
    at.put(p.state_out + (size_t)b * p.C, y, pairs);
    at.put(static_cast<T *>(p.y) + (size_t)b * p.y_stride, y, rows_pairs);
}

// ------------------------------------------------------------------------------------------------
// gradient
// ------------------------------------------------------------------------------------------------

// kAlone: a sequence is one block's (S is 1).  With both in one kernel B8 n2048 C2048 in bf16 takes 117 us instead of 113.
template <typename T, int kLanes, bool kWide, bool kAlone>
__global__ void __launch_bounds__(kThreads, 2) glr_backward_kernel(GlrBwd p, int slabs, int blocks, bool out_pairs) {
    using Sh = Shape<kLanes, 4>;
    constexpr int kTok = Sh::kTok;
    extern __shared__ __align__(128) char ring[];
    __shared__ Runs<kLanes> fwd[2], bwd[2][1];
    __shared__ uint64_t carry[2][kLanes];   // (kAlone)
    __shared__ Exchange<kLanes, 1> others;  // (else)
    let_next_begin();
    after_previous();
    const Glr &f = p.f;
    const int group = Sh::group(), lane = Sh::lane();
    const int S = kAlone ? 1 : blocks;
    const unsigned rank = kAlone ? 0 : cluster_rank(), unit = blockIdx.x / S;
    const int b = unit / slabs;
    const uint32_t channel = (unit - b * slabs) * Sh::kChannels;
    const Lane at(channel, lane, f.C);
    const bool pairs = f.C % 2 == 0;
    const int len = f.lengths ? min(max(f.lengths[b], 0), f.n) : f.n;
    const size_t row0 = (size_t)b * f.n;
    const int step = -S * Sh::kSpan, rounds = (int)(((long long)f.n - step - 1) / -step);
    Tokens<T, Sh, 4, kWide> in;
    int tile = ((rounds - 1) * S + rank) * Sh::kSpan, t0 = tile + group * kTok;
    in.set(0, f.x, f.x_stride, row0, channel, t0, step);
    in.set(1, f.r, f.r_stride, row0, channel, t0, step);
    in.set(2, f.g, f.g_stride, row0, channel, t0, step);
    in.set(3, p.dy, p.dy_stride, row0, channel, t0, step);
    in.open(ring, channel, f.C, len);
    in.begin(t0, step, at);
    const uint64_t dec = at.get(f.decay, pairs);
    const Decay decay(dec);
    // the gradient of the state behind the round
    uint64_t D = p.dstate_out ? at.get(p.dstate_out + (size_t)b * f.C, pairs) : 0;
    // a group's last token of the round
    T *dx = static_cast<T *>(p.dx) + (long long)(row0 + t0 + kTok - 1) * p.dx_stride,
      *dr = static_cast<T *>(p.dr) + (long long)(row0 + t0 + kTok - 1) * p.dr_stride,
      *dg = static_cast<T *>(p.dg) + (long long)(row0 + t0 + kTok - 1) * p.dg_stride;
    const long long dx_step = step * p.dx_stride, dr_step = step * p.dr_stride, dg_step = step * p.dg_stride;
    const float *mark = f.marks + (size_t)b * glr_marks(f.n) * f.C;
    auto state_before = [&](int t) {
        return (unsigned)t < (unsigned)f.n ? at.get(mark + (size_t)(t / kGlrTile) * f.C, pairs) : 0;
    };
    uint64_t first = state_before(tile);  // the state before the tile
    const Joint<Sh, -1> joint;
    if constexpr (!kAlone) {
        open_exchange(others, S, f.missing);
        if (blockIdx.x == 0 && threadIdx.x == 0) *p.header = WsHeader{};  // (waits set it after seconds)
    } else if (joint.last() && joint.speaks()) {
        carry[1][lane] = D;
    }
    const uint64_t minus = twice(-1.f);
    uint64_t dsum = 0;
    bool lost = false;
    auto walk = [&](auto near) {
        for (int round = 0, slot = 0; round < rounds; ++round, t0 += step, tile += step) {
            uint64_t a[kTok], s[kTok], mi[kTok], rest[kTok], add[kTok], over[kTok];  // .., m i, 1 - i, b, i x / m
            // dy, from the ring each time: registers are what this kernel is short of
            auto vd = [&](int u) { return as_pair(in.get(slot, 3, t0, u)); };
            Run forward{0, 0};
            in.next(slot, t0, step, at);
#pragma unroll
            for (int u = 0; u < kTok; ++u) {
                uint64_t w;
                Raw<T, 2> rr = in.get(slot, 1, t0, u);
                if (t0 + u >= len) shut(rr);  // (x and dy are 0 there)
                s[u] = each(one_plus_exp<T>(as_pair(rr)), rcp);
                decay_of<T, near()>(decay, s[u], a[u], w);
                const uint64_t rm = each(add2(w, twice(kTiny)), rsqrt_of), m = mul2(w, rm);
                const uint64_t i = each(one_plus_exp<T>(as_pair(in.get(slot, 2, t0, u))), rcp);
                const uint64_t ix = mul2(i, as_pair(in.get(slot, 0, t0, u)));
                mi[u] = mul2(m, i);
                rest[u] = fma2(i, minus, twice(1.f));
                add[u] = mul2(m, ix);
                over[u] = mul2(rm, ix);
                forward = u ? Run{mul2(a[u], forward.p), fma2(a[u], forward.l, add[u])} : Run{a[u], add[u]};
            }
            const uint64_t own = forward.p;
            uint64_t back = mul2(a[kTok - 1], vd(kTok - 1));
#pragma unroll
            for (int u = kTok - 2; u >= 0; --u) back = mul2(a[u], add2(vd(u), back));
            const int buf = round & 1;
            Run in_warp, mine[1], ahead[1];
            forward = of_warp<Sh, 1>(forward, in_warp);
            if (joint.speaks()) fwd[buf][joint.warp][lane] = forward;
            mine[0] = of_warp<Sh, -1>({own, back}, ahead[0]);
            joint.tell(bwd[buf][0], mine[0]);
            uint64_t h = first;
            first = state_before(tile + step);
            uint64_t later;
            if constexpr (kAlone) {
                later = joint.alone(bwd[buf][0], carry, round, mine[0], ahead[0], D);
            } else {
                uint64_t got[1];
                joint.among(bwd[buf], others, round, S, rank, mine, ahead, lost, D, got);
                later = got[0];
            }
            for (int k = 0; k < joint.warp; ++k) h = after(fwd[buf][k][lane], h);
            if (Sh::kOfWarp > 1) h = after(in_warp, h);
            uint64_t e[kTok];  // the derivative of the state by log a
#pragma unroll
            for (int u = 0; u < kTok; ++u) {
                h = fma2(a[u], h, add[u]);
                e[u] = fma2(over[u], minus, h);
            }
            T *px = dx, *pr = dr, *pg = dg;
            dx += dx_step;
            dr += dr_step;
            dg += dg_step;
            auto put = [&](int u, bool on, bool as_pairs) {
                const uint64_t G = add2(vd(u), later);
                later = mul2(a[u], G);
                const uint64_t es = mul2(mul2(G, e[u]), s[u]);
                if (on) dsum = add2(dsum, es);
                at.put(px, on ? mul2(G, mi[u]) : 0, as_pairs);
                at.put(pg, on ? mul2(mul2(G, add[u]), rest[u]) : 0, as_pairs);
                at.put(pr, on ? mul2(es, fma2(mul2(s[u], dec), minus, dec)) : 0, as_pairs);
            };
            if (t0 + kTok <= len && out_pairs) {
#pragma unroll
                for (int u = kTok - 1; u >= 0; --u, px -= p.dx_stride, pr -= p.dr_stride, pg -= p.dg_stride)
                    put(u, true, true);
            } else {
#pragma unroll
                for (int u = kTok - 1; u >= 0; --u, px -= p.dx_stride, pr -= p.dr_stride, pg -= p.dg_stride)
                    if (t0 + u < f.n) put(u, t0 + u < len, out_pairs);
            }
            if (++slot == kSlots) slot = 0;
        }
    };
    if (decay.near) walk(std::true_type());
    else walk(std::false_type());
    auto put_state = [&](uint64_t v) {
        if (p.dstate_in && rank == 0 && joint.last() && joint.speaks()) at.put(p.dstate_in + (size_t)b * f.C, v, pairs);
    };
    put_state(D);
    // decay's gradient: the block's warps in order, then (another kernel) its blocks
    if (Sh::kOfWarp > 1) dsum = add2(dsum, __shfl_xor_sync(0xffffffffu, dsum, 16));
    __syncthreads();
    if (joint.speaks()) fwd[0][joint.warp][lane].p = dsum;
    __syncthreads();
    if (threadIdx.x < kLanes) {
#pragma unroll
        for (int k = 1; k < kWarps; ++k) dsum = add2(dsum, fwd[0][k][lane].p);
        at.put(p.partial + ((size_t)b * S + rank) * f.C, dsum, pairs);
    }
    ring_wait<0>();
    if constexpr (!kAlone) {
        close_exchange(others);
        if (is_lost(others)) {
            put_state(kLost);
            if (threadIdx.x == 0) {
                p.header->where = 1;
                p.header->detail = blockIdx.x;
                p.header->error = kDevTimeout;
            }
        }
    }
}

// How a call is spread: lanes for a token's channels, and blocks of one sequence
struct Spread {
    int lanes, slabs, S;
};
// As many blocks as two an SM, up to eight for a sequence; where that leaves half of the SMs' room, blocks take half the
// channels; where few clusters are left even so, they are of sixteen blocks (the GPU holds 36 clusters of eight, 14 of
// sixteen, at two blocks an SM; more would be a second wave: B1 n32768 C1024 in clusters of eight of blocks that fill an
// SM, of which it holds 15, 186 us instead of 85).  A sequence is not given more blocks than it has tiles.
Spread spread(int B, int n, int C, int tok) {
    auto units = [&](int lanes) { return (long long)B * ((C + 2 * lanes - 1) / (2 * lanes)); };
    const int span = 8 * tok;
    Spread r{32, 0, 1};
    while (r.S < 8 && units(32) * r.S * 2 <= 2 * kSMs && (long long)r.S * span < n) r.S *= 2;
    if ((r.S == 8 && units(16) <= 36) || C <= 32) r.lanes = 16;
    if (r.S == 8 && units(16) <= 14 && 8LL * 2 * span < n) r.S = 16;
    r.slabs = (C + 2 * r.lanes - 1) / (2 * r.lanes);
    return r;
}
Spread spread_bwd(int B, int n, int C) { return spread(B, n, C, 4); }

template <typename T>
bool pairs_ok(const void *p, long long stride, int C) {
    return C % 2 == 0 && rows_aligned(p, stride, sizeof(T), 2 * sizeof(T));
}
template <typename T>
bool ring_ok(const void *p, long long stride) {
    return rows_aligned(p, stride, sizeof(T), 16);
}

template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kernel)(P...), long long units, int S, int smem, cudaStream_t s, A... args) {
    cudaError_t e = cudaSuccess;
    if (smem > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (!e && S > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e ? e : launch_cluster_after(kernel, (unsigned)(units * S), kThreads, S, smem, s, args...);
}

template <typename T, int kLanes, bool kWide>
cudaError_t forward_as(const Glr &p, const Spread &r, cudaStream_t s) {
    const bool pairs = pairs_ok<T>(p.y, p.y_stride, p.C);
    const long long units = (long long)p.B * r.slabs;
    return r.S == 1 ? launch_clusters(glr_forward_kernel<T, kLanes, kWide, 1>, units, 1,
                                      FwdSmem<T, kLanes, kWide, 1>::kBytes, s, p, r.slabs, 1, pairs)
                    : launch_clusters(glr_forward_kernel<T, kLanes, kWide, 2>, units, r.S,
                                      FwdSmem<T, kLanes, kWide, 2>::kBytes, s, p, r.slabs, r.S, pairs);
}
template <typename T>
cudaError_t forward_of(const Glr &p, cudaStream_t s) {
    const Spread r = spread(p.B, p.n, p.C, FwdShape<T, 32>::kTok);
    if (ring_ok<T>(p.x, p.x_stride) && ring_ok<T>(p.r, p.r_stride) && ring_ok<T>(p.g, p.g_stride))
        return r.lanes == 32 ? forward_as<T, 32, true>(p, r, s) : forward_as<T, 16, true>(p, r, s);
    return r.lanes == 32 ? forward_as<T, 32, false>(p, r, s) : forward_as<T, 16, false>(p, r, s);
}

template <typename T>
cudaError_t step_of(const Glr &p, cudaStream_t s) {
    const int slabs = (p.C + 63) / 64;
    const bool pairs = pairs_ok<T>(p.x, p.x_stride, p.C) && pairs_ok<T>(p.r, p.r_stride, p.C) &&
                       pairs_ok<T>(p.g, p.g_stride, p.C) && pairs_ok<T>(p.y, p.y_stride, p.C);
    return launch_after(glr_step_kernel<T>, (unsigned)(((long long)p.B * slabs + 3) / 4), 128, 0, s, p, slabs, pairs);
}

template <typename T, int kLanes, bool kWide>
cudaError_t backward_as(const GlrBwd &p, const Spread &r, cudaStream_t s) {
    const Glr &f = p.f;
    const bool pairs = pairs_ok<T>(p.dx, p.dx_stride, f.C) && pairs_ok<T>(p.dr, p.dr_stride, f.C) &&
                       pairs_ok<T>(p.dg, p.dg_stride, f.C);
    const cudaError_t e = launch_clusters(r.S == 1 ? glr_backward_kernel<T, kLanes, kWide, true>
                                                   : glr_backward_kernel<T, kLanes, kWide, false>,
                                          (long long)f.B * r.slabs, r.S, Tokens<T, Shape<kLanes, 4>, 4, kWide>::kSmem, s, p,
                                          r.slabs, r.S, pairs);
    if (e) return e;
    // (blocks that wait for one another have cleared the header before)
    return column_sum_launch({p.partial, (long long)f.B * r.S, f.C, 1, {{p.ddecay, 0, nullptr}}, f.dt, r.S > 1 ? nullptr : p.header},
                             s);
}
template <typename T>
cudaError_t backward_of(const GlrBwd &p, cudaStream_t s) {
    const Glr &f = p.f;
    const Spread r = spread_bwd(f.B, f.n, f.C);
    if (ring_ok<T>(f.x, f.x_stride) && ring_ok<T>(f.r, f.r_stride) && ring_ok<T>(f.g, f.g_stride) &&
        ring_ok<T>(p.dy, p.dy_stride))
        return r.lanes == 32 ? backward_as<T, 32, true>(p, r, s) : backward_as<T, 16, true>(p, r, s);
    return r.lanes == 32 ? backward_as<T, 32, false>(p, r, s) : backward_as<T, 16, false>(p, r, s);
}

// testing: the waits of a sequence's second block run out
uint32_t missing_bytes() { return getenv("HLA_TEST_SHORT_COPY") ? 16 : 0; }

}  // namespace

bool glr_fits(int B, int C) { return (long long)B * ((C + 31) / 32) <= (1LL << 27); }
cudaError_t glr_forward_launch(const Glr &q, cudaStream_t s) {
    Glr p = q;
    p.missing = missing_bytes();
    return p.dt == HLA_BF16 ? forward_of<__nv_bfloat16>(p, s) : forward_of<float>(p, s);
}
cudaError_t glr_step_launch(const Glr &p, cudaStream_t s) {
    return p.dt == HLA_BF16 ? step_of<__nv_bfloat16>(p, s) : step_of<float>(p, s);
}
size_t glr_backward_partial_floats(int B, int n, int C) { return (size_t)B * spread_bwd(B, n, C).S * C; }
cudaError_t glr_backward_launch(const GlrBwd &q, cudaStream_t s) {
    GlrBwd p = q;
    p.f.missing = missing_bytes();
    return p.f.dt == HLA_BF16 ? backward_of<__nv_bfloat16>(p, s) : backward_of<float>(p, s);
}

}  // namespace hla
