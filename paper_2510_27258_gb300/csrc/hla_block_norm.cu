// The norms after and before a block with its gate, residual scale and dropout, and their gradients.
//
//   u = y r1, r1 = 1 / sqrt(mean(y^2) + eps)   (u = y without the norm after the block)
//   x' = alpha x + k scale act(gate) u w_post,   h = x' r2 w_pre,  r2 = 1 / sqrt(mean(x'^2) + eps)
// k is 0 or 1 / (1 - p) by 32 bits for each value, Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random
// numbers: as easy as 1, 2, 3") of (column / 4, row, offset) under the seed: word column % 4; both directions make
// the same bits, none are stored.  Backwards, with t the gradient of x':
//   t = dx' + r2 (dh w_pre - x' r2 mean(dh w_pre x' r2)),  dx = alpha t,  q = t k act(gate),
//   dy = r1 (q scale w_post - u mean(q scale w_post u)),  dgate = t k scale u w_post act'(gate),
//   dw_post = scale sum q u,  dscale = w_post sum q u,  dw_pre = sum dh x' r2   (sums over rows).
//
// Every tensor is read and written once.  A row belongs to a block (up to 256 columns: to 4 to 32 lanes), eight columns a
// thread in registers, with the block's next rows in flight; blocks stay for many rows, so that the weights are loaded
// once and the gradient's sums over rows stay in registers.  What does not depend on a row's sum (gate, random bits) is
// done while the sum's barrier is waited for.  Rows of more than 8192 columns are walked several times by one block.
// Statistics, products and sums are fp32; each output is rounded once.
//
// bf16, B8 n2048 C2048, everything on: forward 68 us, 4.9 TB/s, 74 % of what a copy reaches; gradient 125 us, 4.3 TB/s,
// 65 %.  Bound by issue slots and latency (57 % of the slots in use, 16 warps an SM at 120 registers a thread), the random
// bits first: without dropout 64 and 107 us.  fp32, 8192 rows of the same: 54 us (94 %), gradient 91 (89 %), by memory.
#include <type_traits>

#include "hla_vec.cuh"

namespace hla {
namespace {

constexpr int kPer = 8;                        // columns of a thread
constexpr int kNarrow = 32 * kPer, kWide = 1024 * kPer;
constexpr int kMaxWarps = 32, kNarrowThreads = 128;
// threads of an SM at a time, 128 registers each (768 or 1024, on B8 n2048 C2048 bf16: forward 98 us instead of 69,
// gradient 252 instead of 125)
constexpr int kSmThreads = 512;
constexpr int block_of(int kMax) { return kMax > 32 ? kMax : kNarrowThreads; }

constexpr uint32_t kMul0 = 0xD2511F53u, kMul1 = 0xCD9E8D57u;
constexpr int kRounds = 10;

struct Words {
    uint32_t w[4];
};
// the last rounds of Philox4x32-10, from round kFrom on, with the keys of each round
template <int kFrom>
__device__ __forceinline__ Words philox(const BlockNorm &p, uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3) {
#pragma unroll
    for (int i = kFrom; i < kRounds; ++i) {
        const uint64_t p0 = (uint64_t)c0 * kMul0, p1 = (uint64_t)c2 * kMul1;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ p.key[i][0];
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ p.key[i][1];
        c3 = (uint32_t)p0;
    }
    return {{c0, c1, c2, c3}};
}
// What the first three rounds make of a column group is the same for every row, but for one product of the row:
//   round 0: (r0, r1, r2, r3) = (hi(o0 M1) ^ row ^ k, lo(o0 M1), hi(g M0) ^ o1 ^ k', lo(g M0))
//   round 1: (s0, s1, s2, s3) = (hi(r2 M1) ^ r1 ^ k, lo(r2 M1), hi(r0 M0) ^ r3 ^ k', lo(r0 M0))
//   round 2: (hi(s2 M1) ^ s1 ^ k, lo(s2 M1), hi(s0 M0) ^ s3 ^ k', lo(s0 M0))
// where only r0, s2 and s3 know the row.
struct Group {
    uint32_t a, b, c, d;  // r3 ^ k', s1 ^ k, hi(s0 M0) ^ k', lo(s0 M0)
    __device__ __forceinline__ void set(const BlockNorm &p, uint32_t group) {
        const uint64_t g = (uint64_t)group * kMul0;
        const uint64_t r2 = (uint64_t)((uint32_t)(g >> 32) ^ (uint32_t)(p.offset >> 32) ^ p.key[0][1]) * kMul1;
        const uint64_t r1 = (p.offset & 0xffffffffu) * kMul1;
        const uint64_t s0 = (uint64_t)((uint32_t)(r2 >> 32) ^ (uint32_t)r1 ^ p.key[1][0]) * kMul0;
        a = (uint32_t)g ^ p.key[1][1];
        b = (uint32_t)r2 ^ p.key[2][0];
        c = (uint32_t)(s0 >> 32) ^ p.key[2][1];
        d = (uint32_t)s0;
    }
};
// the row's product of round 1
__device__ __forceinline__ uint64_t row_of(const BlockNorm &p, uint32_t row) {
    return (uint64_t)((uint32_t)((p.offset & 0xffffffffu) * kMul1 >> 32) ^ row ^ p.key[0][0]) * kMul0;
}
__device__ __forceinline__ Words words_of(const BlockNorm &p, const Group &g, uint64_t row) {
    const uint64_t p1 = (uint64_t)((uint32_t)(row >> 32) ^ g.a) * kMul1;
    return philox<3>(p, (uint32_t)(p1 >> 32) ^ g.b, (uint32_t)p1, g.c ^ (uint32_t)row, g.d);
}

// whether one value is kept
__device__ __forceinline__ bool kept(const BlockNorm &p, long long row, int col) {
    const Words r = philox<0>(p, (uint32_t)(col >> 2), (uint32_t)row, (uint32_t)p.offset, (uint32_t)(p.offset >> 32));
    const uint32_t w = (col & 2) ? ((col & 1) ? r.w[3] : r.w[2]) : ((col & 1) ? r.w[1] : r.w[0]);
    return w >= p.drop_below;
}

// act(v) and, if asked, its slope, for values of type T
template <typename T, bool kSlope>
__device__ __forceinline__ float activation(int act, float v, float &slope) {
    if (act == HLA_LINEAR) {
        slope = 1.f;
        return v;
    }
    const float s = __fdividef(1.f, 1.f + exp_minus<T>(v));  // (v of -89 and below: 0, as the rounded sigmoid)
    if (act == HLA_SIGMOID) {
        if (kSlope) slope = s * (1.f - s);
        return s;
    }
    if (kSlope) slope = s * (1.f + v * (1.f - s));
    return v * s;
}

constexpr int kPairs = kPer / 2;
using Pairs = uint64_t[kPairs];

__device__ __forceinline__ uint64_t twice(float x) { return pair(x, x); }

// the same of a thread's columns, two at a time
template <typename T, bool kSlope>
__device__ __forceinline__ void activate(int act, Pairs &v, Pairs &slope) {
    if (act == HLA_LINEAR) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) slope[i] = twice(1.f);
        return;
    }
    const uint64_t one = twice(1.f), minus = twice(-1.f);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        float a, b;
        unpair(add2(exp_minus2<T>(v[i]), one), a, b);
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(a));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(b));
        const uint64_t s = pair(a, b), r = fma2(s, minus, one);
        if (act == HLA_SIGMOID) {
            if (kSlope) slope[i] = mul2(s, r);
            v[i] = s;
        } else {
            if (kSlope) slope[i] = mul2(s, fma2(v[i], r, one));
            v[i] = mul2(v[i], s);
        }
    }
}

// A thread's eight columns: kE accesses of kV neighbours (kNear of them lie side by side), `threads` apart
template <typename T, int kV>
struct Cols {
    static constexpr int kE = kPer / kV, kNear = kV;
    Raw<T, kV> r[kE];
    static __device__ __forceinline__ int at(int e, int t, int threads) { return (e * threads + t) * kV; }
    __device__ __forceinline__ void load(const T *row, int t, int threads, int C) {
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            const int c = at(e, t, threads);
            r[e] = c < C ? raw_load<T, kV>(row + c) : raw_zero<T, kV>();
        }
    }
    __device__ __forceinline__ void get(Pairs &v) const {
        if constexpr (kV == 1) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) v[i] = pair(to_f32(r[2 * i].v[0]), to_f32(r[2 * i + 1].v[0]));
        } else {
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                uint64_t f[kV / 2];
                to_pairs(r[e], f);
#pragma unroll
                for (int i = 0; i < kV / 2; ++i) v[e * kV / 2 + i] = f[i];
            }
        }
    }
    static __device__ __forceinline__ void put(T *row, int t, int threads, int C, const Pairs &v) {
        float f[kPer];
#pragma unroll
        for (int i = 0; i < kPairs; ++i) unpair(v[i], f[2 * i], f[2 * i + 1]);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            const int c = at(e, t, threads);
            float o[kV];
#pragma unroll
            for (int i = 0; i < kV; ++i) o[i] = f[e * kV + i];
            if (c < C) VecIo<T, kV>::store(row + c, o);
        }
    }
};

// bf16 rows of blocks that begin anywhere, in the forward (kWords): pairs of neighbours out of the one or two 4-byte words
// that hold them (a word that holds one element of a row is memory of its tensor).  C 2047: 119 us against 191 by the
// element, C 519 175 against 291; not for rows of lanes (C 255: 110 against 81), nor in the gradient, which has no
// registers for the words of its next row (C 2047: 349 against 250).
constexpr int kWords = 0;
template <>
struct Cols<__nv_bfloat16, kWords> {
    using T = __nv_bfloat16;
    static constexpr int kE = kPer / 2, kNear = 2;
    uint32_t a[kE], b[kE], half;  // words; a bit for each pair of which one element is the row's last
    bool odd;                     // the row begins in the middle of a word
    static __device__ __forceinline__ int at(int e, int t, int threads) { return (e * threads + t) * 2; }
    __device__ __forceinline__ void load(const T *row, int t, int threads, int C) {
        odd = reinterpret_cast<uintptr_t>(row) & 2;
        half = 0;
        const uint32_t *words = reinterpret_cast<const uint32_t *>(reinterpret_cast<uintptr_t>(row) & ~uintptr_t(3));
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            const int c = at(e, t, threads);
            a[e] = c < C ? words[c / 2] : 0u;
            b[e] = odd && c + 1 < C ? words[c / 2 + 1] : 0u;
            if (c + 1 == C) half |= 1u << e;
        }
    }
    __device__ __forceinline__ void get(Pairs &v) const {
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            Raw<T, 2> r;
            r.v = odd ? __byte_perm(a[e], b[e], 0x5432) : a[e];
            if (half >> e & 1) r.v &= 0xffffu;
            uint64_t f[1];
            to_pairs(r, f);
            v[e] = f[0];
        }
    }
    // (every lane takes part) where a row begins in the middle of a word, a lane's words are its first element and the
    // lane's before it: whole words, because halves of them by turns cost twice the way to L2
    static __device__ __forceinline__ void put(T *row, int t, int threads, int C, const Pairs &v) {
        const bool odd = reinterpret_cast<uintptr_t>(row) & 2, first = (t & 31) == 0, last = (t & 31) == 31 || t == threads - 1;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            const int c = at(e, t, threads);
            float f[2];
            unpair(v[e], f[0], f[1]);
            const float before = __shfl_up_sync(0xffffffffu, f[1], 1);
            if (!odd) {
                if (c + 1 < C) VecIo<T, 2>::store(row + c, f);
                else if (c < C) from_f32(row + c, f[0]);
            } else {
                const float pair[2] = {before, f[0]};
                if (c < C) {
                    if (first) from_f32(row + c, f[0]);
                    else VecIo<T, 2>::store(row + c - 1, pair);
                }
                // (where the next lane has nothing of the row, the second is this lane's to write, too)
                if (c + 1 < C && (last || c + 2 >= C)) from_f32(row + c + 1, f[1]);
            }
        }
    }
};

// Zeros in the places of dropped values.  Where a thread's accesses are narrower than the generator's four words, the
// lanes that share a group of four columns each make the words of two of their eight groups and exchange them.
template <int kV>
struct Drop {
    static constexpr int kShare = kV >= 4 ? 1 : 4 / kV;  // lanes to a group
    Group group[2];
    __device__ __forceinline__ void open(const BlockNorm &p, int t, int threads) {
        if (!p.drop) return;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int e = kV >= 4 ? 4 * j / kV : t % kShare + j * kShare;
            group[j].set(p, (uint32_t)((e * threads + t) * kV + (kV >= 4 ? 4 * j % kV : 0)) >> 2);
        }
    }
    // lanes o = 0, 1 or 0 .. 3 that share groups, each with the words of group o, come to have their own words of all
    static __device__ __forceinline__ void exchange(Words &w, int t) {
        if constexpr (kV == 2) {
            const bool odd = t & 1;
            const uint32_t a = __shfl_xor_sync(0xffffffffu, odd ? w.w[0] : w.w[2], 1),
                           b = __shfl_xor_sync(0xffffffffu, odd ? w.w[1] : w.w[3], 1);
            w = odd ? Words{{a, b, w.w[2], w.w[3]}} : Words{{w.w[0], w.w[1], a, b}};
        } else if constexpr (kV == 1) {
#pragma unroll
            for (int o = 1; o < 4; o *= 2) {
                const bool high = t & o;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (i & o) continue;
                    const uint32_t got = __shfl_xor_sync(0xffffffffu, high ? w.w[i] : w.w[i | o], o);
                    if (high) w.w[i] = got; else w.w[i | o] = got;
                }
            }
        }
    }
    struct Kept {
        bool on[kPer];
        // selected, not multiplied: what y and gate hold where a value is dropped, NaN and infinities too, reaches nothing
        __device__ __forceinline__ void apply(Pairs &v) const {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                float a, b;
                unpair(v[i], a, b);
                v[i] = pair(on[2 * i] ? a : 0.f, on[2 * i + 1] ? b : 0.f);
            }
        }
    };
    __device__ __forceinline__ Kept of(const BlockNorm &p, long long row, int t) const {
        Kept keep;
        const uint64_t of_row = row_of(p, (uint32_t)row);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            Words w = words_of(p, group[j], of_row);
            exchange(w, t);
#pragma unroll
            for (int i = 0; i < 4; ++i) keep.on[4 * j + i] = w.w[i] >= p.drop_below;
        }
        return keep;
    }
};

// A thread's columns of the rows that its block takes, one every `step`.  kSlots > 1: through a ring of shared memory,
// all rows but the one in use in flight, written and read by the same thread.  1: in registers, a row ahead.  0: loaded
// where they are used.
template <typename T, int kV, int kTensors, int kSlots>
struct Rows {
    using C8 = Cols<T, kV>;
    const T *from[kTensors];  // (null: not there)
    long long stride[kTensors];
    char *ring;
    int t, threads, C;
    long long rows, step;
    C8 ahead[kSlots == 1 ? kTensors : 1];

    __device__ __forceinline__ char *place(int slot, int i, int e) const {
        return ring + ((slot * kTensors + i) * C8::kE + e) * (int)(blockDim.x * sizeof(Raw<T, kV>));
    }
    __device__ __forceinline__ void send(int slot, long long row) const {
        if constexpr (kSlots > 1) {
#pragma unroll
            for (int i = 0; i < kTensors; ++i)
#pragma unroll
                for (int e = 0; e < C8::kE; ++e) {
                    const int c = C8::at(e, t, threads);
                    if (from[i])
                        ring_copy<T, kV>(reinterpret_cast<Raw<T, kV> *>(place(slot, i, e)), from[i] + row * stride[i] + c,
                                         c < C && row < rows);
                }
            ring_commit();
        }
    }
    __device__ __forceinline__ void begin(char *smem, long long row) {
        if constexpr (kSlots > 1) {
            ring = smem + threadIdx.x * sizeof(Raw<T, kV>);
#pragma unroll
            for (int k = 0; k < kSlots - 1; ++k) send(k, row + k * step);
        } else {
            used(row - step);
        }
    }
    // when a row is in registers
    __device__ __forceinline__ void used(long long row) {
        if constexpr (kSlots == 1) {
#pragma unroll
            for (int i = 0; i < kTensors; ++i)
                if (from[i] && row + step < rows) ahead[i].load(from[i] + (row + step) * stride[i], t, threads, C);
        }
    }
    __device__ __forceinline__ void next(int slot, long long row) const {
        if constexpr (kSlots > 1) {
            ring_wait<kSlots - 2>();
            send(slot ? slot - 1 : kSlots - 1, row + (kSlots - 1) * step);
        }
    }
    __device__ __forceinline__ void get(int slot, int i, long long row, Pairs &v) const {
        C8 c;
        if constexpr (kSlots > 1) {
#pragma unroll
            for (int e = 0; e < C8::kE; ++e)
                c.r[e] = C8::at(e, t, threads) < C ? *reinterpret_cast<const Raw<T, kV> *>(place(slot, i, e))
                                                   : raw_zero<T, kV>();
        } else if constexpr (kSlots == 1) {
            c = ahead[i];
        } else {
            c.load(from[i] + row * stride[i], t, threads, row < rows ? C : 0);
        }
        c.get(v);
    }
};
// Slots of the gradient's ring: three, or two where that would take the room of another block (none where rows are
// read an element at a time, or two do not fit).  The forward, with fewer rows to hold, keeps the next row in registers:
// 68.6 us against 75.3 on B8 n2048 C2048 bf16 (the gradient, whose registers would spill: 159 against 124.6).
template <typename T, int kV, int kMax>
constexpr int slots() {
    constexpr int bytes = 5 * block_of(kMax) * kPer * (int)sizeof(T);
    if (sizeof(Raw<T, kV>) < 4) return 0;
    if (3 * bytes <= 64 * 1024 || (kMax == 512 && 3 * bytes <= 160 * 1024)) return 3;
    return 2 * bytes <= 160 * 1024 ? 2 : 0;
}
template <typename T>
__host__ __device__ constexpr size_t ring_bytes(int threads, int slots) { return (size_t)slots * 5 * threads * kPer * sizeof(T); }

// a weight's eight columns, or ones
template <typename T, int kV>
__device__ __forceinline__ void weight(const void *w, int t, int threads, int C, Pairs &v) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) v[i] = twice(1.f);
        return;
    }
    Cols<T, kV> c;
    c.load(static_cast<const T *>(w), t, threads, C);
    c.get(v);
}

// Sums of kN values over a row's lanes, or over a block through `red` (two buffers in turn: one barrier a sum)
template <int kN>
struct Sum {
    float v[kN];
};
template <int kLanes, int kN>
__device__ __forceinline__ void lane_sum(Sum<kN> &s) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < kN; ++i) s.v[i] += __shfl_xor_sync(0xffffffffu, s.v[i], o);
}
__device__ __forceinline__ void add_up(uint64_t v, float &sum) {
    float a, b;
    unpair(v, a, b);
    sum = a + b;
}
// tell: this warp's part; read: the row's sum, behind a barrier
template <int kMax, int kN>
__device__ __forceinline__ void tell(Sum<kN> &s, float (&red)[2][2][kMaxWarps], int turn) {
    lane_sum<(kMax > 32 ? 32 : kMax)>(s);
    if (kMax > 32 && (threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < kN; ++i) red[turn][i][threadIdx.x >> 5] = s.v[i];
}
template <int kMax, int kN>
__device__ __forceinline__ void read(Sum<kN> &s, float (&red)[2][2][kMaxWarps], int &turn) {
    if (kMax <= 32) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kMax / 32; w += 4) {  // (what is behind the block's last warp was cleared)
            const float4 f = *reinterpret_cast<const float4 *>(&red[turn][i][w]);
            sum += (f.x + f.y) + (f.z + f.w);
        }
        s.v[i] = sum;
    }
    turn ^= 1;
}
template <int kMax, int kN>
__device__ __forceinline__ void row_sum(Sum<kN> &s, float (&red)[2][2][kMaxWarps], int &turn) {
    tell<kMax>(s, red, turn);
    read<kMax>(s, red, turn);
}

__device__ __forceinline__ void clear(float (&red)[2][2][kMaxWarps]) {
    float *f = &red[0][0][0];
    for (int i = threadIdx.x; i < 4 * kMaxWarps; i += blockDim.x) f[i] = 0.f;
    __syncthreads();
}

// ------------------------------------------------------------------------------------------------
// forward
// ------------------------------------------------------------------------------------------------

// kMax: the block's threads at most, or (up to 32) the lanes of a row, of which a block of 128 threads has several
template <typename T, int kV, int kMax>
__global__ void __launch_bounds__(block_of(kMax), kMax == 1024 ? 1 : kSmThreads / block_of(kMax))
block_norm_forward_kernel(BlockNorm p) {
    constexpr bool kBlock = kMax > 32;
    // rows of a block, of a warp
    constexpr int kAtOnce = kBlock ? 1 : kNarrowThreads / kMax, kOfWarp = kBlock ? 1 : 32 / kMax;
    __shared__ __align__(16) float red[2][2][kMaxWarps];
    let_next_begin();
    after_previous();
    int turn = 0;
    if (kBlock) clear(red);
    const int threads = kBlock ? blockDim.x : kMax, t = kBlock ? threadIdx.x : threadIdx.x % kMax, C = p.C;
    const long long step = (long long)gridDim.x * kAtOnce;
    const float inv = 1.f / C;
    Pairs scale, w_pre;  // (the first times w_post and the kept values' factor)
    {
        Pairs w_post;
        weight<T, kV>(p.scale, t, threads, C, scale);
        weight<T, kV>(p.w_post, t, threads, C, w_post);
        weight<T, kV>(p.w_pre, t, threads, C, w_pre);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) scale[i] = mul2(mul2(scale[i], w_post[i]), twice(p.keep_scale));
    }
    Drop<Cols<T, kV>::kNear> drop;
    drop.open(p, t, threads);
    Rows<T, kV, 3, 1> in{{static_cast<const T *>(p.x), static_cast<const T *>(p.y), static_cast<const T *>(p.gate)},
                              {p.x_stride, p.y_stride, p.gate_stride}, nullptr, t, threads, C, p.rows, step};
    long long row = (long long)blockIdx.x * kAtOnce + (kBlock ? 0 : threadIdx.x / kMax);
    // a warp's rows together: those behind the last one take part in sums and exchanges alone
    const int in_warp = kBlock ? 0 : (threadIdx.x & 31) / kMax;
    in.begin(nullptr, row);
    for (; row - in_warp < p.rows; row += step) {
        const bool live = kOfWarp == 1 || row < p.rows;
        Pairs x, y, f;
        in.get(0, 0, row, x);
        in.get(0, 1, row, y);
        if (p.gate) in.get(0, 2, row, f);
        in.used(row);
        Sum<1> s1;
        if (p.post) {
            uint64_t sum = mul2(y[0], y[0]);
#pragma unroll
            for (int i = 1; i < kPairs; ++i) sum = fma2(y[i], y[i], sum);
            add_up(sum, s1.v[0]);
            tell<kMax>(s1, red, turn);
        }
        if (p.gate) {
            Pairs slope;
            activate<T, false>(p.act, f, slope);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) f[i] = mul2(mul2(f[i], scale[i]), y[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) f[i] = mul2(scale[i], y[i]);
        }
        if (p.drop) drop.of(p, row, t).apply(f);
        float r1 = 1.f;
        if (p.post) {
            read<kMax>(s1, red, turn);
            r1 = rsqrtf(s1.v[0] * inv + p.eps);
        }
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            x[i] = fma2(f[i], twice(r1), mul2(x[i], twice(p.alpha)));
            sum = fma2(x[i], x[i], sum);
        }
        Sum<1> s2;
        add_up(sum, s2.v[0]);
        if (p.pre) tell<kMax>(s2, red, turn);
        Cols<T, kV>::put(static_cast<T *>(p.x_out) + row * p.x_out_stride, t, threads, live ? C : 0, x);
        if (p.pre) {
            read<kMax>(s2, red, turn);
            const float r2 = rsqrtf(s2.v[0] * inv + p.eps);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) x[i] = mul2(mul2(x[i], twice(r2)), w_pre[i]);
            Cols<T, kV>::put(static_cast<T *>(p.h) + row * p.h_stride, t, threads, live ? C : 0, x);
        }
    }
}

// One column of a wide row: what both passes over it need.  An element a thread, and all four random words of a group for
// one: bf16, 1365 rows of 12288 (as many values as 8192 x 2048) 278 us, gradient 822, of which the random bits take 53 and
// 224; a copy's rate would take 25 and 40.
template <typename T>
struct Wide {
    const BlockNorm &p;
    long long row;
    __device__ __forceinline__ static float of(const void *w, int c) {
        return w ? to_f32(static_cast<const T *>(w)[c]) : 1.f;
    }
    __device__ __forceinline__ float y(int c) const { return to_f32(static_cast<const T *>(p.y)[row * p.y_stride + c]); }
    __device__ __forceinline__ float keep(int c) const { return !p.drop ? 1.f : kept(p, row, c) ? p.keep_scale : 0.f; }
    __device__ __forceinline__ float act(int c, float &slope) const {
        return p.gate ? activation<T, true>(p.act, to_f32(static_cast<const T *>(p.gate)[row * p.gate_stride + c]), slope)
                      : (slope = 0.f, 1.f);
    }
    // x' of one column (k, a and its slope too)
    __device__ __forceinline__ float x_out(int c, float r1, float &k, float &a, float &slope) const {
        k = keep(c);
        a = act(c, slope);
        const float f = k != 0.f ? y(c) * r1 * of(p.w_post, c) * of(p.scale, c) * k * a : 0.f;
        return p.alpha * to_f32(static_cast<const T *>(p.x)[row * p.x_stride + c]) + f;
    }
};

template <typename T>
__global__ void __launch_bounds__(1024) block_norm_wide_forward_kernel(BlockNorm p) {
    __shared__ __align__(16) float red[2][2][kMaxWarps];
    let_next_begin();
    after_previous();
    int turn = 0;
    const float inv = 1.f / p.C;
    float k, a, slope;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const Wide<T> in{p, row};
        float r1 = 1.f, r2 = 1.f;
        if (p.post) {
            Sum<1> s{{0.f}};
            for (int c = threadIdx.x; c < p.C; c += 1024) s.v[0] += in.y(c) * in.y(c);
            row_sum<1024>(s, red, turn);
            r1 = rsqrtf(s.v[0] * inv + p.eps);
        }
        if (p.pre) {
            Sum<1> s{{0.f}};
            for (int c = threadIdx.x; c < p.C; c += 1024) {
                const float x = in.x_out(c, r1, k, a, slope);
                s.v[0] += x * x;
            }
            row_sum<1024>(s, red, turn);
            r2 = rsqrtf(s.v[0] * inv + p.eps);
        }
        for (int c = threadIdx.x; c < p.C; c += 1024) {  // (x_out may be x: a column is read and written by one thread)
            const float x = in.x_out(c, r1, k, a, slope);
            from_f32(static_cast<T *>(p.x_out) + row * p.x_out_stride + c, x);
            if (p.pre) from_f32(static_cast<T *>(p.h) + row * p.h_stride + c, x * r2 * Wide<T>::of(p.w_pre, c));
        }
    }
}

// ------------------------------------------------------------------------------------------------
// gradient
// ------------------------------------------------------------------------------------------------

// what is left of the gradient where the row's sums are known
__device__ __forceinline__ float grad_x_out(float dx_out, float gw, float x_out, float r2, float m2) {
    return dx_out + r2 * (gw - x_out * r2 * m2);
}

template <typename T, int kV, int kMax>
__global__ void __launch_bounds__(block_of(kMax), kMax == 1024 ? 1 : kSmThreads / block_of(kMax))
block_norm_backward_kernel(BlockNormBwd q) {
    constexpr bool kBlock = kMax > 32;
    // rows of a block, of a warp
    constexpr int kAtOnce = kBlock ? 1 : kNarrowThreads / kMax, kOfWarp = kBlock ? 1 : 32 / kMax;
    __shared__ __align__(16) float red[2][2][kMaxWarps];
    __shared__ float sums[kBlock ? 1 : 2 * kNarrow];
    let_next_begin();
    after_previous();
    const BlockNorm &p = q.f;
    int turn = 0;
    if (kBlock) clear(red);
    const int threads = kBlock ? blockDim.x : kMax, t = kBlock ? threadIdx.x : threadIdx.x % kMax, C = p.C;
    const long long step = (long long)gridDim.x * kAtOnce;
    const float inv = 1.f / C;
    Pairs scale, w_pre;  // (the first times w_post and the kept values' factor)
    {
        Pairs w_post;
        weight<T, kV>(p.scale, t, threads, C, scale);
        weight<T, kV>(p.w_post, t, threads, C, w_post);
        if (kMax < 1024) weight<T, kV>(p.w_pre, t, threads, C, w_pre);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) scale[i] = mul2(mul2(scale[i], w_post[i]), twice(p.keep_scale));
    }
    Drop<Cols<T, kV>::kNear> drop;
    drop.open(p, t, threads);
    Pairs qu = {}, dw_pre = {};  // sums over this thread's rows
    // With 64 registers a thread the sums wait in shared memory and w_pre is read where it is used (gradient of C 8190
    // 285 us instead of 354, of C 6144 248 instead of 278, of C 8192 in fp32 148 instead of 170)
    constexpr bool kApart = kMax == 1024;
    constexpr int kSlots = slots<T, kV, kMax>();
    extern __shared__ __align__(16) char ring[];
    Rows<T, kV, 5, kSlots> in{{static_cast<const T *>(p.x), static_cast<const T *>(p.y), static_cast<const T *>(p.gate),
                               static_cast<const T *>(q.dx_out), static_cast<const T *>(q.dh)},
                              {p.x_stride, p.y_stride, p.gate_stride, q.dx_out_stride, q.dh_stride},
                              nullptr, t, threads, C, p.rows, step};
    // (kApart) this thread's sums in shared memory
    ulonglong2 *apart = reinterpret_cast<ulonglong2 *>(ring + ring_bytes<T>(blockDim.x, kSlots)) + threadIdx.x;
    auto keep_sums = [&](int k, const Pairs &v) {
#pragma unroll
        for (int i = 0; i < kPairs; i += 2) apart[(k * 2 + i / 2) * blockDim.x] = make_ulonglong2(v[i], v[i + 1]);
    };
    auto get_sums = [&](int k, Pairs &v) {
#pragma unroll
        for (int i = 0; i < kPairs; i += 2) {
            const ulonglong2 w = apart[(k * 2 + i / 2) * blockDim.x];
            v[i] = w.x;
            v[i + 1] = w.y;
        }
    };
    if (kApart) {
        keep_sums(0, qu);
        keep_sums(1, dw_pre);
    }
    long long row = (long long)blockIdx.x * kAtOnce + (kBlock ? 0 : threadIdx.x / kMax);
    // a warp's rows together: those behind the last one take part in sums and exchanges alone
    const int in_warp = kBlock ? 0 : (threadIdx.x & 31) / kMax;
    in.begin(ring, row);
    for (int slot = 0; row - in_warp < p.rows; row += step, slot = slot + 1 < kSlots ? slot + 1 : 0) {
        const bool live = kOfWarp == 1 || row < p.rows;
        Pairs x, y, d, h, f[2];  // f: act(gate), act'(gate), 0 where dropped
        in.next(slot, row);
        in.get(slot, 0, row, x);
        in.get(slot, 1, row, y);
        if (p.gate) in.get(slot, 2, row, f[0]);
        in.get(slot, 3, row, d);
        if (p.pre) in.get(slot, 4, row, h);
        Sum<1> s1;
        if (p.post) {
            uint64_t sum = mul2(y[0], y[0]);
#pragma unroll
            for (int i = 1; i < kPairs; ++i) sum = fma2(y[i], y[i], sum);
            add_up(sum, s1.v[0]);
            tell<kMax>(s1, red, turn);
        }
        if (p.gate) {
            activate<T, true>(p.act, f[0], f[1]);
        } else {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) f[0][i] = f[1][i] = twice(1.f);
        }
        if (p.drop) {
            const auto keep = drop.of(p, row, t);
            keep.apply(f[0]);
            keep.apply(f[1]);
            if (!p.post) keep.apply(y);  // (with the norm, u of dropped values is part of dy)
        }
        Pairs fs;  // what multiplies u in x', and t in dn (kApart: made where it is used)
        if (!kApart)
#pragma unroll
            for (int i = 0; i < kPairs; ++i) fs[i] = mul2(f[0][i], scale[i]);
        float r1 = 1.f;
        if (p.post) {
            read<kMax>(s1, red, turn);
            r1 = rsqrtf(s1.v[0] * inv + p.eps);
        }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) y[i] = mul2(y[i], twice(r1));  // u
        if (p.pre) {
            uint64_t sum = 0, dot = 0;
            if (kApart) weight<T, kV>(p.w_pre, t, threads, C, w_pre);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                const uint64_t ax = mul2(x[i], twice(p.alpha));
                x[i] = kApart ? fma2(mul2(y[i], f[0][i]), scale[i], ax) : fma2(y[i], fs[i], ax);  // x'
                sum = fma2(x[i], x[i], sum);
                dot = fma2(mul2(h[i], w_pre[i]), x[i], dot);
            }
            Sum<2> s2;
            add_up(sum, s2.v[0]);
            add_up(dot, s2.v[1]);
            row_sum<kMax>(s2, red, turn);
            const float r2 = rsqrtf(s2.v[0] * inv + p.eps), m2 = s2.v[1] * r2 * inv;
            // t = dx' + r2 (dh w_pre - x' r2 m2)
            const uint64_t by = twice(-r2 * r2 * m2);
            if (kApart) {
                get_sums(1, dw_pre);
                weight<T, kV>(p.w_pre, t, threads, C, w_pre);
            }
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                const uint64_t hr = mul2(h[i], twice(r2));
                d[i] = fma2(x[i], by, fma2(hr, w_pre[i], d[i]));
                if (live) dw_pre[i] = fma2(hr, x[i], dw_pre[i]);
            }
            if (kApart) keep_sums(1, dw_pre);
        }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) x[i] = mul2(d[i], twice(p.alpha));
        Cols<T, kV>::put(static_cast<T *>(q.dx) + row * q.dx_stride, t, threads, live ? C : 0, x);
        uint64_t dot = 0;
        if (kApart) get_sums(0, qu);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const uint64_t du = mul2(d[i], y[i]);
            if (live) qu[i] = fma2(du, f[0][i], qu[i]);
            x[i] = kApart ? mul2(mul2(d[i], f[0][i]), scale[i]) : mul2(d[i], fs[i]);  // q scale w_post
            dot = fma2(x[i], y[i], dot);
            f[1][i] = mul2(mul2(du, f[1][i]), scale[i]);  // dgate
        }
        if (kApart) keep_sums(0, qu);
        Sum<1> s3;
        add_up(dot, s3.v[0]);
        if (p.post) tell<kMax>(s3, red, turn);
        if (p.gate) Cols<T, kV>::put(static_cast<T *>(q.dgate) + row * q.dgate_stride, t, threads, live ? C : 0, f[1]);
        if (p.post) {
            read<kMax>(s3, red, turn);
            const uint64_t m = twice(-s3.v[0] * inv);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) x[i] = mul2(fma2(y[i], m, x[i]), twice(r1));
        }
        Cols<T, kV>::put(static_cast<T *>(q.dy) + row * q.dy_stride, t, threads, live ? C : 0, x);
    }
    if (kSlots > 1) ring_wait<0>();
    if (kApart) {
        get_sums(0, qu);
        get_sums(1, dw_pre);
    }
    // this block's sums, in the order of its warps (the blocks' by column_sum_launch)
    constexpr int kNear = Cols<T, kV>::kNear;
    float sum[2][kPer];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        unpair(mul2(qu[i], twice(p.keep_scale)), sum[0][2 * i], sum[0][2 * i + 1]);
        unpair(dw_pre[i], sum[1][2 * i], sum[1][2 * i + 1]);
    }
    if (!kBlock) {
#pragma unroll
        for (int o = kMax; o < 32; o *= 2)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < kPer; ++i) sum[n][i] += __shfl_xor_sync(0xffffffffu, sum[n][i], o);
        for (int w = 0; w < kNarrowThreads / 32; ++w) {
            if ((threadIdx.x >> 5) == w && in_warp == 0) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int c = Cols<T, kV>::at(i / kNear, t, threads) + i % kNear;
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        sum[n][i] += w ? sums[n * kNarrow + c] : 0.f;
                        sums[n * kNarrow + c] = sum[n][i];
                    }
                }
            }
            __syncthreads();
        }
    }
    float *to = q.partial + (size_t)blockIdx.x * 2 * C;
    if (kBlock || (threadIdx.x >= kNarrowThreads - 32 && in_warp == 0)) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int c = Cols<T, kV>::at(i / kNear, t, threads) + i % kNear;
            if (c < C) {
                to[c] = sum[0][i];
                to[(size_t)C + c] = sum[1][i];
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(1024) block_norm_wide_backward_kernel(BlockNormBwd q) {
    __shared__ __align__(16) float red[2][2][kMaxWarps];
    let_next_begin();
    after_previous();
    const BlockNorm &p = q.f;
    int turn = 0;
    const float inv = 1.f / p.C;
    float *to = q.partial + (size_t)blockIdx.x * 2 * p.C;
    float k, a, slope;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const Wide<T> in{p, row};
        float r1 = 1.f, r2 = 1.f, m2 = 0.f, m1 = 0.f;
        if (p.post) {
            Sum<1> s{{0.f}};
            for (int c = threadIdx.x; c < p.C; c += 1024) s.v[0] += in.y(c) * in.y(c);
            row_sum<1024>(s, red, turn);
            r1 = rsqrtf(s.v[0] * inv + p.eps);
        }
        auto dh = [&](int c) { return p.pre ? to_f32(static_cast<const T *>(q.dh)[row * q.dh_stride + c]) : 0.f; };
        if (p.pre) {
            Sum<2> s{{0.f, 0.f}};
            for (int c = threadIdx.x; c < p.C; c += 1024) {
                const float x = in.x_out(c, r1, k, a, slope);
                s.v[0] += x * x;
                s.v[1] += dh(c) * Wide<T>::of(p.w_pre, c) * x;
            }
            row_sum<1024>(s, red, turn);
            r2 = rsqrtf(s.v[0] * inv + p.eps);
            m2 = s.v[1] * r2 * inv;
        }
        // the gradient of x' (and x' itself)
        auto back = [&](int c, float &x) {
            x = in.x_out(c, r1, k, a, slope);
            const float d = to_f32(static_cast<const T *>(q.dx_out)[row * q.dx_out_stride + c]);
            return p.pre ? grad_x_out(d, dh(c) * Wide<T>::of(p.w_pre, c), x, r2, m2) : d;
        };
        if (p.post) {
            Sum<1> s{{0.f}};
            for (int c = threadIdx.x; c < p.C; c += 1024) {
                float x;
                const float tk = back(c, x);
                if (k != 0.f) s.v[0] += tk * k * a * Wide<T>::of(p.scale, c) * Wide<T>::of(p.w_post, c) * in.y(c) * r1;
            }
            row_sum<1024>(s, red, turn);
            m1 = s.v[0] * inv;
        }
        for (int c = threadIdx.x; c < p.C; c += 1024) {
            float x;
            const float tg = back(c, x), u = in.y(c) * r1, w = Wide<T>::of(p.w_post, c), sc = Wide<T>::of(p.scale, c);
            const bool on = k != 0.f;
            const float tk = on ? tg * k : 0.f, through = on ? tk * a : 0.f;
            from_f32(static_cast<T *>(q.dx) + row * q.dx_stride + c, p.alpha * tg);
            from_f32(static_cast<T *>(q.dy) + row * q.dy_stride + c,
                     p.post ? r1 * (through * sc * w - u * m1) : through * sc * w);
            if (p.gate) from_f32(static_cast<T *>(q.dgate) + row * q.dgate_stride + c, on ? tk * sc * u * w * slope : 0.f);
            const float add[2] = {on ? through * u : 0.f, p.pre ? dh(c) * x * r2 : 0.f};
            const bool first = row == blockIdx.x;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float *at = to + (size_t)j * p.C + c;
                *at = first ? add[j] : *at + add[j];
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------------------

constexpr int kSMs = 152;

struct Plan {
    unsigned grid;
    int threads;
};
// lanes of a narrow row: eight columns each
int lanes_of(int C) { return C <= 32 ? 4 : C <= 64 ? 8 : C <= 128 ? 16 : 32; }
// Blocks that the GPU holds, or fewer where there are not so many rows
Plan plan(long long rows, int C) {
    const int threads = C <= kNarrow ? kNarrowThreads : C > kWide ? 1024 : (C + 32 * kPer - 1) / (32 * kPer) * 32;
    const long long at_once = C <= kNarrow ? kNarrowThreads / lanes_of(C) : 1, blocks = (rows + at_once - 1) / at_once;
    const long long most = (long long)kSMs * (kSmThreads / threads > 0 ? kSmThreads / threads : 1);
    return {(unsigned)(blocks < most ? blocks : most), threads};
}

// whether every row begins at `by` bytes and has whole accesses of so many
template <typename T>
bool rows_of(const BlockNorm &p, size_t by) {
    auto ok = [&](const void *q, long long stride) { return !q || rows_aligned(q, stride, sizeof(T), by); };
    return p.C % (by / sizeof(T)) == 0 && ok(p.x, p.x_stride) && ok(p.y, p.y_stride) && ok(p.gate, p.gate_stride) &&
           ok(p.x_out, p.x_out_stride) && ok(p.h, p.h_stride) && ok(p.w_post, 0) && ok(p.scale, 0) && ok(p.w_pre, 0);
}
template <typename T>
bool rows_of(const BlockNormBwd &q, size_t by) {
    auto ok = [&](const void *p, long long stride) { return !p || rows_aligned(p, stride, sizeof(T), by); };
    return rows_of<T>(q.f, by) && ok(q.dx_out, q.dx_out_stride) && ok(q.dh, q.dh_stride) && ok(q.dx, q.dx_stride) &&
           ok(q.dy, q.dy_stride) && ok(q.dgate, q.dgate_stride);
}
// the widest access that every row allows: 16 bytes, two elements, or one
template <typename T, typename P, typename F>
cudaError_t by_access(const P &p, F f) {
    if (rows_of<T>(p, 16)) return f(std::integral_constant<int, 16 / sizeof(T)>());
    return rows_of<T>(p, 2 * sizeof(T)) ? f(std::integral_constant<int, 2>()) : f(std::integral_constant<int, 1>());
}

template <typename F>
cudaError_t by_threads(int C, int threads, F f) {
    return C <= 32          ? f(std::integral_constant<int, 4>())
           : C <= 64        ? f(std::integral_constant<int, 8>())
           : C <= 128       ? f(std::integral_constant<int, 16>())
           : C <= kNarrow   ? f(std::integral_constant<int, 32>())
           : threads <= 256 ? f(std::integral_constant<int, 256>())
           : threads <= 512 ? f(std::integral_constant<int, 512>())
                            : f(std::integral_constant<int, 1024>());
}
template <typename P>
cudaError_t launch_ring(void (*kernel)(P), const Plan &g, size_t smem, cudaStream_t s, const P &p) {
    if (smem > 32 * 1024) {  // (48 KB with what the kernel has besides)
        const cudaError_t e = allow_smem(kernel, smem);
        if (e) return e;
    }
    return launch_after(kernel, g.grid, g.threads, smem, s, p);
}

template <typename T>
cudaError_t forward_of(const BlockNorm &p, cudaStream_t s) {
    const Plan g = plan(p.rows, p.C);
    if (p.C > kWide) return launch_after(block_norm_wide_forward_kernel<T>, g.grid, 1024, 0, s, p);
    auto as = [&](auto V) -> cudaError_t {
        return by_threads(p.C, g.threads, [&](auto M) {
            constexpr int kV = V() == 1 && sizeof(T) == 2 && M() > 32 ? kWords : V();
            return launch_after(block_norm_forward_kernel<T, kV, M()>, g.grid, g.threads, 0, s, p);
        });
    };
    return by_access<T>(p, as);
}

template <typename T>
cudaError_t backward_of(const BlockNormBwd &q, cudaStream_t s) {
    const BlockNorm &p = q.f;
    const Plan g = plan(p.rows, p.C);
    auto as = [&](auto V) -> cudaError_t {
        return by_threads(p.C, g.threads, [&](auto M) {
            const size_t smem = ring_bytes<T>(g.threads, slots<T, V(), M()>()) + (M() == 1024 ? 64 * g.threads : 0);
            return launch_ring(block_norm_backward_kernel<T, V(), M()>, g, smem, s, q);
        });
    };
    const cudaError_t e =
        p.C > kWide ? launch_after(block_norm_wide_backward_kernel<T>, g.grid, 1024, 0, s, q) : by_access<T>(q, as);
    if (e) return e;
    // (what the sum for dscale is of y is none of a weight that is not there)
    const int post = p.post ? 0 : ColumnSum::kNoSum, pre = p.pre ? 1 : ColumnSum::kNoSum;
    const ColumnSum sums{q.partial, g.grid, p.C, 2,
                         {{q.dw_post, post, p.scale}, {q.dscale, 0, p.w_post}, {q.dw_pre, pre, nullptr}}, p.dt, q.header};
    return column_sum_launch(sums, s);
}

}  // namespace

cudaError_t block_norm_forward_launch(const BlockNorm &p, cudaStream_t s) {
    return p.dt == HLA_BF16 ? forward_of<__nv_bfloat16>(p, s) : forward_of<float>(p, s);
}
size_t block_norm_partial_floats(long long rows, int C) { return (size_t)plan(rows, C).grid * 2 * C; }
cudaError_t block_norm_backward_launch(const BlockNormBwd &q, cudaStream_t s) {
    return q.f.dt == HLA_BF16 ? backward_of<__nv_bfloat16>(q, s) : backward_of<float>(q, s);
}

}  // namespace hla
