// Selective state space scan over prompts on the tensor cores (sm_103a): tcgen05 MMAs with TMEM
// accumulators, TMA tile loads and stores.
//
// With L_t = sum_{u <= t} a delta_u inside a 128-token tile and H the state before it, a tile is
//   S = C B^T,   W_ts = S_ts exp(L_t - L_s) delta_s  (s <= t, else 0)
//   Y = W X + diag(exp(L_t)) C H + skip X
//   H' = exp(L_end) H + B^T (w X),   w_s = exp(L_end - L_s) delta_s
// S depends on the group alone and B^T (.), C (.) take any number of columns, so a CTA works on 128
// columns at once: two heads of a group (P <= 64, padded to 64) or one head of 128.
//
// Decays: the exponent of every pair further apart than a 32-token block factors into a row part and
// a column part that are both <= 0 (for a <= 0), so only the diagonal blocks take an exponential a
// pair; all sums of exponents run inside a block or towards the nearer end, so that weights of
// neighbouring tokens do not come from differences of large numbers.
//
// Precision: products accumulate in fp32 and the state is fp32.  W and the copy of H that
// C H reads are rounded to bf16 once, they only reach the bf16 output.  w X, which reaches the fp32
// state, is a pair hi + lo of bf16 (16 bits), two products: a state is 4e-6 (2-norm) from a 64-bit one, where
// fp32 products would leave 1e-7, and a four-hundredth of what the rounding of the bf16 inputs is.  Values of X
// that are not finite are taken out of W X (take_out).
//
// TMEM (512 columns): S (then W of both heads as packed bf16 in its place), H^T, and Y twice.  H is
// transposed (a lane per column), so that its product's N is the number of states: half the time for
// N <= 64, and neighbouring lanes write neighbouring elements of a state (long scan 77 -> 72 us).  It is
// kept multiplied by the coming tile's decay, so that (w X)^T B accumulates onto it; Y is C H, whose rows
// the epilogue multiplies by exp(L_t) before W X accumulates onto it.
//
// Shared memory, N = 128: C, B and X double-buffered, a slot for H in bf16 and then hi, and lo in C's place
// once S and C H are done.  N <= 64: slots of their own for H, hi and lo, three for X and one for C, so that
// the next tile's w X is split while the tensor cores run W X (long scan 72 -> 68 us).  The output is
// staged in X's place.
//
// Roles: warps 0-15 are the epilogue, warp w on TMEM lanes 32 (w % 4) .. (one row each: a token, or a
// column of H) and columns 32 (w / 4) .. (of H^T: its fourth of the states); warp 16 loads B and C and
// issues MMAs, warp 17 stores the output and loads X (one thread each), warps 18 and 19 compute the next
// tile's decays, one half's each.  They meet at mbarriers only.  The chain from tile to tile is H -> C H -> hi, lo (for
// N = 128 in H's slot) -> H'; the epilogue turns S into W while the tensor cores run (w X)^T B, puts the
// new H down while they run W X, and writes the output while they run the next tile's C H.
//
// What bounds it: a tile of N = 128 takes about 5,200 cycles, the chain C H and S (1,250) -> hi, lo to their
// slots (800) -> (w X)^T B (1,200) -> H' and W X (1,000; an MMA of 64 columns takes as long as one of 128)
// with hand-offs of some 200 each, beside 610 KB through shared memory (4,900 cycles of it).  One of
// N <= 64 takes 4,600, all of it the epilogue's work: hi, lo 1,300, W 1,100, output 700, H' 450, C H 150, the
// rest hand-offs.  Measured on a GB300: B8 n2048 H32 P64 G1 N128 52.2 us (43 % of what its bytes take; 9 of them
// outside the loop over the tiles), B1 n32768 H16 P64 G2 N64 68.2 us in three launches (the state sweep 23, the
// chain 7, this kernel 42, each alone).
//
// Few heads: the sequence is cut into segments, one CTA each; a state-only pass (B and X alone) gives
// each segment's own state, chain_kernel the state before each segment.
#include <cstdlib>
#include <utility>

#include "hla_vec.cuh"
#include "sm103_prims.cuh"
#include "tensor_map.h"

namespace hla {
namespace {

using namespace sm103;

constexpr int kTile = 128;
constexpr int kEpiWarps = 16, kEpiThreads = kEpiWarps * 32;
constexpr int kIssuerWarp = kEpiWarps, kStoreWarp = kEpiWarps + 1, kStepWarp = kEpiWarps + 2;  // (two of the last)
constexpr int kStateThreads = kEpiThreads + 4 * 32, kStateLoadWarp = kEpiWarps + 1, kStateStepWarp = kEpiWarps + 2;
constexpr int kThreads = kEpiThreads + 4 * 32;
// decay of a block (a power of two) down to which its diagonal part is factored, too
constexpr float kFactored = 100.f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

enum Bar {
    bLdX = 0, bLdB = 3, bLdC = 5,              // + stage: X, B, C have landed (N = 128: all three, bLdX)
    bEvS = 7, bEvY2 = 8, bEvY1 = 9, bEvU = 10,  // MMA commits
    bEpE = 11, bEpW = 12, bEpX = 13,           // epilogue hand-offs (16 warp arrivals)
    bEpY0 = 14, bEpY1 = 15,                    // ... of the output, staged in X's slot of even, odd tiles
    bStep = 16,                                // a tile's decays are in shared memory (2 warp arrivals)
    bTot0 = 17, bTot1 = 18,                    // ... an even, odd tile's block decays, ahead of the rest
    bTear = 19,
    kNumBars = 20
};

struct Misc {
    // of both halves' tokens: decay up to the token in its 32-token block, step times the decay from the
    // token to its block's end; decay of each block (of even and odd tiles)
    float cum[2][kTile], cf[2][kTile], tot[2][2][4];
    uint64_t bar[kNumBars];
    uint32_t tmem_base;
    int abort_flag;
    // what the epilogue needs now and then of its place in the problem (kept out of its registers):
    // sequence, first head, segment, whether the second 64 columns are a head of this group
    int b, h0, seg, both;
    // of each slot of X: whether its tile holds a value that is not finite, and the first token with one in each
    // column (a byte each, 255: none)
    int odd[3];
    uint32_t first[3][kTile / 4];
};
static_assert(sizeof(Misc) <= 3 * 1024, "fits beside the tiles");

// shared-memory map for N <= 64 (kN = 64) and N = 128.  N <= 64 has room for H's copy and hi, lo apart.
template <int kN>
struct Map {
    static constexpr bool kApart = kN == 64;
    static constexpr int kXs = kApart ? 3 : 2, kCs = kApart ? 1 : 2;  // stages of X and C (B: two)
    static constexpr uint32_t kOperand = kN / 64 * kBlockBytes;       // a C or B tile
    static constexpr uint32_t C(int s) { return s * kOperand; }
    static constexpr uint32_t B(int s) { return (kCs + s) * kOperand; }
    static constexpr uint32_t X(int s) { return (kCs + 2) * kOperand + s * kTileBytes; }
    static constexpr uint32_t kHi = X(kXs), kH = kApart ? kHi + 2 * kTileBytes : kHi;
    static constexpr uint32_t kEnd = kHi + kTileBytes + (kApart ? kTileBytes + kOperand : 0);
    static constexpr uint32_t lo(int j) { return kApart ? kHi + kTileBytes : C(j & 1); }
    static constexpr uint32_t kBytes = kEnd + sizeof(Misc);
};
static_assert(Map<128>::kBytes <= 232448 && Map<64>::kBytes <= 232448, "shared memory");

constexpr uint32_t kTS = 0, kTH = 128, kTY = 256;  // TMEM columns; Y of even tiles, then of odd ones

struct Params {
    int n, H, P, G, N, softplus;
    int per_group;         // units of 128 columns in a group
    int units, segments, seg_tiles;
    long long delta_stride;
    const __nv_bfloat16 *delta;
    __nv_bfloat16 *y;
    long long y_stride;
    const float *a, *skip, *delta_bias;
    const int *lengths;
    const float *state_in;
    float *state_out, *seg_state, *seg_decay;
    WsHeader *err;
    int clear;             // this launch clears the error word
};

constexpr unsigned long long kBarWaitNs = 2000000000ull;

__device__ __forceinline__ void set_error(WsHeader *err, unsigned where, unsigned detail) {
    if (atomicCAS(&err->error, 0u, (unsigned)kDevTimeout) == 0u) {
        err->where = where;
        err->detail = detail;
    }
}

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// max(v, 0) + log(1 + e), e = exp(-|v|), by log(1 + e) = 2 atanh(s) with s = e / (2 + e) <= 1/3 and the
// series of atanh up to s^13 (what follows is below 2^-23 of the sum)
__device__ __forceinline__ float softplus(float v) {
    const float e = ex2(-kLog2e * fabsf(v)), s = __fdividef(e, 2.f + e), q = s * s;
    float y = fmaf(q, 1.f / 13.f, 1.f / 11.f);
    y = fmaf(q, y, 1.f / 9.f);
    y = fmaf(q, y, 1.f / 7.f);
    y = fmaf(q, y, 1.f / 5.f);
    y = fmaf(q, y, 1.f / 3.f);
    y = fmaf(q, y, 1.f);
    return fmaf(2.f * s, y, fmaxf(v, 0.f));
}

constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
constexpr uint32_t kLboK = 1u << 16, kLboMN = (kBlockBytes >> 4) << 16;

// D (+)= A B, KS steps of 16 over K, N columns, both operands in shared memory (low descriptor words)
template <int N, bool A_MN, bool B_MN, int KS>
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t accumulate) {
    constexpr uint32_t id = idesc_bf16(128, N, A_MN, B_MN);
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
        const uint32_t ka = A_MN ? kk * 128u : (kk >> 2) * (kBlockBytes >> 4) + (kk & 3) * 2u;
        const uint32_t kb = B_MN ? kk * 128u : (kk >> 2) * (kBlockBytes >> 4) + (kk & 3) * 2u;
        umma_bf16(d_tmem, (static_cast<uint64_t>(kDescHi) << 32) | (a_lo + ka),
                  (static_cast<uint64_t>(kDescHi) << 32) | (b_lo + kb), id, kk > 0 ? 1u : accumulate);
    }
}

// D += A B with A (128 x 128 bf16) in TMEM: K elements 16 kk .. of a row packed in columns a_tmem + 16 kk .. +7
template <int N>
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo) {
    constexpr uint32_t id = idesc_bf16(128, N, 0, 1);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
        umma_bf16_ts(d_tmem, a_tmem + 16u * kk,
                     (static_cast<uint64_t>(kDescHi) << 32) | (b_lo + kk * 128u), id, 1u);
}

// a CTA's 128 columns and its tiles
struct Unit {
    int b, g, h0, seg, t_lo, t_hi, live, tiles;  // sequence, group, first head; tokens, those that count
    bool one, both;  // one head of 128 columns, else two heads of up to 64; the second one is in the group
};

__device__ __forceinline__ Unit unit_of(const Params &p) {
    Unit u;
    const int unit = blockIdx.x % p.units, group_heads = p.H / p.G, k = unit % p.per_group;
    u.seg = blockIdx.x / p.units;
    u.one = p.P == 128;
    u.g = unit / p.per_group % p.G;
    u.b = unit / p.per_group / p.G;
    u.h0 = u.g * group_heads + (u.one ? k : 2 * k);
    u.both = u.one || 2 * k + 1 < group_heads;
    u.t_lo = u.seg * p.seg_tiles * kTile;
    u.t_hi = min(u.t_lo + p.seg_tiles * kTile, p.n);
    u.live = min(u.t_hi, p.lengths ? min(max(p.lengths[u.b], 0), p.n) : p.n);
    u.tiles = u.live > u.t_lo ? (u.live - u.t_lo + kTile - 1) / kTile : 0;
    return u;
}

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}

// Elements c .. c + 7 of a row of w X as the bf16 pairs hi + lo.  With w = wh + wl in bf16 (to 2^-17): hi = x wh
// rounded, x wh - hi is a bf16 exactly, and lo = x wl + (x wh - hi) rounded, all by fused multiply-adds on
// the packed elements.  odd collects products of neighbours: it becomes infinite or NaN where an element of X is
// (or where products leave the range).
struct Weight {
    uint32_t wh, wl;
    __device__ explicit Weight(float w) : wh(pack_bf16x2(w, w)) {
        const float rest = w - bf16_lo(wh);
        wl = pack_bf16x2(rest, rest);
    }
};

__device__ __forceinline__ void split8(const uint8_t *xs, int r, int c, const Weight &w, uint4 &hi, uint4 &lo,
                                       uint32_t &odd) {
    const uint4 u = *reinterpret_cast<const uint4 *>(xs + tile_off(r, c));
    const uint32_t x[4] = {u.x, u.y, u.z, u.w};
    uint32_t h[4], l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        h[e] = fma_bf16x2(x[e], w.wh, 0x80008000u);  // (plus minus zero)
        l[e] = fma_bf16x2(x[e], w.wl, fma_bf16x2(x[e], w.wh, h[e] ^ 0x80008000u));
    }
    odd = fma_bf16x2(x[2], x[3], fma_bf16x2(x[0], x[1], odd));
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// 32 of them, rows and columns as in the X tile (hi may take its place); returns odd
__device__ __forceinline__ uint32_t split_row(const uint8_t *xs, uint8_t *hi_tile, uint8_t *lo_tile, int r, int c0, float wr) {
    const Weight w(wr);
    uint32_t odd = 0u;
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
        uint4 hi, lo;
        split8(xs, r, c0 + i, w, hi, lo, odd);
        *reinterpret_cast<uint4 *>(hi_tile + tile_off(r, c0 + i)) = hi;
        *reinterpret_cast<uint4 *>(lo_tile + tile_off(r, c0 + i)) = lo;
    }
    return odd;
}

// Values of X that are not finite, in a tile's row r and columns c0 .. c0 + 31: zero instead, and for each such
// column the first token with one.  (This and put_nan are calls: inlined they cost 0.5 us of 51 where all is finite.)
__device__ __noinline__ void take_out(uint8_t *xs, int r, int c0, uint32_t *first, volatile int *odd) {
#pragma unroll 1
    for (int c = c0; c < c0 + 32; ++c) {
        uint16_t *at = reinterpret_cast<uint16_t *>(xs + tile_off(r, c & ~7)) + (c & 7);
        if ((*at & 0x7f80) != 0x7f80) continue;
        *at = 0;
        uint32_t *word = first + c / 4, old = *(volatile uint32_t *)word;
        const int sh = 8 * (c & 3);
        while ((int)((old >> sh) & 255u) > r) {  // (a swap that fails: another thread's has lowered a byte)
            const uint32_t was = old;
            old = atomicCAS(word, was, (was & ~(255u << sh)) | (uint32_t)r << sh);
            if (old == was) break;
        }
    }
    *odd = 1;
}

// NaN in a tile's rows below `rows` from each column's first token with such a value on; none has one after that
__device__ __noinline__ void put_nan(uint8_t *tile, uint8_t *first, int rows) {
#pragma unroll 1
    for (int c = 0; c < kTile; ++c) {
#pragma unroll 1
        for (int r = first[c]; r < rows; ++r) reinterpret_cast<uint16_t *>(tile + tile_off(r, c & ~7))[c & 7] = 0x7fff;
        first[c] = 255;
    }
}

// The state that a segment's tokens leave, from a zero state (all segments but the last): H = B^T (w X)
// with w_s the decay from token s to the segment's end times its step.  The tiles are taken from the
// last to the first, so that the decay of what follows a tile is known and H only accumulates.
// A stage holds a tile's B and X; hi takes X's place.
template <int kN>
struct StateMap {
    static constexpr uint32_t kOperand = kN / 64 * kBlockBytes;
    static constexpr int kStages = kN == 64 ? 3 : 2;
    static constexpr uint32_t B(int s) { return s * kOperand; }
    static constexpr uint32_t X(int s) { return kStages * kOperand + s * kTileBytes; }
    static constexpr uint32_t Lo(int j) { return kStages * (kOperand + kTileBytes) + (j & 1) * kTileBytes; }
    static constexpr uint32_t kEnd = Lo(1) + kTileBytes;
};

struct StateMisc {
    float cf[2][2][kTile], tot[2][2][4];  // of two tiles' tokens, as in Misc
    uint64_t bar[kNumBars];
    uint32_t tmem_base;
    int abort_flag;
};

static_assert(StateMap<64>::kEnd + sizeof(StateMisc) <= 232448 && StateMap<128>::kEnd + sizeof(StateMisc) <= 232448,
              "shared memory");

// Each of these may complete for later tiles before the last thread has waited for an earlier one's, so a
// barrier serves every second or third tile only: its next completion needs that thread's own next step.
enum StateBar {
    sLd0 = 0,                // + stage: B, X have landed
    sEvU0 = 3,               // + stage: the products are done
    sEpX0 = 6, sEpX1 = 7,    // hi, lo of even, odd tiles are there (16 warp arrivals)
    sStep0 = 8, sStep1 = 9,  // their decays are (2 warp arrivals)
    sTear = 10
};

// Steps and decays of a tile's tokens for one head: four consecutive tokens a lane, whose raw steps are
// `raw`; eight lanes hold a 32-token block.  up: decay of the block up to each token; cf: step times the
// decay from the token to the block's end.
__device__ __forceinline__ void block_decays(const __nv_bfloat16 (&raw)[4], int count, float da, float bias, int softplus_on,
                                             float4 &up4, float4 &cf4) {
    const int lane8 = threadIdx.x & 7;
    float d[4], up[4], down[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // the first `count` of the four tokens count
        const float v = to_f32(raw[i]) + bias;
        d[i] = i < count ? (softplus_on ? softplus(v) : v) : 0.f;
        up[i] = i < count ? da * d[i] : 0.f;
    }
    down[3] = 0.f;
#pragma unroll
    for (int i = 2; i >= 0; --i) down[i] = down[i + 1] + up[i + 1];
    float below = down[0] + up[0], above = below;  // of the lane's four; then inclusive over the block's lanes
#pragma unroll
    for (int i = 1; i < 4; ++i) up[i] += up[i - 1];
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
        const float x = __shfl_up_sync(0xffffffffu, below, o), z = __shfl_down_sync(0xffffffffu, above, o);
        if (lane8 >= o) below += x;
        if (lane8 + o < 8) above += z;
    }
    float first = __shfl_up_sync(0xffffffffu, below, 1), last = __shfl_down_sync(0xffffffffu, above, 1);
    first = lane8 > 0 ? first : 0.f;  // what the lanes before and after it hold
    last = lane8 < 7 ? last : 0.f;
    up4 = make_float4(first + up[0], first + up[1], first + up[2], first + up[3]);
    cf4 = make_float4(ex2(last + down[0]) * d[0], ex2(last + down[1]) * d[1], ex2(last + down[2]) * d[2],
                      ex2(last + down[3]) * d[3]);
}

template <typename M>
__device__ __forceinline__ bool bar_wait(M *ms, int b, uint32_t parity, const Params &p) {
    if (mbar_try_wait(&ms->bar[b], parity)) return true;
    if (*(volatile int *)&ms->abort_flag) return false;
    if (mbar_wait(&ms->bar[b], parity, kBarWaitNs)) return true;
    set_error(p.err, 400 + b, parity);
    *(volatile int *)&ms->abort_flag = 1;
    return false;
}

template <typename M>
__device__ __forceinline__ void epi_arrive(M *ms, int b) {
    tc_fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&ms->bar[b]);
}

template <int kN>
__global__ void __launch_bounds__(kStateThreads, 1)
ssm_state_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_b, Params p) {
    using Sm = StateMap<kN>;
    extern __shared__ __align__(1024) uint8_t smem[];
    StateMisc *ms = reinterpret_cast<StateMisc *>(smem + Sm::kEnd);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool issuer = warp == kEpiWarps;
    after_previous();
    let_next_begin();
    const Unit u = unit_of(p);

    if (blockIdx.x == 0 && tid == 0) *p.err = WsHeader{};  // a wait takes seconds to give up
    if (smem_u32(smem) & 1023u) {                          // the tile layout needs 1 KiB alignment
        if (tid == 0) set_error(p.err, 398, smem_u32(smem));
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < kNumBars; ++i) mbar_init(&ms->bar[i], i == sEpX0 || i == sEpX1 ? kEpiWarps : i == sStep0 || i == sStep1 ? 2 : 1);
        ms->abort_flag = 0;
        fence_mbar_init();
    }
    if (issuer) {
        tmem_alloc(&ms->tmem_base, 128);
        tmem_relinquish();
        if (lane == 0) {
            prefetch_tmap(&tm_x);
            prefetch_tmap(&tm_b);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = ms->tmem_base;

    if (issuer) {
        if (lane == 0) {
            const uint32_t sb4 = smem_u32(smem) >> 4;
            auto lm = [&](uint32_t off) { return sb4 + (off >> 4) + kLboMN; };
            for (int j = 0; j < u.tiles; ++j) {
                const int st = j % Sm::kStages;
                if (!bar_wait(ms, sLd0 + st, (j / Sm::kStages) & 1, p)) break;
                if (!bar_wait(ms, sEpX0 + (j & 1), (j >> 1) & 1, p)) break;
                tc_fence_after();
                mma_ss<kN, true, true, 8>(tb, lm(Sm::X(st)), lm(Sm::B(st)), j > 0 ? 1u : 0u);
                mma_ss<kN, true, true, 8>(tb, lm(Sm::Lo(j)), lm(Sm::B(st)), 1u);
                umma_commit(&ms->bar[sEvU0 + st]);
            }
            // MMAs in flight finish (bounded) before TMEM is released: where a wait gave up, here or in the epilogue,
            // nothing else has waited for them
            umma_commit(&ms->bar[sTear]);
            mbar_wait(&ms->bar[sTear], 0, kBarWaitNs);
        }
        __syncwarp();
    } else if (warp == kStateLoadWarp) {
        if (lane == 0) {
            int j = 0;
            for (; j < u.tiles; ++j) {  // the j-th tile from the end
                const int st = j % Sm::kStages, i = j - Sm::kStages, t = u.t_lo + (u.tiles - 1 - j) * kTile;
                // the products of the tile that held the stage are done
                if (i >= 0 && !bar_wait(ms, sEvU0 + st, (i / Sm::kStages) & 1, p)) break;
                uint64_t *bar = &ms->bar[sLd0 + st];
                mbar_arrive_expect_tx(bar, kTileBytes + Sm::kOperand);
                for (int k = 0; k < kN / 64; ++k)
                    tma_load_4d(smem + Sm::B(st) + k * kBlockBytes, &tm_b, bar, 64 * k, u.g, t, u.b);
                tma_load_4d(smem + Sm::X(st), &tm_x, bar, 0, u.h0, t, u.b);
                tma_load_4d(smem + Sm::X(st) + kBlockBytes, &tm_x, bar, u.one ? 64 : 0,
                            u.one || !u.both ? u.h0 : u.h0 + 1, t, u.b);
            }
            // (where a wait gave up) copies in flight finish before shared memory is released
            for (int i = max(j - Sm::kStages, 0); i < j; ++i)
                mbar_wait(&ms->bar[sLd0 + i % Sm::kStages], (i / Sm::kStages) & 1, kBarWaitNs);
        }
        __syncwarp();
    } else if (warp >= kStateStepWarp) {
        // the decays of half e
        const int e = warp - kStateStepWarp, head = u.one || !e || !u.both ? u.h0 : u.h0 + 1;
        const float da = p.a[head] * kLog2e, bias = p.delta_bias ? p.delta_bias[head] : 0.f;
        const __nv_bfloat16 *from = p.delta + (long long)u.b * p.n * p.delta_stride + head;
        __nv_bfloat16 raw[2][4];  // of two tiles
        auto fetch = [&](int j, __nv_bfloat16 (&r)[4]) {  // rows that do not count: another one's, not used
            const int t = u.t_lo + max(u.tiles - 1 - j, 0) * kTile + 4 * lane;
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = from[(long long)min(t + i, u.live - 1) * p.delta_stride];
        };
        if (u.tiles > 0) {
            fetch(0, raw[0]);
            fetch(1, raw[1]);
        }
#pragma unroll 2
        for (int j = 0; j < u.tiles; ++j) {
            float4 up, cf;
            block_decays(raw[j & 1], u.live - (u.t_lo + (u.tiles - 1 - j) * kTile + 4 * lane), da, bias, p.softplus, up, cf);
            fetch(j + 2, raw[j & 1]);
            // every epilogue warp has done with the decays that were here (the lanes leave together, if one gave up)
            if (j >= 2 && !__all_sync(0xffffffffu, bar_wait(ms, sEpX0 + (j & 1), ((j - 2) >> 1) & 1, p))) break;
            *reinterpret_cast<float4 *>(&ms->cf[j & 1][e][4 * lane]) = cf;
            if ((lane & 7) == 7) ms->tot[j & 1][e][lane >> 3] = up.w;
            __syncwarp();
            if (lane == 0) mbar_arrive(&ms->bar[sStep0 + (j & 1)]);
        }
    } else {
        const int qd = warp & 3, cq = warp >> 2, r = 32 * qd + lane, c0 = 32 * cq, hs = cq >> 1;
        const int head = u.one || !hs || !u.both ? u.h0 : u.h0 + 1;  // a second head that is not there: the first
        float run = 0.f;  // decay of the tiles taken so far (a power of two)
        for (int j = 0; j < u.tiles; ++j) {
            const int buf = j & 1, t0 = u.t_lo + (u.tiles - 1 - j) * kTile;
            const bool in = t0 + r < u.live;
            bar_wait(ms, sStep0 + buf, (j >> 1) & 1, p);
            float later = run;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float x = ms->tot[buf][hs][q];
                if (q > qd) later += x;
                run += x;
            }
            const float wr = ms->cf[buf][hs][r] * ex2(later);
            const int st = j % Sm::kStages;
            uint8_t *xs = smem + Sm::X(st);
            bar_wait(ms, sLd0 + st, (j / Sm::kStages) & 1, p);
            if (t0 + kTile > u.live && !in) {  // tokens that do not count: zero rows, whatever was read
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    const uint4 z = make_uint4(0, 0, 0, 0);
                    *reinterpret_cast<uint4 *>(xs + tile_off(r, c0 + i)) = z;
                    if (kN == 128 || cq < 2) *reinterpret_cast<uint4 *>(smem + Sm::B(st) + tile_off(r, c0 + i)) = z;
                }
            }
            if (j >= 2) {  // the products of two tiles ago have read this lo
                bar_wait(ms, sEvU0 + (j - 2) % Sm::kStages, ((j - 2) / Sm::kStages) & 1, p);
                tc_fence_after();
            }
            split_row(xs, xs, smem + Sm::Lo(j), r, c0, wr);
            fence_async_smem();
            epi_arrive(ms, sEpX0 + buf);
        }
        if (u.tiles > 0) {
            const int i = u.tiles - 1;
            bar_wait(ms, sEvU0 + i % Sm::kStages, (i / Sm::kStages) & 1, p);
            tc_fence_after();
        }
        // TMEM lane r holds column r of the states: those of a head are written by neighbouring lanes
        constexpr int kS = kN / 4;
        const int half = qd >> 1, col = u.one ? r : r & 63, s0 = cq * kS;
        const bool mine = (!half || u.both) && col < p.P;
        const long long at = ((long long)u.b * p.H + (u.one || !half ? u.h0 : u.h0 + 1)) * p.segments + u.seg;
        if (r == 0 && (cq == 0 || (cq == 2 && !u.one && u.both)))  // (of half cq / 2)
            p.seg_decay[((long long)u.b * p.H + head) * p.segments + u.seg] = run * kLn2;
        float *to = p.seg_state + (at * p.N + s0) * p.P + col;
#pragma unroll
        for (int o = 0; o < kS; o += 16) {
            uint32_t v[16];
            tmem_ld16(tb + ((uint32_t)(32 * qd) << 16) + s0 + o, v);  // by whole warps, wherever the values go
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (mine && s0 + o + i < p.N)
                    to[(size_t)(o + i) * p.P] = u.tiles > 0 ? __uint_as_float(v[i]) : 0.f;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (issuer) {
        tc_fence_after();
        tmem_dealloc(tb, 128);
    }
}

template <int kN>
__global__ void __launch_bounds__(kThreads, 1)
ssm_tc_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_b,
              const __grid_constant__ CUtensorMap tm_c, const __grid_constant__ CUtensorMap tm_y, Params p) {
    using Sm = Map<kN>;
    extern __shared__ __align__(1024) uint8_t smem[];
    Misc *ms = reinterpret_cast<Misc *>(smem + Sm::kEnd);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool issuer = warp == kIssuerWarp;

    if (p.segments == 1) after_previous();
    let_next_begin();
    const Unit u = unit_of(p);
    const int b = u.b, g = u.g, h0 = u.h0, seg = u.seg, t_lo = u.t_lo, live = u.live, tiles = u.tiles;
    const bool one = u.one, both = u.both;

    if (p.clear && blockIdx.x == 0 && tid == 0) *p.err = WsHeader{};  // a wait takes seconds to give up
    if (smem_u32(smem) & 1023u) {  // the tile layout needs 1 KiB alignment
        if (tid == 0) set_error(p.err, 399, smem_u32(smem));
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < kNumBars; ++i) {
            const bool two = (i >= bStep && i <= bTot1) || (!Sm::kApart && i < bLdB);
            mbar_init(&ms->bar[i], (i >= bEpE && i <= bEpY1) ? kEpiWarps : two ? 2 : 1);
        }
        ms->abort_flag = 0;
        ms->odd[0] = ms->odd[1] = ms->odd[2] = 0;
        ms->b = b; ms->h0 = h0; ms->seg = seg; ms->both = both;
        fence_mbar_init();
    }
    if (tid < 3 * (kTile / 4)) ms->first[tid / (kTile / 4)][tid % (kTile / 4)] = ~0u;
    if (issuer) {
        tmem_alloc(&ms->tmem_base, 512);
        tmem_relinquish();
        if (lane == 0) {
            prefetch_tmap(&tm_x); prefetch_tmap(&tm_b);
            prefetch_tmap(&tm_c); prefetch_tmap(&tm_y);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = ms->tmem_base;

    if (issuer) {
        if (lane == 0) {
            const uint32_t sb4 = smem_u32(smem) >> 4;
            auto lk = [&](uint32_t off) { return sb4 + (off >> 4) + kLboK; };
            auto lm = [&](uint32_t off) { return sb4 + (off >> 4) + kLboMN; };
            auto load_bc = [&](const CUtensorMap *map, int j, uint32_t to, uint64_t *bar) {
                for (int i = 0; i < kN / 64; ++i)
                    tma_load_4d(smem + to + i * kBlockBytes, map, bar, 64 * i, g, t_lo + j * kTile, b);
            };
            auto expect = [&](int bar, uint32_t bytes) {
                mbar_arrive_expect_tx(&ms->bar[bar], bytes);
                return &ms->bar[bar];
            };
            auto scores = [&](int buf, int cb) {  // with H before the tile in its slot and TMEM
                tc_fence_after();
                mma_ss<128, false, false, kN / 16>(tb + kTY + 128 * buf, lk(Sm::C(cb)), lk(Sm::kH), 0u);  // C H
                umma_commit(&ms->bar[bEvY2]);
                mma_ss<128, false, false, kN / 16>(tb + kTS, lk(Sm::C(cb)), lk(Sm::B(buf)), 0u);  // S = C B^T
                umma_commit(&ms->bar[bEvS]);
            };
            auto update = [&](int buf) {
                tc_fence_after();
                mma_ss<kN, true, true, 8>(tb + kTH, lm(Sm::kHi), lm(Sm::B(buf)), 1u);  // H^T += (w X)^T B
                mma_ss<kN, true, true, 8>(tb + kTH, lm(Sm::lo(buf)), lm(Sm::B(buf)), 1u);
                umma_commit(&ms->bar[bEvU]);
            };
            auto output = [&](int buf, int xb) {  // Y += W X
                tc_fence_after();
                const uint32_t y = tb + kTY + 128 * buf;
                if (one) {
                    mma_ts<128>(y, tb + kTS, lm(Sm::X(xb)));
                } else {
                    mma_ts<64>(y, tb + kTS, lm(Sm::X(xb)));
                    mma_ts<64>(y + 64, tb + kTS + 8, lm(Sm::X(xb) + kBlockBytes));
                }
                umma_commit(&ms->bar[bEvY1]);
            };
            bool ok = true;
            int bs = 0, cs = 0;  // tiles whose copies of B, C were issued (N = 128: of both, bs)
            if constexpr (Sm::kApart) {
                auto next_b = [&]() { load_bc(&tm_b, bs, Sm::B(bs & 1), expect(bLdB + (bs & 1), Sm::kOperand)); ++bs; };
                auto next_c = [&]() { load_bc(&tm_c, cs, Sm::C(0), expect(bLdC, Sm::kOperand)); ++cs; };
                if (tiles > 0) { next_c(); next_b(); }
                if (tiles > 1) next_b();
                for (int j = 0; j < tiles; ++j) {
                    const int buf = j & 1, par = j & 1, xb = j % Sm::kXs;
                    if (!(ok = bar_wait(ms, bLdC, par, p) && bar_wait(ms, bLdB + buf, (j >> 1) & 1, p))) break;
                    if (!(ok = bar_wait(ms, bEpE, par, p))) break;
                    scores(buf, 0);
                    if (j > 0 && bs < tiles) next_b();  // the previous tile's (w X)^T B is done
                    if (!(ok = bar_wait(ms, bLdX + xb, (j / Sm::kXs) & 1, p) && bar_wait(ms, bEpX, par, p))) break;
                    update(buf);
                    if (cs < tiles) {
                        if (!(ok = bar_wait(ms, bEvS, par, p))) break;
                        next_c();
                    }
                    if (!(ok = bar_wait(ms, bEpW, par, p))) break;
                    output(buf, xb);
                }
            } else {
                auto next = [&]() {
                    uint64_t *bar = expect(bLdX + (bs & 1), 2 * Sm::kOperand);  // (X is the storing warp's)
                    load_bc(&tm_b, bs, Sm::B(bs & 1), bar);
                    load_bc(&tm_c, bs, Sm::C(bs & 1), bar);
                    ++bs;
                };
                while (bs < 2 && bs < tiles) next();
                ok = tiles == 0 || bar_wait(ms, bLdX, 0, p);
                for (int j = 0; ok && j < tiles; ++j) {
                    const int buf = j & 1, par = j & 1;
                    if (!(ok = bar_wait(ms, bEpE, par, p))) break;
                    scores(buf, buf);
                    if (j > 0 && bs < tiles) next();  // the previous tile's (w X)^T B is done
                    if (!(ok = bar_wait(ms, bEpX, par, p))) break;
                    update(buf);
                    if (!(ok = bar_wait(ms, bEpW, par, p))) break;
                    output(buf, buf);
                    if (j + 1 < tiles) ok = bar_wait(ms, bLdX + (buf ^ 1), ((j + 1) >> 1) & 1, p);
                }
            }
            // copies and MMAs in flight finish (bounded) before shared memory and TMEM are released: where a wait gave
            // up, here or in the epilogue, nothing else has waited for them
            if (!ok) {
                for (int j = max(bs - 2, 0); j < bs; ++j)
                    mbar_wait(&ms->bar[(Sm::kApart ? bLdB : bLdX) + (j & 1)], (j >> 1) & 1, kBarWaitNs);
                if (cs > 0) mbar_wait(&ms->bar[bLdC], (cs - 1) & 1, kBarWaitNs);
            }
            umma_commit(&ms->bar[bTear]);
            mbar_wait(&ms->bar[bTear], 0, kBarWaitNs);
        }
        __syncwarp();
    } else if (warp == kStoreWarp) {
        if (lane == 0) {
            // X's slots are this warp's: a tile's output leaves from one, and then the next X that goes there
            // is sent for
            int xs = 0, j = 0;
            auto next_x = [&]() {
                const int st = xs % Sm::kXs, t = t_lo + xs * kTile;
                uint64_t *bar = &ms->bar[bLdX + st];
                mbar_arrive_expect_tx(bar, kTileBytes);
                // a second head that the group does not have: the first one again, its result unused
                tma_load_4d(smem + Sm::X(st), &tm_x, bar, 0, h0, t, b);
                tma_load_4d(smem + Sm::X(st) + kBlockBytes, &tm_x, bar, one ? 64 : 0, one || !both ? h0 : h0 + 1, t, b);
                ++xs;
            };
            while (xs < Sm::kXs && xs < tiles) next_x();
            for (; j < tiles; ++j) {
                const int st = j % Sm::kXs, t0 = t_lo + j * kTile;
                uint8_t *from = smem + Sm::X(st);
                if (!bar_wait(ms, bEpY0 + (j & 1), (j >> 1) & 1, p)) break;
                const int gave_up = *(volatile int *)&ms->abort_flag, odd = *(volatile int *)&ms->odd[st];
                if (gave_up | odd) {
                    // where a wait of any role gave up, the epilogue no longer waits for X: it may not have landed
                    if (gave_up) break;
                    // columns whose X was taken out, from its token on
                    put_nan(from, reinterpret_cast<uint8_t *>(ms->first[st]), min(kTile, live - t0));
                    ms->odd[st] = 0;
                    fence_async_smem();
                }
                tma_store_4d(&tm_y, from, 0, h0, t0, b);
                if (both) tma_store_4d(&tm_y, from + kBlockBytes, one ? 64 : 0, one ? h0 : h0 + 1, t0, b);
                tma_store_commit();
                tma_store_wait_read();
                if (xs < tiles) next_x();
            }
            // (where a wait gave up) copies in flight finish, or a time limit, before shared memory is released
            for (; j < tiles && j < xs; ++j) mbar_wait(&ms->bar[bLdX + j % Sm::kXs], (j / Sm::kXs) & 1, kBarWaitNs);
            tma_store_wait_all();
        }
        __syncwarp();
    } else if (warp >= kStepWarp) {
        // steps and decays of a tile's tokens for half e, four consecutive tokens a lane
        const int e = warp - kStepWarp, head = one || !e || !both ? h0 : h0 + 1;
        const float da = p.a[head] * kLog2e, bias = p.delta_bias ? p.delta_bias[head] : 0.f;
        const __nv_bfloat16 *raw = p.delta + (long long)b * p.n * p.delta_stride + head;
        __nv_bfloat16 next[4];
        auto fetch = [&](int j) {  // rows that do not count: the last one that does, not used
#pragma unroll
            for (int i = 0; i < 4; ++i)
                next[i] = raw[(long long)min(t_lo + j * kTile + 4 * lane + i, live - 1) * p.delta_stride];
        };
        if (tiles > 0) fetch(0);
        for (int j = 0; j < tiles; ++j) {
            float4 up, cf;
            block_decays(next, live - (t_lo + j * kTile + 4 * lane), da, bias, p.softplus, up, cf);
            fetch(j + 1);
            if ((lane & 7) == 7) ms->tot[j & 1][e][lane >> 3] = up.w;
            __syncwarp();
            if (lane == 0) mbar_arrive(&ms->bar[bTot0 + (j & 1)]);
            // every epilogue warp has done with the previous tile's decays (the lanes leave together, if one gave up)
            if (j > 0 && !__all_sync(0xffffffffu, bar_wait(ms, bEpW, (j - 1) & 1, p))) break;
            *reinterpret_cast<float4 *>(&ms->cum[e][4 * lane]) = up;
            *reinterpret_cast<float4 *>(&ms->cf[e][4 * lane]) = cf;
            __syncwarp();
            if (lane == 0) mbar_arrive(&ms->bar[bStep]);
        }
    } else {
        // ============================ epilogue ============================
        const int qd = warp & 3, cq = warp >> 2;
        const int r = 32 * qd + lane, c0 = 32 * cq;
        const uint32_t lane_base = (uint32_t)(32 * qd) << 16;
        const int hs = cq >> 1;                     // which half of the columns
        constexpr int kS = kN / 4;                  // as rows of H^T (its TMEM lanes): column r, states s0 ..
        const int s0 = cq * kS;
        const int dhead = one || !hs || !both ? h0 : h0 + 1;  // a second head that is not there: the first
        const float skip = p.skip ? p.skip[dhead] : 0.f;
        // this thread's first state within [B, H, segs, N, P], the others P apart; null where it has none
        auto state_at = [&](float *base, int segs, int seg_i) -> float * {
            const volatile Misc *m = ms;
            const int half = p.P == 128 ? 0 : qd >> 1, col = r - 64 * half;
            if (!base || col >= p.P || (half && !m->both)) return nullptr;
            const long long bh = (long long)m->b * p.H + m->h0 + half;
            return base + ((bh * segs + seg_i) * p.N + s0) * p.P + col;
        };
        const uint32_t h_at = tb + lane_base + kTH + s0;
        // decay of the tile's blocks before / after this token's, and (for H^T's row) of the whole tile
        float before = 0.f, later = 0.f, total = 0.f;
        auto decays = [&](int j) {
            bar_wait(ms, bTot0 + (j & 1), (j >> 1) & 1, p);
            const float *tot = ms->tot[j & 1][hs];
            before = later = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (q < qd) before += tot[q];
                if (q > qd) later += tot[q];
            }
            const float *all = ms->tot[j & 1][qd >> 1];
            total = (all[0] + all[1]) + (all[2] + all[3]);
        };
        // the state before a tile: its bf16 copy to EH, handed over at once, and times the tile's decay to
        // TMEM, which is read only after the hand-over of w X
        auto put_state = [&](float (&v)[kS]) {
#pragma unroll
            for (int i = 0; i < kS; i += 8)
                *reinterpret_cast<uint4 *>(smem + Sm::kH + tile_off(r, s0 + i)) =
                    make_uint4(pack_bf16x2(v[i], v[i + 1]), pack_bf16x2(v[i + 2], v[i + 3]),
                               pack_bf16x2(v[i + 4], v[i + 5]), pack_bf16x2(v[i + 6], v[i + 7]));
            fence_async_smem();
            epi_arrive(ms, bEpE);
            const float keep = ex2(total);
            uint32_t u[kS];
#pragma unroll
            for (int i = 0; i < kS; ++i) u[i] = __float_as_uint(v[i] * keep);
            if constexpr (kS == 32) tmem_st32(h_at, u); else tmem_st16(h_at, u);
        };
        if (p.segments > 1) after_previous();  // (nothing is written before this by any role)
        // state 0: from state_in or the segment's chained state
        const float *from = p.segments > 1 ? state_at(p.seg_state, p.segments, seg)
                                           : state_at(const_cast<float *>(p.state_in), 1, 0);
        if (tiles > 0) {
            decays(0);
            float v[kS];
#pragma unroll
            for (int i = 0; i < kS; ++i) v[i] = from && s0 + i < p.N ? from[(size_t)i * p.P] : 0.f;
            put_state(v);
        }

        // waits for tile j's copies; tokens that do not count: zero rows of X and B, whatever was read
        auto landed = [&](int j) {
            const int xb = j % Sm::kXs, buf = j & 1, t0 = t_lo + j * kTile;
            bar_wait(ms, bLdX + xb, (j / Sm::kXs) & 1, p);
            if (t0 + kTile > live) {
                if (Sm::kApart) bar_wait(ms, bLdB + buf, (j >> 1) & 1, p);
                if (t0 + r >= live) {
                    const uint4 z = make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        *reinterpret_cast<uint4 *>(smem + Sm::X(xb) + tile_off(r, c0 + i)) = z;
                        if (kN == 128 || cq < 2) *reinterpret_cast<uint4 *>(smem + Sm::B(buf) + tile_off(r, c0 + i)) = z;
                    }
                }
                fence_async_smem();
            }
        };

        // W = S . decay of tile j, packed bf16 in S's place: this thread's 32 columns of both halves.  A
        // step of 16 columns turns into 8 words of the first half's W and 8 of the second's.
        auto weights = [&](int j) {
            const uint32_t sw = tb + lane_base + kTS + c0;
            // a row's factor: the decay from the end of the columns' block to the token.  In the diagonal
            // block that is the inverse of the decay still to come, finite unless the block decays by
            // more than 2^-kFactored; then every pair takes its own exponential.
            float rf[2];
            bool factored = true;
            if (cq <= qd) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float *tot = ms->tot[j & 1][e];
                    const float own = tot[qd];
                    float x = ms->cum[e][r] - (cq == qd ? own : 0.f);
                    if (cq < 1 && qd > 1) x += tot[1];
                    if (cq < 2 && qd > 2) x += tot[2];
                    rf[e] = ex2(x);
                    if (cq == qd && !(fabsf(own) <= kFactored)) factored = false;
                }
            }
            bar_wait(ms, bEvS, j & 1, p);
            tc_fence_after();
            if (cq > qd) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = 0u;
                tmem_st16(sw, w);
                tmem_st16(sw + 16, w);
            } else if (factored) {
                const uint64_t rf0 = pair(rf[0], rf[0]), rf1 = pair(rf[1], rf[1]);
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    uint32_t sv[16], w[8];
                    tmem_ld16(sw + 16 * o, sv);
                    tmem_ld_wait();
                    if (cq == qd) {  // above the diagonal: zero
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (16 * o + i > lane) sv[i] = 0u;
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (e == 1 && one) break;
                        const ulonglong2 *cf = reinterpret_cast<const ulonglong2 *>(&ms->cf[e][c0 + 16 * o]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const ulonglong2 f = cf[i];
                            w[2 * i] = bf16_of(mul2(pair(sv[4 * i], sv[4 * i + 1]), mul2(e ? rf1 : rf0, f.x)));
                            w[2 * i + 1] = bf16_of(mul2(pair(sv[4 * i + 2], sv[4 * i + 3]), mul2(e ? rf1 : rf0, f.y)));
                        }
                        tmem_st8(sw + 16 * o + 8 * e, w);
                    }
                }
            } else {
                // from the diagonal to the left: the exponents grow by one token's decay a column, so that what is
                // near a token does not come from a difference of what a strong decay made large (or infinite)
                const volatile Misc *m = ms;
                const int tc = t_lo + j * kTile + c0 + lane;  // this lane's column
                float x0 = 0.f, x1 = 0.f;
#pragma unroll
                for (int o = 1; o >= 0; --o) {
                    uint32_t sv[16], w[8];
                    tmem_ld16(sw + 16 * o, sv);
                    tmem_ld_wait();
#pragma unroll 1
                    for (int e = 0; e < 2; ++e) {
                        const int he = m->h0 + (e && m->both && !one ? 1 : 0);
                        float dc = 0.f;  // its step
                        if (tc < live) {
                            dc = to_f32(p.delta[((long long)m->b * p.n + tc) * p.delta_stride + he]) +
                                 (p.delta_bias ? p.delta_bias[he] : 0.f);
                            dc = p.softplus ? softplus(dc) : dc;
                        }
                        const float da = p.a[he] * kLog2e;
                        float x = e ? x1 : x0;
#pragma unroll
                        for (int i = 7; i >= 0; --i) {
                            const int c = 16 * o + 2 * i;
                            const float d0 = __shfl_sync(0xffffffffu, dc, c), d1 = __shfl_sync(0xffffffffu, dc, c + 1);
                            const float w1 = c + 1 <= lane ? ex2(x) * d1 : 0.f;
                            x += c + 1 <= lane ? da * d1 : 0.f;
                            const float w0 = c <= lane ? ex2(x) * d0 : 0.f;
                            x += c <= lane ? da * d0 : 0.f;
                            w[i] = pack_bf16x2(c <= lane ? __uint_as_float(sv[2 * i]) * w0 : 0.f,
                                               c + 1 <= lane ? __uint_as_float(sv[2 * i + 1]) * w1 : 0.f);
                        }
                        (e ? x1 : x0) = x;
                        tmem_st8(sw + 16 * o + 8 * e, w);
                    }
                }
            }
            tmem_st_wait();
            epi_arrive(ms, bEpW);
        };
        // W X multiplies a token's X by weights of zero for the tokens before it: a value that is not finite would
        // make their outputs NaN.  It is taken out of X, once w X has it, and the storing warp makes the outputs from
        // its token on NaN.
        // (a) w X of tile j -> hi, lo
        float yf = 0.f;  // decay of the tile up to this token
        auto split = [&](int j) {
            bar_wait(ms, bStep, j & 1, p);
            const float wr = ms->cf[hs][r] * ex2(later);
            yf = ex2(before + ms->cum[hs][r]);
            landed(j);
            uint32_t odd = 0u;
            if constexpr (Sm::kApart) {
                odd = split_row(smem + Sm::X(j % Sm::kXs), smem + Sm::kHi, smem + Sm::lo(j), r, c0, wr);
            } else {  // in registers until their slots are free
                const Weight w(wr);
                uint4 hi[4], lo[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) split8(smem + Sm::X(j & 1), r, c0 + 8 * i, w, hi[i], lo[i], odd);
                bar_wait(ms, bEvY2, j & 1, p);  // C H has read H, where hi goes,
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(smem + Sm::kHi + tile_off(r, c0 + 8 * i)) = hi[i];
                bar_wait(ms, bEvS, j & 1, p);  // and C B^T has read C, where lo goes
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(smem + Sm::lo(j) + tile_off(r, c0 + 8 * i)) = lo[i];
                tc_fence_after();
            }
            if ((odd & 0x7f80u) == 0x7f80u || (odd & 0x7f800000u) == 0x7f800000u)
                take_out(smem + Sm::X(j % Sm::kXs), r, c0, ms->first[j % Sm::kXs], &ms->odd[j % Sm::kXs]);
            __syncwarp();
            fence_async_smem();
            tmem_st_wait();  // (H times the tile's decay)
            epi_arrive(ms, bEpX);
        };
        if (Sm::kApart && tiles > 0) split(0);
        for (int j = 0; j < tiles; ++j) {
            const int buf = j & 1, par = j & 1, t0 = t_lo + j * kTile;
            uint8_t *xs = smem + Sm::X(j % Sm::kXs);
            const bool in = t0 + r < live;
            if (!Sm::kApart) split(j);
            // (b) C H times the decay up to each token, and W, while the tensor cores run B^T (w X)
            const uint32_t y_at = tb + lane_base + kTY + 128 * buf + c0;
            if (Sm::kApart) {
                bar_wait(ms, bEvY2, par, p);
                tc_fence_after();
            }
            {
                const uint64_t yf2 = pair(yf, yf);
#pragma unroll
                for (int c = 0; c < 32; c += 16) {
                    uint32_t y[16];
                    tmem_ld16(y_at + c, y);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        float a, b2;
                        unpair(mul2(yf2, pair(y[e], y[e + 1])), a, b2);
                        y[e] = __float_as_uint(a);
                        y[e + 1] = __float_as_uint(b2);
                    }
                    tmem_st16(y_at + c, y);
                }
            }
            weights(j);
            // (c) the state after the tile, while they run W X
            bar_wait(ms, bEvU, par, p);
            tc_fence_after();
            if (j + 1 < tiles) {
                decays(j + 1);
                float v[kS];
                uint32_t u[kS];
                if constexpr (kS == 32) tmem_ld32(h_at, u); else tmem_ld16(h_at, u);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < kS; ++i) v[i] = __uint_as_float(u[i]);
                put_state(v);
                if (Sm::kApart) split(j + 1);
            }
            // (d) Y -> bf16 in X's place -> TMA store
            bar_wait(ms, bEvY1, par, p);
            tc_fence_after();
            const uint64_t skip2 = pair(skip, skip);
#pragma unroll
            for (int c = 0; c < 32; c += 16) {
                uint32_t y[16], o[8];
                tmem_ld16(y_at + c, y);
                uint4 *at0 = reinterpret_cast<uint4 *>(xs + tile_off(r, c0 + c));
                uint4 *at1 = reinterpret_cast<uint4 *>(xs + tile_off(r, c0 + c + 8));
                const uint4 u0 = *at0, u1 = *at1;
                const uint32_t x[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = bf16_of(fma2(skip2, of_bf16(x[e]), pair(y[2 * e], y[2 * e + 1])));
                if (t0 + kTile > live && !in) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = 0u;
                }
                *at0 = make_uint4(o[0], o[1], o[2], o[3]);
                *at1 = make_uint4(o[4], o[5], o[6], o[7]);
            }
            fence_async_smem();
            epi_arrive(ms, bEpY0 + buf);
        }

        const volatile Misc *m = ms;
        const int hcol = one ? c0 : (cq & 1) * 32;
        const int head = m->h0 + (one ? 0 : hs);
        const int cols = p.P - hcol;  // columns of the head from this thread's first one on
        if (!hs || m->both) {  // the rest of the segment does not count: zeros
            const int end = min((m->seg + 1) * p.seg_tiles * kTile, p.n);
            for (int t = max(m->seg * p.seg_tiles * kTile, live) + r; t < end; t += kTile) {
                __nv_bfloat16 *row = p.y + ((long long)m->b * p.n + t) * p.y_stride + (long long)head * p.P + hcol;
#pragma unroll
                for (int i = 0; i < 32; i += 8)
                    if (i < cols) *reinterpret_cast<uint4 *>(row + i) = make_uint4(0, 0, 0, 0);
            }
        }
        float *to = m->seg == p.segments - 1 ? state_at(p.state_out, 1, 0) : nullptr;
#pragma unroll
        for (int o = 0; o < kS; o += 16) {
            uint32_t u[16];
            tmem_ld16(h_at + o, u);  // by whole warps, wherever the values go
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (!to || s0 + o + i >= p.N) continue;
                const size_t e = (size_t)(o + i) * p.P;
                to[e] = tiles > 0 ? __uint_as_float(u[i]) : from ? from[e] : 0.f;  // nothing counts: the state as it was
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (issuer) {
        tc_fence_after();
        tmem_dealloc(tb, 512);
    }
}

// rows [B, n] at a row stride, `heads` blocks of `inner` bf16 in each; boxes of 64 columns of one head x
// `rows` tokens, 128-byte swizzle, zero fill past a head's columns and past a sequence's n tokens
bool make_map(CUtensorMap *m, const void *base, int B, int n, int heads, int inner, long long stride, int rows = kTile) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[4] = {(cuuint64_t)inner, (cuuint64_t)heads, (cuuint64_t)n, (cuuint64_t)B};
    cuuint64_t strides[3] = {(cuuint64_t)inner * 2, (cuuint64_t)stride * 2, (cuuint64_t)stride * 2 * (cuuint64_t)n};
    cuuint32_t box[4] = {64, 1, (cuuint32_t)rows, 1};
    cuuint32_t es[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Cut {
    int per_group, units, segments, seg_tiles;
};

// Units of 128 columns, and segments: the number that gives the shortest chain of tiles over 152 SMs,
// where a segmented scan pays a state-only pass (about half a tile's work) on top
Cut cut(const Ssm &p) {
    Cut c{};
    const int group_heads = p.H / p.G;
    c.per_group = p.P == 128 ? group_heads : (group_heads + 1) / 2;
    c.units = p.B * p.G * c.per_group;
    const int tiles = (p.n + kTile - 1) / kTile;
    double best = 0;
    for (int s = 1; s <= tiles && s <= 152; ++s) {
        const int len = (tiles + s - 1) / s, segs = (tiles + len - 1) / len;
        const long long waves = ((long long)c.units * segs + 151) / 152;
        const double cost = waves * (len * (segs > 1 ? 1.5 : 1.0) + (segs > 1 ? 6.0 : 0.0));
        if (s == 1 || cost < best) {
            best = cost;
            c.segments = segs;
            c.seg_tiles = len;
        }
    }
    return c;
}

}  // namespace

size_t ssm_tc_workspace_floats(const Ssm &p) {
    if (p.n <= 0 || p.B <= 0) return 0;
    const Cut c = cut(p);
    return c.segments > 1 ? (size_t)p.B * p.H * c.segments * ((size_t)p.N * p.P + 1) : 0;
}

int ssm_tc_launches(const Ssm &p) { return cut(p).segments > 1 ? 3 : 1; }

bool ssm_tc_applicable(const Ssm &p) {
    if (getenv("HLA_DISABLE_FUSED")) return false;
    if (p.dt != HLA_BF16 || p.n <= 0 || p.B <= 0) return false;
    for (auto [ptr, stride] : {std::pair<const void *, long long>{p.x, p.x_stride}, {p.b, p.b_stride}, {p.c, p.c_stride},
                               {p.y, p.y_stride}})
        if (!rows_aligned(ptr, stride, 2, 16)) return false;
    int dev = 0, major = 0, minor = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
    cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev);
    return major == 10 && minor == 3 && encode_fn() != nullptr;
}

cudaError_t ssm_tc_launch(const Ssm &p, cudaStream_t stream) {
    CUtensorMap mx, mb, mc, my;
    const int x_rows = getenv("HLA_TEST_SHORT_COPY") ? kTile / 2 : kTile;  // testing: the waits for X run out
    if (!make_map(&mx, p.x, p.B, p.n, p.H, p.P, p.x_stride, x_rows) ||
        !make_map(&mb, p.b, p.B, p.n, p.G, p.N, p.b_stride) || !make_map(&mc, p.c, p.B, p.n, p.G, p.N, p.c_stride) ||
        !make_map(&my, p.y, p.B, p.n, p.H, p.P, p.y_stride))
        return cudaErrorInvalidValue;
    const Cut c = cut(p);
    Params q{};
    q.n = p.n; q.H = p.H; q.P = p.P; q.G = p.G; q.N = p.N; q.softplus = p.softplus;
    q.per_group = c.per_group; q.units = c.units; q.segments = c.segments; q.seg_tiles = c.seg_tiles;
    q.delta_stride = p.delta_stride; q.delta = static_cast<const __nv_bfloat16 *>(p.delta);
    q.y = static_cast<__nv_bfloat16 *>(p.y); q.y_stride = p.y_stride;
    q.a = p.a; q.skip = p.skip; q.delta_bias = p.delta_bias; q.lengths = p.lengths;
    q.state_in = p.state_in; q.state_out = p.state_out;
    q.seg_state = reinterpret_cast<float *>(p.ws + kWsHeaderBytes);
    q.seg_decay = q.seg_state + (size_t)p.B * p.H * c.segments * p.N * p.P;
    q.err = reinterpret_cast<WsHeader *>(p.ws);
    q.clear = 1;
    auto launch = [&](auto kern, int blocks, uint32_t smem) -> cudaError_t {
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e) return e;
        return launch_after(kern, blocks, kThreads, smem, stream, mx, mb, mc, my, q);
    };
    const bool wide = p.N == 128;
    if (c.segments > 1) {
        const int blocks = c.units * (c.segments - 1);
        auto run = [&](auto kern, uint32_t smem) -> cudaError_t {
            cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e) return e;
            return launch_after(kern, blocks, kStateThreads, smem, stream, mx, mb, q);
        };
        constexpr uint32_t kMisc = sizeof(StateMisc);
        cudaError_t e = wide ? run(ssm_state_kernel<128>, StateMap<128>::kEnd + kMisc)
                             : run(ssm_state_kernel<64>, StateMap<64>::kEnd + kMisc);
        if (e) return e;
        e = ssm_chain_launch(p.state_in, q.seg_state, q.seg_decay, (long long)p.B * p.H, p.N * p.P, c.segments, stream);
        if (e) return e;
        q.clear = 0;
    }
    const int blocks = c.units * c.segments;
    return wide ? launch(ssm_tc_kernel<128>, blocks, Map<128>::kBytes)
                : launch(ssm_tc_kernel<64>, blocks, Map<64>::kBytes);
}

}  // namespace hla
