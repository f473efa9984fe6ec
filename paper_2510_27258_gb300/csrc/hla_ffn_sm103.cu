// Gated feed-forward projections and their gradients on the tensor cores (bf16).
//
//   kOut   out = act(x Wg^T) (x Wu^T)
//   kGrad  dZ = [dout Zu act'(Zg) | dout act(Zg)], Z computed again, to the workspace in bf16
//   kBack  dx = dZg Wg + dZu Wu (one sum over both), and d[Wg; Wu] = dZ^T x: the tiles of both in one list, which
//          leaves fewer pairs without one at the end than two launches
//
// Each is a product D = A B^T over tiles of 256 x 256, made by a pair of blocks (tcgen05.mma of both their SMs, M = N =
// 256): a block loads 128 rows of A and 128 of B in steps of 64, 32 KB for 8.4 MFLOP of its half.  Where the sum's index is
// not the contiguous one (B of dx, both of dw) the operand is read as it lies (MN-major), so nothing is transposed in
// memory.  The forward's tile has 128 gate columns (the first block's half of B) and the same 128 up columns (the
// second's), so that activation and product happen where the tile is read out.
//
// A block has a loading warp, whose copies count at the first block's barriers, a warp that issues the products (first
// block) and four warps that read finished tiles out of tensor memory, whose 512 columns hold two of them, so that
// reading out is hidden behind the next tile.  Blocks stay for many tiles, which are taken in groups of eight columns so
// that a round of all blocks reads few distinct rows.  Where tiles are few and the sum long, the sum is cut and the
// parts are added in their order by another kernel.
//
// Bound by the tensor cores.  8192 x 2048 x 5632: forward 204 us in a capture of its own, 1.85 PFLOP/s, 97 % of what a
// library product reaches in a burst (225 to 233 us one after another, at the clocks that leaves); gradient 709 to 727 us,
// of which kBack 404 (97 %) and kGrad 223 (89 %), whose read-out of a tile (dout, two planes of dZ) takes as long as the
// products of the next.  dZ lies in bf16 between the products: the error of dx and dw against 64 bits is 0.0023 of their norm
// instead of the 0.0017 that their own rounding makes; fp32 would double its bytes, and the products read it twice.
// Up to 128 tokens, where the weights' bytes count, ffn_few_kernel: 16 tokens 8.6 us on the device where the weights' 46 MB are
// in L2, 11.3 us from memory (4.1 TB/s, 62 % of what a copy reaches).
//
// Every wait has a limit: it sets the workspace's error word and the block's `stop`, after which all roles leave,
// copies and products in flight are waited for (with a limit), and tensor memory is released.
#include <climits>

#include "hla_ffn.h"
#include "hla_vec.cuh"
#include "sm103_prims.cuh"
#include "tensor_map.h"

namespace hla {
namespace {

using namespace sm103;

constexpr int kTile = 256, kHalf = 128, kStep = 64;
constexpr int kThreads = 192;
constexpr uint32_t kHalfBytes = kHalf * kStep * 2, kStageBytes = 2 * kHalfBytes;
constexpr int kStages = 6;
constexpr uint32_t kPitch = 144;                         // a staged row of 128 bytes and what keeps banks apart
constexpr uint32_t kStagingBytes = 32 * kPitch;          // of a warp that reads out
constexpr uint32_t kSmemBytes = 1024 + kStages * kStageBytes + 4 * kStagingBytes + 256;
constexpr long long kWaitCycles = 4000000000ll, kLandCycles = 200000000ll;  // about 2 and 0.1 s

enum Mode { kOut, kGrad, kBack };

struct Work {
    int down, across, parts;   // tiles along A's and B's rows, cuts of the sum
    int steps, per_part;       // steps of the sum, and of a part
    int dw;                    // kBack: of dw, else of dx
    int plane_steps;           // dx: steps of one plane; dw: tiles of one plane
    int rows, cols;            // of the output (kOut, kGrad: cols = F; dw: rows = F, of each plane)
    int act;
    void *out;                 // bf16, or fp32 parts [part][rows][cols] (dw: [part][2][rows][cols]); kGrad: dZ
    long long out_row;         // elements
    long long out_plane;       // kGrad, dw: elements from one plane to the other
    int out_wide;              // whether rows of out allow 16-byte accesses
    const __nv_bfloat16 *dout;  // kGrad
    long long dout_row;
    int dout_wide;
};
struct Call {
    Work w[2];       // kBack: two lists of tiles, one behind the other
    int first, all;  // tiles of the first, of both
    WsHeader *header;
    int clear;       // the call's first product clears the header
};

struct Bars {
    uint64_t full[kStages], empty[kStages];
    uint64_t done[2], taken[2];  // a tile's sums are there, have been read
    uint64_t drain;
    uint32_t tmem;
    int stop;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the first block's barrier in the place of this one
__device__ __forceinline__ uint32_t of_first(uint64_t *bar) {
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(smem_u32(bar)));
    return at;
}
__device__ __forceinline__ void arrive_at(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// a copy into this block's shared memory whose bytes count at the first block's barrier
__device__ __forceinline__ void load_pair(void *dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}
// false: another role gave up, or this wait did
__device__ bool wait(uint64_t *bar, uint32_t parity, Bars *bars, WsHeader *header, unsigned where) {
    if (mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    while (true) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*reinterpret_cast<volatile int *>(&bars->stop)) return false;
        if (clock64() - t0 > kWaitCycles) {
            header->where = where;
            header->detail = blockIdx.x;
            header->error = kDevTimeout;
            *reinterpret_cast<volatile int *>(&bars->stop) = 1;
            return false;
        }
    }
}
// products in flight when a role gives up; not longer than the limit
__device__ void drain(uint64_t *bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity) && clock64() - t0 <= kWaitCycles) {
    }
}

__device__ __forceinline__ void umma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// an arrival at the same barrier of both blocks when the products issued so far are done
__device__ __forceinline__ void commit_pair(uint64_t *bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            smem_u32(bar)),
        "h"((uint16_t)3)
        : "memory");
}

__device__ __forceinline__ float act_of(int act, float v, float &slope) {
    if (act == HLA_LINEAR) {
        slope = 1.f;
        return v;
    }
    const float s = __fdividef(1.f, 1.f + __expf(-v));
    slope = act == HLA_SIGMOID ? s * (1.f - s) : s * (1.f + v * (1.f - s));
    return act == HLA_SIGMOID ? s : v * s;
}

struct Tile {
    int m, n, part;
};
// groups of eight columns; down within a group, a row's columns next to each other
__device__ __forceinline__ Tile tile_of(const Work &w, int i) {
    const int each = w.down * w.across, part = i / each;
    i -= part * each;
    const int group = i / (8 * w.down), first = group * 8, width = min(8, w.across - first);
    i -= group * 8 * w.down;
    const int m = i / width;
    return {m, first + i - m * width, part};
}

// 32 staged rows of kBytes to global memory, row by row: 16 bytes a lane, or an element, eight in flight
template <int kBytes, typename E>
__device__ __forceinline__ void store_rows(const char *staged, E *at, long long row, int rows, int cols, bool wide) {
    const int lane = threadIdx.x & 31;
    constexpr int kLanes = kBytes / 16, kEach = 16 / sizeof(E), kCols = kBytes / (int)sizeof(E);
    if (wide) {
        const int c = (lane % kLanes) * kEach;
#pragma unroll
        for (int r = lane / kLanes; r < 32; r += 32 / kLanes)
            if (r < rows && c < cols)
                *reinterpret_cast<uint4 *>(at + r * row + c) =
                    *reinterpret_cast<const uint4 *>(staged + r * kPitch + c * sizeof(E));
    } else {
#pragma unroll 1
        for (int i0 = lane; i0 < 32 * kCols; i0 += 256) {
            E v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = (i0 + 32 * j) / kCols, c = (i0 + 32 * j) % kCols;
                v[j] = *reinterpret_cast<const E *>(staged + r * kPitch + c * sizeof(E));
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = (i0 + 32 * j) / kCols, c = (i0 + 32 * j) % kCols;
                if (r < rows && c < cols) at[r * row + c] = v[j];
            }
        }
    }
}
// 32 rows of 32 elements from global memory, eight in flight (behind the last row or column: 0)
__device__ __forceinline__ void load_rows(char *staged, const __nv_bfloat16 *at, long long row, int rows, int cols) {
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int r0 = 0; r0 < 32; r0 += 8) {
        __nv_bfloat16 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = r0 + j < rows && lane < cols ? at[(r0 + j) * row + lane] : __float2bfloat16(0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) *reinterpret_cast<__nv_bfloat16 *>(staged + (r0 + j) * kPitch + lane * 2) = v[j];
    }
}

template <Mode kMode>
__global__ void __launch_bounds__(kThreads, 1)
ffn_tile_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_a1, const __grid_constant__ CUtensorMap map_b1,
                const __grid_constant__ Call call) {
    extern __shared__ char raw[];
    char *stages = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    char *staging = stages + kStages * kStageBytes;
    Bars *bars = reinterpret_cast<Bars *>(staging + 4 * kStagingBytes);
    static_assert(sizeof(Bars) <= 256, "the barriers' room");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int clusters = gridDim.x / 2, tiles = call.all;
    WsHeader *header = call.header;
    auto work_of = [&](int i) -> const Work & { return call.w[kMode == kBack && i >= call.first]; };
    auto place_of = [&](int i) { return tile_of(work_of(i), kMode == kBack && i >= call.first ? i - call.first : i); };
    if (threadIdx.x == 0) {
        prefetch_tmap(&map_a);
        prefetch_tmap(&map_b);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&bars->full[s], 1);
            mbar_init(&bars->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&bars->done[b], 1);
            mbar_init(&bars->taken[b], 8);
        }
        mbar_init(&bars->drain, 1);
        bars->stop = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars->tmem))
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_meet();
    tc_fence_after();
    let_next_begin();
    after_previous();
    if (call.clear && blockIdx.x == 0 && threadIdx.x == 0) *header = WsHeader{};  // (waits set it after seconds)
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&bars->tmem);

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 0, sent = 0;
            bool ok = true;
            for (int i = blockIdx.x / 2; i < tiles && ok; i += clusters) {
                const Work &w = work_of(i);
                const Tile t = place_of(i);
                const int k_lo = t.part * w.per_part, k_hi = min(w.steps, k_lo + w.per_part);
                for (int k = k_lo; k < k_hi; ++k) {
                    if (!wait(&bars->empty[s], phase ^ 1, bars, header, 1)) {
                        ok = false;
                        break;
                    }
                    char *a = stages + s * kStageBytes, *b = a + kHalfBytes;
                    const uint32_t bar = of_first(&bars->full[s]);
                    if (rank == 0) mbar_arrive_expect_tx(&bars->full[s], 2 * kStageBytes);
                    if (kMode == kOut || kMode == kGrad) {
                        load_pair(a, &map_a, bar, k * kStep, t.m * kTile + rank * kHalf, 0);
                        load_pair(b, &map_b, bar, k * kStep, t.n * kHalf, rank);
                    } else if (!w.dw) {
                        const CUtensorMap *ma = i < call.first ? &map_a : &map_a1, *mb = i < call.first ? &map_b : &map_b1;
                        const int plane = k >= w.plane_steps, at = (k - plane * w.plane_steps) * kStep;
                        load_pair(a, ma, bar, at, t.m * kTile + rank * kHalf, plane);
                        const int n = t.n * kTile + rank * kHalf;
                        load_pair(b, mb, bar, n, at, plane);
                        load_pair(b + kHalfBytes / 2, mb, bar, n + 64, at, plane);
                    } else {
                        const CUtensorMap *ma = i < call.first ? &map_a : &map_a1, *mb = i < call.first ? &map_b : &map_b1;
                        const int plane = t.m >= w.plane_steps, m = (t.m - plane * w.plane_steps) * kTile + rank * kHalf;
                        load_pair(a, ma, bar, m, k * kStep, plane);
                        load_pair(a + kHalfBytes / 2, ma, bar, m + 64, k * kStep, plane);
                        const int n = t.n * kTile + rank * kHalf;
                        load_pair(b, mb, bar, n, k * kStep, 0);
                        load_pair(b + kHalfBytes / 2, mb, bar, n + 64, k * kStep, 0);
                    }
                    ++sent;
                    if (++s == kStages) {
                        s = 0;
                        phase ^= 1;
                    }
                }
            }
            // Shared memory goes when the last products have read each stage and said so here.  Where a role gave up
            // there is no sign of a copy but its time: one that was sent lands within microseconds
            const long long t0 = clock64();
            for (uint32_t d = 0; ok && d < kStages && d < sent; ++d) {
                if (s == 0) phase ^= 1;
                s = s ? s - 1 : kStages - 1;
                ok = wait(&bars->empty[s], phase, bars, header, 4);
            }
            while (!ok && clock64() - t0 < kLandCycles) {
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            int s = 0, b = 0;
            uint32_t phase = 0, bphase = 0;
            bool ok = true;
            for (int i = blockIdx.x / 2; i < tiles && ok; i += clusters) {
                const Work &w = work_of(i);
                const Tile t = place_of(i);
                const int k_lo = t.part * w.per_part, k_hi = min(w.steps, k_lo + w.per_part);
                if (!wait(&bars->taken[b], bphase ^ 1, bars, header, 2)) break;
                tc_fence_after();
                // operands that are read against the sum's direction: 16 of its indices are 2048 bytes on, else 32
                const bool a_cross = kMode == kBack && w.dw;
                constexpr bool b_cross = kMode == kBack;
                const uint32_t idesc = idesc_bf16(256, 256, a_cross, b_cross), a_step = a_cross ? 2048 : 32,
                               a_lbo = a_cross ? kHalfBytes / 2 : 16;
                constexpr uint32_t b_step = b_cross ? 2048 : 32, b_lbo = b_cross ? kHalfBytes / 2 : 16;
                for (int k = k_lo; k < k_hi; ++k) {
                    if (!wait(&bars->full[s], phase, bars, header, 3)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t a = smem_u32(stages + s * kStageBytes), bb = a + kHalfBytes;
#pragma unroll
                    for (int kk = 0; kk < kStep / 16; ++kk) {
                        const uint64_t da = desc_sw128(a + kk * a_step, a_lbo, 1024);
                        const uint64_t db = desc_sw128(bb + kk * b_step, b_lbo, 1024);
                        umma_pair(tmem + b * 256, da, db, idesc, k > k_lo || kk > 0);
                    }
                    commit_pair(&bars->empty[s]);
                    if (++s == kStages) {
                        s = 0;
                        phase ^= 1;
                    }
                }
                commit_pair(&bars->done[b]);
                b ^= 1;
                if (b == 0) bphase ^= 1;
            }
            // products in flight read both blocks' shared memory and write their tensor memory
            asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                             smem_u32(&bars->drain))
                         : "memory");
            drain(&bars->drain, 0);
        }
        __syncwarp();
    } else {
        char *mine = staging + (warp - 2) * kStagingBytes;
        const int quarter = warp & 3;
        int b = 0;
        uint32_t bphase = 0;
        for (int i = blockIdx.x / 2; i < tiles; i += clusters) {
            const Work &w = work_of(i);
            const Tile t = place_of(i);
            // kGrad: a lane's part of dout's next 32 columns (four rows' 16 bytes, eight rows apart), the first before the
            // tile is there
            uint4 next[4] = {};
            auto fetch = [&](int c) {
                const int n0 = t.n * kHalf + c + lane % 4 * 8, m0 = t.m * kTile + rank * kHalf + quarter * 32 + lane / 4;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (m0 + 8 * j < w.rows && n0 < w.cols)
                        next[j] = *reinterpret_cast<const uint4 *>(w.dout + (m0 + 8 * j) * w.dout_row + n0);
            };
            if (kMode == kGrad && w.dout_wide) fetch(0);
            if (!__all_sync(0xffffffffu, wait(&bars->done[b], bphase, bars, header, 5))) break;
            tc_fence_after();
            const uint32_t from = taddr(tmem + b * 256, quarter * 32, 0);
            const bool dw = kMode == kBack && w.dw;
            const int plane = dw && t.m >= w.plane_steps;
            const int m0 = (t.m - plane * w.plane_steps) * kTile + rank * kHalf + quarter * 32;
            const int rows = w.rows - m0;  // (may be below 1)
            char *row = mine + lane * kPitch;
            if (kMode == kOut) {
#pragma unroll 1
                for (int c = 0; c < kHalf; c += 64) {
                    const int n0 = t.n * kHalf + c;
#pragma unroll
                    for (int h = 0; h < 64; h += 32) {
                        uint32_t g[32], u[32];
                        tmem_ld32(from + c + h, g);
                        tmem_ld32(from + kHalf + c + h, u);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 32; j += 8) {
                            uint32_t o[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float v[2], slope;
#pragma unroll
                                for (int q = 0; q < 2; ++q)
                                    v[q] = act_of(w.act, __uint_as_float(g[j + 2 * e + q]), slope) *
                                           __uint_as_float(u[j + 2 * e + q]);
                                o[e] = pack_bf16x2(v[0], v[1]);
                            }
                            *reinterpret_cast<uint4 *>(row + (h + j) * 2) = make_uint4(o[0], o[1], o[2], o[3]);
                        }
                    }
                    __syncwarp();
                    store_rows<128>(mine, static_cast<__nv_bfloat16 *>(w.out) + m0 * w.out_row + n0, w.out_row, rows,
                                    w.cols - n0, w.out_wide);
                    __syncwarp();
                }
            } else if (kMode == kGrad) {
#pragma unroll 1
                for (int c = 0; c < kHalf; c += 32) {
                    const int n0 = t.n * kHalf + c;
                    if (w.dout_wide) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            *reinterpret_cast<uint4 *>(mine + (lane / 4 + 8 * j) * kPitch + lane % 4 * 16) = next[j];
                        if (c + 32 < kHalf) fetch(c + 32);
                    } else {
                        load_rows(mine, w.dout + m0 * w.dout_row + n0, w.dout_row, rows, w.cols - n0);
                    }
                    __syncwarp();
                    uint32_t g[32], u[32];
                    tmem_ld32(from + c, g);
                    tmem_ld32(from + kHalf + c, u);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; j += 8) {
                        const uint4 d = *reinterpret_cast<const uint4 *>(row + j * 2);
                        const uint32_t dw[4] = {d.x, d.y, d.z, d.w};
                        uint32_t og[4], ou[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float d2[2] = {bf16_lo(dw[e]), bf16_hi(dw[e])};
                            float vg[2], vu[2];
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                float slope;
                                const float a = act_of(w.act, __uint_as_float(g[j + 2 * e + q]), slope);
                                vg[q] = d2[q] * __uint_as_float(u[j + 2 * e + q]) * slope;
                                vu[q] = d2[q] * a;
                            }
                            og[e] = pack_bf16x2(vg[0], vg[1]);
                            ou[e] = pack_bf16x2(vu[0], vu[1]);
                        }
                        *reinterpret_cast<uint4 *>(row + j * 2) = make_uint4(og[0], og[1], og[2], og[3]);
                        *reinterpret_cast<uint4 *>(row + 64 + j * 2) = make_uint4(ou[0], ou[1], ou[2], ou[3]);
                    }
                    __syncwarp();
                    __nv_bfloat16 *to = static_cast<__nv_bfloat16 *>(w.out) + m0 * w.out_row + n0;
                    // (dZ's rows are padded to 16 bytes: what is written behind the last column is not read)
                    const int cols = (w.cols - n0 + 7) & ~7;
                    store_rows<64>(mine, to, w.out_row, rows, cols, true);
                    store_rows<64>(mine + 64, to + w.out_plane, w.out_row, rows, cols, true);
                    __syncwarp();
                }
            } else if (w.parts == 1) {
#pragma unroll 1
                for (int c = 0; c < kTile; c += 64) {
                    const int n0 = t.n * kTile + c;
                    if (n0 >= w.cols) break;
#pragma unroll
                    for (int h = 0; h < 64; h += 32) {
                        uint32_t v[32];
                        tmem_ld32(from + c + h, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 32; j += 8)
                            *reinterpret_cast<uint4 *>(row + (h + j) * 2) = make_uint4(
                                pack_bf16x2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])),
                                pack_bf16x2(__uint_as_float(v[j + 2]), __uint_as_float(v[j + 3])),
                                pack_bf16x2(__uint_as_float(v[j + 4]), __uint_as_float(v[j + 5])),
                                pack_bf16x2(__uint_as_float(v[j + 6]), __uint_as_float(v[j + 7])));
                    }
                    __syncwarp();
                    __nv_bfloat16 *to = static_cast<__nv_bfloat16 *>(w.out) + plane * w.out_plane + m0 * w.out_row + n0;
                    store_rows<128>(mine, to, w.out_row, rows, w.cols - n0, w.out_wide);
                    __syncwarp();
                }
            } else {
                float *out = static_cast<float *>(w.out) +
                             ((long long)t.part * (dw ? 2 : 1) + plane) * w.rows * w.cols + (long long)m0 * w.cols;
#pragma unroll 1
                for (int c = 0; c < kTile; c += 32) {
                    const int n0 = t.n * kTile + c;
                    if (n0 >= w.cols) break;
                    uint32_t v[32];
                    tmem_ld32(from + c, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; j += 4)
                        *reinterpret_cast<uint4 *>(row + j * 4) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    __syncwarp();
                    store_rows<128>(mine, out + n0, w.cols, rows, w.cols - n0, w.cols % 4 == 0);
                    __syncwarp();
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at(of_first(&bars->taken[b]));
            b ^= 1;
            if (b == 0) bphase ^= 1;
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_meet();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// ------------------------------------------------------------------------------------------------
// few rows: the weights are the rows of the product, the tokens its columns
//
// With up to 128 tokens the weights' bytes are what counts.  A block reads 128 of their rows (64 gate and 64 up rows of
// the same features; for dx 128 columns, against the sum's direction) for all tokens, 16 to 128 columns of one
// product, so the products cost what the tokens need, and every SM streams weights: the sum is cut over the blocks of a
// cluster, whose parts meet in shared memory and are added in the blocks' order, each block finishing some of the tokens.
// The cuts are powers of two, so the SMs' shares are uneven: with F 5632 176 blocks, of which 24 SMs have two.
// ------------------------------------------------------------------------------------------------

constexpr int kFewMost = 128, kFewThreads = 192, kFewStages = 8;
constexpr uint32_t kFewABytes = 128 * kStep * 2;

struct Few {
    int cols, stages;   // tokens' columns in the product (a multiple of 16), stages of the ring
    int steps, per;     // steps of the sum, of a block
    int plane_steps;    // kBack: steps of one plane
    int tokens, width;  // rows of the output, and its columns (kOut, kGrad: F; kBack: K)
    int act;
    __nv_bfloat16 *out;
    long long out_row, out_plane;
    const __nv_bfloat16 *dout;
    long long dout_row;
    WsHeader *header;
    int clear;
};

struct FewBars {
    uint64_t full[kFewStages], empty[kFewStages], done;
    uint32_t tmem;
    int stop;
};

__device__ bool wait_few(uint64_t *bar, uint32_t parity, FewBars *bars, WsHeader *header, unsigned where) {
    if (mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    while (true) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*reinterpret_cast<volatile int *>(&bars->stop)) return false;
        if (clock64() - t0 > kWaitCycles) {
            header->where = where;
            header->detail = blockIdx.x;
            header->error = kDevTimeout;
            *reinterpret_cast<volatile int *>(&bars->stop) = 1;
            return false;
        }
    }
}

// kN values of the cluster's blocks' partial sums, added in the blocks' order
template <int kN>
__device__ __forceinline__ void add_blocks(const float *const (&mine)[kN], int S, float (&sum)[kN]) {
    if (S == 1) {
#pragma unroll
        for (int j = 0; j < kN; ++j) sum[j] = *mine[j];
        return;
    }
#pragma unroll
    for (int j = 0; j < kN; ++j) sum[j] = 0.f;
    for (int b = 0; b < S; b += 2) {  // (S is even)
        float v[2][kN];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                uint32_t at;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(mine[j])), "r"(b + q));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[q][j]) : "r"(at) : "memory");
            }
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int j = 0; j < kN; ++j) sum[j] += v[q][j];
    }
}

// grid: tiles of weights' rows x blocks of a cluster
template <Mode kMode>
__global__ void __launch_bounds__(kFewThreads)
ffn_few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_t, Few f, int S) {
    extern __shared__ char raw[];
    __shared__ FewBars bars_;
    FewBars *bars = &bars_;
    char *stages = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = S > 1 ? (int)cluster_rank() : 0, tile = blockIdx.x / S;
    const uint32_t stage_bytes = kFewABytes + f.cols * kStep * 2;
    const uint32_t tmem_cols = f.cols <= 32 ? 32 : f.cols <= 64 ? 64 : 128;
    const int k_lo = min(rank * f.per, f.steps), k_hi = min(k_lo + f.per, f.steps);
    if (threadIdx.x == 0) {
        prefetch_tmap(&map_w);
        prefetch_tmap(&map_t);
        for (int s = 0; s < f.stages; ++s) {
            mbar_init(&bars->full[s], 1);
            mbar_init(&bars->empty[s], 1);
        }
        mbar_init(&bars->done, 1);
        bars->stop = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(&bars->tmem, tmem_cols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    let_next_begin();
    after_previous();
    if (f.clear && blockIdx.x == 0 && threadIdx.x == 0) *f.header = WsHeader{};  // (waits set it after seconds)
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&bars->tmem);

    if (warp == 0 && lane == 0) {
        int s = 0;
        uint32_t phase = 0, sent = 0;
        bool ok = true;
        for (int k = k_lo; k < k_hi; ++k) {
            if (!wait_few(&bars->empty[s], phase ^ 1, bars, f.header, 11)) {
                ok = false;
                break;
            }
            char *a = stages + s * stage_bytes, *b = a + kFewABytes;
            uint64_t *bar = &bars->full[s];
            mbar_arrive_expect_tx(bar, stage_bytes);
            if (kMode == kBack) {
                const int plane = k >= f.plane_steps, at = (k - plane * f.plane_steps) * kStep;
                tma_load_3d(a, &map_w, bar, tile * 128, at, plane);
                tma_load_3d(a + kFewABytes / 2, &map_w, bar, tile * 128 + 64, at, plane);
                tma_load_3d(b, &map_t, bar, at, 0, plane);
            } else {
                tma_load_3d(a, &map_w, bar, k * kStep, tile * 64, 0);
                tma_load_3d(a + kFewABytes / 2, &map_w, bar, k * kStep, tile * 64, 1);
                tma_load_3d(b, &map_t, bar, k * kStep, 0, 0);
            }
            ++sent;
            if (++s == f.stages) {
                s = 0;
                phase ^= 1;
            }
        }
        // (where a role gave up: the copies in flight land before shared memory goes)
        const long long t0 = clock64();
        for (uint32_t d = 0; !ok && d < (uint32_t)f.stages && d < sent; ++d) {
            if (s == 0) phase ^= 1;
            s = s ? s - 1 : f.stages - 1;
            while (!mbar_try_wait(&bars->full[s], phase) && clock64() - t0 < kLandCycles) {
            }
        }
    } else if (warp == 1 && lane == 0) {
        const uint32_t idesc = idesc_bf16(128, f.cols, kMode == kBack, 0);
        int s = 0;
        uint32_t phase = 0;
        for (int k = k_lo; k < k_hi; ++k) {
            if (!wait_few(&bars->full[s], phase, bars, f.header, 12)) break;
            tc_fence_after();
            const uint32_t a = smem_u32(stages + s * stage_bytes), b = a + kFewABytes;
#pragma unroll
            for (int kk = 0; kk < kStep / 16; ++kk) {
                const uint64_t da = kMode == kBack ? desc_sw128(a + kk * 2048, kFewABytes / 2, 1024)
                                                   : desc_sw128(a + kk * 32, 16, 1024);
                umma_bf16(tmem, da, desc_sw128(b + kk * 32, 16, 1024), idesc, k > k_lo || kk > 0);
            }
            umma_commit(&bars->empty[s]);
            if (++s == f.stages) {
                s = 0;
                phase ^= 1;
            }
        }
        umma_commit(&bars->done);
    }
    __syncwarp();
    // every block's sums to its shared memory, [token][row]: the stages are free when the last product is done
    float *sums = reinterpret_cast<float *>(stages);
    const bool some = k_lo < k_hi;
    if (warp >= 2) {
        const int quarter = warp & 3, row = quarter * 32 + lane;
        if (__all_sync(0xffffffffu, wait_few(&bars->done, 0, bars, f.header, 13))) {
            tc_fence_after();
            for (int c = 0; c < f.cols; c += 16) {
                uint32_t v[16];
                tmem_ld16(taddr(tmem, quarter * 32, c), v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j) sums[(c + j) * 128 + row] = some ? __uint_as_float(v[j]) : 0.f;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (S > 1) cluster_meet();
    // the block's tokens, neighbouring threads a row's neighbours, four values of a thread in flight
    const int each = (f.tokens + S - 1) / S, lo = rank * each, hi = min(lo + each, f.tokens);
    constexpr int kPerToken = kMode == kBack ? 128 : 64, kFour = 4;
    const int n0 = tile * kPerToken, all = (hi - lo) * kPerToken;
    for (int i0 = threadIdx.x; i0 < all; i0 += kFewThreads * kFour) {
        const float *at[kFour], *at_up[kFour];
        float v[kFour], up[kFour], d[kFour];
        long long to[kFour];
        bool on[kFour];
#pragma unroll
        for (int j = 0; j < kFour; ++j) {
            const int i = min(i0 + j * kFewThreads, all - 1), token = lo + i / kPerToken, r = i % kPerToken;
            on[j] = i0 + j * kFewThreads < all && n0 + r < f.width;
            at[j] = sums + token * 128 + r;
            at_up[j] = at[j] + 64;
            to[j] = token * f.out_row + n0 + r;
            if (kMode == kGrad) d[j] = on[j] ? to_f32(f.dout[token * f.dout_row + n0 + r]) : 0.f;
        }
        add_blocks(at, S, v);
        if (kMode != kBack) add_blocks(at_up, S, up);
#pragma unroll
        for (int j = 0; j < kFour; ++j) {
            if (!on[j]) continue;
            if (kMode == kBack) {
                from_f32(f.out + to[j], v[j]);
                continue;
            }
            float slope;
            const float a = act_of(f.act, v[j], slope);
            if (kMode == kOut) {
                from_f32(f.out + to[j], a * up[j]);
            } else {
                from_f32(f.out + to[j], d[j] * up[j] * slope);
                from_f32(f.out + f.out_plane + to[j], d[j] * a);
            }
        }
    }
    if (S > 1) cluster_meet();  // the others have read this block's sums
    if (warp == 1) tmem_dealloc(tmem, tmem_cols);
}

// rows of K elements to rows of `stride` (a multiple of 8) elements
__global__ void __launch_bounds__(256) ffn_align_kernel(const __nv_bfloat16 *from, long long from_row, __nv_bfloat16 *to,
                                                       long long to_row, int rows, int K) {
    let_next_begin();
    after_previous();
    for (int r = blockIdx.x; r < rows; r += gridDim.x)
        for (int k = threadIdx.x; k < K; k += 256) to[r * to_row + k] = from[r * from_row + k];
}

// out = the sum of `parts` runs of rows x cols
__global__ void __launch_bounds__(256) ffn_parts_kernel(const float *from, int parts, long long rows, int cols,
                                                       __nv_bfloat16 *out, long long out_row) {
    let_next_begin();
    after_previous();
    const long long all = rows * cols;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        float sum = 0.f;
#pragma unroll 4
        for (int z = 0; z < parts; ++z) sum += from[z * all + i];
        const long long m = i / cols;
        from_f32(out + m * out_row + (i - m * cols), sum);
    }
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------

constexpr int kSMs = 152, kPairs = kSMs / 2;

int up8(int v) { return (v + 7) & ~7; }
int tiles_of(int v, int by) { return (v + by - 1) / by; }

// [planes][rows][cols] of bf16 with rows `row` and planes `plane` elements apart; a box of 64 columns and box_rows rows
cudaError_t map_of(CUtensorMap *map, const void *p, long long cols, long long rows, int planes, long long row,
                   long long plane, int box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)row * 2, (cuuint64_t)plane * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
    const CUresult r = encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), dims, strides, box, one,
                                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : r == CUDA_ERROR_NOT_SUPPORTED ? cudaErrorNotSupported : cudaErrorInvalidValue;
}

template <Mode kMode>
cudaError_t run(const CUtensorMap (&m)[4], Call &c, cudaStream_t s) {
    const cudaError_t e =
        cudaFuncSetAttribute(ffn_tile_kernel<kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e) return e;
    auto tiles = [](const Work &w) { return (long long)w.down * w.across * w.parts; };
    const long long all = tiles(c.w[0]) + (kMode == kBack ? tiles(c.w[1]) : 0);
    if (all > INT_MAX) return cudaErrorInvalidValue;
    c.first = (int)tiles(c.w[0]);
    c.all = (int)all;
    return launch_cluster_after(ffn_tile_kernel<kMode>, 2u * (unsigned)(all < kPairs ? all : kPairs), kThreads, 2,
                                kSmemBytes, s, m[0], m[1], m[2], m[3], c);
}

// Cuts of a sum of `steps`: as many as give every pair a tile, of eight steps or more
int cuts(long long tiles, int steps) {
    const long long by_pairs = kPairs / tiles, by_steps = steps / 8;
    const long long n = by_pairs < by_steps ? by_pairs : by_steps;
    return n < 1 ? 1 : (int)n;
}
struct Cut {
    int parts, per;
};
Cut cut(long long tiles, int steps) {
    const int per = tiles_of(steps, cuts(tiles, steps));
    return {tiles_of(steps, per), per};
}
Cut cut_dx(int M, int K, int F) { return cut((long long)tiles_of(M, kTile) * tiles_of(K, kTile), 2 * tiles_of(F, kStep)); }
Cut cut_dw(int M, int K, int F) { return cut(2LL * tiles_of(F, kTile) * tiles_of(K, kTile), tiles_of(M, kStep)); }

size_t up256(size_t v) { return align_up(v, 256); }
size_t aligned_bytes(int M, int K, int F) {  // x and w in aligned rows
    return up256((size_t)M * up8(K) * 2) + up256((size_t)2 * F * up8(K) * 2);
}

struct Operands {
    const __nv_bfloat16 *x, *w;
    long long x_row, w_row;
};
// x and w as the copies need them: where rows do not begin at 16 bytes, in the workspace (at `at`, moved on)
cudaError_t align_operands(const Ffn &p, char *&at, Operands &o, cudaStream_t s) {
    const int K8 = up8(p.K);
    o = {static_cast<const __nv_bfloat16 *>(p.x), static_cast<const __nv_bfloat16 *>(p.w), p.x_stride, p.K};
    if (p.M == 1) o.x_row = K8;  // (the only row's stride is not used)
    if (!rows_aligned(p.x, o.x_row, 2, 16)) {
        __nv_bfloat16 *to = reinterpret_cast<__nv_bfloat16 *>(at);
        const cudaError_t e = launch_after(ffn_align_kernel, p.M < 8 * kSMs ? p.M : 8 * kSMs, 256, 0, s, o.x, p.x_stride,
                                           to, (long long)K8, p.M, p.K);
        if (e) return e;
        o.x = to;
        o.x_row = K8;
    }
    at += up256((size_t)p.M * K8 * 2);
    if (!rows_aligned(p.w, o.w_row, 2, 16)) {
        __nv_bfloat16 *to = reinterpret_cast<__nv_bfloat16 *>(at);
        const cudaError_t e = launch_after(ffn_align_kernel, 2 * p.F < 8 * kSMs ? 2 * p.F : 8 * kSMs, 256, 0, s, o.w,
                                           (long long)p.K, to, (long long)K8, 2 * p.F, p.K);
        if (e) return e;
        o.w = to;
        o.w_row = K8;
    }
    at += up256((size_t)2 * p.F * K8 * 2);
    return cudaSuccess;
}

bool wide(const void *p, long long row, int cols) { return cols % 8 == 0 && rows_aligned(p, row, 2, 16); }

// Few rows: blocks of a cluster as many as fill two blocks an SM, each with four steps or more
template <Mode kMode>
cudaError_t run_few(const CUtensorMap &weights, const CUtensorMap &tokens, Few f, int tiles, cudaStream_t s) {
    const int bytes = (int)kFewABytes + f.cols * kStep * 2, sums = f.cols * 128 * 4;
    constexpr int kRoom = 100 * 1024;
    f.stages = kRoom / bytes < kFewStages ? kRoom / bytes : kFewStages;
    int S = 1;
    while (S < 8 && (long long)tiles * S * 2 <= 2 * kSMs && f.steps >= S * 2 * 4) S *= 2;
    f.per = tiles_of(f.steps, S);
    const int smem = 1024 + (f.stages * bytes > sums ? f.stages * bytes : sums);
    const cudaError_t e = allow_smem(ffn_few_kernel<kMode>, smem);
    if (e) return e;
    return launch_cluster_after(ffn_few_kernel<kMode>, (unsigned)((long long)tiles * S), kFewThreads, S, smem, s, weights,
                                tokens, f, S);
}

// Up to 128 tokens, where the tiles of 256 x 256 would leave pairs without one (16 x 2048 x 5632: 9 us on the device
// instead of 18, weights in L2; above, the tiles cost no more than the tokens' own products.  1 x 4096 x 14336 by the tiles:
// 74 us, where the weights' bytes take 35)
bool few(int M, int F) { return M <= kFewMost && tiles_of(F, kHalf) < kPairs; }
int few_cols(int M) { return (M + 15) / 16 * 16; }

// kOut and kGrad
template <Mode kMode>
cudaError_t forward_product(const Ffn &p, const Operands &o, Work w, cudaStream_t s) {
    CUtensorMap m[4];
    cudaError_t e;
    if (few(p.M, p.F)) {
        Few f{};
        f.cols = few_cols(p.M);
        f.steps = tiles_of(p.K, kStep);
        f.tokens = p.M;
        f.width = p.F;
        f.act = p.act;
        f.out = static_cast<__nv_bfloat16 *>(w.out);
        f.out_row = w.out_row;
        f.out_plane = w.out_plane;
        f.dout = w.dout;
        f.dout_row = w.dout_row;
        f.header = reinterpret_cast<WsHeader *>(p.ws);
        f.clear = 1;
        e = map_of(&m[0], o.w, p.K, p.F, 2, o.w_row, o.w_row * p.F, kStep);
        if (!e) e = map_of(&m[1], o.x, p.K, p.M, 1, o.x_row, o.x_row * p.M, f.cols);
        return e ? e : run_few<kMode>(m[0], m[1], f, tiles_of(p.F, 64), s);
    }
    e = map_of(&m[0], o.x, p.K, p.M, 1, o.x_row, o.x_row * p.M, kHalf);
    if (!e) e = map_of(&m[1], o.w, p.K, p.F, 2, o.w_row, o.w_row * p.F, kHalf);
    if (e) return e;
    m[2] = m[0];
    m[3] = m[1];
    w.down = tiles_of(p.M, kTile);
    w.across = tiles_of(p.F, kHalf);
    w.parts = 1;
    w.steps = w.per_part = tiles_of(p.K, kStep);
    w.rows = p.M;
    w.cols = p.F;
    w.act = p.act;
    Call c{{w, w}, 0, 0, reinterpret_cast<WsHeader *>(p.ws), 1};
    return run<kMode>(m, c, s);
}

cudaError_t add_parts(const float *from, int parts, long long rows, int cols, void *out, long long out_row,
                      cudaStream_t s) {
    const long long blocks = (rows * cols + 255) / 256;
    return launch_after(ffn_parts_kernel, (unsigned)(blocks < 16 * kSMs ? blocks : 16 * kSMs), 256, 0, s, from, parts, rows,
                        cols, static_cast<__nv_bfloat16 *>(out), out_row);
}

}  // namespace

size_t ffn_tc_forward_scratch_bytes(int M, int K, int F) { return aligned_bytes(M, K, F); }

size_t ffn_tc_backward_scratch_bytes(int M, int K, int F) {
    if (M == 0) return 0;
    const Cut dx = cut_dx(M, K, F), dw = cut_dw(M, K, F);
    return aligned_bytes(M, K, F) + up256((size_t)2 * M * up8(F) * 2) +
           (dx.parts > 1 ? up256(sizeof(float) * dx.parts * M * K) : 0) +
           (dw.parts > 1 ? up256(sizeof(float) * dw.parts * 2 * F * K) : 0);
}

cudaError_t ffn_tc_forward(const Ffn &p, cudaStream_t s) {
    char *at = p.ws + kWsHeaderBytes;
    Operands o;
    const cudaError_t e = align_operands(p, at, o, s);
    if (e) return e;
    Work w{};
    w.out = p.out;
    w.out_row = p.out_stride;
    w.out_wide = wide(p.out, p.out_stride, p.F);
    return forward_product<kOut>(p, o, w, s);
}

cudaError_t ffn_tc_backward(const FfnBwd &q, cudaStream_t s) {
    const Ffn &p = q.f;
    char *at = p.ws + kWsHeaderBytes;
    Operands o;
    cudaError_t e = align_operands(p, at, o, s);
    if (e) return e;
    const int F8 = up8(p.F);
    const long long dz_plane = (long long)p.M * F8;
    __nv_bfloat16 *dz = reinterpret_cast<__nv_bfloat16 *>(at);
    at += up256((size_t)2 * dz_plane * 2);
    {
        Work w{};
        w.out = dz;
        w.out_row = F8;
        w.out_plane = dz_plane;
        w.out_wide = 1;
        w.dout = static_cast<const __nv_bfloat16 *>(q.dout);
        w.dout_row = q.dout_stride;
        w.dout_wide = wide(q.dout, q.dout_stride, p.F);
        e = forward_product<kGrad>(p, o, w, s);
        if (e) return e;
    }
    const Cut dx_cut = cut_dx(p.M, p.K, p.F), dw_cut = cut_dw(p.M, p.K, p.F);
    float *dx_parts = reinterpret_cast<float *>(at);
    at += dx_cut.parts > 1 ? up256(sizeof(float) * dx_cut.parts * p.M * p.K) : 0;
    float *dw_parts = reinterpret_cast<float *>(at);
    Work dx{}, dw{};
    // dx: the sum runs over both planes of dZ and w
    dx.down = tiles_of(p.M, kTile);
    dx.across = tiles_of(p.K, kTile);
    dx.plane_steps = tiles_of(p.F, kStep);
    dx.steps = 2 * dx.plane_steps;
    dx.parts = dx_cut.parts;
    dx.per_part = dx_cut.per;
    dx.rows = p.M;
    dx.cols = p.K;
    dx.out = dx.parts > 1 ? dx_parts : q.dx;
    dx.out_row = q.dx_stride;
    dx.out_wide = wide(q.dx, q.dx_stride, p.K);
    // dw: tiles of either plane, the sum over tokens
    dw.dw = 1;
    dw.plane_steps = tiles_of(p.F, kTile);
    dw.down = 2 * dw.plane_steps;
    dw.across = dx.across;
    dw.steps = tiles_of(p.M, kStep);
    dw.parts = dw_cut.parts;
    dw.per_part = dw_cut.per;
    dw.rows = p.F;
    dw.cols = p.K;
    dw.out = dw.parts > 1 ? dw_parts : q.dw;
    dw.out_row = p.K;
    dw.out_plane = (long long)p.F * p.K;
    dw.out_wide = wide(q.dw, p.K, p.K);
    if (few(p.M, p.F)) {
        Few f{};
        f.cols = few_cols(p.M);
        f.plane_steps = dx.plane_steps;
        f.steps = dx.steps;
        f.tokens = p.M;
        f.width = p.K;
        f.out = static_cast<__nv_bfloat16 *>(q.dx);
        f.out_row = q.dx_stride;
        f.header = reinterpret_cast<WsHeader *>(p.ws);
        CUtensorMap m[4];
        e = map_of(&m[0], o.w, p.K, p.F, 2, o.w_row, o.w_row * p.F, kStep);
        if (!e) e = map_of(&m[1], dz, p.F, p.M, 2, F8, dz_plane, f.cols);
        if (!e) e = run_few<kBack>(m[0], m[1], f, tiles_of(p.K, 128), s);
        if (!e) e = map_of(&m[0], dz, p.F, p.M, 2, F8, dz_plane, kStep);
        if (!e) e = map_of(&m[1], o.x, p.K, p.M, 1, o.x_row, o.x_row * p.M, kStep);
        if (e) return e;
        m[2] = m[0];
        m[3] = m[1];
        dx.down = 0;
        Call c{{dw, dx}, 0, 0, f.header, 0};
        e = run<kBack>(m, c, s);
        return e || dw.parts == 1 ? e : add_parts(dw_parts, dw.parts, 2LL * p.F, p.K, q.dw, p.K, s);
    }
    // the list with the longer sums first
    const int at_dx = dw.per_part > dx.per_part, at_dw = 1 - at_dx;
    CUtensorMap m[4];
    e = map_of(&m[2 * at_dx], dz, p.F, p.M, 2, F8, dz_plane, kHalf);
    if (!e) e = map_of(&m[2 * at_dx + 1], o.w, p.K, p.F, 2, o.w_row, o.w_row * p.F, kStep);
    if (!e) e = map_of(&m[2 * at_dw], dz, p.F, p.M, 2, F8, dz_plane, kStep);
    if (!e) e = map_of(&m[2 * at_dw + 1], o.x, p.K, p.M, 1, o.x_row, o.x_row * p.M, kStep);
    if (e) return e;
    Call c{{at_dx ? dw : dx, at_dx ? dx : dw}, 0, 0, reinterpret_cast<WsHeader *>(p.ws), 0};
    e = run<kBack>(m, c, s);
    if (!e && dx.parts > 1) e = add_parts(dx_parts, dx.parts, p.M, p.K, q.dx, q.dx_stride, s);
    if (!e && dw.parts > 1) e = add_parts(dw_parts, dw.parts, 2LL * p.F, p.K, q.dw, p.K, s);
    return e;
}

}  // namespace hla
