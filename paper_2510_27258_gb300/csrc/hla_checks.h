// Argument checks that the entry points of hla_layer_api.cu and hla_block_api.cu share.
#pragma once

#include "hla_internal.h"

namespace hla {

inline bool aligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline size_t elem_bytes(hla_dtype dt) { return dt == HLA_BF16 ? 2 : 4; }

constexpr long long kMaxRows = (1LL << 31) - 1;
constexpr long long kMaxValues = 1LL << 40;
constexpr int kMaxChannels = (int)kMaxRows - 256;  // a block has up to 256: its last one is within 32 bits

#define HLA_TRY(expr)                       \
    do {                                    \
        const hla_status st_ = (expr);      \
        if (st_ != HLA_OK) return st_;      \
    } while (0)

inline hla_status check_type(hla_dtype dt) {
    return dt == HLA_F32 || dt == HLA_BF16 ? HLA_OK : fail(HLA_ERR_INVALID_ARGUMENT, "unknown dtype %d", (int)dt);
}

inline hla_status check_flag(int v, const char *name) {
    return v == 0 || v == 1 ? HLA_OK : fail(HLA_ERR_INVALID_ARGUMENT, "%s must be 0 or 1, got %d", name, v);
}

inline hla_status check_rows(int B, int n) {
    if (B < 0 || n < 0) return fail(HLA_ERR_INVALID_ARGUMENT, "negative size B=%d n=%d", B, n);
    return n <= (1 << 30) && (long long)B * n <= kMaxRows ? HLA_OK : fail(HLA_ERR_UNSUPPORTED, "problem too large");
}

// a strided token tensor: pointer (where there are rows), element alignment, row stride
inline hla_status check_tensor(const void *p, long long stride, long long width, hla_dtype dt, long long rows, const char *name) {
    if (rows > 0 && !p) return fail(HLA_ERR_INVALID_ARGUMENT, "null %s pointer", name);
    if (!aligned(p, elem_bytes(dt))) return fail(HLA_ERR_INVALID_ARGUMENT, "%s is not aligned to its elements", name);
    if (stride < width)
        return fail(HLA_ERR_INVALID_ARGUMENT, "%s: row stride %lld is below the row's %lld elements", name, stride, width);
    if (stride > kMaxValues || (rows > 0 && stride > kMaxValues / rows))
        return fail(HLA_ERR_UNSUPPORTED, "problem too large");
    return HLA_OK;
}

inline hla_status check_workspace(const void *ws, size_t bytes, size_t need) {
    if (!ws || bytes < need)
        return fail(HLA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, ws ? bytes : (size_t)0);
    if (!aligned(ws, 256)) return fail(HLA_ERR_INVALID_ARGUMENT, "workspace must be 256-byte aligned");
    return HLA_OK;
}

// one multiple of 16 bytes after the workspace header
inline size_t scratch_bytes(size_t floats) { return align_up(kWsHeaderBytes + floats * sizeof(float), 256); }

inline cudaStream_t as_stream(hla_stream_t s) { return reinterpret_cast<cudaStream_t>(s); }

inline hla_status clear_header(void *ws, cudaStream_t s) {
    return cuda_status(cudaMemsetAsync(ws, 0, kWsHeaderBytes, s), "clearing the workspace header");
}

}  // namespace hla
