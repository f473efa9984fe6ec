// C ABI of the operators around the mixers (convolution, selective scan, q/k norm with rotation):
// argument checks, workspace sizing, dispatch.  See include/hla.h for the contracts.
#include <cmath>

#include "hla_internal.h"

namespace hla {
namespace {

bool aligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
size_t elem_bytes(hla_dtype dt) { return dt == HLA_BF16 ? 2 : 4; }
bool size_ok(int v) { return v == 16 || v == 32 || v == 64 || v == 128; }

constexpr long long kMaxRows = (1LL << 31) - 1;
constexpr long long kMaxValues = 1LL << 40;
constexpr int kMaxChannels = (int)kMaxRows - 256;  // a block has up to 256: its last one is within 32 bits

#define HLA_TRY(expr)                       \
    do {                                    \
        const hla_status st_ = (expr);      \
        if (st_ != HLA_OK) return st_;      \
    } while (0)

hla_status check_type(hla_dtype dt) {
    return dt == HLA_F32 || dt == HLA_BF16 ? HLA_OK : fail(HLA_ERR_INVALID_ARGUMENT, "unknown dtype %d", (int)dt);
}

hla_status check_flag(int v, const char *name) {
    return v == 0 || v == 1 ? HLA_OK : fail(HLA_ERR_INVALID_ARGUMENT, "%s must be 0 or 1, got %d", name, v);
}

hla_status check_rows(int B, int n) {
    if (B < 0 || n < 0) return fail(HLA_ERR_INVALID_ARGUMENT, "negative size B=%d n=%d", B, n);
    return n <= (1 << 30) && (long long)B * n <= kMaxRows ? HLA_OK : fail(HLA_ERR_UNSUPPORTED, "problem too large");
}

// a strided token tensor: pointer (where there are rows), element alignment, row stride
hla_status check_tensor(const void *p, long long stride, long long width, hla_dtype dt, long long rows, const char *name) {
    if (rows > 0 && !p) return fail(HLA_ERR_INVALID_ARGUMENT, "null %s pointer", name);
    if (!aligned(p, elem_bytes(dt))) return fail(HLA_ERR_INVALID_ARGUMENT, "%s is not aligned to its elements", name);
    if (stride < width)
        return fail(HLA_ERR_INVALID_ARGUMENT, "%s: row stride %lld is below the row's %lld elements", name, stride, width);
    if (stride > kMaxValues || (rows > 0 && stride > kMaxValues / rows))
        return fail(HLA_ERR_UNSUPPORTED, "problem too large");
    return HLA_OK;
}

hla_status check_workspace(const void *ws, size_t bytes, size_t need) {
    if (!ws || bytes < need)
        return fail(HLA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, ws ? bytes : (size_t)0);
    if (!aligned(ws, 256)) return fail(HLA_ERR_INVALID_ARGUMENT, "workspace must be 256-byte aligned");
    return HLA_OK;
}

hla_status check_conv(const void *x, const void *w, const void *bias, hla_dtype dt, int B, int n, int C, int width,
                      long long x_stride, int silu, const int *lengths) {
    HLA_TRY(check_type(dt));
    HLA_TRY(check_rows(B, n));
    HLA_TRY(check_flag(silu, "silu"));
    if (C <= 0 || width <= 0) return fail(HLA_ERR_INVALID_ARGUMENT, "non-positive size C=%d width=%d", C, width);
    if (width < 2 || width > 4) return fail(HLA_ERR_UNSUPPORTED, "width=%d: supported widths are 2, 3, 4", width);
    if (C > kMaxChannels) return fail(HLA_ERR_UNSUPPORTED, "problem too large");
    // one launch covers B x token blocks x channel blocks
    if (((long long)n / 32 + 1) * B > kMaxRows / (C / 32 + 1)) return fail(HLA_ERR_UNSUPPORTED, "problem too large");
    HLA_TRY(check_tensor(x, x_stride, C, dt, (long long)B * n, "x"));
    if (B > 0 && !w) return fail(HLA_ERR_INVALID_ARGUMENT, "null w pointer");
    if (!aligned(w, elem_bytes(dt)) || !aligned(bias, elem_bytes(dt)) || !aligned(lengths, 4))
        return fail(HLA_ERR_INVALID_ARGUMENT, "w, bias and lengths must be aligned to their elements");
    return HLA_OK;
}

hla_status check_ssm(const Ssm &p, bool step) {
    HLA_TRY(check_type(p.dt));
    HLA_TRY(check_rows(p.B, p.n));
    HLA_TRY(check_flag(p.softplus, "softplus"));
    if (p.H <= 0 || p.G <= 0 || p.P <= 0 || p.N <= 0)
        return fail(HLA_ERR_INVALID_ARGUMENT, "non-positive size H=%d P=%d G=%d N=%d", p.H, p.P, p.G, p.N);
    if (p.H % p.G) return fail(HLA_ERR_INVALID_ARGUMENT, "H=%d is not a multiple of G=%d", p.H, p.G);
    if (!size_ok(p.P) || !size_ok(p.N))
        return fail(HLA_ERR_UNSUPPORTED, "P=%d N=%d: supported sizes are 16, 32, 64, 128", p.P, p.N);
    if ((long long)p.B * p.H > (1LL << 27)) return fail(HLA_ERR_UNSUPPORTED, "problem too large");
    const long long rows = (long long)p.B * p.n;
    HLA_TRY(check_tensor(p.x, p.x_stride, (long long)p.H * p.P, p.dt, rows, "x"));
    HLA_TRY(check_tensor(p.y, p.y_stride, (long long)p.H * p.P, p.dt, rows, "y"));
    HLA_TRY(check_tensor(p.delta, p.delta_stride, p.H, p.dt, rows, "delta"));
    HLA_TRY(check_tensor(p.b, p.b_stride, (long long)p.G * p.N, p.dt, rows, "b"));
    HLA_TRY(check_tensor(p.c, p.c_stride, (long long)p.G * p.N, p.dt, rows, "c"));
    if (rows > 0 && !p.a) return fail(HLA_ERR_INVALID_ARGUMENT, "null a pointer");
    if (!aligned(p.a, 4) || !aligned(p.skip, 4) || !aligned(p.delta_bias, 4) || !aligned(p.lengths, 4))
        return fail(HLA_ERR_INVALID_ARGUMENT, "a, skip, delta_bias and lengths must be 4-byte aligned");
    if (!aligned(p.state_in, 16) || !aligned(p.state_out, 16))
        return fail(HLA_ERR_INVALID_ARGUMENT, "states must be 16-byte aligned");
    if (step && p.B > 0 && !p.state_out) return fail(HLA_ERR_INVALID_ARGUMENT, "null state pointer");
    return HLA_OK;
}

hla_status check_qk(const QkNorm &p) {
    HLA_TRY(check_type(p.dt));
    HLA_TRY(check_rows(p.B, p.n));
    HLA_TRY(check_flag(p.interleaved, "interleaved"));
    if (p.H <= 0 || p.Hk <= 0 || p.d <= 0 || p.rot < 0)
        return fail(HLA_ERR_INVALID_ARGUMENT, "bad size H=%d Hk=%d d=%d rot=%d", p.H, p.Hk, p.d, p.rot);
    if (p.H % p.Hk) return fail(HLA_ERR_INVALID_ARGUMENT, "H=%d is not a multiple of Hk=%d", p.H, p.Hk);
    if (!std::isfinite(p.eps) || p.eps < 0.f) return fail(HLA_ERR_INVALID_ARGUMENT, "eps must be finite and not negative");
    if (p.rot > p.d) return fail(HLA_ERR_INVALID_ARGUMENT, "rot=%d is above d=%d", p.rot, p.d);
    if (!size_ok(p.d)) return fail(HLA_ERR_UNSUPPORTED, "d=%d: supported sizes are 16, 32, 64, 128", p.d);
    if (p.rot % 8) return fail(HLA_ERR_UNSUPPORTED, "rot=%d: supported are multiples of 8", p.rot);
    if (p.H > 65536) return fail(HLA_ERR_UNSUPPORTED, "H=%d: up to 65536 heads", p.H);
    const long long rows = (long long)p.B * p.n;
    HLA_TRY(check_tensor(p.q, p.q_stride, (long long)p.H * p.d, p.dt, rows, "q"));
    HLA_TRY(check_tensor(p.k, p.k_stride, (long long)p.Hk * p.d, p.dt, rows, "k"));
    if (!aligned(p.wq, elem_bytes(p.dt)) || !aligned(p.wk, elem_bytes(p.dt)) || !aligned(p.positions, 4))
        return fail(HLA_ERR_INVALID_ARGUMENT, "weights and positions must be aligned to their elements");
    if (p.rot > 0) {
        if (p.table_rows < 0) return fail(HLA_ERR_INVALID_ARGUMENT, "negative table_rows");
        if (rows > 0 && (!p.cos || !p.sin)) return fail(HLA_ERR_INVALID_ARGUMENT, "null cos or sin pointer");
        if (!aligned(p.cos, 16) || !aligned(p.sin, 16))
            return fail(HLA_ERR_INVALID_ARGUMENT, "cos and sin must be 16-byte aligned");
        if (!p.positions && rows > 0 && (p.pos0 < 0 || (long long)p.pos0 + p.n > p.table_rows))
            return fail(HLA_ERR_INVALID_ARGUMENT, "positions %d..%lld are outside the tables' %d rows", p.pos0,
                        (long long)p.pos0 + p.n - 1, p.table_rows);
    }
    return HLA_OK;
}

// one multiple of 16 bytes after the workspace header
size_t scratch_bytes(size_t floats) { return align_up(kWsHeaderBytes + floats * sizeof(float), 256); }

cudaStream_t as_stream(hla_stream_t s) { return reinterpret_cast<cudaStream_t>(s); }

hla_status clear_header(void *ws, cudaStream_t s) {
    return cuda_status(cudaMemsetAsync(ws, 0, kWsHeaderBytes, s), "clearing the workspace header");
}

}  // namespace
}  // namespace hla

using namespace hla;

extern "C" {

hla_status hla_conv_forward(const void *x, const void *w, const void *bias, void *out, hla_dtype dt, int B, int n,
                            int C, int width, long long x_stride, long long out_stride, int silu, const int *lengths,
                            const void *state_in, void *state_out, hla_stream_t stream) {
    clear_last_error();
    HLA_TRY(check_conv(x, w, bias, dt, B, n, C, width, x_stride, silu, lengths));
    HLA_TRY(check_tensor(out, out_stride, C, dt, (long long)B * n, "out"));
    if (!aligned(state_in, elem_bytes(dt)) || !aligned(state_out, elem_bytes(dt)))
        return fail(HLA_ERR_INVALID_ARGUMENT, "states must be aligned to their elements");
    if (B == 0 || (n == 0 && !state_out)) return HLA_OK;
    const Conv p{x, w, bias, out, dt, B, n, C, width, silu, x_stride, out_stride, lengths, state_in, state_out};
    return cuda_status(conv_forward_launch(p, as_stream(stream)), "convolution");
}

hla_status hla_conv_step(const void *x, const void *w, const void *bias, void *out, hla_dtype dt, int B, int C,
                         int width, long long x_stride, long long out_stride, int silu, void *state,
                         hla_stream_t stream) {
    clear_last_error();
    HLA_TRY(check_conv(x, w, bias, dt, B, 1, C, width, x_stride, silu, nullptr));
    HLA_TRY(check_tensor(out, out_stride, C, dt, B, "out"));
    if (B > 0 && !state) return fail(HLA_ERR_INVALID_ARGUMENT, "null state pointer");
    if (!aligned(state, elem_bytes(dt))) return fail(HLA_ERR_INVALID_ARGUMENT, "state is not aligned to its elements");
    if (B == 0) return HLA_OK;
    const Conv p{x, w, bias, out, dt, B, 1, C, width, silu, x_stride, out_stride, nullptr, state, state};
    return cuda_status(conv_step_launch(p, as_stream(stream)), "convolution step");
}

size_t hla_conv_backward_workspace_bytes(int B, int n, int C, int width, hla_dtype dt) {
    if (B < 0 || n < 0 || C <= 0 || C > kMaxChannels || width < 2 || width > 4 || (dt != HLA_F32 && dt != HLA_BF16)) return 0;
    if ((long long)B * n > kMaxRows) return 0;
    return scratch_bytes(conv_backward_partial_floats(B, n, C, width));
}

hla_status hla_conv_backward(const void *x, const void *w, const void *bias, const void *dout, void *dx, float *dw,
                             float *dbias, hla_dtype dt, int B, int n, int C, int width, long long x_stride,
                             long long dout_stride, long long dx_stride, int silu, const int *lengths,
                             void *workspace, size_t workspace_bytes, hla_stream_t stream) {
    clear_last_error();
    HLA_TRY(check_conv(x, w, bias, dt, B, n, C, width, x_stride, silu, lengths));
    HLA_TRY(check_tensor(dout, dout_stride, C, dt, (long long)B * n, "dout"));
    HLA_TRY(check_tensor(dx, dx_stride, C, dt, (long long)B * n, "dx"));
    if (!dw) return fail(HLA_ERR_INVALID_ARGUMENT, "null dw pointer");
    if (!aligned(dw, 4) || !aligned(dbias, 4)) return fail(HLA_ERR_INVALID_ARGUMENT, "dw and dbias must be 4-byte aligned");
    HLA_TRY(check_workspace(workspace, workspace_bytes, hla_conv_backward_workspace_bytes(B, n, C, width, dt)));
    cudaStream_t s = as_stream(stream);
    if ((long long)B * n == 0) {
        HLA_TRY(clear_header(workspace, s));
        HLA_TRY(cuda_status(cudaMemsetAsync(dw, 0, sizeof(float) * (size_t)C * width, s), "clearing dw"));
        return dbias ? cuda_status(cudaMemsetAsync(dbias, 0, sizeof(float) * (size_t)C, s), "clearing dbias") : HLA_OK;
    }
    const ConvBwd p{x, w, bias, dout, dx, dw, dbias, dt, B, n, C, width, silu, x_stride, dout_stride, dx_stride, lengths,
                    reinterpret_cast<float *>(static_cast<char *>(workspace) + kWsHeaderBytes),
                    static_cast<WsHeader *>(workspace)};
    return cuda_status(conv_backward_launch(p, s), "convolution backward");
}

size_t hla_ssm_workspace_bytes(int B, int n, int H, int P, int G, int N, hla_dtype dt) {
    if (B < 0 || n < 0 || H <= 0 || G <= 0 || H % G || !size_ok(P) || !size_ok(N)) return 0;
    if ((dt != HLA_F32 && dt != HLA_BF16) || (long long)B * n > kMaxRows || (long long)B * H > (1LL << 27)) return 0;
    Ssm p{};
    p.dt = dt; p.B = B; p.n = n; p.H = H; p.P = P; p.G = G; p.N = N;
    const size_t scan = ssm_scan_workspace_floats(p), tc = dt == HLA_BF16 ? ssm_tc_workspace_floats(p) : 0;
    return scratch_bytes(scan > tc ? scan : tc);
}

int hla_ssm_forward_path(int B, int n, int H, int P, int G, int N, hla_dtype dt, int aligned_rows, int *launches) {
    if (launches) *launches = 0;
    if (hla_ssm_workspace_bytes(B, n, H, P, G, N, dt) == 0 || n > (1 << 30)) return -1;
    Ssm p{};
    p.dt = dt; p.B = B; p.n = n; p.H = H; p.P = P; p.G = G; p.N = N;
    p.x = p.b = p.c = reinterpret_cast<const void *>(uintptr_t(aligned_rows ? 256 : 2));
    p.y = reinterpret_cast<void *>(uintptr_t(256));
    if (B == 0 || n == 0) return 0;
    const bool tc = ssm_tc_applicable(p);
    if (launches) *launches = tc ? ssm_tc_launches(p) : ssm_scan_launches(p);
    return tc ? 1 : 0;
}

hla_status hla_ssm_forward(const void *x, const void *delta, const float *a, const void *b, const void *c,
                           const float *skip, const float *delta_bias, void *y, hla_dtype dt, int B, int n, int H,
                           int P, int G, int N, long long x_stride, long long delta_stride, long long b_stride,
                           long long c_stride, long long y_stride, int softplus, const int *lengths,
                           const float *state_in, float *state_out, void *workspace, size_t workspace_bytes,
                           hla_stream_t stream) {
    clear_last_error();
    const Ssm p{x, delta, b, c, a, skip, delta_bias, y, dt, B, n, H, P, G, N, softplus, x_stride, delta_stride, b_stride,
                c_stride, y_stride, lengths, state_in, state_out, static_cast<char *>(workspace)};
    HLA_TRY(check_ssm(p, false));
    HLA_TRY(check_workspace(workspace, workspace_bytes, hla_ssm_workspace_bytes(B, n, H, P, G, N, dt)));
    if (B == 0) return HLA_OK;
    cudaStream_t s = as_stream(stream);
    if (n == 0) {
        HLA_TRY(clear_header(workspace, s));
        if (!state_out || state_out == state_in) return HLA_OK;
        const size_t bytes = sizeof(float) * (size_t)B * H * N * P;
        return cuda_status(state_in ? cudaMemcpyAsync(state_out, state_in, bytes, cudaMemcpyDeviceToDevice, s)
                                    : cudaMemsetAsync(state_out, 0, bytes, s), "copying the state");
    }
    if (ssm_tc_applicable(p)) return cuda_status(ssm_tc_launch(p, s), "selective scan (tensor cores)");
    return cuda_status(ssm_scan_launch(p, s), "selective scan");
}

hla_status hla_ssm_step(const void *x, const void *delta, const float *a, const void *b, const void *c,
                        const float *skip, const float *delta_bias, void *y, hla_dtype dt, int B, int H, int P, int G,
                        int N, long long x_stride, long long delta_stride, long long b_stride, long long c_stride,
                        long long y_stride, int softplus, float *state, hla_stream_t stream) {
    clear_last_error();
    const Ssm p{x, delta, b, c, a, skip, delta_bias, y, dt, B, 1, H, P, G, N, softplus, x_stride, delta_stride, b_stride,
                c_stride, y_stride, nullptr, state, state, nullptr};
    HLA_TRY(check_ssm(p, true));
    if (B == 0) return HLA_OK;
    return cuda_status(ssm_step_launch(p, as_stream(stream)), "selective scan step");
}

hla_status hla_qk_norm_forward(const void *q, const void *k, const void *wq, const void *wk, const float *cos,
                               const float *sin, const int *positions, void *q_out, void *k_out, hla_dtype dt, int B,
                               int n, int H, int Hk, int d, int rot, int interleaved, long long q_stride,
                               long long k_stride, int pos0, int table_rows, float eps, hla_stream_t stream) {
    clear_last_error();
    const QkNorm p{q, k, wq, wk, cos, sin, positions, q_out, k_out, dt, B, n, H, Hk, d, rot, interleaved, q_stride,
                   k_stride, pos0, table_rows, eps};
    HLA_TRY(check_qk(p));
    const long long rows = (long long)B * n;
    if (rows > 0 && (!q_out || !k_out)) return fail(HLA_ERR_INVALID_ARGUMENT, "null q_out or k_out pointer");
    if (!aligned(q_out, 16) || !aligned(k_out, 16))
        return fail(HLA_ERR_INVALID_ARGUMENT, "q_out and k_out must be 16-byte aligned");
    if (rows == 0) return HLA_OK;
    return cuda_status(qk_norm_forward_launch(p, as_stream(stream)), "q/k norm");
}

size_t hla_qk_norm_backward_workspace_bytes(int B, int n, int H, int Hk, int d, hla_dtype dt) {
    if (B < 0 || n < 0 || H <= 0 || Hk <= 0 || H % Hk || H > 65536 || !size_ok(d)) return 0;
    if ((dt != HLA_F32 && dt != HLA_BF16) || (long long)B * n > kMaxRows) return 0;
    return scratch_bytes((long long)B * n ? qk_norm_partial_floats(B, n, H, Hk, d) : 0);
}

hla_status hla_qk_norm_backward(const void *q, const void *k, const void *wq, const void *wk, const float *cos,
                                const float *sin, const int *positions, const void *dq_out, const void *dk_out,
                                void *dq, void *dk, float *dwq, float *dwk, hla_dtype dt, int B, int n, int H, int Hk,
                                int d, int rot, int interleaved, long long q_stride, long long k_stride,
                                long long dq_stride, long long dk_stride, int pos0, int table_rows, float eps,
                                void *workspace, size_t workspace_bytes, hla_stream_t stream) {
    clear_last_error();
    QkNormBwd p{{q, k, wq, wk, cos, sin, positions, nullptr, nullptr, dt, B, n, H, Hk, d, rot, interleaved, q_stride,
                 k_stride, pos0, table_rows, eps}, dq_out, dk_out, dq, dk, dq_stride, dk_stride, dwq, dwk, nullptr,
                static_cast<WsHeader *>(workspace)};
    HLA_TRY(check_qk(p.f));
    const long long rows = (long long)B * n;
    HLA_TRY(check_tensor(dq, dq_stride, (long long)H * d, dt, rows, "dq"));
    HLA_TRY(check_tensor(dk, dk_stride, (long long)Hk * d, dt, rows, "dk"));
    if (rows > 0 && (!dq_out || !dk_out)) return fail(HLA_ERR_INVALID_ARGUMENT, "null dq_out or dk_out pointer");
    if (!aligned(dq_out, 16) || !aligned(dk_out, 16))
        return fail(HLA_ERR_INVALID_ARGUMENT, "dq_out and dk_out must be 16-byte aligned");
    if (!aligned(dwq, 4) || !aligned(dwk, 4)) return fail(HLA_ERR_INVALID_ARGUMENT, "dwq and dwk must be 4-byte aligned");
    HLA_TRY(check_workspace(workspace, workspace_bytes, hla_qk_norm_backward_workspace_bytes(B, n, H, Hk, d, dt)));
    cudaStream_t s = as_stream(stream);
    if (rows == 0) {
        HLA_TRY(clear_header(workspace, s));
        if (dwq) HLA_TRY(cuda_status(cudaMemsetAsync(dwq, 0, sizeof(float) * d, s), "clearing dwq"));
        if (dwk) HLA_TRY(cuda_status(cudaMemsetAsync(dwk, 0, sizeof(float) * d, s), "clearing dwk"));
        return HLA_OK;
    }
    p.partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + kWsHeaderBytes);
    return cuda_status(qk_norm_backward_launch(p, s), "q/k norm backward");
}

}  // extern "C"
