// extern "C" entry points of the rest of a block: the gated recurrence, the norms around a block, the gated
// feed-forward projections.  Argument checks, workspace sizing, dispatch; see include/hla.h for the contracts.
#include <cmath>

#include "hla_checks.h"

namespace hla {
namespace {

bool type_ok(hla_dtype dt) { return dt == HLA_F32 || dt == HLA_BF16; }

hla_status check_aligned16(const void *p, const char *name) {
    return aligned(p, 16) ? HLA_OK : fail(HLA_ERR_INVALID_ARGUMENT, "%s must be 16-byte aligned", name);
}

hla_status check_glr(const Glr &p) {
    HLA_TRY(check_type(p.dt));
    HLA_TRY(check_rows(p.B, p.n));
    if (p.C <= 0) return fail(HLA_ERR_INVALID_ARGUMENT, "C=%d must be above 0", p.C);
    if (p.C > kMaxChannels || !glr_fits(p.B, p.C)) return fail(HLA_ERR_UNSUPPORTED, "problem too large");
    const long long rows = (long long)p.B * p.n;
    HLA_TRY(check_tensor(p.x, p.x_stride, p.C, p.dt, rows, "x"));
    HLA_TRY(check_tensor(p.r, p.r_stride, p.C, p.dt, rows, "r"));
    HLA_TRY(check_tensor(p.g, p.g_stride, p.C, p.dt, rows, "g"));
    if (rows > 0 && !p.decay) return fail(HLA_ERR_INVALID_ARGUMENT, "null decay pointer");
    HLA_TRY(check_aligned16(p.decay, "decay"));
    HLA_TRY(check_aligned16(p.marks, "marks"));
    HLA_TRY(check_aligned16(p.state_in, "state"));
    HLA_TRY(check_aligned16(p.state_out, "state"));
    return aligned(p.lengths, 4) ? HLA_OK : fail(HLA_ERR_INVALID_ARGUMENT, "lengths must be 4-byte aligned");
}

bool glr_sizes(int B, int n, int C, hla_dtype dt) {
    return B >= 0 && n >= 0 && n <= (1 << 30) && C > 0 && C <= kMaxChannels && type_ok(dt) && (long long)B * n <= kMaxRows &&
           glr_fits(B, C);
}

// the state behind no tokens
hla_status keep_state(const float *in, float *out, size_t count, cudaStream_t s) {
    if (!out || out == in || count == 0) return HLA_OK;
    const size_t bytes = sizeof(float) * count;
    return cuda_status(in ? cudaMemcpyAsync(out, in, bytes, cudaMemcpyDeviceToDevice, s) : cudaMemsetAsync(out, 0, bytes, s),
                       "copying the state");
}

constexpr long long kMaxNormColumns = kMaxRows / 3 - 32;  // three sums a column, 32 columns a block

hla_status check_norm(BlockNorm &p, int rows, double dropout) {
    HLA_TRY(check_type(p.dt));
    if (rows < 0 || p.C <= 0) return fail(HLA_ERR_INVALID_ARGUMENT, "bad size rows=%d C=%d", rows, p.C);
    if (p.C > kMaxNormColumns) return fail(HLA_ERR_UNSUPPORTED, "problem too large");
    HLA_TRY(check_flag(p.post, "post_norm"));
    HLA_TRY(check_flag(p.pre, "pre_norm"));
    if (p.act < HLA_LINEAR || p.act > HLA_SILU) return fail(HLA_ERR_INVALID_ARGUMENT, "unknown activation %d", p.act);
    if (!std::isfinite(p.eps) || p.eps < 0.f) return fail(HLA_ERR_INVALID_ARGUMENT, "eps must be finite and not negative");
    if (!std::isfinite(p.alpha)) return fail(HLA_ERR_INVALID_ARGUMENT, "alpha must be finite");
    if (!(dropout >= 0. && dropout < 1.)) return fail(HLA_ERR_INVALID_ARGUMENT, "dropout must be at least 0 and below 1");
    HLA_TRY(check_tensor(p.x, p.x_stride, p.C, p.dt, rows, "x"));
    HLA_TRY(check_tensor(p.y, p.y_stride, p.C, p.dt, rows, "y"));
    if (p.gate) HLA_TRY(check_tensor(p.gate, p.gate_stride, p.C, p.dt, rows, "gate"));
    if (!p.post) p.w_post = nullptr;
    if (!p.pre) p.w_pre = nullptr;
    const size_t eb = elem_bytes(p.dt);
    if (!aligned(p.w_post, eb) || !aligned(p.scale, eb) || !aligned(p.w_pre, eb))
        return fail(HLA_ERR_INVALID_ARGUMENT, "weights must be aligned to their elements");
    p.rows = rows;
    p.drop_below = (uint32_t)(dropout * 4294967296.0);
    p.drop = p.drop_below != 0;
    p.keep_scale = p.drop ? (float)(1.0 / (1.0 - dropout)) : 1.f;
    for (uint32_t i = 0; i < 10; ++i) {
        p.key[i][0] = (uint32_t)p.seed + i * 0x9E3779B9u;
        p.key[i][1] = (uint32_t)(p.seed >> 32) + i * 0xBB67AE85u;
    }
    return HLA_OK;
}

hla_status check_ffn(const Ffn &p) {
    HLA_TRY(check_type(p.dt));
    if (p.M < 0 || p.K <= 0 || p.F <= 0) return fail(HLA_ERR_INVALID_ARGUMENT, "bad size rows=%d K=%d F=%d", p.M, p.K, p.F);
    if (!hla_ffn_backward_workspace_bytes(p.M, p.K, p.F, p.dt)) return fail(HLA_ERR_UNSUPPORTED, "problem too large");
    if (p.act < HLA_LINEAR || p.act > HLA_SILU) return fail(HLA_ERR_INVALID_ARGUMENT, "unknown activation %d", p.act);
    HLA_TRY(check_tensor(p.x, p.x_stride, p.K, p.dt, p.M, "x"));
    if (!p.w) return fail(HLA_ERR_INVALID_ARGUMENT, "null w pointer");
    return aligned(p.w, elem_bytes(p.dt)) ? HLA_OK : fail(HLA_ERR_INVALID_ARGUMENT, "w is not aligned to its elements");
}

// Sizes of the products: each below 2^26 (tiles of them, side by side, are counted in 32 bits)
bool ffn_sizes(int M, int K, int F, hla_dtype dt) {
    constexpr int kMost = 1 << 26;
    return M >= 0 && K > 0 && F > 0 && type_ok(dt) && M <= kMost && K <= kMost && F <= kMost &&
           (long long)K * F <= kMaxValues && (long long)M * K <= kMaxValues && (long long)M * F <= kMaxValues &&
           ((long long)M / 64 + 1) * (F / 32 + 1) <= kMaxRows && ((long long)M / 64 + 1) * (K / 32 + 1) <= kMaxRows &&
           ((long long)F / 32 + 1) * (K / 32 + 1) <= kMaxRows;
}

}  // namespace
}  // namespace hla

using namespace hla;

extern "C" {

int hla_glr_marks(int n) { return n < 0 ? 0 : glr_marks(n); }

hla_status hla_glr_forward(const void *x, const void *r, const void *g, const float *decay, void *y, hla_dtype dt, int B,
                           int n, int C, long long x_stride, long long r_stride, long long g_stride, long long y_stride,
                           const int *lengths, const float *state_in, float *state_out, float *marks,
                           hla_stream_t stream) {
    clear_last_error();
    const Glr p{x, r, g, decay, y, dt, B, n, C, x_stride, r_stride, g_stride, y_stride, lengths, state_in, state_out, marks};
    HLA_TRY(check_glr(p));
    HLA_TRY(check_tensor(y, y_stride, C, dt, (long long)B * n, "y"));
    if (B == 0) return HLA_OK;
    cudaStream_t s = as_stream(stream);
    if (n == 0) return keep_state(state_in, state_out, (size_t)B * C, s);
    return cuda_status(glr_forward_launch(p, s), "gated recurrence");
}

hla_status hla_glr_step(const void *x, const void *r, const void *g, const float *decay, void *y, hla_dtype dt, int B, int C,
                        long long x_stride, long long r_stride, long long g_stride, long long y_stride, float *state,
                        hla_stream_t stream) {
    clear_last_error();
    const Glr p{x, r, g, decay, y, dt, B, 1, C, x_stride, r_stride, g_stride, y_stride, nullptr, state, state, nullptr};
    HLA_TRY(check_glr(p));
    HLA_TRY(check_tensor(y, y_stride, C, dt, B, "y"));
    if (B > 0 && !state) return fail(HLA_ERR_INVALID_ARGUMENT, "null state pointer");
    if (B == 0) return HLA_OK;
    return cuda_status(glr_step_launch(p, as_stream(stream)), "gated recurrence step");
}

size_t hla_glr_backward_workspace_bytes(int B, int n, int C, hla_dtype dt) {
    return glr_sizes(B, n, C, dt) ? scratch_bytes(glr_backward_partial_floats(B, n, C)) : 0;
}

hla_status hla_glr_backward(const void *x, const void *r, const void *g, const float *decay, const void *dy,
                            const float *marks, void *dx, void *dr, void *dg, float *ddecay, hla_dtype dt, int B, int n,
                            int C, long long x_stride, long long r_stride, long long g_stride, long long dy_stride,
                            long long dx_stride, long long dr_stride, long long dg_stride, const int *lengths,
                            const float *dstate_out, float *dstate_in, void *workspace, size_t workspace_bytes,
                            hla_stream_t stream) {
    clear_last_error();
    GlrBwd p{{x, r, g, decay, nullptr, dt, B, n, C, x_stride, r_stride, g_stride, C, lengths, nullptr, nullptr,
              const_cast<float *>(marks)},
             dy, dstate_out, dx, dr, dg, ddecay, dstate_in, dy_stride, dx_stride, dr_stride, dg_stride, nullptr,
             static_cast<WsHeader *>(workspace)};
    HLA_TRY(check_glr(p.f));
    const long long rows = (long long)B * n;
    HLA_TRY(check_tensor(dy, dy_stride, C, dt, rows, "dy"));
    HLA_TRY(check_tensor(dx, dx_stride, C, dt, rows, "dx"));
    HLA_TRY(check_tensor(dr, dr_stride, C, dt, rows, "dr"));
    HLA_TRY(check_tensor(dg, dg_stride, C, dt, rows, "dg"));
    if (rows > 0 && !marks) return fail(HLA_ERR_INVALID_ARGUMENT, "null marks pointer");
    if (!ddecay) return fail(HLA_ERR_INVALID_ARGUMENT, "null ddecay pointer");
    HLA_TRY(check_aligned16(ddecay, "ddecay"));
    HLA_TRY(check_aligned16(dstate_out, "dstate_out"));
    HLA_TRY(check_aligned16(dstate_in, "dstate_in"));
    HLA_TRY(check_workspace(workspace, workspace_bytes, hla_glr_backward_workspace_bytes(B, n, C, dt)));
    cudaStream_t s = as_stream(stream);
    if (rows == 0) {
        HLA_TRY(clear_header(workspace, s));
        HLA_TRY(cuda_status(cudaMemsetAsync(ddecay, 0, sizeof(float) * (size_t)C, s), "clearing ddecay"));
        return keep_state(dstate_out, dstate_in, (size_t)B * C, s);
    }
    p.partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + kWsHeaderBytes);
    return cuda_status(glr_backward_launch(p, s), "gated recurrence backward");
}

hla_status hla_block_norm_forward(const void *x, const void *y, const void *gate, const void *w_post, const void *scale,
                                  const void *w_pre, void *x_out, void *h, hla_dtype dt, int rows, int C,
                                  long long x_stride, long long y_stride, long long gate_stride, long long x_out_stride,
                                  long long h_stride, int post_norm, int pre_norm, int act, float alpha, float eps,
                                  double dropout, unsigned long long seed, unsigned long long offset, hla_stream_t stream) {
    clear_last_error();
    BlockNorm p{x, y, gate, w_post, scale, w_pre, x_out, h, dt, rows, C, post_norm, pre_norm, act, x_stride, y_stride,
                gate_stride, x_out_stride, h_stride, alpha, eps, 0, 0, 1.f, seed, offset, {}};
    HLA_TRY(check_norm(p, rows, dropout));
    HLA_TRY(check_tensor(x_out, x_out_stride, C, dt, rows, "x_out"));
    if (pre_norm) {
        HLA_TRY(check_tensor(h, h_stride, C, dt, rows, "h"));
    } else {
        p.h = nullptr;
    }
    if (rows == 0) return HLA_OK;
    return cuda_status(block_norm_forward_launch(p, as_stream(stream)), "block norm");
}

size_t hla_block_norm_backward_workspace_bytes(int rows, int C, hla_dtype dt) {
    if (rows < 0 || C <= 0 || C > kMaxNormColumns || !type_ok(dt)) return 0;
    return scratch_bytes(rows ? block_norm_partial_floats(rows, C) : 0);
}

hla_status hla_block_norm_backward(const void *x, const void *y, const void *gate, const void *w_post, const void *scale,
                                   const void *w_pre, const void *dx_out, const void *dh, void *dx, void *dy, void *dgate,
                                   float *dw_post, float *dscale, float *dw_pre, hla_dtype dt, int rows, int C,
                                   long long x_stride, long long y_stride, long long gate_stride, long long dx_out_stride,
                                   long long dh_stride, long long dx_stride, long long dy_stride, long long dgate_stride,
                                   int post_norm, int pre_norm, int act, float alpha, float eps, double dropout,
                                   unsigned long long seed, unsigned long long offset, void *workspace,
                                   size_t workspace_bytes, hla_stream_t stream) {
    clear_last_error();
    BlockNormBwd q{{x, y, gate, w_post, scale, w_pre, nullptr, nullptr, dt, rows, C, post_norm, pre_norm, act, x_stride,
                    y_stride, gate_stride, C, C, alpha, eps, 0, 0, 1.f, seed, offset, {}},
                   dx_out, dh, dx, dy, dgate, dw_post, dscale, dw_pre, dx_out_stride, dh_stride, dx_stride, dy_stride,
                   dgate_stride, nullptr, static_cast<WsHeader *>(workspace)};
    HLA_TRY(check_norm(q.f, rows, dropout));
    HLA_TRY(check_tensor(dx_out, dx_out_stride, C, dt, rows, "dx_out"));
    HLA_TRY(check_tensor(dx, dx_stride, C, dt, rows, "dx"));
    HLA_TRY(check_tensor(dy, dy_stride, C, dt, rows, "dy"));
    if (pre_norm) {
        HLA_TRY(check_tensor(dh, dh_stride, C, dt, rows, "dh"));
    } else {
        q.dh = nullptr;
    }
    if (gate) {
        HLA_TRY(check_tensor(dgate, dgate_stride, C, dt, rows, "dgate"));
    } else {
        q.dgate = nullptr;
    }
    if (!aligned(dw_post, 4) || !aligned(dscale, 4) || !aligned(dw_pre, 4))
        return fail(HLA_ERR_INVALID_ARGUMENT, "dw_post, dscale and dw_pre must be 4-byte aligned");
    HLA_TRY(check_workspace(workspace, workspace_bytes, hla_block_norm_backward_workspace_bytes(rows, C, dt)));
    cudaStream_t s = as_stream(stream);
    if (rows == 0) {
        HLA_TRY(clear_header(workspace, s));
        for (float *out : {dw_post, dscale, dw_pre}) {
            if (!out) continue;
            HLA_TRY(cuda_status(cudaMemsetAsync(out, 0, sizeof(float) * (size_t)C, s), "clearing weight gradients"));
        }
        return HLA_OK;
    }
    q.partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + kWsHeaderBytes);
    return cuda_status(block_norm_backward_launch(q, s), "block norm backward");
}

size_t hla_ffn_workspace_bytes(int rows, int K, int F, hla_dtype dt) {
    return ffn_sizes(rows, K, F, dt) ? kWsHeaderBytes + align_up(ffn_forward_scratch_bytes(rows, K, F, dt), 256) : 0;
}

size_t hla_ffn_backward_workspace_bytes(int rows, int K, int F, hla_dtype dt) {
    return ffn_sizes(rows, K, F, dt) ? kWsHeaderBytes + align_up(ffn_backward_scratch_bytes(rows, K, F, dt), 256) : 0;
}

hla_status hla_ffn_forward(const void *x, const void *w, void *out, hla_dtype dt, int rows, int K, int F,
                           long long x_stride, long long out_stride, int act, void *workspace, size_t workspace_bytes,
                           hla_stream_t stream) {
    clear_last_error();
    const Ffn p{x, w, out, dt, rows, K, F, act, x_stride, out_stride, static_cast<char *>(workspace)};
    HLA_TRY(check_ffn(p));
    HLA_TRY(check_tensor(out, out_stride, F, dt, rows, "out"));
    HLA_TRY(check_workspace(workspace, workspace_bytes, hla_ffn_workspace_bytes(rows, K, F, dt)));
    cudaStream_t s = as_stream(stream);
    if (rows == 0) return clear_header(workspace, s);
    return cuda_status(ffn_forward_launch(p, s), "feed-forward");
}

hla_status hla_ffn_backward(const void *x, const void *w, const void *dout, void *dx, void *dw, hla_dtype dt, int rows,
                            int K, int F, long long x_stride, long long dout_stride, long long dx_stride, int act,
                            void *workspace, size_t workspace_bytes, hla_stream_t stream) {
    clear_last_error();
    const FfnBwd p{{x, w, nullptr, dt, rows, K, F, act, x_stride, F, static_cast<char *>(workspace)}, dout, dx, dw,
                   dout_stride, dx_stride};
    HLA_TRY(check_ffn(p.f));
    HLA_TRY(check_tensor(dout, dout_stride, F, dt, rows, "dout"));
    HLA_TRY(check_tensor(dx, dx_stride, K, dt, rows, "dx"));
    if (!dw) return fail(HLA_ERR_INVALID_ARGUMENT, "null dw pointer");
    if (!aligned(dw, elem_bytes(dt))) return fail(HLA_ERR_INVALID_ARGUMENT, "dw is not aligned to its elements");
    HLA_TRY(check_workspace(workspace, workspace_bytes, hla_ffn_backward_workspace_bytes(rows, K, F, dt)));
    cudaStream_t s = as_stream(stream);
    if (rows == 0) {
        HLA_TRY(clear_header(workspace, s));
        return cuda_status(cudaMemsetAsync(dw, 0, elem_bytes(dt) * 2 * (size_t)F * K, s), "clearing dw");
    }
    return cuda_status(ffn_backward_launch(p, s), "feed-forward backward");
}

}  // extern "C"
