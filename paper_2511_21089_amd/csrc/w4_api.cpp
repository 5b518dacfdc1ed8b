// Host side of the 4-bit weights' entry points: argument checks, workspace, launch.
#include <mutex>

#include "internal.h"

using namespace mlpmoe;

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// H of the kernels on 4-bit weights: rows of whole steps of K (128).
int w4_h_ld(int d_inter) { return (int)align_up((size_t)d_inter, 128); }
size_t h_bytes(int T, int d_inter) { return align_up((size_t)T * w4_h_ld(d_inter) * 2, 256); }

constexpr int kW4MaxTokens = 65535 * 16;

// Rows that the kernels on 4-bit weights take: whole blocks, whose scales fit LDS.
bool row_lengths_fit(int d_model, int d_inter)
{
    return d_model % 32 == 0 && d_inter % 32 == 0 && d_model <= kW4MaxK && d_inter <= kW4MaxK;
}

int check_matrix(const void *codes, const void *scales, const void *W, int rows, int cols, int elem_bytes)
{
    if (rows < 0 || cols < 1 || rows > (1 << 22) || cols > (1 << 22) || (long long)rows * cols > (1LL << 40)) return MLPMOE_ERR_SHAPE;
    if ((elem_bytes != 2 && elem_bytes != 4) || cols % 32 != 0) return MLPMOE_ERR_UNSUPPORTED;
    if (rows == 0) return MLPMOE_OK;
    if (!codes || !scales || !W) return MLPMOE_ERR_NULL;
    if (!aligned16(codes) || !aligned16(scales) || !aligned16(W)) return MLPMOE_ERR_ALIGN;
    return MLPMOE_OK;
}

int forward_w4(const void *x, const uint8_t *const w[6], const int32_t *off, const float *alpha, const uint8_t *mask,
               const uint8_t *route, int T, int d_model, int d_inter, int B, int out_bytes, void *out, void *workspace,
               size_t workspace_bytes, bool own, void *stream)
{
    int rc = check_forward(x, w[0], w[2], w[4], off, alpha, mask, T, d_model, d_inter, B, out);
    if (rc != MLPMOE_OK) return rc;
    if ((out_bytes != 2 && out_bytes != 4) || !row_lengths_fit(d_model, d_inter)) return MLPMOE_ERR_UNSUPPORTED;
    if (T == 0) return MLPMOE_OK;
    if (d_inter > 0 && (!w[1] || !w[3] || !w[5])) return MLPMOE_ERR_NULL;
    if (!aligned16(w[1]) || !aligned16(w[3]) || !aligned16(w[5])) return MLPMOE_ERR_ALIGN;
    if (T > kW4MaxTokens) return MLPMOE_ERR_SHAPE;

    (void)hipGetLastError();
    g_err_detail[0] = 0;
    BranchTable bt;
    make_table(off, alpha, mask, B, bt);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (bt.n_runs == 0) {                    // nothing active: the sum over branches is empty
        const size_t n = (size_t)T * d_model;
        const hipError_t e = out_bytes == 2 ? launch_fill_zero16(static_cast<uint16_t *>(out), n, s)
                                            : launch_fill_zero(static_cast<float *>(out), n, s);
        return e == hipSuccess ? MLPMOE_OK : MLPMOE_ERR_HIP;
    }
    const size_t need = mlpmoe_w4_workspace_bytes(T, d_model, d_inter, B);
    std::unique_lock<std::mutex> lock(workspace_mutex(), std::defer_lock);
    if (own) {
        lock.lock();                         // held until the kernels are enqueued
        rc = owned_workspace(need, need, s, &workspace, &workspace_bytes);
        if (rc != MLPMOE_OK) return rc;
    }
    if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return MLPMOE_ERR_WORKSPACE;
    W4Args a;
    a.x = x;
    a.gc = w[0]; a.gs = w[1]; a.uc = w[2]; a.us = w[3]; a.dc = w[4]; a.ds = w[5];
    a.route = route;
    a.T = T; a.d_model = d_model; a.d_inter = d_inter;
    a.H = workspace;
    a.ldh = w4_h_ld(d_inter);
    a.out = out;
    a.out_bf16 = out_bytes == 2;
    a.partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + h_bytes(T, d_inter));
    a.stream = s;
    const hipError_t e = T > 16 ? launch_w4_tiles(a, bt) : launch_w4_forward(a, bt);
    if (e != hipSuccess && g_err_detail[0] == 0) (void)note_hip_error("kernel launch", e);
    return e == hipSuccess ? MLPMOE_OK : MLPMOE_ERR_HIP;
}

}  // namespace

extern "C" {

int mlpmoe_w4_quantize(const void *W, int rows, int cols, int elem_bytes, uint8_t *codes, uint8_t *scales, void *stream)
{
    const int rc = check_matrix(codes, scales, W, rows, cols, elem_bytes);
    if (rc != MLPMOE_OK || rows == 0) return rc;
    (void)hipGetLastError();
    g_err_detail[0] = 0;
    const hipError_t e = launch_w4_quantize(W, (size_t)rows * cols, elem_bytes, codes, scales, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MLPMOE_OK : MLPMOE_ERR_HIP;
}

int mlpmoe_w4_dequantize(const uint8_t *codes, const uint8_t *scales, int rows, int cols, int elem_bytes, void *W, void *stream)
{
    const int rc = check_matrix(codes, scales, W, rows, cols, elem_bytes);
    if (rc != MLPMOE_OK || rows == 0) return rc;
    (void)hipGetLastError();
    g_err_detail[0] = 0;
    const hipError_t e = launch_w4_dequantize(codes, scales, (size_t)rows * cols, elem_bytes, W, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MLPMOE_OK : MLPMOE_ERR_HIP;
}

size_t mlpmoe_w4_workspace_bytes(int T, int d_model, int d_inter, int B)
{
    if (T < 0 || T > kW4MaxTokens || d_model < 1 || d_inter < 0 || B < 1 || B > MLPMOE_MAX_BRANCHES) return 0;
    if (!row_lengths_fit(d_model, d_inter)) return 0;
    return h_bytes(T, d_inter) + align_up(w4_partial_floats(T, d_model, d_inter) * 4, 256) + 256;
}

int mlpmoe_forward_w4(const void *x, const uint8_t *gate_codes, const uint8_t *gate_scales, const uint8_t *up_codes,
                      const uint8_t *up_scales, const uint8_t *down_codes, const uint8_t *down_scales,
                      const int32_t *branch_offsets, const float *alpha, const uint8_t *active_mask, const uint8_t *route,
                      int T, int d_model, int d_inter, int B, int out_bytes, void *out, void *stream)
{
    const uint8_t *const w[6] = {gate_codes, gate_scales, up_codes, up_scales, down_codes, down_scales};
    return forward_w4(x, w, branch_offsets, alpha, active_mask, route, T, d_model, d_inter, B, out_bytes, out, nullptr, 0, true,
                      stream);
}

int mlpmoe_forward_w4_ws(const void *x, const uint8_t *gate_codes, const uint8_t *gate_scales, const uint8_t *up_codes,
                         const uint8_t *up_scales, const uint8_t *down_codes, const uint8_t *down_scales,
                         const int32_t *branch_offsets, const float *alpha, const uint8_t *active_mask, const uint8_t *route,
                         int T, int d_model, int d_inter, int B, int out_bytes, void *out, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    const uint8_t *const w[6] = {gate_codes, gate_scales, up_codes, up_scales, down_codes, down_scales};
    return forward_w4(x, w, branch_offsets, alpha, active_mask, route, T, d_model, d_inter, B, out_bytes, out, workspace,
                      workspace_bytes, false, stream);
}

}  // extern "C"
