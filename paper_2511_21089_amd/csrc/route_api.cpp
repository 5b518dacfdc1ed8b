// Host side of the router's entry points: argument checks, workspace, launch.
#include <mutex>

#include "internal.h"

using namespace mlpmoe;

namespace {

// Partial sums of a call with counts or loss: [blocks][B] pairs, then [blocks] ints.
size_t part_bytes(int blocks, int B) { return align_up((size_t)blocks * B * sizeof(RoutePart), 256); }

bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check_sizes(int T, int B, int elem_bytes)
{
    if (B < 1 || B > MLPMOE_MAX_BRANCHES || T < 0 || T > (1 << 24)) return MLPMOE_ERR_SHAPE;
    if (elem_bytes != 2 && elem_bytes != 4) return MLPMOE_ERR_UNSUPPORTED;
    return MLPMOE_OK;
}

// Bit b set: branch b may be taken.  NULL: all of them.
unsigned long long active_bits(const uint8_t *mask, int B, int *n)
{
    unsigned long long bits = 0;
    *n = 0;
    for (int b = 0; b < B; ++b)
        if (!mask || mask[b]) {
            bits |= 1ULL << b;
            ++*n;
        }
    return bits;
}

int route_topk(const void *logits, int ld, const uint8_t *active_mask, const uint8_t *token_mask, int T, int B, int k,
               int elem_bytes, uint8_t *route, float *probs, int32_t *counts, float *loss, void *workspace,
               size_t workspace_bytes, bool own, void *stream)
{
    int rc = check_sizes(T, B, elem_bytes);
    if (rc != MLPMOE_OK) return rc;
    if (k < 1 || k > B || ld < B || (long long)T * ld > (1LL << 40)) return MLPMOE_ERR_SHAPE;
    const bool stats = counts || loss;
    if (T == 0 && !stats) return MLPMOE_OK;
    if (T > 0 && (!logits || !route)) return MLPMOE_ERR_NULL;
    if (!aligned_to(logits, elem_bytes) || !aligned_to(probs, 4) || !aligned_to(counts, 4) || !aligned_to(loss, 4))
        return MLPMOE_ERR_ALIGN;

    (void)hipGetLastError();
    g_err_detail[0] = 0;
    RouteArgs a;
    a.logits = logits;
    a.ld = ld;
    a.active = active_bits(active_mask, B, &a.n_active);
    a.token_mask = token_mask;
    a.T = T;
    a.B = B;
    a.k = k;
    a.elem_bytes = elem_bytes;
    a.route = route;
    a.probs = probs;
    a.counts = counts;
    a.loss = loss;
    a.part = nullptr;
    a.part_n = nullptr;
    a.stream = static_cast<hipStream_t>(stream);

    const int blocks = route_blocks(T, B);
    std::unique_lock<std::mutex> lock(workspace_mutex(), std::defer_lock);
    if (stats && blocks > 1) {
        const size_t need = mlpmoe_route_workspace_bytes(T, B);
        if (own) {
            lock.lock();                     // held until the kernels are enqueued
            rc = owned_workspace(need, need, a.stream, &workspace, &workspace_bytes);
            if (rc != MLPMOE_OK) return rc;
        }
        if (!workspace || workspace_bytes < need || !aligned_to(workspace, 256)) return MLPMOE_ERR_WORKSPACE;
        a.part = static_cast<RoutePart *>(workspace);
        a.part_n = reinterpret_cast<int *>(static_cast<char *>(workspace) + part_bytes(blocks, B));
    }
    const hipError_t e = launch_route_topk(a);
    if (e != hipSuccess && g_err_detail[0] == 0) (void)note_hip_error("kernel launch", e);
    return e == hipSuccess ? MLPMOE_OK : MLPMOE_ERR_HIP;
}

}  // namespace

extern "C" {

size_t mlpmoe_route_workspace_bytes(int T, int B)
{
    if (T < 0 || T > (1 << 24) || B < 1 || B > MLPMOE_MAX_BRANCHES) return 0;
    const int blocks = route_most_blocks(T, B);
    return part_bytes(blocks, B) + align_up((size_t)blocks * sizeof(int), 256);
}

int mlpmoe_route_topk(const void *logits, int ld, const uint8_t *active_mask, const uint8_t *token_mask, int T, int B, int k,
                      int elem_bytes, uint8_t *route, float *probs, int32_t *counts, float *loss, void *stream)
{
    return route_topk(logits, ld, active_mask, token_mask, T, B, k, elem_bytes, route, probs, counts, loss, nullptr, 0, true,
                      stream);
}

int mlpmoe_route_topk_ws(const void *logits, int ld, const uint8_t *active_mask, const uint8_t *token_mask, int T, int B,
                         int k, int elem_bytes, uint8_t *route, float *probs, int32_t *counts, float *loss, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    return route_topk(logits, ld, active_mask, token_mask, T, B, k, elem_bytes, route, probs, counts, loss, workspace,
                      workspace_bytes, false, stream);
}

int mlpmoe_route_backward(const float *probs, const int32_t *counts, const float *dprobs, const float *dloss,
                          const uint8_t *active_mask, int T, int B, int elem_bytes, void *dlogits, void *stream)
{
    const int rc = check_sizes(T, B, elem_bytes);
    if (rc != MLPMOE_OK) return rc;
    if (T == 0) return MLPMOE_OK;
    if (!probs || !dlogits || (dloss && !counts)) return MLPMOE_ERR_NULL;
    if (!aligned_to(probs, 4) || !aligned_to(counts, 4) || !aligned_to(dprobs, 4) || !aligned_to(dloss, 4) ||
        !aligned_to(dlogits, elem_bytes))
        return MLPMOE_ERR_ALIGN;
    (void)hipGetLastError();
    g_err_detail[0] = 0;
    RouteBackArgs a;
    a.probs = probs;
    a.counts = counts;
    a.dprobs = dprobs;
    a.dloss = dloss;
    (void)active_bits(active_mask, B, &a.n_active);
    a.T = T;
    a.B = B;
    a.elem_bytes = elem_bytes;
    a.dlogits = dlogits;
    a.stream = static_cast<hipStream_t>(stream);
    const hipError_t e = launch_route_backward(a);
    if (e != hipSuccess && g_err_detail[0] == 0) (void)note_hip_error("kernel launch", e);
    return e == hipSuccess ? MLPMOE_OK : MLPMOE_ERR_HIP;
}

}  // extern "C"
