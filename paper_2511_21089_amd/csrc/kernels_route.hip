// The router of a routed layer: which branches every token takes, the softmax probabilities, how many tokens take each
// branch, the balance loss, and the gradient of the logits.
//
//   p[t, b] = exp(x[t, b] - max) / sum        over the active branches of a token that counts
//   loss    = A * sum_b f_b P_b,   f_b = counts[b] / sum counts,   P_b = mean over the counted tokens of p[t, b]
//   dx      = p (.) (g - sum_b p g),          g[t, b] = dprobs[t, b] + dloss * A * f_b / N
//
// Memory bound by intention: a row is at most 64 logits, so a token is worked on by L = 1 .. 16 neighbouring lanes that hold
// four branches each in registers; everything a token needs crosses lanes by DPP inside 16 lanes.  Logits are read once,
// probabilities and route bytes written once.
#include "internal.h"

namespace mlpmoe {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint16_t u16x4;

constexpr float kNegInf = -__builtin_inff();

template <int kCtrl>
__device__ __forceinline__ float dpp(float v)
{
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, kCtrl, 0xf, 0xf, false));
}
template <int kCtrl>
__device__ __forceinline__ int dpp(int v)
{
    return __builtin_amdgcn_update_dpp(v, v, kCtrl, 0xf, 0xf, false);
}

// Reduction over the L lanes of a token, the same value on each: neighbours, pairs, then the mirrored half and the mirrored
// whole of a row of 16.
template <int L, typename V, typename F>
__device__ __forceinline__ V over_token(V v, F f)
{
    if (L >= 2) v = f(v, dpp<0xB1>(v));        // quad_perm 1 0 3 2
    if (L >= 4) v = f(v, dpp<0x4E>(v));        // quad_perm 2 3 0 1
    if (L >= 8) v = f(v, dpp<0x141>(v));       // row_half_mirror
    if (L >= 16) v = f(v, dpp<0x140>(v));      // row_mirror
    return v;
}
struct Add {
    template <typename V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};
struct Max {
    // a not-a-number loses against a number
    __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_fmaxf(a, b); }
};

__device__ __forceinline__ float widen(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
__device__ __forceinline__ float widen(float v) { return v; }

// Four neighbouring values of a row, those past the row's end `fill`.
template <bool kVec, typename E>
__device__ __forceinline__ void load4(const E *row, int b0, int B, float fill, float v[4])
{
    if constexpr (kVec) {
        if (b0 < B) {
            if constexpr (sizeof(E) == 4) {
                const f32x4 w = *reinterpret_cast<const f32x4 *>(row + b0);
                v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w;
            } else {
                const u16x4 w = *reinterpret_cast<const u16x4 *>(row + b0);
                v[0] = widen(w.x), v[1] = widen(w.y), v[2] = widen(w.z), v[3] = widen(w.w);
            }
        } else {
            v[0] = v[1] = v[2] = v[3] = fill;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = b0 + e < B ? widen(row[b0 + e]) : fill;
    }
}

template <bool kVec>
__device__ __forceinline__ void store4(float *row, int b0, int B, const float v[4])
{
    if constexpr (kVec) {
        if (b0 < B) *reinterpret_cast<f32x4 *>(row + b0) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (b0 + e < B) row[b0 + e] = v[e];
    }
}

template <bool kVec>
__device__ __forceinline__ void store4(uint16_t *row, int b0, int B, const float v[4])
{
    u16x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint16_t, (__bf16)v[e]);
    if constexpr (kVec) {
        if (b0 < B) *reinterpret_cast<u16x4 *>(row + b0) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (b0 + e < B) row[b0 + e] = w[e];
    }
}

// Sums of a call with counts and loss from the blocks' partial sums, in the order of the blocks; the probabilities' in
// double, since the number of tokens goes to 2^24.
__device__ __forceinline__ void finish(const float *psum, const int *cnt, int blocks, int B, int n_active, int32_t *counts,
                                       float *loss)
{
    // psum and cnt: [blocks][B + 1], the last entry of a row the block's counted tokens
    __shared__ double s_p[1024];
    __shared__ int s_c[1024];
    __shared__ double s_prod[64];
    __shared__ int s_cnt[65];
    const int cols = B + 1;
    const int parts = (int)blockDim.x / cols;            // threads that share a column
    const int col = threadIdx.x % cols, part = threadIdx.x / cols;
    double p = 0;
    int c = 0;
    if (part < parts)
        for (int i = part; i < blocks; i += parts) {
            p += (double)psum[(size_t)i * cols + col];
            c += cnt[(size_t)i * cols + col];
        }
    s_p[threadIdx.x] = p;
    s_c[threadIdx.x] = c;
    __syncthreads();
    if ((int)threadIdx.x < cols) {
        p = 0, c = 0;
        for (int i = 0; i < parts; ++i) {
            p += s_p[i * cols + threadIdx.x];
            c += s_c[i * cols + threadIdx.x];
        }
        s_cnt[threadIdx.x] = c;
        if (counts) counts[threadIdx.x] = c;
        if ((int)threadIdx.x < B) s_prod[threadIdx.x] = p * (double)c;
    }
    __syncthreads();
    if (threadIdx.x == 0 && loss) {
        double sum = 0;
        long long taken = 0;
        for (int b = 0; b < B; ++b) {
            sum += s_prod[b];
            taken += s_cnt[b];
        }
        const double n = (double)s_cnt[B];
        *loss = taken > 0 ? (float)((double)n_active * sum / ((double)taken * n)) : 0.0f;
    }
}

constexpr int kRouteThreads = 512;

// A token on L lanes, four branches a lane.  kStats: also what the counts and the loss need: with one block the result, else
// the block's partial sums.
template <int L, typename E, bool kVec, bool kStats>
__global__ void __launch_bounds__(kRouteThreads)
route_topk_kernel(const E *__restrict__ logits, int ld, unsigned long long active, const uint8_t *__restrict__ token_mask,
                  int T, int B, int k, uint8_t *__restrict__ route, float *__restrict__ probs, float *__restrict__ part_p,
                  int *__restrict__ part_c, int32_t *__restrict__ counts, float *__restrict__ loss, int n_active)
{
    const int l = threadIdx.x % L, b0 = 4 * l;
    const int per_block = blockDim.x / L;
    float sum_p[4] = {0, 0, 0, 0};
    int sum_c[4] = {0, 0, 0, 0}, sum_n = 0;
    const unsigned on = (unsigned)(active >> b0) & 15u;
    // lanes of this token that come before this one
    const unsigned long long lower = ((1ULL << l) - 1) << ((threadIdx.x & 63) - l);

    for (long long t = (long long)blockIdx.x * per_block + threadIdx.x / L; t < T; t += (long long)gridDim.x * per_block) {
        float x[4];
        load4<kVec>(logits + t * ld, b0, B, kNegInf, x);
        const bool real = !token_mask || token_mask[t] != 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = ((on >> e) & 1u) && real ? x[e] : kNegInf;
        const float m = over_token<L>(__builtin_fmaxf(__builtin_fmaxf(x[0], x[1]), __builtin_fmaxf(x[2], x[3])), Max());
        const bool used = m > kNegInf;

        float p[4] = {0, 0, 0, 0};
        if (probs || kStats) {
            float s = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[e] = __expf(x[e] - m);
                s += p[e];
            }
            s = over_token<L>(s, Add());
            const float inv = 1.0f / s;
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = used && x[e] != kNegInf ? p[e] * inv : 0.0f;
            if (probs) store4<kVec>(probs + t * B, b0, B, p);
        }

        // The k first in the order (larger logit, then lower index).  A lane sorts its four; every round takes the largest head
        // of the token's lanes, of the lowest lane that has it.  What is not a number is never taken.
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = x[e] > kNegInf ? x[e] : kNegInf;
        int rank[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int f = e + 1; f < 4; ++f) {
                const int later = y[e] >= y[f];
                rank[f] += later;
                rank[e] += 1 - later;
            }
        float s0 = __builtin_fmaxf(y[0], y[1]), s1 = __builtin_fminf(y[0], y[1]);
        float s2 = __builtin_fmaxf(y[2], y[3]), s3 = __builtin_fminf(y[2], y[3]);
        float h = __builtin_fminf(s0, s2);
        s0 = __builtin_fmaxf(s0, s2);
        float lo = __builtin_fmaxf(s1, s3);
        s3 = __builtin_fminf(s1, s3);
        s1 = __builtin_fmaxf(h, lo);
        s2 = __builtin_fminf(h, lo);
        int taken = 0;
        for (int i = 0; i < k; ++i) {
            const float best = over_token<L>(s0, Max());
            const bool mine = s0 == best && best > kNegInf;
            const bool first = mine && (__ballot(mine) & lower) == 0;
            taken += first;
            s0 = first ? s1 : s0;
            s1 = first ? s2 : s1;
            s2 = first ? s3 : s2;
            s3 = first ? kNegInf : s3;
        }
        uint32_t bytes = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) bytes |= (rank[e] < taken ? 1u : 0u) << (8 * e);
        if constexpr (kVec) {
            if (b0 < B) *reinterpret_cast<uint32_t *>(route + t * B + b0) = bytes;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (b0 + e < B) route[t * B + b0 + e] = (uint8_t)(bytes >> (8 * e));
        }
        if constexpr (kStats) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum_p[e] += p[e];
                sum_c[e] += (int)((bytes >> (8 * e)) & 1u);
            }
            sum_n += used;
        }
    }

    if constexpr (kStats) {
        // the block's sums, in the order of its tokens' lanes
        __shared__ float s_p[kRouteThreads * 4];
        __shared__ int s_c[kRouteThreads * 4];
        __shared__ int s_n[kRouteThreads];
        __shared__ float s_tp[65];
        __shared__ int s_tc[65];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s_p[threadIdx.x * 4 + e] = sum_p[e];
            s_c[threadIdx.x * 4 + e] = sum_c[e];
        }
        s_n[threadIdx.x] = sum_n;
        __syncthreads();
        if ((int)threadIdx.x <= B) {
            float p = 0;
            int c = 0;
            const int col = threadIdx.x;
            for (int g = 0; g < per_block; ++g) {
                if (col < B) {
                    p += s_p[g * L * 4 + col];
                    c += s_c[g * L * 4 + col];
                } else {
                    c += s_n[g * L];
                }
            }
            if (gridDim.x == 1) {
                s_tp[col] = p;
                s_tc[col] = c;
            } else {
                part_p[(size_t)blockIdx.x * (B + 1) + col] = p;
                part_c[(size_t)blockIdx.x * (B + 1) + col] = c;
            }
        }
        if (gridDim.x == 1) {
            __syncthreads();
            finish(s_tp, s_tc, 1, B, n_active, counts, loss);
        }
    }
}

__global__ void __launch_bounds__(1024)
route_finish_kernel(const float *__restrict__ part_p, const int *__restrict__ part_c, int blocks, int B, int n_active,
                    int32_t *__restrict__ counts, float *__restrict__ loss)
{
    finish(part_p, part_c, blocks, B, n_active, counts, loss);
}

template <int L, typename E, bool kVec>
__global__ void __launch_bounds__(256)
route_backward_kernel(const float *__restrict__ probs, const int32_t *__restrict__ counts, const float *__restrict__ dprobs,
                      const float *__restrict__ dloss, int T, int B, int n_active, E *__restrict__ dlogits)
{
    const int l = threadIdx.x % L, b0 = 4 * l;
    const int per_block = blockDim.x / L;
    // the loss's part of the probabilities' gradient, the same for every token
    float w[4] = {0, 0, 0, 0};
    if (dloss) {
        int c[4], all = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c[e] = b0 + e < B ? counts[b0 + e] : 0;
            all += c[e];
        }
        all = over_token<L>(all, Add());
        const int n = counts[B];
        const double f = all > 0 && n > 0 ? (double)*dloss * n_active / ((double)all * n) : 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (float)(f * c[e]);
    }
    for (long long t = (long long)blockIdx.x * per_block + threadIdx.x / L; t < T; t += (long long)gridDim.x * per_block) {
        float p[4], g[4] = {0, 0, 0, 0};
        load4<kVec>(probs + t * B, b0, B, 0.0f, p);
        if (dprobs) load4<kVec>(dprobs + t * B, b0, B, 0.0f, g);
        float s = 0;
        // a probability of zero has no part in the sum and no gradient, whatever stands in dprobs there
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            g[e] = p[e] == 0.0f ? 0.0f : g[e] + w[e];
            s += p[e] * g[e];
        }
        s = over_token<L>(s, Add());
        float d[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] = p[e] == 0.0f ? 0.0f : p[e] * (g[e] - s);
        store4<kVec>(dlogits + t * B, b0, B, d);
    }
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

template <int L, typename E, bool kVec>
hipError_t launch_topk(const RouteArgs &a, int blocks)
{
    const bool stats = a.counts || a.loss;
    {
        ProfileScope ps(MLPMOE_KERNEL_ROUTE_TOPK, a.stream);
        if (stats)
            route_topk_kernel<L, E, kVec, true><<<blocks, kRouteThreads, 0, a.stream>>>(
                static_cast<const E *>(a.logits), a.ld, a.active, a.token_mask, a.T, a.B, a.k, a.route, a.probs, a.part_p,
                a.part_c, a.counts, a.loss, a.n_active);
        else
            route_topk_kernel<L, E, kVec, false><<<blocks, kRouteThreads, 0, a.stream>>>(
                static_cast<const E *>(a.logits), a.ld, a.active, a.token_mask, a.T, a.B, a.k, a.route, a.probs, nullptr,
                nullptr, nullptr, nullptr, a.n_active);
    }
    hipError_t e = launch_status("route_topk launch");
    if (e != hipSuccess || !stats || blocks == 1) return e;
    ProfileScope ps(MLPMOE_KERNEL_ROUTE_FINISH, a.stream);
    route_finish_kernel<<<1, 1024, 0, a.stream>>>(a.part_p, a.part_c, blocks, a.B, a.n_active, a.counts, a.loss);
    return launch_status("route_finish launch");
}

template <int L, typename E, bool kVec>
hipError_t launch_back(const RouteBackArgs &a)
{
    const int per_block = 256 / L;
    const long long want = ((long long)a.T + per_block - 1) / per_block;
    const int blocks = (int)(want < 2048 ? want : 2048);
    ProfileScope ps(MLPMOE_KERNEL_ROUTE_BACKWARD, a.stream);
    route_backward_kernel<L, E, kVec><<<blocks, 256, 0, a.stream>>>(a.probs, a.counts, a.dprobs, a.dloss, a.T, a.B, a.n_active,
                                                                  static_cast<E *>(a.dlogits));
    return launch_status("route_backward launch");
}

int lanes(int B) { return B <= 4 ? 1 : B <= 8 ? 2 : B <= 16 ? 4 : B <= 32 ? 8 : 16; }

template <typename E, bool kVec>
hipError_t topk_lanes(const RouteArgs &a, int blocks)
{
    switch (lanes(a.B)) {
    case 1: return launch_topk<1, E, kVec>(a, blocks);
    case 2: return launch_topk<2, E, kVec>(a, blocks);
    case 4: return launch_topk<4, E, kVec>(a, blocks);
    case 8: return launch_topk<8, E, kVec>(a, blocks);
    default: return launch_topk<16, E, kVec>(a, blocks);
    }
}

template <typename E, bool kVec>
hipError_t back_lanes(const RouteBackArgs &a)
{
    switch (lanes(a.B)) {
    case 1: return launch_back<1, E, kVec>(a);
    case 2: return launch_back<2, E, kVec>(a);
    case 4: return launch_back<4, E, kVec>(a);
    case 8: return launch_back<8, E, kVec>(a);
    default: return launch_back<16, E, kVec>(a);
    }
}

}  // namespace

int route_blocks(int T, int B)
{
    const int per_block = kRouteThreads / lanes(B);
    const long long want = ((long long)T + per_block - 1) / per_block;
    return (int)(want < 1 ? 1 : want < kRouteMaxBlocks ? want : kRouteMaxBlocks);
}

hipError_t launch_route_topk(const RouteArgs &a)
{
    const int blocks = route_blocks(a.T, a.B);
    const bool f32 = a.elem_bytes == 4;
    // rows of whole 4-branch pieces, each on its own alignment: one load and one store a lane
    const bool vec = a.B % 4 == 0 && a.ld % 4 == 0 && aligned(a.logits, f32 ? 16 : 8) && aligned(a.probs, 16) && aligned(a.route, 4);
    if (f32) return vec ? topk_lanes<float, true>(a, blocks) : topk_lanes<float, false>(a, blocks);
    return vec ? topk_lanes<uint16_t, true>(a, blocks) : topk_lanes<uint16_t, false>(a, blocks);
}

hipError_t launch_route_backward(const RouteBackArgs &a)
{
    const bool f32 = a.elem_bytes == 4;
    const bool vec = a.B % 4 == 0 && aligned(a.probs, 16) && aligned(a.dprobs, 16) && aligned(a.dlogits, f32 ? 16 : 8);
    if (f32) return vec ? back_lanes<float, true>(a) : back_lanes<float, false>(a);
    return vec ? back_lanes<uint16_t, true>(a) : back_lanes<uint16_t, false>(a);
}

}  // namespace mlpmoe
