// The router of a routed layer: which branches every token takes, the softmax probabilities, how many tokens take each
// branch, the balance loss, and the gradient of the logits.
//
//   p[t, b] = exp(x[t, b] - max) / sum        over the active branches of a token that counts
//   loss    = A * sum_b f_b P_b,   f_b = counts[b] / sum counts,   P_b = mean over the counted tokens of p[t, b]
//   dx      = p (.) (g - sum_b p g),          g[t, b] = dprobs[t, b] + dloss * A * f_b / N
//
// A row is at most 64 logits, so a token is worked on by L = 1 .. 16 neighbouring lanes that hold four branches each in
// registers; everything a token needs crosses lanes by DPP inside 16 lanes.  Logits are read once, probabilities and route
// bytes written once.  Few tokens: a launch (1.9 us), or two (4000 x 16: 4.3 and 3.8 us).
#include "internal.h"

namespace mlpmoe {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint16_t u16x4;

constexpr float kNegInf = -__builtin_inff();

template <int kCtrl>
__device__ __forceinline__ int dpp(int v)
{
    return __builtin_amdgcn_update_dpp(0, v, kCtrl, 0xf, 0xf, true);
}
template <int kCtrl>
__device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, dpp<kCtrl>(__builtin_bit_cast(int, v)));
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
    __device__ __forceinline__ int operator()(int a, int b) const { return a > b ? a : b; }
};
struct Or {
    __device__ __forceinline__ int operator()(int a, int b) const { return a | b; }
};

// Logits as integers in the same order, both zeros alike and what is not a number as -inf: the largest of two is one
// instruction that takes its operand across lanes, where a float's needs two more to be quiet about not-a-numbers.
__device__ __forceinline__ int order(float x)
{
    const int i = __builtin_bit_cast(int, (x > kNegInf ? x : kNegInf) + 0.0f);
    return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float value(int o) { return __builtin_bit_cast(float, o ^ ((o >> 31) & 0x7fffffff)); }

// One lane out of each L: of the lanes that are set, the lowest of each L.  Every L has one set, or none and then no later one
// either, so the carry of a sum stays where it began.
template <int L>
__device__ __forceinline__ bool lowest(bool set)
{
    if (L == 1) return set;
    constexpr unsigned long long kOnes = ~0ULL / ((1ULL << L) - 1);
    const unsigned long long m = __ballot(set);
    return __builtin_amdgcn_inverse_ballot_w64(m & (~m + kOnes));
}

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

template <typename V>
__device__ __forceinline__ V over_wave(V v)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
    return v;
}

// Counts and loss from the sums over all tokens: lane b of the first wave has branch b's probabilities and count (zeros past B),
// every lane the number of tokens.
__device__ __forceinline__ void finish(double p, int c, int tokens, int B, int n_active, int32_t *counts, float *loss)
{
    const int lane = threadIdx.x;
    if (counts && lane < B) counts[lane] = c;
    if (counts && lane == 0) counts[B] = tokens;
    const double sum = over_wave(p * (double)c), taken = over_wave((double)c);
    // nothing taken: sum is 0, or not a number if a probability is none
    if (loss && lane == 0) *loss = (float)(taken > 0 ? (double)n_active * sum / (taken * (double)tokens) : sum);
}

constexpr int kRouteThreads = 1024;

// A token on L lanes, four branches a lane; a wave's next tokens are asked for before these are worked on.  Bound by vector
// instructions, some 140 for four tokens of 64 branches and 11 a round of the selection: 131072 x 64 floats, k = 8, with
// probabilities and sums 20.8 us, 3.6 TB/s, some 12 of them instructions and the rest the rounds' chain, each waiting for the one before (30.6 with float maxima, each three instructions a step instead of one, and the last
// token's byte waited for before anything else); twice the blocks 20.0, and 5.5 us instead of 3.8 for the kernel after it.
// kStats: also what the counts and the loss need: with one block the result, else the block's partial sums, rows of B and the
// number of tokens.
template <int L, typename E, bool kVec, bool kStats>
__global__ void __launch_bounds__(kRouteThreads)
route_topk_kernel(const E *__restrict__ logits, int ld, unsigned long long active, const uint8_t *__restrict__ token_mask,
                  int T, int B, int k, uint8_t *__restrict__ route, float *__restrict__ probs, RoutePart *__restrict__ part,
                  int *__restrict__ part_n, int32_t *__restrict__ counts, float *__restrict__ loss, int n_active)
{
    const int l = threadIdx.x % L, b0 = 4 * l;
    const int per_block = blockDim.x / L;
    const long long stride = (long long)gridDim.x * per_block;
    float sum_p[4] = {0, 0, 0, 0};
    int sum_c[4] = {0, 0, 0, 0}, sum_n = 0;
    const unsigned on = (unsigned)(active >> b0) & 15u;

    float ahead[4];
    int real = 1;
    long long t = (long long)blockIdx.x * per_block + threadIdx.x / L;
    const E *row = logits + t * ld;
    const long long row_step = stride * ld, out_step = stride * B;
    const uint8_t *mask = token_mask + (token_mask ? t : 0);
    float *to_probs = probs + (probs ? t * B : 0);
    uint8_t *to_route = route + t * B;
    if (t < T) {
        load4<kVec>(row, b0, B, kNegInf, ahead);
        if (token_mask) real = *mask;
    }
#pragma unroll 1
    for (; t < T; t += stride) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = ((on >> e) & 1u) && real != 0 ? ahead[e] : kNegInf;
        if (t + stride < T) {
            row += row_step;
            load4<kVec>(row, b0, B, kNegInf, ahead);
            if (token_mask) real = *(mask += stride);
        }
        int o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = order(x[e]);
        // sorted, s[0] the largest
        const Max more;
        auto less = [](int a, int b) { return a < b ? a : b; };
        int s[4];
        {
            const int a = more(o[0], o[1]), b = less(o[0], o[1]), c = more(o[2], o[3]), d = less(o[2], o[3]);
            const int e = less(a, c), f = more(b, d);
            s[0] = more(a, c);
            s[1] = more(e, f);
            s[2] = less(e, f);
            s[3] = less(b, d);
        }
        const int none = order(kNegInf);
        const int most = over_token<L>(s[0], more);
        bool used = most > none;

        float p[4] = {0, 0, 0, 0};
        if (probs || kStats) {
            // A token without a number to take is an empty row only if all of its branches are barred: with a not-a-number it counts,
            // and m = -inf makes the probabilities of what is not barred not-a-numbers.  Looked at only where the wave has such a
            // token: padding, mostly.
            if (__ballot(!used) != 0) {
                const bool nan = x[0] != x[0] || x[1] != x[1] || x[2] != x[2] || x[3] != x[3];
                used = over_token<L>((int)(used || nan), Or()) != 0;
            }
            const float m = value(most);
            float sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[e] = __expf(x[e] - m);
                sum += p[e];
            }
            sum = over_token<L>(sum, Add());
            // a reciprocal good to one unit in the last place, then one step of Newton's method
            float inv = __builtin_amdgcn_rcpf(sum);
            inv = inv * (2.0f - sum * inv);
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = used && x[e] != kNegInf ? p[e] * inv : 0.0f;
            if (probs) store4<kVec>(to_probs, b0, B, p);
        }

        // The k first in the order (larger logit, then lower index).  Every round takes the largest head of the token's lanes, of
        // the lowest lane that has it; what is not there (-inf) comes last and is left out at the end.
        int rank[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int f = e + 1; f < 4; ++f) {
                const int later = o[e] >= o[f];
                rank[f] += later;
                rank[e] += 1 - later;
            }
        int taken = 0, best = most;
#pragma unroll 1
        for (int i = k; i > 0; --i) {
            const bool first = lowest<L>(s[0] == best);
            taken += first;
            s[0] = first ? s[1] : s[0];
            s[1] = first ? s[2] : s[1];
            s[2] = first ? s[3] : s[2];
            s[3] = first ? none : s[3];
            best = over_token<L>(s[0], more);
        }
        uint32_t bytes = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) bytes |= (rank[e] < taken && o[e] > none ? 1u : 0u) << (8 * e);
        if constexpr (kVec) {
            if (b0 < B) *reinterpret_cast<uint32_t *>(to_route + b0) = bytes;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (b0 + e < B) to_route[b0 + e] = (uint8_t)(bytes >> (8 * e));
        }
        if constexpr (kStats) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum_p[e] += p[e];
                sum_c[e] += (int)((bytes >> (8 * e)) & 1u);
            }
            sum_n += used;
        }
        to_probs += probs ? out_step : 0;
        to_route += out_step;
    }

    if constexpr (kStats) {
        // over the tokens of a wave by lanes, then over the waves in their order
        __shared__ float s_p[kRouteThreads / 64][64];
        __shared__ int s_c[kRouteThreads / 64][64], s_n[kRouteThreads / 64];
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
#pragma unroll
        for (int d = 32; d >= L; d /= 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum_p[e] += __shfl_xor(sum_p[e], d);
                sum_c[e] += __shfl_xor(sum_c[e], d);
            }
            sum_n += __shfl_xor(sum_n, d);
        }
        if (lane < L) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s_p[wave][b0 + e] = sum_p[e], s_c[wave][b0 + e] = sum_c[e];
        }
        if (lane == 0) s_n[wave] = sum_n;
        __syncthreads();
        if (wave > 0) return;
        float p = 0;
        int c = 0, n = 0;
        for (int w = 0; w < waves; ++w) {
            if (lane < 4 * L) p += s_p[w][lane], c += s_c[w][lane];
            n += s_n[w];
        }
        if (gridDim.x == 1) {
            finish((double)p, c, n, B, n_active, counts, loss);
        } else {
            if (lane < B) part[(size_t)blockIdx.x * B + lane] = RoutePart{p, c};
            if (lane == 0) part_n[blockIdx.x] = n;
        }
    }
}

// The blocks' partial sums, a lane a branch and a wave every 16th block, all asked for at once: the latency of one load and of the
// instructions' first fetch.  Probabilities in double, since the number of tokens goes to 2^24.
__global__ void __launch_bounds__(1024)
route_finish_kernel(const RoutePart *__restrict__ part, const int *__restrict__ part_n, int blocks, int B, int n_active,
                    int32_t *__restrict__ counts, float *__restrict__ loss)
{
    __shared__ double s_p[16][64];
    __shared__ int s_c[16][64], s_n[kRouteMaxBlocks / 64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    constexpr int EACH = kRouteMaxBlocks / 16;
    const int at = threadIdx.x < (unsigned)blocks ? part_n[threadIdx.x] : 0;
    RoutePart v[EACH];
    const RoutePart *from = part + (lane < B ? lane : 0);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int block = wave + 16 * i;
        v[i] = from[(block < blocks ? block : 0) * B];
    }
    double p = 0;
    int c = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const bool in = wave + 16 * i < blocks;
        p += in ? (double)v[i].p : 0.0;
        c += in ? v[i].c : 0;
    }
    s_p[wave][lane] = p;
    s_c[wave][lane] = c;
    if (wave < kRouteMaxBlocks / 64) {
        const int n = over_wave(at);
        if (lane == 0) s_n[wave] = n;
    }
    __syncthreads();
    if (wave > 0) return;
    p = 0, c = 0;
    int n = 0;
    for (int w = 0; w < 16; ++w) p += s_p[w][lane], c += s_c[w][lane];
    for (int w = 0; w < kRouteMaxBlocks / 64; ++w) n += s_n[w];
    finish(lane < B ? p : 0.0, lane < B ? c : 0, n, B, n_active, counts, loss);
}

// Memory bound: 131072 x 64 floats 17.4 us, 5.8 TB/s.
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

int lanes(int B) { return B <= 4 ? 1 : B <= 8 ? 2 : B <= 16 ? 4 : B <= 32 ? 8 : 16; }

// Threads and blocks of a call with counts or loss.  One block, which needs no second kernel, while a thread has at most two
// tokens; then 256 threads while that gives at most kRouteMaxBlocks blocks; then 1024, which fill the chip with a block on every CU.
int route_threads(int T, int B)
{
    const long long all = (long long)T * lanes(B);
    return all > 2 * kRouteThreads && all <= 256LL * kRouteMaxBlocks ? 256 : kRouteThreads;
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

template <int L, typename E, bool kVec>
hipError_t launch_topk(const RouteArgs &a)
{
    const int blocks = route_blocks(a.T, a.B);
    const bool stats = a.counts || a.loss;
    const long long want = ((long long)a.T * L + 255) / 256;
    const int free_blocks = (int)(want < 2048 ? want : 2048);
    {
        ProfileScope ps(MLPMOE_KERNEL_ROUTE_TOPK, a.stream);
        if (stats)
            route_topk_kernel<L, E, kVec, true><<<blocks, route_threads(a.T, a.B), 0, a.stream>>>(
                static_cast<const E *>(a.logits), a.ld, a.active, a.token_mask, a.T, a.B, a.k, a.route, a.probs, a.part,
                a.part_n, a.counts, a.loss, a.n_active);
        else
            route_topk_kernel<L, E, kVec, false><<<free_blocks, 256, 0, a.stream>>>(
                static_cast<const E *>(a.logits), a.ld, a.active, a.token_mask, a.T, a.B, a.k, a.route, a.probs, nullptr,
                nullptr, nullptr, nullptr, a.n_active);
    }
    hipError_t e = launch_status("route_topk launch");
    if (e != hipSuccess || !stats || blocks == 1) return e;
    ProfileScope ps(MLPMOE_KERNEL_ROUTE_FINISH, a.stream);
    route_finish_kernel<<<1, 1024, 0, a.stream>>>(a.part, a.part_n, blocks, a.B, a.n_active, a.counts, a.loss);
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

template <typename E, bool kVec>
hipError_t topk_lanes(const RouteArgs &a)
{
    switch (lanes(a.B)) {
    case 1: return launch_topk<1, E, kVec>(a);
    case 2: return launch_topk<2, E, kVec>(a);
    case 4: return launch_topk<4, E, kVec>(a);
    case 8: return launch_topk<8, E, kVec>(a);
    default: return launch_topk<16, E, kVec>(a);
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

int route_most_blocks(int T, int B)
{
    const long long all = (long long)T * lanes(B), want = (all + 255) / 256;
    return (int)(all <= 2 * kRouteThreads ? 1 : want < kRouteMaxBlocks ? want : kRouteMaxBlocks);
}

int route_blocks(int T, int B)
{
    const long long all = (long long)T * lanes(B);
    if (all <= 2 * kRouteThreads) return 1;
    const int threads = route_threads(T, B);
    const long long want = (all + threads - 1) / threads;
    return (int)(want < kRouteMaxBlocks ? want : kRouteMaxBlocks);
}

hipError_t launch_route_topk(const RouteArgs &a)
{
    const bool f32 = a.elem_bytes == 4;
    // rows of whole 4-branch pieces, each on its own alignment: one load and one store a lane
    const bool vec = a.B % 4 == 0 && a.ld % 4 == 0 && aligned(a.logits, f32 ? 16 : 8) && aligned(a.probs, 16) && aligned(a.route, 4);
    if (f32) return vec ? topk_lanes<float, true>(a) : topk_lanes<float, false>(a);
    return vec ? topk_lanes<uint16_t, true>(a) : topk_lanes<uint16_t, false>(a);
}

hipError_t launch_route_backward(const RouteBackArgs &a)
{
    const bool f32 = a.elem_bytes == 4;
    const bool vec = a.B % 4 == 0 && aligned(a.probs, 16) && aligned(a.dprobs, 16) && aligned(a.dlogits, f32 ? 16 : 8);
    if (f32) return vec ? back_lanes<float, true>(a) : back_lanes<float, false>(a);
    return vec ? back_lanes<uint16_t, true>(a) : back_lanes<uint16_t, false>(a);
}

}  // namespace mlpmoe
