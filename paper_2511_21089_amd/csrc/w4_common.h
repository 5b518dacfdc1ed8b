// Device code that the kernels on 4-bit weights share.
#pragma once

#include <mutex>

#include "internal.h"

namespace mlpmoe {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

typedef const __attribute__((address_space(1))) void *gptr_t;
typedef __attribute__((address_space(3))) void *lptr_t;

__device__ const uint32_t g_zero16[4] = {0, 0, 0, 0};

template <typename V>
__device__ __forceinline__ V ldg(const void *p)
{
    typedef const __attribute__((address_space(1))) V *gptr;
    return *(gptr)p;
}

// One wave-wide load of 16 bytes a lane straight into LDS: lane l's data lands at dst + 16 l.
__device__ __forceinline__ void dma16(const void *src, void *dst)
{
    __builtin_amdgcn_global_load_lds((gptr_t)src, (lptr_t)dst, 16, 0, 0);
}

// No memory operation moves across: the counted waits below rely on the order in which loads are issued.
__device__ __forceinline__ void keep_order()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Waits until at most N of this wave's loads are outstanding (they return in issue order) and none of its LDS operations.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}
// ... and then for the workgroup's other waves.  Written by hand because the compiler's own barrier waits for every load.
template <int N>
__device__ __forceinline__ void pipeline_barrier()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Eight elements of a block as bf16, in order.
__device__ __forceinline__ bf16x8 widen8(uint32_t w, float scale)
{
    union {
        bf16x2 p[4];
        bf16x8 v;
    } r;
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return r.v;
}

__device__ __forceinline__ float silu_mul(float g, float u)
{
    const float e = __builtin_amdgcn_exp2f(g * -1.4426950408889634f);
    return g * __builtin_amdgcn_rcpf(1.0f + e) * u;
}

__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

// K goes by steps of 128: a lane's 16 bytes of codes are a block of 32, group q = lane >> 4 takes block q of the step, and the
// j-th of the step's four MFMAs elements 8 j .. 8 j + 7 of it.  So a step's 16 pieces of x or H (8 values, 16 bytes) are read as
// piece 4 q + j by group q, out of LDS, where they are put by loads whose neighbouring lanes have neighbouring pieces: lanes that
// gather every fourth piece make four requests of one (medians of a trace, 4096 x 14336: w4_down, T = 16, 14.6 us instead of 13.9, w4_tile_down, T = 24,
// 14.3 instead of 13.7).
constexpr int kStepK = 128;

// A load of a step's codes of 16 rows: lane's row and its block of the step, four neighbouring lanes 64 bytes of a row; and where in
// the kilobyte of LDS that it fills the lane finds row r16, block q, so that 16 lanes read different banks.  (Against lanes that load
// what they use, neighbours in different rows, medians of a trace, 4096 x 14336: w4_down T = 1 8.0 us instead of 8.2, T = 16 12.5 and 13.9;
// w4_tile_gate_up T = 24 19.7 and 21.6, T = 500 110 both.)
struct CodeLane {
    int row, block, at;
    __device__ __forceinline__ CodeLane()
    {
        const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
        row = lane >> 2;
        block = (lane & 3) ^ (lane >> 4);
        at = (r16 * 4 + (q ^ (r16 >> 2))) * 16;
    }
};

// The neurons of a call's live branches (on, and some token of the workgroup's takes them).  Mostly they are one range that the
// host knows (kOneRun: no routing, one run of active branches); a workgroup then asks for weights at once, without having seen
// the table, whose arguments take a round trip.  Otherwise the table and the routes are looked through first, and what comes
// of it is kept in LDS.
struct Range {
    int beg, end;
};

// Live branches of the tokens t0 .. t0 + nt - 1, looked through by the whole workgroup (any: two words of LDS).  Ends with a
// barrier.
__device__ __forceinline__ unsigned long long live_of(const BranchTable &bt, const uint8_t *route, int t0, int nt, unsigned *any)
{
    if (!route) return bt.active;
    if (threadIdx.x < 2) any[threadIdx.x] = 0;
    __syncthreads();
    unsigned long long mine = 0;
    int b = (int)threadIdx.x % bt.B;
    const int add = (int)blockDim.x % bt.B;
    for (int i = threadIdx.x; i < nt * bt.B; i += blockDim.x) {
        if (route[(size_t)t0 * bt.B + i]) mine |= 1ULL << b;
        b += add;
        if (b >= bt.B) b -= bt.B;
    }
    if ((unsigned)mine) atomicOr(&any[0], (unsigned)mine);
    if (mine >> 32) atomicOr(&any[1], (unsigned)(mine >> 32));
    __syncthreads();
    return (any[0] | ((unsigned long long)any[1] << 32)) & bt.active;
}

// Lane b of every wave: the offsets of branch b.
struct OffsetLanes {
    int beg, end;
    __device__ __forceinline__ explicit OffsetLanes(const BranchTable &bt)
    {
        const int lane = threadIdx.x & 63;
        beg = bt.off[lane];
        end = bt.off[lane + 1];
    }
    __device__ __forceinline__ int first(int b) const { return __builtin_amdgcn_readlane(beg, b); }
    __device__ __forceinline__ int past(int b) const { return __builtin_amdgcn_readlane(end, b); }
};

// Live branches of at most 16 tokens, every wave for itself: all routes asked for at once.
__device__ __forceinline__ unsigned long long live_of_16(const BranchTable &bt, const uint8_t *route, int t0, int nt)
{
    if (!route) return bt.active;
    const int lane = threadIdx.x & 63, b = lane < bt.B ? lane : 0;
    unsigned any = 0;
#pragma unroll
    for (int t = 0; t < 16; ++t) any |= route[(size_t)(t0 + (t < nt ? t : 0)) * bt.B + b];
    return __ballot(any != 0 && lane < bt.B) & bt.active;
}

// The groups of G neurons, at multiples of G, that a live branch reaches into, numbered in order.
template <int G, bool kOneRun>
struct Groups {
    int beg, upto;           // lane b: first group that branch b adds to those of the live branches before it; their number with it
    int total;
    __device__ __forceinline__ Groups(const Range &run) : beg(run.beg / G), upto(0), total((run.end + G - 1) / G - run.beg / G) {}
    __device__ __forceinline__ Groups(const OffsetLanes &off, unsigned long long live)
    {
        const int lane = threadIdx.x & 63;
        const bool on = (live >> lane) & 1;
        const int lo = on ? off.beg : 0, hi = on ? off.end : 0;
        int end = hi > lo ? (hi + G - 1) / G : 0;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int v = __shfl_up(end, d);
            if (lane >= d && v > end) end = v;
        }
        int before = __shfl_up(end, 1);
        if (lane == 0) before = 0;
        beg = lo / G > before ? lo / G : before;
        upto = hi > lo ? end - beg : 0;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        total = __builtin_amdgcn_readlane(upto, 63);
    }
    // group number i (uniform, i < total)
    __device__ __forceinline__ int operator()(int i) const
    {
        if (kOneRun) return beg + i;
        const int b = __popcll(__ballot(upto <= i));
        return __builtin_amdgcn_readlane(beg, b) + i - (b > 0 ? __builtin_amdgcn_readlane(upto, b - 1) : 0);
    }
};

// h of 4 neurons n .. n + 3 (this lane's) of a group n0 .. n0 + G - 1 (uniform) from gate and up sums, as bf16: alpha SiLU(g) u, or 0 where
// the neuron's branch is off or the token does not take it.  store(8 bytes).  All lanes of the wave call it.
// The one rounding to fewer bits between the products, and the bf16 forward's as well: the second product runs on the bf16 matrix
// instructions, which a float h would need two or three times.  It adds to the result about what its own rounding to bf16 does:
// 4096 x 14336, N(0, 1) and N(0, 0.02^2), rms error over rms of the result 0.0024, 0.0017 of it the bf16 result's, 0.0016 h's.
template <int G, typename Takes, typename Store>
__device__ __forceinline__ void gated(const BranchLanes &br, const BranchTable &bt, int n0, int n, f32x4 g, f32x4 u, Takes takes, Store store)
{
    int b = br.branch(n0), end = br.next(b);
    f32x4 h = {0, 0, 0, 0};
#pragma unroll 1
    for (int beg = n0; beg < n0 + G; beg = end, ++b, end = br.next(b)) {         // mostly once: the group lies in one branch
        if (!((bt.active >> b) & 1) || !takes(b)) continue;
        const float alpha = br.alpha(b);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e >= beg && n + e < end) h[e] = alpha * silu_mul(g[e], u[e]);
    }
    store(uint2{(uint32_t)to_bf16(h[0]) | (uint32_t)to_bf16(h[1]) << 16, (uint32_t)to_bf16(h[2]) | (uint32_t)to_bf16(h[3]) << 16});
}

// The down projection reads H by whole steps of 128 neurons.  Groups of G that a live branch reaches into are written whole;
// here the rest of such a step is set to zero, and all of the branches that only other tokens of a down projection's workgroup
// take (wide, which has live in it).  The branches are shared out to the workgroups (first, step), their tokens to its waves: one
// workgroup with all of them was the last to end (gate+up, routed, T = 16: 896 x 4864 12.0 -> 9.5 us, 4096 x 14336 19.4 -> 15.6).
__device__ __forceinline__ void clear_range(uint16_t *H, int ldh, int nt, int from, int to, int wave, int nw)
{
    for (int t = wave; t < nt; t += nw)
        for (int p = from / 8 * 8 + (threadIdx.x & 63) * 8; p < to; p += 512) {
            uint16_t *h = H + (size_t)t * ldh + p;
            if (p >= from && p + 8 <= to)
                *reinterpret_cast<u32x4 *>(h) = u32x4{0, 0, 0, 0};
            else
#pragma unroll 1
                for (int e = 0; e < 8; ++e)
                    if (p + e >= from && p + e < to) h[e] = 0;
        }
}
__device__ __forceinline__ void clear_edges(const Range &run, uint16_t *H, int ldh, int nt, int wave, int nw)
{
    if (run.beg % kStepK) clear_range(H, ldh, nt, run.beg / kStepK * kStepK, run.beg, wave, nw);
    if (run.end % kStepK) clear_range(H, ldh, nt, run.end, (run.end + kStepK - 1) / kStepK * kStepK, wave, nw);
}
__device__ __forceinline__ void clear_edges(const OffsetLanes &off, int B, unsigned long long live, unsigned long long wide,
                                            uint16_t *H, int ldh, int nt, int wave, int nw, int first, int step)
{
#pragma unroll 1
    for (int b = first; b <= B; b += step) {                       // past the last branch: the rest of its step
        const int from = b < B ? off.first(b) : off.past(B - 1), to = b < B ? off.past(b) : ldh;
        if ((b < B && ((live >> b) & 1)) || to == from) continue;
        const int up = (from + kStepK - 1) / kStepK * kStepK, down = to / kStepK * kStepK;
        const int end = up < to && !(b < B && ((wide >> b) & 1)) ? up : to, beg = down > end ? down : end;
        clear_range(H, ldh, nt, from, end, wave, nw);
        clear_range(H, ldh, nt, beg, to, wave, nw);
    }
}

// A bit a block of the K axis of W_down: whether a live branch has a neuron in it.  Ends with a barrier.
__device__ __forceinline__ void mark_blocks(const OffsetLanes &off, unsigned long long live, uint32_t *bits, int blocks)
{
#pragma unroll 1
    for (int i = threadIdx.x; i < (blocks + 31) / 32; i += blockDim.x) {
        uint32_t w = 0;
        for (unsigned long long m = live; m != 0; m &= m - 1) {
            const int b = __builtin_ctzll(m), lo = off.first(b), hi = off.past(b);
            // blocks lo / 32 .. (hi - 1) / 32 of this word's 32 i .. 32 i + 31
            const int from = lo / 32 - 32 * i, to = (hi + 31) / 32 - 32 * i;
            const uint32_t below = to <= 0 ? 0u : to >= 32 ? ~0u : (1u << to) - 1u;
            const uint32_t less = from <= 0 ? 0u : from >= 32 ? ~0u : (1u << from) - 1u;
            if (hi > lo) w |= below & ~less;
        }
        bits[i] = w;
    }
    __syncthreads();
}

// The steps of K with a live block, in order: every wave counts them, all write the same list.  Ends with a barrier.
__device__ __forceinline__ int list_steps(const uint32_t *bits, int all, uint16_t *list)
{
    int n = 0;
#pragma unroll 1
    for (int s = 0; s < all; s += 64) {
        const int st = s + (threadIdx.x & 63);
        const bool on = st < all && ((bits[st / 8] >> (st % 8 * 4)) & 15u) != 0;
        const unsigned long long m = __ballot(on);
        if (on) list[n + __popcll(m & ((1ULL << (threadIdx.x & 63)) - 1))] = (uint16_t)st;
        n += __popcll(m);
    }
    __syncthreads();
    return n;
}

// Lets a kernel have `bytes` of LDS on the current device: the runtime is asked when a call needs more than those before it
// (2 us a call otherwise, of 8 for a launch or two).
template <auto kernel>
hipError_t allow_lds(int bytes, const char *what)
{
    static std::mutex mu;
    static int given[64] = {0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return note_hip_error("hipGetDevice", e);
    if (dev < 0 || dev >= 64) return note_hip_error("device index", hipErrorInvalidDevice);
    std::lock_guard<std::mutex> lock(mu);
    if (given[dev] >= bytes) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return note_hip_error(what, e);
    given[dev] = bytes;
    return hipSuccess;
}

}  // namespace
}  // namespace mlpmoe
