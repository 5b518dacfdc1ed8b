// The branched SwiGLU forward on 4-bit weights, and the conversion of weight matrices to and from them.
//
// Storage (the public Microscaling format MXFP4): 32 neighbours of a row share a scale 2^(s - 127), s a byte; an element is 4
// bits, sign and magnitude, the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6; low nibble first.  A 16-byte piece of a row is exactly
// one block, so a lane that loads 16 bytes needs one scale.  v_cvt_scalef32_pk_bf16_fp4 turns two elements and the scale into
// two bf16 values, exactly (at most two significant bits), so a weight costs half a vector instruction, and the products run
// on v_mfma_f32_16x16x32_bf16 with x and H as they are in the bf16 forward:
//
//   w4_gate_up   h[t, n] = bf16(alpha_b SiLU(g) u), g and u in float
//   w4_down      out[t, m] = sum_n h[t, n] W_down[m, n] in float
//
// Both are bound by the stream of weights from HBM while few tokens share it.
#include "internal.h"

namespace mlpmoe {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

__device__ const uint32_t g_zero16[4] = {0, 0, 0, 0};

template <typename V>
__device__ __forceinline__ V ldg(const void *p)
{
    typedef const __attribute__((address_space(1))) V *gptr;
    return *(gptr)p;
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

// Branches that are on and that some token of t0 .. t0 + nt - 1 takes, as a word; the same in every lane.
__device__ __forceinline__ unsigned long long live_branches(const BranchTable &bt, const uint8_t *route, int t0, int nt)
{
    if (!route) return bt.active;
    const int b = threadIdx.x & 63;
    bool any = false;
    if (b < bt.B)
        for (int t = 0; t < nt; ++t) any = any || route[(size_t)(t0 + t) * bt.B + b] != 0;
    return __ballot(any) & bt.active;
}

constexpr int kRows = 8;                 // neurons of a gate+up tile: MFMA rows 0-7 W_gate, 8-15 W_up
constexpr int kStep = 512;               // K of a wave's step: each of its four groups of 16 lanes takes 128, four blocks
constexpr int kPad = 8;                  // x rows in LDS are this much longer, so that 16 of them start on different banks

// What a wave loads for a step: four blocks of a row a lane, and their scales.
struct Step {
    u32x4 w[4];
    uint32_t s;
};

// unit: this lane's group of four blocks (128 elements) of the row; blocks: how many blocks the row has.
__device__ __forceinline__ Step load_step(const uint8_t *codes, const uint8_t *scales, int unit, int blocks)
{
    Step r;
    r.s = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int b = unit * 4 + j;
        const bool ok = b < blocks;
        r.w[j] = ldg<u32x4>(ok ? codes + (size_t)b * 16 : reinterpret_cast<const uint8_t *>(g_zero16));
        r.s |= (uint32_t)ldg<uint8_t>(ok ? scales + b : reinterpret_cast<const uint8_t *>(g_zero16)) << (8 * j);
    }
    return r;
}

// Grid (WGs, token tiles of 16).  A wave works out tiles of 8 neurons, wave w of workgroup g the tiles w * grid + g and so on,
// so that what live branches there are is spread over the chip.  x goes through LDS in chunks of kc.
__global__ void __launch_bounds__(512)
w4_gate_up(const uint16_t *__restrict__ x, int T, int K, int kc, const uint8_t *__restrict__ gc, const uint8_t *__restrict__ gs,
           const uint8_t *__restrict__ uc, const uint8_t *__restrict__ us, uint16_t *__restrict__ H, int ldh,
           const uint8_t *__restrict__ route, BranchTable bt)
{
    extern __shared__ __attribute__((aligned(16))) uint16_t s_x[];
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int t0 = 16 * blockIdx.y, nt = T - t0 < 16 ? T - t0 : 16;
    const unsigned long long live = live_branches(bt, route, t0, nt);

    // lane b: tiles of branch b and all before it
    const int width = lane < bt.B ? bt.off[lane + 1] - bt.off[lane] : 0;
    int upto = (live >> lane) & 1 ? (width + kRows - 1) / kRows : 0;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(upto, d);
        if (lane >= d) upto += v;
    }
    const int tiles = __builtin_amdgcn_readlane(upto, 63);

    // H of neurons that no token takes but that share a block of W_down's row with one that is taken has to be zero
    if (blockIdx.x == 0)
        for (int b = wave; b < bt.B; b += nw) {
            if ((live >> b) & 1) continue;
            const int lo = bt.off[b], hi = bt.off[b + 1];
            const int end = (lo + 31) / 32 * 32 < hi ? (lo + 31) / 32 * 32 : hi;
            const int beg = hi / 32 * 32 > end ? hi / 32 * 32 : end;
            for (int t = 0; t < nt; ++t) {
                if (lane < end - lo) H[(size_t)(t0 + t) * ldh + lo + lane] = 0;
                if (lane < hi - beg) H[(size_t)(t0 + t) * ldh + beg + lane] = 0;
            }
        }

    const int blocks = K / 32;
    const int ldx = kc + kPad;
    const int passes = (tiles + nw * (int)gridDim.x - 1) / (nw * (int)gridDim.x);
    const uint16_t *xr = s_x + (r16 < nt ? r16 : 0) * ldx + q * 128;
    for (int pass = 0; pass < passes; ++pass) {
        const int idx = (pass * nw + wave) * gridDim.x + blockIdx.x;
        const bool have = idx < tiles;
        // the branch is the first whose tiles reach past idx
        const int b = have ? __popcll(__ballot(upto <= idx)) : 0;
        const int before = b > 0 ? __builtin_amdgcn_readlane(upto, b - 1) : 0;
        const int n0 = have ? bt.off[b] + (idx - before) * kRows : 0;
        const int n_end = have ? bt.off[b + 1] : 1;
        int n = n0 + (r16 & 7);
        n = n < n_end ? n : n_end - 1;                   // rows past the branch are computed and not stored
        const uint8_t *codes = (r16 < 8 ? gc : uc) + (size_t)n * (K / 2);
        const uint8_t *scales = (r16 < 8 ? gs : us) + (size_t)n * blocks;

        f32x4 acc = {0, 0, 0, 0};
        for (int k0 = 0; k0 < K; k0 += kc) {
            const int kn = K - k0 < kc ? K - k0 : kc;
            if (pass == 0 || kc < K) {
                __syncthreads();
                const int pieces = (kc + 7) / 8;         // of 8 values; past K zeros
                for (int i = threadIdx.x; i < nt * pieces; i += blockDim.x) {
                    const int t = i / pieces, c = (i - t * pieces) * 8;
                    u32x4 v = {0, 0, 0, 0};
                    if (c < kn) v = ldg<u32x4>(x + (size_t)(t0 + t) * K + k0 + c);
                    *reinterpret_cast<u32x4 *>(s_x + t * ldx + c) = v;
                }
                __syncthreads();
            }
            if (!have) continue;
            for (int s = 0; s * kStep < kn; ++s) {
                const Step st = load_step(codes, scales, k0 / 128 + s * 4 + q, blocks);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float sc = scale_of((st.s >> (8 * j)) & 255u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bf16x8 xv = *reinterpret_cast<const bf16x8 *>(xr + s * kStep + j * 32 + i * 8);
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(st.w[j][i], sc), xv, acc, 0, 0, 0);
                    }
                }
            }
        }
        if (!have) continue;
        // rows 4q .. 4q + 3 of token r16: gate in lanes q < 2, up in those 32 lanes on
        const float alpha = bt.alpha[b];
        const int t = t0 + r16;
        const bool take = r16 < nt && (!route || route[(size_t)t * bt.B + b] != 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float up = __shfl_xor(acc[i], 32);
            const int m = n0 + 4 * q + i;
            if (q < 2 && r16 < nt && m < n_end) H[(size_t)t * ldh + m] = take ? to_bf16(alpha * silu_mul(acc[i], up)) : 0;
        }
    }
}

constexpr int kDownWaves = 16;

// Grid (tiles of 16 features, token tiles of 16).  The waves of a workgroup take turns with the steps of K, and their sums are
// added in the order of the waves.  A block of the K axis is live if a live branch has a neuron in it; the others are not read.
__global__ void __launch_bounds__(kDownWaves * 64)
w4_down(const uint16_t *__restrict__ H, int ldh, int T, int K, const uint8_t *__restrict__ dc, const uint8_t *__restrict__ ds,
        int d_model, void *__restrict__ out, int out_bf16, const uint8_t *__restrict__ route, BranchTable bt, int dense)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t s_live[];      // a bit a block, unless all are live
    __shared__ float red[kDownWaves][256];
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t0 = 16 * blockIdx.y, nt = T - t0 < 16 ? T - t0 : 16;
    const int blocks = K / 32;
    if (!dense) {
        const unsigned long long live = live_branches(bt, route, t0, nt);
        for (int i = threadIdx.x; i < (blocks + 31) / 32; i += blockDim.x) s_live[i] = 0;
        __syncthreads();
        for (int b = 0; b < bt.B; ++b) {
            const int lo = bt.off[b], hi = bt.off[b + 1];
            if (!((live >> b) & 1) || hi == lo) continue;
            for (int i = lo / 32 + threadIdx.x; i <= (hi - 1) / 32; i += blockDim.x) atomicOr(&s_live[i / 32], 1u << (i & 31));
        }
        __syncthreads();
    }
    const int m0 = blockIdx.x * 16;
    const int m = m0 + r16 < d_model ? m0 + r16 : d_model - 1;
    const uint8_t *codes = dc + (size_t)m * (K / 2), *scales = ds + (size_t)m * blocks;
    const uint16_t *hr = H + (size_t)(t0 + (r16 < nt ? r16 : 0)) * ldh;
    const uint8_t *zero = reinterpret_cast<const uint8_t *>(g_zero16);
    f32x4 acc = {0, 0, 0, 0};
    for (int s = wave; s * kStep < K; s += kDownWaves) {
        const int unit = s * 4 + q;
        unsigned ok = 0;
        if (unit * 4 < blocks) ok = dense ? 15u : (s_live[unit / 8] >> (unit % 8 * 4)) & 15u;
        if (blocks - unit * 4 < 4 && ok) ok &= (1u << (blocks - unit * 4)) - 1u;
        if (__ballot(ok != 0) == 0) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool on = (ok >> j) & 1u;
            const int b = unit * 4 + j;
            const u32x4 w = ldg<u32x4>(on ? codes + (size_t)b * 16 : zero);
            const float sc = scale_of(ldg<uint8_t>(on ? scales + b : zero));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x8 hv = ldg<bf16x8>(on ? reinterpret_cast<const uint8_t *>(hr + b * 32 + i * 8) : zero);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[i], sc), hv, acc, 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) red[wave][r16 * 16 + 4 * q + i] = acc[i];
    __syncthreads();
    if (threadIdx.x < 256) {
        const int t = threadIdx.x >> 4, f = m0 + (threadIdx.x & 15);
        float v = 0;
#pragma unroll
        for (int w = 0; w < kDownWaves; ++w) v += red[w][threadIdx.x];
        if (t < nt && f < d_model) {
            const size_t at = (size_t)(t0 + t) * d_model + f;
            if (out_bf16)
                static_cast<uint16_t *>(out)[at] = to_bf16(v);
            else
                static_cast<float *>(out)[at] = v;
        }
    }
}

// --- conversion ------------------------------------------------------------------------------------------------------
// A lane takes 8 of a block's 32 values; the block's largest magnitude crosses its four lanes by DPP.
template <typename E>
__global__ void __launch_bounds__(256)
w4_quantize_kernel(const E *__restrict__ W, size_t pieces, uint32_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < pieces; i += (size_t)gridDim.x * blockDim.x) {
        float v[8];
        if constexpr (sizeof(E) == 4) {
            const f32x4 a = ldg<f32x4>(W + i * 8), b = ldg<f32x4>(W + i * 8 + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
        } else {
            const u32x4 a = ldg<u32x4>(W + i * 8);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[2 * e] = __builtin_bit_cast(float, a[e] << 16);
                v[2 * e + 1] = __builtin_bit_cast(float, a[e] & 0xffff0000u);
            }
        }
        // magnitudes compare as their bits; what is not finite has the largest
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;
            top = u > top ? u : top;
        }
        uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)top, (int)top, 0xB1, 0xf, 0xf, false);
        top = o > top ? o : top;
        o = (uint32_t)__builtin_amdgcn_update_dpp((int)top, (int)top, 0x4E, 0xf, 0xf, false);
        top = o > top ? o : top;
        // exponent of the largest value less that of 4 and 6, the largest elements; 255 (not a number) if it is not finite
        const int ex = (int)(top >> 23);
        const int s = ex == 255 ? 255 : ex > 3 ? ex - 2 : 1;
        const float scale = __builtin_bit_cast(float, (uint32_t)(s == 255 ? 254 : s) << 23);
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
        codes[i] = s == 255 ? 0u : w;
        if ((i & 3) == 0) scales[i >> 2] = (uint8_t)s;
    }
}

template <typename E>
__global__ void __launch_bounds__(256)
w4_dequantize_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales, size_t pieces, E *__restrict__ W)
{
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < pieces; i += (size_t)gridDim.x * blockDim.x) {
        const bf16x8 v = widen8(codes[i], scale_of(scales[i >> 2]));
        if constexpr (sizeof(E) == 4) {
            f32x4 a, b;
#pragma unroll
            for (int e = 0; e < 4; ++e) a[e] = (float)v[e], b[e] = (float)v[4 + e];
            *reinterpret_cast<f32x4 *>(W + i * 8) = a;
            *reinterpret_cast<f32x4 *>(W + i * 8 + 4) = b;
        } else {
            *reinterpret_cast<bf16x8 *>(W + i * 8) = v;
        }
    }
}

unsigned convert_blocks(size_t pieces)
{
    const size_t want = (pieces + 255) / 256;
    return (unsigned)(want < 8192 ? want : 8192);
}

// Bytes of LDS for x: all of K if 16 rows (fewer for fewer tokens) fit, else chunks.
constexpr int kXBytes = 144 * 1024;

}  // namespace

hipError_t launch_w4_quantize(const void *W, size_t n, int elem_bytes, uint8_t *codes, uint8_t *scales, hipStream_t s)
{
    ProfileScope ps(MLPMOE_KERNEL_W4_CONVERT, s);
    const size_t pieces = n / 8;
    if (elem_bytes == 4)
        w4_quantize_kernel<float><<<convert_blocks(pieces), 256, 0, s>>>(static_cast<const float *>(W), pieces,
                                                                       reinterpret_cast<uint32_t *>(codes), scales);
    else
        w4_quantize_kernel<uint16_t><<<convert_blocks(pieces), 256, 0, s>>>(static_cast<const uint16_t *>(W), pieces,
                                                                          reinterpret_cast<uint32_t *>(codes), scales);
    return launch_status("w4_quantize launch");
}

hipError_t launch_w4_dequantize(const uint8_t *codes, const uint8_t *scales, size_t n, int elem_bytes, void *W, hipStream_t s)
{
    ProfileScope ps(MLPMOE_KERNEL_W4_CONVERT, s);
    const size_t pieces = n / 8;
    const uint32_t *c = reinterpret_cast<const uint32_t *>(codes);
    if (elem_bytes == 4)
        w4_dequantize_kernel<float><<<convert_blocks(pieces), 256, 0, s>>>(c, scales, pieces, static_cast<float *>(W));
    else
        w4_dequantize_kernel<uint16_t><<<convert_blocks(pieces), 256, 0, s>>>(c, scales, pieces, static_cast<uint16_t *>(W));
    return launch_status("w4_dequantize launch");
}

hipError_t launch_w4_forward(const W4Args &a, const BranchTable &bt)
{
    const int nt = a.T < 16 ? a.T : 16, token_tiles = ceil_div(a.T, 16);
    int kc = (kXBytes / (2 * nt) - kPad) / kStep * kStep;
    const int k_all = ceil_div(a.d_model, kStep) * kStep;
    if (kc > k_all) kc = k_all;
    int tiles = 0;
    for (int b = 0; b < bt.B; ++b)
        if ((bt.active >> b) & 1) tiles += ceil_div(bt.off[b + 1] - bt.off[b], kRows);
    const int nw = 8;
    int grid = ceil_div(tiles, nw);
    const size_t lds = (size_t)nt * (kc + kPad) * 2;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(w4_gate_up), hipFuncAttributeMaxDynamicSharedMemorySize,
                                       160 * 1024);
    if (e != hipSuccess) return note_hip_error("w4_gate_up attribute", e);
    {
        ProfileScope ps(MLPMOE_KERNEL_W4_GATE_UP, a.stream);
        w4_gate_up<<<dim3(grid, token_tiles), nw * 64, lds, a.stream>>>(static_cast<const uint16_t *>(a.x), a.T, a.d_model, kc, a.gc,
                                                                    a.gs, a.uc, a.us, static_cast<uint16_t *>(a.H), a.ldh,
                                                                    a.route, bt);
        e = launch_status("w4_gate_up launch");
        if (e != hipSuccess) return e;
    }
    const bool dense = !a.route && bt.d_eff == a.d_inter;
    const size_t bits = dense ? 0 : (size_t)ceil_div(a.d_inter / 32, 32) * 4;
    ProfileScope ps(MLPMOE_KERNEL_W4_DOWN, a.stream);
    w4_down<<<dim3(ceil_div(a.d_model, 16), token_tiles), kDownWaves * 64, bits, a.stream>>>(
        static_cast<const uint16_t *>(a.H), a.ldh, a.T, a.d_inter, a.dc, a.ds, a.d_model, a.out, a.out_bf16, a.route, bt, dense);
    return launch_status("w4_down launch");
}

}  // namespace mlpmoe
