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
#include "w4_common.h"

namespace mlpmoe {
namespace {

// These kernels live for 5 to 20 us, and code that runs once is fetched as it runs, a 64-byte line in some 170 clocks: a
// kilobyte of straight code costs as much as the latency of a load.  (The down projection with its ring of code registers
// unrolled took 2200 clocks for a chunk of K whose data had arrived.)  So loops stay rolled, what is staged goes straight into
// LDS without registers, and the branch table is looked at beside the first loads.

constexpr int kLdsBytes = 159 * 1024;

// Bytes of LDS for the scales of 16 rows, as they lie in memory.
__host__ __device__ constexpr int scale_bytes(int K) { return (K / 2 + 15) / 16 * 16 + 16; }

// `bytes` of scales to LDS, `wave` of nw waves; 16 bytes a lane if base and size are multiples of 16, else 4 (they are multiples of 8).
__device__ __forceinline__ void stage_scales(const uint8_t *src, char *dst, int bytes, bool by16, int wave, int nw)
{
    const int lane = threadIdx.x & 63;
    if (by16) {
#pragma unroll 1
        for (int i = wave * 1024; i < bytes; i += nw * 1024)
            if (i + lane * 16 < bytes) dma16(src + i + lane * 16, dst + i);
    } else {
#pragma unroll 1
        for (int i = wave * 256; i < bytes; i += nw * 256)
            if (i + lane * 4 < bytes)
                __builtin_amdgcn_global_load_lds((gptr_t)(src + i + lane * 4), (lptr_t)(dst + i), 4, 0, 0);
    }
}

constexpr int kChunkK = 512;             // K of a stage of w4_gate_up: four steps
constexpr int kXRow = kChunkK * 2 + 16;  // bytes of a token's x in it: the lanes of a cycle (eight tokens, two pieces 8 apart) read different banks

// Bytes of LDS: S stages, x of nt tokens in each of them or, whole, beside them.
size_t gate_up_lds(int nt, int nw, int S, int K, bool whole)
{
    return (size_t)S * nw * 4096 + (size_t)(whole ? ceil_div(K, kChunkK) : S) * nt * kXRow + 1024 + (size_t)nw * scale_bytes(K);
}

// Grid (workgroups, tiles of tt tokens).  A wave works out groups of 8 neurons, MFMA rows 0-7 W_gate and 8-15 W_up; wave w of
// workgroup g the groups w * grid + g and so on, so that what live groups there are is spread over the chip.  With x whole in
// LDS (below) several waves can share a group, chunk by chunk of K in turn: as many as the host says or, where the live groups are known
// here only, as have none of their own (T = 1 on one of 8 or 16 branches, us with its events: 4096 x 14336 9.0, not shared 10.8, 8192 x 8192 10.1, 14.2).
// 512 of K at a time, the codes (each wave its own) go through LDS, S - 1 stages ahead, and with them x (for the workgroup), which
// has the waves meet for every stage; XL = 0: x fits LDS whole, and after one meeting every wave goes at its own pace.  A load of codes
// is 256 bytes of four rows each: 4096 x 14336, gate and up codes alone, 10.2 us, and 11.3 us with 64 bytes of 16 rows.  Row r's 16-byte
// piece c lies at place c ^ r of its 256 bytes, and group q of lanes takes piece (block) 4 q + s in step s, so that the lanes of a
// cycle read different banks; x lies in the order in which it is read.  The 16 rows' scales are staged whole: asking for a byte
// a block costs as many requests as the codes (20.8 us).
// Medians of a trace, 4096 x 14336: T = 1 14.4 to 15.0 us (62 MB, 4.2 TB/s), T = 16 17.0, on a part of the branches 13.9 (16.3, 18.0 and 15.6 with
// a step's reads waited for one after the other and 64-bit addresses); 896 x 4864, T = 1 4.6, of which some 4 are the start, the first loads' latency and
// the epilogue's instruction fetch, which no kernel here is without.
template <bool kOneRun, int XL, int S>
__global__ void __launch_bounds__(512)
w4_gate_up(const uint16_t *__restrict__ x, int T, int tt, int K, const uint8_t *__restrict__ gc, const uint8_t *__restrict__ gs,
           const uint8_t *__restrict__ uc, const uint8_t *__restrict__ us, uint16_t *__restrict__ H, int ldh,
           const uint8_t *__restrict__ route, int parts_if_one, Range run, BranchTable bt)
{
    constexpr int PER = 4 + XL, AHEAD = S - 1;
    static_assert((AHEAD - 1) * PER < 63, "loads in flight");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int t0 = tt * blockIdx.y, nt = T - t0 < tt ? T - t0 : tt;
    const int blocks = K / 32, chunks = (K + kChunkK - 1) / kChunkK;
    constexpr bool kWhole = XL == 0;
    const int stage = (kWhole ? 0 : nt * kXRow) + nw * 4096;
    char *all_x = lds + S * stage, *scrap = all_x + (kWhole ? chunks * nt * kXRow : 0);
    Groups<8, kOneRun> groups(run);
    if constexpr (kOneRun) {
        if (blockIdx.x == 0) clear_edges(run, H + (size_t)t0 * ldh, ldh, nt, wave, nw);
    } else {
        const OffsetLanes off(bt);
        const unsigned long long live = live_of_16(bt, route, 0, T);    // of all tokens: the down projection's tiles may be larger
        groups = Groups<8, kOneRun>(off, live);
        clear_edges(off, bt.B, live, live, H + (size_t)t0 * ldh, ldh, nt, wave, nw, blockIdx.x, gridDim.x);
    }

    // this wave's group and part of K, of the parts that a group's waves take in turn
    int parts = kWhole && kOneRun ? parts_if_one : 1, slot = wave, part = 0;
    if constexpr (kWhole && !kOneRun) {
        const int own = __popcll(__ballot(lane < nw && (int)blockIdx.x + lane * (int)gridDim.x < groups.total));
        while (own > 0 && (parts + 1) * own <= nw && parts < chunks) ++parts;
    }
    if (kWhole && parts > 1)
        for (slot = 0, part = wave; part >= parts; part -= parts) ++slot;
    char *my_s = scrap + 1024 + slot * scale_bytes(K);

    // lane of a load of x: place 16 s + 4 q + j of the 64 is piece 16 q + 4 s + j
    const int x_piece = ((lane >> 2) & 3) * 16 + (lane >> 4) * 4 + (lane & 3);
    const char *zero = reinterpret_cast<const char *>(g_zero16);
    const int xr = (r16 < nt ? r16 : 0) * kXRow + q * 64, cb = (kWhole ? 0 : nt * kXRow) + wave * 4096;
#pragma unroll 1
    for (int at = blockIdx.x; at < groups.total; at += nw * (int)gridDim.x) {
        const int idx = at + slot * (int)gridDim.x;
        const bool have = idx < groups.total;
        const int n0 = have ? groups(idx) * 8 : 0;
        if (at != (int)blockIdx.x) pipeline_barrier<0>();               // the last group's stages and scales have been read
        const char *xb = reinterpret_cast<const char *>(x + (size_t)t0 * K);
        // Offsets of this lane in 32 bits from bases that are the same for all lanes.  A wave without a group asks for zeros; in the last
        // chunk what lies past the row's end is zero in x, and in the codes anything, the row's first.
        const char *gb = have ? reinterpret_cast<const char *>(gc + (size_t)n0 * (K / 2)) : zero;
        const char *ub = have ? reinterpret_cast<const char *>(uc + (size_t)n0 * (K / 2)) : zero;
        unsigned x_at[XL > 0 ? XL : 1], code_at[4], code_last[4];
#pragma unroll
        for (int n = 0; n < XL; ++n) x_at[n] = (unsigned)(wave + n * nw < nt ? wave + n * nw : 0) * K * 2 + x_piece * 16;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int piece = r16 ^ (4 * r + q);         // of row 4 r + q
            const unsigned row = (unsigned)(4 * (r & 1) + q) * (K / 2);
            code_at[r] = have ? row + piece * 16 : 0;
            code_last[r] = have ? row + ((chunks - 1) * 16 + piece < blocks ? (chunks - 1) * 16 + piece : 0) * 16 : 0;
        }
        auto issue = [&](int i, char *dst) {             // always PER loads; past the end the last chunk again
            const int c = part + i * parts, k = c < chunks ? c : chunks - 1;
            const bool last = k == chunks - 1;
            const unsigned codes = have ? k * 256 : 0;
#pragma unroll
            for (int n = 0; n < XL; ++n) {
                const char *src = xb + (x_at[n] + k * 1024);
                if (last && K % kChunkK != 0) {
                    asm volatile("");                    // a branch: a select would take these instructions in every chunk
                    src = k * 64 + x_piece < K / 8 ? src : zero;
                }
                dma16(src, wave + n * nw < nt ? dst + (wave + n * nw) * kXRow : scrap);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) dma16((r < 2 ? gb : ub) + (last ? code_last[r] : code_at[r] + codes), dst + cb + r * 1024);
        };
        keep_order();
#pragma unroll 1
        for (int c = 0; c < AHEAD; ++c) {
            issue(c, lds + c * stage);
            if (c == 0) {
                if (kWhole && at == (int)blockIdx.x)
#pragma unroll 1
                    for (int u = wave; u < nt * chunks; u += nw) {
                        const int k = u / nt, t = u - k * nt;
                        dma16(k * 64 + x_piece < K / 8 ? xb + (size_t)t * K * 2 + k * 1024 + x_piece * 16 : zero, all_x + u * kXRow);
                    }
                stage_scales(gs + (size_t)n0 * blocks, my_s, K / 4, K % 64 == 0, part, parts);
                stage_scales(us + (size_t)n0 * blocks, my_s + K / 4, K / 4, K % 64 == 0, part, parts);
            }
            keep_order();
        }
        const char *mine = lds;
        char *fill = lds + AHEAD * stage;
        f32x4 acc = {0, 0, 0, 0};
        if (kWhole && at == (int)blockIdx.x) pipeline_barrier<(AHEAD - 1) * PER>();
#pragma unroll 1
        for (int i = 0, c = part; c < chunks; ++i, c += parts) {
            if (kWhole)
                wait_loads<(AHEAD - 1) * PER>();
            else
                pipeline_barrier<(AHEAD - 1) * PER>();
            issue(i + AHEAD, fill);
            const char *mx = kWhole ? all_x + c * nt * kXRow : mine;
            const char *sc = my_s + r16 * blocks + c * 16 + q * 4;
            if (have) {
                // the next step's reads come after the first product: the compiler waits for all reads of LDS at the first use of one
                uint32_t byte[2];
                u32x4 w[2];
                bf16x8 xv[2][4];
                auto read = [&](int s) {
                    byte[s & 1] = *reinterpret_cast<const uint8_t *>(sc + s);
                    w[s & 1] = *reinterpret_cast<const u32x4 *>(mine + cb + r16 * 256 + ((q * 4 + s) ^ r16) * 16);
#pragma unroll
                    for (int j = 0; j < 4; ++j) xv[s & 1][j] = *reinterpret_cast<const bf16x8 *>(mx + xr + s * 256 + j * 16);
                };
                read(0);
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    __builtin_amdgcn_sched_barrier(0);
                    const float scale = scale_of(c * 16 + q * 4 + s < blocks ? byte[s & 1] : 127u);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[s & 1][j], scale), xv[s & 1][j], acc, 0, 0, 0);
                        if (j == 0 && s < 3) {
                            __builtin_amdgcn_sched_barrier(0);
                            read(s + 1);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
            }
            mine = mine + stage == lds + S * stage ? lds : mine + stage;
            fill = fill + stage == lds + S * stage ? lds : fill + stage;
        }
        if (kWhole && parts > 1) {                       // the parts' sums, in order; a wave's go where its codes were
            wait_loads<0>();
            f32x4 *sums = reinterpret_cast<f32x4 *>(lds + wave * 4096) + lane;
            if (part > 0) *sums = acc;
            pipeline_barrier<0>();
            if (part > 0) continue;
            for (int p = 1; p < parts; ++p) acc += sums[p * 256];
        }
        if (!have) continue;
        // neurons 4q .. 4q + 3 of token r16: gate in groups q < 2, up in the lanes 32 on
        f32x4 up;
#pragma unroll
        for (int i = 0; i < 4; ++i) up[i] = __shfl_xor(acc[i], 32);
        const BranchLanes br(bt);
        gated<8>(
            br, bt, n0, n0 + 4 * (q & 1), acc, up,
            [&](int b) { return kOneRun || !route || (r16 < nt && route[(size_t)(t0 + r16) * bt.B + b] != 0); },
            [&](uint2 h) {
                if (q < 2 && r16 < nt) *reinterpret_cast<uint2 *>(H + (size_t)(t0 + r16) * ldh + n0 + 4 * q) = h;
            });
    }
    pipeline_barrier<0>();                               // loads past the end are still on their way into LDS
}

// Bytes of LDS of w4_down: S stages of codes and of nt tokens' H, or H whole beside them, a kilobyte that loads without a token
// fill, the scales, and for tables that are no single run a bit a block and the list of live steps.
__host__ __device__ constexpr int whole_row(int K) { return (K + 4 * kStepK - 1) / (4 * kStepK) * 1024 + 16; }
size_t down_lds(int W, int S, int nt, int K, bool one, bool whole)
{
    return (size_t)S * (W * 1024 + (whole ? 0 : nt * (W * 256 + 16))) + (whole ? (size_t)nt * whole_row(K) : 0) + 1024 + scale_bytes(K) +
           (one ? 0 : (size_t)ceil_div(K / 32, 32) * 4 + ceil_div(K, kStepK) * 2);
}

// Grid (tiles of 16 features, token tiles of up to 4 NL or 16).  A workgroup of W waves owns 16 rows of W_down; in every chunk of W
// steps of K each wave has one, so that together the waves read W * 64 bytes of a row.  Codes (each wave its own) and H (for the
// workgroup) go through LDS, S - 1 chunks ahead, and the waves meet for every chunk; NL = 0: H of up to 16 tokens lies in LDS whole, and
// after one meeting every wave goes at its own pace.  A step is live if a live branch has a neuron in it; the others are left out.  The waves' sums are added in
// their order.  Medians of a trace, 4096 x 14336: T = 1 7.6 us (31 MB, 4.1 TB/s), T = 16 12.3, bound by H, which every workgroup reads (117 MB out of L2;
// four waves more that only load H, so that codes can be asked for five chunks ahead, do not help).
// Asking for the codes at the end of the kernel before does not help: with all of them in L2 this one takes 7.6 us instead
// of 8.4 (H by chunks), and that one longer by more.
template <bool kOneRun, int W, int NL, int S>
__global__ void __launch_bounds__(W * 64)
w4_down(const uint16_t *__restrict__ H, int ldh, int T, int K, const uint8_t *__restrict__ dc, const uint8_t *__restrict__ ds,
        int d_model, void *__restrict__ out, int out_bf16, const uint8_t *__restrict__ route, Range run, BranchTable bt)
{
    constexpr bool kWhole = NL == 0;
    constexpr int PARTS = W / 4;                         // kilobytes of a token's chunk of H
    constexpr int PER = NL + 1, AHEAD = S - 1;
    static_assert((AHEAD - 1) * PER < 63, "loads in flight");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int TOKENS = kWhole ? 16 : 4 * NL;
    const int t0 = TOKENS * blockIdx.y, nt = T - t0 < TOKENS ? T - t0 : TOKENS;
    const int blocks = K / 32, all = (K + kStepK - 1) / kStepK, m0 = blockIdx.x * 16;
    const int h_row = kWhole ? whole_row(K) : W * 256 + 16, h_stage = kWhole ? 0 : nt * h_row;
    const int stage = h_stage + W * 1024;
    char *all_h = lds + S * stage, *scrap = all_h + (kWhole ? nt * h_row : 0), *scales = scrap + 1024;
    uint32_t *bits = reinterpret_cast<uint32_t *>(scales + scale_bytes(K));
    uint16_t *list = reinterpret_cast<uint16_t *>(bits + (blocks + 31) / 32);
    const int s_beg = kOneRun ? run.beg / kStepK : 0;
    int steps = kOneRun ? (run.end + kStepK - 1) / kStepK - s_beg : 0;
    if constexpr (!kOneRun) {
        const OffsetLanes off(bt);
        mark_blocks(off, live_of_16(bt, route, t0, nt), bits, blocks);
        steps = list_steps(bits, all, list);
    }
    // Offsets of this lane in 32 bits from bases that are the same for all lanes, and past the last step that step again, which
    // nothing reads: few instructions a load (medians of a trace, T = 16: 4096 x 14336 on a part of the branches 11.2 -> 10.2 us, on all 12.5 -> 12.4,
    // 2048 x 7168 6.5 -> 6.3).
    const CodeLane cl;
    const char *codes = reinterpret_cast<const char *>(dc + (size_t)m0 * (K / 2)), *hb = reinterpret_cast<const char *>(H + (size_t)t0 * ldh);
    const unsigned code_at = cl.row * (K / 2) + cl.block * 16;
    const unsigned code_last = cl.row * (K / 2) + (cl.block < blocks - (all - 1) * 4 ? cl.block * 16 : 0);
    unsigned h_at[NL > 0 ? NL : 1];                      // a load of H: four steps of a token, piece r16 of step q
#pragma unroll
    for (int n = 0; n < NL; ++n) {
        const int t = (wave * NL + n) / PARTS;
        h_at[n] = (unsigned)(t < nt ? t : nt - 1) * ldh * 2 + r16 * 16;
    }
    auto step_of = [&](int i) {
        const int k = i < steps ? i : steps > 0 ? steps - 1 : 0;
        return kOneRun ? s_beg + k : steps > 0 ? (int)list[k] : 0;
    };
    auto issue = [&](int c, char *dst) {                 // always PER loads
#pragma unroll
        for (int n = 0; n < NL; ++n) {
            const int unit = wave * NL + n, t = unit / PARTS, part = unit % PARTS;
            dma16(hb + (h_at[n] + (unsigned)step_of(c * W + part * 4 + q) * 256), t < nt ? dst + t * h_row + part * 1024 : scrap);
        }
        const int s = __builtin_amdgcn_readfirstlane(step_of(c * W + wave));
        dma16(codes + ((s == all - 1 ? code_last : code_at) + (unsigned)s * 64), dst + h_stage + wave * 1024);
    };
    const int chunks = (steps + W - 1) / W;
    keep_order();
#pragma unroll 1
    for (int c = 0; c < AHEAD; ++c) {
        issue(c, lds + c * stage);
        if (c == 0) {
            if (kWhole)
#pragma unroll 1
                for (int part = wave; part * 4 < steps; part += W) {
                    const unsigned at = (unsigned)step_of(part * 4 + q) * 256 + r16 * 16;
#pragma unroll 1
                    for (int t = 0; t < nt; ++t) dma16(hb + (at + (unsigned)t * ldh * 2), all_h + t * h_row + part * 1024);
                }
            stage_scales(ds + (size_t)m0 * blocks, scales, K / 2, true, wave, W);
        }
        keep_order();
    }
    f32x4 acc = {0, 0, 0, 0};
    const char *mine = lds, *end = lds + S * stage;
    char *fill = lds + AHEAD * stage;
    const int hr = (r16 < nt ? r16 : 0) * h_row + wave * 256 + q * 64, wr = h_stage + wave * 1024 + cl.at;
    if (kWhole) pipeline_barrier<(AHEAD - 1) * PER>();
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        if (kWhole)
            wait_loads<(AHEAD - 1) * PER>();
        else
            pipeline_barrier<(AHEAD - 1) * PER>();
        issue(c + AHEAD, fill);
        if (c * W + wave < steps) {
            const int b = __builtin_amdgcn_readfirstlane(step_of(c * W + wave)) * 4 + q;
            const uint32_t byte = *reinterpret_cast<const uint8_t *>(scales + r16 * blocks + b);
            // a block that is not live: H is zero there, the scale may be no number
            const bool on = b < blocks && (kOneRun ? b >= run.beg / 32 && b * 32 < run.end : (bits[b / 32] >> (b & 31) & 1) != 0);
            const u32x4 w = *reinterpret_cast<const u32x4 *>(mine + wr);
            const char *mh = kWhole ? all_h + c * W * 256 : mine;
            bf16x8 h[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = *reinterpret_cast<const bf16x8 *>(mh + hr + j * 16);
            __builtin_amdgcn_sched_barrier(0);           // one wait for all of these reads
            const float scale = scale_of(on ? byte : 127u);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[j], scale), h[j], acc, 0, 0, 0);
        }
        mine = mine + stage == end ? lds : mine + stage;
        fill = fill + stage == end ? lds : fill + stage;
    }
    pipeline_barrier<0>();
    float *red = reinterpret_cast<float *>(lds);         // where the stages were
#pragma unroll
    for (int i = 0; i < 4; ++i) red[wave * 256 + r16 * 16 + 4 * q + i] = acc[i];
    __syncthreads();
    if (threadIdx.x < 256) {
        const int t = threadIdx.x >> 4, f = m0 + (threadIdx.x & 15);
        float v = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) v += red[w * 256 + threadIdx.x];
        if (t < nt) {
            const size_t to = (size_t)(t0 + t) * d_model + f;
            if (out_bf16)
                static_cast<uint16_t *>(out)[to] = to_bf16(v);
            else
                static_cast<float *>(out)[to] = v;
        }
    }
}

// --- conversion ------------------------------------------------------------------------------------------------------
// A lane takes 8 of a block's 32 values; the block's largest magnitude crosses its four lanes by DPP.  Memory bound: 14336 x 4096 bf16
// there and back 48.5 us, 266 MB, 5.5 TB/s.
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

template <bool kOneRun, int W, int NL, int S>
hipError_t launch_down(const W4Args &a, const BranchTable &bt, const Range &run)
{
    constexpr int TOKENS = NL == 0 ? 16 : 4 * NL;
    const size_t lds = down_lds(W, S, a.T < TOKENS ? a.T : TOKENS, a.d_inter, kOneRun, NL == 0);
    const hipError_t e = allow_lds<w4_down<kOneRun, W, NL, S>>((int)lds, "w4_down attribute");
    if (e != hipSuccess) return e;
    ProfileScope ps(MLPMOE_KERNEL_W4_DOWN, a.stream);
    w4_down<kOneRun, W, NL, S><<<dim3(a.d_model / 16, ceil_div(a.T, TOKENS)), W * 64, lds, a.stream>>>(
        static_cast<const uint16_t *>(a.H), a.ldh, a.T, a.d_inter, a.dc, a.ds, a.d_model, a.out, a.out_bf16, a.route, run, bt);
    return launch_status("w4_down launch");
}

template <bool kOneRun, int XL, int S>
hipError_t launch_gate_up(const W4Args &a, const BranchTable &bt, const Range &run, int groups, int share, int nw, int tt)
{
    const size_t lds = gate_up_lds(a.T < tt ? a.T : tt, nw, S, a.d_model, XL == 0);
    const hipError_t e = allow_lds<w4_gate_up<kOneRun, XL, S>>((int)lds, "w4_gate_up attribute");
    if (e != hipSuccess) return e;
    const int resident = 256 * (int)(160 * 1024 / lds);
    const int chunks = ceil_div(a.d_model, kChunkK), grid = ceil_div(groups, share) < resident ? ceil_div(groups, share) : resident;
    ProfileScope ps(MLPMOE_KERNEL_W4_GATE_UP, a.stream);
    w4_gate_up<kOneRun, XL, S><<<dim3(grid, ceil_div(a.T, tt)), nw * 64, lds, a.stream>>>(
        static_cast<const uint16_t *>(a.x), a.T, tt, a.d_model, a.gc, a.gs, a.uc, a.us, static_cast<uint16_t *>(a.H), a.ldh, a.route,
        nw / share < chunks ? nw / share : chunks, run, bt);
    return launch_status("w4_gate_up launch");
}

// A wave a group for every CU's share of the groups, up to 8; three stages, x whole if there is room for it.  Where the share is one to
// three groups and a wave would have four or more kilobytes of x to load, up to 8 waves share them, or at least the loads (us with events,
// shared and not: 4096 x 2048, T = 8 9.0, 16.2; 6144 x 2048, T = 1 8.4, 12.0; 2048 x 2048, T = 16 8.1, 14.7; 896 x 4864, T = 16 7.4, 7.7; but four groups: 2048 x 7168,
// T = 4 8.9, 8.0).  (More stages, that
// is requests in flight, take longer: 4096 x 14336, T = 1: four 18.0 us, three 16.8.)  Where three stages with x in them do not fit,
// up to two waves fewer, then two stages.  A wave loads up to four tokens of x.
template <bool kOneRun>
hipError_t gate_up(const W4Args &a, const BranchTable &bt, const Range &run, int groups)
{
    const int nt = a.T < 16 ? a.T : 16, K = a.d_model, least = ceil_div(nt, 4);
    auto fits = [&](int nw, int S, bool whole) { return gate_up_lds(nt, nw, S, K, whole) <= (size_t)kLdsBytes; };
    int want = ceil_div(groups, 256);
    want = want > 8 ? 8 : want;
    const int most = want <= 3 && ceil_div(K, kChunkK) * nt >= 4 * want ? 8 : want;
    for (int n = most; n >= (want <= 2 && want < least ? least : want); --n)
        if (fits(n, 3, true)) return launch_gate_up<kOneRun, 0, 3>(a, bt, run, groups, want, n, 16);
    want = want < least ? least : want;
    for (int n = want; n >= least && n >= want - 2; --n) {
        if (!fits(n, 3, false)) continue;
        const int xl = ceil_div(nt, n);
        return xl <= 2   ? launch_gate_up<kOneRun, 2, 3>(a, bt, run, groups, n, n, 16)
               : xl == 3 ? launch_gate_up<kOneRun, 3, 3>(a, bt, run, groups, n, n, 16)
                         : launch_gate_up<kOneRun, 4, 3>(a, bt, run, groups, n, n, 16);
    }
    for (int n = want; n >= least; --n)
        if (fits(n, 2, false)) return launch_gate_up<kOneRun, 4, 2>(a, bt, run, groups, n, n, 16);
    return launch_gate_up<kOneRun, 4, 2>(a, bt, run, groups, 1, 1, 4);      // scales of a very long K: one wave, four tokens at a time
}

// 16 waves while three stages of their chunks fit, else 8, whose chunks are half as long.  H whole if it fits, us with its events against H by chunks:
// 4096 x 14336, T = 1 9.6, 10.5; 8192 x 8192, T = 1 14.6 and 15.8, T = 4 15.4 and 16.0; 2048 x 7168, T = 1 6.8 and 7.2, T = 12 8.1 and 8.2;
// 896 x 4864, T = 1 6.1 and 6.4.
template <bool kOneRun>
hipError_t down(const W4Args &a, const BranchTable &bt, const Range &run)
{
    const int nt = a.T < 16 ? a.T : 16, K = a.d_inter;
    auto fits = [&](int W, int S, bool whole = false) { return down_lds(W, S, nt, K, kOneRun, whole) <= (size_t)kLdsBytes; };
    if (fits(16, 4, true)) return launch_down<kOneRun, 16, 0, 4>(a, bt, run);
    if (nt <= 4 && fits(16, 4)) return launch_down<kOneRun, 16, 1, 4>(a, bt, run);
    if (nt <= 8 && fits(16, 3)) return launch_down<kOneRun, 16, 2, 3>(a, bt, run);
    if (fits(8, 3)) return launch_down<kOneRun, 8, 4, 3>(a, bt, run);
    return launch_down<kOneRun, 8, 1, 3>(a, bt, run);    // scales of a very long K: four tokens at a time
}

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
    const bool one = !a.route && bt.n_runs == 1;
    const Range run = one ? Range{bt.run_start[0], bt.run_end[0]} : Range{0, 0};
    int groups = 0;                          // an upper bound: a group shared by two branches counts for both
    for (int b = 0; b < bt.B; ++b)
        if (((bt.active >> b) & 1) && bt.off[b + 1] > bt.off[b]) groups += ceil_div(bt.off[b + 1], 8) - bt.off[b] / 8;
    if (one) groups = ceil_div(run.end, 8) - run.beg / 8;
    const hipError_t e = one ? gate_up<true>(a, bt, run, groups) : gate_up<false>(a, bt, run, groups);
    if (e != hipSuccess) return e;
    return one ? down<true>(a, bt, run) : down<false>(a, bt, run);
}

}  // namespace mlpmoe
