// The forward on 4-bit weights for more tokens than one MFMA column block: tiles of rows x tokens.
//
// A workgroup owns 16 NF tokens and, for each of its WR row waves, 16 NA rows of weights.  x (or H) goes through LDS, shared by the
// waves; each wave's codes go through LDS too, read back by the lanes that loaded them, and are widened in registers: a weight
// is widened once for 16 NF tokens, half an instruction a weight against NF MFMA columns.  K goes by steps of 128, AHEAD stages
// of KW steps ahead; with KW = 2 two sets of row waves take the steps in turn and add their sums at the end, which gives a tile
// that is too small for two workgroups on a CU two waves a SIMD.  LDS holds a token's 128 values as 16 pieces of 16 bytes, piece c
// at place c ^ (token mod 16), so that the lanes of a cycle read different banks.
//
// Rows are the MFMA's rows and tokens its columns: a lane ends with four neighbouring neurons (features) of a token, one store.
// Nothing is loaded into registers: beside loads into LDS the compiler waits for every register load at once.
//
// 4096 x 14336, T = 500: gate and up 106 us (1.11 PFLOP/s), down 63 and the sum of its ranges 6.6.  Matrix pipes busy 47 % of it, LDS 40 %;
// without any loads the same loops take 95 us instead of 112 and 51 instead of 66 (with their events); the rest is the meetings
// and the first reads of a stage.  T = 45: 24, 15 and 4 us, start and latency again.
#include "w4_common.h"

namespace mlpmoe {
namespace {

constexpr int kCus = 256, kMostSplits = 8;
constexpr int kScaleBuf = 1280;          // scales of a wave's rows for 512 of K: 16 bytes a row, or 20 in five loads of a dword

constexpr int stage_bytes(int NA, int NF, int KW, int WR) { return KW * NF * 4096 + KW * WR * NA * 1024; }
constexpr int core_lds(int NA, int NF, int AHEAD, int KW, int WR)
{
    return (AHEAD + 1) * (stage_bytes(NA, NF, KW, WR) + KW * WR * kScaleBuf);
}

// acc[a][f] += 16 rows (codes[a], this wave's) x 16 tokens over the n > 0 steps step(0) .. step(n - 1), ascending (past the end
// the last one).  srow: this lane's row of scales, lane 16 a + r for row r of codes[a]; send: their end.  on(b): whether block b is read (the scale of
// another may be no number; x is zero there).  The sum is in the first set's waves.  kWholeSteps: X is H, whose rows are
// whole steps; else a row is K long.
template <int NA, int NF, int AHEAD, int KW, int WR, bool kWholeSteps, typename StepOf, typename On>
__device__ __forceinline__ void sum_steps(f32x4 (&acc)[NA][NF], const uint8_t *const (&codes)[NA], const uint8_t *srow,
                                          const uint8_t *send, const uint16_t *__restrict__ X, int ldx, int last_token, int K,
                                          char *lds, int n, StepOf step_of, On on)
{
    constexpr int STAGE = stage_bytes(NA, NF, KW, WR), NX = NF * 4 / WR, PER = NX + NA;
    static_assert(NF * 4 % WR == 0 && (AHEAD - 1) * PER < 63 && NA <= 4, "loads in flight");
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kw = wave / WR;
    const int blocks = K / 32, all = (K + kStepK - 1) / kStepK;
    const char *xb = reinterpret_cast<const char *>(X), *zero = reinterpret_cast<const char *>(g_zero16);
    // this lane's part of the loads of X: four tokens a load, 16 pieces each
    unsigned x_off[NX];
    int x_k[NX];
#pragma unroll
    for (int i = 0; i < NX; ++i) {
        const int unit = wave * NX + i, t = unit % (NF * 4) * 4 + q, c = r16 ^ (t & 15);
        x_off[i] = (unsigned)((t < last_token ? t : last_token) * ldx * 2 + c * 16);
        x_k[i] = c * 8;
    }
    const CodeLane cl;
    const unsigned w_row = cl.row * (K / 2);
    const int block_last = cl.block < blocks - (all - 1) * 4 ? cl.block : 0;     // in the last step there may be fewer than four
    const bool by16 = K % 512 == 0;
    const int late = by16 ? 0 : (r16 * blocks) & 3;                     // bytes of a dword before a row's
    char *my_s = lds + (AHEAD + 1) * STAGE + wave * ((AHEAD + 1) * kScaleBuf);
    const int w_at = KW * NF * 4096 + wave * (NA * 1024);
    int have = -1, slot = 0;                                            // the last 512 of K whose scales were asked for, and where
    auto issue = [&](int i, char *dst) {                                // stage i: steps KW i ..; always PER loads, and at times scales
        const int s = step_of(i * KW + kw);                             // past the end the last one again
        if (s >> 2 != have) {
            have = s >> 2;
            slot = slot == AHEAD ? 0 : slot + 1;
            char *to = my_s + slot * kScaleBuf;
            if (by16) {
                dma16(srow + have * 16, to);
            } else {
                const uint8_t *p = reinterpret_cast<const uint8_t *>(reinterpret_cast<uintptr_t>(srow + have * 16) & ~(uintptr_t)3);
#pragma unroll 1
                for (int d = 0; d < 5; ++d)
                    __builtin_amdgcn_global_load_lds((gptr_t)(p + d * 4 < send ? p + d * 4 : p), (lptr_t)(to + d * 256), 4, 0, 0);
            }
        }
#pragma unroll
        for (int j = 0; j < NX; ++j) {
            const int u = KW == 1 ? s : step_of(i * KW + (wave * NX + j) / (NF * 4));
            const char *src = xb + (size_t)u * 256 + x_off[j];
            if (!kWholeSteps && u == all - 1) src = u * kStepK + x_k[j] < K ? src : zero;
            // The second set has no step in the last stage where their number is odd: zeros, whatever X holds (a product of zero and an
            // infinity is not a number).
            if (KW > 1 && i * KW + (wave * NX + j) / (NF * 4) >= n) src = zero;
            dma16(src, dst + (wave * NX + j) * 1024);
        }
        const unsigned off = w_row + s * 64 + (s == all - 1 ? block_last : cl.block) * 16;
#pragma unroll
        for (int a = 0; a < NA; ++a) dma16(codes[a] + off, dst + w_at + a * 1024);
    };
    const int stages = (n + KW - 1) / KW;
    keep_order();
#pragma unroll 1
    for (int i = 0; i < AHEAD; ++i) {
        issue(i, lds + i * STAGE);
        keep_order();
    }
    char *mine = lds, *fill = lds + AHEAD * STAGE;
    int read = -1, rslot = 0;
    const int a_step = by16 ? 256 : 64;
#pragma unroll 1
    for (int i = 0; i < stages; ++i) {
        pipeline_barrier<(AHEAD - 1) * PER>();
        const int s = step_of(i * KW + kw);
        if (s >> 2 != read) read = s >> 2, rslot = rslot == AHEAD ? 0 : rslot + 1;
        const int at = late + (s & 3) * 4 + q;
        const char *sc = my_s + rslot * kScaleBuf + (by16 ? r16 * 16 + at : (at >> 2) * 256 + r16 * 4 + (at & 3));
        const char *st = mine + kw * (NF * 4096) + r16 * 256;
        const bool live = on(s * 4 + q), mine_too = KW == 1 || i * KW + kw < n;
        float scale[NA];
        uint32_t byte[NA];
        u32x4 w[NA];
        bf16x8 xv[2][NF];
        auto read_x = [&](int j) {
#pragma unroll
            for (int f = 0; f < NF; ++f) xv[j & 1][f] = *reinterpret_cast<const bf16x8 *>(st + f * 4096 + (((q * 4 + j) ^ r16) * 16));
        };
#pragma unroll
        for (int a = 0; a < NA; ++a) {
            byte[a] = *reinterpret_cast<const uint8_t *>(sc + a * a_step);
            w[a] = *reinterpret_cast<const u32x4 *>(mine + w_at + a * 1024 + cl.at);
        }
        read_x(0);
        __builtin_amdgcn_sched_barrier(0);               // one wait for all of these reads
#pragma unroll
        for (int a = 0; a < NA; ++a) {
            // The set without a step: a scale that is a number.  Zeros in its x would do without the codes, but the compiler then orders the
            // reads otherwise (4096 x 14336, T = 24 gate and up 22.7 us instead of 22.1 with its events).
            if (KW > 1 && !mine_too) w[a] = u32x4{0, 0, 0, 0};
            scale[a] = scale_of(live && mine_too ? byte[a] : 127u);
        }
        // The compiler waits for all reads of LDS at the first use of one, so the next reads come after the first products.
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                const bf16x8 wv = widen8(w[a][j], scale[a]);
#pragma unroll
                for (int f = 0; f < NF; ++f) acc[a][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xv[j & 1][f], acc[a][f], 0, 0, 0);
                if (a == 0) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (j == 0) issue(i + AHEAD, fill);
                    if (j < 3) read_x(j + 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        mine = mine + STAGE == lds + (AHEAD + 1) * STAGE ? lds : mine + STAGE;
        fill = fill + STAGE == lds + (AHEAD + 1) * STAGE ? lds : fill + STAGE;
    }
    pipeline_barrier<0>();                  // what is still on its way into LDS
    if constexpr (KW > 1) {
        static_assert(KW == 2 && WR * NA * NF * 1024 <= (AHEAD + 1) * STAGE, "the second set's sums fit where the stages were");
        f32x4 *sums = reinterpret_cast<f32x4 *>(lds) + (wave % WR) * (NA * NF * 64) + lane;
        if (kw == 1) {
#pragma unroll
            for (int i = 0; i < NA * NF; ++i) sums[i * 64] = acc[i / NF][i % NF];
        }
        pipeline_barrier<0>();
        if (kw == 0) {
#pragma unroll
            for (int i = 0; i < NA * NF; ++i) acc[i / NF][i % NF] += sums[i * 64];
        }
        pipeline_barrier<0>();              // LDS is free again
    }
}

// Calls fn(f, sum) for f = 0 .. NF - 1, sum(a) this lane's acc[a][f], in a loop that is not unrolled, through BYTES of LDS of this
// wave's own: an epilogue that is written out for every sum is thousands of instructions that run once.
template <int NA, int NF, int BYTES, typename Fn>
__device__ __forceinline__ void each_sum(const f32x4 (&acc)[NA][NF], char *lds, Fn fn)
{
    constexpr int F = NA * NF * 1024 <= BYTES ? NF : NA * ((NF + 1) / 2) * 1024 <= BYTES ? (NF + 1) / 2 : NF / 4;
    static_assert(F > 0 && NA * F * 1024 <= BYTES, "room for the sums of some of the tokens");
    f32x4 *mine = reinterpret_cast<f32x4 *>(lds) + (threadIdx.x & 63);
#pragma unroll 1
    for (int f0 = 0; f0 < NF; f0 += F) {
#pragma unroll
        for (int p = 0; p < NF; p += F)
            if (f0 == p) {
#pragma unroll
                for (int a = 0; a < NA; ++a)
#pragma unroll
                    for (int f = 0; f < F; ++f)
                        if (p + f < NF) mine[(a * F + f) * 64] = acc[a][p + f];
            }
#pragma unroll 1
        for (int f = f0; f < f0 + F && f < NF; ++f) fn(f, [&](int a) { return mine[(a * F + f - f0) * 64]; });
    }
}

// Grid (8, token tiles, row tiles / 8): workgroups go to the XCDs in turn, so the token tiles of a row tile, which read the same
// weights, are on one XCD, one after the other.

// A row wave takes NR groups of 16 neurons that a live branch reaches into, at multiples of 16: rows of W_gate, then of W_up.
// reach: tokens of a workgroup of the down projection, which reads what any of them has live, so that a tile's tokens need zeros
// there.
template <int NR, int NF, int AHEAD, int KW, int WR, int W, bool kOneRun>
__global__ void __launch_bounds__(KW * WR * 64, W)
w4_tile_gate_up(const uint16_t *__restrict__ x, int T, int K, int d_inter, const uint8_t *__restrict__ gc, const uint8_t *__restrict__ gs,
                const uint8_t *__restrict__ uc, const uint8_t *__restrict__ us, uint16_t *__restrict__ H, int ldh,
                const uint8_t *__restrict__ route, int reach, int row_tiles, Range run, BranchTable bt)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int row = blockIdx.z * 8 + blockIdx.x;
    if (row >= row_tiles) return;
    const int t0 = blockIdx.y * 16 * NF, nt = T - t0 < 16 * NF ? T - t0 : 16 * NF;
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % WR;
    Groups<16, kOneRun> groups(run);
    if constexpr (kOneRun) {
        if (row == 0) clear_edges(run, H + (size_t)t0 * ldh, ldh, nt, wave, WR);
    } else {
        __shared__ unsigned any[4];
        const OffsetLanes off(bt);
        const unsigned long long live = live_of(bt, route, t0, nt, any);
        const int r0 = t0 / reach * reach, upto = (t0 + nt + reach - 1) / reach * reach, r1 = upto < T ? upto : T;
        const unsigned long long wide = route && (r0 < t0 || r1 > t0 + nt) ? live_of(bt, route, r0, r1 - r0, any + 2) : live;
        groups = Groups<16, kOneRun>(off, live);
        clear_edges(off, bt.B, live, wide, H + (size_t)t0 * ldh, ldh, nt, wave, WR, row, row_tiles);
        if (row * WR * NR >= groups.total) return;
    }

    const int blocks = K / 32;
    const uint8_t *codes[2 * NR], *srow = gs;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int idx = (row * WR + wave) * NR + i;
        const int g = groups(idx < groups.total ? idx : groups.total - 1);
        codes[i] = gc + (size_t)g * 16 * (K / 2);
        codes[NR + i] = uc + (size_t)g * 16 * (K / 2);
        const size_t at = (size_t)(g * 16 + r16) * blocks;
        if (q == i) srow = gs + at;
        if (q == NR + i) srow = us + at;
    }
    f32x4 acc[2 * NR][NF];
#pragma unroll
    for (int a = 0; a < 2 * NR; ++a)
#pragma unroll
        for (int f = 0; f < NF; ++f) acc[a][f] = f32x4{0, 0, 0, 0};
    const int steps = (K + kStepK - 1) / kStepK;
    sum_steps<2 * NR, NF, AHEAD, KW, WR, false>(
        acc, codes, srow, (q < NR || q >= 2 * NR ? gs : us) + (size_t)d_inter * blocks, x + (size_t)t0 * K, K, nt - 1, K, lds, steps,
        [&](int i) { return i < steps ? i : steps - 1; }, [&](int b) { return b < blocks; });
    if (KW > 1 && threadIdx.x >= WR * 64) return;

    const BranchLanes br(bt);
    constexpr int MINE = (AHEAD + 1) * stage_bytes(2 * NR, NF, KW, WR) / WR / 1024 * 1024;
    each_sum<2 * NR, NF, MINE>(acc, lds + wave * MINE, [&](int f, auto sum) {
        const int t = f * 16 + r16;
#pragma unroll 1
        for (int i = 0; i < NR; ++i) {
            const int idx = (row * WR + wave) * NR + i;
            if (idx >= groups.total) break;
            const int n0 = groups(idx) * 16;
            const f32x4 g = sum(i), u = sum(NR + i);
            gated<16>(
                br, bt, n0, n0 + 4 * q, g, u,
                [&](int b) { return kOneRun || !route || (t < nt && route[(size_t)(t0 + t) * bt.B + b] != 0); },
                [&](uint2 h) {
                    if (t < nt) *reinterpret_cast<uint2 *>(H + (size_t)(t0 + t) * ldh + n0 + 4 * q) = h;
                });
        }
    });
}

// K is cut into 2^log_splits ranges; with more than one the sums go to partial [ranges][T][d_model].
template <int NA, int NF, int AHEAD, int KW, int WR, int W, bool kOneRun>
__global__ void __launch_bounds__(KW * WR * 64, W)
w4_tile_down(const uint16_t *__restrict__ H, int ldh, int T, int K, const uint8_t *__restrict__ dc, const uint8_t *__restrict__ ds,
             int d_model, void *__restrict__ out, int out_bf16, float *__restrict__ partial, int log_splits,
             const uint8_t *__restrict__ route, int row_tiles, Range run, BranchTable bt)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int row = blockIdx.z * 8 + blockIdx.x, splits = 1 << log_splits;
    if (row >= row_tiles) return;
    const int z = blockIdx.y & (splits - 1);
    const int t0 = (blockIdx.y >> log_splits) * 16 * NF, nt = T - t0 < 16 * NF ? T - t0 : 16 * NF;
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % WR;
    const int blocks = K / 32, all = (K + kStepK - 1) / kStepK;
    uint32_t *bits = reinterpret_cast<uint32_t *>(lds + core_lds(NA, NF, AHEAD, KW, WR));
    uint16_t *list = reinterpret_cast<uint16_t *>(bits + (blocks + 31) / 32);
    const int s_beg = kOneRun ? run.beg / kStepK : 0;
    int steps = kOneRun ? (run.end + kStepK - 1) / kStepK - s_beg : 0;
    if constexpr (!kOneRun) {
        __shared__ unsigned any[2];
        const OffsetLanes off(bt);
        mark_blocks(off, live_of(bt, route, t0, nt, any), bits, blocks);
        steps = list_steps(bits, all, list);
    }
    const uint8_t *codes[NA], *srow = ds;
#pragma unroll
    for (int a = 0; a < NA; ++a) {
        const int want = (row * WR + wave) * NA + a, g = want * 16 < d_model ? want : d_model / 16 - 1;
        codes[a] = dc + (size_t)g * 16 * (K / 2);
        if (q == a) srow = ds + (size_t)(g * 16 + r16) * blocks;
    }
    f32x4 acc[NA][NF];
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int f = 0; f < NF; ++f) acc[a][f] = f32x4{0, 0, 0, 0};
    const int beg = steps * z >> log_splits, n = (steps * (z + 1) >> log_splits) - beg;
    if (n > 0)
        sum_steps<NA, NF, AHEAD, KW, WR, true>(
            acc, codes, srow, ds + (size_t)d_model * blocks, H + (size_t)t0 * ldh, ldh, nt - 1, K, lds, n,
            [&](int i) {
                const int at = beg + (i < n ? i : n - 1);
                return kOneRun ? s_beg + at : __builtin_amdgcn_readfirstlane((int)list[at]);
            },
            [&](int b) { return b < blocks && (kOneRun ? b >= run.beg / 32 && b * 32 < run.end : (bits[b / 32] >> (b & 31) & 1) != 0); });
    if (KW > 1 && threadIdx.x >= WR * 64) return;

    constexpr int MINE = (AHEAD + 1) * stage_bytes(NA, NF, KW, WR) / WR / 1024 * 1024;
    each_sum<NA, NF, MINE>(acc, lds + wave * MINE, [&](int f, auto sum) {
        const int t = f * 16 + r16;
#pragma unroll 1
        for (int a = 0; a < NA; ++a) {
            const int m = ((row * WR + wave) * NA + a) * 16 + 4 * q;
            const f32x4 v = sum(a);
            if (m >= d_model || t >= nt) continue;
            const size_t to = (size_t)(t0 + t) * d_model + m;
            if (splits > 1)
                *reinterpret_cast<f32x4 *>(partial + (size_t)z * T * d_model + to) = v;
            else if (out_bf16)
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + to) = uint2{(uint32_t)to_bf16(v[0]) | (uint32_t)to_bf16(v[1]) << 16,
                                                                                      (uint32_t)to_bf16(v[2]) | (uint32_t)to_bf16(v[3]) << 16};
            else
                *reinterpret_cast<f32x4 *>(static_cast<float *>(out) + to) = v;
        }
    });
}

// The partial sums of a split, in order.
__global__ void __launch_bounds__(256)
w4_reduce(const float *__restrict__ partial, size_t n4, int splits, void *__restrict__ out, int out_bf16)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (size_t)gridDim.x * 256) {
        f32x4 s = reinterpret_cast<const f32x4 *>(partial)[i];
        for (int z = 1; z < splits; ++z) s += reinterpret_cast<const f32x4 *>(partial)[(size_t)z * n4 + i];
        if (out_bf16)
            reinterpret_cast<uint2 *>(out)[i] = uint2{(uint32_t)to_bf16(s[0]) | (uint32_t)to_bf16(s[1]) << 16,
                                                     (uint32_t)to_bf16(s[2]) | (uint32_t)to_bf16(s[3]) << 16};
        else
            reinterpret_cast<f32x4 *>(out)[i] = s;
    }
}

Range run_of(const W4Args &a, const BranchTable &bt) { return !a.route && bt.n_runs == 1 ? Range{bt.run_start[0], bt.run_end[0]} : Range{0, 0}; }

template <int NR, int NF, int D, int KW, int WR, int W>
hipError_t gate_up(const W4Args &a, const BranchTable &bt, int reach)
{
    int groups = 0;                          // an upper bound: a group shared by two branches counts for both
    const Range run = run_of(a, bt);
    const bool one = run.end > 0;
    for (int b = 0; b < bt.B; ++b)
        if (((bt.active >> b) & 1) && bt.off[b + 1] > bt.off[b]) groups += ceil_div(bt.off[b + 1], 16) - bt.off[b] / 16;
    if (one) groups = ceil_div(run.end, 16) - run.beg / 16;
    const int row_tiles = ceil_div(groups, WR * NR), token_tiles = ceil_div(a.T, 16 * NF);
    const size_t lds = core_lds(2 * NR, NF, D, KW, WR);
    const hipError_t e = one ? allow_lds<w4_tile_gate_up<NR, NF, D, KW, WR, W, true>>((int)lds, "w4_tile_gate_up attribute")
                             : allow_lds<w4_tile_gate_up<NR, NF, D, KW, WR, W, false>>((int)lds, "w4_tile_gate_up attribute");
    if (e != hipSuccess) return e;
    ProfileScope ps(MLPMOE_KERNEL_W4_GATE_UP, a.stream);
    (one ? w4_tile_gate_up<NR, NF, D, KW, WR, W, true> : w4_tile_gate_up<NR, NF, D, KW, WR, W, false>)
        <<<dim3(8, token_tiles, ceil_div(row_tiles, 8)), KW * WR * 64, lds, a.stream>>>(
            static_cast<const uint16_t *>(a.x), a.T, a.d_model, a.d_inter, a.gc, a.gs, a.uc, a.us, static_cast<uint16_t *>(a.H), a.ldh, a.route,
            reach, row_tiles, run, bt);
    return launch_status("w4_tile_gate_up launch");
}

template <int NA, int NF, int D, int KW, int WR, int W>
hipError_t down(const W4Args &a, const BranchTable &bt, int splits)
{
    int log_splits = 0;
    while (1 << log_splits < splits) ++log_splits;
    const int row_tiles = ceil_div(a.d_model, 16 * WR * NA), token_tiles = ceil_div(a.T, 16 * NF);
    const Range run = run_of(a, bt);
    const bool one = run.end > 0;
    const size_t lds = core_lds(NA, NF, D, KW, WR) + (one ? 0 : (size_t)ceil_div(a.d_inter / 32, 32) * 4 + (size_t)ceil_div(a.d_inter, kStepK) * 2);
    hipError_t e = one ? allow_lds<w4_tile_down<NA, NF, D, KW, WR, W, true>>((int)lds, "w4_tile_down attribute")
                       : allow_lds<w4_tile_down<NA, NF, D, KW, WR, W, false>>((int)lds, "w4_tile_down attribute");
    if (e != hipSuccess) return e;
    {
        ProfileScope ps(MLPMOE_KERNEL_W4_DOWN, a.stream);
        (one ? w4_tile_down<NA, NF, D, KW, WR, W, true> : w4_tile_down<NA, NF, D, KW, WR, W, false>)
            <<<dim3(8, token_tiles << log_splits, ceil_div(row_tiles, 8)), KW * WR * 64, lds, a.stream>>>(
                static_cast<const uint16_t *>(a.H), a.ldh, a.T, a.d_inter, a.dc, a.ds, a.d_model, a.out, a.out_bf16, a.partial, log_splits,
                a.route, row_tiles, run, bt);
        e = launch_status("w4_tile_down launch");
        if (e != hipSuccess || splits == 1) return e;
    }
    const size_t n4 = (size_t)a.T * a.d_model / 4;
    const size_t blocks = (n4 + 255) / 256;
    ProfileScope ps(MLPMOE_KERNEL_SPLITK_REDUCE, a.stream);
    w4_reduce<<<(unsigned)(blocks < 2048 ? blocks : 2048), 256, 0, a.stream>>>(a.partial, n4, splits, a.out, a.out_bf16);
    return launch_status("w4_reduce launch");
}

}  // namespace

// Tiles of the down projection: 128 features x 32, 48 or 64 tokens while there are few, 256 x 64 where that gives 64 tiles; and K
// cut until there are two workgroups a CU.  us, down projection and the sum of its ranges, with some 5 of their events:
//   4096 x 14336: T = 24 128 x 32 20.8, 128 x 64 23.7; T = 45 128 x 48 24.2, 128 x 64 24.7; T = 128 128 x 64 32.8, 256 x 64 36.6; T = 200 256 x 64 47.2,
//   128 x 64 48.6; T = 500 75.2 and 82.3; T = 1000 127 and 145
//   896 x 4864: T = 500 128 x 64 22.9, 256 x 64 more than 26; T = 2000 41 and more than 49
struct DownTile {
    int kind, rows, tokens, splits;
};
DownTile down_tile(int T, int d_model, int d_inter)
{
    DownTile t = T <= 32 ? DownTile{0, 128, 32, 1} : T <= 48 ? DownTile{1, 128, 48, 1} : T <= 64 ? DownTile{2, 128, 64, 1} : DownTile{3, 128, 64, 1};
    if (T > 64 && d_model >= 1024 && (long long)ceil_div(d_model, 256) * ceil_div(T, 64) >= 64) t = DownTile{4, 256, 64, 1};
    const long long tiles = (long long)ceil_div(d_model, t.rows) * ceil_div(T, t.tokens);
    while (t.splits < kMostSplits && tiles * t.splits * 2 <= 2 * kCus && d_inter >= kStepK * 8 * t.splits) t.splits *= 2;
    return t;
}

// Room for the partial sums of any call of up to T tokens: at most kMostSplits ranges, and a split leaves at most 2 kCus tiles of 256 x 64.
size_t w4_partial_floats(int T, int d_model, int d_inter)
{
    if (T <= 16 || d_inter < kStepK * 8) return 0;
    const size_t few = (size_t)kMostSplits * T * d_model, many = (size_t)2 * kCus * 256 * 64;
    return few < many ? few : many;
}

// Tiles of gate+up, neurons x tokens: the smallest of 64 x 32, 48 or 64 in two sets of waves with which a workgroup on every CU
// does it in one go; past that 256 x 128 (8 waves, for a K worth its start) where its rounds over the chip are three quarters
// full, 128 x 64 in 4 waves where there is more than one for every CU, else in 8.  us, each with some 2.5 of its events:
//   4096 x 14336: T = 45 64 x 48 22.9, 64 x 64 29.3; T = 64 64 x 64 30.4, 64 x 32 34.7; T = 128 128 x 64 (8) 41.0, 64 x 64 55.1; T = 200
//   128 x 64 (4) 65, (8) 79; T = 300 99.7, 256 x 128 105; T = 500 256 x 128 103.5, 128 x 64 (4) 124; T = 2000 431 and 476
//   4096 x 28672: T = 45 128 x 64 (8) 44.2, 64 x 48 47.6; T = 300 128 x 64 (4) 160, 256 x 128 in two rounds of 1.3 205
//   8192 x 8192: T = 80 64 x 48 38.6, 64 x 64 50.8, 64 x 32 57.6; T = 200 128 x 64 (8) 74.0, (4) 85.9
//   2048 x 7168: T = 45 64 x 32 13.2, 64 x 48 15.0; T = 96 64 x 48 16.1, 64 x 64 18.9; T = 300 128 x 64 (4) 35.1; T = 1000 256 x 128 65.0, 128 x 64 (4) 70.2
//   896 x 4864: T = 96 64 x 32 11.1, 64 x 48 12.9; T = 300 128 x 64 (8) 16.5, (4) 17.2
hipError_t launch_w4_tiles(const W4Args &a, const BranchTable &bt)
{
    const int n = bt.d_eff;
    const DownTile t = down_tile(a.T, a.d_model, a.d_inter);
    auto tiles = [&](int rows, int tokens) { return (long long)ceil_div(n, rows) * ceil_div(a.T, tokens); };
    const long long most = tiles(256, 128);
    hipError_t e;
    if (a.T <= 32 || tiles(64, 32) <= kCus)
        e = gate_up<1, 2, 2, 2, 4, 2>(a, bt, t.tokens);
    else if (tiles(64, 48) <= kCus)
        e = gate_up<1, 3, 2, 2, 4, 2>(a, bt, t.tokens);
    else if (tiles(64, 64) <= kCus)
        e = gate_up<1, 4, 1, 2, 4, 2>(a, bt, t.tokens);
    else if (a.d_model >= 2048 && most * 4 >= (most + kCus - 1) / kCus * kCus * 3)
        e = gate_up<2, 8, 1, 1, 8, 2>(a, bt, t.tokens);
    else if (tiles(128, 64) > kCus)
        e = gate_up<2, 4, 1, 1, 4, 2>(a, bt, t.tokens);
    else
        e = gate_up<1, 4, 2, 1, 8, 2>(a, bt, t.tokens);
    if (e != hipSuccess) return e;
    switch (t.kind) {
    case 0: return down<2, 2, 2, 2, 4, 2>(a, bt, t.splits);
    case 1: return down<2, 3, 2, 2, 4, 2>(a, bt, t.splits);
    case 2: return down<2, 4, 2, 1, 4, 2>(a, bt, t.splits);
    case 3: return down<2, 4, 1, 1, 4, 3>(a, bt, t.splits);
    default: return down<4, 4, 1, 1, 4, 2>(a, bt, t.splits);
    }
}

}  // namespace mlpmoe
