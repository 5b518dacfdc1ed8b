// The forward on 4-bit weights for more tokens than one MFMA column block: tiles of rows x tokens.
//
// A workgroup of four waves owns 16 NF tokens and 16 NA rows of weights a wave.  The tokens' x (or H) goes through LDS, shared
// by the waves, 128 of K at a time and D steps ahead, loaded straight into LDS; each wave loads the codes of its own rows
// straight into registers, 16 bytes a lane = one block of 32, also D steps ahead, and widens them there: a weight is widened
// once for 16 NF tokens, half an instruction a weight against NF MFMA columns.  LDS holds a token's 128 values as 16 pieces of
// 16 bytes, piece c at place c ^ (token mod 16), so that the lanes of a cycle read different banks.
//
// Rows are the MFMA's rows and tokens its columns: a lane ends with four neighbouring neurons (features) of a token, one store.
#include "w4_common.h"

namespace mlpmoe {
namespace {

constexpr int kWaves = 4;
constexpr int kScaleLd = 80;             // bytes of LDS for the scales of 2048 of K of a row: 64, and 16 for other banks

// One set of four waves: the ring of x or H, and the scales of its rows.
constexpr int core_lds(int NA, int NF, int D) { return (D + 1) * NF * 4096 + kWaves * NA * 16 * kScaleLd; }

// The codes and scales of 16 rows.
struct Rows {
    __amdgpu_buffer_rsrc_t codes;
    const uint8_t *scales, *end;             // of these rows, of the matrix
    __device__ __forceinline__ void set(const uint8_t *c, const uint8_t *s, int row, int all_rows, int K)
    {
        end = s + (size_t)all_rows * (K / 32);
        codes = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(c + (size_t)row * (K / 2)), 0, 16u * (unsigned)(K / 2),
                                                 0x00027000);
        scales = s + (size_t)row * (K / 32);
    }
};

// acc[a][f] += rows a x tokens f over steps of K.  KW sets of four waves share the steps out: next() names KW at a time (the first
// of them, or -1: no more) and set kw takes the first + kw unless that is past the end or not live; live(s): the blocks of step
// s to be read, four bits, 0 past the end.  The sum is in the first set's waves.  kPlaced: X is H, whose pieces lie in the
// order in which they are read.
template <int NA, int NF, int D, int KW, bool kPlaced, typename Next, typename Live>
__device__ __forceinline__ void sum_steps(f32x4 (&acc)[NA][NF], const Rows (&rows)[NA], const uint16_t *__restrict__ X, int ldx,
                                          int last_token, int K, char *lds, Next next, Live live)
{
    constexpr int R = D + 1, STAGE = NF * 16 * 256, PER = NF + NA;
    static_assert((D - 1) * PER < 63, "the counter of loads in flight holds six bits");
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kWaves;
    const int kw = KW > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / kWaves : 0;
    char *all_lds = lds;
    lds += kw * core_lds(NA, NF, D);
    // this lane's part of the loads into LDS: four tokens a load, 16 pieces each
    unsigned x_off[NF], x_blk[NF];
#pragma unroll
    for (int n = 0; n < NF; ++n) {
        const int t = (wave * NF + n) * 4 + q;
        const unsigned c = (unsigned)(r16 ^ (t & 15));
        x_off[n] = (unsigned)(t < last_token ? t : last_token) * (unsigned)ldx * 2u + (kPlaced ? (c & 3) * 4 + c / 4 : c) * 16u;
        x_blk[n] = c / 4;
    }
    const unsigned w_off = (unsigned)r16 * (unsigned)(K / 2) + (unsigned)q * 16u;
    const char *xb = reinterpret_cast<const char *>(X), *zero = reinterpret_cast<const char *>(g_zero16);

    u32x4 w[R][NA];
    int step[R];
    bool on[R];                             // this lane's block of the step
    auto issue = [&](int s, int slot) {
        const unsigned ok = s < 0 ? 0u : live(s + kw);
        char *dst = lds + slot * STAGE + wave * (NF * 1024);
        const char *src = xb + (size_t)(s < 0 ? 0 : s + kw) * 256;
#pragma unroll
        for (int n = 0; n < NF; ++n) dma16((ok >> x_blk[n]) & 1u ? src + x_off[n] : zero, dst + n * 1024);
        on[slot] = (ok >> q) & 1u;
        const unsigned wo = on[slot] ? w_off + (unsigned)(s + kw) * 64u : 0xffffffffu;
#pragma unroll
        for (int a = 0; a < NA; ++a) w[slot][a] = __builtin_amdgcn_raw_buffer_load_b128(rows[a].codes, wo, 0, 0);
        step[slot] = s;
    };
    // scales: 16 steps' worth of this wave's rows at a time, four lanes a row
    char *my_s = lds + R * STAGE + wave * (NA * 16 * kScaleLd);
    const int s_row = lane >> 2, s_piece = (lane & 3) * 16;
    ScalePiece ahead[NA];
    int chunk = -1, ahead_of = -1;
    auto load_scales = [&](int c) {
#pragma unroll
        for (int a = 0; a < NA; ++a) ahead[a].load(rows[a].scales + (size_t)s_row * (K / 32) + c * 64 + s_piece, rows[a].end);
        ahead_of = c;
    };
#pragma unroll
    for (int u = 0; u < D; ++u) {
        issue(next(), u);
        keep_order();
    }
    for (bool more = true; more;) {
#pragma unroll
        for (int u = 0; u < R; ++u) {
            if (step[u] < 0) {
                more = false;
                break;
            }
            const int s = step[u] + kw;
            if (s / 16 != chunk) {
                chunk = s / 16;
                if (ahead_of != chunk) load_scales(chunk);
#pragma unroll
                for (int a = 0; a < NA; ++a) ahead[a].place(my_s + (a * 16 + s_row) * kScaleLd + s_piece);
                if ((chunk + 1) * 64 < K / 32) load_scales(chunk + 1);
            }
            pipeline_barrier<(D - 1) * PER>();
            issue(next(), (u + D) % R);
            const char *st = lds + u * STAGE + r16 * 256;
            float scale[NA];
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                scale[a] = scale_of(*reinterpret_cast<const uint8_t *>(my_s + (a * 16 + r16) * kScaleLd + s % 16 * 4 + q));
                scale[a] = on[u] ? scale[a] : 1.0f;      // that of a block that is not read may be no number
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bf16x8 wv[NA];
#pragma unroll
                for (int a = 0; a < NA; ++a) wv[a] = widen8(w[u][a][j], scale[a]);
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    const bf16x8 xv = *reinterpret_cast<const bf16x8 *>(st + f * (16 * 256) + (((q * 4 + j) ^ r16) * 16));
#pragma unroll
                    for (int a = 0; a < NA; ++a) acc[a][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[a], xv, acc[a][f], 0, 0, 0);
                }
            }
        }
    }
    pipeline_barrier<0>();                  // what is still on its way into LDS is zeros; let it land
    if constexpr (KW > 1) {
        static_assert(KW == 2 && kWaves * NA * NF * 1024 <= KW * core_lds(NA, NF, D), "the second set's sums fit where the rings were");
        f32x4 *s = reinterpret_cast<f32x4 *>(all_lds) + wave * (NA * NF * 64) + lane;
        if (kw == 1) {
#pragma unroll
            for (int i = 0; i < NA * NF; ++i) s[i * 64] = acc[i / NF][i % NF];
        }
        pipeline_barrier<0>();
        if (kw == 0) {
#pragma unroll
            for (int i = 0; i < NA * NF; ++i) acc[i / NF][i % NF] += s[i * 64];
        }
    }
}

// Workgroup ids to tiles: the token tiles of a row tile on one XCD, one after the other, since they read the same weights.
// Returns false past the last tile.  grid = 8 * ceil(row_tiles / 8) * token_tiles.
__device__ __forceinline__ bool tile_of(int id, int row_tiles, int token_tiles, int &row, int &token)
{
    const int xcd = id % 8, at = id / 8;
    token = at % token_tiles;
    row = at / token_tiles * 8 + xcd;
    return row < row_tiles;
}

// A wave takes NR groups of 16 neurons that a live branch reaches into, at multiples of 16.
template <int NR, int NF, int D, int KW, int W, bool kOneRun>
__global__ void __launch_bounds__(KW * kWaves * 64, W)
w4_tile_gate_up(const uint16_t *__restrict__ x, int T, int K, int d_inter, const uint8_t *__restrict__ gc, const uint8_t *__restrict__ gs,
                const uint8_t *__restrict__ uc, const uint8_t *__restrict__ us, uint16_t *__restrict__ H, int ldh,
                const uint8_t *__restrict__ route, int row_tiles, int token_tiles, Range run, BranchTable bt)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int row, token;
    if (!tile_of(blockIdx.x, row_tiles, token_tiles, row, token)) return;
    const int t0 = token * 16 * NF, nt = T - t0 < 16 * NF ? T - t0 : 16 * NF;
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kWaves;
    BranchLanes br(bt);
    Groups<16, kOneRun> groups(run);
    if constexpr (kOneRun) {
        if (row == 0) clear_edges(run, H + (size_t)t0 * ldh, ldh, nt, wave, kWaves);
    } else {
        __shared__ unsigned any[2];
        const OffsetLanes off(bt);
        const unsigned long long live = live_of(bt, route, t0, nt, any);
        groups = Groups<16, kOneRun>(off, live);
        if (row == 0) clear_edges(off, bt.B, live, H + (size_t)t0 * ldh, ldh, nt, wave, kWaves);
        if (row * kWaves * NR >= groups.total) return;
    }

    int group[NR];
    Rows rows[2 * NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int idx = (row * kWaves + wave) * NR + i;
        group[i] = groups(idx < groups.total ? idx : groups.total - 1);
        rows[i].set(gc, gs, group[i] * 16, d_inter, K);
        rows[NR + i].set(uc, us, group[i] * 16, d_inter, K);
        if (idx >= groups.total) group[i] = -1;
    }
    f32x4 acc[2 * NR][NF];
#pragma unroll
    for (int a = 0; a < 2 * NR; ++a)
#pragma unroll
        for (int f = 0; f < NF; ++f) acc[a][f] = f32x4{0, 0, 0, 0};
    const int steps = (K + kStepK - 1) / kStepK, blocks = K / 32;
    int at = -KW;
    sum_steps<2 * NR, NF, D, KW, false>(
        acc, rows, x + (size_t)t0 * K, K, nt - 1, K, lds, [&]() { return (at += KW) < steps ? at : -1; },
        [&](int s) { return blocks - s * 4 >= 4 ? 15u : blocks - s * 4 <= 0 ? 0u : (1u << (blocks - s * 4)) - 1u; });
    if (KW > 1 && threadIdx.x >= kWaves * 64) return;

#pragma unroll
    for (int i = 0; i < NR; ++i) {
        if (group[i] < 0) continue;
        const int n0 = group[i] * 16;
        gated<16, NF>(
            br, bt, n0, n0 + 4 * q, [&](int f, int e, float &g, float &u) { g = acc[i][f][e], u = acc[NR + i][f][e]; },
            [&](int f, int b) {
                const int t = f * 16 + r16;
                return kOneRun || !route || (t < nt && route[(size_t)(t0 + t) * bt.B + b] != 0);
            },
            [&](int f, uint2 h) {
                const int t = f * 16 + r16;
                if (t < nt) *reinterpret_cast<uint2 *>(H + (size_t)(t0 + t) * ldh + h_place(n0 + 4 * q)) = h;
            });
    }
}

// K is cut into `splits` ranges; with more than one the sums go to partial [splits][T][d_model].
template <int NA, int NF, int D, int KW, int W, bool kOneRun>
__global__ void __launch_bounds__(KW * kWaves * 64, W)
w4_tile_down(const uint16_t *__restrict__ H, int ldh, int T, int K, const uint8_t *__restrict__ dc, const uint8_t *__restrict__ ds,
             int d_model, void *__restrict__ out, int out_bf16, float *__restrict__ partial, int splits,
             const uint8_t *__restrict__ route, int row_tiles, int token_tiles, Range run, BranchTable bt)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int row, token;
    if (!tile_of(blockIdx.x, row_tiles * splits, token_tiles, row, token)) return;
    const int z = row / row_tiles;
    row -= z * row_tiles;
    const int t0 = token * 16 * NF, nt = T - t0 < 16 * NF ? T - t0 : 16 * NF;
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kWaves;
    const int blocks = K / 32;
    uint32_t *bits = reinterpret_cast<uint32_t *>(lds + KW * core_lds(NA, NF, D));
    if constexpr (!kOneRun) {
        __shared__ unsigned any[2];
        const OffsetLanes off(bt);
        mark_blocks(off, live_of(bt, route, t0, nt, any), bits, blocks);
    }
    const int first = kOneRun ? run.beg / 32 : 0, last = kOneRun ? (run.end + 31) / 32 : blocks;      // live blocks lie here
    Rows rows[NA];
    int group[NA];
#pragma unroll
    for (int a = 0; a < NA; ++a) {
        group[a] = (row * kWaves + wave) * NA + a;
        rows[a].set(dc, ds, (group[a] * 16 < d_model ? group[a] * 16 : d_model - 16), d_model, K);
    }
    f32x4 acc[NA][NF];
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int f = 0; f < NF; ++f) acc[a][f] = f32x4{0, 0, 0, 0};
    const int s_beg = first / 4, steps = (last + 3) / 4 - s_beg;
    const int end = s_beg + (int)((long long)steps * (z + 1) / splits);
    int at = s_beg + (int)((long long)steps * z / splits) - KW;
    auto live = [&](int s) -> unsigned {
        if (s >= end) return 0u;
        if (!kOneRun) return ((unsigned)__builtin_amdgcn_readfirstlane(bits[s / 8]) >> (s % 8 * 4)) & 15u;      // 0 past the last block
        unsigned m = last - s * 4 >= 4 ? 15u : (1u << (last - s * 4)) - 1u;
        if (first > s * 4) m &= ~((1u << (first - s * 4)) - 1u);
        return m;
    };
    sum_steps<NA, NF, D, KW, true>(
        acc, rows, H + (size_t)t0 * ldh, ldh, nt - 1, K, lds,
        [&]() {
            at += KW;
            if (!kOneRun)
                for (; at < end; at += KW) {
                    unsigned any = 0;
#pragma unroll
                    for (int k = 0; k < KW; ++k) any |= live(at + k);
                    if (any) break;
                }
            return at < end ? at : -1;
        },
        live);
    if (KW > 1 && threadIdx.x >= kWaves * 64) return;

#pragma unroll
    for (int a = 0; a < NA; ++a) {
        const int m = group[a] * 16 + 4 * q;
        if (m >= d_model) continue;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int t = f * 16 + r16;
            if (t >= nt) continue;
            const size_t to = (size_t)(t0 + t) * d_model + m;
            if (splits > 1)
                *reinterpret_cast<f32x4 *>(partial + (size_t)z * T * d_model + to) = acc[a][f];
            else if (out_bf16)
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + to) =
                    uint2{(uint32_t)to_bf16(acc[a][f][0]) | (uint32_t)to_bf16(acc[a][f][1]) << 16,
                          (uint32_t)to_bf16(acc[a][f][2]) | (uint32_t)to_bf16(acc[a][f][3]) << 16};
            else
                *reinterpret_cast<f32x4 *>(static_cast<float *>(out) + to) = acc[a][f];
        }
    }
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

template <int NR, int NF, int D, int KW, int W>
hipError_t gate_up(const W4Args &a, const BranchTable &bt)
{
    int groups = 0;                          // an upper bound: a group shared by two branches counts for both
    const Range run = run_of(a, bt);
    const bool one = run.end > 0;
    for (int b = 0; b < bt.B; ++b)
        if (((bt.active >> b) & 1) && bt.off[b + 1] > bt.off[b]) groups += ceil_div(bt.off[b + 1], 16) - bt.off[b] / 16;
    if (one) groups = ceil_div(run.end, 16) - run.beg / 16;
    const int row_tiles = ceil_div(groups, kWaves * NR), token_tiles = ceil_div(a.T, 16 * NF);
    const size_t lds = KW * core_lds(2 * NR, NF, D);
    const hipError_t e = one ? allow_lds<w4_tile_gate_up<NR, NF, D, KW, W, true>>((int)lds, "w4_tile_gate_up attribute")
                             : allow_lds<w4_tile_gate_up<NR, NF, D, KW, W, false>>((int)lds, "w4_tile_gate_up attribute");
    if (e != hipSuccess) return e;
    ProfileScope ps(MLPMOE_KERNEL_W4_GATE_UP, a.stream);
    (one ? w4_tile_gate_up<NR, NF, D, KW, W, true> : w4_tile_gate_up<NR, NF, D, KW, W, false>)
        <<<ceil_div(row_tiles, 8) * 8 * token_tiles, KW * kWaves * 64, lds, a.stream>>>(
            static_cast<const uint16_t *>(a.x), a.T, a.d_model, a.d_inter, a.gc, a.gs, a.uc, a.us, static_cast<uint16_t *>(a.H), a.ldh, a.route,
            row_tiles, token_tiles, run, bt);
    return launch_status("w4_tile_gate_up launch");
}

template <int NA, int NF, int D, int KW, int W>
hipError_t down(const W4Args &a, const BranchTable &bt, int splits)
{
    const int row_tiles = ceil_div(a.d_model, 16 * kWaves * NA), token_tiles = ceil_div(a.T, 16 * NF);
    const Range run = run_of(a, bt);
    const bool one = run.end > 0;
    const size_t lds = KW * core_lds(NA, NF, D) + (one ? 0 : (size_t)ceil_div(a.d_inter / 32, 32) * 4);
    hipError_t e = one ? allow_lds<w4_tile_down<NA, NF, D, KW, W, true>>((int)lds, "w4_tile_down attribute")
                       : allow_lds<w4_tile_down<NA, NF, D, KW, W, false>>((int)lds, "w4_tile_down attribute");
    if (e != hipSuccess) return e;
    {
        ProfileScope ps(MLPMOE_KERNEL_W4_DOWN, a.stream);
        (one ? w4_tile_down<NA, NF, D, KW, W, true> : w4_tile_down<NA, NF, D, KW, W, false>)
            <<<ceil_div(row_tiles * splits, 8) * 8 * token_tiles, KW * kWaves * 64, lds, a.stream>>>(
                static_cast<const uint16_t *>(a.H), a.ldh, a.T, a.d_inter, a.dc, a.ds, a.d_model, a.out, a.out_bf16, a.partial, splits,
                a.route, row_tiles, token_tiles, run, bt);
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

// K ranges of the down projection: enough workgroups to fill the chip twice.
int w4_splits(int T, int d_model, int d_inter)
{
    const int tiles = ceil_div(d_model, 256) * ceil_div(T, 64);
    int s = 1;
    while (s < 8 && tiles * s * 2 <= 512) s *= 2;
    return s;
}

hipError_t launch_w4_tiles(const W4Args &a, const BranchTable &bt)
{
    const int s = w4_splits(a.T, a.d_model, a.d_inter);
    hipError_t e;
    if (a.T <= 48) {
        e = gate_up<1, 3, 3, 2, 2>(a, bt);
        return e == hipSuccess ? down<2, 3, 3, 2, 2>(a, bt, s) : e;
    }
    if (a.T <= 192) {
        e = gate_up<1, 4, 3, 1, 2>(a, bt);
        return e == hipSuccess ? down<2, 4, 3, 1, 2>(a, bt, s) : e;
    }
    e = gate_up<2, 4, 1, 1, 2>(a, bt);
    return e == hipSuccess ? down<4, 4, 1, 1, 2>(a, bt, s) : e;
}

}  // namespace mlpmoe
