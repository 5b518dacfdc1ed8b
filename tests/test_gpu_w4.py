"""4-bit weights on the GPU: conversions exactly against the oracle, the forward through the same checks as the bf16 paths
(every stored h one that fp32 can round to, the result the down projection of the stored H), on the dequantised weights."""
import numpy as np
import pytest

from gpu_util import check_bf16_flip_aware, widen
from oracle import w4
from paper_2511_21089_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mm():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2511_21089_amd import binding
    return binding


# ------------------------------------------------------------------------------------------------ conversions
@pytest.mark.parametrize("elem", [2, 4])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (17, 96), (40, 416), (5, 1056)])
def test_quantize_and_dequantize(mm, rows, cols, elem):
    import torch
    g = torch.Generator().manual_seed(rows)
    W = torch.randn((rows, cols), generator=g) * torch.exp2(torch.randint(-40, 40, (rows, cols // 32), generator=g).float()
                                                           ).repeat_interleave(32, 1)
    W = W.to(torch.bfloat16 if elem == 2 else torch.float32)
    W[0, :8] = torch.tensor([6., 5., 3.5, 2.5, 1.75, 1.25, 0.75, 0.25])      # every halfway case, and both zeros
    W[0, 8:32] = -torch.arange(24) / 4.
    codes, scales = mm.mlpmoe_w4_quantize(W.cuda())
    o_codes, o_scales = w4.quantize(W.double().numpy())
    assert np.array_equal(codes.cpu().numpy(), o_codes) and np.array_equal(scales.cpu().numpy(), o_scales)
    want = w4.dequantize(o_codes, o_scales)
    for dtype in (torch.bfloat16, torch.float32):
        V = mm.mlpmoe_w4_dequantize(codes, scales, dtype)
        assert V.dtype == dtype and np.array_equal(V.double().cpu().numpy(), want)
        assert np.array_equal(torch.signbit(V).cpu().numpy(), np.signbit(want))
    # what is on the grid stays on it
    again = mm.mlpmoe_w4_quantize(mm.mlpmoe_w4_dequantize(codes, scales))
    assert torch.equal(mm.mlpmoe_w4_dequantize(*again), mm.mlpmoe_w4_dequantize(codes, scales))


def test_every_code_and_scale(mm):
    import torch
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1).reshape(256 * 16, 16)
    scales = torch.arange(256, dtype=torch.uint8).repeat_interleave(16).view(-1, 1)
    # elements from 2 on at the scale 2^127, and from 4 on at 2^126, are 2^128 and more, past the largest bf16 value
    # (2 - 2^-7) 2^127: infinity there
    with np.errstate(over="ignore"):
        want = w4.dequantize(codes.numpy(), scales.numpy()).astype(np.float32)
    assert np.isinf(want[254 * 16:255 * 16]).any() and np.isfinite(want[:253 * 16]).all()
    got = mm.mlpmoe_w4_dequantize(codes.cuda(), scales.cuda()).float().cpu().numpy()
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("elem", [2, 4])
def test_quantize_special_blocks(mm, elem):
    import torch
    W = torch.zeros((6, 64))
    W[0, 1], W[1, 33], W[2, 0] = float("inf"), float("nan"), -float("inf")
    W[3, :32] = torch.finfo(torch.bfloat16).max
    W[4, :32] = 2.0 ** -133                                    # below the smallest normal number
    W[5, 32] = 2.0 ** -125
    W = W.to(torch.bfloat16 if elem == 2 else torch.float32)
    codes, scales = mm.mlpmoe_w4_quantize(W.cuda())
    o_codes, o_scales = w4.quantize(W.double().numpy())
    assert np.array_equal(codes.cpu().numpy(), o_codes) and np.array_equal(scales.cpu().numpy(), o_scales)


def test_conversion_of_many(mm):
    """More pieces than a grid has lanes, the last rows checked; and matrices of no rows."""
    import torch
    W = torch.randn((40000, 2048), device="cuda").to(torch.bfloat16)
    codes, scales = mm.mlpmoe_w4_quantize(W)
    for lo in (0, 20011, 39992):
        o = w4.quantize(W[lo:lo + 8].double().cpu().numpy())
        assert np.array_equal(codes[lo:lo + 8].cpu().numpy(), o[0]) and np.array_equal(scales[lo:lo + 8].cpu().numpy(), o[1])
    V = mm.mlpmoe_w4_dequantize(codes, scales)
    assert np.array_equal(V[-8:].double().cpu().numpy(), w4.dequantize(codes[-8:].cpu().numpy(), scales[-8:].cpu().numpy()))
    none = mm.mlpmoe_w4_quantize(W[:0])
    assert none[0].shape == (0, 1024) and mm.mlpmoe_w4_dequantize(*none).shape == (0, 2048)


def test_conversion_past_32_bits(mm):
    import torch
    W = torch.zeros((70000, 32768), dtype=torch.bfloat16, device="cuda")
    W[-3:] = torch.randn((3, 32768), generator=torch.Generator().manual_seed(1)).cuda().to(torch.bfloat16)
    codes, scales = mm.mlpmoe_w4_quantize(W)
    o = w4.quantize(W[-4:].double().cpu().numpy())
    assert np.array_equal(codes[-4:].cpu().numpy(), o[0]) and np.array_equal(scales[-4:].cpu().numpy(), o[1])
    assert not codes[:-3].any()
    V = mm.mlpmoe_w4_dequantize(codes, scales, out=W)
    assert np.array_equal(V[-4:].double().cpu().numpy(), w4.dequantize(codes[-4:].cpu().numpy(), scales[-4:].cpu().numpy()))


# ------------------------------------------------------------------------------------------------ forward
def layer(mm, T, d_model, widths, seed, scale=0.02):
    """x as bf16 bits, packed weights on the GPU, their values as float32, offsets, alpha."""
    import torch
    off = np.concatenate(([0], np.cumsum(widths))).astype(np.int32)
    d_inter = int(off[-1])
    rng = np.random.default_rng(seed)
    x, *W = synth.random_layer(rng, T, d_model, d_inter, "bf16", w_scale=scale)
    packed, values = [], []
    for w in W:
        c, s = mm.mlpmoe_w4_quantize(mm.bf16_tensor(w))
        packed.append((c, s))
        values.append(w4.dequantize(c.cpu().numpy(), s.cpu().numpy()).astype(np.float32))
    return x, packed, values, off, rng.uniform(0.8, 1.2, size=len(widths)).astype(np.float32)


def run(mm, x, packed, off, alpha, mask, route=None, out_dtype=None):
    import torch
    T, d_model = x.shape
    d_inter = int(off[-1])
    ws = torch.full((mm.mlpmoe_w4_workspace_bytes(T, d_model, d_inter, len(alpha)),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((T, d_model), float("nan"), dtype=out_dtype or torch.float32, device="cuda")
    r = None if route is None else torch.from_numpy(route).cuda()
    mm.mlpmoe_forward_w4(mm.bf16_tensor(x), *packed, off, alpha, mask, route=r, out=out, workspace=ws)
    torch.cuda.synchronize()
    # H: rows of whole 128s
    ld = (d_inter + 127) // 128 * 128
    H = ws[:T * ld * 2].view(torch.int16).view(T, ld)[:, :d_inter].contiguous().cpu().numpy().view(np.uint16)
    return out, synth.bf16_bits_to_f32(H).astype(np.float64)


def check(mm, T, d_model, widths, seed=0, off_branches=(), route=None, label=""):
    import torch
    x, packed, values, off, alpha = layer(mm, T, d_model, widths, seed)
    mask = np.ones(len(widths), np.uint8)
    mask[list(off_branches)] = 0
    label = label or "T=%d %dx%d B=%d" % (T, d_model, off[-1], len(widths))
    print(label, flush=True)
    out, H = run(mm, x, packed, off, alpha, mask, route)
    check_bf16_flip_aware(out.cpu().numpy(), H, x, *values, off, alpha, mask, route=route, label=label)
    got, _ = run(mm, x, packed, off, alpha, mask, route, torch.bfloat16)
    assert torch.equal(got, out.to(torch.bfloat16))            # the same sums, rounded once
    return x, packed, values, off, alpha, mask, out


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 33, 64, 65, 100])
@pytest.mark.parametrize("d_model,widths", [(32, [32]), (64, [96, 64]), (416, [100, 60, 0, 224]), (896, [608] * 8)])
def test_sizes(mm, T, d_model, widths):
    check(mm, T, d_model, widths, seed=T)


@pytest.mark.parametrize("T", [1, 5, 16, 31, 130, 300])
@pytest.mark.parametrize("d_model,widths", [(1056, [33, 7, 1, 87, 512]), (4640, [160, 96]), (512, [1500, 1060]), (9248, [64])])
def test_odd_boundaries_and_long_rows(mm, T, d_model, widths):
    check(mm, T, d_model, widths, seed=T + 1)


@pytest.mark.parametrize("T", [1, 9, 16, 40, 200])
def test_inactive_branches(mm, T):
    """Pruned branches hold scales of 255 wherever no active branch shares the block: nothing of them reaches out."""
    import torch
    widths, gone = [70, 90, 300, 4, 20, 156, 512], (1, 3, 5)
    x, packed, values, off, alpha = layer(mm, T, 256, widths, seed=T)
    mask = np.ones(len(widths), np.uint8)
    mask[list(gone)] = 0
    want, _ = run(mm, x, packed, off, alpha, mask)
    live = np.zeros(int(off[-1]) // 32, bool)
    for b in range(len(widths)):
        if mask[b]:
            live[off[b] // 32:(off[b + 1] - 1) // 32 + 1] = True
    for b in gone:
        packed[0][1][off[b]:off[b + 1]] = 255
        packed[1][1][off[b]:off[b + 1]] = 255
        packed[1][0][off[b]:off[b + 1]] = 119
    packed[2][1][:, torch.from_numpy(~live).cuda()] = 255
    got, H = run(mm, x, packed, off, alpha, mask)
    assert torch.equal(got, want)
    check_bf16_flip_aware(got.cpu().numpy(), H, x, *[np.nan_to_num(v) for v in values], off, alpha, mask)


def routes(rng, T, B, k):
    r = np.zeros((T, B), np.uint8)
    for t in range(T):
        r[t, rng.choice(B, size=k, replace=False)] = rng.integers(1, 256)
    return r


@pytest.mark.parametrize("T", [1, 3, 16, 17, 50, 300])
@pytest.mark.parametrize("widths", [[128] * 8, [100, 28, 33, 95, 256, 128, 64, 64]])
def test_routed(mm, T, widths):
    rng = np.random.default_rng(T)
    r = routes(rng, T, 8, 3)
    if T > 2:
        r[T // 2] = 0                                   # a token that takes nothing
        r[0] = 1                                        # one that takes everything
    *_, out = check(mm, T, 224, widths, seed=T, off_branches=(2,), route=r)
    if T > 2:
        assert not out[T // 2].any()
    # few branches taken at all, and none
    few = np.zeros_like(r)
    few[:, 5] = 1
    check(mm, T, 224, widths, seed=T, route=few)
    *_, out = check(mm, T, 224, widths, seed=T, route=0 * few)
    assert not out.any()


@pytest.mark.parametrize("T,run_length,d_model,widths", [
    (T, n, d, w) for T, n in [(16, 5), (40, 9), (64, 32), (64, 10), (300, 20), (300, 48)]
    for d, w in [(224, [100, 28, 33, 95, 256, 128, 64, 64]), (1024, [512] * 8)]
] + [(16, 5, 51200, [128] * 4), (40, 9, 51200, [128] * 4)])
def test_routed_by_sequences(mm, T, run_length, d_model, widths):
    """Neighbouring tokens take the same branches, other runs of tokens others: a branch that part of a workgroup's tokens take
    is there for the rest, whose values in the workspace are nobody's."""
    B = len(widths)
    r = np.zeros((T, B), np.uint8)
    for i, t in enumerate(range(0, T, run_length)):
        r[t:t + run_length, [(2 * i) % B, (2 * i + 1) % B]] = 1
    check(mm, T, d_model, widths, seed=T + run_length, route=r)


@pytest.mark.parametrize("kind", ["one run", "some off", "routed"])
@pytest.mark.parametrize("T", [1, 5, 8, 13, 16])
@pytest.mark.parametrize("d_model,widths", [(4096, [96, 32]), (2080, [500, 524, 1024]), (1024, [2000, 1000, 1096]), (6144, [1100, 948])])
def test_waves_that_share(mm, T, d_model, widths, kind):
    """Few neurons for many waves: K and the loads of x shared out, with and without a part left over."""
    B = len(widths)
    r = None
    if kind == "routed":
        r = np.zeros((T, B), np.uint8)
        r[np.arange(T), np.arange(T) % 2] = 1
    check(mm, T, d_model, widths, seed=T, off_branches=(1,) if kind == "some off" else (), route=r)


@pytest.mark.parametrize("kind", ["one run", "some off", "routed"])
@pytest.mark.parametrize("T,d_model,widths", [(300, 96, [256] * 8), (400, 96, [500, 512, 524, 512]), (600, 160, [256] * 8), (1100, 96, [2000, 48]),
                                              (1600, 2048, [1024, 1000, 1048, 1024])])
def test_many_tokens(mm, T, d_model, widths, kind):
    """Enough tiles for every shape of them."""
    B = len(widths)
    r = None
    if kind == "routed":
        r = routes(np.random.default_rng(T), T, B, 1)
        r[:, 0] = 0
        r[:T // 3, B - 1] = 1
    check(mm, T, d_model, widths, seed=T, off_branches=(1,) if kind == "some off" and B > 2 else (), route=r)


@pytest.mark.parametrize("T", [1, 3, 8, 16, 17, 45, 65])
@pytest.mark.parametrize("d_model,widths,gone", [(131072, [64], ()), (131040, [40, 24], ()), (32, [131072], ()), (32, [50000, 40, 81032], (1,)),
                                                 (64, [131040], ())])
def test_longest_rows(mm, T, d_model, widths, gone):
    rng = np.random.default_rng(T)
    check(mm, T, d_model, widths, seed=T, off_branches=gone)
    if len(widths) > 1:
        check(mm, T, d_model, widths, seed=T, off_branches=gone, route=routes(rng, T, len(widths), 1))


@pytest.mark.parametrize("T", [1, 9, 40])
def test_weights_past_32_bits(mm, T):
    """The largest matrices, 8 GiB of codes each, zero but for the last neurons: the layer that has only these.  The sums over
    d_model may be in another order, so an h may be rounded the other way: 2^-8 of it, and of the result."""
    import torch
    n, some = 131072, 96
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, n), generator=g, device="cuda").to(torch.bfloat16)
    far, near = [], []
    for rows, cols in ((n, n), (n, n), (n, n)):
        codes = torch.zeros((rows, cols // 2), dtype=torch.uint8, device="cuda")
        scales = torch.full((rows, cols // 32), 118, dtype=torch.uint8, device="cuda")
        where = (slice(n - some, n), slice(None)) if len(far) < 2 else (slice(None), slice((n - some) // 2, n // 2))
        codes[where] = torch.randint(256, codes[where].shape, generator=g, dtype=torch.uint8, device="cuda")
        far.append((codes, scales))
        part = scales[where] if len(far) < 3 else scales[:, (n - some) // 32:]
        near.append((codes[where].contiguous(), part.contiguous()))
    al, mk = np.ones(1, np.float32), np.ones(1, np.uint8)
    got = mm.mlpmoe_forward_w4(x, *far, np.array([0, n], np.int32), al, mk, out_dtype=torch.float32)
    want = mm.mlpmoe_forward_w4(x, *near, np.array([0, some], np.int32), al, mk, out_dtype=torch.float32).double()
    rms = want.square().mean().sqrt()
    assert rms > 0 and float((got.double() - want).abs().max()) <= 1e-2 * float(rms)


def test_most_tokens(mm):
    """As many tokens as a call takes, 999 of them again and again: the same bits wherever they stand."""
    import torch
    T, n = 65535 * 16, 999
    x, packed, values, off, alpha = layer(mm, n, 64, [40, 24], seed=8)
    mask = np.ones(2, np.uint8)
    small, _ = run(mm, x, packed, off, alpha, mask)
    xs = mm.bf16_tensor(x).repeat(T // n + 1, 1)[:T].contiguous()
    out = mm.mlpmoe_forward_w4(xs, *packed, off, alpha, mask, out_dtype=torch.float32)
    first = out[:n]
    assert torch.equal(out, first.repeat(T // n + 1, 1)[:T])
    assert float((first - small).abs().max()) <= 1e-2 * float(small.square().mean().sqrt())


@pytest.mark.parametrize("T", [1, 20, 150])
def test_nothing_active_and_no_tokens(mm, T):
    import torch
    x, packed, values, off, alpha = layer(mm, T, 64, [32, 64], seed=1)
    for dtype in (torch.float32, torch.bfloat16):
        out, _ = run(mm, x, packed, off, alpha, np.zeros(2, np.uint8), out_dtype=dtype)
        assert not out.any()
        assert run(mm, x[:0], packed, off, alpha, np.ones(2, np.uint8), out_dtype=dtype)[0].shape == (0, 64)


@pytest.mark.parametrize("T", [4, 16, 40, 200])
def test_tokens_do_not_mix(mm, T):
    """A token of infinities and not-a-numbers leaves the others as they are, bit for bit."""
    import torch
    x, packed, values, off, alpha = layer(mm, T, 288, [200, 120], seed=3)
    mask = np.ones(2, np.uint8)
    want, _ = run(mm, x, packed, off, alpha, mask)
    bad = x.copy()
    bad[1, 7], bad[T - 1, 3] = 0x7FC0, 0x7F80
    got, _ = run(mm, bad, packed, off, alpha, mask)
    others = [t for t in range(T) if t not in (1, T - 1)]
    assert torch.equal(got[others], want[others])
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[T - 1]).all()


@pytest.mark.parametrize("T", [1, 16, 33, 200])
def test_in_place_repeat_and_owned_workspace(mm, T):
    """The result over x, in the library's workspace, and again: the same bits."""
    import torch
    x, packed, values, off, alpha = layer(mm, T, 256, [300, 340], seed=5)
    mask = np.ones(2, np.uint8)
    want, _ = run(mm, x, packed, off, alpha, mask, out_dtype=torch.bfloat16)
    xt = mm.bf16_tensor(x)
    for _ in range(3):
        assert torch.equal(mm.mlpmoe_forward_w4(xt, *packed, off, alpha, mask), want)
    mm.mlpmoe_forward_w4(xt, *packed, off, alpha, mask, out=xt)
    assert torch.equal(xt, want)


@pytest.mark.parametrize("T", [7, 100])
def test_rows_behind_the_last_stay(mm, T):
    import torch
    x, packed, values, off, alpha = layer(mm, T, 96, [64, 64], seed=6)
    for dtype in (torch.float32, torch.bfloat16):
        buf = torch.full((T + 16, 96), 5.0, dtype=dtype, device="cuda")
        mm.mlpmoe_forward_w4(mm.bf16_tensor(x), *packed, off, alpha, np.ones(2, np.uint8), out=buf[:T])
        assert (buf[T:] == 5.0).all() and torch.isfinite(buf).all()


@pytest.mark.parametrize("T", [3, 16, 45, 300])
def test_graph(mm, T):
    """Two captured calls that share a workspace, replayed with new x and routes."""
    import torch
    x, packed, values, off, alpha = layer(mm, T, 256, [128] * 4, seed=8)
    mask = np.ones(4, np.uint8)
    rng = np.random.default_rng(1)
    ra, rb = (torch.from_numpy(routes(rng, T, 4, 2)).cuda() for _ in range(2))
    xa = mm.bf16_tensor(x)
    xb = torch.roll(xa, 3, dims=1)
    ws = torch.empty(mm.mlpmoe_w4_workspace_bytes(T, 256, 512, 4), dtype=torch.uint8, device="cuda")
    eager = {}
    for name, a, r in (("a", xa, ra), ("b", xb, rb)):
        eager[name] = mm.mlpmoe_forward_w4(a, *packed, off, alpha, mask, route=r, workspace=ws)
    torch.cuda.synchronize()
    bx, br = xa.clone(), ra.clone()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            first = mm.mlpmoe_forward_w4(bx, *packed, off, alpha, mask, route=br, workspace=ws)
            second = mm.mlpmoe_forward_w4(xb, *packed, off, alpha, mask, route=rb, workspace=ws)
    torch.cuda.synchronize()
    for rep in range(4):
        which = "ab"[rep % 2]
        bx.copy_(xa if which == "a" else xb)
        br.copy_(ra if which == "a" else rb)
        first.fill_(3)
        second.fill_(3)
        ws.fill_(255)
        graph.replay()
        mm.mlpmoe_forward_w4(xa, *packed, off, alpha, mask, workspace=ws)      # the program's own work between the replays
        torch.cuda.synchronize()
        assert torch.equal(first, eager[which]) and torch.equal(second, eager["b"]), rep


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("T", [2, 40])
def test_two_streams_at_once(mm, T):
    """Two layers on two streams, each with its workspace, again and again: what each gives alone."""
    import torch
    jobs = []
    for seed in (1, 2):
        x, packed, values, off, alpha = layer(mm, T, 512, [300, 212, 512], seed=seed)
        ws = torch.empty(mm.mlpmoe_w4_workspace_bytes(T, 512, int(off[-1]), 3), dtype=torch.uint8, device="cuda")
        args = (mm.bf16_tensor(x), *packed, off, alpha, np.ones(3, np.uint8))
        jobs.append((args, ws, mm.mlpmoe_forward_w4(*args, workspace=ws), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for args, ws, _, stream in jobs:
            with torch.cuda.stream(stream):
                got.append(mm.mlpmoe_forward_w4(*args, workspace=ws))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert torch.equal(out, jobs[i % 2][2])


@pytest.mark.parametrize("T", [1, 16, 70])
def test_router_and_forward_together(mm, T):
    """Logits -> route -> the forward on 4-bit weights, as a server runs them; the counts are those of the routes, and a
    token's result is that of the branches its logits lead in."""
    import torch
    widths = [96, 128, 64, 160, 64]
    x, packed, values, off, alpha = layer(mm, T, 192, widths, seed=11)
    xt = mm.bf16_tensor(x)
    mask = np.array([1, 1, 0, 1, 1], np.uint8)
    logits = (xt.float() @ torch.randn((192, 5), generator=torch.Generator().manual_seed(2)).cuda()).to(torch.bfloat16)
    real = torch.ones(T, dtype=torch.bool, device="cuda")
    real[T - T // 4:] = False
    route, probs, counts, loss = mm.mlpmoe_route_topk(logits, 2, mask, real)
    out, H = run(mm, x, packed, off, alpha, mask, route.cpu().numpy())
    check_bf16_flip_aware(out.cpu().numpy(), H, x, *values, off, alpha, mask, route=route.cpu().numpy())
    assert torch.equal(counts[:5], route.sum(0, dtype=torch.int32)) and int(counts[5]) == int(real.sum())
    assert int(counts[2]) == 0 and not out[~real].any()
    lead = torch.where(torch.from_numpy(mask != 0).cuda(), logits.float(), -float("inf")).argmax(1)
    assert route[real].gather(1, lead[real][:, None]).all()
    d = mm.mlpmoe_route_backward(probs, counts, None, torch.ones(1, device="cuda"), mask)
    assert not d[~real].any() and not d[:, 2].any() and abs(float(d.sum())) < 1e-5
