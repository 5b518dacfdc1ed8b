"""The router on the GPU against the float64 oracle: routes and counts exactly, probabilities, loss and gradient within
bounds counted in roundings."""
import numpy as np
import pytest

from oracle import route as orc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24           # half a step of float


@pytest.fixture(scope="module")
def mm():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2511_21089_amd import binding
    return binding


def logits_of(seed, T, B, dtype, banned=0.0, spread=1.5):
    """(GPU tensor, the same values in float64)."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((T, B), generator=g) * spread).to(dtype)
    if banned:
        x[torch.rand((T, B), generator=g) < banned] = -float("inf")
    return x.cuda(), x.double().numpy()


def prob_bound(x, p):
    """|error| of exp(x - max) / sum in float: x - max and its product with log2(e) are off by a rounding each, which moves the
    exponential by that times |x - max|; the exponential, the sum of B terms (and what it does to the quotient) and the
    division add B + 8 roundings of the value."""
    top = np.max(np.where(np.isnan(x), -np.inf, x), axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        d = np.where(p > 0, np.abs(x - top), 0.0)
    return p * U * (3 * d + 3 * d.max(axis=1, keepdims=True) + x.shape[1] + 8) + 2.0 ** -126


def check(mm, x, host, k, active=None, real=None, **kw):
    import torch
    T, B = host.shape
    rdev = None if real is None else torch.from_numpy(np.asarray(real, np.uint8)).cuda()
    route, probs, counts, loss = mm.mlpmoe_route_topk(x, k, active, rdev, **kw)
    torch.cuda.synchronize()
    o_route, o_p, o_counts, o_loss = orc.route_topk(host, k, active, real)
    assert np.array_equal(route.cpu().numpy(), o_route)
    assert np.array_equal(counts.cpu().numpy(), o_counts)
    got = probs.cpu().numpy().astype(np.float64)
    on = np.ones(B, bool) if active is None else np.asarray(active) != 0
    seen = np.where(on[None, :], host, -np.inf)
    bound = prob_bound(seen, o_p)
    assert np.all(np.abs(got - o_p) <= bound), float(np.max((np.abs(got - o_p) / (bound + 1e-300))))
    assert not got[o_p == 0].any()
    # the loss: the probabilities' errors, at most one rounding for each of the additions a block makes in float, one at the end
    rel = U * (np.max(np.where(o_p > 0, bound / (U * np.maximum(o_p, 1e-300)), 0), initial=0.0) + T / 256 + 1024)
    assert abs(float(loss[0]) - o_loss) <= rel * o_loss, (float(loss[0]), o_loss)
    return route, probs, counts, loss


@pytest.mark.parametrize("elem", [2, 4])
@pytest.mark.parametrize("B", [1, 2, 3, 4, 7, 8, 13, 16, 17, 31, 32, 36, 61, 64])
def test_sizes(mm, B, elem):
    import torch
    dtype = torch.bfloat16 if elem == 2 else torch.float32
    for T in (1, 2, 33, 700):
        for k in sorted({1, min(2, B), (B + 1) // 2, B}):
            print("B=%d T=%d k=%d elem=%d" % (B, T, k, elem), flush=True)
            x, host = logits_of(100 * B + T + k, T, B, dtype)
            check(mm, x, host, k)


@pytest.mark.parametrize("elem", [2, 4])
@pytest.mark.parametrize("T,B,k", [(5, 16, 4), (300, 12, 5), (9000, 64, 8), (40000, 8, 2), (20011, 5, 3)])
def test_masks_bars_and_padding(mm, T, B, k, elem):
    """Branches off with not-a-number and infinities in their places, barred branches, padding, rows with nothing left."""
    import torch
    dtype = torch.bfloat16 if elem == 2 else torch.float32
    x, host = logits_of(T + B, T, B, dtype, banned=0.3)
    rng = np.random.default_rng(T)
    active = np.ones(B, np.uint8)
    active[rng.choice(B, size=B // 3, replace=False)] = 0
    junk = torch.tensor([float("nan"), float("inf"), -float("inf")])[torch.randint(3, (T, B))].to(dtype)
    x[:, torch.from_numpy(active == 0).cuda()] = junk[:, torch.from_numpy(active == 0)].cuda()
    real = (rng.uniform(size=T) < 0.8).astype(np.uint8) * rng.integers(1, 256, size=T).astype(np.uint8)
    x[T // 2] = -float("inf")                                  # a row whose mask leaves nothing
    host = x.double().cpu().numpy()
    check(mm, x, host, k, active, real)


def test_ties_and_lowest_values(mm):
    """Equal logits go to the lowest index; a mask of the type's lowest value is a value like another."""
    import torch
    for dtype in (torch.bfloat16, torch.float32):
        low = torch.finfo(dtype).min
        for B in (4, 10, 40, 64):
            x = torch.randint(0, 3, (257, B), generator=torch.Generator().manual_seed(B)).to(dtype)
            x[5] = low
            x[6] = low
            x[6, B - 1] = 0
            x[7] = torch.finfo(dtype).max
            x[8] = -0.0
            x[8, B // 2] = 0.0                                 # zeros of both signs are equal
            for k in (1, 3, B - 1, B):
                check(mm, x.cuda(), x.double().numpy(), k)


def test_nothing_at_all(mm):
    """No token, none that counts, no branch that is on: zeros."""
    import torch
    for T, B in ((0, 8), (0, 5), (4, 8), (3000, 7)):
        x = torch.randn((T, B), device="cuda")
        for kw in (dict(token_mask=torch.zeros(T, dtype=torch.uint8, device="cuda")), dict(active_mask=np.zeros(B, np.uint8))):
            route, probs, counts, loss = mm.mlpmoe_route_topk(x, 2, **kw)
            assert not route.any() and not probs.any() and not counts.any() and float(loss) == 0.0
            d = mm.mlpmoe_route_backward(probs, counts, torch.full_like(probs, float("nan")), loss, kw.get("active_mask"))
            assert d.shape == (T, B) and not d.any()


def test_not_a_number_stays_in_its_row(mm):
    import torch
    x = torch.randn((40, 16), device="cuda")
    clean = mm.mlpmoe_route_topk(x, 4)
    x[3, 5] = float("nan")
    x[9, 2] = float("inf")
    route, probs, counts, loss = mm.mlpmoe_route_topk(x, 4)
    rows = torch.arange(40, device="cuda")
    others = (rows != 3) & (rows != 9)
    assert torch.equal(route[others], clean[0][others]) and torch.equal(probs[others], clean[1][others])
    assert torch.isnan(probs[3]).all() and torch.isnan(probs[9]).all() and torch.isnan(loss).all()
    assert route[3, 5] == 0 and int(route[3].sum()) == 4 and route[9, 2] == 1


def test_strides_and_alignment(mm):
    """Logits as columns of a wider matrix, at every alignment; outputs of the caller's at odd addresses."""
    import torch
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.randn((130, 41), device="cuda").to(dtype)
        for B, c in ((16, 0), (16, 1), (16, 3), (24, 16), (7, 33)):
            x = wide[:, c:c + B]
            check(mm, x, x.double().cpu().numpy(), min(3, B))
        buf = torch.full((130 * 16 + 3,), 7, dtype=torch.uint8, device="cuda")
        x = wide[:, 4:20]
        route = buf[1:1 + 130 * 16].view(130, 16)
        check(mm, x, x.double().cpu().numpy(), 2, route=route)
        assert buf[0] == 7 and (buf[-2:] == 7).all()


def test_far_rows(mm):
    """Row offsets past 32 bits: rows 2^21 elements apart, the last of them 4 GiB and more from the first."""
    import torch
    ld, T, B = 1 << 21, 1100, 8
    big = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda").view(T, ld)
    x, host = logits_of(5, T, B, torch.bfloat16)
    big[:, :B] = x
    check(mm, big[:, :B], host, 3)


@pytest.mark.parametrize("T,B,k", [(1024, 8, 2), (1025, 8, 3), (100003, 64, 6), (600001, 3, 1)])
def test_many_tokens_a_lane(mm, T, B, k):
    """A lane with more than one token, with sums and without, the last of them missing here and there; most tokens padding."""
    import torch
    x, host = logits_of(T, T, B, torch.float32, banned=0.1)
    real = (np.random.default_rng(T).uniform(size=T) < 0.4).astype(np.uint8)
    route, probs, *_ = check(mm, x, host, k, None, real)
    r, p, *_ = mm.mlpmoe_route_topk(x, k, None, torch.from_numpy(real).cuda(), want_stats=False)
    assert torch.equal(r, route) and torch.equal(p, probs)


def test_most_tokens(mm):
    """2^24 tokens, every count exact and the loss within its bound (the sums of a lane's and a block's tokens in float)."""
    import torch
    T, B = 1 << 24, 4
    x = torch.randn((T, B), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(torch.bfloat16)
    route, probs, counts, loss = mm.mlpmoe_route_topk(x, 1)
    best = x.float().amax(dim=1, keepdim=True)
    want = x.float() == best
    for b in range(1, B):
        want[:, b] &= ~want[:, :b].any(dim=1)                     # the lowest of equal ones
    want = want.to(torch.uint8)
    assert torch.equal(route, want)
    assert torch.equal(counts[:B], want.sum(dim=0, dtype=torch.int32)) and int(counts[B]) == T
    p = torch.softmax(x.double(), dim=1)
    assert float((probs.double() - p).abs().max()) <= U * (3 * 2 * 12 + B + 8)
    exact = float(B * (want.double().mean(dim=0) * p.mean(dim=0)).sum())
    rel = U * (3 * 2 * 12 + B + 8 + T / 256 / 1024 + 1024)         # additions of a lane, then of its block
    assert abs(float(loss) - exact) <= rel * exact


def test_forms_agree_and_repeat(mm):
    """Without sums, without probabilities, with a workspace of the caller's: the same route; every run the same bits."""
    import torch
    for T, B in ((3, 16), (5000, 64), (4999, 9)):
        x, _ = logits_of(T, T, B, torch.bfloat16)
        a = mm.mlpmoe_route_topk(x, 3)
        route, probs, counts, loss = mm.mlpmoe_route_topk(x, 3, want_probs=False, want_stats=False)
        assert torch.equal(route, a[0]) and probs is None and counts is None and loss is None
        ws = torch.full((mm.mlpmoe_route_workspace_bytes(T, B),), 255, dtype=torch.uint8, device="cuda")
        for _ in range(3):
            b = mm.mlpmoe_route_topk(x, 3, workspace=ws)
            assert all(torch.equal(u, v) for u, v in zip(a, b))
        c = mm.mlpmoe_route_topk(x, 3, want_probs=False)
        assert c[1] is None and torch.equal(c[2], a[2]) and torch.equal(c[3], a[3])


def back_bound(p, dp, w, dtype):
    """Roundings of g (one, and w's own), of the products and the sum of B of them, of g - s and its product with p, then the
    result's storage."""
    import torch
    g = np.abs(dp) + np.abs(w)
    s = (np.abs(p) * g).sum(axis=1, keepdims=True)
    half = torch.finfo(dtype).eps / 2
    return p * U * (4 * g + (p.shape[1] + 5) * s), half


@pytest.mark.parametrize("elem", [2, 4])
@pytest.mark.parametrize("T,B", [(1, 1), (1, 16), (77, 3), (1000, 8), (333, 20), (2049, 64), (70000, 12)])
def test_gradient(mm, T, B, elem):
    import torch
    dtype = torch.bfloat16 if elem == 2 else torch.float32
    x, host = logits_of(T, T, B, dtype, banned=0.1 if B > 3 else 0.0)
    active = np.ones(B, np.uint8)
    if B > 4:
        active[1] = 0
    real = torch.ones(T, dtype=torch.uint8, device="cuda")
    real[T // 2:T // 2 + T // 5] = 0
    _, probs, counts, _ = mm.mlpmoe_route_topk(x, min(2, B), active, real)
    p, c = probs.double().cpu().numpy(), counts.cpu().numpy()
    dp = torch.randn((T, B), device="cuda")
    dp[probs == 0] = float("nan")                    # what stands behind a probability of zero is not looked at
    dl = torch.tensor([0.37], device="cuda")
    A = int(active.sum())
    for dprobs, dloss in ((dp, dl), (dp, None), (None, dl), (None, None)):
        d = mm.mlpmoe_route_backward(probs, counts, dprobs, dloss, active, dtype=dtype)
        h = np.zeros((T, B)) if dprobs is None else np.where(p == 0, 0.0, dp.double().cpu().numpy())
        lam = 0.0 if dloss is None else float(dl)
        want = orc.route_backward(p, c, h, lam, A)
        w = np.zeros(B) if c[:B].sum() == 0 else lam * A * c[:B] / c[:B].sum() / c[B]
        bound, half = back_bound(p, h, w, dtype)
        err = np.abs(d.double().cpu().numpy() - want)
        assert d.dtype == dtype and np.all(err <= bound * (1 + half) + half * np.abs(want) + 2.0 ** -126)
        assert not d[probs == 0].any()


def test_gradient_in_a_training_step(mm):
    """Forward and backward together against torch's gradients in float64 of the loss written out."""
    import torch
    T, B, k = 600, 16, 4
    x, host = logits_of(9, T, B, torch.float32)
    real = torch.ones(T, dtype=torch.uint8, device="cuda")
    real[500:] = 0
    route, probs, counts, loss = mm.mlpmoe_route_topk(x, k, None, real)
    mix = torch.randn((T, B), device="cuda")
    d = mm.mlpmoe_route_backward(probs, counts, mix, torch.tensor([0.5], device="cuda"))
    y = torch.from_numpy(host).requires_grad_()
    p = torch.softmax(y, 1) * real.cpu().double()[:, None]
    f = route.cpu().double().sum(0) / route.cpu().sum()
    total = (mix.cpu().double() * p).sum() + 0.5 * B * (f * p.sum(0)).sum() / 500
    total.backward()
    # probabilities are off by prob_bound, everything here is of order one: a hundred roundings
    assert np.max(np.abs(d.cpu().double().numpy() - y.grad.numpy())) < 200 * U * float(mix.abs().max())


def test_graph_and_streams(mm):
    """Recorded into a graph and replayed with other logits; two recorded calls that share a workspace; a call on another stream."""
    import torch
    T, B, k = 5000, 16, 4
    x, _ = logits_of(1, T, B, torch.bfloat16)
    x2, _ = logits_of(2, T, B, torch.bfloat16)
    ws = torch.empty(mm.mlpmoe_route_workspace_bytes(T, B), dtype=torch.uint8, device="cuda")
    dl = torch.ones(1, device="cuda")

    def step(v):
        r = mm.mlpmoe_route_topk(v, k, workspace=ws)
        return list(r) + [mm.mlpmoe_route_backward(r[1], r[2], None, dl)]

    eager = [[t.clone() for t in step(v)] for v in (x, x2)]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    buf, graph = x.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            first = step(buf)
            second = step(x2)
    torch.cuda.synchronize()
    for rep in range(4):
        buf.copy_((x, x2)[rep % 2])
        ws.fill_(255)
        for t in first + second:
            t.fill_(77)
        graph.replay()
        step(x2)                                       # the program's own work between the replays
        torch.cuda.synchronize()
        for got, want in ((first, eager[rep % 2]), (second, eager[1])):
            assert all(torch.equal(u, v) for u, v in zip(got, want)), rep
    with torch.cuda.stream(stream):
        got = step(x)
    stream.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(got, eager[0]))
    got = mm.mlpmoe_route_topk(x, k, stream=stream)
    stream.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(got, eager[0][:4]))
