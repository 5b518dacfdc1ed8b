"""The router and its gradient on the GPU where active logits are not numbers: a token with one counts and shows it, in its
probabilities, the loss and its gradient, also where it has no number at all; padding and inactive branches hide theirs."""
import numpy as np
import pytest

from oracle import route as orc
from test_gpu_route import back_bound, prob_bound

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module")
def mm():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2511_21089_amd import binding
    return binding


def same(a, b):
    """Equal, not-a-numbers alike."""
    import torch
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def broken(T, B, dtype):
    """Rows in turn: nothing but not-a-numbers, those and barred branches, one among numbers, all barred, numbers, numbers."""
    import torch
    g = torch.Generator().manual_seed(T + B)
    x = torch.randn((T, B), generator=g)
    x[0::6] = float("nan")
    x[1::6] = torch.where(torch.rand((len(x[1::6]), B), generator=g) < 0.5, float("nan"), -INF)
    x[2::6, B // 2] = float("nan")
    x[3::6] = -INF
    return x.to(dtype)


@pytest.mark.parametrize("elem", [2, 4])
@pytest.mark.parametrize("T,B,k", [(1, 1, 1), (7, 1, 1), (1, 16, 4), (40, 16, 4), (300, 12, 12), (2100, 64, 8), (9001, 64, 3), (20011, 5, 2)])
def test_rows_without_a_number(mm, T, B, k, elem):
    import torch
    dtype = torch.bfloat16 if elem == 2 else torch.float32
    x = broken(T, B, dtype)
    active = np.ones(B, np.uint8)
    if B > 4:
        active[B // 3] = 0
    real = np.ones(T, np.uint8)
    real[T - T // 5:] = 0
    host = x.double().numpy()
    o_route, o_p, o_counts, o_loss = orc.route_topk(host, k, active, real)
    assert np.isnan(o_loss) and np.isnan(o_p[0]).any()
    print("T=%d B=%d k=%d elem=%d" % (T, B, k, elem), flush=True)
    xd, rd = x.cuda(), torch.from_numpy(real).cuda()
    route, probs, counts, loss = mm.mlpmoe_route_topk(xd, k, active, rd)
    p = probs.double().cpu().numpy()
    assert np.array_equal(route.cpu().numpy(), o_route) and np.array_equal(counts.cpu().numpy(), o_counts)
    assert np.array_equal(np.isnan(p), np.isnan(o_p)) and torch.isnan(loss).all()
    rows = ~np.isnan(o_p).any(axis=1)
    seen = np.where(active[None, :] != 0, host, -np.inf)
    assert np.all(np.abs(p[rows] - o_p[rows]) <= prob_bound(seen[rows], o_p[rows])) and not p[o_p == 0].any()
    # without sums, without probabilities
    r, q, *_ = mm.mlpmoe_route_topk(xd, k, active, rd, want_stats=False)
    assert torch.equal(r, route) and same(q, probs)
    r, _, c, l = mm.mlpmoe_route_topk(xd, k, active, rd, want_probs=False)
    assert torch.equal(r, route) and torch.equal(c, counts) and torch.isnan(l).all()
    r = mm.mlpmoe_route_topk(xd, k, active, rd, want_probs=False, want_stats=False)[0]
    assert torch.equal(r, route)
    # the gradient
    A = int(active.sum())
    dp = torch.randn((T, B), generator=torch.Generator().manual_seed(1))
    for dprobs, lam in ((dp, 0.25), (None, 0.25), (dp, None)):
        d = mm.mlpmoe_route_backward(probs, counts, None if dprobs is None else dprobs.cuda(),
                                     None if lam is None else torch.tensor([lam], device="cuda"), active)
        h = np.zeros((T, B)) if dprobs is None else dprobs.double().numpy()
        want = orc.route_backward(p, counts.cpu().numpy(), h, lam or 0.0, A)
        got = d.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).any()
        assert not got[p == 0].any()
        c = o_counts.astype(np.float64)
        w = np.zeros(B) if lam is None or c[:B].sum() == 0 else lam * A * c[:B] / c[:B].sum() / c[B]
        bound, half = back_bound(p[rows], h[rows], w, torch.float32)
        assert np.all(np.abs(got[rows] - want[rows]) <= bound * (1 + half) + half * np.abs(want[rows]) + 2.0 ** -126)


@pytest.mark.parametrize("T,B", [(1, 4), (5, 16), (5000, 16)])
def test_no_number_at_all(mm, T, B):
    """Nothing is taken and the loss is no number either."""
    import torch
    route, probs, counts, loss = mm.mlpmoe_route_topk(torch.full((T, B), float("nan"), device="cuda"), 2)
    assert not route.any() and torch.isnan(probs).all() and torch.isnan(loss).all()
    assert counts.tolist() == [0] * B + [T]


@pytest.mark.parametrize("T", [6, 3000])
def test_padding_and_inactive_branches_hide_theirs(mm, T):
    import torch
    x = torch.randn((T, 8), generator=torch.Generator().manual_seed(T))
    real = np.arange(T) % 3 != 0
    active = np.array([1, 1, 0, 1, 0, 1, 1, 1], np.uint8)
    rd = torch.from_numpy(real).cuda()
    want = mm.mlpmoe_route_topk(x.cuda(), 2, active, rd)
    x[0::3] = float("nan")
    x[:, [2, 4]] = float("nan")
    got = mm.mlpmoe_route_topk(x.cuda(), 2, active, rd)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.isfinite(got[3]).all()
