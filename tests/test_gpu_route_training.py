"""Router and gradient together as in a training step, against torch's gradients in float64 of the loss written out; the balance
loss weighs as much as the probabilities' own gradient, so that a wrong factor in either shows."""
import numpy as np
import pytest

from test_gpu_route import back_bound, logits_of, prob_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mm():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2511_21089_amd import binding
    return binding


@pytest.mark.parametrize("T,N,B,k", [(600, 500, 16, 4), (5000, 4501, 64, 8), (40, 40, 5, 2)])
def test_both_terms_of_a_training_step(mm, T, N, B, k):
    import torch
    x, _ = logits_of(T, T, B, torch.float32)
    x += torch.linspace(-2, 2, B, device="cuda")            # some branches are taken far more often than others
    host = x.double().cpu().numpy()
    active = np.ones(B, np.uint8)
    active[1] = 0
    A = B - 1
    real = torch.zeros(T, dtype=torch.uint8, device="cuda")
    real[:N] = 1
    route, probs, counts, loss = mm.mlpmoe_route_topk(x, k, active, real)
    mix = torch.randn((T, B), generator=torch.Generator().manual_seed(T))
    weight = float(N)                                       # dloss A f_b / N is then A f_b, of order one as mix is
    d = mm.mlpmoe_route_backward(probs, counts, mix.cuda(), torch.tensor([weight], device="cuda"), active).double().cpu().numpy()

    r = route.cpu().double()
    f = r.sum(0) / r.sum()
    assert int(counts[B]) == N and float(f.max()) > 3 * float(f[[0, *range(2, B)]].min())

    def gradient(mix_part, loss_part):
        y = torch.from_numpy(host).requires_grad_()
        p = torch.softmax(y.masked_fill(torch.from_numpy(active == 0), -float("inf")), 1) * real.cpu().double()[:, None]
        (mix_part * (mix.double() * p).sum() + loss_part * weight * A * (f * p.sum(0)).sum() / N).backward()
        return p.detach().numpy(), y.grad.numpy()

    p, want = gradient(1, 1)
    # d = p (g - sum p g): the gradient's own roundings, and what the probabilities' errors (prob_bound) move it by, to first order
    # and a hundredth more
    h, w = mix.double().numpy(), A * f.numpy()
    g = h + w
    e = prob_bound(np.where(active != 0, host, -np.inf), p)
    bound, half = back_bound(p, h, w, torch.float32)
    bound = bound * (1 + half) + half * np.abs(want) + 2.0 ** -126
    bound += 1.01 * (e * np.abs(g - (p * g).sum(1, keepdims=True)) + p * (e * np.abs(g)).sum(1, keepdims=True))
    assert np.all(np.abs(d - want) <= bound), float(np.max(np.abs(d - want) / bound))
    # a wrong factor in either term is far outside
    for parts in ((1, 0), (1, 0.5), (1, 0.99), (0, 1), (0.99, 1)):
        assert np.mean(np.abs(gradient(*parts)[1] - want) > 4 * bound) > 0.3 * N / T * A / B, parts
