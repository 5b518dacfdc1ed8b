"""The forward on 4-bit weights with infinities in x or in h: a token's result is the infinity that the products and sums
give, however many steps of K there are and however they are shared out.  All weights are positive, so that no product is of
zero and infinity and no sum of opposite ones."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mm():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2511_21089_amd import binding
    return binding


def positive(rows, cols, seed):
    """Weights of 1 .. 6 times 2^-8 (codes 2 .. 7)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    low, high = (torch.randint(2, 8, (rows, cols // 2), generator=g, dtype=torch.uint8, device="cuda") for _ in range(2))
    return low | high << 4, torch.full((rows, cols // 32), 119, dtype=torch.uint8, device="cuda")


def layer(T, d_model, d_inter):
    import torch
    x = (torch.rand((T, d_model), generator=torch.Generator(device="cuda").manual_seed(T), device="cuda") + 0.5).to(torch.bfloat16)
    return x, [positive(d_inter, d_model, 1), positive(d_inter, d_model, 2), positive(d_model, d_inter, 3)]


def calls(mm, x, W, d_inter):
    """Plain, with a branch off, and routed to everything and to a part."""
    import torch
    T = x.shape[0]
    off, al = np.array([0, d_inter // 2, d_inter // 2 + 40, d_inter], np.int32), np.ones(3, np.float32)
    for dtype in (torch.float32, torch.bfloat16):
        yield mm.mlpmoe_forward_w4(x, *W, off, al, np.ones(3, np.uint8), out_dtype=dtype)
        yield mm.mlpmoe_forward_w4(x, *W, off, al, np.array([1, 0, 1], np.uint8), out_dtype=dtype)
        for first in (0, 2):
            route = torch.ones((T, 3), dtype=torch.uint8, device="cuda")
            route[:, :first] = 0
            yield mm.mlpmoe_forward_w4(x, *W, off, al, np.ones(3, np.uint8), route=route, out_dtype=dtype)


TOKENS = [1, 16, 17, 32, 33, 48, 49, 64, 65, 200]


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("d_model", [96, 128, 384, 416, 512])
def test_an_infinity_at_the_end_of_x(mm, T, d_model):
    import torch
    x, W = layer(T, d_model, 256)
    x[T // 2, -1] = float("inf")
    others = torch.arange(T, device="cuda") != T // 2
    for i, out in enumerate(calls(mm, x, W, 256)):
        assert torch.isposinf(out[T // 2]).all(), i
        assert torch.isfinite(out[others]).all() and (out[others] > 0).all(), i


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("d_inter", [128, 384, 416, 1152, 1280, 2176])
def test_an_infinity_at_the_end_of_h(mm, T, d_inter):
    """The last neuron's gate and up sums are near 2^83 each, their product past the largest float."""
    import torch
    x, W = layer(T, 128, d_inter)
    for _, scales in W[:2]:
        scales[-1] = 200
    for i, out in enumerate(calls(mm, x, W, d_inter)):
        assert torch.isposinf(out).all(), i
