"""Sizes and strides of the router's tensors that do not fit the library's 32-bit arguments are refused, never cut short."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mm():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2511_21089_amd import binding
    return binding


def refused(mm, f, *args, **kw):
    with pytest.raises(mm.MlpMoeError) as e:
        f(*args, **kw)
    assert e.value.status == mm.ERR_SHAPE


def test_rows_further_apart_than_32_bits(mm):
    import torch
    ld = (1 << 32) + 8                                     # 8 in its lower 32 bits
    x = torch.empty(ld + 8, dtype=torch.bfloat16, device="cuda").as_strided((2, 8), (ld, 1))
    x[0] = torch.arange(8)
    x[1] = -torch.arange(8)
    refused(mm, mm.mlpmoe_route_topk, x, 2)
    one = mm.mlpmoe_route_topk(x[1:], 2)                   # a single row has no stride
    assert one[0].tolist() == [[1, 1, 0, 0, 0, 0, 0, 0]]


def test_choices_and_tokens_past_32_bits(mm):
    import torch
    refused(mm, mm.mlpmoe_route_topk, torch.zeros((4, 8), device="cuda"), (1 << 32) + 2)
    many = torch.empty(((1 << 32) + 1, 1), dtype=torch.bfloat16, device="cuda")
    refused(mm, mm.mlpmoe_route_topk, many, 1, want_probs=False, want_stats=False)
    del many
    p = torch.empty(((1 << 32) + 1, 1), device="cuda")
    refused(mm, mm.mlpmoe_route_backward, p, None, dtype=torch.bfloat16)
