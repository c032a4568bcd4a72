"""The torch conveniences of quantised inference compute no gradients: tensors that ask for one are refused (CPU only)."""
import pytest
import torch

from paper_2609_24519_amd import awe


def calls():
    """(what asks for a gradient, the call) for every floating-point argument."""
    x, w, s = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(5, 2)
    x8, sx = torch.zeros(3, 64, dtype=torch.int8), torch.zeros(3)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    cache = awe.Cache(torch.zeros(4, 2, 16, 64, dtype=torch.int8), torch.zeros(4, 2, 64, 16, dtype=torch.int8),
                      torch.zeros(4, 2), torch.zeros(4, 2))
    batch = awe.Batch(i32(3), i32(2), i32(2, 4), 5, 3, 64)
    rows = lambda: torch.zeros(5, 2, 64, dtype=torch.bfloat16)  # noqa: E731
    a, b = rows(), rows()
    return [(x, lambda: awe.matmul_w4(x, w, s, 32)), (s, lambda: awe.matmul_w4(x, w, s, 32)),
            (sx, lambda: awe.matmul_w4(x8, w, s, 32, x_scales=sx)), (a, lambda: awe.store_tokens(cache, batch, a, b)),
            (b, lambda: awe.store_tokens(cache, batch, a, b)), (a, lambda: awe.attend(cache, batch, a, 1.0)),
            (b, lambda: awe.attend(cache, batch, a, 1.0, out=b))]


@pytest.mark.parametrize("i", range(7))
def test_a_gradient_is_refused(i):
    wants, call = calls()[i]
    wants.requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        call()
    # without gradients, or without one asked for, the call goes on (to the refusal of tensors of the host)
    with torch.no_grad(), pytest.raises(ValueError, match="device"):
        call()
    with torch.inference_mode(), pytest.raises(ValueError, match="device"):
        call()
    wants.requires_grad_(False)
    with pytest.raises(ValueError, match="device"):
        call()


def test_scales_of_a_cache_with_a_gradient_are_refused():
    k, v = torch.zeros(4, 2, 16, 64, dtype=torch.int8), torch.zeros(4, 2, 64, 16, dtype=torch.int8)
    for i in (0, 1):
        scales = [torch.zeros(4, 2) for _ in range(2)]
        scales[i].requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            awe.Cache(k, v, *scales)
