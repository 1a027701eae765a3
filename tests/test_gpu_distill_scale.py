"""kge_distill_loss at the ends of what its factors can be: T^2 and grad_scale times T beyond what 32 bits hold."""
import math

import numpy as np
import pytest
import torch

from test_gpu_rows import U32, kge  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [0.1, 0.3, 1e10, 2e19, 1e20])
@pytest.mark.parametrize("n", [900, 50_000])
def test_loss_is_multiplied_in_64_bits(kge, n, T):
    """Equal scores: every weight is exactly 1 and the divergence is log(n / m)."""
    x, m = torch.full((1, n), 0.25, device="cuda"), 1000 * n // 1001 if n < 1000 else 1024
    if n > 1024:
        x[:, 1030:] = -math.inf
    there = min(n, 1030)
    ids, t, loss = torch.arange(m, device="cuda")[None], torch.zeros(1, m, device="cuda"), torch.empty(1, device="cuda")
    kge.kge_distill_loss(x, ids, t, None, T, 1.0, loss)
    want = float(np.float32(T)) ** 2 * math.log1p((there - m) / m)
    # (the logarithms of m and of `there` are off by 2^-53 of 7 each)
    assert abs(loss.item() - want) <= 1.01 * U32 * want + float(np.float32(T)) ** 2 * 2.0 ** -49


@pytest.mark.parametrize("n", [100, 9000, 60_000])
def test_a_factor_that_32_bits_do_not_hold(kge, n):
    """grad_scale times T is 1.2e39: gradients that are larger than any number are one (or infinite), those of masked candidates are 0."""
    x = torch.randn(2, n, generator=torch.Generator("cuda").manual_seed(n), device="cuda")
    x[:, 5::3] = -math.inf
    ids, t = torch.tensor([[0, 1, 3]] * 2, device="cuda"), torch.zeros(2, 3, device="cuda")
    grad = torch.empty(2, n, device="cuda")
    for lse in (None, torch.full((2,), 2.0, device="cuda")):
        kge.kge_distill_loss(x, ids, t, lse, 4.0, 3e38, None, grad)
        assert not torch.isnan(grad).any()
        assert (grad[:, 5::3] == 0).all() and (grad[:, [0, 1, 3]] < 0).all()
