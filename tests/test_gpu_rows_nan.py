"""Signalling NaN, of both signs, in rows of scores: masked as any other NaN, and in a distillation NaN."""

import numpy as np
import pytest
import torch

from test_gpu_rows import check_sample, check_top, kge, normal, rows_of, teacher_lists  # noqa: F401

pytestmark = pytest.mark.gpu
BITS = {torch.float32: (torch.int32, [0x7F800001, -0x7FFFFF, -0x3FFFFF, 0x7FC00000]), torch.bfloat16: (torch.int16, [0x7F81, -0x7F, -0x3F, 0x7FC0]),
        torch.float16: (torch.int16, [0x7C01, -0x3FF, -0x1FF, 0x7E00])}


@pytest.mark.parametrize("dtype", list(BITS))
@pytest.mark.parametrize("n", [50, 900, 6000, 15_000, 40_000])
def test_signalling_nan(kge, n, dtype):
    x = rows_of(normal(4, n, n, dtype=dtype), dtype)
    kind, bits = BITS[dtype]
    for i, b in enumerate(bits):
        x.view(kind)[:, i::7] = b
    assert int(torch.isnan(x).sum()) >= 4 * 4 * (n // 7)
    check_top(kge, x, min(n, 30))
    u = np.random.default_rng(n).random((4, 9))
    for setting in (dict(), dict(top_p=0.9), dict(min_p=0.01), dict(top_k=20, top_p=0.9)):
        check_sample(kge, x, u, **setting)
    clean = normal(4, n, n)
    ids, t, lse = teacher_lists(clean.double().numpy(), 5, n, 1.0, unused=False)
    for at, b in ((n // 2, bits[0]), (n - 1, bits[1])):
        for T in (1.0, 30.0):
            x = rows_of(clean, dtype)
            x.view(kind)[2, at] = b
            loss, grad = torch.empty(4, device="cuda"), torch.empty(4, n, dtype=dtype, device="cuda")
            kge.kge_distill_loss(x, torch.from_numpy(ids).cuda(), torch.from_numpy(t).float().cuda(), torch.from_numpy(lse).float().cuda(), T, 1.0, loss, grad)
            assert torch.isnan(loss).tolist() == [False, False, True, False]
            assert torch.isnan(grad[2]).all() and torch.isfinite(grad[[0, 1, 3]]).all()
