"""What the calls on rows of scores refuse, on the host: nothing is enqueued, so no GPU is needed."""
import ctypes
import math

import pytest
import torch

from paper_2004_08532_amd import binding as kge

lib = kge._lib
P = 4096  # an address that nothing reads
BAD = [("dtype", 3), ("dtype", -1), ("rows", -1), ("rows", 1 << 31), ("n", 0), ("n", 1 << 32), ("ld", 99), ("scores", None), ("scores", P + 2)]


def last():
    return kge.kge_last_error(None)


def top(scores=P, dtype=0, rows=4, n=100, ld=100, m=10, temperature=1.0, ids=P, tops=P, lse=None, ws=None, size=0):
    return lib.kge_top_scores(scores, dtype, rows, n, ld, m, temperature, ids, tops, lse, ws, size, None)


def sample(scores=P, dtype=0, rows=4, n=100, ld=100, u=P, draws=2, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, ids=P, logp=None, ws=None,
           size=0):
    return lib.kge_sample_scores(scores, dtype, rows, n, ld, u, draws, temperature, top_k, top_p, min_p, ids, logp, ws, size, None)


def distill(scores=P, dtype=0, rows=4, n=100, ld=100, t_ids=P, t_scores=P, t_lse=None, m=10, temperature=1.0, grad_scale=1.0, loss=P, grad=None,
            ld_grad=100, ws=None, size=0):
    return lib.kge_distill_loss(scores, dtype, rows, n, ld, t_ids, t_scores, t_lse, m, temperature, grad_scale, loss, grad, ld_grad, ws, size, None)


@pytest.mark.parametrize("call", [top, sample, distill])
@pytest.mark.parametrize("name,value", BAD)
def test_rows(call, name, value):
    assert call(**{name: value}) == kge.KGE_ERR_INVALID_ARG and last()


@pytest.mark.parametrize("call", [top, sample, distill])
def test_no_rows_is_no_work(call):
    assert call(rows=0, scores=None) == kge.KGE_OK


@pytest.mark.parametrize("call,bad", [
    (top, dict(m=0)), (top, dict(m=1025)), (top, dict(temperature=0.0)), (top, dict(temperature=-1.0)), (top, dict(temperature=math.nan)),
    (top, dict(temperature=math.inf)), (top, dict(ids=None)), (top, dict(tops=None)),
    (sample, dict(draws=0)), (sample, dict(draws=(1 << 20) + 1)), (sample, dict(temperature=-0.5)), (sample, dict(temperature=math.nan)),
    (sample, dict(temperature=math.inf)), (sample, dict(top_k=-1)), (sample, dict(top_k=1025, n=5000, ld=5000)), (sample, dict(top_p=1.5)),
    (sample, dict(top_p=-0.1)), (sample, dict(top_p=math.nan)), (sample, dict(min_p=1.5)), (sample, dict(min_p=math.nan)), (sample, dict(u=None)),
    (sample, dict(ids=None)),
    (distill, dict(m=0)), (distill, dict(m=1025)), (distill, dict(temperature=0.0)), (distill, dict(temperature=math.inf)),
    (distill, dict(grad_scale=math.nan)), (distill, dict(grad_scale=math.inf)), (distill, dict(t_ids=None)), (distill, dict(t_scores=None)),
    (distill, dict(loss=None)), (distill, dict(grad=P, ld_grad=99)), (distill, dict(grad=P + 2)), (distill, dict(grad=P, ld=120, ld_grad=121)),
])
def test_arguments(call, bad):
    assert call(**bad) == kge.KGE_ERR_INVALID_ARG and last()


@pytest.mark.parametrize("call,size", [
    (top, lambda: lib.kge_top_scores_workspace(4, 50_000, 10)),
    (sample, lambda: lib.kge_sample_scores_workspace(4, 50_000, 2, 0, 1.0)),
    (distill, lambda: lib.kge_distill_loss_workspace(4, 50_000))])
def test_workspace_of_long_rows(call, size):
    long = dict(n=50_000, ld=50_000)
    needed = size()
    assert needed > 0
    assert call(**long) == kge.KGE_ERR_WORKSPACE and "workspace" in last()
    assert call(**long, ws=P, size=needed - 1) == kge.KGE_ERR_WORKSPACE
    assert call(**long, ws=P + 8, size=needed) == kge.KGE_ERR_INVALID_ARG and "aligned" in last()


def test_no_workspace_where_a_workgroup_holds_the_row():
    assert lib.kge_top_scores_workspace(1000, 32_768, 1024) == lib.kge_sample_scores_workspace(1000, 32_768, 64, 50, 0.9) == 0
    assert lib.kge_distill_loss_workspace(1000, 32_768) == 0


@pytest.mark.parametrize("n", [32_769, 40_943, 2_500_000, 86_054_151])
@pytest.mark.parametrize("top_k,top_p", [(0, 1.0), (0, 0.9), (1, 1.0), (1024, 0.9)])
def test_greedy_draws_fit_every_workspace(n, top_k, top_p):
    """Temperature 0 draws as top_k = 1 does, in the workspace that the caller's own settings give."""
    assert lib.kge_sample_scores_workspace(3, n, 2, top_k, top_p) >= lib.kge_sample_scores_workspace(3, n, 2, 1, 1.0)


def test_tensors_that_are_not_on_a_device():
    x, i, u = torch.zeros(2, 8), torch.zeros(2, 3, dtype=torch.int64), torch.zeros(2, 3, dtype=torch.float64)
    with pytest.raises(TypeError):
        kge.kge_top_scores(x, 3, 1.0, i, torch.zeros(2, 3))
    with pytest.raises(TypeError):
        kge.kge_sample_scores(x, u, 1.0, 0, 1.0, 0.0, i)
    with pytest.raises(TypeError):
        kge.kge_distill_loss(x, i, torch.zeros(2, 3), None, 1.0, 1.0, torch.zeros(2))


@pytest.mark.parametrize("model", ["transe_l1", "rotate", "transr"])
def test_models_that_a_teacher_cannot_train(model):
    """Their step forms the coefficients inside of its own launches; the model is looked at before anything else."""
    cfg = kge.kge_config()
    cfg.model = kge.MODEL_IDS[model]
    ctx = ctypes.create_string_buffer(1 << 16)  # stands for a context, whose first member is its configuration
    ctypes.memmove(ctx, ctypes.byref(cfg), ctypes.sizeof(cfg))
    assert lib.kge_distill_step(ctx, P, P, P, P, P, P, P, 4, P, 4, 4, 0, 1.0, 0.1, P, P, None, 2, 1.0, None, None) == kge.KGE_ERR_UNSUPPORTED
