"""How many draws a call of kge_sample_scores takes, on the host: nothing is enqueued."""
import pytest

from paper_2004_08532_amd import binding as kge

lib = kge._lib
P = 4096  # an address that nothing reads


def sample(rows, draws, n, top_k=0, top_p=1.0, min_p=0.0, temperature=1.0):
    return lib.kge_sample_scores(P, kge.KGE_F16, rows, n, n, P, draws, temperature, top_k, top_p, min_p, P, None, None, 0, None)


@pytest.mark.parametrize("setting", [dict(), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=40_000)])
def test_more_draws_than_workgroups_can_be_numbered(setting):
    assert sample((1 << 13) + 1, 1 << 20, 40_000, **setting) == kge.KGE_ERR_INVALID_ARG and "2^33" in kge.kge_last_error(None)
    # the most: the next thing to be looked at is the workspace, of which there is none here
    assert sample(1 << 13, 1 << 20, 40_000, **setting) == kge.KGE_ERR_WORKSPACE


@pytest.mark.parametrize("setting", [dict(top_k=20), dict(temperature=0.0)])
def test_lists_have_a_workgroup_per_row(setting):
    assert sample((1 << 13) + 1, 1 << 20, 40_000, **setting) == kge.KGE_ERR_WORKSPACE
