"""Draws by kge_sample_scores where a search or a rounding can miss."""
import math

import numpy as np
import pytest
import torch

from test_gpu_rows import U32, kge  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- long rows: every group of 4096 scores is reached

def equal_scores(kge, n, buffer, places, want_of, **setting):
    """A row of n equal scores: K of them kept, the first ones, with weights that are exactly 1, so that (j + 1/2) / K falls on j."""
    keep = want_of(n)
    at = np.unique(places[places < keep])
    u = torch.from_numpy((at + 0.5) / keep).cuda()[None]
    ids, logp = torch.full((1, at.size), -7, dtype=torch.int64, device="cuda"), torch.empty(1, at.size, device="cuda")
    kge.kge_sample_scores(buffer[:, :n], u, setting.get("T", 1.0), 0, setting.get("top_p", 1.0), setting.get("min_p", 0.0), ids, logp)
    got = ids[0].cpu().numpy()
    assert np.array_equal(got, at), (n, setting, np.flatnonzero(got != at)[:8], got[got != at][:8], at[got != at][:8])
    assert (np.abs(logp[0].cpu().numpy() + math.log(keep)) <= 1.01 * U32 * math.log(keep) + 1e-12).all()


def ends(n):
    first = np.arange(0, n, 4096)
    return np.concatenate([first, first + 4095, [n - 1]])


KEPT = [(dict(), lambda n: n), (dict(min_p=0.5), lambda n: n), (dict(top_p=0.875), lambda n: math.ceil(0.875 * n))]


@pytest.mark.parametrize("setting,want_of", KEPT, ids=["all", "min_p", "top_p"])
@pytest.mark.parametrize("groups", [9, 63, 64, 65, 66, 127, 128, 129, 130, 192, 193, 194, 1025, 4097, 4098, 4100, 4161, 8257])
def test_first_and_last_candidate_of_every_group(kge, groups, setting, want_of):
    buffer = torch.zeros(1, groups * 4096, dtype=torch.float16, device="cuda")
    for n in (groups * 4096, (groups - 1) * 4096 + 1):
        equal_scores(kge, n, buffer, ends(n), want_of, **setting)


def test_last_group_at_every_number_of_groups(kge):
    most = 330
    buffer = torch.zeros(1, most * 4096, dtype=torch.bfloat16, device="cuda")
    for groups in range(9, most + 1):
        n = groups * 4096 - groups % 3
        equal_scores(kge, n, buffer, np.array([0, n // 2, n - 4096, n - 1]), lambda k: k)
