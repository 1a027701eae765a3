"""Draws by kge_sample_scores where a search or a rounding can miss: every id has to be a candidate that is kept, with a weight of its own."""
import math

import numpy as np
import pytest
import torch

from test_gpu_rows import U32, kge, normal, order, rows_of, weights  # noqa: F401

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


# ---- tiles and entries without a weight

def check_draws(kge, x, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Each id is kept and has a weight; the number lies in the candidate's own part of the sum, to 1e-12 of the whole sum (its weights are off by 4e-14
    and sums of up to 2^17 in 64 bits by less than that); logp is that candidate's."""
    rows = x.shape[0]
    ids = torch.full(u.shape, -7, dtype=torch.int64, device="cuda")
    logp = torch.full(u.shape, 77.0, device="cuda")
    kge.kge_sample_scores(x, torch.from_numpy(u).cuda(), T, top_k, top_p, min_p, ids, logp)
    x, ids, logp = x.double().cpu().numpy(), ids.cpu().numpy(), logp.cpu().numpy()
    T, top_p, min_p = (float(np.float32(v)) for v in (T, top_p, min_p))
    for i in range(rows):
        first = order(x[i])
        w = weights(x[i], T)
        w[w < 2.0 ** -1000] = 0.0
        first = first[:top_k] if top_k else first
        if top_p < 1:
            sums = np.cumsum(w[first])
            first = first[:1 + np.searchsorted(sums[:-1], top_p * sums[-1])]
        kept = np.sort(first[w[first] >= min_p])
        kept = kept[w[kept] > 0]
        sums = np.cumsum(w[kept].astype(np.longdouble))
        want = np.clip(np.nan_to_num(u[i]), 0.0, 1.0 - 2.0 ** -53) * sums[-1]
        for d in range(u.shape[1]):
            at = np.searchsorted(kept, ids[i, d])
            assert at < kept.size and kept[at] == ids[i, d], (i, d, u[i, d], ids[i, d])
            slack = 1e-12 * sums[-1] if want[d] > 0 else 0.0
            assert sums[at] - w[kept[at]] - slack <= want[d] <= sums[at] + slack, (i, d, u[i, d], ids[i, d])
            exact = float(np.log(w[kept[at]] / sums[-1]))
            assert abs(logp[i, d] - exact) <= 1.01 * U32 * abs(exact) + 1e-12, (i, d, logp[i, d], exact)


ALL_KEPT = [dict(), dict(min_p=1e-6), dict(top_p=0.97), dict(top_p=0.9, min_p=0.001, T=2.0), dict(top_k=200), dict(top_k=900, T=0.002)]
NUMBERS = [1.0, 1.0 - 2.0 ** -53, 1.0 - 2.0 ** -52, 5.0, math.inf, 0.0, -1.0, math.nan]


@pytest.mark.parametrize("setting", range(len(ALL_KEPT)))
@pytest.mark.parametrize("n", [200, 700, 1300, 2000, 5000, 8000, 15_000, 30_000, 50_000, 90_000])
def test_numbers_at_the_ends(kge, n, setting):
    x = normal(32, n, n + setting)
    x[8:16, n - n // 3:] = -math.inf
    x[16:24, :n // 3] = -math.inf
    check_draws(kge, rows_of(x), np.tile(NUMBERS, (32, 1)), **ALL_KEPT[setting])


@pytest.mark.parametrize("setting", range(len(ALL_KEPT)))
@pytest.mark.parametrize("n", [1300, 5000, 15_000, 30_000, 70_000])
def test_numbers_at_the_borders_of_masked_tiles(kge, n, setting):
    """Numbers that are the running sums in front of stretches of masked candidates."""
    x = normal(16, n, n + setting)
    part = max(256, n // 6 // 256 * 256)
    for first in range(part, n, 2 * part):
        x[:, first:first + part] = -math.inf
    w = np.stack([weights(r, ALL_KEPT[setting].get("T", 1.0)) for r in x.double().numpy()])
    sums = np.cumsum(w, 1)
    u = sums[:, part - 1::part] / sums[:, -1:]
    check_draws(kge, rows_of(x), np.concatenate([u, np.nextafter(u, 0.0)], 1), **ALL_KEPT[setting])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1024, 2048, 5000, 14_000, 33_000, 80_000, 300_000])
def test_tiles_whose_weights_are_less_than_any(kge, n, dtype):
    """The number 0 falls on the first candidate with a weight of 2^-1000 or more, whatever lies in front of it: tiles of 256 whose weights are a
    little less, beside tiles whose weights are a little more."""
    x = np.full((6, n), -math.inf)
    x[:, n - 3] = 0.0                       # the best one
    x[0, 0:256], x[0, 256 + 9] = -695.0, -600.0    # exp(-693.15) = 2^-1000
    x[1, 0:512], x[1, 512 + 200] = -700.0, -690.0
    x[2, 3], x[2, 300], x[2, 600], x[2, 1000] = -695.0, -694.0, -698.0, -692.0
    x[3, 0:1024:5] = -696.0
    x[3, 700] = -688.0
    x[4, 0:256] = -690.0
    x[4, 256:1000] = -700.0
    x[5] = -694.0
    x[5, n // 2 - 4] = -640.0
    x[5, n - 3:] = 0.0
    check_draws(kge, rows_of(torch.from_numpy(x), dtype), np.tile([0.0, -1.0, 0.5, 1.0 - 2.0 ** -53, 1e-310], (6, 1)))
    check_draws(kge, rows_of(torch.from_numpy(x / 128), dtype), np.tile([0.0, 0.5], (6, 1)), T=1 / 128)


@pytest.mark.parametrize("n", [1500, 2000, 6000, 15_000, 30_000, 40_000, 200_000])
def test_top_p_that_ends_next_to_zero(kge, n):
    """The cut lies among scores of -2^-149, just below many zeros and above a few more: whatever the first bins are, whose borders the row's best and
    lowest score set, the zeros are counted once."""
    g = np.random.default_rng(n)
    for most, T in ((1 << 20, 1e-39), (1 << 23, 1e-38)):
        x = g.choice([0, -1, 9], (64, n), p=[0.2, 0.25, 0.55])
        x = np.where(x == 9, g.integers(-40, 31, x.shape), x).astype(np.float64)
        x[:, 7], x[:, n // 2] = most + np.arange(64) * 3, -most - g.integers(0, 64, 64)
        x[:, -1] = -1
        u = np.concatenate([np.tile([1.0 - 2.0 ** -53, 0.0], (64, 1)), g.random((64, 4))], 1)
        check_draws(kge, rows_of(torch.from_numpy(x * 2.0 ** -149).float()), u, T=T, top_p=0.6)
