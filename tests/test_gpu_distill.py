"""kge_distill_loss where 32-bit weights do not do: masses that lie far below the row's best score, and large temperatures."""
import math

import numpy as np
import pytest
import torch

from test_gpu_rows import HALF_STEP, Q_ERR, TINY, U32, W_ERR, kge, normal, rows_of, teacher_lists  # noqa: F401

pytestmark = pytest.mark.gpu
L = np.longdouble  # 64 bits of fraction, exponents to 2^16384


def exact(row, ids, t, lse, T):
    """Loss and gradient of one row by the definition; the sum of what the gradient is a difference of; and sum |p - q|, what an error of a logarithm
    is multiplied with.  Entries are distinct."""
    used = (ids >= 0) & (ids < row.size) & (t != -np.inf)
    ids, t, x, T = ids[used], t[used].astype(L), row.astype(L), L(T)
    zero = np.zeros(row.size, L)
    there = row > -np.inf
    if not there.any() or (lse is None and not ids.size):
        return L(0), zero, zero, L(0)
    listed = np.zeros(row.size, bool)
    listed[ids] = True

    def shares(mask):  # exponentials relative to the best among them, and the logarithm of their sum
        if not (mask & there).any():
            return zero, L(-np.inf)
        best = x[mask & there].max()
        w = np.where(mask & there, np.exp(np.where(there, x - best, L(0)) / T), L(0))
        return w / w.sum(), best / T + np.log(w.sum())

    rest_share, rest_log = shares(~listed)
    q, log_z = shares(np.ones(row.size, bool))
    if lse is None:
        p = np.exp((t - t.max()) / T)
        log_p = (t - t.max()) / T - np.log(p.sum())
        p, rest = p / p.sum(), L(0)
    else:
        log_p = t / T - L(lse)
        p = np.exp(log_p)
        rest = max(L(0), 1 - p.sum()) if rest_log > -np.inf else L(0)
    with np.errstate(invalid="ignore"):
        loss = np.where(p > 0, p * (log_p - (x[ids] / T - log_z)), L(0)).sum()
    if rest > 0:
        loss += rest * (np.log(rest) - (rest_log - log_z))
    target = rest * rest_share
    target[ids] += p
    mass = p.sum() + rest
    q_rest = np.exp(rest_log - log_z)
    moved = np.abs(p - q[ids]).sum() + abs(rest - q_rest)
    return T * T * loss, T * (mass * q - target), T * (mass * q + target), moved


def check(kge, x, ids, t, lse, T, wide, c=1.0, in_place=False, grad=True, loss=True, **more):
    rows, n = x.shape
    dtype = x.dtype
    x64 = x.double().cpu().numpy()
    d_ids, d_t = torch.as_tensor(ids).cuda(), torch.as_tensor(t, dtype=torch.float32).cuda()
    d_lse = None if lse is None else torch.as_tensor(lse, dtype=torch.float32).cuda()
    got = torch.full((rows,), 77.0, device="cuda")
    out = x if in_place else rows_of(torch.full((rows, n), 77.0), dtype, pad=3) if grad else None
    kge.kge_distill_loss(x, d_ids, d_t, d_lse, T, c, got if loss else None, out, **more)
    got = got.double().cpu().numpy()
    g_out = out.double().cpu().numpy() if grad else None
    ids, t, T = d_ids.cpu().numpy(), d_t.double().cpu().numpy(), float(np.float32(T))
    lse = None if lse is None else d_lse.double().cpu().numpy()
    for i in range(rows):
        want, g, scale, moved = exact(x64[i], ids[i], t[i], None if lse is None else lse[i], T)
        finite = np.isfinite(x64[i])
        size = 1.0 + math.log(n) + (np.abs(x64[i][finite]).max() if finite.any() else 0.0) / T + np.abs(t[i][np.isfinite(t[i])]).max() / T \
            + (0.0 if lse is None else abs(lse[i]))
        if wide:  # weights off by 4e-14; a few roundings of logarithms of that size, 2^-53 of it each
            off = 5e-14 + 2.0 ** -49 * size
            loss_off, grad_off = T * T * float(moved) * off, off * scale.astype(float) + 6 * U32 * np.abs(g.astype(float))
            loss_off += T * T * size * 2.0 ** -60  # (the roundings of `exact`)
        else:
            loss_off, grad_off = T * T * 3 * 2 * W_ERR, (Q_ERR + 4 * U32) * scale.astype(float)
        want, g = float(want), g.astype(float)
        if loss:
            if np.isfinite(want):
                assert abs(got[i] - want) <= 1.01 * U32 * abs(want) + loss_off + 2.0 ** -149, (i, got[i], want, abs(got[i] - want), loss_off)
            else:
                assert got[i] == want
        if grad:
            limit = abs(c) * grad_off + 1.01 * HALF_STEP[dtype] * np.abs(c * g) + TINY[dtype]
            worst = np.abs(g_out[i] - c * g) / limit
            assert np.isfinite(g_out[i]).all() and worst.max() <= 1.0, (i, worst.max(), np.argmax(worst), g_out[i][np.argmax(worst)], c * g[np.argmax(worst)])


# ---- a rest far below the listed candidates

@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("T", [0.1, 1.0, 3.0])
@pytest.mark.parametrize("n,m", [(40, 3), (256, 16), (900, 20), (3000, 64), (8000, 100), (15_000, 64), (30_000, 300), (40_000, 100), (300_000, 40)])
def test_a_rest_far_below_the_list(kge, n, m, T, in_place):
    """All that is not listed lies some T below the list: less than the smallest 32-bit number, then less than the smallest 64-bit one; some of it is
    masked, and so are listed candidates."""
    gaps = np.array([20.0, 44.0, 60.0, 80.0, 88.0, 95.0, 104.0, 110.0, 300.0, 500.0, 800.0, 3000.0])
    rng = np.random.default_rng(n)
    x = rng.normal(0, 1, (gaps.size, n)) * T
    ids = np.stack([rng.permutation(n)[:m] for _ in gaps])
    x -= gaps[:, None] * T
    np.put_along_axis(x, ids, rng.normal(0, 1, ids.shape) * T, 1)
    x[::2, ::3] = -math.inf
    x[np.arange(gaps.size), ids[:, 0]] = 2.0 * T  # (a listed one that is not masked)
    listed = np.zeros(x.shape, bool)
    np.put_along_axis(listed, ids, True, 1)
    x[:, -1] = np.where(listed[:, -1], x[:, -1], -gaps * T)
    t = rng.normal(0, 1, ids.shape) * T
    for i in range(0, gaps.size, 2):  # (a masked candidate with a share would make the loss infinite)
        ids[i][x[i, ids[i]] == -math.inf] = -1
    lse = np.log(np.exp(t / T).sum(1)) + rng.uniform(0.05, 0.5, gaps.size)
    check(kge, rows_of(torch.from_numpy(x).float()), ids, t, lse, T, False, c=-0.5, in_place=in_place)
    if not in_place:
        check(kge, rows_of(torch.from_numpy(x).float(), pad=1, offset=1), ids, t, lse, T, False, grad=False)
        check(kge, rows_of(torch.from_numpy(x).float(), pad=2), ids, t, lse, T, False, loss=False)
        check(kge, rows_of(torch.from_numpy(x), torch.bfloat16), ids, t, lse, T, False)


@pytest.mark.parametrize("n", [100, 5000, 20_000, 50_000])
def test_a_list_far_below_the_rest(kge, n):
    rng = np.random.default_rng(n)
    gaps = np.array([50.0, 95.0, 110.0, 400.0, 900.0])
    x = rng.normal(0, 1, (gaps.size, n))
    ids = np.stack([rng.permutation(n)[:10] for _ in gaps])
    np.put_along_axis(x, ids, rng.normal(0, 1, ids.shape) - gaps[:, None], 1)
    t = rng.normal(0, 1, ids.shape)
    for lse in (None, np.log(np.exp(t).sum(1)) + 0.3):
        check(kge, rows_of(torch.from_numpy(x).float()), ids, t, lse, 1.0, False)


@pytest.mark.parametrize("n", [8, 256, 1024])
def test_a_rest_without_candidates_beside_masked_ones(kge, n):
    """Everything that is not listed is masked: the rest has no candidate, and masked ones get no gradient."""
    rng = np.random.default_rng(n)
    x = rng.normal(0, 2, (4, n))
    ids = np.stack([rng.permutation(n)[:n // 2] for _ in range(4)])
    listed = np.zeros(x.shape, bool)
    np.put_along_axis(listed, ids, True, 1)
    x[~listed] = -math.inf
    t = rng.normal(0, 2, ids.shape)
    check(kge, rows_of(torch.from_numpy(x).float()), ids, t, np.log(np.exp(t).sum(1)) + 0.2, 1.0, False)
