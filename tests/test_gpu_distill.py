"""kge_distill_loss where 32-bit weights do not do: masses that lie far below the row's best score, and large temperatures."""
import math

import numpy as np
import pytest
import torch

from test_gpu_rows import HALF_STEP, Q_ERR, TINY, U32, W_ERR, kge, normal, rows_of, teacher_lists  # noqa: F401

pytestmark = pytest.mark.gpu
L = np.longdouble  # 64 bits of fraction, exponents to 2^16384


def exact(row, ids, t, lse, T):
    """Loss and gradient of one row by the definition; the sum of what the gradient is a difference of; sum |p - q|, what an error of a logarithm
    is multiplied with; and what one of the sum of p is multiplied with.  Entries are distinct."""
    used = (ids >= 0) & (ids < row.size) & (t != -np.inf)
    ids, t, x, T = ids[used], t[used].astype(L), row.astype(L), L(T)
    zero = np.zeros(row.size, L)
    there = row > -np.inf
    if not there.any() or (lse is None and not ids.size):
        return L(0), zero, zero, L(0), 0.0
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
    of_sum = 0.0 if lse is None else abs(float(np.log(rest) - (rest_log - log_z))) if rest > 0 else 1.0
    return T * T * loss, T * (mass * q - target), T * (mass * q + target), moved, of_sum


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
        want, g, scale, moved, of_sum = exact(x64[i], ids[i], t[i], None if lse is None else lse[i], T)
        finite = np.isfinite(x64[i])
        size = 1.0 + math.log(n) + (np.abs(x64[i][finite]).max() if finite.any() else 0.0) / T + np.abs(t[i][np.isfinite(t[i])]).max() / T \
            + (0.0 if lse is None else abs(lse[i]))
        if wide:  # weights off by 4e-14; a few roundings of logarithms of that size, 2^-53 of it each
            off = 5e-14 + 2.0 ** -49 * size
            loss_off, grad_off = T * T * float(moved) * off, off * scale.astype(float) + 6 * U32 * np.abs(g.astype(float))
            loss_off += T * T * size * 2.0 ** -60  # (the roundings of `exact`)
            # With a log-sum-exp the rest is 1 - sum p, or, where there is no rest, the loss contains sum p - 1: its derivative by sum p is `of_sum`.  The sum is near
            # 1, so each of its last additions rounds by up to 2^-54 or 2^-53 and the exponentials' errors of 2^-53 of themselves add up to another 2^-53: 2^-51.
            loss_off += T * T * of_sum * 2.0 ** -51
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


# ---- large temperatures

LARGE_T = [4.5, 20.0, 100.0, 1e3, 1e4, 1e5]


@pytest.mark.parametrize("T", LARGE_T)
@pytest.mark.parametrize("rows,n,m,rest", [(3, 256, 256, False), (3, 256, 255, False), (3, 256, 256, True), (2, 1, 1, False), (2, 300, 20, True), (2, 1024, 1024, False), (3, 900, 900, True),
                                           (2, 4096, 30, True), (2, 6000, 64, False), (2, 14_952, 64, True), (2, 30_000, 500, True), (2, 32_769, 64, True),
                                           (2, 50_000, 300, False), (1, 200_000, 1024, True)])
def test_large_temperatures(kge, rows, n, m, rest, T):
    """What is allowed grows with T times the roundings of 64 bits, and not with T^2 times those of 32."""
    x = normal(rows, n, n + m)
    ids, t, _ = teacher_lists(x.double().numpy(), m, n, T, unused=False)
    lse = None
    if rest:  # the teacher's own log-sum-exp over all candidates, in fp32
        g = np.random.default_rng(n + 1)
        every = x.double().numpy() + g.normal(0, 0.5, x.shape)
        np.put_along_axis(every, ids, t, 1)
        lse = (np.log(np.exp((every.astype(L) - every.max()) / L(T)).sum(1)) + every.max() / T).astype(float)
    check(kge, rows_of(x, pad=n % 3), ids, t, lse, T, True, c=1.0 / rows)
    check(kge, rows_of(x, torch.float16, offset=1), ids, t, lse, T, True, c=-1.0)
    check(kge, rows_of(x), ids, t, lse, T, True, grad=False)
    check(kge, rows_of(x), ids, t, lse, T, True, in_place=True)


@pytest.mark.parametrize("n,m", [(60, 20), (1000, 100), (20_000, 300), (50_000, 64)])
@pytest.mark.parametrize("T", [6.0, 300.0])
def test_large_temperatures_with_masks_and_gaps(kge, n, m, T):
    rng = np.random.default_rng(n)
    x = rng.normal(0, 3, (7, n))
    ids = np.stack([rng.permutation(n)[:m] for _ in range(7)])
    t = rng.normal(0, 3, ids.shape)
    keep = np.take_along_axis(x, ids, 1)
    x[0, ::3] = -math.inf
    x[1] -= 100.0 * T                            # the rest lies far below the list
    x[2] -= 1000.0 * T
    x[3] += 95.0 * T                             # and far above it
    np.put_along_axis(x, ids, keep, 1)
    x[4] = -math.inf
    ids[5] = -1
    t[6, ::2] = -np.inf
    lse = np.log(np.exp(np.where(np.isfinite(t), t, -1e9) / T).sum(1)) + 0.4
    for at in (None, lse):
        check(kge, rows_of(torch.from_numpy(x).float()), ids, t, at, T, True)
        check(kge, rows_of(torch.from_numpy(x).float()), ids, t, at, T, True, in_place=True)


@pytest.mark.parametrize("n", [5, 700, 50_000])
def test_equal_rows_at_the_largest_temperatures(kge, n):
    """T^2 is larger than fp32 holds; a student that is like its teacher has loss 0, not 0 times infinity."""
    m = min(n, 1024)
    x = torch.full((2, n), 1.5)
    x[:, m:] = -math.inf
    ids = torch.arange(m, device="cuda").repeat(2, 1)
    loss, grad = torch.empty(2, device="cuda"), torch.empty(2, n, device="cuda")
    for T in (1e15, 3e19, 1e30, 3.4e38):
        kge.kge_distill_loss(rows_of(x), ids, torch.full((2, m), 0.25, device="cuda"), None, T, 1.0, loss, grad)
        assert (loss == 0).all() and (grad == 0).all()


@pytest.mark.parametrize("n", [100, 20_000, 50_000])
def test_nan_at_large_temperatures(kge, n):
    x = normal(6, n, n)
    ids, t, lse = teacher_lists(x.double().numpy(), 5, n, 50.0, unused=False)
    x[1, n // 2], x[2, n - 1] = math.nan, math.inf
    x[5, int(ids[5, 2])] = math.inf  # listed
    t[3, 2] = math.nan
    loss, grad = torch.empty(6, device="cuda"), torch.empty(6, n, device="cuda")
    for T in (50.0, 1.0):
        for teacher_lse in (None, torch.from_numpy(lse).float().cuda()):
            kge.kge_distill_loss(rows_of(x), torch.from_numpy(ids).cuda(), torch.from_numpy(t).float().cuda(), teacher_lse, T, 1.0, loss, grad)
            assert torch.isnan(loss).tolist() == [False, True, True, True, False, True]
            assert torch.isfinite(grad[[0, 4]]).all() and torch.isnan(grad[[1, 2, 5]]).all()


def test_repeated_entries_at_large_temperatures(kge):
    """The same candidate twice: its masses add up, so the halves of an entry give the gradient of the whole, and the loss of two halves."""
    for n in (400, 40_000):
        x = normal(3, n, n)
        ids, t, lse = teacher_lists(x.double().numpy(), 30, n, 80.0, unused=False)
        T, half = 80.0, 80.0 * math.log(2.0)
        at = rows_of(x)

        def call(ids, t, lse):
            loss, grad = torch.empty(3, device="cuda"), torch.empty(3, n, device="cuda")
            kge.kge_distill_loss(at, torch.from_numpy(ids).cuda(), torch.from_numpy(t).float().cuda(), None if lse is None else torch.from_numpy(lse).float().cuda(),
                                 T, 1.0, loss, grad)
            return loss.double(), grad.double()

        for given in (None, lse + 0.2):
            one, two = call(ids, t, given), call(np.concatenate([ids, ids], 1), np.concatenate([t - half, t - half], 1), given)
            p = np.exp(t / T - given[:, None]).sum(1) if given is not None else np.ones(3)
            less = torch.from_numpy(T * T * p * math.log(2.0)).cuda()  # p log p of two halves
            # t - half is rounded to fp32 (2^-24 of some 60), so p by 2^-18 / T, T^2 of which is in the loss
            # and the two losses themselves, of up to 45,000, are rounded to fp32: by 2^-24 of each
            assert ((one[0] - two[0] - less).abs() <= T * 2.0 ** -17 + 1.01 * U32 * (one[0].abs() + two[0].abs())).all()
            assert (one[1] - two[1]).abs().max() <= 2.0 ** -17


# ---- listed candidates

@pytest.mark.parametrize("T", [0.5, 1.0, 4.0])
@pytest.mark.parametrize("n", [1, 5, 60, 256, 700, 1024])
def test_lists_of_all_candidates(kge, n, T):
    """Weights of listed candidates are formed in 64 bits at every temperature: where all are listed, loss and gradient are off by their rounding, and by the
    2^-53 of each of some 30 steps, the logarithms' of their size."""
    x = normal(4, n, n)
    ids, t, lse = teacher_lists(x.double().numpy(), n, n, T, unused=False)
    for given in (None, lse, lse + 0.3):
        loss, grad = torch.empty(4, device="cuda"), torch.empty(4, n, device="cuda")
        d_lse = None if given is None else torch.from_numpy(given).float().cuda()
        kge.kge_distill_loss(rows_of(x), torch.from_numpy(ids).cuda(), torch.from_numpy(t).float().cuda(), d_lse, T, 1.0, loss, grad)
        t32 = t.astype(np.float32).astype(np.float64)
        for i in range(4):
            want, g, scale, _, of_sum = exact(x[i].double().numpy(), ids[i], t32[i], None if given is None else d_lse[i].item(), T)
            size = 2.0 + math.log(n) + (np.abs(x[i].double().numpy()).max() + np.abs(t[i]).max()) / T
            assert abs(loss[i].item() - float(want)) <= 1.01 * U32 * abs(float(want)) + T * T * (30 * size + 4 * of_sum) * 2.0 ** -53
            off = 1.01 * U32 * np.abs(g.astype(float)) + 30 * size * 2.0 ** -53 * scale.astype(float) + 2.0 ** -149
            assert (np.abs(grad[i].double().cpu().numpy() - g.astype(float)) <= off).all()
