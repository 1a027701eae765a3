"""Operators on rows of scores against their definitions in 64 bits: kge_top_scores, kge_sample_scores, kge_distill_loss."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24  # half a step of fp32
# A weight exp2(x) of the distillation loss: the hardware's exp2 is off by at most a step (2 U32), its argument in [-1/2, 1/2] by U32 / 2, the
# sum of four weights by 3 U32; log and products are formed in 64 bits.  So sums, and quotients of two of them:
W_ERR, Q_ERR = 6 * U32, 12 * U32
HALF_STEP = {torch.float32: U32, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}  # spacing below the normal numbers


@pytest.fixture(scope="module")
def kge():
    import paper_2004_08532_amd as k
    return k


def rows_of(x, dtype=torch.float32, pad=0, offset=0):
    """A device tensor whose rows lie n + pad apart and start `offset` values behind an aligned address; NaN between them."""
    x = torch.as_tensor(x)
    rows, n = x.shape
    buffer = torch.full((offset + rows * (n + pad) + 8,), math.nan, dtype=dtype, device="cuda")
    view = buffer[offset:offset + rows * (n + pad)].view(rows, n + pad)[:, :n]
    view.copy_(x)
    return view


def normal(rows, n, seed, spread=3.0, dtype=torch.float32):
    g = np.random.default_rng(seed)
    return torch.from_numpy(g.normal(-2.0, spread, (rows, n))).to(dtype).float()


def order(row):
    """Positions of the candidates that are not masked, best first, equal ones by position."""
    there = np.flatnonzero(row > -np.inf)
    return there[np.argsort(-row[there], kind="stable")]


def weights(row, T):
    best = row[row > -np.inf].max()
    with np.errstate(invalid="ignore"):
        return np.where(row > -np.inf, np.where(row == best, 1.0, np.exp((row - best) / T)), 0.0)


# ---- top

def check_top(kge, x, m, T=1.0, **more):
    rows, n = x.shape
    ids = torch.full((rows + 1, m), 77, dtype=torch.int64, device="cuda")
    top = torch.full((rows + 1, m), 77.0, device="cuda")
    lse = torch.full((rows + 1,), 77.0, device="cuda")
    kge.kge_top_scores(x, m, T, ids[:rows], top[:rows], lse[:rows], **more)
    assert (ids[rows] == 77).all() and (top[rows] == 77).all() and lse[rows] == 77  # what lies behind stays as it was
    ids, top, lse, x = (y.cpu().numpy() for y in (ids, top, lse, x.double()))
    T = float(np.float32(T))  # (the temperature that the call gets)
    for i in range(rows):
        want = order(x[i])[:m]
        assert np.array_equal(ids[i][:want.size], want), (i, ids[i][:8], want[:8])
        assert np.array_equal(top[i][:want.size], x[i][want].astype(np.float32))
        assert (ids[i][want.size:] == -1).all() and (top[i][want.size:] == -np.inf).all()
        if not want.size:
            assert lse[i] == -np.inf
        elif x[i][want[0]] == np.inf:
            assert lse[i] == np.inf
        else:
            exact = x[i][want[0]] / T + np.log(weights(x[i], T).sum())
            assert abs(lse[i] - exact) <= 1.01 * U32 * abs(exact) + 1e-13 + 2.0 ** -149, (i, lse[i], exact)


SIZES = [(1, 1, 1), (3, 2, 5), (1, 4, 4), (5, 63, 1), (5, 255, 10), (4, 256, 256), (3, 257, 300), (2, 1024, 1024), (4, 1025, 7), (3, 4096, 64),
         (2, 4097, 1000), (2, 8192, 40), (300, 8193, 300), (2, 16384, 33),
         (2, 16385, 1024), (2, 32768, 5), (2, 32769, 1024), (2, 70001, 3), (1, 300_001, 1024), (2, 300_001, 500), (1, 700_001, 1024)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n,m", SIZES)
def test_top(kge, rows, n, m, dtype):
    x = normal(rows, n, n + m, dtype=dtype)
    x[:, ::7] = -math.inf
    check_top(kge, rows_of(x, dtype, pad=n % 5, offset=n % 3), m, T=0.7)


@pytest.mark.parametrize("n,m", [(40, 10), (700, 100), (9000, 512), (20_000, 1024), (50_000, 300), (50_000, 90), (1_300_000, 700)])
def test_top_of_equal_and_extreme_scores(kge, n, m):
    g = np.random.default_rng(n)
    x = np.empty((9, n))
    x[0] = 1.25                                                          # all equal
    x[1] = g.integers(0, 4, n)                                           # a few values
    x[2] = g.choice([0.0, -0.0, -1.0], n)                                # both zeros
    x[3] = g.choice([math.inf, 5.0, -math.inf, math.nan], n)
    x[4] = -math.inf
    x[5] = math.nan
    x[6] = torch.finfo(torch.float32).min                                # the lowest number is no mask
    x[7] = np.where(np.arange(n) == n - 1, 3.0, -math.inf)               # one candidate, the last
    x[8] = g.choice([1e-42, -1e-42, 2e-45, 0.0], n)                      # below the normal numbers
    check_top(kge, rows_of(torch.from_numpy(x).float()), m)


def test_sorted_rows(kge):
    """The best ones all in one wave's tiles, or in the last segment."""
    for n, m in ((5000, 1000), (30_000, 1000), (100_000, 1000), (100_000, 100), (1_100_000, 1000)):
        x = torch.arange(n, dtype=torch.float32)[None] / 7
        check_top(kge, rows_of(torch.cat([x, -x])), m, T=50.0)


# ---- sample

def check_sample(kge, x, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0, want_logp=True, **more):
    """Ids are those of the definition.  Where a number falls within 1e-12 of the border of two candidates (of the whole sum), or a sum
    within that of the border of top-p or min-p, either side is right; the inputs here have no such numbers but by chance."""
    rows, n = x.shape
    un = torch.from_numpy(u).cuda()
    ids = torch.full((rows + 1, u.shape[1]), 77, dtype=torch.int64, device="cuda")
    logp = torch.full((rows + 1, u.shape[1]), 77.0, device="cuda") if want_logp else None
    kge.kge_sample_scores(x, un, T, top_k, top_p, min_p, ids[:rows], logp[:rows] if want_logp else None, **more)
    assert (ids[rows] == 77).all()
    if want_logp:
        assert (logp[rows] == 77).all()
    x, ids = x.double().cpu().numpy(), ids.cpu().numpy()
    T, top_p, min_p = (float(np.float32(v)) for v in (T, top_p, min_p))
    for i in range(rows):
        first = order(x[i])
        if not first.size:
            assert (ids[i] == -1).all()
            if want_logp:
                assert (logp[i] == -math.inf).all()
            continue
        if T == 0:
            assert (ids[i] == first[0]).all()
            continue
        w = weights(x[i], T)
        first = first[:top_k] if top_k else first
        if top_p < 1:
            sums = np.cumsum(w[first])
            first = first[:1 + np.searchsorted(sums[:-1], top_p * sums[-1])]
        kept = np.sort(first[w[first] >= min_p])
        sums = np.cumsum(w[kept].astype(np.longdouble))
        want = np.clip(np.nan_to_num(u[i]), 0.0, 1.0) * sums[-1]
        at = np.minimum(np.searchsorted(sums, want, side="right"), np.flatnonzero(w[kept] > 0)[-1])
        for d in range(u.shape[1]):
            if ids[i, d] != kept[at[d]]:
                assert np.abs(sums - want[d]).min() < 1e-12 * sums[-1], (i, d, ids[i, d], kept[at[d]], kept.size)
                continue
            if want_logp:
                exact = float(np.log(w[kept[at[d]]] / sums[-1]))
                assert abs(logp[i, d].item() - exact) <= 1.01 * U32 * abs(exact) + 1e-12


SETTINGS = [dict(), dict(T=0.0), dict(T=0.6, min_p=0.05), dict(top_p=0.9), dict(top_p=0.5, min_p=0.2, T=2.0), dict(top_p=0.0), dict(top_k=1), dict(top_k=20),
            dict(top_k=50, top_p=0.8, min_p=0.01, T=1.5), dict(min_p=1.0), dict(top_p=0.999, T=5.0)]


@pytest.mark.parametrize("setting", range(len(SETTINGS)))
@pytest.mark.parametrize("rows,n,draws", [(1, 1, 1), (3, 5, 2), (5, 255, 7), (2, 256, 64), (3, 1000, 3), (2, 4096, 5), (2, 5000, 100), (2, 8192, 3), (300, 8193, 4), (3, 16384, 2), (1, 16385, 70),
                                          (2, 32768, 4), (2, 32769, 9), (1, 70_001, 3), (1, 1_000_003, 33)])
def test_sample(kge, rows, n, draws, setting):
    dtype = [torch.float32, torch.bfloat16, torch.float16][(n + setting) % 3]
    x = normal(rows, n, n + setting, dtype=dtype)
    if n > 2:
        x[:, 1::5] = -math.inf
        x[-1, 2::9] = math.nan
    u = np.random.default_rng(n).random((rows, draws))
    check_sample(kge, rows_of(x, dtype, pad=n % 4, offset=n % 3), u, **SETTINGS[setting])


@pytest.mark.parametrize("size", [1e6, 1e10, 1e30])
@pytest.mark.parametrize("n", [50, 900, 6000, 80_000])
def test_sample_of_large_scores(kge, n, size):
    """Neighbouring numbers are further apart than the scores that matter; small temperatures and large ones."""
    g = np.random.default_rng(n)
    x = (size * (1 + 2.0 ** -23 * g.integers(-3, 4, (3, n)))).astype(np.float32)
    x[1] = -x[1]
    for T in (1.0, 1e-3, size * 2.0 ** -23):
        check_sample(kge, rows_of(torch.from_numpy(x)), g.random((3, 9)), T=T)
        check_sample(kge, rows_of(torch.from_numpy(x)), g.random((3, 9)), T=T, top_p=0.8)


@pytest.mark.parametrize("setting", range(len(SETTINGS)))
@pytest.mark.parametrize("n", [50, 900, 6000, 33_000, 80_000])
def test_sample_of_equal_and_extreme_scores(kge, n, setting):
    g = np.random.default_rng(n)
    x = np.empty((9, n))
    x[0] = 1.25
    x[1] = g.integers(0, 4, n)
    x[2] = g.choice([0.0, -0.0, -1.0], n)
    x[3] = g.choice([math.inf, 5.0, -math.inf, math.nan], n)
    x[4] = -math.inf
    x[5] = math.nan
    x[6] = torch.finfo(torch.float32).min
    x[7] = np.where(np.arange(n) == n - 1, 3.0, -math.inf)
    x[8] = np.where(np.arange(n) % 3 == 0, torch.finfo(torch.float32).min, g.normal(0, 30, n))
    u = np.concatenate([g.random((9, 5)), np.broadcast_to([0.0, 1.0 - 2.0 ** -53], (9, 2))], 1)
    check_sample(kge, rows_of(torch.from_numpy(x).float()), u, **SETTINGS[setting])


@pytest.mark.parametrize("top_p", [1e-7, 0.3, 0.9, 0.9999, 1.0 - 2.0 ** -23])
@pytest.mark.parametrize("n", [700, 6000, 20_000, 33_001, 270_000])
def test_where_top_p_ends(kge, n, top_p):
    """Scores as they come, few different ones, one far above many equal ones, all but a few masked; differences below the normal numbers and
    above the largest one."""
    g = np.random.default_rng(n)
    u = g.random((6, 6))
    x = np.full((6, n), -math.inf)
    x[0] = g.normal(0, 3, n)
    x[1] = np.round(g.normal(0, 2, n))
    x[2] = 0.125
    x[3] = np.where(np.arange(n) == n // 3, 7.0, -2.5)
    x[4, ::97] = g.normal(0, 1, x[4, ::97].size)
    x[5] = np.where(g.random(n) < 0.5, 1.0, g.normal(1.0, 2.0 ** -9, n))
    check_sample(kge, rows_of(torch.from_numpy(x).float()), u, top_p=top_p)
    check_sample(kge, rows_of(torch.from_numpy(x).float(), torch.bfloat16), u, T=0.5, top_p=top_p, min_p=1e-4)
    check_sample(kge, rows_of(torch.from_numpy(x).float()), u, T=1e-4, top_p=top_p)
    # (weights from 1 to exp(-8.4) in steps of 2^-149; then to exp(-6.8), whose scores are further apart than any number)
    check_sample(kge, rows_of(torch.from_numpy(2.0 ** -149 * g.integers(-3000, 3000, (6, n))).float()), u, T=1e-42, top_p=top_p)
    check_sample(kge, rows_of(torch.from_numpy(3.4e38 * g.uniform(-1, 1, (6, n))).float()), u, T=1e38, top_p=top_p)


@pytest.mark.parametrize("top_k", [300, 1024])
@pytest.mark.parametrize("n", [1100, 6000, 12_000, 30_000, 40_000, 120_000, 600_000])
def test_sample_of_long_lists(kge, n, top_k):
    g = np.random.default_rng(n)
    x = g.normal(0, 2, (3, n))
    x[1] = np.round(x[1])
    x[2, n // 7:] = -math.inf
    for dtype in (torch.float32, torch.float16):
        check_sample(kge, rows_of(torch.from_numpy(x), dtype), g.random((3, 20)), top_k=top_k)
        check_sample(kge, rows_of(torch.from_numpy(x), dtype), g.random((3, 20)), T=3.0, top_k=top_k, top_p=0.95, min_p=1e-3)


def test_numbers_outside_of_the_unit_interval(kge):
    for n in (100, 2000, 50_000):
        x = normal(2, n, n)
        x[:, -1] = -math.inf
        u = np.array([[-1.0, math.nan, 1.0, 5.0, 0.25]] * 2)
        check_sample(kge, rows_of(x), u, want_logp=False)
        check_sample(kge, rows_of(x), u, top_k=10)
        check_sample(kge, rows_of(x), u, top_p=0.7)


def test_shares_of_many_draws(kge):
    """Numbers at equal distances: every candidate is drawn as often as its share says, to the one draw that a border can cost."""
    x = normal(1, 700, 3)
    draws = 200_000
    u = ((np.arange(draws) + 0.5) / draws)[None]
    ids = torch.empty(1, draws, dtype=torch.int64, device="cuda")
    kge.kge_sample_scores(rows_of(x), torch.from_numpy(u).cuda(), 1.0, 0, 1.0, 0.0, ids)
    got = np.bincount(ids.cpu().numpy()[0], minlength=700)
    w = weights(x[0].double().numpy(), 1.0)
    assert np.abs(got - draws * w / w.sum()).max() <= 1.0 + 1e-6


# ---- distill

def distill64(x, ids, t, lse, T):
    """Loss and its gradient by the definition, row by row."""
    loss, grad, scale = np.zeros(x.shape[0]), np.zeros(x.shape), np.zeros(x.shape)
    for i, row in enumerate(x):
        used = (ids[i] >= 0) & (ids[i] < x.shape[1]) & (t[i] != -np.inf)
        if not (row > -np.inf).any() or (lse is None and not used.any()):
            continue
        listed = ids[i][used]
        w = weights(row, T)
        q = w / w.sum()
        if lse is None:
            p = np.exp((t[i][used] - t[i][used].max()) / T)
            p /= p.sum()
        else:
            p = np.exp(t[i][used] / T - lse[i])
        target = np.bincount(listed, p, x.shape[1])
        with np.errstate(divide="ignore"):
            logs = np.log(p) - ((row[listed] - row[row > -np.inf].max()) / T - np.log(w.sum()))
        loss[i] = (p[p > 0] * logs[p > 0]).sum()
        rest = 0.0 if lse is None else max(0.0, 1.0 - p.sum())
        other = w.copy()
        other[listed] = 0.0
        if other.sum() == 0:
            rest = 0.0
        share = np.zeros_like(w)
        if rest > 0:
            loss[i] += rest * np.log(rest * w.sum() / other.sum())
            share = rest * other / other.sum()
        mass = p.sum() + rest
        loss[i] *= T * T
        grad[i] = T * (mass * q - target - share)
        scale[i] = T * (mass * q + target + share)  # what the gradient is a difference of
    return loss, grad, scale


def check_distill(kge, x, ids, t, lse=None, T=1.0, c=1.0, in_place=False, grad=True, **more):
    rows, n = x.shape
    dtype = x.dtype
    x64 = x.double().cpu().numpy()
    d_ids, d_t = torch.as_tensor(ids).cuda(), torch.as_tensor(t, dtype=torch.float32).cuda()
    d_lse = None if lse is None else torch.as_tensor(lse, dtype=torch.float32).cuda()
    loss = torch.full((rows + 1,), 77.0, device="cuda")
    out = x if in_place else rows_of(torch.full((rows + 1, n), 77.0), dtype, pad=3)[:rows] if grad else None
    between = None if in_place or not grad else out.as_strided((rows, out.stride(0) - n), (out.stride(0), 1), out.storage_offset() + n)
    kge.kge_distill_loss(x, d_ids, d_t, d_lse, T, c, loss[:rows], out, **more)
    assert loss[rows] == 77 and (between is None or torch.isnan(between).all())
    lse64 = None if lse is None else d_lse.double().cpu().numpy()
    want, g, scale = distill64(x64, d_ids.cpu().numpy(), d_t.double().cpu().numpy(), lse64, float(np.float32(T)))
    mass = T * T * (1.0 + 2.0)  # sums of p, p and rest: W_ERR for log Z, twice that for log(Z / Z_r)
    got = loss[:rows].double().cpu().numpy()
    finite = np.isfinite(want)
    assert np.array_equal(got[~finite], want[~finite])
    got, want = got[finite], want[finite]
    assert (np.abs(got - want) <= 1.01 * U32 * np.abs(want) + mass * 2 * W_ERR).all(), np.abs(got - want).max()
    if grad:
        got = out.double().cpu().numpy()
        limit = abs(c) * (scale * (Q_ERR + 4 * U32)) + 1.01 * HALF_STEP[dtype] * np.abs(c * g) + TINY[dtype]
        assert (np.abs(got - c * g) <= limit).all(), (np.abs(got - c * g) / limit).max()


def teacher_lists(x, m, seed, T, unused=True):
    """Lists of a teacher near the student x, and its log-sum-exp."""
    g = np.random.default_rng(seed)
    t = np.where(np.isfinite(x), x + g.normal(0, 0.5, x.shape), g.normal(0, 3, x.shape))
    ids = np.argsort(-t, axis=1, kind="stable")[:, :m].astype(np.int64)
    scores = np.take_along_axis(t, ids, 1)
    lse = np.log(np.exp((t - t.max(1, keepdims=True)) / T).sum(1)) + t.max(1) / T
    if ids.shape[1] < m:  # fewer candidates than entries
        ids = np.pad(ids, ((0, 0), (0, m - ids.shape[1])), constant_values=-1)
        scores = np.pad(scores, ((0, 0), (0, m - scores.shape[1])), constant_values=-np.inf)
    if unused:
        off = g.random(ids.shape) < 0.1
        ids[off] = g.choice([-1, x.shape[1], 1 << 40, -(1 << 40)], off.sum())
    return ids, scores, lse


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n,m", [(1, 1, 1), (3, 2, 5), (5, 255, 10), (4, 256, 256), (3, 257, 300), (2, 1024, 1024), (4, 1025, 7), (3, 4096, 64), (2, 4097, 1000),
                                      (2, 8192, 40), (300, 8193, 20), (2, 16384, 33), (2, 16385, 1024), (2, 32768, 5), (2, 32769, 1024), (2, 70001, 3), (1, 300_001, 100)])
def test_distill(kge, rows, n, m, dtype, rest):
    x = normal(rows, n, n + m, dtype=dtype)
    T = 2.0 if n % 2 else 0.75
    ids, t, lse = teacher_lists(x.double().numpy(), m, n, T)
    check_distill(kge, rows_of(x, dtype, pad=n % 5, offset=n % 3), ids, t, lse if rest else None, T=T, c=-1.5 / rows)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n,m", [(60, 20), (1000, 100), (20_000, 300), (50_000, 1024)])
def test_distill_in_place_with_masks_and_repeated_entries(kge, n, m, rest):
    x = normal(6, n, n)
    x[0, ::3] = -math.inf                                   # masked, some of them listed: an infinite loss
    x[1] = -math.inf                                        # no candidate
    ids, t, lse = teacher_lists(x.double().numpy(), m, n, 1.0)
    x[2, ids[2][(ids[2] >= 0) & (ids[2] < n)]] += 3.0
    ids[3] = np.resize(ids[3][:3], m)                       # the same three again and again
    t[3] -= 4.0
    t[4, ::2] = -np.inf                                     # entries without a share
    ids[5] = -1                                             # an empty list
    check_distill(kge, rows_of(x), ids, t, lse if rest else None, in_place=True)
    check_distill(kge, rows_of(x, pad=5), ids, t, lse if rest else None, grad=False)


@pytest.mark.parametrize("n", [60, 1000, 20_000, 50_000])
def test_distill_of_extreme_scores_and_temperatures(kge, n):
    """Rows of the type's lowest value, alone and beside masked ones; scores as far apart as the type allows and 2^-83 apart, T with them."""
    low, g = torch.finfo(torch.float32).min, np.random.default_rng(n)
    x = np.full((5, n), low)
    x[1, ::2] = -math.inf
    x[2, 1::3] = g.normal(0, 3, x[2, 1::3].size)
    x[3] = 1e30 * (1 + 2.0 ** -23 * g.integers(-3, 4, n))
    x[4] = -x[3]
    ids = np.stack([g.permutation(n)[:20] for _ in range(5)])
    ids[1] = ids[1] // 2 * 2 + 1 - 2 * (ids[1] >= n - n % 2)  # not masked
    t = g.normal(0, 1, ids.shape)
    check_distill(kge, rows_of(torch.from_numpy(x).float()), ids, t)
    for size, T in ((3.4e38, 1e18), (2.0 ** -60, 2.0 ** -60)):
        x = size * np.floor(g.uniform(-1, 1, (5, n)) * 2.0 ** 23) * 2.0 ** -23
        x[0, ::2] = -math.inf
        t = size * g.uniform(-1, 1, ids.shape)
        if size < 1:
            ids[0] = ids[1]
            check_distill(kge, rows_of(torch.from_numpy(x).float()), ids, t, T=T)
        else:  # far beyond each other: the best has all of the mass
            check_distill(kge, rows_of(torch.from_numpy(x).float()), np.argsort(-x, axis=1)[:, :20], np.sort(t, axis=1)[:, ::-1].copy(), T=T)


def test_a_rest_that_has_nowhere_to_go(kge):
    for n in (8, 300, 1024):
        x = normal(2, n, n)
        ids, t, lse = teacher_lists(x.double().numpy(), n, n, 1.0, unused=False)
        check_distill(kge, rows_of(x), ids, t, lse + 0.5)   # the list is everything, and its masses sum to less than one


@pytest.mark.parametrize("n", [100, 20_000, 50_000])
def test_nan_makes_its_row_nan_and_no_other(kge, n):
    x = normal(6, n, n)
    ids, t, lse = teacher_lists(x.double().numpy(), 5, n, 1.0, unused=False)
    x[1, n // 2], x[2, n - 1] = math.nan, math.inf
    t[3, 2], t[4, 0] = math.nan, math.inf
    loss, grad = torch.empty(6, device="cuda"), torch.empty(6, n, device="cuda")
    for teacher_lse in (None, torch.from_numpy(lse).float().cuda()):
        kge.kge_distill_loss(rows_of(x), torch.from_numpy(ids).cuda(), torch.from_numpy(t).float().cuda(), teacher_lse, 1.0, 1.0, loss, grad)
        assert torch.isnan(loss).tolist()[:4] == [False, True, True, True] and not torch.isnan(loss[5])
        assert not torch.isfinite(loss[4])
        assert torch.isfinite(grad[[0, 5]]).all() and torch.isnan(grad[[1, 2]]).all()


def test_gradient_against_differences(kge):
    x = normal(2, 300, 5)
    ids, t, lse = teacher_lists(x.double().numpy(), 20, 5, 1.5, unused=False)
    d_ids, d_t, d_lse = torch.from_numpy(ids).cuda(), torch.from_numpy(t).float().cuda(), torch.from_numpy(lse).float().cuda()
    for teacher_lse in (None, d_lse):
        grad, loss = torch.empty(2, 300, device="cuda"), torch.empty(2, device="cuda")
        kge.kge_distill_loss(rows_of(x), d_ids, d_t, teacher_lse, 1.5, 1.0, loss, grad)
        h = 2.0 ** -4
        for j in (int(ids[0, 0]), int(ids[0, 7]), 17, 123):
            two = []
            for s in (h, -h):
                y = x.clone()
                y[0, j] += s
                kge.kge_distill_loss(rows_of(y), d_ids, d_t, teacher_lse, 1.5, 1.0, loss)
                two.append(loss[0].item())
            # central difference: h^2 / 6 of the third derivative (at most T^2 / T^3 of 1), and the losses' own errors over 2 h
            assert abs((two[0] - two[1]) / (2 * h) - grad[0, j].item()) <= h * h / 6 + 1.5 ** 2 * 3 * 2 * W_ERR / h + 2 * U32 * abs(two[0]) / h


# ---- streams, graphs, workspaces, refusals

def all_three(kge, x, T=1.3, ws=None, stream=None, out=None):
    rows, n = x.shape
    o = out or dict(ids=torch.empty(rows, 40, dtype=torch.int64, device="cuda"), top=torch.empty(rows, 40, device="cuda"),
                    lse=torch.empty(rows, device="cuda"), a=torch.empty(rows, 6, dtype=torch.int64, device="cuda"),
                    b=torch.empty(rows, 6, dtype=torch.int64, device="cuda"), c=torch.empty(rows, 6, dtype=torch.int64, device="cuda"),
                    logp=torch.empty(rows, 6, device="cuda"), loss=torch.empty(rows, device="cuda"), grad=torch.empty(rows, n, device="cuda"))
    u = ((torch.arange(rows * 6, device="cuda", dtype=torch.float64).view(rows, 6) * 0.618034) % 1.0) if "u" not in o else o["u"]
    o["u"] = u
    kge.kge_top_scores(x, 40, T, o["ids"], o["top"], o["lse"], ws, hip_stream=stream)
    kge.kge_sample_scores(x, u, T, 0, 1.0, 0.0, o["a"], o["logp"], ws, hip_stream=stream)
    kge.kge_sample_scores(x, u, T, 0, 0.9, 0.0, o["b"], None, ws, hip_stream=stream)
    kge.kge_sample_scores(x, u, T, 30, 0.9, 0.001, o["c"], None, ws, hip_stream=stream)
    kge.kge_distill_loss(x, o["ids"], o["top"], o["lse"], T, 1.0, o["loss"], o["grad"], ws, hip_stream=stream)
    return o


def size_of_all(kge, rows, n):
    return max(kge.kge_top_scores_workspace(rows, n, 40), kge.kge_sample_scores_workspace(rows, n, 6, 0, 0.9),
               kge.kge_sample_scores_workspace(rows, n, 6, 30, 0.9), kge.kge_distill_loss_workspace(rows, n), 16)


@pytest.mark.parametrize("rows,n", [(64, 200), (8, 15_000), (3, 100_000)])
def test_captured_and_replayed(kge, rows, n):
    """A graph of all the calls, replayed on new scores with eager work in between, gives the bits of the eager calls."""
    x = rows_of(normal(rows, n, 1))
    ws = torch.empty(size_of_all(kge, rows, n), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        out = all_three(kge, x, ws=ws)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        all_three(kge, x, ws=ws, out=out)
    for seed in range(4):
        x.copy_(normal(rows, n, 10 + seed))
        for k in ("ids", "a", "b", "c", "loss", "grad"):
            out[k].fill_(7)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = all_three(kge, x)
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k], eager[k]), (seed, k)


def test_two_streams_at_once(kge):
    xs = [rows_of(normal(4, 90_000, s)) for s in range(2)]
    alone = [all_three(kge, x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    both = []
    for x, st in zip(xs, streams):
        both.append(all_three(kge, x, stream=st, out={k: torch.empty_like(v) if k != "u" else v for k, v in alone[0].items()}))
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for k in a:
            assert torch.equal(a[k], b[k]), k


def test_workspace_of_another_stream(kge):
    """Memory that the current stream still writes to is free for it, not for the stream of the call."""
    x = rows_of(normal(2, 200_000, 3))
    alone = {k: v.clone() for k, v in all_three(kge, x).items()}
    out = {k: torch.empty_like(v) if k != "u" else v for k, v in alone.items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    sizes = {f(2, 200_000, *rest) for f, rest in ((kge.kge_top_scores_workspace, (40,)), (kge.kge_sample_scores_workspace, (6, 0, 0.9)),
                                                  (kge.kge_sample_scores_workspace, (6, 30, 0.9)), (kge.kge_distill_loss_workspace, ()))}
    held = [torch.empty(size, dtype=torch.uint8, device="cuda") for size in sizes for _ in range(4)]
    for _ in range(200):
        for y in held:
            y.fill_(255)
    del held, y
    all_three(kge, x, stream=side, out=out)
    torch.cuda.synchronize()
    for k in alone:
        assert torch.equal(alone[k], out[k]), k


def test_same_call_same_bits(kge):
    for rows, n in [(3, 700), (5, 14_951), (2, 200_000)]:
        x = rows_of(normal(rows, n, n))
        first = {k: v.clone() for k, v in all_three(kge, x).items()}
        for _ in range(3):
            again = all_three(kge, x)
            assert all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("rows,n", [(70_001, 5), (66_000, 300)])
def test_many_rows(kge, rows, n):
    """A row's results do not depend on how many rows the call has."""
    x = torch.randn(rows, n, generator=torch.Generator("cuda").manual_seed(n), device="cuda")
    all_at_once = {k: v.clone() for k, v in all_three(kge, x).items()}
    for first in (0, 40_000, rows - 500):
        part = x[first:first + 500]
        some = all_three(kge, part, out={k: torch.empty_like(v[:500]) if k != "u" else v[first:first + 500].contiguous() for k, v in all_at_once.items()})
        assert all(torch.equal(some[k], all_at_once[k][first:first + 500]) for k in some), first


def test_positions_past_31_bits(kge):
    """A row of more than 2^31 candidates in half precision, its good ones behind that."""
    n = (1 << 31) + 70_000
    x = torch.full((1, n), -60000.0, dtype=torch.float16, device="cuda")
    where = [5, (1 << 31) - 1, 1 << 31, (1 << 31) + 1, n - 1]
    x[0, where] = torch.tensor([1.0, 4.0, 3.0, 4.0, 2.0], dtype=torch.float16, device="cuda")
    ids, top = torch.empty(1, 5, dtype=torch.int64, device="cuda"), torch.empty(1, 5, device="cuda")
    kge.kge_top_scores(x, 5, 1.0, ids, top)
    assert ids[0].tolist() == [where[i] for i in (1, 3, 2, 4, 0)]
    u = torch.tensor([[0.0, 0.01, 0.5, 0.6, 0.99]], dtype=torch.float64, device="cuda")
    w = np.exp(np.array([1.0, 4.0, 3.0, 4.0, 2.0]) - 4.0)
    want = [where[int(np.searchsorted(np.cumsum(w), v * w.sum(), side="right"))] for v in u[0].tolist()]
    got = torch.empty(1, 5, dtype=torch.int64, device="cuda")
    kge.kge_sample_scores(x, u, 1.0, 0, 1.0, 0.0, got)
    assert got[0].tolist() == want
    kge.kge_sample_scores(x, u, 1.0, 0, 0.99999, 0.0, got)
    assert got[0].tolist() == want
    loss = torch.empty(1, device="cuda")
    kge.kge_distill_loss(x, ids, top, None, 1.0, 1.0, loss, x)
    assert abs(loss.item()) <= 3 * 2 * W_ERR  # the list holds all of the mass
    assert (x[0, where].float().abs() <= 12 * U32).all()


def test_refusals_of_tensors(kge):
    x, i, f = torch.zeros(4, 50, device="cuda"), torch.zeros(4, 3, dtype=torch.int64, device="cuda"), torch.zeros(4, 3, device="cuda")
    u, loss = torch.zeros(4, 3, dtype=torch.float64, device="cuda"), torch.zeros(4, device="cuda")
    bad = [lambda: kge.kge_top_scores(x.double(), 3, 1.0, i, f), lambda: kge.kge_top_scores(x[0], 3, 1.0, i, f),
           lambda: kge.kge_top_scores(x.t(), 3, 1.0, i, f), lambda: kge.kge_top_scores(x[:1].expand(4, 50), 3, 1.0, i, f),
           lambda: kge.kge_top_scores(x, 4, 1.0, i, f), lambda: kge.kge_top_scores(x, 3, 1.0, i.int(), f),
           lambda: kge.kge_top_scores(x, 3, 1.0, i, f, torch.zeros(3, device="cuda")),
           lambda: kge.kge_sample_scores(x, u.float(), 1.0, 0, 1.0, 0.0, i), lambda: kge.kge_sample_scores(x, u[:3], 1.0, 0, 1.0, 0.0, i),
           lambda: kge.kge_sample_scores(x, u, 1.0, 0, 1.0, 0.0, i[:, :2]),
           lambda: kge.kge_distill_loss(x, i, f.double(), None, 1.0, 1.0, loss), lambda: kge.kge_distill_loss(x, i, f, f, 1.0, 1.0, loss),
           lambda: kge.kge_distill_loss(x, i, f, None, 1.0, 1.0, loss, x.half()), lambda: kge.kge_distill_loss(x, i, f, None, 1.0, 1.0, loss, x[:, :40])]
    for call in bad:
        with pytest.raises((TypeError, ValueError)):
            call()
    with pytest.raises(kge.KgeError):
        kge.kge_sample_scores(x, u, -1.0, 0, 1.0, 0.0, i)
