"""kge_distill_step over the sizes of its rows, temperatures, contexts, streams and graphs, against 64-bit autograd or against itself."""
import numpy as np
import pytest
import torch

from test_gpu_distill_step import kge, psi  # noqa: F401

pytestmark = pytest.mark.gpu


def grads64(model, E, R, h, r, t, neg, chunk, head, gamma, ids, tops, lse, T):
    """Loss and the tables' gradients; entries with an id of -1 are unused."""
    E, R = (torch.from_numpy(x).double().requires_grad_() for x in (E, R))
    rows = torch.from_numpy(neg).repeat_interleave(chunk, 0)
    s = psi(model, E, R, torch.from_numpy(t if head else h), torch.from_numpy(r), rows, head) + (gamma if model == "transe_l2" else 0.0)
    logq = torch.log_softmax(s / T, 1)
    used, at, tops = torch.from_numpy(ids >= 0), torch.from_numpy(np.maximum(ids, 0)), torch.from_numpy(tops).double()
    masked = torch.where(used, tops, torch.full_like(tops, -1e300))
    log_p = torch.log_softmax(masked / T, 1) if lse is None else masked / T - torch.from_numpy(lse).double()[:, None]
    p = torch.where(used, log_p.exp(), torch.zeros_like(log_p))
    loss = (p * (torch.where(used, log_p, torch.zeros_like(log_p)) - logq.gather(1, at))).sum(1)
    if lse is not None:
        rest = 1 - p.sum(1)
        listed = torch.zeros_like(logq).scatter_add(1, at, used.double()) > 0
        loss = loss + rest * (torch.log(rest) - torch.logsumexp(torch.where(listed, torch.full_like(logq, -1e300), logq), 1))
    loss = T * T * loss.mean()
    loss.backward()
    return loss.item(), E.grad.numpy(), R.grad.numpy()


class Case:
    def __init__(self, kge, model, b, chunk, k, D, m, rest, seed, scale=1.0, T=1.5, **context):
        g = np.random.default_rng(seed)
        n_ent, n_rel = 1200, 5
        self.kge, self.model, self.chunk, self.k, self.T = kge, model, chunk, k, T
        self.E = g.uniform(-scale, scale, (n_ent, D)).astype(np.float32)
        self.R = g.uniform(-1, 1, (n_rel, D * D if model == "rescal" else D)).astype(np.float32)
        self.h, self.t = g.integers(0, n_ent, (2, b))
        self.r, self.neg = g.integers(0, n_rel, b), g.integers(0, n_ent, (b // chunk, k))
        self.ids = np.stack([g.permutation(k)[:m] for _ in range(b)])
        self.tops = g.normal(0, 1, (b, m)).astype(np.float32)
        self.ids[g.random(self.ids.shape) < 0.2] = -1
        self.ids[:, 0] = np.maximum(self.ids[:, 0], 0)
        for i in range(b):  # (distinct)
            self.ids[i, 1:][self.ids[i, 1:] == self.ids[i, 0]] = -1
        of_used = np.where(self.ids >= 0, np.exp(self.tops.astype(np.float64) / T), 0.0).sum(1)
        self.lse = (np.log(of_used) + g.uniform(0.05, 0.7, b)).astype(np.float32) if rest else None
        self.ctx = kge.KgeContext(model, n_ent, n_rel, D, self.R.shape[1], max_batch=b, max_neg_per_chunk=k, max_chunks=b // chunk, **context)
        self.rowwise = context.get("adagrad_mode", 0) == 1
        self.dev = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (self.h, self.r, self.t, self.neg.reshape(-1), self.ids, self.tops)]
        self.dev_lse = None if self.lse is None else torch.from_numpy(self.lse).cuda()
        self.loss = torch.zeros(1, device="cuda")
        self.tables = [torch.empty_like(torch.from_numpy(x)).cuda() for x in (self.E, self.R)]
        self.states = [torch.zeros(x.shape[0] if self.rowwise else x.shape, device="cuda") for x in self.tables]
        self.reset()

    def reset(self):
        for d, x in zip(self.tables, (self.E, self.R)):
            d.copy_(torch.from_numpy(x))
        for x in self.states:
            x.zero_()

    def step(self, head=0, stream=None):
        dh, dr, dt, dn, di, ds = self.dev
        self.ctx.distill_step(self.tables[0], self.states[0], self.tables[1], self.states[1], dh, dr, dt, dn, self.k, self.chunk, head, 6.0, 0.05, di, ds,
                              self.dev_lse, self.T, loss_out=self.loss, stream=stream)

    def results(self):
        torch.cuda.synchronize()
        return [x.clone() for x in (*self.tables, *self.states, self.loss)]

    def check(self, off, head=0):
        self.step(head)
        torch.cuda.synchronize()
        want, *grads = grads64(self.model, self.E, self.R, self.h, self.r, self.t, self.neg, self.chunk, bool(head), 6.0, self.ids, self.tops, self.lse, self.T)
        assert abs(self.loss.item() - want) <= off * max(1.0, abs(want)), (self.loss.item(), want)
        for state, g in zip(self.states, grads):
            assert torch.isfinite(state).all()
            got = state.double().sqrt().cpu().numpy()
            g = np.sqrt((g ** 2).mean(1)) if self.rowwise else np.abs(g)
            assert np.sqrt(((got - g) ** 2).sum()) <= off * np.sqrt((g ** 2).sum())


# Scores are sums of up to 16 products of up to 1 in 32 bits, off by up to 16 * 2^-24 * 4; the shares p and q, of which a gradient is T times the difference, follow them by
# that over T, and the difference is of the size of the scores' own differences (1 and more) over T.
OFF = 4e-5


@pytest.mark.parametrize("T", [1.5, 30.0])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("model", ["distmult", "transe_l2"])
@pytest.mark.parametrize("k,m", [(200, 9), (900, 40), (2500, 40), (6000, 64), (12_000, 64), (20_000, 300), (32_768, 30)])
def test_rows_of_every_size(kge, k, m, model, rest, T):
    case = Case(kge, model, 8, 4, k, 16, m, rest, k, T=T)
    try:
        case.check(OFF, head=k % 2)
    finally:
        case.ctx.close()


@pytest.mark.parametrize("model", ["complex", "rescal"])
@pytest.mark.parametrize("T", [1.5, 30.0])
def test_other_models_at_large_temperatures(kge, model, T):
    case = Case(kge, model, 48, 24, 700, 16, 20, True, 3, T=T)
    try:
        case.check(OFF)
    finally:
        case.ctx.close()


@pytest.mark.parametrize("T", [0.05, 1.0, 5.0])
def test_lists_far_above_the_rest(kge, T):
    """Listed candidates whose scores lie some 20 above the others': 400 T, 20 T and 4 T.  (Scores of up to 40 from 16 products, off by 2e-5, over T.)"""
    case = Case(kge, "distmult", 16, 8, 300, 16, 5, True, 9, T=T)
    try:
        case.R[:] = 1.0
        for i in range(16):
            kept = case.E[case.h[i]]
            for at in case.ids[i][case.ids[i] >= 0]:
                case.E[case.neg[i // 8, at]] = np.sign(kept) * 2.0
        case.reset()
        case.step()
        torch.cuda.synchronize()
        assert torch.isfinite(case.loss).all() and all(torch.isfinite(x).all() for x in (*case.tables, *case.states))
        case.reset()
        case.check(1e-4 / min(T, 1.0))
    finally:
        case.ctx.close()


@pytest.mark.parametrize("model", ["distmult", "transe_l2"])
def test_the_losses_of_the_context_are_not_used(kge, model):
    results = []
    for context in (dict(), dict(adv_temperature=1.0), dict(loss="ranking"), dict(loss="ranking", adv_temperature=0.5), dict(validate_indices=True)):
        case = Case(kge, model, 64, 16, 128, 32, 10, True, 5, **context)
        try:
            case.step()
            results.append(case.results())
        finally:
            case.ctx.close()
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


@pytest.mark.parametrize("model", ["distmult", "transe_l2", "complex"])
def test_one_accumulator_per_row(kge, model):
    case = Case(kge, model, 64, 16, 128, 32, 10, True, 7, adagrad_mode=1)
    try:
        case.check(OFF)
    finally:
        case.ctx.close()


@pytest.mark.parametrize("k,b,T", [(64, 32, 2.0), (3000, 16, 2.0), (900, 512, 12.0)])
def test_another_stream_and_a_graph(kge, k, b, T):
    case = Case(kge, "distmult", b, 8, k, 32, 12, True, 11, T=T)
    try:
        case.step()
        eager = case.results()
        case.reset()
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        case.step(stream=stream)
        assert all(torch.equal(a, b) for a, b in zip(eager, case.results()))
        case.reset()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            case.step(stream=stream)
        torch.cuda.synchronize()
        for _ in range(3):  # on new lists each time, with eager steps between
            case.dev[5].copy_(torch.randn_like(case.dev[5]))
            if case.dev_lse is not None:
                case.dev_lse.copy_(torch.logsumexp(torch.where(case.dev[4] >= 0, case.dev[5], -1e30).double() / T, 1) + 0.3)
            case.reset()
            case.step()
            eager = case.results()
            case.reset()
            torch.cuda.synchronize()
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(eager, case.results()))
    finally:
        case.ctx.close()
