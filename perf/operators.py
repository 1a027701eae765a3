"""Operators on rows of scores, as cases that can be timed and compared.

A row holds a model's scores of the candidates of one query (h, r, ?) or (?, r, t), as kge_score writes them.  Three operators:

  "top"      kge_top_scores: the m best candidates of every row in order, and the row's log-sum-exp (answers to a query; the list
             that a teacher hands to a student)
  "sample"   kge_sample_scores: candidates drawn from the row's softmax with temperature, top-k, top-p and min-p, by given random
             numbers (hard negatives, sampled answers)
  "distill"  kge_distill_loss: divergence of a student's row from a teacher's list of best candidates, and its gradient

`own` chooses between the plain forms below and the library's entry points; both take what `prepare` gives.
"""
import math

import numpy as np
import torch

own = False

_DEFAULTS = dict(kind="top", rows=1024, n=14_951, pad=0, dtype="float32", masked=8, temperature=1.0, m=0, lse=True, draws=0,
                 top_k=0, top_p=1.0, min_p=0.0, rest=False, grad=True)


def _case(**kw):
    return dict(_DEFAULTS, **kw)


def listed():
    return [
        # the smallest mini-batch in use: best ten of the 64 candidates of its chunk, one launch in a loop of small ones
        _case(kind="top", name="top-chunk", rows=256, n=64, m=10, lse=False, masked=0),
        # a teacher's lists for one mini-batch over all entities of an FB15k-sized graph, at the student's temperature
        _case(kind="top", name="top-teacher", m=64, temperature=2.0),
        # the hundred best answers of a few queries over a graph of 2.5 M entities, scores kept in half the bytes
        _case(kind="top", name="top-answers", rows=16, n=2_500_000, m=100, dtype="bfloat16", lse=False),
        # one query answered by a draw: latency is all there is
        _case(kind="sample", name="sample-query", rows=1, temperature=0.7, top_p=0.9, draws=1),
        # sixteen hard negatives for every positive of a mini-batch out of all entities
        _case(kind="sample", name="sample-negatives", draws=16),
        # one answer each for a batch of queries, unlikely ones left out
        _case(kind="sample", name="sample-nucleus", top_p=0.9, draws=1),
        # a few queries over a mid-sized graph, all four settings
        _case(kind="sample", name="sample-all-settings", rows=8, n=2_500_000, dtype="bfloat16", temperature=0.8, top_k=50, top_p=0.95,
              min_p=0.02, draws=4),
        # two queries over ten million entities: a long axis and hardly any rows
        _case(kind="sample", name="sample-freebase", rows=2, n=10_000_000, top_p=0.95, draws=64),
        # the candidates of a chunk (256) for a mini-batch of 1024, the training step on small graphs
        _case(kind="distill", name="distill-chunk", n=256, m=16, masked=0, temperature=2.0),
        # a mini-batch against all entities of an FB15k-sized graph, with the mass that the lists leave out
        _case(kind="distill", name="distill-rest", m=64, rest=True, temperature=2.0),
        # validation loss at odd sizes: rows that start at any address, half precision, no gradient
        _case(kind="distill", name="distill-validation", rows=690, n=40_943, pad=6, dtype="float16", m=100, grad=False),
        # few long rows with their gradient
        _case(kind="distill", name="distill-medium", rows=16, n=2_500_000, dtype="bfloat16", m=256, rest=True),
    ]


_MOST = 40_000_000  # elements of the largest listed case


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    c = _case(kind=rng.choice(["top", "sample", "sample", "distill"]))
    c["n"] = _log(rng, 40, 5_000_000)
    c["rows"] = _log(rng, 1, max(1, min(4_096, _MOST // 2 // c["n"])))
    c["dtype"] = rng.choice(["float32", "float32", "bfloat16", "float16"])
    c["pad"] = rng.choice([0, 0, rng.randrange(1, 40)])
    c["masked"] = rng.choice([0, 0, _log(rng, 1, c["n"] // 8)])
    c["temperature"] = rng.choice([1.0, 1.0, 2.0, 0.7])
    most = min(c["n"], 1_024)
    if c["kind"] == "top":
        c["m"], c["lse"] = _log(rng, 1, most), rng.random() < 0.5
    elif c["kind"] == "sample":
        c["draws"] = _log(rng, 1, 64)
        c["top_k"] = rng.choice([0, 0, _log(rng, 1, most)])
        c["top_p"] = rng.choice([1.0, 0.95, 0.9, 0.5])
        c["min_p"] = rng.choice([0.0, 0.0, 0.02])
    else:
        c["m"], c["rest"], c["grad"] = _log(rng, 1, min(c["n"] // 2, 512)), rng.random() < 0.5, rng.random() < 0.75
    return c


# ---------------------------------------------------------------------------------------------------------------


def _inputs(c, seed):
    """Scores of a trained model: most candidates unlikely, a few dozen far above the others; known answers are masked, and some
    queries that only fill a mini-batch up are masked altogether."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rows, n, dtype = c["rows"], c["n"], getattr(torch, c["dtype"])

    def rand(*shape, dtype=torch.float32):
        return torch.rand(*shape, generator=g, device="cuda", dtype=dtype)

    def some(count):
        return torch.randint(n, (rows, count), generator=g, device="cuda")

    x = torch.randn(rows, n, generator=g, device="cuda").mul_(2.5).sub_(4.0)
    good = some(min(24, n))
    x.scatter_add_(1, good, rand(*good.shape).mul_(8).add_(4))
    s = {}
    if c["kind"] == "distill":
        teacher = x + torch.randn(rows, n, generator=g, device="cuda").mul_(0.7)
        s["teacher_scores"], s["teacher_ids"] = (y.contiguous() for y in torch.topk(teacher, c["m"], dim=1))
        unused = rand(rows, c["m"]) < 0.02  # lists that came out shorter
        s["teacher_ids"].masked_fill_(unused, -1)
        s["teacher_lse"] = torch.logsumexp(teacher.double() / c["temperature"], 1).float() if c["rest"] else None
        del teacher
    elif c["masked"]:
        x.scatter_(1, some(c["masked"]), -math.inf)
    if c["masked"] and rows >= 64:
        x[63::64] = -math.inf
    s["buffer"] = torch.full((rows, n + c["pad"]), math.nan, dtype=dtype, device="cuda")
    s["scores"] = s["buffer"][:, :n]
    s["scores"].copy_(x)
    if c["kind"] == "sample":
        s["u"] = rand(rows, c["draws"], dtype=torch.float64)
    return s


def prepare(case, seed):
    c = case
    s = dict(c, **_inputs(c, seed))
    rows = c["rows"]

    def out(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if c["kind"] == "top":
        s["ids_out"], s["scores_out"] = out(rows, c["m"], dtype=torch.int64), out(rows, c["m"])
        s["lse_out"] = out(rows) if c["lse"] else None
    elif c["kind"] == "sample":
        s["ids_out"], s["logp_out"] = out(rows, c["draws"], dtype=torch.int64), out(rows, c["draws"])
    else:
        s["loss_out"] = out(rows)
        s["grad_out"] = out(rows, c["n"], dtype=s["scores"].dtype) if c["grad"] else None
    s["workspace"] = None
    if own:
        import paper_2004_08532_amd as kge
        size = {"top": lambda: kge.kge_top_scores_workspace(rows, c["n"], c["m"]),
                "sample": lambda: kge.kge_sample_scores_workspace(rows, c["n"], c["draws"], c["top_k"], c["top_p"]),
                "distill": lambda: kge.kge_distill_loss_workspace(rows, c["n"])}[c["kind"]]()
        s["workspace"] = out(size, dtype=torch.uint8) if size else None
    return s


def run(state):
    s = state
    if own:
        return _RUN_OWN[s["kind"]](s)
    return _RUN_PLAIN[s["kind"]](s)


def _top_own(s):
    import paper_2004_08532_amd as kge
    kge.kge_top_scores(s["scores"], s["m"], s["temperature"], s["ids_out"], s["scores_out"], s["lse_out"], s["workspace"])
    return [s["ids_out"], s["scores_out"], s["lse_out"]][:3 if s["lse"] else 2]


def _sample_own(s):
    import paper_2004_08532_amd as kge
    kge.kge_sample_scores(s["scores"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["ids_out"], s["logp_out"],
                          s["workspace"])
    return [s["ids_out"], s["logp_out"]]


def _distill_own(s):
    import paper_2004_08532_amd as kge
    kge.kge_distill_loss(s["scores"], s["teacher_ids"], s["teacher_scores"], s["teacher_lse"], s["temperature"], 1.0 / s["rows"],
                         s["loss_out"], s["grad_out"], s["workspace"])
    return [s["loss_out"], s["grad_out"]][:2 if s["grad"] else 1]


def _ordered(x):
    """Every row in order, best first and equal scores by their position; -inf: left out."""
    return torch.sort(torch.where(torch.isnan(x), -math.inf, x), dim=1, descending=True, stable=True)


def _relative(x, best, temperature):
    """exp((x - best) / temperature); a row without a best has none."""
    return torch.where(best > -math.inf, torch.exp((x - best) / temperature), torch.zeros_like(x))


def _top_plain(s):
    values, order = _ordered(s["scores"].float())
    top, ids = values[:, :s["m"]].contiguous(), order[:, :s["m"]]
    out = [torch.where(top > -math.inf, ids, -1), top]
    if s["lse"]:
        best, temperature = values[:, :1].double(), float(np.float32(s["temperature"]))
        total = _relative(values.double(), best, temperature).sum(1)
        out.append((best[:, 0] / temperature + torch.log(total)).float())
    return out


def _sample_plain(s):
    x = s["scores"].double()
    rows, n = x.shape
    temperature, top_p, min_p = (float(np.float32(s[k])) for k in ("temperature", "top_p", "min_p"))
    if s["top_k"] or top_p < 1 or min_p > 0:
        values, order = _ordered(x)
        w = _relative(values, values[:, :1], temperature)
        w[:, s["top_k"] or n:] = 0
        cut = w.cumsum(1)
        keep = w >= min_p
        if top_p < 1:
            keep[:, 1:] &= cut[:, :-1] < top_p * cut[:, -1:]
        w = torch.zeros_like(x).scatter_(1, order, w * keep)
    else:
        x = torch.where(torch.isnan(x), -math.inf, x)
        w = _relative(x, x.amax(1, keepdim=True), temperature)
    below = w.cumsum(1)
    total = below[:, -1:].clone()
    ids = torch.searchsorted(below, s["u"] * total, right=True)
    ids = torch.minimum(ids, (n - 1) - (w > 0).flip(1).int().argmax(1, keepdim=True))
    logp = torch.log(w.gather(1, ids) / total).float()
    empty = total == 0
    return [torch.where(empty, -1, ids), torch.where(empty, -math.inf, logp)]


def _distill_plain(s):
    # in 64 bits: the rest is what is left of 1, and the loss of a student that is close to its teacher a difference of near values
    T, n = float(np.float32(s["temperature"])), s["n"]
    z = s["scores"].double() / T
    best = z.amax(1, keepdim=True)
    w = _relative(z, best, 1.0)
    Z = w.sum(1, keepdim=True)
    used = (s["teacher_ids"] >= 0) & (s["teacher_ids"] < n) & (best > -math.inf)
    ids = torch.where(used, s["teacher_ids"], 0)
    t = torch.where(used, s["teacher_scores"].double() / T, -math.inf)
    if s["rest"]:
        log_p = t - s["teacher_lse"].double()[:, None]
        p = torch.exp(log_p)
    else:
        e = _relative(t, t.amax(1, keepdim=True), 1.0)
        p = e / e.sum(1, keepdim=True)
        log_p = torch.log(p)
    p = torch.where(used, p, 0)
    log_q = z.gather(1, ids) - best - torch.log(Z)
    loss = torch.where(p > 0, p * (log_p - log_q), 0).sum(1)
    target = torch.zeros_like(z).scatter_add_(1, ids, p)
    mass = p.sum(1, keepdim=True)
    if s["rest"]:
        unlisted = torch.zeros_like(z).scatter_add_(1, ids, used.to(z.dtype)) == 0
        other = (w * unlisted).sum(1, keepdim=True)
        rest = torch.where(best > -math.inf, (1 - mass).clamp(min=0), 0)
        loss = loss + torch.where(rest > 0, rest * torch.log(rest * Z / other), 0)[:, 0]
        target = target + rest * w * unlisted / other
        mass = mass + rest
    live = (best > -math.inf) & (mass > 0)
    out = [(torch.where(live[:, 0], loss, 0) * T * T).float()]
    if s["grad"]:
        out.append(torch.where(live, (mass * w / Z - target) * (T / s["rows"]), 0).to(s["scores"].dtype))
    return out


_RUN_OWN = {"top": _top_own, "sample": _sample_own, "distill": _distill_own}
_RUN_PLAIN = {"top": _top_plain, "sample": _sample_plain, "distill": _distill_plain}


# ---------------------------------------------------------------------------------------------------------------


def exact(case, seed):
    """In 64 bits, row by row, from the definitions."""
    c = case
    s = _inputs(c, seed)
    x = s["scores"].double().cpu().numpy()
    T = float(np.float32(c["temperature"]))
    if c["kind"] == "top":
        ids, top = np.full((c["rows"], c["m"]), -1, np.int64), np.full((c["rows"], c["m"]), -np.inf)
        lse = np.full(c["rows"], -np.inf)
        for i, row in enumerate(x):
            there = np.flatnonzero(row > -np.inf)
            least = np.sort(row[there])[-c["m"]] if there.size > c["m"] else -np.inf
            short = there[row[there] >= least]
            first = short[np.lexsort((short, -row[short]))][:c["m"]]
            ids[i, :first.size], top[i, :first.size] = first, row[first]
            if there.size:
                lse[i] = row[first[0]] / T + np.log(np.exp((row[there] - row[first[0]]) / T).sum())
        return [ids, top, lse][:3 if c["lse"] else 2]
    if c["kind"] == "sample":
        u = s["u"].cpu().numpy()
        ids, logp = np.full(u.shape, -1, np.int64), np.full(u.shape, -np.inf)
        top_p, min_p = float(np.float32(c["top_p"])), float(np.float32(c["min_p"]))
        for i, row in enumerate(x):
            there = np.flatnonzero(row > -np.inf)
            if not there.size:
                continue
            w = np.exp((row[there] - row[there].max()) / T)
            first = np.argsort(-row[there], kind="stable")
            count = first.size
            if c["top_k"]:
                count = min(count, c["top_k"])
            if top_p < 1:
                sums = np.cumsum(w[first[:count]])
                count = min(count, 1 + int(np.searchsorted(sums, top_p * sums[-1])))
            kept = first[:count]
            kept = np.sort(kept[w[kept] >= min_p])
            sums = np.cumsum(w[kept])
            at = np.minimum(np.searchsorted(sums, u[i] * sums[-1], side="right"), kept.size - 1)
            ids[i], logp[i] = there[kept[at]], np.log(w[kept[at]] / sums[-1])
        return [ids, logp]
    t_ids, t = s["teacher_ids"].cpu().numpy(), s["teacher_scores"].double().cpu().numpy()
    loss, grad = np.zeros(c["rows"]), np.zeros(x.shape) if c["grad"] else None
    for i, row in enumerate(x):
        used = (t_ids[i] >= 0) & (t_ids[i] < c["n"])
        listed, best = t_ids[i][used], row.max()
        if best == -np.inf or not listed.size:
            continue  # (a list with no entry leaves nothing to learn; cases with `rest` always have one)
        w = np.exp((row - best) / T)
        q = w / w.sum()
        if c["rest"]:
            p = np.exp(t[i][used] / T - float(s["teacher_lse"][i]))
        else:
            p = np.exp((t[i][used] - t[i][used].max()) / T)
            p /= p.sum()
        target = np.bincount(listed, p, c["n"])
        loss[i] = (p * (np.log(p) - (row[listed] - best) / T + np.log(w.sum()))).sum()
        rest = max(0.0, 1.0 - p.sum()) if c["rest"] else 0.0
        if rest > 0:
            other = w.copy()
            other[listed] = 0
            loss[i] += rest * np.log(rest / (other.sum() / w.sum()))
            target += rest * other / other.sum()
        loss[i] *= T * T
        if c["grad"]:
            grad[i] = (target.sum() * q - target) * T / c["rows"]
    return [loss, grad][:2 if c["grad"] else 1]


def work(case):
    """Bytes: every score is read once, a gradient is written once, lists and random numbers are read or written once.  Flops: a
    comparison per element of a top list; a difference, an exponential and a sum per element of a distribution, and a product
    and a difference per element of its gradient."""
    c = case
    cells, size = c["rows"] * c["n"], 4 if c["dtype"] == "float32" else 2
    if c["kind"] == "top":
        return {"bytes": cells * size + c["rows"] * (12 * c["m"] + 4 * c["lse"]), "flops": cells * (4 if c["lse"] else 1)}
    if c["kind"] == "sample":
        return {"bytes": cells * size + 20 * c["rows"] * c["draws"], "flops": 4 * cells}
    return {"bytes": cells * size * (2 if c["grad"] else 1) + c["rows"] * (12 * c["m"] + 4 + 4 * c["rest"]),
            "flops": cells * (6 if c["grad"] else 4)}
