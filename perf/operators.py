"""The operators on rows of logits as timed cases: the top entries of a row with the
log-sum-exp of the rest (what is kept of a teacher's row), the distillation loss from
such entries with its gradient, and drawing a token from given uniforms under
temperature, top-k, top-p and min-p.

With `own` false `run()` computes them in elementary torch operations, with `own`
true by the binding's entry points.  Rows follow the shape of the library's synthetic
target rows (a power law over the ranks, here with an exponent of each row's own), in
the place of a model's.
"""
import math

import torch

own = False
DEV = "cuda"
VOCABS = (4096, 32000, 50257, 128256, 151936)


def listed():
    return [
        # the smallest call: one row of the tiny drafter; launches count
        dict(name="top_one_row", kind="top", rows=1, vocab=4096, dtype="f32", k=8, T=1.0, pad=0),
        # what one user's verified chain gives to train on later
        dict(name="top_chain_bf16", kind="top", rows=16, vocab=151936, dtype="bf16", k=64, T=1.0, pad=0),
        # an odd vocabulary, whose rows are not aligned, at a training temperature
        dict(name="top_odd_f32", kind="top", rows=60, vocab=50257, dtype="f32", k=33, T=2.0, pad=0),
        # a teacher's pass over a large batch of chains, many entries kept
        dict(name="top_batch_bf16", kind="top", rows=960, vocab=151936, dtype="bf16", k=256, T=1.0, pad=0),
        # a step of the tiny drafter on the teacher's entries alone (no rest)
        dict(name="distill_tiny_f32", kind="distill", rows=15, vocab=4096, dtype="f32", k=16, T=1.0, rest=False,
             grad=True, pad=0),
        # 16 chains of 15 drafted positions, as the training forward leaves their logits
        dict(name="distill_bs16_f32", kind="distill", rows=240, vocab=151936, dtype="f32", k=64, T=2.0, rest=True,
             grad=True, pad=0),
        # an odd vocabulary in bf16, rows of padded width
        dict(name="distill_odd_bf16", kind="distill", rows=75, vocab=50257, dtype="bf16", k=100, T=1.5, rest=True,
             grad=True, pad=7),
        # the loss alone, as an evaluation takes it
        dict(name="distill_eval_bf16", kind="distill", rows=480, vocab=151936, dtype="bf16", k=128, T=1.0, rest=True,
             grad=False, pad=0),
        # one interactive user's next token
        dict(name="sample_one_user", kind="sample", rows=1, vocab=151936, dtype="bf16", filters="top_k+top_p", T=0.8,
             pad=0),
        # a few users under min-p, an odd vocabulary
        dict(name="sample_min_p_odd", kind="sample", rows=33, vocab=50257, dtype="f32", filters="min_p", T=1.0, pad=0),
        # a serving batch under top-p: peaked rows and flat ones whose nucleus is thousands of tokens
        dict(name="sample_top_p_bs512", kind="sample", rows=512, vocab=151936, dtype="bf16", filters="top_p", T=0.9,
             pad=0),
        # a batch whose users each set their own filters, or none
        dict(name="sample_mixed_bs64", kind="sample", rows=64, vocab=128256, dtype="f32", filters="mixed", T=1.0, pad=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["top", "distill", "sample"])
    vocab = rng.choice(VOCABS) if rng.random() < 0.5 else _log_int(rng, 1000, 151936)
    dtype = rng.choice(["f32", "bf16"])
    rows = _log_int(rng, 1, min(1000, 36_000_000 // vocab))
    case = dict(kind=kind, rows=rows, vocab=vocab, dtype=dtype, pad=rng.choice([0, 0, rng.randint(1, 64)]))
    if kind == "sample":
        filters = rng.choice(["none", "top_k", "top_p", "min_p", "top_k+top_p", "mixed"])
        return dict(case, filters=filters, T=round(rng.uniform(0.5, 1.5), 2))
    case.update(k=_log_int(rng, 1, min(1024, vocab)), T=round(rng.uniform(0.7, 3.0), 2))
    if kind == "distill":
        case.update(rest=rng.random() < 0.6, grad=rng.random() < 0.8)
    return case


# --------------------------------------------------------------------------
# inputs, from the seed alone
# --------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 4099 + stream)
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(case, g):
    """[rows, vocab] logits in fp32: a * (-log u), that is a power law of exponent a over the
    ranks, a between 1.1 (flat) and 2.5 (peaked) for each row, moved to values a model has."""
    a = 1.1 + 1.4 * torch.rand(case["rows"], 1, generator=g, device=DEV)
    u = torch.rand(case["rows"], case["vocab"], generator=g, device=DEV).clamp_(min=2.0**-24)
    return u.log_().neg_().mul_(a).sub_(2.0)


def _store(case, x):
    """The rows in their type, a padded width apart."""
    buf = torch.full((case["rows"], case["vocab"] + case["pad"]), -1.0, device=DEV, dtype=_dtype(case))
    buf[:, :case["vocab"]] = x
    return buf[:, :case["vocab"]]


def _uniform(g, n, lo, hi):
    return lo + (hi - lo) * torch.rand(n, generator=g, device=DEV)


def prepare(case, seed):
    g = _gen(seed, 1)
    n, V = case["rows"], case["vocab"]
    s = dict(case=case)
    if case["kind"] == "distill":
        teacher = _rows(case, g)
        noise = torch.randn(n, V, generator=g, device=DEV)
        s["logits"] = _store(case, noise.mul_(0.7).add_(teacher, alpha=0.8))
        teacher = teacher.to(torch.bfloat16).float()   # a teacher's rows are kept from bf16 logits
        vals, ids = torch.sort(teacher, dim=1, descending=True, stable=True)
        s["t_vals"], s["t_ids"] = vals[:, :case["k"]].contiguous(), ids[:, :case["k"]].int().contiguous()
        if case["rest"]:
            others = vals[:, case["k"]:].double() / case["T"]
            s["t_rest"] = torch.logsumexp(others, 1).float() if others.shape[1] else torch.full((n,), -math.inf, device=DEV)
        # the position decay of the training loss over chains of 15, some positions past a chain's end
        w = torch.exp(-(torch.arange(n, device=DEV) % 15) / 15.0)
        s["weights"] = torch.where(torch.rand(n, generator=g, device=DEV) < 0.1, 0.0, w)
        s["weights"][0] = 1.0
    else:
        s["logits"] = _store(case, _rows(case, g))
    if case["kind"] == "sample":
        f = case["filters"]
        on = lambda name: f == "mixed" or name in f  # noqa: E731
        some = lambda: torch.rand(n, generator=g, device=DEV) < (0.5 if f == "mixed" else 1.0)  # noqa: E731
        s["T"] = _uniform(g, n, 0.85, 1.15) * case["T"]
        s["u"] = torch.rand(n, generator=g, device=DEV)
        s["top_k"] = s["top_p"] = s["min_p"] = None
        if on("top_k"):
            k = torch.randint(5, min(101, V), (n,), generator=g, device=DEV, dtype=torch.int32)
            s["top_k"] = torch.where(some(), k, 0)
        if on("top_p"):
            s["top_p"] = torch.where(some(), _uniform(g, n, 0.8, 0.98), 1.0)
        if on("min_p"):
            s["min_p"] = torch.where(some(), _uniform(g, n, 0.01, 0.2), 0.0)
        if f == "mixed":   # some users decode greedily
            s["T"] = torch.where(torch.rand(n, generator=g, device=DEV) < 0.1, 0.0, s["T"])
    return s


# --------------------------------------------------------------------------
# plain forms: elementary operations, in 32 bits; sampling, whose tokens turn on
# borders between running sums, in 64
# --------------------------------------------------------------------------
def _plain_top(case, s):
    vals, ids = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    k = case["k"]
    rest = vals[:, k:] / case["T"]
    if rest.shape[1]:
        m = rest[:, :1]
        rest = m[:, 0] + torch.log(torch.exp(rest - m).sum(1))
    else:
        rest = torch.full((case["rows"],), -math.inf, device=DEV)
    return dict(ids=ids[:, :k].int(), vals=vals[:, :k].contiguous(), rest=rest)


def _plain_distill(case, s):
    T = case["T"]
    z = s["logits"].float() / T
    t = s["t_vals"] / T
    rest = s["t_rest"][:, None] if case["rest"] else torch.full_like(t[:, :1], -math.inf)
    t = torch.cat([t, rest], 1)
    t = t - t.max(1, keepdim=True).values
    log_p = t - torch.log(torch.exp(t).sum(1, keepdim=True))
    p = torch.exp(log_p)
    m = z.max(1, keepdim=True).values
    e = torch.exp(z - m)
    ids = s["t_ids"].long()
    others = e.scatter(1, ids, 0.0).sum(1, keepdim=True)
    total = e.sum(1, keepdim=True)
    log_q = torch.cat([z.gather(1, ids) - m, torch.log(others)], 1) - torch.log(total)
    row_loss = T * T * torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
    w = s["weights"]
    scale = w / w.sum()
    out = dict(loss=(scale * row_loss).sum(), row_loss=row_loss)
    if case["grad"]:
        q = e / total
        q_rest = others / total
        ratio = torch.where(p[:, -1:] > 0, p[:, -1:] / q_rest, 0.0)
        grad = q * (1.0 - ratio)
        grad.scatter_(1, ids, q.gather(1, ids) - p[:, :-1])
        out["grad"] = (grad * (T * scale)[:, None]).to(s["logits"].dtype)
    return out


def _plain_sample(case, s):
    n, V = case["rows"], case["vocab"]
    vals, ids = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    greedy = s["T"] == 0
    T = torch.where(greedy, 1.0, s["T"]).double()[:, None]
    x = (vals.double() - vals[:, :1].double()) / T
    e = torch.exp(x)
    cum = torch.cumsum(e, 1)
    n_k = torch.full((n,), V, device=DEV)
    if s["top_k"] is not None:
        n_k = torch.where(s["top_k"] > 0, s["top_k"].long(), n_k)
    n_k = torch.where(greedy, 1, n_k)
    keep = n_k
    if s["top_p"] is not None:
        mass = cum.gather(1, n_k[:, None] - 1)
        n_p = (cum < s["top_p"].double()[:, None] * mass).sum(1) + 1
        keep = torch.where(s["top_p"] < 1, torch.minimum(keep, n_p), keep)
    if s["min_p"] is not None:
        keep = torch.minimum(keep, (e >= s["min_p"].double()[:, None]).sum(1))
    mass = cum.gather(1, keep[:, None] - 1)
    at = (cum <= s["u"].double()[:, None] * mass).sum(1)
    at = torch.minimum(at, keep - 1)[:, None]
    logprob = x.gather(1, at) - torch.log(mass)
    return dict(token=ids.gather(1, at)[:, 0].int(), logprob=logprob[:, 0].float())


# --------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------
def _held(case, s):
    """Outputs and workspace, as a program allocates them once and keeps them."""
    if "held" not in s:
        from paper_2605_29707_amd import binding as bd
        n, V = case["rows"], case["vocab"]
        f32 = lambda *shape: torch.empty(shape, device=DEV, dtype=torch.float32)  # noqa: E731
        i32 = lambda *shape: torch.empty(shape, device=DEV, dtype=torch.int32)  # noqa: E731
        if case["kind"] == "top":
            out = dict(ids=i32(n, case["k"]), vals=f32(n, case["k"]), rest=f32(n))
            need = bd.domino_top_logits_workspace_bytes(n, V, case["k"])
        elif case["kind"] == "distill":
            out = dict(loss=f32(1)[0], row_loss=f32(n))
            if case["grad"]:
                out["grad"] = torch.empty((n, V), device=DEV, dtype=s["logits"].dtype)
            need = bd.domino_distill_workspace_bytes(n, V, case["k"])
        else:
            out = dict(token=i32(n), logprob=f32(n))
            need = bd.domino_sample_logits_workspace_bytes(n, V)
        s["held"] = bd, out, torch.empty(need, device=DEV, dtype=torch.uint8)
    return s["held"]


def _own_run(case, s):
    bd, out, ws = _held(case, s)
    if case["kind"] == "top":
        bd.domino_top_logits(s["logits"], out["ids"], out["vals"], ws, rest=out["rest"], temperature=case["T"])
    elif case["kind"] == "distill":
        bd.domino_distill_loss(s["logits"], s["t_ids"], s["t_vals"], out["loss"], ws, teacher_rest=s.get("t_rest"),
                               temperature=case["T"], row_weights=s["weights"], row_loss=out["row_loss"],
                               grad=out.get("grad"))
    else:
        bd.domino_sample_logits(s["logits"], s["u"], out["token"], ws, temperature=s["T"], top_k=s["top_k"],
                                top_p=s["top_p"], min_p=s["min_p"], logprobs=out["logprob"])
    return out


def run(state):
    case = state["case"]
    if own:
        return _own_run(case, state)
    return dict(top=_plain_top, distill=_plain_distill, sample=_plain_sample)[case["kind"]](case, state)


def work(case):
    n, V = case["rows"], case["vocab"]
    size = n * V * (2 if case["dtype"] == "bf16" else 4)
    if case["kind"] == "top":
        return {"bytes": size + n * (8 * case["k"] + 4), "flops": 3 * n * V}
    if case["kind"] == "distill":
        entries = n * (8 * case["k"] + 12)
        return {"bytes": size * (2 if case["grad"] else 1) + entries, "flops": (6 if case["grad"] else 3) * n * V}
    return {"bytes": size + n * 28, "flops": 3 * n * V}


# --------------------------------------------------------------------------
# the same outputs in 64 bits
# --------------------------------------------------------------------------
def _exact_top(case, s):
    x = s["logits"].double()
    best = torch.topk(x, case["k"], dim=1).values
    # the others: below the last kept value, and what its ties leave over
    edge = best[:, -1:]
    below = torch.logsumexp(torch.where(x < edge, x, -math.inf) / case["T"], 1)
    over = (x == edge).sum(1) - (best == edge).sum(1)
    rest = torch.logaddexp(below, torch.log(over.double()) + edge[:, 0] / case["T"])
    return dict(ids=None, vals=best, rest=rest)


def _exact_distill(case, s):
    n, V, T = case["rows"], case["vocab"], case["T"]
    with torch.enable_grad():
        x = s["logits"].double().requires_grad_(case["grad"])
        log_q = torch.log_softmax(x / T, 1)
        inside = torch.zeros(n, V, dtype=torch.bool, device=DEV).scatter_(1, s["t_ids"].long(), True)
        kept = torch.gather(log_q, 1, s["t_ids"].long())
        t = s["t_vals"].double() / T
        if case["rest"] and case["k"] < V:
            kept = torch.cat([kept, torch.logsumexp(log_q.masked_fill(inside, -math.inf), 1, keepdim=True)], 1)
            t = torch.cat([t, s["t_rest"].double()[:, None]], 1)
        p = torch.softmax(t, 1)
        row_loss = T**2 * (p * (torch.log_softmax(t, 1) - kept)).sum(1)
        w = s["weights"].double()
        loss = (w * row_loss).sum() / w.sum()
        out = dict(loss=loss.detach(), row_loss=row_loss.detach())
        if case["grad"]:
            out["grad"] = torch.autograd.grad(loss, x)[0]
    return out


def _exact_sample(case, s):
    """Probabilities, filtered and divided by their sum again after each filter; the draw by the running sum."""
    x = s["logits"].double()
    greedy = s["T"] == 0
    prob = torch.softmax(x / torch.where(greedy, 1.0, s["T"]).double()[:, None], 1)
    prob, ids = torch.sort(prob, dim=1, descending=True, stable=True)
    rank = torch.arange(case["vocab"], device=DEV)[None, :]
    ratio = prob / prob[:, :1]
    if s["top_k"] is not None:
        prob = prob.masked_fill((rank >= s["top_k"][:, None]) & (s["top_k"] > 0)[:, None], 0.0)
    prob = prob.masked_fill((rank > 0) & greedy[:, None], 0.0)
    prob = prob / prob.sum(1, keepdim=True)
    kept = prob
    if s["top_p"] is not None:
        before = torch.cumsum(prob, 1) - prob
        kept = kept.masked_fill((before >= s["top_p"].double()[:, None]) & (s["top_p"] < 1)[:, None], 0.0)
    if s["min_p"] is not None:
        kept = kept.masked_fill(ratio < s["min_p"].double()[:, None], 0.0)
    kept = kept / kept.sum(1, keepdim=True)
    last = (kept > 0).sum(1) - 1
    at = torch.minimum((torch.cumsum(kept, 1) <= s["u"].double()[:, None]).sum(1), last)
    return dict(token=None, logprob=torch.log(kept.gather(1, at[:, None]))[:, 0])


def exact(case, seed):
    s = prepare(case, seed)
    return dict(top=_exact_top, distill=_exact_distill, sample=_exact_sample)[case["kind"]](case, s)
