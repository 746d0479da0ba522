"""The operators on a paged KV cache as timed cases: the append of new tokens with their
rotary positions, the attention of new tokens over the pages, eviction by accumulated
attention weight, and the commit of an accepted path.

With `own` false `run()` computes them in elementary torch operations, with `own` true by
the binding's entry points.  Keys, values and queries are normal numbers, queries wide
enough that a row's weights are peaked; a sequence's lengths follow from the case alone.
"""
import math

import torch

own = False
DEV = "cuda"
HEADS = ((4, 2), (8, 8), (12, 4), (16, 1), (32, 8), (40, 8), (64, 8))
PAGES = (1, 8, 16, 32, 64, 128, 256)
THETA = 1e6


def listed():
    base = dict(nq=32, nkv=8, dh=128, dtype="bf16", order="slot", ragged=False)
    return [
        # one interactive user's next token: the smallest call, launches count
        dict(base, name="append_one", kind="append", batch=1, new=1, ctx=1024, page=16, layout="half", rot=128, scaling="none",
             norm=True, weights=False),
        # chunks of several users' prompts far into a stretched context; neighbouring elements rotate, half of the head
        dict(base, name="append_chunks", kind="append", batch=5, new=4096, ctx=60000, page=64, layout="pairs", rot=64,
             scaling="yarn", norm=False, weights=True, order="head", ragged=True),
        # the tiny fp32 target's chain of 16 drafted tokens, for three users
        dict(base, name="attend_tiny_f32", kind="attend", batch=3, new=16, ctx=128, page=8, nq=4, nkv=2, dh=64, dtype="f32",
             tree=False, weights=False, ragged=True),
        # one interactive user's next token
        dict(base, name="attend_one", kind="attend", batch=1, new=1, ctx=1024, page=16, tree=False, weights=False),
        # a serving batch's next tokens at different lengths, their weights kept for eviction
        dict(base, name="attend_decode_bs64", kind="attend", batch=64, new=1, ctx=16384, page=64, tree=False, weights=True,
             ragged=True),
        # verification of trees of four candidates a depth; odd lengths
        dict(base, name="attend_trees", kind="attend", batch=7, new=61, ctx=3001, page=32, tree=True, weights=False,
             order="head", ragged=True),
        # a chunk of a long prompt
        dict(base, name="attend_chunk", kind="attend", batch=1, new=4096, ctx=12288, page=64, tree=False, weights=False),
        # one user's cache a little over its budget, in place
        dict(base, name="evict_in_place", kind="evict", batch=1, layers=5, ctx=1100, budget=1024, sink=4, recent=256, page=16,
             new_pages=False),
        # one long document of an odd length, to other pages (its own are shared with other users)
        dict(base, name="evict_long", kind="evict", batch=1, layers=2, ctx=100003, budget=8192, sink=4, recent=1024, page=64,
             new_pages=True),
        # a serving batch at different lengths, some of them under the budget
        dict(base, name="evict_batch", kind="evict", batch=16, layers=3, ctx=16384, budget=5000, sink=16, recent=512, page=32,
             new_pages=True, order="head", ragged=True),
        # one user's tree of two candidates a depth
        dict(base, name="commit_one", kind="commit", batch=1, layers=36, ctx=1024, branch=2, page=16),
        # a serving batch's trees of four
        dict(base, name="commit_bs32", kind="commit", batch=32, layers=36, ctx=500, branch=4, page=64, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "evict", "commit"])
    nq, nkv = rng.choice(HEADS)
    case = dict(kind=kind, nq=nq, nkv=nkv, dh=rng.choice([64, 128]), page=rng.choice(PAGES), dtype=rng.choice(["bf16", "bf16", "f32"]),
                order=rng.choice(["slot", "head"]), ragged=rng.random() < 0.7)
    if kind == "append":
        rot = rng.choice([0, 16, 32, 48, case["dh"]])
        return dict(case, batch=_log_int(rng, 1, 64), new=_log_int(rng, 1, 4096), ctx=_log_int(rng, 1, 100000), rot=rot,
                    layout=rng.choice(["half", "pairs"]), scaling=rng.choice(["none", "linear", "ntk", "yarn"]) if rot else "none",
                    norm=rng.random() < 0.5, weights=rng.random() < 0.5)
    if kind == "attend":
        new = 1 if rng.random() < 0.3 else _log_int(rng, 1, 4096)
        return dict(case, batch=_log_int(rng, 1, 64), new=new, ctx=_log_int(rng, 1, 32768), tree=new <= 64 and rng.random() < 0.4,
                    weights=rng.random() < 0.3)
    if kind == "evict":
        ctx = _log_int(rng, 64, 100000)
        budget = _log_int(rng, 16, min(ctx, 16384))
        sink = rng.randint(0, budget // 8)
        return dict(case, batch=_log_int(rng, 1, 32), layers=rng.randint(1, 5), ctx=ctx, budget=budget, sink=sink,
                    recent=rng.randint(0, (budget - sink) // 2), new_pages=rng.random() < 0.6)
    return dict(case, batch=_log_int(rng, 1, 32), layers=rng.randint(1, 36), ctx=_log_int(rng, 1, 2000), branch=rng.choice([1, 2, 4]))


def _room(case):
    """Bytes that the padded plain form of a case takes."""
    cells = case["batch"] * (case["ctx"] + case.get("new", 64)) * case["nkv"] * case["dh"] * case.get("layers", 1) * 8
    rows = case["batch"] * case["nq"] * case.get("new", 0) * (case["ctx"] + case.get("new", 0)) * 4 if case["kind"] == "attend" else 0
    return max(cells, rows)


def draw(rng):
    most = {c["kind"]: work(c) for c in listed() if c["name"] in ("append_chunks", "evict_batch", "commit_bs32")}
    most["attend"] = dict(bytes=max(work(c)["bytes"] for c in listed() if c["kind"] == "attend"),
                          flops=max(work(c)["flops"] for c in listed() if c["kind"] == "attend"))
    while True:
        case = _draw(rng)
        w = work(case)
        if all(w[k] <= most[case["kind"]][k] for k in w) and _room(case) <= 9e9:
            return case


# --------------------------------------------------------------------------
# lengths, from the case alone
# --------------------------------------------------------------------------
def _part(b, step):
    return (b * step) % 1.0


def _counts(case):
    """(cached tokens, new tokens) of every sequence: up to three quarters and nine tenths less where ragged; one sequence waits."""
    out = []
    for b in range(case["batch"]):
        ctx, new = case["ctx"], case.get("new", 0)
        if case["ragged"]:
            ctx -= int(0.75 * ctx * _part(b, 0.618034))
            new = 0 if b == 3 and new else max(min(new, 1), new - int(0.9 * new * _part(b, 0.414214)))
        out.append((ctx, new))
    return out


def _nodes(case):
    return 1 + 15 * case["branch"]


def _depths(case):
    return [(7 * b + 5) % 16 for b in range(case["batch"])]


# --------------------------------------------------------------------------
# inputs, from the seed alone
# --------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 4099 + stream)
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _table(g, lens, page, most, pages):
    """A table [batch, most] of random pages for sequences of these lengths, -1 where there is none; the pages used."""
    order = torch.randperm(pages, generator=g, device=DEV).int()
    need = [-(-n // page) for n in lens]
    table, at = torch.full((len(lens), most), -1, dtype=torch.int32, device=DEV), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def _pages(case, g, layers, pages):
    """Keys or values of all pages as [layers, pages, page, nkv, dh], stored by slots or by heads."""
    a, b = (case["page"], case["nkv"]) if case["order"] == "slot" else (case["nkv"], case["page"])
    x = torch.empty((layers, pages, a, b, case["dh"]), dtype=_dtype(case), device=DEV)
    for layer in range(layers):
        x[layer] = torch.randn((pages, a, b, case["dh"]), generator=g, device=DEV)
    return x if case["order"] == "slot" else x.transpose(2, 3)


def _tree_mask(new):
    """Which nodes each node of a tree of four candidates a depth sees: itself and its ancestors, the first of every depth above."""
    i = torch.arange(new, device=DEV)
    depth = (i + 3) // 4
    first = torch.where(i > 0, 1 + 4 * (depth - 1), 0)
    return ((first[None, :] == i[None, :]) & (depth[None, :] < depth[:, None])) | (i[None, :] == i[:, None])


def prepare(case, seed):
    g = _gen(seed, 1)
    counts, page, layers, dt = _counts(case), case["page"], case.get("layers", 1), _dtype(case)
    extra = _nodes(case) if case["kind"] == "commit" else 0
    lens = [c + n + extra for c, n in counts]
    used = sum(-(-n // page) for n in lens)
    kept = -(-case.get("budget", 0) // page) * case["batch"] if case.get("new_pages") else 0
    pages = used + kept + max(2, used // 16)
    most = max(-(-n // page) for n in lens) + 3
    table = _table(g, lens + [kept * page], page, max(most, kept), pages)
    s = dict(case=case, table=table[:-1, :most].contiguous())
    if kept:
        s["new_table"] = table[-1, :kept].reshape(case["batch"], -1).contiguous()
    s["k"], s["v"] = _pages(case, g, layers, pages), _pages(case, g, layers, pages)
    s["max_len"], s["lens"] = max(lens), _i32([n for n in lens] if not extra else [c for c, _ in counts])
    if case.get("weights") or case["kind"] == "evict":
        # what many steps of a peaked softmax leave: a heavy tail, and nothing at all at many slots
        w = torch.exp(2.0 * torch.randn((layers, pages, case["nkv"], page), generator=g, device=DEV) - 2.0)
        s["w"] = torch.where(torch.rand(w.shape, generator=g, device=DEV) < 0.1, 0.0, w)
    if case["kind"] in ("append", "attend"):
        tokens, starts = sum(n for _, n in counts), [0]
        for _, n in counts:
            starts.append(starts[-1] + n)
        s["starts"], s["max_new"] = _i32(starts), max(n for _, n in counts)
        width = case["nq"] + 2 * case["nkv"]
        x = torch.randn((tokens, width, case["dh"]), generator=g, device=DEV)   # a projection's rows: q, k and v side by side
        if case["kind"] == "attend":
            x *= 2.5
        x = x.to(dt)
        s["q"], s["kn"], s["vn"] = x[:, :case["nq"]], x[:, case["nq"]:case["nq"] + case["nkv"]], x[:, case["nq"] + case["nkv"]:]
    if case["kind"] == "append":
        s["q_norm"] = s["k_norm"] = None
        if case["norm"]:
            s["q_norm"], s["k_norm"] = ((1.0 + 0.1 * torch.randn(case["dh"], generator=g, device=DEV)).to(dt) for _ in range(2))
    if case["kind"] == "attend" and case["tree"]:
        s["mask"] = torch.cat([_tree_mask(case["new"])[:n] for _, n in counts]).to(torch.uint8).contiguous()
    if case["kind"] == "commit":
        rank = torch.randint(0, case["branch"], (case["batch"], 15), generator=g, device=DEV)
        node = 1 + torch.arange(15, device=DEV) * case["branch"] + rank
        s["accept"] = _i32(_depths(case))
        s["path"] = torch.where(torch.arange(15, device=DEV) < s["accept"][:, None], node, -1).int().contiguous()
    return s


# --------------------------------------------------------------------------
# plain forms: elementary operations, in 32 bits; angles in 64
# --------------------------------------------------------------------------
def _frequencies(case):
    """The angle a position of each rotated pair, and the factor on the rotated elements."""
    rot, factor, first = case["rot"], 4.0, 16384
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    theta = THETA * factor ** (rot / (rot - 2)) if case["scaling"] == "ntk" else THETA
    f = theta ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "yarn":
        turns = first * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _sequence_of(s, tokens):
    """(sequence, place among its new ones, slot) of every new token."""
    t = torch.arange(tokens, device=DEV)
    starts, lens = s["starts"].long(), s["lens"].long()
    b = (starts[None, 1:] <= t[:, None]).sum(1)
    at = t - starts[b]
    return b, at, lens[b] - (starts[b + 1] - starts[b]) + at


def _plain_rotate(case, x, gain, cos, sin):
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain.float()
    rot = case["rot"]
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if case["layout"] == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([u, v], -1) if case["layout"] == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_append(case, s):
    b, _, slot = _sequence_of(s, s["q"].shape[0])
    cos = sin = torch.zeros((1, 1, 0), device=DEV)
    if case["rot"]:
        f, scale = _frequencies(case)
        angle = slot.double()[:, None, None] * f
        cos, sin = (torch.cos(angle) * scale).float(), (torch.sin(angle) * scale).float()
    page, at = s["table"].long()[b, slot // case["page"]], slot % case["page"]
    dt = _dtype(case)
    q = _plain_rotate(case, s["q"], s["q_norm"], cos, sin).to(dt)
    s["k"][0][page, at] = _plain_rotate(case, s["kn"], s["k_norm"], cos, sin).to(dt)
    s["v"][0][page, at] = s["vn"]
    out = dict(q=q, k=s["k"], v=s["v"])
    if case["weights"]:
        s["w"][0][page, :, at] = 0.0
        out["w"] = s["w"]
    return out


def _plain_attend(case, s):
    lens, most, new = s["lens"].long(), s["max_len"], s["max_new"]
    batch, nq, nkv, dh = case["batch"], case["nq"], case["nkv"], case["dh"]
    b, at, _ = _sequence_of(s, s["q"].shape[0])
    slots = torch.arange(most, device=DEV)
    page, off = s["table"].long()[:, slots // case["page"]], slots % case["page"]
    k = s["k"][0][page, off].float().permute(0, 2, 3, 1).contiguous()     # [batch, nkv, dh, most]
    v = s["v"][0][page, off].float().permute(0, 2, 1, 3).contiguous()
    q = torch.zeros((batch, nkv, new, nq // nkv, dh), device=DEV)
    q[b, :, at] = s["q"].float().reshape(-1, nkv, nq // nkv, dh)
    score = torch.matmul(q.reshape(batch, nkv, -1, dh), k) * (dh ** -0.5)
    count = s["starts"].long().diff()
    place = slots[None, :] - (lens - count)[:, None]                        # among the new tokens, negative in the context
    if case["tree"]:
        rows = torch.zeros((batch, new, new), dtype=torch.bool, device=DEV)
        rows[b, at] = s["mask"].bool()[:, :new]
        seen = rows.gather(2, place.clamp(0, new - 1)[:, None, :].expand(batch, new, most)) | (place < 0)[:, None, :]
    else:
        seen = place[:, None, :] <= torch.arange(new, device=DEV)[None, :, None]
    seen = seen & (slots[None, None, :] < lens[:, None, None])
    score = score.view(batch, nkv, new, nq // nkv, most).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score.sub_(torch.where(top == -math.inf, 0.0, top)))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(batch, nkv, -1, most), v).view(batch, nkv, new, nq // nkv, dh) / total
    lse = (top + torch.log(total))[..., 0]
    out = dict(out=o[b, :, at].reshape(-1, nq, dh).to(_dtype(case)), lse=lse[b, :, at].reshape(-1, nq))
    if case["weights"]:
        alive = torch.arange(new, device=DEV)[None, :] < count[:, None]
        p = torch.where(alive[:, None, :, None, None], p / total, 0.0).sum((2, 3))   # [batch, nkv, most]
        head = torch.arange(nkv, device=DEV)[None, None, :]
        s["w"][0].index_put_((page[:, :, None], head, off[None, :, None]), p.transpose(1, 2), accumulate=True)
        out["w"] = s["w"]
    return out


def _plain_evict(case, s):
    layers, batch, nkv, most, budget = case["layers"], case["batch"], case["nkv"], s["max_len"], case["budget"]
    lens = s["lens"].long()[None, :, None, None]
    layer = torch.arange(layers, device=DEV)[:, None, None, None]
    seq = torch.arange(batch, device=DEV)[None, :, None, None]
    head = torch.arange(nkv, device=DEV)[None, None, :, None]
    slots = torch.arange(most, device=DEV)
    table = s["table"].long()
    w = s["w"][layer, table[:, slots // case["page"]][None, :, None, :], head, slots % case["page"]]
    always = (slots < case["sink"]) | (slots >= lens - case["recent"]) | (lens <= budget)
    free = ~always & (slots < lens)
    order = torch.sort(torch.where(free, w, -1.0), dim=-1, descending=True, stable=True).indices
    best = torch.zeros(w.shape, dtype=torch.bool, device=DEV).scatter_(-1, order[..., :budget - case["sink"] - case["recent"]], True)
    keep = (always | (best & free)) & (slots < lens)
    kept = torch.sort(torch.where(keep, slots, most), dim=-1).values[..., :budget]
    kept = torch.cat([kept, torch.full(kept.shape[:3] + (budget - kept.shape[3],), most, device=DEV)], -1)
    live = kept < most
    # what lies past the kept ones writes slot 0's row once more, to slot 0
    src = torch.where(live, kept, kept[..., :1])
    dst = torch.where(live, torch.arange(budget, device=DEV), 0)
    to = s["new_table"].long() if case["new_pages"] else table
    to, at = to[seq, dst // case["page"]], dst % case["page"]
    page, off = table[seq, src // case["page"]], src % case["page"]
    s["k"][layer, to, at, head] = s["k"][layer, page, off, head]
    s["v"][layer, to, at, head] = s["v"][layer, page, off, head]
    s["w"][layer, to, head, at] = s["w"][layer, page, head, off]
    return dict(lens=torch.clamp(s["lens"], max=budget), kept=torch.where(live, kept, -1).int(), k=s["k"], v=s["v"], w=s["w"])


def _plain_commit(case, s):
    seq = torch.arange(case["batch"], device=DEV)[:, None]
    lens, path = s["lens"].long()[:, None], s["path"].long()
    to = lens + 1 + torch.arange(15, device=DEV)
    src = torch.where(path > 0, lens + path, to)
    table = s["table"].long()
    page, off = table[seq, src // case["page"]], src % case["page"]
    dst, at = table[seq, to // case["page"]], to % case["page"]
    s["k"][:, dst, at] = s["k"][:, page, off]
    s["v"][:, dst, at] = s["v"][:, page, off]
    return dict(lens=s["lens"] + 1 + s["accept"], k=s["k"], v=s["v"])


# --------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------
def _held(case, s):
    """Cache handle, outputs, workspace and table of angles, as a program makes them once and keeps them."""
    if "held" not in s:
        from paper_2605_29707_amd import binding as bd
        cache = bd.PagedCache(s["k"], s["v"], s["table"], weights=s.get("w"))
        need, out, more = bd.DOMINO_PAGED_WORKSPACE_BYTES, {}, {}
        if case["kind"] == "append":
            out["q"] = torch.empty(s["q"].shape, dtype=_dtype(case), device=DEV)
            if case["rot"]:
                scaling = dict(none=bd.DOMINO_ROPE_NONE, linear=bd.DOMINO_ROPE_LINEAR, ntk=bd.DOMINO_ROPE_NTK, yarn=bd.DOMINO_ROPE_YARN)
                f, more["rope_scale"] = bd.domino_rope_frequencies(case["rot"], THETA, scaling[case["scaling"]], factor=4.0,
                                                                   original_ctx=16384, beta_fast=32.0, beta_slow=1.0)
                more["frequencies"] = torch.from_numpy(f).to(DEV)
                more["interleaved"] = case["layout"] == "pairs"
        elif case["kind"] == "attend":
            out["out"] = torch.empty(s["q"].shape, dtype=_dtype(case), device=DEV)
            out["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
            need = bd.domino_paged_attention_workspace_bytes(cache, s["q"].shape[0], case["nq"], s["max_new"], s["max_len"],
                                                             accumulate=case["weights"])
        else:
            out["lens"] = torch.empty_like(s["lens"])
            if case["kind"] == "evict":
                out["kept"] = torch.empty((case["layers"], case["batch"], case["nkv"], case["budget"]), dtype=torch.int32, device=DEV)
                need = bd.domino_paged_evict_workspace_bytes(cache, s["max_len"], case["budget"])
        out.update(k=s["k"], v=s["v"]) if case["kind"] != "attend" else None
        if "w" in s:
            out["w"] = s["w"]
        s["held"] = bd, cache, out, torch.zeros(need, device=DEV, dtype=torch.uint8), more
    return s["held"]


def _own_run(case, s):
    bd, cache, out, ws, more = _held(case, s)
    if case["kind"] == "append":
        bd.domino_paged_append(cache, s["q"], s["kn"], s["vn"], out["q"], s["starts"], s["lens"], ws, q_norm=s["q_norm"],
                               k_norm=s["k_norm"], **more)
    elif case["kind"] == "attend":
        bd.domino_paged_attention(cache, s["q"], out["out"], s["starts"], s["lens"], s["max_new"], s["max_len"], ws, mask=s.get("mask"),
                                  lse=out["lse"], accumulate=case["weights"])
    elif case["kind"] == "evict":
        bd.domino_paged_evict(cache, s["lens"], out["lens"], s["max_len"], case["budget"], ws, sink=case["sink"], recent=case["recent"],
                              new_table=s.get("new_table"), kept=out["kept"])
    else:
        bd.domino_paged_commit(cache, _nodes(case), s["lens"], s["accept"], s["path"], out["lens"], ws)
    return out


def run(state):
    case = state["case"]
    if own:
        return _own_run(case, state)
    return dict(append=_plain_append, attend=_plain_attend, evict=_plain_evict, commit=_plain_commit)[case["kind"]](case, state)


def work(case):
    size, counts, row = (2 if case["dtype"] == "bf16" else 4), _counts(case), case["nkv"] * case["dh"]
    if case["kind"] == "append":
        tokens = sum(n for _, n in counts)
        values = tokens * (case["nq"] + 2 * case["nkv"]) * case["dh"]
        return {"bytes": 2 * size * values + (4 * tokens * case["nkv"] if case["weights"] else 0), "flops": 6 * values}
    if case["kind"] == "attend":
        tokens, slots = sum(n for _, n in counts), sum(c + n for c, n in counts if n)
        pairs = sum(n * c + (n * (n + 1) // 2 if not case["tree"] else sum(1 + (i + 3) // 4 for i in range(n))) for c, n in counts)
        return {"bytes": 2 * size * (slots * row + tokens * case["nq"] * case["dh"]) + 4 * tokens * case["nq"]
                + (8 * slots * case["nkv"] if case["weights"] else 0), "flops": 4 * pairs * case["nq"] * case["dh"]}
    if case["kind"] == "evict":
        kept = sum(min(c, case["budget"]) for c, _ in counts)
        slots = sum(c for c, _ in counts if c > case["budget"])
        if not case["new_pages"]:     # in place only the rows behind the first that goes are moved: all but the first `sink`, about
            kept = sum(case["budget"] - case["sink"] for c, _ in counts if c > case["budget"])
        return {"bytes": case["layers"] * case["nkv"] * (4 * slots + kept * (4 * case["dh"] * size + 12)) + 1,
                "flops": case["layers"] * case["nkv"] * slots}
    moved = sum(_depths(case)) if case["branch"] > 1 else 0
    return {"bytes": case["layers"] * moved * row * size * 4 + case["batch"] * 72, "flops": 0}


# --------------------------------------------------------------------------
# the same outputs in 64 bits, one sequence after another
# --------------------------------------------------------------------------
def _cells(s, b, first, last):
    """(pages, offsets) of a sequence's slots first..last-1."""
    n = torch.arange(first, last, device=DEV)
    size = s["case"]["page"]
    return s["table"][b].long()[torch.div(n, size, rounding_mode="floor")], torch.remainder(n, size)


def _exact_append(case, s):
    q, k, v = s["q"].double().clone(), s["kn"].double().clone(), s["vn"].double()
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    kc, vc = s["k"].double(), s["v"].double()
    wc = s["w"].double() if case["weights"] else None
    rot, half = case["rot"], case["rot"] // 2
    for x, gain in ((q, s["q_norm"]), (k, s["k_norm"])):
        if gain is not None:
            x /= torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / case["dh"] + 1e-6)
            x *= gain.double()
    # every pair as one complex number, turned by exp(i angle)
    if rot:
        i = torch.arange(half, dtype=torch.float64, device=DEV)
        factor, scale = 4.0, 1.0
        f = torch.exp(-2.0 * i / rot * math.log(THETA * (factor ** (rot / (rot - 2)) if case["scaling"] == "ntk" else 1.0)))
        if case["scaling"] == "linear":
            f /= factor
        elif case["scaling"] == "yarn":
            turns, scale = 16384 * f / math.tau, 0.1 * math.log(factor) + 1.0
            mix = torch.where(turns > 32, 1.0, torch.where(turns < 1, 0.0, (turns - 1) / 31))
            f = f * (mix + (1 - mix) / factor)
    for b in range(case["batch"]):
        lo, hi, n = starts[b], starts[b + 1], lens[b]
        if lo == hi:
            continue
        if rot:
            turn = torch.polar(torch.full((hi - lo, half), scale, dtype=torch.float64, device=DEV),
                               torch.outer(torch.arange(n - (hi - lo), n, dtype=torch.float64, device=DEV), f))[:, None]
            first, second = (slice(0, half), slice(half, rot)) if case["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
            for x in (q, k):
                z = torch.complex(x[lo:hi, :, first].contiguous(), x[lo:hi, :, second].contiguous()) * turn
                x[lo:hi, :, first], x[lo:hi, :, second] = z.real, z.imag
        page, at = _cells(s, b, n - (hi - lo), n)
        kc[0, page, at], vc[0, page, at] = k[lo:hi], v[lo:hi]
        if wc is not None:
            wc[0, page, :, at] = 0.0
    return dict(q=q, k=kc, v=vc, **({} if wc is None else dict(w=wc)))


def _exact_attend(case, s):
    starts, lens, group = s["starts"].tolist(), s["lens"].tolist(), case["nq"] // case["nkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    w = s["w"].double() if case["weights"] else None
    for b in range(case["batch"]):
        lo, hi, n = starts[b], starts[b + 1], lens[b]
        if lo == hi:
            continue
        new = hi - lo
        page, at = _cells(s, b, 0, n)
        hidden = torch.zeros((new, n), dtype=torch.bool, device=DEV)
        hidden[:, n - new:] = ~s["mask"][lo:hi, :new].bool() if case["tree"] else torch.ones(new, new, device=DEV).triu(1).bool()
        for h in range(case["nkv"]):
            k, v = s["k"][0, page, at, h].double(), s["v"][0, page, at, h].double()
            for j in range(h * group, (h + 1) * group):
                score = (s["q"][lo:hi, j].double() @ k.t() / math.sqrt(case["dh"])).masked_fill(hidden, -math.inf)
                lse[lo:hi, j] = torch.logsumexp(score, 1)
                p = torch.softmax(score, 1)
                out[lo:hi, j] = p @ v
                if w is not None:
                    w[0, page, h, at] += p.sum(0)
    return dict(out=out, lse=lse, **({} if w is None else dict(w=w)))


def _exact_evict(case, s):
    k, v, w = s["k"].double(), s["v"].double(), s["w"].double()
    lens, budget, sink, recent = s["lens"].tolist(), case["budget"], case["sink"], case["recent"]
    for b, n in enumerate(lens):
        m = min(n, budget)
        page, at = _cells(s, b, 0, n)
        to = dict(s, table=s["new_table"]) if case["new_pages"] else s
        dst, off = _cells(to, b, 0, m)
        for layer in range(case["layers"]):
            for h in range(case["nkv"]):
                keep = torch.arange(n, device=DEV)
                if n > budget:
                    # by (weight desc, slot asc): the slots of equal weight counted from the left
                    mid = s["w"][layer, page, h, at][sink:n - recent].double()
                    take = budget - sink - recent
                    edge = torch.topk(mid, take).values[-1] if take else math.inf
                    ties = mid == edge
                    chosen = (mid > edge) | (ties & (torch.cumsum(ties, 0) <= take - (mid > edge).sum()))
                    keep = torch.cat([keep[:sink], sink + chosen.nonzero()[:, 0], keep[n - recent:]])
                k[layer, dst, off, h] = s["k"][layer, page[keep], at[keep], h].double()
                v[layer, dst, off, h] = s["v"][layer, page[keep], at[keep], h].double()
                w[layer, dst, h, off] = s["w"][layer, page[keep], h, at[keep]].double()
    return dict(lens=None, kept=None, k=k, v=v, w=w)


def _exact_commit(case, s):
    k, v = s["k"].double(), s["v"].double()
    for b, (n, a) in enumerate(zip(s["lens"].tolist(), s["accept"].tolist())):
        page, at = _cells(s, b, n, n + _nodes(case))
        node = s["path"][b, :a].long()
        k[:, page[1:a + 1], at[1:a + 1]] = s["k"][:, page[node], at[node]].double()
        v[:, page[1:a + 1], at[1:a + 1]] = s["v"][:, page[node], at[node]].double()
    return dict(lens=None, k=k, v=v)


def exact(case, seed):
    s = prepare(case, seed)
    return dict(append=_exact_append, attend=_exact_attend, evict=_exact_evict, commit=_exact_commit)[case["kind"]](case, s)
