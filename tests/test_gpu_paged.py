"""The operators on a paged cache against the oracle in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_helpers import log  # noqa: E402
from oracle import paged_oracle as po  # noqa: E402
from paged_helpers import DEV, DT, Pages, dev, half_step, i32, starts_of  # noqa: E402
from paper_2605_29707_amd import binding as bd  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24   # half a step of fp32


def tokens(n, heads, dh, dtype, seed, scale=1.0, pad=0):
    """[n, heads, dh] random rows, `pad` elements wider apart than they are."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, heads * dh + pad, generator=g) * scale).to(DT[dtype]).to(DEV)
    return x[:, :heads * dh].unflatten(1, (heads, dh))


def no_error(ws):
    assert bd.domino_workspace_error(ws) == 0


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,rot,layout,scaling,norm,order,page", [
    (128, 128, "half", "none", True, "slot", 16), (128, 64, "half", "linear", False, "head", 1),
    (128, 48, "pairs", "ntk", True, "slot", 8), (64, 64, "pairs", "yarn", False, "head", 32),
    (64, 16, "half", "yarn", True, "slot", 64), (64, 0, "half", "none", False, "slot", 16),
    (64, 0, "half", "none", True, "slot", 2)])
def test_append(dtype, dh, rot, layout, scaling, norm, order, page):
    lens, news = [37, 5, 1, 90, 64], [3, 5, 1, 0, 33]     # a whole sequence, a single token, a waiting sequence
    nq, nkv, dt = 6, 2, DT[dtype]
    c = Pages(lens, page=page, nkv=nkv, dh=dh, dtype=dtype, order=order, layers=3, weights=True, seed=rot)
    starts, n = starts_of(news), sum(news)
    rows = n + 4                                          # rows behind the last sequence
    x = tokens(rows, nq + 2 * nkv, dh, dtype, 7, pad=16)
    q, k, v = x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:]
    out = torch.full((rows, nq, dh), 7.0, dtype=dt, device=DEV)
    gains = [(1 + 0.2 * torch.randn(dh, generator=torch.Generator().manual_seed(s))).to(dt).to(DEV) if norm else None
             for s in (1, 2)]
    kinds = dict(none=bd.DOMINO_ROPE_NONE, linear=bd.DOMINO_ROPE_LINEAR, ntk=bd.DOMINO_ROPE_NTK, yarn=bd.DOMINO_ROPE_YARN)
    freq, scale = (bd.domino_rope_frequencies(rot, 1e4, kinds[scaling], 8.0, 4096, 32, 1) if rot else (np.zeros(0), 1.0))
    pos = np.random.RandomState(3).randint(0, 2_000_000, rows).astype(np.int32)
    pos[0] = 2**31 - 1
    old_k, old_v, old_w = c.copies()
    ws = c.workspace(bd.DOMINO_PAGED_WORKSPACE_BYTES)
    bd.domino_paged_append(c.cache, q, k, v, out, i32(starts), i32(lens), ws, layer=1, positions=i32(pos),
                           frequencies=dev(freq) if rot else None, rope_scale=scale, interleaved=layout == "pairs",
                           q_norm=gains[0], k_norm=gains[1], rms_eps=1e-5)
    no_error(ws)
    assert (out[n:] == 7.0).all()
    f64 = lambda t: t.float().cpu().numpy()  # noqa: E731
    # errors: an angle in turns is rounded to 2^-25 (2 pi 2^-25 of the operands), the sine and cosine by 2 steps each, the norm's
    # sum of up to 128 squares by 12 roundings (half of that in its root), and 8 products and sums; then the storage type's
    near = 2 * np.pi * 2.0 ** -25 + (4 + 6 + 8) * 2 * U
    rope = lambda t, g: po.rotate(f64(t)[:n], pos[:n], freq, scale, layout == "pairs", None if g is None else f64(g), 1e-5)  # noqa: E731
    want, size = rope(q, gains[0])
    assert (np.abs(f64(out)[:n] - want) <= half_step(dt) * np.abs(want) + 2 * near * size).all()
    want_k, size_k = rope(k, gains[1])
    got_k, got_v, got_w = c.copies()
    for b in range(len(lens)):
        p, r = po.cells(c.table, b, np.arange(lens[b] - news[b], lens[b]), page)
        span = slice(starts[b], starts[b + 1])
        assert (np.abs(got_k[1, p, r] - want_k[span]) <= half_step(dt) * np.abs(want_k[span]) + 2 * near * size_k[span]).all()
        assert (got_v[1, p, r] == f64(v)[span]).all() and (got_w[1, p, :, r] == 0).all()
        old_k[1, p, r], old_v[1, p, r], old_w[1, p, :, r] = got_k[1, p, r], got_v[1, p, r], 0
    for got, old in ((got_k, old_k), (got_v, old_v), (got_w, old_w)):   # nothing else is touched
        np.testing.assert_array_equal(got, old)


def test_append_in_place_without_positions():
    """q in its own place gives what q apart gives; a token without positions takes its slot."""
    c, d = (Pages([70, 9], page=4, nkv=2, dh=128, seed=2) for _ in range(2))
    x = tokens(40, 8, 128, "bf16", 3)
    q, k, v, starts, lens = x[:, :4], x[:, 4:6], x[:, 6:], i32([0, 35, 40]), i32([70, 9])
    freq = dev(bd.domino_rope_frequencies(128, 1e6)[0])
    out = torch.empty(40, 4, 128, dtype=torch.bfloat16, device=DEV)
    ws = c.workspace(16)
    bd.domino_paged_append(c.cache, q, k, v, out, starts, lens, ws, frequencies=freq, q_norm=k[0, 0].contiguous())
    slots = np.concatenate([np.arange(35, 70), np.arange(4, 9)])
    bd.domino_paged_append(d.cache, q, k, v, q, starts, lens, ws, positions=i32(slots), frequencies=freq,
                           q_norm=k[0, 0].contiguous())
    no_error(ws)
    assert torch.equal(out, q) and torch.equal(c.k.nan_to_num(), d.k.nan_to_num())


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def check_attention(c, q, news, lens, layer=0, scale=None, mask=None, max_new=None, max_len=None, accumulate=False, out=None,
                    tail=0, ws=None):
    """One call against the oracle.  Errors: a score's sum of d_h products and its factor are off by (d_h + 2) U of sum |q||k| scale,
    the base-2 argument and the exponential by 4 U of the largest score more, so a weight by e^(2 d) - 1, d their sum; the
    row's sums over n slots by n U at most; bf16 rounds the weights (half a step of |p v|) and the output."""
    starts, dt, dh = starts_of(news), q.dtype, c.dh
    n, nq = q.shape[:2]
    scale = dh ** -0.5 if scale is None else scale
    out = torch.full((n, nq, dh), 7.0, dtype=dt, device=DEV) if out is None else out
    lse = torch.full((n, nq), 7.0, device=DEV)
    old_k, old_v, old_w = c.copies()
    max_new, max_len = max_new or max(max(news), 1), max_len or max(lens)
    need = bd.domino_paged_attention_workspace_bytes(c.cache, n, nq, max_new, max_len, accumulate)
    ws = c.workspace(need) if ws is None else ws
    bd.domino_paged_attention(c.cache, q, out, i32(starts), i32(lens), max_new, max_len, ws, layer=layer, scale=scale, mask=mask,
                              lse=lse, accumulate=accumulate)
    no_error(ws)
    want, want_lse, given, size, spread = po.attention(q.float().cpu().numpy(), old_k, old_v, c.table, starts, lens, layer, scale,
                                                       None if mask is None else mask.reshape(-1, mask.shape[-1]).cpu().numpy())
    live = n - tail
    got, got_lse = out.float().cpu().numpy(), lse.cpu().numpy()
    assert (got[live:] == 7.0).all() and (got_lse[live:] == 7.0).all()
    got, got_lse, want, want_lse, size, spread = (x[:live] for x in (got, got_lse, want, want_lse, size, spread))
    step = half_step(dt) if dt == torch.bfloat16 else 0.0
    d = ((dh + 2) + 4 * 1.5) * U * size + 4 * U
    rel = np.expm1(2 * d) + (max(lens) + 32) * 2 * U
    tol = (rel + step)[..., None] * spread + half_step(dt) * np.abs(want) * (1 + step)
    far = np.abs(got - want) - tol
    assert (far <= 0).all(), (float(np.nanmax(far)), np.unravel_index(np.nanargmax(far), far.shape), np.isnan(got).sum())
    empty = want_lse == -np.inf
    assert (got_lse[empty] == -np.inf).all() and (got[empty] == 0).all()
    tol = (rel + 2 * U * (np.abs(want_lse) + 2))[~empty]
    assert (np.abs(got_lse[~empty] - want_lse[~empty]) <= tol).all()
    new_k, new_v, new_w = c.copies()
    np.testing.assert_array_equal(new_k, old_k)
    np.testing.assert_array_equal(new_v, old_v)
    if accumulate:
        worst = rel.max(initial=0) + 4 * U * (1 + np.abs(want_lse[~empty]).max(initial=0))
        for (b, h), p in given.items():
            pg, r = po.cells(c.table, b, np.arange(lens[b]), c.page)
            w = old_w[layer, pg, h, r] + p
            rows = news[b] * nq // c.nkv
            assert (np.abs(new_w[layer, pg, h, r] - w) <= worst * p + U * (2 * w + rows * p)).all(), (b, h)
            old_w[layer, pg, h, r] = new_w[layer, pg, h, r]
        np.testing.assert_array_equal(new_w, old_w)
    elif old_w is not None:
        np.testing.assert_array_equal(new_w, old_w)
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("most", [1, 3, 40])
def test_many_sequences(dtype, most):
    """More sequences than a wave has lanes, some of them waiting, the rows of all in one call."""
    rng = np.random.RandomState(most)
    news = rng.randint(0, most + 1, 150)
    news[[0, 63, 64, 65, 149]] = [0, most, 0, most, 1]
    lens = news + rng.randint(0, 90, 150)
    c = Pages(lens, page=4, nkv=2, dh=64, dtype=dtype, weights=True, seed=most)
    q = tokens(news.sum() + 2, 4, 64, dtype, 1, scale=2.0)
    check_attention(c, q, list(news), list(lens), accumulate=True, tail=2)
    # and their append
    x, out, ws = tokens(news.sum() + 2, 8, 64, dtype, 2), torch.zeros_like(q), c.workspace(16)
    old_k, old_v, old_w = c.copies()
    bd.domino_paged_append(c.cache, x[:, :4], x[:, 4:6], x[:, 6:], out, i32(starts_of(news)), i32(lens), ws)
    no_error(ws)
    assert torch.equal(out[:-2], x[:-2, :4]) and (out[-2:] == 0).all()
    for b, at in enumerate(starts_of(news)[:-1]):
        p, r = po.cells(c.table, b, np.arange(lens[b] - news[b], lens[b]), 4)
        old_k[0, p, r], old_v[0, p, r] = (x[at:at + news[b], s].float().cpu().numpy() for s in (slice(4, 6), slice(6, 8)))
        old_w[0, p, :, r] = 0
    for got, want in zip(c.copies(), (old_k, old_v, old_w)):
        np.testing.assert_array_equal(got, want)


def test_one_kv_head_for_many_query_heads():
    for news in ([1, 1], [3, 70]):
        c = Pages([90, 300], page=16, nkv=1, dh=128, weights=True)
        check_attention(c, tokens(sum(news), 160, 128, "bf16", 3), news, [90, 300], accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [3, 0, 1, 4], [70, 1, 2, 33]])
@pytest.mark.parametrize("nq,nkv", [(4, 1), (4, 4), (32, 1)])
def test_lengths_far_below_the_limit(dtype, news, nq, nkv):
    """max_len as a captured graph has it: sequences are a small part of it, and cut into other runs than the longest would be."""
    lens = [1100, 1, 129, 640]
    c = Pages(lens, page=16, nkv=nkv, dh=64, dtype=dtype, weights=True, seed=nkv, room=20000)
    q = tokens(sum(news), nq, 64, dtype, 2, scale=2.0)
    check_attention(c, q, news, lens, max_new=80, max_len=20000, accumulate=True)
    mask = (torch.rand(sum(news), 80, generator=torch.Generator().manual_seed(3)) < 0.4).to(torch.uint8)
    check_attention(c, q, news, lens, max_new=max(news), max_len=20000, accumulate=True, mask=mask.to(DEV))


def test_rows_before_the_first_sequence():
    c = Pages([40, 9], page=8, nkv=2, dh=64)
    x, ws = tokens(9, 8, 64, "bf16", 1), c.workspace(1 << 20)
    out = torch.full((9, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    bd.domino_paged_append(c.cache, x[:, :4], x[:, 4:6], x[:, 6:], out, i32([3, 5, 8]), i32([40, 9]), ws)
    assert torch.equal(out[3:8], x[3:8, :4]) and (out[:3] == 7).all() and (out[8:] == 7).all()
    att = torch.full((9, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    bd.domino_paged_attention(c.cache, out, att, i32([3, 5, 8]), i32([40, 9]), 3, 40, ws)
    no_error(ws)
    want = torch.empty(5, 4, 64, dtype=torch.bfloat16, device=DEV)
    bd.domino_paged_attention(c.cache, out[3:8], want, i32([0, 2, 5]), i32([40, 9]), 3, 40, ws)
    assert torch.equal(att[3:8], want) and (att[:3] == 7).all() and (att[8:] == 7).all()


def test_append_of_many_tokens():
    """From 1024 tokens on a workgroup has all heads of a token."""
    lens, news = [1500, 700], [1500, 33]
    c, d = (Pages(lens, page=64, nkv=2, dh=128, seed=1, weights=True) for _ in range(2))
    x = tokens(1533, 24, 128, "bf16", 1)
    freq = dev(bd.domino_rope_frequencies(128, 1e6)[0])
    outs = [torch.empty(1533, 20, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ws = c.workspace(16)
    bd.domino_paged_append(c.cache, x[:, :20], x[:, 20:22], x[:, 22:], outs[0], i32([0, 1500, 1533]), i32(lens), ws, frequencies=freq)
    for lo in range(0, 1533, 500):        # in pieces, with the positions of the whole
        hi = min(lo + 500, 1533)
        cut = [max(0, min(hi, 1500) - lo), max(0, hi - max(lo, 1500))]
        done = [min(hi, 1500), 667 + max(0, hi - 1500)]
        y = x[lo:hi]
        bd.domino_paged_append(d.cache, y[:, :20], y[:, 20:22], y[:, 22:], outs[1][lo:hi], i32(starts_of(cut)), i32(done), ws, frequencies=freq)
    no_error(ws)
    assert torch.equal(outs[0], outs[1])
    for a, b in ((c.k, d.k), (c.v, d.v), (c.w, d.w)):
        assert torch.equal(a.nan_to_num(), b.nan_to_num())


SHAPES = [  # lens, news, heads, kv heads, page
    ([1], [1], 1, 1, 1), ([1, 2, 3], [1, 2, 3], 4, 2, 1), ([33, 128, 129, 127], [1, 1, 1, 1], 8, 2, 16),
    ([40, 5, 300], [0, 5, 7], 6, 3, 8), ([257, 31], [16, 16], 16, 1, 32), ([700, 65, 64], [61, 33, 64], 8, 2, 64),
    ([1025], [1], 8, 8, 256), ([290, 513], [200, 129], 12, 4, 128), ([2300], [3], 40, 8, 16)]


@pytest.mark.parametrize("dtype,dh,order", [("bf16", 128, "slot"), ("bf16", 64, "head"), ("f32", 64, "slot"), ("f32", 128, "head")])
@pytest.mark.parametrize("lens,news,nq,nkv,page", SHAPES)
def test_attention(dtype, dh, order, lens, news, nq, nkv, page):
    c = Pages(lens, page=page, nkv=nkv, dh=dh, dtype=dtype, order=order, layers=2, weights=True, seed=len(lens))
    q = tokens(sum(news) + 3, nq, dh, dtype, 5, scale=2.0, pad=8 * dh)
    check_attention(c, q, news, lens, layer=1, tail=3, accumulate=True)


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("lens,news,nq,nkv,page", [
    ([16, 45, 3], [16, 16, 3], 8, 2, 4), ([61, 500], [61, 61], 8, 2, 32), ([7], [7], 2, 2, 1), ([150, 2], [130, 2], 4, 1, 16)])
def test_attention_masked(dtype, dh, lens, news, nq, nkv, page):
    """Any mask over the new tokens, with rows that see nothing (whole sequences' contexts among them)."""
    c = Pages(lens, page=page, nkv=nkv, dh=dh, dtype=dtype, weights=True, seed=1)
    n, wide = sum(news), max(news) + 3
    mask = (torch.rand(n, wide, generator=torch.Generator().manual_seed(2)) < 0.3).to(torch.uint8) * 3
    mask[::3] = 0
    mask[1] = 1
    check_attention(c, tokens(n, nq, dh, dtype, 6, scale=2.0), news, lens, mask=mask.to(DEV), accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx,new", [(0, 5), (3, 64), (130, 100)])
def test_what_is_hidden_may_be_anything(dtype, ctx, new):
    """NaN and infinities in keys and values of new tokens that a row does not see leave it as it is."""
    lens, news, nq, nkv, dh = [ctx + new], [new], 4, 2, 64
    c = Pages(lens, page=8, nkv=nkv, dh=dh, dtype=dtype, seed=4)
    q = tokens(new, nq, dh, dtype, 8)
    last = new // 2                     # rows before it do not see it
    for slot, kv, bad in ((ctx + last, c.v, float("nan")), (ctx + last + 1, c.k, float("inf")), (ctx + new - 1, c.v, -float("inf"))):
        kv[0, c.table[0, slot // 8], slot % 8] = bad
    out, _ = check_visible(c, q, news, lens, last)
    # ... and rows that see them are NaN
    assert torch.isnan(out[last:]).any(-1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("new", [3, 40])
def test_a_row_of_nan_gives_nothing_to_what_it_does_not_see(dtype, masked, new):
    """The weights of the slots that it sees become NaN, those of later tokens are what the other rows give."""
    c = Pages([50 + new], page=8, nkv=2, dh=64, dtype=dtype, weights=True, stale="", seed=new)
    q = tokens(new, 4, 64, dtype, 1)
    slots = np.arange(50 + new)
    pg, r = po.cells(c.table, 0, slots, 8)
    mask = torch.tril(torch.ones(new, new, dtype=torch.uint8)).to(DEV) if masked else None
    ws = c.workspace(bd.domino_paged_attention_workspace_bytes(c.cache, new, 4, new, 50 + new, True))
    starts, lens, out, got = i32([0, new]), i32([50 + new]), torch.empty_like(q), []
    for bad in (False, True):
        c.w.zero_()
        if bad:
            q[1] = float("nan")
        bd.domino_paged_attention(c.cache, q, out, starts, lens, new, 50 + new, ws, mask=mask, accumulate=True)
        no_error(ws)
        got.append(c.w[0].cpu().numpy()[pg, :, r])
    assert np.isnan(got[1][:52]).all() and np.array_equal(got[1][52:], got[0][52:])
    assert torch.isnan(out[1]).all() and not torch.isnan(out[[0, 2]]).any()


def check_visible(c, q, news, lens, rows):
    """The first `rows` rows of one sequence equal those of a call on a cache without the later tokens' values."""
    starts, dt = i32(starts_of(news)), q.dtype
    res = []
    for clean in (False, True):
        if clean:
            for s in range(lens[0] - news[0] + rows, lens[0]):
                c.k[0, c.table[0, s // c.page], s % c.page] = 0.25
                c.v[0, c.table[0, s // c.page], s % c.page] = 0.5
        out = torch.empty(q.shape, dtype=dt, device=DEV)
        lse = torch.empty(q.shape[:2], device=DEV)
        ws = c.workspace(bd.domino_paged_attention_workspace_bytes(c.cache, q.shape[0], q.shape[1], news[0], lens[0]))
        bd.domino_paged_attention(c.cache, q, out, starts, i32(lens), news[0], lens[0], ws, lse=lse)
        res.append((out, lse))
    assert torch.equal(res[0][0][:rows], res[1][0][:rows]) and torch.equal(res[0][1][:rows], res[1][1][:rows])
    return res[0]


# ---------------------------------------------------------------------------
# eviction and commit: whole rows move
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,dh,order,page", [("bf16", 128, "slot", 16), ("bf16", 64, "head", 1), ("f32", 128, "head", 8),
                                                  ("f32", 64, "slot", 64)])
@pytest.mark.parametrize("new_pages", [False, True])
@pytest.mark.parametrize("budget,sink,recent,values", [
    (40, 4, 8, "random"), (1, 0, 0, "random"), (64, 64, 0, "random"), (33, 0, 33, "few"), (50, 10, 40, "few"), (100, 3, 5, "few"),
    (300, 5, 100, "odd"), (1500, 0, 0, "zero"), (700, 0, 1, "random")])
def test_evict(dtype, dh, order, page, new_pages, budget, sink, recent, values):
    lens = [1, 33, 2000, 0, 100, 769, 64]
    c = Pages(lens, page=page, nkv=2, dh=dh, dtype=dtype, order=order, layers=2, weights=True, seed=budget, stale="", room=0,
              spare=7 * -(-budget // page) + 2)
    g = torch.Generator().manual_seed(9)
    if values == "few":      # many equal weights
        c.w.copy_(torch.randint(0, 3, c.w.shape, generator=g))
    elif values == "zero":
        c.w.zero_()
        c.w[torch.rand(c.w.shape, generator=g).to(DEV) < 0.5] = -0.0
    elif values == "odd":    # NaN, infinities, zeros of both signs and negative numbers
        pick = torch.randint(0, 8, c.w.shape, generator=g)
        odd = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, -1.5, 1e-40, 2.0])
        c.w.copy_(odd[pick])
    k, v, w = c.copies()
    new_table = None
    if new_pages:
        per = -(-budget // page)
        new_table = c.free[:7 * per].reshape(7, per).copy()
    want_lens, want_kept = po.evict(k, v, w, c.table, np.asarray(lens), budget, sink, recent, new_table)
    kept = torch.full((2, 7, 2, budget), 9, dtype=torch.int32, device=DEV)
    out = torch.zeros(7, dtype=torch.int32, device=DEV)
    ws = c.workspace(bd.domino_paged_evict_workspace_bytes(c.cache, 2000, budget))
    bd.domino_paged_evict(c.cache, i32(lens), out, 2000, budget, ws, sink=sink, recent=recent,
                          new_table=None if new_table is None else i32(new_table), kept=kept)
    no_error(ws)
    np.testing.assert_array_equal(out.cpu().numpy(), want_lens)
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    for got, want in zip(c.copies(), (k, v, w)):
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("page,values", [(1, "random"), (2, "few"), (64, "random"), (64, "one"), (512, "few")])
@pytest.mark.parametrize("new_pages", [False, True])
def test_evict_long(page, values, new_pages):
    """Sequences of more slots than one workgroup chooses from, beside short ones."""
    lens, budget, sink, recent = [16384, 16385, 50000, 700, 32768], 1003, 5, 300
    c = Pages(lens, page=page, nkv=2, dh=64, weights=True, stale="", spare=5 * -(-budget // page) + 2)
    g = torch.Generator().manual_seed(9)
    if values != "random":   # equal weights, over all slices or but for a few
        c.w.copy_(torch.randint(0, 4, c.w.shape, generator=g) if values == "few" else torch.ones(c.w.shape))
    k, v, w = c.copies()
    per = -(-budget // page)
    new_table = c.free[:5 * per].reshape(5, per).copy() if new_pages else None
    want_lens, want_kept = po.evict(k, v, w, c.table, np.asarray(lens), budget, sink, recent, new_table)
    kept = torch.full((1, 5, 2, budget), 9, dtype=torch.int32, device=DEV)
    out = torch.zeros(5, dtype=torch.int32, device=DEV)
    ws = c.workspace(bd.domino_paged_evict_workspace_bytes(c.cache, 50000, budget)).fill_(77)
    ws[:16] = 0
    for _ in range(1 if new_table is None else 2):   # (to new pages, the second call finds what the first did)
        bd.domino_paged_evict(c.cache, i32(lens), out, 50000, budget, ws, sink=sink, recent=recent,
                              new_table=None if new_table is None else i32(new_table), kept=kept)
    no_error(ws)
    np.testing.assert_array_equal(out.cpu().numpy(), want_lens)
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    for got, want in zip(c.copies(), (k, v, w)):
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
def test_evict_many_heads_in_place(dtype, dh):
    """More workgroups than where rows are cut into narrow slices, over several rounds."""
    lens, budget = [900, 33, 1700, 1300], 1201
    c = Pages(lens, page=16, nkv=8, dh=dh, dtype=dtype, layers=2, weights=True, stale="", seed=dh)
    k, v, w = c.copies()
    want_lens, want_kept = po.evict(k, v, w, c.table, np.asarray(lens), budget, 3, 77, None)
    kept, out = torch.full((2, 4, 8, budget), 9, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    ws = c.workspace(bd.domino_paged_evict_workspace_bytes(c.cache, 1700, budget))
    bd.domino_paged_evict(c.cache, i32(lens), out, 1700, budget, ws, sink=3, recent=77, kept=kept)
    no_error(ws)
    np.testing.assert_array_equal(out.cpu().numpy(), want_lens)
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    for got, want in zip(c.copies(), (k, v, w)):
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("values", ["random", "few"])
def test_evict_ten_slices(values):
    """More slices than a phase adds up at a time."""
    lens, budget = [150001, 1 << 17, 2000], 20001
    c = Pages(lens, page=256, nkv=1, dh=64, weights=True, stale="", seed=1)
    if values == "few":
        c.w.copy_(torch.randint(0, 3, c.w.shape, generator=torch.Generator().manual_seed(9)))
    k, v, w = c.copies()
    want_lens, want_kept = po.evict(k, v, w, c.table, np.asarray(lens), budget, 3, 777, None)
    kept, out = torch.full((1, 3, 1, budget), 9, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    ws = c.workspace(bd.domino_paged_evict_workspace_bytes(c.cache, 150001, budget)).fill_(77)
    ws[:16] = 0
    bd.domino_paged_evict(c.cache, i32(lens), out, 150001, budget, ws, sink=3, recent=777, kept=kept)
    no_error(ws)
    np.testing.assert_array_equal(out.cpu().numpy(), want_lens)
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    for got, want in zip(c.copies(), (k, v, w)):
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("dtype,dh,order,page,weights", [("bf16", 128, "slot", 16, True), ("bf16", 64, "head", 1, False),
                                                          ("f32", 128, "head", 32, True), ("f32", 64, "slot", 8, True)])
@pytest.mark.parametrize("nodes,depth", [(61, 15), (16, 15), (2, 1), (1024, 63)])
def test_commit(dtype, dh, order, page, weights, nodes, depth):
    lens = [0, 5, 130, 64]
    rng = np.random.RandomState(nodes)
    accept = [0, depth, min(depth, 3), depth // 2]
    path = np.full((4, depth), -1, np.int32)
    for b, a in enumerate(accept):    # ascending ids, the one at depth d at least d
        path[b, :a] = np.maximum(np.sort(rng.choice(np.arange(1, nodes), a, replace=False)), np.arange(1, a + 1))
    c = Pages(lens, page=page, nkv=3, dh=dh, dtype=dtype, order=order, layers=3, weights=weights, stale="", room=nodes)
    k, v, w = c.copies()
    want = po.commit(k, v, w, c.table, lens, accept, path)
    out, ws = torch.zeros(4, dtype=torch.int32, device=DEV), c.workspace(16)
    bd.domino_paged_commit(c.cache, nodes, i32(lens), i32(accept), i32(path), out, ws)
    no_error(ws)
    np.testing.assert_array_equal(out.cpu().numpy(), want)
    for got, old in zip(c.copies(), (k, v, w)):
        if old is not None:
            np.testing.assert_array_equal(got, old)
