"""The operators on a paged cache where a call can go wrong: lengths and pages that are out of range, captured graphs, other
streams, offsets past 32 bits, and a run of all of them as a server makes it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from oracle import paged_oracle as po  # noqa: E402
from paged_helpers import DEV, Pages, dev, i32, starts_of  # noqa: E402
from paper_2605_29707_amd import binding as bd  # noqa: E402
from test_gpu_paged import check_attention, no_error, tokens  # noqa: E402

pytestmark = pytest.mark.gpu


def attend(c, q, starts, lens, max_new, max_len, ws=None, **kw):
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    need = bd.domino_paged_attention_workspace_bytes(c.cache, q.shape[0], q.shape[1], max_new, max_len, kw.get("accumulate", False))
    ws = c.workspace(need) if ws is None else ws
    bd.domino_paged_attention(c.cache, q, out, i32(starts), i32(lens), max_new, max_len, ws, lse=lse, **kw)
    return out, lse, bd.domino_workspace_error(ws)


@pytest.mark.parametrize("starts,lens,bad", [
    ([0, 2, 4, 6], [40, 33, 41], [2]),       # longer than max_len
    ([0, 2, 4, 6], [40, 1, 30], [1]),        # fewer slots than new tokens
    ([0, 2, 4, 6], [-1, 33, 2**31 - 1], [0, 2]),
    ([0, 4, 2, 6], [40, 33, 30], [1, 2]),    # more than max_new; starts that go down
    ([-1, 2, 4, 6], [40, 33, 30], [0]),
    ([0, 2, 4, 2**31 - 1], [40, 33, 30], [2]),
])
def test_lengths_out_of_range(starts, lens, bad):
    """Such a sequence is left out and reported; the others are as they are alone."""
    c = Pages([40, 33, 30], page=8, nkv=2, dh=64, seed=3, weights=True)
    q = tokens(6, 4, 64, "bf16", 1)
    w = c.w.clone()
    out, lse, err = attend(c, q, starts, lens, 3, 40, accumulate=True)
    assert err == bd.DEV_BAD_CTX_LEN
    want, want_lse, e = attend(c, q, [0, 2, 4, 6], [40, 33, 30], 3, 40)
    assert e == 0
    for b in range(3):
        rows = slice(2 * b, 2 * b + 2)
        if b in bad:
            continue
        if starts[b:b + 2] == [2 * b, 2 * b + 2]:
            assert torch.equal(out[rows], want[rows]) and torch.equal(lse[rows], want_lse[rows])
    if bad == [2]:
        assert (out[4:] == 7.0).all() and (lse[4:] == 7.0).all()
        mine = c.table[2][c.table[2] >= 0]
        assert torch.equal(c.w[0, mine], w[0, mine])


def test_append_lengths_and_pages_out_of_range():
    c = Pages([40, 33, 30], page=8, nkv=2, dh=64, seed=3, weights=True)
    x = tokens(6, 8, 64, "bf16", 1)
    q, k, v, ws = x[:, :4], x[:, 4:6], x[:, 6:], c.workspace(16)
    out = torch.full((6, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    before = c.copies()
    room = c.table.shape[1] * 8
    bd.domino_paged_append(c.cache, q, k, v, out, i32([0, 2, 4, 6]), i32([1, room + 1, -5]), ws)
    assert bd.domino_workspace_error(ws) == bd.DEV_BAD_CTX_LEN and (out == 7.0).all()
    # lengths whose last page the table does not name: queries are written, no row is
    bd.domino_workspace_error(ws)
    ws.zero_()
    bd.domino_paged_append(c.cache, q, k, v, out, i32([0, 2, 2, 2]), i32([room, 33, 30]), ws)
    assert bd.domino_workspace_error(ws) == bd.DEV_BAD_PAGE and (out[:2] == q[:2]).all() and (out[2:] == 7.0).all()
    for got, old in zip(c.copies(), before):
        np.testing.assert_array_equal(got, old)


@pytest.mark.parametrize("page_id", [-1, -2**31, 2**31 - 1, "n_pages"])
@pytest.mark.parametrize("new", [1, 40])
def test_pages_out_of_range(page_id, new):
    """A bad table entry of one sequence is reported and changes nothing for the others."""
    c = Pages([70, 64], page=8, nkv=2, dh=128, seed=3, weights=True, stale="")
    q = tokens(new + 1, 4, 128, "bf16", 1)
    args = ([0, new, new + 1], [70, 64], new, 70)
    want, want_lse, err = attend(c, q, *args)
    assert err == 0
    table = c.table.copy()
    table[0, 3] = c.pages if page_id == "n_pages" else page_id
    c.cache = bd.PagedCache(c.k, c.v, i32(table), weights=c.w)
    before = c.copies()
    out, lse, err = attend(c, q, *args, accumulate=True)
    assert err == bd.DEV_BAD_PAGE and torch.equal(out[new:], want[new:]) and torch.equal(lse[new:], want_lse[new:])
    after = c.copies()
    for got, old in zip(after[:2], before[:2]):
        np.testing.assert_array_equal(got, old)
    used = np.unique(c.table[c.table >= 0])
    others = np.setdiff1d(np.arange(c.pages), np.setdiff1d(used, [c.table[0, 3]]))
    np.testing.assert_array_equal(after[2][0, others], before[2][0, others])   # also the page that was lost
    # eviction and commit
    for new_table in (None, c.free[:0]):
        kept, lens, ws = torch.zeros(1, 2, 2, 32, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV), None
        ws = c.workspace(bd.domino_paged_evict_workspace_bytes(c.cache, 70, 32))
        to = None if new_table is None else i32(np.full((2, 4), -1))
        state = c.copies()
        bd.domino_paged_evict(c.cache, i32([70, 20]), lens, 70, 32, ws, sink=30, recent=2, kept=kept, new_table=to)
        assert bd.domino_workspace_error(ws) == bd.DEV_BAD_PAGE and lens.tolist() == [32, 20]
        if to is not None:
            for got, old in zip(c.copies(), state):
                np.testing.assert_array_equal(got, old)
    state = c.copies()
    lens, ws = torch.zeros(2, dtype=torch.int32, device=DEV), c.workspace(16)
    bd.domino_paged_commit(c.cache, 10, i32([22, 60]), i32([2, 0]), i32([[3, 4], [-1, -1]]), lens, ws)
    assert bd.domino_workspace_error(ws) == bd.DEV_BAD_PAGE and lens.tolist() == [22, 61]
    for got, old in zip(c.copies(), state):
        np.testing.assert_array_equal(got, old)


@pytest.mark.parametrize("accept,path,err", [
    ([3, 1], [[1, 2, 1], [5, -1, -1]], bd.DEV_BAD_TREE), ([3, 1], [[1, 2, 16], [5, -1, -1]], bd.DEV_BAD_TREE),
    ([3, 1], [[0, 2, 5], [5, -1, -1]], bd.DEV_BAD_TREE), ([4, 1], [[4, 5, 6], [5, -1, -1]], bd.DEV_BAD_CTX_LEN),
    ([-1, 1], [[4, 5, 6], [5, -1, -1]], bd.DEV_BAD_CTX_LEN)])
def test_commit_of_bad_paths(accept, path, err):
    c = Pages([20, 9], page=4, nkv=2, dh=64, room=16, stale="", layers=2)
    k, v, _ = c.copies()
    lens, ws = torch.zeros(2, dtype=torch.int32, device=DEV), c.workspace(16)
    bd.domino_paged_commit(c.cache, 16, i32([20, 9]), i32(accept), i32(path), lens, ws)
    assert bd.domino_workspace_error(ws) == err and lens.tolist() == [20, 11]
    po.commit(k, v, None, c.table, [20, 9], [0, 1], path)
    for got, want in zip(c.copies(), (k, v)):
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("kw", [dict(lens=[-1, 50]), dict(lens=[51, 50])])
def test_evict_lengths_out_of_range(kw):
    c = Pages([50, 50], page=4, nkv=2, dh=64, stale="", weights=True)
    want = c.copies()
    kept, lens = torch.zeros(1, 2, 2, 8, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    ws = c.workspace(bd.domino_paged_evict_workspace_bytes(c.cache, 50, 8))
    bd.domino_paged_evict(c.cache, i32(kw["lens"]), lens, 50, 8, ws, recent=2, kept=kept)
    assert bd.domino_workspace_error(ws) == bd.DEV_BAD_CTX_LEN and lens.tolist() == [kw["lens"][0], 8]
    assert (kept[:, 0] == -1).all()
    mine = c.table[0][c.table[0] >= 0]
    for got, old in zip(c.copies(), want):
        np.testing.assert_array_equal(got[:, mine], old[:, mine])


def test_shared_pages_are_read():
    """Two sequences with one prefix."""
    c = Pages([64, 70], page=16, nkv=2, dh=64, seed=5)
    c.table[1, :4] = c.table[0, :4]
    c.cache = bd.PagedCache(c.k, c.v, i32(c.table))
    check_attention(c, tokens(2, 4, 64, "bf16", 3), [1, 1], [64, 70])


def test_offsets_past_32_bits():
    """A cache of more than 2^32 elements whose pages in use lie at its ends."""
    pages, page, nkv, dh = (1 << 32) // (64 * 8 * 128) + 40, 64, 8, 128
    k = torch.empty(1, pages, page, nkv, dh, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    ids = [pages - 1, 0, pages - 2, pages // 2]
    g = torch.Generator(device=DEV).manual_seed(1)
    for x in (k, v):
        for p in ids:
            x[0, p] = torch.randn(page, nkv, dh, generator=g, device=DEV)
    small = Pages([200], page=page, nkv=nkv, dh=dh, spare=0, stale="", weights=True)
    for at, p in enumerate(small.table[0, :4]):
        small.k[0, p], small.v[0, p] = k[0, ids[at]], v[0, ids[at]]
    big = Pages.__new__(Pages)
    big.k, big.v, big.w, big.cache = k, v, None, bd.PagedCache(k, v, i32([ids]))
    big.workspace = small.workspace
    for new in (1, 70):
        q = tokens(new, 16, dh, "bf16", new)
        got, want = attend(big, q, [0, new], [200], new, 200), attend(small, q, [0, new], [200], new, 200)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    x, out, ws = tokens(8, 32, dh, "bf16", 9), torch.empty(8, 16, dh, dtype=torch.bfloat16, device=DEV), small.workspace(16)
    for c in (big, small):
        bd.domino_paged_append(c.cache, x[:, :16], x[:, 16:24], x[:, 24:], out, i32([0, 8]), i32([200]), ws)
        bd.domino_paged_commit(c.cache, 16, i32([192]), i32([2]), i32([[5, 7]]), torch.zeros(1, dtype=torch.int32, device=DEV), ws)
    no_error(ws)
    for at, p in enumerate(small.table[0, :4]):
        assert torch.equal(small.k[0, p], k[0, ids[at]]) and torch.equal(small.v[0, p], v[0, ids[at]])


def test_far_apart_rows_of_queries():
    """Token strides that pass 32 bits in bytes."""
    n, nq, dh = 3, 4, 64
    flat = torch.empty(2 * (1 << 30) + (1 << 12), dtype=torch.bfloat16, device=DEV)
    q = flat.as_strided((n, nq, dh), (1 << 30, dh, 1))
    q.copy_(tokens(n, nq, dh, "bf16", 4))
    c = Pages([30], page=8, nkv=2, dh=dh, weights=True)
    check_attention(c, q, [3], [30], accumulate=True)


def step(c, x, out, q_out, starts, lens, ws, wide, freq, kept, new_lens):
    nq, nkv = out.shape[1], c.nkv
    bd.domino_paged_append(c.cache, x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:], q_out, starts, lens, ws, frequencies=freq)
    bd.domino_paged_attention(c.cache, q_out, out, starts, lens, x.shape[0], wide, ws, accumulate=True)
    bd.domino_paged_evict(c.cache, lens, new_lens, wide, 48, ws, sink=2, recent=16, kept=kept)


@pytest.mark.parametrize("new", [1, 33])
def test_captured_and_replayed(new):
    """Append, attention with accumulated weights and eviction in one graph, replayed with other inputs between eager steps."""
    lens = [120, 64]
    c, d = (Pages(lens, page=16, nkv=2, dh=64, weights=True, seed=8, stale="") for _ in range(2))
    n = 2 * new
    x = tokens(n, 8, 64, "bf16", 1).contiguous()
    wide = 120
    need = max(bd.domino_paged_attention_workspace_bytes(c.cache, n, 4, n, wide, True), bd.domino_paged_evict_workspace_bytes(c.cache, wide, 48))
    freq = dev(bd.domino_rope_frequencies(64, 1e4)[0])
    mk = lambda: dict(out=torch.zeros(n, 4, 64, dtype=torch.bfloat16, device=DEV), q_out=torch.zeros(n, 4, 64, dtype=torch.bfloat16, device=DEV),  # noqa: E731
                      starts=i32([0, new, n]), lens=i32(lens), ws=c.workspace(need), wide=wide, freq=freq,
                      kept=torch.zeros(1, 2, 2, 48, dtype=torch.int32, device=DEV), new_lens=i32([0, 0]))
    a, b = mk(), mk()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    saved = [t.clone() for t in (c.k, c.v, c.w)]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(c, x, **a)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        step(c, x, **a)
    for t, s in zip((c.k, c.v, c.w), saved):
        t.copy_(s)
    for i in range(4):
        x.copy_(tokens(n, 8, 64, "bf16", 10 + i))
        graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        step(d, x, **b)
        for s, t in ((c.k, d.k), (c.v, d.v), (c.w, d.w), (a["out"], b["out"]), (a["kept"], b["kept"]), (a["new_lens"], b["new_lens"])):
            assert torch.equal(s, t), i
    no_error(a["ws"])


def test_two_streams_at_once():
    """Calls over one cache on two streams, a workspace each."""
    c = Pages([900, 1500], page=16, nkv=2, dh=128, seed=2)
    q = [tokens(n, 8, 128, "bf16", n) for n in (2, 180)]
    args = [([0, 1, 2], [900, 1500], 1, 1500), ([0, 90, 180], [900, 1500], 90, 1500)]
    want = [attend(c, q[i], *args[i])[0] for i in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ws = [c.workspace(bd.domino_paged_attention_workspace_bytes(c.cache, len(q[i]), 8, args[i][2], 1500)) for i in range(2)]
    outs, ints = [[], []], [[i32(x) for x in a[:2]] for a in args]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            out = torch.zeros_like(q[i])
            streams[i].wait_stream(torch.cuda.current_stream())
            bd.domino_paged_attention(c.cache, q[i], out, *ints[i], args[i][2], 1500, ws[i], stream=streams[i])
            outs[i].append(out)
    torch.cuda.synchronize()
    for i in range(2):
        no_error(ws[i])
        assert all(torch.equal(o, want[i]) for o in outs[i])


def test_repeatable():
    c = Pages([3000, 17, 800], page=32, nkv=2, dh=128, seed=2, weights=True)
    q = tokens(120, 8, 128, "bf16", 3, scale=3.0)
    w0, first = c.w.clone(), None
    for _ in range(5):
        c.w.copy_(w0)
        out, lse, _ = attend(c, q, [0, 100, 110, 120], [3000, 17, 800], 100, 3000, accumulate=True)
        now = (out.clone(), lse.clone(), c.w.clone())
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_served_cycle(dtype):
    """A server's run over two users: prompts in chunks, then cycles of a drafted tree (domino_build_tree's) that is verified over the
    pages, accepted (domino_verify_accept) and committed, then eviction, and decoding on the shortened cache; every call against
    the oracle on the caches as the call before it left them."""
    page, nkv, nq, dh, room = 16, 2, 8, 64, 160
    c = Pages([0, 0], page=page, nkv=nkv, dh=dh, dtype=dtype, room=room, weights=True, stale="", seed=6)
    freq = dev(bd.domino_rope_frequencies(dh, 1e4)[0])
    ws = c.workspace(bd.domino_paged_attention_workspace_bytes(c.cache, 122, nq, 61, room, True))
    lens, pos, seed = np.zeros(2, int), np.zeros(2, int), 0

    def forward(news, mask=None, where=None, accumulate=True):
        nonlocal seed
        seed += 1
        x = tokens(sum(news), nq + 2 * nkv, dh, dtype, seed)
        q = torch.empty(sum(news), nq, dh, dtype=x.dtype, device=DEV)
        at = np.concatenate([p + np.arange(n) for p, n in zip(pos, news)]) if where is None else where
        full = lens + news
        bd.domino_paged_append(c.cache, x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:], q, i32(starts_of(news)), i32(full), ws,
                               positions=i32(at), frequencies=freq)
        check_attention(c, q, list(news), list(full), mask=mask, accumulate=accumulate, ws=ws, max_new=61, max_len=room)
        return full

    for news in ([30, 7], [21, 0], [1, 1]):           # the prompts
        lens = forward(news)
        pos = pos + news
    rng = np.random.RandomState(0)
    for cycle in range(3):
        beta, depth, V = 4, 15, 97
        ids, anchor = i32(rng.randint(0, V, (2, depth, beta))), i32(rng.randint(0, V, 2))
        nn = 1 + depth * beta
        tok, par, dep, npos = (torch.zeros(2, nn, dtype=torch.int32, device=DEV) for _ in range(4))
        anc = torch.zeros(2, nn, nn, dtype=torch.uint8, device=DEV)
        bd.domino_build_tree(ids, anchor, i32(pos), tok, par, dep, npos, ancestor_mask=anc)
        before = i32(lens)
        # (a tree's nodes leave no weights: most of them go)
        forward([nn, nn], mask=anc, where=npos.cpu().numpy().ravel(), accumulate=False)
        logits = torch.randn(2, nn, V, device=DEV)
        logits[0, 0, tok[0, 2]] = 99.0                # some node of each tree is accepted
        logits[1, 0, tok[1, 1]] = 99.0
        logits[1, 1, tok[1, 7]] = 99.0
        acc, nodes, toks = (torch.zeros(2, *s, dtype=torch.int32, device=DEV) for s in ((), (depth,), (depth + 1,)))
        vws = torch.empty(bd.domino_verify_workspace_bytes(2, nn, V), dtype=torch.uint8, device=DEV)
        bd.domino_verify_accept(tok, par, logits, 16, acc, nodes, toks, vws)
        k, v, w = c.copies()
        want = po.commit(k, v, w, c.table, lens, acc.cpu().numpy(), nodes.cpu().numpy())
        new = torch.zeros(2, dtype=torch.int32, device=DEV)
        bd.domino_paged_commit(c.cache, nn, before, acc, nodes, new, ws)
        np.testing.assert_array_equal(new.cpu().numpy(), want)
        assert (acc >= 1).all()
        for got, old in zip(c.copies(), (k, v, w)):
            np.testing.assert_array_equal(got, old)
        pos, lens = pos + 1 + acc.cpu().numpy(), want.astype(int)
    budget = 24
    k, v, w = c.copies()
    want, want_kept = po.evict(k, v, w, c.table, lens, budget, 2, 8)
    new, kept = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(1, 2, nkv, budget, dtype=torch.int32, device=DEV)
    bd.domino_paged_evict(c.cache, i32(lens), new, room, budget, ws, sink=2, recent=8, kept=kept)
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    np.testing.assert_array_equal(new.cpu().numpy(), want)
    for got, old in zip(c.copies(), (k, v, w)):
        np.testing.assert_array_equal(got, old)
    lens = want.astype(int)
    assert lens.max() == budget
    for _ in range(2):                                # slots are no positions any more
        lens = forward([1, 1])
        pos = pos + 1
    no_error(ws)
