"""Calls of the operators on a paged cache that are refused before any HIP call, and what the host launches; needs no GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import host_stub
from oracle import paged_oracle as po
from paper_2605_29707_amd import binding as bd

P = 4096  # never dereferenced: validation fails first
INV, WS, UNS = bd.DOMINO_ERR_INVALID_ARG, bd.DOMINO_ERR_WORKSPACE, bd.DOMINO_ERR_UNSUPPORTED
BIG = 1 << 50


def cache(**kw):
    c = dict(k=P, v=P, weights=P, page_table=P, layer_stride=1 << 20, page_stride=16 * 2 * 64, slot_stride=128, head_stride=64,
             n_layers=2, n_pages=9, page_size=16, n_kv_heads=2, head_dim=64, batch=3, max_pages=4, dtype=1)
    c.update(kw)
    return bd.domino_paged_cache(**c)


APPEND = dict(layer=0, tokens=5, nq=4, q=P, ldq=512, k=P, ldk=512, v=P, ldv=512, out=P + 8192, ldo=256, starts=P, lens=P, pos=None,
              freq=P, rot=64, inter=0, scale=1.0, qn=None, kn=None, eps=1e-6, ws=P, n=BIG, st=None)
ATTEND = dict(layer=0, tokens=5, nq=4, max_new=3, max_len=64, q=P, ldq=512, out=P + 8192, ldo=256, starts=P, lens=P, scale=0.1,
              mask=None, ldm=0, lse=None, acc=0, ws=P, n=BIG, st=None)
EVICT = dict(lens=P, new=P + 64, max_len=64, budget=32, sink=4, recent=8, table=None, pages=0, kept=None, ws=P, n=BIG, st=None)
COMMIT = dict(nodes=16, depth=15, lens=P, acc=P, path=P, new=P + 64, ws=P, n=BIG, st=None)
CACHE = [(dict(k=None), INV), (dict(v=None), INV), (dict(page_table=None), INV), (dict(n_layers=0), INV), (dict(n_pages=0), INV),
         (dict(n_kv_heads=0), INV), (dict(batch=0), INV), (dict(max_pages=0), INV), (dict(dtype=2), INV), (dict(page_size=0), UNS),
         (dict(page_size=24), UNS), (dict(page_size=131072), UNS), (dict(max_pages=1 << 26), UNS), (dict(head_dim=96), UNS),
         (dict(page_stride=63), INV), (dict(slot_stride=132), INV), (dict(head_stride=0), INV), (dict(layer_stride=-8), INV),
         (dict(k=P + 8), INV), (dict(v=P + 2), INV), (dict(weights=P + 4), INV)]


def call(name, args, c=None, **kw):
    assert set(kw) <= set(args)
    c = cache() if c is None else c
    st = getattr(bd.load(), name)(C.byref(c), *[kw.get(n, args[n]) for n in args])
    assert st == bd.DOMINO_OK or bd.last_error()
    return st


@pytest.mark.parametrize("kw,status", CACHE)
def test_cache_refusals(kw, status):
    c = cache(**kw)
    for name, args in (("domino_paged_append", APPEND), ("domino_paged_attention", ATTEND), ("domino_paged_evict", EVICT),
                       ("domino_paged_commit", COMMIT)):
        assert call(name, args, c) == status
    assert bd.load().domino_paged_attention_workspace_bytes(C.byref(c), 5, 4, 3, 64, 0) == 0
    assert bd.load().domino_paged_evict_workspace_bytes(C.byref(c), 64, 32) == 0


WORK = [(dict(ws=None), WS), (dict(ws=P + 8), WS), (dict(n=8), WS)]
ROWS = WORK + [(dict(layer=-1), INV), (dict(layer=2), INV), (dict(tokens=0), INV), (dict(nq=0), INV), (dict(nq=3), INV),
               (dict(q=None), INV), (dict(q=P + 2), INV), (dict(ldq=255), INV), (dict(ldq=260), INV), (dict(out=None), INV),
               (dict(ldo=248), INV), (dict(starts=None), INV), (dict(lens=None), INV), (dict(tokens=1 << 24), UNS)]


@pytest.mark.parametrize("kw,status", ROWS + [
    (dict(k=None), INV), (dict(v=None), INV), (dict(ldk=64), INV), (dict(ldv=130), INV), (dict(out=P), INV), (dict(rot=-16), INV),
    (dict(rot=80), INV), (dict(rot=24), UNS), (dict(freq=None), INV), (dict(freq=P + 4), INV), (dict(scale=float("nan")), INV),
    (dict(qn=P + 4), INV), (dict(qn=P, eps=-1.0), INV), (dict(kn=P, eps=float("inf")), INV)])
def test_append_refusals(kw, status):
    assert call("domino_paged_append", APPEND, **kw) == status


@pytest.mark.parametrize("kw,status", ROWS + [
    (dict(max_new=0), INV), (dict(max_len=0), INV), (dict(max_len=65), INV), (dict(out=P, ldo=512), INV), (dict(scale=0.0), INV),
    (dict(scale=-1.0), INV), (dict(scale=float("inf")), INV), (dict(scale=float("nan")), INV), (dict(mask=P, ldm=2), INV)])
def test_attention_refusals(kw, status):
    assert call("domino_paged_attention", ATTEND, **kw) == status


def test_weights_are_needed():
    c = cache(weights=None)
    assert call("domino_paged_attention", ATTEND, c, acc=1) == INV
    assert call("domino_paged_evict", EVICT, c) == INV
    assert bd.load().domino_paged_evict_workspace_bytes(C.byref(c), 64, 32) == 0


@pytest.mark.parametrize("kw,status", WORK + [
    (dict(lens=None), INV), (dict(new=None), INV), (dict(new=P), INV), (dict(max_len=0), INV), (dict(max_len=65), INV),
    (dict(budget=0), INV), (dict(budget=(1 << 21) + 1), UNS), (dict(sink=-1), INV), (dict(recent=-1), INV), (dict(sink=25), INV),
    (dict(sink=2**31 - 1, recent=2**31 - 1), INV), (dict(table=P, pages=1), INV)])
def test_evict_refusals(kw, status):
    assert call("domino_paged_evict", EVICT, **kw) == status


@pytest.mark.parametrize("kw,status", WORK + [
    (dict(nodes=0), INV), (dict(nodes=1025), INV), (dict(depth=0), INV), (dict(depth=64), INV), (dict(lens=None), INV),
    (dict(acc=None), INV), (dict(path=None), INV), (dict(new=None), INV), (dict(new=P), INV)])
def test_commit_refusals(kw, status):
    assert call("domino_paged_commit", COMMIT, **kw) == status


@pytest.mark.parametrize("kind,name,kw", [
    (bd.DOMINO_ROPE_NONE, "none", {}), (bd.DOMINO_ROPE_LINEAR, "linear", dict(factor=4.0)), (bd.DOMINO_ROPE_NTK, "ntk", dict(factor=8.0)),
    (bd.DOMINO_ROPE_YARN, "yarn", dict(factor=16.0, original_ctx=4096, beta_fast=32.0, beta_slow=1.0)),
    (bd.DOMINO_ROPE_YARN, "yarn", dict(factor=1.0, original_ctx=1, beta_fast=2.0, beta_slow=0.5))])
@pytest.mark.parametrize("rot", [4, 64, 128])
def test_rope_frequencies(kind, name, kw, rot):
    f, scale = bd.domino_rope_frequencies(rot, 1e6, kind, **kw)
    want, want_scale = po.rope_frequencies(rot, 1e6, name, **kw)
    assert np.abs(f / want - 1).max() <= 64 * 2.0**-53   # pow of both libraries, and the products after it
    assert abs(scale - want_scale) <= 2.0**-24 * want_scale * 1.01


@pytest.mark.parametrize("args", [
    (0, 1e4), (3, 1e4), (130, 1e4), (64, 1.0), (64, float("inf")), (64, float("nan")), (64, 1e4, 4), (64, 1e4, 1, 0.5),
    (64, 1e4, 1, float("nan")), (2, 1e4, 2, 2.0), (64, 1e4, 3, 2.0, 0), (64, 1e4, 3, 2.0, 4096, 1.0, 1.0),
    (64, 1e4, 3, 2.0, 4096, 1.0, 0.0), (64, 1e4, 3, 2.0, 4096, float("inf"), 1.0)])
def test_rope_frequencies_refusals(args):
    with pytest.raises(bd.DominoError) as e:
        bd.domino_rope_frequencies(*args)
    assert e.value.status == INV


def test_launches_fit_their_grids(tmp_path):
    """From the smallest to the largest calls: grids below 2^32 threads, a workspace of exactly the query's size is taken, one
    byte less refused."""
    host_stub.run('''
import paper_2605_29707_amd.binding as bd
lib, F = bd.load(), h.FAKE
def cache(**kw):
    c = dict(k=F, v=F, weights=F, page_table=F, layer_stride=1 << 40, page_stride=1 << 30, slot_stride=1 << 14, head_stride=128,
             n_layers=1, n_pages=9, page_size=64, n_kv_heads=8, head_dim=128, batch=1, max_pages=16, dtype=1)
    c.update(kw)
    return C.byref(bd.domino_paged_cache(**c))
def check():
    out = [r for r in h.log() if r[0] == "launch"]
    assert out
    for r in out:
        assert int(r[2]) * int(r[3]) * int(r[4]) * int(r[5]) < 2**32 and int(r[2]) >= 1 and int(r[3]) <= 65535, r
    return out
for batch, tokens, nq, nkv, new, length, dtype in ((1, 1, 8, 8, 1, 1, 1), (1, 1, 64, 1, 1, 1 << 29, 1), (64, 64, 64, 8, 1, 131072, 1),
        (1, 32768, 32, 8, 32768, 131072, 1), (1024, 4096, 32, 8, 64, 4096, 0), (3, 100000, 8, 8, 99999, 99999, 0), (7, 427, 40, 8, 61, 3000, 1)):
    c = cache(batch=batch, max_pages=-(-length // 64), n_kv_heads=nkv, dtype=dtype)
    for acc in (0, 1):
        n = lib.domino_paged_attention_workspace_bytes(c, tokens, nq, new, length, acc)
        assert n >= 16
        args = (c, 0, tokens, nq, new, length, F, nq * 128, F + 8192, nq * 128, F, F, 0.1, None, 0, None, acc, F)
        assert lib.domino_paged_attention(*args, n - 1, None) == -2 and lib.domino_paged_attention(*args, n, None) == 0, bd.last_error()
        check()
    args = (c, 0, tokens, nq, F, nq * 128, F, nkv * 128, F, nkv * 128, F, nq * 128, F, F, None, F, 128, 0, 1.0, None, None, 0.0, F)
    assert lib.domino_paged_append(*args, 15, None) == -2 and lib.domino_paged_append(*args, 16, None) == 0
    check()
    for budget in (1, 5000, 1 << 21):
        n = lib.domino_paged_evict_workspace_bytes(c, length, budget)
        for table in (None, F):
            args = (c, F, F + 64, length, budget, 0, 1, table, 1 << 16, None, F)
            assert lib.domino_paged_evict(*args, n - 1, None) == -2 and lib.domino_paged_evict(*args, n, None) == 0
            check()
    assert lib.domino_paged_commit(c, 61, 15, F, F, F, F + 64, F, 16, None) == 0
    check()
# what no launch holds is refused
c = cache(batch=1 << 20, max_pages=1 << 23)
assert lib.domino_paged_attention_workspace_bytes(c, 1 << 20, 8, 1, 1 << 29, 1) == 0 and "launch" in bd.last_error()
''', tmp_path)


def test_binding_refuses_what_it_cannot_pass_on():
    def refused(fn, *a, **kw):
        with pytest.raises(bd.DominoError) as e:
            fn(*a, **kw)
        assert e.value.status == INV

    k = torch.zeros(9, 16, 2, 64)
    table = torch.zeros(3, 4, dtype=torch.int32)
    refused(bd.PagedCache, k, k.bfloat16(), table)
    refused(bd.PagedCache, k, k[:, :8], table)
    refused(bd.PagedCache, k.double(), k.double(), table)
    refused(bd.PagedCache, k, k.transpose(1, 2).contiguous().transpose(1, 2), table)   # other strides
    refused(bd.PagedCache, k.transpose(2, 3), k.transpose(2, 3), table)                # rows that are not dense
    refused(bd.PagedCache, k, k, table.long())
    refused(bd.PagedCache, k, k, table[0])
    refused(bd.PagedCache, k, k, table.t())
    refused(bd.PagedCache, k, k, table, weights=torch.zeros(9, 16, 2))
    refused(bd.PagedCache, k[0], k[0], table)
    refused(bd.PagedCache, k[:0], k[:0], table)
    c = bd.PagedCache(k, k.clone(), table, weights=torch.zeros(9, 2, 16))
    q, kn, ws = torch.zeros(5, 4, 64), torch.zeros(5, 2, 64), torch.zeros(4096, dtype=torch.uint8)
    starts, lens = torch.zeros(4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    ok = dict(q=q, k=kn, v=kn, q_out=q, seq_starts=starts, kv_lens=lens, workspace=ws)
    for kw in (dict(q=q.bfloat16()), dict(q=q[0]), dict(k=kn[:4]), dict(v=q), dict(q_out=q[:, :2]), dict(seq_starts=lens),
               dict(kv_lens=lens.long()), dict(positions=lens), dict(frequencies=torch.zeros(32)), dict(q_norm=torch.zeros(32)),
               dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), {}):   # (the last: not on a GPU)
        refused(bd.domino_paged_append, c, **{**ok, **kw})
    ok = dict(q=q, out=q.clone(), seq_starts=starts, kv_lens=lens, max_new=3, max_len=9, workspace=ws)
    for kw in (dict(out=q[:, :2]), dict(lse=torch.zeros(5, 3)), dict(mask=torch.zeros(5, 2, dtype=torch.uint8)),
               dict(mask=torch.zeros(5, 3)), dict(mask=torch.zeros(4, 3, dtype=torch.bool)), {}):
        refused(bd.domino_paged_attention, c, **{**ok, **kw})
    refused(bd.domino_paged_attention_workspace_bytes, c, 5, 3, 3, 9)
    refused(bd.domino_paged_evict_workspace_bytes, c, 9, 0)
    refused(bd.domino_paged_evict, c, lens, lens.clone(), 9, 4, ws, kept=torch.zeros(3, 2, 4))
    refused(bd.domino_paged_evict, c, lens, lens.clone(), 9, 4, ws, new_table=lens)
    refused(bd.domino_paged_evict, c, lens, lens.clone(), 9, 4, ws)
    refused(bd.domino_paged_commit, c, 16, lens, lens, lens, lens.clone(), ws)
    refused(bd.domino_paged_commit, c, 16, lens, lens, torch.zeros(3, 15, dtype=torch.int32), lens.clone(), ws)
