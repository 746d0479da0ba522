"""Calls of the row operators that are refused before any HIP call; needs no GPU."""
import ctypes as C

import pytest
import torch

import host_stub
from paper_2605_29707_amd import binding as bd

P = C.c_void_p(4096)  # never dereferenced: validation fails first
INV, WS, UNS = bd.DOMINO_ERR_INVALID_ARG, bd.DOMINO_ERR_WORKSPACE, bd.DOMINO_ERR_UNSUPPORTED
BIG = 1 << 40


def _call(name, args, **kw):
    names = list(args)
    assert set(kw) <= set(names)
    return getattr(bd.load(), name)(*[kw.get(n, args[n]) for n in names])


TOP = dict(rows=3, vocab=100, k=5, logits=P, dtype=1, ld=100, T=1.0, ids=P, vals=P, rest=None, ws=P, nbytes=BIG, st=None)
SAMPLE = dict(rows=3, vocab=100, logits=P, dtype=1, ld=100, T=None, top_k=None, top_p=None, min_p=None, u=P, tokens=P,
              logprobs=None, ws=P, nbytes=BIG, st=None)
DISTILL = dict(rows=3, vocab=100, k=5, logits=P, dtype=0, ld=100, ids=P, vals=P, rest=None, T=1.0, w=None, scale=1.0,
               loss=P, row_loss=None, grad=None, ld_grad=0, ws=P, nbytes=BIG, st=None)
ROWS = [(dict(rows=0), INV), (dict(rows=-1), INV), (dict(vocab=0), INV), (dict(dtype=2), INV), (dict(logits=None), INV),
        (dict(ld=99), INV), (dict(logits=C.c_void_p(4097)), INV), (dict(ws=None), WS), (dict(nbytes=8), WS),
        (dict(ws=C.c_void_p(4100)), WS)]
BAD_T = [(dict(T=t), INV) for t in (0.0, -1.0, float("nan"), float("inf"), 1e-38, 0.9e-30, 1.1e30)]


@pytest.mark.parametrize("kw,status", ROWS + BAD_T + [
    (dict(k=0), INV), (dict(k=101), INV), (dict(k=1025, vocab=2000, ld=2000), INV), (dict(ids=None), INV),
    (dict(vals=None), INV), (dict(vocab=327681, ld=327681), UNS), (dict(rows=1 << 22), UNS)])
def test_top_refusals(kw, status):
    assert _call("domino_top_logits", TOP, **kw) == status and bd.last_error()


@pytest.mark.parametrize("kw,status", ROWS + [
    (dict(u=None), INV), (dict(tokens=None), INV), (dict(vocab=327681, ld=327681), UNS), (dict(rows=1 << 22), UNS)])
def test_sample_refusals(kw, status):
    assert _call("domino_sample_logits", SAMPLE, **kw) == status and bd.last_error()


@pytest.mark.parametrize("kw,status", ROWS + BAD_T + [
    (dict(k=0), INV), (dict(k=101), INV), (dict(k=1025, vocab=2000, ld=2000), INV), (dict(ids=None), INV),
    (dict(vals=None), INV), (dict(loss=None), INV), (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV),
    (dict(grad=P, ld_grad=99), INV), (dict(grad=C.c_void_p(4098), ld_grad=100), INV),
    (dict(grad=P, ld_grad=101), INV),   # in the logits' place with another row stride
    (dict(vocab=2**31 - 1, ld=2**31 - 1, rows=33), UNS), (dict(rows=2**31 - 1), UNS)])
def test_distill_refusals(kw, status):
    assert _call("domino_distill_loss", DISTILL, **kw) == status and bd.last_error()


def test_workspace_queries():
    lib = bd.load()
    for f, n in ((lib.domino_top_logits_workspace_bytes, 3), (lib.domino_distill_workspace_bytes, 3),
                 (lib.domino_sample_logits_workspace_bytes, 2)):
        assert f(*(2, 151936, 64)[:n]) > 0
        assert f(*(0, 100, 4)[:n]) == f(*(2, 0, 1)[:n]) == f(*(2**31 - 1, 2**31 - 1, 4)[:n]) == 0
    for f in (lib.domino_top_logits_workspace_bytes, lib.domino_distill_workspace_bytes):
        assert f(1, 100, 0) == f(1, 100, 101) == f(1, 5000, 1025) == 0


def test_launches_fit_their_grids(tmp_path):
    """At the most rows and vocabularies: every launch's grid holds its workgroups, below 2^32
    threads, and a workspace of exactly the query's size is taken, one byte less refused."""
    host_stub.run('''
import paper_2605_29707_amd.binding as bd
lib, F = bd.load(), h.FAKE
def check(rows, vocab, chunk, extra=0):
    out = [r for r in h.log() if r[0] == "launch"]
    for r in out:
        assert int(r[2]) * int(r[5]) < 2**32 and r[3:5] == ["1", "1"], r
    assert int(out[0][2]) == rows * -(-vocab // chunk) + extra, out
    assert int(out[1][2]) == rows, out
    return out
for rows, vocab in ((1, 1), (262143, 4096), (262143, 327680), (7, 327680), (240, 151936)):
    n = lib.domino_top_logits_workspace_bytes(rows, vocab, 1)
    args = (rows, vocab, 1, F, 1, vocab, 1.0, F, F, F, F)
    assert lib.domino_top_logits(*args, n - 1, None) == -2 and lib.domino_top_logits(*args, n, None) == 0
    check(rows, vocab, 8192)
    n = lib.domino_sample_logits_workspace_bytes(rows, vocab)
    args = (rows, vocab, F, 0, vocab, None, None, None, None, F, F, None, F)
    assert lib.domino_sample_logits(*args, n - 1, None) == -2 and lib.domino_sample_logits(*args, n, None) == 0
    check(rows, vocab, 8192)
for rows, vocab, k in ((1, 1, 1), (240, 151936, 64), (31, 2**31 - 1, 8), (16777214, 4096, 1)):
    n = lib.domino_distill_workspace_bytes(rows, vocab, k)
    for grad in (None, F + 4096):
        args = (rows, vocab, k, F, 1, vocab, F, F, None, 1.0, None, 1.0, F, None, grad, vocab, F)
        assert lib.domino_distill_loss(*args, n - 1, None) == -2 and lib.domino_distill_loss(*args, n, None) == 0
        out = check(rows, vocab, 4096, 1)
        assert int(out[2][2]) == (int(out[0][2]) if grad else 1)
''', tmp_path)


def test_binding_refuses_what_it_cannot_pass_on():
    f = torch.zeros(4, 10)
    ids, vals, ws = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(64, dtype=torch.uint8)

    def refused(fn, *a, **kw):
        with pytest.raises(bd.DominoError) as e:
            fn(*a, **kw)
        assert e.value.status == INV

    refused(bd.domino_top_logits, f.t(), ids, vals, ws)                     # rows that are not dense
    refused(bd.domino_top_logits, f.double(), ids, vals, ws)
    refused(bd.domino_top_logits, f[0], ids, vals, ws)
    refused(bd.domino_top_logits, f, ids.long(), vals, ws)
    refused(bd.domino_top_logits, f, ids, vals[:, :1], ws)
    refused(bd.domino_top_logits, f, ids, vals, ws, rest=torch.zeros(3))
    refused(bd.domino_top_logits, f, ids, vals, ws)                         # not on a GPU
    loss = torch.zeros(1)
    refused(bd.domino_distill_loss, f, ids, vals, loss, ws, grad=torch.zeros(4, 9))
    refused(bd.domino_distill_loss, f, ids, vals, loss, ws, grad=f.bfloat16())
    refused(bd.domino_distill_loss, f, ids, vals, loss, ws, row_weights=torch.zeros(4, dtype=torch.float64))
    refused(bd.domino_distill_loss, f, ids, vals.t().contiguous().t(), loss, ws)
    refused(bd.domino_sample_logits, f, torch.zeros(5), ids[:, 0].contiguous(), ws)
    refused(bd.domino_sample_logits, f, torch.zeros(4), ids[:, 0], ws)      # not contiguous
    refused(bd.domino_sample_logits, f, torch.zeros(4), ids[:, 0].contiguous(), ws, top_k=torch.zeros(4))
