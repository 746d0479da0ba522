"""The row operators on the GPU against their float64 oracle: top entries, the
distillation loss and gradient, filtered sampling.

Tolerances.  A sum of exp over a row is formed from single-precision exponentials: the
difference to the maximum, its product with log2(e)/T and that factor are each off by
2^-24 at most, so a term of 2^-x is off by 3 x ln2 2^-24 of itself, and the exponential
by 2^-23; terms that matter in a row of V have x <= log2(V) + 10 < 29, which bounds the sum's
error by 29 * 0.69 * 3 * 2^-24 + 2^-23 < 4e-6 of itself (EXP).  Outputs are rounded once: 2^-24 (fp32) or
2^-8 (bf16) of the value (HALF)."""
import numpy as np
import pytest

import synth
from oracle import rows_oracle as ro

torch = pytest.importorskip("torch")
from paper_2605_29707_amd import binding as bd  # noqa: E402
from gpu_helpers import log  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EXP = 4e-6
HALF = {"f32": 2.0**-24, "bf16": 2.0**-8}
LOWEST = {"f32": float(np.finfo(np.float32).min), "bf16": -3.3895313892515355e38}


def _dt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _values(dtype, x):
    """x as the type holds it."""
    x = np.asarray(x, np.float32)
    return synth.bf16_round(x) if dtype == "bf16" else x


def _make(kind, rows, V, dtype, seed=0):
    rng = np.random.default_rng([seed, V, rows])
    x = rng.normal(size=(rows, V)) * 2.5
    if kind == "zipf":       # a power law over the ranks, peaked and flat rows
        x = -rng.uniform(1.0, 3.0, size=(rows, 1)) * np.log(rng.uniform(1e-6, 1, size=(rows, V)))
    elif kind == "ties":
        x = rng.integers(-3, 4, size=(rows, V)).astype(float)
    elif kind == "falling":  # the first entries fill the first groups
        x = -np.sort(-x, axis=1)
    elif kind == "equal":
        x = np.full((rows, V), 1.5)
    elif kind == "coarse":   # bf16 values 1/8 apart: thousands of each
        x = 24 + 1.2 * x
    elif kind == "close":    # values that differ in their last bits alone, of both signs
        x = rng.integers(-3000, 3000, size=(rows, V)) * 1e-9
    elif kind in ("masked", "lowest"):   # few ids stay, none in the last row
        low = -np.inf if kind == "masked" else LOWEST[dtype]
        keep = rng.random(size=(rows, V)) < 40.0 / V
        keep[-1] = False
        x = np.where(keep, x, low)
    elif kind == "special":  # NaN, infinities, zeros of both signs among ordinary values
        at = rng.integers(0, V, size=(rows, 6))
        for r in range(rows):
            x[r, at[r]] = [np.nan, -np.inf, 0.0, -0.0, np.nan, LOWEST[dtype]]
        x[0, at[0, 0]] = np.inf
        if rows > 1:
            x[1] = np.nan
    return _values(dtype, x)


def _put(x, dtype, pad=0, offset=0):
    """The rows on the GPU, `pad` values apart, the first one `offset` values into its memory."""
    n, V = x.shape
    flat = torch.full((offset + n * (V + pad),), 7.0, dtype=_dt(dtype), device=DEV)
    rows = flat[offset:].view(n, V + pad)[:, :V]
    rows.copy_(torch.from_numpy(x).to(DEV))
    return rows


def _t(x, dt=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(dt)


def _ws(nbytes):
    """A workspace of just this size with a guard behind it, full of old data."""
    buf = torch.full((nbytes + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    return buf


def _guard(buf, nbytes):
    assert bool((buf[nbytes:] == 0xA5).all()), "written past the workspace"


# --------------------------------------------------------------------------
# top entries
# --------------------------------------------------------------------------
def _top(lg, k, T=1.0, rest=True, stream=None):
    n, V = lg.shape
    nb = bd.domino_top_logits_workspace_bytes(n, V, k)
    buf = _ws(nb)
    ids = torch.full((n, k), -7, dtype=torch.int32, device=DEV)
    vals, r = torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
    bd.domino_top_logits(lg, ids, vals, buf[:nb], rest=r if rest else None, temperature=T, stream=stream)
    torch.cuda.synchronize()
    assert bd.domino_workspace_error(buf) == 0
    _guard(buf, nb)
    return ids.cpu().numpy(), vals.cpu().numpy(), r.cpu().numpy()


def _check_rest(got, want):
    # (the type's lowest value over T = 0.25 is -1.36e39: below fp32's range, and -inf when rounded to it)
    with np.errstate(over="ignore"):
        fin = np.isfinite(want.astype(np.float32))
        np.testing.assert_array_equal(got[~fin], want.astype(np.float32)[~fin])
    tol = EXP + HALF["f32"] * np.abs(want[fin])
    assert np.all(np.abs(got[fin] - want[fin]) <= tol), np.max(np.abs(got[fin] - want[fin]) - tol)


@pytest.mark.parametrize("kind,rows,V,k,dtype,pad,offset,T", [
    ("normal", 1, 1, 1, "f32", 0, 0, 1.0), ("normal", 3, 7, 7, "bf16", 0, 1, 1.0), ("normal", 2, 31, 5, "f32", 1, 3, 0.5),
    ("normal", 5, 33, 33, "bf16", 0, 0, 1.0), ("ties", 4, 255, 100, "bf16", 2, 0, 1.0),
    ("normal", 2, 1024, 1024, "f32", 0, 0, 2.0), ("normal", 2, 4096, 1024, "bf16", 0, 0, 1.0),
    ("zipf", 3, 8193, 17, "f32", 0, 0, 1.0), ("zipf", 40, 4097, 2, "bf16", 0, 0, 3.0),
    ("zipf", 5, 50257, 64, "bf16", 0, 0, 1.0), ("zipf", 3, 50257, 1000, "f32", 5, 2, 0.7),
    ("zipf", 2, 151936, 256, "bf16", 0, 0, 1.0), ("zipf", 2, 327680, 1024, "f32", 0, 0, 1.0),
    ("ties", 3, 151936, 512, "bf16", 0, 0, 1.0), ("ties", 2, 40000, 33, "f32", 0, 0, 1.0),
    ("ties", 3, 5000, 1024, "f32", 0, 0, 1.0), ("ties", 3, 2000, 700, "bf16", 0, 1, 1.0), ("coarse", 2, 151936, 900, "bf16", 0, 0, 2.0),
    ("falling", 2, 50257, 300, "f32", 0, 0, 1.0), ("falling", 2, 151936, 1024, "f32", 0, 0, 1.0),
    ("falling", 2, 20000, 1024, "bf16", 0, 0, 1.0), ("equal", 2, 327680, 1024, "bf16", 0, 0, 1.0),
    ("equal", 2, 5000, 100, "f32", 0, 0, 1.0), ("close", 2, 30000, 700, "f32", 0, 0, 1.0),
    ("masked", 4, 50257, 64, "bf16", 0, 0, 1.0), ("masked", 3, 50257, 512, "f32", 0, 0, 1.0),
    ("lowest", 3, 32000, 128, "bf16", 0, 0, 1.0), ("lowest", 3, 32000, 30, "f32", 0, 0, 0.25),
    ("special", 4, 4099, 20, "f32", 0, 0, 1.0), ("special", 4, 4099, 20, "bf16", 0, 0, 1.0)])
def test_top_logits(kind, rows, V, k, dtype, pad, offset, T):
    x = _make(kind, rows, V, dtype)
    ids, vals, rest = _top(_put(x, dtype, pad, offset), k, T)
    want = ro.top_logits(x, k, T)
    np.testing.assert_array_equal(ids, want["ids"])
    np.testing.assert_array_equal(vals, want["vals"].astype(np.float32))
    _check_rest(rest, want["rest"])


def test_rest_behind_a_wide_gap_keeps_its_value():
    """The others lie so far below the entries that exp of the difference is 0."""
    x = np.full((2, 9000), -3000.0, np.float32)
    x[:, ::1000] = 50.0
    ids, _, rest = _top(_put(x, "f32"), 9)
    assert ids[0].tolist() == list(range(0, 9000, 1000))
    _check_rest(rest, np.full(2, -3000.0 + np.log(8991)))


def test_top_without_rest_and_on_another_stream():
    x = _make("zipf", 6, 32000, "bf16")
    lg = _put(x, "bf16")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    ids, vals, _ = _top(lg, 50, rest=False, stream=st)
    np.testing.assert_array_equal(ids, ro.top_logits(x, 50)["ids"])


def test_top_of_many_rows():
    """More workgroups than the chip holds at once; an id as its row's own maximum."""
    n, V = 5000, 130
    g = torch.Generator(device=DEV).manual_seed(3)
    lg = torch.randn(n, V, generator=g, device=DEV)
    at = torch.randint(0, V, (n,), generator=g, device=DEV)
    lg[torch.arange(n, device=DEV), at] = 30.0
    ids, vals, rest = _top(lg, 1)
    assert np.array_equal(ids[:, 0], at.cpu().numpy()) and np.all(vals == 30.0)
    lg[torch.arange(n, device=DEV), at] = -float("inf")
    _check_rest(rest, torch.logsumexp(lg.double(), 1).cpu().numpy())


# --------------------------------------------------------------------------
# distillation
# --------------------------------------------------------------------------
def _teacher(kind, rows, V, k, seed=1):
    x = _make("zipf" if kind == "zipf" else "normal", rows, V, "bf16", seed).astype(np.float64)
    top = ro.top_logits(x, k)
    return top["ids"], top["vals"].astype(np.float32), x


def _distill(lg, ids, vals, rest=None, T=1.0, w=None, scale=1.0, grad="new", ld_pad=0, stream=None, error=0):
    n, V = lg.shape
    k = ids.shape[1]
    nb = bd.domino_distill_workspace_bytes(n, V, k)
    buf = _ws(nb)
    loss, row_loss = torch.empty(1, device=DEV), torch.empty(n, device=DEV)
    wide = None
    if grad == "new":
        wide = torch.full((n, V + ld_pad), 9.0, dtype=lg.dtype, device=DEV)
        g = wide[:, :V]
    else:
        g = lg if grad == "in place" else None
    bd.domino_distill_loss(lg, _t(ids, torch.int32), _t(vals), loss, buf[:nb], teacher_rest=None if rest is None else _t(rest),
                           temperature=T, row_weights=None if w is None else _t(w), grad_scale=scale, row_loss=row_loss,
                           grad=g, stream=stream)
    torch.cuda.synchronize()
    assert bd.domino_workspace_error(buf) == error
    _guard(buf, nb)
    if wide is not None and ld_pad:
        assert bool((wide[:, V:] == 9.0).all()), "written behind a row"
    return (float(loss[0]), row_loss.cpu().numpy().astype(np.float64),
            None if g is None else g.float().cpu().numpy().astype(np.float64))


def _check_distill(got, x, ids, vals, rest, T, w, scale, dtype):
    want = ro.distill_loss(x, ids, vals, rest, T, w, scale)
    n, V = x.shape
    loss, row_loss, grad = got
    fin = np.isfinite(want["row_loss"])
    np.testing.assert_array_equal(row_loss[~fin], want["row_loss"][~fin])
    # a KL is a mean of differences of logarithms, each off by the sums' error
    tol = 2 * EXP * T * T + HALF["f32"] * np.abs(want["row_loss"][fin])
    assert np.all(np.abs(row_loss[fin] - want["row_loss"][fin]) <= tol)
    if np.isfinite(want["loss"]):
        assert abs(loss - want["loss"]) <= 2 * EXP * T * T + HALF["f32"] * abs(want["loss"])
    else:
        np.testing.assert_array_equal(loss, want["loss"])
    if grad is None:
        return
    ww = np.ones(n) if w is None else np.where((np.asarray(w) >= 0) & np.isfinite(w), w, 0.0)
    W = ww.sum()
    g, ref = grad, want["grad"]
    assert np.array_equal(np.isnan(g), np.isnan(ref))
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(np.isnan(x), -np.inf, x.astype(np.float64)) / T
        z = z - np.where(np.isfinite(z.max(1, keepdims=True)), z.max(1, keepdims=True), 0.0)
        q = np.exp(z)
        q = q / np.maximum(q.sum(1, keepdims=True), 1e-300)
    s = abs(scale) * T * (ww / W if W > 0 else ww)[:, None]
    # a term of 2^-x: 3 x ln2 2^-24 + 2^-23 of itself (x up to 126, below which it is 0 in fp32)
    tol = (HALF[dtype] + 126 * 0.7 * 3 * 2.0**-24 + 2.0**-23) * np.abs(ref) + EXP * s * q + s * 2.0**-120 + 2.0**-126
    bad = np.abs(g - ref) > tol
    assert not bad.any(), (np.argwhere(bad)[:3], g[bad][:3], ref[bad][:3])


@pytest.mark.parametrize("rows,V,k,dtype,rest,T,pad,offset,weights", [
    (1, 1, 1, "f32", False, 1.0, 0, 0, False), (3, 9, 9, "bf16", False, 1.0, 0, 1, True),
    (2, 33, 4, "f32", True, 0.5, 3, 1, True), (15, 4096, 16, "f32", True, 1.0, 0, 0, True),
    (5, 4097, 1, "bf16", True, 2.0, 0, 0, False), (7, 8191, 300, "f32", True, 1.5, 2, 0, True),
    (4, 50257, 100, "bf16", True, 1.5, 7, 3, True), (3, 50257, 1024, "f32", True, 3.0, 0, 0, False),
    (2, 151936, 64, "f32", True, 2.0, 0, 0, True), (2, 151936, 128, "bf16", False, 1.0, 0, 0, False),
    (2, 400000, 8, "bf16", True, 1.0, 0, 0, False), (300, 64, 3, "f32", True, 1.0, 0, 0, True)])
def test_distill(rows, V, k, dtype, rest, T, pad, offset, weights):
    ids, vals, tx = _teacher("zipf", rows, V, k)
    r = ro.top_logits(tx, k, T)["rest"].astype(np.float32) if rest else None
    rng = np.random.default_rng(V)
    x = _values(dtype, 0.8 * tx + 0.7 * rng.normal(size=tx.shape))
    w = np.exp(-(np.arange(rows) % 15) / 15.0).astype(np.float32) if weights else None
    if weights and rows > 2:
        w[1] = 0.0
    got = _distill(_put(x, dtype, pad, offset), ids, vals, r, T, w, scale=1.25, ld_pad=pad)
    _check_distill(got, x, ids, vals, r, T, w, 1.25, dtype)
    if pad == 0 and offset == 0:   # the same bits in the logits' place, and the same loss without a gradient
        again = _distill(_put(x, dtype), ids, vals, r, T, w, scale=1.25, grad="in place")
        assert again[0] == got[0] and np.array_equal(again[1], got[1]) and np.array_equal(again[2], got[2])
        alone = _distill(_put(x, dtype), ids, vals, r, T, w, grad=None)
        assert alone[0] == got[0] and np.array_equal(alone[1], got[1])


@pytest.mark.parametrize("kind", ["masked", "lowest", "special", "equal"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_odd_students(kind, dtype):
    """Masked students (one row wholly), NaN and infinities; the losses are inf or NaN where the formula's are."""
    rows, V, k = 4, 5000, 12
    ids, vals, tx = _teacher("normal", rows, V, k)
    x = _make(kind, rows, V, dtype, seed=4)
    if kind == "special":   # where entries are: NaN is -inf, so that q = 0 under p > 0
        x[2, ids[2, 0]] = np.nan
        x[0] = np.where(np.isposinf(x[0]), 1.0, x[0])
    r = ro.top_logits(tx, k)["rest"].astype(np.float32)
    got = _distill(_put(x, dtype), ids, vals, r)
    _check_distill(got, x, ids, vals, r, 1.0, None, 1.0, dtype)
    inf = _make("normal", rows, V, dtype)
    inf[1, 77] = np.inf     # no distribution: NaN in its row, no other
    loss, row_loss, grad = _distill(_put(inf, dtype), ids, vals, r)
    assert np.isnan(loss) and np.isnan(row_loss[1]) and np.isfinite(row_loss[[0, 2, 3]]).all()
    assert np.isnan(grad[1, 77]) and np.isfinite(grad[[0, 2, 3]]).all()


def test_distill_odd_teachers():
    """Unused places, rows without a teacher, entries of -inf, all the weight in the rest or none."""
    rows, V, k = 6, 3001, 10
    ids, vals, tx = _teacher("normal", rows, V, k)
    r = ro.top_logits(tx, k)["rest"].astype(np.float32)
    ids[0, 3:] = -1
    ids[1] = -1                         # the rest alone: q_rest is 1, so is p_rest
    ids[2], r[2] = -1, -np.inf          # nothing
    vals[3], r[3] = -np.inf, 2.0
    vals[4, :5], r[4] = -np.inf, -np.inf
    vals[5, 2] = np.nan
    x = _make("normal", rows, V, "f32", seed=9)
    got = _distill(_put(x, "f32"), ids, vals, r)
    _check_distill(got, x, ids, vals, r, 1.0, None, 1.0, "f32")
    assert got[1][2] == 0 and not got[2][2].any()


def test_distill_rest_far_below_the_entries():
    """The student's others weigh nothing beside its entries while the teacher puts a third of its weight there."""
    V, k = 6000, 4
    x = np.full((2, V), -200.0, np.float32)
    x[:, :k] = 20.0
    x[1, k:] += np.random.default_rng(0).normal(size=V - k)
    ids, vals = np.tile(np.arange(k, dtype=np.int32), (2, 1)), np.zeros((2, k), np.float32)
    r = np.full(2, np.log(2.0), np.float32)
    got = _distill(_put(x, "f32"), ids, vals, r)
    _check_distill(got, x, ids, vals, r, 1.0, None, 1.0, "f32")


def test_distill_bad_ids_and_weights():
    rows, V, k = 5, 9000, 6
    ids, vals, _ = _teacher("normal", rows, V, k)
    x = _make("normal", rows, V, "f32", seed=2)
    ids[1, 4] = V                   # out of range
    ids[2, 5] = ids[2, 0]           # twice
    ids[3, 1] = -2
    loss, row_loss, grad = _distill(_put(x, "f32"), ids, vals, error=bd.DEV_BAD_TOKEN)
    assert np.isnan(loss) and np.isnan(row_loss[[1, 2, 3]]).all() and np.isfinite(row_loss[[0, 4]]).all()
    assert np.isnan(grad[[1, 2, 3]]).all() and np.isfinite(grad[[0, 4]]).all()
    w = np.array([1.0, 0.0, 0.0, 0.0, 2.0], np.float32)     # the bad rows weigh nothing
    got = _distill(_put(x, "f32"), ids, vals, w=w, error=bd.DEV_BAD_TOKEN)
    assert np.isfinite(got[0]) and not got[2][[1, 2, 3]].any()
    ids, vals, _ = _teacher("normal", rows, V, k)
    w = np.array([1.0, -1.0, np.nan, np.inf, 2.0], np.float32)
    got = _distill(_put(x, "f32"), ids, vals, w=w, error=bd.DEV_BAD_PARAM)
    _check_distill(got, x, ids, vals, None, 1.0, w, 1.0, "f32")
    got = _distill(_put(x, "f32"), ids, vals, w=np.zeros(rows, np.float32))
    assert got[0] == 0 and not got[2].any()


def test_distill_gradient_against_differences():
    """The loss moves by the gradient along a direction: error h^2 of the third derivative (|d| <= 1 and
    probabilities: below h^2) and the losses' own error over 2 h."""
    rows, V, k, T, h = 4, 2000, 30, 1.3, 0.05
    ids, vals, tx = _teacher("normal", rows, V, k)
    r = ro.top_logits(tx, k, T)["rest"].astype(np.float32)
    rng = np.random.default_rng(8)
    x = _values("f32", tx + rng.normal(size=tx.shape))
    d = rng.choice([-1.0, 1.0], size=x.shape).astype(np.float32)
    up, down = (_distill(_put(x + s * h * d, "f32"), ids, vals, r, T, grad=None)[0] for s in (1, -1))
    grad = _distill(_put(x, "f32"), ids, vals, r, T)[2]
    assert abs((up - down) / (2 * h) - float((grad * d).sum())) <= h * h + 2 * (2 * EXP * T * T) / (2 * h)


# --------------------------------------------------------------------------
# sampling
# --------------------------------------------------------------------------
def _sample(lg, u, T=None, top_k=None, top_p=None, min_p=None, stream=None, error=0):
    n, V = lg.shape
    nb = bd.domino_sample_logits_workspace_bytes(n, V)
    buf = _ws(nb)
    tok, lp = torch.full((n,), -7, dtype=torch.int32, device=DEV), torch.empty(n, device=DEV)

    def opt(a, dt=torch.float32):
        return None if a is None else _t(np.broadcast_to(np.asarray(a), (n,)), dt)

    bd.domino_sample_logits(lg, opt(u), tok, buf[:nb], temperature=opt(T), top_k=opt(top_k, torch.int32),
                            top_p=opt(top_p), min_p=opt(min_p), logprobs=lp, stream=stream)
    torch.cuda.synchronize()
    assert bd.domino_workspace_error(buf) == error
    _guard(buf, nb)
    return tok.cpu().numpy(), lp.cpu().numpy().astype(np.float64)


def _check_sample(x, u, T=None, top_k=None, top_p=None, min_p=None, dtype="f32", pad=0, offset=0):
    n = len(x)
    f32 = [None if a is None else np.broadcast_to(np.asarray(a, np.float32), (n,)) for a in (u, T, top_p, min_p)]
    k = None if top_k is None else np.broadcast_to(np.asarray(top_k), (n,))
    tok, lp = _sample(_put(x, dtype, pad, offset), f32[0], f32[1], k, f32[2], f32[3])
    want = ro.sample_logits(x, f32[0], f32[1], k, f32[2], f32[3])
    # both sides hold the running sums to 2^-40 of the kept sum; where the whole row's sum comes
    # from single-precision exponentials (no filter ends among the first entries), to EXP of what lies behind them
    clear = want["margin"] > 1e-11
    log(f"{n} rows, kept {want['kept'].min()}..{want['kept'].max()}, least margin {want['margin'].min():.1e}")
    assert clear.mean() > 0.9 or n < 3
    np.testing.assert_array_equal(tok[clear], want["tokens"][clear])
    fin = clear & np.isfinite(want["logprobs"])
    np.testing.assert_allclose(lp[fin], want["logprobs"][fin], rtol=2 * HALF["f32"], atol=EXP)
    assert np.array_equal(lp[~np.isfinite(want["logprobs"])], want["logprobs"][~np.isfinite(want["logprobs"])])
    return want


FILTERS = [dict(), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=40, top_p=0.95, min_p=0.02),
           dict(top_k=3000, top_p=0.9), dict(top_k=1024), dict(top_k=1), dict(top_k=2000, min_p=0.001)]


@pytest.mark.parametrize("kw", FILTERS, ids=lambda k: "+".join(f"{a}={b}" for a, b in k.items()) or "none")
@pytest.mark.parametrize("V,dtype,kind", [(50257, "bf16", "zipf"), (32000, "f32", "normal"), (4096, "f32", "zipf")])
def test_sample_filters(V, dtype, kind, kw):
    n = 24
    x = _make(kind, n, V, dtype, seed=7)
    u = np.random.default_rng(V).random(n).astype(np.float32)
    u[:3] = [0.0, 1 - 2.0**-24, 0.5]
    _check_sample(x, u, T=np.linspace(0.5, 1.6, n), dtype=dtype, **kw)


@pytest.mark.parametrize("kind,rows,V,dtype,pad,offset", [
    ("normal", 1, 1, "f32", 0, 0), ("normal", 9, 3, "bf16", 1, 1), ("normal", 4, 31, "f32", 0, 3),
    ("ties", 12, 5000, "bf16", 3, 0), ("equal", 12, 20000, "f32", 0, 0), ("equal", 6, 327680, "bf16", 0, 0),
    ("falling", 6, 50257, "bf16", 0, 5), ("close", 8, 30000, "f32", 0, 0), ("masked", 8, 50257, "bf16", 0, 0),
    ("lowest", 8, 32000, "f32", 0, 0), ("special", 12, 6001, "f32", 1, 0), ("special", 12, 6001, "bf16", 0, 0),
    ("normal", 3, 327680, "f32", 0, 0), ("zipf", 3, 151936, "bf16", 0, 0)])
def test_sample_edges(kind, rows, V, dtype, pad, offset):
    x = _make(kind, rows, V, dtype, seed=3)
    rng = np.random.default_rng(V + rows)
    for kw in (dict(), dict(top_p=0.7), dict(top_k=min(V, 1500), top_p=0.6), dict(min_p=0.2)):
        _check_sample(x, rng.random(rows), T=np.linspace(0.8, 1.5, rows), dtype=dtype, pad=pad, offset=offset, **kw)


def test_sample_of_equal_logits_at_exact_borders():
    """1000 equal logits, half of them kept: u on a border takes the entry behind it."""
    x = np.zeros((4, 1000), np.float32)
    tok, lp = _sample(_put(x, "f32"), np.array([0.0, 0.25, 0.5, 0.998], np.float32), top_p=0.5)
    assert tok.tolist() == [0, 125, 250, 499]
    np.testing.assert_allclose(lp, -np.log(500.0), rtol=2 * HALF["f32"])
    x = np.zeros((4, 40000), np.float32)
    tok, lp = _sample(_put(x, "f32"), np.array([0.0, 0.25, 0.5, 1 - 2.0**-24], np.float32), top_p=0.5)
    assert tok.tolist() == [0, 5000, 10000, 19999]


@pytest.mark.parametrize("V,n_inf", [(500, 64), (500, 65), (3000, 2500), (151936, 70), (151936, 151936)])
def test_sample_of_infinities(V, n_inf):
    """Logits of +inf share all the weight, also where they are more than the first entries looked at.  Their running
    sums are whole numbers, and u times one of them (24 bits times 18) is exact on both sides: so is the token, on
    a border too."""
    n = 9
    x = _make("normal", n, V, "f32", seed=6)
    rng = np.random.default_rng(V)
    for r in range(n):
        x[r, rng.permutation(V)[:n_inf]] = np.inf
    u = (rng.integers(0, 60, n) + 0.5) / 60
    for kw in (dict(), dict(top_k=min(V - 1, 1500)), dict(top_k=30), dict(top_p=0.6), dict(min_p=0.5),
               dict(top_k=min(V - 1, 1500), top_p=0.3, min_p=0.1)):
        par = {a: np.full(n, b, np.int64 if a == "top_k" else np.float32) for a, b in kw.items()}
        par["T"] = np.linspace(0.5, 2, n).astype(np.float32)
        tok, lp = _sample(_put(x, "f32"), u.astype(np.float32), **par)
        par["temperature"] = par.pop("T")
        want = ro.sample_logits(x, u.astype(np.float32), **par)
        np.testing.assert_array_equal(tok, want["tokens"])
        np.testing.assert_allclose(lp, want["logprobs"], rtol=2 * HALF["f32"])


def test_sample_greedy_rows_and_per_row_filters():
    n, V = 64, 20011
    x = _make("zipf", n, V, "bf16", seed=5)
    rng = np.random.default_rng(0)
    T = np.where(np.arange(n) % 5 == 0, 0.0, rng.uniform(0.3, 2.0, n))
    top_k = rng.choice([0, -1, 1, 20, 900, 5000, V, V + 5], n)
    top_p = rng.choice([1.0, 0.0, 0.3, 0.9, 0.99], n)
    min_p = rng.choice([0.0, 1.0, 0.1, 0.001], n)
    want = _check_sample(x, rng.random(n), T, top_k, top_p, min_p, dtype="bf16")
    greedy = T == 0
    assert np.array_equal(want["tokens"][greedy], np.argmax(x[greedy], 1)) and np.all(want["logprobs"][greedy] == 0)


def test_sample_parameters_out_of_range():
    n, V = 8, 700
    x = _make("normal", n, V, "f32")
    T = np.array([1, -1, np.nan, np.inf, 1, 1, 1, 1], np.float32)
    top_p = np.array([1, 1, 1, 1, 1.5, np.nan, 1, 1], np.float32)
    min_p = np.array([0, 0, 0, 0, 0, 0, -0.5, 0], np.float32)
    u = np.full(n, 0.3, np.float32)
    u[7] = 1.0
    tok, lp = _sample(_put(x, "f32"), u, T, None, top_p, min_p, error=bd.DEV_BAD_PARAM)
    assert tok[0] == ro.sample_row(x[0].astype(np.float64), u=float(u[0]))[0]
    assert np.all(tok[1:] == -1) and np.isnan(lp[1:]).all() and np.isfinite(lp[0])


def test_sample_temperatures_at_the_ends_of_their_range():
    """1e-30 over logits 1e-32 apart: a hundred entries an e-fold.  1e30: what is not -inf or the type's lowest
    is equal.  Past them: refused."""
    n, V = 6, 4096
    u = np.linspace(0.05, 0.9, n)
    x = np.tile((-1e-32 * np.arange(V)).astype(np.float32), (n, 1))
    for kw in (dict(), dict(top_p=0.8), dict(min_p=0.3), dict(top_k=200)):
        _check_sample(x, u, T=np.full(n, 1e-30), **kw)
    y = _make("normal", n, V, "f32", seed=2)
    y[:, ::3], y[:, 1::3] = -np.inf, LOWEST["f32"]
    for kw in (dict(), dict(top_p=0.8), dict(top_k=1200)):
        want = _check_sample(y, u, T=np.full(n, 1e30), **kw)
        assert np.all(want["tokens"] % 3 == 2)
    T = np.array([0.9e-30, 1.1e30, 1.0, 1e-38, 3e38, 1e-45], np.float32)
    tok, _ = _sample(_put(y, "f32"), u.astype(np.float32), T, error=bd.DEV_BAD_PARAM)
    assert (tok >= 0).tolist() == [False, False, True, False, False, False]


@pytest.mark.parametrize("kind,V,dtype", [("normal", 151936, "f32"), ("falling", 151936, "bf16"), ("close", 262144, "f32"),
                                          ("coarse", 151936, "bf16"), ("ties", 262144, "f32"), ("ties", 9001, "f32")])
def test_sample_few_flat_rows(kind, V, dtype):
    """Rows that several workgroups share, their filters' borders far behind the first entries and, in rows in
    falling order, a border's entries side by side."""
    n = 4
    x = _make(kind, n, V, dtype, seed=11)
    rng = np.random.default_rng(V)
    for kw in (dict(), dict(top_p=0.9), dict(top_k=30000, top_p=0.5, min_p=0.01), dict(top_k=100000), dict(min_p=0.3)):
        _check_sample(x, rng.random(n), T=np.linspace(2, 4, n), dtype=dtype, **kw)


# --------------------------------------------------------------------------
# streams, graphs, and all of them together
# --------------------------------------------------------------------------
def test_two_streams_at_once():
    """Calls with a workspace of their own on two streams give what they give alone."""
    xs = [_make("zipf", 64, 50257, "bf16", seed=s) for s in (1, 2)]
    lgs = [_put(x, "bf16") for x in xs]
    u = _t(np.random.default_rng(0).random(64))
    p = torch.full((64,), 0.9, device=DEV)
    nb = bd.domino_sample_logits_workspace_bytes(64, 50257)
    toks = [torch.empty(64, dtype=torch.int32, device=DEV) for _ in range(2)]
    wss = [_ws(nb) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in (0, 1):
            bd.domino_sample_logits(lgs[i], u, toks[i], wss[i][:nb], top_p=p, stream=streams[i])
    torch.cuda.synchronize()
    for i in (0, 1):
        alone = _sample(lgs[i], u.cpu().numpy(), top_p=0.9)[0]
        np.testing.assert_array_equal(toks[i].cpu().numpy(), alone)


def test_rows_past_32_bit_offsets():
    """The second row begins 2^31 + 3 values after the first, for reading and for the gradient."""
    V, k, ld = 20000, 16, 2**31 + 3
    x = _make("zipf", 2, V, "bf16", seed=1)
    big, gbig = (torch.empty(ld + V, dtype=torch.bfloat16, device=DEV).as_strided((2, V), (ld, 1)) for _ in range(2))
    big.copy_(torch.from_numpy(x))
    near = _put(x, "bf16")
    ids, vals, rest = _top(big, k)
    for a, b in zip((ids, vals, rest), _top(near, k)):
        np.testing.assert_array_equal(a, b)
    u = np.array([0.3, 0.99], np.float32)
    for T in (0.7, 4.0):
        for a, b in zip(_sample(big, u, np.full(2, T), top_p=0.95), _sample(near, u, np.full(2, T), top_p=0.95)):
            np.testing.assert_array_equal(a, b)
    want = _distill(near, ids, vals, rest, 2.0)
    loss, ws = torch.empty(1, device=DEV), torch.empty(bd.domino_distill_workspace_bytes(2, V, k), dtype=torch.uint8, device=DEV)
    bd.domino_distill_loss(big, _t(ids, torch.int32), _t(vals), loss, ws, teacher_rest=_t(rest), temperature=2.0, grad=gbig)
    torch.cuda.synchronize()
    assert float(loss[0]) == want[0]
    np.testing.assert_array_equal(gbig.float().cpu().numpy(), want[2])


def test_a_workspace_elsewhere_is_refused():
    lg = _put(_make("normal", 2, 100, "f32"), "f32")
    tok = torch.empty(2, dtype=torch.int32, device=DEV)
    nb = bd.domino_sample_logits_workspace_bytes(2, 100)
    for ws in (torch.empty(nb, dtype=torch.uint8), torch.empty(2 * nb, dtype=torch.uint8, device=DEV)[::2]):
        with pytest.raises(bd.DominoError) as e:
            bd.domino_sample_logits(lg, torch.zeros(2, device=DEV), tok, ws)
        assert e.value.status == bd.DOMINO_ERR_INVALID_ARG


def test_captured_calls_replay_on_new_inputs():
    """The three calls in one graph, replayed with other inputs between the program's own eager work:
    each replay gives the eager calls' bits."""
    n, V, k = 30, 20000, 32
    lg, st = torch.empty(n, V, device=DEV), torch.empty(n, V, device=DEV)
    ids, vals, rest = torch.empty(n, k, dtype=torch.int32, device=DEV), torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
    loss, grad, u = torch.empty(1, device=DEV), torch.empty(n, V, device=DEV), torch.empty(n, device=DEV)
    tok, lp = torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, device=DEV)
    p = torch.full((n,), 0.95, device=DEV)
    ws = torch.empty(max(bd.domino_top_logits_workspace_bytes(n, V, k), bd.domino_distill_workspace_bytes(n, V, k),
                         bd.domino_sample_logits_workspace_bytes(n, V)), dtype=torch.uint8, device=DEV)

    def calls():
        bd.domino_top_logits(lg, ids, vals, ws, rest=rest)
        bd.domino_distill_loss(st, ids, vals, loss, ws, teacher_rest=rest, grad=grad)
        bd.domino_sample_logits(lg, u, tok, ws, top_p=p, logprobs=lp)

    def fill(s):
        g = torch.Generator(device=DEV).manual_seed(s)
        lg.copy_(3 * torch.randn(n, V, generator=g, device=DEV))
        st.copy_(lg + torch.randn(n, V, generator=g, device=DEV))
        u.copy_(torch.rand(n, generator=g, device=DEV))

    out = (ids, vals, rest, loss, grad, tok, lp)
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for s in (1, 2, 3, 4):
        fill(s)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        calls()
        for a, b in zip(got, out):
            assert torch.equal(a, b)


def test_from_the_targets_rows_to_the_drafters_gradient():
    """As a program uses them: the target scores a chain, its top entries are kept, the drafter's
    teacher-forced forward gives the student rows, the loss from the kept entries their gradient; and the next
    token is drawn from the target's last row."""
    cfg = synth.get_config("tiny").with_(batch=2)
    w, inp = synth.make_weights(cfg, seed=0), synth.make_inputs(cfg, seed=0)
    bs, D, V, B = cfg.batch, cfg.depth, cfg.vocab, cfg.block
    dw = bd.to_device_weights(w, cfg, DEV)
    drafter, target = bd.DominoModel(cfg, dw), bd.DominoModel(cfg, dw, target=True)
    rng = np.random.default_rng(1)
    labels = rng.integers(0, V - 1, size=(bs, D)).astype(np.int32)
    ctx = 64
    lens = torch.full((bs,), ctx, dtype=torch.int32, device=DEV)
    kv = [torch.randn(cfg.n_layers, bs, ctx + B, cfg.n_kv_heads, cfg.head_dim, device=DEV,
                      generator=torch.Generator(device=DEV).manual_seed(s)) for s in (1, 2)]
    # the target's rows of the anchor and the labels but the last: row i scores label i
    tok = np.concatenate([inp["anchor"][:bs, None], labels[:, :-1]], 1).astype(np.int32)
    pos = np.tile(ctx + np.arange(D, dtype=np.int32), (bs, 1))
    mask = np.tile(np.tril(np.ones((D, D), np.uint8)), (bs, 1, 1))
    tlog = torch.empty(bs, D, V, device=DEV)
    ws = torch.empty(bd.domino_target_workspace_bytes(target, bs, D, ctx + B), dtype=torch.uint8, device=DEV)
    bd.domino_target_verify(target, _t(tok, torch.int32), _t(pos, torch.int32), _t(mask, torch.uint8), lens, *kv, ctx + B,
                            tlog, ws)
    fin = torch.empty(bs, D, V, device=DEV)
    tws = torch.empty(bd.domino_train_workspace_bytes(drafter, bs, ctx + B), dtype=torch.uint8, device=DEV)
    loss3 = torch.empty(3, device=DEV)
    bd.domino_train_forward(drafter, _t(inp["anchor"][:bs], torch.int32), lens, *kv, ctx + B, _t(labels, torch.int32), 0.5,
                            15.0, loss3, tws, debug={"final_logits": fin})
    k, T, n = 16, 1.5, bs * D
    teacher, student = tlog.view(n, V), fin.view(n, V)
    nb = bd.domino_top_logits_workspace_bytes(n, V, k)
    ids = torch.empty(n, k, dtype=torch.int32, device=DEV)
    vals, rest = torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
    bd.domino_top_logits(teacher, ids, vals, torch.empty(nb, dtype=torch.uint8, device=DEV), rest=rest, temperature=T)
    torch.cuda.synchronize()
    t, s = teacher.cpu().numpy(), student.cpu().numpy()
    want = ro.top_logits(t, k, T)
    np.testing.assert_array_equal(ids.cpu().numpy(), want["ids"])
    decay = np.exp(-(np.arange(n) % D) / 15.0).astype(np.float32)
    got = _distill(student, ids.cpu().numpy(), vals.cpu().numpy(), rest.cpu().numpy(), T, decay)
    _check_distill(got, s, ids.cpu().numpy(), vals.cpu().numpy(), rest.cpu().numpy(), T, decay, 1.0, "f32")
    # a step against the gradient lowers the loss
    lower = _distill(student - 0.5 * _t(got[2]), ids.cpu().numpy(), vals.cpu().numpy(), rest.cpu().numpy(), T, decay, grad=None)
    assert lower[0] < got[0]
    last = tlog[:, -1]       # rows D * V values apart
    _check_sample(t.reshape(bs, D, V)[:, -1], np.array([0.2, 0.9]), T=0.8, top_k=50, top_p=0.9)
    tok2, _ = _sample(last, np.array([0.2, 0.9], np.float32), np.full(2, 0.8), np.full(2, 50), np.full(2, 0.9))
    np.testing.assert_array_equal(tok2, ro.sample_logits(t.reshape(bs, D, V)[:, -1], np.array([0.2, 0.9], np.float32),
                                                         np.full(2, 0.8, np.float32), np.full(2, 50),
                                                         np.full(2, 0.9, np.float32))["tokens"])
    drafter.close()
    target.close()
