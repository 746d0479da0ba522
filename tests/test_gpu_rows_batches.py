"""Batches and vocabularies at the ends of the sampler's rules: more rows than one workgroup a flat row is for,
vocabularies around a vector, a group of 32, the 64 entries looked at first and the list of 2048."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import rows_oracle as ro  # noqa: E402
from test_gpu_rows import DEV, _check_sample, _make, _put, _sample, _top, _check_rest  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,V,dtype", [(1023, 16384, "bf16"), (1100, 16391, "f32"), (2050, 20000, "bf16")])
def test_sample_of_many_rows(rows, V, dtype):
    """Each row is drawn as it is in a small batch, where several workgroups share the flat ones."""
    kinds = [_make(kind, 10, V, dtype, seed=31) for kind in ("normal", "zipf", "coarse", "equal", "masked")]
    x = np.concatenate(kinds)
    rng = np.random.default_rng(rows)
    at = rng.integers(0, len(x), rows)
    big = _put(x, dtype)[torch.from_numpy(at).to(DEV)].contiguous()
    u, T = rng.random(rows).astype(np.float32), rng.uniform(0.6, 3.0, rows).astype(np.float32)
    p, k = rng.choice([1.0, 0.9, 0.5], rows).astype(np.float32), rng.choice([0, 0, 40, 3000], rows)
    tok, lp = _sample(big, u, T, k, p)
    want = ro.sample_logits(x[at[:64]], u[:64], T[:64], k[:64], p[:64])
    clear = want["margin"] > 1e-8
    np.testing.assert_array_equal(tok[:64][clear], want["tokens"][clear])
    for r0 in range(0, rows, 60):  # 60 rows: up to 2 workgroups a row
        s = slice(r0, min(r0 + 60, rows))
        t2, l2 = _sample(big[s], u[s], T[s], k[s], p[s])
        np.testing.assert_array_equal(tok[s], t2)
        np.testing.assert_array_equal(lp[s], l2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2, 5, 8, 31, 33, 63, 64, 65, 66, 71, 96, 127, 257, 1025, 2047, 2048, 2049, 2080, 4097])
def test_small_vocabularies(V, dtype):
    rng = np.random.default_rng(V)
    for kind in ("normal", "ties", "special", "masked"):
        x = _make(kind, 7, V, dtype, seed=33)
        for kw in (dict(), dict(top_p=0.8), dict(top_k=max(1, V // 2), top_p=0.7), dict(min_p=0.1)):
            _check_sample(x, rng.random(7), T=np.linspace(0.7, 2.5, 7), dtype=dtype, pad=V % 3, offset=V % 2, **kw)
        k = min(V, 1 + V // 3)
        ids, vals, rest = _top(_put(x, dtype, V % 3, V % 2), min(k, 1024))
        want = ro.top_logits(x, min(k, 1024))
        np.testing.assert_array_equal(ids, want["ids"])
        _check_rest(rest, want["rest"])
