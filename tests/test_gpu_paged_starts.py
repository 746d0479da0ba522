"""Starts of packed sequences that go down: every kernel leaves out the first sequence whose starts do and all behind it, and the
ones before it are as they are alone."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paged_helpers import DEV, Pages, i32  # noqa: E402
from paper_2605_29707_amd import binding as bd  # noqa: E402
from test_gpu_paged import tokens  # noqa: E402

pytestmark = pytest.mark.gpu


def many(drop):
    """150 sequences of two rows whose starts go down in sequence `drop`, and rise again behind it."""
    s = 2 * np.arange(151)
    s[drop + 1:] -= 5
    return list(s)


# starts, the sequences before the drop, new tokens at most, slots before the new ones
CASES = [([0, 1, 0, 1, 0, 1], 1, 1, 40), ([0, 3, 2, 5], 1, 3, 30), ([0, 5, 2, 3], 1, 5, 200), ([0, 40, 20, 60], 1, 40, 300),
         ([4, 2, 3], 0, 2, 9), ([0, 2, 2, 4, 3, 6], 3, 3, 33), (many(10), 10, 2, 20), (many(63), 63, 2, 20), (many(70), 70, 2, 20)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("starts,good,most,ctx", CASES, ids=[str(i) for i in range(len(CASES))])
def test_starts_that_go_down(dtype, starts, good, most, ctx):
    n, batch = max(starts), len(starts) - 1
    lens = [ctx + most + b % 3 for b in range(batch)]
    alone = starts[:good + 1] + [starts[good]] * (batch - good)      # the rest waits
    runs = []
    for st in (starts, alone):
        c = Pages(lens, page=8, nkv=2, dh=64, dtype=dtype, weights=True, seed=3, stale="")
        x = tokens(n, 8, 64, dtype, 1)
        q = torch.full((n, 4, 64), 7.0, dtype=x.dtype, device=DEV)
        ws = c.workspace(16)
        bd.domino_paged_append(c.cache, x[:, :4], x[:, 4:6], x[:, 6:], q, i32(st), i32(lens), ws)
        errors = [bd.domino_workspace_error(ws)]
        need = bd.domino_paged_attention_workspace_bytes(c.cache, n, 4, most, max(lens), True)
        ws = c.workspace(need).fill_(0x70)       # (large finite numbers, if something read what nothing wrote)
        ws[:16] = 0
        out, lse = torch.full_like(q, 7.0), torch.full((n, 4), 7.0, device=DEV)
        bd.domino_paged_attention(c.cache, x[:, :4], out, i32(st), i32(lens), most, max(lens), ws, lse=lse, accumulate=True)
        errors.append(bd.domino_workspace_error(ws))
        runs.append((errors, q, out, lse, c.k, c.v, c.w))
    assert runs[0][0] == [bd.DEV_BAD_CTX_LEN] * 2 and runs[1][0] == [0, 0]
    for got, want in zip(runs[0][1:], runs[1][1:]):
        assert torch.equal(got, want)
    if starts[good] < n:
        assert (runs[0][2][starts[good]:] == 7.0).all()
