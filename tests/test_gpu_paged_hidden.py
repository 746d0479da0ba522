"""Values of v that are not finite, over the kernels, page sizes, masks and runs of the attention on pages: they reach every row that
sees their slot, whatever its weight, and no other."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paged_helpers import DEV, Pages, i32  # noqa: E402
from paper_2605_29707_amd import binding as bd  # noqa: E402
from test_gpu_paged import no_error, tokens  # noqa: E402

pytestmark = pytest.mark.gpu
INF = float("inf")


def attend(c, q, n, mask=None):
    """One sequence of n slots, every row of q new: (out, lse)."""
    new, nq = q.shape[:2]
    out, lse = torch.full_like(q, 7.0), torch.full((new, nq), 7.0, device=DEV)
    ws = c.workspace(bd.domino_paged_attention_workspace_bytes(c.cache, new, nq, new, n))
    bd.domino_paged_attention(c.cache, q, out, i32([0, new]), i32([n]), new, n, ws, mask=mask, lse=lse)
    no_error(ws)
    return out, lse


def put(c, x, slot, value):
    x[0, c.table[0, slot // c.page], slot % c.page] = value


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("ctx,new", [(150, 3), (2500, 3), (150, 40), (2500, 40)])
def test_a_score_of_minus_infinity_hides_nothing(dtype, masked, ctx, new):
    """A slot with score -inf and NaN in v, among the context's (steps that every row sees whole) and among the new ones: NaN in the
    rows that see it, and their lse is that of the other slots."""
    n = ctx + new
    mask = torch.tril(torch.ones(new, new, dtype=torch.uint8, device=DEV)) if masked else None
    q = tokens(new, 4, 64, dtype, 1)
    q[..., 0] = 1.0
    for slot in (5, ctx - 2, ctx + new // 2):
        c = Pages([n], page=16, nkv=2, dh=64, dtype=dtype, seed=4, stale="")
        put(c, c.k[..., 0], slot, -INF)
        want, want_lse = attend(c, q, n, mask)
        put(c, c.v, slot, float("nan"))
        out, lse = attend(c, q, n, mask)
        first = max(0, slot - ctx)
        assert torch.equal(lse, want_lse) and torch.isfinite(lse).all()
        assert torch.isnan(out[first:]).all() and torch.equal(out[:first], want[:first])
    # nothing but such slots
    c.k[..., 0] = -INF
    c.v.fill_(float("nan"))
    out, lse = attend(c, q, n, mask)
    assert (out == 0).all() and (lse == -INF).all()
