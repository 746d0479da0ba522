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


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("new", [3, 40])           # the kernel of few rows; the chunks' (of fp32 two tiles of 16)
@pytest.mark.parametrize("ctx", [13, 2500])        # one run; several
@pytest.mark.parametrize("page", [1, 8, 32, 64])   # a page's lookup by slots, loads, halves of a step and steps
def test_values_that_are_not_finite(dtype, dh, masked, new, ctx, page):
    """Single values of new tokens: in the rows that see their slot NaN or the infinity stands in their column, every other number
    is that of a call on finite values."""
    n = ctx + new
    c = Pages([n], page=page, nkv=2, dh=dh, dtype=dtype, seed=page, stale="")
    q = tokens(new, 4, dh, dtype, 1)
    sees = torch.tril(torch.ones(new, new, dtype=torch.bool))
    mask = None
    if masked:     # siblings: tokens that some earlier and some later rows do not see
        sees = (torch.rand(new, new, generator=torch.Generator().manual_seed(new)) < 0.6) & sees | torch.eye(new, dtype=torch.bool)
        sees[new - 1] = True
        mask = sees.to(torch.uint8).to(DEV)
    odd = [(new // 2, 3, float("nan")), (new // 2 + 1, dh // 2 + 1, INF), (new - 1, dh - 1, -INF), (0, 5, INF)]
    want, want_lse = attend(c, q, n, mask)
    want = want.clone()
    for token, col, value in odd:
        put(c, c.v[..., col], ctx + token, value)
        want[sees[:, token].to(DEV), :, col] = value
    out, lse = attend(c, q, n, mask)
    assert torch.equal(lse, want_lse)
    assert torch.equal(out.nan_to_num(123.0, 1e38, -1e38), want.nan_to_num(123.0, 1e38, -1e38))


@pytest.mark.parametrize("dtype,dh,page", [("bf16", 64, 8), ("bf16", 128, 64), ("f32", 128, 32), ("f32", 64, 1)])
@pytest.mark.parametrize("new", [1, 40])
def test_values_of_the_context_that_are_not_finite(dtype, dh, page, new):
    """Every row sees them, in steps without a mask: their columns hold no finite number, the others what they held."""
    n = 700 + new
    c = Pages([n], page=page, nkv=2, dh=dh, dtype=dtype, seed=page, stale="")
    q = tokens(new, 4, dh, dtype, 1)
    want, want_lse = attend(c, q, n)
    for slot, col, value in ((5, 3, float("nan")), (300, 17, INF), (699, dh - 1, -INF)):
        put(c, c.v[..., col], slot, value)
    out, lse = attend(c, q, n)
    cols = torch.zeros(dh, dtype=torch.bool, device=DEV)
    cols[[3, 17, dh - 1]] = True
    assert torch.equal(lse, want_lse) and torch.equal(out[..., ~cols], want[..., ~cols])
    assert not torch.isfinite(out[..., cols]).any() and torch.isnan(out[..., 3]).all()
