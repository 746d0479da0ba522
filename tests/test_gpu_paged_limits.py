"""Attention on pages whose weights cannot come from kept scores: short sequences under a max_len so large that the scores of few
rows would pass 1 GB."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paged_helpers import Pages, i32  # noqa: E402
from paper_2605_29707_amd import binding as bd  # noqa: E402
from test_gpu_paged import check_attention, tokens  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("news", [[1, 1, 1], [4, 0, 3]])
def test_few_rows_under_a_very_long_limit(dtype, dh, masked, news):
    lens, page, limit = [700, 33, 1025], 64, 1 << 24
    c = Pages(lens, page=page, nkv=2, dh=dh, dtype=dtype, weights=True, seed=1)
    table = np.full((3, limit // page), -1, np.int32)
    table[:, :c.table.shape[1]] = c.table
    c.cache = bd.PagedCache(c.k, c.v, i32(table), weights=c.w)
    n, most = sum(news), max(news)
    scores = limit // 32 * 128 * most * 4 * 3 * 2            # bytes that the scores of every slot up to the limit would take
    assert scores > 1e9 and bd.domino_paged_attention_workspace_bytes(c.cache, n, 8, most, limit, True) < scores / 4
    mask = None
    if masked:
        mask = (torch.rand(n, most, generator=torch.Generator().manual_seed(2)) < 0.5).to(torch.uint8).to(c.k.device)
    check_attention(c, tokens(n, 8, dh, dtype, 3, scale=2.0), news, lens, mask=mask, max_new=most, max_len=limit, accumulate=True)
