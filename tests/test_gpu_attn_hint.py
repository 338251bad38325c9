"""A plan whose hint of short rows is wrong, in blocks of so many edges that a wavefront's share passes 32 bits."""
import pytest
import torch

from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu


def test_a_wrong_hint_of_short_rows_changes_no_result():
    """One row of 2^27 edges and 64 heads beside short ones: 2^33 steps to one wavefront, were it not cut."""
    rows, sources, heads, D, long = 300, 1000, 64, 8, 1 << 27
    g = torch.Generator(device="cuda").manual_seed(1)
    degree = torch.full((rows,), 3, dtype=torch.int64)
    degree[150] = long
    ptr = torch.cat((torch.zeros(1, dtype=torch.int64), degree.cumsum(0))).int().cuda()
    col = (torch.arange(int(ptr[-1]), device="cuda") % sources).int()
    Q = torch.randn(rows, heads * D, generator=g, device="cuda").bfloat16()
    K, V = (torch.randn(sources, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    Q[150] = 0
    results = []
    for hint in (0, B.PLAN_SHORT_DST_ROWS):
        plan = B.fastgl_block_plan_create(ptr, col, sources, B.PLAN_FWD | hint)
        results.append(B.fastgl_attn_fwd(ptr, col, Q, K, V, heads, 1, plan=plan))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    O, lse = results[1]
    # all weights are the same: the mean of the neighbours' rows, float32 sums in runs of some hundred, bf16 results
    count = torch.bincount(col[int(ptr[150]):int(ptr[151])].long(), minlength=sources).double()
    mean = (count @ V.double() / long).repeat(heads)
    off = 2.0 ** -24 * 2000 * V.double().abs().mean(0).repeat(heads)
    assert bool(((O[150].double() - mean).abs() <= off + 2.0 ** -8 * (mean.abs() + off)).all())
    assert bool(((lse[150].double() - torch.tensor(float(long)).log().item()).abs() < 1e-3).all())
