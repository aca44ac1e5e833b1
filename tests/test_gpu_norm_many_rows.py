"""heal_block_norm of more rows than one launch takes: 2^21 workgroups, of 16 rows up to 64 wide and of
one row above 512."""
import pytest
import torch

import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("dim,rows_a_workgroup", [(3, 16), (8, 16), (513, 1)])
@pytest.mark.parametrize("add", [False, True])
def test_a_second_launch(dim, rows_a_workgroup, add):
    """Three heads that are one row of h each: the rows of one launch, bit for bit, in all of them."""
    n = (rows_a_workgroup << 21) // 3 + 23
    assert n < rows_a_workgroup << 21 < 3 * n
    g = torch.Generator(device="cuda").manual_seed(dim)
    h = torch.randn(n, dim, generator=g, device="cuda")
    w = 1.0 + 0.1 * torch.randn(dim, generator=g, device="cuda")
    kw = dict(post=w, pre=w, scale=0.5) if add else dict(pre=w)
    announce("%d x 3 rows of %d" % (n, dim))
    wide = h[:, None].expand(n, 3, dim)
    want = heal.heal_block_norm(h, h if add else None, **kw)
    got = heal.heal_block_norm(wide, wide if add else None, **kw)
    for i in (0, 1) if add else (1,):
        for head in range(3):
            assert torch.equal(got[i][:, head], want[i])
    some = h[-5:].double()
    if not add:   # (that they are right at all)
        rms = some / torch.sqrt((some * some).mean(-1, keepdim=True) + 1e-6) * w.double()
        assert torch.all((got[1][-5:, 2].double() - rms).abs() <= 2.0 ** -23 * rms.abs())
