"""heal_block_norm about the mean of rows of up to 2^24, whose first element lies far from the others."""
import numpy as np
import pytest
import torch

import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("n", [16384, 16385, 70001, 1 << 20, (1 << 22) + 3, 1 << 24])
@pytest.mark.parametrize("first", [1000.123, 7.7777, 1e6, -2.5e8, 3.0 + 2.0 ** -20])
def test_one_element_off(n, first):
    """n - 1 threes and another value v: their mean is a / n above three with a = v - 3, their variance
    a^2 (n - 1) / n^2. So the threes give -sign(a) / sqrt(n - 1) and v gives sign(a) sqrt(n - 1), rounded
    once: 2^-24 of them. Besides, the mean is off by its roundings, 2^-53 of |a| <= 2 max(|v|, 3) and twice of
    itself, 4 x 2^-53 max(|v|, 3) in all: 4 n 2^-53 max(|v|, 3) / |a| of what the threes give. Sums
    about the mean cost 2^-26 (2^14 roundings of 2^-53, at most 2^14 times larger by cancellation, halved
    by the root)."""
    x = torch.full((2, n), 3.0, device="cuda")
    x[:, 0] = first
    v = float(x[0, 0])
    a = v - 3.0
    want = np.full(n, -np.sign(a) / np.sqrt(n - 1.0))
    want[0] = np.sign(a) * np.sqrt(n - 1.0)
    bound = (2.0 ** -24 + 2.0 ** -26 + 4 * n * 2.0 ** -53 * max(abs(v), 3.0) / abs(a)) * np.abs(want)
    one = torch.ones(n, device="cuda")
    announce("%d elements, the first %r" % (n, v))
    _, out = heal.heal_block_norm(x, pre=one, eps=0.0, centred=True)
    h, _ = heal.heal_block_norm(torch.zeros_like(x), x, post=one, eps=0.0, centred=True)
    for got in (out, h):
        err = np.abs(got.double().cpu().numpy() - want)
        assert np.all(err <= bound), (err / np.abs(want)).max()


@pytest.mark.parametrize("n", [20000, 1 << 20, (1 << 24) - 1])
def test_random_rows_about_a_far_mean(n):
    """Values around 1000 with the first at 0, against two passes in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(n)
    x = 1000.0 + torch.randn(1, n, generator=g, device="cuda")
    x[:, 0] = 0.0
    w = torch.rand(n, generator=g, device="cuda") + 0.5
    announce("%d elements about 1000" % n)
    _, out = heal.heal_block_norm(x, pre=w, centred=True)
    X = x.double()
    d = X - X.mean()
    want = d / torch.sqrt((d * d).mean() + 1e-6) * w.double()
    # half a step of the result; 2^-26 of the deviation; the mean to 2^-40 of a thousand
    assert torch.all((out.double() - want).abs() <= (2.0 ** -24 + 2.0 ** -26) * want.abs() + 2.0 ** -30)
