"""Attention over values of one size throughout, down to FP32's smallest."""
import numpy as np
import pytest

from gpu_util import needs_gpu
from test_gpu_kv import World, _check_attention, _check_prompts

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("size", [1e-44, 1e-40, 1e-36, 1e-32, 1e-28, 1e30, 1e37])
def test_values_of_one_size(size):
    w = World(3, heads=2, dim=64, block=32, cols=8, seed=1)
    counts = [5, 96, 201]
    w.append(counts, w.rows(302), w.rows(302) * np.float32(size))
    w.check()
    _check_attention(w, [1, 1, 1], w.rows(3, 4))
    _check_attention(w, [1, 1, 1], w.rows(3, 4), chunk=64)
    _check_attention(w, [5, 3, 4], w.rows(12, 4))


@pytest.mark.parametrize("size", [1e-40, 1e-36, 1e30])
def test_prompts_over_values_of_one_size(size):
    w = World(20, heads=8, dim=64, block=32, cols=5, seed=2)
    counts = [100 + i for i in range(20)]
    w.append(counts, w.rows(sum(counts)), w.rows(sum(counts)) * np.float32(size))
    _check_prompts(w, counts, 4)
