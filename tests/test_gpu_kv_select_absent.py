"""heal_kv_select where the cache does not hold some blocks: they score -infinity, whatever
lies where their page would be."""
import numpy as np
import pytest
import torch

import kv_ref
import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu
from test_gpu_kv import dev, ints

pytestmark = [pytest.mark.gpu, needs_gpu]

B, DIM, HEADS, GROUP = 16, 64, 2, 3


def select_and_compare(lens, counts, cols, absent, sizes, ragged, seed=0):
    """absent(i, b): whether block b of sequence i is not held.  Every list whole."""
    rng = np.random.default_rng(seed)
    seqs = len(lens)
    c = heal.KVCache.empty(seqs * cols, seqs, HEADS, DIM, B)
    mean = rng.standard_normal((seqs * cols, HEADS, DIM)).astype(np.float32)
    c.k_mean.copy_(dev(mean))
    table = rng.permutation(seqs * cols).reshape(seqs, cols).astype(np.int32)
    score = mean[table].astype(np.float64)   # (seqs, cols, heads, dim)
    out = [-1, seqs * cols, 2 ** 31 - 1, -2 ** 31]
    for i in range(seqs):
        for b in range(cols):
            if absent(i, b):
                table[i, b] = out[(i + b) % 4]
                score[i, b] = np.nan        # a score that is no number is -infinity
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    q = rng.standard_normal((int(cu[-1]), HEADS * GROUP, DIM)).astype(np.float32)
    for n_sel, first, last in sizes:
        announce("select %d of %d columns, %s tokens" % (n_sel, cols, counts[:4]))
        got = heal.heal_kv_select(c, dev(q), n_sel, dev(table), ints(list(map(int, lens))), cu=dev(cu) if ragged else None,
                                  keep_first=first, keep_last=last).cpu().numpy()
        for i in range(seqs):
            for j in range(counts[i]):
                t = cu[i] + j
                for h in range(HEADS):
                    want = kv_ref.select(q[t, h * GROUP:(h + 1) * GROUP], score[i, :, h], int(lens[i]) - counts[i] + j, B,
                                         n_sel, first, last)
                    assert got[t, h].tolist() == want, (n_sel, i, j, h)


def a_third(i, b):
    return (b * 7 + i) % 3 == 0


def most(i, b):
    return (b * 5 + i) % 16 != 3


def whole_tiles(i, b):
    return b % 64 >= 20


@pytest.mark.parametrize("absent", [a_third, most, whole_tiles])
@pytest.mark.parametrize("seqs,cols", [(3, 32), (3, 100), (3, 200), (140, 130), (2, 700)])
def test_single_tokens(seqs, cols, absent):
    """Two, four and sixteen waves; candidates in registers and (2048 and more) not."""
    lens = [cols * B - 5 * i for i in range(seqs)]
    select_and_compare(lens, [1] * seqs, cols, absent, [(2, 1, 1), (5, 0, 1), (cols // 2, 2, 3), (cols - 1, 1, 1)], False)


@pytest.mark.parametrize("absent", [a_third, most, whole_tiles])
@pytest.mark.parametrize("cols", [30, 200])
def test_several_tokens_of_a_sequence(cols, absent):
    lens, counts = [cols * B, cols * B // 2 + 3, 40], [37, 18, 2]
    select_and_compare(lens, counts, cols, absent, [(2, 1, 1), (5, 0, 1), (cols // 2, 2, 3), (cols - 1, 1, 1)], True)


def test_a_long_table():
    select_and_compare([3000 * B], [1], 3000, whole_tiles, [(2, 1, 1), (700, 1, 1), (1500, 1, 1)], False)


def test_a_query_that_is_no_number():
    """... gives no score; the head's others decide."""
    rng = np.random.default_rng(1)
    cols = 60
    c = heal.KVCache.empty(cols, 1, 1, DIM, B)
    mean = rng.standard_normal((cols, 1, DIM)).astype(np.float32)
    c.k_mean.copy_(dev(mean))
    q = rng.standard_normal((1, 3, DIM)).astype(np.float32)
    table, lens = torch.arange(cols, dtype=torch.int32, device="cuda")[None], ints([cols * B])
    announce("a query that is no number")
    q[0, 1, 5] = np.nan
    got = heal.heal_kv_select(c, dev(q), 9, table, lens).cpu().numpy()[0, 0].tolist()
    assert got == kv_ref.select(q[0, [0, 2]], mean[:, 0].astype(np.float64), cols * B - 1, B, 9, 1, 1)
    q[:] = np.nan
    got = heal.heal_kv_select(c, dev(q), 9, table, lens).cpu().numpy()[0, 0].tolist()
    assert got == list(range(8)) + [cols - 1]
