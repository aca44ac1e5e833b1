"""The pages of a cache at the ends of what their calls take."""
import pytest
import torch

import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu
from test_gpu_kv_pages import World, ints

pytestmark = [pytest.mark.gpu, needs_gpu]


def test_tables_without_columns():
    """Rows that have no entries: nothing is held or taken, and compaction moves the counts alone."""
    pool = heal.KVPool.empty(10, 16)
    pool.refs[::3] = 2
    table, lens = torch.empty((3, 0), dtype=torch.int32, device="cuda"), ints([40, 0, 7])
    announce("no columns")
    heal.heal_kv_release(pool, table, lens)
    heal.heal_kv_fork(pool, table, lens, ints([0]), ints([1]))
    for cu, tokens in ((ints([0, 20, 20, 27]), 27), (None, 3)):
        assert heal.heal_kv_reserve(pool, tokens, table, lens, cu=cu).item() == 0
    assert pool.refs.tolist() == [2, 0, 0] * 3 + [2]
    src, dst, count = heal.heal_kv_compact(pool, table)
    assert pool.refs.tolist() == [2] * 4 + [0] * 6 and count.item() == 2
    assert src.tolist() == [9, 6, -1, -1, -1] and dst.tolist() == [1, 2, -1, -1, -1]


@pytest.mark.parametrize("seqs", [510, 511, 512, 513])
def test_reserve_around_the_units_of_one_workgroup(seqs):
    """A ragged call has two units for each sequence and one for each block of tokens: 1024 of them, a
    few more, a few less."""
    w = World(seqs, 3, 4 * seqs, block=128, seed=seqs, fill=0.6)
    for tokens in (0, 100, 127, 128, 129, 255, 256, 400):
        counts = [0] * seqs
        for i in range(tokens):
            counts[(i * i + seqs - 1) % seqs] += 1
        counts[-1] += tokens - sum(counts)
        announce("reserve %d sequences, %d tokens" % (seqs, tokens))
        w.reserve([n + c for n, c in zip(w.lens, counts)], counts)
