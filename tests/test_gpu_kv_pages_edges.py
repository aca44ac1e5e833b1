"""The pages of a cache at the ends of what their calls take."""
import numpy as np
import pytest
import torch

import pages_ref
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


def test_more_rows_than_one_launch():
    """2^22 rows and more, a workgroup each: rows cut back, then compaction of their tables."""
    rows, blocks, block = (1 << 22) + 300, 5000, 16
    rng = np.random.default_rng(0)
    table = rng.integers(-1, blocks, (rows, 2)).astype(np.int32)
    table[:, 0] = np.where(table[:, 0] % 3 == 1, 7, table[:, 0])   # (blocks that only second entries hold)
    lens = rng.integers(-1, 3 * block, rows).astype(np.int32)
    refs = np.bincount(table[table >= 0], minlength=blocks)
    t, pool = ints(table), heal.KVPool(ints(refs), block)
    announce("release of %d rows" % rows)
    heal.heal_kv_release(pool, t, ints(lens))
    gone = np.arange(2) >= -(-np.maximum(lens, 0)[:, None] // block)
    refs -= np.bincount(table[gone & (table >= 0)], minlength=blocks)
    table[gone] = -1
    assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(pool.refs.cpu().numpy(), refs)
    # one block in four stays
    table[table % 4 != 0] = -1
    refs = np.bincount(table[table >= 0], minlength=blocks)
    t.copy_(ints(table)), pool.refs.copy_(ints(refs))
    announce("compact %d rows" % rows)
    src, dst, count = heal.heal_kv_compact(pool, t)
    refs = refs.tolist()
    moves = pages_ref.compact([], refs)
    to = np.arange(blocks)
    for a, b in moves:
        to[a] = b
    assert len(moves) > 500 and count.item() == len(moves)
    assert src[:len(moves)].tolist() == [a for a, _ in moves] and dst[:len(moves)].tolist() == [b for _, b in moves]
    assert pool.refs.tolist() == refs
    assert np.array_equal(t.cpu().numpy(), np.where(table >= 0, to[table], -1))
