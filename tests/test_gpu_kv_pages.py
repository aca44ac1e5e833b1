"""The pages of a cache on the GPU against their rules (tests/pages_ref.py), and with the
cache's other calls."""
import numpy as np
import pytest
import torch

import pages_ref
import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class World:
    """A table and its counts, here and on the GPU.  Some rows begin as others do, and some
    entries hold nothing.  The device table has columns beyond, which stay as they are."""

    def __init__(self, rows, cols, blocks, block=16, seed=0, fill=0.7, junk=False):
        rng = self.rng = np.random.default_rng(seed)
        self.block, self.blocks, self.cols = block, blocks, cols
        pages, at = rng.permutation(blocks), 0
        self.table, self.lens = [], []
        for i in range(rows):
            n = int(rng.integers(0, int(cols * block * fill) + 1))
            row = [-1] * cols
            held = pages_ref.held_blocks(n, block)
            shared = 0
            if i and rng.random() < 0.4:
                shared = min(int(rng.integers(0, held + 1)), pages_ref.held_blocks(self.lens[i - 1], block))
                row[:shared] = self.table[i - 1][:shared]
            held = min(held, shared + blocks - at)
            n = min(n, held * block)
            row[shared:held] = pages[at:at + held - shared].tolist()
            at += held - shared
            if junk and rng.random() < 0.3:
                row[int(rng.integers(0, cols))] = int(rng.choice([-5, blocks, blocks + 7, 2**31 - 1, -2**31]))
            self.table.append(row)
            self.lens.append(n)
        self.refs = [0] * blocks
        for row in self.table:
            for p in row:
                if 0 <= p < blocks:
                    self.refs[p] += 1
        self.upload()

    def upload(self):
        wide = np.full((len(self.table), self.cols + 3), 77, np.int32)
        for i, row in enumerate(self.table):
            wide[i, :self.cols] = row
        self.wide = ints(wide)
        self.t = self.wide[:, :self.cols]
        guard = np.full(self.blocks + 8, 55, np.int32)
        guard[4:4 + self.blocks] = self.refs
        self.guard = ints(guard)
        self.pool = heal.KVPool(self.guard[4:4 + self.blocks], self.block)

    def check(self):
        torch.cuda.synchronize()
        wide, guard = self.wide.cpu().numpy(), self.guard.cpu().numpy()
        assert np.all(wide[:, self.cols:] == 77) and np.all(guard[:4] == 55) and np.all(guard[4 + self.blocks:] == 55)
        assert wide[:, :self.cols].tolist() == self.table
        assert guard[4:4 + self.blocks].tolist() == self.refs

    def release(self, lens):
        pages_ref.release(self.table, self.refs, lens, self.block)
        heal.heal_kv_release(self.pool, self.t, ints(lens))
        self.check()

    def fork(self, lens, parents, children):
        pages_ref.fork(self.table, self.refs, lens, parents, children, self.block)
        heal.heal_kv_fork(self.pool, self.t, ints(lens), ints(parents).view(-1), ints(children).view(-1))
        self.check()

    def reserve(self, lens, counts, ragged=True):
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64).tolist()
        lack = pages_ref.reserve(self.table, self.refs, lens, cu, self.block)
        got = heal.heal_kv_reserve(self.pool, cu[-1], self.t, ints(lens), cu=ints(cu) if ragged else None)
        self.check()
        assert got.item() == lack
        return lack

    def compact(self):
        held = sum(r > 0 for r in self.refs)
        moves = pages_ref.compact(self.table, self.refs)
        src, dst, count = heal.heal_kv_compact(self.pool, self.t)
        self.check()
        pad = [-1] * (self.blocks // 2 - len(moves))
        assert count.item() == len(moves)
        assert src.tolist() == [m[0] for m in moves] + pad and dst.tolist() == [m[1] for m in moves] + pad
        assert all((r > 0) == (p < held) for p, r in enumerate(self.refs))
        return moves


SIZES = [(1, 1, 1), (1, 3, 2), (3, 5, 7), (7, 33, 150), (64, 70, 3001), (5, 1030, 4100), (130, 9, 4096), (40, 40, 9000)]


@pytest.mark.parametrize("rows,cols,blocks", SIZES)
@pytest.mark.parametrize("junk", [False, True])
def test_release(rows, cols, blocks, junk):
    w = World(rows, cols, blocks, seed=rows, junk=junk)
    announce("release %s" % ((rows, cols, blocks, junk),))
    w.release([max(0, n - int(w.rng.integers(0, 3 * w.block))) for n in w.lens])
    w.release([int(w.rng.choice([0, -3, 2**31 - 1, 5])) for _ in w.lens])
    w.release([0] * rows)
    if not junk:
        assert not any(w.refs)


@pytest.mark.parametrize("rows,cols,blocks", SIZES)
def test_fork(rows, cols, blocks):
    w = World(rows, cols, blocks, seed=rows + 1, junk=True)
    announce("fork %s" % ((rows, cols, blocks),))
    order = w.rng.permutation(rows)
    half = rows // 2
    parents = w.rng.choice(order[:max(half, 1)], rows - half).tolist()
    w.fork(w.lens, parents, order[half:].tolist())   # (one row: its own parent, left out)
    # no pairs; numbers that are no rows; a child twice; a child that is a parent
    w.fork(w.lens, [], [])
    bad = [(-1, 0), (rows, 0), (0, -1), (0, rows), (2**31 - 1, 0), (0, -2**31)]
    w.fork(w.lens, [p for p, _ in bad], [c for _, c in bad])
    any_row = lambda n: w.rng.integers(0, rows, n).tolist()  # noqa: E731
    w.fork(w.lens, any_row(5), any_row(5))
    w.fork([n - 20 for n in w.lens], any_row(3), any_row(3))


def test_more_pairs_than_threads():
    rows = 700
    w = World(rows, 3, 4000, seed=9)
    parents = w.rng.integers(0, 100, 900).tolist()
    children = w.rng.integers(90, rows, 900).tolist()
    w.fork(w.lens, parents, children)


@pytest.mark.parametrize("rows,cols,blocks", SIZES)
@pytest.mark.parametrize("junk", [False, True])
def test_reserve(rows, cols, blocks, junk):
    w = World(rows, cols, blocks, seed=rows + 2, junk=junk)
    announce("reserve %s" % ((rows, cols, blocks, junk),))
    room = cols * w.block
    for step in range(4):
        counts = w.rng.choice([0, 1, 1, 2, 5, 16, 40], rows).tolist()
        lens = [min(n + c, room + (step == 3) * 40) for n, c in zip(w.lens, counts)]
        lens = [n if w.rng.random() < 0.9 else int(w.rng.choice([0, -1, 1])) for n in lens]
        if not w.reserve(lens, counts):
            w.lens = [max(n, 0) for n in lens]
    lens = [min(n + 1, room) for n in w.lens]
    w.reserve(lens, [1] * rows, ragged=False)


def test_reserve_shared_blocks():
    """All of a block's holders in the call: the first keeps it; some: they all leave it."""
    w = World(1, 4, 40, block=16, seed=3)
    w.table = [[5, 6, 7, -1], [5, 6, 7, -1], [5, 6, 7, -1], [5, 6, -1, -1]]
    w.refs = [0] * 40
    w.refs[5] = w.refs[6] = 4
    w.refs[7] = 3
    w.upload()
    w.reserve([41, 41, 41, 30], [1, 1, 1, 0])          # block 7's three holders, all here
    assert w.table[0][2] == 7 and w.table[1][2] == 0 and w.table[2][2] == 1
    w.reserve([41, 30, 41, 33], [0, 1, 0, 1])          # block 6 leaves row 1; row 3 opens its third
    assert w.table[1][1] == 2 and w.refs[6] == 3 and w.table[3][2] == 3
    w.reserve([20, 20, 20, 20], [20, 20, 20, 20])      # everything becomes its row's own
    assert sorted(w.refs) == sorted([1] * sum(w.refs) + [0] * (40 - sum(w.refs)))


def test_reserve_all_or_nothing():
    w = World(6, 8, 20, seed=5, fill=0.3)
    before = [list(r) for r in w.table], list(w.refs)
    assert w.reserve([128] * 6, [128] * 6) > 0
    assert (w.table, w.refs) == before
    w.release([0] * 6)
    assert w.reserve([128, 0, 32, 0, 0, 0], [128, 0, 32, 0, 0, 0]) == 0
    assert w.reserve([0, 160, 0, 0, 0, 0], [0, 160, 0, 0, 0, 0]) == 0   # its table has room for 8 blocks
    assert w.reserve([0, 0, 0, 48, 0, 0], [0, 0, 0, 48, 0, 0]) == 1
    assert w.reserve([0, 0, 0, 32, 0, 0], [0, 0, 0, 32, 0, 0]) == 0
    assert all(w.refs)


def test_counts_that_do_not_agree():
    """Entries whose block is called free, more entries than counted, negative counts."""
    w = World(1, 3, 30, seed=6)
    w.table = [[4, 5, 6], [4, 5, 9], [4, 5, 6], [1, 1, 1]]
    w.refs = [0] * 30
    w.refs[4], w.refs[5], w.refs[6], w.refs[9], w.refs[1], w.refs[2] = 2, 7, 0, -4, 1, -2**30 + 1
    w.upload()
    w.reserve([48, 48, 48, 48], [48, 48, 48, 48])


@pytest.mark.parametrize("tokens", [1, 40])
@pytest.mark.parametrize("seqs", [1023, 1024, 1025, 2500, 5000])
def test_reserve_of_many_sequences(seqs, tokens):
    """As many work units as one workgroup has threads, and more."""
    w = World(seqs, 4, 3 * seqs + 50, seed=seqs, fill=0.2)
    lens = [n + tokens for n in w.lens]
    announce("reserve %d x %d" % (seqs, tokens))
    w.reserve(lens, [tokens] * seqs, ragged=tokens > 1)
    w.reserve([n + 1 for n in lens], [1] * seqs)
    w.compact()


def test_reserve_in_a_large_pool():
    w = World(9, 70, 300001, seed=1, fill=0.5)
    for p in w.rng.permutation(300001)[:250000]:
        w.refs[p] = max(w.refs[p], 1)
    w.upload()
    w.reserve([n + 300 for n in w.lens], [300] * 9)
    w.refs = [max(r, 1) for r in w.refs[:-2]] + w.refs[-2:]
    w.upload()
    w.reserve([n + 600 for n in w.lens], [300] * 9)
    w.compact()


@pytest.mark.parametrize("rows,cols,blocks", SIZES + [(3, 1100, 8191), (2, 4, 4097), (1, 8192, 8192), (3, 2731, 8192), (2, 8, 8193)])
@pytest.mark.parametrize("junk", [False, True])
def test_compact(rows, cols, blocks, junk):
    w = World(rows, cols, blocks, seed=rows + 3, junk=junk, fill=0.5)
    announce("compact %s" % ((rows, cols, blocks, junk),))
    w.compact()
    assert w.compact() == []
    w.release([0 if i % 2 else n for i, n in enumerate(w.lens)])
    w.compact()
    w.release([0] * rows)
    if not junk:
        assert w.compact() == []


def test_compact_of_full_and_empty_pools():
    for held in (range(0), range(100), range(50, 100), range(99, 100), range(0, 100, 2)):
        w = World(1, 2, 100)
        w.table, w.refs = [[-1, -1]], [int(p in held) * (1 + p) for p in range(100)]
        w.upload()
        w.compact()


def test_calls_without_rows():
    pool = heal.KVPool.empty(10, 16)
    none = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    heal.heal_kv_release(pool, none, ints([]))
    heal.heal_kv_fork(pool, none, ints([]), ints([]), ints([]))
    missing = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    assert heal.heal_kv_reserve(pool, 0, none, ints([]), missing=missing) is missing
    assert missing.item() == 0
    assert heal.heal_kv_reserve(pool, 0, none, ints([]), cu=ints([0])).item() == 0
    src, dst, count = heal.heal_kv_compact(pool, none)
    assert count.item() == 0 and src.tolist() == dst.tolist() == [-1] * 5


# ---- copies ---------------------------------------------------------------------

ARRAYS = ("k_codes", "v_codes", "scales", "k_mean", "k_recent", "v_recent")


def random_cache(blocks, slots, heads, dim, block, seed=0):
    torch.manual_seed(seed)
    cache = heal.KVCache.empty(blocks, slots, heads, dim, block)
    for name in ARRAYS:
        t = getattr(cache, name)
        t.copy_(torch.randint(-128, 128, t.shape, device="cuda") if t.dtype == torch.int8 else torch.randn(t.shape, device="cuda"))
    return cache


def check_copy(cache, blocks=((), ()), slots=((), ()), count=None):
    want = [getattr(cache, n).clone() for n in ARRAYS]
    n = len(blocks[0]) if count is None else max(0, min(count, len(blocks[0])))
    for i, t in enumerate(want):
        pairs = list(zip(*blocks))[:n] if i < 4 else zip(*slots)
        old = t.clone()
        for a, b in pairs:
            if 0 <= a < len(t) and 0 <= b < len(t):
                t[b] = old[a]
    heal.heal_kv_copy(cache, blocks=tuple(map(ints, blocks)) if blocks[0] else None,
                      slots=tuple(map(ints, slots)) if slots[0] else None, count=None if count is None else ints([count]))
    torch.cuda.synchronize()
    for name, t in zip(ARRAYS, want):
        assert torch.equal(getattr(cache, name), t), name


@pytest.mark.parametrize("heads,dim,block", [(1, 64, 16), (5, 96, 16), (3, 96, 32), (8, 128, 64), (2, 128, 128), (33, 64, 128),
                                             (1023, 64, 16)])
def test_copy(heads, dim, block):
    cache = random_cache(12, 7, heads, dim, block)
    announce("copy %s" % ((heads, dim, block),))
    check_copy(cache, blocks=((3, 0, 11), (5, 9, 1)), slots=((6, 2), (0, 3)))
    check_copy(cache, blocks=((3, 12, -1, 4, 2**31 - 1, 7), (5, 9, 1, 12, 0, -2**31)))   # two of them no blocks
    check_copy(cache, slots=((1, 7, -1, 2, 4), (3, 0, 5, -9, 4)))
    check_copy(cache, blocks=((1, 2, 3, 4), (8, 9, 10, 11)), count=2)
    for count in (0, -5, 9):
        check_copy(cache, blocks=((5, 6), (1, 2)), count=count)
    heal.heal_kv_copy(cache)


def test_copy_of_more_units_than_workgroups():
    cache = random_cache(3000, 2, 2, 64, 128)
    order = np.random.default_rng(0).permutation(3000)
    check_copy(cache, blocks=(order[:1500].tolist(), order[1500:].tolist()))


def test_copy_of_blocks_past_32_bits():
    cache = heal.KVCache.empty(36000, 2, 8, 128, 64)   # 2.4 GB of codes of each kind, 64 KiB a block
    last = 35999
    assert cache.k_codes.numel() > 1 << 31
    for name in ARRAYS[:4]:
        t = getattr(cache, name)
        t[1].copy_(torch.randint(-99, 99, t[1].shape, device="cuda"))
        t[last].zero_()
    heal.heal_kv_copy(cache, blocks=(ints([1]), ints([last])))
    for name in ARRAYS[:4]:
        t = getattr(cache, name)
        assert torch.equal(t[1], t[last]) and t[last].any()


# ---- refusals that need tensors ----------------------------------------------------

def test_tensors_that_do_not_fit_are_refused():
    pool, cache = heal.KVPool.empty(10, 16), random_cache(10, 3, 1, 64, 16)
    t, n = torch.full((3, 4), -1, dtype=torch.int32, device="cuda"), ints([0, 0, 0])
    two, three = ints([0, 1]), ints([0, 1, 2])
    for f in (lambda: heal.heal_kv_release(pool, t.long(), n), lambda: heal.heal_kv_release(pool, t, two),
              lambda: heal.heal_kv_release(pool, t.t(), ints([0] * 4)), lambda: heal.heal_kv_release(pool, t.cpu(), n),
              lambda: heal.heal_kv_release(pool, t, n.float()), lambda: heal.heal_kv_fork(pool, t, n, two, three),
              lambda: heal.heal_kv_fork(pool, t, n, two, two.long()), lambda: heal.heal_kv_reserve(pool, 4, t, n),
              lambda: heal.heal_kv_reserve(pool, 3, t, n, cu=three), lambda: heal.heal_kv_reserve(pool, 3, t, n, missing=two),
              lambda: heal.heal_kv_compact(pool, t, src=ints([0] * 4)), lambda: heal.heal_kv_compact(pool, t, count=two),
              lambda: heal.heal_kv_copy(cache, blocks=(two, three)), lambda: heal.heal_kv_copy(cache, slots=(two, two.cpu())),
              lambda: heal.heal_kv_copy(cache, count=ints([1])), lambda: heal.heal_kv_copy(cache, blocks=two),
              lambda: heal.heal_kv_copy(cache, slots=(None, two)), lambda: heal.heal_kv_fork(pool, t, n, None, None), lambda: heal.heal_kv_copy(cache, blocks=(two, two), count=two),
              lambda: heal.KVPool(ints([0] * 8)[::2], 16), lambda: heal.KVPool(ints([0] * 8), 17),
              lambda: heal.KVPool(ints([]), 16), lambda: setattr(pool, "refs", n), lambda: delattr(pool, "block")):
        with pytest.raises(heal.HealError):
            f()


# ---- as they are used ----------------------------------------------------------------

def test_forks_of_a_sequence_decode_like_sequences_of_their_own():
    """A prompt forks into three; all four go on with tokens of their own, are cut back and
    compacted, and attend to what sequences that never shared anything attend to, bit for bit."""
    heads, dim, block, rows, cols = 2, 64, 16, 4, 8
    torch.manual_seed(3)
    pool = heal.KVPool.empty(40, block)
    pool.refs[::3] = 1   # (someone else's)
    shared, apart = (random_cache(40, rows, heads, dim, block, seed=s) for s in (1, 2))
    table = torch.full((rows, cols), -1, dtype=torch.int32, device="cuda")
    own = torch.arange(rows * cols, device="cuda").view(rows, cols).to(torch.int32)
    randn = lambda *s: torch.randn(s, device="cuda")  # noqa: E731
    # the prompt, in row 0
    n = 43
    k, v = randn(n, heads, dim), randn(n, heads, dim)
    lens, cu = ints([n, 0, 0, 0]), ints([0, n, n, n, n])
    assert heal.heal_kv_reserve(pool, n, table, lens, cu=cu).item() == 0
    heal.heal_kv_append(shared, k, v, table, lens, cu=cu)
    heal.heal_kv_fork(pool, table, lens, ints([0, 0, 0]), ints([1, 2, 3]))
    heal.heal_kv_copy(shared, slots=(ints([0, 0, 0]), ints([1, 2, 3])))
    heal.heal_kv_append(apart, k.repeat(rows, 1, 1), v.repeat(rows, 1, 1), own, ints([n] * rows),
                        cu=ints([n * i for i in range(rows + 1)]))
    assert (pool.refs > 0).sum().item() == 14 + 3
    length = [n] * rows
    for counts, cut in ([[1, 1, 1, 1], [0, 0, 0, 0]], [[1, 7, 5, 2], [0, 3, 5, 0]], [[20, 1, 0, 1], [0, 0, 0, 0]],
                        [[1, 1, 1, 40], [1, 0, 0, 0]]):
        length = [x + c for x, c in zip(length, counts)]
        T, lens = sum(counts), ints(length)
        cu = ints(np.concatenate([[0], np.cumsum(counts)]))
        k, v, q = randn(T, heads, dim), randn(T, heads, dim), randn(T, 2 * heads, dim)
        assert heal.heal_kv_reserve(pool, T, table, lens, cu=cu).item() == 0
        got = []
        for cache, t in ((shared, table), (apart, own)):
            heal.heal_kv_append(cache, k, v, t, lens, cu=cu)
            got.append(heal.heal_kv_attention(cache, q, t, lens, cu=cu))
        assert torch.equal(*got)
        length = [x - c for x, c in zip(length, cut)]
        heal.heal_kv_release(pool, table, ints(length))
        src, dst, count = heal.heal_kv_compact(pool, table)
        heal.heal_kv_copy(shared, blocks=(src, dst), count=count)
        held = (pool.refs > 0).sum().item()
        assert (pool.refs[:held] > 0).all()
    heal.heal_kv_release(pool, table, ints([0] * rows))
    assert (pool.refs > 0).sum().item() == 14 and (table == -1).all()


def test_a_captured_step():
    """Release, fork, reserve and the copies in a graph, replayed on other contents."""
    w = World(12, 30, 400, seed=8, fill=0.4)
    cache = random_cache(400, 14, 1, 64, 16)
    lens, kept = ints(w.lens), ints(w.lens)
    cu, tokens = ints(range(0, 37, 3)), 36
    parents, children, slots = ints([0, 1]), ints([2, 3]), (ints([0, 1]), ints([2, 3]))
    missing = torch.zeros(1, dtype=torch.int32, device="cuda")
    lists = [torch.zeros(200, dtype=torch.int32, device="cuda") for _ in range(2)]
    count = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step():
        heal.heal_kv_release(w.pool, w.t, kept)
        heal.heal_kv_fork(w.pool, w.t, kept, parents, children)
        heal.heal_kv_copy(cache, slots=slots)
        heal.heal_kv_reserve(w.pool, tokens, w.t, lens, cu=cu, missing=missing)
        heal.heal_kv_compact(w.pool, w.t, *lists, count)
        heal.heal_kv_copy(cache, blocks=lists, count=count)
    graph = torch.cuda.CUDAGraph()
    step_lens = [n + 3 for n in w.lens]
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        kept_now = [max(0, n - turn) for n in step_lens]
        kept_now[2:4] = [0, 0]
        now = list(kept_now)
        now[2:4] = now[0:2]
        now = [n + 3 for n in now]
        kept.copy_(ints(kept_now))
        lens.copy_(ints(now))
        pages_ref.release(w.table, w.refs, kept_now, 16)
        pages_ref.fork(w.table, w.refs, kept_now, [0, 1], [2, 3], 16)
        lack = pages_ref.reserve(w.table, w.refs, now, list(range(0, 37, 3)), 16)
        moves = pages_ref.compact(w.table, w.refs)
        want = [getattr(cache, n).clone() for n in ARRAYS]
        for t in want[4:]:
            t[2:4] = t[0:2]
        for a, b in moves:
            for t in want[:4]:
                t[b] = t[a]
        torch.cuda.synchronize()
        graph.replay()
        w.check()
        assert missing.item() == lack == 0 and count.item() == len(moves)
        for name, t in zip(ARRAYS, want):
            assert torch.equal(getattr(cache, name), t), name
        step_lens = now


def test_on_another_stream():
    w = World(20, 40, 900, seed=4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        w.release([n // 2 for n in w.lens])
        w.reserve([n // 2 + 5 for n in w.lens], [5] * 20)
        w.compact()
