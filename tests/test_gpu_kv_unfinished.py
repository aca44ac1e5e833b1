"""Rows of a block that is not complete, some of which hold infinities, no numbers or numbers
far larger than the others: what a query does not see, and what is no longer there,
does not reach its output."""
import numpy as np
import pytest
import torch

import kv_ref
import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu
from test_gpu_kv import World, dev

pytestmark = [pytest.mark.gpu, needs_gpu]

ODD = [float("nan"), float("inf"), -float("inf"), 1e10, -3e38]


def attention(w, counts, q, **kw):
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    out = torch.full(q.shape, 7.0, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    announce("attention %s of %s, %s %s" % (counts, w.lens(), q.shape, kw))
    heal.heal_kv_attention(w.cache, dev(q), **w.kw(), cu=dev(cu), out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)


def check(w, counts, q, some=False, **kw):
    """Causal attention against its definition.  A key row that is not finite makes a
    row that sees it no number throughout, a value that is not finite only its
    column; the bounds go by the rows that are seen (and complete blocks by all of theirs)."""
    out, lse = attention(w, counts, q, **kw)
    group, scale, window = q.shape[1] // w.heads, w.dim ** -0.5, kw.get("window", 0)
    t0 = 0
    for i, r in enumerate(w.ref):
        n, c = len(r.k), counts[i]
        if not c:
            continue
        rows, t0 = slice(t0, t0 + c), t0 + c
        place, at = np.arange(n - c, n)[:, None], np.arange(n)
        seen = at <= place
        if window:
            seen &= at > place - window
        keys, values = r.values("k"), r.values("v")
        for h in range(q.shape[1]):
            if some and 0 < h % group < group - 1:
                continue
            K, V = keys[:, h // group], values[:, h // group]
            x = q[rows, h].astype(np.float64)
            no_key = seen @ ~np.isfinite(K).all(1) > 0           # (rows)
            no_value = seen.astype(int) @ ~np.isfinite(V) > 0    # (rows, dim)
            K, V = np.where(np.isfinite(K), K, 0.0), np.where(np.isfinite(V), V, 0.0)
            s = np.where(seen, scale * (x @ K.T), -np.inf)
            m = s.max(1)
            e = np.where(seen, np.exp(s - m[:, None]), 0.0)
            p = e / e.sum(1)[:, None]
            S = scale * np.where(seen, np.abs(x) @ np.abs(K).T, 0.0).max(1)
            # the largest value of the complete blocks that are seen and of the other rows that are
            big = np.abs(V).max(1)
            full = n // w.block * w.block
            for b in range(0, full, w.block):
                big[b:b + w.block] = np.abs(r.v[b:b + w.block, h // group]).max()
            v = np.where(seen, big, 0.0).max(1)
            rel, floor, off = kv_ref.bound(S, seen.sum(1), w.dim,
                                           scale * np.abs(x).max(1) * np.where(seen, np.abs(K).sum(1), 0.0).max(1),
                                           scale * np.abs(x).sum(1) * np.where(seen, np.abs(K).max(1), 0.0).max(1), v)
            got = out[rows, h]
            assert np.all(np.isnan(got) == (no_value | no_key[:, None])), (i, h)
            assert np.all(np.isnan(lse[rows, h]) == no_key), (i, h)
            ok = ~(no_value | no_key[:, None])
            err = np.abs(got - p @ V) - (rel[:, None] * (p @ np.abs(V)) + floor[:, None])
            assert np.all(err[ok] <= 0), (i, h, err[ok].max())
            want = m + np.log(e.sum(1))
            assert np.all(np.abs(lse[rows, h] - want)[~no_key] <= (off + 2.0 ** -23 * np.abs(want))[~no_key]), (i, h)


@pytest.mark.parametrize("odd", ODD)
@pytest.mark.parametrize("dim,block", [(64, 16), (96, 32), (128, 64), (64, 128), (128, 16)])
def test_drafts_and_their_refusal(dim, block, odd):
    """Drafts of which one has an odd value (or key), all queries at once; then without the
    refused ones, before anything new arrives and after it."""
    w = World(4, heads=2, dim=dim, block=block, cols=5, seed=dim + block, rot=0)
    w.append([block + 5, 3, 2 * block + block // 2, 0])
    for where in ("v", "k"):
        rows = {"k": w.rows(16), "v": w.rows(16)}
        x = rows[where]
        small = np.float32(np.clip(odd, -1e10, 1e10)) if where == "k" else np.float32(odd)
        x[2, 1, 7] = small              # sequence 0: its third draft, one column
        x[4, 0, [0, dim - 1]] = small   # 1: the first, two columns
        x[11, :, 5] = small             # 2: the last, both heads
        x[12, 1, 3] = small             # 3: its first token of all
        w.append([4, 4, 4, 4], rows["k"], rows["v"])
        for kw in ({}, dict(chunk=64), dict(window=3)):
            check(w, [4, 4, 4, 4], w.rows(16, 4), **kw)
            check(w, [1, 1, 1, 1], w.rows(4, 6), **kw)
        for r, n in zip(w.ref, (2, 4, 1, 4)):
            r.cut(len(r.k) - n)
        check(w, [1, 1, 1, 0], w.rows(3, 4))
        check(w, [2, 3, 4, 0], w.rows(9, 4), chunk=64)
        w.append([1, 2, 1, 1])
        w.check()
        check(w, [1, 2, 1, 1], w.rows(5, 4))
        for r, n in zip(w.ref, (block + 5, 3, 2 * block + block // 2, 0)):
            r.cut(n)
    w.append([block, block, block, block])
    w.check()


@pytest.mark.parametrize("odd", [float("nan"), float("inf")])
def test_a_complete_block_with_an_odd_row(odd):
    """Its codes are no numbers, for every row that sees a token of the block; rows that
    see none of it, and its neighbours, are as ever."""
    w = World(2, heads=2, dim=64, block=16, cols=8, rot=0)
    rows = {"k": w.rows(200), "v": w.rows(200)}
    rows["v"][20, 0, 3] = odd       # sequence 0, block 1, head 0
    rows["k"][100 + 40, 1, 9] = odd   # 1, block 2, head 1
    w.append([100, 100], rows["k"], rows["v"])
    w.ref[0].v[16:32, 0], w.ref[1].k[32:48, 1] = 0.0, 0.0   # (the rest is compared)
    k, v = (x.cpu().numpy() for x in heal.heal_kv_read(w.cache, 200, cu=dev(np.int32([0, 100, 200])), **w.kw()))
    bad = np.zeros((200, 2), bool)
    bad[16:32, 0] = True
    assert np.array_equal(np.isnan(v).all(2), bad) and np.array_equal(np.isnan(v).any(2), bad)
    bad[:] = False
    bad[132:148, 1] = True
    assert np.array_equal(np.isnan(k).all(2), bad) and np.array_equal(np.isnan(k).any(2), bad)
    q = w.rows(100, 4)
    for window in (0, 10):
        out, lse = attention(w, [100, 0], q, window=window)
        first = 31 if window == 0 else 31 + window
        place = np.arange(100)
        sees = (place >= 16) & ((place < first) | (window == 0))
        assert np.array_equal(np.isnan(out).all(2), sees[:, None] & (np.arange(4) < 2))
        assert np.array_equal(np.isnan(out).any(2), np.isnan(out).all(2)) and np.isfinite(lse).all()
        out, lse = attention(w, [0, 100], q, window=window)
        sees = (place >= 32) & ((place < 47 + window) | (window == 0))
        assert np.array_equal(np.isnan(out).all(2), sees[:, None] & (np.arange(4) >= 2))
        assert np.array_equal(np.isnan(out).any(2), np.isnan(out).all(2)) and np.array_equal(np.isnan(lse), np.isnan(out).any(2))


@pytest.mark.parametrize("odd", ODD)
@pytest.mark.parametrize("dim,block", [(64, 16), (96, 32), (128, 64), (64, 128), (128, 16)])
def test_prompts(dim, block, odd):
    """Prompts (tiles of 128 rows) whose last block has an odd row, and without it."""
    heads, group = (8, 4) if dim != 96 else (5, 7)
    w = World(20, heads=heads, dim=dim, block=block, cols=-(-230 // block), seed=dim * block, rot=0)
    counts = [100 + 3 * i + (0 if (100 + 3 * i) % block else 1) for i in range(20)]
    rows = {"k": w.rows(sum(counts)), "v": w.rows(sum(counts))}
    first, at = [], 0
    for i, n in enumerate(counts):
        start = n // block * block
        first.append(start + (n - start) // 2)   # the odd row
        x = rows["v" if i % 3 else "k"]
        value = np.float32(np.clip(odd, -1e10, 1e10)) if i % 3 == 0 else np.float32(odd)
        x[at + first[i], i % heads, (5 * i) % dim] = value
        at += n
    w.append(counts, rows["k"], rows["v"])
    check(w, counts, w.rows(sum(counts), heads * group), some=True)
    check(w, counts, w.rows(sum(counts), heads * group), some=True, window=70)
    for r, n in zip(w.ref, first):
        r.cut(n)
    counts = [min(len(r.k), 90 + i) for i, r in enumerate(w.ref)]
    check(w, counts, w.rows(sum(counts), heads * group), some=True)


def test_a_shared_tile_of_coded_and_other_blocks():
    """Blocks of 16: one tile of 64 tokens with coded blocks, a block that is not held and
    the last rows, far apart in size."""
    w = World(18, heads=8, dim=64, block=16, cols=12, rot=0, seed=3)
    counts = [120 + i for i in range(18)]
    rows = [w.rows(sum(counts)) for _ in range(2)]
    at = 0
    for i, n in enumerate(counts):
        for b in range(0, n, 16):
            rows[1][at + b:min(at + b + 16, at + n)] *= np.float32([1.0, 1e-3, 30.0, 1e4][(b // 16 + i) % 4])
        at += n
    w.append(counts, *rows)
    check(w, counts, w.rows(sum(counts), 32))
    check(w, [3] * 18, w.rows(54, 32))
