"""The key/value cache on the GPU against its definition in 64 bits (tests/kv_ref.py)."""
import numpy as np
import pytest
import torch

import kv_ref
import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

NAN = float("nan")


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


class World:
    """A cache on the GPU and what it should hold.  The arrays start as NaN and any
    codes, pages and slots are handed out in a shuffled order."""

    def __init__(self, seqs, heads=2, dim=64, block=16, cols=12, seed=0, sigma=1.0, places=4096, rot=None,
                 interleaved=False):
        self.rng = np.random.default_rng(seed)
        self.seqs, self.heads, self.dim, self.block, self.cols = seqs, heads, dim, block, cols
        blocks = seqs * cols + 3
        self.cache = heal.KVCache.empty(blocks, seqs + 2, heads, dim, block)
        for t in (self.cache.scales, self.cache.k_mean, self.cache.k_recent, self.cache.v_recent):
            t.fill_(NAN)
        for t in (self.cache.k_codes, self.cache.v_codes):
            t.copy_(torch.randint(-128, 128, t.shape, device="cuda"))
        self.table = self.rng.permutation(blocks)[:seqs * cols].reshape(seqs, cols).astype(np.int32)
        self.slots = self.rng.permutation(seqs + 2)[:seqs].astype(np.int32)
        self.ref = [kv_ref.Sequence(heads, dim, block) for _ in range(seqs)]
        self.ring = [{} for _ in range(seqs)]   # the place whose row is at p % (2 * block)
        self.sigma, self.interleaved = sigma, interleaved
        self.cos = self.sin = None
        rot = dim if rot is None else rot
        if rot:
            angle = np.arange(places)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
            self.cos, self.sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)

    def lens(self):
        return [len(r.k) for r in self.ref]

    def kw(self, lens=None):
        return {"table": dev(self.table), "lens": ints(self.lens() if lens is None else lens),
                "slots": dev(self.slots)}

    def rows(self, n, heads=None):
        return (self.sigma * self.rng.standard_normal((n, heads or self.heads, self.dim))).astype(np.float32)

    def append(self, counts, k=None, v=None, q=None):
        """counts[i] new tokens for sequence i, in one call."""
        T = sum(counts)
        k, v = self.rows(T) if k is None else k, self.rows(T) if v is None else v
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        for i, r in enumerate(self.ref):
            n = len(r.k)
            r.append(k[cu[i]:cu[i + 1]], v[cu[i]:cu[i + 1]], self.cos, self.sin, self.interleaved)
            for p in range(n, len(r.k)):
                self.ring[i][p % (2 * self.block)] = p
        announce("append %s to %s" % (counts, self.lens()))
        one = all(c == 1 for c in counts)
        out = heal.heal_kv_append(self.cache, dev(k), dev(v), cu=None if one else dev(cu), **self.kw(),
                                  cos=None if self.cos is None else dev(self.cos),
                                  sin=None if self.sin is None else dev(self.sin),
                                  interleaved=self.interleaved, q=None if q is None else dev(q))
        torch.cuda.synchronize()
        return out

    def check(self):
        """Every block that a sequence holds, bit for bit."""
        c = self.cache
        kc, vc, sc, mean = (t.cpu().numpy() for t in (c.k_codes, c.v_codes, c.scales, c.k_mean))
        kr, vr = c.k_recent.cpu().numpy(), c.v_recent.cpu().numpy()
        B = self.block
        order = np.array([t % 16 // 4 * (B // 4) + t // 16 * 4 + t % 4 for t in range(B)])
        for i, r in enumerate(self.ref):
            n = len(r.k)
            if n:
                m = r.means()
            for b in range(-(-n // B)):
                page = self.table[i, b]
                k, v = r.k[b * B:(b + 1) * B], r.v[b * B:(b + 1) * B]
                assert np.array_equal(sc[page, :, 0], np.abs(k).max((0, 2))), (i, b)
                assert np.array_equal(sc[page, :, 1], np.abs(v).max((0, 2))), (i, b)
                # an FP64 sum rounded once: half an FP32 step (2^-24 of the value, and 2^-150
                # below 2^-126, where the step stays 2^-149) and the sum's own error
                limit = 2.0 ** -24 * np.abs(m[b]) + 2.0 ** -150 + 2.0 ** -47 * np.abs(k).max()
                assert np.all(np.abs(mean[page] - m[b]) <= limit), (i, b)
                if n >= b * B + B:
                    assert np.array_equal(kc[page].transpose(1, 0, 2), r.block_codes(b, "k")[0]), (i, b)
                    assert np.array_equal(vc[page][..., order].transpose(2, 0, 1), r.block_codes(b, "v")[0]), (i, b)
            # the rows of the last two blocks, but for those whose place in the ring a later
            # block has taken (before the sequence was cut back)
            first = max(0, ((n - 1) // B - 1) * B) if n else 0
            for p in range(first, n):
                if self.ring[i].get(p % (2 * B), p) != p:
                    assert p < n // B * B
                    continue
                assert np.array_equal(kr[self.slots[i], :, p % (2 * B)], r.k[p]), (i, p)
                assert np.array_equal(vr[self.slots[i], :, :, p % (2 * B)], r.v[p]), (i, p)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_append_bits(dim, block):
    """Prompts of any length, one token at a time, drafts, and a prompt that spans many
    blocks after a block that has begun."""
    w = World(4, heads=3, dim=dim, block=block, cols=9, seed=dim + block, interleaved=dim == 96)
    w.append([1, block, 2 * block + 5, 0])
    w.check()
    w.append([1, 1, 1, 1])
    w.check()
    w.append([block - 2, 3, block - 6, 7])
    w.check()
    w.append([3 * block + 7, 2 * block, 0, 4 * block - 9])
    w.check()
    w.append([1, 1, 1, 1])
    w.check()


def test_bits_do_not_depend_on_the_calls():
    """One call for everything, tokens one by one, and pieces of any size: the same cache."""
    n, got = 83, []
    rng = np.random.default_rng(7)
    k, v = (rng.standard_normal((n, 2, 64)).astype(np.float32) for _ in range(2))
    for pieces in ([n], [1] * n, [17, 31, 2, 20, 13], [5] * 16 + [3]):
        w = World(1, seed=1)
        at = 0
        for p in pieces:
            w.append([p], k[at:at + p], v[at:at + p])
            at += p
        w.check()
        pages = w.table[0, :6]
        c = w.cache
        got.append([t[pages].cpu() for t in (c.k_codes[:, :, :, :], c.v_codes, c.scales, c.k_mean)])
    for other in got[1:]:
        assert torch.equal(got[0][2], other[2]) and torch.equal(got[0][3], other[3])
        for j in range(2):   # the sixth block is not complete: no codes
            assert torch.equal(got[0][j][:5], other[j][:5])


@pytest.mark.parametrize("rot,interleaved", [(0, False), (2, False), (2, True), (48, True), (64, False), (64, True)])
def test_rotation_and_queries(rot, interleaved):
    w = World(3, seed=rot, rot=rot, interleaved=interleaved, places=40)
    for counts in ([5, 0, 39], [1, 1, 1], [2, 9, 3]):   # the last places are past the table
        T = sum(counts)
        q = w.rows(T, 5)
        start = w.lens()
        out = w.append(counts, q=q).cpu().numpy()
        t = 0
        for i, n in enumerate(counts):
            for j in range(n):
                assert np.array_equal(out[t], kv_ref.rotate(q[t], start[i] + j, w.cos, w.sin, interleaved))
                t += 1
        w.check()


def test_queries_in_place_and_strided_inputs():
    """k and v as views of one fused projection, in rows that are not 16-byte aligned;
    q rotated where it is."""
    for pad in (0, 1):
        w = World(2, heads=2, dim=96, block=32, seed=pad)
        T, width = 70, 4 * 96 + 2 * 96 + 2 * 96 + pad
        x = w.rng.standard_normal((T, width)).astype(np.float32)
        g = dev(x)
        part = lambda y, lo, h: y[:, lo * 96:(lo + h) * 96].reshape(T, h, 96)  # noqa: E731
        view = lambda lo, h: g[:, lo * 96:(lo + h) * 96].unflatten(1, (h, 96))  # noqa: E731
        w.ref[0].append(part(x, 4, 2)[:45], part(x, 6, 2)[:45], w.cos, w.sin)
        w.ref[1].append(part(x, 4, 2)[45:], part(x, 6, 2)[45:], w.cos, w.sin)
        q = view(0, 4)
        announce("fused projection, pad %d" % pad)
        out = heal.heal_kv_append(w.cache, view(4, 2), view(6, 2), cu=ints([0, 45, 70]), **w.kw(), cos=dev(w.cos),
                                  sin=dev(w.sin), q=q, q_out=q)
        assert out is q
        w.check()
        want = np.stack([kv_ref.rotate(part(x, 0, 4)[t], t if t < 45 else t - 45, w.cos, w.sin, False)
                         for t in range(T)])
        assert np.array_equal(q.cpu().numpy(), want)
        assert np.array_equal(g[:, 4 * 96:].cpu().numpy(), x[:, 4 * 96:])


def test_values_at_the_edges():
    """Ties between codes, zeros, subnormal and huge numbers, one large element."""
    B = 16
    w = World(1, heads=6, dim=64, block=B, rot=0)
    k = w.rows(B)
    k[:, 0] = 0.0
    k[:, 1] = np.round(k[:, 1] * 20) / 2.0   # with m = 127: halves are ties
    k[0, 1, 0] = 127.0
    k[:, 2] *= np.float32(1e-42)
    k[:, 3] *= np.float32(1e37)
    k[:, 4] *= np.float32(1e-30)
    k[5, 4, 7] = -1.0
    k[:, 5] = np.float32(2.0 ** -149)
    w.append([B], k, k.copy())
    w.check()
    got, _ = heal.heal_kv_read(w.cache, B, **w.kw(), cu=ints([0, B]))
    assert np.abs(got.cpu().numpy()[:, 5]).max() <= 2.0 ** -148


def test_cut_back_and_go_on():
    """Refused drafts: the length goes back, over a block's end too, and on again."""
    w = World(2, block=16, cols=8)
    w.append([30, 15])
    for counts, keep in (([4, 4], [31, 16]), ([1, 1], [32, 17]), ([8, 20], [33, 18]), ([14, 14], [40, 20]),
                         ([16, 16], [48, 21])):
        w.append(counts)
        w.check()
        for r, n in zip(w.ref, keep):
            r.cut(n)
        q = w.rows(2, 4)
        _check_attention(w, [1, 1], q)


def test_read():
    w = World(3, heads=2, dim=96, block=32, cols=5, seed=5)
    w.append([100, 0, 33])
    for counts in ([100, 0, 33], [1, 0, 1], [37, 0, 2], [64, 0, 32], [5, 0, 0]):
        T = sum(counts)
        cu = np.concatenate([[0], np.cumsum(counts)])
        announce("read %s" % counts)
        k, v = (t.cpu().numpy().astype(np.float64) for t in heal.heal_kv_read(w.cache, T, cu=ints(cu.tolist()), **w.kw()))
        for i, r in enumerate(w.ref):
            for got, name in ((k, "k"), (v, "v")):
                want = r.values(name)[len(r.k) - counts[i]:]
                # m / 127 and the product are rounded
                assert np.all(np.abs(got[cu[i]:cu[i + 1]] - want) <= 2 * 2.0 ** -24 * np.abs(want))
    # more tokens than there are: zeros in front
    k, v = heal.heal_kv_read(w.cache, 50, cu=ints([0, 0, 10, 50]), **w.kw())
    assert not k[:17].any() and not v[:17].any()
    assert torch.equal(k[17:].cpu(), heal.heal_kv_read(w.cache, 33, cu=ints([0, 0, 0, 33]), **w.kw())[0].cpu())


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_read_a_few_rows(dim, block):
    """The last 1, 8, 9 and more rows of blocks that are not complete, as they came."""
    w = World(3, heads=2, dim=dim, block=block, cols=3, seed=dim + block)
    w.append([block + 13, block - 1, 2 * block + 15])
    for n in (1, 2, 8, 9, 13):
        announce("the last %d rows" % n)
        got = heal.heal_kv_read(w.cache, 3 * n, cu=ints([0, n, 2 * n, 3 * n]), **w.kw())
        for t, name in zip(got, ("k", "v")):
            t = t.cpu().numpy()
            for i, r in enumerate(w.ref):
                assert np.array_equal(t[i * n:(i + 1) * n], getattr(r, name)[len(r.k) - n:]), (n, i, name)


def test_a_shared_beginning():
    """Sequences that list the same complete blocks and go on in their own."""
    w = World(1, heads=2, dim=64, block=32, cols=4, seed=8)
    k, v = w.rows(64 + 40), w.rows(64 + 40)
    w.append([64], k[:64], v[:64])
    table = np.concatenate([w.table, w.table])
    spare = sorted(set(range(7)) - set(w.table[0].tolist()))
    table[1, 2:] = spare[:2]
    slots = [int(w.slots[0]), (int(w.slots[0]) + 1) % 3]
    kw = {"table": dev(table), "lens": ints([64 + 40, 64 + 40]), "slots": ints(slots), "cu": ints([0, 40, 80])}
    announce("append behind a shared beginning")
    two = lambda x: dev(np.concatenate([x[64:], x[64:]]))  # noqa: E731
    heal.heal_kv_append(w.cache, two(k), two(v), cos=dev(w.cos), sin=dev(w.sin), **kw)
    w.ref[0].append(k[64:], v[64:], w.cos, w.sin, w.interleaved)
    for p in range(64, 104):
        w.ring[0][p % 64] = p
    w.check()
    q = dev(w.rows(40, 4))
    out = heal.heal_kv_attention(w.cache, torch.cat([q, q]), **kw)
    assert torch.equal(out[:40], out[40:])
    _check_attention(w, [40], q.cpu().numpy())


# ---- attention ------------------------------------------------------------------


def _check_attention(w, counts, q, scale=None, causal=True, window=0, sel=None, lens=None, hidden=(), **kw):
    """heal_kv_attention of the last counts[i] tokens of every sequence; hidden:
    (sequence, block) that the cache does not hold."""
    T, heads_q = q.shape[0], q.shape[1]
    G = heads_q // w.heads
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    out = torch.full((T, heads_q, w.dim), 7.0, device="cuda")
    lse = torch.full((T, heads_q), 7.0, device="cuda")
    one = all(c == 1 for c in counts) and kw.pop("no_cu", True)
    announce("attention %s of %s, %s causal %s window %d %s" % (counts, w.lens(), q.shape, causal, window, kw))
    got = heal.heal_kv_attention(w.cache, dev(q), **w.kw(lens), cu=None if one else dev(cu), scale=scale, causal=causal,
                                 window=window, sel=None if sel is None else dev(sel), out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    assert got is out
    out, lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    scale = w.dim ** -0.5 if scale is None else scale
    for i, r in enumerate(w.ref):
        K, V, n = r.values("k"), r.values("v"), len(r.k)
        for j in range(counts[i]):
            t, place = cu[i] + j, n - counts[i] + j
            at = np.arange(n)
            seen = (at <= place) if causal else np.full(n, place >= 0)
            if window:
                seen = seen & (at > place - window)
            for i2, b in hidden:
                if i2 == i:
                    seen = seen & (at // w.block != b)
            for h in range(heads_q):
                many = seen.astype(np.float64)
                if sel is not None:
                    times = np.array([(sel[t, h // G] == b).sum() for b in range(w.cols)])
                    many = many * times[at // w.block]
                o, e, S, A = kv_ref.attention(q[t, h], K[:, h // G], V[:, h // G], scale, many)
                Ks, x = np.abs(K[many > 0, h // G]), np.abs(q[t, h]).astype(np.float64)
                top = lambda y: y.max() if y.size else 0.0  # noqa: E731
                # the largest value of the blocks that are seen (of an incomplete one all rows count)
                met = np.unique(np.nonzero(many)[0] // w.block)
                v = top(np.abs(r.v[np.isin(at // w.block, met), h // G]))
                rel, floor, lse_off = kv_ref.bound(S, max(1, many.sum()), w.dim, abs(scale) * x.max() * top(Ks.sum(1)),
                                                   abs(scale) * x.sum() * top(Ks), float(v))
                assert np.all(np.abs(out[t, h] - o) <= rel * A + floor), (i, j, h, np.abs(out[t, h] - o).max())
                if np.isinf(e):
                    assert lse[t, h] == e, (i, j, h)
                else:
                    assert abs(lse[t, h] - e) <= lse_off + 2.0 ** -23 * abs(e), (i, j, h, lse[t, h], e)
    return out


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("group", [1, 3, 4])
def test_single_tokens(dim, block, group):
    w = World(7, heads=2, dim=dim, block=block, cols=-(-400 // block), seed=dim + block + group)
    w.append([1, block - 1, block, block + 1, 65, 130, 399])
    _check_attention(w, [1] * 7, w.rows(7, 2 * group))
    _check_attention(w, [1] * 7, w.rows(7, 2 * group), chunk=64)
    _check_attention(w, [1] * 7, w.rows(7, 2 * group), window=50, chunk=128)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_drafts_and_prompts(dim, block):
    w = World(5, heads=2, dim=dim, block=block, cols=-(-300 // block), seed=dim + block)
    w.append([1, 37, 150, 64, 290])
    counts = [1, 5, 150, 0, 33]
    for group, kw in ((1, {}), (4, {}), (3, dict(window=40)), (2, dict(causal=False)), (5, dict(chunk=64))):
        _check_attention(w, counts, w.rows(sum(counts), 2 * group), **kw)


@pytest.mark.parametrize("group", [8, 15, 16, 17, 40])
def test_many_queries_of_one_head(group):
    w = World(2, heads=1, dim=64, block=32, cols=5, seed=group)
    w.append([70, 129])
    _check_attention(w, [1, 1], w.rows(2, group))
    _check_attention(w, [3, 20], w.rows(23, group))


@pytest.mark.parametrize("heads", [1, 5])
def test_odd_heads_and_every_short_length(heads):
    lens = list(range(1, 36))
    w = World(len(lens), heads=heads, dim=64, block=16, cols=3)
    w.append(lens)
    _check_attention(w, [1] * len(lens), w.rows(len(lens), heads))
    _check_attention(w, lens, w.rows(sum(lens), heads))


@pytest.mark.parametrize("window", [1, 15, 16, 17, 64, 100, 1000])
def test_windows(window):
    w = World(3, dim=64, block=32, cols=10)
    w.append([10, 150, 300])
    _check_attention(w, [1, 1, 1], w.rows(3, 4), window=window)
    _check_attention(w, [10, 20, 140], w.rows(170, 4), window=window)
    with pytest.raises(heal.HealError):
        heal.heal_kv_attention(w.cache, dev(w.rows(3, 4)), **w.kw(), window=window, causal=False)


def test_rows_that_see_nothing():
    """Unused places of the batch (length 0), and more tokens than the length."""
    w = World(4, cols=5)
    w.append([0, 20, 0, 3])
    out = _check_attention(w, [1, 1, 1, 1], w.rows(4, 4))
    assert not out[0].any() and not out[2].any()
    _check_attention(w, [3, 25, 1, 40], w.rows(69, 4))
    _check_attention(w, [3, 25, 1, 40], w.rows(69, 4), causal=False, chunk=64)


@pytest.mark.parametrize("scale", [0.0, -0.7, 3.0, 1e-30])
def test_scales(scale):
    w = World(2, cols=8)
    w.append([100, 40])
    _check_attention(w, [1, 1], w.rows(2, 4), scale=scale)


@pytest.mark.parametrize("kind", ["k", "v", "q"])
def test_magnitudes_from_row_to_row(kind):
    """Blocks (rows) whose numbers differ by many orders of magnitude, and zeros."""
    w = World(1, heads=2, dim=64, block=16, cols=16, rot=0)
    n = 230
    x = {"k": w.rows(n), "v": w.rows(n)}
    q = w.rows(8, 4)
    powers = np.array([1e-20, 1e3, 0.0, 1.0, 1e-38, 1e-3, 1e-8, 30.0, 0.0, 1e-12, 1e4, 1.0, 1e-2, 0.0, 1e-44])
    if kind == "q":
        q *= powers[:8, None, None].astype(np.float32)
        q[:, :, ::2] *= np.float32(1e-5)
    else:
        x[kind] *= np.repeat(powers, 16)[:n, None, None].astype(np.float32)
    w.append([n], x["k"], x["v"])
    w.check()
    scale = 1e-3 if kind != "v" else None
    _check_attention(w, [8], q, scale=scale)
    _check_attention(w, [8], q, scale=scale, chunk=64)
    if kind == "v":   # large values only at places that the first queries do not see
        _check_attention(w, [8], q, window=20)


def test_anything_behind_the_last_token():
    """NaN and infinities in the ring behind the last row, in pages of no sequence, and
    in a row's neighbours: a row's result does not change."""
    w = World(2, dim=64, block=16, cols=4)
    w.append([21, 37])
    q = w.rows(2, 4)
    a = _check_attention(w, [1, 1], q)
    c = w.cache
    c.k_recent[int(w.slots[0]), :, 21:] = NAN
    c.v_recent[int(w.slots[0]), :, :, 21:] = float("inf")
    unused = [p for p in range(c.blocks) if p not in set(w.table[0, :2]) | set(w.table[1, :3])]
    c.scales[unused] = NAN
    c.k_codes[unused] = -128
    w.table[0, 2:] = -1
    w.table[1, 3:] = 1 << 30
    assert np.array_equal(_check_attention(w, [1, 1], q), a)
    q[0, 0, 3] = NAN
    announce("a row that holds a NaN")
    b = heal.heal_kv_attention(c, dev(q), **w.kw()).cpu().numpy()
    assert np.isnan(b[0, 0]).all() and np.array_equal(b[0, 1:], a[0, 1:]) and np.array_equal(b[1], a[1])


def test_pages_that_are_not_there():
    """Table entries out of range, and slots out of range: those tokens are not seen."""
    w = World(3, dim=64, block=16, cols=6)
    w.append([50, 90, 20])
    q = w.rows(3, 4)
    keep = w.table.copy()
    w.table[0, 1], w.table[1, 4], w.table[1, 0], w.table[2, 1] = -5, w.cache.blocks, 2 ** 31 - 1, -2 ** 31
    _check_attention(w, [1, 1, 1], q, hidden=[(0, 1), (1, 4), (1, 0), (2, 1)])
    k, v = heal.heal_kv_read(w.cache, 160, cu=ints([0, 50, 140, 160]), **w.kw())
    assert not k[16:32].any() and not v[50:66].any() and k[:16].any() and not k[156:].any()
    w.table = keep
    w.slots = np.array([-1, 5, 2 ** 31 - 1], np.int32)
    _check_attention(w, [1, 1, 1], q, hidden=[(0, 3), (1, 5), (2, 1)])


def test_append_writes_nothing_elsewhere():
    """Bad pages and slots, places past the table, tokens of no sequence: everything else
    keeps its bits."""
    w = World(4, dim=64, block=16, cols=2)
    w.append([10, 10, 10, 10])
    c = w.cache
    arrays = (c.k_codes, c.v_codes, c.scales, c.k_mean, c.k_recent, c.v_recent)
    before = [t.clone() for t in arrays]
    table, slots = w.table.copy(), w.slots.copy()
    table[0] = [-1, 1 << 30]
    slots[1] = 99
    T = 60
    k = dev(w.rows(T))
    q = dev(w.rows(T, 4))
    q_out = torch.full_like(q, 5.0)
    announce("append with bad entries")
    # sequence 0: bad pages; 1: a bad slot; 2: goes past its table; 3: negative places
    heal.heal_kv_append(c, k, k, dev(table), ints([30, 12, 45, 2]), cu=ints([4, 24, 26, 46, 50]), slots=dev(slots),
                        q=q, q_out=q_out)
    torch.cuda.synchronize()
    assert (q_out[:4] == 5.0).all() and (q_out[50:] == 5.0).all() and torch.equal(q_out[4:50], q[4:50])
    touched = [set(), set(w.table[1, :1]), set(w.table[2]), set(w.table[3, :1])]
    pages = set().union(*touched)
    others = [p for p in range(c.blocks) if p not in pages]
    for t, b in list(zip(arrays, before))[:4]:
        assert torch.equal(t[others].view(torch.uint8), b[others].view(torch.uint8))
    free = [s for s in range(c.slots) if s not in set(w.slots[[0, 2, 3]])]
    for t, b in list(zip(arrays, before))[4:]:
        assert torch.equal(t[free].view(torch.uint8), b[free].view(torch.uint8))


def test_tokens_of_no_sequence_are_left_alone():
    w = World(2, dim=64, block=16, cols=6)
    w.append([40, 90])
    for chunk in (0, 64):
        q = w.rows(20, 4)
        out = torch.full((20, 4, 64), 7.0, device="cuda")
        lse = torch.full((20, 4), 7.0, device="cuda")
        sel = torch.full((20, 2, 2), 9, dtype=torch.int32, device="cuda")
        cu = ints([3, 5, 16])
        announce("rows of no sequence, chunk %d" % chunk)
        heal.heal_kv_attention(w.cache, dev(q), cu=cu, **w.kw(), out=out, lse=lse, chunk=chunk)
        heal.heal_kv_select(w.cache, dev(q), 2, cu=cu, **w.kw(), out=sel)
        for x, y in ((out, 7.0), (lse, 7.0), (sel, 9)):
            assert (x[:3] == y).all() and (x[16:] == y).all() and not (x[3:16] == y).any()


def test_lengths_past_the_table():
    """Places that the table has no block for hold nothing, without columns no place does."""
    w = World(2, dim=64, block=16, cols=4)
    w.append([50, 64])
    q = w.rows(2, 4)
    kw = w.kw([50, 64 + 37])      # the second length is 37 past the table: its query sees all 64
    announce("lengths past the table")
    out = heal.heal_kv_attention(w.cache, dev(q), **kw).cpu().numpy()
    K, V = w.ref[1].values("k"), w.ref[1].values("v")
    for h in range(4):
        o, _, S, A = kv_ref.attention(q[1, h], K[:, h // 2], V[:, h // 2], 0.125, np.ones(64))
        rel, floor, _ = kv_ref.bound(S, 64, 64, v=float(np.abs(V).max()) * 1.01)
        assert np.all(np.abs(out[1, h] - o) <= rel * A + floor)
    sel = heal.heal_kv_select(w.cache, dev(q), 4, **kw).cpu().numpy()
    assert (sel == [0, 1, 2, 3]).all()
    none = dict(kw, table=kw["table"][:, :0])
    for x in (w.rows(2, 4), w.rows(80, 4)):
        cu = ints([0, len(x) // 2, len(x)])
        assert not heal.heal_kv_attention(w.cache, dev(x), **none, cu=cu).any()
        assert (heal.heal_kv_select(w.cache, dev(x), 3, **none, cu=cu) == -1).all()
        k, v = heal.heal_kv_read(w.cache, len(x), **none, cu=cu)
        assert not k.any() and not v.any()


def test_calls_without_tokens():
    w = World(2, dim=64, block=16, cols=4)
    w.append([5, 6])
    kw, cu, q = dict(w.kw(), cu=ints([0, 0, 0])), ints([0, 0, 0]), torch.empty(0, 4, 64, device="cuda")
    assert heal.heal_kv_append(w.cache, q[:, :2], q[:, :2], **kw, q=q).shape == (0, 4, 64)
    assert heal.heal_kv_attention(w.cache, q, **kw).shape == (0, 4, 64)
    assert heal.heal_kv_select(w.cache, q, 3, **kw).shape == (0, 2, 3)
    assert heal.heal_kv_read(w.cache, 0, **kw)[0].shape == (0, 2, 64)
    w.check()


def test_strided_queries_and_outputs():
    w = World(2, heads=2, dim=96, block=32, cols=4)
    w.append([40, 77])
    q = w.rows(9, 6)
    want = heal.heal_kv_attention(w.cache, dev(q), cu=ints([0, 2, 9]), **w.kw())
    for pad in (0, 1, 4):
        wide = torch.full((6, 9, 96 + pad), 3.0, device="cuda")
        wide[:, :, :96] = dev(q).transpose(0, 1)
        out = torch.full((9, 6 * 96 + pad), 3.0, device="cuda")
        view = out[:, :576].unflatten(1, (6, 96))
        announce("strides, pad %d" % pad)
        heal.heal_kv_attention(w.cache, wide[:, :, :96].transpose(0, 1), cu=ints([0, 2, 9]), **w.kw(), out=view)
        assert torch.equal(view, want) and (out[:, 576:] == 3.0).all()
    with pytest.raises(heal.HealError):
        heal.heal_kv_attention(w.cache, dev(q), cu=ints([0, 2, 9]), **w.kw(),
                               out=torch.empty(1, 6, 96, device="cuda").expand(9, 6, 96))


@pytest.mark.parametrize("block,n_sel", [(16, 3), (16, 9), (32, 1), (64, 5), (128, 2)])
def test_listed_blocks(block, n_sel):
    """Lists with -1 anywhere, numbers past the table, and a block listed twice."""
    w = World(3, heads=3, dim=64, block=block, cols=6, seed=n_sel)
    w.append([block * 4 + 3, 5, block * 6])
    for counts, G in (([1, 1, 1], 2), ([4, 2, 7], 4), ([1, 1, 1], 18)):
        T = sum(counts)
        sel = w.rng.integers(-2, 8, (T, 3, n_sel)).astype(np.int32)
        sel[:, 0] = -1
        sel[0, 1, 0] = 2 ** 31 - 1
        _check_attention(w, counts, w.rows(T, 3 * G), sel=sel)
        _check_attention(w, counts, w.rows(T, 3 * G), sel=sel, chunk=64, window=70)


def test_all_blocks_listed_is_all_blocks():
    w = World(2, heads=2, dim=128, block=64, cols=4)
    w.append([200, 130])
    q = dev(w.rows(2, 8))
    sel = torch.arange(4, dtype=torch.int32, device="cuda").expand(2, 2, 4).contiguous()
    assert torch.equal(heal.heal_kv_attention(w.cache, q, **w.kw(), sel=sel, chunk=64),
                       heal.heal_kv_attention(w.cache, q, **w.kw(), chunk=64))


def test_chunk_makes_bits_independent_of_the_batch():
    w = World(6, heads=2, dim=128, block=64, cols=20, seed=3)
    w.append([700, 64, 1200, 1, 300, 999])
    q = dev(w.rows(6, 8))
    for chunk in (64, 256, 1024):
        whole = heal.heal_kv_attention(w.cache, q, **w.kw(), chunk=chunk)
        for i in (0, 2, 5):
            kw = {k: v[i:i + 1].contiguous() for k, v in w.kw().items()}
            kw["table"] = kw["table"][:, :19 + i % 2].contiguous()
            assert torch.equal(heal.heal_kv_attention(w.cache, q[i:i + 1], **kw, chunk=chunk)[0], whole[i])
    assert torch.equal(heal.heal_kv_attention(w.cache, q, **w.kw()), heal.heal_kv_attention(w.cache, q, **w.kw()))


def test_long_sequence():
    """20001 tokens, a few queries; more chunks than a wave has lanes."""
    w = World(1, heads=1, dim=64, block=128, cols=160, places=20100)
    w.append([20001])
    w.check()
    _check_attention(w, [1], w.rows(1, 4))
    _check_attention(w, [3], w.rows(3, 4), chunk=128)


def test_offsets_past_32_bits():
    """A cache whose codes, scales and ring rows lie past 2^32 bytes, pages at its end."""
    blocks, slots = 70000, 70000
    c = heal.KVCache.empty(blocks, slots, 8, 128, 64)      # 4.6 GB of codes each, 37 GB of ring rows each
    w = World(2, heads=8, dim=128, block=64, cols=3)
    w.cache = c
    w.table = np.array([[blocks - 1, blocks - 3, 7], [blocks - 2, 0, blocks - 4]], np.int32)
    w.slots = np.array([slots - 1, 3], np.int32)
    w.append([100, 150])
    _check_attention(w, [1, 1], w.rows(2, 8))
    q = w.rows(2, 8)
    sel = heal.heal_kv_select(c, dev(q), 2, **w.kw()).cpu().numpy()
    assert (sel[0] == [0, 1]).all() and (sel[1] == [0, 2]).all()


# ---- prompts: 128-row tiles ------------------------------------------------------


def _check_prompts(w, counts, group, causal=True, window=0, tile=128, hidden=(), strided=False):
    """As _check_attention for many rows at a time, of a call that takes 128-row tiles."""
    import ctypes
    T, heads_q = sum(counts), w.heads * group
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    kw = w.kw()
    batch = heal._CBatch(w.seqs, T, 1, 1, 1, w.cols, w.cols, 1)
    assert heal.lib().heal_kv_attention_tile(w.cache._ref, ctypes.byref(batch), heads_q, window, 0, 0) == tile
    q = w.rows(T, heads_q)
    g = dev(q)
    out = torch.full((T, heads_q, w.dim), 7.0, device="cuda")
    if strided:   # heads outermost, rows that are not 16-byte aligned
        g = torch.nn.functional.pad(g.transpose(0, 1), (0, 1)).contiguous()[..., :-1].transpose(0, 1)
        out = torch.full((heads_q, T, w.dim + 1), 7.0, device="cuda")[..., :-1].transpose(0, 1)
    lse = torch.full((T, heads_q), 7.0, device="cuda")
    announce("prompts %s of %s, %s causal %s window %d" % (counts, w.lens(), q.shape, causal, window))
    heal.heal_kv_attention(w.cache, g, cu=dev(cu), **kw, causal=causal, window=window, out=out, lse=lse)
    torch.cuda.synchronize()
    out, lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(g.cpu().numpy(), q)
    scale = w.dim ** -0.5
    for i, r in enumerate(w.ref):
        n, t = len(r.k), counts[i]
        if not t:
            continue
        rows = slice(cu[i], cu[i + 1])
        place, at = np.arange(n - t, n)[:, None], np.arange(n)
        seen = (at <= place) if causal else np.repeat(place >= 0, n, 1)
        if window:
            seen = seen & (at > place - window)
        for i2, b in hidden:
            if i2 == i:
                seen = seen & (at // w.block != b)
        for h in range(heads_q):
            K, V = r.values("k")[:, h // group], r.values("v")[:, h // group]
            x = q[rows, h].astype(np.float64)
            s = np.where(seen, scale * (x @ K.T), -np.inf)
            m = s.max(1, initial=-np.inf)
            e = np.where(seen, np.exp(s - np.where(np.isinf(m), 0.0, m)[:, None]), 0.0)
            l = e.sum(1)
            p = e / np.where(l == 0, 1.0, l)[:, None]
            S = scale * np.where(seen, np.abs(x) @ np.abs(K).T, 0.0).max(1, initial=0.0)
            top = np.abs(K).max(initial=0.0)
            rel, floor, off = kv_ref.bound(S, np.maximum(1, seen.sum(1)), w.dim,
                                           scale * np.abs(x).max(1) * np.abs(K).sum(1).max(initial=0.0),
                                           scale * np.abs(x).sum(1) * top, np.abs(V).max(initial=0.0) * 1.01)
            assert np.all(np.abs(out[rows, h] - p @ V) <= rel[:, None] * (p @ np.abs(V)) + floor[:, None]), (i, h)
            empty = l == 0
            assert np.all(np.isneginf(lse[rows, h][empty])) and not out[rows, h][empty].any()
            want = m[~empty] + np.log(l[~empty])
            assert np.all(np.abs(lse[rows, h][~empty] - want) <= off[~empty] + 2.0 ** -23 * np.abs(want)), (i, h)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_prompts(dim, block):
    """Ragged prompts and continued ones, of any length modulo the tiles, none among them."""
    heads, group = (8, 4) if dim != 96 else (5, 7)
    w = World(20, heads=heads, dim=dim, block=block, cols=-(-260 // block), seed=dim * block)
    first = [(i * 37) % 140 for i in range(20)]
    w.append(first)
    counts = [64 + (i * 29) % 50 for i in range(20)]
    counts[3] = 0
    w.append(counts)
    _check_prompts(w, counts, group)
    _check_prompts(w, counts, group, strided=True)


@pytest.mark.parametrize("window", [1, 30, 64, 100])
def test_prompts_with_windows(window):
    w = World(24, heads=8, dim=64, block=32, cols=8, seed=window)
    counts = [150 + i for i in range(24)]
    w.append(counts)
    _check_prompts(w, counts, 2, window=window)


def test_prompts_not_causal_and_beyond_their_length():
    w = World(20, heads=8, dim=64, block=16, cols=14)
    w.append([(i * 23) % 200 for i in range(20)])
    counts = [150] * 20    # longer than some of the sequences: those rows see nothing
    _check_prompts(w, counts, 4, causal=False)
    _check_prompts(w, counts, 4)


def test_prompts_with_pages_that_are_not_there():
    w = World(16, heads=8, dim=128, block=32, cols=8)
    counts = [130 + 5 * i for i in range(16)]
    w.append(counts)
    hidden = [(0, 0), (1, 1), (1, 2), (2, 4), (3, 3)]
    for i, b in hidden:
        w.table[i, b] = -1 if b % 2 else w.cache.blocks + 7
    hidden.append((5, len(w.ref[5].k) // 32))
    w.slots[5] = -3        # its incomplete block
    w.cache.k_codes[[p for p in range(w.cache.blocks) if p not in set(w.table.ravel().tolist())]] = -128
    _check_prompts(w, counts, 4, hidden=hidden)


def test_a_chunk_of_a_long_prompt():
    """Few row tiles, so that each is cut into parts."""
    w = World(1, heads=4, dim=128, block=64, cols=100, places=7000)
    w.append([6123])
    _check_prompts(w, [300], 4, tile=16)
    w = World(1, heads=8, dim=128, block=64, cols=100, places=7000)
    w.append([6123])
    _check_prompts(w, [500], 4)
    _check_prompts(w, [497], 4, strided=True)


@pytest.mark.parametrize("seqs", [256, 257, 700])
def test_many_sequences(seqs):
    """Row tiles found by counting, and (past 256 sequences) from bounds."""
    w = World(seqs, heads=1, dim=64, block=16, cols=9, seed=seqs)
    w.append([1 + (i * 13) % 140 for i in range(seqs)])
    counts = [(i * 7) % 6 for i in range(seqs)]
    counts = [min(c, len(r.k)) for c, r in zip(counts, w.ref)]
    _check_prompts(w, counts, 3, tile=16)
    _check_prompts(w, [min(140, len(r.k)) for r in w.ref], 16, tile=128)


def test_anything_behind_a_prompt():
    """NaN and infinities in the ring behind the last row of a prompt."""
    w = World(16, heads=8, dim=64, block=64, cols=3)
    counts = [100 + i for i in range(16)]
    w.append(counts)
    for i, n in enumerate(counts):
        w.cache.k_recent[int(w.slots[i]), :, n:] = NAN
        w.cache.v_recent[int(w.slots[i]), :, :, n:] = float("inf")
        w.table[i, 2] = -1
    _check_prompts(w, counts, 4)


def test_select_of_more_blocks_than_four_tokens_fit():
    """Past 4096 columns each token is a workgroup's alone, in ragged calls too."""
    w = World(2, heads=1, dim=64, block=16, cols=4100, places=1)
    mean = torch.randn(w.cache.k_mean.shape, device="cuda")
    w.cache.k_mean.copy_(mean)
    lens, cu = [16 * 4099 + 3, 500], [0, 3, 5]
    q = w.rows(5, 2)
    announce("select of 4100 columns")
    got = heal.heal_kv_select(w.cache, dev(q), 9, cu=ints(cu), **w.kw(lens)).cpu().numpy()
    mean = mean.cpu().numpy().astype(np.float64)
    for t, (i, j, n) in enumerate([(0, 0, 3), (0, 1, 3), (0, 2, 3), (1, 0, 2), (1, 1, 2)]):
        want = kv_ref.select(q[t], mean[w.table[i], 0], lens[i] - n + j, 16, 9, 1, 1)
        assert got[t, 0].tolist() == want, t


# ---- which blocks -----------------------------------------------------------------


def _check_select(w, counts, q, n_sel, keep_first=1, keep_last=1):
    T, G = q.shape[0], q.shape[1] // w.heads
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    announce("select %s of %s, %d" % (counts, w.lens(), n_sel))
    got = heal.heal_kv_select(w.cache, dev(q), n_sel, **w.kw(), cu=dev(cu), keep_first=keep_first,
                              keep_last=keep_last).cpu().numpy()
    mean = w.cache.k_mean.cpu().numpy().astype(np.float64)
    for i, r in enumerate(w.ref):
        for j in range(counts[i]):
            for h in range(w.heads):
                t, place = cu[i] + j, len(r.k) - counts[i] + j
                want = kv_ref.select(q[t, h * G:(h + 1) * G], mean[w.table[i], h], place, w.block, n_sel,
                                     keep_first, keep_last)
                assert got[t, h].tolist() == want, (i, j, h)


@pytest.mark.parametrize("dim,block,group", [(64, 16, 1), (96, 16, 4), (128, 32, 8), (64, 32, 9), (128, 16, 20)])
def test_select(dim, block, group):
    w = World(4, heads=2, dim=dim, block=block, cols=70, seed=dim + group)
    w.append([block * 70, 1, block * 33 + 1, block * 9])
    for n_sel, first, last in ((1, 0, 1), (2, 1, 1), (7, 1, 1), (16, 3, 5), (8, 4, 4), (69, 0, 1), (200, 1, 1)):
        _check_select(w, [1, 1, 1, 1], w.rows(4, 2 * group), n_sel, first, last)
    _check_select(w, [40, 1, 5, 9], w.rows(55, 2 * group), 6)
    _check_select(w, [3, 4, 0, 2], w.rows(9, 2 * group), 6)   # more tokens than the length: places below 0


@pytest.mark.parametrize("seqs,cols", [(3, 20), (3, 32), (3, 33), (3, 127), (3, 128), (2, 700), (140, 130)])
@pytest.mark.parametrize("dim,group", [(64, 1), (96, 5), (128, 16), (128, 17)])
def test_select_for_single_tokens(dim, group, seqs, cols):
    """One token of each sequence, without cu: from no block to as many as the table has."""
    rng = np.random.default_rng(dim + group + cols)
    c = heal.KVCache.empty(seqs * cols, seqs, 2, dim, 16)
    mean = rng.standard_normal((seqs * cols, 2, dim)).astype(np.float32)
    c.k_mean.copy_(dev(mean))
    table = rng.permutation(seqs * cols).reshape(seqs, cols).astype(np.int32)
    lens = rng.integers(0, cols * 16 + 1, seqs)
    lens[0], lens[-1] = cols * 16, cols * 8 + 1
    q = rng.standard_normal((seqs, 2 * group, dim)).astype(np.float32)
    for n_sel, first, last in ((2, 1, 1), (17, 2, 3)):
        announce("select %s of %s" % (n_sel, lens[:3]))
        got = heal.heal_kv_select(c, dev(q), n_sel, dev(table), ints(lens.tolist()), keep_first=first,
                                  keep_last=last).cpu().numpy()
        for i in range(seqs):
            for h in range(2):
                want = kv_ref.select(q[i, h * group:(h + 1) * group], mean[table[i], h].astype(np.float64),
                                     int(lens[i]) - 1, 16, n_sel, first, last)
                assert got[i, h].tolist() == want, (i, h)


def test_select_equal_scores_and_no_numbers():
    w = World(1, heads=2, dim=64, block=16, cols=200)
    w.append([16 * 200])
    mean = w.cache.k_mean
    pages = torch.from_numpy(w.table[0].astype(np.int64)).cuda()
    mean[pages[20:120]] = mean[pages[20]].clone()      # a hundred equal blocks
    mean[pages[130:140], 0] = NAN
    mean[pages[140:150], :, 0] = float("inf")
    mean[pages[150:160], :, 0] = -float("inf")
    mean[pages[160:170]] = 0.0
    mean[pages[170:180]] = -0.0
    for sign in (1.0, -1.0):
        q = w.rows(1, 4) * np.float32(0.1) + (sign * mean[pages[20], 0]).cpu().numpy()
        for n_sel in (2, 3, 15, 50, 101, 130, 195, 199):
            _check_select(w, [1], q.astype(np.float32), n_sel)
    w.table[0, 30:60] = -1     # blocks that the cache does not hold come last
    got = heal.heal_kv_select(w.cache, dev(w.rows(1, 4)), 171, **w.kw())[0, 1].cpu().numpy()
    assert not np.isin(np.arange(30, 59), got).all() and np.isin(np.r_[0:30, 60:200], got).sum() >= 140


def test_select_the_longest_table():
    w = World(1, heads=1, dim=64, block=16, cols=1)
    cols = 16384
    c = heal.KVCache.empty(cols, 1, 1, 64, 16)
    c.k_mean.copy_(dev(w.rng.standard_normal((cols, 1, 64)).astype(np.float32)))
    q = w.rng.standard_normal((1, 2, 64)).astype(np.float32)
    table = w.rng.permutation(cols).astype(np.int32)[None]
    announce("select of 16384 blocks")
    got = heal.heal_kv_select(c, dev(q), 1000, dev(table), ints([cols * 16])).cpu().numpy()[0, 0]
    mean = c.k_mean.cpu().numpy().astype(np.float64)[table[0], 0]
    assert got.tolist() == kv_ref.select(q[0], mean, cols * 16 - 1, 16, 1000, 1, 1)


# ---- together, on streams and in graphs ---------------------------------------------


def test_a_sequence_from_prompt_to_selected_decode():
    """As a server uses them: prompts, decode steps with all blocks, then with selected ones."""
    w = World(3, heads=2, dim=64, block=16, cols=24, seed=9)
    counts = [200, 33, 121]
    for step in range(20):
        q = w.append(counts, q=w.rows(sum(counts), 8))
        T = sum(counts)
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        sel = None
        if step > 10:
            sel = heal.heal_kv_select(w.cache, q, 4, **w.kw(), cu=dev(cu), keep_first=1, keep_last=2).cpu().numpy()
            _check_select(w, counts, q.cpu().numpy(), 4, 1, 2)
        _check_attention(w, counts, q.cpu().numpy(), sel=sel)
        counts = [1, 1, 1] if step % 3 else [1, 4, 2]
    w.check()


def _decode_state(seed):
    w = World(3, heads=2, dim=128, block=16, cols=30, seed=seed)
    w.append([300, 15, 100])
    n = 3
    s = {"w": w, "kw": w.kw(), "k": dev(w.rows(n)), "v": dev(w.rows(n)), "q": dev(w.rows(n, 8)), "cos": dev(w.cos),
         "sin": dev(w.sin), "q_out": torch.empty(n, 8, 128, device="cuda"),
         "sel": torch.empty(n, 2, 6, dtype=torch.int32, device="cuda"),
         "out": torch.empty(n, 8, 128, device="cuda"), "out2": torch.empty(n, 8, 128, device="cuda")}
    return s


def _decode_step(s):
    """The next token of every sequence: lens goes up on the device."""
    s["kw"]["lens"] += 1
    c = s["w"].cache
    heal.heal_kv_append(c, s["k"], s["v"], **s["kw"], cos=s["cos"], sin=s["sin"], q=s["q"], q_out=s["q_out"])
    heal.heal_kv_select(c, s["q_out"], 6, **s["kw"], out=s["sel"])
    heal.heal_kv_attention(c, s["q_out"], **s["kw"], out=s["out"], chunk=64)
    heal.heal_kv_attention(c, s["q_out"], **s["kw"], sel=s["sel"], out=s["out2"])


def test_a_decode_step_captured_and_replayed():
    a, b = _decode_state(4), _decode_state(4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _decode_step(a)
        _decode_step(b)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    announce("capture of a decode step")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _decode_step(a)
    torch.cuda.synchronize()
    for r in range(6):
        x = torch.randn(512, 512, device="cuda")
        heal.heal_gemm_f32(x, x)
        _decode_step(b)
        for t in (a["out"], a["out2"], a["q_out"]):
            t.zero_()
        torch.cuda.synchronize()
        announce("replay %d" % r)
        g.replay()
        torch.cuda.synchronize()
        for name in ("out", "out2", "q_out", "sel"):
            assert torch.equal(a[name], b[name]), (r, name)
        assert torch.equal(a["kw"]["lens"], b["kw"]["lens"])


def test_a_prompt_captured_and_replayed():
    """A ragged call of the prompts' kernel in parts, with other lengths at each replay.
    (Its tokens begin at a block's first, so that doing it again changes nothing.)"""
    w = World(3, heads=2, dim=128, block=64, cols=40, seed=12)
    w.append([2500, 900, 2500])
    T, kw = 700, w.kw()
    k, v, q = dev(w.rows(T)), dev(w.rows(T)), dev(w.rows(T, 8))
    cu, cos, sin = ints([0, 640, 640, 690]), dev(w.cos), dev(w.sin)   # (ten tokens are nobody's)
    out, lse, q_out = torch.empty_like(q), torch.empty(T, 8, device="cuda"), torch.empty_like(q)

    def step():
        heal.heal_kv_append(w.cache, k, v, cos=cos, sin=sin, q=q, q_out=q_out, cu=cu, **kw)
        heal.heal_kv_attention(w.cache, q_out, cu=cu, out=out, lse=lse, **kw)

    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    announce("capture of a prompt")
    with torch.cuda.graph(g):
        step()
    for lens in ([2560, 900, 114], [640, 0, 50], [1280, 900, 1970], [2240, 5, 2098]):
        kw["lens"].copy_(ints(lens))
        got = []
        for run in (step, g.replay, g.replay):
            for t in (out, lse, q_out):
                t.fill_(9.0)
            announce("lengths %s %s" % (lens, run.__name__))
            run()
            torch.cuda.synchronize()
            got.append([t.clone() for t in (out, lse, q_out)])
            assert (out[690:] == 9.0).all() and (lse[690:] == 9.0).all() and (q_out[690:] == 9.0).all()
        for x in got[1:]:
            assert all(torch.equal(a, b) for a, b in zip(x, got[0])), lens


def test_a_long_selection_captured():
    """More blocks than a kernel's LDS holds by default, in a graph."""
    c = heal.KVCache.empty(9000, 1, 1, 64, 16)
    c.k_mean.normal_()
    table, lens = torch.arange(9000, dtype=torch.int32, device="cuda")[None], ints([9000 * 16])
    q, out = torch.randn(1, 4, 64, device="cuda"), torch.empty(1, 1, 50, dtype=torch.int32, device="cuda")
    announce("a long selection")
    want = heal.heal_kv_select(c, q, 50, table, lens)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        heal.heal_kv_select(c, q, 50, table, lens, out=out)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_two_streams_at_once():
    """Two batches on two streams, each with its own cache, as each alone."""
    alone = []
    for seed in (1, 2):
        s = _decode_state(seed)
        for _ in range(4):
            _decode_step(s)
        torch.cuda.synchronize()
        alone.append((s["out"].clone(), s["out2"].clone()))
    states = [_decode_state(seed) for seed in (1, 2)]
    streams = [torch.cuda.Stream() for _ in states]
    torch.cuda.synchronize()
    announce("two streams")
    for _ in range(4):
        for s, st in zip(states, streams):
            with torch.cuda.stream(st):
                _decode_step(s)
    torch.cuda.synchronize()
    for s, (o, o2) in zip(states, alone):
        assert torch.equal(s["out"], o) and torch.equal(s["out2"], o2)


def test_binding_refuses_on_the_gpu():
    w = World(2, dim=64, block=16, cols=3)
    w.append([5, 6])
    q, kw, c = dev(w.rows(2, 4)), w.kw(), w.cache
    bad = [
        lambda: heal.heal_kv_attention(c, q, **{**kw, "lens": kw["lens"].long()}),
        lambda: heal.heal_kv_attention(c, q, **{**kw, "lens": kw["lens"][:1]}),
        lambda: heal.heal_kv_attention(c, q, **{**kw, "lens": kw["lens"].cpu()}),
        lambda: heal.heal_kv_attention(c, q, **{**kw, "table": kw["table"].t()}),
        lambda: heal.heal_kv_attention(c, q, **{**kw, "slots": kw["slots"][:1]}),
        lambda: heal.heal_kv_attention(c, q, **kw, cu=ints([0, 2])),
        lambda: heal.heal_kv_attention(c, q.transpose(1, 2), **kw),
        lambda: heal.heal_kv_attention(c, q, **kw, out=q[:, :2]),
        lambda: heal.heal_kv_attention(c, q, **kw, lse=torch.empty(4, 2, device="cuda").t()),
        lambda: heal.heal_kv_attention(c, q, **kw, sel=torch.zeros(2, 2, 0, dtype=torch.int32, device="cuda")),
        lambda: heal.heal_kv_attention(c, q, **kw, sel=torch.zeros(2, 4, 3, dtype=torch.int32, device="cuda")),
        lambda: heal.heal_kv_attention(c, q, **kw, chunk=65),
        lambda: heal.heal_kv_attention(c, q, **kw, window=-1),
        lambda: heal.heal_kv_attention(c, q, **kw, scale=float("nan")),
        lambda: heal.heal_kv_attention(c, dev(w.rows(3, 4)), **kw),
        lambda: heal.heal_kv_select(c, q, 1, **kw),
        lambda: heal.heal_kv_select(c, q, 0, **kw),
        lambda: heal.heal_kv_select(c, q, 4, **kw, keep_last=0),
        lambda: heal.heal_kv_select(c, q, 4, **kw, out=torch.empty(2, 2, 5, dtype=torch.int32, device="cuda")),
        lambda: heal.heal_kv_append(c, q[:, :2], q[:, :2], **kw, cos=dev(w.cos)),
        lambda: heal.heal_kv_append(c, q[:, :2], q[:, :2], **kw, cos=dev(w.cos), sin=dev(w.sin[:5])),
        lambda: heal.heal_kv_append(c, q[:, :2], q[:, :2], **kw, cos=dev(np.ones((9, 33), np.float32)),
                                    sin=dev(np.ones((9, 33), np.float32))),
        lambda: heal.heal_kv_append(c, q[:, :2], q[:, :2], **kw, q_out=q),
        lambda: heal.heal_kv_append(c, q, q, **kw),
        lambda: heal.heal_kv_read(c, 3, **kw),
        lambda: heal.heal_kv_read(heal.KVCache.empty(4, 1, 2, 64, 16), 2, kw["table"], kw["lens"]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(heal.HealError):
            call()
            pytest.fail("call %d was taken" % i)
