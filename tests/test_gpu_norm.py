"""heal_block_norm against its formula in 64 bits.

h' is rounded once from FP64, so it is off by half an FP32 step of itself (2^-24, and 2^-150
below 2^-126) and by what its FP64 terms lose (less than 8 roundings of 2^-53 each, and those
of the first norm).  out is the norm of h' as it was written: the reference takes the
kernel's own h', and the bound is half a step again.  The FP64 sums of a row of n elements are off
by n 2^-53 at most, and about the mean the square of the pivot's distance costs up to n more:
n^2 2^-53 in all, below 2^-25 of 1 for every row here (n <= 2^14) and 2^-21 for the longest; the
terms below take 2^-30 (rows up to 2^11), or n^2 2^-53."""
import numpy as np
import pytest
import torch

import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]


def normed(y, weight, bias, eps, centred):
    """(value, sum of the magnitudes that make it up) in 64 bits.  Where y is near the mean those are not
    the value's: the mean is a sum about the row's first element, rounded in relation to that."""
    y = y.astype(np.float64)
    d = y - y.mean(-1, keepdims=True) if centred else y
    with np.errstate(all="ignore"):
        f = weight.astype(np.float64) / np.sqrt((d * d).mean(-1, keepdims=True) + np.float64(np.float32(eps)))
        terms = (np.abs(y) + np.abs(y[..., :1]) if centred else np.abs(y)) * np.abs(f)
    b = 0.0 if bias is None else bias.astype(np.float64)
    return d * f + b, terms + np.abs(b)


def close(got, want, terms, n, what):
    fp64 = max(2.0 ** -30, n * n * 2.0 ** -53) * 2.0 ** -3
    limit = 2.0 ** -24 * np.abs(want) + fp64 * terms + 2.0 ** -149
    bad = ~(np.abs(got - want) <= limit) & ~(np.isnan(got) & np.isnan(want)) & ~(got == want.astype(np.float32))
    assert not bad.any(), (what, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


def run(h, x=None, post=None, gate=None, scale=1.0, pre=None, eps=1e-6, centred=False, post_bias=None, pre_bias=None, **kw):
    """Runs numpy arrays through the kernel and holds it to the formula; returns (h', out)."""
    dev = lambda a: a if a is None or isinstance(a, torch.Tensor) else torch.from_numpy(np.array(a)).cuda()  # noqa: E731
    host = lambda a: a if a is None or isinstance(a, np.ndarray) else a.cpu().numpy()  # noqa: E731
    h0, x0, g0 = host(h).copy(), None if x is None else host(x).copy(), host(gate)
    ho, out = heal.heal_block_norm(dev(h), dev(x), post=dev(post), gate=dev(gate), scale=scale, pre=dev(pre), eps=eps,
                                   centred=centred, post_bias=dev(post_bias), pre_bias=dev(pre_bias), **kw)
    torch.cuda.synchronize()
    n, after = h0.shape[-1], h0
    if x is not None:
        u, terms = x0.astype(np.float64), np.abs(x0.astype(np.float64))
        if post is not None:
            u, terms = normed(x0, host(post), host(post_bias), eps, centred)
        f = np.float64(np.float32(scale)) * (1.0 if gate is None else g0.astype(np.float64))
        after = ho.cpu().numpy()
        with np.errstate(all="ignore"):
            close(after, h0 + f * u, np.abs(h0.astype(np.float64)) * 2.0 ** -17 + np.abs(f) * terms, n, "h'")
    if pre is not None:
        want, terms = normed(after, host(pre), host(pre_bias), eps, centred)
        close(out.cpu().numpy(), want, terms, n, "out")
    return ho, out


def rows(rng, *shape, sigma=1.0):
    x = (sigma * rng.standard_normal(shape)).astype(np.float32)
    x[..., 0] *= 50.0   # a wide channel
    return x


DIMS = [1, 2, 3, 5, 31, 64, 65, 96, 100, 128, 132, 255, 256, 260, 511, 512, 516, 1000, 1023, 1024, 1028, 2048, 2052, 4095, 4096,
        4100, 8192, 8196, 14336, 16384, 16388, 16385, 40000]


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("n", [1, 3, 70])
def test_rows_of_every_length(dim, n):
    rng = np.random.default_rng(dim + n)
    announce("norm %d x %d" % (n, dim))
    w = lambda: 1.0 + 0.1 * rows(rng, dim)  # noqa: E731
    h, x = rows(rng, n, dim), rows(rng, n, dim)
    run(h, pre=w())
    run(h, x, pre=w())
    run(h, x, post=w(), gate=rows(rng, 1, dim), scale=0.3, pre=w(), pre_bias=w(), post_bias=w(), centred=True)
    run(h, x, post=w(), gate=rows(rng, n, dim), scale=-2.0)


@pytest.mark.parametrize("gate", [None, (1, 1), (1, 300), (9, 1), (9, 300)])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("centred", [False, True])
def test_every_form(gate, post, pre, centred):
    rng = np.random.default_rng(1)
    w = lambda on: 1.0 + 0.1 * rows(rng, 300) if on else None  # noqa: E731
    h, x = rows(rng, 9, 300), rows(rng, 9, 300)
    announce("norm gate %s post %s pre %s centred %s" % (gate, post, pre, centred))
    run(h, x, post=w(post), pre=w(pre), gate=None if gate is None else rng.standard_normal(gate).astype(np.float32), scale=0.7,
        centred=centred, post_bias=w(post and centred), pre_bias=w(pre and not centred), eps=1e-5)


@pytest.mark.parametrize("dim", [64, 96, 128, 100, 256, 257])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (1, 5), (7, 3), (300, 32)])
def test_heads_between_others(tokens, heads, dim):
    """Heads out of a joint projection's rows, written to rows of their own or in place."""
    rng = np.random.default_rng(dim)
    wide = torch.from_numpy(rows(rng, tokens, heads + 3, dim)).cuda()
    before, w = wide.clone(), 1.0 + 0.1 * rows(rng, dim)
    announce("heads %s" % ((tokens, heads, dim),))
    _, out = run(wide[:, 1:heads + 1], pre=w)
    assert torch.equal(wide, before)
    part = wide[:, 1:heads + 1]
    # (in place: the check above has read h before the call)
    _, same = run(part, pre=w, out=part)
    assert same is part and torch.equal(out, part)
    assert torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[:, heads + 1:], before[:, heads + 1:])
    # queries beside keys of the same rows: side by side is not overlapping
    heal.heal_block_norm(wide[:, :1], pre=torch.from_numpy(w).cuda(), out=wide[:, 2:3])
    gate = torch.from_numpy(rng.standard_normal((tokens, 1, dim)).astype(np.float32)).cuda()
    run(wide[:, :heads], wide[:, 3:], gate=gate, pre=w)


@pytest.mark.parametrize("dim", [96, 128, 1000, 4096, 16384, 20000])
def test_strides_alignment_and_places(dim):
    rng = np.random.default_rng(dim)
    base = torch.from_numpy(rows(rng, 6, dim + 9)).cuda()
    other = torch.from_numpy(rows(rng, 12, dim + 9)).cuda()
    w = 1.0 + 0.1 * rows(rng, dim)
    kw = dict(post=w, pre=w, scale=0.5)
    want = run(base[:, :dim].contiguous(), other[:6, :dim].contiguous(), **kw)
    for a, b in ((base[:, :dim], other[:6, :dim]), (base[:, :dim], other[::2, 4:dim + 4])):
        run(a, b, **kw)
    run(base[:, 1:dim + 1], other[:6, 3:dim + 3], **kw)
    # the same rows at other alignments: the same bits
    for off in (1, 2, 3):
        moved = [torch.empty(6, dim + 9, device="cuda")[:, off:off + dim] for _ in range(2)]
        moved[0].copy_(base[:, :dim]), moved[1].copy_(other[:6, :dim])
        got = run(*moved, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # in place, with and without a place for h'
    h, x = base[:, :dim].contiguous(), other[:6, :dim].contiguous()
    got = run(h, x, h_out=h, out=x, **kw)
    assert got[0] is h and got[1] is x and torch.equal(h, want[0]) and torch.equal(x, want[1])
    h, x = base[:, :dim].contiguous(), other[:6, :dim].contiguous()
    got = run(h, x, h_out=x, out=h, **kw)
    assert torch.equal(x, want[0]) and torch.equal(h, want[1])
    # one row of h for all, and outputs among rows that stay
    one = base[:1, :dim].expand(6, dim)
    rest = torch.full((6, 2 * dim + 8), 5.0, device="cuda")
    run(one, x, h_out=rest[:, :dim], out=rest[:, dim:2 * dim], **kw)
    assert (rest[:, 2 * dim:] == 5.0).all()


def test_without_h_out():
    """The last norm of a model needs the sum's norm only (the C entry takes no h')."""
    import ctypes
    torch.manual_seed(0)
    h, x, w = torch.randn(5, 200, device="cuda"), torch.randn(5, 200, device="cuda"), torch.rand(200, device="cuda")
    out = torch.empty_like(h)
    spec = heal._CNorm(w.data_ptr(), None, 1e-6, 0)
    st = heal.lib().heal_block_norm(5, 1, 200, h.data_ptr(), 200, 0, x.data_ptr(), 200, 0, None, None, 0, 0, 0, 1.0,
                                    ctypes.byref(spec), None, 0, 0, out.data_ptr(), 200, 0, heal._stream())
    assert st == 0 and torch.equal(out, heal.heal_block_norm(h, x, pre=w)[1])


@pytest.mark.parametrize("dim", [7, 128, 1000, 4096, 16384, 17000])
def test_magnitudes(dim):
    rng = np.random.default_rng(dim)
    w = 1.0 + 0.1 * rows(rng, dim)
    x = rows(rng, 8, dim)
    scale = np.array([1e-38, 1e-30, 1e-20, 1e-3, 1.0, 1e18, 1e30, 1e36], np.float32)[:, None]
    run(x * scale, pre=w, eps=0.0)
    run(x * scale, pre=w, eps=0.0, centred=True)
    run(x * scale, (x * scale)[::-1].copy(), post=w, pre=w, eps=1e-12, scale=0.1)
    # rows that differ from one number in their last places only
    near = (np.float32(3.0) + np.arange(dim, dtype=np.float32)[None] % 5 * np.float32(2.0 ** -21)) * scale[2:7]
    near = near.astype(np.float32)
    run(near, pre=w, eps=0.0, centred=True)
    near[:, 0] *= 1000.0   # the first one far off
    run(near, pre=w, eps=0.0, centred=True)


@pytest.mark.parametrize("dim", [100, 128, 4096, 20000])
def test_what_is_not_finite_stays_in_its_row(dim):
    rng = np.random.default_rng(dim)
    w = 1.0 + 0.1 * rows(rng, dim)
    h, x = rows(rng, 70, dim), rows(rng, 70, dim)
    clean = heal.heal_block_norm(*(torch.from_numpy(t).cuda() for t in (h, x)), pre=torch.from_numpy(w).cuda())
    bad = {2: np.inf, 5: -np.inf, 9: np.nan, 33: np.inf}
    for r, v in bad.items():
        (h if r % 2 else x)[r, r] = v
    x[33, 7] = np.nan
    ho, out = heal.heal_block_norm(*(torch.from_numpy(t).cuda() for t in (h, x)), pre=torch.from_numpy(w).cuda())
    fine = [i for i in range(70) if i not in bad]
    for got, want in ((ho, clean[0]), (out, clean[1])):
        assert torch.equal(got[fine], want[fine])
    o = out.cpu().numpy()
    # an infinity: no number where it is, zeros elsewhere; a NaN: all of the row
    for r in (2, 5):
        assert np.isnan(o[r, r]) and np.all(np.delete(o[r], r) == 0)
    assert np.isnan(o[9]).all() and np.isnan(o[33]).all()
    c = heal.heal_block_norm(torch.from_numpy(h).cuda(), pre=torch.from_numpy(w).cuda(), centred=True)[1].cpu().numpy()
    assert np.isnan(c[[5, 9, 33]]).all() and np.isfinite(np.delete(c, [5, 9, 33], 0)).all()
    # zeros: the formula's 0 / 0 without eps, 0 with it
    zero = torch.zeros(2, dim, device="cuda")
    assert heal.heal_block_norm(zero, pre=torch.from_numpy(w).cuda(), eps=0.0)[1].isnan().all()
    assert (heal.heal_block_norm(zero, pre=torch.from_numpy(w).cuda())[1] == 0).all()


@pytest.mark.parametrize("dim", [64, 128, 300, 4096, 20000])
def test_a_rows_bits_do_not_depend_on_the_batch(dim):
    torch.manual_seed(dim)
    h, x, w = torch.randn(513, dim, device="cuda"), torch.randn(513, dim, device="cuda"), torch.rand(dim, device="cuda")
    ho, out = heal.heal_block_norm(h, x, post=w, pre=w, centred=True)
    for rows_ in (slice(0, 1), slice(5, 8), slice(512, 513), slice(100, 165)):
        a, b = heal.heal_block_norm(h[rows_], x[rows_], post=w, pre=w, centred=True)
        assert torch.equal(a, ho[rows_]) and torch.equal(b, out[rows_])


def test_many_rows():
    """More rows than one launch takes workgroups."""
    torch.manual_seed(0)
    n = (1 << 22) + 5
    h, w = torch.randn(n, 1, 8, device="cuda").expand(n, 3, 8), torch.rand(8, device="cuda")
    out = heal.heal_block_norm(h, pre=w)[1]
    at = torch.tensor([0, 1, n // 2, n - 1], device="cuda")
    assert torch.equal(out[at], heal.heal_block_norm(h[at], pre=w)[1])
    assert torch.equal(out[:, 0], out[:, 2])


def test_rows_past_32_bits():
    base = torch.empty(3 << 30, device="cuda")   # rows 2^30 elements apart
    h = base.as_strided((3, 500), (1 << 30, 1))
    h.copy_(torch.randn(3, 500, device="cuda"))
    w = torch.rand(500, device="cuda")
    want = heal.heal_block_norm(h.contiguous(), pre=w)[1]
    out = base.as_strided((3, 500), (1 << 30, 1), 512)
    heal.heal_block_norm(h, pre=w, out=out)
    assert torch.equal(out, want)


def test_captured_and_on_another_stream():
    torch.manual_seed(1)
    h, x, w = torch.randn(33, 4096, device="cuda"), torch.randn(33, 4096, device="cuda"), torch.rand(4096, device="cuda")
    ho, out = torch.empty_like(h), torch.empty_like(h)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        heal.heal_block_norm(h, x, post=w, pre=w, h_out=ho, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        heal.heal_block_norm(h, x, post=w, pre=w, h_out=ho, out=out)
    for turn in range(3):
        h.copy_(torch.randn_like(h))
        want = heal.heal_block_norm(h, x, post=w, pre=w)
        ho.zero_(), out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(ho, want[0]) and torch.equal(out, want[1])


def test_empty_calls_and_refusals():
    h, w = torch.randn(4, 64, device="cuda"), torch.rand(64, device="cuda")
    none = h[:0]
    ho, out = heal.heal_block_norm(none, none, pre=w)
    assert ho.shape == out.shape == (0, 64)
    assert heal.heal_block_norm(h, pre=w)[0] is h and heal.heal_block_norm(h, h)[1] is None
    for f in (lambda: heal.heal_block_norm(h), lambda: heal.heal_block_norm(h, post=w, pre=w), lambda: heal.heal_block_norm(h, gate=h, pre=w),
              lambda: heal.heal_block_norm(h, h[:3], pre=w), lambda: heal.heal_block_norm(h, pre=w[:63]),
              lambda: heal.heal_block_norm(h, pre=w.double()), lambda: heal.heal_block_norm(h.half(), pre=w),
              lambda: heal.heal_block_norm(h.t(), pre=w[:4]), lambda: heal.heal_block_norm(h, pre=w, pre_bias=w[1:]),
              lambda: heal.heal_block_norm(h, h, post_bias=w), lambda: heal.heal_block_norm(h, h, gate=h[:, :2]),
              lambda: heal.heal_block_norm(h, h, gate=w), lambda: heal.heal_block_norm(h, h, out=h),
              lambda: heal.heal_block_norm(h, pre=w, h_out=h), lambda: heal.heal_block_norm(h, pre=w, out=h[:, :32]),
              lambda: heal.heal_block_norm(h[:2], h[:2], h_out=h[1:3]), lambda: heal.heal_block_norm(h[0], pre=w),
              lambda: heal.heal_block_norm(h, pre=w, out=w.expand(4, 64)), lambda: heal.heal_block_norm(h, pre=w, eps=-1.0),
              lambda: heal.heal_block_norm(h, h, scale=float("nan")), lambda: heal.heal_block_norm(h, pre=w.cpu())):
        with pytest.raises(heal.HealError):
            f()
