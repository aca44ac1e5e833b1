"""Residual norms and adapters where no GPU is needed: refusals and empty calls."""
import ctypes

import pytest
import torch

import paper_2606_21023_amd as heal

MIB = 1 << 20
H, X, G, HO, OUT, W, W2 = (MIB * i for i in range(1, 8))   # never dereferenced
OK, INVALID = 0, 1
NAN, INF = float("nan"), float("inf")


def _spec(**kw):
    a = dict(weight=W, bias=None, eps=1e-6, centred=0)
    a.update(kw)
    return heal._CNorm(*a.values())


def _name(kw):
    return ",".join("%s=%s" % (k, [getattr(v, f) for f, _ in v._fields_] if isinstance(v, heal._CNorm) else v)
                    for k, v in kw.items())


def _norm(post=_spec(weight=W2), pre=_spec(), **kw):
    a = dict(rows=10, heads=1, dim=100, h=H, h_row=100, h_head=0, x=X, x_row=100, x_head=0, post=post, gate=G, gate_row=100,
             gate_head=0, gate_col=1, scale=0.5, pre=pre, h_out=HO, ho_row=100, ho_head=0, out=OUT, out_row=100, out_head=0)
    a.update(kw)
    for n in ("post", "pre"):
        a[n] = ctypes.byref(a[n]) if a[n] is not None else None
    return heal.lib().heal_block_norm(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(heads=-1), dict(dim=0), dict(dim=(1 << 24) + 1), dict(rows=1 << 20, heads=1 << 11), dict(h=None),
    dict(h=H + 2), dict(x=X + 1), dict(gate=G + 2), dict(h_out=HO + 1), dict(out=OUT + 2), dict(h_row=-1), dict(x_row=-4),
    dict(gate_row=-1), dict(gate_col=2), dict(scale=NAN), dict(scale=INF), dict(ho_row=99), dict(out_row=50),
    dict(h_row=(1 << 40) + 1),
    # what needs x, or pre, or an output
    dict(x=None), dict(x=None, post=None), dict(x=None, post=None, gate=None), dict(pre=None), dict(out=None),
    dict(pre=None, out=None, h_out=None),
    dict(pre=_spec(weight=None)), dict(post=_spec(weight=W + 2)), dict(pre=_spec(bias=W + 1)), dict(pre=_spec(eps=-1.0)),
    dict(post=_spec(eps=NAN)), dict(pre=_spec(eps=INF)), dict(pre=_spec(centred=2)),
    # outputs that overlap something
    dict(h_out=OUT), dict(h_out=H + 4), dict(h_out=H, ho_row=104), dict(out=X + 400), dict(out=G), dict(out=W - 400),
    dict(h_out=W2 + 396), dict(out=HO + 3996), dict(h_out=H, out=H), dict(heads=4, ho_head=100, ho_row=100, out_head=100,
                                                                        out_row=400),
], ids=_name)
def test_bad_norms_are_refused(kw):
    assert _norm(**kw) == INVALID


def test_norms_without_rows_do_nothing():
    assert _norm(rows=0, h=None) == OK and _norm(heads=0) == OK


def _lora(bank=None, **kw):
    b = dict(adapters=4, rank=8, K=100, N=60, type=0, a=W, b=W2, ranks=None, scales=None)
    b.update(bank or {})
    a = dict(tokens=5, seqs=3, cu=MIB * 10, ids=MIB * 11, x=X, ldx=100, y=HO, ldy=60, out=OUT, ldo=60, workspace=MIB * 20,
             size=1 << 40)
    a.update(kw)
    return heal.lib().heal_lora_add(ctypes.byref(heal._CBank(*b.values())), *a.values(), None)


@pytest.mark.parametrize("kw", [dict(bank=b) for b in (
    dict(adapters=0), dict(adapters=1 << 31), dict(rank=0), dict(rank=513), dict(K=0), dict(N=0), dict(K=(1 << 24) + 1),
    dict(N=(1 << 24) + 1), dict(type=3), dict(type=-1), dict(a=None), dict(b=None), dict(a=W + 4), dict(b=W2 + 8),
    dict(ranks=MIB * 12 + 2), dict(scales=MIB * 12 + 1))] + [
    dict(tokens=-1), dict(tokens=(1 << 24) + 1), dict(seqs=-1), dict(seqs=(1 << 24) + 1), dict(cu=None), dict(cu=MIB + 2),
    dict(ids=None), dict(ids=MIB + 2), dict(x=None), dict(y=None), dict(out=None), dict(x=X + 2), dict(out=OUT + 1),
    dict(ldx=99), dict(ldy=59), dict(ldo=59), dict(ldx=(1 << 40) + 1), dict(workspace=None), dict(workspace=MIB + 8), dict(size=0),
    dict(out=HO, ldo=61), dict(out=HO + 4), dict(out=X), dict(out=X + 1996), dict(out=W + 16), dict(out=W2 - 64)], ids=str)
def test_bad_adapters_are_refused(kw):
    assert _lora(**kw) == INVALID


def test_calls_without_tokens_do_nothing():
    assert _lora(tokens=0, seqs=0, cu=None, ids=None, x=None, y=None, out=None, workspace=None) == OK
    assert _lora(tokens=0, x=None) == OK and _lora(seqs=0, ids=None) == OK


def test_lora_workspace():
    f = heal.lib().heal_lora_workspace
    bank = lambda **kw: ctypes.byref(heal._CBank(*{**dict(adapters=4, rank=8, K=100, N=60, type=0, a=None, b=None,  # noqa: E731
                                                         ranks=None, scales=None), **kw}.values()))
    assert f(bank(), 5) >= 5 * 8 * 4 and f(bank(), 0) >= 0
    assert f(bank(rank=0), 5) == -1 and f(bank(), -1) == -1 and f(bank(type=9), 5) == -1
    # it grows with the tokens and the rank, in proportion
    assert f(bank(), 2000) * 2 >= f(bank(), 4000) and f(bank(K=1 << 24, rank=512, N=1), 1 << 24) > 0


def test_the_binding_refuses_what_is_no_cuda_tensor():
    x = torch.zeros(2, 8)
    for f in (lambda: heal.heal_block_norm(x, pre=torch.ones(8)), lambda: heal.LoraBank(torch.zeros(1, 2, 8), torch.zeros(1, 4, 2)),
              lambda: heal.LoraBank(None, None), lambda: heal.heal_lora_add(x, x, None, [0, 0])):
        with pytest.raises(heal.HealError):
            f()
