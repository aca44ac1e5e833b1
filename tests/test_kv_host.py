"""The key/value cache where no GPU is needed: index functions, refusals, workspace."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2606_21023_amd as heal
from paper_2606_21023_amd import build as hbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, OK, INVALID = 0x10000, 0, 1   # FAKE is never dereferenced


def test_index_functions(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "kv_index")
    subprocess.run([gxx, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-D__HIP_PLATFORM_AMD__",
                    "-I", hbuild.INCLUDE, "-I", hbuild.CSRC, "-I", "/opt/rocm/include",
                    os.path.join(ROOT, "tests", "c", "kv_index.cpp"), "-L/opt/rocm/lib", "-lamdhip64", "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.stdout.strip() == "ok", r.stdout + r.stderr


def _cache(**kw):
    a = dict(blocks=10, slots=4, heads=2, dim=128, block=64, k_codes=FAKE, v_codes=FAKE, scales=FAKE,
             k_mean=FAKE, k_recent=FAKE, v_recent=FAKE)
    a.update(kw)
    return heal._CCache(*a.values())


def _batch(**kw):
    a = dict(seqs=3, tokens=5, cu=FAKE, lens=FAKE, table=FAKE, table_ld=7, table_cols=6, slots=FAKE)
    a.update(kw)
    return heal._CBatch(*a.values())


def _append(cache=None, batch=None, **kw):
    a = dict(k=FAKE, k_token=256, k_head=128, v=FAKE, v_token=256, v_head=128, cos=FAKE, sin=FAKE, places=100,
             rot=128, interleaved=0, q=FAKE, q_token=512, q_head=128, heads_q=4, q_out=FAKE + 64, qo_token=512,
             qo_head=128)
    a.update(kw)
    return heal.lib().heal_kv_append(ctypes.byref(cache or _cache()), ctypes.byref(batch or _batch()),
                                     *a.values(), None)


def _read(cache=None, batch=None, k=FAKE, v=FAKE):
    return heal.lib().heal_kv_read(ctypes.byref(cache or _cache()), ctypes.byref(batch or _batch()), k, v, None)


def _select(cache=None, batch=None, **kw):
    a = dict(q=FAKE, q_token=512, q_head=128, heads_q=4, n_sel=4, keep_first=1, keep_last=1, sel=FAKE)
    a.update(kw)
    return heal.lib().heal_kv_select(ctypes.byref(cache or _cache()), ctypes.byref(batch or _batch()),
                                     *a.values(), None)


def _attention(cache=None, batch=None, **kw):
    a = dict(q=FAKE, q_token=512, q_head=128, heads_q=4, scale=ctypes.c_float(0.1), causal=1, window=0, sel=None,
             n_sel=0, out=FAKE, out_token=512, out_head=128, lse=None, chunk=0, workspace=FAKE, size=1 << 40)
    a.update(kw)
    return heal.lib().heal_kv_attention(ctypes.byref(cache or _cache()), ctypes.byref(batch or _batch()),
                                        *a.values(), None)


CALLS = [_append, _read, _select, _attention]

BAD_CACHE = [dict(blocks=0), dict(blocks=1 << 31), dict(slots=0), dict(heads=0), dict(heads=1025), dict(dim=80),
             dict(dim=256), dict(block=8), dict(block=48), dict(k_codes=0), dict(v_codes=FAKE + 8), dict(scales=0),
             dict(k_mean=FAKE + 4), dict(k_recent=0), dict(v_recent=0)]
BAD_BATCH = [dict(seqs=-1), dict(seqs=(1 << 24) + 1), dict(tokens=-1), dict(tokens=(1 << 30) + 1),
             dict(cu=None, tokens=4), dict(cu=FAKE + 2), dict(lens=None), dict(lens=FAKE + 1), dict(table=None),
             dict(table_ld=5), dict(table_cols=-1), dict(table_cols=1 << 25, table_ld=1 << 25), dict(slots=FAKE + 3)]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw", BAD_CACHE, ids=str)
def test_a_bad_cache_is_refused(call, kw):
    assert call(cache=_cache(**kw)) == INVALID


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw", BAD_BATCH, ids=str)
def test_a_bad_batch_is_refused(call, kw):
    assert call(batch=_batch(**kw)) == INVALID


@pytest.mark.parametrize("call,kw", [(_append, kw) for kw in (
    dict(k=0), dict(v=0), dict(k=FAKE + 2), dict(k_token=-1), dict(v_head=-4), dict(rot=130), dict(rot=7),
    dict(rot=-2), dict(interleaved=2), dict(places=-1), dict(cos=0), dict(sin=FAKE + 2), dict(q=0), dict(q_out=0),
    dict(heads_q=0), dict(qo_token=100), dict(qo_head=64), dict(qo_token=384), dict(q_out=FAKE, qo_head=129, qo_token=700),
)] + [(_select, kw) for kw in (
    dict(q=0), dict(sel=0), dict(heads_q=3), dict(heads_q=0), dict(n_sel=1), dict(n_sel=0, keep_first=0),
    dict(keep_first=-1), dict(keep_last=0), dict(keep_first=4), dict(q_token=-1), dict(sel=FAKE + 1),
    dict(batch=_batch(table_cols=16385, table_ld=16385)),
)] + [(_attention, kw) for kw in (
    dict(q=0), dict(out=0), dict(q=FAKE + 2), dict(out=FAKE + 1), dict(lse=FAKE + 2), dict(heads_q=5),
    dict(scale=ctypes.c_float(float("nan"))), dict(scale=ctypes.c_float(float("inf"))), dict(causal=2),
    dict(window=-1), dict(window=5, causal=0), dict(sel=FAKE, n_sel=0), dict(sel=None, n_sel=3), dict(sel=FAKE + 2, n_sel=3),
    dict(sel=FAKE, n_sel=-1), dict(sel=FAKE, n_sel=1 << 30), dict(chunk=-64), dict(chunk=100),
    dict(out_token=100), dict(out_head=100), dict(workspace=None, chunk=64), dict(workspace=FAKE + 8, chunk=64),
    dict(size=64, chunk=64),
)], ids=lambda x: getattr(x, "__name__", None) or ",".join(x))
def test_bad_arguments_are_refused(call, kw):
    assert call(**kw) == INVALID


@pytest.mark.parametrize("call", CALLS)
def test_calls_without_tokens_do_nothing(call):
    null = dict(k_codes=0, v_codes=0, scales=0, k_mean=0, k_recent=0, v_recent=0)
    for kw in (dict(tokens=0), dict(seqs=0), dict(seqs=0, tokens=0, cu=None, lens=None, table=None, slots=None)):
        assert call(cache=_cache(**null), batch=_batch(**kw)) == OK


def test_workspace():
    f = heal.lib().heal_kv_attention_workspace

    def size(heads_q=4, window=0, n_sel=0, chunk=0, cache=None, **kw):
        return f(ctypes.byref(cache or _cache()), ctypes.byref(_batch(**kw)), heads_q, window, n_sel, chunk)
    # chunks x rows x (dim + 2) floats
    assert size(chunk=64, table_cols=6) == 6 * 5 * 4 * 130 * 4
    assert size(chunk=128, table_cols=5) == 3 * 5 * 4 * 130 * 4
    assert size(chunk=1 << 20) == 0 and size(table_cols=1) == 0 and size(table_cols=0, table=None) == 0
    assert size(chunk=64, n_sel=3) == 3 * 5 * 4 * 130 * 4
    assert size(heads_q=3) == -1 and size(window=-1) == -1 and size(chunk=63) == -1 and size(n_sel=-2) == -1
    assert size(cache=_cache(dim=65)) == -1 and size(tokens=-1) == -1
    # pointers do not matter, and a long cache needs no more than 64 chunks of the library's choice
    assert size(lens=None) >= 0
    assert size(table_cols=1 << 24, table_ld=1 << 24) <= 64 * 5 * 4 * 130 * 4
    assert size(tokens=1 << 30, heads_q=2048, chunk=64, table_cols=1 << 24, table_ld=1 << 24) == -1


def test_which_kernel_takes_a_call():
    """16-row tiles for single tokens, drafts and short prompts; 128-row tiles for long ones,
    or many (us on one MI355X with 16-row and 128-row tiles)."""
    f = heal.lib().heal_kv_attention_tile

    def tile(seqs, tokens, length, heads=8, group=4, dim=128, block=64, chunk=0, n_sel=0, window=0, cu=FAKE):
        c = _cache(heads=heads, dim=dim, block=block)
        b = _batch(seqs=seqs, tokens=seqs * tokens, cu=cu, table_cols=-(-length // block),
                   table_ld=-(-length // block))
        return f(ctypes.byref(c), ctypes.byref(b), heads * group, window, n_sel, chunk)
    assert tile(64, 1, 8192) == 16 and tile(64, 1, 8192, cu=None) == 16
    assert tile(8, 4, 4096) == 16 and tile(8, 16, 4096) == 16              # 24, 35; 44, 49
    assert tile(8, 64, 4096) == 128 and tile(32, 512, 2048) == 128         # 117, 90; 1807, 927
    assert tile(1, 256, 256) == 16 and tile(16, 256, 256) == 128           # 14, 22; 140, 60
    assert tile(1, 512, 16001) == 128 and tile(2, 2048, 2048) == 128
    # sums that do not depend on the call's sizes, and blocks of each token's own
    assert tile(2, 2048, 2048, chunk=64) == 16 and tile(2, 2048, 2048, n_sel=4) == 16
    # a window leaves little to read
    assert tile(1, 512, 16001, window=64) == 16
    assert tile(1, 1, 64, dim=65) == 0 and tile(1, 1, 64, group=0) == 0
    assert tile(1, 1 << 30, 64, group=2) == 0


class OnDevice(torch.Tensor):
    """A CPU tensor that the checks take for one on the device."""
    is_cuda = True


def _arrays(blocks=3, slots=2, heads=2, dim=64, block=16):
    shapes = [(blocks, heads, block, dim), (blocks, heads, dim, block), (blocks, heads, 2), (blocks, heads, dim),
              (slots, heads, 2 * block, dim), (slots, heads, dim, 2 * block)]
    return [torch.zeros(s, dtype=torch.int8 if i < 2 else torch.float32).as_subclass(OnDevice)
            for i, s in enumerate(shapes)]


def test_kvcache_checks_its_arrays():
    c = heal.KVCache(*_arrays())
    assert (c.blocks, c.slots, c.heads, c.dim, c.block) == (3, 2, 2, 64, 16)
    for i in range(6):
        a = _arrays()
        a[i] = a[i].to(torch.float16).as_subclass(OnDevice)
        with pytest.raises(heal.HealError):
            heal.KVCache(*a)
        a = _arrays()
        a[i] = torch.zeros([x + 1 for x in a[i].shape], dtype=a[i].dtype).as_subclass(OnDevice)
        with pytest.raises(heal.HealError):
            heal.KVCache(*a)
        a = _arrays()
        a[i] = a[i].as_subclass(torch.Tensor)
        with pytest.raises(heal.HealError):
            heal.KVCache(*a)
    for kw in (dict(dim=80), dict(block=24), dict(blocks=0), dict(slots=0), dict(heads=0)):
        with pytest.raises(heal.HealError):
            heal.KVCache(*_arrays(**kw))


def test_binding_refuses():
    c = heal.KVCache(*_arrays())
    q = torch.zeros((2, 4, 64)).as_subclass(OnDevice)
    for call in (lambda: heal.heal_kv_attention(None, q, None, None),
                 lambda: heal.heal_kv_attention(c, q[..., :32], None, None),
                 lambda: heal.heal_kv_attention(c, q[:, :3], None, None),
                 lambda: heal.heal_kv_attention(c, q.double(), None, None),
                 lambda: heal.heal_kv_select(c, q[0], 2, None, None),
                 lambda: heal.heal_kv_append(c, q, q, None, None),
                 lambda: heal.heal_kv_append(c, q[:, :2], q[:1, :2], None, None),
                 lambda: heal.heal_kv_read(None, 2, None, None)):
        with pytest.raises(heal.HealError):
            call()
