"""Calls of more workgroups than one launch has (2^22), against the same tokens in small calls
and, for what append writes, against the definition."""
import numpy as np
import pytest
import torch

import kv_ref
import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

SEQS, HEADS, GROUP, DIM, B = 70000, 64, 4, 64, 16   # SEQS * HEADS > 2^22
SLICES = [(0, 40), (65530, 65570), (SEQS - 40, SEQS)]


def test_calls_of_many_workgroups():
    """One token of each of 70000 sequences, the last one of a block: the earlier rows are
    zeros (slots that are not there)."""
    g = torch.Generator(device="cuda").manual_seed(5)
    c = heal.KVCache.empty(SEQS, 1, HEADS, DIM, B)
    table = torch.randperm(SEQS, generator=g, device="cuda").to(torch.int32)[:, None].contiguous()
    lens = torch.full((SEQS,), B, dtype=torch.int32, device="cuda")
    none = torch.full((SEQS,), -1, dtype=torch.int32, device="cuda")
    k, v, q = (torch.randn(SEQS, HEADS, DIM, generator=g, device="cuda") for _ in range(3))
    angle = torch.arange(B, device="cuda")[:, None] * 0.1 ** torch.arange(DIM // 2, device="cuda")[None]
    cos, sin = angle.cos().contiguous(), angle.sin().contiguous()
    announce("append")
    q_out = heal.heal_kv_append(c, k, v, table, lens, slots=none, cos=cos, sin=sin, q=q)
    torch.cuda.synchronize()
    co, si = cos.cpu().numpy(), sin.cpu().numpy()
    for lo, hi in SLICES:
        for i in (lo, hi - 1):
            assert np.array_equal(q_out[i].cpu().numpy(), kv_ref.rotate(q[i].cpu().numpy(), B - 1, co, si, False))
            rows = np.zeros((B, HEADS, DIM), np.float32)
            rows[-1] = kv_ref.rotate(k[i].cpu().numpy(), B - 1, co, si, False)
            page = int(table[i, 0])
            for h in (0, HEADS - 1):
                assert np.array_equal(c.k_codes[page, h].cpu().numpy(), kv_ref.codes(rows[:, h])[0])
                assert np.array_equal(c.v_codes[page, h, :, B - 1].cpu().numpy(), kv_ref.codes(v[i, h].cpu().numpy())[0])
                # an FP64 sum of 16, rounded once
                assert np.abs(c.k_mean[page, h].cpu().numpy() - rows[-1, h] / 16.0).max() <= 2.0 ** -24 * np.abs(rows[-1, h] / 16.0).max()
    del k, v, q, q_out

    announce("read")
    whole = heal.heal_kv_read(c, SEQS, table, lens, slots=none)
    for lo, hi in SLICES:
        part = heal.heal_kv_read(c, hi - lo, table[lo:hi], lens[lo:hi], slots=none[lo:hi])
        assert all(torch.equal(x[lo:hi], y) for x, y in zip(whole, part)) and part[0].any()
    del whole

    # nine blocks a sequence, its neighbours' among them: chunks of 64 tokens make three parts
    table = torch.stack([table[:, 0].roll(-j) for j in range(9)], 1).contiguous()
    lens = torch.randint(1, 10, (SEQS,), generator=g, device="cuda").to(torch.int32) * B
    q = torch.randn(SEQS, HEADS * GROUP, DIM, generator=g, device="cuda")
    announce("select")
    sel = heal.heal_kv_select(c, q, 3, table, lens, slots=none)
    for lo, hi in SLICES:
        assert torch.equal(sel[lo:hi], heal.heal_kv_select(c, q[lo:hi], 3, table[lo:hi], lens[lo:hi], slots=none[lo:hi]))
    for kw in (dict(), dict(sel=sel)):
        announce("attention %s" % list(kw))
        lse = torch.empty(SEQS, HEADS * GROUP, device="cuda")
        whole = heal.heal_kv_attention(c, q, table, lens, slots=none, chunk=64, lse=lse, **kw)
        for lo, hi in SLICES:
            kw2 = {n: x[lo:hi] for n, x in kw.items()}
            lse2 = torch.empty(hi - lo, HEADS * GROUP, device="cuda")
            part = heal.heal_kv_attention(c, q[lo:hi], table[lo:hi], lens[lo:hi], slots=none[lo:hi], chunk=64, lse=lse2, **kw2)
            assert torch.equal(whole[lo:hi], part) and torch.equal(lse[lo:hi], lse2) and part.any(2).all()
        del whole
    torch.cuda.empty_cache()
