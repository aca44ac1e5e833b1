"""The calls of a decoder layer one after another, as a server of many requests makes them:
two steps of four requests that share a prompt, against the layer in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2606_21023_amd as heal
from gpu_util import announce, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

D, H, G, DIM, BLOCK, EPS = 512, 2, 2, 64, 16, 1e-5
QKV = (H * G + 2 * H) * DIM


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Layer:
    def __init__(self):
        torch.manual_seed(0)
        r = lambda *s: torch.randn(s, device="cuda")  # noqa: E731
        self.wqkv, self.wo = r(D, QKV) * D ** -0.5, r(H * G * DIM, D) * 0.06
        self.n1, self.n2, self.nq, self.post = (1 + 0.1 * r(n) for n in (D, D, DIM, D))
        self.bank = heal.LoraBank(r(3, 8, D) * D ** -0.5, r(3, QKV, 8) * 0.1, scales=r(3))
        self.obank = heal.LoraBank((r(3, 4, H * G * DIM) * 0.06).bfloat16(), (r(3, D, 4) * 0.1).bfloat16(), ranks=ints([4, 1, 0]))


def step(L, cache, pool, table, lens, cu, h, ids):
    """One layer on the tokens' residual h; returns the residual and what the next block takes."""
    T = len(h)
    _, a = heal.heal_block_norm(h, pre=L.n1, eps=EPS)
    qkv = heal.heal_gemm_f32(a, L.wqkv)
    heal.heal_lora_add(qkv, a, L.bank, ids, cu=cu, out=qkv)
    qkv = qkv.view(T, H * G + 2 * H, DIM)
    q, k, v = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
    heal.heal_block_norm(q, pre=L.nq, eps=EPS, out=q)
    missing = heal.heal_kv_reserve(pool, T, table, lens, cu=cu)
    heal.heal_kv_append(cache, k, v, table, lens, cu=cu)
    o = heal.heal_kv_attention(cache, q, table, lens, cu=cu).view(T, -1)
    y = heal.heal_gemm_f32(o, L.wo)
    heal.heal_lora_add(y, o, L.obank, ids, cu=cu, out=y)
    h, a = heal.heal_block_norm(h, y, post=L.post, scale=0.5, pre=L.n2, eps=EPS)
    return h, a, missing


def rms(x, w):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * w


def layer64(L, past, h, adapter):
    """The layer for one sequence's new tokens h; past: [k, v] rows so far, extended here."""
    n = lambda t: t.double().cpu().numpy()  # noqa: E731
    s = 1.0

    def adapted(x, bank):
        if not 0 <= adapter < bank.adapters:
            return 0.0
        r = bank.rank if bank.ranks is None else int(bank.ranks[adapter])
        s = 1.0 if bank.scales is None else float(bank.scales[adapter])
        return s * (x @ n(bank.a[adapter, :r]).T) @ n(bank.b[adapter, :, :r]).T
    a = rms(h, n(L.n1))
    qkv = (a @ n(L.wqkv) + adapted(a, L.bank)).reshape(len(h), -1, DIM)
    q, k, v = rms(qkv[:, :H * G], n(L.nq)), qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
    past[0], past[1] = np.concatenate([past[0], k]), np.concatenate([past[1], v])
    o = np.zeros_like(q)
    for t in range(len(h)):
        end = len(past[0]) - len(h) + t + 1
        for j in range(H * G):
            x = past[0][:end, j // G] @ q[t, j] * DIM ** -0.5
            p = np.exp(x - x.max())
            o[t, j] = p / p.sum() @ past[1][:end, j // G]
    o = o.reshape(len(h), -1)
    h = h + 0.5 * rms(o @ n(L.wo) + adapted(o, L.obank), n(L.post))
    return h, rms(h, n(L.n2))


def test_steps_of_requests_that_share_a_prompt():
    L, prompt, rows = Layer(), 12, 4
    cache, pool = heal.KVCache.empty(30, rows, H, DIM, BLOCK), heal.KVPool.empty(30, BLOCK)
    table = torch.full((rows, 6), -1, dtype=torch.int32, device="cuda")
    h = torch.randn(prompt, D, device="cuda")
    announce("prompt")
    n = [prompt, 0, 0, 0]
    got, _, missing = step(L, cache, pool, table, ints(n), ints([0] + [prompt] * 4), h, ints([1, -1, -1, -1]))
    past = [np.zeros((0, H, DIM)), np.zeros((0, H, DIM))]
    want, _ = layer64(L, past, h.double().cpu().numpy(), 1)
    assert missing.item() == 0

    def same(got, want):
        # the products keep 16 of 24 bits of each operand (2^-16 of their terms' magnitudes, which over
        # hundreds of random terms is some 2^-16 of the largest results); norms and softmax pass that on
        # with factors of a few, through three products in a row: 2^-10 of the largest result is 20 times that
        got = got.double().cpu().numpy()
        assert np.abs(got - want).max() <= 2.0 ** -10 * np.abs(want).max()
    same(got, want)
    # the others continue the same prompt, with adapters of their own
    heal.heal_kv_fork(pool, table, ints(n), ints([0, 0, 0]), ints([1, 2, 3]))
    heal.heal_kv_copy(cache, slots=(ints([0, 0, 0]), ints([1, 2, 3])))
    pasts = [[p.copy() for p in past] for _ in range(rows)]
    n, ids = [prompt] * rows, [1, 0, -1, 2]
    for counts in ([1, 1, 1, 1], [1, 2, 1, 2]):   # all blocks stay incomplete: FP32 rows throughout
        n = [a + b for a, b in zip(n, counts)]
        cu = np.concatenate([[0], np.cumsum(counts)])
        h = torch.randn(int(cu[-1]), D, device="cuda")
        announce("step %s" % counts)
        got, a, missing = step(L, cache, pool, table, ints(n), ints(cu), h, ints(ids))
        assert missing.item() == 0
        for i in range(rows):
            rows_ = slice(int(cu[i]), int(cu[i + 1]))
            want = layer64(L, pasts[i], h[rows_].double().cpu().numpy(), ids[i])
            same(got[rows_], want[0])
            same(a[rows_], want[1])
    assert (pool.refs > 0).sum().item() == 4   # the prompt's block is whose it was, each other has one
