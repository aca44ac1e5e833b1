"""The work that the key/value cache operators are measured on.

One cache holds the keys and values of many sequences in blocks of tokens:

  k_codes   int8  (blocks, heads, block, dim)       127 x / m of every complete block
  v_codes   int8  (blocks, heads, dim, block)       tokens of a block in the order of `_order`
  scales    fp32  (blocks, heads, 2)                m = max|x| of the block's keys, values
  k_mean    fp32  (blocks, heads, dim)              mean of the block's keys
  k_recent  fp32  (slots, heads, 2 * block, dim)    rows of the last two blocks, at place % (2 * block)
  v_recent  fp32  (slots, heads, dim, 2 * block)

A sequence is a row of `table` (its blocks), a length (`lens`, the new tokens
included) and a slot; its tokens in a call are cu[i] to cu[i + 1].  Complete
blocks are read from their codes, the rows behind them from the FP32 rows.

  append     new keys (rotated by their place) and values enter the cache, the
             queries are rotated too; the rows of every block touched are read back;
  attention  the new tokens' queries against the cache, causal, with a window,
             or (``sel`` > 0) over a list of blocks for each token and head;
  select     that list: the blocks whose mean key scores highest, the first and
             the last block always.

Sizes are those of a Llama-3.1-8B layer (32 heads in groups of 4, 128 wide) or
generic ones; blocks of 64 tokens unless a case says otherwise.
"""
import numpy as np
import torch

own = False


def _case(name, op, seqs, tokens, ctx, heads=8, group=4, dim=128, block=64, **more):
    c = {"name": name, "op": op, "seqs": seqs, "tokens": tokens, "ctx": ctx, "heads": heads,
         "group": group, "dim": dim, "block": block, "pad": 0}
    if op == "append":
        c.update(rot=dim, interleaved=False)
    elif op == "attention":
        c.update(window=0, sel=0)
    c.update(more)
    return c


def listed():
    return [
        # one token of one sequence enters the cache: latency counts
        _case("append-token", "append", 1, 1, 1000),
        # a decode step of 64 sequences, some of which fill a block
        _case("append-batch", "append", 64, 1, 4096),
        # drafted tokens of narrow heads, half of each head rotated, in pairs side by side
        _case("append-drafts", "append", 13, 5, 333, heads=5, group=3, dim=96, block=16, rot=48,
              interleaved=True),
        # four ragged prompts
        _case("append-prompts", "append", 4, 4096, 4096),
        # one token of one long sequence
        _case("decode-one", "attention", 1, 1, 8191),
        # a decode step of 64 sequences of 4096 to 8192 tokens, three places of the batch unused
        _case("decode-batch", "attention", 64, 1, 8192, pad=3),
        # drafted tokens of small odd heads within a window
        _case("decode-drafts", "attention", 13, 5, 3001, heads=5, group=3, dim=64, block=32, window=1000),
        # two ragged prompts against themselves
        _case("prompts", "attention", 2, 2048, 2048),
        # a chunk of a long prompt
        _case("chunk", "attention", 1, 512, 16001),
        # a decode step over 48 of 512 blocks
        _case("decode-selected", "attention", 32, 1, 32768, sel=48),
        # which blocks a decode step of long sequences reads
        _case("select-batch", "select", 32, 1, 32768, sel=48),
        # ... and every token of a chunk of a prompt
        _case("select-chunk", "select", 1, 777, 5000, sel=16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """One more case: 1 to 64 sequences of 1 to 32768 tokens, single tokens, 2 to
    8 drafted ones or prompts; heads 64, 96 or 128 wide, 1 to 8 of them with 1 to
    8 queries each, blocks of 16 to 128 tokens."""
    op = rng.choice(("append", "attention", "attention", "select"))
    kind = rng.choice(("one", "drafts", "prompt"))
    heads, group = rng.choice((1, 2, 3, 4, 5, 8)), rng.choice((1, 2, 3, 4, 7, 8))
    dim, block = rng.choice((64, 96, 128)), rng.choice((16, 32, 64, 64, 128))
    if kind == "prompt":
        tokens, seqs = _log_int(rng, 9, 2048), rng.randint(1, 4)
        # a prompt, or its next part (which begins a block)
        ctx = tokens if op == "append" or rng.random() < 0.5 else tokens + _log_int(rng, 1, 8192)
        while op == "attention" and seqs * tokens * ctx * heads * group * dim > 2 * 2048 * 2048 * 32 * 128:
            tokens, ctx = tokens // 2 + 1, ctx // 2 + 1
    else:
        tokens = 1 if kind == "one" else rng.randint(2, 8)
        seqs = _log_int(rng, 1, 64)
        ctx = max(tokens, _log_int(rng, 1, 32768))
        while seqs * ctx * heads * dim > 64 * 6144 * 8 * 128:
            ctx = max(tokens, ctx // 2 + 1)
    c = _case("", op, seqs, tokens, ctx, heads, group, dim, block)
    del c["name"]
    if op != "append" and kind == "one":
        c["pad"] = rng.choice((0, 0, 1, 5))
    if op == "append":
        c["rot"], c["interleaved"] = rng.choice((dim, dim, dim // 2, 0)), rng.random() < 0.5
    elif op == "attention":
        if rng.random() < 0.25:
            c["window"] = _log_int(rng, 1, 4096)
        elif kind != "prompt" and rng.random() < 0.4:
            c["sel"] = _log_int(rng, 2, 64)
    else:
        c["sel"] = _log_int(rng, 2, 64)
    return c


def _sequences(c):
    """(new tokens, length) of every sequence; `pad` more at the end are unused
    places of the batch: a token each, and no length."""
    n, length = [], []
    for i in range(c["seqs"]):
        t = max(1, c["tokens"] - i * 61 % (c["tokens"] // 2 + 1))
        at = max(t, c["ctx"] - i * 67 % (c["ctx"] // 2 + 1))
        if c["op"] == "append" and t > c["block"]:
            at = t + (at - t) // c["block"] * c["block"]   # a prompt's part begins a block
        n.append(t)
        length.append(at)
    return n + [1] * c["pad"], length + [0] * c["pad"]


def _order(block):
    """The place of each token among the values of a block: token 16 s + 4 g + i
    is at g * block / 4 + 4 s + i."""
    t = torch.arange(block)
    return t % 16 // 4 * (block // 4) + t // 16 * 4 + t % 4


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, H, d, dev = c["block"], c["heads"], c["dim"], "cuda"
    n, length = _sequences(c)
    N, T, heads_q = len(n), sum(n), H * c["group"]
    blocks = [-(-x // B) for x in length]
    cols, total = max(blocks), sum(blocks)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev)

    # every sequence's blocks lie anywhere in the cache, which has a few more
    pages = torch.randperm(total + 5, generator=g, device=dev).to(torch.int32).tolist()
    table, at = [], 0
    for b in blocks:
        table.append(pages[at:at + b] + [-1] * (cols - b))
        at += b
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    slots = torch.randperm(N + 2, generator=g, device=dev)[:N].to(torch.int32)
    cu = [0]
    for t in n:
        cu.append(cu[-1] + t)
    P = total + 5
    s = {"case": c, "B": B, "H": H, "G": c["group"], "d": d, "T": T, "N": N, "cols": cols,
         "table": ints(table), "lens": ints(length), "slots": slots, "cu": None if T == N else ints(cu),
         "scale": d ** -0.5, "q": randn(T, heads_q, d)}
    if c["op"] == "select":   # needs no codes
        codes = lambda *shape: torch.empty(shape, dtype=torch.int8, device=dev)  # noqa: E731
        recent = lambda *shape: torch.empty(shape, device=dev)  # noqa: E731
    else:
        def codes(*shape):
            x = torch.empty(shape, dtype=torch.int8, device=dev)
            for part in x.view(shape[0], -1).split(4096):
                part.copy_(torch.randn(part.shape, generator=g, device=dev).mul_(36.0).round_().clamp_(-127, 127))
            return x
        recent = randn
    # keys have a few wide channels
    wide = torch.ones(d, device=dev)
    wide[torch.randperm(d, generator=g, device=dev)[:2]] = 3.0
    s["cache"] = (codes(P, H, B, d), codes(P, H, d, B),
                  torch.rand((P, H, 2), generator=g, device=dev) * 3.0 + 2.0, randn(P, H, d) * 0.3,
                  recent(N + 2, H, 2 * B, d).mul_(wide), recent(N + 2, H, d, 2 * B))
    # the scale of an incomplete block is the largest of the rows it has
    if c["op"] == "attention":
        for i, (x, slot) in enumerate(zip(length, slots.tolist())):
            if x % B:
                b = x // B
                rows = slice(b % 2 * B, b % 2 * B + x % B)
                kr, vr = s["cache"][4][slot, :, rows], s["cache"][5][slot, :, :, rows]
                s["cache"][2][table[i][b], :, 0] = kr.abs().amax((1, 2))
                s["cache"][2][table[i][b], :, 1] = vr.abs().amax((1, 2))
    # places of the tokens, and the tokens of each sequence side by side
    width = max(n)
    seq = [i for i, t in enumerate(n) for _ in range(t)]
    col = [j for t in n for j in range(t)]
    s["seq"], s["col"], s["width"] = ints(seq).long(), ints(col).long(), width
    s["place"] = ints([length[i] - n[i] + j for i, j in zip(seq, col)])
    if c["op"] == "append":
        s["k"], s["v"] = randn(T, H, d) * wide, randn(T, H, d)
        s.update(_append_plan(n, length, table, slots.tolist(), B, ints))
        places = max(length)
        half = c["rot"] // 2
        if half:
            freq = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)
            angle = torch.arange(places, dtype=torch.float64, device=dev)[:, None] * freq
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        else:
            s["cos"] = s["sin"] = None
    elif c["op"] == "attention" and c["sel"]:
        s["sel"] = _any_blocks(s, c, g)
    return s


def _append_plan(n, length, table, slots, B, ints):
    """What a scheduler knows of the tokens that it appends: every block touched, where
    each of its rows comes from (a new token, or a row of the ring), the rows that stay
    in the ring, and the rows to read back (whole blocks from the first one touched)."""
    T = sum(n)
    block, src, have, full, ring_to, ring_from, cu_read, seqs, first = [], [], [], [], [], [], [0], [], []
    t0 = 0
    for i, (t, x) in enumerate(zip(n, length)):
        start, slot = x - t, slots[i]
        for b in range(start // B, (x - 1) // B + 1):
            block.append(table[i][b])
            row = [p if p < x else -1 for p in range(b * B, b * B + B)]
            have.append([p >= 0 for p in row])
            src.append([0 if p < 0 else t0 + p - start if p >= start else T + slot * 2 * B + p % (2 * B) for p in row])
            full.append(x >= b * B + B)
        for p in range(max(start, ((x - 1) // B - 1) * B), x):
            ring_to.append(slot * 2 * B + p % (2 * B))
            ring_from.append(t0 + p - start)
        seqs.append(i)
        first.append(start // B * B)
        cu_read.append(cu_read[-1] + x - start // B * B)
        t0 += t
    whole = [u for u, f in enumerate(full) if f]
    read_unit, read_row = [], []
    for u, h in enumerate(have):
        k = sum(h)
        read_unit += [u] * k
        read_row += range(k)
    return {"block": ints(block).long(), "src": ints(src).long(), "have": torch.tensor(have, device="cuda"),
            "whole": ints(whole).long(), "ring_to": ints(ring_to).long(), "ring_from": ints(ring_from).long(),
            "cu_read": ints(cu_read), "read": cu_read[-1], "read_unit": ints(read_unit).long(),
            "read_row": ints(read_row).long(), "full": torch.tensor(full, device="cuda")}


def _any_blocks(s, c, g):
    """A list of blocks for each token and head: its last one, the first, and any others, ascending."""
    T, H, B, k = s["T"], s["H"], s["B"], c["sel"]
    last = torch.div(s["place"], B, rounding_mode="floor")
    nb = (last + 1).clamp(min=0)
    key = torch.rand((T, H, s["cols"] + k), generator=g, device="cuda")
    b = torch.arange(s["cols"] + k, device="cuda")
    key = torch.where((b == last[:, None])[:, None] | (b == 0), key - 2.0, key)
    key = torch.where((b >= nb[:, None])[:, None], torch.full_like(key, 3.0), key)
    value, at = key.sort(dim=-1)
    at = torch.where(value[..., :k] < 2.0, at[..., :k], torch.full_like(at[..., :k], 1 << 30))
    at = at.sort(dim=-1).values
    return torch.where(at < 1 << 30, at, torch.full_like(at, -1)).to(torch.int32)


# ---- the operators -----------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"append": _append, "attention": _attention, "select": _select}[op](s)


def _own(s, op):
    import paper_2606_21023_amd as heal
    if "handle" not in s:   # a program keeps its cache
        s["handle"] = heal.KVCache(*s["cache"])
    cache, c = s["handle"], s["case"]
    seqs = {"table": s["table"], "lens": s["lens"], "cu": s["cu"], "slots": s["slots"]}
    if op == "append":
        q = heal.heal_kv_append(cache, s["k"], s["v"], **seqs, cos=s["cos"], sin=s["sin"],
                                interleaved=c["interleaved"], q=s["q"])
        seqs["cu"] = s["cu_read"]
        k, v = heal.heal_kv_read(cache, s["read"], **seqs)
        return {"q": q, "k": k, "v": v, "scales": cache.scales, "mean": cache.k_mean}
    if op == "select":
        return heal.heal_kv_select(cache, s["q"], c["sel"], **seqs, keep_first=1, keep_last=1)
    lse = torch.empty((s["T"], s["H"] * s["G"]), device="cuda")
    out = heal.heal_kv_attention(cache, s["q"], **seqs, scale=s["scale"], window=c["window"], sel=s.get("sel"),
                                 lse=lse)
    return {"out": out, "lse": lse}


def _rotate(x, s):
    """x (tokens, heads, dim) rotated by the tokens' places, in 64 bits, rounded once."""
    if s["cos"] is None:
        return x
    r = s["case"]["rot"]
    at = s["place"].long()
    co, si = s["cos"][at].double()[:, None], s["sin"][at].double()[:, None]
    y = x[..., :r].double()
    if s["case"]["interleaved"]:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack((a * co - b * si, b * co + a * si), -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:]
        y = torch.cat((a * co - b * si, b * co + a * si), -1)
    return torch.cat((y.float(), x[..., r:]), -1)


def _append(s):
    kc, vc, scales, mean, kr, vr = s["cache"]
    B, H, d = s["B"], s["H"], s["d"]
    q, k, v = _rotate(s["q"], s), _rotate(s["k"], s), s["v"]
    krows, vrows = kr.transpose(1, 2).reshape(-1, H, d), vr.permute(0, 3, 1, 2).reshape(-1, H, d)
    have = s["have"][:, :, None, None]
    # the rows of every block touched: units, block, heads, dim
    K = torch.where(have, torch.cat((k, krows))[s["src"]], 0.0)
    V = torch.where(have, torch.cat((v, vrows))[s["src"]], 0.0)
    mk, mv = K.abs().amax((1, 3)), V.abs().amax((1, 3))
    scales[s["block"]] = torch.stack((mk, mv), -1)
    mean[s["block"]] = (K.double().sum(1) / s["have"].sum(1)[:, None, None]).float()
    K8, V8 = _codes(K, mk), _codes(V, mv)
    at, u = s["block"][s["whole"]], s["whole"]
    kc[at] = K8[u].transpose(1, 2).to(torch.int8)
    order = _order(B).to("cuda")
    vc[at] = torch.empty_like(vc[at]).index_copy_(3, order, V8[u].permute(0, 2, 3, 1).to(torch.int8).contiguous())
    # the rows that stay as they are
    to, slot = s["ring_to"] % (2 * B), s["ring_to"] // (2 * B)
    kr[slot, :, to] = k[s["ring_from"]]
    vr[slot, :, :, to] = v[s["ring_from"]]
    # read back what the cache holds
    full = s["full"][:, None, None, None]
    K = torch.where(full, K8 * (mk / 127.0)[:, None, :, None], K)
    V = torch.where(full, V8 * (mv / 127.0)[:, None, :, None], V)
    ru, rr = s["read_unit"], s["read_row"]
    return {"q": q, "k": K[ru, rr], "v": V[ru, rr], "scales": scales, "mean": mean}


def _codes(x, m):
    """Round(127 x / m), ties to even, decided in 64 bits; zeros where m is 0."""
    m = m.double()[:, None, :, None]
    return torch.where(m > 0, torch.round(127.0 * x.double() / m), 0.0).float()


def _rows(s):
    """Keys and values of the whole batch in 32 bits: sequences, heads, dim wide rows of
    every place of the table and one block more."""
    kc, vc, scales, _, kr, vr = s["cache"]
    B, H, d, N = s["B"], s["H"], s["d"], s["N"]
    order = _order(B).to("cuda")
    t = s["table"].long().clamp(min=0)
    t = torch.cat((t, t.new_zeros(N, 1)), 1)
    sc = scales[t] / 127.0
    K = kc[t].float() * sc[..., 0, None, None]
    V = vc[t][..., order].float().mul_(sc[..., 1, None, None]).transpose(-1, -2)
    K, V = K.contiguous(), V.contiguous()
    last = torch.div(s["lens"].long(), B, rounding_mode="floor")
    i = torch.arange(N, device="cuda")
    half = last % 2
    K[i, last] = kr.view(-1, H, 2, B, d)[s["slots"].long(), :, half]
    V[i, last] = vr.view(-1, H, d, 2, B)[s["slots"].long(), :, :, half].transpose(-1, -2)
    flat = lambda x: x.transpose(1, 2).reshape(N, H, -1, d)  # noqa: E731
    return flat(K), flat(V)


def _softmax(x, mask):
    """Weights of the last axis where mask holds (0 in rows without any), and the row's
    logarithm of the sum."""
    x = torch.where(mask, x, -torch.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -torch.inf, 0.0, m))
    l = p.sum(-1, keepdim=True)
    return p / torch.where(l == 0, 1.0, l), (torch.log(l) + m).squeeze(-1)


def _seen(t, place, length, window):
    mask = (t <= place) & (t < length)
    return mask & (t > place - window) if window else mask


def _attention(s):
    c, H, G, d, T = s["case"], s["H"], s["G"], s["d"], s["T"]
    q = s["q"].view(T, H, G, d) * s["scale"]
    if c["sel"]:
        return _attention_selected(s, q)
    K, V = _rows(s)
    Q = q.new_zeros(s["N"], s["width"], H, G, d)
    Q[s["seq"], s["col"]] = q
    place = s["place"].new_full((s["N"], s["width"]), -1)
    place[s["seq"], s["col"]] = s["place"]
    x = Q.permute(0, 2, 1, 3, 4).reshape(s["N"], H, -1, d) @ K.transpose(-1, -2)
    t = torch.arange(K.shape[2], device="cuda")
    mask = _seen(t, place[..., None], s["lens"][:, None, None], c["window"])
    p, lse = _softmax(x.view(s["N"], H, s["width"], G, -1), mask[:, None, :, None])
    o = (p.view(s["N"], H, s["width"] * G, -1) @ V).view(s["N"], H, s["width"], G, d)
    out = o.permute(0, 2, 1, 3, 4)[s["seq"], s["col"]].reshape(T, H * G, d)
    return {"out": out, "lse": lse.permute(0, 2, 1, 3)[s["seq"], s["col"]].reshape(T, H * G)}


def _attention_selected(s, q):
    """Every token and head with its own blocks."""
    kc, vc, scales, _, kr, vr = s["cache"]
    B, H, d, T, k = s["B"], s["H"], s["d"], s["T"], s["case"]["sel"]
    sel = s["sel"].long()
    seq, h = s["seq"][:, None, None], torch.arange(H, device="cuda")[None, :, None]
    page = s["table"][seq, sel.clamp(min=0)].long().clamp(min=0)
    sc = scales[page, h] / 127.0
    K = kc[page, h].float() * sc[..., 0, None, None]
    V = vc[page, h][..., _order(B).to("cuda")].float() * sc[..., 1, None, None]
    length = s["lens"].long()[seq]
    rows = (sel * B + B > length)[..., None, None]   # a block that is not complete
    half, slot = sel.clamp(min=0) % 2, s["slots"].long()[seq]
    K = torch.where(rows, kr.view(-1, H, 2, B, d)[slot, h, half], K)
    V = torch.where(rows, vr.view(-1, H, d, 2, B).permute(0, 1, 3, 2, 4)[slot, h, half], V)
    t = sel[..., None] * B + torch.arange(B, device="cuda")
    mask = _seen(t, s["place"][:, None, None, None], length[..., None], s["case"]["window"]) & (sel >= 0)[..., None]
    K = K.reshape(T, H, k * B, d)
    V = V.transpose(-1, -2).reshape(T, H, k * B, d)
    p, lse = _softmax(q @ K.transpose(-1, -2), mask.reshape(T, H, 1, k * B))
    return {"out": (p @ V).reshape(T, -1, d), "lse": lse.reshape(T, -1)}


def _select(s):
    B, H, G, d, T, k = s["B"], s["H"], s["G"], s["d"], s["T"], s["case"]["sel"]
    mean = s["cache"][3]
    M = mean[s["table"].long().clamp(min=0)].double()          # sequences, blocks, heads, dim
    M = M.permute(0, 2, 3, 1)
    Q = s["q"].new_zeros(s["N"], s["width"], H, G, d, dtype=torch.float64)
    Q[s["seq"], s["col"]] = s["q"].view(T, H, G, d).double()
    x = Q.permute(0, 2, 1, 3, 4).reshape(s["N"], H, -1, d) @ M
    x = x.view(s["N"], H, s["width"], G, -1).amax(3).transpose(1, 2)[s["seq"], s["col"]]   # tokens, heads, blocks
    last = torch.div(s["place"], B, rounding_mode="floor")[:, None, None]
    b = torch.arange(x.shape[-1], device="cuda")
    x = torch.where((b == last) | (b == 0), torch.inf, x)
    x = torch.where(b > last, -torch.inf, x)
    at = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :k]
    at = torch.where(at <= last, at, 1 << 30).sort(dim=-1).values
    at = torch.where(at < 1 << 30, at, -1).to(torch.int32)
    return torch.nn.functional.pad(at, (0, k - at.shape[-1]), value=-1)


# ---- what an operator cannot do without ---------------------------------------

def work(case):
    c, B, H, d = case, case["block"], case["heads"], case["dim"]
    n, length = _sequences(c)
    T, heads_q = sum(n), H * c["group"]
    if c["op"] == "append":
        # new rows and the first block's old ones in, complete blocks' codes and the rows
        # that stay FP32 out; the codes or rows read again, FP32 rows out; queries in and out
        old = sum((x - t) % B for t, x in zip(n, length))
        whole = sum(x // B * B - (x - t) // B * B for t, x in zip(n, length))
        part = sum(x - max(x // B * B, x - t) for t, x in zip(n, length))
        back = sum(x - (x - t) // B * B for t, x in zip(n, length))
        return {"bytes": H * d * (8 * (T + old) + 4 * whole + 8 * part + 8 * (back - whole) + 8 * back)
                + 8 * T * heads_q * d,
                "flops": 3 * T * (H + heads_q) * c["rot"] + 6 * back * H * d}
    if c["op"] == "select":
        blocks = sum(-(-x // B) for x in length)
        scored = sum((x - t + j) // B + 1 for t, x in zip(n, length) for j in range(t) if x)
        return {"bytes": blocks * H * 4 * d + 4 * T * heads_q * d + 4 * T * H * c["sel"],
                "flops": 2 * scored * heads_q * d}
    rows = pairs = 0
    for t, x in zip(n, length):
        if c["sel"]:
            rows += t * min(c["sel"] * B, x)
            pairs += t * min(c["sel"] * B, x)
        elif x:
            w = c["window"] or x
            rows += min(x, w + t - 1)
            pairs += sum(min(x - t + j + 1, w) for j in range(t))
    return {"bytes": rows * H * 2 * d + 8 * T * heads_q * d, "flops": 4 * pairs * heads_q * d}


# ---- from the definitions, in 64 bits -----------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "select": _exact_select}[case["op"]](s)


def _turned(x, place, s):
    """x (heads, dim) of one token at a place, as complex numbers times exp(i angle)."""
    r = s["case"]["rot"]
    y = x.double().clone()
    if not r:
        return y
    z = torch.complex(s["cos"][place].double(), s["sin"][place].double())
    i = torch.arange(r // 2, device="cuda")
    a, b = (2 * i, 2 * i + 1) if s["case"]["interleaved"] else (i, i + r // 2)
    w = torch.complex(y[:, :, a], y[:, :, b]) * z[:, None]
    y[:, :, a], y[:, :, b] = w.real, w.imag
    return y


def _exact_append(s):
    n, length = _sequences(s["case"])
    B, H, d = s["B"], s["H"], s["d"]
    kc, vc, scales, mean, kr, vr = s["cache"]
    scales, mean = scales.double(), mean.double()
    place = s["place"].long()
    q, k = _turned(s["q"], place, s), _turned(s["k"], place, s).float()   # keys are kept in 32 bits
    ks, vs, t0 = [], [], 0
    for i, (t, x) in enumerate(zip(n, length)):
        start, slot = x - t, s["slots"][i].item()
        first = start // B * B
        old = torch.arange(first, start, device="cuda") % (2 * B)
        K = torch.cat((kr[slot][:, old].transpose(0, 1), k[t0:t0 + t])).double()
        V = torch.cat((vr[slot][:, :, old].permute(2, 0, 1), s["v"][t0:t0 + t])).double()
        for b in range(first // B, -(-x // B)):
            rows, page = slice(b * B - first, b * B + B - first), s["table"][i, b].item()
            mean[page] = K[rows].mean(0)
            for j, X in enumerate((K, V)):
                part = X[rows]
                scales[page, :, j] = part.abs().amax((0, 2))
                if b * B + B <= x:
                    m = scales[page, :, j, None]
                    X[rows] = torch.where(m > 0, torch.round(part * 127.0 / m) * m / 127.0, 0.0)
        ks.append(K)
        vs.append(V)
        t0 += t
    return {"q": q, "k": torch.cat(ks), "v": torch.cat(vs), "scales": scales, "mean": mean}


def _exact_attention(s):
    c, B, H, G, d = s["case"], s["B"], s["H"], s["G"], s["d"]
    n, length = _sequences(c)
    kc, vc, scales, _, kr, vr = s["cache"]
    out = torch.zeros((s["T"], H * G, d), dtype=torch.float64, device="cuda")
    lse = torch.full((s["T"], H * G), -torch.inf, dtype=torch.float64, device="cuda")
    order = _order(B).to("cuda")
    t0 = 0
    for i, (t, x) in enumerate(zip(n, length)):
        if x:
            pages, whole = s["table"][i].long(), x // B
            tail = torch.arange(whole * B, x, device="cuda") % (2 * B)
            slot, pages = s["slots"][i].item(), pages[:whole]
            at = torch.arange(x, device="cuda")
            place = torch.arange(x - t, x, device="cuda")[:, None]
            mask = at <= place
            if c["window"]:
                mask &= at > place - c["window"]
            mask = mask[None].expand(H, t, x)
            if c["sel"]:
                listed_ = torch.zeros((t, H, -(-x // B) + 1), dtype=torch.bool, device="cuda")
                sel = s["sel"][t0:t0 + t].long()
                listed_.scatter_(2, torch.where(sel < 0, listed_.shape[2] - 1, sel), True)
                mask = mask & listed_[..., :-1].repeat_interleave(B, -1)[..., :x].transpose(0, 1)
            for h in range(H):
                K = kc[pages, h].double() * (scales[pages, h, 0].double() / 127.0)[:, None, None]
                V = vc[pages, h].double()[:, :, order].transpose(1, 2) * (scales[pages, h, 1].double() / 127.0)[:, None, None]
                K = torch.cat((K.reshape(-1, d), kr[slot, h, tail].double()))
                V = torch.cat((V.reshape(-1, d), vr[slot, h][:, tail].t().double()))
                Q = s["q"][t0:t0 + t, h * G:h * G + G].double()
                a = (Q.reshape(-1, d) @ K.t().contiguous()).view(t, G, x) * d ** -0.5
                a = a.masked_fill(~mask[h][:, None], -torch.inf)
                e = torch.logsumexp(a, -1)
                w = torch.exp(a - e[..., None]).nan_to_num(0.0)
                out[t0:t0 + t, h * G:h * G + G] = (w.view(-1, x) @ V).view(t, G, d)
                lse[t0:t0 + t, h * G:h * G + G] = e
        t0 += t
    return {"out": out, "lse": lse}


def _exact_select(s):
    c, B, H, G, k = s["case"], s["B"], s["H"], s["G"], s["case"]["sel"]
    n, length = _sequences(c)
    found = np.full((s["T"], H, k), -1, np.int32)
    t0 = 0
    for i, (t, x) in enumerate(zip(n, length)):
        if x:
            nb = -(-x // B)
            M = s["cache"][3][s["table"][i, :nb].long()].double()
            for h in range(H):
                Q = s["q"][t0:t0 + t, h * G:h * G + G].double()
                score = (Q.reshape(t * G, -1) @ M[:, h].t().contiguous()).view(t, G, nb).amax(1).cpu().numpy()
                for j in range(t):
                    last = (x - t + j) // B
                    others = np.argsort(-score[j, 1:max(1, last)], kind="stable") + 1
                    pick = np.unique(np.concatenate(([0, last], others[:k - 2])))
                    found[t0 + j, h, :len(pick)] = pick
        t0 += t
    return torch.from_numpy(found).cuda()
