"""The work that the residual norms, the adapters and the cache's pages are measured on.

  norm      the residual stream between two blocks of a layer: the output of the block that
            ends is normed (``post``), gated and scaled, added to the stream, and the sum is
            normed for the block that begins (``pre``); or the norm of every query head;
  lora      low-rank adapters of many requests beside a shared projection: the tokens of
            a sequence get  y + s B (A x)  with their sequence's adapter, or y where it has none;
  branch    the pages of a cache in a step of a server that samples several continuations:
            finished and refused tokens give their blocks up, sequences fork into empty
            rows, their FP32 rows are copied, and the step's tokens get blocks of their own;
  compact   the held blocks move to the front of the cache, tables and counts follow.

Sizes are those of a Llama-3.1-8B layer (hidden 4096, MLP 14336, 32 heads in groups of 4, 128
wide) or generic ones.
"""
import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _norm(name, rows, dim, heads=0, post=False, gate="none", pre=True, centred=False, add=True):
    return {"name": name, "op": "norm", "rows": rows, "dim": dim, "heads": heads, "post": post, "gate": gate,
            "pre": pre, "centred": centred, "add": add}


def _lora(name, seqs, tokens, k, n, rank, adapters, type="fp32", bare=False):
    return {"name": name, "op": "lora", "seqs": seqs, "tokens": tokens, "k": k, "n": n, "rank": rank,
            "adapters": adapters, "type": type, "bare": bare}


def _pages(name, op, rows, ctx, heads=8, dim=128, block=64, tokens=1, forks=0):
    return {"name": name, "op": op, "rows": rows, "ctx": ctx, "heads": heads, "dim": dim, "block": block,
            "tokens": tokens, "forks": forks}


def listed():
    return [
        # one token's residual and the next norm: latency counts
        _norm("norm-token", 1, 4096),
        # a decode step with norms on both sides of the block and a factor for every channel
        _norm("norm-batch", 64, 4096, post=True, gate="column"),
        # the tokens of a prompt, norms on both sides
        _norm("norm-prompts", 4096, 4096, post=True),
        # the query heads of a prompt, out of the rows that a joint projection wrote
        _norm("norm-heads", 2048, 128, heads=32, add=False),
        # one token with an adapter
        _lora("lora-token", 1, 1, 4096, 4096, 16, 8),
        # a decode step of 64 requests with 24 adapters of ranks up to 64, some without any
        _lora("lora-decode", 64, 1, 4096, 14336, 64, 24, type="bf16", bare=True),
        # drafted tokens through an odd, deep projection
        _lora("lora-drafts", 13, 5, 14335, 1001, 24, 5, type="fp16"),
        # ragged prompts of four requests
        _lora("lora-prompts", 4, 1365, 4096, 4096, 16, 8),
        # a prompt that forks into four continuations
        _pages("branch-few", "branch", 4, 1000, forks=3),
        # a decode step of 96 sequences, some of which fork, finish or are cut back
        _pages("branch-batch", "branch", 96, 4096, forks=20, tokens=4),
        # a small cache with holes
        _pages("compact-few", "compact", 13, 700, heads=5, dim=96, block=16),
        # a cache that half emptied
        _pages("compact-half", "compact", 32, 4096),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """One more case: norms of 1 to 16384 rows of 64 to 16384, or of heads; 1 to 64
    sequences of 1 to 4096 tokens with 1 to 32 adapters of ranks up to 128; caches of up to
    128 sequences of 1 to 16384 tokens."""
    op = rng.choice(("norm", "lora", "lora", "branch", "compact"))
    if op == "norm":
        heads = rng.choice((0, 0, 0, 1, 5, 8, 32))
        dim = rng.choice((64, 96, 128)) if heads else _log_int(rng, 64, 16384)
        if not heads and rng.random() < 0.6:
            dim = (dim + 31) // 32 * 32
        rows = _log_int(rng, 1, 16384)
        while rows * dim * max(heads, 1) > 4096 * 4096:
            rows = rows // 2 + 1
        add = not heads and rng.random() < 0.8
        pre = not add or rng.random() < 0.85
        c = _norm("", rows, dim, heads, add and rng.random() < 0.5,
                  rng.choice(("none", "column", "row", "full")) if add else "none", pre, rng.random() < 0.3, add)
    elif op == "lora":
        kind = rng.choice(("one", "drafts", "prompt"))
        seqs = rng.randint(1, 4) if kind == "prompt" else _log_int(rng, 1, 64)
        tokens = _log_int(rng, 9, 4096) if kind == "prompt" else 1 if kind == "one" else rng.randint(2, 8)
        k, n = _log_int(rng, 64, 14336), _log_int(rng, 64, 14336)
        if rng.random() < 0.7:
            k, n = (k + 31) // 32 * 32, (n + 31) // 32 * 32
        rank = rng.choice((1, 4, 8, 8, 16, 16, 24, 32, 64, 128))
        while seqs * tokens * (k + 2 * n + 128 * rank) > 4096 * (3 * 4096 + 128 * 16):
            tokens, k, n = tokens // 2 + 1, k * 3 // 4, n * 3 // 4
        c = _lora("", seqs, tokens, k, n, rank, _log_int(rng, 1, 32), rng.choice(tuple(TYPES)), rng.random() < 0.5)
    else:
        rows, block = _log_int(rng, 2, 128), rng.choice((16, 32, 64, 64, 128))
        heads, dim = rng.choice((1, 2, 5, 8)), rng.choice((64, 96, 128))
        ctx = _log_int(rng, 1, 16384)
        most = 96 * 4096 if op == "branch" else 32 * 4096
        while rows * (ctx + (4 * block if op == "branch" else 0)) * heads * dim > most * 8 * 128 or rows * ctx > 64 * most:
            rows, ctx = rows * 2 // 3 + 1, ctx * 2 // 3 + 1
        c = _pages("", op, rows, ctx, heads, dim, block, rng.choice((1, 1, 1, 3, 8, 40)),
                   rng.randint(0, rows // 2) if op == "branch" else 0)
    del c["name"]
    return c


# ---- what a user's program has ------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    if case["op"] == "norm":
        return _prepare_norm(case, randn)
    if case["op"] == "lora":
        return _prepare_lora(case, seed, randn)
    return _prepare_pages(case, seed, g, randn)


def _prepare_norm(c, randn):
    rows, dim, heads = c["rows"], c["dim"], c["heads"]
    s = {"case": c, "eps": 1e-5}
    if heads:   # queries as they stand beside keys and values
        wide = randn(rows, heads + 2 * max(heads // 4, 1), dim)
        s["h"] = wide[:, :heads]
    else:   # a few channels of the stream are far larger than the others
        s["h"] = randn(rows, dim)
        s["h"][:, :max(1, dim // 1000)] *= 50.0
    weight = lambda: 1.0 + 0.1 * randn(dim)  # noqa: E731
    s["x"] = randn(rows, dim) * 0.3 if c["add"] else None
    s["post"], s["post_bias"] = weight() if c["post"] else None, randn(dim) * 0.1 if c["post"] and c["centred"] else None
    s["pre"], s["pre_bias"] = weight() if c["pre"] else None, randn(dim) * 0.1 if c["pre"] and c["centred"] else None
    s["gate"] = {"none": lambda: None, "column": lambda: randn(1, dim), "row": lambda: randn(rows, 1),
                 "full": lambda: randn(rows, dim)}[c["gate"]]()
    s["scale"] = 0.22 if c["post"] else 1.0
    return s


def _adapters_of(c):
    """The adapter of every sequence (-1: none), the rank of every adapter, the tokens
    of every sequence."""
    seqs, many = c["seqs"], c["adapters"]
    ids = [-1 if c["bare"] and i % 7 == 3 else (i * i + 3 * i) % many for i in range(seqs)]
    ranks = [max(1, c["rank"] >> (a % 4)) for a in range(many)]
    n = [max(1, c["tokens"] - i * 61 % (c["tokens"] // 2 + 1)) for i in range(seqs)]
    return ids, ranks, n


def _prepare_lora(c, seed, randn):
    k, n, r, many = c["k"], c["n"], c["rank"], c["adapters"]
    ids, ranks, count = _adapters_of(c)
    tokens, type_ = sum(count), TYPES[c["type"]]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    cu = np.concatenate([[0], np.cumsum(count)]).tolist()
    rows = {}
    for i, a in enumerate(ids):
        if a >= 0:
            rows.setdefault(a, []).extend(range(cu[i], cu[i + 1]))
    x = randn(tokens, k)
    x[:, :max(1, k // 1000)] *= 50.0
    return {"case": c, "x": x, "y": randn(tokens, n), "a": (randn(many, r, k) * k ** -0.5).to(type_),
            "b": (randn(many, n, r) * 0.1).to(type_), "ranks": ints(ranks), "rank_list": ranks,
            "scales": 16.0 / ints(ranks).float(), "ids": ints(ids),
            "cu": None if max(count) == 1 else ints(cu), "rows": {a: ints(v).long() for a, v in rows.items()}}


def _plan(c, seed):
    """Tables and counts of a cache in use, in host memory: `table` (rows, columns), `length`
    of every row, `refs` of every block."""
    rng = np.random.default_rng(seed)
    rows, B = c["rows"], c["block"]
    length = np.array([max(1, c["ctx"] - i * 67 % (c["ctx"] // 2 + 1)) for i in range(rows)])
    branch = c["op"] == "branch"
    if branch:   # the last rows are still empty, and their number is that of the forks
        length[rows - c["forks"]:] = 0
    held = -(-length // B)
    cols = int(max(held)) + c["tokens"] // B + 2
    P = int(held.sum() * (1.1 if branch else 2.0)) + rows * (c["tokens"] // B + 3)
    pages = rng.permutation(P)
    table = np.full((rows, cols), -1, np.int64)
    at = 0
    for i in range(rows):
        shared = 0
        if i % 3 == 2 and held[i]:   # begins as the row before it
            shared = int(min(length[i - 1], length[i]) // B // 2)
            table[i, :shared] = table[i - 1, :shared]
        table[i, shared:held[i]] = pages[at:at + held[i] - shared]
        at += held[i] - shared
    refs = np.bincount(table[table >= 0], minlength=P)
    return table, length, refs


def _prepare_pages(c, seed, g, randn):
    table, length, refs = _plan(c, seed)
    rows, B, H, d, P = c["rows"], c["block"], c["heads"], c["dim"], len(refs)
    ints = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": c, "table": ints(table), "refs": ints(refs), "P": P, "B": B}
    slots = rows + 2 if c["op"] == "branch" else 1
    if c["op"] == "branch":
        codes = lambda *shape: torch.empty(shape, dtype=torch.int8, device="cuda")  # noqa: E731
        some, ring = lambda *shape: torch.empty(shape, device="cuda"), randn  # noqa: E731
    else:
        codes = lambda *shape: torch.randint(-127, 128, shape, generator=g, dtype=torch.int8, device="cuda")  # noqa: E731
        some, ring = randn, lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
    s["cache"] = (codes(P, H, B, d), codes(P, H, d, B), some(P, H, 2), some(P, H, d), ring(slots, H, 2 * B, d),
                  ring(slots, H, d, 2 * B))
    if c["op"] == "compact":
        held = refs > 0
        s["moves"] = int(held[held.sum():].sum())
        return s
    # some rows are cut back by a token, one in eight finishes, and rows fork into the empty ones
    rng = np.random.default_rng(seed + 1)
    alive = rows - c["forks"]
    kept = length.copy()
    kept[:alive] = np.where(np.arange(alive) % 8 == 7, 0, np.maximum(kept[:alive] - np.arange(alive) % 3, 1))
    able = np.flatnonzero(kept > 0)
    parents = rng.choice(able, c["forks"]) if len(able) else np.zeros(c["forks"], np.int64)
    children = np.arange(alive, rows)
    n = np.zeros(rows, np.int64)
    n[kept > 0] = c["tokens"]
    n[children] = c["tokens"]
    after = kept + n
    after[children] = kept[parents] + c["tokens"]
    cu = np.concatenate([[0], np.cumsum(n)])
    units = [(i, b) for i in range(rows) if n[i] for b in range((after[i] - n[i]) // B, (after[i] - 1) // B + 1)]
    s.update(kept=ints(kept), parents=ints(parents), children=ints(children), after=ints(after), cu=ints(cu),
             tokens=int(n.sum()), unit_row=ints([u[0] for u in units]).long(),
             unit_block=ints([u[1] for u in units]).long(), ring_from=ints(parents + 1), ring_to=ints(children + 1))
    return s


# ---- the operators -------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"norm": _own_norm, "lora": _own_lora, "branch": _own_branch, "compact": _own_compact}[op](s)
    return {"norm": _plain_norm, "lora": _plain_lora, "branch": _plain_branch, "compact": _plain_compact}[op](s)


def _own_norm(s):
    import paper_2606_21023_amd as heal
    h, out = heal.heal_block_norm(s["h"], s["x"], post=s["post"], post_bias=s["post_bias"], gate=s["gate"],
                                  scale=s["scale"], pre=s["pre"], pre_bias=s["pre_bias"], eps=s["eps"],
                                  centred=s["case"]["centred"])
    got = {}
    if s["x"] is not None:
        got["h"] = h
    if s["pre"] is not None:
        got["out"] = out
    return got


def _own_lora(s):
    import paper_2606_21023_amd as heal
    if "bank" not in s:   # a program keeps its adapters
        s["bank"] = heal.LoraBank(s["a"], s["b"], ranks=s["ranks"], scales=s["scales"])
    return heal.heal_lora_add(s["y"], s["x"], s["bank"], s["ids"], cu=s["cu"])


def _handles(s):
    import paper_2606_21023_amd as heal
    if "handle" not in s:   # a program keeps its cache, and the pool of its blocks
        s["handle"], s["working"] = heal.KVCache(*s["cache"]), s["refs"].clone()
        s["pool"] = heal.KVPool(s["working"], s["B"])
    s["working"].copy_(s["refs"])   # a pass begins with the blocks held as they were
    return heal, s["handle"], s["pool"], s["table"].clone()


def _own_branch(s):
    heal, cache, pool, table = _handles(s)
    heal.heal_kv_release(pool, table, s["kept"])
    heal.heal_kv_fork(pool, table, s["kept"], s["parents"], s["children"])
    heal.heal_kv_copy(cache, slots=(s["ring_from"], s["ring_to"]))
    missing = heal.heal_kv_reserve(pool, s["tokens"], table, s["after"], cu=s["cu"])
    return {"table": table, "refs": pool.refs, "missing": missing, "k": cache.k_recent, "v": cache.v_recent}


def _own_compact(s):
    heal, cache, pool, table = _handles(s)
    src, dst, count = heal.heal_kv_compact(pool, table)
    heal.heal_kv_copy(cache, blocks=(src, dst), count=count)
    return {"table": table, "refs": pool.refs, "src": src, "dst": dst, "count": count, "k": cache.k_codes,
            "v": cache.v_codes, "scales": cache.scales, "mean": cache.k_mean}


def _plain_normed(x, weight, bias, eps, centred):
    if centred:
        x = x - x.mean(-1, keepdim=True)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * weight
    return y if bias is None else y + bias


def _plain_norm(s):
    h, got = s["h"], {}
    centred = s["case"]["centred"]
    if s["x"] is not None:
        u = s["x"]
        if s["post"] is not None:
            u = _plain_normed(u, s["post"], s["post_bias"], s["eps"], centred)
        if s["gate"] is not None:
            u = u * s["gate"]
        h = got["h"] = h + s["scale"] * u
    if s["pre"] is not None:
        got["out"] = _plain_normed(h, s["pre"], s["pre_bias"], s["eps"], centred)
    return got


def _plain_lora(s):
    out = s["y"].clone()
    for a, rows in s["rows"].items():
        r = s["rank_list"][a]
        v = s["x"][rows] @ s["a"][a, :r].float().t()
        out[rows] += s["scales"][a] * (v @ s["b"][a, :, :r].float().t())
    return out


def _plain_release(table, refs, lens, B):
    b = torch.arange(table.shape[1], device="cuda")
    gone = (table >= 0) & (table < len(refs)) & (b >= torch.div(lens + B - 1, B, rounding_mode="floor")[:, None])
    refs.scatter_add_(0, table.clamp(min=0).long().flatten(), -gone.flatten().to(torch.int32))
    table.masked_fill_(b >= torch.div(lens + B - 1, B, rounding_mode="floor")[:, None], -1)


def _plain_branch(s):
    table, refs, B, P = s["table"].clone(), s["refs"].clone(), s["B"], s["P"]
    _plain_release(table, refs, s["kept"], B)
    # forks: the children's rows are empty
    p, c = s["parents"].long(), s["children"].long()
    row = table[p]
    held = row >= 0
    table[c] = row
    refs.scatter_add_(0, row.clamp(min=0).long().flatten(), held.flatten().to(torch.int32))
    kr, vr = s["cache"][4], s["cache"][5]
    kr[s["ring_to"].long()] = kr[s["ring_from"].long()]
    vr[s["ring_to"].long()] = vr[s["ring_from"].long()]
    # blocks for the tokens: those that are held by this row alone stay; of a block whose holders
    # are all here the first one keeps it; the others take the lowest free blocks in turn
    i, b = s["unit_row"], s["unit_block"]
    u = torch.arange(len(i), device="cuda")
    page = table[i, b].long()
    at = page.clamp(min=0)
    held = (page >= 0) & (refs[at] >= 1)
    k = torch.zeros(P, dtype=torch.int32, device="cuda").scatter_add_(0, at, held.to(torch.int32))
    first = torch.full((P,), len(i), device="cuda").scatter_reduce_(0, at, torch.where(held, u, len(i)), "amin")
    keep = held & (k[at] >= refs[at]) & (first[at] == u)
    need = ~keep
    rank = torch.cumsum(need, 0) - 1
    order = torch.sort(refs > 0, stable=True).indices
    lack = (need.sum() - (refs <= 0).sum()).clamp(min=0)
    fresh = order[rank.clamp(0, P - 1)]
    now = torch.where(k == 0, refs, torch.where(k >= refs, 1, refs - k))
    now = torch.where((k > 0) & (refs < 1), refs, now)
    now = now.scatter(0, torch.where(need, fresh, at), torch.where(need, 1, now[at]).to(torch.int32))
    new = table.clone()
    new[i, b] = torch.where(need, fresh, page).to(torch.int32)
    fine = lack == 0
    return {"table": torch.where(fine, new, table), "refs": torch.where(fine, now, refs),
            "missing": lack.to(torch.int32).view(1), "k": kr, "v": vr}


def _plain_compact(s):
    table, refs, P = s["table"], s["refs"], s["P"]
    held = refs > 0
    n = held.sum()
    at = torch.arange(P, device="cuda")
    most = P // 2
    src = torch.sort(torch.where(held & (at >= n), at, -1), descending=True).values[:most]
    dst = torch.sort(torch.where(~held & (at < n), at, P)).values[:most]
    dst = torch.where(dst < P, dst, -1)
    m = s["moves"]
    a, b = src[:m], dst[:m]
    to = at.clone()
    to[a] = b
    table = torch.where((table >= 0) & (table < P), to[table.clamp(0, P - 1).long()].to(torch.int32), table)
    new = refs.clone()
    new[b] = refs[a]
    new[a] = 0
    kc, vc, scales, mean = s["cache"][:4]
    for t in (kc, vc, scales, mean):
        t[b] = t[a]
    return {"table": table, "refs": new, "src": src.to(torch.int32), "dst": dst.to(torch.int32),
            "count": (src >= 0).sum().to(torch.int32).view(1), "k": kc, "v": vc, "scales": scales, "mean": mean}


# ---- what an operator cannot do without ------------------------------------------

def work(case):
    c = case
    if c["op"] == "norm":
        n = c["rows"] * max(c["heads"], 1) * c["dim"]
        streams = 1 + 2 * c["add"] + c["pre"] + (c["gate"] == "full")
        small = c["dim"] * (c["post"] + c["pre"]) * (1 + c["centred"]) + {"column": c["dim"], "row": c["rows"]}.get(c["gate"], 0)
        return {"bytes": 4 * (streams * n + small), "flops": n * (4 * c["post"] + 4 * c["pre"] + 3 * c["add"])}
    if c["op"] == "lora":
        ids, ranks, count = _adapters_of(c)
        size = 4 if c["type"] == "fp32" else 2
        with_one = sum(t for a, t in zip(ids, count) if a >= 0)
        return {"bytes": 4 * (with_one * c["k"] + 2 * sum(count) * c["n"])
                + sum(ranks[a] * (c["k"] + c["n"]) * size for a in set(ids) if a >= 0),
                "flops": sum(2 * t * ranks[a] * (c["k"] + c["n"]) for a, t in zip(ids, count) if a >= 0)}
    table, length, refs = _plan(c, 0)
    ints = 8 * (table.size + refs.size)   # each entry and count read and written once
    rows = c["heads"] * c["dim"] * 4
    if c["op"] == "branch":
        return {"bytes": ints + c["forks"] * 2 * 2 * c["block"] * 2 * rows, "flops": table.size}
    held = refs > 0
    moves = int(held[held.sum():].sum())
    block = c["heads"] * (2 * c["block"] * c["dim"] + 8 + 4 * c["dim"])
    return {"bytes": ints + 2 * moves * block, "flops": table.size}


# ---- from the definitions, in 64 bits --------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "lora": _exact_lora, "branch": _exact_branch, "compact": _exact_compact}[case["op"]](s)


def _exact_norm(s):
    c, got = s["case"], {}

    def normed(x, weight, bias):
        mean = x.sum(-1, keepdim=True) / c["dim"] if c["centred"] else 0.0
        square = ((x - mean) ** 2).sum(-1, keepdim=True) / c["dim"]
        y = (x - mean) / torch.sqrt(square + s["eps"]) * weight.double()
        return y + bias.double() if bias is not None else y
    h = s["h"].double()
    if c["add"]:
        u = s["x"].double()
        if c["post"]:
            u = normed(u, s["post"], s["post_bias"])
        h = got["h"] = h + s["scale"] * (u if s["gate"] is None else s["gate"].double() * u)
    if c["pre"]:
        got["out"] = normed(h, s["pre"], s["pre_bias"])
    return got


def _exact_lora(s):
    ids, ranks, count = _adapters_of(s["case"])
    out, t0 = s["y"].double(), 0
    for a, t in zip(ids, count):
        if a >= 0:
            A, B = s["a"][a, :ranks[a]].double(), s["b"][a, :, :ranks[a]].double()
            v = torch.matmul(A, s["x"][t0:t0 + t].double().t().contiguous())
            out[t0:t0 + t] += s["scales"][a].double() * torch.matmul(B, v).t()
        t0 += t
    return out


def _gpu(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _exact_branch(s):
    B, P = s["B"], s["P"]
    table, refs = s["table"].tolist(), s["refs"].tolist()
    kept, after, cu = s["kept"].tolist(), s["after"].tolist(), s["cu"].tolist()
    for row, n in zip(table, kept):
        for b in range(-(-n // B), len(row)):
            if row[b] >= 0:
                refs[row[b]] -= 1
            row[b] = -1
    kr, vr = s["cache"][4].clone(), s["cache"][5].clone()
    for p, c, a, b in zip(s["parents"].tolist(), s["children"].tolist(), s["ring_from"].tolist(), s["ring_to"].tolist()):
        table[c] = list(table[p])
        for page in table[c]:
            if page >= 0:
                refs[page] += 1
        kr[b], vr[b] = kr[a], vr[a]
    # one after another: a block held elsewhere too is left to the others, the last of whom keeps it;
    # of those that are all in this call, the first
    was, here = list(refs), {}
    units = [(i, b) for i in range(len(table)) if cu[i + 1] > cu[i]
             for b in range((after[i] - cu[i + 1] + cu[i]) // B, (after[i] - 1) // B + 1)]
    for i, b in units:
        here.setdefault(table[i][b], []).append((i, b))
    free = [p for p in range(P) if was[p] <= 0]
    take = []
    for i, b in units:
        page = table[i][b]
        if page < 0 or was[page] < 1 or len(here[page]) < was[page] or here[page][0] != (i, b):
            take.append((i, b))
    if len(take) <= len(free):
        for page, who in here.items():
            if page >= 0 and was[page] >= 1:
                refs[page] = 1 if len(who) >= was[page] else was[page] - len(who)
        for (i, b), page in zip(take, free):
            table[i][b], refs[page] = page, 1
    return {"table": _gpu(table), "refs": _gpu(refs), "missing": _gpu([max(0, len(take) - len(free))]), "k": kr, "v": vr}


def _exact_compact(s):
    P, refs = s["P"], s["refs"].tolist()
    table = s["table"].cpu().numpy()
    src, dst = [], []
    lo, hi = 0, P - 1
    while True:
        while lo < P and refs[lo] > 0:
            lo += 1
        while hi >= 0 and refs[hi] <= 0:
            hi -= 1
        if lo >= hi:
            break
        refs[lo], refs[hi] = refs[hi], 0
        src.append(hi)
        dst.append(lo)
    to = np.arange(P)
    to[src] = dst
    pad = [-1] * (P // 2 - len(src))
    kc, vc, scales, mean = (t.clone() for t in s["cache"][:4])
    for t in (kc, vc, scales, mean):
        for a, b in zip(src, dst):
            t[b] = t[a]
    return {"table": _gpu(np.where(table >= 0, to[np.clip(table, 0, None)], -1)), "refs": _gpu(refs),
            "src": _gpu(src + pad), "dst": _gpu(dst + pad), "count": _gpu([len(src)]), "k": kc, "v": vc,
            "scales": scales, "mean": mean}
