"""The calls that keep a paged cache of shared keys and values, attend over it, and add a learned relative position bias.

Every share and every opened masked value is uniform over the ring whatever the plaintext, so the inputs are uniform words.  Where `own`
is false, `run` computes the same words in elementary torch operations on the ring's integers, which wrap as the ring does.

A cached row of K or V is n + 1 words an element: slot 0 is the public F = sum_i (x_i - b_i), slot 1 is b_0 + F, slot 1 + i is b_i.  Pools are
[n + 1][pages][kv heads][tokens a page][dim]; a table [batch][pages a sequence] says which page holds which positions.
"""
import math

import numpy as np
import torch

own = False

F = 16                                     # fractional bits
BUCKETS, REACH = 32, 128                   # of the relative position bias


def listed():
    return [
        # one new token a sequence: what every step of a batch of eight generations appends, latency alone
        dict(name="append_token", kind="append", bits=64, n=3, batch=8, kv=8, dim=128, page=64, rows=1, context=4096),
        # four prompts of up to 2048 tokens enter the cache
        dict(name="append_prompt", kind="append", bits=64, n=2, batch=4, kv=8, dim=128, page=64, rows=2048, context=0),
        # pages copied where a forked sequence is written, or where the pool is compacted
        dict(name="copy_pages", kind="copy", bits=64, n=3, kv=8, dim=128, page=64, pairs=48),
        # the accepted branch of 32 drafted tokens moves to the front, 16 sequences
        dict(name="keep_accepted", kind="compact", bits=64, n=3, batch=16, kv=8, dim=128, page=64, nodes=32, context=1000),
        # scores of a single token over a short cache: the smallest attention call
        dict(name="scores_token", kind="scores", bits=64, n=3, batch=2, heads=8, kv=8, dim=64, page=16, nodes=1, context=700, f=F, bias=False),
        # a tree of eight drafted tokens, four query heads a cached head, with the relative position bias
        dict(name="scores_tree", kind="scores", bits=64, n=3, batch=2, heads=16, kv=4, dim=128, page=64, nodes=8, context=8192, f=F, bias=True),
        # a single token over long caches: the largest call
        dict(name="values_long", kind="values", bits=64, n=3, batch=4, heads=16, kv=8, dim=128, page=64, nodes=1, context=32768, f=F),
        # 32-bit words, heads of 80, an odd number of query rows
        dict(name="values_tree32", kind="values", bits=32, n=2, batch=8, heads=20, kv=4, dim=80, page=16, nodes=7, context=3001, f=12),
        # the bias of one generated token, scores truncated in the same pass
        dict(name="bias_token", kind="bias", bits=64, n=3, batch=4, heads=8, Q=1, K=777, first=776, causal=True, f=F),
        # the scores of a training step of a decoder
        dict(name="bias_causal", kind="bias", bits=64, n=3, batch=2, heads=8, Q=1024, K=1024, first=0, causal=True, f=F),
        # the gradient of the table, 196 tokens of image patches, both directions, 32-bit words
        dict(name="grad_patches", kind="grad", bits=32, n=3, batch=8, heads=4, Q=196, K=196, first=0, causal=False),
        # and of a decoder's training step
        dict(name="grad_causal", kind="grad", bits=64, n=3, batch=4, heads=16, Q=1024, K=1024, first=0, causal=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "copy", "compact", "scores", "scores", "values", "values", "bias", "grad"])
    c = dict(kind=kind, bits=rng.choice([64, 64, 32]), n=rng.randint(2, 5))
    if kind in ("bias", "grad"):
        c.update(batch=rng.randint(1, 8), heads=rng.randint(1, 16), Q=_log(rng, 1, 1500), K=_log(rng, 1, 1500), causal=rng.random() < 0.5)
        c["first"] = max(0, c["K"] - c["Q"]) if rng.random() < 0.5 else 0
        if kind == "bias":
            c["f"] = rng.choice([0, 12, 12, 16])
        while c["n"] * c["batch"] * c["heads"] * c["Q"] * c["K"] > 1.5e8:
            c["Q"], c["K"], c["first"] = c["Q"] // 2 + 1, c["K"] // 2 + 1, c["first"] // 2
        return c
    c.update(kv=rng.choice([1, 2, 4, 8]), dim=rng.choice([16, 32, 64, 64, 80, 128, 128, 256]), page=rng.choice([16, 32, 64, 128]))
    if kind == "copy":
        c["pairs"] = _log(rng, 1, 64)
    elif kind == "append":
        c.update(batch=rng.randint(1, 16), rows=_log(rng, 1, 1024), context=_log(rng, 1, 2000) - 1)
    else:
        c.update(batch=rng.randint(1, 8), nodes=rng.choice([1, 1, 2, 5, 8, 16, 33]), context=_log(rng, 1, 16384) - 1)
        if kind != "compact":
            c.update(heads=c["kv"] * rng.choice([1, 1, 2, 4, 5]), f=rng.choice([0, 12, 12, 16]))
            if kind == "scores":
                c["bias"] = rng.random() < 0.5
            while c["n"] * c["batch"] * c["heads"] * c["nodes"] * (c["context"] + c["nodes"]) * c["dim"] > 1e9:
                c["context"], c["batch"], c["nodes"] = c["context"] // 2, (c["batch"] + 1) // 2, (c["nodes"] + 1) // 2
    return c


# ---- inputs --------------------------------------------------------------------------------------------------
def _contexts(c):
    """Tokens in the cache before the new ones, a sequence each: the longest, then ragged ones, the last of four or more idle at zero."""
    b, most = c["batch"], c["context"]
    got = [most] + [most * (13 + 7 * (i % 5)) // 48 for i in range(1, b)]
    return got[:-1] + [0] if b >= 4 else got


def _counts(c):
    """New rows a sequence of an append."""
    return [c["rows"]] + [max(1, c["rows"] * (29 + 5 * (i % 4)) // 48) for i in range(1, c["batch"])]


def _lengths(c):
    return [c["K"]] + [max(1, c["K"] * (31 + 5 * (i % 4)) // 48) for i in range(1, c["batch"])]


def _pages(c):
    """Pages of a sequence, and of the pool, some of which hold nothing."""
    if c["kind"] == "copy":
        return 0, 2 * c["pairs"] + 3
    each = -(-(c["context"] + c.get("rows", c.get("nodes"))) // c["page"])
    return each, each * c["batch"] + 3


def _bucket_of(both):
    """Bucket of a distance key - query, from -REACH to REACH: the near ones have one each, the far ones share logarithmic ranges whose
    borders are compared in whole numbers.  both: half of the buckets are for keys behind the query; otherwise those have bucket 0."""
    half = BUCKETS // 2 if both else BUCKETS
    near = half // 2
    wide = half - near

    def of(d):
        m = max(d, 0)
        return m if m < near else near + max(j for j in range(wide) if m ** wide * near ** j >= REACH ** j * near ** wide)
    return [(half + of(d) if both and d > 0 else of(abs(d)) if both else of(-d)) for d in range(-REACH, REACH + 1)]


def prepare(case, seed):
    c, n = case, case["n"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    host = np.random.RandomState(seed % (1 << 31))
    word = torch.int32 if c["bits"] == 32 else torch.int64
    low, high = -2 ** (c["bits"] - 1), 2 ** (c["bits"] - 1) - 1

    def u(*shape):
        return torch.empty(shape, dtype=word, device="cuda").random_(low, high, generator=g)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")
    s = {"case": c, "masked": -(1 << (c["bits"] - 4))}
    if c["kind"] in ("bias", "grad"):
        b, h, q, k = c["batch"], c["heads"], c["Q"], c["K"]
        s.update(x=u(n, b, h, q, k), bucket_of=ints(_bucket_of(not c["causal"])), lengths=ints(_lengths(c)))
        if c["kind"] == "bias":
            s.update(table=u(n, h, BUCKETS), tuple=[u(n, b, h, q, k) for _ in range(3)] if c["f"] else None)
        return s
    each, pages = _pages(c)
    pool = (n + 1, pages, c["kv"], c["page"], c["dim"])
    order = host.permutation(pages)
    if c["kind"] == "copy":
        s.update(pools=(u(*pool), u(*pool)), src=ints(order[:c["pairs"]]), dst=ints(order[c["pairs"]:2 * c["pairs"]]))
        return s
    s.update(context=ints(_contexts(c)), table=ints(order[:c["batch"] * each].reshape(c["batch"], each)))
    if c["kind"] == "append":
        rows = (n, c["batch"], c["kv"], c["rows"], c["dim"])
        s.update(pools=(u(*pool), u(*pool)), x=(u(*rows), u(*rows)), b=(u(*rows), u(*rows)), count=ints(_counts(c)))
        return s
    # a random tree: every node but a root descends from an earlier one, and sees its ancestors and itself
    m = c["nodes"]
    parent = [[int(host.randint(-1, j)) for j in range(m)] for _ in range(c["batch"])]
    sees, deep = [], []
    for p in parent:
        bits, depth = [], []
        for j in range(m):
            bits.append((bits[p[j]] if p[j] >= 0 else 0) | 1 << j)
            depth.append(depth[p[j]] + 1 if p[j] >= 0 else 0)
        sees.append(bits)
        deep.append(depth)
    if c["kind"] == "compact":
        kept = [[j for j in range(m) if bits[last] >> j & 1] for bits, last in zip(sees, host.randint(0, m, c["batch"]))]
        s.update(pools=(u(*pool), u(*pool)), kept=ints([k + [0] * (m - len(k)) for k in kept]), kept_count=ints([len(k) for k in kept]))
        return s
    if c["batch"] >= 4:
        sees[-1][0] = 0                    # an idle slot of the batch: a row that sees nothing at all
    s["tree"] = torch.tensor(sees, dtype=torch.int64, device="cuda")
    rows, columns = (n, c["batch"], c["heads"], m), c["context"] + m
    shape = rows + (columns if c["kind"] == "scores" else c["dim"],)
    s.update(pool=u(*pool), C=u(*shape), tuple=[u(*shape) for _ in range(3)] if c["f"] else None)
    s.update(zip(("x", "A"), (u(*rows, c["dim"] if c["kind"] == "scores" else columns) for _ in range(2))))
    if c["kind"] == "scores" and c["bias"]:
        s.update(bias=u(n, c["heads"], BUCKETS), bucket_of=ints(_bucket_of(False)), depth=ints(deep))
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------
def _trunc(y, tup, f, bits):
    """Signed probabilistic truncation of the shares y by f bits."""
    r, top, msb = tup
    c = (y + r).sum(0, dtype=y.dtype) + (1 << (bits - 2))
    c_msb = (c >> (bits - 1)) & 1
    out = ((msb - 2 * c_msb * msb) << (bits - 1 - f)) - top
    out[0] += (c_msb << (bits - 1 - f)) + ((c >> f) & ((1 << (bits - 1 - f)) - 1)) - (1 << (bits - 2 - f))
    return out


def _rows_of(pool, table, columns):
    """[slots][batch][kv heads][columns][dim] of a paged pool."""
    got = pool[:, table.long()].transpose(2, 3)
    return got.reshape(got.shape[:3] + (-1, got.shape[-1]))[:, :, :, :columns]


def _visible(s, columns):
    """[batch][nodes][columns]: the context, and what the tree says of the drafted tokens behind it."""
    at = torch.arange(columns, device="cuda") - s["context"][:, None, None]
    m = s["case"]["nodes"]
    return (at < 0) | ((at < m) & ((s["tree"][:, :, None] >> at.clamp(0, m - 1)) & 1 > 0))


def _attend(s):
    c, n = s["case"], s["case"]["n"]
    m, g, columns = c["nodes"], c["kv"], c["context"] + c["nodes"]
    cached = _rows_of(s["pool"], s["table"], columns)
    seen = _visible(s, columns)[:, None]
    word = s["pool"].dtype
    x, A = s["x"], s["A"]
    if c["kind"] == "values":
        x, A = x * seen, A * seen
    by_kv = (n, c["batch"], g, c["heads"] // g * m, x.shape[-1])
    A = A.reshape(by_kv)
    E = x.reshape(by_kv).sum(0, dtype=word) - A.sum(0, dtype=word)
    if c["kind"] == "scores":
        z = (E[..., None, :] * cached[1:, :, :, None]).sum(-1, dtype=word) + (A[..., None, :] * cached[0][:, :, None]).sum(-1, dtype=word)
    else:
        z = (E[..., None] * cached[1:, :, :, None]).sum(-2, dtype=word) + (A[..., None] * cached[0][:, :, None]).sum(-2, dtype=word)
    z = s["C"] + z.reshape(s["C"].shape)
    if c["f"]:
        z = _trunc(z, s["tuple"], c["f"], c["bits"])
    if c["kind"] == "values":
        return z
    if c["bias"]:
        at = torch.arange(columns, device="cuda") - s["context"][:, None]
        key = torch.where(at < 0, at, s["depth"].long().gather(1, at.clamp(0, m - 1)))
        away = (key[:, None] - s["depth"][:, :, None]).clamp(-REACH, REACH) + REACH
        z = z + s["bias"][:, :, s["bucket_of"][away].long()].transpose(1, 2)
    z = torch.where(seen, z, 0)
    z[0] += torch.where(seen, 0, s["masked"]).to(word)
    return z


def _pairs(s):
    """[batch][1][Q][K]: which scores are there."""
    c = s["case"]
    k = torch.arange(c["K"], device="cuda")
    seen = k < s["lengths"][:, None, None, None]
    return seen & (k <= torch.arange(c["Q"], device="cuda")[:, None] + c["first"]) if c["causal"] else seen.expand(-1, 1, c["Q"], -1)


def _bias(s):
    c = s["case"]
    y = _trunc(s["x"], s["tuple"], c["f"], c["bits"]) if c["f"] else s["x"]
    away = torch.arange(c["K"], device="cuda") - torch.arange(c["Q"], device="cuda")[:, None] - c["first"]
    y = y + s["table"][:, :, s["bucket_of"][away.clamp(-REACH, REACH) + REACH].long()][:, None]
    seen = _pairs(s)
    y = torch.where(seen, y, 0)
    y[0] += torch.where(seen, 0, s["masked"]).to(y.dtype)
    return y


def _grad(s):
    """Sums along the diagonals first (every row pushed right by its own number of places), then over the distances of a bucket."""
    c, x = s["case"], s["x"]
    x = torch.where(_pairs(s), x, 0).sum(1, dtype=x.dtype).flip(-2)
    n, h, q, k = x.shape
    x = torch.nn.functional.pad(x, (0, q)).reshape(n, h, -1)[..., :q * (q + k - 1)].reshape(n, h, q, q + k - 1).sum(-2, dtype=x.dtype)
    away = torch.arange(q + k - 1, device="cuda") - (q - 1) - c["first"]
    return torch.zeros(n, h, BUCKETS, dtype=x.dtype, device="cuda").index_add_(2, s["bucket_of"][away.clamp(-REACH, REACH) + REACH].long(), x)


def _append(s):
    c = s["case"]
    at = torch.arange(c["rows"], device="cuda")
    b, r = (at < s["count"][:, None]).nonzero(as_tuple=True)
    to = r + s["context"][b].long()
    page, place = s["table"][b, to // c["page"]].long(), to % c["page"]

    def into(pool, x, mask):
        opened = x.sum(0, dtype=x.dtype) - mask.sum(0, dtype=x.dtype)
        slots = torch.cat([opened[None], mask])
        slots[1] += opened
        pool[:, page, :, place] = slots[:, b, :, r]
        return pool
    return into(s["pools"][0], s["x"][0], s["b"][0]), into(s["pools"][1], s["x"][1], s["b"][1])


def _copy(s):
    def one(pool):
        pool[:, s["dst"].long()] = pool[:, s["src"].long()]
        return pool
    return one(s["pools"][0]), one(s["pools"][1])


def _compact(s):
    c = s["case"]
    b, j = (torch.arange(c["nodes"], device="cuda") < s["kept_count"][:, None]).nonzero(as_tuple=True)
    old, new = s["context"][b].long() + s["kept"][b, j], s["context"][b].long() + j
    t = c["page"]

    def one(pool):
        pool[:, s["table"][b, new // t].long(), :, new % t] = pool[:, s["table"][b, old // t].long(), :, old % t]
        return pool
    return one(s["pools"][0]), one(s["pools"][1])


def run(s):
    c = s["case"]
    kind = c["kind"]
    if not own:
        return {"append": _append, "copy": _copy, "compact": _compact, "scores": _attend, "values": _attend, "bias": _bias, "grad": _grad}[kind](s)
    from paper_2402_02320_amd import spin
    ring = spin.ring32 if c["bits"] == 32 else spin
    if kind == "append":
        return ring.cache_append(s["pools"], s["table"], s["context"], s["x"], s["b"], count=s["count"])
    if kind == "copy":
        return ring.cache_copy(s["pools"], s["src"], s["dst"])
    if kind == "compact":
        return ring.cache_compact(s["pools"], s["table"], s["context"], s["kept"], s["kept_count"])
    if kind == "scores":
        bias = (s["bias"], s["bucket_of"]) if c["bias"] else None
        return ring.cache_scores(s["pool"], s["table"], s["context"], s["x"], s["A"], s["C"], f=c["f"], tuple_=s["tuple"], tree=s["tree"],
                                 masked=s["masked"], bias=bias, depth=s.get("depth"))
    if kind == "values":
        return ring.cache_values(s["pool"], s["table"], s["context"], s["x"], s["A"], s["C"], f=c["f"], tuple_=s["tuple"], tree=s["tree"])
    if kind == "bias":
        return ring.relbias_trunc(s["x"], s["table"], s["bucket_of"], f=c["f"], tuple_=s["tuple"], first=c["first"], causal=c["causal"],
                                  lengths=s["lengths"], masked=s["masked"])
    return ring.relbias_grad(s["x"], s["bucket_of"], BUCKETS, first=c["first"], causal=c["causal"], lengths=s["lengths"])


def work(case):
    """bytes: every word that a result depends on read once, every returned word written once (of a pool, the rows that change).  flops: two
    per ring multiply-add, of which a party has two a query element and cached row; elsewhere two per word that is added."""
    c, n, w = case, case["n"], case["bits"] // 8
    if c["kind"] in ("bias", "grad"):
        seen = c["heads"] * sum(sum(min(k, q + c["first"] + 1) if c["causal"] else k for q in range(c["Q"])) for k in _lengths(c))
        every = c["heads"] * c["batch"] * c["Q"] * c["K"]
        if c["kind"] == "grad":
            return {"bytes": w * n * (seen + c["heads"] * BUCKETS), "flops": 2.0 * n * seen}
        return {"bytes": w * n * ((4 if c["f"] else 1) * seen + every + c["heads"] * BUCKETS), "flops": 2.0 * n * seen}
    row = c["kv"] * c["dim"] * w
    if c["kind"] == "copy":
        return {"bytes": 4 * (n + 1) * c["pairs"] * c["page"] * row, "flops": 0}
    if c["kind"] == "compact":
        # a path of a random tree of m nodes has about log(m) + 1 of them, the first of which often stays
        return {"bytes": 4 * (n + 1) * c["batch"] * (math.log(c["nodes"]) + 0.5) * row, "flops": 0}
    if c["kind"] == "append":
        return {"bytes": 2 * (3 * n + 1) * sum(_counts(c)) * row, "flops": 2.0 * 2 * 2 * n * sum(_counts(c)) * row / w}
    m, columns = c["nodes"], c["context"] + c["nodes"]
    seen = sum(k + m for k in _contexts(c))
    rows = c["batch"] * c["heads"] * m
    scores, vectors = c["heads"] * m * seen, rows * c["dim"]
    if c["kind"] == "scores":
        words = n * (2 * vectors + (4 if c["f"] else 1) * scores + rows * columns)
    else:
        words = n * (2 * scores + (5 if c["f"] else 2) * vectors)
    return {"bytes": (n + 1) * seen * row + w * words, "flops": 4.0 * n * scores * c["dim"]}


# ---- the definition, word by word on the host -----------------------------------------------------------------
def exact(case, seed):
    c, n = case, case["n"]
    work_of = work(c)
    if work_of["flops"] > 2e9 or work_of["bytes"] > 5e8:
        return None                        # minutes on the host
    unsigned = np.uint32 if c["bits"] == 32 else np.uint64
    signed = np.int32 if c["bits"] == 32 else np.int64
    s = prepare(case, seed)

    def words(t):
        return t.cpu().numpy().view(unsigned)

    def truncated(y, tup, f):
        if not f:
            return y
        top = c["bits"] - 1
        r, r_top, r_msb = (words(t) for t in tup)
        opened = y[0] * unsigned(0) + unsigned(1 << (top - 1))
        for i in range(n):
            opened = opened + y[i] + r[i]
        carry = opened >> unsigned(top)
        out = np.empty_like(y)
        for i in range(n):
            flipped = np.where(carry == 1, unsigned(0) - r_msb[i], r_msb[i]) + (carry if i == 0 else unsigned(0))
            out[i] = flipped * unsigned(1 << (top - f)) - r_top[i]
        out[0] += (opened % unsigned(1 << top)) // unsigned(1 << f) - unsigned(1 << (top - 1 - f))
        return out
    if c["kind"] in ("append", "copy", "compact"):
        pools = [words(p).copy() for p in s["pools"]]
        for k, p in enumerate(pools):
            if c["kind"] == "copy":
                for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
                    p[:, b] = p[:, a]
                continue
            table, start = s["table"].tolist(), s["context"].tolist()
            old = p.copy()
            for b in range(c["batch"]):
                moves = range(s["count"].tolist()[b]) if c["kind"] == "append" else s["kept"].tolist()[b][:s["kept_count"].tolist()[b]]
                for j, row in enumerate(moves):
                    to = start[b] + j
                    dst = p[:, table[b][to // c["page"]], :, to % c["page"]]
                    if c["kind"] == "compact":
                        at = start[b] + row
                        dst[:] = old[:, table[b][at // c["page"]], :, at % c["page"]]
                    else:
                        x, mask = (words(t[k][:, b, :, row]) for t in (s["x"], s["b"]))
                        opened = (x - mask).sum(0, dtype=unsigned)
                        dst[:] = np.concatenate([opened[None], mask])
                        dst[1] += opened
        return tuple(p.view(signed) for p in pools)
    masked = unsigned(s["masked"] % (1 << c["bits"]))
    if c["kind"] in ("bias", "grad"):
        x, lut, lengths = words(s["x"]), s["bucket_of"].tolist(), s["lengths"].tolist()
        away = np.arange(c["K"]) - np.arange(c["Q"])[:, None] - c["first"]
        bucket = np.array(lut)[np.clip(away, -REACH, REACH) + REACH]
        seen = np.stack([np.broadcast_to(np.arange(c["K"]) < k, away.shape) & ((away <= 0) | (not c["causal"])) for k in lengths])
        if c["kind"] == "grad":
            out = np.zeros((n, c["heads"], BUCKETS), unsigned)
            for b in range(c["batch"]):
                for k in range(BUCKETS):
                    out[:, :, k] += (x[:, b] * (seen[b] & (bucket == k)).astype(unsigned)).sum((-1, -2), dtype=unsigned)
            return out.view(signed)
        y, table = truncated(x, s["tuple"], c["f"]), words(s["table"])
        for i in range(n):
            for h in range(c["heads"]):
                y[i, :, h] = np.where(seen, y[i, :, h] + table[i, h][bucket], masked if i == 0 else unsigned(0))
        return y.view(signed)
    pool, table, context, tree = words(s["pool"]), s["table"].tolist(), s["context"].tolist(), s["tree"].tolist()
    x, A, out = words(s["x"]), words(s["A"]), words(s["C"]).copy()
    m, columns, share = c["nodes"], c["context"] + c["nodes"], c["heads"] // c["kv"]
    seen = np.zeros((c["batch"], m, columns), bool)
    for b in range(c["batch"]):
        for j in range(m):
            seen[b, j, :context[b]] = True
            for k in range(m):
                seen[b, j, context[b] + k] = tree[b][j] >> k & 1
        for h in range(c["heads"]):
            cached = np.concatenate([pool[:, p, h // share] for p in table[b]], axis=1)[:, :columns]
            e = (x[:, b, h] - A[:, b, h]).sum(0, dtype=unsigned)
            for i in range(n):
                for j in range(m):
                    a = A[i, b, h, j]
                    if c["kind"] == "scores":
                        out[i, b, h, j] += (cached[1 + i] * e[j]).sum(-1, dtype=unsigned) + (cached[0] * a).sum(-1, dtype=unsigned)
                    else:
                        k = seen[b, j]
                        out[i, b, h, j] += (cached[1 + i][k] * e[j][k][:, None]).sum(0, dtype=unsigned) + (cached[0][k] * a[k][:, None]).sum(0, dtype=unsigned)
    out = truncated(out, s["tuple"], c["f"])
    if c["kind"] == "scores":
        for b in range(c["batch"]):
            place = s["depth"].tolist()[b] if c["bias"] else [0] * m
            for j in range(m):
                key = np.concatenate([np.arange(context[b]), context[b] + np.array(place), np.zeros(columns - context[b] - m, int)]).astype(int)
                if c["bias"]:
                    bucket = np.array(s["bucket_of"].tolist())[np.clip(key - context[b] - place[j], -REACH, REACH) + REACH]
                    out[:, b, :, j] += words(s["bias"])[:, :, bucket]
                out[:, b, :, j] = np.where(seen[b, j], out[:, b, :, j], unsigned(0))
                out[0, b, :, j] = np.where(seen[b, j], out[0, b, :, j], masked)
    return out.view(signed)
