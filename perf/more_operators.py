"""The calls of a transformer block without softmax on shares: linear attention with a decay for each head, and layer norm, forward and backward.

Every share and every opened masked value is uniform over the ring whatever the plaintext, so the inputs are uniform words.  Where `own`
is false, `run` computes the same words in elementary torch operations on the ring's integers, which wrap as the ring does.

A secret x is opened as E = sum_i (x_i - a_i) against its mask a; a product of two opened secrets is a_i . F + E . b_i (+ E . F, party 0) beside the dealt
share c_i of the masks' product.  T(y, f) is the truncation of y by f bits with its tuple (r, r_top, r_msb).
"""
import math

import numpy as np
import torch

own = False

ROW_WORDS, GRAD_ROW_WORDS = 15, 22         # dealt words a row of the norm: a Newton step's (and as many besides), and the gradient's


def listed():
    return [
        # one generated token of two sequences: the smallest call, latency alone
        dict(name="step_token", kind="step", bits=64, n=3, batch=2, heads=8, dk=64, dv=64, f=16, g=12, idle=False),
        # a token of each of 32 sequences: the states go through the chip once
        dict(name="step_batch", kind="step", bits=64, n=3, batch=32, heads=16, dk=128, dv=128, f=16, g=12, idle=True),
        # 32-bit words, keys and values of different odd widths, idle sequences
        dict(name="step_odd32", kind="step", bits=32, n=2, batch=9, heads=5, dk=40, dv=72, f=9, g=6, idle=True),
        # a short prompt: a few chunks, the last of them cut
        dict(name="prompt_short", kind="prompt", bits=64, n=3, batch=1, heads=8, tokens=300, dk=64, dv=64, chunk=64, f=16, g=12),
        # long prompts: the largest call
        dict(name="prompt_long", kind="prompt", bits=64, n=3, batch=2, heads=16, tokens=4096, dk=128, dv=128, chunk=128, f=16, g=12),
        # ragged prompts of 32-bit words, short chunks
        dict(name="prompt_ragged32", kind="prompt", bits=32, n=2, batch=4, heads=6, tokens=777, dk=80, dv=48, chunk=32, f=9, g=6),
        # forward and backward of a training step
        dict(name="train", kind="train", bits=64, n=2, batch=2, heads=8, tokens=1024, dk=64, dv=64, chunk=64, f=16, g=12),
        # the norm before one generated token of two sequences
        dict(name="norm_token", kind="norm", bits=64, n=3, rows=2, dim=1024, f=16, shift=26, iterations=6),
        # a prompt's tokens
        dict(name="norm_rows", kind="norm", bits=64, n=3, rows=4096, dim=1024, f=16, shift=26, iterations=6),
        # odd sizes, 32-bit words
        dict(name="norm_odd32", kind="norm", bits=32, n=2, rows=1001, dim=333, f=9, shift=15, iterations=5),
        # the gradient of a training step, wide rows
        dict(name="norm_grad", kind="norm_grad", bits=64, n=3, rows=2048, dim=2048, f=16, shift=27),
        # five parties, eight images of 196 patches
        dict(name="norm_grad_patches", kind="norm_grad", bits=64, n=5, rows=1568, dim=256, f=16, shift=24),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "prompt", "prompt", "train", "norm", "norm", "norm_grad"])
    bits = rng.choice([64, 64, 32])
    c = dict(kind=kind, bits=bits, n=rng.randint(2, 5), f=16 if bits == 64 else 9)
    if kind in ("norm", "norm_grad"):
        c.update(rows=_log(rng, 1, 6000), dim=_log(rng, 8, 4096))
        c["shift"] = c["f"] + 10 if bits == 64 else 15
        if kind == "norm":
            c["iterations"] = rng.randint(3, 9)
        while c["n"] * c["rows"] * c["dim"] > 1.2e7:
            c["rows"] = c["rows"] // 2 + 1
        return c
    c.update(batch=rng.randint(1, 8), heads=rng.randint(1, 16), dk=rng.choice([16, 32, 40, 64, 64, 80, 128, 128, 256]),
             dv=rng.choice([16, 32, 64, 64, 72, 96, 128, 128, 256]), g=rng.choice([0, 6, 6]) if bits == 32 else rng.choice([0, 12, 12]))
    if kind == "step":
        c["idle"] = rng.random() < 0.5
        return c
    c.update(tokens=_log(rng, 1, 3000), chunk=rng.choice([32, 64, 128]))
    most = 2e8 if kind == "prompt" else 4e7
    while c["n"] * c["batch"] * c["heads"] * c["tokens"] * max(c["chunk"] + c["dk"], c["dk"] * c["dv"] // c["chunk"]) > most:
        c["tokens"], c["batch"] = c["tokens"] // 2 + 1, (c["batch"] + 1) // 2
    return c


# ---- inputs --------------------------------------------------------------------------------------------------
def _lengths(c):
    """Tokens of every sequence: the first has all, the others are ragged; of four or more the last has none."""
    got = [c["tokens"]] + [max(1, c["tokens"] * (23 + 9 * (i % 3)) // 48) for i in range(1, c["batch"])]
    return got[:-1] + [0] if c["batch"] >= 4 else got


def _chunks(c):
    return -(-c["tokens"] // c["chunk"])


def _decay(c, most):
    """w[head][j] = round(lambda^j 2^g), lambda = 1 - 2^-(3 + 5 head / heads); without fractional bits there is no decay."""
    if c["g"] == 0:
        return None
    return [[int(round((1 - 2.0 ** -(3 + 5 * h / c["heads"])) ** j * 2 ** c["g"])) for j in range(most + 1)] for h in range(c["heads"])]


def prepare(case, seed):
    c, n = case, case["n"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    word = torch.int32 if c["bits"] == 32 else torch.int64
    low, high = -2 ** (c["bits"] - 1), 2 ** (c["bits"] - 1) - 1

    def u(*shape):
        return torch.empty((n,) + shape, dtype=word, device="cuda").random_(low, high, generator=g)

    def masked(*shape):
        return u(*shape), u(*shape)

    def tup(*shape):
        return [u(*shape) for _ in range(3)]
    s = {"case": c}
    if c["kind"] in ("norm", "norm_grad"):
        r, d = c["rows"], c["dim"]
        s.update(gamma=masked(d), c=(u(r, d), u(r, d)), tuples=(tup(r, d), tup(r, d)))
        if c["kind"] == "norm":
            s.update(x=u(r, d), beta=u(d), masks=(u(r, d), u(r, d)), row_words=u(ROW_WORDS * (c["iterations"] + 1), r))
        else:
            s.update(dy=u(r, d), xhat=u(r, d), rstd=u(r), masks=(u(r, d), u(r, d), u(r, d)), column_words=u(4, d), row_words=u(GRAD_ROW_WORDS, r))
        return s
    b, h, dk, dv = c["batch"], c["heads"], c["dk"], c["dv"]
    w = _decay(c, 1 if c["kind"] == "step" else c["chunk"])
    s["decay"] = None if w is None else torch.tensor(w, dtype=word, device="cuda")
    state = (b, h, dk, dv)
    if c["kind"] == "step":
        s.update(S=u(*state), q=masked(b, h, dk), k=masked(b, h, dk), v=masked(b, h, dv), mask=u(*state), c=(u(*state), u(b, h, dv)),
                 tuples=(tup(*state), tup(b, h, dv)), active=torch.tensor([0 if c["idle"] and i % 4 == 3 else 1 for i in range(b)], dtype=torch.int32, device="cuda"))
        return s
    nc, C, t = _chunks(c), c["chunk"], c["tokens"]
    keys, values, pairs, states = (b, h, t, dk), (b, h, t, dv), (b, h, nc, C, C), (b, h, nc, dk, dv)
    s.update(lengths=torch.tensor(_lengths(c), dtype=torch.int32, device="cuda"), q=masked(*keys), k=masked(*keys), v=masked(*values), first=u(*state),
             AP=u(*pairs), AS=u(*states), cP=u(*pairs), cS=u(*states), cO=u(*values), tP=tup(*pairs), tS=tup(*states), tO=tup(*values))
    if c["kind"] == "train":
        s.update(dO=masked(*values), dlast=u(*state), AdP=u(*pairs), AdS=u(*states), cdP=u(*pairs), cdS=u(*states), cdQ=u(*keys), cdK=u(*keys),
                 cdV=u(*values), tdP=tup(*pairs), tdS=tup(*states), tdQ=tup(*keys), tdK=tup(*keys), tdV=tup(*values))
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


def _open(x, a):
    return x.sum(0, dtype=x.dtype) - a.sum(0, dtype=x.dtype)


def _mm(x, y):
    """x . y over the last two axes, a few k at a time."""
    out = None
    at_once = max(1, (1 << 27) // max(1, x[..., 0].numel() * y.shape[-1]))
    for k in range(0, x.shape[-1], at_once):
        part = (x[..., :, k:k + at_once, None] * y[..., None, k:k + at_once, :]).sum(-2, dtype=x.dtype)
        out = part if out is None else out.add_(part)
    return out


def _beaver(x, a, y, b):
    """Every party's part of x . y behind the dealt c."""
    e, f = _open(x, a), _open(y, b)
    z = torch.stack([_mm(a[i], f) + _mm(e, b[i]) for i in range(len(a))])
    z[0] += _mm(e, f)
    return z


def _mul(e, a, f, b):
    """The same, elementwise, of opened factors."""
    z = a * f + e * b
    z[0] += e * f
    return z


def _chunked(x, c):
    """[.., tokens, d] -> [.., chunks, chunk, d]"""
    x = torch.nn.functional.pad(x, (0, 0, 0, _chunks(c) * c["chunk"] - x.shape[-2]))
    return x.reshape(x.shape[:-2] + (_chunks(c), c["chunk"], x.shape[-1]))


class _Chunks:
    """Weights and masks of the chunked form."""

    def __init__(self, s):
        c = self.c = s["case"]
        C = c["chunk"]
        i = torch.arange(C, device="cuda")
        self.len = (s["lengths"].long()[:, None] - C * torch.arange(_chunks(c), device="cuda")).clamp(0, C)           # [batch, chunks]
        w = torch.ones(c["heads"], C + 1, dtype=s["AP"].dtype, device="cuda") if s["decay"] is None else s["decay"]
        self.rows = i < self.len[:, None, :, None]                                                # [batch, 1, chunks, C]
        self.pairs = (i[None, :] <= i[:, None]) & self.rows[..., None]                            # j <= i < len
        self.near = w[:, (i[:, None] - i[None, :]).clamp(min=0)][None, :, None]                   # w[i - j]
        at = (self.len[:, :, None] - 1 - i).clamp(min=0)                                          # [batch, chunks, C]
        self.to_end = w[:, at].transpose(0, 1)                                                    # w[len - 1 - i]: [batch, heads, chunks, C]
        self.from_start = w[:, i + 1][None, :, None].expand_as(self.to_end)                       # w[i + 1]
        self.whole = w[:, self.len].transpose(0, 1)                                               # w[len]: [batch, heads, chunks]

    def scores(self, x, y, C, t):
        c = self.c
        X, A, Y, B = (_chunked(v, c) for v in x + y)
        z = C + self.near * _beaver(X, A, Y.transpose(-1, -2), B.transpose(-1, -2))
        return torch.where(self.pairs, _trunc(z, t, c["f"] + c["g"], c["bits"]), 0)

    def states(self, x, y, C, t, first, reverse=False):
        c = self.c
        w = torch.where(self.rows, self.from_start if reverse else self.to_end, 0)[..., None]
        X, A = (w * _chunked(v, c) for v in x)             # rows that are not there weigh nothing
        Y, B = (_chunked(v, c) for v in y)
        z = _beaver(X.transpose(-1, -2), A.transpose(-1, -2), Y, B)
        z += C
        before, now = torch.empty_like(C), first
        for k in reversed(range(_chunks(c))) if reverse else range(_chunks(c)):
            before[:, :, :, k] = now
            new = _trunc(z[:, :, :, k] + (self.whole[:, :, k] << c["f"])[..., None, None] * now, [v[:, :, :, k] for v in t], c["f"] + c["g"], c["bits"])
            now = torch.where((self.len[:, k] > 0)[:, None, None, None], new, now)
        return before, now

    def outputs(self, p, y, x, s, C, t, reverse=False, transposed=False):
        c = self.c
        P, AP = (torch.where(self.pairs, v, 0) for v in p)
        S, AS = s
        if reverse:
            P, AP = P.transpose(-1, -2), AP.transpose(-1, -2)
        if transposed:
            S, AS = S.transpose(-1, -2), AS.transpose(-1, -2)
        Y, B = (torch.where(self.rows[..., None], _chunked(v, c), 0) for v in y)
        w = torch.where(self.rows, self.to_end if reverse else self.from_start, 0)[..., None]
        X, A = (_chunked(v, c) for v in x)
        z = (_beaver(P, AP, Y, B) << c["g"]) + w * _beaver(X, A, S, AS)
        z = z.flatten(3, 4)[:, :, :, :c["tokens"]] + C
        rows = self.rows.flatten(2, 3)[:, :, :c["tokens"], None]
        return torch.where(rows, _trunc(z, t, c["f"] + c["g"], c["bits"]), 0)


class _Calls:
    """The framework's, of the same arguments."""

    def __init__(self, s, ring):
        self.ring = ring
        self.more = dict(decay=s["decay"], g=s["case"]["g"], lengths=s["lengths"])
        self.chunk, self.f = s["case"]["chunk"], s["case"]["f"]

    def scores(self, x, y, C, t):
        return self.ring.linattn_scores(x, y, C, t, self.f, **self.more)

    def states(self, x, y, C, t, first, reverse=False):
        return self.ring.linattn_states(x, y, C, t, self.f, self.chunk, first=first, reverse=reverse, **self.more)

    def outputs(self, p, y, x, s, C, t, reverse=False, transposed=False):
        return self.ring.linattn_outputs(p, y, x, s, C, t, self.f, reverse=reverse, transposed=transposed, **self.more)


def _attend(s, calls):
    P = calls.scores(s["q"], s["k"], s["cP"], s["tP"])
    S, last = calls.states(s["k"], s["v"], s["cS"], s["tS"], s["first"])
    O = calls.outputs((P, s["AP"]), s["v"], s["q"], (S, s["AS"]), s["cO"], s["tO"])
    if s["case"]["kind"] == "prompt":
        return O, last
    dP = calls.scores(s["dO"], s["v"], s["cdP"], s["tdP"])
    dS, dfirst = calls.states(s["q"], s["dO"], s["cdS"], s["tdS"], s["dlast"], reverse=True)
    dp, S, dS = (dP, s["AdP"]), (S, s["AS"]), (dS, s["AdS"])
    dQ = calls.outputs(dp, s["k"], s["dO"], S, s["cdQ"], s["tdQ"], transposed=True)
    dK = calls.outputs(dp, s["q"], s["v"], dS, s["cdK"], s["tdK"], reverse=True, transposed=True)
    dV = calls.outputs((P, s["AP"]), s["dO"], s["k"], dS, s["cdV"], s["tdV"], reverse=True)
    return O, last, dQ, dK, dV, dfirst


def _step(s):
    c = s["case"]
    w0, w1 = (1, 1) if s["decay"] is None else (s["decay"][:, j, None, None] for j in range(2))
    (k, ak), (v, av), (q, aq) = s["k"], s["v"], s["q"]
    z = s["c"][0] + w0 * _mul(_open(k, ak)[..., None], ak[..., None], _open(v, av)[..., None, :], av[..., None, :]) + (w1 << c["f"]) * s["S"]
    live = (s["active"] > 0)[:, None, None]
    S = torch.where(live[..., None], _trunc(z, s["tuples"][0], c["f"] + c["g"], c["bits"]), s["S"])
    o = s["c"][1] + _mul(_open(q, aq)[..., None], aq[..., None], _open(S, s["mask"]), s["mask"]).sum(-2, dtype=S.dtype)
    return torch.where(live, _trunc(o, s["tuples"][1], c["f"], c["bits"]), 0), S


def _inverse(c):
    return ((1 << c["shift"]) + c["dim"] // 2) // c["dim"]


def _line(f):
    """offset and slope of the first guess at 1 / sqrt(v), and eps."""
    return 3 << (f - 1), 1 << (f - 2), 1


def _norm(s):
    c, f = s["case"], s["case"]["f"]
    bits, inv, (offset, slope, eps) = c["bits"], _inverse(c), _line(f)
    w = s["row_words"]
    a1, a2 = s["masks"]

    def public(x, v):
        x = x.clone()
        x[0] += v
        return x

    def at(k):
        return w[:, k]

    def cut(y, k, by):
        return _trunc(y, (w[:, k], w[:, k + 1], w[:, k + 2]), by, bits)
    x = s["x"]
    x = x - cut(x.sum(-1, dtype=x.dtype) * inv, 0, c["shift"])[..., None]
    E = _open(x, a1)
    z = (2 * E * a1).sum(-1, dtype=x.dtype) + at(3)
    z[0] += (E * E).sum(-1, dtype=x.dtype)
    v = public(cut(cut(z, 4, f) * inv, 7, c["shift"]), eps)
    y = cut(public(-slope * v, offset << f), 10, f)
    bv = at(13)
    Fv = _open(v, bv)
    for k in range(14, 14 + 15 * c["iterations"], 15):
        ay, au, ah = at(k), at(k + 5), at(k + 10)
        e = _open(y, ay)
        u = cut(public(at(k + 1) + 2 * e * ay, e * e), k + 2, f)
        t = cut(at(k + 6) + _mul(_open(u, au), au, Fv, bv), k + 7, f)
        h = public(-t, 3 << f)
        y = cut(at(k + 11) + _mul(e, ay, _open(h, ah), ah), k + 12, f + 1)
    b = at(14 + 15 * c["iterations"])
    xhat = _trunc(s["c"][0] + _mul(E, a1, _open(y, b)[..., None], b[..., None]), s["tuples"][0], f, bits)
    gamma, bg = s["gamma"]
    out = _trunc(s["c"][1] + _mul(_open(xhat, a2), a2, _open(gamma, bg), bg[:, None]), s["tuples"][1], f, bits) + s["beta"][:, None]
    return out, xhat, y


def _norm_grad(s):
    c, f = s["case"], s["case"]["f"]
    bits, inv, w = c["bits"], _inverse(c), s["row_words"]
    a1, a2, a3 = s["masks"]
    (gamma, bg), dy, xhat, word = s["gamma"], s["dy"], s["xhat"], s["dy"].dtype

    def cut(y, k, by):
        return _trunc(y, (w[:, k], w[:, k + 1], w[:, k + 2]), by, bits)
    E1, E2 = _open(dy, a1), _open(xhat, a2)
    g = _trunc(s["c"][0] + _mul(E1, a1, _open(gamma, bg), bg[:, None]), s["tuples"][0], f, bits)
    E3 = _open(g, a3)
    cw = s["column_words"]
    dgamma = _trunc(cw[:, 0] + _mul(E1, a1, E2, a2).sum(1, dtype=word), (cw[:, 1], cw[:, 2], cw[:, 3]), f, bits)
    m1 = cut(inv * g.sum(-1, dtype=word), 0, c["shift"])
    m2 = cut(inv * cut(w[:, 3] + _mul(E3, a3, E2, a2).sum(-1, dtype=word), 4, f), 7, c["shift"])
    br, am1, am2, ak = w[:, 10], w[:, 11], w[:, 16], w[:, 21]
    Fr = _open(s["rstd"], br)
    k1 = cut(w[:, 12] + _mul(_open(m1, am1), am1, Fr, br), 13, f)
    k2 = cut(w[:, 17] + _mul(_open(m2, am2), am2, Fr, br), 18, f)
    z = s["c"][1] + _mul(E3, a3, Fr[..., None], br[..., None]) - _mul(E2, a2, _open(k2, ak)[..., None], ak[..., None])
    return _trunc(z, s["tuples"][1], f, bits) - k1[..., None], dgamma, dy.sum(1, dtype=word)


def run(s):
    c = s["case"]
    if not own:
        if c["kind"] in ("prompt", "train"):
            return _attend(s, _Chunks(s))
        return {"step": _step, "norm": _norm, "norm_grad": _norm_grad}[c["kind"]](s)
    from paper_2402_02320_amd import spin
    ring = spin.ring32 if c["bits"] == 32 else spin
    if c["kind"] in ("prompt", "train"):
        return _attend(s, _Calls(s, ring))
    if c["kind"] == "step":
        return ring.linattn_step(s["S"], s["q"], s["k"], s["v"], s["mask"], s["c"], s["tuples"], c["f"], decay=s["decay"], g=c["g"], active=s["active"])
    if c["kind"] == "norm":
        offset, slope, eps = _line(c["f"])
        return ring.layernorm(s["x"], s["gamma"], s["beta"], s["masks"], s["c"], s["tuples"], s["row_words"], c["f"], c["shift"], (offset, slope), eps=eps)
    return ring.layernorm_grad(s["dy"], s["xhat"], s["rstd"], s["gamma"], s["masks"], s["c"], s["tuples"], s["row_words"], s["column_words"], c["f"], c["shift"])


def work(case):
    """bytes: every word that a result depends on read once, every returned word written once; what only passes between the calls of one
    pass (scores, states) is not counted, its dealt masks and tuples are.  flops: two per ring multiply-add, of which a party has two a product."""
    c, n, w = case, case["n"], case["bits"] // 8
    if c["kind"] in ("norm", "norm_grad"):
        r, d = c["rows"], c["dim"]
        if c["kind"] == "norm":
            words = 13 * r * d + 3 * d + r * (15 * c["iterations"] + 16)
            return {"bytes": w * n * words, "flops": 2.0 * n * r * (7 * d + 10 * c["iterations"])}
        return {"bytes": w * n * (12 * r * d + 8 * d + 23 * r), "flops": 2.0 * n * r * 12 * d}
    dk, dv, h = c["dk"], c["dv"], c["heads"]
    if c["kind"] == "step":
        live = sum(0 if c["idle"] and i % 4 == 3 else 1 for i in range(c["batch"])) * h
        idle = c["batch"] * h - live
        return {"bytes": w * n * (live * (7 * dk * dv + 4 * dk + 7 * dv) + idle * (2 * dk * dv + dv)), "flops": 2.0 * n * live * 6 * dk * dv}
    C = c["chunk"]
    parts = [min(C, t - at) for t in _lengths(c) for at in range(0, t, C)]
    tokens, chunks, pairs = h * sum(parts), h * len(parts), h * sum(p * (p + 1) // 2 for p in parts)
    every = h * c["batch"]
    words = tokens * (4 * dk + 2 * dv + 4 * dv) + pairs * 5 + chunks * dk * dv * 5 + every * (2 * dk * dv + c["tokens"] * dv)
    macs = pairs * (dk + dv) + tokens * dk * dv * 2
    if c["kind"] == "train":
        words += tokens * (2 * dv + 8 * dk + 4 * dv) + pairs * 5 + chunks * dk * dv * 5 + every * (2 * dk * dv + c["tokens"] * (2 * dk + dv))
        macs += pairs * (dv + 2 * dk + dv) + tokens * dk * dv * 4
    return {"bytes": w * n * words, "flops": 4.0 * n * macs}


# ---- the definition, word by word on the host -----------------------------------------------------------------
def exact(case, seed):
    c, n = case, case["n"]
    much = work(c)
    if much["flops"] > 1.5e9 or much["bytes"] > 4e8:
        return None                        # minutes on the host
    bits, f = c["bits"], c["f"]
    unsigned, signed = (np.uint32, np.int32) if bits == 32 else (np.uint64, np.int64)

    def host(v):
        if isinstance(v, torch.Tensor):
            return v.cpu().numpy().view(unsigned) if v.dtype != torch.int32 or bits == 32 else v.cpu().numpy()
        return [host(k) for k in v] if isinstance(v, (tuple, list)) else v
    s = {k: host(v) for k, v in prepare(case, seed).items()}

    def word(v):
        return unsigned(v % (1 << bits))

    def total(x, axis):
        return x.sum(axis, dtype=unsigned)

    def truncated(y, tup, by):
        opened = word(1 << (bits - 2)) + total(y, 0) + total(tup[0], 0)
        carry = opened >> unsigned(bits - 1)
        out = np.where(carry == 1, unsigned(0) - tup[2], tup[2])
        out[0] += carry
        out = out * word(1 << (bits - 1 - by)) - tup[1]
        out[0] += (opened % word(1 << (bits - 1))) // word(1 << by) - word(1 << (bits - 2 - by))
        return out

    def product(x, y, times):
        """Shares of x . y behind the dealt word, x and y = (shares, masks), by `times` of (left, right)."""
        (x, a), (y, b) = x, y
        e, g = total(x, 0) - total(a, 0), total(y, 0) - total(b, 0)
        return np.stack([times(e, b[i]) + times(a[i], g) + (times(e, g) if i == 0 else unsigned(0)) for i in range(n)])

    def signed_of(r):
        return tuple(signed_of(v) for v in r) if isinstance(r, tuple) else np.ascontiguousarray(r).view(signed)

    if c["kind"] in ("norm", "norm_grad"):
        d, shift = c["dim"], c["shift"]
        inv = word(((1 << shift) + d // 2) // d)
        w = s["row_words"].transpose(1, 0, 2)

        def times(x, y):
            return x * y

        def three(k):
            return w[k], w[k + 1], w[k + 2]

        def wide(v):
            return np.broadcast_to(v[..., None], v.shape + (d,))
        gamma = [np.broadcast_to(v[:, None], (n, c["rows"], d)) for v in s["gamma"]]
        if c["kind"] == "norm":
            offset, slope, eps = 3 * 2 ** (f - 1), 2 ** (f - 2), 1
            mean = truncated(total(s["x"], -1) * inv, three(0), shift)
            centred = (s["x"] - wide(mean), s["masks"][0])
            square = total(product(centred, centred, times), -1) + w[3]
            var = truncated(truncated(square, three(4), f) * inv, three(7), shift)
            var[0] += word(eps)
            guess = unsigned(0) - var * word(slope)
            guess[0] += word(offset << f)
            y = truncated(guess, three(10), f)
            for k in range(c["iterations"]):
                at = 14 + 15 * k
                u = truncated(w[at + 1] + product((y, w[at]), (y, w[at]), times), three(at + 2), f)
                h = unsigned(0) - truncated(w[at + 6] + product((u, w[at + 5]), (var, w[13]), times), three(at + 7), f)
                h[0] += word(3 << f)
                y = truncated(w[at + 11] + product((y, w[at]), (h, w[at + 10]), times), three(at + 12), f + 1)
            xhat = truncated(s["c"][0] + product(centred, (wide(y), wide(w[14 + 15 * c["iterations"]])), times), s["tuples"][0], f)
            out = truncated(s["c"][1] + product((xhat, s["masks"][1]), gamma, times), s["tuples"][1], f) + s["beta"][:, None]
            return signed_of((out, xhat, y))
        dy, xhat = (s["dy"], s["masks"][0]), (s["xhat"], s["masks"][1])
        g = (truncated(s["c"][0] + product(dy, gamma, times), s["tuples"][0], f), s["masks"][2])
        columns = s["column_words"].transpose(1, 0, 2)
        dgamma = truncated(columns[0] + total(product(dy, xhat, times), 1), columns[1:], f)
        m1 = truncated(total(g[0], -1) * inv, three(0), shift)
        m2 = truncated(truncated(w[3] + total(product(g, xhat, times), -1), three(4), f) * inv, three(7), shift)
        rstd = (s["rstd"], w[10])
        k1 = truncated(w[12] + product((m1, w[11]), rstd, times), three(13), f)
        k2 = truncated(w[17] + product((m2, w[16]), rstd, times), three(18), f)
        z = s["c"][1] + product(g, (wide(s["rstd"]), wide(w[10])), times) - product(xhat, (wide(k2), wide(w[21])), times)
        return signed_of((truncated(z, s["tuples"][1], f) - wide(k1), dgamma, total(dy[0], 1)))

    heads, g = c["heads"], c["g"]

    def w(h, j):
        return word(int(s["decay"][h][j])) if s["decay"] is not None else word(1)

    def pick(pair, b, h, rows=None):
        return tuple(v[:, b, h] if rows is None else v[:, b, h, rows] for v in pair)

    def share(by, x):
        """Shares and masks of rows scaled by public words (one each)."""
        by = np.array(by, unsigned)
        return tuple(v * by[:, None] for v in x)

    def flipped(x):
        return tuple(v.swapaxes(-1, -2) for v in x)

    def matmul(x, y):
        return x @ y if x.shape[-1] else np.zeros((x.shape[0], y.shape[1]), unsigned)

    if c["kind"] == "step":
        S, o = s["S"].copy(), np.zeros_like(s["c"][1])
        for b in range(c["batch"]):
            if s["active"][b] <= 0:
                continue
            for h in range(heads):
                k, v, q = ((tuple(t[:, b, h, :, None] for t in s["k"])), (tuple(t[:, b, h, None] for t in s["v"])), (tuple(t[:, b, h, None] for t in s["q"])))
                z = s["c"][0][:, b, h] + w(h, 0) * product(k, v, matmul) + w(h, 1) * word(1 << f) * S[:, b, h]
                S[:, b, h] = truncated(z, [t[:, b, h] for t in s["tuples"][0]], f + g)
                z = s["c"][1][:, b, h] + product(q, (S[:, b, h], s["mask"][:, b, h]), matmul)[:, 0]
                o[:, b, h] = truncated(z, [t[:, b, h] for t in s["tuples"][1]], f)
        return signed_of((o, S))

    C, nc = c["chunk"], -(-c["tokens"] // c["chunk"])
    lengths = [int(v) for v in s["lengths"]]

    def parts(order):
        for b in range(c["batch"]):
            for h in range(heads):
                for k in order:
                    rows = range(k * C, min((k + 1) * C, max(lengths[b], k * C)))
                    yield b, h, k, slice(rows.start, rows.stop), len(rows)

    def scores(x, y, cc, t):
        out = np.zeros_like(cc)
        for b, h, k, rows, m in parts(range(nc)):
            if m:
                near = np.array([[int(w(h, i - j)) if j <= i else 0 for j in range(m)] for i in range(m)], unsigned)
                z = cc[:, b, h, k, :m, :m] + near * product(pick(x, b, h, rows), flipped(pick(y, b, h, rows)), matmul)
                z = truncated(z, [v[:, b, h, k, :m, :m] for v in t], f + g)
                out[:, b, h, k, :m, :m] = z * (np.tri(m, dtype=unsigned))
        return out

    def states(x, y, cc, t, first, reverse=False):
        before, now = np.zeros_like(cc), first.copy()
        for b, h, k, rows, m in parts(range(nc)[::-1] if reverse else range(nc)):
            before[:, b, h, k] = now[:, b, h]
            if m:
                left = share([int(w(h, j + 1 if reverse else m - 1 - j)) for j in range(m)], pick(x, b, h, rows))
                z = cc[:, b, h, k] + product(flipped(left), pick(y, b, h, rows), matmul) + w(h, m) * word(1 << f) * now[:, b, h]
                now[:, b, h] = truncated(z, [v[:, b, h, k] for v in t], f + g)
        return before, now

    def outputs(p, y, x, S, cc, t, reverse=False, transposed=False):
        out = np.zeros_like(cc)
        for b, h, k, rows, m in parts(range(nc)):
            if m:
                low = tuple(v[:, b, h, k, :m, :m] * np.tri(m, dtype=unsigned) for v in p)
                state = tuple(v[:, b, h, k] for v in S)
                left = share([int(w(h, m - 1 - i if reverse else i + 1)) for i in range(m)], pick(x, b, h, rows))
                z = word(1 << g) * product(flipped(low) if reverse else low, pick(y, b, h, rows), matmul)
                z = z + product(left, flipped(state) if transposed else state, matmul) + cc[:, b, h, rows]
                out[:, b, h, rows] = truncated(z, [v[:, b, h, rows] for v in t], f + g)
        return out

    P = scores(s["q"], s["k"], s["cP"], s["tP"])
    S, last = states(s["k"], s["v"], s["cS"], s["tS"], s["first"])
    O = outputs((P, s["AP"]), s["v"], s["q"], (S, s["AS"]), s["cO"], s["tO"])
    if c["kind"] == "prompt":
        return signed_of((O, last))
    dP = scores(s["dO"], s["v"], s["cdP"], s["tdP"])
    dS, dfirst = states(s["q"], s["dO"], s["cdS"], s["tdS"], s["dlast"], reverse=True)
    dQ = outputs((dP, s["AdP"]), s["k"], s["dO"], (S, s["AS"]), s["cdQ"], s["tdQ"], transposed=True)
    dK = outputs((dP, s["AdP"]), s["q"], s["v"], (dS, s["AdS"]), s["cdK"], s["tdK"], reverse=True, transposed=True)
    dV = outputs((P, s["AP"]), s["dO"], s["k"], (dS, s["AdS"]), s["cdV"], s["tdV"], reverse=True)
    return signed_of((O, last, dQ, dK, dV, dfirst))
