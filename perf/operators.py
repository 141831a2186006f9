"""The operators of a token model of K replicas, as timed cases.

A replica holds one low-rank adapter beside a projection that all replicas share (`adapter`), a gated
linear recurrence that mixes the tokens of a sequence (`recurrence`), dropout whose mask is a function
of a counter, so that both passes of a sharpness-aware step drop the same values (`dropout`), and the
log probabilities of the given tokens with their gradient (`logprobs`).

With `own` false `run` computes the plain form: elementary torch operations in 32 bits, rounded once
at the end.  With `own` true it makes the framework's calls.  `exact` computes the same outputs in 64
bits from the definitions.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ---- the cases --------------------------------------------------------------------------------

def listed():
    return [
        # hidden activations of two workers of the smallest dense model: a call's latency
        dict(name="dropout_batch", op="dropout", K=2, rows=32, cols=784, pad=0, type="fp32", p=0.5, residual=False),
        # hidden states of eight workers, 4096 tokens each, dropped and added to the residual stream
        dict(name="dropout_tokens", op="dropout", K=8, rows=4096, cols=4096, pad=0, type="bf16", p=0.1, residual=True),
        # one new token: its alternatives among the tokens that a grammar allows
        dict(name="logprobs_token", op="logprobs", rows=1, vocab=131072, pad=0, type="bf16", top=20, masked=0.3, grad=False),
        # answers of eight workers, 128 samples each, over 1000 classes, with the five best
        dict(name="logprobs_classes", op="logprobs", rows=1024, vocab=1000, pad=0, type="fp32", top=5, masked=0.0, grad=False),
        # the loss of a training step on 8192 tokens with an entropy bonus, and its gradient; odd vocabulary
        dict(name="logprobs_train", op="logprobs", rows=8192, vocab=49999, pad=1, type="bf16", top=0, masked=0.0, grad=True),
        # one step of 64 sequences that are being generated
        dict(name="recurrence_step", op="recurrence", seqs=64, length=1, dim=4096, type="bf16", ragged=False, grad=False),
        # a training step on eight sequences of equal length
        dict(name="recurrence_train", op="recurrence", seqs=8, length=4096, dim=2048, type="bf16", ragged=False, grad=True),
        # three long documents packed one after the other, of any lengths, on few channels
        dict(name="recurrence_long", op="recurrence", seqs=3, length=43691, dim=1000, type="fp32", ragged=True, grad=True),
        # one new token for each of 32 requests, each with an adapter of its own
        dict(name="adapter_decode", op="adapter", rows=32, inp=4096, out=4096, rank=16, adapters=32, segs=32, type="bf16",
             adapter_type="bf16", bias=False, grad=False),
        # prompts of 21 requests of any lengths, 16 adapters
        dict(name="adapter_prompts", op="adapter", rows=8191, inp=4096, out=8192, rank=32, adapters=16, segs=21, type="bf16",
             adapter_type="bf16", bias=True, grad=False),
        # a training step of eight replicas, 2048 tokens each: adapters and their gradients in 32 bits
        dict(name="adapter_train", op="adapter", rows=16384, inp=4096, out=4096, rank=16, adapters=8, segs=8, type="bf16",
             adapter_type="fp32", bias=False, grad=True),
        # odd widths in 32 bits, so that no tile is full
        dict(name="adapter_odd", op="adapter", rows=777, inp=1000, out=1501, rank=12, adapters=3, segs=5, type="fp32",
             adapter_type="fp32", bias=True, grad=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dropout", "logprobs", "recurrence", "adapter"])
    kind = rng.choice(["fp32", "bf16"])
    if op == "dropout":
        K, cols = rng.randint(1, 8), _log_int(rng, 64, 8192)
        rows = _log_int(rng, 1, max(2, min(16384, 60_000_000 // (K * cols))))
        return dict(op=op, K=K, rows=rows, cols=cols, pad=rng.choice([0, 0, 1, 8]), type=kind, p=rng.choice([0.05, 0.1, 0.25, 0.5]),
                    residual=rng.random() < 0.5)
    if op == "logprobs":
        vocab = _log_int(rng, 10, 131072)
        grad = rng.random() < 0.5
        rows = _log_int(rng, 1, max(2, min(16384, (200_000_000 if grad else 40_000_000) // vocab)))
        return dict(op=op, rows=rows, vocab=vocab, pad=rng.choice([0, 0, 1, 16]), type=kind,
                    top=0 if grad else rng.randint(0, min(32, vocab // 2)), masked=rng.choice([0.0, 0.0, 0.3]), grad=grad)
    if op == "recurrence":
        dim, seqs = _log_int(rng, 64, 4096), _log_int(rng, 1, 64)
        length = 1 if rng.random() < 0.25 else _log_int(rng, 2, max(3, min(40000, 60_000_000 // (dim * seqs))))
        return dict(op=op, seqs=seqs, length=length, dim=dim, type=kind, ragged=length > 1 and rng.random() < 0.5,
                    grad=rng.random() < 0.5)
    rows, segs = _log_int(rng, 1, 8192), rng.randint(1, 40)
    even = rng.random() < 0.6
    inp, out = _log_int(rng, 64, 4096), _log_int(rng, 64, 4096)
    return dict(op=op, rows=rows, inp=inp // 8 * 8 if even else inp, out=out // 8 * 8 if even else out, rank=rng.choice([4, 8, 12, 16, 32, 64]),
                adapters=rng.randint(1, 24), segs=segs, type=kind, adapter_type=rng.choice(["fp32", "fp32" if kind == "fp32" else "bf16"]),
                bias=rng.random() < 0.5, grad=rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------------------------

def _pieces(rng, total, n):
    """n + 1 places that cut `total` rows into n pieces of any lengths, none among them."""
    return [0] + sorted(rng.randint(0, total) for _ in range(n - 1)) + [total]


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    t = TYPES[case["type"]]

    def normal(*shape, std=1.0, mean=0.0, type=t):
        return torch.empty(*shape, device=DEV).normal_(mean, std, generator=g).to(type)

    if case["op"] == "dropout":
        K, rows, cols, ld = case["K"], case["rows"], case["cols"], case["cols"] + case["pad"]
        x = normal(K, rows, ld)[:, :, :cols]
        res = normal(K, rows, ld)[:, :, :cols] if case["residual"] else None
        return dict(x=x, residual=res, p=case["p"], seed=rng.getrandbits(64), step=rng.getrandbits(20), site=rng.randrange(64))
    if case["op"] == "logprobs":
        rows, V, ld = case["rows"], case["vocab"], case["vocab"] + case["pad"]
        z = normal(rows, ld, std=2.5)[:, :V]
        tokens = torch.randint(0, V, (rows,), device=DEV, generator=g, dtype=torch.int32)
        if case["masked"]:
            barred = torch.rand(rows, V, device=DEV, generator=g) < case["masked"]
            barred.scatter_(1, tokens.long()[:, None], False)
            z.masked_fill_(barred, -math.inf)
        d = dict(z=z, tokens=tokens, top=case["top"])
        if case["grad"]:
            tokens[torch.rand(rows, device=DEV, generator=g) < 0.03] = -1          # tokens that do not count
            d["g_logp"] = normal(rows, std=0.3, mean=-1.0, type=torch.float32) / rows
            d["g_entropy"] = normal(rows, std=0.1, type=torch.float32) / rows
        return d
    if case["op"] == "recurrence":
        S, T, D = case["seqs"], case["length"], case["dim"]
        shape = (S * T, D) if case["ragged"] else (S, T, D)
        d = dict(f=normal(*shape, mean=2.0, std=1.5), x=normal(*shape), h0=normal(S, D, type=torch.float32), offsets=None)
        if case["ragged"]:
            d["offsets"] = torch.tensor(_pieces(rng, S * T, S), dtype=torch.int64, device=DEV)
        if case["grad"]:
            d["dh"], d["dlast"] = normal(*shape), normal(S, D, type=torch.float32)
        return d
    n, inp, out, r, m, ta = case["rows"], case["inp"], case["out"], case["rank"], case["adapters"], TYPES[case["adapter_type"]]
    begin = _pieces(rng, n, case["segs"])
    if case["segs"] == m and n % m == 0:            # one adapter for each of the replicas or requests
        begin, which = [k * (n // m) for k in range(m + 1)], list(range(m))
        rng.shuffle(which)
    else:                                           # some requests have none
        which = [rng.randint(-1, m - 1) for _ in range(case["segs"])]
    d = dict(x=normal(n, inp), W=normal(out, inp, std=inp ** -0.5), bias=normal(out, type=torch.float32) if case["bias"] else None,
             A=normal(m, r, inp, std=inp ** -0.5, type=ta), B=normal(m, out, r, std=0.5, type=ta), scale=2.0,
             begin=torch.tensor(begin, dtype=torch.int32, device=DEV), which=torch.tensor(which, dtype=torch.int32, device=DEV))
    if case["grad"]:
        d["dy"] = normal(n, out)
    return d


def prepare(case, seed):
    return dict(op=case["op"], type=TYPES[case["type"]], grad=bool(case.get("grad")), **_inputs(case, seed))


# ---- one pass ---------------------------------------------------------------------------------

def run(state):
    return (OWN if own else PLAIN)[state["op"]](state)


def _own_dropout(s):
    from paper_2509_03110_amd import ops
    return ops.dropout(s["x"], s["p"], seed=s["seed"], step=s["step"], site=s["site"], residual=s["residual"])


def _own_logprobs(s):
    from paper_2509_03110_amd import ops
    r = ops.logprobs(s["z"], s["tokens"], top=s["top"])
    out = dict(logp=r.logp, entropy=r.entropy)
    if s["top"]:
        out.update(ids=r.top_ids, best=r.top_logp)
    if s["grad"]:
        out["dz"] = ops.logprobs_backward(s["z"], s["tokens"], r.lse, r.entropy, s["g_logp"], s["g_entropy"])
    return out


def _own_recurrence(s):
    from paper_2509_03110_amd import ops
    r = ops.recurrence(s["f"], s["x"], h0=s["h0"], offsets=s["offsets"], save=s["grad"])
    out = dict(h=r.h, last=r.last)
    if s["grad"]:
        out["df"], out["dx"], out["dh0"] = ops.recurrence_backward(s["f"], s["x"], s["dh"], r.states, h0=s["h0"], dlast=s["dlast"],
                                                                   offsets=s["offsets"])
    return out


def _own_adapter(s):
    from paper_2509_03110_amd import ops
    y, u = ops.adapter(s["x"], s["W"], s["A"], s["B"], s["begin"], s["which"], s["scale"], bias=s["bias"])
    if not s["grad"]:
        return dict(y=y)
    dx, dA, dB = ops.adapter_backward(s["x"], s["W"], s["A"], s["B"], u, s["dy"], s["begin"], s["which"], s["scale"])
    return dict(y=y, dx=dx, dA=dA, dB=dB)


OWN = dict(dropout=_own_dropout, logprobs=_own_logprobs, recurrence=_own_recurrence, adapter=_own_adapter)


# ---- the plain forms --------------------------------------------------------------------------

def _philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 of 32-bit counters in 64-bit integers: four words for each counter."""
    low = 0xFFFFFFFF
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _plain_dropout(s):
    x = s["x"]
    K, rows, cols = x.shape
    groups = (cols + 7) // 8
    shape = (K, rows, groups)
    at = lambda n, k: torch.arange(n, device=DEV).view([-1 if i == k else 1 for i in range(3)]).expand(shape)  # noqa: E731
    c3 = torch.full(shape, s["step"], device=DEV, dtype=torch.int64)
    words = torch.stack(_philox(at(groups, 2), at(rows, 1), s["site"] | (at(K, 0) << 16), c3, s["seed"]), -1)
    halves = torch.stack((words & 0xFFFF, words >> 16), -1).view(K, rows, groups * 8)[:, :, :cols]
    drop = round(s["p"] * 65536)
    y = torch.where(halves >= drop, x.float() * (65536.0 / (65536 - drop)), 0.0)
    return (y if s["residual"] is None else y + s["residual"].float()).to(s["type"])


def _plain_logprobs(s):
    z, tokens = s["z"].float(), s["tokens"].long()
    counts = tokens >= 0
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    lp = z - lse
    p = e / total
    plp = torch.where(p > 0, p * lp, 0.0)
    entropy = -plp.sum(1)
    logp = torch.where(counts, lp.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0)
    out = dict(logp=logp, entropy=entropy)
    if s["top"]:
        best, ids = torch.sort(z, dim=1, descending=True, stable=True)
        out.update(ids=ids[:, :s["top"]].to(torch.int32), best=best[:, :s["top"]] - lse)
    if s["grad"]:
        g = torch.where(counts, s["g_logp"], 0.0)[:, None]
        dz = -g * p - s["g_entropy"][:, None] * (plp + p * entropy[:, None])
        dz.scatter_add_(1, tokens.clamp(min=0)[:, None], g)
        out["dz"] = dz.to(s["type"])
    return out


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dim 0 from h_{-1} = 0: spans of 1, 2, 4, ... steps joined to the ones before."""
    n = 1
    while n < a.shape[0]:
        b = torch.cat((b[:n], a[n:] * b[:-n] + b[n:]))
        a = torch.cat((a[:n], a[n:] * a[:-n]))
        n *= 2
    return b


def _plain_recurrence(s):
    S, D = s["h0"].shape
    shape = s["f"].shape
    packed = s["offsets"] is not None
    lay = (lambda t: t.float()) if packed else (lambda t: t.float().transpose(0, 1))        # time first
    back = (lambda t: t) if packed else (lambda t: t.transpose(0, 1))
    f, x, h0 = lay(s["f"]), lay(s["x"]), s["h0"]
    a, i = torch.sigmoid(f), torch.sigmoid(-f)
    if packed:
        first, end = s["offsets"][:-1], s["offsets"][1:]
        some = (end > first).nonzero()[:, 0]
        first, final, h0 = first[some], end[some] - 1, h0[some]
    else:
        first, final, some = torch.zeros(1, dtype=torch.int64, device=DEV), torch.full((1,), shape[1] - 1, device=DEV), slice(None)
    one = (lambda t: t) if packed else (lambda t: t[None])
    cut = a.index_fill(0, first, 0.0)                                                       # nothing comes over a first row
    b = i * x
    b[first] += a[first] * one(h0)
    h = _scan(cut, b)
    last = s["h0"].clone()
    last[some] = h[final] if packed else h[-1]
    out = dict(h=back(h).to(s["type"]), last=last)
    if s["grad"]:
        before = torch.cat((torch.zeros_like(h[:1]), h[:-1]))
        before[first] = one(h0)
        dh = lay(s["dh"]).clone()
        dh[final] += one(s["dlast"][some])
        after = torch.cat((cut[1:], torch.zeros_like(a[:1])))
        d = _scan(after.flip(0), dh.flip(0)).flip(0)
        dh0 = s["dlast"].clone()
        dh0[some] = (a[first] * d[first]) if packed else (a[0] * d[0])
        out.update(df=back(a * i * d * (before - x)).to(s["type"]), dx=back(i * d).to(s["type"]), dh0=dh0)
    return out


def _plain_adapter(s):
    x, W, A, B, scale = s["x"].float(), s["W"].float(), s["A"].float(), s["B"].float(), s["scale"]
    m, r, inp = A.shape
    n, out = x.shape[0], W.shape[0]
    seg = torch.searchsorted(s["begin"][1:].contiguous(), torch.arange(n, device=DEV, dtype=torch.int32), right=True)
    which = s["which"].long()[seg]                                                          # the adapter of each row, or -1
    mine = (which[:, None] == torch.arange(m, device=DEV)).float()[:, :, None]              # [n, m, 1]
    A_all, B_all = A.reshape(m * r, inp), B.permute(0, 2, 1).reshape(m * r, out)
    u = ((x @ A_all.t()).view(n, m, r) * mine).view(n, m * r)
    y = x @ W.t() + scale * (u @ B_all)
    if s["bias"] is not None:
        y = y + s["bias"]
    got = dict(y=y.to(s["type"]))
    if s["grad"]:
        dy = s["dy"].float()
        du = ((dy @ B_all.t()).view(n, m, r) * (scale * mine)).view(n, m * r)
        got["dx"] = (dy @ W + du @ A_all).to(s["type"])
        got["dA"] = (du.t() @ x).view(m, r, inp)
        got["dB"] = (scale * (u.t() @ dy)).view(m, r, out).permute(0, 2, 1).contiguous()
    return got


PLAIN = dict(dropout=_plain_dropout, logprobs=_plain_logprobs, recurrence=_plain_recurrence, adapter=_plain_adapter)


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    b = 2 if case["type"] == "bf16" else 4
    if case["op"] == "dropout":
        n = case["K"] * case["rows"] * case["cols"]
        return dict(bytes=n * b * (3 if case["residual"] else 2), flops=2 * n)
    if case["op"] == "logprobs":
        n = case["rows"] * case["vocab"]
        return dict(bytes=n * b * (2 if case["grad"] else 1) + case["rows"] * (12 + 8 * case["top"]), flops=n * (12 if case["grad"] else 6))
    if case["op"] == "recurrence":
        n, state = case["seqs"] * case["length"] * case["dim"], 4 * case["seqs"] * case["dim"]
        return dict(bytes=n * b * (6 if case["grad"] else 3) + state * (4 if case["grad"] else 2), flops=n * (20 if case["grad"] else 8))
    n, i, o, r, m = case["rows"], case["inp"], case["out"], case["rank"], case["adapters"]
    ba = 2 if case["adapter_type"] == "bf16" else 4
    low = 2 * n * r * (i + o)
    if case["grad"]:
        return dict(bytes=b * (2 * n * (i + o) + i * o) + m * r * (i + o) * (ba + 4), flops=4 * n * i * o + 3 * low)
    return dict(bytes=b * (n * (i + o) + i * o) + min(m, case["segs"]) * r * (i + o) * ba, flops=2 * n * i * o + low)


# ---- the definitions in 64 bits -----------------------------------------------------------------

def exact(case, seed):
    return EXACT[case["op"]](case, _inputs(case, seed))


def _exact_dropout(case, s):
    K, rows, cols = s["x"].shape
    if K * rows * cols > 40_000_000:
        return None
    groups = -(-cols // 8)
    u64 = np.uint64
    mask, shift = u64(0xFFFFFFFF), u64(32)
    key = [u64(s["seed"] % 2 ** 32), u64(s["seed"] // 2 ** 32)]
    k, r, c = np.meshgrid(np.arange(K, dtype=u64), np.arange(rows, dtype=u64), np.arange(groups, dtype=u64), indexing="ij")
    v = [c, r, k * u64(65536) + u64(s["site"]), np.full_like(c, s["step"])]
    for n in range(10):
        lo, hi = v[0] * u64(0xD2511F53), v[2] * u64(0xCD9E8D57)
        v = [(hi >> shift) ^ v[1] ^ key[0], hi & mask, (lo >> shift) ^ v[3] ^ key[1], lo & mask]
        key = [(key[0] + u64(0x9E3779B9)) & mask, (key[1] + u64(0xBB67AE85)) & mask]
    draws = np.zeros((K, rows, groups * 8), np.uint32)
    for e in range(8):
        draws[:, :, e::8] = (v[e // 2] >> u64(16 * (e % 2))) & u64(0xFFFF)
    drop = round(case["p"] * 65536)
    x = s["x"].double().cpu().numpy()
    y = np.where(draws[:, :, :cols] < drop, 0.0, x * 65536 / (65536 - drop))
    return y if s["residual"] is None else y + s["residual"].double().cpu().numpy()


def _exact_logprobs(case, s):
    parts = []
    for lo in range(0, case["rows"], 512):
        z, tok = s["z"][lo:lo + 512].double(), s["tokens"][lo:lo + 512].long()
        rows = torch.arange(z.shape[0], device=DEV)
        top = z.max(1).values
        lse = top + (z - top[:, None]).exp().sum(1).log()
        logs = z - lse[:, None]
        p = logs.exp()
        weighted = torch.nan_to_num(p * logs, nan=0.0)
        H = -weighted.sum(1)
        has = tok >= 0
        part = dict(logp=torch.where(has, logs[rows, tok.clamp(min=0)], torch.zeros_like(H)), entropy=H)
        if case["top"]:
            part["best"] = torch.topk(logs, case["top"], dim=1).values
        if case["grad"]:
            gl, ge = s["g_logp"][lo:lo + 512].double() * has, s["g_entropy"][lo:lo + 512].double()
            dz = -(p * gl[:, None]) - ge[:, None] * (weighted + p * H[:, None])
            dz[rows[has], tok[has]] += gl[has]
            part["dz"] = dz
        parts.append(part)
    got = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    return dict(got, ids=None) if case["top"] else got


def _exact_recurrence(case, s):
    S, T, D = case["seqs"], case["length"], case["dim"]
    ends = s["offsets"].tolist() if case["ragged"] else [T * k for k in range(S + 1)]
    lengths = [ends[k + 1] - ends[k] for k in range(S)]
    longest = max(lengths)
    if longest > 150_000 or S * longest * D > 500_000_000:
        return None
    flat = lambda t: t.reshape(S * T, D)  # noqa: E731

    def spread(t, fill):
        """[longest, S, D] with the sequences side by side."""
        out = torch.full((longest, S, D), fill, device=DEV, dtype=torch.float64)
        for k in range(S):
            out[:lengths[k], k] = flat(t)[ends[k]:ends[k + 1]].double()
        return out

    def gather(t):
        return torch.cat([t[:lengths[k], k] for k in range(S)]).reshape(s["f"].shape)

    f, x = spread(s["f"], math.inf), spread(s["x"], 0.0)             # past a sequence's end its state stays as it is
    a = 1 / (1 + torch.exp(-f))
    i = 1 / (1 + torch.exp(f))
    v = i * x
    h = torch.empty(longest + 1, S, D, device=DEV, dtype=torch.float64)
    h[0] = s["h0"]
    for t in range(longest):
        torch.addcmul(v[t], a[t], h[t], out=h[t + 1])
    out = dict(h=gather(h[1:]), last=h[longest])
    if case["grad"]:
        dh = spread(s["dh"], 0.0)
        d = torch.empty_like(dh)
        carry = s["dlast"].double()
        for t in range(longest - 1, -1, -1):
            torch.add(dh[t], carry, out=d[t])
            carry = a[t] * d[t]
        out.update(df=gather(a * i * d * (h[:-1] - x)), dx=gather(i * d), dh0=carry)
    return out


def _exact_adapter(case, s):
    x, W = s["x"].double(), s["W"].double()
    y = x @ W.T
    if s["bias"] is not None:
        y += s["bias"].double()
    begin, which = s["begin"].tolist(), s["which"].tolist()
    if case["grad"]:
        dy = s["dy"].double()
        dx, dA, dB = dy @ W, torch.zeros_like(s["A"], dtype=torch.float64), torch.zeros_like(s["B"], dtype=torch.float64)
    for k, a in enumerate(which):
        rows = slice(begin[k], begin[k + 1])
        if a < 0 or begin[k] == begin[k + 1]:
            continue
        A, B = s["A"][a].double(), s["B"][a].double()
        u = x[rows] @ A.T
        y[rows] += s["scale"] * (u @ B.T)
        if case["grad"]:
            du = s["scale"] * (dy[rows] @ B)
            dx[rows] += du @ A
            dA[a] += du.T @ x[rows]
            dB[a] += s["scale"] * (dy[rows].T @ u)
    return dict(y=y, dx=dx, dA=dA, dB=dB) if case["grad"] else dict(y=y)


EXACT = dict(dropout=_exact_dropout, logprobs=_exact_logprobs, recurrence=_exact_recurrence, adapter=_exact_adapter)
