"""What the operators of a transformer block's training step are measured on: dropout from a counter-based generator,
layer norm (alone, or fused with dropout and the residual add) and the attention softmax with a learned relative
position bias by buckets, each forward and backward.

`run` computes a case with the library's entry points where `own` is true, else in plain torch operations in 32 bits.

Random bits: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011) with the
seed as key and (column // 8, row, step, site) as counter; element (row, column) takes the 16-bit half column % 8 of the
128 bits (low half of a word first), is kept when that is at least T = round(65536 p), and is then multiplied by
65536 / (65536 - T).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SITE = 7            # which of the model's dropouts this is
EPS = 1e-5


# ---------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # activations of a batch of sequences in front of a residual add: the ordinary large call
        dict(name="dropout_bf16", op="dropout", rows=16384, cols=4096, type="bf16", p=0.1),
        # a classifier's ragged hidden layer, rows that start at no vector boundary
        dict(name="dropout_odd_f32", op="dropout", rows=2011, cols=1001, type="f32", p=0.25),
        # the normalisation of four new tokens when a model answers: nothing but latency
        dict(name="norm_tokens", op="norm", back=False, rows=4, cols=4096, type="bf16", param="f32", fused=False, p=0.0),
        # an odd width in binary16
        dict(name="norm_odd_f16", op="norm", back=False, rows=5000, cols=1001, type="f16", param="f16", fused=False, p=0.0),
        # a block's joint in training: residual + dropout(x), then the norm
        dict(name="add_norm", op="norm", back=False, rows=16384, cols=2048, type="bf16", param="f32", fused=True, p=0.1),
        # backward of a plain norm, master parameters in binary32
        dict(name="norm_back", op="norm", back=True, rows=8192, cols=1024, type="bf16", param="f32", fused=False, p=0.0),
        # backward of the joint at the width and batch where it costs most
        dict(name="add_norm_back", op="norm", back=True, rows=16384, cols=4096, type="bf16", param="f32", fused=True, p=0.1),
        # backward at an odd width, everything in binary32, few rows
        dict(name="norm_back_odd_f32", op="norm", back=True, rows=777, cols=1001, type="f32", param="f32", fused=False, p=0.0),
        # encoder self-attention in training: ragged lengths, bias both ways, dropout of the probabilities
        dict(name="softmax", op="softmax", back=False, batch=8, heads=16, q=1024, k=1024, type="bf16", causal=False,
             ragged=True, buckets=32, distance=128, p=0.1),
        # one new token per sequence over a long past
        dict(name="softmax_token", op="softmax", back=False, batch=16, heads=16, q=1, k=16384, type="bf16", causal=True,
             ragged=True, buckets=32, distance=128, p=0.0),
        # the encoder's backward pass, with the bias table's gradient
        dict(name="softmax_back", op="softmax", back=True, batch=8, heads=16, q=1024, k=1024, type="bf16", causal=False,
             ragged=True, buckets=32, distance=128, p=0.1),
        # decoder self-attention at an odd length, backward, binary16
        dict(name="softmax_back_odd", op="softmax", back=True, batch=3, heads=8, q=997, k=997, type="f16", causal=True,
             ragged=False, buckets=32, distance=128, p=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A size between lo and hi, evenly over its logarithm; half of them multiples of 64, the others as they fall."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["dropout", "norm", "norm", "softmax", "softmax"])
    kind = rng.choice(["f32", "bf16", "bf16", "f16"])
    most = 1 << (25 if kind == "f32" else 26)
    p = rng.choice([0.0, 0.05, 0.1, 0.25, 0.5])
    if op != "softmax":
        cols = _width(rng, 64, 16384)
        rows = _log(rng, 1, min(65536, most // cols))
        if op == "dropout":
            return dict(op=op, rows=rows, cols=cols, type=kind, p=p or 0.1)
        fused = rng.random() < 0.6
        return dict(op=op, back=rng.random() < 0.5, rows=rows, cols=cols, type=kind, param=rng.choice(["f32", kind]),
                    fused=fused, p=p if fused else 0.0)
    back = rng.random() < 0.5
    batch, heads = _log(rng, 1, 16), _log(rng, 1, 32)
    token = not back and rng.random() < 0.4
    if token:
        k = min(_width(rng, 64, 65536), most // (batch * heads))
        q, causal, p = 1, True, 0.0
    else:
        k = min(_width(rng, 16, 4096), int(math.sqrt(most / (batch * heads))))
        causal = rng.random() < 0.5
        q = k if rng.random() < 0.6 else max(1, int(k * rng.uniform(0.05, 1.0)))
    return dict(op=op, back=back, batch=batch, heads=heads, q=q, k=k, type=kind, causal=causal, ragged=rng.random() < 0.5,
                buckets=rng.choice([16, 32, 64]), distance=rng.choice([64, 128, 256]), p=p)


# --------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["type"]]

    def normal(*shape, scale=1.0):
        return torch.empty(shape, device="cuda").normal_(0.0, scale, generator=gen)

    s = {"case": case, "rng": torch.tensor([(seed * 0x9E3779B97F4A7C15 + 12345) & (2 ** 62 - 1), 3 + seed % 1000],
                                           dtype=torch.int64, device="cuda")}
    if case["op"] == "dropout":
        s["x"] = normal(case["rows"], case["cols"]).to(dt)
        s["y"] = torch.empty_like(s["x"])
    elif case["op"] == "norm":
        rows, cols, pdt = case["rows"], case["cols"], DTYPES[case["param"]]
        s["weight"] = (1.0 + normal(cols, scale=0.2)).to(pdt)
        s["bias"] = normal(cols, scale=0.2).to(pdt)
        channel = torch.exp(normal(cols, scale=0.5))          # some channels of a trained model are larger than others
        x = normal(rows, cols) * channel + 0.3
        if not case["back"]:
            s["x"] = x.to(dt)
            s["y"] = torch.empty_like(s["x"])
            s["mean"], s["rstd"] = (torch.empty(rows, device="cuda") for _ in range(2))
            if case["fused"]:
                s["residual"] = normal(rows, cols, scale=2.0).to(dt)
                s["h"] = torch.empty_like(s["x"])
        else:
            s["h"] = x.to(dt)
            h = s["h"].float()
            s["mean"] = h.mean(1)
            s["rstd"] = torch.rsqrt((h - s["mean"][:, None]).square().mean(1) + EPS)
            s["dy"] = normal(rows, cols, scale=0.05).to(dt)
            s["dx"] = torch.empty_like(s["h"])
            s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
            if case["fused"]:
                s["dh"] = normal(rows, cols, scale=0.05).to(dt)
                s["dresidual"] = torch.empty_like(s["h"])
            if own:
                from paper_1712_02679_b200 import binding as B
                s["workspace"] = torch.empty(B.adacomp_layer_norm_workspace(rows, cols), dtype=torch.uint8, device="cuda")
    else:
        shape = (case["batch"], case["heads"], case["q"], case["k"])
        s["scores"] = normal(*shape, scale=8.0).to(dt)
        s["scale"] = 0.25
        s["table"] = normal(case["buckets"], case["heads"], scale=0.7)
        s["q_offset"] = case["k"] - case["q"]
        s["key_len"] = None
        if case["ragged"]:
            s["key_len"] = torch.randint((case["k"] + 1) // 2, case["k"] + 1, (case["batch"],), device="cuda", generator=gen,
                                         dtype=torch.int32)
        if own:
            from paper_1712_02679_b200 import binding as B
            s["relpos"] = B.adacomp_relpos_plan(case["buckets"], case["distance"], not case["causal"])
        if not case["back"]:
            s["probs"] = torch.empty_like(s["scores"])
            s["lse"] = torch.empty(shape[:3], device="cuda")
        else:
            s["lse"] = _logits(s)[0].logsumexp(-1)
            s["dprobs"] = normal(*shape, scale=0.05).to(dt)
            s["dscores"] = torch.empty_like(s["scores"])
            s["dtable"] = torch.empty_like(s["table"])
            if own:
                s["workspace"] = torch.empty(B.adacomp_bias_softmax_workspace(*shape, s["relpos"]), dtype=torch.uint8,
                                             device="cuda")
    return s


# ----------------------------------------------------------------------------------------- one pass of a case

def run(state):
    case = state["case"]
    op = case["op"] + ("_back" if case.get("back") else "")
    return (_own if own else _plain)[op](state)


def _own_dropout(s):
    from paper_1712_02679_b200 import binding as B
    B.adacomp_dropout(s["x"], s["y"], s["case"]["p"], s["rng"], site=SITE)
    return {"y": s["y"]}


def _own_norm(s):
    from paper_1712_02679_b200 import binding as B
    c = s["case"]
    B.adacomp_layer_norm(s["x"], s["weight"], s["bias"], s["y"], s["mean"], s["rstd"], eps=EPS, residual=s.get("residual"),
                         h_out=s.get("h"), p=c["p"], rng=s["rng"], site=SITE)
    out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    return {**out, "h": s["h"]} if c["fused"] else out


def _own_norm_back(s):
    from paper_1712_02679_b200 import binding as B
    c = s["case"]
    B.adacomp_layer_norm_backward(s["dy"], s["h"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"],
                                  s["workspace"], dh_in=s.get("dh"), dresidual=s.get("dresidual"), p=c["p"], rng=s["rng"],
                                  site=SITE)
    out = {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    return {**out, "dresidual": s["dresidual"]} if c["fused"] else out


def _own_softmax(s):
    from paper_1712_02679_b200 import binding as B
    c = s["case"]
    B.adacomp_bias_softmax(s["scores"], s["table"], s["relpos"], s["probs"], s["lse"], scale=s["scale"], causal=c["causal"],
                           q_offset=s["q_offset"], key_len=s["key_len"], p=c["p"], rng=s["rng"], site=SITE)
    return {"probs": s["probs"], "lse": s["lse"]}


def _own_softmax_back(s):
    from paper_1712_02679_b200 import binding as B
    c = s["case"]
    B.adacomp_bias_softmax_backward(s["dprobs"], s["scores"], s["table"], s["relpos"], s["lse"], s["dscores"], s["dtable"],
                                    s["workspace"], scale=s["scale"], causal=c["causal"], q_offset=s["q_offset"],
                                    key_len=s["key_len"], p=c["p"], rng=s["rng"], site=SITE)
    return {"dscores": s["dscores"], "dtable": s["dtable"]}


_own = {"dropout": _own_dropout, "norm": _own_norm, "norm_back": _own_norm_back, "softmax": _own_softmax,
        "softmax_back": _own_softmax_back}


# ------------------------------------------------------------------- the plain forms: torch operations, 32 bits

def _kept(rng, rows, cols, p):
    """Which elements of [rows, cols] dropout keeps.  Integers below 2^32 held in int64: the product's high half comes out
    of a wrapped 64-bit product by an arithmetic shift and a mask."""
    low = 0xFFFFFFFF
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    groups = -(-cols // 8)
    zero = torch.zeros(rows, groups, dtype=torch.int64, device="cuda")
    c0 = zero + torch.arange(groups, device="cuda")
    c1 = zero + torch.arange(rows, device="cuda")[:, None]
    c2 = zero + (rng[1] & low)
    c3 = zero + SITE
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    halves = [(c >> sh & 0xFFFF).to(torch.int32) for c in (c0, c1, c2, c3) for sh in (0, 16)]
    return (torch.stack(halves, -1) >= round(65536 * p)).view(rows, groups * 8)[:, :cols]


def _dropped(x, rng, p):
    """Dropout of a 32-bit tensor; rows are all dimensions but the last."""
    if p == 0.0:
        return x
    keep = _kept(rng, x.numel() // x.shape[-1], x.shape[-1], p).view(x.shape)
    return torch.where(keep, x * (65536.0 / (65536 - round(65536 * p))), 0.0)


def _plain_dropout(s):
    return {"y": _dropped(s["x"].float(), s["rng"], s["case"]["p"]).to(s["x"].dtype)}


def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    h = _dropped(s["x"].float(), s["rng"], c["p"])
    if c["fused"]:
        h = h + s["residual"].float()
    mean = h.mean(1)
    centred = h - mean[:, None]
    rstd = torch.rsqrt(centred.square().mean(1) + EPS)
    y = centred * rstd[:, None] * s["weight"].float() + s["bias"].float()
    out = {"y": y.to(dt), "mean": mean, "rstd": rstd}
    return {**out, "h": h.to(dt)} if c["fused"] else out


def _plain_norm_back(s):
    c, dt = s["case"], s["h"].dtype
    dy = s["dy"].float()
    xhat = (s["h"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"].float()
    dh = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if c["fused"]:
        dh = dh + s["dh"].float()
    out = {"dx": _dropped(dh, s["rng"], c["p"]).to(dt), "dweight": (dy * xhat).sum(0).to(s["weight"].dtype),
           "dbias": dy.sum(0).to(s["bias"].dtype)}
    return {**out, "dresidual": dh.to(dt)} if c["fused"] else out


def _first_distances(case):
    """first[k]: the smallest distance whose bucket is k or more, per side.  Half of a side's buckets hold one distance
    each, the others are spaced by equal ratios up to `distance`."""
    n = case["buckets"] if case["causal"] else case["buckets"] // 2
    exact = n // 2
    first = list(range(exact + 1))
    for k in range(1, n - exact):
        v = exact * (case["distance"] / exact) ** (k / (n - exact))
        first.append(math.ceil(v - 1e-9 * v))
    return first


def _bucket_of(case, device="cuda"):
    """Bucket of every (query, key) pair."""
    i = torch.arange(case["q"], device=device)[:, None] + (case["k"] - case["q"])
    j = torch.arange(case["k"], device=device)[None, :]
    first = torch.tensor(_first_distances(case), device=device)
    away = (i - j).clamp(min=0) if case["causal"] else (i - j).abs()
    bucket = torch.searchsorted(first, away, right=True) - 1
    return bucket if case["causal"] else bucket + (j > i) * len(first)


def _logits(s):
    """Logits in 32 bits, -inf where masked; and the buckets."""
    c = s["case"]
    bucket = _bucket_of(c)
    t = s["scores"].float() * s["scale"] + s["table"].t()[:, bucket]
    j = torch.arange(c["k"], device="cuda")
    if c["causal"]:
        t = t.masked_fill(j[None, :] > torch.arange(c["q"], device="cuda")[:, None] + s["q_offset"], -math.inf)
    if s["key_len"] is not None:
        t = t.masked_fill((j[None, :] >= s["key_len"][:, None])[:, None, None, :], -math.inf)
    return t, bucket


def _plain_softmax(s):
    t, _ = _logits(s)
    top = t.amax(-1, keepdim=True)
    e = torch.exp(t - top)
    total = e.sum(-1, keepdim=True)
    probs = _dropped(e / total, s["rng"], s["case"]["p"])
    return {"probs": probs.to(s["scores"].dtype), "lse": (top + torch.log(total)).squeeze(-1)}


def _plain_softmax_back(s):
    c = s["case"]
    t, bucket = _logits(s)
    probs = torch.exp(t - s["lse"][..., None])
    dp = _dropped(s["dprobs"].float(), s["rng"], c["p"])
    ds = probs * (dp - (probs * dp).sum(-1, keepdim=True))
    over = ds.sum(0)
    dtable = torch.stack([(over * (bucket == b)).sum((1, 2)) for b in range(c["buckets"])])
    return {"dscores": (ds * s["scale"]).to(s["scores"].dtype), "dtable": dtable}


_plain = {"dropout": _plain_dropout, "norm": _plain_norm, "norm_back": _plain_norm_back, "softmax": _plain_softmax,
          "softmax_back": _plain_softmax_back}


# ----------------------------------------------------------------------------------------------------- work

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    e = size[case["type"]]
    # the generator: ten rounds of two products, four exclusive ors and two additions per eight elements
    draws = 10.0 if case["p"] else 0.0
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * e, "flops": n * (1 + draws)}
    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        arrays = (5 if case["back"] else 4) if case["fused"] else (3 if case["back"] else 2)
        params = (3 if case["back"] else 2) * case["cols"] * size[case["param"]]
        return {"bytes": arrays * n * e + params + 8 * case["rows"], "flops": n * ((14 if case["back"] else 8) + draws)}
    b, h, q, k = case["batch"], case["heads"], case["q"], case["k"]
    pairs = q * k - (q * (q - 1) // 2 if case["causal"] else 0)
    kept = b * h * pairs * (0.75 if case["ragged"] else 1.0)       # lengths fall evenly between half and all
    written = b * h * q * k
    reads = (2 if case["back"] else 1) * kept
    tables = (2 if case["back"] else 1) * case["buckets"] * h * 4
    return {"bytes": (reads + written) * e + 4 * b * h * q + tables, "flops": kept * ((12 if case["back"] else 8) + draws)}


# ------------------------------------------------------------------ the definitions in 64 bits, written apart

def _mulhilo64(a, m):
    """High and low 32 bits of a * m by 16-bit halves (a: int64 tensor of 32-bit values)."""
    al, ah, ml, mh = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
    mid = ah * ml + (al * ml >> 16)
    mid2 = al * mh + (mid & 0xFFFF)
    return ah * mh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (al * ml & 0xFFFF)


def _mask64(rng, rows, cols, p):
    seed, step = (int(v) for v in rng.cpu())
    col, row = torch.arange(cols, device="cuda"), torch.arange(rows, device="cuda")
    c = [torch.arange(-(-cols // 8), device="cuda")[None, :].expand(rows, -1), row[:, None].expand(-1, -(-cols // 8)),
         torch.tensor(step % 2 ** 32, device="cuda"), torch.tensor(SITE, device="cuda")]
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]
    for r in range(10):
        hi0, lo0 = _mulhilo64(c[0], 0xD2511F53)
        hi1, lo1 = _mulhilo64(c[2], 0xCD9E8D57)
        c = [hi1 ^ c[1] ^ ((key[0] + r * 0x9E3779B9) % 2 ** 32), lo1, hi0 ^ c[3] ^ ((key[1] + r * 0xBB67AE85) % 2 ** 32), lo0]
    bits = torch.empty(rows, cols, dtype=torch.int64, device="cuda")
    for lane in range(8):
        at = col[lane::8]
        bits[:, lane::8] = c[lane // 2][:, at // 8] // 65536 ** (lane % 2) % 65536
    return (bits >= round(65536 * p)).double() * (65536 / (65536 - round(65536 * p)))


def _through64(x, s):
    p = s["case"]["p"]
    if p == 0.0:
        return x
    return x * _mask64(s["rng"], x.numel() // x.shape[-1], x.shape[-1], p).view(x.shape)


def _softmax64(s):
    """Kept probabilities of each pair in 64 bits, the logarithm of the row's sum, and each pair's bucket."""
    c = s["case"]
    q, k = c["q"], c["k"]
    per = {}
    first = _first_distances(c)
    for d in range(-k, q + k + 1):                       # distance query - key
        n = max(d, 0) if c["causal"] else abs(d)
        b = sum(1 for f in first if f <= n) - 1 if n < first[-1] else len(first) - 1
        per[d] = b + (len(first) if d < 0 and not c["causal"] else 0)
    line = torch.tensor([per[d] for d in range(-k, q + k + 1)], device="cuda")
    away = (torch.arange(q, device="cuda") + k - q)[:, None] - torch.arange(k, device="cuda")[None, :]
    bucket = line[away + k]
    keep = torch.ones(c["batch"], 1, q, k, dtype=torch.bool, device="cuda")
    if c["causal"]:
        keep &= away >= 0
    if s["key_len"] is not None:
        keep &= torch.arange(k, device="cuda") < s["key_len"].view(-1, 1, 1, 1)
    logit = s["scores"].double() * s["scale"]
    logit += s["table"].double().t()[:, bucket]
    logit.masked_fill_(~keep, -math.inf)
    lse = torch.logsumexp(logit, -1)
    return logit.sub_(lse[..., None]).exp_(), lse, bucket


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        return {"y": _through64(s["x"].double(), s)}
    if case["op"] == "norm" and not case["back"]:
        h = _through64(s["x"].double(), s)
        if case["fused"]:
            h = h + s["residual"].double()
        var, mean = torch.var_mean(h, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        y = torch.addcmul(s["bias"].double(), (h - mean[:, None]) * rstd[:, None], s["weight"].double())
        out = {"y": y, "mean": mean, "rstd": rstd}
        return {**out, "h": h} if case["fused"] else out
    if case["op"] == "norm":
        # the Jacobian-vector product written out per row: the component along xhat and the mean are taken off g
        n = case["cols"]
        dy, rstd = s["dy"].double(), s["rstd"].double()
        xhat = (s["h"].double() - s["mean"].double()[:, None]) * rstd[:, None]
        g = dy * s["weight"].double()
        along = torch.einsum("rc,rc->r", g, xhat) / n
        dh = (g - torch.outer(g.sum(1) / n, torch.ones(n, dtype=torch.float64, device="cuda")) - xhat * along[:, None])
        dh *= rstd[:, None]
        if case["fused"]:
            dh += s["dh"].double()
        out = {"dx": _through64(dh, s), "dweight": torch.einsum("rc,rc->c", dy, xhat), "dbias": dy.sum(0)}
        return {**out, "dresidual": dh} if case["fused"] else out
    probs, lse, bucket = _softmax64(s)
    if not case["back"]:
        return {"probs": _through64(probs, s), "lse": lse}
    # the rows' statistics are an input of the backward pass
    probs *= torch.exp(lse - s["lse"].double())[..., None]
    dp = _through64(s["dprobs"].double(), s)
    dp -= torch.einsum("bhqk,bhqk->bhq", probs, dp)[..., None]
    ds = probs.mul_(dp)
    over = ds.sum(0).flatten(1)
    dtable = torch.zeros(case["buckets"], case["heads"], dtype=torch.float64, device="cuda")
    dtable.index_add_(0, bucket.flatten(), over.t().contiguous())
    return {"dscores": ds * s["scale"], "dtable": dtable}
