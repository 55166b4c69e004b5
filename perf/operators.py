"""Timed cases of the gradients that a program holds, the relative position bias and the norms of queries and keys.

A case is a dict of plain values; `kind` says what one pass does:

  clip        per-unit gradients of many tensors, [units, ...] each: the squared norm of every unit over all tensors, then
              (`out` = "sum") the clip-weighted sums, on buffers cleared first, or (`out` = "scaled") every unit's gradient scaled
              to the clip norm.  `form` = "stack": the tensors of a transformer stack, "adapters": low-rank pairs beside projections
  bias        a relative position bias [heads, queries, keys] from its table of buckets; the queries are the last positions
  bias_grads  every example's gradient of such a table, shared by `layers` layers, from the gradients of the attention scores
  qk          root-mean-square norm of every head of queries and keys with a gain, and the rotation by position
  qk_grads    its backward: gradients of queries and keys, and every example's gradients of the two gains

`own` false: the plain forms, in elementary torch operations.  `own` true: the calls that a program makes of the library.
"""
import math

import torch

own = False
DEV = "cuda:0"
CLIP = 1.0
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def listed():
    return [
        # the smallest program: the gradient of a single block as one unit; launches and latency are all there is to it
        dict(name="clip_block_f32", kind="clip", form="stack", blocks=1, hidden=64, ffn=256, vocab=0, units=1, dtype="f32", out="sum"),
        # the whole bf16 gradient of one user of a BERT-Large-shaped model, 391 tensors, added to the sum of the step
        dict(name="clip_user_bf16", kind="clip", form="stack", blocks=24, hidden=1024, ffn=4096, vocab=30522, units=1, dtype="bf16", out="sum"),
        # the fp32 gradient of a mid-sized stack, clipped for a program that sends it on or updates without noise
        dict(name="clip_scaled_f32", kind="clip", form="stack", blocks=8, hidden=512, ffn=2048, vocab=30522, units=1, dtype="f32", out="scaled"),
        # per-example gradients of rank-8 adapters beside queries and values of 24 blocks, as a vectorised backward leaves them
        dict(name="clip_adapters_bf16", kind="clip", form="adapters", layers=48, hidden=1024, rank=8, units=128, dtype="bf16", out="sum"),
        # one new token against 513 cached positions
        dict(name="bias_token", kind="bias", heads=16, queries=1, keys=513, per_side=16, reach=128, both=True, dtype="bf16"),
        # the bias of a whole window of 2,048 positions
        dict(name="bias_window", kind="bias", heads=16, queries=2048, keys=2048, per_side=16, reach=128, both=True, dtype="bf16"),
        # the table of 24 encoder layers at the length of the benchmark
        dict(name="bias_grads_128", kind="bias_grads", layers=24, batch=128, heads=16, queries=128, keys=128, per_side=16, reach=128, both=True,
             causal=False, ragged=False, dtype="bf16"),
        # a padded batch of odd length under a causal mask, scores in fp32
        dict(name="bias_grads_ragged", kind="bias_grads", layers=6, batch=24, heads=12, queries=509, keys=509, per_side=32, reach=128, both=False,
             causal=True, ragged=True, dtype="f32"),
        # one new token of 64 sequences, grouped heads, out of a fused projection
        dict(name="qk_token", kind="qk", batch=64, tokens=1, q_heads=32, k_heads=8, width=128, rotated=128, interleaved=False, fused=True, dtype="bf16"),
        # a batch of 32 prompts
        dict(name="qk_prompt", kind="qk", batch=32, tokens=512, q_heads=16, k_heads=16, width=64, rotated=64, interleaved=False, fused=True, dtype="bf16"),
        # the backward of the benchmark's micro-batch: 512 sequences of 128 tokens
        dict(name="qk_grads_large", kind="qk_grads", batch=512, tokens=128, q_heads=16, k_heads=16, width=64, rotated=64, interleaved=False,
             fused=True, dtype="bf16"),
        # fp32, partial rotation of neighbouring pairs, odd length, heads of 80
        dict(name="qk_grads_partial", kind="qk_grads", batch=8, tokens=333, q_heads=12, k_heads=4, width=80, rotated=32, interleaved=True, fused=False,
             dtype="f32"),
    ]


# ---------------------------------------------------------------------------------------------------------------------
# drawn cases
# ---------------------------------------------------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["clip", "clip", "bias", "bias_grads", "bias_grads", "qk", "qk_grads"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "clip":
        c = dict(kind=kind, form=rng.choice(["stack", "adapters"]), dtype=dtype, out=rng.choice(["sum", "sum", "scaled"]))
        if c["form"] == "stack":
            hidden = 8 * _log_int(rng, 4, 128)
            c.update(blocks=_log_int(rng, 1, 24), hidden=hidden, ffn=4 * hidden, vocab=rng.choice([0, _log_int(rng, 500, 30522)]), units=1)
        else:
            c.update(layers=_log_int(rng, 1, 64), hidden=_log_int(rng, 50, 1024), rank=_log_int(rng, 1, 32), units=_log_int(rng, 2, 512))
    elif kind in ("bias", "bias_grads"):
        keys = _log_int(rng, 1, 2048 if kind == "bias" else 1024)
        both = rng.random() < 0.5
        n = rng.choice([4, 8, 16, 32, 64])
        c = dict(kind=kind, heads=_log_int(rng, 1, 32), queries=rng.choice([1, keys, keys, max(1, keys // 3)]), keys=keys, per_side=n,
                 reach=rng.choice([n, 4 * n, 128]), both=both, dtype=dtype)
        if c["reach"] <= n // 2:
            c["reach"] = n
        if kind == "bias_grads":
            c.update(layers=rng.choice([1, 1, 2, 6, 12, 24]), batch=_log_int(rng, 1, 256), causal=not both, ragged=rng.random() < 0.5)
    else:
        width = 8 * rng.randint(2, 32)
        k_heads = _log_int(rng, 1, 16)
        c = dict(kind=kind, batch=_log_int(rng, 1, 256), tokens=rng.choice([1, _log_int(rng, 2, 2048)]), q_heads=k_heads * rng.choice([1, 1, 2, 4]),
                 k_heads=k_heads, width=width, rotated=rng.choice([0, width // 16 * 8, width]), interleaved=rng.random() < 0.3, fused=rng.random() < 0.5,
                 dtype=dtype)
    part = "units" if kind == "clip" else "heads" if kind == "bias" else "batch"
    while work(c)["bytes"] > 1.5e9:
        c[part if c[part] > 1 else "layers" if c.get("layers", 1) > 1 else "blocks"] //= 2
    return c


# ---------------------------------------------------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------------------------------------------------
def _shapes(c):
    """The tensors of a clip case, without their leading axis of units."""
    h = c["hidden"]
    if c["form"] == "adapters":
        return [s for _ in range(c["layers"]) for s in ((h, c["rank"]), (c["rank"], h))]
    f = c["ffn"]
    s = [(c["vocab"], h), (512, h), (h,), (h,)] if c["vocab"] else []
    for _ in range(c["blocks"]):
        s += [(h, h), (h,)] * 4 + [(h,), (h,), (h, f), (f,), (f, h), (h,), (h,), (h,)]
    return s


def _lengths(c):
    """Lengths of a padded batch: from all positions down to a quarter of them, and one empty example if there are three."""
    n, b = c["keys"], c["batch"]
    if not c["ragged"]:
        return [n] * b
    out = [n - (3 * n * i) // (4 * b) for i in range(b)]
    if b >= 3:
        out[1] = 0
    return out


def _places(c):
    """Pairs of a query and a key that count, of one head and all examples."""
    q, k = c["queries"], c["keys"]
    total = 0
    for n in _lengths(c):
        rows = max(0, n - (k - q))  # queries at positions k - q .. n - 1
        total += rows * (k - q) + rows * (rows + 1) // 2 if c["causal"] else rows * n
    return total


def work(c):
    e = SIZE[c["dtype"]]
    if c["kind"] == "clip":
        n = sum(math.prod(s) for s in _shapes(c))
        x = n * c["units"]
        return {"bytes": x * e + (4 * n if c["out"] == "sum" else x * e), "flops": 4 * x}
    if c["kind"] == "bias":
        n = c["heads"] * c["queries"] * c["keys"]
        return {"bytes": n * e, "flops": n}
    if c["kind"] == "bias_grads":
        n = c["layers"] * c["heads"] * _places(c)
        buckets = c["per_side"] * (2 if c["both"] else 1)
        return {"bytes": n * e + 4 * c["batch"] * buckets * c["heads"], "flops": n}
    n = c["batch"] * c["tokens"] * (c["q_heads"] + c["k_heads"]) * c["width"]
    if c["kind"] == "qk":
        return {"bytes": 2 * n * e, "flops": 7 * n}
    return {"bytes": 3 * n * e + 8 * c["batch"] * c["width"], "flops": 16 * n}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _randn(shape, gen):
    return torch.randn(shape, generator=gen, device=DEV)


def _score_grads(c, gen, allowed):
    """Gradients of attention scores, P * (dP - sum P dP), one layer: zero where the mask hides the key, NaN in rows that it leaves empty."""
    shape = (c["batch"], c["heads"], c["queries"], c["keys"])
    scores = _randn(shape, gen).mul_(1.5).masked_fill_(~allowed, -math.inf)
    scores -= scores.amax(-1, keepdim=True)
    p = scores.exp_()
    p /= p.sum(-1, keepdim=True)
    dp = _randn(shape, gen).mul_(1e-2)
    return (p * (dp - (p * dp).sum(-1, keepdim=True))).to(DTYPES[c["dtype"]])


def _allowed(c, lengths):
    """[batch, 1, queries, keys]: the places that count."""
    q = torch.arange(c["queries"], device=DEV) + (c["keys"] - c["queries"])
    k = torch.arange(c["keys"], device=DEV)
    ok = (q[None, :, None] < lengths[:, None, None]) & (k[None, None, :] < lengths[:, None, None])
    if c["causal"]:
        ok = ok & (k[None, None, :] <= q[None, :, None])
    return ok[:, None]


def _inputs(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "clip":
        shapes, u = _shapes(c), c["units"]
        # norms from a fifth of the clip norm to twenty times it, another for every unit
        scale = torch.exp(torch.rand(u, generator=gen, device=DEV) * math.log(100.0)) * 0.2
        scale /= math.sqrt(sum(math.prod(s) for s in shapes))
        return {"X": [(_randn((u, math.prod(s)), gen) * scale[:, None]).to(dt).reshape((u,) + s) for s in shapes]}
    if c["kind"] == "bias":
        return {"table": _randn((c["per_side"] * (2 if c["both"] else 1), c["heads"]), gen)}
    if c["kind"] == "bias_grads":
        order = torch.randperm(c["batch"], generator=gen, device=DEV)
        lengths = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)[order]
        allowed = _allowed(c, lengths)
        return {"dS": [_score_grads(c, gen, allowed) for _ in range(c["layers"])], "lengths": lengths if c["ragged"] else None}
    b, t, hq, hk, d = c["batch"], c["tokens"], c["q_heads"], c["k_heads"], c["width"]
    channel = torch.exp(0.5 * _randn((d,), gen))  # a few channels are larger than the others
    if c["fused"]:  # queries, keys and values of a token next to each other
        qkv = (_randn((b, t, hq + 2 * hk, d), gen) * channel).to(dt)
        s = {"q": qkv[:, :, :hq], "k": qkv[:, :, hq:hq + hk]}
    else:
        s = {"q": (_randn((b, t, hq, d), gen) * channel).to(dt), "k": (_randn((b, t, hk, d), gen) * channel).to(dt)}
    for n in ("gain_q", "gain_k"):
        s[n] = 1 + 0.2 * _randn((d,), gen)
    r = c["rotated"]
    s["cos"] = s["sin"] = s["positions"] = None
    if r:
        most = 4096
        angle = torch.arange(most, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (
            -torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        first = torch.randint(0, most - t + 1, (b, 1), generator=gen, device=DEV)
        s["positions"] = (first + torch.arange(t, device=DEV)).to(torch.int32)
    if c["kind"] == "qk_grads":
        s["dyq"], s["dyk"] = (_randn((b, t, h, d), gen).mul_(1e-2).to(dt) for h in (hq, hk))
    return s


def _starts(c):
    """The first distance of each of a side's buckets: one each up to half of them, then in equal steps of the logarithm up to `reach`."""
    n, exact = c["per_side"], c["per_side"] // 2
    out = list(range(exact))
    d = exact
    for j in range(n - exact):
        # the first d with (d / exact)^(n - exact) >= (reach / exact)^j, in whole numbers
        while d ** (n - exact) * exact ** j < c["reach"] ** j * exact ** (n - exact):
            d += 1
        out.append(d)
    return out


_ctx = None


def _context():
    global _ctx
    if _ctx is None:
        import paper_2108_01624_amd as dp

        _ctx = dp.Context()
    return _ctx


def _places_of(xs, whole):
    """Where the tensors lie in a flat buffer of all units (whole) or of their sums: each from a multiple of 8 numbers on, zeros between."""
    at = [0]
    for x in xs:
        at.append(at[-1] + ((x if whole else x[0]).numel() + 7) // 8 * 8)
    return at[:-1], at[-1]


def prepare(case, seed):
    c, s = case, _inputs(case, seed)
    s["case"] = c
    dt = DTYPES[c["dtype"]]
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEV)
    if c["kind"] == "clip":
        s["sqnorms"] = new(c["units"])
        # one flat buffer of all sums, as the update takes it, or of all scaled gradients
        at, end = _places_of(s["X"], c["out"] == "scaled")
        if c["out"] == "sum":
            s["S"] = new(end)
            s["sums"] = [s["S"][o:o + x[0].numel()].view(x[0].shape) for o, x in zip(at, s["X"])]
        else:
            s["flat"] = torch.zeros(end, dtype=dt, device=DEV)
            s["Y"] = [s["flat"][o:o + x.numel()].view(x.shape) for o, x in zip(at, s["X"])]
    elif c["kind"].startswith("bias"):
        buckets = c["per_side"] * (2 if c["both"] else 1)
        if c["kind"] == "bias":
            s["bias"] = new(c["heads"], c["queries"], c["keys"], dtype=dt)
        else:
            s["grads"] = new(c["batch"], buckets, c["heads"])
        s["starts"] = _starts(c)
    elif c["kind"] == "qk":
        s["yq"], s["yk"] = (new(c["batch"], c["tokens"], h, c["width"], dtype=dt) for h in (c["q_heads"], c["k_heads"]))
    else:
        s["grads"] = new(c["batch"], 2, c["width"])
        if c["fused"]:  # the gradient of the fused projection's output; the values' part is another operator's
            d_qkv = torch.zeros((c["batch"], c["tokens"], c["q_heads"] + 2 * c["k_heads"], c["width"]), dtype=dt, device=DEV)
            s["dq"], s["dk"] = d_qkv[:, :, :c["q_heads"]], d_qkv[:, :, c["q_heads"]:c["q_heads"] + c["k_heads"]]
        else:
            s["dq"], s["dk"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    if own:
        import paper_2108_01624_amd as dp

        _context()
        if "starts" in s:
            s["starts"] = dp.dp_relative_buckets(c["per_side"], c["reach"])
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["kind"]](state)


def _own_clip(s):
    ctx = _context()
    ctx.zero_f32(s["sqnorms"])
    ctx.sqnorms_grads(s["X"], s["sqnorms"])
    if "Y" in s:
        ctx.clip_grads(s["X"], CLIP, s["sqnorms"], s["Y"])
        return {"sqnorms": s["sqnorms"], "Y": s["flat"]}
    ctx.zero_f32(s["S"])
    ctx.clip_accumulate_grads(s["X"], CLIP, s["sqnorms"], s["sums"])
    return {"sqnorms": s["sqnorms"], "S": s["S"]}


def _own_bias(s):
    _context().relative_bias(s["table"], s["starts"], s["case"]["both"], s["bias"])
    return {"bias": s["bias"]}


def _own_bias_grads(s):
    c = s["case"]
    _context().relative_bias_grads(s["dS"], s["starts"], c["both"], s["grads"], lengths=s["lengths"], causal=c["causal"])
    return {"grads": s["grads"]}


def _own_qk(s):
    _context().qk_norm(s["q"], s["k"], s["gain_q"], s["gain_k"], s["cos"], s["sin"], s["yq"], s["yk"], positions=s["positions"],
                       interleaved=s["case"]["interleaved"], eps=EPS)
    return {"yq": s["yq"], "yk": s["yk"]}


def _own_qk_grads(s):
    _context().qk_norm_grads(s["q"], s["k"], s["gain_q"], s["gain_k"], s["cos"], s["sin"], s["dyq"], s["dyk"], s["grads"], s["dq"], s["dk"],
                             positions=s["positions"], interleaved=s["case"]["interleaved"], eps=EPS)
    return {"dq": s["dq"], "dk": s["dk"], "grads": s["grads"]}


_own = {"clip": _own_clip, "bias": _own_bias, "bias_grads": _own_bias_grads, "qk": _own_qk, "qk_grads": _own_qk_grads}


def _plain_clip(s):
    u = s["case"]["units"]
    rows = [x.reshape(u, -1).float() for x in s["X"]]
    n = torch.zeros(u, device=DEV)
    for x in rows:
        n = n + (x * x).sum(1)
    f = torch.where(n > 0, (CLIP / n.sqrt()).clamp(max=1.0), torch.ones_like(n))
    if "Y" in s:
        for x, out in zip(rows, s["Y"]):
            out.copy_((x * f[:, None]).reshape(out.shape))
        return {"sqnorms": n, "Y": s["flat"]}
    s["S"].zero_()
    for x, out in zip(rows, s["sums"]):
        out += (x * f[:, None]).sum(0).reshape(out.shape)
    return {"sqnorms": n, "S": s["S"]}


def _buckets(c, starts, rel):
    """The bucket of a key `rel` positions behind its query (negative: in front of it)."""
    starts = torch.tensor(starts, device=DEV)
    dist = rel.abs() if c["both"] else (-rel).clamp(min=0)
    b = (dist[..., None] >= starts).sum(-1) - 1
    return b + c["per_side"] * (rel > 0) if c["both"] else b


def _plain_bias(s):
    c = s["case"]
    q = torch.arange(c["queries"], device=DEV) + (c["keys"] - c["queries"])
    rel = torch.arange(c["keys"], device=DEV)[None, :] - q[:, None]
    return {"bias": s["table"][_buckets(c, s["starts"], rel)].permute(2, 0, 1).contiguous().to(DTYPES[c["dtype"]])}


def _plain_bias_grads(s):
    c = s["case"]
    b, h, q, k = c["batch"], c["heads"], c["queries"], c["keys"]
    total = torch.zeros((b, h, q, k), device=DEV)
    for x in s["dS"]:
        total += x
    if c["causal"] or s["lengths"] is not None:
        lengths = s["lengths"] if s["lengths"] is not None else torch.full((b,), k, device=DEV)
        total = torch.where(_allowed(c, lengths), total, torch.zeros((), device=DEV))
    # every row one to the left of the row above it: written in rows of k + q - 1 numbers, read behind q - 1 zeros in rows of k + q
    wide = torch.nn.functional.pad(total, (0, q - 1)).reshape(b, h, -1)
    lines = torch.nn.functional.pad(wide, (q - 1, 1)).reshape(b, h, q, k + q)[..., :-1].sum(2)
    idx = _buckets(c, s["starts"], torch.arange(k + q - 1, device=DEV) - (k - 1))  # (column j: the keys j - (k - 1) behind their query)
    n = c["per_side"] * (2 if c["both"] else 1)
    out = torch.zeros((b, h, n), device=DEV)
    for j in range(n):
        out[..., j] = lines[..., idx == j].sum(-1)
    return {"grads": out.transpose(1, 2).contiguous()}


def _pairs(x, c):
    """The two halves of the numbers that are rotated together."""
    r = c["rotated"]
    return (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])


def _rotated(x, c, cos, sin):
    r = c["rotated"]
    if not r:
        return x
    a, b = _pairs(x, c)
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _angles(s):
    if s["cos"] is None:
        return None, None
    p = s["positions"].long()
    return s["cos"][p][:, :, None], s["sin"][p][:, :, None]


def _plain_qk(s):
    c, out = s["case"], {}
    cos, sin = _angles(s)
    for n in ("q", "k"):
        x = s[n].float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["gain_" + n]
        out["y" + n] = _rotated(x, c, cos, sin).to(DTYPES[c["dtype"]])
    return out


def _plain_qk_grads(s):
    c, out, gains = s["case"], {}, []
    cos, sin = _angles(s)
    for n in ("q", "k"):
        x = s[n].float()
        inv = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        x = x * inv
        u = _rotated(s["dy" + n].float(), c, cos, None if sin is None else -sin)
        gains.append((u * x).sum((1, 2)))
        u = u * s["gain_" + n]
        out["d" + n] = (inv * (u - x * (u * x).mean(-1, keepdim=True))).to(DTYPES[c["dtype"]])
    out["grads"] = torch.stack(gains, 1)
    return out


_plain = {"clip": _plain_clip, "bias": _plain_bias, "bias_grads": _plain_bias_grads, "qk": _plain_qk, "qk_grads": _plain_qk_grads}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "clip":
        n = torch.zeros(c["units"], dtype=torch.float64, device=DEV)
        for x in s["X"]:
            n += x.double().flatten(1).square().sum(1)
        f = torch.minimum(torch.ones_like(n), CLIP * n.rsqrt())
        f[n == 0] = 1.0
        at, end = _places_of(s["X"], c["out"] == "scaled")
        out = torch.zeros(end, dtype=torch.float64, device=DEV)
        for o, x in zip(at, s["X"]):
            y = f @ x.double().flatten(1) if c["out"] == "sum" else (x.double().flatten(1) * f[:, None]).flatten()
            out[o:o + y.numel()] = y
        return {"sqnorms": n, "S" if c["out"] == "sum" else "Y": out}
    if c["kind"].startswith("bias"):
        # buckets as runs of distances, the last one open
        n, q, k = c["per_side"], c["queries"], c["keys"]
        edges = _starts(c) + [1 << 40]
        at = torch.arange(k, device=DEV)[None, :] - torch.arange(k - q, k, device=DEV)[:, None]
        member = []
        for side in (-1, 1) if c["both"] else (-1,):
            d = side * at if c["both"] else (-at).clamp(min=0)
            for j in range(n):
                here = (d >= edges[j]) & (d < edges[j + 1])
                member.append(here & (at > 0) if side == 1 else here & (at <= 0) if c["both"] else here)
        if c["kind"] == "bias":
            out = torch.zeros((c["heads"], q, k), dtype=torch.float64, device=DEV)
            for j, here in enumerate(member):
                out += torch.where(here, s["table"][j].double()[:, None, None], out.new_zeros(()))
            return {"bias": out}
        total = torch.zeros((c["batch"], c["heads"], q, k), dtype=torch.float64, device=DEV)
        for x in s["dS"]:
            total += x.double()
        if s["lengths"] is not None:
            rows, cols = torch.arange(k - q, k, device=DEV), torch.arange(k, device=DEV)
            for i, n_i in enumerate(s["lengths"].tolist()):
                total[i, :, rows >= n_i] = 0
                total[i, :, :, cols >= n_i] = 0
        if c["causal"]:
            total.masked_fill_(at > 0, 0.0)
        return {"grads": torch.stack([total.masked_fill(~here, 0.0).sum((2, 3)) for here in member], 1)}
    # queries and keys: the definition of the forward, and its derivatives by automatic differentiation; complex numbers turn the pairs
    out, gains = {}, []
    r = c["rotated"]
    for n in ("q", "k"):
        grad = c["kind"] == "qk_grads"
        x = s[n].double().contiguous().requires_grad_(grad)
        g = s["gain_" + n].double().expand(c["batch"], 1, 1, -1).contiguous().requires_grad_(grad)
        y = x / (x.pow(2).sum(-1, keepdim=True) / c["width"] + EPS).sqrt() * g
        if r:
            turn = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"].long()].unsqueeze(2)
            if c["interleaved"]:
                z = torch.view_as_real(torch.view_as_complex(y[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * turn).flatten(-2)
            else:
                w = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
                z = torch.cat([w.real, w.imag], -1)
            y = torch.cat([z, y[..., r:]], -1)
        if not grad:
            out["y" + n] = y
            continue
        dx, dg = torch.autograd.grad(y, (x, g), s["dy" + n].double())
        out["d" + n] = dx
        gains.append(dg.reshape(c["batch"], -1))
    if gains:
        out["grads"] = torch.stack(gains, 1)
    return out
