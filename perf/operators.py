"""Operators of a token block behind the early layers: layer norm over channels, softmax attention with its backward
pass, and activation checkpoints in 8 bits with what the backward pass computes from them.

A case names one pass through one operator ("op"):

  norm_forward          y, mean, rstd of rows of channels; x as token rows or as an NCHW map, y as rows or as a map
  norm_backward         dx, dgamma, dbeta; x in its own type or as an 8-bit checkpoint
  attention_forward     out and the log-sums; grouped heads, lengths, causal or not; one query of a long cache too
  attention_backward    dq, dk, dv from dout, with the probabilities recomputed
  checkpoint            pack to 8 bits and unpack again, through an activation if one is named
  checkpoint_act        dx = dy f'(x) with x from the checkpoint
  checkpoint_wgrad      dW = dy^T x with x from the checkpoint

Where `own` is false the formulas run as plain torch operations in 32 bits.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_ES = {"f32": 4, "bf16": 2}


def _norm(name, op, outer, inner, channels, dtype, x="rows", y="rows", pad=0, block=0):
    """x, y: "rows" ([outer][inner][channels]) or "map" ([outer][channels][inner]); pad: unused channels behind each row of x;
    block: x is a checkpoint with blocks of that many channels (0: x itself)."""
    return _named(name, {"op": op, "outer": outer, "inner": inner, "channels": channels, "dtype": dtype, "x": x, "y": y,
                         "pad": pad, "block": block})


def _attention(name, op, batch, heads, kv_heads, q_len, kv_len, dim, dtype, causal=False, ragged=False, packed=False):
    """ragged: every image has lengths of its own (see _lengths); packed: q, k, v are slices of one tensor."""
    return _named(name, {"op": op, "batch": batch, "heads": heads, "kv_heads": kv_heads, "q_len": q_len, "kv_len": kv_len,
                         "dim": dim, "dtype": dtype, "causal": causal, "ragged": ragged, "packed": packed})


def _check(name, op, rows, cols, block, dtype, act="none", n=0):
    """n: outputs of the linear layer whose weight gradient is taken (checkpoint_wgrad)."""
    return _named(name, {"op": op, "rows": rows, "cols": cols, "block": block, "dtype": dtype, "act": act, "n": n})


def _named(name, c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # Serving: four tokens, one from each of four streams, through a norm; all latency.
        _norm("norm_tokens_bf16", "norm_forward", 4, 1, 256, "bf16"),
        # The early layers' output map (16 images of 76 x 76) read as a map, normalised and written as token rows.
        _norm("norm_map_to_tokens_f32", "norm_forward", 16, 5776, 128, "f32", x="map"),
        # Training, 64 images of 38 x 38 tokens, 512 channels: dx and both parameter gradients.
        _norm("norm_backward_bf16", "norm_backward", 64, 1444, 512, "bf16"),
        # The same from an 8-bit checkpoint of x; odd everything: 13 images of 37 x 37, 250 channels.
        _norm("norm_backward_checkpoint_f32", "norm_backward", 13, 1369, 250, "f32", block=64),
        # What a first pooled block hands on, kept in 8 bits between forward and backward: 64 images, 32 channels of 304 x 304.
        _check("checkpoint_maps_f32", "checkpoint", 2048, 92416, 128, "f32"),
        # GELU's derivative from the checkpoint of a 1024-wide hidden layer, 32 images of 38 x 38 tokens.
        _check("checkpoint_gelu_bf16", "checkpoint_act", 46208, 1024, 128, "bf16", "gelu"),
        # Weight gradient of a 512 -> 1024 linear layer on the same tokens, its input kept in 8 bits.
        _check("checkpoint_wgrad_bf16", "checkpoint_wgrad", 46208, 512, 128, "bf16", n=1024),
        # A small one on ragged sizes, 32-bit.
        _check("checkpoint_wgrad_odd_f32", "checkpoint_wgrad", 4995, 202, 32, "f32", n=133),
        # Serving: one new token of 8 streams against caches of up to 8192 tokens, 16 heads on 4.
        _attention("attention_token_bf16", "attention_forward", 8, 16, 4, 1, 8192, 128, "bf16", causal=True, ragged=True),
        # Prompts of up to 2704 tokens (52 x 52), 8 heads of 128 on 2.
        _attention("attention_prompt_bf16", "attention_forward", 4, 8, 2, 2704, 2704, 128, "bf16", causal=True, ragged=True),
        # Training on 76 x 76 tokens, every token sees every other: the largest case.
        _attention("attention_backward_bf16", "attention_backward", 8, 8, 8, 5776, 5776, 64, "bf16", packed=True),
        # Training in 32 bits, odd lengths, shared heads, causal, a head size off the powers of two.
        _attention("attention_backward_odd_f32", "attention_backward", 3, 6, 2, 577, 701, 40, "f32", causal=True, ragged=True),
    ]


def _lengths(case):
    """Query and key lengths of every image; a function of the case alone."""
    b, ql, kl = case["batch"], case["q_len"], case["kv_len"]
    if not case["ragged"]:
        return [ql] * b, [kl] * b
    ks = [max(1, kl - (i * 7919) % (kl // 2 + 1)) for i in range(b)]
    qs = [max(1, ql - (i * 7919) % (ql // 2 + 1)) for i in range(b)]
    return qs, ks


def _pairs(case):
    """Pairs of a query and a key it sees, over the batch, for one head."""
    total = 0
    for ql, kl in zip(*_lengths(case)):
        if not case["causal"]:
            total += ql * kl
            continue
        off = kl - ql                                   # query i sees keys 0 .. i + off
        first = max(0, -off)                            # the first query that sees any
        n = ql - first
        total += n * (first + off + 1) + n * (n - 1) // 2
    return total


def work(case):
    op = case["op"]
    es = _ES[case["dtype"]]
    if op.startswith("norm"):
        rows, c = case["outer"] * case["inner"], case["channels"]
        n = rows * c
        if op == "norm_forward":
            return {"bytes": float(2 * n * es + 2 * c * es + 8 * rows), "flops": 8.0 * n}
        x = n * es if not case["block"] else n + rows * -(-c // case["block"])
        return {"bytes": float(2 * n * es + x + 8 * rows + c * es + 8 * c), "flops": 16.0 * n}
    if op.startswith("attention"):
        pairs, d = _pairs(case), case["dim"]
        ql, kl = _lengths(case)
        q = sum(ql) * case["heads"] * d * es
        kv = sum(kl) * case["kv_heads"] * d * es
        lse = sum(ql) * case["heads"] * 4
        if op == "attention_forward":
            return {"bytes": float(2 * q + 2 * kv + lse), "flops": 4.0 * pairs * case["heads"] * d}
        return {"bytes": float(4 * q + 4 * kv + lse), "flops": 10.0 * pairs * case["heads"] * d}
    n = case["rows"] * case["cols"]
    held = n + case["rows"] * -(-case["cols"] // case["block"])
    if op == "checkpoint":
        return {"bytes": float(2 * n * es + 2 * held), "flops": 8.0 * n}
    if op == "checkpoint_act":
        return {"bytes": float(2 * n * es + held), "flops": 20.0 * n}
    return {"bytes": float(held + case["rows"] * case["n"] * es + 4 * case["n"] * case["cols"]),
            "flops": 2.0 * n * case["n"]}


# ---- drawn cases ---------------------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    wk = work(case)
    rate = 3e14 if case["dtype"] == "bf16" else 6e13
    return wk["flops"] / rate + wk["bytes"] / 3e12


_LARGEST = None


def draw(rng):
    """One case of the listed ones' ranges: 1 to 92416 tokens of 8 to 1100 channels, up to 8192 tokens of attention with heads
    of 8 to 128, checkpoints of up to 190 million values."""
    global _LARGEST
    if _LARGEST is None:
        _LARGEST = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("norm_forward", "norm_backward", "attention_forward", "attention_forward", "attention_backward",
                         "attention_backward", "checkpoint", "checkpoint_act", "checkpoint_wgrad"))
        dtype = rng.choice(("f32", "bf16", "bf16"))
        if op.startswith("norm"):
            c = _log(rng, 8, 1100)
            c = rng.choice((c, max(8, c // 8 * 8), max(32, c // 32 * 32)))
            outer, inner = _log(rng, 1, 64), _log(rng, 1, 5776)
            x = y = "rows"
            pad = block = 0
            if rng.random() < 0.35:
                x, y = "map", rng.choice(("map", "rows"))
            elif op == "norm_backward" and rng.random() < 0.4:
                block = rng.choice((32, 64, 128))
            elif rng.random() < 0.3:
                pad = rng.choice((8, 24, c))
            case = _norm(None, op, outer, inner, c, dtype, x, y, pad, block)
            if 4 * outer * inner * c > 1e9:
                continue
        elif op.startswith("attention"):
            kv = rng.choice((1, 1, 2, 4, 8))
            heads = kv * rng.choice((1, 1, 2, 4, 8))
            dim = rng.choice((8 * rng.randint(1, 16), 32, 64, 64, 128, 128))
            batch = _log(rng, 1, 16)
            kv_len = _log(rng, 1, 8192)
            q_len = kv_len if rng.random() < 0.6 else _log(rng, 1, kv_len)
            if op == "attention_forward" and rng.random() < 0.25:
                q_len = 1
            causal, ragged = rng.random() < 0.5, rng.random() < 0.5
            packed = q_len == kv_len and rng.random() < 0.4
            case = _attention(None, op, batch, heads, kv, q_len, kv_len, dim, dtype, causal, ragged, packed)
            if batch * heads * q_len * kv_len > 2.2e9:
                continue
        else:
            block = rng.choice((32, 64, 128, 256))
            if op == "checkpoint_wgrad":
                rows, cols, n = _log(rng, 64, 92416), _log(rng, 16, 1024), _log(rng, 16, 1024)
                if rng.random() < 0.5:
                    cols, n = max(16, cols // 16 * 16), max(16, n // 16 * 16)
                case = _check(None, op, rows, cols, block, dtype, n=n)
            else:
                rows, cols = _log(rng, 1, 46208), _log(rng, 16, 92416)
                act = rng.choice(("leaky", "gelu", "silu") if op == "checkpoint_act" else ("none", "none", "leaky", "gelu", "silu"))
                case = _check(None, op, rows, cols, block, dtype, act)
                if rows * cols > 190e6:
                    continue
        if _cost(case) <= _LARGEST:
            return case


# ---- inputs --------------------------------------------------------------------------------------------------------
_SLOPE = 0.1
_EPS = 1e-5


def _normal(g, shape, std=1.0, mean=0.0):
    return torch.empty(shape, device="cuda").normal_(mean, std, generator=g)


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _DT[case["dtype"]]
    op = case["op"]
    if op.startswith("norm"):
        b, p, c = case["outer"], case["inner"], case["channels"]
        spread = torch.exp(_normal(g, (c,), 0.5))                     # channels of different sizes, off centre
        x = (_normal(g, (b, p, c + case["pad"]))[:, :, :c] * spread + 0.3 * spread).to(dt)
        if case["x"] == "map":
            x = x.transpose(1, 2).contiguous().transpose(1, 2)
        elif case["pad"]:
            wide = torch.zeros((b, p, c + case["pad"]), device="cuda", dtype=dt)
            wide[:, :, :c] = x
            x = wide[:, :, :c]
        t = {"x": x, "gamma": _normal(g, (c,), 0.2, 1.0).to(dt), "beta": _normal(g, (c,), 0.2).to(dt)}
        if op == "norm_backward":
            dy = _normal(g, (b, p, c)).to(dt)
            t["dy"] = dy if case["y"] == "rows" else dy.transpose(1, 2).contiguous().transpose(1, 2)
            # the statistics that the forward pass left, of x before any checkpoint
            x32 = x.float()
            t["mean"] = x32.mean(2)
            t["rstd"] = torch.rsqrt(((x32 - t["mean"][:, :, None]) ** 2).mean(2) + _EPS)
            if case["block"]:
                t["codes"], t["exponents"] = _pack(x.reshape(b * p, c), case["block"])
        return t
    if op.startswith("attention"):
        b, h, kv, ql, kl, d = (case[k] for k in ("batch", "heads", "kv_heads", "q_len", "kv_len", "dim"))
        if case["packed"]:
            all_ = _normal(g, (b, ql, h + 2 * kv, d)).to(dt)
            q, k, v = all_[:, :, :h], all_[:, :, h:h + kv], all_[:, :, h + kv:]
        else:
            q, k, v = (_normal(g, s).to(dt) for s in ((b, ql, h, d), (b, kl, kv, d), (b, kl, kv, d)))
        t = {"q": q, "k": k, "v": v, "q_lens": None, "kv_lens": None}
        if case["ragged"]:
            t["q_lens"], t["kv_lens"] = (torch.tensor(n, dtype=torch.int32, device="cuda") for n in _lengths(case))
        if op == "attention_backward":
            t["dout"] = _normal(g, (b, ql, h, d)).to(dt)
        return t
    rows, cols = case["rows"], case["cols"]
    # activations: a few large values in each row's neighbourhood, none or both signs after the layer
    x = _normal(g, (rows, cols))
    x.mul_(torch.exp(_normal(g, (rows, 1), 0.5)))
    t = {}
    if op == "checkpoint":
        t["x"] = x.to(dt)
        return t
    t["codes"], t["exponents"] = _pack(x.to(dt), case["block"])
    del x
    t["dy"] = _normal(g, (rows, case["n"] if op == "checkpoint_wgrad" else cols)).to(dt)
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    op = case["op"]
    state = {"case": case, "t": t}
    if not own:
        return state
    from paper_2409_09083_amd import tokens
    if op.startswith("norm"):
        state["norm"] = tokens.Norm(case["outer"], case["inner"], case["channels"], case["dtype"], eps=_EPS,
                                    y_layout=case["y"], x_layout=case["x"])
        if case["block"]:
            state["ckpt"] = tokens.Checkpoint(case["outer"] * case["inner"], case["channels"], case["dtype"], case["block"])
    elif op.startswith("attention"):
        at = tokens.Attention(case["batch"], case["heads"], case["kv_heads"], case["q_len"], case["kv_len"], case["dim"],
                              case["dtype"], causal=case["causal"], training=op == "attention_backward")
        if op == "attention_backward":                  # what the forward pass leaves for the backward pass
            at.forward(t["q"], t["k"], t["v"], t["q_lens"], t["kv_lens"])
        state["attention"] = at
    else:
        state["ckpt"] = tokens.Checkpoint(case["rows"], case["cols"], case["dtype"], case["block"], outputs=case["n"])
    if "ckpt" in state and "codes" in t:
        state["ckpt"].codes.copy_(t["codes"])
        state["ckpt"].exponents.copy_(t["exponents"])
    return state


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _power(e):
    """2^e in 32 bits for -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _blocks(x, block):
    rows, cols = x.shape
    nb = -(-cols // block)
    if nb * block == cols:
        return x.reshape(rows, nb, block)
    full = torch.zeros((rows, nb * block), device=x.device, dtype=x.dtype)
    full[:, :cols] = x
    return full.view(rows, nb, block)


def _pack(x, block):
    """Codes and exponents of [rows][cols]: per block of a row the smallest e >= -126 with max|x| <= 127 * 2^e, and x / 2^e rounded
    to the nearest whole number, ties to even.  At e = 122 codes stop at 63, so that no value that they stand for passes the
    largest finite one.  A block with an infinity or a NaN has e = 127 and codes 0, and stands for NaN in all its places."""
    cols = x.shape[1]
    v = _blocks(x.float(), block)
    amax = v.abs().amax(2)
    bad = ~(v.abs() < math.inf).all(2)
    m, p = torch.frexp(torch.where(bad, torch.zeros_like(amax), amax))
    e = torch.where(m > 0.9921875, p - 6, p - 7)
    e = torch.where(m == 0, torch.full_like(e, -126), e).clamp(-126, 122)
    top = torch.where(e == 122, 63.0, 127.0)[:, :, None]
    q = torch.round(v * _power(-e)[:, :, None])
    q = torch.minimum(torch.maximum(q, -top), top)
    q = torch.where(bad[:, :, None], torch.zeros_like(q), q)
    e = torch.where(bad, torch.full_like(e, 127), e)
    return q.to(torch.int8).reshape(x.shape[0], -1)[:, :cols].contiguous(), e.to(torch.int8)


def _unpack(codes, e, block):
    scale = torch.where(e == 127, torch.full(e.shape, math.nan, device=e.device), _power(e))
    return (_blocks(codes.float(), block) * scale[:, :, None]).reshape(codes.shape[0], -1)[:, :codes.shape[1]]


def _act(x, act):
    if act == "leaky":
        return torch.where(x > 0, x, x * _SLOPE)
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _act_derivative(x, act):
    if act == "leaky":
        return torch.where(x > 0, 1.0, _SLOPE)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-x))
    return s * (1 + x * (1 - s))


def _visible(case, t):
    """[images][q_len][kv_len]: query i sees key j."""
    b, dev = case["batch"], "cuda"
    ql = torch.full((b,), case["q_len"], device=dev) if t["q_lens"] is None else t["q_lens"]
    kl = torch.full((b,), case["kv_len"], device=dev) if t["kv_lens"] is None else t["kv_lens"]
    i = torch.arange(case["q_len"], device=dev)[None, :, None]
    j = torch.arange(case["kv_len"], device=dev)[None, None, :]
    seen = (i < ql[:, None, None]) & (j < kl[:, None, None])
    if case["causal"]:
        seen = seen & (j <= i + (kl - ql)[:, None, None])
    return seen


def _heads(x):
    """[images][tokens][heads][d] -> [images][heads][tokens][d] in 32 bits."""
    return x.float().transpose(1, 2).contiguous()


def _plain_attention(case, t):
    b, h, kv, ql, kl, d = (case[k] for k in ("batch", "heads", "kv_heads", "q_len", "kv_len", "dim"))
    dt = _DT[case["dtype"]]
    scale = 1 / math.sqrt(d)
    q, k, v = _heads(t["q"]).view(b, kv, -1, d), _heads(t["k"]), _heads(t["v"])      # the heads that share one lie behind each other
    s = torch.matmul(q, k.transpose(2, 3)).view(b, h, ql, kl) * scale
    s = torch.where(_visible(case, t)[:, None], s, -math.inf)
    m = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = p.sum(3, keepdim=True)
    lse = (m + torch.log(total)).squeeze(3)
    p = (p / torch.where(total == 0, torch.ones_like(total), total)).view(b, kv, -1, kl)
    if case["op"] == "attention_forward":
        out = torch.matmul(p, v).view(b, h, ql, d)
        return {"out": out.transpose(1, 2).to(dt).contiguous(), "lse": lse}
    del s
    do = _heads(t["dout"]).view(b, kv, -1, d)
    dv = torch.matmul(p.transpose(2, 3), do)
    dp = torch.matmul(do, v.transpose(2, 3))
    ds = p * (dp - (p * dp).sum(3, keepdim=True))
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(2, 3), q) * scale
    return {n: x.transpose(1, 2).to(dt).contiguous() for n, x in (("dq", dq.view(b, h, ql, d)), ("dk", dk), ("dv", dv))}


def _plain_norm(case, t):
    dt = _DT[case["dtype"]]
    g = t["gamma"].float()
    if case["op"] == "norm_forward":
        x = t["x"].float()
        mean = x.mean(2, keepdim=True)
        rstd = torch.rsqrt(((x - mean) ** 2).mean(2, keepdim=True) + _EPS)
        y = ((x - mean) * rstd * g + t["beta"].float()).to(dt)
        if case["y"] == "map":
            y = y.transpose(1, 2).contiguous()
        return {"y": y.contiguous(), "mean": mean.squeeze(2), "rstd": rstd.squeeze(2)}
    x = _unpack(t["codes"], t["exponents"], case["block"]).view(t["dy"].shape) if case["block"] else t["x"].float()
    dy = t["dy"].float()
    rstd = t["rstd"][:, :, None]
    xh = (x - t["mean"][:, :, None]) * rstd
    a = dy * g
    dx = rstd * (a - a.mean(2, keepdim=True) - xh * (a * xh).mean(2, keepdim=True))
    dx = dx.to(dt)
    if case["x"] == "map":
        dx = dx.transpose(1, 2)
    return {"dx": dx.contiguous(), "dgamma": (dy * xh).sum((0, 1)), "dbeta": dy.sum((0, 1))}


def _plain_checkpoint(case, t):
    dt = _DT[case["dtype"]]
    if case["op"] == "checkpoint":
        codes, e = _pack(t["x"], case["block"])
        return {"x": _act(_unpack(codes, e, case["block"]), case["act"]).to(dt), "exponents": e}
    x = _unpack(t["codes"], t["exponents"], case["block"])
    if case["op"] == "checkpoint_act":
        return {"dx": (t["dy"].float() * _act_derivative(x, case["act"])).to(dt)}
    return {"dw": torch.matmul(t["dy"].float().t(), x)}


def run(state):
    case, t = state["case"], state["t"]
    op = case["op"]
    if not own:
        if op.startswith("norm"):
            return _plain_norm(case, t)
        if op.startswith("attention"):
            return _plain_attention(case, t)
        return _plain_checkpoint(case, t)
    if op == "norm_forward":
        n = state["norm"]
        n.forward(t["x"], t["gamma"], t["beta"])
        return {"y": n.y_buffer, "mean": n.mean, "rstd": n.rstd}
    if op == "norm_backward":
        n = state["norm"]
        n.backward(t["dy"], state["ckpt"] if case["block"] else t["x"], t["gamma"], t["mean"], t["rstd"])
        return {"dx": n.dx_buffer, "dgamma": n.dgamma, "dbeta": n.dbeta}
    if op == "attention_forward":
        a = state["attention"]
        a.forward(t["q"], t["k"], t["v"], t["q_lens"], t["kv_lens"])
        return {"out": a.out, "lse": a.lse}
    if op == "attention_backward":
        a = state["attention"]
        a.backward(t["dout"], t["q"], t["k"], t["v"], t["q_lens"], t["kv_lens"])
        return {"dq": a.dq, "dk": a.dk, "dv": a.dv}
    c = state["ckpt"]
    if op == "checkpoint":
        c.pack(t["x"])
        return {"x": c.unpack(act=case["act"], slope=_SLOPE), "exponents": c.exponents}
    if op == "checkpoint_act":
        return {"dx": c.act_backward(t["dy"], act=case["act"], slope=_SLOPE)}
    return {"dw": c.wgrad(t["dy"])}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def _exact_values(x, block):
    """What a checkpoint of x stands for, and its exponents: the smallest e is looked for from below."""
    rows, cols = x.shape
    out = torch.empty((rows, cols), dtype=torch.float64, device=x.device)
    exps = torch.empty((rows, -(-cols // block)), dtype=torch.int8, device=x.device)
    for i in range(exps.shape[1]):
        v = x[:, i * block:(i + 1) * block].double()
        top = v.abs().max(1).values
        e = torch.floor(torch.log2(torch.clamp(top, min=2.0 ** -200) / 127)) - 2
        for _ in range(4):
            e = torch.where(top > 127 * torch.exp2(e), e + 1, e)
        e = torch.clamp(e, -126, 122)
        unit = torch.exp2(e)[:, None]
        most = torch.where(e == 122, 63.0, 127.0).double()[:, None]
        out[:, i * block:(i + 1) * block] = torch.clamp(torch.round(v / unit), -most, most) * unit
        exps[:, i] = e.to(torch.int8)
    return out, exps


def _exact_held(codes, exponents, block):
    unit = torch.exp2(exponents.double())
    return codes.double() * torch.repeat_interleave(unit, block, 1)[:, :codes.shape[1]]


def _exact_act(x, act, derivative):
    if act == "none":
        return x
    if act == "leaky":
        unit = torch.where(x > 0, torch.ones_like(x), torch.full_like(x, _SLOPE))
        return unit if derivative else x * unit
    if act == "gelu":
        phi = torch.special.ndtr(x)
        return phi + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi) if derivative else x * phi
    s = torch.sigmoid(x)
    return s + x * s * torch.sigmoid(-x) if derivative else x * s


def _exact_attention(case, t):
    b, h, kv, ql, kl, d = (case[k] for k in ("batch", "heads", "kv_heads", "q_len", "kv_len", "dim"))
    backward = case["op"] == "attention_backward"
    g = h // kv
    new = lambda *s: torch.zeros(s, dtype=torch.float64, device="cuda")     # noqa: E731
    out, lse = new(b, ql, h, d), new(b, h, ql) - math.inf
    dq, dk, dv = new(b, ql, h, d), new(b, kl, kv, d), new(b, kl, kv, d)
    for n, (qn, kn) in enumerate(zip(*_lengths(case))):
        for j in range(h):
            q, k, v = t["q"][n, :qn, j].double(), t["k"][n, :kn, j // g].double(), t["v"][n, :kn, j // g].double()
            s = (q @ k.t().contiguous()) / math.sqrt(d)
            if case["causal"]:
                late = torch.ones((qn, kn), dtype=torch.bool, device="cuda").triu(kn - qn + 1)
                s = s.masked_fill(late, -math.inf)
            total = torch.logsumexp(s, 1)
            p = torch.nan_to_num(torch.exp(s - total[:, None]))           # a query that sees nothing: no probabilities
            o = p @ v
            out[n, :qn, j], lse[n, j, :qn] = o, total
            if backward:
                do = t["dout"][n, :qn, j].double()
                dv[n, :kn, j // g] += p.t().contiguous() @ do
                ds = p * (do @ v.t().contiguous() - (do * o).sum(1, keepdim=True)) / math.sqrt(d)
                dq[n, :qn, j] = ds @ k
                dk[n, :kn, j // g] += ds.t().contiguous() @ q
    return {"dq": dq, "dk": dk, "dv": dv} if backward else {"out": out, "lse": lse}


def exact(case, seed):
    t = _inputs(case, seed)
    op = case["op"]
    if op.startswith("attention"):
        return _exact_attention(case, t)
    if op == "norm_forward":
        x = t["x"].double()
        var, mean = torch.var_mean(x, 2, correction=0)
        rstd = (var + _EPS) ** -0.5
        y = (x - mean[:, :, None]) * rstd[:, :, None] * t["gamma"].double() + t["beta"].double()
        return {"y": y.transpose(1, 2).contiguous() if case["y"] == "map" else y, "mean": mean, "rstd": rstd}
    if op == "norm_backward":
        dy, g = t["dy"].double(), t["gamma"].double()
        x = _exact_held(t["codes"], t["exponents"], case["block"]).view(dy.shape) if case["block"] else t["x"].double()
        # the derivative of y with the statistics given: through the centring, then through the scaling
        r = t["rstd"].double()[:, :, None]
        h = (x - t["mean"].double()[:, :, None]) * r
        a = dy * g
        dx = r * a
        dx = dx - dx.mean(2, keepdim=True) - r * h * (a * h).mean(2, keepdim=True)
        return {"dx": dx.transpose(1, 2).contiguous() if case["x"] == "map" else dx, "dgamma": (dy * h).sum((0, 1)),
                "dbeta": dy.sum((0, 1))}
    if op == "checkpoint":
        v, e = _exact_values(t["x"], case["block"])
        return {"x": _exact_act(v, case["act"], False), "exponents": e}
    x = _exact_held(t["codes"], t["exponents"], case["block"])
    if op == "checkpoint_act":
        return {"dx": t["dy"].double() * _exact_act(x, case["act"], True)}
    return {"dw": t["dy"].double().t().contiguous() @ x}
