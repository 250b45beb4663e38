"""Operators of training a token block on a vocabulary: embedding rows looked up and their gradient, the softmax cross entropy of a
linear layer over the vocabulary with its gradient, and the orthogonal part of a weight's update by Newton-Schulz products.

A case names one pass through one operator ("op"):

  embedding_forward     out[r] = scale * table[ids[r]]; a row without an id (outside 0 .. vocab - 1) is zero
  embedding_backward    dtable in 32 bits: scale * the sum of the dy of the rows with that id
  loss_forward          per row log sum_v exp(s_v) - s_label with s = scale * weight x, that log-sum, and the mean over the labelled rows
  loss_backward         dx, dweight of the sum of dloss[r] * loss[r], with the logits computed again; without dloss, of the mean
  orthogonal            x / (|x| + eps), then `steps` times x <- a x + (b (x x^T) + c (x x^T)^2) x

Where `own` is false the formulas run as plain torch operations in 32 bits.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_IDS = {"i32": torch.int32, "i64": torch.int64}
_ES = {"f32": 4, "bf16": 2}
_COEFFICIENTS = (3.4445, -4.775, 2.0315)
_EPS = 1e-7


def _named(name, c):
    if name:
        c["name"] = name
    return c


def _embedding(name, op, rows, vocab, channels, dtype, ids="i64", missing=0.0, pad=0):
    """missing: share of the rows that have no id; pad: unused channels behind each row of dy (backward)."""
    return _named(name, {"op": op, "rows": rows, "vocab": vocab, "channels": channels, "dtype": dtype, "ids": ids, "missing": missing,
                         "scale": 0.5 if channels % 2 else math.sqrt(channels), "pad": pad})


def _loss(name, op, rows, vocab, channels, dtype, ids="i64", missing=0.0, weighted=False, scale=1.0, pad=0):
    """missing: share of the rows that have no label; weighted: dloss is given; pad: unused channels behind each row of x."""
    return _named(name, {"op": op, "rows": rows, "vocab": vocab, "channels": channels, "dtype": dtype, "ids": ids, "missing": missing,
                         "weighted": weighted, "scale": scale, "pad": pad})


def _orthogonal(name, count, rows, cols, dtype, steps=5):
    return _named(name, {"op": "orthogonal", "count": count, "rows": rows, "cols": cols, "dtype": dtype, "steps": steps})


def listed():
    return [
        # Serving: the embedding rows of one new token of each of 8 streams; all latency.
        _embedding("embedding_tokens_bf16", "embedding_forward", 8, 32768, 1024, "bf16"),
        # Codes of 32 images of 38 x 38 places, a third of them unknown, looked up in 32 bits.
        _embedding("embedding_codes_f32", "embedding_forward", 46208, 8192, 512, "f32", missing=0.33),
        # Training, 64 images of 38 x 38 places, a few codes much more often than the others: the table's gradient.
        _embedding("embedding_backward_bf16", "embedding_backward", 92416, 16384, 512, "bf16", missing=0.1),
        # The same on odd sizes in 32 bits, rows of dy inside wider ones.
        _embedding("embedding_backward_odd_f32", "embedding_backward", 4995, 1001, 250, "f32", ids="i32", pad=3),
        # Serving: how likely the next token of each of 4 streams was; reading the weight is all the work.
        _loss("loss_tokens_bf16", "loss_forward", 4, 32768, 512, "bf16"),
        # Evaluation: 8 images of 38 x 38 tokens on a vocabulary of 16384.
        _loss("loss_forward_bf16", "loss_forward", 11552, 16384, 512, "bf16"),
        # Training where most places are given and only the others have labels; 32 bits, odd sizes.
        _loss("loss_backward_odd_f32", "loss_backward", 4995, 10007, 202, "f32", ids="i32", missing=0.4, weighted=True, pad=5),
        # Training, 8 images of 38 x 38 tokens of 1024 channels on a vocabulary of 32768, every token labelled: the largest loss.
        _loss("loss_backward_bf16", "loss_backward", 11552, 32768, 1024, "bf16"),
        # The update of 64 filters of 64 x 3 x 3: a chain of small products.
        _orthogonal("orthogonal_filters_f32", 1, 64, 576, "f32"),
        # Three layers of odd sizes at once, taller than wide.
        _orthogonal("orthogonal_odd_f32", 3, 707, 133, "f32"),
        # The update of a perceptron's weights in 32 bits, four layers at once.
        _orthogonal("orthogonal_layers_f32", 4, 512, 2048, "f32"),
        # A large square weight's update held in 16 bits: the largest case.
        _orthogonal("orthogonal_large_bf16", 1, 4096, 4096, "bf16"),
    ]


def work(case):
    op, es = case["op"], _ES[case["dtype"]]
    if op == "orthogonal":
        n, k = sorted((case["rows"], case["cols"]))
        # x x^T and its square are symmetric: half of each
        return {"bytes": 2.0 * case["count"] * n * k * es, "flops": float(case["count"] * case["steps"]) * (n * n * k + n ** 3 + 2 * n * n * k)}
    rows, vocab, c = case["rows"], case["vocab"], case["channels"]
    known = rows * (1 - case["missing"])
    ids = rows * (8 if case["ids"] == "i64" else 4)
    if op == "embedding_forward":
        return {"bytes": float(ids + min(known, vocab) * c * es + rows * c * es), "flops": float(rows * c)}
    if op == "embedding_backward":
        return {"bytes": float(ids + known * c * es + 4 * vocab * c), "flops": float(known * c)}
    if op == "loss_forward":
        return {"bytes": float(ids + known * c * es + vocab * c * es + 8 * rows), "flops": 2.0 * known * vocab * c}
    return {"bytes": float(ids + (known + rows) * c * es + 2 * vocab * c * es + 4 * rows), "flops": 6.0 * known * vocab * c}


# ---- drawn cases ---------------------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    wk = work(case)
    return wk["flops"] / (3e14 if case["dtype"] == "bf16" else 1e14) + wk["bytes"] / 3e12


_LARGEST = None


def draw(rng):
    """One case of the listed ones' ranges: 1 to 92416 rows of 8 to 1024 channels on vocabularies of 64 to 32768, matrices of 8 to
    4096 rows and columns."""
    global _LARGEST
    if _LARGEST is None:
        _LARGEST = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("embedding_forward", "embedding_backward", "loss_forward", "loss_forward", "loss_backward", "loss_backward",
                         "orthogonal", "orthogonal"))
        dtype, ids = rng.choice(("f32", "bf16")), rng.choice(("i32", "i64"))
        if op == "orthogonal":
            n, k = _log(rng, 8, 4096), _log(rng, 8, 4096)
            if rng.random() < 0.5:
                n, k = max(8, n // 64 * 64), max(8, k // 64 * 64)
            case = _orthogonal(None, _log(rng, 1, 16), n, k, dtype, rng.choice((5, 5, 5, 3, 6)))
            if case["count"] * n * k > 64e6:
                continue
        else:
            c = _log(rng, 8, 1024)
            if rng.random() < 0.6:
                c = c // 64 * 64 if c >= 64 else c // 8 * 8
            vocab = _log(rng, 64, 32768)
            missing = rng.choice((0.0, 0.0, 0.15, 0.6))
            pad = rng.choice((0, 0, 0, 3, 8))
            if op.startswith("embedding"):
                case = _embedding(None, op, _log(rng, 1, 92416), vocab, c, dtype, ids, missing, pad if op.endswith("backward") else 0)
            else:
                rows = _log(rng, 1, 16) if rng.random() < 0.25 else _log(rng, 1, 11552)
                case = _loss(None, op, rows, vocab, c, dtype, ids, missing if rows > 16 else 0.0, rng.random() < 0.5,
                             rng.choice((1.0, 1.0, 0.25)), pad)
        if _cost(case) <= _LARGEST:
            return case


# ---- inputs --------------------------------------------------------------------------------------------------------
def _normal(g, shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


def _ids(g, case, rows, vocab):
    """Ids of which a few are much more frequent than the others; -1 where there is none."""
    u = torch.rand((rows,), device="cuda", generator=g)
    ids = (u ** 3 * vocab).long().clamp_(max=vocab - 1)
    if case["missing"]:
        ids[torch.rand((rows,), device="cuda", generator=g) < case["missing"]] = -1
        ids[0] = vocab - 1                              # (one at least is there)
    return ids


def _inside(x, pad):
    """x in rows that are `pad` elements longer."""
    if not pad:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), device="cuda", dtype=x.dtype)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, op = _DT[case["dtype"]], case["op"]
    if op == "orthogonal":
        b, n, k = case["count"], case["rows"], case["cols"]
        # a gradient: singular values over three decades, rows of different sizes
        x = _normal(g, (b, n, k)) * torch.exp(_normal(g, (b, n, 1), 0.7)) * torch.exp(_normal(g, (b, 1, k), 0.7))
        return {"x": (x * 1e-3).to(dt)}
    rows, vocab, c = case["rows"], case["vocab"], case["channels"]
    ids = _ids(g, case, rows, vocab)
    t = {"ids": ids.to(_IDS[case["ids"]])}
    if op.startswith("embedding"):
        if op == "embedding_forward":
            t["table"] = _normal(g, (vocab, c), c ** -0.5).to(dt)
        else:
            t["dy"] = _inside(_normal(g, (rows, c)).to(dt), case["pad"])
        return t
    w = _normal(g, (vocab, c), c ** -0.5)
    # tokens that lean towards their labels, some of them much: probabilities from nearly none to nearly one
    x = _normal(g, (rows, c)) + 12 / case["scale"] * torch.rand((rows, 1), device="cuda", generator=g) * w[ids.clamp(min=0)]
    t["x"], t["weight"] = _inside(x.to(dt), case["pad"]), w.to(dt)
    if op == "loss_backward":
        t["dloss"] = torch.rand((rows,), device="cuda", generator=g) / rows if case["weighted"] else None
        t["lse"] = _plain_loss(case, t)[1]              # (what the forward pass left)
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    state = {"case": case, "t": t}
    if not own:
        return state
    from paper_2409_09083_amd import orthogonal, vocabulary
    if case["op"] == "orthogonal":
        state["object"] = orthogonal.Orthogonal(case["rows"], case["cols"], case["dtype"], count=case["count"], steps=case["steps"],
                                                coefficients=_COEFFICIENTS, eps=_EPS)
    elif case["op"].startswith("embedding"):
        state["object"] = vocabulary.Embedding(case["rows"], case["vocab"], case["channels"], case["dtype"], scale=case["scale"],
                                               training=case["op"] == "embedding_backward")
    else:
        state["object"] = vocabulary.TokenLoss(case["rows"], case["vocab"], case["channels"], case["dtype"], scale=case["scale"],
                                               training=case["op"] == "loss_backward")
    return state


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _plain_embedding(case, t):
    ids, dt = t["ids"].long(), _DT[case["dtype"]]
    there = (ids >= 0) & (ids < case["vocab"])
    if case["op"] == "embedding_forward":
        rows = t["table"][torch.where(there, ids, 0)].float() * case["scale"]
        return {"out": torch.where(there[:, None], rows, 0.0).to(dt)}
    d = torch.zeros((case["vocab"] + 1, case["channels"]), device="cuda")
    d.index_add_(0, torch.where(there, ids, case["vocab"]), t["dy"].float())
    return {"dtable": d[:-1] * case["scale"]}


def _plain_logits(case, t):
    return torch.matmul(t["x"].float(), t["weight"].float().t()) * case["scale"]


def _plain_loss(case, t):
    """Losses (0 where there is no label), log-sums (there too), mean."""
    ids = t["ids"].long()
    there = (ids >= 0) & (ids < case["vocab"])
    s = _plain_logits(case, t)
    m = s.amax(1, keepdim=True)
    lse = (m + torch.log(torch.exp(s - m).sum(1, keepdim=True))).squeeze(1)
    loss = lse - s.gather(1, torch.where(there, ids, 0)[:, None]).squeeze(1)
    loss, lse = torch.where(there, loss, 0.0), torch.where(there, lse, 0.0)
    return loss, lse, (loss.double().sum() / there.sum().clamp(min=1)).float()


def _plain_loss_backward(case, t):
    ids, dt = t["ids"].long(), _DT[case["dtype"]]
    there = (ids >= 0) & (ids < case["vocab"])
    weight = torch.where(there, t["dloss"] if case["weighted"] else 1 / there.sum().clamp(min=1).float(), 0.0) * case["scale"]
    p = torch.exp(_plain_logits(case, t) - t["lse"][:, None])
    p.scatter_add_(1, torch.where(there, ids, 0)[:, None], torch.full_like(weight, -1.0)[:, None])
    p = torch.where(there[:, None], p * weight[:, None], 0.0)
    return {"dx": torch.matmul(p, t["weight"].float()).to(dt), "dweight": torch.matmul(p.t(), t["x"].float()).to(dt)}


def _plain_orthogonal(case, t):
    a, b, c = _COEFFICIENTS
    x = t["x"].float()
    tall = case["rows"] > case["cols"]
    x = x / (x.double().square().sum((1, 2), keepdim=True).sqrt() + _EPS).float()
    x = x.transpose(1, 2).contiguous() if tall else x
    for _ in range(case["steps"]):
        s = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * s + c * torch.matmul(s, s), x)
    x = x.transpose(1, 2).contiguous() if tall else x
    return {"out": x.to(_DT[case["dtype"]])}


def run(state):
    case, t = state["case"], state["t"]
    op = case["op"]
    if not own:
        if op == "orthogonal":
            return _plain_orthogonal(case, t)
        if op == "loss_forward":
            loss, lse, mean = _plain_loss(case, t)
            return {"loss": loss, "lse": lse, "mean": mean}
        return _plain_loss_backward(case, t) if op == "loss_backward" else _plain_embedding(case, t)
    o = state["object"]
    if op == "orthogonal":
        return {"out": o.forward(t["x"])}
    if op == "embedding_forward":
        return {"out": o.forward(t["ids"], t["table"])}
    if op == "embedding_backward":
        return {"dtable": o.backward(t["ids"], t["dy"])}
    if op == "loss_forward":
        mean = o.forward(t["x"], t["weight"], t["ids"])
        return {"loss": o.losses, "lse": o.lse, "mean": mean}
    dx, dw = o.backward(t["x"], t["weight"], t["ids"], dloss=t["dloss"], lse=t["lse"])
    return {"dx": dx, "dweight": dw}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    t = _inputs(case, seed)
    op = case["op"]
    if op == "orthogonal":
        a, b, c = _COEFFICIENTS
        out = []
        for x in t["x"].double():
            x = x / (torch.linalg.vector_norm(x) + _EPS)
            for _ in range(case["steps"]):
                # from the smaller side: (x x^T) x = x (x^T x)
                if case["rows"] <= case["cols"]:
                    s = x @ x.t().contiguous()
                    x = a * x + (b * s + c * (s @ s)) @ x
                else:
                    s = x.t().contiguous() @ x
                    x = a * x + x @ (b * s + c * (s @ s))
            out.append(x)
        return {"out": torch.stack(out)}
    ids = t["ids"].long()
    there = ((ids >= 0) & (ids < case["vocab"])).nonzero().squeeze(1)
    known = ids[there]
    rows, c = case["rows"], case["channels"]
    if op == "embedding_forward":
        out = torch.zeros((rows, c), dtype=torch.float64, device="cuda")
        out[there] = t["table"][known].double() * case["scale"]
        return {"out": out}
    if op == "embedding_backward":
        order = torch.argsort(known, stable=True)
        total = torch.zeros((len(known) + 1, c), dtype=torch.float64, device="cuda")
        torch.cumsum(t["dy"][there[order]].double(), 0, out=total[1:])
        ends = torch.cumsum(torch.bincount(known, minlength=case["vocab"]), 0)
        starts = torch.cat((ends.new_zeros(1), ends[:-1]))
        return {"dtable": (total[ends] - total[starts]) * case["scale"]}
    # only the labelled rows
    x, w = t["x"][there].double(), t["weight"].double()
    s = x @ w.t().contiguous() * case["scale"]
    if op == "loss_forward":
        some = torch.logsumexp(s, 1)
        loss, lse = (torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(2))
        lse[there] = some
        loss[there] = some - s[torch.arange(len(known), device="cuda"), known]
        return {"loss": loss, "lse": lse, "mean": loss.sum() / max(1, len(known))}
    p = torch.exp(s - t["lse"][there].double()[:, None])
    p[torch.arange(len(known), device="cuda"), known] -= 1
    share = t["dloss"][there].double() if case["weighted"] else torch.full((len(known),), 1 / max(1, len(known)), dtype=torch.float64, device="cuda")
    p *= case["scale"] * share[:, None]
    dx = torch.zeros((rows, c), dtype=torch.float64, device="cuda")
    dx[there] = p @ w
    return {"dx": dx, "dweight": p.t().contiguous() @ x}
