"""The operators that train a head on the cached rows, and what they are timed on.

A head is fitted to the labels of some vertices, minibatch by minibatch: learned rows looked up beside the cached ones, a norm, a
linear layer over the classes and its loss; then the way back.

lookup   y = scale * table[ids];  dtable[r] = scale * sum of dy over the rows i with ids[i] = r
norm     of n = norm(x[ids]): dx (+ what reaches x past the norm), dweight, dbias from dn
loss     loss = logsumexp(x W + b) - (x W + b)[label];  dx, dW, db from dloss
"""
import math

import torch

own = False

_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


def _lookup(name, rows, table, d, dtype, grad_dtype, skew, scale=1.0):
    c = {"op": "lookup", "rows": rows, "table": table, "d": d, "dtype": dtype, "grad_dtype": grad_dtype, "skew": skew, "scale": scale}
    return {"name": name, **c} if name else c


def _norm(name, rows, d, dtype, x_dtype, kind, by_id=False, add=False):
    c = {"op": "norm", "rows": rows, "d": d, "dtype": dtype, "x_dtype": x_dtype, "kind": kind, "by_id": by_id, "add": add}
    return {"name": name, **c} if name else c


def _loss(name, rows, k, classes, dtype, bias=True, grad=True):
    c = {"op": "loss", "rows": rows, "k": k, "classes": classes, "dtype": dtype, "bias": bias, "grad": grad}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one vertex of one of a thousand kinds
        _lookup("lookup-one-row", 1, 1000, 128, "fp32", "fp32", 1.0),
        # learned rows of a vertex's kind or place, named as often as vertices have neighbours: a few rows by thousands
        _lookup("lookup-skewed", 300_007, 50_000, 256, "bf16", "bf16", 3.0, scale=16.0),
        # learned feature rows of the social graph, a minibatch of its vertices
        _lookup("lookup-features", 20_011, 232_965, 602, "fp32", "fp32", 1.0),
        # one vertex
        _norm("norm-grad-one-row", 1, 128, "fp32", "fp32", "layer", by_id=True),
        # the social graph's feature width, rows that no vector width divides
        _norm("norm-grad-odd-602", 10_001, 602, "fp32", "fp32", "layer"),
        # a 16-bit head on the fp32 rows of the cache
        _norm("norm-grad-cached-rows", 150_003, 256, "bf16", "fp32", "rms", by_id=True),
        # a wide head, with the gradient of the residual stream
        _norm("norm-grad-wide", 32_768, 4096, "bf16", "bf16", "layer", add=True),
        # one vertex (the sparse graph's widths)
        _loss("loss-one-row", 1, 128, 40, "fp32"),
        # a minibatch on the social graph's features
        _loss("loss-batch-602", 1000, 602, 41, "fp32"),
        # every labelled vertex at once (the dense graph's widths)
        _loss("loss-cached-rows", 200_000, 256, 47, "fp32"),
        # links: which of many vertices is at the other end; a number of classes that no vector width divides
        _loss("loss-links", 6001, 512, 32_003, "fp16"),
        # as many classes as a large vocabulary has
        _loss("loss-wide", 16_384, 1024, 65_536, "bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    which = rng.random()
    dtype = rng.choice(("fp32", "bf16", "bf16", "fp16"))
    if which < 0.3:
        d = rng.choice((32, 100, 128, 256, 602, 1024, _log_uniform(rng, 1, 4096), 8 * _log_uniform(rng, 1, 512)))
        table = _log_uniform(rng, 1, min(2_500_000, 150_000_000 // d))
        rows = _log_uniform(rng, 1, min(400_000, 120_000_000 // d))
        return _lookup(None, rows, table, d, dtype, rng.choice((dtype, "fp32")), rng.choice((1.0, 1.0, 2.0, 3.0)), rng.choice((1.0, 16.0, math.sqrt(d))))
    if which < 0.6:
        d = rng.choice((32, 100, 128, 256, 602, 1024, 4096, _log_uniform(rng, 8, 5000), 8 * _log_uniform(rng, 2, 1000)))
        rows = _log_uniform(rng, 1, min(300_000, (1 << 27) // (_BYTES[dtype] * d)))
        return _norm(None, rows, d, dtype, rng.choice((dtype, "fp32")), rng.choice(("layer", "rms")), rng.random() < 0.5, rng.random() < 0.5)
    k = rng.choice((32, 100, 128, 256, 602, 1024, _log_uniform(rng, 16, 2048), 8 * _log_uniform(rng, 2, 256)))
    classes = rng.choice((2, 40, 41, 47, _log_uniform(rng, 5, 100_000), _log_uniform(rng, 1000, 100_000), 8 * _log_uniform(rng, 2, 8192)))
    most = min((1 << 39) // (k * classes) if dtype != "fp32" else (1 << 36) // (k * classes), (1 << 29) // classes, (1 << 27) // k)
    return _loss(None, _log_uniform(rng, 1, max(2, min(most, 200_000))), k, classes, dtype, rng.random() < 0.7, rng.random() < 0.8)


def _inputs(case, seed):
    """The values of a case, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, rows = _DTYPES[case["dtype"]], case["rows"]

    def normal(*shape, scale=1.0, to=dtype):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(to)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    v = {}
    if case["op"] == "lookup":
        v["table"] = normal(case["table"], case["d"])
        at = (uniform(rows).double() ** case["skew"] * case["table"]).to(torch.int32).clamp(max=case["table"] - 1)
        # popular rows lie anywhere in the table; one id in 64 is padding
        ids = torch.randperm(case["table"], generator=g, device="cuda")[at.long()].to(torch.int32)
        v["ids"] = torch.where(uniform(rows) < 1 / 64, -1, ids)
        v["dy"] = normal(rows, case["d"])
        return v
    if case["op"] == "norm":
        d, x_dtype = case["d"], _DTYPES[case["x_dtype"]]
        table = rows
        if case["by_id"]:
            table = rows + rows // 4 + 3
            v["ids"] = torch.randperm(table, generator=g, device="cuda")[:rows].to(torch.int32)
        v["x"] = normal(table, d, to=x_dtype, scale=2.0) + 0.25
        v["dn"] = normal(rows, d)
        v["add"] = normal(rows, d, to=x_dtype) if case["add"] else None
        v["weight"], v["norm_bias"] = 1 + 0.1 * normal(d, to=torch.float32), 0.1 * normal(d, to=torch.float32) if case["kind"] == "layer" else None
        return v
    k, classes = case["k"], case["classes"]
    v["x"] = normal(rows, k)
    v["W"] = normal(k, classes, scale=2 / math.sqrt(k))
    v["bias"] = normal(classes, scale=0.1, to=torch.float32) if case["bias"] else None
    v["labels"] = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    if rows > 1:               # some vertices of a minibatch have no label
        v["labels"] = torch.where(uniform(rows) < 1 / 16, -1, v["labels"])
    v["dloss"] = 0.5 + uniform(rows)
    return v


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if own and case["op"] == "norm":
        from paper_2601_12347_b200 import serve
        s["norm"] = serve.Norm(serve.NORM_LAYER if case["kind"] == "layer" else serve.NORM_RMS, s["weight"], s["norm_bias"], eps=1e-5)
    return s


def _run_lookup(s):
    c = s["case"]
    if own:
        from paper_2601_12347_b200 import train
        return [train.lookup_rows(s["table"], s["ids"], scale=c["scale"]),
                train.lookup_rows_grad(s["dy"], s["ids"], c["table"], scale=c["scale"], out_dtype=_DTYPES[c["grad_dtype"]])]
    real = (s["ids"] >= 0)[:, None]
    at = s["ids"].long().clamp(min=0)
    y = torch.where(real, s["table"][at].float() * c["scale"], 0.0)
    dtable = torch.zeros(c["table"], c["d"], device="cuda")
    dtable.index_add_(0, at, torch.where(real, s["dy"].float() * c["scale"], 0.0))
    return [y.to(s["table"].dtype), dtable.to(_DTYPES[c["grad_dtype"]])]


def _run_norm(s):
    c = s["case"]
    if own:
        from paper_2601_12347_b200 import train
        dx, dweight, dbias = train.norm_rows_grad(s["dn"], s["x"], s["norm"], ids=s.get("ids"), add=s["add"])
        return [t for t in (dx, dweight, dbias) if t is not None]
    x = s["x"].float()[s["ids"].long()] if c["by_id"] else s["x"].float()
    dn = s["dn"].float()
    if c["kind"] == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    inv = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + 1e-5)
    x = x * inv
    dxn = dn * s["weight"]
    dx = dxn - x * (dxn * x).mean(dim=1, keepdim=True)
    if c["kind"] == "layer":
        dx = dx - dxn.mean(dim=1, keepdim=True)
    dx = dx * inv
    if s["add"] is not None:
        dx = dx + s["add"].float()
    got = [dx.to(s["x"].dtype), (dn * x).sum(dim=0)]
    return got + [dn.sum(dim=0)] if c["kind"] == "layer" else got


def _run_loss(s):
    c = s["case"]
    if own:
        from paper_2601_12347_b200 import train
        loss, lse = train.loss_rows(s["x"], s["W"], s["labels"], bias=s["bias"])
        if not c["grad"]:
            return [loss, lse]
        dx, dW, dbias = train.loss_rows_grad(s["x"], s["W"], s["labels"], lse, s["dloss"], bias=s["bias"])
        return [t for t in (loss, lse, dx, dW, dbias) if t is not None]
    x, W = s["x"].float(), s["W"].float()
    z = x @ W
    if s["bias"] is not None:
        z = z + s["bias"]
    real = s["labels"] >= 0
    at = s["labels"].long().clamp(min=0)[:, None]
    top = z.max(dim=1, keepdim=True).values
    lse = top + torch.log(torch.exp(z - top).sum(dim=1, keepdim=True))
    loss = torch.where(real, (lse - z.gather(1, at))[:, 0], 0.0)
    if not c["grad"]:
        return [loss, lse[:, 0]]
    g = torch.exp(z - lse)
    g.scatter_add_(1, at, torch.full_like(lse, -1.0))
    g = g * torch.where(real, s["dloss"], 0.0)[:, None]
    got = [loss, lse[:, 0], (g @ W.T).to(s["x"].dtype), (x.T @ g).to(s["W"].dtype)]
    return got + [g.sum(dim=0)] if s["bias"] is not None else got


_RUN = {"lookup": _run_lookup, "norm": _run_norm, "loss": _run_loss}


def run(state):
    return _RUN[state["case"]["op"]](state)


def exact(case, seed):
    v = _inputs(case, seed)
    f64 = torch.float64
    if case["op"] == "lookup":
        ids = v["ids"].long()
        padded = torch.cat([v["table"], torch.zeros_like(v["table"][:1])])
        y = padded.index_select(0, torch.where(ids < 0, case["table"], ids)).to(f64) * case["scale"]
        mine = (ids >= 0).nonzero()[:, 0]
        sums = torch.zeros(case["table"], case["d"], dtype=f64, device="cuda")
        sums.index_put_((ids[mine],), v["dy"][mine].to(f64), accumulate=True)
        return [y, sums * case["scale"]]
    if case["op"] == "norm":
        x = (v["x"].index_select(0, v["ids"].long()) if case["by_id"] else v["x"]).to(f64)
        dn, w, d = v["dn"].to(f64), v["weight"].to(f64), case["d"]
        layer = case["kind"] == "layer"
        centred = x - x.sum(1, True) / d if layer else x
        spread = ((centred ** 2).sum(1, True) / d + 1e-5).sqrt()
        up = dn * w
        along = (up * centred).sum(1, True) / (d * spread ** 2)
        dx = (up - centred * along - (up.sum(1, True) / d if layer else 0.0)) / spread
        if v["add"] is not None:
            dx = dx + v["add"].to(f64)
        got = [dx, (dn * centred / spread).sum(0)]
        return got + [dn.sum(0)] if layer else got
    W = v["W"].to(f64)
    b = torch.zeros(case["classes"], dtype=f64, device="cuda") if v["bias"] is None else v["bias"].to(f64)
    loss, lse, dx = [], [], []
    dW, db = torch.zeros_like(W), torch.zeros_like(b)
    some = max(1, (1 << 28) // case["classes"])
    for r in range(0, case["rows"], some):
        x, labels = v["x"][r:r + some].to(f64), v["labels"][r:r + some].long()
        z = torch.addmm(b, x, W)
        l = torch.logsumexp(z, 1)
        has = (labels >= 0).nonzero()[:, 0]
        here = torch.zeros_like(l)
        here[has] = l[has] - z[has, labels[has]]
        loss.append(here)
        lse.append(l)
        if case["grad"]:
            p = torch.softmax(z, 1)
            p[has, labels[has]] -= 1
            weight = torch.zeros_like(l)
            weight[has] = v["dloss"][r:r + some].to(f64)[has]
            p *= weight[:, None]
            dx.append(p @ W.T)
            dW += x.T @ p
            db += p.sum(0)
    got = [torch.cat(loss), torch.cat(lse)]
    if case["grad"]:
        got += [torch.cat(dx), dW] + ([db] if v["bias"] is not None else [])
    return got


def work(case):
    rows, size = case["rows"], _BYTES[case["dtype"]]
    if case["op"] == "lookup":
        d, table = case["d"], case["table"]
        named = min(rows, table)
        return {"bytes": 4 * rows + d * (size * (named + 2 * rows) + _BYTES[case["grad_dtype"]] * table), "flops": 2 * rows * d}
    if case["op"] == "norm":
        d, xs = case["d"], _BYTES[case["x_dtype"]]
        moved = rows * d * (size + xs * (3 if case["add"] else 2)) + (4 * rows if case["by_id"] else 0)
        return {"bytes": moved + 4 * d * (4 if case["kind"] == "layer" else 2), "flops": 15 * rows * d}
    k, classes = case["k"], case["classes"]
    moved = size * (rows * k + k * classes) * (2 if case["grad"] else 1) + rows * (16 if case["grad"] else 12)
    moved += (8 if case["grad"] else 4) * classes if case["bias"] else 0
    return {"bytes": moved, "flops": (6 if case["grad"] else 2) * rows * k * classes}
