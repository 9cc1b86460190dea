"""The operators that answer requests from the cached rows, and what they are timed on.

A serving process holds the rows of every vertex; a request names vertices (`ids`) and the head it wants run on their
rows.  A block of such a head is a normalisation, a projection shared by all tenants with a low-rank adapter of the
request's tenant beside it, and the way back into the residual stream: norm, gate, scale, sum, and the norm that the
next block begins with.

norm_rows      s = residual[ids] + scale * act(gate) * post(y);  n = pre(s)
project_rows   y = act(x[ids] W + b + scale_a (x[ids] A_a) B_a),  a = the row's adapter, or none
"""
import math

import torch

own = False

_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


def _norm(name, rows, d, dtype, residual, post, pre, gate="none", gate_act="identity", vector=False, by_id=False):
    c = {"op": "norm", "rows": rows, "d": d, "dtype": dtype, "residual": residual, "post": post, "pre": pre,
         "gate": gate, "gate_act": gate_act, "vector": vector, "by_id": by_id}
    return {"name": name, **c} if name else c


def _project(name, rows, k, n, dtype, rank, tenants, run, act="identity", by_id=False):
    c = {"op": "project", "rows": rows, "k": k, "n": n, "dtype": dtype, "rank": rank, "tenants": tenants, "run": run,
         "act": act, "by_id": by_id}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one vertex is asked for: its cached row enters the first block
        _norm("norm-one-row", 1, 128, "fp32", "fp32", "none", "layer", by_id=True),
        # a small batch of requests between two blocks
        _norm("norm-batch-64", 64, 256, "bf16", "bf16", "rms", "rms", gate="full", gate_act="silu", vector=True),
        # the features of the social graph: rows that no vector width divides, a gate for each row
        _norm("norm-odd-602", 10_001, 602, "fp32", "fp32", "layer", "layer", gate="row", gate_act="sigmoid"),
        # 16-bit blocks over the fp32 rows of the cache
        _norm("norm-cached-rows", 150_003, 256, "bf16", "fp32", "rms", "rms", vector=True, by_id=True),
        # an offline pass of a wide head
        _norm("norm-wide", 32_768, 4096, "bf16", "bf16", "rms", "rms", gate="full", gate_act="silu"),
        # logits of one vertex for one tenant (the sparse graph's widths)
        _project("project-one-row", 1, 128, 40, "fp32", 8, 4, 1, by_id=True),
        # single rows of many tenants at once
        _project("project-batch-64", 64, 256, 256, "bf16", 16, 64, 1, act="relu"),
        # requests of some thirty vertices each on the social graph's features
        _project("project-odd-602", 1000, 602, 41, "fp32", 8, 32, 31, by_id=True),
        # short requests, tenants in any order, a rank of 32
        _project("project-short-runs", 30_011, 512, 768, "fp16", 32, 64, 20),
        # logits of a large share of the cached vertices (the dense graph's widths)
        _project("project-cached-rows", 200_000, 256, 47, "fp32", 16, 64, 1000, by_id=True),
        # fp32 all the way, hidden widths
        _project("project-fp32-hidden", 40_000, 256, 256, "fp32", 16, 16, 300, act="relu"),
        # an offline pass of a wide head
        _project("project-wide", 65_536, 1024, 1024, "bf16", 16, 128, 512),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.45:
        dtype = rng.choice(("fp32", "bf16", "bf16", "fp16"))
        d = rng.choice((32, 100, 128, 256, 602, 1024, 4096, _log_uniform(rng, 8, 5000), 8 * _log_uniform(rng, 2, 1000)))
        most = (1 << 27) * 2 // (_BYTES[dtype] * d)
        return _norm(None, _log_uniform(rng, 1, min(most // 2, 300_000)), d, dtype, rng.choice((dtype, "fp32")),
                     rng.choice(("none", "layer", "rms")), rng.choice(("none", "layer", "rms")),
                     rng.choice(("none", "row", "full")), rng.choice(("identity", "sigmoid", "silu", "tanh")),
                     rng.random() < 0.5, rng.random() < 0.5)
    dtype = rng.choice(("fp32", "fp32", "bf16", "fp16"))
    k = rng.choice((32, 100, 128, 256, 602, _log_uniform(rng, 16, 1024), 8 * _log_uniform(rng, 2, 128)))
    n = rng.choice((16, 40, 41, 47, 256, _log_uniform(rng, 5, 1024), 8 * _log_uniform(rng, 2, 128)))
    most = (1 << 35) // (k * n) if dtype != "fp32" else (1 << 32) // (k * n)
    rows = _log_uniform(rng, 1, max(2, min(most, 200_000)))
    run = _log_uniform(rng, 1, 1024)
    tenants = min(_log_uniform(rng, 1, 128), 2 * max(1, rows // run))
    return _project(None, rows, k, n, dtype, rng.choice((4, 8, 16, 16, 32, 64, rng.randint(1, 64))), tenants, run,
                    rng.choice(("identity", "relu")), rng.random() < 0.5)


def _inputs(case, seed):
    """The values of a case, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, rows = _DTYPES[case["dtype"]], case["rows"]

    def normal(*shape, scale=1.0, to=dtype):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(to)

    v = {}
    if case["by_id"]:     # distinct vertices of a table with a quarter more rows
        v["table"] = rows + rows // 4 + 3
        v["ids"] = torch.randperm(v["table"], generator=g, device="cuda")[:rows].to(torch.int32)
    if case["op"] == "norm":
        d = case["d"]
        if case["post"] != "none" or case["gate"] != "none" or case["vector"] or not case["by_id"]:
            v["y"] = normal(rows, d, scale=2.0)
            if case["gate"] != "none":
                v["gate"] = normal(rows, d if case["gate"] == "full" else 1)
            v["scale"] = 0.1 + 0.02 * normal(d, to=torch.float32) if case["vector"] else 0.5
        v["residual"] = normal(v.get("table", rows), d, to=_DTYPES[case["residual"]]) + 0.25
        for which in ("post", "pre"):
            if case[which] != "none":
                v[which] = (1 + 0.1 * normal(d, to=torch.float32), 0.1 * normal(d, to=torch.float32) if case[which] == "layer" else None)
        return v
    k, n, r, tenants, run = (case[x] for x in ("k", "n", "rank", "tenants", "run"))
    v["x"] = normal(v.get("table", rows), k)
    v["W"] = normal(k, n, scale=math.sqrt(2.0 / (k + n)))
    v["bias"] = normal(n, scale=0.1, to=torch.float32)
    v["A"] = normal(tenants, k, r, scale=1 / math.sqrt(k))
    v["B"] = normal(tenants, r, n, scale=0.5 / math.sqrt(r))
    v["scales"] = [(0.5, 1.0, 2.0)[t % 3] for t in range(tenants)]
    # requests of `run` rows, each of some tenant; one in sixteen asks for the shared projection alone
    requests = rows // run + 2
    tenant = torch.randint(0, tenants, (requests,), generator=g, device="cuda", dtype=torch.int32)
    tenant[torch.rand(requests, generator=g, device="cuda") < 1 / 16] = -1
    first = int(torch.randint(0, run, (1,), generator=g, device="cuda"))
    v["slots"] = tenant[(torch.arange(rows, device="cuda") + first) // run].contiguous()
    return v


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if own:
        from paper_2601_12347_b200 import serve
        if case["op"] == "norm":
            kinds = {"layer": serve.NORM_LAYER, "rms": serve.NORM_RMS}
            s["norms"] = {w: serve.Norm(kinds[case[w]], *s[w], eps=1e-5) for w in ("post", "pre") if w in s}
        else:
            s["projection"] = serve.Projection(s["W"], s["bias"], act=serve.ACT_RELU if case["act"] == "relu" else serve.ACT_IDENTITY)
            s["bank"] = serve.AdapterBank(s["projection"], case["tenants"], case["rank"])
            s["bank"].set(0, s["A"], s["B"], s["scales"])
    elif case["op"] == "project":
        s["scales"] = torch.tensor(s["scales"], device="cuda")
    return s


def _plain_norm(v, kind, weight_bias):
    if kind == "none":
        return v
    weight, bias = weight_bias
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + 1e-5) * weight
    return v if bias is None else v + bias


def _plain_gate(gate, act):
    if act == "sigmoid":
        return 1 / (1 + torch.exp(-gate))
    if act == "silu":
        return gate / (1 + torch.exp(-gate))
    return torch.tanh(gate) if act == "tanh" else gate


def _run_norm(s):
    c = s["case"]
    if own:
        from paper_2601_12347_b200 import serve
        acts = {"identity": serve.GATE_IDENTITY, "sigmoid": serve.GATE_SIGMOID, "silu": serve.GATE_SILU, "tanh": serve.GATE_TANH}
        stream, normed = serve.norm_rows(s.get("y"), post=s["norms"].get("post"), gate=s.get("gate"), gate_act=acts[c["gate_act"]],
                                         scale=s.get("scale", 1.0), residual=s["residual"], ids=s.get("ids"),
                                         pre=s["norms"].get("pre"), normed_dtype=_DTYPES[c["dtype"]])
        return [t for t in (stream, normed) if t is not None]
    t = s["residual"].float()[s["ids"].long()] if c["by_id"] else s["residual"].float()
    got = []
    if "y" in s:
        p = _plain_norm(s["y"].float(), c["post"], s.get("post"))
        if "gate" in s:
            p = p * _plain_gate(s["gate"].float(), c["gate_act"])
        t = t + s["scale"] * p
        got.append(t.to(s["residual"].dtype))
    if c["pre"] != "none":
        got.append(_plain_norm(t, c["pre"], s["pre"]).to(_DTYPES[c["dtype"]]))
    return got if got else [t.to(s["residual"].dtype)]


def _run_project(s):
    c = s["case"]
    if own:
        from paper_2601_12347_b200 import serve
        return serve.project_rows(s["x"], s["projection"], bank=s["bank"], slots=s["slots"], ids=s.get("ids"))
    x = s["x"][s["ids"].long()].float() if c["by_id"] else s["x"].float()
    y = x @ s["W"].float() + s["bias"]
    slots = s["slots"].long()
    at, has = slots.clamp(min=0), (slots >= 0)[:, None]
    if c["rows"] <= 1024:       # each row with its own adapter's matrices
        t = torch.bmm(x[:, None, :], s["A"].float()[at]) * s["scales"][at][:, None, None]
        delta = torch.bmm(t, s["B"].float()[at])[:, 0, :]
    else:                       # every adapter for every row, and all but the row's own dropped
        k, n, r, tenants = c["k"], c["n"], c["rank"], c["tenants"]
        t = (x @ s["A"].float().permute(1, 0, 2).reshape(k, tenants * r)).view(-1, tenants, r) * s["scales"][:, None]
        t = torch.where((at[:, None] == torch.arange(tenants, device=at.device))[:, :, None], t, 0.0)
        delta = t.view(-1, tenants * r) @ s["B"].float().reshape(tenants * r, n)
    y = y + torch.where(has, delta, 0.0)
    return (torch.relu(y) if c["act"] == "relu" else y).to(s["x"].dtype)


def run(state):
    return _run_norm(state) if state["case"]["op"] == "norm" else _run_project(state)


def exact(case, seed):
    v = _inputs(case, seed)
    f64 = torch.float64
    if case["op"] == "norm":
        def normed(t, kind, wb):
            w = wb[0].to(f64)
            b = torch.zeros_like(w) if wb[1] is None else wb[1].to(f64)
            centre = t.mean(1, True) if kind == "layer" else 0.0
            spread = ((t - centre) ** 2).sum(1, True) / t.shape[1] + 1e-5
            return (t - centre) / spread.sqrt() * w + b
        t = v["residual"].to(f64)
        t = t.index_select(0, v["ids"].long()) if case["by_id"] else t
        got = []
        if "y" in v:
            p = v["y"].to(f64)
            p = normed(p, case["post"], v["post"]) if "post" in v else p
            if "gate" in v:
                gate = v["gate"].to(f64)
                p = p * {"identity": gate, "sigmoid": gate.sigmoid(), "silu": gate * gate.sigmoid(), "tanh": gate.tanh()}[case["gate_act"]]
            scale = v["scale"]
            t = t + p * (scale.to(f64) if case["vector"] else scale)
            got.append(t)
        if "pre" in v:
            got.append(normed(t, case["pre"], v["pre"]))
        return got if got else [t]
    x = v["x"].to(f64)
    x = x.index_select(0, v["ids"].long()) if case["by_id"] else x
    y = torch.addmm(v["bias"].to(f64), x, v["W"].to(f64))
    for a in range(case["tenants"]):
        mine = (v["slots"] == a).nonzero()[:, 0]
        if mine.numel():
            y[mine] += v["scales"][a] * ((x[mine] @ v["A"][a].to(f64)) @ v["B"][a].to(f64))
    return y.clamp(min=0) if case["act"] == "relu" else y


def work(case):
    rows, size = case["rows"], _BYTES[case["dtype"]]
    moved = 4 * rows if case["by_id"] else 0
    if case["op"] == "norm":
        d, res = case["d"], _BYTES[case["residual"]]
        has_y = case["post"] != "none" or case["gate"] != "none" or case["vector"] or not case["by_id"]
        moved += rows * d * res                                                   # residual rows
        if has_y:
            moved += rows * d * (size + res)                                      # y, and the new stream
            moved += rows * size * {"none": 0, "row": 1, "full": d}[case["gate"]]
        if case["pre"] != "none":
            moved += rows * d * size
        elif not has_y:
            moved += rows * d * res
        moved += 4 * d * (case["vector"] + sum({"none": 0, "rms": 1, "layer": 2}[case[w]] for w in ("post", "pre")))
        return {"bytes": moved, "flops": rows * d * 12}
    k, n, r = case["k"], case["n"], case["rank"]
    used = min(case["tenants"], -(-rows // case["run"]) + 1)
    moved += 4 * rows + size * (rows * (k + n) + k * n + used * r * (k + n)) + 4 * n
    return {"bytes": moved, "flops": 2 * rows * (k * n + r * (k + n))}
