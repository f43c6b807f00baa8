"""The operators of a mixture-of-experts feed-forward between two norms, as measurable cases.

  kind "norm"     the norm behind a block, its gate, the scaled residual and the norm before
                  the next block in one pass (fb_op_sandwich_norm); with parts > 0 the block's
                  output is a weighted sum of expert rows
  kind "route"    the router: the top-k experts of each token, their weights, and the rows
                  sorted by expert (fb_op_route)
  kind "experts"  matrix products grouped by expert with ragged sizes (fb_op_expert_gemm)

The plain forms are elementary torch operations in 32 bits; exact() is float64.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS_POST, EPS_PRE, RESID_SCALE = 1e-6, 1e-6, 0.875


# ---- the cases ------------------------------------------------------------------------

def listed():
    return [
        # One token between two blocks: latency alone.
        _norm("norm_one_token", rows=1, D=1536),
        # One candidate's tokens behind two experts each: the combination fused with the norms.
        _norm("norm_combine_1560", rows=1560, D=1536, parts=2),
        # A pool of 32 candidates, each with modulation of its own.
        _norm("norm_pool_49920", rows=49920, D=1536, group=1560),
        # An odd width, padded rows and a residual stream in bf16: nothing is 16-byte aligned.
        _norm("norm_odd_2049", rows=2049, D=1235, h_type="bf16", post="layer", pre="rms", pad=6),
        # The router of one token.
        _route("route_one_token", T=1, E=8, k=2),
        # The router of a pool, many small experts, padding tokens among the rest.
        _route("route_pool_49920", T=49920, E=64, k=8, masked=0.1, renorm=True),
        # Both experts of one token, gated: every weight read serves one row.
        _experts("experts_one_token", T=1, E=8, k=2, N=4096, K=1536, act="swiglu"),
        # Expert FFN up of one candidate's refine: 390 rows an expert on average.
        _experts("experts_up_1560", T=1560, E=8, k=2, N=8960, K=1536, act="gelu"),
        # Its FFN down: few output features, a long sum.
        _experts("experts_down_1560", T=1560, E=8, k=2, N=1536, K=8960, gather=False),
        # Many small gated experts, unevenly loaded, a ragged token count.
        _experts("experts_fine_1041", T=1041, E=64, k=8, N=1024, K=1536, act="swiglu", skew=1.0),
        # A few tokens over many experts, most of them with a row or two or none; fp32 results.
        _experts("experts_sparse_33", T=33, E=64, k=4, N=1000, K=1032, out_type="f32", skew=1.5,
                 bias=False),
        # The up-projection of a pool of 16 candidates.
        _experts("experts_pool_24960", T=24960, E=8, k=2, N=8960, K=1536, act="gelu"),
    ]


def draw(rng):
    """One more case of the listed ones' ranges."""
    most = work(listed()[-1])
    while True:
        case = _draw_any(rng)
        w = work(case)
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and _plain_bytes(case) < 2e10:
            return case


def _draw_any(rng):
    pick = rng.random()
    if pick < 0.35:
        D = rng.choice([256, 1536, 5120, _log_int(rng, 33, 6000), 8 * _log_int(rng, 8, 640)])
        rows = _log_int(rng, 1, 49920)
        return _norm(None, rows=rows, D=D, parts=rng.choice([0, 0, 1, 2, 3, 8]),
                     y_type=rng.choice(["bf16", "bf16", "f32"]),
                     h_type=rng.choice(["f32", "f32", "bf16"]),
                     a_type=rng.choice(["bf16", "bf16", "f32"]),
                     post=rng.choice(["rms", "rms", "layer", "none"]),
                     pre=rng.choice(["layer", "rms", "none"]),
                     group=rng.choice([0, _log_int(rng, 1, rows)]), pad=rng.choice([0, 0, 8, 3]))
    if pick < 0.55:
        E = rng.choice([2, 8, 64, 256, _log_int(rng, 1, 512)])
        return _route(None, T=_log_int(rng, 1, 49920), E=E, k=min(E, rng.choice([1, 2, 4, 6, 8])),
                      l_type=rng.choice(["f32", "f32", "bf16"]), masked=rng.choice([0, 0.1, 0.9]),
                      banned=rng.choice([0, 0, 0.5]), renorm=rng.random() < 0.5)
    E = rng.choice([4, 8, 64, 128, _log_int(rng, 1, 160)])
    gather = rng.random() < 0.6
    act = rng.choice(["none", "gelu", "swiglu", "geglu"]) if gather else rng.choice(["none", "gelu"])
    N = 16 * _log_int(rng, 4, 560) if act in ("swiglu", "geglu") else 8 * _log_int(rng, 8, 1120)
    return _experts(None, T=_log_int(rng, 1, 24960), E=E, k=min(E, rng.choice([1, 2, 4, 8])), N=N,
                    K=rng.choice([1536, 8 * _log_int(rng, 8, 1120)]), act=act, gather=gather,
                    out_type=rng.choice(["bf16", "bf16", "f32"]), bias=rng.random() < 0.7,
                    skew=rng.choice([0.0, 0.5, 1.0, 1.5]), masked=rng.choice([0, 0, 0.3]))


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _named(name, **case):
    return dict(name=name, **case) if name else case


def _norm(name, rows, D, parts=0, y_type="bf16", h_type="f32", a_type="bf16", post="rms",
          pre="layer", group=0, pad=0):
    return _named(name, kind="norm", rows=rows, D=D, parts=parts, y_type=y_type, h_type=h_type,
                  a_type=a_type, post=post, pre=pre, group=group, pad=pad)


def _route(name, T, E, k, l_type="f32", masked=0.0, banned=0.0, renorm=False):
    return _named(name, kind="route", T=T, E=E, k=k, l_type=l_type, masked=masked, banned=banned,
                  renorm=renorm)


def _experts(name, T, E, k, N, K, act="none", gather=True, out_type="bf16", bias=True, skew=0.0,
             masked=0.0):
    return _named(name, kind="experts", T=T, E=E, k=k, N=N, K=K, act=act, gather=gather,
                  out_type=out_type, bias=bias, skew=skew, masked=masked)


def _size(t):
    return 2 if t == "bf16" else 4


def work(case):
    if case["kind"] == "norm":
        n, parts = case["rows"] * case["D"], case["parts"]
        groups = -(-case["rows"] // case["group"]) if case["group"] else 1
        b = n * (2 * _size(case["h_type"]) + max(1, parts) * _size(case["y_type"]))
        b += 8 * case["rows"] * parts + 4 * case["D"] * (2 + groups)
        if case["pre"] != "none":
            b += n * _size(case["a_type"]) + 8 * case["D"] * groups
        return {"bytes": b, "flops": n * (20 + 2 * parts)}
    if case["kind"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": T * E * _size(case["l_type"]) + T + 16 * T * k + 4 * (E + 1),
                "flops": T * E * (4 + k)}
    T, E, k, N, K = (case[f] for f in ("T", "E", "k", "N", "K"))
    live = T * (1 - case["masked"])
    rows = max(1, round(live * k))
    Nw = 2 * N if case["act"] in ("swiglu", "geglu") else N
    active = E * (1 - (1 - k / E) ** live) if k < E else E
    b = active * Nw * K * 2 + (live if case["gather"] else rows) * K * 2
    b += rows * N * _size(case["out_type"]) + rows * 4
    return {"bytes": b, "flops": 2.0 * rows * Nw * K}


def _plain_bytes(case):
    """About what the plain form holds at once."""
    if case["kind"] == "norm":
        return 4.0 * case["rows"] * case["D"] * (6 + 2 * case["parts"])
    if case["kind"] == "route":
        return 40.0 * case["T"] * case["E"]
    Nw = 2 * case["N"] if case["act"] in ("swiglu", "geglu") else case["N"]
    most = min(case["T"], 4 + 2 * case["T"] * case["k"] / case["E"] * math.exp(case["skew"] * 2.5))
    return 6.0 * case["E"] * Nw * case["K"] + case["E"] * most * (16.0 * Nw + 8.0 * case["K"])


# ---- inputs ---------------------------------------------------------------------------

def _padded(x, pad):
    """x with rows pad elements further apart than they are long."""
    if not pad:
        return x.contiguous()
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _inputs(case, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 13)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = {"case": case}
    if case["kind"] == "norm":
        rows, D, parts, pad = case["rows"], case["D"], case["parts"], case["pad"]
        # a residual stream: a mean of its own, and a few channels far larger than the rest
        h = randn(rows, D) + 0.3
        h[:, :: max(7, D // 6)] *= 20.0
        s["h"] = _padded(h.to(TYPES[case["h_type"]]), pad)
        y = 0.5 * randn(rows * max(1, parts), D)
        if parts:
            slot = torch.randperm(rows * parts, generator=g, device="cuda").view(rows, parts)
            drop = rand(rows, parts) < 0.05  # tokens without some of their experts, or any
            drop[:: 97] |= rand(drop[:: 97].shape) < 0.5
            weight = rand(rows, parts) + 0.05
            y[slot[drop]] = float("nan")  # rows that nothing points to, weights of no row
            s["weight"] = weight.masked_fill(drop, float("nan"))
            s["slot"] = slot.masked_fill(drop, -1).to(torch.int32)
        s["y"] = _padded(y.to(TYPES[case["y_type"]]), pad)
        groups = -(-rows // case["group"]) if case["group"] else 1
        s["post_w"] = 1 + 0.2 * randn(D)
        s["post_b"] = 0.1 * randn(D) if case["post"] == "layer" else None
        s["gate"] = 0.5 * randn(groups, D)
        s["mul"], s["add"] = 0.3 * randn(groups, D), 0.3 * randn(groups, D)
        s["h_out"] = torch.zeros(rows, D, dtype=TYPES[case["h_type"]], device="cuda")
        s["a"] = (torch.zeros(rows, D, dtype=TYPES[case["a_type"]], device="cuda")
                  if case["pre"] != "none" else None)
    elif case["kind"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        logits = randn(T, E) + 0.5 * randn(E)
        logits = torch.where(rand(T, E) < 0.3, (logits * 4).round() / 4, logits)  # ties
        if case["banned"]:
            logits[rand(T, E) < case["banned"]] = -math.inf
        s["valid"] = None
        if case["masked"]:  # padding tokens hold anything
            s["valid"] = (rand(T) >= case["masked"]).to(torch.uint8)
            logits[s["valid"] == 0] = float("nan")
        s["logits"] = logits.to(TYPES[case["l_type"]])
        for name, n in (("expert", k), ("slot", k)):
            s[name] = torch.zeros(T, n, dtype=torch.int32, device="cuda")
        s["weight"] = torch.zeros(T, k, device="cuda")
        s["token"] = torch.zeros(T * k, dtype=torch.int32, device="cuda")
        s["offsets"] = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    else:
        T, E, k, N, K = (case[f] for f in ("T", "E", "k", "N", "K"))
        Nw = 2 * N if case["act"] in ("swiglu", "geglu") else N
        score = case["skew"] * randn(E) - torch.log(-torch.log(rand(T, E).clamp(1e-9, 1 - 1e-7)))
        chosen = score.argsort(1, descending=True)[:, :k]
        live = rand(T) >= case["masked"]
        flat = chosen.masked_fill(~live[:, None], E).reshape(-1)
        order = flat.sort(stable=True).indices
        counts = torch.bincount(flat, minlength=E + 1)[:E]
        s["offsets"] = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
        s["offsets"][1:] = counts.cumsum(0)
        rows, s["most"] = int(counts.sum()), int(counts.max())  # what the plain form pads to
        s["A"] = randn(T if case["gather"] else T * k, K).to(torch.bfloat16)
        s["index"] = None
        if case["gather"]:
            s["index"] = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
            s["index"][:rows] = (order[:rows] // k).to(torch.int32)
        s["W"] = torch.empty(E, Nw, K, dtype=torch.bfloat16, device="cuda")
        s["W"].normal_(0.0, K ** -0.5, generator=g)
        s["bias"] = 0.2 * randn(E, Nw) if case["bias"] else None
        s["out"] = torch.zeros(T * k, N, dtype=TYPES[case["out_type"]], device="cuda")
    return s


_kept = {}


def _model():
    """The library handle that a program keeps: its stream, workspaces and errors."""
    if "model" not in _kept:
        from paper_2607_04461_gb300 import flashbon, synth
        _kept["model"] = flashbon.Model(synth.TINY, synth.make_weights(synth.TINY))
    return _kept["model"]


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2607_04461_gb300 import flashbon as fb
        s["model"] = _model()
        if case["kind"] == "norm":
            s["args"] = fb.make_sandwich(
                s["h"], y=s["y"], slot=s.get("slot"), weight=s.get("weight"), post=case["post"],
                post_eps=EPS_POST, post_w=s["post_w"], post_b=s["post_b"], gate=s["gate"],
                resid_scale=RESID_SCALE, h_out=s["h_out"], pre=case["pre"], pre_eps=EPS_PRE,
                mul_base=1.0, mul=s["mul"], add=s["add"], a=s["a"], group_rows=case["group"])
        elif case["kind"] == "route":
            s["args"] = fb.make_route(
                s["logits"], s["expert"], s["weight"], s["slot"], s["token"], s["offsets"],
                valid=s["valid"], renorm=case["renorm"])
        else:
            s["args"] = fb.make_experts(
                s["A"], s["W"], s["offsets"], s["out"], index=s["index"], bias=s["bias"],
                act=case["act"])
    return s


def run(s):
    kind = s["case"]["kind"]
    if kind == "norm":
        if own:
            s["model"].op_sandwich_norm(s["args"])
            return {"h": s["h_out"], "a": s["a"]}
        return _plain_norm(s)
    if kind == "route":
        if own:
            s["model"].op_route(s["args"])
            return {f: s[f] for f in ("expert", "weight", "slot", "token", "offsets")}
        return _plain_route(s)
    if own:
        s["model"].op_expert_gemm(s["args"])
        return {"out": s["out"]}
    return _plain_experts(s)


# ---- the plain forms ------------------------------------------------------------------

def _normed(x, kind, eps):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(1, keepdim=True) + eps)


def _plain_norm(s):
    c = s["case"]
    y = s["y"].float()
    if c["parts"]:
        picked = y[s["slot"].clamp(min=0).long()] * s["weight"][:, :, None]
        y = picked.masked_fill((s["slot"] < 0)[:, :, None], 0.0).sum(1)
    u = _normed(y, c["post"], EPS_POST) * s["post_w"]
    if s["post_b"] is not None:
        u = u + s["post_b"]
    gate, mul, add = s["gate"], s["mul"], s["add"]
    if c["group"]:
        of = torch.arange(c["rows"], device="cuda") // c["group"]
        gate, mul, add = gate[of], mul[of], add[of]
    h = RESID_SCALE * s["h"].float() + gate * u
    a = None
    if c["pre"] != "none":
        a = (_normed(h, c["pre"], EPS_PRE) * (1.0 + mul) + add).to(TYPES[c["a_type"]])
    return {"h": h.to(TYPES[c["h_type"]]), "a": a}


def _plain_route(s):
    c = s["case"]
    T, E, k = c["T"], c["E"], c["k"]
    logits = s["logits"].float()
    if s["valid"] is not None:
        logits = logits.masked_fill(s["valid"][:, None] == 0, -math.inf)
    top, expert = logits.sort(dim=1, descending=True, stable=True)  # ties: the lowest index first
    top, expert = top[:, :k], expert[:, :k]
    none = top == -math.inf
    shift = top[:, :1].masked_fill(none[:, :1], 0.0)
    e = torch.exp(top - shift)
    total = (e if c["renorm"] else torch.exp(logits - shift)).sum(1, keepdim=True)
    weight = (e / total).masked_fill(none, 0.0)
    flat = expert.masked_fill(none, E).reshape(-1)
    by, order = flat.sort(stable=True)
    offsets = torch.searchsorted(by, torch.arange(E + 1, device="cuda")).to(torch.int32)
    token = (order // k).masked_fill(by == E, -1).to(torch.int32)
    slot = torch.empty_like(order)
    slot[order] = torch.arange(T * k, device="cuda")
    slot = slot.view(T, k).masked_fill(none, -1).to(torch.int32)
    return {"expert": expert.masked_fill(none, -1).to(torch.int32), "weight": weight, "slot": slot,
            "token": token, "offsets": offsets}


def _gelu(x):
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))


def _act(x, act, N):
    if act == "none":
        return x
    if act == "gelu":
        return _gelu(x)
    gate, up = x[..., :N], x[..., N:]
    return (_gelu(gate) if act == "geglu" else gate / (1 + torch.exp(-gate))) * up


def _plain_experts(s):
    c = s["case"]
    E, N = c["E"], c["N"]
    # the experts' rows side by side, all padded to the fullest one's count
    first, end = s["offsets"][:-1].long(), s["offsets"][1:].long()
    row = first[:, None] + torch.arange(s["most"], device="cuda")
    inside = row < end[:, None]
    src = row.masked_fill(~inside, 0)
    if s["index"] is not None:
        src = s["index"][src].long().masked_fill(~inside, 0)
    x = torch.bmm(s["A"][src].float(), s["W"].float().transpose(1, 2))
    if s["bias"] is not None:
        x = x + s["bias"][:, None, :]
    x = _act(x, c["act"], N).to(TYPES[c["out_type"]])
    # rows of no expert go to one behind the last
    out = torch.zeros(s["out"].shape[0] + 1, N, dtype=x.dtype, device="cuda")
    out[row.masked_fill(~inside, s["out"].shape[0]).view(-1)] = x.view(E * s["most"], N)
    return {"out": out[:-1]}


# ---- 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] == "experts" and work(case)["flops"] > 8e12:
        return None
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "route": _exact_route, "experts": _exact_experts}[case["kind"]](s)


def _exact_norm(s):
    c = s["case"]
    rows, D = c["rows"], c["D"]
    h_new = torch.empty(rows, D, dtype=torch.float64, device="cuda")
    a = torch.empty_like(h_new) if c["pre"] != "none" else None
    step = max(1, 40_000_000 // D)

    def stats(x, kind, eps):
        if kind == "none":
            return x
        mean = x.sum(1, keepdim=True) / D if kind == "layer" else 0.0
        var = ((x - mean) ** 2).sum(1, keepdim=True) / D
        return (x - mean) / (var + eps).sqrt()

    for r0 in range(0, rows, step):
        r = torch.arange(r0, min(rows, r0 + step), device="cuda")
        of = r // c["group"] if c["group"] else torch.zeros_like(r)
        if c["parts"]:
            y = torch.zeros(len(r), D, dtype=torch.float64, device="cuda")
            for j in range(c["parts"]):
                got = (s["slot"][r, j] >= 0).nonzero()[:, 0]
                y[got] += s["weight"][r, j][got, None].double() * s["y"][s["slot"][r, j][got].long()].double()
        else:
            y = s["y"][r].double()
        u = stats(y, c["post"], EPS_POST) * s["post_w"].double()
        if s["post_b"] is not None:
            u += s["post_b"].double()
        h_new[r] = RESID_SCALE * s["h"][r].double() + s["gate"][of].double() * u
        if a is not None:
            a[r] = stats(h_new[r], c["pre"], EPS_PRE) * (1 + s["mul"][of].double()) + s["add"][of].double()
    return {"h": h_new, "a": a}


def _exact_route(s):
    """By hand: k times the largest logit left, then the experts' lists one after the other."""
    c = s["case"]
    T, E, k = c["T"], c["E"], c["k"]
    left = s["logits"].double().clone()
    if s["valid"] is not None:
        left[s["valid"] == 0] = -math.inf
    every = left.clone()
    at = torch.arange(E, device="cuda").expand(T, E)
    expert = torch.full((T, k), -1, dtype=torch.int64, device="cuda")
    value = torch.full((T, k), -math.inf, dtype=torch.float64, device="cuda")
    for j in range(k):
        best = left.amax(1)
        first = torch.where(left == best[:, None], at, E).amin(1)
        some = best > -math.inf
        expert[some, j], value[some, j] = first[some], best[some]
        left.scatter_(1, first.clamp(max=E - 1)[:, None], -math.inf)
    weight = torch.zeros(T, k, dtype=torch.float64, device="cuda")
    some = expert[:, 0] >= 0
    of = value if c["renorm"] else every
    weight[some] = torch.exp(value[some] - torch.logsumexp(of[some], 1, keepdim=True))
    slot = torch.full((T, k), -1, dtype=torch.int64, device="cuda")
    token = torch.full((T * k,), -1, dtype=torch.int64, device="cuda")
    offsets = [0]
    for e in range(E):
        t, j = (expert == e).nonzero(as_tuple=True)
        rows = offsets[-1] + torch.arange(len(t), device="cuda")
        slot[t, j], token[rows] = rows, t
        offsets.append(offsets[-1] + len(t))
    whole = torch.int32
    return {"expert": expert.to(whole), "weight": weight, "slot": slot.to(whole),
            "token": token.to(whole), "offsets": torch.tensor(offsets, dtype=whole)}


def _exact_experts(s):
    c = s["case"]
    N = c["N"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    offsets = s["offsets"].tolist()
    for e in range(c["E"]):
        r0, r1 = offsets[e], offsets[e + 1]
        if r0 == r1:
            continue
        A = s["A"][r0:r1] if s["index"] is None else s["A"][s["index"][r0:r1].long()]
        v = A.double() @ s["W"][e].double().T
        if s["bias"] is not None:
            v += s["bias"][e].double()
        if c["act"] in ("gelu", "geglu"):
            g = v[:, :N]
            v[:, :N] = g / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
        elif c["act"] == "swiglu":
            v[:, :N] *= torch.sigmoid(v[:, :N])
        out[r0:r1] = v[:, :N] * v[:, N:] if v.shape[1] > N else v
    return {"out": out}
