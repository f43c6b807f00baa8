"""Operators of a pool that serves several requests at once, as measurable cases.

  kind "cross"    attention to encoder states of another length: every sequence of queries has a
                  prompt of its own length, may share it with others, keys may be masked
                  (fb_op_cross_attention)
  kind "adapter"  a projection with low-rank adapters: every segment of rows has an adapter of its
                  own, or none, beside the shared weights (fb_op_adapter_gemm)

The plain forms are elementary torch operations in 32 bits; exact() is float64.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases ------------------------------------------------------------------------

def listed():
    return [
        # One token asks a padded prompt: latency alone.
        _cross("cross_one_token", queries=[1], keys=[512]),
        # 64 sequences of one token each over encoder states of very different lengths, four query
        # heads a key head: every key is read once.
        _cross("cross_tokens_64", queries=[1] * 64, keys=_lengths(64, 32, 4096, 1), heads=16, kv_heads=4),
        # A block of one candidate's refine.
        _cross("cross_candidate_1560", queries=[1560], keys=[512]),
        # A pool of 32 candidates of 8 prompts, and no prompt is padded.
        _cross("cross_prompts_49920", queries=[1560] * 32, keys=_lengths(8, 20, 512, 2), shared=True),
        # Odd lengths, sequences without a query or a key, padding keys inside the prompts, heads of
        # 64, three query heads a key head, rows further apart than they are long.
        _cross("cross_masked_odd", queries=_lengths(23, 0, 700, 3), keys=_lengths(23, 0, 400, 4),
               heads=6, kv_heads=2, D=64, masked=0.3, pad=8),
        # 4096 tokens of one large image over the states of a long reference.
        _cross("cross_long_8191", queries=[4096], keys=[8191]),
        # One row: every weight serves it alone.
        _adapter("adapter_one_row", segments=[1], N=1536, K=1536, rank=16),
        # The modulation of 64 requests, a row and an adapter each.
        _adapter("adapter_rows_64", segments=[1] * 64, N=9216, K=1536, rank=16, adapters=64),
        # FFN down of one candidate, gated into the residual stream.
        _adapter("adapter_down_1560", segments=[1560], N=1536, K=8960, rank=32, resid=True),
        # The prompts of 16 requests through the text projection, some without an adapter.
        _adapter("adapter_prompts_16", segments=_lengths(16, 5, 512, 5), N=1536, K=4096, rank=16,
                 adapters=8, none=0.25, act="gelu"),
        # Odd sizes, fp32 results, empty segments.
        _adapter("adapter_odd_613", segments=_lengths(9, 0, 150, 6), N=1000, K=1032, rank=8,
                 adapters=5, out_type="f32", bias=False, pad=8),
        # FFN up of 16 candidates of 4 requests.
        _adapter("adapter_pool_24960", segments=[6240] * 4, N=8960, K=1536, rank=64, adapters=4,
                 act="gelu"),
    ]


def draw(rng):
    """One more case of the listed ones' ranges."""
    every = [work(c) for c in listed()]
    flops, moved = max(w["flops"] for w in every), max(w["bytes"] for w in every)
    while True:
        case = _draw_cross(rng) if rng.random() < 0.5 else _draw_adapter(rng)
        w = work(case)
        rows = sum(_numbers(case["queries" if case["kind"] == "cross" else "segments"]))
        if rows and w["flops"] <= flops and w["bytes"] <= moved and _plain_bytes(case) < 2e10:
            return case


def _draw_cross(rng):
    seqs = _log_int(rng, 1, 64)
    most = rng.choice([1, 4, 64, 1560, 4096])
    queries = _lengths(seqs, rng.choice([0, 1]), most, rng.randrange(1 << 30))
    shared = rng.random() < 0.4
    states = _log_int(rng, 1, seqs) if shared else seqs
    keys = _lengths(states, rng.choice([0, 1, 20]), rng.choice([77, 512, 512, 4096, 8191]),
                    rng.randrange(1 << 30))
    kv_heads = rng.choice([1, 2, 4, 8, 12])
    group = rng.choice([1, 1, 1, 2, 3, 4, 8])
    return _cross(None, queries, keys, heads=kv_heads * group, kv_heads=kv_heads,
                  D=rng.choice([128, 128, 64]), shared=shared, masked=rng.choice([0, 0, 0.1, 0.6]),
                  pad=rng.choice([0, 0, 8, 24]))


def _draw_adapter(rng):
    count = _log_int(rng, 1, 128)
    segments = _lengths(count, rng.choice([0, 1]), rng.choice([1, 1, 8, 64, 512, 1560, 6240]),
                        rng.randrange(1 << 30))
    resid = rng.random() < 0.3
    return _adapter(None, segments, N=8 * _log_int(rng, 8, 1152), K=8 * _log_int(rng, 8, 1120),
                    rank=8 * _log_int(rng, 1, 16), adapters=_log_int(rng, 1, count),
                    none=rng.choice([0, 0, 0.3]), act="none" if resid else rng.choice(["none", "gelu"]),
                    out_type=rng.choice(["bf16", "bf16", "f32"]), resid=resid,
                    bias=rng.random() < 0.7, pad=rng.choice([0, 0, 8]))


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _lengths(n, lo, hi, seed):
    """n lengths of [lo, hi], spread over their logarithm."""
    rng = random.Random(seed)
    return [max(lo, min(hi, _log_int(rng, max(lo, 0.7), hi))) if rng.random() > 0.1 or lo else 0
            for _ in range(n)]


def _text(numbers):
    """Lengths as one plain value of a case: "1560*32" or "5 17 9"."""
    if len(set(numbers)) == 1:
        return f"{numbers[0]}*{len(numbers)}"
    return " ".join(str(n) for n in numbers)


def _numbers(text):
    if "*" in text:
        n, count = text.split("*")
        return [int(n)] * int(count)
    return [int(n) for n in text.split()]


def _named(name, **case):
    return dict(name=name, **case) if name else case


def _cross(name, queries, keys, heads=12, kv_heads=None, D=128, shared=False, masked=0.0, pad=0):
    return _named(name, kind="cross", queries=_text(queries), keys=_text(keys), heads=heads,
                  kv_heads=kv_heads or heads, D=D, shared=shared, masked=masked, pad=pad)


def _adapter(name, segments, N, K, rank, adapters=1, none=0.0, act="none", out_type="bf16",
             resid=False, bias=True, pad=0):
    return _named(name, kind="adapter", segments=_text(segments), N=N, K=K, rank=rank,
                  adapters=adapters, none=none, act=act, out_type="f32" if resid else out_type,
                  resid=resid, bias=bias, pad=pad)


def _states_of(case):
    """The encoder states that each sequence attends to."""
    n, states = len(_numbers(case["queries"])), len(_numbers(case["keys"]))
    return [s * states // n for s in range(n)] if case["shared"] else list(range(n))


def _adapters_of(case):
    """The adapter of each segment, -1 for none."""
    segments = _numbers(case["segments"])
    rng = random.Random(len(segments) * 31 + case["adapters"])
    return [-1 if rng.random() < case["none"] else s % case["adapters"] for s in range(len(segments))]


def work(case):
    if case["kind"] == "cross":
        queries, keys, of = _numbers(case["queries"]), _numbers(case["keys"]), _states_of(case)
        live = 1 - case["masked"]
        used = sum(keys[s] for s in {of[i] for i, q in enumerate(queries) if q})
        b = 4.0 * sum(queries) * case["heads"] * case["D"]
        b += 4.0 * used * live * case["kv_heads"] * case["D"] + (used if case["masked"] else 0)
        b += 4 * (len(queries) + len(keys) + 2)
        pairs = sum(q * keys[of[i]] for i, q in enumerate(queries))
        return {"bytes": b, "flops": 4.0 * case["D"] * case["heads"] * pairs * live}
    N, K, rank = case["N"], case["K"], case["rank"]
    segments, of = _numbers(case["segments"]), _adapters_of(case)
    rows = sum(segments)
    adapted = sum(n for n, e in zip(segments, of) if e >= 0)
    used = len({e for n, e in zip(segments, of) if n and e >= 0})
    b = 2.0 * (rows * K + N * K + used * rank * (N + K)) + 8 * len(segments)
    b += rows * N * ((8 if case["resid"] else 4) if case["out_type"] == "f32" else 2)
    b += 4.0 * N * (case["bias"] + case["resid"])
    return {"bytes": b, "flops": 2.0 * rows * N * K + 2.0 * adapted * rank * (N + K)}


def _plain_bytes(case):
    """About what the plain form holds at once."""
    if case["kind"] == "cross":
        queries, keys, of = _numbers(case["queries"]), _numbers(case["keys"]), _states_of(case)
        most = max(q * keys[of[i]] for i, q in enumerate(queries))
        return 12.0 * sum(queries) * case["heads"] * case["D"] + 16.0 * most * case["heads"]
    rows = sum(_numbers(case["segments"]))
    return 6.0 * case["N"] * case["K"] + rows * (6.0 * case["K"] + 24.0 * case["N"])


# ---- inputs ---------------------------------------------------------------------------

def _padded(x, pad):
    """x with rows pad elements further apart than they are long."""
    if not pad:
        return x
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _whole(numbers):
    return torch.tensor(numbers, dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 17)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = {"case": case}
    if case["kind"] == "cross":
        queries, keys = _numbers(case["queries"]), _numbers(case["keys"])
        heads, kv_heads, D, pad = case["heads"], case["kv_heads"], case["D"], case["pad"]
        s["q_at"], s["k_at"], s["of"] = _offsets(queries), _offsets(keys), _states_of(case)
        rows, kv_rows = s["q_at"][-1], s["k_at"][-1]
        # normed queries and keys; some heads look at few keys, some at all alike
        peak = torch.linspace(0.5, 4.0, heads, device="cuda").repeat_interleave(D)
        s["q"] = _padded((randn(rows, heads * D) * peak).to(torch.bfloat16), pad)
        # keys and values side by side, as one projection leaves them
        kv = randn(kv_rows, 2 * kv_heads * D)
        kv[:, kv_heads * D:] += 0.2
        s["valid"] = None
        if case["masked"]:  # padding keys hold anything
            s["valid"] = (torch.rand(kv_rows, generator=g, device="cuda") >= case["masked"]).to(torch.uint8)
            kv[s["valid"] == 0] = float("nan")
        kv = _padded(kv.to(torch.bfloat16), pad)
        s["k"], s["v"] = kv[:, :kv_heads * D], kv[:, kv_heads * D:]
        s["q_offsets"], s["kv_offsets"] = _whole(s["q_at"]), _whole(s["k_at"])
        s["kv_of"] = _whole(s["of"]) if case["shared"] else None
        s["out"] = torch.zeros(rows, heads * D, dtype=torch.bfloat16, device="cuda")
        return s
    N, K, rank, adapters = case["N"], case["K"], case["rank"], case["adapters"]
    s["at"], s["of"] = _offsets(_numbers(case["segments"])), _adapters_of(case)
    rows = s["at"][-1]
    s["x"] = _padded(randn(rows, K).to(torch.bfloat16), case["pad"])
    s["w"] = (randn(N, K) * K ** -0.5).to(torch.bfloat16)
    # the adapters' product adds about a third of what the shared one gives
    s["a"] = (randn(adapters, rank, K) * K ** -0.5).to(torch.bfloat16)
    s["b"] = (randn(adapters, N, rank) * rank ** -0.5).to(torch.bfloat16)
    s["scale"] = 0.25 + 0.25 * torch.rand(adapters, generator=g, device="cuda")
    s["bias"] = 0.2 * randn(N) if case["bias"] else None
    s["resid"] = 2.0 * randn(rows, N) if case["resid"] else None
    s["gate"] = 0.5 * randn(N) if case["resid"] else None
    s["offsets"], s["adapter"] = _whole(s["at"]), _whole(s["of"])
    s["out"] = torch.zeros(rows, N, dtype=TYPES[case["out_type"]], device="cuda")
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
        if case["kind"] == "cross":
            s["args"] = fb.make_cross(s["q"], s["k"], s["v"], s["out"], s["q_offsets"],
                                      s["kv_offsets"], head_dim=case["D"], kv_of=s["kv_of"],
                                      valid=s["valid"])
        else:
            s["args"] = fb.make_adapters(s["x"], s["w"], s["a"], s["b"], s["offsets"], s["adapter"],
                                         s["out"], scale=s["scale"], bias=s["bias"], act=case["act"],
                                         resid=s["resid"], gate=s["gate"])
    return s


def run(s):
    if own:
        if s["case"]["kind"] == "cross":
            s["model"].op_cross_attention(s["args"])
        else:
            s["model"].op_adapter_gemm(s["args"])
        return {"out": s["out"]}
    return _plain_cross(s) if s["case"]["kind"] == "cross" else _plain_adapter(s)


# ---- the plain forms ------------------------------------------------------------------

def _plain_cross(s):
    c = s["case"]
    heads, kv_heads, D = c["heads"], c["kv_heads"], c["D"]
    out = torch.zeros_like(s["out"])
    for i, of in enumerate(s["of"]):
        q0, q1, k0, k1 = s["q_at"][i], s["q_at"][i + 1], s["k_at"][of], s["k_at"][of + 1]
        if q0 == q1 or k0 == k1:
            continue
        # [kv head][query of a group's heads][D]
        q = s["q"][q0:q1].float().view(q1 - q0, kv_heads, heads // kv_heads, D)
        q = q.permute(1, 2, 0, 3).reshape(kv_heads, -1, D)
        k = s["k"][k0:k1].float().view(k1 - k0, kv_heads, D).permute(1, 2, 0)
        v = s["v"][k0:k1].float().view(k1 - k0, kv_heads, D).permute(1, 0, 2)
        score = torch.bmm(q, k) * D ** -0.5
        if s["valid"] is not None:
            padding = s["valid"][k0:k1] == 0
            score = score.masked_fill(padding, -math.inf)
            v = v.masked_fill(padding[:, None], 0.0)
        top = score.amax(2, keepdim=True)
        p = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
        total = p.sum(2, keepdim=True)
        o = torch.bmm(p, v) / total.masked_fill(total == 0, 1.0)
        o = o.view(kv_heads, heads // kv_heads, q1 - q0, D).permute(2, 0, 1, 3)
        out[q0:q1] = o.reshape(q1 - q0, heads * D).to(out.dtype)
    return {"out": out}


def _plain_adapter(s):
    x = s["x"].float()
    y = x @ s["w"].float().T
    if s["bias"] is not None:
        y = y + s["bias"]
    for i, e in enumerate(s["of"]):
        r0, r1 = s["at"][i], s["at"][i + 1]
        if e >= 0 and r0 < r1:
            y[r0:r1] += s["scale"][e] * ((x[r0:r1] @ s["a"][e].float().T) @ s["b"][e].float().T)
    if s["case"]["act"] == "gelu":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    if s["resid"] is not None:
        y = s["resid"] + s["gate"] * y
    return {"out": y.to(s["out"].dtype)}


# ---- 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_cross(s) if case["kind"] == "cross" else _exact_adapter(s)


def _exact_cross(s):
    """Head by head, on the valid keys alone."""
    c = s["case"]
    D, group = c["D"], c["heads"] // c["kv_heads"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for i, of in enumerate(s["of"]):
        rows = slice(s["q_at"][i], s["q_at"][i + 1])
        keys = torch.arange(s["k_at"][of], s["k_at"][of + 1], device="cuda")
        if s["valid"] is not None:
            keys = keys[s["valid"][keys] != 0]
        if rows.start == rows.stop or len(keys) == 0:
            continue
        for h in range(c["heads"]):
            at, kv = slice(h * D, (h + 1) * D), slice(h // group * D, (h // group + 1) * D)
            score = s["q"][rows, at].double() @ s["k"][keys, kv].double().T / math.sqrt(D)
            p = torch.exp(score - torch.logsumexp(score, 1, keepdim=True))
            out[rows, at] = p @ s["v"][keys, kv].double()
    return {"out": out}


def _exact_adapter(s):
    """Each adapter merged into the weights, for the rows that have it."""
    c = s["case"]
    x = s["x"].double()
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    row_of = torch.full((x.shape[0],), -1, dtype=torch.int64, device="cuda")
    for i, e in enumerate(s["of"]):
        row_of[s["at"][i]:s["at"][i + 1]] = e
    for e in sorted(set(s["of"])):
        rows = (row_of == e).nonzero()[:, 0]
        w = s["w"].double()
        if e >= 0:
            w = w + s["scale"][e].double() * (s["b"][e].double() @ s["a"][e].double())
        out[rows] = x[rows] @ w.T
    if s["bias"] is not None:
        out += s["bias"].double()
    if c["act"] == "gelu":
        out = out / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (out + 0.044715 * out ** 3)))
    if s["resid"] is not None:
        out = s["resid"].double() + s["gate"].double() * out
    return {"out": out}
