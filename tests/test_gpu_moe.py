"""The operators of a mixture-of-experts feed-forward between two norms, through the public
calls, against their definitions in float64.

Tolerances, from the arithmetic:
  * fp32 elementwise chains and row sums: a row of D values is summed in at most D / 32 + 16
    additions that follow one another, so a statistic is off by at most (D / 32 + 16) 6e-8
    (the row sums' errors are random: half of it covers them); every further operation adds 6e-8 of
    its operands' size. Each element is compared with the sum of its terms' sizes.
  * rounding to bf16: 2^-8 of the value (8 significant bits, half a unit of the last one).
  * products: a 64-wide K block is four MMAs, each of which may cut the running sum by one
    fp32 unit, 1.2e-7 of it. The largest result stands for the running sum.
  * bf16 results of GELU and SiLU may be off by 2^-10.9 of the tanh that x / 2 multiplies, as with
    the hardware tanh; that they keep bf16's precision where that cancels has a test of its own.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2607_04461_gb300 import flashbon as fb
from paper_2607_04461_gb300 import synth

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def model():
    m = fb.Model(synth.TINY, synth.make_weights(synth.TINY))
    yield m
    m.close()


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def padded(x, pad, fill=7.0):
    wide = torch.full((x.shape[0], x.shape[1] + pad), fill, dtype=x.dtype, device="cuda")
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


# ---- norms around a block -------------------------------------------------------------

def norm64(x, size, kind, eps):
    """The norm in float64, and the size of its terms."""
    if kind == "none":
        return x, size
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    rstd = 1 / (((x - mean) ** 2).mean(1, keepdim=True) + eps).sqrt()
    return (x - mean) * rstd, (size + mean.abs()) * rstd


def sandwich_case(model, rows, D, parts=0, y_t=BF, h_t=F32, a_t=BF, post="rms", pre="layer",
                  group=0, pad=0, seed=0, gate=True, mods=True, affine=True, in_place=False,
                  with_y=True, drop=0.2, y_off=0.0, scale=0.75, mul_base=1.0, eps=1e-6):
    g = gen(1000 + seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    h = padded((3 * randn(rows, D) + 0.5).to(h_t), pad)
    h0 = h.clone()
    y = slot = weight = None
    if with_y:
        y = padded((randn(rows * max(1, parts) + 3, D) + y_off).to(y_t), pad)
    if parts:
        slot = torch.randperm(rows * parts, generator=g, device="cuda").view(rows, parts)
        gone = torch.rand(rows, parts, generator=g, device="cuda") < drop
        if rows > 2:
            gone[1] = True  # a token without any expert
        weight = torch.rand(rows, parts, generator=g, device="cuda")
        y[slot[gone]] = float("nan")
        slot, weight = slot.masked_fill(gone, -1).int(), weight.masked_fill(gone, math.inf)
    groups = -(-rows // group) if group else 1
    wide = randn(groups, 3 * D + 4) if mods else None  # gate, mul, add side by side
    gt = wide[:, :D] if gate and mods else None
    mul, add = (wide[:, D:2 * D], wide[:, 2 * D:3 * D]) if mods else (None, None)
    pw, pb = (1 + 0.2 * randn(D), 0.1 * randn(D)) if affine else (None, None)
    h_out = h if in_place else padded(torch.full((rows, D), 5.0, device="cuda").to(h_t), pad)
    a = padded(torch.full((rows, D), 5.0, device="cuda").to(a_t), pad) if pre is not None else None
    s = fb.make_sandwich(h, y=y, slot=slot, weight=weight, post=post, post_eps=eps, post_w=pw,
                         post_b=pb, gate=gt, resid_scale=scale, h_out=h_out, pre=pre or "none",
                         pre_eps=eps, mul_base=mul_base, mul=mul, add=add, a=a, group_rows=group)
    model.op_sandwich_norm(s)
    torch.cuda.synchronize()

    of = torch.arange(rows, device="cuda") // group if group else torch.zeros(rows, device="cuda").long()
    per = lambda x, none: torch.full((1, 1), none, device="cuda").double() if x is None else x.double()[of]  # noqa: E731
    hd = h0.double()
    want, size = scale * hd, (scale * hd).abs()
    if with_y:
        if parts:
            yd, ysize = torch.zeros_like(hd), torch.zeros_like(hd)
            for j in range(parts):
                ok = (slot[:, j] >= 0).nonzero()[:, 0]
                t = weight[ok, j, None].double() * y[slot[ok, j].long()].double()
                yd[ok] += t
                ysize[ok] += t.abs()
        else:
            yd = y[:rows].double()
            ysize = yd.abs()
        u, usize = norm64(yd, ysize, post, eps)
        if affine:
            u, usize = u * pw.double() + pb.double(), usize * pw.double().abs() + pb.double().abs()
        want = want + per(gt, 1.0) * u
        size = size + per(gt, 1.0).abs() * usize
    unit = 0.5 * (D / 32 + 16) * 6e-8 + 10 * 6e-8
    check(h_out, want, unit * size, h_t)
    if a is not None:
        n, nsize = norm64(want, size, pre, eps)
        f = mul_base + (mul.double()[of] if mods else 0.0)
        want_a = n * f + per(add, 0.0)
        check(a, want_a, 2 * unit * (nsize * (abs(f) if not mods else f.abs()) + per(add, 0.0).abs()), a_t)
    if pad:  # what lies between the rows
        for x in (h_out, a):
            if x is not None:
                base = x.as_strided((rows, D + pad), (D + pad, 1))
                assert torch.all(base[:, D:] == 7.0)


def check(got, want, tol, dtype):
    assert torch.isfinite(got.float()).all()
    if dtype == BF:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    bad = (got.double() - want).abs() - tol
    assert bad.max().item() <= 0, f"{bad.max().item():.3e} over, {(bad > 0).sum().item()} elements"


@pytest.mark.parametrize("rows,D", [
    (1, 1), (3, 7), (5, 8), (2, 33), (9, 128), (1, 1536), (7, 1536), (300, 1536), (1561, 1536),
    (33, 1000), (12, 1235), (65, 2048), (17, 2056), (31, 5120), (6, 6001), (5, 8192), (3, 9000), (2, 16384),
    (4, 16383),
])
@pytest.mark.parametrize("post,pre", [("rms", "layer"), ("layer", "rms"), ("none", "none")])
def test_sandwich_widths(model, rows, D, post, pre):
    sandwich_case(model, rows, D, post=post, pre=pre, seed=D)


@pytest.mark.parametrize("y_t", [BF, F32])
@pytest.mark.parametrize("h_t", [BF, F32])
@pytest.mark.parametrize("a_t", [BF, F32])
@pytest.mark.parametrize("D,pad", [(256, 0), (256, 8), (256, 3), (1536, 4), (777, 1)])
def test_sandwich_types_and_strides(model, y_t, h_t, a_t, D, pad):
    sandwich_case(model, 37, D, y_t=y_t, h_t=h_t, a_t=a_t, pad=pad, parts=0, seed=pad)
    sandwich_case(model, 37, D, y_t=y_t, h_t=h_t, a_t=a_t, pad=pad, parts=2, seed=pad, in_place=True)


@pytest.mark.parametrize("parts", [1, 2, 3, 8, 16])
@pytest.mark.parametrize("rows,D", [(1, 256), (40, 1536), (130, 515)])
def test_sandwich_combines_expert_rows(model, parts, rows, D):
    """Rows without some of their experts, or any; rows that nothing points to hold NaN and
    the weights of missing ones infinity."""
    sandwich_case(model, rows, D, parts=parts, seed=parts)
    sandwich_case(model, rows, D, parts=parts, seed=parts, drop=1.1, y_t=F32)


@pytest.mark.parametrize("group", [1, 7, 100, 4000])
def test_sandwich_modulation_groups(model, group):
    sandwich_case(model, 100, 1536, group=group, seed=group)
    sandwich_case(model, 100, 100, group=group, seed=group, h_t=BF)


@pytest.mark.parametrize("kw", [
    dict(with_y=False), dict(with_y=False, scale=1.0, pre="rms"), dict(pre=None), dict(gate=False),
    dict(mods=False), dict(affine=False), dict(affine=False, mods=False, post="layer"),
    dict(mul_base=0.0), dict(scale=0.0), dict(scale=-1.5, in_place=True),
    dict(y_off=100.0, post="layer"), dict(y_off=-30.0, post="rms", eps=1e-3),
])
@pytest.mark.parametrize("D", [640, 1536, 1001])
def test_sandwich_parts_left_out(model, D, kw):
    sandwich_case(model, 50, D, seed=5, **kw)


def test_sandwich_many_rows(model):
    """More rows than one wave holds, for each row's own place in the outputs."""
    sandwich_case(model, 49920, 1536, group=1560, seed=3)
    sandwich_case(model, 20001, 1536, parts=2, seed=4)
    sandwich_case(model, 9001, 5120, seed=6)


def test_sandwich_special_values(model):
    """A row with a NaN or an infinity stays its own; a constant row has no variance."""
    D = 1536
    y = torch.randn(6, D, device="cuda").to(BF)
    y[1, 5], y[2, 700] = float("nan"), float("inf")
    y[3] = 3.0
    h = torch.randn(6, D, device="cuda")
    a, h_out = torch.zeros(6, D, device="cuda"), torch.zeros(6, D, device="cuda")
    model.op_sandwich_norm(fb.make_sandwich(h, y=y, post="layer", pre="rms", a=a, h_out=h_out))
    assert torch.isnan(a[1]).all() and torch.isnan(a[2]).all()
    assert torch.equal(h_out[3], h[3])  # (3 - 3) rstd = 0
    for r in (0, 3, 4, 5):
        assert torch.isfinite(a[r]).all() and torch.isfinite(h_out[r]).all()


def test_sandwich_slot_out_of_range(model):
    y, h = torch.randn(4, 256, device="cuda").to(BF), torch.randn(3, 256, device="cuda")
    slot = torch.tensor([[0], [4], [1]], dtype=torch.int32, device="cuda")
    w = torch.ones(3, 1, device="cuda")
    h_out = torch.zeros_like(h)
    with pytest.raises(fb.FlashBonError) as e:
        model.op_sandwich_norm(fb.make_sandwich(h, y=y, slot=slot, weight=w, h_out=h_out))
    assert e.value.status == fb.FB_EINVAL
    slot[1] = 3  # the next call finds nothing left of it
    model.op_sandwich_norm(fb.make_sandwich(h, y=y, slot=slot, weight=w, h_out=h_out))
    assert torch.allclose(h_out, h + y[slot[:, 0].long()].float())


# ---- router ---------------------------------------------------------------------------

def route64(logits, valid, k, renorm):
    """One token and one expert at a time, in numpy."""
    x = logits.float().cpu().numpy().astype(np.float64)
    T, E = x.shape
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, np.finfo(np.float32).max))
    if valid is not None:
        x[valid.cpu().numpy() == 0] = -np.inf
    expert, weight = np.full((T, k), -1), np.zeros((T, k))
    slot, lists = np.full((T, k), -1), [[] for _ in range(E)]
    for t in range(T):
        order = [e for e in np.argsort(-x[t], kind="stable") if x[t, e] > -np.inf]
        got = order[:k]
        if got:
            p = np.exp(x[t, got if renorm else order] - x[t, got[0]])
            weight[t, :len(got)] = np.exp(x[t, got] - x[t, got[0]]) / p.sum()
        expert[t, :len(got)] = got
        for j, e in enumerate(got):
            lists[e].append((t, j))
    offsets, token = np.cumsum([0] + [len(v) for v in lists]), np.full(T * k, -1)
    for e, v in enumerate(lists):
        for i, (t, j) in enumerate(v):
            slot[t, j], token[offsets[e] + i] = offsets[e] + i, t
    return expert, weight, slot, token, offsets


def route_buffers(T, E, k):
    i32 = dict(dtype=torch.int32, device="cuda")
    return (torch.full((T, k), 99, **i32), torch.full((T, k), 9.0, device="cuda"),
            torch.full((T, k), 99, **i32), torch.full((T * k,), 99, **i32), torch.full((E + 1,), 99, **i32))


def route_case(model, logits, k, valid=None, renorm=False):
    T, E = logits.shape
    out = route_buffers(T, E, k)
    r = fb.make_route(logits, *out, valid=valid, renorm=renorm)
    want = route64(logits, valid, k, renorm)
    for _ in range(2):  # (the second call finds the workspace as the first left it)
        model.op_route(r)
        for name, g, w in zip(("expert", "weight", "slot", "token", "offsets"), out, want):
            if name != "weight":
                assert np.array_equal(g.cpu().numpy(), w), name
        # exp of a difference: 2 units and 6e-8 of its size; a sum of E / 32 + 5 terms
        tol = 6e-8 * (4 + E / 32 + 5 + 40)
        assert (np.abs(out[1].cpu().numpy() - want[1]) <= tol * want[1] + 1e-37).all()


@pytest.mark.parametrize("T,E,k", [
    (1, 1, 1), (1, 8, 2), (1, 512, 16), (2, 3, 3), (5, 33, 4), (31, 8, 8), (100, 64, 8),
    (257, 256, 8), (513, 2, 1), (1000, 5, 2), (1560, 8, 2), (3000, 160, 6), (4097, 64, 1),
    (700, 512, 16), (9001, 16, 4), (33000, 8, 2),
])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_route(model, T, E, k, dtype):
    g = gen(T * 7 + E)
    x = torch.randn(T, E, generator=g, device="cuda")
    route_case(model, x.to(dtype), k, renorm=bool(T % 2))


@pytest.mark.parametrize("k", [1, 2, 6])
@pytest.mark.parametrize("E", [6, 40, 300])
def test_route_ties_masks_and_padding(model, E, k):
    g = gen(E + k)
    T = 400
    x = torch.randint(-3, 4, (T, E), generator=g, device="cuda").float() * 0.25  # many ties
    x[::5] = x[::5] * -0.0                                 # -0 and +0 are equal
    x[torch.rand(T, E, generator=g, device="cuda") < 0.6] = -math.inf
    x[3] = -math.inf                                       # no expert left
    x[7] = float("nan")
    x[8, 1], x[9, 2], x[9, 4] = float("nan"), math.inf, math.inf
    x[10] = torch.finfo(F32).min                           # the lowest value is a value
    x[11] = -math.inf
    x[11, E - 1] = -1e30
    route_case(model, x, k)
    route_case(model, x, k, renorm=True)
    valid = (torch.rand(T, generator=g, device="cuda") < 0.5).to(torch.uint8)
    x[valid == 0] = float("nan")
    route_case(model, x, k, valid=valid)
    route_case(model, x, k, valid=torch.zeros_like(valid))
    route_case(model, padded(x, 5, float("nan")), k, valid=valid * 3)


def test_route_all_to_one_expert(model):
    x = torch.full((5000, 64), -1.0, device="cuda")
    x[:, 63], x[:, 0] = 5.0, 4.0
    route_case(model, x, 2)


def test_route_without_tokens(model):
    out = route_buffers(0, 9, 2)
    model.op_route(fb.make_route(torch.zeros(0, 9, device="cuda"), *out))
    assert torch.equal(out[4].cpu(), torch.zeros(10, dtype=torch.int32))


# ---- products grouped by expert -------------------------------------------------------

def act64(v, act, n):
    if act in ("gelu", "geglu"):
        f = lambda x: 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))  # noqa: E731
    else:
        f = lambda x: x * torch.sigmoid(x)  # noqa: E731
    if act == "none":
        return v
    return f(v) if act == "gelu" else f(v[:, :n]) * v[:, n:]


def experts_case(model, sizes, n, k, act="none", gather=True, out_t=BF, bias=True, pad=0, seed=0,
                 spare=0, tail=0):
    """sizes: rows of each expert; spare: rows of out that no expert has; tail: elements
    between the rows."""
    g = gen(seed + 17 * n + k)
    E, S = len(sizes), sum(sizes)
    nw = 2 * n if act in ("swiglu", "geglu") else n
    T = max(1, S // 2 + 1) if gather else S + spare
    a = padded(torch.randn(max(T, 1), k, generator=g, device="cuda").to(BF), pad)
    w = torch.empty(E, nw, k, dtype=BF, device="cuda").normal_(0, k ** -0.5, generator=g)
    b = 0.3 * torch.randn(E, nw, generator=g, device="cuda") if bias else None
    off = torch.tensor([0] + list(np.cumsum(sizes)), dtype=torch.int32, device="cuda")
    idx = None
    if gather:
        idx = torch.full((S + spare,), -9, dtype=torch.int32, device="cuda")
        idx[:S] = torch.randint(0, T, (S,), generator=g, device="cuda").int()
    out = padded(torch.full((S + spare, n), 3.0, device="cuda").to(out_t), tail)
    args = fb.make_experts(a, w, off, out, index=idx, bias=b, act=act)
    model.op_expert_gemm(args)
    torch.cuda.synchronize()
    first = out.clone()
    r0 = 0
    for e, r in enumerate(sizes):
        if r:
            x = (a[idx[r0:r0 + r].long()] if gather else a[r0:r0 + r]).double()
            v = x @ w[e].double().T
            if bias:
                v = v + b[e].double()
            want = act64(v, act, n)
            tol = 4 * -(-k // 64) * 1.2e-7 * v.abs().max() * torch.ones_like(want)
            if act != "none":
                tol = tol * 1.2
                if out_t == BF:
                    tol = tol + 2.0 ** -10.9 * 0.5 * v[:, :n].abs()
                tol = tol + 6e-7 * v[:, :n].abs()
            if nw > n:
                tol = tol * v[:, n:].abs() + 1.2 * v[:, :n].abs() * 4 * -(-k // 64) * 1.2e-7 * v.abs().max()
            tol = tol + 3e-7 * want.abs()
            check(out[r0:r0 + r], want, tol, out_t)
        r0 += r
    assert torch.all(out[S:] == 3.0)
    if tail:
        base = out.as_strided((S + spare, n + tail), (n + tail, 1))
        assert torch.all(base[:, n:] == 7.0)
    model.op_expert_gemm(args)  # the same bits every time
    torch.cuda.synchronize()
    assert torch.equal(out, first)


ACTS = ["none", "gelu", "swiglu", "geglu"]


@pytest.mark.parametrize("sizes", [
    [1], [0, 1], [2, 0, 0, 3], [8, 8], [1, 1, 1, 1, 0, 1], [15, 17], [16, 33, 1], [40] * 3,
    [130, 0, 257, 5], [600], [300, 17, 0, 0, 255, 256],
])
@pytest.mark.parametrize("act", ACTS)
def test_experts_sizes(model, sizes, act):
    experts_case(model, sizes, 256, 128, act=act, seed=len(sizes))


@pytest.mark.parametrize("n,k", [(16, 8), (48, 40), (64, 64), (112, 72), (144, 1000), (256, 1536),
                                 (272, 136), (1000 // 16 * 16, 1032), (1536, 4096)])
@pytest.mark.parametrize("sizes", [[3, 0, 2], [70, 5, 141]])
@pytest.mark.parametrize("act", ["none", "geglu"])
@pytest.mark.parametrize("out_t", [BF, F32])
def test_experts_widths(model, n, k, sizes, act, out_t):
    experts_case(model, sizes, n, k, act=act, out_t=out_t, seed=1)


@pytest.mark.parametrize("n", [8, 24, 200, 1000])
def test_experts_n_multiple_of_8(model, n):
    experts_case(model, [20, 0, 3], n, 96, seed=2)
    experts_case(model, [20, 0, 3], n, 96, act="gelu", gather=False, out_t=F32, seed=2)


@pytest.mark.parametrize("out_t", [BF, F32])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gather", [True, False])
def test_experts_types_strides_and_spare_rows(model, act, gather, out_t):
    experts_case(model, [5, 0, 90, 260], 160, 200, act=act, gather=gather, out_t=out_t, pad=8,
                 spare=40, tail=16, seed=3)
    experts_case(model, [1, 2], 160, 200, act=act, gather=gather, out_t=out_t, pad=8, spare=4,
                 tail=16, bias=False, seed=4)
    experts_case(model, [0, 0], 160, 200, act=act, gather=gather, out_t=out_t, spare=4, seed=4)


@pytest.mark.parametrize("sizes,n,k,act", [
    ([390] * 8, 8960, 1536, "gelu"),
    ([390] * 8, 1536, 8960, "none"),
    ([0, 4000, 3, 700], 2048, 1536, "swiglu"),
    (list(range(64)), 1024, 1536, "swiglu"),
    ([(i * 37) % 11 for i in range(512)], 256, 512, "none"),
    ([2] * 4, 4096, 1536, "swiglu"),
    ([1, 1], 1536, 8960, "none"),
    ([13], 1536, 8960, "none"),
])
def test_experts_at_size(model, sizes, n, k, act):
    experts_case(model, sizes, n, k, act=act, gather=act != "none", seed=9)


@pytest.mark.parametrize("k", [4096, 8960])
@pytest.mark.parametrize("sizes", [[4, 1], [200, 31]])
def test_experts_long_sums_fp32(model, k, sizes):
    """A long K in fp32: the error is that of sums no longer than 80 K blocks."""
    a = torch.randn(sum(sizes), k, generator=gen(k), device="cuda").to(BF)
    w = torch.empty(2, 512, k, dtype=BF, device="cuda").normal_(0, k ** -0.5, generator=gen(k + 1))
    off = torch.tensor([0, sizes[0], sum(sizes)], dtype=torch.int32, device="cuda")
    out = torch.zeros(sum(sizes), 512, device="cuda")
    model.op_expert_gemm(fb.make_experts(a, w, off, out))
    want = torch.cat([a[:sizes[0]].double() @ w[0].double().T, a[sizes[0]:].double() @ w[1].double().T])
    assert ((out.double() - want).norm() / want.norm()).item() <= 80 * 1.2e-7


def test_experts_infinities_and_nan_stay_in_their_rows(model):
    a = torch.randn(40, 128, device="cuda").to(BF)
    a[3, 5], a[17, 0] = float("nan"), float("inf")
    w = torch.randn(2, 256, 128, device="cuda").to(BF)
    off = torch.tensor([0, 18, 40], dtype=torch.int32, device="cuda")
    out = torch.zeros(40, 256, dtype=BF, device="cuda")
    model.op_expert_gemm(fb.make_experts(a, w, off, out))
    fine = torch.isfinite(out.float()).all(1)
    assert not fine[3] and not fine[17] and fine.sum() == 38


@pytest.mark.parametrize("offsets", [[1, 5, 9], [0, 9, 5], [0, 5, 12], [0, -3, 9], [0, 1 << 30, 9]])
@pytest.mark.parametrize("rows", [10, 200])
def test_experts_bad_offsets(model, offsets, rows):
    scale = rows // 10
    a, w = torch.randn(rows, 64, device="cuda").to(BF), torch.randn(2, 64, 64, device="cuda").to(BF)
    out = torch.zeros(rows, 64, dtype=BF, device="cuda")
    off = torch.tensor([min(o * scale, 1 << 30) for o in offsets], dtype=torch.int32, device="cuda")
    with pytest.raises(fb.FlashBonError) as e:
        model.op_expert_gemm(fb.make_experts(a, w, off, out))
    assert e.value.status == fb.FB_EINVAL
    off.copy_(torch.tensor([0, 5, 9]) * scale)
    model.op_expert_gemm(fb.make_experts(a, w, off, out))


@pytest.mark.parametrize("rows", [4, 100])
@pytest.mark.parametrize("bad", [-1, 50, 1 << 30])
def test_experts_bad_index(model, rows, bad):
    a, w = torch.randn(50, 64, device="cuda").to(BF), torch.randn(2, 64, 64, device="cuda").to(BF)
    out = torch.zeros(rows, 64, dtype=BF, device="cuda")
    off = torch.tensor([0, 2, rows], dtype=torch.int32, device="cuda")
    idx = torch.zeros(rows, dtype=torch.int32, device="cuda")
    idx[rows - 1] = bad
    with pytest.raises(fb.FlashBonError) as e:
        model.op_expert_gemm(fb.make_experts(a, w, off, out, index=idx))
    assert e.value.status == fb.FB_EINVAL
    idx[rows - 1] = 49
    model.op_expert_gemm(fb.make_experts(a, w, off, out, index=idx))


def test_stream_budget_repeat_and_counters(model):
    """On a caller's stream and a few SMs, launched several times back to back."""
    st = torch.cuda.Stream()
    before = model.stats()
    try:
        model.set_stream(st)
        model.set_sm_budget(10)
        fb.fb_set_op_repeat(model.handle, 3)
        with torch.cuda.stream(st):
            experts_case(model, [70, 3, 400], 512, 256, act="swiglu", seed=30)
            sandwich_case(model, 500, 1536, parts=2, seed=30)
            route_case(model, torch.randn(700, 32, device="cuda"), 4)
    finally:
        fb.fb_set_op_repeat(model.handle, 1)
        model.set_sm_budget(0)
        model.set_stream(None)
    after = model.stats()
    n = {k: after[k]["launches"] - before[k]["launches"] for k in ("sandwich_norm", "route", "expert_gemm")}
    # (700 tokens over 32 experts are routed in three launches)
    assert n == {"sandwich_norm": 3, "route": 18, "expert_gemm": 6}


# ---- all of it ------------------------------------------------------------------------

@pytest.mark.parametrize("T,D,H,E,k,act,pad_to", [
    (1, 256, 512, 8, 2, "gelu", 8), (77, 256, 128, 4, 1, "swiglu", 128),
    (500, 1536, 1024, 16, 4, "swiglu", 128), (301, 144, 80, 5, 3, "geglu", 8),
])
def test_moe_forward(model, T, D, H, E, k, act, pad_to):
    """The feed-forward in one call against float64 on the router's own choice."""
    g = gen(T)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    nw = H if act == "gelu" else 2 * H
    rows = -(-E // pad_to) * pad_to
    router = (randn(rows, D) * D ** -0.5).to(BF)
    router[E:] = float("nan")  # ignored
    w1, w2 = (randn(E, nw, D) * D ** -0.5).to(BF), (randn(E, D, H) * H ** -0.5).to(BF)
    b1, b2 = 0.1 * randn(E, nw), 0.1 * randn(E, D)
    a, h = randn(T, D).to(BF), randn(T, D)
    gate, mul, add = randn(1, D), 0.3 * randn(1, D), 0.3 * randn(1, D)
    valid = torch.ones(T, dtype=torch.uint8, device="cuda")
    valid[T // 2 + 1:: 7] = 0
    moe = fb.make_moe(router, w1, w2, k, b1=b1, b2=b2, act=act, renorm=True)
    h_out, a_out = torch.zeros_like(h), torch.zeros_like(a)
    s = fb.make_sandwich(h, post="rms", gate=gate, resid_scale=0.875, h_out=h_out, pre="layer",
                         mul=mul, add=add, a=a_out)
    model.moe_forward(moe, a, s, valid=valid)

    logits = torch.zeros(T, rows, device="cuda")
    fb.fb_op_gemm(model.handle, T, rows, D, a, router, None, 2, logits)
    out = route_buffers(T, E, k)
    model.op_route(fb.make_route(logits[:, :E], *out, valid=valid, renorm=True))
    expert, weight = out[0].long(), out[1].double()
    y = torch.zeros(T, D, dtype=torch.float64, device="cuda")
    for e in range(E):
        t, j = (expert == e).nonzero(as_tuple=True)
        x = act64(a[t].double() @ w1[e].double().T + b1[e].double(), act, H)
        y[t] += weight[t, j, None] * (x @ w2[e].double().T + b2[e].double())
    u = norm64(y, y, "rms", 1e-6)[0]
    want = 0.875 * h.double() + gate.double() * u
    want_a = norm64(want, want, "layer", 1e-6)[0] * (1 + mul.double()) + add.double()
    # two bf16 roundings on the way (hidden rows, expert rows), each 2^-9 at most of what
    # the norm scales to one, random over a sum: 2^-9 sqrt(2) of the rms, five times that
    # at the largest of all elements
    assert ((h_out.double() - want) / gate.abs().clamp(min=1e-3)).abs().max().item() <= 5 * 2 ** -8.5 * max(1.0, u.abs().max().item())
    err = (h_out.double() - want).norm() / (gate.double() * u).norm()
    assert err.item() <= 2 ** -8.5
    assert ((a_out.double() - want_a).norm() / want_a.norm()).item() <= 2 ** -7.5


def test_moe_forward_rejects(model):
    w1, w2 = torch.zeros(4, 64, 32, dtype=BF, device="cuda"), torch.zeros(4, 32, 64, dtype=BF, device="cuda")
    moe = fb.make_moe(torch.zeros(8, 32, dtype=BF, device="cuda"), w1, w2, 2)
    h, a = torch.zeros(3, 32, device="cuda"), torch.zeros(3, 32, dtype=BF, device="cuda")
    with pytest.raises(fb.FlashBonError):  # y belongs to the call
        model.moe_forward(moe, a, fb.make_sandwich(h, y=a, h_out=h))
    with pytest.raises(fb.FlashBonError):  # more experts a token than there are
        model.moe_forward(fb.make_moe(torch.zeros(8, 32, dtype=BF, device="cuda"), w1, w2, 5), a,
                          fb.make_sandwich(h, h_out=h))
    with pytest.raises(fb.FlashBonError):  # fewer router rows than experts
        model.moe_forward(fb.make_moe(torch.zeros(0, 32, dtype=BF, device="cuda"), w1, w2, 2), a,
                          fb.make_sandwich(h, h_out=h))
    with pytest.raises(ValueError):
        model.moe_forward(moe, a[:2].contiguous(), fb.make_sandwich(h, h_out=h))


def test_example_runs_the_operators_together(capsys):
    """The example's chain of layers. Its error: three bf16 roundings (normed input, hidden
    rows, expert rows), each 2^-8 / sqrt(3) rms of its values, and a token whose second and
    third logits nearly tie may go elsewhere (few enough to fit in twice that)."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "moe_feed_forward.py")
    spec = importlib.util.spec_from_file_location("moe_feed_forward", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    assert mod.main(["--tokens", "200", "--layers", "2", "--experts", "6"]) <= 2 * 3 ** 0.5 * 2 ** -8 / 3 ** 0.5
    assert "off by" in capsys.readouterr().out


def test_experts_bad_index_in_copied_rows(model):
    """Groups so large that their rows are copied first."""
    a, w = torch.randn(50, 64, device="cuda").to(BF), torch.randn(2, 64, 64, device="cuda").to(BF)
    out = torch.zeros(1000, 64, dtype=BF, device="cuda")
    off = torch.tensor([0, 400, 1000], dtype=torch.int32, device="cuda")
    idx = torch.zeros(1000, dtype=torch.int32, device="cuda")
    idx[999] = 50
    with pytest.raises(fb.FlashBonError) as e:
        model.op_expert_gemm(fb.make_experts(a, w, off, out, index=idx))
    assert e.value.status == fb.FB_EINVAL
    idx[999] = 49
    model.op_expert_gemm(fb.make_experts(a, w, off, out, index=idx))
    want = a[idx.long()].double()
    want = torch.cat([want[:400] @ w[0].double().T, want[400:] @ w[1].double().T])
    check(out, want, 4 * 1.2e-7 * want.abs().max() * torch.ones_like(want), BF)


@pytest.mark.parametrize("sizes", [[200, 300, 0], [0, 1000], [193, 193]])
@pytest.mark.parametrize("act", ACTS)
def test_experts_copied_rows(model, sizes, act):
    experts_case(model, sizes, 144, 136, act=act, spare=7, pad=8, seed=40)


def test_scratch_failure_leaves_the_model_usable():
    """A scratch buffer that cannot be had: FB_ENOMEM, and the next call grows it."""
    with fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as m:
        x = torch.randn(3000, 40, device="cuda")
        out = route_buffers(3000, 40, 3)
        r = fb.make_route(x, *out)
        try:
            fb.fb_test_fail_alloc(0)
            with pytest.raises(fb.FlashBonError) as e:
                m.op_route(r)
            assert e.value.status == fb.FB_ENOMEM
        finally:
            fb.fb_test_fail_alloc(-1)
        route_case(m, x, 3)
        n = fb.fb_test_alloc_calls()
        m.op_route(r)
        assert fb.fb_test_alloc_calls() == n  # (nothing more to allocate)


def test_two_models_at_once():
    """Operators of two models from two threads, each with scratch and errors of its own."""
    import threading
    failed = []

    def work(seed):
        try:
            with fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as m:
                st = torch.cuda.Stream()
                m.set_stream(st)
                with torch.cuda.stream(st):
                    for i in range(4):
                        experts_case(m, [250, 3, 400 + seed], 256, 192, act="swiglu", seed=seed + i)
                        route_case(m, torch.randn(2000 + seed, 12, device="cuda"), 3)
                        sandwich_case(m, 700, 520, parts=2, seed=seed + i)
                m.set_stream(None)
        except BaseException as e:  # noqa: BLE001
            failed.append(e)
    ts = [threading.Thread(target=work, args=(k,)) for k in (50, 60)]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    assert not failed, failed


@pytest.mark.parametrize("sizes", [[200, 300, 0], [0, 1000], [193, 193]])
@pytest.mark.parametrize("n,act", [(1600, "none"), (1544, "gelu"), (800, "swiglu")])
@pytest.mark.parametrize("out_t", [BF, F32])
def test_experts_copied_rows_of_wide_experts(model, sizes, n, act, out_t):
    """Weight rows enough that large groups' rows are copied first."""
    experts_case(model, sizes, n, 136, act=act, out_t=out_t, spare=7, pad=8, seed=41)


def test_experts_bad_index_in_copied_rows_of_wide_experts(model):
    a, w = torch.randn(50, 64, device="cuda").to(BF), torch.randn(2, 1600, 64, device="cuda").to(BF)
    out = torch.zeros(1000, 1600, dtype=BF, device="cuda")
    off = torch.tensor([0, 400, 1000], dtype=torch.int32, device="cuda")
    idx = torch.zeros(1000, dtype=torch.int32, device="cuda")
    for bad in (-1, 50):
        idx[999] = bad
        with pytest.raises(fb.FlashBonError) as e:
            model.op_expert_gemm(fb.make_experts(a, w, off, out, index=idx))
        assert e.value.status == fb.FB_EINVAL
    idx[999] = 49
    for offsets in ([0, 1000, 400], [0, 400, 1001], [0, -1, 1000]):
        bad_off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        with pytest.raises(fb.FlashBonError) as e:
            model.op_expert_gemm(fb.make_experts(a, w, bad_off, out, index=idx))
        assert e.value.status == fb.FB_EINVAL
    model.op_expert_gemm(fb.make_experts(a, w, off, out, index=idx))
    want = a[idx.long()].double()
    want = torch.cat([want[:400] @ w[0].double().T, want[400:] @ w[1].double().T])
    check(out, want, 4 * 1.2e-7 * want.abs().max() * torch.ones_like(want), BF)


@pytest.mark.parametrize("n,k", [(1200, 8960), (520, 40000), (2100 // 8 * 8, 8000)])
@pytest.mark.parametrize("sizes", [[300, 17, 0, 520], [700, 600]])
def test_experts_weights_in_bands(model, n, k, sizes):
    """Experts of more weights than the product takes before it turns to the next tokens."""
    experts_case(model, sizes, n, k, seed=42)


@pytest.mark.parametrize("T,E", [(2, 3), (31, 64), (40, 100), (1000, 512), (17000, 8)])
def test_moe_forward_router_sizes(model, T, E):
    """Few and many rows and experts: the router's product takes other forms."""
    test_moe_forward(model, T, 256, 64, E, min(E, 2), "gelu", 128)


def test_moe_forward_router_on_two_sms(model):
    """As few SMs as a budget can name, and experts for more tiles than these take at once."""
    try:
        model.set_sm_budget(2)
        test_moe_forward(model, 20, 256, 64, 500, 2, "gelu", 8)
        test_moe_forward(model, 40, 256, 64, 500, 2, "gelu", 8)
    finally:
        model.set_sm_budget(0)


def activation_rows(act, out_t, rows):
    """Outputs of one expert at chosen values v before the activation, and v's two parts in float64.
    A row of `a` has one element that is not zero, so that products and sums are exact."""
    n, k = 2048, 64
    grid = torch.cat([torch.linspace(-20, 4, n - 256), torch.linspace(-90, 90, 256)]).to(BF)
    gated = act in ("swiglu", "geglu")
    w = torch.zeros(1, 2 * n if gated else n, k, dtype=BF, device="cuda")
    w[0, :n, 0] = grid.cuda()
    if gated:
        w[0, n:, 0] = torch.tensor([1.0, -2.5, 0.375, 96.0]).repeat(n // 4).to(BF).cuda()
    a = torch.zeros(rows, k, dtype=BF, device="cuda")
    a[:, 0] = torch.tensor([1.0, 0.75, 0.5, -1.0]).repeat(rows)[:rows].to(BF)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    out = torch.full((rows, n), 3.0, device="cuda").to(out_t)
    return a, w, off, out, a[:, :1].double() * w[0, :n, 0].double(), \
        a[:, :1].double() * w[0, n:, 0].double() if gated else None


@pytest.mark.parametrize("act", ["gelu", "swiglu", "geglu"])
@pytest.mark.parametrize("out_t", [BF, F32])
@pytest.mark.parametrize("rows", [4, 70])
def test_experts_activations_keep_their_precision(model, act, out_t, rows):
    """Every result within its type's rounding and a few fp32 units, the small ones at negative
    arguments too, where x / 2 (1 + tanh) cancels. x sigmoid(z), z = x or the tanh form's 2 u:
    z is off by up to 8 roundings, 2^-24 each, which the exponential turns into a relative error of
    8 |z| 2^-24; the exponential, 1 + it, the quotient and the product with `up` add less than 16
    units. Past z = -86 the quotient's divisor passes 2^125 and the result may be 0."""
    a, w, off, out, v, up = activation_rows(act, out_t, rows)
    model.op_expert_gemm(fb.make_experts(a, w, off, out, act=act))
    torch.cuda.synchronize()
    z = v if act == "swiglu" else 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
    want = v / (1 + torch.exp(-z))
    tol = 2.0 ** -24 * (16 + 8 * z.abs().clamp(max=90)) * want.abs() + (z < -86) * want.abs()
    if up is not None:
        want, tol = want * up, tol * up.abs()
    check(out, want, tol + 1e-37, out_t)


@pytest.mark.parametrize("rows", [12, 200, 8000])
@pytest.mark.parametrize("at,value", [(1, 1 << 30), (7, 1 << 30), (7, -4), (33, 1 << 30), (40, 1 << 30),
                                      (40, 0), (0, 2)])
def test_experts_bad_offsets_write_nothing(model, rows, at, value):
    """One bad offset among many good ones, met by any lane that looks: no group is taken out of
    such a table, in the streamed form, in tiles and with copied rows."""
    n = 1600 if rows == 8000 else 256
    a, w = torch.randn(rows, 64, device="cuda").to(BF), torch.randn(40, n, 64, device="cuda").to(BF)
    off = (torch.arange(41) * rows // 40).int()
    good = off.cuda()
    off[at] = value
    idx = torch.zeros(rows, dtype=torch.int32, device="cuda")
    for index in (None, idx):
        out = torch.full((rows, n), 3.0, device="cuda").to(BF)
        with pytest.raises(fb.FlashBonError) as e:
            model.op_expert_gemm(fb.make_experts(a, w, off.cuda(), out, index=index))
        assert e.value.status == fb.FB_EINVAL
        assert torch.all(out == 3.0)
        model.op_expert_gemm(fb.make_experts(a, w, good, out, index=index))
        assert torch.all((out != 3.0).any(1))


def test_stats_keep_to_the_room_that_they_have(model):
    """fb_get_stats writes the ten kinds that it had before there were more; fb_get_stats_n as
    many as it is told."""
    lib, size = fb.load_library(), ctypes.sizeof(fb.fb_kstat)
    arr = (fb.fb_kstat * 16)()
    p = ctypes.cast(arr, ctypes.c_void_p)
    for call, kinds in ((lambda: lib.fb_get_stats(model.handle, p), 10),
                        (lambda: lib.fb_get_stats_n(model.handle, p, 0), 0),
                        (lambda: lib.fb_get_stats_n(model.handle, p, 12), 12),
                        (lambda: lib.fb_get_stats_n(model.handle, p, 15), 15)):
        ctypes.memset(arr, 0xa5, 16 * size)
        assert call() == fb.FB_OK
        raw = bytes(arr)
        assert raw[kinds * size:] == b"\xa5" * ((16 - kinds) * size)
        assert all(a.launches == s["launches"] for a, s in zip(arr[:kinds], model.stats().values()))
        assert all(a.launches == 0 for a in arr[len(fb.KERNEL_KINDS):kinds])
    assert lib.fb_get_stats_n(model.handle, p, -1) == fb.FB_EINVAL


def test_one_row_of_a_wider_matrix(model):
    """A matrix of one row has no row stride: a view of an odd-sized buffer is taken."""
    k, n = 64, 128
    buf, obuf = torch.randn(3, k + 3, device="cuda").to(BF), torch.zeros(2, n + 5, dtype=BF, device="cuda")
    w = torch.randn(1, n, k, device="cuda").to(BF)
    off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    model.op_expert_gemm(fb.make_experts(buf[:1, :k], w, off, obuf[:1, :n]))
    want = buf[:1, :k].double() @ w[0].double().T
    check(obuf[:1, :n], want, 4 * 1.2e-7 * want.abs().max() * torch.ones_like(want), BF)
    assert torch.all(obuf[0, n:] == 0) and torch.all(obuf[1] == 0)
    one = torch.randn(k, device="cuda").to(BF).expand(1, k)  # (a row repeated: stride 0)
    model.op_expert_gemm(fb.make_experts(one, w, off, obuf[:1, :n]))
    want = one.double() @ w[0].double().T
    check(obuf[:1, :n], want, 4 * 1.2e-7 * want.abs().max() * torch.ones_like(want), BF)


def route_sorted(x, valid, k, renorm):
    """route64 for many tokens at once."""
    x = x.float().cpu().numpy().astype(np.float64)
    T, E = x.shape
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, np.finfo(np.float32).max))
    if valid is not None:
        x[valid.cpu().numpy() == 0] = -np.inf
    expert = np.argsort(-x, axis=1, kind="stable")[:, :k]
    top = np.take_along_axis(x, expert, 1)
    none = top == -np.inf
    shift = np.where(none[:, :1], 0, top[:, :1])
    e = np.where(none, 0, np.exp(top - shift))
    total = e.sum(1, keepdims=True) if renorm else np.exp(x - shift).sum(1, keepdims=True)
    weight = e / np.where(none[:, :1], 1, total)
    flat = np.where(none, E, expert).reshape(-1)
    order = np.argsort(flat, kind="stable")
    offsets = np.searchsorted(flat[order], np.arange(E + 1))
    token = np.where(flat[order] == E, -1, order // k)
    slot = np.empty(T * k, dtype=np.int64)
    slot[order] = np.arange(T * k)
    return (np.where(none, -1, expert), weight, np.where(none, -1, slot.reshape(T, k)), token, offsets)


@pytest.mark.parametrize("T,k,dtype,pad", [(12289, 1, F32, 0), (12300, 8, BF, 0), (20000, 8, F32, 0),
                                           (12289, 16, F32, 4), (20000, 16, BF, 3)])
@pytest.mark.parametrize("E", [9, 16, 17, 32, 33, 64, 100, 128, 200, 256, 300])
def test_route_of_a_pool(model, T, E, k, dtype, pad):
    """Several lanes a token, several experts a lane, with ties, masked experts, padding tokens and
    rows of any stride."""
    g = gen(T + E + k)
    k = min(k, E)
    x = torch.randn(T, E, generator=g, device="cuda")
    x = torch.where(torch.rand(T, E, generator=g, device="cuda") < 0.4, (2 * x).round() / 2, x)
    x[::3][torch.rand(x[::3].shape, generator=g, device="cuda") < 0.7] = -math.inf
    x[5:8], x[9, 1], x[9, 3] = float("nan"), math.inf, math.inf
    x[11], x[12, :] = -math.inf, 0.25
    x[12345 % T:] += 0.5
    valid = (torch.rand(T, generator=g, device="cuda") < 0.8).to(torch.uint8)
    x[valid == 0] = float("nan")
    x = x.to(dtype)
    if pad:
        x = padded(x, pad, float("nan"))
    out = route_buffers(T, E, k)
    for v, renorm in ((valid, False), (None, True)):
        want = route_sorted(x, v, k, renorm)
        model.op_route(fb.make_route(x, *out, valid=v, renorm=renorm))
        for name, got, w in zip(("expert", "weight", "slot", "token", "offsets"), out, want):
            if name != "weight":
                assert np.array_equal(got.cpu().numpy(), w), name
        tol = 6e-8 * (4 + E / 32 + 5 + 40)  # (as in route_case; a lane's own terms number E / 8 at most)
        tol = tol + 6e-8 * E / 8
        assert (np.abs(out[1].cpu().numpy() - want[1]) <= tol * want[1] + 1e-37).all()


@pytest.mark.parametrize("rows", [3, 700, 2500])
@pytest.mark.parametrize("D", [200, 256, 412, 512, 700, 768, 1000, 1024, 1280, 1500, 1536, 2000, 2048,
                               2816, 4000, 4096, 5120, 8192, 12000])
@pytest.mark.parametrize("odd", [0, 1])
def test_sandwich_forms(model, rows, D, odd):
    """Few, a middle number and many rows of every width's form, aligned and not, in modulation
    groups (which many rows take in segments) and with expert rows."""
    sandwich_case(model, rows, D - odd, group=max(1, rows // 3 - 1), seed=rows + D)
    sandwich_case(model, rows, D - odd, parts=2, post="layer", pre="rms", seed=rows - D, a_t=F32)


def launches(model, kind):
    return model.stats()[kind]["launches"]


@pytest.mark.parametrize("T,E,k,H,act", [(500, 4, 2, 1600, "gelu"), (901, 4, 2, 800, "swiglu")])
def test_moe_forward_copies_rows(model, T, E, k, H, act):
    """Groups and experts so large that the layer's rows are copied to expert order first."""
    before = launches(model, "small")
    test_moe_forward(model, T, 256, H, E, k, act, 128)
    assert launches(model, "small") == before + 1


def test_copied_rows_back_to_back(model):
    """Copies and products that follow one another without a wait reuse one scratch buffer: a
    product starts beside the copy, the next copy behind the product."""
    st = torch.cuda.Stream()
    before = launches(model, "small")
    try:
        model.set_stream(st)
        fb.fb_set_op_repeat(model.handle, 7)
        with torch.cuda.stream(st):
            experts_case(model, [900, 0, 700], 1600, 512, act="gelu", seed=50)
            experts_case(model, [300, 450], 800, 512, act="swiglu", out_t=F32, seed=51)
    finally:
        fb.fb_set_op_repeat(model.handle, 1)
        model.set_stream(None)
    assert launches(model, "small") == before + 28


def test_two_models_copy_rows_at_once():
    import threading
    failed = []

    def work(seed):
        try:
            with fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as m:
                st = torch.cuda.Stream()
                m.set_stream(st)
                before = launches(m, "small")
                with torch.cuda.stream(st):
                    for i in range(6):
                        experts_case(m, [500, 3, 700 + seed], 1600, 256, act="gelu", seed=seed + i)
                assert launches(m, "small") == before + 12
                m.set_stream(None)
        except BaseException as e:  # noqa: BLE001
            failed.append(e)
    ts = [threading.Thread(target=work, args=(k,)) for k in (70, 90)]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    assert not failed, failed


@pytest.mark.parametrize("k", [4096, 8960])
@pytest.mark.parametrize("sizes", [[4, 1], [20, 3], [200, 31]])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_experts_fp32_sums_are_short(model, k, sizes, act):
    """2-norm of the error of fp32 results. Four K blocks are 16 MMAs, the j-th of which cuts up to
    one unit (half of one on average, 0.7 x 6e-8) off a running sum of sqrt(j / 16) of the part's:
    16 x 2/3 x 4.3e-8 = 4.6e-7 of the part, and of the whole, as parts are independent. Up to 35
    parts added in order round another 0.7 x 3.4e-8 sqrt(35) = 1.4e-7: together less than 6e-7
    (one chain over K loses 6e-8 a K block: 3.8e-6 and 8.4e-6). The two factors of a gated result
    carry that each, and 3e-7 by the activation: 1e-6."""
    n = 512
    nw = 2 * n if act == "swiglu" else n
    a = torch.randn(sum(sizes), k, generator=gen(k), device="cuda").to(BF)
    w = torch.empty(2, nw, k, dtype=BF, device="cuda").normal_(0, k ** -0.5, generator=gen(k + 1))
    off = torch.tensor([0, sizes[0], sum(sizes)], dtype=torch.int32, device="cuda")
    out = torch.zeros(sum(sizes), n, device="cuda")
    model.op_expert_gemm(fb.make_experts(a, w, off, out, act=act))
    want = torch.cat([act64(x.double() @ w[e].double().T, act, n)
                      for e, x in enumerate((a[:sizes[0]], a[sizes[0]:]))])
    err = ((out.double() - want).norm() / want.norm()).item()
    assert err <= (6e-7 if act == "none" else 1e-6)


def test_experts_wait_runs_out_then_recovers(model):
    """Tiles of 2048 K blocks, all at once, take their mainloop 0.67 ms, past a limit of a microsecond
    on the epilogue's wait for it (whose clock is looked at every 64 polls, 0.3 ms): the call reports
    it, and the next ones are as before."""
    rows, n, k = 1024, 4864, 1 << 17
    a = torch.randn(rows, k, generator=gen(80), device="cuda").to(BF)
    w = torch.empty(1, n, k, dtype=BF, device="cuda").normal_(generator=gen(81))
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    out = torch.zeros(rows, n, dtype=BF, device="cuda")
    args = fb.make_experts(a, w, off, out)
    model.op_expert_gemm(args)
    ref = out.clone()
    torch.cuda.synchronize()
    fb.fb_set_device_wait_limit(1000)
    try:
        with pytest.raises(fb.FlashBonError) as e:
            model.op_expert_gemm(args)
    finally:
        fb.fb_set_device_wait_limit(0)
    assert e.value.status == fb.FB_ECUDA and "device wait timed out" in str(e.value)
    for _ in range(2):
        out.zero_()
        model.op_expert_gemm(args)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
    experts_case(model, [70, 3, 400], 512, 256, act="swiglu", seed=82)


def test_moe_forward_of_millions_of_rows(model):
    """More rows than a grid's second dimension has tiles for, with a router weight that is not
    padded: every row as in a call of few."""
    T, D, H, E = 65535 * 64 + 70, 16, 16, 2
    g = gen(90)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    router = torch.zeros(8, D, dtype=BF, device="cuda")
    router[:E] = randn(E, D).to(BF)
    moe = fb.make_moe(router, randn(E, H, D).to(BF), randn(E, D, H).to(BF), 1, renorm=True)
    a, h = randn(T, D).to(BF), randn(T, D)
    h_out, part = torch.zeros_like(h), torch.zeros(3000, D, device="cuda")
    model.moe_forward(moe, a, fb.make_sandwich(h, h_out=h_out))
    for r in (slice(0, 3000), slice(T - 3000, T)):
        model.moe_forward(moe, a[r].contiguous(), fb.make_sandwich(h[r].contiguous(), h_out=part))
        torch.cuda.synchronize()
        assert torch.equal(h_out[r], part)
    assert torch.all((h_out != h).any(1))


def test_gemm_of_millions_of_rows(model):
    M = 65535 * 64 + 70
    A, W = torch.randn(M, 8, device="cuda").to(BF), torch.randn(8, 8, device="cuda").to(BF)
    out = torch.zeros(M, 8, device="cuda")
    fb.fb_op_gemm(model.handle, M, 8, 8, A, W, None, 2, out)
    want = A.double() @ W.double().T
    # (eight products and sums of fp32, each off by 2^-24 of at most the terms' sizes)
    assert ((out.double() - want).abs() <= 16 * 2 ** -24 * (A.double().abs() @ W.double().abs().T)).all()


@pytest.mark.parametrize("k", [(1 << 20) + 40, 1 << 21])
@pytest.mark.parametrize("rows", [8, 40])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_experts_very_long_sums_bf16(model, k, rows, act):
    """bf16 results of a K so long that one chain of the tensor core loses more than their rounding,
    6e-9 of the result per element where all terms have one sign. Sums in parts: 16 cuts of up to
    2^-23 in each, and the parts (at most k / 192, in the streamed form) added in order, half of
    2^-24 each."""
    g = gen(k + rows)
    a = torch.randn(rows, k, generator=g, device="cuda").abs().to(BF)
    w = torch.empty(1, 32, k, dtype=BF, device="cuda").normal_(generator=g).abs_()
    n = 16 if act == "swiglu" else 32
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    out = torch.zeros(rows, n, dtype=BF, device="cuda")
    model.op_expert_gemm(fb.make_experts(a, w, off, out, act=act))
    v = sum(a[:, i:i + (1 << 19)].double() @ w[0, :, i:i + (1 << 19)].double().T
            for i in range(0, k, 1 << 19))
    want = act64(v, act, n)
    check(out, want, (2 if act == "swiglu" else 1) * (16 * 2 ** -23 + k / 192 * 2 ** -25) * want, BF)
