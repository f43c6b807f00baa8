"""The operators for several requests in one batch, through the public calls, against their
definitions in float64.

Tolerances, from the arithmetic (A = sum_j w_j |v_j|, the size of an attention result's terms):
  * cross attention: a key's weight and the result are rounded to bf16, 2^-8 of the term each:
    2^-8 (A + |o|). A score's fp32 sum may lose one unit, 1.2e-7 of its terms' sum, per 16 of
    head_dim; with the rounding of the exponent's argument (2^-24 of at most |scale s| + |m|) and
    the hardware exponential (2^-22) that is an absolute error d of the exponent, and 2 d A of the
    result (numerator and sum).
  * adapters: a product's fp32 sum may lose one unit, 1.2e-7 of its terms' sum, per 16 of K, and as
    much for each other operation on the way (bias, scale, the two sums' sum, activation: 16 of
    them at most). t = x A^T is a sum of two (fp32 results: three) bf16 values: 2^-16 (2^-24) of
    t, times |B|. bf16 results: 2^-8 of the value more. GELU's slope is at most 1.13, and its
    own error 2^-14 of the value for bf16 results.
"""
import math

import pytest
import torch

from paper_2607_04461_gb300 import flashbon as fb
from paper_2607_04461_gb300 import synth

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
NAN = float("nan")


@pytest.fixture(scope="module")
def model():
    m = fb.Model(synth.TINY, synth.make_weights(synth.TINY))
    yield m
    m.close()


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def whole(x):
    return torch.tensor(x, dtype=I32, device="cuda")


def offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def padded(x, pad, fill=NAN):
    if not pad:
        return x
    wide = torch.full((x.shape[0], x.shape[1] + pad), fill, dtype=x.dtype, device="cuda")
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


# ---- cross attention ------------------------------------------------------------------

class Cross:
    """Inputs, the result in float64 and its tolerance."""

    def __init__(self, queries, keys, heads=2, kv_heads=None, D=128, kv_of=None, valid=None, pad=0,
                 seed=0, scale=0.0, spread=1.0, extra_rows=3, packed=True):
        g = gen(seed)
        kv_heads = kv_heads or heads
        self.heads, self.kv_heads, self.D, self.scale = heads, kv_heads, D, scale
        self.q_at, self.k_at = offsets(queries), offsets(keys)
        self.of = list(range(len(queries))) if kv_of is None else list(kv_of)
        rows, kv_rows = self.q_at[-1] + extra_rows, self.k_at[-1] + extra_rows
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.q = padded((spread * randn(rows, heads * D)).to(BF), pad)
        kv = (randn(kv_rows, 2 * kv_heads * D)).to(BF)
        kv[self.k_at[-1]:] = NAN  # rows of no states
        self.valid = None
        if valid is not None:
            self.valid = (valid if torch.is_tensor(valid) else
                          (torch.rand(kv_rows, generator=g, device="cuda") >= valid)).to(torch.uint8).cuda()
            masked = self.valid == 0
            kv[masked] = torch.where(torch.rand(kv[masked].shape, generator=g, device="cuda") < 0.5,
                                     NAN, math.inf).to(BF)
        if packed:
            kv = padded(kv, pad)
            self.k, self.v = kv[:, :kv_heads * D], kv[:, kv_heads * D:]
        else:
            self.k, self.v = (padded(x.contiguous(), pad) for x in kv.chunk(2, 1))
        self.kv_of = None if kv_of is None else whole(self.of)
        self.out = padded(torch.full((rows, heads * D), 7.0, dtype=BF, device="cuda"), pad)
        self.args = fb.make_cross(self.q, self.k, self.v, self.out, whole(self.q_at), whole(self.k_at),
                                  head_dim=D, kv_of=self.kv_of, valid=self.valid, scale=scale)

    def want(self):
        D, G = self.D, self.heads // self.kv_heads
        scale = self.scale or 1 / math.sqrt(D)
        o = torch.full(self.out.shape, 7.0, dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(o)
        for s, u in enumerate(self.of):
            r = slice(self.q_at[s], self.q_at[s + 1])
            keys = torch.arange(self.k_at[u], self.k_at[u + 1], device="cuda")
            if self.valid is not None:
                keys = keys[self.valid[keys] != 0]
            o[r] = 0.0
            if r.start == r.stop or len(keys) == 0:
                continue
            for h in range(self.heads):
                c, kc = slice(h * D, (h + 1) * D), slice(h // G * D, (h // G + 1) * D)
                q, k, v = self.q[r, c].double(), self.k[keys, kc].double(), self.v[keys, kc].double()
                x = scale * (q @ k.T)
                w = torch.softmax(x, 1)
                o[r, c], size = w @ v, w @ v.abs()
                d = 1.2e-7 * (D / 16) * scale * (q.abs() @ k.abs().T) + 2.0 ** -22 + \
                    2.0 ** -23 * (x.abs() + x.abs().amax(1, keepdim=True))
                tol[r, c] = 2.0 ** -8 * (size + o[r, c].abs()) + 2 * d.amax(1, keepdim=True) * size
        return o, tol

    def check(self, model):
        model.op_cross_attention(self.args)
        want, tol = self.want()
        got = self.out.double()
        bad = ~((got - want).abs() <= tol)
        assert not bad.any(), (bad.nonzero()[:5].tolist(), got[bad][:5], want[bad][:5], tol[bad][:5])
        if self.out.stride(0) > self.out.shape[1]:  # what lies between the rows is as it was
            whole_rows = self.out.as_strided((self.out.shape[0] - 1, self.out.stride(0)), self.out.stride())
            assert whole_rows[:, self.out.shape[1]:].isnan().all()


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("queries,keys", [
    ([1], [1]), ([1], [512]), ([3], [2]), ([1, 1, 1, 1], [5, 128, 129, 1000]), ([128], [128]),
    ([129], [127]), ([256], [16]), ([257], [17]), ([31, 33], [33, 31]), ([300, 5, 260], [15, 640, 130]),
    ([0, 7, 0], [4, 0, 9]), ([0, 200, 1], [0, 300, 0]), ([5], [0]), ([1041], [77]), ([130] * 5, [512, 1, 64, 250, 113]),
])
def test_cross_lengths(model, D, queries, keys):
    Cross(queries, keys, D=D, seed=len(queries)).check(model)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 2), (3, 1), (12, 4), (5, 1), (8, 8), (64, 1), (100, 1), (128, 1)])
def test_cross_head_groups(model, D, heads, kv_heads):
    Cross([1, 40, 9, 130], [70, 200, 0, 33], heads=heads, kv_heads=kv_heads, D=D, seed=heads).check(model)


@pytest.mark.parametrize("D", [128, 64])
def test_cross_shared_states(model, D):
    """Sequences that share a prompt, prompts out of order, one that nobody asks."""
    Cross([20, 1, 300, 7, 0, 130], [100, 257, 30, 3], kv_of=[1, 0, 1, 3, 0, 1], D=D, seed=3).check(model)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("valid", [0.0, 0.3, 0.9, 1.0])
@pytest.mark.parametrize("queries,keys", [([1], [700]), ([200, 33], [300, 129]), ([9, 9, 300], [1, 16, 128])])
def test_cross_masked_keys(model, D, valid, queries, keys):
    """Keys and values that are masked hold NaN and infinities; at 1.0 no key is left."""
    Cross(queries, keys, heads=4, kv_heads=2, D=D, valid=valid, seed=int(valid * 10)).check(model)


@pytest.mark.parametrize("first", [True, False])
def test_cross_masked_tiles(model, first):
    """Whole stretches of keys masked before or behind the ones that are left."""
    valid = torch.ones(700 + 3)
    valid[:400] = 0
    Cross([150, 2], [640, 60], valid=valid if first else valid.flip(0), seed=5).check(model)


@pytest.mark.parametrize("pad,packed", [(8, True), (24, False), (0, False)])
def test_cross_strides(model, pad, packed):
    Cross([33, 200], [64, 190], heads=3, pad=pad, packed=packed, seed=7).check(model)
    Cross([1, 6], [64, 190], heads=6, kv_heads=3, D=64, pad=pad, packed=packed, seed=8).check(model)


@pytest.mark.parametrize("scale,spread", [(1.0, 1.0), (0.01, 1.0), (0.0, 12.0)])
def test_cross_scales(model, scale, spread):
    """Flat and peaked rows, scores of hundreds."""
    Cross([70, 140], [300, 65], scale=scale, spread=spread, seed=9).check(model)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("queries,heads,kv_heads", [([1], 8, 1), ([1], 4, 4), ([300], 2, 2), ([5, 700], 2, 1)])
def test_cross_long_states(model, D, queries, heads, kv_heads):
    """Long states, whose keys several SMs share."""
    Cross(queries, [9001] + [300] * (len(queries) - 1), heads=heads, kv_heads=kv_heads, D=D, seed=11).check(model)


def test_cross_many_sequences(model):
    rng = torch.Generator().manual_seed(1)
    queries = torch.randint(0, 4, (700,), generator=rng).tolist()
    keys = torch.randint(0, 60, (700,), generator=rng).tolist()
    Cross(queries, keys, heads=2, kv_heads=1, D=64, seed=12).check(model)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (3, 3), (20, 5)])
@pytest.mark.parametrize("valid", [None, 0.3])
@pytest.mark.parametrize("long", [False, True])
def test_cross_kv_heads_side_by_side(model, D, heads, kv_heads, valid, long):
    """More sequences of one query tile than SMs, among them some of several tiles, of no query and of
    no key; with one long prompt, whose keys several SMs share."""
    rng = torch.Generator().manual_seed(kv_heads)
    queries = torch.randint(0, 5, (160,), generator=rng).tolist()
    keys = torch.randint(0, 400, (160,), generator=rng).tolist()
    queries[7], queries[90], queries[91], queries[159] = 300, 130, 700, 129
    if long:
        keys[3], keys[100], queries[3] = 9000, 2500, 1
    keys[20] = 0
    Cross(queries, keys, heads=heads, kv_heads=kv_heads, D=D, valid=valid, seed=17).check(model)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("queries,keys", [([1] * 9, [700] * 9), ([2, 300, 1, 1, 40], [1, 130, 2000, 16, 513])])
def test_cross_on_few_sms(model, D, queries, keys):
    model.set_sm_budget(4)
    try:
        Cross(queries, keys, heads=6, kv_heads=3, D=D, valid=0.1, seed=18).check(model)
        Cross(queries, keys, heads=6, kv_heads=2, D=D, seed=19).check(model)
    finally:
        model.set_sm_budget(0)


def test_cross_same_result_every_time_and_on_few_sms(model):
    """The same bits on every call, with a repeat count, and on a budget of few SMs within the
    tolerance."""
    c = Cross([1, 513, 64], [4000, 700, 129], heads=4, kv_heads=2, valid=0.1, seed=13)
    c.check(model)
    first = c.out.clone()
    fb.fb_set_op_repeat(model.handle, 3)
    try:
        c.out.fill_(7.0)
        c.check(model)
    finally:
        fb.fb_set_op_repeat(model.handle, 1)
    assert torch.equal(first, c.out)
    model.set_sm_budget(8)
    try:
        c.out.fill_(7.0)
        c.check(model)
    finally:
        model.set_sm_budget(0)


def test_cross_on_another_stream(model):
    side = torch.cuda.Stream()
    c = Cross([70, 3], [200, 90], seed=14)
    torch.cuda.synchronize()
    model.set_stream(side.cuda_stream)
    try:
        c.check(model)
    finally:
        model.set_stream(None)


@pytest.mark.parametrize("q_at,k_at,of", [
    ([0, 5, 3], [0, 4, 8], None), ([1, 2, 3], [0, 4, 8], None), ([0, 5, 300], [0, 4, 8], None),
    ([0, 2, 5], [0, 9, 8], None), ([0, 2, 5], [2, 4, 8], None), ([0, 2, 5], [0, 4, 900], None),
    ([0, 2, 5], [0, 4, 8], [0, 2]), ([0, 2, 5], [0, 4, 8], [-1, 0]), ([0, -3, 5], [0, 4, 8], None),
    ([0, 2, -5], [0, 4, 8], None), ([0, 2, 5], [0, -4, 8], None),
])
def test_cross_bad_offsets(model, q_at, k_at, of):
    """Refused on the device; the model stays usable."""
    c = Cross([2, 3], [4, 4], kv_of=None if of is None else [0, 1], seed=15)
    q_bad, k_bad, of_bad = whole(q_at), whole(k_at), None if of is None else whole(of)
    args = fb.make_cross(c.q, c.k, c.v, c.out, q_bad, k_bad, kv_of=of_bad)
    with pytest.raises(fb.FlashBonError) as e:
        model.op_cross_attention(args)
    assert e.value.status == fb.FB_EINVAL
    c.out.fill_(7.0)
    c.check(model)


# ---- adapters -------------------------------------------------------------------------

class Adapters:
    def __init__(self, segments, of, N=256, K=192, rank=8, adapters=None, act="none", out_t=BF,
                 resid=False, gate=False, bias=True, scale=True, pad=0, seed=0, extra_rows=3,
                 in_place=False, big=1.0):
        g = gen(seed)
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        adapters = adapters or max(max(of, default=0), 0) + 1
        self.at, self.of, self.act = offsets(segments), list(of), act
        rows = self.at[-1] + extra_rows
        self.x = padded(randn(rows, K).to(BF), pad)
        self.w = (randn(N, K) * K ** -0.5).to(BF)
        self.a = (big * randn(adapters, rank, K) * K ** -0.5).to(BF)
        self.b = (randn(adapters, N, rank) * rank ** -0.5).to(BF)
        unused = [e for e in range(adapters) if e not in of]
        self.a[unused] = NAN  # nobody's adapters
        self.b[unused] = NAN
        self.scale = 0.5 + torch.rand(adapters, generator=g, device="cuda") if scale else None
        self.bias = randn(N) if bias else None
        self.gate = randn(N) if gate else None
        self.out = padded(torch.full((rows, N), 7.0, dtype=out_t, device="cuda"), pad)
        self.resid = None
        if resid:
            self.resid = self.out if in_place else padded(randn(rows, N), pad)
            if in_place:
                self.out.copy_(randn(rows, N))
        self.before = self.out.clone()
        self.resid_before = None if self.resid is None else self.resid.clone()
        self.args = fb.make_adapters(self.x, self.w, self.a, self.b, whole(self.at), whole(self.of),
                                     self.out, scale=self.scale, bias=self.bias, act=act,
                                     resid=self.resid, gate=self.gate)

    def want(self):
        f32 = self.out.dtype == F32
        K, N = self.w.shape[1], self.w.shape[0]
        x = self.x.double()
        y, size = x @ self.w.double().T, x.abs() @ self.w.double().abs().T
        if self.bias is not None:
            y, size = y + self.bias.double(), size + self.bias.double().abs()
        unit = 1.2e-7 * (K / 16 + 16)
        tol = unit * size
        for i, e in enumerate(self.of):
            if e < 0:
                continue
            r = slice(self.at[i], self.at[i + 1])
            s = 1.0 if self.scale is None else self.scale[e].double()
            a, b = self.a[e].double(), self.b[e].double()
            t, t_size = x[r] @ a.T, x[r].abs() @ a.abs().T
            y[r] += s * (t @ b.T)
            tol[r] += s * (unit * t_size @ b.abs().T + (2.0 ** (-24 if f32 else -16) + 1.2e-7 * (b.shape[1] / 16 + 4))
                           * (t.abs() @ b.abs().T))
        if self.act == "gelu":
            z = 2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)
            y = y * torch.sigmoid(z)
            tol = 1.13 * tol + (16 * 1.2e-7 if f32 else 2.0 ** -14) * y.abs() + 1e-30
        if self.gate is not None:
            y, tol = y * self.gate.double(), tol * self.gate.double().abs() + 1.2e-7 * (y * self.gate.double()).abs()
        if self.resid is not None:
            y = self.resid_before.double() + y
            tol = tol + 1.2e-7 * (self.resid_before.double().abs() + y.abs())
        tol = tol + (2.0 ** -24 if f32 else 2.0 ** -8) * y.abs()
        end = self.at[-1]
        y[end:], tol[end:] = self.before[end:].double(), 0.0
        return y, tol

    def check(self, model):
        model.op_adapter_gemm(self.args)
        self.compare()

    def compare(self):
        want, tol = self.want()
        got = self.out.double()
        bad = ~((got - want).abs() <= tol)
        assert not bad.any(), (int(bad.sum()), bad.nonzero()[:5].tolist(), got[bad][:5], want[bad][:5], tol[bad][:5])
        if self.out.stride(0) > self.out.shape[1]:
            whole_rows = self.out.as_strided((self.out.shape[0] - 1, self.out.stride(0)), self.out.stride())
            assert whole_rows[:, self.out.shape[1]:].isnan().all()


# (too many rows for streamed weights, segments too short for tiles of their own)
MANY = [2] * 45 + [0, 17, 1], [i % 3 - (i % 7 == 0) for i in range(48)]
LONG = [1400, 33, 700, 5, 900], [0, 1, -1, 0, 1]  # (long enough for t as K blocks of the product)


@pytest.mark.parametrize("out_t", [BF, F32])
@pytest.mark.parametrize("segments,of", [
    ([1], [0]), ([1], [-1]), ([2, 1], [1, 0]), ([1] * 9, [0, 1, 2, -1, 2, 2, 0, -1, 1]), ([33], [0]),
    ([16, 17], [0, 1]), ([0, 5, 0, 0, 11, 0], [0, 1, 2, -1, 0, 1]), ([300], [0]), ([129, 1, 257], [1, -1, 0]),
    ([40] * 6, [0, 1, 2, 3, 4, 5]), ([1] * 70, list(range(70))), ([3] * 50, [i % 7 - 1 for i in range(50)]),
    ([600, 2, 2, 2], [0, 1, 0, -1]), ([2000], [0]), ([700, 900, 31], [1, 0, -1]),
    ([1, 1500, 0, 15, 2049, 17], [0, 2, 1, 0, -1, 1]),
])
def test_adapter_segments(model, out_t, segments, of):
    Adapters(segments, of, out_t=out_t, seed=len(segments)).check(model)


@pytest.mark.parametrize("out_t", [BF, F32])
@pytest.mark.parametrize("segments,of", [([5], [0]), ([1] * 40, [i % 3 for i in range(40)]), MANY, ([200, 150], [0, 1]), LONG])
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 72, 128, 200, 256])
def test_adapter_ranks(model, out_t, segments, of, rank):
    Adapters(segments, of, out_t=out_t, rank=rank, seed=rank).check(model)


@pytest.mark.parametrize("out_t", [BF, F32])
@pytest.mark.parametrize("segments,of", [([1], [0]), ([20], [0]), ([1] * 40, [i % 3 for i in range(40)]), MANY, ([260, 90], [0, 1]), LONG])
@pytest.mark.parametrize("N,K", [(8, 8), (8, 520), (264, 8), (1000, 1032), (136, 64), (520, 72), (2048, 4104)])
def test_adapter_odd_sizes(model, out_t, segments, of, N, K):
    Adapters(segments, of, N=N, K=K, out_t=out_t, seed=N + K).check(model)


@pytest.mark.parametrize("segments,of", [([1], [0]), ([7, 9], [0, -1]), ([1] * 40, [i % 4 - 1 for i in range(40)]), MANY, ([300, 140], [1, 0]), LONG])
@pytest.mark.parametrize("kw", [
    dict(act="gelu"), dict(act="gelu", out_t=F32), dict(out_t=F32, resid=True, gate=True),
    dict(out_t=F32, resid=True, gate=True, in_place=True), dict(out_t=F32, resid=True),
    dict(out_t=F32, gate=True, act="gelu"), dict(bias=False, scale=False), dict(pad=8), dict(pad=24, out_t=F32),
    dict(pad=8, out_t=F32, resid=True, gate=True, act="gelu"), dict(big=30.0), dict(extra_rows=0),
])
def test_adapter_epilogues(model, segments, of, kw):
    Adapters(segments, of, N=328, K=448, rank=16, seed=21, **kw).check(model)


@pytest.mark.parametrize("out_t", [BF, F32])
@pytest.mark.parametrize("N,K", [(264, 1032), (264, 4160), (1536, 2056)])
@pytest.mark.parametrize("segments,of", [LONG, ([1300], [0]), ([80, 90, 70], [0, -1, 1]), ([3000, 1, 400], [0, 1, -1])])
def test_adapter_cut_tiles(model, out_t, N, K, segments, of):
    """Few tiles of a long sum, which several SM pairs share."""
    Adapters(segments, of, N=N, K=K, rank=40, out_t=out_t, seed=26).check(model)


@pytest.mark.parametrize("segments,of,K", [([1300], [0], 4160), ([3000, 1, 400], [0, 1, -1], 1032), LONG + (8200,)])
def test_adapter_cut_tiles_of_t_and_the_product(model, segments, of, K):
    """Both kernels' cut tiles share their scratch: every call gives the same bits."""
    c = Adapters(segments, of, N=1536, K=K, rank=16, seed=38)
    c.check(model)
    first = c.out.clone()
    for _ in range(20):
        c.out.copy_(c.before)
        model.op_adapter_gemm(c.args)
        torch.cuda.synchronize()
        assert torch.equal(first, c.out)


@pytest.mark.parametrize("sms", [2, 4, 6, 16])
@pytest.mark.parametrize("segments,of,N", [([100], [0], 264), ([100], [0], 8), ([90, 100, 3], [1, -1, 0], 520)])
def test_adapter_as_many_tiles_as_clusters(model, sms, segments, of, N):
    """Every cluster of the few has a tile of the product, or nearly: t's kernel still has one."""
    model.set_sm_budget(sms)
    try:
        Adapters(segments, of, N=N, K=64, rank=256, seed=39).check(model)
    finally:
        model.set_sm_budget(0)


def test_adapter_same_result_every_time_and_on_few_sms(model):
    for segments, of in (([1] * 50, [i % 5 for i in range(50)]), ([400, 300, 9], [0, -1, 1]), ([6], [0]), LONG):
        c = Adapters(segments, of, N=1536, K=1544, rank=16, seed=22)
        c.check(model)
        first = c.out.clone()
        fb.fb_set_op_repeat(model.handle, 3)
        try:
            c.check(model)
        finally:
            fb.fb_set_op_repeat(model.handle, 1)
        assert torch.equal(first, c.out)
        model.set_sm_budget(8)
        try:
            c.check(model)
        finally:
            model.set_sm_budget(0)


def test_adapter_on_another_stream(model):
    side = torch.cuda.Stream()
    c = Adapters([70, 3], [0, 1], seed=23)
    torch.cuda.synchronize()
    model.set_stream(side.cuda_stream)
    try:
        c.check(model)
    finally:
        model.set_stream(None)


@pytest.mark.parametrize("rows", [4, 40, 400, 4000])
@pytest.mark.parametrize("at,of", [
    ([0, 3, 2], [0, 0]), ([1, 2, 3], [0, 0]), ([0, 3, 50000], [0, 0]), ([0, 2, 4], [0, 2]), ([0, 2, 4], [-2, 0]),
    ([0, -1, 4], [0, 0]), ([0, 2, -4], [0, 0]),
])
def test_adapter_bad_segments(model, rows, at, of):
    """Refused on the device; the model stays usable."""
    c = Adapters([rows // 2, rows // 2], [0, 1], seed=24)
    args = fb.make_adapters(c.x, c.w, c.a, c.b, whole(at), whole(of), c.out)
    with pytest.raises(fb.FlashBonError) as e:
        model.op_adapter_gemm(args)
    assert e.value.status == fb.FB_EINVAL
    c.out.copy_(c.before)
    c.check(model)


def test_scratch_failure_leaves_the_model_usable():
    with fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as m:
        c = Adapters([300, 200], [0, 1], N=512, K=512, rank=16, seed=25)
        fb.fb_test_fail_alloc(0)
        try:
            with pytest.raises(fb.FlashBonError) as e:
                m.op_adapter_gemm(c.args)
            assert e.value.status == fb.FB_ENOMEM
        finally:
            fb.fb_test_fail_alloc(-1)
        c.out.copy_(c.before)
        c.check(m)


def test_cross_scratch_failure_leaves_the_model_usable():
    with fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as m:
        c = Cross([3], [4000], seed=26)  # (its keys shared by SMs, the parts in the scratch)
        fb.fb_test_fail_alloc(0)
        try:
            with pytest.raises(fb.FlashBonError) as e:
                m.op_cross_attention(c.args)
            assert e.value.status == fb.FB_ENOMEM
        finally:
            fb.fb_test_fail_alloc(-1)
        assert (c.out == 7.0).all()
        c.check(m)


def test_cross_wait_runs_out_then_recovers(model):
    """More than four items for each SM, of 32 key tiles: an item's place in the ring of four comes free
    after some 40 us, past a limit of a microsecond on that wait. The call reports it, and the next ones are as
    before, with whole items and with cut ones."""
    whole_items = Cross([200] * 300, [4096], heads=4, kv_of=[0] * 300, seed=27)
    cut_items = Cross([3, 40], [4000, 9000], seed=28)
    model.op_cross_attention(whole_items.args)
    ref = whole_items.out.clone()
    torch.cuda.synchronize()
    fb.fb_set_device_wait_limit(1000)
    try:
        with pytest.raises(fb.FlashBonError) as e:
            model.op_cross_attention(whole_items.args)
    finally:
        fb.fb_set_device_wait_limit(0)
    assert e.value.status == fb.FB_ECUDA and "device wait timed out" in str(e.value)
    for _ in range(2):
        whole_items.out.fill_(7.0)
        model.op_cross_attention(whole_items.args)
        torch.cuda.synchronize()
        assert torch.equal(whole_items.out, ref)
        cut_items.check(model)


def test_adapter_wait_runs_out_then_recovers(model):
    """Tiles of 2048 K blocks, all at once, take their mainloop 0.6 ms, past a limit of a microsecond on
    the epilogue's wait for it (whose clock is looked at every 64 polls, 0.3 ms): the call reports it,
    and the next ones are as before."""
    rows, n, k = 1024, 4864, 1 << 17
    g = gen(29)
    x = torch.randn(rows, k, generator=g, device="cuda").to(BF)
    w = torch.empty(n, k, dtype=BF, device="cuda").normal_(generator=g)
    a, b = (torch.randn(*size, generator=g, device="cuda").to(BF) for size in ((1, 8, k), (1, n, 8)))
    out = torch.zeros(rows, n, dtype=BF, device="cuda")
    args = fb.make_adapters(x, w, a, b, whole([0, rows]), whole([0]), out)
    model.op_adapter_gemm(args)
    ref = out.clone()
    torch.cuda.synchronize()
    fb.fb_set_device_wait_limit(1000)
    try:
        with pytest.raises(fb.FlashBonError) as e:
            model.op_adapter_gemm(args)
    finally:
        fb.fb_set_device_wait_limit(0)
    assert e.value.status == fb.FB_ECUDA and "device wait timed out" in str(e.value)
    for _ in range(2):
        out.zero_()
        model.op_adapter_gemm(args)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
    Adapters(*LONG, N=1536, K=1544, rank=16, seed=30).check(model)


def test_statistics_of_both(model):
    """Launches, operations and bytes under the operators' own kinds."""
    c, a = Cross([70, 3], [200, 90], seed=32), Adapters([300, 20], [0, 1], rank=16, seed=33)
    model.reset_stats()
    c.check(model)
    a.check(model)
    stats = model.stats()
    assert {kind: x["launches"] for kind, x in stats.items() if x["launches"]} == \
        {"cross_attention": 1, "adapter_gemm": 2}
    assert stats["cross_attention"]["flops"] > 0 and stats["adapter_gemm"]["bytes"] > 0


def test_two_models_at_once():
    """Calls of two models on streams of their own, from two threads: each has its scratch and counters."""
    import threading
    with fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as one, \
            fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as two:
        work = [(m, torch.cuda.Stream(), Cross([3, 300], [6000, 700], seed=34 + i),
                 Adapters(*LONG, N=1536, K=1544, rank=16, seed=36 + i)) for i, m in enumerate((one, two))]
        torch.cuda.synchronize()
        failures = []

        def run(m, stream, c, a):
            try:
                m.set_stream(stream.cuda_stream)
                for _ in range(20):
                    m.op_cross_attention(c.args)
                    m.op_adapter_gemm(a.args)
            except Exception as e:  # noqa: BLE001
                failures.append(e)

        threads = [threading.Thread(target=run, args=w) for w in work]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not failures
        for m, _, c, a in work:
            c.check(m)
            a.check(m)
            m.set_stream(None)


def test_cross_cache_past_32_bits(model):
    """Keys, values, masks and rows behind 2^32 elements: as in buffers of their own."""
    far, D, keys = 34_000_000, 64, 700
    g = gen(40)
    kv = torch.zeros(far + keys, 2 * D, dtype=BF, device="cuda")
    kv[far:] = torch.randn(keys, 2 * D, generator=g, device="cuda").to(BF)
    valid = torch.ones(far + keys, dtype=torch.uint8, device="cuda")
    valid[far + 5::3] = 0
    wide = 1 << 16  # row stride of q and out
    rows = 66_000
    q = torch.zeros(rows, wide, dtype=BF, device="cuda")[:, :2 * D]
    out = torch.full((rows, wide), 7.0, dtype=BF, device="cuda")[:, :2 * D]
    q[rows - 150:] = torch.randn(150, 2 * D, generator=g, device="cuda").to(BF)
    assert (rows - 150) * wide > 1 << 32 and far * 2 * D > 1 << 32
    model.op_cross_attention(fb.make_cross(q, kv[:, :D], kv[:, D:], out, whole([0, rows - 150, rows]),
                                           whole([0, 0, far, far + keys]), head_dim=D, kv_of=whole([0, 2]), valid=valid))
    near = torch.empty(150, 2 * D, dtype=BF, device="cuda")
    model.op_cross_attention(fb.make_cross(q[rows - 150:].contiguous(), kv[far:, :D].contiguous(),
                                           kv[far:, D:].contiguous(), near, whole([0, 150]), whole([0, keys]),
                                           head_dim=D, valid=valid[far:].contiguous()))
    assert (out[:rows - 150] == 0).all() and near.abs().sum() > 0
    assert torch.allclose(out[rows - 150:].double(), near.double(), rtol=2 ** -7, atol=2 ** -7)


@pytest.mark.parametrize("out_t", [BF, F32])
def test_adapter_results_past_32_bits(model, out_t):
    """More results than 2^32: the last rows as in a call of few."""
    rows, N, K, rank = (1 << 21) + 77, 2056, 16, 8
    g = gen(41)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, w, a, b = randn(rows, K).to(BF), randn(N, K).to(BF), randn(2, rank, K).to(BF), randn(2, N, rank).to(BF)
    out = torch.zeros(rows, N, dtype=out_t, device="cuda")
    assert rows * N > 1 << 32
    model.op_adapter_gemm(fb.make_adapters(x, w, a, b, whole([0, 1000, rows]), whole([0, 1]), out))
    for r, e in ((slice(0, 1000), 0), (slice(rows - 3000, rows), 1)):
        part = torch.zeros(r.stop - r.start, N, dtype=out_t, device="cuda")
        n = r.stop - r.start
        model.op_adapter_gemm(fb.make_adapters(x[r].contiguous(), w, a, b, whole([0, n]), whole([e]), part))
        size = x[r].double().abs() @ w.double().abs().T + \
            (x[r].double().abs() @ a[e].double().abs().T) @ b[e].double().abs().T
        unit = 2.0 ** -7 if out_t == BF else 1e-6
        assert ((out[r].double() - part.double()).abs() <= unit * part.double().abs() + 2.0 ** -15 * size).all()


# ---- together -------------------------------------------------------------------------

def test_cross_sublayer_of_several_requests(model):
    """The cross-attention part of a block for four requests, each with its own prompt and adapter
    (one without): keys and values from the prompts, queries, attention, the projection back into
    the gated residual stream; two candidates a request share its prompt."""
    D, H, rank, T = 256, 2, 16, 150
    prompts, adapter = [77, 5, 130, 31], [0, -1, 2, 1]
    g = gen(31)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    weights = {n: (randn(o, i) * i ** -0.5).to(BF) for n, o, i in
               (("q", D, D), ("kv", 2 * D, 192), ("o", D, D))}
    low = {n: ((randn(3, rank, w.shape[1]) * w.shape[1] ** -0.5).to(BF),
               (0.3 * randn(3, w.shape[0], rank) * rank ** -0.5).to(BF)) for n, w in weights.items()}
    h = randn(8 * T, D)
    a = h.to(BF)
    ctx = randn(sum(prompts), 192).to(BF)
    gate = randn(D)
    rows_at, per_candidate = whole(offsets([2 * T] * 4)), whole(offsets([T] * 8))
    ctx_at, e = whole(offsets(prompts)), whole(adapter)
    q, kv, o, out = (torch.zeros(n, w, dtype=t, device="cuda") for n, w, t in
                     ((8 * T, D, BF), (sum(prompts), 2 * D, BF), (8 * T, D, BF), (8 * T, D, F32)))
    model.op_adapter_gemm(fb.make_adapters(ctx, weights["kv"], *low["kv"], ctx_at, e, kv))
    model.op_adapter_gemm(fb.make_adapters(a, weights["q"], *low["q"], rows_at, e, q))
    model.op_cross_attention(fb.make_cross(q, kv[:, :D], kv[:, D:], o, per_candidate, ctx_at,
                                           kv_of=whole([0, 0, 1, 1, 2, 2, 3, 3])))
    model.op_adapter_gemm(fb.make_adapters(o, weights["o"], *low["o"], rows_at, e, out, resid=h, gate=gate))

    def project(x, name, i):
        y = x @ weights[name].double().T
        if adapter[i] >= 0:
            la, lb = (t[adapter[i]].double() for t in low[name])
            y = y + x @ la.T @ lb.T
        return y

    at = offsets(prompts)
    for i in range(4):
        rows = slice(2 * T * i, 2 * T * (i + 1))
        keys = project(ctx[at[i]:at[i + 1]].double(), "kv", i)
        query = project(a[rows].double(), "q", i)
        y = torch.cat([torch.softmax(query[:, c] @ keys[:, c].T / math.sqrt(128), 1) @ keys[:, D:][:, c]
                       for c in (slice(0, 128), slice(128, 256))], 1)
        step = gate.double() * project(y, "o", i)
        err = (out[rows].double() - h[rows].double() - step).norm() / step.norm()
        # four roundings to bf16 on the way (k, v, q, weights, o), 2^-8 each at most
        assert err < 5 * 2.0 ** -8, (i, err)


@pytest.mark.parametrize("D,queries,keys", [(128, [1] * 3, [4000, 1300, 900]), (128, [300], [5000]), (64, [2, 200], [6000, 2100])])
def test_cross_first_tiles_of_every_cta(model, D, queries, keys):
    """More key tiles for a CTA than its rings hold, from the first one on, over many launches: K's ring
    may be ahead of V's first load by as much as it holds."""
    c = Cross(queries, keys, heads=4, kv_heads=4, D=D, valid=0.1, seed=50)
    c.check(model)
    first = c.out.clone()
    fb.fb_set_op_repeat(model.handle, 50)
    try:
        for _ in range(4):
            c.out.fill_(7.0)
            model.op_cross_attention(c.args)
            torch.cuda.synchronize()
            assert torch.equal(first, c.out)
    finally:
        fb.fb_set_op_repeat(model.handle, 1)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (4, 2), (3, 1), (5, 1), (6, 2)])
@pytest.mark.parametrize("valid", [None, 0.2])
def test_cross_row_does_not_depend_on_its_neighbours(model, D, heads, kv_heads, valid):
    """A few rows of a tile, with other sequences' behind them, or none: the same bits. The neighbours'
    scores grow from key tile to key tile by far more than the rows' own."""
    c = Cross([5, 60, 1], [700, 300], heads=heads, kv_heads=kv_heads, D=D, kv_of=[0, 0, 1], valid=valid, seed=51)
    own = c.q[:5].clone()
    results = []
    for spread, signs in ((0.0, 1.0), (1.0, 1.0), (30.0, 1.0), (30.0, -1.0)):
        c.q[5:] = (spread * signs * torch.randn(c.q[5:].shape, generator=gen(52), device="cuda")).to(BF)
        assert torch.equal(c.q[:5], own)
        c.out.fill_(7.0)
        c.check(model)
        results.append(c.out[:5].clone())
    alone = Cross([5], [700, 300], heads=heads, kv_heads=kv_heads, D=D, kv_of=[0], seed=51, extra_rows=0)
    alone.args = fb.make_cross(own, c.k, c.v, alone.out, whole([0, 5]), whole([0, 700, 1000]), head_dim=D,
                               kv_of=whole([0]), valid=c.valid)
    model.op_cross_attention(alone.args)
    results.append(alone.out)
    for r in results[1:]:
        assert torch.equal(results[0], r)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("queries,heads,kv_heads,D,sms", [
    ([4096], 12, 12, 128, 0), ([5], 6, 6, 64, 4), ([1] * 200, 4, 2, 64, 0), ([3, 0, 300], 3, 1, 128, 2), ([1], 1, 1, 64, 0),
])
def test_cross_no_key_at_all(model, queries, heads, kv_heads, D, sms, masked):
    """Key buffers of no row, with more items than SMs and fewer: zeros."""
    rows = sum(queries) + 2
    q = torch.randn(rows, heads * D, generator=gen(53), device="cuda").to(BF)
    k = torch.empty(0, kv_heads * D, dtype=BF, device="cuda")
    out = torch.full_like(q, 7.0)
    valid = torch.empty(0, dtype=torch.uint8, device="cuda") if masked else None
    args = fb.make_cross(q, k, k, out, whole(offsets(queries)), whole([0] * (len(queries) + 1)), head_dim=D, valid=valid)
    model.set_sm_budget(sms)
    try:
        model.op_cross_attention(args)
    finally:
        model.set_sm_budget(0)
    assert (out[:-2] == 0).all() and (out[-2:] == 7.0).all()


def test_device_of_a_model(model):
    assert fb.fb_model_device(model.handle) == torch.cuda.current_device()
    args = Cross([3], [5], seed=54).args
    assert args._device == torch.cuda.current_device()
    args._device += 1  # as if the tensors lay on the next one
    with pytest.raises(ValueError, match="device"):
        model.op_cross_attention(args)


@pytest.mark.parametrize("queries,sms", [([3], 0), ([300] * 40, 0), ([5, 40], 2)])
def test_cross_bad_offset_of_a_state_that_nobody_asks_for(model, queries, sms):
    states = 100_000
    c = Cross(queries, [40, 100, 7], kv_of=[i % 2 for i in range(len(queries))], seed=55)
    of = c.kv_of
    k_at = torch.full((states + 1,), 147, dtype=I32, device="cuda")
    k_at[:3] = whole([0, 40, 140])
    c.args = fb.make_cross(c.q, c.k, c.v, c.out, whole(c.q_at), k_at, kv_of=of)
    model.set_sm_budget(sms)
    try:
        c.check(model)
        for at, n in ((3, 139), (31, 141), (32, 146), (33, 148 + len(c.k)), (5000, 12), (12345, -1), (99_999, 1 << 30), (states, 146)):
            bad = k_at.clone()
            bad[at] = n
            with pytest.raises(fb.FlashBonError) as e:
                model.op_cross_attention(fb.make_cross(c.q, c.k, c.v, c.out, whole(c.q_at), bad, kv_of=of))
            assert e.value.status == fb.FB_EINVAL, (at, n)
        c.out.fill_(7.0)
        c.check(model)
    finally:
        model.set_sm_budget(0)


def test_cross_very_many_states(model):
    """2^24 states, two of which are asked for: no role waits for the check of the others (under a limit of
    3 ms for each wait; one warp alone would look at them for longer)."""
    c = Cross([3, 200], [40, 100], seed=56)
    k_at = torch.full(((1 << 24) + 1,), 140, dtype=I32, device="cuda")
    k_at[:2] = whole([0, 40])
    c.args = fb.make_cross(c.q, c.k, c.v, c.out, whole(c.q_at), k_at, kv_of=whole([0, 1]))
    torch.cuda.synchronize()
    fb.fb_set_device_wait_limit(3_000_000)
    try:
        c.check(model)
    finally:
        fb.fb_set_device_wait_limit(0)


def test_cross_very_long_state_loses_nothing(model):
    """2^22 keys on two SMs, values of one sign: a single accumulator would lose 1 % to the tensor core's
    truncated sums. The result is rounded to bf16, 2^-8, and its sums lose 1e-4 at most."""
    keys, D = 1 << 22, 64
    g = gen(57)
    k = torch.zeros(keys, D, dtype=BF, device="cuda")
    v = (1 + torch.rand(keys, D, generator=g, device="cuda")).to(BF)
    q, out = torch.ones(3, D, dtype=BF, device="cuda"), torch.zeros(3, D, dtype=BF, device="cuda")
    args = fb.make_cross(q, k, v, out, whole([0, 3]), whole([0, keys]), head_dim=D)
    want = v.double().mean(0)
    for sms in (2, 0):
        model.set_sm_budget(sms)
        try:
            model.op_cross_attention(args)
        finally:
            model.set_sm_budget(0)
        assert ((out.double() - want).abs() <= (2.0 ** -8 + 1e-4) * want).all(), sms


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("valid", [None, 0.4])
@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (2, 2), (3, 3)])
@pytest.mark.parametrize("queries,sms", [([3] * 5, 2), ([1, 2, 1, 1, 2], 4), ([140, 0, 300, 5, 1], 2), ([2, 0, 130, 2, 1], 0)])
def test_cross_long_states_in_parts(model, D, valid, heads, kv_heads, queries, sms):
    """States on both sides of the parts' 128 key tiles, and of several parts, with scores whose maxima grow;
    whole items, cut ones and key heads side by side."""
    model.set_sm_budget(sms)
    try:
        Cross(queries, [16384, 16385, 33000, 4, 49153], heads=heads, kv_heads=kv_heads, D=D, valid=valid,
              scale=0.5, seed=58).check(model)
    finally:
        model.set_sm_budget(0)


def test_cross_long_state_masked_to_its_last_part(model):
    """Nothing left in the first parts, then nothing in the last ones."""
    valid = torch.zeros(70_000 + 3)
    valid[60_000:60_100] = 1
    for v in (valid, valid.flip(0)):
        model.set_sm_budget(2)
        try:
            Cross([1, 200], [70_000], kv_of=[0, 0], D=64, valid=v, seed=59).check(model)
        finally:
            model.set_sm_budget(0)


def test_cross_long_states_same_result_every_time(model):
    c = Cross([200] * 40, [70_000], kv_of=[0] * 40, D=64, valid=0.1, seed=60)
    model.op_cross_attention(c.args)
    first = c.out.clone()
    for _ in range(5):
        c.out.fill_(7.0)
        model.op_cross_attention(c.args)
        torch.cuda.synchronize()
        assert torch.equal(first, c.out)


def test_both_on_sm_partitions_side_by_side():
    """A model on each part of the GPU, with its budget, two threads at once: the results of the whole one
    within the tolerance, the same bits every time."""
    import threading
    with fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as one, \
            fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as two, fb.SmSplit(40) as sp:
        work = [(m, part, Cross([3, 300, 5], [6000, 700, 70_000], seed=61 + part),
                 [Adapters(*a, N=1536, K=1544, rank=16, seed=63 + part) for a in (LONG, MANY, ([6], [0]))])
                for part, m in enumerate((one, two))]
        torch.cuda.synchronize()
        failures = []

        def run(m, part, c, adapters):
            try:
                m.set_stream(sp.streams[part])
                m.set_sm_budget(sp.sms[part])
                for _ in range(10):
                    m.op_cross_attention(c.args)
                    for a in adapters:
                        m.op_adapter_gemm(a.args)
            except Exception as e:  # noqa: BLE001
                failures.append(e)

        threads = [threading.Thread(target=run, args=w) for w in work]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not failures
        for m, _, c, adapters in work:
            first = c.out.clone()
            c.check(m)
            assert torch.equal(first, c.out)
            for a in adapters:
                first = a.out.clone()
                a.check(m)
                assert torch.equal(first, a.out)
            m.set_stream(None)
