"""Arguments of the mixture-of-experts calls that are refused before anything runs (no GPU
needed: the model handle and the pointers are never read)."""
import ctypes
import os

import pytest

from paper_2607_04461_gb300 import flashbon as fb

P = 4096  # an aligned address; a refused call reads nothing there


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2607_04461_gb300 import build
        build.build()
    return fb.load_library()


def sandwich(**kw):
    d = dict(rows=4, dim=64, h=P, h_type=1, ldh=64, y=P, y_type=0, y_rows=4, parts=0, ldy=64,
             post=1, pre=2, resid_scale=1.0, h_out=P, ldho=64, a=P, a_type=0, lda=64, ldm=64)
    d.update(kw)
    return fb.fb_sandwich(**d)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(dim=0), dict(dim=16385, ldh=20000, ldy=20000, ldho=20000, lda=20000),
    dict(h=None), dict(h_out=None, a=None), dict(h_type=2), dict(y_type=-1), dict(a_type=7),
    dict(post=3), dict(pre=-1), dict(ldh=63), dict(ldho=0), dict(lda=63), dict(ldy=63),
    dict(group_rows=-1), dict(group_rows=2, gate=P, ldm=63), dict(parts=-1),
    dict(parts=17, slot=P, weight=P), dict(parts=2), dict(parts=2, slot=P), dict(y_rows=3),
    dict(y_rows=-1, parts=1, slot=P, weight=P),
])
def test_sandwich_refusals(lib, bad):
    assert lib.fb_op_sandwich_norm(P, ctypes.byref(sandwich(**bad))) == fb.FB_EINVAL
    assert lib.fb_last_error()


def route(**kw):
    d = dict(tokens=4, experts=8, top_k=2, logits=P, logits_type=1, ldl=8, expert=P, weight=P,
             slot=P, token=P, offsets=P)
    d.update(kw)
    return fb.fb_route(**d)


@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(experts=0), dict(experts=513, ldl=513), dict(top_k=0), dict(top_k=9),
    dict(top_k=17, experts=64, ldl=64), dict(tokens=(1 << 25) + 1), dict(logits=None),
    dict(expert=None), dict(weight=None), dict(slot=None), dict(token=None), dict(offsets=None),
    dict(logits_type=2), dict(ldl=7),
])
def test_route_refusals(lib, bad):
    assert lib.fb_op_route(P, ctypes.byref(route(**bad))) == fb.FB_EINVAL
    assert lib.fb_last_error()


def experts(**kw):
    d = dict(experts=2, n=64, k=64, max_rows=8, a_rows=8, a=P, lda=64, offsets=P, w=P, act=0, out=P,
             out_type=0, ldo=64)
    d.update(kw)
    return fb.fb_experts(**d)


@pytest.mark.parametrize("bad", [
    dict(experts=0), dict(experts=513), dict(n=0), dict(k=0), dict(n=60), dict(k=60),
    dict(n=56, act=2), dict(act=4), dict(act=-1), dict(max_rows=-1), dict(max_rows=(1 << 26) + 1),
    dict(a_rows=7), dict(a_rows=-1), dict(a_rows=0, index=P), dict(a=None), dict(w=None),
    dict(out=None), dict(offsets=None), dict(out_type=3), dict(lda=56), dict(lda=68),
    dict(ldo=56), dict(ldo=66), dict(a=P + 2), dict(w=P + 8), dict(out=P + 4),
])
def test_experts_refusals(lib, bad):
    assert lib.fb_op_expert_gemm(P, ctypes.byref(experts(**bad))) == fb.FB_EINVAL
    assert lib.fb_last_error()


def test_null_arguments(lib):
    for f, make in ((lib.fb_op_sandwich_norm, sandwich), (lib.fb_op_route, route),
                    (lib.fb_op_expert_gemm, experts)):
        assert f(None, ctypes.byref(make())) == fb.FB_EINVAL
        assert f(P, None) == fb.FB_EINVAL
    moe = fb.fb_moe(dim=64, hidden=64, experts=4, top_k=2, router_rows=8, router_w=P, w1=P, w2=P)
    assert lib.fb_moe_forward(P, ctypes.byref(moe), None, None, None) == fb.FB_EINVAL


@pytest.mark.parametrize("bad", [
    dict(dim=32), dict(hidden=0), dict(hidden=72), dict(experts=9), dict(top_k=0), dict(top_k=5),
    dict(router_rows=12), dict(act=9), dict(router_w=None), dict(w1=None), dict(w2=P + 8),
])
def test_moe_forward_refusals(lib, bad):
    d = dict(dim=64, hidden=64, experts=4, top_k=2, router_rows=8, router_w=P, w1=P, w2=P)
    d.update(bad)
    s = sandwich(y=None)
    assert lib.fb_moe_forward(P, ctypes.byref(fb.fb_moe(**d)), P, None,
                              ctypes.byref(s)) == fb.FB_EINVAL


def test_make_functions_check_their_tensors():
    torch = pytest.importorskip("torch")
    with pytest.raises(TypeError, match="CUDA"):
        fb.make_sandwich(torch.zeros(2, 8))
    with pytest.raises(TypeError, match="CUDA"):
        fb.make_experts(torch.zeros(2, 8), torch.zeros(1, 8, 8), None, torch.zeros(2, 8))


@pytest.mark.parametrize("bad", [
    dict(n=(1 << 30) + 8, ldo=(1 << 30) + 8), dict(n=(1 << 31) - 8, ldo=1 << 31),
    dict(n=(1 << 29) + 16, ldo=1 << 30, act=2), dict(n=1 << 30, ldo=1 << 30, act=3),
    dict(k=(1 << 30) + 8, lda=(1 << 30) + 8), dict(k=(1 << 31) - 8, lda=1 << 31),
])
def test_experts_sizes_past_the_kernels_counters(lib, bad):
    """Weight rows or a K that the kernels' 32-bit counters would not hold."""
    assert lib.fb_op_expert_gemm(P, ctypes.byref(experts(**bad))) == fb.FB_EINVAL
    assert b"at most" in lib.fb_last_error()
    moe = fb.fb_moe(dim=64, hidden=(1 << 29) + 16, experts=4, top_k=2, router_rows=8, router_w=P,
                    w1=P, w2=P, act=2)
    assert lib.fb_moe_forward(P, ctypes.byref(moe), P, None,
                              ctypes.byref(sandwich(y=None))) == fb.FB_EINVAL
    assert b"at most" in lib.fb_last_error()
