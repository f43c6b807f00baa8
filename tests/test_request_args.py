"""Arguments of the calls for several requests that are refused before anything runs (no GPU
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


def cross(**kw):
    d = dict(seqs=2, states=2, heads=4, kv_heads=2, head_dim=64, q_rows=8, kv_rows=8, q=P, ldq=256,
             k=P, ldk=128, v=P, ldv=128, q_offsets=P, kv_offsets=P, out=P, ldo=256)
    d.update(kw)
    return fb.fb_cross(**d)


@pytest.mark.parametrize("bad", [
    dict(seqs=-1), dict(seqs=4097, states=5000), dict(states=-1, kv_of=P), dict(states=1),
    dict(heads=0), dict(heads=4104, kv_heads=4104, ldq=1 << 20, ldo=1 << 20, ldk=1 << 20, ldv=1 << 20),
    dict(kv_heads=0), dict(kv_heads=3), dict(kv_heads=8), dict(heads=129, kv_heads=1, ldq=1 << 14, ldo=1 << 14),
    dict(head_dim=96), dict(head_dim=32), dict(head_dim=0), dict(q_rows=-1), dict(q_rows=(1 << 26) + 1),
    dict(kv_rows=-1), dict(kv_rows=(1 << 26) + 1), dict(scale=-1.0), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(q=None), dict(k=None), dict(v=None), dict(out=None),
    dict(q_offsets=None), dict(kv_offsets=None), dict(ldq=248), dict(ldk=120), dict(ldv=120),
    dict(ldo=0), dict(ldq=260), dict(ldk=132), dict(ldv=130), dict(ldo=257), dict(q=P + 8),
    dict(k=P + 2), dict(v=P + 4), dict(out=P + 8),
])
def test_cross_refusals(lib, bad):
    assert lib.fb_op_cross_attention(P, ctypes.byref(cross(**bad))) == fb.FB_EINVAL
    assert lib.fb_last_error()


def adapters(**kw):
    d = dict(rows=8, n=64, k=64, rank=8, adapters=2, segments=2, x=P, ldx=64, w=P, a=P, b=P,
             offsets=P, adapter=P, out=P, out_type=0, ldo=64)
    d.update(kw)
    return fb.fb_adapters(**d)


@pytest.mark.parametrize("bad", [
    dict(segments=-1), dict(segments=1025), dict(adapters=0), dict(adapters=-1), dict(rows=-1),
    dict(rows=(1 << 26) + 1), dict(n=0), dict(n=60), dict(k=0), dict(k=60), dict(rank=0),
    dict(rank=12), dict(rank=264), dict(n=(1 << 30) + 8, ldo=1 << 31), dict(k=(1 << 30) + 8, ldx=1 << 31),
    dict(act=2), dict(act=-1), dict(out_type=2), dict(resid=P, ldr=64), dict(gate=P),
    dict(x=None), dict(w=None), dict(a=None), dict(b=None), dict(out=None), dict(offsets=None),
    dict(adapter=None), dict(ldx=56), dict(ldx=68), dict(ldo=56), dict(ldo=66),
    dict(resid=P, ldr=56, out_type=1), dict(resid=P, ldr=66, out_type=1),
    dict(resid=P + 4, ldr=64, out_type=1), dict(x=P + 2), dict(w=P + 8), dict(a=P + 8),
    dict(b=P + 8), dict(out=P + 4),
])
def test_adapter_refusals(lib, bad):
    assert lib.fb_op_adapter_gemm(P, ctypes.byref(adapters(**bad))) == fb.FB_EINVAL
    assert lib.fb_last_error()


def test_null_arguments(lib):
    for f, make in ((lib.fb_op_cross_attention, cross), (lib.fb_op_adapter_gemm, adapters)):
        assert f(None, ctypes.byref(make())) == fb.FB_EINVAL
        assert f(P, None) == fb.FB_EINVAL


def test_calls_without_rows_do_nothing(lib):
    """No row, or no sequence: nothing is read, the model handle neither."""
    for c in (cross(q_rows=0, q=None, out=None), cross(seqs=0), cross(seqs=0, states=0, kv_rows=0, k=None, v=None)):
        assert lib.fb_op_cross_attention(P, ctypes.byref(c)) == fb.FB_OK
    for g in (adapters(rows=0, x=None, w=None, a=None, b=None, out=None), adapters(segments=0, adapter=None)):
        assert lib.fb_op_adapter_gemm(P, ctypes.byref(g)) == fb.FB_OK


def test_make_functions_check_their_tensors():
    torch = pytest.importorskip("torch")
    z, i = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA"):
        fb.make_cross(z, z, z, z, i, i)
    with pytest.raises(ValueError, match="whole heads"):
        fb.make_cross(z, z, z, z, i, i, head_dim=96)
    with pytest.raises(TypeError, match="CUDA"):
        fb.make_adapters(z, z, torch.zeros(1, 8, 128), torch.zeros(1, 4, 8), i, i[:1], z)


class _OnDevice:
    """A tensor's device and nothing else."""

    def __init__(self, index):
        self.device = type("device", (), {"index": index})


class _ModelOnDeviceOne:
    """The library of a model on device 1, whose calls count."""
    calls = 0

    def fb_model_device(self, model):
        return 1

    def fb_op_cross_attention(self, model, args):
        self.calls += 1
        return fb.FB_OK

    fb_op_adapter_gemm = fb_op_cross_attention


@pytest.mark.parametrize("call,make", [(fb.fb_op_cross_attention, cross), (fb.fb_op_adapter_gemm, adapters)])
def test_tensors_of_another_device_than_the_models(monkeypatch, call, make):
    """Refused by the binding before the library reads an address."""
    lib = _ModelOnDeviceOne()
    monkeypatch.setattr(fb, "load_library", lambda: lib)
    assert fb._one_device(q=_OnDevice(2), valid=None, k=_OnDevice(2)) == 2
    with pytest.raises(ValueError, match="several devices"):
        fb._one_device(q=_OnDevice(1), k=_OnDevice(0))
    args = make()
    args._device = 0
    with pytest.raises(ValueError, match="device 0.*device 1"):
        call(P, args)
    assert lib.calls == 0
    args._device = 1
    call(P, args)
    assert lib.calls == 1
    call(P, make())  # (filled in by hand: taken as it is)
    assert lib.calls == 2


def test_null_model_has_no_device(lib):
    assert lib.fb_model_device(None) == -1


def test_cross_refuses_more_states_than_rows_can_be(lib):
    for states in ((1 << 26) + 1, (1 << 31) - 1):
        assert lib.fb_op_cross_attention(P, ctypes.byref(cross(states=states, kv_of=P))) == fb.FB_EINVAL
        assert b"states" in lib.fb_last_error()


@pytest.mark.parametrize("call,make", [(fb.fb_op_cross_attention, cross), (fb.fb_op_adapter_gemm, adapters)])
def test_no_model_is_refused_by_the_library(lib, call, make):
    """As before the tensors' device was looked at (a closed Model has no handle)."""
    args = make()
    args._device = 0
    with pytest.raises(fb.FlashBonError) as e:
        call(None, args)
    assert e.value.status == fb.FB_EINVAL
