"""ctypes binding of libflashbon.so (include/flashbon.h). Argument marshalling only:
every step of the draft path runs in the library's CUDA kernels. There is no CPU
fallback: if the library is missing, loading raises.

Buffers may be numpy arrays (host memory) or torch tensors (host or CUDA); they are
passed to the library as raw pointers and must be contiguous float32 / uint8 / int32.
The make_sandwich, make_route and make_experts arguments are CUDA tensors, whose rows may be
further apart than they are long.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

from . import synth

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libflashbon.so")

FB_OK, FB_EINVAL, FB_ENOMEM, FB_ECUDA, FB_EPLAN, FB_ESTATE = range(6)
KERNEL_KINDS = ["gemm_tc", "gemm_simt", "attn_self", "attn_cross", "ln_mod", "qk_norm_rope",
                "proxy_add", "patch_embed", "head_euler", "small", "sandwich_norm", "route",
                "expert_gemm", "cross_attention", "adapter_gemm"]
K = {name: i for i, name in enumerate(KERNEL_KINDS)}


class FlashBonError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"flashbon status {status}: {msg}")
        self.status = status


class fb_cfg(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in (
        "depth", "dim", "heads", "head_dim", "ffn", "text_len", "text_dim", "latent_c",
        "latent_h", "latent_w", "patch", "max_n", "freq_dim")] + [
        ("eps_ln", ctypes.c_float), ("eps_rms", ctypes.c_float), ("rope_theta", ctypes.c_float)]


class fb_sampler_opts(ctypes.Structure):
    _fields_ = [("guidance", ctypes.c_float), ("text_uncond", ctypes.c_void_p),
                ("sde_a", ctypes.c_float), ("noise", ctypes.c_void_p),
                ("keep_state", ctypes.c_int), ("state", ctypes.c_void_p),
                ("warm_steps", ctypes.c_int)]


class fb_kstat(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_uint64), ("ms", ctypes.c_double),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double)]


class fb_sandwich(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("dim", ctypes.c_int),
                ("h", ctypes.c_void_p), ("h_type", ctypes.c_int), ("ldh", ctypes.c_int64),
                ("y", ctypes.c_void_p), ("y_type", ctypes.c_int), ("y_rows", ctypes.c_int),
                ("parts", ctypes.c_int), ("ldy", ctypes.c_int64), ("slot", ctypes.c_void_p),
                ("weight", ctypes.c_void_p), ("post", ctypes.c_int), ("post_eps", ctypes.c_float),
                ("post_w", ctypes.c_void_p), ("post_b", ctypes.c_void_p),
                ("gate", ctypes.c_void_p), ("resid_scale", ctypes.c_float),
                ("h_out", ctypes.c_void_p), ("ldho", ctypes.c_int64), ("pre", ctypes.c_int),
                ("pre_eps", ctypes.c_float), ("mul_base", ctypes.c_float),
                ("mul", ctypes.c_void_p), ("add", ctypes.c_void_p), ("a", ctypes.c_void_p),
                ("a_type", ctypes.c_int), ("lda", ctypes.c_int64), ("group_rows", ctypes.c_int),
                ("ldm", ctypes.c_int64)]


class fb_route(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int), ("experts", ctypes.c_int), ("top_k", ctypes.c_int),
                ("logits", ctypes.c_void_p), ("logits_type", ctypes.c_int),
                ("ldl", ctypes.c_int64), ("valid", ctypes.c_void_p), ("renorm", ctypes.c_int),
                ("expert", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("slot", ctypes.c_void_p), ("token", ctypes.c_void_p),
                ("offsets", ctypes.c_void_p)]


class fb_experts(ctypes.Structure):
    _fields_ = [("experts", ctypes.c_int), ("n", ctypes.c_int), ("k", ctypes.c_int),
                ("max_rows", ctypes.c_int), ("a_rows", ctypes.c_int), ("a", ctypes.c_void_p),
                ("lda", ctypes.c_int64), ("index", ctypes.c_void_p), ("offsets", ctypes.c_void_p),
                ("w", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("act", ctypes.c_int),
                ("out", ctypes.c_void_p), ("out_type", ctypes.c_int), ("ldo", ctypes.c_int64)]


class fb_moe(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("dim", "hidden", "experts", "top_k", "renorm", "act",
                                            "router_rows")] + [
        (n, ctypes.c_void_p) for n in ("router_w", "w1", "w2", "b1", "b2")]


class fb_cross(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("seqs", "states", "heads", "kv_heads", "head_dim",
                                            "q_rows", "kv_rows")] + [
        ("q", ctypes.c_void_p), ("ldq", ctypes.c_int64), ("k", ctypes.c_void_p),
        ("ldk", ctypes.c_int64), ("v", ctypes.c_void_p), ("ldv", ctypes.c_int64),
        ("q_offsets", ctypes.c_void_p), ("kv_offsets", ctypes.c_void_p),
        ("kv_of", ctypes.c_void_p), ("valid", ctypes.c_void_p), ("scale", ctypes.c_float),
        ("out", ctypes.c_void_p), ("ldo", ctypes.c_int64)]


class fb_adapters(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("rows", "n", "k", "rank", "adapters", "segments")] + [
        ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64)] + [
        (n, ctypes.c_void_p) for n in ("w", "a", "b", "bias", "scale", "offsets", "adapter")] + [
        ("act", ctypes.c_int), ("resid", ctypes.c_void_p), ("ldr", ctypes.c_int64),
        ("gate", ctypes.c_void_p), ("out", ctypes.c_void_p), ("out_type", ctypes.c_int),
        ("ldo", ctypes.c_int64)]


FB_BF16, FB_F32 = 0, 1
NORMS = {"none": 0, "rms": 1, "layer": 2}
ACTS = {"none": 0, "gelu": 1, "swiglu": 2, "geglu": 3}

EXPORTS = ["fb_weights_count", "fb_weights_entry", "fb_init_model", "fb_free", "fb_set_stream",
           "fb_encode_text", "fb_draft", "fb_refine", "fb_plan_from_phi", "fb_block_forward",
           "fb_last_error", "fb_set_timing", "fb_get_stats", "fb_get_stats_n", "fb_reset_stats",
           "fb_kernel_name",
           "fb_op_gemm", "fb_op_attention", "fb_draft_ex", "fb_refine_ex", "fb_select_elo",
           "fb_set_op_repeat", "fb_gemm_streamk_noalloc", "fb_state_bytes", "fb_state_offload",
           "fb_state_wait", "fb_set_sm_budget", "fb_sm_split_create", "fb_sm_split_info",
           "fb_sm_split_free", "fb_pipeline_step", "fb_set_device_wait_limit",
           "fb_test_fail_alloc", "fb_test_alloc_calls", "fb_test_poison_counters",
           "fb_test_request_handover", "fb_test_attention_split", "fb_test_plan_traffic",
           "fb_probe_mma_rate", "fb_probe_mma_gap", "fb_probe_mufu", "fb_probe_tmem_load",
           "fb_probe_mma_mix", "fb_op_sandwich_norm", "fb_op_route", "fb_op_expert_gemm",
           "fb_moe_forward", "fb_op_cross_attention", "fb_op_adapter_gemm", "fb_model_device"]

PAIR_VERIFIER = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                 ctypes.POINTER(ctypes.c_int))

_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Loads libflashbon.so (raises FileNotFoundError if it was not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} not built: run paper_2607_04461_gb300.build.build()")
    L = ctypes.CDLL(path)
    P, I, S, F, D = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_float, ctypes.c_double
    sig = {
        "fb_weights_count": (I, [ctypes.POINTER(fb_cfg), ctypes.POINTER(I), ctypes.POINTER(S)]),
        "fb_weights_entry": (I, [ctypes.POINTER(fb_cfg), I, ctypes.POINTER(ctypes.c_char_p),
                                 ctypes.POINTER(S), ctypes.POINTER(S)]),
        "fb_init_model": (I, [ctypes.POINTER(fb_cfg), P, ctypes.POINTER(P)]),
        "fb_free": (None, [P]),
        "fb_set_stream": (I, [P, P]),
        "fb_encode_text": (I, [P, P]),
        "fb_draft": (I, [P, P, I, P, P, I, P, P]),
        "fb_refine": (I, [P, P, P, P, I]),
        "fb_draft_ex": (I, [P, P, I, P, P, I, P, P, ctypes.POINTER(fb_sampler_opts)]),
        "fb_refine_ex": (I, [P, P, P, P, I, ctypes.POINTER(fb_sampler_opts)]),
        "fb_select_elo": (I, [P, I, D, D, D, D, PAIR_VERIFIER, P, ctypes.POINTER(I),
                              ctypes.POINTER(ctypes.c_double), ctypes.POINTER(I)]),
        "fb_plan_from_phi": (I, [I, I, I, I, I, I, I, I, P, P]),
        "fb_block_forward": (I, [P, I, P, I, F]),
        "fb_last_error": (ctypes.c_char_p, []),
        "fb_set_timing": (I, [P, I]),
        "fb_set_op_repeat": (I, [P, I]),
        "fb_get_stats": (I, [P, P]),
        "fb_get_stats_n": (I, [P, P, I]),
        "fb_reset_stats": (I, [P]),
        "fb_kernel_name": (ctypes.c_char_p, [I]),
        "fb_op_gemm": (I, [P, I, I, I, P, P, P, I, P, P, P, P, P, I]),
        "fb_op_attention": (I, [P, P, I, P, I, P, I, P, I, I, I, I, I, I, I, I]),
        "fb_gemm_streamk_noalloc": (I, [P, I, I, I, P, P, P, I, P, P, P, P, P]),
        "fb_state_bytes": (I, [P, ctypes.POINTER(S)]),
        "fb_state_offload": (I, [P, I, I, ctypes.POINTER(P)]),
        "fb_state_wait": (I, [P]),
        "fb_set_sm_budget": (I, [P, I]),
        "fb_model_device": (I, [P]),
        "fb_sm_split_create": (I, [I, ctypes.POINTER(P)]),
        "fb_sm_split_info": (I, [P, I, ctypes.POINTER(P), ctypes.POINTER(I)]),
        "fb_sm_split_free": (None, [P]),
        "fb_pipeline_step": (I, [P, P, I, P, P, I, P, P, ctypes.POINTER(fb_sampler_opts),
                                 P, P, P, I, ctypes.POINTER(fb_sampler_opts)]),
        "fb_set_device_wait_limit": (I, [ctypes.c_ulonglong]),
        "fb_test_fail_alloc": (I, [ctypes.c_long]),
        "fb_test_alloc_calls": (ctypes.c_long, []),
        "fb_test_poison_counters": (I, [P]),
        "fb_test_request_handover": (I, [P, I]),
        "fb_test_plan_traffic": (I, [ctypes.POINTER(fb_cfg), P, I, P, P, S, ctypes.POINTER(I),
                                     ctypes.POINTER(I), ctypes.POINTER(D)]),
        "fb_test_attention_split": (I, [P, I, I, I, I, I, ctypes.POINTER(I)]),
        "fb_op_sandwich_norm": (I, [P, ctypes.POINTER(fb_sandwich)]),
        "fb_op_route": (I, [P, ctypes.POINTER(fb_route)]),
        "fb_op_expert_gemm": (I, [P, ctypes.POINTER(fb_experts)]),
        "fb_moe_forward": (I, [P, ctypes.POINTER(fb_moe), P, P, ctypes.POINTER(fb_sandwich)]),
        "fb_op_cross_attention": (I, [P, ctypes.POINTER(fb_cross)]),
        "fb_op_adapter_gemm": (I, [P, ctypes.POINTER(fb_adapters)]),
        "fb_probe_mma_rate": (I, [I, I, I, ctypes.POINTER(ctypes.c_double)]),
        "fb_probe_mma_gap": (I, [I, ctypes.POINTER(ctypes.c_double)]),
        "fb_probe_mufu": (I, [I, ctypes.POINTER(ctypes.c_double)]),
        "fb_probe_tmem_load": (I, [I, ctypes.POINTER(ctypes.c_double)]),
        "fb_probe_mma_mix": (I, [I, I, I, ctypes.POINTER(ctypes.c_double)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    _lib = L
    return L


def _check(status):
    if status != FB_OK:
        raise FlashBonError(status, load_library().fb_last_error().decode())


def _ptr(x, dtype=None):
    """Raw pointer of a numpy array or torch tensor (must be contiguous)."""
    if x is None:
        return None
    if isinstance(x, np.ndarray):
        if dtype is not None and x.dtype != dtype:
            raise TypeError(f"expected {dtype}, got {x.dtype}")
        if not x.flags["C_CONTIGUOUS"]:
            raise ValueError("array must be C-contiguous")
        return x.ctypes.data
    if hasattr(x, "data_ptr"):
        if not x.is_contiguous():
            raise ValueError("tensor must be contiguous")
        return x.data_ptr()
    if isinstance(x, int):
        return x
    raise TypeError(f"unsupported buffer type {type(x)}")


def make_cfg(cfg: synth.Cfg) -> fb_cfg:
    c = fb_cfg()
    for f, _ in fb_cfg._fields_:
        setattr(c, f, getattr(cfg, f))
    return c


def pack_weights(cfg: synth.Cfg, weights: dict):
    """Packs named weights into the library's fp32 layout (fb_weights_entry order): a
    numpy buffer, or a CUDA tensor when the weights are CUDA tensors."""
    L = load_library()
    c = make_cfg(cfg)
    count, total = ctypes.c_int(), ctypes.c_size_t()
    _check(L.fb_weights_count(ctypes.byref(c), ctypes.byref(count), ctypes.byref(total)))
    first = next(iter(weights.values()))
    if getattr(first, "is_cuda", False):
        import torch
        buf = torch.empty(total.value, dtype=torch.float32, device=first.device)
        name, off, numel = ctypes.c_char_p(), ctypes.c_size_t(), ctypes.c_size_t()
        for i in range(count.value):
            _check(L.fb_weights_entry(ctypes.byref(c), i, ctypes.byref(name),
                                      ctypes.byref(off), ctypes.byref(numel)))
            w = weights[name.value.decode()].reshape(-1)
            if w.numel() != numel.value:
                raise ValueError(f"{name.value.decode()}: {w.numel()} elements, "
                                 f"expected {numel.value}")
            buf[off.value: off.value + numel.value].copy_(w)
        return buf
    buf = np.empty(total.value, np.float32)
    name, off, numel = ctypes.c_char_p(), ctypes.c_size_t(), ctypes.c_size_t()
    for i in range(count.value):
        _check(L.fb_weights_entry(ctypes.byref(c), i, ctypes.byref(name), ctypes.byref(off),
                                  ctypes.byref(numel)))
        w = np.asarray(weights[name.value.decode()], np.float32).ravel()
        if w.size != numel.value:
            raise ValueError(f"{name.value.decode()}: {w.size} elements, expected {numel.value}")
        buf[off.value: off.value + numel.value] = w
    return buf


# ---- functions with the C-ABI names -------------------------------------------------

def fb_init_model(cfg: synth.Cfg, weights) -> int:
    """weights: dict of named arrays, or an already packed fp32 buffer."""
    L = load_library()
    packed = weights if isinstance(weights, np.ndarray) or hasattr(weights, "data_ptr") \
        else pack_weights(cfg, weights)
    c = make_cfg(cfg)
    h = ctypes.c_void_p()
    _check(L.fb_init_model(ctypes.byref(c), _ptr(packed, np.float32), ctypes.byref(h)))
    return h.value


def fb_free(model: int) -> None:
    load_library().fb_free(model)


def fb_set_stream(model: int, stream) -> None:
    """stream: a torch.cuda.Stream, a raw cudaStream_t int, or None (model's own)."""
    s = getattr(stream, "cuda_stream", stream)
    _check(load_library().fb_set_stream(model, s))


def fb_model_device(model: int) -> int:
    """The device that the model lives on."""
    return load_library().fb_model_device(model)


def fb_set_sm_budget(model: int, n_sms: int) -> None:
    _check(load_library().fb_set_sm_budget(model, int(n_sms)))


class SmSplit:
    """Two disjoint SM partitions of the current device (green contexts), each with its
    own stream: part 0 holds n_sms SMs, part 1 the rest. streams[i] is a raw
    cudaStream_t handle (int) for Model.set_stream; sms[i] the part's SM count."""

    def __init__(self, n_sms: int):
        L = load_library()
        h = ctypes.c_void_p()
        _check(L.fb_sm_split_create(int(n_sms), ctypes.byref(h)))
        self.handle = h.value
        self.streams, self.sms = [], []
        for part in (0, 1):
            st, n = ctypes.c_void_p(), ctypes.c_int()
            _check(L.fb_sm_split_info(self.handle, part, ctypes.byref(st), ctypes.byref(n)))
            self.streams.append(st.value)
            self.sms.append(n.value)

    def close(self):
        if self.handle:
            load_library().fb_sm_split_free(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def fb_encode_text(model: int, text_ctx) -> None:
    _check(load_library().fb_encode_text(model, _ptr(text_ctx, np.float32)))


def fb_draft(model: int, latents, n: int, text_ctx, schedule, skip_mask=None,
             proxy_plan=None) -> None:
    sched = np.ascontiguousarray(schedule, np.float32)
    sk = None if skip_mask is None else np.ascontiguousarray(skip_mask, np.uint8)
    px = None if proxy_plan is None else np.ascontiguousarray(proxy_plan, np.int32)
    n_steps = len(sched) - 1
    for a in (sk, px):
        if a is not None and a.shape[0] != n_steps:
            raise ValueError("plan rows must equal len(schedule) - 1")
    _check(load_library().fb_draft(model, _ptr(latents, np.float32), n,
                                   _ptr(text_ctx, np.float32), _ptr(sched), n_steps,
                                   _ptr(sk), _ptr(px)))


def fb_refine(model: int, latent, text_ctx, full_schedule) -> None:
    sched = np.ascontiguousarray(full_schedule, np.float32)
    _check(load_library().fb_refine(model, _ptr(latent, np.float32), _ptr(text_ctx, np.float32),
                                    _ptr(sched), len(sched) - 1))


def make_opts(guidance=1.0, text_uncond=None, sde_a=0.0, noise=None, keep_state=False,
              state=None, warm_steps=0):
    """fb_sampler_opts; keeps references to the buffers it points to. state is a cached
    state buffer (fb_state_offload layout: numpy uint8 array or torch tensor)."""
    o = fb_sampler_opts(float(guidance), _ptr(text_uncond, np.float32), float(sde_a),
                        _ptr(noise, np.float32), int(bool(keep_state)), _ptr(state),
                        int(warm_steps))
    o._keep = (text_uncond, noise, state)
    return o


def fb_state_bytes(model) -> int:
    n = ctypes.c_size_t()
    _check(load_library().fb_state_bytes(model, ctypes.byref(n)))
    return n.value


def fb_state_offload(model, first: int, dsts) -> None:
    """Starts the copies of candidates first .. first + len(dsts) - 1's cached states into
    dsts (fb_state_bytes bytes each; pinned host memory lets them overlap later work);
    fb_state_wait waits for them."""
    arr = (ctypes.c_void_p * len(dsts))(*[_ptr(d) for d in dsts])
    _check(load_library().fb_state_offload(model, first, len(dsts), arr))


def fb_state_wait(model) -> None:
    _check(load_library().fb_state_wait(model))


def fb_draft_ex(model: int, latents, n: int, text_ctx, schedule, skip_mask=None,
                proxy_plan=None, opts=None) -> None:
    sched = np.ascontiguousarray(schedule, np.float32)
    sk = None if skip_mask is None else np.ascontiguousarray(skip_mask, np.uint8)
    px = None if proxy_plan is None else np.ascontiguousarray(proxy_plan, np.int32)
    _check(load_library().fb_draft_ex(model, _ptr(latents, np.float32), n,
                                      _ptr(text_ctx, np.float32), _ptr(sched), len(sched) - 1,
                                      _ptr(sk), _ptr(px),
                                      None if opts is None else ctypes.byref(opts)))


def fb_refine_ex(model: int, latent, text_ctx, full_schedule, opts=None) -> None:
    sched = np.ascontiguousarray(full_schedule, np.float32)
    _check(load_library().fb_refine_ex(model, _ptr(latent, np.float32),
                                       _ptr(text_ctx, np.float32), _ptr(sched), len(sched) - 1,
                                       None if opts is None else ctypes.byref(opts)))


def fb_pipeline_step(drafter: int, latents, n: int, text_ctx, draft_schedule, skip_mask,
                     proxy_plan, refiner=None, refine_latent=None, refine_schedule=None,
                     draft_opts=None, refine_opts=None) -> None:
    """Drafts `latents` with `drafter` while `refiner` refines `refine_latent` (the
    previous pool's selected candidate) on a worker thread of the library; returns when
    both are done. refine_latent None: the draft alone."""
    ds = np.ascontiguousarray(draft_schedule, np.float32)
    sk = None if skip_mask is None else np.ascontiguousarray(skip_mask, np.uint8)
    px = None if proxy_plan is None else np.ascontiguousarray(proxy_plan, np.int32)
    rsched = (np.zeros(1, np.float32) if refine_schedule is None
              else np.ascontiguousarray(refine_schedule, np.float32))
    _check(load_library().fb_pipeline_step(
        drafter, _ptr(latents, np.float32), n, _ptr(text_ctx, np.float32), _ptr(ds),
        len(ds) - 1, _ptr(sk), _ptr(px), None if draft_opts is None else ctypes.byref(draft_opts),
        refiner, _ptr(refine_latent, np.float32), _ptr(rsched), len(rsched) - 1,
        None if refine_opts is None else ctypes.byref(refine_opts)))


def fb_select_elo(scores, compare, rho1=0.5, rho2=0.5, kappa=1.5, k_base=32.0):
    """Stage 2 selection. compare(a, b) -> (a_preferred, confidence 0/1/2).
    Returns (winner, ratings [M], pairwise calls)."""
    sc = np.ascontiguousarray(scores, np.int32)
    M = sc.size

    def cb(user, a, b, conf_ptr):
        pref, conf = compare(a, b)
        conf_ptr[0] = int(conf)
        return 1 if pref else 0
    fn = PAIR_VERIFIER(cb)
    winner, calls = ctypes.c_int(), ctypes.c_int()
    ratings = np.zeros(M, np.float64)
    _check(load_library().fb_select_elo(_ptr(sc), M, rho1, rho2, kappa, k_base, fn, None,
                                        ctypes.byref(winner),
                                        ratings.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                        ctypes.byref(calls)))
    return winner.value, ratings, calls.value


def fb_plan_from_phi(S, S_prime, n_skip, l_start, l_end, f_full, order, depth):
    skip = np.zeros((S_prime, depth), np.uint8)
    proxy = np.zeros((S_prime, depth), np.int32)
    _check(load_library().fb_plan_from_phi(S, S_prime, n_skip, l_start, l_end, f_full, order,
                                           depth, _ptr(skip), _ptr(proxy)))
    return skip, proxy


def fb_block_forward(model: int, layer: int, h, n: int, t: float) -> None:
    _check(load_library().fb_block_forward(model, layer, _ptr(h), n, float(t)))


def fb_set_timing(model: int, mask: int) -> None:
    _check(load_library().fb_set_timing(model, int(mask)))


def fb_set_op_repeat(model: int, n: int) -> None:
    _check(load_library().fb_set_op_repeat(model, int(n)))


def fb_set_device_wait_limit(ns: int) -> None:
    """Device-side wait limit in nanoseconds (0 = the default 2 s); a testing hook."""
    _check(load_library().fb_set_device_wait_limit(int(ns)))


def fb_test_fail_alloc(k: int) -> None:
    """Makes the library's k-th device allocation from now fail (k < 0 disarms)."""
    _check(load_library().fb_test_fail_alloc(int(k)))


def fb_test_alloc_calls() -> int:
    """Device allocations the library made since the last fb_test_fail_alloc."""
    return int(load_library().fb_test_alloc_calls())


def fb_test_poison_counters(model) -> None:
    """Sets the stream-K counters of `model` (None: the allocation-free entry point's) to
    a large negative value, so the next stream-K finisher's wait cannot complete."""
    _check(load_library().fb_test_poison_counters(model))


def fb_test_plan_traffic(cfg, schedule, skip_mask, proxy_plan, elems):
    """(slots, sums, bytes per element) of the contribution cache under a plan."""
    sched = np.ascontiguousarray(schedule, np.float32)
    skip = np.ascontiguousarray(skip_mask, np.uint8)
    proxy = np.ascontiguousarray(proxy_plan, np.int32)
    slots, sums, nbytes = ctypes.c_int(), ctypes.c_int(), ctypes.c_double()
    c = make_cfg(cfg)
    _check(load_library().fb_test_plan_traffic(
        ctypes.byref(c), sched.ctypes.data, len(sched) - 1, skip.ctypes.data, proxy.ctypes.data,
        int(elems), ctypes.byref(slots), ctypes.byref(sums), ctypes.byref(nbytes)))
    return slots.value, sums.value, nbytes.value


def fb_test_attention_split(model, batch, Lq, Lkv, heads, impl=0) -> int:
    """CTAs among which fb_op_attention cuts its items by key range (0: none is cut)."""
    ctas = ctypes.c_int()
    _check(load_library().fb_test_attention_split(model, batch, Lq, Lkv, heads, impl,
                                                  ctypes.byref(ctas)))
    return ctas.value


def fb_test_request_handover(model, on: bool) -> None:
    """Makes the contributors of the next launch's cut stream-K tiles hand their shares over
    to the last one (on), or clears the counters (off)."""
    _check(load_library().fb_test_request_handover(model, int(on)))


def fb_probe_mma_rate(issuers: int, n: int, reps: int = 16384) -> float:
    """Tensor-pipe MACs per SM clock with `issuers` issuing warps and M=128 x n MMAs."""
    out = ctypes.c_double()
    _check(load_library().fb_probe_mma_rate(int(issuers), int(n), int(reps), ctypes.byref(out)))
    return out.value


def fb_probe_mma_gap(gap: int) -> float:
    """Tensor-pipe MACs per SM clock with a gap of `gap` clocks after every 8 MMAs."""
    out = ctypes.c_double()
    _check(load_library().fb_probe_mma_gap(int(gap), ctypes.byref(out)))
    return out.value


def fb_probe_mufu(op: int) -> float:
    """Results per SM clock of ex2 (0), tanh (1), rcp (2) or ex2 on f16 pairs (3)."""
    out = ctypes.c_double()
    _check(load_library().fb_probe_mufu(int(op), ctypes.byref(out)))
    return out.value


def fb_probe_tmem_load(busy: bool) -> float:
    """SM clocks of a 128-column TMEM load and its wait (tensor pipe idle or running)."""
    out = ctypes.c_double()
    _check(load_library().fb_probe_tmem_load(1 if busy else 0, ctypes.byref(out)))
    return out.value


def fb_probe_mma_mix(form: int, loaders: int = 0, loader_gap: int = 0) -> float:
    """Tensor-pipe MACs per SM clock of attention-step-shaped MMA batches (form 0: both
    operands K-major in shared memory, 1: B MN-major, 2: B MN-major and A from TMEM, 3: a
    whole attention step, 4: the same with its commits, 5 and 6: forms 3 and 4 with hoisted
    descriptor words; 7-13: forms 0-6 with softmax arithmetic in the loaders) with `loaders`
    warps reading and writing TMEM meanwhile."""
    out = ctypes.c_double()
    _check(load_library().fb_probe_mma_mix(int(form), int(loaders), int(loader_gap),
                                           ctypes.byref(out)))
    return out.value


def fb_get_stats(model: int) -> dict:
    arr = (fb_kstat * len(KERNEL_KINDS))()
    _check(load_library().fb_get_stats_n(model, ctypes.cast(arr, ctypes.c_void_p), len(arr)))
    return {KERNEL_KINDS[i]: dict(launches=int(arr[i].launches), ms=arr[i].ms,
                                  flops=arr[i].flops, bytes=arr[i].bytes)
            for i in range(len(KERNEL_KINDS))}


def fb_reset_stats(model: int) -> None:
    _check(load_library().fb_reset_stats(model))


def fb_op_gemm(model, M, N, K, A, W, bias, epi, out, resid=None, gate=None, base=None,
               delta=None, impl=0) -> None:
    _check(load_library().fb_op_gemm(model, M, N, K, _ptr(A), _ptr(W), _ptr(bias), epi,
                                     _ptr(out), _ptr(resid), _ptr(gate), _ptr(base),
                                     _ptr(delta), impl))


def fb_gemm_streamk_noalloc(stream, M, N, K, A, W, bias, epi, out, resid=None, gate=None,
                            base=None, delta=None) -> None:
    """The allocation-free stream-K GEMM (no model); `stream` is a cudaStream_t handle
    (int) or None for the legacy default stream. Waits for the result."""
    _check(load_library().fb_gemm_streamk_noalloc(stream, M, N, K, _ptr(A), _ptr(W),
                                                  _ptr(bias), epi, _ptr(out), _ptr(resid),
                                                  _ptr(gate), _ptr(base), _ptr(delta)))


def fb_op_attention(model, Q, ldq, Kt, ldk, V, ldv, O, ldo, batch, Lq, Lkv, kv_batch_rows,
                    heads, head_dim, impl=0) -> None:
    _check(load_library().fb_op_attention(model, _ptr(Q), ldq, _ptr(Kt), ldk, _ptr(V), ldv,
                                          _ptr(O), ldo, batch, Lq, Lkv, kv_batch_rows, heads,
                                          head_dim, impl))


# ---- mixture-of-experts feed-forward between two norms ----------------------------------
# make_* build the argument structures from CUDA tensors; they keep references to the tensors
# and can be used for any number of calls.

def _tensor(name, x, dtypes, shape, rows=False):
    """The pointer of CUDA tensor x (None: null) after a check of its type and shape (None in
    shape: any size); contiguous, or with `rows` only along each row."""
    if x is None:
        return None
    if not getattr(x, "is_cuda", False):
        raise TypeError(f"{name}: expected a CUDA tensor")
    if str(x.dtype).removeprefix("torch.") not in dtypes:
        raise TypeError(f"{name}: expected {' or '.join(dtypes)}, got {x.dtype}")
    if x.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, x.shape)):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(x.shape)}")
    if rows:
        if x.shape[1] > 1 and x.stride(1) != 1:
            raise ValueError(f"{name}: rows must be contiguous")
    elif not x.is_contiguous():
        raise ValueError(f"{name}: tensor must be contiguous")
    return x.data_ptr()


_FLOATS = ("bfloat16", "float32")


def _row_stride(x):
    """Elements from a row to the next; one row alone has no stride of its own (torch's may be
    anything), and its width will do."""
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


def _type(x):
    return FB_F32 if x.dtype.itemsize == 4 else FB_BF16


def make_sandwich(h, y=None, slot=None, weight=None, post="none", post_eps=1e-6, post_w=None,
                  post_b=None, gate=None, resid_scale=1.0, h_out=None, pre="none", pre_eps=1e-6,
                  mul_base=1.0, mul=None, add=None, a=None, group_rows=0):
    """fb_sandwich for fb_op_sandwich_norm. h [rows][dim] bf16 or fp32; y [rows][dim], or with
    slot and weight ([rows][parts] int32 and fp32) the rows that slot points to; norms "none",
    "rms" or "layer"; gate, mul and add [groups][dim] fp32, row r // group_rows of them for row
    r (one row and group_rows 0: the same for all); h_out (may be h) and a [rows][dim]."""
    rows, dim = h.shape
    s = fb_sandwich(rows=rows, dim=dim, resid_scale=resid_scale, post=NORMS[post],
                    post_eps=post_eps, pre=NORMS[pre], pre_eps=pre_eps, mul_base=mul_base,
                    group_rows=group_rows)
    s.h, s.h_type, s.ldh = _tensor("h", h, _FLOATS, (rows, dim), True), _type(h), _row_stride(h)
    if y is not None:
        s.y, s.y_type = _tensor("y", y, _FLOATS, (None, dim), True), _type(y)
        s.y_rows, s.ldy = y.shape[0], _row_stride(y)
    if slot is not None:
        if y is None or weight is None:
            raise ValueError("slot needs y and weight")
        s.parts = slot.shape[1]
        if s.parts < 1:
            raise ValueError("slot: at least one part")
        s.slot = _tensor("slot", slot, ("int32",), (rows, s.parts))
        s.weight = _tensor("weight", weight, ("float32",), (rows, s.parts))
    s.post_w = _tensor("post_w", post_w, ("float32",), (dim,))
    s.post_b = _tensor("post_b", post_b, ("float32",), (dim,))
    groups = -(-rows // group_rows) if group_rows > 0 else 1
    strides = set()
    for name, x in (("gate", gate), ("mul", mul), ("add", add)):
        if x is None:
            continue
        setattr(s, name, _tensor(name, x, ("float32",), (None, dim), True))
        if x.shape[0] < groups:
            raise ValueError(f"{name}: {x.shape[0]} rows for {groups} groups")
        strides.add(_row_stride(x))
    if len(strides) > 1 and groups > 1:
        raise ValueError("gate, mul and add must have the same row stride")
    s.ldm = max(strides, default=dim)
    if h_out is not None:
        s.h_out = _tensor("h_out", h_out, (str(h.dtype).removeprefix("torch."),), (rows, dim), True)
        s.ldho = _row_stride(h_out)
    if a is not None:
        s.a, s.a_type = _tensor("a", a, _FLOATS, (rows, dim), True), _type(a)
        s.lda = _row_stride(a)
    s._keep = (h, y, slot, weight, post_w, post_b, gate, mul, add, h_out, a)
    return s


def make_route(logits, expert, weight, slot, token, offsets, valid=None, renorm=False):
    """fb_route for fb_op_route. logits [tokens][experts] bf16 or fp32; expert, slot int32 and
    weight fp32 [tokens][top_k], token int32 [tokens * top_k], offsets int32 [experts + 1];
    valid [tokens] uint8 or None."""
    tokens, experts = logits.shape
    k = expert.shape[1]
    r = fb_route(tokens=tokens, experts=experts, top_k=k, renorm=int(bool(renorm)))
    r.logits = _tensor("logits", logits, _FLOATS, (tokens, experts), True)
    r.logits_type, r.ldl = _type(logits), _row_stride(logits)
    r.valid = _tensor("valid", valid, ("uint8",), (tokens,))
    r.expert = _tensor("expert", expert, ("int32",), (tokens, k))
    r.weight = _tensor("weight", weight, ("float32",), (tokens, k))
    r.slot = _tensor("slot", slot, ("int32",), (tokens, k))
    r.token = _tensor("token", token, ("int32",), (tokens * k,))
    r.offsets = _tensor("offsets", offsets, ("int32",), (experts + 1,))
    r._keep = (logits, valid, expert, weight, slot, token, offsets)
    return r


def make_experts(a, w, offsets, out, index=None, bias=None, act="none"):
    """fb_experts for fb_op_expert_gemm. a [a_rows][k] bf16; w [experts][n or 2 n][k] bf16;
    offsets [experts + 1] and index [max_rows] int32; bias [experts][n or 2 n] fp32; out
    [max_rows][n] bf16 or fp32; act "none", "gelu", "swiglu" or "geglu" (the last two: the n
    gate rows of w and bias before the n up rows)."""
    experts, nw, k = w.shape
    gated = ACTS[act] >= ACTS["swiglu"]
    if gated and nw % 2:
        raise ValueError("w: gate rows and up rows differ in number")
    n = nw // 2 if gated else nw
    g = fb_experts(experts=experts, n=n, k=k, max_rows=out.shape[0], a_rows=a.shape[0],
                   act=ACTS[act])
    g.a, g.lda = _tensor("a", a, ("bfloat16",), (None, k), True), _row_stride(a)
    g.w = _tensor("w", w, ("bfloat16",), (experts, nw, k))
    g.offsets = _tensor("offsets", offsets, ("int32",), (experts + 1,))
    g.index = _tensor("index", index, ("int32",), (out.shape[0],))
    g.bias = _tensor("bias", bias, ("float32",), (experts, nw))
    g.out, g.out_type = _tensor("out", out, _FLOATS, (None, n), True), _type(out)
    g.ldo = _row_stride(out)
    g._keep = (a, w, offsets, out, index, bias)
    return g


def make_moe(router_w, w1, w2, top_k, b1=None, b2=None, act="gelu", renorm=False):
    """fb_moe for fb_moe_forward. router_w [router_rows][dim] bf16 (padded rows behind the
    experts are ignored); w1 [experts][hidden or 2 hidden][dim], w2 [experts][dim][hidden] bf16;
    biases fp32."""
    experts, dim, hidden = w2.shape
    nw = 2 * hidden if ACTS[act] >= ACTS["swiglu"] else hidden
    p = fb_moe(dim=dim, hidden=hidden, experts=experts, top_k=top_k, renorm=int(bool(renorm)),
               act=ACTS[act], router_rows=router_w.shape[0])
    p.router_w = _tensor("router_w", router_w, ("bfloat16",), (None, dim))
    p.w1 = _tensor("w1", w1, ("bfloat16",), (experts, nw, dim))
    p.w2 = _tensor("w2", w2, ("bfloat16",), (experts, dim, hidden))
    p.b1 = _tensor("b1", b1, ("float32",), (experts, nw))
    p.b2 = _tensor("b2", b2, ("float32",), (experts, dim))
    p._keep = (router_w, w1, w2, b1, b2)
    return p


def fb_op_sandwich_norm(model: int, args: fb_sandwich) -> None:
    _check(load_library().fb_op_sandwich_norm(model, ctypes.byref(args)))


def fb_op_route(model: int, args: fb_route) -> None:
    _check(load_library().fb_op_route(model, ctypes.byref(args)))


def fb_op_expert_gemm(model: int, args: fb_experts) -> None:
    _check(load_library().fb_op_expert_gemm(model, ctypes.byref(args)))


def fb_moe_forward(model: int, moe: fb_moe, a, sandwich: fb_sandwich, valid=None) -> None:
    """a: the normed input, bf16 [rows][dim]; valid: uint8 [rows] or None."""
    _check(load_library().fb_moe_forward(
        model, ctypes.byref(moe), _tensor("a", a, ("bfloat16",), (sandwich.rows, moe.dim)),
        _tensor("valid", valid, ("uint8",), (sandwich.rows,)), ctypes.byref(sandwich)))


# ---- several requests in one batch --------------------------------------------------------

def _one_device(**tensors):
    """The one device that all tensors lie on (the library reads them on the model's, see
    _on_model)."""
    found = {name: x.device.index for name, x in tensors.items() if x is not None}
    if len(set(found.values())) > 1:
        raise ValueError(f"tensors on several devices: {found}")
    return next(iter(found.values()))


def _on_model(model, args):
    """Refuses tensors of another device than the model's, whose addresses mean nothing there.
    (Structures filled in by hand say nothing about their device, and no model is the library's to
    refuse.)"""
    device = getattr(args, "_device", None)
    if model and device is not None and device != load_library().fb_model_device(model):
        raise ValueError(f"tensors on device {device}, the model on device "
                         f"{load_library().fb_model_device(model)}")


def make_cross(q, k, v, out, q_offsets, kv_offsets, head_dim=128, kv_of=None, valid=None, scale=0.0):
    """fb_cross for fb_op_cross_attention. q and out [q_rows][heads * head_dim], k and v
    [kv_rows][kv_heads * head_dim] bf16 (k and v may be columns of one buffer); q_offsets [seqs + 1],
    kv_offsets [states + 1] and kv_of [seqs] (None: sequence s attends to states s) int32; valid
    [kv_rows] uint8, 0 where a key is padding, or None; scale 0: 1 / sqrt(head_dim)."""
    if q.dim() != 2 or k.dim() != 2 or q.shape[1] % head_dim or k.shape[1] % head_dim:
        raise ValueError(f"q and k: rows of whole heads of {head_dim}")
    wq, wk = q.shape[1], k.shape[1]
    c = fb_cross(seqs=q_offsets.shape[0] - 1, states=kv_offsets.shape[0] - 1, heads=wq // head_dim,
                 kv_heads=wk // head_dim, head_dim=head_dim, q_rows=q.shape[0], kv_rows=k.shape[0],
                 scale=scale)
    bf16 = ("bfloat16",)
    c.q, c.ldq = _tensor("q", q, bf16, (None, wq), True), _row_stride(q)
    c.k, c.ldk = _tensor("k", k, bf16, (None, wk), True), _row_stride(k)
    c.v, c.ldv = _tensor("v", v, bf16, (k.shape[0], wk), True), _row_stride(v)
    c.out, c.ldo = _tensor("out", out, bf16, (q.shape[0], wq), True), _row_stride(out)
    c.q_offsets = _tensor("q_offsets", q_offsets, ("int32",), (None,))
    c.kv_offsets = _tensor("kv_offsets", kv_offsets, ("int32",), (None,))
    c.kv_of = _tensor("kv_of", kv_of, ("int32",), (c.seqs,))
    c.valid = _tensor("valid", valid, ("uint8",), (k.shape[0],))
    c._device = _one_device(q=q, k=k, v=v, out=out, q_offsets=q_offsets, kv_offsets=kv_offsets,
                            kv_of=kv_of, valid=valid)
    c._keep = (q, k, v, out, q_offsets, kv_offsets, kv_of, valid)
    return c


def make_adapters(x, w, a, b, offsets, adapter, out, scale=None, bias=None, act="none", resid=None,
                  gate=None):
    """fb_adapters for fb_op_adapter_gemm. x [rows][k], w [n][k], a [adapters][rank][k], b
    [adapters][n][rank] bf16; offsets [segments + 1] and adapter [segments] (-1: none) int32; scale
    [adapters], bias and gate [n], resid [rows][n] fp32 or None; out [rows][n] bf16 or fp32 (may be
    resid); act "none" or "gelu"."""
    rows, (n, k), (adapters, rank) = x.shape[0], w.shape, a.shape[:2]
    g = fb_adapters(rows=rows, n=n, k=k, rank=rank, adapters=adapters, segments=offsets.shape[0] - 1,
                    act=ACTS[act])
    bf16, f32 = ("bfloat16",), ("float32",)
    g.x, g.ldx = _tensor("x", x, bf16, (None, k), True), _row_stride(x)
    g.w = _tensor("w", w, bf16, (n, k))
    g.a = _tensor("a", a, bf16, (adapters, rank, k))
    g.b = _tensor("b", b, bf16, (adapters, n, rank))
    g.scale = _tensor("scale", scale, f32, (adapters,))
    g.bias = _tensor("bias", bias, f32, (n,))
    g.gate = _tensor("gate", gate, f32, (n,))
    g.offsets = _tensor("offsets", offsets, ("int32",), (None,))
    g.adapter = _tensor("adapter", adapter, ("int32",), (g.segments,))
    if resid is not None:
        g.resid, g.ldr = _tensor("resid", resid, f32, (rows, n), True), _row_stride(resid)
    g.out, g.out_type = _tensor("out", out, _FLOATS, (rows, n), True), _type(out)
    g.ldo = _row_stride(out)
    g._device = _one_device(x=x, w=w, a=a, b=b, scale=scale, bias=bias, gate=gate, offsets=offsets,
                            adapter=adapter, resid=resid, out=out)
    g._keep = (x, w, a, b, offsets, adapter, out, scale, bias, resid, gate)
    return g


def fb_op_cross_attention(model: int, args: fb_cross) -> None:
    _on_model(model, args)
    _check(load_library().fb_op_cross_attention(model, ctypes.byref(args)))


def fb_op_adapter_gemm(model: int, args: fb_adapters) -> None:
    _on_model(model, args)
    _check(load_library().fb_op_adapter_gemm(model, ctypes.byref(args)))


class Model:
    """Owns an fb_model handle; methods forward to the fb_* functions."""

    def __init__(self, cfg: synth.Cfg, weights):
        self.cfg = cfg
        self.handle = fb_init_model(cfg, weights)

    def close(self):
        if self.handle:
            fb_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def set_stream(self, stream):
        fb_set_stream(self.handle, stream)

    def set_sm_budget(self, n_sms):
        fb_set_sm_budget(self.handle, n_sms)

    def encode_text(self, ctx):
        fb_encode_text(self.handle, ctx)

    def draft(self, latents, text_ctx, schedule, skip_mask=None, proxy_plan=None, n=None,
              opts=None):
        n = latents.shape[0] if n is None else n
        if opts is None:
            fb_draft(self.handle, latents, n, text_ctx, schedule, skip_mask, proxy_plan)
        else:
            fb_draft_ex(self.handle, latents, n, text_ctx, schedule, skip_mask, proxy_plan, opts)

    def refine(self, latent, text_ctx, schedule, opts=None):
        if opts is None:
            fb_refine(self.handle, latent, text_ctx, schedule)
        else:
            fb_refine_ex(self.handle, latent, text_ctx, schedule, opts)

    def state_bytes(self) -> int:
        return fb_state_bytes(self.handle)

    def state_offload(self, first, dsts):
        fb_state_offload(self.handle, first, dsts)

    def state_wait(self):
        fb_state_wait(self.handle)

    def block_forward(self, layer, h, n, t):
        fb_block_forward(self.handle, layer, h, n, t)

    def op_sandwich_norm(self, args):
        fb_op_sandwich_norm(self.handle, args)

    def op_route(self, args):
        fb_op_route(self.handle, args)

    def op_expert_gemm(self, args):
        fb_op_expert_gemm(self.handle, args)

    def moe_forward(self, moe, a, sandwich, valid=None):
        fb_moe_forward(self.handle, moe, a, sandwich, valid)

    def op_cross_attention(self, args):
        fb_op_cross_attention(self.handle, args)

    def op_adapter_gemm(self, args):
        fb_op_adapter_gemm(self.handle, args)

    def set_timing(self, mask):
        fb_set_timing(self.handle, mask)

    def stats(self):
        return fb_get_stats(self.handle)

    def reset_stats(self):
        fb_reset_stats(self.handle)
