"""Thin binding of libdrf's C ABI (see include/drf.h): ctypes, and a CPython module for the skip calls' arguments.

Argument marshalling only: torch supplies device buffers and the current HIP stream;
every step of the path runs in the library's kernels.  There is no CPU fallback: a
missing library raises at load.  The module is built for one interpreter; another one, or a build
without Python's headers, marshals the skip calls with ctypes too."""
import ctypes as C
import math
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdrf.so")

CONSERVATIVE, AGGRESSIVE = 0, 1
F32, BF16 = 0, 1
COND_VECTOR, COND_CLASS, COND_TEXT = 0, 1, 2
PLAN_ROW = 5
PROF_GEMM, PROF_ATTN, PROF_ELEMWISE, PROF_UPDATE, PROF_PASS_FULL, PROF_PASS_OTHER = 0, 1, 2, 3, 4, 5
DDIM, DDPM, EULER = 0, 1, 2
ROPE_PAIRS, ROPE_HALVES = 0, 1
QK_NONE, QK_RMS, QK_LAYER = 0, 1, 2
_QK = {"none": QK_NONE, "rms": QK_RMS, "layer": QK_LAYER}
_LAYOUTS = {"pairs": ROPE_PAIRS, "halves": ROPE_HALVES}

# include/drf.h: the method's calls
SYMBOLS = ["drf_denoiser_weight_count", "drf_denoiser_create", "drf_denoiser_destroy", "drf_denoiser_reserve", "drf_denoiser_use_graphs",
           "drf_eps_batched", "drf_eps_batched_static", "drf_skip_transition", "drf_refine_step", "drf_sample",
           "drf_skip_transition_noise", "drf_normal_fill", "drf_sample_noise", "drf_noise_count",
           "drf_plan_build", "drf_last_error",
           "drf_rope", "drf_qk_norm_rope", "drf_block_words", "drf_block_select_scratch_bytes", "drf_block_select", "drf_block_attention", "drf_block_attention_scratch_bytes", "drf_block_attention_split",
           "drf_denoiser_weight_count_attn", "drf_denoiser_create_attn"]
# include/drf_measure.h: test and measurement hooks
MEASURE_SYMBOLS = ["drf_eps_trace", "drf_profile_enable", "drf_profile_read", "drf_probe_gemm_bf16",
                   "drf_probe_attn_bf16", "drf_probe_cross_attn_bf16", "drf_probe_attn_route", "drf_probe_gemm_route", "drf_probe_block_route", "drf_probe_update_fused", "drf_graph_stats", "drf_calibrate_mfma_bf16", "drf_calibrate_copy"]
STATIC_SCRATCH_BYTES = 48 << 20


class DitConfig(C.Structure):
    _fields_ = [(k, C.c_int) for k in ("depth", "hidden", "heads", "mlp_ratio", "patch", "in_ch", "lat_h",
                                         "lat_w", "dtype", "cond", "cond_dim", "ctx_len")]


class SchedConfig(C.Structure):
    _fields_ = [("train_steps", C.c_int), ("beta_start", C.c_double), ("beta_end", C.c_double),
                ("steps", C.c_int), ("eta", C.c_double), ("sampler", C.c_int), ("shift", C.c_double)]


class Noise(C.Structure):
    _fields_ = [("z", C.c_void_p), ("seed", C.c_uint64), ("field0", C.c_uint32)]


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("slot_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class AttnShape(C.Structure):
    _fields_ = [(k, C.c_int) for k in ("dtype", "slots", "q_tokens", "kv_tokens", "q_heads", "kv_heads", "head_dim")] + [
        ("q_lens", C.c_void_p), ("kv_lens", C.c_void_p)]


class RopeConfig(C.Structure):
    _fields_ = [("n_axes", C.c_int), ("dim", C.c_int * 3), ("extent", C.c_int * 3), ("origin", C.c_double * 3), ("step", C.c_double * 3),
                ("theta", C.c_double), ("layout", C.c_int)]


class QkConfig(C.Structure):
    _fields_ = [("norm", C.c_int), ("eps", C.c_double), ("q_scale", C.c_float)] + [(k, C.c_void_p) for k in ("q_gain", "q_bias", "k_gain", "k_bias")]


class AttnConfig(C.Structure):
    _fields_ = [("qk_norm", C.c_int), ("norm_eps", C.c_double), ("rope_dim", C.c_int * 2), ("rope_theta", C.c_double), ("rope_layout", C.c_int),
                ("additive_pos", C.c_int), ("q_block", C.c_int), ("kv_block", C.c_int), ("topk", C.c_int)]


class DrfError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("libdrf status %d: %s" % (status, msg))
        self.status = status


_lib = None
_skip = None            # _native.skip or _skip_ctypes, once the library is loaded


def lib():
    """Load libdrf.so (built by paper_2603_25872_amd/build.py); raises if absent."""
    global _lib, _skip
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libdrf.so is not built: run `python -m paper_2603_25872_amd.build`")
        L = C.CDLL(LIB_PATH)
        L.drf_denoiser_weight_count.restype = C.c_size_t
        L.drf_denoiser_weight_count.argtypes = [C.c_void_p]
        L.drf_denoiser_create.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.drf_denoiser_destroy.argtypes = [C.c_void_p]
        L.drf_denoiser_destroy.restype = None
        L.drf_denoiser_reserve.argtypes = [C.c_void_p, C.c_int]
        L.drf_denoiser_use_graphs.argtypes = [C.c_void_p, C.c_int]
        L.drf_eps_batched.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
        L.drf_eps_batched_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
        L.drf_probe_update_fused.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_float, C.c_size_t, C.c_void_p,
                                             C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.drf_graph_stats.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.drf_calibrate_mfma_bf16.argtypes = [C.c_int, C.c_int, C.c_void_p, C.c_void_p]
        L.drf_calibrate_copy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int, C.c_void_p, C.c_void_p]
        L.drf_eps_trace.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p,
                                    C.c_void_p]
        L.drf_skip_transition.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int,
                                          C.c_size_t, C.c_void_p, C.c_void_p]
        L.drf_refine_step.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_size_t, C.c_void_p,
                                      C.c_void_p]
        L.drf_sample.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                 C.c_void_p, C.c_float, C.c_void_p, C.c_void_p]
        L.drf_plan_build.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        L.drf_skip_transition_noise.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int,
                                                C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p]
        L.drf_normal_fill.argtypes = [C.c_uint64, C.c_uint32, C.c_size_t, C.c_size_t, C.c_void_p, C.c_void_p]
        L.drf_sample_noise.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
        L.drf_noise_count.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_void_p]
        L.drf_profile_enable.argtypes = [C.c_void_p, C.c_int]
        L.drf_profile_read.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        L.drf_probe_gemm_bf16.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                          C.c_int, C.c_void_p]
        L.drf_probe_attn_bf16.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p]
        L.drf_probe_cross_attn_bf16.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p] + [C.c_int] * 7 + [C.c_void_p]
        L.drf_probe_attn_route.argtypes = [C.c_int] * 6
        L.drf_probe_block_route.argtypes = [C.c_int] * 5
        L.drf_probe_gemm_route.argtypes = [C.c_int] * 5 + [C.c_void_p]
        L.drf_last_error.restype = C.c_char_p
        L.drf_denoiser_weight_count_attn.restype = C.c_size_t
        L.drf_denoiser_weight_count_attn.argtypes = [C.c_void_p, C.c_void_p]
        L.drf_denoiser_create_attn.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.drf_rope.argtypes = [C.c_void_p] + [C.c_int] * 5 + [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p]
        L.drf_qk_norm_rope.argtypes = [C.c_void_p] * 4 + [C.c_size_t] + [C.c_void_p] * 5
        L.drf_block_words.restype = L.drf_block_select_scratch_bytes.restype = C.c_size_t
        L.drf_block_words.argtypes = [C.c_int, C.c_int]
        L.drf_block_select_scratch_bytes.argtypes = [C.c_void_p, C.c_int, C.c_int]
        L.drf_block_select.argtypes = [C.c_void_p] + [C.c_int] * 3 + [C.c_void_p] * 3 + [C.c_size_t, C.c_void_p, C.c_void_p]
        L.drf_block_attention.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_float] + [C.c_void_p] * 6
        L.drf_block_attention_scratch_bytes.argtypes = [C.c_void_p]
        L.drf_block_attention_scratch_bytes.restype = C.c_size_t
        L.drf_block_attention_split.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_float] + [C.c_void_p] * 6 + [C.c_size_t, C.c_void_p]
        try:
            from . import _native               # built beside the library
            _native.bind(C.cast(L.drf_skip_transition_noise, C.c_void_p).value)
            _skip = _native.skip
        except ImportError:
            _skip = _skip_ctypes
        _lib = L
    return _lib


def _check(status):
    if status != 0:
        raise DrfError(status, lib().drf_last_error().decode())


def dit_config(d):
    return DitConfig(d["depth"], d["hidden"], d["heads"], d["mlp_ratio"], d["patch"], d["in_ch"], d["lat_h"],
                     d["lat_w"], d["dtype"], d["cond"], d["cond_dim"], d["ctx_len"])


def attn_config(dit):
    """drf_attn_config of a model whose dict has an "attn" entry (see I.param_shapes), else None."""
    a = dit.get("attn")
    if a is None:
        return None
    rope, blocks = a.get("rope_dim", (0, 0)), a.get("blocks", (0, 0, 0))
    return AttnConfig(_QK[a.get("qk_norm", "none")], float(a.get("norm_eps", 1e-6)), (C.c_int * 2)(*rope), float(a.get("rope_theta", 10000.0)),
                      _LAYOUTS[a.get("rope_layout", "pairs")], int(a.get("additive_pos", True)), *blocks)


def sched_config(d):
    return SchedConfig(d["train_steps"], d["beta_start"], d["beta_end"], d["steps"], float(d.get("eta", 0.0)),
                       int(d.get("sampler", DDIM)), float(d.get("shift", 1.0)))


def _noise(z=None, seed=None, field0=0):
    """drf_noise from explicit device fields z, or (seed, field0) of the library's stream; None when neither is given."""
    import torch
    if z is not None:
        return Noise(_dev(z, torch.float32), 0, 0)
    if seed is not None:
        return Noise(None, int(seed), int(field0))
    return None


def _stream():
    """Handle of the current stream (torch.cuda.current_stream() makes a Stream object of it: 3.0 us a call against 0.2)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _dev(t, dtype=None):
    """Device pointer of a contiguous CUDA tensor."""
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "need a contiguous device tensor"
    if dtype is not None:
        assert t.dtype == dtype, "expected %s, got %s" % (dtype, t.dtype)
    return t.data_ptr()


def denoiser_weight_count(dit):
    cfg, attn = dit_config(dit), attn_config(dit)
    return int(lib().drf_denoiser_weight_count_attn(C.byref(cfg), None if attn is None else C.byref(attn)))


def plan_build(sched, mode, n):
    """The bookkeeping table of drf_sample as an int32 array [rows, 5] (host only)."""
    sc = sched_config(sched)
    cnt = C.c_size_t(0)
    _check(lib().drf_plan_build(C.byref(sc), mode, n, None, 0, C.byref(cnt)))
    rows = np.zeros((cnt.value, PLAN_ROW), np.int32)
    _check(lib().drf_plan_build(C.byref(sc), mode, n, rows.ctypes.data_as(C.c_void_p), cnt.value, C.byref(cnt)))
    return rows


def _targets(s_to):
    """s_to as a tuple of the call's own: what sizes the output is what is launched, whatever becomes of the caller's list meanwhile."""
    m, to = len(s_to), tuple(s_to)
    if len(to) != m:
        raise IndexError("invalid index")
    return to


def _skip_ctypes(sched, x_from, net_from, s_from, s_to, noise, out, dtype, stream):
    """_native.skip where that module is not there (8.1 us a call against 6.3): status of drf_skip_transition_noise on these arguments."""
    sc = sched_config(sched)
    m = len(s_to)
    to = (C.c_int * max(m, 1))(*_targets(s_to))
    batch = x_from.shape[0] if len(x_from.shape) else 1
    elems = math.prod(x_from.shape[1:]) if batch else 0
    return _lib.drf_skip_transition_noise(C.byref(sc), _dev(x_from, dtype), _dev(net_from, dtype), s_from, to, m, batch, elems, noise,
                                          _dev(out, dtype), stream() if callable(stream) else stream)


def skip_transition(sched, x_from, eps_from, s_from, s_to, out=None):
    """x_from, eps_from: fp32 device tensors [batch, ...]; s_to: list of target indices.
    Returns [len(s_to), batch, ...]."""
    import torch
    s_to = _targets(s_to)
    if out is None:
        out = torch.empty((len(s_to),) + tuple(x_from.shape), dtype=torch.float32, device=x_from.device)
    if _lib is None:
        lib()
    _check(_skip(sched, x_from, eps_from, s_from, s_to, None, out, torch.float32, _stream))
    return out


def skip_transition_noise(sched, x_from, net_from, s_from, s_to, z=None, seed=None, field0=0, out=None):
    """Skip transitions of the configured sampler with their fresh noise: explicit fields z [len(s_to), batch, ...]
    or the library's stream (seed, field0)."""
    import torch
    s_to = _targets(s_to)
    if out is None:
        out = torch.empty((len(s_to),) + tuple(x_from.shape), dtype=torch.float32, device=x_from.device)
    if _lib is None:
        lib()
    nz = _noise(z, seed, field0)
    _check(_skip(sched, x_from, net_from, s_from, s_to, None if nz is None else C.addressof(nz), out, torch.float32, _stream))
    return out


def normal_fill(seed, field0, n_fields, field_elems, out=None):
    """Fields field0 .. field0 + n_fields - 1 of the library's normal stream as a device tensor [n_fields, field_elems]."""
    import torch
    if out is None:
        out = torch.empty((n_fields, field_elems), dtype=torch.float32, device="cuda")
    _check(lib().drf_normal_fill(int(seed), int(field0), n_fields, field_elems, _dev(out, torch.float32), _stream()))
    return out


def noise_count(sched, mode, n):
    """Number of fresh-noise fields one drf_sample_noise call draws (host only)."""
    sc = sched_config(sched)
    cnt = C.c_size_t(0)
    _check(lib().drf_noise_count(C.byref(sc), mode, n, C.byref(cnt)))
    return int(cnt.value)


def refine_step(sched, x, eps, s_from, out=None):
    import torch
    sc = sched_config(sched)
    batch = x.shape[0]
    if out is None:
        out = torch.empty_like(x)
    _check(lib().drf_refine_step(C.byref(sc), _dev(x, torch.float32), _dev(eps, torch.float32), s_from, batch,
                                 x.numel() // batch if batch else 0, _dev(out, torch.float32), _stream()))
    return out


# ---- attention operators: what _native does, where that module is not there ----
# (Like every call of this module they work on the tensors' memory and are unknown to autograd: results require no gradient.)

def _heads(t, like=None, same=False):
    """(drf_heads, dtype, shape) of a device tensor [slots, tokens, heads, head_dim] whose head columns are contiguous."""
    import torch
    assert t.is_cuda and t.dim() == 4, "need a device tensor [slots, tokens, heads, head_dim]"
    ss, ts, hs, cs = t.stride()
    assert cs == 1 or t.shape[3] < 2, "a head's columns must be contiguous"
    assert t.dtype in (torch.bfloat16, torch.float32), "expected bfloat16 or float32"
    if like is not None:
        assert t.dtype == like.dtype, "tensors of two types"
        assert t.device == like.device, "tensors on two devices"
        assert not same or t.shape == like.shape, "an output must have the shape of its input"
    return Heads(t.data_ptr(), ss, ts, hs)


def _vector(t, dtype, n, like, what):
    """Device pointer of a contiguous tensor of n elements on the device of `like`, or None."""
    if t is None:
        return None
    p = _dev(t, dtype)
    assert t.device == like.device, "tensors on two devices"
    assert t.numel() == n, "%s must have %d elements" % (what, n)
    return p


def _current(x):
    """The current stream, if x is on the current device."""
    import torch
    device = torch.cuda.current_device()
    assert x.device.index == device, "the tensors are not on the current device"
    return torch._C._cuda_getCurrentRawStream(device)


class _OperatorsCtypes:
    """The operators' marshalling with ctypes."""

    @staticmethod
    def _positions(t, config, x):
        import torch
        if t is None:
            return None, 0
        if config is None:
            raise ValueError("positions without a rotation")
        axes = RopeConfig.from_address(config).n_axes
        want = (x.shape[1], axes)
        assert tuple(t.shape) in (want, (x.shape[0],) + want), "positions must be [tokens, axes] or [slots, tokens, axes]"
        return _vector(t, torch.float32, t.numel(), x, "positions"), x.shape[1] * axes if t.dim() == 3 else 0

    @staticmethod
    def _shape(q, k, q_lens, kv_lens):
        import torch
        hq, hk = _heads(q), _heads(k, q)
        assert q.shape[0] == k.shape[0] and q.shape[3] == k.shape[3], "k must have the slots and head width of q"
        S = q.shape[0]
        return hq, hk, AttnShape(BF16 if q.dtype == torch.bfloat16 else F32, S, q.shape[1], k.shape[1], q.shape[2], k.shape[2], q.shape[3],
                                 _vector(q_lens, torch.int32, S, q, "q_lens"), _vector(kv_lens, torch.int32, S, q, "kv_lens"))

    @staticmethod
    def _words(shape, q_block, kv_block):
        return (-(-shape.q_tokens // q_block) if q_block > 0 else 0) * shape.slots * shape.q_heads * _lib.drf_block_words(shape.kv_tokens, kv_block)

    @classmethod
    def rope(cls, x, out, config, positions, lens):
        import torch
        hx, ho = _heads(x), _heads(out, x, True)
        p, stride = cls._positions(positions, config, x)
        ln = _vector(lens, torch.int32, x.shape[0], x, "lens")
        return _lib.drf_rope(config, BF16 if x.dtype == torch.bfloat16 else F32, *x.shape, ln, p, stride, C.byref(hx), C.byref(ho), _current(x))

    @classmethod
    def qk_norm_rope(cls, q, k, q_out, k_out, norm, eps, q_scale, q_gain, q_bias, k_gain, k_bias, config, positions, lens):
        import torch
        hq, hk, hqo, hko = _heads(q), _heads(k, q), _heads(q_out, q, True), _heads(k_out, k, True)
        assert q.shape[:2] == k.shape[:2] and q.shape[3] == k.shape[3], "k must have the slots, tokens and head width of q"
        cfg = QkConfig(norm, eps, q_scale, *(_vector(t, torch.float32, q.shape[3], q, "a norm's parameters") for t in (q_gain, q_bias, k_gain, k_bias)))
        p, stride = cls._positions(positions, config, q)
        S, N, H, d = q.shape
        shape = AttnShape(BF16 if q.dtype == torch.bfloat16 else F32, S, N, N, H, k.shape[2], d, _vector(lens, torch.int32, S, q, "lens"), None)
        return _lib.drf_qk_norm_rope(C.byref(cfg), config, C.byref(shape), p, stride, C.byref(hq), C.byref(hk), C.byref(hqo), C.byref(hko), _current(q))

    @classmethod
    def block_select(cls, q, k, out, q_block, kv_block, topk, q_lens, kv_lens, scratch):
        import torch
        hq, hk, shape = cls._shape(q, k, q_lens, kv_lens)
        n = _lib.drf_block_select_scratch_bytes(C.byref(shape), q_block, kv_block)
        o = _vector(out, torch.int32, cls._words(shape, q_block, kv_block), q, "the blocks' words")
        sc = _vector(scratch, torch.float32, n // 4, q, "scratch")
        return _lib.drf_block_select(C.byref(shape), q_block, kv_block, topk, C.byref(hq), C.byref(hk), sc, n, o, _current(q))

    @classmethod
    def block_attention(cls, q, k, v, blocks, out, q_block, kv_block, scale, q_lens, kv_lens, scratch):
        import torch
        hq, hk, shape = cls._shape(q, k, q_lens, kv_lens)
        hv, ho = _heads(v, k, True), _heads(out, q, True)
        w = _vector(blocks, torch.int32, cls._words(shape, q_block, kv_block), q, "the blocks' words")
        n = 0 if scratch is None else _lib.drf_block_attention_scratch_bytes(C.byref(shape))
        return _lib.drf_block_attention_split(C.byref(shape), q_block, kv_block, scale, w, C.byref(hq), C.byref(hk), C.byref(hv), C.byref(ho),
                                              _vector(scratch, torch.float32, n // 4, q, "scratch"), n, _current(q))


_ops = None             # _native or _OperatorsCtypes, at the first operator


def _operators():
    global _ops
    import torch
    L = lib()
    try:
        from . import _native
        _native.bind_operators(tuple(C.cast(f, C.c_void_p).value for f in (L.drf_rope, L.drf_qk_norm_rope, L.drf_block_words, L.drf_block_select_scratch_bytes,
                                                                           L.drf_block_select, L.drf_block_attention_scratch_bytes, L.drf_block_attention_split)),
                               torch.float32, torch.bfloat16, torch.int32, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
        _ops = _native
    except ImportError:
        _ops = _OperatorsCtypes
    return _ops


def rope_config(dims, extents, theta=10000.0, layout="pairs", origin=None, step=None):
    """The rotation of rope() and qk_norm_rope(): columns, grid extent, origin and step of up to three axes (see include/drf.h)."""
    n = len(dims)
    if not 1 <= n <= 3 or len(extents) != n:
        raise ValueError("one to three axes, with an extent for each")
    rc = RopeConfig(n_axes=n, theta=float(theta), layout=_LAYOUTS[layout])
    for a in range(n):
        rc.dim[a], rc.extent[a] = int(dims[a]), int(extents[a])
        rc.origin[a] = 0.0 if origin is None else float(origin[a])
        rc.step[a] = 1.0 if step is None else float(step[a])
    return rc


def rope(x, config, positions=None, lens=None, out=None):
    """x [slots, tokens, heads, head_dim] (any strides but the last) with its columns turned by their positions; out may be x.  Rows behind a
    slot's length are left as they were: those of x in an output made here.  No gradient is recorded; that of x is the result's, turned back by the
    rotation with origin and step negated."""
    import torch
    if out is None:
        out = torch.empty_like(x) if lens is None else x.detach().clone()
    _check((_ops or _operators()).rope(x, out, C.addressof(config), positions, lens))
    return out


def qk_norm_rope(q, k, norm, config=None, q_gain=None, k_gain=None, q_bias=None, k_bias=None, eps=1e-6, q_scale=1.0, positions=None, lens=None,
                 q_out=None, k_out=None):
    """Norm ("none", "rms", "layer") of every head of q and k [slots, tokens, heads, head_dim], then the rotation; returns (q_out, k_out).  Outputs may
    be their inputs; rows behind a slot's length as in rope().  No gradient is recorded."""
    import torch
    if q_out is None:
        q_out = torch.empty_like(q) if lens is None else q.detach().clone()
    if k_out is None:
        k_out = torch.empty_like(k) if lens is None else k.detach().clone()
    _check((_ops or _operators()).qk_norm_rope(q, k, q_out, k_out, _QK[norm], float(eps), float(q_scale), q_gain, q_bias, k_gain, k_bias,
                                               None if config is None else C.addressof(config), positions, lens))
    return q_out, k_out


def block_select(q, k, q_block, kv_block, topk, q_lens=None, kv_lens=None, out=None):
    """Bit words [slots, heads, query blocks, words] (int32) of the topk key blocks whose mean lies nearest each query block's mean."""
    import torch
    ops = _ops or _operators()
    S, N, H, d = q.shape
    if out is None:
        out = torch.empty((S, H, -(-N // q_block) if q_block > 0 else 0, _lib.drf_block_words(k.shape[1], kv_block)), dtype=torch.int32, device=q.device)
    shape = AttnShape(F32, S, N, k.shape[1], H, k.shape[2], d, None, None)
    scratch = torch.empty(_lib.drf_block_select_scratch_bytes(C.byref(shape), q_block, kv_block) // 4, dtype=torch.float32, device=q.device)
    _check(ops.block_select(q, k, out, q_block, kv_block, topk, q_lens, kv_lens, scratch))
    return out


def block_attention(q, k, v, blocks, q_block, kv_block, scale=None, q_lens=None, kv_lens=None, out=None, split=False):
    """softmax(scale q k^T) v over the key blocks that the words `blocks` (as block_select gives them) name for each query block; scale
    1 / sqrt(head_dim) by default.  No gradient is recorded.  Rows behind a slot's q length are left as they were: zeros in an output made here.  split: several workgroups
    share a head where its queries are few and its keys many (for lists from about 1500 keys on, in bf16 over 8192 tokens or more; other calls are as without)."""
    import torch
    if out is None:
        out = (torch.empty if q_lens is None else torch.zeros)(q.shape, dtype=q.dtype, device=q.device)
    ops, scratch = _ops or _operators(), None
    if split:
        shape = AttnShape(BF16 if q.dtype == torch.bfloat16 else F32, q.shape[0], q.shape[1], k.shape[1], q.shape[2], k.shape[2], q.shape[3], None, None)
        n = _lib.drf_block_attention_scratch_bytes(C.byref(shape))
        scratch = torch.empty(n // 4, dtype=torch.float32, device=q.device) if n else None
    _check(ops.block_attention(q, k, v, blocks, out, q_block, kv_block, q.shape[3] ** -0.5 if scale is None else scale, q_lens, kv_lens, scratch))
    return out


def probe_gemm_bf16(A, W, bias, out=None, variant=0):
    """out[M,N] = A[M,K] @ W[N,K]^T + bias with the library's bf16 GEMM (measurement hook)."""
    import torch
    M, K = A.shape
    N = W.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    _check(lib().drf_probe_gemm_bf16(_dev(A, torch.bfloat16), _dev(W, torch.bfloat16), M, N, K,
                                     _dev(out, torch.bfloat16), _dev(bias, torch.float32), variant, _stream()))
    return out


def probe_gemm_route(M, N, K, kind=0, rows_per_slot=256):
    """(tile, parts of K, tile of the first rows, first rows) of a bf16 GEMM (host only, see include/drf_measure.h)."""
    route = (C.c_int * 4)()
    _check(lib().drf_probe_gemm_route(M, N, K, kind, rows_per_slot, route))
    return tuple(route)


def probe_attn_bf16(qkv, slots, tokens, heads, head_dim, out=None):
    """Self-attention of the library on a packed bf16 [slots*tokens, 3*heads*head_dim] tensor (measurement hook)."""
    import torch
    if out is None:
        out = torch.empty((slots * tokens, heads * head_dim), dtype=torch.bfloat16, device=qkv.device)
    _check(lib().drf_probe_attn_bf16(_dev(qkv, torch.bfloat16), _dev(out, torch.bfloat16), slots, tokens, heads, head_dim,
                                     _stream()))
    return out


def probe_cross_attn_bf16(q, kv, slots, kv_slots, q_rows, kv_rows, heads, head_dim, q_scaled=False, out=None):
    """Attention of bf16 q [slots*q_rows, heads*head_dim] over bf16 kv [kv_slots*kv_rows, 2*heads*head_dim], slot j over kv
    slot j % kv_slots (measurement hook)."""
    import torch
    if out is None:
        out = torch.empty((slots * q_rows, heads * head_dim), dtype=torch.bfloat16, device=q.device)
    _check(lib().drf_probe_cross_attn_bf16(_dev(q, torch.bfloat16), _dev(kv, torch.bfloat16), _dev(out, torch.bfloat16), slots, kv_slots,
                                           q_rows, kv_rows, heads, head_dim, int(q_scaled), _stream()))
    return out


def probe_attn_route(slots, q_rows, kv_rows, heads, head_dim, q_scaled=False):
    """Number of the bf16 attention kernel that takes a launch of these sizes (host only, see include/drf_measure.h)."""
    return lib().drf_probe_attn_route(slots, q_rows, kv_rows, heads, head_dim, int(q_scaled))


def probe_block_route(slots, tokens, hidden, heads, mlp_ratio=4):
    """How a bf16 pass of these sizes runs its blocks (host only, see include/drf_measure.h)."""
    return lib().drf_probe_block_route(slots, tokens, hidden, heads, mlp_ratio)


def probe_update_fused(sched, s_from, n_chain, n_draft, g, w, x_base, eps, x_out=None, draft_out=None):
    """One launch of the fused guidance + refine-chain + draft update kernel (measurement hook).
    x_base [field...], eps [max(n_chain,1), g, field...]; returns (x_out, draft_out [n_draft, field...])."""
    import torch
    sc = sched_config(sched)
    field = x_base.numel()
    if x_out is None:
        x_out = torch.empty_like(x_base)
    if draft_out is None and n_draft > 0:
        draft_out = torch.empty((n_draft,) + tuple(x_base.shape), dtype=torch.float32, device=x_base.device)
    _check(lib().drf_probe_update_fused(C.byref(sc), s_from, n_chain, n_draft, g, float(w), field, _dev(x_base, torch.float32),
                                        _dev(eps, torch.float32), _dev(x_out, torch.float32), _dev(draft_out, torch.float32),
                                        _stream()))
    return x_out, draft_out


def calibrate_mfma_bf16(random_operands=True, iters=5):
    """TFLOP/s of a loop of nothing but the GEMM kernel's MFMA instruction on this GPU (measurement hook)."""
    v = C.c_double(0)
    _check(lib().drf_calibrate_mfma_bf16(1 if random_operands else 0, iters, C.byref(v), _stream()))
    return v.value


def calibrate_copy(src, dst, iters=5):
    """GB/s (read + written) of a plain copy kernel between two device tensors of equal size (measurement hook)."""
    v = C.c_double(0)
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == nbytes
    _check(lib().drf_calibrate_copy(_dev(src), _dev(dst), nbytes, iters, C.byref(v), _stream()))
    return v.value


class Denoiser:
    """Owns a drf_denoiser handle."""

    def __init__(self, dit, host_weights):
        self.dit = dict(dit)
        w = np.ascontiguousarray(host_weights, np.float32)
        cfg, attn = dit_config(dit), attn_config(dit)
        h = C.c_void_p()
        _check(lib().drf_denoiser_create_attn(C.byref(cfg), None if attn is None else C.byref(attn), w.ctypes.data_as(C.c_void_p), w.size, _stream(), C.byref(h)))
        self.h = h

    def close(self):
        h, self.h = getattr(self, "h", None), None
        if h and _lib is not None:              # at interpreter exit the module may already be torn down
            _lib.drf_denoiser_destroy(h)

    __del__ = close

    def reserve(self, max_slots):
        _check(lib().drf_denoiser_reserve(self.h, max_slots))

    def use_graphs(self, mode):
        """0: sample() launches kernel by kernel; 1 (default): replays a captured graph from the second identical
        call on; 2: captures at the first call."""
        _check(lib().drf_denoiser_use_graphs(self.h, int(mode)))

    def graph_stats(self):
        a, b, c = C.c_int(0), C.c_int(0), C.c_longlong(0)
        _check(lib().drf_graph_stats(self.h, C.byref(a), C.byref(b), C.byref(c)))
        return dict(captured=a.value, failed=b.value, replays=c.value)

    def _cond_dtype(self):
        import torch
        return torch.int32 if self.dit["cond"] == COND_CLASS else torch.float32

    def eps_batched(self, x, t, cond, out=None):
        import torch
        if out is None:
            out = torch.empty_like(x)
        _check(lib().drf_eps_batched(self.h, _dev(x, torch.float32), _dev(t, torch.int32),
                                     _dev(cond, self._cond_dtype()), x.shape[0], _dev(out, torch.float32), _stream()))
        return out

    def eps_batched_static(self, x, t, cond, out):
        """drf_eps_batched on the library's static scratch array: the call allocates nothing, so `out` is required."""
        import torch
        _check(lib().drf_eps_batched_static(self.h, _dev(x, torch.float32), _dev(t, torch.int32),
                                            _dev(cond, self._cond_dtype()), x.shape[0], _dev(out, torch.float32), _stream()))
        return out

    def eps_trace(self, x, t, cond, n_blocks):
        import torch
        d = self.dit
        T = (d["lat_h"] // d["patch"]) * (d["lat_w"] // d["patch"])
        out = torch.empty((x.shape[0], T, d["hidden"]), dtype=torch.float32, device=x.device)
        _check(lib().drf_eps_trace(self.h, _dev(x, torch.float32), _dev(t, torch.int32),
                                   _dev(cond, self._cond_dtype()), x.shape[0], n_blocks, _dev(out), _stream()))
        return out

    def sample(self, sched, mode, n, x_T, cond, null_cond=None, cfg_scale=0.0, out=None):
        import torch
        sc = sched_config(sched)
        if out is None:
            out = torch.empty_like(x_T)
        _check(lib().drf_sample(self.h, C.byref(sc), mode, n, x_T.shape[0], _dev(x_T, torch.float32),
                                _dev(cond, self._cond_dtype()), _dev(null_cond, self._cond_dtype()),
                                float(cfg_scale or 0.0), _dev(out, torch.float32), _stream()))
        return out

    def sample_noise(self, sched, mode, n, x_T, cond, null_cond=None, cfg_scale=0.0, z=None, seed=None, field0=0,
                     out=None):
        import torch
        sc = sched_config(sched)
        if out is None:
            out = torch.empty_like(x_T)
        nz = _noise(z, seed, field0)
        _check(lib().drf_sample_noise(self.h, C.byref(sc), mode, n, x_T.shape[0], _dev(x_T, torch.float32),
                                      _dev(cond, self._cond_dtype()), _dev(null_cond, self._cond_dtype()),
                                      float(cfg_scale or 0.0), C.byref(nz) if nz is not None else None,
                                      _dev(out, torch.float32), _stream()))
        return out

    def profile_enable(self, on=1):
        """0 off, 1 (True) per launch, 2 per predictor pass of sample()"""
        _check(lib().drf_profile_enable(self.h, int(on)))

    def profile_read(self, which):
        n, ms, work = C.c_longlong(0), C.c_double(0), C.c_double(0)
        _check(lib().drf_profile_read(self.h, which, C.byref(n), C.byref(ms), C.byref(work)))
        return dict(launches=n.value, ms=ms.value, work=work.value)
