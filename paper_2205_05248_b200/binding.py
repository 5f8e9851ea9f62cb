"""Thin Python binding of the C-ABI actor library (``include/marl_actor.h``).

Argument marshalling only: torch supplies device memory and streams, every step of the path runs in the
library's CUDA kernels.  The shared object is built in-tree by ``paper_2205_05248_b200.build``; if it is
missing, or no CUDA device is present, calls fail with an exception - there is no CPU path.

The module-level functions carry the C names (``marl_actor_create`` ...); ``Actor`` wraps a handle together
with the torch tensors that back its ring, state and staging memory.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmarl_actor.so")

PRECISION = {"fp32": 0, "bf16": 1}
KERNEL = {"auto": 0, "ffma": 1, "tensor": 2, "pipelined": 3, "dual": 4}
STATUS_NO_AVAIL, STATUS_TIMEOUT, STATUS_BAD_INDEX = 1, 2, 4

# Debug aid: with GUARD_BYTES > 0 (a multiple of 256; the test-suite sets it) every buffer an Actor hands to the
# library gets that many guard bytes of a fixed pattern in front of it and behind it, and ``Actor.check_guards``
# (called by ``destroy``) raises if the library has written outside a buffer.
GUARD_BYTES = 0
GUARD_PATTERN = 0xA5

EXPORTS = [
    "marl_actor_query_sizes", "marl_actor_create", "marl_actor_set_weights", "marl_actor_set_weights_typed",
    "marl_actor_publish_weights",
    "marl_actor_weights_version",
    "marl_actor_step", "marl_actor_step_subset", "marl_actor_step_lagged", "marl_actor_step_host", "marl_env_generate", "marl_rollout_staged", "marl_rollout",
    "marl_actor_set_trace", "marl_ring_view", "marl_ring_sample", "marl_actor_get_state", "marl_actor_set_state",
    "marl_actor_status", "marl_actor_reset", "marl_actor_destroy", "marl_actor_kernel_name",
    "marl_actor_step_kernel",
    "marl_actor_launch_count", "marl_last_error", "marl_rollout_noalloc", "marl_selftest_bounded_wait",
    "marl_measure_ffma_tflops", "marl_policy_logprob", "marl_policy_logprob_backward",
    "marl_linear_scan_query", "marl_linear_scan", "marl_linear_scan_backward",
    "marl_orthogonalise",
]
DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
MAX_TOP = 32
SCAN_FORM = {"raw": 0, "blend": 1}
SCAN_INTERVAL = 64


class MarlError(RuntimeError):
    pass


class Config(C.Structure):
    _fields_ = [("n_envs", C.c_int32), ("n_agents", C.c_int32), ("obs_dim", C.c_int32), ("n_actions", C.c_int32),
                ("hidden", C.c_int32), ("ring_episodes", C.c_int32), ("ring_steps", C.c_int32),
                ("precision", C.c_int32), ("kernel", C.c_int32), ("n_agent_types", C.c_int32), ("seed", C.c_uint64),
                ("stream", C.c_void_p), ("ring_mem", C.c_void_p), ("ring_bytes", C.c_size_t),
                ("state_mem", C.c_void_p), ("state_bytes", C.c_size_t), ("work_mem", C.c_void_p),
                ("work_bytes", C.c_size_t)]


class Sizes(C.Structure):
    _fields_ = [("ring_bytes", C.c_size_t), ("state_bytes", C.c_size_t), ("work_bytes_min", C.c_size_t),
                ("work_bytes_per_step", C.c_size_t)]


class SynthEnv(C.Structure):
    _fields_ = [("seed", C.c_uint64), ("obs_law", C.c_int32), ("done_thresh24", C.c_uint32),
                ("avail_thresh_first", C.c_uint32), ("avail_thresh_rest", C.c_uint32), ("avail_split", C.c_int32),
                ("n_type0", C.c_int32), ("type_block_start", C.c_int32), ("type_block_len", C.c_int32)]


class SampleBatch(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("obs", "avail", "action", "q", "reward", "done", "slot", "len", "epid")]


class RingView(C.Structure):
    _fields_ = [("base", C.c_void_p), ("slot_stride", C.c_size_t), ("step_stride", C.c_size_t),
                ("off_obs", C.c_size_t), ("off_avail", C.c_size_t), ("off_action", C.c_size_t),
                ("off_q", C.c_size_t), ("off_reward", C.c_size_t), ("off_done", C.c_size_t),
                ("episodes", C.c_int32), ("steps", C.c_int32), ("slots_per_env", C.c_int32), ("n_envs", C.c_int32),
                ("n_agents", C.c_int32), ("obs_dim", C.c_int32), ("n_actions", C.c_int32), ("reserved", C.c_int32),
                ("slot_epid", C.c_void_p), ("slot_len", C.c_void_p), ("slot_complete", C.c_void_p)]


class StateView(C.Structure):
    _fields_ = [("h", C.c_void_p), ("last_action", C.c_void_p), ("slot", C.c_void_p), ("pos", C.c_void_p),
                ("ep_count", C.c_void_p), ("step", C.c_uint64)]


class PolicyRows(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("avail", C.c_void_p), ("action", C.c_void_p), ("rows", C.c_int64),
                ("row_stride", C.c_int64), ("avail_stride", C.c_int64), ("n_actions", C.c_int32), ("dtype", C.c_int32),
                ("temperature", C.c_float), ("reserved", C.c_int32)]


class Scan(C.Structure):
    _fields_ = [("gate", C.c_void_p), ("x", C.c_void_p), ("gate_b", C.c_int64), ("gate_t", C.c_int64), ("x_b", C.c_int64),
                ("x_t", C.c_int64), ("gate_c", C.c_int32), ("x_c", C.c_int32), ("h0", C.c_void_p), ("done", C.c_void_p),
                ("length", C.c_void_p), ("B", C.c_int32), ("L", C.c_int32), ("C", C.c_int32), ("dtype", C.c_int32),
                ("form", C.c_int32), ("reverse", C.c_int32)]


class Matrix(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("out", C.c_void_p), ("in_batch", C.c_int64), ("in_row", C.c_int64), ("out_batch", C.c_int64),
                ("out_row", C.c_int64), ("batch", C.c_int32), ("rows", C.c_int32), ("cols", C.c_int32), ("scale", C.c_float)]


class Counters(C.Structure):
    _fields_ = [("agent_steps", C.c_uint64), ("episodes", C.c_uint64), ("explored", C.c_uint64),
                ("no_avail", C.c_uint64), ("truncated", C.c_uint64)]


_lib = None


def load_library():
    """Loads libmarl_actor.so (no CUDA call is made by loading).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MarlError(f"{LIB_PATH} is missing: run `python -m paper_2205_05248_b200.build` (there is no "
                            "CPU fallback)")
        lib = C.CDLL(LIB_PATH)
        P = C.c_void_p
        lib.marl_last_error.restype = C.c_char_p
        lib.marl_actor_kernel_name.restype = C.c_char_p
        lib.marl_actor_kernel_name.argtypes = [P]
        lib.marl_actor_step_kernel.restype = C.c_char_p
        lib.marl_actor_step_kernel.argtypes = [P]
        lib.marl_actor_launch_count.restype = C.c_uint64
        lib.marl_actor_launch_count.argtypes = [P]
        lib.marl_actor_weights_version.restype = C.c_uint64
        lib.marl_actor_weights_version.argtypes = [P]
        lib.marl_actor_destroy.restype = None
        lib.marl_actor_destroy.argtypes = [P]
        lib.marl_actor_query_sizes.argtypes = [C.POINTER(Config), C.POINTER(Sizes)]
        lib.marl_actor_create.argtypes = [C.POINTER(Config), C.POINTER(P)]
        lib.marl_actor_set_weights.argtypes = [P] + [P] * 8 + [C.c_uint64]
        lib.marl_actor_set_weights_typed.argtypes = [P, C.c_int32, P] + [P] * 8 + [C.c_uint64]
        lib.marl_actor_publish_weights.argtypes = [P] + [P] * 8 + [C.c_uint64, C.c_uint64]
        lib.marl_actor_step.argtypes = [P, P, P, P, P, C.c_float, P]
        lib.marl_actor_step_host.argtypes = [P, P, P, P, P, C.c_float, P]
        lib.marl_actor_step_subset.argtypes = [P, P, C.c_int32, P, P, P, P, C.c_float, P]
        lib.marl_actor_step_lagged.argtypes = [P, P, C.c_int32, P, P, P, P, C.c_float, P]
        lib.marl_env_generate.argtypes = [P, C.POINTER(SynthEnv), C.c_uint32, C.c_int32, P, P, P, P]
        lib.marl_rollout_staged.argtypes = [P, P, P, P, P, C.c_int32, C.c_double, C.c_double, C.c_int32]
        lib.marl_rollout.argtypes = [P, C.POINTER(SynthEnv), C.c_int32, C.c_double, C.c_double, C.c_int32]
        lib.marl_rollout_noalloc.argtypes = [P, C.POINTER(SynthEnv), C.c_int32, C.c_double, C.c_double, C.c_int32]
        lib.marl_measure_ffma_tflops.argtypes = [P, C.POINTER(C.c_double)]
        lib.marl_selftest_bounded_wait.argtypes = [P, C.c_uint32, C.POINTER(C.c_uint32)]
        lib.marl_actor_set_trace.argtypes = [P, P, P, C.c_int32]
        lib.marl_ring_view.argtypes = [P, C.POINTER(RingView)]
        lib.marl_ring_sample.argtypes = [P, C.c_uint32, C.c_int32, C.POINTER(SampleBatch)]
        lib.marl_actor_get_state.argtypes = [P, C.POINTER(StateView)]
        lib.marl_actor_set_state.argtypes = [P, C.POINTER(StateView)]
        lib.marl_actor_status.argtypes = [P, C.POINTER(C.c_uint32), C.POINTER(Counters)]
        lib.marl_actor_reset.argtypes = [P]
        lib.marl_policy_logprob.argtypes = [P, C.POINTER(PolicyRows), C.c_int32, P, P, P, P, P]
        lib.marl_policy_logprob_backward.argtypes = [P, C.POINTER(PolicyRows), P, P, P, P, P, C.c_int64]
        lib.marl_orthogonalise.argtypes = [P, C.POINTER(Matrix), C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_float), C.c_float]
        lib.marl_linear_scan_query.argtypes = [C.POINTER(Scan), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        lib.marl_linear_scan.argtypes = [P, C.POINTER(Scan), P, P, P, P, C.c_size_t]
        lib.marl_linear_scan_backward.argtypes = [P, C.POINTER(Scan), P, P, C.c_int64, C.c_int64, P, P, P, P, P, C.c_size_t]
        _lib = lib
    return _lib


def _check(rc: int):
    if rc != 0:
        raise MarlError(f"marl error {rc}: {load_library().marl_last_error().decode()}")


def make_env(env: dict) -> SynthEnv:
    return SynthEnv(int(env["seed"]), int(env["obs_law"]), int(env["done_thresh24"]),
                    int(env["avail_thresh_first"]), int(env["avail_thresh_rest"]), int(env["avail_split"]),
                    int(env["n_type0"]), int(env["type_block_start"]), int(env["type_block_len"]))


def make_config(cfg: dict, kernel: str = "auto") -> Config:
    prec = cfg["precision"]
    prec = PRECISION.get(prec, prec)
    c = Config()
    c.n_envs, c.n_agents, c.obs_dim, c.n_actions, c.hidden = cfg["E"], cfg["n"], cfg["D"], cfg["A"], cfg["H"]
    c.ring_episodes, c.ring_steps, c.precision, c.kernel = cfg["C"], cfg["L"], int(prec), KERNEL[kernel]
    c.seed = int(cfg["seed"])
    c.n_agent_types = (max(cfg["agent_type"]) + 1) if cfg.get("agent_type") is not None else 0
    return c


def marl_actor_query_sizes(cfg: dict) -> dict:
    s = Sizes()
    c = make_config(cfg)
    _check(load_library().marl_actor_query_sizes(C.byref(c), C.byref(s)))
    return {k: getattr(s, k) for k, _ in Sizes._fields_}


def marl_measure_ffma_tflops() -> float:
    """fp32 FMA peak of the current device under load, in TFLOP/s (measured by the library)."""
    out = C.c_double(0)
    stream = torch.cuda.current_stream().cuda_stream
    _check(load_library().marl_measure_ffma_tflops(C.c_void_p(stream), C.byref(out)))
    return float(out.value)


def marl_selftest_bounded_wait(poll_limit: int = 20000) -> int:
    """Runs the bounded-wait self-test on the current stream; returns the reported status word."""
    st = C.c_uint32(0)
    stream = torch.cuda.current_stream().cuda_stream
    _check(load_library().marl_selftest_bounded_wait(C.c_void_p(stream), C.c_uint32(poll_limit), C.byref(st)))
    return int(st.value)


def _dptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


# ---- the learner's operators (device tensors, on the current stream of their device) ------------------------------------
# They are not part of autograd: results carry no graph, whether or not the inputs require gradients, and a gradient is asked for with
# the *_backward function of the same name.  marl_orthogonalise has none.
# Calls of a few microseconds of GPU work are common here, so the marshalling is kept short: no text is made unless a check
# fails, the stream is asked for as a number, and dense outputs are made with their strides.
_F32, _I32 = torch.float32, torch.int32


def _device_call(dev, fn, *args):
    """fn(stream, *args) with the tensors' device current, on its current stream."""
    index = dev.index
    stream = torch._C._cuda_getCurrentRawStream(index)
    if torch._C._cuda_getDevice() == index:
        rc = fn(stream, *args)
    else:
        with torch.cuda.device(dev):
            rc = fn(stream, *args)
    if rc != 0:
        _check(rc)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _new(shape, dtype, dev):
    """A dense tensor."""
    stride, n = [], 1
    for s in reversed(shape):
        stride.append(n)
        n *= s if s > 1 else 1
    return torch.empty_strided(shape, stride[::-1], dtype=dtype, device=dev)


def _rows_of(t, name: str):
    """t[..., A] as rows: (number of rows, elements between rows); the elements of a row must be neighbours."""
    shape, strides = t.shape, t.stride()
    A = shape[-1]
    if A < 1 or (strides[-1] != 1 and A != 1):
        raise MarlError(f"{name} has no entries, or the entries of a row are not neighbours")
    rows, stride = 1, None
    for k in range(len(shape) - 2, -1, -1):
        n = shape[k]
        if n == 0:
            return 0, A
        if n == 1:
            continue
        if stride is None:
            stride = strides[k]
        elif strides[k] != stride * rows:
            raise MarlError(f"{name} cannot be walked as rows at one distance")
        rows *= n
    return rows, (A if stride is None else stride)


def _dense(t, dtype, shape, dev, name: str):
    """The address of a dense tensor of that type and shape on that device; None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.device != dev or not t.is_contiguous():
        raise MarlError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {dev}")
    return t.data_ptr()


def _policy_rows(logits, action, avail, temperature: float):
    if not logits.is_cuda:
        raise MarlError("logits must be a CUDA tensor: there is no CPU path")
    dt = DTYPE.get(logits.dtype)
    if dt is None or logits.dim() < 1:
        raise MarlError("logits must be a float32, bfloat16 or float16 tensor of at least one dimension")
    shape, dev = logits.shape, logits.device
    lead = shape[:-1]
    rows, stride = _rows_of(logits, "logits")
    if action is None:
        raise MarlError("action is None")
    act = _dense(action, _I32, lead, dev, "action")
    av, astride = None, 0
    if avail is not None:
        if avail.dtype not in (torch.uint8, torch.bool) or avail.shape != shape or avail.device != dev:
            raise MarlError(f"avail must be a uint8 or bool tensor of shape {tuple(shape)} on {dev}")
        av, astride = avail.data_ptr(), _rows_of(avail, "avail")[1]
    return lead, dev, PolicyRows(logits.data_ptr(), av, act, rows, stride, astride, shape[-1], dt, temperature, 0)


def marl_policy_logprob(logits, action, avail=None, temperature: float = 1.0, top: int = 0) -> dict:
    """Log probability of the action taken, entropy and the `top` best alternatives of each row of logits [..., A] (the q of a
    sampled batch).  action int32 [...], avail uint8 or bool [..., A].  Returns logp, entropy float32 [...], stats float32
    [..., 2] (for the gradient), top_index int32 and top_logp float32 [..., top] (None with top = 0).  Not recorded by autograd: the
    gradient is marl_policy_logprob_backward."""
    lead, dev, p = _policy_rows(logits, action, avail, temperature)
    if not 0 <= top <= MAX_TOP:
        raise MarlError(f"top must be in [0, {MAX_TOP}]")
    logp, entropy, stats = _new(lead, _F32, dev), _new(lead, _F32, dev), _new((*lead, 2), _F32, dev)
    index = tops = None
    if top:
        index, tops = _new((*lead, top), _I32, dev), _new((*lead, top), _F32, dev)
    _device_call(dev, load_library().marl_policy_logprob, p, top, logp.data_ptr(), entropy.data_ptr(), stats.data_ptr(), _ptr(index),
                 _ptr(tops))
    return dict(logp=logp, entropy=entropy, stats=stats, top_index=index, top_logp=tops)


def marl_policy_logprob_backward(logits, action, stats, entropy, g_logp=None, g_entropy=None, avail=None,
                                 temperature: float = 1.0, out=None):
    """The gradient of marl_policy_logprob with respect to the logits, from its stats and entropy and the gradients of logp and
    entropy float32 [...] (either may be None).  Returns a tensor like logits (dense, or `out`, whose rows may be further apart; `out`
    may be the logits)."""
    lead, dev, p = _policy_rows(logits, action, avail, temperature)
    if stats is None or entropy is None:
        raise MarlError("stats or entropy is None")
    st = _dense(stats, _F32, (*lead, 2), dev, "stats")
    en, gl, ge = _dense(entropy, _F32, lead, dev, "entropy"), _dense(g_logp, _F32, lead, dev, "g_logp"), _dense(g_entropy, _F32, lead, dev, "g_entropy")
    if out is None:
        out, stride = _new(logits.shape, logits.dtype, dev), logits.shape[-1]
    else:
        if out.dtype is not logits.dtype or out.shape != logits.shape or out.device != dev:
            raise MarlError("out must be like logits")
        stride = _rows_of(out, "out")[1]
    _device_call(dev, load_library().marl_policy_logprob_backward, p, st, en, gl, ge, out.data_ptr(), stride)
    return out


def _scan_args(gate, x, h0, done, length, form: str, reverse: bool):
    if not x.is_cuda:
        raise MarlError("x must be a CUDA tensor: there is no CPU path")
    dt, shape, dev = DTYPE.get(x.dtype), x.shape, x.device
    if dt is None or gate.dtype is not x.dtype:
        raise MarlError("gate and x must both be float32, bfloat16 or float16")
    if len(shape) != 3 or gate.shape != shape or gate.device != dev:
        raise MarlError("gate and x must have the same shape [B, L, C], on one device")
    f = SCAN_FORM.get(form)
    if f is None:
        raise MarlError(f"form must be one of {sorted(SCAN_FORM)}")
    B, L, Cn = shape
    h, n = _dense(h0, _F32, (B, Cn), dev, "h0"), _dense(length, _I32, (B,), dev, "length")
    d = None
    if done is not None:
        d = _dense(done, torch.bool if done.dtype is torch.bool else torch.uint8, (B, L), dev, "done")
    gb, gt, gc = gate.stride()
    xb, xt, xc = x.stride()
    if Cn <= 1:
        gc = xc = 1
    if gc not in (0, 1) or xc not in (0, 1):
        raise MarlError("the channels of gate and of x must be neighbours, or one value for all")
    return Scan(gate.data_ptr(), x.data_ptr(), gb, gt, xb, xt, gc, xc, h, d, n, B, L, Cn, dt, f, 1 if reverse else 0)


def _scan_work(s, dev):
    """Scratch of a call and its size (none where the time axis is short or the other axes are large, as most often)."""
    if s.L <= SCAN_INTERVAL:
        return None, 0
    need = C.c_size_t()
    _check(load_library().marl_linear_scan_query(s, None, need))
    n = need.value
    return (torch.empty(n, dtype=torch.uint8, device=dev) if n else None), n


def marl_linear_scan(gate, x, h0=None, done=None, length=None, form: str = "blend", reverse: bool = False, keep: bool = False) -> dict:
    """The gated linear recurrence of x [B, L, C] (its rows and those of gate may be strided; gate may be expanded).  h0 float32 [B, C],
    done uint8 or bool [B, L], length int32 [B], each may be None.  Returns y like x (dense), last float32 [B, C] and, with
    keep, the states that marl_linear_scan_backward takes.  Not recorded by autograd."""
    s = _scan_args(gate, x, h0, done, length, form, reverse)
    dev = x.device
    B, L, Cn = x.shape
    y, last = _new((B, L, Cn), x.dtype, dev), _new((B, Cn), _F32, dev)
    states = _new((B, -(-L // SCAN_INTERVAL), Cn), _F32, dev) if keep else None
    work, need = _scan_work(s, dev)
    _device_call(dev, load_library().marl_linear_scan, s, y.data_ptr(), last.data_ptr(), _ptr(states), _ptr(work), need)
    return dict(y=y, last=last, states=states)


def marl_linear_scan_backward(gate, x, states, dy, dlast=None, h0=None, done=None, length=None, form: str = "blend",
                              reverse: bool = False) -> dict:
    """The gradients of marl_linear_scan (called with the same arguments and keep=True) from those of y and, if not None, of last:
    dgate and dx like x (dense; the caller sums them where the inputs were expanded) and dh0 float32 [B, C]."""
    s = _scan_args(gate, x, h0, done, length, form, reverse)
    dev = x.device
    B, L, Cn = x.shape
    if states is None:
        raise MarlError("states is None: call marl_linear_scan with keep=True")
    st = _dense(states, _F32, (B, -(-L // SCAN_INTERVAL), Cn), dev, "states")
    dl = _dense(dlast, _F32, (B, Cn), dev, "dlast")
    if dy.dtype is not x.dtype or dy.shape != x.shape or dy.device != dev or (Cn > 1 and dy.stride(2) != 1):
        raise MarlError("dy must be like x, its channels neighbours")
    dgate, dx, dh0 = _new((B, L, Cn), x.dtype, dev), _new((B, L, Cn), x.dtype, dev), _new((B, Cn), _F32, dev)
    work, need = _scan_work(s, dev)
    _device_call(dev, load_library().marl_linear_scan_backward, s, st, dy.data_ptr(), dy.stride(0), dy.stride(1), dl, dgate.data_ptr(),
                 dx.data_ptr(), dh0.data_ptr(), _ptr(work), need)
    return dict(dgate=dgate, dx=dx, dh0=dh0)


def marl_orthogonalise(mats, steps: int = 5, coeffs=(3.4445, -4.7750, 2.0315), eps: float = 1e-7, scale=1.0, out=None) -> list:
    """Orthogonalised updates of a list of matrices [r, c] or batches of them [k, r, c] (one dtype; rows may be strided), in one
    call.  scale: one factor, or one for each entry of the list.  out: a list of tensors like mats (the same ones: in place).
    Returns the list of results, which autograd does not record."""
    mats = list(mats)
    if not mats:
        return []
    dev, dtype = mats[0].device, mats[0].dtype
    dt = DTYPE.get(dtype)
    if not mats[0].is_cuda or dt is None:
        raise MarlError("matrices must be float32, bfloat16 or float16 CUDA tensors: there is no CPU path")
    if len(coeffs) != 3:
        raise MarlError("coeffs must be three numbers")
    outs = [_new(m.shape, dtype, dev) for m in mats] if out is None else list(out)
    scales = scale if isinstance(scale, (list, tuple)) else [scale] * len(mats)
    if not len(outs) == len(mats) == len(scales):
        raise MarlError("out and scale must be as long as the list")
    entries = []
    for m, o, f in zip(mats, outs, scales):
        shape = m.shape
        if len(shape) not in (2, 3) or 0 in shape:
            raise MarlError("a matrix has shape [r, c] or [k, r, c]")
        if m.device != dev or o.device != dev or m.dtype is not dtype or o.dtype is not dtype or o.shape != shape:
            raise MarlError("the matrices must share a device and a dtype, and out must be like them")
        ms, os_ = m.stride(), o.stride()
        if shape[-1] != 1 and (ms[-1] != 1 or os_[-1] != 1):
            raise MarlError("the entries of a row must be neighbours")
        if len(shape) == 3:
            entries.append((m.data_ptr(), o.data_ptr(), ms[0], ms[1], os_[0], os_[1], shape[0], shape[1], shape[2], f))
        else:
            entries.append((m.data_ptr(), o.data_ptr(), 0, ms[0], 0, os_[0], 1, shape[0], shape[1], f))
    _device_call(dev, load_library().marl_orthogonalise, (Matrix * len(entries))(*entries), len(entries), dt, steps, (C.c_float * 3)(*coeffs), eps)
    return outs


class Actor:
    """A library handle plus the torch tensors that back it.

    work_steps: how many environment steps of staging to allocate for ``rollout`` (default: cfg['T'] if it
    fits in ``work_budget_bytes``, else as many as fit).
    """

    def __init__(self, cfg: dict, device: str = "cuda:0", kernel: str = "auto", work_steps: int | None = None,
                 work_budget_bytes: int = 24 << 30):
        if not torch.cuda.is_available():
            raise MarlError("no CUDA device: the actor library has no CPU path")
        self.lib = load_library()
        self.cfg = dict(cfg)
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        sizes = marl_actor_query_sizes(cfg)
        steps = cfg.get("T", 1) if work_steps is None else work_steps
        per = sizes["work_bytes_per_step"]
        steps = max(1, min(steps, (work_budget_bytes - sizes["work_bytes_min"]) // per + 1))
        wbytes = sizes["work_bytes_min"] + (steps - 1) * per
        u8 = dict(dtype=torch.uint8, device=self.device)
        self._guards = []

        def alloc(nbytes, zero):
            g = GUARD_BYTES
            if g <= 0:
                return torch.zeros(nbytes, **u8) if zero else torch.empty(nbytes, **u8)
            assert g % 256 == 0
            full = torch.zeros(nbytes + 2 * g, **u8) if zero else torch.empty(nbytes + 2 * g, **u8)
            full[:g] = GUARD_PATTERN
            full[g + nbytes:] = GUARD_PATTERN
            self._guards.append((full, g, nbytes))
            return full[g:g + nbytes]

        self.ring_mem = alloc(sizes["ring_bytes"], True)   # padding bytes are never written
        self.state_mem = alloc(sizes["state_bytes"], False)
        self.work_mem = alloc(wbytes, False)
        c = make_config(cfg, kernel)
        self.stream = torch.cuda.current_stream(self.device)
        c.stream = self.stream.cuda_stream
        c.ring_mem, c.ring_bytes = self.ring_mem.data_ptr(), self.ring_mem.numel()
        c.state_mem, c.state_bytes = self.state_mem.data_ptr(), self.state_mem.numel()
        c.work_mem, c.work_bytes = self.work_mem.data_ptr(), self.work_mem.numel()
        h = C.c_void_p()
        _check(self.lib.marl_actor_create(C.byref(c), C.byref(h)))
        self.handle = h
        self._trace = None
        self._keep = []

    # -- lifetime ---------------------------------------------------------------------------------
    def destroy(self):
        if getattr(self, "handle", None):
            self.lib.marl_actor_destroy(self.handle)      # synchronises the stream
            self.handle = None
            self.check_guards()

    def check_guards(self):
        """Raises if any guard byte around the ring, state or work buffer has changed (GUARD_BYTES > 0 only)."""
        for name, (full, g, nbytes) in zip(("ring_mem", "state_mem", "work_mem"), getattr(self, "_guards", [])):
            front_ok = bool((full[:g] == GUARD_PATTERN).all())
            back_ok = bool((full[g + nbytes:] == GUARD_PATTERN).all())
            if not (front_ok and back_ok):
                raise MarlError(f"the library wrote outside {name} ({'before' if not front_ok else 'behind'} the buffer)")

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # -- weights ----------------------------------------------------------------------------------
    def set_weights(self, w: dict, version: int = 1):
        import numpy as np
        arrs = [np.ascontiguousarray(w[k], dtype=np.float32)
                for k in ("W1", "b1", "W_ih", "b_ih", "W_hh", "b_hh", "W2", "b2")]
        _check(self.lib.marl_actor_set_weights(self.handle, *[a.ctypes.data_as(C.c_void_p) for a in arrs],
                                               C.c_uint64(version)))

    def set_weights_typed(self, ws: list, agent_type=None, version: int = 1):
        """marl_actor_set_weights_typed: one network (a dict like ``set_weights`` takes) per unit type; agent_type
        defaults to the configuration's."""
        import numpy as np
        types = np.ascontiguousarray(self.cfg["agent_type"] if agent_type is None else agent_type, dtype=np.int32)
        arrs = [np.ascontiguousarray(np.stack([w[k] for w in ws]), dtype=np.float32)
                for k in ("W1", "b1", "W_ih", "b_ih", "W_hh", "b_hh", "W2", "b2")]
        _check(self.lib.marl_actor_set_weights_typed(self.handle, C.c_int32(len(ws)), types.ctypes.data_as(C.c_void_p),
                                                     *[a.ctypes.data_as(C.c_void_p) for a in arrs], C.c_uint64(version)))

    def publish_weights(self, w: dict, version: int, effective_step: int):
        """marl_actor_publish_weights: the network in use from global step effective_step on."""
        import numpy as np
        arrs = [np.ascontiguousarray(w[k], dtype=np.float32)
                for k in ("W1", "b1", "W_ih", "b_ih", "W_hh", "b_hh", "W2", "b2")]
        _check(self.lib.marl_actor_publish_weights(self.handle, *[a.ctypes.data_as(C.c_void_p) for a in arrs],
                                                   C.c_uint64(version), C.c_uint64(effective_step)))

    @property
    def weights_version(self) -> int:
        return int(self.lib.marl_actor_weights_version(self.handle))

    # -- stepping ---------------------------------------------------------------------------------
    def step(self, obs, avail, reward, done, eps: float, actions_out=None):
        """marl_actor_step on device tensors; returns the int32 [E][n] action tensor."""
        E, n = self.cfg["E"], self.cfg["n"]
        if actions_out is None:
            actions_out = torch.empty((E, n), dtype=torch.int32, device=self.device)
        for t, dt in ((obs, torch.float32), (avail, torch.uint8), (reward, torch.float32), (done, torch.uint8)):
            assert t.is_cuda and t.dtype == dt and t.is_contiguous()
        _check(self.lib.marl_actor_step(self.handle, _dptr(obs), _dptr(avail), _dptr(reward), _dptr(done),
                                        C.c_float(eps), _dptr(actions_out)))
        return actions_out

    def step_lagged(self, env_ids, obs, avail, prev_reward, prev_done, eps: float, actions_out=None):
        """marl_actor_step_lagged: step_subset with the outcome of each environment's previous action."""
        return self.step_subset(env_ids, obs, avail, prev_reward, prev_done, eps, actions_out, lagged=True)

    def step_subset(self, env_ids, obs, avail, reward, done, eps: float, actions_out=None, lagged=False):
        """marl_actor_step_subset: env_ids is a host int32 array [M]; the other tensors are device tensors over the
        list.  Returns the int32 [M][n] action tensor."""
        import numpy as np
        ids = np.ascontiguousarray(env_ids, dtype=np.int32)
        M, n = int(ids.shape[0]), self.cfg["n"]
        if actions_out is None:
            actions_out = torch.empty((M, n), dtype=torch.int32, device=self.device)
        for t, dt in ((obs, torch.float32), (avail, torch.uint8), (reward, torch.float32), (done, torch.uint8)):
            assert t.is_cuda and t.dtype == dt and t.is_contiguous() and t.shape[0] == M
        fn = self.lib.marl_actor_step_lagged if lagged else self.lib.marl_actor_step_subset
        _check(fn(self.handle, ids.ctypes.data_as(C.c_void_p), C.c_int32(M), _dptr(obs), _dptr(avail), _dptr(reward),
                  _dptr(done), C.c_float(eps), _dptr(actions_out)))
        return actions_out

    def step_host(self, obs, avail, reward, done, eps: float, actions_out):
        """marl_actor_step_host on host tensors (pinned for asynchronous copies); synchronises."""
        for t in (obs, avail, reward, done, actions_out):
            assert not t.is_cuda and t.is_contiguous()
        _check(self.lib.marl_actor_step_host(self.handle, _dptr(obs), _dptr(avail), _dptr(reward), _dptr(done),
                                             C.c_float(eps), _dptr(actions_out)))
        return actions_out

    def env_generate(self, env: dict, t0: int, n_steps: int, out=None):
        """marl_env_generate into fresh (or given) device tensors laid out [step][E]..."""
        c = self.cfg
        E, n, D, A = c["E"], c["n"], c["D"], c["A"]
        if out is None:
            out = (torch.empty((n_steps, E, n, D), dtype=torch.float32, device=self.device),
                   torch.empty((n_steps, E, n, A), dtype=torch.uint8, device=self.device),
                   torch.empty((n_steps, E), dtype=torch.float32, device=self.device),
                   torch.empty((n_steps, E), dtype=torch.uint8, device=self.device))
        ev = make_env(env)
        _check(self.lib.marl_env_generate(self.handle, C.byref(ev), C.c_uint32(t0), C.c_int32(n_steps),
                                          *[_dptr(t) for t in out]))
        return out

    def rollout_staged(self, obs, avail, reward, done, T: int, eps_start: float, eps_end: float | None = None,
                       anneal_steps: int = 0):
        eps_end = eps_start if eps_end is None else eps_end
        _check(self.lib.marl_rollout_staged(self.handle, _dptr(obs), _dptr(avail), _dptr(reward), _dptr(done),
                                            C.c_int32(T), C.c_double(eps_start), C.c_double(eps_end),
                                            C.c_int32(anneal_steps)))

    def rollout(self, env: dict, T: int, eps_start: float, eps_end: float | None = None, anneal_steps: int = 0):
        eps_end = eps_start if eps_end is None else eps_end
        ev = make_env(env)
        _check(self.lib.marl_rollout(self.handle, C.byref(ev), C.c_int32(T), C.c_double(eps_start),
                                     C.c_double(eps_end), C.c_int32(anneal_steps)))

    def rollout_noalloc(self, env: dict, T: int, eps_start: float, eps_end: float | None = None,
                        anneal_steps: int = 0):
        """marl_rollout_noalloc: same results as ``rollout``, staged through the library's fixed scratch array
        (for callers that may not allocate device memory).  On failure the exception carries the return code, so
        "too large for the scratch" (-4, MARL_ENOMEM) can be told from other errors."""
        eps_end = eps_start if eps_end is None else eps_end
        ev = make_env(env)
        rc = self.lib.marl_rollout_noalloc(self.handle, C.byref(ev), C.c_int32(T), C.c_double(eps_start),
                                           C.c_double(eps_end), C.c_int32(anneal_steps))
        if rc != 0:
            raise MarlError(f"marl_rollout_noalloc failed with code {rc}")

    # -- verification trace -----------------------------------------------------------------------
    def set_trace(self, capacity_steps: int, want_q: bool = True):
        c = self.cfg
        if capacity_steps <= 0:
            self._trace = None
            _check(self.lib.marl_actor_set_trace(self.handle, None, None, 0))
            return None
        acts = torch.full((capacity_steps, c["E"], c["n"]), -7, dtype=torch.int32, device=self.device)
        q = (torch.full((capacity_steps, c["E"], c["n"], c["A"]), float("nan"), dtype=torch.float32,
                        device=self.device) if want_q else None)
        self._trace = (acts, q)
        _check(self.lib.marl_actor_set_trace(self.handle, _dptr(acts), _dptr(q), C.c_int32(capacity_steps)))
        return self._trace

    # -- views ------------------------------------------------------------------------------------
    def ring_view(self) -> dict:
        """marl_ring_view as strided torch views over the ring memory (no copies)."""
        v = RingView()
        _check(self.lib.marl_ring_view(self.handle, C.byref(v)))
        base_off = v.base - self.ring_mem.data_ptr()
        Cn, L, n, D, A = v.episodes, v.steps, v.n_agents, v.obs_dim, v.n_actions
        u8 = self.ring_mem
        f32 = u8[: u8.numel() // 4 * 4].view(torch.float32)
        i32 = u8[: u8.numel() // 4 * 4].view(torch.int32)
        ss, ps = v.slot_stride, v.step_stride

        # (as_strided offsets count from the start of the storage, and ring_mem may itself start inside one)
        so4, so1 = f32.storage_offset(), u8.storage_offset()

        def f(off, shape_tail, stride_tail):
            return torch.as_strided(f32, (Cn, L, *shape_tail), (ss // 4, ps // 4, *stride_tail), so4 + (base_off + off) // 4)

        def hdr(ptr, dtype, count):
            o = ptr - u8.data_ptr()
            nb = torch.empty((), dtype=dtype).element_size() * count
            return u8[o:o + nb].view(dtype)

        out = dict(
            obs=f(v.off_obs, (n, D), (D, 1)), q=f(v.off_q, (n, A), (A, 1)), reward=f(v.off_reward, (), ()),
            action=torch.as_strided(i32, (Cn, L, n), (ss // 4, ps // 4, 1), so4 + (base_off + v.off_action) // 4),
            avail=torch.as_strided(u8, (Cn, L, n, A), (ss, ps, A, 1), so1 + base_off + v.off_avail),
            done=torch.as_strided(u8, (Cn, L), (ss, ps), so1 + base_off + v.off_done),
            slot_epid=hdr(v.slot_epid, torch.int64, Cn), slot_len=hdr(v.slot_len, torch.int32, Cn),
            slot_complete=hdr(v.slot_complete, torch.uint8, Cn))
        out["meta"] = {k: getattr(v, k) for k, _ in RingView._fields_}
        return out

    def ring_sample(self, draw_index: int, B: int) -> dict:
        """marl_ring_sample into fresh device tensors: a dense batch of B episodes drawn from the ring."""
        c = self.cfg
        L, n, D, A = c["L"], c["n"], c["D"], c["A"]
        dev = self.device
        out = dict(obs=torch.empty((B, L, n, D), dtype=torch.float32, device=dev),
                   avail=torch.empty((B, L, n, A), dtype=torch.uint8, device=dev),
                   action=torch.empty((B, L, n), dtype=torch.int32, device=dev),
                   q=torch.empty((B, L, n, A), dtype=torch.float32, device=dev),
                   reward=torch.empty((B, L), dtype=torch.float32, device=dev),
                   done=torch.empty((B, L), dtype=torch.uint8, device=dev),
                   slot=torch.empty((B,), dtype=torch.int32, device=dev),
                   len=torch.empty((B,), dtype=torch.int32, device=dev),
                   epid=torch.empty((B,), dtype=torch.int64, device=dev))
        sb = SampleBatch(*[_dptr(out[k]) for k, _ in SampleBatch._fields_])
        _check(self.lib.marl_ring_sample(self.handle, C.c_uint32(draw_index), C.c_int32(B), C.byref(sb)))
        return out

    def get_state(self) -> dict:
        s = StateView()
        _check(self.lib.marl_actor_get_state(self.handle, C.byref(s)))
        c = self.cfg
        E, n, H = c["E"], c["n"], c["H"]
        u8 = self.state_mem
        base = u8.data_ptr()

        def arr(ptr, dtype, shape):
            cnt = 1
            for x in shape:
                cnt *= x
            nb = torch.empty((), dtype=dtype).element_size() * cnt
            return u8[ptr - base: ptr - base + nb].view(dtype).view(shape)

        return dict(h=arr(s.h, torch.float32, (E, n, H)), last_action=arr(s.last_action, torch.int32, (E, n)),
                    slot=arr(s.slot, torch.int32, (E,)), pos=arr(s.pos, torch.int32, (E,)),
                    ep_count=arr(s.ep_count, torch.int64, (E,)), step=int(s.step))

    def set_state(self, st: dict):
        s = StateView(st["h"].data_ptr(), st["last_action"].data_ptr(), st["slot"].data_ptr(), st["pos"].data_ptr(),
                      st["ep_count"].data_ptr(), int(st["step"]))
        _check(self.lib.marl_actor_set_state(self.handle, C.byref(s)))

    def status(self):
        st = C.c_uint32(0)
        cn = Counters()
        _check(self.lib.marl_actor_status(self.handle, C.byref(st), C.byref(cn)))
        return int(st.value), {k: int(getattr(cn, k)) for k, _ in Counters._fields_}

    def reset(self):
        _check(self.lib.marl_actor_reset(self.handle))

    @property
    def kernel_name(self) -> str:
        return self.lib.marl_actor_kernel_name(self.handle).decode()

    @property
    def step_kernel(self) -> str:
        """The CUDA kernel of the latest step ("" before the first)."""
        return self.lib.marl_actor_step_kernel(self.handle).decode()

    @property
    def launch_count(self) -> int:
        return int(self.lib.marl_actor_launch_count(self.handle))
