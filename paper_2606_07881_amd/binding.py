"""ctypes binding of libpaci_stage.so (argument marshalling only).

Every step of the stage runs in the HIP library. This module only converts
configs to ``paci_shapes``, hands device pointers of torch tensors and the
current HIP stream to the C ABI, and turns negative status codes into
exceptions. Importing it raises if the library has not been built.
"""
import ctypes
import os
import re

import numpy as np

# torch ships its own HIP runtime. It must be loaded before the library so
# that the library's libamdhip64 dependency resolves to that same copy. Two
# runtimes in one process do not share device allocations.
import torch  # noqa: F401

from . import inputs

# PACI_STAGE_LIB: another build of the same library (e.g. one with host-side
# sanitizers for the host-only tests); the in-tree build otherwise
LIB_PATH = os.environ.get("PACI_STAGE_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)),
                                                             "libpaci_stage.so")
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "paci_stage.h")

OK, STEP_DUE = 0, 1
E_INVAL, E_UNSUPPORTED, E_NOMEM, E_ORDER, E_BACKPRESSURE, E_STEP_PENDING, E_NOT_DUE, E_HIP, E_SCRATCH = range(-1, -10, -1)
MIDDLE, FIRST, LAST = 0, 1, 2
FP32, BF16 = 0, 1
PARAMS, GRADS, EXP_AVG, EXP_AVG_SQ = 0, 1, 2, 3
KINDS = {"middle": MIDDLE, "first": FIRST, "last": LAST}
DTYPES = {"fp32": FP32, "bf16": BF16}
ROPE_PAIRS = {"half": 0, "adjacent": 1}


class PaciShapes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "d_model", "n_heads", "head_dim", "d_ff", "seq",
                                              "micro_batch", "vocab", "max_pos", "kind", "dtype")] + \
               [(n, ctypes.c_float) for n in ("lr", "beta1", "beta2", "eps", "weight_decay", "ln_eps")] + \
               [("recompute", ctypes.c_int32), ("lr_warmup", ctypes.c_int32), ("lr_total", ctypes.c_int32),
                ("lr_min_ratio", ctypes.c_float), ("fused_head", ctypes.c_int32), ("dropout", ctypes.c_float),
                ("dropout_seed", ctypes.c_uint32), ("window", ctypes.c_int32), ("qk_norm", ctypes.c_int32),
                ("rope_dims", ctypes.c_int32), ("rope_theta", ctypes.c_float), ("rope_pairs", ctypes.c_int32),
                ("rel_buckets", ctypes.c_int32), ("rel_max_distance", ctypes.c_int32)]


class PaciCounters(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("version", "c", "q", "next_f", "next_b", "K", "delay")]


class PaciParamInfo(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("rows", ctypes.c_int32), ("cols", ctypes.c_int32),
                ("offset", ctypes.c_int64), ("numel", ctypes.c_int64), ("decay", ctypes.c_int32)]


class PaciQkShapes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "tokens", "seq", "q_heads", "k_heads", "head_dim", "norm")] + \
               [("eps", ctypes.c_float), ("rope_dims", ctypes.c_int32), ("rope_pairs", ctypes.c_int32)]


class PaciAttnShapes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "batch", "seq", "n_heads", "head_dim", "n_buckets",
                                              "max_distance")]


class PaciError(RuntimeError):
    def __init__(self, code, where="", hip=0):
        self.code = code
        self.hip = hip
        extra = f", hipError_t {hip}" if hip else ""
        super().__init__(f"{where}: {strerror(code)} ({code}{extra})")


def _load():
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2606_07881_amd.build` "
                           "(the stage has no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I, I32P, I64, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(ctypes.c_int32), ctypes.c_int64, ctypes.c_size_t
    DP = ctypes.POINTER(ctypes.c_double)
    sig = {
        "paci_fsm_create": (I, [I, I, ctypes.POINTER(P)]),
        "paci_fsm_forward": (I, [P, I, ctypes.POINTER(I)]),
        "paci_fsm_backward": (I, [P, I, ctypes.POINTER(I)]),
        "paci_fsm_step": (I, [P, ctypes.POINTER(I)]),
        "paci_fsm_counters": (I, [P, ctypes.POINTER(PaciCounters)]),
        "paci_fsm_destroy": (I, [P]),
        "paci_schedule": (I, [I, I, I, I32P, I32P, I, ctypes.POINTER(I)]),
        "paci_schedule_flush": (I, [I, I, I, I32P, I32P, I, ctypes.POINTER(I)]),
        "paci_partition": (I, [I, I, DP, DP, DP, ctypes.c_double, I32P, DP, DP]),
        "paci_eta_flush": (ctypes.c_double, [ctypes.c_double, I]),
        "paci_eta_interleaved": (ctypes.c_double, [ctypes.c_double, I, I]),
        "paci_throughput_proxy": (ctypes.c_double, [ctypes.c_double, ctypes.c_double, I]),
        "paci_param_count": (I, [ctypes.POINTER(PaciShapes), ctypes.POINTER(I), ctypes.POINTER(I64)]),
        "paci_param_info_at": (I, [ctypes.POINTER(PaciShapes), I, ctypes.POINTER(PaciParamInfo)]),
        "paci_stage_arena_bytes": (I, [ctypes.POINTER(PaciShapes), I, I, ctypes.POINTER(SZ)]),
        "paci_stage_init": (I, [ctypes.POINTER(PaciShapes), I, I, P, SZ, P, ctypes.POINTER(P)]),
        "paci_stage_destroy": (I, [P]),
        "paci_stage_load": (I, [P, I, P, I64, I]),
        "paci_stage_read": (I, [P, I, P, I64, I]),
        "paci_stage_forward": (I, [P, I, P, P, P, ctypes.POINTER(I)]),
        "paci_stage_backward": (I, [P, I, P, P, ctypes.POINTER(I)]),
        "paci_stage_backward_static": (I, [P, I, P, P, ctypes.POINTER(I)]),
        "paci_stage_step": (I, [P, ctypes.POINTER(I)]),
        "paci_stage_run": (I, [P, I, P, P, P, P, P, I32P]),
        "paci_stage_run_events": (I, [P, I, I32P, I32P, P, P, P, P, P, I32P]),
        "paci_stage_reset_counters": (I, [P]),
        "paci_stage_updates": (I, [P, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]),
        "paci_stage_resume": (I, [P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
        "paci_stage_counters": (I, [P, ctypes.POINTER(PaciCounters)]),
        "paci_stage_sync": (I, [P]),
        "paci_last_hip_error": (I, [P]),
        "paci_strerror": (ctypes.c_char_p, [I]),
        "paci_rope_freqs": (I, [ctypes.c_double, I, DP]),
        "paci_qk_norm_rope_forward": (I, [ctypes.POINTER(PaciQkShapes), P, I64, P, P, P, P, P, I64, P]),
        "paci_qk_norm_rope_workspace": (I, [ctypes.POINTER(PaciQkShapes), ctypes.POINTER(SZ)]),
        "paci_qk_norm_rope_backward": (I, [ctypes.POINTER(PaciQkShapes), P, I64, P, I64, P, P, P, P, P, I64, P, P, P, P,
                                           SZ, P]),
        "paci_rel_bounds": (I, [I, I, I32P]),
        "paci_attn_forward": (I, [ctypes.POINTER(PaciAttnShapes), P, I64, P, I64, P, I64, P, P, P, P, P]),
        "paci_attn_workspace": (I, [ctypes.POINTER(PaciAttnShapes), ctypes.POINTER(SZ)]),
        "paci_attn_backward": (I, [ctypes.POINTER(PaciAttnShapes), P, I64, P, I64, P, I64, P, P, P, P, P, P, I64, P, I64, P,
                                   I64, P, P, SZ, P]),
        "paci_kernel_family_count": (I, []),
        "paci_kernel_family_name": (ctypes.c_char_p, [I]),
        "paci_stage_set_timing": (I, [P, I]),
        "paci_stage_kernel_times": (I, [P, I, ctypes.POINTER(I64), ctypes.POINTER(ctypes.c_double),
                                        ctypes.POINTER(ctypes.c_double)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


def strerror(code):
    return lib.paci_strerror(code).decode()


def _check(code, where):
    if code < 0:
        raise PaciError(code, where)
    return code


def header_symbols():
    """Names of the functions include/paci_stage.h declares."""
    with open(HEADER) as fh:
        text = fh.read()
    return sorted(set(re.findall(r"\b(paci_[a-z_]+)\s*\(", text)))


def shapes(cfg):
    s = PaciShapes()
    for k in ("n_layers", "d_model", "n_heads", "head_dim", "d_ff", "seq", "micro_batch"):
        setattr(s, k, int(cfg[k]))
    s.vocab = int(cfg.get("vocab", 0))
    s.max_pos = int(cfg.get("max_pos", 0))
    s.kind = KINDS[cfg["kind"]]
    s.dtype = DTYPES[cfg["dtype"]]
    for k in ("lr", "beta1", "beta2", "eps", "weight_decay", "ln_eps"):
        setattr(s, k, float(cfg[k]))
    s.recompute = int(bool(cfg.get("recompute", False)))
    s.lr_warmup = int(cfg.get("lr_warmup", 0))
    s.lr_total = int(cfg.get("lr_total", 0))
    s.lr_min_ratio = float(cfg.get("lr_min_ratio", 0.1))
    s.fused_head = int(bool(cfg.get("fused_head", False)))
    s.dropout = float(cfg.get("dropout", 0.0))
    s.dropout_seed = int(cfg.get("dropout_seed", 0)) & 0xFFFFFFFF
    s.window = int(bool(cfg.get("window", False)))
    s.qk_norm = int(bool(cfg.get("qk_norm", False)))
    s.rope_dims = int(cfg.get("rope_dims", 0))
    s.rope_theta = float(cfg.get("rope_theta", 10000.0))
    s.rope_pairs = ROPE_PAIRS[cfg.get("rope_pairs", "half")]
    s.rel_buckets = int(cfg.get("rel_buckets", 0))
    s.rel_max_distance = int(cfg.get("rel_max_distance", 0))
    return s


# ---- host-only calls ----------------------------------------------------------------------
def partition(t, s, a, N, budget=float("inf")):
    """paci_partition: returns (cuts, max_time, max_overshoot); max_overshoot == 0
    exactly when every stage fits the budget."""
    t, s, a = (np.ascontiguousarray(x, np.float64) for x in (t, s, a))
    assert t.shape == s.shape == a.shape and t.ndim == 1
    cuts = np.zeros(max(N, 0) + 1, np.int32)
    mt, mo = ctypes.c_double(), ctypes.c_double()
    dp = ctypes.POINTER(ctypes.c_double)
    _check(lib.paci_partition(t.size, N, t.ctypes.data_as(dp), s.ctypes.data_as(dp), a.ctypes.data_as(dp),
                              float(budget), cuts.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                              ctypes.byref(mt), ctypes.byref(mo)), "paci_partition")
    return cuts, mt.value, mo.value


def schedule(M, K, delay, flush=False):
    """paci_schedule (asynchronous 1F1B) or, with ``flush``, paci_schedule_flush
    (synchronous 1F1B with a flush per window): returns (kinds, idx) int32
    arrays (0 = F, 1 = B, 2 = step)."""
    n = ctypes.c_int(0)
    cap = 2 * M + M // max(K, 1) + 1
    kinds = np.zeros(cap, np.int32)
    idx = np.zeros(cap, np.int32)
    name = "paci_schedule_flush" if flush else "paci_schedule"
    _check(getattr(lib, name)(M, K, delay, kinds.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                              idx.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), cap, ctypes.byref(n)), name)
    return kinds[:n.value].copy(), idx[:n.value].copy()


class Fsm:
    """The host-only protocol object (paci_fsm_*)."""

    def __init__(self, K, delay):
        self.h = ctypes.c_void_p()
        _check(lib.paci_fsm_create(K, delay, ctypes.byref(self.h)), "paci_fsm_create")

    def forward(self, mb):
        v = ctypes.c_int(-1)
        return lib.paci_fsm_forward(self.h, mb, ctypes.byref(v)), v.value

    def backward(self, mb):
        v = ctypes.c_int(-1)
        return lib.paci_fsm_backward(self.h, mb, ctypes.byref(v)), v.value

    def step(self):
        v = ctypes.c_int(-1)
        return lib.paci_fsm_step(self.h, ctypes.byref(v)), v.value

    def counters(self):
        c = PaciCounters()
        _check(lib.paci_fsm_counters(self.h, ctypes.byref(c)), "paci_fsm_counters")
        return {k: getattr(c, k) for k, _ in PaciCounters._fields_}

    def __del__(self):
        if getattr(self, "h", None) and lib is not None:
            lib.paci_fsm_destroy(self.h)
            self.h = None


def param_table(cfg):
    """paci_param_info_at for every tensor: list of dicts in canonical order."""
    s = shapes(cfg)
    n, tot = ctypes.c_int(0), ctypes.c_int64(0)
    _check(lib.paci_param_count(ctypes.byref(s), ctypes.byref(n), ctypes.byref(tot)), "paci_param_count")
    out = []
    for i in range(n.value):
        info = PaciParamInfo()
        _check(lib.paci_param_info_at(ctypes.byref(s), i, ctypes.byref(info)), "paci_param_info_at")
        out.append(dict(name=info.name.decode(), rows=info.rows, cols=info.cols, offset=info.offset,
                        numel=info.numel, decay=bool(info.decay)))
    return out


def arena_bytes(cfg, K=None, delay=None):
    s = shapes(cfg)
    b = ctypes.c_size_t(0)
    _check(lib.paci_stage_arena_bytes(ctypes.byref(s), cfg["K"] if K is None else K,
                                      cfg["delay"] if delay is None else delay, ctypes.byref(b)),
           "paci_stage_arena_bytes")
    return b.value


def kernel_families():
    return [lib.paci_kernel_family_name(i).decode() for i in range(lib.paci_kernel_family_count())]


# ---- the stage (device) --------------------------------------------------------------------
def _ptr(t):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


class Stage:
    """stage_init(shapes, K, delay) on the current torch device and stream."""

    def __init__(self, cfg, K=None, delay=None, device="cuda"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("the PACI stage needs a HIP device")
        self.torch = torch
        self.cfg = dict(cfg)
        self.K = cfg["K"] if K is None else K
        self.delay = cfg["delay"] if delay is None else delay
        self.s = shapes(cfg)
        nbytes = arena_bytes(cfg, self.K, self.delay)
        self.arena = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        base = self.arena.data_ptr()
        self.arena_ptr = (base + 255) // 256 * 256
        self.stream = torch.cuda.current_stream(self.arena.device)
        self.h = ctypes.c_void_p()
        r = lib.paci_stage_init(ctypes.byref(self.s), self.K, self.delay, ctypes.c_void_p(self.arena_ptr),
                                nbytes, ctypes.c_void_p(self.stream.cuda_stream), ctypes.byref(self.h))
        if r < 0:
            raise PaciError(r, "paci_stage_init", lib.paci_last_hip_error(None) if r == E_HIP else 0)
        self.n_params = sum(p["numel"] for p in param_table(cfg))
        self.act_dtype = torch.bfloat16 if cfg["dtype"] == "bf16" else torch.float32
        self.T = cfg["micro_batch"] * cfg["seq"]

    def close(self):
        if getattr(self, "h", None) and lib is not None:
            lib.paci_stage_destroy(self.h)
            self.h = None

    def __del__(self):
        self.close()

    # state transfer
    def load(self, what, values):
        """values: a float32 torch tensor on the device, or a numpy array on the host."""
        if isinstance(values, np.ndarray):
            a = np.ascontiguousarray(values, dtype=np.float32)
            _check(lib.paci_stage_load(self.h, what, ctypes.c_void_p(a.ctypes.data), a.size, 0), "paci_stage_load")
        else:
            assert values.dtype == self.torch.float32 and values.is_contiguous()
            _check(lib.paci_stage_load(self.h, what, _ptr(values), values.numel(), 1), "paci_stage_load")

    def load_params(self, params):
        self.load(PARAMS, inputs.flat_params(self.cfg, params))

    def read(self, what):
        out = np.empty(self.n_params, np.float32)
        _check(lib.paci_stage_read(self.h, what, ctypes.c_void_p(out.ctypes.data), out.size, 0), "paci_stage_read")
        return out

    # events of Alg. 1
    def forward(self, mb, inp, out, targets=None):
        v = ctypes.c_int(-1)
        _check(lib.paci_stage_forward(self.h, mb, _ptr(inp), _ptr(targets), _ptr(out), ctypes.byref(v)),
               "paci_stage_forward")
        return v.value

    def backward(self, mb, grad_out=None, grad_in=None):
        v = ctypes.c_int(-1)
        r = _check(lib.paci_stage_backward(self.h, mb, _ptr(grad_out), _ptr(grad_in), ctypes.byref(v)),
                   "paci_stage_backward")
        return v.value, r == STEP_DUE

    def backward_static(self, mb, grad_out=None, grad_in=None):
        """paci_stage_backward_static: the backward with its attention scratch in the
        library's static buffer (no allocation at call time)."""
        v = ctypes.c_int(-1)
        r = _check(lib.paci_stage_backward_static(self.h, mb, _ptr(grad_out), _ptr(grad_in), ctypes.byref(v)),
                   "paci_stage_backward_static")
        return v.value, r == STEP_DUE

    def step(self):
        v = ctypes.c_int(-1)
        _check(lib.paci_stage_step(self.h, ctypes.byref(v)), "paci_stage_step")
        return v.value

    def try_forward(self, mb, inp, out, targets=None):
        """Like forward but returns the raw status instead of raising."""
        v = ctypes.c_int(-1)
        return lib.paci_stage_forward(self.h, mb, _ptr(inp), _ptr(targets), _ptr(out), ctypes.byref(v))

    def try_backward(self, mb, grad_out=None, grad_in=None):
        v = ctypes.c_int(-1)
        return lib.paci_stage_backward(self.h, mb, _ptr(grad_out), _ptr(grad_in), ctypes.byref(v))

    def try_step(self):
        v = ctypes.c_int(-1)
        return lib.paci_stage_step(self.h, ctypes.byref(v))

    def run(self, M, in_all, grad_out_all=None, out_all=None, grad_in_all=None, targets_all=None):
        """paci_stage_run: replays the canonical order; returns stamps [M, 3] (t^F, t^B, Delta)."""
        stamps = np.zeros((M, 3), np.int32)
        _check(lib.paci_stage_run(self.h, M, _ptr(in_all), ctypes.cast(_ptr(targets_all), ctypes.POINTER(ctypes.c_int32)),
                                  _ptr(grad_out_all), _ptr(out_all), _ptr(grad_in_all),
                                  stamps.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))),
               "paci_stage_run")
        return stamps

    def run_events(self, kinds, idx, in_all, grad_out_all=None, out_all=None, grad_in_all=None, targets_all=None):
        """paci_stage_run_events: replays the (kinds, idx) list; returns stamps [M, 3]
        for micro-batch indices 0 .. max(idx)."""
        kinds = np.ascontiguousarray(kinds, np.int32)
        idx = np.ascontiguousarray(idx, np.int32)
        M = int(idx.max()) + 1 if idx.size else 0
        stamps = np.zeros((max(M, 1), 3), np.int32)
        i32 = ctypes.POINTER(ctypes.c_int32)
        _check(lib.paci_stage_run_events(self.h, kinds.size, kinds.ctypes.data_as(i32), idx.ctypes.data_as(i32),
                                         _ptr(in_all), ctypes.cast(_ptr(targets_all), i32), _ptr(grad_out_all),
                                         _ptr(out_all), _ptr(grad_in_all), stamps.ctypes.data_as(i32)),
               "paci_stage_run_events")
        return stamps[:M]

    def reset_counters(self):
        _check(lib.paci_stage_reset_counters(self.h), "paci_stage_reset_counters")

    def resume(self, version, next_mb, applied, skipped=0):
        """paci_stage_resume: continue a checkpoint of a drained stage."""
        _check(lib.paci_stage_resume(self.h, version, next_mb, applied, skipped), "paci_stage_resume")

    def updates(self):
        """(applied, skipped): updates the step applied and skipped (non-finite G)."""
        a, k = ctypes.c_int32(), ctypes.c_int32()
        _check(lib.paci_stage_updates(self.h, ctypes.byref(a), ctypes.byref(k)), "paci_stage_updates")
        return a.value, k.value

    def counters(self):
        c = PaciCounters()
        _check(lib.paci_stage_counters(self.h, ctypes.byref(c)), "paci_stage_counters")
        return {k: getattr(c, k) for k, _ in PaciCounters._fields_}

    def sync(self):
        _check(lib.paci_stage_sync(self.h), "paci_stage_sync")

    def set_timing(self, on):
        _check(lib.paci_stage_set_timing(self.h, 1 if on else 0), "paci_stage_set_timing")

    def kernel_times(self):
        out = {}
        for i, name in enumerate(kernel_families()):
            n, ms, w = ctypes.c_int64(0), ctypes.c_double(0), ctypes.c_double(0)
            _check(lib.paci_stage_kernel_times(self.h, i, ctypes.byref(n), ctypes.byref(ms), ctypes.byref(w)),
                   "paci_stage_kernel_times")
            out[name] = dict(launches=n.value, ms=ms.value, work=w.value)
        return out


# ---- attention operators (device) ------------------------------------------------------------
# Each runs on the tensors' device and its current torch stream. Matrices are
# [rows, columns] with contiguous rows (any row stride the C ABI admits, e.g. a
# column range of a fused projection); vectors are contiguous. They know nothing of
# autograd: results are written into the caller's tensors and carry no graph, also
# where an operand requires gradients; the *_backward calls give those. The checks are
# written for few Python operations: a small call costs more here than on the GPU.
_TORCH_DTYPES = {torch.bfloat16: BF16, torch.float32: FP32}
_F32, _I32, _F64 = torch.float32, torch.int32, torch.float64
def _stream_handle(dev):
    return torch.cuda.current_stream(dev).cuda_stream


# the current stream's handle without the Stream object that torch.cuda.current_stream makes around it (1 us of a 9 us
# call); a torch that lacks this private name has the other way, and one without devices this module's host calls
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream_handle)
_INT_MAX = 2 ** 31 - 1   # sizes are int32 in the C structures, which would keep the low bits of larger ones


def _int32(what, *sizes):
    """ctypes passes the low 32 bits of an int: others than these would make the C call fill more than the array holds."""
    if max(sizes) > _INT_MAX or min(sizes) < -_INT_MAX:
        _refuse(f"{what}: {sizes}")


def rope_freqs(theta, rope_dims):
    """paci_rope_freqs: theta^(-2 i / rope_dims), i < rope_dims / 2, as a float64 array."""
    _int32("rope_freqs", rope_dims)
    f = np.zeros(max(rope_dims // 2, 1), np.float64)
    _check(lib.paci_rope_freqs(float(theta), rope_dims, f.ctypes.data_as(ctypes.POINTER(ctypes.c_double))),
           "paci_rope_freqs")
    return f


def rel_bounds(n_buckets, max_distance):
    """paci_rel_bounds: the first distance of every bucket, as an int32 array."""
    _int32("rel_bounds", n_buckets, max_distance)
    b = np.zeros(max(n_buckets, 1), np.int32)
    _check(lib.paci_rel_bounds(n_buckets, max_distance, b.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))),
           "paci_rel_bounds")
    return b


def _refuse(what, code=E_INVAL):
    raise PaciError(code, what)


def _mat(t, shape, dtype, dev, what):
    """Address of a matrix of this shape, dtype and device index (its stride is the caller's to pass)."""
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev or (t.stride(1) != 1 and shape[1] > 1):
        _refuse(f"{what}: {tuple(shape)} {dtype} on device {dev} with contiguous rows expected")
    return t.data_ptr()


def _vec(t, shape, dtype, dev, what):
    """Address of a contiguous tensor of this shape (None: null)."""
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev or not t.is_contiguous():
        _refuse(f"{what}: contiguous {tuple(shape)} {dtype} on device {dev} expected")
    return t.data_ptr()


def _operand(x, what):
    """The PACI dtype of an operator's first tensor, a matrix on a device."""
    if not x.is_cuda or x.dim() != 2:
        _refuse(f"{what}: a device matrix expected")
    dt = _TORCH_DTYPES.get(x.dtype)
    return _refuse(what, E_UNSUPPORTED) if dt is None else dt


def _launch(fn, dev, *args):
    """Calls a C operator on a device's current stream."""
    st = _raw_stream(dev)
    if dev == torch.cuda.current_device():
        r = fn(*args, st)
    else:
        with torch.cuda.device(dev):
            r = fn(*args, st)
    if r < 0:
        raise PaciError(r, fn.__name__, lib.paci_last_hip_error(None) if r == E_HIP else 0)


def _bytes(fn, shapes):
    n = ctypes.c_size_t(0)
    _check(fn(ctypes.byref(shapes), ctypes.byref(n)), fn.__name__)
    return n.value


def _workspace(ws, fn, shapes, like):
    """The caller's workspace (any contiguous tensor on the device), or one of the needed
    size from torch's allocator on the current stream: (tensor, bytes)."""
    if ws is None:
        n = _bytes(fn, shapes)
        return like.new_empty((n + 3) // 4, dtype=_F32), n
    if ws.device != like.device or not ws.is_contiguous():
        _refuse(f"{fn.__name__}: a contiguous workspace on {like.device} expected")
    return ws, ws.numel() * ws.element_size()


def _qk_shapes(x, q_heads, k_heads, seq, norm, eps, freq, pairs):
    dt = _operand(x, "qk_norm_rope x")
    tokens, cols = x.shape
    heads = q_heads + k_heads
    if heads < 1 or min(q_heads, k_heads, seq) < 0 or cols % heads or pairs not in ROPE_PAIRS or max(tokens, cols, seq) > _INT_MAX:
        _refuse(f"qk_norm_rope: {cols} columns of {heads} heads, pairs {pairs!r}")
    return PaciQkShapes(dt, tokens, seq, q_heads, k_heads, cols // heads, norm, eps, 0 if freq is None else 2 * freq.numel(),
                        ROPE_PAIRS[pairs])


def qk_norm_rope(x, y, q_heads, k_heads, seq=1, q_gain=None, k_gain=None, eps=1e-5, freq=None, pairs="half", pos=None):
    """paci_qk_norm_rope_forward: y = the normalised and rotated heads of x
    [tokens, (q_heads + k_heads) * head_dim]. Gains ([head_dim] float32): norm, None:
    no norm. freq ([rope_dims / 2] float64): rotation, None: none. pos ([tokens] int32)
    or, without it, row % seq. y may be x. y carries no autograd graph:
    qk_norm_rope_backward gives the gradients."""
    s = _qk_shapes(x, q_heads, k_heads, seq, q_gain is not None or k_gain is not None, eps, freq, pairs)
    dh, shape, dt, dev = (s.head_dim,), x.shape, x.dtype, x.get_device()
    _launch(lib.paci_qk_norm_rope_forward, dev, ctypes.byref(s), _mat(x, shape, dt, dev, "qk_norm_rope x"), x.stride(0),
            _vec(q_gain, dh, _F32, dev, "q_gain"), _vec(k_gain, dh, _F32, dev, "k_gain"),
            _vec(pos, (s.tokens,), _I32, dev, "pos"), _vec(freq, (s.rope_dims // 2,), _F64, dev, "freq"),
            _mat(y, shape, dt, dev, "qk_norm_rope y"), y.stride(0))
    return y


def qk_norm_rope_workspace(x, q_heads, k_heads, seq=1, norm=True, freq=None, pairs="half"):
    """Bytes of workspace that qk_norm_rope_backward needs for these operands."""
    return _bytes(lib.paci_qk_norm_rope_workspace, _qk_shapes(x, q_heads, k_heads, seq, norm, 0.0, freq, pairs))


def qk_norm_rope_backward(x, dy, dx, q_heads, k_heads, seq=1, q_gain=None, k_gain=None, eps=1e-5, freq=None, pairs="half",
                          pos=None, g_q_gain=None, g_k_gain=None, g_bias=None, ws=None):
    """paci_qk_norm_rope_backward: dx from dy and the forward's arguments; g_q_gain, g_k_gain
    and g_bias (float32, optional) are added to. dx may be dy. ws: a workspace of
    qk_norm_rope_workspace bytes (None: from torch's allocator)."""
    s = _qk_shapes(x, q_heads, k_heads, seq, q_gain is not None or k_gain is not None, eps, freq, pairs)
    dh, shape, dt, dev = (s.head_dim,), x.shape, x.dtype, x.get_device()
    ws, n = _workspace(ws, lib.paci_qk_norm_rope_workspace, s, x)
    _launch(lib.paci_qk_norm_rope_backward, dev, ctypes.byref(s), _mat(x, shape, dt, dev, "qk_norm_rope x"), x.stride(0),
            _mat(dy, shape, dt, dev, "qk_norm_rope dy"), dy.stride(0), _vec(q_gain, dh, _F32, dev, "q_gain"),
            _vec(k_gain, dh, _F32, dev, "k_gain"), _vec(pos, (s.tokens,), _I32, dev, "pos"),
            _vec(freq, (s.rope_dims // 2,), _F64, dev, "freq"), _mat(dx, shape, dt, dev, "qk_norm_rope dx"), dx.stride(0),
            _vec(g_q_gain, dh, _F32, dev, "g_q_gain"), _vec(g_k_gain, dh, _F32, dev, "g_k_gain"),
            _vec(g_bias, shape[1:], _F32, dev, "g_bias"), ws.data_ptr(), n)
    return dx


def _attn_shapes(q, batch, n_heads, table, max_distance):
    dt = _operand(q, "attention q")
    T, d = q.shape
    if (min(batch, max_distance) < 0 or n_heads < 1 or d % n_heads or (T % batch if batch else T) or
            max(T, d, batch, max_distance) > _INT_MAX):
        _refuse(f"attention: {(T, d)} is not {batch} sequences of {n_heads} heads")
    return PaciAttnShapes(dt, batch, T // batch if batch else 0, n_heads, d // n_heads, 0 if table is None else table.shape[0],
                          max_distance)


def _attn_inputs(s, q, k, v, table, bounds):
    shape, dt, dev = q.shape, q.dtype, q.get_device()
    return (_mat(q, shape, dt, dev, "attention q"), q.stride(0), _mat(k, shape, dt, dev, "attention k"), k.stride(0),
            _mat(v, shape, dt, dev, "attention v"), v.stride(0), _vec(table, (s.n_buckets, s.n_heads), _F32, dev, "table"),
            _vec(bounds, (s.n_buckets,), _I32, dev, "bounds"))


def attention(q, k, v, o, lse2, batch, n_heads, table=None, bounds=None, max_distance=0):
    """paci_attn_forward: causal attention of q, k and v [batch * seq, n_heads * head_dim]
    into o (contiguous) and lse2 [batch * n_heads, seq] float32, with the relative position
    bias table [n_buckets, n_heads] float32 and its bounds [n_buckets] int32 (rel_bounds
    gives the usual ones), or without. o and lse2 carry no autograd graph:
    attention_backward gives the gradients."""
    s = _attn_shapes(q, batch, n_heads, table, max_distance)
    dev = q.get_device()
    _launch(lib.paci_attn_forward, dev, ctypes.byref(s), *_attn_inputs(s, q, k, v, table, bounds),
            _vec(o, q.shape, q.dtype, dev, "o"), _vec(lse2, (batch * n_heads, s.seq), _F32, dev, "lse2"))
    return o


def attention_workspace(q, batch, n_heads, table=None, max_distance=0):
    """Bytes of workspace that attention_backward needs for these operands."""
    return _bytes(lib.paci_attn_workspace, _attn_shapes(q, batch, n_heads, table, max_distance))


def attention_backward(q, k, v, o, lse2, do, dq, dk, dv, batch, n_heads, table=None, bounds=None, max_distance=0,
                       g_table=None, ws=None):
    """paci_attn_backward: dq, dk and dv from do (contiguous like o) and the forward's operands,
    o and lse2; g_table (float32, optional) is added to. ws: a workspace of
    attention_workspace bytes (None: from torch's allocator)."""
    s = _attn_shapes(q, batch, n_heads, table, max_distance)
    shape, dt, dev = q.shape, q.dtype, q.get_device()
    ws, n = _workspace(ws, lib.paci_attn_workspace, s, q)
    _launch(lib.paci_attn_backward, dev, ctypes.byref(s), *_attn_inputs(s, q, k, v, table, bounds),
            _vec(o, shape, dt, dev, "o"), _vec(lse2, (batch * n_heads, s.seq), _F32, dev, "lse2"),
            _vec(do, shape, dt, dev, "do"), _mat(dq, shape, dt, dev, "dq"), dq.stride(0), _mat(dk, shape, dt, dev, "dk"),
            dk.stride(0), _mat(dv, shape, dt, dev, "dv"), dv.stride(0),
            _vec(g_table, (s.n_buckets, n_heads), _F32, dev, "g_table"), ws.data_ptr(), n)
    return dq, dk, dv


# The C ABI's names for the three events and the constructor.
def stage_init(cfg, K=None, delay=None):
    return Stage(cfg, K, delay)


def stage_forward(stage, mb, inp, out, targets=None):
    return stage.forward(mb, inp, out, targets)


def stage_backward(stage, mb, grad_out=None, grad_in=None):
    return stage.backward(mb, grad_out, grad_in)


def stage_step(stage):
    return stage.step()
