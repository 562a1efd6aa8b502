"""ctypes binding of ``libtre.so`` (the C ABI declared in ``include/tre.h``); lists
of tensors are read by ``_tensors.so``.

Argument marshalling only: torch supplies device memory and the stream, and
every step of the path runs in the library's HIP kernels.  There is no CPU
fallback; a missing library raises at load time.
"""
from __future__ import annotations

import ctypes
import os
from array import array
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# TRE_HOST_SANITIZED=1 loads the host-only AddressSanitizer / UBSan build
# (no device code) for the CPU tests; see build.build_host_sanitized
SANITIZED = os.environ.get("TRE_HOST_SANITIZED") == "1"
LIB_PATH = os.path.join(_HERE, "libtre_host_san.so" if SANITIZED else "libtre.so")

STATUS = {
    0: "TRE_OK", 1: "TRE_E_ARG", 2: "TRE_E_PARSE", 3: "TRE_E_SPLIT", 4: "TRE_E_SHAPE", 5: "TRE_E_DTYPE",
    6: "TRE_E_UNSORTED", 7: "TRE_E_DUPKEY", 8: "TRE_E_KEYRANGE", 9: "TRE_E_CAPACITY", 10: "TRE_E_WORKSPACE",
    11: "TRE_E_DEVICE", 12: "TRE_E_STATE",
}
STATUS_CODE = {v: k for k, v in STATUS.items()}
DTYPE = {"f32": 0, "bf16": 1, "mxfp4": 2}

# every symbol include/tre.h declares
EXPORTS = [
    "tre_plan", "tre_plan_get_info", "tre_plan_destroy", "tre_workspace_bytes", "tre_workspace_max_pairs",
    "tre_join", "tre_join_keys", "tre_contract", "tre_execute", "tre_timing_read", "tre_cast_f32_bf16", "tre_scale_f32",
    "tre_stack_workspace_bytes", "tre_stack_rows",
    "tre_tiles_from_entries", "tre_status_str", "tre_last_error", "tre_version",
    "tre_repartition_workspace_bytes", "tre_repartition", "tre_execute3_workspace_bytes", "tre_execute3",
    "tre_noalloc_scratch_bytes", "tre_execute_noalloc", "tre_output_bounds", "tre_execute_async",
    "tre_tile_bytes", "tre_mx_quantize", "tre_mx_dequantize", "tre_lookup", "tre_lookup_grad_workspace_bytes",
    "tre_lookup_grad", "tre_log_probs_workspace_bytes", "tre_log_probs", "tre_log_probs_grad",
    "tre_grad_norm_workspace_bytes", "tre_grad_norm", "tre_adamw_state_bytes", "tre_adamw", "tre_adamw_moments",
]


class TreError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        self.status = STATUS.get(code, str(code))
        super().__init__(f"{where}: {self.status}" + (f" ({detail})" if detail else ""))


class Options(ctypes.Structure):
    _fields_ = [("validate_keys", ctypes.c_int32), ("max_pairs_per_unit", ctypes.c_int32),
                ("u_ranges", ctypes.c_int32), ("pace_windows", ctypes.c_int32), ("w_bf16", ctypes.c_int32),
                ("small_join", ctypes.c_int32), ("reserved", ctypes.c_int32 * 2)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("key_arity", ctypes.c_int32 * 3), ("tile_elems", ctypes.c_int64 * 3), ("n_join", ctypes.c_int32),
                ("kernel_class", ctypes.c_int32), ("batch", ctypes.c_int64), ("m", ctypes.c_int64),
                ("n", ctypes.c_int64), ("k", ctypes.c_int64), ("flops_per_pair", ctypes.c_int64),
                ("key_labels", (ctypes.c_char * 27) * 3), ("roles", ctypes.c_char * 27),
                ("group_needs_sort", ctypes.c_int32), ("v_needs_sort", ctypes.c_int32), ("w_dtype", ctypes.c_int32),
                ("join_outer", ctypes.c_int32)]


class JoinResult(ctypes.Structure):
    _fields_ = [("n_u", ctypes.c_int64), ("n_v", ctypes.c_int64), ("n_pairs", ctypes.c_int64), ("n_w", ctypes.c_int64),
                ("internal", ctypes.c_uint64 * 16)]


class AdamwOptions(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("grad_scale", ctypes.c_double), ("step", ctypes.c_int64),
                ("lr_dev", ctypes.c_void_p), ("step_dev", ctypes.c_void_p), ("grad_scale_dev", ctypes.c_void_p),
                ("seed", ctypes.c_uint64), ("stochastic", ctypes.c_int32), ("bits", ctypes.c_int32),
                ("reserved", ctypes.c_int32 * 2)]


class Timing(ctypes.Structure):
    _fields_ = [("join_ms", ctypes.c_float), ("units_ms", ctypes.c_float), ("contract_ms", ctypes.c_float),
                ("reduce_ms", ctypes.c_float), ("total_ms", ctypes.c_float), ("deferred", ctypes.c_int32),
                ("pending", ctypes.c_int32), ("contract_block", ctypes.c_int32), ("n_units", ctypes.c_int64), ("n_split_segments", ctypes.c_int64),
                ("n_partials", ctypes.c_int64), ("events", ctypes.c_void_p * 4), ("contract_path", ctypes.c_int32),
                ("join_path", ctypes.c_int32)]

    PATHS = {0: "gemm", 1: "vec", 2: "gemm128", 3: "gemm128_paced", 4: "gemm128_u_ranges", 5: "mx"}
    JOIN_PATHS = {0: "u_driven", 1: "v_driven", 2: "v_driven_one_match", 3: "v_driven_dense", 4: "keyed_by_u",
                  5: "one_workgroup", 6: "u_driven_dense"}

    def read(self):
        """Wait for deferred events and fill the millisecond fields."""
        _check(lib().tre_timing_read(ctypes.byref(self)), "tre_timing_read")
        return self

    def as_dict(self):
        d = {k: getattr(self, k) for k, _ in self._fields_ if k not in ("events", "deferred", "pending")}
        d["contract_path"] = self.PATHS.get(self.contract_path, self.contract_path)
        d["join_path"] = self.JOIN_PATHS.get(self.join_path, self.join_path)
        d["contract_block"] = (self.contract_block >> 16, self.contract_block & 0xffff)
        return d


_lib = None


def lib():
    """Load libtre.so; raises if it has not been built (no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2603_08957_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
        L.tre_plan.argtypes = [ctypes.c_char_p, ctypes.c_char_p, P, P, ctypes.c_int, P, P]
        L.tre_plan_get_info.argtypes = [P, P]
        L.tre_plan_destroy.argtypes = [P]
        L.tre_plan_destroy.restype = None
        L.tre_workspace_bytes.argtypes = [P, i64, i64, i64]
        L.tre_workspace_bytes.restype = sz
        L.tre_workspace_max_pairs.argtypes = [P, i64, i64, sz]
        L.tre_workspace_max_pairs.restype = i64
        L.tre_join.argtypes = [P, P, i64, P, i64, P, sz, P, P, P]
        L.tre_join_keys.argtypes = [P, P, P, i64, P]
        L.tre_contract.argtypes = [P, P, P, P, P, i64, P, P, i64, P, P]
        L.tre_execute.argtypes = [P, P, i64, P, P, i64, P, P, P, i64, P, P, i64, P, P, sz, P, P]
        L.tre_output_bounds.argtypes = [P, i64, i64, sz, P, P, P]
        L.tre_execute_async.argtypes = [P, P, i64, P, P, P, i64, P, P, P, i64, P, i64, P, P, sz, P, P]
        L.tre_timing_read.argtypes = [P]
        L.tre_cast_f32_bf16.argtypes = [P, P, i64, P]
        L.tre_scale_f32.argtypes = [P, P, i64, ctypes.c_float, P]
        L.tre_stack_workspace_bytes.argtypes = [i64]
        L.tre_stack_workspace_bytes.restype = sz
        L.tre_stack_rows.argtypes = [P, i64, P, i64, i32, i32, P, P, i64, P, P, sz, P]
        L.tre_tiles_from_entries.argtypes = [P, P, P, i64, i32, P, i64, i64, P]
        cs = ctypes.c_char_p
        L.tre_repartition_workspace_bytes.argtypes = [cs, cs, cs, P, P, P, i64]
        L.tre_repartition_workspace_bytes.restype = sz
        L.tre_repartition.argtypes = [cs, cs, cs, P, P, P, i32, P, i64, P, P, P, i64, P, P, sz, P]
        L.tre_execute3_workspace_bytes.argtypes = [cs, cs, P, P, i64]
        L.tre_execute3_workspace_bytes.restype = sz
        L.tre_execute3.argtypes = [cs, cs, P, P, ctypes.c_int, P, i64, P, P, i64, P, P, i64, P, P, P, i64, P, P, P, sz,
                                   P, P]
        L.tre_noalloc_scratch_bytes.argtypes = []
        L.tre_noalloc_scratch_bytes.restype = sz
        L.tre_execute_noalloc.argtypes = [P, P, i64, P, P, i64, P, P, P, i64, P, P, i64, P, P]
        L.tre_tile_bytes.argtypes = [P, i32]
        L.tre_tile_bytes.restype = i64
        L.tre_mx_quantize.argtypes = [P, i32, P, i32, i64, P, P]
        L.tre_mx_dequantize.argtypes = [P, i32, P, i64, P, i32, P]
        L.tre_lookup.argtypes = [P, i32, i64, i64, i64, P, i32, i64, ctypes.c_float, P, i32, P, P]
        L.tre_lookup_grad_workspace_bytes.argtypes = [i64, i64, i64]
        L.tre_lookup_grad_workspace_bytes.restype = sz
        L.tre_lookup_grad.argtypes = [P, i32, P, i32, i64, ctypes.c_float, P, i32, i64, i64, i32, P, P, sz, P]
        f32 = ctypes.c_float
        L.tre_log_probs_workspace_bytes.argtypes = [i64, i64, i64, i32, i32]
        L.tre_log_probs_workspace_bytes.restype = sz
        L.tre_log_probs.argtypes = [P, i32, i64, i64, i64, i64, i64, P, i32, f32, P, P, P, P, i32, P, P, P, P, sz, P]
        L.tre_log_probs_grad.argtypes = [P, i32, i64, i64, i64, i64, i64, P, P, i32, f32, P, P, P, P, P, i32, i64, i64, P, P]
        L.tre_grad_norm_workspace_bytes.argtypes = [i32, P]
        L.tre_grad_norm_workspace_bytes.restype = sz
        L.tre_grad_norm.argtypes = [i32, P, P, P, f32, P, P, sz, P]
        L.tre_adamw_state_bytes.argtypes = [i32, P, i32]
        L.tre_adamw_state_bytes.restype = sz
        L.tre_adamw.argtypes = [i32, P, P, P, P, P, P, P, P]
        L.tre_adamw_moments.argtypes = [P, i64, P, P, i32, P]
        L.tre_status_str.restype = ctypes.c_char_p
        L.tre_last_error.restype = ctypes.c_char_p
        L.tre_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(rc: int, where: str):
    if rc != 0:
        raise TreError(rc, where, lib().tre_last_error().decode())


def _ptr(t):
    """Device pointer of a torch tensor (or None)."""
    if t is None:
        return None
    return ctypes.c_void_p(t.data_ptr())


def _at(t):
    """The same as a number, which costs a small call less."""
    return None if t is None else t.data_ptr()


def _stream(stream=None, device=None):
    """The hipStream_t of a torch stream, or of the (current) device's current
    one, whose handle torch gives without making a stream object (3 us less)."""
    import torch

    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)
    return ctypes.c_void_p(raw(torch.cuda.current_device() if device is None else device.index))


def _buffer(stream, device, make, result=True):
    """The tensor that ``make()`` allocates, out of the memory of the stream that
    will use it: a block that the current stream has just given back may still
    be in use by what is queued there, which a caller's stream does not wait
    for.  A result is the current stream's too: its memory is not given out
    again before what that stream does with it is done."""
    import torch

    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        t = make()
    if result:
        t.record_stream(torch.cuda.current_stream(device))
    return t


class Plan:
    """A parsed, classified binary EinSum (host object, see tre_plan)."""

    def __init__(self, einsum: str, upper: str, extents: dict, tiles: dict, dtype: str = "f32",
                 validate: bool = True, max_pairs_per_unit: int = 0, u_ranges: int = 0, pace_windows: int = 0,
                 w_bf16: bool = False, small_join: int = 0):
        L = lib()
        ext = np.zeros(26, dtype=np.int64)
        til = np.ones(26, dtype=np.int32)
        for k, v in extents.items():
            ext[ord(k) - 97] = v
        for k, v in (tiles or {}).items():
            til[ord(k) - 97] = v
        opt = Options(int(validate), int(max_pairs_per_unit), int(u_ranges), int(pace_windows), int(w_bf16),
                      int(small_join))
        self.w_bf16 = bool(w_bf16)
        h = ctypes.c_void_p(0)
        rc = L.tre_plan(einsum.encode(), upper.encode(), ext.ctypes.data_as(ctypes.c_void_p),
                        til.ctypes.data_as(ctypes.c_void_p), DTYPE[dtype], ctypes.byref(opt), ctypes.byref(h))
        _check(rc, "tre_plan")
        self._h = h
        self.einsum, self.upper, self.dtype = einsum, upper, dtype
        info = PlanInfo()
        _check(L.tre_plan_get_info(h, ctypes.byref(info)), "tre_plan_get_info")
        self.key_arity = list(info.key_arity)
        self.tile_elems = list(info.tile_elems)
        self.n_join = info.n_join
        self.kernel_class = {0: "gemm", 1: "vec", 2: "gemm128", 3: "mx"}[info.kernel_class]
        self.bmnk = (info.batch, info.m, info.n, info.k)
        self.flops_per_pair = info.flops_per_pair
        self.key_labels = [bytes(info.key_labels[o]).split(b"\0")[0].decode() for o in range(3)]
        self.roles = bytes(info.roles).split(b"\0")[0].decode()
        self.group_needs_sort = bool(info.group_needs_sort)
        self.v_needs_sort = bool(info.v_needs_sort)
        self.w_dtype = {0: "f32", 1: "bf16"}[info.w_dtype]
        self.join_outer = "v" if info.join_outer else "u"
        # whether U's and V's tuples are rows of a table: W keeps one of its labels, and no other is promoted
        ins, w = einsum.replace(" ", "").split("->")
        kept = [[c for c in lab if c in w] for lab in ins.split(",")]
        self.token_keyed = [len(k) == 1 and self.key_labels[o] in ("", k[0]) for o, k in enumerate(kept)]
        # bytes of one tile of U, V and W as the calls take it
        self.tile_bytes = [int(L.tre_tile_bytes(h, o)) for o in range(3)]

    @classmethod
    def from_spec(cls, spec: dict, **kw):
        return cls(spec["einsum"], spec["upper"], spec["extents"], spec["tiles"], spec["dtype"], **kw)

    @property
    def handle(self):
        return self._h

    def workspace_bytes(self, n_u: int, n_v: int, max_pairs: int) -> int:
        return int(lib().tre_workspace_bytes(self._h, n_u, n_v, max_pairs))

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _lib is not None:
            _lib.tre_plan_destroy(h)
            self._h = None


def alloc_workspace(nbytes: int, device="cuda"):
    import torch

    ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    return ws


def _mx_operands(plan: Plan, u_tiles, v_tiles):
    """4-bit tiles come as uint8 rows of the plan's tile size, on the GPU that the
    call runs on (the current one): anything else is an array that was not
    quantised for this plan, or not for here."""
    import torch

    if plan.dtype != "mxfp4":
        return
    for o, t in ((0, u_tiles), (1, v_tiles)):
        if t is None:
            continue
        if t.dtype != torch.uint8 or t.dim() != 2 or t.shape[1] != plan.tile_bytes[o] or not t.is_contiguous():
            raise TreError(STATUS_CODE["TRE_E_SHAPE"], "tre.contract",
                           f"operand {'uv'[o]} of an mxfp4 plan: contiguous uint8 [n, {plan.tile_bytes[o]}] wanted, "
                           f"got {t.dtype} {tuple(t.shape)}")
        if not t.is_cuda or t.device.index != torch.cuda.current_device():
            raise TreError(STATUS_CODE["TRE_E_ARG"], "tre.contract",
                           f"operand {'uv'[o]} of an mxfp4 plan: on {t.device}, wanted on the current GPU")


def join(plan: Plan, u_keys, n_u: int, v_keys, n_v: int, ws, stream=None, timing: Timing | None = None) -> JoinResult:
    jr = JoinResult()
    rc = lib().tre_join(plan.handle, _ptr(u_keys), n_u, _ptr(v_keys), n_v, _ptr(ws), ws.numel(), _stream(stream),
                        ctypes.byref(jr), ctypes.byref(timing) if timing is not None else None)
    if rc != 0:
        err = TreError(rc, "tre_join", lib().tre_last_error().decode())
        err.join_result = jr
        raise err
    return jr


def contract(plan: Plan, jr: JoinResult, u_tiles, v_tiles, w_keys, w_tiles, pairs_out=None, stream=None,
             timing: Timing | None = None):
    _mx_operands(plan, u_tiles, v_tiles)
    w_cap = w_tiles.shape[0] if w_tiles is not None else 0
    pair_cap = pairs_out.shape[0] if pairs_out is not None else 0
    rc = lib().tre_contract(plan.handle, ctypes.byref(jr), _ptr(u_tiles), _ptr(v_tiles), _ptr(w_keys), w_cap,
                            _ptr(w_tiles), _ptr(pairs_out), pair_cap, _stream(stream),
                            ctypes.byref(timing) if timing is not None else None)
    _check(rc, "tre_contract")


def join_keys(plan: Plan, jr: JoinResult, w_keys, stream=None):
    """Write the join's output keys (tre_join_keys) into w_keys [>= n_w, r_W]."""
    w_cap = w_keys.shape[0] if w_keys is not None else 0
    _check(lib().tre_join_keys(plan.handle, ctypes.byref(jr), _ptr(w_keys), w_cap, _stream(stream)),
           "tre_join_keys")


def execute(plan: Plan, u_keys, u_tiles, v_keys, v_tiles, w_keys, w_tiles, ws, pairs_out=None, stream=None,
            timing: Timing | None = None):
    """tre_execute into caller-owned outputs and workspace (their row counts
    are the capacities): the join and the contraction in one call.  Returns
    (n_w, n_pairs); a TreError carries them when a capacity is short."""
    _mx_operands(plan, u_tiles, v_tiles)
    n_u, n_v = int(u_tiles.shape[0]), int(v_tiles.shape[0])
    n_w, n_p = ctypes.c_int64(0), ctypes.c_int64(0)
    rc = lib().tre_execute(plan.handle, _ptr(u_keys), n_u, _ptr(u_tiles), _ptr(v_keys), n_v, _ptr(v_tiles),
                           _ptr(w_keys), _ptr(w_tiles), int(w_tiles.shape[0]) if w_tiles is not None else 0,
                           ctypes.byref(n_w), _ptr(pairs_out), int(pairs_out.shape[0]) if pairs_out is not None else 0,
                           ctypes.byref(n_p), _ptr(ws), ws.numel(), _stream(stream),
                           ctypes.byref(timing) if timing is not None else None)
    if rc != 0:
        err = TreError(rc, "tre_execute", lib().tre_last_error().decode())
        err.n_w, err.n_pairs = int(n_w.value), int(n_p.value)
        raise err
    return int(n_w.value), int(n_p.value)


def output_bounds(plan: Plan, n_u: int, n_v: int, ws_bytes: int):
    """tre_output_bounds: (pair bound, key bound, whether tre_execute_async
    runs without a read-back for these sizes)."""
    pb, kb, ok = ctypes.c_int64(0), ctypes.c_int64(0), ctypes.c_int32(0)
    _check(lib().tre_output_bounds(plan.handle, int(n_u), int(n_v), int(ws_bytes), ctypes.byref(pb), ctypes.byref(kb),
                                   ctypes.byref(ok)), "tre_output_bounds")
    return int(pb.value), int(kb.value), bool(ok.value)


def execute_async(plan: Plan, u_keys, u_tiles, v_keys, v_tiles, w_keys, w_tiles, ws, counts, pairs_out=None,
                  n_u=None, n_u_dev=None, stream=None, timing: Timing | None = None):
    """tre_execute_async: join and contraction enqueued with no wait; the
    counts ([pairs, keys, status, 0]) land in ``counts`` (device int64 [4]).
    ``n_u`` defaults to u_tiles' rows; ``n_u_dev`` (a device int64 tensor)
    holds U's actual count when n_u is only a bound."""
    _mx_operands(plan, u_tiles, v_tiles)
    n_u = int(u_tiles.shape[0]) if n_u is None else int(n_u)
    n_v = int(v_tiles.shape[0])
    rc = lib().tre_execute_async(plan.handle, _ptr(u_keys), n_u, _ptr(n_u_dev), _ptr(u_tiles), _ptr(v_keys), n_v,
                                 _ptr(v_tiles), _ptr(w_keys), _ptr(w_tiles),
                                 int(w_tiles.shape[0]) if w_tiles is not None else 0, _ptr(pairs_out),
                                 int(pairs_out.shape[0]) if pairs_out is not None else 0, _ptr(counts), _ptr(ws),
                                 ws.numel(), _stream(stream), ctypes.byref(timing) if timing is not None else None)
    _check(rc, "tre_execute_async")


@dataclass
class Output:
    w_keys: object      # torch int32 [n_w, r_W]
    w_tiles: object     # torch float32 [n_w, tile_elems(W)]
    pairs: object       # torch int32 [n_pairs, 2] or None
    n_pairs: int
    n_w: int
    timing: dict | None
    ws: object


def einsum(plan: Plan, u_keys, u_tiles, v_keys, v_tiles, want_pairs: bool = False, ws=None, stream=None,
           timing: bool = False, pair_hint: int | None = None) -> Output:
    """Join + contract with output buffers allocated by torch.  The workspace
    is grown and the join repeated once if the pair list does not fit."""
    import torch

    _mx_operands(plan, u_tiles, v_tiles)
    n_u, n_v = int(u_tiles.shape[0]), int(v_tiles.shape[0])
    dev = u_tiles.device
    if ws is None:
        hint = pair_hint if pair_hint is not None else max(n_u, n_v, 1) * 2
        ws = _buffer(stream, dev, lambda: alloc_workspace(plan.workspace_bytes(n_u, n_v, hint), dev))
    tm = Timing() if timing else None
    try:
        jr = join(plan, u_keys, n_u, v_keys, n_v, ws, stream, tm)
    except TreError as e:
        if e.code != 10 or e.join_result.n_pairs <= 0:
            raise
        need = int(e.join_result.n_pairs)
        ws = _buffer(stream, dev, lambda: alloc_workspace(plan.workspace_bytes(n_u, n_v, need), dev))
        jr = join(plan, u_keys, n_u, v_keys, n_v, ws, stream, tm)
    n_w, n_p = int(jr.n_w), int(jr.n_pairs)
    rw = plan.key_arity[2]
    w_keys = _buffer(stream, dev, lambda: torch.empty((n_w, rw), dtype=torch.int32, device=dev))
    w_tiles = _buffer(stream, dev, lambda: torch.empty((n_w, plan.tile_elems[2]),
                                                       dtype=torch.bfloat16 if plan.w_bf16 else torch.float32, device=dev))
    pairs = _buffer(stream, dev, lambda: torch.empty((n_p, 2), dtype=torch.int32, device=dev)) if want_pairs else None
    contract(plan, jr, u_tiles, v_tiles, w_keys if rw > 0 else None, w_tiles, pairs, stream, tm)
    return Output(w_keys, w_tiles, pairs, n_p, n_w, tm.as_dict() if tm is not None else None, ws)


def execute_noalloc(plan: Plan, u_keys, u_tiles, v_keys, v_tiles, w_keys, w_tiles, pairs_out=None, stream=None):
    """tre_execute_noalloc: join + contract with the library's static device
    scratch as workspace; every output buffer is the caller's (their row
    counts are the capacities).  Returns (n_w, n_pairs)."""
    _mx_operands(plan, u_tiles, v_tiles)
    n_u, n_v = int(u_tiles.shape[0]), int(v_tiles.shape[0])
    n_w, n_p = ctypes.c_int64(0), ctypes.c_int64(0)
    rc = lib().tre_execute_noalloc(plan.handle, _ptr(u_keys), n_u, _ptr(u_tiles), _ptr(v_keys), n_v, _ptr(v_tiles),
                                   _ptr(w_keys), _ptr(w_tiles), int(w_tiles.shape[0]), ctypes.byref(n_w),
                                   _ptr(pairs_out), int(pairs_out.shape[0]) if pairs_out is not None else 0,
                                   ctypes.byref(n_p), _stream(stream))
    if rc != 0:
        err = TreError(rc, "tre_execute_noalloc", lib().tre_last_error().decode())
        err.n_w, err.n_pairs = int(n_w.value), int(n_p.value)
        raise err
    return int(n_w.value), int(n_p.value)


def noalloc_scratch_bytes() -> int:
    return int(lib().tre_noalloc_scratch_bytes())


# ------------------------------------------------ 4-bit tiles, rows by token

def _value_type(t, where, what):
    """0 / 1 for fp32 / bf16, of a tensor or a type."""
    import torch

    dt = getattr(t, "dtype", t)
    if dt == torch.float32:
        return 0
    if dt == torch.bfloat16:
        return 1
    raise TreError(STATUS_CODE["TRE_E_DTYPE"], where, f"{what}: float32 or bfloat16 wanted, got {dt}")


def _want(t, where, what, shape=None, dtype=None, device=None):
    """A contiguous GPU tensor, of this shape, type and device where given."""
    if not t.is_cuda or (device is not None and t.device != device):
        raise TreError(STATUS_CODE["TRE_E_ARG"], where, f"{what}: on {t.device}, wanted on {device or 'a GPU'}")
    if dtype is not None and t.dtype != dtype:
        raise TreError(STATUS_CODE["TRE_E_DTYPE"], where, f"{what}: {dtype} wanted, got {t.dtype}")
    if (shape is not None and t.shape != shape) or not t.is_contiguous():
        raise TreError(STATUS_CODE["TRE_E_SHAPE"], where,
                       f"{what}: contiguous {tuple(shape) if shape is not None else 'tensor'} wanted, got {tuple(t.shape)}"
                       f" with strides {tuple(t.stride())}")
    return t


class _Here:
    """The device of a call's tensors made current for it (nothing where it is
    already: that check costs a tenth of the context), and its stream: the
    caller's, else the device's current one."""

    def __init__(self, device, stream, where):
        import torch

        if stream is not None and stream.device != device:
            raise TreError(STATUS_CODE["TRE_E_ARG"], where, f"stream: on {stream.device}, the tensors on {device}")
        self.device, self.stream = device, stream
        self.guard = torch.cuda.device(device) if torch.cuda.current_device() != device.index else None
        self.ptr = _stream(stream, device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return self

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)

    def buffer(self, make, result=True):
        return _buffer(self.stream, self.device, make, result)

    def uses(self, *tensors):
        """The caller's tensors: given back while a caller's stream still has the
        call queued, their memory stays theirs until it is done."""
        if self.stream is not None:
            for t in tensors:
                if t is not None:
                    t.record_stream(self.stream)


def _operand(plan, operand, where):
    if plan.dtype != "mxfp4":
        raise TreError(STATUS_CODE["TRE_E_DTYPE"], where, f"the plan's tiles are {plan.dtype}, not mxfp4")
    if operand not in ("u", "v"):
        raise TreError(STATUS_CODE["TRE_E_ARG"], where, f"operand 'u' or 'v' wanted, got {operand!r}")
    return "uv".index(operand)


def mx_quantize(plan: Plan, operand: str, tiles, out=None, stream=None):
    """Tiles [n, tile_elems] (float32 or bfloat16) of the mxfp4 plan's operand
    "u" or "v" in 4 bits (see tre_mx_quantize): uint8 [n, plan.tile_bytes],
    which the plan's calls take."""
    import torch

    w = "tre.mx_quantize"
    o = _operand(plan, operand, w)
    dt = _value_type(tiles, w, "tiles")
    n = int(tiles.shape[0]) if tiles.dim() else -1
    _want(tiles, w, "tiles", (n, plan.tile_elems[o]))
    with _Here(tiles.device, stream, w) as here:
        if out is None:
            out = here.buffer(lambda: torch.empty((n, plan.tile_bytes[o]), dtype=torch.uint8, device=tiles.device))
        else:
            _want(out, w, "out", (n, plan.tile_bytes[o]), torch.uint8, tiles.device)
        here.uses(tiles, out)
        _check(lib().tre_mx_quantize(plan.handle, o, _ptr(tiles), dt, n, _ptr(out), here.ptr), "tre_mx_quantize")
    return out


def mx_dequantize(plan: Plan, operand: str, mx_tiles, dtype=None, out=None, stream=None):
    """The values of 4-bit tiles of the plan's operand "u" or "v" (see
    tre_mx_dequantize): [n, tile_elems] in ``dtype`` (float32, the default, or
    bfloat16; ``out``'s where that is given)."""
    import torch

    w = "tre.mx_dequantize"
    o = _operand(plan, operand, w)
    n = int(mx_tiles.shape[0]) if mx_tiles.dim() else -1
    _want(mx_tiles, w, "mx_tiles", (n, plan.tile_bytes[o]), torch.uint8)
    dt = _value_type(out if out is not None else dtype or torch.float32, w, "out")
    with _Here(mx_tiles.device, stream, w) as here:
        if out is None:
            out = here.buffer(lambda: torch.empty((n, plan.tile_elems[o]), dtype=dtype or torch.float32,
                                                  device=mx_tiles.device))
        else:
            _want(out, w, "out", (n, plan.tile_elems[o]), dtype, mx_tiles.device)
        here.uses(mx_tiles, out)
        _check(lib().tre_mx_dequantize(plan.handle, o, _ptr(mx_tiles), n, _ptr(out), dt, here.ptr), "tre_mx_dequantize")
    return out


def _ids(ids, where, device):
    import torch

    if ids.dtype not in (torch.int32, torch.int64):
        raise TreError(STATUS_CODE["TRE_E_DTYPE"], where, f"ids: int32 or int64 wanted, got {ids.dtype}")
    return _want(ids, where, "ids", device=device)


def _status(status, where, device):
    import torch

    if status is not None:
        _want(status, where, "status", (1,), torch.int64, device)
    return status


def lookup(table, ids, scale: float = 1.0, dtype=None, out=None, plan: Plan | None = None, operand: str = "u",
           status=None, stream=None):
    """Rows of a table by token, ids.shape + [row] (see tre_lookup):
    scale * table[ids], zero where an id is negative.  ``table`` is [n_rows, row]
    in float32 or bfloat16, or 4-bit tiles of an mxfp4 ``plan``'s operand, which
    keeps one label, the token's, and contracts the row's.  ``dtype``: of the
    result (the table's; float32 for 4-bit tiles).  ``status`` (int64 [1]) is
    set to TRE_E_KEYRANGE where an id is n_rows or more; such rows are zero."""
    import torch

    w = "tre.lookup"
    tile_rows = 1
    if plan is not None:
        o = _operand(plan, operand, w)
        b, m, n, k = plan.bmnk
        if b != 1:
            raise TreError(STATUS_CODE["TRE_E_SHAPE"], w, "the plan's operands share a label that W keeps in its tile")
        if not plan.token_keyed[o]:
            raise TreError(STATUS_CODE["TRE_E_SHAPE"], w,
                           f"operand {operand!r} of {plan.einsum!r} ({plan.upper!r} promoted): one label that W keeps, the "
                           "token's, and the others whole in the tile wanted")
        tile_rows, elems, tdt = (m, n)[o], k, 2
        n_tiles = int(table.shape[0]) if table.dim() else -1
        _want(table, w, "table", (n_tiles, plan.tile_bytes[o]), torch.uint8)
        n_rows = n_tiles * tile_rows
    else:
        tdt = _value_type(table, w, "table")
        if table.dim() != 2:
            raise TreError(STATUS_CODE["TRE_E_SHAPE"], w, f"table: [rows, row] wanted, got {tuple(table.shape)}")
        n_rows, elems = int(table.shape[0]), int(table.shape[1])
        _want(table, w, "table")
    _ids(ids, w, table.device)
    _status(status, w, table.device)
    shape = tuple(ids.shape) + (elems,)
    dtype = dtype or (out.dtype if out is not None else torch.float32 if plan is not None else table.dtype)
    odt = _value_type(dtype, w, "out")
    with _Here(table.device, stream, w) as here:
        if out is None:
            out = here.buffer(lambda: torch.empty(shape, dtype=dtype, device=table.device))
        else:
            _want(out, w, "out", shape, dtype, table.device)
        here.uses(table, ids, out, status)
        _check(lib().tre_lookup(_ptr(table), tdt, n_rows, elems, tile_rows, _ptr(ids), ids.element_size(), ids.numel(),
                                float(scale), _ptr(out), odt, _ptr(status), here.ptr), "tre_lookup")
    return out


def lookup_grad_workspace_bytes(n_ids: int, n_rows: int, row_elems: int) -> int:
    return int(lib().tre_lookup_grad_workspace_bytes(int(n_ids), int(n_rows), int(row_elems)))


def lookup_grad(grad, ids, n_rows: int, scale: float = 1.0, dtype=None, out=None, accumulate: bool = False,
                status=None, ws=None, stream=None):
    """The gradient of `lookup` by its table, [n_rows, row] (see
    tre_lookup_grad): scale times the rows of ``grad`` (ids.shape + [row],
    float32 or bfloat16) summed by token in fp32.  ``dtype``: of the result
    (float32); with ``accumulate`` the sums are added to ``out``."""
    import torch

    w = "tre.lookup_grad"
    gdt = _value_type(grad, w, "grad")
    _want(grad, w, "grad")
    _ids(ids, w, grad.device)
    if grad.dim() != ids.dim() + 1 or tuple(grad.shape[:-1]) != tuple(ids.shape):
        raise TreError(STATUS_CODE["TRE_E_SHAPE"], w,
                       f"grad: ids' shape {tuple(ids.shape)} and a row wanted, got {tuple(grad.shape)}")
    if accumulate and out is None:
        raise TreError(STATUS_CODE["TRE_E_ARG"], w, "accumulate needs out")
    _status(status, w, grad.device)
    n, elems, n_rows = ids.numel(), int(grad.shape[-1]), int(n_rows)
    dtype = dtype or (out.dtype if out is not None else torch.float32)
    odt = _value_type(dtype, w, "out")
    with _Here(grad.device, stream, w) as here:
        if out is None:
            out = here.buffer(lambda: torch.empty((n_rows, elems), dtype=dtype, device=grad.device))
        else:
            _want(out, w, "out", (n_rows, elems), dtype, grad.device)
        if ws is None:
            ws = here.buffer(lambda: alloc_workspace(lookup_grad_workspace_bytes(n, n_rows, elems), grad.device),
                             result=False)
        else:
            _want(ws, w, "ws", device=grad.device)
        here.uses(grad, ids, out, status, ws)
        _check(lib().tre_lookup_grad(_ptr(grad), gdt, _ptr(ids), ids.element_size(), n, float(scale), _ptr(out), odt, n_rows,
                                     elems, int(accumulate), _ptr(status), _ptr(ws), ws.numel() * ws.element_size(),
                                     here.ptr), "tre_lookup_grad")
    return out


_tensors = None


def _reader():
    """The reader of tensors, _tensors.so (no other path)."""
    global _tensors
    if _tensors is None:
        import torch  # noqa: F401  (whose libraries it uses)

        try:
            from . import _tensors as t
        except ImportError as e:
            raise RuntimeError(f"_tensors.so is missing: build it with `python -m paper_2603_08957_amd.build` ({e})") from None
        _tensors = t
    return _tensors


# ------------------------------------------------- probabilities of scores

def _scores(x, where, what):
    """(type, n, vocab, cols, row stride, tile stride, address, GPU) of scores
    [n, vocab] or in tiles [tiles, n, cols], whose last dimension is contiguous."""
    got = _reader().scores(x)
    if got is not None:
        return got
    _value_type(x, where, what)
    if x.dim() not in (2, 3) or 0 in (x.shape[-1], x.shape[0] if x.dim() == 3 else 1):
        raise TreError(STATUS_CODE["TRE_E_SHAPE"], where, f"{what}: [n, vocab] or tiles [tiles, n, cols] wanted, got {tuple(x.shape)}")
    if not x.is_cuda:
        raise TreError(STATUS_CODE["TRE_E_ARG"], where, f"{what}: on {x.device}, wanted on a GPU")
    raise TreError(STATUS_CODE["TRE_E_SHAPE"], where, f"{what}: a last stride of 1 wanted, got strides {x.stride()}")


def _words(ids, where, n, gpu, device):
    """(address, bytes of one) of words [n], (None, 0) for none."""
    if ids is None:
        return None, 0
    at = _reader().vector(ids, 1, gpu, n, 0)
    if at is None:
        _ids(ids, where, device)
        raise TreError(STATUS_CODE["TRE_E_SHAPE"], where, f"ids: [{n}] wanted, got {tuple(ids.shape)}")
    return (at, 8) if at > 0 or ids.element_size() == 8 else (-at, 4)


def _floats(t, where, what, n, row, gpu, device):
    """The address of a float32 tensor [n] or [n, row], None for none."""
    import torch

    if t is None:
        return None
    at = _reader().vector(t, 0, gpu, n, row)
    if at is None:
        _want(t, where, what, (n, row) if row else (n,), torch.float32, device)
    return at


@dataclass
class LogProbs:
    """What `log_probs` gives of each token, in float32: views of one allocation.
    They share its memory, which one that is kept keeps whole, and torch's count of
    writes, so that writing one counts for all: clone what is kept long or written."""
    log_prob: object        # [n]: its given word's, or None
    lse: object             # [n]: log of the sum of e^(scale x)
    stats: object           # [n, 2]: what log_probs_grad takes
    entropy: object         # [n], or None
    top_ids: object         # int32 [n, top], or None
    top_log_probs: object   # [n, top], or None


def log_probs_workspace_bytes(n: int, vocab: int, cols: int | None = None, dtype=None, top: int = 0) -> int:
    """For scores [n, vocab], or in tiles of ``cols`` words, of ``dtype`` (float32)."""
    import torch

    dt = _value_type(dtype or torch.float32, "tre.log_probs_workspace_bytes", "dtype")
    return int(lib().tre_log_probs_workspace_bytes(int(n), int(vocab), int(cols or vocab), dt, int(top)))


def log_probs(scores, ids=None, scale: float = 1.0, top: int = 0, entropy: bool = False, status=None, ws=None,
              stream=None) -> LogProbs:
    """Log probabilities out of scores (see tre_log_probs): softmax of scale *
    scores, [n, vocab] or in the tiles [tiles, n, cols] that a score EinSum gives,
    float32 or bfloat16, rows and tiles at any stride.  Of each token the given
    word's (``ids`` [n], int32 or int64; 0 where negative), the log of the sum, the
    entropy and the ``top`` (up to 64) best words, where asked for.  ``status``
    (int64 [1]) is set to TRE_E_KEYRANGE where an id is vocab or more."""
    import torch

    w = "tre.log_probs"
    dt, n, vocab, cols, rows, tiles, at, gpu = _scores(scores, w, "scores")
    dev = scores.device
    ids_at, id_bytes = _words(ids, w, n, gpu, dev)
    if status is not None:
        _status(status, w, dev)
    top = int(top)
    if not 0 <= top <= min(64, vocab):
        raise TreError(STATUS_CODE["TRE_E_SHAPE"], w, f"top: 0 to {min(64, vocab)} wanted, got {top}")
    given, entropy = ids is not None, bool(entropy)
    L = lib()
    with _Here(dev, stream, w) as here:
        # views of one allocation: what several take is most of a small call
        flat = here.buffer(lambda: torch.empty(n * (3 + given + entropy + 2 * top), dtype=torch.float32, device=dev))
        stats, lse, log_prob, h, top_log_probs, top_ids = _reader().views(flat, n, given, entropy, top)
        if ws is not None:
            _want(ws, w, "ws", device=dev)
            need = ws.numel() * ws.element_size()
        else:
            need = L.tre_log_probs_workspace_bytes(n, vocab, cols, dt, top)
            if need:
                ws = here.buffer(lambda: alloc_workspace(need, dev), result=False)
        if stream is not None:
            here.uses(scores, ids, status, ws)
        base = flat.data_ptr()
        _check(L.tre_log_probs(at, dt, n, vocab, cols, rows, tiles, ids_at, id_bytes, float(scale), _at(log_prob), base + 8 * n,
                               base, _at(h), top, _at(top_ids), _at(top_log_probs), _at(status), _at(ws), need, here.ptr),
               "tre_log_probs")
    return LogProbs(log_prob, lse, stats, h, top_ids, top_log_probs)


def log_probs_grad(scores, stats, ids=None, grad_log_prob=None, grad_lse=None, grad_entropy=None, entropy=None,
                   scale: float = 1.0, dtype=None, out=None, status=None, stream=None):
    """The gradient by the scores of a loss whose gradients by `log_probs`'s
    log_prob, lse and entropy are given (see tre_log_probs_grad): ``stats`` and
    ``entropy`` are those that it gave.  In the scores' layout and ``dtype`` (the
    scores'); ``out`` may have strides of its own, and be ``scores``.  torch counts
    the write into ``out`` as one in place."""
    import torch

    w = "tre.log_probs_grad"
    dt, n, vocab, cols, rows, tiles, at, gpu = _scores(scores, w, "scores")
    if grad_log_prob is None and grad_lse is None and grad_entropy is None:
        raise TreError(STATUS_CODE["TRE_E_ARG"], w, "no gradient given")
    dev = scores.device
    stats_at = _floats(stats, w, "stats", n, 2, gpu, dev)
    ids_at, id_bytes = _words(ids, w, n, gpu, dev)
    g, gl, gh, h = (_floats(t, w, what, n, 0, gpu, dev) for t, what in (
        (grad_log_prob, "grad_log_prob"), (grad_lse, "grad_lse"), (grad_entropy, "grad_entropy"), (entropy, "entropy")))
    if status is not None:
        _status(status, w, dev)
    dtype = dtype or (out.dtype if out is not None else scores.dtype)
    odt = _value_type(dtype, w, "out")
    given = out is not None
    with _Here(dev, stream, w) as here:
        if not given:
            out = here.buffer(lambda: torch.empty(scores.shape, dtype=dtype, device=dev))
            out_rows, out_tiles = cols, n * cols
        elif out.shape != scores.shape or out.device != dev or out.dtype != dtype:
            raise TreError(STATUS_CODE["TRE_E_SHAPE"], w, f"out: {dtype} {tuple(scores.shape)} on {dev} wanted, got {out.dtype} "
                                                          f"{tuple(out.shape)} on {out.device}")
        else:
            out_rows, out_tiles = _scores(out, w, "out")[4:6]
        if stream is not None:
            here.uses(scores, stats, ids, grad_log_prob, grad_lse, grad_entropy, entropy, out, status)
        _check(lib().tre_log_probs_grad(at, dt, n, vocab, cols, rows, tiles, stats_at, ids_at, id_bytes, float(scale), g, gl, gh, h,
                                        out.data_ptr(), odt, out_rows, out_tiles, _at(status), here.ptr), "tre_log_probs_grad")
        if given:
            _reader().written(out)
    return out


# ------------------------------------------- a training step of many tensors

class _Many:
    """Host arrays of contiguous GPU tensors' addresses, types and elements, all
    on one device, as the calls over many tensors take them."""

    _WHY = {1: ("TRE_E_ARG", "a list of tensors wanted"), 2: ("TRE_E_ARG", "wanted on one GPU"),
            3: ("TRE_E_SHAPE", "contiguous tensors wanted"), 4: ("TRE_E_DTYPE", "float32 or bfloat16 wanted")}

    def __init__(self, tensors, where, what):
        import torch

        if isinstance(tensors, torch.Tensor):
            tensors = [tensors]
        self.tensors = tensors = tensors if isinstance(tensors, (list, tuple)) else list(tensors)
        why, *got = _reader().gather(tensors)
        if why:
            status, text = self._WHY[why]
            raise TreError(STATUS_CODE[status], where, f"{what}[{got[0]}]: {text}")
        device, self.addresses, self.types, self.sizes = got
        self.n = len(tensors)
        self.device = torch.device("cuda", device) if device >= 0 else None


def grad_norm_workspace_bytes(sizes) -> int:
    """For tensors of these numbers of elements."""
    sizes = array("q", sizes)
    return int(lib().tre_grad_norm_workspace_bytes(len(sizes), sizes.tobytes()))


def grad_norm(tensors, max_norm: float | None = None, out=None, ws=None, stream=None):
    """The norm of a list of tensors (float32 or bfloat16, contiguous, on one GPU)
    taken together, and the factor that brings it to ``max_norm`` at most (1
    without), float32 [2] on their device (see tre_grad_norm).  The factor,
    ``out[1:]``, is what `adamw` takes as ``grad_scale``; it is NaN where the norm
    is not finite, and then `adamw` takes no step."""
    import torch

    w = "tre.grad_norm"
    many = _Many(tensors, w, "tensors")
    if many.device is None:
        raise TreError(STATUS_CODE["TRE_E_ARG"], w, "tensors: none")
    max_norm = -1.0 if max_norm is None else float(max_norm)
    given = out is not None
    with _Here(many.device, stream, w) as here:
        if not given:
            out = here.buffer(lambda: torch.empty(2, dtype=torch.float32, device=many.device))
        else:
            _want(out, w, "out", (2,), torch.float32, many.device)
        if ws is None:
            need = int(lib().tre_grad_norm_workspace_bytes(many.n, many.sizes))
            ws = here.buffer(lambda: alloc_workspace(need, many.device), result=False)
        else:
            _want(ws, w, "ws", device=many.device)
        if stream is not None:
            here.uses(*many.tensors, out, ws)
        _check(lib().tre_grad_norm(many.n, many.addresses, many.types, many.sizes, max_norm, _ptr(out), _ptr(ws),
                                   ws.numel() * ws.element_size(), here.ptr), "tre_grad_norm")
        if given:
            _reader().written(out)
    return out


def adamw_state(params, bits: int = 32, stream=None):
    """Moments of no step yet for a list of tensors (see tre_adamw): zeros,
    float32 [2 T] for 32 bits, uint8 [2 T + T / 16] for 8."""
    import torch

    w = "tre.adamw_state"
    many = _Many(params, w, "params")
    if bits not in (8, 32) or many.device is None:
        raise TreError(STATUS_CODE["TRE_E_ARG"], w, f"tensors and 8 or 32 bits wanted, got {many.n} and {bits}")
    need = int(lib().tre_adamw_state_bytes(many.n, many.sizes, bits))
    with _Here(many.device, stream, w) as here:
        return here.buffer(lambda: torch.zeros(need // 4 if bits == 32 else need, device=many.device,
                                               dtype=torch.float32 if bits == 32 else torch.uint8))


def _device_value(x, where, what, dtype, device):
    """(host value, tensor) of a number or a device tensor of one."""
    if isinstance(x, (int, float)):
        return x, None
    import torch

    if not isinstance(x, torch.Tensor):
        return x, None
    if x.numel() != 1:
        raise TreError(STATUS_CODE["TRE_E_SHAPE"], where, f"{what}: one value wanted, got {tuple(x.shape)}")
    return 0, _want(x, where, what, dtype=dtype, device=device)


def adamw(params, grads, state, step, lr, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
          weight_decay: float = 0.0, grad_scale=1.0, seed: int | None = None, stream=None):
    """One AdamW step of a list of tensors, in place (see tre_adamw): ``params``
    and ``grads`` of the same shapes, float32 or bfloat16, contiguous, on one GPU;
    ``state`` from `adamw_state`, whose type says how many bits the moments have.
    ``step`` (the first is 1), ``lr`` and ``grad_scale`` are numbers or tensors of
    one value (int64, float32, float32) on the device, read when the step runs.
    With a ``seed`` 8-bit moments and bfloat16 weights are rounded by chance, by
    (seed, step, element); else to the nearest.  torch counts the step as one in
    place of ``params`` and ``state``: a backward pass that saved a weight before
    it is an error."""
    import torch

    w = "tre.adamw"
    p, g = _Many(params, w, "params"), _Many(grads, w, "grads")
    if p.device != g.device or p.device is None:
        raise TreError(STATUS_CODE["TRE_E_ARG"], w, f"params and grads wanted on one GPU, got {p.device} and {g.device}")
    if not _reader().same_shapes(p.tensors, g.tensors):
        raise TreError(STATUS_CODE["TRE_E_SHAPE"], w, "grads: params' shapes wanted")
    if state.dtype not in (torch.float32, torch.uint8):
        raise TreError(STATUS_CODE["TRE_E_DTYPE"], w, f"state: float32 or uint8 wanted, got {state.dtype}")
    bits = 32 if state.dtype == torch.float32 else 8
    need = int(lib().tre_adamw_state_bytes(p.n, p.sizes, bits)) // (4 if bits == 32 else 1)
    _want(state, w, "state", (need,), device=p.device)
    step, step_dev = _device_value(step, w, "step", torch.int64, p.device)
    lr, lr_dev = _device_value(lr, w, "lr", torch.float32, p.device)
    scale, scale_dev = _device_value(grad_scale, w, "grad_scale", torch.float32, p.device)
    opt = AdamwOptions(float(lr), float(beta1), float(beta2), float(eps), float(weight_decay), float(scale), int(step),
                       _ptr(lr_dev), _ptr(step_dev), _ptr(scale_dev), (seed or 0) & (1 << 64) - 1, int(seed is not None), bits)
    with _Here(p.device, stream, w) as here:
        if stream is not None:
            here.uses(*p.tensors, *g.tensors, state, step_dev, lr_dev, scale_dev)
        _check(lib().tre_adamw(p.n, p.addresses, p.types, g.addresses, g.types, p.sizes, _ptr(state), ctypes.byref(opt),
                               here.ptr), "tre_adamw")
    _reader().written(p.tensors, state)


def adamw_moments(state, dtype=None, stream=None):
    """The moments m and v that a state of `adamw` holds, [T] each: views of a
    float32 state's; of an 8-bit state's the values (see tre_adamw_moments), in
    ``dtype`` (float32, the default, or bfloat16).  Tensor i's begin at the sum of
    the elements before it, each tensor's taken up to a multiple of 32."""
    import torch

    w = "tre.adamw_moments"
    if state.dtype not in (torch.float32, torch.uint8):
        raise TreError(STATUS_CODE["TRE_E_DTYPE"], w, f"state: float32 or uint8 wanted, got {state.dtype}")
    if state.dtype == torch.float32:
        _want(state, w, "state")
        if dtype not in (None, torch.float32) or state.numel() % 64:
            raise TreError(STATUS_CODE["TRE_E_DTYPE"], w, "32-bit moments are float32, 64 k of them")
        return state.view(2, -1).unbind()
    _want(state, w, "state")
    total = state.numel() * 16 // 33
    if state.numel() % 66 or total % 32:
        raise TreError(STATUS_CODE["TRE_E_SHAPE"], w, f"state: a state of 8 bits wanted, got {state.numel()} bytes")
    dtype = dtype or torch.float32
    dt = _value_type(dtype, w, "moments")
    with _Here(state.device, stream, w) as here:
        m, v = (here.buffer(lambda: torch.empty(total, dtype=dtype, device=state.device)) for _ in range(2))
        here.uses(state)
        _check(lib().tre_adamw_moments(_ptr(state), total, _ptr(m), _ptr(v), dt, here.ptr), "tre_adamw_moments")
    return m, v


def cast_f32_bf16(x, out=None, stream=None):
    import torch

    y = out
    if y is None:
        y = _buffer(stream, x.device, lambda: torch.empty(x.shape, dtype=torch.bfloat16, device=x.device))
    _check(lib().tre_cast_f32_bf16(_ptr(x), _ptr(y), x.numel(), _stream(stream)), "tre_cast_f32_bf16")
    return y


def scale_f32(x, scale: float, out=None, stream=None):
    """out = scale * x (fp32, elementwise; out may be x)."""
    import torch

    y = out if out is not None else _buffer(stream, x.device, lambda: torch.empty_like(x))
    _check(lib().tre_scale_f32(_ptr(x), _ptr(y), x.numel(), float(scale), _stream(stream)), "tre_scale_f32")
    return y


def stack_rows(keys, tiles, group: int, stream=None):
    """STACK re-composition (see tre_stack_rows); keys [n] or [n,1] int32."""
    import torch

    n = int(keys.shape[0])
    row = int(tiles.numel() // max(n, 1)) if n else int(tiles.shape[1])
    eb = tiles.element_size()
    dev = tiles.device
    ws = _buffer(stream, dev, lambda: alloc_workspace(int(lib().tre_stack_workspace_bytes(n)), dev), result=False)
    cap = n
    out_keys = _buffer(stream, dev, lambda: torch.empty((cap, 1), dtype=torch.int32, device=dev))
    out_tiles = _buffer(stream, dev, lambda: torch.empty((cap, group * row), dtype=tiles.dtype, device=dev))
    n_out = ctypes.c_int64(0)
    rc = lib().tre_stack_rows(_ptr(keys), n, _ptr(tiles), row, group, eb, _ptr(out_keys), _ptr(out_tiles), cap,
                              ctypes.byref(n_out), _ptr(ws), ws.numel(), _stream(stream))
    _check(rc, "tre_stack_rows")
    k = int(n_out.value)
    return out_keys[:k], out_tiles[:k]


def repartition(labels: str, upper_in: str, upper_out: str, extents: dict, tiles_in: dict, tiles_out: dict,
                keys, tiles, stream=None, in_place: bool = False):
    """The relation (keys, tiles) under the target decomposition (see
    tre_repartition).  Returns (keys_out [n_out, r_out] int32, tiles_out
    [n_out, tile_elems_out], same dtype as ``tiles``).  ``in_place``: the
    target tiles are a view of ``tiles`` (a regrouping of whole tiles in
    order, nothing missing; TreError otherwise)."""
    import numpy as _np
    import torch

    ext = _np.zeros(26, dtype=_np.int64)
    tin = _np.ones(26, dtype=_np.int32)
    tout = _np.ones(26, dtype=_np.int32)
    for k, v in extents.items():
        ext[ord(k) - 97] = v
    for k, v in (tiles_in or {}).items():
        tin[ord(k) - 97] = v
    for k, v in (tiles_out or {}).items():
        tout[ord(k) - 97] = v
    args = (labels.encode(), upper_in.encode(), upper_out.encode(), ext.ctypes.data_as(ctypes.c_void_p),
            tin.ctypes.data_as(ctypes.c_void_p), tout.ctypes.data_as(ctypes.c_void_p))
    n = int(keys.shape[0]) if keys is not None else int(tiles.shape[0])
    wsb = int(lib().tre_repartition_workspace_bytes(*args, n))
    n_out = ctypes.c_int64(0)
    if wsb == 0:  # bad arguments: let the call itself name the error
        rc = lib().tre_repartition(*args, tiles.element_size(), _ptr(keys), n, _ptr(tiles), None, None, 0,
                                   ctypes.byref(n_out), None, 0, _stream(stream))
        _check(rc if rc else STATUS_CODE["TRE_E_ARG"], "tre_repartition")
    dev = tiles.device
    ws = _buffer(stream, dev, lambda: alloc_workspace(wsb, dev), result=False)
    te_in = te_out = 1
    grid = cover = 1
    for c in labels:
        e, ti, to = int(ext[ord(c) - 97]), int(tin[ord(c) - 97]), int(tout[ord(c) - 97])
        ti = ti if c in upper_in else e
        te_in *= ti
        te_out *= to if c in upper_out else e
        if c in upper_out and to > 0:
            grid *= e // to
            cover *= min(e // to, (ti - 1) // to + 2)
    if in_place:
        cap = (n * te_in) // max(te_out, 1)
        out_keys = _buffer(stream, dev, lambda: torch.empty((max(cap, 1), len(upper_out)), dtype=torch.int32, device=dev))
        rc = lib().tre_repartition(*args, tiles.element_size(), _ptr(keys), n, _ptr(tiles), _ptr(out_keys),
                                   _ptr(tiles), cap, ctypes.byref(n_out), _ptr(ws), ws.numel(), _stream(stream))
        _check(rc, "tre_repartition")
        k = int(n_out.value)
        return out_keys[:k], tiles.reshape(-1)[:k * te_out].view(k, te_out)
    # first call with room for every target tile the sources can meet when
    # that costs little memory; otherwise the call reports the count first
    bound = min(grid, n * cover)
    esz = tiles.element_size()
    cap = bound if bound * te_out * esz <= max(2 * n * te_in * esz, 1 << 26) else 0
    while True:
        out_keys = _buffer(stream, dev, lambda: torch.empty((max(cap, 1), len(upper_out)), dtype=torch.int32, device=dev))
        out_tiles = _buffer(stream, dev, lambda: torch.empty((max(cap, 1), te_out), dtype=tiles.dtype, device=dev))
        rc = lib().tre_repartition(*args, tiles.element_size(), _ptr(keys), n, _ptr(tiles), _ptr(out_keys),
                                   _ptr(out_tiles), cap, ctypes.byref(n_out), _ptr(ws), ws.numel(), _stream(stream))
        if rc == STATUS_CODE["TRE_E_CAPACITY"] and n_out.value > cap:
            cap = int(n_out.value)
            continue
        _check(rc, "tre_repartition")
        k = int(n_out.value)
        return out_keys[:k], out_tiles[:k]


def tiles_from_entries(slot, offset, values, n_tiles: int, tile_elems: int, stream=None):
    """Dense tiles [n_tiles, tile_elems] (dtype of ``values``) from scalar entries."""
    import torch

    tiles = _buffer(stream, values.device,
                    lambda: torch.empty((n_tiles, tile_elems), dtype=values.dtype, device=values.device))
    rc = lib().tre_tiles_from_entries(_ptr(slot), _ptr(offset), _ptr(values), int(values.numel()),
                                      values.element_size(), _ptr(tiles), n_tiles, tile_elems, _stream(stream))
    _check(rc, "tre_tiles_from_entries")
    return tiles


class Einsum3:
    """One three-operand EinSum "U,V,X->W" (see tre_execute3): U joined with V
    and X in one pass, one fused contraction per matched triple.  Holds the
    letter-indexed shape arrays and a workspace sized for ``n_u_max``."""

    def __init__(self, einsum: str, upper: str, extents: dict, tiles: dict, n_u_max: int, device="cuda"):
        import numpy as _np

        self.einsum, self.upper = einsum, upper
        self._ext = _np.zeros(26, dtype=_np.int64)
        self._tile = _np.ones(26, dtype=_np.int32)
        for k, v in extents.items():
            self._ext[ord(k) - 97] = v
        for k, v in (tiles or {}).items():
            self._tile[ord(k) - 97] = v
        w = einsum.split("->")[1]
        self.w_arity = sum(1 for c in w if c in upper)
        self.w_tile_elems = 1
        self.w_key_space = 1
        for c in w:
            e, t = int(self._ext[ord(c) - 97]), int(self._tile[ord(c) - 97])
            self.w_tile_elems *= t if c in upper else e
            if c in upper:
                self.w_key_space *= e // t
        self.n_u_max = int(n_u_max)
        wsb = int(lib().tre_execute3_workspace_bytes(*self._args(), self.n_u_max))
        if wsb == 0:  # bad arguments: let the call itself name the error
            n_w, n_t = ctypes.c_int64(0), ctypes.c_int64(0)
            rc = lib().tre_execute3(*self._args(), 0, None, 0, None, None, 0, None, None, 0, None, None, None, 0,
                                    ctypes.byref(n_w), ctypes.byref(n_t), None, 0, None, None)
            _check(rc if rc else STATUS_CODE["TRE_E_ARG"], "tre_execute3")
        self.ws = alloc_workspace(wsb, device)

    def _args(self):
        return (self.einsum.encode(), self.upper.encode(), self._ext.ctypes.data_as(ctypes.c_void_p),
                self._tile.ctypes.data_as(ctypes.c_void_p))

    def __call__(self, u_keys, u_tiles, v_keys, v_tiles, x_keys, x_tiles, stream=None, timing: Timing | None = None,
                 out=None):
        """Returns (w_keys int32 [n_w, r_W], w_tiles float32 [n_w, tile_elems(W)], n_triples).
        ``out`` = (w_keys, w_tiles) preallocated buffers (their row count is the capacity)."""
        import torch

        n_u, n_v, n_x = int(u_tiles.shape[0]), int(v_tiles.shape[0]), int(x_tiles.shape[0])
        if n_u > self.n_u_max:
            raise ValueError(f"n_u {n_u} above the workspace sizing {self.n_u_max}")
        dev = u_tiles.device
        if stream is not None:
            self.ws.record_stream(stream)
        if out is None:
            cap = min(n_u, self.w_key_space)
            out = (_buffer(stream, dev, lambda: torch.empty((max(cap, 1), self.w_arity), dtype=torch.int32, device=dev)),
                   _buffer(stream, dev, lambda: torch.empty((max(cap, 1), self.w_tile_elems), dtype=torch.float32,
                                                            device=dev)))
            cap_given = cap
        else:
            cap_given = int(out[1].shape[0])
        n_w, n_t = ctypes.c_int64(0), ctypes.c_int64(0)
        rc = lib().tre_execute3(*self._args(), 0, _ptr(u_keys), n_u, _ptr(u_tiles), _ptr(v_keys), n_v, _ptr(v_tiles),
                                _ptr(x_keys), n_x, _ptr(x_tiles), _ptr(out[0]) if self.w_arity else None,
                                _ptr(out[1]), cap_given, ctypes.byref(n_w), ctypes.byref(n_t), _ptr(self.ws),
                                self.ws.numel(), _stream(stream), ctypes.byref(timing) if timing is not None else None)
        _check(rc, "tre_execute3")
        k = int(n_w.value)
        return out[0][:k], out[1][:k], int(n_t.value)


def execute3(einsum: str, upper: str, extents: dict, tiles: dict, u_keys, u_tiles, v_keys, v_tiles, x_keys, x_tiles,
             stream=None, timing: bool = False):
    """One-shot tre_execute3 with a fresh workspace; returns (w_keys, w_tiles,
    n_triples[, timing dict])."""
    import contextlib

    import torch

    with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():  # its workspace is that stream's
        op = Einsum3(einsum, upper, extents, tiles, int(u_tiles.shape[0]), u_tiles.device)
    tm = Timing() if timing else None
    wk, wt, nt = op(u_keys, u_tiles, v_keys, v_tiles, x_keys, x_tiles, stream, tm)
    return (wk, wt, nt, tm.as_dict()) if timing else (wk, wt, nt)
