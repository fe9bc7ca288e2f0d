"""Python binding of liblx (the C ABI declared in include/lx.h).

Argument marshalling only: every step of the forward runs in the CUDA library.
PyTorch provides device memory and the current stream.  There is no fallback:
if liblx.so is missing or cannot load, every call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, NamedTuple, Optional

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "liblx.so")

LX_OK, LX_ERR_ARG, LX_ERR_SHAPE, LX_ERR_CUDA, LX_ERR_OOM, LX_ERR_TIMEOUT, LX_ERR_STATE, \
    LX_ERR_UNSUPPORTED = range(8)
STATUS_NAMES = ["LX_OK", "LX_ERR_ARG", "LX_ERR_SHAPE", "LX_ERR_CUDA", "LX_ERR_OOM",
                "LX_ERR_TIMEOUT", "LX_ERR_STATE", "LX_ERR_UNSUPPORTED"]
LX_F32, LX_BF16, LX_E4M3 = 0, 1, 2
LX_PATH_AUTO, LX_PATH_GENERIC = 0, 1
LX_MAX_DEPTH, LX_MAX_K, LX_MAX_EXPERTS = 4, 32, 1024
LX_MAX_WIDTH, LX_MAX_TEACHER = 65536, 1024
LX_GATE_NONE, LX_GATE_CHANNEL, LX_GATE_TOKEN, LX_GATE_FULL = range(4)
LX_ACT_NONE, LX_ACT_RELU, LX_ACT_SILU, LX_ACT_GELU = range(4)

# every symbol include/lx.h declares
EXPORTS = [
    "lx_load_compressed_layer", "lx_free_layer", "lx_reserve", "lx_route", "lx_bucket",
    "lx_moe_forward", "lx_get_buckets", "lx_layer_info", "lx_set_path", "lx_set_profiling",
    "lx_read_profile", "lx_last_error", "lx_bucket_noalloc", "lx_coact_accumulate",
    "lx_coact_npmi", "lx_align_cost", "lx_lap_solve", "lx_lap_solve_batch", "lx_permute_neurons",
    "lx_compress_workspace", "lx_compress_factor", "lx_set_wait_limit", "lx_inject_unmet_wait",
    "lx_clear_device_error", "lx_inject_unmet_wait_call", "lx_residual_norm",
    "lx_residual_norm_workspace", "lx_residual_norm_backward", "lx_router_balance_workspace",
    "lx_router_balance", "lx_router_balance_backward", "lx_distill_loss", "lx_residual_norm_q8",
    "lx_linear", "lx_linear_workspace", "lx_linear_backward", "lx_head_loss_workspace", "lx_head_loss",
]
(LX_WAIT_NONE, LX_WAIT_STREAM_DEP, LX_WAIT_TC_MMA, LX_WAIT_ROUTER, LX_WAIT_CALL_PRODUCT,
 LX_WAIT_CALL_JACOBI, LX_WAIT_CALL_SUMS, LX_WAIT_CALL_ENTRIES, LX_WAIT_CALL_WRITTEN,
 LX_WAIT_CALL_AGAIN) = range(10)
LX_NOALLOC_SCRATCH_BYTES = 16 << 20


class LxError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < 8 else status}: {msg}")
        self.status = status


class LayerDesc(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32),
                ("n_experts", ctypes.c_int32), ("n_nodes", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("node_parent", ctypes.POINTER(ctypes.c_int32)),
                ("node_rank", ctypes.POINTER(ctypes.c_int32)),
                ("expert_node", ctypes.POINTER(ctypes.c_int32)),
                ("node_sign", ctypes.POINTER(ctypes.c_int8))]


class LayerInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "d_model", "d_ff", "n_experts", "n_nodes", "dtype", "n_anchors", "n_corrections",
        "max_depth", "max_rank")] + [("weight_bytes", ctypes.c_int64)] + [
        (n, ctypes.c_int32) for n in ("last_T", "last_k", "last_rows", "device_error",
                                      "stream_path")]


class ResnormDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "T", "H", "gate_kind")] + [
        (n, ctypes.c_int64) for n in ("ldr", "ldy", "ldg")] + [
        (n, ctypes.c_void_p) for n in ("r", "y", "gate", "w_post", "w_pre")] + [
        (n, ctypes.c_float) for n in ("res_scale", "weight_offset", "eps")]


class LinearDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "T", "N", "K", "act")] + [
        (n, ctypes.c_int64) for n in ("ldx", "ldw", "ldr")] + [
        (n, ctypes.c_void_p) for n in ("x", "w", "x_scale", "w_scale", "bias", "residual")]


class KernelTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("ms", ctypes.c_float)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load liblx.so; raises if it is missing (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2608_07814_gb300.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        u64, f32 = ctypes.c_uint64, ctypes.c_float
        sig = {
            "lx_load_compressed_layer": [ctypes.POINTER(LayerDesc), vp, vp, vp, vp,
                                         ctypes.POINTER(vp)],
            "lx_free_layer": [vp],
            "lx_reserve": [vp, i32, i32],
            "lx_route": [vp, vp, i32, i32, vp, vp, vp, vp],
            "lx_bucket": [vp, vp, i32, i32, vp],
            "lx_moe_forward": [vp, vp, i32, i32, vp, vp],
            "lx_get_buckets": [vp, vp, vp, vp, vp, vp, vp],
            "lx_layer_info": [vp, ctypes.POINTER(LayerInfo)],
            "lx_set_path": [vp, i32],
            "lx_set_profiling": [vp, i32],
            "lx_set_wait_limit": [vp, ctypes.c_uint64],
            "lx_inject_unmet_wait": [vp, i32],
            "lx_inject_unmet_wait_call": [i32, ctypes.c_uint64],
            "lx_clear_device_error": [vp],
            "lx_read_profile": [vp, ctypes.POINTER(KernelTime), i32, ctypes.POINTER(i32)],
            "lx_bucket_noalloc": [vp, vp, i32, i32, vp, vp, vp, vp, vp, vp],
            "lx_coact_accumulate": [vp, i32, i32, i32, vp, vp, vp],
            "lx_coact_npmi": [vp, i32, ctypes.c_int64, vp, vp],
            "lx_align_cost": [i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp],
            "lx_lap_solve": [vp, i32, vp, ctypes.POINTER(ctypes.c_double)],
            "lx_lap_solve_batch": [vp, i32, i32, vp, vp, i32],
            "lx_permute_neurons": [i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp],
            "lx_compress_workspace": [i32, i32, i32, i32, ctypes.POINTER(ctypes.c_uint64)],
            "lx_compress_factor": [i32, i32, i32, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp,
                                   ctypes.c_uint64, vp],
            "lx_residual_norm": [ctypes.POINTER(ResnormDesc), vp, vp, vp, vp],
            "lx_residual_norm_workspace": [i32, i32, ctypes.POINTER(u64)],
            "lx_residual_norm_backward": [ctypes.POINTER(ResnormDesc), vp, vp, i64, vp, i64, vp, vp,
                                          vp, vp, vp, vp, u64, vp],
            "lx_router_balance_workspace": [i32, i32, ctypes.POINTER(u64)],
            "lx_router_balance": [i32, vp, i64, vp, vp, i32, i32, i32, f32, f32, vp, vp, vp, vp, vp,
                                  u64, vp],
            "lx_router_balance_backward": [i32, vp, i64, vp, vp, vp, i32, i32, i32, f32, f32, vp, vp],
            "lx_distill_loss": [i32, vp, i64, vp, vp, vp, vp, vp, i32, i32, i32, f32, f32, f32, vp,
                                vp, i64, vp],
            "lx_residual_norm_q8": [ctypes.POINTER(ResnormDesc), vp, vp, vp, vp, vp, vp],
            "lx_linear": [ctypes.POINTER(LinearDesc), vp, i64, vp, vp],
            "lx_linear_workspace": [i32, i32, i32, ctypes.POINTER(u64)],
            "lx_linear_backward": [ctypes.POINTER(LinearDesc), vp, i64, vp, vp, vp, vp, vp, u64, vp],
            "lx_head_loss_workspace": [i32, i32, i32, i32, i32, ctypes.POINTER(u64)],
            "lx_head_loss": [vp, i64, vp, i64, vp, vp, i32, i32, i32, vp, vp, vp, vp, u64, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = ctypes.c_int
        L.lx_last_error.argtypes = []
        L.lx_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != LX_OK:
        raise LxError(status, lib().lx_last_error().decode())


def _stream(stream: Optional[torch.cuda.Stream]) -> ctypes.c_void_p:
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def host_to_torch(a: np.ndarray, dtype: str) -> torch.Tensor:
    """Storage array (bf16 as uint16 bits, or float32) -> CPU torch tensor."""
    if dtype == "bf16":
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))


class Layer:
    """A compressed MoE layer installed on the current CUDA device.

    ``src`` is any object with the fields of ``synth.CompressedLayer``
    (d_model, d_ff, n_experts, dtype in {'f32','bf16'}, node_parent, node_rank,
    expert_node, node_w, router_w, router_bias, and optionally node_sign)."""

    def __init__(self, src, stream: Optional[torch.cuda.Stream] = None):
        L = lib()
        if src.dtype not in ("f32", "bf16"):
            raise ValueError("liblx stores f32 or bf16 layers")
        self.dtype = src.dtype
        self.torch_dtype = torch.bfloat16 if src.dtype == "bf16" else torch.float32
        self.d_model, self.d_ff, self.n_experts = src.d_model, src.d_ff, src.n_experts
        want = np.uint16 if src.dtype == "bf16" else np.float32
        self._keep = []
        parent = np.ascontiguousarray(src.node_parent, np.int32)
        rank = np.ascontiguousarray(src.node_rank, np.int32)
        enode = np.ascontiguousarray(src.expert_node, np.int32)
        self._keep += [parent, rank, enode]
        sign = getattr(src, "node_sign", None)
        if sign is not None:
            sign = np.ascontiguousarray(sign, np.int8)
            self._keep.append(sign)
        N = parent.shape[0]
        ptrs = (ctypes.c_void_p * (6 * N))()
        for n, ws in enumerate(src.node_w):
            for j, a in enumerate(ws):
                a = np.ascontiguousarray(a, dtype=want)
                self._keep.append(a)
                ptrs[6 * n + j] = a.ctypes.data
        rw = np.ascontiguousarray(src.router_w, dtype=want)
        self._keep.append(rw)
        bias = None
        if src.router_bias is not None:
            bias = np.ascontiguousarray(src.router_bias, np.float32)
            self._keep.append(bias)
        desc = LayerDesc(src.d_model, src.d_ff, src.n_experts, N,
                         LX_BF16 if src.dtype == "bf16" else LX_F32,
                         parent.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                         rank.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                         enode.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                         None if sign is None else sign.ctypes.data_as(
                             ctypes.POINTER(ctypes.c_int8)))
        h = ctypes.c_void_p()
        st = L.lx_load_compressed_layer(ctypes.byref(desc), ptrs, ctypes.c_void_p(rw.ctypes.data),
                                        None if bias is None else ctypes.c_void_p(bias.ctypes.data),
                                        _stream(stream) if torch.cuda.is_available() else None,
                                        ctypes.byref(h))
        self._keep = None
        _check(st)
        self.handle = h
        self.info_cache = self.info()

    # ---- lifetime
    def free(self) -> None:
        if getattr(self, "handle", None):
            _check(lib().lx_free_layer(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    # ---- calls
    def info(self) -> Dict[str, int]:
        inf = LayerInfo()
        _check(lib().lx_layer_info(self.handle, ctypes.byref(inf)))
        return {n: getattr(inf, n) for n, _ in LayerInfo._fields_}

    def reserve(self, max_tokens: int, k: int) -> None:
        _check(lib().lx_reserve(self.handle, max_tokens, k))

    def set_wait_limit(self, cycles: int) -> None:
        """Bound (SM clock cycles) of the kernels' device-side waits; 0 = default."""
        _check(lib().lx_set_wait_limit(self.handle, int(cycles)))

    def inject_unmet_wait(self, site: int) -> None:
        """Test hook: make the wait at `site` (LX_WAIT_*) run out."""
        _check(lib().lx_inject_unmet_wait(self.handle, int(site)))

    def clear_device_error(self) -> None:
        _check(lib().lx_clear_device_error(self.handle))

    def set_path(self, path: int) -> None:
        _check(lib().lx_set_path(self.handle, path))

    def set_profiling(self, on: bool) -> None:
        _check(lib().lx_set_profiling(self.handle, 1 if on else 0))

    def read_profile(self, cap: int = 4096):
        buf = (KernelTime * cap)()
        n = ctypes.c_int32()
        _check(lib().lx_read_profile(self.handle, buf, cap, ctypes.byref(n)))
        return [(buf[i].name.decode(), float(buf[i].ms)) for i in range(n.value)]

    def route(self, x: torch.Tensor, k: int, want_logits: bool = False, stream=None):
        T = x.shape[0]
        dev = x.device
        ids = torch.empty((T, k), dtype=torch.int32, device=dev)
        w = torch.empty((T, k), dtype=torch.float32, device=dev)
        logits = torch.empty((T, self.n_experts), dtype=torch.float32, device=dev) \
            if want_logits else None
        _check(lib().lx_route(self.handle, _ptr(x), T, k, _ptr(ids), _ptr(w), _ptr(logits),
                              _stream(stream)))
        return (ids, w, logits) if want_logits else (ids, w)

    def bucket(self, topk_id: torch.Tensor, stream=None) -> None:
        T, k = topk_id.shape
        _check(lib().lx_bucket(self.handle, _ptr(topk_id), T, k, _stream(stream)))

    def moe_forward(self, x: torch.Tensor, k: int, y: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
        if y is None:
            y = torch.empty_like(x)
        _check(lib().lx_moe_forward(self.handle, _ptr(x), x.shape[0], k, _ptr(y),
                                    _stream(stream)))
        return y

    def get_buckets(self, stream=None) -> Dict[str, torch.Tensor]:
        inf = self.info()
        T, k, D = inf["last_T"], inf["last_k"], inf["max_depth"]
        dev = torch.device("cuda", torch.cuda.current_device())
        z = lambda n: torch.empty(max(1, n), dtype=torch.int32, device=dev)
        out = dict(node_off=z(inf["n_nodes"] + 1), node_tok=z(T * k * D), node_row=z(T * k * D),
                   expert_off=z(self.n_experts + 1), perm=z(T * k))
        _check(lib().lx_get_buckets(self.handle, _ptr(out["node_off"]), _ptr(out["node_tok"]),
                                    _ptr(out["node_row"]), _ptr(out["expert_off"]),
                                    _ptr(out["perm"]), _stream(stream)))
        out["node_tok"] = out["node_tok"][:inf["last_rows"]]
        out["node_row"] = out["node_row"][:T * k * D]
        out["perm"] = out["perm"][:T * k]
        return out


# ----------------------------------------------------------------------------
# router profiling statistics (standalone calls, no layer)
# ----------------------------------------------------------------------------
def coact_accumulate(topk_id: torch.Tensor, E: int, fire: Optional[torch.Tensor] = None,
                     coact: Optional[torch.Tensor] = None, stream=None):
    """Adds the batch topk_id [T, k] (int32, device) to the uint64 counters
    fire [E] and coact [E, E] (int64 tensors holding the unsigned counts;
    allocated zeroed when omitted).  Returns (fire, coact)."""
    dev = topk_id.device
    if fire is None:
        fire = torch.zeros(E, dtype=torch.int64, device=dev)
    if coact is None:
        coact = torch.zeros((E, E), dtype=torch.int64, device=dev)
    T, k = topk_id.shape
    _check(lib().lx_coact_accumulate(_ptr(topk_id), T, k, E, _ptr(fire), _ptr(coact),
                                     _stream(stream)))
    return fire, coact


def coact_npmi(coact: torch.Tensor, n_tokens: int, stream=None) -> torch.Tensor:
    """float64 [E, E] NPMI of the counts coact [E, E] over n_tokens tokens."""
    E = coact.shape[0]
    out = torch.empty((E, E), dtype=torch.float64, device=coact.device)
    _check(lib().lx_coact_npmi(_ptr(coact), E, n_tokens, _ptr(out), _stream(stream)))
    return out


# ----------------------------------------------------------------------------
# neuron alignment (standalone calls on plain expert matrices)
# ----------------------------------------------------------------------------
def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return LX_BF16
    if t.dtype == torch.float32:
        return LX_F32
    raise ValueError("expert matrices must be bf16 or fp32")


def align_cost(dom, mem, stream=None) -> torch.Tensor:
    """fp32 [I, I] cost of matching dominant neurons (rows) with member neurons
    (columns); dom and mem are (gate [I,H], up [I,H], down [H,I]) device tensors."""
    g = dom[0]
    I, H = g.shape
    cost = torch.empty((I, I), dtype=torch.float32, device=g.device)
    _check(lib().lx_align_cost(_dtype_code(g), H, I, *[_ptr(t) for t in dom],
                               *[_ptr(t) for t in mem], _ptr(cost), _stream(stream)))
    return cost


def inject_unmet_wait_call(site: int, cycles: int = 0) -> None:
    """Test hook: in this thread's next align_cost / compress_factor / distill_loss the wait at
    `site` (LX_WAIT_CALL_*) runs out after `cycles` SM clock cycles."""
    _check(lib().lx_inject_unmet_wait_call(int(site), int(cycles)))


def lap_solve(cost: np.ndarray):
    """(assign int32 [n], total float) of the exact assignment of a host cost."""
    c = np.ascontiguousarray(cost, dtype=np.float32)
    n = c.shape[0]
    out = np.empty(n, np.int32)
    tot = ctypes.c_double()
    _check(lib().lx_lap_solve(ctypes.c_void_p(c.ctypes.data), n,
                              ctypes.c_void_p(out.ctypes.data), ctypes.byref(tot)))
    return out, tot.value


def lap_solve_batch(costs: np.ndarray, threads: int = 0):
    """(assign int32 [count, n], totals float64 [count]) of independent host
    costs [count, n, n], solved on `threads` host threads (0: all cores)."""
    c = np.ascontiguousarray(costs, dtype=np.float32)
    count, n = c.shape[0], c.shape[1]
    out = np.empty((count, n), np.int32)
    tot = np.empty(count, np.float64)
    _check(lib().lx_lap_solve_batch(ctypes.c_void_p(c.ctypes.data), n, count,
                                    ctypes.c_void_p(out.ctypes.data),
                                    ctypes.c_void_p(tot.ctypes.data), threads))
    return out, tot


def permute_neurons(perm: torch.Tensor, gate: torch.Tensor, up: torch.Tensor,
                    down: torch.Tensor, stream=None, out=None):
    """(gate, up, down) of the member with neuron i taken from neuron perm[i]
    (into ``out`` when given)."""
    I, H = gate.shape
    outs = out if out is not None else (torch.empty_like(gate), torch.empty_like(up),
                                        torch.empty_like(down))
    _check(lib().lx_permute_neurons(_dtype_code(gate), H, I, _ptr(perm), _ptr(gate), _ptr(up),
                                    _ptr(down), *[_ptr(t) for t in outs], _stream(stream)))
    return outs


# ----------------------------------------------------------------------------
# compression of one member projection
# ----------------------------------------------------------------------------
def compress_workspace_bytes(rows: int, cols: int, l: int, r: int) -> int:
    b = ctypes.c_uint64()
    _check(lib().lx_compress_workspace(rows, cols, l, r, ctypes.byref(b)))
    return int(b.value)


def compress_factor(w_dom: torch.Tensor, w_mem: torch.Tensor, omega: torch.Tensor, r: int,
                    power_iters: int = 2, workspace: Optional[torch.Tensor] = None,
                    stream=None, out=None):
    """(U [rows, r], V [cols, r], s [r]) fp32 with U V^T ~ w_mem - w_dom; omega
    is the fp32 [cols, l] Gaussian test matrix.  ``out`` = preallocated
    (U, V, s); independent projections may run concurrently on their own
    streams, each with its own workspace."""
    rows, cols = w_dom.shape
    l = omega.shape[1]
    need = compress_workspace_bytes(rows, cols, l, r)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=w_dom.device)
    dev = w_dom.device
    if out is None:
        out = (torch.empty((rows, r), dtype=torch.float32, device=dev),
               torch.empty((cols, r), dtype=torch.float32, device=dev),
               torch.empty(r, dtype=torch.float32, device=dev))
    U, V, s = out
    _check(lib().lx_compress_factor(_dtype_code(w_dom), rows, cols, _ptr(w_dom), _ptr(w_mem),
                                    _ptr(omega), l, r, power_iters, _ptr(U), _ptr(V), _ptr(s),
                                    _ptr(workspace), workspace.numel(), _stream(stream)))
    return U, V, s


_MEMBER_STREAMS: Dict[int, list] = {}


def compress_member(w_doms, w_mems, omegas, r: int, power_iters: int = 2, workspaces=None,
                    outs=None):
    """The gate, up and down projections of one member, each through
    lx_compress_factor on a stream of its own (the three are independent), the
    calling stream waiting for all three.  Lists of three: dominant and member
    matrices, fp32 Gaussian test matrices, optional workspaces and outputs.
    Returns the three (U, V, s)."""
    dev = w_doms[0].device
    main = torch.cuda.current_stream(dev)
    key = dev.index if dev.index is not None else torch.cuda.current_device()
    if key not in _MEMBER_STREAMS:
        _MEMBER_STREAMS[key] = [torch.cuda.Stream(device=dev) for _ in range(3)]
    streams = _MEMBER_STREAMS[key]
    start = torch.cuda.Event()
    start.record(main)
    res = []
    for j in range(3):
        st = streams[j]
        st.wait_event(start)
        ws = workspaces[j] if workspaces is not None else None
        out = outs[j] if outs is not None else None
        with torch.cuda.stream(st):
            res.append(compress_factor(w_doms[j], w_mems[j], omegas[j], r, power_iters,
                                       workspace=ws, stream=st, out=out))
        done = torch.cuda.Event()
        done.record(st)
        main.wait_event(done)
        if out is None:
            for t in res[-1]:  # allocated on the side stream, used on the caller's
                t.record_stream(main)
    return res


# ----------------------------------------------------------------------------
# the operators around a layer: block norms, router balance loss, distillation
# ----------------------------------------------------------------------------
# The tensors of a call, a workspace among them, lie on the current device: the library
# launches there.
_DTYPES = {torch.bfloat16: LX_BF16, torch.float32: LX_F32}

# the current device, and the cudaStream_t of a device's current stream
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _device(t: torch.Tensor, name: str) -> int:
    """Checks that a tensor is on the current device, where the launches go; its index."""
    dev = t.get_device()
    if dev < 0 or dev != _current_device():
        raise ValueError(f"{name} must be a CUDA tensor on the current device")
    return dev


def _rows(t: torch.Tensor, name: str, dev: int, shape=None, dtype=None) -> int:
    """Checks a matrix of rows (unit stride inside a row) on device dev and returns their distance."""
    if t.dim() != 2 or t.get_device() != dev:
        raise ValueError(f"{name} must be a matrix on cuda:{dev}")
    have = t.shape
    if shape is not None and have != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have the dtype {dtype}")
    T, n = have
    ld, inner = t.stride()
    if inner != 1 and n > 1:
        raise ValueError(f"{name} must have unit stride inside a row")
    return ld if T > 1 else max(n, 1)


def _flat(t: Optional[torch.Tensor], name: str, dev: int, n: int, dtype=torch.float32):
    """Checks a contiguous array of n elements (or None) on device dev and returns its address."""
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous array of {n} {dtype} elements on cuda:{dev}")
    return t.data_ptr()


def _check_workspace(t: torch.Tensor, dev: int) -> None:
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous array on cuda:{dev}")


def _type(dtype: torch.dtype, name: str) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"{name} must be bf16 or fp32")
    return code


def _elsewhere(stream, fn, args, kwargs):
    """fn(*args, **kwargs) with `stream` current.  What it allocates belongs to that
    stream; its inputs there, and its outputs on the caller's stream, are marked as used,
    so that no memory is given away early.  The order of the streams is the caller's."""
    here = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        if stream != here:
            for t in (*args, *kwargs.values()):
                for u in t if isinstance(t, tuple) else (t,):
                    if isinstance(u, torch.Tensor) and u.is_cuda:
                        u.record_stream(stream)
        out = fn(*args, **kwargs)
    if stream != here:
        for t in out if isinstance(out, tuple) else (out,):
            if t is not None:
                t.record_stream(here)
    return out


def _resnorm_desc(dev, r, y, w_post, gate, w_pre, res_scale, weight_offset, eps):
    """(descriptor, r's shape, its dtype)."""
    ldr = _rows(r, "r", dev)
    shape, dtype = r.shape, r.dtype
    T, H = shape
    kind = ldy = ldg = 0
    yp = gp = None
    if y is not None:
        ldy, yp = _rows(y, "y", dev, shape, dtype), y.data_ptr()
    if gate is not None:
        if gate.dim() == 1:
            kind, gp = LX_GATE_CHANNEL, _flat(gate, "a gate of one dimension", dev, H)
        elif gate.shape == (T, 1) and (H != 1 or gate.dtype == torch.float32):
            kind, ldg, gp = LX_GATE_TOKEN, _rows(gate, "gate", dev, None, torch.float32), gate.data_ptr()
        else:
            kind, ldg, gp = LX_GATE_FULL, _rows(gate, "gate", dev, shape, dtype), gate.data_ptr()
    return ResnormDesc(_type(dtype, "r"), T, H, kind, ldr, ldy, ldg, r.data_ptr(), yp, gp,
                       _flat(w_post, "w_post", dev, H), _flat(w_pre, "w_pre", dev, H), res_scale,
                       weight_offset, eps), shape, dtype


def residual_norm(r: torch.Tensor, y: Optional[torch.Tensor] = None, *, w_post=None, gate=None,
                  w_pre=None, res_scale: float = 1.0, weight_offset: float = 0.0, eps: float = 1e-6,
                  r_out=None, h_out=None, stats=None, stream=None):
    """The norm after a block, its gate and residual, and the norm before the next:

        u = rms_norm(y) * (weight_offset + w_post)        (y itself without w_post)
        r_out = res_scale * r + gate * u
        h = rms_norm(r_out) * (weight_offset + w_pre)

    r and y are [T, H] (bf16 or fp32, rows may be slices of wider ones); w_post and
    w_pre fp32 [H]; gate fp32 [H], fp32 [T, 1] or [T, H] in r's type.  Returns (r_out,
    h); h is None without w_pre.  Without y only the norm is taken, and r_out is r
    itself unless res_scale is not 1 or a buffer is given.  ``r_out`` may be r (in
    place).  ``stats``: fp32 [2, T] for residual_norm_backward."""
    if stream is not None:
        return _elsewhere(stream, residual_norm, (r, y), dict(
            w_post=w_post, gate=gate, w_pre=w_pre, res_scale=res_scale, weight_offset=weight_offset,
            eps=eps, r_out=r_out, h_out=h_out, stats=stats))
    dev = _device(r, "r")
    d, shape, dtype = _resnorm_desc(dev, r, y, w_post, gate, w_pre, res_scale, weight_offset, eps)
    n = shape[0] * shape[1]
    rp, hp = _flat(r_out, "r_out", dev, n, dtype), _flat(h_out, "h_out", dev, n, dtype)
    if r_out is None and (y is not None or res_scale != 1.0):
        r_out, rp = _empty_for(r, shape)
    if h_out is None and w_pre is not None:
        h_out, hp = _empty_for(r, shape)
    status = lib().lx_residual_norm(d, rp, hp, _flat(stats, "stats", dev, 2 * shape[0]), _raw_stream(dev))
    if status:
        _check(status)
    return (r if r_out is None else r_out), h_out


class ResidualNormGrads(NamedTuple):
    """Gradients of residual_norm; None where the input was absent."""
    dr: torch.Tensor
    dy: Optional[torch.Tensor]
    dw_post: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dw_pre: Optional[torch.Tensor]


def _empty_for(t: Optional[torch.Tensor], shape):
    """(uninitialised tensor of t's type, its address), or Nones for None."""
    if t is None:
        return None, None
    e = torch.empty(shape, dtype=t.dtype, device=t.device)
    return e, e.data_ptr()


def residual_norm_workspace_bytes(T: int, H: int) -> int:
    b = ctypes.c_uint64()
    _check(lib().lx_residual_norm_workspace(T, H, b))
    return b.value


def residual_norm_backward(dr_out, dh, r, y, stats, *, w_post=None, gate=None, w_pre=None,
                           res_scale: float = 1.0, weight_offset: float = 0.0, workspace=None,
                           stream=None) -> ResidualNormGrads:
    """Gradients of residual_norm with respect to r, y, w_post, gate and w_pre, from
    those of r_out and h (either may be None for zero).  The other arguments are the
    forward's (r as it was before the call) and the stats it wrote."""
    if stream is not None:
        return _elsewhere(stream, residual_norm_backward, (dr_out, dh, r, y, stats), dict(
            w_post=w_post, gate=gate, w_pre=w_pre, res_scale=res_scale, weight_offset=weight_offset,
            workspace=workspace))
    dev = _device(r, "r")
    d, shape, dtype = _resnorm_desc(dev, r, y, w_post, gate, w_pre, res_scale, weight_offset, 0.0)
    T, H = shape
    lddr = lddh = 0
    drp = dhp = None
    if dr_out is not None:
        lddr, drp = _rows(dr_out, "dr_out", dev, shape, dtype), dr_out.data_ptr()
    if dh is not None:
        lddh, dhp = _rows(dh, "dh", dev, shape, dtype), dh.data_ptr()
    dr, p0 = _empty_for(r, shape)
    dy, p1 = _empty_for(y, shape)
    dw_post, p2 = _empty_for(w_post, H)
    dgate, p3 = _empty_for(gate, None if gate is None else gate.shape)
    dw_pre, p4 = _empty_for(w_pre, H)
    if workspace is None:
        workspace = torch.empty(residual_norm_workspace_bytes(T, H), dtype=torch.uint8, device=r.device)
    else:
        _check_workspace(workspace, dev)
    status = lib().lx_residual_norm_backward(
        d, _flat(stats, "stats", dev, 2 * T), drp, lddr, dhp, lddh, p0, p1, p2, p3, p4,
        workspace.data_ptr(), workspace.nbytes, _raw_stream(dev))
    if status:
        _check(status)
    return ResidualNormGrads(dr, dy, dw_post, dgate, dw_pre)


class RouterBalance(NamedTuple):
    """What router_balance computes: loss fp32 [3] (the loss, its balance and z parts),
    counts int32 [E + 1] (tokens of each expert, then the tokens that counted), prob
    fp32 [E] (mean router probability), lse fp32 [T] (log-sum-exp of each token, -inf
    where it did not count)."""
    loss: torch.Tensor
    counts: torch.Tensor
    prob: torch.Tensor
    lse: torch.Tensor


def router_balance_workspace_bytes(T: int, E: int) -> int:
    b = ctypes.c_uint64()
    _check(lib().lx_router_balance_workspace(T, E, b))
    return b.value


def router_balance(logits: torch.Tensor, topk_id: torch.Tensor, *, mask=None,
                   balance_coef: float = 0.01, z_coef: float = 0.0, workspace=None,
                   stream=None) -> RouterBalance:
    """Balance loss E sum_e (c_e / (n k)) P_e and z loss mean(lse^2) of the router's
    logits [T, E] (fp32 as Layer.route gives them, or bf16) and its int32 ids [T, k],
    over the tokens whose mask (bool or uint8 [T]) is not 0."""
    if stream is not None:
        return _elsewhere(stream, router_balance, (logits, topk_id), dict(
            mask=mask, balance_coef=balance_coef, z_coef=z_coef, workspace=workspace))
    at = _device(logits, "logits")
    ld = _rows(logits, "logits", at)
    T, E = logits.shape
    if topk_id.dim() != 2 or topk_id.shape[0] != T:
        raise ValueError("topk_id must be [T, k]")
    k, dev = topk_id.shape[1], logits.device
    ids = _flat(topk_id, "topk_id", at, T * k, torch.int32)
    if mask is not None:
        if mask.dtype not in (torch.bool, torch.uint8):
            raise ValueError("mask must be bool or uint8")
        mask = _flat(mask, "mask", at, T, mask.dtype)
    loss = torch.empty(3, dtype=torch.float32, device=dev)
    counts = torch.empty(E + 1, dtype=torch.int32, device=dev)
    prob = torch.empty(E, dtype=torch.float32, device=dev)
    lse = torch.empty(T, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = torch.empty(router_balance_workspace_bytes(T, E), dtype=torch.uint8, device=dev)
    else:
        _check_workspace(workspace, at)
    status = lib().lx_router_balance(
        _type(logits.dtype, "logits"), logits.data_ptr(), ld, ids, mask, T, E, k, balance_coef, z_coef,
        counts.data_ptr(), prob.data_ptr(), lse.data_ptr(), loss.data_ptr(), workspace.data_ptr(),
        workspace.nbytes, _raw_stream(at))
    if status:
        _check(status)
    return RouterBalance(loss, counts, prob, lse)


def router_balance_backward(logits: torch.Tensor, state: RouterBalance, k: int, *, dloss=None,
                            balance_coef: float = 0.01, z_coef: float = 0.0, out=None,
                            stream=None) -> torch.Tensor:
    """Gradient of router_balance's loss with respect to the logits, in their type,
    times dloss (an fp32 device scalar; 1 when omitted); the counts are held fixed.
    `state` and the coefficients are the forward's, k its ids per token.  ``out`` may
    be the logits themselves."""
    if stream is not None:
        return _elsewhere(stream, router_balance_backward, (logits, state, k), dict(
            dloss=dloss, balance_coef=balance_coef, z_coef=z_coef, out=out))
    dev = _device(logits, "logits")
    ld = _rows(logits, "logits", dev)
    T, E = logits.shape
    op = _flat(out, "out", dev, T * E, logits.dtype)
    if out is None:
        out, op = _empty_for(logits, (T, E))
    status = lib().lx_router_balance_backward(
        _type(logits.dtype, "logits"), logits.data_ptr(), ld, _flat(state.lse, "lse", dev, T),
        _flat(state.counts, "counts", dev, E + 1, torch.int32), _flat(dloss, "dloss", dev, 1), T, E, k,
        balance_coef, z_coef, op, _raw_stream(dev))
    if status:
        _check(status)
    return out


def distill_loss(logits: torch.Tensor, teacher_id: torch.Tensor, teacher_logit: torch.Tensor, *,
                 temperature: float = 1.0, teacher_lse=None, kd_weight: float = 1.0, labels=None,
                 ce_weight: float = 0.0, row_weight=None, want_grad: bool = True, dlogits=None,
                 stream=None):
    """Distillation of the student's logits [T, V] (bf16 or fp32) from a teacher's
    stored top entries (int32 ids and fp32 logits [T, K]), optionally mixed with the
    cross-entropy of int32 labels [T]:

        loss = row_weight * (kd_weight * temperature^2 * KL + ce_weight * CE)

    teacher_lse (fp32 [T]): log-sum-exp of the teacher's logits over the temperature;
    the entries then keep their share of its whole distribution, otherwise they are
    normalised among themselves.  Returns (loss fp32 [T], gradient of its sum with
    respect to the logits, or None).  ``dlogits`` may be the logits themselves."""
    if stream is not None:
        return _elsewhere(stream, distill_loss, (logits, teacher_id, teacher_logit), dict(
            temperature=temperature, teacher_lse=teacher_lse, kd_weight=kd_weight, labels=labels,
            ce_weight=ce_weight, row_weight=row_weight, want_grad=want_grad, dlogits=dlogits))
    at = _device(logits, "logits")
    ld = _rows(logits, "logits", at)
    T, V = logits.shape
    dtype = logits.dtype
    if teacher_id.dim() != 2 or teacher_id.shape[0] != T:
        raise ValueError("teacher_id must be [T, K]")
    K, dev = teacher_id.shape[1], logits.device
    code = _type(dtype, "logits")
    ids = _flat(teacher_id, "teacher_id", at, T * K, torch.int32)
    top = _flat(teacher_logit, "teacher_logit", at, T * K)
    loss = torch.empty(T, dtype=torch.float32, device=dev)
    ldd, dp = V, None
    if dlogits is not None:
        ldd, dp = _rows(dlogits, "dlogits", at, logits.shape, dtype), dlogits.data_ptr()
    elif want_grad:
        dlogits = torch.empty((T, V), dtype=dtype, device=dev)
        dp = dlogits.data_ptr()
    status = lib().lx_distill_loss(
        code, logits.data_ptr(), ld, ids, top, _flat(teacher_lse, "teacher_lse", at, T),
        _flat(labels, "labels", at, T, torch.int32), _flat(row_weight, "row_weight", at, T), T, V, K,
        temperature, kd_weight, ce_weight, loss.data_ptr(), dp, ldd, _raw_stream(at))
    if status:
        _check(status)
    return loss, dlogits


# ----------------------------------------------------------------------------
# products around a layer: the norm's output in 8 bits, dense products, the head's loss
# ----------------------------------------------------------------------------
class ResidualNormQ8(NamedTuple):
    """What residual_norm_q8 gives: r_out, and h as e4m3 [T, H] with a scale fp32 [T]."""
    r_out: torch.Tensor
    q: torch.Tensor
    scale: torch.Tensor


def residual_norm_q8(r: torch.Tensor, y: Optional[torch.Tensor] = None, *, w_pre, w_post=None, gate=None,
                     res_scale: float = 1.0, weight_offset: float = 0.0, eps: float = 1e-6, r_out=None,
                     q_out=None, scale_out=None, h_out=None, stats=None, stream=None) -> ResidualNormQ8:
    """residual_norm with h in 8 bits, as `linear` reads it:

        scale = max(max|h| / 448, 2^-126) of each token,  q = e4m3(h / scale)

    The other arguments are residual_norm's; ``h_out`` (in r's type) takes h itself too
    where one is given.  For weights in 8 bits, a scale for each output:
    ``s = (w.float().abs().amax(1) / 448).clamp(min=2**-126)``,
    ``(w.float() / s[:, None]).to(torch.float8_e4m3fn)``."""
    if stream is not None:
        return _elsewhere(stream, residual_norm_q8, (r, y), dict(
            w_pre=w_pre, w_post=w_post, gate=gate, res_scale=res_scale, weight_offset=weight_offset, eps=eps,
            r_out=r_out, q_out=q_out, scale_out=scale_out, h_out=h_out, stats=stats))
    dev = _device(r, "r")
    d, shape, dtype = _resnorm_desc(dev, r, y, w_post, gate, w_pre, res_scale, weight_offset, eps)
    T, H = shape
    n = T * H
    rp, hp = _flat(r_out, "r_out", dev, n, dtype), _flat(h_out, "h_out", dev, n, dtype)
    if r_out is None and (y is not None or res_scale != 1.0):
        r_out, rp = _empty_for(r, shape)
    if q_out is None:
        q_out = torch.empty(shape, dtype=torch.float8_e4m3fn, device=r.device)
    if scale_out is None:
        scale_out = torch.empty(T, dtype=torch.float32, device=r.device)
    status = lib().lx_residual_norm_q8(
        d, rp, _flat(q_out, "q_out", dev, n, torch.float8_e4m3fn), _flat(scale_out, "scale_out", dev, T), hp,
        _flat(stats, "stats", dev, 2 * T), _raw_stream(dev))
    if status:
        _check(status)
    return ResidualNormQ8(r if r_out is None else r_out, q_out, scale_out)


_ACTS = {"none": LX_ACT_NONE, "relu": LX_ACT_RELU, "silu": LX_ACT_SILU, "gelu": LX_ACT_GELU}
_LINEAR_TYPES = {torch.bfloat16: LX_BF16, torch.float8_e4m3fn: LX_E4M3}


def _linear_args(dev, x, w, act):
    """(type, T, N, K, activation, ldx, ldw): what a product is described by."""
    dtype = x.dtype
    code = _LINEAR_TYPES.get(dtype)
    if code is None:
        raise ValueError("x must be bf16 or e4m3")
    a = _ACTS.get(act)
    if a is None:
        raise ValueError("act must be one of " + ", ".join(_ACTS))
    ldx, ldw = _rows(x, "x", dev), _rows(w, "w", dev, None, dtype)
    T, K = x.shape
    N, k = w.shape
    if k != K:
        raise ValueError(f"w must be [N, {K}]")
    return code, T, N, K, a, ldx, ldw


def linear(x: torch.Tensor, w: torch.Tensor, *, x_scale=None, w_scale=None, bias=None, act: str = "none",
           residual=None, y=None, pre=None, stream=None) -> torch.Tensor:
    """y = act(x w^T + bias) + residual, bf16 [T, N], of x [T, K] and w [N, K] in bf16, or in
    e4m3 with x_scale fp32 [T] and w_scale fp32 [N] (the product times both).

    act: "none", "relu", "silu" or "gelu" (by the error function); bias bf16 [N]; residual
    bf16 [T, N]; rows of x, w, residual and y may be slices of wider ones (x's and w's on
    16-byte boundaries, K a multiple of 16 bytes).  ``y`` may be the residual (in place);
    ``pre`` (bf16 [T, N]) takes the sum before the activation for linear_backward."""
    if stream is not None:
        return _elsewhere(stream, linear, (x, w), dict(x_scale=x_scale, w_scale=w_scale, bias=bias, act=act,
                                                       residual=residual, y=y, pre=pre))
    dev = _device(x, "x")
    code, T, N, K, a, ldx, ldw = _linear_args(dev, x, w, act)
    bf = torch.bfloat16
    xs = ws = bp = rp = pp = None
    if code == LX_E4M3:
        if x_scale is None or w_scale is None:
            raise ValueError("x_scale and w_scale go with e4m3")
        xs, ws = _flat(x_scale, "x_scale", dev, T), _flat(w_scale, "w_scale", dev, N)
    elif x_scale is not None or w_scale is not None:
        raise ValueError("x_scale and w_scale go with e4m3")
    if bias is not None:
        bp = _flat(bias, "bias", dev, N, bf)
    ldr = 0
    if residual is not None:
        ldr, rp = _rows(residual, "residual", dev, (T, N), bf), residual.data_ptr()
    if pre is not None:
        pp = _flat(pre, "pre", dev, T * N, bf)
    if y is None:
        y, ldy = torch.empty((T, N), dtype=bf, device=x.device), N
    else:
        ldy = _rows(y, "y", dev, (T, N), bf)
    status = lib().lx_linear(
        LinearDesc(code, T, N, K, a, ldx, ldw, ldr, x.data_ptr(), w.data_ptr(), xs, ws, bp, rp), y.data_ptr(), ldy, pp,
        _raw_stream(dev))
    if status:
        _check(status)
    return y


class LinearGrads(NamedTuple):
    """Gradients of linear; None where not asked for.  (The residual's is dy.)"""
    dx: Optional[torch.Tensor]
    dw: Optional[torch.Tensor]
    dbias: Optional[torch.Tensor]


def linear_workspace_bytes(T: int, N: int, K: int) -> int:
    b = ctypes.c_uint64()
    _check(lib().lx_linear_workspace(T, N, K, b))
    return b.value


def linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, *, act: str = "none", pre=None,
                    want_dx: bool = True, want_dw: bool = True, want_dbias: bool = False, workspace=None,
                    stream=None) -> LinearGrads:
    """Gradients of linear (bf16) with respect to x, w and bias from that of y [T, N]; x, w,
    act and pre are the forward's (pre with an activation alone)."""
    if stream is not None:
        return _elsewhere(stream, linear_backward, (dy, x, w), dict(
            act=act, pre=pre, want_dx=want_dx, want_dw=want_dw, want_dbias=want_dbias, workspace=workspace))
    dev = _device(x, "x")
    code, T, N, K, a, ldx, ldw = _linear_args(dev, x, w, act)
    bf = torch.bfloat16
    lddy = _rows(dy, "dy", dev, (T, N), bf)
    dx, p0 = _empty_for(x if want_dx else None, (T, K))
    dw, p1 = _empty_for(w if want_dw else None, (N, K))
    dbias, p2 = _empty_for(w if want_dbias else None, N)
    if workspace is None:
        workspace = torch.empty(linear_workspace_bytes(T, N, K), dtype=torch.uint8, device=x.device)
    else:
        _check_workspace(workspace, dev)
    d = LinearDesc(code, T, N, K, a, ldx, ldw, 0, x.data_ptr(), w.data_ptr())
    status = lib().lx_linear_backward(d, dy.data_ptr(), lddy, _flat(pre, "pre", dev, T * N, bf), p0, p1, p2,
                                      workspace.data_ptr(), workspace.nbytes, _raw_stream(dev))
    if status:
        _check(status)
    return LinearGrads(dx, dw, dbias)


class HeadLoss(NamedTuple):
    """What head_loss computes: loss fp32 [T], and the gradients of its sum (None where not
    asked for)."""
    loss: torch.Tensor
    dh: Optional[torch.Tensor]
    dw: Optional[torch.Tensor]


def head_loss_workspace_bytes(T: int, V: int, H: int, want_dh: bool = True, want_dw: bool = True) -> int:
    b = ctypes.c_uint64()
    _check(lib().lx_head_loss_workspace(T, V, H, int(want_dh), int(want_dw), b))
    return b.value


def head_loss(h: torch.Tensor, w: torch.Tensor, labels: torch.Tensor, *, row_weight=None, want_dh: bool = True,
              want_dw: bool = True, workspace=None, stream=None) -> HeadLoss:
    """Softmax cross-entropy of the logits h w^T against int32 labels [T], of the last hidden states
    h [T, H] and the head's weights w [V, H] (bf16), without a [T, V] array of logits (for gradients they
    are kept, in the workspace, where they take up to 256 MiB):

        loss = row_weight * (logsumexp(h w^T) - (h w^T)[label])

    with the gradients of its sum.  A token whose label is outside [0, V) or whose weight is
    0 takes no part (loss and gradient 0, its hidden state not used) and costs no products."""
    if stream is not None:
        return _elsewhere(stream, head_loss, (h, w, labels), dict(
            row_weight=row_weight, want_dh=want_dh, want_dw=want_dw, workspace=workspace))
    dev = _device(h, "h")
    if h.dtype != torch.bfloat16:
        raise ValueError("h must be bf16")
    ldh = _rows(h, "h", dev)
    T, H = h.shape
    ldw = _rows(w, "w", dev, None, torch.bfloat16)
    V = w.shape[0]
    if w.shape[1] != H:
        raise ValueError(f"w must be [V, {H}]")
    lp, rp = _flat(labels, "labels", dev, T, torch.int32), _flat(row_weight, "row_weight", dev, T)
    loss = torch.empty(T, dtype=torch.float32, device=h.device)
    dh, p0 = _empty_for(h if want_dh else None, (T, H))
    dw, p1 = _empty_for(w if want_dw else None, (V, H))
    if workspace is None:
        workspace = torch.empty(head_loss_workspace_bytes(T, V, H, want_dh, want_dw), dtype=torch.uint8,
                                device=h.device)
    else:
        _check_workspace(workspace, dev)
    status = lib().lx_head_loss(h.data_ptr(), ldh, w.data_ptr(), ldw, lp, rp, T, V, H, loss.data_ptr(), p0, p1,
                                workspace.data_ptr(), workspace.nbytes, _raw_stream(dev))
    if status:
        _check(status)
    return HeadLoss(loss, dh, dw)
