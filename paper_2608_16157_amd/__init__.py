"""Python binding of libftmoe: the MoE layer executed against a GPU expert cache on gfx950.

Argument marshalling only.  Every step of the layer runs in the HIP kernels of
``libftmoe.so``; torch provides device memory and streams.  The entry points keep the names
of the C ABI declared in ``include/ftmoe.h``:

    ft_moe_workspace_bytes(desc, max_tokens) -> int
    ft_route_only(desc, logits, slot_table, T, route, ws, stream=None)
    ft_moe_forward(desc, banks, logits, slot_table, x, T, out_partial, route, ws, stream=None)
    ft_moe_forward_profiled(desc, banks, logits, slot_table, x, T, out_partial, route, ws,
                            events, stream=None)
    ft_moe_forward_noalloc(desc, banks, logits, slot_table, x, T, out_partial, route, stream=None)
    ft_miss_list_to_host(desc, route, T, host, stream=None)
    ft_cache_plan(desc, route, T, slot_table, state, policy, plan, stream=None)
    ft_cpu_pool_create(n_threads=0, pin=True) -> CpuPool;  ft_cpu_pool_destroy(pool)
    ft_cpu_experts(desc, host_pool, x, T, topk_ids, topk_w, experts, out, pool=None)
    ft_cache_fill(desc, host_pool, dev_banks, plan, max_fill, stream=None)
    ft_moe_step_hybrid(desc, dev_banks, host_pool, logits, slot_table, state, b_pcie, b_host,
                       max_fill, step, x, T, out, route, plan, host, ws, pool, stream=None)
    ft_prefill_layers(desc, host_layers, dev_bufs, slot_table, logits, x, T, out, route, ws,
                      overlap=True, stream=None, copy_stream=None)
    ft_act_quantize(x, T, C, row=None, col=None, stream=None)
    ft_linear_workspace_bytes(desc, max_tokens) -> int
    ft_linear(desc, weight, x, T, y, ws=None, stream=None)
    ft_linear_transpose(out_features, in_features, weight, weight_t, stream=None)
    ft_linear_weight_grad(out_features, in_features, T, dy_col, x_col, dw, accumulate=False, stream=None)
    ft_swiglu_quantize(gu, T, inter, h, saved=None, stream=None)
    ft_swiglu_backward(saved, dh, T, inter, dgu_row=None, dgu_col=None, h_col=None, stream=None)
    ft_balance_workspace_bytes(desc, max_tokens) -> int
    ft_balance_loss(desc, logits, topk_ids, T, out, ws, seq_off=None, mask=None, stream=None)
    ft_router_backward(desc, logits, topk_ids, T, balance, d_loss, d_logits, topk_w=None, d_topk_w=None,
                       seq_off=None, mask=None, stream=None)
    ft_expert_sort_rows(desc, T) -> int;  ft_expert_sort_workspace_bytes(desc, max_tokens) -> int
    ft_expert_sort(desc, topk_ids, T, out, ws, mask=None, stream=None)
    ft_expert_gather(desc, sort, x, T, C, weights=None, rows=None, row=None, col=None, stream=None)
    ft_expert_combine(desc, sort, rows, T, C, y, weights=None, base=None, stream=None)
    ft_expert_gate_grad(desc, sort, rows, dy, T, C, d_weights, stream=None)
    ft_expert_linear(desc, linear, weight, x, sort, T, y, stream=None)
    ft_expert_linear_transpose(n, out_features, in_features, weight, weight_t, stream=None)
    ft_expert_weight_grad(desc, out_features, in_features, dy_col, x_col, sort, T, dw, accumulate=False, stream=None)
    ft_block_norm(desc, params, x, block, T, r=None, n=None, n_row=None, stream=None)
    ft_block_norm_workspace_bytes(desc, max_tokens) -> int
    ft_block_norm_backward(desc, params, r, block, dr, dn, T, dx=None, d_block=None, grads=None, ws=None, stream=None)
    ft_status_string(status) -> str

``desc`` is a dict with the ft_moe_desc_t fields; ``route`` a RouteBuffers; ``banks`` a dict
with w13, w2 (and s13, s2 for fp8) device tensors; a ``weight`` of the dense product a dict with w and
s; 8-bit forms ActCodes; ``ft_balance_loss``'s outputs a BalanceBuffers; the ``desc`` of the ft_expert calls a dict
with the ft_sort_desc_t fields and ``sort`` a SortBuffers; the ``desc`` of the norms one with the ft_norm_desc_t
fields, ``params`` and ``grads`` dicts of pre, post, gate and token_gate; everything else device tensors.  A non-OK status raises FtError.  If the library is not built, importing works but every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libftmoe.so")

FT_OK, FT_ERR_NULL, FT_ERR_SHAPE, FT_ERR_DTYPE, FT_ERR_CAPACITY, FT_ERR_HIP = range(6)
FT_GATE_SOFTMAX_TOPK_RENORM, FT_GATE_SIGMOID_TOPK_RENORM = 0, 1
FT_COMBINE_ORDERED, FT_COMBINE_ATOMIC = 0, 1
FT_ACT_EXACT, FT_ACT_FP8_1x128_POW2 = 0, 1
FT_DT_F32, FT_DT_BF16, FT_DT_FP8E4M3FN_B128, FT_DT_MXFP4, FT_DT_FP8_ACT = 0, 1, 2, 3, 4
FT_SLOT_MISS = -1
FT_DEV_SLOT_RANGE, FT_DEV_SLOT_DUP, FT_DEV_SLOT_SHARED = 1, 2, 4

EXPORTED = ("ft_moe_workspace_bytes", "ft_route_only", "ft_moe_forward", "ft_moe_forward_noalloc",
            "ft_moe_forward_profiled", "ft_miss_list_to_host", "ft_cache_plan", "ft_cpu_experts",
            "ft_cache_fill", "ft_moe_step_hybrid", "ft_prefill_layers", "ft_status_string",
            "ft_cpu_pool_create", "ft_cpu_pool_destroy", "ft_act_quantize", "ft_linear_workspace_bytes",
            "ft_linear", "ft_linear_transpose", "ft_linear_weight_grad", "ft_swiglu_quantize",
            "ft_swiglu_backward", "ft_balance_workspace_bytes", "ft_balance_loss", "ft_router_backward",
            "ft_expert_sort_rows", "ft_expert_sort_workspace_bytes", "ft_expert_sort", "ft_expert_gather",
            "ft_expert_combine", "ft_expert_gate_grad", "ft_expert_linear", "ft_expert_linear_transpose",
            "ft_expert_weight_grad", "ft_block_norm", "ft_block_norm_workspace_bytes", "ft_block_norm_backward")
FT_PROF_STAGES = 4
FT_NOALLOC_SCRATCH_BYTES = 64 << 20


class FtError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {_status_text(status)}")


class ft_moe_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("hidden", "inter", "n_experts", "top_k", "gating",
                                              "w_dtype", "x_dtype", "n_slots", "shared_slot",
                                              "combine", "act_quant")]


class ft_banks_t(ctypes.Structure):
    _fields_ = [("w13", ctypes.c_void_p), ("w2", ctypes.c_void_p), ("s13", ctypes.c_void_p),
                ("s2", ctypes.c_void_p)]


class ft_route_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("topk_ids", "topk_w", "topk_slot", "hit_pairs",
                                               "miss_pairs", "hit_off", "miss_off", "counts")]


class ft_prof_events_t(ctypes.Structure):
    _fields_ = [("ev", ctypes.c_void_p * 5)]


class ft_host_miss_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("counts", "miss_pairs", "miss_off", "topk_ids",
                                               "topk_w")]


class ft_cache_state_t(ctypes.Structure):
    _fields_ = [("slot_expert", ctypes.c_void_p), ("slot_stamp", ctypes.c_void_p),
                ("clock", ctypes.c_void_p)]


class ft_cache_policy_t(ctypes.Structure):
    _fields_ = [("b_pcie", ctypes.c_double), ("b_host", ctypes.c_double),
                ("max_fill", ctypes.c_int32), ("step", ctypes.c_uint32)]


class ft_fill_plan_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("fill_expert", "fill_slot", "evict_expert",
                                               "cpu_expert", "counts")]


class ft_hybrid_host_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("plan_counts", "cpu_expert", "topk_ids", "topk_w", "x",
                                               "cpu_out", "task")]


FT_HYBRID_TASK_BYTES = 24 * 8


class ft_act_codes_t(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


class ft_linear_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("out_features", "in_features", "x_dtype", "y_dtype")]


class ft_balance_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_experts", "top_k", "gating", "n_seq")] + \
               [("coef", ctypes.c_float)]


class ft_balance_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("counts", "tokens", "prob", "frac", "loss")]


class ft_sort_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_experts", "top_k", "first", "local", "align", "rows")]


class ft_sort_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("row_pair", "pair_row", "off", "count", "dropped")]


class ft_norm_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("channels", "x_dtype", "y_dtype", "w_dtype", "post_norm")] + \
               [("eps", ctypes.c_float), ("scale", ctypes.c_float)]


class ft_norm_params_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("pre", "post", "gate", "token_gate")]


class ft_norm_grads_t(ctypes.Structure):
    _fields_ = ft_norm_params_t._fields_


_lib: Optional[ctypes.CDLL] = None


def load(path: str = None) -> ctypes.CDLL:
    """Load libftmoe.so once (FTMOE_LIBRARY may name another build); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or os.environ.get("FTMOE_LIBRARY") or LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"libftmoe.so not built ({path}); run __graft_entry__.build() or "
                           "python paper_2608_16157_amd/build.py")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    lib.ft_moe_workspace_bytes.restype = ctypes.c_size_t
    lib.ft_moe_workspace_bytes.argtypes = [P(ft_moe_desc_t), ctypes.c_int32]
    lib.ft_route_only.restype = ctypes.c_int
    lib.ft_route_only.argtypes = [P(ft_moe_desc_t), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                  P(ft_route_t), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    lib.ft_moe_forward.restype = ctypes.c_int
    lib.ft_moe_forward.argtypes = [P(ft_moe_desc_t), P(ft_banks_t), ctypes.c_void_p, ctypes.c_void_p,
                                   ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, P(ft_route_t),
                                   ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    lib.ft_moe_forward_noalloc.restype = ctypes.c_int
    lib.ft_moe_forward_noalloc.argtypes = [P(ft_moe_desc_t), P(ft_banks_t), ctypes.c_void_p,
                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                           ctypes.c_void_p, P(ft_route_t), ctypes.c_void_p]
    lib.ft_moe_forward_profiled.restype = ctypes.c_int
    lib.ft_moe_forward_profiled.argtypes = lib.ft_moe_forward.argtypes + [P(ft_prof_events_t)]
    lib.ft_miss_list_to_host.restype = ctypes.c_int
    lib.ft_miss_list_to_host.argtypes = [P(ft_moe_desc_t), P(ft_route_t), ctypes.c_int32,
                                         P(ft_host_miss_t), ctypes.c_void_p]
    lib.ft_cache_plan.restype = ctypes.c_int
    lib.ft_cache_plan.argtypes = [P(ft_moe_desc_t), P(ft_route_t), ctypes.c_int32, ctypes.c_void_p,
                                  P(ft_cache_state_t), P(ft_cache_policy_t), P(ft_fill_plan_t),
                                  ctypes.c_void_p]
    lib.ft_cpu_pool_create.restype = ctypes.c_void_p
    lib.ft_cpu_pool_create.argtypes = [ctypes.c_int32, ctypes.c_int32]
    lib.ft_cpu_pool_destroy.restype = None
    lib.ft_cpu_pool_destroy.argtypes = [ctypes.c_void_p]
    lib.ft_cpu_experts.restype = ctypes.c_int
    lib.ft_cpu_experts.argtypes = [P(ft_moe_desc_t), P(ft_banks_t), ctypes.c_void_p, ctypes.c_int32,
                                   ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                   ctypes.c_void_p, ctypes.c_void_p]
    lib.ft_cache_fill.restype = ctypes.c_int
    lib.ft_cache_fill.argtypes = [P(ft_moe_desc_t), P(ft_banks_t), P(ft_banks_t), P(ft_fill_plan_t),
                                  ctypes.c_int32, ctypes.c_void_p]
    lib.ft_moe_step_hybrid.restype = ctypes.c_int
    lib.ft_moe_step_hybrid.argtypes = [P(ft_moe_desc_t), P(ft_banks_t), P(ft_banks_t), ctypes.c_void_p,
                                       ctypes.c_void_p, P(ft_cache_state_t), P(ft_cache_policy_t),
                                       ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p,
                                       P(ft_route_t), P(ft_fill_plan_t), P(ft_hybrid_host_t),
                                       ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]
    lib.ft_prefill_layers.restype = ctypes.c_int
    lib.ft_prefill_layers.argtypes = [P(ft_moe_desc_t), ctypes.c_int32, P(ft_banks_t), P(ft_banks_t),
                                      ctypes.c_void_p, P(ctypes.c_void_p), P(ctypes.c_void_p),
                                      ctypes.c_int32, P(ctypes.c_void_p), P(ft_route_t), ctypes.c_void_p,
                                      ctypes.c_size_t, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
    p, i, z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    codes, bal = P(ft_act_codes_t), P(ft_balance_t)
    lib.ft_act_quantize.restype = ctypes.c_int
    lib.ft_act_quantize.argtypes = [p, i, i, i, codes, codes, p]
    lib.ft_linear_workspace_bytes.restype = z
    lib.ft_linear_workspace_bytes.argtypes = [P(ft_linear_desc_t), i]
    lib.ft_linear.restype = ctypes.c_int
    lib.ft_linear.argtypes = [P(ft_linear_desc_t), p, p, p, p, i, p, p, z, p]
    lib.ft_linear_transpose.restype = ctypes.c_int
    lib.ft_linear_transpose.argtypes = [i, i, p, p, p, p, p]
    lib.ft_linear_weight_grad.restype = ctypes.c_int
    lib.ft_linear_weight_grad.argtypes = [i, i, i, codes, codes, p, i, i, p]
    lib.ft_swiglu_quantize.restype = ctypes.c_int
    lib.ft_swiglu_quantize.argtypes = [p, i, i, i, codes, codes, p]
    lib.ft_swiglu_backward.restype = ctypes.c_int
    lib.ft_swiglu_backward.argtypes = [codes, p, i, i, i, codes, codes, codes, p]
    lib.ft_balance_workspace_bytes.restype = z
    lib.ft_balance_workspace_bytes.argtypes = [P(ft_balance_desc_t), i]
    lib.ft_balance_loss.restype = ctypes.c_int
    lib.ft_balance_loss.argtypes = [P(ft_balance_desc_t), p, p, i, p, p, bal, p, z, p]
    lib.ft_router_backward.restype = ctypes.c_int
    lib.ft_router_backward.argtypes = [P(ft_balance_desc_t), p, p, i, p, p, bal, p, p, p, p, p]
    sd, st, ld, nd = P(ft_sort_desc_t), P(ft_sort_t), P(ft_linear_desc_t), P(ft_norm_desc_t)
    lib.ft_expert_sort_rows.restype = i
    lib.ft_expert_sort_rows.argtypes = [sd, i]
    lib.ft_expert_sort_workspace_bytes.restype = z
    lib.ft_expert_sort_workspace_bytes.argtypes = [sd, i]
    lib.ft_block_norm_workspace_bytes.restype = z
    lib.ft_block_norm_workspace_bytes.argtypes = [nd, i]
    for name, args in (("ft_expert_sort", [sd, p, i, p, st, p, z, p]),
                       ("ft_expert_gather", [sd, st, p, i, i, i, p, p, i, codes, codes, p]),
                       ("ft_expert_combine", [sd, st, p, i, i, i, p, p, p, i, p]),
                       ("ft_expert_gate_grad", [sd, st, p, i, p, i, i, i, p, p]),
                       ("ft_expert_linear", [sd, ld, p, p, codes, st, i, p, p]),
                       ("ft_expert_linear_transpose", [i, i, i, p, p, p, p, p]),
                       ("ft_expert_weight_grad", [sd, i, i, codes, codes, st, i, p, i, i, p]),
                       ("ft_block_norm", [nd, P(ft_norm_params_t), p, p, i, p, p, codes, p]),
                       ("ft_block_norm_backward", [nd, P(ft_norm_params_t), p, p, p, p, i, p, p, P(ft_norm_grads_t), p, z, p])):
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = args
    lib.ft_status_string.restype = ctypes.c_char_p
    lib.ft_status_string.argtypes = [ctypes.c_int]
    _lib = lib
    return lib


def _status_text(status: int) -> str:
    try:
        return load().ft_status_string(status).decode()
    except RuntimeError:
        return f"status {status}"


def ft_status_string(status: int) -> str:
    return load().ft_status_string(status).decode()


# ------------------------------------------------------------------------------ marshalling

def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libftmoe must be contiguous")
    return t.data_ptr()


# ------------------------------------------------------------------------------ validation
# The C ABI carries device pointers without capacities, so every wrapper checks the tensors it
# passes (device, dtype, element count) against the sizes the call will touch, and raises
# ValueError before the library is entered.

_X_DTYPES = {FT_DT_F32: torch.float32, FT_DT_BF16: torch.bfloat16}
_W_DTYPES = {FT_DT_F32: (torch.float32,), FT_DT_BF16: (torch.bfloat16, torch.int16),
             FT_DT_FP8E4M3FN_B128: (torch.uint8, torch.float8_e4m3fn), FT_DT_MXFP4: (torch.uint8,)}
_S_DTYPES = {FT_DT_FP8E4M3FN_B128: (torch.float32,), FT_DT_MXFP4: (torch.uint8,)}


def expert_bank_bytes(desc: dict) -> tuple:
    """Bytes of one expert in each bank (w13, w2, s13, s2) for the layout of ``desc``."""
    H, I, wd = int(desc["hidden"]), int(desc["inter"]), int(desc["w_dtype"])
    if wd == FT_DT_F32:
        return 8 * I * H, 4 * H * I, 0, 0
    if wd == FT_DT_BF16:
        return 4 * I * H, 2 * H * I, 0, 0
    if wd == FT_DT_FP8E4M3FN_B128:
        return 2 * I * H, H * I, (2 * I // 128) * (H // 128) * 4, (H // 128) * (I // 128) * 4
    return I * H, H * I // 2, 2 * I * (H // 32), H * (I // 32)


def _need(t, name: str, dtypes, numel: int, device: str = "cuda") -> None:
    """Raise ValueError unless ``t`` is a tensor on ``device`` of one of ``dtypes`` holding at
    least ``numel`` elements."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if device == "cuda" and not t.is_cuda:
        raise ValueError(f"{name}: must be a device (cuda) tensor")
    if device == "cpu" and t.is_cuda:
        raise ValueError(f"{name}: must be a host tensor")
    if not isinstance(dtypes, tuple):
        dtypes = (dtypes,)
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    if t.numel() < numel:
        raise ValueError(f"{name}: {t.numel()} elements, the call needs {numel}")


def _need_bytes(t, name: str, dtypes, nbytes: int, device: str = "cuda") -> None:
    _need(t, name, dtypes, 0, device)
    if t.numel() * t.element_size() < nbytes:
        raise ValueError(f"{name}: {t.numel() * t.element_size()} bytes, the call needs {nbytes}")


def _need_banks(desc: dict, banks: dict, rows: int, name: str, device: str = "cuda") -> None:
    """Every bank holds ``rows`` expert rows of the layout of ``desc``."""
    if rows <= 0:
        return
    wd = int(desc["w_dtype"])
    b13, b2, bs13, bs2 = expert_bank_bytes(desc)
    _need_bytes(banks.get("w13"), f"{name}['w13']", _W_DTYPES[wd], rows * b13, device)
    _need_bytes(banks.get("w2"), f"{name}['w2']", _W_DTYPES[wd], rows * b2, device)
    if wd in _S_DTYPES:
        _need_bytes(banks.get("s13"), f"{name}['s13']", _S_DTYPES[wd], rows * bs13, device)
        _need_bytes(banks.get("s2"), f"{name}['s2']", _S_DTYPES[wd], rows * bs2, device)


def _need_route(route, desc: dict, T: int) -> None:
    if not isinstance(route, RouteBuffers):
        raise ValueError("route: expected a RouteBuffers")
    E, k = int(desc["n_experts"]), int(desc["top_k"])
    if route.E != E or route.k != k or route.T < T:
        raise ValueError(f"route: sized for T={route.T}, k={route.k}, E={route.E}; the call needs "
                         f"T={T}, k={k}, E={E}")


def _need_layer_inputs(desc: dict, logits, slot_table, T: int, x=None, out=None) -> None:
    E, H = int(desc["n_experts"]), int(desc["hidden"])
    _need(logits, "logits", torch.float32, T * E)
    _need(slot_table, "slot_table", torch.int32, E)
    if x is not None or out is not None:
        xd = _X_DTYPES.get(int(desc["x_dtype"]))
        if xd is None:
            raise ValueError(f"x_dtype {desc['x_dtype']} is not supported")
        _need(x, "x", xd, T * H)
        _need(out, "out_partial", torch.float32, T * H)


def _stream(stream) -> Optional[int]:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_desc(d: dict) -> ft_moe_desc_t:
    """ft_moe_desc_t from a dict; ``combine`` defaults to FT_COMBINE_ORDERED and ``act_quant`` to
    FT_ACT_EXACT."""
    return ft_moe_desc_t(**{f: int(d.get(f, 0) if f in ("combine", "act_quant") else d[f])
                            for f, _ in ft_moe_desc_t._fields_})


class RouteBuffers:
    """Device tensors behind one ft_route_t, sized for T tokens."""

    def __init__(self, T: int, top_k: int, n_experts: int, device="cuda"):
        pk = max(T * top_k, 1)
        i32 = dict(dtype=torch.int32, device=device)
        self.T, self.k, self.E = T, top_k, n_experts
        self.topk_ids = torch.empty(pk, **i32)
        self.topk_w = torch.empty(pk, dtype=torch.float32, device=device)
        self.topk_slot = torch.empty(pk, **i32)
        self.hit_pairs = torch.empty(pk, **i32)
        self.miss_pairs = torch.empty(pk, **i32)
        self.hit_off = torch.empty(n_experts + 1, **i32)
        self.miss_off = torch.empty(n_experts + 1, **i32)
        self.counts = torch.empty(4, **i32)

    def c(self) -> ft_route_t:
        return ft_route_t(*[_ptr(getattr(self, n)) for n, _ in ft_route_t._fields_])


class HostMissBuffers:
    """Pinned host buffers behind one ft_host_miss_t."""

    def __init__(self, T: int, top_k: int, n_experts: int):
        pk = max(T * top_k, 1)
        kw = dict(pin_memory=True)
        self.counts = torch.empty(4, dtype=torch.int32, **kw)
        self.miss_pairs = torch.empty(pk, dtype=torch.int32, **kw)
        self.miss_off = torch.empty(n_experts + 1, dtype=torch.int32, **kw)
        self.topk_ids = torch.empty(pk, dtype=torch.int32, **kw)
        self.topk_w = torch.empty(pk, dtype=torch.float32, **kw)

    def c(self) -> ft_host_miss_t:
        return ft_host_miss_t(*[_ptr(getattr(self, n)) for n, _ in ft_host_miss_t._fields_])


def _check(status: int, where: str):
    if status != FT_OK:
        raise FtError(status, where)


def ft_moe_workspace_bytes(desc: dict, max_tokens: int) -> int:
    return int(load().ft_moe_workspace_bytes(ctypes.byref(make_desc(desc)), int(max_tokens)))


def alloc_workspace(desc: dict, max_tokens: int, device="cuda") -> torch.Tensor:
    n = ft_moe_workspace_bytes(desc, max_tokens)
    if n == 0:
        raise FtError(FT_ERR_SHAPE, "ft_moe_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def ft_route_only(desc: dict, logits: torch.Tensor, slot_table: torch.Tensor, T: int,
                  route: RouteBuffers, ws: torch.Tensor, stream=None) -> None:
    _need_layer_inputs(desc, logits, slot_table, T)
    _need_route(route, desc, T)
    _need(ws, "ws", torch.uint8, 0)
    st = load().ft_route_only(ctypes.byref(make_desc(desc)), _ptr(logits), _ptr(slot_table), int(T),
                              ctypes.byref(route.c()), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "ft_route_only")


def _need_forward(desc, banks, logits, slot_table, x, T, out_partial, route, ws) -> None:
    if int(T) <= 0:
        return
    _need_layer_inputs(desc, logits, slot_table, T, x, out_partial)
    _need_route(route, desc, T)
    _need(ws, "ws", torch.uint8, 0)
    _need_banks(desc, banks, int(desc["n_slots"]), "banks")


def ft_moe_forward(desc: dict, banks: dict, logits: torch.Tensor, slot_table: torch.Tensor,
                   x: torch.Tensor, T: int, out_partial: torch.Tensor, route: RouteBuffers,
                   ws: torch.Tensor, stream=None) -> None:
    _need_forward(desc, banks, logits, slot_table, x, T, out_partial, route, ws)
    b = ft_banks_t(_ptr(banks.get("w13")), _ptr(banks.get("w2")), _ptr(banks.get("s13")),
                   _ptr(banks.get("s2")))
    st = load().ft_moe_forward(ctypes.byref(make_desc(desc)), ctypes.byref(b), _ptr(logits),
                               _ptr(slot_table), _ptr(x), int(T), _ptr(out_partial),
                               ctypes.byref(route.c()), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "ft_moe_forward")


def ft_moe_forward_noalloc(desc: dict, banks: dict, logits: torch.Tensor, slot_table: torch.Tensor,
                           x: torch.Tensor, T: int, out_partial: torch.Tensor, route: RouteBuffers,
                           stream=None) -> None:
    """ft_moe_forward on the library's own device scratch array (no workspace argument)."""
    if int(T) > 0:
        _need_layer_inputs(desc, logits, slot_table, T, x, out_partial)
        _need_route(route, desc, T)
        _need_banks(desc, banks, int(desc["n_slots"]), "banks")
    b = ft_banks_t(_ptr(banks.get("w13")), _ptr(banks.get("w2")), _ptr(banks.get("s13")),
                   _ptr(banks.get("s2")))
    st = load().ft_moe_forward_noalloc(ctypes.byref(make_desc(desc)), ctypes.byref(b), _ptr(logits),
                                       _ptr(slot_table), _ptr(x), int(T), _ptr(out_partial),
                                       ctypes.byref(route.c()), _stream(stream))
    _check(st, "ft_moe_forward_noalloc")


def ft_moe_forward_profiled(desc: dict, banks: dict, logits: torch.Tensor, slot_table: torch.Tensor,
                            x: torch.Tensor, T: int, out_partial: torch.Tensor, route: RouteBuffers,
                            ws: torch.Tensor, events, stream=None) -> None:
    """``events``: FT_PROF_STAGES + 1 hipEvent_t handles (ints) or None entries."""
    _need_forward(desc, banks, logits, slot_table, x, T, out_partial, route, ws)
    b = ft_banks_t(_ptr(banks.get("w13")), _ptr(banks.get("w2")), _ptr(banks.get("s13")),
                   _ptr(banks.get("s2")))
    ev = ft_prof_events_t()
    for i, e in enumerate(events):
        ev.ev[i] = e
    st = load().ft_moe_forward_profiled(ctypes.byref(make_desc(desc)), ctypes.byref(b), _ptr(logits),
                                        _ptr(slot_table), _ptr(x), int(T), _ptr(out_partial),
                                        ctypes.byref(route.c()), _ptr(ws), ws.numel(),
                                        _stream(stream), ctypes.byref(ev))
    _check(st, "ft_moe_forward_profiled")


def ft_miss_list_to_host(desc: dict, route: RouteBuffers, T: int, host: HostMissBuffers,
                         stream=None) -> None:
    _need_route(route, desc, T)
    pk, E = int(T) * int(desc["top_k"]), int(desc["n_experts"])
    for n, dt, cnt in (("counts", torch.int32, 4), ("miss_pairs", torch.int32, pk),
                       ("miss_off", torch.int32, E + 1), ("topk_ids", torch.int32, pk),
                       ("topk_w", torch.float32, pk)):
        _need(getattr(host, n, None), f"host.{n}", dt, cnt, "cpu")
    st = load().ft_miss_list_to_host(ctypes.byref(make_desc(desc)), ctypes.byref(route.c()), int(T),
                                     ctypes.byref(host.c()), _stream(stream))
    _check(st, "ft_miss_list_to_host")


class CacheState:
    """Device tensors behind one ft_cache_state_t: slot -> expert (-1 empty), the slot stamps
    (uint32 in the ABI; held as int32 here, stamps stay below 2**31) and an optional one-element
    device step clock."""

    def __init__(self, slot_expert: torch.Tensor, slot_stamp: torch.Tensor,
                 clock: Optional[torch.Tensor] = None):
        self.slot_expert = slot_expert
        self.slot_stamp = slot_stamp
        self.clock = clock

    def c(self) -> ft_cache_state_t:
        return ft_cache_state_t(_ptr(self.slot_expert), _ptr(self.slot_stamp), _ptr(self.clock))


class FillPlanBuffers:
    """Device tensors behind one ft_fill_plan_t (max_fill fills, n_experts CPU entries)."""

    def __init__(self, max_fill: int, n_experts: int, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.fill_expert = torch.empty(max_fill, **i32)
        self.fill_slot = torch.empty(max_fill, **i32)
        self.evict_expert = torch.empty(max_fill, **i32)
        self.cpu_expert = torch.empty(max(n_experts, 1), **i32)
        self.counts = torch.empty(4, **i32)

    def c(self) -> ft_fill_plan_t:
        return ft_fill_plan_t(*[_ptr(getattr(self, n)) for n, _ in ft_fill_plan_t._fields_])


def _need_plan(desc: dict, slot_table, state, plan, max_fill: int) -> None:
    E, S = int(desc["n_experts"]), int(desc["n_slots"])
    _need(slot_table, "slot_table", torch.int32, E)
    _need(state.slot_expert, "state.slot_expert", torch.int32, S)
    _need(state.slot_stamp, "state.slot_stamp", (torch.int32, torch.uint32), S)
    for n in ("fill_expert", "fill_slot", "evict_expert"):
        _need(getattr(plan, n), f"plan.{n}", torch.int32, int(max_fill))
    _need(plan.cpu_expert, "plan.cpu_expert", torch.int32, E)
    _need(plan.counts, "plan.counts", torch.int32, 4)


def ft_cache_plan(desc: dict, route: RouteBuffers, T: int, slot_table: torch.Tensor,
                  state: CacheState, b_pcie: float, b_host: float, max_fill: int, step: int,
                  plan: FillPlanBuffers, stream=None) -> None:
    _need_route(route, desc, T)
    _need_plan(desc, slot_table, state, plan, max_fill)
    pol = ft_cache_policy_t(float(b_pcie), float(b_host), int(max_fill), int(step))
    st = load().ft_cache_plan(ctypes.byref(make_desc(desc)), ctypes.byref(route.c()), int(T),
                              _ptr(slot_table), ctypes.byref(state.c()), ctypes.byref(pol),
                              ctypes.byref(plan.c()), _stream(stream))
    _check(st, "ft_cache_plan")


class CpuPool:
    """A persistent CPU worker pool (ft_cpu_pool_t); destroyed with ft_cpu_pool_destroy or when
    garbage-collected."""

    def __init__(self, handle: int, n_threads: int, pin: bool):
        self.handle, self.n_threads, self.pin = handle, n_threads, pin

    def close(self) -> None:
        if self.handle:
            load().ft_cpu_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def ft_cpu_pool_create(n_threads: int = 0, pin: bool = True) -> CpuPool:
    h = load().ft_cpu_pool_create(int(n_threads), 1 if pin else 0)
    if not h:
        raise RuntimeError("ft_cpu_pool_create failed")
    return CpuPool(h, n_threads, pin)


def ft_cpu_pool_destroy(pool: CpuPool) -> None:
    pool.close()


def _pool_handle(pool) -> Optional[int]:
    if pool is None:
        return None
    if not isinstance(pool, CpuPool) or not pool.handle:
        raise ValueError("pool: expected an open CpuPool or None")
    return pool.handle


def ft_cpu_experts(desc: dict, host_pool: dict, x: torch.Tensor, T: int, topk_ids: torch.Tensor,
                   topk_w: torch.Tensor, experts: torch.Tensor, out: torch.Tensor,
                   pool: Optional[CpuPool] = None) -> None:
    """CPU branch on host tensors: ``host_pool`` holds w13, w2 (s13, s2) indexed by expert id;
    runs on ``pool``'s workers, or on the calling thread without one."""
    if int(T) > 0:
        E, H, k = int(desc["n_experts"]), int(desc["hidden"]), int(desc["top_k"])
        xd = _X_DTYPES.get(int(desc["x_dtype"]))
        if xd is None:
            raise ValueError(f"x_dtype {desc['x_dtype']} is not supported")
        _need(x, "x", xd, int(T) * H, "cpu")
        _need(topk_ids, "topk_ids", torch.int32, int(T) * k, "cpu")
        _need(topk_w, "topk_w", torch.float32, int(T) * k, "cpu")
        _need(experts, "experts", torch.int32, 0, "cpu")
        _need(out, "out", torch.float32, int(T) * H, "cpu")
        if experts.numel() > 0:
            _need_banks(desc, host_pool, E, "host_pool", "cpu")
    b = ft_banks_t(_ptr(host_pool.get("w13")), _ptr(host_pool.get("w2")), _ptr(host_pool.get("s13")),
                   _ptr(host_pool.get("s2")))
    st = load().ft_cpu_experts(ctypes.byref(make_desc(desc)), ctypes.byref(b), _ptr(x), int(T),
                               _ptr(topk_ids), _ptr(topk_w), _ptr(experts), int(experts.numel()),
                               _ptr(out), _pool_handle(pool))
    _check(st, "ft_cpu_experts")


def _banks(b: dict) -> ft_banks_t:
    return ft_banks_t(_ptr(b.get("w13")), _ptr(b.get("w2")), _ptr(b.get("s13")), _ptr(b.get("s2")))


def ft_cache_fill(desc: dict, host_pool: dict, dev_banks: dict, plan: FillPlanBuffers, max_fill: int,
                  stream=None) -> None:
    _need_banks(desc, host_pool, int(desc["n_experts"]), "host_pool", "cpu")
    _need_banks(desc, dev_banks, int(desc["n_slots"]), "dev_banks")
    for n in ("fill_expert", "fill_slot"):
        _need(getattr(plan, n), f"plan.{n}", torch.int32, int(max_fill))
    _need(plan.counts, "plan.counts", torch.int32, 4)
    st = load().ft_cache_fill(ctypes.byref(make_desc(desc)), ctypes.byref(_banks(host_pool)),
                              ctypes.byref(_banks(dev_banks)), ctypes.byref(plan.c()), int(max_fill),
                              _stream(stream))
    _check(st, "ft_cache_fill")


class HybridHostBuffers:
    """Pinned host staging behind one ft_hybrid_host_t, for T tokens."""

    def __init__(self, T: int, top_k: int, n_experts: int, hidden: int, x_dtype=torch.bfloat16):
        kw = dict(pin_memory=True)
        pk = max(T * top_k, 1)
        self.plan_counts = torch.empty(4, dtype=torch.int32, **kw)
        self.cpu_expert = torch.empty(n_experts, dtype=torch.int32, **kw)
        self.topk_ids = torch.empty(pk, dtype=torch.int32, **kw)
        self.topk_w = torch.empty(pk, dtype=torch.float32, **kw)
        self.x = torch.empty(max(T, 1), hidden, dtype=x_dtype, **kw)
        self.cpu_out = torch.empty(max(T, 1), hidden, dtype=torch.float32, **kw)
        self.task = torch.zeros(FT_HYBRID_TASK_BYTES, dtype=torch.uint8)   # plain host memory
        self.T, self.k, self.E, self.H = T, top_k, n_experts, hidden

    def c(self) -> ft_hybrid_host_t:
        return ft_hybrid_host_t(*[_ptr(getattr(self, n)) for n, _ in ft_hybrid_host_t._fields_])


def ft_moe_step_hybrid(desc: dict, dev_banks: dict, host_pool: dict, logits: torch.Tensor,
                       slot_table: torch.Tensor, state: CacheState, b_pcie: float, b_host: float,
                       max_fill: int, step: int, x: torch.Tensor, T: int, out: torch.Tensor,
                       route: RouteBuffers, plan: FillPlanBuffers,
                       host: HybridHostBuffers, ws: torch.Tensor, pool: Optional[CpuPool],
                       stream=None) -> None:
    """One complete hybrid layer step, enqueued on ``stream`` without waiting for the device."""
    if int(T) > 0:
        _need_layer_inputs(desc, logits, slot_table, T, x, out)
        _need_route(route, desc, T)
        _need(ws, "ws", torch.uint8, 0)
        _need_banks(desc, dev_banks, int(desc["n_slots"]), "dev_banks")
        _need_banks(desc, host_pool, int(desc["n_experts"]), "host_pool", "cpu")
        _need_plan(desc, slot_table, state, plan, max_fill)
        if host.T < T or host.k != int(desc["top_k"]) or host.E != int(desc["n_experts"]) or \
                host.H != int(desc["hidden"]):
            raise ValueError("host: HybridHostBuffers sized for another layer or fewer tokens")
        if state.clock is not None:
            _need(state.clock, "state.clock", (torch.int32, torch.uint32), 1)
    pol = ft_cache_policy_t(float(b_pcie), float(b_host), int(max_fill), int(step))
    st = load().ft_moe_step_hybrid(ctypes.byref(make_desc(desc)), ctypes.byref(_banks(dev_banks)),
                                   ctypes.byref(_banks(host_pool)), _ptr(logits), _ptr(slot_table),
                                   ctypes.byref(state.c()), ctypes.byref(pol), _ptr(x), int(T),
                                   _ptr(out), ctypes.byref(route.c()),
                                   ctypes.byref(plan.c()), ctypes.byref(host.c()), _ptr(ws),
                                   ws.numel(), _pool_handle(pool), _stream(stream))
    _check(st, "ft_moe_step_hybrid")


def banks_of(layer) -> dict:
    """The bank tensors of a synthetic layer object (w13, w2, s13, s2 attributes)."""
    return {"w13": layer.w13, "w2": layer.w2, "s13": layer.s13, "s2": layer.s2}


def ft_prefill_layers(desc: dict, host_layers: list, dev_bufs: list, slot_table: torch.Tensor,
                      logits: list, x: list, T: int, out: list, route: RouteBuffers, ws: torch.Tensor,
                      overlap: bool = True, stream=None, copy_stream=None) -> None:
    """``host_layers``: one dict of pinned host tensors (w13, w2, s13, s2) per layer;
    ``dev_bufs``: two dicts of device tensors; ``logits``, ``x``, ``out``: one device tensor per
    layer.  ``copy_stream``: a torch stream or raw handle, required when ``overlap``."""
    n = len(host_layers)
    if not (len(logits) == len(x) == len(out) == n) or len(dev_bufs) != 2:
        raise ValueError("one logits, x and out tensor per layer and two device buffers")
    if int(T) > 0:
        for l in range(n):
            _need_banks(desc, host_layers[l], int(desc["n_slots"]), f"host_layers[{l}]", "cpu")
            _need_layer_inputs(desc, logits[l], slot_table, T, x[l], out[l])
        for b in range(2):
            _need_banks(desc, dev_bufs[b], int(desc["n_slots"]), f"dev_bufs[{b}]")
        _need_route(route, desc, T)
        _need(ws, "ws", torch.uint8, 0)
    hl = (ft_banks_t * max(n, 1))(*[_banks(h) for h in host_layers])
    db = (ft_banks_t * 2)(*[_banks(d) for d in dev_bufs])
    arr = lambda ts: (ctypes.c_void_p * max(n, 1))(*[_ptr(t) for t in ts])
    cs = None if copy_stream is None else _stream(copy_stream)
    st = load().ft_prefill_layers(ctypes.byref(make_desc(desc)), n, hl, db, _ptr(slot_table),
                                  arr(logits), arr(x), int(T), arr(out), ctypes.byref(route.c()),
                                  _ptr(ws), ws.numel(), 1 if overlap else 0, _stream(stream), cs)
    _check(st, "ft_prefill_layers")


# ------------------------------------------------------------ dense layers next to the experts

_FLOATS = {torch.float32: FT_DT_F32, torch.bfloat16: FT_DT_BF16}
_FLOAT_TYPES = tuple(_FLOATS)
_CODES = (torch.uint8, torch.float8_e4m3fn)
_BYTES, _F32, _I32, _MASKS = (torch.uint8,), (torch.float32,), (torch.int32,), (torch.uint8, torch.bool)


def _pad128(n: int) -> int:
    return (n + 127) // 128 * 128


class ActCodes:
    """8-bit form of a matrix of ``rows`` x ``cols`` (ft_act_codes_t): ``codes`` uint8 [rows][Kp] and
    ``scales`` uint8 [Kp/128][Rp], Kp and Rp being cols and rows rounded up to multiples of 128.  The row
    form of x [T][C] is ActCodes(T, C), its column form ActCodes(C, T)."""

    def __init__(self, rows: int, cols: int, device="cuda"):
        kp = _pad128(cols)
        self.rows, self.cols = rows, cols
        self.codes = torch.empty(rows, kp, dtype=torch.uint8, device=device)
        self.scales = torch.empty(kp // 128, _pad128(rows), dtype=torch.uint8, device=device)

    @classmethod
    def of(cls, codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int) -> "ActCodes":
        """A form over existing tensors."""
        self = cls.__new__(cls)
        self.rows, self.cols, self.codes, self.scales = rows, cols, codes, scales
        return self


def _arg(dev: int, t, name: str, dtypes: tuple, numel: int):
    """The checks of _need, contiguity and one device for the whole call (``dev``: the one so far, -1 before the
    first), in one frame per tensor: at a call's few microseconds they count.  -> (device, address)."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.numel() < numel:
        _need(t, name, dtypes, numel)
    d = t.get_device()
    if d != dev or d < 0:
        if d < 0:
            raise ValueError(f"{name}: must be a device (cuda) tensor")
        if dev >= 0:
            raise ValueError(f"{name}: tensors on devices {dev} and {d}; a call works on one device")
    if not t.is_contiguous():
        raise ValueError("tensors passed to libftmoe must be contiguous")
    return d, t.data_ptr()


# a torch.cuda.Stream object costs a call more than its kernel's launch does
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on(device: int, call, *args) -> int:
    """``call(*args, stream)`` with ``device`` current; the last of ``args`` is the caller's stream or
    None for that device's current one."""
    stream = args[-1]
    stream = _raw_stream(device) if stream is None else _stream(stream)
    if device == _current_device():
        return call(*args[:-1], stream)
    with torch.cuda.device(device):
        return call(*args[:-1], stream)


def _need_codes(c, name: str, rows: int, cols: int, dev: int = -1):
    """The 8-bit form of a rows x cols matrix.  -> (device, address of codes, of scales)."""
    if not isinstance(c, ActCodes):
        raise ValueError(f"{name}: expected an ActCodes, got {type(c).__name__}")
    if c.rows != rows or c.cols != cols:
        raise ValueError(f"{name}: the form of a {c.rows} x {c.cols} matrix, the call needs {rows} x {cols}")
    kp = _pad128(cols)
    dev, codes = _arg(dev, c.codes, name + ".codes", _CODES, rows * kp)
    dev, scales = _arg(dev, c.scales, name + ".scales", _BYTES, kp // 128 * _pad128(rows))
    return dev, codes, scales


def _codes_arg(dev: int, c, name: str, rows: int, cols: int, optional: bool = False):
    """-> (device, the ft_act_codes_t to pass); None passes as NULL where the call may leave the form out."""
    if c is None and optional:
        return dev, None
    dev, codes, scales = _need_codes(c, name, rows, cols, dev)
    return dev, ctypes.byref(ft_act_codes_t(codes, scales))


def _in_rows(t: torch.Tensor, stream) -> torch.Tensor:
    """A copy of a strided 2-D tensor of bytes in rows.  The transpose of rows goes through the weight transpose where its
    sizes are ones of a weight: 7168 x 36864 in 112 us, 2048 x 28160 in 19, in 1032 and 259 by torch's copy, which moves single
    bytes.  Small ones wait for the host, which takes longer here: 1024 x 1024 12.7 us, 6.8 by torch's copy."""
    rows, kp = t.shape
    if t.is_cuda and t.numel() >= 1 << 22 and t.t().is_contiguous() and rows % 128 == 0 and kp % 128 == 0 and \
            max(rows, kp) <= 65536 and t.data_ptr() % 16 == 0:
        new = lambda *shape, dtype: torch.empty(*shape, dtype=dtype, device=t.device)
        out = new(rows, kp, dtype=torch.uint8)
        unused = {"s": new(kp // 128, rows // 128, dtype=torch.float32)}, {"s": new(rows // 128, kp // 128, dtype=torch.float32)}
        ft_linear_transpose(kp, rows, {"w": t.t(), **unused[0]}, {"w": out, **unused[1]}, stream)
        return out
    return t.contiguous()


def _laid_out(c, stream):
    """An input form whose tensors are strided views, as quantising a transposed matrix leaves them, in rows: a copy that
    lives on the call's stream.  Everything else goes on as it is, to be refused where it does not fit."""
    if not isinstance(c, ActCodes) or not all(isinstance(t, torch.Tensor) for t in (c.codes, c.scales)):
        return c
    if c.codes.is_contiguous() and c.scales.is_contiguous():
        return c
    kp = _pad128(c.cols)
    if c.codes.shape != (c.rows, kp) or c.scales.shape != (kp // 128, _pad128(c.rows)):
        return c
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, c.codes.device)
    with torch.cuda.stream(stream):   # None: no change
        rows = [t if t.is_contiguous() else _in_rows(t, stream) for t in (c.codes, c.scales)]
    return ActCodes.of(*rows, c.rows, c.cols)


def _need_sizes(T: int, *features: int) -> None:
    """Sizes the library refuses (FT_ERR_SHAPE) would make the element counts here meaningless."""
    if not 0 <= T <= 1048576 or any(not 16 <= f <= 65536 or f % 16 for f in features):
        raise FtError(FT_ERR_SHAPE, "sizes")


def ft_act_quantize(x: torch.Tensor, T: int, C: int, row: Optional[ActCodes] = None,
                    col: Optional[ActCodes] = None, stream=None) -> None:
    T, C = int(T), int(C)
    _need_sizes(T, C)
    if T == 0:
        return
    dev, xp = _arg(-1, x, "x", _FLOAT_TYPES, T * C)
    dev, rp = _codes_arg(dev, row, "row", T, C, True)
    dev, cp = _codes_arg(dev, col, "col", C, T, True)
    st = _on(dev, load().ft_act_quantize, xp, _FLOATS[x.dtype], T, C, rp, cp, stream)
    _check(st, "ft_act_quantize")


@functools.lru_cache(maxsize=256)   # a struct per set of values
def _linear_struct(*values: int) -> ft_linear_desc_t:
    return ft_linear_desc_t(*values)


def _linear_desc(d: dict) -> ft_linear_desc_t:
    return _linear_struct(int(d["out_features"]), int(d["in_features"]), int(d["x_dtype"]), int(d["y_dtype"]))


def ft_linear_workspace_bytes(desc: dict, max_tokens: int) -> int:
    return int(load().ft_linear_workspace_bytes(ctypes.byref(_linear_desc(desc)), int(max_tokens)))


def alloc_linear_workspace(desc: dict, max_tokens: int, device="cuda") -> torch.Tensor:
    """Workspace of ft_linear for up to max_tokens tokens."""
    n = ft_linear_workspace_bytes(desc, max_tokens)
    if n == 0:
        raise FtError(FT_ERR_SHAPE, "ft_linear_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _weight_args(dev: int, weight: dict, name: str, N: int, K: int):
    kp = _pad128(K)
    dev, w = _arg(dev, weight.get("w"), name + "['w']", _CODES, N * kp)
    dev, s = _arg(dev, weight.get("s"), name + "['s']", _F32, _pad128(N) // 128 * (kp // 128))
    return dev, w, s


def ft_linear(desc: dict, weight: dict, x, T: int, y: torch.Tensor, ws: Optional[torch.Tensor] = None,
              stream=None) -> None:
    """``x``: a device tensor [T][in_features] of x_dtype, or with FT_DT_FP8_ACT its row form
    (ActCodes); ``ws`` may be None with the latter only."""
    d, T = _linear_desc(desc), int(T)
    N, K = d.out_features, d.in_features
    _need_sizes(T, N, K)
    if T == 0:
        return
    dev, w, scales = _weight_args(-1, weight, "weight", N, K)
    if d.x_dtype == FT_DT_FP8_ACT:
        dev, xp, xs = _need_codes(x, "x", T, K, dev)
    else:
        if d.x_dtype not in _X_DTYPES:
            raise FtError(FT_ERR_DTYPE, "ft_linear")
        dev, xp = _arg(dev, x, "x", (_X_DTYPES[d.x_dtype],), T * K)
        xs = None
    if d.y_dtype not in _X_DTYPES:
        raise FtError(FT_ERR_DTYPE, "ft_linear")
    dev, yp = _arg(dev, y, "y", (_X_DTYPES[d.y_dtype],), T * N)
    wp, room = None, 0
    if ws is not None or d.x_dtype != FT_DT_FP8_ACT:
        dev, wp = _arg(dev, ws, "ws", _BYTES, 0)
        room = ws.numel()
    st = _on(dev, load().ft_linear, ctypes.byref(d), w, scales, xp, xs, T, yp, wp, room, stream)
    _check(st, "ft_linear")


def ft_linear_transpose(out_features: int, in_features: int, weight: dict, weight_t: dict, stream=None) -> None:
    N, K = int(out_features), int(in_features)
    _need_sizes(0, N, K)
    dev, w, scales = _weight_args(-1, weight, "weight", N, K)
    dev, wt, scales_t = _weight_args(dev, weight_t, "weight_t", K, N)
    st = _on(dev, load().ft_linear_transpose, N, K, w, scales, wt, scales_t, stream)
    _check(st, "ft_linear_transpose")


def ft_linear_weight_grad(out_features: int, in_features: int, T: int, dy_col: ActCodes, x_col: ActCodes,
                          dw: torch.Tensor, accumulate: bool = False, stream=None) -> None:
    """``dw``: float32 or bfloat16 [out_features][in_features].  ``dy_col``, ``x_col``: forms whose tensors are strided
    views (a transposed matrix was quantised) are brought into rows by the call, at the price of a copy."""
    N, K, T = int(out_features), int(in_features), int(T)
    _need_sizes(T, N, K)
    dev, out = _arg(-1, dw, "dw", _FLOAT_TYPES, N * K)
    yp = xp = None
    if T > 0:
        dy_col, x_col = _laid_out(dy_col, stream), _laid_out(x_col, stream)
        dev, yp = _codes_arg(dev, dy_col, "dy_col", N, T)
        dev, xp = _codes_arg(dev, x_col, "x_col", K, T)
    st = _on(dev, load().ft_linear_weight_grad, N, K, T, yp, xp, out, _FLOATS[dw.dtype], 1 if accumulate else 0, stream)
    _check(st, "ft_linear_weight_grad")


def _need_inter(T: int, inter: int) -> None:
    if inter % 128:
        raise FtError(FT_ERR_SHAPE, "sizes")
    _need_sizes(T, inter, 2 * inter)


def ft_swiglu_quantize(gu: torch.Tensor, T: int, inter: int, h: ActCodes, saved: Optional[ActCodes] = None,
                       stream=None) -> None:
    T, I = int(T), int(inter)
    _need_inter(T, I)
    if T == 0:
        return
    dev, gp = _arg(-1, gu, "gu", _FLOAT_TYPES, T * 2 * I)
    dev, hp = _codes_arg(dev, h, "h", T, I)
    dev, sp = _codes_arg(dev, saved, "saved", T, 2 * I, True)
    st = _on(dev, load().ft_swiglu_quantize, gp, _FLOATS[gu.dtype], T, I, hp, sp, stream)
    _check(st, "ft_swiglu_quantize")


def ft_swiglu_backward(saved: ActCodes, dh: torch.Tensor, T: int, inter: int, dgu_row: Optional[ActCodes] = None,
                       dgu_col: Optional[ActCodes] = None, h_col: Optional[ActCodes] = None, stream=None) -> None:
    T, I = int(T), int(inter)
    _need_inter(T, I)
    if T == 0:
        return
    dev, sp = _codes_arg(-1, saved, "saved", T, 2 * I)
    dev, dp = _arg(dev, dh, "dh", _FLOAT_TYPES, T * I)
    dev, rp = _codes_arg(dev, dgu_row, "dgu_row", T, 2 * I, True)
    dev, cp = _codes_arg(dev, dgu_col, "dgu_col", 2 * I, T, True)
    dev, hp = _codes_arg(dev, h_col, "h_col", I, T, True)
    st = _on(dev, load().ft_swiglu_backward, sp, dp, _FLOATS[dh.dtype], T, I, rp, cp, hp, stream)
    _check(st, "ft_swiglu_backward")


class BalanceBuffers:
    """Device tensors behind one ft_balance_t: counts, prob, frac [n_seq][E], tokens, loss [n_seq]."""

    def __init__(self, n_seq: int, n_experts: int, device="cuda"):
        i32, f32 = dict(dtype=torch.int32, device=device), dict(dtype=torch.float32, device=device)
        self.counts = torch.empty(n_seq, n_experts, **i32)
        self.tokens = torch.empty(n_seq, **i32)
        self.prob = torch.empty(n_seq, n_experts, **f32)
        self.frac = torch.empty(n_seq, n_experts, **f32)
        self.loss = torch.empty(n_seq, **f32)

    @classmethod
    def of(cls, counts, tokens, prob, frac, loss) -> "BalanceBuffers":
        """Buffers over existing tensors."""
        self = cls.__new__(cls)
        self.counts, self.tokens, self.prob, self.frac, self.loss = counts, tokens, prob, frac, loss
        return self


@functools.lru_cache(maxsize=256)
def _balance_struct(*values) -> ft_balance_desc_t:
    return ft_balance_desc_t(*values)


def _balance_desc(d: dict) -> ft_balance_desc_t:
    return _balance_struct(int(d["n_experts"]), int(d["top_k"]), int(d["gating"]), int(d["n_seq"]),
                           float(d.get("coef", 1.0)))


def ft_balance_workspace_bytes(desc: dict, max_tokens: int) -> int:
    return int(load().ft_balance_workspace_bytes(ctypes.byref(_balance_desc(desc)), int(max_tokens)))


def alloc_balance_workspace(desc: dict, max_tokens: int, device="cuda") -> torch.Tensor:
    n = ft_balance_workspace_bytes(desc, max_tokens)
    if n == 0:
        raise FtError(FT_ERR_SHAPE, "ft_balance_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _token_args(d: ft_balance_desc_t, logits, topk_ids, T: int, seq_off, mask):
    """-> (device, addresses of logits, topk_ids, seq_off, mask)."""
    if T < 0:
        raise FtError(FT_ERR_SHAPE, "sizes")
    dev, lp, ip, sp, mp = -1, None, None, None, None
    if T > 0:
        dev, lp = _arg(dev, logits, "logits", _F32, T * d.n_experts)
        if topk_ids is not None:
            dev, ip = _arg(dev, topk_ids, "topk_ids", _I32, T * d.top_k)
        if mask is not None:
            dev, mp = _arg(dev, mask, "mask", _MASKS, T)
    if seq_off is not None:
        dev, sp = _arg(dev, seq_off, "seq_off", _I32, d.n_seq + 1)
    return dev, lp, ip, sp, mp


def _balance_arg(dev: int, d: ft_balance_desc_t, b, names):
    """The buffers ``names`` of a BalanceBuffers as an ft_balance_t, the others left out."""
    if not isinstance(b, BalanceBuffers):
        raise ValueError("expected a BalanceBuffers")
    out = ft_balance_t()
    for n in names:
        dev, at = _arg(dev, getattr(b, n), n, _I32 if n in ("counts", "tokens") else _F32,
                       d.n_seq * (1 if n in ("tokens", "loss") else d.n_experts))
        setattr(out, n, at)
    return dev, ctypes.byref(out)


def ft_balance_loss(desc: dict, logits: torch.Tensor, topk_ids: torch.Tensor, T: int, out: BalanceBuffers,
                    ws: torch.Tensor, seq_off: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                    stream=None) -> None:
    """``topk_ids``: the routing's (RouteBuffers.topk_ids); ``mask``: uint8 or bool per token."""
    d, T = _balance_desc(desc), int(T)
    if T > 0 and topk_ids is None:
        raise ValueError("topk_ids: required")
    dev, lp, ip, sp, mp = _token_args(d, logits, topk_ids, T, seq_off, mask)
    dev, bp = _balance_arg(dev, d, out, ("counts", "tokens", "prob", "frac", "loss"))
    dev, wp = _arg(dev, ws, "ws", _BYTES, 0)
    st = _on(dev, load().ft_balance_loss, ctypes.byref(d), lp, ip, T, sp, mp, bp, wp, ws.numel(), stream)
    _check(st, "ft_balance_loss")


def ft_router_backward(desc: dict, logits: torch.Tensor, topk_ids: Optional[torch.Tensor], T: int,
                       balance: Optional[BalanceBuffers], d_loss: Optional[torch.Tensor], d_logits: torch.Tensor,
                       topk_w: Optional[torch.Tensor] = None, d_topk_w: Optional[torch.Tensor] = None,
                       seq_off: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, stream=None) -> None:
    """``balance`` and ``d_loss`` may be None (gates only), or ``d_topk_w`` (loss only)."""
    d, T = _balance_desc(desc), int(T)
    dev, lp, ip, sp, mp = _token_args(d, logits, topk_ids, T, seq_off, mask)
    if T == 0:
        return
    dev, op = _arg(dev, d_logits, "d_logits", _F32, T * d.n_experts)
    bp = dl = wp = dw = None
    if d_loss is not None:
        dev, dl = _arg(dev, d_loss, "d_loss", _F32, d.n_seq)
        dev, bp = _balance_arg(dev, d, balance, ("tokens", "frac"))
    if d_topk_w is not None:
        if topk_ids is None:
            raise ValueError("topk_ids: required with d_topk_w")
        dev, wp = _arg(dev, topk_w, "topk_w", _F32, T * d.top_k)
        dev, dw = _arg(dev, d_topk_w, "d_topk_w", _F32, T * d.top_k)
    st = _on(dev, load().ft_router_backward, ctypes.byref(d), lp, ip, T, sp, mp, bp, dl, wp, dw, op, stream)
    _check(st, "ft_router_backward")


# ------------------------------------------------------------ the routed experts in training, and norms

@functools.lru_cache(maxsize=256)   # a struct per set of values
def _sort_struct(E, k, first, local, align, rows) -> ft_sort_desc_t:
    return ft_sort_desc_t(int(E), int(k), int(first), int(E if local is None else local), int(align), int(rows))


def _sort_desc(d: dict) -> ft_sort_desc_t:
    """``first`` and ``local`` may be left out (every expert is here)."""
    return _sort_struct(d["n_experts"], d["top_k"], d.get("first", 0), d.get("local"), d["align"], d["rows"])


def ft_expert_sort_rows(desc: dict, T: int) -> int:
    """Rows that hold every pair of T tokens (``rows`` is not needed in ``desc``); 0 where the library refuses."""
    return int(load().ft_expert_sort_rows(ctypes.byref(_sort_desc({"rows": 0, **desc})), int(T)))


class SortBuffers:
    """Device tensors behind one ft_sort_t for T tokens: row_pair [rows], pair_row [T][top_k], off [local + 1],
    count [local], dropped [1], all int32."""

    def __init__(self, desc: dict, T: int, device="cuda"):
        d = _sort_desc(desc)
        kw = dict(dtype=torch.int32, device=device)
        self.row_pair = torch.empty(d.rows, **kw)
        self.pair_row = torch.empty(T, d.top_k, **kw)
        self.off = torch.empty(d.local + 1, **kw)
        self.count = torch.empty(d.local, **kw)
        self.dropped = torch.empty(1, **kw)

    @classmethod
    def of(cls, row_pair, pair_row, off, count, dropped) -> "SortBuffers":
        """Buffers over existing tensors."""
        self = cls.__new__(cls)
        self.row_pair, self.pair_row, self.off, self.count, self.dropped = row_pair, pair_row, off, count, dropped
        return self


def ft_expert_sort_workspace_bytes(desc: dict, max_tokens: int) -> int:
    return int(load().ft_expert_sort_workspace_bytes(ctypes.byref(_sort_desc(desc)), int(max_tokens)))


def alloc_sort_workspace(desc: dict, max_tokens: int, device="cuda") -> torch.Tensor:
    """Workspace of ft_expert_sort for up to max_tokens tokens."""
    n = ft_expert_sort_workspace_bytes(desc, max_tokens)
    if n == 0:
        raise FtError(FT_ERR_SHAPE, "ft_expert_sort_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _need_tokens(d: ft_sort_desc_t, T: int, *features: int) -> None:
    _need_sizes(T, *features)
    if d.rows < 16 or d.top_k < 1 or d.local < 1:
        raise FtError(FT_ERR_SHAPE, "sizes")


def _need_sort(sort) -> None:
    if not isinstance(sort, SortBuffers):
        raise ValueError(f"sort: expected a SortBuffers, got {type(sort).__name__}")


def _groups_arg(dev: int, d: ft_sort_desc_t, sort):
    """What a product reads of a SortBuffers, as an ft_sort_t."""
    _need_sort(sort)
    local = d.local
    dev, off = _arg(dev, sort.off, "off", _I32, local + 1)
    dev, count = _arg(dev, sort.count, "count", _I32, local)
    return dev, ctypes.byref(ft_sort_t(None, None, off, count))


def _pairs_arg(dev: int, d: ft_sort_desc_t, T: int, sort):
    """What a call that goes by tokens reads of it."""
    _need_sort(sort)
    dev, at = _arg(dev, sort.pair_row, "pair_row", _I32, T * d.top_k)
    return dev, ctypes.byref(ft_sort_t(None, at))


def _optional(dev: int, t, name: str, dtypes: tuple, numel: int):
    return (dev, None) if t is None else _arg(dev, t, name, dtypes, numel)


def ft_expert_sort(desc: dict, topk_ids: torch.Tensor, T: int, out: SortBuffers, ws: torch.Tensor,
                   mask: Optional[torch.Tensor] = None, stream=None) -> None:
    """``topk_ids``: the routing's (RouteBuffers.topk_ids); ``mask``: uint8 or bool per token."""
    d, T = _sort_desc(desc), int(T)
    _need_tokens(d, T)
    dev, ip, mp = -1, None, None
    if T > 0:
        dev, ip = _arg(dev, topk_ids, "topk_ids", _I32, T * d.top_k)
        dev, mp = _optional(dev, mask, "mask", _MASKS, T)
    _need_sort(out)
    local, pairs = d.local, None
    dev, rows = _arg(dev, out.row_pair, "row_pair", _I32, d.rows)
    if T > 0:
        dev, pairs = _arg(dev, out.pair_row, "pair_row", _I32, T * d.top_k)
    dev, off = _arg(dev, out.off, "off", _I32, local + 1)
    dev, count = _arg(dev, out.count, "count", _I32, local)
    dev, dropped = _arg(dev, out.dropped, "dropped", _I32, 1)
    dev, wp = _arg(dev, ws, "ws", _BYTES, 0)
    st = _on(dev, load().ft_expert_sort, ctypes.byref(d), ip, T, mp, ctypes.byref(ft_sort_t(rows, pairs, off, count, dropped)),
             wp, ws.numel(), stream)
    _check(st, "ft_expert_sort")


def ft_expert_gather(desc: dict, sort: SortBuffers, x: torch.Tensor, T: int, C: int,
                     weights: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
                     row: Optional[ActCodes] = None, col: Optional[ActCodes] = None, stream=None) -> None:
    """``rows``: the plain rows, float32 or bfloat16 [desc rows][C]; ``row``, ``col``: their 8-bit forms."""
    d, T, C = _sort_desc(desc), int(T), int(C)
    _need_tokens(d, T, C)
    if T == 0:
        return
    dev, xp = _arg(-1, x, "x", _FLOAT_TYPES, T * C)
    _need_sort(sort)
    dev, at = _arg(dev, sort.row_pair, "row_pair", _I32, d.rows)
    dev, off = _arg(dev, sort.off, "off", _I32, d.local + 1)
    sp = ctypes.byref(ft_sort_t(at, None, off))
    dev, wp = _optional(dev, weights, "weights", _F32, T * d.top_k)
    dev, pp = _optional(dev, rows, "rows", _FLOAT_TYPES, d.rows * C)
    dev, rp = _codes_arg(dev, row, "row", d.rows, C, True)
    dev, cp = _codes_arg(dev, col, "col", C, d.rows, True)
    st = _on(dev, load().ft_expert_gather, ctypes.byref(d), sp, xp, _FLOATS[x.dtype], T, C, wp, pp,
             0 if rows is None else _FLOATS[rows.dtype], rp, cp, stream)
    _check(st, "ft_expert_gather")


def ft_expert_combine(desc: dict, sort: SortBuffers, rows: torch.Tensor, T: int, C: int, y: torch.Tensor,
                      weights: Optional[torch.Tensor] = None, base: Optional[torch.Tensor] = None, stream=None) -> None:
    """``base``: of y's type, or y itself."""
    d, T, C = _sort_desc(desc), int(T), int(C)
    _need_tokens(d, T, C)
    if T == 0:
        return
    dev, rp = _arg(-1, rows, "rows", _FLOAT_TYPES, d.rows * C)
    dev, sp = _pairs_arg(dev, d, T, sort)
    dev, yp = _arg(dev, y, "y", _FLOAT_TYPES, T * C)
    dev, wp = _optional(dev, weights, "weights", _F32, T * d.top_k)
    dev, bp = _optional(dev, base, "base", (y.dtype,), T * C)
    st = _on(dev, load().ft_expert_combine, ctypes.byref(d), sp, rp, _FLOATS[rows.dtype], T, C, wp, bp, yp,
             _FLOATS[y.dtype], stream)
    _check(st, "ft_expert_combine")


def ft_expert_gate_grad(desc: dict, sort: SortBuffers, rows: torch.Tensor, dy: torch.Tensor, T: int, C: int,
                        d_weights: torch.Tensor, stream=None) -> None:
    d, T, C = _sort_desc(desc), int(T), int(C)
    _need_tokens(d, T, C)
    if T == 0:
        return
    dev, rp = _arg(-1, rows, "rows", _FLOAT_TYPES, d.rows * C)
    dev, sp = _pairs_arg(dev, d, T, sort)
    dev, yp = _arg(dev, dy, "dy", _FLOAT_TYPES, T * C)
    dev, wp = _arg(dev, d_weights, "d_weights", _F32, T * d.top_k)
    st = _on(dev, load().ft_expert_gate_grad, ctypes.byref(d), sp, rp, _FLOATS[rows.dtype], yp, _FLOATS[dy.dtype], T, C, wp,
             stream)
    _check(st, "ft_expert_gate_grad")


def _expert_weights(dev: int, weight: dict, name: str, n: int, N: int, K: int):
    kp = _pad128(K)
    dev, w = _arg(dev, weight.get("w"), name + "['w']", _CODES, n * N * kp)
    dev, s = _arg(dev, weight.get("s"), name + "['s']", _F32, n * (_pad128(N) // 128) * (kp // 128))
    return dev, w, s


def ft_expert_linear(desc: dict, linear: dict, weight: dict, x: ActCodes, sort: SortBuffers, T: int, y: torch.Tensor,
                     stream=None) -> None:
    """``weight``: ``w`` [local][N][Kp] codes and ``s`` their block scales; ``x``: the row form of the rows."""
    d, l, T = _sort_desc(desc), _linear_desc(linear), int(T)
    N, K = l.out_features, l.in_features
    _need_tokens(d, T, N, K)
    if T == 0:
        return
    if l.x_dtype != FT_DT_FP8_ACT or l.y_dtype not in _X_DTYPES:
        raise FtError(FT_ERR_DTYPE, "ft_expert_linear")
    dev, w, s = _expert_weights(-1, weight, "weight", d.local, N, K)
    dev, xp = _codes_arg(dev, x, "x", d.rows, K)
    dev, sp = _groups_arg(dev, d, sort)
    dev, yp = _arg(dev, y, "y", (_X_DTYPES[l.y_dtype],), d.rows * N)
    st = _on(dev, load().ft_expert_linear, ctypes.byref(d), ctypes.byref(l), w, s, xp, sp, T, yp, stream)
    _check(st, "ft_expert_linear")


def ft_expert_linear_transpose(n: int, out_features: int, in_features: int, weight: dict, weight_t: dict, stream=None) -> None:
    n, N, K = int(n), int(out_features), int(in_features)
    _need_sizes(0, N, K)
    if not 1 <= n <= 1024:
        raise FtError(FT_ERR_SHAPE, "sizes")
    dev, w, s = _expert_weights(-1, weight, "weight", n, N, K)
    dev, wt, ts = _expert_weights(dev, weight_t, "weight_t", n, K, N)
    st = _on(dev, load().ft_expert_linear_transpose, n, N, K, w, s, wt, ts, stream)
    _check(st, "ft_expert_linear_transpose")


def ft_expert_weight_grad(desc: dict, out_features: int, in_features: int, dy_col: ActCodes, x_col: ActCodes,
                          sort: SortBuffers, T: int, dw: torch.Tensor, accumulate: bool = False, stream=None) -> None:
    """``dw``: float32 or bfloat16 [local][out_features][in_features].  ``dy_col``, ``x_col``: strided views are brought
    into rows by the call, as in ft_linear_weight_grad."""
    d, N, K, T = _sort_desc(desc), int(out_features), int(in_features), int(T)
    _need_tokens(d, T, N, K)
    dev, out = _arg(-1, dw, "dw", _FLOAT_TYPES, d.local * N * K)
    yp = xp = sp = None
    if T > 0:
        dy_col, x_col = _laid_out(dy_col, stream), _laid_out(x_col, stream)
        dev, yp = _codes_arg(dev, dy_col, "dy_col", N, d.rows)
        dev, xp = _codes_arg(dev, x_col, "x_col", K, d.rows)
        dev, sp = _groups_arg(dev, d, sort)
    st = _on(dev, load().ft_expert_weight_grad, ctypes.byref(d), N, K, yp, xp, sp, T, out, _FLOATS[dw.dtype],
             1 if accumulate else 0, stream)
    _check(st, "ft_expert_weight_grad")


@functools.lru_cache(maxsize=256)
def _norm_struct(C, x, y, w, post, eps, scale) -> ft_norm_desc_t:
    return ft_norm_desc_t(int(C), int(x), int(y), int(w), int(post), float(eps), float(scale))


def _norm_desc(d: dict) -> ft_norm_desc_t:
    return _norm_struct(d["channels"], d["x_dtype"], d["y_dtype"], d["w_dtype"], d.get("post_norm", 0), d["eps"],
                        d.get("scale", 1.0))


def _norm_types(d: ft_norm_desc_t, T: int, where: str):
    """-> the tensor types of x, y and the weights."""
    _need_sizes(T, d.channels)
    kinds = [_X_DTYPES.get(v) for v in (d.x_dtype, d.y_dtype, d.w_dtype)]
    if None in kinds:
        raise FtError(FT_ERR_DTYPE, where)
    return kinds


def _norm_params(dev: int, d: ft_norm_desc_t, T: int, params: dict, kind):
    C, kinds, at = d.channels, (kind,), [None] * 4
    for i, n in enumerate(("pre", "post", "gate", "token_gate")):
        t = params.get(n)
        if t is not None:
            dev, at[i] = _arg(dev, t, n, kinds if i < 3 else _F32, C if i < 3 else T)
    return dev, ctypes.byref(ft_norm_params_t(*at))


def ft_block_norm(desc: dict, params: dict, x: torch.Tensor, block: Optional[torch.Tensor], T: int,
                  r: Optional[torch.Tensor] = None, n: Optional[torch.Tensor] = None, n_row: Optional[ActCodes] = None,
                  stream=None) -> None:
    """``params``: ``pre``, ``post``, ``gate``, ``token_gate``, each a tensor or left out (ones)."""
    d, T = _norm_desc(desc), int(T)
    xk, yk, wk = _norm_types(d, T, "ft_block_norm")
    if T == 0:
        return
    size = T * d.channels
    dev, xp = _arg(-1, x, "x", (xk,), size)
    dev, pp = _norm_params(dev, d, T, params, wk)
    dev, bp = _optional(dev, block, "block", (yk,), size)
    dev, rp = _optional(dev, r, "r", (xk,), size)
    dev, np_ = _optional(dev, n, "n", (yk,), size)
    dev, cp = _codes_arg(dev, n_row, "n_row", T, d.channels, True)
    st = _on(dev, load().ft_block_norm, ctypes.byref(d), pp, xp, bp, T, rp, np_, cp, stream)
    _check(st, "ft_block_norm")


def ft_block_norm_workspace_bytes(desc: dict, max_tokens: int) -> int:
    return int(load().ft_block_norm_workspace_bytes(ctypes.byref(_norm_desc(desc)), int(max_tokens)))


def alloc_block_norm_workspace(desc: dict, max_tokens: int, device="cuda") -> torch.Tensor:
    """Workspace of ft_block_norm_backward for up to max_tokens tokens."""
    n = ft_block_norm_workspace_bytes(desc, max_tokens)
    if n == 0:
        raise FtError(FT_ERR_SHAPE, "ft_block_norm_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def ft_block_norm_backward(desc: dict, params: dict, r: torch.Tensor, block: Optional[torch.Tensor],
                           dr: Optional[torch.Tensor], dn: Optional[torch.Tensor], T: int,
                           dx: Optional[torch.Tensor] = None, d_block: Optional[torch.Tensor] = None,
                           grads: Optional[dict] = None, ws: Optional[torch.Tensor] = None, stream=None) -> None:
    """``grads``: float32 tensors for the gradients of ``params``, those left out or None are not formed."""
    d, T = _norm_desc(desc), int(T)
    xk, yk, wk = _norm_types(d, T, "ft_block_norm_backward")
    size, g, dev = T * d.channels, [None] * 4, -1
    for i, n in enumerate(("pre", "post", "gate", "token_gate")):
        t = (grads or {}).get(n)
        if t is not None:
            dev, g[i] = _arg(dev, t, "d_" + n, _F32, d.channels if i < 3 else T)
    if T == 0 and not any(g[:3]):
        return
    dev, pp = _norm_params(dev, d, T, params, wk)
    rp = bp = drp = dnp = dxp = dbp = None
    if T > 0:
        dev, rp = _arg(dev, r, "r", (xk,), size)
        dev, bp = _optional(dev, block, "block", (yk,), size)
        dev, drp = _optional(dev, dr, "dr", (xk,), size)
        dev, dnp = _optional(dev, dn, "dn", (yk,), size)
        dev, dxp = _optional(dev, dx, "dx", (xk,), size)
        dev, dbp = _optional(dev, d_block, "d_block", (yk,), size)
    dev, wp = _optional(dev, ws, "ws", _BYTES, 0)
    st = _on(dev, load().ft_block_norm_backward, ctypes.byref(d), pp, rp, bp, drp, dnp, T, dxp, dbp, ctypes.byref(ft_norm_grads_t(*g)), wp,
             0 if ws is None else ws.numel(), stream)
    _check(st, "ft_block_norm_backward")
