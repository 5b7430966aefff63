"""Thin Python binding of libmetro.so (see include/metro.h): argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI; torch supplies device
memory and the current stream.  There is no CPU fallback: if the library has not been
built, loading fails.

The calls of a serving step (routing, FFN, combine, gate) are marshalled by native code (csrc/call.cpp) when every
argument is the plain case and all buffers are given; anything else goes through the checks below, which decide what
is refused and say why.  The checks cost about 0.6 us a tensor here, more than the launches: a small fp32 layer (three
calls, four kernels, 18 us on the device) took 31 us for the host's sake, and takes 17 us with the native way.
"""
from __future__ import annotations

import ctypes
import importlib
import os
from typing import Dict, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmetro.so")
CALL_PATH = os.path.join(_HERE, "_call.so")
_lib = None
_native = None              # csrc/call.cpp
_fn: Dict[str, int] = {}    # addresses of the library's functions, for it

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP, ERR_TOO_LARGE = 0, -1, -2, -3, -4, -5
FLAG_BAD_ID, FLAG_NO_REPLICA, FLAG_BAD_PLACEMENT = 1, 2, 4
DTYPE_F32, DTYPE_BF16 = 0, 1

EXPORTS = ("metro_status_string", "metro_route", "metro_route_token_balanced", "moe_permute",
           "moe_grouped_ffn_workspace_bytes", "moe_grouped_ffn", "moe_grouped_ffn_gate_up",
           "moe_grouped_ffn_down", "moe_unpermute", "moe_gate_topk_workspace_bytes", "moe_gate_topk",
           "moe_grouped_ffn_static_ws_bytes", "moe_grouped_ffn_static_ws", "metro_route_permute",
           "metro_route_token_balanced_permute", "moe_permute_rows", "moe_permute_rows_backward", "moe_unpermute_backward",
           "moe_quantize_fp8", "moe_quantize_weights_fp8", "moe_grouped_mm_fp8", "moe_grouped_ffn_fp8_workspace_bytes",
           "moe_grouped_ffn_fp8")


class MetroError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"libmetro: {text} (status {status})")
        self.status = status


def load() -> ctypes.CDLL:
    """Load the in-tree library; raises if it was not built (python -m paper_2512_09277_amd.build)."""
    global _lib, _native
    if _lib is None:
        for path in (LIB_PATH, CALL_PATH):
            if not os.path.exists(path):
                raise RuntimeError(f"{path} is missing: build it with `python -m paper_2512_09277_amd.build` "
                                   "(there is no fallback path)")
        lib = ctypes.CDLL(LIB_PATH)
        vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        lib.metro_status_string.restype = ctypes.c_char_p
        lib.metro_status_string.argtypes = [ci]
        lib.metro_route.restype = ci
        lib.metro_route.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp]
        lib.metro_route_token_balanced.restype = ci
        lib.metro_route_token_balanced.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, vp, vp, vp, vp, vp]
        lib.metro_route_permute.restype = ci
        lib.metro_route_permute.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.metro_route_token_balanced_permute.restype = ci
        lib.metro_route_token_balanced_permute.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.moe_permute.restype = ci
        lib.moe_permute.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp, vp]
        lib.moe_grouped_ffn_workspace_bytes.restype = sz
        lib.moe_grouped_ffn_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci]
        lib.moe_grouped_ffn.restype = ci
        lib.moe_grouped_ffn.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, ci, vp, ci, vp, ci, vp, vp, sz, vp]
        lib.moe_grouped_ffn_gate_up.restype = ci
        lib.moe_grouped_ffn_gate_up.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, ci, vp, ci, vp, sz, vp]
        lib.moe_grouped_ffn_down.restype = ci
        lib.moe_grouped_ffn_down.argtypes = [vp, ci, ci, ci, ci, ci, ci, vp, ci, vp, vp, sz, vp]
        lib.moe_grouped_ffn_static_ws_bytes.restype = sz
        lib.moe_grouped_ffn_static_ws_bytes.argtypes = []
        lib.moe_grouped_ffn_static_ws.restype = ci
        lib.moe_grouped_ffn_static_ws.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, ci, vp, ci, vp, ci, vp, vp]
        lib.moe_unpermute.restype = ci
        lib.moe_unpermute.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp, vp]
        lib.moe_gate_topk_workspace_bytes.restype = sz
        lib.moe_gate_topk_workspace_bytes.argtypes = [ci, ci, ci, ci]
        lib.moe_gate_topk.restype = ci
        lib.moe_gate_topk.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, vp, vp, vp, vp, vp, sz, vp]
        lib.moe_permute_rows.restype = ci
        lib.moe_permute_rows.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp]
        lib.moe_permute_rows_backward.restype = ci
        lib.moe_permute_rows_backward.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp]
        lib.moe_unpermute_backward.restype = ci
        lib.moe_unpermute_backward.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, vp]
        lib.moe_quantize_fp8.restype = ci
        lib.moe_quantize_fp8.argtypes = [vp, ci, ci, ci, ci, vp, vp, ci, vp, vp]
        lib.moe_quantize_weights_fp8.restype = ci
        lib.moe_quantize_weights_fp8.argtypes = [vp, ci, ci, ci, ci, ci, vp, ci, vp, vp]
        lib.moe_grouped_mm_fp8.restype = ci
        lib.moe_grouped_mm_fp8.argtypes = [vp, ci, vp, vp, vp, ci, ci, ci, ci, ci, vp, ci, vp, ci, vp, vp]
        lib.moe_grouped_ffn_fp8_workspace_bytes.restype = sz
        lib.moe_grouped_ffn_fp8_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
        lib.moe_grouped_ffn_fp8.restype = ci
        lib.moe_grouped_ffn_fp8.argtypes = [vp, ci, vp, vp, vp, ci, ci, ci, ci, ci, vp, ci, vp, vp, ci, vp, ci, vp, vp, sz, vp]
        _fn.update({name: ctypes.cast(getattr(lib, name), vp).value for name in EXPORTS})
        _native = importlib.import_module("._call", __package__)
        _lib = lib
    return _lib


_UNUSUAL = 1                # of the native calls: not the plain case, nothing enqueued


def _check(status: int) -> None:
    if status != OK:
        raise MetroError(status, load().metro_status_string(status).decode())


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _dev(t: torch.Tensor, dtype: torch.dtype, name: str) -> int:
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name}: expected a contiguous {dtype} device tensor, got {t.dtype} on {t.device}")
    return t.data_ptr()


def _weights(t: torch.Tensor, dtype: torch.dtype, name: str):
    """Weights [slots, rows, K]: K contiguous, rows `ld` elements apart, slots rows*ld apart (a dense
    tensor, or a [:, :, :K] view of a buffer with padded rows).  Returns (pointer, ld)."""
    if not (t.is_cuda and t.dtype == dtype and t.dim() == 3):
        raise TypeError(f"{name}: expected a 3-d {dtype} device tensor")
    slots, rows, K = t.shape
    ld = t.stride(1) if rows > 1 else max(K, t.stride(1))
    if t.stride(2) != 1 or ld < K or (slots > 1 and t.stride(0) != rows * ld):
        raise TypeError(f"{name}: rows must be K-contiguous with a uniform pitch (strides {t.stride()})")
    return t.data_ptr(), ld


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    if t.dtype == torch.float32:
        return DTYPE_F32
    raise TypeError("activations and weights are bfloat16 or float32")


def route_buffers(L: int, T: int, k: int, N: int, G: int, device) -> Dict[str, torch.Tensor]:
    """Output buffers of the routing calls (reusable across calls of the same shape)."""
    return dict(pair_slot=torch.empty((L, T, k), dtype=torch.int32, device=device),
                expert_slot=torch.empty((L, N), dtype=torch.int32, device=device),
                rank_active=torch.empty((L, G), dtype=torch.int32, device=device),
                rank_bitmap=torch.empty((L, G), dtype=torch.int64, device=device),
                err_flag=torch.empty((L,), dtype=torch.int32, device=device))


def _route(fn_name: str, topk_ids: torch.Tensor, slot_to_expert: torch.Tensor, N: int, G: int, spr: int,
           out: Optional[Dict[str, torch.Tensor]]) -> Dict[str, torch.Tensor]:
    lib = load()
    if out is not None:
        status = _native.route(_fn[fn_name], int(fn_name == "metro_route"), topk_ids, slot_to_expert, N, G, spr, out)
        if status != _UNUSUAL:
            _check(status)
            return out
    if topk_ids.dim() == 2:
        topk_ids = topk_ids.unsqueeze(0)
    if slot_to_expert.dim() == 1:
        slot_to_expert = slot_to_expert.unsqueeze(0)
    L, T, k = topk_ids.shape
    if tuple(slot_to_expert.shape) != (L, G * spr):
        raise ValueError(f"slot_to_expert must be [L={L}, G*spr={G * spr}]")
    if out is None:
        out = route_buffers(L, T, k, N, G, topk_ids.device)
    ids_p = _dev(topk_ids, torch.int32, "topk_ids")
    s2e_p = _dev(slot_to_expert, torch.int32, "slot_to_expert")
    ps = _dev(out["pair_slot"], torch.int32, "pair_slot")
    ra = _dev(out["rank_active"], torch.int32, "rank_active")
    rb = _dev(out["rank_bitmap"], torch.int64, "rank_bitmap")
    ef = _dev(out["err_flag"], torch.int32, "err_flag")
    if fn_name == "metro_route":
        es = _dev(out["expert_slot"], torch.int32, "expert_slot")
        _check(lib.metro_route(ids_p, s2e_p, L, T, k, N, G, spr, ps, es, ra, rb, ef, _stream()))
    else:
        _check(lib.metro_route_token_balanced(ids_p, s2e_p, L, T, k, N, G, spr, ps, ra, rb, ef, _stream()))
    return out


def metro_route(topk_ids, slot_to_expert, N: int, G: int, spr: int, out=None) -> Dict[str, torch.Tensor]:
    """topk_ids [L,T,k] (or [T,k]) int32, slot_to_expert [L,S] (or [S]) int32 -> dict of device tensors
    pair_slot [L,T,k], expert_slot [L,N], rank_active [L,G], rank_bitmap [L,G] (int64 bits), err_flag [L]."""
    return _route("metro_route", topk_ids, slot_to_expert, N, G, spr, out)


def metro_route_token_balanced(topk_ids, slot_to_expert, N: int, G: int, spr: int, out=None):
    """Same as metro_route for the token-balanced baseline; expert_slot is left untouched."""
    return _route("metro_route_token_balanced", topk_ids, slot_to_expert, N, G, spr, out)


def permute_buffers(T: int, k: int, spr: int, device) -> Dict[str, torch.Tensor]:
    return dict(group_offsets=torch.empty((spr + 1,), dtype=torch.int32, device=device),
                perm_pair=torch.empty((T * k,), dtype=torch.int32, device=device),
                pair_row=torch.empty((T, k), dtype=torch.int32, device=device),
                n_pairs=torch.empty((1,), dtype=torch.int32, device=device))


def moe_permute(pair_slot: torch.Tensor, rank: int, spr: int, out=None) -> Dict[str, torch.Tensor]:
    """pair_slot [T,k] int32 -> dict(group_offsets [spr+1], perm_pair [T*k], pair_row [T,k], n_pairs [1])."""
    T, k = pair_slot.shape
    if out is None:
        out = permute_buffers(T, k, spr, pair_slot.device)
    _check(load().moe_permute(_dev(pair_slot, torch.int32, "pair_slot"), T, k, rank, spr,
                              _dev(out["group_offsets"], torch.int32, "group_offsets"),
                              _dev(out["perm_pair"], torch.int32, "perm_pair"),
                              _dev(out["pair_row"], torch.int32, "pair_row"),
                              _dev(out["n_pairs"], torch.int32, "n_pairs"), _stream()))
    return out


def _route_permute(fn_name: str, topk_ids, slot_to_expert, N: int, G: int, spr: int, rank: int, out, lists):
    lib = load()
    if out is not None and lists is not None:
        status = _native.route_permute(_fn[fn_name], int(fn_name == "metro_route_permute"), topk_ids, slot_to_expert, N, G,
                                       spr, rank, out, lists)
        if status != _UNUSUAL:
            _check(status)
            return out, lists
    if topk_ids.dim() == 3:
        if topk_ids.shape[0] != 1:
            raise ValueError("the fused call takes one layer")
        topk_ids = topk_ids[0]
    if slot_to_expert.dim() == 2:
        slot_to_expert = slot_to_expert[0]
    T, k = topk_ids.shape
    if slot_to_expert.numel() != G * spr:
        raise ValueError(f"slot_to_expert must hold G*spr={G * spr} entries")
    if out is None:
        out = route_buffers(1, T, k, N, G, topk_ids.device)
    if lists is None:
        lists = permute_buffers(T, k, spr, topk_ids.device)
    head = [_dev(topk_ids, torch.int32, "topk_ids"), _dev(slot_to_expert, torch.int32, "slot_to_expert"), T, k, N, G, spr,
            rank, _dev(out["pair_slot"], torch.int32, "pair_slot")]
    tail = [_dev(out["rank_active"], torch.int32, "rank_active"), _dev(out["rank_bitmap"], torch.int64, "rank_bitmap"),
            _dev(out["err_flag"], torch.int32, "err_flag"), _dev(lists["group_offsets"], torch.int32, "group_offsets"),
            _dev(lists["perm_pair"], torch.int32, "perm_pair"), _dev(lists["pair_row"], torch.int32, "pair_row"),
            _dev(lists["n_pairs"], torch.int32, "n_pairs"), _stream()]
    if fn_name == "metro_route_permute":
        _check(lib.metro_route_permute(*head, _dev(out["expert_slot"], torch.int32, "expert_slot"), *tail))
    else:
        _check(lib.metro_route_token_balanced_permute(*head, *tail))
    return out, lists


def metro_route_permute(topk_ids, slot_to_expert, N: int, G: int, spr: int, rank: int, out=None, lists=None):
    """metro_route (one layer) and moe_permute(rank) in one launch -> (routing dict, token-list dict)."""
    return _route_permute("metro_route_permute", topk_ids, slot_to_expert, N, G, spr, rank, out, lists)


def metro_route_token_balanced_permute(topk_ids, slot_to_expert, N: int, G: int, spr: int, rank: int, out=None,
                                       lists=None):
    """metro_route_token_balanced (one layer) and moe_permute(rank) in one launch."""
    return _route_permute("metro_route_token_balanced_permute", topk_ids, slot_to_expert, N, G, spr, rank, out, lists)


def moe_grouped_ffn_workspace_bytes(T: int, k: int, spr: int, H: int, I: int, dtype: torch.dtype) -> int:
    code = DTYPE_BF16 if dtype == torch.bfloat16 else DTYPE_F32
    return int(load().moe_grouped_ffn_workspace_bytes(T, k, spr, H, I, code))


def moe_grouped_ffn(x: torch.Tensor, perm_pair: torch.Tensor, group_offsets: torch.Tensor, k: int,
                    w13: torch.Tensor, w2: torch.Tensor, y_perm: Optional[torch.Tensor] = None,
                    ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [T,H], w13 [spr,2I,H], w2 [spr,H,I] (bf16 or f32) -> y_perm [T*k,H] (rows < n_pairs written)."""
    load()
    if y_perm is not None and ws is not None:
        status = _native.ffn(_fn["moe_grouped_ffn"], x, perm_pair, group_offsets, k, w13, w2, y_perm, ws)
        if status != _UNUSUAL:
            _check(status)
            return y_perm
    T, H = x.shape
    spr, two_i, _ = w13.shape
    I = two_i // 2
    if tuple(w13.shape) != (spr, 2 * I, H) or tuple(w2.shape) != (spr, H, I):
        raise ValueError("weight shapes must be w13 [spr,2I,H] and w2 [spr,H,I]")
    if perm_pair.numel() < T * k or group_offsets.numel() != spr + 1:
        raise ValueError("perm_pair must hold T*k entries and group_offsets spr+1")
    code = _dtype_code(x)
    if y_perm is None:
        y_perm = torch.empty((T * k, H), dtype=x.dtype, device=x.device)
    need = int(load().moe_grouped_ffn_workspace_bytes(T, k, spr, H, I, code))
    if ws is None:
        ws = torch.empty((need,), dtype=torch.uint8, device=x.device)
    p13, ld13 = _weights(w13, x.dtype, "w13")
    p2, ld2 = _weights(w2, x.dtype, "w2")
    _check(load().moe_grouped_ffn(_dev(x, x.dtype, "x"), _dev(perm_pair, torch.int32, "perm_pair"),
                                  _dev(group_offsets, torch.int32, "group_offsets"), T, k, spr, H, I, code,
                                  p13, ld13, p2, ld2, _dev(y_perm, x.dtype, "y_perm"),
                                  _dev(ws, torch.uint8, "ws"), ws.numel(), _stream()))
    return y_perm


def moe_grouped_ffn_static_ws(x: torch.Tensor, perm_pair: torch.Tensor, group_offsets: torch.Tensor, k: int,
                              w13: torch.Tensor, w2: torch.Tensor, y_perm: torch.Tensor) -> torch.Tensor:
    """moe_grouped_ffn on the library's built-in workspace: the caller passes inputs and the output only."""
    T, H = x.shape
    spr, two_i, _ = w13.shape
    I = two_i // 2
    if tuple(w13.shape) != (spr, 2 * I, H) or tuple(w2.shape) != (spr, H, I):
        raise ValueError("weight shapes must be w13 [spr,2I,H] and w2 [spr,H,I]")
    if perm_pair.numel() < T * k or group_offsets.numel() != spr + 1 or tuple(y_perm.shape) != (T * k, H):
        raise ValueError("perm_pair must hold T*k entries, group_offsets spr+1, y_perm [T*k,H]")
    p13, ld13 = _weights(w13, x.dtype, "w13")
    p2, ld2 = _weights(w2, x.dtype, "w2")
    _check(load().moe_grouped_ffn_static_ws(_dev(x, x.dtype, "x"), _dev(perm_pair, torch.int32, "perm_pair"),
                                            _dev(group_offsets, torch.int32, "group_offsets"), T, k, spr, H, I,
                                            _dtype_code(x), p13, ld13, p2, ld2, _dev(y_perm, x.dtype, "y_perm"),
                                            _stream()))
    return y_perm


def moe_grouped_ffn_stages(x, perm_pair, group_offsets, k: int, w13, w2, y_perm, ws, between=None):
    """moe_grouped_ffn as its two stage calls; `between(i)` (i = 0..2) is called before, between and
    after the stages, e.g. to record events on the current stream."""
    T, H = x.shape
    spr, two_i, _ = w13.shape
    I = two_i // 2
    code = _dtype_code(x)
    lib = load()
    go = _dev(group_offsets, torch.int32, "group_offsets")
    wsp, wsn = _dev(ws, torch.uint8, "ws"), ws.numel()
    mark = between if between is not None else (lambda i: None)
    p13, ld13 = _weights(w13, x.dtype, "w13")
    p2, ld2 = _weights(w2, x.dtype, "w2")
    mark(0)
    _check(lib.moe_grouped_ffn_gate_up(_dev(x, x.dtype, "x"), _dev(perm_pair, torch.int32, "perm_pair"), go, T, k,
                                       spr, H, I, code, p13, ld13, wsp, wsn, _stream()))
    mark(1)
    _check(lib.moe_grouped_ffn_down(go, T, k, spr, H, I, code, p2, ld2, _dev(y_perm, x.dtype, "y_perm"), wsp, wsn,
                                    _stream()))
    mark(2)
    return y_perm


def moe_unpermute(y_perm: torch.Tensor, pair_row: torch.Tensor, topk_w: torch.Tensor,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y_perm [T*k,H], pair_row [T,k] int32, topk_w [T,k] float32 -> out [T,H]."""
    load()
    if out is not None:
        status = _native.unpermute(_fn["moe_unpermute"], y_perm, pair_row, topk_w, out)
        if status != _UNUSUAL:
            _check(status)
            return out
    T, k = pair_row.shape
    H = y_perm.shape[1]
    code = _dtype_code(y_perm)
    if out is None:
        out = torch.empty((T, H), dtype=y_perm.dtype, device=y_perm.device)
    _check(load().moe_unpermute(_dev(y_perm, y_perm.dtype, "y_perm"), _dev(pair_row, torch.int32, "pair_row"),
                                _dev(topk_w, torch.float32, "topk_w"), T, k, H, code,
                                _dev(out, y_perm.dtype, "out"), _stream()))
    return out


def moe_gate_topk(x: torch.Tensor, w_gate: torch.Tensor, k: int, out: Optional[dict] = None,
                  ws: Optional[torch.Tensor] = None, n_valid: Optional[torch.Tensor] = None) -> dict:
    """x [T,H], w_gate [N,H] (bf16 or f32; rows may be strided) -> dict(topk_ids [T,k] int32,
    topk_w [T,k] float32, expert_count [N] int32).  n_valid: int32 device tensor of one element, the number of
    real tokens of a padded batch (tokens past it get ids -1 and weights 0)."""
    load()
    if out is not None and ws is not None:
        status = _native.gate_topk(_fn["moe_gate_topk"], x, w_gate, k, out, ws, n_valid)
        if status != _UNUSUAL:
            _check(status)
            return out
    T, H = x.shape
    N = w_gate.shape[0]
    if w_gate.shape[1] != H or w_gate.stride(1) != 1:
        raise ValueError("w_gate must be [N,H] with contiguous rows")
    code = _dtype_code(x)
    if out is None:
        out = dict(topk_ids=torch.empty((T, k), dtype=torch.int32, device=x.device),
                   topk_w=torch.empty((T, k), dtype=torch.float32, device=x.device),
                   expert_count=torch.empty((N,), dtype=torch.int32, device=x.device))
    if ws is None:
        ws = torch.empty((int(load().moe_gate_topk_workspace_bytes(T, H, N, code)),), dtype=torch.uint8,
                         device=x.device)
    if not (w_gate.is_cuda and w_gate.dtype == x.dtype):
        raise TypeError(f"w_gate: expected a {x.dtype} device tensor")
    ldw = w_gate.stride(0) if N > 1 else H
    nv = None if n_valid is None else _dev(n_valid, torch.int32, "n_valid")
    _check(load().moe_gate_topk(_dev(x, x.dtype, "x"), w_gate.data_ptr(), ldw, T, H, N, k, code, nv,
                                _dev(out["topk_ids"], torch.int32, "topk_ids"),
                                _dev(out["topk_w"], torch.float32, "topk_w"),
                                _dev(out["expert_count"], torch.int32, "expert_count"),
                                _dev(ws, torch.uint8, "ws"), ws.numel(), _stream()))
    return out


# ------------------------------------------------------------------------------------------ sorted rows and gradients
def _on_current_device(**tensors) -> None:
    """A launch goes to the current device's stream, so that is where its tensors have to be."""
    on_gpu = {name: t.device for name, t in tensors.items() if t is not None and t.is_cuda}
    here = torch.cuda.current_device() if on_gpu else None
    for name, device in on_gpu.items():
        if device.index != here:
            raise ValueError(f"{name} is on {device}, the current device is cuda:{here}")


def _shaped(t: torch.Tensor, shape, name: str) -> torch.Tensor:
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    return t


def moe_permute_rows(x: torch.Tensor, pair_row: torch.Tensor, x_perm: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [T,H] (bf16 or f32), pair_row [T,k] int32 -> x_perm [T*k,H]: row pair_row[t,j] is x[t].  Rows that no pair names (those past
    n_pairs) are left as they were."""
    load()
    if x_perm is not None:
        status = _native.rows(_fn["moe_permute_rows"], 0, x, pair_row, x_perm)
        if status != _UNUSUAL:
            _check(status)
            return x_perm
    T, H = x.shape
    k = _shaped(pair_row, (T, pair_row.shape[-1]), "pair_row").shape[1]
    code = _dtype_code(x)
    if x_perm is None:
        x_perm = torch.empty((T * k, H), dtype=x.dtype, device=x.device)
    _on_current_device(x=x, pair_row=pair_row, x_perm=x_perm)
    _check(load().moe_permute_rows(_dev(x, x.dtype, "x"), _dev(pair_row, torch.int32, "pair_row"), T, k, H, code,
                                   _dev(_shaped(x_perm, (T * k, H), "x_perm"), x.dtype, "x_perm"), _stream()))
    return x_perm


def moe_permute_rows_backward(dx_perm: torch.Tensor, pair_row: torch.Tensor, dx: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of moe_permute_rows: dx_perm [T*k,H], pair_row [T,k] -> dx [T,H], the sum of a token's rows."""
    load()
    if dx is not None:
        status = _native.rows(_fn["moe_permute_rows_backward"], 1, dx_perm, pair_row, dx)
        if status != _UNUSUAL:
            _check(status)
            return dx
    T, k = pair_row.shape
    H = dx_perm.shape[-1]
    _shaped(dx_perm, (T * k, H), "dx_perm")
    code = _dtype_code(dx_perm)
    if dx is None:
        dx = torch.empty((T, H), dtype=dx_perm.dtype, device=dx_perm.device)
    _on_current_device(dx_perm=dx_perm, pair_row=pair_row, dx=dx)
    _check(load().moe_permute_rows_backward(_dev(dx_perm, dx_perm.dtype, "dx_perm"), _dev(pair_row, torch.int32, "pair_row"), T, k, H,
                                            code, _dev(_shaped(dx, (T, H), "dx"), dx_perm.dtype, "dx"), _stream()))
    return dx


def moe_unpermute_backward(dout: torch.Tensor, y_perm: torch.Tensor, pair_row: torch.Tensor, topk_w: torch.Tensor,
                           dy_perm: Optional[torch.Tensor] = None, dtopk_w: Optional[torch.Tensor] = None):
    """The gradient of moe_unpermute: dout [T,H], y_perm [T*k,H], pair_row [T,k], topk_w [T,k] float32 -> (dy_perm [T*k,H], of which
    rows that no pair names are left as they were; dtopk_w [T,k] float32, 0 for pairs of other ranks)."""
    load()
    if dy_perm is not None and dtopk_w is not None:
        status = _native.unpermute_backward(_fn["moe_unpermute_backward"], dout, y_perm, pair_row, topk_w, dy_perm, dtopk_w)
        if status != _UNUSUAL:
            _check(status)
            return dy_perm, dtopk_w
    T, H = dout.shape
    k = _shaped(pair_row, (T, pair_row.shape[-1]), "pair_row").shape[1]
    code = _dtype_code(dout)
    if dy_perm is None:
        dy_perm = torch.empty((T * k, H), dtype=dout.dtype, device=dout.device)
    if dtopk_w is None:
        dtopk_w = torch.empty((T, k), dtype=torch.float32, device=dout.device)
    _on_current_device(dout=dout, y_perm=y_perm, pair_row=pair_row, topk_w=topk_w, dy_perm=dy_perm, dtopk_w=dtopk_w)
    _check(load().moe_unpermute_backward(
        _dev(dout, dout.dtype, "dout"), _dev(_shaped(y_perm, (T * k, H), "y_perm"), dout.dtype, "y_perm"),
        _dev(pair_row, torch.int32, "pair_row"), _dev(_shaped(topk_w, (T, k), "topk_w"), torch.float32, "topk_w"), T, k, H, code,
        _dev(_shaped(dy_perm, (T * k, H), "dy_perm"), dout.dtype, "dy_perm"),
        _dev(_shaped(dtopk_w, (T, k), "dtopk_w"), torch.float32, "dtopk_w"), _stream()))
    return dy_perm, dtopk_w


# ------------------------------------------------------------------------------------------ 8-bit experts
FP8 = torch.float8_e4m3fn
BLOCK = 128                 # values of a row that share a scale; rows and columns of a weight block


def _blocks(n: int) -> int:
    return (n + BLOCK - 1) // BLOCK


def _fp8_matrix(t: torch.Tensor, name: str):
    """e4m3 [.., rows, K]: K contiguous, rows `ld` bytes apart (a multiple of 16), matrices rows*ld apart, and the last row's bytes up
    to a multiple of 16 inside the storage.  Returns (pointer, ld)."""
    if not (t.is_cuda and t.dtype == FP8 and t.dim() in (2, 3)):
        raise TypeError(f"{name}: expected a {FP8} device tensor of rows, got {t.dtype} on {t.device}")
    lead = t.shape[0] if t.dim() == 3 else 1
    rows, K = t.shape[-2:]
    k16 = (K + 15) // 16 * 16
    one = rows <= 1
    ld = t.stride(-2) if not one else t.stride(0) if t.dim() == 3 and lead > 1 else k16
    if (K > 1 and t.stride(-1) != 1) or ld < K or ld % 16 or ld >= 1 << 31 or (t.dim() == 3 and lead > 1 and t.stride(0) != rows * ld):
        raise TypeError(f"{name}: rows must be K-contiguous, a multiple of 16 bytes apart (strides {t.stride()})")
    if t.numel() and t.storage_offset() + (lead * rows - 1) * ld + k16 > t.untyped_storage().nbytes():
        raise ValueError(f"{name}: the last row must be readable up to a multiple of 16 bytes")
    return t.data_ptr(), ld


def quantize_buffers(R: int, K: int, device) -> Dict[str, torch.Tensor]:
    """Output buffers of moe_quantize_fp8: rows padded to a multiple of 16 bytes."""
    q = torch.empty((R, (K + 15) // 16 * 16), dtype=torch.uint8, device=device).view(FP8)
    return dict(q=q[:, :K], scale=torch.empty((R, _blocks(K)), dtype=torch.float32, device=device))


def quantize_weights_buffers(slots: int, rows: int, K: int, device) -> Dict[str, torch.Tensor]:
    """Output buffers of moe_quantize_weights_fp8: rows a multiple of 16 bytes and not of 4096 bytes apart."""
    pitch = K + BLOCK if K % 4096 == 0 else (K + 15) // 16 * 16
    q = torch.empty((slots, rows, pitch), dtype=torch.uint8, device=device).view(FP8)
    return dict(q=q[:, :, :K], scale=torch.empty((slots, _blocks(rows), _blocks(K)), dtype=torch.float32, device=device))


def moe_quantize_fp8(x: torch.Tensor, n_rows: Optional[torch.Tensor] = None,
                     out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """x [R,K] (bf16 or f32; rows may be strided) -> dict(q [R,K] e4m3, scale [R,ceil(K/128)] float32).  n_rows: int32 device tensor of
    one element, the rows to convert (those past it are left as they were)."""
    load()
    if out is not None:
        status = _native.quantize(_fn["moe_quantize_fp8"], x, n_rows, out)
        if status != _UNUSUAL:
            _check(status)
            return out
    R, K = x.shape
    code = _dtype_code(x)
    if out is None:
        out = quantize_buffers(R, K, x.device)
    _on_current_device(x=x, n_rows=n_rows, q=out["q"], scale=out["scale"])
    if not x.is_cuda or (K > 1 and x.stride(1) != 1) or (R > 1 and not K <= x.stride(0) < 1 << 31):
        raise TypeError(f"x: expected a device tensor with contiguous rows, got strides {x.stride()} on {x.device}")
    q, ldq = _fp8_matrix(_shaped(out["q"], (R, K), "q"), "q")
    nr = None if n_rows is None else _dev(_shaped(n_rows, (1,), "n_rows"), torch.int32, "n_rows")
    _check(load().moe_quantize_fp8(x.data_ptr(), x.stride(0) if R > 1 else K, R, K, code, nr, q, ldq,
                                   _dev(_shaped(out["scale"], (R, _blocks(K)), "scale"), torch.float32, "scale"), _stream()))
    return out


def moe_quantize_weights_fp8(w: torch.Tensor, out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """w [slots,rows,K] (bf16 or f32; rows may be padded) -> dict(q [slots,rows,K] e4m3, scale [slots,ceil(rows/128),ceil(K/128)]
    float32).  For w13 [spr,2I,H], whose gate and up halves have blocks of their own, pass w13.view(2*spr, I, H)."""
    S, rows, K = w.shape
    code = _dtype_code(w)
    if out is None:
        out = quantize_weights_buffers(S, rows, K, w.device)
    _on_current_device(w=w, q=out["q"], scale=out["scale"])
    p, ld = _weights(w, w.dtype, "w")
    if ld >= 1 << 31:
        raise TypeError(f"w: rows are too far apart (strides {w.stride()})")
    q, ldq = _fp8_matrix(_shaped(out["q"], (S, rows, K), "q"), "q")
    _check(load().moe_quantize_weights_fp8(p, ld, S, rows, K, code, q, ldq,
                                           _dev(_shaped(out["scale"], (S, _blocks(rows), _blocks(K)), "scale"), torch.float32, "scale"),
                                           _stream()))
    return out


def moe_grouped_mm_fp8(x: torch.Tensor, xs: torch.Tensor, group_offsets: torch.Tensor, w: torch.Tensor, ws: torch.Tensor,
                       y: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16,
                       perm_pair: Optional[torch.Tensor] = None, k: int = 1) -> torch.Tensor:
    """Rows sorted by group times their group's weights: x [R,K] e4m3, xs [R,ceil(K/128)], w [groups,N,K] e4m3,
    ws [groups,ceil(N/128),ceil(K/128)] -> y [R,N] (bf16 or f32, `dtype` where y is not given; rows past the last group are left as they
    were).  With perm_pair, x holds tokens [T,K], row r is that of token perm_pair[r] // k, and y is [T*k,N]."""
    load()
    if y is not None:
        status = _native.mm_fp8(_fn["moe_grouped_mm_fp8"], x, xs, group_offsets, w, ws, y, perm_pair, k)
        if status != _UNUSUAL:
            _check(status)
            return y
    T, K = x.shape
    groups, N, _ = w.shape
    if perm_pair is None and k != 1:
        raise ValueError("k without perm_pair")
    if k < 1 or (perm_pair is not None and perm_pair.numel() < T * k):
        raise ValueError("perm_pair must hold T*k entries")
    if y is None:
        y = torch.empty((T * k, N), dtype=dtype, device=x.device)
    _on_current_device(x=x, xs=xs, group_offsets=group_offsets, w=w, ws=ws, y=y, perm_pair=perm_pair)
    px, ldx = _fp8_matrix(x, "x")
    pw, ldw = _fp8_matrix(_shaped(w, (groups, N, K), "w"), "w")
    _check(load().moe_grouped_mm_fp8(
        px, ldx, _dev(_shaped(xs, (T, _blocks(K)), "xs"), torch.float32, "xs"),
        None if perm_pair is None else _dev(perm_pair, torch.int32, "perm_pair"),
        _dev(_shaped(group_offsets, (groups + 1,), "group_offsets"), torch.int32, "group_offsets"), T, k, groups, K, N, pw, ldw,
        _dev(_shaped(ws, (groups, _blocks(N), _blocks(K)), "ws"), torch.float32, "ws"), _dtype_code(y),
        _dev(_shaped(y, (T * k, N), "y"), y.dtype, "y"), _stream()))
    return y


def moe_grouped_ffn_fp8_workspace_bytes(T: int, k: int, spr: int, H: int, I: int) -> int:
    return int(load().moe_grouped_ffn_fp8_workspace_bytes(T, k, spr, H, I))


def moe_grouped_ffn_fp8(x: torch.Tensor, xs: torch.Tensor, perm_pair: torch.Tensor, group_offsets: torch.Tensor, k: int,
                        w13: torch.Tensor, s13: torch.Tensor, w2: torch.Tensor, s2: torch.Tensor,
                        y_perm: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                        dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """moe_grouped_ffn on 8-bit experts: x [T,H] e4m3 with xs [T,ceil(H/128)], w13 [spr,2I,H] e4m3 with s13 [spr,2*ceil(I/128),
    ceil(H/128)], w2 [spr,H,I] e4m3 with s2 [spr,ceil(H/128),ceil(I/128)] -> y_perm [T*k,H] (bf16 or f32, `dtype` where it is not given;
    rows < n_pairs written)."""
    load()
    if y_perm is not None and ws is not None:
        status = _native.ffn_fp8(_fn["moe_grouped_ffn_fp8"], x, xs, perm_pair, group_offsets, k, w13, s13, w2, s2, y_perm, ws)
        if status != _UNUSUAL:
            _check(status)
            return y_perm
    T, H = x.shape
    spr, two_i, _ = w13.shape
    I = two_i // 2
    _shaped(w13, (spr, 2 * I, H), "w13")
    _shaped(w2, (spr, H, I), "w2")
    if perm_pair.numel() < T * k:
        raise ValueError("perm_pair must hold T*k entries")
    if y_perm is None:
        y_perm = torch.empty((T * k, H), dtype=dtype, device=x.device)
    if ws is None:
        ws = torch.empty((moe_grouped_ffn_fp8_workspace_bytes(T, k, spr, H, I),), dtype=torch.uint8, device=x.device)
    _on_current_device(x=x, xs=xs, perm_pair=perm_pair, group_offsets=group_offsets, w13=w13, s13=s13, w2=w2, s2=s2, y_perm=y_perm, ws=ws)
    px, ldx = _fp8_matrix(x, "x")
    p13, ld13 = _fp8_matrix(w13, "w13")
    p2, ld2 = _fp8_matrix(w2, "w2")
    _check(load().moe_grouped_ffn_fp8(
        px, ldx, _dev(_shaped(xs, (T, _blocks(H)), "xs"), torch.float32, "xs"), _dev(perm_pair, torch.int32, "perm_pair"),
        _dev(_shaped(group_offsets, (spr + 1,), "group_offsets"), torch.int32, "group_offsets"), T, k, spr, H, I,
        p13, ld13, _dev(_shaped(s13, (spr, 2 * _blocks(I), _blocks(H)), "s13"), torch.float32, "s13"),
        p2, ld2, _dev(_shaped(s2, (spr, _blocks(H), _blocks(I)), "s2"), torch.float32, "s2"), _dtype_code(y_perm),
        _dev(_shaped(y_perm, (T * k, H), "y_perm"), y_perm.dtype, "y_perm"), _dev(ws, torch.uint8, "ws"), ws.numel(), _stream()))
    return y_perm
