"""Binding of libheterospec.so: argument marshalling only.

Every function has the name and the arguments of the C entry point it calls (see
include/heterospec.h); tensors are torch tensors on the GPU, used purely as device memory.  What a call makes
for itself (outputs and a workspace that were not given) belongs to the stream that it runs on, `stream` or the
current one, as tensors made under torch.cuda.stream(stream) do.
There is no CPU path: if the library is not built, importing this module's functions raises.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
from typing import Dict, Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libheterospec.so")
MARSHAL_PATH = os.path.join(_PKG, "_marshal.so")

HS_F32, HS_BF16 = 0, 1
HS_ERR_WORKSPACE = 4
HS_ACCEPT_GREEDY, HS_ACCEPT_STOCHASTIC, HS_ACCEPT_STOCHASTIC_POINTMASS = 0, 1, 2
HS_PSTAR_CUMULATIVE, HS_PSTAR_LOCAL = 0, 1
HS_MAX_TOPK = 64
HS_MX_E4M3, HS_MX_E2M1 = 0, 1
HS_MX_PAGE, HS_MX_BLOCK = 64, 32
HS_ROTARY_HALF, HS_ROTARY_NEIGHBOURS = 0, 1
HS_ROTARY_SCALINGS = {"none": 0, "linear": 1, "base": 2, "wavelength": 3, "yarn": 4}

_c = ctypes
_vp, _i32, _i64, _f32, _sz = _c.c_void_p, _c.c_int32, _c.c_int64, _c.c_float, _c.c_size_t

_SIGNATURES = {
    "hs_status_string": (_c.c_char_p, [_c.c_int]),
    "hs_last_error": (_c.c_char_p, []),
    "hs_version": (_c.c_char_p, []),
    "hs_draft_entropy_topk_workspace": (_sz, [_i32, _i32, _i32]),
    "hs_draft_entropy_topk": (_c.c_int, [_vp, _i64, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "hs_draft_entropy_topk_rows": (_c.c_int, [_vp, _i64, _vp, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                                              _vp]),
    "hs_draft_entropy_topk_fused": (_c.c_int, [_vp, _i64, _vp, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                                               _vp]),
    "hs_workspace_prepare": (_c.c_int, [_vp, _sz, _vp]),
    "hs_tree_prune_workspace": (_sz, [_i32, _i32]),
    "hs_tree_prune": (_c.c_int, [_vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "hs_tree_prune_static": (_c.c_int, [_vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "hs_tree_prune_counted": (_c.c_int, [_vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                         _sz, _vp]),
    "hs_tree_expand": (_c.c_int, [_vp] * 15 + [_i32] * 5 + [_vp]),
    "hs_adaptive_control": (_c.c_int, [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _i32, _vp, _i32, _i32, _i32, _i32,
                                       _c.c_int, _vp, _vp, _vp, _vp, _vp, _vp]),
    "hs_adaptive_policy": (_c.c_int, [_i32, _vp, _i32, _i32, _i32, _i32, _vp, _vp]),
    "hs_tree_attention_workspace": (_sz, [_i32, _i32, _i64, _i32, _i32, _i32, _c.c_int]),
    "hs_tree_attention": (_c.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32,
                                     _c.c_int, _f32, _vp, _vp, _vp, _sz, _vp]),
    "hs_tree_attention_shared_tree": (_c.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32,
                                                 _i32, _c.c_int, _f32, _vp, _vp, _vp, _sz, _vp]),
    "hs_tree_attention_lens": (_c.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32,
                                          _i32, _c.c_int, _f32, _vp, _vp, _vp, _sz, _vp]),
    "hs_tree_attention_paged": (_c.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp, _i32, _i32,
                                           _i32, _i32, _c.c_int, _f32, _vp, _vp, _vp, _sz, _vp]),
    "hs_kv_commit_paged": (_c.c_int, [_vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _i32, _i32, _vp, _i32, _i32, _i32,
                                      _c.c_int, _vp]),
    "hs_kv_commit": (_c.c_int, [_vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _c.c_int, _vp]),
    "hs_rotary": (_c.c_int, [_vp, _i64, _vp, _i64, _vp, _i32, _i32, _i32, _i32, _c.c_int, _vp, _i32, _c.c_int, _f32, _vp, _i64,
                             _vp, _i64, _vp]),
    "hs_tree_rotary": (_c.c_int, [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _c.c_int, _vp, _i32,
                                  _c.c_int, _f32, _vp, _i64, _vp, _i64, _vp]),
    "hs_rotary_frequencies": (_c.c_int, [_i32, _c.c_double, _c.c_int, _c.c_double, _c.c_double, _c.c_double, _c.c_double, _vp, _vp]),
    "hs_kv_append_mx": (_c.c_int, [_vp, _i64, _vp, _i64, _vp, _i32, _vp, _vp, _vp, _vp, _c.c_int, _vp, _i32, _i32, _vp, _vp, _i32,
                                   _i32, _i32, _c.c_int, _vp]),
    "hs_kv_commit_mx": (_c.c_int, [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _c.c_int, _vp, _i32, _i32, _vp,
                                   _vp, _i32, _i32, _i32, _c.c_int, _vp]),
    "hs_kv_read_mx": (_c.c_int, [_vp, _vp, _vp, _vp, _c.c_int, _vp, _i32, _i32, _vp, _vp, _i64, _vp, _vp, _i32, _i32, _i32,
                                 _c.c_int, _vp]),
    "hs_tree_attention_mx_workspace": (_sz, [_vp, _vp, _i32, _i32, _i32, _i32]),
    "hs_tree_attention_mx": (_c.c_int, [_vp, _i64, _vp, _vp, _vp, _vp, _c.c_int, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _i32, _i32,
                                        _vp, _vp, _i32, _i32, _i32, _i32, _c.c_int, _f32, _vp, _vp, _vp, _sz, _vp]),
    "hs_block_tables": (_c.c_int, [_vp, _i32, _vp, _i32, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _i32, _vp]),
    "hs_slot_map": (_c.c_int, [_vp, _i32, _vp, _vp, _i32, _vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _i32, _vp]),
    "hs_latent_store": (_c.c_int, [_vp, _i64, _vp, _i64, _vp, _i32, _vp, _i64, _i32, _i32, _c.c_int, _vp]),
    "hs_latent_read": (_c.c_int, [_vp, _i64, _vp, _i32, _vp, _i64, _vp, _i64, _i32, _i32, _c.c_int, _vp]),
    "hs_tree_attention_latent_workspace": (_sz, [_vp, _vp, _i32, _i32, _i32, _i32]),
    "hs_tree_attention_latent": (_c.c_int, [_vp, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp,
                                            _i32, _i32, _i32, _i32, _c.c_int, _f32, _vp, _i64, _i64, _vp, _vp, _sz, _vp]),
    "hs_prompt_attention_latent_workspace": (_sz, [_vp, _vp, _i32, _i32, _i32]),
    "hs_prompt_attention_latent": (_c.c_int, [_vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _vp, _i32,
                                              _i32, _i32, _i32, _i32, _c.c_int, _f32, _vp, _i64, _i64, _vp, _vp, _sz, _vp]),
    "hs_tree_validate": (_c.c_int, [_vp, _vp, _vp, _i32, _i32, _vp, _vp]),
    "hs_time_next_attention": (_c.c_int, [_vp, _vp]),
    "hs_tree_attention_last_kernel": (_c.c_int32, []),
    "hs_tree_attention_last_form": (_c.c_int32, []),
    "hs_tree_attention_plan": (_c.c_int, [_vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _i32, _c.c_int, _vp, _vp]),
    "hs_verify_accept_workspace": (_sz, [_i32, _i32, _i32]),
    "hs_verify_accept_workspace_mode": (_sz, [_i32, _i32, _i32, _c.c_int]),
    "hs_verify_accept": (_c.c_int, [_vp, _vp, _i64, _vp, _vp, _vp, _i32, _i32, _i32, _c.c_int, _f32, _vp, _i32,
                                    _vp, _vp, _vp, _vp, _sz, _vp]),
}

_lib_handle = None


class HsError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__("%s failed with status %d: %s" % (where, status, detail))
        self.status = status


def lib():
    """The loaded library; raises if it has not been built (there is no fallback)."""
    global _lib_handle
    if _lib_handle is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libheterospec.so is not built: run `python -m paper_2505_13254_amd.build` "
                               "(or __graft_entry__.build()) first")
        h = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(h, name)
            fn.restype, fn.argtypes = res, args
        _lib_handle = h
    return _lib_handle


def exported_symbols():
    return sorted(_SIGNATURES)


def _check(status: int, where: str):
    if status != 0:
        raise HsError(status, where, lib().hs_last_error().decode())


class _Calls:
    """The library's calls as functions of tensors and numbers (csrc/marshal.cpp): one native function checks the
    tensors, takes their addresses and makes the call, which returns its status.  The short calls are bound by
    what happens on the host (four calls of a tiny step: 31.9 us checked and converted in Python, now 19.6)."""
    _module = None

    def __getattr__(self, name):
        address = ctypes.cast(getattr(lib(), name), _vp).value
        if _Calls._module is None:
            if not os.path.exists(MARSHAL_PATH):
                raise RuntimeError("_marshal.so is not built: run `python -m paper_2505_13254_amd.build` first")
            spec = importlib.util.spec_from_file_location(__package__ + "._marshal", MARSHAL_PATH)
            _Calls._module = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(_Calls._module)
        fn = _Calls._module.function(name, address)
        setattr(self, name, fn)
        return fn


_calls = _Calls()


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _dev(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor on the GPU" % (name, dtype))
    return t


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """A tensor of the stream that uses it: its memory is free for that stream's next tensor alone once it is dropped, and what used
    it before ran on that stream, too.  (Memory of the current stream could be written by both at once.)"""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream)):
        return torch.empty(shape, dtype=dtype, device=device)


def workspace(nbytes: int, device, stream=None) -> Optional[torch.Tensor]:
    """A 256-byte aligned scratch buffer (torch's allocator aligns to at least 512 bytes), for calls on `stream`."""
    if nbytes == 0:
        return None
    return _empty(nbytes, torch.uint8, device, stream)


def hs_workspace_prepare(ws: Optional[torch.Tensor], stream=None) -> None:
    """Clears a workspace tensor on the GPU (what hs_draft_entropy_topk_fused asks of its workspace)."""
    if ws is None:
        return
    _check(lib().hs_workspace_prepare(_ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), "hs_workspace_prepare")


def hs_draft_entropy_topk(logits: torch.Tensor, K: int, temperature: float = 1.0, *, want_full: bool = True,
                          out: Optional[Dict[str, torch.Tensor]] = None, ws: Optional[torch.Tensor] = None,
                          row_index: Optional[torch.Tensor] = None, fused: bool = False,
                          stream=None) -> Dict[str, torch.Tensor]:
    """logits float32 [N, V] (row stride may exceed V).  Returns topk_idx, topk_logp, ent_topk, ent_full, lse
    for its N rows, or, with row_index int32 [R] (GPU), for the R rows that row_index names
    (hs_draft_entropy_topk_rows; a negative entry leaves that result row untouched).
    fused: hs_draft_entropy_topk_fused (one launch); `ws` must then be given and PREPARED
    (hs_workspace_prepare, and only completed fused calls on it since)."""
    if logits.dim() != 2 or logits.dtype != torch.float32 or not logits.is_cuda or logits.stride(1) != 1:
        raise ValueError("logits must be a float32 [R, V] GPU tensor with unit inner stride")
    N, V = logits.shape
    R = N
    if row_index is not None:
        R = row_index.numel()
    if out is None:
        dev = logits.device
        out = dict(topk_idx=_empty((R, K), torch.int32, dev, stream),
                   topk_logp=_empty((R, K), torch.float32, dev, stream),
                   ent_topk=_empty(R, torch.float32, dev, stream))
        if want_full:
            out["ent_full"] = _empty(R, torch.float32, dev, stream)
            out["lse"] = _empty(R, torch.float32, dev, stream)
    if ws is None and not fused:
        ws = workspace(lib().hs_draft_entropy_topk_workspace(R, V, K), logits.device, stream)
    stride = logits.stride(0) if N > 1 else max(V, logits.stride(0))
    tail = (R, V, K, temperature, out["topk_idx"], out["topk_logp"], out["ent_topk"], out.get("ent_full"), out.get("lse"), ws,
            stream)
    if fused:
        st = HS_ERR_WORKSPACE if ws is None else _calls.hs_draft_entropy_topk_fused(logits, stride, row_index, *tail)
        if st == HS_ERR_WORKSPACE:
            need = lib().hs_draft_entropy_topk_workspace(R, V, K)
            if ws is None or ws.numel() < need:
                raise ValueError("the fused call needs a prepared workspace of at least %d bytes" % need)
    elif row_index is None:
        st = _calls.hs_draft_entropy_topk(logits, stride, *tail)
    else:
        st = _calls.hs_draft_entropy_topk_rows(logits, stride, row_index, *tail)
    _check(st, "hs_draft_entropy_topk")
    return out


def hs_tree_prune(parent: torch.Tensor, logc: torch.Tensor, node_offsets: torch.Tensor, d_max: torch.Tensor,
                  theta: torch.Tensor, max_nodes: torch.Tensor, *, node_counts: Optional[torch.Tensor] = None,
                  out: Optional[Dict[str, torch.Tensor]] = None,
                  ws: Optional[torch.Tensor] = None, stream=None) -> Dict[str, torch.Tensor]:
    """All arguments are GPU tensors: parent int32 [NN], logc float32 [NN], node_offsets int32 [B+1],
    d_max int32 [B], theta float32 [B], max_nodes int32 [B].  Returns depth, cumlogp, keep, out_offsets,
    out_src, out_parent (the last two sized NN; the first out_offsets[B] entries are valid).
    With node_counts int32 [B] the call is hs_tree_prune_counted (trees stored with spare capacity)."""
    NN, B = parent.numel(), node_offsets.numel() - 1
    if out is None:
        dev = parent.device
        out = dict(depth=_empty(NN, torch.int32, dev, stream),
                   cumlogp=_empty(NN, torch.float32, dev, stream),
                   keep=_empty(NN, torch.uint8, dev, stream),
                   out_offsets=_empty(B + 1, torch.int32, dev, stream),
                   out_src=_empty(max(NN, 1), torch.int32, dev, stream),
                   out_parent=_empty(max(NN, 1), torch.int32, dev, stream))
    if ws is None:
        ws = workspace(lib().hs_tree_prune_workspace(B, NN), parent.device, stream)
    tail = (B, NN, d_max, theta, max_nodes, out["depth"], out["cumlogp"], out["keep"], out["out_offsets"], out["out_src"],
            out["out_parent"], ws, stream)
    if node_counts is None:
        st = _calls.hs_tree_prune(parent, logc, node_offsets, *tail)
    else:
        st = _calls.hs_tree_prune_counted(parent, logc, node_offsets, node_counts, *tail)
    _check(st, "hs_tree_prune")
    return out


def hs_tree_prune_static(parent: torch.Tensor, logc: torch.Tensor, node_offsets: torch.Tensor, d_max: torch.Tensor,
                         theta: torch.Tensor, max_nodes: torch.Tensor, *, out: Dict[str, torch.Tensor],
                         stream=None) -> Dict[str, torch.Tensor]:
    """hs_tree_prune on the library's own static scratch: no workspace, and `out` (depth, cumlogp, keep,
    out_offsets, out_src, out_parent as hs_tree_prune returns them) must be given, so the call allocates
    nothing."""
    _dev(parent, torch.int32, "parent"); _dev(logc, torch.float32, "logc")
    _dev(node_offsets, torch.int32, "node_offsets"); _dev(d_max, torch.int32, "d_max")
    _dev(theta, torch.float32, "theta"); _dev(max_nodes, torch.int32, "max_nodes")
    NN, B = parent.numel(), node_offsets.numel() - 1
    st = lib().hs_tree_prune_static(_ptr(parent), _ptr(logc), _ptr(node_offsets), B, NN, _ptr(d_max), _ptr(theta),
                                    _ptr(max_nodes), _ptr(out["depth"]), _ptr(out["cumlogp"]), _ptr(out["keep"]),
                                    _ptr(out["out_offsets"]), _ptr(out["out_src"]), _ptr(out["out_parent"]),
                                    _stream(stream))
    _check(st, "hs_tree_prune_static")
    return out


def new_tree_state(B: int, cap: int, F: int, device) -> Dict[str, torch.Tensor]:
    """Device arrays of hs_tree_expand's draft-tree state (uninitialised: the first call initialises them)."""
    i32 = dict(dtype=torch.int32, device=device)
    f32 = dict(dtype=torch.float32, device=device)
    return dict(parent=torch.empty(B * cap, **i32), token=torch.empty(B * cap, **i32), depth=torch.empty(B * cap, **i32),
                logc=torch.empty(B * cap, **f32), cumlogp=torch.empty(B * cap, **f32), ent=torch.empty(B * cap, **f32),
                n_nodes=torch.empty(B, **i32), level=torch.empty(B, **i32), frontier=torch.empty(B * F, **i32),
                n_frontier=torch.empty(B, **i32), frontier_rows=torch.empty(B * F, **i32),
                node_offsets=(torch.arange(B + 1, dtype=torch.int64) * cap).to(torch.int32).to(device))


def hs_tree_expand(state: Dict[str, torch.Tensor], topk_idx, topk_logp, ent_topk, d_limit, B: int, cap: int, F: int,
                   K: int, first: bool, *, stream=None) -> Dict[str, torch.Tensor]:
    """state: the tensors of new_tree_state(); topk_idx int32 [B*F, K], topk_logp float32 [B*F, K], ent_topk
    float32 [B*F] (hs_draft_entropy_topk's results for the frontier slots); d_limit int32 [B] or None."""
    if topk_idx.numel() < B * F * K or ent_topk.numel() < B * F:
        raise ValueError("Top-K results must cover B * F frontier slots")
    if state["parent"].numel() < B * cap or state["frontier"].numel() < B * F:
        raise ValueError("state arrays are smaller than B * cap / B * F")
    st = _calls.hs_tree_expand(state["parent"], state["token"], state["logc"], state["cumlogp"], state["depth"], state["ent"],
                               state["n_nodes"], state["level"], state["frontier"], state["n_frontier"], state["frontier_rows"],
                               topk_idx, topk_logp, ent_topk, d_limit, B, cap, F, K, 1 if first else 0, stream)
    _check(st, "hs_tree_expand")
    return state


def hs_adaptive_control(parent, logc, ent, node_offsets, node_counts, bin_edges, gamma, alpha: int, d_base: int,
                        n_default: int, mode: int = 0, *, out: Optional[Dict[str, torch.Tensor]] = None,
                        stream=None) -> Dict[str, torch.Tensor]:
    """parent int32 [NN], logc / ent float32 [NN], node_offsets int32 [B+1], node_counts int32 [B] or None (GPU);
    bin_edges (ascending, n_bins - 1 values) and gamma are host sequences of floats.
    Returns phi float32 [B] and pstar, bin, d_prime, n_prime int32 [B]."""
    B, NN = node_offsets.numel() - 1, parent.numel()
    if out is None:
        dev = parent.device
        out = dict(phi=_empty(B, torch.float32, dev, stream))
        for k in ("pstar", "bin", "d_prime", "n_prime"):
            out[k] = _empty(B, torch.int32, dev, stream)
    st = _calls.hs_adaptive_control(parent, logc, ent, node_offsets, node_counts, B, NN, bin_edges, len(bin_edges) + 1, gamma,
                                    len(gamma), int(alpha), int(d_base), int(n_default), int(mode), out["phi"], out["pstar"],
                                    out["bin"], out["d_prime"], out["n_prime"], stream)
    _check(st, "hs_adaptive_control")
    return out


def hs_adaptive_policy(bin: int, gamma, alpha: int, d_base: int, n_default: int):
    """(d_prime, n_prime) of entropy bin `bin`, from the library's own formula (host arithmetic only)."""
    gam = (_f32 * max(1, len(gamma)))(*[float(x) for x in gamma])
    dp, np_ = _i32(0), _i32(0)
    st = lib().hs_adaptive_policy(int(bin), _c.cast(gam, _vp), len(gamma), int(alpha), int(d_base), int(n_default),
                                  _c.byref(dp), _c.byref(np_))
    _check(st, "hs_adaptive_policy")
    return int(dp.value), int(np_.value)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return HS_F32
    if t.dtype == torch.bfloat16:
        return HS_BF16
    raise ValueError("q/k/v must be float32 or bfloat16")


def hs_tree_attention(q, k_prefix, v_prefix, k_tree, v_tree, parent, node_offsets, prefix_offsets,
                      host_node_offsets, host_prefix_offsets, scale: float, *, want_lse: bool = False,
                      out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                      ws: Optional[torch.Tensor] = None, stream=None,
                      prefix_lens: Optional[torch.Tensor] = None, host_prefix_lens: Optional[torch.Tensor] = None,
                      shared_tree: bool = False):
    """q [NN,Hq,D]; k_prefix, v_prefix [total_prefix,Hkv,D]; k_tree, v_tree [NN,Hkv,D] (float32 or bfloat16, GPU);
    parent int32 [NN], node_offsets int32 [B+1], prefix_offsets int64 [B+1] on the GPU and the same two offset
    arrays on the host (CPU tensors).  Returns (o [NN,Hq,D], lse [NN,Hq] or None).
    With prefix_lens (int64 [B], GPU) and host_prefix_lens (the same on the CPU) the call is
    hs_tree_attention_lens: prefix_offsets then delimit cache regions with spare capacity.
    shared_tree: the call is hs_tree_attention_shared_tree: parent int32 [M] is one tree that all B entries
    (of M rows each) use."""
    NN, Hq, D = q.shape
    Hkv = k_tree.shape[1]
    B = host_node_offsets.numel() - 1
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    if want_lse and lse is None:
        lse = _empty((NN, Hq), torch.float32, q.device, stream)
    if ws is None:
        ws = workspace(lib().hs_tree_attention_workspace(B, NN, int(host_prefix_offsets[-1]), Hq, Hkv, D, _dtype_code(q)), q.device, stream)
    if shared_tree:
        if prefix_lens is not None:
            raise ValueError("shared_tree and prefix_lens cannot be combined")
        st = _calls.hs_tree_attention_shared_tree(q, k_prefix, v_prefix, k_tree, v_tree, parent, node_offsets, prefix_offsets,
                                                  host_node_offsets, host_prefix_offsets, B, Hq, Hkv, D, scale, out, lse, ws, stream)
    elif prefix_lens is None:
        st = _calls.hs_tree_attention(q, k_prefix, v_prefix, k_tree, v_tree, parent, node_offsets, prefix_offsets,
                                      host_node_offsets, host_prefix_offsets, B, Hq, Hkv, D, scale, out, lse, ws, stream)
    else:
        st = _calls.hs_tree_attention_lens(q, k_prefix, v_prefix, k_tree, v_tree, parent, node_offsets, prefix_offsets,
                                           host_node_offsets, host_prefix_offsets, prefix_lens, host_prefix_lens, B, Hq, Hkv, D,
                                           scale, out, lse, ws, stream)
    _check(st, "hs_tree_attention")
    return out, lse


def hs_tree_attention_paged(q, k_pages, v_pages, k_tree, v_tree, parent, node_offsets, host_node_offsets, block_table,
                            prefix_lens, host_prefix_lens, scale: float, *, want_lse: bool = False,
                            out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                            ws: Optional[torch.Tensor] = None, stream=None):
    """q [NN,Hq,D]; k_pages, v_pages [n_pages, page_tokens, Hkv, D]; k_tree, v_tree [NN,Hkv,D]; parent int32 [NN],
    node_offsets int32 [B+1], block_table int32 [B, max_blocks], prefix_lens int64 [B] on the GPU;
    host_node_offsets and host_prefix_lens the same on the CPU.  Returns (o, lse or None)."""
    NN, Hq, D = q.shape
    Hkv = k_tree.shape[1]
    B = host_node_offsets.numel() - 1
    if block_table.dim() != 2 or block_table.shape[0] != B or k_pages.dim() != 4:
        raise ValueError("block_table must be [B, max_blocks] and the pools [n_pages, page_tokens, Hkv, D]")
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    if want_lse and lse is None:
        lse = _empty((NN, Hq), torch.float32, q.device, stream)
    if ws is None:
        ws = workspace(lib().hs_tree_attention_workspace(B, NN, int(host_prefix_lens.sum()), Hq, Hkv, D, _dtype_code(q)), q.device, stream)
    st = _calls.hs_tree_attention_paged(q, k_pages, v_pages, k_tree, v_tree, parent, node_offsets, host_node_offsets, block_table,
                                        block_table.shape[1], k_pages.shape[1], prefix_lens, host_prefix_lens, B, Hq, Hkv, D,
                                        scale, out, lse, ws, stream)
    _check(st, "hs_tree_attention_paged")
    return out, lse


def hs_kv_commit_paged(k_tree, v_tree, node_offsets, accept_path, accept_len, k_pages, v_pages, block_table, cache_lens,
                       *, stream=None):
    """As hs_kv_commit, into pools k_pages, v_pages [n_pages, page_tokens, Hkv, D] through block_table int32
    [B, max_blocks]; cache_lens int64 [B] is updated in place."""
    Hkv, D = k_tree.shape[1], k_tree.shape[2]
    st = _calls.hs_kv_commit_paged(k_tree, v_tree, node_offsets, accept_path, accept_len, accept_path.shape[1], k_pages, v_pages,
                                   block_table, block_table.shape[1], k_pages.shape[1], cache_lens, node_offsets.numel() - 1,
                                   Hkv, D, stream)
    _check(st, "hs_kv_commit_paged")
    return cache_lens


def hs_kv_commit(k_tree, v_tree, node_offsets, accept_path, accept_len, k_cache, v_cache, cache_offsets, cache_lens,
                 *, stream=None):
    """k_tree, v_tree [NN,Hkv,D] and k_cache, v_cache [capacity,Hkv,D] of one element type; node_offsets int32
    [B+1], accept_path int32 [B,max_depth], accept_len int32 [B], cache_offsets int64 [B+1], cache_lens int64
    [B] (updated in place); all on the GPU."""
    B = node_offsets.numel() - 1
    if accept_path.dim() != 2 or accept_path.shape[0] != B or accept_len.numel() != B or cache_lens.numel() != B:
        raise ValueError("accept_path must be [B, max_depth]; accept_len and cache_lens [B]")
    Hkv, D = k_tree.shape[1], k_tree.shape[2]
    st = _calls.hs_kv_commit(k_tree, v_tree, node_offsets, accept_path, accept_len, accept_path.shape[1], k_cache, v_cache,
                             cache_offsets, cache_lens, B, Hkv, D, stream)
    _check(st, "hs_kv_commit")
    return cache_lens


def hs_rotary_frequencies(rot_dim: int, base: float = 10000.0, *, scaling: str = "none", factor: float = 1.0, context: float = 0.0,
                          low: float = 1.0, high: float = 4.0, device=None):
    """The table of a rotation: (inv_freq float64 [rot_dim / 2] on `device`, mscale).  scaling: "none", "linear", "base",
    "wavelength" or "yarn" (whose usual low and high are 1 and 32)."""
    if scaling not in HS_ROTARY_SCALINGS:
        raise ValueError("scaling must be one of %s" % ", ".join(HS_ROTARY_SCALINGS))
    table = torch.empty(max(0, int(rot_dim)) // 2, dtype=torch.float64)
    m = _f32(1.0)
    _check(lib().hs_rotary_frequencies(int(rot_dim), float(base), HS_ROTARY_SCALINGS[scaling], float(factor), float(context), float(low),
                                       float(high), table.data_ptr(), _c.byref(m)), "hs_rotary_frequencies")
    return table if device is None else table.to(device), float(m.value)


def _rotary_args(q, k, inv_freq, q_out, k_out, stream):
    if q.dim() != 3 or (k is not None and (k.dim() != 3 or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2])):
        raise ValueError("q and k must be [N, heads, D] with the same N and D")
    if q_out is None:
        q_out = _empty(q.shape, q.dtype, q.device, stream)
    if k_out is None and k is not None:
        k_out = _empty(k.shape, k.dtype, k.device, stream)
    if q_out.shape != q.shape or (k_out is None) != (k is None) or (k is not None and k_out.shape != k.shape):
        raise ValueError("outputs must have their inputs' shapes")
    return q_out, k_out, (0 if k is None else k.shape[1])


def hs_rotary(q, k, positions, inv_freq, *, interleaved: bool = False, mscale: float = 1.0, q_out=None, k_out=None, stream=None):
    """q [N,Hq,D], k [N,Hkv,D] or None (float32 or bfloat16, GPU; rows may have a stride of their own, e.g. slices of a fused
    projection), positions int64 [N], inv_freq float64 [rot_dim / 2] on the GPU (hs_rotary_frequencies).  interleaved: pairs
    are neighbours, otherwise halves.  q_out / k_out may be q / k themselves.  Returns (q_out, k_out)."""
    q_out, k_out, Hkv = _rotary_args(q, k, inv_freq, q_out, k_out, stream)
    N, Hq, D = q.shape
    if positions.numel() != N:
        raise ValueError("positions must hold N values")
    _check(_calls.hs_rotary(q, k, positions, N, Hq, Hkv, D, inv_freq, 2 * inv_freq.numel(),
                            HS_ROTARY_NEIGHBOURS if interleaved else HS_ROTARY_HALF, mscale, q_out, k_out, stream), "hs_rotary")
    return q_out, k_out


def hs_tree_rotary(q, k, parent, node_offsets, prefix_lens, inv_freq, *, interleaved: bool = False, mscale: float = 1.0, q_out=None,
                   k_out=None, stream=None):
    """hs_rotary of the rows of draft trees (parent int32 [N], node_offsets int32 [B+1], GPU): a row's position is
    prefix_lens[s] (int64 [B], GPU) plus its depth."""
    q_out, k_out, Hkv = _rotary_args(q, k, inv_freq, q_out, k_out, stream)
    N, Hq, D = q.shape
    B = node_offsets.numel() - 1
    if parent.numel() != N or prefix_lens.numel() != B:
        raise ValueError("parent must hold N values, prefix_lens B")
    _check(_calls.hs_tree_rotary(q, k, parent, node_offsets, prefix_lens, B, N, Hq, Hkv, D, inv_freq, 2 * inv_freq.numel(),
                                 HS_ROTARY_NEIGHBOURS if interleaved else HS_ROTARY_HALF, mscale, q_out, k_out, stream), "hs_tree_rotary")
    return q_out, k_out


def new_mx_cache(n_pages: int, Hkv: int, D: int, fmt: int = HS_MX_E4M3, device="cuda:0") -> Dict[str, torch.Tensor]:
    """Pools of a quantised cache (uninitialised): k_codes, v_codes [n_pages, Hkv, 64, D] float8_e4m3fn, or
    [n_pages, Hkv, 64, D / 2] uint8 (two 4-bit elements to a byte), and k_scales, v_scales uint8 [n_pages, Hkv, 64, D / 32]."""
    if fmt not in (HS_MX_E4M3, HS_MX_E2M1) or D % HS_MX_BLOCK != 0:
        raise ValueError("fmt must be HS_MX_E4M3 or HS_MX_E2M1, D a multiple of %d" % HS_MX_BLOCK)
    wide, kind = (D, torch.float8_e4m3fn) if fmt == HS_MX_E4M3 else (D // 2, torch.uint8)
    c = {}
    for n in ("k", "v"):
        c[n + "_codes"] = torch.empty((n_pages, Hkv, HS_MX_PAGE, wide), dtype=kind, device=device)
        c[n + "_scales"] = torch.empty((n_pages, Hkv, HS_MX_PAGE, D // HS_MX_BLOCK), dtype=torch.uint8, device=device)
    return c


def _mx_cache(cache, block_table, B):
    """(k_codes, k_scales, v_codes, v_scales, format), pages, Hkv, D of a cache as new_mx_cache makes it."""
    kc, ks, vc, vs = cache["k_codes"], cache["k_scales"], cache["v_codes"], cache["v_scales"]
    fmt = HS_MX_E4M3 if kc.dtype == torch.float8_e4m3fn else HS_MX_E2M1
    if kc.dim() != 4 or ks.dim() != 4 or kc.shape[2] != HS_MX_PAGE:
        raise ValueError("a cache's codes must be [n_pages, Hkv, %d, D] and its scales [n_pages, Hkv, %d, D / %d]" % (HS_MX_PAGE, HS_MX_PAGE, HS_MX_BLOCK))
    n_pages, Hkv, _, wide = kc.shape
    D = wide if fmt == HS_MX_E4M3 else 2 * wide
    if vc.dtype != kc.dtype or vc.shape != kc.shape or vs.shape != ks.shape or tuple(ks.shape) != (n_pages, Hkv, HS_MX_PAGE, D // HS_MX_BLOCK):
        raise ValueError("the cache's four tensors do not fit each other")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table must be [B, max_blocks]")
    return (kc, ks, vc, vs, fmt), n_pages, Hkv, D


def _mx_store_args(k, v, cache, block_table, cache_lens, new_lens, B):
    pool, n_pages, Hkv, D = _mx_cache(cache, block_table, B)
    if k.dim() != 3 or k.shape != v.shape or k.shape[1] != Hkv or k.shape[2] != D:
        raise ValueError("k and v must be [NN, Hkv, D] of the cache's Hkv and D")
    if cache_lens.numel() != B or (new_lens is not None and new_lens.numel() != B):
        raise ValueError("cache_lens and new_lens must hold B values")
    return pool, (block_table, block_table.shape[1], n_pages, cache_lens, new_lens, B, Hkv, D)


def hs_kv_append_mx(k, v, node_offsets, cache, block_table, cache_lens, *, new_lens=None, stream=None) -> None:
    """k, v [NN,Hkv,D] (float32 or bfloat16, GPU; rows may have a stride of their own): rows node_offsets[s] .. of sequence s
    (int32 [B+1]) become its tokens cache_lens[s] .. (int64 [B], left alone) in `cache` (new_mx_cache) through block_table int32
    [B, max_blocks].  new_lens (int64 [B] or None) receives the lengths afterwards."""
    pool, rest = _mx_store_args(k, v, cache, block_table, cache_lens, new_lens, node_offsets.numel() - 1)
    _check(_calls.hs_kv_append_mx(k, v, node_offsets, k.shape[0], *pool, *rest, stream), "hs_kv_append_mx")


def hs_kv_commit_mx(k_tree, v_tree, node_offsets, accept_path, accept_len, cache, block_table, cache_lens, *, new_lens=None,
                    stream=None) -> None:
    """As hs_kv_append_mx, with the tree's root and the accepted rows (accept_path int32 [B, max_depth], accept_len int32 [B], as
    hs_verify_accept writes them)."""
    B = node_offsets.numel() - 1
    pool, rest = _mx_store_args(k_tree, v_tree, cache, block_table, cache_lens, new_lens, B)
    if accept_path.dim() != 2 or accept_path.shape[0] != B or accept_len.numel() != B:
        raise ValueError("accept_path must be [B, max_depth], accept_len [B]")
    _check(_calls.hs_kv_commit_mx(k_tree, v_tree, node_offsets, accept_path, accept_len, accept_path.shape[1], *pool, *rest, stream),
           "hs_kv_commit_mx")


def hs_kv_read_mx(cache, block_table, out_offsets, total: int, *, first=None, dtype=torch.bfloat16, out=None, stream=None):
    """Tokens first[s] .. (int64 [B], GPU; None: from 0) of sequence s as rows out_offsets[s] .. out_offsets[s+1] - 1 (int64 [B+1],
    GPU; total = the last) of two tensors [total, Hkv, D], `out` or new ones of `dtype`.  Returns (k, v)."""
    B = out_offsets.numel() - 1
    pool, n_pages, Hkv, D = _mx_cache(cache, block_table, B)
    if out is None:
        out = tuple(_empty((total, Hkv, D), dtype, block_table.device, stream) for _ in range(2))
    if any(tuple(t.shape) != (total, Hkv, D) for t in out) or (first is not None and first.numel() != B):
        raise ValueError("out must be two tensors [total, Hkv, D], first must hold B values")
    _check(_calls.hs_kv_read_mx(*pool, block_table, block_table.shape[1], n_pages, first, out_offsets, total, out[0], out[1], B, Hkv, D,
                                stream), "hs_kv_read_mx")
    return out[0], out[1]


def hs_tree_attention_mx_workspace(host_node_offsets, host_prefix_lens, Hq: int, Hkv: int, D: int, device, *, stream=None) -> Optional[torch.Tensor]:
    """A workspace for hs_tree_attention_mx calls of these row counts and lengths (CPU tensors) on `stream`; None where none is needed."""
    if host_node_offsets.numel() != host_prefix_lens.numel() + 1:
        raise ValueError("the offsets must hold B + 1 values, the lengths B")
    no, pl = host_node_offsets.to("cpu", torch.int32).contiguous(), host_prefix_lens.to("cpu", torch.int64).contiguous()
    n = lib().hs_tree_attention_mx_workspace(no.data_ptr(), pl.data_ptr(), no.numel() - 1, int(Hq), int(Hkv), int(D))
    return workspace(n, device, stream)


def hs_tree_attention_mx(q, cache, k_tree, v_tree, parent, node_offsets, host_node_offsets, block_table, prefix_lens,
                         host_prefix_lens, scale: float, *, want_lse: bool = False, out: Optional[torch.Tensor] = None,
                         lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """hs_tree_attention_paged on a quantised cache (new_mx_cache): q [NN,Hq,D], k_tree, v_tree [NN,Hkv,D] bfloat16 (GPU; rows may
    have a stride of their own).  Returns (o [NN,Hq,D], lse [NN,Hq] or None)."""
    if q.dim() != 3:
        raise ValueError("q must be [NN, Hq, D]")
    NN, Hq, D = q.shape
    B = host_node_offsets.numel() - 1
    pool, n_pages, Hkv, cache_D = _mx_cache(cache, block_table, B)
    if cache_D != D or tuple(k_tree.shape) != (NN, Hkv, D) or v_tree.shape != k_tree.shape:
        raise ValueError("k_tree and v_tree must be [NN, Hkv, D] of the cache's Hkv, and D that of q")
    if parent.numel() != NN or node_offsets.numel() != B + 1 or prefix_lens.numel() != B or host_prefix_lens.numel() != B or \
            int(host_node_offsets[B]) != NN:
        raise ValueError("parent must hold NN values, the offsets B + 1 (the last one NN), the lengths B")
    if out is None:
        out = _empty((NN, Hq, D), q.dtype, q.device, stream)
    if want_lse and lse is None:
        lse = _empty((NN, Hq), torch.float32, q.device, stream)
    if out.shape != q.shape or (lse is not None and lse.numel() != NN * Hq):
        raise ValueError("out must be [NN, Hq, D], lse [NN, Hq]")
    if ws is None:
        ws = hs_tree_attention_mx_workspace(host_node_offsets, host_prefix_lens, Hq, Hkv, D, q.device, stream=stream)
    _check(_calls.hs_tree_attention_mx(q, *pool, k_tree, v_tree, parent, node_offsets, host_node_offsets, block_table,
                                       block_table.shape[1], n_pages, prefix_lens, host_prefix_lens, B, Hq, Hkv, D, scale, out, lse, ws,
                                       stream), "hs_tree_attention_mx")
    return out, lse


def new_page_tables(B: int, max_blocks: int, n_pages: int, device="cuda:0") -> Dict[str, torch.Tensor]:
    """The tables of B sequences over a pool of n_pages free pages, as hs_block_tables takes them: block_table int32 [B, max_blocks], held
    int32 [B], free_pages int32 [n_pages] (page 0 comes first), free_count int32 [1]."""
    i32 = dict(dtype=torch.int32, device=device)
    return dict(block_table=torch.full((B, max_blocks), -1, **i32), held=torch.zeros(B, **i32), free_pages=torch.arange(n_pages - 1, -1, -1, **i32),
                free_count=torch.full((1,), n_pages, **i32))


def hs_block_tables(want, block_table, held, free_pages, free_count, *, page_tokens: int = HS_MX_PAGE, new_held=None, new_free_count=None, refused=None,
                    stream=None):
    """Pages for want[s] tokens (int64 [B], GPU) of every sequence: block_table int32 [B, max_blocks] and free_pages int32 [n_pages] are updated in
    place, held int32 [B] and free_count int32 [1] are left alone.  refused: int32 [B] or None.  Returns (new_held, new_free_count); of no
    sequences the count as it was."""
    B = want.numel()
    if block_table.dim() != 2 or block_table.shape[0] != B or held.numel() != B:
        raise ValueError("block_table must be [B, max_blocks], held [B]")
    if new_held is None:
        new_held = _empty(B, torch.int32, want.device, stream)
    if new_free_count is None:
        new_free_count = _empty(1, torch.int32, want.device, stream)
    if new_held.numel() != B or free_count.numel() != 1 or new_free_count.numel() != 1 or (refused is not None and refused.numel() != B):
        raise ValueError("new_held and refused must hold B values, the counts one")
    _check(_calls.hs_block_tables(want, page_tokens, block_table, block_table.shape[1], held, new_held, free_pages, free_pages.numel(), free_count,
                                  new_free_count, refused, B, stream), "hs_block_tables")
    return new_held, new_free_count


def hs_slot_map(node_offsets, NN: int, cache_lens, block_table, n_pages: int, *, page_tokens: int = HS_MX_PAGE, held=None, accept_path=None,
                accept_len=None, slots=None, new_lens=None, stream=None):
    """Slots (int64 [NN]) of the rows node_offsets[s] .. of sequence s (int32 [B+1]) behind its cache_lens[s] tokens (int64 [B]) in a pool of n_pages
    pages, -1 for a row without one.  With accept_path int32 [B, max_depth] and accept_len int32 [B]: of a tree's root and accepted rows.  held int32 [B]
    or None: pages of block_table int32 [B, max_blocks] that a sequence has.  new_lens (int64 [B] or None) receives the lengths afterwards."""
    B = node_offsets.numel() - 1
    if block_table.dim() != 2 or block_table.shape[0] != B or cache_lens.numel() != B:
        raise ValueError("block_table must be [B, max_blocks], cache_lens [B]")
    if (held is not None and held.numel() != B) or (new_lens is not None and new_lens.numel() != B):
        raise ValueError("held and new_lens must hold B values")
    if (accept_path is None) != (accept_len is None) or (accept_path is not None and
                                                         (accept_path.dim() != 2 or accept_path.shape[0] != B or accept_len.numel() != B)):
        raise ValueError("accept_path must be [B, max_depth], accept_len [B], both or neither")
    if slots is None:
        slots = _empty(NN, torch.int64, node_offsets.device, stream)
    if slots.numel() != NN:
        raise ValueError("slots must hold NN values")
    _check(_calls.hs_slot_map(node_offsets, NN, accept_path, accept_len, 0 if accept_path is None else accept_path.shape[1], block_table,
                              block_table.shape[1], page_tokens, n_pages, held, cache_lens, slots, new_lens, B, stream), "hs_slot_map")
    return slots


def new_latent_cache(n_pages: int, R: int, Dr: int, dtype=torch.bfloat16, device="cuda:0") -> torch.Tensor:
    """The pool of a paged cache of latents (uninitialised): [n_pages, 64, R + Dr], a token's latent and behind it its rotary part."""
    return torch.empty((n_pages, HS_MX_PAGE, R + Dr), dtype=dtype, device=device)


def _latent_pool(pool, R: int, Dr: int):
    if pool.dim() != 3 or pool.shape[2] != R + Dr:
        raise ValueError("the pool must be [n_pages, page_tokens, R + Dr]")
    return pool.shape[0] * pool.shape[1]


def hs_latent_store(c, r, slots, pool, *, stream=None) -> None:
    """Rows c [N, R] and r [N, Dr] (float32 or bfloat16, GPU; rows may have a stride of their own) go to slots (int64 [N]; one that the pool does not
    have: the row goes nowhere) of `pool` (new_latent_cache)."""
    if c.dim() != 2 or r.dim() != 2 or r.shape[0] != c.shape[0] or slots.numel() != c.shape[0]:
        raise ValueError("c must be [N, R], r [N, Dr], slots [N]")
    n = _latent_pool(pool, c.shape[1], r.shape[1])
    _check(_calls.hs_latent_store(c, r, slots, c.shape[0], pool, n, c.shape[1], r.shape[1], stream), "hs_latent_store")


def hs_latent_read(pool, slots, R: int, *, out=None, stream=None):
    """Rows (c [N, R], r [N, Dr]) at slots (int64 [N]) of a pool, `out` or new ones.  Rows without a slot are left as they were."""
    N = slots.numel()
    if out is None:
        out = tuple(_empty((N, n), pool.dtype, pool.device, stream) for n in (R, pool.shape[-1] - R))
    c, r = out
    if c.dim() != 2 or r.dim() != 2 or c.shape[0] != N or r.shape[0] != N or c.shape[1] != R:
        raise ValueError("out must be two tensors [N, R] and [N, Dr]")
    n = _latent_pool(pool, R, r.shape[1])
    _check(_calls.hs_latent_read(pool, n, slots, N, c, r, R, r.shape[1], stream), "hs_latent_read")
    return c, r


def hs_tree_attention_latent_workspace(host_node_offsets, host_prefix_lens, Hq: int, R: int, Dr: int, device, *, stream=None) -> Optional[torch.Tensor]:
    """A workspace for hs_tree_attention_latent calls of these row counts and lengths (CPU tensors) on `stream`; None where none is needed."""
    if host_node_offsets.numel() != host_prefix_lens.numel() + 1:
        raise ValueError("the offsets must hold B + 1 values, the lengths B")
    no, pl = host_node_offsets.to("cpu", torch.int32).contiguous(), host_prefix_lens.to("cpu", torch.int64).contiguous()
    n = lib().hs_tree_attention_latent_workspace(no.data_ptr(), pl.data_ptr(), no.numel() - 1, int(Hq), int(R), int(Dr))
    return workspace(n, device, stream)


def hs_tree_attention_latent(q, q_rope, pool, c_tree, r_tree, parent, node_offsets, host_node_offsets, block_table, prefix_lens, host_prefix_lens,
                             scale: float, *, want_lse: bool = False, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                             ws: Optional[torch.Tensor] = None, stream=None):
    """Absorbed latent attention of tree rows: q [NN,Hq,R], q_rope [NN,Hq,Dr], c_tree [NN,R], r_tree [NN,Dr], `pool` [n_pages,64,R+Dr] (float32 or
    bfloat16, GPU; all but the pool may have strides of their own, heads included), the rest as in hs_tree_attention_paged.  Returns (o [NN,Hq,R], lse
    [NN,Hq] or None)."""
    if q.dim() != 3 or q_rope.dim() != 3 or pool.dim() != 3:
        raise ValueError("q must be [NN, Hq, R], q_rope [NN, Hq, Dr], the pool [n_pages, 64, R + Dr]")
    NN, Hq, R = q.shape
    Dr = q_rope.shape[2]
    B = host_node_offsets.numel() - 1
    if pool.shape[1] != HS_MX_PAGE or pool.shape[2] != R + Dr or tuple(q_rope.shape[:2]) != (NN, Hq) or tuple(c_tree.shape) != (NN, R) or \
            tuple(r_tree.shape) != (NN, Dr):
        raise ValueError("q_rope must be [NN, Hq, Dr], c_tree [NN, R], r_tree [NN, Dr], the pool [n_pages, %d, R + Dr]" % HS_MX_PAGE)
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table must be [B, max_blocks]")
    if parent.numel() != NN or node_offsets.numel() != B + 1 or prefix_lens.numel() != B or host_prefix_lens.numel() != B or \
            int(host_node_offsets[B]) != NN:
        raise ValueError("parent must hold NN values, the offsets B + 1 (the last one NN), the lengths B")
    if out is None:
        out = _empty((NN, Hq, R), q.dtype, q.device, stream)
    if want_lse and lse is None:
        lse = _empty((NN, Hq), torch.float32, q.device, stream)
    if out.shape != q.shape or (lse is not None and lse.numel() != NN * Hq):
        raise ValueError("out must be [NN, Hq, R], lse [NN, Hq]")
    if ws is None:
        ws = hs_tree_attention_latent_workspace(host_node_offsets, host_prefix_lens, Hq, R, Dr, q.device, stream=stream)
    _check(_calls.hs_tree_attention_latent(q, q_rope, pool, c_tree, r_tree, parent, node_offsets, host_node_offsets, block_table, block_table.shape[1],
                                           pool.shape[0], prefix_lens, host_prefix_lens, B, Hq, R, Dr, scale, out, lse, ws, stream),
           "hs_tree_attention_latent")
    return out, lse


def hs_prompt_attention_latent_workspace(host_q_offsets, host_kv_offsets, H: int, Dv: int, device, *, stream=None) -> Optional[torch.Tensor]:
    """A workspace for hs_prompt_attention_latent calls of these offsets (CPU tensors) on `stream`; None where none is needed."""
    if host_q_offsets.numel() != host_kv_offsets.numel():
        raise ValueError("both offsets must hold B + 1 values")
    qo, ko = host_q_offsets.to("cpu", torch.int32).contiguous(), host_kv_offsets.to("cpu", torch.int64).contiguous()
    n = lib().hs_prompt_attention_latent_workspace(qo.data_ptr(), ko.data_ptr(), qo.numel() - 1, int(H), int(Dv))
    return workspace(n, device, stream)


def hs_prompt_attention_latent(q, q_rope, k, k_rope, v, q_offsets, kv_offsets, host_q_offsets, host_kv_offsets, scale: float, *, want_lse: bool = False,
                               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Expanded latent attention of prompt rows, causal: q [N,H,Dn], q_rope [N,H,Dr], k [T,H,Dn], k_rope [T,Dr], v [T,H,Dv] (float32 or bfloat16, GPU;
    strides of their own, e.g. k and v slices of one product's result), q_offsets int32 [B+1] and kv_offsets int64 [B+1] on the GPU and the same on the
    CPU.  Returns (o [N,H,Dv], lse [N,H] or None)."""
    if q.dim() != 3 or q_rope.dim() != 3 or k.dim() != 3 or k_rope.dim() != 2 or v.dim() != 3:
        raise ValueError("q must be [N, H, Dn], q_rope [N, H, Dr], k [T, H, Dn], k_rope [T, Dr], v [T, H, Dv]")
    N, H, Dn = q.shape
    T, Dr, Dv = k.shape[0], q_rope.shape[2], v.shape[2]
    B = host_q_offsets.numel() - 1
    if tuple(q_rope.shape[:2]) != (N, H) or tuple(k.shape[1:]) != (H, Dn) or tuple(k_rope.shape) != (T, Dr) or tuple(v.shape[:2]) != (T, H):
        raise ValueError("q must be [N, H, Dn], q_rope [N, H, Dr], k [T, H, Dn], k_rope [T, Dr], v [T, H, Dv]")
    if q_offsets.numel() != B + 1 or kv_offsets.numel() != B + 1 or host_kv_offsets.numel() != B + 1 or int(host_q_offsets[B]) != N or \
            int(host_kv_offsets[B]) != T:
        raise ValueError("the offsets must hold B + 1 values, the last ones N and T")
    if out is None:
        out = _empty((N, H, Dv), q.dtype, q.device, stream)
    if want_lse and lse is None:
        lse = _empty((N, H), torch.float32, q.device, stream)
    if tuple(out.shape) != (N, H, Dv) or (lse is not None and lse.numel() != N * H):
        raise ValueError("out must be [N, H, Dv], lse [N, H]")
    if ws is None:
        ws = hs_prompt_attention_latent_workspace(host_q_offsets, host_kv_offsets, H, Dv, q.device, stream=stream)
    _check(_calls.hs_prompt_attention_latent(q, q_rope, k, k_rope, v, q_offsets, kv_offsets, host_q_offsets, host_kv_offsets, B, H, Dn, Dr, Dv, scale, out,
                                             lse, ws, stream), "hs_prompt_attention_latent")
    return out, lse


def hs_verify_accept(target_logits, draft_logits, token, parent, node_offsets, mode: int, temperature: float,
                     uniforms, max_depth: int, *, out: Optional[Dict[str, torch.Tensor]] = None,
                     ws: Optional[torch.Tensor] = None, stream=None) -> Dict[str, torch.Tensor]:
    """target_logits / draft_logits float32 [NN, V] (draft and uniforms may be None when greedy; rows may be
    padded: unit stride along the vocabulary, the same row stride in both), token and parent int32 [NN],
    node_offsets int32 [B+1], uniforms float32 [NN + B].  Returns accept_len [B], accept_path [B, max_depth],
    bonus_token [B]."""
    def rows(t, name):
        if not t.is_cuda or t.dtype != torch.float32 or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
            raise ValueError("%s must be a float32 [NN, V] GPU tensor with unit stride along V" % name)
        return t.stride(0) if t.shape[0] > 1 else t.shape[1]
    row_stride = rows(target_logits, "target_logits")
    NN, V = target_logits.shape
    B = node_offsets.numel() - 1
    if draft_logits is not None:
        if draft_logits.shape != target_logits.shape or rows(draft_logits, "draft_logits") != row_stride:
            raise ValueError("draft_logits must have the shape and row stride of target_logits")
    if uniforms is not None and uniforms.numel() != NN + B:
        raise ValueError("uniforms must hold NN + B values")
    if out is None:
        dev = target_logits.device
        out = dict(accept_len=_empty(B, torch.int32, dev, stream),
                   accept_path=_empty((B, max_depth), torch.int32, dev, stream),
                   bonus_token=_empty(B, torch.int32, dev, stream))
    if ws is None:
        ws = workspace(lib().hs_verify_accept_workspace_mode(B, NN, V, int(mode)), target_logits.device, stream)
    st = _calls.hs_verify_accept(target_logits, draft_logits, row_stride, token, parent, node_offsets, B, NN, V, int(mode),
                                 temperature, uniforms, int(max_depth), out["accept_len"], out["accept_path"],
                                 out["bonus_token"], ws, stream)
    _check(st, "hs_verify_accept")
    return out


def hs_time_next_attention(start_event, stop_event) -> None:
    """start_event, stop_event: torch.cuda.Event(enable_timing=True) that have been recorded at least once
    (torch creates the HIP event at the first record), or both None.  The next tree-attention call of this
    thread attaches them to its attention kernel; start_event.elapsed_time(stop_event) is then the
    kernel's own duration."""
    if start_event is None and stop_event is None:
        _check(lib().hs_time_next_attention(None, None), "hs_time_next_attention")
        return
    h0, h1 = start_event.cuda_event, stop_event.cuda_event
    if not h0 or not h1:
        raise ValueError("hs_time_next_attention: record each event once before handing it over")
    _check(lib().hs_time_next_attention(_c.c_void_p(h0), _c.c_void_p(h1)), "hs_time_next_attention")


def hs_tree_attention_plan(host_node_offsets, host_prefix_offsets, Hq, Hkv, D, dtype, *, host_prefix_lens=None,
                           paged=False, max_blocks=0):
    """Host only.  host_node_offsets int32 [B+1], host_prefix_offsets int64 [B+1] (None when paged),
    host_prefix_lens int64 [B] or None: CPU tensors.  Returns (totals int64 [6], per_seq int32 [B,4]) as the
    header describes them."""
    B = host_node_offsets.numel() - 1
    totals = torch.zeros(6, dtype=torch.int64)
    per_seq = torch.zeros(max(B, 1), 4, dtype=torch.int32)
    hp = None if host_prefix_offsets is None else host_prefix_offsets.data_ptr()
    hl = None if host_prefix_lens is None else host_prefix_lens.data_ptr()
    _check(lib().hs_tree_attention_plan(host_node_offsets.data_ptr(), hp, hl, 1 if paged else 0, int(max_blocks), B,
                                        int(Hq), int(Hkv), int(D), int(dtype), totals.data_ptr(), per_seq.data_ptr()),
           "hs_tree_attention_plan")
    return totals, per_seq[:B]


def hs_tree_attention_last_kernel() -> int:
    """1: this thread's last tree-attention call ran the bfloat16 matrix-core kernel, 2: the any-shape kernel, 0: it launched nothing."""
    return int(lib().hs_tree_attention_last_kernel())


def hs_tree_attention_last_form() -> int:
    """Workgroups to a work item (1, 2, 4) of this thread's last tree-attention call or plan query, plus 16 or 32 where row
    groups share blocks among waves, as the header describes it; 0: not the matrix-core kernel."""
    return int(lib().hs_tree_attention_last_form())


def hs_tree_validate(parent, token, node_offsets, *, stream=None) -> torch.Tensor:
    """parent int32 [NN], token int32 [NN] or None, node_offsets int32 [B+1] (GPU).  Returns the device
    report int32 [2]: number of offending rows, global index of the first (-1 if none)."""
    _dev(parent, torch.int32, "parent"); _dev(node_offsets, torch.int32, "node_offsets")
    if token is not None:
        _dev(token, torch.int32, "token")
    report = _empty(2, torch.int32, parent.device, stream)
    st = lib().hs_tree_validate(_ptr(parent), _ptr(token), _ptr(node_offsets), node_offsets.numel() - 1,
                                parent.numel(), _ptr(report), _stream(stream))
    _check(st, "hs_tree_validate")
    return report
