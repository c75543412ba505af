"""Thin ctypes layer over ``libgs.so``: same names as ``include/gs.h``.

Argument marshalling only.  Tensors are torch CUDA tensors used as plain
device buffers; each call passes ``data_ptr()`` values and the current torch
stream to the C entry point.  There is no CPU or torch fallback: if the shared
library is missing, or a tensor is not on the GPU, the call raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgs.so")

GS_OK, GS_EINVAL, GS_EWORKSPACE, GS_EOVERFLOW, GS_EHIP = 0, -1, -2, -3, -4
GS_SYMMETRIZE, GS_DROP_SELF_LOOPS, GS_DEDUPE = 1, 2, 4
GS_F32, GS_BF16, GS_F16 = 0, 1, 2

EXPORTS = (
    "gs_last_hip_error",
    "gs_csr_build_workspace_bytes", "gs_csr_build",
    "gs_alias_build_workspace_bytes", "gs_alias_build", "gs_alias_pack",
    "gs_random_walk", "gs_node2vec_walk",
    "gs_make_pairs_workspace_bytes", "gs_make_pairs",
    "gs_sample_negatives", "gs_sample_edges",
    "gs_sgns_step_workspace_bytes", "gs_sgns_step", "gs_sgns_step_static", "gs_sgns_momentum_step",
    "gs_sgns_adam_step",
    "gs_sgns_step_fused_workspace_bytes", "gs_sgns_step_fused",
    "gs_pair_offsets_workspace_bytes", "gs_pair_offsets",
    "gs_sgns_step_from_walks_workspace_bytes", "gs_sgns_step_from_walks",
    "gs_line1_step_workspace_bytes", "gs_line1_step",
    "gs_unique_ids_workspace_bytes", "gs_unique_ids", "gs_get_rows", "gs_put_rows",
    "gs_table_mult", "gs_table_mult_add", "gs_sort_pairs_workspace_bytes", "gs_sort_pairs",
    "gs_softmax_loss_workspace_bytes", "gs_softmax_loss", "gs_scores_workspace_bytes", "gs_scores",
    "gs_sample_scores_workspace_bytes", "gs_sample_scores",
    "gs_clip_grads_workspace_bytes", "gs_clip_grads",
    "gs_q8_pitch", "gs_q8_scale_pitch", "gs_quantize_rows", "gs_scores_q8_workspace_bytes", "gs_scores_q8",
    "gs_beam_select_workspace_bytes", "gs_beam_select", "gs_beam_reorder",
)


class GsError(RuntimeError):
    def __init__(self, what: str, status: int, hip: int = 0):
        names = {-1: "GS_EINVAL", -2: "GS_EWORKSPACE", -3: "GS_EOVERFLOW", -4: "GS_EHIP"}
        msg = f"{what}: {names.get(status, status)}"
        if status == GS_EHIP:
            msg += f" (hip error {hip})"
        super().__init__(msg)
        self.status = status


class CsrStruct(C.Structure):
    _fields_ = [("num_nodes", C.c_int64), ("num_entries", C.c_int64),
                ("offsets", C.c_void_p), ("offset_bits", C.c_int32),
                ("nbrs", C.c_void_p), ("weights", C.c_void_p)]


class AliasStruct(C.Structure):
    _fields_ = [("prob", C.c_void_p), ("alias", C.c_void_p), ("packed", C.c_void_p)]


class TensorStruct(C.Structure):
    _fields_ = [("data", C.c_void_p), ("out", C.c_void_p), ("count", C.c_int64), ("dtype", C.c_int32)]


class StateStruct(C.Structure):
    _fields_ = [("data", C.c_void_p), ("out", C.c_void_p), ("row_bytes", C.c_int64), ("append_at", C.c_int64)]


# Arguments of the calls that are made once for every token or walk: p pointer, q int64, i int32, f float, z size.
SIGNATURES = {
    "gs_quantize_rows": "pqiipqpppp", "gs_scores_q8_workspace_bytes": "qqi", "gs_scores_q8": "ppqppqipqpfpipzp",
    "gs_beam_select_workspace_bytes": "qiqii", "gs_beam_select": "pqiqippippppzp", "gs_beam_reorder": "piqiippp",
}
_TYPES = {"p": C.c_void_p, "q": C.c_int64, "i": C.c_int32, "f": C.c_float, "z": C.c_size_t}

_lib = None


def lib() -> C.CDLL:
    """Opens libgs.so (built by ``paper_2407_15452_amd.build``); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2407_15452_amd.build`; "
                "there is no fallback path")
        l = C.CDLL(LIB_PATH)
        for name in EXPORTS:
            fn = getattr(l, name)
            fn.restype = C.c_size_t if name.endswith("_workspace_bytes") else C.c_int32
            if name in SIGNATURES:
                fn.argtypes = [_TYPES[t] for t in SIGNATURES[name]]
        _lib = l
    return _lib


def _dev(t, dtype=None, name="tensor"):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(rc, what):
    if rc != GS_OK:
        raise GsError(what, rc, lib().gs_last_hip_error() if rc == GS_EHIP else 0)


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


class Csr:
    """Device CSR (tensors + the host descriptor handed to the library)."""

    def __init__(self, offsets: torch.Tensor, nbrs: torch.Tensor, weights=None, num_entries=None):
        assert offsets.dtype in (torch.int32, torch.int64)
        self.offsets, self.nbrs, self.weights = offsets, nbrs, weights
        self.num_nodes = offsets.numel() - 1
        self.num_entries = int(nbrs.numel() if num_entries is None else num_entries)
        self.offset_bits = 64 if offsets.dtype == torch.int64 else 32
        self.struct = CsrStruct(self.num_nodes, self.num_entries, offsets.data_ptr(),
                                self.offset_bits, nbrs.data_ptr() if nbrs.numel() else None,
                                weights.data_ptr() if weights is not None else None)


class Alias:
    def __init__(self, prob: torch.Tensor, alias: torch.Tensor, packed=None):
        _dev(prob, torch.float32, "prob")
        _dev(alias, torch.int32, "alias")
        _dev(packed, torch.int64, "packed")
        self.prob, self.alias, self.packed = prob, alias, packed
        self.struct = AliasStruct(prob.data_ptr(), alias.data_ptr(),
                                  None if packed is None else packed.data_ptr())


def gs_csr_build(src, dst, w, num_nodes: int, flags: int, offset_bits: int = 32, ws=None) -> Csr:
    l = lib()
    m = int(src.numel())
    dev = src.device
    cap = max(1, m * (2 if flags & GS_SYMMETRIZE else 1))
    offsets = torch.empty(num_nodes + 1, dtype=torch.int64 if offset_bits == 64 else torch.int32,
                          device=dev)
    nbrs = torch.empty(cap, dtype=torch.int32, device=dev)
    w_out = torch.empty(cap, dtype=torch.float32, device=dev) if w is not None else None
    n_out = torch.zeros(1, dtype=torch.int64, device=dev)
    need = l.gs_csr_build_workspace_bytes(C.c_int64(m), C.c_int64(num_nodes), C.c_uint32(flags))
    if ws is None:
        ws = _workspace(need, dev)
    rc = l.gs_csr_build(_dev(src, torch.int32, "src"), _dev(dst, torch.int32, "dst"),
                        _dev(w, torch.float32, "w"), C.c_int64(m), C.c_int64(num_nodes),
                        C.c_uint32(flags), C.c_int32(offset_bits), _dev(offsets), _dev(nbrs),
                        _dev(w_out), _dev(n_out), _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_csr_build")
    n = int(n_out.item())
    return Csr(offsets, nbrs[:n], None if w_out is None else w_out[:n], n)


def gs_alias_pack(prob, alias) -> torch.Tensor:
    """The table as one 8-byte word per entry (see gs.h)."""
    total = int(prob.numel())
    packed = torch.empty(max(1, total), dtype=torch.int64, device=prob.device)
    rc = lib().gs_alias_pack(_dev(prob, torch.float32, "prob"), _dev(alias, torch.int32, "alias"),
                             C.c_int64(total), _dev(packed), _stream())
    _check(rc, "gs_alias_pack")
    return packed[:total]


def gs_alias_build(seg_offsets, weights, ws=None, pack: bool = True) -> Alias:
    l = lib()
    dev = weights.device
    total = int(weights.numel())
    nseg = int(seg_offsets.numel()) - 1
    bits = 64 if seg_offsets.dtype == torch.int64 else 32
    prob = torch.empty(max(1, total), dtype=torch.float32, device=dev)
    alias = torch.empty(max(1, total), dtype=torch.int32, device=dev)
    need = l.gs_alias_build_workspace_bytes(C.c_int64(nseg), C.c_int64(total))
    if ws is None:
        ws = _workspace(need, dev)
    rc = l.gs_alias_build(_dev(seg_offsets, None, "seg_offsets"), C.c_int32(bits), C.c_int64(nseg),
                          C.c_int64(total), _dev(weights, torch.float32, "weights"), _dev(prob),
                          _dev(alias), _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_alias_build")
    prob, alias = prob[:total], alias[:total]
    return Alias(prob, alias, gs_alias_pack(prob, alias) if pack and total > 0 else None)


def _alias_ref(a):
    return None if a is None else C.byref(a.struct)


def gs_random_walk(g: Csr, a, starts, walk_len: int, seed: int, walk_id_base: int = 0, out=None):
    nw = int(starts.numel())
    if out is None:
        out = torch.empty((nw, walk_len), dtype=torch.int32, device=starts.device)
    rc = lib().gs_random_walk(C.byref(g.struct), _alias_ref(a), _dev(starts, torch.int32, "starts"),
                              C.c_int64(nw), C.c_uint64(walk_id_base), C.c_int32(walk_len),
                              C.c_uint64(seed), _dev(out, torch.int32, "walks_out"), _stream())
    _check(rc, "gs_random_walk")
    return out


def gs_node2vec_walk(g: Csr, a, starts, walk_len: int, p: float, q: float, seed: int,
                     walk_id_base: int = 0, out=None):
    nw = int(starts.numel())
    if out is None:
        out = torch.empty((nw, walk_len), dtype=torch.int32, device=starts.device)
    rc = lib().gs_node2vec_walk(C.byref(g.struct), _alias_ref(a),
                                _dev(starts, torch.int32, "starts"), C.c_int64(nw),
                                C.c_uint64(walk_id_base), C.c_int32(walk_len), C.c_float(p),
                                C.c_float(q), C.c_uint64(seed), _dev(out, torch.int32, "walks_out"),
                                _stream())
    _check(rc, "gs_node2vec_walk")
    return out


def pair_capacity(num_walks: int, walk_len: int, window: int) -> int:
    """Capacity gs_make_pairs requires of its output arrays (see gs.h)."""
    if walk_len > window:
        return num_walks * (2 * window * walk_len - window * (window + 1))
    return num_walks * walk_len * (walk_len - 1)


def gs_make_pairs(walks, window: int, centers=None, contexts=None, num_pairs_out=None, ws=None,
                  sync: bool = True):
    """Returns (centers, contexts, num_pairs).  With sync=False num_pairs is the
    device scalar and the outputs are left at full capacity."""
    l = lib()
    nw, walk_len = int(walks.shape[0]), int(walks.shape[1])
    dev = walks.device
    cap = max(1, pair_capacity(nw, walk_len, window))
    if centers is None:
        centers = torch.empty(cap, dtype=torch.int32, device=dev)
    if contexts is None:
        contexts = torch.empty(cap, dtype=torch.int32, device=dev)
    if num_pairs_out is None:
        num_pairs_out = torch.zeros(1, dtype=torch.int64, device=dev)
    if ws is None:
        ws = _workspace(l.gs_make_pairs_workspace_bytes(C.c_int64(nw)), dev)
    rc = l.gs_make_pairs(_dev(walks, torch.int32, "walks"), C.c_int64(nw), C.c_int32(walk_len),
                         C.c_int32(window), _dev(centers, torch.int32), _dev(contexts, torch.int32),
                         _dev(num_pairs_out, torch.int64), _dev(ws), C.c_size_t(ws.numel()),
                         _stream())
    _check(rc, "gs_make_pairs")
    if not sync:
        return centers, contexts, num_pairs_out
    n = int(num_pairs_out.item())
    return centers[:n], contexts[:n], n


def gs_sample_negatives(noise, num_nodes: int, num_pairs: int, k: int, seed: int,
                        pair_index_base: int = 0, out=None, device=None):
    if out is None:
        dev = noise.prob.device if noise is not None else device
        out = torch.empty((num_pairs, k), dtype=torch.int32, device=dev)
    rc = lib().gs_sample_negatives(_alias_ref(noise), C.c_int64(num_nodes), C.c_int64(num_pairs),
                                   C.c_uint64(pair_index_base), C.c_int32(k), C.c_uint64(seed),
                                   _dev(out, torch.int32, "negs_out"), _stream())
    _check(rc, "gs_sample_negatives")
    return out


def gs_sample_edges(g: Csr, edge_alias, num_samples: int, seed: int, sample_index_base: int = 0,
                    centers_out=None, contexts_out=None):
    """LINE positive pairs: returns (centers, contexts), one CSR entry per sample."""
    dev = g.nbrs.device
    if centers_out is None:
        centers_out = torch.empty(max(num_samples, 0), dtype=torch.int32, device=dev)
    if contexts_out is None:
        contexts_out = torch.empty(max(num_samples, 0), dtype=torch.int32, device=dev)
    rc = lib().gs_sample_edges(C.byref(g.struct), _alias_ref(edge_alias), C.c_int64(num_samples),
                               C.c_uint64(sample_index_base), C.c_uint64(seed),
                               _dev(centers_out, torch.int32, "centers_out"),
                               _dev(contexts_out, torch.int32, "contexts_out"), _stream())
    _check(rc, "gs_sample_edges")
    return centers_out, contexts_out


def gs_sgns_step_workspace_bytes(num_pairs: int, num_nodes: int, k: int, dim: int,
                                 dtype: int = GS_F32) -> int:
    return int(lib().gs_sgns_step_workspace_bytes(C.c_int64(num_pairs), C.c_int64(num_nodes),
                                                  C.c_int32(k), C.c_int32(dim), C.c_int32(dtype)))


def gs_sgns_step(w_in, w_out, centers, contexts, negs, lr: float, loss_out=None, ws=None):
    """Updates w_in / w_out in place; returns the device scalar holding the summed loss."""
    dtype = _table_dtype(w_in)
    num_nodes, dim = int(w_in.shape[0]), int(w_in.shape[1])
    num_pairs = int(centers.numel())
    k = int(negs.shape[1]) if negs.dim() == 2 else 0
    dev = w_in.device
    if loss_out is None:
        loss_out = torch.zeros(1, dtype=torch.float64, device=dev)
    if ws is None:
        ws = _workspace(gs_sgns_step_workspace_bytes(num_pairs, num_nodes, k, dim, dtype), dev)
    rc = lib().gs_sgns_step(_dev(w_in, None, "w_in"), _dev(w_out, w_in.dtype, "w_out"),
                            C.c_int64(num_nodes), C.c_int32(dim), C.c_int32(dtype),
                            _dev(centers, torch.int32, "centers"),
                            _dev(contexts, torch.int32, "contexts"),
                            _dev(negs, torch.int32, "negs") if negs.numel() else None,
                            C.c_int64(num_pairs), C.c_int32(k), C.c_float(lr),
                            _dev(loss_out, torch.float64, "loss_sum_out"), _dev(ws),
                            C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_sgns_step")
    return loss_out


def gs_sgns_step_static(w_in, w_out, centers, contexts, negs, lr: float, loss_out=None):
    """gs_sgns_step on the library's own static scratch array (small batches; see gs.h)."""
    dtype = _table_dtype(w_in)
    num_nodes, dim = int(w_in.shape[0]), int(w_in.shape[1])
    num_pairs = int(centers.numel())
    k = int(negs.shape[1]) if negs.dim() == 2 else 0
    if loss_out is None:
        loss_out = torch.zeros(1, dtype=torch.float64, device=w_in.device)
    rc = lib().gs_sgns_step_static(_dev(w_in, None, "w_in"), _dev(w_out, w_in.dtype, "w_out"),
                                   C.c_int64(num_nodes), C.c_int32(dim), C.c_int32(dtype),
                                   _dev(centers, torch.int32, "centers"),
                                   _dev(contexts, torch.int32, "contexts"),
                                   _dev(negs, torch.int32, "negs") if negs.numel() else None,
                                   C.c_int64(num_pairs), C.c_int32(k), C.c_float(lr),
                                   _dev(loss_out, torch.float64, "loss_sum_out"), _stream())
    _check(rc, "gs_sgns_step_static")
    return loss_out


def gs_sgns_momentum_step(w_in, w_out, m_in, m_out, centers, contexts, negs, lr: float, mu: float,
                          loss_out=None, ws=None):
    """SGD-with-momentum iteration (see gs.h); the four tables are updated in place."""
    dtype = _table_dtype(w_in)
    num_nodes, dim = int(w_in.shape[0]), int(w_in.shape[1])
    num_pairs = int(centers.numel())
    k = int(negs.shape[1]) if negs.dim() == 2 else 0
    dev = w_in.device
    if loss_out is None:
        loss_out = torch.zeros(1, dtype=torch.float64, device=dev)
    if ws is None:
        ws = _workspace(gs_sgns_step_workspace_bytes(num_pairs, num_nodes, k, dim, dtype), dev)
    rc = lib().gs_sgns_momentum_step(
        _dev(w_in, None, "w_in"), _dev(w_out, w_in.dtype, "w_out"), _dev(m_in, w_in.dtype, "m_in"),
        _dev(m_out, w_in.dtype, "m_out"), C.c_int64(num_nodes), C.c_int32(dim), C.c_int32(dtype),
        _dev(centers, torch.int32, "centers"), _dev(contexts, torch.int32, "contexts"),
        _dev(negs, torch.int32, "negs") if negs.numel() else None, C.c_int64(num_pairs),
        C.c_int32(k), C.c_float(lr), C.c_float(mu), _dev(loss_out, torch.float64, "loss_sum_out"),
        _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_sgns_momentum_step")
    return loss_out


def gs_unique_ids_workspace_bytes(n: int, num_nodes: int) -> int:
    return int(lib().gs_unique_ids_workspace_bytes(C.c_int64(n), C.c_int64(num_nodes)))


def gs_unique_ids(ids, num_nodes: int, want_inverse: bool = True, ws=None):
    """Returns (unique_out [n], num_unique device int64[1], inverse [n] or None); only the
    first num_unique entries of unique_out are meaningful."""
    n = int(ids.numel())
    dev = ids.device
    unique_out = torch.empty(max(n, 1), dtype=torch.int32, device=dev)
    count = torch.zeros(1, dtype=torch.int64, device=dev)
    inverse = torch.empty(max(n, 1), dtype=torch.int32, device=dev) if want_inverse else None
    if ws is None:
        ws = _workspace(gs_unique_ids_workspace_bytes(n, num_nodes), dev)
    rc = lib().gs_unique_ids(_dev(ids, torch.int32, "ids"), C.c_int64(n), C.c_int64(num_nodes),
                             _dev(unique_out, torch.int32), _dev(count, torch.int64),
                             _dev(inverse, torch.int32) if inverse is not None else None,
                             _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_unique_ids")
    return unique_out[:n], count, (inverse[:n] if inverse is not None else None)


def _table_dtype(table):
    if table.dtype == torch.float32:
        return GS_F32
    if table.dtype == torch.bfloat16:
        return GS_BF16
    if table.dtype == torch.float16:
        return GS_F16
    raise TypeError(f"tables are float32, bfloat16 or float16, not {table.dtype}")


def gs_get_rows(table, ids, count=None, out=None):
    """out[i] = table[ids[i]] as float32; `count` (device int64[1]) limits the rows processed."""
    n, dim = int(ids.numel()), int(table.shape[1])
    if out is None:
        out = torch.empty((n, dim), dtype=torch.float32, device=table.device)
    rc = lib().gs_get_rows(_dev(table), C.c_int64(table.shape[0]), C.c_int32(dim),
                           C.c_int32(_table_dtype(table)), _dev(ids, torch.int32, "ids"), C.c_int64(n),
                           _dev(count, torch.int64) if count is not None else None,
                           _dev(out, torch.float32, "out"), _stream())
    _check(rc, "gs_get_rows")
    return out


def gs_put_rows(table, ids, rows, scale: float, count=None):
    """table[ids[i]] += scale * rows[i] in place; the ids must be distinct."""
    n, dim = int(ids.numel()), int(table.shape[1])
    rc = lib().gs_put_rows(_dev(table), C.c_int64(table.shape[0]), C.c_int32(dim),
                           C.c_int32(_table_dtype(table)), _dev(ids, torch.int32, "ids"), C.c_int64(n),
                           _dev(count, torch.int64) if count is not None else None,
                           _dev(rows, torch.float32, "rows"), C.c_float(scale), _stream())
    _check(rc, "gs_put_rows")


def gs_sgns_adam_step(w_in, w_out, m_in, m_out, v_in, v_out, centers, contexts, negs, lr: float,
                      beta1: float, beta2: float, eps: float, t: int, loss_out=None, ws=None):
    """Adam iteration number t on six float32 tables, in place; returns the device loss scalar."""
    num_nodes, dim = int(w_in.shape[0]), int(w_in.shape[1])
    num_pairs = int(centers.numel())
    k = int(negs.shape[1]) if negs.dim() == 2 else 0
    dev = w_in.device
    for tb in (w_in, w_out, m_in, m_out, v_in, v_out):
        if tb.dtype != torch.float32 or tuple(tb.shape) != (num_nodes, dim) or not tb.is_contiguous():
            raise TypeError("Adam tables must be contiguous float32 [num_nodes, dim]")
    if loss_out is None:
        loss_out = torch.zeros(1, dtype=torch.float64, device=dev)
    if ws is None:
        ws = _workspace(gs_sgns_step_workspace_bytes(num_pairs, num_nodes, k, dim, GS_F32), dev)
    rc = lib().gs_sgns_adam_step(
        _dev(w_in), _dev(w_out), _dev(m_in), _dev(m_out), _dev(v_in), _dev(v_out),
        C.c_int64(num_nodes), C.c_int32(dim), _dev(centers, torch.int32, "centers"),
        _dev(contexts, torch.int32, "contexts"), _dev(negs, torch.int32, "negs"),
        C.c_int64(num_pairs), C.c_int32(k), C.c_float(lr), C.c_float(beta1), C.c_float(beta2),
        C.c_float(eps), C.c_int64(t), _dev(loss_out, torch.float64), _dev(ws),
        C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_sgns_adam_step")
    return loss_out


def gs_sgns_step_fused_workspace_bytes(num_pairs: int, num_nodes: int, k: int, dim: int,
                                       dtype: int = GS_F32) -> int:
    return int(lib().gs_sgns_step_fused_workspace_bytes(C.c_int64(num_pairs), C.c_int64(num_nodes),
                                                        C.c_int32(k), C.c_int32(dim), C.c_int32(dtype)))


def gs_sgns_step_fused(w_in, w_out, centers, contexts, noise, k: int, neg_seed: int, lr: float,
                       pair_index_base: int = 0, loss_out=None, ws=None):
    """gs_sample_negatives + gs_sgns_step in one call; returns the device loss scalar."""
    dtype = _table_dtype(w_in)
    num_nodes, dim = int(w_in.shape[0]), int(w_in.shape[1])
    num_pairs = int(centers.numel())
    dev = w_in.device
    if loss_out is None:
        loss_out = torch.zeros(1, dtype=torch.float64, device=dev)
    if ws is None:
        ws = _workspace(gs_sgns_step_fused_workspace_bytes(num_pairs, num_nodes, k, dim, dtype), dev)
    rc = lib().gs_sgns_step_fused(
        _dev(w_in), _dev(w_out), C.c_int64(num_nodes), C.c_int32(dim), C.c_int32(dtype),
        _dev(centers, torch.int32, "centers"), _dev(contexts, torch.int32, "contexts"),
        C.c_int64(num_pairs), _alias_ref(noise), C.c_uint64(pair_index_base), C.c_uint64(neg_seed),
        C.c_int32(k), C.c_float(lr), _dev(loss_out, torch.float64), _dev(ws), C.c_size_t(ws.numel()),
        _stream())
    _check(rc, "gs_sgns_step_fused")
    return loss_out


def gs_pair_offsets(walks, window: int, out=None, ws=None):
    """int64[num_walks + 1]: pairs emitted for the walks before each walk, and for all of them."""
    num_walks, walk_len = int(walks.shape[0]), int(walks.shape[1])
    dev = walks.device
    if out is None:
        out = torch.empty(num_walks + 1, dtype=torch.int64, device=dev)
    if ws is None:
        ws = _workspace(int(lib().gs_pair_offsets_workspace_bytes(C.c_int64(num_walks))), dev)
    rc = lib().gs_pair_offsets(_dev(walks, torch.int32, "walks"), C.c_int64(num_walks), C.c_int32(walk_len),
                               C.c_int32(window), _dev(out, torch.int64, "offsets_out"), _dev(ws),
                               C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_pair_offsets")
    return out


def gs_sgns_step_from_walks_workspace_bytes(num_pairs: int, num_nodes: int, k: int, dim: int,
                                            dtype: int = GS_F32) -> int:
    return int(lib().gs_sgns_step_from_walks_workspace_bytes(
        C.c_int64(num_pairs), C.c_int64(num_nodes), C.c_int32(k), C.c_int32(dim), C.c_int32(dtype)))


def gs_sgns_step_from_walks(w_in, w_out, walks, window: int, pair_offsets, first_pair: int,
                            num_pairs: int, noise, k: int, neg_seed: int, lr: float,
                            pair_index_base: int = 0, loss_out=None, ws=None):
    """Pairs from the walk buffer, negatives from the counters, and the iteration, in one call."""
    dtype = _table_dtype(w_in)
    num_nodes, dim = int(w_in.shape[0]), int(w_in.shape[1])
    num_walks, walk_len = int(walks.shape[0]), int(walks.shape[1])
    dev = w_in.device
    if loss_out is None:
        loss_out = torch.zeros(1, dtype=torch.float64, device=dev)
    if ws is None:
        ws = _workspace(gs_sgns_step_from_walks_workspace_bytes(num_pairs, num_nodes, k, dim, dtype), dev)
    rc = lib().gs_sgns_step_from_walks(
        _dev(w_in), _dev(w_out), C.c_int64(num_nodes), C.c_int32(dim), C.c_int32(dtype),
        _dev(walks, torch.int32, "walks"), C.c_int64(num_walks), C.c_int32(walk_len), C.c_int32(window),
        _dev(pair_offsets, torch.int64, "pair_offsets"), C.c_int64(first_pair), C.c_int64(num_pairs),
        _alias_ref(noise), C.c_uint64(pair_index_base), C.c_uint64(neg_seed), C.c_int32(k),
        C.c_float(lr), _dev(loss_out, torch.float64), _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_sgns_step_from_walks")
    return loss_out


def gs_line1_step_workspace_bytes(num_pairs: int, num_nodes: int, k: int, dim: int,
                                  dtype: int = GS_F32) -> int:
    return int(lib().gs_line1_step_workspace_bytes(C.c_int64(num_pairs), C.c_int64(num_nodes),
                                                   C.c_int32(k), C.c_int32(dim), C.c_int32(dtype)))


def gs_line1_step(w, sources, targets, negs, lr: float, loss_out=None, ws=None):
    """First-order LINE iteration on the single table w, in place; returns the device loss scalar."""
    dtype = _table_dtype(w)
    num_nodes, dim = int(w.shape[0]), int(w.shape[1])
    num_pairs = int(sources.numel())
    k = int(negs.shape[1]) if negs.dim() == 2 else 0
    dev = w.device
    if loss_out is None:
        loss_out = torch.zeros(1, dtype=torch.float64, device=dev)
    if ws is None:
        ws = _workspace(gs_line1_step_workspace_bytes(num_pairs, num_nodes, k, dim, dtype), dev)
    rc = lib().gs_line1_step(
        _dev(w), C.c_int64(num_nodes), C.c_int32(dim), C.c_int32(dtype),
        _dev(sources, torch.int32, "sources"), _dev(targets, torch.int32, "targets"),
        _dev(negs, torch.int32, "negs"), C.c_int64(num_pairs), C.c_int32(k), C.c_float(lr),
        _dev(loss_out, torch.float64), _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_line1_step")
    return loss_out


def gs_table_mult(table, factor: float):
    """table *= factor in place, every row."""
    rc = lib().gs_table_mult(_dev(table), C.c_int64(table.shape[0]), C.c_int32(table.shape[1]),
                             C.c_int32(_table_dtype(table)), C.c_float(factor), _stream())
    _check(rc, "gs_table_mult")


def gs_table_mult_add(dst, src, factor: float):
    """dst += factor * src in place, every row (two tables of the same shape and dtype)."""
    if dst.shape != src.shape or dst.dtype != src.dtype:
        raise TypeError("gs_table_mult_add needs two tables of the same shape and dtype")
    rc = lib().gs_table_mult_add(_dev(dst), _dev(src), C.c_int64(dst.shape[0]),
                                 C.c_int32(dst.shape[1]), C.c_int32(_table_dtype(dst)),
                                 C.c_float(factor), _stream())
    _check(rc, "gs_table_mult_add")


def gs_sort_pairs_workspace_bytes(n: int) -> int:
    return int(lib().gs_sort_pairs_workspace_bytes(C.c_int64(n)))


def gs_sort_pairs(centers, contexts, num_nodes: int, centers_out=None, contexts_out=None, ws=None):
    """Pairs reordered by centre id (stable); returns (centers_out, contexts_out)."""
    n = int(centers.numel())
    dev = centers.device
    if centers_out is None:
        centers_out = torch.empty(max(n, 1), dtype=torch.int32, device=dev)[:n]
    if contexts_out is None:
        contexts_out = torch.empty(max(n, 1), dtype=torch.int32, device=dev)[:n]
    if ws is None:
        ws = _workspace(gs_sort_pairs_workspace_bytes(n), dev)
    rc = lib().gs_sort_pairs(_dev(centers, torch.int32, "centers"), _dev(contexts, torch.int32, "contexts"),
                             C.c_int64(n), C.c_int64(num_nodes), _dev(centers_out, torch.int32),
                             _dev(contexts_out, torch.int32), _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_sort_pairs")
    return centers_out, contexts_out


def gs_softmax_loss_workspace_bytes(num_pairs: int, num_nodes: int, dim: int, dtype: int = GS_F32,
                                    want_grad: bool = True) -> int:
    return int(lib().gs_softmax_loss_workspace_bytes(C.c_int64(num_pairs), C.c_int64(num_nodes), C.c_int32(dim),
                                                     C.c_int32(dtype), C.c_int32(bool(want_grad))))


def _two_tables(w_in, w_out, bias):
    if w_in.dim() != 2 or w_out.dim() != 2 or w_in.shape[1] != w_out.shape[1] or w_in.dtype != w_out.dtype:
        raise TypeError("w_in and w_out must be [rows, dim] with the same dim and dtype")
    if bias is not None and tuple(bias.shape) != (w_out.shape[0],):
        raise ValueError("bias must have one value per row of w_out")
    return _table_dtype(w_in)


def _out(t, shape, dtype, device, name):
    """A new output, or the caller's, checked."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"{name} must have shape {tuple(shape)} and dtype {dtype}")
    return t


def gs_softmax_loss(w_in, w_out, centers, contexts, bias=None, scale: float = 1.0, grad_scale: float = 1.0,
                    want_grad=True, loss_out=None, g_in=None, g_out=None, ws=None):
    """Softmax loss of every pair over all nodes; returns (loss [n] float32, g_in [n, dim], g_out [nodes, dim]).
    want_grad: True for both gradients, "in" or "out" for one alone, False for none; the others are None (see gs.h)."""
    if isinstance(want_grad, str) and want_grad not in ("in", "out"):
        raise ValueError('want_grad must be True, False, "in" or "out"')
    dtype = _two_tables(w_in, w_out, bias)
    (num_in, dim), num_nodes, n = w_in.shape, int(w_out.shape[0]), int(centers.numel())
    if int(contexts.numel()) != n:
        raise ValueError("centers and contexts must have the same length")
    dev = w_in.device
    loss_out = _out(loss_out, (n,), torch.float32, dev, "loss_out")
    g_in = _out(g_in, (n, dim), w_in.dtype, dev, "g_in") if want_grad and want_grad != "out" else None
    g_out = _out(g_out, (num_nodes, dim), w_out.dtype, dev, "g_out") if want_grad and want_grad != "in" else None
    if ws is None:
        ws = _workspace(gs_softmax_loss_workspace_bytes(n, num_nodes, dim, dtype, want_grad), dev)
    rc = lib().gs_softmax_loss(
        _dev(w_in, None, "w_in"), C.c_int64(num_in), _dev(w_out, None, "w_out"), C.c_int64(num_nodes), C.c_int32(dim),
        C.c_int32(dtype), _dev(centers, torch.int32, "centers"), _dev(contexts, torch.int32, "contexts"), C.c_int64(n),
        _dev(bias, torch.float32, "bias"), C.c_float(scale), _dev(loss_out, None, "loss_out"), _dev(g_in, None, "g_in"),
        _dev(g_out, None, "g_out"), C.c_float(grad_scale), _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_softmax_loss")
    return loss_out, g_in, g_out


def gs_scores_workspace_bytes(num_centers: int, num_nodes: int, dim: int, dtype: int = GS_F32) -> int:
    return int(lib().gs_scores_workspace_bytes(C.c_int64(num_centers), C.c_int64(num_nodes), C.c_int32(dim), C.c_int32(dtype)))


def gs_scores(w_in, w_out, centers, bias=None, scale: float = 1.0, out=None, ws=None):
    """float32 [n, nodes]: scale * <w_in[centers[i]], w_out[j]> + bias[j]."""
    dtype = _two_tables(w_in, w_out, bias)
    (num_in, dim), num_nodes, n = w_in.shape, int(w_out.shape[0]), int(centers.numel())
    dev = w_in.device
    out = _out(out, (n, num_nodes), torch.float32, dev, "out")
    if ws is None:
        ws = _workspace(gs_scores_workspace_bytes(n, num_nodes, dim, dtype), dev)
    rc = lib().gs_scores(
        _dev(w_in, None, "w_in"), C.c_int64(num_in), _dev(w_out, None, "w_out"), C.c_int64(num_nodes), C.c_int32(dim),
        C.c_int32(dtype), _dev(centers, torch.int32, "centers"), C.c_int64(n), _dev(bias, torch.float32, "bias"),
        C.c_float(scale), _dev(out, None, "out"), _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_scores")
    return out


def gs_sample_scores_workspace_bytes(rows: int, n: int, dtype: int = GS_F32) -> int:
    return int(lib().gs_sample_scores_workspace_bytes(C.c_int64(rows), C.c_int64(n), C.c_int32(dtype)))


def gs_sample_scores(scores, uniforms, temperature=None, top_k=None, top_p=None, min_p=None, ids_out=None,
                     probs_out=None, ws=None):
    """One node per row of scores [rows, n]; returns (ids int32 [rows], probs float32 [rows]).  The filters are
    tensors with one value per row, or None (see gs.h)."""
    if scores.dim() != 2:
        raise ValueError("scores must be [rows, n]")
    dtype = _table_dtype(scores)
    rows, n = int(scores.shape[0]), int(scores.shape[1])
    dev = scores.device
    for name, t in (("uniforms", uniforms), ("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p)):
        if t is not None and tuple(t.shape) != (rows,):
            raise ValueError(f"{name} must have one value per row of scores")
    ids_out = _out(ids_out, (rows,), torch.int32, dev, "ids_out")
    probs_out = _out(probs_out, (rows,), torch.float32, dev, "probs_out")
    if ws is None:
        ws = _workspace(gs_sample_scores_workspace_bytes(rows, n, dtype), dev)
    rc = lib().gs_sample_scores(
        _dev(scores, None, "scores"), C.c_int64(rows), C.c_int64(n), C.c_int32(dtype),
        _dev(uniforms, torch.float32, "uniforms"), _dev(temperature, torch.float32, "temperature"),
        _dev(top_k, torch.int32, "top_k"), _dev(top_p, torch.float32, "top_p"), _dev(min_p, torch.float32, "min_p"),
        _dev(ids_out), _dev(probs_out), _dev(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_sample_scores")
    return ids_out, probs_out


class GradList:
    """Gradients (and, where given, the tensors that receive them clipped) as the host array gs_clip_grads takes;
    built once for tensors that stay where they are."""

    def __init__(self, grads, outs=None):
        self.grads, self.outs = list(grads), None if outs is None else list(outs)
        if self.outs is not None and len(self.outs) != len(self.grads):
            raise ValueError("one output per gradient")
        if not self.grads:
            raise ValueError("no gradients")
        self.device = self.grads[0].device
        self.array = (TensorStruct * len(self.grads))()
        for i, g in enumerate(self.grads):
            _dev(g, None, "gradient")
            o = None if self.outs is None else self.outs[i]
            if o is not None and (o.dtype != g.dtype or o.numel() != g.numel()):
                raise TypeError("an output must have its gradient's size and dtype")
            if g.device != self.device or (o is not None and o.device != self.device):
                raise ValueError("gradients and outputs must be on one device")
            self.array[i] = TensorStruct(g.data_ptr(), None if o is None else _dev(o, None, "output").value, g.numel(), _table_dtype(g))


def gs_clip_grads_workspace_bytes(num_tensors: int) -> int:
    return int(lib().gs_clip_grads_workspace_bytes(C.c_int32(num_tensors)))


def gs_clip_grads(grads, max_norm: float, norm_out=None, ws=None):
    """Clips a GradList (or a list of tensors, in place) to the norm max_norm; returns the norm before, float64 [1]."""
    if not isinstance(grads, GradList):
        grads = GradList(grads)
    n = len(grads.grads)
    norm_out = _out(norm_out, (1,), torch.float64, grads.device, "norm_out")
    if ws is None:
        ws = _workspace(gs_clip_grads_workspace_bytes(n), grads.device)
    rc = lib().gs_clip_grads(grads.array, C.c_int32(n), C.c_double(max_norm), _dev(norm_out), _dev(ws),
                             C.c_size_t(ws.numel()), _stream())
    _check(rc, "gs_clip_grads")
    return norm_out


GS_Q8_MAX_DIM = 8192
MOST_BEAMS = 256                 # and the most places of a selection; checked here, since what is passed on has 32 bits


def _one_device(dev, **tensors):
    """All of a call's tensors on its device, which is the current one: streams and workspaces are of that."""
    for name, t in tensors.items():
        if isinstance(t, torch.Tensor) and t.device != dev:
            raise ValueError(f"{name} must be on {dev}, not on {t.device}")
    if dev.type == "cuda" and dev.index != torch.cuda.current_device():
        raise ValueError(f"{dev} must be the current device")


def _at(t, dtype, name):
    """The address of a tensor, or None; its type is checked where one is given."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream_of(dev):
    return torch._C._cuda_getCurrentRawStream(dev.index)     # torch.cuda.current_stream takes as long as a launch


class Table8:
    """Rows of 8-bit values for answers: data float8_e4m3fn [rows, pitch], scales float8_e8m0fnu [rows, scale pitch], a scale for
    each block of 128 of the `dim` columns (see gs.h).  ``Table8.empty`` makes room for one."""

    def __init__(self, data: torch.Tensor, scales: torch.Tensor, dim: int):
        _at(data, torch.float8_e4m3fn, "data")
        _at(scales, torch.float8_e8m0fnu, "scales")
        pitch, scale_pitch = self.pitches(dim)
        if data.dim() != 2 or data.shape[1] != pitch or tuple(scales.shape) != (data.shape[0], scale_pitch):
            raise ValueError(f"rows of {dim} columns are data [rows, {pitch}] and scales [rows, {scale_pitch}]")
        if data.device != scales.device:
            raise ValueError("data and scales must be on one device")
        self.data, self.scales, self.dim, self.num_nodes, self.device = data, scales, int(dim), int(data.shape[0]), data.device

    @staticmethod
    def pitches(dim: int):
        if not 1 <= dim <= GS_Q8_MAX_DIM:
            raise ValueError(f"dim must be from 1 to {GS_Q8_MAX_DIM}")
        blocks = -(-dim // 128)
        return -(-dim // 16) * 16, blocks if blocks <= 2 else -(-blocks // 4) * 4

    @classmethod
    def empty(cls, num_nodes: int, dim: int, device):
        pitch, scale_pitch = cls.pitches(dim)
        return cls(torch.empty(num_nodes, pitch, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn),
                   torch.empty(num_nodes, scale_pitch, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu), dim)


def gs_quantize_rows(table, ids=None, count=None, out=None) -> Table8:
    """table [nodes, dim] as a Table8: all of it, or (with ids int32 [n], and out) the rows ids, the others as they are."""
    if table.dim() != 2:
        raise ValueError("table must be [nodes, dim]")
    dtype = _table_dtype(table)
    num_nodes, dim = int(table.shape[0]), int(table.shape[1])
    _one_device(table.device, out=None if out is None else out.data, ids=ids, count=count)
    if out is None:
        if ids is not None:
            raise ValueError("rows by their ids are written to an existing copy: pass out")
        out = Table8.empty(num_nodes, dim, table.device)
    if out.num_nodes != num_nodes or out.dim != dim:
        raise ValueError(f"out must have {num_nodes} rows of {dim} columns")
    n = num_nodes if ids is None else int(ids.numel())
    rc = lib().gs_quantize_rows(_at(table, None, "table"), num_nodes, dim, dtype, _at(ids, torch.int32, "ids"), n, _at(count, torch.int64, "count"),
                                out.data.data_ptr(), out.scales.data_ptr(), _stream_of(table.device))
    _check(rc, "gs_quantize_rows")
    return out


def gs_scores_q8_workspace_bytes(num_centers: int, num_nodes: int, dim: int) -> int:
    return int(lib().gs_scores_q8_workspace_bytes(num_centers, num_nodes, dim)) if 1 <= dim <= GS_Q8_MAX_DIM else 0


def gs_scores_q8(t_in: Table8, t_out: Table8, centers, bias=None, scale: float = 1.0, dtype=torch.float32, out=None, ws=None):
    """[n, nodes] of dtype (float32, bfloat16, float16): scale * <row centers[i] of t_in, row j of t_out> + bias[j]."""
    if t_in.dim != t_out.dim:
        raise ValueError("t_in and t_out must have the same dim")
    if bias is not None and tuple(bias.shape) != (t_out.num_nodes,):
        raise ValueError("bias must have one value per row of t_out")
    n, dev = int(centers.numel()), t_in.device
    _one_device(dev, t_out=t_out.data, centers=centers, bias=bias, out=out, ws=ws)
    out = _out(out, (n, t_out.num_nodes), dtype, dev, "out")
    if ws is None:
        ws = _workspace(gs_scores_q8_workspace_bytes(n, t_out.num_nodes, t_out.dim), dev)
    rc = lib().gs_scores_q8(
        t_in.data.data_ptr(), t_in.scales.data_ptr(), t_in.num_nodes, t_out.data.data_ptr(), t_out.scales.data_ptr(), t_out.num_nodes, t_out.dim,
        _at(centers, torch.int32, "centers"), n, _at(bias, torch.float32, "bias"), scale, _at(out, None, "out"), _table_dtype(out),
        _at(ws, torch.uint8, "ws"), ws.numel(), _stream_of(dev))
    _check(rc, "gs_scores_q8")
    return out


def gs_beam_select_workspace_bytes(groups: int, beams: int, n: int, width: int, dtype: int = GS_F32) -> int:
    if not (1 <= beams <= MOST_BEAMS and 1 <= width <= MOST_BEAMS):
        return 0
    return int(lib().gs_beam_select_workspace_bytes(groups, beams, n, width, dtype))


def gs_beam_select(scores, logp, beams: int, width: int, ended=None, parents_out=None, nodes_out=None, logp_out=None, ws=None):
    """The `width` best continuations of each group of `beams` walks, from scores [groups * beams, n] and logp float32
    [groups * beams]; ended: bool or uint8 [groups * beams].  Returns (parents, nodes int32, logp float32), [groups, width] each."""
    if scores.dim() != 2 or beams < 1 or scores.shape[0] % beams != 0:
        raise ValueError("scores must be [groups * beams, n]")
    if not 1 <= width <= MOST_BEAMS:
        raise ValueError(f"width must be from 1 to {MOST_BEAMS}")
    dtype = _table_dtype(scores)
    rows, n, dev = int(scores.shape[0]), int(scores.shape[1]), scores.device
    groups = rows // beams
    for name, t in (("logp", logp), ("ended", ended)):
        if t is not None and tuple(t.shape) != (rows,):
            raise ValueError(f"{name} must have one value per row of scores")
    if ended is not None and ended.dtype == torch.bool:
        ended = ended.view(torch.uint8)
    _one_device(dev, logp=logp, ended=ended, parents_out=parents_out, nodes_out=nodes_out, logp_out=logp_out, ws=ws)
    parents_out = _out(parents_out, (groups, width), torch.int32, dev, "parents_out")
    nodes_out = _out(nodes_out, (groups, width), torch.int32, dev, "nodes_out")
    logp_out = _out(logp_out, (groups, width), torch.float32, dev, "logp_out")
    if ws is None:
        ws = _workspace(gs_beam_select_workspace_bytes(groups, beams, n, width, dtype), dev)
    rc = lib().gs_beam_select(
        _at(scores, None, "scores"), groups, beams, n, dtype, _at(logp, torch.float32, "logp"), _at(ended, torch.uint8, "ended"), width,
        _at(parents_out, None, "parents_out"), _at(nodes_out, None, "nodes_out"), _at(logp_out, None, "logp_out"), _at(ws, torch.uint8, "ws"),
        ws.numel(), _stream_of(dev))
    _check(rc, "gs_beam_select")
    return parents_out, nodes_out, logp_out


def gs_beam_reorder(states, parents, beams: int, outs=None, nodes=None, columns=None):
    """Row g * width + k of each output becomes row g * beams + parents[g, k] of its state; a parent that is none leaves the row as it
    is.  states: tensors [groups * beams, ...] of any type; outs: tensors [groups * width, ...], or None (also one of them): in
    place.  columns: for each state None, or the column of an int32 state [rows, columns] at which nodes[g, k] is written."""
    if parents.dim() != 2:
        raise ValueError("parents must be [groups, width]")
    groups, width = int(parents.shape[0]), int(parents.shape[1])
    if nodes is not None and nodes.shape != parents.shape:
        raise ValueError("nodes must have the shape of parents")
    states, outs = list(states), [None] * len(states) if outs is None else list(outs)
    columns = [None] * len(states) if columns is None else list(columns)
    if len(outs) != len(states) or len(columns) != len(states):
        raise ValueError("one output and one column per state")
    _one_device(parents.device, nodes=nodes, **{f"states[{i}]": x for i, x in enumerate(states)}, **{f"outs[{i}]": x for i, x in enumerate(outs)})
    array = (StateStruct * len(states))()
    for i, (x, out, column) in enumerate(zip(states, outs, columns)):
        data = _at(x, None, "state")
        if x.dim() < 1 or x.shape[0] != groups * beams:
            raise ValueError(f"a state must have {groups * beams} rows")
        if out is not None and (out.dtype != x.dtype or tuple(out.shape) != (groups * width, *x.shape[1:])):
            raise ValueError("an output must have its state's type and rows")
        if out is None and beams != width:
            raise ValueError("in place there are as many walks as before: pass outs")
        row_bytes = math.prod(x.shape[1:]) * x.element_size()
        if column is not None and (x.dim() != 2 or x.dtype != torch.int32 or not 0 <= column < x.shape[1] or nodes is None):
            raise ValueError("nodes are written to a column of an int32 state [rows, columns]")
        array[i] = StateStruct(data, _at(out, None, "output"), row_bytes, -1 if column is None else 4 * column)
    rc = lib().gs_beam_reorder(C.addressof(array), len(states), groups, beams, width, _at(parents, torch.int32, "parents"),
                               _at(nodes, torch.int32, "nodes"), _stream_of(parents.device))
    _check(rc, "gs_beam_reorder")
