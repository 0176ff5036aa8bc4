"""ctypes binding of libtreelstm.so: same entry points as include/treelstm.h.

Argument marshalling only - every step of the forward pass runs in the HIP library.
PyTorch is used for device memory and for the stream handle.  There is no CPU
fallback: if the library has not been built, loading fails with an error.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtreelstm.so")

TL_TREELSTM, TL_TREERNN, TL_RNTN = 0, 1, 2
TL_F32, TL_BF16_IN = 0, 1
TL_SCHED_READY, TL_SCHED_LEVEL_DEVICE, TL_SCHED_LEVEL_HOST, TL_SCHED_READY_PRIORITY, TL_SCHED_DATAFLOW = 0, 1, 2, 3, 4
TL_OK, TL_EINVAL, TL_ENOMEM, TL_EHIP, TL_ESTRUCT, TL_ESTALL, TL_ELIMIT = 0, -1, -2, -3, -4, -5, -6
TL_NOALLOC_MAX_NODES = 16384
TL_N_STAGES, TL_PROFILE_RING = 5, 128
TL_DT_F32, TL_DT_BF16, TL_DT_F16 = 0, 1, 2
TL_GATE_SIGMOID, TL_GATE_GIVEN = 0, 1
SCHEDULERS = {"ready": TL_SCHED_READY, "level_device": TL_SCHED_LEVEL_DEVICE, "level_host": TL_SCHED_LEVEL_HOST,
              "ready_priority": TL_SCHED_READY_PRIORITY, "dataflow": TL_SCHED_DATAFLOW}

EXPORTS = ("tl_create", "tl_forward", "tl_forward_noalloc", "tl_status", "tl_set_profiling", "tl_stage_ms", "tl_last_stats", "tl_backward",
           "tl_set_keep_gates", "tl_set_async_backward", "tl_sgd_update", "tl_get_params", "tl_classify", "tl_classify_backward", "tl_td_create", "tl_td_generate", "tl_td_status", "tl_td_destroy", "tl_strerror", "tl_destroy",
           "tl_attend", "tl_attend_backward", "tl_attend_workspace", "tl_sample",
           "tl_recur", "tl_recur_backward", "tl_recur_workspace", "tl_score", "tl_score_backward", "tl_score_workspace", "tl_dropout")


class tl_config(ctypes.Structure):
    _fields_ = [("cell", ctypes.c_int), ("precision", ctypes.c_int), ("scheduler", ctypes.c_int),
                ("validate", ctypes.c_int), ("vocab", ctypes.c_int), ("embed_dim", ctypes.c_int),
                ("hidden", ctypes.c_int), ("spin_limit", ctypes.c_int),
                ("emb", ctypes.c_void_p), ("w_leaf", ctypes.c_void_p), ("b_leaf", ctypes.c_void_p),
                ("u", ctypes.c_void_p), ("b", ctypes.c_void_p), ("v", ctypes.c_void_p)]


class tl_rows(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class tl_attention(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("n_trees", ctypes.c_int), ("n_q", ctypes.c_int), ("n_kv", ctypes.c_int),
                ("n_heads", ctypes.c_int), ("n_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("scale", ctypes.c_float),
                ("q_off", ctypes.c_void_p), ("kv_off", ctypes.c_void_p), ("kv_mask", ctypes.c_void_p),
                ("q", tl_rows), ("k", tl_rows), ("v", tl_rows)]


class tl_recurrence(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("gate", ctypes.c_int), ("n_trees", ctypes.c_int), ("n_rows", ctypes.c_int), ("channels", ctypes.c_int),
                ("spin_limit", ctypes.c_int), ("off", ctypes.c_void_p), ("g", ctypes.c_void_p), ("x", ctypes.c_void_p), ("g_row", ctypes.c_int64), ("x_row", ctypes.c_int64)]


_lib = None


def lib():
    """The loaded library; raises if it has not been built (python -m paper_1809_00832_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libtreelstm.so is missing: build it with `python -m paper_1809_00832_amd.build` "
                               "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, ci = ctypes.c_void_p, ctypes.c_int
        L.tl_create.restype = ci
        L.tl_create.argtypes = [ctypes.POINTER(tl_config), ctypes.POINTER(vp)]
        L.tl_forward.restype = ci
        L.tl_forward.argtypes = [vp, ci, ci] + [vp] * 10
        L.tl_forward_noalloc.restype = ci
        L.tl_forward_noalloc.argtypes = [vp, ci, ci] + [vp] * 10
        L.tl_status.restype = ci
        L.tl_status.argtypes = [vp]
        L.tl_set_profiling.restype = ci
        L.tl_set_profiling.argtypes = [vp, ci]
        L.tl_stage_ms.restype = ci
        L.tl_stage_ms.argtypes = [vp, ci, ctypes.POINTER(ctypes.c_float)]
        L.tl_last_stats.restype = ci
        L.tl_last_stats.argtypes = [vp] + [ctypes.POINTER(ci)] * 3
        L.tl_strerror.restype = ctypes.c_char_p
        L.tl_backward.restype = ci
        L.tl_backward.argtypes = [vp, ci, ci] + [vp] * 13
        L.tl_sgd_update.restype = ci
        L.tl_sgd_update.argtypes = [vp, ctypes.c_float, ci] + [vp] * 8
        L.tl_get_params.restype = ci
        L.tl_get_params.argtypes = [vp] * 7
        L.tl_set_keep_gates.restype = ci
        L.tl_set_keep_gates.argtypes = [vp, ci]
        L.tl_set_async_backward.restype = ci
        L.tl_set_async_backward.argtypes = [vp, ci]
        L.tl_td_create.restype = ci
        L.tl_td_create.argtypes = [ci, vp, vp, vp, ctypes.c_float, ci, ctypes.POINTER(vp)]
        L.tl_td_generate.restype = ci
        L.tl_td_generate.argtypes = [vp, ci, ci, ci] + [vp] * 9
        L.tl_td_status.restype = ci
        L.tl_td_status.argtypes = [vp]
        L.tl_td_destroy.restype = ci
        L.tl_td_destroy.argtypes = [vp]
        L.tl_classify.restype = ci
        L.tl_classify.argtypes = [vp, ci, vp, vp, vp, ci, vp, vp]
        L.tl_classify_backward.restype = ci
        L.tl_classify_backward.argtypes = [vp, ci, vp, vp, vp, ci] + [vp] * 7
        L.tl_strerror.argtypes = [ci]
        attn, rows, i64 = vp, vp, ctypes.c_int64            # the structures by reference, or their bytes
        L.tl_attend_workspace.restype = ci
        L.tl_attend_workspace.argtypes = [attn, ci, ctypes.POINTER(i64)]
        L.tl_attend.restype = ci
        L.tl_attend.argtypes = [attn, rows, vp, vp, i64, vp]
        L.tl_attend_backward.restype = ci
        L.tl_attend_backward.argtypes = [attn, rows, vp, rows, rows, rows, rows, vp, i64, vp]
        L.tl_sample.restype = ci
        L.tl_sample.argtypes = [ci, ci, ci, vp, i64] + [vp] * 9
        f32 = ctypes.c_float
        for name, args in (("tl_recur_workspace", [vp, ci, ctypes.POINTER(i64)]), ("tl_recur", [vp, vp, vp, i64, vp, vp, vp, i64, vp]),
                           ("tl_recur_backward", [vp, vp, vp, i64, vp, vp, i64, vp, i64, vp, vp, i64, vp]),
                           ("tl_score_workspace", [ci, ci, ci, ci, ctypes.POINTER(i64)]),
                           ("tl_score", [ci, ci, ci, vp, i64, vp, ci, vp, vp, vp, vp, vp, i64, vp]),
                           ("tl_score_backward", [ci, ci, ci, vp, i64, vp, vp, vp, vp, vp, i64, vp]),
                           ("tl_dropout", [ci, ci, ci, vp, i64, vp, i64, vp, i64, f32, vp, vp])):
            getattr(L, name).restype, getattr(L, name).argtypes = ci, args
        L.tl_destroy.restype = ci
        L.tl_destroy.argtypes = [vp]
        _lib = L
    return _lib


class TLError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (%d)" % (where, lib().tl_strerror(code).decode(), code))


def _check(code: int, where: str):
    if code != TL_OK:
        raise TLError(code, where)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def tl_create(cell, precision, scheduler, vocab, embed_dim, hidden, emb, w_leaf=None, b_leaf=None, u=None, b=None,
              v=None, validate=0, spin_limit=0) -> int:
    """Device tensors (fp32, contiguous) in, context handle out."""
    for t in (emb, w_leaf, b_leaf, u, b, v):
        if t is not None:
            assert t.is_cuda and t.is_contiguous() and t.dtype.is_floating_point and t.element_size() == 4
    cfg = tl_config(cell, precision, scheduler, validate, vocab, embed_dim, hidden, spin_limit,
                    _ptr(emb), _ptr(w_leaf), _ptr(b_leaf), _ptr(u), _ptr(b), _ptr(v))
    out = ctypes.c_void_p()
    _check(lib().tl_create(ctypes.byref(cfg), ctypes.byref(out)), "tl_create")
    return out.value


def tl_forward(ctx, n_trees, n_nodes, tree_off, left, right, word, h, c=None, h_root=None, c_root=None, root=None,
               stream=None) -> None:
    """int32 / fp32 device tensors in and out; `stream` is a raw hipStream_t (int) or None for torch's current one."""
    import torch
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    _check(lib().tl_forward(ctx, n_trees, n_nodes, _ptr(tree_off), _ptr(left), _ptr(right), _ptr(word), _ptr(h),
                            _ptr(c), _ptr(h_root), _ptr(c_root), _ptr(root), stream), "tl_forward")


def tl_forward_noalloc(ctx, n_trees, n_nodes, tree_off, left, right, word, h, c=None, h_root=None, c_root=None, root=None,
                       stream=None) -> None:
    """Same arguments as tl_forward; the library allocates nothing during the call (fixed per-GPU workspace)."""
    import torch
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    _check(lib().tl_forward_noalloc(ctx, n_trees, n_nodes, _ptr(tree_off), _ptr(left), _ptr(right), _ptr(word), _ptr(h),
                                    _ptr(c), _ptr(h_root), _ptr(c_root), _ptr(root), stream), "tl_forward_noalloc")


def tl_status(ctx) -> int:
    return lib().tl_status(ctx)


def tl_set_profiling(ctx, on: bool) -> None:
    _check(lib().tl_set_profiling(ctx, int(on)), "tl_set_profiling")


def tl_stage_ms(ctx, back: int = 0):
    ms = (ctypes.c_float * TL_N_STAGES)()
    _check(lib().tl_stage_ms(ctx, back, ms), "tl_stage_ms")
    return dict(zip(("structure", "leaves", "internal", "roots", "total"), [float(x) for x in ms]))


def tl_last_stats(ctx):
    a, b, c = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(lib().tl_last_stats(ctx, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)), "tl_last_stats")
    return {"n_levels": a.value, "n_tiles": b.value, "n_workgroups": c.value}


def tl_backward(ctx, batch, g_h, embed_dim, rntn=False, stream=None):
    """Gradients for a batch that tl_forward has evaluated (`batch` is the dict TreeNet.load returns, holding h and
    c); g_h [N x H] float32 CUDA tensor.  Returns dict(d_u, d_b, d_w_leaf, d_b_leaf, d_x) of CUDA tensors for a
    TreeLSTM, dict(d_u [2H x H], d_b [H], d_x) for a TreeRNN (batch["c"] is None there), and with rntn=True also
    d_w_leaf [d x 2d x 2d], the gradient of the tensor V."""
    import torch
    N, H, E = batch["N"], int(batch["h"].shape[1]), int(embed_dim)
    assert g_h.is_cuda and g_h.dtype == torch.float32 and g_h.is_contiguous() and tuple(g_h.shape) == (N, H)
    dev = g_h.device
    lstm = batch.get("c") is not None
    ng = 5 if lstm else 1
    out = {"d_u": torch.empty((2 * H, ng * H), device=dev), "d_b": torch.empty(ng * H, device=dev),
           "d_x": torch.empty((N, E), device=dev)}
    if lstm:
        out["d_w_leaf"] = torch.empty((E, 3 * H), device=dev)
        out["d_b_leaf"] = torch.empty(3 * H, device=dev)
    elif rntn:
        out["d_w_leaf"] = torch.empty((H, 2 * H, 2 * H), device=dev)        # gradient of the tensor V
    st = (stream or torch.cuda.current_stream()).cuda_stream
    _check(lib().tl_backward(ctx, batch["B"], N, batch["tree_off"].data_ptr(), batch["left"].data_ptr(),
                             batch["right"].data_ptr(), batch["word"].data_ptr(), batch["h"].data_ptr(),
                             _ptr(batch.get("c")), g_h.data_ptr(), out["d_u"].data_ptr(), out["d_b"].data_ptr(),
                             _ptr(out.get("d_w_leaf")), _ptr(out.get("d_b_leaf")), out["d_x"].data_ptr(), st), "tl_backward")
    return out


def tl_sgd_update(ctx, lr, batch, grads, with_embedding=True, stream=None) -> None:
    """theta -= lr * gradient for the parameters the context holds; `grads` is what tl_backward returned, `batch`
    the dict TreeNet.load returned."""
    import torch
    st = (stream or torch.cuda.current_stream()).cuda_stream
    _check(lib().tl_sgd_update(ctx, float(lr), batch["N"], batch["left"].data_ptr(), batch["word"].data_ptr(),
                               grads["d_u"].data_ptr(), grads["d_b"].data_ptr(), _ptr(grads.get("d_w_leaf")),
                               _ptr(grads.get("d_b_leaf")), grads["d_x"].data_ptr() if with_embedding else None, st),
           "tl_sgd_update")


def tl_get_params(ctx, vocab, embed_dim, hidden, cell=TL_TREELSTM, stream=None):
    """The context's current parameters as new CUDA tensors: dict(u, b, w_leaf, b_leaf, emb); dict(u, b, emb) for a
    TreeRNN; dict(u, b, w_leaf = V [d x 2d x 2d], emb) for an RNTN."""
    import torch
    H, E = int(hidden), int(embed_dim)
    ng = 5 if cell == TL_TREELSTM else 1
    new = lambda *shape: torch.empty(shape, dtype=torch.float32, device="cuda")
    out = {"u": new(2 * H, ng * H), "b": new(ng * H), "emb": new(int(vocab), E)}
    if cell == TL_TREELSTM:
        out["w_leaf"], out["b_leaf"] = new(E, 3 * H), new(3 * H)
    elif cell == TL_RNTN:
        out["w_leaf"] = new(H, 2 * H, 2 * H)
    st = (stream or torch.cuda.current_stream()).cuda_stream
    _check(lib().tl_get_params(ctx, out["u"].data_ptr(), out["b"].data_ptr(), _ptr(out.get("w_leaf")), _ptr(out.get("b_leaf")),
                               out["emb"].data_ptr(), st), "tl_get_params")
    return out


def tl_set_keep_gates(ctx, on: bool) -> None:
    _check(lib().tl_set_keep_gates(ctx, 1 if on else 0), "tl_set_keep_gates")


def tl_set_async_backward(ctx, on) -> None:
    """True / 1: TreeLSTM and TreeRNN do not wait (RNTN returns the structure pass's status all the same); False / 0: the default;
    -1: always launches per height, which need no workgroups resident together."""
    _check(lib().tl_set_async_backward(ctx, int(on)), "tl_set_async_backward")


def tl_classify(ctx, h, w_s, b_s, probs=None, stream=None):
    """probs = softmax(h @ w_s + b_s) row by row; all arguments are float32 CUDA tensors.  Returns probs."""
    import torch
    n_rows, n_classes = int(h.shape[0]), int(w_s.shape[1])
    for t in (h, w_s, b_s):
        assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()
    if probs is None:
        probs = torch.empty((n_rows, n_classes), dtype=torch.float32, device=h.device)
    st = (stream or torch.cuda.current_stream()).cuda_stream
    _check(lib().tl_classify(ctx, n_rows, h.data_ptr(), w_s.data_ptr(), b_s.data_ptr(), n_classes, probs.data_ptr(), st),
           "tl_classify")
    return probs


def tl_classify_backward(ctx, h, w_s, b_s, label, stream=None):
    """Cross-entropy over the rows with a label in [0, C) on top of tl_classify.  h, w_s, b_s float32 and label
    int32 CUDA tensors.  Returns dict(loss [1], d_logits, g_h, d_w_s, d_b_s) of new float32 CUDA tensors."""
    import torch
    n_rows, n_classes = int(h.shape[0]), int(w_s.shape[1])
    for t in (h, w_s, b_s):
        assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()
    assert label.is_cuda and label.dtype == torch.int32 and label.is_contiguous() and label.numel() == n_rows
    new = lambda *shape: torch.empty(shape, dtype=torch.float32, device=h.device)
    out = {"loss": new(1), "d_logits": new(n_rows, n_classes), "g_h": new(n_rows, int(h.shape[1])),
           "d_w_s": new(int(h.shape[1]), n_classes), "d_b_s": new(n_classes)}
    st = (stream or torch.cuda.current_stream()).cuda_stream
    _check(lib().tl_classify_backward(ctx, n_rows, h.data_ptr(), w_s.data_ptr(), b_s.data_ptr(), n_classes,
                                      label.data_ptr(), out["d_logits"].data_ptr(), out["g_h"].data_ptr(),
                                      out["d_w_s"].data_ptr(), out["d_b_s"].data_ptr(), out["loss"].data_ptr(), st),
           "tl_classify_backward")
    return out


def tl_td_create(hidden, u_td, b_td, w_stop, b_stop, spin_limit=0):
    """Context of the top-down generator; u_td [H x 8H], b_td [8H], w_stop [H] float32 CUDA tensors."""
    import torch
    for t in (u_td, b_td, w_stop):
        assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()
    assert tuple(u_td.shape) == (hidden, 8 * hidden) and b_td.numel() == 8 * hidden and w_stop.numel() == hidden
    ctx = ctypes.c_void_p()
    _check(lib().tl_td_create(int(hidden), u_td.data_ptr(), b_td.data_ptr(), w_stop.data_ptr(), float(b_stop), int(spin_limit),
                              ctypes.byref(ctx)), "tl_td_create")
    return ctx


def tl_td_generate(ctx, h_root, c_root, max_nodes, max_depth, stream=None):
    """Grows one tree per row of h_root / c_root (float32 CUDA tensors [B x H]).  Returns a dict of new CUDA tensors
    with max_nodes rows each (h, c, parent, left, right, depth, score) and counts [4]; asynchronous."""
    import torch
    B, H = int(h_root.shape[0]), int(h_root.shape[1])
    assert h_root.is_cuda and c_root.is_cuda and h_root.dtype == torch.float32 and tuple(c_root.shape) == (B, H)
    dev = h_root.device
    out = {"h": torch.empty((max_nodes, H), device=dev), "c": torch.empty((max_nodes, H), device=dev),
           "score": torch.empty(max_nodes, device=dev), "counts": torch.zeros(4, dtype=torch.int32, device=dev)}
    for k in ("parent", "left", "right", "depth"):
        out[k] = torch.empty(max_nodes, dtype=torch.int32, device=dev)
    out["h"][:B].copy_(h_root)
    out["c"][:B].copy_(c_root)
    tl_td_generate_into(ctx, B, max_depth, out, stream)
    return out


def tl_td_generate_into(ctx, n_trees, max_depth, out, stream=None):
    """The call itself on buffers that tl_td_generate allocated (root rows in place)."""
    import torch
    st = (stream or torch.cuda.current_stream()).cuda_stream
    _check(lib().tl_td_generate(ctx, int(n_trees), int(out["h"].shape[0]), int(max_depth), out["h"].data_ptr(), out["c"].data_ptr(),
                                out["parent"].data_ptr(), out["left"].data_ptr(), out["right"].data_ptr(),
                                out["depth"].data_ptr(), out["score"].data_ptr(), out["counts"].data_ptr(), st), "tl_td_generate")


def tl_td_status(ctx) -> int:
    return lib().tl_td_status(ctx)


def tl_td_destroy(ctx) -> None:
    _check(lib().tl_td_destroy(ctx), "tl_td_destroy")


def _dtype(t) -> int:
    import torch
    d = t.dtype
    if d is torch.float32:
        return TL_DT_F32
    assert d is torch.bfloat16 or d is torch.float16, "float32, bfloat16 or float16"
    return TL_DT_BF16 if d is torch.bfloat16 else TL_DT_F16


def _raw_stream(index) -> int:
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)        # (the public call takes 3 us, as long as a launch)
    return raw(index) if raw else torch.cuda.current_stream(index).cuda_stream


def _elsewhere(index, stream):
    """A context in which launches go to the given stream, or to the device `index` where that is not the current one.  (The callers compare with
    torch._C._cuda_getDevice, which is torch.cuda.current_device without its check of the set-up: a short call is bound by the host's time.)"""
    import torch
    assert index >= 0 and (stream is None or stream.device_index == index), "CUDA tensors, and a stream of their device"
    return torch.cuda.stream(stream) if stream is not None else torch.cuda.device(index)


# tl_attention and tl_rows as bytes: packing takes a quarter of the time of filling the structures
_PACK_ATTENTION, _PACK_ROWS = struct.Struct("7if3Q9q").pack, struct.Struct("Q2q").pack
assert struct.calcsize("7if3Q9q") == ctypes.sizeof(tl_attention) and struct.calcsize("Q2q") == ctypes.sizeof(tl_rows)


def _rows(t, like, shape, index):
    assert t.get_device() == index and t.dtype == like.dtype and t.shape == shape and (shape[2] == 1 or t.stride(2) == 1), "rows, heads and a contiguous head_dim"
    return _PACK_ROWS(t.data_ptr(), t.stride(0), t.stride(1))


def _attention(q, k, v, q_off, kv_off, kv_mask, scale, index) -> bytes:
    import torch
    n_q, n_heads, d = q.shape
    n_kv, n_kv_heads, dk = k.shape
    dtype = q.dtype
    assert index == k.get_device() == v.get_device() == q_off.get_device() == kv_off.get_device(), "tensors of one device"
    assert k.dtype == dtype and v.dtype == dtype and dk == d and v.shape == k.shape
    q_row, q_head, q_d = q.stride()
    k_row, k_head, k_d = k.stride()
    v_row, v_head, v_d = v.stride()
    assert d == 1 or q_d == k_d == v_d == 1, "head_dim must be contiguous"
    int32 = torch.int32
    assert q_off.dtype == int32 and q_off.is_contiguous() and kv_off.dtype == int32 and kv_off.is_contiguous()
    n_off = q_off.numel()
    assert n_off == kv_off.numel() >= 1
    mask = 0
    if kv_mask is not None:
        assert kv_mask.get_device() == index and kv_mask.dtype in (torch.uint8, torch.bool) and kv_mask.is_contiguous() and kv_mask.numel() == n_kv
        mask = kv_mask.data_ptr()
    return _PACK_ATTENTION(_dtype(q), n_off - 1, n_q, n_kv, n_heads, n_kv_heads, d, d ** -0.5 if scale is None else scale, q_off.data_ptr(),
                           kv_off.data_ptr(), mask, q.data_ptr(), q_row, q_head, k.data_ptr(), k_row, k_head, v.data_ptr(), v_row, v_head)


def _attend_workspace(a, backward, device):
    import torch
    size = ctypes.c_int64()
    _check(lib().tl_attend_workspace(a, backward, ctypes.byref(size)), "tl_attend_workspace")
    n = size.value
    return (torch.empty(n, dtype=torch.uint8, device=device), n) if n else (None, 0)


def tl_attend(q, k, v, q_off, kv_off, kv_mask=None, scale=None, o=None, with_lse=False, stream=None):
    """Cross attention of every tree's queries to its nodes.  q [n_q, heads, D], k and v [n_kv, kv_heads, D]: CUDA tensors of one type
    (float32, bfloat16, float16) with any strides of rows and heads; q_off, kv_off [n_trees + 1] int32; kv_mask [n_kv] uint8 or bool,
    0 for nodes that are not read; scale: 1 / sqrt(D) if None.  All on one device, where the call goes, on its current stream or `stream`.
    Returns o, or (o, lse [n_q, heads] float32)."""
    import torch
    index = q.get_device()
    if stream is not None or torch._C._cuda_getDevice() != index:
        with _elsewhere(index, stream):
            return tl_attend(q, k, v, q_off, kv_off, kv_mask, scale, o, with_lse)
    a = _attention(q, k, v, q_off, kv_off, kv_mask, scale, index)
    shape, device = q.shape, q.device
    if o is None:
        o = torch.empty_like(q) if q.is_contiguous() else q.new_empty(shape)
    lse = torch.empty(shape[:2], dtype=torch.float32, device=device) if with_lse else None
    call, rows, at, st = lib().tl_attend, _rows(o, q, shape, index), _ptr(lse), _raw_stream(index)
    code = call(a, rows, at, None, 0, st)
    if code == TL_ELIMIT:                                       # (most calls need no workspace: asking first would cost them a call)
        ws, n = _attend_workspace(a, 0, device)
        code = call(a, rows, at, _ptr(ws), n, st)
    _check(code, "tl_attend")
    return (o, lse) if with_lse else o


def tl_attend_backward(q, k, v, o, lse, d_o, q_off, kv_off, kv_mask=None, scale=None, stream=None):
    """Gradients of tl_attend for its arguments and what it returned; d_o like o.  Returns dict(d_q, d_k, d_v) of new tensors."""
    import torch
    index = q.get_device()
    if stream is not None or torch._C._cuda_getDevice() != index:
        with _elsewhere(index, stream):
            return tl_attend_backward(q, k, v, o, lse, d_o, q_off, kv_off, kv_mask, scale)
    a = _attention(q, k, v, q_off, kv_off, kv_mask, scale, index)
    q_shape, kv_shape, device = q.shape, k.shape, q.device
    assert lse.get_device() == index and lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == q_shape[:2]
    d_q, d_k, d_v = q.new_empty(q_shape), q.new_empty(kv_shape), q.new_empty(kv_shape)
    ws, n = _attend_workspace(a, 1, device)
    _check(lib().tl_attend_backward(a, _rows(o, q, q_shape, index), lse.data_ptr(), _rows(d_o, q, q_shape, index), _rows(d_q, q, q_shape, index), _rows(d_k, q, kv_shape, index),
                                    _rows(d_v, q, kv_shape, index), _ptr(ws), n, _raw_stream(index)), "tl_attend_backward")
    return {"d_q": d_q, "d_k": d_k, "d_v": d_v}


def tl_sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    """One word per row of logits [n, vocab] (float32, bfloat16 or float16; rows any stride apart) from the uniform numbers u [n] float32;
    temperature, top_p, min_p [n] float32 and top_k [n] int32 CUDA tensors, None: off.  Returns dict(token int32, logprob float32,
    kept int32) of new tensors [n]."""
    import torch
    index = logits.get_device()
    if stream is not None or torch._C._cuda_getDevice() != index:
        with _elsewhere(index, stream):
            return tl_sample(logits, u, temperature, top_k, top_p, min_p)
    n, vocab = logits.shape
    device = logits.device
    assert vocab == 1 or logits.stride(1) == 1
    for t, dt in ((u, torch.float32), (temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32)):
        assert t is None or (t.get_device() == index and t.dtype == dt and t.is_contiguous() and t.numel() == n)
    out = {"token": torch.empty(n, dtype=torch.int32, device=device), "logprob": torch.empty(n, dtype=torch.float32, device=device),
           "kept": torch.empty(n, dtype=torch.int32, device=device)}
    _check(lib().tl_sample(_dtype(logits), n, vocab, logits.data_ptr(), logits.stride(0), u.data_ptr(), _ptr(temperature), _ptr(top_k),
                           _ptr(top_p), _ptr(min_p), out["token"].data_ptr(), out["logprob"].data_ptr(), out["kept"].data_ptr(),
                           _raw_stream(index)), "tl_sample")
    return out


_PACK_RECURRENCE = struct.Struct("6i3Q2q").pack
assert struct.calcsize("6i3Q2q") == ctypes.sizeof(tl_recurrence)


def _recurrence(g, x, off, gate, index, spin_limit=0) -> bytes:
    import torch
    n, channels = g.shape
    dtype = g.dtype
    assert index == x.get_device() == off.get_device(), "tensors of one device"
    assert x.dtype is dtype and x.shape == g.shape
    g_row, g_c = g.stride()
    x_row, x_c = x.stride()
    assert channels == 1 or g_c == x_c == 1, "channels must be contiguous"
    n_off = off.numel()
    assert off.dtype is torch.int32 and off.is_contiguous() and n_off >= 1
    return _PACK_RECURRENCE(_dtype(g), gate, n_off - 1, n, channels, spin_limit, off.data_ptr(), g.data_ptr(), x.data_ptr(), g_row, x_row)


def _recur_workspace(r, backward, device):
    import torch
    size = ctypes.c_int64()
    _check(lib().tl_recur_workspace(r, backward, ctypes.byref(size)), "tl_recur_workspace")
    n = size.value
    return (torch.empty(n, dtype=torch.uint8, device=device), n) if n else (None, 0)


def _states(t, index, shape):
    import torch
    if t is None:
        return None
    assert t.get_device() == index and t.dtype is torch.float32 and t.is_contiguous() and t.shape == shape
    return t.data_ptr()


def _like(t, like, index):
    """Rows of the type and shape of `like`: address and stride."""
    row, c = t.stride()
    assert t.get_device() == index and t.dtype is like.dtype and t.shape == like.shape and (c == 1 or t.shape[1] == 1)
    return t.data_ptr(), row


def _floats(t, shape):
    """A new float32 tensor on the device of t.  (new_empty of t's own type takes a quarter less than torch.empty with a type and a device.)"""
    import torch
    return t.new_empty(shape) if t.dtype is torch.float32 else t.new_empty(shape, dtype=torch.float32)


def _new_like(t, shape):
    """A new contiguous tensor of the type of t."""
    import torch
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(shape)


def tl_recur(g, x, off, h0=None, gate=TL_GATE_SIGMOID, h=None, h_last=None, with_last=False, with_tape=False, stream=None, spin_limit=0):
    """h_t = f_t h_(t-1) + i_t x_t along the rows of every sentence.  g, x [n, channels]: CUDA tensors of one type (float32, bfloat16, float16)
    with rows any stride apart; off [sentences + 1] int32, from 0 to at most n; h0 [sentences, channels] float32, None: zero.  Returns dict(h,
    h_last with with_last or where one is given, tape with with_tape): h is new unless given (its rows behind the last sentence are left
    as they were, of a new one undefined), h_last [sentences, channels] float32 may be h0 itself, the tape is for tl_recur_backward.  spin_limit: most polls of
    a wait between workgroups (0: default, below 0: none)."""
    import torch
    index = g.get_device()
    if stream is not None or torch._C._cuda_getDevice() != index:
        with _elsewhere(index, stream):
            return tl_recur(g, x, off, h0, gate, h, h_last, with_last, with_tape, None, spin_limit)
    r = _recurrence(g, x, off, gate, index, spin_limit)
    n, channels = g.shape
    trees, device = off.numel() - 1, g.device
    state = (trees, channels)
    if h is None:
        h = _new_like(g, (n, channels))
        at, row = h.data_ptr(), channels
    else:
        at, row = _like(h, g, index)
    out = {"h": h}
    first, last, tape = _states(h0, index, state), None, None
    if h_last is not None:
        last = _states(h_last, index, state)
    elif with_last:
        h_last = torch.empty_like(h0) if h0 is not None else _floats(g, state)
        last = h_last.data_ptr()
    if last is not None:
        out["h_last"] = h_last
    if with_tape:
        out["tape"] = t = _floats(g, (n // 64 + trees, channels))
        tape = t.data_ptr()
    call, st = lib().tl_recur, _raw_stream(index)
    code = call(r, first, at, row, last, tape, None, 0, st)
    if code == TL_ELIMIT:
        ws, size = _recur_workspace(r, 0, device)
        code = call(r, first, at, row, last, tape, _ptr(ws), size, st)
    _check(code, "tl_recur")
    return out


def tl_recur_backward(g, x, off, tape, d_h=None, d_last=None, gate=TL_GATE_SIGMOID, stream=None, spin_limit=0):
    """Gradients of tl_recur for its arguments and its tape: d_h [n, channels] of the type of g, d_last [sentences, channels] float32, None: zero.
    Returns dict(d_g, d_x, d_h0) of new tensors; rows of d_g and d_x behind the last sentence are zero."""
    import torch
    index = g.get_device()
    if stream is not None or torch._C._cuda_getDevice() != index:
        with _elsewhere(index, stream):
            return tl_recur_backward(g, x, off, tape, d_h, d_last, gate, None, spin_limit)
    r = _recurrence(g, x, off, gate, index, spin_limit)
    n, channels = g.shape
    trees, device = off.numel() - 1, g.device
    state = (trees, channels)
    d_g = _new_like(g, (n, channels))
    d_x = torch.empty_like(d_g)
    d_h0 = torch.empty_like(d_last) if d_last is not None else _floats(g, state)
    at, row = _like(d_h, g, index) if d_h is not None else (None, 0)
    call, kept, last, st = lib().tl_recur_backward, _states(tape, index, (n // 64 + trees, channels)), _states(d_last, index, state), _raw_stream(index)
    rest = (d_g.data_ptr(), channels, d_x.data_ptr(), channels, d_h0.data_ptr())
    code = call(r, kept, at, row, last, *rest, None, 0, st)
    if code == TL_ELIMIT:
        ws, size = _recur_workspace(r, 1, device)
        code = call(r, kept, at, row, last, *rest, _ptr(ws), size, st)
    _check(code, "tl_recur_backward")
    return {"d_g": d_g, "d_x": d_x, "d_h0": d_h0}


def _words(t, n, index):
    import torch
    if t is None:
        return None
    assert t.get_device() == index and t.dtype is torch.int32 and t.is_contiguous() and t.numel() == n
    return t.data_ptr()


def tl_score(logits, word=None, n_top=0, stream=None):
    """Log probabilities of given words, entropies, and the n_top (up to 64) most probable words of rows of logits [n, vocab] (float32, bfloat16 or
    float16; rows any stride apart); word [n] int32, outside [0, vocab) where a row has none.  Returns dict(entropy [n], stats [3, n] for
    tl_score_backward, logprob [n] with words, top_word [n, n_top] int32 and top_logprob [n, n_top] with n_top > 0) of new tensors; entropy is a row
    of stats."""
    import torch
    index = logits.get_device()
    if stream is not None or torch._C._cuda_getDevice() != index:
        with _elsewhere(index, stream):
            return tl_score(logits, word, n_top)
    n, vocab = logits.shape
    device, dtype = logits.device, _dtype(logits)
    row, c = logits.stride()
    assert vocab == 1 or c == 1
    words = _words(word, n, index)
    stats = _floats(logits, (3, n))
    at = stats.data_ptr()
    out = {"entropy": stats[2], "stats": stats}
    log_at = top_at = top_log_at = None
    if words is not None:
        out["logprob"] = t = _floats(stats, (n,))
        log_at = t.data_ptr()
    if n_top > 0:
        shape = (n, n_top)
        out["top_word"] = t = word.new_empty(shape) if word is not None else torch.empty(shape, dtype=torch.int32, device=device)
        out["top_logprob"] = p = _floats(stats, shape)
        top_at, top_log_at = t.data_ptr(), p.data_ptr()
    call, st = lib().tl_score, _raw_stream(index)
    args = (dtype, n, vocab, logits.data_ptr(), row, words, n_top, log_at, at, top_at, top_log_at)
    code = call(*args, None, 0, st)
    if code == TL_ELIMIT:
        size = ctypes.c_int64()
        _check(lib().tl_score_workspace(dtype, n, vocab, n_top, ctypes.byref(size)), "tl_score_workspace")
        ws = torch.empty(size.value, dtype=torch.uint8, device=device)
        code = call(*args, ws.data_ptr(), size.value, st)
    _check(code, "tl_score")
    return out


def tl_score_backward(logits, word, stats, d_logprob=None, d_entropy=None, d_logits=None, stream=None):
    """Gradient of the logits from those of tl_score's logprob and entropy ([n] float32, None: zero), its arguments and its stats.  d_logits may be
    logits itself (new if None) and is returned."""
    import torch
    index = logits.get_device()
    if stream is not None or torch._C._cuda_getDevice() != index:
        with _elsewhere(index, stream):
            return tl_score_backward(logits, word, stats, d_logprob, d_entropy, d_logits)
    n, vocab = logits.shape
    x_row, c = logits.stride()
    assert vocab == 1 or c == 1
    if d_logits is None:
        d_logits = _new_like(logits, (n, vocab))
        at, row = d_logits.data_ptr(), vocab
    else:
        at, row = _like(d_logits, logits, index)
    _check(lib().tl_score_backward(_dtype(logits), n, vocab, logits.data_ptr(), x_row, _words(word, n, index), _states(stats, index, (3, n)),
                                   _states(d_logprob, index, (n,)), _states(d_entropy, index, (n,)), at, row, _raw_stream(index)), "tl_score_backward")
    return d_logits


def tl_dropout(x, p, numbers, residual=None, y=None, stream=None):
    """y = residual + dropout(x): x, residual, y [n, columns] CUDA tensors of one type (float32, bfloat16, float16) with rows any stride apart; p: share of
    dropped values; numbers [2] int64: seed and step.  y may be x or residual (new if None) and is returned.  The gradient of x is the same
    call on that of y without a residual."""
    import torch
    index = x.get_device()
    if stream is not None or torch._C._cuda_getDevice() != index:
        with _elsewhere(index, stream):
            return tl_dropout(x, p, numbers, residual, y)
    n, cols = x.shape
    assert numbers.get_device() == index and numbers.dtype in (torch.int64, torch.uint64) and numbers.is_contiguous() and numbers.numel() == 2
    x_row, c = x.stride()
    assert cols == 1 or c == 1
    r_at, r_row = _like(residual, x, index) if residual is not None else (None, 0)
    if y is None:
        y = _new_like(x, (n, cols))
        y_at, y_row = y.data_ptr(), cols
    else:
        y_at, y_row = _like(y, x, index)
    _check(lib().tl_dropout(_dtype(x), n, cols, x.data_ptr(), x_row, r_at, r_row, y_at, y_row, p, numbers.data_ptr(), _raw_stream(index)), "tl_dropout")
    return y


def tl_strerror(code: int) -> str:
    return lib().tl_strerror(code).decode()


def tl_destroy(ctx) -> None:
    _check(lib().tl_destroy(ctx), "tl_destroy")


class TreeNet:
    """Holds a context plus device copies of a batch; thin convenience over the calls above."""

    def __init__(self, params, scheduler="ready", precision=TL_F32, validate=0, spin_limit=0, device="cuda:0"):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        dev = lambda a: None if a is None else torch.from_numpy(a).to(self.device).contiguous()
        self.cell, self.H = params.cell, params.hidden
        self.ctx = tl_create(params.cell, precision, SCHEDULERS[scheduler], params.vocab, params.embed_dim,
                             params.hidden, dev(params.emb), dev(params.w_leaf), dev(params.b_leaf), dev(params.u),
                             dev(params.b), dev(params.v), validate=validate, spin_limit=spin_limit)
        self.batch = None

    def load(self, trees):
        """Copies a batch (numpy int32 arrays) to the device and allocates the outputs."""
        torch = self.torch
        dev = lambda a: torch.from_numpy(a).to(self.device).contiguous()
        B, N, H = trees.n_trees, trees.n_nodes, self.H
        out = lambda *s: torch.empty(*s, dtype=torch.float32, device=self.device)
        self.batch = dict(B=B, N=N, tree_off=dev(trees.tree_off), left=dev(trees.left), right=dev(trees.right),
                          word=dev(trees.word), h=out(N, H), c=out(N, H) if self.cell == TL_TREELSTM else None,
                          h_root=out(B, H), c_root=out(B, H) if self.cell == TL_TREELSTM else None,
                          root=torch.empty(B, dtype=torch.int32, device=self.device))
        return self.batch

    def forward(self, stream=None):
        b = self.batch
        tl_forward(self.ctx, b["B"], b["N"], b["tree_off"], b["left"], b["right"], b["word"], b["h"], b["c"],
                   b["h_root"], b["c_root"], b["root"], stream)

    def run(self, trees):
        """load + forward + status check; returns host numpy copies of the outputs."""
        self.load(trees)
        self.forward()
        code = tl_status(self.ctx)
        if code != TL_OK:
            raise TLError(code, "tl_forward (device)")
        b = self.batch
        host = lambda t: None if t is None else t.cpu().numpy()
        return {k: host(b[k]) for k in ("h", "c", "h_root", "c_root", "root")}

    def close(self):
        if self.ctx:
            tl_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
