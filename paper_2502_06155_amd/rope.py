"""Python binding of the C ABI in include/head_rope.h: norms of queries and keys for each head, rotation by
positions, and the layout of the attention entry points (argument marshalling, checks and workspaces only).

The functions named as in the header take its arguments; the torch wrappers below them (head_rope,
head_rope_grad) check shapes, types and devices, allocate outputs and workspaces and run on the current
stream of the tensors' device. rope_freqs and grid_positions make what they take, once for a program.
"""
from __future__ import annotations

import ctypes
import functools
import struct

from ._lib import lib
from .api import _check, _ptr, _stream
from .blocks import _current, _on, _unrecorded, _want, _workspace

try:
    import torch
except ImportError:  # the functions of the C ABI take addresses and do without
    torch = None

ROPE_AXES = 4
NORMS = {None: 0, "rms": 1, "layer": 2}
ROPE_LAYOUTS = {None: 0, "interleaved": 1, "halves": 2, "split": 3}


class Rows(ctypes.Structure):
    """ta_rows: an address and the strides of sequence, token and head, in values."""

    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64),
                ("head", ctypes.c_int64)]


class HeadRopeSpec(ctypes.Structure):
    """head_rope_spec."""

    _fields_ = [("B", ctypes.c_int), ("S", ctypes.c_int), ("H", ctypes.c_int), ("Hkv", ctypes.c_int),
                ("d", ctypes.c_int), ("norm", ctypes.c_int), ("eps", ctypes.c_float),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("q_bias", ctypes.c_void_p),
                ("k_bias", ctypes.c_void_p), ("layout", ctypes.c_int), ("axes", ctypes.c_int),
                ("dims", ctypes.c_int * ROPE_AXES), ("freqs", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("positions_batch", ctypes.c_int64), ("lens", ctypes.c_void_p)]


def _ref(x):
    """The address of a struct: a Structure's, or bytes laid out alike."""
    return x if x is None or type(x) is bytes else ctypes.byref(x)


def head_rope_fwd(spec, q, k, v, q_out, k_out, v_out, stream=None) -> None:
    """head_rope_fwd of the C ABI: q, k, v are Rows or None."""
    _check(lib.head_rope_fwd(_ref(spec), _ref(q), _ref(k), _ref(v), _ptr(q_out), _ptr(k_out), _ptr(v_out),
                             _stream(stream)), "head_rope_fwd")


def head_rope_bwd_workspace(spec) -> int:
    """Bytes of workspace that head_rope_bwd needs for this spec."""
    n = ctypes.c_size_t(0)
    _check(lib.head_rope_bwd_workspace(_ref(spec), ctypes.byref(n)), "head_rope_bwd_workspace")
    return n.value


@functools.lru_cache(maxsize=1024)
def _grad_workspace(B: int, S: int, H: int, Hkv: int, d: int) -> int:
    """head_rope_bwd_workspace of a spec of these sizes with a norm."""
    return head_rope_bwd_workspace(HeadRopeSpec(B=B, S=S, H=H, Hkv=Hkv, d=d, norm=1, eps=1.0))


def head_rope_bwd(spec, q, k, dq_out, dk_out, dv_out, dq, dk, dv, dq_weight=None, dk_weight=None, dq_bias=None,
                  dk_bias=None, workspace=None, workspace_bytes: int = 0, stream=None) -> None:
    """head_rope_bwd of the C ABI: q, k, dq, dk, dv are Rows or None."""
    _check(lib.head_rope_bwd(_ref(spec), _ref(q), _ref(k), _ptr(dq_out), _ptr(dk_out), _ptr(dv_out), _ref(dq),
                             _ref(dk), _ref(dv), _ptr(dq_weight), _ptr(dk_weight), _ptr(dq_bias), _ptr(dk_bias),
                             _ptr(workspace), workspace_bytes, _stream(stream)), "head_rope_bwd")


# ---------------------------------------------------------------------------------------------
# torch wrappers


def rope_freqs(dims, theta: float = 10000.0, device="cuda"):
    """The usual frequencies of axes of `dims` values: theta^(-2 j / n) for pair j of an axis of n, fp64
    [sum(dims) / 2]."""
    return torch.cat([theta ** (-torch.arange(0, n, 2, dtype=torch.float64) / n) for n in dims]).to(device)


def grid_positions(frames: int, height: int, width: int, text: int = 0, device="cuda"):
    """int32 [text + frames * height * width, 3]: time, height and width of a video's tokens, frame after
    frame; `text` tokens before it stand at 0 and are not turned."""
    f, h, w = (torch.arange(n, dtype=torch.int32) for n in (frames, height, width))
    grid = torch.stack(torch.meshgrid(f, h, w, indexing="ij"), -1).reshape(-1, 3)
    return torch.cat([torch.zeros(text, 3, dtype=torch.int32), grid]).to(device)


# The structs as bytes, which ctypes passes by address: a third of the time that building a Structure takes.
_PACKED_ROWS = struct.Struct("Pqqq")
_PACKED_SPEC = struct.Struct("6if4x4P2i4i2PqP")
_WEIGHTS = ("q_weight", "k_weight", "q_bias", "k_bias")


def _rows(t, name: str, B: int, S: int, heads: int, d: int, device) -> bytes:
    """t is a bf16 [B, S, heads, d] tensor on this GPU whose values of a head lie together."""
    if t.dtype is not torch.bfloat16 or t.shape != (B, S, heads, d) or t.device != device:
        if t.shape != (B, S, heads, d):
            raise ValueError(f"{name} must have the shape {(B, S, heads, d)}, got {tuple(t.shape)}")
        if t.dtype is not torch.bfloat16:
            raise ValueError(f"{name} must be {torch.bfloat16}, got {t.dtype}")
        raise ValueError(f"{name} must be on the GPU {device}, got {t.device}")
    batch, token, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    # (The stride of a dimension of one place says nothing.)
    return _PACKED_ROWS.pack(t.data_ptr(), batch if B > 1 else 0, token if S > 1 else 0, head if heads > 1 else 0)


_STILL = (0,) * 9


def _spec(q, k, v, positions, freqs, dims, layout, weights, norm, eps, lens):
    """(spec, device, B, S, H, Hkv, d) of the wrappers' arguments."""
    some = q if q is not None else k if k is not None else v
    if some is None:
        raise ValueError("one of q, k and v must be given")
    if some.dim() != 4 or not some.is_cuda:
        raise ValueError("expected [B, S, heads, d] tensors on a GPU")
    B, S, H, d = some.shape
    device = some.device
    if q is None:
        Hkv, H = H, 1
    else:
        heads = k if k is not None else v
        Hkv = heads.shape[2] if heads is not None and heads.dim() == 4 else 1
    if norm not in NORMS:
        raise ValueError(f"norm must be one of {list(NORMS)}, got {norm!r}")
    if layout not in ROPE_LAYOUTS:
        raise ValueError(f"layout must be one of {list(ROPE_LAYOUTS)}, got {layout!r}")
    at = [0, 0, 0, 0]
    for i, t in enumerate(weights):
        if t is not None:
            _want(t, _WEIGHTS[i], (d,), torch.float32, device)
            at[i] = t.data_ptr()
    turn = _STILL
    if positions is not None:
        dims = (d,) if dims is None else tuple(dims)
        n = len(dims)
        if not 1 <= n <= ROPE_AXES:
            raise ValueError(f"dims must name 1 to {ROPE_AXES} axes")
        if freqs is None or layout is None:
            raise ValueError("positions need freqs and a layout")
        _want(freqs, "freqs", (sum(dims) // 2,), torch.float64, device)
        shared = positions.dim() == 2
        _want(positions, "positions", (S, n) if shared else (B, S, n), torch.int32, device)
        turn = (ROPE_LAYOUTS[layout], n, *dims, *_STILL[n:ROPE_AXES], freqs.data_ptr(), positions.data_ptr(),
                0 if shared else S * n)
    if lens is not None:
        _want(lens, "lens", (B,), torch.int32, device)
        lens = lens.data_ptr()
    return _PACKED_SPEC.pack(B, S, H, Hkv, d, NORMS[norm], eps, *at, *turn, lens or 0), device, B, S, H, Hkv, d


def head_rope(q, k, v, positions=None, freqs=None, dims=None, layout="interleaved", norm=None, q_weight=None,
              k_weight=None, q_bias=None, k_bias=None, eps: float = 1e-6, lens=None, out=None):
    """Norms, rotation and layout of a projection's heads: q [B, S, H, d], k and v [B, S, Hkv, d] bf16, of any
    strides that keep a head's values together (views of one projection), to (q [B, H, S, d], k, v
    [B, Hkv, S, d]) as attention takes them. Any of the three may be None.

    norm: None, "rms" or "layer" over the d values of every head of q and k, with fp32 weights (and, "layer",
    biases) [d]. positions: int32 [S, axes] or [B, S, axes]; freqs: fp64 [sum(dims) / 2] (rope_freqs); dims: how many
    values of a head turn with each axis, (d,) if not given, the rest stays; layout: which values are pairs,
    "interleaved" (2 j, 2 j + 1), "halves" (j and n / 2 + j of an axis' n) or "split" (p and R / 2 + p of all R turned
    values). Without positions nothing is turned. lens (int32 [B]): tokens behind a sequence's end give zeros.
    out: the three results' tensors. Autograd does not record it (it warns where it would have): head_rope_grad
    gives the gradients."""
    weights = (q_weight, k_weight, q_bias, k_bias)
    spec, device, B, S, H, Hkv, d = _spec(q, k, v, positions, freqs, dims, layout, weights, norm, eps, lens)
    _unrecorded("head_rope", "head_rope_grad gives the gradients", (q, k, v, *weights))
    rows, outs, at = [None, None, None], [None, None, None], [None, None, None]
    for i, t in enumerate((q, k, v)):
        if t is None:
            continue
        heads = Hkv if i else H
        rows[i] = _rows(t, "qkv"[i], B, S, heads, d, device)
        if out is None:
            y = t.new_empty((B, heads, S, d))
        else:
            y = out[i]
            _want(y, "out", (B, heads, S, d), torch.bfloat16, device)
        outs[i], at[i] = y, y.data_ptr()
    with _on(device):
        _check(lib.head_rope_fwd(spec, *rows, *at, _current(device)), "head_rope_fwd")
    return tuple(outs)


def head_rope_grad(q, k, v, dq, dk, dv, positions=None, freqs=None, dims=None, layout="interleaved", norm=None,
                   q_weight=None, k_weight=None, q_bias=None, k_bias=None, eps: float = 1e-6, lens=None, out=None):
    """Gradients of head_rope for the same arguments: dq [B, H, S, d], dk and dv [B, Hkv, S, d] are those of its
    results. Returns (of q, of k, of v, of q_weight, of k_weight, of q_bias, of k_bias); the first three as
    [B, S, heads, d], parts of one [B, S, H + 2 Hkv, d] tensor, the gradient of a projection of everything, or
    written to `out`, three tensors of any strides that keep a head's values together. What was None, or has
    no weight or bias, is None; v's own values are not read, only its shape. It has no second derivative (and warns where
    autograd would have recorded one)."""
    spec, device, B, S, H, Hkv, d = _spec(q, k, v, positions, freqs, dims, layout, (q_weight, k_weight, q_bias, k_bias),
                                          norm, eps, lens)
    _unrecorded("head_rope_grad", "it has no second derivative", (dq, dk, dv), (q, k, v, q_weight, k_weight))
    rows, grads, to, outs = [None, None, None], [None, None, None], [None, None, None], out
    if out is None:
        # Rows of one new tensor: their places are known.
        heads = [n if t is not None else 0 for t, n in ((q, H), (k, Hkv), (v, Hkv))]
        n = sum(heads)
        one = torch.empty((B, S, n, d), dtype=torch.bfloat16, device=device)
        outs = one.split_with_sizes(heads, 2)
        place, token = one.data_ptr(), n * d
    outs = [y if t is not None else None for t, y in zip((q, k, v), outs)]
    for i, (t, g) in enumerate(((q, dq), (k, dk), (v, dv))):
        if (t is None) != (g is None):
            raise ValueError(f"{'qkv'[i]} and d{'qkv'[i]} go together")
        if t is None:
            continue
        n = Hkv if i else H
        rows[i] = _rows(t, "qkv"[i], B, S, n, d, device)
        _want(g, ("dq", "dk", "dv")[i], (B, n, S, d), torch.bfloat16, device)
        grads[i] = g.data_ptr()
        if out is None:
            to[i] = _PACKED_ROWS.pack(place, S * token, token, d)
            place += 2 * n * d
        else:
            to[i] = _rows(out[i], "out", B, S, n, d, device)
    sums, at = [None, None, None, None], [None, None, None, None]
    wanted = [i for i, w in enumerate((q_weight, k_weight, q_bias, k_bias))
              if w is not None and (k if i % 2 else q) is not None]
    if wanted:
        for i, w in zip(wanted, torch.empty((len(wanted), d), dtype=torch.float32, device=device).unbind()):
            sums[i], at[i] = w, w.data_ptr()
    n = 0 if norm is None else _grad_workspace(B, S, H, Hkv, d)
    with _on(device):
        workspace = _workspace(n, device)
        _check(lib.head_rope_bwd(spec, rows[0], rows[1], *grads, *to, *at, workspace.data_ptr() if n else None, n,
                                 _current(device)), "head_rope_bwd")
    return (*outs, *sums)
