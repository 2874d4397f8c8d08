"""The operators around a verify call: conditioning of logits, attention over an 8-bit paged cache, and appending to it.

Argument marshalling only, as in binding.py: tensors are checked and handed to the C ABI (`include/fsd.h` has the
definitions).  What a program keeps from step to step is an object here (`Conditions`, `Cache`, `Rotation`): its tensors are
checked once, when it is made, and are read at every call, so their contents may change between calls and their memory may not.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import FsdError, _ptr, _stream, _workspace, library

F16 = 2
CACHE_BLOCK = 64
CACHE_GROUP = 16
ROPE_HALVES, ROPE_PAIRS = 0, 1
ROW_BAD_CACHE = 32

_vp, _i = ctypes.c_void_p, ctypes.c_int


class _Conditions(ctypes.Structure):
    _fields_ = [("history", _vp), ("history_len", _vp), ("prompt_len", _vp), ("history_stride", _i), ("bias_count", _i),
                ("bias_tokens", _vp), ("bias_values", _vp), ("repetition", _vp), ("presence", _vp), ("frequency", _vp),
                ("allowed", _vp), ("allowed_contexts", _i)]


class _Cache(ctypes.Structure):
    _fields_ = [("k_codes", _vp), ("v_codes", _vp), ("k_scale", _vp), ("v_scale", _vp), ("block_table", _vp), ("cache_len", _vp),
                ("layers", _i), ("num_blocks", _i), ("kv_heads", _i), ("head_dim", _i), ("max_blocks", _i)]


class _Rotation(ctypes.Structure):
    _fields_ = [("table", _vp), ("rows", _i), ("dim", _i), ("style", _i)]


def _torch():
    if binding.torch is None:
        binding._use_torch()
    return binding.torch


def _check(t, name, shape=None, dtype=None, device=None):
    binding._check(t, name, shape, dtype)
    if device is not None and t.device != device:
        raise ValueError(f"{name} lives on {t.device}, the others on {device}")


def _on_current(device, stream):
    if device.index != _torch().cuda.current_device():
        raise ValueError(f"the tensors live on {device}, which is not the current device")
    if stream is not None and stream.device != device:
        raise ValueError(f"the stream is one of {stream.device}, the tensors live on {device}")


def _new(stream, device, **tensors):
    """Tensors (shape, dtype) that a call of `stream` writes, out of that stream's memory: what the current stream has given back may be in use there
    still.  Nor are they given out again before the current stream, whose program has them, is done with them."""
    torch = _torch()
    if stream is None:
        return {n: torch.empty(shape, dtype=dtype, device=device) for n, (shape, dtype) in tensors.items()}
    with torch.cuda.stream(stream):
        out = {n: torch.empty(shape, dtype=dtype, device=device) for n, (shape, dtype) in tensors.items()}
    for t in out.values():
        t.record_stream(torch.cuda.current_stream())
    return out


class Conditions:
    """Penalties, biases and grammar masks of a batch (fsd_conditions).  All of them are optional.

    history int32 [B, n] token ids; history_len, prompt_len int32 [B]; repetition, presence, frequency float32 [B];
    bias_tokens int32 / bias_values float32 [B, m]; allowed int32 [B, 1 or contexts, ceil(V / 32)] bit masks."""

    def __init__(self, *, history=None, history_len=None, prompt_len=None, repetition=None, presence=None, frequency=None,
                 bias_tokens=None, bias_values=None, allowed=None):
        torch = _torch()
        given = [t for t in (history, history_len, prompt_len, repetition, presence, frequency, bias_tokens, bias_values, allowed)
                 if t is not None]
        self.batch, self.device = (given[0].shape[0], given[0].device) if given else (None, None)
        B, dev = self.batch, self.device
        for name, t, dtype in (("history_len", history_len, torch.int32), ("prompt_len", prompt_len, torch.int32),
                               ("repetition", repetition, torch.float32), ("presence", presence, torch.float32),
                               ("frequency", frequency, torch.float32)):
            if t is not None:
                _check(t, name, (B,), dtype, dev)
        if (history_len is not None or prompt_len is not None) and history is None:
            raise ValueError("history_len and prompt_len need a history")
        if (bias_tokens is None) != (bias_values is None):
            raise ValueError("bias_tokens and bias_values come together")
        for name, t, dtype, dims in (("history", history, torch.int32, 2), ("bias_tokens", bias_tokens, torch.int32, 2),
                                     ("bias_values", bias_values, torch.float32, 2), ("allowed", allowed, torch.int32, 3)):
            if t is not None:
                if t.dim() != dims:
                    raise ValueError(f"{name} has {t.dim()} dimensions, expected {dims}")
                _check(t, name, (B, *t.shape[1:]), dtype, dev)
        if bias_tokens is not None and bias_tokens.shape != bias_values.shape:
            raise ValueError("bias_tokens and bias_values differ in shape")
        if allowed is not None and allowed.shape[1] == 0:
            raise ValueError("allowed has no context")       # (and no memory: it would count as absent)
        self._held = given
        self.words = allowed.shape[2] if allowed is not None else None
        self.contexts = allowed.shape[1] if allowed is not None else 0
        self._c = _Conditions(_ptr(history), _ptr(history_len), _ptr(prompt_len), history.shape[1] if history is not None else 0,
                              bias_tokens.shape[1] if bias_tokens is not None else 0, _ptr(bias_tokens), _ptr(bias_values),
                              _ptr(repetition), _ptr(presence), _ptr(frequency), _ptr(allowed), self.contexts)
        self._ref = ctypes.byref(self._c)

    def _fits(self, B, V, device, contexts):
        if self.batch is not None and (self.batch != B or self.device != device):
            raise ValueError(f"the conditions are those of {self.batch} sequences on {self.device}, the logits have {B} on {device}")
        if self.words is not None and self.words != (V + 31) // 32:
            raise ValueError(f"allowed has {self.words} words a row, {(V + 31) // 32} hold {V} entries")
        if self.contexts not in (0, 1, contexts):
            raise ValueError(f"allowed has {self.contexts} contexts, expected 1 or {contexts}")


class Cache:
    """The 8-bit paged cache (fsd_cache): uint8 codes, float32 scales, the block table and the lengths of a batch.

    k_codes uint8 [layers, num_blocks, kv_heads, 64, head_dim], v_codes uint8 [layers, num_blocks, kv_heads, 4, head_dim, 16],
    k_scale / v_scale float32 [layers, num_blocks, kv_heads], block_table int32 [B, max_blocks], cache_len int32 [B]."""

    def __init__(self, k_codes, v_codes, k_scale, v_scale, block_table, cache_len):
        torch = _torch()
        if k_codes.dim() != 5 or block_table.dim() != 2:
            raise ValueError("k_codes has 5 dimensions and block_table 2")
        L, P, H, T, D = k_codes.shape
        B, M = block_table.shape
        dev = k_codes.device
        _check(k_codes, "k_codes", (L, P, H, CACHE_BLOCK, D), torch.uint8)
        _check(v_codes, "v_codes", (L, P, H, CACHE_BLOCK // CACHE_GROUP, D, CACHE_GROUP), torch.uint8, dev)
        _check(k_scale, "k_scale", (L, P, H), torch.float32, dev)
        _check(v_scale, "v_scale", (L, P, H), torch.float32, dev)
        _check(block_table, "block_table", (B, M), torch.int32, dev)
        _check(cache_len, "cache_len", (B,), torch.int32, dev)
        self.k_codes, self.v_codes, self.k_scale, self.v_scale = k_codes, v_codes, k_scale, v_scale
        self.block_table, self.cache_len = block_table, cache_len
        self.layers, self.num_blocks, self.kv_heads, self.head_dim = L, P, H, D
        self.batch, self.max_blocks, self.device = B, M, dev
        self._c = _Cache(_ptr(k_codes), _ptr(v_codes), _ptr(k_scale), _ptr(v_scale), _ptr(block_table), _ptr(cache_len),
                         L, P, H, D, M)
        self._ref = ctypes.byref(self._c)

    def with_tables(self, block_table, cache_len):
        """The same codes and scales under other tables and lengths (those that fsd_cache_fork gives)."""
        return Cache(self.k_codes, self.v_codes, self.k_scale, self.v_scale, block_table, cache_len)

    @classmethod
    def empty(cls, layers, num_blocks, kv_heads, head_dim, block_table, cache_len):
        """A cache without contents on the device of block_table; scales start at 1."""
        torch = _torch()
        dev = block_table.device
        shape = (layers, num_blocks, kv_heads)
        return cls(torch.zeros((*shape, CACHE_BLOCK, head_dim), dtype=torch.uint8, device=dev),
                   torch.zeros((*shape, CACHE_BLOCK // CACHE_GROUP, head_dim, CACHE_GROUP), dtype=torch.uint8, device=dev),
                   torch.ones(shape, dtype=torch.float32, device=dev), torch.ones(shape, dtype=torch.float32, device=dev),
                   block_table, cache_len)


class Rotation:
    """Rotation by position (fsd_rotation): table float32 [rows, dim], dim/2 cosines and dim/2 sines of every position."""

    def __init__(self, table, style=ROPE_HALVES):
        if table.dim() != 2:
            raise ValueError("table has 2 dimensions")
        _check(table, "table", None, _torch().float32)
        self.table, self.style, self.device = table, style, table.device
        self._c = _Rotation(_ptr(table), table.shape[0], table.shape[1], style)
        self._ref = ctypes.byref(self._c)


def _condition(call, logits, tokens, parent, conditions, out, stream):
    torch = _torch()
    if logits.dim() != 3:
        raise ValueError("logits have 3 dimensions")
    B, rows, V = logits.shape
    dt = binding._dtype_code(logits)
    dev = logits.device
    _check(logits, "logits")
    _on_current(dev, stream)
    n = 0
    if tokens is not None:
        n = tokens.shape[-1]
        _check(tokens, "tokens", (B, n), torch.int32, dev)
    if rows not in (n, n + 1):
        raise ValueError(f"{rows} rows of logits go with {rows - 1} or {rows} candidates, got {n}")
    if parent is not None:
        _check(parent, "parent", (B, n), torch.int32, dev)
    conditions._fits(B, V, dev, n + 1)
    if out is None:
        out = _new(stream, dev, out=(logits.shape, logits.dtype))
    else:
        _check(out["out"], "out", logits.shape, logits.dtype, dev)
    L = library()
    if call == "fsd_condition_tree":
        st = L.fsd_condition_tree(_ptr(logits), _ptr(tokens), _ptr(parent), B, n, rows, V, dt, conditions._ref, _ptr(out["out"]),
                                  _stream(stream))
    else:
        st = L.fsd_condition_chain(_ptr(logits), _ptr(tokens), B, n, rows, V, dt, conditions._ref, _ptr(out["out"]), _stream(stream))
    if st != 0:
        raise FsdError(st, call)
    return out


def fsd_condition_chain(logits, cand, conditions, *, out=None, stream=None):
    """logits [B,K+1,V] (target rows) or [B,K,V] (draft rows), cand int32 [B,K] (None: no candidates, one row) -> dict with
    out, the conditioned logits.  out=dict(out=logits) works in place."""
    return _condition("fsd_condition_chain", logits, cand, None, conditions, out, stream)


def fsd_condition_tree(logits, node_tokens, parent, conditions, *, out=None, stream=None):
    """logits [B,N+1,V] (target rows) or [B,N,V] (draft rows), node_tokens / parent int32 [B,N] -> dict with out."""
    return _condition("fsd_condition_tree", logits, node_tokens, parent, conditions, out, stream)


_codes = {}


def _dtype_code(t, floats):
    if not _codes:
        torch = _torch()
        _codes.update({torch.float32: binding.F32, torch.bfloat16: binding.BF16, torch.float16: F16})
    code = _codes.get(t.dtype)
    if code is None or (code == binding.F32 and not floats):
        raise TypeError(f"{'float32, ' if floats else ''}bfloat16 or float16 wanted, got {t.dtype}")
    return code


def _token_stride(t, name, shape, dtype, device):
    """Elements between tokens of [..., B, R, heads, head_dim]: heads lie side by side, and the tokens at one distance."""
    if t.device != device:                   # (the others': a GPU)
        raise ValueError(f"{name} lives on {t.device}, the others on {device}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    stride = t.stride()
    if shape[-1] > 1 and stride[-1] != 1 or shape[-2] > 1 and stride[-2] != shape[-1]:
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    step, run = None, 1                      # run: tokens that the dimensions behind the current one hold
    for i in range(len(shape) - 3, -1, -1):
        n = shape[i]
        if n > 1:
            if step is None:
                step = stride[i] // run
            if stride[i] != step * run:
                raise ValueError(f"{name}: tokens must lie at one distance from one another")
            run *= n
    return step if step is not None else shape[-1] * shape[-2]


def _laid_out_alike(a, b):
    return a.stride() == b.stride() and a.shape == b.shape and a.dtype == b.dtype and a.device == b.device


def fsd_cache_append(k, v, cache, accept_len, *, path_nodes=None, rotation=None, out=None, stream=None):
    """k, v [B,R,kv_heads,head_dim] or [layers,B,R,kv_heads,head_dim] (tokens at any one distance), accept_len int32 [B] and
    path_nodes int32 [B,max_depth] as a verify call gives them -> dict with cache_len (the new lengths, to be
    copied into the cache's own once no call reads those) and row_status."""
    torch = _torch()
    dt = _dtype_code(k, True)
    dev = cache.device
    _on_current(dev, stream)
    if k.dim() not in (4, 5):
        raise ValueError("k has 4 or 5 dimensions")
    B, R = k.shape[-4:-2]
    shape = (cache.batch, R, cache.kv_heads, cache.head_dim)
    if k.dim() == 5 or cache.layers != 1:
        shape = (cache.layers, *shape)
    step = _token_stride(k, "k", shape, k.dtype, dev)
    if not _laid_out_alike(v, k) and _token_stride(v, "v", shape, k.dtype, dev) != step:
        raise ValueError("k and v differ in the distance between tokens")
    _check(accept_len, "accept_len", (B,), torch.int32, dev)
    depth = 0
    if path_nodes is not None:
        depth = path_nodes.shape[-1]
        _check(path_nodes, "path_nodes", (B, depth), torch.int32, dev)
    if rotation is not None and rotation.device != dev:
        raise ValueError(f"the rotation lives on {rotation.device}, the cache on {dev}")
    if out is None:
        out = _new(stream, dev, cache_len=((B,), torch.int32), row_status=((B,), torch.int32))
    for name in ("cache_len", "row_status"):
        if out.get(name) is not None:
            _check(out[name], name, (B,), torch.int32, dev)
    st = library().fsd_cache_append(_ptr(k), _ptr(v), step, B, R, dt, _ptr(accept_len), _ptr(path_nodes), depth,
                                    rotation._ref if rotation is not None else None, cache._ref, _ptr(out.get("cache_len")),
                                    _ptr(out.get("row_status")), _stream(stream))
    if st != 0:
        raise FsdError(st, "fsd_cache_append")
    return out


_attend_bytes = {}


def fsd_attend_workspace_bytes(B: int, R: int, heads: int, kv_heads: int, head_dim: int) -> int:
    key = (B, R, heads, kv_heads, head_dim)
    n = _attend_bytes.get(key)
    if n is None:   # the library's answer for a shape does not change: asked once
        n = _attend_bytes[key] = int(library().fsd_attend_workspace_bytes(*key))
    return n


def _attend(call, q, k, v, parent, cache, layer, row_count, rotation, scale, out, workspace, stream):
    torch = _torch()
    dt = _dtype_code(q, False)
    dev = cache.device
    _on_current(dev, stream)
    if q.dim() != 4:
        raise ValueError("q has 4 dimensions")
    B, R, heads, D = q.shape
    q_step = _token_stride(q, "q", (cache.batch, R, heads, cache.head_dim), q.dtype, dev)
    shape = (B, R, cache.kv_heads, D)
    kv_step = _token_stride(k, "k", shape, q.dtype, dev)
    if not _laid_out_alike(v, k) and _token_stride(v, "v", shape, q.dtype, dev) != kv_step:
        raise ValueError("k and v differ in the distance between tokens")
    if parent is not None:
        _check(parent, "parent", (B, R - 1), torch.int32, dev)
    if row_count is not None:
        _check(row_count, "row_count", (B,), torch.int32, dev)
    if rotation is not None and rotation.device != dev:
        raise ValueError(f"the rotation lives on {rotation.device}, the cache on {dev}")
    if out is None:
        out = _new(stream, dev, out=((B, R, heads, D), q.dtype), row_status=((B,), torch.int32))
    else:
        _check(out["out"], "out", q.shape, q.dtype, dev)
        if out.get("row_status") is not None:
            _check(out["row_status"], "row_status", (B,), torch.int32, dev)
    if workspace is None:
        need = fsd_attend_workspace_bytes(B, R, heads, cache.kv_heads, D) + 256
        workspace = _new(stream, dev, workspace=((need,), torch.uint8))["workspace"]
    elif not workspace.is_cuda or workspace.device != dev or not workspace.is_contiguous() or workspace.dtype != torch.uint8:
        raise ValueError(f"workspace: contiguous uint8 on {dev} wanted")
    workspace, base, size = _workspace(workspace, 0, dev)
    scale = D ** -0.5 if scale is None else float(scale)
    rot = rotation._ref if rotation is not None else None
    L = library()
    if call == "fsd_attend_tree":
        st = L.fsd_attend_tree(_ptr(q), _ptr(k), _ptr(v), q_step, kv_step, _ptr(parent), B, R, heads, dt, _ptr(row_count), scale, rot,
                               cache._ref, layer, _ptr(out["out"]), _ptr(out.get("row_status")), base, size,
                               _stream(stream))
    else:
        st = L.fsd_attend_chain(_ptr(q), _ptr(k), _ptr(v), q_step, kv_step, B, R, heads, dt, _ptr(row_count), scale, rot, cache._ref,
                                layer, _ptr(out["out"]), _ptr(out.get("row_status")), base, size, _stream(stream))
    if st != 0:
        raise FsdError(st, call)
    out["_workspace"] = workspace
    return out


def fsd_attend_chain(q, k, v, cache, *, layer=0, row_count=None, rotation=None, scale=None, out=None, workspace=None, stream=None):
    """q [B,R,heads,head_dim], k, v [B,R,kv_heads,head_dim] (tokens at any one distance: parts of one projection's output will
    do) of the token emitted last and the candidates behind it -> dict with out [B,R,heads,head_dim] and row_status.
    scale: 1 / sqrt(head_dim) unless given."""
    return _attend("fsd_attend_chain", q, k, v, None, cache, layer, row_count, rotation, scale, out, workspace, stream)


def fsd_attend_tree(q, k, v, parent, cache, *, layer=0, row_count=None, rotation=None, scale=None, out=None, workspace=None, stream=None):
    """fsd_attend_chain over a token tree: R = N+1 rows, parent int32 [B,N]."""
    return _attend("fsd_attend_tree", q, k, v, parent, cache, layer, row_count, rotation, scale, out, workspace, stream)
