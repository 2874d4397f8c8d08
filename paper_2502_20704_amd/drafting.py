"""The operators around drafting: the best continuations of beams, the states that follow them, and the pages of the 8-bit cache.

Argument marshalling only, as in operators.py: tensors are checked and handed to the C ABI (`include/fsd.h` has the definitions).

The outputs that a call of fsd_beam_select, fsd_cache_fork or fsd_cache_compact makes are parts of one tensor, with its workspace behind them where that is of 64 KB at
most: whoever keeps one of them keeps all of that.  A program that keeps the parents of every step, for tracing back, clones them or hands in tensors by `out`.
"""
from __future__ import annotations

import math

from . import binding
from .binding import FsdError, _ptr, _stream, _workspace, library
from .operators import _check, _new, _on_current, _torch

ROW_NO_BLOCKS = 64

_bytes = {}
_MOST_KEPT = 1000           # shapes: a program has a few; one that has more pays for them again


def _asked_once(call, *key):
    n = _bytes.get((call, key))
    if n is None:   # the library's answer for a shape does not change
        if len(_bytes) > _MOST_KEPT:
            _bytes.clear()
        fits = all(-0x80000000 <= size <= 0x7FFFFFFF for size in key)   # (another size would arrive there in its place)
        n = _bytes[call, key] = int(getattr(library(), call)(*key)) if fits else 0
    return n


def fsd_beam_workspace_bytes(B: int, beams: int, V: int, n: int, dtype: int) -> int:
    return _asked_once("fsd_beam_workspace_bytes", B, beams, V, n, dtype)


def fsd_cache_fork_workspace_bytes(num_blocks: int, n: int) -> int:
    return _asked_once("fsd_cache_fork_workspace_bytes", num_blocks, n)


def fsd_cache_compact_workspace_bytes(num_blocks: int) -> int:
    return _asked_once("fsd_cache_compact_workspace_bytes", num_blocks)


_layouts = {}
_WITH_OUTPUTS = 1 << 16     # bytes of a workspace that is made together with the outputs, and so lives as long as any of them


def _layout(space, tensors):
    """how `_parts` divides a tensor: each part's name, whether it is int32, shape, strides and begin; where the space begins; the words of all; whether
    a part is float32"""
    torch = _torch()
    parts, size = [], 0
    for name, (shape, dtype) in tensors.items():
        parts.append((name, dtype == torch.int32, shape, (shape[1], 1) if len(shape) == 2 else (1,), size))
        size += (math.prod(shape) + 15) // 16 * 16
    begin = (size * 4 + 255) // 256 * 256
    return parts, begin, (begin + space + 256 if space else size * 4) // 4 + 1, any(not part[1] for part in parts)


def _parts(stream, device, space, layout=None, **tensors):
    """New tensors of 32-bit numbers, of one or two dimensions, and `space` bytes behind them, as parts of one (a new tensor takes the host 1.7 us, a
    part of one 0.8): them, and where the space begins."""
    torch = _torch()
    parts, begin, words, any_float = layout or _layout(space, tensors)
    whole = torch.empty(words, dtype=torch.int32, device=device) if stream is None else _new(stream, device, whole=((words,), torch.int32))["whole"]
    floats = whole.view(torch.float32) if any_float else None
    at = whole.data_ptr() + begin
    return {name: torch.as_strided(whole if is_int else floats, shape, stride, offset) for name, is_int, shape, stride, offset in parts}, whole, at + -at % 256


def _results(call, sizes, specs, out, optional, workspace, need, device, stream):
    """the caller's outputs (those in `optional` may be missing) and workspace, checked, or new ones -> outputs, their addresses, workspace, its first address
    and size.  specs(*sizes): the outputs' shapes and types, in the order of the call's arguments (asked for once for a call's sizes: host time of forking one
    sequence's beams 19.0 -> 16.8 us, with `_want`)"""
    if out is None:
        space = need if workspace is None and need <= _WITH_OUTPUTS else 0
        layout = _layouts.get((call, space, sizes))
        if layout is None:
            if len(_layouts) > _MOST_KEPT:
                _layouts.clear()
            layout = _layouts[call, space, sizes] = _layout(space, specs(*sizes))
        out, whole, base = _parts(stream, device, space, layout)
        at = whole.data_ptr()
        addresses = [at + 4 * part[4] for part in layout[0]]
        if space:
            return out, addresses, whole, base, need
    else:
        tensors = specs(*sizes)
        _outputs(out, stream, device, optional, None, **tensors)
        addresses = [_ptr(out.get(name)) for name in tensors]
    if workspace is None:
        workspace = _new(stream, device, workspace=((need + 256,), _torch().uint8))["workspace"]
    elif not workspace.is_cuda or workspace.device != device or not workspace.is_contiguous() or workspace.dtype != _torch().uint8:
        raise ValueError(f"workspace: contiguous uint8 on {device} wanted")
    return out, addresses, *_workspace(workspace, 0, device)


def _outputs(given, stream, device, optional, new, /, **tensors):
    """the caller's outputs, checked, or new ones; optional: those that a caller may leave out"""
    if given is None:
        return new(stream, device, **tensors)
    for name, (shape, dtype) in tensors.items():
        if name not in optional or given.get(name) is not None:
            _check(given[name], name, shape, dtype, device)
    return given


def _want(t, name, shape, dtype, device):
    """(the usual case in one look; _check says what is wrong)"""
    if not (t.dtype == dtype and t.shape == shape and t.device == device and t.is_contiguous() and t.is_cuda):
        _check(t, name, shape, dtype, device)


def _counts(call, *sizes):
    """what the library takes as int: a larger one would arrive as another"""
    if max(sizes) > 0x7FFFFFFF:
        raise FsdError(-2, call)


def _row_stride(t, name):
    """elements between rows of [B, beams, V]: entries lie side by side, and the rows at one distance"""
    B, W, V = t.shape
    s = t.stride()
    step = s[1] if W > 1 else s[0] if B > 1 else V
    if V > 1 and s[2] != 1 or B > 1 and s[0] != W * step:
        raise ValueError(f"{name}: entries must lie side by side and rows at one distance from one another")
    return step


def _select_outputs(B, n):
    torch = _torch()
    return dict(scores=((B, n), torch.float32), parent=((B, n), torch.int32), tokens=((B, n), torch.int32), row_status=((B,), torch.int32))


def fsd_beam_select(logits, scores, n, *, weights=None, done=None, out=None, workspace=None, stream=None):
    """logits [B,beams,V] (rows at any one distance: the front of a padded vocabulary will do), scores float32 [B,beams] (None: 0),
    weights float32 and done int32 [B,beams] -> dict with scores float32, parent and tokens int32 [B,n], best first, and row_status (new ones: parts
    of one tensor, see above).  Masked entries are best -inf: a finite number costs up to 50 times the time where it leaves a row fewer than n."""
    torch = _torch()
    if logits.dim() != 3:
        raise ValueError("logits have 3 dimensions")
    if not logits.is_cuda:
        raise ValueError("logits must live on the GPU")
    B, W, V = logits.shape
    dt = binding._dtype_code(logits)
    dev = logits.device
    _on_current(dev, stream)
    step = _row_stride(logits, "logits")
    for name, t, dtype in (("scores", scores, torch.float32), ("weights", weights, torch.float32), ("done", done, torch.int32)):
        if t is not None:
            _want(t, name, (B, W), dtype, dev)
    _counts("fsd_beam_select", B, W, V, n)
    need = fsd_beam_workspace_bytes(B, W, V, n, dt)
    if need == 0:
        raise FsdError(-2, "fsd_beam_select")                 # (before tensors of such sizes are made)
    out, to, workspace, base, size = _results("fsd_beam_select", (B, n), _select_outputs, out, ("row_status",), workspace, need, dev, stream)
    st = library().fsd_beam_select(logits.data_ptr(), step, _ptr(scores), _ptr(weights), _ptr(done), B, W, V, dt, n, *to, base, size, _stream(stream))
    if st != 0:
        raise FsdError(st, "fsd_beam_select")
    out["_workspace"] = workspace
    return out


def fsd_beam_reorder(states, parent, *, batch_dim=0, out=None, stream=None):
    """states [..., B, beams, ...] of any type with B at batch_dim, parent int32 [B,n] -> dict with out [..., B, n, ...] (zeros where
    parent is -1) and row_status [B]."""
    torch = _torch()
    if not 0 <= batch_dim <= states.dim() - 2:
        raise ValueError("batch_dim names the sequences' dimension, with the beams' behind it")
    dev = states.device
    _check(states, "states")
    _on_current(dev, stream)
    if parent.dim() != 2:
        raise ValueError("parent has 2 dimensions")
    shape = tuple(states.shape)
    B, W = shape[batch_dim:batch_dim + 2]
    n = parent.shape[1]
    _counts("fsd_beam_reorder", *shape[:batch_dim + 2], math.prod(shape[:batch_dim]), n)
    _want(parent, "parent", (B, n), torch.int32, dev)
    out = _outputs(out, stream, dev, ("row_status",), _new, out=((*shape[:batch_dim + 1], n, *shape[batch_dim + 2:]), states.dtype),
                   row_status=((B,), torch.int32))
    st = library().fsd_beam_reorder(_ptr(states), _ptr(parent), math.prod(shape[:batch_dim]), B, W, n,
                                    math.prod(shape[batch_dim + 2:]) * states.element_size(), _ptr(out["out"]), _ptr(out.get("row_status")),
                                    _stream(stream))
    if st != 0:
        raise FsdError(st, "fsd_beam_reorder")
    return out


def _fork_outputs(n, M, P):
    i32 = _torch().int32
    return dict(block_table=((n, M), i32), cache_len=((n,), i32), refs=((P,), i32), free_blocks=((1,), i32), row_status=((n,), i32))


def fsd_cache_fork(cache, parent, refs, *, lengths=None, room=None, out=None, workspace=None, stream=None):
    """parent int32 [n] (rows of the cache's table; -1: none), refs int32 [num_blocks], lengths and room int32 [n] -> dict with block_table
    [n,max_blocks], cache_len [n], refs [num_blocks], free_blocks [1] and row_status [n].  `cache.with_tables(block_table, cache_len)`
    is the cache of the new sequences.  (New outputs: parts of one tensor, see above.)"""
    torch = _torch()
    dev = cache.device
    _on_current(dev, stream)
    if parent.dim() != 1:
        raise ValueError("parent has 1 dimension")
    n, P = parent.shape[0], cache.num_blocks
    _counts("fsd_cache_fork", n)
    _want(parent, "parent", (n,), torch.int32, dev)
    _want(refs, "refs", (P,), torch.int32, dev)
    for name, t in (("lengths", lengths), ("room", room)):
        if t is not None:
            _want(t, name, (n,), torch.int32, dev)
    out, to, workspace, base, size = _results("fsd_cache_fork", (n, cache.max_blocks, P), _fork_outputs, out, ("free_blocks", "row_status"), workspace,
                                              fsd_cache_fork_workspace_bytes(P, n), dev, stream)
    st = library().fsd_cache_fork(cache._ref, cache.batch, refs.data_ptr(), parent.data_ptr(), _ptr(lengths), _ptr(room), n, *to, base, size, _stream(stream))
    if st != 0:
        raise FsdError(st, "fsd_cache_fork")
    out["_workspace"] = workspace
    return out


def fsd_cache_copy(src, dst, src_blocks, dst_blocks, *, tokens=None, out=None, stream=None):
    """Blocks src_blocks int32 [n] of the cache src become blocks dst_blocks of dst (which may be src), their first tokens int32 [n] tokens
    (None: all) -> dict with page_status [n]."""
    torch = _torch()
    dev = src.device
    _on_current(dev, stream)
    if dst.device != dev:
        raise ValueError(f"the caches live on {dev} and {dst.device}")
    if (src.layers, src.kv_heads, src.head_dim) != (dst.layers, dst.kv_heads, dst.head_dim):
        raise ValueError("the caches differ in layers, kv_heads or head_dim")
    if src_blocks.dim() != 1:
        raise ValueError("src_blocks has 1 dimension")
    n = src_blocks.shape[0]
    _counts("fsd_cache_copy", n)
    for name, t in (("src_blocks", src_blocks), ("dst_blocks", dst_blocks), ("tokens", tokens)):
        if t is not None:
            _want(t, name, (n,), torch.int32, dev)
    out = _outputs(out, stream, dev, ("page_status",), _new, page_status=((n,), torch.int32))
    st = library().fsd_cache_copy(src._ref, dst._ref, _ptr(src_blocks), _ptr(dst_blocks), _ptr(tokens), n, _ptr(out.get("page_status")),
                                  _stream(stream))
    if st != 0:
        raise FsdError(st, "fsd_cache_copy")
    return out


def _compact_outputs(B, M, P):
    i32 = _torch().int32
    return dict(block_table=((B, M), i32), refs=((P,), i32), remap=((P,), i32), used_blocks=((1,), i32), row_status=((B,), i32))


def fsd_cache_compact(cache, refs, *, out=None, workspace=None, stream=None):
    """refs int32 [num_blocks] -> dict with block_table [B,max_blocks], refs and remap [num_blocks], used_blocks [1] and row_status [B].
    out=dict(block_table=cache.block_table, refs=refs) works in place.  (New outputs: parts of one tensor, see above.)"""
    torch = _torch()
    dev = cache.device
    _on_current(dev, stream)
    B, P = cache.batch, cache.num_blocks
    _want(refs, "refs", (P,), torch.int32, dev)
    out, to, workspace, base, size = _results("fsd_cache_compact", (B, cache.max_blocks, P), _compact_outputs, out, ("remap", "used_blocks", "row_status"), workspace,
                                              fsd_cache_compact_workspace_bytes(P), dev, stream)
    st = library().fsd_cache_compact(cache._ref, B, refs.data_ptr(), *to, base, size, _stream(stream))
    if st != 0:
        raise FsdError(st, "fsd_cache_compact")
    out["_workspace"] = workspace
    return out
