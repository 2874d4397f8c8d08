"""Refusals of the operators around a verify call: argument errors of the C ABI and of the binding, found before anything is
launched (no GPU needed)."""
import ctypes
import math

import pytest

import paper_2502_20704_amd as fsd
from paper_2502_20704_amd import operators as ops

A = 0x1000      # an address that is never dereferenced: every case below fails validation first


def _chain(**kw):
    c = ops._Conditions()
    a = dict(logits=A, tokens=A, B=2, K=4, rows=5, V=1000, dtype=fsd.F32, out=A, parent=None, tree=False)
    for k, v in kw.items():
        if k in a:
            a[k] = v
        else:
            setattr(c, k, v)
    L, ref = fsd.library(), ctypes.byref(c) if kw.get("conditions", True) else None
    if a["tree"]:
        return L.fsd_condition_tree(a["logits"], a["tokens"], a["parent"], a["B"], a["K"], a["rows"], a["V"], a["dtype"], ref, a["out"], None)
    return L.fsd_condition_chain(a["logits"], a["tokens"], a["B"], a["K"], a["rows"], a["V"], a["dtype"], ref, a["out"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), -1), (dict(out=None), -1), (dict(tokens=None), -1), (dict(conditions=None), -1),
    (dict(tree=True), -1), (dict(bias_count=3, bias_values=A), -1), (dict(bias_count=3, bias_tokens=A), -1),
    (dict(B=0), -2), (dict(B=65536), -2), (dict(K=-1, rows=0), -2), (dict(K=2049, rows=2049), -2), (dict(rows=3), -2), (dict(rows=6), -2),
    (dict(K=0, rows=0), -2), (dict(V=0), -2), (dict(V=524289), -2), (dict(B=60000, K=300, rows=300), -2),
    (dict(tree=True, parent=A, K=0, rows=1), -2), (dict(history_stride=-1), -2), (dict(bias_count=-1), -2),
    (dict(allowed=A, allowed_contexts=4), -2), (dict(allowed=A, allowed_contexts=0), -2),
    (dict(dtype=fsd.F16), -3), (dict(dtype=7), -3), (dict(logits=A + 2), -9), (dict(out=A + 1, dtype=fsd.BF16), -9),
])
def test_condition_refusals(kw, status):
    assert _chain(**kw) == status


def _cache(**kw):
    c = ops._Cache(A, A, A, A, A, 2 * A, 2, 10, 2, 128, 4)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


CACHE = [
    (dict(k_codes=None), -1), (dict(v_codes=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1), (dict(block_table=None), -1),
    (dict(cache_len=None), -1), (dict(layers=0), -2), (dict(num_blocks=0), -2), (dict(kv_heads=0), -2), (dict(head_dim=96), -2),
    (dict(max_blocks=0), -2), (dict(max_blocks=1 << 26), -2), (dict(k_codes=A + 8), -9), (dict(v_codes=A + 1), -9), (dict(k_scale=A + 2), -9),
]
ROTATION = [
    (ops._Rotation(A, 0, 64, 0), -2), (ops._Rotation(A, 9, 24, 0), -2), (ops._Rotation(A, 9, 0, 0), -2), (ops._Rotation(A, 9, 144, 0), -2),
    (ops._Rotation(A, 9, 64, 2), -6), (ops._Rotation(A + 4, 9, 64, 0), -9),
]


def _append(cache=None, rotation=None, **kw):
    a = dict(k=A, v=A, stride=256, B=2, R=9, dtype=fsd.BF16, accept=A, path=None, depth=0, len_out=A)
    a.update(kw)
    return fsd.library().fsd_cache_append(a["k"], a["v"], a["stride"], a["B"], a["R"], a["dtype"], a["accept"], a["path"], a["depth"],
                                          ctypes.byref(rotation) if rotation is not None else None, cache or _cache(), a["len_out"], None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(accept=None), -1), (dict(B=0), -2), (dict(R=0), -2), (dict(R=(1 << 20) + 1), -2),
    (dict(path=A, depth=0), -2), (dict(path=A, depth=2049), -2), (dict(dtype=3), -3), (dict(stride=248), -9), (dict(stride=260), -9),
    (dict(k=A + 8), -9), (dict(v=A + 2), -9), (dict(len_out=2 * A), -9), (dict(B=65535, R=1 << 20), -2),
])
def test_append_refusals(kw, status):
    assert _append(**kw) == status


def _attend(cache=None, rotation=None, **kw):
    a = dict(q=A, k=A, v=A, q_stride=8 * 128, kv_stride=256, B=2, R=9, heads=8, dtype=fsd.BF16, scale=0.1, layer=1, out=A, ws=A, bytes=1 << 40,
             tree=False, parent=None)
    a.update(kw)
    L, rot = fsd.library(), ctypes.byref(rotation) if rotation is not None else None
    if a["tree"]:
        return L.fsd_attend_tree(a["q"], a["k"], a["v"], a["q_stride"], a["kv_stride"], a["parent"], a["B"], a["R"], a["heads"], a["dtype"], None,
                                 a["scale"], rot, cache or _cache(), a["layer"], a["out"], None, a["ws"], a["bytes"], None)
    return L.fsd_attend_chain(a["q"], a["k"], a["v"], a["q_stride"], a["kv_stride"], a["B"], a["R"], a["heads"], a["dtype"], None, a["scale"],
                              rot, cache or _cache(), a["layer"], a["out"], None, a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(out=None), -1), (dict(tree=True), -1),
    (dict(B=0), -2), (dict(B=65536), -2), (dict(R=0), -2), (dict(R=2050), -2), (dict(B=60000, R=300), -2), (dict(heads=7), -2), (dict(heads=1), -2),
    (dict(heads=130, q_stride=130 * 128), -2), (dict(layer=-1), -2), (dict(layer=2), -2), (dict(scale=math.inf), -2), (dict(scale=math.nan), -2),
    (dict(dtype=fsd.F32), -3), (dict(dtype=5), -3), (dict(q_stride=1016), -9), (dict(q_stride=1028), -9), (dict(kv_stride=255), -9),
    (dict(q=A + 8), -9), (dict(out=A + 4), -9), (dict(ws=None), -5), (dict(ws=A + 16), -5), (dict(bytes=1000), -5),
])
def test_attend_refusals(kw, status):
    assert _attend(**kw) == status


@pytest.mark.parametrize("kw,status", CACHE)
def test_cache_refusals(kw, status):
    assert _append(cache=_cache(**kw)) == status
    assert _attend(cache=_cache(**kw)) == status


@pytest.mark.parametrize("rotation,status", ROTATION)
def test_rotation_refusals(rotation, status):
    assert _append(rotation=rotation) == status
    assert _attend(rotation=rotation) == status


def test_limits_of_a_launch():
    """Calls whose grids or counts would not fit: refused before anything is launched."""
    assert _append(cache=_cache(layers=65536)) == -2
    assert _append(cache=_cache(layers=1 << 22), R=17) == -2
    assert _attend(scale=3.0e38) == -2
    assert _attend(cache=_cache(kv_heads=128, max_blocks=1 << 24), heads=128, q_stride=128 * 128, kv_stride=128 * 128) == -2


def test_workspace_planning():
    f = fsd.fsd_attend_workspace_bytes
    assert f(1, 1, 1, 1, 64) > 0 and f(64, 9, 32, 8, 128) % 256 == 0
    assert f(3, 2049, 64, 1, 256) > 0
    assert f(0, 1, 1, 1, 64) == 0 and f(1, 2050, 1, 1, 64) == 0 and f(1, 1, 3, 2, 64) == 0 and f(1, 1, 1, 1, 80) == 0


def test_status_string():
    L = fsd.library()
    assert L.fsd_status_string(-9) not in (L.fsd_status_string(-8), L.fsd_status_string(-100))


def test_binding_refuses_host_tensors():
    import torch

    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        fsd.fsd_condition_chain(torch.zeros(1, 1, 8), None, fsd.Conditions())
    with pytest.raises(ValueError):
        fsd.Conditions(history=torch.zeros((1, 4), dtype=torch.int32))
    with pytest.raises(ValueError):
        fsd.Conditions(history_len=i)
    with pytest.raises(ValueError):
        fsd.Cache.empty(1, 1, 1, 64, torch.zeros((1, 1), dtype=torch.int32), i)
    with pytest.raises(ValueError):
        fsd.Rotation(torch.zeros(4, 64))


def test_distance_between_tokens():
    """What the binding takes for one distance between tokens, and what it refuses."""
    import types

    import torch

    def step(t, lead):
        fake = types.SimpleNamespace(is_cuda=True, device="d", shape=t.shape, dtype=t.dtype, stride=t.stride)
        return ops._token_stride(fake, "k", lead, t.dtype, "d")

    whole = torch.zeros(3, 2, 5, 6, 64)
    assert step(whole, (3, 2, 5, 6, 64)) == 6 * 64
    assert step(whole[..., 1:3, :], (3, 2, 5, 2, 64)) == 6 * 64
    assert step(whole[:1, :, :, :4], (1, 2, 5, 4, 64)) == 6 * 64
    assert step(torch.zeros(1, 1, 1, 4, 64), (1, 1, 1, 4, 64)) == 256
    assert step(torch.zeros(2, 1, 1, 4, 64)[:, :, :, :2], (2, 1, 1, 2, 64)) == 256      # layers at that distance
    with pytest.raises(ValueError):
        step(whole[:, :, :3], (3, 2, 3, 6, 64))                  # sequences further apart than their tokens
    with pytest.raises(ValueError):
        step(whole[..., :32], (3, 2, 5, 6, 32))
    with pytest.raises(ValueError):
        step(whole.transpose(0, 1), (2, 3, 5, 6, 64))
    with pytest.raises(ValueError):
        step(whole, (3, 2, 5, 6, 128))


@pytest.mark.parametrize("at,size", [(1, 1), (16, 100), (1, 254)])
def test_workspace_that_ends_before_the_first_aligned_address(at, size):
    """A view that holds no aligned address has room for nothing, not for 2^64 bytes."""
    import torch

    from paper_2502_20704_amd import binding

    arena = torch.zeros(1024, dtype=torch.uint8)
    at += (-arena.data_ptr()) % 256
    assert binding._workspace(arena[at:at + size], 0, arena.device)[2] == 0
    assert ops._workspace is binding._workspace


def test_reports_that_lie_in_what_a_call_reads():
    """cache_len_out and row_status, byte by byte beside and inside every array that other workgroups read, and one another."""
    B, blocks, depth = 2, 4, 3
    at = dict(cache_len=0x10000, block_table=0x20000, accept_len=0x30000, path_nodes=0x40000, parent=0x50000, row_count=0x60000)
    size = dict(cache_len=4 * B, block_table=4 * B * blocks, accept_len=4 * B, path_nodes=4 * B * depth, parent=4 * B * 8, row_count=4 * B)
    cache = _cache(cache_len=at["cache_len"], block_table=at["block_table"])
    L = fsd.library()

    def append(length, status):
        return L.fsd_cache_append(A, A, 256, B, 9, fsd.BF16, at["accept_len"], at["path_nodes"], depth, None, cache, length, status, None)

    def attend(status):
        return L.fsd_attend_tree(A, A, A, 8 * 128, 256, at["parent"], B, 9, 8, fsd.BF16, at["row_count"], 0.1, None, cache, 0, A, status, A, 1 << 40, None)

    for name in ("cache_len", "block_table", "accept_len", "path_nodes"):
        for where in (at[name], at[name] - 4, at[name] + size[name] - 4):
            assert append(where, None) == -9 and append(None, where) == -9, (name, where)
    for where in (0x70000, 0x70004, 0x6fffc):
        assert append(0x70000, where) == -9
    for name in ("cache_len", "block_table", "parent", "row_count"):
        for where in (at[name], at[name] - 4, at[name] + size[name] - 4):
            assert attend(where) == -9, (name, where)


@pytest.mark.parametrize("dtype,step", [(fsd.F32, 4), (fsd.BF16, 2)])
def test_conditioned_logits_that_overlap_the_logits_by_a_part(dtype, step):
    """In place is one address for both; rows that another workgroup writes before this one reads them are not."""
    size, at = 2 * 5 * 1000 * step, 1 << 20
    for tree in (False, True):
        for out in (at + step, at - step, at + size - step, at - size + step):
            assert _chain(logits=at, out=out, dtype=dtype, tree=tree, parent=A) == -9


def test_streams_of_another_device(monkeypatch):
    import types

    import torch

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    here, there = torch.device("cuda", 0), torch.device("cuda", 1)
    ops._on_current(here, None)
    ops._on_current(here, types.SimpleNamespace(device=here))
    for device, stream in ((there, None), (here, types.SimpleNamespace(device=there))):
        with pytest.raises(ValueError):
            ops._on_current(device, stream)
