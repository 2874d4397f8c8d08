"""Refusals of the operators around drafting: argument errors of the C ABI and of the binding, found before anything is launched (no
GPU needed)."""
import ctypes
import types

import pytest

import paper_2502_20704_amd as fsd
from paper_2502_20704_amd import drafting
from paper_2502_20704_amd import operators as ops

A = 1 << 32     # addresses that are never dereferenced: every case below fails validation first.  Each argument has 2^32 bytes of its own
LOGITS, SCORES, WEIGHTS, DONE, OUT, PARENT, TOKENS, STATUS, SPACE = (A * (k + 1) for k in range(9))
GB = 1 << 30


def _select(**kw):
    a = dict(logits=LOGITS, stride=1000, scores=SCORES, weights=WEIGHTS, done=DONE, B=2, W=4, V=1000, dtype=fsd.BF16, n=8, out=OUT, parent=PARENT,
             tokens=TOKENS, status=STATUS, ws=SPACE, bytes=GB)
    a.update(kw)
    return fsd.library().fsd_beam_select(a["logits"], a["stride"], a["scores"], a["weights"], a["done"], a["B"], a["W"], a["V"], a["dtype"], a["n"], a["out"],
                                         a["parent"], a["tokens"], a["status"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), -1), (dict(out=None), -1), (dict(parent=None), -1), (dict(tokens=None), -1),
    (dict(B=0), -2), (dict(B=65536), -2), (dict(W=0), -2), (dict(W=257), -2), (dict(n=0), -2), (dict(n=129), -2), (dict(V=0), -2), (dict(V=524289, stride=524289), -2),
    (dict(dtype=fsd.F16), -3), (dict(dtype=9), -3),
    (dict(stride=999), -9), (dict(stride=(1 << 32) + 1), -9), (dict(logits=LOGITS + 1), -9), (dict(logits=LOGITS + 2, dtype=fsd.F32), -9), (dict(scores=SCORES + 2), -9),
    (dict(weights=WEIGHTS + 1), -9), (dict(done=DONE + 2), -9), (dict(out=OUT + 2), -9), (dict(parent=PARENT + 1), -9), (dict(tokens=TOKENS + 3), -9), (dict(status=STATUS + 2), -9),
    (dict(ws=None), -5), (dict(ws=SPACE + 16), -5), (dict(bytes=100), -5),
])
def test_select_refusals(kw, status):
    assert _select(**kw) == status


def test_select_outputs_that_lie_in_what_it_reads():
    lists = dict(scores=SCORES, weights=WEIGHTS, done=DONE)
    for name in ("out", "parent", "tokens"):
        for at in lists.values():
            for where in (at, at - 60, at + 28):
                assert _select(**{name: where}) == -9, (name, where)
        for where in (LOGITS, LOGITS + 8 * 2000 - 4, SPACE, SPACE + 700, STATUS, STATUS + 4):
            assert _select(**{name: where}) == -9, (name, where)
    assert _select(out=PARENT + 60) == -9 and _select(tokens=PARENT - 60) == -9 and _select(status=TOKENS + 60) == -9
    need = fsd.fsd_beam_workspace_bytes(2, 4, 1000, 8, fsd.BF16)
    assert _select(ws=LOGITS + 15872) == -9 and _select(logits=SPACE + need - 2) == -9
    # the last row's end, not a whole stride's
    assert _select(stride=1 << 20, out=LOGITS + 7 * (1 << 21) + 1996) == -9 and _select(stride=1 << 20, out=LOGITS + 7 * (1 << 21) + 2000, parent=None) == -1


def test_workspace_sizes():
    assert fsd.fsd_beam_workspace_bytes(1, 1, 1, 1, fsd.F32) > 0 and fsd.fsd_beam_workspace_bytes(64, 8, 128256, 16, fsd.BF16) > 0
    for bad in ((0, 1, 1, 1, 0), (1, 257, 1, 1, 0), (1, 1, 0, 1, 0), (1, 1, 1, 129, 0), (1, 1, 1, 1, 2), (1, 1, 524289, 1, 1), (65536, 1, 1, 1, 1)):
        assert fsd.fsd_beam_workspace_bytes(*bad) == 0
    for B in (1, 3, 17, 64, 500, 65535):
        for W in (1, 2, 8, 100, 256):
            for V in (1, 7, 2049, 32000, 128257, 524288):
                for dtype in (fsd.F32, fsd.BF16):
                    n = fsd.fsd_beam_workspace_bytes(B, W, V, 128, dtype)
                    assert n > 0 and n % 256 == 0
                    for smaller in ((max(1, B // 2), W, V, 128), (B, max(1, W - 1), V, 128), (B, W, max(1, V - 1000), 128), (B, W, V // 2 + 1, 100)):
                        assert fsd.fsd_beam_workspace_bytes(*smaller, dtype) <= n
    assert fsd.fsd_cache_fork_workspace_bytes(1, 1) > 0 and fsd.fsd_cache_fork_workspace_bytes(1 << 24, 65535) > 0
    assert fsd.fsd_cache_fork_workspace_bytes(0, 1) == fsd.fsd_cache_fork_workspace_bytes(5, 0) == fsd.fsd_cache_fork_workspace_bytes((1 << 24) + 1, 1) == 0
    assert fsd.fsd_cache_fork_workspace_bytes(5, 65536) == fsd.fsd_cache_compact_workspace_bytes(0) == fsd.fsd_cache_compact_workspace_bytes((1 << 24) + 1) == 0


def _reorder(**kw):
    a = dict(states=LOGITS, parent=PARENT, layers=2, B=3, W=4, n=5, row=100, out=OUT, status=STATUS)
    a.update(kw)
    return fsd.library().fsd_beam_reorder(a["states"], a["parent"], a["layers"], a["B"], a["W"], a["n"], a["row"], a["out"], a["status"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(states=None), -1), (dict(parent=None), -1), (dict(out=None), -1), (dict(layers=0), -2), (dict(layers=65536), -2), (dict(B=0), -2), (dict(B=65536), -2),
    (dict(W=0), -2), (dict(W=65536), -2), (dict(n=0), -2), (dict(n=65536), -2), (dict(row=0), -2), (dict(row=(1 << 40) + 1), -2), (dict(layers=60000, B=60000), -2),
    (dict(layers=30000, B=60000, row=1 << 40), -2), (dict(parent=PARENT + 2), -9), (dict(status=STATUS + 1), -9),
    (dict(out=LOGITS), -9), (dict(out=LOGITS + 2399), -9), (dict(out=LOGITS - 2999), -9), (dict(out=PARENT + 59), -9), (dict(status=PARENT + 56), -9),
    (dict(status=LOGITS + 2396), -9), (dict(status=OUT + 2996), -9),
])
def test_reorder_refusals(kw, status):
    assert _reorder(**kw) == status


KC, VC, KS, VS, TABLE, LENS, REFS, KEEP, ROOM, TABLE_OUT, LEN_OUT, REFS_OUT, FREE = (A * (k + 20) for k in range(13))


def _cache(**kw):
    c = ops._Cache(KC, VC, KS, VS, TABLE, LENS, 2, 100, 2, 128, 4)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


CACHE = [
    (dict(k_codes=None), -1), (dict(v_codes=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1), (dict(block_table=None), -1), (dict(cache_len=None), -1),
    (dict(layers=0), -2), (dict(num_blocks=0), -2), (dict(kv_heads=0), -2), (dict(head_dim=96), -2), (dict(max_blocks=0), -2), (dict(k_codes=KC + 8), -9), (dict(v_codes=VC + 1), -9),
    (dict(k_scale=KS + 2), -9),
]


def _fork(cache=None, **kw):
    a = dict(B=3, refs=REFS, parent=PARENT, keep=KEEP, room=ROOM, n=5, table=TABLE_OUT, lens=LEN_OUT, refs_out=REFS_OUT, free=FREE, status=STATUS, ws=SPACE, bytes=GB)
    a.update(kw)
    return fsd.library().fsd_cache_fork(cache or _cache(), a["B"], a["refs"], a["parent"], a["keep"], a["room"], a["n"], a["table"], a["lens"], a["refs_out"], a["free"],
                                        a["status"], a["ws"], a["bytes"], None)


def _compact(cache=None, **kw):
    a = dict(B=3, refs=REFS, table=TABLE_OUT, refs_out=REFS_OUT, remap=LEN_OUT, used=FREE, status=STATUS, ws=SPACE, bytes=GB)
    a.update(kw)
    return fsd.library().fsd_cache_compact(cache or _cache(), a["B"], a["refs"], a["table"], a["refs_out"], a["remap"], a["used"], a["status"], a["ws"], a["bytes"], None)


def _copy(src=None, dst=None, **kw):
    a = dict(a=PARENT, b=KEEP, tokens=ROOM, n=5, status=STATUS)
    a.update(kw)
    other = _cache(k_codes=KC + 50 * A, v_codes=VC + 50 * A, k_scale=KS + 50 * A, v_scale=VS + 50 * A, num_blocks=70)
    return fsd.library().fsd_cache_copy(src or _cache(), dst or other, a["a"], a["b"], a["tokens"], a["n"], a["status"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(refs=None), -1), (dict(parent=None), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(refs_out=None), -1), (dict(B=0), -2), (dict(B=65536), -2), (dict(n=0), -2),
    (dict(n=65536), -2), (dict(cache=_cache(num_blocks=(1 << 24) + 1)), -2), (dict(n=65535, cache=_cache(max_blocks=32769)), -2), (dict(refs=REFS + 2), -9),
    (dict(parent=PARENT + 1), -9), (dict(keep=KEEP + 2), -9), (dict(room=ROOM + 2), -9), (dict(table=TABLE_OUT + 2), -9), (dict(lens=LEN_OUT + 2), -9), (dict(refs_out=REFS_OUT + 2), -9),
    (dict(free=FREE + 2), -9), (dict(status=STATUS + 2), -9), (dict(cache=_cache(block_table=TABLE + 2)), -9), (dict(cache=_cache(cache_len=LENS + 2)), -9), (dict(ws=None), -5),
    (dict(ws=SPACE + 128), -5), (dict(bytes=1000), -5),
])
def test_fork_refusals(kw, status):
    assert _fork(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(refs=None), -1), (dict(table=None), -1), (dict(refs_out=None), -1), (dict(B=0), -2), (dict(B=65536), -2), (dict(cache=_cache(num_blocks=(1 << 24) + 1)), -2),
    (dict(refs=REFS + 2), -9), (dict(table=TABLE_OUT + 2), -9), (dict(refs_out=REFS_OUT + 1), -9), (dict(remap=LEN_OUT + 2), -9), (dict(used=FREE + 2), -9), (dict(status=STATUS + 2), -9),
    (dict(cache=_cache(block_table=TABLE + 2)), -9), (dict(ws=None), -5), (dict(ws=SPACE + 8), -5), (dict(bytes=500), -5),
])
def test_compact_refusals(kw, status):
    assert _compact(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(a=None), -1), (dict(b=None), -1), (dict(n=0), -2), (dict(n=-1), -2), (dict(src=_cache(layers=1)), -2), (dict(src=_cache(kv_heads=1)), -2), (dict(src=_cache(head_dim=64)), -2),
    (dict(n=(1 << 31) - 1, src=_cache(layers=1 << 9), dst=_cache(layers=1 << 9)), -2),
    (dict(a=PARENT + 2), -9), (dict(b=KEEP + 1), -9), (dict(tokens=ROOM + 2), -9), (dict(status=STATUS + 2), -9), (dict(status=PARENT + 16), -9), (dict(status=KEEP - 16), -9),
    (dict(status=ROOM), -9), (dict(status=KC + 50 * A + 16), -9),
    # caches that share some of their memory
    (dict(dst=_cache(k_codes=KC + 16)), -9), (dict(dst=_cache(v_codes=VC + 50 * A)), -9), (dict(dst=_cache(k_scale=KS + 4)), -9), (dict(dst=_cache(num_blocks=99)), -9),
    (dict(dst=_cache(k_codes=KC + 2 * 100 * 2 * 64 * 128 - 16, v_codes=VC + 50 * A, k_scale=KS + 50 * A, v_scale=VS + 50 * A)), -9),
    (dict(src=_cache(k_codes=VC + 50 * A, v_codes=KC + 50 * A)), -9),
])
def test_copy_refusals(kw, status):
    assert _copy(**kw) == status


@pytest.mark.parametrize("kw,status", CACHE)
def test_cache_refusals(kw, status):
    assert _fork(cache=_cache(**kw)) == status and _compact(cache=_cache(**kw)) == status and _copy(src=_cache(**kw)) == status
    assert _copy(dst=_cache(**kw)) == status


def test_outputs_that_lie_in_what_a_call_reads():
    size = dict(table=5 * 16, lens=20, refs_out=400, free=4, status=20)
    inputs = dict(refs=(REFS, 400), parent=(PARENT, 20), keep=(KEEP, 20), room=(ROOM, 20), block_table=(TABLE, 48), cache_len=(LENS, 12), ws=(SPACE, 256))
    own = dict(table=TABLE_OUT, lens=LEN_OUT, refs_out=REFS_OUT, free=FREE, status=STATUS)
    for name, n in size.items():
        for what, (at, m) in inputs.items():
            for where in (at, at - n + 4, at + m - 4):
                if name == "refs_out" and where == REFS:
                    continue                                  # in place
                assert _fork(**{name: where}) == -9, (name, what)
        for what, at in own.items():
            if what != name:
                for where in (at, at - n + 4, at + size[what] - 4):
                    assert _fork(**{name: where}) == -9, (name, what)
    assert _fork(refs_out=REFS, table=None) == -1
    size = dict(table=48, refs_out=400, remap=400, used=4, status=12)
    inputs = dict(refs=(REFS, 400), block_table=(TABLE, 48), ws=(SPACE, 256))
    own = dict(table=TABLE_OUT, refs_out=REFS_OUT, remap=LEN_OUT, used=FREE, status=STATUS)
    for name, n in size.items():
        for what, (at, m) in inputs.items():
            for where in (at, at - n + 4, at + m - 4):
                if (name, where) in (("refs_out", REFS), ("table", TABLE)):
                    continue
                assert _compact(**{name: where}) == -9, (name, what)
        for what, at in own.items():
            if what != name:
                for where in (at, at - n + 4, at + size[what] - 4):
                    assert _compact(**{name: where}) == -9, (name, what)


def test_outputs_that_lie_in_the_pages():
    codes, scales = 2 * 100 * 2 * 64 * 128, 2 * 100 * 2 * 4
    for at, m in ((KC, codes), (VC, codes), (KS, scales), (VS, scales)):
        for where in (at, at + m - 4):
            for name in ("table", "lens", "refs_out", "free", "status"):
                assert _fork(**{name: where}) == -9, name
            for name in ("table", "refs_out", "remap", "used", "status"):
                assert _compact(**{name: where}) == -9, name
        assert _fork(ws=at) == -9 and _compact(ws=at + m // 256 * 256 - 256) == -9


def test_row_strides():
    import torch

    whole = torch.zeros(3, 4, 50)
    assert drafting._row_stride(whole, "z") == 50 and drafting._row_stride(whole[:, :, :7], "z") == 50 and drafting._row_stride(whole[:1, :, 3:], "z") == 50
    assert drafting._row_stride(whole[:, :1, :9], "z") == 200 and drafting._row_stride(torch.zeros(1, 1, 9), "z") == 9 and drafting._row_stride(whole[:, :, :1], "z") == 50
    for bad in (whole[:, :2], whole[:, :, ::2], whole.transpose(0, 1)):
        with pytest.raises(ValueError):
            drafting._row_stride(bad, "z")


def test_sizes_are_refused_before_outputs_are_made(monkeypatch):
    """(the sizes of a call come from the caller's n: outputs of 2^40 numbers are not asked for)"""
    import torch

    class OnGpu:
        is_cuda, device, dtype, shape = True, types.SimpleNamespace(index=0), torch.float32, (2, 3, 10)

        def dim(self):
            return 3

        def stride(self):
            return 30, 10, 1

    monkeypatch.setattr(drafting, "_on_current", lambda device, stream: None)
    monkeypatch.setattr(drafting, "_new", lambda *a, **k: pytest.fail("made"))
    for n in (-1, 0, 129, 1 << 30, 1 << 40, (1 << 32) + 4):
        with pytest.raises(fsd.FsdError, match="fsd_beam_select"):
            fsd.fsd_beam_select(OnGpu(), None, n)
    OnGpu.shape = 2, 3, (1 << 32) + 10
    with pytest.raises(fsd.FsdError, match="fsd_beam_select"):
        fsd.fsd_beam_select(OnGpu(), None, 4)


def test_binding_refusals():
    import torch

    z, s = torch.zeros(2, 3, 10), torch.zeros(2, 3)
    with pytest.raises(ValueError):
        fsd.fsd_beam_select(z, s, 4)                          # not on the GPU
    with pytest.raises(ValueError):
        fsd.fsd_beam_select(z[0], s, 4)
    with pytest.raises(ValueError):
        fsd.fsd_beam_reorder(z, torch.zeros((2, 3), dtype=torch.int32))
    with pytest.raises(ValueError):
        fsd.fsd_beam_reorder(z, torch.zeros((2, 3), dtype=torch.int32), batch_dim=2)
    with pytest.raises(ValueError):
        fsd.fsd_beam_reorder(z, torch.zeros((2, 3), dtype=torch.int32), batch_dim=-1)


def test_parts_of_one_tensor():
    """outputs that the binding makes are apart, aligned and of the shapes asked for"""
    import torch

    shapes = dict(a=((3, 5), torch.float32), b=((7,), torch.int32), c=((1,), torch.int32), d=((2, 2), torch.int32))
    for space in (0, 1, 300, 4096):
        got, whole, base = drafting._parts(None, torch.device("cpu"), space, **shapes)
        end = max(t.data_ptr() + 4 * t.numel() for t in got.values())
        assert base % 256 == 0 and base >= end and (not space or base + space <= whole.data_ptr() + 4 * whole.numel())
    assert got["a"].shape == (3, 5) and got["a"].dtype == torch.float32 and got["a"].is_contiguous() and got["d"].is_contiguous()
    for k, t in enumerate(got.values()):
        t.fill_(k + 1)
    assert [int(t.sum()) for t in got.values()] == [15, 14, 3, 16]
    assert all((t.data_ptr() - got["a"].data_ptr()) % 64 == 0 for t in got.values())


def test_tables_of_a_cache_are_taken_over():
    assert types.FunctionType is type(fsd.Cache.with_tables) and fsd.ROW_NO_BLOCKS == 64
