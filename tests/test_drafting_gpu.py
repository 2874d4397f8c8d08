"""The operators around drafting on the GPU, against plain implementations (drafting_ref.py)."""
import numpy as np
import pytest
import torch

import paper_2502_20704_amd as fsd
from tests import drafting_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _host(t):
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def _dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ------------------------------------------------------------------------------------------ selection


def _same_selection(got, want, what=""):
    """Whole numbers equal; scores within their one rounding to binary32 (2^-24) and the normaliser's error: the row's sum of exponentials is off
    by 2^-33 of it at most, its logarithm by as much, the binary64 sums by next to nothing."""
    scores, parent, tokens, status, nearest = want
    assert nearest > 2.0 ** -31 or nearest == 0.0, "two beams' entries lie too near to one another for a test of their order"
    torch.cuda.synchronize()
    assert (_host(got["row_status"]) == status).all(), what
    assert (_host(got["parent"]) == parent).all(), what
    assert (_host(got["tokens"]) == tokens).all(), what
    s = _host(got["scores"])
    with np.errstate(over="ignore"):
        fine = np.isfinite(scores.astype(np.float32))         # (what lies below binary32's range is rounded to -inf)
    assert (np.isneginf(s) == ~fine).all(), what
    bound = 2.0 ** -24 * np.abs(scores[fine]) * (1 + 2.0 ** -20) + 2.0 ** -32 + 2.0 ** -149
    assert (np.abs(s[fine] - scores[fine]) <= bound).all(), what


def _logits(rng, B, W, V, dtype, spread=3.0):
    return torch.from_numpy((rng.standard_normal((B, W, V)) * spread).astype(np.float32)).to(DT[dtype])


def _scores(rng, B, W):
    return -np.sort(rng.uniform(0, 12, (B, W))).astype(np.float32)


SELECT = [
    # B, beams, V, n, dtype
    (1, 1, 1, 1, "f32"), (1, 1, 1, 5, "bf16"), (2, 3, 7, 4, "f32"), (2, 2, 3, 128, "bf16"), (3, 4, 1000, 8, "bf16"), (1, 4, 32000, 8, "bf16"),
    (1, 1, 32001, 1, "f32"), (5, 2, 2049, 3, "bf16"), (2, 8, 128257, 16, "bf16"), (2, 3, 128256, 60, "f32"), (1, 1, 262145, 128, "f32"),
    (1, 256, 515, 128, "bf16"), (70, 16, 999, 20, "f32"), (40, 32, 2056, 64, "bf16"), (1, 2, 524288, 33, "bf16"), (300, 1, 515, 2, "bf16"),
    (130, 9, 16385, 100, "bf16"),
]


@pytest.mark.parametrize("B,W,V,n,dtype", SELECT)
def test_select(B, W, V, n, dtype):
    rng = np.random.default_rng(B * 7 + W * 11 + V + n)
    z = _logits(rng, B, W, V, dtype)
    scores = _scores(rng, B, W)
    got = fsd.fsd_beam_select(z.cuda(), _dev(scores), n)
    _same_selection(got, ref.select(_host(z), scores, None, None, n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [100, 40001])
def test_select_finished_weighted_masked(V, dtype):
    rng = np.random.default_rng(V)
    B, W, n = 9, 6, 12
    z = _logits(rng, B, W, V, dtype)
    z[torch.from_numpy(rng.random((B, W, V)) < 0.9)] = -float("inf")
    z[0, 2] = -float("inf")                                   # a beam that a grammar has ended
    z[1] = -float("inf")                                      # all of them
    z[2, :, 5:] = -float("inf")                               # few continuations
    z[2, :, :5] = 1.0
    scores, weights = _scores(rng, B, W), rng.uniform(0.05, 2.0, (B, W)).astype(np.float32)
    scores[3, 2:] = -np.inf
    scores[4] = -np.inf
    done = (rng.random((B, W)) < 0.3).astype(np.int32)
    done[5] = -1                                              # (anything but 0)
    done[3, 3] = 1                                            # finished, and does not count
    weights[4, 1], weights[3, 4] = np.nan, -1.0               # of beams that do not count
    for w, d in ((weights, done), (None, done), (weights, None)):
        got = fsd.fsd_beam_select(z.cuda(), _dev(scores), n, weights=_dev(w), done=_dev(d))
        _same_selection(got, ref.select(_host(z), scores, w, d, n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_equal_entries(dtype):
    """ties go to the lowest beam and entry, also where more entries are equal than a workgroup's list holds"""
    V, n = 40000, 100
    z = torch.zeros((7, 2, V), dtype=DT[dtype])
    z[1] = -2.5
    z[2, :, ::2] = 1.0
    z[3, 0], z[3, 1] = torch.arange(V) // 64 / 16.0, -(torch.arange(V) // 64) / 16.0   # in order, either way
    z[4, :, :30000] = -float("inf")
    z[4, :, 20000:20050] = 3.0                                # a part of the best, then equal ones
    z[5, :, ::3], z[5, :, 1::3] = -0.0, -1.0                  # 0 and -0 are equal
    z[6, 1] = -float("inf")
    scores = np.zeros((7, 2), np.float32)
    want = ref.select(_host(z), scores, None, None, n)
    _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(scores), n), (*want[:4], np.inf))
    _same_selection(fsd.fsd_beam_select(z.cuda(), None, n), (*want[:4], np.inf))
    for short in (1, 3, 17):
        want = ref.select(_host(z), scores, None, None, short)
        _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(scores), short), (*want[:4], np.inf))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_sizes_of_numbers(dtype):
    """logits of any size: the normaliser is formed from distances"""
    rng = np.random.default_rng(5)
    V = 5000
    z = _logits(rng, 6, 1, V, dtype)
    z[0] *= 1e30
    z[1] = -3e38
    z[1, 0, 7] = 3e38
    z[2] += 2.0 ** 22
    z[3] *= 1e-38
    z[4] *= 300.0
    z[5, 0, 0], z[5, 0, 1:] = 0.0, -700.0
    scores = np.array([[0.0], [-3e38], [-1e-30], [-5.0], [1e6], [-0.0]], np.float32)
    _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(scores), 9), ref.select(_host(z), scores, None, None, 9))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [9, 33333])
def test_select_reports(V, dtype):
    rng = np.random.default_rng(V)
    B, W, n = 14, 3, 4
    z = _logits(rng, B, W, V, dtype)
    scores, weights, done = _scores(rng, B, W), np.ones((B, W), np.float32), np.zeros((B, W), np.int32)
    nan, inf = float("nan"), float("inf")
    z[0, 1, V - 1], z[1, 0, 0], z[2, 2, V // 2] = nan, inf, -nan
    z[3, 1] = nan
    z[4, 1], z[4, 1, 3] = -inf, nan
    z[5, 0], done[5, 0] = nan, 1                              # rows that are not read
    z[6, 2], scores[6, 2] = nan, -inf
    scores[7, 1], scores[8, 0] = nan, inf
    weights[9, 0], weights[10, 2], weights[11, 1], weights[12, 1] = 0.0, inf, nan, -2.0
    done[11, 1], done[7, 1] = 1, 1
    got = fsd.fsd_beam_select(z.cuda(), _dev(scores), n, weights=_dev(weights), done=_dev(done))
    want = ref.select(_host(z), scores, weights, done, n)
    assert [b for b in range(B) if want[3][b]] == [0, 1, 2, 3, 4, 7, 8, 9, 10, 11, 12]
    _same_selection(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_strides(dtype):
    rng = np.random.default_rng(8)
    wide = _logits(rng, 3, 4, 1000, dtype).cuda()
    scores = _scores(rng, 3, 4)
    for z in (wide[:, :, :777], wide[:, :, 3:], wide[:, :, 1:2], wide[1:2, :, 5:900], wide[:, :1, 7:]):
        s = scores[:z.shape[0], :z.shape[1]]
        if z.shape[1] == 1 and z.shape[0] > 1:
            got = fsd.fsd_beam_select(z, _dev(s), 6)          # one beam: the sequences' distance counts
        else:
            got = fsd.fsd_beam_select(z, _dev(s), 6)
        _same_selection(got, ref.select(_host(z), s, None, None, 6))


def test_select_rows_far_apart():
    """elements beyond 2^32 bytes and 2^31 elements"""
    stride = (1 << 31) + 24
    buffer = torch.zeros(2 * stride + 4096, dtype=torch.bfloat16, device="cuda")
    z = torch.as_strided(buffer, (1, 3, 1000), (3 * stride, stride, 1))
    rng = np.random.default_rng(1)
    z.copy_(_logits(rng, 1, 3, 1000, "bf16"))
    scores = _scores(rng, 1, 3)
    _same_selection(fsd.fsd_beam_select(z, _dev(scores), 20), ref.select(_host(z), scores, None, None, 20))


# ------------------------------------------------------------------------------------------ states


@pytest.mark.parametrize("row,dtype", [(1, torch.uint8), (3, torch.uint8), (16, torch.uint8), (17, torch.int16), (500, torch.float32), (16384, torch.uint8),
                                       (16385, torch.uint8), (50001, torch.bfloat16)])
@pytest.mark.parametrize("layers,B,W,n", [(1, 1, 1, 1), (3, 5, 4, 7), (2, 1, 300, 2)])
def test_reorder(row, dtype, layers, B, W, n):
    rng = np.random.default_rng(row + W)
    size = row * torch.empty((), dtype=dtype).element_size()
    flat = torch.from_numpy(rng.integers(0, 256, layers * B * W * size + 1, dtype=np.uint8)).cuda()
    parent = rng.integers(-1, W, (B, n)).astype(np.int32)
    if B > 2:
        parent[1, 0], parent[2, n - 1] = W, -2
    for odd in ([0, 1] if dtype == torch.uint8 else [0]):     # any address
        bytes_in = flat[odd:odd + layers * B * W * size]
        out = dict(out=torch.full((layers * B * n * size + 1,), 77, dtype=torch.uint8, device="cuda")[odd:odd + layers * B * n * size].view(dtype).view(layers, B, n, row),
                   row_status=torch.full((B,), 9, dtype=torch.int32, device="cuda"))
        got = fsd.fsd_beam_reorder(bytes_in.view(dtype).view(layers, B, W, row), _dev(parent), batch_dim=1, out=out)
        want, status = ref.reorder(bytes_in.cpu().numpy().reshape(layers, B, W, size), parent)
        torch.cuda.synchronize()
        assert (got["out"].contiguous().view(torch.uint8).cpu().numpy().reshape(want.shape) == want).all()
        assert (_host(got["row_status"]) == status).all()


def test_reorder_dimensions():
    states = torch.arange(4 * 3 * 5, device="cuda", dtype=torch.float32).view(4, 3, 5)
    parent = torch.tensor([[2, 0], [1, 1], [-1, 0], [0, 2]], dtype=torch.int32, device="cuda")
    got = fsd.fsd_beam_reorder(states, parent)["out"]
    assert torch.equal(got[0, 0], states[0, 2]) and torch.equal(got[1], states[1, [1, 1]]) and not got[2, 0].any()
    flat = states.view(4, 15)[:, :3].contiguous()             # one number a beam
    assert torch.equal(fsd.fsd_beam_reorder(flat, parent)["out"][3], flat[3, [0, 2]])


# ------------------------------------------------------------------------------------------ pages


def _pages(rng, L, P, H, D):
    return dict(k_codes=rng.integers(0, 256, (L, P, H, 64, D), dtype=np.uint8), v_codes=rng.integers(0, 256, (L, P, H, 4, D, 16), dtype=np.uint8),
                k_scale=rng.random((L, P, H), dtype=np.float32), v_scale=rng.random((L, P, H), dtype=np.float32))


def _cache(pages, table, lens):
    return fsd.Cache(*(_dev(pages[k]) for k in ("k_codes", "v_codes", "k_scale", "v_scale")), _dev(table), _dev(lens))


def _same_pages(cache, pages):
    for k, v in pages.items():
        assert (getattr(cache, k).cpu().numpy() == v).all(), k


def _sequences(rng, B, M, P, share=0.3, most=None):
    """tables and counts as calls leave them: some full blocks shared, some places reserved; and counts of others"""
    order = list(rng.permutation(P))
    table, lens = np.full((B, M), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        n = int(rng.integers(0, (most or 64 * M) + 1))
        lens[b] = n
        first = int(rng.integers(0, b)) if b and rng.random() < share else None
        for j in range(-(-n // 64)):
            if first is not None and j < min(n, lens[first]) // 64 and rng.random() < 0.9:
                table[b, j] = table[first, j]
            else:
                table[b, j] = order.pop()
        for j in range(-(-n // 64), min(M, -(-n // 64) + int(rng.integers(0, 3)))):
            if order:
                table[b, j] = order.pop()
    refs = np.bincount(table[table >= 0], minlength=P).astype(np.int32)
    for e in rng.choice(P, max(1, P // 10), replace=False):   # a store of prompts holds these too
        refs[e] += int(rng.integers(1, 3))
    return table, lens, refs


def _fork(rng, table, lens, refs, parent, lengths, room, L=1, H=1, D=64, **kw):
    B, M = table.shape
    pages = _pages(rng, L, len(refs), H, D)
    cache = _cache(pages, table, lens)
    want = ref.fork(table, lens, refs, parent, lengths, room)
    got = fsd.fsd_cache_fork(cache, _dev(parent), _dev(refs), lengths=_dev(lengths), room=_dev(room), **kw)
    torch.cuda.synchronize()
    for name, w in zip(("block_table", "cache_len", "refs", "free_blocks", "row_status"), want):
        assert (_host(got[name]) == w).all(), name
    ref.move_pages({k: v.copy() for k, v in pages.items()}, pages, want[5])
    _same_pages(cache, pages)
    assert (cache.block_table.cpu().numpy() == table).all()
    return got, want


FORK = [
    # B, n, M, P, layers, heads, head_dim
    (1, 1, 1, 3, 1, 1, 64), (1, 4, 3, 20, 2, 3, 64), (6, 6, 5, 60, 1, 2, 128), (6, 11, 5, 100, 2, 1, 256), (9, 3, 4, 50, 1, 1, 64),
    (40, 70, 3, 400, 1, 1, 64), (3, 5, 600, 3000, 1, 1, 64), (300, 600, 2, 2500, 1, 1, 64), (5, 5, 2, 5000, 1, 1, 64),
]


@pytest.mark.parametrize("B,n,M,P,L,H,D", FORK)
@pytest.mark.parametrize("seed", [0, 1])
def test_fork(B, n, M, P, L, H, D, seed):
    rng = np.random.default_rng(1000 * seed + B + n + M + P)
    table, lens, refs = _sequences(rng, B, M, P)
    parent = rng.integers(-1, B, n).astype(np.int32)
    have = np.where(parent >= 0, lens[np.maximum(parent, 0)], 0)
    lengths = np.where(rng.random(n) < 0.5, have, rng.integers(0, have + 1)).astype(np.int32)
    room = np.minimum(rng.choice([0, 1, 9, 70, 200], n), 64 * M - lengths).astype(np.int32)
    _fork(rng, table, lens, refs, parent, lengths, room, L, H, D)
    _fork(rng, table, lens, refs, parent, None, None, L, H, D)
    same = np.arange(min(n, B)).astype(np.int32)              # every sequence goes on
    _fork(rng, table, lens, refs, same, None, None, L, H, D)


def test_fork_beams_of_all_lengths():
    """one sequence, copied for each length of its last block, and for one behind a full block"""
    for length in (1, 15, 16, 17, 63, 64, 65, 128):
        rng = np.random.default_rng(length)
        table = np.array([[4, 2, -1, -1]], np.int32) if length <= 128 else None
        refs = np.zeros(12, np.int32)
        refs[[4, 2]] = 1
        _, want = _fork(rng, table, np.array([length], np.int32), refs, np.zeros(3, np.int32), None, np.array([1, 0, 100], np.int32), 2, 2, 128)
        assert len(want[5]) == (2 if length % 64 else 0)


def test_fork_order_of_claims():
    """A block may be kept by the first that wants it only if no one else names it: not another batch, not a full place of a
    longer sibling; and what a shorter sibling would overwrite is copied."""
    rng = np.random.default_rng(3)
    table = np.array([[1, 2, 3, 4], [5, -1, -1, -1]], np.int32)
    lens = np.array([200, 30], np.int32)
    refs = np.array([0, 1, 1, 1, 1, 2, 0, 0, 0, 0, 0, 0], np.int32)      # block 5: another batch has it too
    parent, lengths = np.array([0, 0, 0, 1, -1], np.int32), np.array([100, 200, 70, 30, 0], np.int32)
    _, want = _fork(rng, table, lens, refs, parent, lengths, np.array([10, 10, 0, 1, 64], np.int32))
    assert want[0][1].tolist() == [1, 2, 3, 4] and want[0][0][1] != 2 and want[0][2][1] != 2 and want[0][3][0] != 5 and len(want[5]) == 3


def test_fork_reports():
    rng = np.random.default_rng(4)
    table = np.array([[1, 2, 3], [4, -1, 5], [6, 99, -1], [7, 8, -1], [9, 10, 11]], np.int32)
    lens = np.array([130, 150, 70, 200, -4], np.int32)
    refs = np.bincount(np.arange(1, 12), minlength=30).astype(np.int32)
    parent = np.array([0, 1, 2, 3, 4, 5, -2, 0, 0, 0, -1, 2, -1], np.int32)
    lengths = np.array([130, 150, 70, 10, 0, 0, 0, 131, -1, 5, 77, 64, 0], np.int32)
    room = np.array([62, 0, 0, 0, 0, 0, 0, 0, 0, 188, 192, 0, 193], np.int32)
    _, want = _fork(rng, table, lens, refs, parent, lengths, room)
    assert want[4].tolist() == [0, 32, 32, 32, 32, 2, 2, 32, 32, 32, 0, 0, 32]


def test_fork_without_blocks():
    rng = np.random.default_rng(6)
    table = np.array([[0, 1], [2, -1]], np.int32)
    lens, refs = np.array([100, 10], np.int32), np.array([1, 1, 1, 0, 0], np.int32)
    parent = np.array([0, 0, 0, 7], np.int32)
    _, want = _fork(rng, table, lens, refs, parent, None, None)          # two copies, block 2 free again: enough
    assert want[3] == 1
    _, want = _fork(rng, table, lens, refs, np.array([0, 0, 0, 0, 0, 7], np.int32), None, None)
    assert want[3] == -1 and want[4].tolist() == [64] * 5 + [66] and (want[0] == -1).all()
    # the counts may be brought up to date in place, also then
    for p in (parent, np.array([0, 0, 0, 0, 0], np.int32)):
        r = _dev(refs)
        pages = _pages(rng, 1, 5, 1, 64)
        cache = _cache(pages, table, lens)
        n = len(p)
        out = dict(block_table=torch.empty((n, 2), dtype=torch.int32, device="cuda"), cache_len=torch.empty(n, dtype=torch.int32, device="cuda"), refs=r)
        fsd.fsd_cache_fork(cache, _dev(p), r, out=out)
        torch.cuda.synchronize()
        assert (_host(r) == ref.fork(table, lens, refs, p, None, None)[2]).all()


def test_fork_of_inconsistent_tables():
    """one block at two places, counts that are too small: nothing out of range, and what is said holds"""
    rng = np.random.default_rng(7)
    table = np.array([[3, 3, 3], [3, 4, 4]], np.int32)
    lens = np.array([128, 70], np.int32)
    for refs in (np.array([0, 0, 0, 4, 2, 0, 0, 0, 0, 0, 0, 0], np.int32), np.zeros(12, np.int32), np.full(12, -5, np.int32)):
        _fork(rng, table, lens, refs, np.array([1, 0, 1, 1], np.int32), np.array([70, 100, 30, 64], np.int32), np.array([60, 70, 100, 100], np.int32))


@pytest.mark.parametrize("L,P,Q,H,D,n", [(1, 5, 5, 1, 64, 1), (3, 9, 20, 2, 128, 9), (2, 30, 7, 3, 256, 6)])
def test_copy(L, P, Q, H, D, n):
    rng = np.random.default_rng(P + Q)
    a, b = _pages(rng, L, P, H, D), _pages(rng, L, Q, H, D)
    empty = np.full((1, 1), -1, np.int32), np.zeros(1, np.int32)
    src, dst = _cache(a, *empty), _cache(b, *empty)
    come, go = rng.choice(P, n, replace=False).astype(np.int32), rng.choice(Q, n, replace=False).astype(np.int32)
    tokens = rng.integers(0, 65, n).astype(np.int32)
    status = np.zeros(n, np.int64)
    pairs = [(int(x), int(y), -(-int(t) // 16)) for x, y, t in zip(come, go, tokens)]
    if n > 5:
        come[0], go[1], come[2], go[3], tokens[4], tokens[5] = -1, -1, P, Q, 65, -1
        status[2:6] = 32
        pairs = pairs[6:]
    got = fsd.fsd_cache_copy(src, dst, _dev(come), _dev(go), tokens=_dev(tokens))
    torch.cuda.synchronize()
    ref.move_pages(a, b, pairs)
    assert (_host(got["page_status"]) == status).all()
    _same_pages(src, a)
    _same_pages(dst, b)
    # whole pages, within one cache
    k = P // 2
    fsd.fsd_cache_copy(src, src, _dev(np.arange(k, dtype=np.int32)), _dev(np.arange(P - k, P, dtype=np.int32)))
    torch.cuda.synchronize()
    ref.move_pages({x: y.copy() for x, y in a.items()}, a, [(i, P - k + i, 4) for i in range(k)])
    _same_pages(src, a)


@pytest.mark.parametrize("P,share", [(1, 0.0), (1, 1.0), (2, 0.5), (40, 0.0), (40, 1.0), (40, 0.4), (1024, 0.5), (1025, 0.9), (3000, 0.1), (3000, 0.7)])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(P, share, in_place):
    rng = np.random.default_rng(P)
    L, H, D, B, M = 2, 1, 64, 7, 9
    refs = np.where(rng.random(P) < share, rng.integers(1, 5, P), -(rng.random(P) < 0.1).astype(np.int32)).astype(np.int32)
    used = np.flatnonzero(refs > 0)
    table = np.full((B, M), -1, np.int32)
    if len(used):
        table[:, :6] = rng.choice(used, (B, 6))
    table[1, 2], table[2, 7], table[3, 8] = -9, P, 1 << 30
    free = np.flatnonzero(refs <= 0)
    if len(free):
        table[4, 3] = free[-1]
    pages = _pages(rng, L, P, H, D)
    cache, r = _cache(pages, table, np.zeros(B, np.int32)), _dev(refs)
    want = ref.compact(table, refs)
    kw = dict(out=dict(block_table=cache.block_table, refs=r, remap=torch.empty_like(r), used_blocks=torch.empty(1, dtype=torch.int32, device="cuda"),
                       row_status=torch.empty(B, dtype=torch.int32, device="cuda"))) if in_place else {}
    got = fsd.fsd_cache_compact(cache, r, **kw)
    torch.cuda.synchronize()
    for name, w in zip(("block_table", "refs", "remap", "used_blocks", "row_status"), want):
        assert (_host(got[name]) == w).all(), name
    ref.move_pages({k: v.copy() for k, v in pages.items()}, pages, want[5])
    _same_pages(cache, pages)
