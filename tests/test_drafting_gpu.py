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
    (130, 9, 16385, 100, "bf16"), (65535, 1, 5, 3, "bf16"), (1, 256, 70000, 128, "bf16"),
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
@pytest.mark.parametrize("B,W,V", [(3, 2, 50), (4, 3, 9001), (12, 8, 100003)])
def test_select_masks_of_the_lowest_number(B, W, V, dtype):
    """masked places that hold the type's lowest number are entries, behind all others; a row of nothing else has them all equal"""
    rng = np.random.default_rng(V)
    z = _logits(rng, B, W, V, dtype)
    keep = rng.random((B, W, V)) < 12.0 / V
    z[torch.from_numpy(~keep)] = torch.finfo(DT[dtype]).min
    z[0] = torch.finfo(DT[dtype]).min
    z[1, 0] = torch.finfo(DT[dtype]).min
    scores = _scores(rng, B, W)
    for n in (5, 40, 128):
        got, want = fsd.fsd_beam_select(z.cuda(), _dev(scores), n), ref.select(_host(z), scores, None, None, n)
        _same_selection(got, want)
    got, want = fsd.fsd_beam_select(z[:1].cuda(), None, 40), ref.select(_host(z[:1]), None, None, None, 40)   # (equal to the last bit)
    _same_selection(got, (*want[:4], np.inf))
    assert (want[1] == 0).all() and (want[2] == np.arange(40)).all()


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
    # more than one workgroup takes: many blocks, many places, many sequences
    (12, 30, 5, 4500, 2, 2, 64), (8, 8, 1500, 13000, 1, 1, 64), (300, 600, 20, 6500, 1, 1, 64), (1100, 1200, 2, 4000, 1, 1, 64), (7, 1, 3, 4097, 2, 3, 128),
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


@pytest.mark.parametrize("P,share", [(1, 0.0), (1, 1.0), (2, 0.5), (40, 0.0), (40, 1.0), (40, 0.4), (1024, 0.5), (1025, 0.9), (3000, 0.1), (3000, 0.7),
                                     (4097, 0.5), (5000, 0.0), (5000, 1.0), (9000, 0.3), (6144, 0.8)])
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


# ------------------------------------------------------------------------------------------ larger rows


def _long_rows():
    """bfloat16 rows that go to the kernel with the table of exponentials, and what it does not hold"""
    rng = np.random.default_rng(12)
    B, W, V = 12, 8, 100003
    z = torch.from_numpy(rng.standard_normal((B, W, V)).astype(np.float32) * 3)
    z[1] *= 30.0                                              # largest beyond 64
    z[2] -= 100.0                                             # largest under -20
    z[3] *= 1e-4                                              # nearer to 0 than the table goes
    z[4] = 0.0
    z[5] = (torch.arange(V) // 64 / 64.0)                     # in order
    z[6][torch.from_numpy(rng.random((W, V)) < 0.99)] = -float("inf")
    z[7, :, :60000] -= 1000.0                                 # nothing like the rest in front
    z[8, :, 50000:] += 80.0
    z[9] = -float("inf")
    z[9, 3, V - 1], z[9, 5, 0] = -3000.0, 7.0
    z[10] = -70.0 - z[10].abs()                               # under the table's end, every one
    z[11, :, 1:] = -63.9
    z[11, :, 0] = 1e-30
    return z.to(torch.bfloat16), _scores(rng, B, W)


@pytest.mark.parametrize("n", [1, 16, 128])
def test_select_long_rows(n):
    z, scores = _long_rows()
    wide = torch.full((12, 8, 100104), 7.0, dtype=torch.bfloat16, device="cuda")
    got = []
    for rows in (z.cuda(), wide[:, :, 1:100004].copy_(z)):    # whole, and at odd addresses
        got.append(fsd.fsd_beam_select(rows, _dev(scores), n))
    want = ref.select(_host(z), scores, None, None, n)
    for g in got:
        _same_selection(g, (*want[:4], np.inf))
    assert want[4] > 2.0 ** -31


def test_select_long_rows_reports():
    z, scores = _long_rows()
    z[3, 4, 99].view(torch.int16).fill_(0x7F81)               # a signalling NaN
    z[0, 7, 100002], z[1, 0, 3], z[4, 2, 77], z[6, 6, 50001] = float("nan"), float("inf"), -float("nan"), float("nan")
    done = np.zeros((12, 8), np.int32)
    done[6, 6], done[2, 1] = 1, 1
    got = fsd.fsd_beam_select(z.cuda(), _dev(scores), 5, done=_dev(done))
    want = ref.select(_host(z), scores, None, done, 5)
    assert [b for b in range(12) if want[3][b]] == [0, 1, 3, 4]
    _same_selection(got, (*want[:4], np.inf))


@pytest.mark.parametrize("spread", [3.0, 300.0])
def test_select_long_binary32_rows(spread):
    """slices of several chunks"""
    rng = np.random.default_rng(9)
    z = _logits(rng, 11, 8, 100003, "f32", spread)
    z[3, :, 40000:60000] = -float("inf")
    z[4] = 1.25
    z[5] = torch.arange(100003) / 1000.0
    scores = _scores(rng, 11, 8)
    want = ref.select(_host(z), scores, None, None, 37)
    _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(scores), 37), (*want[:4], np.inf))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_one_beam_has_all_of_the_best(dtype):
    """most of the best entries in the lists of one beam, and of one slice"""
    rng = np.random.default_rng(10)
    z = _logits(rng, 3, 60, 6000, dtype, 0.5)
    z[0, 17] *= 8
    z[1, 59, 4000:4500] += 9.0
    scores = np.zeros((3, 60), np.float32)
    scores[0, 17] = 12.0
    scores[2] = -np.arange(60) * 3.0
    want = ref.select(_host(z), scores, None, None, 128)
    _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(scores), 128), (*want[:4], np.inf))


@pytest.mark.parametrize("far", [0.0, 40.0])
@pytest.mark.parametrize("B,W,V,n,dtype", [(1, 4, 32000, 128, "bf16"), (2, 4, 15375, 82, "bf16"), (1, 1, 128256, 128, "bf16"), (1, 30, 3000, 128, "f32"), (3, 24, 13697, 99, "f32"),
                                           (1, 64, 32000, 128, "bf16"), (2, 256, 1500, 128, "f32"), (1, 3, 200001, 100, "f32"), (64, 8, 9000, 128, "bf16")])
def test_select_one_list_has_most_of_the_best(B, W, V, n, dtype, far):
    """side by side in one row, and in order, so that one slice's list gives most of the answer, and to its end where the other beams' scores are far below"""
    rng = np.random.default_rng(W + V + n)
    z = torch.from_numpy(rng.standard_normal((B, W, V)).astype(np.float32))
    at = V // 3 // 64 * 64
    z[:, W - 1, at:at + n] = 9.0 + torch.arange(n) * 0.0625
    z[-1, 0, 5] = 9.03
    z = z.to(torch.bfloat16) if dtype == "bf16" else z
    scores = rng.random((B, W)).astype(np.float32) * 0.01
    scores[:, :W - 1] -= np.float32(far)
    want = ref.select(_host(z), scores, None, None, n)
    _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(scores), n), want)
    assert far == 0.0 or (want[1][0] == W - 1).all()


@pytest.mark.parametrize("n", [1, 17, 100, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_last_slices_of_all_lengths(dtype, n):
    """rows whose last slice has fewer slots than a workgroup has threads, or than one of its wavefronts"""
    rng = np.random.default_rng(n)
    for V in (8, 120, 505, 1000, 1776, 2040, 2055, 2300, 3200, 4100, 6151, 128256):
        z, scores = _logits(rng, 1, 2, V, dtype), _scores(rng, 1, 2)
        _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(scores), n), ref.select(_host(z), scores, None, None, n), V)


# ------------------------------------------------------------------------------------------ the largest


def test_fork_and_compact_largest_batch():
    """as many sequences as there may be, before and after"""
    rng = np.random.default_rng(17)
    n, P = 65535, 140000
    table, lens, refs = _sequences(rng, n, 2, P, most=100)
    parent = rng.integers(-1, n, n).astype(np.int32)
    codes = lambda: torch.empty((1, P, 1, 64 * 64), dtype=torch.uint8, device="cuda")  # noqa: E731
    scale = torch.arange(P, dtype=torch.float32, device="cuda").view(1, P, 1)
    cache = fsd.Cache(codes().view(1, P, 1, 64, 64), codes().view(1, P, 1, 4, 64, 16), scale.clone(), -scale, _dev(table), _dev(lens))
    want = ref.fork(table, lens, refs, parent, None, None)
    got = fsd.fsd_cache_fork(cache, _dev(parent), _dev(refs))
    torch.cuda.synchronize()
    for name, w in zip(("block_table", "cache_len", "refs", "free_blocks", "row_status"), want):
        assert (_host(got[name]) == w).all(), name
    scales = np.arange(P, dtype=np.float32)
    for a, b, _ in want[5]:
        scales[b] = a
    assert len(want[5]) > 10000 and (_host(cache.k_scale).reshape(-1) == scales).all() and (_host(cache.v_scale).reshape(-1) == -scales).all()
    cache = cache.with_tables(got["block_table"], got["cache_len"])
    want = ref.compact(want[0], want[2])
    got = fsd.fsd_cache_compact(cache, got["refs"])
    torch.cuda.synchronize()
    for name, w in zip(("block_table", "refs", "remap", "used_blocks", "row_status"), want):
        assert (_host(got[name]) == w).all(), name


def test_pages_beyond_32_bits_of_bytes():
    """5 GB of codes: pages from behind 2^32 to the front, and back"""
    L, P, H, D = 1, 40000, 16, 128
    k, v = (torch.empty((L, P, H * 64 * D), dtype=torch.uint8, device="cuda") for _ in range(2))
    scale = torch.rand((2, L, P, H), device="cuda")
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = fsd.Cache(k.view(L, P, H, 64, D), v.view(L, P, H, 4, D, 16), scale[0], scale[1], ints(39998, 39999)[None], ints(100))
    some = [0, 1, 2, 7231, 7232, 32767, 32768, 39997, 39998, 39999]    # (block 7232 is where the low 32 bits of block 40000 would be)

    def fill():
        for e in some:
            k[0, e], v[0, e] = (torch.randint(0, 256, (H * 64 * D,), dtype=torch.uint8, device="cuda") for _ in range(2))
        return {e: (k[0, e].clone(), v[0, e].clone(), scale[:, 0, e].clone()) for e in some}

    def check(was, moved, tokens=None):
        torch.cuda.synchronize()
        for e in some:
            if e in (tokens or {}):                           # the first groups of 16 tokens of each head
                g = tokens[e]
                for x, y in ((k[0, e], was[moved[e]][0]), (v[0, e], was[moved[e]][1])):
                    assert torch.equal(x.view(H, 4, 16 * D)[:, :g], y.view(H, 4, 16 * D)[:, :g]), e
            else:
                assert torch.equal(k[0, e], was[moved.get(e, e)][0]) and torch.equal(v[0, e], was[moved.get(e, e)][1]), e
            assert torch.equal(scale[:, 0, e], was[moved.get(e, e)][2]), e

    was = fill()
    fsd.fsd_cache_copy(cache, cache, ints(39999, 0), ints(1, 39997))
    check(was, {1: 39999, 39997: 0})
    was = fill()
    refs = torch.ones(P, dtype=torch.int32, device="cuda")
    refs[[0, 7232]] = 0                                       # a copy of the begun block goes to block 0
    got = fsd.fsd_cache_fork(cache, ints(0, 0), refs)
    assert got["block_table"].tolist() == [[39998, 39999], [39998, 0]] and got["refs"][39998] == 2
    check(was, {0: 39999}, {0: 3})
    was = fill()
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    refs[[2, 39998, 39999]] = 1
    got = fsd.fsd_cache_compact(cache, refs)
    assert got["block_table"].tolist() == [[0, 1]] and int(got["used_blocks"]) == 3
    check(was, {0: 39998, 1: 39999})


def test_reorder_rows_beyond_32_bits_of_bytes():
    row = (1 << 30) + 48
    states = torch.randint(0, 256, (1, 6, row // 8), dtype=torch.int64, device="cuda")
    got = fsd.fsd_beam_reorder(states, torch.tensor([[5, -1, 0, 4, 5]], dtype=torch.int32, device="cuda"))["out"]
    for i, w in enumerate((5, None, 0, 4, 5)):
        assert torch.equal(got[0, i], states[0, w] if w is not None else torch.zeros_like(got[0, i])), i


# ------------------------------------------------------------------------------------------ calls beside one another


def _select_args(rng, B=5, W=6, V=40009, dtype="bf16"):
    z, s = _logits(rng, B, W, V, dtype), _scores(rng, B, W)
    return z, s


def test_workspaces_may_hold_anything():
    rng = np.random.default_rng(21)
    z, s = _select_args(rng)
    want = ref.select(_host(z), s, None, None, 9)
    ws = torch.full((fsd.fsd_beam_workspace_bytes(40, 8, 128256, 60, fsd.F32) + 256,), 255, dtype=torch.uint8, device="cuda")
    _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(s), 9, workspace=ws), want)
    fsd.fsd_beam_select(torch.randn((30, 8, 90000), device="cuda"), None, 60, workspace=ws)
    _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(s), 9, workspace=ws), want)
    table, lens, refs = _sequences(rng, 9, 4, 60)
    for fill in (255, 0, 127):
        ws = torch.full((fsd.fsd_cache_fork_workspace_bytes(60, 20) + 256,), fill, dtype=torch.uint8, device="cuda")
        _fork(rng, table, lens, refs, rng.integers(-1, 9, 20).astype(np.int32), None, None, workspace=ws)


def test_smallest_workspaces():
    """the sizes that the library asks for are enough, to the byte"""
    rng = np.random.default_rng(22)
    z, s = _select_args(rng, 3, 4, 5000)
    need = fsd.fsd_beam_workspace_bytes(3, 4, 5000, 7, fsd.BF16)
    arena = torch.full((need + 512,), 99, dtype=torch.uint8, device="cuda")
    at = (-arena.data_ptr()) % 256
    _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(s), 7, workspace=arena[at:at + need]), ref.select(_host(z), s, None, None, 7))
    assert (arena[at + need:] == 99).all() and (arena[:at] == 99).all()
    with pytest.raises(fsd.FsdError):
        fsd.fsd_beam_select(z.cuda(), _dev(s), 7, workspace=arena[at:at + need - 1])
    for P, n, M in ((50, 9, 4), (5000, 9, 4), (2000, 30, 400)):
        table, lens, refs = _sequences(rng, 4, M, P)
        need = fsd.fsd_cache_fork_workspace_bytes(P, n)
        arena = torch.full((need + 512,), 99, dtype=torch.uint8, device="cuda")
        at = (-arena.data_ptr()) % 256
        _fork(rng, table, lens, refs, rng.integers(-1, 4, n).astype(np.int32), None, None, workspace=arena[at:at + need])
        assert (arena[at + need:] == 99).all() and (arena[:at] == 99).all()
        need = fsd.fsd_cache_compact_workspace_bytes(P)
        arena = torch.full((need + 512,), 99, dtype=torch.uint8, device="cuda")
        at = (-arena.data_ptr()) % 256
        cache = _cache(_pages(rng, 1, P, 1, 64), table, lens)
        got = fsd.fsd_cache_compact(cache, _dev(refs), workspace=arena[at:at + need])
        want = ref.compact(table, refs)
        torch.cuda.synchronize()
        assert (_host(got["remap"]) == want[2]).all() and (_host(got["block_table"]) == want[0]).all()
        assert (arena[at + need:] == 99).all() and (arena[:at] == 99).all()


def test_reports_may_be_left_out():
    rng = np.random.default_rng(23)
    z, s = _select_args(rng, 2, 3, 700, "f32")
    new = lambda shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    out = dict(scores=new((2, 5), torch.float32), parent=new((2, 5)), tokens=new((2, 5)))
    got = dict(fsd.fsd_beam_select(z.cuda(), _dev(s), 5, out=out), row_status=torch.zeros(2))
    _same_selection(got, ref.select(_host(z), s, None, None, 5))
    parent = out["parent"]
    fsd.fsd_beam_reorder(z.cuda(), parent, out=dict(out=torch.empty((2, 5, 700), device="cuda")))
    for P, M in ((40, 4), (6000, 4)):
        table, lens, refs = _sequences(rng, 3, M, P)
        cache = _cache(_pages(rng, 1, P, 1, 64), table, lens)
        got = fsd.fsd_cache_fork(cache, _dev(np.array([0, 2], np.int32)), _dev(refs), out=dict(block_table=new((2, M)), cache_len=new(2), refs=new(P)))
        torch.cuda.synchronize()
        want = ref.fork(table, lens, refs, np.array([0, 2]), None, None)
        assert (_host(got["block_table"]) == want[0]).all() and (_host(got["refs"]) == want[2]).all()
        got = fsd.fsd_cache_compact(cache, _dev(refs), out=dict(block_table=new((3, M)), refs=new(P)))
        torch.cuda.synchronize()
        assert (_host(got["refs"]) == ref.compact(table, refs)[1]).all()


def test_two_streams_at_once():
    rng = np.random.default_rng(24)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    calls = [_select_args(rng, 6, 7, 90001) for _ in streams]
    on = [(z.cuda(), _dev(s)) for z, s in calls]
    tables = [_sequences(rng, 20, 5, 300) for _ in streams]
    parents = [rng.integers(-1, 20, 33).astype(np.int32) for _ in streams]
    pages = [_pages(rng, 2, 300, 1, 64) for _ in streams]
    caches = [_cache(p, t[0], t[1]) for p, t in zip(pages, tables)]
    refs, par = [_dev(t[2]) for t in tables], [_dev(p) for p in parents]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            got[i].append((fsd.fsd_beam_select(*on[i], 30, stream=st), fsd.fsd_cache_fork(caches[i], par[i], refs[i], stream=st),
                           fsd.fsd_beam_reorder(on[i][0], par[i][:6].view(6, 1).clamp(0, 6), stream=st)))
    torch.cuda.synchronize()
    for i in range(2):
        want, forked = ref.select(_host(calls[i][0]), calls[i][1], None, None, 30), ref.fork(*tables[i], parents[i], None, None)
        ref.move_pages({k: v.copy() for k, v in pages[i].items()}, pages[i], forked[5])
        _same_pages(caches[i], pages[i])
        for s, f, r in got[i]:
            _same_selection(s, want)
            assert (_host(f["block_table"]) == forked[0]).all() and (_host(f["refs"]) == forked[2]).all()
            assert torch.equal(r["out"][:, 0], on[i][0][torch.arange(6, device="cuda"), par[i][:6].clamp(0, 6).long()])


@pytest.mark.parametrize("P,M", [(200, 5), (6000, 5), (200, 900)])
def test_replays_from_a_graph(P, M):
    """A captured step, replayed with other contents of the same tensors, and eager work in between."""
    rng = np.random.default_rng(P + M)
    B, W, V, n = 4, 3, 70001, 3
    z, s = torch.empty((B, W, V), dtype=torch.bfloat16, device="cuda"), torch.empty((B, W), device="cuda")
    state = torch.randn((2, B, W, 50), device="cuda")
    offset = (torch.arange(B, dtype=torch.int32, device="cuda") * W)[:, None]
    pages = _pages(rng, 1, P, 1, 64)
    cache = _cache(pages, np.full((B * W, M), -1, np.int32), np.zeros(B * W, np.int32))
    refs, room = torch.zeros(P, dtype=torch.int32, device="cuda"), torch.full((B * n,), 9, dtype=torch.int32, device="cuda")

    def step():
        best = fsd.fsd_beam_select(z, s, n)
        states = fsd.fsd_beam_reorder(state, best["parent"], batch_dim=1)
        rows = torch.where(best["parent"] < 0, -1, best["parent"] + offset).view(-1)
        forked = fsd.fsd_cache_fork(cache, rows, refs, room=room)
        packed = fsd.fsd_cache_compact(cache.with_tables(forked["block_table"], forked["cache_len"]), forked["refs"])
        return best, states, forked, packed

    def fill(k):
        g = np.random.default_rng(100 + k)
        z.copy_(_logits(g, B, W, V, "bf16"))
        s.copy_(torch.from_numpy(_scores(g, B, W)))
        table, lens, r = _sequences(g, B * W, M, P, most=min(64 * M - 9, 300))
        cache.block_table.copy_(torch.from_numpy(table))
        cache.cache_len.copy_(torch.from_numpy(lens))
        refs.copy_(torch.from_numpy(r))
        for name, v in pages.items():
            getattr(cache, name).copy_(torch.from_numpy(v))

    fill(0)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = step()
    for k in (1, 2, 3, 1):
        fill(k)
        g.replay()
        torch.cuda.synchronize()
        got = [{name: t.clone() for name, t in part.items() if name != "_workspace"} for part in captured]
        after = {name: getattr(cache, name).clone() for name in pages}
        fill(k)
        eager = step()
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            for name, t in a.items():
                assert torch.equal(t, b[name]), (k, name)
        for name in pages:
            assert torch.equal(after[name].view(torch.uint8), getattr(cache, name).view(torch.uint8)), (k, name)
        _same_selection(eager[0], ref.select(_host(z), _host(s), None, None, n))


def test_streams_of_their_own_memory():
    """`stream`: what the binding allocates stays allocated until that stream has used it"""
    rng = np.random.default_rng(26)
    side = torch.cuda.Stream()
    z, s = _select_args(rng, 3, 4, 20000)
    zd, sd = z.cuda(), _dev(s)
    torch.cuda.synchronize()
    got = fsd.fsd_beam_select(zd, sd, 8, stream=side)
    for _ in range(8):
        torch.full((got["_workspace"].numel(),), 255, dtype=torch.uint8, device="cuda")
    side.synchronize()
    _same_selection(got, ref.select(_host(z), s, None, None, 8))


# ------------------------------------------------------------------------------------------ together


def test_beam_search_over_the_cache():
    """Prompts appended, each continued by beams: attention over the forked cache, the best continuations, histories and pages that follow
    them.  Every beam's pages in the end are those of a sequence that was never forked."""
    rng = np.random.default_rng(30)
    B, W, V, H, G, D, L, P, M = 3, 4, 600, 2, 2, 64, 1, 120, 6
    emb = {k: torch.from_numpy(rng.standard_normal((V, h, D)).astype(np.float32) * 0.7).to(torch.bfloat16).cuda() for k, h in (("q", H * G), ("k", H), ("v", H))}
    head = torch.from_numpy(rng.standard_normal((H * G * D, V)).astype(np.float32) * 0.4).cuda()
    prompts = [rng.integers(0, V, k) for k in (70, 1, 130)]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    def append(cache, tokens, counts):                        # tokens [S, R]: the first counts[s] of them
        t = torch.as_tensor(tokens, dtype=torch.long, device="cuda")
        out = fsd.fsd_cache_append(emb["k"][t].contiguous(), emb["v"][t].contiguous(), cache, ints(counts) - 1)
        assert not out["row_status"].any()
        cache.cache_len.copy_(out["cache_len"])

    def prompt_into(cache, rows):                             # all but a prompt's last token
        R = max(len(p) for p in rows)
        append(cache, [list(p) + [0] * (R - len(p)) for p in rows], [len(p) - 1 for p in rows])

    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    cache = fsd.Cache.empty(L, P, H, D, torch.full((1, M), -1, dtype=torch.int32, device="cuda"), ints([0]))

    def fork(cache, refs, parent, room):
        out = fsd.fsd_cache_fork(cache, ints(parent) if isinstance(parent, list) else parent, refs, room=ints(room))
        assert not out["row_status"].any()
        table = out["block_table"]
        count = torch.bincount(table[table >= 0].long(), minlength=P).int()
        assert torch.equal(out["refs"], count) and int(out["free_blocks"]) == int((count == 0).sum())
        return cache.with_tables(table, out["cache_len"]), out["refs"]

    cache, refs = fork(cache, refs, [-1] * B, [len(p) for p in prompts])
    prompt_into(cache, prompts)
    cache, refs = fork(cache, refs, [b for b in range(B) for _ in range(W)], [1] * (B * W))
    scores = torch.full((B, W), -float("inf"), device="cuda")
    scores[:, 0] = 0.0                                        # the first step has one beam
    history = torch.zeros((B, W, 200), dtype=torch.int32, device="cuda")
    for b, p in enumerate(prompts):
        history[b, :, :len(p)] = ints(p.tolist())
    length = torch.tensor([len(p) for p in prompts], device="cuda")
    last = torch.stack([history[b, :, len(p) - 1] for b, p in enumerate(prompts)])
    offset = (torch.arange(B, dtype=torch.int32, device="cuda") * W)[:, None]
    for _ in range(70):
        t = last.long().view(B * W, 1)
        x = fsd.fsd_attend_chain(emb["q"][t].contiguous(), emb["k"][t].contiguous(), emb["v"][t].contiguous(), cache)
        assert not x["row_status"].any()
        logits = (x["out"].float().view(B, W, -1) @ head).contiguous()
        best = fsd.fsd_beam_select(logits, scores, W)
        want = ref.select(_host(logits), _host(scores), None, None, W)
        _same_selection(best, (*want[:4], max(want[4], 2.0 ** -30)))
        append(cache, last.long().view(B * W, 1), [1] * (B * W))
        cache, refs = fork(cache, refs, (best["parent"] + offset).view(-1).contiguous(), [1] * (B * W))
        scores, last = best["scores"].clone(), best["tokens"].clone()
        history = fsd.fsd_beam_reorder(history, best["parent"])["out"]
        history.scatter_(2, length.view(B, 1, 1).expand(B, W, 1), last[:, :, None])
        length = length + 1
    # put together, and each beam again by itself
    packed = fsd.fsd_cache_compact(cache, refs)
    assert int(packed["used_blocks"]) == int((refs > 0).sum()) and int(packed["block_table"].max()) < int(packed["used_blocks"])
    cache = cache.with_tables(packed["block_table"], cache.cache_len)
    lens = cache.cache_len.tolist()
    for b in range(B):
        for w in range(W):
            tokens = history[b, w, :int(length[b])].tolist()
            n = len(tokens) - 1
            assert lens[b * W + w] == n
            alone = fsd.Cache.empty(L, M, H, D, torch.arange(M, dtype=torch.int32, device="cuda")[None], ints([0]))
            prompt_into(alone, [np.array(tokens[:len(prompts[b])])])
            for x in tokens[len(prompts[b]) - 1:-1]:
                append(alone, [[x]], [1])
            for j in range(-(-n // 64)):
                blk, held = int(cache.block_table[b * W + w, j]), min(64, n - 64 * j)
                assert torch.equal(cache.k_codes[:, blk, :, :held], alone.k_codes[:, j, :, :held])
                v = [c.v_codes[:, e].transpose(-1, -2).reshape(L, H, 64, D)[:, :, :held] for c, e in ((cache, blk), (alone, j))]
                assert torch.equal(*v)
                assert torch.equal(cache.k_scale[:, blk], alone.k_scale[:, j]) and torch.equal(cache.v_scale[:, blk], alone.v_scale[:, j])


def test_a_tree_from_the_selection_is_verified():
    """two levels of a token tree by the selection, verified against the same model: the divergences are 0 and a path of two is accepted"""
    rng = np.random.default_rng(31)
    B, V, first, second = 5, 3000, 4, 7
    root = _logits(rng, B, 1, V, "bf16").cuda()
    level1 = fsd.fsd_beam_select(root, None, first)
    below = _logits(rng, B, first, V, "bf16").cuda()          # the model's rows behind the nodes of the first level
    level2 = fsd.fsd_beam_select(below, level1["scores"], second)
    behind = _logits(rng, B, second, V, "bf16").cuda()
    tokens = torch.cat([level1["tokens"], level2["tokens"]], 1).contiguous()
    parent = torch.cat([torch.full_like(level1["parent"], -1), level2["parent"]], 1).contiguous()
    target = torch.cat([root, below, behind], 1).contiguous()
    draft = torch.cat([fsd.fsd_beam_reorder(root, level1["parent"])["out"], fsd.fsd_beam_reorder(below, level2["parent"])["out"]], 1).contiguous()
    got = fsd.fsd_verify_tree(target, draft, tokens, parent, 3, 0.0, fsd.DIV_JS, fsd.GREEDY)
    torch.cuda.synchronize()
    assert not got["row_status"].any() and (got["divergences"] == 0).all() and (got["path_len"] == 2).all()
    assert torch.equal(got["path_nodes"][:, 1], torch.full_like(got["path_nodes"][:, 1], first))   # the best node of the second level
