"""The operators around drafting on the GPU: numbers at the ends of their ranges, rows of few entries, the merge's other ways, memory of other
streams, and runs of them together."""
import math

import numpy as np
import pytest
import torch

import paper_2502_20704_amd as fsd
from tests import drafting_ref as ref
from tests.test_drafting_gpu import DT, _cache, _dev, _host, _logits, _pages, _same_selection, _select_args, _sequences

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------ normalisers


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,times", [(50, 1), (9002, 1), (100002, 10)])   # (30 long rows a number: by the kernel with the table)
def test_select_rows_of_one_large_number(V, times, dtype):
    """A row is as likely as it is a number higher up or lower down, however large that number is: where a mask of the type's lowest number leaves a beam
    nothing, each of its V entries has the score -log V, and does not stand in front of beams that have something."""
    numbers = [torch.finfo(DT[dtype]).min, -1e30, 2.0 ** 100, -(2.0 ** 60)] * times
    B, n = len(numbers), 8
    z = torch.empty((B, 3, V), dtype=DT[dtype])
    z[:, 0] = torch.tensor(numbers, dtype=DT[dtype])[:, None]
    z[:, 1], z[:, 1, 5:8] = -math.inf, 0.25
    z[:, 2], z[:, 2, ::2] = -math.inf, torch.tensor(numbers, dtype=DT[dtype])[:, None]
    scores = np.array([[-1.0, -1.5, -1.75]] * B, np.float32)
    got = fsd.fsd_beam_select(z.cuda(), _dev(scores), n)
    torch.cuda.synchronize()
    assert not got["row_status"].any()
    # -1.5 - log 3; then -1.75 - log V + log 2 = -1.057 - log V is behind -1 - log V
    assert (_host(got["parent"]) == [1, 1, 1, 0, 0, 0, 0, 0]).all() and (_host(got["tokens"]) == [5, 6, 7, 0, 1, 2, 3, 4]).all()
    want = np.array([-1.5 - math.log(3)] * 3 + [-1.0 - math.log(V)] * 5)
    # one rounding to binary32, and the normaliser's error
    assert (np.abs(_host(got["scores"]) - want) <= 2.0 ** -24 * np.abs(want) * (1 + 2.0 ** -20) + 2.0 ** -32).all()


def test_select_normaliser_within_its_bound():
    """The sum of a row's exponentials is off by less than 2^-33 of it, also where every entry's exponential is formed from a wavefront's largest entry, that
    from the slice's and that from the row's, each at a distance at which the polynomial is off the most.  (Rows beyond the range of e^z; parts of
    256 entries are the wavefronts' of a call of this size.)"""
    V, far = 65536, 218 * 2.0 ** -14                          # a multiple of the numbers' distance there
    z = np.full((V // 1024, 4, 256), 1000.0 - 3 * far)
    z[:, :, 0] += far                                         # a part's largest
    z[:, 0] = -np.inf
    z[:, 0, 0] = 1000.0 - far                                 # a slice's, alone in its part
    z[0, 0, 0] = 1000.0                                       # the row's
    z = z.reshape(1, 1, V).astype(np.float32)
    least = z[0, 0].astype(np.float64) - 1000.0
    norm = math.log(math.fsum(np.exp(least[least > -np.inf]).tolist()))
    scores = np.array([[norm]], np.float32)                   # (so that the result is near 0, and its rounding small)
    got = fsd.fsd_beam_select(_dev(z), _dev(scores), 1)
    want = float(scores[0, 0]) - norm
    assert int(got["tokens"][0, 0]) == 0
    assert abs(float(got["scores"][0, 0]) - want) <= 2.0 ** -33 + 2.0 ** -24 * abs(want) + 2.0 ** -45


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,B", [(40, 4), (9000, 4), (100003, 14)])
def test_select_only_continuations_are_certain(V, B, dtype):
    """A row with one entry gives the beam's score itself, so that it ties with a finished beam of that score and with other such rows: the lowest beam comes
    first, whatever the logits are."""
    rng = np.random.default_rng(V)
    W = 6
    z = torch.full((B, W, V), -math.inf, dtype=DT[dtype])
    at = rng.integers(0, V, (B, W))
    values = rng.standard_normal((B, W)) * 4
    values[1] = rng.standard_normal(W) * 300                  # beyond the table's range, and e^z's
    values[2] = rng.uniform(-1e30, 1e30, W)
    values[3, :3], values[3, 3:] = [0.0, 64.0, -63.5], [1e-30, -2.0 ** -13, 600.0]
    for b in range(B):
        for w in range(W):
            z[b, w, at[b, w]] = float(values[b, w])
    scores = np.full((B, W), -2.3, np.float32)
    done = np.zeros((B, W), np.int32)
    done[0, 2] = done[2, 3] = 1
    for n in (1, 4, 9):
        got = fsd.fsd_beam_select(z.cuda(), _dev(scores), n, done=_dev(done))
        k = min(n, W)
        assert not got["row_status"].any()
        assert (_host(got["parent"])[:, :k] == np.arange(k)).all() and (_host(got["parent"])[:, k:] == -1).all()
        assert (_host(got["tokens"])[:, :k] == np.where(done[:, :k] != 0, -1, at[:, :k])).all()
        assert (_host(got["scores"])[:, :k] == scores[:, :k]).all()
    # (0 is no size to measure an error of 2^-33 by: exactly 0)
    got = fsd.fsd_beam_select(z.cuda(), None, 4)
    assert (got["scores"] == 0.0).all() and (_host(got["parent"]) == np.arange(4)).all()


# ------------------------------------------------------------------------------------------ merging


@pytest.mark.parametrize("W,finished", [(256, 256), (256, 200), (200, 150), (129, 129)])
@pytest.mark.parametrize("n", [1, 3, 15, 100, 128])
def test_select_many_finished_beams(W, finished, n):
    """more finished beams than n, than 128, and as many as there are beams, with equal ranks among them"""
    rng = np.random.default_rng(W + finished + n)
    B, V = 4, 90
    z = _logits(rng, B, W, V, "f32")
    done = np.zeros((B, W), np.int32)
    for b in range(B):
        done[b, rng.permutation(W)[:finished]] = 1
    scores = np.stack([rng.uniform(-12, 0, W), np.full(W, -1.5), rng.integers(-9, 0, W), rng.uniform(-3, 0, W)]).astype(np.float32)
    weights = rng.uniform(0.5, 2.0, (B, W)).astype(np.float32)
    scores[3, ::7] = -np.inf
    for by in (None, weights):
        want = ref.select(_host(z), scores, by, done, n)
        # (equal ranks of finished beams are equal to the last bit; ranks of entries are as far from one another as the assertion says)
        _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(scores), n, weights=_dev(by), done=_dev(done)), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("W,V", [(64, 300), (64, 100), (200, 50), (256, 131)])
def test_select_equal_rows_of_many_beams(W, V, dtype):
    """rows that are equal from beam to beam: more equal ranks than the merge orders at once, in its kernel for lists that go deep"""
    n = 128
    steps = torch.arange(V) // 8 / 4.0
    z = torch.stack([torch.zeros(V), -steps, steps, steps % 3.0]).to(DT[dtype])[:, None].expand(4, W, V).contiguous()
    scores = np.zeros((4, W), np.float32)
    done = np.zeros((4, W), np.int32)
    done[:, 5:W // 2] = 1                                     # (rank 0: in front of all entries)
    for d in (None, done):
        want = ref.select(_host(z), scores, None, d, n)
        _same_selection(fsd.fsd_beam_select(z.cuda(), _dev(scores), n, done=_dev(d)), (*want[:4], np.inf))


# ------------------------------------------------------------------------------------------ memory


def _calls():
    """name -> a call that takes a stream (its inputs are there: no stream has work on them), and the outputs that it is known by"""
    rng = np.random.default_rng(41)
    z, s = _select_args(rng, 6, 7, 90001)
    small, large = (z[:2].cuda(), _dev(s[:2])), (z.cuda(), _dev(s))
    P, M = 6000, 12
    table, lens, refs = _sequences(rng, 40, M, P)
    cache, refs = _cache(_pages(rng, 1, P, 1, 64), table, lens), _dev(refs)
    parent = _dev(rng.integers(-1, 40, 90).astype(np.int32))
    best, counts = parent[:6].view(6, 1).clamp(-1, 6), refs.clone()
    one = dict(out=torch.empty((6, 50), device="cuda"), parent=torch.empty((6, 50), dtype=torch.int32, device="cuda"))
    given = dict(scores=one["out"], parent=one["parent"], tokens=torch.empty_like(one["parent"]))
    torch.cuda.synchronize()
    return {
        "select": (lambda stream: fsd.fsd_beam_select(*small, 2, stream=stream), ("scores", "parent", "tokens")),
        "select_large": (lambda stream: fsd.fsd_beam_select(*large, 50, stream=stream), ("scores", "parent", "tokens")),
        "select_into": (lambda stream: fsd.fsd_beam_select(*large, 50, out=dict(given), stream=stream), ("scores", "parent", "tokens")),
        "fork": (lambda stream: fsd.fsd_cache_fork(cache, parent, refs, stream=stream), ("block_table", "cache_len", "refs")),
        "reorder": (lambda stream: fsd.fsd_beam_reorder(large[0], best, stream=stream), ("out",)),
        "compact": (lambda stream: fsd.fsd_cache_compact(cache, counts, stream=stream), ("block_table", "remap")),
    }


def _sizes(got):
    return sorted({t.untyped_storage().nbytes() for t in got.values()})


@pytest.mark.parametrize("name", ["select", "select_large", "select_into", "fork", "reorder"])
def test_memory_of_a_call_on_another_stream_is_not_given_out(name):
    """What the binding makes for a call of `stream` is not given out on the current one before the call is over, also where its caller has dropped the workspace."""
    run, known = _calls()[name]
    side = torch.cuda.Stream()
    want = {k: v.clone() for k, v in run(None).items() if k in known}
    sizes = _sizes(run(None))
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = {k: v for k, v in run(side).items() if k in known}      # (the workspace goes)
    held = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(6)]
    torch.cuda.current_stream().synchronize()
    side.synchronize()
    assert held and all(torch.equal(got[k], want[k]) for k in known)


@pytest.mark.parametrize("name", ["select", "select_large", "select_into", "fork", "reorder", "compact"])
def test_a_call_on_another_stream_leaves_the_current_streams_memory(name):
    """What the binding makes for a call of `stream` is not memory that the current stream has given back and still has work on."""
    run, _ = _calls()[name]
    side = torch.cuda.Stream()
    sizes = _sizes(run(None))
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(6)]
    kept = [torch.zeros_like(t) for t in held]
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    for a, b in zip(held, kept):
        b.copy_(a)
    del held, a                                                   # given back while the copies are under way
    got = run(side)
    torch.cuda.synchronize()
    assert got is not None and all((t == 7).all() for t in kept)


# ------------------------------------------------------------------------------------------ together


def test_another_table_over_the_same_pages():
    """with_tables shares codes and scales and replaces table and lengths"""
    rng = np.random.default_rng(44)
    cache = _cache(_pages(rng, 2, 9, 1, 64), np.array([[3, 1]], np.int32), np.array([70], np.int32))
    table, lens = _dev(np.array([[5, -1, -1], [3, 1, 0]], np.int32)), _dev(np.array([64, 100], np.int32))
    other = cache.with_tables(table, lens)
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        assert getattr(other, name) is getattr(cache, name)
    assert other.block_table is table and other.cache_len is lens and (other.batch, other.max_blocks, other.num_blocks) == (2, 3, 9)
    assert cache.block_table.shape == (1, 2)                  # (as it was)
    want = ref.fork(_host(table), _host(lens), np.ones(9, np.int32), np.array([1, 0]), None, None)
    got = fsd.fsd_cache_fork(other, _dev(np.array([1, 0], np.int32)), torch.ones(9, dtype=torch.int32, device="cuda"))
    assert (_host(got["block_table"]) == want[0]).all() and (_host(got["cache_len"]) == want[1]).all()
    with pytest.raises(ValueError):
        cache.with_tables(table, lens[:1].contiguous())


def test_a_tree_is_made_verified_and_appended():
    """A tree of two levels by the selection; the path that the verify call accepts is appended to a forked cache as the same tokens in a row are to another."""
    rng = np.random.default_rng(45)
    B, V, first, second, H, D, P, M = 5, 3000, 4, 7, 2, 64, 40, 3
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    root, below, behind = (_logits(rng, B, k, V, "bf16").cuda() for k in (1, first, second))
    level1 = fsd.fsd_beam_select(root, None, first)
    level2 = fsd.fsd_beam_select(below, level1["scores"], second)
    tokens = torch.cat([level1["tokens"], level2["tokens"]], 1).contiguous()
    parent = torch.cat([torch.full_like(level1["parent"], -1), level2["parent"]], 1).contiguous()
    target = torch.cat([root, below, behind], 1).contiguous()
    draft = torch.cat([fsd.fsd_beam_reorder(root, level1["parent"])["out"], fsd.fsd_beam_reorder(below, level2["parent"])["out"]], 1).contiguous()
    found = fsd.fsd_verify_tree(target, draft, tokens, parent, 3, 0.0, fsd.DIV_JS, fsd.GREEDY)
    assert (found["path_len"] == 2).all()

    emb = torch.from_numpy(rng.standard_normal((V, H, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    rows = emb[torch.cat([tokens[:, :1] * 0, tokens], 1).long()].contiguous()         # the token before (0) and the nodes
    empty = fsd.Cache.empty(1, P, H, D, torch.full((1, M), -1, dtype=torch.int32, device="cuda"), ints([0]))
    begun = fsd.fsd_cache_fork(empty, ints([-1] * B), torch.zeros(P, dtype=torch.int32, device="cuda"), room=ints([3] * B))
    made = empty.with_tables(begun["block_table"], begun["cache_len"])
    out = fsd.fsd_cache_append(rows, rows, made, found["path_len"], path_nodes=found["path_nodes"])
    assert not out["row_status"].any() and (out["cache_len"] == 3).all()

    nodes = found["path_nodes"][:, :2].long()
    chain = rows.gather(1, torch.cat([nodes[:, :1] * 0, nodes + 1], 1)[:, :, None, None].expand(B, 3, H, D)).contiguous()
    alone = fsd.Cache.empty(1, B, H, D, torch.arange(B, dtype=torch.int32, device="cuda")[:, None], torch.zeros(B, dtype=torch.int32, device="cuda"))
    assert not fsd.fsd_cache_append(chain, chain, alone, ints([2] * B))["row_status"].any()
    at = made.block_table[:, 0].long()
    assert torch.equal(made.k_codes[:, at, :, :3], alone.k_codes[:, :, :, :3]) and torch.equal(made.k_scale[:, at], alone.k_scale)
    assert torch.equal(made.v_codes[:, at, :, 0, :, :3], alone.v_codes[:, :, :, 0, :, :3]) and torch.equal(made.v_scale[:, at], alone.v_scale)
