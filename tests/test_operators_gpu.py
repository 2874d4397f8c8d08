"""The operators around a verify call on the GPU, against plain 64-bit implementations (operators_ref.py)."""
import numpy as np
import pytest
import torch

import paper_2502_20704_amd as fsd
from tests import operators_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _host(t):
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def _rand_parents(rng, B, N, deep=False):
    p = np.empty((B, N), dtype=np.int32)
    for b in range(B):
        for j in range(N):
            p[b, j] = rng.integers(max(-1, j - 3) if deep else -1, j)
    return p


def _close(got, want, err, dtype, what=""):
    """within `err` before the last rounding, which is off by half a step; non-finite values equal"""
    got = _host(got)
    assert got.shape == want.shape
    fine = np.isfinite(want)
    assert (np.isfinite(got) == fine).all(), f"{what}: finite places differ"
    assert (np.isnan(got) == np.isnan(want)).all() and (got[~fine & ~np.isnan(want)] == want[~fine & ~np.isnan(want)]).all(), what
    d = np.abs(got[fine] - want[fine])
    bound = err[fine] * (1 + ref.HALF_STEP[dtype]) + ref.HALF_STEP[dtype] * np.abs(want[fine]) + 2.0 ** -140
    assert (d <= bound).all(), f"{what}: off by {(d / np.maximum(bound, 1e-300)).max():.2f} bounds"


# ------------------------------------------------------------------------------------------ conditioning


def _conditions(rng, B, V, contexts, *, history=0, biases=0, mask=None, bad_ids=False, few=None):
    few = few or V
    c = dict.fromkeys(("history", "history_len", "prompt_len", "repetition", "presence", "frequency", "bias_tokens", "bias_values", "allowed"))
    if history:
        c["history"] = rng.integers(-2 if bad_ids else 0, few + (3 if bad_ids and few == V else 0), (B, history)).astype(np.int32)
        c["history_len"] = rng.integers(0, history + 1, B).astype(np.int32)
        c["prompt_len"] = rng.integers(0, history + 1, B).astype(np.int32)
        if B > 1:
            c["history_len"][0], c["prompt_len"][0] = history + 5, -3         # taken as within the list
    c["repetition"] = rng.uniform(0.5, 2.0, B).astype(np.float32)
    c["presence"] = rng.uniform(-1.0, 2.0, B).astype(np.float32)
    c["frequency"] = rng.uniform(-0.5, 1.0, B).astype(np.float32)
    if biases:
        c["bias_tokens"] = rng.integers(-2, few, (B, biases)).astype(np.int32)
        c["bias_values"] = (rng.standard_normal((B, biases)) * 4).astype(np.float32)
    if mask:
        n = contexts if mask == "contexts" else 1
        w = rng.integers(0, 1 << 32, (B, n, (V + 31) // 32), dtype=np.uint64).astype(np.uint32)
        w[:, ::3] &= rng.integers(0, 1 << 32, w[:, ::3].shape, dtype=np.uint64).astype(np.uint32)
        w[0, n - 1] = 0                                                        # nothing is allowed
        c["allowed"] = w.view(np.int32)
    return c


def _dev(c):
    return fsd.Conditions(**{k: torch.from_numpy(v).cuda() if v is not None else None for k, v in c.items()})


CONDITION = [
    # B, N, V, dtype, tree, target, history, biases, mask
    (1, 0, 1, "f32", False, True, 0, 0, None),
    (2, 0, 31, "bf16", False, True, 5, 3, "sequence"),
    (1, 1, 32000, "bf16", False, True, 700, 0, None),
    (3, 4, 4097, "bf16", False, True, 100, 9, "contexts"),
    (3, 4, 4097, "f32", False, False, 100, 9, "contexts"),
    (2, 16, 12291, "f32", False, True, 3000, 300, "sequence"),
    (2, 3, 5, "f32", False, True, 40, 7, "contexts"),
    (2, 7, 7, "bf16", True, True, 40, 7, "contexts"),
    (3, 13, 8200, "bf16", True, True, 100, 0, "contexts"),
    (3, 13, 8199, "bf16", True, False, 100, 5, "contexts"),
    (1, 60, 33000, "f32", True, False, 64, 0, "contexts"),
    (1, 200, 2050, "f32", True, True, 10, 0, None),
    (5, 8, 1000, "bf16", True, False, 0, 0, "sequence"),
    (40, 2, 9000, "bf16", False, True, 33, 0, None),
]


@pytest.mark.parametrize("B,N,V,dtype,tree,target,history,biases,mask", CONDITION)
@pytest.mark.parametrize("in_place", [False, True])
def test_condition(B, N, V, dtype, tree, target, history, biases, mask, in_place):
    rng = np.random.default_rng(B * 1000 + N * 100 + V)
    rows = N + 1 if target else N
    z = torch.from_numpy((rng.standard_normal((B, rows, V)) * 3).astype(np.float32)).to(DT[dtype])
    z[0, 0, :: 7] = -float("inf")
    z[0, rows - 1, 0] = 0.0
    tokens = rng.integers(-1, min(V, 50), (B, N)).astype(np.int32)      # candidates that repeat one another, and one that is none
    parent = _rand_parents(rng, B, N, deep=True) if tree else None
    if tree and N > 4:
        parent[0, 3], parent[0, 4] = 3, -7                                # malformed: children of the root
    c = _conditions(rng, B, V, N + 1, history=history, biases=biases, mask=mask, bad_ids=True, few=min(V, 60))
    want, err = ref.condition(_host(z), tokens, parent, target, c)
    zd = z.cuda()
    out = dict(out=zd if in_place else torch.full_like(zd, 7.0))
    if tree:
        got = fsd.fsd_condition_tree(zd, torch.from_numpy(tokens).cuda(), torch.from_numpy(parent).cuda(), _dev(c), out=out)["out"]
    else:
        got = fsd.fsd_condition_chain(zd, torch.from_numpy(tokens).cuda() if N else None, _dev(c), out=out)["out"]
    torch.cuda.synchronize()
    _close(got, want, err, DT[dtype])
    same = (err == 0) & ~np.isneginf(want)                                # what nothing touches keeps its bits
    assert (_host(got)[same] == _host(z)[same]).all()
    if not in_place:
        assert torch.equal(zd.cpu(), z)


def test_condition_without_conditions_copies():
    z = torch.randn(2, 4, 1003, device="cuda")
    z[0, 0, 0], z[1, 3, 1002] = float("nan"), float("inf")
    got = fsd.fsd_condition_chain(z, torch.zeros((2, 3), dtype=torch.int32, device="cuda"), fsd.Conditions())["out"]
    assert torch.equal(got.view(torch.int32), z.view(torch.int32))


def test_condition_masked_places_hold_anything():
    """A NaN or an infinity in a masked place does not come through; elsewhere it does."""
    V = 300
    z = torch.zeros(1, 1, V, device="cuda")
    z[0, 0, 0], z[0, 0, 1], z[0, 0, 2], z[0, 0, 299] = float("nan"), float("inf"), float("nan"), float("inf")
    w = torch.zeros((1, 1, 10), dtype=torch.int32, device="cuda")
    w[0, 0, 0] = 0b1100
    hist = torch.tensor([[0, 1, 2, 299]], dtype=torch.int32, device="cuda")
    got = fsd.fsd_condition_chain(z, None, fsd.Conditions(allowed=w, history=hist, repetition=torch.full((1,), 2.0, device="cuda")))["out"].cpu()
    assert torch.isnan(got[0, 0, 2]) and got[0, 0, 3] == 0
    assert (got[0, 0, [0, 1, 4, 299]] == -float("inf")).all()


def test_condition_long_chain_and_deep_tree():
    """The most candidates a call takes; a tree that is a chain gives the chain's result."""
    rng = np.random.default_rng(5)
    N, V = 2048, 203
    z = torch.from_numpy(rng.standard_normal((1, N + 1, V)).astype(np.float32)).cuda()
    tokens = torch.from_numpy(rng.integers(0, V, (1, N)).astype(np.int32)).cuda()
    c = fsd.Conditions(frequency=torch.full((1,), 0.01, device="cuda"), presence=torch.full((1,), 0.5, device="cuda"))
    chain = fsd.fsd_condition_chain(z, tokens, c)["out"]
    parent = torch.arange(-1, N - 1, dtype=torch.int32, device="cuda")[None]
    tree = fsd.fsd_condition_tree(z, tokens, parent, c)["out"]
    assert torch.equal(chain, tree)
    count = torch.nn.functional.one_hot(tokens[0].long().cpu(), V).cumsum(0).double().numpy()
    want = _host(z)[0, 1:] - 0.01 * count - 0.5 * (count > 0)
    _close(chain[0, 1:], want, 5 * 2.0 ** -24 * (np.abs(_host(z)[0, 1:]) + 0.02 * count + 0.5), torch.float32)


def test_condition_unaligned_base_and_verify_agree():
    """Rows that begin in the middle of a word; the result is what a verify call takes."""
    rng = np.random.default_rng(9)
    B, K, V = 2, 3, 1001
    buf = torch.zeros(B * (K + 1) * V + 1, dtype=torch.bfloat16, device="cuda")
    z = buf[1:].view(B, K + 1, V)
    z.copy_(torch.from_numpy(rng.standard_normal((B, K + 1, V))).cuda())
    c = _conditions(rng, B, V, K + 1, history=50, biases=4, mask="sequence", few=100)
    c["allowed"][:] = -1
    tokens = rng.integers(0, V, (B, K)).astype(np.int32)
    want, err = ref.condition(_host(z), tokens, None, True, c)
    dt = torch.from_numpy(tokens).cuda()
    got = fsd.fsd_condition_chain(z, dt, _dev(c))["out"]
    _close(got, want, err, torch.bfloat16)
    draft = got[:, :K].contiguous()
    v = fsd.fsd_verify_chain(got, draft, dt, 0.0, mode=fsd.GREEDY)
    assert (v["accept_len"] == K).all() and (v["out_tokens"][:, K] == got[:, K].float().argmax(1)).all()


# ------------------------------------------------------------------------------------------ the cache


def _turns(rows, dim):
    if dim == 0:
        return None
    freq = 10000.0 ** (-np.arange(0, dim, 2) / dim)
    a = np.arange(rows)[:, None] * freq
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def _rotation(turns, halves):
    return None if turns is None else fsd.Rotation(torch.from_numpy(turns).cuda(), fsd.ROPE_HALVES if halves else fsd.ROPE_PAIRS)


def _random_cache(rng, L, P, H, D, table, lens, top=0x7F):
    """every code but the NaNs, and what lies behind the lengths is NaN"""
    kc = rng.integers(0, top, (L, P, H, 64, D)).astype(np.uint8) | (rng.integers(0, 2, (L, P, H, 64, D)) << 7).astype(np.uint8)
    vc = rng.integers(0, top, (L, P, H, 4, D, 16)).astype(np.uint8) | (rng.integers(0, 2, (L, P, H, 4, D, 16)) << 7).astype(np.uint8)
    c = dict(k_codes=kc, v_codes=vc, k_scale=np.exp2(rng.integers(-9, -5, (L, P, H))).astype(np.float32),
             v_scale=np.exp2(rng.integers(-9, -5, (L, P, H))).astype(np.float32))
    for b, n in enumerate(lens):
        if n % 64 and table.shape[1] > n // 64:
            i = table[b, n // 64]
            kc[:, i, :, n % 64:] = 0x7F
            vc.transpose(0, 1, 2, 3, 5, 4).reshape(L, P, H, 64, D)  # (a copy: the places are set below)
            for t in range(n % 64, 64):
                vc[:, i, :, t // 16, :, t % 16] = 0xFF
    return c


def _to_cache(c, table, lens):
    return fsd.Cache(*(torch.from_numpy(c[k]).cuda() for k in ("k_codes", "v_codes", "k_scale", "v_scale")),
                     torch.from_numpy(table).cuda(), torch.from_numpy(np.asarray(lens, dtype=np.int32)).cuda())


def _tables(rng, B, per, extra=3):
    at = rng.permutation(B * per + extra)[:B * per]
    return at.reshape(B, per).astype(np.int32), B * per + extra


ATTEND = [
    # lens, R, heads, kv_heads, D, dtype, tree, turn, halves
    ([0], 1, 1, 1, 64, "bf16", False, 0, True),
    ([1, 63, 64, 65], 1, 8, 2, 128, "bf16", False, 128, True),
    ([129, 0, 700], 5, 8, 2, 128, "f16", False, 64, False),
    ([300, 1], 9, 4, 1, 64, "bf16", False, 64, True),                      # 36 rows: 3 tiles
    ([257, 64], 4, 16, 1, 128, "f16", False, 32, True),                    # 64 rows: 4 tiles
    ([130, 5], 17, 7, 1, 128, "bf16", False, 128, True),                   # 119 rows, more than one tile of the fours
    ([70, 511], 65, 10, 2, 64, "f16", False, 64, False),                   # rows of two tails
    ([70, 200], 130, 4, 2, 128, "bf16", False, 128, True),
    ([100, 0], 3, 8, 4, 256, "bf16", False, 256, True),
    ([65, 300], 20, 4, 2, 256, "f16", False, 128, False),
    ([65, 90], 40, 8, 2, 256, "bf16", False, 256, True),
    ([33, 128, 0], 14, 8, 4, 128, "bf16", True, 128, True),
    ([200, 10], 61, 8, 2, 128, "f16", True, 128, True),
    ([63, 1], 150, 3, 3, 64, "bf16", True, 64, False),
    ([4000], 2, 4, 1, 128, "bf16", False, 128, True),                      # many pieces
    ([3000, 10, 900], 6, 6, 2, 64, "f16", True, 64, True),
]


@pytest.mark.parametrize("lens,R,heads,kv_heads,D,dtype,tree,turn,halves", ATTEND)
def test_attend(lens, R, heads, kv_heads, D, dtype, tree, turn, halves):
    rng = np.random.default_rng(sum(lens) + R * 7 + D)
    B, dt = len(lens), DT[dtype]
    table, P = _tables(rng, B, max(1, (max(lens) + 63) // 64))
    c = _random_cache(rng, 2, P, kv_heads, D, table, lens, top=0x70)
    mixed = torch.from_numpy(rng.standard_normal((B, R, heads + 2 * kv_heads, D)) * 0.7).to(dt).cuda()
    q, k, v = mixed[:, :, :heads], mixed[:, :, heads:heads + kv_heads], mixed[:, :, heads + kv_heads:]
    parent = _rand_parents(rng, B, R - 1, deep=True) if tree else None
    turns = _turns(max(lens) + R, turn)
    rows = rng.integers(0, R + 1, B).astype(np.int32)
    rows[0] = R
    cache = _to_cache(c, table, lens)
    for count in (None, rows):
        out = dict(out=torch.full((B, R, heads, D), 7.0, dtype=dt, device="cuda"), row_status=torch.full((B,), -1, dtype=torch.int32, device="cuda"))
        more = dict(layer=1, rotation=_rotation(turns, halves), out=out, scale=0.11, row_count=torch.from_numpy(count).cuda() if count is not None else None)
        if tree:
            fsd.fsd_attend_tree(q, k, v, torch.from_numpy(parent).cuda(), cache, **more)
        else:
            fsd.fsd_attend_chain(q, k, v, cache, **more)
        torch.cuda.synchronize()
        n = count if count is not None else np.full(B, R)
        want, bound = ref.attend(_host(q), _host(k), _host(v), parent, n, c, 1, lens, table, 0.11, turns, halves, dt)
        got = _host(out["out"])
        assert (out["row_status"].cpu().numpy() == 0).all()
        for b in range(B):
            d = np.abs(got[b, :n[b]] - want[b, :n[b]])
            assert np.isfinite(got[b, :n[b]]).all()
            assert (d <= bound[b, :n[b]]).all(), f"sequence {b}: {(d / np.maximum(bound[b, :n[b]], 1e-30)).max():.2f} bounds"
            assert (got[b, n[b]:] == 7.0).all(), "rows behind the last were written"


# ------------------------------------------------------------------------------------------ appending

APPEND = [
    # counts, lens, R, kv_heads, D, dtype, layers, tree, turn, halves
    ([1], [0], 1, 1, 64, "bf16", 1, False, 0, True),
    ([1, 1, 1, 1], [0, 63, 64, 100], 1, 2, 128, "bf16", 1, False, 128, True),
    ([0, 5, 9, 3], [10, 60, 120, 0], 9, 2, 128, "f16", 3, False, 64, False),
    ([4, 1, 3], [62, 128, 13], 14, 3, 64, "f32", 2, True, 64, True),
    ([6, 2], [61, 5], 40, 2, 256, "bf16", 2, True, 256, True),
    ([70, 200, 0, 64], [0, 30, 64, 1], 200, 2, 128, "bf16", 1, False, 128, True),
    ([130, 17], [63, 127], 130, 1, 256, "f32", 2, False, 128, False),
    ([33, 20], [5, 40], 33, 4, 64, "f16", 1, False, 16, True),
]


@pytest.mark.parametrize("big", [False, True])
@pytest.mark.parametrize("counts,lens,R,H,D,dtype,L,tree,turn,halves", APPEND)
def test_append(counts, lens, R, H, D, dtype, L, tree, turn, halves, big):
    """big: what is appended is larger than what the blocks hold, so that their codes are rounded again."""
    rng = np.random.default_rng(sum(lens) + R * 3 + D + big)
    B, dt = len(lens), DT[dtype]
    table, P = _tables(rng, B, (max(n + c for n, c in zip(lens, counts)) + 63) // 64 + 1)
    c = _random_cache(rng, L, P, H, D, table, lens)
    mixed = torch.from_numpy(rng.standard_normal((L, B, R, 2 * H + 1, D)) * (30.0 if big else 0.02)).to(dt).cuda()
    k, v = mixed[:, :, :, :H], mixed[:, :, :, H:2 * H]
    path, paths = None, [list(range(n)) for n in counts]
    if tree:
        path = np.full((B, 9), -1, dtype=np.int32)
        for b, n in enumerate(counts):
            path[b, :n - 1] = np.sort(rng.choice(R - 1, n - 1, replace=False))
            paths[b] = [0] + [int(j) + 1 for j in path[b, :n - 1]]
    turns = _turns(512, turn)
    cache = _to_cache(c, table, lens)
    got = fsd.fsd_cache_append(k, v, cache, torch.tensor([n - 1 for n in counts], dtype=torch.int32, device="cuda"),
                               path_nodes=torch.from_numpy(path).cuda() if tree else None, rotation=_rotation(turns, halves))
    torch.cuda.synchronize()
    assert (got["row_status"].cpu().numpy() == 0).all()
    assert got["cache_len"].tolist() == [n + m for n, m in zip(lens, counts)]
    kh, vh = _host(k), _host(v)
    want = {n: a.copy() for n, a in c.items()}
    new_k, new_v = cache.k_codes.cpu().numpy(), cache.v_codes.cpu().numpy()
    ks, vs = cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy()
    touched = set()
    for b in range(B):
        for i in range((lens[b] + 0) // 64, (lens[b] + counts[b] - 1) // 64 + 1 if counts[b] else 0):
            lo, hi = max(lens[b], 64 * i), min(lens[b] + counts[b], 64 * i + 64)
            if lo >= hi:
                continue
            rows, fill, at = [paths[b][t - lens[b]] for t in range(lo, hi)], lo - 64 * i, table[b, i]
            touched.add(int(at))
            for layer in range(L):
                for h in range(H):
                    x = ref.turned(kh[layer, b, rows, h], turns, np.arange(lo, hi), halves)
                    y = vh[layer, b, rows, h]
                    old = dict(k=ref.block_keys(c["k_codes"][layer, at, h]), v=ref.block_values(c["v_codes"][layer, at, h]))
                    now = dict(k=ref.block_keys(new_k[layer, at, h]), v=ref.block_values(new_v[layer, at, h]))
                    for name, val, scales in (("k", x, ks), ("v", y, vs)):
                        s, s_old = ref.block_scale(val), float(c[name + "_scale"][layer, at, h])
                        s = max(s, s_old) if fill else s
                        # (a rotated key is off by 3 roundings of 2^-24: its largest does not lie that near a border in these inputs)
                        assert scales[layer, at, h] == s, (name, b, i)
                        g = now[name]
                        assert np.array_equal(g[:fill], ref.nearest_code_value(old[name][:fill] * s_old / s) if fill else g[:0])
                        if name == "v" or turns is None:
                            assert np.array_equal(g[fill:fill + hi - lo], ref.nearest_code_value(val / s))
                        else:
                            # half a step of e4m3, 2^-4 of the value or 2^-10 s at the low end, and the rotation's own error
                            off = np.abs(g[fill:fill + hi - lo] * s - val)
                            size = np.abs(val) + np.abs(kh[layer, b, rows, h]) * 2
                            assert (off <= np.maximum(2.0 ** -4 * np.abs(val), 2.0 ** -10 * s) * (1 + 2.0 ** -20) + 3 * 2.0 ** -24 * np.maximum(size, np.abs(kh[layer, b, rows, h]).max(-1, keepdims=True) * 2)).all()
                        # what lies behind is left as it was
                        if name == "k":
                            assert np.array_equal(new_k[layer, at, h, fill + hi - lo:], c["k_codes"][layer, at, h, fill + hi - lo:])
                        else:
                            a = np.swapaxes(new_v[layer, at, h], -1, -2).reshape(64, D)[fill + hi - lo:]
                            assert np.array_equal(a, np.swapaxes(c["v_codes"][layer, at, h], -1, -2).reshape(64, D)[fill + hi - lo:])
    rest = [i for i in range(P) if i not in touched]
    for name, a in (("k_codes", new_k), ("v_codes", new_v), ("k_scale", ks), ("v_scale", vs)):
        assert np.array_equal(a[:, rest], c[name][:, rest]), name
