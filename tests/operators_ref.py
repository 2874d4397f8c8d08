"""Plain 64-bit implementations of the operators around a verify call (numpy, from their definitions in include/fsd.h) and the
bounds their tests use."""
import numpy as np
import torch

BLOCK, GROUP = 64, 16
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def way(parent, j):
    """nodes on the way to node j, itself included; a parent outside [-1, j) counts as -1"""
    out = []
    while j >= 0:
        out.append(j)
        p = int(parent[j])
        j = p if -1 <= p < j else -1
    return out[::-1]


def condition(logits, tokens, parent, target, c):
    """logits float64 [B,rows,V]; c: a dict of numpy arrays (or None) named as in fsd.Conditions -> (result, error of 32-bit
    arithmetic allowed for, before the last rounding).  Five operations, each off by 2^-24 of the magnitudes that meet in it."""
    B, rows, V = logits.shape
    out, err = np.empty_like(logits), np.zeros_like(logits)
    N = tokens.shape[1]
    for b in range(B):
        def per(name, d):
            return float(c[name][b]) if c.get(name) is not None else d
        r_, f_, p_ = per("repetition", 1.0), per("frequency", 0.0), per("presence", 0.0)
        prompt, said = np.zeros(V), np.zeros(V)
        if c.get("history") is not None:
            h = c["history"][b]
            n = max(0, min(int(per("history_len", len(h))), len(h)))
            k = max(0, min(int(per("prompt_len", 0)), n))
            for part, to in ((h[:k], prompt), (h[k:n], said)):
                ok = part[(part >= 0) & (part < V)]
                np.add.at(to, ok, 1.0)
        bias = np.zeros(V)
        if c.get("bias_tokens") is not None:
            for t, x in zip(c["bias_tokens"][b], c["bias_values"][b]):
                if 0 <= t < V:
                    bias[t] = x                                   # of equal ids the last counts
        for r in range(rows):
            if parent is None:
                nodes, context = list(range(min(r, N))), r
            else:
                last = r - 1 if target else int(parent[b][r])
                if not target and not -1 <= last < r:
                    last = -1
                nodes, context = way(parent[b], last), last + 1
            count = said.copy()
            for j in nodes:
                if 0 <= tokens[b, j] < V:
                    count[tokens[b, j]] += 1
            z = logits[b, r].copy()
            hit = (prompt + count) > 0
            with np.errstate(invalid="ignore"):
                pos, neg = hit & (z > 0), hit & ~(z > 0)
                z[pos] /= r_
                z[neg] *= r_
                size = np.abs(z) + abs(f_) * count + abs(p_) + np.abs(bias)
                z = np.where(count > 0, z - f_ * count - p_ * (count > 0), z)
                z = z + bias
            touched = hit | (bias != 0)
            e = np.where(touched & np.isfinite(size), 5 * 2.0 ** -24 * size, 0.0)
            if c.get("allowed") is not None:
                w = c["allowed"][b, context if c["allowed"].shape[1] > 1 else 0].astype(np.int64)
                v = np.arange(V)
                no = (w[v // 32] >> (v % 32)) & 1 == 0
                z[no], e[no] = -np.inf, 0.0
            out[b, r], err[b, r] = z, e
    return out, err


def turned(x, table, pos, halves):
    """x float64 [..., D] at integer positions pos [...]"""
    if table is None:
        return x
    n = table.shape[1] // 2
    t = table[np.clip(pos, 0, table.shape[0] - 1)].astype(np.float64)
    c, s = t[..., :n], t[..., n:]
    y = x.copy()
    lo, hi = (slice(0, n), slice(n, 2 * n)) if halves else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y[..., lo] = x[..., lo] * c - x[..., hi] * s
    y[..., hi] = x[..., hi] * c + x[..., lo] * s
    return y


def code_values(codes):
    """values of e4m3 codes (uint8), from the format's definition"""
    codes = codes.astype(np.int64)
    sign, e, m = np.where(codes & 128, -1.0, 1.0), (codes >> 3) & 15, codes & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e.astype(np.float64) - 10))
    return np.where((codes & 127) == 127, np.nan, sign * v)


def nearest_code_value(y):
    """y (|y| <= 448 but for rounding) as the nearest e4m3 value, ties to even; NaN where y is not finite"""
    y = np.asarray(y, dtype=np.float64)
    a = np.where(np.isfinite(y), np.abs(y), 1.0)
    unit = np.exp2(np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    v = np.sign(y) * np.minimum(np.rint(a / unit) * unit, 448.0)
    return np.where(np.isfinite(y), v, np.nan)


def block_scale(x):
    a = np.abs(x[np.isfinite(x)])
    most = float(a.max()) if a.size else 0.0
    e = -100
    while most > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def block_keys(k_codes):
    """[..., 64, D] codes -> values"""
    return code_values(k_codes)


def block_values(v_codes):
    """[..., 4, D, 16] codes -> values [..., 64, D]"""
    v = code_values(v_codes)
    return np.swapaxes(v, -1, -2).reshape(*v.shape[:-3], BLOCK, v.shape[-2])


def attend(q, k, v, parent, rows, cache, layer, lens, table, scale, turns, halves, dtype, left_out=(), by_contribution=False):
    """(out [B,R,heads,D], bound) in 64 bits; left_out: (sequence, block of it) pairs none of whose tokens counts.  cache: dict of numpy arrays as fsd.Cache names them.

    The bound: a product's error is scale * sum |q||k| times (one rounding of q to 11 bits, for the rows' keys one of k as well,
    4 more of 2^-24 each for the rotation of either, D sums of 2^-24), delta for the row's largest.  Weights then lie within
    exp(+-delta), so their shares within exp(+-2 delta); their rounding to 11 bits and the exponential's and sums' own errors (under 2^-14
    together) come on top, all relative to sum w |v|; a weight under 2^-24 of the row's largest is lost to binary16 (2^-24 of max |v|
    each).  Last the rounding to the result's type.

    by_contribution: where value scales lie far apart, max |v| says little.  A token's weight times its block's value scale is what binary16
    holds, 2^7 or more for the largest of them: what is lost is at most 2^-32 of the largest such product, times codes of up to 512, a
    token.  The sum of weights loses at most 2^-26 a token: 2^-25 beside 2^7 where its scale is up to 2^6 below another's, nothing else."""
    B, R, heads, D = q.shape
    H = k.shape[2]
    G = heads // H
    out, bound = np.zeros_like(q), np.zeros_like(q)
    for b in range(B):
        n, count = int(lens[b]), int(rows[b])
        par = parent[b] if parent is not None else np.arange(-1, R - 2)
        ways = [[0] + [j + 1 for j in way(par, r - 1)] for r in range(count)]
        pos = np.array([n + len(w) - 1 for w in ways], dtype=np.int64)
        if count == 0:
            continue
        qr, kr = turned(q[b, :count], turns, pos[:, None], halves), turned(k[b, :count], turns, pos[:, None], halves)
        qa, ka = np.abs(q[b, :count]), np.abs(k[b, :count])
        if turns is not None:                                    # |a cos - b sin| is at most |a| + |b|
            qa, ka = qa + np.abs(qr), ka + np.abs(kr)
        blocks = table[b, :(n + BLOCK - 1) // BLOCK].copy()
        held = np.ones(n, dtype=bool)
        for bb, j in left_out:
            if bb == b:
                blocks[j], held[64 * j:64 * j + 64] = 0, False
        sees = np.zeros((count, count), dtype=bool)
        for r, w in enumerate(ways):
            sees[r, w] = True
        for h in range(H):
            ck = (block_keys(cache["k_codes"][layer, blocks, h]) * cache["k_scale"][layer, blocks, h][:, None, None].astype(np.float64))
            cv = (block_values(cache["v_codes"][layer, blocks, h]) * cache["v_scale"][layer, blocks, h][:, None, None].astype(np.float64))
            kk = np.concatenate([ck.reshape(-1, D)[:n], kr[:, h]])
            vv = np.concatenate([cv.reshape(-1, D)[:n], v[b, :count, h]])
            kabs = np.concatenate([np.abs(ck.reshape(-1, D)[:n]) * 1.0, ka[:, h] * 2.0])
            own = [np.abs(v[b, t // BLOCK * BLOCK:min(count, t // BLOCK * BLOCK + BLOCK), h]).max() / 256 for t in range(count)]
            vscale = np.concatenate([np.repeat(cache["v_scale"][layer, blocks, h].astype(np.float64), BLOCK)[:n], own])
            seen = np.concatenate([np.broadcast_to(held, (count, n)), sees], 1)
            for i in range(h * G, h * G + G):
                with np.errstate(invalid="ignore", over="ignore"):
                    s = qr[:, i] @ np.nan_to_num(kk, nan=0.0, posinf=0.0, neginf=0.0).T * scale
                    s = np.where(np.isfinite(kk).all(1)[None, :], s, np.nan)
                    s = np.where(seen, s, -np.inf)
                    off = abs(scale) * (qa[:, i] @ np.nan_to_num(kabs, nan=0.0, posinf=0.0, neginf=0.0).T) * (2.0 ** -11 + (8 + D) * 2.0 ** -24)
                    delta = np.where(seen, off, 0.0).max(1)
                    w = np.exp(s - s.max(1, keepdims=True))
                    w = w / w.sum(1, keepdims=True)
                for r in range(count):
                    at = seen[r]
                    o = w[r, at] @ vv[at]
                    size = w[r, at] @ np.abs(vv[at])
                    out[b, r, i] = o
                    vmax = np.abs(vv[at]).max()
                    lost = 2.0 ** -24 * vmax * min(at.sum(), 64)
                    if by_contribution:
                        lost = 2.0 ** -32 * 512 * (w[r, at] * vscale[at]).max() * at.sum() + 2.0 ** -26 * at.sum() * size
                    bound[b, r, i] = (np.expm1(2 * delta[r]) + 2.0 ** -11 + 2.0 ** -14) * size + lost + HALF_STEP[dtype] * np.abs(o)
    return out, bound
