"""Plain implementations of the operators around drafting (numpy, from their definitions in include/fsd.h)."""
import numpy as np

BLOCK, GROUP = 64, 16
BAD_PARENT, BAD_CACHE, NO_BLOCKS, NONFINITE = 2, 32, 64, 1


def select(logits, scores, weights, done, n):
    """logits float64 [B,W,V] -> scores float64, parent, tokens [B,n], status [B], and the smallest distance of two neighbouring ranks of
    different beams (what the normalisers' errors have to stay below for the order to be theirs)"""
    B, W, V = logits.shape
    out = np.full((B, n), -np.inf), np.full((B, n), -1, np.int64), np.full((B, n), -1, np.int64), np.zeros(B, np.int64)
    nearest = np.inf
    for b in range(B):
        found, bad = [], False
        for w in range(W):
            s = 0.0 if scores is None else float(scores[b, w])
            if s == -np.inf:
                continue
            by = 1.0 if weights is None else float(weights[b, w])
            if not (s < np.inf) or not (0.0 < by < np.inf):
                bad = True
                continue
            if done is not None and done[b, w]:
                found.append((np.array([s * by]), np.array([s]), w, np.array([-1]), np.zeros(1)))
                continue
            z = logits[b, w]
            if np.isnan(z).any() or (z == np.inf).any():
                bad = True
                continue
            at = np.flatnonzero(z > -np.inf)
            if len(at) == 0:
                continue
            top = z.max()
            with np.errstate(under="ignore"):
                rest = np.log(np.sort(np.exp(z[at] - top)).sum())
            # (top + rest in one number would lose rest's last bits beside a top of 2^20, all of it beside one of 2^53)
            t = s + (z[at] - (top + rest) if abs(top) < 2.0 ** 20 else (z[at] - top) - rest)
            found.append((t * by, t, w, at, z[at]))
        if bad:
            out[3][b] = NONFINITE
            continue
        if not found:
            continue
        rank, score, tok, z = (np.concatenate([f[k] for f in found]) for k in (0, 1, 3, 4))
        beam = np.concatenate([np.full(len(f[3]), f[2]) for f in found])
        order = np.lexsort((tok, -z, beam, -rank))[:n + 1]
        with np.errstate(invalid="ignore"):
            gaps = np.abs(np.diff(rank[order]))[beam[order][1:] != beam[order][:-1]]
        if len(gaps):
            nearest = min(nearest, gaps.min())
        order = order[:n]
        k = len(order)
        out[0][b, :k], out[1][b, :k], out[2][b, :k] = score[order], beam[order], tok[order]
    return (*out, nearest)


def reorder(states, parent):
    """states [layers,B,W,...]"""
    L, B, W = states.shape[:3]
    n = parent.shape[1]
    out = np.zeros((L, B, n, *states.shape[3:]), states.dtype)
    status = np.zeros(B, np.int64)
    for b in range(B):
        for i in range(n):
            p = int(parent[b, i])
            if 0 <= p < W:
                out[:, b, i] = states[:, b, p]
            elif p != -1:
                status[b] = BAD_PARENT
    return out, status


def fork(table, lens, refs, parent, lengths, room):
    """-> table, lens, refs, free, status, [(block, block, groups of 16 tokens) copied]"""
    B, M = table.shape
    P, n = len(refs), len(parent)
    other = refs.astype(np.int64).copy()
    for e in table[(table >= 0) & (table < P)]:
        other[e] -= 1
    other = np.maximum(other, 0)
    seqs = []
    for i in range(n):
        p, status = int(parent[i]), 0
        if not -1 <= p < B:
            seqs.append((0, 0, BAD_PARENT, None))
            continue
        held = int(lens[p]) if p >= 0 else 0
        r = int(room[i]) if room is not None else 0
        have = held if lengths is None or p < 0 else int(lengths[i])
        row = table[p] if p >= 0 else np.full(M, -1)
        if not (0 <= held <= BLOCK * M and 0 <= have <= held and 0 <= r <= BLOCK * M - have):
            status = BAD_CACHE
        elif any(not 0 <= e < P for e in row[:-(-have // BLOCK)]):
            status = BAD_CACHE
        seqs.append((0, 0, status, None) if status else (have, -(-(have + r) // BLOCK), 0, row))
    named = np.zeros(P, np.int64)
    for have, need, status, row in seqs:
        for j in range(have // BLOCK):
            named[row[j]] += 1
    keeper = {}
    for i, (have, need, status, row) in enumerate(seqs):
        for j in range(have // BLOCK, need):
            e = int(row[j])
            if 0 <= e < P and other[e] == 0 and named[e] == 0 and e not in keeper:
                keeper[e] = (i, j)
    free = [e for e in range(P) if other[e] == 0 and named[e] == 0 and e not in keeper]
    out = np.full((n, M), -1, np.int64)
    copies, taken = [], 0
    for i, (have, need, status, row) in enumerate(seqs):
        full = have // BLOCK
        for j in range(need):
            if j < full or keeper.get(int(row[j])) == (i, j):
                out[i, j] = row[j]
                continue
            if taken < len(free):
                out[i, j] = free[taken]
                if j == full and have % BLOCK:
                    copies.append((int(row[j]), free[taken], -(-(have % BLOCK) // GROUP)))
            taken += 1
    left = len(free) - taken
    status = np.array([s[2] for s in seqs], np.int64)
    if left < 0:
        return np.full((n, M), -1), np.zeros(n, np.int64), refs.astype(np.int64), left, status | NO_BLOCKS, []
    counts = other.copy()
    for e in out[out >= 0]:
        counts[e] += 1
    return out, np.array([s[0] for s in seqs], np.int64), counts, left, status, copies


def move_pages(src, dst, pairs):
    """pages: dicts of k_codes [L,P,H,64,D], v_codes [L,P,H,4,D,16], k_scale, v_scale [L,P,H]; pairs (from, to, groups)"""
    for a, b, groups in pairs:
        dst["k_codes"][:, b, :, :groups * GROUP] = src["k_codes"][:, a, :, :groups * GROUP]
        dst["v_codes"][:, b, :, :groups] = src["v_codes"][:, a, :, :groups]
        for name in ("k_scale", "v_scale"):
            dst[name][:, b] = src[name][:, a]


def compact(table, refs):
    """-> table, refs, remap, used, status, [(from, to, 4)]"""
    P = len(refs)
    used = [e for e in range(P) if refs[e] > 0]
    U = len(used)
    movers, holes = [e for e in used if e >= U], [e for e in range(U) if refs[e] <= 0]
    remap = np.array([e if refs[e] > 0 else -1 for e in range(P)])
    counts = np.maximum(refs.astype(np.int64), 0)
    for a, b in zip(movers, holes):
        remap[a] = b
        counts[b], counts[a] = counts[a], 0
    out = np.full(table.shape, -1, np.int64)
    status = np.zeros(len(table), np.int64)
    for b in range(len(table)):
        for j, e in enumerate(table[b]):
            if 0 <= e < P:
                out[b, j] = remap[e]
            if e >= 0 and out[b, j] < 0:
                status[b] = BAD_CACHE
    return out, counts, remap, U, status, [(a, b, 4) for a, b in zip(movers, holes)]
