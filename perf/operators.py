"""What the speed of the operators around a verify call is measured on.

A serving step of speculative decoding runs the target model over the candidates (their attention reads the
cache), brings penalties, biases and grammar masks onto the logits, verifies, and puts the keys and values of
what was accepted into the cache.  A case is one call of one of these operators:

  condition   penalties for repeated tokens, biases and grammar masks on the rows of a verify call's logits,
              each row in its own context (the history, and the candidates on the way to that row);
  attend      attention of the candidates of a step (chain or tree, with the last emitted token as row 0) over
              a paged cache of 8-bit keys and values with one scale for each block of tokens and head, and over
              one another;
  append      the accepted rows' keys and values into that cache, with the rotation by position on the way.

Where `own` is false `run` computes these with elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 64            # tokens of a cache block
GROUP = 16            # tokens whose values lie side by side in a block
CODE_MAX = 448.0      # largest finite e4m3 value
LEAST = -100          # smallest exponent of a block's scale
DEPTH, BRANCH = 6, 4  # layers of a token tree, contexts a layer expands


def _condition(name, call, B, rows, V, dtype, **more):
    c = dict(name=name, op="condition", call=call, B=B, rows=rows, V=V, dtype=dtype, side="target", history=512,
             biases=0, mask="none")
    c.update(more)
    return c


def _append(name, call, layers, B, rows, heads, D, dtype, **more):
    c = dict(name=name, op="append", call=call, layers=layers, B=B, rows=rows, heads=heads, D=D, dtype=dtype, most=192,
             turn=D, style="halves")
    c.update(more)
    return c


def _attend(name, call, B, rows, heads, kv_heads, D, dtype, shortest, longest, **more):
    c = dict(name=name, op="attend", call=call, B=B, rows=rows, heads=heads, kv_heads=kv_heads, D=D, dtype=dtype,
             shortest=shortest, longest=longest, turn=D, style="halves")
    c.update(more)
    return c


def listed():
    return [
        # one user, no candidates: the smallest call, its latency
        _condition("condition_single", "chain", 1, 0, 32000, "bf16"),
        # the target rows of the serving batch of the benchmark
        _condition("condition_batch", "chain", 64, 8, 128256, "bf16", history=4096, biases=16),
        # the draft rows of a batch of token trees under grammars: a mask for every context
        _condition("condition_tree", "tree", 32, 60, 128256, "bf16", side="draft", history=2048, mask="contexts"),
        # binary32 logits, long candidates, rows that are not 16-byte aligned, long histories, one mask a sequence
        _condition("condition_ragged", "chain", 48, 16, 128259, "f32", history=32768, biases=100, mask="sequence"),
        # one user, one token, one layer: the smallest call, its latency
        _append("append_token", "chain", 1, 1, 1, 8, 128, "bf16"),
        # what a batch of trees left accepted, all layers of a model in one call
        _append("append_tree", "tree", 32, 64, 61, 8, 128, "bf16"),
        # prompts of a few sequences, one of them empty
        _append("append_prompt", "chain", 1, 5, 8192, 8, 128, "f16", most=100),
        # one user, one token, a short cache: latency
        _attend("attend_single", "chain", 1, 1, 32, 8, 128, "bf16", 2048, 2048),
        # the candidates of the serving batch
        _attend("attend_batch", "chain", 64, 9, 32, 8, 128, "bf16", 1024, 8192),
        # a batch of token trees
        _attend("attend_tree", "tree", 32, 61, 32, 8, 128, "bf16", 512, 4096),
        # two users with long contexts, an odd number of heads to a group
        _attend("attend_long", "chain", 2, 5, 28, 4, 128, "f16", 100000, 131072),
        # pieces of prompts behind what is cached of them, as many key heads as query heads, part of a head rotated in pairs
        _attend("attend_prompt", "chain", 3, 1000, 16, 16, 64, "bf16", 0, 7000, turn=32, style="pairs"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["condition", "append", "attend", "attend"])
    tree = rng.random() < 0.35
    call = "tree" if tree else "chain"
    if op == "condition":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        V = _log_uniform(rng, 32000, 256000)
        V = V | 1 if rng.random() < 0.3 else V // 64 * 64
        rows = rng.randint(8, 64) if tree else rng.randint(0, 16)
        side = rng.choice(["target", "draft"]) if rows else "target"
        B = max(1, min(_log_uniform(rng, 1, 128), int(4.0e8 / ((rows + 1) * V * (2 if dtype == "bf16" else 4)))))
        c = _condition(None, call, B, rows, V, dtype, side=side, history=_log_uniform(rng, 16, 16384),
                       biases=rng.choice([0, 0, rng.randint(1, 300)]), mask=rng.choice(["none", "sequence", "contexts"]))
    elif op == "append":
        D = rng.choice([64, 128, 128, 256])
        heads, layers = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 1, 4, 16])
        rows = rng.randint(8, 64) if tree else _log_uniform(rng, 1, 4096)
        B = max(1, min(_log_uniform(rng, 1, 128), int(3.0e7 / (layers * (rows + 192) * heads * D))))
        c = _append(None, call, layers, B, rows, heads, D, rng.choice(["bf16", "bf16", "f16", "f32"]),
                    most=rng.randint(0, 192), turn=rng.choice([0, D // 2, D, D]), style=rng.choice(["halves", "halves", "pairs"]))
    else:
        D = rng.choice([64, 128, 128, 128, 256])
        kv_heads, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
        rows = rng.randint(9, 65) if tree else rng.choice([1, 1, rng.randint(2, 17), _log_uniform(rng, 18, 1000)])
        longest = _log_uniform(rng, 1, 40000)
        B = max(1, min(_log_uniform(rng, 1, 128), int(2.0e8 / (longest * kv_heads * D)),
                       int(1.0e9 / ((longest + rows) * kv_heads * group * rows))))
        longest = min(longest, int(1.0e9 / (B * kv_heads * group * rows)))
        c = _attend(None, call, B, rows, kv_heads * group, kv_heads, D, rng.choice(["bf16", "bf16", "f16"]),
                    rng.choice([0, longest // 2, longest]), longest, turn=rng.choice([0, D // 2, D, D]),
                    style=rng.choice(["halves", "halves", "pairs"]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------- inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _trees(seed, B, N):
    """Parents of the N nodes of B token trees of DEPTH layers, numbered layer by layer: a layer expands its BRANCH
    best contexts into BRANCH tokens each, and the N best proposals are kept."""
    rng = random.Random(seed)
    parents = []
    for _ in range(B):
        props, frontier = [], [(-1, 0.0)]
        for layer in range(DEPTH):
            new = []
            for pid, score in frontier:
                for r in range(BRANCH):
                    s = score - 0.4 * (r + 1) * (0.5 + rng.random())
                    props.append((pid, s, layer))
                    new.append((len(props) - 1, s))
            frontier = sorted(new, key=lambda x: -x[1])[:BRANCH]
        keep = sorted(sorted(range(len(props)), key=lambda i: -props[i][1])[:N], key=lambda i: (props[i][2], i))
        number = {i: k for k, i in enumerate(keep)}
        parents.append([number.get(props[i][0], -1) for i in keep])
    return parents


def _path(rng, parent):
    """node indices from the root to some node"""
    at, path = rng.randrange(len(parent)), []
    while at >= 0:
        path.append(at)
        at = parent[at]
    return path[::-1]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _rotation(dim, rows):
    """cosines, then sines, of the angles of every position (formed in 64 bits)"""
    if dim == 0:
        return None
    freq = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    angle = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()


def _prepare_condition(c, seed):
    g, rng = _generator(seed), random.Random(seed)
    B, K, V, L = c["B"], c["rows"], c["V"], c["history"]
    s = dict(tree=c["call"] == "tree")
    rows = K + 1 if c["side"] == "target" else K
    s["logits"] = torch.randn((B, rows, V), generator=g, device="cuda").mul_(3.0).to(DTYPES[c["dtype"]])
    s["side"] = c["side"]
    # a user's tokens come back again and again: a square law over the vocabulary, another order for every seed
    ids = lambda *n: (torch.rand(n, generator=g, device="cuda").square_().mul_(V).long().mul_(7919).add_(seed) % V).int()  # noqa: E731
    s["tokens"] = ids(B, K)
    s["parent"] = _ints(_trees(seed, B, K)) if s["tree"] else None
    s["history"] = ids(B, L)
    lens = [rng.randint(L // 2, L) for _ in range(B)]
    s["history_len"], s["prompt_len"] = _ints(lens), _ints([rng.randint(0, n) for n in lens])
    s["repetition"] = torch.rand((B,), generator=g, device="cuda").add_(0.8)
    s["presence"] = torch.rand((B,), generator=g, device="cuda")
    s["frequency"] = torch.rand((B,), generator=g, device="cuda").mul_(0.5)
    s["bias_tokens"] = s["bias_values"] = s["allowed"] = None
    if c["biases"]:
        n = c["biases"]
        first = torch.randint(0, V, (B, 1), generator=g, device="cuda")
        s["bias_tokens"] = ((first + torch.arange(n, device="cuda") * (V // n)) % V).int()
        s["bias_tokens"][:, n - n // 4:] = -1                      # lists of other lengths
        s["bias_values"] = torch.randn((B, n), generator=g, device="cuda").mul_(5.0)
    if c["mask"] != "none":
        # a free text leaves nearly everything, a rule of the grammar a few hundred tokens
        n = K + 1 if c["mask"] == "contexts" else 1
        share = torch.rand((B, n, 1), generator=g, device="cuda")
        share = torch.where(share < 0.5, 0.002, 0.95)
        words = (V + 31) // 32
        bits = torch.zeros((B, n, words), dtype=torch.int64, device="cuda")
        for k in range(32):
            bits |= (torch.rand((B, n, words), generator=g, device="cuda") < share).long() << k
        s["allowed"] = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()
    s["out"] = torch.zeros_like(s["logits"])
    if own:
        import paper_2502_20704_amd as fsd

        s["conditions"] = fsd.Conditions(**{k: s[k] for k in ("history", "history_len", "prompt_len", "repetition", "presence",
                                                              "frequency", "bias_tokens", "bias_values", "allowed")})
    return s


def _codes(g, shape, spread=60.0):
    """e4m3 codes as a cache holds them: a bell whose largest values come near the end of the range"""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16).mul_(spread)
    return x.clamp_(-CODE_MAX, CODE_MAX).to(torch.float8_e4m3fn).view(torch.uint8)


def _cache(g, layers, blocks, heads, D):
    scale = lambda: torch.exp2(torch.randint(-7, -4, (layers, blocks, heads), generator=g, device="cuda").float())  # noqa: E731
    return dict(k_codes=_codes(g, (layers, blocks, heads, BLOCK, D)), v_codes=_codes(g, (layers, blocks, heads, BLOCK // GROUP, D, GROUP)),
                k_scale=scale(), v_scale=scale())


def _handles(s):
    import paper_2502_20704_amd as fsd

    s["cache"] = fsd.Cache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["table"], s["cache_len"])
    s["rotation"] = None
    if s["turns"] is not None:
        s["rotation"] = fsd.Rotation(s["turns"], fsd.ROPE_HALVES if s["style"] == "halves" else fsd.ROPE_PAIRS)


def _prepare_append(c, seed):
    g, rng = _generator(seed), random.Random(seed)
    L, B, R, H, D = c["layers"], c["B"], c["rows"], c["heads"], c["D"]
    s = dict(tree=c["call"] == "tree", style=c["style"])
    if s["tree"]:
        paths = [_path(rng, p) for p in _trees(seed, B, R - 1)]
        counts = [len(p) + 1 for p in paths]
        depth = max(DEPTH, 1)
        s["path"] = _ints([p + [-1] * (depth - len(p)) for p in paths])
    else:
        counts = [rng.randint((R + 1) // 2, R) for _ in range(B)]
        if B > 2:
            counts[1] = 0
        s["path"] = None
    s["accept_len"] = _ints([n - 1 for n in counts])
    lens = [rng.randint(0, c["most"]) for _ in range(B)]
    s["cache_len"] = _ints(lens)
    per = (c["most"] + R + BLOCK - 1) // BLOCK if not s["tree"] else (c["most"] + DEPTH + 1 + BLOCK - 1) // BLOCK
    s["per"] = per
    at = list(range(B * per))
    rng.shuffle(at)
    s["table"] = _ints([at[b * per:(b + 1) * per] for b in range(B)])
    s.update(_cache(g, L, B * per, H, D))
    values = lambda: torch.randn((L, B, R, H, D), generator=g, device="cuda", dtype=torch.float32 if c["dtype"] == "f32" else torch.float16).to(DTYPES[c["dtype"]])  # noqa: E731
    s["k"], s["v"] = values(), values()
    s["turns"] = _rotation(c["turn"], c["most"] + R + 1)
    s["len_out"], s["row_status"] = torch.zeros_like(s["cache_len"]), torch.zeros_like(s["cache_len"])
    if own:
        _handles(s)
    return s


def _prepare_attend(c, seed):
    g, rng = _generator(seed), random.Random(seed)
    B, R, Hq, H, D = c["B"], c["rows"], c["heads"], c["kv_heads"], c["D"]
    s = dict(tree=c["call"] == "tree", style=c["style"])
    s["parent"] = _ints(_trees(seed, B, R - 1)) if s["tree"] else None
    lens = [rng.randint(c["shortest"], c["longest"]) for _ in range(B)]
    lens[0] = c["longest"]
    if c["shortest"] == 0 and B > 1:
        lens[1] = 0
    s["cache_len"] = _ints(lens)
    # prompts' last pieces are shorter than the others
    s["row_count"] = _ints([R] + [rng.randint(R // 2, R) for _ in range(B - 1)]) if R > 100 else None
    per = max(1, (c["longest"] + BLOCK - 1) // BLOCK)
    need = [(n + BLOCK - 1) // BLOCK for n in lens]
    at = list(range(sum(need) + 1))
    rng.shuffle(at)
    table, used = [], 0
    for n in need:
        table.append(at[used:used + n] + [0] * (per - n))
        used += n
    s["table"] = _ints(table)
    s.update(_cache(g, 1, len(at), H, D))
    dt = DTYPES[c["dtype"]]
    mixed = torch.randn((B, R, Hq + 2 * H, D), generator=g, device="cuda").to(dt)    # one product gives all three
    s["q"], s["k"], s["v"] = mixed[:, :, :Hq], mixed[:, :, Hq:Hq + H], mixed[:, :, Hq + H:]
    s["turns"] = _rotation(c["turn"], c["longest"] + R)
    s["scale"] = D ** -0.5
    s["out"] = torch.zeros((B, R, Hq, D), dtype=dt, device="cuda")
    s["row_status"] = torch.zeros_like(s["cache_len"])
    if own:
        import paper_2502_20704_amd as fsd

        _handles(s)
        s["workspace"] = torch.empty(fsd.fsd_attend_workspace_bytes(B, R, Hq, H, D), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    s = {"condition": _prepare_condition, "append": _prepare_append, "attend": _prepare_attend}[case["op"]](case, seed)
    s["op"] = case["op"]
    return s


# ---------------------------------------------------------------------------------------------------- plain forms


def _ancestors(parent):
    """[B, N+1, N+1], 1 where the context of the second index lies on the way to that of the first (itself included);
    context 0 is the root, j+1 ends with node j.  Trees have at most 15 layers here."""
    B, N = parent.shape
    step = torch.eye(N + 1, device=parent.device).expand(B, N + 1, N + 1).clone()
    step[:, 1:].scatter_add_(2, (parent + 1).long()[:, :, None], torch.ones((B, N, 1), device=parent.device))
    return (torch.linalg.matrix_power(step, 15) > 0).float()


def _turned(x, turns, at, style):
    """x [..., rows, heads, D] in 32 bits, rotated by the angles of the positions `at` [..., rows]"""
    if turns is None:
        return x
    n = turns.shape[1] // 2
    t = turns[at.clamp(0, turns.shape[0] - 1)]
    cos, sin = t[..., None, :n], t[..., None, n:]
    if style == "halves":
        a, b = x[..., :n], x[..., n:2 * n]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * n:]], -1)
    a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., 2 * n:]], -1)


def _plain_condition(s):
    z = s["logits"].float()
    B, rows, V = z.shape
    tokens = s["tokens"].long()
    N = tokens.shape[1]
    if s["tree"]:
        on_way = _ancestors(s["parent"])[:, :, 1:]                                    # [B, context, node]
        context = torch.arange(rows, device=z.device).expand(B, rows) if s["side"] == "target" else (s["parent"] + 1).long()
    else:
        on_way = torch.ones((N + 1, N), device=z.device).tril(-1).expand(B, N + 1, N)
        context = torch.arange(rows, device=z.device).expand(B, rows)
    on_way = on_way.gather(1, context[:, :, None].expand(B, rows, N)).contiguous()
    at = torch.arange(s["history"].shape[1], device=z.device)
    held = (at < s["history_len"][:, None]).float()
    said = held * (at >= s["prompt_len"][:, None])
    history = s["history"].long()
    seen = torch.zeros((B, V), device=z.device).scatter_add_(1, history, held)
    count = torch.zeros((B, V), device=z.device).scatter_add_(1, history, said)
    more = torch.zeros((B, rows, V), device=z.device).scatter_add_(2, tokens[:, None, :].expand(B, rows, N).contiguous(), on_way)
    seen = seen[:, None] + more
    count = count[:, None] + more
    r = s["repetition"][:, None, None]
    z = torch.where(seen > 0, torch.where(z > 0, z / r, z * r), z)
    z = z - s["frequency"][:, None, None] * count - s["presence"][:, None, None] * (count > 0)
    if s["bias_tokens"] is not None:
        bias = torch.zeros((B, V + 1), device=z.device)
        where = torch.where(s["bias_tokens"] < 0, V, s["bias_tokens"]).long()
        z = z + bias.scatter_(1, where, s["bias_values"])[:, None, :V]
    if s["allowed"] is not None:
        bits = (s["allowed"][..., None] >> torch.arange(32, device=z.device, dtype=torch.int32)) & 1
        bits = bits.flatten(2)[:, :, :V].bool()
        bits = bits.expand(B, rows, V) if bits.shape[1] == 1 else bits.gather(1, context[:, :, None].expand(B, rows, V))
        z = z.masked_fill(~bits, -math.inf)
    s["out"].copy_(z.to(s["logits"].dtype))
    return s["out"]


def _exponent(most):
    """the smallest e with most <= 448 * 2^e, but not under LEAST"""
    m, e = torch.frexp(most / CODE_MAX)
    return torch.where(most > 0, torch.where(m == 0.5, e - 1, e), LEAST).clamp(min=LEAST)


def _plain_append(s):
    k, v = s["k"].float(), s["v"].float()
    L, B, R, H, D = k.shape
    dev = k.device
    count = s["accept_len"].long() + 1
    per = s["per"]
    # token t of the table's blocks holds row t - cache_len of the accepted ones
    t = torch.arange(per * BLOCK, device=dev)
    row = t - s["cache_len"][:, None].long()
    new = (row >= 0) & (row < count[:, None])
    row = row.clamp(0, max(R - 1, 0))
    if s["path"] is not None:
        path = torch.cat([torch.zeros((B, 1), dtype=torch.long, device=dev), s["path"].long() + 1], 1)
        row = path.gather(1, row.clamp(max=path.shape[1] - 1)).clamp(min=0)
    pick = row[None, :, :, None, None].expand(L, B, per * BLOCK, H, D)
    k = _turned(k.gather(2, pick), s["turns"], t.expand(B, -1), s["style"])
    v = v.gather(2, pick)
    touched = new.view(B, per, BLOCK).any(2)
    begun = (t[::BLOCK] < s["cache_len"][:, None]) & touched                           # holds tokens already
    table = s["table"].long()

    def put(x, codes, scale, by_token):
        x = x.view(L, B, per, BLOCK, H, D).transpose(3, 4)                            # [L, B, per, H, BLOCK, D]
        is_new = new.view(B, per, 1, BLOCK, 1)
        e = _exponent(torch.where(is_new, x.abs(), torch.zeros((), device=dev)).amax((4, 5)))
        old_scale = scale[:, table]                                                   # [L, B, per, H]
        one = torch.exp2(e.float())
        one = torch.where(begun[:, :, None], torch.maximum(one, old_scale), one)
        held = codes[:, table].view(torch.float8_e4m3fn).float()
        if not by_token:
            held = held.permute(0, 1, 2, 3, 4, 6, 5).reshape(L, B, per, H, BLOCK, D)
        value = torch.where(is_new, x / one[..., None, None], held * (old_scale / one)[..., None, None])
        keep = ~(is_new | (begun[:, :, None, None, None] & (t.view(per, 1, BLOCK, 1) < s["cache_len"].view(B, 1, 1, 1, 1))))
        value = torch.where(keep, held, value).to(torch.float8_e4m3fn).view(torch.uint8)
        if not by_token:
            value = value.view(L, B, per, H, BLOCK // GROUP, GROUP, D).transpose(5, 6)
        codes[:, table[touched]] = value[:, touched]
        scale[:, table[touched]] = one[:, touched]

    put(k, s["k_codes"], s["k_scale"], True)
    put(v, s["v_codes"], s["v_scale"], False)
    s["len_out"].copy_(s["cache_len"] + count)
    return _append_outputs(s)


def _append_outputs(s):
    return [s["k_codes"].view(torch.float8_e4m3fn), s["v_codes"].view(torch.float8_e4m3fn), s["k_scale"], s["v_scale"],
            s["len_out"], s["row_status"]]


def _plain_attend(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    B, R, Hq, D = q.shape
    H = k.shape[2]
    dev = q.device
    if s["tree"]:
        sees = _ancestors(s["parent"])
    else:
        sees = torch.ones((R, R), device=dev).tril().expand(B, R, R)
    at = s["cache_len"][:, None].long() + sees.sum(2).long() - 1
    q, k = _turned(q, s["turns"], at, s["style"]), _turned(k, s["turns"], at, s["style"])
    table = s["table"].long()
    per = table.shape[1]
    kc = s["k_codes"][0, table].view(torch.float8_e4m3fn).float() * s["k_scale"][0, table][..., None, None]
    vc = s["v_codes"][0, table].view(torch.float8_e4m3fn).float() * s["v_scale"][0, table][..., None, None, None]
    kc = kc.transpose(1, 2).reshape(B, H, per * BLOCK, D)
    vc = vc.permute(0, 2, 1, 3, 5, 4).reshape(B, H, per * BLOCK, D)
    held = torch.arange(per * BLOCK, device=dev) < s["cache_len"][:, None]
    rows = q.view(B, R, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, H, R * (Hq // H), D)
    kc = torch.cat([kc, k.transpose(1, 2)], 2).transpose(2, 3).contiguous()
    vc = torch.cat([vc.masked_fill(~held[:, None, :, None], 0.0), v.transpose(1, 2)], 2)
    score = (rows @ kc).view(B, H, R, Hq // H, -1) * s["scale"]
    seen = torch.cat([held[:, None, :].expand(B, R, per * BLOCK), sees > 0], 2)
    score = score.masked_fill(~seen[:, None, :, None, :], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = (p.view(B, H, R * (Hq // H), -1) @ vc).view(B, H, R, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, R, Hq, D)
    o = o.to(s["out"].dtype)
    if s["row_count"] is not None:
        o = torch.where((torch.arange(R, device=dev) < s["row_count"][:, None])[:, :, None, None], o, s["out"])
    s["out"].copy_(o)
    return [s["out"], s["row_status"]]


def _own(s):
    import paper_2502_20704_amd as fsd

    if s["op"] == "condition":
        out = dict(out=s["out"])
        if s["tree"]:
            fsd.fsd_condition_tree(s["logits"], s["tokens"], s["parent"], s["conditions"], out=out)
        else:
            fsd.fsd_condition_chain(s["logits"], s["tokens"], s["conditions"], out=out)
        return s["out"]
    if s["op"] == "append":
        fsd.fsd_cache_append(s["k"], s["v"], s["cache"], s["accept_len"], path_nodes=s["path"], rotation=s["rotation"],
                             out=dict(cache_len=s["len_out"], row_status=s["row_status"]))
        return _append_outputs(s)
    more = dict(rotation=s["rotation"], scale=s["scale"], out=dict(out=s["out"], row_status=s["row_status"]), workspace=s["workspace"])
    if s["tree"]:
        fsd.fsd_attend_tree(s["q"], s["k"], s["v"], s["parent"], s["cache"], **more)
    else:
        fsd.fsd_attend_chain(s["q"], s["k"], s["v"], s["cache"], row_count=s["row_count"], **more)
    return [s["out"], s["row_status"]]


def run(state):
    if own:
        return _own(state)
    return {"condition": _plain_condition, "append": _plain_append, "attend": _plain_attend}[state["op"]](state)


# ---------------------------------------------------------------------------------------------------- work


def work(case):
    c = case
    if c["op"] == "condition":
        B, K, V = c["B"], c["rows"], c["V"]
        rows = K + 1 if c["side"] == "target" else K
        masks = {"none": 0, "sequence": 1, "contexts": K + 1}[c["mask"]]
        per = 4 if c["dtype"] == "f32" else 2
        return dict(bytes=B * (2 * rows * V * per + 3 * c["history"] + 8 * c["biases"] + masks * ((V + 31) // 32) * 4),
                    flops=B * rows * V)
    width = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "append":
        rows = 4 if c["call"] == "tree" else 0.75 * c["rows"] * (1 if c["B"] < 3 else (c["B"] - 1) / c["B"])
        rows = max(1.0, rows)
        values = c["layers"] * c["B"] * rows * c["heads"] * c["D"] * 2
        return dict(bytes=int(values * (width + 1)), flops=int(values * 3))
    tokens = c["longest"] + (c["B"] - 1) * (c["shortest"] + c["longest"]) / 2
    R, B, D = c["rows"], c["B"], c["D"]
    rows = R if R <= 100 else (R + (B - 1) * 0.75 * R) / B
    fresh = DEPTH / 2 if c["call"] == "tree" else (rows + 1) / 2
    return dict(bytes=int(2 * tokens * c["kv_heads"] * (D + 4 / BLOCK) + B * rows * D * width * 2 * (c["heads"] + c["kv_heads"])),
                flops=int(4 * D * c["heads"] * rows * (tokens + B * fresh)))


# ---------------------------------------------------------------------------------------------------- in 64 bits


def _walk(parent, j):
    way = []
    while j >= 0:
        way.append(j)
        j = parent[j]
    return way[::-1]


def _exact_condition(case, seed):
    s = _prepare_condition(case, seed)
    B, rows, V = s["logits"].shape
    N = s["tokens"].shape[1]
    out = torch.empty((B, rows, V), dtype=torch.float64, device="cuda")
    host = {k: s[k].tolist() for k in ("history_len", "prompt_len", "repetition", "presence", "frequency")}
    for b in range(B):
        parent = s["parent"][b].tolist() if s["tree"] else list(range(-1, N - 1))
        n, p = host["history_len"][b], host["prompt_len"][b]
        prompt = torch.bincount(s["history"][b, :min(p, n)].long(), minlength=V)
        said = torch.bincount(s["history"][b, min(p, n):n].long(), minlength=V)
        bias = torch.zeros(V, dtype=torch.float64, device="cuda")
        if s["bias_tokens"] is not None:
            good = s["bias_tokens"][b] >= 0
            bias[s["bias_tokens"][b][good].long()] = s["bias_values"][b][good].double()
        for r in range(rows):
            last = r - 1 if s["side"] == "target" or not s["tree"] else parent[r]
            way = _walk(parent, last)
            count = said + torch.bincount(s["tokens"][b].long()[torch.tensor(way, dtype=torch.long, device="cuda")], minlength=V)
            z = s["logits"][b, r].double()
            hit = (count + prompt) > 0
            z = torch.where(hit & (z > 0), z / host["repetition"][b], torch.where(hit, z * host["repetition"][b], z))
            z = z - host["frequency"][b] * count.double() - host["presence"][b] * (count > 0).double() + bias
            if s["allowed"] is not None:
                w = s["allowed"][b, last + 1 if s["allowed"].shape[1] > 1 else 0].long()
                j = torch.arange(V, device="cuda")
                z = torch.where((w[j // 32] >> (j % 32)) % 2 == 0, -math.inf, z)
            out[b, r] = z
    return out


def _turn64(x, turns, positions, style):
    """x [n, H, D] in 64 bits"""
    if turns is None:
        return x
    n = turns.shape[1] // 2
    t = turns[positions].double()
    c, sn = t[:, None, :n], t[:, None, n:]
    y = x.clone()
    lo, hi = (slice(0, n), slice(n, 2 * n)) if style == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y[..., lo] = x[..., lo] * c - x[..., hi] * sn
    y[..., hi] = x[..., hi] * c + x[..., lo] * sn
    return y


def _to_code64(y):
    """nearest e4m3 value, ties to even; |y| <= 448"""
    a = y.abs()
    unit = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(y) * torch.round(a / unit) * unit


def _exact_append(case, seed):
    s = _prepare_append(case, seed)
    L, B, R, H, D = s["k"].shape
    if L * B * H > 20000:
        return None
    kc = s["k_codes"].view(torch.float8_e4m3fn).double()
    vc = s["v_codes"].view(torch.float8_e4m3fn).double()
    ks, vs = s["k_scale"].double(), s["v_scale"].double()
    lens, counts, table = s["cache_len"].tolist(), [n + 1 for n in s["accept_len"].tolist()], s["table"].tolist()
    for b in range(B):
        rows = list(range(counts[b])) if s["path"] is None else ([0] + [j + 1 for j in s["path"][b].tolist()])[:counts[b]]
        t = 0
        while t < counts[b]:
            at = lens[b] + t
            fill, n = at % BLOCK, min(BLOCK - at % BLOCK, counts[b] - t)
            block = table[b][at // BLOCK]
            pick = torch.tensor(rows[t:t + n], device="cuda")
            for layer in range(L):
                where = torch.arange(at, at + n, device="cuda")
                xk = _turn64(s["k"][layer, b, pick].double(), s["turns"], where, s["style"]).transpose(0, 1)
                xv = s["v"][layer, b, pick].double().transpose(0, 1)
                old_v = vc[layer, block].transpose(2, 3).reshape(H, BLOCK, D).clone()
                for x, codes, scales in ((xk, kc[layer, block], ks), (xv, old_v, vs)):
                    most = x.abs().amax((1, 2))
                    e = torch.ceil(torch.log2(most.clamp(min=2.0 ** -200) / CODE_MAX)).clamp(min=LEAST)
                    e = e + (most > CODE_MAX * torch.exp2(e)).double()                # (log2's own rounding at a border)
                    e = torch.where((most <= CODE_MAX * torch.exp2(e - 1)) & (e > LEAST), e - 1, e)
                    one = torch.exp2(e)
                    if fill:
                        one = torch.maximum(one, scales[layer, block])
                        codes[:, :fill] = _to_code64(codes[:, :fill] * (scales[layer, block] / one)[:, None, None])
                    codes[:, fill:fill + n] = _to_code64(x / one[:, None, None])
                    scales[layer, block] = one
                vc[layer, block] = old_v.view(H, BLOCK // GROUP, GROUP, D).transpose(2, 3)
            t += n
    return [kc, vc, ks, vs, None, None]


def _exact_attend(case, seed):
    s = _prepare_attend(case, seed)
    B, R, Hq, D = s["q"].shape
    H = s["k"].shape[2]
    out = s["out"].double()
    counts = s["row_count"].tolist() if s["row_count"] is not None else [R] * B
    for b in range(B):
        n, R1 = int(s["cache_len"][b]), counts[b]
        parent = s["parent"][b].tolist() if s["tree"] else list(range(-1, R - 2))
        ways = [[0] + [j + 1 for j in _walk(parent, r - 1)] for r in range(R1)] if s["tree"] else None
        depth = torch.tensor([len(w) - 1 for w in ways] if s["tree"] else list(range(R1)), device="cuda")
        where = n + depth
        q = _turn64(s["q"][b, :R1].double(), s["turns"], where, s["style"])
        k = _turn64(s["k"][b, :R1].double(), s["turns"], where, s["style"])
        v = s["v"][b, :R1].double()
        if s["tree"]:
            sees = torch.zeros((R1, R1), dtype=torch.bool)
            for r, w in enumerate(ways):
                sees[r, w] = True
            sees = sees.cuda()
        else:
            sees = torch.arange(R1, device="cuda")[None, :] <= torch.arange(R1, device="cuda")[:, None]
        blocks = s["table"][b, :(n + BLOCK - 1) // BLOCK].long()
        for h in range(H):
            kh = s["k_codes"][0, blocks, h].view(torch.float8_e4m3fn).double() * s["k_scale"][0, blocks, h].double()[:, None, None]
            vh = s["v_codes"][0, blocks, h].view(torch.float8_e4m3fn).double().transpose(2, 3) * s["v_scale"][0, blocks, h].double()[:, None, None, None]
            kh = torch.cat([kh.reshape(-1, D)[:n], k[:, h]])
            vh = torch.cat([vh.reshape(-1, D)[:n], v[:, h]])
            seen = torch.cat([torch.ones((R1, n), dtype=torch.bool, device="cuda"), sees], 1)
            for i in range(h * (Hq // H), (h + 1) * (Hq // H)):
                score = (q[:, i] @ kh.t()) * s["scale"]
                out[b, :R1, i] = torch.softmax(score.masked_fill(~seen, -math.inf), 1) @ vh
    return [out, None]


def exact(case, seed):
    return {"condition": _exact_condition, "append": _exact_append, "attend": _exact_attend}[case["op"]](case, seed)
