"""The calls around a language model service's attention as a user's program makes them, for timing and checking.

Five operators: norm and rotation of query and key heads, the fork of requests that share a paged cache's blocks, its compaction, the
copy of blocks in the caches of all layers, and what rows of logits say about tokens (log probabilities, entropy, alternatives).  Where `own`
is false they are computed in their plain form, with elementary torch operations in 32 bits, angles in 64.

Lengths, parents and the like of a case come from its own `lengths` number, data and the places of blocks from the seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one user's next token at a far position: all latency
        dict(name="rotate_one", op="rotate", tokens=1, prompts=0, farthest=131071, q_heads=32, kv_heads=8, dim=128, rotary=128, neighbours=False, norm=True,
             dtype="bf16", lengths=1),
        # a decode step of a busy service, heads of 64 of which half is rotated, neighbours as pairs
        dict(name="rotate_step", op="rotate", tokens=256, prompts=0, farthest=16384, q_heads=16, kv_heads=16, dim=64, rotary=32, neighbours=True, norm=True,
             dtype="f16", lengths=2),
        # packed prompts of very different lengths
        dict(name="rotate_prompts", op="rotate", tokens=23171, prompts=24, farthest=0, q_heads=32, kv_heads=8, dim=128, rotary=128, neighbours=False, norm=True,
             dtype="bf16", lengths=3),
        # a beam search's step: 32 prompts with 4 beams each
        dict(name="fork_beams", op="fork", groups=32, beams=4, children=4, ended=0.1, prompt_most=2048, own_most=256, block=64, spare=0.25, lengths=4),
        # very many requests over a large cache of small blocks; some have ended, the others are sampled twice
        dict(name="fork_many", op="fork", groups=4096, beams=1, children=2, ended=0.3, prompt_most=4096, own_most=512, block=32, spare=0.1, lengths=5),
        # a small service's cache after some hours
        dict(name="compact_small", op="compact", groups=32, beams=4, prompt_most=2048, own_most=256, block=64, spare=1.0, lengths=6),
        # a large cache of small blocks, nearly full
        dict(name="compact_large", op="compact", groups=3001, beams=1, prompt_most=4096, own_most=512, block=16, spare=0.25, lengths=7),
        # the last blocks of the beams that a step has forked, in all layers
        dict(name="copy_beams", op="copy", layers=4, copies=61, rest=67, block=64, kv_heads=8, dim=128, lengths=8),
        # what a compaction moves, in a model's first layers
        dict(name="copy_moved", op="copy", layers=3, copies=5000, rest=300, block=16, kv_heads=8, dim=128, lengths=9),
        # one user's next token: a single row
        dict(name="scores_one", op="scores", rows=1, vocabulary=131072, top=20, masked=0.0, scale=1.0, dtype="bf16", lengths=10),
        # a step's rows in 32 bits, an odd vocabulary of which a grammar leaves little, at a temperature
        dict(name="scores_step", op="scores", rows=256, vocabulary=50001, top=5, masked=0.9, scale=1.25, dtype="f32", lengths=11),
        # a batch of prompts is scored
        dict(name="scores_prompts", op="scores", rows=2999, vocabulary=100003, top=20, masked=0.0, scale=1.0, dtype="bf16", lengths=12),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rotate", "fork", "compact", "copy", "scores"])
    case = {"op": op, "lengths": rng.randrange(1 << 30)}
    if op == "rotate":
        dim = rng.choice([64, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 5, 8])
        q_heads = kv_heads * rng.choice([1, 3, 4, 6, 8])
        tokens = _log(rng, 1, min(24000, 118_000_000 // ((q_heads + kv_heads) * dim)))
        return dict(case, tokens=tokens, prompts=rng.choice([0, 0, 1, _log(rng, 1, min(64, tokens))]), farthest=_log(rng, 1, 1 << 20), q_heads=q_heads, kv_heads=kv_heads,
                    dim=dim, rotary=rng.choice([16, dim // 2, dim - 16, dim]), neighbours=rng.random() < 0.5, norm=rng.random() < 0.7,
                    dtype=rng.choice(["bf16", "f16"]))
    if op in ("fork", "compact"):
        beams = rng.choice([1, 1, 2, 3, 4, 8])
        groups = _log(rng, 1, 4096 // beams)
        case.update(groups=groups, beams=beams, prompt_most=_log(rng, 1, min(65536, (1 << 24) // groups)), own_most=_log(rng, 1, min(2048, (1 << 21) // (groups * beams))),
                    block=rng.choice([32, 64, 128, 256]), spare=rng.choice([0.1, 0.5, 1.0]))
        return dict(case, children=rng.choice([1, beams, 2]), ended=rng.choice([0.0, 0.1, 0.5])) if op == "fork" else case
    if op == "copy":
        layers, block, kv_heads, dim = rng.choice([1, 2, 5, 16]), rng.choice([16, 32, 64, 128, 256]), rng.choice([1, 2, 5, 8]), rng.choice([64, 128])
        return dict(case, layers=layers, copies=_log(rng, 1, min(5000, 240_000_000 // (layers * block * kv_heads * dim))), rest=_log(rng, 1, 300), block=block,
                    kv_heads=kv_heads, dim=dim)
    rows = _log(rng, 1, 4096)
    return dict(case, rows=rows, vocabulary=_log(rng, 1, min(200_000, 299_000_000 // rows)), top=rng.choice([0, 1, 5, 20, 32]), masked=rng.choice([0.0, 0.0, 0.5, 0.999]),
                scale=rng.choice([1.0, 0.7, 2.0]), dtype=rng.choice(["bf16", "f16", "f32"]))


# ---- what a case's own number gives, on the host ------------------------------------------------------------------

def _positions(case):
    rng = np.random.default_rng(case["lengths"])
    n = case["tokens"]
    if case["prompts"] == 0:                                                # a token each for as many requests
        return np.exp(rng.uniform(0, math.log(case["farthest"] + 1), n)).astype(np.int64) if n > 1 else np.array([case["farthest"]])
    cuts = np.sort(rng.integers(0, n + 1, case["prompts"] - 1))             # (a prompt may be empty)
    starts = np.concatenate([[0], cuts])
    return np.arange(n) - np.repeat(starts, np.diff(np.concatenate([starts, [n]])))


def _requests(case):
    """(lengths of requests, whole blocks that a request shares with the others of its group, parents of the children)."""
    rng = np.random.default_rng(case["lengths"])
    groups, beams, b = case["groups"], case["beams"], case["block"]
    prompt = np.exp(rng.uniform(0, math.log(case["prompt_most"]), groups)).round().astype(np.int64)
    lengths = np.repeat(prompt + rng.integers(0, case["own_most"] + 1, groups), beams)      # a group's beams are equally long
    shared = np.repeat(prompt // b if beams > 1 else prompt * 0, beams)
    if case["op"] == "compact":
        return lengths, shared, None
    children = case["children"]
    parents = np.arange(groups)[:, None] * beams + rng.integers(0, beams, (groups, children))
    parents[rng.random(groups) < case["ended"]] = -1
    return lengths, shared, parents.reshape(-1)


def _blocks(case, lengths, shared):
    """The table's entries as numbers from 0 on, -1 behind the requests, and how many blocks there are in use."""
    b, beams = case["block"], case["beams"]
    pages = -(-lengths // b)
    width = int(pages.max()) + 1
    page = np.arange(width)
    first = np.arange(lengths.size) // beams * beams
    of = np.where(page[None, :] < shared[:, None], first[:, None], np.arange(lengths.size)[:, None]) * width + page        # whose page it is
    there = page[None, :] < pages[:, None]
    used = np.zeros(lengths.size * width, dtype=bool)
    used[of[there]] = True
    number = np.cumsum(used) - 1
    return np.where(there, number[of], -1), int(used.sum())


def _cache_sizes(case):
    n_blocks = 2 * case["copies"] + case["rest"]
    return (n_blocks, case["kv_heads"], case["block"], case["dim"])


def work(case):
    op = case["op"]
    if op == "rotate":
        values = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 4 * values + 4 * case["tokens"] + 2 * case["rotary"] + 4 * case["dim"] * case["norm"], "flops": 6 * values}
    if op in ("fork", "compact"):
        lengths, shared, parents = _requests(case)
        table, used = _blocks(case, lengths, shared)
        pages, free = int((-(-lengths // case["block"])).sum()), int(used * case["spare"]) + 5
        if op == "compact":
            return {"bytes": 4 * (lengths.size + pages + table.size + 2 * free) + 8 * min(free, (used + free) // 2) + 8, "flops": 0}
        return {"bytes": 4 * (lengths.size + pages + 2 * parents.size + parents.size * table.shape[1] + free + used + free) + 8 * parents.size + 12, "flops": 0}
    if op == "copy":
        _, hkv, b, d = _cache_sizes(case)
        return {"bytes": case["layers"] * case["copies"] * 2 * 2 * (hkv * b * d + hkv) + 8 * case["copies"], "flops": 0}
    size = {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    return {"bytes": case["rows"] * (case["vocabulary"] * size + 4 + 12 + 8 * case["top"]), "flops": 8 * case["rows"] * case["vocabulary"]}


def _int32(v):
    return torch.from_numpy(np.ascontiguousarray(v).astype(np.int32)).to(DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    state = {"op": op, "status": torch.zeros(1, dtype=torch.int32, device=DEV)}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)
    if op == "rotate":
        dtype, hq, hkv, d, rotary = DTYPES[case["dtype"]], case["q_heads"], case["kv_heads"], case["dim"], case["rotary"]
        # queries and keys lie in one product's output, in front of its values; some tokens and channels are much larger
        qkv = normal(case["tokens"], hq + 2 * hkv, d)
        qkv *= torch.exp(normal(case["tokens"], 1, 1)) * torch.exp(normal(1, hq + 2 * hkv, d))
        qkv = qkv.to(dtype)
        state.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], positions=_int32(_positions(case)), neighbours=case["neighbours"], epsilon=1e-6,
                     frequencies=(10000.0 ** (-torch.arange(0, rotary, 2, device=DEV, dtype=torch.float64) / rotary)).float())
        state.update({name: (1 + 0.2 * normal(d)).to(dtype) if case["norm"] else None for name in ("q_weight", "k_weight")})
        return state
    if op in ("fork", "compact"):
        lengths, shared, parents = _requests(case)
        table, used = _blocks(case, lengths, shared)
        n_free = int(used * case["spare"]) + 5
        n_blocks = used + n_free + 3                                         # three that the service keeps for itself
        order = torch.randperm(n_blocks, generator=gen, device=DEV).to(torch.int32)
        table = _int32(table)
        table = torch.where(table >= 0, order[table.clamp(min=0).long()], -1)
        state.update(table=table, requests=_int32(lengths), block=case["block"], n_blocks=n_blocks, free=order[used:used + n_free].contiguous())
        if op == "fork":
            state["parents"] = _int32(parents)
        return state
    if op == "copy":
        shape = _cache_sizes(case)
        order = torch.randperm(shape[0], generator=gen, device=DEV).to(torch.int32)
        n = case["copies"]
        copies = torch.full((n + 7, 2), -1, dtype=torch.int32, device=DEV)   # the list has room for more
        copies[:n, 0], copies[:n, 1] = order[:n], order[n:2 * n]
        caches = []
        for _ in range(case["layers"]):
            codes = [torch.randint(0, 0x78, shape, generator=gen, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn) for _ in range(2)]
            caches.append((*codes, *(torch.randint(110, 130, shape[:2], generator=gen, device=DEV, dtype=torch.uint8) for _ in range(2))))
        state.update(caches=caches, copies=copies)
        return state
    rows, n = case["rows"], case["vocabulary"]
    logits = normal(rows, n).mul_(2.5)
    if case["masked"] > 0:
        logits.masked_fill_(torch.rand((rows, n), generator=gen, device=DEV) < case["masked"], -math.inf)
        if rows > 4:
            logits[rows // 2] = -math.inf                                    # a row that the grammar leaves nothing
    tokens = torch.randint(0, n, (rows,), generator=gen, device=DEV, dtype=torch.int32)
    tokens[3::16] = -1                                                       # the last tokens of prompts have none behind them
    state.update(logits=logits.to(DTYPES[case["dtype"]]), tokens=tokens, scale=case["scale"], top=case["top"])
    return state


# ---- plain forms ------------------------------------------------------------------------------------------------

def _rotate_plain_one(x, weight, epsilon, cos, sin, neighbours):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + epsilon) * weight.float()
    half = cos.shape[-1]
    turned, rest = y[..., :2 * half], y[..., 2 * half:]
    if neighbours:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turned[..., :half], turned[..., half:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, rest], -1).to(x.dtype)


def _rotate_plain(s):
    angles = s["positions"].double()[:, None, None] * s["frequencies"].double()
    cos, sin = torch.cos(angles).float(), torch.sin(angles).float()
    return {"q": _rotate_plain_one(s["q"], s["q_weight"], s["epsilon"], cos, sin, s["neighbours"]),
            "k": _rotate_plain_one(s["k"], s["k_weight"], s["epsilon"], cos, sin, s["neighbours"])}


def _marked(n_blocks, blocks, there):
    """Which blocks the entries name that are there."""
    marks = torch.zeros(n_blocks + 1, dtype=torch.bool, device=DEV)
    marks[torch.where(there, blocks, n_blocks).reshape(-1).long()] = True
    return marks[:n_blocks]


def _listed(marks, room):
    """The marked blocks ascending, -1 behind them."""
    out = torch.full((room + 1,), -1, dtype=torch.long, device=DEV)
    out.scatter_(0, torch.where(marks, torch.cumsum(marks, 0) - 1, room).clamp(max=room), torch.arange(marks.numel(), device=DEV))
    return torch.cat([out[:room], out.new_full((1,), -1)])


def _fork_plain(s):
    table, lengths, b, n_blocks, free = s["table"].long(), s["requests"].long(), s["block"], s["n_blocks"], s["free"].long()
    alive, parent = s["parents"] >= 0, s["parents"].clamp(min=0).long()
    (n, width), children = table.shape, parent.numel()
    page, order = torch.arange(width, device=DEV), torch.arange(children, device=DEV)
    length = torch.where(alive, lengths[parent], 0)
    pages = (length + b - 1) // b
    there = page[None, :] < pages[:, None]
    rows = torch.where(there, table[parent], -1)
    first = torch.full((n,), children, device=DEV).scatter_reduce_(0, parent, torch.where(alive, order, children), "amin")
    need = alive & (length % b > 0) & (order > first[parent])
    taken = need.sum()
    given = _marked(n_blocks, table, page[None, :] < ((lengths + b - 1) // b)[:, None]) & ~_marked(n_blocks, rows, there)
    pool = torch.cat([free, _listed(given, n_blocks)])
    total = free.numel() + given.sum()
    mine = torch.where(need, torch.cumsum(need, 0) - 1, children)
    source = rows[order, (pages - 1).clamp(min=0)]
    target = pool[mine.clamp(max=pool.numel() - 1)]
    copies = torch.full((children + 1, 2), -1, dtype=torch.long, device=DEV)
    copies.scatter_(0, mine[:, None].expand(-1, 2), torch.stack([source, target], 1))
    rows = torch.where((page[None, :] == pages[:, None] - 1) & need[:, None], target[:, None], rows)
    at = torch.arange(n_blocks, device=DEV) + taken
    left = torch.where(at < total, pool[at.clamp(max=pool.numel() - 1)], -1)
    return {"table": rows.int(), "lengths": length.int(), "copies": copies[:children].int(), "free": left.int(),
            "counts": torch.stack([taken, given.sum(), total - taken]).int()}


def _compact_plain(s):
    table, b, n_blocks, free = s["table"].long(), s["block"], s["n_blocks"], s["free"].long()
    there = torch.arange(table.shape[1], device=DEV)[None, :] < ((s["requests"].long() + b - 1) // b)[:, None]
    used = _marked(n_blocks, table, there)
    spare = _marked(n_blocks, free, torch.ones_like(free, dtype=torch.bool))
    n_used = used.sum()
    behind = torch.cumsum(used | spare, 0) > n_used
    moved, holes = used & behind, spare & ~behind
    room = min(free.numel(), n_blocks // 2)
    copies = torch.stack([_listed(moved, room)[:room], _listed(holes, room)[:room]], 1)
    goes = torch.arange(n_blocks + 1, device=DEV)
    goes[torch.where(copies[:, 0] >= 0, copies[:, 0], n_blocks)] = copies[:, 1]
    left = _listed((used | spare) & behind, free.numel())[:free.numel()]
    return {"table": torch.where(there, goes[table.clamp(min=0)], -1).int(), "copies": copies.int(), "free": left.int(),
            "counts": torch.stack([moved.sum(), n_used]).int()}


def _copy_plain(s):
    copies = s["copies"].long()
    copies = torch.where(copies >= 0, copies, copies[:1])                    # an unused entry repeats the first one
    for cache in s["caches"]:
        for t in cache:
            raw = t.view(torch.uint8)
            raw[copies[:, 1]] = raw[copies[:, 0]]
    return s["caches"]


def _scores_plain(s):
    logits, tokens, top = s["logits"], s["tokens"].long(), s["top"]
    rows, n = logits.shape
    z = logits.float() * s["scale"]
    most = z.amax(1, keepdim=True)
    d = z - torch.where(torch.isfinite(most), most, 0.0)
    e = torch.exp(d)
    total = e.sum(1)
    some = total > 0
    lse = torch.where(some, most[:, 0] + torch.log(total), -math.inf)
    entropy = torch.where(some, torch.log(total) - (e * torch.where(e > 0, d, 0.0)).sum(1) / torch.where(some, total, 1.0), 0.0)
    del d, e

    def logprob(x):
        return torch.where(torch.isfinite(x), x - torch.where(some, lse, 0.0)[:, None], -math.inf)
    given = logprob(z.gather(1, tokens.clamp(min=0)[:, None]))[:, 0]
    # values ascending as integers, a lower token before an equal one
    bits = (logits.float() + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() * (1 << 32) + (n - 1 - torch.arange(n, device=DEV))
    k = min(top, n)
    first = n - 1 - (torch.topk(key, k, 1).values & 0xffffffff) if k else tokens.new_zeros((rows, 0))
    values = logprob(z.gather(1, first))
    rest = top - k
    return {"logprob": torch.where(tokens >= 0, given, 0.0), "entropy": entropy, "lse": lse,
            "top_tokens": torch.nn.functional.pad(torch.where(values > -math.inf, first, -1), (0, rest), value=-1).int(),
            "top_logprob": torch.nn.functional.pad(values, (0, rest), value=-math.inf)}


def run(state):
    s = state
    if own:
        from paper_2311_10359_amd import binding
        if s["op"] == "rotate":
            got = binding.fikit_rotate_heads(s["q"], s["k"], s["positions"], s["frequencies"], s["status"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                                             epsilon=s["epsilon"], neighbours=s["neighbours"])
            return {"q": got.q, "k": got.k}
        if s["op"] == "fork":
            got = binding.fikit_cache_fork(s["table"], s["requests"], s["parents"], s["block"], s["n_blocks"], s["free"], s["status"])
            return {"table": got.block_table, "lengths": got.lengths, "copies": got.copies, "free": got.free_blocks, "counts": got.counts}
        if s["op"] == "compact":
            got = binding.fikit_cache_compact(s["table"], s["requests"], s["block"], s["n_blocks"], s["free"], s["status"])
            return {"table": got.block_table, "copies": got.copies, "free": got.free_blocks, "counts": got.counts}
        if s["op"] == "copy":
            binding.fikit_cache_copy(s["caches"], s["copies"], s["status"])
            return s["caches"]
        got = binding.fikit_token_scores(s["logits"], s["tokens"], s["status"], scale=s["scale"], n_top=s["top"])
        return {"logprob": got.logprob, "entropy": got.entropy, "lse": got.lse, "top_tokens": got.top_tokens, "top_logprob": got.top_logprob}
    return {"rotate": _rotate_plain, "fork": _fork_plain, "compact": _compact_plain, "copy": _copy_plain, "scores": _scores_plain}[s["op"]](s)


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------

def _exact_rotate(x, weight, epsilon, positions, frequencies, neighbours):
    """As products of complex numbers, a head at a time."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    half = frequencies.numel()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), positions.double()[:, None] * frequencies.double()[None, :])
    for h in range(x.shape[1]):
        y = x[:, h].double()
        if weight is not None:
            y = y / torch.sqrt(y.square().sum(1, keepdim=True) / y.shape[1] + epsilon) * weight.double()
        out[:, h] = y
        i = torch.arange(half, device=x.device)
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
        z = torch.complex(y[:, a], y[:, b]) * turn
        out[:, h, a], out[:, h, b] = z.real, z.imag
    return out


def exact(case, seed):
    if case["op"] not in ("rotate", "scores"):
        return None                                                          # whole numbers and copies only
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return {name: _exact_rotate(s[name], s[name + "_weight"], s["epsilon"], s["positions"], s["frequencies"], s["neighbours"]) for name in ("q", "k")}
    outs = {"logprob": [], "entropy": [], "lse": [], "top_logprob": []}
    for r in range(0, case["rows"], 256):
        z = s["logits"][r:r + 256].double() * s["scale"]
        tokens = s["tokens"][r:r + 256].long()
        lse = torch.logsumexp(z, 1)
        log_p = torch.where(torch.isfinite(z), z - lse[:, None], -math.inf)
        outs["lse"].append(lse)
        outs["entropy"].append(torch.special.entr(torch.exp(log_p)).sum(1))
        outs["logprob"].append(torch.where(tokens >= 0, log_p[torch.arange(tokens.numel(), device=DEV), tokens.clamp(min=0)], 0.0))
        k = min(case["top"], case["vocabulary"])
        outs["top_logprob"].append(torch.nn.functional.pad(torch.topk(log_p, k, 1).values, (0, case["top"] - k), value=-math.inf))
    return {"logprob": torch.cat(outs["logprob"]), "entropy": torch.cat(outs["entropy"]), "lse": torch.cat(outs["lse"]), "top_tokens": None,
            "top_logprob": torch.cat(outs["top_logprob"])}
