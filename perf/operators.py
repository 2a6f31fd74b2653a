"""The attention operators of a language model service as a user's program calls them, for timing and checking.

Four operators: the plan of a step over a paged cache (block tables, slots), the append of new keys and values into the
8-bit cache, the attention of a decode step over that cache, and the causal attention of packed prompts.  Where `own` is
false they are computed in their plain form, with elementary torch operations in 32 bits.

The cache holds OCP E4M3 codes, [blocks, kv heads, block tokens, head dim], and a biased power-of-two exponent per block
and head: a value is code * 2 ** (exponent - 127).  Lengths of a case come from its own `lengths` number, data from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
MOST_CODE = 448.0                      # largest E4M3 value


def listed():
    return [
        # the plan of one decode step of a busy service: every request gets one token; all latency
        dict(name="plan_step", op="plan", requests=256, cached_most=16384, added_most=1, prompts=0.0, block=64, lengths=1),
        # a batch of new prompts, nothing cached, odd lengths, small blocks
        dict(name="plan_prompts", op="plan", requests=64, cached_most=0, added_most=4096, prompts=1.0, block=16, lengths=2),
        # very many requests, most of them decoding, a tenth with a prompt or a continued prompt
        dict(name="plan_many", op="plan", requests=16384, cached_most=2048, added_most=1024, prompts=0.1, block=32, lengths=3),
        # the keys and values of one decode step: one token per request behind what its block holds
        dict(name="append_step", op="append", requests=256, cached_most=2048, added_most=1, prompts=0.0, block=64, kv_heads=8, dim=128,
             dtype="bf16", lengths=4),
        # new and continued prompts, several thousand tokens each
        dict(name="append_prompts", op="append", requests=16, cached_most=1000, added_most=4096, prompts=1.0, block=64, kv_heads=8, dim=128,
             dtype="bf16", lengths=5),
        # one user alone at an odd length: the latency of a token
        dict(name="decode_one", op="decode", requests=1, shortest=4097, longest=4097, block=64, q_heads=32, kv_heads=8, dim=128,
             dtype="bf16", lengths=6),
        # a batch of lengths from one token to 16384, heads of 64, every query head with keys of its own, small blocks
        dict(name="decode_ragged", op="decode", requests=64, shortest=1, longest=16384, block=16, q_heads=16, kv_heads=16, dim=64,
             dtype="f16", lengths=7),
        # two users with a very long context, many query heads to a key head
        dict(name="decode_long", op="decode", requests=2, shortest=65536, longest=131071, block=128, q_heads=64, kv_heads=4, dim=128,
             dtype="bf16", lengths=8),
        # a full service: the cache's bytes are all that counts
        dict(name="decode_full", op="decode", requests=128, shortest=4096, longest=16384, block=64, q_heads=32, kv_heads=8, dim=128,
             dtype="bf16", lengths=9),
        # a few short prompts, the first tokens of a chat
        dict(name="prompt_short", op="prompt", requests=5, shortest=1, longest=120, q_heads=16, kv_heads=16, dim=64, dtype="f16", lengths=10),
        # a batch of prompts of very different lengths
        dict(name="prompt_ragged", op="prompt", requests=24, shortest=1, longest=2048, q_heads=32, kv_heads=8, dim=128, dtype="bf16", lengths=11),
        # one long document
        dict(name="prompt_long", op="prompt", requests=1, shortest=8192, longest=8192, q_heads=32, kv_heads=8, dim=128, dtype="bf16", lengths=12),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["plan", "append", "decode", "prompt"])
    case = {"op": op, "lengths": rng.randrange(1 << 30)}
    dim = rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 5, 8])
    group = rng.choice([1, 3, 4, 6, 8, 16])
    dtype = rng.choice(["bf16", "f16"])
    block = rng.choice([16, 32, 64, 128])
    if op == "plan":
        requests = _log(rng, 1, 16384)
        return dict(case, requests=requests, cached_most=_log(rng, 1, 16384), added_most=_log(rng, 1, min(4096, max(1, 400000 // requests))),
                    prompts=rng.choice([0.0, 0.1, 1.0]), block=block)
    if op == "append":
        requests = _log(rng, 1, 512)
        return dict(case, requests=requests, cached_most=_log(rng, 1, 2048), added_most=_log(rng, 1, min(4096, max(1, 16384 // requests))),
                    prompts=rng.choice([0.1, 1.0]), block=block, kv_heads=kv_heads, dim=dim, dtype=dtype)
    if op == "decode":
        requests = _log(rng, 1, 256)
        return dict(case, requests=requests, shortest=1, longest=_log(rng, 1, min(131072, (1 << 23) // (requests * kv_heads))), block=block,
                    q_heads=kv_heads * group, kv_heads=kv_heads, dim=dim, dtype=dtype)
    kv_heads = min(kv_heads, 4)
    group = min(group, 8)
    longest = _log(rng, 1, 4096)
    requests = _log(rng, 1, min(64, max(1, (1 << 24) // longest ** 2)))
    return dict(case, requests=requests, shortest=1, longest=longest, q_heads=kv_heads * group, kv_heads=kv_heads, dim=dim, dtype=dtype)


def _spread(rng, low, high):
    """A length from low to high, spread over its logarithm."""
    return min(high, max(low, _log(rng, low, high)))


def _lengths(case):
    """(cached, added) per request for plan and append, the requests' lengths for the others."""
    rng = random.Random(case["lengths"])
    if case["op"] in ("plan", "append"):
        cached, added = [], []
        for _ in range(case["requests"]):
            prompt = rng.random() < case["prompts"]
            cached.append(rng.randint(0, case["cached_most"]))
            added.append(_spread(rng, 1, case["added_most"]) if prompt else 1)
        return cached, added
    return [_spread(rng, case["shortest"], case["longest"]) for _ in range(case["requests"])]


def _pieces(case):
    """How many pieces the new tokens are cut into by the blocks, and how many blocks are new."""
    b = case["block"]
    cached, added = _lengths(case)
    return (sum((c + a - 1) // b - c // b + 1 for c, a in zip(cached, added)),
            sum(-(-(c + a) // b) - -(-c // b) for c, a in zip(cached, added)))


def work(case):
    op = case["op"]
    if op == "plan":
        cached, added = _lengths(case)
        n, tokens = len(cached), sum(added)
        pieces, blocks = _pieces(case)
        return {"bytes": 8 * n + 4 * blocks + 4 * n + 4 * (n + 1) + 8 * tokens + 16 * pieces + 4 * blocks, "flops": 0}
    if op == "append":
        _, added = _lengths(case)
        pieces, _ = _pieces(case)
        values = 2 * sum(added) * case["kv_heads"] * case["dim"]
        return {"bytes": 3 * values + 16 * pieces + 2 * pieces * case["kv_heads"], "flops": 2 * values}
    lengths, hq, hkv, d = _lengths(case), case["q_heads"], case["kv_heads"], case["dim"]
    if op == "decode":
        blocks = sum(-(-n // case["block"]) for n in lengths)
        return {"bytes": 2 * sum(lengths) * hkv * d + 2 * blocks * hkv + 4 * blocks + 4 * len(lengths) * hq * (d + 1), "flops": 4 * sum(lengths) * hq * d}
    tokens = sum(lengths)
    return {"bytes": 2 * tokens * d * (2 * hq + 2 * hkv) + 4 * tokens * hq, "flops": 2 * d * hq * sum(n * (n + 1) for n in lengths)}


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _cache(case, gen, n_blocks):
    """A cache that earlier steps have filled: codes of normal values, exponents of values about one."""
    shape = (n_blocks, case["kv_heads"], case["block"], case["dim"])

    def codes():
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16).mul_(100.0).clamp_(-MOST_CODE, MOST_CODE).to(torch.float8_e4m3fn)

    def exponents():
        return torch.randint(119, 122, shape[:2], generator=gen, device=DEV, dtype=torch.uint8)
    return {"k_cache": codes(), "v_cache": codes(), "k_exp": exponents(), "v_exp": exponents()}


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    state = {"op": case["op"], "case": case, "status": torch.zeros(1, dtype=torch.int32, device=DEV)}
    if case["op"] in ("plan", "append"):
        b = case["block"]
        cached, added = _lengths(case)
        lengths = [c + a for c, a in zip(cached, added)]
        width = -(-max(lengths) // b)
        before = _int32([-(-c // b) for c in cached])
        n_blocks = sum(-(-n // b) for n in lengths) + 7
        order = torch.randperm(n_blocks, generator=gen, device=DEV).to(torch.int32)     # blocks are spread by earlier requests
        column = torch.arange(width, device=DEV)
        held = column[None, :] < before[:, None]
        n_held = int(held.sum())
        table = torch.full((len(cached), width), -1, dtype=torch.int32, device=DEV)
        table[held] = order[:n_held]
        state.update(cached=_int32(cached), added=_int32(added), n_tokens=sum(added), block=b, table=table, free=order[n_held:].contiguous())
        if case["op"] == "plan":
            return state
        dtype, hkv, d, n = DTYPES[case["dtype"]], case["kv_heads"], case["dim"], sum(added)
        # keys and values lie in one product's output, between its queries; some tokens and channels are much larger
        qkv = torch.randn((n, 3 * hkv, d), generator=gen, device=DEV, dtype=torch.float32)
        qkv *= torch.exp(torch.randn((n, 1, 1), generator=gen, device=DEV)) * torch.exp(torch.randn((1, 3 * hkv, d), generator=gen, device=DEV))
        qkv = qkv.to(dtype)
        state.update(_cache(case, gen, n_blocks), k=qkv[:, hkv:2 * hkv], v=qkv[:, 2 * hkv:])
        plan = _plan_plain(state)
        state["pieces"] = plan["pieces"]
        return state
    lengths, dtype, hq, hkv, d = _lengths(case), DTYPES[case["dtype"]], case["q_heads"], case["kv_heads"], case["dim"]
    state["scale"] = 1.0 / math.sqrt(d)
    state["longest"] = max(lengths)
    if case["op"] == "decode":
        b = case["block"]
        width = -(-max(lengths) // b)
        used = _int32([-(-n // b) for n in lengths])
        n_blocks = sum(-(-n // b) for n in lengths)
        order = torch.randperm(n_blocks, generator=gen, device=DEV).to(torch.int32)
        table = torch.full((len(lengths), width), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(width, device=DEV)[None, :] < used[:, None]] = order
        state.update(_cache(case, gen, n_blocks), lens=_int32(lengths), table=table,
                     q=torch.randn((len(lengths), hq, d), generator=gen, device=DEV, dtype=torch.float32).to(dtype))
        return state
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    qkv = torch.randn((int(offsets[-1]), hq + 2 * hkv, d), generator=gen, device=DEV, dtype=torch.float32).to(dtype)
    state.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], offsets=_int32(offsets.tolist()))
    return state


# ---- plain forms ------------------------------------------------------------------------------------------------

def _plan_plain(s):
    cached, added, b, n, table = s["cached"].long(), s["added"].long(), s["block"], s["n_tokens"], s["table"]
    requests, width = table.shape
    lengths = cached + added
    offsets = torch.cat([cached.new_zeros(1), torch.cumsum(added, 0)])
    before = (cached + b - 1) // b
    need = (lengths + b - 1) // b - before
    base = torch.cumsum(need, 0) - need
    token = torch.arange(n, device=DEV)
    request = torch.searchsorted(offsets, token, right=True) - 1
    index = token - offsets[request]
    at = cached[request] + index
    page = at // b
    opens = at % b == 0
    free = s["free"].long()
    fresh = torch.where(page >= before[request], free[(base[request] + page - before[request]).clamp(0, max(0, free.numel() - 1))], 0)
    flat = torch.cat([table.reshape(-1).long(), cached.new_zeros(1)])
    flat.scatter_(0, torch.where(opens, request * width + page, requests * width), fresh)
    full = flat[:-1].reshape(requests, width)
    block = full[request, page]
    # the pieces: a token leads one if it is its request's first or the first of its block
    leads = opens | (index == 0)
    rank = torch.cumsum(leads.long(), 0) - 1
    count = torch.minimum(b - at % b, lengths[request] - at)
    piece = torch.stack([block, token, at % b, count], 1)
    room = _room(n, requests, b)
    pieces = torch.full((room + 1, 4), -1, dtype=torch.int64, device=DEV)
    pieces.scatter_(0, torch.where(leads, rank, room)[:, None].expand(-1, 4), piece)
    return {"table": full.int(), "lengths": lengths.int(), "offsets": offsets.int(), "slots": block * b + at % b, "pieces": pieces[:room].int(),
            "counts": torch.stack([need.sum(), leads.sum()]).int()}


def _room(n_tokens, requests, block):
    """Most pieces that so many new tokens of so many requests can be cut into."""
    return min(n_tokens, n_tokens // block + 2 * requests)


def _power(exponents):
    return torch.exp2(exponents.float() - 127.0)


def _append_plain_one(codes, exponents, x, pieces):
    """Puts the pieces of x into the cache, in place."""
    b = codes.shape[2]
    raw = codes.view(torch.uint8)
    pieces = torch.where(pieces[:, :1] >= 0, pieces, pieces[:1]).long()                    # an unused entry repeats the first piece
    block, first, at, count = pieces[:, 0], pieces[:, 1:2], pieces[:, 2:3], pieces[:, 3:4]
    place = torch.arange(b, device=DEV)[None, :]
    new = (place >= at) & (place < at + count)                                              # [pieces, b]
    values = x.float()[torch.where(new, first + place - at, 0)].transpose(1, 2)             # [pieces, heads, b, d]
    new, earlier = new[:, None, :, None], (place < at)[:, None, :, None]
    most = torch.where(torch.isfinite(values) & new, values.abs(), 0.0).amax((2, 3))        # [pieces, heads]
    _, e = torch.frexp(most / MOST_CODE)                                                    # most / 448 = f * 2 ** e, f in [0.5, 1)
    e = torch.where(torch.ldexp(torch.full_like(most, MOST_CODE), e - 1) >= most, e - 1, e)  # (f = 0.5 needs one less)
    need = torch.where(most > 0, e + 127, 1).clamp(1, 254).long()
    old = exponents[block].long()
    chosen = torch.where(at > 0, torch.maximum(need, old), need)
    held = raw[block].view(torch.float8_e4m3fn).float()
    kept = held * torch.exp2((old - chosen).float())[:, :, None, None]
    scaled = torch.where(torch.isfinite(values), values * torch.exp2((127 - chosen).float())[:, :, None, None], math.nan)
    out = torch.where(new, scaled, torch.where(earlier, kept, held)).to(torch.float8_e4m3fn)
    raw[block] = out.view(torch.uint8)
    exponents[block] = chosen.to(torch.uint8)
    return codes, exponents


def _softmax_plain(scores, seen, values):
    """(rows' outputs, log of the rows' sums) of scores where `seen`; a row that sees nothing has outputs of zero."""
    scores = torch.where(seen, scores, -math.inf)
    most = scores.amax(-1, keepdim=True)
    most = torch.where(torch.isfinite(most), most, 0.0)
    p = torch.exp(scores - most)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, values) / torch.where(total > 0, total, 1.0)
    return out, (most + torch.log(total)).squeeze(-1)


def _decode_plain(s):
    table, lens = s["table"], s["lens"].long()
    requests, width = table.shape
    _, hkv, b, d = s["k_cache"].shape
    hq = s["q"].shape[1]
    block = table.clamp(min=0).long()

    def whole(codes, exponents):
        x = codes.view(torch.uint8)[block].view(torch.float8_e4m3fn).float() * _power(exponents[block])[..., None, None]    # [requests, width, hkv, b, d]
        return x.transpose(1, 2).reshape(requests, hkv, width * b, d)
    seen = torch.arange(width * b, device=DEV)[None, :] < lens[:, None]
    k = whole(s["k_cache"], s["k_exp"])
    q = s["q"].float().reshape(requests, hkv, hq // hkv, d)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    del k
    v = torch.where(seen[:, None, :, None], whole(s["v_cache"], s["v_exp"]), 0.0)
    out, lse = _softmax_plain(scores, seen[:, None, None, :], v)
    return {"out": out.reshape(requests, hq, d).to(s["q"].dtype), "lse": lse.reshape(requests, hq)}


def _prompt_plain(s):
    offsets = s["offsets"].long()
    longest = s["longest"]
    starts, counts = offsets[:-1], offsets[1:] - offsets[:-1]
    requests = starts.numel()
    n, hq, d = s["q"].shape
    hkv = s["k"].shape[1]
    place = torch.arange(longest, device=DEV)
    there = place[None, :] < counts[:, None]
    token = torch.where(there, starts[:, None] + place, 0)

    def padded(x):
        return torch.where(there[:, :, None, None], x.float()[token], 0.0).transpose(1, 2)      # [requests, heads, longest, d]
    q = padded(s["q"]).reshape(requests, hkv, hq // hkv * longest, d)
    scores = torch.matmul(q, padded(s["k"]).transpose(2, 3).contiguous()) * s["scale"]
    seen = (place[None, :] <= place[:, None]).repeat(hq // hkv, 1)
    out, lse = _softmax_plain(scores, seen, padded(s["v"]))
    out = out.reshape(requests, hq, longest, d).transpose(1, 2).reshape(requests * longest, hq, d)
    lse = lse.reshape(requests, hq, longest).transpose(1, 2).reshape(requests * longest, hq)
    token = torch.arange(n, device=DEV)
    request = torch.searchsorted(offsets, token, right=True) - 1
    row = request * longest + token - starts[request]
    return {"out": out[row].to(s["q"].dtype), "lse": lse[row]}


def run(state):
    s = state
    if own:
        from paper_2311_10359_amd import binding
        if s["op"] == "plan":
            plan = binding.fikit_cache_plan(s["cached"], s["added"], s["n_tokens"], s["block"], s["table"], s["free"], s["status"])
            return {"table": s["table"], "lengths": plan.lengths, "offsets": plan.token_offsets, "slots": plan.slots, "pieces": plan.pieces, "counts": plan.counts}
        if s["op"] == "append":
            binding.fikit_cache_append(s["k_cache"], s["v_cache"], s["k_exp"], s["v_exp"], s["k"], s["v"], s["pieces"], s["status"])
            return {"k": s["k_cache"], "v": s["v_cache"], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}
        if s["op"] == "decode":
            got = binding.fikit_cache_attention(s["q"], s["k_cache"], s["v_cache"], s["k_exp"], s["v_exp"], s["table"], s["lens"], s["scale"],
                                                s["status"], max_length=s["longest"])
            return {"out": got.out, "lse": got.lse}
        got = binding.fikit_prompt_attention(s["q"], s["k"], s["v"], s["offsets"], s["scale"], s["status"])
        return {"out": got.out, "lse": got.lse}
    if s["op"] == "plan":
        return _plan_plain(s)
    if s["op"] == "append":
        k, k_exp = _append_plain_one(s["k_cache"], s["k_exp"], s["k"], s["pieces"])
        v, v_exp = _append_plain_one(s["v_cache"], s["v_exp"], s["v"], s["pieces"])
        return {"k": k, "v": v, "k_exp": k_exp, "v_exp": v_exp}
    return _decode_plain(s) if s["op"] == "decode" else _prompt_plain(s)


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------

def _exact_rows(q, k, v, scale, causal):
    """Attention of the rows of q [rows, heads, d] over k, v [keys, kv heads, d], everything in 64 bits, a head at a time."""
    rows, hq, d = q.shape
    group = hq // k.shape[1]
    out, lse = q.new_zeros(q.shape), q.new_zeros((rows, hq))
    for h in range(hq):
        scores = (q[:, h] @ k[:, h // group].T) * scale
        if causal:
            scores.masked_fill_(torch.ones(scores.shape, dtype=torch.bool, device=scores.device).triu_(1), -math.inf)
        lse[:, h] = torch.logsumexp(scores, 1)
        out[:, h] = torch.exp(scores - lse[:, h, None]) @ v[:, h // group]
    return out, lse


def _exact_append(codes, exponents, x, pieces):
    """The codes before they are rounded."""
    new, old = codes.double().cpu().numpy(), exponents.cpu().numpy()
    x = x.double().cpu().numpy()
    for block, first, at, count in pieces.cpu().numpy():
        if block < 0:
            continue
        values = x[first:first + count].transpose(1, 0, 2)                       # [heads, count, d]
        for h in range(values.shape[0]):
            most = np.abs(values[h]).max()
            e = 1
            if most > 0:
                e = max(1, min(254, 127 + math.ceil(math.log2(most / MOST_CODE))))
                e += most > MOST_CODE * 2.0 ** (e - 127)
            if at > 0:
                e = max(e, int(old[block, h]))
                new[block, h, :at] *= 2.0 ** (int(old[block, h]) - e)
            new[block, h, at:at + count] = values[h] * 2.0 ** (127 - e)
    return torch.from_numpy(new)


def exact(case, seed):
    if case["op"] == "plan":
        return None                                                                # whole numbers only
    if case["op"] == "append":
        if sum(_lengths(case)[1]) * case["kv_heads"] > 400000:
            return None
        s = prepare(case, seed)
        return {"k": _exact_append(s["k_cache"], s["k_exp"], s["k"], s["pieces"]), "v": _exact_append(s["v_cache"], s["v_exp"], s["v"], s["pieces"]),
                "k_exp": None, "v_exp": None}
    lengths = _lengths(case)
    if case["op"] == "decode" and case["requests"] * case["q_heads"] > 100000:
        return None
    s = prepare(case, seed)
    outs, sums = [], []
    for r, n in enumerate(lengths):
        if case["op"] == "decode":
            pages = s["table"][r, :-(-n // case["block"])].long()

            def values(codes, exponents):
                x = codes.view(torch.uint8)[pages].view(torch.float8_e4m3fn).double() * torch.exp2(exponents[pages].double() - 127.0)[:, :, None, None]
                return x.transpose(1, 2).reshape(-1, case["kv_heads"], case["dim"])[:n]
            q, k, v = s["q"][r:r + 1].double(), values(s["k_cache"], s["k_exp"]), values(s["v_cache"], s["v_exp"])
        else:
            start = sum(lengths[:r])
            q, k, v = (s[x][start:start + n].double() for x in "qkv")
        out, lse = _exact_rows(q, k, v, s["scale"], case["op"] == "prompt")
        outs.append(out)
        sums.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(sums)}
