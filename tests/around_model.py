"""Plain implementations of the calls around the attention, on the CPU in 64 bits, and how far the calls may be from them.

Rotation.  With u the unit roundoff of the 16-bit type, a value of a pair (a, b) of normed values differs by its rounding, u |y|, and by
what 32 bits lose on the way, relative to |a| + |b|: the sum of squares of 16 values in a lane and over 4 steps of lanes (20 * 2^-24, halved
by the root), the root's reciprocal (2 * 2^-24), two products (2 * 2^-24), the rotation's three operations, and cosine and sine, which are within 4 * 2^-24:
below 2^-19 in all.  Below the smallest normal value a rounding is half a subnormal step: 2^-134 for bfloat16, 2^-25 for float16.
"""
import torch

ROUNDOFF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def rotate(x, weight, epsilon, positions, frequencies, neighbours):
    """(outputs, bounds) of x [tokens, heads, dim]; a token of negative position has NaN."""
    dtype, y = x.dtype, x.double().cpu()
    if weight is not None:
        e = float(torch.tensor(epsilon, dtype=torch.float32))
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + e) * weight.double().cpu()
    half = 0 if frequencies is None else frequencies.numel()
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
    out, size = y.clone(), y.abs()
    if half:
        t = (positions.double().cpu()[:, None] * frequencies.double().cpu())[:, None, :]
        ya, yb = y[..., a], y[..., b]
        out[..., a], out[..., b] = ya * t.cos() - yb * t.sin(), yb * t.cos() + ya * t.sin()
        size[..., a] = size[..., b] = ya.abs() + yb.abs()
    out[positions.cpu() < 0] = float("nan")
    return out, ROUNDOFF[dtype] * out.abs() + 2.0 ** -19 * size + SMALLEST[dtype]


def near(got, want, bound):
    """Within the bound where the wanted value is finite, equal in kind where it is not."""
    got = got.double().cpu()
    fine = torch.isfinite(want)
    kinds = torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    return kinds and bool(((got - want).abs()[fine] <= bound[fine]).all())


def fork(table, lengths, parents, block, n_blocks, free):
    """Everything fikit_cache_fork writes, from the definitions, a child at a time; lists of Python numbers in and out.  None: too few blocks."""
    def pages(n):
        return -(-n // block)
    continued = {p for p in parents if p >= 0}
    kept = {b for p in continued for b in table[p][:pages(lengths[p])]}
    given = sorted({b for r, row in enumerate(table) for b in row[:pages(lengths[r])]} - kept)
    pool, taken, seen, copies, rows, new_lengths = list(free) + given, 0, set(), [], [], []
    for p in parents:
        n = lengths[p] if p >= 0 else 0
        row = list(table[p][:pages(n)]) if p >= 0 else []
        if n % block and p in seen:
            if taken == len(pool):
                return None
            copies.append([row[-1], pool[taken]])
            row[-1] = pool[taken]
            taken += 1
        seen.add(p)
        rows.append(row + [-1] * (len(table[0]) - len(row) if table else 0))
        new_lengths.append(n)
    left = pool[taken:]
    return {"block_table": rows, "lengths": new_lengths, "copies": copies + [[-1, -1]] * (len(parents) - len(copies)),
            "free_blocks": left + [-1] * (n_blocks - len(left)), "counts": [taken, len(given), len(left)]}


def compact(table, lengths, block, n_blocks, free):
    """Everything fikit_cache_compact writes, from the definitions."""
    held = [row[:-(-n // block)] for row, n in zip(table, lengths)]
    used = sorted({b for row in held for b in row})
    both = sorted(used + list(free))
    front, rest = set(both[:len(used)]), both[len(used):]
    moves = dict(zip([b for b in used if b not in front], sorted(front - set(used))))
    room = min(len(free), n_blocks // 2)
    return {"block_table": [[moves.get(b, b) for b in row] + [-1] * (len(table[0]) - len(row)) for row in held],
            "copies": [list(m) for m in moves.items()] + [[-1, -1]] * (room - len(moves)), "free_blocks": rest, "counts": [len(moves), len(used)]}


class Scores:
    """What fikit_token_scores says about logits [rows, V], in 64 bits, and how far it may be off.

    A term exp(z_j - max z) has the relative error e_j = 2^-22 (1 + |z_j| + |z_j - max z|) at most: the difference of logits and its product with scale * log2(e),
    itself rounded twice, are off by 4 * 2^-24 |z_j - max z|, as are the moves of sums from one largest logit to another, which add up to that difference at
    most; the exponentials of term and moves are within 2^-23 each, of which n below has its share.  Sums: a lane adds up V / 64 terms at most, then 20
    steps join lanes, waves and parts, n = (V / 64 + 20) 2^-24 in all.  So the sum's logarithm is off by sum p e + n and its own rounding 2^-22 (1 + |lse|),
    a log probability by e of its token besides, and the entropy sum p (-log p) by 2 sum p e (1 + |log p|) + 2 n (1 + sum p |z - max z|) + 2^-21 (1 + H)."""

    def __init__(self, logits, tokens, scale, top):
        x = logits.double().cpu()
        rows, v = x.shape
        inf = float("inf")
        z = x * float(torch.tensor(scale, dtype=torch.float32))
        odd = (torch.isnan(x) | (x == inf)).any(1)
        nothing = (x == -inf).all(1)
        fine = ~odd & ~nothing
        zz = torch.where(fine[:, None], z, torch.zeros(()).double())
        most = zz.amax(1, keepdim=True) if v else zz.new_zeros((rows, 1))
        beyond = torch.logsumexp(zz - most, 1)                      # (relative to the largest, whatever its size)
        lse = most[:, 0] + beyond
        log_p = zz - most - beyond[:, None]
        p = log_p.exp()
        size, away = torch.where(p > 0, zz.abs(), 0.0), torch.where(p > 0, (zz - most).abs(), 0.0)
        e = 2.0 ** -22 * (1 + size + away)
        n = (v / 64 + 20) * 2.0 ** -24
        minus_log = torch.where(p > 0, -log_p, 0.0)
        h = (p * minus_log).sum(1)
        self.bound = {"lse": (p * e).sum(1) + n + 2.0 ** -22 * (1 + lse.abs())}
        self.bound["entropy"] = 2 * (p * e * (1 + minus_log)).sum(1) + 2 * n * (1 + (p * away).sum(1)) + 2.0 ** -21 * (1 + h)

        def whole(values, of_nothing):
            return torch.where(odd, torch.nan, torch.where(nothing, of_nothing, values))
        self.want = {"lse": whole(lse, -inf), "entropy": whole(h, 0.0)}
        of_token = self.bound["lse"][:, None] + 2.0 ** -22 * (1 + z.abs() + (z - most).abs())
        values = torch.where(torch.isfinite(z) & fine[:, None], log_p, torch.full((), -inf).double())
        values = torch.where(odd[:, None], torch.nan, values)
        if tokens is not None:
            t = tokens.long().cpu()
            at = t.clamp(min=0)[:, None]
            given = t >= 0
            self.want["logprob"] = torch.where(given, values.gather(1, at)[:, 0], 0.0) if v else torch.zeros(rows).double()
            self.bound["logprob"] = torch.where(given, of_token.gather(1, at)[:, 0], 0.0) if v else torch.zeros(rows).double()
        order = torch.sort(torch.where(torch.isnan(x), -inf, x + 0.0), dim=1, descending=True, stable=True).indices[:, :top]
        there = torch.zeros((rows, top), dtype=torch.bool)
        there[:, :order.shape[1]] = torch.isfinite(z.gather(1, order)) & fine[:, None]
        order = torch.nn.functional.pad(order, (0, top - order.shape[1]))
        self.want["top_tokens"] = torch.where(there, order, -1)
        if v:
            self.want["top_logprob"] = torch.where(odd[:, None], torch.nan, torch.where(there, values.gather(1, order), -inf))
            self.bound["top_logprob"] = of_token.gather(1, order)
        else:
            self.want["top_logprob"], self.bound["top_logprob"] = torch.full((rows, top), -inf).double(), torch.zeros((rows, top)).double()

    def differs(self, got):
        """Names of the outputs that are not as wanted."""
        bad = []
        for name, want in self.want.items():
            g = getattr(got, name).cpu()
            if not (torch.equal(g.long(), want) if name == "top_tokens" else near(g, want, self.bound[name])):
                bad.append(name)
        return bad
