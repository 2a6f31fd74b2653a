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
