"""Plain implementations of the attention calls, on the CPU in 64 bits, and how far the calls may be from them.

The bounds.  With u the unit roundoff of the 16-bit type (2^-8 for bfloat16, 2^-11 for float16), A = sum_j p_j |v_j| / sum_j p_j
per output, E the largest error of a score (as an exponent, so a relative error of its weight):

  a score is a product of `dim` exact 16-bit products summed in 32 bits, scaled, and an exponential of it:
      E = (dim + 8) 2^-24 scale sum |q_i| |k_i| + 2^-21 (1 + |score|)
  an output differs by the weights' rounding (u A), the outputs' rounding (u A), the scores' error in numerator and denominator
  (2 E A) and sums of n terms in 32 bits (2 n 2^-24 A); 1.1 times that for terms of second order, and 2^-24 for the f16 values
  and weights that are subnormal (n 2^-30 max |v| of the latter).
  the logarithm of the sum differs by E, n 2^-24 and its own rounding, 2^-21 (1 + |lse|).
"""
import math

import numpy as np
import torch

ROUNDOFF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
MOST_CODE = 448.0


def pieces_room(n_tokens, n_requests, block):
    return min(n_tokens, n_tokens // block + 2 * n_requests)


def plan(cached, added, block, table, free):
    """Everything fikit_cache_plan writes, from the definitions, a token at a time; `table` (numpy) is changed."""
    free = list(free)
    taken, slots, pieces, offsets = 0, [], [], [0]
    for r, (c, a) in enumerate(zip(cached, added)):
        held = -(-c // block)
        for page in range(held, -(-(c + a) // block)):
            table[r, page] = free[taken]
            taken += 1
        for i in range(a):
            place = c + i
            b = int(table[r, place // block])
            slots.append(b * block + place % block)
            if i == 0 or place % block == 0:
                pieces.append([b, offsets[-1] + i, place % block, 0])
            pieces[-1][3] += 1
        offsets.append(offsets[-1] + a)
    n = offsets[-1]
    counts = [taken, len(pieces)]
    pieces += [[-1] * 4] * (pieces_room(n, len(cached), block) - len(pieces))
    return {"lengths": [c + a for c, a in zip(cached, added)], "offsets": offsets, "slots": slots, "pieces": pieces, "counts": counts}


def round_codes(x):
    """The E4M3 bytes nearest to 64-bit values (|x| <= 448 or not finite), ties to even; NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    grid = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()      # 0 .. 448, ascending
    mag = np.where(np.isfinite(x), np.abs(x), 0.0)
    up = np.clip(np.searchsorted(grid, mag), 0, 126)
    down = np.maximum(up - 1, 0)
    to_up, to_down = grid[up] - mag, mag - grid[down]
    code = np.where((to_up < to_down) | ((to_up == to_down) & (up % 2 == 0)), up, down)
    code = np.where(mag == grid[up], up, code)
    code = code | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isfinite(x), code, 0x7f).astype(np.uint8)


def same_codes(a, b):
    """Equal bytes, NaN being equal to NaN of either sign."""
    return bool((((a == b) | (((a & 0x7f) == 0x7f) & ((b & 0x7f) == 0x7f)))).all())


def exponent_for(most):
    x = 1
    while x < 254 and most > MOST_CODE * 2.0 ** (x - 127):
        x += 1
    return x


def append(codes, exps, x, pieces):
    """Puts `pieces` of x [tokens, heads, dim] into the bytes codes [blocks, heads, block, dim], exps [blocks, heads]; in place."""
    x = x.double().numpy()
    for block, first, at, count in pieces:
        if block < 0:
            continue
        for h in range(codes.shape[1]):
            new = x[first:first + count, h]
            finite = np.abs(new[np.isfinite(new)])
            e = exponent_for(finite.max() if finite.size else 0.0)
            if at > 0:
                old = int(exps[block, h])
                if old > e:
                    e = old
                elif e > old:
                    held = torch.from_numpy(codes[block, h, :at].copy()).view(torch.float8_e4m3fn).double().numpy()
                    codes[block, h, :at] = round_codes(held * 2.0 ** (old - e))
            codes[block, h, at:at + count] = round_codes(new * 2.0 ** (127 - e))
            exps[block, h] = e


def cache_values(codes, exps, table_row, length, block):
    """[length, heads, dim] in 64 bits."""
    pages = table_row[:-(-length // block)].long()
    x = codes[pages].view(torch.float8_e4m3fn).double() * torch.exp2(exps[pages].double() - 127.0)[:, :, None, None]
    return x.transpose(1, 2).reshape(-1, codes.shape[1], codes.shape[3])[:length]


class Rows:
    """Attention of query rows [rows, heads, dim] over keys and values [keys, kv heads, dim], all in 64 bits; row i sees the first
    `sees[i]` keys."""

    def __init__(self, q, k, v, scale, sees, dtype):
        q, k, v = q.double(), k.double(), v.double()
        rows, heads, dim = q.shape
        group = heads // k.shape[1] if k.shape[1] else 1
        self.out, self.bound = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
        self.lse, self.lse_bound = torch.full((rows, heads), -math.inf, dtype=torch.float64), torch.zeros((rows, heads), dtype=torch.float64)
        u = ROUNDOFF[dtype]
        for i in range(rows):
            n = int(sees[i])
            if n == 0:
                continue
            kk = k[:n].repeat_interleave(group, 1)
            vv = v[:n].repeat_interleave(group, 1)
            s = (kk * q[i]).sum(2) * scale                                    # [n, heads]
            lse = torch.logsumexp(s, 0)
            p = torch.exp(s - lse)
            self.out[i] = (p[:, :, None] * vv).sum(0)
            self.lse[i] = lse
            e = ((dim + 8) * 2.0 ** -24 * abs(scale) * (kk * q[i]).abs().sum(2) + 2.0 ** -21 * (1 + s.abs())).amax(0)     # [heads]
            a = (p[:, :, None] * vv.abs()).sum(0)
            self.bound[i] = 1.1 * a * (2 * u + 2 * e[:, None] + 2 * n * 2.0 ** -24) + 2.0 ** -24 + n * 2.0 ** -30 * vv.abs().amax(0)
            self.lse_bound[i] = 1.1 * (e + n * 2.0 ** -24) + 2.0 ** -21 * (1 + lse.abs())


def near(got, want, bound):
    """Within the bound where the wanted value is finite, equal in kind where it is not."""
    got = got.double().cpu()
    fine = torch.isfinite(want)
    kinds = torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    return kinds and bool(((got - want).abs()[fine] <= bound[fine]).all())
