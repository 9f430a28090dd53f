"""Plain models of the device-driven path for its tests: the free stacks and tables as Python lists, the
cache as logical rows, attention in 64 bits. They share nothing with the library but the block format's
definition (a unit of 8 elements u of token row r is stored at unit u ^ (r & 7) of its 64 elements)."""
from __future__ import annotations

import math

import numpy as np

NO_SLOT = -(1 << 63)
EINVAL, ENOSPC = -1, -2


def ceil_div(a, b):
    return -(-a // b)


class PoolModel:
    """Two stacks (lists, top at the end) and the calls' effect on tables, stated one block at a time."""

    def __init__(self, ids0, ids1, capacity=(math.inf, math.inf)):
        self.stacks = [list(ids0), list(ids1)]
        self.capacity = capacity

    def step(self, T, lens, new_lens, tables, max_tokens):
        """tables: list of dicts {block: entry}, changed in place. Returns (status, offsets, slots, positions)."""
        n, width = len(lens), self.width
        bad = any(x < 0 or x > width * T for x in list(lens) + list(new_lens))
        total = sum(max(0, b - a) for a, b in zip(lens, new_lens))
        empty = ([0] * (n + 1), [NO_SLOT] * max_tokens, [-1] * max_tokens)
        if bad or total > max_tokens:
            return (EINVAL,) + empty
        need = sum(max(0, ceil_div(b, T) - ceil_div(a, T)) for a, b in zip(lens, new_lens))
        if need > len(self.stacks[0]) + len(self.stacks[1]):
            return (ENOSPC,) + empty
        for i in range(n):
            for j in range(ceil_div(lens[i], T), ceil_div(new_lens[i], T)):
                tables[i][j] = self.stacks[0].pop() if self.stacks[0] else ~self.stacks[1].pop()
        offsets, slots, positions = [0], [], []
        for i in range(n):
            for pos in range(lens[i], new_lens[i]):
                e = tables[i][pos // T]
                slots.append(e * T + pos % T if e >= 0 else ~(~e * T + pos % T))
                positions.append(pos)
            offsets.append(len(slots))
        slots += [NO_SLOT] * (max_tokens - len(slots))
        positions += [-1] * (max_tokens - len(positions))
        status = 0
        for i in reversed(range(n)):
            for j in reversed(range(ceil_div(new_lens[i], T), ceil_div(lens[i], T))):
                e = tables[i][j]
                k = 0 if e >= 0 else 1
                if len(self.stacks[k]) < self.capacity[k]:
                    self.stacks[k].append(e if e >= 0 else ~e)
                else:
                    status = EINVAL
        return status, offsets, slots, positions


def stored_place(row, width):
    """Stored position of each of `width` columns in token row `row` of a block."""
    c = np.arange(width)
    return (c // 64) * 64 + ((((c % 64) // 8) ^ (row & 7)) * 8) + c % 8


def logical_rows(local, lent, table, length, T):
    """K and V rows of one sequence in 64 bits, [length][Hkv][D] each, read cell by cell from torch arenas."""
    import torch
    ref = local if local is not None and local.shape[0] else lent
    Hkv, D = ref.shape[3], ref.shape[4]
    out = torch.empty((2, length, Hkv * D), dtype=torch.float64, device=ref.device)
    place = torch.from_numpy(np.stack([stored_place(r, Hkv * D) for r in range(T)])).to(ref.device)
    for j in range(ceil_div(length, T)):
        e = int(table[j])
        block = local[e] if e >= 0 else lent[~e]
        rows = block.reshape(2, T, Hkv * D).double().gather(2, place[None].expand(2, -1, -1))
        k = min(T, length - j * T)
        out[:, j * T:j * T + k] = rows[:, :k]
    return out[0].reshape(length, Hkv, D), out[1].reshape(length, Hkv, D)


def attend(q, k, v, scale):
    """q [Hq][D], k and v [n][Hkv][D] in 64 bits: (out, lse, sum over dims of |q k| * |scale| at its largest)."""
    import torch
    Hq, Hkv = q.shape[0], k.shape[1]
    G = Hq // Hkv
    z = torch.einsum("hgd,nhd->hgn", q.reshape(Hkv, G, -1), k) * scale
    size = float((torch.einsum("hgd,nhd->hgn", q.reshape(Hkv, G, -1).abs(), k.abs()) * abs(scale)).max())
    w = torch.softmax(z, -1)
    out = torch.einsum("hgn,nhd->hgd", w, v).reshape(Hq, -1)
    return out, torch.logsumexp(z, -1).reshape(Hq), size


def row_error(n, D, size, vmax):
    """Bound on the error of one unrounded output element. The scores are f32 sums of D exact products (relative 2^-23 for each
    addition, as a tensor core may truncate), so each is off by at most D 2^-23 size, plus 2^-23 size for the scaling and 2^-22 for the
    exponential; a weight enters as two 16-bit numbers, the second one's rounding being 2^-16 of the weight (bf16); sums of n
    weights and n products are off by n 2^-23 of their size at most. A relative error d of every weight moves a weighted mean
    of numbers below vmax by at most 2 d vmax."""
    d = (D + 1) * 2.0 ** -23 * size + 2.0 ** -22 + 2.0 ** -16 + n * 2.0 ** -23
    return 2 * d * vmax


def close(got, ref, slack, eps):
    """|got - ref| <= half a step of the output type, relative to the value, plus slack (a number or an array); and in the 2-norm."""
    err = (got.double() - ref).abs()
    ok = bool((err <= eps / 2 * (ref.abs() + slack) + slack + 2.0 ** -25).all())
    return ok, float(err.max()) if err.numel() else 0.0


def lse_slack(n, D, size):
    return (D + 1) * 2.0 ** -23 * size + 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -22 * (size + math.log(max(n, 1)) + 1)
