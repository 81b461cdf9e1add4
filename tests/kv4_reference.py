"""The 4-bit cache by hand, in 64 bits: the format, the plan as a list of free blocks and a table, and the attention."""
import numpy as np
import torch

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
E_MIN, E_MAX = -111, 125


def held(x: torch.Tensor) -> torch.Tensor:
    """What x [..., head_dim] stands for once it is held in 4 bits (float64, CPU): groups of 32 with the least power of two
    2^e >= max|x| / 7, the nearest level, ties to the level with the even index."""
    a = np.ascontiguousarray(x.detach().cpu().double().numpy())
    g = a.reshape(*a.shape[:-1], -1, 32)
    out = np.empty_like(g)
    flat_in, flat_out = g.reshape(-1, 32), out.reshape(-1, 32)
    finite = np.isfinite(flat_in).all(1)
    top = np.where(finite, np.abs(np.where(np.isfinite(flat_in), flat_in, 0)).max(1), 1.0)
    m, e = np.frexp(top / 7.0 * (1 - 2.0 ** -50))   # top / 7 in [2^(e-1), 2^e), a power of two itself counted below
    e = np.where(top == 0, E_MIN, e)
    e = np.where((top > 0) & (np.ldexp(7.0, e - 1) >= top), e - 1, e)
    e = np.clip(e, E_MIN, E_MAX)
    unit = np.ldexp(1.0, e)[:, None]
    r = np.abs(np.where(finite[:, None], flat_in, 0)) / unit
    d = np.abs(r[..., None] - LEVELS)
    near = d.min(-1, keepdims=True)
    tie = d == near
    best = np.where(tie & (np.arange(8) % 2 == 0), 0, np.where(tie, 1, 2)).argmin(-1)
    flat_out[:] = np.where(finite[:, None], np.sign(flat_in) * LEVELS[best] * unit, np.nan)
    return torch.from_numpy(out.reshape(a.shape))


class Blocks:
    """Table and stack of free blocks, kept one request after the other."""

    def __init__(self, n_blocks, max_seqs, max_positions, block):
        self.block, self.max_positions = block, max_positions
        self.stack = list(range(n_blocks - 1, -1, -1))
        self.table = [[] for _ in range(max_seqs)]

    def need(self, tokens):
        return -(-tokens // self.block)

    def plan(self, held_, start, end, n_rows, max_rows_per_seq=None):
        n = len(held_)
        most = n_rows if max_rows_per_seq is None else min(n_rows, max_rows_per_seq)
        rows, ok = [], []
        at = 0
        for h, s, e in zip(held_, start, end):
            in_range = 0 <= s <= e <= self.max_positions
            r = e - s if in_range else 0
            ok.append(in_range and (s <= h or s == e) and 0 <= h <= self.max_positions and r <= most and (r == 0 or at + r <= n_rows))
            rows.append(r)
            at += r
        need = [self.need(end[i]) if ok[i] else len(self.table[i]) for i in range(n)]
        for i in reversed(range(n)):
            assert len(self.table[i]) == self.need(max(0, min(held_[i], self.max_positions))), "the lengths contradict the table"
            while len(self.table[i]) > need[i]:
                self.stack.append(self.table[i].pop())
        have, asked, served = len(self.stack), 0, []
        for i in range(n):
            want = need[i] - len(self.table[i])
            asked += want
            served.append(ok[i] and (want == 0 or asked <= have))
        for i in range(n):
            while served[i] and len(self.table[i]) < need[i]:
                self.table[i].append(self.stack.pop())
        slots, positions, row_seq, row_start = [], [], [], []
        for i in range(n):
            row_start.append(min(len(slots), n_rows))
            for p in range(start[i], start[i] + rows[i]):
                if len(slots) < n_rows:
                    slots.append(self.table[i][p // self.block] * self.block + p % self.block if served[i] else -1)
                    positions.append(p if served[i] else -1)
                    row_seq.append(i)
        row_start.append(len(slots))
        pad = [-1] * (n_rows - len(slots))
        return dict(slots=slots + pad, positions=positions + pad, row_seq=row_seq + pad, row_start=row_start, served=[int(s) for s in served],
                    held_next=[e if s else h for s, e, h in zip(served, end, held_)], n_free=[len(self.stack)])


def attend(q, k, v, positions, group, scale, window=0):
    """q [rows][heads][hd]; k, v [ctx][kv_heads][hd] (values as held); positions: of the rows, -1: sees nothing.
    -> out, lse, weight (the same sum over |v|: what errors of the weights are measured against), z_abs (largest sum of |q k| scale)"""
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    rows, heads, hd = q.shape
    out = torch.zeros(rows, heads, hd, dtype=torch.float64)
    weight = torch.zeros_like(out)
    lse = torch.full((rows, heads), -np.inf, dtype=torch.float64)
    pos = torch.as_tensor(positions)
    back = pos[:, None] - torch.arange(k.shape[0])[None, :]
    seen = (back >= 0) & (back < (window or 1 << 30)) & (pos[:, None] >= 0)
    some = seen.any(1)
    z_abs = 0.0
    for h in range(heads):
        kk, vv = k[:, h // group], v[:, h // group]
        z = torch.where(seen, q[:, h] @ kk.T * scale, -torch.inf)
        z_abs = max(z_abs, float(torch.where(seen, q[:, h].abs() @ kk.abs().T, 0.0).nan_to_num().max() * scale))
        lse[:, h] = torch.logsumexp(z, 1)
        w = torch.where(seen, torch.exp(z - torch.where(some, lse[:, h], 0.0)[:, None]), 0.0)
        out[:, h] = w @ vv
        weight[:, h] = w @ vv.abs()
    return out, lse, weight, z_abs
