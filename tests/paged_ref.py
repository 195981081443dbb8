"""Paged cache and attention over it in float64 on the CPU, from the definitions, and the inputs of their tests.  Nothing here calls the library."""
import math

import torch

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Case:
    """Sequences with `new` tokens behind `past` ones in a pool whose pages lie in any order; slots that hold no token are NaN."""

    def __init__(self, dtype, H, H_kv, d_h, page, new, past, *, seed=0, order="heads", pad_rows=0, spare_columns=0, scale=1.0, value_shift=0.0):
        g = torch.Generator().manual_seed(1234 + seed)
        self.dtype, self.H, self.H_kv, self.d_h, self.page, self.new, self.past = DT[dtype], H, H_kv, d_h, page, list(new), list(past)
        self.B, self.G = len(new), H // H_kv
        self.total = [a + b for a, b in zip(new, past)]
        held = [-(-t // page) for t in self.total]
        self.pages = sum(held) + 3
        number = torch.randperm(self.pages, generator=g)
        width = max(max(held), 1) + spare_columns
        self.table = torch.full((self.B, width), -7, dtype=torch.int32)        # (entries behind a sequence's last page are nobody's)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = number[at:at + n].int()
            at += n
        self.start = torch.tensor([sum(new[:b]) for b in range(self.B + 1)], dtype=torch.int32)
        self.past_t = torch.tensor(past, dtype=torch.int32)
        self.rows = int(self.start[-1]) + pad_rows
        self.longest = max(new)
        randn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.k = [(randn(t, H_kv, d_h) + 0.5 * randn(1, H_kv, d_h)).to(self.dtype) for t in self.total]     # by sequence
        self.v = [(randn(t, H_kv, d_h) + value_shift).to(self.dtype) for t in self.total]
        self.Q = (scale * randn(max(self.rows, 1), H * d_h)).to(self.dtype)
        self.order = order
        self.K, self.V, self.bounds = self.pool()
        for b in range(self.B):
            self.fill(b, 0, self.total[b])

    def pool(self):
        shape = (self.pages, self.H_kv, self.page, self.d_h)
        kv = [torch.full(shape, math.nan, dtype=self.dtype) for _ in range(2)]
        return kv[0], kv[1], torch.full((self.pages, self.H_kv, 2, self.d_h), math.nan, dtype=self.dtype)

    def fill(self, b, lo, hi):
        """Tokens lo .. hi - 1 of sequence b into the pool, and the bounds of their pages."""
        for p in range(lo, hi):
            at = int(self.table[b, p // self.page])
            self.K[at, :, p % self.page] = self.k[b][p]
            self.V[at, :, p % self.page] = self.v[b][p]
        for j in range(lo // self.page, -(-hi // self.page) if hi > lo else 0):
            keys = self.k[b][j * self.page:min((j + 1) * self.page, hi)]
            at = int(self.table[b, j])
            self.bounds[at, :, 0] = keys.amin(0)
            self.bounds[at, :, 1] = keys.amax(0)

    def rows_of(self, b):
        return int(self.start[b]), int(self.start[b + 1])

    def on_gpu(self, pa):
        """cache and chunk on the device, the pool in the case's order."""
        def lay(x):
            x = x.cuda()
            return x if self.order == "heads" else x.transpose(1, 2).contiguous().transpose(1, 2)
        cache = pa.PagedCache(lay(self.K), lay(self.V), self.bounds.cuda())
        chunk = pa.Chunk(self.table.cuda(), self.start.cuda(), self.past_t.cuda(), rows=self.rows, longest=self.longest)
        return cache, chunk


def attend(c, causal, lists=None, drop=()):
    """out [rows, H * d_h] in float64 and, beside it, sum_s p_s |v_s| and the largest error that fp32 sums can make in a score.  lists: pages of
    every row and head of the cache; drop: (sequence, page) whose keys count as masked."""
    out = torch.zeros(c.rows, c.H, c.d_h, dtype=torch.float64)
    weight, err = torch.zeros_like(out), torch.zeros(c.rows, c.H, 1, dtype=torch.float64)
    for b in range(c.B):
        r0, r1 = c.rows_of(b)
        if r0 == r1:
            continue
        n, past, L = r1 - r0, c.past[b], c.total[b]
        see = torch.ones(n, L, dtype=torch.bool)
        if causal:
            see = torch.arange(L)[None] <= past + torch.arange(n)[:, None]
        for bb, j in drop:
            if bb == b:
                see[:, j * c.page:(j + 1) * c.page] = False
        for h in range(c.H):
            kv = h // c.G
            q = c.Q[r0:r1].view(n, c.H, c.d_h)[:, h].double()
            k, v = c.k[b][:, kv].double(), c.v[b][:, kv].double()
            mine = see
            if lists is not None:
                named = torch.zeros(n, -(-L // c.page), dtype=torch.bool)
                for i in range(n):
                    named[i, lists[r0 + i][kv]] = True
                mine = see & named.repeat_interleave(c.page, dim=1)[:, :L]
            s = (q @ k.t() / math.sqrt(c.d_h)).masked_fill(~mine, -math.inf)
            p = torch.nan_to_num(torch.softmax(s, dim=1))
            out[r0:r1, h] = p @ v
            weight[r0:r1, h] = p @ v.abs()
            size = ((q.abs() @ k.abs().t()) / math.sqrt(c.d_h)).masked_fill(~mine, 0.0)
            err[r0:r1, h, 0] = size.amax(1) * (c.d_h + 8) * 2.0 ** -24
    return out.flatten(1), weight.flatten(1), err.expand(-1, -1, c.d_h).flatten(1)


def tolerance(c, ref, weight, err, weight_step):
    """An output is rounded by half a step of its type.  A weight's relative error is its score's absolute one, twice (numerator and sum), what the
    exponential (2^-22, its argument's rounding included), the sum of up to `longest` of them and the weights' own rounding (weight_step) add."""
    half = torch.finfo(c.dtype).eps / 2
    n = max(c.total)
    return half * ref.abs() + (2 * err + 2 * weight_step + 2.0 ** -20 + (n + 64) * 2.0 ** -24) * weight + 1e-30


def scores(c, b, row, kv):
    """score of every page of sequence b for a row and a head of the cache, in float64."""
    q = c.Q[row].view(c.H, c.d_h)[kv * c.G:(kv + 1) * c.G].double()
    at = c.table[b, :-(-c.total[b] // c.page)].long()
    low, high = c.bounds[at, kv, 0].double(), c.bounds[at, kv, 1].double()
    return torch.maximum(q[:, None] * low, q[:, None] * high).sum(-1).amax(0)


def select(c, budget, first, last, causal, bad=()):
    """The chosen pages of every row and head of the cache; bad: (sequence, page) with no page in the pool."""
    lists = []
    for row in range(c.rows):
        b = next((b for b in range(c.B) if c.rows_of(b)[0] <= row < c.rows_of(b)[1]), None)
        if b is None:
            lists.append(None)
            continue
        pos = c.past[b] + row - c.rows_of(b)[0]
        have = (pos if causal else c.total[b] - 1) // c.page + 1
        mine = []
        for kv in range(c.H_kv):
            s = scores(c, b, row, kv).tolist()
            lo = min(first, have)
            hi = max(lo, have - last)
            ok = [j for j in range(have) if (b, j) not in bad]
            forced = [j for j in ok if j < lo or j >= hi]
            free = budget - lo - (have - hi)
            best = sorted((j for j in ok if lo <= j < hi), key=lambda j: (-s[j], j))[:max(free, 0)]
            mine.append(sorted(forced + best))
        lists.append(mine)
    return lists


def rope_table(positions, rot, theta=10000.0):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.stack((angle.cos(), angle.sin()), dim=-1).float()


def head(x, w, eps, table, pos, pairs):
    """Norm and rotation of rows x [n, heads, d_h] at positions pos, in float64, and the sum of magnitudes that each output column is made of."""
    x = x.double()
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    size = x.abs()
    if table is None:
        return x, size
    half = table.shape[1]
    cos, sin = table[pos][:, None, :, 0].double(), table[pos][:, None, :, 1].double()
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
    y, size = x.clone(), size.clone()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size
