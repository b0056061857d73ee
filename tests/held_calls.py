"""Attention calls on pools in 4 bits that are compared so that nothing passes which is not within its bounds, NaN among it, and whose positions below the
prefix are the prefix row's."""
import math

import torch

import held_model as held
import serving_model as model
from test_gpu_held import Attend, HeldPool, i32

TORCH = held.TORCH


def compare(got, norm, want):
    """got, norm (None: not asked for): what the library gives; want: what the model does, with its bounds."""
    out, lse, off, lse_off = want
    far = ~((got.double() - out).abs() <= off)
    assert not far.any(), (int(far.sum()), float(((got.double() - out).abs() / off).max()))
    if norm is not None:
        none = lse == -math.inf
        assert torch.equal(norm == -math.inf, none)
        far = ~((norm.double() - lse)[~none].abs() <= lse_off[~none])
        assert not far.any(), (int(far.sum()), float(((norm.double() - lse).abs() / lse_off)[~none].max()))


class Call(Attend):
    def seen_of(self, row, hidden=None):
        """Keys and values of a row's positions, [0, its length) in whole pages, and which of them are not seen whatever the token."""
        d = self.d
        n = d.host_lens[row]
        pages = model.pages_of(n, d.block)
        kinds = [[], []]
        gone = torch.zeros(pages * d.block, dtype=torch.bool)
        cache = d.cache[1].cpu()
        tables = [d.host_tables[0], d.host_tables[row]]
        for table in tables:
            ok = [p if 0 <= p < d.blocks else 0 for p in (table + [-1] * pages)[:pages]]
            for kind in range(2):
                kinds[kind].append([x.flatten(0, 1) for x in d.form.get(cache[kind, ok], TORCH[self.dtype])])
        pos = torch.arange(pages * d.block)
        shared = pos < self.prefix
        for p in range(pages):
            for own in (0, 1):
                entry = tables[own][p] if p < len(tables[own]) else -1
                if not 0 <= entry < d.blocks:
                    gone |= (pos // d.block == p) & (shared != bool(own))
        gone |= shared & (pos >= d.host_lens[0])
        if hidden:
            gone |= torch.tensor([hidden(row, int(p)) for p in pos], dtype=torch.bool)
        pick = [[torch.where(shared.view(-1, *[1] * (x.dim() - 1)), x, y) for x, y in zip(*kind)] for kind in kinds]
        return pick, gone

    def model(self, hidden=None):
        d, H, G = self.d, self.H, self.G
        out, lse = torch.zeros((self.n, H * G, self.D), dtype=torch.float64), torch.full((self.n, H * G), -math.inf, dtype=torch.float64)
        off, lse_off = torch.zeros_like(out), torch.zeros((self.n, H * G), dtype=torch.float64)
        most = float(self.q.float().abs().max())
        for i, row in enumerate(self.rows):
            first, end, n = self.starts[i], self.starts[i + 1], d.host_lens[row]
            if first == end:
                continue
            (k, v), gone = self.seen_of(row, hidden)
            last = (n - (end - first) + torch.arange(end - first)).clamp(max=self.most_tokens - 1)
            seen = (torch.arange(len(gone))[None] <= last[:, None]) & ~gone[None]
            for h in range(H):
                part = held.attention(self.q[first:end, h * G:h * G + G], [x[:, h] for x in k], [x[:, h] for x in v], seen, self.scale, most)
                for whole, y in zip((out, lse, off, lse_off), part):
                    whole[first:end, h * G:h * G + G] = y
        return out, lse, off, lse_off

    def check(self, fault=0, hidden=None, **kw):
        got, norm = self.run(**kw)
        assert self.d.fault() == fault
        compare(got, norm, self.model(hidden))
        return got, norm

    def far(self):
        """The same call on a pool of more than 4 GiB of keys, its pages on both sides of 2 and 4 GiB."""
        small, form = self.d, self.d.form
        page = 4 * form.count
        blocks = (1 << 32) // page + 3 * small.blocks + 8
        half, whole = (1 << 31) // page, (1 << 32) // page
        places = [[i, half - i, half + 1 + i, whole - i, whole + 1 + i, blocks - 1 - i][i % 6] for i in range(small.blocks)]
        assert len(set(places)) == len(places) and max(places) < blocks and min(places) >= 0
        d = HeldPool.__new__(HeldPool)
        d.form, d.H, d.D, d.block, d.blocks, d.dtype, d.L = form, small.H, small.D, small.block, blocks, small.dtype, 2
        d.cache = torch.empty((2, blocks, form.count), dtype=torch.int32, device="cuda")
        d.cache[:, places] = small.cache[1]
        d.ptrs = torch.tensor([d.cache.data_ptr()] * 2, dtype=torch.int64, device="cuda")
        d.host_tables = [[places[p] if 0 <= p < small.blocks else -1 for p in t] for t in small.host_tables]
        d.tables, d.lens, d.err = i32(d.host_tables), small.lens, torch.zeros(1, dtype=torch.int32, device="cuda")
        p = small.pool
        d.pool = type(p)(2, self.H, self.D, p.dtype, blocks, small.block, len(small.host_lens), len(d.host_tables[0]), d.ptrs.data_ptr(), d.tables.data_ptr(),
                         d.lens.data_ptr(), None, d.err.data_ptr())
        return d
