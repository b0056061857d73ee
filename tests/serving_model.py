"""The books of a pool and attention over its rows, written from their definitions: plain Python and 64-bit numpy / torch on the
CPU.  Nothing here is shared with the library."""
import math

import torch

FAULT_PAGE, FAULT_LIST, FAULT_NO_ROOM = 1, 2, 4


def pages_of(tokens, block):
    return -(-tokens // block)


class Books:
    """tables [rows][length], lens, refs as lists; `moved` collects what a call does to the data: (from, to, tokens)."""

    def __init__(self, n_rows, length, block, blocks):
        self.block, self.blocks, self.length = block, blocks, length
        self.tables = [[-1] * length for _ in range(n_rows)]
        self.lens, self.refs = [0] * n_rows, [0] * blocks
        self.err, self.moved = 0, []

    def free_list(self):
        return [p for p in range(self.blocks) if self.refs[p] <= 0]

    def _ok(self, page):
        return 0 <= page < self.blocks

    def grow(self, rows, counts=None):
        counts = [1] * len(rows) if counts is None else counts
        fault = 0
        fault |= FAULT_LIST if any(r < 0 for r in self.refs) else 0
        noted, needs, seen = fault, [], set()
        fault = 0
        for row, more in zip(rows, counts):
            if not 0 <= row < len(self.lens) or row in seen or not 0 <= self.lens[row] <= self.length * self.block or more < 0:
                fault |= FAULT_LIST
                continue
            seen.add(row)
            n = self.lens[row]
            if n + more > self.length * self.block:
                fault |= FAULT_NO_ROOM
                continue
            if n % self.block and more:
                page = self.tables[row][n // self.block]
                if not self._ok(page):
                    noted |= FAULT_PAGE
                elif self.refs[page] > 1:
                    fault |= FAULT_LIST
            needs.append(pages_of(n + more, self.block) - pages_of(n, self.block))
        free = self.free_list()
        if not fault and sum(needs) > len(free):
            fault |= FAULT_NO_ROOM
        self.err |= fault | noted
        if fault:
            return
        at = 0
        for row, more, need in zip(rows, counts, needs):
            held = pages_of(self.lens[row], self.block)
            for j in range(need):
                self.tables[row][held + j] = free[at]
                self.refs[free[at]] = 1
                at += 1
            self.lens[row] += more

    def fork(self, parents, children):
        self.err |= FAULT_LIST if any(r < 0 for r in self.refs) else 0
        fault, n_rows = 0, len(self.lens)
        for c in children:
            if not 0 <= c < n_rows or children.count(c) > 1 or self.lens[c] != 0:
                fault |= FAULT_LIST
        for p in parents:
            if not 0 <= p < n_rows or p in children or not 0 <= self.lens[p] <= self.length * self.block:
                fault |= FAULT_LIST
        free = self.free_list()
        if not fault and sum(self.lens[p] % self.block != 0 for p in parents) > len(free):
            fault |= FAULT_NO_ROOM
        self.err |= fault
        if fault:
            return
        at = 0
        for p, c in zip(parents, children):
            whole, part = divmod(self.lens[p], self.block)
            for j in range(whole):
                page = self.tables[p][j]
                self.tables[c][j] = page
                if self._ok(page):
                    self.refs[page] += 1
                else:
                    self.err |= FAULT_PAGE
            if part:
                self.tables[c][whole] = free[at]
                self.refs[free[at]] = 1
                if self._ok(self.tables[p][whole]):
                    self.moved.append((self.tables[p][whole], free[at], part))
                else:
                    self.err |= FAULT_PAGE
                at += 1
            self.lens[c] = self.lens[p]

    def free(self, rows):
        for row in rows:
            if not 0 <= row < len(self.lens):
                self.err |= FAULT_LIST
                continue
            n, self.lens[row] = self.lens[row], 0
            if not 0 <= n <= self.length * self.block:
                self.err |= FAULT_LIST
                continue
            for page in self.tables[row][:pages_of(n, self.block)]:
                if not self._ok(page):
                    self.err |= FAULT_PAGE
                elif self.refs[page] <= 0:
                    self.err |= FAULT_LIST
                else:
                    self.refs[page] -= 1

    def compact(self):
        """-> map, tables, refs; the books themselves stay."""
        self.err |= FAULT_LIST if any(r < 0 for r in self.refs) else 0
        used = [p for p in range(self.blocks) if self.refs[p] > 0]
        n = len(used)
        places = [p for p in range(n) if self.refs[p] <= 0]
        to = [-1] * self.blocks
        for p in used:
            to[p] = p
        for p, place in zip([p for p in used if p >= n], places):
            to[p] = place
            self.moved.append((p, place, self.block))
        refs = [0] * self.blocks
        for p in used:
            refs[to[p]] = self.refs[p]
        tables = [list(t) for t in self.tables]
        for t, k in zip(tables, self.lens):
            if not 0 <= k <= self.length * self.block:
                self.err |= FAULT_LIST
                continue
            for j in range(pages_of(k, self.block)):
                if not self._ok(t[j]):
                    self.err |= FAULT_PAGE
                elif to[t[j]] < 0:
                    self.err |= FAULT_LIST
                else:
                    t[j] = to[t[j]]
        return to, tables, refs


def attention(q, keys, values, seen, scale):
    """One row of a table and one KV head, in 64 bits.  q [n][G][D]; keys, values [tokens][D]; seen [n][tokens] bool.
    -> out [n][G][D], lse [n][G], and what the bounds of its rounding need: sum_j p_j |v_j|, the sum of |v_j| over the sum of
    weights, and the largest sum of |q k| that a row sees."""
    q, keys, values = q.double(), keys.double(), values.double()
    none = torch.full((), -math.inf, dtype=torch.float64)
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    spread, thin, size = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64)
    for i in range(q.shape[0]):
        k, v = keys[seen[i]], values[seen[i]]  # what is masked does not take part, whatever it holds
        if k.shape[0] == 0:
            continue
        s = q[i] @ k.T * scale
        top = s.amax(dim=-1, keepdim=True)
        w = torch.exp(s - torch.where(top == none, torch.zeros_like(top), top))
        total = w.sum(dim=-1, keepdim=True)
        out[i], lse[i] = (w / total) @ v, (top + torch.log(total))[:, 0]
        spread[i], thin[i] = (w / total) @ v.abs(), v.abs().sum(dim=0) / total
        size[i] = (q[i].abs() @ k.abs().T).amax(dim=-1) * scale
    return out, lse, spread, thin, size


def attention_bounds(out, lse, spread, thin, size, tokens, head_dim, dtype):
    """How far a result may be off.  u is half a step of the type, e = 2^-24 of 32-bit sums.
    Scores: head_dim products, exact, are summed in 32 bits, and scaled and shifted with one rounding each: e (head_dim + 4) times the sum of
    the terms' magnitudes; exp2 is off by 2 steps more.  Weights, numerator and denominator are off by twice that; the rounded
    weights by u (fp16 below 2^-14: by 2^-25); sums of `tokens` terms by e each; joining pieces and dividing by 16 e; the result by u."""
    u, e = torch.finfo(dtype).eps / 2, 2.0 ** -24
    score = e * ((head_dim + 4) * size + 4)
    share = (2 * score + (tokens + 16) * e).unsqueeze(-1) + u
    extra = 2.0 ** -25 * thin if dtype == torch.float16 else 0.0
    smallest = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134  # half the last step of the type
    return u * out.abs() + share * (1 + u) * spread + extra + smallest, score + (tokens + 16) * e + 4 * e * lse.abs()
