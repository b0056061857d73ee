"""Pools in 4 bits: tokens written and read back, pages moved between 16 and 4 bits, the page calls, and attention, against tests/held_model.py."""
import math
import random

import pytest
import torch

import held_model as held
import kvc_harness as hz
import paper_2602_09725_amd as kvc
import serving_model as model

pytestmark = pytest.mark.gpu
TORCH = held.TORCH


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class HeldPool:
    """A pool in 4 bits whose pages are `words` (int32 [L][2][blocks][count] on the CPU; random ones by default)."""

    def __init__(self, tables, lens, H, D, block, blocks, dtype="f16", L=1, words=None, refs=None, seed=1):
        self.form = held.Words(H, D, block)
        self.H, self.D, self.block, self.blocks, self.dtype, self.L = H, D, block, blocks, dtype, L
        if words is None:
            g = torch.Generator().manual_seed(seed)
            words = torch.randint(-2 ** 31, 2 ** 31, (L, 2, blocks, self.form.count), generator=g, dtype=torch.int64).to(torch.int32)
        self.cache = words.cuda()
        self.ptrs = torch.tensor([c.data_ptr() for c in self.cache], dtype=torch.int64, device="cuda")
        length = max(len(t) for t in tables)
        self.host_tables, self.host_lens = [t + [-1] * (length - len(t)) for t in tables], list(lens)
        self.tables, self.lens = i32(self.host_tables), i32(self.host_lens)
        self.refs = None if refs is None else i32(refs)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.pool = kvc.Pool(L, H, D, (kvc.KVC_F16 if dtype == "f16" else kvc.KVC_BF16) | kvc.KVC_HELD_Q4, blocks, block, len(lens), length,
                             self.ptrs.data_ptr(), self.tables.data_ptr(), self.lens.data_ptr(), self.refs.data_ptr() if refs is not None else None,
                             self.err.data_ptr())
        assert kvc.page_bytes(self.pool) == 4 * self.form.count

    def fault(self):
        torch.cuda.synchronize()
        return int(self.err.item())

    def host(self):
        return self.cache.cpu().long() & 0xffffffff


def tokens_like(n, H, D, dtype, seed):
    """Tokens with heads of every kind: ordinary ones, one value all over, zeros of both signs, tiny and large ranges, one far element."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, H, D), generator=g).mul_(torch.exp(torch.rand((H, D), generator=g) * 2 - 1))
    kinds = torch.randint(0, 12, (n, H), generator=g)
    x[kinds == 1] = 1.2345
    x[kinds == 2] = 0.0
    x[kinds == 3] *= 1e-3 if dtype == "f16" else 1e-20
    x[kinds == 4] *= 3000.0 if dtype == "f16" else 1e20
    x[kinds == 5] += 100.0
    x[kinds == 6] = torch.where(x[kinds == 6] > 0, 1.0, -0.0)
    x[..., -1][kinds == 7] = 500.0
    x[kinds == 8] = torch.round(x[kinds == 8] * 4) / 4  # many ties
    x = x.to(TORCH[dtype])
    if dtype == "f16":
        x[kinds == 9] = torch.where(x[kinds == 9] > 0, 65504.0, -65504.0).to(torch.float16)
        x[kinds == 10] = torch.where(x[kinds == 10] > 0, 2.0 ** -24, -(2.0 ** -23)).to(torch.float16)
    return x


def paged(lens, block, blocks, seed, spare=1):
    order = list(range(blocks))
    random.Random(seed).shuffle(order)
    return [[order.pop() for _ in range(model.pages_of(n, block) + spare)] for n in lens]


SHAPES = [  # H, D, block
    (8, 128, 16), (1, 8, 4), (2, 40, 20), (3, 64, 8), (4, 96, 12), (1, 256, 32), (5, 24, 4), (2, 200, 64), (16, 16, 16),
]


@pytest.mark.parametrize("H,D,block", SHAPES)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_tokens_are_held_to_the_bit(kvc_lib, H, D, block, dtype):
    """Ragged requests at all places of a quad, in any order of rows; every other word of the pool stays."""
    rng = random.Random(H * D + block)
    new = [1, 2, 3, 4, 5, 0, 7, 13, 2 * block + 3, 1, 1, 6, 33]
    old = [rng.randint(0, 3 * block) for _ in new]
    lens = [n + o for n, o in zip(new, old)]
    d = HeldPool(paged(lens, block, 200, 3), lens, H, D, block, 200, dtype, L=2)
    rows = list(range(len(new)))
    rng.shuffle(rows)
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + new[r])
    n = starts[-1]
    k, v = tokens_like(n, H, D, dtype, 1), tokens_like(n, H, D, dtype, 2)
    want = d.host()
    for i, r in enumerate(rows):
        for j in range(new[r]):
            at = old[r] + j
            page, t = d.host_tables[r][at // block], starts[i] + j
            d.form.put(want[1, 0, page], at % block, k[t])
            d.form.put(want[1, 1, page], at % block, v[t])
    wide = torch.zeros((n, 2 * H + 1, D), dtype=TORCH[dtype], device="cuda")  # K and V of a projection, side by side
    wide[:, :H], wide[:, H:2 * H] = k.cuda(), v.cuda()
    at, begin = i32(rows), i32(starts)
    b = kvc.Batch(len(rows), n, max(new), at.data_ptr(), begin.data_ptr())
    kvc.kvc_append_paged(d.pool, b, 1, wide.data_ptr(), wide[:, H:].data_ptr(), wide.stride(0), hz.stream_handle())
    assert d.fault() == 0
    assert torch.equal(d.host(), want)
    # and back, into rows with room between them
    out = torch.full((2, n, H + 2, D), 7.0, dtype=TORCH[dtype], device="cuda")
    kvc.kvc_read_paged(d.pool, b, None, 1, out[0].data_ptr(), out[1].data_ptr(), out.stride(1), hz.stream_handle())
    assert d.fault() == 0
    for got, x in zip(out.cpu(), (k, v)):
        assert torch.equal(got[:, :H], held.rounded(held.stands_for(*held.quantized(x)), TORCH[dtype]))
        assert (got[:, H:] == 7.0).all()


def test_single_tokens(kvc_lib):
    """A step without a list of starts: request r is row r."""
    H, D, block, R = 2, 64, 8, 70
    lens = [1 + i for i in range(R)]
    d = HeldPool(paged(lens, block, 500, 5), lens, H, D, block, 500)
    k, v = tokens_like(R, H, D, "f16", 3), tokens_like(R, H, D, "f16", 4)
    want = d.host()
    for r in range(R):
        for kind, x in enumerate((k, v)):
            d.form.put(want[0, kind, d.host_tables[r][r // block]], r % block, x[r])
    kd, vd = k.cuda(), v.cuda()
    b = kvc.Batch(R)
    kvc.kvc_append_paged(d.pool, b, 0, kd.data_ptr(), vd.data_ptr(), H * D, hz.stream_handle())
    assert d.fault() == 0 and torch.equal(d.host(), want)
    out = torch.empty((2, R, H, D), dtype=torch.float16, device="cuda")
    kvc.kvc_read_paged(d.pool, b, None, 0, out[0].data_ptr(), out[1].data_ptr(), H * D, hz.stream_handle())
    assert torch.equal(out[0].cpu(), held.rounded(held.stands_for(*held.quantized(k)), torch.float16))
    assert torch.equal(out[1].cpu(), held.rounded(held.stands_for(*held.quantized(v)), torch.float16))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_heads_that_are_not_finite_read_back_as_nan(kvc_lib, dtype):
    H, D, block = 4, 40, 4
    x = torch.randn((4, H, D), generator=torch.Generator().manual_seed(1)).to(TORCH[dtype])
    x[0, 1, 7], x[1, 2, 0], x[2, 3, 39], x[3, 0, 3] = math.nan, math.inf, -math.inf, -math.nan
    if dtype == "bf16":
        x[3, 1, 0], x[3, 1, 1] = 3e38, -3e38  # their difference has no number in 32 bits
    d = HeldPool([[2]], [4], H, D, block, 5, dtype)
    xd, begin = x.cuda(), i32([0, 4])
    b = kvc.Batch(1, 4, 4, None, begin.data_ptr())
    kvc.kvc_append_paged(d.pool, b, 0, xd.data_ptr(), xd.data_ptr(), H * D, hz.stream_handle())
    out = torch.empty((2, 4, H, D), dtype=TORCH[dtype], device="cuda")
    kvc.kvc_read_paged(d.pool, b, None, 0, out[0].data_ptr(), out[1].data_ptr(), H * D, hz.stream_handle())
    want = held.rounded(held.stands_for(*held.quantized(x)), TORCH[dtype])
    assert int(torch.isnan(want).any(dim=-1).sum()) == (5 if dtype == "bf16" else 4)
    for got in out.cpu():
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())


def test_faults_of_writing_and_reading(kvc_lib):
    """A bad page, a row outside the table, a row shorter than its new tokens, tokens beyond the bound and between no requests."""
    H, D, block = 1, 64, 4
    tables = [[3, 99, 5], [-1, 7, 8], [9, 10, 11], [12, 13, 14]]
    lens = [10, 9, 2, 12]
    for what, rows, starts, most, first, want_fault, left_out in (
            ("page", [0, 1], [0, 10, 19], 10, None, model.FAULT_PAGE, set(range(4, 8)) | set(range(10, 14))),
            ("row", [4, 0], [0, 2, 4], 2, None, model.FAULT_LIST, {0, 1}),
            ("short", [2, 3], [0, 5, 8], 5, None, model.FAULT_LIST, {0, 1, 2}),
            ("bound", [3, 2], [0, 6, 7], 4, None, model.FAULT_LIST, {4, 5}),
            ("uncovered", [3, 2], [1, 3, 4], 4, None, model.FAULT_LIST, {0, 4}),
            ("first", [3, 3], [0, 3, 6], 3, [11, -1], model.FAULT_LIST, {1, 2, 3})):
        n = max(7, starts[-1]) if what in ("uncovered",) else starts[-1]
        if what == "uncovered":
            n, left_out = 5, {0, 4}
        d = HeldPool(tables, lens, H, D, block, 20)
        k = tokens_like(n, H, D, "f16", 5).cuda()
        at, begin, from_ = i32(rows), i32(starts), None if first is None else i32(first)
        b = kvc.Batch(len(rows), n, most, at.data_ptr(), begin.data_ptr())
        before = d.host()
        code, scale, mn = d.form.get(before[0].flatten(0, 1), torch.float16)
        values = held.rounded(held.stands_for(code, scale, mn), torch.float16).view(2, 20, block, H, D)
        out = torch.full((2, n, H, D), 7.0, dtype=torch.float16, device="cuda")
        kvc.kvc_read_paged(d.pool, b, None if first is None else from_.data_ptr(), 0, out[0].data_ptr(), out[1].data_ptr(), H * D, hz.stream_handle())
        assert d.fault() == want_fault, what
        where = {}
        for i, row in enumerate(rows):
            for t in range(starts[i], starts[i + 1]):
                at_ = (first[i] if first else (lens[row] if row < 4 else 0) - (starts[i + 1] - starts[i])) + t - starts[i]
                where[t] = (row, at_)
        for t in range(n):
            for kind in range(2):
                if t in left_out:
                    assert (out[kind, t] == 7.0).all(), (what, t)
                else:
                    row, pos = where[t]
                    want = values[kind, tables[row][pos // block], pos % block]
                    assert torch.equal(out[kind, t].cpu().nan_to_num(), want.nan_to_num()), (what, t)
        if first is not None:
            continue
        d.err.zero_()
        kvc.kvc_append_paged(d.pool, b, 0, k.data_ptr(), k.data_ptr(), H * D, hz.stream_handle())
        assert d.fault() == want_fault, what
        want = before
        for t in range(n):
            if t not in left_out:
                row, pos = where[t]
                for kind in range(2):
                    d.form.put(want[0, kind, tables[row][pos // block]], pos % block, k[t].cpu())
        assert torch.equal(d.host(), want), what


@pytest.mark.parametrize("block", [1, 4, 5, 33])
def test_reading_a_pool_of_16_bits(kvc_lib, block):
    H, D, blocks = 3, 40, 120
    lens = [50, 3 * block, 17, 1]
    tables = paged(lens, block, blocks, 4)
    length = max(len(t) for t in tables)
    cache = torch.randint(-32768, 32768, (2, blocks, block, H, D), dtype=torch.int16, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    tab, ln, ptr, err = i32([t + [-1] * (length - len(t)) for t in tables]), i32(lens), torch.tensor([cache.data_ptr()], device="cuda"), i32([0])
    pool = kvc.Pool(1, H, D, kvc.KVC_BF16, blocks, block, 4, length, ptr.data_ptr(), tab.data_ptr(), ln.data_ptr(), None, err.data_ptr())
    counts, first = [50, 2, 9, 1], [0, 1, 3, 0]
    starts = [0, 50, 52, 61, 62]
    begin, from_ = i32(starts), i32(first)
    out = torch.zeros((2, 62, H, D), dtype=torch.int16, device="cuda")
    b = kvc.Batch(4, 62, 50, None, begin.data_ptr())
    kvc.kvc_read_paged(pool, b, from_.data_ptr(), 0, out[0].data_ptr(), out[1].data_ptr(), H * D, hz.stream_handle())
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    for r in range(4):
        for i in range(counts[r]):
            pos = first[r] + i
            assert torch.equal(out[:, starts[r] + i], cache[:, tables[r][pos // block], pos % block]), (r, i)


@pytest.mark.parametrize("H,D,block", SHAPES)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_pages_between_the_pools(kvc_lib, H, D, block, dtype):
    L, blocks, other = 3, 9, 7
    wide = torch.stack([tokens_like(2 * blocks * block, H, D, dtype, 20 + i).view(2, blocks, block, H, D) for i in range(L)])
    d = HeldPool([[0]], [0], H, D, block, other, dtype, L=L)
    cache = wide.cuda()
    ptrs, err = torch.tensor([c.data_ptr() for c in cache], device="cuda"), i32([0])
    pool = kvc.Pool(L, H, D, kvc.KVC_F16 if dtype == "f16" else kvc.KVC_BF16, blocks, block, 1, 1, ptrs.data_ptr(), d.tables.data_ptr(),
                    d.lens.data_ptr(), None, err.data_ptr())
    src, dst = [8, 0, 3, 9, -1, 5], [6, 2, 0, 1, 4, 7]  # three pairs of pages that both pools have
    a, b = i32(src), i32(dst)
    want = d.host()
    for s, t in ((8, 6), (0, 2), (3, 0)):
        for layer in range(L):
            for kind in range(2):
                for slot in range(block):
                    d.form.put(want[layer, kind, t], slot, wide[layer, kind, s, slot])
    kvc.kvc_pages_convert(pool, d.pool, a.data_ptr(), b.data_ptr(), 6, hz.stream_handle())
    assert d.fault() == model.FAULT_PAGE and int(err.item()) == model.FAULT_PAGE
    assert torch.equal(d.host(), want) and torch.equal(cache.cpu().view(torch.int16), wide.view(torch.int16))
    d.err.zero_()
    err.zero_()
    again, back = i32([6, 2, 0]), i32([1, 2, 4])
    kvc.kvc_pages_convert(d.pool, pool, again.data_ptr(), back.data_ptr(), 3, hz.stream_handle())
    assert d.fault() == 0 and int(err.item()) == 0
    expect = wide.clone()
    for s, t in ((8, 1), (0, 2), (3, 4)):
        expect[:, :, t] = held.rounded(held.stands_for(*held.quantized(wide[:, :, s])), TORCH[dtype])
    assert torch.equal(cache.cpu().view(torch.int16), expect.view(torch.int16)) and torch.equal(d.host(), want)


@pytest.mark.parametrize("blocks", [40, 20000])
def test_page_calls_move_held_pages(kvc_lib, blocks):
    """A fork copies the parent's last page whole, copy and compact move pages as they are."""
    H, D, block = 2, 40, 4
    books = model.Books(6, 8, block, blocks)
    lens = [10, 0, 8, 0, 3, 0]
    order = list(range(5, blocks))
    random.Random(7).shuffle(order)
    for row, n in enumerate(lens):
        for j in range(model.pages_of(n, block)):
            books.tables[row][j] = order.pop()
            books.refs[books.tables[row][j]] = 1
        books.lens[row] = n
    d = HeldPool(books.tables, books.lens, H, D, block, blocks, L=2, refs=books.refs)
    space = torch.empty(kvc.pages_workspace(d.pool), dtype=torch.uint8, device="cuda")
    room = space.data_ptr(), space.numel(), hz.stream_handle()
    before = d.cache.clone()

    def check():
        assert d.fault() == books.err == 0
        assert (d.tables.tolist(), d.lens.tolist(), d.refs.tolist()) == (books.tables, books.lens, books.refs)
        want = before.clone()
        for source, place, _ in books.moved:
            want[:, :, place] = before[:, :, source]
        assert bool((d.cache == want).all())

    parents, children, rows, counts = i32([0, 0, 2]), i32([1, 3, 5]), i32([1, 3]), i32([1, 6])
    kvc.kvc_pages_fork(d.pool, parents.data_ptr(), children.data_ptr(), 3, *room)
    books.fork([0, 0, 2], [1, 3, 5])
    check()
    kvc.kvc_pages_grow(d.pool, rows.data_ptr(), counts.data_ptr(), 2, *room)
    books.grow([1, 3], [1, 6])
    check()
    gone, source, place = i32([0, 2]), i32([0, 1]), i32([33, 34])
    kvc.kvc_pages_free(d.pool, gone.data_ptr(), 2, hz.stream_handle())
    books.free([0, 2])
    check()
    before, books.moved = d.cache.clone(), []
    to = torch.empty(blocks, dtype=torch.int32, device="cuda")
    kvc.kvc_pages_compact(d.pool, to.data_ptr(), d.tables.data_ptr(), d.refs.data_ptr(), *room)
    places, books.tables, books.refs = books.compact()
    check()
    assert to.tolist() == places
    before, books.moved = d.cache.clone(), [(0, 33, block), (1, 34, block)]
    kvc.kvc_pages_copy(d.pool, source.data_ptr(), place.data_ptr(), 2, hz.stream_handle())
    check()


# ---- attention


def words_of(form, L, blocks, dtype, seed, pages=None):
    """Pages of tokens of every ordinary kind."""
    g = torch.Generator().manual_seed(seed)
    n = blocks * form.block
    out = torch.empty((L, 2, blocks, form.count), dtype=torch.int64)
    W, H, b = form.D // 8, form.H, form.block
    for layer in range(L):
        for kind in range(2):
            x = torch.randn((n, H, form.D), generator=g).mul_(torch.exp(torch.rand((H, form.D), generator=g) * 1.9 - 1.2))
            far = torch.rand((n, H), generator=g) < 0.05
            x[far] = x[far] * 4 + 3
            code, scale, mn = held.quantized(x.to(TORCH[dtype]))
            bits = lambda v: v.to(TORCH[dtype]).view(torch.int16).long() & 0xffff  # noqa: E731
            word = (code.view(n, H, W, 8) << torch.tensor([held.shift_of(i) for i in range(8)])).sum(dim=-1)
            word = word.view(blocks, b // 4, 4, H, W).permute(0, 3, 1, 4, 2).reshape(blocks, -1)
            pair = (bits(scale) | bits(mn) << 16).view(blocks, b, H).transpose(1, 2).reshape(blocks, -1)
            out[layer, kind] = torch.cat([word, pair], dim=1)
    return (out - (out >= 2 ** 31).long() * 2 ** 32).to(torch.int32)


class Attend:
    """A call of kvc_attend_paged on a held pool, and what the model says of it."""

    def __init__(self, new, owned, prefix, H, G, D, block, dtype, seed=1, most_tokens=None, cover=None):
        lens = [prefix + o for o in owned]
        shared = prefix // block
        rows = [model.pages_of(prefix, block)] + [max(0, model.pages_of(n, block) - shared) + 1 for n in lens]
        blocks = sum(rows) + 3
        order = list(range(blocks))
        random.Random(seed).shuffle(order)
        first = [order.pop() for _ in range(rows[0])]
        tables = [first] + [first[:shared] + [order.pop() for _ in range(k)] for k in rows[1:]]
        form = held.Words(H, D, block)
        words = words_of(form, 2, blocks, dtype, seed)
        if prefix % block:  # the prompt's last page, filled in part, is each row's own
            for t in tables[1:]:
                for slot in range(prefix % block):
                    at = [form.word(h, slot, w) for h in range(H) for w in range(D // 8)] + [form.pair(h, slot) for h in range(H)]
                    words[:, :, t[shared], at] = words[:, :, first[shared], :][:, :, at]
        self.d = HeldPool(tables, [prefix] + lens, H, D, block, blocks, dtype, L=2, words=words)
        self.H, self.G, self.D, self.dtype, self.prefix, self.new = H, G, D, dtype, prefix, new
        self.rows = list(range(1, len(new) + 1))
        random.Random(seed + 1).shuffle(self.rows)
        self.starts = [0]
        for r in self.rows:
            self.starts.append(self.starts[-1] + new[r - 1])
        self.n = self.starts[-1]
        g = torch.Generator().manual_seed(seed + 2)
        self.q = torch.randn((self.n, H * G, D), generator=g).to(TORCH[dtype])
        self.scale = 1 / math.sqrt(D)
        self.most_tokens = max(lens + [prefix]) if most_tokens is None else most_tokens
        self.at, self.begin = i32(self.rows), i32(self.starts)
        one = max(new) == 1 and min(new) == 1
        self.batch = kvc.Batch(len(new), self.n, max(new), self.at.data_ptr(), None if one else self.begin.data_ptr())

    def run(self, lse=True, q_pad=0, stream=None):
        H, G, D = self.H, self.G, self.D
        q = torch.full((self.n, H * G, D + q_pad), 9.0, dtype=TORCH[self.dtype], device="cuda")
        q[..., :D] = self.q.cuda()
        out = torch.full((self.n, H * G, D + q_pad), 7.0, dtype=TORCH[self.dtype], device="cuda")
        norm = torch.full((self.n, H * G), 7.0, device="cuda")
        a = kvc.Attention(H * G, self.scale, self.most_tokens, self.prefix, 0, q.stride()[:2], out.stride()[:2])
        size = kvc.attention_workspace(self.d.pool, self.batch, a)
        space = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
        kvc.kvc_attend_paged(self.d.pool, self.batch, a, 1, q.data_ptr(), out.data_ptr(), norm.data_ptr() if lse else None, space.data_ptr(), size,
                             hz.stream_handle())
        torch.cuda.synchronize()
        assert (out[..., D:] == 7.0).all()
        return out[..., :D].cpu(), norm.cpu() if lse else None

    def model(self, hidden=None):
        """hidden(row, position) -> bool: positions that are not seen for another reason."""
        d, H, G = self.d, self.H, self.G
        out, lse = torch.zeros((self.n, H * G, self.D), dtype=torch.float64), torch.zeros((self.n, H * G), dtype=torch.float64)
        off, lse_off = torch.zeros_like(out), torch.zeros_like(lse)
        cache = d.cache.cpu()
        for i, row in enumerate(self.rows):
            first, end, n = self.starts[i], self.starts[i + 1], d.host_lens[row]
            if first == end:
                continue
            pages = d.host_tables[row][:model.pages_of(n, d.block)]
            ok = [p if 0 <= p < d.blocks else 0 for p in pages]
            k, v = ([x.flatten(0, 1) for x in d.form.get(cache[1, kind, ok], TORCH[self.dtype])] for kind in range(2))
            seen = torch.zeros((end - first, len(pages) * d.block), dtype=torch.bool)
            for t in range(end - first):
                seen[t, :max(0, min(n - (end - first) + t + 1, self.most_tokens))] = True
            if hidden:
                for pos in range(seen.shape[1]):
                    if hidden(row, pos):
                        seen[:, pos] = False
            for h in range(H):
                part = held.attention(self.q[first:end, h * G:h * G + G], [x[:, h] for x in k], [x[:, h] for x in v], seen, self.scale, float(self.q.float().abs().max()))
                for whole, y in zip((out, lse, off, lse_off), part):
                    whole[first:end, h * G:h * G + G] = y
        return out, lse, off, lse_off

    def check(self, fault=0, hidden=None, **kw):
        got, norm = self.run(**kw)
        assert self.d.fault() == fault
        out, lse, off, lse_off = self.model(hidden)
        bad = (got.double() - out).abs() > off
        assert not bad.any(), (int(bad.sum()), float(((got.double() - out).abs() / off).max()))
        if norm is not None:
            none = lse == -math.inf
            assert torch.equal(norm.double() == -math.inf, none)
            wrong = (norm.double() - lse)[~none].abs() > lse_off[~none]
            assert not wrong.any(), (int(wrong.sum()), float(((norm.double() - lse).abs() / lse_off)[~none].max()))
        return got, norm


GRID = [  # new, owned, prefix, H, G, D, block
    ([1], [1], 0, 1, 1, 8, 4),
    ([1, 1, 1], [1, 64, 65], 0, 2, 4, 128, 16),
    ([1] * 4, [60, 1, 17, 33], 1000, 8, 4, 128, 16),
    ([1] * 5, [9, 300, 700, 1, 64], 333, 2, 7, 64, 8),
    ([1] * 20, [3 + 7 * i for i in range(20)], 130, 1, 8, 128, 32),
    ([3, 1, 9, 2], [3, 70, 200, 5], 77, 2, 3, 40, 20),
    ([40, 7, 64], [40, 90, 64], 0, 1, 4, 128, 16),
    ([33, 1], [500, 2], 600, 2, 2, 256, 32),
    ([1] * 3, [2000, 1500, 40], 0, 2, 16, 96, 16),
    ([5, 5], [5, 700], 4000, 1, 1, 24, 4),
    ([150], [150], 50, 1, 3, 200, 64),
    ([1], [20000], 0, 1, 2, 128, 16),
    ([1] * 130, [1 + i % 9 for i in range(130)], 515, 1, 2, 64, 16),
]


@pytest.mark.parametrize("case", range(len(GRID)))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention(kvc_lib, case, dtype):
    Attend(*GRID[case], dtype, seed=case).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_into_rows_with_gaps_and_without_logarithms(kvc_lib, dtype, D):
    Attend([2, 1, 30], [50, 3, 30], 100, 2, 2, D, 8, dtype).check(lse=False, q_pad=16)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("prefix", [0, 300])
def test_what_is_not_seen_may_be_held_with_anything(kvc_lib, dtype, prefix):
    """Slots behind a row's end, and pages that no row has, stand for NaN and infinities; a token that only later ones see likewise."""
    a = Attend([1, 6, 3, 20], [5, 70, 3, 400], prefix, 2, 4, 128, 16, dtype)
    d = a.d
    inf, nan = (0x7c00, 0x7e00) if dtype == "f16" else (0x7f80, 0x7fc0)
    taken = set()
    for row, table in enumerate(d.host_tables):
        for pos in range(d.host_lens[row]):
            taken.add((table[pos // d.block], pos % d.block))
    words = d.cache.cpu()
    for page in range(d.blocks):
        for slot in range(d.block):
            if (page, slot) not in taken:
                for h in range(a.H):
                    words[:, :, page, d.form.pair(h, slot)] = [nan, inf | nan << 16, inf | inf << 16, nan | 0x3c00 << 16][(page + slot + h) % 4]
    d.cache.copy_(words)
    a.check()
    row = max(range(1, 5), key=lambda r: d.host_lens[r])  # its last token: only the last new one sees it
    last = d.host_lens[row] - 1
    words[:, :, d.host_tables[row][last // d.block], [d.form.pair(h, last % d.block) for h in range(a.H)]] = nan
    d.cache.copy_(words)
    got, norm = a.run()
    out, lse, off, _ = a.model()
    i = a.rows.index(row)
    t = a.starts[i + 1] - 1
    assert torch.isnan(got[t]).all() and torch.isnan(norm[t]).all()
    others = [j for j in range(a.n) if j != t]
    assert ((got.double() - out).abs() <= off)[others].all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows_that_see_nothing(kvc_lib, dtype):
    """A row shorter than its new tokens, an empty one, a row outside the table: 0 and -inf, and the list is told to be at fault."""
    a = Attend([4, 1, 2], [4, 1, 2], 0, 2, 4, 64, 8, dtype)
    a.d.host_lens[1], a.d.host_lens[2] = 2, 0
    a.d.lens.copy_(i32(a.d.host_lens))
    got, norm = a.check(fault=0)
    assert (norm == -math.inf).any() and (got[norm == -math.inf] == 0).all()
    a.at[0] = 99
    got, norm = a.run()
    assert a.d.fault() == model.FAULT_LIST
    n = a.starts[1]
    assert (got[:n] == 0).all() and (norm[:n] == -math.inf).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("prefix", [0, 200])
def test_pages_outside_the_pool_are_not_seen(kvc_lib, dtype, prefix):
    a = Attend([1, 5, 40], [300, 90, 40], prefix, 2, 4, 128, 8, dtype)
    d = a.d
    bad = {}
    for row, places in ((1, [prefix // 8 + 2, prefix // 8 + 9]), (2, [prefix // 8 + 1])):
        for j in places:
            d.host_tables[row][j] = -1 if j % 2 else d.blocks
            bad.setdefault(row, set()).add(j)
    if prefix:
        for row in range(4):
            d.host_tables[row][3] = d.blocks + 5
            bad.setdefault(row, set()).add(3)
    d.tables.copy_(i32(d.host_tables))
    a.check(fault=model.FAULT_PAGE, hidden=lambda row, pos: pos // 8 in bad.get(row, ()))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_bound_below_the_rows(kvc_lib, dtype):
    a = Attend([1, 1, 2], [100, 300, 250], 0, 1, 4, 128, 16, dtype, most_tokens=256)
    a.check(fault=model.FAULT_LIST)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("size", [0, 1])
def test_queries_and_scales_of_all_sizes(kvc_lib, dtype, size):
    """Queries far from 1, one element far from the others, and values whose scales differ by powers of two from token to token."""
    a = Attend([2, 1, 3], [90, 200, 40], 150, 2, 4, 128, 16, dtype, seed=5)
    g = torch.Generator().manual_seed(9)
    power = torch.randint(-12, 5, (a.n, a.H * a.G, 1), generator=g).float() if dtype == "f16" else torch.randint(-60, 5, (a.n, a.H * a.G, 1), generator=g).float()
    a.q = (a.q.float() * torch.exp2(power)).to(TORCH[dtype]) if size else a.q * 8
    a.q[:, 0, 5] = 30.0
    a.q[:, 1] = 0.0
    d = a.d
    words = d.cache.cpu()
    lo = torch.randint(-8, 4, (d.blocks, d.block, a.H), generator=g) if dtype == "f16" else torch.randint(-60, 20, (d.blocks, d.block, a.H), generator=g)
    shared = {p for t in d.host_tables for p in t}
    for page in shared:  # the scale and the least value of a token move by the same power of two, exactly
        if page < 0:
            continue
        code, s, m = d.form.get(words[1, 1, page][None], TORCH[dtype])
        f = torch.exp2(lo[page].double())
        bits = lambda v: v.to(TORCH[dtype]).view(torch.int16).long() & 0xffff  # noqa: E731
        s, m = (s[0] * f).to(TORCH[dtype]), (m[0] * f).to(TORCH[dtype])
        for h in range(a.H):
            at = [d.form.pair(h, slot) for slot in range(d.block)]
            w = bits(s[:, h]) | bits(m[:, h]) << 16
            words[1, 1, page, at] = (w - (w >= 2 ** 31).long() * 2 ** 32).to(torch.int32)
    first = d.host_tables[0]
    if a.prefix % d.block:
        for t in d.host_tables[1:]:
            at = [d.form.pair(h, slot) for h in range(a.H) for slot in range(a.prefix % d.block)]
            words[1, 1, t[a.prefix // d.block], at] = words[1, 1, first[a.prefix // d.block], at]
    d.cache.copy_(words)
    a.check()
