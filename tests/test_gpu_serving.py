"""Pages of a pool, appended tokens and attention over pages, against tests/serving_model.py."""
import math
import random

import pytest
import torch

import kvc_harness as hz
import paper_2602_09725_amd as kvc
import serving_model as model

pytestmark = pytest.mark.gpu
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class DevicePool:
    """Books and caches on the device; the caches hold `fill` where a test writes nothing."""

    def __init__(self, books, L, H, D, dtype="f16", caches=None, refs=True):
        self.books, self.L, self.H, self.D, self.dtype = books, L, H, D, dtype
        self.caches = caches
        if caches is None:
            g = torch.Generator(device="cuda")
            g.manual_seed(7)
            self.caches = [torch.randint(-32768, 32768, (2, books.blocks, books.block, H * D), generator=g, device="cuda", dtype=torch.int16)
                           for _ in range(L)]
        self.ptrs = torch.tensor([c.data_ptr() for c in self.caches], dtype=torch.int64, device="cuda")
        self.tables, self.lens, self.refs = i32(books.tables), i32(books.lens), i32(books.refs)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.pool = kvc.Pool(L, H, D, kvc.KVC_F16 if dtype == "f16" else kvc.KVC_BF16, books.blocks, books.block, len(books.lens), books.length,
                             self.ptrs.data_ptr(), self.tables.data_ptr(), self.lens.data_ptr(), self.refs.data_ptr() if refs else None,
                             self.err.data_ptr())
        self.space = torch.full((kvc.pages_workspace(self.pool),), 0xA5, dtype=torch.uint8, device="cuda")

    def room(self):
        return self.space.data_ptr(), self.space.numel(), hz.stream_handle()

    def check(self, before=None):
        torch.cuda.synchronize()
        assert int(self.err.item()) == self.books.err
        assert self.lens.tolist() == self.books.lens
        assert self.refs.tolist() == self.books.refs
        assert self.tables.tolist() == self.books.tables
        if before is not None:
            self.check_data(before)

    def check_data(self, before):
        """The pages are as they were, but for what the model moved."""
        for c, b in zip(self.caches, before):
            want = b.clone()
            for source, place, tokens in self.books.moved:
                want[:, place, :tokens] = b[:, source, :tokens]
            assert torch.equal(c, want)

    def copy(self):
        return [c.clone() for c in self.caches]


def filled(n_rows, length, block, blocks, lens, seed, shared=0):
    """Books whose rows have pages of their own in random order; the first `shared` rows' pages have another holder."""
    rng = random.Random(seed)
    books = model.Books(n_rows, length, block, blocks)
    free = list(range(blocks))
    rng.shuffle(free)
    for row, n in enumerate(lens):
        for j in range(model.pages_of(n, block)):
            books.tables[row][j] = free.pop()
            books.refs[books.tables[row][j]] = 1 + (row < shared)
        books.lens[row] = n
    return books


SHAPES = [  # L, H, D, block
    (2, 2, 16, 16), (1, 1, 8, 1), (3, 8, 128, 16), (2, 3, 40, 5), (1, 4, 128, 64), (5, 1, 256, 33),
]


@pytest.mark.parametrize("L,H,D,block", SHAPES)
def test_copy(kvc_lib, L, H, D, block):
    books = model.Books(1, 1, block, 40)
    d = DevicePool(books, L, H, D)
    before = d.copy()
    src, dst = [3, 39, 7, 0, 7], [4, 5, 38, 1, 2]
    d.books.moved = [(s, t, block) for s, t in zip(src, dst)]
    a, b = i32(src), i32(dst)
    kvc.kvc_pages_copy(d.pool, a.data_ptr(), b.data_ptr(), len(src), hz.stream_handle())
    d.check(before)


def test_copy_leaves_out_pages_beyond_the_pool(kvc_lib):
    books = model.Books(1, 1, 16, 12)
    d = DevicePool(books, 2, 2, 64)
    before = d.copy()
    a, b = i32([-1, 12, 3, 4, 5]), i32([1, 2, 12, -7, 6])
    books.moved, books.err = [(5, 6, 16)], model.FAULT_PAGE
    kvc.kvc_pages_copy(d.pool, a.data_ptr(), b.data_ptr(), 5, hz.stream_handle())
    d.check(before)


@pytest.mark.parametrize("L,H,D,block", SHAPES)
@pytest.mark.parametrize("blocks", [70, 4096, 4097, 9000])
def test_fork_grow_and_free(kvc_lib, L, H, D, block, blocks):
    if blocks > 4096 and H * D * block * L > 10000:
        L, H, D = 1, 1, 8
    lens = [5 * block + 3 % block, 0, 1, 2 * block, 0, 0, 0, 0, block - 1, 0]
    books = filled(10, 9, block, blocks, lens, seed=blocks + block)
    for page in range(blocks // 2, blocks - 5):  # few are free at the low end, and they lie in all segments
        if books.refs[page] == 0 and page % 7:
            books.refs[page] = 1
    d = DevicePool(books, L, H, D)
    before = d.copy()
    parents, children = i32([0, 0, 2, 3, 8]), i32([7, 1, 5, 4, 9])
    kvc.kvc_pages_fork(d.pool, parents.data_ptr(), children.data_ptr(), 5, *d.room())
    books.fork([0, 0, 2, 3, 8], [7, 1, 5, 4, 9])
    d.check(before)
    rows = i32([5, 7, 6, 1, 9])
    counts = i32([1, 2 * block, block + 1, 0, 1])
    kvc.kvc_pages_grow(d.pool, rows.data_ptr(), counts.data_ptr(), 5, *d.room())
    books.grow([5, 7, 6, 1, 9], [1, 2 * block, block + 1, 0, 1])
    d.check(before)
    kvc.kvc_pages_grow(d.pool, rows.data_ptr(), None, 2, *d.room())
    books.grow([5, 7])
    d.check(before)
    gone = i32([0, 7, 7, 6, 1, 4])  # row 7 twice
    kvc.kvc_pages_free(d.pool, gone.data_ptr(), 6, hz.stream_handle())
    books.free([0, 7, 7, 6, 1, 4])
    d.check(before)
    assert books.err == 0


LONG = 700


def test_long_lists(kvc_lib):
    """More entries than a workgroup has threads, and rows that take many pages from several segments."""
    books = filled(2 * LONG + 1, 40, 4, 20000, [4 * (i % 9) + i % 4 for i in range(LONG)], seed=3)
    for page in range(20000):
        if books.refs[page] == 0 and page % 3 == 0:
            books.refs[page] = 1
    d = DevicePool(books, 1, 1, 8)
    before = d.copy()
    parents, children = list(range(LONG)), list(range(2 * LONG - 1, LONG - 1, -1))
    a, b = i32(parents), i32(children)
    kvc.kvc_pages_fork(d.pool, a.data_ptr(), b.data_ptr(), LONG, *d.room())
    books.fork(parents, children)
    d.check(before)
    counts = [(7 * i) % 100 for i in range(LONG)]
    c = i32(counts)
    kvc.kvc_pages_grow(d.pool, b.data_ptr(), c.data_ptr(), LONG, *d.room())
    books.grow(children, counts)
    d.check(before)
    kvc.kvc_pages_free(d.pool, a.data_ptr(), LONG, hz.stream_handle())
    books.free(parents)
    d.check(before)
    assert books.err == 0


@pytest.mark.parametrize("what", ["twice", "row", "not empty", "chain", "no room", "length"])
def test_a_fork_that_cannot_be_changes_nothing(kvc_lib, what):
    books = filled(8, 6, 4, 12, [9, 10, 11, 0, 0, 0, 0, 3], seed=1)
    parents, children = [0, 1, 2], [3, 4, 5]
    if what == "twice":
        children = [3, 4, 3]
    elif what == "row":
        parents = [0, 8, 2]
    elif what == "not empty":
        children = [3, 7, 5]
    elif what == "chain":
        parents = [0, 3, 2]
    elif what == "no room":
        for page in range(12):
            books.refs[page] = max(books.refs[page], 1)
        books.refs[books.tables[7][0]] = 0
    else:
        books.lens[1] = 25
    d = DevicePool(books, 1, 1, 8)
    before = d.copy()
    a, b = i32(parents), i32(children)
    kvc.kvc_pages_fork(d.pool, a.data_ptr(), b.data_ptr(), 3, *d.room())
    books.fork(parents, children)
    assert books.err == (model.FAULT_NO_ROOM if what == "no room" else model.FAULT_LIST)
    d.check(before)


@pytest.mark.parametrize("what", ["twice", "row", "negative", "full", "no room", "shared", "length", "huge"])
def test_a_grow_that_cannot_be_changes_nothing(kvc_lib, what):
    books = filled(5, 6, 4, 16, [9, 0, 23, 4, 5], seed=2, shared=1 if what == "shared" else 0)
    rows, counts = [0, 1, 3], [1, 9, 4]
    want = model.FAULT_LIST
    if what == "twice":
        rows = [0, 1, 0]
    elif what == "row":
        rows = [0, -1, 3]
    elif what == "negative":
        counts = [1, -1, 4]
    elif what == "full":
        rows, want = [0, 1, 2], model.FAULT_NO_ROOM
    elif what == "no room":
        counts, want = [15, 24, 20], model.FAULT_NO_ROOM
    elif what == "length":
        books.lens[1] = -3
    elif what == "huge":
        counts, want = [1, 2 ** 31 - 1, 4], model.FAULT_NO_ROOM
    d = DevicePool(books, 1, 1, 8)
    before = d.copy()
    a, b = i32(rows), i32(counts)
    kvc.kvc_pages_grow(d.pool, a.data_ptr(), b.data_ptr(), 3, *d.room())
    books.grow(rows, counts)
    assert books.err == want
    d.check(before)


def test_free_and_fork_leave_out_what_is_wrong(kvc_lib):
    books = filled(6, 4, 4, 20, [9, 12, 5, 0, 8, 0], seed=4)
    books.tables[0][1], books.tables[1][0] = 20, -5
    books.refs[books.tables[2][0]] = 0
    books.lens[4] = 17
    d = DevicePool(books, 2, 1, 16)
    before = d.copy()
    a, b = i32([0, 1]), i32([3, 5])
    kvc.kvc_pages_fork(d.pool, a.data_ptr(), b.data_ptr(), 2, *d.room())
    books.fork([0, 1], [3, 5])
    assert books.err == model.FAULT_PAGE
    d.check(before)
    gone = [0, 9, 1, 2, 4, -1, 3]
    c = i32(gone)
    kvc.kvc_pages_free(d.pool, c.data_ptr(), len(gone), hz.stream_handle())
    books.free(gone)
    assert books.err == model.FAULT_PAGE | model.FAULT_LIST
    d.check(before)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("L,H,D,block,blocks,used", [
    (2, 2, 16, 16, 60, 25), (1, 1, 8, 1, 9000, 4100), (1, 1, 8, 4, 8192, 4096), (3, 8, 128, 16, 70, 69), (2, 3, 40, 5, 100, 0), (1, 1, 8, 2, 64, 64),
    (1, 1, 8, 4, 5000, 1), (2, 1, 256, 200, 20, 9),
])
def test_compact(kvc_lib, L, H, D, block, blocks, used, in_place):
    rows = 7
    cut = [used * i // rows for i in range(rows + 1)]
    lens = [max(0, (b - a) * block - (i if block > i and b > a else 0)) for i, (a, b) in enumerate(zip(cut, cut[1:]))]
    books = filled(rows + 3, max(1, max(model.pages_of(n, block) for n in lens)) + 2, block, blocks, lens, seed=used + blocks)
    if lens[0] > block:  # a fork of two rows' first pages
        for row in (0, 1):
            books.tables[rows + row][0] = books.tables[row][0]
            books.refs[books.tables[row][0]] += 1
            books.lens[rows + row] = block
    d = DevicePool(books, L, H, D)
    before = d.copy()
    where = torch.full((blocks,), 77, dtype=torch.int32, device="cuda")
    tables, refs = (d.tables, d.refs) if in_place else (torch.full_like(d.tables, 55), torch.full_like(d.refs, 55))
    kvc.kvc_pages_compact(d.pool, where.data_ptr(), tables.data_ptr(), refs.data_ptr(), *d.room())
    want = books.compact()
    torch.cuda.synchronize()
    assert (where.tolist(), tables.tolist(), refs.tolist()) == want
    assert int(d.err.item()) == books.err == 0
    d.check_data(before)
    if not in_place:
        d.check()


def test_compact_goes_on_where_entries_are_wrong(kvc_lib):
    books = filled(4, 5, 4, 30, [17, 9, 20, 4], seed=9)
    books.tables[0][1], books.tables[1][2] = 30, -2
    books.refs[books.tables[2][1]] = 0
    books.refs[29 if books.refs[29] == 0 else 28] = -3
    books.lens[3] = 21
    d = DevicePool(books, 2, 1, 16)
    before = d.copy()
    where, tables, refs = torch.empty_like(d.refs), torch.empty_like(d.tables), torch.empty_like(d.refs)
    kvc.kvc_pages_compact(d.pool, where.data_ptr(), tables.data_ptr(), refs.data_ptr(), *d.room())
    want = books.compact()
    torch.cuda.synchronize()
    assert (where.tolist(), tables.tolist(), refs.tolist()) == want
    assert int(d.err.item()) == books.err == model.FAULT_PAGE | model.FAULT_LIST
    d.check_data(before)


# ---- pools on both sides of what one workgroup looks after: 16384 pages, lists of 1024 entries


def half_taken(books, seed):
    rng = random.Random(seed)
    for page in range(books.blocks):
        if books.refs[page] == 0 and rng.random() < 0.6:
            books.refs[page] = 1
    return books


@pytest.mark.parametrize("entries", [1, 1024, 1025])
@pytest.mark.parametrize("blocks", [16383, 16384, 16385, 50000])
def test_lists_and_pools_of_many_pages(kvc_lib, blocks, entries):
    lens = [3 * (i % 5) + i % 3 for i in range(entries)]
    books = half_taken(filled(2 * entries + 1, 24, 3, blocks, lens, seed=entries), blocks)
    d = DevicePool(books, 1, 1, 8)
    before = d.copy()
    parents, children = list(range(entries)), list(range(2 * entries - 1, entries - 1, -1))
    a, b = i32(parents), i32(children)
    kvc.kvc_pages_fork(d.pool, a.data_ptr(), b.data_ptr(), entries, *d.room())
    books.fork(parents, children)
    d.check(before)
    counts = [(5 * i + 1) % 12 for i in range(entries)]
    c = i32(counts)
    kvc.kvc_pages_grow(d.pool, b.data_ptr(), c.data_ptr(), entries, *d.room())
    books.grow(children, counts)
    d.check(before)
    kvc.kvc_pages_free(d.pool, a.data_ptr(), entries, hz.stream_handle())
    books.free(parents)
    d.check(before)
    assert books.err == 0


@pytest.mark.parametrize("blocks", [40, 20000])
@pytest.mark.parametrize("what", ["twice", "no room", "exactly enough", "bad page", "count below 0"])
def test_faults_in_pools_of_any_size(kvc_lib, blocks, what):
    """A list at fault changes nothing, in small pools as in large ones; the last free page can be taken."""
    books = filled(8, 5, 4, blocks, [9, 6, 4, 0, 0, 0], seed=blocks)
    free = [page for page in range(blocks) if books.refs[page] == 0]
    if what in ("no room", "exactly enough"):  # two forks need a page each
        for page in free[:-2] if what == "exactly enough" else free[:-1]:
            books.refs[page] = 1
    if what == "bad page":
        books.tables[0][2] = blocks
    if what == "count below 0":
        books.refs[free[3]] = -1
    children = [3, 3, 5] if what == "twice" else [3, 4, 5]
    d = DevicePool(books, 2, 1, 16)
    before = d.copy()
    a, b = i32([0, 1, 2]), i32(children)
    kvc.kvc_pages_fork(d.pool, a.data_ptr(), b.data_ptr(), 3, *d.room())
    books.fork([0, 1, 2], children)
    want = {"twice": model.FAULT_LIST, "no room": model.FAULT_NO_ROOM, "exactly enough": 0, "bad page": model.FAULT_PAGE,
            "count below 0": model.FAULT_LIST}[what]
    assert books.err == want
    d.check(before)
    if what == "exactly enough":  # and now there is none
        c, counts = i32([2, 0]), i32([1, 1])
        kvc.kvc_pages_grow(d.pool, c.data_ptr(), counts.data_ptr(), 2, *d.room())
        books.grow([2, 0], [1, 1])
        assert books.err == model.FAULT_NO_ROOM
        d.check(before)


@pytest.mark.parametrize("blocks,used", [(16384, 1), (16384, 16384), (16384, 5000), (16385, 8191), (16385, 16385), (40000, 0), (33000, 20000)])
def test_compact_of_many_pages(kvc_lib, blocks, used):
    lens = [2 * (used // 4)] * 4 + [2 * (used % 4)]
    books = filled(6, max(1, used), 2, blocks, lens, seed=used)
    d = DevicePool(books, 1, 1, 8)
    before = d.copy()
    where, tables, refs = torch.empty_like(d.refs), torch.empty_like(d.tables), torch.empty_like(d.refs)
    kvc.kvc_pages_compact(d.pool, where.data_ptr(), tables.data_ptr(), refs.data_ptr(), *d.room())
    want = books.compact()
    torch.cuda.synchronize()
    assert (where.tolist(), refs.tolist()) == (want[0], want[2])
    assert torch.equal(tables, i32(want[1]))
    assert int(d.err.item()) == books.err == 0
    d.check_data(before)


# ---- append

BATCHES = [  # tokens of the rows after the call, new ones of each (None: one each)
    ([1, 40, 17, 5], None), ([7], [7]), ([30, 64, 1, 33, 20], [30, 0, 1, 17, 20]), ([300, 299, 40], [290, 250, 3]),
]


def starts_of(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


@pytest.mark.parametrize("L,H,D,block", SHAPES)
@pytest.mark.parametrize("lens,new", BATCHES)
def test_append(kvc_lib, L, H, D, block, lens, new):
    n_rows = len(lens) + 2
    order = list(range(n_rows))
    random.Random(block).shuffle(order)
    rows = order[:len(lens)]
    by_row = [0] * n_rows
    for r, n in zip(rows, lens):
        by_row[r] = n
    books = filled(n_rows, max(model.pages_of(n, block) for n in lens), block, 20 + sum(model.pages_of(n, block) for n in lens), by_row, seed=block)
    d = DevicePool(books, L, H, D, refs=False)
    before = d.copy()
    counts = [1] * len(lens) if new is None else new
    n, wide = sum(counts), H * D * 2 + 24
    x = torch.randint(-32768, 32768, (n, wide), device="cuda", dtype=torch.int16)
    k, v = x[:, 8:8 + H * D], x[:, 16 + H * D:16 + 2 * H * D]
    where, starts = i32(rows), i32(starts_of(counts))
    layer = L - 1
    kvc.kvc_append_paged(d.pool, kvc.Batch(len(lens), n, max(counts), where.data_ptr(), None if new is None else starts.data_ptr()), layer, k.data_ptr(),
                         v.data_ptr(), wide, hz.stream_handle())
    want = before[layer].clone()
    t = 0
    for r, length, c in zip(rows, lens, counts):
        for i in range(c):
            at = length - c + i
            page = books.tables[r][at // block]
            want[0, page, at % block], want[1, page, at % block] = k[t], v[t]
            t += 1
    d.check()
    for i, c in enumerate(d.caches):
        assert torch.equal(c, want if i == layer else before[i])


def test_append_leaves_out_what_has_no_place(kvc_lib):
    books = filled(4, 3, 4, 20, [9, 3, 12, 5], seed=6)
    books.tables[0][2], books.lens[3] = 20, 13
    d = DevicePool(books, 1, 1, 8, refs=False)
    before = d.copy()
    rows, starts = i32([0, 1, 2, 3, 9]), i32([0, 2, 6, 8, 9, 10])  # row 1 has three tokens and should have four new ones
    x = torch.randint(-32768, 32768, (10, 8), device="cuda", dtype=torch.int16)
    kvc.kvc_append_paged(d.pool, kvc.Batch(5, 10, 4, rows.data_ptr(), starts.data_ptr()), 0, x.data_ptr(), x.data_ptr(), 8, hz.stream_handle())
    want = before[0].clone()
    t = books.tables
    want[:, t[0][1], 3] = x[0]
    for i in range(3):
        want[:, t[1][0], i] = x[3 + i]
    want[:, t[2][2], 2], want[:, t[2][2], 3] = x[6], x[7]
    books.err = model.FAULT_PAGE | model.FAULT_LIST
    d.check()
    assert torch.equal(d.caches[0], want)


# ---- attention


class Attend:
    """A pool of one or more layers whose rows share a prefix held by row 0, and a batch of its other rows.  Slots that hold no
    token hold NaN."""

    def __init__(self, H, G, D, dtype, block, prefix, lens, new, seed=0, most_tokens=None, slack=3, spare=0, scale=None, layers=1, spread=1.0,
                 first_page=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rng = random.Random(seed)
        self.H, self.G, self.D, self.dtype, self.block, self.prefix = H, G, D, TORCH[dtype], block, prefix
        self.new = [1] * len(lens) if new is None else new
        self.one_each = new is None
        n_rows = len(lens) + 2
        self.rows = list(range(1, n_rows))
        rng.shuffle(self.rows)
        self.rows = self.rows[:len(lens)]
        shared = prefix // block
        longest = max([prefix, 1, most_tokens or 0] + lens)
        length = model.pages_of(longest, block) + 1
        need = model.pages_of(prefix, block) + sum(max(0, model.pages_of(n, block) - shared) for n in lens)
        blocks = first_page + need + slack
        books = model.Books(n_rows, length, block, blocks)
        free = list(range(first_page, blocks))
        rng.shuffle(free)
        for j in range(model.pages_of(prefix, block)):
            books.tables[0][j] = free.pop()
        books.lens[0] = prefix
        for r, n in zip(self.rows, lens):
            for j in range(model.pages_of(n, block)):
                books.tables[r][j] = books.tables[0][j] if j < shared else free.pop()
            books.lens[r] = n
        self.books, self.lens = books, lens
        self.caches = [torch.full((2, blocks, block, H, D), math.nan, dtype=self.dtype, device="cuda") for _ in range(layers)]
        self.layer = layers - 1
        cache = self.caches[self.layer]
        for r in [0] + self.rows:
            n = books.lens[r]
            start = 0 if r == 0 else min(n, shared * block)
            for at in range(start, n, block):
                page, count = books.tables[r][at // block], min(block, n - at)
                x = torch.randn((2, count, H, D), generator=g, device="cuda") * spread
                if r and at < prefix:  # what a fork copied
                    same = min(prefix - at, count)
                    x[:, :same] = cache[:, books.tables[0][at // block], :same].float()
                cache[:, page, :count] = x.to(self.dtype)
        n = sum(self.new)
        heads = H * G
        self.q_store = torch.full((n, heads + 1, D + 8), math.nan, dtype=self.dtype, device="cuda")
        self.q = self.q_store[:, :heads, :D]
        self.q.copy_(torch.randn((n, heads, D), generator=g, device="cuda").to(self.dtype))
        self.out_store = torch.full((n, heads, D + 16), 7.0, dtype=self.dtype, device="cuda")
        self.out = self.out_store[:, :, :D]
        self.lse = torch.full((n + 1, heads), 7.0, device="cuda")
        self.scale = D ** -0.5 if scale is None else scale
        self.device = DevicePool(books, layers, H, D, dtype, self.caches, refs=False)
        self.where, self.starts = i32(self.rows), i32(starts_of(self.new))
        self.batch = kvc.Batch(len(lens), n, max(self.new + [1]), self.where.data_ptr(), None if self.one_each else self.starts.data_ptr())
        self.most = max([prefix] + lens) if most_tokens is None else most_tokens
        self.attention = kvc.Attention(heads, self.scale, self.most, prefix, 0, self.q.stride()[:2], self.out.stride()[:2])
        self.space = torch.full((kvc.attention_workspace(self.device.pool, self.batch, self.attention),), 0xFF, dtype=torch.uint8, device="cuda")

    def call(self, lse=True):
        kvc.kvc_attend_paged(self.device.pool, self.batch, self.attention, self.layer, self.q.data_ptr(), self.out.data_ptr(),
                             self.lse.data_ptr() if lse else None, self.space.data_ptr(), self.space.numel(), hz.stream_handle())

    def check(self, err=0, lens=None, missing=None, skip=()):
        """missing: (row or None for the prefix, position) pairs that are not seen.  skip: requests that are not looked at."""
        torch.cuda.synchronize()
        assert int(self.device.err.item()) == err
        assert bool((self.out_store[:, :, self.D:] == 7.0).all()) and bool((self.lse[-1] == 7.0).all()), "wrote beside the result"
        lens = self.lens if lens is None else lens
        cache = self.caches[self.layer].cpu()
        flat = cache.flatten(1, 2)
        got, got_lse, q = self.out.double().cpu(), self.lse[:-1].double().cpu(), self.q.double().cpu()
        starts = starts_of(self.new)
        for request, (r, n) in enumerate(zip(self.rows, lens)):
            if request in skip:
                continue
            t0, c = starts[request], self.new[request]
            if c == 0:
                continue
            positions = torch.arange(n)
            blocks = positions // self.block
            own, front = torch.tensor(self.books.tables[r]), torch.tensor(self.books.tables[0])
            page = torch.where(positions < self.prefix, front[blocks], own[blocks]).long()
            there = (page >= 0) & (page < self.books.blocks)
            for who, at in missing or ():
                if at < n and (who is None or who == r):
                    there[at] = False
            slots = page.clamp(0, self.books.blocks - 1) * self.block + positions % self.block
            seen = (positions[None] <= (n - c + torch.arange(c))[:, None]) & there[None]
            for h in range(self.H):
                heads = slice(h * self.G, h * self.G + self.G)
                want = model.attention(q[t0:t0 + c, heads], flat[0, slots, h], flat[1, slots, h], seen, self.scale)
                far, far_lse = model.attention_bounds(*want, n, self.D, self.dtype)
                self.near(f"out of request {request}, head {h}", got[t0:t0 + c, heads], want[0], far)
                self.near(f"lse of request {request}, head {h}", got_lse[t0:t0 + c, heads], want[1], far_lse)

    @staticmethod
    def near(name, got, want, far):
        finite = torch.isfinite(want)
        assert bool((torch.isnan(got) == torch.isnan(want)).all()), name
        assert bool((got[~finite & ~torch.isnan(want)] == want[~finite & ~torch.isnan(want)]).all()), name
        off = (got - want).abs()[finite]
        assert bool((off <= far[finite]).all()), f"{name}: off by {float((off / far[finite]).max()):.3g} times what rounding allows"


# H, G, D, block, prefix, lens of the rows, new tokens of each
ATTEND = [
    (2, 4, 128, 16, 100, [101, 140, 117], None),           # decoding: four rows of queries a head
    (1, 1, 64, 16, 0, [1], None),                          # one token sees itself
    (1, 1, 128, 1, 3, [4, 5], None),                       # pages of one token
    (2, 1, 64, 16, 40, [41, 60, 300], [1, 20, 250]),       # ragged questions
    (1, 7, 128, 32, 70, [75, 71, 200], [5, 1, 33]),        # seven query heads a KV head
    (3, 1, 80, 5, 33, [34, 50], None),                     # head_dim between two kernels', pages that end inside a tile
    (1, 2, 8, 8, 20, [25, 90], [3, 8]),
    (2, 2, 256, 16, 130, [131, 190, 150], None),
    (1, 3, 136, 16, 64, [90, 65], [20, 1]),
    (1, 8, 256, 64, 70, [200, 300], [100, 90]),            # more rows than a wave has
    (1, 71, 128, 16, 40, [45, 60, 41], None),              # more query heads a KV head than a wave has rows
    (8, 4, 128, 16, 1500, [1501 + 30 * i for i in range(9)], None),
    (2, 4, 128, 16, 640, [641 + 7 * i for i in range(40)], None),  # 160 rows over the prefix
    (1, 4, 64, 33, 5000, [5001, 5400, 9000], [1, 2, 3]),
    (1, 1, 128, 16, 0, [700], [700]),                      # a prompt
    (2, 1, 40, 16, 0, [300, 1, 257], [300, 1, 257]),
    (1, 2, 128, 16, 128, [128, 127, 1, 0, 64, 129], None),  # rows that end inside the prefix, one that is empty
    (1, 2, 64, 16, 50, [3, 60, 0, 20], [5, 4, 2, 30]),     # more new tokens than there are: the first of them see nothing
    (1, 4, 128, 16, 96, [96, 50], None),                   # nothing beyond the prefix
    (1, 1, 128, 16, 0, [0, 0], None),                      # nothing at all
    (1, 2, 128, 16, 30, [64, 40, 90], [0, 3, 0]),          # requests without a new token
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", ATTEND, ids=[f"c{i}" for i in range(len(ATTEND))])
def test_attention(kvc_lib, case, dtype):
    hz.say(f"[case] attention {case} {dtype}")
    a = Attend(*case[:3], dtype, *case[3:], seed=len(case[5]))
    a.call()
    a.check()


@pytest.mark.parametrize("new", [None, [2, 40]])
def test_attention_without_the_sums(kvc_lib, new):
    a = Attend(1, 4, 128, "f16", 16, 300, [340, 420], new, layers=3)
    a.call(lse=False)
    torch.cuda.synchronize()
    first = a.out.clone()
    assert bool((a.lse == 7.0).all())
    a.call()
    a.check()
    assert torch.equal(first, a.out)


@pytest.mark.parametrize("new", [None, [3, 50, 9]])
def test_attention_within_looser_bounds(kvc_lib, new):
    a = Attend(2, 2, 128, "bf16", 16, 200, [230, 290, 215], new, most_tokens=300)
    a.call()
    a.check()


@pytest.mark.parametrize("spread", [30.0, 1e-3])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_of_extreme_scores(kvc_lib, dtype, spread):
    """One token gets all the weight, and scores of thousands do not overflow; or all get the same."""
    a = Attend(1, 4, 128, dtype, 16, 500, [520, 600], [3, 20], spread=spread, seed=5)
    a.call()
    a.check()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("G", [2, 40])
def test_what_a_query_does_not_see_does_not_reach_it(kvc_lib, value, kind, G):
    """New tokens whose key or value is no number: queries before them know nothing of it, and those that see it do."""
    a = Attend(1, G, 128, "bf16", 16, 60, [90, 75], [20, 9], seed=1)
    cache = a.caches[0]
    for request, at, dim in ((0, 84, 3), (1, 70, 100), (1, 73, 100)):
        page = a.books.tables[a.rows[request]][at // 16]
        cache[kind, page, at % 16, 0, dim] = value
    if kind == 0:
        a.q[..., 3], a.q[..., 100] = 1.0, 1.0  # the score has the key's sign
    a.call()
    torch.cuda.synchronize()
    clean = Attend(1, G, 128, "bf16", 16, 60, [90, 75], [20, 9], seed=1)
    if kind == 0:
        clean.q[..., 3], clean.q[..., 100] = 1.0, 1.0
    clean.call()
    clean.check()
    assert int(a.device.err.item()) == 0
    for t in range(29):
        position = 70 + t if t < 20 else 66 + t - 20
        sees = position >= (84 if t < 20 else 70)
        dims = slice(None) if kind == 0 else [3 if t < 20 else 100]
        if not sees:
            assert torch.equal(a.out[t], clean.out[t]) and torch.equal(a.lse[t], clean.lse[t])
        elif kind == 0 and value == -math.inf:
            assert bool(torch.isfinite(a.out[t]).all())
        else:
            assert not bool(torch.isfinite(a.out[t][:, dims]).any())
            if kind == 1:
                rest = [d for d in range(128) if d not in dims]
                assert torch.equal(a.out[t][:, rest], clean.out[t][:, rest])


@pytest.mark.parametrize("new", [None, [4, 90]])
def test_pages_outside_the_pool_are_not_seen(kvc_lib, new):
    a = Attend(2, 2, 64, "f16", 16, 100, [260, 210], new, seed=3)
    a.books.tables[0][2] = a.books.blocks           # positions 32 .. 47 of the prefix
    a.books.tables[a.rows[0]][9] = -1               # 144 .. 159 of a row
    a.books.tables[a.rows[1]][3] = 10 ** 6          # below the prefix: read through row 0
    a.device.tables.copy_(i32(a.books.tables))
    a.call()
    a.check(err=model.FAULT_PAGE, missing=[(None, p) for p in range(32, 48)] + [(a.rows[0], p) for p in range(144, 160)])


def test_books_that_contradict_the_call(kvc_lib):
    """Lengths beyond the bound are cut to it, a row outside the table is empty; both are told."""
    a = Attend(1, 2, 64, "f16", 16, 40, [70, 60, 50], None, seed=8, most_tokens=64)
    a.call()
    torch.cuda.synchronize()
    cut = a.out.clone()
    assert int(a.device.err.item()) == model.FAULT_LIST
    a.device.err.zero_()
    a.check(lens=[64, 60, 50])
    a.where[1] = 99
    a.call()
    torch.cuda.synchronize()
    assert int(a.device.err.item()) == model.FAULT_LIST
    assert bool((a.out[1] == 0).all()) and bool((a.lse[1] == -math.inf).all())
    assert torch.equal(a.out[0], cut[0]) and torch.equal(a.out[2], cut[2])
    b = Attend(1, 2, 64, "f16", 16, 40, [70, 60], None, seed=8)
    b.device.lens[0] = 30  # the prefix's row is shorter than the prefix: positions 30 .. 39 are not there
    b.call()
    b.check(err=model.FAULT_LIST, missing=[(None, p) for p in range(30, 40)])
    c = Attend(1, 1, 64, "f16", 16, 0, [70, 60, 50], [3, 9, 2], seed=8)
    c.starts[1] = 14  # beyond the end, and descending
    c.call()
    torch.cuda.synchronize()
    assert int(c.device.err.item()) == model.FAULT_LIST


def test_a_graph_follows_the_books(kvc_lib):
    """Lengths, tables and rows change between replays; every replay equals a call of its own."""
    a = Attend(2, 4, 128, "f16", 16, 700, [701 + 20 * i for i in range(6)], None, seed=4, most_tokens=1000)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        a.call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        a.call()
    for turn in range(3):
        lens = [n - 150 * turn - i for i, n in enumerate(a.lens)]
        a.device.lens.copy_(i32([700] + [dict(zip(a.rows, lens)).get(r, 0) for r in range(1, len(a.books.lens))]))
        a.out.zero_()
        a.space.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        a.check(lens=lens)
        replayed = a.out.clone()
        a.out.zero_()
        a.call()
        torch.cuda.synchronize()
        assert torch.equal(replayed, a.out)


def test_offsets_beyond_32_bits(kvc_lib):
    """A layer's cache of 9 GB, its pages in use at the end, K and V more than 4 GB apart."""
    first = (1 << 32) // (2 * 64 * 128 * 2) + 5  # pages of 32 KB
    a = Attend(2, 2, 128, "f16", 64, 200, [230, 300], [1, 20], seed=2, first_page=first)
    assert a.caches[0].numel() * 2 > 2 * (1 << 32)
    a.call()
    a.check()
    lens = a.lens
    x = torch.randn((21, 2, 2, 128), device="cuda").to(torch.float16)
    kvc.kvc_append_paged(a.device.pool, a.batch, 0, x[:, 0].data_ptr(), x[:, 1].data_ptr(), 512, hz.stream_handle())
    torch.cuda.synchronize()
    t = 0
    for r, n, c in zip(a.rows, lens, a.new):
        for at in range(n - c, n):
            assert torch.equal(a.caches[0][:, a.books.tables[r][at // 64], at % 64], x[t])
            t += 1
    a.call()
    a.check()
    src, dst = i32([a.books.tables[0][0]]), i32([0])
    kvc.kvc_pages_copy(a.device.pool, src.data_ptr(), dst.data_ptr(), 1, hz.stream_handle())
    torch.cuda.synchronize()
    assert torch.equal(a.caches[0][:, 0], a.caches[0][:, a.books.tables[0][0]])


# ---- many new tokens over a short prefix: each row's tokens are one sequence, and no pieces are joined

ONE_SEQUENCE = [
    (8, 8, 128, 16, 100, [320, 260, 140, 290], [200, 150, 0, 170]),
    (4, 16, 64, 5, 33, [300, 280, 33, 40], [260, 240, 3, 20]),
    (8, 8, 128, 16, 128, [60, 300, 290, 0], [60, 250, 210, 5]),  # rows that end inside the prefix
    (8, 8, 256, 32, 70, [300, 330], [250, 270]),
    (8, 8, 72, 1, 64, [200, 450], [130, 390]),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", ONE_SEQUENCE, ids=[f"c{i}" for i in range(len(ONE_SEQUENCE))])
def test_attention_of_one_sequence(kvc_lib, case, dtype):
    hz.say(f"[case] one sequence {case} {dtype}")
    a = Attend(*case[:3], dtype, *case[3:], seed=len(case[5]))
    assert a.space.numel() == 0
    a.call()
    a.check()


def test_faults_of_one_sequence(kvc_lib):
    """Pages outside the pool are not seen, below the prefix those of the prefix's row; nor is what that row lacks."""
    a = Attend(8, 8, 64, "f16", 16, 100, [320, 290], [270, 250], seed=3)
    assert a.space.numel() == 0
    a.books.tables[0][2] = a.books.blocks           # positions 32 .. 47 of the prefix
    a.books.tables[a.rows[0]][9] = -1               # 144 .. 159 of a row
    a.books.tables[a.rows[1]][3] = 10 ** 6          # below the prefix: read through row 0
    a.device.tables.copy_(i32(a.books.tables))
    a.call()
    a.check(err=model.FAULT_PAGE, missing=[(None, p) for p in range(32, 48)] + [(a.rows[0], p) for p in range(144, 160)])
    b = Attend(8, 8, 128, "bf16", 16, 100, [320, 290], [270, 250], seed=4)
    b.device.lens[0] = 71
    b.call()
    b.check(err=model.FAULT_LIST, missing=[(None, p) for p in range(71, 100)])


def test_wild_values_of_one_sequence(kvc_lib):
    """What a query does not see does not reach it, be it infinite."""
    a, clean = (Attend(8, 8, 128, "f16", 16, 90, [300, 310], [260, 270], seed=6) for _ in range(2))
    page = a.books.tables[a.rows[0]][280 // 16]
    a.caches[0][1, page, 280 % 16, :, 5] = math.inf
    a.call()
    clean.call()
    clean.check()
    torch.cuda.synchronize()
    first = 280 - 40  # the token at position 280 is the request's 241st
    assert torch.equal(a.out[:first], clean.out[:first]) and torch.equal(a.out[260:], clean.out[260:])
    assert bool((a.out[first:260, :, 5] == math.inf).all())
    rest = [d for d in range(128) if d != 5]
    assert torch.equal(a.out[first:260][:, :, rest], clean.out[first:260][:, :, rest])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", [
    (32, 1, 128, 16, 70, [71 + (5 * i) % 60 for i in range(20)], None),           # a wave each has a head of a request
    (32, 3, 64, 5, 33, [40 + (7 * i) % 90 for i in range(17)], [1 + i % 4 for i in range(17)]),
    (16, 8, 256, 32, 100, [101 + (i * 31) % 128 if i % 5 else 90 + i % 3 for i in range(33)], None),  # some end inside the prefix
    (40, 1, 72, 1, 0, [(3 * i) % 129 for i in range(15)], [min((3 * i) % 129, i % 6) for i in range(15)]),
    (32, 1, 128, 16, 64, [64, 64, 65, 192, 0, 1] + [70] * 11, None),
], ids=[f"c{i}" for i in range(5)])
def test_many_rows_of_few_tokens(kvc_lib, case, dtype):
    hz.say(f"[case] few tokens {case} {dtype}")
    a = Attend(*case[:3], dtype, *case[3:], seed=len(case[5]))
    a.call()
    a.check()
    a.books.tables[a.rows[3]][case[4] // case[3]] = -1  # the page of the first own token, and of what the prefix has in it
    a.device.tables.copy_(i32(a.books.tables))
    a.call()
    block = case[3]
    first = case[4] // block * block
    lost = [(a.rows[3], p) for p in range(max(first, case[4]), first + block)]
    seen = a.lens[3] > case[4] and a.new[3] > 0
    a.check(err=model.FAULT_PAGE if seen else 0, missing=lost)
