"""Serving calls where books, lists and pages are not what a call may rely on, and attention at the ends of its types and addresses."""
import math
import random

import pytest
import torch

import kvc_harness as hz
import paper_2602_09725_amd as kvc
import serving_model as model
from test_gpu_serving import Attend, DevicePool, filled, i32, starts_of

pytestmark = pytest.mark.gpu


# ---- a page outside the pool behind tokens that are all seen


def facing_away(a, nats, seed=11):
    """Every key points away from every query: scores lie around -nats, below those of a key of zeros."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    u = torch.full((a.D,), a.D ** -0.5, device="cuda")
    a.q.copy_((u + 0.01 * torch.randn(a.q.shape, generator=g, device="cuda")).to(a.dtype))
    keys = a.caches[a.layer][0]
    keys.copy_((0.3 * keys.float() - nats * u).to(a.dtype))  # (NaN stays where no token is)


BEHIND = [  # case, pages of the prefix and of each row that lie outside the pool: first half of a piece's third or fifth tile of 64 tokens
    ((8, 16, 64, 16, 5200, [5210 + i for i in range(16)], None), [8, 88], []),          # a prefix in pieces of 384 tokens
    ((8, 8, 64, 16, 100, [700, 650], [270, 250]), [], [[8], [16]]),                     # one sequence a row
    ((8, 8, 128, 16, 200, [700, 650], [270, 250]), [8], []),                            # the same, below the prefix
    ((2, 4, 128, 16, 0, [6000], [300]), [], [[8, 176]]),                                # a row's own tokens in pieces of 512
    ((2, 8, 256, 16, 0, [6000], [150]), [], [[8, 176]]),
]


@pytest.mark.parametrize("dtype,nats", [("f16", 25.0), ("f16", 120.0), ("bf16", 120.0)])
@pytest.mark.parametrize("case", BEHIND, ids=[f"c{i}" for i in range(len(BEHIND))])
def test_a_page_outside_the_pool_takes_nothing_from_those_before(kvc_lib, case, dtype, nats):
    hz.say(f"[case] behind {case} {dtype} {nats}")
    shape, front, rows = case
    a = Attend(*shape[:3], dtype, *shape[3:], seed=5, scale=1.0)
    facing_away(a, nats)
    for page in front:
        a.books.tables[0][page] = a.books.blocks
    for r, pages in zip(a.rows, rows):
        for page in pages:
            a.books.tables[r][page] = -1
    a.device.tables.copy_(i32(a.books.tables))
    a.call()
    a.check(err=model.FAULT_PAGE)


# ---- new tokens that no request covers


def rows_near(a, request, tokens, seen):
    """The results of these tokens of a request are those of the first seen[i] positions of its row."""
    r, n = a.rows[request], max(seen)
    got, got_lse = a.out[tokens].double().cpu(), a.lse[tokens].double().cpu()
    positions = torch.arange(n)
    own, front = torch.tensor(a.books.tables[r])[positions // a.block], torch.tensor(a.books.tables[0])[positions // a.block]
    slots = torch.where(positions < a.prefix, front, own) * a.block + positions % a.block
    flat = a.caches[a.layer].flatten(1, 2)[:, slots.cuda()].cpu()
    visible = positions[None] < torch.tensor(seen)[:, None]
    for h in range(a.H):
        heads = slice(h * a.G, h * a.G + a.G)
        want = model.attention(a.q[tokens, heads].cpu(), flat[0, :, h], flat[1, :, h], visible, a.scale)
        far, far_lse = model.attention_bounds(*want, n, a.D, a.dtype)
        a.near(f"out of request {request}, head {h}", got[:, heads], want[0], far)
        a.near(f"lse of request {request}, head {h}", got_lse[:, heads], want[1], far_lse)


UNCOVERED = {
    "pieces": (2, 4, 128, 16, 700, [760, 720, 900], [6, 5, 9]),
    "one wave": (2, 2, 64, 16, 0, [40, 60, 100], [6, 5, 9]),
    "four waves": (2, 16, 128, 16, 0, [40, 60, 100], [6, 5, 9]),
    "a wave each": (32, 1, 128, 16, 0, [40 + i for i in range(20)], [6, 5] + [4] * 17 + [9]),
    "prefix alone": (2, 4, 128, 16, 90, [90, 80, 85], [6, 5, 9]),
    "one sequence": (8, 8, 64, 16, 100, [320, 290, 300], [270, 250, 280]),
}


@pytest.mark.parametrize("wrong", ["tail", "head", "many", "descending"])
@pytest.mark.parametrize("form", UNCOVERED)
def test_tokens_that_no_request_covers_have_no_result(kvc_lib, form, wrong):
    """They get 0 and -inf, whatever the workspace and the results held before, and the list is told to be at fault."""
    hz.say(f"[case] uncovered {form} {wrong}")
    case = UNCOVERED[form]
    a = Attend(*case[:3], "f16", *case[3:], seed=7)
    starts, most = starts_of(a.new), max(a.new)
    if wrong == "tail":
        starts[-1] -= 3
    elif wrong == "head":
        starts[0] = 2
    elif wrong == "many":
        most -= 2
    else:
        starts[1], starts[2] = starts[2], starts[1]
    a.starts.copy_(i32(starts))
    a.batch = kvc.Batch(len(a.new), sum(a.new), most, a.where.data_ptr(), a.starts.data_ptr())
    a.space = torch.empty(kvc.attention_workspace(a.device.pool, a.batch, a.attention), dtype=torch.uint8, device="cuda")
    a.space.view(torch.float32).fill_(1.5)
    a.call()
    torch.cuda.synchronize()
    assert int(a.device.err.item()) == model.FAULT_LIST
    assert bool((a.out_store[:, :, a.D:] == 7.0).all()) and bool((a.lse[-1] == 7.0).all())
    if wrong == "descending":  # the requests overlap: their tokens' results are open, but they are results
        assert not bool((a.out == 7.0).any()) and not bool((a.lse[:-1] == 7.0).any())
        return
    covered = torch.zeros(sum(a.new), dtype=torch.bool)
    for request, (first, end) in enumerate(zip(starts, starts[1:])):
        n = end - first
        tokens = list(range(first, first + min(n, most)))
        covered[tokens] = True
        length = a.books.lens[a.rows[request]]
        if request in (0, 1, len(a.new) - 1):
            rows_near(a, request, tokens, [length - n + i + 1 for i in range(len(tokens))])
    assert int((~covered).sum()) >= 2
    assert bool((a.out[~covered.cuda()] == 0).all()) and bool((a.lse[:-1][~covered.cuda()] == -math.inf).all())


def test_books_at_fault_are_told_where_nothing_may_be_seen(kvc_lib):
    """No position lies below a bound of 0 tokens: all rows are empty, and those that are not are told."""
    for lens, err in (([0, 0, 0], 0), ([0, 9, 0], model.FAULT_LIST)):
        a = Attend(2, 2, 64, "f16", 16, 0, lens, None, seed=2)
        a.most = 0
        a.attention = kvc.Attention(4, a.scale, 0, 0, 0, a.q.stride()[:2], a.out.stride()[:2])
        a.call()
        torch.cuda.synchronize()
        assert int(a.device.err.item()) == err
        assert bool((a.out == 0).all()) and bool((a.lse[:-1] == -math.inf).all())


@pytest.mark.parametrize("H,D", [(1, 8), (40, 128)])  # (a vector a thread, and four)
@pytest.mark.parametrize("wrong", ["head", "tail", "many"])
def test_append_leaves_out_what_no_request_covers(kvc_lib, wrong, H, D):
    books = filled(3, 80, 4, 200, [280, 290, 9], seed=6)
    d = DevicePool(books, 1, H, D, refs=False)
    before = d.copy()
    new, most = [250, 200, 4], 250
    starts = starts_of(new)
    if wrong == "head":
        starts[0] = 5
    elif wrong == "tail":
        starts[-1] -= 2
    else:
        most = 230
    n, where = sum(new), i32(starts)
    x = torch.randint(-32768, 32768, (n, H * D), device="cuda", dtype=torch.int16)
    kvc.kvc_append_paged(d.pool, kvc.Batch(3, n, most, None, where.data_ptr()), 0, x.data_ptr(), x.data_ptr(), H * D, hz.stream_handle())
    want = before[0].clone()
    for r, (first, end) in enumerate(zip(starts, starts[1:])):
        for t in range(first, min(end, first + most)):
            at = books.lens[r] - end + t
            want[:, books.tables[r][at // 4], at % 4] = x[t]
    books.err = model.FAULT_LIST
    d.check()
    assert torch.equal(d.caches[0], want)


# ---- tables that hold free pages


class Books(model.Books):
    """A fork whose parent holds a free page: of a last page filled in part the list is at fault, a whole one is copied as it is and shared
    with nobody."""

    def fork(self, parents, children):
        free = set(self.free_list())
        lost = [self.tables[p][j] for p in parents for j in range(self.lens[p] // self.block) if self.tables[p][j] in free]
        if any(self.lens[p] % self.block and self.tables[p][self.lens[p] // self.block] in free for p in parents):
            self.err |= model.FAULT_LIST
            return
        taken = self.free_list()[:sum(self.lens[p] % self.block != 0 for p in parents)]
        was = list(self.refs)
        super().fork(parents, children)
        for page in lost:
            self.refs[page] = 1 if page in taken else was[page]
            self.err |= model.FAULT_LIST


def books_of(blocks, lens, seed):
    books = filled(8, 6, 4, blocks, lens, seed=seed)
    books.__class__ = Books
    return books


@pytest.mark.parametrize("blocks", [40, 20000])
@pytest.mark.parametrize("count", [0, -2])
def test_a_grow_into_a_free_page_changes_nothing(kvc_lib, blocks, count):
    """A last page that is filled in part and held by nobody could be another row's by now."""
    books = books_of(blocks, [9, 8, 6, 0], blocks)
    books.refs[books.tables[2][1]] = count
    books.refs[books.tables[1][1]] = 0  # filled to its end: nobody writes to it
    d = DevicePool(books, 1, 1, 8)
    before = d.copy()
    for more in ([3, 1, 5], [3, 2, 0]):
        rows, counts = i32([0, 2, 3]), i32(more)
        kvc.kvc_pages_grow(d.pool, rows.data_ptr(), counts.data_ptr(), 3, *d.room())
        books.err = model.FAULT_LIST
        d.check(before)
    if count == 0:
        d.err.zero_()
        books.err = 0
        rows, counts = i32([2, 0]), i32([0, 5])  # a row that gets no token is not written to
        kvc.kvc_pages_grow(d.pool, rows.data_ptr(), counts.data_ptr(), 2, *d.room())
        books.grow([2, 0], [0, 5])
        assert books.err == 0
        d.check(before)


@pytest.mark.parametrize("blocks", [40, 20000])
@pytest.mark.parametrize("count", [0, -2])
@pytest.mark.parametrize("what", ["part", "whole"])
def test_a_fork_of_a_free_page(kvc_lib, blocks, count, what):
    books = books_of(blocks, [9, 12, 6, 0, 0, 0, 0], blocks + 1)
    if what == "part":
        books.refs[books.tables[2][1]] = count
    else:  # the lowest free page, which the call takes for a child too
        books.refs[books.tables[0][0]] = books.refs[books.tables[1][1]] = 0
        books.tables[1][1] = books.free_list()[0]
        books.refs[books.tables[1][1]] = count
    d = DevicePool(books, 2, 1, 16)
    before = d.copy()
    parents, children = [1, 0, 1, 2], [3, 4, 6, 5]
    a, b = i32(parents), i32(children)
    kvc.kvc_pages_fork(d.pool, a.data_ptr(), b.data_ptr(), 4, *d.room())
    books.fork(parents, children)
    assert books.err == model.FAULT_LIST and (books.lens[3] == 12) == (what == "whole")
    d.check(before)


# ---- weights far below a row's largest


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("G,new,tokens", [(1, 1, 300), (3, 20, 300), (2, 1, 20), (40, 1, 3000)])
def test_small_weights_count(kvc_lib, dtype, G, new, tokens):
    """One token outweighs each of the others 2^26 times and has the value 0: what is left is theirs.  Weights are held with a relative
    error of half a step of the type down to 2^-21 of the largest, and to 2^-32 of it below that."""
    a = Attend(2, G, 64, dtype, 16, 0, [tokens], [new], seed=3, scale=math.log(2.0))
    keys, values = a.caches[0][0].flatten(0, 1), a.caches[0][1].flatten(0, 1)
    positions = torch.arange(tokens)
    slots = (torch.tensor(a.books.tables[a.rows[0]])[positions // 16] * 16 + positions % 16).cuda()
    a.q.zero_()
    a.q[..., 0] = 1.0
    keys[slots] = 0
    keys[slots[1:], :, 0] = -26.0
    values[slots[:1]] = 0
    values[slots[1:]] = (512.0 + torch.arange(64, device="cuda")).to(a.dtype)
    a.call()
    torch.cuda.synchronize()
    assert int(a.device.err.item()) == 0
    seen = torch.arange(tokens - new + 1, tokens + 1, dtype=torch.float64)[:, None, None]  # tokens that each query sees
    others = (seen - 1) * 2.0 ** -26
    value = values[slots[-1]].double().cpu()[0]
    want = (others / (1 + others) * value).expand(new, 2 * G, 64)
    u, e = torch.finfo(a.dtype).eps / 2, 2.0 ** -24
    size, smallest = 26.0 * math.log(2.0), 2.0 ** -25 if dtype == "f16" else 2.0 ** -134
    held = (seen - 1) * 2.0 ** -32 * value if dtype == "f16" else 0.0
    far = (2 * u + 2 * u * u + 2 * e * (68 * size + 4) + (tokens + 16) * e) * want + held + smallest
    assert bool(((a.out.double().cpu() - want).abs() <= far).all())
    want_lse = torch.log1p(others)[..., 0].expand(new, 2 * G)
    assert bool(((a.lse[:-1].double().cpu() - want_lse).abs() <= e * (68 * size + 4) + (tokens + 20) * e).all())


# ---- caches whose K and V pass 32 bits of offsets


@pytest.fixture(scope="module")
def large():
    """Memory of a layer whose K and V have 4.6 GB each."""
    yield torch.full((2 * 4600 << 20,), 0x7E, dtype=torch.uint8, device="cuda")  # (NaN in both types)


LARGE = [  # H, G, block, prefix, lens, new
    (2, 4, 16, 900, [901 + 30 * i for i in range(3)], None),              # one wave along the rows, for both parts
    (4, 4, 16, 0, [700, 90, 1500], None),
    (32, 1, 16, 70, [71 + (5 * i) % 60 for i in range(20)], None),        # a wave each for a head of a request
    (32, 3, 8, 33, [40 + (7 * i) % 90 for i in range(17)], [1 + i % 4 for i in range(17)]),
    (2, 4, 32, 640, [641 + 7 * i for i in range(40)], None),              # four waves over the prefix
    (2, 4, 16, 300, [600, 450], [40, 90]),                                # and over the rows' own tokens
    (8, 8, 16, 100, [320, 260, 140, 290], [200, 150, 0, 170]),            # one sequence a row
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256, 40])
@pytest.mark.parametrize("case", LARGE, ids=[f"c{i}" for i in range(len(LARGE))])
def test_every_body_beyond_32_bits(kvc_lib, large, case, D, dtype):
    """Pages all over 4.6 GB of K and of V, so that neighbours lie on both sides of 2 and 4 GiB: results are those of the same pages side by side."""
    hz.say(f"[case] large {case} {D} {dtype}")
    H, G, block, prefix, lens, new = case
    a = Attend(H, G, D, dtype, block, prefix, lens, new, seed=9)
    a.call()
    torch.cuda.synchronize()
    near, near_lse = a.out.clone(), a.lse.clone()
    page_bytes = block * H * D * 2
    blocks = large.numel() // 2 // page_bytes
    assert blocks * page_bytes > 1 << 32
    rng = random.Random(D)
    to = [0, blocks - 1] + [edge // page_bytes + i for edge in (1 << 31, 1 << 32) for i in (-1, 0, 1)]
    to += rng.sample([page for page in range(1, blocks - 1, 7) if page not in to], a.books.blocks - len(to))
    rng.shuffle(to)
    cache = large[:2 * blocks * page_bytes].view(a.dtype).unflatten(0, (2, blocks, block, H, D))
    cache[:, torch.tensor(to, device="cuda")] = a.caches[0]
    a.device.tables.copy_(i32([[to[page] if page >= 0 else -1 for page in t] for t in a.books.tables]))
    a.device.ptrs.fill_(large.data_ptr())
    a.device.pool.num_blocks = blocks
    a.out_store.fill_(7.0)
    a.lse.fill_(7.0)
    a.call()
    torch.cuda.synchronize()
    assert int(a.device.err.item()) == 0
    assert torch.equal(a.out, near) and torch.equal(a.lse, near_lse)
