"""Pools in 4 bits where it is easy to go wrong: heads of one value, rows that end inside the prefix, tokens that no request covers, graphs, streams, long
and large pools."""
import math

import pytest
import torch

import held_model as held
import kvc_harness as hz
import paper_2602_09725_amd as kvc
import serving_model as model
from test_gpu_held import Attend, HeldPool, i32, tokens_like, words_of

pytestmark = pytest.mark.gpu
TORCH = held.TORCH
BODIES = [([1, 1, 1], 4), ([1, 30, 7], 4), ([200, 40, 190], 8)]  # a wave's, a few blocks of rows, rows by the hundred


def put_pairs(a, kind, change):
    """change(scale, mn, page, slot, head) -> the pair a token is held with; kind 0: keys, 1: values."""
    d = a.d
    words = d.cache.cpu()
    code, s, m = d.form.get(words[1, kind], TORCH[a.dtype])
    bits = lambda v: torch.tensor(v, dtype=torch.float64).to(TORCH[a.dtype]).view(torch.int16).item() & 0xffff  # noqa: E731
    for page in range(d.blocks):
        for slot in range(d.block):
            for h in range(a.H):
                new = change(float(s[page, slot, h]), float(m[page, slot, h]), page, slot, h)
                if new is not None:
                    w = bits(new[0]) | bits(new[1]) << 16
                    words[1, kind, page, d.form.pair(h, slot)] = w - (w >= 2 ** 31) * 2 ** 32
    d.cache.copy_(words)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("body", range(len(BODIES)))
@pytest.mark.parametrize("D", [40, 64, 128, 256])
def test_heads_of_one_value(kvc_lib, dtype, body, D):
    """Scale 0, whatever the codes: values of 0, of one number, of a small one; and all heads so."""
    new, G = BODIES[body]
    new = new if D < 256 else [n // 4 + 1 for n in new]
    a = Attend(new, [n + 60 for n in new], 70, 1, G, D, 8, dtype, seed=body)

    def some(s, m, page, slot, h):
        return (0.0, [0.0, m, 0.01 * m, -3.0][(page * 3 + slot) % 4]) if (page * 5 + slot) % 3 == 0 else None

    put_pairs(a, 0, some)
    put_pairs(a, 1, some)
    same_prefix(a)
    a.check()
    put_pairs(a, 1, lambda s, m, page, slot, h: (0.0, 0.0))
    got, _ = a.check()
    # Codes are taken less 8, and 8 times the weights' sum is added.  A head of zeros counts as scale 2^-60 and codes of 0, so that what is left is 2^-60 of the
    # rounding of two sums of 8 w over n tokens: each within n 2^-23 of itself, the weights' own sum being 1.
    n = 70 + max(new) + 60
    assert got.double().abs().max() <= 2.0 ** -60 * 16 * n * 2.0 ** -23


def same_prefix(a):
    """What a fork copies: the prompt's last page, filled in part, is each row's own."""
    d, part = a.d, a.prefix % a.d.block
    words = d.cache.cpu()
    first = d.host_tables[0]
    for t in d.host_tables[1:]:
        for slot in range(part):
            at = [d.form.word(h, slot, w) for h in range(a.H) for w in range(a.D // 8)] + [d.form.pair(h, slot) for h in range(a.H)]
            words[:, :, t[a.prefix // d.block], at] = words[:, :, first[a.prefix // d.block], :][:, :, at]
    d.cache.copy_(words)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows_far_from_zero(kvc_lib, dtype):
    """Values and keys whose least value is thousands of steps away, as a head of few nearby numbers has."""
    a = Attend([1, 20, 3], [90, 40, 300], 90, 2, 4, 128, 16, dtype, seed=3)
    far = 800.0 if dtype == "bf16" else 3000.0
    put_pairs(a, 1, lambda s, m, page, slot, h: (s, far * s) if (page + slot) % 4 == 0 else None)
    put_pairs(a, 0, lambda s, m, page, slot, h: (s / 256, m) if (page + slot) % 4 == 1 else None)
    same_prefix(a)
    a.check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("G", [1, 4, 40])
def test_rows_that_end_inside_the_prefix(kvc_lib, dtype, G):
    """Of rows shorter than the prefix only what is there is seen; some end on a quad, some inside."""
    a = Attend([1, 3, 5, 2], [4, 4, 9, 4], 301, 1, G, 64, 8, dtype, seed=G)
    for row, n in ((1, 100), (2, 7), (3, 300), (4, 302)):
        a.d.host_lens[row] = n
    a.d.lens.copy_(i32(a.d.host_lens))
    a.check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_prefix_row_that_is_too_short(kvc_lib, dtype):
    a = Attend([1, 1], [40, 9], 200, 1, 4, 64, 8, dtype, seed=2)
    a.d.host_lens[0] = 120
    a.d.lens.copy_(i32(a.d.host_lens))
    a.check(fault=model.FAULT_LIST, hidden=lambda row, pos: 120 <= pos < 200)


@pytest.mark.parametrize("new,G", [([1, 2, 3], 4), ([40, 30, 60], 4)])
@pytest.mark.parametrize("prefix", [0, 100])
def test_tokens_that_no_request_covers(kvc_lib, new, G, prefix):
    a = Attend(new, [n + 20 for n in new], prefix, 2, G, 64, 8, "f16", seed=4)
    whole, _ = a.check()
    n = a.n
    starts = list(a.starts)
    for wrong in ("front", "back"):
        a.begin.copy_(i32([1] + starts[1:] if wrong == "front" else starts[:-1] + [n - 1]))
        a.d.err.zero_()
        got, norm = a.run()
        assert a.d.fault() == model.FAULT_LIST
        t = 0 if wrong == "front" else n - 1
        assert (got[t] == 0).all() and (norm[t] == -math.inf).all(), wrong
        keep = range(starts[1], n) if wrong == "front" else range(0, starts[-2])  # (the other request sees other positions now)
        assert torch.equal(got[list(keep)], whole[list(keep)])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_lengths_of_zero_and_bounds_of_zero(kvc_lib, dtype):
    a = Attend([1, 1], [5, 9], 0, 1, 4, 64, 8, dtype, most_tokens=0)
    got, norm = a.run()
    assert a.d.fault() == model.FAULT_LIST and (got == 0).all() and (norm == -math.inf).all()


@pytest.mark.parametrize("case", [([1] * 6, [900, 30, 1, 400, 64, 65], 700, 2, 4, 128), ([60, 1, 30], [300, 90, 30], 0, 1, 8, 128),
                                  ([100, 90], [100, 400], 300, 1, 8, 64)])
def test_a_graph_follows_the_books(kvc_lib, case):
    """A step (append, attend, read) captured once, replayed while lengths change: every replay equals calls of its own."""
    new, owned, prefix, H, G, D = case
    a = Attend(new, owned, prefix, H, G, D, 16, "f16", seed=6)
    d, n = a.d, a.n
    g = torch.Generator("cuda").manual_seed(1)
    k, v = (torch.randn((n, H, D), generator=g, device="cuda").half() for _ in range(2))
    q = a.q.cuda()
    out, norm = torch.zeros_like(q), torch.zeros((n, H * G), device="cuda")
    back = torch.zeros((2, n, H, D), dtype=torch.float16, device="cuda")
    call = kvc.Attention(H * G, a.scale, a.most_tokens, prefix, 0, q.stride()[:2], out.stride()[:2])
    size = kvc.attention_workspace(d.pool, a.batch, call)
    space = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step():
        at = hz.stream_handle()
        kvc.kvc_append_paged(d.pool, a.batch, 1, k.data_ptr(), v.data_ptr(), H * D, at)
        kvc.kvc_attend_paged(d.pool, a.batch, call, 1, q.data_ptr(), out.data_ptr(), norm.data_ptr(), space.data_ptr(), size, at)
        kvc.kvc_read_paged(d.pool, a.batch, None, 1, back[0].data_ptr(), back[1].data_ptr(), H * D, at)

    before = d.cache.clone()
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for turn in range(3):
        lens = [prefix] + [prefix + max(x, o - 11 * turn) for x, o in zip(new, owned)]
        d.lens.copy_(i32(lens))
        d.host_lens = lens
        results = []
        for replay in (True, False):
            d.cache.copy_(before)
            out.zero_(), norm.zero_(), back.zero_(), space.fill_(0xFF)
            torch.cuda.synchronize()
            if replay:
                graph.replay()
            else:
                step()
            torch.cuda.synchronize()
            results.append([x.clone() for x in (out, norm, back, d.cache)])
        for x, y in zip(*results):
            assert torch.equal(x, y)
        want, want_lse, far, far_lse = a.model()
        assert bool(((out.double().cpu() - want).abs() <= far).all()) and bool(((norm.double().cpu() - want_lse).abs() <= far_lse).all())
        assert torch.equal(back[0].cpu(), held.rounded(held.stands_for(*held.quantized(k.cpu())), torch.float16))
    assert d.fault() == 0


def test_calls_on_two_streams(kvc_lib):
    """Each with its own workspace, over one pool: the same results as after one another."""
    a = Attend([1, 1, 3], [500, 70, 40], 900, 2, 4, 128, 16, "bf16", seed=8)
    b = Attend([70, 1, 30], [500, 70, 40], 200, 2, 4, 128, 16, "f16", seed=9)
    alone = [x.run() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    jobs = []
    for x, s in zip((a, b), streams):
        H = x.H * x.G
        q = x.q.cuda()
        out, norm = torch.zeros_like(q), torch.zeros((x.n, H), device="cuda")
        call = kvc.Attention(H, x.scale, x.most_tokens, x.prefix, 0, q.stride()[:2], out.stride()[:2])
        size = kvc.attention_workspace(x.d.pool, x.batch, call)
        jobs.append((x, s, q, out, norm, call, torch.empty(size, dtype=torch.uint8, device="cuda"), size))
    torch.cuda.synchronize()
    for _ in range(5):
        for x, s, q, out, norm, call, space, size in jobs:
            kvc.kvc_attend_paged(x.d.pool, x.batch, call, 1, q.data_ptr(), out.data_ptr(), norm.data_ptr(), space.data_ptr(), size, s.cuda_stream)
    torch.cuda.synchronize()
    for (x, _, _, out, norm, *_), (want, want_lse) in zip(jobs, alone):
        assert torch.equal(out.cpu(), want) and torch.equal(norm.cpu(), want_lse)


def test_results_do_not_change_from_call_to_call(kvc_lib):
    a = Attend([1] * 9, [900 + 90 * i for i in range(9)], 3000, 2, 4, 128, 16, "bf16", seed=10)
    first = a.run()
    for _ in range(3):
        again = a.run()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("D,H,G,new", [(128, 2, 4, [1, 5]), (64, 1, 40, [1, 9]), (256, 1, 2, [1, 40]), (128, 1, 8, [60, 40])])
def test_layers_beyond_4_gib(kvc_lib, D, H, G, new):
    """Keys and values more than 4 GiB apart, the pages in use on both sides of 2 and 4 GiB."""
    block, dtype = 64, "bf16"
    form = held.Words(H, D, block)
    page = 4 * form.count
    blocks = (1 << 32) // page + 40
    cache = torch.empty((1, 2, blocks, form.count), dtype=torch.int32, device="cuda")
    places = [0, blocks - 1, (1 << 31) // page, (1 << 31) // page + 1, (1 << 32) // page, (1 << 32) // page - 1, 7, blocks - 2, (1 << 32) // page + 3, 11]
    words = words_of(form, 1, len(places), dtype, 3).cuda()
    cache[:, :, places] = words
    prefix, owned = 130, [max(60, new[0]), max(200, new[1])]
    tables = [places[:3], places[:2] + places[3:6], places[:2] + places[6:10]]
    part = prefix % block
    for t in tables[1:]:
        for slot in range(part):
            at = [form.word(h, slot, w) for h in range(H) for w in range(D // 8)] + [form.pair(h, slot) for h in range(H)]
            cache[0][:, t[2], at] = cache[0][:, places[2]][:, at]
    a = Attend.__new__(Attend)
    d = a.d = HeldPool.__new__(HeldPool)
    d.form, d.H, d.D, d.block, d.blocks, d.dtype, d.L, d.cache = form, H, D, block, blocks, dtype, 2, cache
    d.ptrs = torch.tensor([cache[0].data_ptr()] * 2, dtype=torch.int64, device="cuda")
    length = max(len(t) for t in tables)
    d.host_tables, d.host_lens = [t + [-1] * (length - len(t)) for t in tables], [prefix] + [prefix + o for o in owned]
    d.tables, d.lens, d.err = i32(d.host_tables), i32(d.host_lens), torch.zeros(1, dtype=torch.int32, device="cuda")
    d.pool = kvc.Pool(2, H, D, kvc.KVC_BF16 | kvc.KVC_HELD_Q4, blocks, block, 3, length, d.ptrs.data_ptr(), d.tables.data_ptr(), d.lens.data_ptr(), None,
                      d.err.data_ptr())
    a.H, a.G, a.D, a.dtype, a.prefix, a.new, a.rows, a.scale, a.most_tokens = H, G, D, dtype, prefix, new, [1, 2], 1 / math.sqrt(D), prefix + max(owned)
    a.starts, a.n = [0, new[0], sum(new)], sum(new)
    a.q = torch.randn((a.n, H * G, D), generator=torch.Generator().manual_seed(2)).to(TORCH[dtype])
    a.at, a.begin = i32(a.rows), i32(a.starts)
    a.batch = kvc.Batch(2, a.n, max(new), a.at.data_ptr(), a.begin.data_ptr())

    def check():
        got, norm = a.run()
        used = sorted({p for t in tables for p in t})
        small = a.d
        a.d = HeldPool.__new__(HeldPool)  # the same pages, one after the other, for the model
        a.d.form, a.d.block, a.d.blocks = form, block, len(used)
        a.d.cache = cache[0][:, used][None].expand(2, 2, len(used), form.count)
        a.d.host_tables = [[used.index(p) if p >= 0 else -1 for p in t] for t in small.host_tables]
        a.d.host_lens = small.host_lens
        want, want_lse, far, far_lse = a.model()
        a.d = small
        assert d.fault() == 0
        assert bool(((got.double() - want).abs() <= far).all()) and bool(((norm.double() - want_lse).abs() <= far_lse).all())

    check()
    k, v = tokens_like(a.n, H, D, dtype, 5), tokens_like(a.n, H, D, dtype, 6)
    kd, vd = k.cuda(), v.cuda()
    kvc.kvc_append_paged(d.pool, a.batch, 1, kd.data_ptr(), vd.data_ptr(), H * D, hz.stream_handle())
    out = torch.empty((2, a.n, H, D), dtype=TORCH[dtype], device="cuda")
    kvc.kvc_read_paged(d.pool, a.batch, None, 1, out[0].data_ptr(), out[1].data_ptr(), H * D, hz.stream_handle())
    assert d.fault() == 0
    for got, x in zip(out.cpu(), (k, v)):
        assert torch.equal(got, held.rounded(held.stands_for(*held.quantized(x)), TORCH[dtype]))
    source, place = i32([places[1], places[8]]), i32([3, 4])
    kvc.kvc_pages_copy(d.pool, source.data_ptr(), place.data_ptr(), 2, hz.stream_handle())
    torch.cuda.synchronize()
    assert torch.equal(cache[0][:, [3, 4]], cache[0][:, [places[1], places[8]]])


def check_all_sizes(a):
    """Against the model, where values are of all sizes: rows that see a bf16 head with a scale above 2^40, or of one number above it, are NaN; a result may be
    beyond the type, the largest number or infinity then (x_hat of 65504 and its like reaches 65536), if the bound reaches it."""
    got, norm = a.run()
    assert a.d.fault() == 0
    out, lse, off, lse_off = a.model()
    code, s, m = a.d.form.get(a.d.cache[1, 1].cpu(), TORCH[a.dtype])
    wild = (s > 2.0 ** 40) | ((s * 2 ** 15 <= m.abs()) & (m.abs() > 2.0 ** 40))
    bad = torch.zeros(norm.shape, dtype=torch.bool)
    for r, row in enumerate(a.rows):
        table, total, n = a.d.host_tables[row], a.d.host_lens[row], a.starts[r + 1] - a.starts[r]
        for i in range(n):
            last = total - n + i
            for h in range(a.H):
                bad[a.starts[r] + i, h * a.G:(h + 1) * a.G] = any(bool(wild[table[t // a.d.block], t % a.d.block, h]) for t in range(last + 1))
    assert torch.isnan(got[bad]).all() and torch.isnan(norm[bad]).all()
    most = torch.finfo(TORCH[a.dtype]).max
    far, ok = off[~bad], got[~bad].double()
    ok = torch.where(ok.isinf(), ok.sign() * most, ok)
    assert bool(((ok - out[~bad].clamp(-most, most)).abs() <= far).all())
    assert bool(((norm[~bad].double() - lse[~bad]).abs() <= lse_off[~bad]).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("G,D,new", [(4, 64, [0, 3, 0, 1, 0]), (8, 128, [0, 60, 0, 45, 0]), (2, 256, [0, 70, 0, 90, 0])])
@pytest.mark.parametrize("prefix", [0, 101])
def test_requests_without_tokens(kvc_lib, dtype, G, D, new, prefix):
    """First, last and between others; a row of nothing among them.  Written, attended to and read back."""
    a = Attend(new, [0, 90, 10, 100, 5], prefix, 2, G, D, 8, dtype, seed=7)
    k, v = tokens_like(a.n, 2, D, dtype, 8), tokens_like(a.n, 2, D, dtype, 9)
    kd, vd = k.cuda(), v.cuda()
    kvc.kvc_append_paged(a.d.pool, a.batch, 1, kd.data_ptr(), vd.data_ptr(), 2 * D, hz.stream_handle())
    check_all_sizes(a)
    out = torch.zeros((2, a.n, 2, D), dtype=TORCH[dtype], device="cuda")
    kvc.kvc_read_paged(a.d.pool, a.batch, None, 1, out[0].data_ptr(), out[1].data_ptr(), 2 * D, hz.stream_handle())
    assert a.d.fault() == 0
    for got, x in zip(out.cpu(), (k, v)):
        assert torch.equal(got, held.rounded(held.stands_for(*held.quantized(x)), TORCH[dtype]))
