"""Pools in 4 bits, calls of many tokens, where a thread takes several quads side by side: written and read back, ragged, with what is at fault among them."""
import random

import pytest
import torch

import held_model as held
import kvc_harness as hz
import paper_2602_09725_amd as kvc
import serving_model as model
from test_gpu_held import HeldPool, i32, paged, tokens_like

pytestmark = pytest.mark.gpu
TORCH = held.TORCH
SHAPES = [(16, 40, 20, 20000), (8, 128, 16, 13500), (4, 256, 8, 13000), (64, 8, 4, 25000)]  # H, D, block, tokens


def places(d, page, slot):
    """Where the words [n][H][W] and pairs [n][H] of tokens on these pages and slots lie, in a kind's pages one after the other."""
    H, W, b = d.H, d.D // 8, d.block
    h = torch.arange(H)
    base = page * d.form.count
    word = base[:, None, None] + ((h[:, None] * (b // 4) + (slot // 4)[:, None, None]) * W + torch.arange(W)) * 4 + (slot % 4)[:, None, None]
    return word, base[:, None] + H * b * W + h * b + slot[:, None]


def put(d, kind_words, page, slot, x):
    """kind_words: [blocks * words] of a kind (int64)."""
    code, scale, mn = held.quantized(x)
    bits = lambda v: v.to(x.dtype).view(torch.int16).long() & 0xffff  # noqa: E731
    nan = 0x7e00 if x.dtype == torch.float16 else 0x7fc0
    word, pair = places(d, page, slot)
    kind_words[word] = (code.view(*code.shape[:2], -1, 8) << torch.tensor([held.shift_of(i) for i in range(8)])).sum(dim=-1)
    kind_words[pair] = torch.where(torch.isnan(scale), torch.full_like(bits(scale), nan), bits(scale) | bits(mn) << 16)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_many_tokens(kvc_lib, shape, dtype):
    H, D, block, most = SHAPES[shape]
    hz.say(f"[case] {SHAPES[shape]} {dtype}")
    rng = random.Random(shape)
    new = [1, 2, 0, 3, 5]
    while sum(new) < most:
        new.append(rng.choice([1, 4, rng.randint(2, 40), rng.randint(100, 1500)]))
    old = [rng.randint(0, 2 * block) for _ in new]
    lens = [n + o for n, o in zip(new, old)]
    blocks = sum(model.pages_of(n, block) + 1 for n in lens) + 5
    d = HeldPool(paged(lens, block, blocks, 3), lens, H, D, block, blocks, dtype, L=1)
    rows = list(range(len(new)))
    rng.shuffle(rows)
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + new[r])
    n = starts[-1]
    row = torch.tensor([r for r in rows for _ in range(new[r])])
    pos = torch.tensor([old[r] + j for r in rows for j in range(new[r])])
    # two rows have a page that the pool has not
    tables = torch.tensor(d.host_tables)
    for r, page in ((len(new) - 1, blocks), (len(new) // 2, -1)):
        tables[r, lens[r] // 2 // block] = page
    d.tables.copy_(tables.to(torch.int32))
    page = tables[row, pos // block]
    ok = (page >= 0) & (page < blocks)
    k, v = tokens_like(n, H, D, dtype, 1), tokens_like(n, H, D, dtype, 2)
    kd, vd, at, begin = k.cuda(), v.cuda(), i32(rows), i32(starts)
    batch = kvc.Batch(len(rows), n, max(new), at.data_ptr(), begin.data_ptr())
    want = d.host()
    for kind, x in enumerate((k, v)):
        put(d, want[0, kind].view(-1), page[ok], (pos % block)[ok], x[ok])
    write = lambda: kvc.kvc_append_paged(d.pool, batch, 0, kd.data_ptr(), vd.data_ptr(), H * D, hz.stream_handle())  # noqa: E731
    assert hz.kernels_of(write)[0][1][-1] > 1
    write()
    bad = 0 if ok.all() else model.FAULT_PAGE
    assert d.fault() == bad and torch.equal(d.host(), want)

    out = torch.full((2, n, H, D), 7.0, dtype=TORCH[dtype], device="cuda")
    read = lambda first, out: kvc.kvc_read_paged(d.pool, batch, first, 0, out[0].data_ptr(), out[1].data_ptr(), H * D, hz.stream_handle())  # noqa: E731
    assert hz.kernels_of(lambda: read(None, out))[0][1][-1] > 1
    read(None, out)
    assert d.fault() == bad
    for got, x in zip(out.cpu(), (k, v)):
        assert torch.equal(got[ok], held.rounded(held.stands_for(*held.quantized(x[ok])), TORCH[dtype])) and (got[~ok] == 7.0).all()

    # the rows' first tokens instead of their last ones; one request begins in front of its row, one ends behind it
    first = [0] * len(rows)
    begins = [i for i, r in enumerate(rows) if new[r] > 2]
    first[begins[0]], first[begins[1]] = -2, lens[rows[begins[1]]] - new[rows[begins[1]]] + 1
    pos = torch.cat([torch.arange(new[r]) + first[i] for i, r in enumerate(rows)])
    there = (pos >= 0) & (pos < torch.tensor(lens)[row])
    page = tables[row, pos.clamp(min=0) // block]
    there &= (page >= 0) & (page < blocks)
    d.err.zero_()
    out.fill_(7.0)
    read(i32(first).data_ptr(), out)
    assert d.fault() & model.FAULT_LIST
    word, pair = places(d, page[there], (pos % block)[there])
    value = lambda x: (x - (x >= 0x8000).long() * 0x10000).to(torch.int16).view(TORCH[dtype]).double()  # noqa: E731
    for kind in range(2):
        words = want[0, kind].view(-1)
        code = (words[word][..., None] >> torch.tensor([held.shift_of(i) for i in range(8)]) & 15).flatten(2)
        expect = held.rounded(held.stands_for(code, value(words[pair] & 0xffff), value(words[pair] >> 16)), TORCH[dtype])
        got = out[kind].cpu()
        assert torch.equal(got[there].nan_to_num(7e3), expect.nan_to_num(7e3)) and (got[~there] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_one_token_of_each_row_from_anywhere(kvc_lib, dtype):
    """No list of starts, but positions: request r reads the token at first[r]."""
    H, D, block, lens = 3, 64, 8, [1, 9, 30, 4, 17]
    d = HeldPool(paged(lens, block, 40, 5), lens, H, D, block, 40, dtype)
    first = [0, 8, 13, 4, -1]  # the last two are in no row
    out = torch.full((2, 5, H, D), 7.0, dtype=TORCH[dtype], device="cuda")
    kvc.kvc_read_paged(d.pool, kvc.Batch(5), i32(first).data_ptr(), 0, out[0].data_ptr(), out[1].data_ptr(), H * D, hz.stream_handle())
    assert d.fault() == model.FAULT_LIST
    code, scale, mn = d.form.get(d.host()[0].flatten(0, 1), TORCH[dtype])
    values = held.rounded(held.stands_for(code, scale, mn), TORCH[dtype]).view(2, 40, block, H, D)
    for r in range(3):
        want = values[:, d.host_tables[r][first[r] // block], first[r] % block]
        assert torch.equal(out[:, r].cpu().nan_to_num(7e3), want.nan_to_num(7e3))
    assert (out[:, 3:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,G", [([1, 1, 3], 4), ([60, 30, 61], 8)])
def test_queries_that_are_not_finite_reach_no_other_row(kvc_lib, dtype, new, G):
    from held_calls import Call, compare

    a = Call(new, [n + 50 for n in new], 203, 2, G, 128, 16, dtype, seed=3)
    wild = [(0, 1, 5, float("nan")), (1, 2, 127, float("inf")), (a.n - 1, 3, 8, float("-inf"))]
    clean = a.q.clone()
    for t, h, e, x in wild:
        a.q[t, h, e] = x
    got, norm = a.run()
    assert a.d.fault() == 0
    a.q = clean
    want = a.model()
    for t, h, _, _ in wild:
        assert not torch.isfinite(got[t, h]).any()
        got[t, h], norm[t, h] = want[0][t, h].to(got.dtype), want[1][t, h].float()
    compare(got, norm, want)
