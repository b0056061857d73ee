"""Pools in 4 bits: many tokens of small weight behind one that has nearly all of it."""
import math

import pytest
import torch

import held_model as held
import kvc_harness as hz
from held_calls import Call, compare

pytestmark = pytest.mark.gpu
TORCH = held.TORCH
SHAPES = [  # new, owned, prefix, H, G, D, block: 16 rows a workgroup, a wave each, 128 rows
    ([1, 3], [1500, 400], 0, 1, 2, 64, 16),
    ([1, 2, 1], [40, 9, 70], 1000, 1, 4, 128, 16),
    ([1, 9], [300, 900], 0, 1, 2, 256, 8),
    ([1] * 70, [230 + 4 * i for i in range(70)], 0, 8, 1, 64, 8),
    ([180, 33, 120], [480, 70, 150], 0, 8, 8, 64, 16),
    ([150, 90, 160], [150, 200, 160], 701, 4, 8, 128, 16),
    ([180, 33, 120], [480, 70, 150], 0, 8, 8, 256, 16),
]


def put(a, pair_of):
    """pair_of(kind, first): scale and least value of a token; first: whether it is the first of its row."""
    d = a.d
    words = d.cache.cpu()
    bits = lambda v: torch.tensor(v, dtype=torch.float64).to(TORCH[a.dtype]).view(torch.int16).item() & 0xffff  # noqa: E731
    at = [d.form.pair(h, 0) for h in range(a.H)]
    for kind in range(2):
        for first in (False, True):
            s, m = pair_of(kind, first)
            w = bits(s) | bits(m) << 16
            w -= (w >= 2 ** 31) * 2 ** 32
            if first:
                for t in d.host_tables[0 if a.prefix else 1:]:  # (row 0 of no prefix has no page)
                    words[1, kind, t[0], at] = w
            else:
                words[1, kind, :, d.form.count - a.H * d.block:] = w
    d.cache.copy_(words)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("gap", [16.05, 18.0, 13.0])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_small_weights_behind_a_large_one(kvc_lib, dtype, gap, shape):
    """The first token has 2^gap times the weight of each other one, and values of steps of 1, the others 4 and a few steps of 2^-9.  A weight times its value's
    scale counts down to 2^-33 of the largest one: what the bound of held_model.attention has for fp16, which for bf16 allows 2^-25 (here that is all that the others have)."""
    hz.say(f"[case] {SHAPES[shape]} {dtype} {gap}")
    a = Call(*SHAPES[shape], dtype, seed=shape)
    a.q = torch.full_like(a.q, 0.25)  # a query's product with a key of one value c: 0.25 sqrt(D) c
    c = gap * math.log(2) / (0.25 * math.sqrt(a.D))
    put(a, lambda kind, first: ((1.0, 0.0) if first else (2.0 ** -9, 4.0)) if kind else ((0.0, c) if first else (0.0, 0.0)))
    got, norm = a.run()
    assert a.d.fault() == 0
    out, lse, off, lse_off = a.model()
    if dtype == "bf16":
        gap = float(torch.tensor(c, dtype=torch.bfloat16)) * 0.25 * math.sqrt(a.D) / math.log(2)
        for r, row in enumerate(a.rows):
            n = a.starts[r + 1] - a.starts[r]
            seen = a.d.host_lens[row] - n + 1 + torch.arange(n, dtype=torch.float64)
            most = 1 / (1 + (seen - 1) * 2.0 ** -gap)  # the first token's share, times its scale of 1
            steps = most * (seen - 1) * 2.0 ** 11      # what a step of all the others' weights adds, at least
            off[a.starts[r]:a.starts[r + 1]] -= (2.0 ** -25 - 2.0 ** -33) * steps[:, None, None]
        assert (off > 0).all()
    compare(got, norm, (out, lse, off, lse_off))


@pytest.mark.parametrize("element", range(1, 9))
@pytest.mark.parametrize("new", [1, 150])
def test_small_elements_of_a_query_beside_a_large_one(kvc_lib, element, new):
    """Of 2^-34 of the largest: it still counts, at each place of a word.  Keys of steps of 2^33 that only it meets make a product of 7/2 of it."""
    a = Call([new], [new + 1], 0, 1, 2, 64, 8, "bf16")
    a.q = torch.zeros_like(a.q)
    a.q[..., 0], a.q[..., element] = 1.0, 2.0 ** -34
    d = a.d
    words = d.cache.cpu()
    form, table = d.form, d.host_tables[1]
    value = lambda v: torch.tensor(v, dtype=torch.bfloat16).view(torch.int16).item() & 0xffff  # noqa: E731
    s, m = value(2.0 ** 33), value(-2.0 ** 36)
    for t in range(new + 1):
        page, slot = table[t // d.block], t % d.block
        words[1, 0, page, form.pair(0, slot)] = 0
        if t == 0:
            w = s | m << 16
            words[1, 0, page, form.pair(0, slot)] = w - (w >= 2 ** 31) * 2 ** 32
            for i in range(8):  # codes of 8, which with the least value stand for 0, and one of 15
                codes = [15 if 8 * i + k == element else 8 for k in range(8)]
                w = sum(c << held.shift_of(k) for k, c in enumerate(codes))
                words[1, 0, page, form.word(0, slot, i)] = w - (w >= 2 ** 31) * 2 ** 32
    d.cache.copy_(words)
    _, norm = a.run()
    assert a.d.fault() == 0
    # the first token's score is 7 / 2 * scale, exact but for a few roundings of 32 bits; of n others it is 0
    others = torch.arange(1, new + 1, dtype=torch.float64)[:, None]
    want = torch.log(math.exp(3.5 * a.scale) + others)
    assert bool(((norm.double() - want).abs() <= 2.0 ** -24 * (40 + new) * (1 + want.abs())).all())
