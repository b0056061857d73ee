"""Pools in 4 bits: positions below the prefix are the prefix row's, also where the prefix ends inside four tokens that a page has side by side."""
import pytest
import torch

import kvc_harness as hz
import serving_model as model
from held_calls import Call

pytestmark = pytest.mark.gpu
SHAPES = [  # new, owned beyond the prefix, H, G, D, block: 16 rows a workgroup, 128 rows, a wave each
    ([1, 1, 3], [40, 9, 70], 2, 4, 128, 16),
    ([1, 2, 1], [40, 9, 70], 1, 4, 64, 8),
    ([1, 9], [40, 30], 1, 2, 256, 8),
    ([60, 30, 61], [60, 80, 70], 2, 8, 64, 16),
    ([150, 90, 160], [150, 200, 160], 4, 8, 200, 16),
    ([150, 90, 160], [150, 200, 160], 4, 8, 128, 16),
    ([1] * 70, [1 + 4 * i for i in range(70)], 8, 1, 40, 8),
]
BOTH = pytest.mark.parametrize("dtype", ["f16", "bf16"])
ALL = pytest.mark.parametrize("shape", range(len(SHAPES)))


def call(shape, prefix, dtype, more=None):
    new, owned, *rest = SHAPES[shape]
    hz.say(f"[case] prefix {prefix} {SHAPES[shape]} {dtype}")
    return Call(new, owned if more is None else more, prefix, *rest, dtype, seed=shape + prefix)


def others(a):
    """Slots below the prefix in the rows' own pages hold other tokens than the prefix row's, some of them NaN or infinite."""
    d, part = a.d, a.prefix % a.d.block
    words = d.cache.cpu()
    g = torch.Generator().manual_seed(99)
    inf, nan = (0x7c00, 0x7e00) if a.dtype == "f16" else (0x7f80, 0x7fc0)
    for r, t in enumerate(d.host_tables[1:]):
        for slot in range(part):
            at = [d.form.word(h, slot, w) for h in range(a.H) for w in range(a.D // 8)]
            words[:, :, t[a.prefix // d.block], at] = torch.randint(-2 ** 31, 2 ** 31, (2, 2, len(at)), generator=g).to(torch.int32)
            for kind in range(2):
                pair = [nan, inf | nan << 16, None, inf][(r + slot + kind) % 4]
                if pair is not None:
                    words[:, kind, t[a.prefix // d.block], [d.form.pair(h, slot) for h in range(a.H)]] = pair
    d.cache.copy_(words)


@ALL
@BOTH
@pytest.mark.parametrize("prefix", [301, 302, 303, 257, 514, 130, 67, 3, 1])
def test_the_prefix_is_read_through_its_row(kvc_lib, shape, dtype, prefix):
    """Rows' tables that lack the prefix's whole pages, and own pages with something else in its last slots: neither is looked at, nor told."""
    a = call(shape, prefix, dtype)
    others(a)
    shared = prefix // a.d.block
    for r, t in enumerate(a.d.host_tables[1:]):
        t[:shared] = [[10 ** 6, -1, a.d.blocks][r % 3]] * shared
    a.d.tables.copy_(torch.tensor(a.d.host_tables, dtype=torch.int32))
    a.check()


@ALL
@BOTH
@pytest.mark.parametrize("prefix,there", [(301, 300), (303, 301), (259, 257), (513, 512), (302, 300), (302, 299), (3, 2), (2, 0)])
def test_a_prefix_row_that_ends_a_little_early(kvc_lib, shape, dtype, prefix, there):
    """What it lacks is seen by nobody, whatever the rows' own pages have there, and is told."""
    a = call(shape, prefix, dtype)
    a.d.host_lens[0] = there
    a.d.lens.copy_(torch.tensor(a.d.host_lens, dtype=torch.int32))
    a.check(fault=model.FAULT_LIST)


@ALL
@BOTH
def test_rows_that_end_where_the_prefix_does(kvc_lib, shape, dtype):
    """Rows of the prefix's length, of a token more and of less: a table's entry for a quad that has none of the row's own tokens is not looked at."""
    a = call(shape, 302, dtype)
    lens = [[302, 303, 301, 304, 300, 305][r % 6] for r in range(len(a.new))]
    a.d.host_lens[1:] = lens
    a.d.lens.copy_(torch.tensor(a.d.host_lens, dtype=torch.int32))
    for r, n in enumerate(lens):
        if n <= 302:
            a.d.host_tables[r + 1] = [-1] * len(a.d.host_tables[0])
    a.d.tables.copy_(torch.tensor(a.d.host_tables, dtype=torch.int32))
    a.check()


@ALL
@BOTH
@pytest.mark.parametrize("prefix", [302, 2])
def test_a_bound_that_is_the_prefix(kvc_lib, shape, dtype, prefix):
    """No token lies beyond the prefix: there is nothing of the rows' own, and only the prefix's row is read."""
    a = call(shape, prefix, dtype)
    a.most_tokens = prefix
    a.d.host_lens[1:] = [prefix] * len(a.new)
    a.d.lens.copy_(torch.tensor(a.d.host_lens, dtype=torch.int32))
    for t in a.d.host_tables[1:]:
        t[:] = [-1] * len(t)
    a.d.tables.copy_(torch.tensor(a.d.host_tables, dtype=torch.int32))
    a.check()


@BOTH
@pytest.mark.parametrize("shape", [0, 4, 6])
def test_a_page_outside_the_pool_at_the_end(kvc_lib, shape, dtype):
    """The prefix's last page: it alone is not seen, and is told."""
    a = call(shape, 302, dtype)
    a.d.host_tables[0][302 // a.d.block] = a.d.blocks + 7
    a.d.tables.copy_(torch.tensor(a.d.host_tables, dtype=torch.int32))
    a.check(fault=model.FAULT_PAGE)
