"""Serving calls where books, lists and pages are not what a call may rely on, and attention at the ends of its types and addresses."""
import pytest
import torch

import kvc_harness as hz
import serving_model as model
from test_gpu_serving import Attend, i32

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
