"""The example that serves from a restored cache, with its cache in 4 bits: every call of such a pool after one another, against dense copies of the
tokens that are quantized by tests/held_model.py."""
import os
import sys

import pytest
import torch

import held_model as held
from test_gpu_serving_example import restored

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import serve_shared_prefix as serve  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,block,prompt,D", [("f16", 16, 75, 64), ("bf16", 20, 300, 128), ("bf16", 4, 64, 32), ("f16", 32, 130, 256)])
def test_requests_over_a_restored_prompt_in_4_bits(kvc_lib, dtype, block, prompt, D):
    L, Q, H = 3, 8, 2
    m = serve.Model(L, Q, H, D, dtype)
    layout, frames, meta = serve.packed_prompt(m, prompt)
    kind = serve.DTYPES[dtype][0]
    server = serve.Server(m, 4, prompt + 60, -(-prompt // block) + 4 * (-(-60 // block) + 2), block, held=True)
    server.restore(layout, frames, meta, prompt)
    dense = {0: restored(layout, frames, meta, prompt, H, D, kind).cpu()}
    g = torch.Generator(device="cuda")
    g.manual_seed(3)

    def admit(rows):
        server.admit(rows)
        for row in rows:
            dense[row] = dense[0]

    def look_at(row):
        for layer in range(L):
            for got, want in zip(server.read_back(row, layer), dense[row][layer]):
                assert torch.equal(got.cpu(), held.rounded(held.stands_for(*held.quantized(want)), kind)), (row, layer)

    def step(rows, new):
        x = torch.randn((sum(new), m.width), generator=g, device="cuda").to(kind)
        server.step(x, rows, new)
        at = 0
        for row, n in zip(rows, new):
            more = torch.stack([torch.stack([k[at:at + n], v[at:at + n]]) for _, k, v, _, _ in server.seen]).cpu()
            dense[row] = torch.cat([dense[row], more], dim=2)
            total = dense[row].shape[2]
            seen = torch.arange(total)[None] <= (total - n + torch.arange(n))[:, None]
            for layer, (q, _, _, out, lse) in enumerate(server.seen):
                keys, values = dense[row][layer]
                for h in range(H):
                    heads = slice(h * Q // H, (h + 1) * Q // H)
                    want, want_lse, far, far_lse = held.attention(q[at:at + n, heads].cpu(), held.quantized(keys[:, h]), held.quantized(values[:, h]), seen,
                                                                  D ** -0.5, float(q.float().abs().max()))
                    assert bool(((out[at:at + n, heads].double().cpu() - want).abs() <= far).all()), (row, layer, h)
                    assert bool(((lse[at:at + n, heads].double().cpu() - want_lse).abs() <= far_lse).all()), (row, layer, h)
            at += n
        assert int(server.err.item()) == 0

    look_at(0)
    admit([1, 2, 3])
    step([1, 2, 3], [1, 9, 20])
    step([3, 1, 2], [1, 1, 1])
    server.finish([2])
    admit([4, 2])
    step([4, 2], [7, 1])
    server.compact()
    step([1, 2, 3, 4], [1, 1, 1, 1])
    for row in (0, 1, 2, 3, 4):
        look_at(row)
    server.finish([1, 2, 3, 4])
    assert int((server.refs > 0).sum()) == -(-prompt // block) and int(server.refs.max()) == 1
    server.compact()
    admit([1])
    step([1], [2])
    look_at(1)
