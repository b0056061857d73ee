"""The example that serves from a restored cache, against dense caches that are kept beside it."""
import os
import sys

import pytest
import torch

import serving_model as model

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import serve_shared_prefix as serve  # noqa: E402

pytestmark = pytest.mark.gpu


def restored(layout, frames, meta, n, heads, dim, dtype):
    """The prompt's cache, restored to a contiguous one: [layers][2][n][heads][dim]."""
    import paper_2602_09725_amd as kvc

    out = torch.empty((layout.num_layers, 2, n, heads, dim), dtype=dtype, device="cuda")
    width = heads * dim
    kvc.kvc_restore(layout, frames.data_ptr(), meta.data_ptr(), n, out.data_ptr(), (2 * n * width, n * width, width), serve.stream())
    return out


@pytest.mark.parametrize("dtype,block,prompt", [("f16", 16, 75), ("bf16", 5, 300), ("bf16", 32, 64)])
def test_requests_over_a_restored_prompt(kvc_lib, dtype, block, prompt):
    L, Q, H, D = 3, 8, 2, 64
    m = serve.Model(L, Q, H, D, dtype)
    layout, frames, meta = serve.packed_prompt(m, prompt)
    kind = serve.DTYPES[dtype][0]
    server = serve.Server(m, 4, prompt + 60, -(-prompt // block) + 4 * (-(-60 // block) + 2), block)
    server.restore(layout, frames, meta, prompt)
    dense = {0: restored(layout, frames, meta, prompt, H, D, kind)}
    g = torch.Generator(device="cuda")
    g.manual_seed(3)

    def admit(rows):
        server.admit(rows)
        for row in rows:
            dense[row] = dense[0]

    def step(rows, new):
        x = torch.randn((sum(new), m.width), generator=g, device="cuda").to(kind)
        server.step(x, rows, new)
        at = 0
        for row, n in zip(rows, new):
            more = torch.stack([torch.stack([k[at:at + n], v[at:at + n]]) for _, k, v, _, _ in server.seen])
            dense[row] = torch.cat([dense[row], more], dim=2)
            total = dense[row].shape[2]
            seen = torch.arange(total)[None] <= (total - n + torch.arange(n))[:, None]
            for layer, (q, _, _, out, lse) in enumerate(server.seen):
                keys, values = dense[row][layer].cpu()
                for h in range(H):
                    heads = slice(h * Q // H, (h + 1) * Q // H)
                    want = model.attention(q[at:at + n, heads].cpu(), keys[:, h], values[:, h], seen, D ** -0.5)
                    far, far_lse = model.attention_bounds(*want, total, D, kind)
                    assert bool(((out[at:at + n, heads].double().cpu() - want[0]).abs() <= far).all()), (row, layer, h)
                    assert bool(((lse[at:at + n, heads].double().cpu() - want[1]).abs() <= far_lse).all()), (row, layer, h)
            at += n
        assert int(server.err.item()) == 0

    admit([1, 2, 3])
    step([1, 2, 3], [1, 9, 20])
    step([3, 1, 2], [1, 1, 1])
    server.finish([2])
    admit([4, 2])
    step([4, 2], [7, 1])
    server.compact()
    step([1, 2, 3, 4], [1, 1, 1, 1])
    server.finish([1, 2, 3, 4])
    assert int((server.refs > 0).sum()) == -(-prompt // block) and int(server.refs.max()) == 1
    server.compact()
    admit([1])
    step([1], [2])
