"""The example's pool in 4 bits: a prompt of several chunks comes into it without its 16-bit cache being there at any time."""
import os
import sys

import pytest
import torch

import held_model as held
from test_gpu_serving_example import restored

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import serve_shared_prefix as serve  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,block,prompt,D", [("f16", 16, 9000, 64), ("bf16", 20, 8192, 128), ("f16", 4096, 9001, 32), ("bf16", 32, 6143, 64)])
def test_a_prompt_comes_in_piece_by_piece(kvc_lib, dtype, block, prompt, D):
    L, Q, H = 2, 4, 2
    m = serve.Model(L, Q, H, D, dtype)
    kind = serve.DTYPES[dtype][0]
    layout, frames, meta = serve.packed_prompt(m, prompt)
    want = restored(layout, frames, meta, prompt, H, D, kind).cpu()
    server = serve.Server(m, 2, prompt + 8, -(-prompt // block) + 4, block, held=True)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before, wide = torch.cuda.memory_allocated(), want.numel() * 2
    server.restore(layout, frames, meta, prompt)
    # (a chunk of 2048 tokens and two pages of 16 bits, and lists)
    most = L * 2 * H * D * 2 * (2048 + 2 * block) + (1 << 20)
    assert torch.cuda.max_memory_allocated() - before <= most and (most < wide or block > 2048)
    assert torch.cuda.memory_allocated() - before <= 1 << 16
    for layer in range(L):
        for got, x in zip(server.read_back(0, layer), want[layer]):
            assert torch.equal(got.cpu(), held.rounded(held.stands_for(*held.quantized(x)), kind))
    assert int(server.err.item()) == 0
