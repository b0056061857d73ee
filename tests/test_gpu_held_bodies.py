"""Every body of the attention over 4 bits (held_cases.py): results, tokens that no request covers, pages more than 4 GiB apart, and calls side by side on one pool."""
import math

import pytest
import torch

import kvc_harness as hz
import paper_2602_09725_amd as kvc
import serving_model as model
from held_calls import Call, compare
from held_cases import CASES
from test_gpu_held import i32

pytestmark = pytest.mark.gpu
ALL = pytest.mark.parametrize("case", range(len(CASES)))
DIRECT = [i for i, c in enumerate(CASES) if c[2] == 0]  # (test_host_held_bodies.py checks that these write results)


@ALL
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_results(kvc_lib, case, dtype):
    hz.say(f"[case] {CASES[case]} {dtype}")
    Call(*CASES[case], dtype, seed=case).check(q_pad=8)


@pytest.mark.parametrize("case", DIRECT)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_tokens_that_no_request_covers(kvc_lib, case, dtype):
    """Where results are written at once: those in front of the first request, behind the last one, and beyond a request's bound."""
    hz.say(f"[case] uncovered {CASES[case]} {dtype}")
    a = Call(*CASES[case], dtype, seed=case)
    starts, n, most = list(a.starts), a.n, max(a.new)

    def batch(most):
        a.batch = kvc.Batch(len(a.new), n, most, a.at.data_ptr(), a.begin.data_ptr())

    batch(max(2, most))
    whole, norms = a.run()
    assert a.d.fault() == 0
    for wrong in ("front", "back"):
        a.begin.copy_(i32([1] + starts[1:] if wrong == "front" else starts[:-1] + [n - 1]))
        got, norm = a.run()
        assert a.d.fault() == model.FAULT_LIST
        a.d.err.zero_()
        t = 0 if wrong == "front" else n - 1
        assert (got[t] == 0).all() and (norm[t] == -math.inf).all(), wrong
        keep = list(range(starts[1], n) if wrong == "front" else range(0, starts[-2]))  # (the other request sees other positions now)
        assert torch.equal(got[keep], whole[keep]) and torch.equal(norm[keep], norms[keep])
    if n > (most - 1) * len(a.new):  # (no such bound can be told)
        return
    a.begin.copy_(i32(starts))
    batch(most - 1)
    got, norm = a.run()
    assert a.d.fault() == model.FAULT_LIST
    want = a.model()
    for i in range(len(a.new)):
        if starts[i + 1] - starts[i] == most:
            want[0][starts[i + 1] - 1], want[1][starts[i + 1] - 1] = 0.0, -math.inf
    compare(got, norm, want)


@ALL
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_pages_beyond_4_gib(kvc_lib, case, dtype):
    hz.say(f"[case] far {CASES[case]} {dtype}")
    a = Call(*CASES[case], dtype, seed=case)
    near, a.d = a.d, a.far()
    got, norm = a.run()
    assert a.d.fault() == 0
    a.d = near
    compare(got, norm, a.model())


def test_calls_on_two_streams_over_one_pool(kvc_lib):
    """Decoding rows and a prompt of the same pool, each call with rows, queries, results and a workspace of its own: what each gives alone."""
    a = Call([1, 1, 3, 70, 1, 30], [500, 70, 40, 300, 70, 40], 333, 2, 4, 128, 16, "bf16", seed=8)
    heads, d = a.H * a.G, a.d
    q = a.q.cuda()

    def part(requests):
        rows = [a.rows[r] for r in requests]
        tokens = [t for r in requests for t in range(a.starts[r], a.starts[r + 1])]
        new = [a.starts[r + 1] - a.starts[r] for r in requests]
        starts = [0]
        for m in new:
            starts.append(starts[-1] + m)
        at, begin, own = i32(rows), i32(starts), q[tokens].contiguous()
        batch = kvc.Batch(len(rows), len(tokens), max(new), at.data_ptr(), begin.data_ptr())
        call = kvc.Attention(heads, a.scale, a.most_tokens, a.prefix, 0, own.stride()[:2], own.stride()[:2])
        size = kvc.attention_workspace(d.pool, batch, call)
        space = torch.empty(size, dtype=torch.uint8, device="cuda")

        def run(stream):
            out, norm = torch.full_like(own, 7.0), torch.full((len(tokens), heads), 7.0, device="cuda")
            torch.cuda.synchronize()
            return out, norm, lambda: kvc.kvc_attend_paged(d.pool, batch, call, 1, own.data_ptr(), out.data_ptr(), norm.data_ptr(), space.data_ptr(), size, stream)

        return tokens, run, (at, begin)

    few = [r for r in range(6) if a.starts[r + 1] - a.starts[r] <= 3]
    parts = [part(few), part([r for r in range(6) if r not in few])]
    want = a.model()
    alone = []
    for tokens, run, _ in parts:
        out, norm, call = run(hz.stream_handle())
        call()
        torch.cuda.synchronize()
        compare(out.cpu(), norm.cpu(), [x[tokens] for x in want])
        alone.append((out, norm))
    streams = [torch.cuda.Stream() for _ in parts]
    for _ in range(5):
        jobs = [run(s.cuda_stream) for (_, run, _), s in zip(parts, streams)]
        for _, _, call in jobs:
            call()
        torch.cuda.synchronize()
        for (out, norm, _), (first, first_norm) in zip(jobs, alone):
            assert torch.equal(out, first) and torch.equal(norm, first_norm)
    assert d.fault() == 0
