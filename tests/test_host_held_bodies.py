"""The cases of test_gpu_held_bodies.py meet every body of the attention over 4 bits (sizes x bodies x results written or pieces), in both types."""
import pytest

from held_cases import CASES
from held_plans import bodies_of, plan_of, size_of


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("far", [False, True])
def test_every_body_is_met(kvc_lib, dtype, far):
    met = set()
    for case in CASES:
        _, _, _, H, _, D, block = case
        blocks = (1 << 32) // (block * H * (D // 2 + 4)) + 3000 if far else 4096
        met |= {(size_of(D), *body) for body in bodies_of(plan_of(*case, dtype, blocks=blocks))}
    lacks = {(size, body, what) for size in (64, 128, 256) for body in ("rows", "wave", "block") for what in ("results", "pieces")} - met
    assert not lacks, sorted(lacks)
    for case in CASES:  # (without a prefix there is one piece: what no request covers is written by the same kernel)
        assert case[2] or {what for _, what in bodies_of(plan_of(*case, dtype))} == {"results"}
