"""Which bodies of the attention over 4 bits a call takes: the library's own planner, asked through tests/held_plan.cpp."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

import paper_2602_09725_amd as kvc
from paper_2602_09725_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
A = 0x7F0000000000  # an aligned address that nothing reads


class Part(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("waves", "splits", "lone", "tokens")]


class Plan(C.Structure):
    _fields_ = [("pieces", C.c_int32), ("part", Part * 2)]


@functools.lru_cache(None)
def _planner():
    with tempfile.TemporaryDirectory() as at:
        out = os.path.join(at, "held_plan.so")
        rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-I", os.path.join(build.ROOT, "include"),
                        "-I", build.CSRC, os.path.join(HERE, "held_plan.cpp"), build.LIB, "-Wl,-rpath," + build.HERE, "-o", out], check=True)
        kvc.load()
        return C.CDLL(out).held_plan


def plan_of(new, owned, prefix, H, G, D, block, dtype, blocks=4096):
    """The plan of requests of so many new tokens, on rows of so many tokens beyond the prefix; blocks: pages of the pool."""
    most, code = prefix + max(owned), kvc.KVC_F16 if dtype == "f16" else kvc.KVC_BF16
    pool = kvc.Pool(2, H, D, code | kvc.KVC_HELD_Q4, blocks, block, len(new) + 1, -(-most // block) + 1, A, A, A, A, A)
    batch = kvc.Batch(len(new), sum(new), max(new), A, None if max(new) == 1 and min(new) == 1 else A)
    plan = Plan()
    status = _planner()(C.byref(pool), C.byref(batch), C.byref(kvc.Attention(H * G, 1.0, most, prefix, 0, (H * G * D, D), (H * G * D, D))), C.byref(plan))
    assert status == 0
    return plan


def bodies_of(plan):
    """The bodies of a call's parts: of 128 rows a workgroup, of 16 rows a workgroup, or of 16 rows a wave; each with whether it writes results or pieces."""
    found = set()
    for part in plan.part:
        if part.splits:
            found.add(("block" if part.waves == 4 else "wave" if part.lone else "rows", "results" if plan.pieces == 1 else "pieces"))
    return found


def size_of(D):
    return 64 if D <= 64 else 128 if D <= 128 else 256
