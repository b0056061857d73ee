"""Serving calls larger than a launch: 2^24 workgroups of 256 threads are one too many, and are refused before anything is enqueued."""
import ctypes

import pytest

import paper_2602_09725_amd as kvc
from test_host_serving import A, UNSUPPORTED, attention, batch, pool, status

BIG = 1 << 60


@pytest.mark.parametrize("layers,n", [(80, 104858), (1 << 20, 8)])  # workgroups of 2 * layers pieces each
def test_copy(kvc_lib, layers, n):
    assert status(kvc.kvc_pages_copy, pool(num_layers=layers), A, A, n) == UNSUPPORTED


def test_fork(kvc_lib):
    assert status(kvc.kvc_pages_fork, pool(num_layers=80, n_rows=200000), A, A, 104858, A, BIG) == UNSUPPORTED


def test_free(kvc_lib):
    assert status(kvc.kvc_pages_free, pool(), A, (1 << 26) - 3) == UNSUPPORTED


def test_append(kvc_lib):
    n = (1 << 26) - 3  # 256 vectors a token, 1024 a workgroup
    assert status(kvc.kvc_append_paged, pool(), batch(n_requests=1, n_new=n, most_new=n, starts_ptr=A), 0, A, A, 1024) == UNSUPPORTED


@pytest.mark.parametrize("b,a,p", [
    (dict(n_requests=1 << 21), dict(prefix_tokens=0), {}),                                    # 8 units of the rows' own tokens a request
    (dict(n_requests=1 << 21), dict(num_q_heads=64, most_tokens=1100, prefix_tokens=1000), dict(num_kv_heads=1)),  # the join's workgroups of 8 rows
    (dict(n_requests=1 << 20), dict(num_q_heads=64, most_tokens=1100, prefix_tokens=1000), dict(num_kv_heads=1, head_dim=256)),  # of 4
])
def test_attention(kvc_lib, b, a, p):
    p, b, a = pool(**p), batch(**b), attention(**a)
    assert kvc.load().kvc_attention_workspace(ctypes.byref(p), ctypes.byref(b), ctypes.byref(a)) == ctypes.c_size_t(-1).value
    assert status(kvc.kvc_attend_paged, p, b, a, 0, A, A, A, A, BIG) == UNSUPPORTED


def test_the_largest_launches_are_not_refused(kvc_lib):
    """Their workspaces are told."""
    assert kvc.attention_workspace(pool(), batch(n_requests=(1 << 21) - 8), attention(prefix_tokens=0)) == 0
    p = pool(num_kv_heads=1)
    assert kvc.attention_workspace(p, batch(n_requests=(1 << 21) - 1), attention(num_q_heads=64, most_tokens=1100, prefix_tokens=1000)) > 0
