"""Calls on pools in 4 bits without a GPU: sizes, and every fault that the host can see."""
import pytest

import paper_2602_09725_amd as kvc
from test_host_serving import A, INVALID, SMALL, UNSUPPORTED, attention, batch, pool, status

Q4 = kvc.KVC_HELD_Q4


def test_bytes_of_a_page(kvc_lib):
    for H, D, b in ((8, 128, 16), (1, 8, 4), (2, 40, 20), (3, 256, 64)):
        assert kvc.page_bytes(pool(num_kv_heads=H, head_dim=D, block_size=b)) == 2 * H * D * b
        for dtype in (0, 1):
            assert kvc.page_bytes(pool(num_kv_heads=H, head_dim=D, block_size=b, dtype=dtype | Q4)) == H * b * (D // 2 + 4)
    with pytest.raises(kvc.KvcError):
        kvc.page_bytes(pool(dtype=2))


BAD = [(dict(dtype=2 | Q4), INVALID), (dict(dtype=Q4 << 1), INVALID), (dict(dtype=-1), INVALID), (dict(dtype=Q4, block_size=18), UNSUPPORTED),
       (dict(dtype=Q4, block_size=2), UNSUPPORTED), (dict(dtype=Q4, head_dim=264), UNSUPPORTED), (dict(dtype=Q4 | 1, head_dim=12), UNSUPPORTED),
       (dict(dtype=Q4, num_layers=0), INVALID), (dict(dtype=Q4, lens_ptr=None), INVALID)]


@pytest.mark.parametrize("kw,want", BAD)
def test_bad_pools_are_refused(kvc_lib, kw, want):
    p, b, a = pool(**kw), batch(), attention(prefix_tokens=0, most_tokens=16)
    wide = pool(**{k: v for k, v in kw.items() if k != "dtype"}) if kw.get("num_layers", 1) and kw.get("lens_ptr", A) else pool()
    assert kvc.pool_validate(p) == want
    assert status(kvc.kvc_append_paged, p, b, 0, A, A, 1024) == want
    assert status(kvc.kvc_read_paged, p, b, None, 0, A, A, 1024) == want
    assert status(kvc.kvc_attend_paged, p, b, a, 0, A, A, A, A, 1 << 40) == want
    assert status(kvc.kvc_pages_convert, p, wide, A, A, 1) == want
    assert status(kvc.kvc_pages_copy, p, A, A, 1) == want


def test_held_pools_are_taken(kvc_lib):
    for kw in (dict(), dict(head_dim=256), dict(head_dim=8, num_kv_heads=1, block_size=4), dict(block_size=20)):
        for dtype in (0, 1):
            assert kvc.pool_validate(pool(dtype=dtype | Q4, **kw)) == 0


def test_read_refuses(kvc_lib):
    for dtype in (0, 1, Q4, 1 | Q4):
        def call(**k):
            return status(kvc.kvc_read_paged, pool(dtype=dtype), k.get("batch", batch()), k.get("first"), k.get("layer", 0), k.get("k", A), k.get("v", A),
                          k.get("stride", 1024))

        assert call(layer=-1) == INVALID and call(layer=32) == INVALID
        assert call(k=None) == INVALID and call(v=None) == INVALID and call(k=A + 8) == INVALID and call(v=A + 2) == INVALID
        assert call(stride=1016) == INVALID and call(stride=0) == INVALID and call(stride=-1024) == INVALID and call(stride=1028) == INVALID
        assert call(first=A + 2) == INVALID
        assert call(batch=batch(n_new=9)) == INVALID
        assert call(batch=batch(n_requests=0), k=None, v=None) == 0
        assert call(batch=batch(n_requests=(1 << 31) - 1, n_new=5, starts_ptr=A)) == UNSUPPORTED


def test_append_to_a_held_pool_refuses(kvc_lib):
    def call(**k):
        return status(kvc.kvc_append_paged, pool(dtype=Q4), k.get("batch", batch()), k.get("layer", 0), k.get("k", A), k.get("v", A), k.get("stride", 1024))

    assert call(layer=32) == INVALID and call(k=None) == INVALID and call(v=A + 8) == INVALID and call(stride=1028) == INVALID and call(stride=-8) == INVALID
    assert call(batch=batch(n_requests=0), k=None) == 0
    assert call(batch=batch(n_requests=1 << 30, n_new=1 << 30, starts_ptr=A)) == UNSUPPORTED  # workgroups beyond a launch


def test_convert_refuses(kvc_lib):
    wide, held = pool(), pool(dtype=Q4, num_blocks=99)

    def call(a=wide, b=held, src=A, dst=A, n=1):
        return status(kvc.kvc_pages_convert, a, b, src, dst, n)

    assert call(b=pool()) == INVALID and call(a=held) == INVALID  # alike in form
    for kw in (dict(num_layers=31), dict(num_kv_heads=4), dict(head_dim=64), dict(block_size=32), dict(dtype=Q4 | 1)):
        assert call(b=pool(**{"dtype": Q4, **kw})) == INVALID
        assert call(a=pool(**{"dtype": Q4, **kw}), b=wide) == INVALID
    assert call(n=-1) == INVALID and call(n=1 << 31) == INVALID
    for args in (dict(src=None), dict(dst=None), dict(src=A + 2), dict(dst=A + 1)):
        assert call(**args) == INVALID
    assert call(src=None, dst=None, n=0) == 0
    assert call(n=1 << 27) == UNSUPPORTED and call(a=held, b=wide, n=1 << 27) == UNSUPPORTED  # workgroups beyond a launch


def test_attention_on_a_held_pool_refuses(kvc_lib):
    def call(**k):
        own = {n: k.pop(n) for n in list(k) if n in ("batch", "layer", "q", "out", "lse", "w", "bytes")}
        return status(kvc.kvc_attend_paged, pool(dtype=Q4), own.get("batch", batch()), attention(**k), own.get("layer", 0), own.get("q", A),
                      own.get("out", A), own.get("lse", A), own.get("w", A), own.get("bytes", 1 << 40))

    assert call(num_q_heads=36) == INVALID and call(scale=0.0) == INVALID and call(most_tokens=8193) == INVALID and call(prefix_tokens=8001) == INVALID
    assert call(layer=32) == INVALID and call(q=None) == INVALID and call(out=A + 8) == INVALID and call(lse=A + 2) == INVALID
    need = kvc.attention_workspace(pool(dtype=Q4), batch(), attention())
    assert need > 0 and call(w=None) == INVALID and call(w=A + 16) == INVALID and call(bytes=need - 1) == SMALL
    assert call(batch=batch(n_requests=0), q=None, out=None, w=None) == 0
