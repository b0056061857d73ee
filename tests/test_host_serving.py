"""Serving calls without a GPU: structures, workspaces, and every fault that the host can see, refused before anything is enqueued."""
import ctypes

import pytest

import paper_2602_09725_amd as kvc

A = 0x7F0000000000  # an aligned address that nothing reads
INVALID, UNSUPPORTED, SMALL = 1, 2, 3


def pool(**kw):
    base = dict(num_layers=32, num_kv_heads=8, head_dim=128, dtype=0, num_blocks=4096, block_size=16, n_rows=64, table_len=512,
                layer_cache_ptrs_dev=A, tables_ptr=A, lens_ptr=A, refs_ptr=A, err_ptr=A)
    base.update(kw)
    return kvc.Pool(**base)


def batch(**kw):
    base = dict(n_requests=8, n_new=None, most_new=1, rows_ptr=A, starts_ptr=None)
    base.update(kw)
    return kvc.Batch(**base)


def attention(**kw):
    base = dict(num_q_heads=32, scale=0.09, most_tokens=8000, prefix_tokens=4000, prefix_row=0, q_strides=(4096, 128), out_strides=(4096, 128))
    base.update(kw)
    return kvc.Attention(**base)


def status(call, *a):
    try:
        call(*a)
    except kvc.KvcError as e:
        return e.status
    return 0


def test_structures_match_the_header(kvc_lib):
    assert (ctypes.sizeof(kvc.Pool), ctypes.sizeof(kvc.Batch), ctypes.sizeof(kvc.Attention)) == (88, 40, 72)
    assert kvc.pool_validate(pool()) == 0
    for part in (pool(), batch(), attention()):
        for field, wrong in (("struct_size", ctypes.sizeof(part) - 8), ("abi_version", 1)):
            was = getattr(part, field)
            setattr(part, field, wrong)
            args = {kvc.Pool: (part, batch(), attention()), kvc.Batch: (pool(), part, attention()), kvc.Attention: (pool(), batch(), part)}[type(part)]
            assert status(kvc.attention_workspace, *args) == INVALID
            setattr(part, field, was)


BAD_POOLS = [
    (dict(num_layers=0), INVALID), (dict(num_kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(dtype=2), INVALID),
    (dict(num_blocks=0), INVALID), (dict(block_size=0), INVALID), (dict(n_rows=0), INVALID), (dict(table_len=0), INVALID),
    (dict(num_blocks=-1), INVALID), (dict(layer_cache_ptrs_dev=None), INVALID), (dict(tables_ptr=None), INVALID), (dict(lens_ptr=None), INVALID),
    (dict(tables_ptr=A + 2), INVALID), (dict(lens_ptr=A + 1), INVALID), (dict(refs_ptr=A + 2), INVALID), (dict(err_ptr=A + 2), INVALID),
    (dict(layer_cache_ptrs_dev=A + 4), INVALID), (dict(head_dim=12), UNSUPPORTED), (dict(n_rows=1 << 18), UNSUPPORTED),
    (dict(num_blocks=1 << 28), UNSUPPORTED), (dict(table_len=1 << 27), UNSUPPORTED),
    (dict(num_blocks=1 << 31, block_size=1, table_len=4), UNSUPPORTED), (dict(num_kv_heads=1 << 14), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,want", BAD_POOLS)
def test_bad_pools_are_refused_by_every_call(kvc_lib, kw, want):
    p, b, a = pool(**kw), batch(), attention(prefix_tokens=0, most_tokens=16)
    assert kvc.pool_validate(p) == want
    assert status(kvc.pages_workspace, p) == want
    big = 1 << 40
    assert status(kvc.kvc_pages_copy, p, A, A, 1) == want
    assert status(kvc.kvc_pages_fork, p, A, A, 1, A, big) == want
    assert status(kvc.kvc_pages_grow, p, A, None, 1, A, big) == want
    assert status(kvc.kvc_pages_free, p, A, 1) == want
    assert status(kvc.kvc_pages_compact, p, A, A, A, A, big) == want
    assert status(kvc.kvc_append_paged, p, b, 0, A, A, 1024) == want
    assert status(kvc.kvc_attend_paged, p, b, a, 0, A, A, A, A, big) == want


def test_the_largest_pools_are_taken(kvc_lib):
    for kw in (dict(num_blocks=(1 << 28) - 1), dict(table_len=(1 << 27) - 1), dict(n_rows=(1 << 18) - 1), dict(num_blocks=(1 << 31) - 1, block_size=1),
               dict(refs_ptr=None), dict(err_ptr=None), dict(head_dim=8, num_kv_heads=1)):
        assert kvc.pool_validate(pool(**kw)) == 0


def test_pages_calls_refuse(kvc_lib):
    p, need = pool(), kvc.pages_workspace(pool())
    for call in (lambda **k: status(kvc.kvc_pages_fork, k.get("pool", p), k.get("a", A), k.get("b", A), k.get("n", 4), k.get("w", A), k.get("bytes", need)),
                 lambda **k: status(kvc.kvc_pages_grow, k.get("pool", p), k.get("a", A), k.get("b", A), k.get("n", 4), k.get("w", A), k.get("bytes", need))):
        assert call(pool=pool(refs_ptr=None)) == INVALID
        assert call(a=None) == INVALID and call(a=A + 2) == INVALID and call(b=A + 2) == INVALID
        assert call(n=-1) == INVALID and call(n=65) == INVALID
        assert call(w=None) == INVALID and call(w=A + 128) == INVALID and call(bytes=need - 1) == SMALL
        assert call(n=0, a=None, w=None) == 0
    assert status(kvc.kvc_pages_fork, p, A, None, 4, A, need) == INVALID
    assert status(kvc.kvc_pages_fork, pool(num_layers=1 << 20, n_rows=5000), A, A, 4096, A, 1 << 40) == UNSUPPORTED
    assert status(kvc.kvc_pages_free, p, None, 1) == INVALID and status(kvc.kvc_pages_free, p, A + 1, 1) == INVALID
    assert status(kvc.kvc_pages_free, p, A, -1) == INVALID and status(kvc.kvc_pages_free, pool(refs_ptr=None), A, 1) == INVALID
    assert status(kvc.kvc_pages_free, p, None, 0) == 0
    for args in ((None, A, A), (A, None, A), (A, A, None), (A + 2, A, A), (A, A + 2, A), (A, A, A + 2)):
        assert status(kvc.kvc_pages_compact, p, *args, A, need) == INVALID
    assert status(kvc.kvc_pages_compact, p, A, A, A, A, need - 1) == SMALL
    assert status(kvc.kvc_pages_compact, pool(refs_ptr=None), A, A, A, A, need) == INVALID
    for args in ((None, A, 3), (A, None, 3), (A + 2, A, 3), (A, A + 2, 3), (A, A, -1), (A, A, 1 << 31)):
        assert status(kvc.kvc_pages_copy, p, *args) == INVALID
    assert status(kvc.kvc_pages_copy, p, None, None, 0) == 0
    assert status(kvc.kvc_pages_copy, p, A, A, 1 << 27) == UNSUPPORTED  # workgroups beyond a launch


BAD_BATCHES = [dict(n_requests=-1), dict(n_new=-1), dict(n_new=9), dict(n_new=9, starts_ptr=A + 2), dict(rows_ptr=A + 1), dict(most_new=-1),
               dict(n_new=9, starts_ptr=A, most_new=1), dict(n_new=9, starts_ptr=A, most_new=0), dict(n_new=1 << 31, starts_ptr=A, most_new=1 << 30)]


@pytest.mark.parametrize("kw", BAD_BATCHES)
def test_bad_batches_are_refused(kvc_lib, kw):
    assert status(kvc.kvc_append_paged, pool(), batch(**kw), 0, A, A, 1024) == INVALID
    assert status(kvc.kvc_attend_paged, pool(), batch(**kw), attention(), 0, A, A, A, A, 1 << 40) == INVALID


def test_append_refuses(kvc_lib):
    call = lambda **k: status(kvc.kvc_append_paged, pool(), k.get("batch", batch()), k.get("layer", 0), k.get("k", A), k.get("v", A), k.get("stride", 1024))  # noqa: E731
    assert call(layer=-1) == INVALID and call(layer=32) == INVALID
    assert call(k=None) == INVALID and call(v=None) == INVALID and call(k=A + 8) == INVALID and call(v=A + 2) == INVALID
    assert call(stride=-8) == INVALID and call(stride=1028) == INVALID
    assert call(batch=batch(n_requests=0), k=None, v=None) == 0


def test_attention_refuses(kvc_lib):
    def call(**k):
        own = {n: k.pop(n) for n in list(k) if n in ("batch", "pool", "layer", "q", "out", "lse", "w", "bytes")}
        return status(kvc.kvc_attend_paged, own.get("pool", pool()), own.get("batch", batch()), attention(**k), own.get("layer", 0), own.get("q", A),
                      own.get("out", A), own.get("lse", A), own.get("w", A), own.get("bytes", 1 << 40))

    assert call(num_q_heads=0) == INVALID and call(num_q_heads=36) == INVALID
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert call(scale=scale) == INVALID
    assert call(most_tokens=-1) == INVALID and call(most_tokens=8193) == INVALID  # 512 pages of 16
    assert call(prefix_tokens=-1) == INVALID and call(prefix_tokens=8001) == INVALID
    assert call(prefix_row=-1) == INVALID and call(prefix_row=64) == INVALID
    for name in ("q_strides", "out_strides"):
        for strides in ((4100, 128), (4096, 12), (-8, 128), (4096, -128)):
            assert call(**{name: strides}) == INVALID
    assert call(pool=pool(head_dim=264, num_kv_heads=1)) == UNSUPPORTED
    assert call(layer=32) == INVALID and call(layer=-1) == INVALID
    assert call(q=None) == INVALID and call(out=None) == INVALID and call(q=A + 8) == INVALID and call(out=A + 8) == INVALID and call(lse=A + 2) == INVALID
    need = kvc.attention_workspace(pool(), batch(), attention())
    assert need > 0 and call(w=None) == INVALID and call(w=A + 16) == INVALID and call(bytes=need - 1) == SMALL
    assert call(batch=batch(n_requests=0), q=None, out=None, w=None) == 0


def test_attention_workspace_holds_the_pieces(kvc_lib):
    """One piece needs none; more need a sum a channel and two numbers a row each."""
    line = lambda n, D=128: (n * 32 * D * 4 + 255) // 256 * 256 + n * 32 * 8  # noqa: E731
    assert kvc.attention_workspace(pool(), batch(), attention(prefix_tokens=0, most_tokens=0)) == 0
    assert kvc.attention_workspace(pool(), batch(), attention(prefix_tokens=0, most_tokens=100)) == 0
    assert kvc.attention_workspace(pool(), batch(), attention(prefix_tokens=100, most_tokens=100)) == 0
    assert kvc.attention_workspace(pool(), batch(), attention(prefix_tokens=100, most_tokens=120)) == line(16)
    for n in (1, 8, 64):
        need = kvc.attention_workspace(pool(), batch(n_requests=n), attention())
        assert need >= line(2 * n) and need <= line(130 * n)
    assert kvc.attention_workspace(pool(), batch(n_requests=0), attention()) == 0
