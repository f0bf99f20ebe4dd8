"""include/mars_cache.h: every function is exported, the binding's structs are the header's, and bad arguments are
refused on the host (no GPU: no call here reaches a kernel)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "mars_cache.h")).read()
CODE = re.sub(r"/\*.*?\*/", "", HEADER, flags=re.S)
ARG, DTYPE, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def C():
    from paper_2601_15498_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2601_15498_amd import build
        build.build()
    from paper_2601_15498_amd import cache
    return cache


def test_every_declared_function_is_exported(C):
    names = set(re.findall(r"\b(mars_[a-z_]+)\s*\(", CODE))
    assert names == {"mars_kv_head_bytes", "mars_kv_append", "mars_kv_read", "mars_tree_mask", "mars_kv_attention_workspace_bytes",
                     "mars_kv_attention", "mars_kv_commit", "mars_kv_reserve_workspace_bytes", "mars_kv_reserve", "mars_kv_fork",
                     "mars_kv_release", "mars_kv_copy_pages"}
    for name in names:
        assert hasattr(C.lib(), name)


def fields(struct):
    text = re.search(r"typedef struct %s \{(.*?)\}" % struct, CODE, re.S).group(1)
    return [(kind, name.strip()) for kind, names in re.findall(r"(void\*|int32_t\*|int32_t|int64_t)\s+([^;]+);", text) for name in names.split(",")]


def test_structs_and_codes_are_the_headers(C):
    size = {"void*": 8, "int32_t*": 8, "int64_t": 8, "int32_t": 4}
    for struct, cls in (("mars_kv_cache", C.CacheStruct), ("mars_kv_rows", C.RowsStruct)):
        want = fields(struct)
        assert [n for _, n in want] == [n for n, _ in cls._fields_]
        assert [size[t] for t, _ in want] == [ctypes.sizeof(t) for _, t in cls._fields_]
    for name, value in re.findall(r"(MARS_KV_[A-Z_]+)\s*=\s*(\d+)", CODE):
        assert getattr(C, name) == int(value)
    assert int(re.search(r"MARS_KV_MAX_REQUESTS (\d+)", CODE).group(1)) == C.MARS_KV_MAX_REQUESTS


def test_head_bytes(C):
    f = C.lib().mars_kv_head_bytes
    assert f(128, 64) == 64 * 136 and f(64, 8) == 544 and f(256, 256) == 256 * 272
    for d, p in ((96, 64), (0, 8), (128, 4), (128, 24), (128, 512), (-64, 8)):
        assert f(d, p) == 0
        with pytest.raises(C.MarsError):
            C.mars_kv_head_bytes(d, p)


P = 0x1000  # never dereferenced: every call below fails a check first


def a_cache(C, **kw):
    f = dict(pool=P, page_table=P, lens=P, held=P, refs=P, layers=2, pages=9, heads=4, dim=128, page=16, sequences=3, width=5)
    f.update(kw)
    return C.CacheStruct(*(f[n] for n, _ in C.CacheStruct._fields_))


def some_rows(C, **kw):
    f = dict(data=P, request=4096, node=512, head=128)
    f.update(kw)
    return C.RowsStruct(*(f[n] for n, _ in C.RowsStruct._fields_))


BAD_CACHES = [dict(layers=0), dict(pages=0), dict(heads=0), dict(dim=96), dict(page=12), dict(sequences=0), dict(width=0), dict(page_table=None),
              dict(width=1 << 30), dict(heads=1 << 27)]


def test_append_and_read_refuse(C):
    L = C.lib()

    def append(cache=None, layer=0, k=None, v=None, dtype=1, B=2, N=3):
        return L.mars_kv_append(cache or a_cache(C), layer, None, k or some_rows(C), v or some_rows(C), dtype, None, B, N, None, None)

    def read(cache=None, layer=0, k=None, v=None, dtype=1, B=2, N=3):
        return L.mars_kv_read(cache or a_cache(C), layer, None, None, k or some_rows(C), v or some_rows(C), dtype, B, N, None)

    for f in (append, read):
        for kw in BAD_CACHES + [dict(pool=None), dict(pool=P + 8)]:
            assert f(a_cache(C, **kw)) == ARG, kw
        assert f(layer=-1) == ARG and f(layer=2) == ARG and f(dtype=3) == DTYPE
        assert f(B=0) == ARG and f(B=4097) == ARG and f(N=0) == ARG and f(N=1 << 25) == ARG
        for bad in (dict(data=None), dict(data=P + 2), dict(node=12), dict(request=3), dict(head=1)):
            assert f(k=some_rows(C, **bad)) == ARG and f(v=some_rows(C, **bad)) == ARG
        assert f(k=some_rows(C, node=6), dtype=0) == ARG
    assert append(a_cache(C, lens=None)) == ARG
    assert L.mars_kv_append(None, 0, None, some_rows(C), some_rows(C), 1, None, 1, 1, None, None) == ARG


def test_attention_refuses(C):
    L = C.lib()

    def call(cache=None, layer=0, q=None, dtype=1, q_heads=8, mask=None, scale=1.0, max_len=0, out=None, B=2, N=3, ws=0x100000, n=1 << 40):
        return L.mars_kv_attention(cache or a_cache(C), layer, None, q or some_rows(C), dtype, q_heads, None, mask, scale, max_len,
                                   out or some_rows(C), None, B, N, ws, n, None)

    for kw in BAD_CACHES + [dict(pool=None), dict(lens=None)]:
        assert call(a_cache(C, **kw)) == ARG, kw
    assert call(layer=2) == ARG and call(dtype=2) == DTYPE and call(q_heads=6) == ARG and call(q_heads=2) == ARG and call(q_heads=0) == ARG
    assert call(B=0) == ARG and call(N=0) == ARG and call(max_len=-1) == ARG
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=scale) == ARG
    assert call(q=some_rows(C, data=P + 4)) == ARG and call(out=some_rows(C, head=4)) == ARG
    assert call(mask=P, N=1025) == ARG
    assert call(ws=None) == WORKSPACE and call(ws=0x100010) == WORKSPACE and call(n=255) == WORKSPACE
    f = L.mars_kv_attention_workspace_bytes
    assert f(1, 1, 32, 8, 128, 1) % 256 == 0 and f(1, 1, 32, 8, 128, 1) > 0
    for bad in ((0, 1, 32, 8, 128, 1), (1, 0, 32, 8, 128, 1), (1, 1, 33, 8, 128, 1), (1, 1, 32, 8, 80, 1), (1, 1, 32, 8, 128, 2), (1, 1, 32, 0, 128, 1)):
        assert f(*bad) == 0


def test_the_calls_on_tables_refuse(C):
    L = C.lib()
    assert L.mars_tree_mask(None, None, 1, 4, P, None, None) == ARG and L.mars_tree_mask(P, None, 1, 4, None, None, None) == ARG
    assert L.mars_tree_mask(P, None, 1, 1025, P, None, None) == ARG and L.mars_tree_mask(P, None, 0, 4, P, None, None) == ARG
    commit = lambda cache=None, a=P, p=P, n=P, B=1, N=4: L.mars_kv_commit(cache or a_cache(C), None, a, p, B, N, n, None, None)  # noqa: E731
    assert commit(a=None) == ARG and commit(p=None) == ARG and commit(n=None) == ARG and commit(B=0) == ARG and commit(N=0) == ARG
    reserve = lambda cache=None, B=1, N=4, ws=0x100000, n=1 << 30: L.mars_kv_reserve(cache or a_cache(C), None, None, B, N, None, ws, n, None)  # noqa: E731
    assert reserve(B=0) == ARG and reserve(N=0) == ARG and reserve(ws=None) == WORKSPACE and reserve(n=100) == WORKSPACE
    assert reserve(ws=0x100001) == WORKSPACE
    fork = lambda cache=None, s=P, d=P, B=1: L.mars_kv_fork(cache or a_cache(C), s, d, B, None, None)  # noqa: E731
    assert fork(s=None) == ARG and fork(d=None) == ARG and fork(B=0) == ARG
    release = lambda cache=None, B=1: L.mars_kv_release(cache or a_cache(C), P, B, None, None)  # noqa: E731
    assert release(B=0) == ARG
    for f in (commit, reserve, fork, release):
        for kw in BAD_CACHES + [dict(lens=None)]:
            assert f(a_cache(C, **kw)) == ARG, kw
    for f in (reserve, fork, release):
        assert f(a_cache(C, held=None)) == ARG and f(a_cache(C, refs=None)) == ARG
    assert L.mars_kv_copy_pages(a_cache(C, pool=None), P, P, 1, None) == ARG and L.mars_kv_copy_pages(a_cache(C), None, P, 1, None) == ARG
    assert L.mars_kv_copy_pages(a_cache(C), P, P, 0, None) == ARG
    assert L.mars_kv_reserve_workspace_bytes(0, 1) == 0 and L.mars_kv_reserve_workspace_bytes(1, 0) == 0


def test_the_binding_refuses(C):
    """Wrong shapes, types, layouts, and tensors that are not on the GPU."""
    import torch
    kv = C.KVCache(2, 9, 4, 128, 16, 3, 80, device="cpu")
    assert kv.pool.shape == (2, 9, 4, 16 * 136) and kv.page_table.shape == (3, 5)
    k = torch.zeros((2, 3, 4, 128), dtype=torch.bfloat16)
    append = lambda k, v, lens=kv.lens: C.mars_kv_append(kv.pool, kv.page_table, lens, k, v)  # noqa: E731
    for call in (lambda: append(k, k.float()), lambda: append(k[:, :, :3], k[:, :, :3]), lambda: append(k, k, kv.lens.long()),
                 lambda: append(k.transpose(2, 3), k.transpose(2, 3)), lambda: append(k, k),
                 lambda: C.mars_kv_commit(kv.pool, kv.page_table, kv.lens, kv.lens, torch.zeros((3, 4), dtype=torch.int32), page_size=24),
                 lambda: C.mars_kv_release(kv.page_table, kv.lens, kv.held, kv.refs, kv.lens),
                 lambda: C.mars_tree_mask(torch.zeros((2, 3), dtype=torch.int32))):
        with pytest.raises(AssertionError):
            call()
    q = torch.zeros((2, 3, 6, 128), dtype=torch.bfloat16)
    with pytest.raises(C.MarsError):
        C.alloc_attention_workspace(kv.pool, kv.page_table, q)          # six query heads over four of the cache
    with pytest.raises(TypeError):
        C.alloc_attention_workspace(kv.pool, kv.page_table, q.half())
