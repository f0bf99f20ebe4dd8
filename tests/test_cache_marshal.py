"""The native part of the cache's binding (csrc/cache_marshal.cpp) against its general way through ctypes, on the CPU: the library's functions
are replaced by ones that write down what they are given."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2601_15498_amd import cache as C

PTR = ctypes.c_void_p
NAMES = ("mars_kv_append", "mars_kv_read", "mars_tree_mask", "mars_kv_attention", "mars_kv_commit", "mars_kv_reserve", "mars_kv_fork",
         "mars_kv_release")
CALLS = ("append", "read", "tree_mask", "attention", "commit", "reserve", "fork", "release")
STRUCTS = {"mars_kv_append": {0: C.CacheStruct, 3: C.RowsStruct, 4: C.RowsStruct}, "mars_kv_read": {0: C.CacheStruct, 4: C.RowsStruct, 5: C.RowsStruct},
           "mars_tree_mask": {}, "mars_kv_attention": {0: C.CacheStruct, 3: C.RowsStruct, 10: C.RowsStruct},
           **{n: {0: C.CacheStruct} for n in NAMES[4:]}}


@pytest.fixture
def recorder(monkeypatch):
    real, native = C.lib(), C._calls()
    if native is C._NoNative:
        pytest.skip("the native part was not built here")
    got, keep = [], []

    def stub(name):
        types = [PTR if hasattr(t, "contents") else t for t in getattr(real, name).argtypes]

        def run(*args):
            vals = list(args)
            for i, struct in STRUCTS[name].items():
                x = struct.from_address(vals[i])
                vals[i] = tuple(getattr(x, f) for f, _ in struct._fields_)
            got.append((name, *vals))
            return 0
        keep.append(ctypes.CFUNCTYPE(ctypes.c_int, *types)(run))
        return keep[-1]

    stubs = {n: stub(n) for n in NAMES}
    native.bind(*(ctypes.cast(stubs[n], PTR).value for n in NAMES), False)
    general = {n: (lambda c: lambda *a: c(*[ctypes.cast(ctypes.byref(x), PTR) if isinstance(x, ctypes.Structure) else x for x in a]))(stubs[n]) for n in NAMES}
    monkeypatch.setattr(C, "_stream", lambda: 0x7F)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)       # the general way's own question
    yield got, native, SimpleNamespace(**general)
    native.bind(*(ctypes.cast(getattr(real, n), PTR).value for n in NAMES), True)


def tensors(D=128, P=16, B=2, N=3, dtype=torch.bfloat16):
    S, W, pages, heads = 4, 5, 9, 2
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    qkv = torch.zeros((B, N, 8, D)).to(dtype)
    return SimpleNamespace(pool=torch.zeros((3, pages, heads, P * (D + D // 16)), dtype=torch.uint8), table=i32(S, W), lens=i32(S), held=i32(S), refs=i32(pages),
                           k=qkv[:, :, 4:6], v=qkv[:, :, 6:], q=qkv[:, :, :4], out=torch.zeros((B, N, 4, D)).to(dtype), lse=torch.zeros((B, N, 4)),
                           seqs=i32(B), n_new=i32(B), status=i32(B), parent=i32(B, N), mask=torch.zeros((B, N, 1), dtype=torch.int64), accept=i32(B),
                           new=i32(S), ws=torch.zeros(4096, dtype=torch.uint8), P=P, D=D, scale=0.25, layer=2)


def entries(s, some):
    """Every call, with its optional arguments or without."""
    o = lambda x: x if some else None  # noqa: E731
    return {
        "append": lambda: C.mars_kv_append(s.pool, s.table, s.lens, s.k, s.v, layer=s.layer, seqs=o(s.seqs), n_new=o(s.n_new), status=o(s.status)),
        "read": lambda: C.mars_kv_read(s.pool, s.table, o(s.held), layer=s.layer, seqs=o(s.seqs), first=o(s.n_new), out=(s.k, s.v)),
        "tree_mask": lambda: C.mars_tree_mask(s.parent, n_new=o(s.n_new), mask=s.mask, status=o(s.status)),
        "attention": lambda: C.mars_kv_attention(s.pool, s.table, s.lens, s.q, layer=s.layer, seqs=o(s.seqs), n_new=o(s.n_new), mask=o(s.mask),
                                                 scale=o(s.scale), max_len=7 if some else 0, out=s.out, lse=o(s.lse), workspace=s.ws),
        "commit": lambda: C.mars_kv_commit(s.pool, s.table, s.lens, s.accept, s.parent, page_size=s.P, seqs=o(s.seqs), new_lens=o(s.new), status=o(s.status)),
        "reserve": lambda: C.mars_kv_reserve(s.pool, s.table, s.lens, s.held, s.refs, s.n_new if some else 60, page_size=s.P, seqs=s.seqs, status=s.status,
                                             workspace=s.ws),
        "fork": lambda: C.mars_kv_fork(s.table, s.lens, s.held, s.refs, s.seqs, s.accept, page_size=s.P, status=o(s.status)),
        "release": lambda: C.mars_kv_release(s.table, s.lens, s.held, s.refs, s.seqs, status=o(s.status)),
    }


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("some", [True, False])
@pytest.mark.parametrize("form", [dict(), dict(D=64, P=8, dtype=torch.float32), dict(D=256, P=256, dtype=torch.int16)])
def test_a_regular_call_hands_over_the_same_either_way(recorder, monkeypatch, call, some, form):
    got, native, general = recorder
    s = tensors(**form)
    run = entries(s, some)[call]
    run()
    assert len(got) == 1
    monkeypatch.setattr(C, "_lib", general)
    monkeypatch.setattr(C, "_native", C._NoNative)
    run()
    assert len(got) == 2 and got[0] == got[1]


class Sub(torch.Tensor):
    pass


IRREGULAR = {
    "a subclass": ("lens", lambda t: t.as_subclass(Sub)), "another type": ("lens", lambda t: t.long()), "another length": ("lens", lambda t: t[:-1]),
    "not contiguous": ("lens", lambda t: torch.zeros((4, 2), dtype=torch.int32)[:, 0]), "nothing": ("lens", lambda t: None),
    "a table of another rank": ("table", lambda t: t[0]), "a table of another type": ("table", lambda t: t.short()),
}
PER_CALL = {
    "append": [("k", lambda t: t.transpose(2, 3)), ("k", lambda t: t.double()), ("v", lambda t: t[:, 1:]), ("v", lambda t: t.float()), ("pool", lambda t: t[:, :, :, :-1]),
               ("pool", lambda t: t[:, ::2]), ("layer", lambda x: 1.0), ("n_new", lambda t: t[:1])],
    "attention": [("q", lambda t: t[:, :, 0]), ("out", lambda t: t.float()), ("out", lambda t: t[:, :, :2]), ("lse", lambda t: t.double()), ("mask", lambda t: t[:, :2]),
                  ("mask", lambda t: t.int()), ("scale", lambda x: 1), ("ws", lambda t: t[::2]), ("ws", lambda t: None)],
    "commit": [("accept", lambda t: t.long()), ("accept", lambda t: None), ("parent", lambda t: t[:, ::2]), ("new", lambda t: t[:2])],
    "reserve": [("refs", lambda t: t[:3]), ("held", lambda t: t.long()), ("status", lambda t: None), ("ws", lambda t: t.int()), ("n_new", lambda t: t.float())],
}


def test_a_call_that_is_not_regular_is_left_alone(recorder, monkeypatch):
    got, native, _ = recorder
    monkeypatch.setattr(C, "_check", lambda rc: None)
    general = []
    monkeypatch.setattr(C, "_native", SimpleNamespace(**{c: (lambda f: lambda *a: general.append(f(*a)) or 0)(getattr(native, c)) for c in CALLS}))
    cases = [(c, f) for c in ("append", "attention", "commit", "reserve", "fork", "release") for f in IRREGULAR.values()]
    cases += [(c, f) for c, fs in PER_CALL.items() for f in fs]
    for call, (name, change) in cases:
        s = tensors()
        setattr(s, name, change(getattr(s, name)))
        entries(s, True)[call]()
        assert general.pop() is None and not got, (call, name)
    assert all(getattr(native, c)(1) is None for c in CALLS) and not got


def test_tensors_that_are_not_on_the_gpu_are_left_to_the_general_way():
    if C._calls() is C._NoNative:
        pytest.skip("the native part was not built here")
    s = tensors()
    for call in CALLS:
        with pytest.raises(AssertionError):
            entries(s, True)[call]()
