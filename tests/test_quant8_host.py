"""Host-side checks of the entry points of the operators in 8-bit floats (no GPU
needed): every call here fails validation, or has nothing to do, before any launch."""
import ctypes

import pytest
import torch

from paper_1907_02154_amd import miconv, quant
from test_quant_host import FAKE, NAN, call, placed


@pytest.fixture(scope="module")
def L():
    return quant.lib()


def cache8(pages=4, heads=2, page_size=16, head_dim=64, block=16, kc=FAKE, ke=FAKE, vc=FAKE, ve=FAKE):
    return quant._Kv8(kc, ke, vc, ve, pages, heads, page_size, head_dim, block)


def test_f8_declared_and_exported(L):
    names = miconv.header_functions()
    for n in ("quant_rmsnorm_f8", "quant_rows_f8", "quant_matmul_f8", "quant_matmul_f8_workspace_bytes", "quant_matmul_f8_describe",
              "quant_kv8_write", "quant_kv8_read", "quant_attention_kv8", "quant_attention_kv8_workspace_bytes",
              "quant_attention_kv8_describe"):
        assert n in names and hasattr(L, n), n
    assert ctypes.sizeof(quant._Kv8) == 56 and quant._Kv8.block.offset == 52


def test_rmsnorm_f8_refusals(L):
    d = [("rows", 2), ("cols", 200), ("dtype", 1), ("x", FAKE), ("xs", 200), ("res", FAKE), ("rs", 200), ("w", FAKE),
         ("eps", 1e-6), ("h", FAKE), ("hs", 200), ("q", FAKE), ("qs", 200), ("e", FAKE), ("es", 2), ("scale", FAKE), ("st", None)]
    f = lambda **k: call(L.quant_rmsnorm_f8, d, **k)  # noqa: E731
    for k in (dict(rows=-1), dict(cols=0), dict(xs=199), dict(rs=199), dict(hs=199), dict(qs=199), dict(es=1), dict(eps=-1.0),
              dict(eps=NAN)):
        assert f(**k) == miconv.ERR_SHAPE, k
    for k in (dict(x=None), dict(q=None), dict(e=None), dict(scale=None), dict(h=None), dict(res=None)):
        assert f(**k) == miconv.ERR_NULL, k
    for k in (dict(x=FAKE + 1), dict(res=FAKE + 1), dict(h=FAKE + 1), dict(w=FAKE + 2), dict(scale=FAKE + 2), dict(dtype=0, x=FAKE + 2)):
        assert f(**k) == miconv.ERR_ALIGN, k
    assert f(dtype=2) == miconv.ERR_UNSUPPORTED
    assert f(rows=1 << 31) == miconv.ERR_TOO_LARGE
    big = 1 << 31
    assert f(cols=big, xs=big, rs=big, hs=big, qs=big, es=big) == miconv.ERR_TOO_LARGE
    assert f(rows=0, x=None, q=None, e=None, scale=None) == miconv.OK
    d = [d[i] for i in (0, 1, 2, 3, 4, 11, 12, 13, 14, 16)]
    f = lambda **k: call(L.quant_rows_f8, d, **k)  # noqa: E731
    assert f(x=None) == f(q=None) == f(e=None) == miconv.ERR_NULL
    assert f(cols=0) == f(xs=4) == f(qs=4) == f(es=1) == miconv.ERR_SHAPE
    assert f(dtype=3) == miconv.ERR_UNSUPPORTED and f(rows=0) == miconv.OK


def test_matmul_f8_refusals(L):
    d = [("M", 4), ("N", 8), ("K", 144), ("a", FAKE), ("as", 144), ("ea", FAKE), ("eas", 2), ("sa", None), ("w", FAKE), ("ws_", 144),
         ("ew", FAKE), ("ews", 2), ("bias", None), ("res", None), ("rs", 0), ("dtype", 1), ("y", FAKE), ("ys", 8), ("relu", 0),
         ("ws", None), ("wsb", 0), ("st", None)]
    f = lambda **k: call(L.quant_matmul_f8, d, **k)  # noqa: E731
    for k in (dict(M=-1), dict(N=0), dict(K=0), {"as": 143}, dict(ws_=143), dict(ys=7), dict(res=FAKE, rs=7), dict(eas=1), dict(ews=1)):
        assert f(**k) == miconv.ERR_SHAPE, k
    for n in ("a", "ea", "w", "ew", "y"):
        assert f(**{n: None}) == miconv.ERR_NULL, n
    for k in (dict(sa=FAKE + 2), dict(bias=FAKE + 2), dict(res=FAKE + 1, rs=8), dict(y=FAKE + 1), dict(dtype=0, y=FAKE + 2)):
        assert f(**k) == miconv.ERR_ALIGN, k
    assert f(dtype=7) == miconv.ERR_UNSUPPORTED
    far = 1 << 23
    assert f(K=far, eas=far, ews=far, **{"as": far, "ws_": far}) == miconv.ERR_TOO_LARGE
    assert f(M=1 << 31) == f(N=(1 << 31) - 255, ys=1 << 31) == miconv.ERR_TOO_LARGE
    assert f(M=0, a=None, y=None) == miconv.OK
    w = lambda M, N, K, a=FAKE, sa=None, p=FAKE, sw=None: L.quant_matmul_f8_workspace_bytes(  # noqa: E731
        M, N, K, a, K if sa is None else sa, p, K if sw is None else sw)
    assert w(-1, 8, 16) == w(4, 0, 16) == w(4, 8, 0) == w(4, 8, 16, sa=15) == w(4, 8, 16, sw=0) == miconv.ERR_SHAPE
    assert w(0, 8, 17) == w(4, 8, 16) == w(4, 8, 32, sa=48) == 0
    assert w(4, 8, 17) == 2 * 256 and w(4, 8, 16, a=FAKE + 1) == w(4, 8, 16, sw=17) == w(4, 8, 16, sa=far) == 256
    for k in (dict(ws=None), dict(wsb=255), dict(ws=FAKE + 16)):
        assert f(**{"a": FAKE + 1, "ws": FAKE, "wsb": 1024, **k}) == miconv.ERR_WORKSPACE, k


@pytest.mark.parametrize("write", [True, False])
def test_cache8_refusals(L, write):
    if write:
        d = [("c", cache8()), ("seqs", 3), ("tokens", 3), ("dtype", 1), ("k", FAKE), ("ks", 128), ("v", FAKE), ("vs", 128),
             ("starts", None), ("lens", FAKE), ("table", FAKE), ("ts", 2), ("max_new", 1), ("st", None)]
        f = lambda **k: call(L.quant_kv8_write, d, **k)  # noqa: E731
        assert f(lens=None) == f(table=None) == miconv.ERR_NULL
        assert f(seqs=-1) == f(ts=0) == f(max_new=0) == miconv.ERR_SHAPE
        assert f(starts=FAKE + 2) == f(lens=FAKE + 1) == f(table=FAKE + 2) == miconv.ERR_ALIGN
        assert f(seqs=65536) == f(c=cache8(block=1), max_new=(1 << 31) - 1) == miconv.ERR_TOO_LARGE
        assert f(seqs=0, k=None) == miconv.OK
    else:
        d = [("c", cache8()), ("tokens", 3), ("slots", FAKE), ("dtype", 1), ("k", FAKE), ("ks", 128), ("v", FAKE), ("vs", 128),
             ("st", None)]
        f = lambda **k: call(L.quant_kv8_read, d, **k)  # noqa: E731
        assert f(slots=None) == miconv.ERR_NULL and f(slots=FAKE + 2) == miconv.ERR_ALIGN
    assert f(c=None) == f(k=None) == f(v=None) == miconv.ERR_NULL
    for n in ("kc", "ke", "vc", "ve"):
        assert f(c=cache8(**{n: None})) == miconv.ERR_NULL, n
    for k in (dict(tokens=-1), dict(ks=127), dict(vs=127), dict(c=cache8(pages=0)), dict(c=cache8(heads=0)), dict(c=cache8(page_size=0)),
              dict(c=cache8(block=0)), dict(c=cache8(block=5)), dict(c=cache8(block=32))):
        assert f(**k) == miconv.ERR_SHAPE, k
    for D in (0, 16, 48, 160, 512):
        assert f(c=cache8(head_dim=D)) == miconv.ERR_UNSUPPORTED, D
    assert f(dtype=2) == f(c=cache8(page_size=514, block=257)) == miconv.ERR_UNSUPPORTED
    assert f(c=cache8(kc=FAKE + 8)) == f(c=cache8(vc=FAKE + 4)) == f(k=FAKE + 1) == miconv.ERR_ALIGN
    assert f(c=cache8(pages=1 << 20, page_size=1 << 11)) == f(tokens=1 << 31) == miconv.ERR_TOO_LARGE
    assert f(c=cache8(pages=1, heads=16, page_size=1 << 28)) == miconv.ERR_TOO_LARGE
    assert f(tokens=0, k=None, v=None) == miconv.OK


def test_attention8_refusals_and_plans(L):
    big = 1 << 30
    d = [("c", cache8()), ("seqs", 2), ("heads", 4), ("tokens", 2), ("q", FAKE), ("qs", 256), ("starts", None),
         ("lens", FAKE), ("table", FAKE), ("ts", 3), ("max_new", 1), ("max_len", 48), ("scale", 1.0), ("causal", 1),
         ("window", 0), ("out", FAKE), ("os", 256), ("ws", FAKE), ("wsb", big), ("st", None)]
    f = lambda **k: call(L.quant_attention_kv8, d, **k)  # noqa: E731
    for n in ("c", "q", "lens", "table", "out"):
        assert f(**{n: None}) == miconv.ERR_NULL, n
    for k in (dict(seqs=-1), dict(heads=3), dict(heads=0), dict(tokens=-1), dict(qs=255), dict(os=255), dict(ts=0),
              dict(max_new=0), dict(max_len=0), dict(scale=NAN), dict(scale=3e38), dict(c=cache8(block=3))):
        assert f(**k) == miconv.ERR_SHAPE, k
    for k in (dict(q=FAKE + 1), dict(out=FAKE + 1), dict(starts=FAKE + 2), dict(lens=FAKE + 2), dict(table=FAKE + 1)):
        assert f(**k) == miconv.ERR_ALIGN, k
    assert f(c=cache8(head_dim=48), qs=192, os=192) == miconv.ERR_UNSUPPORTED
    assert f(seqs=70000) == f(max_new=1 << 30) == f(max_len=1 << 30) == f(tokens=1 << 31) == miconv.ERR_TOO_LARGE
    assert f(seqs=0) == f(tokens=0) == miconv.OK
    need = L.quant_attention_kv8_workspace_bytes(cache8(pages=4096, page_size=64), 1, 4, 1, 65536, 1, 0)
    assert need > 0
    for k in (dict(wsb=need - 1), dict(ws=None), dict(ws=FAKE + 16)):
        assert f(c=cache8(pages=4096, page_size=64), seqs=1, tokens=1, ts=1024, max_len=65536, **k) == miconv.ERR_WORKSPACE
    from paper_1907_02154_amd import traffic
    seen = set()
    buf, n = ctypes.create_string_buffer(256), ctypes.c_int()
    for D in quant.HEAD_DIMS:
        for rows in (1, 16, 17, 32, 33, 64, 65, 5000):
            for max_len in (100, 100000):
                rc = L.quant_attention_kv8_describe(cache8(pages=9999, head_dim=D), 1, 2, rows, max_len, 1, 0, buf, 256, ctypes.byref(n))
                names = buf.value.decode().split(" + ")
                assert rc == miconv.OK and n.value == len(names)
                seen |= set(names)
    assert len(seen) == 6 + 4 + 2 + 6 + 6 and all(k.split("<")[0] in traffic.SOURCES for k in seen)
    seen = set()
    for M, N in ((1, 16), (1, 8193), (33, 5441), (897, 513), (65, 5441), (129, 6529), (129, 10881), (257, 13057), (769, 14081)):
        for dtype in (torch.float32, torch.bfloat16):
            name, n = quant.matmul_f8_describe(M, N, 64, dtype)
            assert n == 1 and quant.matmul_f8_describe(M, N, 63, dtype) == ("matmul_i8_align_kernel + " + name, 2)
            seen.add(name)
    assert all(k.split("<")[0] in traffic.SOURCES for k in seen)


def test_f8_binding_refuses_operands_on_another_device(monkeypatch):
    """Each operand in turn on GPU 1 where GPU 0 is the current one: a ValueError, and no call."""
    monkeypatch.setattr(quant, "_getdevice", lambda: 0)

    class Called(Exception):
        pass

    class Library:
        def __getattr__(self, name):
            if name.endswith("_workspace_bytes"):
                return lambda *a: 256
            raise Called(name)
    monkeypatch.setattr(quant, "lib", Library)
    f32, i32, u8, bf, f8 = torch.float32, torch.int32, torch.uint8, torch.bfloat16, quant.F8

    def kv(at):
        return quant.KV8Cache(*(placed(at, 2, 2, 16, *([64] if d is f8 else []), dtype=d) if d is f8 else placed(at, 2, 2, 2, dtype=d)
                                for d in (f8, u8, f8, u8)))

    calls = {
        "norm": (lambda x, w, r, h, q, e, s: quant.rmsnorm_f8(x, w, r, h=h, q=q, exps=e, scale=s, stream=0),
                 [((4, 64), bf), ((64,), f32), ((4, 64), bf), ((4, 64), bf), ((4, 64), f8), ((4, 1), u8), ((4,), f32)]),
        "rows": (lambda x, q, e: quant.rows_f8(x, q=q, exps=e, stream=0), [((4, 64), bf), ((4, 64), f8), ((4, 1), u8)]),
        "product": (lambda a, ea, w, ew, sa, b, r, o: quant.matmul_f8(a, ea, w, ew, a_scale=sa, bias=b, residual=r, out=o, stream=0),
                    [((4, 64), f8), ((4, 1), u8), ((8, 64), f8), ((8, 1), u8), ((4,), f32), ((8,), f32), ((4, 8), bf), ((4, 8), bf)]),
        "write": (lambda k, v, t, n, s, c: quant.kv8_write(k, v, c, t, n, starts=s, stream=0),
                  [((3, 2, 64), bf), ((3, 2, 64), bf), ((2, 2), i32), ((2,), i32), ((3,), i32), kv]),
        "read": (lambda s, k, v, c: quant.kv8_read(s, c, k=k, v=v, stream=0), [((3,), i32), ((3, 2, 64), bf), ((3, 2, 64), bf), kv]),
        "attend": (lambda q, t, n, s, o, w, c: quant.attention_kv8(q, c, t, n, starts=s, out=o, ws=w, stream=0),
                   [((2, 4, 64), bf), ((2, 2), i32), ((2,), i32), ((3,), i32), ((2, 4, 64), bf), ((512,), u8), kv]),
    }
    for name, (f, kinds) in calls.items():
        make = lambda at: [k(d) if callable(k) else placed(d, *k[0], dtype=k[1]) for k, d in zip(kinds, at)]  # noqa: E731
        if name != "attend":   # its workspace's address is the host allocator's
            with pytest.raises(Called):
                f(*make([0] * len(kinds)))
        for i in range(len(kinds)):
            with pytest.raises(ValueError, match="device"):
                f(*make([int(i == j) for j in range(len(kinds))]))
    assert kv(1).device == 1 and kv(0).block == 8


def test_f8_binding_refuses_numbers_of_more_than_32_bits(monkeypatch):
    monkeypatch.setattr(quant, "_getdevice", lambda: 0)
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0
    monkeypatch.setattr(quant, "lib", Library)
    f8, u8 = quant.F8, torch.uint8
    c = quant.KV8Cache(placed(0, 2, 2, 16, 64, dtype=f8), placed(0, 2, 2, 1, dtype=u8), placed(0, 2, 2, 16, 64, dtype=f8),
                       placed(0, 2, 2, 1, dtype=u8))
    q, o = (placed(0, 2, 4, 64, dtype=torch.bfloat16) for _ in range(2))
    kv = placed(0, 2, 2, 64, dtype=torch.bfloat16)
    t, n = placed(0, 2, 2, dtype=torch.int32), placed(0, 2, dtype=torch.int32)
    for v in (1 << 31, (1 << 32) + 5, -(1 << 31) - 1):
        for k in ("max_new", "max_len", "window"):
            with pytest.raises(ValueError, match=k):
                quant.attention_kv8(q, c, t, n, out=o, stream=0, **{k: v})
            with pytest.raises(ValueError, match=k):
                quant.attention_kv8_workspace_bytes(c, 2, 4, **{"max_new": 1, "max_len": 32, k: v})
        with pytest.raises(ValueError, match="max_new"):
            quant.kv8_write(kv, kv, c, t, n, max_new=v, stream=0)
    assert not calls
    with pytest.raises(TypeError, match="KV8Cache"):
        quant.attention_kv8(q, None, t, n, out=o, stream=0)
    with pytest.raises(ValueError, match="device"):
        quant.rows_f8(torch.zeros(2, 8))
    with pytest.raises(ValueError, match="block"):
        quant.KV8Cache.allocate(1, 1, 16, 64, 5)
