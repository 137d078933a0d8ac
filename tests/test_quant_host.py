"""Host-side checks of the quantised operators' entry points (no GPU needed):
every call here fails validation, or has nothing to do, before any launch."""
import ctypes

import pytest
import torch

from paper_1907_02154_amd import miconv, quant

FAKE = 4096   # aligned, non-null, never touched
NAN = float("nan")


@pytest.fixture(scope="module")
def L():
    return quant.lib()


def cache(pages=4, heads=2, page_size=16, head_dim=64, kc=FAKE, ke=FAKE, vc=FAKE, ve=FAKE):
    return quant._Kv4(kc, ke, vc, ve, pages, heads, page_size, head_dim)


def call(f, defaults, **k):
    assert set(k) <= set(dict(defaults)), k
    return f(*[k.get(n, d) for n, d in defaults])


def test_declared_and_exported(L):
    names = miconv.header_functions()
    for n in ("quant_rmsnorm_i8", "quant_rows_i8", "quant_matmul_i8", "quant_matmul_workspace_bytes", "quant_kv4_write",
              "quant_kv4_read", "quant_attention_kv4", "quant_attention_workspace_bytes"):
        assert n in names and hasattr(L, n), n


def test_rmsnorm_refusals(L):
    d = [("rows", 2), ("cols", 8), ("dtype", 1), ("x", FAKE), ("xs", 8), ("res", FAKE), ("rs", 8), ("w", FAKE),
         ("eps", 1e-6), ("h", FAKE), ("hs", 8), ("q", FAKE), ("qs", 8), ("scale", FAKE), ("st", None)]
    f = lambda **k: call(L.quant_rmsnorm_i8, d, **k)  # noqa: E731
    for k in (dict(rows=-1), dict(cols=0), dict(xs=7), dict(rs=7), dict(hs=7), dict(qs=7), dict(eps=-1.0), dict(eps=NAN)):
        assert f(**k) == miconv.ERR_SHAPE, k
    for k in (dict(x=None), dict(q=None), dict(scale=None), dict(h=None), dict(res=None)):
        assert f(**k) == miconv.ERR_NULL, k
    for k in (dict(x=FAKE + 1), dict(res=FAKE + 1), dict(h=FAKE + 1), dict(w=FAKE + 2), dict(scale=FAKE + 2),
              dict(dtype=0, x=FAKE + 2)):
        assert f(**k) == miconv.ERR_ALIGN, k
    assert f(dtype=2) == miconv.ERR_UNSUPPORTED
    assert f(rows=1 << 31) == miconv.ERR_TOO_LARGE
    assert f(cols=1 << 31, xs=1 << 31, rs=1 << 31, hs=1 << 31, qs=1 << 31) == miconv.ERR_TOO_LARGE
    assert f(rows=0, x=None, q=None, scale=None) == miconv.OK


def test_rows_refusals(L):
    d = [("rows", 2), ("cols", 8), ("dtype", 1), ("x", FAKE), ("xs", 8), ("q", FAKE), ("qs", 8), ("scale", FAKE), ("st", None)]
    f = lambda **k: call(L.quant_rows_i8, d, **k)  # noqa: E731
    assert f(x=None) == f(q=None) == f(scale=None) == miconv.ERR_NULL
    assert f(cols=0) == f(xs=4) == f(qs=4) == miconv.ERR_SHAPE
    assert f(dtype=3) == miconv.ERR_UNSUPPORTED
    assert f(rows=0) == miconv.OK


def test_matmul_refusals(L):
    d = [("M", 4), ("N", 8), ("K", 16), ("a", FAKE), ("as", 16), ("sa", FAKE), ("w", FAKE), ("ws_", 16), ("sw", FAKE),
         ("bias", None), ("res", None), ("rs", 0), ("dtype", 1), ("y", FAKE), ("ys", 8), ("relu", 0), ("ws", None),
         ("wsb", 0), ("st", None)]
    f = lambda **k: call(L.quant_matmul_i8, d, **k)  # noqa: E731
    for k in (dict(M=-1), dict(N=0), dict(K=0), {"as": 15}, dict(ws_=15), dict(ys=7), dict(res=FAKE, rs=7)):
        assert f(**k) == miconv.ERR_SHAPE, k
    for n in ("a", "sa", "w", "sw", "y"):
        assert f(**{n: None}) == miconv.ERR_NULL, n
    for k in (dict(sa=FAKE + 2), dict(sw=FAKE + 1), dict(bias=FAKE + 2), dict(res=FAKE + 1, rs=8), dict(y=FAKE + 1),
              dict(dtype=0, y=FAKE + 2)):
        assert f(**k) == miconv.ERR_ALIGN, k
    assert f(dtype=7) == miconv.ERR_UNSUPPORTED
    assert f(K=131072, **{"as": 131072, "ws_": 131072}) == miconv.ERR_TOO_LARGE
    assert f(M=1 << 31) == miconv.ERR_TOO_LARGE
    assert f(M=0, a=None, y=None) == miconv.OK
    w = lambda M, N, K, a=FAKE, sa=None, p=FAKE, sw=None: L.quant_matmul_workspace_bytes(  # noqa: E731
        M, N, K, a, K if sa is None else sa, p, K if sw is None else sw)
    assert w(-1, 8, 16) == w(4, 0, 16) == w(4, 8, 0) == w(4, 8, 16, sa=15) == w(4, 8, 16, sw=0) == miconv.ERR_SHAPE
    assert w(4, 8, 131072) == miconv.ERR_TOO_LARGE
    assert w(0, 8, 17) == w(4, 8, 16) == w(4, 8, 32, sa=48) == 0      # rows that can be read as they are
    assert w(4, 8, 17) == 2 * 256                                     # both copied: 4 and 8 rows of 32 bytes
    assert w(4, 8, 16, a=FAKE + 1) == w(4, 8, 16, sw=17) == 256       # one of them
    for k in (dict(ws=None), dict(wsb=255), dict(ws=FAKE + 16)):
        assert f(**{"a": FAKE + 1, "ws": FAKE, "wsb": 256, **k}) == miconv.ERR_WORKSPACE, k


@pytest.mark.parametrize("write", [True, False])
def test_cache_refusals(L, write):
    d = [("c", cache()), ("tokens", 3), ("dtype", 1), ("k", FAKE), ("ks", 128), ("v", FAKE), ("vs", 128), ("slots", FAKE),
         ("st", None)]
    if not write:
        d = d[:2] + [d[7], d[2]] + d[3:7] + d[8:]
    f = lambda **k: call(L.quant_kv4_write if write else L.quant_kv4_read, d, **k)  # noqa: E731
    assert f(c=None) == f(k=None) == f(v=None) == f(slots=None) == miconv.ERR_NULL
    for n in ("kc", "ke", "vc", "ve"):
        assert f(c=cache(**{n: None})) == miconv.ERR_NULL, n
    for k in (dict(tokens=-1), dict(ks=127), dict(vs=127), dict(c=cache(pages=0)), dict(c=cache(heads=0)),
              dict(c=cache(page_size=0))):
        assert f(**k) == miconv.ERR_SHAPE, k
    for D in (0, 16, 48, 160, 512):
        assert f(c=cache(head_dim=D)) == miconv.ERR_UNSUPPORTED, D
    assert f(dtype=2) == miconv.ERR_UNSUPPORTED
    assert f(c=cache(kc=FAKE + 8)) == f(c=cache(vc=FAKE + 4)) == f(k=FAKE + 1) == f(slots=FAKE + 2) == miconv.ERR_ALIGN
    assert f(c=cache(pages=1 << 20, page_size=1 << 11)) == miconv.ERR_TOO_LARGE
    assert f(tokens=1 << 31) == miconv.ERR_TOO_LARGE
    assert f(tokens=0, k=None, v=None, slots=None) == miconv.OK


def test_attention_refusals(L):
    big = 1 << 30
    d = [("c", cache()), ("seqs", 2), ("heads", 4), ("tokens", 2), ("q", FAKE), ("qs", 256), ("starts", None),
         ("lens", FAKE), ("table", FAKE), ("ts", 3), ("max_new", 1), ("max_len", 48), ("scale", 1.0), ("causal", 1),
         ("window", 0), ("out", FAKE), ("os", 256), ("ws", FAKE), ("wsb", big), ("st", None)]
    f = lambda **k: call(L.quant_attention_kv4, d, **k)  # noqa: E731
    for n in ("c", "q", "lens", "table", "out"):
        assert f(**{n: None}) == miconv.ERR_NULL, n
    for k in (dict(seqs=-1), dict(heads=3), dict(heads=0), dict(tokens=-1), dict(qs=255), dict(os=255), dict(ts=0),
              dict(max_new=0), dict(max_len=0)):
        assert f(**k) == miconv.ERR_SHAPE, k
    for k in (dict(q=FAKE + 1), dict(out=FAKE + 1), dict(starts=FAKE + 2), dict(lens=FAKE + 2), dict(table=FAKE + 1)):
        assert f(**k) == miconv.ERR_ALIGN, k
    assert f(c=cache(head_dim=48), qs=192, os=192) == miconv.ERR_UNSUPPORTED
    assert f(seqs=70000) == f(max_new=1 << 30) == f(max_len=1 << 30) == f(tokens=1 << 31) == miconv.ERR_TOO_LARGE
    assert f(seqs=0) == f(tokens=0) == miconv.OK
    w = L.quant_attention_workspace_bytes
    c = cache(pages=4096, page_size=64)
    assert w(c, 1, 4, 1, 16, 1, 0) == 0                 # one split: nothing to join
    need = w(c, 1, 4, 1, 65536, 1, 0)
    assert need > 0                                     # one sequence, many places: split over the work-groups
    assert f(c=c, seqs=1, tokens=1, ts=1024, max_len=65536, wsb=need - 1) == miconv.ERR_WORKSPACE
    assert f(c=c, seqs=1, tokens=1, ts=1024, max_len=65536, ws=None) == miconv.ERR_WORKSPACE
    assert f(c=c, seqs=1, tokens=1, ts=1024, max_len=65536, ws=FAKE + 16) == miconv.ERR_WORKSPACE
    assert w(c, 1, 4, 1, 65536, 1, 100) == 0            # a short window: nothing to split
    assert w(c, 1, 4, 1, 65536, 0, 100) == need         # which bounds nothing ahead of the query
    assert w(None, 1, 4, 1, 16, 1, 0) == miconv.ERR_NULL
    assert w(c, 1, 3, 1, 16, 1, 0) == miconv.ERR_SHAPE


def test_matmul_refuses_rows_that_a_tile_numbers_past_32_bits(L):
    """The last tile's rows that are not there have numbers too: 255 of them at most."""
    w = L.quant_matmul_workspace_bytes
    most = (1 << 31) - 256
    assert w(most, 1, 16, FAKE, 16, FAKE, 16) == w(1, most, 16, FAKE, 16, FAKE, 16) == 0
    for M, N in ((most + 1, 1), (1, most + 1), ((1 << 31) - 1, 8)):
        assert w(M, N, 16, FAKE, 16, FAKE, 16) == miconv.ERR_TOO_LARGE
        assert L.quant_matmul_i8(M, N, 16, FAKE, 16, FAKE, FAKE, 16, FAKE, None, None, 0, 1, FAKE, N, 0, None, 0,
                                 None) == miconv.ERR_TOO_LARGE


def test_matmul_workspace_of_rows_far_apart(L, monkeypatch):
    """Aligned rows 2^23 bytes apart are copied: the query says so, and the binding brings the workspace."""
    w = L.quant_matmul_workspace_bytes
    far = 1 << 23
    assert w(4, 8, 16, FAKE, far - 16, FAKE, far - 16) == 0
    assert w(4, 8, 16, FAKE, far, FAKE, 16) == w(4, 8, 16, FAKE, 16, FAKE, far) == 256 and w(4, 8, 16, FAKE, far, FAKE, far) == 512
    given = []

    class Library:
        quant_matmul_workspace_bytes = staticmethod(w)

        def quant_matmul_i8(self, *a):
            given.append(a[-2])
            return 0
    monkeypatch.setattr(quant, "_getdevice", lambda: 0)
    monkeypatch.setattr(quant, "lib", Library)
    i8, f32 = torch.int8, torch.float32
    for sa, sw in ((far, 16), (16, far), (far, far), (16, 16)):
        a, b = (placed(0, r, st, dtype=i8)[:, :16] for r, st in ((4, sa), (8, sw)))
        a.at = b.at = 0
        ws = placed(0, 1024, dtype=torch.uint8)
        ws.data_ptr = lambda: FAKE                  # the host allocator aligns to 64 bytes only
        quant.matmul_i8(a, placed(0, 4, dtype=f32), b, placed(0, 8, dtype=f32), out=placed(0, 4, 8, dtype=f32), ws=ws, stream=0)
        assert (given[-1] >= w(4, 8, 16, a.data_ptr(), sa, b.data_ptr(), sw)) and (given[-1] > 0) == (max(sa, sw) >= far)


def test_described_kernels(L):
    """Every kernel of the product and of attention is reached by some shape, under the name of its source."""
    from paper_1907_02154_amd import traffic
    seen = set()
    for M, N in ((1, 16), (1, 8193), (33, 5441), (897, 513), (65, 5441), (129, 6529), (129, 10881), (257, 13057), (769, 14081)):
        for dtype in (torch.float32, torch.bfloat16):
            name, n = quant.matmul_describe(M, N, 64, dtype)
            assert n == 1 and " + " not in name
            assert quant.matmul_describe(M, N, 63, dtype) == ("matmul_i8_align_kernel + " + name, 2)
            assert quant.matmul_describe(M, N, 64, dtype, w_stride=72) == ("matmul_i8_align_kernel + " + name, 2)
            seen.add(name)
    assert len(seen) == 18
    buf, n = ctypes.create_string_buffer(256), ctypes.c_int()
    for d in quant.HEAD_DIMS:
        for rows in (1, 16, 17, 32, 33, 64, 65, 5000):
            for max_len in (100, 100000):
                rc = L.quant_attention_describe(cache(pages=9999, head_dim=d), 1, 2, rows, max_len, 1, 0, buf, 256, ctypes.byref(n))
                names = buf.value.decode().split(" + ")
                assert rc == miconv.OK and n.value == len(names) == 1 + (
                    L.quant_attention_workspace_bytes(cache(pages=9999, head_dim=d), 1, 2, rows, max_len, 1, 0) > 0)
                seen |= set(names)
    assert len(seen) == 18 + 6 + 4 + 2 + 6 + 6          # few rows by 1, 2 and 4 blocks; many; the joins
    assert all(k.split("<")[0] in traffic.SOURCES for k in seen)
    assert quant.matmul_describe(0, 8, 16) == ("", 0)
    d = lambda *a, dt=0, b=buf, k=256, p=ctypes.byref(n): L.quant_matmul_describe(*a, None, a[2], None, a[2], dt, b, k, p)  # noqa: E731
    assert d(4, 8, 0) == miconv.ERR_SHAPE and d(4, 8, 16, dt=2) == miconv.ERR_UNSUPPORTED and d(4, 8, 131072) == miconv.ERR_TOO_LARGE
    assert d(4, 8, 16, b=None) == d(4, 8, 16, k=0) == d(4, 8, 16, p=None) == miconv.ERR_NULL
    short = ctypes.create_string_buffer(b"x" * 12, 12)
    assert d(4, 8, 16, b=short, k=8) == miconv.OK and short.raw == b"matmul_\0xxxx"
    f = lambda c, *a, b=buf, k=256, p=ctypes.byref(n): L.quant_attention_describe(c, *a, b, k, p)  # noqa: E731
    assert f(None, 1, 2, 1, 8, 1, 0) == f(cache(), 1, 2, 1, 8, 1, 0, b=None) == f(cache(), 1, 2, 1, 8, 1, 0, p=None) == miconv.ERR_NULL
    assert f(cache(), 1, 3, 1, 8, 1, 0) == miconv.ERR_SHAPE and f(cache(head_dim=48), 1, 2, 1, 8, 1, 0) == miconv.ERR_UNSUPPORTED
    assert f(cache(), 0, 2, 1, 8, 1, 0) == miconv.OK and buf.value == b"" and n.value == 0


@pytest.mark.parametrize("scale", [NAN, float("inf"), -float("inf"), 3e38, -3e38])
def test_attention_refuses_scales_that_are_not_finite(L, scale):
    assert L.quant_attention_kv4(cache(), 2, 4, 2, FAKE, 256, None, FAKE, FAKE, 3, 1, 48, scale, 1, 0, FAKE, 256, None, 0,
                                 None) == miconv.ERR_SHAPE


def test_attention_refuses_pages_of_more_rows_than_32_bits_hold(L):
    """heads * page_size >= 2^31: too many for attention's kernels, though the cache's own take them."""
    w = L.quant_attention_workspace_bytes
    assert w(cache(pages=1, heads=8, page_size=(1 << 28) - 1, head_dim=32), 1, 8, 1, 16, 1, 0) == 0
    for heads, page in ((8, 1 << 28), (65535, 1 << 15 | 1), (16, 1 << 28)):
        c = cache(pages=1, heads=heads, page_size=page, head_dim=32)
        assert w(c, 1, heads, 1, 16, 1, 0) == miconv.ERR_TOO_LARGE
        n = heads * 32
        assert L.quant_attention_kv4(c, 1, heads, 1, FAKE, n, None, FAKE, FAKE, 1, 1, 16, 1.0, 1, 0, FAKE, n, None, 0,
                                     None) == miconv.ERR_TOO_LARGE
        assert L.quant_kv4_read(c, 0, FAKE, 1, FAKE, n, FAKE, n, None) == miconv.OK


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("max_new", [1, 12, 300])
def test_attention_plans_of_windows_wider_than_any_length(L, head_dim, max_new):
    """A window that bounds nothing leaves the splits, and so the workspace, as they are without one."""
    c = cache(pages=40, heads=1, head_dim=head_dim)
    for max_len in (300, 2000, 30000):
        want = L.quant_attention_workspace_bytes(c, 2, 4, max_new, max_len, 1, 0)
        for window in (1 << 30, (1 << 31) - 300, (1 << 31) - 80, (1 << 31) - 2, (1 << 31) - 1):
            assert L.quant_attention_workspace_bytes(c, 2, 4, max_new, max_len, 1, window) == want, (max_len, window)


class Placed(torch.Tensor):
    """A host tensor that says it is on GPU `at`: what the binding checks before it passes a pointer on."""
    at = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.at


def placed(at, *shape, dtype):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(Placed)
    t.at = at
    return t


def test_binding_refuses_operands_on_another_device(monkeypatch):
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
    f32, i32, i8, u8, bf = torch.float32, torch.int32, torch.int8, torch.uint8, torch.bfloat16

    def kv(at):
        return quant.KV4Cache(*(placed(at, 2, 2, 16, n, dtype=u8) for n in (32, 2, 32, 2)))

    calls = {
        "norm": (lambda x, w, r, h, q, s: quant.rmsnorm_i8(x, w, r, h=h, q=q, scale=s, stream=0),
                 [((4, 64), bf), ((64,), f32), ((4, 64), bf), ((4, 64), bf), ((4, 64), i8), ((4,), f32)]),
        "rows": (lambda x, q, s: quant.rows_i8(x, q=q, scale=s, stream=0), [((4, 64), bf), ((4, 64), i8), ((4,), f32)]),
        "product": (lambda a, sa, w, sw, b, r, o: quant.matmul_i8(a, sa, w, sw, bias=b, residual=r, out=o, stream=0),
                    [((4, 64), i8), ((4,), f32), ((8, 64), i8), ((8,), f32), ((8,), f32), ((4, 8), bf), ((4, 8), bf)]),
        "write": (lambda k, v, s, c: quant.kv4_write(k, v, s, c, stream=0), [((3, 2, 64), bf), ((3, 2, 64), bf), ((3,), i32), kv]),
        "read": (lambda s, k, v, c: quant.kv4_read(s, c, k=k, v=v, stream=0), [((3,), i32), ((3, 2, 64), bf), ((3, 2, 64), bf), kv]),
        "attend": (lambda q, t, n, s, o, w, c: quant.attention_kv4(q, c, t, n, starts=s, out=o, ws=w, stream=0),
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
    with pytest.raises(ValueError, match="device"):          # a cache on two devices
        quant.KV4Cache(*(placed(int(i == 2), 2, 2, 16, n, dtype=u8) for i, n in enumerate((32, 2, 32, 2))))
    assert kv(1).device == 1                                 # kept on another device than the current one: right until used


def test_binding_refuses_numbers_of_more_than_32_bits(monkeypatch):
    """ctypes takes the low 32 bits of a number: a window of 2^32 + 5 would be one of 5."""
    monkeypatch.setattr(quant, "_getdevice", lambda: 0)
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0
    monkeypatch.setattr(quant, "lib", Library)
    c = quant.KV4Cache(*(placed(0, 2, 2, 16, n, dtype=torch.uint8) for n in (32, 2, 32, 2)))
    q, o = (placed(0, 2, 4, 64, dtype=torch.bfloat16) for _ in range(2))
    t, n = placed(0, 2, 2, dtype=torch.int32), placed(0, 2, dtype=torch.int32)
    for k in ("max_new", "max_len", "window"):
        for v in (1 << 31, (1 << 32) + 5, -(1 << 31) - 1):
            with pytest.raises(ValueError, match=k):
                quant.attention_kv4(q, c, t, n, out=o, stream=0, **{k: v})
            with pytest.raises(ValueError, match=k):
                quant.attention_workspace_bytes(c, 2, 4, **{"max_new": 1, "max_len": 32, k: v})
    assert not calls
    quant.attention_kv4(q, c, t, n, out=o, stream=0, window=(1 << 31) - 1)
    assert calls == ["quant_attention_workspace_bytes", "quant_attention_kv4"]


def test_binding_refuses_host_tensors_and_wrong_types():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="device"):
        quant.rmsnorm_i8(x)
    with pytest.raises(TypeError):
        quant.rows_i8([1.0])
    with pytest.raises(ValueError, match="device"):
        quant.matmul_i8(x.to(torch.int8), x[:, 0], x.to(torch.int8), x[:, 0])
    with pytest.raises(ValueError):
        quant.KV4Cache.allocate(1, 1, 16, 48)
    with pytest.raises(ValueError, match="device"):
        quant.KV4Cache.allocate(1, 1, 16, 64, device="cpu")
    with pytest.raises(TypeError, match="KV4Cache"):
        quant.kv4_read(x, None)
    assert ctypes.sizeof(quant._Kv4) == 56
