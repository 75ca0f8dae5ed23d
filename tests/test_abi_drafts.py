"""Refusals of the entry points of a drafted step and of their Python forms, on
the CPU (nothing reaches the GPU), and the size queries."""
import ctypes
import os

import pytest
import torch

FAKE = ctypes.c_void_p(4096)   # never dereferenced: every call fails validation
ODD = ctypes.c_void_p(4098)
F = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    from paper_2410_19123_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libreadme.so not built")
    return _lib.load()


@pytest.mark.parametrize("bad,status", [
    (dict(rot=0), 2), (dict(rot=24), 2), (dict(rot=528), 2), (dict(rot=-16), 2),
    (dict(scaling=3), 2), (dict(scaling=-1), 2), (dict(theta=0.0), 1), (dict(theta=-1.0), 1),
    (dict(theta=float("inf")), 1), (dict(factor=0.0), 1), (dict(factor=float("nan")), 1),
    (dict(out=None), 1), (dict(scaling=2, trained_len=0.0), 1), (dict(scaling=2, low=2.0, high=2.0), 1),
    (dict(scaling=2, low=float("-inf")), 1), (dict(scaling=2, high=float("nan")), 1),
])
def test_freqs_refuse(lib, bad, status):
    g = dict(rot=32, theta=1e4, scaling=0, factor=1.0, trained_len=64.0, low=1.0, high=32.0,
             out=(ctypes.c_double * 16)())
    g.update(bad)
    assert lib.readme_rotary_freqs(g["rot"], g["theta"], g["scaling"], g["factor"], g["trained_len"],
                                   g["low"], g["high"], g["out"]) == status


def _rotary(lib, **k):
    g = lambda n, d: k.get(n, d)  # noqa: E731
    return lib.readme_rotary(
        g("dt", 1), g("T", 16), g("H", 8), g("D", 128), g("rot", 64), g("layout", 0), g("inverse", 0),
        F(g("amplitude", 1.0)), g("pos", FAKE), g("freqs", FAKE), g("x", FAKE), g("ld_x", 1024),
        g("y", ctypes.c_void_p(1 << 20)), g("ld_y", 1024), None)


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), 1), (dict(H=-1), 1), (dict(dt=2), 2), (dict(H=65536), 2), (dict(D=120), 2),
    (dict(D=528), 2), (dict(D=0), 2), (dict(rot=0), 2), (dict(rot=144), 2), (dict(rot=24), 2),
    (dict(layout=2), 2), (dict(layout=-1), 2), (dict(inverse=2), 1), (dict(inverse=-1), 1),
    (dict(amplitude=float("inf")), 1), (dict(amplitude=float("nan")), 1), (dict(T=(1 << 28) + 1), 2),
    (dict(T=(1 << 26) + 1, D=512, ld_x=4096, ld_y=4096), 2), (dict(pos=None), 1), (dict(freqs=None), 1),
    (dict(x=None), 1), (dict(y=None), 1), (dict(x=ODD), 1), (dict(y=ODD), 1), (dict(pos=ODD), 1),
    (dict(freqs=ctypes.c_void_p(4100)), 1), (dict(ld_x=1016), 1), (dict(ld_y=1020), 1),
    (dict(ld_x=1028), 1), (dict(y=FAKE, ld_y=2048), 1), (dict(dt=0, ld_x=1026), 1),
])
def test_rotary_refuses(lib, bad, status):
    assert _rotary(lib, **bad) == status


def test_rotary_of_nothing(lib):
    none = dict(pos=None, freqs=None, x=None, y=None)
    assert _rotary(lib, T=0, **none) == 0 and _rotary(lib, H=0, **none) == 0
    assert _rotary(lib, T=0, rot=8, **none) == 2


def _append(lib, **k):
    g = lambda n, d: k.get(n, d)  # noqa: E731
    return lib.readme_kv_append(
        g("kt", 0), g("dt", 1), g("T", 16), g("R", 2), g("Hk", 8), g("D", 128), g("rot", 64),
        g("layout", 1), F(g("amplitude", 1.0)), g("pos", None), g("freqs", FAKE), g("k", FAKE),
        g("ld_k", 1024), g("v", FAKE), g("ld_v", 1024), g("offsets", FAKE), g("lens", FAKE),
        g("table", FAKE), g("mb", 4), g("nb", 9), g("codes", FAKE), g("scales", FAKE), None)


CACHE = [
    (dict(T=-1), 1), (dict(R=-1), 1), (dict(R=0), 1), (dict(Hk=0), 1), (dict(mb=0), 1),
    (dict(nb=0), 1), (dict(kt=2), 2), (dict(D=96), 2), (dict(Hk=65536), 2),
    (dict(R=(1 << 22) + 1), 2), (dict(T=(1 << 27) + 1), 2), (dict(mb=1 << 26), 2),
    (dict(nb=1 << 32), 2), (dict(offsets=None), 1), (dict(lens=None), 1), (dict(table=None), 1),
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(codes=ODD), 1), (dict(offsets=ODD), 1),
]


@pytest.mark.parametrize("bad,status", CACHE + [
    (dict(dt=2), 2), (dict(rot=0), 2), (dict(rot=144), 2), (dict(rot=40), 2), (dict(layout=2), 2),
    (dict(amplitude=float("nan")), 1), (dict(freqs=None), 1), (dict(freqs=ctypes.c_void_p(4100)), 1),
    (dict(pos=ODD), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(k=ODD), 1), (dict(ld_k=1016), 1),
    (dict(ld_v=1028), 1),
])
def test_append_refuses(lib, bad, status):
    assert _append(lib, **bad) == status


def test_append_of_nothing(lib):
    none = dict(T=0, R=0, k=None, v=None, offsets=None, lens=None, table=None, codes=None,
                scales=None, freqs=None, mb=0, nb=0)
    assert _append(lib, **none) == 0
    assert _append(lib, **{**none, "rot": 0}) == 2


def _tree(lib, **k):
    g = lambda n, d: k.get(n, d)  # noqa: E731
    return lib.readme_attention_kv_tree(
        g("kt", 0), g("T", 16), g("R", 2), g("H", 16), g("Hk", 8), g("D", 128), g("q", FAKE),
        g("ld_q", 2048), g("offsets", FAKE), g("lens", FAKE), g("table", FAKE), g("mb", 4),
        g("nb", 9), g("codes", FAKE), g("scales", FAKE), g("tree", FAKE), g("words", 1),
        g("pos", None), F(g("scale", 0.1)), g("window", 0), g("o", FAKE), g("ld_o", 2048),
        g("ws", FAKE), g("wsb", 1 << 40), None)


@pytest.mark.parametrize("bad,status", CACHE + [
    (dict(H=15), 1), (dict(H=0), 1), (dict(scale=0.0), 1), (dict(scale=float("nan")), 1),
    (dict(window=-1), 1), (dict(q=None), 1), (dict(o=ODD), 1), (dict(ld_q=2040), 1),
    (dict(ld_o=2052), 1), (dict(ws=None), 1), (dict(wsb=16), 3), (dict(tree=None), 1),
    (dict(tree=ctypes.c_void_p(4100)), 1), (dict(words=0), 1), (dict(words=-1), 1),
    (dict(words=65537), 2), (dict(pos=ODD), 1), (dict(T=1 << 27, H=8), 2),
])
def test_tree_refuses(lib, bad, status):
    assert _tree(lib, **bad) == status


def test_tree_workspace(lib):
    w = lib.readme_attention_kv_tree_workspace_bytes
    for size in ((64, 64, 32, 8, 128, 64), (4096, 4, 8, 8, 128, 2000)):
        need = w(*size)
        assert need > 0
        T, R, H, Hk, D, mb = size
        assert _tree(lib, T=T, R=R, H=H, Hk=Hk, mb=mb, ld_q=H * 128, ld_o=H * 128, wsb=need - 1) == 3
    assert w(64, 64, 32, 7, 128, 64) == 0 and w(64, 0, 32, 8, 128, 64) == 0
    assert _tree(lib, T=0, R=0, q=None, o=None, offsets=None, lens=None, table=None, codes=None,
                 scales=None, tree=None, ws=None, wsb=0, mb=0, nb=0) == 0


def _verify(lib, **k):
    g = lambda n, d: k.get(n, d)  # noqa: E731
    return lib.readme_verify_drafts(
        g("dt", 0), g("T", 16), g("R", 2), g("V", 1000), g("offsets", FAKE), g("tokens", FAKE),
        g("parent", FAKE), g("p", FAKE), g("ld_p", 1000), g("q", FAKE), g("ld_q", 1000),
        g("u", FAKE), g("distinct", 0), g("path", FAKE), g("accepted", FAKE), g("token", FAKE),
        g("ws", FAKE), g("wsb", 1 << 40), None)


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), 1), (dict(R=-1), 1), (dict(R=0), 1), (dict(V=0), 1), (dict(dt=2), 2),
    (dict(distinct=2), 1), (dict(T=(1 << 27) + 1), 2), (dict(R=(1 << 20) + 1), 2),
    (dict(V=1 << 31), 2), (dict(R=1 << 20, V=(1 << 16) + 1), 2), (dict(offsets=None), 1),
    (dict(tokens=None), 1), (dict(parent=None), 1), (dict(p=None), 1), (dict(u=None), 1),
    (dict(path=None), 1), (dict(accepted=None), 1), (dict(token=None), 1), (dict(p=ODD), 1),
    (dict(q=ctypes.c_void_p(4104)), 1), (dict(u=ODD), 1), (dict(tokens=ODD), 1), (dict(token=ODD), 1),
    (dict(ld_p=996), 1), (dict(ld_p=1001), 1), (dict(ld_q=999), 1), (dict(dt=1, ld_p=1004), 1),
    (dict(ws=ODD), 1),
])
def test_verify_refuses(lib, bad, status):
    assert _verify(lib, **bad) == status


def test_verify_workspace(lib):
    w = lib.readme_verify_drafts_workspace_bytes
    assert w(-1, 2, 1000) == 0 and w(16, 0, 1000) == 0 and w(16, 2, 0) == 0 and w(16, 2, 1 << 31) == 0
    need = w(16, 2, 100000)
    if need:
        big = dict(V=100000, ld_p=100000, ld_q=100000)
        assert _verify(lib, wsb=need - 1, **big) == 3 and _verify(lib, ws=None, **big) == 1
    assert _verify(lib, T=0, R=0, offsets=None, accepted=None, token=None, ws=None, wsb=0) == 0


def test_python_forms_refuse():
    from paper_2410_19123_amd import _lib as L
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    x, f = torch.zeros((5, 128), dtype=torch.bfloat16), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="device tensors"):
        L.readme_rotary(x, i(5), f, 64)
    with pytest.raises(L.ReadmeError) as e:
        L.readme_rotary_freqs(24)
    assert e.value.status == 2
    codes, scales = torch.zeros((4, 2, 2, 64 * 64), dtype=torch.uint8), torch.zeros((4, 2, 2))
    with pytest.raises(ValueError, match="device tensors"):
        L.readme_kv_append(0, x, x, i(2), i(1), i(1, 3), codes, scales, f)
    with pytest.raises(ValueError, match="device tensors"):
        L.readme_attention_kv_tree(0, x, i(2), i(1), i(1, 3), codes, scales, 2,
                                   torch.zeros((5, 1), dtype=torch.int64))
    with pytest.raises(ValueError, match="device tensors"):
        L.readme_verify_drafts(i(2), i(5), i(5), torch.zeros(5, 8), None, torch.zeros(5))
