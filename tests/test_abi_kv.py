"""Refusals of the cache's entry points and of their Python form, on the CPU
(nothing reaches the GPU), and the size queries."""
import ctypes
import os

import pytest
import torch

FAKE = ctypes.c_void_p(4096)   # never dereferenced: every call fails validation
ODD = ctypes.c_void_p(4100)


@pytest.fixture(scope="module")
def lib():
    from paper_2410_19123_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libreadme.so not built")
    return _lib.load()


def test_sizes(lib):
    assert lib.readme_kv_codes_bytes(7, 8, 128) == 7 * 8 * 2 * 64 * 128
    assert lib.readme_kv_codes_bytes(1 << 21, 8, 128) == (1 << 21) * 8 * 2 * 64 * 128
    assert lib.readme_kv_scales_bytes(7, 8) == 7 * 8 * 2 * 4
    assert lib.readme_kv_codes_bytes(7, 8, 96) == 0
    assert lib.readme_kv_codes_bytes(-1, 8, 128) == 0
    assert lib.readme_kv_codes_bytes(7, 0, 128) == 0
    assert lib.readme_kv_scales_bytes(7, 0) == 0
    w = lib.readme_attention_kv_workspace_bytes
    assert w(64, 64, 32, 8, 128, 64) > 0
    assert w(64, 64, 32, 7, 128, 64) == 0
    assert w(64, 64, 32, 8, 80, 64) == 0
    assert w(-1, 64, 32, 8, 128, 64) == 0
    assert w(64, 0, 32, 8, 128, 64) == 0
    assert w(1 << 26, 64, 32, 8, 128, 64) == 0


def _write(lib, read=False, **k):
    g = lambda n, d: k.get(n, d)  # noqa: E731
    rows = [g("k", FAKE), g("ld_k", 1024), g("v", FAKE), g("ld_v", 1024)]
    where = [g("offsets", FAKE), g("lens", FAKE), g("table", FAKE), g("mb", 4), g("nb", 9)]
    store = [g("codes", FAKE), g("scales", FAKE)]
    head = [g("kt", 0), g("dt", 1), g("T", 16), g("R", 2), g("Hk", 8), g("D", 128)]
    if read:
        return lib.readme_kv_read(*head, *where, *store, *rows, None)
    return lib.readme_kv_write(*head, *rows, *where, *store, None)


BAD = [
    (dict(T=-1), 1), (dict(R=-1), 1), (dict(R=0), 1), (dict(Hk=0), 1), (dict(mb=0), 1),
    (dict(nb=0), 1), (dict(mb=-1), 1), (dict(kt=2), 2), (dict(kt=-1), 2), (dict(dt=2), 2),
    (dict(D=96), 2), (dict(D=0), 2), (dict(Hk=65536), 2), (dict(R=(1 << 22) + 1), 2),
    (dict(T=(1 << 27) + 1), 2), (dict(mb=1 << 26), 2), (dict(nb=1 << 32), 2),
    (dict(k=None), 1), (dict(v=None), 1), (dict(offsets=None), 1), (dict(lens=None), 1),
    (dict(table=None), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(k=ODD), 1),
    (dict(v=ODD), 1), (dict(codes=ODD), 1), (dict(scales=ODD), 1), (dict(ld_k=1023), 1),
    (dict(ld_v=1016), 1), (dict(ld_k=1028), 1), (dict(offsets=ctypes.c_void_p(4098)), 1),
]


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("bad,status", BAD)
def test_write_and_read_refuse(lib, read, bad, status):
    assert _write(lib, read, **bad) == status


def test_no_rows_is_no_work(lib):
    none = dict(T=0, R=0, k=None, v=None, offsets=None, lens=None, table=None, codes=None,
                scales=None, mb=0, nb=0)
    assert _write(lib, **none) == 0
    assert _write(lib, True, **none) == 0
    assert _attention(lib, T=0, R=0, q=None, o=None, offsets=None, lens=None, table=None,
                      codes=None, scales=None, ws=None, wsb=0, mb=0, nb=0) == 0


def _attention(lib, **k):
    g = lambda n, d: k.get(n, d)  # noqa: E731
    return lib.readme_attention_kv(
        g("kt", 0), g("T", 16), g("R", 2), g("H", 16), g("Hk", 8), g("D", 128), g("q", FAKE),
        g("ld_q", 2048), g("offsets", FAKE), g("lens", FAKE), g("table", FAKE), g("mb", 4),
        g("nb", 9), g("codes", FAKE), g("scales", FAKE), ctypes.c_float(g("scale", 0.1)),
        g("causal", 1), g("window", 0), g("o", FAKE), g("ld_o", 2048), g("ws", FAKE),
        g("wsb", 1 << 40), None)


@pytest.mark.parametrize("bad,status", [b for b in BAD if not {"k", "v", "ld_k", "ld_v", "dt"} &
                                        set(b[0])] + [
    (dict(H=15), 1), (dict(H=0), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(scale=3.4e38), 1),
    (dict(causal=2), 1), (dict(causal=-1), 1), (dict(window=-1), 1), (dict(q=None), 1),
    (dict(o=None), 1), (dict(q=ODD), 1), (dict(o=ODD), 1), (dict(ld_q=2040), 1),
    (dict(ld_o=2052), 1), (dict(ws=None), 1), (dict(ws=ODD), 1), (dict(wsb=16), 3),
    (dict(T=1 << 26, H=32), 2),
])
def test_attention_refuses(lib, bad, status):
    assert _attention(lib, **bad) == status


@pytest.mark.parametrize("T,R,H,Hk", [
    (1 << 27, 1, 8, 8),              # row tiles times heads past the grids
    (1 << 20, 1 << 20, 64, 64),      # and requests times heads
    (16, 1 << 22, 8, 8),
    (16, 129, 65535, 65535),
])
def test_attention_refuses_what_its_grids_cannot_hold(lib, T, R, H, Hk):
    assert _attention(lib, T=T, R=R, H=H, Hk=Hk, ld_q=H * 128, ld_o=H * 128) == 2
    assert lib.readme_attention_kv_workspace_bytes(T, R, H, Hk, 128, 4) == 0


def test_a_window_needs_no_more_workspace(lib):
    """The workspace query knows no window; a call with one takes what it
    says for the same sizes (any smaller one is refused)."""
    w = lib.readme_attention_kv_workspace_bytes
    for T, R, mb in ((64, 64, 2000), (4096, 4, 2000), (1000, 3, 40), (1 << 23, 1, 1 << 20)):
        need = w(T, R, 8, 8, 128, mb)
        assert need > 0
        for window in (0, 1, 1000, (1 << 63) - 1):
            assert _attention(lib, T=T, R=R, H=8, Hk=8, mb=mb, window=window, wsb=need - 1) == 3


def test_python_form_refuses():
    from paper_2410_19123_amd import _lib as L
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    codes, scales = torch.zeros((4, 2, 2, 64 * 64), dtype=torch.uint8), torch.zeros((4, 2, 2))
    k = torch.zeros((5, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensors"):
        L.readme_kv_write(0, k, k, i(2), i(1), i(1, 3), codes, scales)
    with pytest.raises(ValueError, match="device tensors"):
        L.readme_attention_kv(0, k, i(2), i(1), i(1, 3), codes, scales, H=2)


def _router(lib, **k):
    g = lambda n, d: k.get(n, d)  # noqa: E731
    return lib.readme_router_tf_cached(
        g("kt", 0), g("T", 16), g("R", 2), g("D", 256), g("F", 64), g("E", 8), g("V", 100),
        g("tokens", FAKE), g("offsets", FAKE), g("lens", FAKE), g("table", FAKE), g("mb", 4),
        g("nb", 9), g("codes", FAKE), g("scales", FAKE), g("emb", FAKE), g("packed", FAKE),
        g("w_router", FAKE), None, ctypes.c_float(g("eps", 1e-5)), g("ids", FAKE), None,
        g("ws", FAKE), g("wsb", 1 << 40), None)


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), 1), (dict(R=-1), 1), (dict(R=0), 1), (dict(mb=0), 1), (dict(nb=0), 1),
    (dict(kt=2), 2), (dict(D=0), 1), (dict(D=192), 2), (dict(D=32768), 2), (dict(F=0), 1),
    (dict(E=0), 2), (dict(E=257), 2), (dict(V=0), 1), (dict(eps=-1.0), 1),
    (dict(T=1 << 27), 2), (dict(R=(1 << 22) + 1), 2), (dict(mb=1 << 26), 2), (dict(nb=1 << 32), 2),
    (dict(tokens=None), 1), (dict(offsets=None), 1), (dict(lens=None), 1), (dict(table=None), 1),
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(emb=None), 1), (dict(packed=None), 1),
    (dict(w_router=None), 1), (dict(ids=None), 1), (dict(ws=None), 1), (dict(ws=ODD), 1),
    (dict(codes=ODD), 1), (dict(emb=ODD), 1), (dict(wsb=64), 3),
])
def test_cached_router_refuses(lib, bad, status):
    assert _router(lib, **bad) == status


def test_cached_router_workspace(lib):
    w = lib.readme_router_tf_cached_workspace_bytes
    need = w(16, 2, 256, 64, 4)
    assert need == (lib.readme_router_tf_workspace_bytes(16, 256, 64) +
                    lib.readme_attention_kv_workspace_bytes(16, 2, 2, 2, 128, 4))
    assert _router(lib, wsb=need - 1) == 3
    assert w(16, 2, 192, 64, 4) == 0 and w(16, 0, 256, 64, 4) == 0 and w(-1, 2, 256, 64, 4) == 0
    none = dict(T=0, R=0, mb=0, nb=0, tokens=None, offsets=None, lens=None, table=None, codes=None,
                scales=None, emb=None, packed=None, w_router=None, ids=None, ws=None, wsb=0)
    assert _router(lib, **none) == 0
