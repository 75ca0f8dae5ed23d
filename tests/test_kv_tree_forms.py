"""The form of the attention of draft trees by its sizes alone (no GPU: the rule
is host code): chains of few drafts, where tiles of rows are far from full, and the
largest calls, whose launches keep below 2^32 threads."""
import ctypes
import os

import pytest

MAX_PAIRS = 1 << 23  # T H / 16 + R Hk, as the header states it


@pytest.fixture(scope="module")
def form():
    from paper_2410_19123_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libreadme.so not built")
    fn = _lib.load().readme_internal_attention_kv_tree_form
    fn.restype = ctypes.c_int32
    fn.argtypes = [ctypes.c_int64] + [ctypes.c_int32] * 4 + [ctypes.c_int64] * 2
    return lambda T, R, H, Hk, D, blocks, window=0: divmod(fn(T, R, H, Hk, D, blocks, window), 256)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R,n,G,Hk,blocks,waves", [
    # Chains: every request has tiles of its own, so that 64 to 256 requests fill the
    # chip with 4 waves a pair or, many of them on tables of few blocks, 2
    (64, 1, 1, 8, 32, 4), (64, 3, 1, 8, 64, 4), (64, 5, 2, 8, 32, 4), (128, 1, 1, 8, 32, 4),
    (128, 3, 1, 8, 40, 4), (256, 1, 1, 8, 32, 4), (256, 1, 1, 8, 64, 4), (256, 5, 1, 8, 32, 4),
    (64, 5, 1, 32, 64, 4), (64, 8, 1, 8, 16, 4), (256, 5, 1, 8, 8, 2), (64, 1, 1, 32, 8, 2),
    (1024, 1, 1, 8, 32, 4),
    # Few pairs take as many as there are blocks for
    (64, 3, 2, 2, 64, 8), (16, 5, 1, 8, 64, 8), (128, 5, 1, 2, 8, 4),
    # Full tiles, one pair each
    (16, 16, 4, 8, 64, 4), (64, 8, 4, 8, 64, 2), (128, 8, 4, 8, 8, 1), (16, 16, 4, 8, 8, 4), (48, 12, 7, 4, 13, 2),
    (40, 1, 4, 32, 4, 1)])
def test_rows_in_tiles_of_16(form, R, n, G, Hk, blocks, waves, D):
    assert form(R * n, R, Hk * G, Hk, D, blocks) == (16, waves)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R,n,G,Hk,blocks,window,waves", [
    (16, 32, 4, 8, 64, 0, 4), (128, 32, 4, 8, 8, 0, 1), (40, 130, 1, 4, 16, 0, 2), (64, 32, 4, 4, 32, 0, 2), (64, 40, 4, 4, 4, 0, 1)])
def test_rows_in_tiles_of_32(form, R, n, G, Hk, blocks, window, waves, D):
    assert form(R * n, R, Hk * G, Hk, D, blocks, window) == (32, waves)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("blocks", [1, 4, 8, 16, 32, 64, 65, 4000])
@pytest.mark.parametrize("T,R,G,Hk", [
    (1, 1 << 22, 1, 2), (1 << 21, 1 << 22, 1, 1), (1 << 22, 1 << 22, 1, 1), (1 << 20, 1 << 20, 2, 7),
    (8, 1 << 7, 1, 65535), ((1 << 27) - 16, 1, 1, 1), ((1 << 23) - 16, (1 << 17) - 1, 8, 1),
    ((1 << 21) - 16, (1 << 18) - 1, 16, 3), (128, 1, 1, 65535)])
def test_threads_of_the_largest_calls(form, T, R, G, Hk, blocks, D):
    """The grid of whole pairs: a workgroup for every slot of the requests' tiles and
    key head, in eights of up to 16 slots or, tiles of 128 rows, a column a request."""
    assert (T * G // 16 + R) * Hk <= MAX_PAIRS
    rows, waves = form(T, R, Hk * G, Hk, D, blocks)
    if waves:
        slots = T * G // rows + R
        if rows == 128:
            threads = -(-slots // R) * R * Hk * 256
        else:
            threads = (slots * Hk + 128) * 64 * min(waves, 4 if D == 256 else 8)
        assert threads < 1 << 32
