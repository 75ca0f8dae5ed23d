"""The form of the cache attention by its sizes alone (no GPU: the rule is host
code): the sizes of the GPU tests take the forms they are named after."""
import os

import pytest

from tests.kv_forms import AT_128_ONLY, AT_256_TOO, SIZES, WINDOWS, form, kind


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2410_19123_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libreadme.so not built")


@pytest.mark.parametrize("name", SIZES)
def test_sizes_take_their_forms(name):
    assert SIZES[name].form(128) == kind(name)
    if name not in AT_128_ONLY:
        assert SIZES[name].form(64) == kind(name)


@pytest.mark.parametrize("name", WINDOWS)
def test_and_so_with_their_windows(name):
    assert SIZES[name].form(128, WINDOWS[name]) == name
    assert SIZES[name].form(64, WINDOWS[name]) == name


@pytest.mark.parametrize("name", AT_256_TOO)
def test_at_heads_of_256(name):
    assert SIZES[name].form(256, WINDOWS.get(name, 0)) == name


def test_sizes_of_far_apart_scales():
    from tests.test_gpu_kv_scales import FORMS
    for name, (new, _, R, Hk, G, mb, window) in FORMS.items():
        for D in (64, 128):
            for w in (0, window):
                assert form(new * R, R, Hk * G, Hk, D, mb, w) == name, (name, D, w)


@pytest.mark.parametrize("sizes,want", [
    # rows of a call, requests, query and key heads, head dims, blocks of the table
    ((1, 1, 4, 4, 128, 9), "rows/8"),             # one request's next token
    ((64, 64, 32, 8, 128, 64), "rows/4"),         # a decode step
    ((8, 8, 32, 8, 128, 2048), "rows/0"),         # of long requests
    ((8192, 256, 4, 4, 128, 1), "rows/1"),        # many short prompts
    ((8192, 4, 32, 8, 128, 32), "tiles/1"),       # prompts
    ((1400, 3, 28, 4, 64, 313), "tiles/0"),       # pieces of long prompts
])
def test_what_a_server_calls(sizes, want):
    assert form(*sizes) == want
