"""Sizes at which readme_attention_kv takes each of its forms: `rows/W` is the
kernel of 16 query rows with W waves to a whole (rows, key head) pair, `tiles/1`
the one of 128 rows, `rows/0` and `tiles/0` the two with the work dealt in shares.
`form` asks the library, so that a size named after a form takes that form."""
import ctypes

import numpy as np


def form(T, R, H, Hk, D, max_blocks, window=0) -> str:
    from paper_2410_19123_amd import _lib
    fn = _lib.load().readme_internal_attention_kv_form
    fn.restype = ctypes.c_int32
    fn.argtypes = [ctypes.c_int64] + [ctypes.c_int32] * 4 + [ctypes.c_int64] * 2
    rows, waves = divmod(fn(T, R, H, Hk, D, max_blocks, window), 256)
    return f"{ {16: 'rows', 128: 'tiles'}[rows]}/{waves}"


def _spread(lo, hi, R):
    return [lo + int((r + 0.5) * 0.6180339887 % 1.0 * (hi - lo + 1)) for r in range(R)]


class Size:
    """A call: new rows and lengths of the requests, key heads, query heads to
    each, the table's width (blocks past the lengths are absent)."""

    def __init__(self, new, lens, Hk, G, max_blocks):
        self.new, self.lens, self.Hk, self.G, self.max_blocks = list(new), list(lens), Hk, G, max_blocks

    def form(self, D, window=0):
        return form(sum(self.new), len(self.new), self.Hk * self.G, self.Hk, D, self.max_blocks, window)

    def cache(self, make, kt, D, seed):
        """A cache from tests.test_gpu_kv's makers with a table as wide as the
        size says: blocks of their own for the first six requests, the others
        share a few."""
        R, held = len(self.new), (max(max(self.lens), 1) + 63) // 64
        own = min(R, 6) * held
        c = make(kt, 1, self.Hk, D, own + (24 if R > 6 else 0), seed)
        table = np.full((R, self.max_blocks), -1, np.int32)
        table[:6, :held] = c.table[0, :own].reshape(-1, held)
        if R > 6:
            table[6:, :held] = c.rng.choice(c.table[0, own:], (R - 6, held))
        c.table = table
        return c


def _more(new, extra):
    return [n + e for n, e in zip(new, extra)]


# Requests of no rows, of more rows than tokens (rows before position 0), and of
# lengths at a block's border among them.
_T1 = [50, 70, 0, 33, 64, 100, 65, 40]
_T0 = [50, 70, 0, 33, 64, 100, 65, 40, 48, 51, 39, 128, 17, 1, 60, 44]
SIZES = {
    "rows/1": Size([1] * 300, _spread(0, 190, 300), 5, 1, 3),
    "rows/2": Size([1] * 200, _spread(0, 190, 200), 4, 2, 3),
    "rows/4": Size([1, 2] * 50, _spread(1, 380, 100), 4, 3, 6),
    "rows/8": Size([1, 3, 1], [640, 577, 64], 2, 7, 10),
    "rows/0": Size([1, 8, 0], [2100, 512, 77], 2, 2, 66),
    "rows/0 of 300": Size([1] * 300, _spread(0, 190, 300), 2, 4, 65),
    "tiles/1": Size(_T1, _more(_T1, [100, 0, 10, 95, 64, 200, -30, 3]), 13, 4, 6),
    "tiles/0": Size(_T0, _more(_T0, [250, 0, 10, 350, 64, 280, -30, 3] * 2), 13, 1, 20),
    "tiles/0 of 70": Size(_spread(0, 50, 70), _more(_spread(0, 50, 70), _spread(-9, 150, 70)), 2, 1, 70),
    "tiles/0 of 300": Size(_spread(4, 40, 300), _more(_spread(4, 40, 300), _spread(0, 90, 300)), 1, 1, 66),
}
# A window that leaves the form as it is, and hides tokens.
WINDOWS = {"rows/1": 20, "rows/2": 70, "rows/4": 90, "rows/8": 450, "tiles/1": 50, "tiles/0": 200}
# Up to 25 rows a request are few at heads of 64; at heads of 256 fewer waves fit.
AT_128_ONLY = ("tiles/0 of 70", "tiles/0 of 300")
AT_256_TOO = ("rows/0", "tiles/1", "tiles/0")


def kind(name: str) -> str:
    return name.split()[0]
