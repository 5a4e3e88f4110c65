"""Paged 8-bit cache, written down plainly in numpy with 64-bit arithmetic -- TEST INFRASTRUCTURE, as the rest of this package.

Values, blocks and pages follow the description in include/fspad.h. The page map and the attention are those of the 4-bit cache:
paged.page_map and paged.tree_attn, which takes Fp8Pages as well.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32


def _element(code: int) -> float:
    e, m = (code >> 3) & 15, code & 7
    x = np.nan if e == 15 and m == 7 else np.ldexp(m, -9) if e == 0 else np.ldexp(8 + m, e - 10)
    return -x if code & 128 else x


ELEMENTS = np.array([_element(c) for c in range(256)])
FINITE = ELEMENTS[:127]   # ascending, code after code


def block_scale(x) -> int:
    """Scale byte for values: of the finite ones the largest magnitude decides."""
    a = np.abs(np.asarray(x, np.float64)).reshape(-1)
    a = a[np.isfinite(a)]
    top = a.max() if len(a) else 0.0
    for s in range(10, 246):
        if top <= np.ldexp(448.0, s - 127):
            return s
    return 246


def codes_of(x, s: int) -> np.ndarray:
    """The nearest elements, ties to even codes, at most 448; all bits below the sign where x is not finite."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x)
    y = np.where(bad, 0.0, np.abs(x) / np.ldexp(1.0, int(s) - 127))
    up = np.minimum(np.searchsorted(FINITE, y), 126)          # the first element that is not below
    down = np.maximum(up - 1, 0)
    a, b = y - FINITE[down], FINITE[up] - y
    code = np.where(a < b, down, np.where(b < a, up, np.where(down % 2 == 0, down, up)))
    return (np.where(bad, 127, code) | (np.signbit(x) * 128)).astype(np.uint8)


def values_of(codes, s) -> np.ndarray:
    return ELEMENTS[np.asarray(codes)] * np.ldexp(1.0, np.asarray(s, np.int64) - 127)


def page_head_bytes(D: int, P: int) -> int:
    return 2 * P * D + 16


class Fp8Pages:
    """A pool [n_pages, Hkv, page_head_bytes] of bytes."""

    def __init__(self, raw: np.ndarray, D: int, P: int):
        assert raw.dtype == np.uint8 and raw.shape[2] == page_head_bytes(D, P)
        self.raw, self.D, self.P = raw, D, P

    def places(self, which: str, t: int):
        """Byte of every channel's code, and of the block's scale, of token t in a head's part of a page."""
        D, P, E, c = self.D, self.P, self.D // 32, np.arange(self.D)
        if which == "k":
            return ((t // 32 * (D // 16) + c // 16) * 32 + t % 32) * 16 + c % 16, 2 * P * D + t // 32
        return P * D + (((t // 32 * E + c % E) * 2 + t % 32 // 16) * 32 + c // E) * 16 + t % 16, 2 * P * D + 8 + t // 32

    def store(self, which: str, x, slots):
        """Rows x [rows, Hkv, D] into slots, block by block."""
        slots = np.asarray(slots, np.int64)
        blocks = {}
        for r in range(len(slots)):
            if 0 <= slots[r] < len(self.raw) * self.P:
                blocks.setdefault(int(slots[r]) // BLOCK, []).append(r)
        for block, rows in blocks.items():
            begun = any(slots[r] % BLOCK == 0 for r in rows)
            first = block * BLOCK
            for head in range(self.raw.shape[1]):
                part = self.raw[first // self.P, head]
                at_scale = self.places(which, first % self.P)[1]
                had, s = int(part[at_scale]), block_scale([x[r, head] for r in rows])
                if not begun:
                    s = max(s, had)
                    if s > had:
                        for t in range(first % self.P, first % self.P + BLOCK):
                            at = self.places(which, t)[0]
                            part[at] = codes_of(values_of(part[at], had), s)
                for r in rows:
                    part[self.places(which, int(slots[r]) % self.P)[0]] = codes_of(x[r, head], s)
                part[at_scale] = s

    def get_many(self, which: str, slots) -> np.ndarray:
        """[len(slots), Hkv, D]"""
        slots = np.asarray(slots, np.int64)
        out = np.zeros((len(slots), self.raw.shape[1], self.D))
        for t in range(self.P):   # all slots of one place in their pages at once
            here = np.flatnonzero(slots % self.P == t)
            if len(here):
                part = self.raw[slots[here] // self.P]
                code_at, scale_at = self.places(which, t)
                out[here] = values_of(part[:, :, code_at], part[:, :, scale_at][:, :, None])
        return out
