"""CPU pins of the oracle's paged 8-bit cache: the format by hand-written bytes, the rounding's bound, blocks that grow."""
import numpy as np
import pytest

from oracle import paged, paged_fp8


def test_elements():
    e = paged_fp8.ELEMENTS
    assert e[0] == 0 and e[1] == 2.0 ** -9 and e[8] == 2.0 ** -6 and e[0x38] == 1.0 and e[0x7e] == 448 and np.isnan(e[0x7f]) and np.isnan(e[0xff])
    assert np.all(np.diff(paged_fp8.FINITE) > 0) and np.array_equal(e[128:255], -e[:127])


@pytest.mark.parametrize("top,s", [(0.0, 10), (2.0 ** -133, 10), (448 * 2.0 ** -117, 10), (450 * 2.0 ** -117, 11), (448.0, 127), (450.0, 128), (1.75, 119),
                                   (448 * 2.0 ** 119, 246), (255 * 2.0 ** 120, 246), (np.inf, 10), (np.nan, 10)])
def test_scales(top, s):
    assert paged_fp8.block_scale([0.0, -top, 0.0]) == s


def test_codes_by_hand():
    x = [448, -1.0, 1.0625, 1.1875, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, -0.0, np.nan, np.inf]
    assert list(paged_fp8.codes_of(x, 127)) == [0x7e, 0xb8, 0x38, 0x3a, 0x58, 0x5a, 0, 2, 0x80, 0x7f, 0x7f]   # ties to the even code
    assert list(paged_fp8.codes_of([255 * 2.0 ** 120], 246)) == [0x7e]


def test_rounding_is_off_by_at_most_a_sixteenth():
    rng = np.random.default_rng(1)
    x = rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 8, 20000)
    s = paged_fp8.block_scale(x)
    off = np.abs(paged_fp8.values_of(paged_fp8.codes_of(x, s), s) - x)
    assert np.all(off <= np.maximum(np.abs(x) / 16, 2.0 ** (s - 137)))


@pytest.mark.parametrize("D,P", [(64, 32), (128, 32), (64, 256), (128, 64)])
def test_a_page_holds_every_token_in_bytes_of_its_own(D, P):
    p = paged_fp8.Fp8Pages(np.zeros((1, 1, paged_fp8.page_head_bytes(D, P)), np.uint8), D, P)
    seen, scales = np.zeros(p.raw.shape[2], int), set()
    for which in "kv":
        for t in range(P):
            code, scale = p.places(which, t)
            np.add.at(seen, code, 1)
            scales.add((which, t // 32, scale))
    assert np.all(seen[:2 * P * D] == 1) and np.all(seen[2 * P * D:] == 0)
    assert len({s for _, _, s in scales}) == len(scales) == 2 * (P // 32) and min(s for _, _, s in scales) == 2 * P * D


def test_bytes_of_a_page_by_hand():
    D, P = 128, 64
    p = paged_fp8.Fp8Pages(np.zeros((1, 1, paged_fp8.page_head_bytes(D, P)), np.uint8), D, P)
    x = np.zeros((1, 1, D))
    x[0, 0, 19] = 448.0
    p.store("k", x, [32 + 5])
    p.store("v", x, [32 + 21])
    raw = p.raw[0, 0]
    assert raw[32 * 128 + (1 * 32 + 5) * 16 + 3] == 0x7e and raw[2 * 64 * 128 + 1] == 127                  # K: block 1, piece 1, token 5
    assert raw[64 * 128 + 32 * 128 + ((3 * 2 + 1) * 32 + 4) * 16 + 5] == 0x7e and raw[2 * 64 * 128 + 9] == 127   # V: channel 19 = 4 * 4 + 3


def test_a_block_that_grows():
    D, P = 64, 32
    p = paged_fp8.Fp8Pages(np.full((1, 1, paged_fp8.page_head_bytes(D, P)), 0xff, np.uint8), D, P)
    x = np.full((2, 1, D), 1.0)
    x[1] = 1.0 / 64 + 1.0 / 512
    p.store("k", x, [0, 1])                                  # begins: 1.0 needs 2^(119-127), whatever the byte held
    assert p.raw[0, 0, 2 * P * D] == 119
    assert np.array_equal(p.get_many("k", [0, 1]), x)
    p.store("k", np.full((1, 1, D), 0.25), [2])              # needs less: the scale stays
    assert p.raw[0, 0, 2 * P * D] == 119
    p.store("k", np.full((1, 1, D), 448.0), [3])             # 256 times as much: 1/64 + 1/512 is 2^-6 + 2^-9 of the new scale
    assert p.raw[0, 0, 2 * P * D] == 127
    assert np.array_equal(p.get_many("k", [0, 1, 2, 3])[:, 0, 0], [1.0, 1 / 64 + 1 / 512, 0.25, 448.0])
    p.store("k", np.full((1, 1, D), 448.0 * 2), [4])         # 9 of the smallest elements become 4, the even one of 4 and 5
    assert p.get_many("k", [1])[0, 0, 0] == 4 / 256
    p.store("k", np.full((1, 1, D), 0.5), [0])               # the first token again: a new beginning
    assert p.raw[0, 0, 2 * P * D] == 118 and p.get_many("k", [0])[0, 0, 0] == 0.5


def test_attention_takes_these_pages():
    rng = np.random.default_rng(3)
    D, P = 64, 32
    p = paged_fp8.Fp8Pages(rng.integers(0, 256, (3, 1, paged_fp8.page_head_bytes(D, P)), dtype=np.uint8), D, P)
    k, v = rng.standard_normal((2, 40, 1, D))
    slots = np.array([[2, 0][t // P] * P + t % P for t in range(40)])
    p.store("k", k, slots)
    p.store("v", v, slots)
    q, kt, vt = (rng.standard_normal((1, 1, 1, D)) for _ in range(3))
    out, bound = paged.tree_attn(q, kt, vt, p, [[2, 0]], [40], [1], np.ones((1, 1), np.uint64), 64)
    kk, vv = np.concatenate([p.get_many("k", slots)[:, 0], kt[0, 0]]), np.concatenate([p.get_many("v", slots)[:, 0], vt[0, 0]])
    w = np.exp(kk @ q[0, 0, 0] / 8)
    assert np.allclose(out[0, 0, 0], w @ vv / w.sum()) and np.all(bound > 0)
