"""CPU pins of the oracle's paged 4-bit cache: the format by hand-written bytes, the rounding's bound, the page map's rules."""
import numpy as np
import pytest

from oracle import paged


def test_block_by_hand():
    x = np.zeros(32)
    x[:8] = [6.0, -0.25, 0.75, 5.0, 1.25, -7.0, 2.5, 0.26]
    s = paged.block_scale(x)
    assert s == 127                                     # 7 <= 7 * 2^0
    assert list(paged.block_codes(x, s)[:8]) == [7, 8, 2, 6, 2, 15, 4, 1]
    assert list(paged.block_values([7, 8, 2, 6, 2, 15, 4, 1], s)) == [6, 0, 1, 4, 1, -6, 2, 0.5]
    assert paged.block_scale([7.0625] + [0.0] * 31) == 128


@pytest.mark.parametrize("top,s", [(0.0, 2), (2.0 ** -133, 2), (7 * 2.0 ** -125, 2), (7.03125 * 2.0 ** -125, 3), (7 * 2.0 ** 125, 252),
                                   (255 * 2.0 ** 120, 252), (np.inf, 255), (np.nan, 255)])
def test_scales_at_the_ends(top, s):
    x = np.zeros(32)
    x[5] = top
    assert paged.block_scale(x) == s
    if s == 255:
        assert np.all(np.isnan(paged.block_values(paged.block_codes(x, s), s)))
    else:
        assert abs(paged.block_values(paged.block_codes(x, s), s)[5]) <= 6 * 2.0 ** (s - 127)


def test_rounding_is_off_by_at_most_the_scale():
    rng = np.random.default_rng(1)
    for _ in range(200):
        x = rng.standard_normal(32) * 2.0 ** rng.integers(-30, 30)
        s = paged.block_scale(x)
        off = np.abs(paged.block_values(paged.block_codes(x, s), s) - x).max()
        assert off <= 2.0 ** (s - 127) < np.abs(x).max() * 2 / 7


@pytest.mark.parametrize("D,P", [(64, 16), (128, 16), (64, 256), (128, 64)])
def test_a_page_holds_every_token_in_bytes_of_its_own(D, P):
    rng = np.random.default_rng(2)
    raw = rng.integers(0, 256, (2, 1, paged.page_head_bytes(D, P)), dtype=np.uint8)
    p = paged.Pages(raw, D, P)
    seen = np.zeros(raw.shape[2], int)
    for which in "kv":
        for t in range(P):
            code, shift, scale = p._places(which, t)
            np.add.at(seen, code, shift // 4 * 2 - 1 + 2)   # 1 for the low half, 3 for the high one
            seen[scale] += 4
    assert np.all(seen == 4)
    x = rng.standard_normal((2, D))
    p.put("k", P + 3, 0, x[0])
    p.put("v", P + 3, 0, x[1])
    for which, row in zip("kv", x):
        got = p.get(which, P + 3, 0)
        assert np.array_equal(got, p.get_many(which, [P + 3])[0, 0])
        assert np.abs(got - row).max() < np.abs(row).max() * 2 / 7


def test_bytes_of_a_page_by_hand():
    D, P = 128, 16
    p = paged.Pages(np.zeros((1, 1, paged.page_head_bytes(D, P)), np.uint8), D, P)
    x = np.zeros(D)
    x[9], x[8], x[127] = 6.0, 3.0, -1.5
    p.put("k", 2, 0, x)
    p.put("v", 6, 0, x)
    raw = p.raw[0, 0]
    assert raw[2 * 64 + 4] == 0x75                       # K: row of token 2, channels 8 (3.0) and 9 (6.0)
    assert raw[16 * 64 + ((6 // 4 * 16 + 1) * 4 + 6 % 4) * 4] == 0x75   # V: group 1, run 1 (channels 8..15), token 2 of the group
    assert raw[16 * 128 + 2] == 127 and raw[16 * 128 + 16 + 2] == 2     # K scales of block 0 and of the empty block 1
    assert raw[16 * 128 + 16 * 4 + 3 * 16 + 6] == 125    # V scale of block 3: 1.5 <= 7 * 2^-2


def test_page_map_by_hand():
    table = [[4, 1, -1], [0, -1, -1], [3, -1, -1]]
    free = [2, 5, -9, -9, -9, -9]
    # b0 grows past its page, b1 ends, b2 grows by three pages: one more than there are
    slots, lens, top, granted, t, f = paged.page_map([17, 5, 16], [20, -1, 40], table, free, [2], 16, max_new=40)
    assert list(f[:3]) == [2, 5, 0] and int(top[0]) == 2 and list(granted) == [1, 0, 0] and list(lens) == [37, 0, 16]
    assert list(t[0]) == [4, 1, 0] and list(t[2]) == [3, -1, -1]
    assert list(slots[0, :16]) == [16 + 1 + j for j in range(15)] + [0] and slots[0, 20] == -1 and np.all(slots[1:] == -1)
    # by path: nodes 0, 4 and 2 take the next three places
    slots, *_ = paged.page_map([30], [3], [[4, 1, -1]], free, [2], 16, path=[[0, 4, 2, -1, -1]], max_new=5)
    assert list(slots[0]) == [16 + 14, -1, 5 * 16, -1, 16 + 15]
    # packed: refused rows keep their places
    slots, *_ = paged.page_map([0, 0, 0], [2, 100, 1], [[-1], [-1], [-1]], free, [2], 16, n_slots=110)
    assert list(slots[:3]) == [80, 81, -1] and slots[102] == 32 and slots[103] == -1


def test_attention_leaves_out_what_is_not_seen():
    rng = np.random.default_rng(3)
    D, P = 64, 16
    p = paged.Pages(rng.integers(0, 256, (4, 1, paged.page_head_bytes(D, P)), dtype=np.uint8), D, P)
    for t in range(20):
        for w in "kv":
            p.put(w, [2, 0][t // P] * P + t % P, 0, rng.standard_normal(D))
    q, kt, vt = (rng.standard_normal((1, 3, 1, D)) for _ in range(3))
    vt[0, 2] = np.nan
    mask = np.array([[1, 3, 5]], np.uint64)
    out, bound = paged.tree_attn(q, kt, vt, p, [[2, 0]], [20], [3], mask, 32)
    assert np.all(np.isfinite(out[0, :2])) and np.all(np.isnan(out[0, 2])) and np.all(bound[0, :2] > 0)
    bad, _ = paged.tree_attn(q, kt, vt, p, [[2, 7]], [20], [3], mask, 32)
    short, _ = paged.tree_attn(q, kt, vt, p, [[2, 7]], [16], [3], mask, 32)
    assert np.array_equal(bad[0, :2], short[0, :2])
    none, _ = paged.tree_attn(q, kt, vt, p, [[2, 0]], [0], [3], np.array([[1, 0, 0]], np.uint64), 32)
    assert np.all(none[0, 1] == 0) and np.allclose(none[0, 0, 0], vt[0, 0, 0])
