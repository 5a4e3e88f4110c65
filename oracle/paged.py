"""Paged 4-bit cache, written down plainly in numpy with 64-bit arithmetic -- TEST INFRASTRUCTURE, as the rest of this package.

Values, pages and the page map follow the description in include/fspad.h, one value or one token at a time.
"""
from __future__ import annotations

import numpy as np

ELEMENTS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def block_scale(x) -> int:
    """Scale byte of one block of 32 values."""
    a = np.abs(np.asarray(x, np.float64))
    if not np.all(np.isfinite(a)):
        return 255
    for s in range(2, 253):
        if a.max() <= np.ldexp(7.0, s - 127):
            return s
    return 252


def block_codes(x, s: int) -> np.ndarray:
    """4-bit codes of a block under scale byte s: the nearest element, ties to the even code, at most 6."""
    x = np.asarray(x, np.float64)
    if s == 255:
        return np.zeros(len(x), np.uint8)
    y = np.abs(x) / np.ldexp(1.0, s - 127)
    far = np.abs(y[:, None] - ELEMENTS[None, :])
    best = far.min(axis=1, keepdims=True)
    code = np.array([min(np.flatnonzero(row), key=lambda c: c % 2) for row in far == best], np.uint8)
    return code | (np.signbit(x).astype(np.uint8) << 3)


def block_values(codes, s: int) -> np.ndarray:
    codes = np.asarray(codes)
    if s == 255:
        return np.full(len(codes), np.nan)
    v = ELEMENTS[codes & 7] * np.ldexp(1.0, int(s) - 127)
    return np.where(codes & 8, -v, v)


def page_head_bytes(D: int, P: int) -> int:
    return P * D * 17 // 16


class Pages:
    """A pool [n_pages, Hkv, page_head_bytes] of bytes, read and written token by token."""

    def __init__(self, raw: np.ndarray, D: int, P: int):
        assert raw.dtype == np.uint8 and raw.shape[2] == page_head_bytes(D, P)
        self.raw, self.D, self.P = raw, D, P

    def _places(self, which: str, t: int):
        """Byte and half-byte shift of every channel's code, and byte of every block's scale, of token t in a head's part of a page."""
        D, P = self.D, self.P
        c, b = np.arange(D), np.arange(D // 32)
        if which == "k":
            code, scale = t * (D // 2) + c // 2, P * D + b * P + t
        else:
            group, run = 512 // D, D // 16
            code = P * D // 2 + (((t // group) * 16 + c // run) * group + t % group) * (D // 32) + (c % run) // 2
            scale = P * D + P * D // 32 + b * P + t
        return code, 4 * (c % 2), scale

    def put(self, which: str, slot: int, head: int, x):
        part = self.raw[slot // self.P, head]
        code_at, shift, scale_at = self._places(which, slot % self.P)
        for blk in range(self.D // 32):
            r = slice(32 * blk, 32 * blk + 32)
            s = block_scale(x[r])
            part[scale_at[blk]] = s
            for at, sh, code in zip(code_at[r], shift[r], block_codes(x[r], s)):
                part[at] = (int(part[at]) & (0xF0 >> sh)) | (int(code) << sh)

    def get(self, which: str, slot: int, head: int) -> np.ndarray:
        part = self.raw[slot // self.P, head]
        code_at, shift, scale_at = self._places(which, slot % self.P)
        codes = (part[code_at] >> shift) & 15
        return np.concatenate([block_values(codes[32 * i:32 * i + 32], int(part[scale_at[i]])) for i in range(self.D // 32)])

    def get_many(self, which: str, slots) -> np.ndarray:
        """[len(slots), Hkv, D]"""
        slots = np.asarray(slots, np.int64)
        out = np.zeros((len(slots), self.raw.shape[1], self.D))
        for t in range(self.P):   # all slots of one place in their pages at once
            here = np.flatnonzero(slots % self.P == t)
            if len(here) == 0:
                continue
            part = self.raw[slots[here] // self.P]
            code_at, shift, scale_at = self._places(which, t)
            codes = (part[:, :, code_at] >> shift) & 15
            s = np.repeat(part[:, :, scale_at].astype(np.int64), 32, axis=2)
            v = np.ldexp(ELEMENTS[codes & 7], s - 127)
            out[here] = np.where(s == 255, np.nan, np.where(codes & 8, -v, v))
        return out


def page_map(kv_len, n_new, table, free, n_free, P, path=None, max_new=None, n_slots=None):
    """(slots, kv_len_out, n_free_out, granted, table, free): copies, the arguments stay as they are."""
    table, free = np.array(table, np.int64), np.array(free, np.int64)
    B, width = table.shape
    n_pages = len(free)
    top = int(min(max(int(np.asarray(n_free).reshape(-1)[0]), 0), n_pages))
    lens = [max(int(x), 0) for x in kv_len]
    out_len, granted = list(lens), [0] * B
    for b in range(B):                       # pages come back first
        if n_new[b] < 0:
            for i in range(min(-(-lens[b] // P), width)):
                if top < n_pages:
                    free[top] = table[b, i]
                    top += 1
            out_len[b] = 0
    slots = np.full(n_slots if max_new is None else (B, max_new), -1, np.int64)
    asked, avail, first = 0, top, 0
    for b in range(B):
        add, row0 = int(n_new[b]), first
        first += max(add, 0)
        if add < 0:
            continue
        have = min(-(-lens[b] // P), width)
        if lens[b] + add > width * P or (add > max_new if max_new is not None else row0 + add > n_slots):
            continue
        need = -(-(lens[b] + add) // P) - have
        asked += need
        if need and asked > avail:
            continue
        granted[b], out_len[b] = 1, lens[b] + add
        for i in range(need):
            top -= 1
            table[b, have + i] = free[top]
        seen = set()
        for j in range(add):
            page = int(table[b, (lens[b] + j) // P])
            slot = page * P + (lens[b] + j) % P if 0 <= page < n_pages else -1
            if max_new is None:
                slots[row0 + j] = slot
            elif path is None:
                slots[b, j] = slot
            else:
                node = int(path[b][j])
                if 0 <= node < max_new and node not in seen:
                    slots[b, node] = slot
                    seen.add(node)
    return slots, np.array(out_len), np.array([top]), np.array(granted), table, free


def tree_attn(q, k_tree, v_tree, pages: Pages, table, kv_len, n_nodes, mask, max_kv_len, scale=None):
    """(out [B,N,Hq,D], bound): the attention in 64 bits over what each row sees, and how far a computation may be off that

      - rounds every weight to bf16, relative error r = 2^-8 each, and divides by the sum of the rounded weights:
            |out' - out| <= r (1 + 2 r) sum_j w_j |v_j - out|,    w_j the exact weights, summing to 1
      - drops weights, and products of one with a value, below the smallest normal fp32 number (the largest weight being 1 at least, and the
        pieces of a row joined by factors that are dropped alike): n 2^-125 (1 + 2 max_j |v_j|)
      - holds a query as the sum of two fp8 values, off by 2^-22 of the row's largest at most, and sums its 2 D products in fp32, in any
        order and cut where it is not rounded: a score's error e <= (2 D + 8) 2^-23 scale sum_d |q_d k_jd| + 2^-22 scale max_d |q_d| sum_d
        |k_jd| moves its weight by a factor within 1 +- 2 e, an exponential by 2^-22, and the two sums over n keys by n 2^-24 of sum_j w_j |v_j| (numerator) and of |out| (denominator).
    Rounding of the output itself is the caller's."""
    B, N, Hq, D = q.shape
    Hkv = k_tree.shape[2]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(D) if not scale else float(scale)
    out, bound = np.zeros((B, N, Hq, D)), np.zeros((B, N, Hq, D))
    n_pages = pages.raw.shape[0]
    for b in range(B):
        n, L = min(max(int(n_nodes[b]), 0), N), min(max(int(kv_len[b]), 0), max_kv_len)
        t = np.arange(L)
        page = np.asarray(table[b], np.int64)[t // pages.P] if L else np.zeros(0, np.int64)
        there = (page >= 0) & (page < n_pages)
        slots = page[there] * pages.P + t[there] % pages.P
        kp, vp = pages.get_many("k", slots), pages.get_many("v", slots)
        for i in range(n):
            see = [x for x in range(n) if (int(mask[b, i]) >> x) & 1]
            for g in range(Hkv):
                k = np.concatenate([kp[:, g], k_tree[b, see, g]]).astype(np.float64)
                v = np.concatenate([vp[:, g], v_tree[b, see, g]]).astype(np.float64)
                if len(k) == 0:
                    continue
                qq = q[b, i, g * G:(g + 1) * G].astype(np.float64)
                with np.errstate(invalid="ignore", over="ignore"):
                    s = qq @ k.T * scale
                    top = s.max(axis=1, keepdims=True)
                    w = np.exp(s - np.where(np.isfinite(top), top, 0.0))
                    w = np.where(np.isnan(s) | (top == np.inf), np.nan, w)
                    total = w.sum(axis=1, keepdims=True)
                    w = np.where(total == 0, 0.0, w / np.where(total == 0, 1.0, total))
                    o = w @ v
                    e = abs(scale) * ((2 * D + 8) * 2.0 ** -23 * (np.abs(qq) @ np.abs(k).T)
                                      + 2.0 ** -22 * np.abs(qq).max(axis=1, keepdims=True) * np.abs(k).sum(axis=1)).max(axis=1, keepdims=True)
                    spread = np.stack([(w[h][:, None] * np.abs(v - o[h])).sum(axis=0) for h in range(G)])
                    r = 2.0 ** -8
                    bound[b, i, g * G:(g + 1) * G] = ((r * (1 + 2 * r) + 2 * e + 2.0 ** -22) * spread
                                                      + len(k) * 2.0 ** -24 * (w @ np.abs(v) + np.abs(o))
                                                      + len(k) * 2.0 ** -125 * (1 + 2 * np.abs(v).max(axis=0)))
                out[b, i, g * G:(g + 1) * G] = o
    return out, bound
