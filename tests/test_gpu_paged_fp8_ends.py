"""The paged 8-bit attention and forks at the ends of what they take: sequences, query heads on a kv head, forks of a call."""
import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import pages
from test_gpu_attn_paged_fp8 import DEV, _compare
from test_gpu_attn_paged_fp8_cuts import Quick

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,top", [((1024, 1, 4, 2, 64, 32), 90), ((1024, 1, 4, 2, 128, 64), 90), ((1024, 3, 2, 1, 64, 32), 40)])
def test_as_many_sequences_as_a_call_takes(shape, top):
    rng = np.random.default_rng(top)
    kv_len, nodes = rng.integers(0, top + 1, 1024).astype(np.int32), rng.integers(0, shape[1] + 1, 1024).astype(np.int32)
    kv_len[[0, 1023]], nodes[[0, 1023]] = top, shape[1]
    c = Quick(top, *shape, kv_len, nodes)
    want, off = c.reference()
    for workgroups in (0, 4096):
        got, _ = c.cut(top, workgroups)
        _compare(got, want, off)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,Hq,L", [(64, 128, 100), (1, 4096, 500), (3, 700, 33)])
def test_many_query_heads_on_one(N, Hq, L, D):
    """Rows of a kv head in hundreds of groups."""
    c = Quick(N + D, 2, N, Hq, 1, D, 32, np.array([L, 7], np.int32), np.array([N, N // 2], np.int32))
    want, off = c.reference()
    for workgroups in (0, 500):
        got, _ = c.cut(L, workgroups)
        _compare(got, want, off)


@pytest.mark.parametrize("n_pages", [9000, 40000])
@pytest.mark.parametrize("place", ["apart", "in place"])
def test_as_many_forks_as_a_call_takes(n_pages, place):
    """2048 forks in a table of 2048 rows: refused ones of every kind among them, more of them than rows without tokens."""
    rng = np.random.default_rng(n_pages)
    B, F, P, width = 2048, 2048, 16, 8
    lens, order = np.zeros(B, np.int64), rng.permutation(n_pages)
    with_tokens = rng.permutation(B)[:300]
    lens[with_tokens] = rng.integers(1, width * P + 1, 300)
    table, at = rng.integers(-5, 2 * n_pages, (B, width)), 0
    for b in with_tokens:
        n = -(-lens[b] // P)
        table[b, :n], at = order[at:at + n], at + n
    free = np.concatenate([order[at:], np.full(at, -1)])
    n_free, shared = np.array([min(n_pages - at, 900)]), np.zeros(n_pages, np.int64)
    src, dst = rng.choice(with_tokens, F), rng.permutation(B)
    odd = rng.permutation(F)
    src[odd[:20]], dst[odd[20:40]], dst[odd[40:80]] = -3, B + 7, dst[odd[80:120]]
    n_tokens = np.minimum(rng.integers(-1, width * P + 2, F), np.where(rng.random(F) < 0.9, np.maximum(lens[np.clip(src, 0, B - 1)], 0), 1 << 30))
    want = pages.fork(src, dst, lens, table, free, n_free, shared, P, n_tokens=n_tokens)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)  # noqa: E731
    args = [dev(a) for a in (lens, table, free, n_free, shared)]
    new = lambda: torch.empty(F, dtype=torch.int32, device=DEV)  # noqa: E731
    outputs = (new(), new(), args[0], args[3], args[4], new()) if place == "in place" else None
    got = fspad.fspad_page_fork(dev(src), dev(dst), *args, P, n_tokens=dev(n_tokens), outputs=outputs)
    torch.cuda.synchronize()
    for name, g, w in zip(("copy_src", "copy_dst", "kv_len", "n_free", "shared", "granted", "table"), (*got, args[1]), want):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert 100 < want[5].sum() < F and want[4].max() > 0
