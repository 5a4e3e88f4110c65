"""GPU parity of the tree attention over the paged 8-bit cache against the oracle, element by element within the bound that the
oracle derives for bf16 weights and fp32 sums (outputs in fp32; the bf16 output is that one rounded once)."""
import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import paged, paged_fp8
from workloads import gen_trees

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


class Case:
    """Random tables with junk behind their pages; tokens that are there hold N(0,spread), rounded under their block's scale; everything else
    of a page is random bytes (codes of NaN and scales of 255 among them)."""

    def __init__(self, seed, B, N, Hq, Hkv, D, P, kv_len, n_nodes=None, spread=1.0):
        rng = np.random.default_rng(seed)
        self.shape, self.P = (B, N, Hq, Hkv, D), P
        self.kv_len = np.asarray(kv_len, np.int32)
        self.n_nodes = np.full(B, N, np.int32) if n_nodes is None else np.asarray(n_nodes, np.int32)
        held = -(-np.maximum(self.kv_len, 0) // P)
        width, n_pages = int(held.max()) + 1, int(held.sum()) + 2
        order = rng.permutation(n_pages)
        self.table = rng.integers(-3, 2 * n_pages, (B, width)).astype(np.int32)
        raw = rng.integers(0, 256, (n_pages, Hkv, paged_fp8.page_head_bytes(D, P)), dtype=np.uint8)
        self.raw, at, p = raw, 0, paged_fp8.Fp8Pages(raw, D, P)
        places = [[p.places(w, t) for t in range(P)] for w in "kv"]
        for b in range(B):
            self.table[b, :held[b]] = order[at:at + held[b]]
            at += held[b]
            for i in range(held[b]):
                fill, page = min(P, int(self.kv_len[b]) - i * P), raw[self.table[b, i]]
                for w in range(2):
                    for t0 in range(0, fill, 32):
                        n = min(32, fill - t0)
                        x = rng.standard_normal((n, Hkv, D)) * (spread if w == 0 else 1.0)
                        s = paged_fp8.block_scale(x) + int(rng.integers(0, 3))   # (a block may have held larger tokens)
                        code = paged_fp8.codes_of(x, s)
                        for t in range(n):
                            page[:, places[w][t0 + t][0]] = code[t]
                        page[:, places[w][t0][1]] = s
        self.q, self.kt, self.vt = (_bf16(rng.standard_normal(s)) for s in ((B, N, Hq, D), (B, N, Hkv, D), (B, N, Hkv, D)))
        parent, _ = gen_trees(seed, B, N, 6, min(10, max(1, N - 1)), n_nodes=np.maximum(self.n_nodes, 1))
        self.mask = fspad.fspad_tree_build_mask(parent, np.maximum(self.n_nodes, 1))

    def run(self, out_dtype=torch.float32, scale=0.0, workgroups=0, max_kv_len=None, poison=True, pages=None, guard=0):
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
        pages = dev(self.raw) if pages is None else pages
        q, kt, vt, table = self.q.to(DEV), self.kt.to(DEV), self.vt.to(DEV), dev(self.table)
        if max_kv_len is None:
            max_kv_len = max(0, int(self.kv_len.max()))
        desc = fspad.make_paged_desc(q, kt, pages, table, max_kv_len, out_dtype, scale, workgroups, fp8=True)
        size = fspad.fspad_tree_attn_paged_byte_workspace_bytes(desc)
        ws = torch.full((size + guard,), 0xFF if poison else 0, dtype=torch.uint8, device=DEV)
        out = torch.full(q.shape, float("nan"), dtype=out_dtype, device=DEV)
        fspad.fspad_tree_attn_paged_byte(q, kt, vt, pages, table, dev(self.kv_len), dev(self.n_nodes), dev(self.mask.view(np.int64)), out=out,
                                         workspace=ws[:size], desc=desc)
        torch.cuda.synchronize()
        assert bool((ws[size:] == (0xFF if poison else 0)).all())
        return out

    def reference(self, scale=None, max_kv_len=1 << 30):
        D, f = self.shape[4], lambda t: t.double().numpy()  # noqa: E731
        return paged.tree_attn(f(self.q), f(self.kt), f(self.vt), paged_fp8.Fp8Pages(self.raw, D, self.P), self.table, self.kv_len, self.n_nodes,
                               self.mask, max_kv_len, scale)

    def check(self, **kw):
        got = self.run(**kw).double().cpu().numpy()
        want, bound = self.reference(kw.get("scale", 0.0), kw.get("max_kv_len") or 1 << 30)
        _compare(got, want, bound)
        return got


def _compare(got, want, bound):
    assert np.array_equal(np.isfinite(got), np.isfinite(want))
    f = np.isfinite(want)
    off = np.abs(got[f] - want[f])
    over = off - bound[f]
    assert over.size == 0 or over.max() <= 0.0, f"off by {off.max():.3g}, {over.max():.3g} more than the bound allows"


@pytest.mark.parametrize("D,P", [(128, 32), (64, 32), (64, 64), (128, 64), (128, 256), (64, 256)])
@pytest.mark.parametrize("N,Hq,Hkv", [(1, 2, 2), (1, 8, 1), (5, 2, 1), (26, 2, 2), (37, 1, 1), (60, 2, 2), (64, 2, 1), (60, 4, 1), (33, 8, 1)])
def test_shapes(N, Hq, Hkv, D, P):
    """Every row tiling, one to two row groups, both head dims; lengths that end inside a page and inside a block."""
    Case(N + Hq + D + P, 2, N, Hq, Hkv, D, P, [331, 97]).check()


@pytest.mark.parametrize("L", [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 127, 128, 129, 255, 511, 1000])
@pytest.mark.parametrize("P", [32, 128])
def test_lengths(L, P):
    Case(L + P, 1, 3, 2, 1, 128, P, [L]).check()
    Case(L + P, 3, 1, 4, 2, 64, P, [L, 0, 7]).check()
    Case(L + P, 2, 20, 2, 2, 128, P, [L, 19]).check()


@pytest.mark.parametrize("workgroups", [1, 2, 3, 7, 40, 256, 1000, 4096])
@pytest.mark.parametrize("N,Hq,Hkv,D", [(26, 3, 3, 128), (60, 4, 1, 64), (64, 8, 1, 128)])
def test_any_cut_of_the_keys(N, Hq, Hkv, D, workgroups):
    Case(9, 3, N, Hq, Hkv, D, 32, [700, 33, 0], [N, 1, N // 2]).check(workgroups=workgroups)


def test_ragged_batches():
    """More sequences than a wavefront has lanes; trees that fill none, some or all row groups; padded sequences without nodes."""
    rng = np.random.default_rng(3)
    for B, N, Hq, Hkv, D, P, top in ((70, 1, 2, 1, 64, 32, 90), (130, 3, 1, 1, 128, 32, 60), (6, 64, 8, 1, 64, 32, 400), (9, 20, 16, 1, 128, 64, 130)):
        kv_len = rng.integers(0, top, B)
        kv_len[rng.integers(B)] = 0
        nodes = rng.integers(0, N + 1, B)
        got = Case(B, B, N, Hq, Hkv, D, P, kv_len, nodes).check(max_kv_len=(-(-int(kv_len.max()) // P) + 1) * P)   # all the table holds
        for b in range(B):
            assert np.all(got[b, nodes[b]:] == 0)


@pytest.mark.parametrize("B,N,Hq,Hkv,D,P,top", [
    (130, 1, 16, 8, 128, 32, 100), (130, 1, 16, 8, 64, 128, 300), (520, 1, 2, 2, 64, 32, 33), (100, 9, 16, 8, 128, 32, 90), (100, 9, 16, 8, 64, 64, 200),
    (50, 20, 16, 8, 128, 64, 400), (50, 20, 16, 8, 64, 32, 400), (40, 20, 32, 8, 128, 32, 300), (40, 20, 32, 8, 64, 256, 300), (12, 60, 32, 8, 128, 32, 200)])
def test_as_many_rows_as_the_device_has_wavefronts(B, N, Hq, Hkv, D, P, top):
    """Wavefronts then have rows for themselves: one slab a workgroup, or four; sequences of no node, of no token, of all."""
    rng = np.random.default_rng(B + N + D)
    kv_len, nodes = rng.integers(0, top + 1, B), rng.integers(0, N + 1, B)
    kv_len[:4], nodes[:4] = (0, top, 0, top), (N, N, 0, 0)
    got = Case(B, B, N, Hq, Hkv, D, P, kv_len, nodes).check()
    for b in range(B):
        assert np.all(got[b, nodes[b]:] == 0)


@pytest.mark.parametrize("B,N,Hq,Hkv,D,top", [
    (130, 1, 8, 8, 128, 400), (130, 2, 8, 8, 64, 700), (100, 9, 16, 8, 128, 600), (50, 20, 16, 8, 64, 600), (2, 60, 4, 1, 128, 700), (3, 60, 4, 1, 64, 900), (1, 60, 4, 2, 128, 3000),
    (2, 26, 4, 4, 64, 2600), (11, 60, 16, 8, 64, 500), (11, 60, 16, 8, 128, 1300)])
def test_keys_of_a_slab_between_two_wavefronts_four_and_eight(B, N, Hq, Hkv, D, top):
    rng = np.random.default_rng(B + N + D + top)
    kv_len, nodes = rng.integers(0, top + 1, B) // (1 + rng.integers(0, 8, B)), rng.integers(0, N + 1, B)
    kv_len[0], nodes[0] = top, N
    case = Case(B + top, B, N, Hq, Hkv, D, 32, kv_len, nodes)
    case.check()
    case.check(workgroups=1500)


@pytest.mark.parametrize("workgroups", [0, 1, 9, 1000, 4096])
@pytest.mark.parametrize("D", [128, 64])
def test_long_ones_among_many(workgroups, D):
    """Four slabs a workgroup, and a sequence that is cut: by itself, or as the call asks."""
    rng, B = np.random.default_rng(workgroups + D), 34 if D == 128 else 66
    kv_len, nodes = rng.integers(0, 80, B), rng.integers(0, 21, B)
    kv_len[5], nodes[5], nodes[6] = 3500, 20, 0
    Case(workgroups + D, B, 20, 32, 8, D, 64, kv_len, nodes).check(workgroups=workgroups)


@pytest.mark.parametrize("workgroups", [0, 1, 33, 4096])
@pytest.mark.parametrize("N,Hq,D,L", [(33, 1, 128, 160), (60, 4, 128, 130), (60, 4, 64, 250), (64, 1, 64, 0), (60, 4, 64, 251), (33, 1, 128, 161)])
def test_few_keys_of_a_tree(N, Hq, D, L, workgroups):
    """Up to where a wavefront takes all keys of its rows, and one more."""
    Case(N + D + L, 2, N, Hq, 1, D, 32, [L, L // 2], [N, N // 2]).check(workgroups=workgroups)


def test_lengths_and_counts_outside_their_ranges_are_clamped():
    c = Case(4, 4, 6, 2, 1, 128, 32, [100, 60, 30, 5])
    c.kv_len = np.array([10 ** 6, -7, 30, 2 ** 31 - 1], np.int32)
    c.n_nodes = np.array([6, 100, -1, 2 ** 31 - 1], np.int32)
    c.table[0, :] = c.table[0, 0]
    c.table[3, :] = c.table[0, 0]
    got = c.run(max_kv_len=50).double().cpu().numpy()
    want, bound = c.reference(max_kv_len=50)
    _compare(got, want, bound)
    assert np.all(got[2] == 0)


def test_rows_that_see_nothing_are_zero():
    c = Case(5, 3, 7, 4, 2, 128, 32, [0, 0, 20])
    c.mask[0, 2] = 0
    c.mask[1, :] = 0
    c.mask[2, 3] = 0                                   # still sees the prefix
    c.vt[0, 6] = float("inf")                          # and a value that only node 6 sees
    got = c.check()
    assert np.all(got[0, 2] == 0) and np.all(got[1] == 0) and np.any(got[2, 3] != 0)


@pytest.mark.parametrize("D,N,Hq", [(128, 40, 1), (64, 40, 1), (128, 60, 4), (64, 60, 4), (64, 3, 2), (128, 3, 2)])
@pytest.mark.parametrize("what", ["nan", "inf", "-inf", "all"])
def test_what_a_row_does_not_see_has_no_part(D, N, Hq, what):
    """NaN and infinity in tree keys and values of nodes that some rows see, in rows of unused nodes, in query rows, and in unused
    places of the pages (codes of NaN and any scale, which the case's random bytes hold anyway)."""
    c = Case(6, 2, N, Hq, 1, D, 32, [70, 13], [N, N - 2])
    bad = {"nan": [np.nan], "inf": [np.inf], "-inf": [-np.inf], "all": [np.nan, np.inf, -np.inf]}[what]
    for i, x in enumerate(bad * 2):
        c.vt[0, (N - 1 - 3 * i) % N, 0, (5 * i + 1) % D] = x
        c.vt[1, 1 + i % max(1, N - 4), 0, D - 1 - i] = x
    c.kt[0, N - 1, 0, 3] = bad[0]
    c.kt[1, N - 2:] = float("nan")                     # unused
    c.vt[1, N - 2:] = float("inf")
    c.q[0, 1, 0, 7] = float("nan")
    c.q[1, N - 1] = float("nan")
    c.check()


@pytest.mark.parametrize("N,D", [(5, 128), (20, 128), (60, 64), (1, 64)])
def test_nan_in_the_prefix_reaches_every_row(N, D):
    """One code of V makes one channel NaN, one of K every channel."""
    c = Case(7, 1, N, 2, 1, D, 64, [75])
    p, page = paged_fp8.Fp8Pages(c.raw, D, 64), c.raw[c.table[0, 0]]
    at = p.places("v", 41)[0][37]
    kept, page[0, at] = page[0, at], 0xff
    got = c.check()
    assert np.all(np.isnan(got[0, :, :, 37])) and np.isnan(got).sum() == N * 2
    page[0, at] = kept
    page[0, p.places("k", 63)[0][3]] = 0x7f
    assert np.all(np.isnan(c.check()))


def test_positions_on_bad_pages_are_left_out():
    for P, entry in ((32, 1), (32, 4), (64, 0), (128, 1)):
        for bad in (-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1):
            c = Case(8, 1, 9, 2, 1, 128, P, [150])
            c.table[0, entry] = bad
            c.check()
    c = Case(8, 2, 9, 2, 1, 64, 32, [150, 40])
    c.table[0, :] = -1                                 # none of a sequence's prefix is there
    c.check()


@pytest.mark.parametrize("spread", [1.0, 64.0, 2.0 ** 20])
@pytest.mark.parametrize("scale", [0.0, 0.3, -0.2])
def test_scores_of_any_size(spread, scale):
    """From flat to one-hot weights, and a softmax scale below zero."""
    Case(10, 1, 20, 2, 1, 128, 32, [600], spread=spread).check(scale=scale)
    Case(10, 1, 3, 2, 1, 64, 32, [600], spread=spread).check(scale=scale)


@pytest.mark.parametrize("s", [10, 246])
def test_scales_at_their_ends(s):
    """The smallest scale, whose smallest element is the smallest normal bf16, and the largest, whose elements up to 1 times a weight stay finite."""
    c = Case(16, 1, 3, 2, 1, 128, 32, [40])
    p = paged_fp8.Fp8Pages(c.raw, 128, 32)
    rng = np.random.default_rng(s)
    for t in range(40):
        page = c.raw[c.table[0, t // 32], 0]
        at, at_scale = p.places("v", t % 32)
        page[at] = rng.integers(0, 0x39, 128) | (rng.integers(0, 2, 128) * 128)
        page[at_scale] = s
    if s == 246:
        c.vt[:] = 0
    else:
        c.mask[:] = 0                                 # only the prefix
    got = c.check()
    assert np.abs(got).max() > 0


def test_equal_keys_average_their_values():
    c = Case(11, 1, 1, 1, 1, 64, 32, [64])
    c.q[:] = 0
    got = c.check()
    p = paged_fp8.Fp8Pages(c.raw, 64, 32)
    v = p.get_many("v", [int(c.table[0, t // 32]) * 32 + t % 32 for t in range(64)])[:, 0]
    assert np.abs(got[0, 0, 0] - (v.sum(0) + c.vt[0, 0, 0].double().numpy()) / 65).max() < 1e-5


def test_a_sink_and_a_long_flat_tail():
    """One key takes half of the weight, 30000 others share the rest: what each of them adds is kept."""
    c = Case(17, 1, 1, 1, 1, 128, 256, [30000], spread=1e-3)
    c.q[:] = 0
    c.q[0, 0, 0, 0] = 8.0
    c.kt[:] = 0
    c.kt[0, 0, 0, 0] = float(np.log(30000.0) / 8 * np.sqrt(128))
    c.check()


def test_shared_pages_and_page_strides():
    """Two sequences on one prefix; pools of three layers interleaved page by page."""
    c = Case(12, 2, 8, 4, 2, 128, 32, [90, 90])
    c.table[1] = c.table[0]
    pools = torch.randint(0, 256, (c.raw.shape[0], 3, *c.raw.shape[1:]), dtype=torch.uint8, device=DEV)
    pools[:, 1] = torch.from_numpy(c.raw).to(DEV)
    got = c.run(pages=pools[:, 1]).double().cpu().numpy()
    _compare(got, *c.reference())
    assert np.array_equal(c.run().double().cpu().numpy(), got)


def test_bf16_output_is_the_fp32_one_rounded_and_runs_repeat():
    c = Case(13, 3, 26, 8, 4, 128, 64, [900, 17, 400])
    a, b = c.run(), c.run(torch.bfloat16)
    assert torch.equal(a.to(torch.bfloat16), b) and torch.equal(a, c.run(poison=False))


def test_pool_past_32_bits_of_bytes():
    """A sequence whose pages lie on both sides of 4 GB."""
    c = Case(14, 1, 5, 8, 8, 128, 256, [700])
    per = c.raw[0].nbytes
    n_pages = (1 << 32) // per + 9
    pool = torch.zeros((n_pages, *c.raw.shape[1:]), dtype=torch.uint8, device=DEV)
    used = c.table[0, :3].copy()
    far = np.array([1, n_pages - 1, n_pages - 4], np.int32)
    for u, f in zip(used, far):
        pool[int(f)] = torch.from_numpy(c.raw[u]).to(DEV)
    want, bound = c.reference()
    c.table[0, :3] = far
    _compare(c.run(pages=pool).double().cpu().numpy(), want, bound)


def test_long_prefix_single_token():
    c = Case(15, 1, 1, 8, 1, 128, 256, [40000])
    c.check()
    c.check(workgroups=1)


@pytest.mark.parametrize("B,N,Hq,Hkv,D,P,top", [(24, 64, 16, 8, 128, 64, 1500), (24, 40, 16, 8, 128, 32, 1300), (20, 64, 32, 8, 64, 32, 2300), (70, 33, 8, 4, 128, 32, 1100),
                                                (17, 32, 16, 8, 128, 128, 4100), (20, 26, 16, 16, 128, 32, 1400), (20, 17, 16, 16, 64, 64, 1400)])
def test_more_units_than_workgroups(B, N, Hq, Hkv, D, P, top):
    """Row groups of all heads and sequences in equal windows: units that start and end in any place of one, whole ones, ones without
    nodes, last groups of a few rows. Twice the same bits."""
    rng = np.random.default_rng(B + top)
    kv_len, nodes = rng.integers(0, top // 2, B), rng.integers(1, N + 1, B)
    kv_len[:3], kv_len[3:6] = top, [0, 1, 33]
    nodes[:2], nodes[-2:] = N, [0, 1]
    if B == 17:
        kv_len[:], nodes[:] = top - np.arange(B), N
    c = Case(B, B, N, Hq, Hkv, D, P, kv_len, nodes)
    got = c.check()
    for b in range(B):
        assert np.all(got[b, nodes[b]:] == 0)
    assert torch.equal(c.run(), c.run(poison=False))


@pytest.mark.parametrize("D,P", [(64, 32), (128, 32), (64, 64), (128, 256)])
@pytest.mark.parametrize("N,Hq,Hkv", [(1, 2, 2), (1, 16, 1), (3, 4, 1)])
@pytest.mark.parametrize("workgroups", [0, 3, 300])
def test_few_rows_of_long_sequences(N, Hq, Hkv, D, P, workgroups):
    """16 rows or less on eight wavefronts, whole and cut, beside sequences of a few tokens and of none."""
    c = Case(N + D + P, 4, N, Hq, Hkv, D, P, [3000, 1601, 5, 0])
    c.table[0, 1600 // P] = -1
    c.check(workgroups=workgroups)


@pytest.mark.parametrize("B,N,Hq,Hkv,D,P,top,workgroups", [(24, 64, 16, 8, 128, 64, 1300, 0), (20, 40, 16, 8, 64, 32, 2300, 0), (2, 60, 2, 2, 128, 32, 3000, 0), (3, 1, 8, 2, 64, 32, 6000, 0),
                                                           (5, 1, 8, 8, 128, 32, 300, 0), (2, 33, 4, 2, 128, 32, 700, 3), (2, 5, 4, 2, 64, 32, 700, 4096)])
def test_writes_stay_inside_the_workspace(B, N, Hq, Hkv, D, P, top, workgroups):
    rng = np.random.default_rng(top)
    kv_len, nodes = rng.integers(top // 2, top, B), rng.integers(1, N + 1, B)
    kv_len[0], nodes[0] = top, N
    c = Case(B, B, N, Hq, Hkv, D, P, kv_len, nodes)
    assert torch.equal(c.run(workgroups=workgroups, guard=1 << 20), c.run(workgroups=workgroups, guard=1 << 20, poison=False))


@pytest.mark.parametrize("B,N,Hq,Hkv,P,top", [(3, 60, 2, 2, 32, 500), (20, 64, 16, 16, 64, 450), (2, 33, 8, 2, 32, 520)])
def test_two_slabs_on_four_wavefronts(B, N, Hq, Hkv, P, top):
    """More than 32 rows, D = 128, short sequences: whole units of few blocks, last groups of one slab, forced cuts."""
    rng = np.random.default_rng(top)
    kv_len, nodes = rng.integers(0, top, B), rng.integers(0, N + 1, B)
    kv_len[0], nodes[0] = top, N
    c = Case(top, B, N, Hq, Hkv, 128, P, kv_len, nodes)
    c.check()
    c.check(workgroups=5)
