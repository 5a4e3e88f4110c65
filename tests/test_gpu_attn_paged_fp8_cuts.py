"""GPU parity of the tree attention over the paged 8-bit cache in every kernel that a call can be dealt to (rows of a wavefront, slabs and wavefronts of a workgroup, split or
not) and in every way that its keys are cut: units whole because no length allows a cut, whole because of the lengths at hand, in equal pieces, and on one line of windows. What a call was cut into is
read from the workspace. That the list has every kernel is tested on the host, in test_paged_fp8_plan.py."""
import numpy as np
import pytest
import torch

import _paged_reference
import paper_2408_15562_amd as fspad
from oracle import paged_fp8
from test_gpu_attn_paged_fp8 import Case, DEV, _bf16, _compare
from workloads import gen_trees

pytestmark = pytest.mark.gpu

# batch, nodes, query heads, kv heads, head dim, page tokens; longest sequence, how many others are as long, up to how many tokens the rest has, from how many nodes on most
# have; bound on the lengths (0: the longest); rows of a wavefront, slabs, wavefronts, split; how the call is cut
CASES = [
    # 64 rows a wavefront (D = 64), eight and four wavefronts
    ((5, 60, 32, 8, 64, 32), (2400, 1, 700), 0, (64, 1, 8, 1), "pieces"),
    ((16, 60, 16, 4, 64, 64), (14000, 0, 300, 45), 0, (64, 1, 8, 1), "windows"),
    ((5, 60, 32, 8, 64, 32), (1200, 1, 700), 2400, (64, 1, 8, 1), "whole"),
    ((9, 60, 32, 8, 64, 32), (2400, 1, 300), 0, (64, 1, 4, 1), "pieces"),
    ((70, 33, 16, 4, 64, 32), (3200, 4, 200), 0, (64, 1, 4, 1), "windows"),
    ((9, 60, 32, 8, 64, 128), (900, 2, 700), 2400, (64, 1, 4, 1), "whole"),
    # two slabs of 32 rows (D = 128) on eight and on four
    ((5, 60, 32, 8, 128, 32), (2400, 1, 700), 0, (32, 2, 8, 1), "pieces"),
    ((11, 60, 32, 8, 128, 64), (2400, 2, 900, 45), 0, (32, 2, 8, 1), "windows"),
    ((70, 33, 8, 2, 128, 32), (2600, 3, 200, 25), 0, (32, 2, 8, 1), "windows"),
    ((5, 60, 32, 8, 128, 32), (900, 1, 700), 2400, (32, 2, 8, 1), "whole"),
    ((20, 64, 16, 16, 128, 64), (450, 5, 300), 0, (32, 2, 4, 1), "uncut"),
    # four slabs of their own
    ((70, 20, 32, 8, 128, 32), (3200, 3, 200), 0, (32, 4, 4, 0), "windows"),
    ((66, 60, 16, 4, 128, 256), (3300, 2, 300), 0, (32, 4, 4, 0), "windows"),
    ((66, 60, 16, 4, 128, 32), (1500, 2, 300), 4000, (32, 4, 4, 0), "whole"),
    ((12, 60, 32, 8, 128, 32), (3200, 1, 100), 0, (32, 4, 4, 0), "pieces"),
    ((100, 20, 32, 8, 64, 32), (3200, 3, 100), 0, (32, 4, 4, 0), "windows"),
    ((70, 40, 32, 8, 64, 64), (3300, 2, 100), 0, (32, 4, 4, 0), "windows"),
    ((20, 60, 32, 8, 64, 32), (1000, 2, 300), 0, (32, 4, 4, 0), "uncut"),
    # one slab of 32 rows: four wavefronts, eight, two, one
    ((100, 20, 8, 8, 128, 32), (3200, 3, 200), 0, (32, 1, 4, 1), "windows"),
    ((100, 20, 8, 8, 64, 32), (3200, 3, 200), 0, (32, 1, 4, 1), "windows"),
    ((4, 60, 16, 2, 128, 32), (6000, 0, 900), 0, (32, 1, 8, 1), "pieces"),
    ((4, 60, 16, 2, 64, 32), (6000, 0, 900), 0, (32, 1, 8, 1), "pieces"),
    ((12, 20, 16, 16, 128, 32), (8300, 1, 300), 0, (32, 1, 8, 1), "pieces"),
    ((50, 20, 16, 8, 128, 64), (400, 9, 200), 0, (32, 1, 2, 1), "uncut"),
    ((50, 20, 16, 8, 64, 64), (420, 9, 200), 0, (32, 1, 2, 1), "uncut"),
    ((2, 60, 4, 1, 128, 32), (100, 0, 50), 0, (32, 1, 1, 0), "uncut"),
    ((2, 60, 4, 1, 64, 32), (100, 0, 50), 0, (32, 1, 1, 0), "uncut"),
    # 16 rows
    ((130, 1, 16, 8, 128, 32), (100, 9, 60), 0, (16, 1, 1, 0), "uncut"),
    ((130, 1, 16, 8, 64, 32), (100, 9, 60), 0, (16, 1, 1, 0), "uncut"),
    ((130, 1, 8, 8, 128, 32), (400, 9, 300), 0, (16, 1, 2, 1), "uncut"),
    ((130, 2, 8, 8, 64, 32), (400, 9, 300), 0, (16, 1, 2, 1), "uncut"),
    ((70, 1, 8, 4, 128, 32), (6000, 1, 300), 0, (16, 1, 4, 1), "pieces"),
    ((70, 1, 8, 4, 64, 64), (6000, 1, 300), 0, (16, 1, 4, 1), "pieces"),
    ((3, 2, 8, 2, 128, 32), (4000, 1, 300), 0, (16, 1, 8, 1), "pieces"),
    ((3, 2, 8, 2, 64, 256), (4000, 1, 300), 0, (16, 1, 8, 1), "pieces"),
]
IDS = [f"{'x'.join(map(str, dealt))}-{how}-{'_'.join(map(str, shape))}" for shape, _, _, dealt, how in CASES]


def sequences(shape, lengths):
    """Lengths and nodes: empty sequences, trees of no node, of one and of all, last groups of one row, of one slab and of more."""
    (B, N, Hq, Hkv, *_), (top, more, short, *least) = shape, lengths
    rng = np.random.default_rng(B + N + top)
    kv_len, nodes = rng.integers(0, short + 1, B), rng.integers(least[0] if least else 0, N + 1, B)
    at = rng.permutation(B)[:more + 1]
    kv_len[at], nodes[at[0]] = top, N
    for i, n in zip([b for b in range(B) if b != at[0]], (0, 1, -(-64 * Hkv // Hq), N)):   # (the third one: rows of one group, or a few more)
        nodes[i] = min(n, N)
    if B > 8:
        kv_len[[b for b in range(B) if b not in at][:2]] = 0, 1
    return kv_len.astype(np.int32), nodes.astype(np.int32)


class Quick(Case):
    """Case with elements of 1/8 to 4 at random instead of rounded normal ones: many tokens at once. What is not there is random bytes all the same."""

    def __init__(self, seed, B, N, Hq, Hkv, D, P, kv_len, n_nodes):
        rng = np.random.default_rng(seed)
        self.shape, self.P, self.kv_len, self.n_nodes = (B, N, Hq, Hkv, D), P, kv_len, n_nodes
        held = -(-kv_len // P)
        width, n_pages = int(held.max()) + 1, int(held.sum()) + 2
        order, at = rng.permutation(n_pages), 0
        self.table = rng.integers(-3, 2 * n_pages, (B, width)).astype(np.int32)
        junk = rng.integers(0, 256, (n_pages, Hkv, paged_fp8.page_head_bytes(D, P)), dtype=np.uint8)
        raw = rng.integers(4 << 3, 9 << 3, junk.shape, dtype=np.uint8) | (junk & 128)
        raw[:, :, 2 * P * D:] = rng.integers(126, 129, (n_pages, Hkv, 16))
        raw[order[int(held.sum()):]] = junk[order[int(held.sum()):]]
        p = paged_fp8.Fp8Pages(raw, D, P)
        for b in range(B):
            self.table[b, :held[b]] = order[at:at + held[b]]
            at += held[b]
            if kv_len[b] % P:
                page, fill = order[at - 1], int(kv_len[b] % P)
                for w in "kv":
                    there = [p.places(w, t) for t in range(P)]
                    behind = np.concatenate([there[t][0] for t in range(fill, P)] + [[there[t][1] for t in range(-(-fill // 32) * 32, P, 32)]]).astype(int)
                    raw[page][:, behind] = junk[page][:, behind]
        self.raw = raw
        self.q, self.kt, self.vt = (_bf16(rng.standard_normal(s)) for s in ((B, N, Hq, D), (B, N, Hkv, D), (B, N, Hkv, D)))
        parent, _ = gen_trees(seed, B, N, 6, min(10, max(1, N - 1)), n_nodes=np.maximum(n_nodes, 1))
        self.mask = fspad.fspad_tree_build_mask(parent, np.maximum(n_nodes, 1))

    def reference(self, device=DEV):
        D, f = self.shape[4], lambda t: t.double().numpy()  # noqa: E731
        return _paged_reference.tree_attn(f(self.q), f(self.kt), f(self.vt), paged_fp8.Fp8Pages(self.raw, D, self.P), self.table, self.kv_len, self.n_nodes, self.mask, 1 << 30,
                                          device=device)

    def cut(self, bound, workgroups=0):
        """The output, and the pieces of each unit as the workspace has them (0: whole, below zero: of windows)."""
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
        q, kt, vt, pages, table = self.q.to(DEV), self.kt.to(DEV), self.vt.to(DEV), dev(self.raw), dev(self.table)
        if bound > self.table.shape[1] * self.P:   # (a wider table, whose other entries are junk)
            wide = np.full((len(self.table), -(-bound // self.P)), 1 << 30, np.int32)
            wide[:, :self.table.shape[1]] = self.table
            table = dev(wide)
        desc = fspad.make_paged_desc(q, kt, pages, table, bound, torch.float32, 0.0, workgroups, fp8=True)
        ws = torch.full((fspad.fspad_tree_attn_paged_byte_workspace_bytes(desc),), 0xFF, dtype=torch.uint8, device=DEV)
        out = torch.full(q.shape, float("nan"), dtype=torch.float32, device=DEV)
        fspad.fspad_tree_attn_paged_byte(q, kt, vt, pages, table, dev(self.kv_len), dev(self.n_nodes), dev(self.mask.view(np.int64)), out=out, workspace=ws, desc=desc)
        torch.cuda.synchronize()
        return out.double().cpu().numpy(), lambda units: ws[:8 * units].cpu().numpy().view(np.int32).reshape(units, 2)[:, 1]


@pytest.mark.parametrize("shape,lengths,bound,dealt,how", CASES, ids=IDS)
def test_every_kernel_and_cut(shape, lengths, bound, dealt, how):
    B, N, Hq, Hkv, D, P = shape
    kv_len, nodes = sequences(shape, lengths)
    c = Quick(B + D + lengths[0], *shape, kv_len, nodes)
    got, pieces = c.cut(bound or lengths[0])
    want, off = c.reference()
    _compare(got, want, off)
    for b in range(B):
        assert np.all(got[b, nodes[b]:] == 0)
    pieces = pieces(B * Hkv * -(-N * (Hq // Hkv) // (dealt[0] * dealt[1])))
    assert not np.any(pieces == -1)                      # (each unit's are written down)
    assert {"uncut": not pieces.any(), "whole": not pieces.any(), "pieces": pieces.min() == 0 and pieces.max() > 1, "windows": pieces.min() < -1 and pieces.max() == 0}[how]
    again, _ = c.cut(bound or lengths[0])
    assert np.array_equal(got, again)
    forced, pieces = c.cut(bound or lengths[0], workgroups=300)   # the same kernel, cut as the call asks
    _compare(forced, want, off)
