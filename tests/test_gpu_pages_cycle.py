"""Shared pages and the paged caches together, as a server makes the calls that answers each prompt several times: prompts get pages and are
stored, are forked, every branch goes its own way (attention, new pages, stores), some end, the pool is compacted. In 8-bit pages and in 4-bit ones,
two layers interleaved in one pool; every step against the oracle; then a step of all of it captured into a graph, and calls on two streams at once."""
import os
import re

import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import paged, paged_fp8, pages

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def _np(t):
    return t.cpu().numpy()


class Server:
    """State of a server on the device, and the same in the oracle's hands."""

    def __init__(self, fp8, B, N, Hq, Hkv, D, P, width, n_pages, seed):
        self.fp8, self.shape, self.P, self.width, self.rng = fp8, (B, N, Hq, Hkv, D), P, width, np.random.default_rng(seed)
        per = paged_fp8.page_head_bytes(D, P) if fp8 else paged.page_head_bytes(D, P)
        self.pool = torch.from_numpy(self.rng.integers(0, 256, (n_pages, 2, Hkv, per), dtype=np.uint8)).to(DEV)   # pages of two layers
        self.table, self.kv_len = torch.full((B, width), -1, dtype=torch.int32, device=DEV), _dev(np.zeros(B))
        self.free, self.n_free, self.shared = _dev(self.rng.permutation(n_pages)), _dev([n_pages]), _dev(np.zeros(n_pages))
        self.host = dict(table=_np(self.table).astype(np.int64), kv_len=np.zeros(B, np.int64), free=_np(self.free).astype(np.int64), n_free=np.array([n_pages]),
                         shared=np.zeros(n_pages, np.int64))
        self.ref = [self._pages(layer) for layer in range(2)]
        if fp8:
            self.attn, self.store = fspad.fspad_tree_attn_paged_byte, fspad.fspad_kv_store_paged_byte
        else:
            self.attn, self.store = fspad.fspad_tree_attn_paged, fspad.fspad_kv_store_paged

    def _pages(self, layer):
        cls = paged_fp8.Fp8Pages if self.fp8 else paged.Pages
        return cls(_np(self.pool[:, layer]).copy(), self.shape[4], self.P)

    def same_state(self):
        torch.cuda.synchronize()
        for name, want in self.host.items():
            assert np.array_equal(_np(getattr(self, name)), want), name
        holders = np.zeros(len(self.host["free"]), int)
        for b, n in enumerate(self.host["kv_len"]):
            np.add.at(holders, self.host["table"][b, :-(-n // self.P)], 1)
        top = int(self.host["n_free"][0])
        assert sorted([*self.host["free"][:top], *np.flatnonzero(holders)]) == list(range(len(holders)))
        assert np.array_equal(self.host["shared"], np.maximum(holders - 1, 0))

    def grow(self, n_new):
        """Pages and slots for new tokens, which are stored in both layers."""
        h, Hkv, D = self.host, self.shape[3], self.shape[4]
        most = max(1, int(max(n_new)))
        slots, *_ = fspad.fspad_page_map(self.kv_len, _dev(n_new), self.table, self.free, self.n_free, self.P, max_new=most,
                                         outputs=(_dev(np.zeros((len(n_new), most))), self.kv_len, self.n_free, _dev(np.zeros(len(n_new)))))
        want, h["kv_len"], h["n_free"], granted, h["table"], h["free"] = paged.page_map(h["kv_len"], n_new, h["table"], h["free"], h["n_free"], self.P, max_new=most)
        assert np.array_equal(_np(slots), want)
        flat = want.reshape(-1)
        for layer in range(2):
            k, v = (torch.from_numpy(self.rng.standard_normal((flat.size, Hkv, D)).astype(np.float32)).to(torch.bfloat16) for _ in range(2))
            self.store(k.to(DEV), v.to(DEV), slots.view(-1), self.pool[:, layer])
            if self.fp8:
                self.ref[layer].store("k", k.double().numpy(), flat)
                self.ref[layer].store("v", v.double().numpy(), flat)
            else:
                for r in np.flatnonzero(flat >= 0):
                    for g in range(Hkv):
                        self.ref[layer].put("k", int(flat[r]), g, k[r, g].double().numpy())
                        self.ref[layer].put("v", int(flat[r]), g, v[r, g].double().numpy())
        self.same_state()
        return granted

    def fork(self, src, dst, n_tokens=None):
        h, F = self.host, len(src)
        out = [_dev(np.zeros(F)) for _ in range(3)]
        got = fspad.fspad_page_fork(_dev(src), _dev(dst), self.kv_len, self.table, self.free, self.n_free, self.shared, self.P,
                                    n_tokens=None if n_tokens is None else _dev(n_tokens), outputs=(out[0], out[1], self.kv_len, self.n_free, self.shared, out[2]))
        fspad.fspad_page_copy(got[0], got[1], self.pool)                       # both layers at once
        cs, cd, h["kv_len"], h["n_free"], h["shared"], granted, h["table"] = pages.fork(src, dst, h["kv_len"], h["table"], h["free"], h["n_free"], h["shared"], self.P, n_tokens)
        self._copied(cs, cd)
        assert np.array_equal(_np(got[5]), granted)
        return granted

    def release(self, ended):
        h = self.host
        fspad.fspad_page_release(_dev(ended), self.kv_len, self.table, self.free, self.n_free, self.shared, self.P, outputs=(self.kv_len, self.n_free, self.shared))
        h["kv_len"], h["n_free"], h["shared"], h["free"] = pages.release(ended, h["kv_len"], h["table"], h["free"], h["n_free"], h["shared"], self.P)
        self.same_state()

    def compact(self):
        h, n = self.host, len(self.host["free"])
        cs, cd = _dev(np.zeros(n // 2)), _dev(np.zeros(n // 2))
        fspad.fspad_page_compact(self.kv_len, self.table, self.free, self.n_free, self.shared, self.P, outputs=(cs, cd, self.table, self.free, self.shared))
        for layer in range(2):                                                 # each layer by itself
            fspad.fspad_page_copy(cs, cd, self.pool[:, layer])
        cs, cd, h["table"], h["free"], h["shared"] = pages.compact(h["kv_len"], h["table"], h["free"], h["n_free"], h["shared"], self.P)
        self._copied(cs, cd)
        held = {int(p) for b, m in enumerate(h["kv_len"]) for p in h["table"][b, :-(-m // self.P)]}
        assert held == set(range(n - int(h["n_free"][0])))

    def _copied(self, cs, cd):
        for ref in self.ref:
            ref.raw = pages.copy(ref.raw, cs, cd)
        self.same_state()

    def inputs(self):
        B, N, Hq, Hkv, D = self.shape
        q, kt, vt = (torch.from_numpy(self.rng.standard_normal(s).astype(np.float32)).to(torch.bfloat16) for s in ((B, N, Hq, D), (B, N, Hkv, D), (B, N, Hkv, D)))
        return q, kt, vt, np.tile((2 << np.arange(N, dtype=np.uint64)) - np.uint64(1), (B, 1))   # a chain of nodes

    def attend(self):
        B, N = self.shape[:2]
        q, kt, vt, mask = self.inputs()
        nodes = np.where(self.host["kv_len"] > 0, N, 0)
        for layer in range(2):
            out = self.attn(q.to(DEV), kt.to(DEV), vt.to(DEV), self.pool[:, layer], self.table, self.kv_len, _dev(nodes), _dev(mask.view(np.int64), torch.int64),
                            out_dtype=torch.float32)
            torch.cuda.synchronize()
            want, bound = paged.tree_attn(*(t.double().numpy() for t in (q, kt, vt)), self.ref[layer], self.host["table"], self.host["kv_len"], nodes, mask, 1 << 30)
            assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound)


@pytest.mark.parametrize("fp8,N,Hq,Hkv,D,P", [(True, 1, 4, 2, 128, 32), (True, 5, 4, 1, 64, 64), (False, 3, 2, 2, 128, 16)])
def test_answers_to_shared_prompts(fp8, N, Hq, Hkv, D, P):
    B = 7
    s = Server(fp8, B, N, Hq, Hkv, D, P, width=-(-260 // P), n_pages=5 * (-(-260 // P)), seed=P)
    s.grow([100, 3 * P, 0, 0, 0, 0, 0])                          # two prompts, one of whole pages
    assert s.fork([0, 0, 1], [2, 3, 4]).all()
    s.attend()
    for _ in range(3):                                           # branches apart
        s.grow(list(s.rng.integers(0, 12, 2)) + [7, 1, 9, 0, 0])
        s.attend()
    assert s.fork([2, 2, 0], [5, 6, 6], n_tokens=[40, int(s.host["kv_len"][2]), 5]).tolist() == [1, 1, 0]   # of a branch, in part and whole
    s.attend()
    s.release([1, 0, 1, 0, 0, 0, 0])                             # the prompt itself ends, its branches do not
    s.attend()
    s.compact()
    s.attend()
    s.grow([0, 5, 30, 2, 2, 2, 2])                               # a new sequence on released pages
    s.attend()
    s.release([0, 1, 1, 1, 1, 1, 1])
    s.compact()
    assert int(s.host["n_free"][0]) == len(s.host["free"])


def test_fork_refused_for_lack_of_pages_and_granted_later():
    s = Server(True, 4, 1, 2, 1, 128, 32, width=4, n_pages=6, seed=1)
    s.grow([100, 33, 0, 0])                                      # four pages and two
    assert s.fork([0, 1], [2, 3]).tolist() == [0, 0]
    s.release([0, 1, 0, 0])
    assert s.fork([0, 0], [2, 3]).tolist() == [1, 1] and int(s.host["n_free"][0]) == 0
    s.attend()


@pytest.mark.parametrize("fp8,P", [(True, 32), (False, 16)])
def test_a_captured_step_replays(fp8, P):
    """Fork of a sequence, copy, one token of attention on both, growth of the branch, store, end of the branch: captured once and replayed with eager
    work between; each replay does what the calls do eagerly from the same state."""
    Hq, Hkv, D, B, width = 4, 2, 128, 3, 8
    s = Server(fp8, B, 1, Hq, Hkv, D, P, width, n_pages=20, seed=3)
    s.grow([3 * P + 5, 0, 9])
    q, kt, vt, mask = s.inputs()
    q, kt, vt, mask, nodes = q.to(DEV), kt.to(DEV), vt.to(DEV), _dev(mask.view(np.int64), torch.int64), _dev([1, 1, 1])
    src, dst, ended, n_new = _dev([0]), _dev([1]), _dev([0, 1, 0]), _dev([1, 1, 0])
    cs, cd, granted, slots, ok = _dev([0]), _dev([0]), _dev([0]), _dev(np.zeros((B, 1))), _dev(np.zeros(B))
    out = torch.zeros((B, 1, Hq, D), device=DEV)
    k, v = (torch.randn((B, Hkv, D), device=DEV).to(torch.bfloat16) for _ in range(2))

    def step(run):
        kw = dict(prepare=True)
        return [c() if run else c for c in (
            fspad.fspad_page_fork(src, dst, s.kv_len, s.table, s.free, s.n_free, s.shared, P, outputs=(cs, cd, s.kv_len, s.n_free, s.shared, granted), **kw),
            fspad.fspad_page_copy(cs, cd, s.pool, **kw),
            s.attn(q, kt, vt, s.pool[:, 0], s.table, s.kv_len, nodes, mask, out=out, **kw),
            fspad.fspad_page_map(s.kv_len, n_new, s.table, s.free, s.n_free, P, max_new=1, outputs=(slots, s.kv_len, s.n_free, ok), **kw),
            s.store(k, v, slots.view(-1), s.pool[:, 0], **kw),
            fspad.fspad_page_release(ended, s.kv_len, s.table, s.free, s.n_free, s.shared, P, outputs=(s.kv_len, s.n_free, s.shared), **kw))]

    buffers = (s.pool, s.table, s.kv_len, s.free, s.n_free, s.shared, out, cs, cd, granted, slots)
    start = [b.clone() for b in buffers]
    eager = []
    for _ in range(4):
        step(True)
        torch.cuda.synchronize()
        eager.append([b.clone() for b in buffers])
    for b, x in zip(buffers, start):
        b.copy_(x)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        calls = step(False)
        for c in calls:
            c()
    for b, x in zip(buffers, start):
        b.copy_(x)
    for want in eager:
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(buffers, want):
            assert torch.equal(got, w)
        torch.randn(1 << 16, device=DEV).sum().item()            # eager work between
    assert int(granted) == 1 and int(cs) >= 0


def test_calls_on_two_streams_at_once():
    """Two servers, each on a stream of its own with workspaces of its own, interleaved call by call: what they get alone."""
    def make(seed):
        s = Server(True, 4, 3, 4, 2, 128, 32, width=10, n_pages=40, seed=seed)
        s.grow([200, 150, 0, 0])
        q, kt, vt, mask = s.inputs()
        return s, [q.to(DEV), kt.to(DEV), vt.to(DEV), _dev(mask.view(np.int64), torch.int64), _dev([3, 3, 3, 3])]

    def calls(s, x, ended, src, dst):
        f = fspad.fspad_page_fork(src, dst, s.kv_len, s.table, s.free, s.n_free, s.shared, 32, prepare=True)
        r = fspad.fspad_page_release(ended, f.result[2], s.table, s.free, f.result[3], f.result[4], 32, prepare=True)
        c = fspad.fspad_page_compact(r.result[0], s.table, s.free, r.result[1], r.result[2], 32, prepare=True)
        a = s.attn(x[0], x[1], x[2], s.pool[:, 0], c.result[2], r.result[0], x[4], x[3], prepare=True)
        return [f, fspad.fspad_page_copy(f.result[0], f.result[1], s.pool, prepare=True), r, c, fspad.fspad_page_copy(c.result[0], c.result[1], s.pool, prepare=True), a]

    args = _dev([0, 1, 0, 0]), _dev([0, 1]), _dev([2, 3])
    alone = []
    for seed in (5, 6):
        s, x = make(seed)
        alone.append([c() for c in calls(s, x, *args)])
        torch.cuda.synchronize()
        alone[-1] = [t.clone() for r in alone[-1] for t in (r if isinstance(r, tuple) else (r,))]
    streams, sides = [torch.cuda.Stream() for _ in range(2)], [make(seed) for seed in (5, 6)]
    torch.cuda.synchronize()
    made = []
    for stream, (s, x) in zip(streams, sides):
        with torch.cuda.stream(stream):
            made.append(calls(s, x, *args))
    torch.cuda.synchronize()
    got = [[], []]
    for i in range(len(made[0])):
        for side in range(2):
            got[side].append(made[side][i]())
    torch.cuda.synchronize()
    for side in range(2):
        flat = [t for r in got[side] for t in (r if isinstance(r, tuple) else (r,))]
        for a, b in zip(flat, alone[side]):
            assert torch.equal(a, b)


def test_the_documented_calls():
    """README's lines about shared pages, as they stand there."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        block = next(b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "fspad_page_fork" in b)
    s = Server(True, 4, 1, 2, 1, 128, 32, width=5, n_pages=14, seed=2)
    s.grow([101, 40, 0, 0])
    parts = re.split(r"(?m)^# ", block)
    ns = dict(torch=torch, fspad=fspad, i32=dict(dtype=torch.int32, device=DEV), n_pages=14, P=32, table=s.table, free=s.free, n_free=s.n_free, kv_len=s.kv_len, pages=s.pool)
    h = s.host
    exec(parts[0], ns)
    s.shared = ns["shared"]
    cs, cd, h["kv_len"], h["n_free"], h["shared"], granted, h["table"] = pages.fork([0, 0], [2, 3], h["kv_len"], h["table"], h["free"], h["n_free"], h["shared"], 32)
    s._copied(cs, cd)
    assert granted.all() and ns["granted"].tolist() == [1, 1]
    s.attend()
    exec("# " + parts[1], ns)
    h["kv_len"], h["n_free"], h["shared"], h["free"] = pages.release([0, 0, 1, 0], h["kv_len"], h["table"], h["free"], h["n_free"], h["shared"], 32)
    s.same_state()
    exec("# " + parts[2], ns)
    cs, cd, h["table"], h["free"], h["shared"] = pages.compact(h["kv_len"], h["table"], h["free"], h["n_free"], h["shared"], 32)
    s._copied(cs, cd)
    s.attend()
