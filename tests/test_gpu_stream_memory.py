"""Calls that go to another stream than the current one and take workspaces and outputs for themselves: the current stream's memory stays its own, before and behind
the call, and results are those of a call on the current stream."""
import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import paged_fp8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def _release(rng):
    B, P, width, n_pages = 16, 32, 1000, 20000
    table, kv_len = rng.permutation(n_pages)[:B * width].reshape(B, width), rng.integers(1, width * P, B)
    free = np.setdiff1d(np.arange(n_pages), [p for b in range(B) for p in table[b, :-(-kv_len[b] // P)]])
    stack = np.concatenate([free, np.full(n_pages - len(free), -1)])
    args = (_dev(rng.integers(0, 2, B)), _dev(kv_len), _dev(table))
    n_free, shared = _dev([len(free)]), _dev(np.zeros(n_pages))

    def call(free_pages, stream):
        return (*fspad.fspad_page_release(*args, free_pages, n_free, shared, P, stream=stream), free_pages)
    return lambda: _dev(stack), call, fspad.fspad_page_release_workspace_bytes(B, n_pages, width)


def _store(rng):
    Hkv, D, P, n_pages, rows = 2, 64, 32, 100, 2100
    slots = _dev(rng.permutation(n_pages * P)[:rows])
    k, v = (torch.randn((rows, Hkv, D), device=DEV).to(torch.bfloat16) for _ in range(2))

    def fresh():   # (scales of 2^-27: they grow)
        return torch.full((n_pages, Hkv, paged_fp8.page_head_bytes(D, P)), 100, dtype=torch.uint8, device=DEV)
    return fresh, lambda pages, stream: (fspad.fspad_kv_store_paged_byte(k, v, slots, pages, stream=stream),), 4 * n_pages * P


def _attention(rng):
    B, N, Hq, Hkv, D, P, width = 2, 3, 4, 2, 128, 32, 40
    codes, scales = rng.integers(0, 120, (B * width, Hkv, 2 * P * D), dtype=np.uint8), rng.integers(118, 128, (B * width, Hkv, 16), dtype=np.uint8)
    pages = torch.from_numpy(np.concatenate([codes, scales], 2)).to(DEV)
    table, kv_len, n_nodes = _dev(rng.permutation(B * width).reshape(B, width)), _dev([1000, 1200]), _dev([3, 2])
    q, kt, vt = (torch.randn((B, N, h, D), device=DEV).to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    mask = _dev(np.tile([1, 3, 5], (B, 1)), torch.int64)
    desc = fspad.make_paged_desc(q, kt, pages, table, out_dtype=torch.float32, workgroups=32, fp8=True)

    def call(_, stream):
        return fspad.fspad_tree_attn_paged_byte(q, kt, vt, pages, table, kv_len, n_nodes, mask, desc=desc, stream=stream),
    return lambda: None, call, fspad.fspad_tree_attn_paged_byte_workspace_bytes(desc)


def _topk(rng):   # (a call of the bf16 path)
    logits = torch.randn((6, 128256), device=DEV)
    return lambda: None, lambda _, stream: fspad.fspad_draft_topk(logits, 10, stream=stream), fspad.fspad_draft_topk_workspace_bytes(6, 128256, 10)


MAKERS = {"release": _release, "store": _store, "attention": _attention, "top-k": _topk}


class Busy:
    """Some milliseconds of work for a stream."""

    def __init__(self):
        self.x = torch.zeros(1 << 28, device=DEV)

    def __call__(self):
        for _ in range(12):
            self.x.add_(1.0)


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("name", MAKERS)
def test_memory_of_the_current_stream_stays_its_own(name, handle):
    fresh, call, workspace = MAKERS[name](np.random.default_rng(5))
    assert workspace > 0
    want = [t.clone() for t in call(fresh(), None)]
    side, busy, inputs = torch.cuda.Stream(), Busy(), [fresh() for _ in range(2)]
    stream = side.cuda_stream if handle else side
    sizes = sorted({workspace, *(t.numel() * t.element_size() for t in want)})
    torch.cuda.synchronize()
    # what the current stream is given behind the call, which waits for its own stream's other work
    with torch.cuda.stream(side):
        busy()
    got = call(inputs[0], stream)
    given = [torch.full((n,), 77, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(3)]
    torch.cuda.synchronize()
    assert all(bool((g == 77).all()) for g in given)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # what the current stream had before the call, and still reads
    del given, got
    had = [torch.full((n,), 78, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(3)]
    torch.cuda.synchronize()
    busy()
    read = [h.clone() for h in had]
    del had
    got = call(inputs[1], stream)
    torch.cuda.synchronize()
    assert all(bool((r == 78).all()) for r in read)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
