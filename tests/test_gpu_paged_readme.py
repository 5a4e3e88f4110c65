"""README's step over the paged cache, as it stands there: run, captured into a graph and replayed, against the oracle's page map."""
import os
import re

import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import paged
from workloads import gen_draft_tokens, gen_logits, gen_trees

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def _example():
    """The example's set-up with the prompts, and its step."""
    with open(README) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    block = next(b for b in blocks if "fspad_tree_attn_paged" in b)
    before, step = block.split("# a step")
    return before, "#" + step


def test_the_documented_step_replays():
    B, Nmax, Hq, Hkv, D, V = 3, 26, 4, 2, 128, 500
    rng = np.random.default_rng(1)
    bf16 = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DEV, torch.bfloat16)  # noqa: E731
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV, torch.int32)  # noqa: E731
    new = np.array([130, 0, 61])
    parent, nodes = gen_trees(1, B, Nmax, 6, 10)
    ns = dict(torch=torch, fspad=fspad, B=B, Nmax=Nmax, Hkv=Hkv, D=D, n_new=i32(new), k=bf16(int(new.sum()), Hkv, D), v=bf16(int(new.sum()), Hkv, D),
              q=bf16(B, Nmax, Hq, D), k_tree=bf16(B, Nmax, Hkv, D), v_tree=bf16(B, Nmax, Hkv, D), n_nodes=i32(nodes), parent=i32(parent),
              anc_mask=torch.from_numpy(fspad.fspad_tree_build_mask(parent, nodes).view(np.int64)).to(DEV),
              logits=torch.zeros((B, Nmax, V), device=DEV), tokens=i32(np.zeros((B, Nmax))))

    def fill(seed):
        logits = gen_logits(seed, B, Nmax, V, peak=3.0)
        ns["logits"].copy_(torch.from_numpy(logits))
        ns["tokens"].copy_(i32(gen_draft_tokens(seed, logits, parent, nodes, noise=0.2)))
        ns["k_tree"].copy_(bf16(B, Nmax, Hkv, D))
        torch.cuda.synchronize()

    before, step = _example()
    exec(before, ns)
    torch.cuda.synchronize()
    assert ns["kv_len"].tolist() == new.tolist() and ns["granted"].tolist() == [1, 1, 1]
    fill(0)
    exec(step, ns)
    torch.cuda.synchronize()
    names = ("kv_len", "n_free", "granted", "table", "free")
    now = lambda: [ns[n].cpu().numpy() for n in names]  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    state = now()
    with torch.cuda.graph(graph):
        exec(step, ns)
    torch.cuda.synchronize()
    for seed in range(1, 5):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        path, taken = ns["path"].cpu().numpy(), ns["path_len"].cpu().numpy()
        assert taken.min() >= 1
        slots, *want = paged.page_map(state[0], taken, state[3], state[4], state[1], ns["P"], path=path, max_new=Nmax)
        state = now()
        for name, got, w in zip(names, state, want):
            assert np.array_equal(got, w), (seed, name)
        pages = paged.Pages(ns["pages"].cpu().numpy(), D, ns["P"])
        for b in range(B):   # the accepted root lies in its slot
            node = int(path[b, 0])
            blocks = ns["k_tree"][b, node, 0].double().cpu().numpy().reshape(-1, 32)
            scales = [paged.block_scale(x) for x in blocks]
            row = np.concatenate([paged.block_values(paged.block_codes(x, s), s) for x, s in zip(blocks, scales)])
            assert np.array_equal(pages.get("k", int(slots[b, node]), 0), row)
