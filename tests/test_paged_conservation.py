"""Page map: no page is lost, doubled or handed out twice, and the stack's height is what the pages say, for the oracle (CPU) and for the
call. Batches that ask for more pages than there are, where sequences behind a refused one need none or are refused for another reason."""
import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import paged

DEV = "cuda:0"
FORMS = ["rows", "path", "packed"]


def _draw(seed, form):
    rng = np.random.default_rng(seed)
    B, P = int(rng.choice([1, 3, 17, 70, 300])), int(rng.choice([16, 64, 256]))
    top, new_max = int(rng.integers(0, 9 * P)), int(rng.integers(1, 64 if form == "path" else 4 * P))
    kv_len = rng.integers(0, top + 1, B)
    n_new = rng.integers(0, new_max + 1, B)
    n_new[rng.random(B) < 0.3] = rng.integers(0, 3)         # tokens that mostly fit the page a sequence has
    n_new[rng.random(B) < 0.15] = -1
    if form != "path" and B > 1:
        n_new[rng.integers(B)] = 2 * new_max + 10 * P       # fits no row
    width = -(-(top + new_max) // P)
    held = -(-kv_len // P)
    want = int(np.maximum(-(-(kv_len + np.maximum(n_new, 0)) // P) - held, 0).sum())
    spare = int(rng.integers(0, want + 2))
    order = rng.permutation(max(1, int(held.sum()) + spare))
    table = np.full((B, max(1, width)), -1)
    at = 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    free = np.full(len(order), -1)
    free[:len(order) - at] = order[at:]
    kw = dict(n_slots=int(np.maximum(n_new, 0).sum())) if form == "packed" else dict(max_new=new_max)
    if form == "path":
        kw["path"] = np.stack([rng.permutation(new_max) for _ in range(B)])
    return kv_len, n_new, table, free, len(order) - at, P, kw


def _check(case, got):
    """None, or what is wrong with (slots, kv_len_out, n_free_out, granted, table, free)."""
    kv_len, n_new, table0, free0, n_free, P, _ = case
    _, len_out, height, granted, table, free = (np.asarray(x) for x in got)
    height, n_pages = int(height.reshape(-1)[0]), len(free0)
    if not 0 <= height <= n_pages:
        return f"height {height} of {n_pages}"
    had, has = -(-kv_len // P), -(-len_out // P)
    if height != n_free + int(had[n_new < 0].sum()) - int((has - had)[granted == 1].sum()):
        return "height and pages handed out differ"
    held = np.concatenate([table[b, :has[b]] for b in range(len(kv_len))] + [free[:height]])
    if not np.array_equal(np.sort(held), np.arange(n_pages)):
        return "pages lost or doubled"
    for b in range(len(kv_len)):
        if not np.array_equal(table[b, :min(had[b], has[b])], table0[b, :min(had[b], has[b])]):
            return f"row {b} lost a page it had"
    if any(len_out[b] != (0 if n_new[b] < 0 else kv_len[b] + granted[b] * n_new[b]) for b in range(len(kv_len))):
        return "lengths"
    return None


@pytest.mark.parametrize("form", FORMS)
def test_the_oracle_keeps_every_page(form):
    refused = wrong = 0
    for seed in range(150):
        case = _draw(seed, form)
        kv_len, n_new, table, free, n_free, P, kw = case
        got = paged.page_map(kv_len, n_new, table, free, [n_free], P, **kw)
        assert _check(case, got) is None, seed
        refused += int(((got[3] == 0) & (n_new > 0)).any())
        # the largest running demand of a granted sequence is no measure of what was taken: behind a refused one it holds that one's too
        fits = (n_new >= 0) & (kv_len + n_new <= table.shape[1] * P) & (True if form == "packed" else n_new <= kw["max_new"])
        need = np.where(fits, -(-(kv_len + n_new) // P) - -(-kv_len // P), 0)
        demand = int(np.where(got[3] == 1, need.cumsum(), 0).max())
        avail = n_free + int((-(-kv_len // P))[n_new < 0].sum())
        if avail - demand != int(got[2][0]):
            wrong += 1
            assert avail - demand < 0 and _check(case, (*got[:2], np.array([avail - demand]), *got[3:])) is not None
    assert refused >= 10 and wrong >= 5   # (the draws reach both)


@pytest.mark.gpu
@pytest.mark.parametrize("form", FORMS)
def test_the_call_keeps_every_page(form):
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)  # noqa: E731
    for seed in range(60):
        case = _draw(seed, form)
        kv_len, n_new, table, free, n_free, P, kw = case
        t, f = dev(table), dev(free)
        path = dev(kw["path"]) if form == "path" else None
        got = fspad.fspad_page_map(dev(kv_len), dev(n_new), t, f, dev([n_free]), P, path=path, max_new=kw.get("max_new"), n_slots=kw.get("n_slots"))
        torch.cuda.synchronize()
        got = [x.cpu().numpy() for x in (*got, t, f)]
        assert _check(case, got) is None, seed
        want = paged.page_map(kv_len, n_new, table, free, [n_free], P, **kw)
        for name, g, w in zip(("slots", "kv_len_out", "n_free_out", "granted", "table", "free"), got, want):
            assert np.array_equal(g, w), (seed, name)
