"""What the paged 8-bit cache and sequences that share pages are timed on.

Five kinds of pass, all through the public entry points of the package:

  attn     fspad_tree_attn_paged_byte: the draft tree's queries (or one token's) against 8-bit pages and the tree itself
  store    fspad_kv_store_paged_byte, then fspad_kv_load_paged_byte of the blocks that were written to: what the cache holds of them
           is returned as the values that it stands for
  fork     fspad_page_fork, then fspad_page_copy in a layer's pool: sequences begin as copies of others, whose full pages they share
  release  fspad_page_release: sequences end, pages that nobody else holds go back to the stack
  compact  fspad_page_compact, then fspad_page_copy in a layer's pool: what is held moves to the front of the pool

Geometries are those of the repository's own workloads (Vicuna 7B / 33B, LLaMA3 8B / 70B heads). Keys and values are N(0,1),
cached through the rounding that the store applies; what no token occupies of a page holds random bytes, as memory does.

The cache's format. A block is 32 neighbouring tokens of a page and one kv head, K and V apart. An element is an 8-bit float (1 sign, 4
exponent, 3 mantissa bits, largest 448, no infinity), a block's scale 2^(s-127) for a byte s. Of values whose largest finite magnitude is a,
s is the smallest of 10..246 with a <= 448 * 2^(s-127), 246 where that is too small; values are rounded to the nearest element (ties to
even, at most 448), NaN and infinity become NaN. A call that stores a block's first token begins the block: its scale is that of the call's tokens in it. Otherwise it is
the larger of that and of the scale the block has; where it grows, the tokens that the block held are rounded again under the new one.
Where a page of P tokens keeps one kv head's D channels (E = D/32):

  K codes [P/32][D/16][32][16]      token t, channel c at [t/32][c/16][t%32][c%16]
  V codes [P/32][E][2][32][16]      token t, channel c at [t/32][c%E][t%32/16][c/E][t%16]
  K scales [8] | V scales [8]       one byte for each of the P/32 blocks, the rest of the eight unused

A page that several sequences hold has shared[page] holders beside the first; a sequence's last page, if it is not full, is its own.
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F32, F64, I32, I64, U8, FP8 = (torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64, torch.uint8,
                                     torch.float8_e4m3fn)


# --------------------------------------------------------------------------------------------------- the cases

def _attn(name, **kw):
    case = {"name": name, "kind": "attn", "prompts": 1, "branches": 1, "n_q_heads": 32, "n_kv_heads": 32, "head_dim": 128, "kv_min": 0,
            "kv_max": 0, "nodes_min": 0, "nodes_max": 1, "page_tokens": 64, "shape_seed": 1}
    case.update(kw)
    case["kv_min"] = case["kv_min"] or case["kv_max"]
    case["nodes_min"] = case["nodes_min"] or case["nodes_max"]
    return case


def _pages(name, kind, **kw):
    case = {"name": name, "kind": kind, "prompts": 1, "branches": 1, "kv_min": 0, "kv_max": 0, "page_tokens": 64, "n_kv_heads": 8, "head_dim": 128,
            "shape_seed": 1}
    case.update(kw)
    case["kv_min"] = case["kv_min"] or case["kv_max"]
    return case


def listed():
    return [
        # plain decoding of one sequence, short prompt: launches and latency
        _attn("one token", n_kv_heads=8, kv_max=511, page_tokens=32),
        # four sequences of a 33B model: the largest cache traffic
        _attn("33B trees of 4 sequences", prompts=4, n_q_heads=52, n_kv_heads=52, kv_max=4096, nodes_max=60),
        # long retrieval-augmented prompt of a 70B model: the most arithmetic
        _attn("70B tree, long prompt", n_q_heads=64, n_kv_heads=8, kv_max=16384, nodes_max=60, page_tokens=128),
        # several answers to each of eight prompts, a token at a time, smaller heads: branches share their prompt's pages
        _attn("64 forked single tokens", prompts=8, branches=8, n_kv_heads=8, head_dim=64, kv_min=100, kv_max=4000, shape_seed=3),
        # commit behind a verification step: a few nodes of every tree go to the cache
        {"name": "store accepted paths", "kind": "store", "batch": 4, "rows": 60, "stored": 5, "n_kv_heads": 52, "head_dim": 128,
         "page_tokens": 64, "shape_seed": 1},
        # a prompt goes to the cache
        {"name": "store a prompt", "kind": "store", "batch": 1, "rows": 8191, "stored": 8191, "n_kv_heads": 32, "head_dim": 128,
         "page_tokens": 64, "shape_seed": 2},
        # one prompt, three more answers to it
        _pages("fork one prompt", "fork", branches=3, kv_max=2000, spare=1.0),
        # a batch of prompts with eight answers each
        _pages("fork 32 prompts", "fork", prompts=32, branches=7, kv_min=300, kv_max=6011, page_tokens=128, spare=1.0, shape_seed=2),
        # some of a few answers are finished
        _pages("release some of 16", "release", prompts=4, branches=4, kv_min=1000, kv_max=2048, ended=0.3),
        # half of a large batch is
        _pages("release half of 1024", "release", prompts=256, branches=4, kv_min=1000, kv_max=8000, page_tokens=32, ended=0.5, shape_seed=5),
        # a small pool gives memory back
        _pages("compact a small pool", "compact", prompts=4, branches=2, kv_min=500, kv_max=1500, page_tokens=32, n_kv_heads=4, head_dim=64, fill=0.6),
        # a large one does (half a gigabyte of one layer)
        _pages("compact a large pool", "compact", prompts=32, branches=2, kv_min=1000, kv_max=6011, fill=0.6, shape_seed=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges the listed ones stand for, never dearer than the largest of them."""
    kind = rng.choice(["attn", "attn", "attn", "attn", "store", "store", "fork", "fork", "release", "release", "compact", "compact"])
    seed, page, D = rng.randrange(1 << 20), rng.choice([32, 64, 64, 128, 256]), rng.choice([64, 128, 128])
    if kind == "attn":
        hq, hkv = rng.choice([(8, 8), (16, 16), (32, 32), (40, 40), (52, 52), (12, 2), (28, 4), (32, 8), (40, 8), (64, 8), (16, 1)])
        nodes = rng.choice([1, 1, 64, 60, 60, 48, 26, rng.randint(1, 64)])
        prompts, branches, kv = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 4, 8]), _log_int(rng, 1, 16384)
        while prompts * branches * hkv * kv > 8.5e5 or prompts * branches * hq * kv * nodes > 5e7:
            if prompts > 1:
                prompts //= 2
            elif branches > 1:
                branches //= 2
            else:
                kv //= 2
        return _attn("drawn", prompts=prompts, branches=branches, n_q_heads=hq, n_kv_heads=hkv, head_dim=D, kv_min=rng.choice([kv, max(1, kv // 16)]),
                     kv_max=kv, nodes_min=rng.choice([nodes, rng.randint(1, nodes)]), nodes_max=nodes, page_tokens=page, shape_seed=seed)
    if kind == "store":
        hkv = rng.choice([1, 2, 4, 8, 32, 52])
        rows = _log_int(rng, 1, 8191 * 32 * 128 // (hkv * D) if hkv * D > 2048 else 16384)
        batch = rng.choice([1, 1, 2, 5])
        rows = max(1, rows // batch)
        return {"name": "drawn", "kind": kind, "batch": batch, "rows": rows, "stored": rng.choice([rows, rng.randint(1, rows)]), "n_kv_heads": hkv,
                "head_dim": D, "page_tokens": page, "shape_seed": seed}
    kv = _log_int(rng, 1, 6000)
    case = dict(kv_min=rng.choice([kv, max(1, kv // 4)]), kv_max=kv, page_tokens=page, n_kv_heads=rng.choice([1, 2, 4, 8]), head_dim=D, shape_seed=seed)
    if kind == "fork":
        prompts, branches = _log_int(rng, 1, 48), rng.randint(1, 9)
        while prompts * kv > 40000 or prompts * branches > 240:
            prompts, branches = max(1, prompts // 2), max(1, branches // 2)
            if prompts == branches == 1:
                break
        return _pages("drawn", kind, prompts=prompts, branches=branches, spare=rng.choice([1.0, 1.0, 0.5]), **case)
    if kind == "release":
        return _pages("drawn", kind, prompts=_log_int(rng, 1, 256), branches=rng.randint(1, 4), ended=rng.choice([0.1, 0.3, 0.5, 1.0]), **case)
    prompts, branches = _log_int(rng, 1, 48), rng.randint(1, 4)
    while prompts > 1 and prompts * branches * kv > 120000:
        prompts //= 2
    return _pages("drawn", kind, prompts=prompts, branches=branches, fill=rng.uniform(0.4, 0.95), **case)


# ------------------------------------------------------------------------------------------------------ inputs

def _spread(case, lo, hi, n, salt):
    """n sizes between lo and hi (the first one hi), from the case alone."""
    r = np.random.default_rng([case["shape_seed"], salt])
    x = r.integers(lo, hi + 1, n)
    x[0] = hi
    return x.astype(np.int64)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.empty(shape, dtype=BF16, device="cuda").normal_(generator=g)


def _cuda(a, dtype=I32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)


def _pool(g, n_pages, hkv, P, D):
    return torch.randint(0, 256, (n_pages, hkv, 2 * P * D + 16), dtype=U8, device="cuda", generator=g)


def _held(case):
    """Lengths of all sequences (prompts x branches) and how many full pages the branches of each prompt share: all but the last few."""
    n, b, P = case["prompts"], case["branches"], case["page_tokens"]
    kv = _spread(case, case["kv_min"], case["kv_max"], n * b, 1).reshape(n, b)
    common = kv.min(1) * 7 // 8 // P if b > 1 else np.zeros(n, np.int64)
    return kv, common


def _sequences(case, g, n_pages=None):
    """Block tables [B, width] whose pages lie anywhere in the pool (-1 behind a sequence's last one), lengths, the other holders of every page,
    the stack of free pages and its height. n_pages from the number of pages held."""
    kv, common = _held(case)
    P, (n, b) = case["page_tokens"], kv.shape
    pages_of = -(-kv // P)
    used = int(common.sum() + (pages_of - common[:, None]).sum())
    n_pages = used + 3 if n_pages is None else n_pages(used)
    table, shared = np.full((n * b, int(pages_of.max())), -1, np.int64), np.zeros(n_pages, np.int64)
    at = 0
    for i in range(n):
        shared[at:at + common[i]] = b - 1
        table[i * b:(i + 1) * b, :common[i]] = np.arange(at, at + common[i])
        at += common[i]
        for j in range(b):
            table[i * b + j, common[i]:pages_of[i, j]] = np.arange(at, at + pages_of[i, j] - common[i])
            at += pages_of[i, j] - common[i]
    order = torch.randperm(n_pages, generator=g, device="cuda")
    t = _cuda(table, I64)
    s = {"case": case, "kv_len": _cuda(kv.reshape(-1)), "n_pages": n_pages, "n_free": _cuda(np.array([n_pages - used]))}
    s["table"] = torch.where(t >= 0, order[t.clamp(min=0)], -1).int().contiguous()
    s["shared"] = torch.zeros(n_pages, dtype=I32, device="cuda")
    s["shared"][order] = _cuda(shared)
    s["free"] = torch.nn.functional.pad(order[used:].int(), (0, used), value=-1).contiguous()
    return s


def _fill(g, pages, fill, P, D):
    """Tokens below fill[page] of every page: values N(0,1), rounded block by block. The rest of a page stays as it is."""
    kc, vc, ks, vs = _regions(pages, P, D)
    step = max(1, (1 << 25) // (pages.shape[1] * P * D))      # (the rounding's temporaries are 32-bit copies)
    for p0 in range(0, len(pages), step):
        part = slice(p0, min(p0 + step, len(pages)))
        there = (torch.arange(P, device="cuda") < fill[part, None])[:, None, :, None]
        for codes, scales, store in ((kc, ks, _k_order), (vc, vs, _v_order)):
            x = _normal(g, part.stop - p0, pages.shape[1], P, D)
            x = torch.where(there, x, 0).float().unflatten(2, (P // 32, 32))
            s = _scale_of(x.abs().amax((-1, -2)))
            scales[part] = torch.where(there[:, :, ::32, 0].expand_as(s), s, scales[part].int()).to(U8)
            x = torch.ldexp(x, 127 - s[..., None, None]).to(FP8).view(U8)
            codes[part] = torch.where(store(there.unflatten(2, (P // 32, 32)).expand_as(x), D), store(x, D), codes[part])


def _prepare_attn(case, seed):
    g = _gen(seed)
    s = _sequences(case, g)
    B, N, Hq, Hkv, D, P = case["prompts"] * case["branches"], *(case[k] for k in ("nodes_max", "n_q_heads", "n_kv_heads", "head_dim", "page_tokens"))
    nodes = _spread(case, case["nodes_min"], N, B, 2)
    s["nodes"], s["max_kv_len"] = _cuda(nodes), int(case["kv_max"])
    s["pages"] = _pool(g, s["n_pages"], Hkv, P, D)
    fill = torch.zeros(s["n_pages"], dtype=I64, device="cuda")
    at = torch.arange(s["table"].shape[1], device="cuda")
    left = (s["kv_len"].long()[:, None] - at * P).clamp(0, P)
    fill[s["table"][left > 0].long()] = left[left > 0]
    _fill(g, s["pages"], fill, P, D)
    s["q"], s["k_tree"], s["v_tree"] = _normal(g, B, N, Hq, D), _normal(g, B, N, Hkv, D), _normal(g, B, N, Hkv, D)
    # random trees: node i hangs on one of the nodes before it; a node sees its ancestors and itself
    rng = np.random.default_rng([seed, 5])
    mask = np.zeros((B, N), np.uint64)
    mask[:, 0] = 1
    for i in range(1, N):
        parent = rng.integers(max(0, i - 12), i, B)
        mask[:, i] = mask[np.arange(B), parent] | (np.uint64(1) << np.uint64(i))
    mask[np.arange(N)[None, :] >= nodes[:, None]] = 0
    s["mask"] = torch.from_numpy(mask.view(np.int64)).cuda()
    return s


def _prepare_store(case, seed):
    g = _gen(seed)
    B, R, Hkv, D, P = (case[k] for k in ("batch", "rows", "n_kv_heads", "head_dim", "page_tokens"))
    # `stored` rows of every sequence go to the slots behind what it holds already, the others nowhere
    rng = np.random.default_rng([case["shape_seed"], seed])
    held = np.random.default_rng([case["shape_seed"], 4]).integers(0, 4 * P, B)
    n, pages_of = case["stored"], -(-(held + case["stored"]) // P)
    first = np.cumsum(pages_of) - pages_of
    order = torch.randperm(int(pages_of.sum()) + 2, generator=g, device="cuda")
    pick = np.sort(np.argsort(rng.random((B, R)), axis=1)[:, :n], axis=1)
    slot_of = lambda t: order[_cuda(first[:, None] + t // P, I64)] * P + _cuda(t % P, I64)  # noqa: E731
    slots = torch.full((B, R), -1, dtype=I64, device="cuda")
    slots.scatter_(1, _cuda(pick, I64), slot_of(held[:, None] + np.arange(n)[None, :]))
    # what is read back: from the start of the block that the first new token lies in
    back = np.concatenate([np.arange(h // 32 * 32, h + n) for h in held]), np.repeat(np.arange(B), held % 32 + n)
    s = {"case": case, "k": _normal(g, B * R, Hkv, D), "v": _normal(g, B * R, Hkv, D), "slots": slots.view(B * R).int(),
         "pages": _pool(g, len(order), Hkv, P, D)}
    s["back"] = (order[_cuda(first[back[1]] + back[0] // P, I64)] * P + _cuda(back[0] % P, I64)).int()
    fill = torch.zeros(len(order), dtype=I64, device="cuda")
    for b in range(B):
        at = np.arange(-(-held[b] // P))
        fill[order[_cuda(first[b] + at, I64)]] = _cuda(np.minimum(held[b] - at * P, P), I64)
    _fill(g, s["pages"], fill, P, D)
    return s


def _prepare_fork(case, seed):
    g = _gen(seed)
    n, b, P = case["prompts"], case["branches"], case["page_tokens"]
    prompts = dict(case, branches=1)
    copies = int((_held(prompts)[0] % P > 0).sum()) * b     # forks that need a page
    s = _sequences(prompts, g, lambda used: used + max(1, int(copies * case["spare"])))
    s["case"] = case
    # rows [0, n) of the table hold the prompts, the branches' rows behind them are empty
    s["table"] = torch.nn.functional.pad(s["table"], (0, 3, 0, n * b), value=-1).contiguous()
    s["kv_len"] = torch.nn.functional.pad(s["kv_len"], (0, n * b))
    s["src"] = torch.arange(n, device="cuda").repeat_interleave(b).int()
    s["dst"] = n + torch.randperm(n * b, generator=g, device="cuda").int()
    s["pages"] = _pool(g, s["n_pages"], case["n_kv_heads"], P, case["head_dim"])
    return s


def _prepare_release(case, seed):
    g = _gen(seed)
    s = _sequences(case, g)
    B = len(s["kv_len"])
    s["ended"] = (torch.rand(B, generator=g, device="cuda") < case["ended"]).int()
    s["ended"][0] = 1
    return s


def _prepare_compact(case, seed):
    g = _gen(seed)
    s = _sequences(case, g, lambda used: max(used + 1, int(used / case["fill"])))
    s["pages"] = _pool(g, s["n_pages"], case["n_kv_heads"], case["page_tokens"], case["head_dim"])
    return s


def prepare(case, seed):
    return {"attn": _prepare_attn, "store": _prepare_store, "fork": _prepare_fork, "release": _prepare_release,
            "compact": _prepare_compact}[case["kind"]](case, seed)


# ------------------------------------------------------------------------------------------------- plain forms

def _regions(pages, P, D):
    """Views of a pool [n_pages, Hkv, bytes]: K codes, V codes, K scales, V scales (of the blocks there are)."""
    c, nb = P * D, P // 32
    return (pages[..., :c].unflatten(2, (nb, D // 16, 32, 16)), pages[..., c:2 * c].unflatten(2, (nb, D // 32, 2, 32, 16)),
            pages[..., 2 * c:2 * c + nb], pages[..., 2 * c + 8:2 * c + 8 + nb])


def _k_order(x, D):
    """Blocks [..., 32 tokens, D channels] in the order of K's codes, and back."""
    return x.unflatten(-1, (D // 16, 16)).transpose(-2, -3)


def _k_back(c):
    return c.transpose(-2, -3).flatten(-2)


def _v_order(x, D):
    x = x.unflatten(-2, (2, 16)).unflatten(-1, (32, D // 32))              # ..., 2, 16, 32, E
    return x.movedim(-1, -4).transpose(-1, -2)                             # ..., E, 2, 32, 16


def _v_back(c):
    return c.transpose(-1, -2).movedim(-4, -1).flatten(-2).flatten(-3, -2)


def _scale_of(top):
    m, e = torch.frexp(top)                                                # top = m 2^e, 1/2 <= m < 1; 448 * 2^z = 7/8 * 2^(z+9)
    return torch.where(top > 0, e - 9 + (m > 0.875).int() + 127, 0).clamp(10, 246)


def _plain_store(k, v, slots, pages, P):
    D = k.shape[-1]
    kc, vc, ks, vs = _regions(pages, P, D)
    live = (slots >= 0).nonzero().squeeze(1)
    slot = slots[live].long()
    block, of = torch.unique(slot // 32, return_inverse=True)
    page, nth, t = block // (P // 32), block % (P // 32), slot % 32
    begun = torch.zeros(len(block), dtype=torch.bool, device="cuda")
    begun[of[t == 0]] = True
    for x, codes, scales, order, back in ((k, kc, ks, _k_order, _k_back), (v, vc, vs, _v_order, _v_back)):
        x = x[live].float()
        x = torch.where(torch.isfinite(x), x, math.nan)
        top = torch.zeros(len(block), x.shape[1], device="cuda").scatter_reduce_(0, of[:, None].expand(-1, x.shape[1]), x.abs().nan_to_num(0.0).amax(-1), "amax")
        had, s = scales[page, :, nth].int(), _scale_of(top)
        s = torch.where(begun[:, None], s, torch.maximum(had, s))
        was = back(codes[page, :, nth])                                    # [blocks, Hkv, 32, D]
        again = torch.ldexp(was.view(FP8).float(), (had - s)[..., None, None]).to(FP8).view(U8)
        new = torch.where((~begun[:, None] & (s > had))[..., None, None], again, was)
        new[of, :, t] = torch.ldexp(x, 127 - s[of][..., None]).clamp(-448, 448).to(FP8).view(U8)
        codes[page, :, nth] = order(new, D)
        scales[page, :, nth] = s.to(U8)


def _plain_load(slots, pages, P, D):
    slot = slots.long()
    p, nth, t = slot // P, slot % P // 32, slot % 32
    out = []
    for codes, scales, back in zip(_regions(pages, P, D)[:2], _regions(pages, P, D)[2:], (_k_back, _v_back)):
        x = back(codes)[p, :, nth, t].view(FP8).float()                    # [rows, Hkv, D]
        out.append(torch.ldexp(x, scales[p, :, nth].int()[..., None] - 127).to(BF16))
    return tuple(out)


def _plain_attn(s):
    case = s["case"]
    N, Hq, Hkv, D, P = (case[k] for k in ("nodes_max", "n_q_heads", "n_kv_heads", "head_dim", "page_tokens"))
    (B, W), G = s["table"].shape, Hq // Hkv
    kc, vc, ks, vs = _regions(s["pages"], P, D)
    t = s["table"].long().clamp(min=0)
    seen = torch.arange(W * P, device="cuda")[None, :] < s["kv_len"][:, None]
    kv = []
    for codes, scales, back, tree in ((kc, ks, _k_back, s["k_tree"]), (vc, vs, _v_back, s["v_tree"])):
        x = torch.ldexp(back(codes[t]).view(FP8).float(), scales[t].int()[..., None, None] - 127)   # [B, W, Hkv, P/32, 32, D]
        x = x.transpose(1, 2).reshape(B, Hkv, W * P, D)
        kv.append(torch.cat([torch.where(seen[:, None, :, None], x, 0), tree.float().transpose(1, 2)], 2))
    k, v = kv
    q = s["q"].float().view(B, N, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, N * G, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, Hkv, N, G, -1).mul_(1 / math.sqrt(D))
    alive = torch.arange(N, device="cuda")[None, :] < s["nodes"][:, None]
    tree = ((s["mask"][:, :, None] >> torch.arange(N, device="cuda")) & 1).bool() & alive[:, None, :]
    see = torch.cat([seen[:, None, :].expand(B, N, -1), tree], 2) & alive[:, :, None]
    x.masked_fill_(~see[:, None, :, None, :], -math.inf)
    x.sub_(x.amax(-1, keepdim=True).clamp_(min=-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.view(B, Hkv, N * G, -1), v).view(B, Hkv, N, G, D)
    out = torch.where(total > 0, out / total, 0)
    return out.transpose(1, 2).reshape(B, N, Hq, D).to(BF16)


def _plain_copy(pages, src, dst):
    live = src >= 0
    pages[dst[live].long()] = pages[src[live].long()]


def _plain_fork(s):
    P, table, kv_len, n_pages = s["case"]["page_tokens"], s["table"], s["kv_len"].long(), s["n_pages"]
    src, dst, n_free = s["src"].long(), s["dst"].long(), s["n_free"].long()
    n = kv_len[src]
    need = (n % P > 0).long()
    upto = need.cumsum(0)
    granted = (need == 0) | (upto <= n_free)
    takes = granted & (need > 0)
    full = torch.where(granted, n // P, 0)
    page = s["free"].long()[(n_free - upto).clamp(min=0)]
    i = torch.arange(table.shape[1], device="cuda")
    shares = i < full[:, None]
    rows = table[src]
    shared = s["shared"].long().scatter_add(0, rows[shares].long(), torch.ones_like(rows[shares], dtype=I64))
    tail = rows.gather(1, (n // P).clamp(max=table.shape[1] - 1)[:, None]).squeeze(1).long()
    copy_src, copy_dst = torch.where(takes, tail, -1), torch.where(takes, page, -1)
    entries = torch.where(shares, rows, torch.where(takes[:, None] & (i == full[:, None]), page[:, None].int(), table[dst]))
    table[dst] = entries
    lens = kv_len.clone()
    lens[dst] = torch.where(granted, n, kv_len[dst])
    _plain_copy(s["pages"], copy_src, copy_dst)
    return copy_src.int(), copy_dst.int(), lens.int(), (n_free - takes.sum()).int(), shared.int(), granted.int(), table, s["pages"]


def _plain_release(s):
    P, table, kv_len, n_pages = s["case"]["page_tokens"], s["table"], s["kv_len"].long(), s["n_pages"]
    ended, n_free = s["ended"] != 0, s["n_free"].long()
    drop = (torch.arange(table.shape[1], device="cuda") < -(-kv_len // P)[:, None]) & ended[:, None]
    page = table[drop].long()
    drops = torch.zeros(n_pages, dtype=I64, device="cuda").scatter_add_(0, page, torch.ones_like(page))
    gone = drops > s["shared"]
    back = gone.nonzero().squeeze(1)                                       # lowest number first
    s["free"][n_free + torch.arange(len(back), device="cuda")] = back.int()
    shared = torch.where(gone, 0, s["shared"] - drops)
    return torch.where(ended, 0, kv_len).int(), (n_free + len(back)).int(), shared.int(), s["free"]


def _plain_compact(s):
    P, table, kv_len, n_pages = s["case"]["page_tokens"], s["table"], s["kv_len"].long(), s["n_pages"]
    number = torch.arange(n_pages, device="cuda")
    keep = n_pages - s["n_free"].long()
    free = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
    free[s["free"][number < s["n_free"]].long()] = True
    holes, movers = (free & (number < keep)).nonzero().squeeze(1), (~free & (number >= keep)).nonzero().squeeze(1)
    to = number.clone()
    to[movers] = holes
    copy_src = torch.full((n_pages // 2,), -1, dtype=I64, device="cuda")
    copy_dst = copy_src.clone()
    copy_src[:len(movers)], copy_dst[:len(movers)] = movers, holes
    held = torch.arange(table.shape[1], device="cuda") < -(-kv_len // P)[:, None]
    table = torch.where(held, to[table.long().clamp(min=0)], table.long())
    shared = s["shared"].long().clone()
    shared[holes], shared[movers] = shared[movers], 0
    # the stack: what is left over at the end of the pool, lowest number on top
    stack = torch.where(number < s["n_free"], n_pages - 1 - number, -1)
    _plain_copy(s["pages"], copy_src, copy_dst)
    return copy_src.int(), copy_dst.int(), table.int(), stack.int(), shared.int(), s["pages"]


# -------------------------------------------------------------------------------------------------------- pass

def _calls(s):
    """The calls of a pass with their arguments in place, made once for a state's buffers as a serving loop keeps them (lengths, tables
    and slots are on the device, so a step changes no argument), and the pass's outputs."""
    import paper_2408_15562_amd as fspad
    case = s["case"]
    kind, P = case["kind"], case["page_tokens"]
    if kind == "attn":
        call = fspad.fspad_tree_attn_paged_byte(s["q"], s["k_tree"], s["v_tree"], s["pages"], s["table"], s["kv_len"], s["nodes"], s["mask"],
                                               max_kv_len=s["max_kv_len"], prepare=True)
        return [call], call.result
    if kind == "store":
        store = fspad.fspad_kv_store_paged_byte(s["k"], s["v"], s["slots"], s["pages"], prepare=True)
        load = fspad.fspad_kv_load_paged_byte(s["back"], s["pages"], case["head_dim"], prepare=True)
        return [store, load], load.result
    if kind == "release":
        call = fspad.fspad_page_release(s["ended"], s["kv_len"], s["table"], s["free"], s["n_free"], s["shared"], P, prepare=True)
        return [call], (*call.result, s["free"])
    if kind == "fork":
        call = fspad.fspad_page_fork(s["src"], s["dst"], s["kv_len"], s["table"], s["free"], s["n_free"], s["shared"], P, prepare=True)
        outputs = (*call.result, s["table"], s["pages"])
    else:
        call = fspad.fspad_page_compact(s["kv_len"], s["table"], s["free"], s["n_free"], s["shared"], P, prepare=True)
        outputs = (*call.result, s["pages"])
    return [call, fspad.fspad_page_copy(call.result[0], call.result[1], s["pages"], prepare=True)], outputs


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if own:
        if "calls" not in s:
            s["calls"], s["outputs"] = _calls(s)
        for call in s["calls"]:
            call()
        return s["outputs"]
    if kind == "store":
        _plain_store(s["k"], s["v"], s["slots"], s["pages"], case["page_tokens"])
        return _plain_load(s["back"], s["pages"], case["page_tokens"], case["head_dim"])
    return {"attn": _plain_attn, "fork": _plain_fork, "release": _plain_release, "compact": _plain_compact}[kind](s)


def work(case):
    kind, P = case["kind"], case["page_tokens"]
    if kind == "store":
        each = case["n_kv_heads"] * case["head_dim"]
        stored = case["batch"] * case["stored"]
        back = stored + case["batch"] * 16                                  # the blocks the first new tokens lie in: half full
        return {"bytes": stored * (4 + 2) * each + back * (2 + 4) * each + 4 * (case["batch"] * case["rows"] + back), "flops": 0}
    kv, common = _held(case)
    pages_of = -(-kv // P)
    if kind == "attn":
        N, Hq, Hkv, D = (case[k] for k in ("nodes_max", "n_q_heads", "n_kv_heads", "head_dim"))
        n, B = _spread(case, case["nodes_min"], N, kv.size, 2), kv.size
        tokens = int(kv.sum() - ((case["branches"] - 1) * common * P).sum())   # what branches share is read once
        live = int(n.sum())
        return {"bytes": tokens * Hkv * D * 2 + live * (Hq * D * 2 + 2 * Hkv * D * 2 + 8) + B * N * Hq * D * 2 + int(pages_of.sum()) * 4,
                "flops": 4 * Hq * D * int((n * (kv.reshape(-1) + n)).sum())}
    page = case["n_kv_heads"] * (2 * P * case["head_dim"] + 16)
    used = int(common.sum() + (pages_of - common[:, None]).sum())
    if kind == "fork":
        kv, b = _held(dict(case, branches=1))[0], case["branches"]
        copies = max(1, int(int((kv % P > 0).sum()) * b * case["spare"])) if (kv % P > 0).any() else 0
        full = int((kv // P).sum())
        return {"bytes": copies * 2 * page + 4 * (full + full * b + 2 * int((-(-kv // P)).sum())) + 16 * kv.size * (b + 1), "flops": 0}
    if kind == "release":
        return {"bytes": int(4 * (case["ended"] * pages_of.sum() + 2 * used + 3 * kv.size)), "flops": 0}
    n_pages = max(used + 1, int(used / case["fill"]))
    moved = used * (n_pages - used) // n_pages                              # of pages anywhere in the pool, so many lie too far back
    return {"bytes": moved * 2 * page + 4 * int(2 * pages_of.sum() + 4 * n_pages), "flops": 0}


# ------------------------------------------------------------------------------------------------------- exact

def _elements():
    """All 256 elements in 64 bits, from their bits."""
    x = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.nan if e == 15 and m == 7 else math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        x.append(-v if c > 127 else v)
    return torch.tensor(x, dtype=F64, device="cuda")


def _exact_pages(pages, P, D):
    """All K and V of some pages in 64 bits, [n, Hkv, P, D], byte by byte from the format's description."""
    element, E = _elements(), D // 32
    t, c = torch.arange(P, device="cuda")[:, None], torch.arange(D, device="cuda")[None, :]
    at_k = ((t // 32 * (D // 16) + c // 16) * 32 + t % 32) * 16 + c % 16
    at_v = P * D + (((t // 32 * E + c % E) * 2 + t % 32 // 16) * 32 + c // E) * 16 + t % 16
    at_s = 2 * P * D + (t // 32).expand(P, D)
    return [element[pages[:, :, at].long()] * torch.pow(torch.tensor(2.0, dtype=F64, device="cuda"), pages[:, :, sc].double() - 127)
            for at, sc in ((at_k, at_s), (at_v, at_s + 8))]


def _exact_round(x, s):
    """x in 64 bits rounded under scale bytes s (broadcast): to multiples of the spacing that elements of its size have."""
    y = x / torch.pow(torch.tensor(2.0, dtype=F64, device="cuda"), s.double() - 127)
    _, e = torch.frexp(y)
    step = torch.pow(torch.tensor(2.0, dtype=F64, device="cuda"), (e.double() - 4).clamp(min=-9))
    return (torch.round(y / step) * step).clamp(-448, 448) * torch.pow(torch.tensor(2.0, dtype=F64, device="cuda"), s.double() - 127)   # (round: ties to even)


def _exact_store(s, P, D):
    """What the blocks that are read back hold after the store: slot by slot, [rows, Hkv, D] each."""
    back, slots = s["back"].long(), s["slots"].long()
    new = torch.full((len(s["pages"]) * P,), -1, dtype=I64, device="cuda")
    live = (slots >= 0).nonzero().squeeze(1)
    new[slots[live]] = live
    before = _exact_pages(s["pages"], P, D)
    block = torch.arange(32, device="cuda") + back[:, None] // 32 * 32                     # the slots of every slot's block
    out = []
    powers = torch.pow(torch.tensor(2.0, dtype=F64, device="cuda"), torch.arange(10, 247, device="cuda").double() - 127)
    for x, old, at in ((s["k"], before[0], 0), (s["v"], before[1], 8)):
        had = s["pages"][back // P, :, 2 * P * D + at + back % P // 32].long()             # [rows, Hkv]
        top_of_row = torch.cat([x.double().abs().amax(-1), torch.zeros(1, x.shape[1], dtype=F64, device="cuda")])
        top = top_of_row[new[block]].amax(1)                                               # (-1: the row of zeros)
        scale = torch.searchsorted(448 * powers, top).clamp(max=236) + 10
        begun = (new[block[:, 0]] >= 0)[:, None]
        scale = torch.where(begun, scale, torch.maximum(scale, had))[..., None]
        mine = new[back]
        stored = _exact_round(x[mine.clamp(min=0)].double(), scale)
        kept = old[back // P, :, back % P]
        kept = torch.where(scale > had[..., None], _exact_round(kept, scale), kept)
        out.append(torch.where((mine >= 0)[:, None, None], stored, kept))
    return out


def exact(case, seed):
    if case["kind"] not in ("attn", "store"):
        return None          # whole numbers: there is nothing between them
    s = prepare(case, seed)
    P, D = case["page_tokens"], case["head_dim"]
    if case["kind"] == "store":
        return _exact_store(s, P, D)
    N, Hq, Hkv = (case[k] for k in ("nodes_max", "n_q_heads", "n_kv_heads"))
    B, G = len(s["kv_len"]), Hq // Hkv
    kv_len, nodes, table = s["kv_len"].tolist(), s["nodes"].tolist(), s["table"].tolist()
    mask = s["mask"].cpu().numpy().view(np.uint64)
    out = torch.zeros(B, N, Hq, D, dtype=F64, device="cuda")
    for b in range(B):
        n, L = nodes[b], kv_len[b]
        see = np.zeros((n, L + n), bool)
        see[:, :L] = True
        see[:, L:] = (mask[b, :n, None] >> np.arange(n, dtype=np.uint64)) & np.uint64(1)
        see = torch.from_numpy(see).cuda()
        kv = [x.transpose(0, 1).flatten(1, 2)[:, :L] for x in _exact_pages(s["pages"][table[b][:-(-L // P)]], P, D)]
        for g in range(Hkv):
            k = torch.cat([kv[0][g], s["k_tree"][b, :n, g].double()])
            v = torch.cat([kv[1][g], s["v_tree"][b, :n, g].double()])
            x = torch.mm(s["q"][b, :n, g * G:(g + 1) * G].double().reshape(n * G, D), k.t()) / math.sqrt(D)
            x = x.view(n, G, L + n).masked_fill(~see[:, None, :], -math.inf)
            out[b, :n, g * G:(g + 1) * G] = torch.mm(torch.softmax(x, -1).view(n * G, L + n), v).view(n, G, D)
    return out
