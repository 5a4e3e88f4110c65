"""What the paged 4-bit cache is timed on: its page map, its store and load, and the tree attention that reads it.

Four kinds of pass, all through the public entry points of the package:

  attn   fspad_tree_attn_paged: the draft tree's queries (or one token's) against the pages and the tree itself
  store  fspad_kv_store_paged, then fspad_kv_load_paged of the same slots: what was written is returned as the values
         that it stands for
  load   fspad_kv_load_paged of a prefix that lies in the pages
  map    fspad_page_map: block tables, slots, lengths and the stack of free pages from request lengths

Geometries are those of the repository's own workloads (Vicuna 7B / 33B, LLaMA3 8B / 70B heads). Keys and values are N(0,1),
cached through the same rounding the store applies; what no token occupies of a page holds random bytes, as memory does.

The cache's format. A block is 32 neighbouring channels of one token and head, an element one of 0, 1/2, 1, 3/2, 2, 3, 4, 6
with a sign (4 bits, the sign on top), a block's scale 2^(s-127) for a byte s; s = 255 makes the block NaN. For a block whose
largest magnitude is a, s is the smallest of 2..252 with a <= 7 * 2^(s-127) (252 where that is too small), and every value is
rounded to the nearest element (ties to the even code, at most 6). Where a page of P tokens keeps one kv head's D channels:

  K codes [P][D/2] | V codes [P*D/512][16][512/D][D/32] | K scales [D/32][P] | V scales [D/32][P]      (bytes)

with the even channel of a byte in its low half; V's codes are groups of 512/D tokens, in a group 16 runs of D/16 channels.
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F32, F64, I32, I64, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64, torch.uint8


# --------------------------------------------------------------------------------------------------- the cases

def _attn(name, **kw):
    case = {"name": name, "kind": "attn", "batch": 1, "n_q_heads": 32, "n_kv_heads": 32, "head_dim": 128, "kv_min": 0,
            "kv_max": 0, "nodes_min": 0, "nodes_max": 1, "page_tokens": 64, "shape_seed": 1}
    case.update(kw)
    case["kv_min"] = case["kv_min"] or case["kv_max"]
    case["nodes_min"] = case["nodes_min"] or case["nodes_max"]
    return case


def listed():
    return [
        # plain decoding of one sequence, short prompt: launches and latency
        _attn("one token", n_kv_heads=8, kv_max=511, page_tokens=16),
        # interactive verification of a 7B model's layer
        _attn("7B tree", kv_max=2048, nodes_max=26),
        # four sequences of a 33B model: the largest cache traffic
        _attn("33B trees of 4 sequences", batch=4, n_q_heads=52, n_kv_heads=52, kv_max=4096, nodes_max=60),
        # long retrieval-augmented prompt of a 70B model: the most arithmetic
        _attn("70B tree, long prompt", n_q_heads=64, n_kv_heads=8, kv_max=16384, nodes_max=60, page_tokens=128),
        # a serving batch as it comes
        _attn("ragged trees of 16", batch=16, n_kv_heads=8, kv_min=131, kv_max=6011, nodes_min=17, nodes_max=60, page_tokens=32,
              shape_seed=7),
        # plain decoding of a batch, smaller heads
        _attn("64 single tokens", batch=64, n_kv_heads=8, head_dim=64, kv_min=100, kv_max=4000, page_tokens=256, shape_seed=3),
        # commit behind a verification step: a few nodes of every tree go to the cache
        {"name": "store accepted paths", "kind": "store", "batch": 4, "rows": 60, "stored": 5, "n_kv_heads": 52, "head_dim": 128,
         "page_tokens": 64, "shape_seed": 1},
        # a prompt goes to the cache
        {"name": "store a prompt", "kind": "store", "batch": 1, "rows": 8191, "stored": 8191, "n_kv_heads": 32, "head_dim": 128,
         "page_tokens": 64, "shape_seed": 2},
        # the last tokens of a sequence come back (a draft model takes them up)
        {"name": "load a tail", "kind": "load", "rows": 26, "n_kv_heads": 8, "head_dim": 64, "page_tokens": 16, "shape_seed": 1},
        # a whole prefix comes back (it moves to a bf16 cache)
        {"name": "load a prefix", "kind": "load", "rows": 16384, "n_kv_heads": 8, "head_dim": 128, "page_tokens": 128, "shape_seed": 1},
        # behind the acceptance of a step: slots of the accepted nodes, a page now and then
        {"name": "map a step", "kind": "map", "batch": 16, "new_min": 1, "new_max": 7, "rows": 60, "kv_max": 6000, "page_tokens": 32,
         "form": "path", "ended": 0.0, "spare": 1.0, "shape_seed": 1},
        # prompts enter while others end
        {"name": "map prompts", "kind": "map", "batch": 256, "new_min": 0, "new_max": 2048, "rows": 0, "kv_max": 4096, "page_tokens": 16,
         "form": "packed", "ended": 0.25, "spare": 1.0, "shape_seed": 2},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges the listed ones stand for, never dearer than the largest of them."""
    kind = rng.choice(["attn", "attn", "attn", "attn", "store", "store", "load", "map", "map"])
    seed, page, D = rng.randrange(1 << 20), rng.choice([16, 32, 64, 64, 128, 256]), rng.choice([64, 128, 128])
    if kind == "attn":
        hq, hkv = rng.choice([(8, 8), (16, 16), (32, 32), (40, 40), (52, 52), (12, 2), (28, 4), (32, 8), (40, 8), (64, 8), (16, 1)])
        nodes = rng.choice([1, 1, 64, 60, 60, 48, 26, rng.randint(1, 64)])
        batch, kv = _log_int(rng, 1, 64), _log_int(rng, 1, 16384)
        while batch * hkv * kv > 8.5e5 or batch * hq * kv * nodes > 5e7:
            batch, kv = (max(1, batch // 2), kv) if batch > 1 else (batch, kv // 2)
        return _attn("drawn", batch=batch, n_q_heads=hq, n_kv_heads=hkv, head_dim=D, kv_min=rng.choice([kv, max(1, kv // 16)]), kv_max=kv,
                     nodes_min=rng.choice([nodes, rng.randint(1, nodes)]), nodes_max=nodes, page_tokens=page, shape_seed=seed)
    if kind == "map":
        form = rng.choice(["path", "rows", "packed"])
        batch, rows = _log_int(rng, 1, 512), rng.randint(1, 64) if form == "path" else 0
        new = rng.randint(1, rows) if form == "path" else _log_int(rng, 1, 2048)
        return {"name": "drawn", "kind": kind, "batch": batch, "new_min": rng.choice([0, min(1, new), new]), "new_max": new, "rows": rows or new,
                "kv_max": _log_int(rng, 1, 4096), "page_tokens": page, "form": form, "ended": rng.choice([0.0, 0.1, 0.3]),
                "spare": rng.choice([1.0, 1.0, 0.5]), "shape_seed": seed}
    hkv = rng.choice([1, 2, 4, 8, 32, 52])
    rows = _log_int(rng, 1, 8191 * 32 * 128 // (hkv * D) if hkv * D > 2048 else 16384)
    if kind == "load":
        return {"name": "drawn", "kind": kind, "rows": rows, "n_kv_heads": hkv, "head_dim": D, "page_tokens": page, "shape_seed": seed}
    batch = rng.choice([1, 1, 2, 5])
    rows = max(1, rows // batch)
    return {"name": "drawn", "kind": kind, "batch": batch, "rows": rows, "stored": rng.choice([rows, rng.randint(1, rows)]), "n_kv_heads": hkv,
            "head_dim": D, "page_tokens": page, "shape_seed": seed}


# ------------------------------------------------------------------------------------------------------ inputs

def _spread(case, lo, hi, salt):
    """One size per sequence between lo and hi (the first one hi), from the case alone."""
    r = np.random.default_rng([case["shape_seed"], salt])
    n = r.integers(lo, hi + 1, case["batch"])
    n[0] = hi
    return n.astype(np.int64)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.empty(shape, dtype=BF16, device="cuda").normal_(generator=g)


def _cuda(a, dtype=I32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)


def _pool(g, n_pages, hkv, page, D):
    return torch.randint(0, 256, (n_pages, hkv, page * D * 17 // 16), dtype=U8, device="cuda", generator=g)


def _tables(g, pages_of, page, spare):
    """Block tables [B, width] of pages in random order, -1 behind a sequence's last page, and the pages left over."""
    width, total = max(1, int(pages_of.max())), int(pages_of.sum())
    order = torch.randperm(total + spare, generator=g, device="cuda").to(I32)
    first = np.cumsum(pages_of) - pages_of
    at = np.arange(width)[None, :]
    table = torch.where(_cuda(at < pages_of[:, None], torch.bool), order[_cuda(np.minimum(first[:, None] + at, total + spare - 1), I64)], -1)
    return table.contiguous(), order[total:].contiguous()


def _prepare_attn(case, seed):
    g = _gen(seed)
    B, N, Hq, Hkv, D, P = (case[k] for k in ("batch", "nodes_max", "n_q_heads", "n_kv_heads", "head_dim", "page_tokens"))
    kv_len, nodes = _spread(case, case["kv_min"], case["kv_max"], 1), _spread(case, case["nodes_min"], N, 2)
    pages_of = -(-kv_len // P)
    table, _ = _tables(g, pages_of, P, 3)
    s = {"case": case, "table": table, "kv_len": _cuda(kv_len), "nodes": _cuda(nodes), "max_kv_len": int(kv_len.max())}
    s["pages"] = _pool(g, int(pages_of.sum()) + 3, Hkv, P, D)
    b = np.repeat(np.arange(B), kv_len)
    at = np.arange(len(b)) - np.repeat(np.cumsum(kv_len) - kv_len, kv_len)
    b, at = _cuda(b, I64), _cuda(at, I64)
    slots = s["table"][b, at // P].long() * P + at % P
    for part in slots.split(1 << 14):   # (the rounding's temporaries are 32-bit copies of what it rounds)
        _plain_store(_normal(g, len(part), Hkv, D), _normal(g, len(part), Hkv, D), part, s["pages"], P)
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
    held = rng.integers(0, 4 * P, B)
    pages_of = -(-(held + case["stored"]) // P)
    table, _ = _tables(g, pages_of, P, 2)
    pick = np.sort(np.argsort(rng.random((B, R)), axis=1)[:, :case["stored"]], axis=1)
    at = _cuda(held[:, None] + np.arange(case["stored"])[None, :], I64)
    slots = torch.full((B, R), -1, dtype=I32, device="cuda")
    slots.scatter_(1, _cuda(pick, I64), (table.long().gather(1, at // P) * P + at % P).int())
    return {"case": case, "k": _normal(g, B * R, Hkv, D), "v": _normal(g, B * R, Hkv, D), "slots": slots.view(B * R),
            "pages": _pool(g, int(pages_of.sum()) + 2, Hkv, P, D)}


def _prepare_load(case, seed):
    g = _gen(seed)
    R, Hkv, D, P = (case[k] for k in ("rows", "n_kv_heads", "head_dim", "page_tokens"))
    n_pages = -(-R // P) + 3
    at = torch.arange(R, device="cuda")
    s = {"case": case, "pages": _pool(g, n_pages, Hkv, P, D)}
    s["slots"] = (torch.randperm(n_pages, generator=g, device="cuda")[at // P] * P + at % P).int()
    for part in s["slots"].split(1 << 14):
        _plain_store(_normal(g, len(part), Hkv, D), _normal(g, len(part), Hkv, D), part, s["pages"], P)
    return s


def _prepare_map(case, seed):
    g, rng = _gen(seed), np.random.default_rng([case["shape_seed"], 9])
    B, P, rows, path = case["batch"], case["page_tokens"], case["rows"], case["form"] == "path"
    kv_len = rng.integers(0, case["kv_max"] + 1, B)
    new = rng.integers(case["new_min"], case["new_max"] + 1, B)
    ended = rng.random(B) < case["ended"]
    held = -(-kv_len // P)
    need = np.where(ended, 0, -(-(kv_len + new) // P) - held)
    table, free = _tables(g, held, P, max(1, int(need.sum() * case["spare"])))
    width = -(-(case["kv_max"] + case["new_max"]) // P)
    s = {"case": case, "kv_len": _cuda(kv_len), "n_new": _cuda(np.where(ended, -1, new)), "n_slots": int(np.where(ended, 0, new).sum()) + 5}
    s["table"] = torch.nn.functional.pad(table, (0, width - table.shape[1]), value=-1).contiguous()
    s["n_free"] = _cuda(np.array([len(free)]))
    s["free"] = torch.nn.functional.pad(free, (0, int(held.sum())), value=-1).contiguous()
    if path:   # the accepted nodes of every tree, root first
        nodes = np.sort(np.argsort(np.random.default_rng([seed, 9]).random((B, rows)), axis=1)[:, :case["new_max"]], axis=1)
        nodes = np.pad(nodes, ((0, 0), (0, rows - nodes.shape[1])))
        s["path"] = _cuda(np.where(np.arange(rows)[None, :] < new[:, None], nodes, -1))
    s["rows"] = rows if path else case["new_max"]
    return s


def prepare(case, seed):
    return {"attn": _prepare_attn, "store": _prepare_store, "load": _prepare_load, "map": _prepare_map}[case["kind"]](case, seed)


# ------------------------------------------------------------------------------------------------- plain forms

def _regions(pages, P, D):
    """Views of a pool [n_pages, Hkv, bytes]: K codes, V codes, K scales, V scales."""
    c, sc = P * D // 2, P * D // 32
    k, v, ks, vs = pages[..., :c], pages[..., c:2 * c], pages[..., 2 * c:2 * c + sc], pages[..., 2 * c + sc:]
    return (k.unflatten(2, (P, D // 2)), v.unflatten(2, (P * D // 512, 16, 512 // D, D // 32)), ks.unflatten(2, (D // 32, P)),
            vs.unflatten(2, (D // 32, P)))


def _encode(x):
    """Codes [..., D/2] and scale bytes [..., D/32] of x [..., D]."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)                                              # top = m 2^e, 1/2 <= m < 1; 7 * 2^z = 7/8 * 2^(z+3)
    s = torch.where(top > 0, e - 3 + (m > 0.875).int(), -1000) + 127
    s = torch.where(torch.isfinite(top), s.clamp(2, 252), 255)
    y = torch.ldexp(x, 127 - s).abs()
    code = ((y > 0.25).to(U8) + (y >= 0.75).to(U8) + (y > 1.25).to(U8) + (y >= 1.75).to(U8) + (y > 2.5).to(U8) + (y >= 3.5).to(U8) + (y > 5).to(U8)
            + 8 * torch.signbit(x).to(U8))
    code = torch.where(s == 255, 0, code).to(U8).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], s.squeeze(-1).to(U8)


def _decode(code, scale):
    """Values [..., D] of codes [..., D/2] and scale bytes [..., D/32]."""
    c = torch.stack([code & 15, code >> 4], -1).flatten(-2)
    h = (c & 7).float()
    v = torch.where(h < 2, h / 2, torch.ldexp(1 + (h % 2) / 2, (h / 2).floor() - 1))   # 0, .5, 1, 1.5, 2, 3, 4, 6
    v = torch.where(c > 7, -v, v).unflatten(-1, (-1, 32))
    s = scale.int().unsqueeze(-1)
    return torch.where(s == 255, math.nan, torch.ldexp(v, s - 127)).flatten(-2)


def _plain_store(k, v, slots, pages, P):
    D = k.shape[-1]
    kc, vc, ks, vs = _regions(pages, P, D)
    live = (slots >= 0).nonzero().squeeze(1)
    slot = slots[live].long()
    p, t, g = slot // P, slot % P, 512 // D
    kc[p, :, t], scale = _encode(k[live])
    ks[p, :, :, t] = scale
    code, scale = _encode(v[live])
    vc[p, :, t // g, :, t % g] = code.unflatten(-1, (16, D // 32))
    vs[p, :, :, t] = scale


def _plain_load(slots, pages, P, D):
    kc, vc, ks, vs = _regions(pages, P, D)
    live = (slots >= 0)[:, None, None]
    slot = slots.long().clamp(min=0)
    p, t, g = slot // P, slot % P, 512 // D
    k = _decode(kc[p, :, t], ks[p, :, :, t])
    v = _decode(vc[p, :, t // g, :, t % g].flatten(-2), vs[p, :, :, t])
    return torch.where(live, k, 0).to(BF16), torch.where(live, v, 0).to(BF16)


def _plain_attn(s):
    case = s["case"]
    B, N, Hq, Hkv, D, P = (case[k] for k in ("batch", "nodes_max", "n_q_heads", "n_kv_heads", "head_dim", "page_tokens"))
    G, W = Hq // Hkv, s["table"].shape[1]
    kc, vc, ks, vs = _regions(s["pages"], P, D)
    t = s["table"].long().clamp(min=0)
    k = _decode(kc[t], ks[t].transpose(-1, -2))                            # [B, W, Hkv, P, D]
    v = vc[t].transpose(-2, -3).flatten(-2).flatten(-3, -2)                # token groups, tokens, runs of channels -> [B, W, Hkv, P, D/2]
    v = _decode(v, vs[t].transpose(-1, -2))
    seen = torch.arange(W * P, device="cuda")[None, :] < s["kv_len"][:, None]
    k = torch.where(seen[:, None, :, None], k.transpose(1, 2).flatten(2, 3), 0)
    v = torch.where(seen[:, None, :, None], v.transpose(1, 2).flatten(2, 3), 0)
    k = torch.cat([k, s["k_tree"].float().transpose(1, 2)], 2)             # [B, Hkv, L, D]
    v = torch.cat([v, s["v_tree"].float().transpose(1, 2)], 2)
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


def _plain_map(s):
    case, P, width = s["case"], s["case"]["page_tokens"], s["table"].shape[1]
    new, kv_len, n_free, n_pages = s["n_new"].long(), s["kv_len"].long(), s["n_free"].long(), len(s["free"])
    ended, have = new < 0, -(-s["kv_len"].long() // P)
    add = new.clamp(min=0)
    pages = torch.arange(width, device="cuda")
    # pages of ended sequences go on the stack first
    back = torch.where(ended, have, 0)
    at = n_free + (back.cumsum(0) - back)[:, None] + pages
    gone = pages < back[:, None]
    s["free"][at[gone]] = s["table"][gone]
    avail = n_free + back.sum()
    # and new ones come off it, sequence after sequence
    fits = kv_len + add <= width * P
    need = torch.where(fits & ~ended, -(-(kv_len + add) // P) - have, 0)
    upto = need.cumsum(0)
    granted = fits & ~ended & ((need == 0) | (upto <= avail))
    taken = torch.where(granted, upto, 0).amax()
    i = pages - have[:, None]
    fresh = granted[:, None] & (i >= 0) & (i < need[:, None])
    s["table"][fresh] = s["free"][(avail - 1 - (upto - need)[:, None] - i)[fresh]]
    first = add.cumsum(0) - add
    j = torch.arange(max(1, case["new_max"]), device="cuda")
    where = kv_len[:, None] + j
    slot = s["table"].gather(1, (where // P).clamp(max=width - 1)).long() * P + where % P
    live = granted[:, None] & (j < add[:, None])
    if case["form"] == "packed":
        slots = torch.full((s["n_slots"],), -1, dtype=I64, device="cuda")
        slots[(first[:, None] + j)[live]] = slot[live]
    elif case["form"] == "path":
        slots = torch.full((len(new), s["rows"]), -1, dtype=I64, device="cuda")
        node = s["path"].long()[:, :len(j)]
        slots[torch.arange(len(new), device="cuda")[:, None].expand_as(node)[live], node[live]] = slot[live]
    else:
        slots = torch.where(live, slot, -1)
    length = torch.where(ended, 0, torch.where(granted, kv_len + add, kv_len))
    return slots.int(), length.int(), (avail - taken).int(), granted.int(), s["table"], s["free"]


# -------------------------------------------------------------------------------------------------------- pass

def _calls(s):
    """The calls of a pass with their arguments in place, made once for a state's buffers as a serving loop keeps them (lengths, tables
    and slots are on the device, so a step changes no argument), and the pass's outputs."""
    import paper_2408_15562_amd as fspad
    case = s["case"]
    if case["kind"] == "attn":
        call = fspad.fspad_tree_attn_paged(s["q"], s["k_tree"], s["v_tree"], s["pages"], s["table"], s["kv_len"], s["nodes"], s["mask"],
                                           max_kv_len=s["max_kv_len"], prepare=True)
        return [call], call.result
    if case["kind"] == "map":
        packed = case["form"] == "packed"
        call = fspad.fspad_page_map(s["kv_len"], s["n_new"], s["table"], s["free"], s["n_free"], case["page_tokens"], path=s.get("path"),
                                    max_new=None if packed else s["rows"], n_slots=s["n_slots"] if packed else None, prepare=True)
        return [call], (*call.result, s["table"], s["free"])
    load = fspad.fspad_kv_load_paged(s["slots"], s["pages"], case["head_dim"], prepare=True)
    if case["kind"] == "load":
        return [load], load.result
    return [fspad.fspad_kv_store_paged(s["k"], s["v"], s["slots"], s["pages"], prepare=True), load], load.result


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if own:
        if "calls" not in s:
            s["calls"], s["outputs"] = _calls(s)
        for call in s["calls"]:
            call()
        return s["outputs"]
    if kind == "attn":
        return _plain_attn(s)
    if kind == "map":
        return _plain_map(s)
    if kind == "store":
        _plain_store(s["k"], s["v"], s["slots"], s["pages"], case["page_tokens"])
    return _plain_load(s["slots"], s["pages"], case["page_tokens"], case["head_dim"])


def work(case):
    if case["kind"] == "attn":
        B, N, Hq, Hkv, D = (case[k] for k in ("batch", "nodes_max", "n_q_heads", "n_kv_heads", "head_dim"))
        kv, n = _spread(case, case["kv_min"], case["kv_max"], 1), _spread(case, case["nodes_min"], N, 2)
        cache = int(kv.sum()) * Hkv * D * 17 // 16
        live = int(n.sum())
        return {"bytes": cache + live * (Hq * D * 2 + 2 * Hkv * D * 2 + 8) + B * N * Hq * D * 2 + int((-(-kv // case["page_tokens"])).sum()) * 4,
                "flops": 4 * Hq * D * int((n * (kv + n)).sum())}
    if case["kind"] == "map":
        tokens = case["batch"] * (case["new_min"] + case["new_max"]) // 2
        slots = case["batch"] * case["rows"] if case["form"] != "packed" else tokens
        return {"bytes": 4 * (4 * case["batch"] + slots + 2 * tokens // case["page_tokens"]), "flops": 0}
    each = case["n_kv_heads"] * case["head_dim"]
    wide, narrow = 4 * each, each * 17 // 16
    if case["kind"] == "load":
        return {"bytes": case["rows"] * (wide + narrow + 4), "flops": 0}
    stored, rows = case["batch"] * case["stored"], case["batch"] * case["rows"]
    return {"bytes": stored * (wide + 2 * narrow) + rows * (wide + 4), "flops": 0}


# ------------------------------------------------------------------------------------------------------- exact

def _exact_pages(s, P, D):
    """All K and V of a pool in 64 bits, [n_pages, Hkv, P, D], byte by byte from the format's description."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=F64, device="cuda")
    scales = torch.tensor([math.ldexp(1.0, e - 127) for e in range(255)] + [math.nan], dtype=F64, device="cuda")
    tok, ch = torch.arange(P, device="cuda")[:, None], torch.arange(D, device="cuda")[None, :]
    group, run_ = 512 // D, D // 16
    at_k = tok * (D // 2) + ch // 2
    at_v = P * D // 2 + ((tok // group * 16 + ch // run_) * group + tok % group) * (run_ // 2) + ch % run_ // 2
    at_ks = P * D + ch // 32 * P + tok
    half = (4 * (ch % 2)).expand(P, D)
    values = [table[((s["pages"][:, :, at].int() >> half) & 15).long()] * scales[s["pages"][:, :, at_s].long()]
              for at, at_s in ((at_k, at_ks), (at_v, at_ks + P * D // 32))]
    return values


def _exact_round(x):
    """What the store makes of x [T, Hkv, D], in 64 bits: every element against all fifteen values of its block's scale."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    powers = torch.tensor([math.ldexp(1.0, e - 127) for e in range(2, 253)], dtype=F64, device="cuda")
    scale = powers[torch.searchsorted(7 * powers, top).clamp(max=250)]
    y = x / scale
    even, odd = [0.0, 1.0, 2.0, 4.0], [0.5, 1.5, 3.0, 6.0]
    best, far = torch.zeros_like(y), y.abs()
    for value in even[1:] + odd:         # values with even codes first: they keep a tie
        d = (y.abs() - value).abs()
        best, far = torch.where(d < far, value, best), torch.minimum(d, far)
    return (torch.copysign(best, y) * scale).flatten(-2)


def exact(case, seed):
    if case["kind"] == "map":
        return None          # whole numbers: there is nothing between them
    s = prepare(case, seed)
    P, D = case["page_tokens"], case["head_dim"]
    if case["kind"] == "store":
        live = (s["slots"] >= 0)[:, None, None]
        return [torch.where(live, _exact_round(s[n]), 0.0) for n in ("k", "v")]
    if case["kind"] == "load":
        slots = s["slots"].long()
        return [x[slots // P, :, slots % P] for x in _exact_pages(s, P, D)]
    B, N, Hq, Hkv = (case[k] for k in ("batch", "nodes_max", "n_q_heads", "n_kv_heads"))
    G = Hq // Hkv
    kv_len, nodes, table = s["kv_len"].tolist(), s["nodes"].tolist(), s["table"].tolist()
    mask = s["mask"].cpu().numpy().view(np.uint64)
    out = torch.zeros(B, N, Hq, D, dtype=F64, device="cuda")
    for b in range(B):
        n, L = nodes[b], kv_len[b]
        pages = {"pages": s["pages"][table[b][:-(-L // P)]]}
        see = np.zeros((n, L + n), bool)
        see[:, :L] = True
        see[:, L:] = (mask[b, :n, None] >> np.arange(n, dtype=np.uint64)) & np.uint64(1)
        see = torch.from_numpy(see).cuda()
        kv = [x.transpose(0, 1).flatten(1, 2)[:, :L] for x in _exact_pages(pages, P, D)]
        for g in range(Hkv):
            k = torch.cat([kv[0][g], s["k_tree"][b, :n, g].double()])
            v = torch.cat([kv[1][g], s["v_tree"][b, :n, g].double()])
            x = torch.mm(s["q"][b, :n, g * G:(g + 1) * G].double().reshape(n * G, D), k.t()) / math.sqrt(D)
            x = x.view(n, G, L + n).masked_fill(~see[:, None, :], -math.inf)
            out[b, :n, g * G:(g + 1) * G] = torch.mm(torch.softmax(x, -1).view(n * G, L + n), v).view(n, G, D)
    return out
