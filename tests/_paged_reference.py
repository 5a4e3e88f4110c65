"""The paged attention's oracle (oracle.paged.tree_attn) for cases of many rows: the same output and bound in 64 bits, all rows of a sequence and kv head at once. For finite
inputs."""
from __future__ import annotations

import numpy as np
import torch


def tree_attn(q, k_tree, v_tree, pages, table, kv_len, n_nodes, mask, max_kv_len, scale=None, device="cpu"):
    B, N, Hq, D = q.shape
    Hkv = k_tree.shape[2]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(D) if not scale else float(scale)
    out, bound = np.zeros((B, N, Hq, D)), np.zeros((B, N, Hq, D))
    n_pages = pages.raw.shape[0]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)  # noqa: E731
    for b in range(B):
        n, L = min(max(int(n_nodes[b]), 0), N), min(max(int(kv_len[b]), 0), max_kv_len)
        if n == 0:
            continue
        t = np.arange(L)
        page = np.asarray(table[b], np.int64)[t // pages.P] if L else np.zeros(0, np.int64)
        there = (page >= 0) & (page < n_pages)
        slots = page[there] * pages.P + t[there] % pages.P
        kp, vp = pages.get_many("k", slots), pages.get_many("v", slots)
        see = np.ones((n, len(slots) + n), bool)
        see[:, len(slots):] = (mask[b, :n, None] >> np.arange(n, dtype=np.uint64)) & np.uint64(1)
        see = dev(np.repeat(see, G, axis=0))                                # rows: node by node, head by head
        keys = see.sum(1, keepdim=True)
        for g in range(Hkv):
            k, v = dev(np.concatenate([kp[:, g], k_tree[b, :n, g]])), dev(np.concatenate([vp[:, g], v_tree[b, :n, g]]))
            qq = dev(q[b, :n, g * G:(g + 1) * G].astype(np.float64).reshape(n * G, D))
            s = torch.where(see, torch.mm(qq, k.t()) * scale, -torch.inf)
            w = (s - s.amax(1, keepdim=True).clamp(min=-1e300)).exp()
            total = w.sum(1, keepdim=True)
            w /= torch.where(total == 0, 1.0, total)
            o = torch.mm(w, v)
            e = abs(scale) * ((2 * D + 8) * 2.0 ** -23 * torch.mm(qq.abs(), k.abs().t()) + 2.0 ** -22 * qq.abs().amax(1, keepdim=True) * k.abs().sum(1))
            e = torch.where(see, e, 0.0).amax(1, keepdim=True)
            spread, most = torch.zeros_like(o), torch.zeros_like(o)
            for r in range(n * G):
                mine = v[see[r]]
                if len(mine):
                    spread[r], most[r] = torch.mv((mine - o[r]).abs().t(), w[r][see[r]]), mine.abs().amax(0)
            r = 2.0 ** -8
            off = (r * (1 + 2 * r) + 2 * e + 2.0 ** -22) * spread + keys * 2.0 ** -24 * (torch.mm(w, v.abs()) + o.abs()) + keys * 2.0 ** -125 * (1 + 2 * most)
            out[b, :n, g * G:(g + 1) * G], bound[b, :n, g * G:(g + 1) * G] = (x.cpu().numpy().reshape(n, G, D) for x in (o, off))
    return out, bound
