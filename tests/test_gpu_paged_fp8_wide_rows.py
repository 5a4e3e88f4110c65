"""Store into (and load from) the paged 8-bit cache where a workgroup takes two heads at a time (launch_store: from 65536 rows times heads on, or 2048 in 1024 workgroups): heads by two
and by four a workgroup, odd numbers of them, by the scan of all slots and by the list. Every head byte for byte against the oracle."""
import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import paged_fp8
from test_gpu_paged_fp8_rows import DEV, _bf16, _pool, _rows, _same

pytestmark = pytest.mark.gpu
OWN = 7   # heads that differ: head h is head h % 7 again, so that places of a workgroup's heads have all of them


def _store(k, v, slots, raw, D, P):
    """Store, load; what the oracle has of the heads that differ, and the pool as it came out."""
    heads = np.arange(k.shape[1]) % OWN
    dev, s = torch.from_numpy(raw).to(DEV), torch.from_numpy(slots).to(DEV)
    size = fspad.fspad_kv_store_paged_byte_workspace_bytes(fspad.binding._pool_desc(dev, D, True), len(slots))
    ws = torch.full((size + 64,), 1, dtype=torch.uint8, device=DEV)
    fspad.fspad_kv_store_paged_byte(k.to(DEV), v.to(DEV), s, dev, workspace=ws[:size])
    back = fspad.fspad_kv_load_paged_byte(s, dev, D)
    torch.cuda.synchronize()
    assert bool((ws[size:] == 1).all())
    ref = paged_fp8.Fp8Pages(raw[:, :OWN].copy(), D, P)
    ref.store("k", k[:, :OWN].double().numpy(), slots)
    ref.store("v", v[:, :OWN].double().numpy(), slots)
    got = dev.cpu().numpy()
    _same(got, np.ascontiguousarray(ref.raw[:, heads]), D, P, slots)
    inside = (slots >= 0) & (slots < raw.shape[0] * P)
    for which, x in zip("kv", back):
        want = np.where(inside[:, None, None], ref.get_many(which, np.where(inside, slots, 0)), 0.0)[:, heads]
        assert np.array_equal(x.cpu().double().numpy(), want, equal_nan=True)
    return got


@pytest.mark.parametrize("order", ["from inside a block on", "scattered"])
@pytest.mark.parametrize("rows,Hkv,D", [(2048, 33, 128), (2048, 40, 64), (2048, 67, 64), (2100, 33, 64), (2100, 64, 128), (4100, 35, 64), (8191, 9, 128), (8191, 17, 64), (2048, 1, 128),
                                        (1024, 2, 64)])
def test_two_heads_at_a_time(rows, Hkv, D, order):
    """Heads two (or four) a workgroup: the second group's are stored, the last workgroup's odd one by the first group alone. Blocks begun and full, added to, with scales that stay and
    that grow, with NaN, infinity and large values in heads of both groups, rows outside the pool."""
    P, rng = 64, np.random.default_rng(rows + Hkv + D)
    heads, n_pages = np.arange(Hkv) % OWN, -(-rows // P) + 2
    raw = _pool(rows, n_pages, OWN, P, D)[:, heads]
    k, v = (_rows(rng, rows, OWN, D)[:, torch.from_numpy(heads)].contiguous() for _ in range(2))
    k[rows // 5, 3 % Hkv::OWN, 9] = float("inf")
    v[rows // 7, 1 % Hkv::OWN, 2] = float("nan")
    v[rows // 2 + 40, 2 % Hkv::OWN] *= 2.0 ** 100
    slots = (np.arange(rows) + 37 if order != "scattered" else rng.permutation(n_pages * P)[:rows]).astype(np.int32)
    slots[[1, 300]] = [-1, n_pages * P]
    got = _store(k, v, slots, np.ascontiguousarray(raw), D, P)
    # and again, larger ones in part of them: scales grow, what is held is rounded again
    some = np.where(rng.random(rows) < 0.3, slots, -1).astype(np.int32)
    some[some % 32 == 0] = -1                              # (no block is begun)
    again = [(x.float().nan_to_num(0, 0, 0).clamp(-2.0 ** 60, 2.0 ** 60) * f).to(torch.bfloat16) for x, f in ((k, 16.0), (v, 0.25))]
    _store(*again, some, got, D, P)


@pytest.mark.parametrize("rows,Hkv,D", [(37, 3, 64), (37, 3, 128), (2100, 40, 64)])
def test_one_head_for_all(rows, Hkv, D):
    """Keys and values with a head stride of zero: every head of the pool gets the one there is, blocks begun and added to."""
    P, rng = 32, np.random.default_rng(rows + D)
    n_pages = -(-rows // P) + 1
    slots = (np.arange(rows) + 5).astype(np.int32)
    one = torch.from_numpy(np.zeros((n_pages, Hkv, paged_fp8.page_head_bytes(D, P)), np.uint8)).to(DEV)
    k, v = (_bf16(rng.standard_normal((rows, 1, D)) * 2.0 ** rng.integers(-4, 5, (rows, 1, 1))) for _ in range(2))
    fspad.fspad_kv_store_paged_byte(k.to(DEV).expand(rows, Hkv, D), v.to(DEV).expand(rows, Hkv, D), torch.from_numpy(slots).to(DEV), one)
    torch.cuda.synchronize()
    ref = paged_fp8.Fp8Pages(np.zeros((n_pages, 1, paged_fp8.page_head_bytes(D, P)), np.uint8), D, P)
    ref.store("k", k.double().numpy(), slots)
    ref.store("v", v.double().numpy(), slots)
    got = one.cpu().numpy()
    for g in range(Hkv):
        _same(np.ascontiguousarray(got[:, g:g + 1]), ref.raw, D, P, slots)
    assert got[:, 0].any() and all(np.array_equal(got[:, 0], got[:, g]) for g in range(Hkv))
