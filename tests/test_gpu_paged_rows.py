"""GPU store to and load from the paged 4-bit cache against the oracle: byte for byte, and nothing else of the pool touched."""
import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


def _rows(rng, rows, Hkv, D):
    """Rows whose blocks span the range: ordinary ones, tiny and huge ones, zeros, one with infinity and one with NaN."""
    x = rng.standard_normal((rows, Hkv, D // 32, 32)) * 2.0 ** rng.integers(-20, 20, (rows, Hkv, D // 32, 1))
    flat = x.reshape(-1, 32)
    for i, f in enumerate((0.0, 2.0 ** -126, 2.0 ** 124, -0.0)):
        flat[(7 * i + 1) % len(flat)] *= f
    if len(flat) > 40:
        flat[35, 3] = np.inf
        flat[38, 31] = np.nan
    return _bf16(x.reshape(rows, Hkv, D))


def _pool(seed, n_pages, Hkv, P, D):
    return np.random.default_rng(seed).integers(0, 256, (n_pages, Hkv, paged.page_head_bytes(D, P)), dtype=np.uint8)


def _put_all(pool, D, P, k, v, slots):
    ref = paged.Pages(pool.copy(), D, P)
    for r, slot in enumerate(slots):
        if 0 <= slot < pool.shape[0] * P:
            for g in range(pool.shape[1]):
                ref.put("k", int(slot), g, k[r, g].double().numpy())
                ref.put("v", int(slot), g, v[r, g].double().numpy())
    return ref


@pytest.mark.parametrize("rows,Hkv,D,P", [(1, 1, 64, 16), (1, 1, 128, 16), (17, 3, 64, 32), (33, 5, 128, 64), (16, 1, 128, 256), (47, 2, 64, 256),
                                          (9, 52, 128, 16)])
@pytest.mark.parametrize("order", ["in a row", "scattered"])
def test_store_then_load(rows, Hkv, D, P, order):
    rng = np.random.default_rng(rows + D)
    n_pages = -(-rows // P) + 2
    pool = _pool(rows, n_pages, Hkv, P, D)
    k, v = _rows(rng, rows, Hkv, D), _rows(rng, rows, Hkv, D)
    slots = np.arange(P - 3, P - 3 + rows) if order == "in a row" else rng.permutation(n_pages * P)[:rows]
    slots = slots.astype(np.int32)
    if rows > 4:
        slots[[1, 3]] = [-1, n_pages * P]                 # one row before the pool, one behind it: neither is written
    dev = torch.from_numpy(pool).to(DEV)
    s = torch.from_numpy(slots).to(DEV)
    fspad.fspad_kv_store_paged(k.to(DEV), v.to(DEV), s, dev)
    torch.cuda.synchronize()
    ref = _put_all(pool, D, P, k, v, slots)
    assert np.array_equal(dev.cpu().numpy(), ref.raw)
    got = fspad.fspad_kv_load_paged(s, dev, D)
    torch.cuda.synchronize()
    inside = (slots >= 0) & (slots < n_pages * P)
    for which, x in zip("kv", got):
        want = np.where(inside[:, None, None], ref.get_many(which, np.where(inside, slots, 0)), 0.0)
        assert np.array_equal(x.cpu().double().numpy(), want, equal_nan=True)


def test_every_bf16_value_is_rounded_as_the_format_says():
    """All 65536 bit patterns, in blocks whose largest value sets scales around them."""
    bits = np.arange(1 << 16).astype(np.uint16)
    x = torch.from_numpy(bits.view(np.int16).copy()).view(torch.bfloat16)
    finite = torch.isfinite(x.float())
    x = x[finite]
    rng = np.random.default_rng(5)
    x = torch.cat([x, x[torch.from_numpy(rng.permutation(len(x)))], x.abs().sort().values])
    x = torch.nn.functional.pad(x, (0, -len(x) % (2 * 128)))
    k = x.view(-1, 2, 128)
    P, n_pages = 64, -(-len(k) // 64)
    dev = torch.zeros((n_pages, 2, paged.page_head_bytes(128, P)), dtype=torch.uint8, device=DEV)
    s = torch.arange(len(k), dtype=torch.int32, device=DEV)
    fspad.fspad_kv_store_paged(k.to(DEV), k.neg().to(DEV), s, dev)
    gk, gv = (t.cpu() for t in fspad.fspad_kv_load_paged(s, dev, 128))
    blocks = k.double().reshape(-1, 32).numpy()
    want = np.empty_like(blocks)
    for i, row in enumerate(blocks):
        sc = paged.block_scale(row)
        want[i] = paged.block_values(paged.block_codes(row, sc), sc)
    assert np.array_equal(gk.double().reshape(-1, 32).numpy(), want)
    assert np.array_equal(gv.double().reshape(-1, 32).numpy(), -want)


@pytest.mark.parametrize("D", [64, 128])
def test_strided_rows_and_pages(D):
    """Keys and values as slices of one projection's output, pages of two layers interleaved, and a load into a cache's own layout."""
    rng = np.random.default_rng(6)
    rows, Hq, Hkv, P, n_pages, L = 37, 4, 3, 32, 4, 64
    qkv = _bf16(rng.standard_normal((rows, (Hq + 2 * Hkv) * D))).to(DEV)
    k = qkv[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
    v = qkv[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
    both = torch.from_numpy(np.concatenate([_pool(1, n_pages, Hkv, P, D)[:, None], _pool(2, n_pages, Hkv, P, D)[:, None]], axis=1)).to(DEV)
    before = both.clone()
    slots = rng.permutation(n_pages * P)[:rows].astype(np.int32)
    s = torch.from_numpy(slots).to(DEV)
    fspad.fspad_kv_store_paged(k, v, s, both[:, 1])
    torch.cuda.synchronize()
    assert torch.equal(both[:, 0], before[:, 0])
    ref = _put_all(before[:, 1].cpu().numpy(), D, P, k.cpu(), v.cpu(), slots)
    assert np.array_equal(both[:, 1].cpu().numpy(), ref.raw)
    cache = torch.full((2, 2, Hkv, L, D), 7.0, dtype=torch.bfloat16, device=DEV)     # K and V caches [B, Hkv, L, D]
    part = [c[1, :, 5:5 + rows].transpose(0, 1) for c in cache]
    fspad.fspad_kv_load_paged(s, both[:, 1], D, outputs=part)
    torch.cuda.synchronize()
    for which, p, c in zip("kv", part, cache):
        assert np.array_equal(p.cpu().double().numpy(), ref.get_many(which, slots))
        assert bool((c[0] == 7).all()) and bool((c[1, :, :5] == 7).all()) and bool((c[1, :, 5 + rows:] == 7).all())
    # one head for all: a stride of zero is read as often as there are rows
    wide = k[:, :1].expand(rows, Hkv, D)
    fspad.fspad_kv_store_paged(wide, wide, s, both[:, 0])
    got = fspad.fspad_kv_load_paged(s, both[:, 0], D)
    assert torch.equal(got[0], got[1]) and all(torch.equal(got[0][:, 0], got[0][:, g]) for g in range(Hkv))


def test_no_rows_and_repeated_loads():
    pool = torch.from_numpy(_pool(3, 2, 2, 16, 128)).to(DEV)
    before = pool.clone()
    none = torch.empty((0, 2, 128), dtype=torch.bfloat16, device=DEV)
    fspad.fspad_kv_store_paged(none, none, torch.empty(0, dtype=torch.int32, device=DEV), pool)
    k, v = fspad.fspad_kv_load_paged(torch.empty(0, dtype=torch.int32, device=DEV), pool, 128)
    assert k.shape == v.shape == (0, 2, 128) and torch.equal(pool, before)
    k, v = fspad.fspad_kv_load_paged(torch.tensor([5, 5, 31, 5], dtype=torch.int32, device=DEV), pool, 128)
    assert torch.equal(k[0].view(torch.int16), k[3].view(torch.int16)) and torch.equal(v[0].view(torch.int16), v[1].view(torch.int16))


def test_slots_and_pages_past_32_bits_of_bytes():
    """A pool of more than 4 GB: what goes to its last page does not come round to its first."""
    D, P, Hkv = 128, 256, 8
    per = fspad.fspad_kv_page_bytes(Hkv, D, P)
    n_pages = (1 << 32) // per + 40
    pool = torch.zeros((n_pages, Hkv, per // Hkv), dtype=torch.uint8, device=DEV)
    x = _bf16(np.random.default_rng(8).standard_normal((3, Hkv, D))).to(DEV)
    slots = torch.tensor([n_pages * P - 1, 0, (n_pages - 30) * P + 17], dtype=torch.int32, device=DEV)
    fspad.fspad_kv_store_paged(x, -x, slots, pool)
    k, v = fspad.fspad_kv_load_paged(slots, pool, D)
    torch.cuda.synchronize()
    ref = _put_all(np.zeros((1, Hkv, per // Hkv), np.uint8), D, P, x.cpu(), -x.cpu(), [P + 1, 0, P + 1])
    assert np.array_equal(pool[:1].cpu().numpy(), ref.raw)
    assert torch.equal(k, -v) and float((k - x).abs().max()) < float(x.abs().max()) * 2 / 7
    used = torch.zeros(n_pages, dtype=torch.bool, device=DEV)
    used[[0, n_pages - 30, n_pages - 1]] = True
    assert bool((pool.view(n_pages, -1).amax(1) > 0).eq(used).all())


def test_more_rows_than_a_launch_has_workgroups():
    """One row, repeated by a stride of zero, into every slot of more than a million; then all of them back."""
    D, P, rows = 128, 64, (1 << 20) + 77
    n_pages = -(-rows // P)
    rng = np.random.default_rng(1)
    k, v = (_rows(rng, 1, 1, D).to(DEV) for _ in range(2))
    pages = torch.zeros((n_pages, 1, paged.page_head_bytes(D, P)), dtype=torch.uint8, device=DEV)
    slots = torch.arange(rows, dtype=torch.int32, device=DEV).flip(0).contiguous()
    fspad.fspad_kv_store_paged(k.expand(rows, 1, D), v.expand(rows, 1, D), slots, pages)
    got = fspad.fspad_kv_load_paged(slots, pages, D)
    one = _pool(0, 1, 1, P, D)
    ref = _put_all(one, D, P, k.cpu(), v.cpu(), [0])
    for g, name in zip(got, "kv"):
        want = torch.from_numpy(ref.get(name, 0, 0)).to(torch.bfloat16).to(DEV)
        assert bool((g[:, 0] == want).all())
    assert bool((pages[-1, 0, (rows % P) * D // 2:P * D // 2] == 0).all())   # K codes of slots that got no row
