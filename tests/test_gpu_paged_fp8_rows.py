"""GPU store to and load from the paged 8-bit cache against the oracle: byte for byte, and nothing else of the pool touched."""
import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import paged_fp8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _bf16(a):
    with np.errstate(over="ignore"):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


def _rows(rng, rows, Hkv, D, spread=4):
    """Ordinary rows of different sizes, zeros, tiny and huge ones, one with infinity and one with NaN."""
    x = rng.standard_normal((rows, Hkv, D)) * 2.0 ** rng.integers(-spread, spread + 1, (rows, Hkv, 1))
    for i, f in enumerate((0.0, 2.0 ** -120, -0.0)):
        x[(7 * i + 1) % rows] *= f
    if rows > 20:
        x[rows // 2, 0, 3] = np.inf
        x[rows // 3, -1, D - 1] = np.nan
        x[rows - 1] *= 2.0 ** 118
    return _bf16(x)


def _pool(seed, n_pages, Hkv, P, D):
    """Random codes under scales that a cache may hold."""
    rng = np.random.default_rng(seed)
    raw = rng.integers(0, 256, (n_pages, Hkv, paged_fp8.page_head_bytes(D, P)), dtype=np.uint8)
    raw[:, :, 2 * P * D:] = rng.integers(105, 125, (n_pages, Hkv, 16))
    return raw


def _same(got, want, D, P, slots):
    """Bytes equal but for the signs and kinds of NaN, and for tokens of a begun block that the call did not store."""
    live = slots[(slots >= 0) & (slots < got.shape[0] * P)]
    got, want = got.copy(), want.copy()
    for b in {int(s) // 32 for s in live if s % 32 == 0}:
        for t in set(range(32 * b, 32 * b + 32)) - {int(s) for s in live}:
            for which in "kv":
                at = paged_fp8.Fp8Pages(got, D, P).places(which, t % P)[0]
                got[t // P][:, at] = want[t // P][:, at] = 0
    code = np.arange(got.shape[2]) < 2 * P * D
    for x in (got, want):
        x[(x & 0x7f == 0x7f) & code] = 0x7f
    assert np.array_equal(got, want)


def _store_and_check(k, v, slots, pool, D, P):
    dev, s = torch.from_numpy(pool).to(DEV), torch.from_numpy(slots).to(DEV)
    ws = torch.full((fspad.fspad_kv_store_paged_byte_workspace_bytes(fspad.binding._pool_desc(dev, D, True), len(slots)) + 64,), 1, dtype=torch.uint8, device=DEV)
    fspad.fspad_kv_store_paged_byte(k.to(DEV), v.to(DEV), s, dev, workspace=ws[:-64])
    torch.cuda.synchronize()
    ref = paged_fp8.Fp8Pages(pool.copy(), D, P)
    ref.store("k", k.double().numpy(), slots)
    ref.store("v", v.double().numpy(), slots)
    _same(dev.cpu().numpy(), ref.raw, D, P, slots)
    assert bool((ws[-64:] == 1).all())
    got = fspad.fspad_kv_load_paged_byte(s, dev, D)
    torch.cuda.synchronize()
    inside = (slots >= 0) & (slots < pool.shape[0] * P)
    for which, x in zip("kv", got):
        want = np.where(inside[:, None, None], ref.get_many(which, np.where(inside, slots, 0)), 0.0)
        assert np.array_equal(x.cpu().double().numpy(), want, equal_nan=True)
    return dev


@pytest.mark.parametrize("rows,Hkv,D,P", [(1, 1, 64, 32), (1, 1, 128, 32), (17, 3, 64, 32), (33, 5, 128, 64), (16, 1, 128, 256), (47, 2, 64, 256), (9, 52, 128, 32),
                                          (100, 2, 128, 64), (1024, 1, 64, 64), (1025, 1, 64, 64), (1100, 2, 128, 32), (2000, 1, 128, 256), (17000, 1, 64, 64)])
@pytest.mark.parametrize("order", ["in a row", "scattered", "from a block on"])
def test_store_then_load(rows, Hkv, D, P, order):
    rng = np.random.default_rng(rows + D)
    n_pages = -(-rows // P) + 2
    pool = _pool(rows, n_pages, Hkv, P, D)
    k, v = _rows(rng, rows, Hkv, D), _rows(rng, rows, Hkv, D)
    slots = np.arange(P - 3, P - 3 + rows) if order == "in a row" else np.arange(rows) + 32 if order != "scattered" else rng.permutation(n_pages * P)[:rows]
    slots = slots.astype(np.int32)
    if rows > 4:
        slots[[1, 3]] = [-1, n_pages * P]                 # one row before the pool, one behind it: neither is written
    _store_and_check(k, v, slots, pool, D, P)


@pytest.mark.parametrize("D,P,spread", [(128, 64, 0), (64, 32, 3), (128, 32, 12)])
def test_token_by_token(D, P, spread):
    """A sequence that grows by a few tokens a call: blocks begin, fill, and grow as larger tokens come. What is held is that of the oracle after
    every call, and in the end within its bound of what was stored."""
    rng = np.random.default_rng(spread)
    pool, at, rows = _pool(3, 3, 2, P, D), 0, []
    pool[:, :, 2 * P * D:] = 255                          # (what no call has begun may hold anything)
    while at < 2 * P - 5:
        n = int(rng.integers(1, 6))
        k, v = (_bf16(rng.standard_normal((n, 2, D)) * 2.0 ** rng.integers(-spread, spread + 1, (n, 2, 1))) for _ in range(2))
        slots = np.arange(at, at + n, dtype=np.int32)
        pool = _store_and_check(k, v, slots, pool, D, P).cpu().numpy()
        rows.append((k, v))
        at += n
    ref = paged_fp8.Fp8Pages(pool, D, P)
    for which, x in zip("kv", (torch.cat(r).double().numpy() for r in zip(*rows))):
        held = ref.get_many(which, np.arange(at))
        s = np.stack([pool[t // P][:, ref.places(which, t % P)[1]] for t in range(at)]).astype(np.int64)[:, :, None]
        assert np.all(np.abs(held - x) <= np.abs(x) / 16 + 2 * 2.0 ** (s - 137))    # (halves of steps that double add up to less than a step)


def test_rows_of_a_block_anywhere_in_a_call():
    """Two sequences' tokens interleaved, backwards and between rows that go nowhere, by the scan and by the list."""
    D, P, rng = 128, 64, np.random.default_rng(2)
    for rows in (200, 3000, 20000):
        slots = np.full(rows, -1, np.int32)
        places = rng.permutation(rows)[:150]
        slots[places] = np.concatenate([np.arange(40, 115), np.arange(64 * 4 + 74, 64 * 4 - 1, -1)])
        _store_and_check(_rows(rng, rows, 1, D), _rows(rng, rows, 1, D), slots, _pool(rows, 6, 1, P, D), D, P)


def test_every_bf16_value_is_rounded_as_the_format_says():
    """All 65536 bit patterns, sorted by magnitude (blocks of neighbours) and shuffled in blocks of a few exponents, subnormal ones and the ends among them."""
    bits = np.arange(1 << 16).astype(np.uint16)
    x = torch.from_numpy(bits.view(np.int16).copy()).view(torch.bfloat16)
    order = x.float().abs().nan_to_num(0.0, posinf=0.0).argsort(stable=True)
    near = x[order]
    rng = np.random.default_rng(5)
    mixed = near.view(-1, 1 << 13)[:, torch.from_numpy(rng.permutation(1 << 13))].reshape(-1)   # (a few dozen exponents a block)
    P, D = 64, 128
    k, v = torch.cat([near, mixed]).view(-1, 1, D), torch.cat([mixed.neg(), near]).view(-1, 1, D)
    slots = np.arange(len(k), dtype=np.int32)
    _store_and_check(k, v, slots, np.zeros((len(k) // P, 1, paged_fp8.page_head_bytes(D, P)), np.uint8), D, P)


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
    fspad.fspad_kv_store_paged_byte(k, v, s, both[:, 1])
    torch.cuda.synchronize()
    assert torch.equal(both[:, 0], before[:, 0])
    ref = paged_fp8.Fp8Pages(before[:, 1].cpu().numpy().copy(), D, P)
    ref.store("k", k.cpu().double().numpy(), slots)
    ref.store("v", v.cpu().double().numpy(), slots)
    _same(both[:, 1].cpu().numpy(), ref.raw, D, P, slots)
    cache = torch.full((2, 2, Hkv, L, D), 7.0, dtype=torch.bfloat16, device=DEV)     # K and V caches [B, Hkv, L, D]
    part = [c[1, :, 5:5 + rows].transpose(0, 1) for c in cache]
    fspad.fspad_kv_load_paged_byte(s, both[:, 1], D, outputs=part)
    torch.cuda.synchronize()
    for which, p, c in zip("kv", part, cache):
        assert np.array_equal(p.cpu().double().numpy(), ref.get_many(which, slots))
        assert bool((c[0] == 7).all()) and bool((c[1, :, :5] == 7).all()) and bool((c[1, :, 5 + rows:] == 7).all())
    # one head for all: a stride of zero is read as often as there are rows
    wide = k[:, :1].expand(rows, Hkv, D)
    fspad.fspad_kv_store_paged_byte(wide, wide, s, both[:, 0])
    got = fspad.fspad_kv_load_paged_byte(s, both[:, 0], D)
    assert all(torch.equal(got[0][:, 0], got[0][:, g]) for g in range(Hkv) if bool((both[:, 0, 0, 2 * P * D:] == both[:, 0, g, 2 * P * D:]).all()))


def test_no_rows_repeated_loads_and_any_order():
    D, P, rng = 128, 64, np.random.default_rng(4)
    raw = _pool(3, 5, 2, P, D)
    pool = torch.from_numpy(raw).to(DEV)
    none = torch.empty((0, 2, D), dtype=torch.bfloat16, device=DEV)
    fspad.fspad_kv_store_paged_byte(none, none, torch.empty(0, dtype=torch.int32, device=DEV), pool)
    k, v = fspad.fspad_kv_load_paged_byte(torch.empty(0, dtype=torch.int32, device=DEV), pool, D)
    assert k.shape == v.shape == (0, 2, D) and np.array_equal(pool.cpu().numpy(), raw)
    ref = paged_fp8.Fp8Pages(raw, D, P)
    for slots in ([5, 5, 31, 5], rng.integers(0, 5 * P, 77), np.arange(7, 300), [17, -5, 5 * P, 2 ** 31 - 1, 18]):
        slots = np.asarray(slots, np.int32)
        got = fspad.fspad_kv_load_paged_byte(torch.from_numpy(slots).to(DEV), pool, D)
        inside = (slots >= 0) & (slots < 5 * P)
        for which, x in zip("kv", got):
            want = np.where(inside[:, None, None], ref.get_many(which, np.where(inside, slots, 0)), 0.0)
            assert np.array_equal(x.cpu().double().numpy(), want, equal_nan=True)


def test_slots_and_pages_past_32_bits_of_bytes():
    """A pool of more than 4 GB: what goes to its last page does not come round to its first."""
    D, P, Hkv = 128, 256, 8
    per = fspad.fspad_kv_page_bytes_byte(Hkv, D, P)
    n_pages = (1 << 32) // per + 40
    pool = torch.zeros((n_pages, Hkv, per // Hkv), dtype=torch.uint8, device=DEV)
    x = _bf16(np.random.default_rng(8).standard_normal((3, Hkv, D))).to(DEV)
    slots = torch.tensor([n_pages * P - 32, 0, (n_pages - 30) * P + 64], dtype=torch.int32, device=DEV)
    fspad.fspad_kv_store_paged_byte(x, -x, slots, pool)
    k, v = fspad.fspad_kv_load_paged_byte(slots, pool, D)
    torch.cuda.synchronize()
    assert torch.equal(k, -v) and bool(((k - x).abs() <= x.abs() / 16 + 2.0 ** -16).all())
    used = torch.zeros(n_pages, dtype=torch.bool, device=DEV)
    used[[0, n_pages - 30, n_pages - 1]] = True
    assert bool((pool.view(n_pages, -1).amax(1) > 0).eq(used).all())


def test_as_many_rows_as_a_call_takes():
    """One row, repeated by a stride of zero, into every slot of a million; then all of them back."""
    D, P, rows = 64, 64, 1048560
    rng = np.random.default_rng(1)
    k, v = (_bf16(rng.standard_normal((1, 1, D))).to(DEV) for _ in range(2))
    pages = torch.zeros((-(-rows // P), 1, paged_fp8.page_head_bytes(D, P)), dtype=torch.uint8, device=DEV)
    slots = torch.arange(rows, dtype=torch.int32, device=DEV).flip(0).contiguous()
    fspad.fspad_kv_store_paged_byte(k.expand(rows, 1, D), v.expand(rows, 1, D), slots, pages)
    got = fspad.fspad_kv_load_paged_byte(slots, pages, D)
    one = paged_fp8.Fp8Pages(np.zeros((1, 1, paged_fp8.page_head_bytes(D, P)), np.uint8), D, P)
    for which, x, g in zip("kv", (k, v), got):
        one.store(which, x.cpu().double().numpy(), [0])
        want = torch.from_numpy(one.get_many(which, [0])[0, 0]).to(torch.bfloat16).to(DEV)
        assert bool((g[:, 0] == want).all())
