"""CPU-only checks of the paged cache's boundary: sizes, and everything that is refused before a launch."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from paper_2408_15562_amd import binding

P16 = 4096      # stands for a device address that is 16-byte aligned: no call below gets as far as using it
OK, NULL, SHAPE, DTYPE, WORKSPACE = 0, 1, 2, 4, 5


@pytest.fixture(scope="module")
def lib():
    return binding._lib()


def _desc(**kw):
    d = fspad.fspad_paged_desc()
    values = dict(batch=2, n_nodes_max=26, n_q_heads=8, n_kv_heads=2, head_dim=128, io_dtype=1, out_dtype=1, softmax_scale=0.0, page_tokens=16,
                  n_pages=10, page_stride=2 * 2176, table_width=5, max_kv_len=80, table_stride=5, workgroups=0)
    values.update(kw)
    for name, value in values.items():
        setattr(d, name, value)
    return d


@pytest.mark.parametrize("hkv,D,P,want", [(1, 64, 16, 1088), (8, 128, 64, 8 * 8704), (52, 128, 256, 52 * 34816), (0, 64, 16, 0), (1, 96, 16, 0),
                                          (1, 64, 8, 0), (1, 64, 48, 0), (1, 64, 512, 0), (-1, 64, 16, 0)])
def test_page_bytes(hkv, D, P, want):
    assert fspad.fspad_kv_page_bytes(hkv, D, P) == want


@pytest.mark.parametrize("change", [dict(n_kv_heads=0), dict(head_dim=96), dict(page_tokens=24), dict(page_tokens=8), dict(n_pages=0),
                                    dict(page_stride=2 * 2176 - 16), dict(page_stride=2 * 2176 + 8), dict(page_stride=1 << 32), dict(n_pages=1 << 27), dict(n_kv_heads=65536),
                                    dict(n_kv_heads=1 << 30)])
def test_store_and_load_refuse_shapes(lib, change):
    d = _desc(**change)
    assert lib.fspad_kv_store_paged(ctypes.byref(d), 3, P16, P16, 256, 128, P16, P16, None) == SHAPE
    assert lib.fspad_kv_load_paged(ctypes.byref(d), 3, P16, P16, P16, P16, 256, 128, None) == SHAPE


def test_store_and_load_refuse_arguments(lib):
    d = ctypes.byref(_desc())
    store = lambda rows=3, k=P16, v=P16, rs=256, hs=128, slots=P16, pages=P16, desc=d: lib.fspad_kv_store_paged(desc, rows, k, v, rs, hs, slots, pages, None)  # noqa: E731
    load = lambda rows=3, k=P16, v=P16, rs=256, hs=128, slots=P16, pages=P16, desc=d: lib.fspad_kv_load_paged(desc, rows, slots, pages, k, v, rs, hs, None)  # noqa: E731
    for call in (store, load):
        assert call(desc=None) == NULL
        assert call(desc=ctypes.byref(_desc(io_dtype=0))) == DTYPE
        assert call(rows=-1) == SHAPE
        assert call(rows=0, k=None, v=None, slots=None, pages=None) == OK
        for name in ("k", "v", "slots", "pages"):
            assert call(**{name: None}) == NULL
        for name in ("k", "v", "pages"):
            assert call(**{name: P16 + 8}) == SHAPE
        for bad in (dict(rs=252), dict(hs=4), dict(rs=-256), dict(hs=-128)):
            assert call(**bad) == SHAPE
    assert load(hs=64) == SHAPE and load(rs=64) == SHAPE     # rows that overlap


ATTN_SHAPES = [dict(batch=0), dict(batch=1025), dict(n_nodes_max=0), dict(n_nodes_max=65), dict(n_q_heads=0), dict(n_q_heads=7), dict(head_dim=32),
               dict(page_tokens=0), dict(n_pages=0), dict(page_stride=64), dict(table_width=0, max_kv_len=0), dict(table_stride=4), dict(max_kv_len=81),
               dict(max_kv_len=-1), dict(workgroups=-1), dict(workgroups=4097), dict(n_q_heads=2 * (1 << 17), n_nodes_max=64),
               dict(batch=1024, n_kv_heads=64, n_q_heads=64, page_stride=64 * 2176, table_width=1 << 20, table_stride=1 << 20, max_kv_len=1 << 24)]


@pytest.mark.parametrize("change", ATTN_SHAPES)
def test_attention_refuses_shapes(lib, change):
    d = _desc(**change)
    assert fspad.fspad_tree_attn_paged_workspace_bytes(d) == 0
    assert lib.fspad_tree_attn_paged(ctypes.byref(d), *[P16] * 9, P16, 1 << 40, None) == SHAPE


def test_attention_refuses_arguments(lib):
    d = _desc()
    need = fspad.fspad_tree_attn_paged_workspace_bytes(d)
    assert need > 0

    def call(at=None, value=None, desc=d, ws=P16, ws_bytes=need):
        args = [P16] * 9
        if at is not None:
            args[at] = value
        return lib.fspad_tree_attn_paged(ctypes.byref(desc) if desc is not None else None, *args, ws, ws_bytes, None)
    assert call(desc=None) == NULL
    for at in range(9):
        assert call(at, None) == NULL
    for at in (0, 1, 2, 3, 8):
        assert call(at, P16 + 8) == SHAPE
    for scale in (float("nan"), float("inf"), -float("inf"), 1e-45, 3e38):
        assert call(desc=_desc(softmax_scale=scale)) == SHAPE
    assert call(desc=_desc(io_dtype=0)) == DTYPE and call(desc=_desc(out_dtype=2)) == DTYPE
    assert call(ws=None) == WORKSPACE and call(ws_bytes=need - 1) == WORKSPACE and call(ws=P16 + 4) == WORKSPACE


@pytest.mark.parametrize("change", [dict(B=0), dict(B=2049), dict(P=12), dict(n_pages=0), dict(n_pages=1 << 28), dict(width=0), dict(stride=4),
                                    dict(width=1 << 28, stride=1 << 28), dict(B=2048, width=1 << 20, stride=1 << 20), dict(max_new=-1),
                                    dict(max_new=65, path=P16), dict(max_new=0, path=P16), dict(max_new=0, n_slots=-1), dict(max_new=0, n_slots=(1 << 22) + 1),
                                    dict(B=2048, max_new=1 << 20)])
def test_page_map_refuses_shapes(lib, change):
    a = dict(B=3, P=16, n_pages=20, width=5, stride=5, path=None, max_new=4, n_slots=0)
    a.update(change)
    assert lib.fspad_page_map(a["B"], a["P"], a["n_pages"], a["width"], a["stride"], P16, P16, a["path"], a["max_new"], a["n_slots"], *[P16] * 7,
                              None) == SHAPE


def test_page_map_refuses_arguments(lib):
    for at in range(9):       # kv_len, n_new, then block_table .. granted
        p = [P16] * 9
        p[at] = None
        assert lib.fspad_page_map(3, 16, 20, 5, 5, p[0], p[1], None, 4, 0, *p[2:], None) == NULL


@pytest.mark.parametrize("N,Hq,Hkv,D", [(1, 8, 8, 64), (1, 64, 1, 128), (26, 8, 8, 128), (60, 32, 8, 128), (64, 64, 8, 64), (64, 71, 1, 128)])
@pytest.mark.parametrize("B,L", [(1, 0), (1, 1), (3, 700), (64, 4096)])
@pytest.mark.parametrize("workgroups", [0, 1, 333])
def test_workspace_holds_a_slot_for_every_piece(N, Hq, Hkv, D, B, L, workgroups):
    """Where units can be cut: a slot for every unit and for every workgroup asked for beside them (or for every block, if there are fewer)."""
    d = _desc(batch=B, n_nodes_max=N, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, page_stride=Hkv * 17 * D, max_kv_len=L, table_width=300, table_stride=300,
              workgroups=workgroups)
    need = fspad.fspad_tree_attn_paged_workspace_bytes(d)
    rows = N * (Hq // Hkv)
    per_group = next(r for r in (16, 32, 64) if rows <= r or r == 64)
    units = B * Hkv * -(-rows // per_group)
    blocks = units * (-(-L // 32) + -(-N // 32))
    slot = per_group * (D + 2) * 4
    if workgroups or L >= 4096:
        assert need >= units * 8 + (units + min(workgroups or 256, blocks)) * slot
    assert units * 8 <= need <= 16 + units * 8 + (units + (workgroups or 2048)) * slot


def test_binding_refuses_tensors():
    pages = torch.zeros((4, 2, 2176), dtype=torch.uint8)
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        fspad.fspad_kv_store_paged(k, k, slots, pages)                       # host tensors
    with pytest.raises(ValueError):
        fspad.fspad_kv_store_paged(k.float(), k, slots, pages)
    with pytest.raises(ValueError):
        fspad.fspad_kv_store_paged(k, k[:2], slots, pages)
    with pytest.raises(ValueError):
        fspad.fspad_kv_store_paged(k, k, slots.long(), pages)
    with pytest.raises(ValueError):
        fspad.fspad_kv_store_paged(k, k, slots, pages[:, :1])
    with pytest.raises(ValueError):
        fspad.fspad_kv_store_paged(k, torch.zeros((3, 2, 256), dtype=torch.bfloat16)[:, :, ::2], slots, pages)
    with pytest.raises(ValueError):
        fspad.fspad_kv_load_paged(slots, pages[:, :, :2000], 128)
    with pytest.raises(ValueError):
        fspad.fspad_kv_load_paged(slots, pages.permute(1, 0, 2), 128)
    q = torch.zeros((1, 3, 4, 128), dtype=torch.bfloat16)
    kt = torch.zeros((1, 3, 2, 128), dtype=torch.bfloat16)
    one, mask, table = torch.ones(1, dtype=torch.int32), torch.ones((1, 3), dtype=torch.int64), torch.zeros((1, 2), dtype=torch.int32)
    good = dict(q=q, k_tree=kt, v_tree=kt, pages=pages, block_table=table, kv_len=one, n_nodes=one, anc_mask=mask)
    for name, bad in (("k_tree", kt[:, :2]), ("v_tree", kt.float()), ("pages", pages[:, :1]), ("block_table", table.long()), ("kv_len", one.long()),
                      ("n_nodes", torch.ones(2, dtype=torch.int32)), ("anc_mask", mask.int()), ("anc_mask", mask[:, :2]), ("q", q.transpose(1, 2))):
        with pytest.raises(ValueError):
            fspad.fspad_tree_attn_paged(**{**good, name: bad})
    with pytest.raises(ValueError):
        fspad.fspad_tree_attn_paged(**good, out=torch.zeros((1, 3, 4, 64), dtype=torch.bfloat16))
    length = torch.zeros(2, dtype=torch.int32)
    table, free = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(6, dtype=torch.int32)
    for kw in (dict(), dict(max_new=2, n_slots=3), dict(max_new=0), dict(n_slots=4, path=table), dict(max_new=2, path=table)):
        with pytest.raises(ValueError):
            fspad.fspad_page_map(length, length, table, free, one, 16, **kw)
    with pytest.raises(ValueError):
        fspad.fspad_page_map(length, length, table[:1], free, one, 16, max_new=2)
    assert np.array_equal(table.numpy(), np.zeros((2, 3)))
