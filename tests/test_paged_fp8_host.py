"""CPU-only checks of the paged 8-bit cache's boundary: sizes, and everything that is refused before a launch."""
import ctypes

import pytest
import torch

import paper_2408_15562_amd as fspad
from paper_2408_15562_amd import binding

P16 = 4096      # stands for a device address that is 16-byte aligned: no call below gets as far as using it
OK, NULL, SHAPE, DTYPE, WORKSPACE = 0, 1, 2, 4, 5
PER = 2 * 32 * 128 + 16


@pytest.fixture(scope="module")
def lib():
    return binding._lib()


def _desc(**kw):
    d = fspad.fspad_paged_desc()
    values = dict(batch=2, n_nodes_max=26, n_q_heads=8, n_kv_heads=2, head_dim=128, io_dtype=1, out_dtype=1, softmax_scale=0.0, page_tokens=32,
                  n_pages=10, page_stride=2 * PER, table_width=5, max_kv_len=160, table_stride=5, workgroups=0)
    values.update(kw)
    for name, value in values.items():
        setattr(d, name, value)
    return d


@pytest.mark.parametrize("hkv,D,P,want", [(1, 64, 32, 4112), (8, 128, 64, 8 * 16400), (52, 128, 256, 52 * 65552), (0, 64, 32, 0), (1, 96, 32, 0),
                                          (1, 64, 16, 0), (1, 64, 48, 0), (1, 64, 512, 0), (-1, 64, 32, 0)])
def test_page_bytes(hkv, D, P, want):
    assert fspad.fspad_kv_page_bytes_byte(hkv, D, P) == want


@pytest.mark.parametrize("change", [dict(n_kv_heads=0), dict(head_dim=96), dict(page_tokens=48), dict(page_tokens=16), dict(n_pages=0),
                                    dict(page_stride=2 * PER - 16), dict(page_stride=2 * PER + 8), dict(page_stride=1 << 32), dict(n_pages=1 << 26),
                                    dict(n_kv_heads=65536), dict(n_kv_heads=1 << 30)])
def test_store_and_load_refuse_shapes(lib, change):
    d = _desc(**change)
    assert lib.fspad_kv_store_paged_byte(ctypes.byref(d), 3, P16, P16, 256, 128, P16, P16, None, 0, None) == SHAPE
    assert lib.fspad_kv_load_paged_byte(ctypes.byref(d), 3, P16, P16, P16, P16, 256, 128, None) == SHAPE
    assert fspad.fspad_kv_store_paged_byte_workspace_bytes(d, 50000) == 0


def test_store_and_load_refuse_arguments(lib):
    d = ctypes.byref(_desc())
    store = lambda rows=3, k=P16, v=P16, rs=256, hs=128, slots=P16, pages=P16, desc=d: lib.fspad_kv_store_paged_byte(  # noqa: E731
        desc, rows, k, v, rs, hs, slots, pages, None, 0, None)
    load = lambda rows=3, k=P16, v=P16, rs=256, hs=128, slots=P16, pages=P16, desc=d: lib.fspad_kv_load_paged_byte(  # noqa: E731
        desc, rows, slots, pages, k, v, rs, hs, None)
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
    assert store(rows=1048561) == SHAPE


def test_store_of_many_rows_needs_a_workspace(lib):
    d = _desc()
    assert [fspad.fspad_kv_store_paged_byte_workspace_bytes(d, r) for r in (0, 1, 2048, 2049, 90000)] == [0, 0, 0, 1280, 1280]
    call = lambda ws, n: lib.fspad_kv_store_paged_byte(ctypes.byref(d), 2049, P16, P16, 256, 128, P16, P16, ws, n, None)  # noqa: E731
    assert call(None, 1280) == WORKSPACE and call(P16, 1279) == WORKSPACE and call(P16 + 8, 1280) == WORKSPACE


ATTN_SHAPES = [dict(batch=0), dict(batch=1025), dict(n_nodes_max=0), dict(n_nodes_max=65), dict(n_q_heads=0), dict(n_q_heads=7), dict(head_dim=32),
               dict(page_tokens=0), dict(page_tokens=16), dict(n_pages=0), dict(page_stride=64), dict(table_width=0, max_kv_len=0), dict(table_stride=4),
               dict(max_kv_len=161), dict(max_kv_len=-1), dict(workgroups=-1), dict(workgroups=4097), dict(n_q_heads=2 * (1 << 17), n_nodes_max=64),
               dict(batch=1024, n_kv_heads=64, n_q_heads=64, page_stride=64 * PER, table_width=1 << 19, table_stride=1 << 19, max_kv_len=1 << 24)]


@pytest.mark.parametrize("change", ATTN_SHAPES)
def test_attention_refuses_shapes(lib, change):
    d = _desc(**change)
    assert fspad.fspad_tree_attn_paged_byte_workspace_bytes(d) == 0
    assert lib.fspad_tree_attn_paged_byte(ctypes.byref(d), *[P16] * 9, P16, 1 << 40, None) == SHAPE


@pytest.mark.parametrize("batch,nodes,heads,group,max_kv_len,rows,cut", [
    (12, 60, 8, 4, 2000, 128, False), (12, 60, 8, 4, 100000, 128, True),     # 768 slabs of 32 rows: four of them a workgroup, whatever the length
    (11, 60, 8, 4, 2000, 32, False), (11, 60, 8, 4, 34 * 32, 64, False), (11, 60, 8, 4, 70 * 32 + 1, 64, True),   # fewer
    (12, 8, 32, 8, 2000, 32, False), (12, 8, 32, 8, 71 * 32, 32, False),     # rows of one slab or two: one a workgroup, up to 72 blocks
    (12, 8, 32, 8, 71 * 32 + 1, 64, True),
    (4, 60, 8, 4, 70 * 32, 32, False), (4, 60, 8, 4, 254 * 32, 32, False), (4, 60, 8, 4, 254 * 32 + 1, 32, True), (5, 60, 8, 4, 100000, 64, True), (1, 20, 32, 8, 9946, 64, True),
    (1, 60, 8, 4, 160, 32, False), (4, 40, 8, 1, 160, 32, False)])
def test_attention_groups_rows(lib, batch, nodes, heads, group, max_kv_len, rows, cut):
    _groups_rows(128, batch, nodes, heads, group, max_kv_len, rows, cut)


@pytest.mark.parametrize("batch,nodes,heads,group,max_kv_len,rows,cut", [
    (12, 60, 8, 4, 94 * 32, 128, False), (12, 60, 8, 4, 94 * 32 + 1, 64, True), (24, 60, 8, 4, 94 * 32 + 1, 128, True), (11, 60, 8, 4, 34 * 32, 32, False),
    (1, 60, 8, 4, 256, 32, False), (1, 60, 8, 4, 257, 32, False)])
def test_attention_groups_rows_of_64_channels(lib, batch, nodes, heads, group, max_kv_len, rows, cut):
    _groups_rows(64, batch, nodes, heads, group, max_kv_len, rows, cut)


def _groups_rows(D, batch, nodes, heads, group, max_kv_len, rows, cut):
    """The workspace has a word pair for each unit, and slots of a unit's rows where units may be cut: it tells how rows are grouped."""
    d = _desc(batch=batch, n_kv_heads=heads, n_q_heads=heads * group, n_nodes_max=nodes, max_kv_len=max_kv_len, head_dim=D, page_stride=heads * (2 * 32 * D + 16),
              table_width=4096, table_stride=4096)
    need, words = fspad.fspad_tree_attn_paged_byte_workspace_bytes(d), batch * heads * -(-nodes * group // rows) * 8
    assert (need > words) == cut and (need - words) % (rows * (D + 2) * 4) == 0


def test_attention_refuses_arguments(lib):
    d = _desc()
    need = fspad.fspad_tree_attn_paged_byte_workspace_bytes(d)
    assert need > 0

    def call(at=None, value=None, desc=d, ws=P16, ws_bytes=need):
        args = [P16] * 9
        if at is not None:
            args[at] = value
        return lib.fspad_tree_attn_paged_byte(ctypes.byref(desc) if desc is not None else None, *args, ws, ws_bytes, None)
    assert call(desc=None) == NULL
    for at in range(9):
        assert call(at, None) == NULL
    for at in (0, 1, 2, 3, 8):
        assert call(at, P16 + 8) == SHAPE
    for scale in (float("nan"), float("inf"), -float("inf"), 1e-45, 3e38):
        assert call(desc=_desc(softmax_scale=scale)) == SHAPE
    assert call(desc=_desc(io_dtype=0)) == DTYPE and call(desc=_desc(out_dtype=2)) == DTYPE
    assert call(ws=None) == WORKSPACE and call(ws_bytes=need - 1) == WORKSPACE and call(ws=P16 + 4) == WORKSPACE


def test_binding_refuses_tensors():
    pages = torch.zeros((4, 2, PER), dtype=torch.uint8)
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int32)
    for args in ((k, k, slots, pages), (k.float(), k, slots, pages), (k, k[:2], slots, pages), (k, k, slots.long(), pages), (k, k, slots, pages[:, :1]),
                 (k, k, slots, pages[:, :, :PER - 2]), (k, k, slots, pages[:, :, :8])):
        with pytest.raises(ValueError):      # (the first: host tensors)
            fspad.fspad_kv_store_paged_byte(*args)
    with pytest.raises(ValueError):
        fspad.fspad_kv_load_paged_byte(slots, pages[:, :, :2000], 128)
    with pytest.raises(ValueError):
        fspad.fspad_kv_load_paged_byte(slots, pages.permute(1, 0, 2), 128)
    q = torch.zeros((1, 3, 4, 128), dtype=torch.bfloat16)
    kt = torch.zeros((1, 3, 2, 128), dtype=torch.bfloat16)
    one, mask, table = torch.ones(1, dtype=torch.int32), torch.ones((1, 3), dtype=torch.int64), torch.zeros((1, 2), dtype=torch.int32)
    good = dict(q=q, k_tree=kt, v_tree=kt, pages=pages, block_table=table, kv_len=one, n_nodes=one, anc_mask=mask)
    desc = fspad.make_paged_desc(q, kt, pages, table, fp8=True)
    assert desc.page_tokens == 32 and desc.page_stride == 2 * PER and desc.max_kv_len == 64
    four = fspad.make_paged_desc(q, kt, torch.zeros((4, 2, 4352), dtype=torch.uint8), table)
    assert four.page_tokens == 32
    for name, bad in (("k_tree", kt[:, :2]), ("v_tree", kt.float()), ("pages", pages[:, :1]), ("pages", torch.zeros((4, 2, 4352 + 2), dtype=torch.uint8)),
                      ("block_table", table.long()), ("kv_len", one.long()), ("n_nodes", torch.ones(2, dtype=torch.int32)), ("anc_mask", mask.int()),
                      ("anc_mask", mask[:, :2]), ("q", q.transpose(1, 2))):
        with pytest.raises(ValueError):
            fspad.fspad_tree_attn_paged_byte(**{**good, name: bad})
    bad = fspad.make_paged_desc(q, kt, pages, table, fp8=True)
    bad.n_pages = 5
    with pytest.raises(ValueError):
        fspad.fspad_tree_attn_paged_byte(**good, desc=bad)
