"""CPU-only checks of the shared pages' boundary: sizes, and everything that is refused before a launch."""
import pytest
import torch

import paper_2408_15562_amd as fspad
from paper_2408_15562_amd import binding

A = 4096      # stands for a device address: no call below gets as far as using it
OK, NULL, SHAPE, WORKSPACE = 0, 1, 2, 5


@pytest.fixture(scope="module")
def lib():
    return binding._lib()


TABLES = [dict(B=0), dict(B=2049), dict(P=12), dict(P=512), dict(n_pages=0), dict(n_pages=(1 << 19) + 1), dict(width=0), dict(stride=4), dict(width=1 << 28, stride=1 << 28),
          dict(B=2048, width=1 << 20, stride=1 << 20)]


def _table(change):
    a = dict(B=3, P=16, n_pages=20, width=5, stride=5)
    a.update(change)
    return a["B"], a["P"], a["n_pages"], a["width"], a["stride"]


@pytest.mark.parametrize("change", TABLES)
def test_tables_are_refused(lib, change):
    t = _table(change)
    assert lib.fspad_page_fork(*t, 2, *[A] * 14, None) == SHAPE
    assert lib.fspad_page_release(*t, *[A] * 9, A, 1 << 30, None) == SHAPE
    assert lib.fspad_page_compact(*t, t[4], *[A] * 10, None) == SHAPE


def test_fork_refuses_arguments(lib):
    t = _table({})
    for n in (2049, -1):
        assert lib.fspad_page_fork(*t, n, *[A] * 14, None) == SHAPE
    for at in range(14):
        p = [A] * 14
        p[at] = None
        if at != 2:                # n_tokens
            assert lib.fspad_page_fork(*t, 2, *p, None) == NULL


def test_release_refuses_arguments(lib):
    t = _table({})
    assert fspad.fspad_page_release_workspace_bytes(3, 20, 5) == 0 == fspad.fspad_page_release_workspace_bytes(0, 20, 5)
    need = fspad.fspad_page_release_workspace_bytes(3, 40000, 5)
    assert need == 4 * (1 + 10) and fspad.fspad_page_release_workspace_bytes(1024, 16384, 300) == 0
    for at in range(9):
        p = [A] * 9
        p[at] = None
        assert lib.fspad_page_release(*t, *p, None, 0, None) == NULL
    big = _table(dict(n_pages=40000))
    assert [lib.fspad_page_release(*big, *[A] * 9, ws, n, None) for ws, n in ((None, need), (A, need - 1), (A + 8, need))] == [WORKSPACE] * 3


def test_compact_refuses_arguments(lib):
    t = _table({})
    for at in range(10):
        p = [A] * 10
        p[at] = None
        assert lib.fspad_page_compact(*t, 5, *p, None) == NULL
    assert lib.fspad_page_compact(*t, 4, *[A] * 10, None) == SHAPE
    assert lib.fspad_page_compact(*t, 6, *[A] * 10, None) == SHAPE         # the table in place with a stride of its own


def test_copy_refuses_arguments(lib):
    call = lambda pages=A, n_pages=4, stride=64, size=48, n=3, src=A, dst=A: lib.fspad_page_copy(pages, n_pages, stride, size, n, src, dst, None)  # noqa: E731
    for bad in (dict(n_pages=0), dict(size=0), dict(size=40), dict(size=80), dict(stride=72), dict(stride=1 << 32), dict(stride=1 << 31, size=1 << 31), dict(n=-1), dict(pages=A + 8)):
        assert call(**bad) == SHAPE
    for name in ("pages", "src", "dst"):
        assert call(**{name: None}) == NULL
    assert call(n=0, pages=None, src=None, dst=None) == OK


def test_binding_refuses_tensors():
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    good = dict(src=i(2), dst=i(2), kv_len=i(3), block_table=i(3, 4), free_pages=i(9), n_free=i(1), shared=i(9))
    for name, bad in (("src", i(3)), ("dst", i(2).long()), ("kv_len", i(4)), ("block_table", i(4, 3).t()), ("n_free", i(2)), ("shared", i(8)), ("n_tokens", i(3))):
        with pytest.raises(ValueError):
            fspad.fspad_page_fork(**{**good, name: bad}, page_tokens=16)
    with pytest.raises(ValueError, match="device tensor"):
        fspad.fspad_page_fork(**good, page_tokens=16)                     # host tensors
    rest = {k: v for k, v in good.items() if k not in ("src", "dst")}
    for name, bad in (("ended", i(2)), ("ended", torch.zeros(3, dtype=torch.bool)), ("kv_len", i(2)), ("free_pages", i(10)), ("shared", i(9).float())):
        with pytest.raises(ValueError):
            fspad.fspad_page_release(**{**rest, "ended": i(3), name: bad}, page_tokens=16)
    for outputs in ((i(4), i(4), i(3, 5), i(9), i(9)), (i(5), i(4), i(3, 4), i(9), i(9)), (i(4), i(4), i(3, 4), i(8), i(9))):
        with pytest.raises(ValueError):
            fspad.fspad_page_compact(**rest, page_tokens=16, outputs=outputs)
    for src, pages in ((i(2), torch.zeros((4, 64), dtype=torch.int8)), (i(3), torch.zeros((4, 64), dtype=torch.uint8)), (i(2), torch.zeros(64, dtype=torch.uint8)),
                       (i(2), torch.zeros((4, 64, 2), dtype=torch.uint8).transpose(1, 2))):
        with pytest.raises(ValueError):
            fspad.fspad_page_copy(src, i(2), pages)
