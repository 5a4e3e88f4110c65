"""CPU-only: a descriptor that the caller of fspad_tree_attn_paged brings has to agree with the tensors beside it."""
import pytest
import torch

import paper_2408_15562_amd as fspad


def _attn_tensors(B=2, n_pages=4, width=3):
    q, kt = torch.zeros((B, 3, 4, 128), dtype=torch.bfloat16), torch.zeros((B, 3, 2, 128), dtype=torch.bfloat16)
    one = torch.ones(B, dtype=torch.int32)
    return dict(q=q, k_tree=kt, v_tree=kt, pages=torch.zeros((n_pages, 2, 2176), dtype=torch.uint8), block_table=torch.zeros((B, width), dtype=torch.int32),
                kv_len=one, n_nodes=one, anc_mask=torch.ones((B, 3), dtype=torch.int64))


def _call_with(desc, tensors, **kw):
    """What the call refuses; a call that gets past the descriptor is refused for its tensors, which lie on the host."""
    with pytest.raises(ValueError) as e:
        fspad.fspad_tree_attn_paged(**tensors, desc=desc, **kw)
    return str(e.value) != "q must be a device tensor", str(e.value)


def _made(t, **kw):
    return fspad.make_paged_desc(t["q"], t["k_tree"], t["pages"], t["block_table"], **kw)


def test_binding_refuses_a_descriptor_of_other_tensors():
    """Shapes of the descriptor that are not the tensors': pools, tables and trees that the call would read or write past."""
    t = _attn_tensors()
    assert not _call_with(_made(t), t)[0]
    for name, value in (("batch", 3), ("batch", 1), ("n_nodes_max", 4), ("n_nodes_max", 2), ("n_q_heads", 8), ("n_kv_heads", 4), ("n_kv_heads", 1), ("head_dim", 64),
                        ("io_dtype", 0), ("page_tokens", 32), ("n_pages", 5), ("page_stride", 2 * 2 * 2176), ("table_width", 4), ("table_stride", 4)):
        desc = _made(t)
        setattr(desc, name, value)
        refused, why = _call_with(desc, t)
        assert refused and name in why, (name, value, why)
    for name, value in (("n_pages", 3), ("table_width", 2), ("max_kv_len", 7)):   # less than there is
        desc = _made(t)
        setattr(desc, name, value)
        assert not _call_with(desc, t)[0]
    one = _attn_tensors(B=1, n_pages=1)
    for name in ("page_stride", "table_stride"):   # (of one page, of one row)
        desc = _made(one)
        setattr(desc, name, 1 << 16)
        assert not _call_with(desc, one)[0]


@pytest.mark.parametrize("name,bad", [("block_table", lambda t: t["block_table"].long()), ("block_table", lambda t: t["block_table"][:1]),
                                      ("block_table", lambda t: t["block_table"][:, :2]), ("block_table", lambda t: torch.zeros((2, 6), dtype=torch.int32)[:, ::2]),
                                      ("block_table", lambda t: torch.zeros((2, 6), dtype=torch.int32)[:, :3]), ("pages", lambda t: t["pages"][:3]),
                                      ("pages", lambda t: t["pages"][:, :1]), ("pages", lambda t: torch.zeros((4, 2, 4352), dtype=torch.uint8)),
                                      ("pages", lambda t: torch.zeros((8, 2, 2176), dtype=torch.uint8)[::2]), ("pages", lambda t: t["pages"].char())])
def test_binding_refuses_tensors_beside_a_descriptor(name, bad):
    t = _attn_tensors()
    refused, why = _call_with(_made(t), {**t, name: bad(t)})
    assert refused, why


def test_binding_refuses_arguments_that_a_descriptor_contradicts():
    t = _attn_tensors()
    desc = _made(t, max_kv_len=40, softmax_scale=0.3, out_dtype=torch.float32, workgroups=7)
    for kw in (dict(max_kv_len=41), dict(softmax_scale=0.25), dict(out_dtype=torch.bfloat16), dict(workgroups=6)):
        refused, why = _call_with(desc, t, **kw)
        assert refused and next(iter(kw)) in why
    for kw in (dict(), dict(max_kv_len=40), dict(softmax_scale=0.3), dict(out_dtype=torch.float32), dict(workgroups=7)):
        assert not _call_with(desc, t, **kw)[0]
