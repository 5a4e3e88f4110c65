"""CPU-only: what a call takes for itself (workspaces and outputs that are not given) belongs to the stream that the call goes to, and outputs are held for the
current one too. Streams are stood in for by names; nothing is launched."""
import contextlib
import inspect

import numpy as np
import pytest
import torch

import paper_2408_15562_amd as fspad
from oracle import paged, paged_fp8
from paper_2408_15562_amd import binding

B, N, Hq, Hkv, D, V, Hd, I = 2, 4, 4, 2, 64, 256, 128, 128
WIDTH, N_PAGES, P = 3, 20000, 32   # pages for a release that needs a workspace


def _t(*shape, dtype=torch.int32):
    return torch.empty(shape, dtype=dtype, device="meta")


def _bf(*shape):
    return _t(*shape, dtype=torch.bfloat16)


def _f32(*shape):
    return _t(*shape, dtype=torch.float32)


def _i64(*shape):
    return _t(*shape, dtype=torch.int64)


HOST = np.full(B, 3, np.int32)
TREE = dict(draft_tokens=_t(B, N), parent=_t(B, N), n_nodes=_t(B))
TABLES = dict(kv_len=_t(B), block_table=_t(B, WIDTH), free_pages=_t(N_PAGES), n_free=_t(1), shared=_t(N_PAGES), page_tokens=P)
QKV = dict(q=_bf(B, N, Hq, D), k_tree=_bf(B, N, Hkv, D), v_tree=_bf(B, N, Hkv, D))
PAGED = dict(**QKV, block_table=_t(B, WIDTH), kv_len=_t(B), n_nodes=_t(B), anc_mask=_i64(B, N), workgroups=8)
FP4, FP8 = (_t(64, Hkv, per, dtype=torch.uint8) for per in (paged.page_head_bytes(D, P), paged_fp8.page_head_bytes(D, P)))
LAYER = {"w_qkv": _bf((Hq + 2 * Hkv) * D, Hd), "w_o": _bf(Hd, Hq * D), "w_gate": _bf(I, Hd), "w_up": _bf(I, Hd), "w_down": _bf(2 * Hd, I), "gain_attn": _bf(Hd),
         "gain_mlp": _bf(Hd)}
ROWS = 2100   # more than a store takes without a workspace

# entry point: its arguments, and how many tensors it takes for itself
CALLS = {
    "fspad_tree_attn": (dict(**QKV, k_cache=_bf(B, Hkv, 8, D), v_cache=_bf(B, Hkv, 8, D), kv_len=HOST, n_nodes=HOST, anc_mask=_i64(B, N)), 2),
    "fspad_tree_accept_greedy": (dict(logits=_f32(B, N, V), **TREE), 5),
    "fspad_tree_accept_greedy_static": (dict(logits=_f32(B, N, V), **TREE, outputs=(_t(B, N), _t(B), _t(B, N), _t(B))), 0),
    "fspad_tree_accept_sample": (dict(logits=_f32(B, N, V), **TREE, temperature=1.0, uniforms=_f32(B, 2, N)), 5),
    "fspad_tree_accept_sample_draft": (dict(logits=_f32(B, N, V), draft_logits=_f32(B, N, V), **TREE, temperature=1.0, uniforms=_f32(B, 2, N)), 5),
    "fspad_tree_accept_greedy_lm_head": (dict(hidden=_bf(B, N, Hd), lm_head=_bf(V, Hd), **TREE), 7),
    "fspad_tree_accept_sample_lm_head": (dict(hidden=_bf(B, N, Hd), lm_head=_bf(V, Hd), **TREE, temperature=1.0, uniforms=_f32(B, 2, N)), 5),
    "fspad_kv_commit": (dict(k_tree=QKV["k_tree"], v_tree=QKV["v_tree"], k_cache=_bf(B, Hkv, 8, D), v_cache=_bf(B, Hkv, 8, D), kv_len=HOST, path=_t(B, N),
                             path_len=_t(B)), 0),
    "fspad_pack_weight": (dict(w=_bf(32, 128)), 1),
    "fspad_feature_sampler": (dict(f=_bf(3, Hd), e=_bf(3, Hd), w_up=_bf(I, Hd), w_gate=_bf(I, Hd), w_down=_bf(Hd, I)), 2),
    "fspad_draft_layer": (dict(eta=_bf(B, N, Hd), positions=_t(B, N), weights=LAYER, k_cache=None, v_cache=None, kv_len=HOST * 0, n_nodes=HOST, anc_mask=_i64(B, N),
                               n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D), 5),
    "fspad_tree_attn_paged": (dict(**PAGED, pages=FP4), 2),
    "fspad_kv_store_paged": (dict(k=_bf(ROWS, Hkv, D), v=_bf(ROWS, Hkv, D), slots=_t(ROWS), pages=FP4), 0),
    "fspad_kv_load_paged": (dict(slots=_t(ROWS), pages=FP4, head_dim=D), 2),
    "fspad_page_map": (dict({k: TABLES[k] for k in ("kv_len", "block_table", "free_pages", "n_free", "page_tokens")}, n_new=_t(B), max_new=3), 4),
    "fspad_tree_attn_paged_byte": (dict(**PAGED, pages=FP8), 2),
    "fspad_kv_store_paged_byte": (dict(k=_bf(ROWS, Hkv, D), v=_bf(ROWS, Hkv, D), slots=_t(ROWS), pages=FP8), 1),
    "fspad_kv_load_paged_byte": (dict(slots=_t(ROWS), pages=FP8, head_dim=D), 2),
    "fspad_page_fork": (dict(src=_t(1), dst=_t(1), **TABLES), 6),
    "fspad_page_release": (dict(ended=_t(B), **TABLES), 4),
    "fspad_page_compact": (dict(**TABLES), 5),
    "fspad_page_copy": (dict(copy_src=_t(5), copy_dst=_t(5), pages=FP8), 0),
    "fspad_draft_topk": (dict(logits=_f32(3, V), k=4), 3),
    "fspad_tree_build": (dict(cand_parent=_t(B, 6), cand_token=_t(B, 6), cand_logp=_f32(B, 6), n_cand=_t(B), n_keep=3, n_max=4), 5),
}


class Stream:
    def __init__(self, cuda_stream):
        self.cuda_stream = cuda_stream


@pytest.fixture
def streams(monkeypatch):
    """Two streams, the first one current; what is taken while which is current, and which tensors are held for which."""
    class Seen:
        here, side, now, taken, held = Stream(1), Stream(2), None, [], []

    seen = Seen()
    seen.now, seen.taken, seen.held = seen.here, [], []

    @contextlib.contextmanager
    def use(stream):
        before, seen.now = seen.now, stream
        yield
        seen.now = before

    empty = torch.empty

    def taking(*shape, **kw):
        t = empty(*shape, **kw)
        seen.taken.append((seen.now.cuda_stream, t))
        return t

    monkeypatch.setattr(torch, "empty", taking)
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: seen.now)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda ptr, device=None: Stream(ptr))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: seen.held.append((stream.cuda_stream, id(t))))
    monkeypatch.setattr(binding, "_dev_ptr", lambda t, name, dtype=None: None)
    monkeypatch.setattr(binding, "_on_current_device", lambda *tensors: None)
    monkeypatch.setattr(binding, "_check", lambda status, where: None)   # (the one call that is not issued by _issue: refused for its pointers)
    monkeypatch.setattr(binding, "_issue", lambda fn, where, args, keep, result, prepare: args[-1])
    return seen


def test_every_call_with_a_stream_is_here():
    takes = {name for name, fn in vars(fspad).items() if name.startswith("fspad_") and callable(fn) and not inspect.isclass(fn)
             and "stream" in inspect.signature(fn).parameters}
    assert takes == set(CALLS)


@pytest.mark.parametrize("which", ["stream", "handle", "default"])
@pytest.mark.parametrize("name", CALLS)
def test_memory_is_taken_on_the_stream_of_the_call(streams, name, which):
    args, own = CALLS[name]
    ptr = 0 if which == "default" else streams.side.cuda_stream
    went_to = getattr(fspad, name)(**args, stream=streams.side if which == "stream" else ptr)
    assert name == "fspad_pack_weight" or went_to == ptr
    assert [at for at, _ in streams.taken] == [ptr] * own
    assert streams.held == [(streams.here.cuda_stream, id(t)) for _, t in streams.taken]


@pytest.mark.parametrize("which", ["none", "current", "its handle"])
@pytest.mark.parametrize("name", CALLS)
def test_nothing_is_held_on_the_current_stream(streams, name, which):
    args, own = CALLS[name]
    getattr(fspad, name)(**args, stream={"none": None, "current": Stream(1), "its handle": 1}[which])
    assert [at for at, _ in streams.taken] == [streams.here.cuda_stream] * own and not streams.held


def test_tensors_of_the_host_are_refused_as_before():
    args = {k: torch.zeros(v.shape, dtype=v.dtype) if isinstance(v, torch.Tensor) else v for k, v in CALLS["fspad_kv_store_paged_byte"][0].items()}
    with pytest.raises(ValueError, match="k must be a device tensor"):
        fspad.fspad_kv_store_paged_byte(**args, stream=Stream(2))
