"""The paged attention under bounds far above its lengths, which stay on the device: the kernels that the bound chooses (wavefronts, whole units
or cut ones, the join) against the oracle, with as long a table as the bound needs and junk in it."""
import numpy as np
import pytest

from test_gpu_attn_paged import Case, _compare
from test_paged_plan import SHAPES, WIDE

pytestmark = pytest.mark.gpu


def _case(shape, seed=21):
    B, N, Hq, Hkv, D, P, lengths = shape
    rng = np.random.default_rng(seed)
    if isinstance(lengths, tuple):
        kv_len, nodes = np.array(lengths), np.full(B, N)
    else:
        kv_len, nodes = rng.integers(0, lengths + 1, B), rng.integers(0, N + 1, B)
        kv_len[0], nodes[0], nodes[1] = lengths, N, 1
    c = Case(seed, B, N, Hq, Hkv, D, P, kv_len, nodes)
    junk = rng.integers(-3, 2 * c.raw.shape[0], (B, WIDE // P - c.table.shape[1])).astype(np.int32)
    c.table = np.concatenate([c.table, junk], axis=1)
    return c


@pytest.mark.parametrize("shape", [s for s, _, _ in SHAPES], ids=lambda s: "-".join(map(str, s[:6])))
def test_a_bound_far_above_the_lengths(shape):
    c = _case(shape)
    want, bound = c.reference()
    for most in (max(1, int(c.kv_len.max())), WIDE):
        got = c.run(max_kv_len=most, guard=1 << 20)
        _compare(got.double().cpu().numpy(), want, bound)
        for b in range(shape[0]):
            assert np.all(got[b, c.n_nodes[b]:].cpu().numpy() == 0)


@pytest.mark.parametrize("shape", [(5, 1, 8, 2, 128, 64), (3, 26, 8, 8, 128, 32), (3, 60, 8, 8, 128, 64), (3, 60, 16, 16, 64, 64)], ids=lambda s: "-".join(map(str, s)))
def test_one_layout_serves_lengths_of_any_size(shape):
    """One bound, then lengths from none to a long one among short ones: what is whole in one call is cut in the next."""
    for seed, top in enumerate((0, 20, 3000)):
        c = _case((*shape, tuple([top] + [7 * i for i in range(1, shape[0])])), seed)
        want, bound = c.reference()
        _compare(c.run(max_kv_len=WIDE, guard=1 << 20).double().cpu().numpy(), want, bound)
