"""How a call of the paged attention is laid out (csrc/paged_plan.h) under a bound on its lengths: exact, and that of a wide table. CPU;
the shapes are run with both bounds in test_gpu_paged_bound.py."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# batch, nodes, query heads, kv heads, head dim, page tokens, prefix lengths (a tuple: those; else up to so many), and of the exact and the wide
# bound: rows of a wavefront, slabs, wavefronts, whether units may be cut
WIDE = 16384
SHAPES = [
    ((1, 1, 8, 2, 128, 16, (301,)), (16, 1, 4, 0), (16, 1, 8, 1)),
    ((3, 3, 4, 1, 64, 64, (700, 0, 33)), (16, 1, 4, 0), (16, 1, 8, 1)),
    ((70, 1, 8, 8, 64, 32, 200), (16, 1, 4, 0), (16, 1, 4, 1)),
    ((2, 26, 2, 2, 128, 32, (500, 96)), (32, 1, 4, 0), (32, 1, 4, 1)),
    ((2, 26, 16, 16, 128, 16, (500, 96)), (32, 1, 4, 0), (32, 1, 8, 1)),
    ((20, 26, 16, 16, 128, 64, 250), (32, 1, 4, 0), (32, 1, 4, 1)),
    ((2, 20, 12, 12, 64, 64, (400, 31)), (32, 1, 4, 0), (32, 1, 8, 1)),
    ((2, 60, 8, 8, 128, 64, (450, 100)), (32, 2, 4, 0), (32, 2, 8, 1)),
    ((20, 40, 16, 8, 128, 128, 400), (32, 2, 4, 0), (32, 2, 8, 1)),
    ((2, 60, 16, 16, 64, 32, (450, 100)), (64, 1, 4, 0), (64, 1, 8, 1)),
    ((20, 40, 16, 8, 64, 16, 400), (64, 1, 4, 0), (64, 1, 4, 1)),
    ((2, 60, 4, 4, 128, 32, (0, 0)), (32, 2, 4, 0), (32, 2, 8, 1)),
]

DRIVER = r"""
#include <cstdio>
#include "paged_plan.h"
using namespace fspad_detail;
int main() {
  fspad_paged_desc d{};
  d.io_dtype = d.out_dtype = FSPAD_BF16;
  d.n_pages = 1000;
  while (std::scanf("%d %d %d %d %d %d %d", &d.batch, &d.n_nodes_max, &d.n_q_heads, &d.n_kv_heads, &d.head_dim, &d.page_tokens, &d.max_kv_len) == 7) {
    d.page_stride = (int64_t)d.n_kv_heads * page_head_bytes(d.head_dim, d.page_tokens);
    d.table_stride = d.table_width = d.max_kv_len / d.page_tokens + 1;
    const PagedPlan pl = plan_paged(d);
    const int64_t units = (int64_t)d.batch * d.n_kv_heads * pl.groups;
    std::printf("%d %d %d %d %d %d %d %lld %d\n", check_paged_attn(d), pl.rows_per_wave, pl.WS, pl.waves, pl.may_cut, pl.lines, pl.max_pieces, (long long)units, pl.resident);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    at = tmp_path_factory.mktemp("paged_plan")
    (at / "plan.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2408_15562_amd", "csrc"), "-o", str(at / "plan"), str(at / "plan.cpp")], check=True)

    def run(shapes):
        text = "".join(" ".join(map(str, s)) + "\n" for s in shapes)
        out = subprocess.run([str(at / "plan")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def _longest(lengths):
    return max(lengths) if isinstance(lengths, tuple) else lengths


def test_the_shapes_reach_every_layout_with_a_bound_of_either_kind(plan):
    exact = plan([(*s[:6], _longest(s[6])) for s, _, _ in SHAPES])
    wide = plan([(*s[:6], WIDE) for s, _, _ in SHAPES])
    for (shape, e, w), pe, pw in zip(SHAPES, exact, wide):
        assert pe[0] == pw[0] == 0 and pe[1:5] == e and pw[1:5] == w, shape
    # windows of a line: of more units than workgroups, and where all go in one round
    assert any(p[5] and p[7] > p[8] for p in wide) and any(p[5] and p[7] <= p[8] for p in wide)


def test_a_window_has_two_slots(plan):
    """Where workgroups may take windows of the line of units, the workspace has two slots for each; else one for every piece of equal length."""
    shapes = [(B, N, q, kv, D, 32, L) for B in (1, 3, 16, 64, 300) for N in (1, 17, 33, 64) for q, kv in ((8, 8), (16, 2), (52, 52), (64, 8)) for D in (64, 128)
              for L in (0, 31, 500, 4000, 60000)]
    for shape, (status, rows, WS, waves, may_cut, lines, pieces, units, resident) in zip(shapes, plan(shapes)):
        assert status == 0 and rows in (16, 32, 64) and waves in (4, 8) and units <= pieces <= units + 2 * resident, shape
        assert not lines or (rows > 16 and pieces >= 2 * resident), shape
        assert may_cut or pieces == units, shape
