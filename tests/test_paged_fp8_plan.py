"""How calls over the paged 8-bit cache are dealt to kernels (csrc/paged_plan.h), and the attention's many-row reference. CPU; the cases are run in
test_gpu_attn_paged_fp8_cuts.py."""
import os
import re
import subprocess

import numpy as np
import pytest

import _paged_reference
from oracle import paged, paged_fp8
from test_gpu_attn_paged_fp8_cuts import CASES, IDS, Quick, sequences

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2408_15562_amd", "csrc")

DRIVER = r"""
#include <cstdio>
#include "paged_plan.h"
using namespace fspad_detail;
int main() {
  fspad_paged_desc d{};
  d.io_dtype = d.out_dtype = FSPAD_BF16;
  d.n_pages = 1000;
  while (std::scanf("%d %d %d %d %d %d %d", &d.batch, &d.n_nodes_max, &d.n_q_heads, &d.n_kv_heads, &d.head_dim, &d.page_tokens, &d.max_kv_len) == 7) {
    d.page_stride = (int64_t)d.n_kv_heads * page_head_bytes_fp8(d.head_dim, d.page_tokens);
    d.table_stride = d.table_width = d.max_kv_len / d.page_tokens + 1;
    const PagedPlan pl = plan_paged(d, PagedFormat::kFp8);
    std::printf("%d %d %d %d %d %d\n", check_paged_attn(d, PagedFormat::kFp8), pl.rows_per_wave, pl.WS, pl.waves, pl.split, pl.may_cut);
  }
}
"""


def test_cases_reach_the_kernels_that_they_name_and_all_that_there_are(tmp_path):
    (tmp_path / "plan.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", str(tmp_path / "plan"), str(tmp_path / "plan.cpp")], check=True)
    text = "".join(" ".join(map(str, (*shape, bound or lengths[0]))) + "\n" for shape, lengths, bound, _, _ in CASES)
    out = subprocess.run([str(tmp_path / "plan")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    kernels = set()
    for (shape, _, _, dealt, how), line in zip(CASES, out):
        status, *got, may_cut = map(int, line.split())
        assert (status, tuple(got), bool(may_cut)) == (0, dealt, how != "uncut"), (shape, line)
        rows, slabs, waves, split = dealt
        kernels.add((f"Form16Fp8<{shape[4]}>" if rows == 16 else f"Form32Fp8<{shape[4]}, {rows // 32}>", waves, split))
    # the launcher's, from its lines
    with open(os.path.join(CSRC, "fspad_attn_paged_fp8.hip")) as f:
        found = re.findall(r"launch<(Form\d+Fp8<[^>]+>), (\d), true(, false)?>", f.read())
    there = set()
    for form, waves, unsplit in found:
        for D in (64, 128):
            if not ("<64" in form and D == 128):
                there.add((form.replace("<D", f"<{D}"), int(waves), 0 if unsplit else 1))
    assert len(found) == 11 and kernels == there


@pytest.mark.parametrize("shape", [(3, 9, 8, 2, 64, 32), (2, 5, 2, 2, 128, 64)])
def test_many_row_reference_is_the_oracle(shape):
    kv_len, nodes = sequences(shape, (150, 0, 60))
    c = Quick(5, *shape, kv_len, nodes)
    c.table[0, 0] = -1
    c.mask[1, 0] = 0
    out, bound = c.reference("cpu")
    f = lambda t: t.double().numpy()  # noqa: E731
    want, off = paged.tree_attn(f(c.q), f(c.kt), f(c.vt), paged_fp8.Fp8Pages(c.raw, shape[4], shape[5]), c.table, c.kv_len, c.n_nodes, c.mask, 1 << 30)
    assert np.abs(out - want).max() < 1e-12 and np.any(want != 0)
    assert np.abs(bound - off).max() < 1e-12


def test_ids_are_their_own():
    assert len(set(IDS)) == len(CASES)
