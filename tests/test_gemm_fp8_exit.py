"""A block of the 8-bit product ends with no arrival on its way to its barriers: its producer waits for the last hand-over of every stage.
Read from the source, and the stages and parities that it waits for against a model of the barriers."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _source():
    text = open(os.path.join(ROOT, "paper_2512_23087_b200", "csrc", "dvp_gemm_fp8.cu")).read()
    return re.sub(r"/\*.*?\*/|//[^\n]*", "", text, flags=re.S)


def test_every_kernel_with_stages_that_are_handed_back_waits_for_them():
    text = _source()
    kernels = re.split(r"__global__", text)[1:]
    staged = [k for k in kernels if re.search(r"umma_commit(_pair)?\(smem_u32\(&sh->empty", k)]
    assert len(staged) == 2
    for k in staged:
        # behind the loop that fills the stages, in the branch of the thread that does
        loads = max(m.end() for m in re.finditer(r"tma_load_2d(_pair)?\(", k))
        wait = k.find("wait_for_last(sh->empty, it, abort_flag, p.status)")
        assert loads < wait < k.find("warp == 1 && lane == 0" if "warp == 1 && lane == 0" in k else "} else if (warp == 1)")


@pytest.mark.parametrize("stages", [1, 2, 4, 6, 11])
@pytest.mark.parametrize("n", range(0, 30))
def test_the_waits_are_for_the_last_phases(stages, n):
    text = _source()
    assert "for (uint32_t it = n > kStages ? n - kStages : 0; it < n && !*abort_flag; ++it)" in text
    assert "mbar_wait(smem_u32(&empty[it % kStages]), (it / kStages) & 1, abort_flag)" in text
    phases = [0] * stages   # hand-overs that have arrived, one a fill
    for it in range(n):
        phases[it % stages] += 1
    waits = [(it % stages, (it // stages) & 1) for it in range(n - stages if n > stages else 0, n)]
    assert len(waits) == len(set(s for s, _ in waits)) == min(n, stages)
    for s, parity in waits:
        # the last phase of the stage, which no earlier one with the same parity can be taken for: that one was waited for before the last fill
        assert (phases[s] - 1) & 1 == parity
