"""Registers, spills, LDS and occupancy of the gfx950 kernels on rows of logits (CPU only): what their launch rules count
on."""
import re

import pytest

from test_operators_build_resources import OCCUPANCY, SCRATCH, _remarks

LDS = "LDS Size [bytes/block]"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    outdir = str(tmp_path_factory.mktemp("ru"))
    return {k: v for u in ("logit_logprobs", "logit_distill", "logit_distill_step") for k, v in _remarks(u, outdir).items()}


def test_nothing_spills(kernels):
    assert len(kernels) >= 24 + 3 + 1 + 12 + 3 + 6 + 1 + 18
    for name, r in kernels.items():
        assert r[SCRATCH] == 0, (name, r)


def test_streaming_kernels_fill_the_chip(kernels):
    """Eight waves per SIMD, but for the second gradient pass that mostly ends at once, and for alternatives, where the LDS
    of 512 threads leaves room for four workgroups a CU (2-byte logits) or three."""
    seen = 0
    for name, r in kernels.items():
        if re.search(r"logprob_kernelI\w+Li512ELb[01]ELb1E", name):
            seen += 1
            assert r[LDS] <= 160 * 1024 // (3 if "IfL" in name else 4), (name, r)
            assert r[OCCUPANCY] >= (6 if "IfL" in name else 8), (name, r)
        elif re.search(r"logprob_kernelI\w+ELb0EEE|logprob_grad|distill_kernel|distill_grad_kernelI\w+Lb0E|join", name):
            seen += 1
            assert r[OCCUPANCY] == 8, (name, r)
    assert seen >= 6 + 12 + 3 + 12 + 3 + 1


def test_the_fused_step_keeps_two_workgroups_a_cu(kernels):
    seen = 0
    for name, r in kernels.items():
        m = re.search(r"distill_step_kernelI\w+?Li(\d+)ELi(\d+)E", name)
        if m:
            seen += 1
            assert r[OCCUPANCY] >= (6 if m.group(2) == "4" else 4), (name, r)
            assert r[LDS] <= 160 * 1024 // 2 - 33792, (name, r)   # besides the marks
    assert seen == 18
