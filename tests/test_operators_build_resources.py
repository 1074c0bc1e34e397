"""Registers, spills and occupancy of the operators' gfx950 kernels (CPU only), from the compiler's resource remarks:
what the rules that pick a kernel count on."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from paper_2606_20005_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KEY_DIMS, VALUE_DIMS = range(32, 129, 32), range(32, 257, 32)
UNITS = ("norm_rope", "diff_fwd_merge", "diff_bwd_prep",
         *(f"diff_{k}_d{d}" for k in ("fwd", "bwd_dq", "bwd_dkv") for d in KEY_DIMS), "diff_bwd_wide_d96", "diff_bwd_wide_d128")
SCRATCH, OCCUPANCY = "ScratchSize [bytes/lane]", "Occupancy [waves/SIMD]"


def _remarks(unit, outdir):
    try:
        cc = build.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    src = os.path.join(build.CSRC, unit + ".hip")
    cmd = [cc, *build.CFLAGS, *build.unit_flags(src), "--offload-device-only", "-c", src, "-o",
           os.path.join(outdir, unit + ".o"), "-Rpass-analysis=kernel-resource-usage"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    out, cur = {}, None
    for line in r.stderr.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            cur = out.setdefault(m.group(1), {})
            continue
        m = re.search(r"remark:\s+([A-Za-z /\[\]]+?):\s+(\d+)", line)
        if m and cur is not None:
            cur[m.group(1).strip()] = int(m.group(2))
    return out


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    outdir = str(tmp_path_factory.mktemp("ru"))
    with cf.ThreadPoolExecutor(max_workers=8) as ex:
        parts = list(ex.map(lambda u: _remarks(u, outdir), UNITS))
    return {k: v for p in parts for k, v in p.items()}


def test_small_kernels_never_spill_and_keep_the_chip_full(kernels):
    seen = 0
    for name, r in kernels.items():
        if re.search(r"norm_rope|merge|prep|dlam|join", name):
            seen += 1
            assert r[SCRATCH] == 0, (name, r)
            assert r[OCCUPANCY] >= 4, (name, r)
    assert seen >= 36 + 72 + 7   # norm and rotation: types x lanes a row x rotations, with the gradients' two types


def test_diff_forward(kernels):
    """No spills; two waves per SIMD in the workgroups of four waves. Those of two waves, for few rows, stream a cache
    and may be held to one by their LDS stages."""
    seen = set()
    for name, r in kernels.items():
        m = re.search(r"diff_fwd_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E", name)
        if m:
            d, dv, rb, nw = map(int, m.groups())
            seen.add((d, dv, rb, nw))
            assert r[SCRATCH] == 0, (name, r)
            assert r[OCCUPANCY] >= (2 if nw == 4 else 1), (name, r)
    assert {s[:2] for s in seen} == {(d, dv) for d in KEY_DIMS for dv in VALUE_DIMS}


def test_diff_backward(kernels):
    """Two waves per SIMD where the split rule counts on them; spills only where they are known and measured: d 64/64
    (two waves with a small spill beat one without)."""
    seen = set()
    for name, r in kernels.items():
        m = re.search(r"diff_bwd_(dq|dq16|dkv|dkv16)_kernelILi(\d+)ELi(\d+)E", name)
        if not m:
            continue
        kind, d, dv = m.group(1), int(m.group(2)), int(m.group(3))
        seen.add((kind.replace("16", ""), d, dv))
        if kind.startswith("dq"):   # 16 rows a wave where 32 leave room for one wave per SIMD
            assert (kind == "dq16") == (d > 64 or (d == 64 and dv > 160)), name
        else:
            small = (d, dv) in ((32, 32), (32, 64), (32, 96), (64, 32), (64, 64))   # 32 keys a wave, two per SIMD
            assert (kind == "dkv16") == (2 * d + dv <= 384 and not small), name
        assert r[OCCUPANCY] >= (1 if kind == "dkv" and 2 * d + dv > 384 else 2), (name, r)
        assert r[SCRATCH] <= (96 if (kind, d, dv) == ("dkv", 64, 64) else 0), (name, r)
    assert len(seen) == 2 * len(KEY_DIMS) * len(VALUE_DIMS)
