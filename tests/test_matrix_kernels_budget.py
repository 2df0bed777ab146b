"""The kernels of a training step's matrices keep what they work on in registers: nothing is spilled (the large tiles count
the loads that are under way), and as many waves fit as their layout counts on; loads that go straight to the LDS are
waited for in front of the barriers that other waves read behind.  From the compiler's own reports; no GPU is needed."""
import os
import re
import subprocess

import pytest

from paper_2605_17879_amd import build as hip_build
from test_staged_loads import barriers_with_loads_under_way, kernels

SOURCES = ("pack.hip", "packed_product.hip", "muon.hip")
HEADERS = ("gd_operators.h", "gd_tiles.h")
LDS = 160 * 1024


@pytest.fixture(scope="module")
def report():
    written = max(os.path.getmtime(os.path.join(hip_build.CSRC, s)) for s in SOURCES + HEADERS)
    paths = [hip_build.resource_file(s) for s in SOURCES]
    if not all(os.path.exists(p) and os.path.getmtime(p) >= written for p in paths):
        hip_build.build()                       # (the build writes the reports)
    out = {}
    for p in paths:
        with open(p) as f:
            out.update(hip_build.parse_resources(f.read()))
    return out


def test_nothing_is_spilled(report):
    assert len(report) > 60
    for name, r in report.items():
        assert r["VGPRs Spill"] == 0 and r["ScratchSize [bytes/lane]"] == 0 and not r["Dynamic Stack"], name
        assert r["VGPRs"] + r["AGPRs"] <= 256 and r["LDS Size [bytes/block]"] <= LDS, name


@pytest.mark.parametrize("kind,count,waves,groups", [
    # (waves a SIMD, workgroups that a CU's LDS has to hold)
    ("10large_tile", 17, 2, 1), ("10small_tile", 17, 2, 2), ("13direct_kernel", 80, 2, 1), ("11pack_kernel", 6, 4, 4), ("11tiny_kernel", 1, 2, 1),
])
def test_waves_that_fit(report, kind, count, waves, groups):
    found = {k: r for k, r in report.items() if kind in k}
    assert len(found) == count, sorted(found)
    for name, r in found.items():
        assert r["Occupancy [waves/SIMD]"] >= waves, (name, r)
        assert r["LDS Size [bytes/block]"] * groups <= LDS, (name, r)
        if re.search(r"direct_kernel.*Li4EEE", name):
            assert r["LDS Size [bytes/block]"] * 2 <= LDS, (name, r)


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = {}
    for s in SOURCES[1:]:
        to = tmp_path_factory.mktemp("asm") / (s + ".s")
        flags = [f for f in hip_build.FLAGS if f != "-Rpass-analysis=kernel-resource-usage"]
        subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--cuda-device-only", "-S", os.path.join(hip_build.CSRC, s), "-o", str(to)],
                       check=True, stderr=subprocess.DEVNULL)
        out.update(kernels(to.read_text()))
    return out


def test_no_barrier_is_met_with_loads_to_the_lds_under_way(assembly):
    found = {k: v for k, v in assembly.items() if "small_tile" in k or "direct_kernel" in k}
    assert len(found) == 97
    for name, lines in found.items():
        assert barriers_with_loads_under_way(lines) == [], name


def test_sums_of_the_scaled_instruction_are_not_read_too_early(assembly):
    """In the large tile sixteen of them stand together in a piece of assembly that the compiler does not look into: the
    waits at its end are part of it."""
    found = {k: v for k, v in assembly.items() if "large_tile" in k and "of_codes" in k}
    assert len(found) == 8
    for name, lines in found.items():
        ends = [i for i, l in enumerate(lines) if l.startswith("v_mfma_scale") and not lines[i + 1].startswith("v_mfma_scale")]
        assert ends, name
        for i in ends:
            assert all(l.startswith("v_mfma_scale") for l in lines[i - 15:i + 1]), name
            assert lines[i + 1:i + 3] == ["s_nop 15", "s_nop 3"], name
