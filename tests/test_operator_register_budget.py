"""The kernels of a sweep's own training step keep what they work on in registers: nothing is spilled, and as many waves fit as
their layout counts on.  A spill in a product's loop would be slow, and wrong too: the large tiles count the loads
that are under way, and one to scratch memory would be counted with them.  The compiler's resource report (written
beside the objects by the build) is parsed here; no GPU is needed."""
import os

import pytest

from paper_2605_17879_amd import build as hip_build

SOURCES = ("embed.hip", "vocab_loss.hip", "adamw.hip")
HEADERS = ("gd_operators.h", "gd_vocab_plan.h", "gd_lanes.h")
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
    assert len(report) > 80
    for name, r in report.items():
        assert r["VGPRs Spill"] == 0 and r["ScratchSize [bytes/lane]"] == 0 and not r["Dynamic Stack"], name
        assert r["VGPRs"] + r["AGPRs"] <= 512 and r["LDS Size [bytes/block]"] <= LDS, name


@pytest.mark.parametrize("kind,count,waves,groups", [
    # (waves a SIMD, workgroups that a CU's LDS has to hold)
    ("10large_tile", 8, 2, 1), ("10small_tile", 8, 2, 2), ("15few_rows_kernel", 12, 2, 4), ("12adamw_kernel", 1, 4, 1), ("8grad_sum", 12, 4, 1),
    ("8grad_few", 24, 5, 1), ("12embed_kernel", 6, 8, 1), ("10sort_alone", 6, 4, 1), ("9sort_pass", 6, 4, 1),
])
def test_waves_that_fit(report, kind, count, waves, groups):
    found = {k: r for k, r in report.items() if kind in k}
    assert len(found) == count, sorted(found)
    for name, r in found.items():
        assert r["Occupancy [waves/SIMD]"] >= waves, (name, r)
        assert r["LDS Size [bytes/block]"] * groups <= LDS, (name, r)
