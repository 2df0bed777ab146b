"""The tiled products' loads that go from memory straight to the LDS, in the compiler's own output: no wave of a tile of
128 x 128 meets a barrier with such loads still under way, since behind it the other waves read what they bring.
(A barrier does not wait for them by itself.)  No GPU is needed."""
import os
import re
import subprocess

import pytest

from paper_2605_17879_amd import build as hip_build


def kernels(assembly):
    """{symbol: instruction lines with labels} of the kernels that load to the LDS."""
    out = {}
    for m in re.finditer(r"^(_Z\w+):\s*; @", assembly, re.M):
        body = assembly[m.end():assembly.index(".Lfunc_end", m.end())]
        lines = [l.split(";")[0].strip() for l in body.splitlines()]
        lines = [l for l in lines if l and (not l.startswith(".") or l.startswith(".LBB"))]
        if any(re.match(r"buffer_load\S* .*\blds$", l) for l in lines):
            out[m.group(1)] = lines
    return out


def barriers_with_loads_under_way(lines):
    """Lines of the barriers that some path reaches with loads to the LDS that were not waited for."""
    at = {l[:-1]: i for i, l in enumerate(lines) if l.startswith(".LBB") and l.endswith(":")}
    seen, todo, bad = set(), [(0, False)], set()
    while todo:
        i, under_way = todo.pop()
        while i < len(lines) and (i, under_way) not in seen:
            seen.add((i, under_way))
            l = lines[i]
            wait = re.match(r"s_waitcnt .*vmcnt\((\d+)\)", l)
            if re.match(r"buffer_load\S* .*\blds$", l):
                under_way = True
            elif wait and int(wait.group(1)) == 0:
                under_way = False
            elif l.startswith("s_barrier") and under_way:
                bad.add(i)
            elif l.startswith("s_endpgm"):
                break
            branch = re.match(r"s_(c?branch)\S* (\.LBB\w+)", l)
            if branch:
                todo.append((at[branch.group(2)], under_way))
                if branch.group(1) == "branch":
                    break
            i += 1
    return sorted(bad)


PLAIN = ["s_mov_b32 s0, 0", ".LBB0_1:", "buffer_load_dwordx4 v1, s[8:11], 0 offen lds", "ds_read_b64 v[2:3], v4", "WAIT", "s_barrier",
         "s_cbranch_scc1 .LBB0_1", "s_endpgm"]


@pytest.mark.parametrize("wait,bad", [("s_waitcnt vmcnt(0) lgkmcnt(0)", []), ("s_waitcnt lgkmcnt(0)", [5]), ("s_waitcnt vmcnt(8)", [5])])
def test_the_check_itself(wait, bad):
    assert barriers_with_loads_under_way([wait if l == "WAIT" else l for l in PLAIN]) == bad


def test_a_wait_in_front_of_a_loop_is_not_one_inside():
    lines = ["buffer_load_dwordx4 v1, s[8:11], 0 offen lds", "s_waitcnt vmcnt(0)", ".LBB0_1:", "s_barrier",
             "buffer_load_dwordx4 v1, s[8:11], 0 offen lds", "s_cbranch_vccnz .LBB0_1", "s_endpgm"]
    assert barriers_with_loads_under_way(lines) == [3]


def test_no_barrier_is_met_with_loads_to_the_lds_under_way(tmp_path):
    out = tmp_path / "vocab_loss.s"
    flags = [f for f in hip_build.FLAGS if f != "-Rpass-analysis=kernel-resource-usage"]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--cuda-device-only", "-S",
                    os.path.join(hip_build.CSRC, "vocab_loss.hip"), "-o", str(out)], check=True, stderr=subprocess.DEVNULL)
    found = kernels(out.read_text())
    small = {k: v for k, v in found.items() if "small_tile" in k}
    # two types: logits twice (sums, G), both gradients
    assert len(small) == 8 and len(found) == 16
    for name, lines in small.items():
        assert sum(l.startswith("s_barrier") for l in lines) >= 5, name
        assert barriers_with_loads_under_way(lines) == [], name
