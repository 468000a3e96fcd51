"""The plan by which the FP8 linear's gradients are cut (csrc/grad_rules.hpp) is worked out on the host, for the launches, and in each block again: it has
to be made of whole numbers, which are the same on both."""
import os
import re
import subprocess

from paper_2512_07710_amd.build import CSRC, HIPCC, ROOT

# the rule for the rest of many tiles, as a fraction: cut into `most` parts if stages (0.55 - 1 / most) >= 24
PROGRAM = r"""
#include <hip/hip_runtime.h>
#include "grad_rules.hpp"
#include <cstdio>
using namespace moe355;
int main() {
    int tiles, stages;
    while (scanf("%d %d", &tiles, &stages) == 2) {
        const split_plan p = plan_of(tiles, stages, 10, 100);
        printf("%d %d %d\n", p.whole, p.cut, p.parts);
    }
}
"""


def test_no_floating_point():
    text = open(os.path.join(CSRC, "grad_rules.hpp")).read()
    code = re.sub(r"//[^\n]*", "", text)
    assert not re.findall(r"\b(?:float|double)\b|\d\.\d|\d\.?f\b", code)


def test_rest_of_many_tiles(tmp_path):
    (tmp_path / "rules.hip").write_text(PROGRAM)
    exe = tmp_path / "rules"
    subprocess.run([HIPCC, "--cuda-host-only", "-O2", "-std=c++17", "-I", CSRC, "-I", ROOT + "/include", str(tmp_path / "rules.hip"), "-o", str(exe)],
                   check=True, capture_output=True)
    cases = [(512 + rest, stages) for rest in list(range(1, 40)) + [64, 100, 127, 128, 170, 171, 200, 256, 400, 511] for stages in range(4, 140)]
    out = subprocess.run([str(exe)], input="\n".join(f"{t} {s}" for t, s in cases), check=True, capture_output=True, text=True).stdout.splitlines()
    for (tiles, stages), line in zip(cases, out):
        rest = tiles - 512
        most = min(512 // rest, stages // 4)
        cut = most >= 3 and stages * (11 * most - 20) >= 24 * 20 * most
        assert tuple(map(int, line.split())) == ((512, rest, most) if cut else (tiles, 0, 1)), (tiles, stages)
