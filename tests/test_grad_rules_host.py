"""How the FP8 linear's gradients are cut and dealt (csrc/grad_rules.hpp), compiled for the host: every unit has one block, whole tiles and
parts make up the result, parts fit the workspace and none is without stages.  And the entries' refusals that need no device."""
import ctypes
import random
import subprocess

import pytest

import paper_2512_07710_amd as moe
from paper_2512_07710_amd.build import CSRC, HIPCC, ROOT

PROGRAM = r"""
#include <hip/hip_runtime.h>
#include "grad_rules.hpp"
#include <cstdio>
#include <vector>
using namespace moe355;
int main() {
    int cut, turns, room, tiles, stages;                       // room: units that the launch is made for
    while (scanf("%d %d %d %d %d", &cut, &turns, &room, &tiles, &stages) == 5) {
        const split_plan p = cut ? plan_of(tiles, stages, stages % 2 ? 25 : 10, stages % 3 ? 100 : stages % 7 * 15) : split_plan{tiles, 0, 1};
        const int units = p.whole + p.cut * p.parts;
        std::vector<char> seen(units);
        int bad = p.whole + p.cut != tiles || p.parts < 1, idle = 0;
        for (long b = 0; b < blocks_of(room ? room : units, turns); ++b) {
            const int n = unit_of_block(p, turns, (int)b);
            if (n < 0) ++idle;
            else if (n >= units || seen[n]++) bad |= 2;
        }
        for (char s : seen) if (!s) bad |= 4;
        printf("%d %d %d %d %d\n", p.whole, p.cut, p.parts, bad, idle);
    }
}
"""


@pytest.fixture(scope="module")
def deal(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.hip").write_text(PROGRAM)
    subprocess.run([HIPCC, "--cuda-host-only", "-O2", "-std=c++17", "-I", CSRC, "-I", ROOT + "/include", str(d / "rules.hip"), "-o",
                    str(d / "rules")], check=True, capture_output=True)

    def ask(cases):
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = subprocess.run([str(d / "rules")], input=text, check=True, capture_output=True, text=True).stdout.splitlines()
        return [tuple(map(int, line.split())) for line in out]
    return ask


def test_every_unit_has_one_block(deal):
    rng = random.Random(5)
    cases = []
    for tiles in list(range(0, 20)) + [255, 256, 257, 511, 512, 513, 1023, 1024, 1025] + [int(2 ** rng.uniform(0, 15)) for _ in range(300)]:
        for stages in (1, 2, 7, 8, 16, 40, 64, 500, int(2 ** rng.uniform(0, 13))):
            cases.append((1, 0, 0, tiles, stages))             # one matrix
            cases.append((0, 1, 0, tiles, stages))             # experts' weights' gradient
            cases.append((0, 0, tiles + rng.randint(0, 300), tiles, stages))        # experts' rows: fewer tiles than there could be
            if tiles <= 512:
                cases.append((1, 0, 512, tiles, stages))       # the same in parts
    cut = 0
    for case, (whole, n, parts, bad, _) in zip(cases, deal(cases)):
        assert bad == 0, (case, bad)
        assert n * parts <= 512, case                          # places in the workspace
        assert parts == 1 or parts * 4 <= case[4], case
        cut += n > 0
    assert cut > 500


def test_entries_refuse_without_a_context():
    lib = moe.load_library()
    n = None
    assert lib.moe_reserve_gradients(n) == -1
    assert lib.moe_add_rmsnorm(n, n, n, n, 1, 128, 128, 128, 0, 1e-6, *[n] * 5) == -1
    assert lib.moe_add_rmsnorm_backward(*[n] * 6, 1, 128, 0, n, n) == -1
    assert lib.moe_dispatch(n, n, n, 0, n) == -1
    assert lib.moe_dispatch_backward(n, n, n, n, 0, n) == -1
    assert lib.moe_combine_backward(*[n] * 6, 0, n, n, n) == -1
    assert lib.moe_policy_loss(n, n, 128, 0, 1, 128, *[n] * 6, *[ctypes.c_float(0.1)] * 4, 1.0, *[n] * 5, 128, 0) == -1
    assert lib.moe_linear_fp8_dgrad(n, n, 1, 128, n, n, 128, n, 1, n) == -1
    assert lib.moe_linear_fp8_wgrad(n, n, 1, 128, n, n, 128, n, 1, 0, 0, n) == -1
