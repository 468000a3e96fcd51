"""How the norm's rows are dealt to blocks and launches (csrc/grad_rules.hpp), compiled for the host: every row once, whatever their number."""
import random
import subprocess

import pytest

from paper_2512_07710_amd.build import CSRC, HIPCC, ROOT

PROGRAM = r"""
#include <hip/hip_runtime.h>
#include "grad_rules.hpp"
#include <cstdio>
using namespace moe355;
int main() {
    long long rows;
    int cols, threads, codes;
    while (scanf("%lld %d %d %d", &rows, &cols, &threads, &codes) == 4) {
        const int per = norm_rows_per_block(rows, cols, threads, codes);
        long long first = 0, most = 0, launches = 0, blocks;
        for (; first < rows; first += blocks * per, ++launches) {
            blocks = norm_blocks(rows - first, threads, per);
            if (blocks < 1) break;
            if (blocks * threads > most) most = blocks * threads;
        }
        printf("%d %lld %lld %lld\n", per, first, most, launches);
    }
}
"""


@pytest.fixture(scope="module")
def deal(tmp_path_factory):
    d = tmp_path_factory.mktemp("norm")
    (d / "rules.hip").write_text(PROGRAM)
    subprocess.run([HIPCC, "--cuda-host-only", "-O2", "-std=c++17", "-I", CSRC, "-I", ROOT + "/include", str(d / "rules.hip"), "-o", str(d / "rules")],
                   check=True, capture_output=True)

    def ask(cases):
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = subprocess.run([str(d / "rules")], input=text, check=True, capture_output=True, text=True).stdout.splitlines()
        return [tuple(map(int, line.split())) for line in out]
    return ask


def test_every_row_is_in_a_launch(deal):
    rng = random.Random(3)
    cases = [(2 ** 29, 128, 64, 1), (2 ** 30, 128, 64, 1), (2 ** 30, 128, 64, 0), (2 ** 29 + 3, 128, 64, 1), (2 ** 30, 32768, 1024, 1), (1, 128, 64, 1)]
    for _ in range(500):
        cols = 128 * rng.randint(1, 256)
        threads = rng.choice([64, 128, 256, 448, 1024])
        cases.append((int(2 ** rng.uniform(0, 30)), cols, threads, rng.randint(0, 1)))
    for case, (per, reached, grid, launches) in zip(cases, deal(cases)):
        rows, _, _, codes = case
        assert 1 <= per <= (16 if codes else 1), case
        assert rows <= reached < rows + per, case
        assert grid < 2 ** 32, case
        assert launches <= 1 + rows * case[2] // per // 2 ** 30, case
