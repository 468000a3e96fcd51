"""How the two ends of a policy step deal their work (csrc/step_rules.hpp), compiled for the host: no place outside a row, whatever its length."""
import subprocess

import pytest

from paper_2512_07710_amd.build import CSRC, HIPCC, ROOT

PROGRAM = r"""
#include <hip/hip_runtime.h>
#include "step_rules.hpp"
#include <cstdio>
#include <cstring>
using namespace moe355;
int main() {
    char what[16];
    while (scanf("%15s", what) == 1) {
        if (!strcmp(what, "row")) {                            // V, N, parts, threads: what the parts and their threads have of a row
            int V, N, parts, threads, bad = 0;
            if (scanf("%d %d %d %d", &V, &N, &parts, &threads) != 4) return 1;
            const int part_vecs = parts == 1 ? V : (V / N + parts - 1) / parts;
            int64_t covered = 0, next = 0;
            for (int q = 0; q < parts; ++q) {
                const row_part p = part_of_row(V, N, q, parts, part_vecs);
                bad |= p.begin != next || p.end < p.begin || (int64_t)p.end * N > V || p.place != (int64_t)p.end * N;
                covered += (int64_t)(p.end - p.begin) * N;
                next = p.end;
                int64_t expect = p.place;
                for (int t = 0; t < threads; ++t) {
                    const int at = p.behind(t);
                    if (q < parts - 1 || expect >= V) bad |= 2 * (at != -1);
                    else bad |= 4 * (at != expect++);
                }
                covered += expect - p.place;
            }
            printf("%d\n", bad | 8 * (covered != V));
        }
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.hip").write_text(PROGRAM)
    subprocess.run([HIPCC, "--cuda-host-only", "-O2", "-std=c++17", "-I", CSRC, "-I", ROOT + "/include", str(d / "rules.hip"), "-o",
                    str(d / "rules")], check=True, capture_output=True)

    def answers(what, cases):
        text = "\n".join(" ".join(map(str, (what, *c))) for c in cases)
        out = subprocess.run([str(d / "rules")], input=text, check=True, capture_output=True, text=True).stdout.splitlines()
        return [int(line) if " " not in line else tuple(map(int, line.split())) for line in out]
    return answers


LENGTHS = [1, 2, 3, 4, 5, 7, 8, 9, 63, 64, 65, 1000, 50001, 131072, 262143, 10 ** 9 + 7, *(2 ** 31 - n for n in (1, 2, 3, 4, 5, 8, 9, 64, 255, 256, 257, 1023, 1024, 1025, 4097))]


@pytest.mark.parametrize("N", [4, 8])
@pytest.mark.parametrize("threads", [64, 256, 512, 1024])
def test_every_logit_of_a_row_has_one_place(ask, N, threads):
    cases = [(V, N, parts, threads) for V in LENGTHS for parts in (1, 2, 3, 16, 64, 2048)]
    for case, bad in zip(cases, ask("row", cases)):
        assert bad == 0, (case, bad)
