"""How the two ends of a policy step deal their work (csrc/step_rules.hpp), compiled for the host: no place outside a row, whatever its length, and blocks for every
row of a table, however many there are."""
import subprocess
import sys

import pytest
import torch

from paper_2512_07710_amd.build import CSRC, HIPCC, ROOT

TICKETS, WORKSPACE = (1 + 64 + 512) * 32, 64 << 20             # of a context
PROGRAM = f"constexpr int TICKETS = {TICKETS};\n" + r"""
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
        } else if (!strcmp(what, "clear")) {                   // V, tokens, bytes of a row: rows to a block, blocks
            int V;
            int64_t T, bytes;
            if (scanf("%d %ld %ld", &V, &T, &bytes) != 3) return 1;
            const clear_plan p = clearing(V, T, bytes);
            printf("%d %d\n", p.rows, p.blocks);
        } else if (!strcmp(what, "runs")) {                    // T, parts and columns of a thread, room: a run, rows of it to a fold, runs of a group
            int parts, columns;
            int64_t T, room;
            if (scanf("%ld %d %d %ld", &T, &parts, &columns, &room) != 4) return 1;
            const int64_t run = run_of_tokens(T, parts, columns, room, TICKETS);
            printf("%ld %d %d\n", run, rows_of_fold(run), runs_of_group((T + run - 1) / run));
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


def test_every_row_of_a_table_is_cleared_by_one_block(ask):
    cases = [(V, T, bytes) for V in LENGTHS + [8191, 8192, 8193, 2 ** 25, 2 ** 25 + 1, 2 ** 31 - 8192, 2 ** 31 - 8191, 2 ** 31 - 8193] for T in (0, 1, 1024, 2 ** 21)
             for bytes in (2, 4, 14336, 262144)]
    for (V, T, bytes), (rows, blocks) in zip(cases, ask("clear", cases)):
        assert 1 <= rows <= 4096 and (blocks - 1) * rows < V <= blocks * rows and blocks <= 2 ** 19, (V, T, bytes, rows, blocks)
        assert rows == min(4096, max(-(-V // 8192), -(-8 * T // bytes))), (V, T, bytes, rows)


@pytest.mark.skipif(torch.cuda.is_available(), reason="for machines without a GPU: the call would run on made-up pointers")
@pytest.mark.parametrize("V", [2 ** 31 - 8192, 2 ** 31 - 8191, 2 ** 31 - 1])
@pytest.mark.parametrize("T", [0, 1])
def test_the_gradient_of_the_largest_tables_comes_back(V, T):
    """With a status: the plan of its launches is the host's own arithmetic, and no launch succeeds here."""
    code = f"""
import ctypes
import paper_2512_07710_amd as moe
ctx = ctypes.create_string_buffer(b"\x40" * 4096, 4096)
P = 1 << 20
print("status", moe.load_library().moe_embed_backward(ctypes.addressof(ctx), P, P, {T}, {V}, 1, 1, 0, 1.0, 0, P, 1, 0))
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT)
    assert r.returncode == 0 and "status -2" in r.stdout, (r.returncode, r.stdout, r.stderr[-300:])


def _additions(ask, cases):
    """For (T, d, both arrays bf16): additions one after another that a row's share of its token's sum goes through at most."""
    asked = []
    for T, d, narrow in cases:
        columns = 8 if narrow else 4
        room = (WORKSPACE - 16 * (T + 1)) // (8 * -(-d // 8) * 8)
        asked.append((T, -(-d // (columns * 256)), columns, room))
    for (T, d, _), (_, parts, _, room), (run, fold, group) in zip(cases, asked, ask("runs", asked)):
        runs = -(-T // run)
        assert runs <= room and runs * parts <= TICKETS and run & (run - 1) == 0 and fold & (fold - 1) == 0 and fold % 64 == 0
        groups = max(1, runs // group)
        yield min(run, fold) + (run // fold if run > fold else 0) + (runs if runs < 32 else runs - (groups - 1) * group + groups)


def test_sums_of_a_frequent_token_are_short_chains(ask):
    small = [(2 ** 21, 64, False), (2 ** 21, 64, True), (2 ** 20, 512, False), (2 ** 20 + 77, 131, False), (2 ** 20 + 77, 131, True), (32768, 7168, True), (4096, 5120, False)]
    assert max(_additions(ask, small)) <= 200
    every = [(T, d, narrow) for T in (1025, 2049, 4096, 30000, 131072, 10 ** 6, 2 ** 20 + 1, 2 ** 21) for d in (1, 8, 100, 1000, 5120, 7168, 20000, 65536) for narrow in (True, False)]
    chains = dict(zip(every, _additions(ask, every)))
    assert max(n for (T, d, _), n in chains.items() if d <= 7168) <= 320 and max(chains.values()) <= 900, sorted(chains.items(), key=lambda c: -c[1])[:5]
