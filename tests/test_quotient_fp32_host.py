"""The norm's codes are made from fp32 values over fp32 maxima: the short quotient (csrc/e4m3.hpp) against the division there, on the host.

Where the refined reciprocal is the fp32 number next to 1/s, the corrected quotient is the division's (a remainder of the estimate that is exact, times a
reciprocal that is right to half an ulp).  So: all 2^23 significands of s with estimates up to 2 ulp off; where the reciprocal is another, every
significand of v, at every binade that a code can come from; and random pairs over the whole range of scales."""
import os
import subprocess

from paper_2512_07710_amd.build import HIPCC

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "e4m3.hpp"
#include <cmath>
#include <cstdio>
#include <cstring>
static float from_bits(uint32_t b) { float f; memcpy(&f, &b, 4); return f; }
static uint32_t to_bits(float f) { uint32_t b; memcpy(&b, &f, 4); return b; }
static float coded(float q) {                                  // what the code of q >= 0 stands for
    if (q >= 448.f) return 448.f;
    int e;
    frexpf(q, &e);
    const float ulp = q < 0x1p-6f ? 0x1p-9f : ldexpf(1.f, e - 4);
    return rintf(q / ulp) * ulp;
}
static uint64_t state = 88172645463325252ull;
static uint64_t next() { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return state; }
int main() {
    long others = 0, wrong_codes = 0, left_out = 0;
    for (uint32_t m = 0; m < 1u << 23; ++m) {
        const float s = from_bits(127u << 23 | m), nearest = (float)(1.0 / (double)s);
        for (int off = -2; off <= 2; ++off) {
            const float inv = moe355::refined_reciprocal(s, from_bits(to_bits(1.0f / s) + off));
            if (inv == nearest) continue;
            ++others;
            for (uint32_t v = 0; v < 1u << 24; ++v) {          // two binades: every quotient's significand
                const float x = from_bits((127u << 23) + v), q = moe355::corrected_quotient(x, s, inv), t = x / s;
                if (q == t) continue;
                for (int k = -12; k < 9; ++k)
                    if (coded(ldexpf(q, k)) != coded(ldexpf(t, k))) ++(moe355::significand_all_ones(s) ? left_out : wrong_codes);
            }
        }
    }
    long wrong = 0, cases = 0;
    const float ends[3] = {1.f, moe355::SCALE_MID_MIN * 1.01f, moe355::SCALE_MID_MAX / 2.02f};
    for (int which = 0; which < 3; ++which)
        for (int i = 0; i < 20000000; ++i) {
            const uint64_t r = next();
            const float s = ends[which] * from_bits(127u << 23 | (uint32_t)(r & 0x7FFFFF)) / (which ? 1.f : 448.f);
            if (moe355::significand_all_ones(s)) continue;
            const float inv = moe355::refined_reciprocal(s, from_bits(to_bits(1.0f / s) + (int)((r >> 60) % 5) - 2));
            float v = ldexpf(448.f * s, -(int)((r >> 23) % 20)) * from_bits(126u << 23 | (uint32_t)((r >> 30) & 0x7FFFFF));
            if (r >> 59 & 1) v = -v;
            ++cases;
            wrong += coded(fabsf(moe355::corrected_quotient(v, s, inv))) != coded(fabsf(v / s));
        }
    printf("%ld %ld %ld %ld %ld\n", others, wrong_codes, left_out, cases, wrong);
    return 0;
}
"""


def test_codes_of_fp32_values_are_the_divisions(tmp_path):
    src, exe = tmp_path / "quotient.hip", tmp_path / "quotient"
    src.write_text(PROGRAM)
    subprocess.run([HIPCC, "--cuda-host-only", "-O2", "-mfma", "-std=c++17", "-ffp-contract=off", "-I",
                    os.path.join(ROOT, "paper_2512_07710_amd", "csrc"), str(src), "-o", str(exe)], check=True, capture_output=True)
    others, wrong_codes, left_out, cases, wrong = map(int, subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split())
    assert 0 < others < 200 and cases > 50_000_000
    assert wrong_codes == 0 and wrong == 0
    assert left_out > 0                                        # (the case that the division itself is taken for)
