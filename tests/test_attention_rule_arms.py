"""Where the prompt attention's waves share queries in halves: both sides of every border of the rule, compiled for the host.

Blocks of 128 queries up to which they do: 256 with heads up to 64 x 96 and 128 with wider ones, twice as many where 1,024
tokens are seen, and in a ragged batch twice as many once more where 512 are."""
import os
import subprocess

import pytest

from test_gpu_window import run

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROBE = r"""
#include "token_rules.hpp"
#include <cstdio>
int main() {
  long long a, b, c, d, w, s, r;
  while (scanf("%lld %lld %lld %lld %lld %lld %lld", &a, &b, &c, &d, &w, &s, &r) == 7)
    printf("%d\n", (int)nc::window_halves(a, b, c, d, w, s, r != 0));
}
"""

# tokens, window, sinks, ragged, and the factor of the blocks
ARMS = [(128, 0, 0, 0, 1), (511, 0, 0, 0, 1), (511, 0, 0, 1, 1), (512, 0, 0, 0, 1), (512, 0, 0, 1, 2), (1023, 0, 0, 0, 1),
        (1023, 0, 0, 1, 2), (1024, 0, 0, 0, 2), (1024, 0, 0, 1, 4), (5000, 0, 0, 1, 4), (5000, 0, 700, 0, 2),
        (5000, 500, 11, 0, 1), (5000, 500, 11, 1, 1), (5000, 500, 12, 1, 2), (5000, 1000, 23, 0, 1), (5000, 1000, 23, 1, 2),
        (5000, 1000, 24, 0, 2), (5000, 1000, 24, 1, 4), (5000, 6000, 0, 1, 4), (600, 1000, 24, 0, 1), (600, 1000, 24, 1, 2),
        (1024, 512, 0, 0, 1), (1024, 512, 0, 1, 2)]
HEADS = [(64, 64, 256), (64, 96, 256), (1, 1, 256), (64, 97, 128), (65, 64, 128), (128, 128, 128)]


def test_the_rule(tmp_path):
    (tmp_path / "p.cpp").write_text(PROBE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2502_20762_amd", "csrc"), str(tmp_path / "p.cpp"),
                    "-o", str(tmp_path / "p")], check=True)
    lines, want = [], []
    for D, V, fit in HEADS:
        for T, window, sinks, ragged, factor in ARMS:
            most = fit * factor // -(-T // 128)  # sequences and heads whose blocks are no more than that
            for bh in (1, most, most + 1, 4 * most):
                lines.append(f"{bh} {T} {D} {V} {window} {sinks} {ragged}")
                want.append(bh <= most)
        lines += [f"1 {T} {D} {V} 0 0 0" for T in (1, 64, 65)]
        want += [False, False, True]
    out = subprocess.run([str(tmp_path / "p")], input="\n".join(lines), check=True, capture_output=True, text=True).stdout
    got = [x == "1" for x in out.split()]
    assert len(got) == len(want) and all(a == b for a, b in zip(got, want)), [x for x, a, b in zip(lines, got, want) if a != b]


@pytest.mark.gpu
@pytest.mark.parametrize("H,K", [(32, 8), (64, 16)])
def test_ragged_batches_on_both_sides_of_a_border(H, K):
    # two sequences of 520 tokens are 5 blocks a head: 320 blocks share queries in halves as a ragged batch only, 640 do not
    run(2, 520, H, K, 32, 32, "bf16", None, 0, lengths=[520, 3])
    run(2, 520, H, K, 64, 96, "fp16", 600, 5, lengths=[1, 519])
    run(2, 520, H, K, 64, 64, "bf16", 200, 70, lengths=[517, 520])  # 270 tokens seen: neither does
