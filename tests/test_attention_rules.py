"""The sizes of ``test_gpu_window.py`` and ``test_gpu_paged.py`` reach the forms that they are meant for: the rules
themselves, compiled for the host, say which."""
import os
import subprocess

from test_gpu_window import FORMS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROBE = r"""
#include "token_rules.hpp"
#include <cstdio>
int main() {
  long long a, b, c, d;
  while (scanf("%lld %lld %lld %lld", &a, &b, &c, &d) == 4) printf("%d\n", (int)nc::window_halves(a, b, c, d));
}
"""


def test_every_form_of_the_window_has_its_sizes(tmp_path):
    (tmp_path / "p.cpp").write_text(PROBE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2502_20762_amd", "csrc"), str(tmp_path / "p.cpp"),
                    "-o", str(tmp_path / "p")], check=True)
    lines = [f"{B * H} {130 if halves else 129} {D} {V}" for (_, _, halves), (B, H, K, D, V) in FORMS.items()]
    out = subprocess.run([str(tmp_path / "p")], input="\n".join(lines), check=True, capture_output=True, text=True).stdout
    assert [x == "1" for x in out.split()] == [halves for _, _, halves in FORMS]
    # padded head width, tiles of values, direct loads, halves: all of them
    have = {(64 if D <= 64 else 128, (V + 31) // 32, D % 8 == 0 and V % 8 == 0, halves) for D, V, halves in FORMS}
    assert len(have) == 2 * 4 * 2 * 2
