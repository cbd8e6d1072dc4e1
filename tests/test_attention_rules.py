"""The sizes of ``test_gpu_window.py`` and ``test_gpu_paged.py`` reach the forms that they are meant for: the rules
themselves, compiled for the host, say which."""
import os
import random
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


TILES = r"""
#include "token_rules.hpp"
#include <cstdio>
int main() {
  long long i0, queries, len, window, sinks;
  while (scanf("%lld %lld %lld %lld %lld", &i0, &queries, &len, &window, &sinks) == 5) {
    const nc::WindowTiles w = nc::window_tiles((int)i0, (int)queries, len, (int)window, (int)sinks);
    printf("%d", w.whole);
    for (int t = 0; t < w.count; ++t) printf(" %d", w.key0(t));
    printf("\n");
  }
}
"""


def test_the_tiles_of_a_window_hold_every_token_seen_once_and_whole_ones_no_other(tmp_path):
    (tmp_path / "p.cpp").write_text(TILES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2502_20762_amd", "csrc"), str(tmp_path / "p.cpp"),
                    "-o", str(tmp_path / "p")], check=True)
    r = random.Random(1)
    cases = []
    while len(cases) < 20000:
        q = r.choice([32, 64, 128])
        i0, n = q * r.randrange(12), r.randrange(1, 1400)
        if i0 < n:
            cases.append((i0, q, n, r.choice([0, r.randrange(1, 40), r.randrange(1, 400), r.randrange(1, 2000), 2 ** 31 - 1]),
                          r.choice([0, 1, r.randrange(70), r.randrange(600), 5000, 2 ** 31 - 1])))
    text = "\n".join(" ".join(map(str, c)) for c in cases)
    out = subprocess.run([str(tmp_path / "p")], input=text, check=True, capture_output=True, text=True).stdout.strip().split("\n")
    assert len(out) == len(cases)
    for (i0, q, n, window, sinks), line in zip(cases, out):
        whole, *tiles = map(int, line.split())
        what = (i0, q, n, window, sinks, whole, tiles)
        assert len(set(tiles)) == len(tiles) and all(0 <= x < n for x in tiles) and whole <= len(tiles), what
        need = set()
        for i in range(i0, min(i0 + q, n)):
            need.update(range((max(0, i + 1 - window) if window else 0) // 64, i // 64 + 1))
            need.update(range(0, min(sinks - 1, i) // 64 + 1 if sinks else 0))
        assert {64 * x for x in need} <= set(tiles), what
        for j in (x + y for x in tiles[:whole] for y in (0, 31, 63)):
            for i in (i0, i0 + q - 1):
                assert j <= i and (window == 0 or i - j < window or j < sinks), what
