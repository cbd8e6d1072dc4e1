"""The sizes of ``test_gpu_tokens_tiles.py`` reach the kernels that they are meant for: the rules themselves, compiled for
the host, say which."""
import os
import subprocess

import pytest

from test_gpu_tokens_tiles import DECAY, FORMS, LINEAR

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNELS = ["rows16", "rows32", "rows64", "reg128x64", "reg128x128", "reg256x256", "dma128x64", "dma128x128", "dma256x128k32",
           "dma256x128k64", "dma256x256"]
PROBE = r"""
#include "token_rules.hpp"
#include <cstdio>
#include <cstring>
int main() {
  using nc::LinearKernel;
  char what[16];
  long long a, b, c, d;
  printf("%d\n", (int)LinearKernel::dma256x256 + 1);
  while (scanf("%15s", what) == 1) {
    if (!strcmp(what, "linear") && scanf("%lld %lld %lld %lld", &a, &b, &c, &d) == 4) {
      const char* names[] = {NAMES};
      const LinearKernel kinds[] = {KINDS};
      for (int i = 0; i < (int)(sizeof(kinds) / sizeof(kinds[0])); ++i)
        if (kinds[i] == nc::linear_rule(a, b, c, d)) printf("%s\n", names[i]);
    } else if (scanf("%lld %lld %lld", &a, &b, &c) == 3) {
      const nc::DecayPlan p = nc::decay_rule(a, b, c);
      printf("%d %d %d\n", p.chunked, p.seg_chunks, p.nseg);
    }
  }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    text = PROBE.replace("NAMES", ", ".join(f'"{k}"' for k in KERNELS)).replace(
        "KINDS", ", ".join(f"LinearKernel::{k}" for k in KERNELS))
    (d / "p.cpp").write_text(text)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2502_20762_amd", "csrc"), str(d / "p.cpp"),
                    "-o", str(d / "p")], check=True)

    def run(lines):
        out = subprocess.run([str(d / "p")], input="\n".join(lines), check=True, capture_output=True, text=True).stdout
        out = out.strip().split("\n")
        assert int(out[0]) == len(KERNELS)  # no kernel that the names leave out
        assert len(out) == len(lines) + 1
        return out[1:]

    return run


def test_every_kernel_of_the_product_has_its_sizes(rules):
    assert list(LINEAR) == KERNELS
    asked = [(kernel, *size) for kernel, sizes in LINEAR.items() for size in sizes]
    got = rules([f"linear {m} {rows} {k} {int(k % 8 == 0 and pad % 8 == 0)}" for _, m, k, rows, pad in asked])
    assert [a[0] for a in asked] == got
    assert all(rows % 2 == 0 for _, _, _, rows, _ in asked)  # so that each can be gated
    for kernel, sizes in LINEAR.items():
        if "x" in kernel:  # remainders of tokens and weight rows, and along K
            tokens, stage = int(kernel.split("x")[1].split("k")[0]), 64 if kernel in ("dma128x64", "dma256x128k64", "dma256x256") else 32
            assert all(m % tokens for m, _, _, _ in sizes)
            assert any(rows % 64 for _, _, rows, _ in sizes) and any(k % stage for _, k, _, _ in sizes)


def plans(rules):
    got = rules([f"decay {B * H} {T} {V}" for B, T, H, K, D, V, _ in DECAY.values()])
    return {case: tuple(map(int, p.split())) for case, p in zip(DECAY, got)}


def test_long_sequences_have_the_chunks_and_segments_that_they_name(rules):
    p = plans(rules)
    assert all(x[0] == 1 for x in p.values())
    assert {case: x[1:] for case, x in p.items() if "one segment" in case} == {
        "one segment of 18 chunks": (18, 1), "one segment of 18 chunks, wide": (18, 1), "one segment, narrow values": (19, 1)}
    assert p["two segments of 19 chunks"][1:] == (19, 2) and p["segments of 17 chunks, odd"][1:] == (17, 2)
    for case in p:
        if case.split()[0].isdigit():
            assert p[case][2] == int(case.split()[0]), case
    # the scan: a second and a third round of 64 segments, and a state that is no multiple of 4 in both of these
    assert p["odd state of many segments"][2] > 1
    D, V = DECAY["67 segments, odd"][4:6]
    assert D * V % 4 and DECAY["odd state of many segments"][4] * DECAY["odd state of many segments"][5] % 4


def test_ragged_segments_end_before_at_and_after_a_round(rules):
    B, T, H, K, D, V, lengths = DECAY["67 segments"]
    _, per, nseg = plans(rules)["67 segments"]
    last = [min(-(-n // (64 * per)), nseg) - 1 for n in lengths]
    assert {62, 63, 64, 65, 66} <= set(last)


def test_every_width_is_cut_into_segments(rules):
    got = [tuple(map(int, p.split())) for p in rules([f"decay 4 400 {V}" for _, V in FORMS])]
    assert all(chunked and nseg > 1 for chunked, _, nseg in got)
    # padded head width, waves, and direct loads or not: all twelve
    have = {(64 if D <= 64 else 128, 1 if V <= 32 else 2 if V <= 64 else 4, D % 8 == 0 and V % 8 == 0) for D, V in FORMS}
    assert len(have) == 12
