"""Which outputs of the token operators may be given: the check that operands lie apart, against the bytes themselves,
and the refusals of the entry points, which come before anything touches the GPU."""
import os
import random
import subprocess

import pytest

from paper_2502_20762_amd import ncodec as nc
from test_tokens_host import FAKE, decay, decay_shape, linear, linear_shape, qk_shape, rope

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROBE = r"""
#include "areas.hpp"
#include <cstdio>
int main() {
  long long v[16];
  for (;;) {
    for (long long& x : v)
      if (scanf("%lld", &x) != 1) return 0;
    const nc::Area a((const void*)(v[0]), v[1], {v[2], v[3], v[4], v[5], v[6], v[7]}),
        b((const void*)(v[8]), v[9], {v[10], v[11], v[12], v[13], v[14], v[15]});
    printf("%d %d\n", nc::apart(a, b), nc::apart(b, a));
  }
}
"""


@pytest.fixture(scope="module")
def apart(tmp_path_factory):
    d = tmp_path_factory.mktemp("areas")
    (d / "p.cpp").write_text(PROBE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2502_20762_amd", "csrc"), str(d / "p.cpp"),
                    "-o", str(d / "p")], check=True)

    def run(pairs):
        text = "\n".join(" ".join(map(str, (*a, *b))) for a, b in pairs)
        out = subprocess.run([str(d / "p")], input=text, check=True, capture_output=True, text=True).stdout.split()
        assert len(out) == 2 * len(pairs) and out[::2] == out[1::2]  # either way round
        return [x == "1" for x in out[::2]]

    return run


def elements(a):
    base, run, *dims = a
    at = {base}
    for n, s in zip(dims[::2], dims[1::2]):
        at = {x + 2 * s * i for x in at for i in range(n)}
    return {x + 2 * i for x in at for i in range(run)}


def test_apart_is_never_said_of_operands_that_share_a_byte(apart):
    rng = random.Random(1)
    pairs = [tuple((1000 + 2 * rng.randrange(60), rng.randrange(1, 6),
                    *(x for _ in range(3) for x in (rng.choice([1, 1, 2, 3, 5]), rng.randrange(0, 40)))) for _ in range(2))
             for _ in range(4000)]
    said = apart(pairs)
    assert 200 < sum(said) < 3800
    for (a, b), ok in zip(pairs, said):
        assert not ok or not elements(a) & elements(b), (a, b)


def test_parts_of_one_buffer_are_apart(apart):
    # columns, heads, tokens and batches of a (batch, tokens, heads, dim) buffer, in either order of tokens and heads
    rng = random.Random(2)
    pairs = []
    for _ in range(1000):
        size = [rng.randrange(1, 7) for _ in range(4)]  # batch, two dimensions, columns
        cut = rng.randrange(4)
        size[cut] += 1
        stride = [size[1] * size[2] * size[3], size[2] * size[3], size[3], 1]
        first, rest = list(size), list(size)
        first[cut] = rng.randrange(1, size[cut])
        rest[cut] = size[cut] - first[cut]
        order = [0, 1, 2] if rng.random() < 0.5 else [0, 2, 1]

        def area(base, n):
            return (base, n[3], *(x for d in order for x in (n[d], stride[d])))

        pairs.append((area(4096, first), area(4096 + 2 * first[cut] * stride[cut], rest)))
    for (a, b), ok in zip(pairs, apart(pairs)):
        assert ok and not elements(a) & elements(b), (a, b)


def test_linear_refuses_an_output_over_an_input():
    # x is 4 x 16 at FAKE, y 4 x 8
    far = FAKE + (1 << 20)
    s = linear_shape(ldx=16, ldy=16)
    for y in (FAKE, FAKE + 16, FAKE + 100, FAKE - 100):
        assert linear(s, w=far, y=y) == nc.NCODEC_EINVAL
    assert linear(linear_shape(ldy=24, ldx=24), w=far, y=FAKE + 2 * 15) == nc.NCODEC_EINVAL
    assert linear(linear_shape(), x=far, y=FAKE) == nc.NCODEC_EINVAL  # w
    assert linear(linear_shape(), x=far, w=2 * far, b=FAKE + 2, y=FAKE) == nc.NCODEC_EINVAL
    assert linear(linear_shape(), x=far, w=2 * far, r=FAKE + 16, y=FAKE) == nc.NCODEC_EINVAL
    assert "overlaps" in nc.ncodec_last_error(None)


def test_rope_refuses_outputs_over_what_they_are_not():
    far = [FAKE + (i << 20) for i in range(1, 9)]
    free = dict(q=far[0], k=far[1], wq=far[2], wk=far[3], pos=far[4], freq=far[5], qo=far[6], ko=far[7])
    for out in ("qo", "ko"):
        for name in free:
            if name != out and (out, name) not in (("qo", "q"), ("ko", "k")):
                assert rope(qk_shape(), **{**free, out: free[name]}) == nc.NCODEC_EINVAL, (out, name)
    assert rope(qk_shape(), **{**free, "qo": free["q"] + 2}) == nc.NCODEC_EINVAL
    # the same memory at other strides is not in place
    assert rope(qk_shape(qo_token_stride=32), **{**free, "qo": free["q"]}) == nc.NCODEC_EINVAL


def test_decay_refuses_outputs_over_what_they_are_not():
    far = [FAKE + (i << 20) for i in range(1, 9)]
    free = dict(q=far[0], k=far[1], v=far[2], ld=far[3], lengths=far[4], si=far[5], so=far[6], o=far[7])
    for out in ("o", "so"):
        for name in free:
            if name != out and (out, name) != ("so", "si"):
                assert decay(decay_shape(), **{**free, out: free[name]}) == nc.NCODEC_EINVAL, (out, name)
    assert decay(decay_shape(), **{**free, "so": free["si"] + 4}) == nc.NCODEC_EINVAL
