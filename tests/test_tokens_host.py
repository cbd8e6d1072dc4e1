"""Token operators, host side: descriptor structs, and the refusals, which come before anything touches the GPU."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2502_20762_amd import ncodec as nc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000000000  # never dereferenced: every call below is refused, or has nothing to do


@pytest.mark.parametrize("name", ["ncodec_linear_shape", "ncodec_qk_shape", "ncodec_decay_shape"])
def test_struct_matches_header(name, tmp_path):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ncodec.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, text, re.S).group(1)
    names = [re.sub(r"\[.*?\]", "", f).strip() for line in body.split(";") if line.strip()
             for f in re.sub(r"^\s*\w+\s", "", line.strip()).split(",")]
    struct = getattr(nc, name)
    assert names == [f for f, _ in struct._fields_]
    src = tmp_path / "s.c"
    probes = "".join(f'printf("%zu ", offsetof({name}, {n}));' for n in names)
    src.write_text(f'#include "{ROOT}/include/ncodec.h"\n#include <stdio.h>\n'
                   f'int main(void) {{ {probes} printf("%zu\\n", sizeof({name})); return 0; }}')
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "s")], check=True)
    out = subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [getattr(struct, n).offset for n in names] + [ctypes.sizeof(struct)]


def linear_shape(**kw):
    s = dict(dtype=0, act=0, gated=0, reserved=0, m=4, n=8, k=16, ldx=16, ldw=16, ldr=8, ldy=8)
    s.update(kw)
    return nc.ncodec_linear_shape(**s)


def linear(shape, x=FAKE, w=FAKE, b=0, r=0, y=FAKE):
    with pytest.raises(nc.NcodecError) as e:
        nc.ncodec_linear(shape, x, w, b, r, y)
    assert "linear" in nc.ncodec_last_error(None)
    return e.value.status


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(act=5), dict(act=-1), dict(gated=2), dict(reserved=1)])
def test_linear_refuses_values(bad):
    assert linear(linear_shape(**bad)) == nc.NCODEC_EINVAL


@pytest.mark.parametrize("bad", [dict(m=-1), dict(m=1 << 31), dict(n=0), dict(k=0), dict(n=(1 << 20) + 1, ldy=1 << 21),
                                 dict(k=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), dict(ldx=15), dict(ldw=15),
                                 dict(ldy=7), dict(ldy=(1 << 40) + 1)])
def test_linear_refuses_shapes(bad):
    assert linear(linear_shape(**bad)) == nc.NCODEC_ESHAPE


def test_linear_refuses_pointers():
    s = linear_shape()
    for kw in (dict(x=0), dict(w=0), dict(y=0), dict(x=FAKE + 1), dict(b=FAKE + 1), dict(y=FAKE + 1)):
        assert linear(s, **kw) == nc.NCODEC_EINVAL
    assert linear(linear_shape(ldr=7), r=FAKE + 64) == nc.NCODEC_ESHAPE
    assert linear(linear_shape(ldr=9), r=FAKE) == nc.NCODEC_EINVAL  # in place with another stride
    with pytest.raises(nc.NcodecError):
        lib = nc.load_library()
        nc._check(lib.ncodec_linear(None, FAKE, FAKE, None, None, FAKE, None))
    nc.ncodec_linear(linear_shape(m=0), 0, 0, 0, 0, 0)  # no rows: nothing to do


def qk_shape(**kw):
    s = dict(dtype=1, norm=1, axes=3, section=(ctypes.c_int32 * 3)(2, 1, 1), interleaved=0, q_heads=2, k_heads=1,
             head_dim=8, eps=1e-6, reserved=0, tokens=4, q_token_stride=16, q_head_stride=8, k_token_stride=8,
             k_head_stride=8, qo_token_stride=16, qo_head_stride=8, ko_token_stride=8, ko_head_stride=8)
    s.update(kw)
    if isinstance(s["section"], tuple):
        s["section"] = (ctypes.c_int32 * 3)(*s["section"])
    return nc.ncodec_qk_shape(**s)


def rope(shape, q=FAKE, k=FAKE, wq=0, wk=0, pos=FAKE, freq=FAKE, qo=FAKE, ko=FAKE):
    with pytest.raises(nc.NcodecError) as e:
        nc.ncodec_qk_norm_rope(shape, q, k, wq, wk, pos, freq, qo, ko)
    assert "qk_norm_rope" in nc.ncodec_last_error(None)
    return e.value.status


@pytest.mark.parametrize("bad", [dict(dtype=-1), dict(norm=2), dict(interleaved=3), dict(eps=-1.0), dict(reserved=4),
                                 dict(eps=float("nan")), dict(eps=float("inf"))])
def test_qk_refuses_values(bad):
    assert rope(qk_shape(**bad)) == nc.NCODEC_EINVAL


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(tokens=1 << 31), dict(q_heads=-1), dict(k_heads=4097),
                                 dict(head_dim=0), dict(head_dim=257), dict(axes=4), dict(axes=-1),
                                 dict(section=(2, 2, 1)), dict(section=(-1, 1, 1)), dict(axes=2),
                                 dict(q_token_stride=-8), dict(qo_token_stride=7), dict(qo_head_stride=7),
                                 dict(ko_token_stride=0)])
def test_qk_refuses_shapes(bad):
    assert rope(qk_shape(**bad)) == nc.NCODEC_ESHAPE


def test_qk_refuses_pointers():
    s = qk_shape()
    for kw in (dict(q=0), dict(k=0), dict(pos=0), dict(freq=0), dict(qo=0), dict(ko=0), dict(q=FAKE + 1),
               dict(wq=FAKE + 1), dict(pos=FAKE + 2)):
        assert rope(s, **kw) == nc.NCODEC_EINVAL
    nc.ncodec_qk_norm_rope(qk_shape(tokens=0), 0, 0, 0, 0, 0, 0, 0, 0)
    nc.ncodec_qk_norm_rope(qk_shape(q_heads=0, k_heads=0), 0, 0, 0, 0, 0, 0, 0, 0)


def decay_shape(**kw):
    s = dict(dtype=0, heads=4, kv_heads=2, head_dim=16, value_dim=8, scale=0.25, batch=2, tokens=5)
    for t, h, d in (("q", 4, 16), ("k", 2, 16), ("v", 2, 8), ("o", 4, 8)):
        s.update({t + "_batch_stride": 5 * h * d, t + "_token_stride": h * d, t + "_head_stride": d})
    s.update(kw)
    return nc.ncodec_decay_shape(**s)


def decay(shape, q=FAKE, k=FAKE, v=FAKE, ld=FAKE, lengths=0, si=0, so=0, o=FAKE, ws=FAKE, nb=1 << 40):
    with pytest.raises(nc.NcodecError) as e:
        nc.ncodec_decay_attention(shape, q, k, v, ld, lengths, si, so, o, ws, nb)
    assert "decay_attention" in nc.ncodec_last_error(None)
    return e.value.status


@pytest.mark.parametrize("bad", [dict(dtype=7), dict(scale=float("inf")), dict(scale=float("nan"))])
def test_decay_refuses_values(bad):
    assert decay(decay_shape(**bad)) == nc.NCODEC_EINVAL
    assert nc.ncodec_decay_attention_workspace_bytes(decay_shape(**bad)) == 0


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(tokens=1 << 31), dict(heads=0), dict(heads=4098, kv_heads=2),
                                 dict(kv_heads=3), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=129),
                                 dict(value_dim=129), dict(batch=-1), dict(batch=1 << 22), dict(q_batch_stride=-1),
                                 dict(o_token_stride=7), dict(o_head_stride=7), dict(o_batch_stride=0)])
def test_decay_refuses_shapes(bad):
    assert decay(decay_shape(**bad)) == nc.NCODEC_ESHAPE


def test_decay_refuses_pointers():
    s = decay_shape()
    for kw in (dict(q=0), dict(k=0), dict(v=0), dict(ld=0), dict(o=0), dict(q=FAKE + 1), dict(ld=FAKE + 2),
               dict(lengths=FAKE + 2), dict(si=FAKE + 2), dict(so=FAKE + 2)):
        assert decay(s, **kw) == nc.NCODEC_EINVAL
    nc.ncodec_decay_attention(decay_shape(batch=0), 0, 0, 0, 0, 0, 0, 0, 0)
    # one long sequence of few heads is split over workgroups, which meet in the workspace
    long = decay_shape(batch=1, tokens=100000, head_dim=64, value_dim=64)
    need = nc.ncodec_decay_attention_workspace_bytes(long)
    if need:
        for kw in (dict(ws=0), dict(nb=need - 1), dict(ws=FAKE + 16)):
            assert decay(long, **kw) == nc.NCODEC_ENOMEM
