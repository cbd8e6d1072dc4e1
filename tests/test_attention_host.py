"""Attention with a window and over a cache, and the cache's upkeep, host side: descriptor structs, and the refusals, which
come before anything touches the GPU."""
import pytest

import test_tokens_host as host
from paper_2502_20762_amd import ncodec as nc

FAKE = host.FAKE
FAR = [FAKE + (i << 30) for i in range(1, 14)]


@pytest.mark.parametrize("name", ["ncodec_window_shape", "ncodec_cache_shape", "ncodec_paged_shape", "ncodec_append_shape",
                                  "ncodec_evict_shape"])
def test_struct_matches_header(name, tmp_path):
    host.test_struct_matches_header(name, tmp_path)


def refused(fn, what, *args):
    with pytest.raises(nc.NcodecError) as e:
        fn(*args)
    assert what in nc.ncodec_last_error(None)
    return e.value.status


def window_shape(**kw):
    s = dict(dtype=0, heads=4, kv_heads=2, head_dim=16, value_dim=8, scale=0.25, batch=2, tokens=5, window=3, sinks=1)
    for t, h, d in (("q", 4, 16), ("k", 2, 16), ("v", 2, 8), ("o", 4, 8)):
        s.update({t + "_batch_stride": 5 * h * d, t + "_token_stride": h * d, t + "_head_stride": d})
    s.update(kw)
    return nc.ncodec_window_shape(**s)


def window(shape, **kw):
    p = dict(q=FAR[0], k=FAR[1], v=FAR[2], lengths=0, o=FAR[3])
    p.update(kw)
    return refused(nc.ncodec_window_attention, "window_attention", shape, *p.values())


@pytest.mark.parametrize("bad", [dict(dtype=7), dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=-2e30)])
def test_window_refuses_values(bad):
    assert window(window_shape(**bad)) == nc.NCODEC_EINVAL


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(tokens=1 << 31), dict(heads=0), dict(heads=4098, kv_heads=2),
                                 dict(kv_heads=3), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=129),
                                 dict(value_dim=129), dict(batch=-1), dict(batch=1 << 22), dict(q_batch_stride=-1),
                                 dict(o_token_stride=7), dict(o_head_stride=7), dict(o_batch_stride=0), dict(window=-1),
                                 dict(sinks=-1), dict(window=1 << 31), dict(sinks=1 << 31), dict(k_token_stride=(1 << 40) + 1)])
def test_window_refuses_shapes(bad):
    assert window(window_shape(**bad)) == nc.NCODEC_ESHAPE


def test_window_refuses_pointers():
    s = window_shape()
    for kw in (dict(q=0), dict(k=0), dict(v=0), dict(o=0), dict(q=FAKE + 1), dict(lengths=FAKE + 2)):
        assert window(s, **kw) == nc.NCODEC_EINVAL
    for i, name in enumerate(("q", "k", "v", "lengths")):
        assert window(s, **{name: FAR[5], "o": FAR[5]}) == nc.NCODEC_EINVAL, name
    nc.ncodec_window_attention(window_shape(tokens=0), 0, 0, 0, 0, 0)
    nc.ncodec_window_attention(window_shape(batch=0), 0, 0, 0, 0, 0)


def cache_shape(**kw):
    s = dict(dtype=0, kv_heads=2, head_dim=16, value_dim=8, page_size=4, reserved=0, pages=10, k_page_stride=128,
             k_token_stride=32, k_head_stride=16, v_page_stride=64, v_token_stride=16, v_head_stride=8)
    s.update(kw)
    return nc.ncodec_cache_shape(**s)


def paged_shape(**kw):
    s = dict(heads=4, scale=0.25, batch=3, columns=3, table_stride=3, window=0, sinks=0, q_batch_stride=64, q_head_stride=16,
             o_batch_stride=32, o_head_stride=8)
    s.update(kw)
    return nc.ncodec_paged_shape(**s)


def append_shape(**kw):
    s = dict(batch=3, tokens=2, columns=3, table_stride=3, k_batch_stride=64, k_token_stride=32, k_head_stride=16,
             v_batch_stride=32, v_token_stride=16, v_head_stride=8)
    s.update(kw)
    return nc.ncodec_append_shape(**s)


def evict_shape(**kw):
    s = dict(batch=3, columns=3, table_stride=3, new_columns=2, new_table_stride=2, keep=6, sinks=1, recent=2)
    s.update(kw)
    return nc.ncodec_evict_shape(**s)


def paged(cache, shape, **kw):
    p = dict(q=FAR[0], k=FAR[1], v=FAR[2], table=FAR[3], lengths=FAR[4], mass=0, o=FAR[5], ws=FAR[6], nb=1 << 60)
    p.update(kw)
    return refused(nc.ncodec_paged_attention, "paged_attention", cache, shape, *p.values())


def append(cache, shape, **kw):
    p = dict(k=FAR[0], v=FAR[1], kc=FAR[2], vc=FAR[3], table=FAR[4], starts=FAR[5], counts=0, mass=0)
    p.update(kw)
    return refused(nc.ncodec_cache_append, "cache_append", cache, shape, *p.values())


def evict(cache, shape, **kw):
    p = dict(kc=FAR[0], vc=FAR[1], table=FAR[2], lengths=FAR[3], mass=FAR[4], new_table=FAR[5], new_lengths=FAR[6],
             new_mass=FAR[7], kept=FAR[8], ws=FAR[9], nb=1 << 60)
    p.update(kw)
    return refused(nc.ncodec_cache_evict, "cache_evict", cache, shape, *p.values())


CALLS = [(paged, paged_shape), (append, append_shape), (evict, evict_shape)]


@pytest.mark.parametrize("call,shape", CALLS)
@pytest.mark.parametrize("bad", [dict(dtype=2), dict(dtype=-1), dict(reserved=1)])
def test_cache_refuses_values(bad, call, shape):
    assert call(cache_shape(**bad), shape()) == nc.NCODEC_EINVAL


@pytest.mark.parametrize("call,shape", CALLS)
@pytest.mark.parametrize("bad", [dict(kv_heads=0), dict(kv_heads=4097), dict(head_dim=0), dict(head_dim=129), dict(value_dim=0),
                                 dict(value_dim=129), dict(page_size=0), dict(page_size=-4), dict(page_size=3),
                                 dict(page_size=8192), dict(pages=-1), dict(pages=1 << 31), dict(k_page_stride=-1),
                                 dict(v_head_stride=(1 << 40) + 1)])
def test_cache_refuses_shapes(bad, call, shape):
    assert call(cache_shape(**bad), shape()) == nc.NCODEC_ESHAPE


@pytest.mark.parametrize("call,shape", CALLS[1:])
@pytest.mark.parametrize("bad", [dict(k_page_stride=15), dict(k_token_stride=0), dict(k_head_stride=15), dict(v_page_stride=0),
                                 dict(v_token_stride=7), dict(v_head_stride=7)])
def test_rows_that_are_written_are_different_ones(bad, call, shape):
    assert call(cache_shape(**bad), shape()) == nc.NCODEC_ESHAPE


@pytest.mark.parametrize("call,shape", CALLS)
@pytest.mark.parametrize("bad", [dict(batch=-1), dict(batch=1 << 24), dict(batch=1 << 23), dict(columns=-1), dict(columns=1 << 29),
                                 dict(columns=1 << 62), dict(table_stride=-1)])
def test_tables_are_refused(bad, call, shape):
    assert call(cache_shape(), shape(**bad)) == nc.NCODEC_ESHAPE


def test_paged_refuses():
    for bad in (dict(heads=0), dict(heads=3), dict(heads=4098), dict(window=-1), dict(sinks=-1), dict(window=1 << 31),
                dict(sinks=1 << 31), dict(q_head_stride=-1), dict(o_head_stride=7), dict(o_batch_stride=7), dict(batch=1 << 22)):
        assert paged(cache_shape(), paged_shape(**bad)) == nc.NCODEC_ESHAPE, bad
        assert nc.ncodec_paged_attention_workspace_bytes(cache_shape(), paged_shape(**bad), 1) == 0
    for bad in (float("nan"), float("-inf"), 2e30):
        assert paged(cache_shape(), paged_shape(scale=bad)) == nc.NCODEC_EINVAL
    for kw in (dict(q=0), dict(k=0), dict(v=0), dict(table=0), dict(lengths=0), dict(o=0), dict(q=FAKE + 1), dict(k=FAKE + 1),
               dict(table=FAKE + 2), dict(lengths=FAKE + 2), dict(mass=FAKE + 2)):
        assert paged(cache_shape(), paged_shape(), **kw) == nc.NCODEC_EINVAL, kw
    for name in ("q", "k", "v", "table", "lengths"):
        assert paged(cache_shape(), paged_shape(), **{name: FAR[9], "o": FAR[9]}) == nc.NCODEC_EINVAL, name
        assert paged(cache_shape(), paged_shape(), **{name: FAR[9], "mass": FAR[9]}) == nc.NCODEC_EINVAL, name
    assert paged(cache_shape(), paged_shape(), mass=FAR[9], o=FAR[9]) == nc.NCODEC_EINVAL
    nc.ncodec_paged_attention(cache_shape(), paged_shape(batch=0), 0, 0, 0, 0, 0, 0, 0)
    # a long cache of few rows is split over workgroups, and weights need the scores, which meet in the workspace
    big = paged_shape(columns=100000)
    for mass in (0, 1):
        need = nc.ncodec_paged_attention_workspace_bytes(cache_shape(), big, mass)
        assert need > 0
        for kw in (dict(ws=0), dict(nb=need - 1), dict(ws=FAR[6] + 16)):
            assert paged(cache_shape(), big, mass=FAR[9] if mass else 0, **kw) == nc.NCODEC_ENOMEM


def test_append_refuses():
    for bad in (dict(tokens=-1), dict(tokens=1 << 31), dict(k_batch_stride=-1), dict(v_token_stride=(1 << 40) + 1)):
        assert append(cache_shape(), append_shape(**bad)) == nc.NCODEC_ESHAPE, bad
    for kw in (dict(k=0), dict(v=0), dict(kc=0), dict(vc=0), dict(table=0), dict(starts=0), dict(k=FAKE + 1), dict(kc=FAKE + 1),
               dict(starts=FAKE + 2), dict(counts=FAKE + 2), dict(mass=FAKE + 2)):
        assert append(cache_shape(), append_shape(), **kw) == nc.NCODEC_EINVAL, kw
    for out in ("kc", "vc", "mass"):
        for name in ("k", "v", "kc", "vc", "table", "starts", "counts", "mass"):
            if name != out:
                assert append(cache_shape(), append_shape(), **{name: FAR[9], out: FAR[9]}) == nc.NCODEC_EINVAL, (out, name)
    for kw in (dict(batch=0), dict(tokens=0), dict(columns=0)):
        nc.ncodec_cache_append(cache_shape(), append_shape(**kw), 0, 0, 0, 0, 0, 0)
    nc.ncodec_cache_append(cache_shape(pages=0), append_shape(), 0, 0, 0, 0, 0, 0)


def test_evict_refuses():
    for bad in (dict(keep=0), dict(keep=9), dict(sinks=-1), dict(recent=-1), dict(sinks=7), dict(sinks=3, recent=4),
                dict(new_columns=-1), dict(new_columns=1 << 29), dict(new_table_stride=-1), dict(sinks=1 << 62, recent=1 << 62)):
        assert evict(cache_shape(), evict_shape(**bad)) == nc.NCODEC_ESHAPE, bad
    names = ("kc", "vc", "table", "lengths", "mass", "new_table", "new_lengths", "new_mass", "kept")
    for name in names:
        assert evict(cache_shape(), evict_shape(), **{name: 0}) == nc.NCODEC_EINVAL, name
        assert evict(cache_shape(), evict_shape(), **{name: FAKE + 1}) == nc.NCODEC_EINVAL, name
    for out in ("kc", "vc", "new_lengths", "new_mass", "kept"):
        for name in names:
            if name != out:
                assert evict(cache_shape(), evict_shape(), **{name: FAR[10], out: FAR[10]}) == nc.NCODEC_EINVAL, (out, name)
    # a long sequence is shared by workgroups, which meet in the workspace
    big = evict_shape(columns=100000)
    need = nc.ncodec_cache_evict_workspace_bytes(cache_shape(), big)
    assert need > 0 and nc.ncodec_cache_evict_workspace_bytes(cache_shape(), evict_shape(columns=100000, keep=0)) == 0
    for kw in (dict(ws=0), dict(nb=need - 1), dict(ws=FAR[9] + 16)):
        assert evict(cache_shape(), big, **kw) == nc.NCODEC_ENOMEM
    nc.ncodec_cache_evict(cache_shape(), evict_shape(batch=0), 0, 0, 0, 0, 0, 0, 0, 0, 0)


def test_keys_and_values_beside_each_other_in_a_page_are_apart():
    # nothing is enqueued: no tokens fit a table without columns, but the caches are looked at first where there are some
    beside = cache_shape(k_page_stride=192, k_token_stride=48, k_head_stride=24, v_page_stride=192, v_token_stride=48,
                         v_head_stride=24)
    assert append(beside, append_shape(), kc=FAR[2], vc=FAR[2] + 2 * 15) == nc.NCODEC_EINVAL
    assert append(beside, append_shape(), kc=FAR[2], vc=FAR[2] + 2 * 16, starts=FAKE + 2) == nc.NCODEC_EINVAL
    assert "aligned" in nc.ncodec_last_error(None)
    assert append(beside, append_shape(), kc=FAR[2], vc=FAR[2] + 2 * 16, k=FAR[2] + 2) == nc.NCODEC_EINVAL
    assert "overlaps" in nc.ncodec_last_error(None)
