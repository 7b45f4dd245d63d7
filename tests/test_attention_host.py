"""Refusals of the attention operators' entry points: they come from the host before any launch, so none of this needs a
GPU. Addresses here are never followed."""
import ctypes

import pytest

from paper_2007_06919_amd import aqd

A = 1 << 24   # an address for each tensor, far from the others
ADDR = {name: A * (i + 1) for i, name in enumerate((
    "q", "k", "v", "q_weight", "k_weight", "position", "table", "yq", "yk", "slots", "cache", "tables", "lengths", "q_start",
    "k_start", "y", "workspace"))}


def heads_call(**kw):
    d = dict(tokens=4, q_heads=6, k_heads=2, dim=64, rot=32, pairs=aqd.PAIRS_HALVES, type=aqd.BF16, positions=100, eps=1e-6,
             q_token=640, q_head=64, k_token=640, k_head=64, yq_token=384, yq_head=64, yk_token=128, yk_head=64, **ADDR)
    d.update(kw)
    aqd.heads_run(d["tokens"], d["q_heads"], d["k_heads"], d["dim"], d["rot"], d["pairs"], d["type"], d["positions"], d["eps"],
                  d["q"], d["q_token"], d["q_head"], d["k"], d["k_token"], d["k_head"], d["q_weight"], d["k_weight"], d["position"],
                  d["table"], d["yq"], d["yq_token"], d["yq_head"], d["yk"], d["yk_token"], d["yk_head"], 0)


def shape(kw):
    c = {n: kw.pop(n) for n in ("heads", "dim", "group", "page", "pages") if n in kw}
    return aqd.QcacheDesc(*(c.get(n, v) for n, v in (("heads", 2), ("dim", 64), ("group", 32), ("page", 16), ("pages", 5))))


def write_call(call=aqd.qcache_write, **kw):
    c = shape(kw)
    d = dict(tokens=4, type=aqd.BF16, k_token=128, k_head=64, v_token=128, v_head=64, **ADDR)
    d.update(kw)
    rows = (d["k"], d["k_token"], d["k_head"], d["v"], d["v_token"], d["v_head"])
    if call is aqd.qcache_write:
        call(c, d["tokens"], d["type"], *rows, d["slots"], d["cache"], 0)
    else:
        call(c, d["tokens"], d["type"], d["cache"], d["slots"], *rows, 0)


def read_call(**kw):
    write_call(aqd.qcache_read, **kw)


def qattn_call(**kw):
    c = shape(kw)
    d = dict(batch=3, q_heads=4, queries=3, max_queries=1, max_keys=60, type=aqd.F16, scale=0.125, ld_table=4, q_token=256,
             q_head=64, y_token=256, y_head=64, ws_bytes=1 << 20, **ADDR)
    d["q_start"] = None
    d.update(kw)
    aqd.qattn_run(c, d["batch"], d["q_heads"], d["queries"], d["max_queries"], d["max_keys"], d["type"], d["scale"], d["q"],
                  d["q_token"], d["q_head"], d["q_start"], d["cache"], d["tables"], d["ld_table"], d["lengths"], d["y"], d["y_token"],
                  d["y_head"], d["workspace"], d["ws_bytes"], 0)


def attn_call(**kw):
    d = dict(batch=2, q_heads=4, heads=2, dim=64, queries=10, keys=12, max_queries=6, max_keys=7, causal=1, type=aqd.BF16, scale=0.125,
             q_token=256, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64, y_token=256, y_head=64, ws_bytes=1 << 20, **ADDR)
    d.update(kw)
    aqd.attn_run(d["batch"], d["q_heads"], d["heads"], d["dim"], d["queries"], d["keys"], d["max_queries"], d["max_keys"], d["causal"],
                 d["type"], d["scale"], d["q"], d["q_token"], d["q_head"], d["k"], d["k_token"], d["k_head"], d["v"], d["v_token"],
                 d["v_head"], d["q_start"], d["k_start"], d["y"], d["y_token"], d["y_head"], d["workspace"], d["ws_bytes"], 0)


def refused(call, status=aqd.AQD_ERR_INVALID, **kw):
    with pytest.raises(aqd.AqdError) as e:
        call(**kw)
    assert e.value.status == status and aqd.last_error()


@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(q_heads=0), dict(k_heads=-1), dict(dim=63), dict(dim=0), dict(dim=1026), dict(rot=31), dict(rot=66), dict(rot=-2),
    dict(pairs=2), dict(type=3), dict(eps=-1e-9), dict(eps=float("nan")), dict(positions=-1), dict(q=None), dict(k=None), dict(yq=None),
    dict(yk=None), dict(position=None), dict(table=None), dict(q=A + 1), dict(k_weight=ADDR["k_weight"] + 1), dict(table=ADDR["table"] + 2),
    dict(tokens=1 << 28, q_heads=8),
    # strides: heads that share elements, tokens that do, an expanded tensor, far too large
    dict(q_head=63), dict(q_token=320), dict(q_token=0), dict(q_head=0), dict(yq_token=300), dict(yk_head=32), dict(q_token=-640),
    dict(k_token=1 << 60), dict(yq_head=1 << 62),
    # overlaps: in place with other strides, over the keys, over one another, over the table or a weight
    dict(yq=A), dict(yq=A + 128, yq_token=640), dict(yq=ADDR["k"] - 2), dict(yk=ADDR["yq"] + 16), dict(yq=ADDR["table"]), dict(yk=ADDR["q_weight"]),
    dict(yk=ADDR["q"], yk_token=640), dict(yk=ADDR["position"]),
])
def test_heads_refuses(bad):
    refused(heads_call, **bad)


SHAPES = [dict(heads=0), dict(dim=96), dict(dim=512), dict(group=16), dict(group=128), dict(page=8), dict(page=48), dict(page=512), dict(pages=-1),
          dict(pages=1 << 27, page=16), dict(heads=70000)]


@pytest.mark.parametrize("bad", SHAPES)
def test_cache_shapes_are_refused(bad):
    with pytest.raises(aqd.AqdError):
        aqd.qcache_bytes(shape(dict(bad)))
    for call in (write_call, read_call, qattn_call):
        refused(call, **bad)


@pytest.mark.parametrize("call", [write_call, read_call])
@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(type=4), dict(k=None), dict(v=None), dict(slots=None), dict(cache=None), dict(k=ADDR["k"] + 1), dict(slots=ADDR["slots"] + 2),
    dict(cache=ADDR["cache"] + 8), dict(k_token=100), dict(v_head=60), dict(k_token=0), dict(v_token=1 << 59), dict(k=ADDR["cache"] + 64),
    dict(tokens=1 << 30, heads=2),
])
def test_cache_rows_are_refused(call, bad):
    refused(call, **bad)


def test_a_read_refuses_outputs_that_meet():
    refused(read_call, v=ADDR["k"] + 64)
    refused(read_call, k=ADDR["slots"])
    refused(write_call, slots=ADDR["cache"] + 32)


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(queries=-1), dict(max_queries=-1), dict(max_keys=-1), dict(q_heads=0), dict(q_heads=3), dict(type=5), dict(q_heads=65538),
    dict(scale=float("inf")), dict(scale=float("nan")), dict(queries=4), dict(q=None), dict(y=None), dict(cache=None), dict(tables=None),
    dict(lengths=None), dict(q=A + 1), dict(y=ADDR["y"] + 1), dict(cache=ADDR["cache"] + 4), dict(workspace=ADDR["workspace"] + 8),
    dict(lengths=ADDR["lengths"] + 1), dict(ld_table=0), dict(q_token=255), dict(y_head=32), dict(y=A), dict(y=ADDR["lengths"]),
    dict(y=ADDR["cache"]), dict(y=ADDR["tables"]), dict(q_start=ADDR["q_start"] + 2), dict(q_start=ADDR["y"]), dict(max_keys=2 ** 31 - 1),
])
def test_qattn_refuses(bad):
    refused(qattn_call, **bad)


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(queries=-1), dict(keys=-1), dict(max_queries=-1), dict(max_keys=-1), dict(heads=0), dict(heads=3), dict(dim=0), dict(causal=2),
    dict(type=9), dict(scale=float("nan")), dict(q=None), dict(k=None), dict(v=None), dict(y=None), dict(q_start=None), dict(k_start=None),
    dict(k=ADDR["k"] + 1), dict(k_start=ADDR["k_start"] + 2), dict(workspace=ADDR["workspace"] + 4), dict(k_token=100), dict(v_token=0), dict(y_token=64),
    dict(q_head=8), dict(y=ADDR["q"]), dict(y=ADDR["v"] + 128), dict(y=ADDR["k_start"]), dict(y=ADDR["k"] - 2), dict(q_heads=65538),
])
def test_attn_refuses(bad):
    refused(attn_call, **bad)


def test_attention_in_fp32_is_not_there():
    refused(qattn_call, aqd.AQD_ERR_UNSUPPORTED, type=aqd.F32)
    refused(attn_call, aqd.AQD_ERR_UNSUPPORTED, type=aqd.F32)


@pytest.mark.parametrize("dim", [1, 60, 100, 264])
def test_attention_of_other_head_sizes_is_not_there(dim):
    wide = 4 * dim
    refused(attn_call, aqd.AQD_ERR_UNSUPPORTED, dim=dim, q_head=dim, k_head=dim, v_head=dim, y_head=dim, q_token=wide, k_token=wide, v_token=wide,
            y_token=wide)


def test_null_descriptions_are_refused():
    L, size = aqd.lib(), ctypes.c_size_t(5)
    assert L.aqd_heads_run(None, A, A, A, A, A, A, A, A, None) == aqd.AQD_ERR_INVALID
    assert L.qcache_bytes(None, ctypes.byref(size)) == aqd.AQD_ERR_INVALID
    assert L.qcache_bytes(ctypes.byref(aqd.QcacheDesc(1, 64, 32, 16, 1)), None) == aqd.AQD_ERR_INVALID
    assert L.qcache_write(None, A, A, A, A, None) == aqd.AQD_ERR_INVALID
    assert L.qcache_read(None, A, A, A, A, None) == aqd.AQD_ERR_INVALID
    assert L.qattn_workspace(None, ctypes.byref(size)) == aqd.AQD_ERR_INVALID
    assert L.qattn_run(None, A, A, A, A, A, A, A, 0, None) == aqd.AQD_ERR_INVALID
    assert L.aqd_attn_workspace(None, ctypes.byref(size)) == aqd.AQD_ERR_INVALID
    assert L.aqd_attn_run(None, A, A, A, A, A, A, A, 0, None) == aqd.AQD_ERR_INVALID


def test_nothing_is_no_work():
    none = dict.fromkeys(ADDR)
    heads_call(tokens=0, **none)
    write_call(tokens=0, **none)
    read_call(tokens=0, **none)
    write_call(pages=0, **none)
    qattn_call(batch=0, queries=0, **none)
    qattn_call(max_queries=0, **none)
    attn_call(batch=0, **none)
    attn_call(queries=0, **none)


def test_cache_sizes():
    for heads, dim, group, page, pages in ((1, 64, 64, 16, 1), (8, 128, 32, 64, 1000), (3, 256, 128, 256, 7), (2, 128, 64, 32, 0)):
        want = pages * heads * page * 2 * (dim // 2 + 2 * (dim // group))
        assert aqd.qcache_bytes(aqd.QcacheDesc(heads, dim, group, page, pages)) == want


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("batch", [1, 3, 64, 300])
def test_the_workspaces_have_a_bound(batch, dim):
    for q_heads in (8, 64):
        for each in (1, 4, 200):
            for keys in (0, 1, 100, 5000, 131072, 1 << 24):
                cache = aqd.QcacheDesc(8, dim, 32, 16, 1000)
                b = aqd.qattn_workspace(cache, batch, q_heads, batch * each, each, keys, aqd.F16)
                assert 0 <= b <= aqd.ATTN_WORKSPACE_BYTES
                b = aqd.attn_workspace(batch, q_heads, 8, dim, batch * each, min(batch * keys, 1 << 30), each, keys, True, aqd.F16)
                assert 0 <= b <= aqd.ATTN_WORKSPACE_BYTES


def test_keys_far_from_one_another_are_not_there():
    """Offsets within a tile of 32 keys are 32-bit numbers."""
    far = (1 << 26) + 2
    refused(attn_call, aqd.AQD_ERR_UNSUPPORTED, k_token=far, k=1 << 40)
    refused(attn_call, aqd.AQD_ERR_UNSUPPORTED, v_token=far, v=1 << 40)
    # one key has no stride
    attn_call(keys=1, k_token=far, v_token=far, max_queries=0)


@pytest.mark.parametrize("sizes", [
    dict(batch=1 << 20, max_queries=65, heads=4), dict(batch=1 << 23, max_queries=1, heads=1), dict(queries=1 << 28, max_queries=1 << 28, batch=2, heads=4),
    dict(batch=1, queries=1 << 29, max_queries=1 << 29),
])
def test_launches_have_a_bound(sizes):
    """A workgroup has 128 rows (16 of single tokens), and a launch less than 2^32 threads of 256 a workgroup."""
    few = dict(queries=sizes.get("queries", 70))
    refused(attn_call, y_token=256, y=1 << 44, **{**few, **sizes})
    refused(qattn_call, y=1 << 44, q_start=ADDR["q_start"], **{**few, **sizes})


def test_long_sequences_have_a_workspace():
    """The sizes that qattn_run splits by: a row's dim sums and two more numbers for each part."""
    cache = aqd.QcacheDesc(2, 128, 64, 64, 200)
    row = 6 * (128 + 2) * 4
    for queries, keys in ((1, 9000), (4, 9000), (1, 600)):
        b = aqd.qattn_workspace(cache, 1, 6, queries, queries, keys, aqd.BF16)
        assert b and b % (row * queries) == 0 and b <= -(-keys // 128) * row * queries
    assert aqd.qattn_workspace(cache, 1, 6, 1, 1, 100, aqd.BF16) == 0
    assert aqd.attn_workspace(1, 6, 2, 128, 4, 9000, 4, 9000, True, aqd.BF16) % (row * 4) == 0


@pytest.mark.parametrize("batch", [9, 64, 700, 1024, 1025])
def test_shared_workspaces_have_a_bound(batch):
    for heads, per, each in ((1, 1, 1), (8, 8, 1), (8, 4, 500), (64, 1, 20000), (2, 32, 7)):
        for keys in (600, 5000, 131072, 1 << 24, 1 << 30):
            if batch * heads * (each * per / 16 + 1) <= 1 << 23:
                b = aqd.qattn_workspace(aqd.QcacheDesc(heads, 128, 32, 16, 1000), batch, heads * per, batch * each, each, keys, aqd.F16)
                assert 0 <= b <= aqd.ATTN_WORKSPACE_BYTES
