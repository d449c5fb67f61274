"""Calls of the serving operators whose outputs or scratch lie over something else that the same call uses are refused on the host (no GPU
needed): parts of the call run at the same time, so what they read would depend on timing."""
import pytest

from paper_2607_21042_b200 import binding as B
from test_serving_ops_refusals import _append, _cross, _shared, lib  # noqa: F401

MB = 1 << 20


def _refused(lib, fn, args):
    return fn(*args) == B.E_ARG and b"overlap" in lib.tts_gpt_last_error(None)


@pytest.mark.parametrize("fmt,block", [(0, 8192), (1, 4352)])
def test_rows_inside_the_pool_they_are_written_to(lib, fmt, block):
    apart = dict(k=1 * MB, v=2 * MB, slot=3 * MB, pool=4 * MB)         # 4 rows of 2 heads, 3 pages
    size, fn = 3 * 2 * 2 * block, lib.tts_gpt_op_kv_append
    for name in ("k", "v", "slot"):
        for at in (apart["pool"], apart["pool"] + size - 16):
            assert _refused(lib, fn, _append(**{**apart, "fmt": fmt, name: at})), (name, at)
    # the last of 4 rows, whose stride is 384 and whose values are 128
    assert _refused(lib, fn, _append(**{**apart, "fmt": fmt, "v": apart["pool"] - (3 * 384 + 128) * 4 + 16}))
    # next to each other: not refused for that (a call without a GPU fails later)
    for kw in ({"v": apart["pool"] - (3 * 384 + 128) * 4}, {"k": apart["pool"] + size}, {"k": apart["v"]}):
        assert not _refused(lib, fn, _append(**{**apart, "fmt": fmt, **kw})), kw


@pytest.mark.parametrize("fmt,block", [(0, 8192), (1, 4352)])
def test_shared_prefix_attention(lib, fmt, block):
    apart = {n: (i + 1) * 64 * MB for i, n in enumerate(["q", "pool", "table", "rs", "rp", "out", "scratch"])}
    fn, last = lib.tts_gpt_op_attention_shared, 9 * 2 * 2 * block - 16
    for name, at in [("pool", 0), ("pool", last), ("rs", 0), ("rp", 0), ("table", 0), ("scratch", 0), ("scratch", 2048), ("q", 0)]:
        assert _refused(lib, fn, _shared(**{**apart, "fmt": fmt, "out": apart[name] + at})), (name, at)
    for name, at in [("pool", 0), ("rs", 0), ("rp", 0), ("table", 0), ("q", 0)]:
        assert _refused(lib, fn, _shared(**{**apart, "fmt": fmt, "scratch": apart[name] + at})), (name, at)
    assert not _refused(lib, fn, _shared(**{**apart, "fmt": fmt, "out": apart["pool"] + last + 16}))


@pytest.mark.parametrize("q_max", [4, 9])
def test_cross_attention(lib, q_max):
    apart = {n: (i + 1) * 64 * MB for i, n in enumerate(["q", "k", "v", "q0", "k0", "out", "scratch"])}
    fn = lib.tts_gpt_op_attention_cross
    for name in ("q", "k", "v", "q0", "k0", "scratch"):
        assert _refused(lib, fn, _cross(**{**apart, "q_max": q_max, "out": apart[name]})), name
        if name != "scratch":
            assert _refused(lib, fn, _cross(**{**apart, "q_max": q_max, "scratch": apart[name]})), name
    assert _refused(lib, fn, _cross(**{**apart, "q0": apart["out"] + 9 * 256 * 2 - 16}))
    assert not _refused(lib, fn, _cross(**{**apart, "q0": apart["out"] + 9 * 256 * 2}))
