"""Calls of the serving operators that are refused on the host, before anything is enqueued (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2607_21042_b200 import binding as B

P = 1 << 20       # an address that is never followed: aligned, not null


@pytest.fixture(scope="module")
def lib():
    from paper_2607_21042_b200 import build
    build.build()
    return B.load()


def _tables(**kw):
    a = dict(n=4, ids=P, new=P, streams=8, ctx=P, ctx_out=P, n_pages=10, free=P, top=P, top_out=P, n_shared=2, shared=P, pps=4, table=P, rows=16,
             start=P, rs=P, rp=P, sl=P, info=P, stream=0)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


@pytest.mark.parametrize("code,kw", [
    (B.E_ARG, dict(n=0)), (B.E_ARG, dict(new=0)), (B.E_ARG, dict(ctx=0)), (B.E_ARG, dict(ctx_out=0)), (B.E_ARG, dict(free=0)), (B.E_ARG, dict(top=0)),
    (B.E_ARG, dict(top_out=0)), (B.E_ARG, dict(shared=0)), (B.E_ARG, dict(table=0)), (B.E_ARG, dict(start=0)), (B.E_ARG, dict(rs=0)), (B.E_ARG, dict(rp=0)),
    (B.E_ARG, dict(sl=0)), (B.E_ARG, dict(info=0)), (B.E_ARG, dict(info=P + 2)), (B.E_ARG, dict(ids=P + 1)), (B.E_ARG, dict(streams=0)),
    (B.E_ARG, dict(ids=0, n=9)), (B.E_ARG, dict(n_pages=0)), (B.E_ARG, dict(n_pages=2 ** 26)), (B.E_ARG, dict(rows=0)), (B.E_ARG, dict(n_shared=-1)),
    (B.E_ARG, dict(n_shared=5)), (B.E_ARG, dict(pps=0)), (B.E_UNSUPPORTED, dict(n=4097)), (B.E_UNSUPPORTED, dict(streams=32769)), (B.E_UNSUPPORTED, dict(pps=32769)),
])
def test_page_tables(lib, code, kw):
    assert lib.tts_gpt_op_page_tables(*_tables(**kw)) == code
    assert b"op_page_tables" in lib.tts_gpt_last_error(None)


def _append(**kw):
    a = dict(R=4, heads=2, type=B.T_F32, k=P, ks=128, v=P, vs=384, slot=P, fmt=0, pages=3, pool=P, stream=0)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


@pytest.mark.parametrize("code,kw", [
    (B.E_ARG, dict(R=0)), (B.E_ARG, dict(heads=0)), (B.E_ARG, dict(type=B.T_F16)), (B.E_ARG, dict(type=7)), (B.E_ARG, dict(k=0)), (B.E_ARG, dict(v=0)),
    (B.E_ARG, dict(slot=0)), (B.E_ARG, dict(pool=0)), (B.E_ARG, dict(fmt=2)), (B.E_ARG, dict(pages=0)), (B.E_ARG, dict(pages=2 ** 26)), (B.E_ARG, dict(ks=127)),
    (B.E_ARG, dict(vs=64)), (B.E_ARG, dict(ks=130)), (B.E_ARG, dict(type=B.T_BF16, ks=132)), (B.E_ARG, dict(k=P + 8)), (B.E_ARG, dict(pool=P + 4)),
    (B.E_ARG, dict(slot=P + 2)), (B.E_UNSUPPORTED, dict(R=2 ** 30, heads=4, ks=256)),
])
def test_kv_append(lib, code, kw):
    assert lib.tts_gpt_op_kv_append(*_append(**kw)) == code
    assert b"op_kv_append" in lib.tts_gpt_last_error(None)


def _shared(**kw):
    a = dict(R=4, heads=4, kv=2, type=B.T_F32, q=P, qs=256, fmt=0, pages=9, pool=P, n_shared=2, table=P, pps=4, rs=P, rp=P, out=P, scratch=P, size=1 << 30, stream=0)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


@pytest.mark.parametrize("code,kw", [
    (B.E_ARG, dict(R=0)), (B.E_ARG, dict(heads=0)), (B.E_ARG, dict(kv=0)), (B.E_ARG, dict(kv=3)), (B.E_UNSUPPORTED, dict(heads=34, qs=34 * 64)),
    (B.E_UNSUPPORTED, dict(R=4097)), (B.E_UNSUPPORTED, dict(heads=1040, kv=65, qs=1040 * 64)), (B.E_ARG, dict(type=B.T_F16)), (B.E_ARG, dict(q=0)), (B.E_ARG, dict(pool=0)),
    (B.E_ARG, dict(table=0)), (B.E_ARG, dict(rs=0)), (B.E_ARG, dict(rp=0)), (B.E_ARG, dict(out=0)), (B.E_ARG, dict(scratch=0)), (B.E_ARG, dict(fmt=3)), (B.E_ARG, dict(pages=0)),
    (B.E_ARG, dict(n_shared=-1)), (B.E_ARG, dict(n_shared=5)), (B.E_ARG, dict(pps=0)), (B.E_ARG, dict(qs=255)), (B.E_ARG, dict(qs=258)), (B.E_ARG, dict(q=P + 8)),
    (B.E_ARG, dict(out=P + 2)), (B.E_ARG, dict(scratch=P + 128)), (B.E_ARG, dict(table=P + 2)), (B.E_UNSUPPORTED, dict(pages=2 ** 30)), (B.E_UNSUPPORTED, dict(pps=2 ** 25)),
    (B.E_UNSUPPORTED, dict(R=4096, pps=2 ** 20)), (B.E_WORKSPACE, dict(size=4096)),
])
def test_attention_shared(lib, code, kw):
    assert lib.tts_gpt_op_attention_shared(*_shared(**kw)) == code
    assert b"op_attention_shared" in lib.tts_gpt_last_error(None)


def _cross(**kw):
    a = dict(n=3, heads=4, kv=2, type=B.T_BF16, qr=9, q=P, qs=256, kr=50, k=P, ks=128, kh=64, v=P, vs=128, vh=64, q0=P, k0=P, q_max=4, scale=0.125, out=P,
             scratch=P, size=1 << 30, stream=0)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


@pytest.mark.parametrize("code,kw", [
    (B.E_ARG, dict(n=0)), (B.E_ARG, dict(heads=3)), (B.E_UNSUPPORTED, dict(heads=34, qs=34 * 64)), (B.E_ARG, dict(type=B.T_F32)), (B.E_ARG, dict(qr=0)), (B.E_ARG, dict(q=0)),
    (B.E_ARG, dict(k=0)), (B.E_ARG, dict(v=0)), (B.E_ARG, dict(kr=-1)), (B.E_ARG, dict(q0=0)), (B.E_ARG, dict(k0=0)), (B.E_ARG, dict(q_max=0)), (B.E_ARG, dict(out=0)),
    (B.E_ARG, dict(scale=0.0)), (B.E_ARG, dict(scale=-1.0)), (B.E_ARG, dict(scale=float("nan"))), (B.E_ARG, dict(scale=float("inf"))), (B.E_ARG, dict(qs=248)),
    (B.E_ARG, dict(qs=260)), (B.E_ARG, dict(ks=132)), (B.E_ARG, dict(kh=32)), (B.E_ARG, dict(vh=68)), (B.E_ARG, dict(vs=8)), (B.E_ARG, dict(k=P + 8)),
    (B.E_ARG, dict(scratch=P + 16)), (B.E_ARG, dict(scratch=0)), (B.E_UNSUPPORTED, dict(n=4097)), (B.E_WORKSPACE, dict(size=1 << 20)),
    (B.E_UNSUPPORTED, dict(qr=2 ** 24, q_max=2 ** 24, kr=2 ** 20)), (B.E_UNSUPPORTED, dict(qr=2 ** 30)), (B.E_UNSUPPORTED, dict(kr=2 ** 30)), (B.E_UNSUPPORTED, dict(n=1, heads=1, kv=1, qr=2 ** 22, q_max=2 ** 22, kr=2 ** 23)),
])
def test_attention_cross(lib, code, kw):
    assert lib.tts_gpt_op_attention_cross(*_cross(**kw)) == code
    assert b"op_attention_cross" in lib.tts_gpt_last_error(None)


def test_outputs_that_overlap_what_is_read(lib):
    """Addresses 1 MB apart are refused for nothing but an overlap, and with one only for that."""
    def refused(fn, args):
        return fn(*args) == B.E_ARG and b"overlap" in lib.tts_gpt_last_error(None)

    apart = {name: (i + 1) << 20 for i, name in enumerate(["ids", "new", "ctx", "ctx_out", "free", "top", "top_out", "shared", "table", "start", "rs", "rp", "sl", "info"])}
    for a, b in [("rs", "ids"), ("start", "new"), ("ctx_out", "new"), ("info", "top"), ("table", "free"), ("rp", "rs"), ("sl", "shared"), ("top_out", "ctx"), ("info", "start")]:
        assert refused(lib.tts_gpt_op_page_tables, _tables(**{**apart, a: apart[b]})), (a, b)
    assert refused(lib.tts_gpt_op_page_tables, _tables(**{**apart, "top": apart["info"] + 12}))            # the height that a call reports, as the next call's
    assert refused(lib.tts_gpt_op_page_tables, _tables(**{**apart, "ctx_out": apart["ctx"] + 4}))
    assert refused(lib.tts_gpt_op_page_tables, _tables(**{**apart, "rs": apart["rp"] - 60}))                # the last of 16 rows
    Q = P + (1 << 24)
    assert refused(lib.tts_gpt_op_attention_shared, _shared(q=Q, out=Q))
    assert refused(lib.tts_gpt_op_attention_shared, _shared(q=Q, out=Q + 4 * 1024 - 16))
    assert refused(lib.tts_gpt_op_attention_shared, _shared(q=Q, out=Q - 4 * 512 + 16))
    for name in ("q", "k", "v"):
        far = dict(q=P + (1 << 24), k=P + (2 << 24), v=P + (3 << 24))
        assert refused(lib.tts_gpt_op_attention_cross, _cross(**far, out=far[name])), name
        assert refused(lib.tts_gpt_op_attention_cross, _cross(**far, out=far[name] - 9 * 512 + 16)), name


def test_scratch_sizes(lib):
    n, m = C.c_size_t(0), C.c_size_t(0)
    assert lib.tts_gpt_op_attention_shared_scratch_bytes(C.c_int32(1), C.c_int32(4), C.c_int32(4), C.byref(n)) == B.OK
    assert lib.tts_gpt_op_attention_shared_scratch_bytes(C.c_int32(4096), C.c_int32(4), C.c_int32(4), C.byref(m)) == B.OK
    assert 0 < n.value < m.value
    assert lib.tts_gpt_op_attention_shared_scratch_bytes(C.c_int32(0), C.c_int32(4), C.c_int32(4), C.byref(n)) == B.E_ARG
    assert lib.tts_gpt_op_attention_shared_scratch_bytes(C.c_int32(1), C.c_int32(5), C.c_int32(4), C.byref(n)) == B.E_ARG
    assert lib.tts_gpt_op_attention_shared_scratch_bytes(C.c_int32(1), C.c_int32(4), C.c_int32(4), None) == B.E_ARG
    assert lib.tts_gpt_op_attention_cross_scratch_bytes(C.byref(n)) == B.OK and n.value > 0
    assert lib.tts_gpt_op_attention_cross_scratch_bytes(None) == B.E_ARG


def test_the_binding_checks_its_tensors(lib):
    i = torch.zeros(8, dtype=torch.int32)
    pool = torch.zeros(2, 2, 4, 64, 64, dtype=torch.bfloat16)
    q = torch.zeros(3, 256)
    refused = [
        lambda: B.op_attention_shared(q, pool[:, :, :2], torch.zeros(3, 4, dtype=torch.int32), i, i, 1),          # a pool that is not contiguous
        lambda: B.op_attention_shared(q, pool.float(), torch.zeros(3, 4, dtype=torch.int32), i, i, 1),
        lambda: B.op_attention_shared(q.half(), pool, torch.zeros(3, 4, dtype=torch.int32), i, i, 1),
        lambda: B.op_attention_shared(q[:, ::2], pool, torch.zeros(3, 4, dtype=torch.int32), i, i, 1),
        lambda: B.op_attention_shared(q, pool, i, i, i, 1),
        lambda: B.op_attention_shared(q, pool, torch.zeros(3, 4, dtype=torch.int64), i, i, 1),
        lambda: B.op_attention_shared(q, pool, torch.zeros(3, 4, dtype=torch.int32), i[:2], i, 1),
        lambda: B.op_attention_shared(q, pool, torch.zeros(3, 4, dtype=torch.int32), i, i, 1, out=torch.zeros(3, 256)),
        lambda: B.op_kv_append(q, q[:2], pool, i),
        lambda: B.op_kv_append(q, q.bfloat16(), pool, i),
        lambda: B.op_kv_append(q, q, pool, i[:2]),
        lambda: B.op_kv_append(q[:, :128], q[:, :128], pool, i),
        lambda: B.op_page_tables(i, i, i, i, i, i, i, i, i, i),
        lambda: B.op_page_tables(i, i, torch.zeros(8, 4, dtype=torch.int32), i, i, i, i, i, i, i),                # row_start too short
        lambda: B.op_page_tables(i[:4], i, torch.zeros(8, 4, dtype=torch.int32), i, i, i, i, i[:7], i, i),
        lambda: B.op_attention_cross(q.view(3, 4, 64), q.view(3, 4, 64), q.view(3, 4, 64), i[:2], i[:2], 3),      # fp32
        lambda: B.op_attention_cross(q.half().view(3, 4, 64), q.half().view(3, 4, 64), q.view(3, 4, 64).bfloat16(), i[:2], i[:2], 3),
        lambda: B.op_attention_cross(q.half().view(3, 4, 64), q.half().view(3, 4, 64), q.half().view(3, 4, 64), i[:2], i[:3], 3),
        lambda: B.op_attention_cross(q.half().view(3, 4, 64), q.half().view(3, 4, 64), q.half().view(3, 4, 64), i[:1], i[:1], 3),
    ]
    for call in refused:
        with pytest.raises(B.TtsGptError) as e:
            call()
        assert e.value.code == B.E_ARG
    # and everything in order but on the CPU
    with pytest.raises(B.TtsGptError) as e:
        B.op_kv_append(q, q, pool, i)
    assert e.value.code == B.E_ARG and "CUDA" in str(e.value)
