"""The draft operators on the host: calls that are refused before anything is enqueued, and the table of rotary frequencies (no GPU needed)."""
import ctypes as C
import math
from fractions import Fraction

import pytest
import torch

from paper_2607_21042_b200 import binding as B

M = 1 << 20
ADDR = {name: (i + 1) << 32 for i, name in enumerate(
    "q k v pos slot turns qo pool start ids kv parent mask info table out scratch draft target kvo free top topo path acc nxt".split())}   # far apart, never followed


@pytest.fixture(scope="module")
def lib():
    from paper_2607_21042_b200 import build
    build.build()
    return B.load()


def _call(defaults, kw):
    assert set(kw) <= set(defaults)
    a = {**defaults, **kw}
    # an address is given by name, or as (name, offset)
    return [ADDR[x] if isinstance(x, str) else ADDR[x[0]] + x[1] if isinstance(x, tuple) else x for x in a.values()]


ROPE = dict(R=4, heads=4, kv=2, type=B.T_F32, q="q", qs=256, k="k", ks=128, v="v", vs=384, pos="pos", slot="slot", n_rot=64, turns="turns", inter=0, mag=1.0, ot=B.T_BF16, qo="qo", os=256,
            fmt=0, pages=3, pool="pool", stream=0)
TABLES = dict(n=4, R=16, start="start", ids="ids", streams=8, kv="kv", parent="parent", words=1, mask="mask", pos="pos", info="info", stream=0)
TREE = dict(n=3, R=16, heads=4, kv=2, type=B.T_BF16, q="q", qs=256, fmt=0, pages=9, pool="pool", streams=8, table="table", pps=4, start="start", ids="ids", len="kv", words=1, mask="mask",
            t_max=8, scale=0.125, out="out", scratch="scratch", size=1 << 30, stream=0)
ACCEPT = dict(n=4, R=16, start="start", ids="ids", draft="draft", target="target", parent="parent", streams=8, kv="kv", kvo="kvo", table="table", pps=4, n_pages=10, free="free", top="top",
              topo="topo", path="path", acc="acc", nxt="nxt", info="info", stream=0)
MOVE = dict(n=4, R=16, start="start", path="path", slot="slot", heads=2, fmt=0, pages=3, layers=2, apart=3 * 4 * 8192, pool="pool", stream=0)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("code,kw", [
    (B.E_ARG, dict(R=0)), (B.E_ARG, dict(heads=-1)), (B.E_ARG, dict(kv=0)), (B.E_ARG, dict(type=B.T_F16)), (B.E_ARG, dict(ot=B.T_F16)), (B.E_ARG, dict(q=0)), (B.E_ARG, dict(qo=0)),
    (B.E_ARG, dict(k=0)), (B.E_ARG, dict(v=0)), (B.E_ARG, dict(pos=0)), (B.E_ARG, dict(slot=0)), (B.E_ARG, dict(turns=0)), (B.E_ARG, dict(pool=0)), (B.E_ARG, dict(fmt=2)),
    (B.E_ARG, dict(pages=0)), (B.E_ARG, dict(pages=2 ** 26)), (B.E_ARG, dict(qs=252)), (B.E_ARG, dict(os=255)), (B.E_ARG, dict(ks=124)), (B.E_ARG, dict(vs=64)), (B.E_ARG, dict(ks=130)),
    (B.E_ARG, dict(qs=258)), (B.E_ARG, dict(os=260)), (B.E_ARG, dict(type=B.T_BF16, qs=260)), (B.E_ARG, dict(n_rot=0)), (B.E_ARG, dict(n_rot=66)), (B.E_ARG, dict(n_rot=31)),
    (B.E_ARG, dict(mag=NAN)), (B.E_ARG, dict(mag=INF)), (B.E_ARG, dict(q=("q", 8))), (B.E_ARG, dict(k=("k", 4))), (B.E_ARG, dict(v=("v", 2))), (B.E_ARG, dict(qo=("qo", 8))),
    (B.E_ARG, dict(pool=("pool", 8))), (B.E_ARG, dict(turns=("turns", 4))), (B.E_ARG, dict(pos=("pos", 2))), (B.E_ARG, dict(slot=("slot", 1))),
    (B.E_UNSUPPORTED, dict(heads=4097, qs=1 << 20, os=1 << 20)), (B.E_UNSUPPORTED, dict(kv=4097, ks=1 << 20, vs=1 << 20))])
def test_rope_kv_append(lib, code, kw):
    assert lib.tts_gpt_op_rope_kv_append(*_call(ROPE, kw)) == code
    assert b"op_rope_kv_append" in lib.tts_gpt_last_error(None)


@pytest.mark.parametrize("code,kw", [
    (B.E_ARG, dict(n=0)), (B.E_ARG, dict(R=0)), (B.E_ARG, dict(start=0)), (B.E_ARG, dict(kv=0)), (B.E_ARG, dict(parent=0)), (B.E_ARG, dict(mask=0)), (B.E_ARG, dict(pos=0)),
    (B.E_ARG, dict(info=0)), (B.E_ARG, dict(streams=0)), (B.E_ARG, dict(ids=0, n=9)), (B.E_ARG, dict(words=0)), (B.E_ARG, dict(mask=("mask", 2))), (B.E_ARG, dict(ids=("ids", 1))),
    (B.E_UNSUPPORTED, dict(n=4097)), (B.E_UNSUPPORTED, dict(words=9)), (B.E_UNSUPPORTED, dict(streams=32769))])
def test_tree_tables(lib, code, kw):
    assert lib.tts_gpt_op_tree_tables(*_call(TABLES, kw)) == code
    assert b"op_tree_tables" in lib.tts_gpt_last_error(None)


@pytest.mark.parametrize("code,kw", [
    (B.E_ARG, dict(n=0)), (B.E_ARG, dict(R=0)), (B.E_ARG, dict(heads=0)), (B.E_ARG, dict(heads=3)), (B.E_ARG, dict(kv=0)), (B.E_ARG, dict(type=B.T_F16)), (B.E_ARG, dict(q=0)),
    (B.E_ARG, dict(pool=0)), (B.E_ARG, dict(table=0)), (B.E_ARG, dict(start=0)), (B.E_ARG, dict(len=0)), (B.E_ARG, dict(mask=0)), (B.E_ARG, dict(out=0)), (B.E_ARG, dict(scratch=0)),
    (B.E_ARG, dict(fmt=-1)), (B.E_ARG, dict(pages=0)), (B.E_ARG, dict(streams=0)), (B.E_ARG, dict(ids=0, n=9)), (B.E_ARG, dict(pps=0)), (B.E_ARG, dict(words=0)), (B.E_ARG, dict(t_max=0)),
    (B.E_ARG, dict(qs=248)), (B.E_ARG, dict(qs=260)), (B.E_ARG, dict(type=B.T_F32, qs=258)), (B.E_ARG, dict(scale=0.0)), (B.E_ARG, dict(scale=-1.0)), (B.E_ARG, dict(scale=NAN)),
    (B.E_ARG, dict(scale=INF)), (B.E_ARG, dict(q=("q", 8))), (B.E_ARG, dict(out=("out", 8))), (B.E_ARG, dict(pool=("pool", 8))), (B.E_ARG, dict(scratch=("scratch", 128))),
    (B.E_ARG, dict(mask=("mask", 2))), (B.E_UNSUPPORTED, dict(heads=34, qs=34 * 64)), (B.E_UNSUPPORTED, dict(heads=1040, kv=65, qs=1040 * 64)), (B.E_UNSUPPORTED, dict(n=2049)),
    (B.E_UNSUPPORTED, dict(words=33)), (B.E_UNSUPPORTED, dict(pps=2 ** 25)), (B.E_UNSUPPORTED, dict(pages=2 ** 30)), (B.E_UNSUPPORTED, dict(R=2 ** 28)),
    (B.E_UNSUPPORTED, dict(R=2 ** 20, pps=2 ** 14)), (B.E_WORKSPACE, dict(size=4096))])
def test_attention_tree(lib, code, kw):
    assert lib.tts_gpt_op_attention_tree(*_call(TREE, kw)) == code
    assert b"op_attention_tree" in lib.tts_gpt_last_error(None)


@pytest.mark.parametrize("code,kw", [(B.E_ARG, {k: 0}) for k in ("n", "R", "start", "draft", "target", "parent", "streams", "kv", "kvo", "table", "pps", "n_pages", "free", "top", "topo",
                                                                "path", "acc", "nxt", "info")] + [
    (B.E_ARG, dict(ids=0, n=9)), (B.E_ARG, dict(n_pages=2 ** 26)), (B.E_ARG, dict(path=("path", 2))), (B.E_ARG, dict(info=("info", 1))), (B.E_UNSUPPORTED, dict(n=4097)),
    (B.E_UNSUPPORTED, dict(streams=32769)), (B.E_UNSUPPORTED, dict(pps=32769))])
def test_tree_accept(lib, code, kw):
    assert lib.tts_gpt_op_tree_accept(*_call(ACCEPT, kw)) == code
    assert b"op_tree_accept" in lib.tts_gpt_last_error(None)


@pytest.mark.parametrize("code,kw", [(B.E_ARG, {k: 0}) for k in ("n", "R", "start", "path", "slot", "heads", "pages", "layers", "pool")] + [
    (B.E_ARG, dict(fmt=2)), (B.E_ARG, dict(pages=2 ** 26)), (B.E_ARG, dict(apart=3 * 4 * 8192 - 16)), (B.E_ARG, dict(apart=3 * 4 * 8192 + 8)), (B.E_ARG, dict(pool=("pool", 8))),
    (B.E_ARG, dict(path=("path", 2))), (B.E_UNSUPPORTED, dict(n=2 ** 20 + 1)), (B.E_UNSUPPORTED, dict(layers=65536)), (B.E_UNSUPPORTED, dict(heads=4097, apart=1 << 40))])
def test_kv_move(lib, code, kw):
    assert lib.tts_gpt_op_kv_move(*_call(MOVE, kw)) == code
    assert b"op_kv_move" in lib.tts_gpt_last_error(None)


def test_overlaps(lib):
    """Nothing but the overlap is wrong: its first and its last byte."""
    def refused(fn, defaults, kw):
        return fn(*_call(defaults, kw)) == B.E_ARG and b"overlap" in lib.tts_gpt_last_error(None)

    rope, tables, tree, accept, move = (getattr(lib, "tts_gpt_op_" + n) for n in ("rope_kv_append", "tree_tables", "attention_tree", "tree_accept", "kv_move"))
    pool = 3 * 4 * 8192
    for name, n in (("q", 4 * 1024), ("k", 3 * 512 + 512), ("v", 3 * 1536 + 512), ("pos", 16), ("slot", 16), ("turns", 256), ("qo", 4 * 512)):
        step = 16 if name in ("q", "k", "v", "qo", "turns") else 4
        assert refused(rope, ROPE, {name: ("pool", pool - step)}) and refused(rope, ROPE, {name: ("pool", step - n)}), name
    for name, n in (("q", 4 * 1024), ("k", 3 * 512 + 512), ("v", 3 * 1536 + 512), ("pos", 16), ("slot", 16), ("turns", 256)):
        step = 4 if name in ("pos", "slot") else 16
        assert refused(rope, ROPE, {name: ("qo", 4 * 512 - step)}) and refused(rope, ROPE, {name: ("qo", step - n)}), name
    assert refused(rope, ROPE, dict(qo="q"))                                       # another type than q's
    assert refused(rope, ROPE, dict(qo="q", ot=B.T_F32, os=512))                   # another stride
    assert refused(rope, ROPE, dict(qo=("q", 16), ot=B.T_F32))
    for name in ("start", "ids", "kv", "parent"):
        for out in ("mask", "pos", "info"):
            assert refused(tables, TABLES, {name: out}), (name, out)
    assert refused(tables, TABLES, dict(mask=("pos", 60))) and refused(tables, TABLES, dict(info=("mask", 60)))
    for name in ("q", "pool", "table", "start", "ids", "len", "mask"):
        assert refused(tree, TREE, {name: ("out", 16 * 512 - 16)}) and refused(tree, TREE, {name: "scratch"}), name
    assert refused(tree, TREE, dict(out=("scratch", 1024)))
    for name in ("start", "ids", "draft", "target", "parent", "kv", "table", "top"):
        for out in ("kvo", "topo", "free", "path", "acc", "nxt", "info"):
            if (name, out) not in (("kv", "kvo"), ("top", "topo")):
                assert refused(accept, ACCEPT, {name: out}), (name, out)
    assert refused(accept, ACCEPT, dict(kvo=("kv", 4))) and refused(accept, ACCEPT, dict(acc=("nxt", 12))) and refused(accept, ACCEPT, dict(top=("info", 12)))
    for name in ("start", "path", "slot"):
        assert refused(move, MOVE, {name: ("pool", 2 * pool - 4)}), name


def test_scratch_size(lib):
    n, other = C.c_size_t(0), C.c_size_t(0)
    assert lib.tts_gpt_op_attention_tree_scratch_bytes(C.byref(n)) == B.OK and n.value > 0
    assert lib.tts_gpt_op_attention_tree_scratch_bytes(None) == B.E_ARG
    assert lib.tts_gpt_op_attention_tree(*_call(TREE, dict(size=n.value - 1))) == B.E_WORKSPACE


def test_the_binding_checks_its_tensors(lib):
    def i(*shape):
        return torch.zeros(shape or (8,), dtype=torch.int32)

    pool, bytes_ = torch.zeros(2, 2, 4, 64, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 2, 4, 4352, dtype=torch.uint8)
    x, table, turns = torch.zeros(3, 256), i(8, 4), torch.zeros(32, dtype=torch.int64)
    start, mask = i(4), i(3, 1)
    refused = [
        lambda: B.op_rope_kv_append(x, x, x, pool, i(2), i(3), turns), lambda: B.op_rope_kv_append(x, x, x, pool, i(3), i(2), turns),
        lambda: B.op_rope_kv_append(x, x, x.bfloat16(), pool, i(), i(), turns), lambda: B.op_rope_kv_append(x.bfloat16(), x, x, pool, i(), i(), turns),
        lambda: B.op_rope_kv_append(x, x, x, pool, i(), i(), turns.double()), lambda: B.op_rope_kv_append(x[:2], x, x, pool, i(), i(), turns),
        lambda: B.op_rope_kv_append(x[:, :100], x, x, pool, i(), i(), turns), lambda: B.op_rope_kv_append(x, x[:, :128], x, pool, i(), i(), turns),
        lambda: B.op_rope_kv_append(x, x, x, pool, i(), i(), turns, q_out=x.half()), lambda: B.op_rope_kv_append(x, x, x, pool, i(), i(), turns, q_out=x[:2]),
        lambda: B.op_rope_kv_append(None, x, x, pool, i(), i(), turns, q_out=x), lambda: B.op_rope_kv_append(x, x, x, pool[:, :, :2], i(), i(), turns),
        lambda: B.op_rope_kv_append(torch.zeros(3, 512)[:, ::2], x, x, pool, i(), i(), turns), lambda: B.op_rope_kv_append(x, x, x, bytes_[:, :, :, :, 0], i(), i(), turns),
        lambda: B.op_rope_kv_append(x.half(), x.half(), x.half(), pool, i(), i(), turns),
        lambda: B.op_tree_tables(i(3), start, i(), mask, i(4), i()), lambda: B.op_tree_tables(i(3), start, i(), i(4, 1), i(3), i()), lambda: B.op_tree_tables(i(3), start, i(), i(3), i(3), i()),
        lambda: B.op_tree_tables(i(3), i(1), i(), mask, i(3), i()), lambda: B.op_tree_tables(i(3), start, i(), mask, i(3), i(), stream_ids=i(2)),
        lambda: B.op_tree_tables(i(3).long(), start, i(), mask, i(3), i()), lambda: B.op_tree_tables(i(6)[::2], start, i(), mask, i(3), i()),
        lambda: B.op_attention_tree(x.half(), pool, table, start, i(), mask, 3), lambda: B.op_attention_tree(x[:, :100], pool, table, start, i(), mask, 3),
        lambda: B.op_attention_tree(x, pool, i(7, 4), start, i(), mask, 3), lambda: B.op_attention_tree(x, pool, table, start, i(), mask[:2], 3),
        lambda: B.op_attention_tree(x, pool, table, start, i(), mask[:, 0], 3), lambda: B.op_attention_tree(x, pool, table, start, i(), mask, 3, out=x),
        lambda: B.op_attention_tree(x, pool, table, start, i(), mask, 3, stream_ids=i(4), out=x.bfloat16()), lambda: B.op_attention_tree(x, pool.float(), table, start, i(), mask, 3),
        lambda: B.op_attention_tree(x, pool, table, start, i(), mask, 3, out=x.bfloat16(), scratch=i(100)),
        lambda: B.op_tree_accept(i(3), i(2), i(3), start, i(), table, i(), i(1), i(3), i(3), i(3), i()), lambda: B.op_tree_accept(i(3), i(3), i(3), start, i(), i(7, 4), i(), i(1), i(3), i(3), i(3), i()),
        lambda: B.op_tree_accept(i(3), i(3), i(3), start, i(), table, i(), i(1), i(3), i(2), i(3), i()), lambda: B.op_tree_accept(i(3), i(3), i(3), start, i(), table, i(), i(1), i(3), i(3), i(3), i(7)),
        lambda: B.op_tree_accept(i(3), i(3), i(3), start, i(), table, i(), i(1), i(4), i(3), i(3), i()), lambda: B.op_tree_accept(i(3), i(3), i(3), start, i(), table, i(), i(0), i(3), i(3), i(3), i()),
        lambda: B.op_tree_accept(i(3), i(3), i(3), start, i(), table, i(), i(1), i(3), i(3), i(3), i(), kv_len_out=i(7)),
        lambda: B.op_kv_move(bytes_, start, i(3), i(2)), lambda: B.op_kv_move(bytes_[:0], start, i(3), i(3)), lambda: B.op_kv_move(bytes_[:, :, :, :3], start, i(3), i(3)),
        lambda: B.op_kv_move(bytes_[..., :4096], start, i(3), i(3)), lambda: B.op_kv_move(bytes_, i(1), i(3), i(3)), lambda: B.op_kv_move(pool.float(), start, i(3), i(3)),
        lambda: B.op_kv_move(pool.unsqueeze(0).float(), start, i(3), i(3)),
    ]
    for k, call in enumerate(refused):
        with pytest.raises(B.TtsGptError) as e:
            call()
        assert e.value.code == B.E_ARG and "CUDA" not in str(e.value), k
    fine = [                                   # and everything in order but on the CPU
        lambda: B.op_rope_kv_append(x, x, x, pool, i(), i(), turns, q_out=x), lambda: B.op_tree_tables(i(3), start, i(), mask, i(3), i()),
        lambda: B.op_attention_tree(x, pool, table, start, i(), mask, 3, out=x.bfloat16(), scratch=torch.zeros(256, dtype=torch.uint8)),
        lambda: B.op_tree_accept(i(3), i(3), i(3), start, i(), table, i(), i(1), i(3), i(3), i(3), i()),
        lambda: B.op_kv_move(bytes_, start, i(3), i(3)), lambda: B.op_kv_move(bytes_[::2], start, i(3), i(3)), lambda: B.op_kv_move(bytes_[0], start, i(3), i(3)),
        lambda: B.op_kv_move(pool, start, i(3), i(3)), lambda: B.op_kv_move(pool.expand(3, -1, -1, -1, -1, -1)[:1], start, i(3), i(3))]
    for call in fine:
        with pytest.raises(B.TtsGptError) as e:
            call()
        assert e.value.code == B.E_ARG and "CUDA" in str(e.value)


# ---------------------------------------------------------------------------------------------
# rotary frequencies
# ---------------------------------------------------------------------------------------------
PI = Fraction(3141592653589793238462643383279502884197169399375105820974944592, 10 ** 63)


def _turns(*args, **kw):
    table, mag = B.op_rope_frequencies(*args, device="cpu", **kw)
    assert table.dtype == torch.int64
    return [t % 2 ** 64 for t in table.tolist()], mag


def _near(turns, w):
    """w is off by at most 4 of its last places (two logarithms and a power here, as many there), and the product with 1 / 2 pi is rounded once more."""
    for i, (t, x) in enumerate(zip(turns, w)):
        assert abs(t - x / (2 * math.pi) * 2.0 ** 64) <= 8 * 2.0 ** -53 * x * 2.0 ** 64 / (2 * math.pi) + 1, i


@pytest.mark.parametrize("n_rot", [2, 4, 30, 64])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequencies(lib, n_rot, base):
    w = [base ** (-2 * i / n_rot) for i in range(n_rot // 2)]
    turns, mag = _turns(n_rot, base=base)
    assert mag == 1.0
    _near(turns, w)
    turns, mag = _turns(n_rot, base=base, scaling="linear", factor=4.0)
    assert mag == 1.0
    _near(turns, [x / 4.0 for x in w])
    if n_rot >= 4:
        turns, _ = _turns(n_rot, base=base, scaling="ntk", factor=8.0)
        raised = base * 8.0 ** (n_rot / (n_rot - 2))
        assert abs(turns[-1] / 2.0 ** 64 - w[-1] / 8.0 / (2 * math.pi)) <= 1e-14 * w[-1]     # the slowest is divided by the factor
        assert all(abs(t / 2.0 ** 64 - raised ** (-2 * i / n_rot) / (2 * math.pi)) <= 1e-14 * w[i] for i, t in enumerate(turns))


def test_frequencies_by_bands_and_blended(lib):
    """The table's step is 2^-64 of a turn: 2 pi 2^-64 radians, which is 1.3e-12 of the slowest frequency here, come on top of the roundings."""
    step = 2 * math.pi * 2.0 ** -64
    n_rot, base, original, factor = 64, 500000.0, 8192, 8.0
    w = [base ** (-2 * i / n_rot) for i in range(32)]
    turns, mag = _turns(n_rot, base=base, scaling="bands", factor=factor, original=original, low=1.0, high=4.0)
    want = []
    for x in w:
        rounds = original * x / (2 * math.pi)
        s = min(max((rounds - 1.0) / 3.0, 0.0), 1.0)
        want.append((1 - s) * x / factor + s * x)
    assert mag == 1.0 and want[0] == w[0] and want[-1] == w[-1] / factor
    assert all(abs(t / 2.0 ** 64 * 2 * math.pi - x) <= 1e-13 * x + step for t, x in zip(turns, want))
    turns, mag = _turns(n_rot, base=10000.0, scaling="yarn", factor=16.0, original=4096)
    w = [10000.0 ** (-2 * i / n_rot) for i in range(32)]
    pair = lambda rounds: n_rot * math.log(4096 / (rounds * 2 * math.pi)) / (2 * math.log(10000.0))  # noqa: E731
    first, last = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), n_rot - 1)
    want = []
    for i, x in enumerate(w):
        slow = min(max((i - first) / (last - first), 0.0), 1.0)
        want.append(x / 16.0 * slow + x * (1 - slow))
    assert 0 < first < last < 32 and abs(mag - (0.1 * math.log(16.0) + 1.0)) <= 2.0 ** -23
    assert all(abs(t / 2.0 ** 64 * 2 * math.pi - x) <= 1e-13 * x + step for t, x in zip(turns, want))


def test_given_frequencies_modulo_a_turn(lib):
    """Any angle: negative ones, more than a turn; the fraction is good to 2 units of 2^-64 for what is below a turn, and to the long double's 2^-64 of the turns
    beyond (three operations)."""
    given = [1.0, 0.0, -1.0, 100.0, -2.5e-5, 1e-12, 6.283185307179586, 3.0]
    turns, mag = _turns(16, inv_freq=given)
    assert mag == 1.0 and turns[1] == 0
    for t, w in zip(turns, given):
        exact = Fraction(w) / (2 * PI)
        off = (Fraction(t, 2 ** 64) - exact) % 1
        assert min(off, 1 - off) <= Fraction(2 + 3 * int(abs(exact) + 1), 2 ** 64)


@pytest.mark.parametrize("kw", [
    dict(n_rot=0), dict(n_rot=3), dict(n_rot=66), dict(n_rot=64.0), dict(scaling="other"), dict(base=1.0), dict(base=INF), dict(base=NAN), dict(scaling="linear", factor=0.5),
    dict(scaling="linear", factor=NAN), dict(scaling="ntk", factor=2.0, n_rot=2), dict(scaling="yarn", factor=2.0), dict(scaling="yarn", factor=2.0, original=100, low=4.0, high=2.0),
    dict(scaling="bands", factor=2.0, original=100, low=0.0), dict(inv_freq=[1.0] * 31), dict(inv_freq=[1.0] * 31 + [INF])])
def test_frequencies_refused(lib, kw):
    with pytest.raises(B.TtsGptError) as e:
        B.op_rope_frequencies(**{"n_rot": 64, "device": "cpu", **kw})
    assert e.value.code == B.E_ARG
