"""The operators of a program that assembles its own step over a paged cache, each against its formula in 64 bits: page lists
and slot maps, K/V rows into their slots, attention of a batch that shares a prefix, attention to an encoder's states.

Tolerances of the attentions.  With p_j the softmax weights, o = sum p_j v_j and A = sum p_j |v_j| (all exact), what the
kernels round is: each weight to the 16-bit type (relative half step h: 2^-8 bf16, 2^-11 fp16), which moves o by at most h A;
the output, by at most h (|o| + h A); fp32 queries to 16 bits (two bf16 parts; the second is rounded, 2^-8 of 2^-8) and the
sums to fp32, which move a score by at most d = scale (2^-16 + 64 2^-24) sum |q| |k|, a weight by the factor e^(2 d), so
o by at most (e^(2 d) - 1) A.  The exponential is good to 2^-22.  Together, with 1 % for the products of two of these and the
fp32 sums over the keys:  |error| <= 1.01 (h (A + |o|) + (e^(2 d) - 1) A) + 2^-20 A.  Below 2^-14 fp16 has steps of 2^-24, so that there
a rounding is off by up to 2^-25 whatever the value: of the output, and of weights whose sum is at least 1 (the largest of a row is),
which adds 2^-25 (1 + sum |v_j|).
"""
import numpy as np
import pytest
import torch

from paper_2607_21042_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
E4M3_BLOCK = 4352


def _bound(q, k, v, scale, h):
    """o and the tolerance for q [a, 64] against k, v [b, 64] (fp64)."""
    if k.shape[0] == 0:
        return np.zeros_like(q), np.zeros_like(q)
    s = q @ k.T * scale
    d = (np.abs(q) @ np.abs(k).T).max(-1, keepdims=True) * scale * (2.0 ** -16 + 64 * 2.0 ** -24)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o, A = p @ v, p @ np.abs(v)
    small = 2.0 ** -25 * (1 + np.abs(v).sum(0)) if h == HALF[torch.float16] else 0.0
    return o, 1.01 * (h * (A + np.abs(o)) + np.expm1(2 * d) * A) + 2.0 ** -20 * A + small


def _check(got, ref, tol, what):
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got)), what
    over = np.abs(got - ref) - tol
    assert over.max() <= 0, "%s: off by %.3g, %.3g allowed, at %s" % (what, np.abs(got - ref).flat[over.argmax()], tol.flat[over.argmax()],
                                                                    np.unravel_index(over.argmax(), over.shape))


def _gen(seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return g


def _dev(x):
    return torch.as_tensor(x).to(DEV)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------------------------
# attention of a batch that shares a prefix
# ---------------------------------------------------------------------------------------------
class Cache:
    """Rows with their own pages behind n_shared common ones; what no row may read is NaN (in the 8-bit cache: NaN scales)."""

    def __init__(self, seed, fmt, kv_heads, n_shared, own, pad=0, same_stream=()):
        g = _gen(seed)
        R, self.n_shared = len(own), n_shared
        need = [(t + 63) // 64 for t in own]
        pages = torch.randperm(n_shared + sum(need) + 3, generator=g).tolist()
        self.n_pages = len(pages)
        pps = n_shared + max(need + [0]) + 1
        table = np.full((R, pps), 0, dtype=np.int32)
        streams = torch.randperm(R, generator=g).tolist()
        kv = torch.randn(self.n_pages, 2, kv_heads, 64, 64, generator=g)
        live = np.zeros((self.n_pages, 64), dtype=bool)
        live[pages[:n_shared]] = True
        at = n_shared
        for i, m in enumerate(need):
            table[streams[i], :n_shared] = pages[:n_shared]
            table[streams[i], n_shared:n_shared + m] = pages[at:at + m]
            for j in range(m):
                live[pages[at + j], :min(64, own[i] - 64 * j)] = True
            at += m
        if fmt == "bf16":
            pool = kv.bfloat16()
            self.values = pool.double().numpy()
            pool[~torch.from_numpy(live)[:, None, None].expand(-1, 2, kv_heads, -1)] = float("nan")
        else:
            s = kv.abs().amax(-1) / 448
            codes = (kv / s[..., None]).to(torch.float8_e4m3fn)
            self.values = codes.double().numpy() * s.double().numpy()[..., None]
            dead = ~torch.from_numpy(live)[:, None, None].expand(-1, 2, kv_heads, -1)
            bits = codes.view(torch.uint8)
            bits[dead] = 0x7F
            s[dead] = float("nan")
            pool = torch.empty(self.n_pages, 2, kv_heads, E4M3_BLOCK, dtype=torch.uint8)
            pool[..., :4096] = bits.flatten(-2)
            pool[..., 4096:] = s.view(torch.uint8).flatten(-2).view(self.n_pages, 2, kv_heads, 256)
        self.pos = [64 * n_shared + t - 1 for t in own]
        for a, b, pos in same_stream:         # row a reads row b's keys up to pos
            streams[a], self.pos[a] = streams[b], pos
        self.streams = streams + [-1] * pad
        self.pos += [-1] * pad
        self.table, self.kv_heads, self.pool = table, kv_heads, pool.to(DEV)
        self.args = (_dev(table), _i32(self.streams), _i32(self.pos), n_shared)

    def keys(self, r, h):
        n = self.pos[r] + 1
        pages = self.table[self.streams[r]][:(n + 63) // 64]
        return [self.values[pages, x, h].reshape(-1, 64)[:n] for x in (0, 1)]

    def check(self, got, q, what):
        H = q.shape[1] // 64
        G = H // self.kv_heads
        ref, tol = np.zeros(q.shape), np.zeros(q.shape)
        qd = q.double().cpu().numpy()
        for r in range(q.shape[0]):
            if self.pos[r] < 0:
                continue
            for h in range(self.kv_heads):
                k, v = self.keys(r, h)
                sl = slice(h * G * 64, (h + 1) * G * 64)
                o, t = _bound(qd[r, sl].reshape(G, 64), k, v, 0.125, HALF[torch.bfloat16])
                ref[r, sl], tol[r, sl] = o.reshape(-1), t.reshape(-1)
        _check(got.view(torch.bfloat16), ref, tol, what)


def _q(seed, R, H, dtype, std=2.0):
    return (torch.randn(R, H * 64, generator=_gen(seed + 1000)) * std).to(dtype).to(DEV)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("qt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,kv,n_shared,own", [
    (4, 4, 0, [1]), (4, 4, 1, [0]), (20, 20, 7, [1]), (20, 20, 2, [64, 1, 0, 65, 31, 33, 32]),
    (4, 4, 3, [17] * 16), (4, 4, 1, [5] * 17), (2, 2, 5, [300, 0, 129]), (20, 4, 2, [9, 200, 64]), (12, 4, 1, list(range(0, 40, 3))),
    (16, 1, 2, [70, 3, 1]), (7, 1, 0, [1, 63, 64, 65, 500]), (1, 1, 30, [100, 77]), (20, 20, 0, [530, 2, 1000]), (3, 3, 4, [1] * 130),
])
def test_shared_prefix_attention(H, kv, n_shared, own, qt, fmt):
    c = Cache(H + len(own) + n_shared, fmt, kv, n_shared, own)
    q = _q(H, len(own), H, qt)
    c.check(B.op_attention_shared(q, c.pool, *c.args), q, "shared")


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_shared_prefix_padding_short_rows_and_rows_of_one_stream(fmt):
    # rows 1 and 2 end inside the shared pages, row 3 reads row 4's stream up to an earlier position, the last two rows are padding
    own = [40, 0, 0, 0, 100, 0, 64]
    c = Cache(5, fmt, 4, 2, own, pad=2, same_stream=[(1, 1, 70), (2, 2, 0), (3, 4, 150), (5, 4, 200)])
    q = _q(3, len(own) + 2, 8, torch.float32)
    out = torch.full((9, 512), 7.0, dtype=torch.bfloat16, device=DEV)
    got = B.op_attention_shared(q, c.pool, *c.args, out=out)
    assert got is out
    c.check(out, q, "mixed rows")
    assert torch.all(out[7:] == 0)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_shared_prefix_padding_rows_whose_positions_were_left(fmt):
    # a row of no stream is padding whatever its position says: it has no keys, and its length, the longest, says nothing about the others
    c = Cache(7, fmt, 2, 2, [40, 0, 9], pad=3, same_stream=[(1, 1, 70)])
    pos = c.args[2].clone()
    pos[3:] = torch.tensor([500, 0, 2 ** 31 - 1], dtype=torch.int32)
    q = _q(5, 6, 4, torch.float32)
    got = B.op_attention_shared(q, c.pool, c.args[0], c.args[1], pos, 2)
    c.check(got, q, "left positions")
    assert torch.all(got[3:].view(torch.bfloat16) == 0)


def test_shared_prefix_of_padding_rows_alone():
    c = Cache(6, "bf16", 2, 3, [], pad=5)
    c.args = (torch.zeros(1, 4, dtype=torch.int32, device=DEV),) + c.args[1:]
    q = _q(1, 5, 2, torch.bfloat16)
    assert torch.all(B.op_attention_shared(q, c.pool, *c.args).view(torch.bfloat16) == 0)


def test_shared_prefix_rows_of_a_wider_array_and_peaked_scores():
    c = Cache(8, "bf16", 4, 1, [30, 90, 2])
    wide = _q(2, 3, 12, torch.float32, std=30.0)        # scores up to hundreds: weights from 1 down to zero
    q = wide[:, 256:512]
    c.check(B.op_attention_shared(q, c.pool, *c.args), q, "strided")


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_shared_prefix_leaves_out_pages_that_are_none(fmt):
    c = Cache(9, fmt, 2, 1, [130, 64])
    table = c.args[0].clone()
    s = c.streams[0]
    table[s, 2] = 10 ** 6          # keys 128 .. 191 of row 0 lie on no page
    table[c.streams[1], 1] = -1
    q = _q(4, 2, 2, torch.float32)
    got = B.op_attention_shared(q, c.pool, table, *c.args[1:])
    ref, tol = np.zeros((2, 128)), np.zeros((2, 128))
    for r, keep in enumerate([[*range(0, 128), *range(192, 194)], [*range(0, 64)]]):
        for h in range(2):
            k, v = c.keys(r, h)
            ref[r, 64 * h:64 * h + 64], tol[r, 64 * h:64 * h + 64] = [x[0] for x in _bound(q[r:r + 1, 64 * h:64 * h + 64].double().cpu().numpy(), k[keep], v[keep], 0.125, 2.0 ** -8)]
    _check(got.view(torch.bfloat16), ref, tol, "bad pages")


def test_shared_prefix_agrees_with_the_attention_that_reads_the_prefix_for_each_row():
    c = Cache(10, "bf16", 20, 9, [3, 77, 400, 64, 1])
    q = _q(5, 5, 20, torch.float32)
    want = B.op_attention(q, c.pool.view(torch.int16), c.args[0], c.args[1], c.args[2])
    got = B.op_attention_shared(q, c.pool, *c.args).view(torch.bfloat16)
    c.check(got, q, "shared")
    c.check(want, q, "each row for itself")


def test_scratch_serves_calls_of_all_sizes_and_both_kinds_bit_for_bit():
    big, small = Cache(11, "bf16", 20, 4, [50 + 7 * i for i in range(60)]), Cache(12, "e4m3", 4, 11, [5, 0, 300])
    qb, qs = _q(6, 60, 20, torch.float32), _q(7, 3, 20, torch.bfloat16)
    x = CrossCase(13, torch.bfloat16, 4, 4, [1, 3, 1], [700, 0, 2000])
    fresh = [B.op_attention_shared(qb, big.pool, *big.args).clone(), B.op_attention_shared(qs, small.pool, *small.args).clone(), x.run().clone()]
    n = max(B.op_attention_shared_scratch(60, 20, 20, DEV).numel(), B.op_attention_cross_scratch(DEV).numel())
    scratch = torch.zeros(n, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        again = [B.op_attention_shared(qb, big.pool, *big.args, scratch=scratch), B.op_attention_shared(qs, small.pool, *small.args, scratch=scratch), x.run(scratch=scratch)]
        for a, b in zip(fresh, again):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert int(scratch[:4].view(torch.int32)) == 0


def test_results_do_not_depend_on_timing():
    """The same calls many times over, behind each other and beside other work: the same bits, whichever CTA comes last at a tile."""
    c = Cache(12, "e4m3", 4, 11, [5, 0, 300])
    q = _q(7, 3, 20, torch.bfloat16)
    xs = [CrossCase(14, torch.bfloat16, 20, 4, [1, 2], [900, 333]), CrossCase(15, torch.float16, 3, 3, [16, 5, 9], [2000, 100, 31]),
          CrossCase(16, torch.bfloat16, 6, 2, [90, 300], [700, 1500])]
    scratch = torch.zeros(max(B.op_attention_shared_scratch(3, 20, 4, DEV).numel(), B.op_attention_cross_scratch(DEV).numel()), dtype=torch.uint8, device=DEV)
    want = [B.op_attention_shared(q, c.pool, *c.args, scratch=scratch).clone()] + [x.run(scratch=scratch).clone() for x in xs]
    other, busy = torch.cuda.Stream(), torch.randn(2048, 2048, device=DEV)
    for k in range(30):
        with torch.cuda.stream(other):
            busy = busy @ busy.t() * 1e-3
        got = [B.op_attention_shared(q, c.pool, *c.args, scratch=scratch)] + [x.run(scratch=scratch) for x in xs]
        for w, y in zip(want, got):
            assert torch.equal(w.view(torch.int16), y.view(torch.int16)), k


# ---------------------------------------------------------------------------------------------
# attention to an encoder's states
# ---------------------------------------------------------------------------------------------
class CrossCase:
    def __init__(self, seed, dtype, heads, kv, ql, kl, layout="rows", gap_q=0, scale=0.125, std=2.0, q_max=None):
        g = _gen(seed)
        self.heads, self.kv, self.ql, self.kl, self.scale, self.dtype = heads, kv, ql, kl, scale, dtype
        self.q = (torch.randn(gap_q + sum(ql) + 3, heads, 64, generator=g) * std).to(dtype).to(DEV)
        T = sum(kl) + 2
        k, v = torch.randn(T, kv, 64, generator=g).to(dtype), torch.randn(T, kv, 64, generator=g).to(dtype)
        k[sum(kl):] = float("nan")             # behind the last sequence
        v[sum(kl):] = float("nan")
        self.kd, self.vd = k.double().numpy(), v.double().numpy()
        if layout == "rows":
            self.k, self.v = k.to(DEV), v.to(DEV)
        elif layout == "fused":
            kv2 = torch.stack([k, v], 1).to(DEV)
            self.k, self.v = kv2[:, 0], kv2[:, 1]
        elif layout == "heads":                # [heads, rows, 64]
            self.k, self.v = k.transpose(0, 1).contiguous().to(DEV).transpose(0, 1), v.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
        else:                                  # an odd row stride, K and V laid out differently
            wide = torch.zeros(T, kv * 64 + 40, dtype=dtype)
            wide[:, 16:16 + kv * 64] = k.reshape(T, -1)
            self.k = wide.to(DEV)[:, 16:16 + kv * 64].unflatten(1, (kv, 64))
            self.v = v.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
        self.qs = [gap_q + sum(ql[:i]) for i in range(len(ql) + 1)]
        self.ks = [sum(kl[:i]) for i in range(len(kl) + 1)]
        self.args = (self.q, self.k, self.v, _i32(self.qs), _i32(self.ks), max(ql) if q_max is None else q_max)

    def run(self, **kw):
        out = torch.full(self.q.shape, 9.0, dtype=self.dtype, device=DEV)
        return B.op_attention_cross(*self.args, scale=self.scale, out=out, **kw)

    def check(self, got, what="cross"):
        G = self.heads // self.kv
        ref, tol = np.full(got.shape, 9.0), np.zeros(got.shape)
        qd = self.q.double().cpu().numpy()
        for i in range(len(self.ql)):
            a, b, c, d = self.qs[i], self.qs[i + 1], self.ks[i], self.ks[i + 1]
            for h in range(self.heads):
                ref[a:b, h], tol[a:b, h] = _bound(qd[a:b, h], self.kd[c:d, h // G], self.vd[c:d, h // G], self.scale, HALF[self.dtype])
        _check(got, ref, tol, what)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,ql,kl", [
    (4, 4, [1], [1]), (20, 20, [1, 1, 1], [700, 1, 33]), (2, 2, [1, 0, 5, 1], [0, 40, 64, 65]), (3, 3, [16, 17, 1, 33], [31, 32, 33, 1000]),
    (20, 4, [1, 2, 7], [129, 0, 600]), (16, 1, [1, 3], [90, 1500]), (6, 2, [40, 5], [100, 17]), (20, 20, [32] * 5, [90, 200, 1, 0, 555]),
    (4, 4, [128], [128]), (4, 4, [129, 127, 1], [300, 129, 127]), (2, 2, [700, 0, 513], [1000, 5, 1]), (8, 2, [200, 65], [65, 777]), (1, 1, [300], [0]),
    (5, 1, [140, 300], [64, 257]), (3, 3, [256, 255, 257], [127, 384, 513]),
])
def test_cross_attention(heads, kv, ql, kl, dtype):
    c = CrossCase(len(ql) + heads, dtype, heads, kv, ql, kl)
    c.check(c.run())


@pytest.mark.parametrize("ql", [[1, 4, 2], [300, 64, 129]])
@pytest.mark.parametrize("layout", ["fused", "heads", "odd"])
def test_cross_attention_layouts_gaps_and_scale(layout, ql):
    c = CrossCase(21, torch.bfloat16, 6, 3, ql, [100, 31, 250], layout=layout, gap_q=5, scale=0.3)
    c.check(c.run(), layout)
    one = CrossCase(22, torch.float16, 2, 1, ql, [40, 0, 77], layout=layout, q_max=10 ** 6)
    one.check(one.run(), layout + ", one head of keys")


@pytest.mark.parametrize("ql", [[2, 2, 2], [150, 200, 150]])
def test_cross_attention_neighbours_infinities_and_peaked_scores(ql):
    c = CrossCase(23, torch.bfloat16, 2, 2, ql, [37, 50, 41], std=40.0)
    c.check(c.run(), "peaked")
    # what is not finite in one sequence stays there
    c.k[40:60] = float("inf")
    c.v[37:87] = float("nan")
    got = c.run()
    assert torch.isnan(got[c.qs[1]:c.qs[2]]).all()
    c.vd[37:87] = 0
    c.kd[37:87] = 0
    a, b = c.qs[1], c.qs[2]
    got[a:b] = 0
    c.check(got, "neighbours")


@pytest.mark.parametrize("ql", [[2, 2, 2], [150, 200, 150]])
def test_cross_attention_writes_nothing_where_starts_do_not_ascend(ql):
    c = CrossCase(24, torch.bfloat16, 2, 2, ql, [37, 50, 41])
    scratch = B.op_attention_cross_scratch(DEV)
    for at in (3, 4):
        args = list(c.args)
        args[at] = args[at][[0, 2, 1, 3]].contiguous()
        out = torch.full(c.q.shape, 9.0, dtype=c.dtype, device=DEV)
        B.op_attention_cross(*args, out=out, scratch=scratch)
        assert torch.all(out == 9.0)
    c.check(c.run(scratch=scratch), "after them")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("layout", ["rows", "fused", "heads", "odd"])
@pytest.mark.parametrize("heads,kv", [(2, 2), (10, 2), (16, 1), (3, 1)])
def test_cross_attention_of_long_and_short_sequences(heads, kv, layout, dtype):
    # many keys on average, and sequences with none, one, a block, a block and one
    ql, kl = [300, 64, 129, 40, 0, 257, 2, 513], [40, 0, 77, 1, 9, 128, 700, 129]
    c = CrossCase(26, dtype, heads, kv, ql, kl, layout=layout, gap_q=3, scale=0.2)
    c.check(c.run(), layout)
    short = CrossCase(27, dtype, heads, kv, [130, 90, 40], [0, 400, 0], layout=layout, q_max=129)
    short.ql[0] = 129                       # the row beyond q_max is not computed
    qs = short.qs
    got = short.run()
    assert torch.all(got[129] == 9.0) and torch.all(got[:129] == 0) and torch.all(got[qs[2]:qs[3]] == 0) and torch.all(got[qs[3]:] == 9.0)


def test_cross_attention_of_many_keys_neighbours_infinities_and_peaked_scores():
    c = CrossCase(28, torch.bfloat16, 2, 2, [150, 200, 150], [137, 150, 141], std=40.0)
    c.check(c.run(), "peaked")
    c.k[140:160] = float("inf")
    c.v[137:287] = float("nan")
    got = c.run()
    a, b = c.qs[1], c.qs[2]
    assert torch.isnan(got[a:b]).all()
    c.vd[137:287] = c.kd[137:287] = 0
    got[a:b] = 0
    c.check(got, "neighbours")
    # starts that do not ascend
    for at in (3, 4):
        args = list(c.args)
        args[at] = args[at][[0, 2, 1, 3]].contiguous()
        out = torch.full(c.q.shape, 9.0, dtype=c.dtype, device=DEV)
        B.op_attention_cross(*args, out=out)
        assert torch.all(out == 9.0)


@pytest.mark.parametrize("heads,kv,n,q", [(16, 1, 6, 1), (20, 4, 16, 3), (20, 20, 1, 16), (8, 8, 13, 9), (20, 20, 8, 16)])
def test_cross_attention_tiles_of_many_parts(heads, kv, n, q):
    c = CrossCase(29, torch.bfloat16, heads, kv, [q] * n, [700 + 37 * i for i in range(n)])
    got = c.run()
    c.check(got, "many parts")
    for _ in range(5):
        assert torch.equal(got.view(torch.int16), c.run().view(torch.int16))


@pytest.mark.parametrize("ql", [[5, 5], [60, 70]])
@pytest.mark.parametrize("key", [0, 5, 6, 7, 37, 130])
def test_cross_attention_keeps_nan(ql, key):
    # wherever the key lies that has it
    c = CrossCase(25, torch.bfloat16, 2, 2, ql, [140, 33])
    c.k[key] = float("nan")
    got = c.run()
    assert torch.isnan(got[:c.qs[1]]).all()
    assert torch.isfinite(got[c.qs[1]:c.qs[2]]).all()


def test_cross_attention_with_no_keys_at_all_and_no_queries():
    q = torch.ones(3, 4, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.empty(0, 4, 64, dtype=torch.bfloat16, device=DEV)
    out = B.op_attention_cross(q, k, k, _i32([0, 3]), _i32([0, 0]), 3)
    assert torch.all(out == 0)
    q = torch.ones(90, 4, 64, dtype=torch.bfloat16, device=DEV)
    assert torch.all(B.op_attention_cross(q, k, k, _i32([0, 40, 90]), _i32([0, 0, 0]), 50) == 0)
    out = torch.full_like(q, 5.0)
    k = torch.ones(8, 4, 64, dtype=torch.bfloat16, device=DEV)
    B.op_attention_cross(q, k, k, _i32([0, 0, 0]), _i32([0, 8, 8]), 1, out=out)
    assert torch.all(out == 5.0)


# ---------------------------------------------------------------------------------------------
# page lists and slot maps
# ---------------------------------------------------------------------------------------------
class Tables:
    """The device's arrays and, beside them, the same state kept by plain loops."""

    def __init__(self, streams, pps, n_pages, n_shared=0, max_rows=4096, seed=0, offset=0):
        perm = torch.randperm(n_pages + n_shared, generator=_gen(seed)).tolist()
        self.shared, self.free = perm[:n_shared], perm[n_shared:]
        self.pps, self.n_shared, self.max_rows = pps, n_shared, max_rows
        self.ctx, self.lists = [0] * streams, [[] for _ in range(streams)]
        self.d_ctx, self.d_table = _i32(self.ctx), torch.zeros(streams, pps, dtype=torch.int32, device=DEV)
        self.d_free, self.d_top, self.d_info = _i32(self.free), _i32([len(self.free)]), torch.zeros(8, dtype=torch.int32, device=DEV)
        self.d_shared = _i32(self.shared) if n_shared else None
        self.rows = [torch.full((max_rows + offset,), -5, dtype=torch.int32, device=DEV)[offset:] for _ in range(3)]

    def call(self, new, ids=None, **kw):
        n = len(new)
        self.row_start = torch.full((n + 1,), -5, dtype=torch.int32, device=DEV)
        B.op_page_tables(_i32(new), self.d_ctx, self.d_table, self.d_free, self.d_top, self.row_start, *self.rows, self.d_info,
                         stream_ids=None if ids is None else _i32(ids), shared_pages=self.d_shared, **kw)

    def step(self, new, ids=None):
        for x in self.rows:
            x.fill_(-5)
        self.call(new, ids)
        ids = list(range(len(new))) if ids is None else ids
        stream, pos, slot, start, taken = [], [], [], [0], 0
        for s, t in zip(ids, new):
            if self.ctx[s] == 0 and t > 0:
                self.lists[s] = list(self.shared)
                self.ctx[s] = 64 * self.n_shared
            for _ in range(t):
                c = self.ctx[s]
                if c // 64 == len(self.lists[s]):
                    self.lists[s].append(self.free.pop())
                    taken += 1
                stream.append(s); pos.append(c); slot.append(self.lists[s][c // 64] * 64 + c % 64)
                self.ctx[s] = c + 1
            start.append(len(stream))
        assert self.d_info.tolist()[:4] == [B.OK, len(stream), taken, len(self.free)]
        assert self.d_info.tolist()[7] == 0 and self.d_top.tolist() == [len(self.free)]
        assert self.row_start.tolist() == start and self.d_ctx.tolist() == self.ctx
        for got, want in zip(self.rows, (stream, pos, slot)):
            assert got.tolist() == want + [-5] * (self.max_rows - len(want))
        table = self.d_table.cpu().numpy()
        for s, pages in enumerate(self.lists):
            assert table[s, :len(pages)].tolist() == pages
        return stream, pos, slot


@pytest.mark.parametrize("n_shared", [0, 3])
@pytest.mark.parametrize("streams,offset", [(1, 0), (7, 1), (130, 0), (700, 3)])
def test_page_tables_over_several_passes(streams, offset, n_shared):
    t = Tables(streams, 20, 20 * streams, n_shared, max_rows=400 * streams, seed=streams, offset=offset)
    rng = np.random.default_rng(streams)
    t.step([int(x) for x in rng.integers(0, 200, streams)])
    for _ in range(3):
        n = int(rng.integers(1, streams + 1))
        ids = rng.permutation(streams)[:n].tolist()
        t.step([int(x) for x in rng.choice([0, 1, 1, 1, 63, 64, 65, 100], n)], ids)
    t.step([1] * streams)


def test_page_tables_exact_fit_and_largest_call():
    t = Tables(2, 2, 4, max_rows=256)
    t.step([128, 128])
    t = Tables(4096, 4, 3 * 4096, max_rows=130 * 4096, seed=2)
    t.step([130] * 4096, np.random.default_rng(3).permutation(4096).tolist())
    t.step([0] * 4096)


def test_page_tables_refuses_as_a_whole():
    def refused(code, new, ids=None, ctx=None, top=None, **size):
        t = Tables(**{"streams": 5, "pps": 3, "n_pages": 6, "n_shared": 1, "max_rows": 300, **size})
        t.step([10, 60, 0, 64, 1])
        if ctx is not None:
            t.d_ctx[2] = ctx
        if top is not None:
            t.d_top.fill_(top)
        for x in t.rows:
            x.fill_(-5)
        before = [x.clone() for x in (t.d_ctx, t.d_table, t.d_top, t.d_free)]
        t.call(new, ids)
        info = t.d_info.tolist()
        assert info[0] == code and info[1] == info[2] == info[7] == 0, info
        assert all(torch.equal(a, b) for a, b in zip(before, (t.d_ctx, t.d_table, t.d_top, t.d_free)))
        assert all((x == -5).all() for x in t.rows) and (t.row_start == -5).all()

    refused(B.E_ARG, [1, -1])
    refused(B.E_ARG, [1, 1, 1], ctx=-3)
    refused(B.E_ARG, [1], top=-1)
    refused(B.E_ARG, [1], top=7)
    refused(B.E_STREAM, [1, 1], [0, 5])
    refused(B.E_STREAM, [1, 1], [-1, 0])
    refused(B.E_STREAM, [1, 1, 0], [3, 0, 3])
    refused(B.E_CTX_OVERFLOW, [0, 69])            # 64 shared + 60 + 69 > 192
    refused(B.E_CTX_OVERFLOW, [0, 0, 129])        # opening: 64 shared + 129
    refused(B.E_CTX_OVERFLOW, [2 ** 31 - 1])
    refused(B.E_WORKSPACE, [100, 60, 100, 60, 100], max_rows=136)
    refused(B.E_NO_PAGES, [55, 5, 128])


def test_page_tables_with_separate_outputs_repeat():
    t = Tables(3, 4, 9, n_shared=1)
    ctx, top = torch.full((3,), -9, dtype=torch.int32, device=DEV), _i32([0])
    for _ in range(2):
        t.call([70, 0, 3], ids=[2, 1, 0], ctx_len_out=ctx, free_top_out=top)
        assert ctx.tolist() == [67, 0, 134] and top.tolist() == [6] and t.d_ctx.tolist() == [0, 0, 0] and t.d_top.tolist() == [9]
        assert t.d_table[2].tolist()[:3] == [t.shared[0], t.free[-1], t.free[-2]] and t.d_table[0].tolist()[:2] == [t.shared[0], t.free[-3]]


# ---------------------------------------------------------------------------------------------
# K and V rows into their slots
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("R,heads,strided", [(1, 1, False), (1, 20, True), (17, 3, True), (130, 20, False), (700, 5, True)])
def test_kv_append_matches_the_formats(R, heads, strided, fmt, dtype):
    g = _gen(R + heads)
    n_pages = (R + 63) // 64 + 2
    if strided:
        x = (torch.randn(R, 3, heads * 64, generator=g) * 3).to(dtype)
        x[0, 1, :64] = 0                       # a head whose values are all zero
        x = x.to(DEV)
        k, v = x[:, 1], x[:, 2]
    else:
        k, v = torch.randn(R, heads * 64, generator=g).to(dtype).to(DEV), (torch.randn(R, heads * 64, generator=g) * 1e-3).to(dtype).to(DEV)
    slot = torch.randperm(n_pages * 64, generator=g)[:R].int()
    for i, bad in ((3, -1), (5, n_pages * 64), (6, 2 ** 31 - 1), (7, -2 ** 31)):   # rows that belong nowhere
        if R > 10:
            slot[i] = bad
    pool = torch.randint(0, 100, (n_pages, 2, heads, 8192 if fmt == "bf16" else E4M3_BLOCK), generator=g).to(torch.uint8).to(DEV)
    want = pool.clone()
    arg = pool.view(torch.bfloat16).view(n_pages, 2, heads, 64, 64) if fmt == "bf16" else pool
    B.op_kv_append(k, v, arg, slot.to(DEV))
    ok = (slot >= 0) & (slot < n_pages * 64)
    rows, slots = torch.nonzero(ok)[:, 0].to(DEV), slot[ok].long().to(DEV)
    page, off = slots // 64, slots % 64
    for part, src in enumerate((k, v)):
        y = src[rows].float().view(-1, heads, 64)
        if fmt == "bf16":
            want.view(torch.bfloat16).view(n_pages, 2, heads, 64, 64)[page, part, :, off] = y.bfloat16()
        else:
            s = y.abs().amax(-1)
            s = s / torch.full_like(s, 448.0)      # by a tensor: a number's reciprocal would be rounded first
            s = torch.where(s > 0, s, torch.ones_like(s))
            want[..., :4096].unflatten(-1, (64, 64))[page, part, :, off] = (y / s[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
            want[..., 4096:].view(torch.float32)[page, part, :, off] = s
    assert torch.equal(pool, want)


# ---------------------------------------------------------------------------------------------
# together, on other streams, captured
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_a_served_batch_step_by_step(fmt):
    """Prefix prefilled once, four streams opened behind it, then decode steps: lists, rows and attention against plain arrays."""
    H, kv, shared, streams = 8, 4, 2, 4
    t = Tables(streams, 8, 14, n_shared=shared, max_rows=16, seed=1)
    pool = torch.zeros(20, 2, kv, 64, 64, dtype=torch.bfloat16, device=DEV) if fmt == "bf16" else torch.zeros(20, 2, kv, E4M3_BLOCK, dtype=torch.uint8, device=DEV)
    g = _gen(7)
    prefix = torch.randn(2, shared * 64, kv * 64, generator=g).to(DEV)
    slots = torch.cat([torch.arange(64) + 64 * p for p in t.shared]).int().to(DEV)
    B.op_kv_append(prefix[0], prefix[1], pool, slots)

    def stored(x):
        if fmt == "bf16":
            return x.bfloat16().double()
        y = x.view(-1, kv, 64)
        s = y.abs().amax(-1, keepdim=True)
        s = s / torch.full_like(s, 448.0)
        return ((y / s).to(torch.float8_e4m3fn).double() * s.double()).reshape(x.shape)

    held = [[stored(prefix[0])], [stored(prefix[1])]]
    keys = [[list(held[0]), list(held[1])] for _ in range(streams)]
    ids = [2, 0, 3, 1]
    for new in ([3, 1, 7, 2], [1, 1, 1, 1], [1, 0, 1, 1], [1, 1, 1, 1]):
        stream, pos, _ = t.step(new, ids)
        R = len(stream)
        qkv = torch.randn(R, (H + 2 * kv) * 64, generator=g).to(DEV)
        q, k, v = qkv[:, :H * 64], qkv[:, H * 64:(H + kv) * 64], qkv[:, (H + kv) * 64:]
        B.op_kv_append(k, v, pool, t.rows[2])
        out = B.op_attention_shared(q, pool, t.d_table, t.rows[0], t.rows[1], shared).view(torch.bfloat16)
        for r, s in enumerate(stream):
            keys[s][0].append(stored(k[r:r + 1])); keys[s][1].append(stored(v[r:r + 1]))
        for r, s in enumerate(stream):
            K, V = (torch.cat(x)[:pos[r] + 1].cpu().numpy() for x in keys[s])
            for h in range(H):
                c = slice(h // 2 * 64, h // 2 * 64 + 64)
                o, tol = _bound(q[r:r + 1, 64 * h:64 * h + 64].double().cpu().numpy(), K[:, c], V[:, c], 0.125, 2.0 ** -8)
                _check(out[r:r + 1, 64 * h:64 * h + 64], o, tol, "row %d head %d" % (r, h))


def test_captured_steps_on_a_stream_of_their_own():
    """A step captured once and replayed: lengths advance on the device, the last replay's rows are what plain calls give."""
    H, streams = 4, 3
    st = torch.cuda.Stream()
    t = Tables(streams, 4, 10, n_shared=1, max_rows=streams, seed=4)
    t.d_ctx.fill_(64 + 62)
    for s in range(streams):
        t.d_table[s, 0], t.d_table[s, 1] = t.shared[0], t.free[-1 - s]
    t.d_top.fill_(len(t.free) - streams)
    pool = torch.randn(11, 2, H, 64, 64, generator=_gen(3)).bfloat16().to(DEV)
    start = pool.clone()
    q, k, v = (torch.randn(streams, H * 64, generator=_gen(i)).to(DEV) for i in range(3))
    out = torch.zeros(streams, H * 64, dtype=torch.bfloat16, device=DEV)
    new, row_start, scratch = _i32([1] * streams), torch.zeros(streams + 1, dtype=torch.int32, device=DEV), B.op_attention_shared_scratch(streams, H, H, DEV)

    def step(o, scr):
        B.op_page_tables(new, t.d_ctx, t.d_table, t.d_free, t.d_top, row_start, *t.rows, t.d_info, shared_pages=t.d_shared)
        B.op_kv_append(k, v, pool, t.rows[2])
        B.op_attention_shared(q, pool, t.d_table, t.rows[0], t.rows[1], 1, scratch=scr, out=o)

    state = [x.clone() for x in (t.d_ctx, t.d_table, t.d_top)]
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        step(out, scratch)                     # warm
        st.synchronize()
        for x, y in zip((t.d_ctx, t.d_table, t.d_top, pool), state + [start]):
            x.copy_(y)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step(out, scratch)
        for _ in range(5):
            graph.replay()
    st.synchronize()
    assert t.d_ctx.tolist() == [64 + 67] * 3 and t.d_info.tolist()[0] == B.OK and t.rows[1].tolist() == [64 + 66] * 3
    got, replayed = out.clone(), pool.clone()
    for x, y in zip((t.d_ctx, t.d_table, t.d_top, pool), state + [start]):
        x.copy_(y)
    for _ in range(5):
        step(out, None)
    assert torch.equal(out, got) and torch.equal(pool, replayed)


def test_calls_on_a_stream_that_is_not_the_current_one():
    """Memory that a call makes for itself belongs to the stream it runs on."""
    st, c, x = torch.cuda.Stream(), Cache(41, "bf16", 4, 2, [70, 3, 200]), CrossCase(42, torch.float16, 4, 2, [3, 80], [600, 90])
    q = _q(43, 3, 4, torch.float32)
    want, wx = B.op_attention_shared(q, c.pool, *c.args).clone(), B.op_attention_cross(*x.args, scale=x.scale).clone()
    torch.cuda.synchronize()
    for _ in range(5):
        st.wait_stream(torch.cuda.current_stream())
        got = [B.op_attention_shared(q, c.pool, *c.args, stream=st), B.op_attention_cross(*x.args, scale=x.scale, stream=st)]
        junk = [torch.full((1 << 22,), 3.0, device=DEV) for _ in range(4)]      # what the current stream allocates meanwhile
        st.synchronize()
        assert torch.equal(got[0], want) and torch.equal(got[1][:x.qs[-1]], wx[:x.qs[-1]])
        del junk


def test_many_sequences_and_a_large_batch():
    """The largest numbers of sequences and of rows, with small work for each."""
    g = _gen(50)
    for n in (2049, 4096):
        ql, kl = torch.randint(0, 4, (n,), generator=g).tolist(), torch.randint(0, 40, (n,), generator=g).tolist()
        ql[7] = 45                             # more than two tiles of the warp-level kernel
        x = CrossCase(51, torch.bfloat16, 2, 1, ql, kl)
        x.check(x.run(), "%d sequences" % n)
    own = torch.randint(0, 70, (4096,), generator=g).tolist()
    c = Cache(52, "bf16", 1, 1, own)
    q = _q(53, 4096, 2, torch.bfloat16)
    c.check(B.op_attention_shared(q, c.pool, *c.args), q, "4096 rows")


def test_cross_attention_captured_and_on_two_streams_at_once():
    a, b = CrossCase(31, torch.bfloat16, 20, 20, [1] * 9, [900 - 70 * i for i in range(9)]), CrossCase(32, torch.float16, 20, 20, [300, 200], [500, 700])
    want = [a.run(), b.run()]
    streams, scratch = [torch.cuda.Stream(), torch.cuda.Stream()], [B.op_attention_cross_scratch(DEV) for _ in range(2)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c, st, sc in zip((a, b), streams, scratch):
        with torch.cuda.stream(st):
            out = torch.full(c.q.shape, 9.0, dtype=c.dtype, device=DEV)
            st.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                B.op_attention_cross(*c.args, scratch=sc, out=out)
            graphs.append(g); outs.append(out)
    for _ in range(10):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)
