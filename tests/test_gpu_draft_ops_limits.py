"""The draft operators where short things follow one another and where long ones end.  Tolerances as in test_gpu_draft_ops."""
from decimal import Decimal as D, localcontext

import numpy as np
import pytest
import torch

from paper_2607_21042_b200 import binding as B
from test_gpu_draft_ops import E4M3_BLOCK, Drafts, _empty_pool, _forest, _masks, _sees
from test_gpu_serving_ops import HALF, _bound, _check, _gen, _i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _check_tree(d, i, out, q, m):
    """Tree i's rows against the formula; m [t, t]: which nodes a row sees."""
    a, b, heads = d.start[i], d.start[i + 1], q.shape[1] // 64
    G = heads // d.kv_heads
    k, v = d.keys_of(i)
    x = q[a:b].double().cpu().numpy().reshape(-1, heads, 64)
    ref, tol = np.zeros_like(x), np.zeros_like(x)
    for r in range(b - a):
        on = np.concatenate([np.ones(d.ctx[i], bool), m[r]])
        for h in range(d.kv_heads):
            s = slice(h * G, h * G + G)
            ref[r, s], tol[r, s] = _bound(x[r, s], k[on, h], v[on, h], 0.125, HALF[torch.bfloat16])
    _check(out[a:b].view(-1, heads, 64), ref, tol, "tree %d" % i)


# ---------------------------------------------------------------------------------------------
# many tiles of a page or two in every CTA
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("t,H,K,ctx", [
    (4, 20, 20, [0, 3, 60, 17]), (4, 20, 20, [0, 90, 10, 60, 64]), (9, 12, 4, [0, 50, 70, 20, 130]), (11, 20, 4, [40, 0, 53]), (60, 12, 12, [4, 0, 3, 30])])
def test_tiles_of_few_pages(fmt, dtype, t, H, K, ctx):
    """Trees of one page, of one and two by turns, with trees without keys and pages that are none among them: a CTA has ten tiles and more, whose sums meet where the next
    ones' pages come."""
    n = 3200 // K if t < 60 else 200
    lens = [max(1, t - i % 3) for i in range(n)]
    ctx = [ctx[i % len(ctx)] if i % 9 != 4 else 0 for i in range(n)]
    d = Drafts(n + t, fmt, K, lens, ctx)
    _, parent = _forest(n, lens)
    sees = [_sees(parent[a:b]) for a, b in zip(d.start[:-1], d.start[1:])]
    for i in range(4, n, 9):                   # their only page is none, and every second has no stream
        d.table[d.ids[i], 0] = (-1, d.pages)[i % 2]
        if i % 2:
            d.kv_len[d.ids[i]] = 0
    q = d.queries(5, H, dtype)
    mask = _masks(sees, (max(lens) + 31) // 32)
    scratch = B.op_attention_tree_scratch(DEV)
    out = [d.run(q, mask, scratch=scratch) for _ in range(4)]
    assert int(scratch[:4].view(torch.int32)) == 0
    assert all(torch.equal(out[0].view(torch.int16), x.view(torch.int16)) for x in out[1:])
    for i in sorted({*range(0, n, n // 12), *range(4, n, 9)[:6]}):
        if i % 9 == 4:
            assert not out[0][d.start[i]:d.start[i + 1]].any()
        else:
            _check_tree(d, i, out[0], q, sees[i])
    assert torch.all(out[0][d.start[-1]:] == 9.0)


# ---------------------------------------------------------------------------------------------
# acceptance that is refused, and what follows it
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n", [3, 40, 300])
@pytest.mark.parametrize("code,what", [(B.E_ARG, "parent"), (B.E_ARG, "short"), (B.E_STREAM, "stream"), (B.E_STREAM, "twice"), (B.E_CTX_OVERFLOW, "long"), (B.E_WORKSPACE, "nodes"),
                                       (B.E_ARG, "height"), (B.E_ARG, "places"), (B.E_ARG, "starts"), (B.E_ARG, "end")])
def test_a_refused_acceptance_leaves_no_path(code, what, n):
    """Rows of trees that a step before would have moved: behind a refused call there is no path, and the same step's moves leave the cache as it is."""
    lens = [4] * n
    if what == "nodes":
        lens[1] = 257
    start, parent = _forest(1, lens)
    ids, kv, top, places, R = list(range(n)), [66] * n, 3, 3 + n, sum(lens) + 2
    path = np.full(R, -9)
    for a, b in zip(start[:-1], start[1:]):
        path[a:b - 1], path[b - 1] = np.arange(a + 1, b), -1       # every row to the place before
    if what == "nodes":
        kv[1] = 257 + 62
    if what == "parent":
        parent[4 + 2] = 2
    if what == "short":
        kv[1] = 3
    if what == "stream":
        ids[1] = n
    if what == "twice":
        ids[1] = 0
    if what == "long":
        kv[1] = 8 * 64 + 1
    if what == "height":
        top = places + 1
    if what == "places":                       # some pages come back, for which there is no place
        places = top
    if what == "starts":
        start[2] = 3
    if what == "end":
        start[n] += 3
    pages = (R + 63) // 64
    pool = torch.randint(0, 255, (2, pages, 2, 3, 8192), generator=_gen(1), dtype=torch.uint8).to(DEV).view(torch.bfloat16).unflatten(-1, (64, 64))
    before, slot = pool.clone(), torch.randperm(pages * 64, generator=_gen(2))[:R].to(torch.int32).to(DEV)
    start_d, path_d, kv_d, free, top_d = _i32(start.tolist()), _i32(path.tolist()), _i32(kv), _i32([0] * places), _i32([top])
    acc, nxt, info = _i32([-9] * n), _i32([-9] * n), _i32([0] * 8)
    # every drafted token agrees with what is said after its parent, so that other trees have paths that move
    B.op_tree_accept(_i32([1] * R), _i32([1] * R), _i32(parent.tolist() + [0, 0]), start_d, kv_d, torch.arange(8 * n, dtype=torch.int32, device=DEV).view(n, 8), free, top_d, path_d, acc, nxt,
                     info, stream_ids=_i32(ids))
    B.op_kv_move(pool, start_d, path_d, slot)
    assert info.tolist() == [code, 0, 0, top, 0, 0, 0, 0] and kv_d.tolist() == kv and top_d.item() == top and not free.any()
    last = min(int(start[n]), R)
    assert torch.all(path_d[:last] == -1) and torch.all(path_d[last:] == -9)
    assert torch.equal(pool.view(torch.int16), before.view(torch.int16))


# ---------------------------------------------------------------------------------------------
# moves
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,heads,lens,ends", [(0, 1, [9], [1]), (0, 20, [9, 30, 64], [1, 29, 0]), (1, 1, [130, 200, 3], [1, 64, 0]), (1, 20, [300, 257], [63, 161]), (0, 4, [700, 2], [65, 1]),
                                                 (0, 40, [700, 600], [513, 511])])
def test_a_path_ends_at_its_first_hole(fmt, heads, lens, ends):
    """Whatever stands behind the first -1 (or another negative number), in the same reach of a CTA's threads or a later one, moves nothing."""
    start = np.concatenate([[0], np.cumsum(lens)])
    R = int(start[-1])
    pages = (R + 63) // 64 + 1
    path = np.full(R, -1)
    for i, (t, end) in enumerate(zip(lens, ends)):
        path[start[i]:start[i + 1] - 1] = np.arange(start[i] + 1, start[i + 1])      # all rows one place on
        path[start[i] + end] = -1 - 5 * (i % 2)
    slot = np.random.default_rng(3).permutation(pages * 64)[:R]
    pool = torch.randint(0, 255, (pages, 2, heads, E4M3_BLOCK if fmt else 8192), generator=_gen(1), dtype=torch.uint8).to(DEV)
    want = pool.clone()
    views = (lambda x: [x[..., :4096].unflatten(-1, (64, 64)), x[..., 4096:].unflatten(-1, (64, 4))]) if fmt else (lambda x: [x.unflatten(-1, (64, 128))])  # noqa: E731
    for v in views(want):
        old = v.clone()
        for i, end in enumerate(ends):
            for k in range(min(end, lens[i] - 1)):
                a, b = slot[path[start[i] + k]], slot[start[i] + k]
                v[b // 64, :, :, b % 64] = old[a // 64, :, :, a % 64]
    B.op_kv_move(pool if fmt else pool.view(torch.bfloat16).unflatten(-1, (64, 64)), _i32(start.tolist()), _i32(path.tolist()), _i32(slot.tolist()))
    assert torch.equal(pool, want)


# ---------------------------------------------------------------------------------------------
# far positions
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_rot", [4, 26, 64])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_cosine_and_sine_of_far_positions(base, n_rot):
    """Pairs (1, 0) turn into cosine and sine.  The phase is that of the formula with 60 digits, modulo a turn, in whole numbers.  Off by: the table's two units of 2^-64 turns a
    position, 2^31 times, 2 pi 2^-32 radians or 0.025 2^-24; what is left of the angle rounded to fp32, pi 2^-27 or 0.4 2^-24; an ulp of sincospif, 2^-24 (the product with a
    magnitude of 1 is exact)."""
    rows, g = 400, np.random.default_rng(n_rot)
    pos = np.concatenate([[2 ** 31 - 1, -2 ** 31, 0, 1, -1, 2 ** 30], g.integers(-2 ** 31, 2 ** 31, rows - 6)])
    with localcontext() as c:
        c.prec = 60
        two_pi = 2 * D("3.14159265358979323846264338327950288419716939937510582097494459")
        turn = [int((-D(2 * i) / D(n_rot) * D(base).ln()).exp() / two_pi * 2 ** 128) for i in range(n_rot // 2)]
    part = np.array([[int(p) * t % 2 ** 128 / 2 ** 128 for t in turn] for p in pos])
    q = torch.zeros(rows, 64, device=DEV)
    q[:, :n_rot // 2] = 1.0
    got = B.op_rope_kv_append(q, q, q, _empty_pool(0, 8, 1), torch.arange(rows, dtype=torch.int32, device=DEV), _i32(pos.tolist()), B.op_rope_frequencies(n_rot, base=base, device=DEV)[0],
                              q_out=torch.empty_like(q)).double().cpu().numpy()
    off = max(np.abs(got[:, :n_rot // 2] - np.cos(2 * np.pi * part)).max(), np.abs(got[:, n_rot // 2:n_rot] - np.sin(2 * np.pi * part)).max())
    assert off <= 1.43 * 2.0 ** -24, off * 2 ** 24
    assert not got[:, n_rot:].any()


# ---------------------------------------------------------------------------------------------
# keys that are not finite
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("lens,ctx", [([20, 7], [33, 200]), ([64, 50], [10, 0]), ([100, 128], [70, 1])])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_key_that_is_not_finite(fmt, lens, ctx, value):
    """Queries are positive, so that an infinite key has an infinite score: NaN in the rows that see it, or no weight where it is -infinity."""
    d = Drafts(12, fmt, 2, lens, ctx)
    _, parent = _forest(4, lens)
    sees = [_sees(parent[a:b]) for a, b in zip(d.start[:-1], d.start[1:])]
    q = d.queries(9, 4, torch.bfloat16).abs()
    mask, odd = _masks(sees, (max(lens) + 31) // 32), [t // 3 for t in lens]
    for i, j in enumerate(odd):
        page, off = int(d.table[d.ids[i], (ctx[i] + j) // 64]), (ctx[i] + j) % 64
        if fmt:
            d.pool[page, 0, :, 64 * off:64 * off + 64] = 0xB8 if value < 0 else 0x38                       # minus or plus one
            d.pool[page, 0, :, 4096:].view(torch.float32)[:, off] = abs(value)
        else:
            d.pool[page, 0, :, off, 17] = value
    out = d.run(q, mask)
    rows = [r for i, (a, b) in enumerate(zip(d.start[:-1], d.start[1:])) for r in range(a, b) if value < 0 or not sees[i][r - a, odd[i]]]
    others = [r for r in range(int(d.start[-1])) if r not in set(rows)]
    for i, m in enumerate(sees):
        m[:, odd[i]] = False
    d.check(out, q, sees, rows=rows)
    assert bool(others) == (not value < 0) and torch.all(torch.isnan(out[others]))


# ---------------------------------------------------------------------------------------------
# large trees
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,H,K,dtype,lens,ctx,words", [
    (0, 2, 2, torch.bfloat16, [257, 1], [100, 30], 9), (1, 1, 1, torch.bfloat16, [500, 300], [0, 77], 16), (0, 1, 1, torch.float32, [1024, 40], [65, 500], 32),
    (1, 4, 1, torch.float32, [700], [300], 22), (0, 5, 1, torch.bfloat16, [1023, 1, 513], [1, 900, 128], 32), (1, 3, 1, torch.bfloat16, [1100, 20], [50, 64], 32)])
def test_trees_of_hundreds_of_nodes(fmt, H, K, dtype, lens, ctx, words):
    """Masks of up to 32 words; nodes behind the 1024th count as not seen, and the rows of such nodes see others all the same."""
    d = Drafts(sum(lens), fmt, K, lens, ctx)
    rng = np.random.default_rng(3)
    _, parent = _forest(sum(lens) + 1, lens, 9)
    sees = [_sees(parent[a:b]) for a, b in zip(d.start[:-1], d.start[1:])]
    for m in sees:
        m[rng.random(len(m)) < 0.05] = False   # some see nothing of the tree, some all before them
        m[rng.random(len(m)) < 0.05] = True
        m[:, 32 * words:] = False
    q, mask = d.queries(5, H, dtype), _masks([m[:, :32 * words] for m in sees], words)
    out = d.run(q, mask)
    for i, m in enumerate(sees):
        _check_tree(d, i, out, q, m)
    assert torch.all(out[d.start[-1]:] == 9.0)


@pytest.mark.parametrize("n,words", [(1024, 32), (1100, 32), (600, 19), (600, 10)])
def test_values_of_far_nodes_that_are_not_finite(n, words):
    """Only rows whose masks name such a node see it, in the last words too; nodes that the masks cannot name are seen by none."""
    d = Drafts(n, 0, 1, [n], [40])
    rng = np.random.default_rng(4)
    bad = [0, 31, 32, 300, min(n, 32 * words) - 1] + [j for j in (550, 1023, 1024, 1099) if j < n]
    for j, value in zip(bad, [float("nan"), float("inf"), -float("inf")] * 3):
        d.pool[int(d.table[0, (40 + j) // 64]), 1, 0, (40 + j) % 64, j % 64] = value
    m = rng.random((n, n)) < 0.02
    m[:, bad] = False
    named = [j for j in bad if j < 32 * words]
    for k, j in enumerate(named):
        m[20 + 50 * k:24 + 50 * k, j] = True
    m[:, 32 * words:] = False
    q = d.queries(5, 2, torch.bfloat16)
    out = d.run(q, _masks([m[:, :32 * words]], words))
    lost = m[:, named].any(1)
    want = np.isnan(out[:n].double().cpu().numpy()).reshape(n, -1)
    assert np.array_equal(want.all(1), lost) and np.array_equal(want.any(1), lost) and lost.sum() == 4 * len(named)
    for r in np.flatnonzero(~lost)[::7]:
        k, v = d.keys_of(0)
        on = np.concatenate([np.ones(40, bool), m[r]])
        ref, tol = _bound(q[r].double().cpu().numpy().reshape(2, 64), k[on, 0], v[on, 0], 0.125, HALF[torch.bfloat16])
        _check(out[r].view(2, 64), ref, tol, r)
