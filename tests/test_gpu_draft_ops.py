"""The operators of a program that decodes several drafted tokens a step, each against its formula in 64 bits: rotary positions on the way into
the cache, trees' masks and positions, attention of trees, acceptance, and the accepted rows' moves.

Rotation.  The phase is exact to 2^-64 turns a position.  What is left of it behind the nearest quarter turn is rounded to fp32, at most 2^-27 half turns, which
is pi 2^-27 radians; sincospif is good to an ulp, 2^-24; the product with the magnitude m rounds by 2^-24 m: cosine and sine are off by at most (0.4 + 1 + 1) 2^-24 m.  A
rotated value a c - b s rounds b s once and the sum once more.  Together at most 4.5 2^-24 m (|a| + |b|), then half a step of the type it is stored in.

Attention: as in test_gpu_serving_ops (weights rounded to bf16, of the 8-bit cache with V's scale in them, which is the same relative step)."""
import numpy as np
import pytest
import torch

from paper_2607_21042_b200 import binding as B
from test_gpu_serving_ops import HALF, _bound, _check, _gen, _i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4M3_BLOCK = 4352


# ---------------------------------------------------------------------------------------------
# rotary positions into the cache
# ---------------------------------------------------------------------------------------------
def _rotated(x, pos, w, mag, interleaved):
    """x [R, heads, 64] in 64 bits, rotated, and |a| + |b| of each value's pair (zero where nothing turns)."""
    half = len(w)
    i, j = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), np.arange(half, 2 * half))
    t = pos[:, None].astype(np.float64) * w[None]
    c, s = mag * np.cos(t)[:, None], mag * np.sin(t)[:, None]
    y, size = x.copy(), np.zeros_like(x)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    size[..., i] = size[..., j] = mag * (np.abs(x[..., i]) + np.abs(x[..., j]))
    return y, size


def _views(pool):
    return pool[..., :4096].unflatten(-1, (64, 64)).view(torch.float8_e4m3fn), pool[..., 4096:].view(torch.float32)


def _empty_pool(fmt, pages, heads, *layers):
    if fmt:
        return torch.full((*layers, pages, 2, heads, E4M3_BLOCK), 0x55, dtype=torch.uint8, device=DEV)
    return torch.full((*layers, pages, 2, heads, 64, 64), 7.0, dtype=torch.bfloat16, device=DEV)


def _close(got, ref, tol, what):
    got = np.asarray(got, np.float64)
    assert np.all(np.abs(got - ref) <= tol), (what, np.max(np.abs(got - ref) - tol))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,H,K,src,out,fmt,n_rot,fused,top", [
    (1, 20, 20, torch.float32, torch.float32, 0, 64, False, 1), (1, 4, 1, torch.bfloat16, torch.bfloat16, 1, 2, True, 2 ** 31 - 1),
    (5, 20, 20, torch.float32, torch.bfloat16, 0, 64, True, 2048), (77, 20, 4, torch.bfloat16, torch.bfloat16, 1, 32, True, 200000),
    (130, 12, 4, torch.float32, torch.float32, 1, 30, False, 2 ** 20), (33, 16, 1, torch.bfloat16, torch.float32, 0, 16, True, 2 ** 31 - 1),
    (9, 0, 3, torch.float32, torch.float32, 0, 62, False, 5000), (600, 1, 1, torch.bfloat16, torch.bfloat16, 0, 48, False, 10 ** 6),
    (3, 70, 70, torch.float32, torch.bfloat16, 1, 64, True, 10 ** 9)])
def test_rope_kv_append(rows, H, K, src, out, fmt, n_rot, fused, top, interleaved):
    g = _gen(rows * 7 + n_rot)
    pages = (rows + 63) // 64 + 2
    pool = _empty_pool(fmt, pages, K)
    before = pool.clone()
    slot = torch.randperm(pages * 64, generator=g)[:rows].to(torch.int32)
    out_of_it = torch.rand(rows, generator=g) < 0.2
    slot[out_of_it] = torch.tensor([-1, pages * 64, -2 ** 31, 2 ** 31 - 1])[torch.arange(rows) % 4].to(torch.int32)[out_of_it]
    pos = torch.randint(-top, top, (rows,), generator=g, dtype=torch.int64).clamp(-2 ** 31, 2 ** 31 - 1).to(torch.int32)
    x = torch.randn(rows, (H + 2 * K) * 64, generator=g).to(src).to(DEV)
    q, k, v = x.split([H * 64, K * 64, K * 64], 1)
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    w = 10000.0 ** (-np.arange(0, n_rot, 2) / n_rot)
    turns, mag = B.op_rope_frequencies(n_rot, device=DEV)
    assert mag == 1.0
    q_out = torch.full((rows, H * 64), 5.0, dtype=out, device=DEV) if H else None
    B.op_rope_kv_append(q if H else None, k, v, pool, slot.to(DEV), pos.to(DEV), turns, magnitude=1.25, interleaved=interleaved, q_out=q_out)
    torch.cuda.synchronize()
    live = ((slot >= 0) & (slot < pages * 64)).numpy()
    at, p = slot.numpy().astype(np.int64)[live], pos.numpy()[live]
    h = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
    if H:
        ref, size = _rotated(q.double().cpu().numpy().reshape(rows, H, 64)[live], p, w, 1.25, interleaved)
        got = q_out.double().cpu().numpy().reshape(rows, H, 64)
        _close(got[live], ref, 4.5 * 2.0 ** -24 * size + h[out] * np.abs(ref), "q")
        assert np.all(got[~live] == 5.0)
    parts = [_rotated(k.double().cpu().numpy().reshape(rows, K, 64)[live], p, w, 1.25, interleaved), (v.double().cpu().numpy().reshape(rows, K, 64)[live], 0.0)]
    for part, (ref, size) in enumerate(parts):
        if fmt:
            codes, scales = _views(pool)
            c, s = codes[at // 64, part, :, at % 64].double().cpu().numpy(), scales[at // 64, part, :, at % 64].double().cpu().numpy()
            most = np.abs(ref).max(-1)
            _close(s, most / 448, 2.0 ** -22 * np.max(np.abs(ref) + size, -1) / 448, "scales")
            _close(c * s[..., None], ref, 2.0 ** -4 * np.abs(ref) * (1 + 2.0 ** -10) + s[..., None] * 2.0 ** -10 + 2.0 ** -21 * (size + np.abs(ref)), "codes")
        else:
            _close(pool[at // 64, part, :, at % 64].double().cpu().numpy(), ref, 4.5 * 2.0 ** -24 * size + 2.0 ** -8 * np.abs(ref), "pool")
    # nothing else is written
    if fmt:
        for x0, x1 in zip(_views(before), _views(pool)):
            x0, x1 = x0.view(torch.uint8) if x0.dtype is torch.float8_e4m3fn else x0.contiguous().view(torch.int32), x1.view(torch.uint8) if x1.dtype is torch.float8_e4m3fn else x1.contiguous().view(torch.int32)
            x1 = x1.clone()
            x1[at // 64, :, :, at % 64] = x0[at // 64, :, :, at % 64]
            assert torch.equal(x0, x1)
    else:
        y = pool.clone()
        y[at // 64, :, :, at % 64] = 7.0
        assert torch.equal(y, before)


def test_rope_in_place_and_back():
    """q_out may be q, a part of the array that K and V are parts of; turning back by the negative position gives q again, to two roundings."""
    g = _gen(3)
    rows, H = 50, 8
    x = torch.randn(rows, 3, H * 64, generator=g).to(DEV)
    first = x.clone()
    q, k, v = x[:, 0], x[:, 1], x[:, 2]
    slot, pos = torch.arange(rows, dtype=torch.int32, device=DEV), torch.randint(0, 100000, (rows,), generator=g).to(torch.int32).to(DEV)
    turns, _ = B.op_rope_frequencies(64, device=DEV)
    apart = torch.empty(rows, H * 64, device=DEV)
    pools = [_empty_pool(0, 2, H) for _ in range(3)]
    B.op_rope_kv_append(q, k, v, pools[0], slot, pos, turns, q_out=apart)
    B.op_rope_kv_append(q, k, v, pools[1], slot, pos, turns, q_out=q)
    assert torch.equal(q, apart) and torch.equal(pools[0], pools[1]) and torch.equal(x[:, 1:], first[:, 1:])
    B.op_rope_kv_append(q, k, v, pools[2], slot, -pos, turns, q_out=q)
    size = (first[:, 0].view(rows, H, 2, 32).abs().sum(2, keepdim=True)).expand(-1, -1, 2, -1).reshape(rows, -1)
    assert torch.all((q - first[:, 0]).abs() <= 4 * 4.5 * 2.0 ** -24 * size)


def test_rope_values_that_are_not_numbers_stay_in_their_pair():
    rows, H = 4, 2
    x = torch.ones(rows, H * 64, device=DEV)
    x[1, 5] = float("nan")
    x[2, 40] = float("inf")                    # not rotated
    turns, _ = B.op_rope_frequencies(32, device=DEV)
    q = B.op_rope_kv_append(x, torch.ones_like(x), torch.ones_like(x), _empty_pool(0, 1, H), torch.arange(4, dtype=torch.int32, device=DEV),
                            torch.full((4,), 3, dtype=torch.int32, device=DEV), turns, q_out=torch.empty_like(x))
    bad = ~torch.isfinite(q)
    assert bad.sum() == 3 and bad[1, 5] and bad[1, 21] and q[2, 40] == float("inf")


# ---------------------------------------------------------------------------------------------
# trees
# ---------------------------------------------------------------------------------------------
def _forest(seed, lens, reach=6, roots=0.0):
    """Row starts and parents (numbers inside the tree); `roots`: how many of the later nodes have no parent."""
    g = np.random.default_rng(seed)
    parent = [-1 if j == 0 or g.random() < roots else j - 1 - int(g.integers(0, min(j, reach))) for t in lens for j in range(t)]
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), np.array(parent, np.int32)


def _sees(parent):
    """[t, t]: node j is i or an ancestor of i."""
    t = len(parent)
    m = np.zeros((t, t), bool)
    for i in range(t):
        j = i
        while j >= 0:
            m[i, j] = True
            j = parent[j]
    return m


def _words(m, words):
    out = np.zeros((m.shape[0], words), np.uint32)
    for j in range(m.shape[1]):
        out[:, j // 32] |= m[:, j].astype(np.uint32) << np.uint32(j % 32)
    return out.view(np.int32)


@pytest.mark.parametrize("lens,words,reach", [([1], 1, 1), ([32, 1, 0, 31, 17], 1, 3), ([33, 64, 2], 2, 64), ([65, 96, 1, 0, 7], 3, 1), ([256, 129, 255, 256], 8, 9), ([256], 8, 1),
                                              ([5] * 300, 1, 2), ([128, 100], 4, 128)])
def test_tree_tables(lens, words, reach):
    start, parent = _forest(sum(lens), lens, reach, 0.05)
    n, R = len(lens), sum(lens) + 3
    rng = np.random.default_rng(1)
    ids = rng.permutation(n + 2)[:n]
    kv = rng.integers(300, 2000, n + 2)
    mask, pos, info = torch.full((R, words), 77, dtype=torch.int32, device=DEV), torch.full((R,), -5, dtype=torch.int32, device=DEV), _i32([0] * 8)
    B.op_tree_tables(_i32(parent.tolist() + [9] * 3), _i32(start.tolist()), _i32(kv.tolist()), mask, pos, info, stream_ids=_i32(ids.tolist()))
    mask, pos = mask.cpu().numpy(), pos.cpu().numpy()
    assert info[0] == 0
    for i in range(n):
        a, b = start[i], start[i + 1]
        m = _sees(parent[a:b])
        assert np.array_equal(mask[a:b], _words(m, words))
        assert np.array_equal(pos[a:b], kv[ids[i]] - (b - a) + m.sum(1) - 1)
    assert np.all(mask[start[-1]:] == 77) and np.all(pos[start[-1]:] == -5)


@pytest.mark.parametrize("code,what", [(B.E_ARG, "parent"), (B.E_ARG, "negative"), (B.E_ARG, "short"), (B.E_STREAM, "stream"), (B.E_WORKSPACE, "nodes"), (B.E_ARG, "starts"), (B.E_ARG, "end")])
def test_tree_tables_leaves_a_wrong_tree_as_it_was(code, what):
    lens = [4, 6, 5]
    start, parent = _forest(2, lens)
    ids, kv, R, words = [0, 1, 2], [100, 200, 300], 15, 1
    if what == "parent":
        parent[4 + 3] = 3
    if what == "negative":
        parent[4 + 3] = -2
    if what == "short":
        kv[1] = 5
    if what == "stream":
        ids[1] = 3
    if what == "nodes":
        lens[1] = 40
        start, parent = _forest(2, lens)
        R = 49
    if what == "starts":
        start[2] = 3
    if what == "end":
        start[3] = 16
    mask, pos, info = torch.full((R, words), 77, dtype=torch.int32, device=DEV), torch.full((R,), -5, dtype=torch.int32, device=DEV), _i32([0] * 8)
    B.op_tree_tables(_i32(parent.tolist()), _i32(start.tolist()), _i32(kv), mask, pos, info, stream_ids=_i32(ids))
    assert info[0] == code
    pos = pos.cpu().numpy()
    wrong = 2 if what == "end" else 1
    for i in range(3):
        if i == wrong:
            assert what == "starts" or np.all(pos[start[i]:min(start[i + 1], R)] == -5)
        elif not (what == "starts" and i == 2):
            assert np.all(pos[start[i]:start[i + 1]] >= 0)


def _accept_oracle(start, parent, draft, target):
    paths, nxt = [], []
    for a, b in zip(start[:-1], start[1:]):
        path, at, said = [], 0 if b > a else -1, -1
        while at >= 0:
            path.append(at)
            said = target[a + at]
            at = next((j for j in range(b - a) if parent[a + j] == at and draft[a + j] == said), -1)
        paths.append(path)
        nxt.append(said)
    return paths, nxt


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lens,vocab,reach", [([1], 2, 1), ([5, 0, 9, 1], 2, 3), ([64] * 16, 3, 8), ([40, 256, 255, 1, 32, 33] * 7, 3, 20), ([256], 1, 1), ([3] * 600, 2, 2), ([7] * 4096, 2, 3)])
def test_tree_accept(lens, vocab, reach, in_place):
    n = len(lens)
    start, parent = _forest(n + sum(lens), lens, reach, 0.03)
    rng = np.random.default_rng(n)
    R, pps, streams = sum(lens) + 2, 9, n + 3
    draft, target = rng.integers(0, vocab, R), rng.integers(0, vocab, R)
    ids = rng.permutation(streams)[:n]
    kv = np.full(streams, -1)
    kv[ids] = [int(rng.integers(0, pps * 64 - t + 1)) + t for t in lens]
    table = rng.permutation(streams * pps).reshape(streams, pps)
    top, places = 5, streams * pps + 5
    free = rng.integers(0, 1000, places)
    dev = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)  # noqa: E731
    kv_d, top_d, free_d, path, acc, nxt, info = dev(kv), dev([top]), dev(free), dev([-9] * R), dev([-9] * n), dev([-9] * n), dev([0] * 8)
    kv_out, top_out = (None, None) if in_place else (kv_d.clone(), dev([-9]))
    for _ in range(1 if in_place else 2):      # (a second time: what the first left in info does not matter)
        B.op_tree_accept(dev(draft), dev(target), dev(parent.tolist() + [0, 0]), dev(start), kv_d, dev(table), free_d, top_d, path, acc, nxt, info, stream_ids=dev(ids),
                         kv_len_out=kv_out, free_top_out=top_out)
    kv_got, top_got = (kv_d, top_d) if in_place else (kv_out, top_out)
    paths, said = _accept_oracle(start, parent, draft, target)
    want_path, want_kv, want_free = np.full(R, -9), kv.copy(), list(free[:top])
    for i, p in enumerate(paths):
        want_path[start[i]:start[i + 1]] = -1
        want_path[start[i]:start[i] + len(p)] = np.array(p, int) + start[i]
        s = ids[i]
        want_kv[s] = kv[s] - lens[i] + len(p)
        for e in range((kv[s] + 63) // 64 - 1, (want_kv[s] + 63) // 64 - 1, -1):
            want_free.append(table[s, e])
    assert info.tolist() == [0, sum(map(len, paths)), len(want_free) - top, len(want_free), 0, 0, 0, 0]
    assert np.array_equal(path.cpu().numpy(), want_path) and acc.tolist() == [len(p) for p in paths] and nxt.tolist() == said
    assert np.array_equal(kv_got.cpu().numpy(), want_kv) and top_got.item() == len(want_free)
    assert free_d.cpu().numpy()[:len(want_free)].tolist() == [int(x) for x in want_free] and np.array_equal(free_d.cpu().numpy()[len(want_free):], free[len(want_free):])


@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("code,what", [(B.E_ARG, "parent"), (B.E_ARG, "short"), (B.E_STREAM, "stream"), (B.E_STREAM, "twice"), (B.E_CTX_OVERFLOW, "long"), (B.E_WORKSPACE, "nodes"),
                                       (B.E_ARG, "height"), (B.E_ARG, "places"), (B.E_ARG, "end")])
def test_tree_accept_is_refused_as_a_whole(code, what, n):
    lens = [4] * n
    if what == "nodes":
        lens[1] = 257
    start, parent = _forest(1, lens)
    ids, kv, top, places = list(range(n)), [66] * n, 3, 3 + n
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
    if what == "places":
        places = 3 + n - 1
    if what == "end":
        start[n] += 5
    R = sum(lens)
    kv_d, free, top_d = _i32(kv), _i32([0] * places), _i32([top])
    path, acc, nxt, info = _i32([-9] * R), _i32([-9] * n), _i32([-9] * n), _i32([0] * 8)
    # no drafted token agrees: one node each, and a page back
    B.op_tree_accept(_i32([1] * R), _i32([2] * R), _i32(parent.tolist()), _i32(start.tolist()), kv_d, torch.arange(8 * n, dtype=torch.int32, device=DEV).view(n, 8), free, top_d, path, acc,
                     nxt, info, stream_ids=_i32(ids))
    assert info.tolist() == [code, 0, 0, top, 0, 0, 0, 0]
    assert kv_d.tolist() == kv and top_d.item() == top and not free.any()
    bad = {"parent": 1, "nodes": 1, "end": n - 1}.get(what)
    assert acc.tolist() == [0 if i == bad else 1 for i in range(n)] and nxt.tolist() == [-1 if i == bad else 2 for i in range(n)]


# ---------------------------------------------------------------------------------------------
# moves
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,lens,heads,layers", [(0, [1], 1, 1), (1, [9, 0, 64, 5], 4, 1), (0, [256, 40, 1, 300], 20, 3), (1, [300, 64], 20, 2), (0, [12] * 50, 3, 5), (1, [700], 1, 1)])
def test_kv_move(fmt, lens, heads, layers):
    rng = np.random.default_rng(len(lens))
    start = np.concatenate([[0], np.cumsum(lens)])
    R = int(start[-1]) + 4
    pages = (R + 63) // 64 + 2
    slot = rng.permutation(pages * 64)[:R]
    slot[rng.random(R) < 0.05] = -1
    slot[rng.random(R) < 0.05] = pages * 64
    path = np.full(R, -1)
    for i, t in enumerate(lens):
        p = np.flatnonzero(rng.random(t) < (0.3, 0.9)[i % 2])
        path[start[i]:start[i] + len(p)] = p + start[i]
    pool = torch.randint(0, 255, (layers, pages + 1, 2, heads, E4M3_BLOCK if fmt else 8192), generator=_gen(1), dtype=torch.uint8).to(DEV)
    whole = pool if fmt else pool.view(torch.bfloat16).unflatten(-1, (64, 64))
    want = pool.clone()
    views = (lambda x: [x[:, :pages, ..., :4096].unflatten(-1, (64, 64)), x[:, :pages, ..., 4096:].unflatten(-1, (64, 4))]) if fmt else \
        (lambda x: [x[:, :pages].unflatten(-1, (64, 128))])  # noqa: E731
    for i in range(len(lens)):
        rows = [r for r in path[start[i]:start[i + 1]] if r >= 0]
        for v in views(want):
            old = v.clone()
            for k, r in enumerate(rows):
                a, b = slot[r], slot[start[i] + k]
                if min(a, b) >= 0 and max(a, b) < pages * 64:
                    v[:, b // 64, :, :, b % 64] = old[:, a // 64, :, :, a % 64]
    args = _i32(start.tolist()), _i32(path.tolist()), _i32(slot.tolist())
    if layers == 1:
        B.op_kv_move(whole[0, :pages], *args)
    else:
        B.op_kv_move(whole[:, :pages], *args)      # layers a page further apart than they are long
    assert torch.equal(pool, want)


# ---------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------
class Drafts:
    """Streams of a paged cache with a tree of drafted tokens each; slots that hold no token are NaN (8-bit cache: NaN scales), as are rows outside trees."""

    def __init__(self, seed, fmt, kv_heads, lens, ctx, pps=None, extra=2):
        rng = np.random.default_rng(seed)
        self.lens, self.ctx, self.fmt, self.kv_heads, n = lens, ctx, fmt, kv_heads, len(lens)
        self.start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.R = int(self.start[-1]) + extra
        keys = [c + t for c, t in zip(ctx, lens)]
        held = [(k + 63) // 64 for k in keys]
        self.pps = pps or max(held) + 1
        self.pages = sum(held) + 2
        self.ids = rng.permutation(n)
        self.kv_len = np.zeros(n, np.int32)
        self.kv_len[self.ids] = keys
        perm, at = rng.permutation(self.pages), 0
        self.table = np.full((n, self.pps), self.pages - 1, np.int32)
        live = np.zeros((self.pages, 64), bool)
        for i, h in enumerate(held):
            mine = perm[at:at + h]
            self.table[self.ids[i], :min(h, self.pps)] = mine[:self.pps]
            live.reshape(-1)[(mine[:, None] * 64 + np.arange(64)).reshape(-1)[:keys[i]]] = True
            at += h
        kv = torch.randn(self.pages, 2, kv_heads, 64, 64, generator=_gen(seed))
        if fmt:
            s = kv.abs().amax(-1) / 448
            codes = (kv / s[..., None]).to(torch.float8_e4m3fn)
            self.kv = (codes.double() * s.double()[..., None]).numpy()
            s[~torch.tensor(live)[:, None, None].expand_as(s)] = float("nan")
            pool = torch.empty(self.pages, 2, kv_heads, E4M3_BLOCK, dtype=torch.uint8)
            pool[..., :4096] = codes.view(torch.uint8).flatten(-2)
            pool[..., 4096:].view(torch.float32).copy_(s)
        else:
            pool = kv.bfloat16()
            self.kv = pool.double().numpy()
            pool[~torch.tensor(live)[:, None, None].expand(*kv.shape[:-1])] = float("nan")
        self.pool = pool.to(DEV)

    def keys_of(self, i):
        """K and V [keys, heads, 64] of tree i's stream."""
        n = self.ctx[i] + self.lens[i]
        pages = self.table[self.ids[i]][:(n + 63) // 64]
        return [self.kv[pages, w].transpose(0, 2, 1, 3).reshape(-1, self.kv_heads, 64)[:n] for w in (0, 1)]

    def queries(self, seed, heads, dtype):
        q = torch.randn(self.R, heads * 64, generator=_gen(seed)).mul_(2).to(dtype)
        q[self.start[-1]:] = float("nan")
        return q.to(DEV)

    def run(self, q, mask, **kw):
        out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device=DEV)
        kw.setdefault("t_max", max(self.lens))
        B.op_attention_tree(q, self.pool, _i32(self.table.tolist()), _i32(self.start.tolist()), _i32(self.kv_len.tolist()), mask, stream_ids=_i32(self.ids.tolist()), out=out, **kw)
        torch.cuda.synchronize()
        return out

    def check(self, out, q, sees, scale=0.125, rows=None):
        """sees: of each tree, [t, t] which nodes a row sees."""
        heads = q.shape[1] // 64
        G = heads // self.kv_heads
        qn = q.double().cpu().numpy().reshape(self.R, heads, 64)
        ref, tol = np.full((self.R, heads, 64), 9.0), np.zeros((self.R, heads, 64))
        for i, m in enumerate(sees):
            k, v = self.keys_of(i)
            a = self.start[i]
            for r in range(self.lens[i]):
                on = np.concatenate([np.ones(self.ctx[i], bool), m[r]])
                for h in range(self.kv_heads):
                    s = slice(h * G, h * G + G)
                    ref[a + r, s], tol[a + r, s] = _bound(qn[a + r, s], k[on, h], v[on, h], scale, HALF[torch.bfloat16])
        got = out.view(self.R, heads, 64)
        pick = slice(None) if rows is None else rows
        _check(got[pick], ref[pick], tol[pick], "attention")
        assert torch.all(out[self.start[-1]:] == 9.0)


def _masks(sees, words, extra=2):
    out = np.concatenate([_words(m, words) for m in sees if len(m)] + [np.full((extra, words), -1, np.int32)])
    return torch.tensor(out, device=DEV)


CASES = [  # format, query heads, heads of keys, query type, nodes, committed tokens
    (0, 1, 1, torch.bfloat16, [1], [0]), (1, 1, 1, torch.float32, [1], [0]), (0, 4, 4, torch.float32, [8], [333]),
    (0, 2, 2, torch.bfloat16, [32, 1, 7, 0, 31], [64, 0, 127, 50, 128]), (1, 2, 2, torch.bfloat16, [32, 1, 7, 0, 31], [64, 0, 127, 50, 128]),
    (0, 2, 2, torch.float32, [64, 33, 1, 50], [100, 700, 1900, 0]), (1, 2, 2, torch.float32, [64, 33, 1, 50], [100, 700, 1900, 0]),
    (0, 2, 2, torch.bfloat16, [128, 100, 65], [5, 1000, 321]), (1, 2, 2, torch.bfloat16, [128, 100, 65], [5, 1000, 321]),
    (0, 1, 1, torch.float32, [256, 3, 200], [500, 1500, 0]), (1, 1, 1, torch.bfloat16, [256, 3, 200], [500, 1500, 0]),
    (0, 12, 4, torch.bfloat16, [25, 5, 10, 11, 1, 1], [60, 1900, 400, 63, 64, 65]), (1, 20, 4, torch.bfloat16, [25, 5, 10, 6, 1, 1], [60, 1900, 400, 63, 64, 65]),
    (0, 16, 1, torch.float32, [2, 9, 1], [1000, 30, 2]), (1, 16, 1, torch.bfloat16, [2, 9, 1, 40], [1000, 30, 2, 7]), (0, 6, 2, torch.bfloat16, [21, 22, 43, 10], [33, 200, 500, 129]),
    (0, 2, 2, torch.bfloat16, [3] * 400, [17 + 3 * i for i in range(400)]), (1, 2, 1, torch.float32, [5] * 300, [1 + 5 * i for i in range(300)])]


@pytest.mark.parametrize("fmt,H,K,dtype,lens,ctx", CASES)
def test_attention_tree(fmt, H, K, dtype, lens, ctx):
    d = Drafts(H + sum(lens), fmt, K, lens, ctx)
    _, parent = _forest(sum(lens) + 1, lens)
    sees = [_sees(parent[a:b]) for a, b in zip(d.start[:-1], d.start[1:])]
    q = d.queries(5, H, dtype)
    scratch = B.op_attention_tree_scratch(DEV)
    out = d.run(q, _masks(sees, (max(lens) + 31) // 32), scratch=scratch)
    d.check(out, q, sees)
    again = d.run(q, _masks(sees, (max(lens) + 31) // 32), scratch=scratch)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and scratch[:256 + 65536].count_nonzero() == 0


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("lens,ctx", [([20, 7, 1], [0, 200, 0]), ([64, 64], [0, 90]), ([100, 128], [0, 64])])
def test_attention_tree_any_mask(fmt, lens, ctx):
    """Masks that are no trees: rows that see nothing, all, or one node; words and bits behind the last node do not matter."""
    d = Drafts(7, fmt, 2, lens, ctx)
    rng = np.random.default_rng(8)
    sees = []
    for t in lens:
        m = rng.random((t, t)) < rng.random((t, 1))
        m[0] = False
        m[t // 2] = np.arange(t) == t - 1
        m[t - 1] = t > 1
        sees.append(m)
    words = (max(lens) + 31) // 32 + 1
    mask = _masks(sees, words).cpu().numpy().view(np.uint32)
    at = 0
    for t in lens:
        for j in range(t, 32 * words):
            mask[at:at + t, j // 32] |= np.uint32(1) << np.uint32(j % 32)
        at += t
    q = d.queries(9, 4, torch.bfloat16)
    d.check(d.run(q, torch.tensor(mask.view(np.int32), device=DEV)), q, sees)
    # nodes behind the mask's words count as not seen
    few = [m & (np.arange(m.shape[1]) < 32) for m in sees]
    d.check(d.run(q, _masks(sees, words)[:, :1].contiguous()), q, few)


@pytest.mark.parametrize("lens,ctx", [([20, 7, 30], [33, 200, 0]), ([64, 50], [10, 200]), ([100, 128], [70, 1])])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_attention_tree_of_nodes_that_were_never_written(lens, ctx, value):
    """A tree padded to a size: the last nodes hold anything, and only they see themselves."""
    d = Drafts(3, 0, 2, lens, ctx)
    pad = [t // 3 for t in lens]
    for i, (t, p) in enumerate(zip(lens, pad)):
        for pos in range(ctx[i] + t - p, ctx[i] + t):
            page = int(d.table[d.ids[i], pos // 64])
            d.pool[page, :, :, pos % 64] = value
    _, parent = _forest(4, lens)
    sees, rows = [], []
    for i, (a, b) in enumerate(zip(d.start[:-1], d.start[1:])):
        m = _sees(parent[a:b])
        m[:, lens[i] - pad[i]:] = False        # no other row sees them
        m[lens[i] - pad[i]:] = False
        m[np.arange(lens[i] - pad[i], lens[i]), np.arange(lens[i] - pad[i], lens[i])] = True
        sees.append(m)
        rows += list(range(a, b - pad[i]))
    q = d.queries(9, 4, torch.bfloat16)
    out = d.run(q, _masks(sees, (max(lens) + 31) // 32))
    d.check(out, q, sees, rows=rows)
    padded = [r for r in range(int(d.start[-1])) if r not in set(rows)]
    assert torch.all(torch.isnan(out[padded].view(len(padded), 4, 64)).all(-1))
