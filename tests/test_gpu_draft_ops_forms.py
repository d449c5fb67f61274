"""The draft operators in the forms a program has them: a whole loop of drafting and accepting, captured and replayed, on two streams at once, views with strides, pools of more than
4 GB, lists and lengths that are wrong, waits that run out.  Tolerances as in test_gpu_draft_ops."""
import numpy as np
import pytest
import torch

from paper_2607_21042_b200 import binding as B
from test_gpu_draft_ops import Drafts, E4M3_BLOCK, _close, _empty_pool, _forest, _masks, _rotated, _sees, _views
from test_gpu_serving_ops import HALF, _bound, _gen, _i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# ---------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------
class Loop:
    """Streams that draft and accept over one paged cache.  A token's queries, keys and values are rows of tables (two layers), its logits a product of both layers'
    attention with a matrix, so that what is said depends on every token before.  All state lives on the device; `step` makes only calls that can be captured."""

    H, K, V, LAYERS = 4, 2, 7, 2

    def __init__(self, seed, fmt, streams, pages, max_rows, words, interleaved=False):
        g = _gen(seed)
        self.fmt, self.streams, self.words, self.max_rows, self.interleaved, H, K = fmt, streams, words, max_rows, interleaved, self.H, self.K
        self.qkv = torch.randn(self.LAYERS, self.V, (H + 2 * K) * 64, generator=g).to(DEV)
        self.out_w = torch.randn(self.LAYERS * H * 64, self.V, generator=g).to(DEV)
        self.w = 10000.0 ** (-np.arange(0, 48, 2) / 48)
        self.turns, self.mag = B.op_rope_frequencies(48, device=DEV)
        self.pool = _empty_pool(fmt, pages, K, self.LAYERS)
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)  # noqa: E731
        self.pages, self.kv_len, self.table, self.free, self.top = pages, i32(streams), i32(streams, 30), torch.randperm(pages, generator=g).to(torch.int32).to(DEV), _i32([pages])
        self.rows = [i32(max_rows) for _ in range(3)]
        self.start, self.draft, self.parent, self.new = i32(streams + 1), i32(max_rows), i32(max_rows), i32(streams)
        self.mask, self.pos, self.path, self.n_acc, self.next = i32(max_rows, words), i32(max_rows), i32(max_rows), i32(streams), i32(streams)
        self.info, self.tree_info, self.acc_info = i32(8), i32(8), i32(8)
        self.scratch = B.op_attention_tree_scratch(DEV)
        self.outs = torch.zeros(max_rows, self.LAYERS, H * 64, dtype=torch.bfloat16, device=DEV)
        self.q_out = torch.zeros(max_rows, H * 64, device=DEV)
        self.o = [torch.zeros(max_rows, H * 64, dtype=torch.bfloat16, device=DEV) for _ in range(self.LAYERS)]

    def step(self):
        H, K = self.H, self.K
        self.rows[2].fill_(-1)                 # rows behind the last tree have no slot
        B.op_page_tables(self.new, self.kv_len, self.table, self.free, self.top, self.start, *self.rows, self.info)
        B.op_tree_tables(self.parent, self.start, self.kv_len, self.mask, self.pos, self.tree_info)
        for layer in range(self.LAYERS):
            x = self.qkv[layer].index_select(0, self.draft)
            q, k, v = x.split([H * 64, K * 64, K * 64], 1)
            B.op_rope_kv_append(q, k, v, self.pool[layer], self.rows[2], self.pos, self.turns, self.mag, self.interleaved, q_out=self.q_out)
            B.op_attention_tree(self.q_out, self.pool[layer], self.table, self.start, self.kv_len, self.mask, 32 * self.words, scratch=self.scratch, out=self.o[layer])
        logits = torch.cat(self.o, 1).float() @ self.out_w
        self.target = B.op_sample(logits)
        B.op_tree_accept(self.draft, self.target, self.parent, self.start, self.kv_len, self.table, self.free, self.top, self.path, self.n_acc, self.next, self.acc_info)
        B.op_kv_move(self.pool, self.start, self.path, self.rows[2])

    def guess(self, rng, lens, last):
        """Trees of random guesses whose node 0 is what was said last."""
        start, parent = _forest(int(rng.integers(1 << 30)), lens, 5)
        draft = rng.integers(0, self.V, len(parent))
        for i, t in enumerate(lens):
            if t:
                draft[start[i]] = last[i]
        n = len(parent)
        self.parent[:n] = _i32(parent.tolist())
        self.draft[:n] = _i32(draft.tolist())
        self.new.copy_(_i32(list(lens)))
        return draft

    def stored(self, layer, pages):
        """K and V [tokens, heads, 64] of a list of pages, in 64 bits."""
        if self.fmt:
            codes, scales = _views(self.pool[layer][pages])
            kv = codes.double() * scales.double()[..., None]
        else:
            kv = self.pool[layer][pages].double()
        return kv.permute(1, 0, 3, 2, 4).reshape(2, -1, self.K, 64).cpu().numpy()


def _outputs(loop, tokens, layer, k, v):
    """The layer's attention [tokens, heads * 64] of a stream's tokens over its stored keys, and how far the operators may be off: the queries' rotation
    (4.5 2^-24 of a pair's sizes, which moves every score by at most that times the keys' sizes), and what _bound allows."""
    n, G = len(tokens), loop.H // loop.K
    q = loop.qkv[layer, :, :loop.H * 64].double().cpu().numpy()[tokens].reshape(n, loop.H, 64)
    q, size = _rotated(q, np.arange(n), loop.w, loop.mag, loop.interleaved)
    ref, tol = np.zeros((n, loop.H, 64)), np.zeros((n, loop.H, 64))
    for p in range(n):
        for h in range(loop.K):
            s = slice(h * G, h * G + G)
            o, t = _bound(q[p, s], k[:p + 1, h], v[:p + 1, h], 0.125, HALF[torch.bfloat16])
            d = 0.125 * 4.5 * 2.0 ** -24 * (size[p, s] @ np.abs(k[:p + 1, h]).T).max(-1, keepdims=True)
            ref[p, s], tol[p, s] = o, t + np.expm1(2 * d) * np.abs(v[:p + 1, h]).max(0)
    return ref.reshape(n, -1), tol.reshape(n, -1)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("words,sizes", [(1, [9, 1, 32, 17]), (2, [64, 40, 0, 5])])
def test_drafting_and_accepting(fmt, words, sizes):
    """What the loop says is what its tokens lead to: every token has the highest logit after those before it, up to what the operators' roundings allow; the cache
    holds the accepted tokens' keys at their positions; pages that no stream holds are on the stack."""
    rng = np.random.default_rng(words + fmt)
    loop = Loop(3 + fmt, fmt, 4, 40, sum(sizes) * 2, words, interleaved=bool(fmt))
    told = [[int(t)] for t in rng.integers(0, loop.V, 4)]
    most = 0
    for turn in range(12):
        lens = [s if turn % 3 else max(1, s // 2) if s else turn % 2 for s in sizes]
        loop.guess(rng, lens, [t[-1] for t in told])
        before = loop.kv_len.tolist()
        loop.step()
        assert loop.info[0] == 0 and loop.tree_info[0] == 0 and loop.acc_info[0] == 0
        start, path, acc, nxt, draft = loop.start.tolist(), loop.path.tolist(), loop.n_acc.tolist(), loop.next.tolist(), loop.draft.tolist()
        for i, t in enumerate(lens):
            rows = path[start[i]:start[i] + acc[i]]
            most = max(most, acc[i])
            told[i] += [draft[r] for r in rows[1:]] + ([nxt[i]] if t else [])
            assert loop.kv_len[i] == before[i] + acc[i] == len(told[i]) - 1 and acc[i] >= min(t, 1)
    assert most > 2                            # paths that moved were among them
    held = set()
    for i in range(4):
        n = len(told[i]) - 1
        pages = loop.table[i, :(n + 63) // 64].long()
        held |= set(pages.tolist())
        tokens, logits, slack = np.array(told[i][:n], int), 0.0, 0.0
        for layer in range(loop.LAYERS):
            k, v = (x[:n] for x in loop.stored(layer, pages))
            x = loop.qkv[layer].double().cpu().numpy()[tokens]
            at = loop.H * 64
            want, size = _rotated(x[:, at:at + loop.K * 64].reshape(n, loop.K, 64), np.arange(n), loop.w, loop.mag, loop.interleaved)
            for got, ref, sz in ((k, want, size), (v, x[:, at + loop.K * 64:].reshape(n, loop.K, 64), 0.0)):
                near = 2.0 ** -4 * np.abs(ref) * (1 + 2.0 ** -10) + np.abs(ref).max(-1, keepdims=True, initial=0) / 448 * 2.0 ** -9 if fmt else 2.0 ** -8 * np.abs(ref)
                _close(got, ref, near + 2.0 ** -21 * (sz + np.abs(ref)), "cache")
            o, tol = _outputs(loop, tokens, layer, k, v)
            w = loop.out_w.double().cpu().numpy()[layer * at:(layer + 1) * at]
            logits = logits + o @ w
            # sums of 512 products in fp32, in whatever order
            slack = slack + tol @ np.abs(w) + 512 * 2.0 ** -24 * ((np.abs(o) + tol) @ np.abs(w))
        said = np.array(told[i][1:], int)
        if n:
            best, mine = logits.max(-1), logits[np.arange(n), said]
            assert np.all(mine >= best - 2 * slack.max(-1))
    top = int(loop.top.item())
    assert sorted(loop.free[:top].tolist() + list(held)) == list(range(loop.pages))


@pytest.mark.parametrize("fmt", [0, 1])
def test_steps_captured_and_replayed_beside_others(fmt):
    """Two loops, each captured once with its own scratch and replayed on a stream of its own at the same time, do what plain calls do, bit for bit."""
    def state(loop):
        return [x.clone() for x in (loop.pool.view(torch.uint8), loop.kv_len, loop.table, loop.free, loop.top, loop.path, loop.n_acc, loop.next, loop.target)]

    sizes = [(30, 64, 1), (25, 11, 60)]
    runs = []
    for captured in (False, True):
        loops = [Loop(11 + i, fmt, 3, 30, sum(s), 2) for i, s in enumerate(sizes)]
        rng = np.random.default_rng(5)
        streams, graphs = [torch.cuda.Stream() for _ in loops], []
        if captured:
            for loop, st, s in zip(loops, streams, sizes):
                first = [loop.pool, loop.kv_len, loop.table, loop.free, loop.top]
                kept = [x.clone() for x in first]
                loop.guess(np.random.default_rng(1), s, [0] * 3)
                torch.cuda.synchronize()
                with torch.cuda.stream(st):
                    loop.step()                # warm
                    st.synchronize()
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=st):
                        loop.step()
                    graphs.append(graph)
                    for x, y in zip(first, kept):
                        x.copy_(y)
                torch.cuda.synchronize()
        last = [[1, 2, 3], [4, 5, 6]]
        for turn in range(6):
            for i, loop in enumerate(loops):
                loop.guess(rng, sizes[i], last[i])
            torch.cuda.synchronize()
            for i, loop in enumerate(loops):
                with torch.cuda.stream(streams[i]):
                    graphs[i].replay() if captured else loop.step()
            torch.cuda.synchronize()
            last = [loop.next.tolist() for loop in loops]
        assert all(x[0] == 0 for loop in loops for x in (loop.info, loop.tree_info, loop.acc_info))
        runs.append([state(loop) for loop in loops])
        del graphs
    for a, b in zip(*runs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_on_a_stream_that_is_not_the_current_one():
    """Memory that a call makes for itself belongs to the stream it runs on."""
    st, d = torch.cuda.Stream(), Drafts(1, 0, 4, [30, 7], [500, 900])
    sees = [np.tril(np.ones((t, t), bool)) for t in d.lens]
    q, mask = d.queries(2, 4, torch.float32), _masks(sees, 1)
    args = q, d.pool, _i32(d.table.tolist()), _i32(d.start.tolist()), _i32(d.kv_len.tolist()), mask, 32
    ids, turns = _i32(d.ids.tolist()), B.op_rope_frequencies(64, device=DEV)[0]
    pool, slot = _empty_pool(0, 2, 4), torch.arange(d.R, dtype=torch.int32, device=DEV)
    want = B.op_attention_tree(*args, stream_ids=ids).clone(), B.op_rope_kv_append(q, q, q, pool, slot, slot, turns).clone()
    torch.cuda.synchronize()
    for _ in range(5):
        st.wait_stream(torch.cuda.current_stream())
        got = B.op_attention_tree(*args, stream_ids=ids, stream=st), B.op_rope_kv_append(q, q, q, pool, slot, slot, turns, stream=st)
        junk = [torch.full((1 << 22,), 3.0, device=DEV) for _ in range(4)]      # what the current stream allocates meanwhile
        st.synchronize()
        n = sum(d.lens)
        assert torch.equal(got[0][:n], want[0][:n]) and torch.equal(got[1][:n], want[1][:n])
        del junk


# ---------------------------------------------------------------------------------------------
# forms of the arguments
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,K", [(12, 4), (0, 12), (40, 40)])
@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_rot,interleaved", [(64, False), (30, False), (62, True)])
@pytest.mark.parametrize("fmt", [0, 1])
def test_rope_of_a_large_pass_is_that_of_its_parts(fmt, n_rot, interleaved, src, H, K):
    """More rows than CTAs of the other size have place for: bit for bit what calls of 100 rows give."""
    g, rows = _gen(n_rot + H), 30000 // (H + 2 * K) * 2 + 77
    pages = (rows + 63) // 64 + 1
    q, k, v = torch.randn(rows, (H + 2 * K) * 64, generator=g).to(src).to(DEV).split([H * 64, K * 64, K * 64], 1)
    slot = torch.randperm(pages * 64, generator=g)[:rows].to(torch.int32)
    slot[::17] = -1
    slot, pos = slot.to(DEV), torch.randint(-10 ** 6, 10 ** 6, (rows,), generator=g, dtype=torch.int32).to(DEV)
    turns, _ = B.op_rope_frequencies(n_rot, device=DEV)
    pools, outs = [_empty_pool(fmt, pages, K) for _ in range(2)], [torch.full((rows, H * 64), 5.0, dtype=src, device=DEV) if H else None for _ in range(2)]
    for pool, out, step in zip(pools, outs, (rows, 100)):
        for i in range(0, rows, step):
            s = slice(i, i + step)
            B.op_rope_kv_append(q[s] if H else None, k[s], v[s], pool, slot[s], pos[s], turns, interleaved=interleaved, q_out=out[s] if H else None)
    assert torch.equal(pools[0].view(torch.uint8), pools[1].view(torch.uint8))
    assert not H or torch.equal(outs[0], outs[1]) and torch.all(outs[0][::17] == 5.0) and not torch.any((outs[0] == 5.0).all(-1)[torch.arange(rows) % 17 != 0])


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n_rot", [64, 30])
@pytest.mark.parametrize("fmt", [0, 1])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(fmt, n_rot, interleaved, src):
    """A chain of six nodes behind nothing: from the node on whose key or value is not finite, the head's rows are NaN, and no others."""
    x = torch.randn(6, 3 * 128, generator=_gen(4)).to(src).to(DEV)
    q, k, v = x.split(128, 1)
    k[3, 64 + 17], v[1, 5], v[4, 64 + 60] = float("nan"), float("nan"), float("inf")
    pool, table = _empty_pool(fmt, 2, 2), _i32([[1]])
    slot, pos = torch.arange(64, 70, dtype=torch.int32, device=DEV), torch.arange(6, dtype=torch.int32, device=DEV)
    q_out = B.op_rope_kv_append(q, k, v, pool, slot, pos, B.op_rope_frequencies(n_rot, device=DEV)[0], interleaved=interleaved)
    out = B.op_attention_tree(q_out, pool, table, _i32([0, 6]), _i32([6]), _masks([np.tril(np.ones((6, 6), bool))], 1, extra=0), 6).view(6, 2, 64)
    bad = torch.isnan(out)
    for head, first in ((0, 1), (1, 3)):
        assert not bad[:first, head].any() and bad[first:, head].all()


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,K,lens,ctx", [(4, 4, [20, 31], [70, 200]), (6, 2, [20, 9], [130, 64]), (2, 2, [100, 3], [0, 300]), (3, 3, [1], [90])])
def test_attention_of_rows_of_a_wider_array(fmt, dtype, H, K, lens, ctx):
    d = Drafts(13, fmt, K, lens, ctx, extra=0 if len(lens) == 1 else 2)
    sees = [np.tril(np.ones((t, t), bool)) for t in lens]
    q = d.queries(3, H, dtype)
    wide = torch.full((d.R, H * 64 + 8 * 5), float("nan"), dtype=dtype, device=DEV)
    wide[:, 16:16 + H * 64] = q
    mask = _masks(sees, (max(lens) + 31) // 32, extra=d.R - sum(lens))
    out = d.run(wide[:, 16:16 + H * 64], mask, scale=0.3)
    d.check(out, q, sees, scale=0.3)
    assert torch.equal(out.view(torch.int16), d.run(q, mask, scale=0.3).view(torch.int16))


@pytest.mark.parametrize("fmt", [0, 1])
def test_pages_and_streams_that_are_none(fmt):
    """Keys on pages outside the pool, and behind the list's pages, are left out; a stream that is none has no keys."""
    lens, ctx = [10, 20, 30, 9], [200, 300, 130, 100]
    d = Drafts(21, fmt, 2, lens, ctx, pps=4)
    sees = [np.tril(np.ones((t, t), bool)) for t in lens]
    d.table[d.ids[0], 1], d.table[d.ids[2], 0], d.table[d.ids[2], 2] = -1, d.pages, -2 ** 31
    q = d.queries(3, 4, torch.bfloat16)
    ids = d.ids.copy()
    ids[3] = 4
    args = q, d.pool, _i32(d.table.tolist()), _i32(d.start.tolist()), _i32(d.kv_len.tolist()), _masks(sees, 1), 32
    out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device=DEV)
    B.op_attention_tree(*args, stream_ids=_i32(ids.tolist()), out=out)
    got = out.double().cpu().numpy().reshape(d.R, 4, 64)
    qn = q.double().cpu().numpy().reshape(d.R, 4, 64)
    for i, t in enumerate(lens):
        n = ctx[i] + t
        where = np.arange(n)
        held = (where < 4 * 64) & ~np.isin(where // 64, {0: [1], 2: [0, 2]}.get(i, []))
        pages = np.concatenate([d.table[d.ids[i]], [0]])[:(n + 63) // 64]
        pages[(pages < 0) | (pages >= d.pages)] = 0
        k, v = (d.kv[pages, x].transpose(0, 2, 1, 3).reshape(-1, 2, 64)[:n] for x in (0, 1))
        for r in range(t):
            on = held & np.concatenate([np.ones(ctx[i], bool), sees[i][r]]) & (i != 3)
            for h in range(2):
                s = slice(2 * h, 2 * h + 2)
                ref, tol = _bound(qn[d.start[i] + r, s], k[on, h], v[on, h], 0.125, HALF[torch.bfloat16])
                _close(got[d.start[i] + r, s], ref, tol, (i, r))
    assert torch.all(out[d.start[-1]:] == 9.0)


@pytest.mark.parametrize("fmt", [0, 1])
def test_streams_that_hold_fewer_tokens_than_the_tree_has_nodes(fmt):
    """The nodes are the last tokens of the stream: of 20 nodes and 15 tokens, the first 5 have no key.  Lengths of zero and below: none has."""
    lens = [20, 8, 6]
    d = Drafts(5, fmt, 1, lens, [0, 0, 0])
    kv = d.kv_len.copy()
    kv[d.ids[0]], kv[d.ids[1]], kv[d.ids[2]] = 15, 0, -7
    mask = _masks([np.tril(np.ones((t, t), bool)) for t in lens], 1)
    q = d.queries(3, 1, torch.bfloat16)
    d.kv_len = kv
    out = d.run(q, mask)
    k, v = d.keys_of(0)
    for r in range(20):
        n = max(0, r - 4)
        ref, tol = _bound(q[r:r + 1].double().cpu().numpy(), k[:n, 0], v[:n, 0], 0.125, HALF[torch.bfloat16])
        _close(out[r:r + 1].double().cpu().numpy(), ref, tol, r)
    assert not out[20:34].any() and torch.all(out[34:] == 9.0)


@pytest.mark.parametrize("t_max", [5, 40])
def test_rows_beyond_t_max_are_left(t_max):
    lens = [20, 64, 4]
    d = Drafts(6, 0, 2, lens, [100, 10, 300])
    sees = [np.tril(np.ones((t, t), bool)) for t in lens]
    q = d.queries(3, 2, torch.float32)
    out = d.run(q, _masks(sees, 2), t_max=t_max)
    whole = d.run(q, _masks(sees, 2))
    d.check(whole, q, sees)
    left = np.concatenate([np.arange(t) >= t_max for t in lens] + [np.ones(2, bool)])
    assert torch.all(out[torch.tensor(left)] == 9.0)
    d.check(out, q, sees, rows=np.flatnonzero(~left))


@pytest.mark.parametrize("start", [[0, 5, 3, 9], [0, 4, 8, 40], [-1, 4, 8, 9]])
def test_attention_writes_nothing_where_starts_do_not_ascend(start):
    d = Drafts(6, 0, 2, [3, 3, 3], [100, 10, 300])
    q, out = d.queries(3, 2, torch.float32), torch.full((d.R, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    B.op_attention_tree(q, d.pool, _i32(d.table.tolist()), _i32(start), _i32(d.kv_len.tolist()), torch.full((d.R, 1), -1, dtype=torch.int32, device=DEV), 8, out=out)
    assert torch.all(out == 9.0)


@pytest.mark.parametrize("fmt,t", [(0, 1), (1, 3)])
def test_the_largest_number_of_trees(fmt, t):
    n = 2048
    d = Drafts(6, fmt, 1, [t if i % 5 else 0 for i in range(n)], [i % 90 for i in range(n)])
    sees = [np.tril(np.ones((x, x), bool)) for x in d.lens]
    q = d.queries(3, 2, torch.bfloat16)
    d.check(d.run(q, _masks(sees, 1)), q, sees)


def test_two_trees_of_one_stream():
    """Nothing forbids it: both see the same last tokens as their nodes."""
    d = Drafts(6, 0, 2, [6], [100], extra=8)
    tri = np.tril(np.ones((6, 6), bool))
    q = torch.randn(14, 128, generator=_gen(1)).to(DEV)
    q[6:12] = q[:6]
    out = torch.full((14, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    B.op_attention_tree(q, d.pool, _i32(d.table.tolist()), _i32([0, 6, 12]), _i32(d.kv_len.tolist()), _masks([tri, tri], 1), 6, stream_ids=_i32([0, 0]), out=out)
    assert torch.equal(out[:6], out[6:12]) and torch.isfinite(out[:6]).all() and torch.all(out[12:] == 9.0)


@pytest.mark.parametrize("fmt", [0, 1])
def test_a_pool_of_more_than_four_gigabytes(fmt):
    """Pages whose offsets do not fit 32 bits: a tree written, read and moved at the end of the pool gives what it gives at the start of a small one."""
    H = K = 20
    page = 2 * K * (E4M3_BLOCK if fmt else 8192)
    pages = (1 << 32) // page + 70
    g = _gen(9)
    x = torch.randn(70, 3 * H * 64, generator=g).to(DEV)
    q, k, v = x.split(H * 64, 1)
    turns, _ = B.op_rope_frequencies(64, device=DEV)
    pos = torch.arange(70, dtype=torch.int32, device=DEV)
    mask, start, kv_len = _masks([np.tril(np.ones((70, 70), bool))], 3, extra=0), _i32([0, 70]), _i32([70])
    path = _i32([0, 3, 9, 33, 68] + [-1] * 65)
    got = []
    for n in (5, pages):
        shape = (n, 2, K, E4M3_BLOCK) if fmt else (n, 2, K, 64, 64)
        pool = torch.empty(shape, dtype=torch.uint8 if fmt else torch.bfloat16, device=DEV)
        table = _i32([[n - 1, n - 3]])
        slot = torch.cat([torch.arange(64) + 64 * (n - 1), torch.arange(6) + 64 * (n - 3)]).to(torch.int32).to(DEV)
        q_out = torch.empty(70, H * 64, device=DEV)
        B.op_rope_kv_append(q, k, v, pool, slot, pos, turns, q_out=q_out)
        out = B.op_attention_tree(q_out, pool, table, start, kv_len, mask, 70)
        B.op_kv_move(pool, start, path, slot)
        again = B.op_attention_tree(q_out[:5], pool, table, _i32([0, 5]), _i32([5]), mask[:5].contiguous(), 5)
        got.append((q_out, out, again, pool[n - 1, :, :, :E4M3_BLOCK].clone()))
        if fmt:
            assert torch.isfinite(_views(pool[n - 1])[1]).all()
        del pool
    assert all(torch.equal(a, b) for a, b in zip(*got)) and torch.isfinite(got[0][1]).all()


# ---------------------------------------------------------------------------------------------
# waits that run out
# ---------------------------------------------------------------------------------------------
def _expire_call(fmt, H, K, dtype, lens, ctx):
    d = Drafts(31, fmt, K, lens, ctx)
    sees = [np.tril(np.ones((t, t), bool)) for t in lens]
    q, mask = d.queries(3, H, dtype), _masks(sees, (max(lens) + 31) // 32)
    rows = torch.arange(d.R, device=DEV) < int(d.start[-1])
    return (lambda **kw: d.run(q, mask, **kw)), B.op_attention_tree_scratch(DEV), rows


EXPIRE = {  # every CTA of the first two has pages to read
    "one tree": (0, 20, 20, torch.float32, [8], [2000]), "8-bit, grouped": (1, 20, 4, torch.bfloat16, [20, 9, 25], [1500, 1900, 700]),
    "64 rows": (0, 20, 20, torch.bfloat16, [64, 50, 1, 60], [500, 900, 40, 1000]), "128 rows": (0, 4, 4, torch.bfloat16, [128, 200, 90], [1500, 700, 900]),
    "128 rows, 8-bit": (1, 8, 4, torch.float32, [100, 70, 128], [1500, 900, 1100]), "many trees": (0, 4, 4, torch.bfloat16, [3] * 300, [200] * 300)}


@pytest.mark.parametrize("name", EXPIRE)
def test_a_scratch_of_a_failed_call_gives_nan_until_it_is_zeroed(name):
    call, scratch, rows = _expire_call(*EXPIRE[name])
    want = call(scratch=scratch).clone()
    scratch[:4].view(torch.int32).fill_(1)
    got = call(scratch=scratch)
    assert bool(torch.isnan(got[rows]).all()) and torch.equal(got[~rows], want[~rows])
    assert int(scratch[:4].view(torch.int32)) == 1
    scratch.zero_()
    assert torch.equal(call(scratch=scratch), want)


@pytest.mark.parametrize("cta", [0, 5])
@pytest.mark.parametrize("name", EXPIRE)
def test_rows_behind_an_expired_wait_are_nan(name, cta):
    """The copies of one CTA never count as complete: the call ends, says so in its scratch, and every head of a row is whole or NaN."""
    call, scratch, rows = _expire_call(*EXPIRE[name])
    want = call(scratch=scratch).clone()
    try:
        B.debug_expire_op(cta, 20000)
        got = [call(scratch=scratch).clone(), call().clone()]
    finally:
        B.debug_expire_op(-1)
    assert int(scratch[:4].view(torch.int32)) == 1
    for y in got:
        lost = torch.isnan(y).view(y.shape[0], -1, 64).all(-1)
        assert bool(lost[rows].any()) and not bool(lost[~rows].any())
        assert torch.equal(y.view(y.shape[0], -1, 64)[~lost], want.view(y.shape[0], -1, 64)[~lost])
    assert bool(torch.isnan(call(scratch=scratch)[rows]).all())
    scratch.zero_()
    assert torch.equal(call(scratch=scratch), want) and torch.equal(call()[rows], want[rows])


def test_one_scratch_serves_the_attentions_by_turns():
    call, scratch, rows = _expire_call(*EXPIRE["64 rows"])
    other, _, _ = _expire_call(*EXPIRE["8-bit, grouped"])
    x = torch.randn(300, 4, 64, generator=_gen(2)).bfloat16().to(DEV)
    big = B.op_attention_cross_scratch(DEV)
    big = big if big.numel() >= scratch.numel() else scratch
    cross = lambda: B.op_attention_cross(x, x, x, _i32([0, 100, 300]), _i32([0, 170, 300]), 200, scratch=big)  # noqa: E731
    want = call().clone(), other().clone(), cross().clone()
    for _ in range(3):
        assert torch.equal(call(scratch=big), want[0]) and torch.equal(cross(), want[2]) and torch.equal(other(scratch=big), want[1])
