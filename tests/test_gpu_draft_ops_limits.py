"""The draft operators where short things follow one another and where long ones end.  Tolerances as in test_gpu_draft_ops."""
import numpy as np
import pytest
import torch

from paper_2607_21042_b200 import binding as B
from test_gpu_draft_ops import Drafts, _forest, _masks, _sees
from test_gpu_serving_ops import HALF, _bound, _check

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
