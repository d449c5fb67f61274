"""Operators of a program that decodes several drafted tokens a step from the paged cache: which cases are timed.

A draft is a tree: node 0 is the token that the stream has sampled last, every other node a guess at what follows its parent.
One step runs all nodes of all requests through the model at once and keeps the path on which the model agrees:

  rope     a pass's queries and keys rotated by their positions, keys and values into their slots (``op_rope_kv_append``)
  tables   the nodes' ancestors as bit masks, and their positions, from the parents (``op_tree_tables``)
  attend   attention of the nodes to what the stream holds and to their ancestors (``op_attention_tree``)
  accept   the path that the model agrees with; lengths and unused pages go back (``op_tree_accept``)
  move     keys and values of that path to where the stream's next tokens belong, in all layers (``op_kv_move``)

Sizes are those of the decode engine (20 heads of 64, pages of 64 tokens, contexts up to 2048, 24 layers, up to 128 streams, passes
of up to 3584 rows) and of the ranges around them.
"""
from __future__ import annotations

import math
import random

import torch

DEV = "cuda"
PAGE, HD = 64, 64
PPS = 32                       # pages a stream may hold: contexts up to 2048
VOCAB = 8194
E4M3_MAX = 448.0
E4M3_BLOCK = PAGE * HD + 4 * PAGE   # codes and fp32 scales of one (page, K|V, head) block
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

own = False


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def _rope(name, rows, heads, kv_heads, src, q_out, cache, fused, pad, rot, order, scaling, pos_hi):
    """`fused`: q, k and v are parts of one array.  The last `pad` rows belong to no slot.  `rot` values of a head are rotated, in pairs
    of neighbours or of halves (`order`)."""
    c = {"op": "rope", "rows": rows, "heads": heads, "kv_heads": kv_heads, "src": src, "q_out": q_out, "cache": cache, "fused": fused, "pad": pad, "rot": rot,
         "order": order, "scaling": scaling, "pos_hi": pos_hi}
    return dict(c, name=name) if name else c


def _tables(name, n, nodes, reach):
    """n trees of nodes[0]..nodes[1] nodes; a node's parent is one of the `reach` before it (1: a chain)."""
    c = {"op": "tables", "n": n, "t_lo": nodes[0], "t_hi": nodes[1], "reach": reach}
    return dict(c, name=name) if name else c


def _attend(name, n, nodes, reach, heads, kv_heads, q, cache, ctx):
    c = {"op": "attend", "n": n, "t_lo": nodes[0], "t_hi": nodes[1], "reach": reach, "heads": heads, "kv_heads": kv_heads, "q": q, "cache": cache, "ctx_lo": ctx[0],
         "ctx_hi": ctx[1]}
    return dict(c, name=name) if name else c


def _accept(name, n, nodes, reach, agree):
    """`agree`: per cent of the drafted tokens that are what the model says after their parent."""
    c = {"op": "accept", "n": n, "t_lo": nodes[0], "t_hi": nodes[1], "reach": reach, "agree": agree}
    return dict(c, name=name) if name else c


def _move(name, n, nodes, layers, kv_heads, cache):
    c = {"op": "move", "n": n, "t_lo": nodes[0], "t_hi": nodes[1], "layers": layers, "kv_heads": kv_heads, "cache": cache}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the decode step of a small server, straight from the fp32 output of the QKV linear
        _rope("rope_f32_r16", 16, 20, 20, "f32", "f32", "bf16", True, 0, 64, "half", "none", 2048),
        # the rows of a prefill pass of 3584 rows, queries rounded for the tensor cores
        _rope("rope_f32_r3584", 3584, 20, 20, "f32", "bf16", "bf16", True, 0, 64, "half", "none", 2048),
        # grouped heads, half of each rotated, positions far beyond the trained ones, 8-bit cache, padded to a captured size
        _rope("rope_gqa_r777_e4m3", 777, 20, 4, "bf16", "bf16", "e4m3", False, 40, 32, "neighbours", "yarn", 200000),
        # a small server's drafts of one step
        _tables("tables_n16_t40", 16, (24, 40), 8),
        # a full server's
        _tables("tables_n128_t200", 128, (100, 200), 20),
        # one speaker, eight drafted tokens early in the answer
        _attend("attend_n1_t8", 1, (8, 8), 1, 20, 20, "f32", "bf16", (333, 333)),
        # sixteen requests, each with a tree of up to 64 nodes
        _attend("attend_n16_t64", 16, (48, 64), 12, 20, 20, "bf16", "bf16", (150, 1900)),
        # a full server with grouped heads and the 8-bit cache, small trees of all sizes
        _attend("attend_gqa_n128_t25_e4m3", 128, (5, 25), 6, 20, 4, "bf16", "e4m3", (60, 1900)),
        _accept("accept_n16_t40", 16, (24, 40), 8, 70),
        _accept("accept_n128_t200", 128, (100, 200), 20, 70),
        # one layer, right behind its attention
        _move("move_n16_l1", 16, (24, 40), 1, 20, "bf16"),
        # all layers of the model at the end of the step
        _move("move_n32_l24", 32, (24, 64), 24, 20, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = [(c["op"], work(c)) for c in listed()]
    while True:
        c = _draw(rng)
        w = work(c)
        if all(w[k] <= max(t[k] for o, t in top if o == c["op"]) for k in ("bytes", "flops")):
            return c


def _draw(rng):
    op = rng.choice(["rope", "rope", "tables", "attend", "attend", "attend", "accept", "move"])
    heads, kv = rng.choice([(20, 20), (20, 20), (4, 4), (20, 4), (16, 4), (12, 4), (16, 1)])
    cache = rng.choice(["bf16", "bf16", "e4m3"])
    if op == "rope":
        rows = _log(rng, 1, 3584)
        return _rope(None, rows, heads, kv, rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"]), cache, rng.random() < 0.5, rng.choice([0, rng.randint(0, rows - 1)]),
                     rng.choice([64, 64, 2 * rng.randint(1, 32)]), rng.choice(["half", "neighbours"]), rng.choice(["none", "linear", "yarn"]), _log(rng, 1, 1 << 20))
    if op in ("tables", "accept"):
        t = _log(rng, 1, 256)
        n, lo, reach = _log(rng, 1, 300), rng.randint(1, t), _log(rng, 1, 64)
        return _tables(None, n, (lo, t), reach) if op == "tables" else _accept(None, n, (lo, t), reach, rng.randint(0, 100))
    if op == "attend":
        t = rng.choice([_log(rng, 1, 32), _log(rng, 1, 128), _log(rng, 64, 256)])
        hi = _log(rng, 1, PPS * PAGE - t)
        return _attend(None, _log(rng, 1, 160), (rng.randint(1, t), t), _log(rng, 1, 32), heads, kv, rng.choice(["f32", "bf16"]), cache, (rng.randint(0, hi), hi))
    t = _log(rng, 1, 128)
    return _move(None, _log(rng, 1, 128), (rng.randint(1, t), t), _log(rng, 1, 24), kv, cache)


def _spread(n, lo, hi):
    """n whole numbers from lo to hi, evenly spread: their sum is the case's, only their order the seed's."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [(lo + hi) // 2] * n


def _pages(tokens):
    return -(-tokens // PAGE)


def _token_bytes(case):
    """K and V of a token, in one layer."""
    return case["kv_heads"] * 2 * (2 * HD if case["cache"] == "bf16" else HD + 4)


def work(case):
    op = case["op"]
    if op == "rope":
        rows, size = case["rows"] - case["pad"], {"f32": 4, "bf16": 2}
        values = (case["heads"] + 2 * case["kv_heads"]) * HD
        return {"bytes": rows * (values * size[case["src"]] + case["heads"] * HD * size[case["q_out"]] + _token_bytes(case)) + 8 * case["rows"] + 4 * case["rot"],
                "flops": 3 * rows * (case["heads"] + case["kv_heads"]) * case["rot"]}
    lens = _spread(case["n"], case["t_lo"], case["t_hi"])
    rows, words = sum(lens), -(-max(lens) // 32)
    if op == "tables":
        return {"bytes": rows * (4 + 4 + 4 * words) + 12 * case["n"], "flops": 0}
    if op == "attend":
        ctx = _spread(case["n"], case["ctx_lo"], case["ctx_hi"])
        keys = [c + t for c, t in zip(ctx, lens)]
        return {"bytes": _token_bytes(case) * sum(keys) + rows * (case["heads"] * HD * ((4 if case["q"] == "f32" else 2) + 2) + 4 * words) + 4 * sum(_pages(k) for k in keys),
                "flops": 4 * HD * case["heads"] * sum(t * k for t, k in zip(lens, keys))}
    if op == "accept":
        return {"bytes": rows * (4 + 4 + 4 + 4) + 24 * case["n"], "flops": 0}
    count = [(t + 5) // 6 for t in lens]               # nodes of the paths, a third of which stay where they are: see prepare
    return {"bytes": 2 * case["layers"] * _token_bytes(case) * sum(c - (c + 2) // 3 for c in count) + 8 * rows, "flops": 0}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _normal(gen, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32) * std).to(dtype)


def _e4m3(x):
    """Values [..., 64] as e4m3 codes and one fp32 scale for each 64."""
    s = x.abs().amax(-1) / E4M3_MAX
    s = torch.where(s > 0, s, torch.ones_like(s))
    return (x / s[..., None]).to(torch.float8_e4m3fn), s


def _e4m3_views(pool):
    """The codes [..., pages, 2, heads, 64, 64] (bytes) and the scales [..., pages, 2, heads, 64] inside the pool."""
    return pool[..., :PAGE * HD].unflatten(-1, (PAGE, HD)), pool[..., PAGE * HD:].view(torch.float32)


def _pool(gen, cache, n_pages, heads, *layers):
    """Pages filled with keys and values, of one layer or of several."""
    if cache == "bf16":
        return torch.randn(*layers, n_pages, 2, heads, PAGE, HD, generator=gen, device=DEV, dtype=torch.bfloat16)
    pool = torch.empty(*layers, n_pages, 2, heads, E4M3_BLOCK, dtype=torch.uint8, device=DEV)
    c, s = _e4m3(_normal(gen, *layers, n_pages, 2, heads, PAGE, HD))
    codes, scales = _e4m3_views(pool)
    codes.copy_(c.view(torch.uint8))
    scales.copy_(s)
    return pool


def _pool_out(s):
    if s["case"]["cache"] == "bf16":
        return {"pool": s["pool"]}
    codes, scales = _e4m3_views(s["pool"])
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales}


def _inv_freq(rot, scaling):
    """Radians a position, and what cosine and sine are multiplied by: with ``linear`` positions are divided by 8; ``yarn`` divides
    slow pairs by 40, which turn less than once in the 4096 trained positions, leaves those that turn more than 32 times, and blends between."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    f = 10000.0 ** (-2.0 * i / rot)
    if scaling == "linear":
        return f / 8.0, 1.0
    if scaling == "none":
        return f, 1.0
    where = lambda turns: rot * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))  # noqa: E731
    low, high = max(math.floor(where(32.0)), 0), min(math.ceil(where(1.0)), rot - 1)
    ramp = ((i - low) / max(high - low, 0.001)).clamp(0, 1)
    return f / 40.0 * ramp + f * (1 - ramp), 0.1 * math.log(40.0) + 1.0


def _trees(case, gen, rng, extra=3):
    """Ragged trees: row starts, parents (inside their tree), the rows' trees and places in them; a few rows behind the last."""
    lens = _spread(case["n"], case["t_lo"], case["t_hi"])
    rng.shuffle(lens)
    starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
    R = starts[-1] + extra
    seq = torch.repeat_interleave(torch.arange(case["n"], device=DEV), torch.tensor(lens, device=DEV), output_size=starts[-1])
    at = torch.arange(starts[-1], device=DEV) - torch.tensor(starts, device=DEV)[seq]
    back = (torch.rand(starts[-1], generator=gen, device=DEV) * at.clamp(max=case["reach"])).long() if case.get("reach") else torch.zeros_like(at)
    parent = torch.full((R,), -7, dtype=torch.int32, device=DEV)
    parent[:starts[-1]] = (at - 1 - back).int()
    return {"lens": lens, "R": R, "row_start": _ints(starts), "parent": parent, "seq": seq, "at": at}


def _lists(rng, gen, lens, pps):
    """Page lists of streams that hold `lens` tokens, in a pool of no more pages than needed and three."""
    held = [_pages(t) for t in lens]
    pages = torch.randperm(sum(held) + 3, generator=gen, device=DEV, dtype=torch.int32).cpu()
    table, at = torch.zeros(len(lens), pps, dtype=torch.int32), 0
    for i, h in enumerate(held):
        table[i, :h] = pages[at:at + h]
        at += h
    return table.to(DEV), sum(held) + 3, pages[at:]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    op = case["op"]
    s = {"op": op, "case": case}
    if op == "rope":
        rows, H, K = case["rows"], case["heads"], case["kv_heads"]
        n_pages = _pages(rows) + 3
        slot = torch.randperm(n_pages * PAGE, generator=gen, device=DEV, dtype=torch.int32)[:rows].clone()
        if case["pad"]:
            slot[rows - case["pad"]:] = -1
        t = TYPES[case["src"]]
        x = _normal(gen, rows, (H + 2 * K) * HD, dtype=t)
        q, k, v = x.split([H * HD, K * HD, K * HD], 1)
        if not case["fused"]:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        inv, mag = _inv_freq(case["rot"], case["scaling"])
        s.update(q=q, k=k, v=v, pool=_pool(gen, case["cache"], n_pages, K), slot=slot, pos=torch.randint(0, case["pos_hi"], (rows,), generator=gen, device=DEV, dtype=torch.int32),
                 inv_freq=inv.to(DEV), magnitude=mag, q_out=torch.zeros(rows, H * HD, dtype=TYPES[case["q_out"]], device=DEV))
        return s
    n = case["n"]
    s.update(_trees(case, gen, rng))
    s["t_max"] = max(s["lens"])
    s["words"] = -(-s["t_max"] // 32)
    streams = rng.sample(range(n), n)
    s["ids"] = _ints(streams)
    if op == "move":
        # the path has a sixth of the nodes, of which the first third lies where it belongs and the others farther on
        table, n_pages, _ = _lists(rng, gen, [40 + t for t in s["lens"]], PPS)
        path = torch.full((s["R"],), -1, dtype=torch.int32, device=DEV)
        count = (torch.tensor(s["lens"], device=DEV)[s["seq"]] + 5) // 6
        node = torch.where(s["at"] < (count + 2) // 3, s["at"], 2 * s["at"] + 1)
        path[:s["seq"].numel()] = torch.where(s["at"] < count, s["row_start"].long()[:-1][s["seq"]] + node, torch.full_like(node, -1)).int()
        pos = 40 + s["at"]
        slot = torch.full((s["R"],), -1, dtype=torch.int32, device=DEV)
        slot[:s["seq"].numel()] = (table.long()[s["seq"], pos // PAGE] * PAGE + pos % PAGE).int()
        s.update(pool=_pool(gen, case["cache"], n_pages, case["kv_heads"], case["layers"]), path=path, row_slot=slot)
        return s
    if op == "attend":
        ctx = _spread(n, case["ctx_lo"], case["ctx_hi"])
        rng.shuffle(ctx)
    else:
        ctx = [rng.randint(70, 1700) for _ in range(n)]
    kv_len = [0] * n
    for i in range(n):
        kv_len[streams[i]] = ctx[i] + s["lens"][i]
    s["kv_len"] = _ints(kv_len)
    if op == "tables":
        s.update(mask=torch.full((s["R"], s["words"]), -1, dtype=torch.int32, device=DEV), row_pos=torch.full((s["R"],), -1, dtype=torch.int32, device=DEV), info=_ints([0] * 8))
        return s
    s["table"], n_pages, left = _lists(rng, gen, kv_len, PPS)
    if op == "attend":
        s["mask"], _ = _ancestors(s)
        s["keys_max"] = max(kv_len)
        s.update(q=_normal(gen, s["R"], case["heads"] * HD, dtype=TYPES[case["q"]], std=2.0), pool=_pool(gen, case["cache"], n_pages, case["kv_heads"]),
                 out=torch.zeros(s["R"], case["heads"] * HD, dtype=torch.bfloat16, device=DEV))
        return s
    rows = s["seq"].numel()
    free = torch.zeros(n * PPS + 3, dtype=torch.int32, device=DEV)        # a place for every page there may be
    free[:left.numel()] = left.to(DEV)
    target = torch.randint(0, VOCAB, (s["R"],), generator=gen, device=DEV, dtype=torch.int32)
    draft = torch.randint(0, VOCAB, (s["R"],), generator=gen, device=DEV, dtype=torch.int32)
    up = (s["row_start"].long()[:-1][s["seq"]] + s["parent"][:rows].clamp(min=0)).long()
    agree = torch.rand(rows, generator=gen, device=DEV) * 100 < case["agree"]
    draft[:rows] = torch.where(agree, target[up], draft[:rows])
    s.update(draft=draft, target=target, free=free, top=_ints([left.numel()]), kv_len_out=s["kv_len"].clone(), top_out=_ints([0]), path=torch.full((s["R"],), -9, dtype=torch.int32, device=DEV),
             n_accepted=_ints([0] * n), next_token=_ints([0] * n), info=_ints([0] * 8))
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)[state["op"]](state)


def _rotate(x, cos, sin, rot, order):
    """x [rows, heads, 64]; cos, sin [rows, rot / 2]."""
    cos, sin = cos[:, None], sin[:, None]
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if order == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.cat([a, b], -1) if order == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_rope(s):
    c = s["case"]
    H, K = c["heads"], c["kv_heads"]
    angle = s["pos"].double()[:, None] * s["inv_freq"]            # far positions: 64 bits
    cos, sin = (torch.cos(angle) * s["magnitude"]).float(), (torch.sin(angle) * s["magnitude"]).float()
    q, k = (_rotate(x.float().reshape(-1, h, HD), cos, sin, c["rot"], c["order"]) for x, h in ((s["q"], H), (s["k"], K)))
    v = s["v"].float().reshape(-1, K, HD)
    # a row without a slot goes where row 0 goes, with its values (row 0 always has one), and has no queries
    slot = s["slot"].long()
    there = slot >= 0
    slot = torch.where(there, slot, slot[:1])
    page, off = slot // PAGE, slot % PAGE
    k, v = torch.where(there[:, None, None], k, k[:1]), torch.where(there[:, None, None], v, v[:1])
    q_out = torch.where(there[:, None], q.reshape(-1, H * HD).to(s["q_out"].dtype), s["q_out"])
    if c["cache"] == "bf16":
        s["pool"][page, 0, :, off] = k.bfloat16()
        s["pool"][page, 1, :, off] = v.bfloat16()
    else:
        codes, scales = _e4m3_views(s["pool"])
        kc, ks = _e4m3(k)
        vc, vs = _e4m3(v)
        codes[page, 0, :, off] = kc.view(torch.uint8)
        codes[page, 1, :, off] = vc.view(torch.uint8)
        scales[page, 0, :, off] = ks
        scales[page, 1, :, off] = vs
    return {"q": q_out, **_pool_out(s)}


def _own_rope(s):
    from paper_2607_21042_b200 import binding as B
    c = s["case"]
    if "turns" not in s:
        more = {"none": {}, "linear": {"factor": 8.0}, "yarn": {"factor": 40.0, "original": 4096}}[c["scaling"]]
        s["turns"], s["mag"] = B.op_rope_frequencies(c["rot"], base=10000.0, scaling=c["scaling"], device=s["q"].device, **more)
    B.op_rope_kv_append(s["q"], s["k"], s["v"], s["pool"], s["slot"], s["pos"], s["turns"], magnitude=s["mag"], interleaved=c["order"] == "neighbours", q_out=s["q_out"])
    return {"q": s["q_out"], **_pool_out(s)}


def _padded(s):
    """Rows of tree i's nodes [n, t_max], which of them exist, and the parents there (-1 where none)."""
    start = s["row_start"].long()
    j = torch.arange(s["t_max"], device=DEV)
    ok = j < (start[1:] - start[:-1])[:, None]
    rows = torch.where(ok, start[:-1, None] + j, torch.zeros_like(start[:1]))
    return rows, ok, torch.where(ok, s["parent"].long()[rows], torch.full_like(rows, -1))


def _closure(parent):
    """[n, t, t]: 1 where the second node is the first one or one of its ancestors."""
    t = parent.shape[1]
    m = (parent[:, :, None] == torch.arange(t, device=DEV)).float() + torch.eye(t, device=DEV)
    for _ in range(max(t - 1, 1).bit_length()):        # paths of twice the length each time
        m = (torch.bmm(m, m) > 0).float()
    return m


def _ancestors(s):
    """The masks [R, words] and the depths [R] of all rows; of rows of no tree: -1."""
    rows, ok, parent = _padded(s)
    m = _closure(parent)
    n, t = rows.shape
    bits = (torch.nn.functional.pad(m, (0, 32 * s["words"] - t)).long().view(n, t, s["words"], 32) << torch.arange(32, device=DEV)).sum(-1)
    bits = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()
    mask = torch.full((s["R"], s["words"]), -1, dtype=torch.int32, device=DEV)
    depth = torch.full((s["R"],), -1, dtype=torch.int64, device=DEV)
    mask[:s["seq"].numel()] = bits[s["seq"], s["at"]]
    depth[:s["seq"].numel()] = (m.sum(-1).long() - 1)[s["seq"], s["at"]]
    return mask, depth


def _plain_tables(s):
    start = s["row_start"].long()
    mask, depth = _ancestors(s)
    committed = s["kv_len"].long()[s["ids"].long()] - (start[1:] - start[:-1])
    pos = s["row_pos"].clone()
    m = s["seq"].numel()
    pos[:m] = (committed[s["seq"]] + depth[:m]).int()
    return {"mask": mask, "row_pos": pos}


def _own_tables(s):
    from paper_2607_21042_b200 import binding as B
    B.op_tree_tables(s["parent"], s["row_start"], s["kv_len"], s["mask"], s["row_pos"], s["info"], stream_ids=s["ids"])
    return {"mask": s["mask"], "row_pos": s["row_pos"]}


def _plain_attend(s):
    c = s["case"]
    n, H, G = c["n"], c["kv_heads"], c["heads"] // c["kv_heads"]
    rows, ok, _ = _padded(s)
    ids, start = s["ids"].long(), s["row_start"].long()
    kv_len = s["kv_len"].long()[ids]
    pages = s["table"].long()[ids, :_pages(s["keys_max"])]                            # [n, P]
    if c["cache"] == "bf16":
        kv = s["pool"][pages].float()
    else:
        codes, scales = _e4m3_views(s["pool"])
        kv = codes[pages].view(torch.float8_e4m3fn).float() * scales[pages][..., None]
    k, v = (kv[:, :, p].transpose(1, 2).reshape(n, H, -1, HD) for p in (0, 1))         # [n, H, keys, 64]
    q = (s["q"].float() / math.sqrt(HD))[rows].unflatten(2, (H, G, HD))                # [n, t, H, G, 64]
    x = torch.einsum("nthgd,nhkd->nhgtk", q, k)
    key = torch.arange(k.shape[2], device=DEV)
    d = key[None] - (kv_len - (start[1:] - start[:-1]))[:, None]                       # [n, keys]: drafted key number, negative where committed
    word = (s["mask"][rows].long())[:, :, :, None] >> torch.arange(32, device=DEV) & 1
    bit = word.flatten(2).gather(2, d.clamp(0, 32 * s["words"] - 1)[:, None].expand(-1, rows.shape[1], -1)) > 0
    seen = ((d < 0)[:, None] | bit) & (key[None] < kv_len[:, None])[:, None]           # [n, t, keys]
    x = torch.where(seen[:, None, None], x, torch.full_like(x, -math.inf))
    m = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(torch.isfinite(m), m, torch.zeros_like(m)))
    total = w.sum(-1, keepdim=True)
    o = torch.einsum("nhgtk,nhkd->nhgtd", w, v)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).permute(0, 3, 1, 2, 4)
    out = s["out"].clone()
    out[:s["seq"].numel()] = o[s["seq"], s["at"]].flatten(1).bfloat16()
    return out


def _own_attend(s):
    from paper_2607_21042_b200 import binding as B
    if "scratch" not in s:
        s["scratch"] = B.op_attention_tree_scratch(s["q"].device)
    return B.op_attention_tree(s["q"], s["pool"], s["table"], s["row_start"], s["kv_len"], s["mask"], s["t_max"], stream_ids=s["ids"], scratch=s["scratch"], out=s["out"])


def _plain_accept(s):
    rows, ok, parent = _padded(s)
    n, t = rows.shape
    j = torch.arange(t, device=DEV)
    draft, target = s["draft"].long()[rows], s["target"].long()[rows]
    says = draft == target.gather(1, parent.clamp(min=0))
    # of several children with that token the first
    twin = (parent[:, :, None] == parent[:, None]) & (draft[:, :, None] == draft[:, None]) & (j[None, :] < j[:, None])
    good = torch.where(parent >= 0, says & ~twin.any(-1), (j == 0)[None]) & ok
    on = (torch.bmm(_closure(parent), (~good).float()[..., None])[..., 0] == 0) & ok
    count = on.sum(-1)
    local = torch.where(on, j[None], torch.full_like(rows, t)).sort(-1).values
    start, ids = s["row_start"].long(), s["ids"].long()
    where = torch.where(local < t, local + start[:-1, None], torch.full_like(local, -1))
    path = s["path"].clone()
    path[:s["seq"].numel()] = where[s["seq"], s["at"]].int()
    last = local.gather(1, (count - 1).clamp(min=0)[:, None])[:, 0].clamp(max=t - 1)
    token = torch.where(count > 0, target.gather(1, last[:, None])[:, 0], torch.full_like(count, -1))
    # lengths, and the pages behind them
    before = s["kv_len"].long()[ids]
    after = before - (start[1:] - start[:-1]) + count
    held, keep = (before + PAGE - 1) // PAGE, (after + PAGE - 1) // PAGE
    end = torch.cumsum(held - keep, 0)
    top = s["top"].long()
    e = torch.arange(PPS, device=DEV)
    to = top + (end - (held - keep))[:, None] + held[:, None] - 1 - e[None]
    back = (e[None] >= keep[:, None]) & (e[None] < held[:, None])
    spare = s["free"].numel()                          # entries that stay go behind the stack's last place
    free = torch.cat([s["free"].long(), top * 0]).index_put((torch.where(back, to, torch.full_like(to, spare)).flatten(),), s["table"].long()[ids].flatten())[:spare]
    return {"path": path, "n_accepted": count.int(), "next_token": token.int(), "kv_len": s["kv_len"].long().index_copy(0, ids, after).int(), "top": (top + end[-1:]).int(), "free": free.int()}


def _own_accept(s):
    from paper_2607_21042_b200 import binding as B
    B.op_tree_accept(s["draft"], s["target"], s["parent"], s["row_start"], s["kv_len"], s["table"], s["free"], s["top"], s["path"], s["n_accepted"], s["next_token"], s["info"],
                     stream_ids=s["ids"], kv_len_out=s["kv_len_out"], free_top_out=s["top_out"])
    return {"path": s["path"], "n_accepted": s["n_accepted"], "next_token": s["next_token"], "kv_len": s["kv_len_out"], "top": s["top_out"], "free": s["free"]}


def _plain_move(s):
    m = s["seq"].numel()
    path, slot = s["path"][:m].long(), s["row_slot"].long()
    to = slot[:m]
    source = torch.where(path >= 0, slot[path.clamp(min=0)], to)                      # where nothing comes, a slot keeps its row
    a, b, c, d = to // PAGE, to % PAGE, source // PAGE, source % PAGE
    if s["case"]["cache"] == "bf16":
        s["pool"][:, a, :, :, b] = s["pool"][:, c, :, :, d]                           # all are read before one is written
    else:
        codes, scales = _e4m3_views(s["pool"])
        codes[:, a, :, :, b] = codes[:, c, :, :, d]
        scales[:, a, :, :, b] = scales[:, c, :, :, d]
    return _pool_out(s)


def _own_move(s):
    from paper_2607_21042_b200 import binding as B
    B.op_kv_move(s["pool"], s["row_start"], s["path"], s["row_slot"])
    return _pool_out(s)


_run_plain = {"rope": _plain_rope, "tables": _plain_tables, "attend": _plain_attend, "accept": _plain_accept, "move": _plain_move}
_run_own = {"rope": _own_rope, "tables": _own_tables, "attend": _own_attend, "accept": _own_accept, "move": _own_move}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_frequencies(rot, scaling):
    out = []
    for i in range(rot // 2):
        w = math.exp(-2.0 * i / rot * math.log(10000.0))
        if scaling == "linear":
            w /= 8.0
        if scaling == "yarn":
            lo = max(math.floor(rot * math.log(4096 / (64 * math.pi)) / math.log(1e8)), 0)
            hi = min(math.ceil(rot * math.log(4096 / (2 * math.pi)) / math.log(1e8)), rot - 1)
            slow = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            w = slow * w / 40.0 + (1.0 - slow) * w
        out.append(w)
    return out, 1.0 + 0.1 * math.log(40.0) if scaling == "yarn" else 1.0


def _exact_rope(case, s):
    rows, rot = case["rows"] - case["pad"], case["rot"]
    w, mag = _exact_frequencies(rot, case["scaling"])
    angle = s["pos"][:rows].double()[:, None, None] * torch.tensor(w, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(angle, mag), angle)
    half = rot // 2
    first = list(range(half)) if case["order"] == "half" else list(range(0, rot, 2))
    second = list(range(half, rot)) if case["order"] == "half" else list(range(1, rot, 2))

    def turned(x, h):
        x = x[:rows].double().reshape(rows, h, HD).clone()
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    slot = s["slot"][:rows].long()
    q = s["q_out"].double()
    q[:rows] = turned(s["q"], case["heads"]).flatten(1)
    k, v = turned(s["k"], case["kv_heads"]), s["v"][:rows].double().reshape(rows, -1, HD)
    if case["cache"] == "bf16":
        pool = s["pool"].double()
        pool[slot // PAGE, 0, :, slot % PAGE] = k
        pool[slot // PAGE, 1, :, slot % PAGE] = v
        return {"q": q, "pool": pool}
    codes, scales = _e4m3_views(s["pool"])
    codes, scales = codes.view(torch.float8_e4m3fn).double(), scales.double()
    for part, x in enumerate((k, v)):
        sc = x.abs().amax(-1) / E4M3_MAX
        codes[slot // PAGE, part, :, slot % PAGE] = x / sc[..., None]
        scales[slot // PAGE, part, :, slot % PAGE] = sc
    return {"q": q, "codes": codes, "scales": scales}


def _exact_attend(case, s):
    """A request at a time; the ancestors by walking from each node to the first."""
    H, G = case["kv_heads"], case["heads"] // case["kv_heads"]
    out = s["out"].double()
    starts, parent, ids, kv_len = (s[k].tolist() for k in ("row_start", "parent", "ids", "kv_len"))
    for i in range(case["n"]):
        a, b = starts[i], starts[i + 1]
        keys = kv_len[ids[i]]
        pages = s["table"][ids[i]].long()[:_pages(keys)]
        if case["cache"] == "bf16":
            kv = s["pool"][pages].double()
        else:
            codes, scales = _e4m3_views(s["pool"])
            kv = codes[pages].view(torch.float8_e4m3fn).double() * scales[pages].double()[..., None]
        kv = kv.permute(1, 2, 0, 3, 4).reshape(2, H, -1, HD)[:, :, :keys]              # [2, H, keys, 64]
        seen = [[False] * (b - a) for _ in range(b - a)]
        for j in range(b - a):
            at = j
            while at >= 0:
                seen[j][at] = True
                at = parent[a + at]
        hidden = torch.zeros(b - a, keys, dtype=torch.bool, device=DEV)
        hidden[:, keys - (b - a):] = ~torch.tensor(seen, device=DEV)
        q = s["q"][a:b].double().reshape(b - a, H, G, HD).permute(1, 2, 0, 3)          # [H, G, t, 64]
        x = (q @ kv[0][:, None].transpose(-1, -2) / 8.0).masked_fill(hidden, -math.inf)
        out[a:b] = (torch.softmax(x, -1) @ kv[1][:, None]).permute(2, 0, 1, 3).flatten(1)
    return out


def _exact_move(case, s):
    starts, path, slot = (s[k].tolist() for k in ("row_start", "path", "row_slot"))
    pairs = [(slot[r], slot[path[r]]) for r in range(starts[-1]) if path[r] >= 0]
    to, source = (torch.tensor(x, dtype=torch.long, device=DEV) for x in zip(*pairs))
    found = {}
    for name, x in _pool_out(s).items():
        y = x.double()
        y[:, to // PAGE, :, :, to % PAGE] = x.double()[:, source // PAGE, :, :, source % PAGE]
        found[name] = y
    return found


def exact(case, seed):
    if case["op"] in ("tables", "accept"):
        return None
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attend": _exact_attend, "move": _exact_move}[case["op"]](case, s)
