"""Forms of the serving operators that only unusual values, large passes or failures reach."""
import pytest
import torch

from paper_2607_21042_b200 import binding as B
from test_gpu_serving_ops import DEV, E4M3_BLOCK, Cache, CrossCase, _gen, _q

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------
# K and V rows into their slots
# ---------------------------------------------------------------------------------------------
def _encoded(y):
    """e4m3 codes and scales of values [..., 64] in fp32: s = max / 448, 1 where that is zero; finite codes."""
    s = y.abs().amax(-1)
    s = s / torch.full_like(s, 448.0)              # by a tensor: a number's reciprocal would be rounded first
    s = torch.where(s > 0, s, torch.ones_like(s))
    return (y / s[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), s


def test_kv_append_of_values_whose_scale_vanishes():
    """Below 448 * 2^-150 the largest value of a head divided by 448 is zero in fp32: all codes are then zero and the scale is 1, as for zeros;
    just above it the scale is the smallest number there is.  No code may be NaN (0x7F, 0xFF)."""
    tiny = 2.0 ** -149
    x = torch.zeros(8, 128, dtype=torch.float32)
    for r, top in enumerate([1, 200, 224, 225, 300, 448, 1000, 2 ** 20]):      # 224 * 2^-149 is the border itself, a tie that goes to zero
        x[r, 3] = top * tiny
        x[r, 40] = -tiny
        x[r, 64 + r] = -top * tiny
    x = x.to(DEV)
    pool = torch.full((1, 2, 2, E4M3_BLOCK), 77, dtype=torch.uint8, device=DEV)
    B.op_kv_append(x, x, pool, torch.arange(8, dtype=torch.int32, device=DEV))
    codes, scales = pool[0, :, :, :4096].unflatten(-1, (64, 64))[:, :, :8], pool[0, :, :, 4096:].contiguous().view(torch.float32)[:, :, :8]
    want_codes, want_scales = _encoded(x.cpu().view(8, 2, 64))                  # on the host, whose division keeps such numbers
    for part in range(2):
        assert torch.equal(scales[part].cpu(), want_scales.t())
        assert torch.equal(codes[part].cpu(), want_codes.transpose(0, 1))
    assert not bool(((codes & 0x7F) == 0x7F).any()) and bool((scales > 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("R,heads,strided", [(6315, 3, True), (1001, 20, False), (3584, 20, True)])
def test_kv_append_of_large_passes(R, heads, strided, fmt, dtype):
    """From 8 * 256 * SMs lanes on a thread writes four pieces, of rows a quarter of the pass apart.  6315 rows of 3 heads are 37 890 pieces, not a
    multiple of four; rows without a slot lie in all four quarters, at their ends too."""
    assert R * 2 * heads * 8 >= 8 * 256 * torch.cuda.get_device_properties(DEV).multi_processor_count
    g = _gen(R + heads)
    n_pages = (R + 63) // 64 + 2
    if strided:
        x = (torch.randn(R, 3, heads * 64, generator=g) * 3).to(dtype).to(DEV)
        k, v = x[:, 1], x[:, 2]
    else:
        k, v = torch.randn(R, heads * 64, generator=g).to(dtype).to(DEV), (torch.randn(R, heads * 64, generator=g) * 1e-3).to(dtype).to(DEV)
    k[R // 2, :64] = 0                              # a head whose values are all zero
    slot = torch.randperm(n_pages * 64, generator=g)[:R].int()
    for i in range(4):
        a, b = i * R // 4, (i + 1) * R // 4
        for at, bad in zip((a, a + 1, (a + b) // 2, b - 2, b - 1), (-1, n_pages * 64, 2 ** 31 - 1, -2 ** 31, -64)):
            slot[at] = bad
    pool = torch.randint(0, 100, (n_pages, 2, heads, 8192 if fmt == "bf16" else E4M3_BLOCK), generator=g, dtype=torch.uint8).to(DEV)
    want = pool.clone()
    B.op_kv_append(k, v, pool.view(torch.bfloat16).view(n_pages, 2, heads, 64, 64) if fmt == "bf16" else pool, slot.to(DEV))
    ok = (slot >= 0) & (slot < n_pages * 64)
    assert int(ok.sum()) == R - 20
    rows, slots = torch.nonzero(ok)[:, 0].to(DEV), slot[ok].long().to(DEV)
    page, off = slots // 64, slots % 64
    for part, src in enumerate((k, v)):
        y = src[rows].float().view(-1, heads, 64)
        if fmt == "bf16":
            want.view(torch.bfloat16).view(n_pages, 2, heads, 64, 64)[page, part, :, off] = y.bfloat16()
        else:
            codes, scales = _encoded(y)
            want[..., :4096].unflatten(-1, (64, 64))[page, part, :, off] = codes
            want[..., 4096:].view(torch.float32)[page, part, :, off] = scales
    assert torch.equal(pool, want)


# ---------------------------------------------------------------------------------------------
# attention whose parts a second kernel adds
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("qt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,H,kv,n_shared", [(130, 20, 20, 0), (130, 20, 20, 3), (300, 20, 4, 0), (300, 20, 4, 5), (520, 12, 4, 1), (1300, 16, 1, 2), (2600, 3, 3, 0)])
def test_shared_prefix_attention_of_large_batches(R, H, kv, n_shared, qt, fmt):
    """More units of 32 keys than CTAs can merge themselves (52 an SM): rows finished by one warp, rows cut by a range's end, rows whose own keys
    are none, rows that end inside the shared pages, rows of another's stream, padding."""
    own = [(0, 1, 31, 32, 33, 64, 65, 90, 17, 128)[i % 10] if i % 7 else 150 for i in range(R)]
    if n_shared == 0:
        own = [max(1, x) for x in own]
    # rows 1, 12: end inside the shared pages (or, without any, early); row 3 reads row 7's stream up to its third key from the end
    short = [(1, 1, 64 * n_shared // 2 if n_shared else 0), (12, 12, 64 * n_shared - 1 if n_shared else 5), (3, 7, 64 * n_shared + own[7] - 3)]
    c = Cache(R + n_shared, fmt, kv, n_shared, own, pad=3, same_stream=short)
    R += 3
    rpt, pps = 16 // (H // kv), c.args[0].shape[1]
    units = kv * -(-R // rpt) * (2 * n_shared + 1) + R * kv * (2 * (pps - n_shared) + 1)
    assert units > 52 * min(160, torch.cuda.get_device_properties(DEV).multi_processor_count)
    q = _q(R, R, H, qt)
    got = B.op_attention_shared(q, c.pool, *c.args)
    c.check(got, q, "large batch")
    assert torch.all(got[-3:].view(torch.bfloat16) == 0)


def test_shared_prefix_attention_of_sixty_rows():
    c = Cache(11, "bf16", 20, 4, [50 + 7 * i for i in range(60)])
    q = _q(6, 60, 20, torch.float32)
    c.check(B.op_attention_shared(q, c.pool, *c.args), q, "sixty rows")


# ---------------------------------------------------------------------------------------------
# strides that address nothing
# ---------------------------------------------------------------------------------------------
def _cross_c(x, scratch, out, **kw):
    """The C entry point on a CrossCase's arrays, with some arguments replaced."""
    a = dict(n=len(x.ql), heads=x.heads, kv=x.kv, type=B.T_BF16, qr=x.q.shape[0], q=x.q.data_ptr(), qs=x.q.stride(0), kr=x.k.shape[0], k=x.k.data_ptr(), ks=x.k.stride(0),
             kh=x.k.stride(1), v=x.v.data_ptr(), vs=x.v.stride(0), vh=x.v.stride(1), q0=x.args[3].data_ptr(), k0=x.args[4].data_ptr(), q_max=max(x.ql), scale=x.scale,
             out=out.data_ptr(), scratch=scratch.data_ptr(), size=scratch.numel(), stream=0)
    assert set(kw) <= set(a)
    return B.load().tts_gpt_op_attention_cross(*{**a, **kw}.values())


@pytest.mark.parametrize("ql", [[1, 3], [70, 40]])
@pytest.mark.parametrize("stride", [0, 8, -64, 3])
def test_the_stride_of_a_single_head_or_row_is_not_looked_at(ql, stride):
    scratch = B.op_attention_cross_scratch(DEV)
    x = CrossCase(61, torch.bfloat16, 4, 1, ql, [150, 90])                       # one head of keys
    out = torch.full(x.q.shape, 9.0, dtype=x.dtype, device=DEV)
    torch.cuda.synchronize()
    assert _cross_c(x, scratch, out, kh=stride, vh=stride) == B.OK, B.load().tts_gpt_last_error(None)
    torch.cuda.synchronize()
    x.check(out, "one head")
    x = CrossCase(62, torch.bfloat16, 4, 2, [3], [1])                            # one row of keys, one of queries: its first row alone
    out = torch.full(x.q.shape, 9.0, dtype=x.dtype, device=DEV)
    torch.cuda.synchronize()
    assert _cross_c(x, scratch, out, kr=1, ks=stride, vs=stride) == B.OK, B.load().tts_gpt_last_error(None)
    torch.cuda.synchronize()
    x.check(out, "one row of keys")
    one = torch.full(x.q.shape, 9.0, dtype=x.dtype, device=DEV)
    torch.cuda.synchronize()
    assert _cross_c(x, scratch, one, qr=1, qs=stride) == B.OK, B.load().tts_gpt_last_error(None)
    torch.cuda.synchronize()
    assert torch.equal(one[:1], out[:1]) and torch.all(one[1:] == 9.0)


@pytest.mark.parametrize("stride", [0, 8, -64, 3])
def test_the_stride_of_a_single_row_is_not_looked_at(stride):
    c = Cache(63, "bf16", 2, 1, [40])
    q = _q(64, 1, 4, torch.float32)
    want = B.op_attention_shared(q, c.pool, *c.args)
    out, scratch = torch.empty_like(want), B.op_attention_shared_scratch(1, 4, 2, DEV)
    torch.cuda.synchronize()
    lib = B.load()
    assert lib.tts_gpt_op_attention_shared(1, 4, 2, B.T_F32, q.data_ptr(), stride, 0, c.n_pages, c.pool.data_ptr(), 1, c.args[0].data_ptr(), c.args[0].shape[1], c.args[1].data_ptr(),
                                           c.args[2].data_ptr(), out.data_ptr(), scratch.data_ptr(), scratch.numel(), 0) == B.OK, lib.tts_gpt_last_error(None)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    kv = torch.randn(2, 128, generator=_gen(65)).to(DEV)
    slot, pool = torch.tensor([70], dtype=torch.int32, device=DEV), torch.zeros(2, 2, 2, 64, 64, dtype=torch.bfloat16, device=DEV)
    want = pool.clone()
    B.op_kv_append(kv[:1], kv[1:], want, slot)
    torch.cuda.synchronize()
    assert lib.tts_gpt_op_kv_append(1, 2, B.T_F32, kv.data_ptr(), stride, kv.data_ptr() + 512, stride, slot.data_ptr(), 0, 2, pool.data_ptr(), 0) == B.OK, lib.tts_gpt_last_error(None)
    torch.cuda.synchronize()
    assert torch.equal(pool, want) and bool(pool.any())


# ---------------------------------------------------------------------------------------------
# waits that run out
# ---------------------------------------------------------------------------------------------
def _shared_call(seed, fmt, H, kv, n_shared, own, qt, pad=0):
    c = Cache(seed, fmt, kv, n_shared, own, pad=pad)
    q = _q(seed + 1, len(own) + pad, H, qt)
    scratch = B.op_attention_shared_scratch(len(own) + pad, H, kv, DEV)
    rows = torch.ones(q.shape[0], dtype=torch.bool, device=DEV)
    return lambda **kw: B.op_attention_shared(q, c.pool, *c.args, **kw).view(torch.bfloat16).view(-1, H, 64), scratch, rows


def _cross_call(seed, dtype, heads, kv, ql, kl):
    x = CrossCase(seed, dtype, heads, kv, ql, kl, gap_q=2)
    rows = torch.zeros(x.q.shape[0], dtype=torch.bool, device=DEV)
    rows[x.qs[0]:x.qs[-1]] = True
    return x.run, B.op_attention_cross_scratch(DEV), rows


CALLS = {
    "five rows": lambda: _shared_call(71, "bf16", 20, 20, 7, [1, 40, 130, 0, 64], torch.float32),
    "8-bit, grouped, padding": lambda: _shared_call(72, "e4m3", 20, 4, 2, [300, 9, 64], torch.bfloat16, pad=2),
    "no prefix": lambda: _shared_call(73, "bf16", 4, 4, 0, [530, 2, 1000, 1], torch.float32),
    "second kernel": lambda: _shared_call(74, "bf16", 20, 20, 3, [1 + 7 * i % 90 for i in range(130)], torch.float32),
    "second kernel, no prefix, 8-bit": lambda: _shared_call(75, "e4m3", 20, 20, 0, [1 + 7 * i % 150 for i in range(130)], torch.bfloat16),
    "one token each": lambda: _cross_call(76, torch.bfloat16, 20, 20, [1] * 9, [900 - 70 * i for i in range(9)]),
    "latents": lambda: _cross_call(77, torch.float16, 6, 2, [32, 5, 0, 17], [90, 0, 50, 700]),
    "tiles": lambda: _cross_call(78, torch.bfloat16, 3, 3, [300, 64, 0, 129], [700, 0, 100, 257]),
    "tiles, one sequence, grouped": lambda: _cross_call(79, torch.float16, 10, 2, [700], [1500]),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_scratch_of_a_failed_call_gives_nan_until_it_is_zeroed(name):
    call, scratch, rows = CALLS[name]()
    want = call(scratch=scratch).clone()
    scratch[:4].view(torch.int32).fill_(1)
    got = call(scratch=scratch)
    assert bool(torch.isnan(got[rows]).all()) and torch.equal(got[~rows], want[~rows])
    assert int(scratch[:4].view(torch.int32)) == 1
    scratch.zero_()
    assert torch.equal(call(scratch=scratch), want)


@pytest.mark.parametrize("cta", [1, 5])       # both copy something in each of the calls; CTA 0's range may end before a tile's first block
@pytest.mark.parametrize("name", CALLS)
def test_rows_behind_an_expired_wait_are_nan(name, cta):
    """The copies of one CTA never count as complete: the call ends, says so in its scratch, and every head of a row is whole or NaN, also
    where the caller gave no scratch to look into.  (Calls on tiles of 256 rows take the two seconds of an ordinary wait.)"""
    call, scratch, rows = CALLS[name]()
    want = call(scratch=scratch).clone()
    try:
        B.debug_expire_op(cta, 20000)
        got = [call(scratch=scratch).clone()] + ([call().clone()] if cta == 1 else [])
    finally:
        B.debug_expire_op(-1)
    assert int(scratch[:4].view(torch.int32)) == 1
    for y in got:
        lost = torch.isnan(y).all(-1)
        assert bool(lost[rows].any()) and not bool(lost[~rows].any())
        assert torch.equal(y[~lost], want[~lost])
    after = call(scratch=scratch)
    assert bool(torch.isnan(after[rows]).all())
    scratch.zero_()
    assert torch.equal(call(scratch=scratch), want) and torch.equal(call()[rows], want[rows])


def test_expire_op_refuses():
    for bad in ((-2, 10), (0, 0), (0, 100001)):
        with pytest.raises(B.TtsGptError) as e:
            B.debug_expire_op(*bad)
        assert e.value.code == B.E_ARG
