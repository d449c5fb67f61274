"""Forms of the serving operators that only unusual values, large passes or failures reach."""
import pytest
import torch

from paper_2607_21042_b200 import binding as B
from test_gpu_serving_ops import DEV, E4M3_BLOCK

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
