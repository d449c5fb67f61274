"""The 128-row tcgen05 attention of prefill passes at and beyond the 256 pages that the runs of a tile may have together (a tile of an
engine's pass has 190 at most: two streams of 32 pages that are not in it from their start, and whole streams)."""
import numpy as np
import pytest
import torch

from paper_2607_21042_b200 import binding as B
from test_gpu_ops import DEV, _attention_case, _attention_ref, bits_dev, bits_to_f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [2, 80])        # two CTAs, and more than one an SM: both forms of the kernel
@pytest.mark.parametrize("ctx,whole", [(128, True), (129, False), (200, False)])
def test_pages_of_a_tile(ctx, whole, H):
    """128 streams of one row each behind contexts of 2, 3 and 4 pages, then a tile of one stream."""
    rng = np.random.default_rng(82)
    S = 8                                         # whose pages the 128 streams share
    kv, pt, Ks, Vs = _attention_case(rng, H, [ctx] * S + [60], 8 * S + 4, 4)
    pt = np.concatenate([pt[:S]] * 16 + [pt[S:]])
    rows = [(s, ctx - 1) for s in range(128)] + [(128, p) for p in range(60)]
    q = rng.standard_normal(size=(len(rows), H * 64)).astype(np.float32)
    out = B.op_attention_cluster(torch.from_numpy(q).to(DEV), bits_dev(kv), torch.from_numpy(pt).to(DEV),
                                 torch.tensor([s for s, _ in rows], dtype=torch.int32, device=DEV),
                                 torch.tensor([p for _, p in rows], dtype=torch.int32, device=DEV), -3)
    got = bits_to_f64(out)
    if not whole:
        assert np.isnan(got[:128]).all()
    for r, (s, p) in enumerate(rows):
        if (r < 128 and not whole) or r % 9:
            continue
        k = s % S if r < 128 else S
        ref = _attention_ref(q[r].astype(np.float64), Ks[k][:p + 1], Vs[k][:p + 1], H)
        assert np.max(np.abs(got[r] - ref)) <= 2.0 ** -7 * np.abs(ref).max() + 1e-5, (r, s, p)
