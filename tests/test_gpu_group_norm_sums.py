"""Group norm's sums over samples, dweight and dbias, of more samples than fp32 sums of one after the other would bear."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import U, padded_ckpt, values, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("samples", [(1 << 20) + 37, 70000])
@pytest.mark.parametrize("alike", [True, False])
def test_sums_over_many_samples(samples, alike):
    """One pixel a sample, no activation and no weight: a sample's terms are dy and dy h, rounded once, whose sum over the samples is rounded once more (and where it is added to what
    is there).  Sums of 64 bits add 2^-53 of the terms' magnitudes for each of up to 2^21 additions."""
    channels = 8
    rng = np.random.default_rng(samples)
    dy = np.full((samples, channels), 0.1, np.float32) if alike else (0.5 + rng.standard_normal((samples, channels))).astype(np.float32)
    q = np.full((samples, channels), 111, np.int8) if alike else rng.integers(-127, 128, (samples, channels)).astype(np.int8)
    e = np.full((samples, 1), 127 - 6, np.uint8)
    h = q * 2.0**-6
    gw, gb = torch.full((channels,), 7.0, device="cuda"), torch.full((channels,), 7.0, device="cuda")
    ws = torch.full((ff.ff_group_norm_workspace_bytes(samples, 1, channels, 2),), 0x5A, dtype=torch.uint8, device="cuda")
    rstd, kept, of = torch.ones((samples, 2), device="cuda"), padded_ckpt(q, e), torch.from_numpy(dy).cuda()
    run = lambda acc: ff.ff_group_norm_backward(of, None, None, None, *kept, rstd, samples, 2, None, None, ff.ACT_IDENTITY, None, gw, gb, acc, ws)  # noqa: E731
    run(False)
    dw, db = dy * h, dy.astype(np.float64)
    long = 2.0**-53 * 2**21
    bw, bb = U * np.abs(dw).sum(0) + long * np.abs(dw).sum(0) + 2 * U * np.abs(dw.sum(0)), long * np.abs(db).sum(0) + 2 * U * np.abs(db.sum(0))
    within(values(gw), dw.sum(0), bw, "dweight")
    within(values(gb), db.sum(0), bb, "dbias")
    run(True)
    within(values(gw), 2 * dw.sum(0), 2 * bw + 4 * U * np.abs(dw.sum(0)), "dweight added")
    within(values(gb), 2 * db.sum(0), 2 * bb + 4 * U * np.abs(db.sum(0)), "dbias added")
