"""A weight gradient of no rows is zero, however large: of more elements than one launch has lanes for, too."""
import pytest
import torch

import paper_2506_22771_amd as ff

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n, k", [(3, 5), (65535, 262160)])
def test_no_rows(n, k):
    assert n * k < 1 << 20 or n * k > 1 << 34
    if torch.cuda.mem_get_info()[0] < 5 * n * k:
        pytest.skip("not enough memory")
    dy, (q, e) = torch.empty((0, n), device="cuda"), ff.ckpt_empty(0, k)
    dw, db = torch.full((n, k), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    ws = torch.empty(ff.ff_ckpt_weight_grad_workspace_bytes(0, n, k), dtype=torch.uint8, device="cuda")
    ff.ff_ckpt_weight_grad(dy, q, e, None, None, dw, db, True, ws)
    assert all(bool((part == 7).all()) for part in dw.split(4096)) and bool((db == 7).all())
    ff.ff_ckpt_weight_grad(dy, q, e, None, None, dw, db, False, ws)
    assert not any(bool(part.any()) for part in dw.split(4096)) and not bool(db.any())
    del dw
    torch.cuda.empty_cache()
