"""Shared by the tests of layer norm and checkpoints: typed matrices in wider buffers, and bounds on rounding errors."""
import numpy as np
import torch

import paper_2506_22771_amd as ff

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
HALF_ULP = {name: torch.finfo(of).eps / 2 for name, of in DTYPES.items()}       # relative error of one rounding
TINY = {"float32": 2.0**-149, "bfloat16": 2.0**-133, "float16": 2.0**-25}      # absolute error of one rounding near zero
U = 2.0**-24


def typed(a: np.ndarray, dtype: str) -> torch.Tensor:
    """On the device, in a type."""
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DTYPES[dtype]).cuda()


def values(t: torch.Tensor) -> np.ndarray:
    return t.detach().float().cpu().numpy().astype(np.float64)


class Framed:
    """A [rows, cols] view of a buffer of junk, `left` elements into it and `right` elements short of each row's end.  intact(): nothing
    but the view has changed."""

    def __init__(self, rows, cols, dtype, left=0, right=0, data=None):
        of = DTYPES.get(dtype, dtype)
        self.buffer = torch.full(((rows + 2) * (cols + left + right) + left,), 77, dtype=of, device="cuda")
        self.view = self.buffer[left + cols + left + right:][: rows * (cols + left + right)].view(rows, cols + left + right)[:, :cols] \
            if rows else self.buffer[:0].view(0, cols)
        if data is not None:
            self.view.copy_(data)
        self.mask = torch.ones_like(self.buffer, dtype=torch.bool)
        if rows:
            self.mask.as_strided(self.view.shape, self.view.stride(), self.view.storage_offset()).fill_(False)

    def intact(self):
        return bool((self.buffer[self.mask] == 77).all())


def junk_ckpt(rows, cols):
    q, e = ff.ckpt_empty(rows, cols)
    return q.fill_(0x5A), e.fill_(0x5A)


def split_ckpt(q, e, cols):
    """numpy (codes, exponent bytes) without the pad, which has to be zero."""
    nb = (cols + 31) // 32
    q, e = q.cpu().numpy(), e.cpu().numpy()
    assert not q[:, cols:].any() and not e[:, nb:].any(), "pad bytes not zero"
    return q[:, :cols], e[:, :nb]


def padded_ckpt(q: np.ndarray, e: np.ndarray):
    """numpy codes and exponent bytes to the device, padded."""
    rows, cols = q.shape
    dq = np.zeros((rows, ff.ff_pitch(cols)), np.int8)
    de = np.zeros((rows, ff.ff_pitch(ff.ff_ckpt_blocks(cols))), np.uint8)
    dq[:, :cols], de[:, :e.shape[1]] = q, e
    return torch.from_numpy(dq).cuda(), torch.from_numpy(de).cuda()


def within(got: np.ndarray, ref: np.ndarray, bound: np.ndarray, what: str) -> None:
    assert got.shape == ref.shape, what
    odd = ~np.isfinite(ref)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(ref), err_msg=what)
    np.testing.assert_array_equal(got[odd & ~np.isnan(ref)], ref[odd & ~np.isnan(ref)], err_msg=what)
    over = np.abs(got - ref)[~odd] - np.broadcast_to(bound, ref.shape)[~odd]
    assert over.size == 0 or over.max() <= 0, f"{what}: {over.max()} beyond its bound, {np.abs(got - ref)[~odd].max()} in all"
