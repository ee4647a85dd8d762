"""Residual norm on matrices that begin and end inside a 16-byte word, with enough rows that
every warp's stages are filled again after the first and before the last row, whose edge
words are filled in element by element.  Bounds and references: test_gpu_residual_norm."""
import pytest
import torch

from test_gpu_residual_norm import BF, F, HF, make, run_both

pytestmark = pytest.mark.gpu


def shifted(t, by):
    """The same rows in memory that begins `by` elements after a 16-byte boundary."""
    if t is None or t.dim() != 2 or t.shape[1] == 1:
        return t
    buf = torch.full((t.numel() + by,), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[by:].view(t.shape)
    v.copy_(t)
    return v


@pytest.mark.parametrize("post,gate", [(False, "none"), (False, "token"), (False, "full"), (True, "channel")])
@pytest.mark.parametrize("dtype,res", [(BF, BF), (HF, F), (F, F)])
@pytest.mark.parametrize("H,by", [(33, 1), (250, 2), (511, 3)])
def test_rows_of_one_warp(H, by, dtype, res, post, gate):
    T = 15001
    s = make(T, H, dtype, res, F, post, gate, True, True, 0.0, seed=H)
    run_both({k: shifted(v, by) if torch.is_tensor(v) else v for k, v in s.items()}, T)


@pytest.mark.parametrize("H,by", [(1031, 1), (1030, 2)])
def test_rows_of_several_warps(H, by):
    T = 3001
    s = make(T, H, BF, F, F, False, "full", True, True, 0.0, seed=H)
    run_both({k: shifted(v, by) if torch.is_tensor(v) else v for k, v in s.items()}, T)
