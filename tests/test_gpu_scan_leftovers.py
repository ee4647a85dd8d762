"""The recurrence's gradients of rows that TMA cannot take, after other kernels: lanes without a channel
read shared memory that no copy has written, and what is left there decides no bit of a result."""
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu


def leave(value, dtype):
    """Every SM's tiles hold this value: a channel's gates, its values and (a is next to 0, or the value 0) its results."""
    x = torch.full((4096, 16384), value, dtype=dtype, device=dev())
    assert (molt.gated_scan_fwd(x, x)["y"] == value).all()


@pytest.mark.parametrize("kind", ["sigmoid", "log"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H,off", [(65, 0), (65, 1), (56, 3), (1, 0), (300, 1)])
def test_gradients_do_not_depend_on_what_ran_before(H, off, dtype, kind):
    T = 4001
    g = torch.Generator(device=dev()).manual_seed(H)
    n = lambda *s: torch.randn(*s, device=dev(), generator=g)
    wide = lambda x: torch.nn.functional.pad(x, (off, 3)).to(dtype)[:, off:off + H]
    # down to gates whose a has the fewest digits as 1 + (a - 1)
    gate, value, dy = wide(-4.75 * torch.rand(T, H, device=dev(), generator=g)), wide(n(T, H)), wide(n(T, H))
    cu = torch.tensor([0, 700, 701, 3000, T], dtype=torch.int32, device=dev())
    states = molt.gated_scan_fwd(gate, value, cu_seqlens=cu, kind=kind, want_states=True)["states"]
    got = []
    for left in (0.0, -20.0, 0.0, -1024.0):
        leave(left, dtype)
        got.append(molt.gated_scan_bwd(dy, gate, value, states, cu_seqlens=cu, kind=kind))
    for other in got[1:]:
        for k in ("dgate", "dvalue"):
            assert torch.equal(other[k], got[0][k]), (k, int((other[k] != got[0][k]).sum()))
    assert molt.device_status() == 0
