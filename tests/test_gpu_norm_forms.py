"""Every form of the residual norm's persistent kernels with several rows to a block: rows by
the vector (H % 8 == 0), the pair and the element, of one warp and of several, 8 and 16
elements to a thread, one stage and two; with each part left out, each gate and the
types.  The forward takes these kernels for rows of whole vectors from 16 rows an SM on, which
is why T is 2600 here.  Bounds and references: test_gpu_residual_norm."""
import pytest
import torch

from test_gpu_residual_norm import BF, F, HF, dev, run_both

pytestmark = pytest.mark.gpu


def make(T, H, dtype, res, ptype, post, gate, pre, residual, seed):
    g = torch.Generator(device=dev()).manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=dev())
    return {"x": n(T, H).to(dtype), "residual": (2 * n(T, H)).to(res) if residual else None, "eps": 1e-5, "alpha": 0.75, "offset": 0.0,
            "w_post": (1 + 0.3 * n(H)).to(ptype) if post else None, "w_pre": (1 + 0.3 * n(H)).to(ptype) if pre else None,
            "gate": {"none": lambda: None, "channel": lambda: n(H).to(ptype), "token": lambda: n(T, 1),
                     "full": lambda: n(T, H).to(dtype)}[gate](),
            "dy": (0.5 * n(T, H)).to(dtype) if pre else None, "dr": n(T, H).to(res)}


# (dtype, res, ptype, post, gate, pre, residual): every part left out, gate and type with each other at least once
FORMS = [(BF, BF, BF, True, "none", True, True), (BF, F, BF, False, "channel", True, True), (BF, F, F, True, "token", True, True),
         (BF, BF, F, True, "full", True, True), (HF, HF, F, False, "none", True, False), (HF, F, HF, True, "channel", False, True),
         (HF, HF, HF, False, "token", True, True), (HF, F, F, False, "full", False, True), (F, F, F, True, "channel", True, True),
         (F, F, F, False, "token", False, True), (F, F, F, True, "full", True, False), (BF, BF, BF, False, "full", True, True)]
IDS = ["-".join(str(v).replace("torch.", "") for v in f) for f in FORMS]


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("H", [64, 256, 264, 512, 1024, 2048, 4096, 5120, 8192])
def test_rows_of_vectors(H, form):
    run_both(make(2600, H, *form, seed=H), 2600)


@pytest.mark.parametrize("form", FORMS[1::3] + FORMS[8:9], ids=IDS[1::3] + IDS[8:9])
@pytest.mark.parametrize("H", [130, 514, 2050, 5122, 8190, 131, 513, 2049, 5121, 8191])
def test_rows_of_pairs_and_elements(H, form):
    run_both(make(2600, H, *form, seed=H), 2600)


@pytest.mark.parametrize("T,H", [(1217, 8192), (1217, 8190), (1217, 8191)])
@pytest.mark.parametrize("gate", ["channel", "full"])
def test_one_stage(T, H, gate):
    """fp32 rows of which shared memory holds one at a time, eight or nine to a block."""
    run_both(make(T, H, F, F, F, True, gate, True, True, seed=H), T)
