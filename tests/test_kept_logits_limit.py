"""The limit on the logits that the cross entropy keeps between forward and backward."""
import ctypes

import pytest
import torch

import paper_2607_21653_gb300 as molt
from paper_2607_21653_gb300.cross_entropy import CrossEntropyOptions

BF, F = torch.bfloat16, torch.float32
TILE = 16 * (16 * 512 + 4 * 128)   # bytes of 256 x 256 kept logits


@pytest.fixture(scope="module")
def lib():
    molt.build()
    return molt.load()


def size(lib, T, H, V, limit, back=1, dt=2):
    return lib.molt_cross_entropy_workspace_bytes_ex(T, H, V, back, dt, ctypes.byref(CrossEntropyOptions(-100, 0.0, 0.0, limit)))


@pytest.mark.parametrize("T,H,V", [(8192, 4096, 151936), (300, 640, 700), (1 << 20, 1024, 50257), (5000, 576, 50000)])
def test_workspace_follows_the_limit(lib, T, H, V):
    whole = lib.molt_cross_entropy_workspace_bytes(T, H, V, 1, 2)
    assert size(lib, T, H, V, 0) == whole
    assert lib.molt_cross_entropy_workspace_bytes_ex(T, H, V, 1, 2, None) == whole
    assert size(lib, T, H, V, 1 << 62) == whole   # no more than the default
    none = size(lib, T, H, V, -1)
    kept = min(-(-T // 256) * -(-V // 256) * TILE, 4 << 30) if H >= 640 else 0
    assert abs(whole - none - kept) < 256
    limits = [1, 1000, TILE, 1 << 24, 1 << 28, 1 << 30, 4 << 30]
    sizes = [size(lib, T, H, V, n) for n in limits]
    assert sizes == sorted(sizes) and all(none <= n <= none + lim + 256 for n, lim in zip(sizes, limits))
    # the forward alone keeps none
    assert size(lib, T, H, V, 0, back=0) == size(lib, T, H, V, -1, back=0)


@pytest.mark.parametrize("limit", [-1, 1 << 28])
def test_limited_workspace_never_shrinks_as_tokens_grow(lib, limit):
    for H in (320, 1024):
        sizes = [size(lib, T, H, 50257, limit, dt=dt) for dt in (2, 0) for T in range(0, 20000, 77)]
        half = len(sizes) // 2
        assert sizes[:half] == sorted(sizes[:half]) and sizes[half:] == sorted(sizes[half:])


def test_binding_refuses_a_negative_limit():
    with pytest.raises(ValueError, match="max_kept_bytes"):
        molt.cross_entropy._options(-100, 0.0, 0.0, -1)


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,V", [(1100, 640, 3000), (700, 1088, 5003)])
def test_results_with_few_and_no_logits_kept(T, H, V):
    """Kept in part (two token tiles), not at all, and whole: the forward's outputs are the same
    bits, the gradients those of the formulas.  Bounds: test_gpu_cross_entropy."""
    from test_gpu_cross_entropy import check, make, reference
    h, W, x, _ = make(T, H, V, 0.2)
    ref = reference(h, W, x)
    outs = []
    for limit in (None, 0, 2 * -(-V // 256) * TILE, 1000):
        out = molt.cross_entropy_fwd_bwd(h, W, x, max_kept_bytes=limit)
        check(out, ref)
        outs.append(out)
    for o in outs[1:]:
        for k in ("loss", "logp", "lse", "stats"):
            assert torch.equal(o[k], outs[0][k]), k
    assert not torch.equal(outs[1]["dhidden"], outs[0]["dhidden"])   # formed again, not read in steps
    ws = torch.empty(size(molt.load(), T, H, V, -1), dtype=torch.uint8, device="cuda")
    check(molt.cross_entropy_fwd_bwd(h, W, x, max_kept_bytes=0, workspace=ws), ref)
    with pytest.raises(molt.MoltError) as err:
        molt.cross_entropy_fwd_bwd(h, W, x, workspace=ws)
    assert err.value.status == 9 and molt.device_status() == 0
