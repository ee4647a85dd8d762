"""Token embedding and its gradient by sorted tokens, against fp64 sums on the host.

Tolerances, before any run: u is the output type's unit roundoff (bf16 2^-8, fp16
2^-11, fp32 2^-24).  Forward: one fp32 product and one rounding, |err| <= (u + 2^-23)
|ref| (fp16: plus half its smallest subnormal, 2^-25).  Gradient: a sum of n fp32
terms in any order is off by at most n 2^-24 times the sum of their absolute values
(here with 4 more for the scale and the parts), plus the output's rounding."""
import numpy as np
import pytest
import torch

import paper_2607_21653_gb300 as molt

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11, torch.float32: 2.0**-24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0**-25, torch.float32: 0.0}
PAIRS = [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
         (torch.float16, torch.float32), (torch.float32, torch.float32)]


def dev():
    return torch.device("cuda", torch.cuda.current_device())


def ids_of(kind, T, V, rng):
    if kind == "one":
        return np.full(T, V // 2, dtype=np.int32)
    if kind == "sorted":
        return np.sort(rng.integers(0, V, T)).astype(np.int32)
    if kind == "zipf":
        r = (np.exp(rng.random(T) * np.log(V + 1.0)) - 1).astype(np.int64).clip(0, V - 1)
        return rng.permutation(V)[r].astype(np.int32)
    return rng.integers(0, V, T).astype(np.int32)


@pytest.mark.parametrize("dtype,out", PAIRS)
@pytest.mark.parametrize("T,H,V", [(1, 1, 1), (1, 4096, 50), (3, 7, 5), (64, 320, 1000), (1031, 896, 333),
                                   (5000, 2048, 700), (257, 4099, 40), (2, 20001, 3)])
def test_forward(T, H, V, dtype, out):
    rng = np.random.default_rng(T + H)
    E = torch.from_numpy(rng.normal(size=(V, H))).to(dev(), dtype)
    x = torch.from_numpy(ids_of("any", T, V, rng)).to(dev())
    for scale in (1.0, 22.6274):
        got = molt.token_embedding(E, x, scale=scale, out_dtype=out)
        assert got.dtype == out and got.shape == (T, H)
        ref = E.double()[x.long()] * float(np.float32(scale))
        assert ((got.double() - ref).abs() <= (U[out] + 2.0**-23) * ref.abs() + TINY[out]).all()
    assert molt.device_status() == 0


def check_grad(ids, V, H, dtype, out, scale, padding, seed, unaligned=False, expect_flag=0):
    rng = np.random.default_rng(seed)
    T = ids.size
    d = torch.from_numpy(rng.normal(size=(T, H)).astype(np.float32)).to(dev(), dtype)
    x = torch.from_numpy(ids).to(dev())
    dW = None
    if unaligned:   # rows that start one element past a 16-byte boundary
        dW = torch.full((V * H + 1,), 7.0, dtype=out, device=dev())[1:].view(V, H)
    got = molt.token_embedding_bwd(d, x, V, scale=scale, padding_idx=padding, dtype=out, dW=dW)
    again = molt.token_embedding_bwd(d, x, V, scale=scale, padding_idx=padding, dtype=out)
    assert molt.device_status() == expect_flag
    assert torch.equal(got, again)
    keep = (ids >= 0) & (ids < V) & (ids != (-1 if padding is None else padding))
    d64 = d.double().cpu()[torch.from_numpy(keep)]
    k = torch.from_numpy(ids[keep].astype(np.int64))
    s = float(np.float32(scale))
    ref = torch.zeros(V, H, dtype=torch.float64).index_add_(0, k, d64 * s)
    mag = torch.zeros(V, H, dtype=torch.float64).index_add_(0, k, d64.abs() * s)
    n = torch.zeros(V, dtype=torch.float64).index_add_(0, k, torch.ones(k.numel(), dtype=torch.float64))
    err = (got.double().cpu() - ref).abs()
    assert (err <= U[out] * ref.abs() + (n[:, None] + 4) * 2.0**-24 * mag + TINY[out]).all()
    assert (got.cpu()[n == 0] == 0).all()
    return d, x, ref, mag, n


@pytest.mark.parametrize("dtype,out", PAIRS)
@pytest.mark.parametrize("kind", ["any", "zipf", "one", "sorted"])
@pytest.mark.parametrize("T,H,V", [(1, 8, 3), (700, 320, 1000), (1031, 127, 50)])
def test_gradient(T, H, V, kind, dtype, out):
    rng = np.random.default_rng(T)
    check_grad(ids_of(kind, T, V, rng), V, H, dtype, out, 3.5, None, 1)


@pytest.mark.parametrize("T,H,V,kind", [
    (8, 64, 2, "any"), (9, 64, 1, "any"), (8191, 72, 5000, "zipf"), (8192, 64, 31, "any"), (8193, 64, 50000, "zipf"),
    (8200, 24, 255, "any"), (20000, 2056, 3000, "zipf"), (40000, 8, 151936, "any"), (131072, 8, 256, "any"),
    (131073, 8, 65535, "zipf"), (150001, 16, 70000, "zipf"), (140000, 8, 9, "one"), (3000, 5121, 100, "zipf")])
def test_gradient_over_chunks_of_the_sort(T, H, V, kind):
    """One sorted chunk and many, one round of merging and two, runs that cross units."""
    rng = np.random.default_rng(T)
    check_grad(ids_of(kind, T, V, rng), V, H, torch.float32, torch.float32, 1.0, None, 2)


@pytest.mark.parametrize("T,H,V", [(500, 33, 100), (9000, 64, 100)])
def test_gradient_padding_and_alignment(T, H, V):
    rng = np.random.default_rng(3)
    ids = ids_of("zipf", T, V, rng)
    ids[::3] = 0
    check_grad(ids, V, H, torch.bfloat16, torch.bfloat16, 1.0, 0, 3)
    check_grad(ids, V, H, torch.bfloat16, torch.float32, 2.0, 7, 3, unaligned=True)
    check_grad(np.full(T, 4, dtype=np.int32), V, H, torch.float32, torch.float32, 1.0, 4, 3)   # nothing left


@pytest.mark.parametrize("dtype,out", PAIRS)
@pytest.mark.parametrize("T,H,V", [(1, 76, 3001), (2, 1566, 700), (700, 34, 5000), (5, 33, 4100), (1500, 2052, 60), (40, 2, 100000)])
def test_rows_of_every_vector_length(T, H, V, dtype, out):
    """Even rows that are no multiple of eight; few tokens of many, so that rows are zeroed in long runs."""
    rng = np.random.default_rng(T + H)
    ids = ids_of("zipf", T, V, rng)
    for unaligned in (False, True):
        check_grad(ids, V, H, dtype, out, 1.5, None, 6, unaligned=unaligned)
    E = torch.from_numpy(rng.normal(size=(V, H))).to(dev(), dtype)
    x = torch.from_numpy(ids).to(dev())
    ref = E.double()[x.long()] * 1.5
    for at in (0, 1, 2, 4):   # rows that start at any element
        buf = torch.empty(T * H + 8, dtype=out, device=dev())[at:at + T * H].view(T, H)
        got = molt.token_embedding(E, x, scale=1.5, out_dtype=out, out=buf)
        assert ((got.double() - ref).abs() <= (U[out] + 2.0**-23) * ref.abs() + TINY[out]).all()
    assert molt.device_status() == 0


@pytest.mark.parametrize("T", [300, 9001])
def test_tokens_out_of_range(T):
    V, H = 70, 40
    rng = np.random.default_rng(4)
    ids = ids_of("any", T, V, rng)
    ids[5], ids[T - 1], ids[17] = -1, V, 2**31 - 1
    check_grad(ids, V, H, torch.float32, torch.float32, 1.0, None, 4, expect_flag=molt.DEV_FLAGS["token_range"])
    E = torch.randn(V, H, device=dev())
    out = molt.token_embedding(E, torch.from_numpy(ids).to(dev()))
    assert molt.device_status() == molt.DEV_FLAGS["token_range"]
    bad = torch.from_numpy((ids < 0) | (ids >= V)).to(dev())
    assert (out[bad] == 0).all() and torch.equal(out[~bad], E[torch.from_numpy(ids).to(dev())[~bad].long()])


@pytest.mark.parametrize("H", [64, 65])
def test_gradient_added_to(H):
    T, V = 9000, 500
    rng = np.random.default_rng(5)
    ids = ids_of("zipf", T, V, rng)
    d, x, ref, mag, n = check_grad(ids, V, H, torch.bfloat16, torch.float32, 0.5, None, 5)
    base = torch.randn(V, H, device=dev())
    got = molt.token_embedding_bwd(d, x, V, scale=0.5, dW=base.clone(), accumulate_dW=True)
    err = (got.double() - base.double() - ref.to(dev())).abs().cpu()
    assert (err <= 2.0**-24 * (base.double().cpu() + ref).abs() + (n[:, None] + 4) * 2.0**-24 * mag).all()
    assert torch.equal(got[n.to(dev()) == 0], base[n.to(dev()) == 0])


def test_non_finite_gradients_stay_in_their_rows():
    T, V, H = 400, 20, 64
    ids = np.arange(T, dtype=np.int32) % V
    d = torch.ones(T, H, device=dev())
    d[3] = float("inf")
    d[24] = float("nan")
    got = molt.token_embedding_bwd(d, torch.from_numpy(ids).to(dev()), V)
    assert torch.isinf(got[3]).all() and torch.isnan(got[4]).all()
    rest = [v for v in range(V) if v not in (3, 4)]
    assert (got[rest] == T // V).all()


def test_no_tokens():
    empty = torch.empty(0, dtype=torch.int32, device=dev())
    dW = torch.ones(4, 8, device=dev())
    assert torch.equal(molt.token_embedding_bwd(torch.empty(0, 8, device=dev()), empty, 4, dW=dW, accumulate_dW=True),
                       torch.ones(4, 8, device=dev()))
    assert (molt.token_embedding_bwd(torch.empty(0, 8, device=dev()), empty, 4) == 0).all()
    assert molt.token_embedding(torch.ones(4, 8, device=dev()), empty).shape == (0, 8)


def test_gradient_by_differences():
    """<dout, E'[x] - E[x]> = <dE, E' - E>: the forward is linear, so one step of any size serves."""
    T, V, H = 900, 60, 48
    rng = np.random.default_rng(6)
    x = torch.from_numpy(ids_of("zipf", T, V, rng)).to(dev())
    E, step, d = (torch.from_numpy(rng.normal(size=s).astype(np.float32)).to(dev()) for s in ((V, H), (V, H), (T, H)))
    up = (molt.token_embedding(E + step, x, scale=2.0).double() - molt.token_embedding(E, x, scale=2.0).double())
    lhs = (up * d.double()).sum()
    rhs = (molt.token_embedding_bwd(d, x, V, scale=2.0).double() * ((E + step).double() - E.double())).sum()
    # T H products, each off by a few 2^-24 of its size
    scale = (up.abs() * d.double().abs()).sum()
    assert abs(float(lhs - rhs)) <= 1e-5 * float(scale)


def test_other_stream_and_workspace():
    T, V, H = 5000, 300, 128
    rng = np.random.default_rng(7)
    x = torch.from_numpy(ids_of("zipf", T, V, rng)).to(dev())
    d = torch.randn(T, H, device=dev())
    ref = molt.token_embedding_bwd(d, x, V)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = molt.token_embedding_bwd(d, x, V)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, ref)
    small = torch.empty(512, dtype=torch.uint8, device=dev())
    with pytest.raises(molt.MoltError) as e:
        molt.token_embedding_bwd(d, x, V, workspace=small)
    assert e.value.status == 9
    poisoned = torch.full((molt.load().molt_token_embedding_bwd_workspace_bytes(T, H, V),), 255, dtype=torch.uint8,
                          device=dev())
    assert torch.equal(molt.token_embedding_bwd(d, x, V, workspace=poisoned), ref)
