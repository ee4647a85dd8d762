"""Dropout from a counter, against the generator restated in numpy.

The mask is exact.  Values, before any run: the factor 1 / (1 - q) is rounded once and the
product once in fp32 (2^-23 together), the residual's product and the sum once each (fused:
2^-24), the result once to its type (bf16 2^-8, fp16 2^-11 and half its smallest
subnormal, fp32 2^-24)."""
import numpy as np
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11, torch.float32: 2.0**-24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0**-25, torch.float32: 0.0}
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def philox(counter, key):
    """Philox4x32-10 on arrays of 32-bit words (SC 2011)."""
    c = [np.asarray(x, dtype=np.uint64) for x in np.broadcast_arrays(*counter)]
    k0, k1 = int(key[0]), int(key[1])
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def kept(T, H, p, seed, offset=0, first_row=0):
    g = np.arange((H + 7) // 8, dtype=np.uint64)[None, :]
    r = np.arange(first_row, first_row + T, dtype=np.uint64)[:, None]
    w = philox((g, r, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.stack([x >> np.uint64(s) & np.uint64(0xFFFF) for x in w for s in (0, 16)], 2).reshape(T, -1)[:, :H]
    return torch.from_numpy(bits >= np.floor(p * 65536 + 0.5)).to(dev())


def test_the_generator_restated():
    """The published answers for a counter and a key of all zeros, and of all ones."""
    assert [int(x) for x in philox((0, 0, 0, 0), (0, 0))] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert [int(x) for x in philox((ones,) * 4, (ones, ones))] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def reference(x, keep, p, residual=None, res_scale=1.0):
    q = np.floor(p * 65536 + 0.5) / 65536
    out = torch.where(keep, x.double() / (1 - q) if q < 1 else x.double() * 0, 0.0)
    return out if residual is None else out + float(np.float32(res_scale)) * residual.double()


def check(got, ref, x, residual, dtype, q):
    mag = x.double().abs() / (1 - q) if q < 1 else torch.zeros_like(ref)
    bound = 2.0**-23 * torch.where(mag.isfinite(), mag, 0.0) + U[dtype] * ref.abs() * (1 + 2.0**-20) + TINY[dtype]
    if residual is not None:
        bound = bound + 2.0**-23 * residual.double().abs() * 2 + U[dtype] * 2.0**-20
    assert got.dtype == dtype and ((got.double() - ref).abs() <= bound).all(), float(((got.double() - ref).abs() - bound).max())


@pytest.mark.parametrize("dtype,res", [(BF, None), (HF, None), (F32, None), (BF, BF), (HF, HF), (BF, F32), (HF, F32), (F32, F32),
                                       (F32, BF)])
@pytest.mark.parametrize("T,H", [(1, 1), (1, 8), (3, 7), (5, 64), (64, 2048), (257, 1031), (1000, 320), (33, 8200), (4000, 9)])
def test_forward(T, H, dtype, res):
    rng = torch.Generator(device=dev()).manual_seed(T + H)
    x = torch.randn(T, H, device=dev(), generator=rng).to(dtype)
    r = None if res is None else torch.randn(T, H, device=dev(), generator=rng).to(res)
    for p, seed, offset, first, scale in ((0.1, 1, 0, 0, 1.0), (0.5, (1 << 63) + 12345678901, (1 << 40) + 7, 1 << 20, 0.7071),
                                          (0.0, 5, 0, 0, 1.0), (1.0, 5, 3, 0, -2.0), (0.9999999, 7, 0, 0, 1.0)):
        keep = kept(T, H, p, seed, offset, first)
        if p == 0.0:
            assert keep.all()
        if p > 0.999:
            assert not keep.any()
        got = molt.dropout_fwd(x, p, seed, offset=offset, residual=r, res_scale=scale, first_row=first)
        ref = reference(x, keep, p, r, scale)
        check(got, ref, x, r, x.dtype if res is None else res, np.floor(p * 65536 + 0.5) / 65536)
        if r is None:
            assert torch.equal(got != 0, keep & (x != 0))
    assert molt.device_status() == 0


@pytest.mark.parametrize("dtype,to", [(BF, BF), (HF, HF), (F32, F32), (F32, BF), (F32, HF), (BF, F32)])
@pytest.mark.parametrize("T,H", [(1, 5), (300, 320), (70, 1031)])
def test_backward_has_the_forwards_mask(T, H, dtype, to):
    g = torch.Generator(device=dev()).manual_seed(T)
    d = (1.0 + torch.rand(T, H, device=dev(), generator=g)).to(dtype)
    dx = molt.dropout_bwd(d, 0.25, 99, offset=8, dtype=to)
    check(dx, reference(d, kept(T, H, 0.25, 99, 8), 0.25), d, None, to, 0.25)
    ones = molt.dropout_fwd(torch.ones(T, H, device=dev()), 0.25, 99, offset=8)
    assert torch.equal(dx != 0, ones != 0)
    # along a direction, out is linear in x: its difference quotient is the gradient
    v = torch.randn(T, H, device=dev(), generator=g)
    a = molt.dropout_fwd(v, 0.25, 99, offset=8)
    left, right = float((a.double() * d.double()).sum()), float((v.double() * dx.double()).sum())
    # both sides' roundings, of the terms
    assert abs(left - right) <= (U[to] + 2.0**-22) * float((v.double() * dx.double()).abs().sum())


def test_share_of_the_dropped():
    """Half a million elements: five standard deviations."""
    x = torch.ones(512, 1024, device=dev())
    for p in (0.05, 0.1, 0.5, 0.9):
        n = x.numel()
        dropped = int((molt.dropout_fwd(x, p, 3) == 0).sum())
        q = np.floor(p * 65536 + 0.5) / 65536
        assert abs(dropped - q * n) <= 5 * (n * q * (1 - q))**0.5
    a, b = molt.dropout_fwd(x, 0.5, 3) != 0, molt.dropout_fwd(x, 0.5, 3, offset=1) != 0
    c = molt.dropout_fwd(x, 0.5, 4) != 0
    for other in (b, c, a.roll(1, 0), a.roll(1, 1), a.roll(8, 1)):
        assert abs(int((a == other).sum()) - n / 2) <= 5 * (n / 4)**0.5


def test_parts_of_a_batch():
    """Rows taken apart drop what they drop together."""
    x = torch.randn(700, 333, device=dev())
    whole = molt.dropout_fwd(x, 0.3, 11, offset=2)
    parts = [molt.dropout_fwd(x[a:b], 0.3, 11, offset=2, first_row=a) for a, b in ((0, 1), (1, 300), (300, 700))]
    assert torch.equal(whole, torch.cat(parts))
    # the last rows that a 32-bit counter has
    last = molt.dropout_fwd(x[:10, :64], 0.3, 11, first_row=(1 << 32) - 10)
    assert torch.equal(last != 0, kept(10, 64, 0.3, 11, 0, (1 << 32) - 10))


@pytest.mark.parametrize("H", [64, 37])
def test_dropped_values_are_left_out(H):
    """Infinities and NaN that are dropped leave no trace."""
    T = 50
    keep = kept(T, H, 0.5, 21)
    x = torch.where(keep, 1.0, float("nan"))
    x[::2] = torch.where(keep[::2], 1.0, float("inf"))
    out = molt.dropout_fwd(x, 0.5, 21)
    assert torch.equal(out, torch.where(keep, 2.0, 0.0))
    r = torch.randn(T, H, device=dev())
    assert molt.dropout_fwd(x, 0.5, 21, residual=r).isfinite().all()


def test_strides_alignment_and_in_place():
    T = 130
    for H, pad in ((64, 64), (64, 3), (72, 8), (51, 1)):
        for dtype in (BF, F32):
            base = torch.randn(T, H + pad, device=dev()).to(dtype)
            x, r = base[:, :H], torch.randn(T, H + pad, device=dev()).to(dtype)[:, pad:]
            want = molt.dropout_fwd(x.contiguous(), 0.2, 5, residual=r.contiguous(), res_scale=0.5)
            assert torch.equal(molt.dropout_fwd(x, 0.2, 5, residual=r, res_scale=0.5), want)
            off = torch.empty(T * H + 1, dtype=dtype, device=dev())[1:].view(T, H)
            assert torch.equal(molt.dropout_fwd(x, 0.2, 5, residual=r, res_scale=0.5, out=off), want)
            xc, rc = x.contiguous(), r.contiguous()
            assert molt.dropout_fwd(xc, 0.2, 5, residual=rc, res_scale=0.5, out=rc) is rc and torch.equal(rc, want)
            plain = molt.dropout_fwd(x, 0.2, 5)
            assert molt.dropout_fwd(xc, 0.2, 5, out=xc) is xc and torch.equal(xc, plain)
    with pytest.raises(molt.MoltError, match="in place"):
        molt.dropout_fwd(base[:, :H], 0.2, 5, out=torch.as_strided(base, (T, H), (H, 1)))
    with pytest.raises(ValueError, match="shape"):
        molt.dropout_fwd(base, 0.2, 5, out=base[:3])
    with pytest.raises(ValueError, match="seed"):
        molt.dropout_fwd(base, 0.2, -1)
    with pytest.raises(ValueError, match="offset"):
        molt.dropout_fwd(base, 0.2, torch.zeros(2, dtype=torch.int64, device=dev()), offset=3)
    with pytest.raises(TypeError, match="seed"):
        molt.dropout_fwd(base, 0.2, torch.zeros(2, dtype=torch.int32, device=dev()))


@pytest.mark.parametrize("H", [5, 8])
def test_rows_far_apart(H):
    """160 rows, 2^25 elements from one to the next: offsets past 32 bits within a tile."""
    T, ld = 160, 1 << 25
    x = torch.empty(T * ld, dtype=BF, device=dev()).as_strided((T, H), (ld, 1))
    x.copy_(torch.arange(1, T * H + 1, device=dev()).view(T, H))
    for r in (None, x):
        got = molt.dropout_fwd(x, 0.3, 11, residual=r)
        assert torch.equal(got, molt.dropout_fwd(x.contiguous(), 0.3, 11, residual=None if r is None else r.contiguous()))
    assert float(got.float().abs().sum()) > 0


def test_no_rows():
    assert molt.dropout_fwd(torch.empty(0, 64, device=dev()), 0.1, 1).shape == (0, 64)


def test_a_replayed_graph_draws_what_its_seed_says():
    T, H = 300, 320
    x, r = torch.randn(T, H, device=dev()).to(BF), torch.randn(T, H, device=dev())
    words = torch.tensor([1, 2], dtype=torch.int64, device=dev())

    def calls():
        return molt.dropout_fwd(x, 0.1, words, residual=r), molt.dropout_bwd(x, 0.1, words)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    for seed, offset in ((1, 2), (5, 0), (-3, 1 << 40)):
        words.copy_(torch.tensor([seed, offset]))
        graph.replay()
        torch.cuda.synchronize()
        n = seed % (1 << 64)
        assert torch.equal(out[0], molt.dropout_fwd(x, 0.1, n, offset=offset, residual=r))
        assert torch.equal(out[1], molt.dropout_bwd(x, 0.1, n, offset=offset))
