"""`stream` of the calls around the LM head: what they return is allocated and filled on that stream (the current one
is held back by a kernel that counts clocks)."""
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
HOLD = 200_000_000   # clocks
NAMES = ["embedding", "embedding bwd", "norm", "norm bwd added", "ce", "ce bwd", "logprobs", "loss", "advantages"]


def calls():
    g = torch.Generator(device=dev()).manual_seed(1)
    n = lambda *s: torch.randn(*s, device=dev(), generator=g)
    T, H, V = 512, 512, 1024
    x, dy, r, W = n(T, H).to(BF), n(T, H).to(BF), n(T, H), (n(V, H) * H ** -0.5).to(BF)
    w = 1 + 0.1 * n(H)
    tokens = torch.randint(0, V, (T,), device=dev(), generator=g).to(torch.int32)
    s = molt.residual_norm_fwd(x, r, w_pre=w)
    logp, adv = molt.token_logprobs(x, W, tokens)[0], n(T)
    rewards, groups = n(64), (torch.arange(64, device=dev()) // 8).to(torch.int32)
    pair = lambda t: dict(zip("ab", t))
    return {
        "embedding": lambda **k: {"x": molt.token_embedding(W, tokens, **k)},
        "embedding bwd": lambda **k: {"dW": molt.token_embedding_bwd(dy, tokens, V, **k)},
        "norm": lambda **k: molt.residual_norm_fwd(x, r, w_pre=w, **k),
        "norm bwd added": lambda **k: molt.residual_norm_bwd(dy, r, x, s["residual"], s["rstd_pre"], w_pre=w, accumulate=True, **k),
        "ce": lambda **k: molt.cross_entropy_fwd(x, W, tokens, **k),
        "ce bwd": lambda **k: molt.cross_entropy_fwd_bwd(x, W, tokens, dW_dtype=BF, **k),
        "logprobs": lambda **k: pair(molt.token_logprobs(x, W, tokens, **k)),
        "loss": lambda **k: molt.policy_loss_fwd_bwd(x, W, tokens, logp, adv, **k),
        "advantages": lambda **k: {"a": molt.group_advantages(rewards, groups, **k)},
    }


def held(out):
    return {k: t for k, t in out.items() if t is not None}


@pytest.mark.parametrize("name", NAMES)
def test_outputs_belong_to_the_stream(name):
    f = calls()[name]
    want = held(f())
    shapes = [(t.shape, t.dtype) for t in want.values()]
    s = torch.cuda.Stream()
    f(stream=s)                       # (workspaces, and s's own pool)
    torch.cuda.synchronize()
    here = [torch.full(shape, 3.0, device=dev()).to(dtype) for shape, dtype in shapes for _ in range(3)]
    read = [torch.empty_like(t) for t in here]
    torch.cuda.synchronize()
    torch.cuda._sleep(HOLD)
    for i, t in enumerate(here):
        read[i].copy_(t)              # still to come
    del here, t
    out = held(f(stream=s))
    s.synchronize()
    assert not torch.cuda.current_stream().query(), "the current stream was not held back for long enough"
    torch.cuda.synchronize()
    assert all((t == 3).all() for t in read) and set(out) == set(want)
    # (the loss's fp32 sums have no fixed order: a bf16 result may fall to the next number, 2^-7 of it)
    for k, v in want.items():
        assert torch.allclose(out[k].double(), v.double(), rtol=1e-2, atol=1e-5), k
    assert molt.device_status() == 0
