"""Token embedding, residual norm and their gradients in one captured graph, as a training or
decoding loop would replay them: on new inputs, with the bits of the calls outside of it."""
import ctypes

import pytest
import torch

import paper_2607_21653_gb300 as molt
from paper_2607_21653_gb300 import stream as S
from parity import dev

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T,H,V", [(1, 4096, 1000), (700, 320, 3000), (5000, 1031, 700)])
def test_in_a_captured_graph(T, H, V):
    g = torch.Generator(device=dev()).manual_seed(T)
    n = lambda *s: torch.randn(*s, device=dev(), generator=g)
    E, w, gate = n(V, H).to(BF), 1 + 0.1 * n(H), n(H)
    x = torch.randint(0, V, (T,), device=dev(), generator=g).to(torch.int32)
    r, dy, dr = n(T, H), n(T, H).to(BF), n(T, H)
    desc = S.NormDesc(T, H, 0, 0, 0, 0, 2, 2, S.GATE_CHANNEL, 1.0, 1e-6, 0.0)
    nbytes = molt.load().molt_residual_norm_bwd_workspace_bytes(ctypes.byref(desc))
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev())
    ws_e = torch.empty(molt.load().molt_token_embedding_bwd_workspace_bytes(T, H, V), dtype=torch.uint8, device=dev())

    def calls():
        kw = dict(w_post=w, gate=gate, w_pre=w, gate_kind="channel")
        e = molt.token_embedding(E, x, scale=2.0)
        o = molt.residual_norm_fwd(e, r, **kw)
        b = molt.residual_norm_bwd(dy, dr, e, o["residual"], o["rstd_pre"], rstd_post=o["rstd_post"], workspace=ws, **kw)
        dE = molt.token_embedding_bwd(b["dx"], x, V, scale=2.0, workspace=ws_e)
        return {"e": e, **{"f_" + k: v for k, v in o.items()}, **b, "dE": dE}

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    for seed in (1, 2):
        g.manual_seed(seed)
        x.copy_(torch.randint(0, V, (T,), device=dev(), generator=g))
        r.copy_(n(T, H))
        dy.copy_(n(T, H))
        graph.replay()
        got = {k: v.clone() for k, v in out.items()}
        want = calls()
        assert set(got) == set(want)
        for k, v in want.items():
            assert torch.equal(v, got[k]), k
    assert molt.device_status() == 0
