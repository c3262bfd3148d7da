"""A split product under capture: refused with what to do about it while its stream has no workspace, and after
one call there recorded, with replays that give the eager result."""
import numpy as np
import pytest

from oracle import q8
from test_gpu_q8 import env, operand  # noqa: F401

pytestmark = pytest.mark.gpu


def test_refused_then_recorded(env):  # noqa: F811
    torch, L = env
    rng = np.random.default_rng(53)
    M, K, N = 40, 8192, 64
    a, _ = operand(torch, L, rng, M, K, q8.E4M3, q8.POW2, 1)
    b, _ = operand(torch, L, rng, N, K, q8.E4M3, q8.POW2, 128)
    want, c = torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda")
    L.ds_q8_matmul(a, b, want)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    err = None
    print("refused capture", flush=True)
    try:
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=st):
            try:
                L.ds_q8_matmul(a, b, c, stream=st)
            except RuntimeError as e:                  # raised before anything is recorded
                err = e
            c.zero_()                                  # keeps the captured graph non-empty
    finally:
        torch.cuda.synchronize()
    assert "DS_EUNSUPPORTED" in str(err) and "same call once on that stream" in str(err)
    L.ds_q8_matmul(a, b, c, stream=st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        L.ds_q8_matmul(a, b, c, stream=st)
    for i in range(3):
        c.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c, want), i
        L.ds_q8_matmul(a, b, want)                     # eager work between replays
        torch.cuda.synchronize()
