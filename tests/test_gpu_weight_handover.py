"""Weights that were written on the stream a moment ago: the products read theirs ahead of the kernel in front, and a norm between the two
is enough to keep them apart."""
import pytest
import torch

from operator_helpers import DEV, gen, heavy
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("op", ["matvec", "gated_matvec", "gated_gemm"])
@pytest.mark.parametrize("M,rows,K", [(1, 256, 4096), (3, 2048, 1024), (12, 256, 2048), (40, 8192, 512)])
def test_a_norm_keeps_the_writer_of_the_weights_and_the_product_apart(op, M, rows, K):
    """The writer is a rotation, which lets the kernel behind it start at once; new weights in the same place at every step.  Each
    step gives what it gives when the host waits in between."""
    g, steps = gen(M + rows), 12
    V = (heavy(g, steps, rows, K) * 0.1).to(torch.bfloat16)
    R = torch.eye(K, dtype=torch.bfloat16, device=DEV)[torch.randperm(K, generator=g, device=DEV)]
    x = heavy(g, steps, M, K).to(torch.bfloat16)
    weight = torch.ones(K, dtype=torch.bfloat16, device=DEV)
    codes = torch.empty(rows, K // 2, dtype=torch.uint8, device=DEV)
    Ws = torch.empty(torq.torq_scales_bytes(rows, K), dtype=torch.uint8, device=DEV)
    y = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    a = torq.torq_quantize_mxfp4(x[0].float())
    Y = torch.empty(2, steps, M, rows if op == "matvec" else rows // 2, dtype=torch.float32, device=DEV)

    def step(i, out, wait=lambda: None):
        torq.torq_rotate_quantize(V[i], R, None, out_codes=codes, out_scales=Ws)
        wait()
        torq.torq_add_rmsnorm(x[i], weight, out=y)
        if op == "gated_gemm":
            torq.torq_mxfp4_gated_gemm(*a, codes, Ws, Y=out)
        else:
            getattr(torq, f"torq_mxfp4_{op}")(y, codes, Ws, Y=out)
        wait()

    for i in range(steps):
        step(i, Y[0, i], torch.cuda.synchronize)
    assert not any(torch.equal(Y[0, i], Y[0, i - 1]) for i in range(1, steps))
    graph = torch.cuda.CUDAGraph()                       # without the host between them
    with torch.cuda.graph(graph):
        for i in range(steps):
            step(i, Y[1, i])
    for _ in range(5):
        Y[1].zero_()
        codes.fill_(0x77)                                # 6 everywhere
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y[0], Y[1])
    assert torq.torq_last_device_error() == 0
