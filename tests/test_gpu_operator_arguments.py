"""Arguments of the operators that are refused where they used to pass or to fail as something else."""
import pytest
import torch

from operator_helpers import DEV, gen, heavy, quantized
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
def test_refusals(native, monkeypatch):
    if not native:
        monkeypatch.setattr(torq, "_product_native", lambda *a: -1)
    g = gen(1)
    W = quantized(g, 256, 256, "mxfp4")
    X = heavy(g, 8, 256).to(torch.bfloat16)
    A = quantized(g, 8, 256, "mxfp4")
    ws = torch.empty(torq.torq_matvec_workspace_bytes(8, 256, 256), dtype=torch.uint8, device=DEV)
    bad = [lambda: torq.torq_mxfp4_matvec(X, W[0], W[1], out_dtype=None), lambda: torq.torq_mxfp4_gated_gemm(A[0], A[1], W[0], W[1], out_dtype=None),
           lambda: torq.torq_mxfp4_matvec(X, W[0], W[1], workspace="a name"), lambda: torq.torq_mxfp4_gated_matvec(X, W[0], W[1], workspace=4096),
           lambda: torq.torq_mxfp4_matvec(X, W[0], W[1], workspace=ws.cpu()), lambda: torq.torq_mxfp4_matvec(X, W[0], W[1], workspace=ws[::2])]
    before = torq.torq_launch_count()
    for f in bad:
        with pytest.raises(ValueError):
            f()
    assert torq.torq_launch_count() == before
