"""What the gated products leave of the host's work for the plain GEMMs beside them."""
import time

import pytest
import torch

from operator_helpers import DEV
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu


def test_gated_calls_leave_the_plans_of_plain_gemms_alone():
    """The tile lists of the last eight shapes are kept, as their search takes longer than the rest of a call: eight plain GEMMs cost the
    host the same whether gated ones of other shapes come between or not (10.0 us each; 16.4 when the gated ones took places in the list).
    The quickest of many rounds on either side, taken in turn."""
    def operands(M, N, K=128):
        full = lambda n, v: torch.full((n,), v, dtype=torch.uint8, device=DEV)
        return (full(M * K // 2, 0x22).view(M, -1), full(torq.torq_scales_bytes(M, K), 120), full(N * K // 2, 0x22).view(N, -1),
                full(torq.torq_scales_bytes(N, K), 120))

    plain = [operands(1024 + 256 * i, 256 * (37 + 3 * i)) for i in range(8)]
    gated = [operands(1500 + 256 * i, 256 * (40 + 2 * i)) for i in range(2)]

    def host_time(between):
        total = 0.0
        for _ in range(5):
            for o in between:
                torq.torq_mxfp4_gated_gemm(*o)
            start = time.perf_counter()
            for o in plain:
                torq.torq_mxfp4_gemm(*o)
            total += time.perf_counter() - start
        torch.cuda.synchronize()
        return total

    host_time(gated), host_time([])
    alone, beside = (min(t) for t in zip(*((host_time([]), host_time(gated)) for _ in range(40))))
    assert beside < 1.35 * alone, (alone, beside)
