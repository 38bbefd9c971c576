"""Root-mean-square norm with the residual's addition on a GPU, against its definition in 64 bits on the same inputs."""
import math

import pytest
import torch

from paper_2605_19561_b200 import torq
from operator_helpers import DEV, NORM_REL, check_mxfp8, e4m3, gen, heavy, norm_inputs, norm_ref, tile, untile

pytestmark = pytest.mark.gpu
SIZES = [(1, 32), (3, 96), (5, 128), (2, 256), (9, 480), (4, 1024), (130, 1056), (7, 4096), (2, 5120), (500, 5120), (3, 8192), (400, 8192),
         (3, 8224), (2, 14336), (1, 16384), (333, 16384)]


@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("r_dtype", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,d", SIZES)
def test_norm(M, d, x_dtype, r_dtype):
    x, r, w = norm_inputs(M, d, x_dtype, r_dtype)
    ref = norm_ref(x, r, w, 1e-5)
    out = torch.full((M * d + 64,), 7.0, dtype=torch.bfloat16, device=DEV)
    before = torq.torq_launch_count()
    got = torq.torq_add_rmsnorm(x, w, r, 1e-5, out=out[:M * d].view(M, d))
    assert torq.torq_launch_count() == before + 1
    y = got if r is None else got[0]
    assert ((y.double() - ref).abs() <= (2.0 ** -8 + NORM_REL) * ref.abs() + 1e-40).all()
    assert (out[M * d:] == 7).all()
    if r is not None:                                    # one IEEE addition, one rounding
        assert torch.equal(got[1], (x.float() + r.float()).to(r_dtype))


@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("r_dtype", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,d", SIZES)
def test_norm_mxfp8(M, d, x_dtype, r_dtype):
    x, r, w = norm_inputs(M, d, x_dtype, r_dtype, seed=1)
    x[0, :32] = 0                                        # a block of zeros
    if r is not None:
        r[0, :32] = 0
    ref = norm_ref(x, r, w, 1e-6)
    n = torq.torq_scales_bytes(M, d)
    codes = torch.full((M * d + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    scales = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    before = torq.torq_launch_count()
    got = torq.torq_add_rmsnorm_mxfp8(x, w, r, 1e-6, out_bytes=codes[:M * d].view(M, d), out_scales=scales[:n])
    assert torq.torq_launch_count() == before + 1
    check_mxfp8(codes[:M * d].view(M, d), scales[:n], ref)
    assert (codes[M * d:] == 0xA5).all() and (scales[n:] == 0xA5).all()
    if r is not None:
        assert torch.equal(got[2], (x.float() + r.float()).to(r_dtype))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("M,d", [(1, 512), (5, 4096), (700, 5120)])
def test_norm_in_place(M, d, mx):
    f = torq.torq_add_rmsnorm_mxfp8 if mx else torq.torq_add_rmsnorm
    x, r, w = norm_inputs(M, d, torch.bfloat16, torch.bfloat16)
    want = f(x, w, r)
    for alias in ("residual", "x"):
        a, b = x.clone(), r.clone()
        got = f(a, w, b, residual_out=b if alias == "residual" else a)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        assert got[-1].data_ptr() == (b if alias == "residual" else a).data_ptr()


def test_values_at_the_ends():
    d = 256
    w = torch.ones(d, dtype=torch.bfloat16, device=DEV)
    x = torch.zeros(6, d, device=DEV)
    x[1] = 1e-30                                         # far below eps
    x[2] = 1e15                                          # squares of 1e30
    x[3, 0] = 5.0                                        # one element alone
    x[4] = torch.tensor([1.0, -1.0], device=DEV).repeat(d // 2)
    x[5, 5] = float("nan")
    y = torq.torq_add_rmsnorm(x, w)
    assert not y[0].any()
    ref = norm_ref(x, None, w, 1e-6)
    assert ((y.double() - ref).abs()[:5] <= (2.0 ** -8 + NORM_REL) * ref.abs()[:5] + 1e-40).all()
    assert y[5].isnan().all()                            # of one row alone
    codes, scales = torq.torq_add_rmsnorm_mxfp8(x, w)
    check_mxfp8(codes[:5], tile(untile(scales, 5, d // 32)), ref[:5])
    assert e4m3(codes[5]).isnan().all()


def test_refusals():
    X = heavy(gen(1), 4, 256).to(torch.bfloat16)
    w = X[0].contiguous()
    bad = [lambda: torq.torq_add_rmsnorm(X, w.float()), lambda: torq.torq_add_rmsnorm(X, w[:128]), lambda: torq.torq_add_rmsnorm(X.half(), w),
           lambda: torq.torq_add_rmsnorm(X.cpu(), w), lambda: torq.torq_add_rmsnorm(X.t().contiguous().t(), w),
           lambda: torq.torq_add_rmsnorm(X[0], w), lambda: torq.torq_add_rmsnorm(X, w, X[:3].contiguous()),
           lambda: torq.torq_add_rmsnorm(X, w, residual_out=X), lambda: torq.torq_add_rmsnorm(X, w, X, residual_out=X.float()),
           lambda: torq.torq_add_rmsnorm(X, w, out=X.float()),
           lambda: torq.torq_add_rmsnorm_mxfp8(X, w, out_scales=torch.empty(8, dtype=torch.uint8, device=DEV))]
    before = torq.torq_launch_count()
    for f in bad:
        with pytest.raises(ValueError):
            f()
    # a tensor without elements has no address
    for f, code in ((lambda: torq.torq_add_rmsnorm(X, w, eps=-1.0), 2), (lambda: torq.torq_add_rmsnorm(X, w, eps=math.nan), 2),
                    (lambda: torq.torq_add_rmsnorm(X[:0], w), 1)):
        with pytest.raises(torq.TorqError) as e:
            f()
        assert e.value.code == code
    assert torq.torq_launch_count() == before


@pytest.mark.parametrize("native", [True, False])
def test_stream_argument(native, monkeypatch):
    if not native:
        monkeypatch.setattr(torq, "_norm_native", lambda *a: -1)
    x, r, w = norm_inputs(64, 2048, torch.bfloat16, torch.bfloat16)
    want = torq.torq_add_rmsnorm_mxfp8(x, w, r)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        got = torq.torq_add_rmsnorm_mxfp8(x, w, r, stream=s)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
