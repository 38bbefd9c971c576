"""The operators around the layer, what needs no GPU: argument errors of the C entry points are status codes before anything
touches a device, and the Python calls refuse tensors that are not the current GPU's."""
import ctypes
import os
import re

import pytest
import torch

from paper_2605_19561_b200 import torq

CSRC = os.path.join(os.path.dirname(torq.__file__), "csrc")
ONE, ODD = ctypes.c_void_p(16), ctypes.c_void_p(24)      # never dereferenced on these paths
NULL, SHAPE, ALIGN, WORKSPACE = 1, 2, 3, 7


@pytest.mark.parametrize("mx", [False, True])
def test_norm_argument_errors(mx):
    L = torq.lib()

    def call(X=ONE, xt=1, r=None, ro=None, rt=1, w=ONE, eps=1e-6, M=4, d=64, out=ONE, scales=ONE):
        if mx:
            return L.torq_add_rmsnorm_mxfp8(X, xt, r, ro, rt, w, eps, M, d, out, scales, None)
        return L.torq_add_rmsnorm(X, xt, r, ro, rt, w, eps, M, d, out, None)

    assert call(X=None) == NULL and call(w=None) == NULL and call(out=None) == NULL
    if mx:
        assert call(scales=None) == NULL and call(scales=ODD) == ALIGN
    assert call(r=ONE) == NULL and call(ro=ONE) == NULL                            # one without the other
    assert call(M=0) == SHAPE and call(M=-3) == SHAPE and call(M=1 << 40) == SHAPE
    assert call(d=0) == SHAPE and call(d=48) == SHAPE and call(d=16416) == SHAPE
    assert call(xt=2) == SHAPE and call(r=ONE, ro=ONE, rt=5) == SHAPE
    assert call(eps=-1e-6) == SHAPE and call(eps=float("nan")) == SHAPE and call(eps=float("inf")) == SHAPE
    assert call(X=ODD) == ALIGN and call(w=ODD) == ALIGN and call(out=ODD) == ALIGN and call(r=ODD, ro=ONE) == ALIGN
    assert call(r=ONE, ro=ODD) == ALIGN


def test_norm_refuses_host_tensors():
    x = torch.zeros(2, 128, dtype=torch.bfloat16)
    for f in (lambda: torq.torq_add_rmsnorm(x, x[0]), lambda: torq.torq_add_rmsnorm_mxfp8(x, x[0]), lambda: torq.torq_add_rmsnorm(None, x[0])):
        with pytest.raises(ValueError):
            f()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4", "mxint4"])
def test_matvec_argument_errors(fmt, gated):
    f = getattr(torq.lib(), f"torq_{fmt}_{'gated_' if gated else ''}matvec")

    def call(X=ONE, W=ONE, s=ONE, ts=1.0, M=3, N=128, K=256, Y=ONE, t=0, ws=None, n=0):
        return f(X, W, s, *((ts,) if fmt == "nvfp4" else ()), M, N, K, Y, t, ws, n, None)

    for k in ("X", "W", "s", "Y"):
        assert call(**{k: None}) == NULL and call(**{k: ODD}) == ALIGN
    assert call(M=0) == SHAPE and call(M=(1 << 18) + 1) == SHAPE
    assert call(K=192) == SHAPE and call(K=0) == SHAPE and call(K=65536 + 128) == SHAPE and call(K=1 << 25) == SHAPE
    assert call(N=0) == SHAPE and call(N=-128) == SHAPE and call(N=132) == SHAPE and call(N=1 << 30) == SHAPE
    if gated:
        assert call(N=64) == SHAPE and call(N=192) == SHAPE
    assert call(t=2) == SHAPE
    need = torq.torq_matvec_workspace_bytes(5, 128, 256)
    assert torq.torq_matvec_workspace_bytes(4, 128, 256) == 0 and need >= 5 * 8 * 128 + 512
    assert torq.torq_matvec_workspace_bytes(1, 51200, 5120) > 0 and torq.torq_matvec_workspace_bytes(0, 128, 256) == 0   # a long range for one CTA
    big = ctypes.c_void_p(256)
    assert call(M=5) == WORKSPACE and call(M=5, ws=big, n=need - 1) == WORKSPACE and call(M=5, ws=None, n=need) == WORKSPACE
    assert call(M=5, ws=ctypes.c_void_p(128), n=need) == ALIGN
    if fmt == "nvfp4":
        assert call(ts=0.0) == SHAPE and call(ts=-1.0) == SHAPE and call(ts=float("inf")) == SHAPE and call(ts=float("nan")) == SHAPE


def test_matvec_refuses_host_tensors():
    x, w, s = torch.zeros(2, 128, dtype=torch.bfloat16), torch.zeros(128, 64, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    for f in (lambda: torq.torq_mxfp4_matvec(x, w, s), lambda: torq.torq_mxint4_gated_matvec(x, w, s), lambda: torq.torq_nvfp4_matvec(None, w, s, 1.0)):
        with pytest.raises(ValueError):
            f()


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4", "mxint4"])
def test_gated_gemm_argument_errors(fmt):
    f = getattr(torq.lib(), f"torq_{fmt}_gated_gemm")

    def call(A=ONE, sa=ONE, W=ONE, s=ONE, ta=1.0, tw=1.0, M=3, N=128, K=256, Y=ONE, t=0):
        if fmt == "nvfp4":
            return f(A, sa, ta, W, s, tw, M, N, K, Y, t, None)
        return f(A, sa, W, s, M, N, K, Y, t, None)

    for k in ("A", "sa", "W", "s", "Y"):
        assert call(**{k: None}) == NULL and call(**{k: ODD}) == ALIGN
    assert call(M=0) == SHAPE and call(M=(1 << 30) + 1) == SHAPE and call(M=1 << 30, N=1 << 29) == SHAPE
    assert call(K=192) == SHAPE and call(N=64) == SHAPE and call(N=192) == SHAPE and call(N=1 << 30) == SHAPE and call(t=7) == SHAPE
    if fmt == "nvfp4":
        assert call(ta=0.0) == SHAPE and call(tw=float("nan")) == SHAPE


def test_gated_gemm_refuses_host_tensors():
    w, s = torch.zeros(256, 64, dtype=torch.uint8), torch.zeros(1024, dtype=torch.uint8)
    for f in (torq.torq_mxfp4_gated_gemm, torq.torq_mxint4_gated_gemm):
        with pytest.raises(ValueError):
            f(w, s, w, s)


def test_every_role_waits_for_the_kernel_before_in_every_instance():
    """The few-token kernel's roles pass griddepcontrol.wait before their first wait that has a limit, and not only in some instances of
    the template."""
    body = re.sub(r"//.*", "", open(os.path.join(CSRC, "matvec.cuh")).read())
    body = body[re.search(r"^  griddep_launch_dependents\(\);", body, re.M).start():]
    while (m := re.search(r"(?:else )?if constexpr \([^{;]*\) \{", body)):
        end, depth = m.end(), 1
        while depth:
            depth += {"{": 1, "}": -1}.get(body[end], 0)
            end += 1
        body = body[:m.start()] + body[end:]
    roles = re.split(r"^  (?:if \(warp == \d+\) \{|\} else if \(warp == \d+\) \{|\} else \{)$", body, flags=re.M)[1:4]   # behind them the teardown
    assert len(roles) == 3
    for role in roles:
        assert "griddep_wait();" in role[:role.index("mbar_wait")]


@pytest.mark.parametrize("name", ["add_rmsnorm.cuh", "matvec.cuh", "mxfp4_gemm_pair.cuh"])
def test_nothing_that_the_kernel_before_may_write_is_read_as_read_only(name):
    """These kernels may start before the one in front has written their operands: no load of the read-only path, by name or by a
    pointer that the compiler may take for one."""
    code = re.sub(r"//.*", "", open(os.path.join(CSRC, name)).read())
    assert "__ldg" not in code and "ld.global.nc" not in code
    assert not re.search(r"const uint32_t\* __restrict__", code)


def test_the_norm_lets_the_next_kernel_start_behind_the_kernel_before():
    """What stands behind a norm reads its weights ahead of its wait: the norm, which may be all that is between it and what wrote them,
    passes griddepcontrol.wait first."""
    norm, ptx = (re.sub(r"//.*", "", open(os.path.join(CSRC, f)).read()) for f in ("add_rmsnorm.cuh", "sm100_ptx.cuh"))
    kernel = norm[norm.index("add_rmsnorm_kernel("):]
    calls = re.findall(r"griddep_\w+|griddepcontrol\.\w+", kernel)
    order = []
    for c in calls:
        body = re.search(r"void " + c + r"\(\) \{(.*?)\n?\}", ptx, re.S).group(1)
        order += re.findall(r"griddep_wait|griddep_launch_dependents", body) if "asm" not in body else [c]
    assert order == ["griddep_wait", "griddep_launch_dependents"]
