"""Products of few tokens with 4-bit weights, plain and gated, on a GPU, against their definition in 64 bits on the same inputs."""
import pytest
import torch

from operator_helpers import (DEV, check_gated, check_sums, code_values, gen, heavy, matvec_error, quantized, tile, values)
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu
FMTS = ("mxfp4", "nvfp4", "mxint4")


def matvec(fmt, X, W, gated=False, **kw):
    f = getattr(torq, f"torq_{fmt}_{'gated_' if gated else ''}matvec")
    return f(X, W[0], W[1], W[2], **kw) if fmt == "nvfp4" else f(X, W[0], W[1], **kw)


def launches(M, N, K):
    return 2 if torq.torq_matvec_workspace_bytes(M, N, K) else 1


def tokens(g, M, K):
    x = heavy(g, M, K)
    x[:, torch.randperm(K, generator=g, device=DEV)[:2]] *= 100
    if M > 2:
        x[1] = 0                                         # a token of zeros
    if M > 4:
        x[3] *= 1e-30                                    # one of tiny numbers
        x[4] *= 1e25                                     # one of huge ones
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("N,K", [(8, 128), (136, 256), (200, 384), (1000, 640), (264, 1408), (4096, 1024), (512, 14336), (20480, 2304)])
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 33, 70])
def test_matvec(fmt, M, N, K):
    g = gen(M * 1000 + N)
    W = quantized(g, N, K, fmt, pad=0xFF)                # padding rows whose scales are not numbers
    X = tokens(g, M, K)
    dtype = torch.float32 if (M + N // 8) % 2 else torch.bfloat16
    buf = torch.full((M * N + 64,), 7.0, dtype=dtype, device=DEV)
    before = torq.torq_launch_count()
    Y = matvec(fmt, X, W, Y=buf[:M * N].view(M, N))
    assert torq.torq_launch_count() == before + launches(M, N, K)
    check_sums(Y, X.double(), W[3], *matvec_error(fmt, X.double()))
    assert (buf[M * N:] == 7).all()
    assert torq.torq_last_device_error() == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("N,K", [(128, 128), (256, 384), (384, 1408), (2048, 4096), (14336, 512), (25600, 2304)])
@pytest.mark.parametrize("M", [1, 5, 8, 13, 17, 40])
def test_gated_matvec(fmt, M, N, K):
    g = gen(M * 1000 + N + 1)
    W = quantized(g, 2 * N, K, fmt)
    X = tokens(g, M, K)
    X = (X.double() * 0.05).to(torch.bfloat16)
    dtype = torch.bfloat16 if (M + N // 128) % 2 else torch.float32
    buf = torch.full((M * N + 64,), 7.0, dtype=dtype, device=DEV)
    before = torq.torq_launch_count()
    Y = matvec(fmt, X, W, gated=True, Y=buf[:M * N].view(M, N))
    assert torq.torq_launch_count() == before + launches(M, N, K)
    fine = [m for m in range(M) if m != 4 or M <= 4]     # the product of two huge sums has no float32
    check_gated(Y[fine], X.double()[fine], W[3], *matvec_error(fmt, X.double()[fine]))
    assert (buf[M * N:] == 7).all()


@pytest.mark.parametrize("fmt", ["mxfp4", "mxint4"])
def test_block_scales_at_the_ends(fmt):
    """E8M0 bytes 0 (2^-127) and far apart from one another: each block keeps its own power of two."""
    g, N, K = gen(5), 128, 512
    codes = quantized(g, N, K, fmt)[0]
    lin = torch.randint(0, 200, (N, K // 32), generator=g, device=DEV).to(torch.uint8)
    lin[:64] = torch.randint(0, 3, (64, K // 32), generator=g, device=DEV).to(torch.uint8)
    X = heavy(g, 3, K).to(torch.bfloat16)
    X[1] = (X[1].double() * 2.0 ** 40).to(torch.bfloat16)
    Y = matvec(fmt, X, (codes, tile(lin), 1.0), out_dtype=torch.float32)
    check_sums(Y, X.double(), values(codes, lin, fmt), *matvec_error(fmt, X.double()))


@pytest.mark.parametrize("fmt", FMTS)
def test_small_elements_beside_large_ones(fmt):
    """Elements down to 2^-14 of their block's largest count in full: the large ones meet codes of zero."""
    g, N, K = gen(6), 64, 256
    large = 2.0 ** 12
    codes, Ws, ts, v = quantized(g, N, K, fmt)
    codes[:, 0] = 0
    v[:, :2] = 0
    X = heavy(g, 2, K).to(torch.bfloat16).clamp(-1, 1)
    X[X.abs() < 0.25] = 0.5
    X[:, 0] = large
    Y = matvec(fmt, X, (codes, Ws, ts), out_dtype=torch.float32)
    rest = torch.cat([X[:, :2] * 0, X[:, 2:]], 1).double()
    check_sums(Y, rest, v, matvec_error(fmt, rest)[0])


def test_every_code_and_position():
    """One element of x at a time: every code of every position of a block arrives with its own value."""
    K, N = 256, 16
    for fmt in FMTS:
        codes = torch.arange(16, device=DEV, dtype=torch.uint8).view(N, 1) * 0x11
        codes = codes.expand(N, K // 2).contiguous()
        lin = torch.full((N, K // (16 if fmt == "nvfp4" else 32)), 0x38 if fmt == "nvfp4" else 127, dtype=torch.uint8, device=DEV)
        X = torch.eye(K, device=DEV, dtype=torch.bfloat16)
        Y = matvec(fmt, X, (codes, tile(lin), 1.0), out_dtype=torch.float32)
        assert torch.equal(Y.double(), code_values(codes, fmt).t())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("gated", [False, True])
def test_what_is_not_a_number_stays_in_its_token(fmt, gated):
    g, N, K = gen(7), 256, 640
    W = quantized(g, 2 * N if gated else N, K, fmt)
    X = heavy(g, 6, K).to(torch.bfloat16)
    clean = matvec(fmt, X, W, gated)
    X[2, 130] = float("nan")
    X[4, 7] = float("inf")
    Y = matvec(fmt, X, W, gated)
    assert not torch.isfinite(Y[2]).any() and not torch.isfinite(Y[4]).all()
    for m in (0, 1, 3, 5):
        assert torch.equal(Y[m], clean[m])


@pytest.mark.parametrize("fmt", FMTS)
def test_a_token_does_not_depend_on_its_batch(fmt):
    """Bit for bit at every batch that the same instance of the kernel serves, and from call to call."""
    g, N, K = gen(8), 1024, 2048
    W = quantized(g, N, K, fmt)
    X = heavy(g, 8, K).to(torch.bfloat16)
    for some, one in (((0, 8), 6), ((0, 4), 2)):
        x = X[some[0]:some[1]].contiguous()
        Y = matvec(fmt, x, W, out_dtype=torch.float32)
        for _ in range(5):
            assert torch.equal(matvec(fmt, x, W, out_dtype=torch.float32), Y)
        x[one] = X[one + 1 if one > 4 else 0]            # another token changes nothing in the others
        Z = matvec(fmt, x, W, out_dtype=torch.float32)
        rest = [m for m in range(x.shape[0]) if m != one]
        assert torch.equal(Z[rest], Y[rest])
    assert torch.equal(matvec(fmt, X[3:4].contiguous(), W, out_dtype=torch.float32), matvec(fmt, X[2:4].contiguous(), W, out_dtype=torch.float32)[1:])


@pytest.mark.parametrize("fmt", FMTS)
def test_workspace(fmt):
    """The caller's own is enough, whatever it held; too small a one is refused."""
    g, M, N, K = gen(11), 6, 256, 640
    W = quantized(g, N, K, fmt)
    X = heavy(g, M, K).to(torch.bfloat16)
    want = matvec(fmt, X, W)
    ws = torch.full((torq.torq_matvec_workspace_bytes(M, N, K) + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    assert torch.equal(matvec(fmt, X, W, workspace=ws[:-64]), want)
    assert (ws[-64:] == 0xFF).all()
    with pytest.raises(torq.TorqError) as e:
        matvec(fmt, X, W, workspace=ws[:256])
    assert e.value.code == 7


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,K", [(3, 65536), (12, 40960), (20, 28672), (40, 57344)])
def test_long_contractions(fmt, gated, M, K):
    """Where fewer tokens go together than otherwise."""
    g, N = gen(K), 128
    W = quantized(g, 2 * N if gated else N, K, fmt)
    X = (heavy(g, M, K) * 0.02).to(torch.bfloat16)
    Y = matvec(fmt, X, W, gated, out_dtype=torch.float32)
    (check_gated if gated else check_sums)(Y, X.double(), W[3], *matvec_error(fmt, X.double()))


@pytest.mark.parametrize("native", [True, False])
def test_stream_argument(native, monkeypatch):
    """A call on another stream than the current one, its workspace taken from the current one's pool: calls on both at once, with
    the memory that the first has given back taken and overwritten at once."""
    if not native:
        monkeypatch.setattr(torq, "_product_native", lambda *a: -1)
    g, M = gen(3), 7
    W = quantized(g, 4096, 4096, "mxfp4")
    X = heavy(g, M, 4096).to(torch.bfloat16)
    want = matvec("mxfp4", X, W)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    size = torq.torq_matvec_workspace_bytes(M, 4096, 4096)
    for _ in range(20):
        got = [matvec("mxfp4", X, W, stream=s) for _ in range(3)]
        torch.full((size,), 0x55, dtype=torch.uint8, device=DEV)
        also = matvec("mxfp4", X, W)
        torch.cuda.synchronize()
        assert all(torch.equal(y, want) for y in (*got, also))


def test_refusals():
    g = gen(1)
    W = quantized(g, 256, 256, "mxfp4")
    X = heavy(g, 4, 256).to(torch.bfloat16)
    bad = [lambda: torq.torq_mxfp4_matvec(X.float(), W[0], W[1]),                     # type
           lambda: torq.torq_mxfp4_matvec(X.cpu(), W[0], W[1]),                       # device
           lambda: torq.torq_mxfp4_matvec(X.t().contiguous().t(), W[0], W[1]),        # strides
           lambda: torq.torq_mxfp4_matvec(X[:, :128].contiguous(), W[0], W[1]),       # K
           lambda: torq.torq_mxfp4_matvec(X[0], W[0], W[1]),                          # dimensions
           lambda: torq.torq_mxfp4_matvec(X, W[0], W[1][:-1]),                        # too few scales
           lambda: torq.torq_mxfp4_matvec(X, W[0].float(), W[1]),
           lambda: torq.torq_mxfp4_matvec(X, W[0], W[1], Y=torch.empty(4, 255, dtype=torch.bfloat16, device=DEV)),
           lambda: torq.torq_mxfp4_matvec(X, W[0], W[1], Y=torch.empty(4, 256, dtype=torch.float16, device=DEV)),
           lambda: torq.torq_mxfp4_matvec(X, W[0], W[1], out_dtype=torch.float16),
           lambda: torq.torq_nvfp4_matvec(X, W[0], W[1], 1.0),                        # NVFP4 has twice the scale bytes
           lambda: torq.torq_mxfp4_gated_matvec(X, W[0][:255], W[1])]                 # an odd number of rows
    before = torq.torq_launch_count()
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f, code in ((lambda: torq.torq_mxfp4_matvec(X[:0], W[0], W[1]), 1),           # no elements, no address
                    (lambda: torq.torq_mxfp4_gated_matvec(X, W[0][:128], W[1]), 2),   # 64 features: no whole scale tiles
                    (lambda: torq.torq_mxfp4_matvec(X, W[0][:250], W[1]), 2),
                    (lambda: torq.torq_nvfp4_matvec(X, W[0][:64], torch.zeros(4096, dtype=torch.uint8, device=DEV), 0.0), 2)):
        with pytest.raises(torq.TorqError) as e:
            f()
        assert e.value.code == code
    assert torq.torq_launch_count() == before


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("gated,M,N,K", [(False, 17, 13320, 128), (False, 32, 13832, 640), (False, 33, 6920, 1408), (False, 64, 20480, 384), (False, 100, 3336, 2048),
                                         (False, 513, 1000, 384), (False, 2085, 136, 128), (True, 9, 19072, 128), (True, 17, 3840, 640), (True, 31, 5632, 1152),
                                         (True, 100, 1024, 2048), (True, 257, 384, 384), (True, 1027, 128, 128)])
def test_more_tokens(fmt, gated, M, N, K):
    """Where 32 tokens share a tile: workspaces and padding scales that hold no numbers, nothing written behind Y, a token that is not a
    number, a captured call."""
    g = gen(M + N + K)
    W = quantized(g, 2 * N if gated else N, K, fmt, pad=0xFF)
    X = (heavy(g, M, K) * 0.1).to(torch.bfloat16)
    X[2] = 0
    buf = torch.full((M * N + 64,), 7.0, dtype=torch.float32 if M % 2 else torch.bfloat16, device=DEV)
    Y = buf[:M * N].view(M, N)
    ws = torch.full((torq.torq_matvec_workspace_bytes(M, N, K),), 0xFF, dtype=torch.uint8, device=DEV)
    matvec(fmt, X, W, gated, Y=Y, workspace=ws)
    (check_gated if gated else check_sums)(Y, X.double(), W[3], *matvec_error(fmt, X.double()))
    clean = Y.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        matvec(fmt, X, W, gated, Y=Y, workspace=ws)
    X[M - 2, K // 2] = float("nan")
    Y.zero_()
    graph.replay()
    rest = [m for m in range(M) if m != M - 2]
    assert not torch.isfinite(Y[M - 2]).any() and torch.equal(Y[rest], clean[rest])
    assert (buf[M * N:] == 7).all()
    assert torq.torq_last_device_error() == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 256, 512), (4, 128, 1024), (6, 256, 512), (24, 13824, 512), (17, 3840, 512)])
def test_calls_in_a_row_share_memory(fmt, gated, M, N, K):
    """Launches overlap: a norm writes x while the product before it may still run and the one behind it has been started, all on one x
    and one workspace.  Each gives what it gives alone."""
    g, calls = gen(M + N), 40
    W = quantized(g, 2 * N if gated else N, K, fmt)
    X = (heavy(g, calls, M, K) * 3).to(torch.bfloat16)
    weight = torch.ones(K, dtype=torch.bfloat16, device=DEV)
    x = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(torq.torq_matvec_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV)
    Y = torch.empty(2, calls, M, N, dtype=torch.bfloat16, device=DEV)

    def both(i, y):
        torq.torq_add_rmsnorm(X[i], weight, out=x)
        matvec(fmt, x, W, gated, Y=y[i], workspace=ws)

    for i in range(calls):
        both(i, Y[0])
        torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()                       # without the host between them
    with torch.cuda.graph(graph):
        for i in range(calls):
            both(i, Y[1])
    for _ in range(3):
        Y[1].zero_()
        graph.replay()
        assert torch.equal(Y[0], Y[1])
    assert torq.torq_last_device_error() == 0
