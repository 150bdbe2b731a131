"""cat_linear against the formula in 64 bits.

Tolerance, written down before the first run.  S = sum_k |x w| + |b| bounds every partial sum of an output; the kernel adds K products
and the bias in some order, and each addition, rounded or truncated to fp32, errs by at most 2^-23 S: (K + 8) 2^-23 S in all.  The
activations' slopes are at most 1.13, and evaluating one in fp32 errs by at most 2^-19 of max(|y|, 2^-19) (a few functions of 2 ulp each,
arguments of exp up to 16 whose rounding counts sixteenfold).  The result is rounded once: eps / 2 of its magnitude, in fp16 at least
half its smallest number 2^-25, after one more addition of the residual (2^-24 of the result)."""
import math

import pytest
import torch

from paper_2509_26277_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, FH, F32 = torch.bfloat16, torch.float16, torch.float32
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def act64(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if act == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def want_and_bound(X, W, bias, residual, act, out_dtype):
    x, w = X.double(), W.double()
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    y = act64(z, act)
    err = 1.13 * (X.shape[1] + 8) * 2.0 ** -23 * size + (2.0 ** -19 * y.abs().clamp(min=2.0 ** -19) if act not in ("none", "relu") else 0)
    if residual is not None:
        y = y + residual.double()
    half = torch.finfo(out_dtype).eps / 2
    return y, err * 1.01 + (half + 2.0 ** -24) * (y.abs() + err) + torch.finfo(out_dtype).smallest_normal * half


def check(X, W, bias, residual, act, out_dtype, got):
    assert got.dtype == out_dtype
    want, bound = want_and_bound(X, W, bias, residual, act, out_dtype)
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside the bound, worst {float((off / bound).max()):.3g} of it"


def data(m, n, k, dtype, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000 * m + 10 * n + k)
    X = (torch.randn((m, k), generator=g, device="cuda") * scale).to(dtype)
    W = (torch.randn((n, k), generator=g, device="cuda") * k ** -0.5).to(dtype)
    return X, W, g


# one output; one token over one slab, many, none full; 16-token chunks and their edges; the last form of one CTA and the first of pairs;
# tiles of columns that are not full; inner dimensions off every boundary; more tiles than CTAs
SHAPES = [(1, 1, 1), (1, 8, 64), (1, 1000, 512), (2, 129, 63), (1, 4097, 65), (15, 128, 100), (16, 130, 4096), (17, 1000, 1001), (33, 64, 4104),
          (64, 300, 24), (100, 2048, 520), (127, 257, 999), (128, 256, 2048), (129, 255, 72), (160, 1000, 512), (255, 1024, 1000), (256, 512, 2056),
          (257, 513, 136), (300, 1, 4000), (1000, 3, 7), (513, 2049, 1003), (4100, 1000, 576), (5, 20000, 256), (2, 70_001, 40), (20_001, 333, 65)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [BF, FH])
def test_product(m, n, k, dtype):
    for i, out_dtype in enumerate([dtype, F32, FH if dtype == BF else BF]):
        X, W, g = data(m, n, k, dtype, seed=i)
        got = B.cat_linear(X, W, out_dtype=out_dtype)
        check(X, W, None, None, "none", out_dtype, got)
        bias = torch.randn((n,), generator=g, device="cuda").to([dtype, F32, BF][i])
        residual = torch.randn((m, n), generator=g, device="cuda").to(out_dtype)
        act = ACTS[(m + n + k + i) % 5]
        got = B.cat_linear(X, W, bias=bias, residual=residual, activation=act, out_dtype=out_dtype)
        check(X, W, bias, residual, act, out_dtype, got)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m", [1, 40, 200, 600])
@pytest.mark.parametrize("scale", [0.1, 3.0, 30.0])
def test_activations(act, m, scale):
    X, W, g = data(m, 384, 256, BF, scale=scale)
    bias = torch.randn((384,), generator=g, device="cuda")
    for out_dtype in (BF, F32):
        check(X, W, bias, None, act, out_dtype, B.cat_linear(X, W, bias=bias, activation=act, out_dtype=out_dtype))


@pytest.mark.parametrize("m", [1, 24, 150, 700])
@pytest.mark.parametrize("k", [64, 121, 1000])
def test_rows_any_distance_apart(m, k):
    """Views: column ranges of wider matrices at odd and even offsets, every other row, an output inside a larger buffer."""
    n = 301
    g = torch.Generator(device="cuda").manual_seed(m * k)
    for offset, step in [(0, 1), (1, 1), (8, 1), (3, 2)]:
        wide_x = torch.randn((m * step, k + offset + 5), generator=g, device="cuda").to(FH)
        wide_w = (torch.randn((n * step, k + offset + 8), generator=g, device="cuda") * k ** -0.5).to(FH)
        X, W = wide_x[::step, offset:offset + k], wide_w[::step, offset:offset + k]
        buffer = torch.full((m + 2, n + 7), -7.0, device="cuda", dtype=FH)
        out, residual = buffer[1:m + 1, 2:n + 2], torch.randn((m, n + 3), generator=g, device="cuda").to(FH)[:, 1:n + 1]
        want_res = residual.clone()
        got = B.cat_linear(X, W, residual=residual, activation="silu", out=out)
        assert got.data_ptr() == out.data_ptr()
        check(X, W, None, want_res, "silu", FH, got)
        buffer[1:m + 1, 2:n + 2] = -7.0
        assert (buffer == -7.0).all(), "something outside the output was written"


@pytest.mark.parametrize("m", [3, 500])
def test_residual_in_place(m):
    X, W, g = data(m, 512, 256, BF)
    stream = torch.randn((m, 512), generator=g, device="cuda").to(BF)
    before = stream.clone()
    B.cat_linear(X, W, residual=stream, out=stream)
    check(X, W, None, before, "none", BF, stream)


@pytest.mark.parametrize("m", [2, 400])
def test_what_is_not_finite_stays_in_its_rows_and_columns(m):
    X, W, _ = data(m, 300, 200, BF)
    X[0, 5], X[1, 199], W[7, 0] = math.inf, math.nan, -math.inf
    for act in ("none", "relu"):
        got = B.cat_linear(X, W, activation=act, out_dtype=F32)
        want = act64(X.double() @ W.double().t(), act)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got[torch.isinf(want)].double(), want[torch.isinf(want)])
        rest = torch.isfinite(want)
        assert torch.isfinite(got[rest]).all()
    big = B.cat_linear(torch.full((m, 64), 100.0, device="cuda", dtype=FH), torch.full((3, 64), 100.0, device="cuda", dtype=FH))
    assert torch.isinf(big).all()      # 640 000 in fp16


def test_no_rows_and_a_workspace_of_ones_own():
    X, W, _ = data(8, 40, 72, BF)
    assert B.cat_linear(X[:0], W).shape == (0, 40)
    ws = torch.full((256,), 255, dtype=torch.uint8, device="cuda")
    a = B.cat_linear(X, W, ws=ws)
    assert torch.equal(a, B.cat_linear(X, W)) and B.cat_workspace_report(ws)["device_status"] == 0
    odd = torch.randn((8, 73), device="cuda").to(BF)[:, 1:]
    with pytest.raises(B.CatError) as e:
        B.cat_linear(odd, W, ws=ws)     # needs room for a copy
    assert e.value.status == 4


@pytest.mark.parametrize("m,n,k", [(1, 2000, 4096), (64, 1000, 2048), (500, 1000, 520), (77, 300, 333)])
def test_the_same_bits_every_time_and_on_another_stream(m, n, k):
    X, W, g = data(m, n, k, BF)
    bias = torch.randn((n,), generator=g, device="cuda")
    first = B.cat_linear(X, W, bias=bias, activation="gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = [B.cat_linear(X, W, bias=bias, activation="gelu") for _ in range(20)]
    here = [B.cat_linear(X, W, bias=bias, activation="gelu") for _ in range(20)]
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs + here)


@pytest.mark.parametrize("m,k", [(1, 512), (200, 512), (30, 333)])
def test_captured_and_replayed_on_new_inputs(m, k):
    X, W, g = data(m, 700, k, BF)
    out = torch.empty((m, 700), device="cuda", dtype=F32)
    B.cat_linear(X, W, activation="relu", out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            B.cat_linear(X, W, activation="relu", out=out)
    for i in range(3):
        X.copy_(torch.randn((m, k), generator=g, device="cuda"))
        W.copy_(torch.randn((700, k), generator=g, device="cuda") * k ** -0.5)
        graph.replay()
        torch.cuda.synchronize()
        check(X, W, None, None, "relu", F32, out)


def test_refusals_on_the_device():
    X, W, _ = data(8, 40, 72, BF)
    with pytest.raises(TypeError):
        B.cat_linear(X, W.to(FH))
    with pytest.raises(TypeError):
        B.cat_linear(X.float(), W.float())
    with pytest.raises(ValueError):
        B.cat_linear(X, W[:, :71])
    with pytest.raises(ValueError):
        B.cat_linear(X.t().contiguous().t(), W)     # rows that are not contiguous
    with pytest.raises(ValueError):
        B.cat_linear(X, W, activation="tanh")
    with pytest.raises(ValueError):
        B.cat_linear(X, W, bias=torch.zeros(41, device="cuda"))
    with pytest.raises(TypeError):
        B.cat_linear(X, W, residual=torch.zeros((8, 40), device="cuda"))
    with pytest.raises(TypeError):
        B.cat_linear(X, W, out=torch.zeros((8, 40), device="cuda", dtype=torch.float64))
    with pytest.raises(TypeError):
        B.cat_linear(X, W.cpu())
    with pytest.raises(B.CatError) as e:
        B.cat_linear(X, W, out=torch.zeros((1, 40), device="cuda", dtype=BF).expand(8, 40))   # one row for all
    assert e.value.status == 2


@pytest.mark.parametrize("m", [1, 5, 300])
def test_columns_of_one_buffer(m):
    """X, the result and the weights' rows side by side in one buffer share no memory; a shifted residual and the result itself do."""
    for first, second in [(0, 128), (136, 0)]:
        buffer = torch.full((m + 1, 300), 7.0, dtype=BF, device="cuda")
        X, W, _ = data(m, 136, 120, BF)
        x, y = buffer[:m, first:first + 120], buffer[1:, second:second + 136]
        x.copy_(X)
        B.cat_linear(x, W, out=y)
        check(X, W, None, None, "none", BF, y)
        assert torch.equal(x, X) and bool((buffer[1:, 264:] == 7.0).all())
    X, W, _ = data(m, 120, 120, BF)
    for kwargs in [dict(out=X), dict(out=W[:m] if m <= 120 else X), dict(out=buffer[:m, :120], residual=buffer[:m, 8:128])]:
        with pytest.raises(B.CatError) as e:
            B.cat_linear(X, W, **kwargs)
        assert e.value.status == 2


# the largest number of rows, of columns, and the longest inner dimension
@pytest.mark.parametrize("m,n,k", [(1 << 24, 1, 8), (1 << 24, 2, 3), (1, 1 << 20, 8), (3, 1 << 20, 5), (2, 3, 1 << 20), (150, 5, (1 << 20) - 1)])
@pytest.mark.parametrize("out_dtype", [BF, F32])
def test_the_largest_sizes(m, n, k, out_dtype):
    X, W, _ = data(m, n, k, BF)
    check(X, W, None, None, "none", out_dtype, B.cat_linear(X, W, out_dtype=out_dtype))
