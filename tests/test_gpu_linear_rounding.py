"""cat_linear: 16-bit results over long inner dimensions, how often they are the wrong neighbour of the exact value; few tokens over many tiles.

Tolerance, written down before the first run.  The tensor cores add 16 inner columns at a step and truncate the sum: a step drops ulp / 2 on
average, 2^-24 * 0.72 of the sum's size (0.72: a number's mean distance above its binade's lower end).  Products of independent numbers make the
sum a random walk: over a run of n steps of T in all it has 0.53 of its final size on average, which is s sqrt(n / T) for results of size s.
So a run is off by 2.3e-8 n s sqrt(n / T), and T / n runs that are added to nearest, signs independent, by 2.3e-8 n s.  An error e moves a
result to another neighbour with probability e / ulp and by one ulp then: a 2-norm of sqrt(e E[ulp]) / s, with E[ulp] = 2^-7 * 0.72 * 0.8 s in bf16
(0.8 s: mean size).  Runs of up to 24 slabs of four steps, n = 96: 9.9e-5 at most.  One run over 512 steps gives 2.3e-4.  The line lies between."""
import pytest
import torch

from paper_2509_26277_b200 import binding as B
from tests.test_gpu_linear import BF, F32, FH, check, data

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n", [(2048, 2048), (600, 1000), (70, 4000), (16, 16384)])
@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("k", [8192, 20_000])
def test_long_sums_round_to_the_nearest_neighbour(m, n, dtype, k):
    X, W, _ = data(m, n, k, dtype)
    exact = X.double() @ W.double().t()
    off = B.cat_linear(X, W).double() - exact.to(dtype).double()
    line = 1.3e-4 * (torch.finfo(dtype).eps / 2.0 ** -7) ** 0.5      # (fp16's steps are an eighth of bf16's)
    assert float(off.norm() / exact.norm()) < line


@pytest.mark.parametrize("m", [9, 17, 32, 33, 64, 65])
@pytest.mark.parametrize("n,k", [(19_000, 300), (40_000, 130)])
def test_few_tokens_and_more_tiles_than_ctas(m, n, k):
    """Single CTAs that take several tiles, one and two to an SM."""
    X, W, g = data(m, n, k, FH)
    residual = torch.randn((m, n), generator=g, device="cuda")
    check(X, W, None, residual, "silu", F32, B.cat_linear(X, W, residual=residual, activation="silu", out_dtype=F32))
    check(X, W, None, None, "none", FH, B.cat_linear(X, W))
