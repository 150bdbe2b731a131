"""cat_verify_drafts at the ends of its ranges."""
import pytest
import torch

from tests.test_gpu_verify import BF, F32, agree, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1e-37, 4.3e-39, 4.1e-39, 1e-39, 1e-42, 1.4e-45])
@pytest.mark.parametrize("b,v", [(24, 3000), (3, 50_001)])
def test_temperatures_down_to_the_smallest_float(T, b, v):
    """All mass on the largest entry (softmax(logits / T) is defined for every T > 0); and logits as small as T, whose rows are spread as ever."""
    for target, draft in [(F32, BF), (BF, F32), (F32, None)]:
        p = problem(b, 2, v, target, draft)
        p["temperature"][:] = T
        tokens, _ = agree(p)
        assert (tokens[:, 0] >= 0).all()
    p = problem(b, 2, v, F32, F32)
    p["temperature"][:] = T
    p["target"], p["draft"] = p["target"] * T, p["draft"] * T
    agree(p)


@pytest.mark.parametrize("T", [1.0, 3e38, float("inf")])
def test_rows_that_span_all_floats(T):
    """Entries at both ends of fp32 with temperatures as large: differences of logits pass the largest float, their quotients do not."""
    p = problem(12, 1, 700, F32, F32, greedy_every=0)
    p["temperature"][:] = T
    p["target"][:, :, ::2], p["target"][:, :, 1::2] = 3.4e38, -3.4e38
    p["draft"][:, :, ::2], p["draft"][:, :, 1::2] = -3.4e38, 3.4e38
    p["draft_tokens"][::2] = 1
    agree(p)
