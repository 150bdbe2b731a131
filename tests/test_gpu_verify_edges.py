"""cat_verify_drafts at the ends of its ranges."""
import numpy as np
import pytest
import torch

from paper_2509_26277_b200 import binding as B
from tests.test_gpu_verify import BF, F32, agree, host, problem

pytestmark = pytest.mark.gpu

LN2 = float(np.log(2.0))


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
    p["u_sample"][:] = 0
    p["target"][:, :, :4] = -3.4e38
    p["draft_lengths"][:] = 0
    tokens, _ = B.cat_verify_drafts(**p)
    assert (host(tokens)[:, 0] == (4 if T == 1.0 else 0)).all()


@pytest.mark.parametrize("b,v", [(1, 2000), (40, 2000), (200, 2000), (200, 40_000), (3, 40_000)])
@pytest.mark.parametrize("top", [-420.0, 0.0, 346.0])
def test_mass_ends_relative_to_the_rows_largest(b, v, top):
    """u = 0 draws the first entry with mass: one of 2^-900 of its row's largest has some, one of 2^-1100 has none, wherever the largest lies."""
    g = torch.Generator(device="cuda").manual_seed(v + b)
    row = top - 4000 - 100 * torch.rand((b, 2, v), generator=g, device="cuda")
    row[:, :, 3], row[:, :, 5], row[:, :, 9] = top - 1100 * LN2, top - 900 * LN2, top
    none = torch.full((b, 1, v), -torch.inf, device="cuda")
    zero, one = torch.zeros((b,), device="cuda"), torch.ones((b, 1), device="cuda")
    drafts = torch.full((b, 1), 9, dtype=torch.int32, device="cuda")
    # plain sampling; a refused draft that is the largest entry; one of a draft row without mass, refused since 3 has none itself
    tokens, kept = B.cat_verify_drafts(row[:, :1], None, drafts[:, :0].contiguous(), one[:, :0].contiguous(), zero)
    assert (tokens[:, 0] == 5).all()
    tokens, kept = B.cat_verify_drafts(row, None, torch.full_like(drafts, v), one, zero)
    assert (tokens[:, 0] == 5).all() and not kept.any()
    tokens, kept = B.cat_verify_drafts(row, none, torch.full_like(drafts, 3), one, zero)
    assert (tokens[:, 0] == 5).all() and not kept.any()
    tokens, kept = B.cat_verify_drafts(row, none, torch.full_like(drafts, 5), one, zero)
    assert (tokens[:, 0] == 5).all() and (kept == 1).all() and (tokens[:, 1] == 5).all()
    # the numbers of fp32 on both sides of 2^-1000
    if top == 0.0:
        row[:, :, 3], row[:, :, 5] = -693.14722, -693.14716      # (2^-1000.00006 and 2^-999.99997)
        tokens, kept = B.cat_verify_drafts(row[:, :1], None, drafts[:, :0].contiguous(), one[:, :0].contiguous(), zero)
        assert (tokens[:, 0] == 5).all()


@pytest.mark.parametrize("b,v", [(1, 500), (40, 2000), (200, 2000), (3, 40_000), (160, 40_000), (60, 90_000)])
@pytest.mark.parametrize("target", [F32, BF])
def test_drafts_at_the_end_of_mass_against_rows_without_any(b, v, target):
    """A draft whose target entry lies next to 2^-1000 of its row's largest, from a draft row that is masked whole: refused just below, accepted just
    above; the refused one's token is drawn from the target's row."""
    p = problem(b, 2, v, target, F32, sharp=1.0, greedy_every=0)
    p["temperature"], p["draft_lengths"] = None, None
    t = p["target"]
    t.copy_((t.float() - t.float().amax(-1, keepdim=True)).to(target))
    p["draft"][:] = -torch.inf
    p["draft_tokens"][:, 0], p["draft_tokens"][:, 1] = 7, 11
    for first, second in [(1000.5, 1000.5), (999.5, 1000.5), (1003.0, 999.5), (999.5, 999.5)]:
        # (one step of bf16 here is 4: the values that it has are 692 = 998.35 ln 2 and 696 = 1004.1 ln 2)
        t[:, 0, 7], t[:, 1, 11] = -first * LN2, -second * LN2
        tokens, kept = agree(p)
        if target == F32:
            assert (kept == (0 if first > 1000 else 1 if second > 1000 else 2)).all()
        assert (tokens[np.arange(b), kept] >= 0).all()


def test_calls_from_several_host_threads():
    """Vocabularies whose calls want different amounts of shared memory of the same kernel (64 to 127 KB), from threads that do nothing but call."""
    import threading

    failures = []

    def loop(v):
        try:
            p = problem(8, 4, v, BF, BF)
            want = B.cat_verify_drafts(**p)
            tokens, kept = torch.empty_like(want[0]), torch.empty_like(want[1])
            ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
            stream = torch.cuda.Stream()
            torch.cuda.synchronize()
            at = lambda t: t.data_ptr()
            args = (at(p["target"]), 1, 5 * v, v, at(p["draft"]), 1, 4 * v, v, at(p["draft_tokens"]), at(p["draft_lengths"]), at(p["temperature"]),
                    at(p["u_accept"]), at(p["u_sample"]), 8, 4, v, at(tokens), at(kept), at(ws), 256, stream.cuda_stream)
            call = B.lib().cat_verify_drafts
            assert [s for s in (call(*args) for _ in range(3000)) if s] == []
            stream.synchronize()
            assert torch.equal(tokens, want[0]) and torch.equal(kept, want[1])
        except BaseException as e:      # (an assertion in a thread is lost otherwise)
            failures.append(e)

    threads = [threading.Thread(target=loop, args=(v,)) for v in (32_000, 48_000, 40_000, 63_000)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, str(failures[0])[:300]


@pytest.mark.parametrize("b,s,v", [(1, 3, 1000), (8, 4, 32_000), (30, 6, 20_000), (200, 3, 2000), (64, 5, 100_000), (300, 0, 5000)])
def test_inputs_that_change_during_calls(b, s, v):
    """What a call reads then is either value; it ends all the same, and its tokens are tokens."""
    p = problem(b, s, v, BF, BF)
    g = torch.Generator(device="cuda").manual_seed(v)
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")
    sets = []
    for i in range(8):
        T = 2 * rand(b)
        T[rand(b) < 0.2], T[rand(b) < 0.1], T[rand(b) < 0.1] = 0.0, 1e-40, 1e30
        u, a = rand(b), rand(b, s)
        u[rand(b) < 0.2], a[rand(b, s) < 0.2] = 0.0, float("nan")
        x = (rand(b, s) * v).int()
        x[rand(b, s) < 0.1] = -5
        keep = rand(b, s) < 0.7
        x[keep] = p["draft_tokens"][keep]
        n = torch.randint(-1, s + 2, (b,), generator=g, device="cuda", dtype=torch.int32)
        sets.append(dict(temperature=T, u_sample=u, u_accept=a, draft_tokens=x, draft_lengths=n))
    here, side = torch.cuda.Stream(), torch.cuda.Stream()
    tokens, kept = torch.full((b, s + 1), -1, dtype=torch.int32, device="cuda"), torch.zeros((b,), dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    for i in range(150):
        with torch.cuda.stream(here):
            B.cat_verify_drafts(**p, tokens_out=tokens, accepted_out=kept)
        with torch.cuda.stream(side):
            for k, x in sets[i % 8].items():
                p[k].copy_(x)
    torch.cuda.synchronize()
    assert int(tokens.min()) >= -1 and int(tokens.max()) < v
    p["draft_lengths"][:] = s
    agree(p, allow=b)


@pytest.mark.parametrize("b,v", [(4, 1000), (200, 40_000)])
def test_the_status_of_a_workspace_as_it_comes(b, v):
    """The status word is this call's, whatever the workspace held; the count is the running total over a block that was zeroed."""
    ws = torch.full((256,), 255, dtype=torch.uint8, device="cuda")
    p = problem(b, 1, v, F32, F32, sharp=0.1, noise=0.05, greedy_every=0)
    p["draft_lengths"][0] = -1
    agree(p, got=B.cat_verify_drafts(**p, ws=ws, tokens_out=torch.full((b, 2), -9, dtype=torch.int32, device="cuda"),
                                     accepted_out=torch.full((b,), -9, dtype=torch.int32, device="cuda")))
    assert B.cat_workspace_report(ws)["device_status"] == 0
    ws.zero_()
    for i in range(3):
        B.cat_verify_drafts(**p, ws=ws)
        if i == 0:
            once = B.cat_workspace_report(ws)["refined_rows_total"]
    assert B.cat_workspace_report(ws) == dict(B.cat_workspace_report(ws), device_status=0, refined_rows_total=3 * once)


def test_workspaces_elsewhere_are_refused():
    p = problem(2, 1, 100, BF, BF)
    X, W = torch.zeros((4, 64), device="cuda", dtype=BF), torch.zeros((8, 64), device="cuda", dtype=BF)
    for ws in (torch.zeros(256, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8, device="cuda")[::2], torch.zeros(1, device="cuda").expand(256)):
        with pytest.raises(TypeError):
            B.cat_verify_drafts(**p, ws=ws)
        with pytest.raises(TypeError):
            B.cat_linear(X, W, ws=ws)
