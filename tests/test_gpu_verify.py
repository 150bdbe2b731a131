"""cat_verify_drafts against the definitions in 64 bits (verify_oracle).  Outputs are whole numbers and have to be equal, except in
sequences where a decision is closer than 1e-11 in mass, which sums in 64 bits in another order may tell either way (there are none in
most runs; the tests count them)."""
import numpy as np
import pytest
import torch

from paper_2509_26277_b200 import binding as B
from tests import verify_oracle as O

pytestmark = pytest.mark.gpu

BF, FH, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [BF, FH, F32]


def problem(b, s, v, target=BF, draft=BF, noise=0.5, sharp=3.0, seed=0, greedy_every=5):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * b + 1000 * s + v)
    t = (sharp * torch.randn((b, s + 1, v), generator=g, device="cuda")).to(target)
    q = None if draft is None else (t[:, :s].float() + noise * torch.randn((b, s, v), generator=g, device="cuda")).to(draft)
    T = 0.5 + torch.rand((b,), generator=g, device="cuda")
    if greedy_every and b > 1:
        T[::greedy_every] = 0
    guess = t[:, :s].float() if q is None else q.float()
    gumbel = -torch.log(-torch.log(torch.rand(guess.shape, generator=g, device="cuda").clamp(1e-20, 1 - 1e-7)))
    x = (guess + T[:, None, None] * gumbel).argmax(-1).int() if s else torch.zeros((b, 0), dtype=torch.int32, device="cuda")
    n = torch.randint(0, s + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
    n[torch.rand((b,), generator=g, device="cuda") < 0.7] = s
    return dict(target=t, draft=q, draft_tokens=x, u_accept=torch.rand((b, s), generator=g, device="cuda"),
                u_sample=torch.rand((b,), generator=g, device="cuda"), draft_lengths=n, temperature=T)


def host(t):
    return None if t is None else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def want_of(p):
    return O.verify(host(p["target"]), host(p["draft"]), host(p["draft_tokens"]), host(p["u_accept"]), host(p["u_sample"]),
                    host(p.get("draft_lengths")), host(p.get("temperature")))


def agree(p, got=None, allow=0):
    tokens, kept = B.cat_verify_drafts(**p) if got is None else got
    want, want_kept, margin = want_of(p)
    here = want_kept > -9
    same = ((host(tokens) == want).all(1) & (host(kept) == want_kept)) | ~here
    close = margin < 1e-11
    assert (same | close).all(), (np.flatnonzero(~same & ~close)[:5], host(tokens)[~same][:3], want[~same][:3], margin[~same][:3])
    assert close.sum() <= allow, f"{int(close.sum())} decisions too close to test"
    return host(tokens), host(kept)


# one entry; lanes, warps and parts that stay empty; vocabularies at the edges of a chunk; odd row lengths (rows on any even address)
@pytest.mark.parametrize("v", [1, 2, 31, 33, 500, 1000, 1023, 1024, 1025, 4095, 4096, 5001, 16384, 32000, 50_001])
@pytest.mark.parametrize("b,s", [(1, 0), (1, 1), (3, 4), (40, 2)])
def test_vocabularies(b, s, v):
    for i in range(3):
        agree(problem(b, s, v, TYPES[i], TYPES[(i + b) % 3], seed=i, sharp=1.0 + i))


@pytest.mark.parametrize("b,s,v", [(5, 8, 128_000), (300, 3, 2000), (150, 5, 9001), (64, 7, 16_385), (20, 12, 20_000), (1, 64, 1500), (1500, 1, 257),
                                   (37, 1, 100_003), (75, 2, 30_011)])
def test_batches(b, s, v):
    agree(problem(b, s, v, BF, F32 if b % 2 else BF))


@pytest.mark.parametrize("target", TYPES)
@pytest.mark.parametrize("draft", TYPES + [None])
def test_types(target, draft):
    tokens, kept = agree(problem(48, 5, 3001, target, draft, noise=1.0))
    assert kept.min() == 0 and kept.max() >= (1 if draft is None else 3)


@pytest.mark.parametrize("sharp", [0.01, 0.3, 8.0, 40.0])
def test_flat_and_peaked_rows(sharp):
    agree(problem(64, 3, 20_000, F32, F32, sharp=sharp, noise=0.3 * sharp))


def test_draws_next_to_a_border():
    """Flat rows, and uniform numbers on, just below and just above the border between two tokens: sums in fp32 cannot decide these."""
    v, b = 4096, 96
    p = problem(b, 0, v, F32, None, greedy_every=0)
    p["target"] = torch.full((b, 1, v), 2.5, device="cuda")
    k = torch.arange(b, device="cuda") * 37
    p["u_sample"] = (k.double() / v).float()          # (exact: a border in exact arithmetic; the token behind it)
    p["u_sample"][1::3] += 2.0 ** -22
    p["u_sample"][2::3] -= 2.0 ** -22
    p["temperature"] = None
    tokens, _ = B.cat_verify_drafts(**p)
    want = torch.floor(p["u_sample"].double() * v).int()
    assert torch.equal(tokens[1::3, 0], want[1::3]) and torch.equal(tokens[2::3, 0], want[2::3])
    off = (tokens[0::3, 0] - want[0::3])
    assert ((off == 0) | (off == -1)).all()            # 64-bit sums of 4096 equal terms, either side of the border
    p["u_sample"][:] = 0
    assert (B.cat_verify_drafts(**p)[0] == 0).all()
    p["u_sample"][:] = 1 - 2.0 ** -24
    assert (B.cat_verify_drafts(**p)[0] == v - 1).all()


def test_masks():
    """Vocabularies cut to a few tokens, with -inf, the type's lowest value and NaN; whole rows masked; +inf."""
    for dtype in TYPES:
        p = problem(60, 3, 2500, dtype, dtype)
        low = torch.finfo(dtype).min
        t, q = p["target"], p["draft"]
        keep = torch.rand((2500,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) < 0.01
        keep[17] = True
        t[0:10, :, ~keep], q[0:10, :, ~keep] = -torch.inf, -torch.inf
        t[10:20, :, ~keep], q[10:20, :, ~keep] = low, low
        t[20:30, :, ~keep] = torch.nan
        q[20:25, :, ~keep] = torch.nan
        t[30:35, 0] = -torch.inf
        t[35:40, 1] = -torch.inf
        t[36, 2] = torch.nan
        q[40:45, 1] = -torch.inf
        t[45:50] = low
        q[47:52] = low
        t[52:55, :, 100] = torch.inf
        t[53, :, 2400] = torch.inf
        q[54, :, 7] = torch.inf
        for x in (torch.zeros(60, 3), torch.full((60, 3), 17), torch.full((60, 3), 100)):
            p["draft_tokens"] = x.int().cuda()
            agree(p)
        t[:] = -torch.inf
        tokens, kept = agree(p)
        assert (tokens == -1).all() and (kept == 0).all()


def test_identical_rows_accept_everything_and_leave_no_residual():
    p = problem(50, 4, 3000, BF, BF)
    p["draft"] = p["target"][:, :4].clone()
    tokens, kept = agree(p)
    n = host(p["draft_lengths"])
    warm = host(p["temperature"]) > 0
    assert (kept[warm] == n[warm]).all()
    p["draft_tokens"][:] = 3000                        # refused, and p - q has no mass: the draw is from p
    tokens, kept = agree(p)
    assert (kept == 0).all() and (tokens[:, 0] >= 0).all()
    # the same distributions, shifted: what is left of p - q is rounding
    p["target"], p["draft"] = p["target"].float(), p["target"][:, :4].float() + 1.0
    agree(p)


def test_tokens_outside_the_vocabulary_are_refused():
    p = problem(12, 3, 700, F32, F32)
    p["draft_tokens"][::2, 1] = 700
    p["draft_tokens"][1::4, 0] = -1
    p["draft_tokens"][3::4, 0] = -2 ** 31
    tokens, kept = agree(p)
    for q in (dict(p, draft=None), dict(p, u_accept=torch.zeros_like(p["u_accept"]))):
        tokens, kept = agree(q)
        assert (kept[::2] <= 1).all() and (kept[1::2] == 0).all()


def test_lengths_and_sequences_that_are_not_there():
    p = problem(30, 4, 1200, BF, BF)
    p["draft_lengths"] = torch.tensor([-1, 0, 1, 2, 3, 4, 5, 1000, -2 ** 31, 4] * 3, dtype=torch.int32, device="cuda")
    want, want_kept, _ = want_of(p)
    gone = want_kept == -9
    # what lies behind a length is not looked at: NaN there changes nothing
    for b, n in enumerate(p["draft_lengths"].tolist()):
        n = min(n, 4)
        p["target"][b, max(n + 1, 0):], p["draft"][b, max(n, 0):] = torch.nan, torch.nan
        p["u_accept"][b, max(n, 0):] = torch.nan
    tokens = torch.full((30, 5), -9, dtype=torch.int32, device="cuda")
    kept = torch.full((30,), -9, dtype=torch.int32, device="cuda")
    got = B.cat_verify_drafts(**p, tokens_out=tokens, accepted_out=kept)
    assert got[0] is tokens and got[1] is kept
    assert (host(tokens) == want).all() and (host(kept) == want_kept).all() and gone.sum() == 6


def test_uniform_numbers_outside_their_range():
    p = problem(16, 2, 900, F32, F32)
    p["u_sample"][:4], p["u_sample"][4:8], p["u_sample"][8:12] = 1.0, -0.5, torch.nan
    p["u_accept"][:8, 0], p["u_accept"][8:, 0] = torch.nan, 2.0
    agree(p)
    p["temperature"][::3] = torch.nan
    p["temperature"][1::3] = -1.0
    agree(p)


@pytest.mark.parametrize("T", [1e-30, 1e-6, 1e-3, 50.0, 1e6, 1e30])
def test_extreme_temperatures(T):
    p = problem(24, 2, 3000, F32, BF)
    p["temperature"][:] = T
    agree(p)
    p["target"] *= 1e30
    agree(p)


@pytest.mark.parametrize("T", [0.003, 0.01, 0.05, 0.2])
@pytest.mark.parametrize("v", [6, 104, 1630, 48_003])
def test_low_temperatures(T, v):
    """Logits / T of some hundreds to some thousands: probabilities from one to nothing, and exponents up to the ends of fp64."""
    for i, (target, draft) in enumerate([(BF, F32), (FH, F32), (BF, FH), (F32, None)]):
        p = problem(300 if v < 2000 else 40, 2, v, target, draft, seed=i, noise=0.3 * (1 + i), sharp=2.0 + 6 * i, greedy_every=0)
        p["temperature"][:] = T * (1 + torch.rand(p["temperature"].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)))
        # (rows with nearly all their mass on one entry leave residuals of down to 2^-40 in all: any decision within one is within 1e-12)
        agree(p, allow=len(p["u_sample"]) // 5)


def test_views_of_larger_buffers():
    b, s, v = 9, 3, 1501
    p = problem(b, s, v, BF, F32)
    wide = torch.full((b + 1, s + 3, v + 6), torch.nan, device="cuda", dtype=BF)
    wide[:b, 1:s + 2, 3:v + 3] = p["target"]
    other = torch.full((s, b, v + 1), torch.nan, device="cuda")
    other[:, :, 1:] = p["draft"].transpose(0, 1)
    q = dict(p, target=wide[:b, 1:s + 2, 3:v + 3], draft=other[:, :, 1:].transpose(0, 1))
    got = B.cat_verify_drafts(**q)
    agree(p, got=got)


def test_the_same_outputs_every_time_and_on_another_stream():
    p = problem(33, 4, 30_000, BF, BF, sharp=0.5)
    first = B.cat_verify_drafts(**p)
    agree(p, got=first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = [B.cat_verify_drafts(**p) for _ in range(10)]
    outs += [B.cat_verify_drafts(**p) for _ in range(10)]
    torch.cuda.synchronize()
    assert all(torch.equal(first[0], o[0]) and torch.equal(first[1], o[1]) for o in outs)


def test_captured_and_replayed_on_new_inputs():
    p = problem(6, 3, 8000, BF, BF)
    outs = B.cat_verify_drafts(**p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cat_verify_drafts(**p, tokens_out=outs[0], accepted_out=outs[1])
        B.cat_verify_drafts(**p, tokens_out=outs[0], accepted_out=outs[1])
    for i in range(4):
        new = problem(6, 3, 8000, BF, BF, seed=i + 1, sharp=0.2 + i)
        for k, x in new.items():
            p[k].copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        agree(p, got=outs)


def test_offsets_beyond_32_bits():
    """Rows of a buffer of more than 2^32 elements: a sequence far from the first."""
    v = 70_000
    seq = 2 ** 31 + 5 * v + 3
    big = torch.empty((2 * seq + 3 * v,), dtype=BF, device="cuda")
    target = torch.as_strided(big, (3, 2, v), (seq, v, 1))
    p = problem(3, 1, v, BF, BF, greedy_every=0)
    target.copy_(p["target"])
    agree(p, got=B.cat_verify_drafts(**dict(p, target=target)))
    del big, target
    torch.cuda.empty_cache()


@pytest.mark.parametrize("b,s,v,dtype", [(1, 1, 1 << 22, F32), (2, 2, 1_000_003, BF), (3, 0, 600_001, FH), (40, 1, 300_000, BF)])
def test_large_vocabularies(b, s, v, dtype):
    agree(problem(b, s, v, dtype, dtype))


@pytest.mark.parametrize("v", [600, 20_000, 40_000, 90_000])
def test_both_passes_are_reached(v):
    """Flat rows: fp32 sums leave draws undecided; the fp64 pass settles them, in the same launch or in one of its own."""
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    p = problem(200, 1, v, F32, F32, sharp=0.1, noise=0.05, greedy_every=0)
    got = B.cat_verify_drafts(**p, ws=ws)
    agree(p, got=got)
    settled = B.cat_workspace_report(ws)["refined_rows_total"]
    assert (0 < settled < 200) if v > 600 else settled < 200
    B.cat_verify_drafts(**dict(p, target=p["target"] * 300, draft=p["draft"] * 300), ws=ws)       # peaked: hardly any
    assert B.cat_workspace_report(ws)["refined_rows_total"] - settled < 20
    wild = dict(p, target=p["target"] * 1e30, draft=p["draft"] * 1e30)                            # beyond what fp32 exponents hold: all
    agree(wild, got=B.cat_verify_drafts(**wild, ws=ws))


def test_an_output_among_the_inputs_is_refused():
    p = problem(1, 3, 100, BF, BF)
    both = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
    with pytest.raises(B.CatError) as e:
        B.cat_verify_drafts(**dict(p, draft_tokens=both[:, :3]), tokens_out=both)
    assert e.value.status == 2


def test_refusals_on_the_device():
    p = problem(4, 2, 100, BF, BF)
    for key, bad, error in [("draft_tokens", p["draft_tokens"].long(), TypeError), ("draft_tokens", p["draft_tokens"][:, :1], ValueError),
                            ("u_accept", p["u_accept"].double(), TypeError), ("u_sample", p["u_sample"][:3], ValueError),
                            ("temperature", p["temperature"].cpu(), TypeError), ("draft", p["draft"].double(), TypeError),
                            ("draft", p["draft"][:, :1], ValueError), ("target", p["target"].double(), TypeError),
                            ("target", p["target"][0], ValueError), ("target", p["target"][:, :0], ValueError),
                            ("target", p["target"].transpose(1, 2).contiguous().transpose(1, 2), ValueError)]:
        with pytest.raises(error):
            B.cat_verify_drafts(**dict(p, **{key: bad}))
    with pytest.raises(B.CatError) as e:
        B.cat_verify_drafts(**dict(p, target=p["target"][:, :1].expand(4, 3, 100)))   # one row for all
    assert e.value.status == 2


@pytest.mark.parametrize("b,s,v", [(2, 256, 600), (1, 256, 33_000), (1, 0, 1 << 22)])
def test_the_most_drafts_and_the_largest_vocabulary(b, s, v):
    p = problem(b, s, v, FH, BF, noise=0.02)
    p["draft_lengths"] = None
    agree(p)


@pytest.mark.parametrize("v", [1, 7, 40])
def test_the_largest_batch(v):
    """2^20 sequences, every third of them greedy, against whole-batch arithmetic in 64 bits."""
    b = 1 << 20
    g = torch.Generator(device="cuda").manual_seed(v)
    t = torch.randn((b, 1, v), generator=g, device="cuda").to(BF)
    T = torch.ones((b,), device="cuda")
    T[::3] = 0
    u = torch.rand((b,), generator=g, device="cuda")
    none = torch.empty((b, 0), device="cuda")
    tokens, kept = B.cat_verify_drafts(t, None, none.int(), none, u, temperature=T)
    mass = torch.exp(t[:, 0].double() - t[:, 0].double().amax(1, keepdim=True))
    total = mass.cumsum(1)
    drawn = (total > u.double()[:, None] * total[:, -1:]).int().argmax(1)
    largest = t[:, 0] == t[:, 0].amax(1, keepdim=True)
    want = torch.where(T > 0, drawn, largest.int().argmax(1))
    close = (T > 0) & ((total - u.double()[:, None] * total[:, -1:]).abs().amin(1) < 1e-11)
    same = tokens[:, 0] == want
    assert bool((same | close).all()) and int(close.sum()) <= 1 and not bool(kept.any())


def test_outputs_among_the_logits_are_refused():
    p = problem(1, 1, 100, BF, F32)
    for kwargs in [dict(tokens_out=p["draft"].view(torch.int32)[0, :, :2]), dict(accepted_out=p["target"].view(torch.int32)[0, 1, 49:])]:
        with pytest.raises(B.CatError) as e:
            B.cat_verify_drafts(**p, **kwargs)
        assert e.value.status == 2
