"""The output end of a low-bit network that drafts for its full-precision counterpart, as a serving loop runs it: hidden rows through
the head (cat_linear, fp32 rows), the correction of the draft's rows (cat_apply), the verification (cat_verify_drafts) -- eagerly, and
captured once and replayed on new hidden rows."""
import numpy as np
import pytest
import torch

from oracle import cat_oracle as O
from paper_2509_26277_b200 import binding as B
from tests import verify_oracle as V
from tests.test_gpu_linear import want_and_bound

pytestmark = pytest.mark.gpu

SEQS, DRAFTS, WIDTH, VOCAB, K = 6, 3, 256, 1000, 4


def model(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn((VOCAB, WIDTH), generator=g, device="cuda") * 2 * WIDTH ** -0.5)
    step = W.abs().amax(1, keepdim=True) / 3.5
    Wq = ((torch.floor(W / step) + 0.5).clamp(-3.5, 3.5) * step)          # 3-bit weights
    bias = torch.randn((VOCAB,), generator=g, device="cuda")
    X = torch.randn((600, WIDTH), generator=g, device="cuda")
    rows_q = B.cat_linear(X.bfloat16(), Wq.bfloat16(), bias=bias, out_dtype=torch.float32)
    rows_fp = B.cat_linear(X.bfloat16(), W.bfloat16(), bias=bias, out_dtype=torch.float32)
    C, G, Bt, _ = B.cat_fit(rows_q, rows_fp, K, 5)
    return dict(W=W.bfloat16(), Wq=Wq.bfloat16(), bias=bias, C=C, G=G, Bt=Bt, g=g)


def inputs(m):
    g = m["g"]
    hidden = torch.randn((SEQS * (DRAFTS + 1), WIDTH), generator=g, device="cuda").bfloat16()
    return dict(hidden=hidden, ua=torch.rand((SEQS, DRAFTS), generator=g, device="cuda"), us=torch.rand((SEQS,), generator=g, device="cuda"),
                draw=torch.rand((SEQS * DRAFTS,), generator=g, device="cuda"))


def step(m, x, outs):
    """One step; every buffer is the caller's."""
    B.cat_linear(x["hidden"], m["W"], bias=m["bias"], out=outs["target"])
    B.cat_linear(x["hidden"][:SEQS * DRAFTS], m["Wq"], bias=m["bias"], out=outs["low"])
    B.cat_apply(outs["low"], m["C"], m["G"], m["Bt"], out=outs["draft"])
    # drafts are drawn from the corrected rows: sequences without drafts of their own
    B.cat_verify_drafts(outs["draft"].view(SEQS * DRAFTS, 1, VOCAB), None, outs["none"], outs["no_u"], x["draw"], tokens_out=outs["drawn"],
                        accepted_out=outs["no_kept"])
    B.cat_verify_drafts(outs["target"].view(SEQS, DRAFTS + 1, VOCAB), outs["draft"].view(SEQS, DRAFTS, VOCAB), outs["drawn"].view(SEQS, DRAFTS),
                        x["ua"], x["us"], tokens_out=outs["tokens"], accepted_out=outs["kept"])


def buffers():
    f = dict(device="cuda", dtype=torch.float32)
    i = dict(device="cuda", dtype=torch.int32)
    n = SEQS * DRAFTS
    return dict(target=torch.empty((SEQS * (DRAFTS + 1), VOCAB), **f), low=torch.empty((n, VOCAB), **f), draft=torch.empty((n, VOCAB), **f),
                none=torch.empty((n, 0), **i), no_u=torch.empty((n, 0), **f), drawn=torch.empty((n, 1), **i), no_kept=torch.empty((n,), **i),
                tokens=torch.empty((SEQS, DRAFTS + 1), **i), kept=torch.empty((SEQS,), **i))


def check(m, x, o):
    h = lambda t: t.detach().cpu().numpy()
    for rows, W, out in ((x["hidden"], m["W"], o["target"]), (x["hidden"][:SEQS * DRAFTS], m["Wq"], o["low"])):
        want, bound = want_and_bound(rows, W, m["bias"], None, "none", torch.float32)
        assert ((out.double() - want).abs() <= bound).all()
    want, _, _, _ = O.apply(h(o["low"]), h(m["C"]), h(m["G"]), h(m["Bt"]))
    np.testing.assert_array_equal(h(o["draft"]), want)
    drawn, _, margin = V.verify(h(o["draft"])[:, None], None, h(o["none"]), h(o["no_u"]), h(x["draw"]))
    assert ((h(o["drawn"]) == drawn).all(1) | (margin < 1e-11)).all()
    tokens, kept, margin = V.verify(h(o["target"]).reshape(SEQS, DRAFTS + 1, VOCAB), h(o["draft"]).reshape(SEQS, DRAFTS, VOCAB),
                                    h(o["drawn"]).reshape(SEQS, DRAFTS), h(x["ua"]), h(x["us"]))
    fine = margin >= 1e-11
    assert (h(o["tokens"])[fine] == tokens[fine]).all() and (h(o["kept"])[fine] == kept[fine]).all()
    return int(kept.sum())


def test_a_step_of_the_chain_and_its_replay():
    m = model()
    x, o = inputs(m), buffers()
    step(m, x, o)
    torch.cuda.synchronize()
    accepted = check(m, x, o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(m, x, o)
    for _ in range(4):
        for k, v in inputs(m).items():
            x[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        accepted += check(m, x, o)
    assert accepted > 0


def test_two_steps_at_once_on_two_streams():
    m = model(1)
    sides = [torch.cuda.Stream() for _ in range(2)]
    work = [(inputs(m), buffers()) for _ in sides]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (x, o) in zip(sides, work):
            with torch.cuda.stream(s):
                # (workspaces of the correction are kept by shape: one of its own per stream)
                B.cat_linear(x["hidden"], m["W"], bias=m["bias"], out=o["target"])
                B.cat_linear(x["hidden"][:SEQS * DRAFTS], m["Wq"], bias=m["bias"], out=o["low"])
                o.setdefault("ws", torch.empty(B.workspace("apply", SEQS * DRAFTS, VOCAB, K, "cuda").numel(), dtype=torch.uint8, device="cuda"))
                B.cat_apply(o["low"], m["C"], m["G"], m["Bt"], out=o["draft"], ws=o["ws"])
                B.cat_verify_drafts(o["draft"].view(SEQS * DRAFTS, 1, VOCAB), None, o["none"], o["no_u"], x["draw"], tokens_out=o["drawn"],
                                    accepted_out=o["no_kept"])
                B.cat_verify_drafts(o["target"].view(SEQS, DRAFTS + 1, VOCAB), o["draft"].view(SEQS, DRAFTS, VOCAB), o["drawn"].view(SEQS, DRAFTS),
                                    x["ua"], x["us"], tokens_out=o["tokens"], accepted_out=o["kept"])
    torch.cuda.synchronize()
    for x, o in work:
        check(m, x, o)
