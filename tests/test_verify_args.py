"""cat_verify_drafts' checks of arguments (host only), and the definitions it is tested against."""
import numpy as np
import pytest

from paper_2509_26277_b200 import binding as B
from tests import verify_oracle as O

AT = 0x100000          # never dereferenced: every call below fails validation first


def call(**over):
    a = dict(target=AT, tt=1, ts=500, tr=100, draft=AT, dt=0, ds=400, dr=100, tokens=AT, lengths=None, temperature=None, ua=AT, us=AT, B=2, S=4,
             V=100, out=AT + 4096, kept=AT + 8192, ws=AT, ws_bytes=256)
    a.update(over)
    return B.lib().cat_verify_drafts(a["target"], a["tt"], a["ts"], a["tr"], a["draft"], a["dt"], a["ds"], a["dr"], a["tokens"], a["lengths"],
                                     a["temperature"], a["ua"], a["us"], a["B"], a["S"], a["V"], a["out"], a["kept"], a["ws"], a["ws_bytes"], None)


BAD = [(dict(target=None), 1), (dict(us=None), 1), (dict(out=None), 1), (dict(kept=None), 1), (dict(tokens=None), 1), (dict(ua=None), 1),
       (dict(B=-1), 2), (dict(S=-1), 2), (dict(V=0), 2), (dict(tt=3), 2), (dict(dt=-1), 2), (dict(tr=99), 2), (dict(dr=99), 2), (dict(ts=99), 2),
       (dict(ds=0), 2), (dict(B=(1 << 20) + 1), 7), (dict(S=257), 7), (dict(V=(1 << 22) + 1), 7),
       (dict(target=AT + 1), 3), (dict(draft=AT + 2), 3), (dict(tokens=AT + 2), 3), (dict(lengths=AT + 1), 3), (dict(temperature=AT + 2), 3),
       (dict(ua=AT + 1), 3), (dict(us=AT + 2), 3), (dict(out=AT + 2), 3), (dict(kept=AT + 3), 3),
       (dict(tokens=AT + 4096 + 36), 2), (dict(ua=AT + 4064 + 4), 2), (dict(us=AT + 8196), 2), (dict(lengths=AT + 8192), 2), (dict(temperature=AT + 4096), 2),
       (dict(kept=AT + 4096 + 36), 2), (dict(ws=None), 4), (dict(ws_bytes=255), 4), (dict(ws=AT + 4), 4)]


@pytest.mark.parametrize("over,status", BAD)
def test_argument_errors_return_before_any_device_work(over, status):
    before = B.lib().cat_kernel_launches()
    assert call(**over) == status
    assert B.lib().cat_kernel_launches() == before


def test_an_empty_batch_is_no_error():
    assert call(B=0, target=None, out=None, kept=None) == 0


def test_binding_refuses_cpu_tensors():
    import torch
    with pytest.raises(TypeError):
        B.cat_verify_drafts(torch.zeros((1, 1, 4)), None, torch.zeros((1, 0), dtype=torch.int32), torch.zeros((1, 0)), torch.zeros(1))


def test_oracle_a_sequence_without_drafts_is_a_draw_from_its_row():
    row = np.log(np.array([0.1, 0.2, 0.3, 0.4]))
    for u, want in [(0.0, 0), (0.05, 0), (0.15, 1), (0.31, 2), (0.59, 2), (0.61, 3), (0.999, 3)]:
        out, kept, _ = O.verify(row[None, None], None, np.zeros((1, 0)), np.zeros((1, 0)), [u])
        assert out[0, 0] == want and kept[0] == 0


def test_oracle_the_tokens_are_distributed_as_the_target_draws_them():
    """The theorem behind the rule: over the draft's draws and the uniform numbers, the first token has the target's distribution."""
    rng = np.random.default_rng(0)
    p, q = rng.dirichlet(np.ones(5)), rng.dirichlet(np.ones(5))
    n = 200_000
    x = rng.choice(5, size=n, p=q)
    ua, us = rng.random(n), rng.random(n)
    rest = np.maximum(p - q, 0)
    first = np.where(ua * q[x] < p[x], x, np.array([O.draw(rest, u)[0] for u in us]))
    assert np.abs(np.bincount(first, minlength=5) / n - p).max() < 5 * np.sqrt(0.25 / n)
    for i in range(200):
        out, kept, _ = O.verify(np.log(np.stack([p, p]))[None], np.log(q)[None, None], x[i:i + 1, None], ua[i:i + 1, None], us[i:i + 1])
        assert out[0, 0] == first[i] and kept[0] == int(ua[i] * q[x[i]] < p[x[i]])


def test_oracle_masks_greedy_and_rows_without_mass():
    inf, nan = np.inf, np.nan
    t = np.array([[[1.0, 3.0, 3.0, nan], [0.0, -inf, 5.0, 5.0], [-inf, -inf, -inf, nan]]])
    out, kept, _ = O.verify(t, t[:, :2], np.array([[1, 2]]), np.zeros((1, 2)), [0.5], temperature=[0.0])
    assert out.tolist() == [[1, 2, -1]] and kept[0] == 2
    out, kept, _ = O.verify(t, t[:, :2], np.array([[2, 2]]), np.zeros((1, 2)), [0.5], temperature=[0.0])
    assert out.tolist() == [[1, -1, -1]] and kept[0] == 0
    out, kept, _ = O.verify(t, None, np.array([[9, 0]]), np.zeros((1, 2)), [0.0], lengths=[1])
    assert out.tolist() == [[0, -1, -1]] and kept[0] == 0
    assert O.masses([inf, 1.0, inf], 1.0).tolist() == [0.5, 0.0, 0.5]
    assert O.masses([-3.4e38, -3.4e38], 1.0).tolist() == [0.5, 0.5]


@pytest.mark.parametrize("over", [dict(out=AT), dict(kept=AT + 1996), dict(draft=AT + 16384, out=AT + 16384 + 3196), dict(draft=AT + 16384, kept=AT + 16384),
                                  dict(target=AT + 4096 - 1996), dict(ts=1 << 61, target=AT + 65536, out=AT + 131072)])
def test_outputs_among_the_logits_are_refused(over):
    """The first and the last of 2 x (5 rows of 100 bf16) and 2 x (4 rows of 100 fp32); distances whose bytes pass 64 bits."""
    assert call(**over) == 2


def test_outputs_next_to_the_logits_are_not():
    assert call(out=AT + 3200, kept=AT + 3240, ws=None) == 4
    assert call(target=AT + 4096 + 40, ws=None) == 4
