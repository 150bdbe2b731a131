"""cat_linear's checks of arguments: on the host, before anything reaches a GPU."""
import ctypes

import pytest

from paper_2509_26277_b200 import binding as B

AT = 0x100000          # never dereferenced: every call below fails validation first


def call(**over):
    a = dict(X=AT, ldx=64, W=AT, ldw=64, in_type=1, bias=None, bias_type=0, residual=None, ldr=0, act=0, M=8, N=16, K=64, Y=AT, ldy=16,
             out_type=0, ws=AT, ws_bytes=1 << 20)
    a.update(over)
    return B.lib().cat_linear(a["X"], a["ldx"], a["W"], a["ldw"], a["in_type"], a["bias"], a["bias_type"], a["residual"], a["ldr"], a["act"],
                              a["M"], a["N"], a["K"], a["Y"], a["ldy"], a["out_type"], a["ws"], a["ws_bytes"], None)


BAD = [(dict(X=None), 1), (dict(W=None), 1), (dict(Y=None), 1),
       (dict(M=-1), 2), (dict(N=0), 2), (dict(K=0), 2), (dict(ldx=63), 2), (dict(ldw=0), 2), (dict(ldy=15), 2), (dict(residual=AT, ldr=15), 2),
       (dict(in_type=0), 2), (dict(in_type=3), 2), (dict(out_type=-1), 2), (dict(out_type=3), 2), (dict(bias=AT, bias_type=3), 2),
       (dict(act=5), 2), (dict(act=-1), 2), (dict(residual=AT, Y=AT, ldr=20), 2),
       (dict(X=AT + 1), 3), (dict(W=AT + 1), 3), (dict(Y=AT + 2), 3), (dict(bias=AT + 2, bias_type=0), 3), (dict(residual=AT + 2, ldr=16), 3),
       (dict(ws=None), 4), (dict(ws_bytes=255), 4), (dict(ws=AT + 8), 4), (dict(X=AT + 2, ws_bytes=256), 4), (dict(ldw=65, ws_bytes=256), 4),
       (dict(M=(1 << 24) + 1), 7), (dict(N=(1 << 20) + 1, ldy=1 << 21), 7), (dict(K=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), 7),
       (dict(ldx=1 << 31), 7), (dict(ldw=1 << 31), 7)]


@pytest.mark.parametrize("over,status", BAD)
def test_argument_errors_return_before_any_device_work(over, status):
    before = B.lib().cat_kernel_launches()
    assert call(**over) == status
    assert B.lib().cat_kernel_launches() == before


def test_an_empty_batch_is_no_error():
    assert call(M=0, X=None, Y=None) == 0


def test_workspace_query_looks_at_the_addresses():
    q = B.lib().cat_linear_workspace_bytes
    assert q(AT, 64, AT, 64, 8, 16, 64) == 256
    assert q(AT + 2, 64, AT, 64, 8, 16, 64) == 256 + 8 * 64 * 2
    assert q(AT, 65, AT, 64, 8, 16, 64) == 256 + 8 * 64 * 2
    assert q(AT, 64, AT, 61, 8, 16, 61) == 256 + 16 * 64 * 2
    assert q(AT, 1, AT, 64, 1, 16, 61) == 256          # the distance of one row says nothing
    assert q(AT, 64, AT, 64, 8, 0, 64) == 0 and q(AT, 63, AT, 64, 8, 16, 64) == 0


def test_binding_refuses_cpu_tensors():
    import torch
    x = torch.zeros((8, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        B.cat_linear(x, x)
    assert ctypes.sizeof(ctypes.c_void_p) == 8


@pytest.mark.parametrize("over", [dict(Y=AT), dict(X=AT + 65536, Y=AT), dict(X=AT + 65536, Y=AT + 8 * 16 * 4 - 4, bias=AT + 65536 * 2, W=AT + 8 * 16 * 4),
                                  dict(X=AT + 65536, W=AT + 131072, bias=AT + 4, Y=AT), dict(X=AT + 65536, W=AT + 131072, residual=AT + 64, ldr=16, Y=AT),
                                  dict(X=AT, ldx=128, Y=AT + 124, ldy=64), dict(X=AT + 128, ldx=128, W=AT + 65536, Y=AT + 192, ldy=64),
                                  dict(X=AT, ldx=128, W=AT + 65536, Y=AT + 256 * 7 + 64, ldy=100), dict(M=1, X=AT + 65536, W=AT + 128, Y=AT + 124, ldy=1)])
def test_results_among_what_is_read_are_refused(over):
    assert call(**over) == 2


@pytest.mark.parametrize("over", [dict(ldy=1 << 62), dict(ldy=(1 << 36) + 1), dict(residual=AT + (1 << 40), ldr=1 << 62), dict(M=2, ldy=(1 << 63) - 1)])
def test_row_distances_whose_bytes_pass_64_bits_are_refused(over):
    assert call(**dict(dict(Y=AT + (1 << 30)), **over)) == 7
