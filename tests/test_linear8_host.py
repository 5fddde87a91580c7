"""Refusals of the 8-bit linear operators and the token log probabilities: bad
arguments come back as statuses before anything reaches the GPU."""
import ctypes
import types

import pytest
import torch


@pytest.fixture(scope="module")
def L():
    from paper_2609_00049_gb300 import build as b
    b.build()
    import paper_2609_00049_gb300 as rq
    return rq.lib()


FAKE = ctypes.c_void_p(0x10000)   # never dereferenced: every call below fails validation first
ODD = ctypes.c_void_p(0x10001)
BIG = 1 << 40
INVALID, WORKSPACE, UNSUPPORTED = 1, 2, 7


def test_product_refusals(L):
    def call(T=4, n=64, m=32, x=FAKE, xs=FAKE, w=FAKE, bits=8, ws=FAKE, wz=None, y=FAKE, dt=1, buf=FAKE, size=BIG):
        return L.realq_int8_product(None, T, n, m, x, xs, w, bits, ws, wz, y, dt, buf, size)
    for bad in (dict(T=-1), dict(n=0), dict(m=0), dict(bits=2), dict(bits=5), dict(dt=2), dict(x=None), dict(xs=None),
                dict(w=None), dict(ws=None), dict(y=None), dict(y=ODD)):
        assert call(**bad) == INVALID, bad
    assert call(n=131072) == UNSUPPORTED and call(T=1 << 30) == UNSUPPORTED and call(m=1 << 30) == UNSUPPORTED
    assert call(buf=None) == WORKSPACE and call(buf=ODD) == WORKSPACE and call(size=0) == WORKSPACE
    assert call(T=0, x=None) == 0
    import paper_2609_00049_gb300 as rq
    assert "int8_product" in (call(n=0), rq.realq_last_error())[1]
    assert rq.realq_int8_product_workspace_size(0, 8, 8) == 0 and rq.realq_int8_product_workspace_size(8, 8, 8, 3) == 0
    assert rq.realq_int8_product_workspace_size(8, 8, 8) > 0


def test_logprobs_refusals(L):
    def call(T=4, V=100, ld=100, x=FAKE, dt=1, y=FAKE, lp=FAKE, norm=FAKE, H=FAKE, k=2, ids=FAKE, top=FAKE):
        return L.realq_token_logprobs(None, T, V, ld, x, dt, y, lp, norm, H, k, ids, top)
    for bad in (dict(T=-1), dict(V=0), dict(ld=99), dict(dt=3), dict(k=-1), dict(k=33), dict(x=None), dict(y=None),
                dict(ids=None), dict(x=ODD)):
        assert call(**bad) == INVALID, bad
    assert call(V=2 ** 31, ld=2 ** 31) == UNSUPPORTED and call(T=2 ** 29) == UNSUPPORTED
    assert call(T=0, x=None) == 0

    def grad(T=4, V=100, ld=100, x=FAKE, dt=0, y=FAKE, norm=FAKE, g=FAKE, H=FAKE, gH=FAKE, k=2, ids=FAKE, gt=FAKE, ldd=100,
             d=ctypes.c_void_p(0x20000)):
        return L.realq_token_logprobs_grad(None, T, V, ld, x, dt, y, norm, g, H, gH, k, ids, gt, ldd, d)
    for bad in (dict(T=-1), dict(V=0), dict(ld=99), dict(ldd=99), dict(dt=3), dict(k=33), dict(x=None), dict(y=None),
                dict(norm=None), dict(H=None), dict(ids=None), dict(gt=None), dict(d=None), dict(d=ODD),
                dict(d=FAKE, ldd=104)):
        assert grad(**bad) == INVALID, bad
    assert grad(V=2 ** 31, ld=2 ** 31, ldd=2 ** 31) == UNSUPPORTED
    assert grad(T=0, x=None) == 0


def test_checkpoint_refusals(L):
    for call in (lambda T=4, n=64, x=FAKE, dt=1, c=FAKE, e=FAKE: L.realq_checkpoint_pack(None, T, n, x, dt, c, e),
                 lambda T=4, n=64, x=FAKE, dt=1, c=FAKE, e=FAKE: L.realq_checkpoint_unpack(None, T, n, c, e, x, dt)):
        for bad in (dict(T=-1), dict(n=0), dict(dt=2), dict(x=None), dict(c=None), dict(e=None), dict(x=ODD)):
            assert call(**bad) == INVALID, bad
        assert call(T=1 << 45) == UNSUPPORTED and call(T=0, x=None) == 0

    def grad(T=4, m=8, n=64, dy=FAKE, dt=1, c=FAKE, e=FAKE, dW=FAKE, buf=FAKE, size=BIG):
        return L.realq_checkpoint_weight_grad(None, T, m, n, dy, dt, c, e, dW, 0, buf, size)
    for bad in (dict(T=-1), dict(m=0), dict(n=0), dict(dt=2), dict(dy=None), dict(c=None), dict(e=None), dict(dW=None),
                dict(dy=ctypes.c_void_p(0x10004))):
        assert grad(**bad) == INVALID, bad
    assert grad(T=1 << 29) == UNSUPPORTED and grad(m=1 << 30) == UNSUPPORTED
    assert grad(buf=None) == WORKSPACE and grad(size=16) == WORKSPACE and grad(buf=ODD) == WORKSPACE


def test_binding_refusals(L):
    import paper_2609_00049_gb300 as rq
    c, s = torch.zeros(2, 8, dtype=torch.uint8), torch.zeros(2)
    with pytest.raises(ValueError):      # W_codes of another width
        rq.realq_int8_product(c, s, torch.zeros(3, 9, dtype=torch.uint8), torch.zeros(3), torch.zeros(2, 3))
    with pytest.raises(ValueError):      # host tensors
        rq.realq_int8_product(c, s, torch.zeros(3, 8, dtype=torch.uint8), torch.zeros(3), torch.zeros(2, 3),
                              stream=types.SimpleNamespace(cuda_stream=0))
    with pytest.raises(ValueError):
        rq.realq_token_logprobs(torch.zeros(4, 3).t(), torch.zeros(3, dtype=torch.int64), torch.zeros(3))
    with pytest.raises(ValueError):
        rq.realq_checkpoint_pack(torch.zeros(2, 40), torch.zeros(2, 40, dtype=torch.int8), torch.zeros(2, 1, dtype=torch.uint8))
