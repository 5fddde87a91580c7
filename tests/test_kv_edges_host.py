"""Refusals of the 8-bit key/value cache's operators that go by more than one argument."""
import ctypes

import pytest
import torch

import paper_2609_00049_gb300 as rq

FAKE = ctypes.c_void_p(0x10000)   # never dereferenced
INVALID, WORKSPACE = 1, 2


@pytest.fixture(scope="module")
def L():
    from paper_2609_00049_gb300 import build as b
    b.build()
    return rq.lib()


def test_a_scale_that_base_two_cannot_hold(L):
    """Scores are formed in base 2: scale log2(e) has to be a number too."""
    cache = rq.KvCache(2, 10, 2, 64, 64, 16, 0x10000, 0x20000, 0x30000, 0x40000)
    call = lambda scale: L.realq_kv_attention(None, ctypes.byref(cache), 0, 3, 5, 8, FAKE, 512, 64, 1, FAKE, FAKE, FAKE, 5, scale, 1, 0, 5, FAKE, None, None, 0)  # noqa: E731
    for scale in (2.4e38, -2.4e38, 3.4e38):
        assert call(scale) == INVALID, scale
    for scale in (2.3e38, -2.3e38, 0.0, 1.0):          # (past the scale, the missing workspace)
        assert call(scale) == WORKSPACE, scale


def test_a_pool_and_a_cache_on_different_devices():
    cache, pages = rq.KvCache(2, 10, 2, 64, 64, 16, 0x10000, 0x20000, 0x30000, 0x40000), rq.KvPages(10, 3, 5, 0x10000, 0x20000, 0x30000)
    cache.device, pages.device = 0, 1
    i = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: rq.realq_pages_reserve(pages, i, i.long(), cache), lambda: rq.realq_pages_compact(pages, cache, i, i, i)):
        with pytest.raises(ValueError, match="cache and pool"):
            call()
