"""Refusals of the 8-bit key/value cache's operators: bad arguments come back as
statuses before anything reaches the GPU."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def L():
    from paper_2609_00049_gb300 import build as b
    b.build()
    import paper_2609_00049_gb300 as rq
    return rq.lib()


FAKE, OTHER = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x20000)   # never dereferenced
ODD = ctypes.c_void_p(0x10001)
OFF2 = ctypes.c_void_p(0x10002)
BIG = 1 << 40
INVALID, WORKSPACE, UNSUPPORTED = 1, 2, 7


def cache(**kw):
    import paper_2609_00049_gb300 as rq
    c = dict(n_layers=2, n_pages=10, n_kv=2, page_size=64, head_dim=64, scale_block=16, k_codes=0x10000, v_codes=0x20000,
             k_scale=0x30000, v_scale=0x40000)
    c.update(kw)
    return ctypes.byref(rq.KvCache(*c.values()))


def pages(**kw):
    import paper_2609_00049_gb300 as rq
    p = dict(n_pages=10, n_rows=3, max_pages=5, used=0x10000, tables=0x20000, lengths=0x30000)
    p.update(kw)
    return ctypes.byref(rq.KvPages(*p.values()))


BAD_CACHES = [dict(n_layers=0), dict(n_pages=0), dict(n_kv=0), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(scale_block=0),
              dict(scale_block=12), dict(scale_block=128), dict(head_dim=0), dict(head_dim=40), dict(head_dim=272), dict(k_codes=None),
              dict(v_codes=None), dict(k_scale=None), dict(v_scale=None), dict(k_codes=0x10008), dict(v_codes=0x10001), dict(k_scale=0x10002),
              dict(v_scale=0x10001)]
LARGE_CACHES = [dict(n_kv=5000), dict(n_pages=1 << 30), dict(n_layers=1 << 20)]


def every_cache(call):
    for bad in BAD_CACHES:
        assert call(c=cache(**bad)) == INVALID, bad
    for big in LARGE_CACHES:
        assert call(c=cache(**big)) == UNSUPPORTED, big
    assert call(c=None) == INVALID


def test_rotary_refusals(L):
    def call(T=4, D=64, R=64, pos=FAKE, f=FAKE, il=0, amp=1.0, back=0, dt=1, nq=4, q=FAKE, qld=256, qhs=64, qo=OTHER, qold=256, qohs=64, nk=2,
             k=FAKE, kld=128, khs=64, ko=OTHER, kold=128, kohs=64):
        return L.realq_rotary(None, T, D, R, pos, f, il, amp, back, dt, nq, q, qld, qhs, qo, qold, qohs, nk, k, kld, khs, ko, kold, kohs)
    for bad in (dict(T=-1), dict(D=1), dict(D=1025), dict(R=0), dict(R=7), dict(R=66), dict(dt=2), dict(amp=math.nan), dict(amp=math.inf),
                dict(nq=0, nk=0), dict(nq=-1), dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(q=ODD), dict(qo=ODD),
                dict(k=ODD), dict(pos=None), dict(f=None), dict(pos=ctypes.c_void_p(0x10004)), dict(f=ctypes.c_void_p(0x10004)), dict(qhs=63),
                dict(qld=255), dict(qold=64), dict(khs=-64), dict(kohs=10), dict(qo=FAKE, qold=300), dict(ko=FAKE, kohs=64, kold=129),
                dict(dt=0, q=OFF2)):
        assert call(**bad) == INVALID, bad
    assert call(T=(1 << 30) + 1) == UNSUPPORTED and call(nq=70000, qld=1 << 30, qold=1 << 30) == UNSUPPORTED
    assert call(qld=1 << 41) == UNSUPPORTED
    assert call(T=0, q=None, pos=None) == 0
    out = (ctypes.c_double * 64)()
    freq = lambda R=64, base=1e4, sc=0, factor=2.0, ctx=8192.0, lo=1.0, hi=4.0, o=out: L.realq_rotary_frequencies(R, base, sc, factor, ctx, lo, hi, o)  # noqa: E731
    for bad in (dict(R=0), dict(R=5), dict(R=2048), dict(base=0.0), dict(base=math.nan), dict(sc=4), dict(sc=-1), dict(sc=1, factor=0.0),
                dict(sc=3, factor=math.inf), dict(sc=3, ctx=0.0), dict(sc=3, lo=4.0), dict(sc=3, hi=math.nan), dict(o=None)):
        assert freq(**bad) == INVALID, bad
    assert freq() == 0 and freq(factor=-1.0) == 0      # plain: the factor is not read


def test_append_and_read_refusals(L):
    def app(c=None, layer=1, S=3, T=5, k=FAKE, kld=128, khs=64, v=FAKE, vld=128, vhs=64, dt=1, st=FAKE, pos=FAKE, tab=FAKE, M=5):
        return L.realq_kv_append(None, c, layer, S, T, k, kld, khs, v, vld, vhs, dt, st, pos, tab, M)

    def read(c=None, layer=1, S=3, T=5, st=FAKE, pos=FAKE, tab=FAKE, M=5, k=FAKE, v=OTHER, dt=1):
        return L.realq_kv_read(None, c, layer, S, T, st, pos, tab, M, k, v, dt)
    every_cache(app)
    every_cache(read)
    both = (dict(layer=-1), dict(layer=2), dict(S=-1), dict(T=-1), dict(M=-1), dict(dt=2), dict(st=None), dict(pos=None), dict(tab=None),
            dict(st=ODD), dict(tab=OFF2), dict(pos=ctypes.c_void_p(0x10004)), dict(k=ODD), dict(v=ODD))
    for bad in both + (dict(k=None), dict(v=None), dict(kld=127), dict(khs=63), dict(vld=1), dict(dt=0, v=OFF2)):
        assert app(**{"c": cache(), **bad}) == INVALID, bad
    for bad in both:
        assert read(**{"c": cache(), **bad}) == INVALID, bad
    for call in (app, read):
        assert call(c=cache(), S=(1 << 24) + 1) == UNSUPPORTED and call(c=cache(), T=(1 << 30) + 1) == UNSUPPORTED
        assert call(c=cache(), M=(1 << 24) + 1) == UNSUPPORTED
        assert call(c=cache(), T=0, st=None, pos=None, tab=None) == 0


def test_attention_refusals(L):
    import paper_2609_00049_gb300 as rq

    def call(c=None, layer=0, S=3, T=5, H=8, q=FAKE, ld=512, hs=64, dt=1, st=FAKE, ln=FAKE, tab=FAKE, M=5, scale=0.1, causal=1, window=0,
             mx=5, out=FAKE, lse=FAKE, ws=FAKE, size=BIG):
        return L.realq_kv_attention(None, c, layer, S, T, H, q, ld, hs, dt, st, ln, tab, M, scale, causal, window, mx, out, lse, ws, size)
    every_cache(call)
    for bad in (dict(layer=2), dict(S=-1), dict(T=-1), dict(M=-1), dict(H=0), dict(H=7), dict(dt=3), dict(scale=math.nan), dict(scale=math.inf),
                dict(window=-1), dict(window=5, causal=0), dict(mx=0), dict(q=None), dict(q=ODD), dict(ld=511), dict(hs=32), dict(st=None),
                dict(ln=None), dict(tab=None), dict(out=None), dict(out=ODD), dict(lse=OFF2), dict(ln=ODD), dict(dt=0, q=OFF2)):
        assert call(**{"c": cache(), **bad}) == INVALID, bad
    assert call(c=cache(n_kv=1), H=2048, ld=1 << 20) == UNSUPPORTED and call(c=cache(n_kv=1), T=1 << 29, H=4) == UNSUPPORTED
    for bad in (dict(ws=None), dict(ws=ODD), dict(size=100)):
        assert call(**{"c": cache(), **bad}) == WORKSPACE, bad
    assert call(c=cache(), T=0, q=None, st=None) == 0 and call(c=cache(), S=0) == 0
    size = L.realq_kv_attention_workspace_size
    assert size(cache(), 3, 5, 8) > 0 and size(cache(), 3, 5, 7) == 0 and size(cache(), 0, 5, 8) == 0 and size(cache(page_size=8), 3, 5, 8) == 0
    assert "kv_attention" in (call(c=cache(), H=7), rq.realq_last_error())[1]


def test_page_refusals(L):
    def reserve(p=None, st=FAKE, T=4, pos=FAKE, c=None, ws=FAKE, size=BIG):
        return L.realq_pages_reserve(None, p, st, T, pos, cache() if c is None else c, ws, size)

    def fork(p=None, n=2, src=FAKE, dst=OTHER, ws=FAKE, size=BIG):
        return L.realq_pages_fork(None, p, n, src, dst, ws, size)

    def release(p=None, n=2, rows=FAKE):
        return L.realq_pages_release(None, p, n, rows)

    def compact(p=None, c=None, u=FAKE, t=OTHER, m=ctypes.c_void_p(0x50000), ws=FAKE, size=BIG):
        return L.realq_pages_compact(None, p, cache() if c is None else c, u, t, m, ws, size)
    for call in (reserve, fork, release, compact):
        for bad in (dict(n_pages=0), dict(n_rows=0), dict(max_pages=0), dict(used=None), dict(tables=None), dict(lengths=None), dict(used=0x10001),
                    dict(tables=0x10002), dict(lengths=0x10001)):
            assert call(p=pages(**bad)) == INVALID, bad
        for big in (dict(n_pages=1 << 30), dict(n_rows=(1 << 24) + 1), dict(max_pages=(1 << 24) + 1)):
            assert call(p=pages(**big)) == UNSUPPORTED, big
        assert call(p=None) == INVALID
        if call is not release:
            for bad in (dict(ws=None), dict(ws=ODD), dict(size=8)):
                assert call(p=pages(), **bad) == WORKSPACE, bad
    for call in (reserve, compact):
        assert call(p=pages(), c=cache(n_pages=11)) == INVALID
        for bad in BAD_CACHES:
            assert call(p=pages(), c=cache(**bad)) == INVALID, bad
    for bad in (dict(st=None), dict(T=-1), dict(pos=None), dict(st=ODD), dict(pos=ctypes.c_void_p(0x10004))):
        assert reserve(p=pages(), **bad) == INVALID, bad
    assert reserve(p=pages(), T=(1 << 30) + 1) == UNSUPPORTED
    for bad in (dict(n=-1), dict(src=None), dict(dst=None), dict(src=ODD), dict(dst=OFF2)):
        assert fork(p=pages(), **bad) == INVALID, bad
    assert fork(p=pages(), n=0, src=None) == 0 and fork(p=pages(), n=(1 << 24) + 1) == UNSUPPORTED
    for bad in (dict(n=-1), dict(rows=None), dict(rows=ODD)):
        assert release(p=pages(), **bad) == INVALID, bad
    assert release(p=pages(), n=0, rows=None) == 0 and release(p=pages(), n=(1 << 24) + 1) == UNSUPPORTED
    for bad in (dict(u=None), dict(t=None), dict(m=None), dict(u=ODD), dict(t=OFF2), dict(m=ODD), dict(m=FAKE), dict(m=OTHER), dict(m=ctypes.c_void_p(0x20000))):
        assert compact(p=pages(), **bad) == INVALID, bad
    copy = lambda c=None, n=2, src=FAKE, dst=FAKE: L.realq_pages_copy(None, c, n, src, dst)  # noqa: E731
    every_cache(copy)
    for bad in (dict(n=-1), dict(src=None), dict(dst=None), dict(src=ODD), dict(dst=OFF2)):
        assert copy(c=cache(), **bad) == INVALID, bad
    assert copy(c=cache(), n=0, src=None) == 0 and copy(c=cache(), n=(1 << 30) + 1) == UNSUPPORTED
    assert L.realq_pages_workspace_size(10, 3, 5) > 0 and L.realq_pages_workspace_size(0, 3, 5) == 0 and L.realq_pages_workspace_size(10, 3, 0) == 0


def test_binding_refusals(L):
    import paper_2609_00049_gb300 as rq
    codes, scale = torch.zeros(1, 4, 2, 16, 32, dtype=torch.uint8), torch.zeros(1, 4, 2, 2)
    for bad in (dict(k_codes=codes[0]), dict(k_scale=scale[..., :0]), dict(k_scale=torch.zeros(1, 4, 2, 3)), dict()):   # the last: host tensors
        with pytest.raises(ValueError):
            rq.kv_cache(**{**dict(k_codes=codes, v_codes=codes, k_scale=scale, v_scale=scale), **bad})
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        rq.kv_pages(i, i, i)
    with pytest.raises(ValueError):
        rq.kv_pages(i, i.view(2, 2), i[:2])      # host tensors
    x = torch.zeros(3, 2, 32)
    with pytest.raises(ValueError):
        rq.realq_rotary(x, torch.zeros(3, dtype=torch.int64), torch.zeros(16, dtype=torch.float64), x)
    with pytest.raises(ValueError):
        rq.realq_rotary_frequencies(64, scaling="something")
    with pytest.raises(rq.RealqError):
        rq.realq_rotary_frequencies(7)
    assert rq.realq_status_string(rq.REALQ_ERR_NO_PAGES) == "too few free pages or table entries"


def test_layouts_and_limits(L):
    """Heads within a token's row or tokens within a head's; neither where they meet."""
    T, H, D = 5, 8, 64
    call = lambda ld, hs, S=3, ws=None: L.realq_kv_attention(   # noqa: E731
        None, cache(), 0, S, T, H, FAKE, ld, hs, 1, FAKE, FAKE, FAKE, 5, 0.1, 1, 0, 5, FAKE, None, ws, 0)
    assert call(D, T * D) == WORKSPACE and call(H * D, D) == WORKSPACE       # (past the layout, the missing workspace)
    assert call(2 * D, 2 * T * D) == WORKSPACE and call(D, T * D - 1) == INVALID and call(D - 1, T * D) == INVALID
    assert call(H * D - 1, D) == INVALID and call(2 * D, T * D) == INVALID and call(0, T * D) == INVALID
    assert call(H * D, D, S=(1 << 20) + 1) == UNSUPPORTED
