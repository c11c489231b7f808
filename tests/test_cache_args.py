"""What the windowed-attention and cache entry points refuse, and the calls that
have nothing to do (CPU only: the checks run before any HIP call)."""
import ctypes
import math

import pytest

import paper_2602_02071_amd as baps

BAD, NOT, OK = baps.BAPS_INVALID_ARGUMENT, baps.BAPS_UNSUPPORTED, baps.BAPS_OK
A = 4096                               # an aligned address that no call may reach


@pytest.fixture(scope="module")
def lib():
    return baps.load()


def _cache(**kw):
    c = dict(k=A, v=A, k_exp=A, v_exp=A, layers=2, num_pages=8, Hkv=2, page=16, D=64)
    c.update(kw)
    return baps.baps_cache_t(*(c[f] for f, _ in baps.baps_cache_t._fields_))


BAD_CACHES = [(dict(k=None), BAD), (dict(v_exp=None), BAD), (dict(k=A + 8), BAD), (dict(v=A + 1), BAD), (dict(layers=-1), BAD),
              (dict(num_pages=-2), BAD), (dict(Hkv=-1), BAD), (dict(page=48), NOT), (dict(page=8), NOT), (dict(D=96), NOT),
              (dict(D=256), NOT), (dict(Hkv=40000), NOT)]


def test_window(lib):
    def call(q=A, k=A, v=A, o=A, B=1, Hq=4, Hkv=2, Sq=8, Sk=64, D=64, window=5, sinks=0, block=64, prm=None, ws=None, n=0):
        return lib.baps_attention_window(q, k, v, o, None, B, Hq, Hkv, Sq, Sk, D, window, sinks, block,
                                         ctypes.byref(prm) if prm else None, ws, n, None)
    assert call(window=0) == BAD and call(window=-1) == BAD and call(sinks=-1) == BAD
    assert call(q=None) == BAD and call(k=A + 2) == BAD and call(o=None) == BAD and call(Hq=3) == BAD and call(B=-1) == BAD
    assert call(D=96) == NOT and call(block=48) == NOT and call(block=256) == NOT
    assert call(B=0, q=None) == OK and call(Sq=0, q=None, o=None) == OK
    assert call(prm=baps._params(mode=baps.BAPS_MODE_EXP2_HIF8)) == NOT
    assert call(prm=baps._params(lam=9)) == NOT
    assert call(prm=baps._params(tie_mode=baps.BAPS_TIES_EVEN)) == NOT
    assert call(prm=baps._params(qk_scales=(1.0, 1.0))) == NOT
    assert call(prm=baps._params(restart_rows=2)) == NOT
    assert call(prm=baps._params(mode=5)) == BAD and call(prm=baps._params(scale_log2=-1.0)) == BAD
    # a workspace that is needed: missing, short, misaligned
    d = baps._params(mode=baps.BAPS_MODE_DEFAULT)
    long = dict(Sq=1, Sk=9000, window=5000, D=128, prm=d)
    need = baps.baps_attention_window_workspace(1, 4, 2, 1, 9000, 128, 5000, 0, 64, mode=baps.BAPS_MODE_DEFAULT)
    assert need > 0 and need % 256 == 0
    assert call(**long) == BAD and call(**long, ws=A, n=need - 1) == BAD and call(**long, ws=A + 16, n=need) == BAD
    assert baps.baps_attention_window_workspace(1, 4, 2, 90000, 90000, 128, 5000, 0, 64, mode=baps.BAPS_MODE_DEFAULT) == 0
    assert baps.baps_attention_window_workspace(1, 4, 2, 1, 9000, 128, 0, 0, 64, mode=baps.BAPS_MODE_DEFAULT) == 0
    assert baps.baps_attention_window_workspace(1, 4, 2, 1, 9000, 128, 5000, 0, 64) == 0


def test_append(lib):
    def call(c=None, layer=0, k=A, v=A, stride=128, cu=A, lens=A, table=A, width=4, B=2, total=5, most=3):
        c = c or _cache()
        return lib.baps_cache_append(ctypes.byref(c), layer, k, v, stride, cu, lens, table, width, B, total, most, None)
    for kw, status in BAD_CACHES:
        assert call(_cache(**kw)) == status, kw
    assert lib.baps_cache_append(None, 0, A, A, 128, A, A, A, 4, 2, 5, 3, None) == BAD
    assert call(layer=2) == BAD and call(layer=-1) == BAD
    for name in ("k", "v", "cu", "lens", "table"):
        assert call(**{name: None}) == BAD, name
    assert call(k=A + 2) == BAD and call(v=A + 8) == BAD
    assert call(stride=127) == BAD and call(stride=132) == BAD and call(stride=120) == BAD
    for name in ("width", "B", "total", "most"):
        assert call(**{name: -1}) == BAD, name
    assert call(most=2 ** 31 - 1, B=1000) == NOT and call(width=1 << 27) == NOT
    # nothing to do
    for kw in (dict(B=0), dict(total=0), dict(most=0), dict(width=0)):
        assert call(**kw) == OK, kw
    assert call(_cache(num_pages=0)) == OK and call(_cache(Hkv=0)) == OK


def test_attention(lib):
    def call(c=None, layer=1, q=A, stride=256, o=A, cu=A, lens=A, table=A, width=4, B=2, Hq=4, T=6, mq=3, ml=60, window=0, sinks=0,
             scale=0.0, ws=None, n=0):
        c = c or _cache()
        return lib.baps_cache_attention(ctypes.byref(c), layer, q, stride, o, None, cu, lens, table, width, B, Hq, T, mq, ml, window,
                                        sinks, scale, ws, n, None)
    for kw, status in BAD_CACHES:
        assert call(_cache(**kw), Hq=2 * kw.get("Hkv", 2), stride=1 << 24) == status, kw
    assert call(layer=2) == BAD and call(layer=-1) == BAD
    for name in ("q", "o", "cu", "lens", "table"):
        assert call(**{name: None}) == BAD, name
    assert call(q=A + 2) == BAD and call(o=A + 8) == BAD and call(stride=252) == BAD and call(stride=260) == BAD
    for name in ("width", "B", "Hq", "T", "mq", "ml", "window", "sinks"):
        assert call(**{name: -1}) == BAD, name
    for scale in (-1.0, math.inf, math.nan):
        assert call(scale=scale) == BAD
    assert call(Hq=3) == BAD and call(_cache(Hkv=0)) == BAD
    assert call(B=70000) == NOT and call(width=0) == NOT and call(_cache(num_pages=0)) == NOT and call(mq=2 ** 31 - 1) == NOT
    assert call(width=1 << 27) == NOT
    for kw in (dict(B=0), dict(Hq=0), dict(T=0), dict(mq=0)):
        assert call(**kw) == OK, kw
    need = baps.baps_cache_attention_workspace(_cache(), 2, 4, 6, 3, 20000)
    assert need > 0
    assert call(ml=20000) == BAD and call(ml=20000, ws=A, n=need - 1) == BAD and call(ml=20000, ws=A + 128, n=need) == BAD
    assert baps.baps_cache_attention_workspace(_cache(), 2, 4, 6, 3, 20000, 100, 4) == 0        # a short window: no split
    assert baps.baps_cache_attention_workspace(_cache(), 200, 4, 600, 3, 20000) == 0            # enough sequences
    assert baps.baps_cache_attention_workspace(_cache(page=7), 2, 4, 6, 3, 20000) == 0


def test_fork(lib):
    def call(c=None, tin=A, nin=A, rin=A, B_in=2, par=A, grow=None, B_out=3, width=4, tout=2 * A, nout=2 * A, rout=3 * A, miss=A,
             ws=A, n=1 << 20):
        c = c or _cache()
        return lib.baps_cache_fork(ctypes.byref(c), tin, nin, rin, B_in, par, grow, B_out, width, tout, nout, rout, miss, ws, n, None)
    for kw, status in BAD_CACHES:
        assert call(_cache(**kw)) == status, kw
    for name in ("tin", "nin", "rin", "par", "tout", "nout", "rout", "miss", "ws"):
        assert call(**{name: None}) == BAD, name
    for name in ("B_in", "B_out", "width"):
        assert call(**{name: -1}) == BAD, name
    assert call(n=baps.baps_cache_pages_workspace(0, 3) - 1) == BAD and call(ws=A + 64) == BAD
    # outputs over inputs: tables, lengths; counts that overlap without being the same
    assert call(tout=A) == BAD and call(tout=A + 28) == BAD and call(nout=A + 4) == BAD and call(rout=A + 4) == BAD
    assert call(_cache(layers=70000)) == NOT and call(B_out=1 << 20, width=1 << 12) == NOT and call(width=1 << 27) == NOT


def test_compact(lib):
    def call(c=None, tin=A, entries=8, rin=A, tout=2 * A, rout=3 * A, remap=4 * A, live=A, ws=A, n=1 << 20):
        c = c or _cache()
        return lib.baps_cache_compact(ctypes.byref(c), tin, entries, rin, tout, rout, remap, live, ws, n, None)
    for kw, status in BAD_CACHES:
        assert call(_cache(**kw)) == status, kw
    for name in ("tin", "rin", "tout", "rout", "remap", "live", "ws"):
        assert call(**{name: None}) == BAD, name
    assert call(entries=-1) == BAD and call(n=baps.baps_cache_pages_workspace(8, 0) - 1) == BAD and call(ws=A + 4) == BAD
    assert call(tout=A + 4) == BAD and call(rout=A + 4) == BAD


def test_pages_workspace():
    assert baps.baps_cache_pages_workspace(0, 0) >= 0 and baps.baps_cache_pages_workspace(-1, 0) == 0
    assert baps.baps_cache_pages_workspace(1000, 0) >= 12000 and baps.baps_cache_pages_workspace(0, 1000) >= 20000


def test_tensor_helpers_refuse():
    """The tensor helpers refuse what is no device tensor, or of another shape or type, before any call."""
    import torch
    z = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    with pytest.raises(ValueError):
        baps.PagedCache(z(1, 4, 2, 16, 64), z(1, 4, 2, 1, 64, 16), z(1, 4, 2), z(1, 4, 2))       # not on a device
    with pytest.raises(ValueError):
        baps.PagedCache(z(4, 2, 16, 64), z(4, 2, 1, 64, 16), z(4, 2), z(4, 2))
    q = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        baps.attention_window(q, q, q, 4)
