"""The paged cache's entry points on the host: what they refuse before anything is enqueued, their
workspace sizes, and the rotary frequencies (CPU only: no call here launches a kernel)."""
import ctypes
import math

import pytest
import torch

from paper_2609_23733_amd import vp

FAKE, FAKE_ODD = 0x10000, 0x10002     # device addresses that are never dereferenced


@pytest.fixture(scope="module")
def lib():
    return vp.load_library()


def cache(**kw):
    d = dict(K=FAKE, V=FAKE, weight=FAKE, stamp=FAKE, npages=100, page=64, Hkv=4, d=64, dtype=vp.VP_BF16)
    d.update(kw)
    return vp.vp_cache(*[d[f[0]] for f in vp.vp_cache._fields_])


def batch(**kw):
    d = dict(table=FAKE, length=FAKE, seen=FAKE, q_start=FAKE, B=2, max_pages=10, T=8, max_q=5, max_len=600)
    d.update(kw)
    return vp.vp_cache_batch(*[d[f[0]] for f in vp.vp_cache_batch._fields_])


def spec(**kw):
    d = dict(pos=FAKE, freq=FAKE, dim=64, axes=1, layout=1, mag=1.0)
    d.update(kw)
    return vp.vp_rotary_spec(*[d[f[0]] for f in vp.vp_rotary_spec._fields_])


R = ctypes.byref
BAD_CACHE = [
    (dict(K=None), 1), (dict(V=None), 1), (dict(K=FAKE_ODD), 1), (dict(weight=FAKE_ODD), 1), (dict(dtype=5), 1),
    (dict(npages=0), 1), (dict(Hkv=0), 1), (dict(page=0), 1), (dict(page=48), 2), (dict(page=8), 2),
    (dict(page=8192), 2), (dict(d=128), 2), (dict(Hkv=129), 2), (dict(npages=1 << 31), 2),
]
BAD_BATCH = [
    (dict(table=None), 1), (dict(length=None), 1), (dict(q_start=None), 1), (dict(B=0), 1), (dict(max_pages=0), 1),
    (dict(T=-1), 1), (dict(max_q=-1), 1), (dict(max_q=9), 1), (dict(max_len=-1), 1), (dict(max_len=641), 1),
    (dict(max_pages=1 << 25, max_len=1), 2), (dict(B=30000), 2), (dict(T=(1 << 23) + 1), 2),
    (dict(table=FAKE_ODD), 1), (dict(length=FAKE_ODD), 1),
]


def attend(lib, c, b, Hq=8, Q=FAKE, qs=512, scale=0.0, O=FAKE, lse=FAKE, wo=None, ws=FAKE, n=1 << 30):
    return lib.vp_cache_attend(R(c), R(b), Hq, Q, qs, 1, scale, O, lse, wo, ws, n, None)


def append(lib, c, b, Hq=8, Q=FAKE, qs=512, K=FAKE, ks=256, V=FAKE, vs=256, rot=None, Qo=FAKE):
    return lib.vp_cache_append(R(c), R(b), Hq, Q, qs, K, ks, V, vs, R(rot) if rot is not None else None, Qo, None)


def evict(lib, c, b, keep=10, sink=0, recent=0, wo=FAKE, so=FAKE, lo=FAKE, ws=FAKE, n=1 << 30):
    return lib.vp_cache_evict(R(c), R(b), keep, sink, recent, wo, so, lo, ws, n, None)


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_bad_cache(lib, kw, code):
    c = cache(**kw)
    assert attend(lib, c, batch()) == code
    assert append(lib, c, batch()) == code
    assert evict(lib, c, batch()) == code
    assert lib.vp_cache_attend_workspace_bytes(R(c), R(batch()), 8) == 0


@pytest.mark.parametrize("kw,code", BAD_BATCH)
def test_bad_batch(lib, kw, code):
    b = batch(**kw)
    assert attend(lib, cache(), b) == code
    assert append(lib, cache(), b) == code
    assert lib.vp_cache_attend_workspace_bytes(R(cache()), R(b), 8) == 0
    if not set(kw) & {"q_start", "T", "max_q"}:       # the eviction has no chunk
        assert evict(lib, cache(), b) == code


def test_bad_attend(lib):
    c, b = cache(), batch()
    for kw, code in [(dict(Hq=6), 1), (dict(Hq=0), 1), (dict(Hq=2), 1), (dict(Hq=132), 2), (dict(Q=None), 1),
                     (dict(Q=FAKE_ODD), 1), (dict(qs=504), 1), (dict(qs=516), 1), (dict(scale=-1.0), 1),
                     (dict(scale=math.inf), 1), (dict(scale=math.nan), 1),
                     (dict(scale=2.0 ** -101), 1), (dict(scale=2.0 ** 101), 1), (dict(O=None), 1), (dict(O=FAKE_ODD), 1),
                     (dict(lse=None), 1), (dict(wo=FAKE_ODD), 1), (dict(ws=None), 1), (dict(ws=FAKE + 16), 1),
                     (dict(n=0), 3)]:
        assert attend(lib, c, b, **kw) == code, kw
    assert attend(lib, cache(weight=None), b, wo=FAKE) == 1
    assert attend(lib, c, batch(T=0, max_q=0), Q=None, O=None, lse=None) == 0     # nothing to do
    assert lib.vp_cache_attend(None, R(b), 8, FAKE, 512, 1, 0.0, FAKE, FAKE, None, FAKE, 1 << 30, None) == 1
    assert lib.vp_cache_attend(R(c), None, 8, FAKE, 512, 1, 0.0, FAKE, FAKE, None, FAKE, 1 << 30, None) == 1


def test_bad_append(lib):
    c, b = cache(), batch()
    for kw, code in [(dict(Hq=6), 1), (dict(K=None), 1), (dict(V=None), 1), (dict(K=FAKE_ODD), 1), (dict(ks=248), 1),
                     (dict(vs=260), 1), (dict(qs=100), 1), (dict(Qo=None), 1), (dict(Q=FAKE, Qo=FAKE, qs=520), 1),
                     (dict(rot=spec(dim=-2)), 1), (dict(rot=spec(dim=66)), 2), (dict(rot=spec(dim=3)), 2),
                     (dict(rot=spec(axes=0)), 1), (dict(rot=spec(axes=5)), 2), (dict(rot=spec(dim=34, axes=2)), 2),
                     (dict(rot=spec(layout=2)), 1), (dict(rot=spec(mag=math.inf)), 1), (dict(rot=spec(pos=None)), 1),
                     (dict(rot=spec(freq=None)), 1), (dict(rot=spec(freq=FAKE + 4)), 1)]:
        assert append(lib, c, b, **kw) == code, kw
    assert append(lib, c, batch(seen=None)) == 1          # stamps need the tokens' numbers
    assert append(lib, c, batch(T=0, max_q=0), Q=None, K=None, V=None) == 0


def test_bad_evict(lib):
    c, b = cache(), batch()
    for kw, code in [(dict(keep=0), 1), (dict(sink=-1), 1), (dict(recent=-1), 1), (dict(wo=None), 1), (dict(so=None), 1),
                     (dict(lo=None), 1), (dict(wo=FAKE_ODD), 1), (dict(ws=None), 1), (dict(ws=FAKE + 128), 1), (dict(n=0), 3)]:
        assert evict(lib, c, b, **kw) == code, kw
    assert evict(lib, cache(weight=None), b) == 1
    assert evict(lib, cache(stamp=None), b) == 1
    assert evict(lib, c, batch(seen=None)) == 1


def test_bad_rotary(lib):
    go = lambda r=None, dt=vp.VP_BF16, T=4, H=2, x=FAKE, xs=128, y=FAKE, ys=128: \
        lib.vp_rotary(R(spec() if r is None else r), dt, T, H, x, xs, y, ys, 0, None)
    for kw, code in [(dict(dt=3), 1), (dict(T=-1), 1), (dict(H=0), 1), (dict(H=129), 2), (dict(x=None), 1),
                     (dict(y=None), 1), (dict(xs=64), 1), (dict(ys=132), 1), (dict(xs=136, ys=144), 1),
                     (dict(x=FAKE_ODD), 1), (dict(r=spec(dim=65)), 2), (dict(r=spec(pos=None)), 1)]:
        assert go(**kw) == code, kw
    assert lib.vp_rotary(None, 1, 4, 2, FAKE, 128, FAKE, 128, 0, None) == 1
    assert go(T=0) == 0


def test_workspaces(lib):
    f = lambda **kw: lib.vp_cache_attend_workspace_bytes(R(cache()), R(batch(**kw)), 8)
    assert f() > 0 and f() % 256 == 0
    assert f(T=0, max_q=0) > 0
    g = lib.vp_cache_evict_workspace_bytes
    assert g(0, 4, 100) == 0 and g(1, 0, 100) == 0 and g(1, 4, -1) == 0 and g(40000, 4, 1) == 0
    last = 0
    for n in [0, 1, 4096, 4097, 10000, 137400, 1 << 20]:
        assert g(2, 4, n) >= last and g(2, 4, n) % 256 == 0
        last = g(2, 4, n)


def freqs(lib, dim=64, axes=1, base=10000.0, scaling=0, factor=1.0, original=0.0, low=1.0, high=32.0):
    out = (ctypes.c_uint64 * 32)()
    mag = ctypes.c_float(-1)
    code = lib.vp_rotary_frequencies(dim, axes, base, scaling, factor, original, low, high, out, R(mag))
    return code, list(out), mag.value


@pytest.mark.parametrize("kw", [dict(), dict(dim=48), dict(dim=64, axes=2, base=100.0), dict(scaling=1, factor=8.0),
                                dict(scaling=2, factor=8.0, original=4096.0), dict(dim=2),
                                dict(scaling=2, factor=32.0, original=8192.0, low=2.0, high=16.0)])
def test_frequencies(lib, kw):
    """base^(-2j / section), scaled; a double carries 53 bits of the 64."""
    code, got, mag = freqs(lib, **kw)
    assert code == 0
    dim, axes, base = kw.get("dim", 64), kw.get("axes", 1), kw.get("base", 10000.0)
    n = dim // axes // 2
    for p in range(dim // 2):
        f = base ** (-(p % n) / n)
        if kw.get("scaling") == 1:
            f /= kw["factor"]
        if kw.get("scaling") == 2:
            low, high = kw.get("low", 1.0), kw.get("high", 32.0)
            k = min(1.0, max(0.0, (kw["original"] * f / (2 * math.pi) - low) / (high - low)))
            f *= k + (1 - k) / kw["factor"]
        assert abs(got[p] / 2.0 ** 64 * 2 * math.pi / f - 1) < 1e-13
    assert mag == pytest.approx(0.1 * math.log(kw["factor"]) + 1 if kw.get("scaling") == 2 else 1.0, rel=1e-6)


def test_bad_frequencies(lib):
    for kw, code in [(dict(dim=0), 1), (dict(dim=66), 2), (dict(dim=3), 2), (dict(axes=0), 1), (dict(base=1.0), 1),
                     (dict(base=math.nan), 1), (dict(scaling=3), 1), (dict(scaling=1, factor=0.5), 1),
                     (dict(scaling=2, factor=2.0, original=0.0), 1),
                     (dict(scaling=2, factor=2.0, original=9.0, low=4.0, high=4.0), 1)]:
        assert freqs(lib, **kw)[0] == code, kw


def test_python_checks():
    """The binding refuses what the kernels could not run on, before the library is asked."""
    from paper_2609_23733_amd import cache as c
    cpu = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        c.Rotary(torch.zeros(32, dtype=torch.int64))
    with pytest.raises(ValueError, match="GPU"):
        c.PagedCache(torch.zeros(2, 1, 16, 64), torch.zeros(2, 1, 16, 64))
    with pytest.raises(ValueError, match="GPU"):
        c._rows(cpu, "x", 2, 4, torch.bfloat16)
    with pytest.raises(TypeError):
        c._rows(None, "x", 2, 4, torch.bfloat16)
    with pytest.raises(vp.VPError):
        c.Rotary.make(65, device="cpu")


def test_attend_launches_fit(lib):
    """Bounds that would take 2^24 workgroups or more, 2^32 threads, are refused."""
    f = lambda **kw: lib.vp_cache_attend_workspace_bytes(R(cache(npages=1 << 30, Hkv=4)), R(batch(**kw)), 8)
    big = 1 << 23
    assert f(B=1, T=big, max_q=big, max_pages=1 << 20, max_len=1 << 25) > 0
    assert f(B=16000, T=big, max_q=big, max_pages=1 << 20, max_len=1 << 25) == 0
    assert f(B=1, T=8, max_q=8, max_pages=1 << 24, max_len=1 << 30) == 0
    assert f(B=1, T=8, max_q=8, max_pages=1 << 24, max_len=(1 << 30) - 64) > 0
