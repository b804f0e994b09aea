"""Per-head norms and the 8-bit paged cache on the host: what their entry points refuse before anything is enqueued,
workspace sizes and plans, and the references of the GPU tests against torch (CPU only: no call here launches a kernel)."""
import ctypes
import math

import pytest
import torch

import codes64
from paper_2609_23733_amd import cache, vp
from test_cache_abi import BAD_BATCH, BAD_CACHE, FAKE, FAKE_ODD, R, batch, spec
from test_cache_abi import cache as plain

FAKE2 = 0x20000


@pytest.fixture(scope="module")
def lib():
    return vp.load_library()


def coded(scale=FAKE, rows=vp.VP_BF16, **kw):
    return vp.vp_cache8(plain(**dict(dict(dtype=vp.VP_INT8), **kw)), scale, rows)


def norm(kind=0, gain=FAKE, bias=FAKE, per_head=0, eps=1e-6):
    return vp.vp_head_norm(kind, gain, bias, per_head, eps)


def attend(lib, c, b, Hq=8, Q=FAKE, qs=512, scale=0.0, O=FAKE, lse=FAKE, wo=None, ws=FAKE, n=1 << 30):
    return lib.vp_cache8_attend(R(c), R(b), Hq, Q, qs, 1, scale, O, lse, wo, ws, n, None)


def append(lib, c, b, Hq=8, Q=FAKE, qs=512, K=FAKE, ks=256, V=FAKE, vs=256, qn=None, kn=None, rot=None, Qo=FAKE):
    ref = lambda x: None if x is None else R(x)
    return lib.vp_cache8_append(R(c), R(b), Hq, Q, qs, K, ks, V, vs, ref(qn), ref(kn), ref(rot), Qo, None)


def evict(lib, c, b, keep=10, sink=0, recent=0, wo=FAKE, so=FAKE, lo=FAKE, ws=FAKE, n=1 << 30):
    return lib.vp_cache8_evict(R(c), R(b), keep, sink, recent, wo, so, lo, ws, n, None)


def read(lib, c, b, dtype=vp.VP_BF16, K=FAKE, V=FAKE2):
    return lib.vp_cache8_read(R(c), R(b), dtype, K, V, None)


def every(lib, c, b, code, chunk_only=False):
    assert attend(lib, c, b) == code
    assert append(lib, c, b) == code
    assert read(lib, c, b) == code
    assert lib.vp_cache8_attend_workspace_bytes(R(c), R(b), 8) == 0
    if not chunk_only:
        assert evict(lib, c, b) == code


@pytest.mark.parametrize("kw,code", [x for x in BAD_CACHE if "dtype" not in x[0]])
def test_bad_cache(lib, kw, code):
    every(lib, coded(**kw), batch(), code)


@pytest.mark.parametrize("kw,code", BAD_BATCH)
def test_bad_batch(lib, kw, code):
    every(lib, coded(), batch(**kw), code, chunk_only=bool(set(kw) & {"q_start", "T", "max_q"}))


@pytest.mark.parametrize("c", [
    coded(scale=None), coded(scale=FAKE + 8), coded(rows=vp.VP_INT8), coded(rows=7), coded(dtype=4), coded(dtype=-1),
    coded(dtype=vp.VP_BF16), coded(dtype=vp.VP_F32, scale=None), coded(dtype=vp.VP_BF16, scale=None, rows=vp.VP_F32)])
def test_bad_codes(lib, c):
    """Codes without scales, rows of no row type, plain caches with scales or rows of another type."""
    every(lib, c, batch(), 1)


def test_plain_entry_points_refuse_codes(lib):
    c = plain(dtype=vp.VP_INT8)
    assert lib.vp_cache_attend(R(c), R(batch()), 8, FAKE, 512, 1, 0.0, FAKE, FAKE, None, FAKE, 1 << 30, None) == 1
    assert lib.vp_cache_append(R(c), R(batch()), 8, FAKE, 512, FAKE, 256, FAKE, 256, None, FAKE, None) == 1
    assert lib.vp_cache_evict(R(c), R(batch()), 1, 0, 0, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == 1
    for f in (lib.vp_cache8_attend_plan, lib.vp_cache_attend_plan):
        assert f(None, R(batch()), 8, R(vp.vp_cache_plan())) == 1
    assert lib.vp_cache8_attend_workspace_bytes(None, R(batch()), 8) == 0
    assert lib.vp_cache_attend_workspace_bytes(None, R(batch()), 8) == 0


def test_bad_calls(lib):
    c, b = coded(), batch()
    for kw, code in [(dict(Hq=6), 1), (dict(Hq=132), 2), (dict(Q=None), 1), (dict(qs=504), 1), (dict(qs=516), 1),
                     (dict(scale=-1.0), 1), (dict(scale=math.nan), 1), (dict(scale=2.0 ** -101), 1), (dict(O=FAKE_ODD), 1),
                     (dict(lse=None), 1), (dict(wo=FAKE_ODD), 1), (dict(wo=FAKE), 1), (dict(ws=FAKE + 16), 1), (dict(n=0), 3)]:
        assert attend(lib, c, b, **kw) == code, kw      # (wo: with O the same as Q)
    for kw, code in [(dict(Hq=6), 1), (dict(K=None), 1), (dict(V=FAKE_ODD), 1), (dict(ks=260), 1), (dict(Qo=None), 1),
                     (dict(qs=520), 1), (dict(rot=spec(dim=63)), 2), (dict(rot=spec(pos=None)), 1),
                     (dict(qn=norm(kind=2)), 1), (dict(kn=norm(gain=FAKE + 4)), 1), (dict(kn=norm(bias=FAKE + 8)), 1),
                     (dict(kn=norm(eps=-1.0)), 1), (dict(kn=norm(eps=math.nan)), 1), (dict(kn=norm(eps=math.inf)), 1),
                     (dict(qn=norm(per_head=2)), 1)]:
        assert append(lib, c, b, **kw) == code, kw      # (qs=520: Q_out is Q)
    assert append(lib, c, batch(seen=None)) == 1
    for kw, code in [(dict(dtype=vp.VP_INT8), 1), (dict(K=None), 1), (dict(V=FAKE_ODD), 1), (dict(V=FAKE), 1)]:
        assert read(lib, c, b, **kw) == code, kw
    for kw in (dict(keep=0), dict(sink=-1), dict(wo=None), dict(ws=FAKE + 8)):
        assert evict(lib, c, b, **kw) == 1, kw
    assert evict(lib, c, b, n=0) == 3
    many = batch(B=4000, T=1 << 23, max_q=1 << 23, max_len=640)       # 2^32 threads and more
    assert append(lib, c, many) == 2 and read(lib, c, many) == 2 and attend(lib, c, many) == 2
    # workgroups of 512 threads: 2^23 of them are too many
    wide, plan = coded(Hkv=64, page=4096, npages=1 << 30), vp.vp_cache_plan()
    for B, code in ((500, 0), (600, 2)):
        b2 = batch(B=B, T=72, max_q=72, max_len=69100000, max_pages=17000)
        assert lib.vp_cache8_attend_plan(R(wide), R(b2), 128, R(plan)) == code, B
        assert plan.shared == 1 and plan.ranges == 256 and plan.row_tiles == 1
    empty = batch(T=0, max_q=0)
    assert attend(lib, c, empty) == 0 and append(lib, c, empty) == 0 and read(lib, c, empty) == 0


def test_bad_norms(lib):
    def fwd(n=norm(), rot=spec(), dtype=vp.VP_BF16, T=3, H=4, x=FAKE, xs=256, y=FAKE2, ys=256):
        return lib.vp_norm_rotary(None if n is None else R(n), None if rot is None else R(rot), dtype, T, H, x, xs, y, ys, None)

    def grad(n=norm(), rot=spec(), dtype=vp.VP_BF16, T=3, H=4, x=FAKE, xs=256, g=FAKE, gs=256, dx=FAKE2, dg=FAKE, db=FAKE + 1024,
             ws=FAKE, n_ws=1 << 30):
        return lib.vp_norm_rotary_grad(None if n is None else R(n), R(rot), dtype, T, H, x, xs, g, gs, dx, dg, db, ws, n_ws, None)

    bad = [(dict(n=None), 1), (dict(n=norm(kind=-1)), 1), (dict(n=norm(gain=FAKE + 4)), 1), (dict(rot=spec(axes=5, dim=40)), 2),
           (dict(dtype=vp.VP_E4M3), 1), (dict(T=-1), 1), (dict(H=0), 1), (dict(H=129), 2), (dict(x=None), 1),
           (dict(x=FAKE_ODD), 1), (dict(xs=252), 1), (dict(xs=260), 1)]
    for kw, code in bad:
        assert fwd(**kw) == code, kw
        assert grad(**kw) == code, kw
    for kw in (dict(y=None), dict(ys=128), dict(y=FAKE, ys=512)):
        assert fwd(**kw) == 1, kw
    for kw, code in [(dict(g=None), 1), (dict(gs=255), 1), (dict(dx=FAKE), 1), (dict(dx=FAKE_ODD), 1), (dict(dg=FAKE_ODD), 1),
                     (dict(db=FAKE_ODD), 1), (dict(db=FAKE), 1), (dict(ws=None), 1), (dict(ws=FAKE + 8), 1), (dict(n_ws=0), 3)]:
        assert grad(**kw) == code, kw
    assert fwd(T=0) == 0 and grad(dx=None, dg=None, db=None, ws=None, n_ws=0) == 0
    size = lib.vp_norm_rotary_grad_workspace_bytes
    assert size(-1, 4, 0) == size(4, 0, 0) == size(4, 129, 0) == size(4, 4, 2) == 0
    assert size(0, 4, 0) > 0 and size(43968, 16, 1) >= size(1374, 16, 1) > size(1374, 16, 0) > 0


def test_plan(lib):
    """Few rows: 16 or 32 a workgroup; the workspace holds the parts and, for the weights, kept logits."""
    for G, q, rows in [(1, 1, 16), (4, 4, 16), (16, 1, 16), (17, 1, 32), (1, 17, 32)]:
        c, b = coded(Hkv=4), batch(B=1, T=q, max_q=q)
        plan = vp.vp_cache_plan()
        assert lib.vp_cache8_attend_plan(R(c), R(b), 4 * G, R(plan)) == 0
        assert (plan.shared, plan.rows) == (0, rows), (G, q)
        assert plan.ranges * plan.range_slots >= b.max_len and plan.range_slots % 64 == 0
        assert lib.vp_cache8_attend_workspace_bytes(R(c), R(b), 4 * G) >= plan.ranges * q * 4 * G * 66 * 4 * (plan.ranges > 1)


def test_python_refusals():
    t = torch.zeros(64)
    with pytest.raises(ValueError, match="GPU"):
        cache.HeadNorm("layer", t)
    with pytest.raises(KeyError):
        cache.HeadNorm("batch")
    for eps in (0.0, -1.0, float("nan"), float("inf"), 1e-50, 1e39):
        with pytest.raises(ValueError, match="eps"):
            cache.HeadNorm("rms", eps=eps)
    n = cache.HeadNorm("rms")
    with pytest.raises(ValueError, match="GPU"):
        cache.norm_rotary(torch.zeros(2, 3, 64), n)
    with pytest.raises(ValueError, match="positions"):
        cache.norm_rotary(torch.zeros(2, 3, 64), n, pos=torch.zeros(2, 1, dtype=torch.int32))


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_reference_codes(kind):
    """The reference quantiser: its codes decode to what torch's own types hold, scales at the borders."""
    top = codes64.LARGEST[kind]
    x = torch.randn(400, 64, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
    x *= torch.exp2(torch.arange(400)[:, None].double() - 200).clamp(1e-28, 1e28)
    x[:3, 0] = torch.tensor([top, top * (1 + 1e-12), -top], dtype=torch.float64)
    x[:3, 1:] = torch.rand(3, 63).double() * 2
    code, s, v = codes64.quantise64(x, kind)
    assert s[:3].tolist() == [1.0, 2.0, 1.0]
    own = code.view(codes64.CODES[kind]).double() * s[:, None]
    assert torch.equal(own, v)
    assert ((v - x).abs() <= codes64.step64(x / s[:, None], kind) * s[:, None] / 2).all()
    if kind == "e4m3":
        again = (x / s[:, None]).to(torch.float8_e4m3fn).double() * s[:, None]
        near = (x / s[:, None]).float().double() == x / s[:, None]       # (torch rounds through fp32)
        assert torch.equal(again[near], v[near])
    big = torch.tensor([[f * 2.0 ** 127] + [1e38] * 63 for f in (1.0, 1.74, 1.76, 1.98, 1.99, 1.9999999)], dtype=torch.float64)
    v = codes64.quantise64(big, kind)[2]
    # (below 2^128 at most a step: 16 times 2^120, or 2^122)
    assert (v.abs() < 2.0 ** 128).all() and ((v - big).abs() <= 2.0 ** (124 if kind == "e4m3" else 122)).all()
    code, s, v = codes64.quantise64(torch.tensor([[0.0] * 64, [math.inf] + [1.0] * 63, [math.nan] * 64]), kind)
    assert s[0] == 2.0 ** -100 and (v[0] == 0).all() and torch.isnan(s[1:]).all() and torch.isnan(v[1:]).all()
