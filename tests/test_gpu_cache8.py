"""The paged cache of 8-bit codes on the GPU against 64-bit computations: append (norms, rotation, codes), reading
back, attention with its weights, eviction, and the stream layer that runs them.

Tolerances (set before the first run).  Codes are exact: V's have to be those of the definition; K's, quantised from the
normalised and turned row that the kernel has in fp64, lie within half a step of the scale in use (plus the t that
test_gpu_head_norm.py has for fp32) and are the definition's where that is no near tie; scales likewise.  Attention: those of
test_gpu_cache.py over the values that the codes stand for, as code times scale is exact; the kernel's two products by
scales add two roundings, within the 16 u of E."""
import math

import numpy as np
import pytest
import torch

import codes64
from paper_2609_23733_amd import vp
from test_gpu_cache import BF, F32, U, Pool, _gpu, cache, gen, i32, log, normal, radians, rot_tol, rotate64  # noqa: F401
from test_gpu_cache import bf16_tol
from test_gpu_cache_wide import check, whole64
from test_gpu_head_norm import forward64, tolerances

pytestmark = pytest.mark.gpu
KINDS = ["int8", "e4m3"]


class Pool8(Pool):
    """A pool of codes; `k`, `v`: the values that the sequences' codes stand for.  Everything else in it: codes and scales
    of NaN (int8: -128), or random bits."""

    def __init__(self, cache, lens, Hkv, page, kind, seed, rows=BF, spare=3, cap=0, std=1.0, vstd=1.0, junk="nan"):  # noqa: F811
        self.kind, self.code, self.junk = kind, codes64.CODES[kind], junk
        Pool.__init__(self, cache, lens, Hkv, page, rows, seed, spare, 0.0, cap, std, vstd)

    def put(self, b, k, v):
        if b == 0 and not self.k:
            shape = tuple(self.K.shape)
            byte = 127 if self.kind == "e4m3" else 128
            if self.junk == "nan":
                self.K, self.V = (torch.full(shape, byte, dtype=torch.uint8) for _ in range(2))
                self.scale = torch.full(shape[:3] + (2,), math.nan, dtype=BF)
            else:
                self.K, self.V = (torch.randint(0, 256, shape, generator=gen(77 + j)).to(torch.uint8) for j in range(2))
                self.scale = torch.randint(-32768, 32768, shape[:3] + (2,), generator=gen(79)).to(torch.int16).view(BF)
        p, s = self.at(b, k.shape[0])
        kc, ks, kv = codes64.quantise64(k.double(), self.kind)
        vc, vs, vv = codes64.quantise64(v.double(), self.kind)
        self.put_codes(b, p, s, kc, ks, kv, vc, vs, vv)

    def put_codes(self, b, p, s, kc, ks, kv, vc, vs, vv):
        self.K[p, :, s], self.V[p, :, s] = kc, vc
        self.scale[p, :, s] = torch.stack([ks, vs], dim=2).to(BF)
        for have, new in ((self.k, kv), (self.v, vv)):
            if len(have) <= b:
                have.append(new)
            else:
                have[b] = new

    def cuda(self):
        g = lambda t: t.cuda()
        self.gK, self.gV = g(self.K).view(self.code), g(self.V).view(self.code)
        self.gW, self.gS, self.gscale = g(self.W), g(self.S), g(self.scale)
        self.gtable = torch.from_numpy(self.table).cuda()
        return self.c.PagedCache(self.gK, self.gV, self.gW, self.gS, scale=self.gscale, rows=self.dtype)


# ------------------------------------------------------------------ append and read

APPEND = [
    # lens, chunks, Hq, Hkv, page, kind, rows, norm, gain, dim, axes, layout, fused
    ([1], [1], 1, 1, 16, "int8", BF, "layer", "shared", 64, 1, "half", False),
    ([40, 3, 700], [40, 2, 0], 4, 2, 16, "e4m3", F32, "rms", "heads", 48, 1, "interleaved", True),
    ([130, 257, 64], [64, 3, 64], 16, 4, 32, "int8", BF, "layer", "heads", 64, 2, "half", True),
    ([900], [300], 6, 2, 64, "e4m3", BF, None, "none", 60, 2, "half", False),
    ([77, 12], [77, 1], 3, 1, 16, "int8", F32, "rms", "none", 10, 1, "interleaved", False),
    ([3000], [1374], 16, 16, 64, "e4m3", BF, "layer", "shared", 64, 2, "half", False),
    ([50, 9], [33, 9], 2, 2, 128, "int8", F32, "layer", "shared", 0, 1, "half", True),
    ([2] * 40, [1] * 40, 128, 128, 16, "e4m3", BF, "rms", "shared", 32, 1, "half", True),
]


def gains(norm, gain, H, seed):
    if gain == "none":
        return None, None
    shape = (H, 64) if gain == "heads" else (64,)
    ga = 1 + 0.3 * torch.randn(*shape, generator=gen(seed))
    return ga, (0.3 * torch.randn(*shape, generator=gen(seed + 1)) if norm == "layer" else None)


@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,kind,rows,norm,gain,dim,axes,layout,fused", APPEND)
def test_append_and_read(cache, lens, qs, Hq, Hkv, page, kind, rows, norm, gain, dim, axes, layout, fused):  # noqa: F811
    log("append8 %s %s Hq=%d Hkv=%d page=%d %s %s %s" % (lens, qs, Hq, Hkv, page, kind, rows, norm))
    pool = Pool8(cache, lens, Hkv, page, kind, seed=5 + sum(lens), rows=rows)
    before = [t.clone() for t in (pool.K, pool.V, pool.scale, pool.W, pool.S)]
    T = sum(qs)
    x = torch.randn(T, Hq + 2 * Hkv, 64, generator=gen(T + Hq)) * torch.exp(0.5 * torch.randn(T, Hq + 2 * Hkv, 1, generator=gen(2)))
    x = x.to(rows)
    Q, K, V = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    pos = torch.randint(-9999, 9999, (T, axes), generator=gen(4)).to(torch.int32)
    rot = cache.Rotary.make(dim, 10000.0, axes, layout) if dim else None
    dev = lambda t: None if t is None else t.cuda()
    mk = lambda ga, bi: cache.HeadNorm(norm, dev(ga), dev(bi)) if norm else None
    (qga, qbi), (kga, kbi) = gains(norm, gain, Hq, 50), gains(norm, gain, Hkv, 60)
    pc, batch = pool.cuda(), pool.batch(qs, seen=[n + 11 for n in lens])
    gx = x.cuda()
    parts = (gx[:, :Hq], gx[:, Hq:Hq + Hkv], gx[:, Hq + Hkv:]) if fused else (Q.cuda(), K.cuda(), V.cuda())
    got = cache.append(pc, batch, *parts, dev(pos) if rot else None, rot, q_norm=mk(qga, qbi), k_norm=mk(kga, kbi))

    def turned(t, ga, bi):
        if norm:
            y, n, r, S = forward64(t, ga, bi, pos, rot, norm)
            return y, tolerances(y, n, r, S, ga, bi, 1.0, F32)
        one = torch.ones(t.shape[0], t.shape[1], 1, dtype=torch.float64)
        y = t.double() if rot is None else rotate64(t, pos, radians(rot), axes, layout, 1.0)
        return y, 24 * U * t.double().abs().amax(dim=2, keepdim=True) * one + 1e-30

    yq, tq = turned(Q, qga, qbi)
    tq = tq + (2.0 ** -8 * (yq.abs() + tq) if rows == BF else 0)
    assert ((got.cpu().double() - yq).abs() <= tq).all()
    yk, tk = turned(K, kga, kbi)
    vc, vs, vv = codes64.quantise64(V.double(), kind)
    hK, hV, hS = pool.gK.cpu().view(torch.uint8), pool.gV.cpu().view(torch.uint8), pool.gscale.cpu()
    hW, hStamp = pool.gW.cpu(), pool.gS.cpu()
    t = 0
    for b, m in enumerate(qs):
        n = lens[b]
        p, s = (v[n - m:] for v in pool.at(b, n))
        assert torch.equal(hV[p, :, s], vc[t:t + m]), b
        assert torch.equal(hS[p, :, s, 1].double(), vs[t:t + m]), b
        ks, y, ty = hS[p, :, s, 0].double(), yk[t:t + m], tk[t:t + m]
        big = y.abs().amax(dim=2)
        far = ty.expand(y.shape).amax(dim=2)
        assert ((ks == codes64.scale64(big - far, kind)) | (ks == codes64.scale64(big + far, kind))).all(), b
        held = codes64.decode64(hK[p, :, s], ks, kind)
        step = codes64.step64((y.abs() + ty) / ks[..., None], kind) * ks[..., None]
        assert ((held - y).abs() <= step / 2 + ty).all(), b
        # the definition's code, but within 1e-6 of a step of a border (fp64 rows are off by less than 1e-9)
        _, s64, want = codes64.quantise64(y, kind)
        top = big / (codes64.LARGEST[kind] * s64)
        assert (ks == s64)[(top < 1 - 1e-9) & (top > 0.5 + 1e-9)].all(), b
        place = y.abs() / (codes64.step64(y / s64[..., None], kind) * s64[..., None])
        clear = ((place - place.floor() - 0.5).abs() > 1e-6) & (ks == s64)[..., None]
        assert torch.equal(held[clear], want[clear]) and (m == 0 or clear.double().mean() > 0.99), b
        assert (hW[p, :, s] == 0).all()
        assert torch.equal(hStamp[p, :, s], (n + 11 - m + torch.arange(m, dtype=torch.int32))[:, None].expand(m, Hkv))
        before[0][p, :, s], before[1][p, :, s], before[2][p, :, s] = hK[p, :, s], hV[p, :, s], hS[p, :, s]
        before[3][p, :, s], before[4][p, :, s] = hW[p, :, s], hStamp[p, :, s]
        t += m
    bits = lambda v: v.view(torch.int16) if v.dtype == BF else v
    assert all(torch.equal(bits(a), bits(c)) for a, c in zip(before, (hK, hV, hS, hW, hStamp)))   # no other slot
    # what was appended, read back; all there is, and rows past the last sequence's left alone
    for dtype in (BF, F32):
        k, v = cache.read(pc, batch, T, dtype)
        rk = [codes64.decode64(hK[p, :, s], hS[p, :, s, 0], kind) for p, s in (pool.at(b, n) for b, n in enumerate(lens))]
        assert torch.equal(k.cpu().double(), torch.cat([r[n - m:] for r, n, m in zip(rk, lens, qs)]))
        assert torch.equal(v.cpu().double(), vv)
    every = pool.batch(lens)
    R = sum(lens)
    ko, vo = (torch.full((R + 2, Hkv, 64), 7.0, dtype=F32, device="cuda") for _ in range(2))
    cache.read(pc, every, R + 2, K_out=ko, V_out=vo)
    assert torch.equal(ko[:R].cpu().double(), torch.cat(rk)) and (ko[R:] == 7).all() and (vo[R:] == 7).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_plain_caches_with_norms(cache, dtype):  # noqa: F811
    """Norms in the append of a bf16 or fp32 cache are norm_rotary's, to the bit; read returns what is held."""
    log("append norms, plain %s" % dtype)
    pool = Pool(cache, [70, 9], 2, 16, dtype, seed=1)
    pc, batch = pool.cuda(), pool.batch([33, 9], seen=[70, 9])
    Q, K, V = (normal(i, (42, h, 64), dtype).cuda() for i, h in ((1, 4), (2, 2), (3, 2)))
    pos = torch.arange(42, dtype=torch.int32, device="cuda")[:, None]
    rot = cache.Rotary.make(48)
    qn = cache.HeadNorm("rms", 1 + normal(5, (4, 64), F32).cuda())
    kn = cache.HeadNorm("layer", 1 + normal(6, (64,), F32).cuda(), normal(7, (64,), F32).cuda())
    q = cache.append(pc, batch, Q, K, V, pos, rot, q_norm=qn, k_norm=kn)
    k, v = cache.read(pc, batch, 42)
    assert torch.equal(q, cache.norm_rotary(Q, qn, pos, rot))
    assert torch.equal(k, cache.norm_rotary(K, kn, pos, rot)) and torch.equal(v, V)
    only_k = cache.append(pc, batch, Q, K, V, pos, rot, k_norm=kn)
    # (without a norm: the rotation of cache.rotary, whose compiler fuses one product of each pair's two of its own choice;
    # both lie within rot_tol of the exact one, so within twice that of each other)
    ref = cache.rotary(Q, pos, rot).cpu().double()
    assert ((only_k.cpu().double() - ref).abs() <= 2 * rot_tol(Q.cpu(), ref, 1.0, dtype)).all()
    assert cache.append(pc, batch, None, K, V, pos, rot, k_norm=kn) is None
    for other in (F32, BF):
        assert torch.equal(cache.read(pc, batch, 42, other)[0], k.to(other))
    same = Q.clone()
    assert torch.equal(cache.append(pc, batch, same, K, V, pos, rot, Q_out=same, q_norm=qn, k_norm=kn), q)


@pytest.mark.parametrize("kind", KINDS)
def test_rows_at_the_ends(cache, kind):  # noqa: F811
    """Rows of zeros, of tiny, huge and uneven values, and with NaN or infinities, as V: codes of the definition."""
    log("append8 extremes %s" % kind)
    pool = Pool8(cache, [64], 1, 16, kind, seed=2, rows=F32)
    pc, batch = pool.cuda(), pool.batch([64], seen=[64])
    V = normal(3, (64, 1, 64), F32)
    V *= torch.exp2(torch.linspace(-140, 126, 64))[:, None, None]
    V[0] = 0.0
    V[1, 0, 5], V[2, 0, 6], V[3, 0, 7] = math.nan, math.inf, -math.inf
    V[5] = 0.0
    V[5, 0, 63] = -3e38
    top = codes64.LARGEST[kind]
    V[7, 0] = torch.linspace(-top, top, 64)
    V[8, 0] = torch.nextafter(V[7, 0], torch.tensor(math.inf))
    V[9, 0, :] = torch.arange(64) / 2 + 0.5         # ties
    V[9, 0, 0] = top
    V[10:14] = torch.tensor([1.74, 1.76, 1.98, 1.99])[:, None, None] * 2.0 ** 127 * torch.linspace(-1, 1, 64)
    V[14] = torch.finfo(F32).max
    V[15] = torch.finfo(BF).max
    cache.append(pc, batch, None, torch.zeros(64, 1, 64, device="cuda"), V.cuda())
    code, s, v = codes64.quantise64(V.double(), kind)
    p, at = pool.at(0, 64)
    assert torch.equal(pool.gV.cpu().view(torch.uint8)[p, :, at], code)
    hs = pool.gscale.cpu()[p, :, at].double()
    assert torch.equal(torch.nan_to_num(hs[..., 1], nan=-1.0), torch.nan_to_num(s, nan=-1.0))
    assert (hs[..., 0] == 2.0 ** -100).all()
    got = cache.read(pc, batch, 64)[1].cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(v)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(v))


def test_read_of_missing_slots(cache):  # noqa: F811
    """More rows than slots, and pages that do not exist: zeros."""
    log("read8 missing")
    pool = Pool8(cache, [40, 0, 90], 2, 16, "e4m3", seed=6)
    pc, batch = pool.cuda(), pool.batch([50, 5, 90])
    pool.gtable[2, 1], pool.gtable[2, 3] = -1, 1 << 30
    k, v = (t.cpu().double() for t in cache.read(pc, batch, 145))
    for x, have in ((k, pool.k), (v, pool.v)):
        want = torch.zeros(145, 2, 64, dtype=torch.float64)
        want[10:50], want[55:] = have[0], have[2]
        want[55 + 16:55 + 32] = want[55 + 48:55 + 64] = 0.0
        assert torch.equal(x, want)


# ------------------------------------------------------------------ attention

ATTEND = [
    # lens, chunks, Hq, Hkv, page, kind, rows, causal
    ([1], [1], 1, 1, 16, "e4m3", BF, True), ([1], [1], 16, 16, 64, "int8", F32, False),
    ([31], [1], 4, 4, 16, "int8", BF, True), ([33, 64, 65], [1, 1, 1], 16, 4, 16, "e4m3", BF, True),
    ([300], [1], 16, 16, 64, "e4m3", BF, True), ([1374, 5, 700, 0], [1, 1, 0, 0], 16, 8, 32, "int8", BF, True),
    ([2500, 1], [1, 1], 6, 2, 128, "e4m3", F32, True), ([5000], [1], 16, 1, 256, "int8", BF, True),
    ([40], [40], 2, 1, 16, "int8", BF, True), ([40], [40], 2, 1, 16, "e4m3", F32, True),
    ([130, 257, 64], [64, 3, 64], 4, 4, 16, "e4m3", BF, True), ([130, 257, 64], [64, 3, 64], 4, 4, 16, "int8", F32, True),
    ([640], [257], 3, 1, 64, "int8", BF, True), ([640], [257], 3, 1, 64, "e4m3", F32, True),
    ([1000], [300], 2, 2, 4096, "e4m3", BF, False), ([777, 100], [130, 90], 12, 4, 32, "int8", F32, False),
    ([4100], [70], 2, 2, 32, "int8", BF, False), ([9000], [2], 2, 2, 64, "e4m3", BF, True),
    ([2050], [66], 4, 1, 1024, "int8", F32, True), ([6000], [9], 4, 2, 32, "int8", BF, True),
    ([30000, 17], [1, 1], 4, 1, 16, "e4m3", BF, True), ([100], [1], 128, 1, 16, "int8", BF, True),
    ([200, 350], [1, 7], 34, 2, 16, "e4m3", BF, False),
]


@pytest.mark.parametrize("junk", ["nan", "bits"])
@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,kind,rows,causal", ATTEND)
def test_attend(cache, lens, qs, Hq, Hkv, page, kind, rows, causal, junk):  # noqa: F811
    log("attend8 %s %s Hq=%d Hkv=%d page=%d %s %s causal=%d %s" % (lens, qs, Hq, Hkv, page, kind, rows, causal, junk))
    pool = Pool8(cache, lens, Hkv, page, kind, seed=100 + sum(lens), rows=rows, junk=junk)
    check(cache, pool, normal(7, (sum(qs), Hq, 64), rows), qs, causal, 0)


@pytest.mark.parametrize("rows", [BF, F32])
@pytest.mark.parametrize("q", [3, 200])
def test_attend_rows_that_see_nothing(cache, rows, q):  # noqa: F811
    log("attend8 empty rows q=%d %s" % (q, rows))
    pool = Pool8(cache, [2, 0, 150], 2, 16, "int8", seed=31, rows=rows)
    O, lse = check(cache, pool, normal(8, (3 * q, 4, 64), rows), [q, q, q], True, 0)
    assert (O[:q - 2] == 0).all() and torch.isneginf(lse[:q - 2]).all()


def odd_scales(pool, n):
    """Slots whose scale is NaN: a value's at n - 9 (head 0) and n - 40 (1), a key's at n - 5 (0)."""
    p, s = pool.at(0, n)
    for at, h, j in ((n - 9, 0, 1), (n - 40, 1, 1), (n - 5, 0, 0)):
        pool.scale[p[at], h, s[at], j] = math.nan
        (pool.v if j else pool.k)[0][at, h] = math.nan


@pytest.mark.parametrize("rows", [BF, F32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq", [2, 6])
def test_attend_scales_of_nan(cache, rows, kind, Hq):  # noqa: F811
    """They reach the rows that see their slots, and no others."""
    log("attend8 NaN scales %s %s" % (kind, rows))
    n, q = 150, 140
    pool = Pool8(cache, [n], 2, 32, kind, seed=33, rows=rows)
    odd_scales(pool, n)
    check(cache, pool, normal(9, (q, Hq, 64), rows), [q], True, 0)


def test_attend_codes_of_nan(cache):  # noqa: F811
    """An e4m3 NaN among a slot's values: rows that see it get NaN at least in its feature; rows that do not are
    right.  (Not to the bit those of a cache without it: a wave's rows move their references together.)"""
    log("attend8 NaN codes")
    n, q = 150, 140
    for rows in (BF, F32):
        pool = Pool8(cache, [n], 1, 32, "e4m3", seed=33, rows=rows)
        Q = normal(9, (q, 3, 64), rows)
        p, s = pool.at(0, n)
        pool.K[p[n - 3], 0, s[n - 3], 9] = 255
        pool.V[p[n - 9], 0, s[n - 9], 5], pool.V[p[n - 40], 0, s[n - 40], 33] = 127, 255
        pc, batch = pool.cuda(), pool.batch([q])
        O, lse = (t.cpu().double() for t in cache.attend(pc, batch, Q.cuda(), True))
        see = n - q + torch.arange(q) + 1
        assert torch.isnan(O[see > n - 40][:, :, 33]).all() and torch.isnan(O[see > n - 9][:, :, 5]).all()
        assert torch.isnan(lse[see > n - 3]).all()
        sees = torch.arange(n) < see[:, None]
        for h in range(3):
            ro, rl, _, A, X = whole64(Q[:, h], pool.k[0][:, 0], pool.v[0][:, 0], sees, 0.125)
            E = (64 * X + n / 16 + 16 + rl.abs()) * U
            tol = torch.from_numpy(bf16_tol((2 * E[:, None] * A).numpy(), A.numpy(), ro.numpy(), rows == BF))
            few, some = see <= n - 40, see <= n - 3
            assert ((O[:, h] - ro).abs() <= tol)[few].all()
            assert ((lse[:, h] - rl).abs() <= 2 * E)[some].all()


@pytest.mark.parametrize("rows", [BF, F32])
@pytest.mark.parametrize("q", [1, 90])
def test_attend_pages_that_do_not_exist(cache, rows, q):  # noqa: F811
    log("attend8 bad pages %s q=%d" % (rows, q))
    n = 700
    pool = Pool8(cache, [n], 1, 16, "int8", seed=35, rows=rows)
    gone = [s for p in (2, 17, 42) for s in range(16 * p, 16 * p + 16)]
    pc = pool.cuda()
    Q = normal(13, (q, 2, 64), rows).cuda()
    W = pool.W.cuda()
    batch = pool.batch([q])
    for i, p in enumerate((2, 17, 42)):
        pool.gtable[0, p] = [-1, pool.npages, 2 ** 31 - 1][i]
    O, lse = cache.attend(pc, batch, Q, True, weight_out=W)
    keep = np.array([i for i in range(n) if i not in set(gone)])
    sees = torch.from_numpy(keep[None, :] <= (n - q + np.arange(q))[:, None])
    for h in range(2):
        ro, rl, rp, A, X = whole64(Q[:, h].cpu(), pool.k[0][keep, 0], pool.v[0][keep, 0], sees, 0.125)
        E = (64 * X + n / 16 + 16 + rl.abs()) * U
        tol = bf16_tol((2 * E[:, None] * A).numpy(), A.numpy(), ro.numpy(), rows == BF)
        assert ((O[:, h].cpu().double() - ro).abs().numpy() <= tol).all()
        assert ((lse[:, h].cpu().double() - rl).abs() <= 2 * E).all()


@pytest.mark.parametrize("rows", [BF, F32])
@pytest.mark.parametrize("kind", KINDS)
def test_attend_large_logits(cache, rows, kind):  # noqa: F811
    """Logits of some hundreds, the largest late in the sequence, so that the reference has to move; other scales."""
    log("attend8 large logits %s %s" % (kind, rows))
    pool = Pool8(cache, [900], 2, 64, kind, seed=36, rows=rows, std=6.0)
    k = pool.k[0].clone()
    k[800:] *= 4
    pool.put(0, k, pool.v[0])
    check(cache, pool, normal(14, (70, 4, 64), rows, 6.0), [70], False, 0)
    check(cache, pool, normal(15, (1, 4, 64), rows, 6.0), [1], True, 0, scale=0.5)


@pytest.mark.parametrize("rows", [BF, F32])
@pytest.mark.parametrize("vstd", [1e-20, 2e37])
def test_attend_values_of_any_size(cache, rows, vstd):  # noqa: F811
    """Values near the largest (their sums leave fp32's range before the division) and tiny ones."""
    log("attend8 values %g %s" % (vstd, rows))
    pool = Pool8(cache, [700], 1, 16, "int8", seed=37, rows=rows, vstd=1.0)
    pool.put(0, pool.k[0], torch.clamp(pool.v[0], -4, 4) * vstd)
    pool.k[0][650:] *= 1.0
    check(cache, pool, normal(16, (1, 2, 64), rows, 3.0), [1], True, 0)
    check(cache, pool, normal(17, (20, 2, 64), rows, 3.0), [20], True, 0)


WIDE = [
    # lens, chunks, Hq, Hkv, page, kind, causal
    ([1374], [1374], 16, 16, 64, "e4m3", True), ([3000, 2000, 700, 50], [1100, 900, 300, 0], 8, 4, 32, "int8", True),
    ([3300, 90, 2000], [1500, 77, 900], 12, 4, 16, "e4m3", True), ([10000, 300], [260, 17], 16, 4, 64, "int8", False),
    ([2500], [2000], 64, 16, 16, "int8", True), ([2400, 1300], [1300, 1300], 16, 8, 16, "e4m3", True),
    ([9001], [500], 16, 2, 128, "e4m3", False),
]


@pytest.mark.parametrize("junk", ["nan", "bits"])
@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,kind,causal", WIDE)
def test_attend_wide(cache, lens, qs, Hq, Hkv, page, kind, causal, junk):  # noqa: F811
    log("attend8 wide %s %s Hq=%d Hkv=%d page=%d %s causal=%d %s" % (lens, qs, Hq, Hkv, page, kind, causal, junk))
    pool = Pool8(cache, lens, Hkv, page, kind, seed=100 + sum(lens), junk=junk)
    check(cache, pool, normal(7, (sum(qs), Hq, 64), BF), qs, causal, 1)


@pytest.mark.parametrize("kind", KINDS)
def test_attend_wide_odd(cache, kind):  # noqa: F811
    """Whole-view calls with what is rare: scales of NaN in the chunk, missing pages, logits that rise late, values near
    the largest."""
    log("attend8 wide, odd contents %s" % kind)
    n, q = 4000, 1500
    Q = normal(9, (q, 16, 64), BF)
    pool = Pool8(cache, [n], 2, 32, kind, seed=33)
    odd_scales(pool, n)
    check(cache, pool, Q, [q], True, 1)
    pool = Pool8(cache, [n], 2, 32, kind, seed=34)
    check(cache, pool, Q, [q], True, 1, gone=[s for p in (0, 3, 70, 124) for s in range(32 * p, 32 * p + 32) if s < n])
    pool = Pool8(cache, [n], 2, 32, kind, seed=35, std=3.0)
    k = pool.k[0].clone()
    k[2500:] *= 8
    pool.put(0, k, pool.v[0])
    check(cache, pool, normal(10, (q, 16, 64), BF, 3.0), [q], False, 1)
    pool = Pool8(cache, [n], 2, 32, kind, seed=36)
    pool.put(0, pool.k[0], torch.clamp(pool.v[0], -4, 4) * 2e37)
    check(cache, pool, Q, [q], True, 1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("q", [513, 545, 640, 641])
def test_attend_wide_few_rows(cache, kind, q):  # noqa: F811
    """A last tile of 1, 33, 128 and 129 rows; sequences that are no more than that; what is rare in such tiles."""
    log("attend8 wide, few rows %s q=%d" % (kind, q))
    n, lens, qs = 7000, [7000, 300, 64, 1], [q, q - 512, 1, 0]
    pool = Pool8(cache, lens, 8, 32, kind, seed=41, junk="bits")
    check(cache, pool, normal(9, (sum(qs), 8, 64), BF), qs, True, 1)
    Q = normal(10, (q, 8, 64), BF)
    pool = Pool8(cache, [n], 8, 32, kind, seed=42)
    odd_scales(pool, n)
    check(cache, pool, Q, [q], True, 1)
    pool = Pool8(cache, [n], 8, 32, kind, seed=43)
    check(cache, pool, Q, [q], False, 1, gone=[s for p in (0, 3, 70, 124) for s in range(32 * p, 32 * p + 32) if s < n])
    pool = Pool8(cache, [n], 8, 32, kind, seed=44, std=3.0)
    k = pool.k[0].clone()
    k[2500:] *= 8
    pool.put(0, k, torch.clamp(pool.v[0], -4, 4) * 2e37)
    Q = normal(11, (q, 8, 64), BF, 3.0).cuda()
    pc, batch = pool.cuda(), pool.batch([q])
    assert cache.attend_plan(pc, batch, 8, q).shared == 1
    O, lse = cache.attend(pc, batch, Q, True)
    # The tolerance of test_gpu_cache.py and what underflow takes: a power below 2^-126 counts as 0 in the products, and the
    # powers' sum is 1 at least (the reference is one of the row's logits, and grows with them), so each of n slots loses at
    # most 2^-126 of the largest |v|, below 2^126 here: n, where most results are of the size of 1e37.
    sees = torch.arange(n, device="cuda") < (n - q + torch.arange(q, device="cuda") + 1)[:, None]
    for h in range(8):
        v = pool.v[0][:, h].cuda()
        ro, rl, _, A, X = whole64(Q[:, h], pool.k[0][:, h].cuda(), v, sees, 0.125)
        E = (64 * X + n / 16 + 16 + rl.abs()) * U
        tol = (2 * E[:, None] * A + n * 2.0 ** -126 * v.abs().max()).cpu().numpy()
        tol = torch.from_numpy(bf16_tol(tol, A.cpu().numpy(), ro.cpu().numpy())).cuda()
        assert ((O[:, h].double() - ro).abs() <= tol).all(), h
        assert ((lse[:, h].double() - rl).abs() <= 2 * E + 2 * U * rl.abs()).all(), h


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("q", [5, 1500])
def test_attend_scales_of_other_origin(cache, kind, q):  # noqa: F811
    """Scales that are no powers of two: within another bf16 rounding of every value (2^-8) and key (2^-8 of a
    logit's absolute sum X) where rows are many."""
    log("attend8 other scales %s q=%d" % (kind, q))
    n = 9000
    pool = Pool8(cache, [n], 2, 64, kind, seed=38)
    p, s = pool.at(0, n)
    for j, have in ((0, pool.k), (1, pool.v)):
        f = (1 + torch.rand(n, 2, generator=gen(40 + j))).to(BF)
        code = (pool.K if j == 0 else pool.V)[p, :, s]
        sc = (pool.scale[p, :, s, j].float() * f.float()).to(BF)
        pool.scale[p, :, s, j] = sc
        have[0] = codes64.decode64(code, sc.double(), kind)
    Q = normal(9, (q, 4, 64), BF)
    pc, batch = pool.cuda(), pool.batch([q])
    assert cache.attend_plan(pc, batch, 4, q).shared == (q > 64)
    O, lse = cache.attend(pc, batch, Q.cuda(), False)
    for h in range(4):
        one = torch.ones(q, n, dtype=torch.bool, device="cuda")
        ro, rl, _, A, X = whole64(Q[:, h].cuda(), pool.k[0][:, h // 2].cuda(), pool.v[0][:, h // 2].cuda(), one, 0.125)
        shift = 2.0 ** -8 * X + (64 * X + n / 16 + 16 + rl.abs()) * U       # of a logit
        assert ((lse[:, h].double() - rl).abs() <= 2 * shift).all()
        tol = (2 * (torch.exp(2 * shift) - 1))[:, None] * A + 2.0 ** -7 * A
        assert ((O[:, h].double() - ro).abs() <= tol + 2.0 ** -8 * (ro.abs() + tol)).all()


def test_attend_logits_of_minus_infinity(cache):  # noqa: F811
    """Keys of huge scale against fitting queries: weight 0; a row with no other logit gives zeros."""
    log("attend8 -inf logits")
    pool = Pool8(cache, [70, 3], 1, 16, "int8", seed=34)
    for b, which in ((0, [0, 40, 69]), (1, [0, 1, 2])):
        k = pool.k[b].clone()
        k[which] = -3e38
        pool.put(b, k, pool.v[b])
    Q = normal(12, (4, 1, 64), BF).abs() * 8 + 8
    pc, batch = pool.cuda(), pool.batch([2, 2])
    O, lse = cache.attend(pc, batch, Q.cuda(), False)
    assert (O[2:] == 0).all() and torch.isneginf(lse[2:]).all()
    keep = [i for i in range(70) if i not in (0, 40, 69)]
    pool.k[0][[0, 40, 69]] = 0.0
    ro, rl, _, A, X = whole64(Q[:2, 0], pool.k[0][keep, 0], pool.v[0][keep, 0], torch.ones(2, 67, dtype=torch.bool), 0.125)
    E = (64 * X + 21 + rl.abs()) * U
    assert ((lse[:2, 0].cpu().double() - rl).abs() <= 2 * E).all()
    assert ((O[:2, 0].cpu().double() - ro).abs() <= 2 * E[:, None] * A + 2.0 ** -8 * A + 2.0 ** -7 * ro.abs()).all()


@pytest.mark.parametrize("kind", KINDS)
def test_attend_strides_and_in_place(cache, kind):  # noqa: F811
    """Queries as slices of a projection; O may be Q; equal bits every time."""
    log("attend8 strides %s" % kind)
    pool = Pool8(cache, [500, 60], 2, 16, kind, seed=40)
    pc, batch = pool.cuda(), pool.batch([33, 7])
    fused = normal(18, (40, 12, 64), BF).cuda()
    O, lse = cache.attend(pc, batch, fused[:, 2:8], True)
    Q = fused[:, 2:8].contiguous()
    O2, lse2 = cache.attend(pc, batch, Q, True, O=Q)
    assert torch.equal(O, O2) and torch.equal(lse, lse2) and O2 is Q
    with pytest.raises(Exception):
        cache.attend(pc, batch, Q, True, O=Q, weight_out=pool.gW)


def test_long_offsets(cache):  # noqa: F811
    """A pool of more than 2^32 bytes of codes and of scales' elements times four: slots at its end."""
    log("attend8 past 32 bits")
    npages, Hkv, page = 17000, 4, 1024         # 4.46e9 bytes of K
    K, V = (torch.zeros(npages, Hkv, page, 64, dtype=torch.int8, device="cuda") for _ in range(2))
    scale = torch.ones(npages, Hkv, page, 2, dtype=BF, device="cuda")
    pc = cache.PagedCache(K, V, None, None, scale=scale)
    table = torch.tensor([[npages - 1, 3], [npages - 2, npages - 3]], dtype=torch.int32, device="cuda")
    k, v, q = (normal(i, (2000, h, 64), BF).cuda() for i, h in ((1, 4), (2, 4), (3, 8)))
    batch = cache.Batch(table, i32([1500, 500]), i32([0, 1500, 2000]), 1500, 1500)
    cache.append(pc, batch, q, k, v)
    rk, rv = cache.read(pc, batch, 2000)
    for x, r in ((k, rk), (v, rv)):
        assert torch.equal(r.cpu().double(), codes64.quantise64(x.cpu(), "int8")[2])
    one = cache.Batch(table, i32([1500, 500]), i32([0, 1, 2]), 1, 1500)
    O, _ = cache.attend(pc, one, q[:2])
    for b, (a, e) in enumerate(((0, 1500), (1500, 2000))):
        for h in range(8):
            x = (rk[a:e, h // 2].double() @ q[b, h].double()) / 8
            want = torch.softmax(x, 0) @ rv[a:e, h // 2].double()
            assert (O[b, h].double() - want).abs().max() <= 2.0 ** -7 * want.abs().max()
    assert (K[:3] == 0).all() and (K[4:npages - 3] == 0).all()


def test_graphs_streams_and_workspaces(cache):  # noqa: F811
    """A decoding step captured once and replayed with other contents, on another stream, with workspaces of its own; two
    captured graphs that share a workspace, one after the other."""
    log("cache8 graphs")
    pool = Pool8(cache, [2000, 900], 2, 16, "e4m3", seed=41)
    pc, batch = pool.cuda(), pool.batch([1, 1], seen=[2000, 900])
    Q, K, V = (normal(i, (2, h, 64), BF).cuda() for i, h in ((1, 8), (2, 2), (3, 2)))
    pos = torch.tensor([[1999], [899]], dtype=torch.int32, device="cuda")
    rot, norm = cache.Rotary.make(64), cache.HeadNorm("rms", 1 + normal(9, (64,), F32).cuda())
    ws = cache.attend_workspace(pc, batch, 8, 2)

    def step():
        q = cache.append(pc, batch, Q, K, V, pos, rot, q_norm=norm, k_norm=norm)
        O, lse = cache.attend(pc, batch, q, True, weight_out=pool.gW, ws=ws)
        return O, lse, cache.read(pc, batch, 2)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = [t.clone() for t in step()]
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    W0 = pool.gW.clone()
    for k in range(4):
        Q.copy_(normal(30 + k, (2, 8, 64), BF))
        K.copy_(normal(40 + k, (2, 2, 64), BF))
        results = []
        for g, out in graphs:
            pool.gW.copy_(W0)
            g.replay()
            results.append([t.clone() for t in out] + [pool.gW.clone()])
        pool.gW.copy_(W0)
        results.append(list(step()) + [pool.gW])
        torch.cuda.synchronize()
        for r in results[:2]:
            assert all(torch.equal(a, b) for a, b in zip(r, results[2])), k
    assert len(eager) == 3


# ------------------------------------------------------------------ eviction and the layer

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,keep,sink,recent", [([300, 20, 0, 77], 64, 3, 9), ([45000, 17000], 9000, 100, 1000)])
def test_evict(cache, kind, lens, keep, sink, recent):  # noqa: F811
    """As of a plain cache whose rows are the codes, with their scales."""
    log("evict8 %s %s" % (lens, kind))
    pool = Pool8(cache, [0] * len(lens), 2, 16, kind, seed=50, cap=max(lens), spare=sum(-(-n // 16) for n in lens) + 3)
    ids = torch.randperm(pool.npages, generator=gen(1)).to(torch.int32)
    at = 0
    for b, n in enumerate(lens):
        m = -(-n // 16)
        pool.table[b, :m] = ids[at:at + m].numpy()
        at += m
    pool.lens = list(lens)
    shape = (pool.npages, 2, 16)
    pool.K, pool.V = (torch.randint(0, 256, shape + (64,), generator=gen(5 + j)).to(torch.uint8) for j in range(2))
    pool.scale = torch.randint(0, 32000, shape + (2,), generator=gen(7)).to(torch.int16).view(BF)
    pool.W = torch.rand(shape, generator=gen(8))
    pool.W[torch.rand(shape, generator=gen(9)) < 0.3] = 0.25
    for b, n in enumerate(lens):
        p, s = pool.at(b, n)
        for h in range(2):
            pool.S[p, h, s] = torch.randperm(n, generator=gen(10 + b + h)).to(torch.int32)
    # the same codes as the first 64 bf16 features of a plain cache: its eviction is the reference
    wide = lambda t: torch.cat([t.to(BF)], dim=3)
    rk, rv = wide(pool.K), wide(pool.V)
    rk2 = rk.clone()
    rk2[..., :1], rv2 = pool.scale[..., :1], rv.clone()
    rv2[..., :1] = pool.scale[..., 1:]
    outs = []
    for K, V in ((rk, rv), (rk2, rv2)):
        W, S, length = pool.W.cuda(), pool.S.cuda(), i32(lens)
        pc = cache.PagedCache(K.cuda(), V.cuda(), W, S)
        cache.evict(pc, torch.from_numpy(pool.table).cuda(), length, i32(lens), keep, max(lens), sink, recent)
        outs.append((pc.K.cpu(), pc.V.cpu(), W.cpu(), S.cpu(), length.cpu()))
    pc = pool.cuda()
    length = i32(lens)
    cache.evict(pc, pool.gtable, length, i32(lens), keep, max(lens), sink, recent)
    (k, v, W, S, n), (k2, v2, *_) = outs
    assert torch.equal(length.cpu(), n) and torch.equal(pool.gW.cpu(), W) and torch.equal(pool.gS.cpu(), S)
    assert torch.equal(pool.gK.cpu().view(torch.uint8).to(BF), k) and torch.equal(pool.gV.cpu().view(torch.uint8).to(BF), v)
    bits = lambda t: t.contiguous().view(torch.int16)
    assert torch.equal(bits(pool.gscale.cpu()[..., 0]), bits(k2[..., 0]))
    assert torch.equal(bits(pool.gscale.cpu()[..., 1]), bits(v2[..., 0]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [BF, F32])
def test_stream_layer(cache, kind, rows):  # noqa: F811
    """Chunks of two scenes through a bounded 8-bit cache with norms and positions, each step against a plain cache that is
    given the same values: outputs as attention of the values that the codes stand for."""
    log("stream layer 8 bits %s %s" % (kind, rows))
    rot = cache.Rotary.make(64, 100.0, 2)
    qn = cache.HeadNorm("layer", 1 + normal(1, (64,), F32, 0.2).cuda(), normal(2, (64,), F32, 0.2).cuda())
    kn = cache.HeadNorm("rms", 1 + normal(3, (2, 64), F32, 0.2).cuda())
    layer = cache.StreamLayer(2, keep=120, max_chunk=50, Hq=4, Hkv=2, page=16, dtype=codes64.CODES[kind], sink=10, recent=20,
                              rot=rot, q_norm=qn, k_norm=kn, rows=rows)
    plain = cache.StreamLayer(2, keep=120, max_chunk=50, Hq=4, Hkv=2, page=16, dtype=F32, sink=10, recent=20)
    for step in range(7):
        counts = [50, 1] if step % 2 else [31, 50]
        T = sum(counts)
        Q, K, V = (normal(100 * step + i, (T, h, 64), rows).cuda() for i, h in ((1, 4), (2, 2), (3, 2)))
        pos = torch.randint(0, 30, (T, 2), generator=gen(step)).to(torch.int32).cuda()
        O = layer.step(Q, K, V, pos, counts=counts)
        assert O.dtype == rows
        # the values of this chunk as codes hold them
        q = cache.norm_rotary(Q.float(), qn, pos, rot)
        k = cache.norm_rotary(K.float(), kn, pos, rot)
        held = lambda t: codes64.quantise64(t.cpu(), kind)[2].float().cuda()
        P = plain.step(q if rows == F32 else q.to(BF).float(), held(k), held(V.float()), counts=counts)
        assert layer.lens == plain.lens
        # (the layers may choose other victims among equal weights; few of these are)
        assert (O.float() - P).abs().max() <= (2.0 ** -6 if rows == BF else 1e-4) * max(1.0, P.abs().max().item()), step


@pytest.mark.parametrize("kind", KINDS)
def test_stream_example(cache, kind):  # noqa: F811
    """examples/stream_views.py over codes: three small views through a block; the attention of every view against 64 bits
    over the values that the codes of all views' keys and values stand for (tolerance of test_gpu_cache.py's)."""
    log("stream example %s" % kind)
    import importlib.util
    import os
    from paper_2609_23733_amd import synth
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "stream_views.py")
    spec = importlib.util.spec_from_file_location("stream_views", at)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    P = 90
    outs = ex.main(3, 10 * P, P, kind)
    w = {k: v.cuda() for k, v in synth.make_block_weights((1, 0)).items()}
    pos = torch.from_numpy(synth.token_positions(1, P)).cuda()
    ws = torch.empty(vp.block_workspace_bytes(1, P), dtype=torch.uint8, device="cuda")
    ks, vs = [], []
    for v in range(3):
        X = synth.make_block_input(1, P, (1, v), device="cuda")
        Q, K, V = (t.cpu() for t in vp.block_qkv(X, pos, w, 1, P, ws))
        ks.append(codes64.quantise64(K.double(), kind)[2]), vs.append(codes64.quantise64(V.double(), kind)[2])
        K, V = torch.cat(ks), torch.cat(vs)
        Y = torch.empty(P, 16, 64, dtype=BF)
        every = torch.ones(P, K.shape[0], dtype=torch.bool)
        for h in range(16):
            Y[:, h] = whole64(Q[:, h], K[:, h], V[:, h], every, 0.125)[0].to(BF)
        ref = vp.block_out(X, Y.cuda(), w, 1, P, ws).float()
        err = (outs[v].float() - ref).abs().max().item()
        assert err <= 2.0 ** -5 * ref.abs().max().item(), (v, err)


def test_other_devices(cache, monkeypatch):  # noqa: F811
    """Tensors that are not on the current device are refused (the current device's number is what is changed here)."""
    K, V = (torch.zeros(4, 2, 16, 64, dtype=torch.int8, device="cuda") for _ in range(2))
    pc = cache.PagedCache(K, V, scale=torch.ones(4, 2, 16, 2, dtype=BF, device="cuda"))
    batch = cache.Batch(i32([[0]]), i32([5]), i32([0, 2]), 2, 5)
    rows = normal(1, (2, 2, 64), BF).cuda()
    full = cache.PagedCache.empty(4, 2, 16, torch.int8)
    n = cache.HeadNorm("rms")
    ws = cache.attend_workspace(pc, batch, 2, 2)
    k, v = torch.empty_like(rows), torch.empty_like(rows)
    calls = [lambda: cache.append(pc, batch, rows, rows, rows, Q_out=k), lambda: cache.read(pc, batch, 2, K_out=k, V_out=v),
             lambda: cache.norm_rotary(rows, n, out=k), lambda: cache.attend(pc, batch, rows, O=k, ws=ws),
             lambda: cache.evict(full, batch.table, batch.length, i32([5]), 4, 5)]
    for call in calls:
        call()
    # (frequencies elsewhere: what a Rotary made while another device was the current one has)
    rot, pos = cache.Rotary.make(64), torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    rot.freq = rot.freq.cpu()
    for call in (lambda: cache.norm_rotary(rows, n, pos, rot), lambda: cache.append(pc, batch, rows, rows, rows, pos, rot)):
        with pytest.raises(ValueError, match="device"):
            call()
    real = cache._device()
    with monkeypatch.context() as m:
        m.setattr(cache, "_device", lambda: real + 1)
        for call in calls:
            with pytest.raises(ValueError, match="device"):
                call()


def test_refusals(cache):  # noqa: F811
    mk = lambda *s, dtype=torch.int8: torch.zeros(*s, dtype=dtype, device="cuda")
    K, V, s = mk(4, 2, 16, 64), mk(4, 2, 16, 64), mk(4, 2, 16, 2, dtype=BF)
    pc = cache.PagedCache(K, V, scale=s)
    assert pc.dtype is BF and cache.PagedCache(K, V, scale=s, rows=F32).dtype is F32
    for args in (dict(), dict(scale=s[:3]), dict(scale=s.float()), dict(scale=s, rows=torch.float16)):
        with pytest.raises(ValueError):
            cache.PagedCache(K, V, **args)
    with pytest.raises(ValueError):
        cache.PagedCache(K, V.view(torch.float8_e4m3fn), scale=s)
    with pytest.raises(ValueError):
        cache.PagedCache(mk(4, 2, 16, 64, dtype=BF), mk(4, 2, 16, 64, dtype=BF), scale=s)
    with pytest.raises(ValueError):
        cache.PagedCache(mk(4, 2, 16, 64, dtype=BF), mk(4, 2, 16, 64, dtype=BF), rows=F32)
    batch = cache.Batch(i32([[0]]), i32([5]), i32([0, 2]), 2, 5)
    rows = normal(1, (2, 2, 64), F32).cuda()
    with pytest.raises(ValueError):
        cache.append(pc, batch, rows, rows, rows)              # rows are bf16 here
    with pytest.raises(ValueError):
        cache.attend(pc, batch, rows)
    with pytest.raises(ValueError):
        cache.read(pc, batch, 2, torch.float16)
    with pytest.raises(ValueError):
        cache.read(pc, batch, 2, BF, K_out=rows)
    with pytest.raises(ValueError):
        cache.read(pc, batch, 2, K_out=rows[:1], V_out=rows)
    with pytest.raises(ValueError, match="heads"):
        cache.append(pc, batch, rows.to(BF), rows.to(BF), rows.to(BF), k_norm=cache.HeadNorm("rms", torch.ones(3, 64, device="cuda")))
    with pytest.raises(TypeError):
        cache.StreamLayer(1, 10, 10, 2, dtype=torch.float16)


# ------------------------------------------------------------------ precision of many rows

def check_rms(cache, pool, Q, n, q, causal, below=0.0):  # noqa: F811
    """Mean squares over the call: of the errors no more than what two roundings leave, in units of a row's largest output
    (so that rows of small outputs count as others do).  The output's own, to bf16, is taken from the reference itself.
    Probabilities of more than 2^-14 of the largest in fp16 or finer: off by 2^-11 of themselves, each apart, so by a third of that squared
    on the average, and an output by sum p^2 v^2 times it (single bf16 values: 2^-8 for 2^-11); logits, each
    apart, by 64 u X, sums by (n / 16 + 16 + |lse|) u of the output.  `below`: what smaller probabilities may take, together, of a row's
    largest output.  1 % for the sample, some 300,000 values, whose root of the mean square varies by 0.2 %."""
    Hq, Hkv = Q.shape[1], pool.k[0].shape[1]
    pc, batch = pool.cuda(), pool.batch([q])
    assert cache.attend_plan(pc, batch, Hq, q).shared == 1
    O, lse = cache.attend(pc, batch, Q.cuda(), causal)
    see = n - q + torch.arange(q, device="cuda") + 1 if causal else torch.full((q,), n, device="cuda")
    sees = torch.arange(n, device="cuda") < see[:, None]
    err = own = rest = 0.0
    for h in range(Hq):
        k, v = (t[0][:, h * Hkv // Hq].cuda() for t in (pool.k, pool.v))
        ro, rl, p, A, X = whole64(Q[:, h].cuda(), k, v, sees, 0.125)
        E = (64 * X + n / 16 + 16 + rl.abs()) * U
        assert ((lse[:, h].double() - rl).abs() <= 2 * E).all(), h
        unit = ro.abs().amax(dim=1, keepdim=True)
        top = v.abs().max()                                   # (squares stay in range)
        term = torch.sqrt((p * p) @ (v / top) ** 2) * top * (2.0 ** -11 / 3 ** 0.5 + 64 * X[:, None] * U)
        term += 2 * ro.abs() * (n / 16 + 16 + rl.abs())[:, None] * U + below * unit
        mean = lambda e: ((e / unit) ** 2).mean().item() / Hq
        err, own, rest = err + mean(O[:, h].double() - ro), own + mean(ro.to(BF).double() - ro), rest + mean(term)
    got, most = math.sqrt(err), math.sqrt(own) + math.sqrt(rest)
    log("errors %.2e of a row's largest output, at most %.2e + %.2e" % (got, math.sqrt(own), math.sqrt(rest)))
    assert got <= 1.01 * most


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("q,causal", [(700, False), (520, True)])
def test_attend_wide_precision(cache, kind, q, causal):  # noqa: F811
    """Outputs of many rows are as exact as those of few: their own rounding, and little more."""
    log("attend8 wide precision %s q=%d" % (kind, q))
    n = 6000
    pool = Pool8(cache, [n], 4, 32, kind, seed=61, junk="bits")
    check_rms(cache, pool, normal(62, (q, 8, 64), BF), n, q, causal)


RISE = [
    # logit of the first slot, of slot 3,001, values of the first slot, of the first 64, exponents of the others
    (16.0, 0.0, 0.0, 1.0, 0), (40.0, 0.0, 0.0, 1.0, 0), (0.0, 13.0, 1.0, 1.0, 0), (0.0, 30.0, 1.0, 1.0, 0), (20.0, 45.0, 0.0, 1.0, 0),
    (0.0, 0.0, 0.0, 0.0, 0), (0.0, 0.0, 1.0, 1.0, 30), (16.0, 0.0, 0.0, 2.0 ** -40, 8), (9.0, 12.0, 0.0, 2.0 ** 20, 0),
    (0.0, 0.0, 1.0, 2.0 ** -9, 0), (0.0, 0.0, 1.0, 2.0 ** -11, 0), (0.0, 0.0, 1.0, 2.0 ** 12, 1),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("q", [700, 520])
@pytest.mark.parametrize("first,later,v0,v64,spread", RISE)
def test_attend_wide_precision_of_uneven_slots(cache, kind, q, first, later, v0, v64, spread):  # noqa: F811
    """The same where one slot has most of the weight, early or late, with values or without, and where values
    differ by many powers of two from slot to slot."""
    log("attend8 wide precision %s q=%d %s" % (kind, q, (first, later, v0, v64, spread)))
    n = 6000
    pool = Pool8(cache, [n], 4, 32, kind, seed=63)
    k, v = normal(64, (n, 4, 64), F32), normal(65, (n, 4, 64), F32)
    Q = normal(66, (q, 8, 64), BF)
    Q[..., 0] = 8.0
    k[..., 0] = 0.0
    for at, x in ((0, first), (3000, later)):
        if x:
            k[at], k[at, :, 0] = 0.0, x          # (a logit of x with every query)
    v *= torch.exp2(torch.randint(-spread, spread + 1, (n, 1, 1), generator=gen(67)).float())
    v[:64] *= v64
    v[0] *= v0
    pool.put(0, k, v)
    check_rms(cache, pool, Q, n, q, False, 2.0 ** -10)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("up", [-40, 8, 9, 10, 11, 12, 13, 40])
def test_attend_wide_precision_of_the_last_slots(cache, kind, up):  # noqa: F811
    """The same where the slots of the last tile, which is not full, have larger values than all others, or smaller ones and
    nearly all of the weight."""
    log("attend8 wide precision %s, last slots 2^%d" % (kind, up))
    n, q = 6000, 700
    pool = Pool8(cache, [n], 4, 32, kind, seed=68)
    k, v = normal(69, (n, 4, 64), F32), normal(70, (n, 4, 64), F32)
    v[n - 40:] *= 2.0 ** up
    Q = normal(71, (q, 8, 64), BF)
    if up < 0:
        Q[..., 0], k[..., 0], k[n - 40:, :, 0] = 8.0, 0.0, 50.0
    pool.put(0, k, v)
    check_rms(cache, pool, Q, n, q, False, 2.0 ** -10)


class Elsewhere(torch.Tensor):
    """A tensor that says to be on the next device."""

    def get_device(self):
        return torch.cuda.current_device() + 1


def test_batches_and_norms_of_other_devices(cache):  # noqa: F811
    """Every tensor of a batch, and a norm's gain or bias as exchanged, are looked at before a call passes them on."""
    there = lambda t: t.as_subclass(Elsewhere)
    pc = cache.PagedCache.empty(4, 2, 16, torch.int8)
    rows = normal(1, (2, 2, 64), BF).cuda()
    own = [i32([[0]]), i32([5]), i32([0, 2]), i32([5])]
    mk = lambda *t: cache.Batch(*t[:3], 2, 5, t[3])
    calls = [lambda b: cache.append(pc, b, rows, rows, rows), lambda b: cache.read(pc, b, 2),
             lambda b: cache.attend(pc, b, rows)]
    for call in calls:
        call(mk(*own))
        for i in range(4):
            with pytest.raises(ValueError, match="device"):
                call(mk(*[there(t) if i == j else t for j, t in enumerate(own)]))
    for plain in (pc, cache.PagedCache.empty(4, 2, 16)):
        for which in ("q_norm", "k_norm"):
            for name in ("gain", "bias"):
                n = cache.HeadNorm("rms", **{name: torch.ones(64, device="cuda")})
                call = lambda: cache.append(plain, mk(*own), rows, rows, rows, **{which: n})
                call()
                setattr(n, name, there(torch.ones(64, device="cuda")))
                with pytest.raises(ValueError, match="device"):
                    call()
    # a plain cache's tensors, in the calls that it shares with codes
    full = cache.PagedCache.empty(4, 2, 16)
    for i in range(1, 4):
        t = [full.K, full.V, full.weight, full.stamp]
        t[i] = there(t[i])
        odd = cache.PagedCache(*t)
        for call in (lambda: cache.append(odd, mk(*own), rows, rows, rows, q_norm=cache.HeadNorm("rms")),
                     lambda: cache.read(odd, mk(*own), 2)):
            with pytest.raises(ValueError, match="device"):
                call()


def test_gradients_are_refused(cache):  # noqa: F811
    """Calls that have no gradients to give, with something that requires them: refused, where a graph would be
    expected; taken under no_grad.  The plain cache's own calls take them as ever."""
    own = (i32([[0]]), i32([5]), i32([0, 2]), 2, 5, i32([5]))
    batch = cache.Batch(*own)
    rows, leaf = normal(1, (2, 2, 64), BF).cuda(), normal(1, (2, 2, 64), BF).cuda().requires_grad_()
    codes, plain = cache.PagedCache.empty(4, 2, 16, torch.int8), cache.PagedCache.empty(4, 2, 16)
    one = torch.ones(64, device="cuda")
    gain, bias = cache.HeadNorm("rms", one.clone().requires_grad_()), cache.HeadNorm("rms", one, one.clone().requires_grad_())
    calls = [lambda x=x: cache.append(codes, batch, *x) for x in ((leaf, rows, rows), (rows, leaf, rows), (rows, rows, leaf))]
    calls += [lambda pc=pc, n=n, w=w: cache.append(pc, batch, rows, rows, rows, **{w: n})
              for pc in (codes, plain) for n in (gain, bias) for w in ("q_norm", "k_norm")]
    calls += [lambda: cache.append(plain, batch, leaf, rows, rows, q_norm=cache.HeadNorm("rms")),
              lambda: cache.append(codes, batch, rows, rows, rows, Q_out=leaf.detach().clone().requires_grad_()),
              lambda: cache.attend(codes, batch, leaf), lambda: cache.attend(codes, batch, rows, O=leaf.detach().clone().requires_grad_()),
              lambda: cache.read(codes, batch, 2, K_out=leaf.detach().clone().requires_grad_()),
              lambda: cache.StreamLayer(1, 10, 10, 2, q_norm=gain).step(rows, rows, rows),
              lambda: cache.StreamLayer(1, 10, 10, 2, dtype=torch.int8).step(leaf, rows, rows)]
    for call in calls:
        with pytest.raises(ValueError, match="no_grad"):
            call()
        with torch.no_grad():
            call()
    for call in (lambda: cache.append(plain, batch, leaf, leaf, leaf), lambda: cache.attend(plain, batch, leaf)[0]):
        assert not call().requires_grad
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(rows, rows)
        for call in (lambda: cache.append(codes, batch, rows, dual, rows), lambda: cache.attend(codes, batch, dual)):
            with pytest.raises(ValueError, match="forward-mode"):
                call()


@pytest.mark.parametrize("rows", [BF, F32])
@pytest.mark.parametrize("dim,axes,layout", [(None, 1, "half"), (32, 1, "half"), (32, 2, "interleaved"), (10, 1, "half"), (10, 1, "interleaved")])
def test_features_that_are_not_turned(cache, rows, dim, axes, layout):  # noqa: F811
    """Without a norm they pass unchanged, as in the plain append: an infinity or a NaN stays in its feature."""
    T = 40
    pos = torch.randint(-1000, 1000, (T, axes), generator=gen(1)).to(torch.int32).cuda()
    turn = (None, None) if dim is None else (pos, cache.Rotary.make(dim, 100.0, axes, layout))
    Q, K, V = (normal(s, (T, h, 64), rows) for s, h in ((2, 4), (3, 2), (4, 2)))
    for x in (Q, K):
        x[3, 1, 63], x[5, 0, 40], x[6, 1, 33], x[7, 0, 62] = math.inf, -math.inf, math.nan, math.inf
    Q, K, V = Q.cuda(), K.cuda(), V.cuda()
    batch = cache.Batch(i32([[0, 1, 2]]), i32([T]), i32([0, T]), T, T, i32([T]))
    plain = cache.PagedCache.empty(3, 2, 16, rows)
    want = cache.append(plain, batch, Q, K, V, *turn)
    # (the turned features: the compiler fuses either product of a pair)
    same = lambda a, b: torch.allclose(a.float(), b.float(), rtol=2.0 ** -7 if rows == BF else 1e-5, atol=1e-5, equal_nan=True)
    codes = cache.PagedCache.empty(3, 2, 16, torch.int8, rows=rows)
    assert same(cache.append(codes, batch, Q, K, V, *turn), want)
    norm = cache.HeadNorm("rms")
    other = cache.PagedCache.empty(3, 2, 16, rows)
    assert same(cache.append(other, batch, Q, K, V, *turn, k_norm=norm), want)
    cache.append(other, batch, Q, K, V, *turn, q_norm=norm)
    for a, b in zip(cache.read(other, batch, T), cache.read(plain, batch, T)):
        assert same(a, b)


@pytest.mark.parametrize("where", ["chunk", "before"])
def test_attend_wide_codes_of_nan(cache, where):  # noqa: F811
    """e4m3 NaN codes by the kernel of many rows: in the chunk, where some rows see their slots and others do not, and before
    it, where all do.  Features without one are right wherever the row's logits are numbers."""
    log("attend8 wide, NaN codes %s" % where)
    n, q = 4000, 1500
    pool = Pool8(cache, [n], 4, 32, "e4m3", seed=45)
    Q = normal(46, (q, 16, 64), BF)
    p, s = pool.at(0, n)
    end = n if where == "chunk" else n - q
    kn, v1, v2 = end - 3, end - 9, end - 400
    pool.K[p[kn], 1, s[kn], 9] = 255
    pool.V[p[v1], 0, s[v1], 5], pool.V[p[v2], 2, s[v2], 33] = 127, 255
    pc, batch = pool.cuda(), pool.batch([q])
    assert cache.attend_plan(pc, batch, 16, q).shared == 1
    O, lse = (t.double() for t in cache.attend(pc, batch, Q.cuda(), True))
    see = n - q + torch.arange(q, device="cuda") + 1
    sees = torch.arange(n, device="cuda") < see[:, None]
    for h in range(16):
        k, v = pool.k[0][:, h // 4].cuda(), pool.v[0][:, h // 4].cuda()
        ro, rl, _, A, X = whole64(Q[:, h].cuda(), k, v, sees, 0.125)
        E = (64 * X + n / 16 + 16 + rl.abs()) * U
        tol = torch.from_numpy(bf16_tol((2 * E[:, None] * A).cpu().numpy(), A.cpu().numpy(), ro.cpu().numpy())).cuda()
        nan = torch.zeros(q, 64, dtype=torch.bool, device="cuda")
        lost = torch.zeros(q, dtype=torch.bool, device="cuda")
        for hk, at, f in ((0, v1, 5), (2, v2, 33)):
            if h // 4 == hk:
                nan[:, f] = see > at
        if h // 4 == 1:
            lost = see > kn
            nan[lost] = True
        assert torch.equal(torch.isnan(O[:, h]), nan), h
        assert ((O[:, h] - ro).abs() <= tol)[~nan].all(), h
        assert torch.equal(torch.isnan(lse[:, h]), lost) and ((lse[:, h] - rl).abs() <= 2 * E)[~lost].all(), h


@pytest.mark.parametrize("rows", [BF, F32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("q", [1, 5, 90])
def test_weights_over_pages_that_do_not_exist(cache, rows, kind, q):  # noqa: F811
    """Logits kept (one and five tokens) and formed again: slots on missing pages keep their weights, the others get theirs."""
    log("attend8 weights, bad pages %s %s q=%d" % (rows, kind, q))
    n = 4700
    gone = [s for p in (2, 17, 42) for s in range(16 * p, 16 * p + 16)]
    pool = Pool8(cache, [n], 1, 16, kind, seed=35, rows=rows)
    pc, batch = pool.cuda(), pool.batch([q])
    assert cache.attend_plan(pc, batch, 2, q).logits_kept == (q < 90)
    check(cache, pool, normal(13, (q, 2, 64), rows), [q], True, 0, gone=gone)


def test_another_stream_and_workspace(cache):  # noqa: F811
    """The same step on the default stream and, at the same time, on two others with workspaces and caches of their own."""
    log("cache8 streams")
    rot, norm = cache.Rotary.make(64), cache.HeadNorm("rms", 1 + normal(9, (64,), F32).cuda())
    pos = torch.tensor([[1999], [899]], dtype=torch.int32, device="cuda")
    steps = []
    for k in range(3):
        pool = Pool8(cache, [2000, 900], 2, 16, "e4m3", seed=41)
        pc, batch = pool.cuda(), pool.batch([1, 1], seen=[2000, 900])
        Q, K, V = (normal(i, (2, h, 64), BF).cuda() for i, h in ((1, 8), (2, 2), (3, 2)))
        steps.append((pool, pc, batch, Q, K, V, cache.attend_workspace(pc, batch, 8, 2).fill_(255)))

    def run(pool, pc, batch, Q, K, V, ws):
        out = []
        for _ in range(20):
            q = cache.append(pc, batch, Q, K, V, pos, rot, q_norm=norm, k_norm=norm)
            O, lse = cache.attend(pc, batch, q, True, weight_out=pool.gW, ws=ws)
            out += [O, lse, *cache.read(pc, batch, 2)]
        return out + [pool.gW]

    torch.cuda.synchronize()
    outs = []
    streams = [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
    for st, args in zip(streams, steps):
        with torch.cuda.stream(st):
            outs.append(run(*args))
    torch.cuda.synchronize()
    for other in outs[1:]:
        assert len(other) == len(outs[0]) and all(torch.equal(a, b) for a, b in zip(outs[0], other))
