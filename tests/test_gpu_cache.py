"""The paged key-value cache on the GPU against plain 64-bit computations on the CPU: rotary
positions, append, attention with its weights, eviction, and the stream layer that runs them.

Tolerances (set before the first run).  u = 2^-24.  A logit of 64 products accumulated in
fp32 is off by at most 64 u X, X = scale sum_i |q_i k_i| at its largest over the row's slots; the
exponential, its argument and the sum of n probabilities in chains of n / 16 add (16 + n / 16) u.
So with E = (64 X + n / 16 + 16 + |lse|) u an output is off by at most 2 E A, A = sum_j p_j |v_j|, lse
by 2 E, and a weight by 2 E plus its own chain of R rows, R u, times its value.  bf16 (8 significant
bits, rounding error up to 2^-8 of the value) rounds every probability, 2^-8 A, and the
output, 2^-8 |O|."""
import math
import sys

import numpy as np
import pytest
import torch

from paper_2609_23733_amd import vp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BFU = 2.0 ** -8
BF, F32 = torch.bfloat16, torch.float32


def log(msg):
    sys.stdout.write("[gpu-case] %s\n" % msg)
    sys.stdout.flush()


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    vp.load_library()


@pytest.fixture()
def cache():
    from paper_2609_23733_amd import cache as c
    return c


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(seed, shape, dtype=BF, std=1.0):
    return (torch.randn(*shape, generator=gen(seed)) * std).to(dtype)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ rotary

def rotate64(x, pos, f, axes, layout, mag, sign=1.0):
    """x [T, H, 64] in 64 bits; f radians per position, in the order of the pairs."""
    y = x.double().clone()
    n = len(f) // axes
    for p in range(len(f)):
        a, j = p // n, p % n
        i0, i1 = (2 * a * n + j, 2 * a * n + j + n) if layout == "half" else (2 * p, 2 * p + 1)
        ang = sign * pos[:, a].double() * f[p]
        c, s = torch.cos(ang)[:, None] * mag, torch.sin(ang)[:, None] * mag
        x0, x1 = x[:, :, i0].double(), x[:, :, i1].double()
        y[:, :, i0], y[:, :, i1] = x0 * c - x1 * s, x1 * c + x0 * s
    return y


def radians(rot):
    return [(int(v) & ((1 << 64) - 1)) / 2.0 ** 64 * 2 * math.pi for v in rot.freq.cpu().tolist()]


def rot_tol(x, ref, mag, dtype):
    """Angles to 2^-24 of half a turn (pi 2^-24) and 2 ulp of sine and cosine: 6 u per feature of the
    pair, three roundings; bf16 outputs are rounded."""
    pair = float(mag) * 2.0 * x.double().abs().amax(dim=2, keepdim=True)
    t = 12 * U * pair
    return t + (BFU * (ref.abs() + t) if dtype == BF else 0) + 1e-30


@pytest.mark.parametrize("T,H,dtype,dim,axes,layout,scaling", [
    (1, 1, F32, 64, 1, "half", "none"), (13, 16, F32, 64, 1, "half", "parts"),
    (257, 3, BF, 48, 1, "interleaved", "linear"), (77, 16, BF, 64, 2, "half", "none"),
    (5, 4, F32, 12, 1, "half", "none"), (5, 4, F32, 60, 2, "half", "none"),
    (9, 2, BF, 24, 4, "interleaved", "none"), (9, 2, F32, 6, 3, "half", "none"),
    (33, 8, BF, 10, 1, "interleaved", "none"), (3, 128, BF, 2, 1, "half", "none"),
    (4099, 16, BF, 64, 1, "half", "none"), (20011, 2, F32, 64, 1, "interleaved", "parts")])
def test_rotary(cache, T, H, dtype, dim, axes, layout, scaling):
    log("rotary T=%d H=%d dim=%d axes=%d %s %s" % (T, H, dim, axes, layout, scaling))
    rot = cache.Rotary.make(dim, 10000.0, axes, layout, scaling, 8.0, 4096.0)
    x = normal(T + dim, (T, H, 64), dtype)
    pos = torch.randint(-(1 << 20), 1 << 20, (T, axes), generator=gen(T)).to(torch.int32)
    for transpose in (False, True):
        ref = rotate64(x, pos, radians(rot), axes, layout, rot.mag, -1.0 if transpose else 1.0)
        y = cache.rotary(x.cuda(), pos.cuda(), rot, transpose=transpose).cpu().double()
        err = (y - ref).abs()
        assert (err <= rot_tol(x, ref, rot.mag, dtype)).all(), (transpose, err.max().item())
        assert torch.equal(y[:, :, dim:], x[:, :, dim:].double())


def test_rotary_any_position(cache):
    """Positions at the ends of int32: the angle from exact integer arithmetic."""
    log("rotary extreme positions")
    rot = cache.Rotary.make(64, 10000.0)
    pos = torch.tensor([[0], [1], [-1], [2 ** 31 - 1], [-2 ** 31], [123456789], [-987654321]],
                       dtype=torch.int32)
    x = normal(5, (7, 2, 64), F32)
    y = cache.rotary(x.cuda(), pos.cuda(), rot).cpu().double()
    fixed = [int(v) & ((1 << 64) - 1) for v in rot.freq.cpu().tolist()]
    for t in range(7):
        turns = [((int(pos[t, 0]) * f) % (1 << 64)) / 2.0 ** 64 for f in fixed]
        ref = rotate64(x[t:t + 1], torch.ones(1, 1), [2 * math.pi * v for v in turns], 1, "half", 1.0)
        assert (y[t:t + 1] - ref).abs().max() <= 12 * U * 2 * x.abs().max(), t


def test_rotary_strided_and_in_place(cache):
    log("rotary strides")
    rot = cache.Rotary.make(32, 10000.0, 1, "interleaved")
    fused = normal(6, (41, 10, 64), BF).cuda()
    pos = torch.arange(41, dtype=torch.int32, device="cuda")[:, None]
    a = cache.rotary(fused[:, 2:7], pos, rot)
    b = cache.rotary(fused[:, 2:7].contiguous(), pos, rot)
    assert torch.equal(a, b)
    whole = fused.clone()
    cache.rotary(whole[:, 2:7], pos, rot, out=whole[:, 2:7])
    assert torch.equal(whole[:, 2:7], b)
    assert torch.equal(whole[:, :2], fused[:, :2]) and torch.equal(whole[:, 7:], fused[:, 7:])
    assert cache.rotary(fused[:0, 2:7], pos[:0], rot).shape == (0, 5, 64)


def test_rotary_gradient_by_differences(cache):
    """sum(g y(x)) differentiated by x: central differences of the kernel's own forward (the map is
    linear, so a step of 1 has no truncation error) against the transposed map of g."""
    log("rotary gradient")
    rot = cache.Rotary.make(64, 100.0, 2, "half", "parts", 4.0, 64.0)
    pos = torch.randint(0, 500, (6, 2), generator=gen(9)).to(torch.int32).cuda()
    x, g = normal(10, (6, 2, 64), F32), normal(11, (6, 2, 64), F32).cuda()
    dx = cache.rotary(g, pos, rot, transpose=True).cpu().double()
    base = x.cuda()
    for j in range(64):
        up, dn = base.clone(), base.clone()
        up[:, :, j] += 1
        dn[:, :, j] -= 1
        d = (cache.rotary(up, pos, rot).double() - cache.rotary(dn, pos, rot).double()) * g.double()
        num = d.sum(dim=2).cpu() / 2
        scale = 12 * U * 2 * 2 * rot.mag * (x.abs().max() + 1) * g.abs().max().cpu() * 2 + 2 * U * 8
        assert (num - dx[:, :, j]).abs().max() <= scale, j


# ------------------------------------------------------------------ pools and batches

class Pool:
    """A pool with the sequences' pages scattered over it, and everything outside the sequences'
    slots filled with `junk`."""

    def __init__(self, cache, lens, Hkv, page, dtype, seed, spare=3, junk=float("nan"), cap=0,
                 std=1.0, vstd=1.0):
        r = np.random.RandomState(seed)
        self.lens, self.page, self.Hkv, self.dtype = list(lens), page, Hkv, dtype
        need = [-(-n // page) for n in lens]
        self.npages = sum(need) + spare
        ids = r.permutation(self.npages)
        width = max(need + [-(-cap // page), 1])
        self.table = np.full((len(lens), width), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        shape = (self.npages, Hkv, page)
        self.K = torch.full(shape + (64,), junk, dtype=dtype)
        self.V = torch.full(shape + (64,), junk, dtype=dtype)
        self.W = torch.rand(shape, generator=gen(seed + 3)) * 0.1
        self.S = torch.full(shape, -7, dtype=torch.int32)
        self.k, self.v = [], []
        for b, n in enumerate(lens):
            k, v = normal(seed + 10 + b, (n, Hkv, 64), dtype, std), normal(seed + 500 + b, (n, Hkv, 64), dtype, vstd)
            self.put(b, k, v)
        self.c = cache

    def at(self, b, n):
        s = np.arange(n)
        return torch.from_numpy(self.table[b, s // self.page].astype(np.int64)), torch.from_numpy(s % self.page)

    def put(self, b, k, v):
        p, s = self.at(b, k.shape[0])
        self.K[p, :, s], self.V[p, :, s] = k, v
        if len(self.k) <= b:
            self.k.append(k), self.v.append(v)
        else:
            self.k[b], self.v[b] = k, v

    def cuda(self):
        g = lambda t: t.cuda()
        self.gK, self.gV, self.gW, self.gS = g(self.K), g(self.V), g(self.W), g(self.S)
        self.gtable = torch.from_numpy(self.table).cuda()
        return self.c.PagedCache(self.gK, self.gV, self.gW, self.gS)

    def batch(self, qs, seen=None, slack=0):
        start = [0]
        for q in qs:
            start.append(start[-1] + q)
        return self.c.Batch(self.gtable, i32(self.lens), i32(start), max(qs),
                            max(max(self.lens) + slack, 0), None if seen is None else i32(seen))


def attend64(q, k, v, vis, scale=0.125):
    """One head: q [R, 64], the first vis[r] slots: (O, lse, p, A, X) in 64 bits; slots a row does
    not see are left out of its sums."""
    R, n = q.shape[0], k.shape[0]
    O, A = np.zeros((R, 64)), np.zeros((R, 64))
    lse, X, p = np.full(R, -np.inf), np.zeros(R), np.zeros((R, n))
    q, k, v = q.double().numpy(), k.double().numpy(), v.double().numpy()
    for m in sorted(set(vis.tolist())):
        if m <= 0:
            continue
        r = np.nonzero(vis == m)[0]
        with np.errstate(all="ignore"):
            x = scale * q[r] @ k[:m].T
            top = x.max(axis=1, keepdims=True)
            top = np.where(np.isneginf(top), 0, top)
            e = np.exp(x - top)
            s = e.sum(axis=1, keepdims=True)
            pr = np.where(s > 0, e / np.where(s == 0, 1, s), np.where(np.isnan(s), np.nan, 0))
            O[r], A[r] = pr @ v[:m], np.abs(pr) @ np.abs(v[:m])
            lse[r] = np.where(s[:, 0] == 0, -np.inf, top[:, 0] + np.log(s[:, 0]))
            X[r] = scale * (np.abs(q[r]) @ np.abs(k[:m]).T).max(axis=1)
        p[r, :m] = pr
    return O, lse, p, A, X


def check_attend(cache, pool, Q, qs, causal, scale=0.0, weights=True, slack=0, ws=None):
    """Runs attend on the pool and compares everything with attend64."""
    pc = pool.cuda()
    batch = pool.batch(qs, slack=slack)
    T, Hq, Hkv = Q.shape[0], Q.shape[1], pool.Hkv
    G = Hq // Hkv
    W = pool.W.cuda()
    W_out = W.clone() if weights else None
    O, lse = cache.attend(pc, batch, Q.cuda() if not Q.is_cuda else Q, causal, scale, weight_out=W_out, ws=ws)
    torch.cuda.synchronize()
    O, lse = O.cpu().double().numpy(), lse.cpu().double().numpy()
    Wref, Wtol = pool.W.double().numpy().copy(), np.zeros(pool.W.shape)
    s = 0.125 if scale == 0 else scale
    Qc = Q.cpu()
    t = 0
    for b, m in enumerate(qs):
        n = pool.lens[b]
        p_, s_ = (x.numpy() for x in pool.at(b, n))
        vis = np.clip(n - m + np.arange(m) + 1, 0, n) if causal else np.full(m, n)
        for h in range(Hq):
            if m == 0:
                continue
            hk = h // G
            ro, rl, rp, A, X = attend64(Qc[t:t + m, h], pool.k[b][:, hk], pool.v[b][:, hk], vis, s)
            fin = np.where(np.isfinite(rl), np.abs(rl), 0)
            E = (64 * X + n / 16 + 16 + fin) * U
            tol = 2 * E[:, None] * A + 1e-30
            if pool.dtype == BF:
                tol = bf16_tol(tol, A, ro)
            got = O[t:t + m, h]
            bad = ~(np.abs(got - ro) <= tol)
            assert not bad.any(), (b, h, np.argwhere(bad)[:4].tolist(), got[bad][:4], ro[bad][:4], tol[bad][:4])
            gl, same = lse[t:t + m, h], np.isneginf(rl)
            assert (np.isneginf(gl) == same).all(), (b, h)
            assert (np.abs(gl[~same] - rl[~same]) <= 2 * E[~same] + 2 * U * fin[~same]).all(), (b, h)
            Wref[p_, hk, s_] += rp.sum(axis=0)
            Wtol[p_, hk, s_] += (rp * (2 * E[:, None] + m * G * U)).sum(axis=0)
        t += m
    if weights:
        got = W_out.cpu().double().numpy()
        assert (np.abs(got - Wref) <= Wtol + 4 * U * np.abs(Wref) + 1e-30).all(), np.abs(got - Wref).max()
    return O, lse


def bf16_tol(tol, A, ro, on=True):
    """`tol` with the roundings of a bf16 cache: probabilities, then the output."""
    if not on:
        return tol
    tol = tol + BFU * A
    return tol + BFU * (np.abs(ro) + tol)


# ------------------------------------------------------------------ attention

ATTEND = [
    # lens, chunk sizes, Hq, Hkv, page, dtype, causal
    ([1], [1], 1, 1, 16, BF, True), ([1], [1], 16, 16, 64, F32, False),
    ([31], [1], 4, 4, 16, BF, True), ([33, 64, 65], [1, 1, 1], 16, 4, 16, BF, True),
    ([300], [1], 16, 16, 64, BF, True), ([1374, 5, 700, 0], [1, 1, 0, 0], 16, 8, 32, BF, True),
    ([2500, 1], [1, 1], 6, 2, 128, F32, True), ([5000], [1], 16, 1, 256, BF, True),
    ([40], [40], 2, 1, 16, BF, True), ([40], [40], 2, 1, 16, F32, True),
    ([130, 257, 64], [64, 3, 64], 4, 4, 16, BF, True), ([130, 257, 64], [64, 3, 64], 4, 4, 16, F32, True),
    ([640], [257], 3, 1, 64, BF, True), ([640], [257], 3, 1, 64, F32, True),
    ([1000], [300], 2, 2, 4096, BF, False), ([777, 100], [130, 90], 12, 4, 32, F32, False),
    ([3000, 61, 900], [129, 61, 1], 8, 2, 16, BF, True), ([4100], [70], 2, 2, 32, BF, False),
    ([9000], [2], 2, 2, 64, BF, True), ([2050], [66], 4, 1, 1024, F32, True),
]


@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,dtype,causal", ATTEND)
def test_attend(cache, lens, qs, Hq, Hkv, page, dtype, causal):
    log("attend %s %s Hq=%d Hkv=%d page=%d %s causal=%d" % (lens, qs, Hq, Hkv, page, dtype, causal))
    pool = Pool(cache, lens, Hkv, page, dtype, seed=100 + sum(lens))
    check_attend(cache, pool, normal(7, (sum(qs), Hq, 64), dtype), qs, causal)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("q", [3, 200])
def test_attend_rows_that_see_nothing(cache, dtype, q):
    """More new tokens than slots (their start was dropped): the first rows see nothing."""
    log("attend empty rows q=%d %s" % (q, dtype))
    pool = Pool(cache, [2, 0, 150], 2, 16, dtype, seed=31)
    O, lse = check_attend(cache, pool, normal(8, (3 * q, 4, 64), dtype), [q, q, q], True)
    assert (O[:q - 2] == 0).all() and np.isneginf(lse[:q - 2]).all()
    assert (O[q:2 * q] == 0).all() and np.isneginf(lse[q:2 * q]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq", [2, 6])
def test_attend_unseen_tokens_may_hold_anything(cache, dtype, Hq):
    """Values of later tokens of the chunk that are infinite or NaN, and keys, reach the rows that
    see them and no others."""
    log("attend nonfinite later tokens %s" % dtype)
    n, q = 150, 140
    pool = Pool(cache, [n], 2, 32, dtype, seed=33)
    k, v = pool.k[0].clone(), pool.v[0].clone()
    v[n - 9, 0, 5], v[n - 7, 1, 63], v[n - 40, 0, 33] = float("nan"), float("inf"), float("-inf")
    k[n - 5, 0, 3], k[n - 3, 1, 60] = float("nan"), float("inf")
    pool.put(0, k, v)
    Q = normal(9, (q, Hq, 64), dtype)
    pc, batch = pool.cuda(), pool.batch([q])
    W = pool.W.cuda()
    O, lse = cache.attend(pc, batch, Q.cuda(), True, weight_out=W)
    O, lse = O.cpu().double().numpy(), lse.cpu().double().numpy()
    G = Hq // 2
    vis = n - q + np.arange(q) + 1
    for h in range(Hq):
        ro, rl, rp, A, X = attend64(Q[:, h], k[:, h // G], v[:, h // G], vis)
        want, got = np.isfinite(ro), np.isfinite(O[:, h])
        assert (want == got).all(), (h, np.argwhere(want != got)[:5].tolist())
        assert (np.isnan(ro) == np.isnan(O[:, h])).all(), h
        inf = np.isinf(ro)
        assert (ro[inf] == O[:, h][inf]).all()
        E = (64 * X + n / 16 + 16) * U
        with np.errstate(invalid="ignore"):
            tol = bf16_tol(2 * E[:, None] * A, A, ro, dtype == BF)
            assert (np.abs(O[:, h] - ro)[want] <= tol[want]).all(), h
            assert (np.isnan(rl) == np.isnan(lse[:, h])).all(), h


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_logits_of_minus_infinity(cache, dtype):
    """Keys with an infinite component against queries of the opposite sign: weight 0; a row
    with no other logit gives zeros; +inf logits give NaN."""
    log("attend -inf logits %s" % dtype)
    pool = Pool(cache, [70, 3], 1, 16, dtype, seed=34)
    for b, rows in ((0, [0, 40, 69]), (1, [0, 1, 2])):
        k = pool.k[b].clone()
        k[rows, 0] = 0.5
        k[rows, 0, 2] = float("-inf")
        pool.put(b, k, pool.v[b])
    Q = normal(12, (4, 1, 64), dtype).abs()
    Q[3, 0, 2] = -1.0
    pc, batch = pool.cuda(), pool.batch([2, 2])
    O, lse = cache.attend(pc, batch, Q.cuda(), False)
    O, lse = O.cpu().double().numpy()[:, 0], lse.cpu().double().numpy()[:, 0]
    keep = [i for i in range(70) if i not in (0, 40, 69)]
    ro, rl, _, A, X = attend64(Q[:2, 0], pool.k[0][keep, 0], pool.v[0][keep, 0], np.full(2, 67))
    E = (64 * X + 21) * U
    assert (np.abs(O[:2] - ro) <= bf16_tol(2 * E[:, None] * A, A, ro, dtype == BF)).all()
    assert (np.abs(lse[:2] - rl) <= 2 * E + 2 * U * np.abs(rl)).all()
    assert (O[2] == 0).all() and np.isneginf(lse[2])
    assert np.isnan(O[3]).all() and np.isnan(lse[3])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("q", [1, 90])
def test_attend_pages_that_do_not_exist(cache, dtype, q):
    """Numbers outside the pool in the table: their slots are not seen, nothing else changes."""
    log("attend bad pages %s q=%d" % (dtype, q))
    n = 700
    pool = Pool(cache, [n], 1, 16, dtype, seed=35)
    bad = [2, 17, 43]
    seen = np.array([i for i in range(n) if i // 16 not in bad])
    pc, batch = pool.cuda(), pool.batch([q])
    for i, p in enumerate(bad):
        pool.gtable[0, p] = [-1, pool.npages, 2 ** 31 - 1][i]
    Q = normal(13, (q, 2, 64), dtype)
    W = pool.W.cuda()
    O, lse = cache.attend(pc, batch, Q.cuda(), True, weight_out=W)
    O, lse = O.cpu().double().numpy(), lse.cpu().double().numpy()
    vis = np.array([(seen <= n - q + i).sum() for i in range(q)])
    for h in range(2):
        ro, rl, rp, A, X = attend64(Q[:, h], pool.k[0][seen, 0], pool.v[0][seen, 0], vis)
        E = (64 * X + n / 16 + 16 + np.abs(rl)) * U
        tol = bf16_tol(2 * E[:, None] * A, A, ro, dtype == BF)
        assert (np.abs(O[:, h] - ro) <= tol).all()
        assert (np.abs(lse[:, h] - rl) <= 2 * E).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_large_logits(cache, dtype):
    """Sharp rows: logits of some hundreds, the largest late in the sequence, so that the running
    reference has to move; the 64-bit result on the same inputs."""
    log("attend large logits %s" % dtype)
    pool = Pool(cache, [900], 2, 64, dtype, seed=36, std=6.0)
    k = pool.k[0].clone()
    k[800:] *= 4
    pool.put(0, k, pool.v[0])
    check_attend(cache, pool, normal(14, (70, 4, 64), dtype, 6.0), [70], False)
    check_attend(cache, pool, normal(15, (1, 4, 64), dtype, 6.0), [1], True, scale=0.5)


@pytest.mark.parametrize("ks,qs,vs", [(1, 1, 1e-30), (1, 1, 1e-36), (1, 1, 1e35), (1e30, 1e-30, 1), (1e-30, 1e30, 1e-33),
                                      (1e35, 1e-35, 1), (1e-36, 1e36, 1), (3, 3, 1)])
def test_attend_fp32_ranges(cache, ks, qs, vs):
    """fp32 operands far from 1 and of unequal size keep their bits, in chunks (whose products are
    made of bf16 parts where those hold them) as in single tokens."""
    log("attend fp32 ranges k=%g q=%g v=%g" % (ks, qs, vs))
    pool = Pool(cache, [333, 200], 1, 32, F32, seed=41, std=ks, vstd=vs)
    check_attend(cache, pool, normal(42, (333, 1, 64), F32, qs), [200, 133], True)
    check_attend(cache, pool, normal(43, (2, 1, 64), F32, qs), [1, 1], True)


def test_attend_fp32_small_parts(cache):
    """One feature whose key is far below the others and whose query makes up for it; values that are 0
    but for slots of vanishing probability; large values at such slots."""
    log("attend fp32 small parts")
    pool = Pool(cache, [300], 1, 32, F32, seed=44)
    k, v = pool.k[0].clone(), pool.v[0].clone()
    k[:, 0, 7] *= 2.0 ** -112
    pool.put(0, k, v)
    Q = normal(45, (100, 1, 64), F32)
    Q[:, 0, 7] *= 2.0 ** 113
    check_attend(cache, pool, Q, [100], False)
    k = normal(46, (300, 1, 64), F32)
    k[100:200] *= 0.01
    k[:, 0, 0] = 0
    k[100:200, 0, 0] = -8 * 78.0        # logits 78 below the others for queries of 1
    Q = normal(47, (100, 1, 64), F32)
    Q[:, 0, 0] = 1
    for big in (1.0, 1e30):
        v = torch.zeros(300, 1, 64)
        v[100:200] = normal(48, (100, 1, 64), F32) * big
        pool.put(0, k, v)
        check_attend(cache, pool, Q, [100], False)


def test_attend_strided_queries_streams_and_bounds(cache):
    """Queries as a slice of a projection's output; a stream of its own; bounds above the sizes."""
    log("attend strides, streams, bounds")
    pool = Pool(cache, [500, 77], 2, 32, BF, seed=37, cap=4000)
    qs = [33, 60]
    x = normal(16, (93, 8, 64), BF).cuda()
    check_attend(cache, pool, x[:, 2:6], qs, True)
    check_attend(cache, pool, x[:, 2:6].contiguous(), qs, True, slack=3000)
    pc, batch = pool.cuda(), pool.batch(qs)
    a, la = cache.attend(pc, batch, x[:, 2:6])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b, lb = cache.attend(pc, batch, x[:, 2:6])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_attend_weights_in_place_and_idle_sequences(cache):
    log("attend weights in place")
    pool = Pool(cache, [200, 90, 64], 2, 16, BF, seed=38)
    pc, batch = pool.cuda(), pool.batch([5, 0, 9])
    Q = normal(17, (14, 4, 64), BF).cuda()
    W = pool.W.cuda()
    cache.attend(pc, batch, Q, True, weight_out=W)
    cache.attend(pc, batch, Q, True, weight_out=pc.weight)
    assert torch.equal(W, pc.weight)
    p, s = pool.at(1, 90)
    assert torch.equal(W.cpu()[p, :, s], pool.W[p, :, s])
    # sums: every row gives 1
    used = torch.zeros_like(pool.W, dtype=torch.bool)
    for b in (0, 2):
        p, s = pool.at(b, pool.lens[b])
        used[p, :, s] = True
    total = (W.cpu().double() - pool.W.double())[used].sum().item()
    assert abs(total - 14 * 4) <= 14 * 4 * 1e-4
    assert torch.equal(W.cpu()[~used], pool.W[~used])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_past_32_bit_offsets(cache, dtype):
    """Pages whose elements lie past 2^32: a pool of 2^32 + elements of which two sequences use the last
    pages."""
    log("attend large offsets %s" % dtype)
    page, Hkv = 256, 8
    npages = (1 << 32) // (page * Hkv * 64) + 40
    K = torch.empty(npages, Hkv, page, 64, dtype=dtype, device="cuda")
    V = torch.empty_like(K)
    lens, qs = [1000, 300], [1, 100]
    small = Pool(cache, lens, Hkv, page, dtype, seed=39, junk=0.0)
    K[-small.npages:], V[-small.npages:] = small.K.cuda(), small.V.cuda()
    Q = normal(18, (101, Hkv, 64), dtype).cuda()
    small.cuda()
    shift = torch.where(small.gtable >= 0, small.gtable + (npages - small.npages), -1).to(torch.int32)
    pc = cache.PagedCache(K, V)
    b = small.batch(qs)
    big = cache.Batch(shift, b.length, b.q_start, b.max_q, b.max_len)
    want = cache.attend(cache.PagedCache(small.gK, small.gV), b, Q)
    got = cache.attend(pc, big, Q)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    new = normal(19, (101, Hkv, 64), dtype).cuda()
    cache.append(pc, big, None, new, new)
    p = shift[1, 299 // page].item()
    assert torch.equal(K[p, :, 299 % page], new[100])


def test_attend_graph_replays(cache):
    """Append and attend captured as a graph: every replay gives the eager pass's result, also with
    eager work between, and with other tokens in the same buffers."""
    log("cache graph")
    pool = Pool(cache, [600, 90, 1374], 4, 16, BF, seed=40)
    pc, qs = pool.cuda(), [1, 1, 1]
    batch = pool.batch(qs, seen=[700, 90, 1374])
    Q, K, V = (normal(20 + i, (3, h, 64), BF).cuda() for i, h in enumerate((8, 4, 4)))
    rot = cache.Rotary.make(64, 10000.0)
    pos = i32([[699], [89], [1373]])
    O, lse = torch.empty_like(Q), torch.empty(3, 8, device="cuda")
    ws = cache.attend_workspace(pc, batch, 8, 3)
    W = pool.W.cuda()

    def step():
        q = cache.append(pc, batch, Q, K, V, pos, rot, Q_out=Qr)
        cache.attend(pc, batch, q, True, O=O, lse=lse, weight_out=W2, ws=ws)

    Qr, W2 = torch.empty_like(Q), W.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for k in range(4):
        if k == 2:
            Q.copy_(normal(60, (3, 8, 64), BF))
            K.copy_(normal(61, (3, 4, 64), BF))
        step()
        want = [t.clone() for t in (O, lse, W2)]
        for t in (O, lse):
            t.fill_(float("nan"))
        W2.copy_(W)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (O, lse, W2)):
            assert torch.equal(a, b), k


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,dtype,layout,dim", [
    ([1], [1], 1, 1, 16, F32, "half", 64), ([65, 16, 300, 9], [5, 16, 0, 1], 8, 2, 16, BF, "interleaved", 48),
    ([1400], [1374], 16, 16, 64, BF, "half", 64), ([10, 2], [3, 5], 4, 4, 32, F32, "half", 20)])
def test_append(cache, lens, qs, Hq, Hkv, page, dtype, layout, dim):
    log("append %s %s Hq=%d Hkv=%d %s" % (lens, qs, Hq, Hkv, dtype))
    pool = Pool(cache, lens, Hkv, page, dtype, seed=50, junk=0.25)
    T = sum(qs)
    seen = [n + 11 for n in lens]
    x = normal(51, (T, Hq + 2 * Hkv, 64), dtype)
    pos = torch.randint(0, 9999, (T, 1), generator=gen(52)).to(torch.int32)
    rot = cache.Rotary.make(dim, 10000.0, 1, layout, "parts", 8.0, 1024.0)
    pc = pool.cuda()
    g = x.cuda()
    Q = cache.append(pc, pool.batch(qs, seen), g[:, :Hq], g[:, Hq:Hq + Hkv], g[:, Hq + Hkv:], pos.cuda(), rot)
    ref = rotate64(x, pos, radians(rot), 1, layout, rot.mag)
    tol = rot_tol(x, ref, rot.mag, dtype)
    assert ((Q.cpu().double() - ref[:, :Hq]).abs() <= tol[:, :Hq]).all()
    K, V, W, S = pool.K.clone().double(), pool.V.clone(), pool.W.clone(), pool.S.clone()
    Kt = torch.zeros_like(K)
    t = 0
    for b, (n, m) in enumerate(zip(lens, qs)):
        for i in range(m):
            s = n - m + i
            if s >= 0:
                p = pool.table[b, s // page]
                K[p, :, s % page], Kt[p, :, s % page] = ref[t, Hq:Hq + Hkv], tol[t, Hq:Hq + Hkv]
                V[p, :, s % page] = x[t, Hq + Hkv:]
                W[p, :, s % page] = 0
                S[p, :, s % page] = seen[b] - m + i
            t += 1
    assert ((pool.gK.cpu().double() - K).abs() <= Kt).all()
    assert torch.equal(pool.gV.cpu(), V) and torch.equal(pool.gW.cpu(), W) and torch.equal(pool.gS.cpu(), S)


def test_append_plain(cache):
    """No rotation, no queries, no weights and stamps; pages that do not exist are left out."""
    log("append plain")
    pool = Pool(cache, [40], 2, 16, BF, seed=53, junk=0.5)
    pool.cuda()
    pool.gtable[0, 1] = 99
    x = normal(54, (40, 2, 64), BF).cuda()
    pc = cache.PagedCache(pool.gK, pool.gV)
    assert cache.append(pc, pool.batch([40]), None, x, x) is None
    K = pool.K.clone()
    for s in list(range(16)) + list(range(32, 40)):
        K[pool.table[0, s // 16], :, s % 16] = x[s].cpu()
    assert torch.equal(pool.gK.cpu(), K)


# ------------------------------------------------------------------ eviction

def evict64(pool, K, V, W, S, seen, keep, sink, recent):
    """The definition, slot by slot, in place on CPU tensors; returns the new lengths."""
    out = []
    for b, n in enumerate(pool.lens):
        left = min(n, keep)
        out.append(left)
        p, s = pool.at(b, n)
        for h in range(pool.Hkv):
            w, st = W[p, h, s].tolist(), S[p, h, s].tolist()
            safe = [t < sink or t >= seen[b] - recent for t in st]

            def rank(i):
                v = w[i]
                return (0, 0.0, i) if safe[i] else (1, -math.inf, i - 2 * n) if v != v else (1, -v, i)

            kept = set(sorted(range(n), key=rank)[:left])
            holes = [i for i in range(left) if i not in kept]
            movers = sorted(i for i in kept if i >= left)
            assert len(holes) == len(movers)
            for d, i in zip(holes, movers):
                for x in (K, V, W, S):
                    x[p[d], h, s[d]] = x[p[i], h, s[i]].clone()
    return out


EVICT = [
    # lens, keep, sink, recent, Hkv, page, dtype, kind of weights
    ([1], 1, 0, 0, 1, 16, BF, "plain"), ([5], 1, 0, 0, 2, 16, F32, "plain"),
    ([100, 30, 0, 64], 40, 2, 7, 3, 16, BF, "ties"), ([1000], 999, 0, 0, 1, 32, F32, "plain"),
    ([1000, 900], 300, 500, 0, 2, 64, BF, "plain"), ([1000], 300, 0, 500, 2, 64, BF, "ties"),
    ([4096, 4097], 2000, 5, 100, 2, 128, BF, "odd"), ([13000, 700], 5000, 10, 64, 2, 64, F32, "ties"),
    ([9000], 4500, 0, 0, 1, 256, BF, "equal"), ([8193], 8192, 0, 1, 1, 16, BF, "odd"),
    ([30000], 100, 0, 0, 1, 64, BF, "plain"),
]


def weights_of(kind, shape, seed):
    w = torch.exp(2 * torch.randn(shape, generator=gen(seed)))
    if kind == "ties":
        w = torch.floor(w * 2) / 2
    if kind == "equal":
        w = torch.ones(shape)
    if kind == "odd":
        r = torch.rand(shape, generator=gen(seed + 1))
        w = torch.where(r < 0.05, torch.full(shape, float("nan")), w)
        w = torch.where((r > 0.05) & (r < 0.1), torch.full(shape, float("inf")), w)
        w = torch.where((r > 0.1) & (r < 0.3), torch.full(shape, -0.0), w)
        w = torch.where((r > 0.3) & (r < 0.5), torch.full(shape, 0.0), w)
        w = torch.where((r > 0.5) & (r < 0.6), -w, w)
        w = torch.where((r > 0.6) & (r < 0.65), torch.full(shape, float("-inf")), w)
    return w


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("lens,keep,sink,recent,Hkv,page,dtype,kind", EVICT)
def test_evict(cache, lens, keep, sink, recent, Hkv, page, dtype, kind, in_place):
    log("evict %s keep=%d sink=%d recent=%d Hkv=%d page=%d %s %s" %
        (lens, keep, sink, recent, Hkv, page, dtype, kind))
    pool = Pool(cache, lens, Hkv, page, dtype, seed=70, junk=0.5)
    pool.W = weights_of(kind, pool.W.shape, 71)
    seen = [n + n // 2 for n in lens]
    for b, n in enumerate(lens):
        p, s = pool.at(b, n)
        for h in range(Hkv):
            o = torch.randperm(n, generator=gen(72 + b + 10 * h))
            pool.S[p, h, s] = torch.where(o < sink, o, o + n // 2).to(torch.int32)
    pc = pool.cuda()
    K, V, W, S = pool.K.clone(), pool.V.clone(), pool.W.clone(), pool.S.clone()
    left = evict64(pool, K, V, W, S, seen, keep, sink, recent)
    length = i32(lens)
    if in_place:
        wo, so, lo = pool.gW, pool.gS, length
        got = cache.evict(pc, pool.gtable, length, i32(seen), keep, max(lens), sink, recent)
    else:
        wo, so, lo = torch.full_like(pool.gW, 3.0), torch.full_like(pool.gS, -9), torch.zeros_like(length)
        got = cache.evict(pc, pool.gtable, length, i32(seen), keep, max(lens) + 0, sink, recent, wo, so, lo)
        assert torch.equal(pool.gW.cpu().view(torch.int32), pool.W.view(torch.int32))
    assert got is lo and got.tolist() == left
    assert torch.equal(pool.gK.cpu(), K) and torch.equal(pool.gV.cpu(), V)
    for b, n in enumerate(left):
        p, s = pool.at(b, n)
        assert torch.equal(wo.cpu()[p, :, s].view(torch.int32), W[p, :, s].view(torch.int32)), b
        assert torch.equal(so.cpu()[p, :, s], S[p, :, s]), b
    if not in_place:       # nothing but the slots that stay is written
        mask = torch.ones_like(pool.W, dtype=torch.bool)
        for b, n in enumerate(left):
            p, s = pool.at(b, n)
            mask[p, :, s] = False
        assert (wo.cpu()[mask] == 3.0).all() and (so.cpu()[mask] == -9).all()


def test_evict_graph_replays(cache):
    log("evict graph")
    pool = Pool(cache, [3000, 900], 2, 64, BF, seed=75, junk=0.5)
    pool.W = weights_of("ties", pool.W.shape, 76)
    pc = pool.cuda()
    length, seen, lo = i32([3000, 900]), i32([3000, 900]), i32([0, 0])
    wo, so = pool.gW.clone(), pool.gS.clone()
    ws = cache.evict_workspace(pc, 2, 3000)
    go = lambda: cache.evict(pc, pool.gtable, length, seen, 700, 3000, 0, 0, wo, so, lo, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    want = [t.clone() for t in (pool.gK, wo, so, lo)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    for k in range(4):
        pool.gK.copy_(pool.K.cuda())
        pool.gV.copy_(pool.V.cuda())
        lo.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (pool.gK, wo, so, lo)):
            assert torch.equal(a, b), k
        ws.random_(0, 255)     # the workspace holds nothing from call to call


# ------------------------------------------------------------------ the stream layer

@pytest.mark.parametrize("dtype,causal,Hq,Hkv", [(BF, False, 4, 4), (F32, True, 4, 2)])
def test_stream_layer(cache, dtype, causal, Hq, Hkv):
    """Chunks of two sequences through a cache that overflows: every step's output against 64-bit
    attention over what the cache held, every eviction against the definition on the weights
    that were gathered."""
    log("stream layer %s causal=%d" % (dtype, causal))
    rot = cache.Rotary.make(64, 10000.0)
    layer = cache.StreamLayer(2, keep=150, max_chunk=70, Hq=Hq, Hkv=Hkv, page=16, dtype=dtype, sink=3,
                              recent=20, causal=causal, rot=rot)
    table = layer.table.cpu().numpy()
    lens, G = [0, 0], Hq // Hkv
    for step, counts in enumerate([[70, 1], [60, 33], [1, 70], [70, 70], [0, 65], [70, 0], [1, 1]]):
        T = sum(counts)
        Q, K, V = (normal(900 + 3 * step + i, (T, h, 64), dtype) for i, h in enumerate((Hq, Hkv, Hkv)))
        pos = torch.cat([torch.arange(c) + 70 * step for c in counts]).to(torch.int32)[:, None]
        before = [t.clone() for t in (layer.pc.K, layer.pc.V, layer.pc.weight, layer.pc.stamp)]
        O = layer.step(Q.cuda(), K.cuda(), V.cuda(), pos.cuda(), counts).cpu()
        # the cache before the eviction, from the parts
        Qr = cache.rotary(Q.cuda(), pos.cuda(), rot).cpu()
        Kr = cache.rotary(K.cuda(), pos.cuda(), rot).cpu()
        Kb, Vb, Wb, Sb = (t.cpu() for t in before)
        t = 0
        seen = layer.seen.tolist()
        for b, m in enumerate(counts):
            n0 = lens[b]
            lens[b] += m
            s = np.arange(n0, lens[b])
            p, s = torch.from_numpy(table[b, s // 16].astype(np.int64)), torch.from_numpy(s % 16)
            Kb[p, :, s], Vb[p, :, s], Wb[p, :, s] = Kr[t:t + m], V[t:t + m], 0.0
            Sb[p, :, s] = torch.arange(seen[b] - m, seen[b], dtype=torch.int32)[:, None].expand(m, Hkv)
            t += m
        t = 0
        for b, m in enumerate(counts):
            n = lens[b]
            s = np.arange(n)
            p, s = torch.from_numpy(table[b, s // 16].astype(np.int64)), torch.from_numpy(s % 16)
            vis = n - m + np.arange(m) + 1 if causal else np.full(m, n)
            for h in range(Hq):
                if m == 0:
                    continue
                ro, rl, rp, A, X = attend64(Qr[t:t + m, h], Kb[p, h // G, s], Vb[p, h // G, s], vis)
                E = (64 * X + n / 16 + 16 + np.abs(rl)) * U
                tol = bf16_tol(2 * E[:, None] * A, A, ro, dtype == BF)
                assert (np.abs(O[t:t + m, h].double().numpy() - ro) <= tol).all(), (step, b, h)
                Wb[p, h // G, s] += torch.from_numpy(rp.sum(axis=0)).float()
            t += m
        # what stayed: the protected slots all, the others by weight (the smallest kept is not below
        # the largest dropped beyond the weights' error)
        left = [min(n, 150) for n in lens]
        assert layer.length.tolist() == left
        Sn, Wn = layer.pc.stamp.cpu(), layer.pc.weight.cpu()
        for b, n in enumerate(lens):
            s = np.arange(n)
            p, s = torch.from_numpy(table[b, s // 16].astype(np.int64)), torch.from_numpy(s % 16)
            for h in range(Hkv):
                old = {int(x): (float(w), i) for i, (x, w) in enumerate(zip(Sb[p, h, s], Wb[p, h, s]))}
                now = Sn[p, h, s][:left[b]].tolist()
                assert len(set(now)) == left[b] and set(now) <= set(old), (step, b, h)
                safe = {x for x in old if x < 3 or x >= seen[b] - 20}
                assert safe <= set(now)
                drop = [old[x][0] for x in set(old) - set(now)]
                kept = [old[x][0] for x in set(now) - safe]
                if drop and kept:
                    assert min(kept) >= max(drop) - 1e-3 * max(drop), (step, b, h)
                kn, vn = layer.pc.K.cpu()[p, h, s], layer.pc.V.cpu()[p, h, s]
                for j, x in enumerate(now):
                    assert torch.equal(kn[j], Kb[p, h, s][old[x][1]]) and torch.equal(vn[j], Vb[p, h, s][old[x][1]])
                    w = float(Wn[p, h, s][j])
                    assert abs(w - old[x][0]) <= 1e-4 * abs(old[x][0]) + 1e-6
            lens[b] = left[b]


def test_stream_example(cache):
    """examples/stream_views.py: three small views through a block; the attention of every view
    against 64 bits over all views' keys and values, formed by the block's own first stage."""
    log("stream example")
    import importlib.util
    import os
    from paper_2609_23733_amd import synth
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "stream_views.py")
    spec = importlib.util.spec_from_file_location("stream_views", at)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    P = 150
    outs = ex.main(3, 10 * P, P)
    w = {k: v.cuda() for k, v in synth.make_block_weights((1, 0)).items()}
    pos = torch.from_numpy(synth.token_positions(1, P)).cuda()
    ws = torch.empty(vp.block_workspace_bytes(1, P), dtype=torch.uint8, device="cuda")
    ks, vs = [], []
    for v in range(3):
        X = synth.make_block_input(1, P, (1, v), device="cuda")
        Q, K, V = (t.cpu() for t in vp.block_qkv(X, pos, w, 1, P, ws))
        ks.append(K), vs.append(V)
        K, V = torch.cat(ks), torch.cat(vs)
        Y = torch.empty(P, 16, 64, dtype=BF)
        for h in range(16):
            ro = attend64(Q[:, h], K[:, h], V[:, h], np.full(P, K.shape[0]))[0]
            Y[:, h] = torch.from_numpy(ro).to(BF)
        ref = vp.block_out(X, Y.cuda(), w, 1, P, ws).float()
        err = (outs[v].float() - ref).abs().max().item()
        # Y's two roundings (at most 2^-7 of its largest entry, most of it random) through W_O, LayerScale
        # (at most 1.5), LN_2 and the FFN: a few 2^-7 of the output's largest entry, 2^-5 as the bar
        assert err <= 2.0 ** -5 * ref.abs().max().item(), (v, err)


def test_stream_layer_refused_chunk(cache):
    """A chunk that is refused leaves the layer as it was: the steps after it equal those of a
    layer that never saw it."""
    log("stream layer refused chunk")
    rot = cache.Rotary.make(64, 10000.0)
    a, b = (cache.StreamLayer(1, keep=60, max_chunk=40, Hq=4, Hkv=2, page=16, rot=rot) for _ in range(2))
    pos = torch.arange(40, dtype=torch.int32, device="cuda")[:, None]
    for step in range(3):
        Q, K, V = (normal(950 + 3 * step + i, (40, h, 64)).cuda() for i, h in enumerate((4, 2, 2)))
        for bad in (dict(K=K[:, :1]), dict(V=V.float()), dict(pos=None), dict(pos=pos[:39]), dict(Q=Q[:, :3]), dict(counts=[41])):
            kw = dict(dict(Q=Q, K=K, V=V, pos=pos, counts=[40]), **bad)
            with pytest.raises((ValueError, vp.VPError)):
                a.step(**kw)
        assert torch.equal(a.step(Q, K, V, pos), b.step(Q, K, V, pos))
        assert a.lens == b.lens and a.length.tolist() == b.length.tolist() == a.lens
        assert a.seen.tolist() == [40 * (step + 1)]


@pytest.mark.parametrize("G,q,dtype", [(3, 70, BF), (5, 41, BF), (7, 19, F32), (48, 5, BF), (65, 3, F32), (128, 2, BF), (2, 300, F32), (3, 5, BF)])
def test_attend_weights_any_group(cache, G, q, dtype):
    """Weights of chunks whose groups do not divide the tiles of rows: heads and tokens step together."""
    log("attend weights G=%d q=%d %s" % (G, q, dtype))
    lens, qs = [q + 130, q + 3], [q, max(1, q // 2)]
    pool = Pool(cache, lens, 1, 16, dtype, seed=G)
    check_attend(cache, pool, normal(G + 1, (sum(qs), G, 64), dtype), qs, True)


@pytest.mark.parametrize("B,q", [(9, 1), (17, 3), (5, 90)])
def test_attend_ragged_batches(cache, B, q):
    """Many sequences, one long, most short, some idle: ranges past a sequence's end."""
    log("attend ragged B=%d q=%d" % (B, q))
    lens = [2000] + [q + 37 * b for b in range(1, B)]
    qs = [q] + [(0 if b % 4 == 3 else max(1, q - b)) for b in range(1, B)]
    pool = Pool(cache, lens, 2, 16, BF, seed=B)
    check_attend(cache, pool, normal(B + 1, (sum(qs), 6, 64), BF), qs, True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("q,H", [(1, 64), (5, 32)])
def test_attend_many_short_pages(cache, dtype, q, H):
    """Ranges of more than 64 pages: the window of page numbers moves on within a range."""
    log("attend many short pages %s q=%d" % (dtype, q))
    pool = Pool(cache, [9011, 4700], H, 16, dtype, seed=71 + q)
    check_attend(cache, pool, normal(72, (2 * q, H, 64), dtype), [q, q], True)


@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,dtype,causal", [
    # many rows over few slots: both kernels' divisions of rows, ragged and equal
    ([200], [200], 2, 2, 16, BF, True), ([700, 700], [300, 300], 4, 2, 32, BF, False), ([90, 1, 300], [90, 1, 70], 3, 1, 16, F32, True),
    ([1374, 1374], [1374, 1374], 8, 8, 64, BF, False), ([3000, 2000, 100], [400, 17, 100], 8, 4, 64, BF, True),
    ([9000], [150], 16, 16, 64, BF, True), ([600], [200], 2, 2, 16, F32, True)])
def test_attend_many_rows(cache, lens, qs, Hq, Hkv, page, dtype, causal):
    log("attend many rows %s %s %s" % (lens, qs, dtype))
    pool = Pool(cache, lens, Hkv, page, dtype, seed=300 + sum(lens))
    check_attend(cache, pool, normal(8, (sum(qs), Hq, 64), dtype), qs, causal)


@pytest.mark.parametrize("q,H,dtype", [(9, 2, BF), (32, 1, BF), (33, 1, BF), (17, 2, F32), (64, 1, F32)])
def test_attend_weights_of_kept_logits(cache, q, H, dtype):
    """Long caches: up to 32 (fp32: 64) rows of a key head keep their logits for the weights."""
    log("attend weights of kept logits q=%d %s" % (q, dtype))
    pool = Pool(cache, [4500, 4097], H, 64, dtype, seed=400 + q)
    check_attend(cache, pool, normal(9, (q + 3, H, 64), dtype), [q, 3], True)
