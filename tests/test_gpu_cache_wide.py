"""The attention of chunks of many rows over many slots, whose workgroups share every tile, and the eviction of
long caches, in six launches: the cases of test_gpu_cache.py that the plan sends elsewhere at their sizes.  Every
attention case states the kernel it is meant for, and the plan has to agree.

References in 64 bits on the GPU, all rows of all heads; tolerances of test_gpu_cache.py."""
import numpy as np
import pytest
import torch

from test_gpu_cache import BF, F32, U, Pool, _gpu, bf16_tol, cache, gen, i32, log, normal  # noqa: F401

pytestmark = pytest.mark.gpu


def whole64(q, k, v, sees, scale):
    """One head, q [R, 64], k and v [n, 64], sees [R, n]: (O, lse, p, A, X) in 64 bits; what a row does not see
    does not reach it, whatever it holds."""
    q, k, v = q.double(), k.double(), v.double()
    x = torch.where(sees, scale * (q @ k.t()), -torch.inf)
    top = x.amax(dim=1, keepdim=True)
    top = torch.where(top == -torch.inf, 0.0, top)
    e = torch.where(sees, torch.exp(x - top), 0.0)
    s = e.sum(dim=1, keepdim=True)
    p = torch.where(sees, e / torch.where(s == 0, 1.0, s), 0.0)
    lse = torch.where(s == 0, -torch.inf, top + torch.log(s))[:, 0]
    fin = torch.isfinite(v)
    vf = torch.where(fin, v, 0.0)
    O, A = p @ vf, p @ vf.abs()
    for j in (~fin).any(dim=1).nonzero()[:, 0].tolist():
        O += torch.where(sees[:, j:j + 1] & ~fin[j], p[:, j:j + 1] * torch.where(fin[j], 0.0, v[j]), 0.0)
    X = scale * (q.abs() @ k.abs().t())
    X = torch.where(sees & torch.isfinite(X), X, 0.0).amax(dim=1)     # (infinite: no weight, or NaN)
    return O, lse, p, A, X


def check(c, pool, Q, qs, causal, shared, scale=0.0, slack=0, gone=(), reach=None):
    """attend with the weights in a copy, everything against whole64.  `gone`: slots of sequence 0 whose pages do
    not exist; `reach`: called with every head's logits."""
    pc, batch = pool.cuda(), pool.batch(qs, slack=slack)
    T, Hq, _ = Q.shape
    G = Hq // pool.Hkv
    assert c.attend_plan(pc, batch, Hq, T).shared == shared
    if len(gone):
        for i, page in enumerate(sorted({s // pool.page for s in gone})):
            pool.gtable[0, page] = [-1, pool.npages, 2 ** 31 - 1][i % 3]
    Q = Q.cuda()
    W = pool.W.cuda()
    O, lse = c.attend(pc, batch, Q, causal, scale, weight_out=W)
    Wref, Wtol = pool.W.double().cuda(), torch.zeros(pool.W.shape, dtype=torch.float64, device="cuda")
    s, t = 0.125 if scale == 0 else scale, 0
    for b, m in enumerate(qs):
        n = pool.lens[b]
        if m == 0 or n == 0:
            assert (O[t:t + m] == 0).all() and torch.isneginf(lse[t:t + m]).all()
            t += m
            continue
        slot, i = torch.arange(n, device="cuda"), torch.arange(m, device="cuda")
        sees = (slot < (n - m + i + 1)[:, None]) if causal else torch.ones(m, n, dtype=torch.bool, device="cuda")
        if b == 0 and len(gone):
            sees = sees & ~torch.isin(slot, torch.tensor(list(gone), device="cuda"))
        p_, s_ = (x.cuda() for x in pool.at(b, n))
        for h in range(Hq):
            hk = h // G
            ro, rl, rp, A, X = whole64(Q[t:t + m, h], pool.k[b][:, hk].cuda(), pool.v[b][:, hk].cuda(), sees, s)
            if reach:
                reach(b, h, torch.where(sees, s * (Q[t:t + m, h].double() @ pool.k[b][:, hk].cuda().double().t()), -torch.inf))
            E = (64 * X + n / 16 + 16 + torch.where(torch.isfinite(rl), rl.abs(), 0.0)) * U
            tol = (2 * E[:, None] * A + 1e-30).cpu().numpy()
            tol = torch.from_numpy(bf16_tol(tol, A.cpu().numpy(), ro.cpu().numpy(), pool.dtype == BF)).cuda()
            got, fin = O[t:t + m, h].double(), torch.isfinite(ro)
            assert torch.equal(torch.isnan(got), torch.isnan(ro)) and torch.equal(torch.isfinite(got), fin), (b, h)
            assert torch.equal(got[torch.isinf(ro)], ro[torch.isinf(ro)]), (b, h)
            err = torch.where(fin, (got - ro).abs(), 0.0)
            bad = fin & ~(err <= tol)
            assert not bad.any(), (b, h, bad.nonzero()[:4].tolist(), err.max().item())
            gl, fl = lse[t:t + m, h].double(), torch.isfinite(rl)
            assert torch.equal(gl[torch.isinf(rl)], rl[torch.isinf(rl)]) and torch.equal(torch.isnan(gl), torch.isnan(rl)), (b, h)
            assert ((gl - rl).abs()[fl] <= (2 * E + 2 * U * rl.abs())[fl]).all(), (b, h)
            Wref[p_, hk, s_] += rp.sum(dim=0)
            Wtol[p_, hk, s_] += (rp * (2 * E[:, None] + m * G * U)).sum(dim=0)
        t += m
    if len(gone):     # (slots without a page are not written: they are the old page's, which no one names now)
        p_, s_ = (x.cuda() for x in pool.at(0, pool.lens[0]))
        lost = torch.isin(torch.arange(pool.lens[0], device="cuda"), torch.tensor(list(gone), device="cuda"))
        assert torch.equal(W[p_[lost], :, s_[lost]], pool.gW[p_[lost], :, s_[lost]])
    W = W.double()
    fin = torch.isfinite(Wref)
    assert torch.equal(torch.isnan(W), torch.isnan(Wref))
    bad = fin & ~((W - Wref).abs() <= Wtol + 4 * U * Wref.abs() + 1e-30)
    assert not bad.any(), (bad.nonzero()[:4].tolist(), (W - Wref).abs()[fin].max().item())
    return O, lse


WIDE = [
    # lens, chunk sizes, Hq, Hkv, page, dtype, causal
    ([1374], [1374], 16, 16, 64, BF, True),                              # a view over itself
    ([3000, 2000, 700, 50], [1100, 900, 300, 0], 8, 4, 32, BF, True),    # ragged, an idle sequence, eight ranges
    ([3300, 90, 2000], [1500, 77, 900], 12, 4, 16, BF, True),            # groups that do not divide the tiles
    ([10000, 300], [260, 17], 16, 4, 64, BF, False),                     # a last tile of a few rows, 23 ranges
    ([2500], [2000], 64, 16, 16, BF, True),                              # one range of 157 pages
    ([2400, 1300], [1300, 1300], 16, 8, 16, BF, True),                   # ranges of more than 64 pages; a chunk alone
    ([3000], [2500], 64, 16, 16, F32, True),                             # the same in fp32
    ([2400, 1300], [1300, 400], 6, 2, 16, F32, True),
    ([6000, 90], [300, 90], 6, 2, 32, F32, False),
]


@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,dtype,causal", WIDE)
def test_attend_wide(cache, lens, qs, Hq, Hkv, page, dtype, causal):  # noqa: F811
    log("wide %s %s Hq=%d Hkv=%d page=%d %s causal=%d" % (lens, qs, Hq, Hkv, page, dtype, causal))
    pool = Pool(cache, lens, Hkv, page, dtype, seed=100 + sum(lens))
    check(cache, pool, normal(7, (sum(qs), Hq, 64), dtype), qs, causal, 1)


def test_attend_wide_ranges_of_many_pages(cache):  # noqa: F811
    """The cases above that are meant to pass 64 pages within a range do."""
    for (lens, qs, Hq, Hkv, page, dtype, causal), n in ((WIDE[4], 64), (WIDE[5], 64), (WIDE[6], 64)):
        pool = Pool(cache, lens, Hkv, page, dtype, seed=1)
        assert cache.attend_plan(pool.cuda(), pool.batch(qs), Hq, sum(qs)).range_slots > n * page


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_wide_rows_that_see_nothing(cache, dtype):  # noqa: F811
    """More new tokens than slots: the first rows see nothing, alone in their workgroups and beside others."""
    log("wide empty rows %s" % dtype)
    pool = Pool(cache, [1000, 0, 1500], 8, 32, dtype, seed=31)
    O, lse = check(cache, pool, normal(8, (4500, 16, 64), dtype), [1500, 1500, 1500], True, 1)
    assert (O[:500] == 0).all() and torch.isneginf(lse[:500]).all()
    assert (O[1500:3000] == 0).all() and torch.isneginf(lse[1500:3000]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq", [16, 24])
def test_attend_wide_unseen_tokens_may_hold_anything(cache, dtype, Hq):  # noqa: F811
    """Values and keys of the chunk's tokens that are infinite or NaN, on the diagonal's tiles and in tiles that
    all rows see, reach the rows that see them and no others; each in a head of its own."""
    log("wide nonfinite %s Hq=%d" % (dtype, Hq))
    n, q, H = 2400, 1300, 8
    pool = Pool(cache, [n, 1300], H, 32, dtype, seed=33)
    k, v = pool.k[0].clone(), pool.v[0].clone()
    nan, inf = float("nan"), float("inf")
    v[n - 9, 0, 5], v[n - 1, 0, 63], v[n - 700, 0, 33], v[n - 701, 0, 34] = nan, inf, -inf, inf
    v[n - 1299, 1, 0], v[n - 64, 1, 17] = inf, nan
    k[n - 5, 2, 3], k[n - 600, 3, 60] = nan, inf
    v[40, 4, 7], v[41, 5, 7] = nan, -inf                     # every row sees these
    pool.put(0, k, v)
    check(cache, pool, normal(9, (q + 1300, Hq, 64), dtype), [q, 1300], True, 1)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_wide_logits_of_minus_infinity(cache, dtype):  # noqa: F811
    """Slots of weight 0 because of a key, among others, in the whole first tile of a range, and in all slots."""
    log("wide -inf logits %s" % dtype)
    n = 2400
    pool = Pool(cache, [n], 8, 32, dtype, seed=34)
    k = pool.k[0].clone()
    k[:, :, 2] = 0.5
    k[::7, 0, 2] = float("-inf")
    k[:900, 1, 2] = float("-inf")
    k[:, 2, 2] = float("-inf")
    pool.put(0, k, pool.v[0])
    Q = normal(12, (1300, 16, 64), dtype)
    Q[:, :, 2] = 1.0
    O, lse = check(cache, pool, Q, [1300], True, 1)
    assert (O[:, 4:6] == 0).all() and torch.isneginf(lse[:, 4:6]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_wide_pages_that_do_not_exist(cache, dtype):  # noqa: F811
    """Numbers outside the pool in the table: their slots are not seen and their weights are not written."""
    log("wide bad pages %s" % dtype)
    n, page = 2400, 16
    pool = Pool(cache, [n, 1300], 8, page, dtype, seed=35)
    gone = [s for s in range(n) if s // page in (0, 17, 70, 71, 72, 73, 149)]
    check(cache, pool, normal(13, (2600, 16, 64), dtype), [1300, 1300], True, 1, gone=gone)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_narrow_pages_that_do_not_exist(cache, dtype):  # noqa: F811
    """The same for few rows, whose logits are kept, and for more over few slots."""
    log("narrow bad pages %s" % dtype)
    for n, q in ((700, 1), (5000, 20), (700, 60 if dtype == BF else 30)):
        pool = Pool(cache, [n, 90], 1, 16, dtype, seed=36)
        gone = [s for s in range(n) if s // 16 in (2, 17, 43)]
        check(cache, pool, normal(13, (q + 1, 2, 64), dtype), [q, 1], True, 0, gone=gone)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_wide_large_logits(cache, dtype):  # noqa: F811
    """Sharp rows whose logits grow by far more than 41 past the first tile of a range, so that what the first
    reference holds leaves fp32's range and the range is done again with one that moves."""
    log("wide large logits %s" % dtype)
    n = 2400
    pool = Pool(cache, [n], 8, 64, dtype, seed=36, std=6.0)
    k = pool.k[0].clone()
    k[:64] *= 0.05
    k[1800:] *= 4
    pool.put(0, k, pool.v[0])

    def reach(b, h, x):
        assert (x.amax(dim=1) - x[:, :64].amax(dim=1) > 45).float().mean() > 0.9

    check(cache, pool, normal(14, (1300, 16, 64), dtype, 6.0), [1300], False, 1, reach=reach)
    check(cache, pool, normal(15, (1300, 16, 64), dtype, 6.0), [1300], True, 1, scale=0.25)


def test_attend_wide_bounds_and_streams(cache):  # noqa: F811
    """Bounds above the lengths, queries as a slice of a projection's output, another stream."""
    log("wide bounds, strides, streams")
    pool = Pool(cache, [2400, 700], 4, 32, BF, seed=37, cap=9000)
    qs = [1300, 60]
    x = normal(16, (1360, 24, 64), BF).cuda()
    check(cache, pool, x[:, 4:20], qs, True, 1, slack=6000)
    pc, batch = pool.cuda(), pool.batch(qs, slack=6000)
    a, la = cache.attend(pc, batch, x[:, 4:20])
    b, lb = cache.attend(pc, batch, x[:, 4:20].contiguous())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        d, ld = cache.attend(pc, batch, x[:, 4:20])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, b) and torch.equal(la, lb) and torch.equal(a, d) and torch.equal(la, ld)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_wide_graph_replays(cache, dtype):  # noqa: F811
    """A chunk's append and attention with weights as a graph: every replay gives the eager pass's result."""
    log("wide graph %s" % dtype)
    pool = Pool(cache, [2400, 1300], 8, 16, dtype, seed=40)
    qs = [1300, 700]
    pc, batch = pool.cuda(), pool.batch(qs, seen=[2500, 1300])
    Q, K, V = (normal(20 + i, (2000, h, 64), dtype).cuda() for i, h in enumerate((16, 8, 8)))
    assert cache.attend_plan(pc, batch, 16, 2000).shared == 1
    O, lse = torch.empty_like(Q), torch.empty(2000, 16, device="cuda")
    ws, W = cache.attend_workspace(pc, batch, 16, 2000), pool.W.cuda()
    W2, Qr = W.clone(), torch.empty_like(Q)

    def step():
        q = cache.append(pc, batch, Q, K, V, Q_out=Qr)
        cache.attend(pc, batch, q, True, O=O, lse=lse, weight_out=W2, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for r in range(3):
        if r == 2:
            Q.copy_(normal(60, Q.shape, dtype))
            K.copy_(normal(61, K.shape, dtype))
        step()
        want = [t.clone() for t in (O, lse, W2)]
        for t in (O, lse):
            t.fill_(float("nan"))
        W2.copy_(W)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (O, lse, W2)):
            assert torch.equal(a, b), r
        ws.random_(0, 255)     # the workspace holds nothing from call to call


# ------------------------------------------------------------------ eviction in six launches

def keep64(w, safe, keep):
    """Indices that stay: the protected ones, then NaN, then by weight; lower ones among equals."""
    n, nan = len(w), np.isnan(w)
    group = np.where(safe, 0, np.where(nan, 1, 2))
    order = np.lexsort((np.arange(n), np.where(group < 2, 0.0, -w.astype(np.float64)), group))
    return np.sort(order[:min(n, keep)])


def evict64(pool, seen, keep, sink, recent):
    """The pool after the eviction (CPU): (K, V, W, S, lengths)."""
    K, V, W, S = pool.K.clone(), pool.V.clone(), pool.W.clone(), pool.S.clone()
    left = [min(n, keep) for n in pool.lens]
    for b, n in enumerate(pool.lens):
        p, s = pool.at(b, n)
        for h in range(pool.Hkv):
            st = pool.S[p, h, s].numpy().astype(np.int64)
            kept = keep64(pool.W[p, h, s].numpy(), (st < sink) | (st >= seen[b] - recent), keep)
            src = torch.from_numpy(kept[kept >= left[b]])
            dst = torch.from_numpy(np.setdiff1d(np.arange(left[b]), kept))
            assert len(src) == len(dst)
            for x, y in ((K, pool.K), (V, pool.V), (W, pool.W), (S, pool.S)):
                x[p[dst], h, s[dst]] = y[p[src], h, s[src]]
    return K, V, W, S, left


# Past 40,960 slots: their keys do not fit the LDS of a workgroup.
LONG = [
    # lens, keep, sink, recent, Hkv, page, dtype, kind of weights
    ([45000, 700, 20481], 9001, 5, 257, 2, 64, BF, "ties"), ([45000, 700, 20481], 9001, 0, 0, 2, 16, F32, "odd"),
    ([43001], 43000, 0, 0, 3, 32, BF, "plain"), ([49152, 49152], 24576, 1374, 1374, 1, 128, BF, "equal"),
    ([50003, 0, 50003], 1, 0, 0, 1, 256, F32, "ties"), ([61440, 4096], 4096, 6000, 0, 1, 64, BF, "odd"),
    ([41001, 41001, 12000], 30005, 0, 35000, 2, 64, F32, "equal"), ([43000, 5], 43000, 2, 2, 1, 64, BF, "ties"),
]


def long_pool(c, lens, Hkv, page, dtype, kind, sink):
    from test_gpu_cache import weights_of
    pool = Pool(c, lens, Hkv, page, dtype, seed=70, junk=0.5)
    pool.W = weights_of(kind, pool.W.shape, 71)
    for b, n in enumerate(lens):
        p, s = pool.at(b, n)
        for h in range(Hkv):
            o = torch.randperm(n, generator=gen(72 + b + 10 * h))
            pool.S[p, h, s] = torch.where(o < sink, o, o + n // 2).to(torch.int32)
    return pool


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("lens,keep,sink,recent,Hkv,page,dtype,kind", LONG)
def test_evict_long(cache, lens, keep, sink, recent, Hkv, page, dtype, kind, in_place):  # noqa: F811
    log("evict long %s keep=%d sink=%d recent=%d %s" % (lens, keep, sink, recent, kind))
    pool = long_pool(cache, lens, Hkv, page, dtype, kind, sink)
    seen = [n + n // 2 for n in lens]
    pc, length = pool.cuda(), i32(lens)
    K, V, W, S, left = evict64(pool, seen, keep, sink, recent)
    ws = cache.evict_workspace(pc, len(lens), max(lens))
    ws.random_(0, 255)
    if in_place:
        wo, so, lo = pool.gW, pool.gS, length
        cache.evict(pc, pool.gtable, length, i32(seen), keep, max(lens), sink, recent, ws=ws)
    else:
        wo, so, lo = torch.full_like(pool.gW, 3.0), torch.full_like(pool.gS, -9), torch.zeros_like(length)
        cache.evict(pc, pool.gtable, length, i32(seen), keep, max(lens), sink, recent, wo, so, lo, ws)
        assert torch.equal(pool.gW.cpu().view(torch.int32), pool.W.view(torch.int32))
    assert lo.tolist() == left
    assert torch.equal(pool.gK.cpu(), K) and torch.equal(pool.gV.cpu(), V)
    wo, so, rest = wo.cpu(), so.cpu(), torch.ones(W.shape, dtype=torch.bool)
    for b, n in enumerate(left):
        p, s = pool.at(b, n)
        assert torch.equal(wo[p, :, s].view(torch.int32), W[p, :, s].view(torch.int32)), b
        assert torch.equal(so[p, :, s], S[p, :, s]), b
        rest[p, :, s] = False
    if not in_place:       # nothing but the slots that stay is written
        assert (wo[rest] == 3.0).all() and (so[rest] == -9).all()


def test_evict_long_graph_replays(cache):  # noqa: F811
    """Captured, with a workspace that holds something else before every replay."""
    log("evict long graph")
    lens, keep = [45000, 9000], 12000
    pool = long_pool(cache, lens, 2, 64, BF, "ties", 3)
    pc = pool.cuda()
    length, seen, lo = i32(lens), i32([n + n // 2 for n in lens]), i32([0, 0])
    wo, so, ws = pool.gW.clone(), pool.gS.clone(), cache.evict_workspace(pc, 2, 45000)
    go = lambda: cache.evict(pc, pool.gtable, length, seen, keep, 45000, 3, 64, wo, so, lo, ws)
    K, V, W, S, left = evict64(pool, seen.tolist(), keep, 3, 64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    for k in range(4):
        pool.gK.copy_(pool.K)
        pool.gV.copy_(pool.V)
        wo.fill_(3.0), so.fill_(-9), lo.zero_()
        ws.random_(0, 255)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool.gK.cpu(), K) and torch.equal(pool.gV.cpu(), V) and lo.tolist() == left, k
        for b, n in enumerate(left):
            p, s = pool.at(b, n)
            assert torch.equal(wo.cpu()[p, :, s], W[p, :, s]) and torch.equal(so.cpu()[p, :, s], S[p, :, s]), k


# ------------------------------------------------------------------ rotary positions past the caches

@pytest.mark.parametrize("T,H,dtype,dim,axes,layout", [
    (33001, 16, BF, 64, 2, "half"), (33001, 16, BF, 48, 1, "interleaved"), (17003, 16, F32, 64, 1, "interleaved"),
    (17003, 16, F32, 40, 1, "half"), (44001, 3, F32, 12, 1, "half"), (44001, 3, F32, 20, 2, "interleaved")])
def test_rotary_large(cache, T, H, dtype, dim, axes, layout):  # noqa: F811
    """Outputs of more than 64 MiB (bf16), 33 MiB: stored past the caches; the transpose in place, rows that
    lie apart and (fp32) start 16, not 32 bytes into one another's multiples."""
    from test_gpu_cache import radians, rot_tol, rotate64
    log("rotary large T=%d H=%d %s dim=%d %s" % (T, H, dtype, dim, layout))
    assert T * H * 64 * (2 if dtype == BF else 4) > 32 << 20
    rot = cache.Rotary.make(dim, 10000.0, axes, layout, "linear", 8.0)
    step = 16 // (2 if dtype == BF else 4)
    room = torch.zeros(T * (H * 64 + step) + step, dtype=dtype, device="cuda")
    x = room[step:].view(T, H * 64 + step)[:, :H * 64].unflatten(1, (H, 64))
    x.copy_(normal(T, (T, H, 64), dtype))
    pos = torch.randint(-(1 << 20), 1 << 20, (T, axes), generator=gen(T)).to(torch.int32).cuda()
    before = x.clone()
    f = radians(rot)
    ref = rotate64(before, pos, f, axes, layout, rot.mag)
    y = cache.rotary(x, pos, rot)
    assert ((y.double() - ref).abs() <= rot_tol(before, ref, rot.mag, dtype)).all()
    assert torch.equal(y[:, :, dim:], before[:, :, dim:]) and torch.equal(x, before)
    ref = rotate64(before, pos, f, axes, layout, rot.mag, -1.0)
    assert cache.rotary(x, pos, rot, out=x, transpose=True) is x
    assert ((x.double() - ref).abs() <= rot_tol(before, ref, rot.mag, dtype)).all()
    assert torch.equal(x[:, :, dim:], before[:, :, dim:])
    assert (room[:step] == 0).all() and (room[step:].view(T, -1)[:, H * 64:] == 0).all()
