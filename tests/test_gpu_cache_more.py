"""More of the paged key-value cache on the GPU against the 64-bit computations of test_gpu_cache.py, with
its tolerances: u = 2^-24, a row's E, one bf16 rounding up to 2^-8 of a value."""
import numpy as np
import pytest
import torch

from paper_2609_23733_amd import vp
from test_gpu_cache import BF, BFU, F32, U, Pool, _gpu, attend64, cache, check_attend, gen, log, normal  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,dtype,causal", [
    ([200], [1], 2, 2, 16, BF, True), ([9000, 40], [1, 1], 4, 1, 64, BF, True), ([9000, 40], [1, 1], 4, 1, 64, F32, True),
    ([700], [40], 2, 1, 32, F32, True), ([700], [130], 2, 2, 32, BF, True), ([2000, 300], [150, 90], 2, 2, 16, F32, True),
    ([40000], [1], 1, 1, 256, BF, True), ([1374, 1374], [1374, 1374], 8, 8, 64, BF, False)])
def test_attend_values_near_the_largest(cache, lens, qs, Hq, Hkv, page, dtype, causal):  # noqa: F811
    """Values of 1e38 to 3e38 under flat logits: sums of them pass fp32's range, their means do not."""
    log("attend large values %s %s %s" % (lens, qs, dtype))
    pool = Pool(cache, lens, Hkv, page, dtype, seed=820 + sum(lens))
    for b, n in enumerate(lens):
        v = (1e38 + 2e38 * torch.rand(n, Hkv, 64, generator=gen(b))) * torch.tensor([1.0, -1.0]).repeat(32)
        v[:, :, :4] = normal(821 + b, (n, Hkv, 4), F32).clamp(-3, 3) * 1e38     # of either sign in the first features
        pool.put(b, pool.k[b], v.to(dtype))
    check_attend(cache, pool, normal(822, (sum(qs), Hq, 64), dtype), qs, causal)


@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,causal", [
    ([3], [1], 16, 16, 16, True), ([40, 31, 64], [1, 1, 1], 16, 4, 16, True), ([300], [1], 16, 16, 64, True),
    ([90, 5, 200, 0], [1, 1, 0, 0], 16, 8, 32, False), ([120], [20], 3, 1, 64, True), ([64, 257], [33, 1], 2, 2, 16, False)])
def test_attend_bf16_rows_to_the_outputs_rounding(cache, lens, qs, Hq, Hkv, page, causal):  # noqa: F811
    """Up to 64 rows of a key head: the probabilities of the value product as sums of two bf16 values, each within
    2^-16, so that beside fp32's errors only the output's rounding is left."""
    log("attend bf16 two parts %s %s" % (lens, qs))
    pool = Pool(cache, lens, Hkv, page, BF, seed=800 + sum(lens))
    Q = normal(801, (sum(qs), Hq, 64), BF)
    O, _ = cache.attend(pool.cuda(), pool.batch(qs), Q.cuda(), causal)
    O, t = O.cpu().double().numpy(), 0
    for b, m in enumerate(qs):
        n = pool.lens[b]
        vis = np.clip(n - m + np.arange(m) + 1, 0, n) if causal else np.full(m, n)
        for h in range(Hq if m else 0):
            ro, rl, _, A, X = attend64(Q[t:t + m, h], pool.k[b][:, h * Hkv // Hq], pool.v[b][:, h * Hkv // Hq], vis)
            E = (64 * X + n / 16 + 16 + np.abs(rl)) * U
            tol = (2 * E[:, None] + 2.0 ** -16) * A
            tol += BFU * (np.abs(ro) + tol)
            assert (np.abs(O[t:t + m, h] - ro) <= tol).all(), (b, h)
        t += m


@pytest.mark.parametrize("lens,qs,H,page,dtype", [
    ([70], [2], 2, 16, BF), ([5000, 3], [1, 1], 2, 64, BF), ([5000, 3], [1, 1], 2, 64, F32), ([700], [130], 2, 32, F32),
    ([1374, 1374], [1374, 1374], 8, 64, BF)])
def test_attend_only_logits_of_minus_infinity_over_any_values(cache, lens, qs, H, page, dtype):  # noqa: F811
    """A row whose logits are all -inf gives zeros, also where the values are not finite; the other heads' rows
    are not touched."""
    log("attend -inf logits over NaN values %s %s %s" % (lens, qs, dtype))
    pool = Pool(cache, lens, H, page, dtype, seed=840 + sum(lens))
    Q = normal(841, (sum(qs), H, 64), dtype)
    Q[:, 0, 2] = 1.0
    for b, n in enumerate(lens):
        k, v = pool.k[b].clone(), pool.v[b].clone()
        k[:, 0, 2] = float("-inf")
        v[::3, 0], v[1::3, 0] = float("nan"), float("inf")
        pool.put(b, k, v)
    O, lse = cache.attend(pool.cuda(), pool.batch(qs), Q.cuda(), True)
    assert (O[:, 0] == 0).all() and torch.isneginf(lse[:, 0]).all()
    assert torch.isfinite(O[:, 1:]).all() and torch.isfinite(lse[:, 1:]).all()


# ------------------------------------------------------------------ the stream layer

def test_stream_layer_refuses_other_heads_and_idle_positions(cache):  # noqa: F811
    """Queries of another number of heads, also one that the key heads divide, and positions that nothing would
    turn; the layer stays as it was.  Numbers that no step could work with are refused when the layer is made."""
    log("stream layer refusals")
    layer = cache.StreamLayer(1, keep=60, max_chunk=40, Hq=4, Hkv=2, page=16)
    Q, K, V = (normal(860 + i, (20, h, 64)).cuda() for i, h in enumerate((8, 2, 2)))
    pos = torch.arange(20, dtype=torch.int32, device="cuda")[:, None]
    layer.step(Q[:, :4], K, V)
    state = lambda: [t.view(torch.uint8).clone() for t in (layer.pc.K, layer.pc.V, layer.pc.weight, layer.pc.stamp)]
    held = state()     # (as bytes: slots not in use may hold NaN)
    for bad in (Q[:, :2], Q, Q[:, :6]):
        with pytest.raises(ValueError, match="heads"):
            layer.step(bad, K, V)
    with pytest.raises(ValueError, match="rot"):
        layer.step(Q[:, :4], K, V, pos)
    assert layer.lens == [20] and layer.length.tolist() == [20] and layer.seen.tolist() == [20]
    assert all(torch.equal(a, b) for a, b in zip(held, state()))
    for bad in (dict(keep=0), dict(max_chunk=0), dict(sink=-1), dict(recent=-1), dict(Hq=6, Hkv=4), dict(Hq=2, Hkv=4), dict(B=0)):
        with pytest.raises(ValueError):
            cache.StreamLayer(**dict(dict(B=1, keep=60, max_chunk=40, Hq=4, Hkv=2, page=16), **bad))


def test_append_refuses_positions_without_rotation(cache):  # noqa: F811
    log("append positions without rotation")
    pool = Pool(cache, [40], 2, 16, BF, seed=870)
    pc, x = pool.cuda(), normal(871, (5, 2, 64)).cuda()
    with pytest.raises(ValueError, match="rot"):
        cache.append(pc, pool.batch([5], [40]), x, x, x, pos=torch.zeros(5, 1, dtype=torch.int32, device="cuda"))


def test_stream_layer_does_not_wait(cache):  # noqa: F811
    """A step is enqueued without waiting for the stream, with equal chunks and others, with and without an
    eviction, and its results do not depend on how far ahead the host is."""
    log("stream layer does not wait")
    rot = cache.Rotary.make(64, 10000.0)
    steps = []
    for i, counts in enumerate([[30, 10], [20, 20], [7, 33], [40, 1], None, [1, 1]]):
        T = 40 if counts is None else sum(counts)
        x = [normal(880 + 3 * i + j, (T, 4, 64)).cuda() for j in range(3)]
        steps.append((x, torch.arange(T, dtype=torch.int32, device="cuda")[:, None], counts))
    ahead, waiting = (cache.StreamLayer(2, keep=60, max_chunk=40, Hq=4, page=16, rot=rot) for _ in range(2))
    for x, pos, counts in steps[:2]:      # (workspaces grow in the first steps)
        assert torch.equal(ahead.step(*x, pos, counts), waiting.step(*x, pos, counts))
    busy = normal(879, (4096, 4096)).cuda()
    torch.cuda.synchronize()
    for _ in range(8):
        busy = busy @ busy
    torch.cuda.set_sync_debug_mode("error")
    try:
        got = [ahead.step(*x, pos, counts) for x, pos, counts in steps[2:]]
    finally:
        torch.cuda.set_sync_debug_mode("default")
    for (x, pos, counts), O in zip(steps[2:], got):
        want = waiting.step(*x, pos, counts)
        torch.cuda.synchronize()
        assert torch.equal(O, want)


# ------------------------------------------------------------------ rotary

@pytest.mark.parametrize("dtype,layout,axes", [(F32, "half", 2), (BF, "interleaved", 1)])
@pytest.mark.parametrize("transpose", [False, True])
def test_rotary_in_a_graph(cache, dtype, layout, axes, transpose):  # noqa: F811
    """An input that requires gradients gets the transposed map of the output's, also of one that is
    broadcast or lies apart, and the gradient's gradient; `out` would leave the graph and is refused."""
    log("rotary in a graph %s %s" % (dtype, layout))
    rot = cache.Rotary.make(32, 100.0, axes, layout, "parts", 4.0, 64.0)
    pos = torch.randint(0, 500, (9, axes), generator=gen(890)).to(torch.int32).cuda()
    fused = normal(891, (9, 6, 64), dtype).cuda().requires_grad_()
    x = fused[:, 1:4]
    g = normal(892, (9, 6, 64), dtype).cuda()[:, 2:5]
    y = cache.rotary(x, pos, rot, transpose=transpose)
    with torch.no_grad():
        assert torch.equal(y, cache.rotary(x, pos, rot, transpose=transpose)) and y.requires_grad
        want = cache.rotary(g, pos, rot, transpose=not transpose)
        ones = cache.rotary(torch.ones_like(y), pos, rot, transpose=not transpose)
    dx, = torch.autograd.grad(y, fused, g, retain_graph=True)
    assert torch.equal(dx[:, 1:4], want) and (dx[:, :1] == 0).all() and (dx[:, 4:] == 0).all()
    odd = torch.empty(g.numel() + 1, dtype=dtype, device="cuda")[1:].view_as(g).copy_(g)
    dx, = torch.autograd.grad(y, fused, odd, retain_graph=True)
    assert torch.equal(dx[:, 1:4], want)
    dx, = torch.autograd.grad(y.float().sum(), fused, retain_graph=True)
    assert torch.equal(dx[:, 1:4], ones)
    h = g.detach().clone().requires_grad_()
    dx, = torch.autograd.grad(y, fused, h, create_graph=True)
    dh, = torch.autograd.grad(dx[:, 1:4], h, g)
    with torch.no_grad():
        assert torch.equal(dh, cache.rotary(g, pos, rot, transpose=transpose))
    for kw in (dict(x=x, out=torch.empty_like(y).detach()), dict(x=x.detach(), out=h)):
        with pytest.raises(ValueError, match="gradient"):
            cache.rotary(pos=pos, rot=rot, **kw)


@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,dtype", [
    ([300, 40], [1, 20], 4, 2, 16, BF), ([300, 40], [1, 20], 4, 2, 16, F32), ([9000], [1], 4, 2, 64, BF),
    ([2500], [2000], 64, 16, 16, BF), ([700], [130], 2, 2, 32, F32)])
def test_attend_into_its_queries(cache, lens, qs, Hq, Hkv, page, dtype):  # noqa: F811
    """O may be Q; with weights, whose logits may be formed again, it is refused."""
    log("attend O is Q %s %s %s" % (lens, qs, dtype))
    pool = Pool(cache, lens, Hkv, page, dtype, seed=900 + sum(lens))
    pc, batch, Q = pool.cuda(), pool.batch(qs), normal(901, (sum(qs), Hq, 64), dtype).cuda()
    want, lse = cache.attend(pc, batch, Q)
    with pytest.raises(vp.VPError):
        cache.attend(pc, batch, Q, O=Q, weight_out=pc.weight)
    got, l2 = cache.attend(pc, batch, Q, O=Q)
    assert got is Q and torch.equal(got, want) and torch.equal(lse, l2)
