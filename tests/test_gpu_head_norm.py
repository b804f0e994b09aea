"""Per-head norms with rotary positions on the GPU, and their gradients, against 64-bit computations on the CPU.

Tolerances (set before the first run), u = 2^-24, per row of 64 features.  S = max |x|, r = 1 / rms (eps included), N =
max |n|.  Mean: 11 roundings, so a centred value is off by 12 u S; rms relatively by 12 u S r + 16 u (the sum, a root, a
quotient); n by e_n = 24 u S r (1 + N) + 16 u N.  y, before the rotation, by |gain| e_n + 2 u (|gain| N + |bias|), and the rotation of a
pair doubles that and adds 12 u per feature.  Backward: h = R^T g by e_h = 24 u max |g|, z = h gain by
e_z = |gain| e_h + u Z, the two means by e_z + 12 u Z and N e_z + e_n Z + 12 u N Z, so with Z = max |z|
    |dx| is off by r ((2 + N^2) e_z + (2 N + 1) e_n Z + 32 u Z (1 + N^2)) + |dx| (12 u S r + 20 u).
Sums over R rows: each term by e_h N + max |h| e_n + u, and (64 + R / 256) u of the absolute sum for the chains of a
slot (R / 256 rows at most: 32 slots of 8 workgroups or more) and of a workgroup.  bf16 outputs: 2^-8 of the value more."""
import copy
import pickle

import numpy as np
import pytest
import torch

from paper_2609_23733_amd import synth, vp
from test_gpu_cache import BF, BFU, F32, U, _gpu, cache, gen, log, normal, radians, rotate64  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = [
    # T, H, dtype, kind, gain, dim, axes, layout
    (1, 1, F32, "layer", "shared", 64, 1, "half"), (1, 16, BF, "rms", "heads", 64, 1, "interleaved"),
    (13, 16, F32, "layer", "heads", 64, 2, "half"), (13, 3, F32, "rms", "none", 32, 1, "interleaved"),
    (257, 3, BF, "layer", "heads", 48, 1, "interleaved"), (77, 16, BF, "layer", "shared", 64, 2, "half"),
    (5, 4, F32, "rms", "shared", 12, 1, "half"), (5, 6, F32, "layer", "heads", 60, 2, "half"),
    (9, 2, BF, "layer", "shared", 24, 4, "interleaved"), (9, 2, F32, "rms", "heads", 6, 3, "half"),
    (33, 8, BF, "layer", "none", 10, 1, "interleaved"), (3, 128, BF, "rms", "heads", 2, 1, "half"),
    (70, 48, F32, "layer", "heads", 16, 1, "half"), (41, 33, F32, "rms", "heads", 64, 1, "half"),
    (300, 5, F32, "layer", "shared", 0, 1, "half"), (4099, 16, BF, "layer", "shared", 64, 1, "half"),
    (3001, 12, F32, "rms", "heads", 64, 1, "interleaved"), (20011, 16, BF, "rms", "heads", 32, 1, "half"),
]
IDS = ["T%d-H%d-%s-%s-%s-%d-%d-%s" % (c[0], c[1], "bf16" if c[2] is BF else "f32", *c[3:]) for c in CASES]


def inputs(T, H, dtype, kind, gain, dim, axes, seed=0):
    x = torch.randn(T, H, 64, generator=gen(T + H + seed))
    x = (x * torch.exp(0.5 * torch.randn(T, H, 1, generator=gen(seed + 1))) + 0.5).to(dtype)
    g = normal(seed + 2, (T, H, 64), dtype)
    shape = (H, 64) if gain == "heads" else (64,)
    ga = None if gain == "none" else 1 + 0.3 * torch.randn(*shape, generator=gen(seed + 3))
    bi = None if gain == "none" else 0.3 * torch.randn(*shape, generator=gen(seed + 4))
    pos = torch.randint(-(1 << 20), 1 << 20, (T, axes), generator=gen(seed + 5)).to(torch.int32)
    return x, g, ga, bi, pos


def spec(cache, dim, axes, layout):  # noqa: F811
    if dim:
        return cache.Rotary.make(dim, 10000.0, axes, layout, "parts", 8.0, 4096.0)
    return cache.Rotary(torch.zeros(0, dtype=torch.int64, device="cuda"), layout, axes, 1.0)


def forward64(x, ga, bi, pos, rot, kind, eps=1e-6):
    """(y, n, r, S) in 64 bits."""
    f = x.double()
    if kind == "layer":
        f = f - f.mean(dim=2, keepdim=True)
    r = 1 / torch.sqrt((f * f).mean(dim=2, keepdim=True) + eps)
    n = f * r
    v = n if ga is None else n * ga.double()
    v = v if bi is None else v + bi.double()
    y = v if rot is None else rotate64(v, pos, radians(rot), rot.axes, rot.layout, rot.mag)
    return y, n, r, x.double().abs().amax(dim=2, keepdim=True)


def backward64(g, n, r, ga, pos, rot, kind):
    """(dx, h, z)."""
    h = g.double() if rot is None else rotate64(g, pos, radians(rot), rot.axes, rot.layout, rot.mag, -1.0)
    z = h if ga is None else h * ga.double()
    dx = z - n * (z * n).mean(dim=2, keepdim=True)
    if kind == "layer":
        dx = dx - z.mean(dim=2, keepdim=True)
    return dx * r, h, z


def top(v):
    return v.abs().amax(dim=2, keepdim=True)


def tolerances(y, n, r, S, ga, bi, mag, dtype, g=None, dx=None, h=None, z=None):
    """(tol_y, tol_dx, tol of an h n term, tol of an h term)."""
    N = top(n)
    A = 1.0 if ga is None else ga.abs().max().item()
    B = 0.0 if bi is None else bi.abs().max().item()
    e_n = 24 * U * S * r * (1 + N) + 16 * U * N
    ty = mag * (2 * (A * e_n + 2 * U * (A * N + B)) + 24 * U * (A * N + B))
    bf = lambda t, v: t + (BFU * (v.abs() + t) if dtype == BF else 0) + 1e-30
    if g is None:
        return bf(ty, y)
    e_h = 24 * U * mag * top(g.double())
    Z = top(z)
    e_z = A * e_h + U * Z
    td = r * ((2 + N * N) * e_z + (2 * N + 1) * e_n * Z + 32 * U * Z * (1 + N * N)) + dx.abs() * (12 * U * S * r + 20 * U)
    return bf(ty, y), bf(td, dx), e_h * N + top(h) * e_n + U * top(h) * N, e_h


def check_sums(got, terms, term_tol, gain):
    over = (0,) if gain == "heads" else (0, 1)
    rows = terms.shape[0] * (1 if gain == "heads" else terms.shape[1])
    ref, size = terms.sum(dim=over), terms.abs().sum(dim=over)
    tol = (term_tol.expand(terms.shape).sum(dim=over)) + (64 + rows / 256) * U * size + 1e-30
    assert got.shape == ref.shape and got.dtype == F32
    err = (got.cpu().double() - ref).abs()
    assert (err <= tol).all(), (err.max().item(), (err / tol).max().item())


@pytest.mark.parametrize("T,H,dtype,kind,gain,dim,axes,layout", CASES, ids=IDS)
def test_norm_and_gradient(cache, T, H, dtype, kind, gain, dim, axes, layout):  # noqa: F811
    log("norm T=%d H=%d %s %s dim=%d axes=%d %s %s" % (T, H, kind, gain, dim, axes, layout, dtype))
    rot = spec(cache, dim, axes, layout)
    x, g, ga, bi, pos = inputs(T, H, dtype, kind, gain, dim, axes)
    dev = lambda t: None if t is None else t.cuda()
    X, GA, BI, POS = dev(x), dev(ga), dev(bi), dev(pos)
    y, n, r, S = forward64(x, ga, bi, pos, rot, kind)
    dx, h, z = backward64(g, n, r, ga, pos, rot, kind)
    mag = max(1.0, rot.mag)
    ty, td, tn, th = tolerances(y, n, r, S, ga, bi, mag, dtype, g, dx, h, z)
    norm = cache.HeadNorm(kind, GA, BI)
    plain = cache.norm_rotary(X, norm, POS, rot)
    err = (plain.cpu().double() - y).abs()
    assert (err <= ty).all(), err.max().item()
    leaves = [t.requires_grad_() for t in (X, GA, BI) if t is not None]
    out = cache.norm_rotary(X, norm, POS, rot)
    assert torch.equal(out.detach(), plain)
    d = torch.autograd.grad(out, leaves, g.cuda())
    err = (d[0].cpu().double() - dx).abs()
    assert d[0].dtype == dtype and (err <= td).all(), (err.max().item(), (err / td).max().item())
    if ga is not None:
        check_sums(d[1], h * n, tn, gain)
        check_sums(d[2], h, th, gain)
    again = torch.autograd.grad(cache.norm_rotary(X, norm, POS, rot), leaves, g.cuda())
    assert all(torch.equal(a, b) for a, b in zip(d, again))     # one order of all sums


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gradient_by_differences(cache, kind):  # noqa: F811
    """Along random directions of x, gain and bias: central differences of the kernel's own forward at steps s and
    s / 2, combined so that their s^2 error cancels; what is left is below the correction that this makes, and the
    forward's roundings over the step."""
    log("norm gradient by differences %s" % kind)
    T, H = 7, 4
    rot = cache.Rotary.make(64, 100.0, 2, "half")
    x, g, ga, bi, pos = inputs(T, H, F32, kind, "heads", 64, 2, seed=20)
    X, GA, BI, POS, G = (t.cuda() for t in (x, ga, bi, pos, g))
    leaves = [t.clone().requires_grad_() for t in (X, GA, BI)]
    d = torch.autograd.grad(cache.norm_rotary(leaves[0], cache.HeadNorm(kind, leaves[1], leaves[2]), POS, rot), leaves, G)
    r = top(X.double()).cpu() / forward64(x, ga, bi, pos, rot, kind)[2]

    def loss(v, a, b):
        return (cache.norm_rotary(v, cache.HeadNorm(kind, a, b), POS, rot).double() * G.double()).sum().item()

    for trial in range(6):
        for i, base in enumerate((X, GA, BI)):
            w = torch.randn(base.shape, generator=gen(100 + 3 * trial + i)).cuda()
            args = lambda s: [t + s * w if j == i else t for j, t in enumerate((X, GA, BI))]
            D = lambda s: (loss(*args(s)) - loss(*args(-s))) / (2 * s)
            step = 2.0 ** -5
            one, half = D(step), D(step / 2)
            best = (4 * half - one) / 3
            want = (d[i].double() * w.double()).sum().item()
            y = forward64(x, ga, bi, pos, rot, kind)
            ty = tolerances(*y, ga, bi, 1.0, F32)
            # (inputs base + s w are rounded as well: u of them, through a derivative of at most |d|)
            noise = 2 * ((ty * g.double().abs()).sum().item() + (U * (base.abs() + w.abs()).double() * d[i].abs().double()).sum().item()) / step
            assert abs(best - want) <= abs(best - half) + noise, (trial, i, best, want)


def test_strides_in_place_and_empty(cache):  # noqa: F811
    log("norm strides")
    rot = cache.Rotary.make(32, 10000.0, 1, "interleaved")
    norm = cache.HeadNorm("layer", 1 + normal(1, (64,), F32).cuda(), normal(2, (64,), F32).cuda())
    fused = normal(6, (41, 10, 64), BF).cuda()
    pos = torch.arange(41, dtype=torch.int32, device="cuda")[:, None]
    a = cache.norm_rotary(fused[:, 2:7], norm, pos, rot)
    b = cache.norm_rotary(fused[:, 2:7].contiguous(), norm, pos, rot)
    assert torch.equal(a, b)
    whole = fused.clone()
    cache.norm_rotary(whole[:, 2:7], norm, pos, rot, out=whole[:, 2:7])
    assert torch.equal(whole[:, 2:7], b)
    assert torch.equal(whole[:, :2], fused[:, :2]) and torch.equal(whole[:, 7:], fused[:, 7:])
    assert cache.norm_rotary(fused[:0, 2:7], norm, pos[:0], rot).shape == (0, 5, 64)
    none = cache.norm_rotary(fused[:, 2:7], norm)                 # without positions
    zero = cache.norm_rotary(fused[:, 2:7], norm, torch.zeros_like(pos), rot)
    assert torch.equal(none, zero)
    # gradients of a strided leaf, from a broadcast gradient, and of no rows
    x = fused[:, 2:7].detach().requires_grad_()
    ga, bi = norm.gain.clone().requires_grad_(), norm.bias.clone().requires_grad_()
    n2 = cache.HeadNorm("layer", ga, bi)
    d = torch.autograd.grad(cache.norm_rotary(x, n2, pos, rot).sum(), [x, ga, bi])
    xc = fused[:, 2:7].contiguous().requires_grad_()
    e = torch.autograd.grad(cache.norm_rotary(xc, n2, pos, rot), [xc, ga, bi], torch.ones(41, 5, 64, dtype=BF, device="cuda"))
    assert all(torch.equal(p, q) for p, q in zip(d, e))
    empty = fused[:0, 2:7].detach().requires_grad_()
    d = torch.autograd.grad(cache.norm_rotary(empty, n2, pos[:0], rot).sum(), [empty, ga, bi])
    assert d[0].shape == (0, 5, 64) and (d[1] == 0).all() and (d[2] == 0).all()
    # only some of the gradients asked for
    d = torch.autograd.grad(cache.norm_rotary(fused[:, 2:7], n2, pos, rot), [ga], torch.ones(41, 5, 64, dtype=BF, device="cuda"))
    assert torch.equal(d[0], e[1])
    n3 = cache.HeadNorm("layer", norm.gain, norm.bias)
    d = torch.autograd.grad(cache.norm_rotary(x, n3, pos, rot), [x], torch.ones(41, 5, 64, dtype=BF, device="cuda"))
    assert torch.equal(d[0], e[0])


def test_refusals(cache):  # noqa: F811
    x = normal(1, (3, 4, 64), BF).cuda()
    pos = torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    rot = cache.Rotary.make(64)
    f = lambda *s: torch.ones(*s, device="cuda")
    for bad in (f(32), f(2, 2, 64), f(64).to(BF), f(64, 64)[:, 0], f(65)[1:]):
        with pytest.raises(ValueError):
            cache.HeadNorm("layer", bad)
    with pytest.raises(ValueError):
        cache.HeadNorm("layer", f(64), f(4, 64))
    with pytest.raises(ValueError, match="heads"):
        cache.norm_rotary(x, cache.HeadNorm("rms", f(3, 64)), pos, rot)
    n = cache.HeadNorm("rms", f(64).requires_grad_())
    for args in ((x, n, pos), (x, n, None, rot), (x, n, pos[:2], rot), (x.to(torch.float16), n, pos, rot),
                 (x[:, :, :32], n, pos, rot), (x.transpose(0, 1), n, pos, rot)):
        with pytest.raises((ValueError, TypeError)):
            with torch.no_grad():
                cache.norm_rotary(*args)
    with pytest.raises(ValueError, match="graph"):
        cache.norm_rotary(x, n, pos, rot, out=torch.empty_like(x))
    # a second derivative, and inputs changed between forward and backward
    xg = x.float().requires_grad_()
    y = cache.norm_rotary(xg, n, pos, rot)
    d, = torch.autograd.grad(y.sum(), xg, create_graph=True)
    with pytest.raises(RuntimeError):
        d.sum().backward()
    y = cache.norm_rotary(xg, n, pos, rot)
    with torch.no_grad():
        n.gain.add_(1.0)
    with pytest.raises(RuntimeError):
        y.sum().backward()


def test_parameters_whose_storage_changes(cache):  # noqa: F811
    """A gain that gets other memory after the norm was made (as moving a module does) is read from there."""
    x = normal(1, (5, 4, 64), F32).cuda()
    gain = torch.nn.Parameter(torch.ones(64, device="cuda"))
    norm = cache.HeadNorm("rms", gain)
    one = cache.norm_rotary(x, norm).detach()
    gain.data = torch.full((4, 64), 2.0, device="cuda")
    two = cache.norm_rotary(x, norm)
    assert torch.equal(two.detach(), 2 * one) and norm.heads == 4
    two.sum().backward()
    assert gain.grad.shape == (4, 64)
    gain.data = torch.ones(3, 64, device="cuda")
    with pytest.raises(ValueError, match="heads"):
        cache.norm_rotary(x, norm)
    gain.data = torch.ones(32, device="cuda")
    with pytest.raises(ValueError):
        cache.norm_rotary(x, norm)


def test_copies(cache):  # noqa: F811
    """A copied module's norm has the copy's parameters."""
    class Heads(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.gain = torch.nn.Parameter(torch.full((64,), 2.0, device="cuda"))
            self.norm = cache.HeadNorm("rms", self.gain, None, 1e-5)

    one = Heads()
    two = copy.deepcopy(one)
    assert two.norm.gain is two.gain and two.gain is not one.gain and (two.norm.kind, two.norm.eps) == ("rms", 1e-5)
    x = normal(1, (5, 4, 64), F32).cuda()
    with torch.no_grad():
        two.gain.fill_(4.0)
        assert torch.equal(cache.norm_rotary(x, two.norm), 2 * cache.norm_rotary(x, one.norm))
        back = pickle.loads(pickle.dumps(cache.HeadNorm("layer", torch.ones(4, 64, device="cuda"))))
        assert torch.equal(cache.norm_rotary(x, back), cache.norm_rotary(x, cache.HeadNorm("layer")))


def test_parameters_exchanged_before_the_gradient(cache):  # noqa: F811
    """A graph's gradients are of the gain and bias of its forward pass, whatever the norm holds by then."""
    rot = cache.Rotary.make(64)
    pos = torch.arange(9, dtype=torch.int32, device="cuda")[:, None]
    x = normal(1, (9, 4, 64), F32).cuda().requires_grad_()
    leaf = lambda s, *sh: (1 + normal(s, sh, F32).cuda()).requires_grad_()
    ga, bi, g = leaf(2, 4, 64), leaf(3, 4, 64), normal(4, (9, 4, 64), F32).cuda()
    step = lambda n: cache.norm_rotary(x, n, pos, rot)
    want = torch.autograd.grad(step(cache.HeadNorm("layer", ga, bi)), [x, ga, bi], g)
    same = lambda d: all(torch.equal(p, q) for p, q in zip(d, want))
    norm = cache.HeadNorm("layer", ga, bi)
    y = step(norm)
    norm.gain, norm.bias = leaf(5, 4, 64), None
    other = step(norm)
    assert same(torch.autograd.grad(y, [x, ga, bi], g))
    assert not torch.equal(torch.autograd.grad(other, [x], g)[0], want[0])
    # other sizes at the same address
    norm = cache.HeadNorm("layer", ga, bi)
    y = step(norm)
    norm.gain, norm.bias = ga.detach()[0], bi.detach()[0]
    one = step(norm).detach()
    assert torch.equal(one, step(cache.HeadNorm("layer", ga.detach()[0].clone(), bi.detach()[0].clone())).detach())
    assert same(torch.autograd.grad(y, [x, ga, bi], g))
    norm.gain, norm.bias = ga.detach()[:3], bi.detach()[:3]
    with pytest.raises(ValueError, match="heads"):
        step(norm)
    # copies that the graph kept on the host
    norm = cache.HeadNorm("layer", ga, bi)
    with torch.autograd.graph.save_on_cpu():
        y = step(norm)
    with torch.no_grad():
        ga.add_(1.0)
    assert same(torch.autograd.grad(y, [x, ga, bi], g))
    for name in ("kind", "eps"):
        with pytest.raises(AttributeError):
            setattr(norm, name, 1)


def test_rows_that_are_not_finite_or_tiny(cache):  # noqa: F811
    """A NaN or an infinity stays in its row; rows of zeros give the bias, of equal values (layer) too."""
    x = normal(3, (40, 3, 64), F32)
    x[3, 1, 7], x[5, 2, 63], x[9, 0] = float("nan"), float("inf"), 0.0
    x[11, 1], x[12, 1] = 3.0, 1e-30
    bi = normal(4, (64,), F32)
    for kind in ("layer", "rms"):
        y = cache.norm_rotary(x.cuda(), cache.HeadNorm(kind, None, bi.cuda())).cpu()
        odd = torch.zeros(40, 3, dtype=torch.bool)
        odd[3, 1] = odd[5, 2] = True
        assert torch.isnan(y[odd]).any(dim=1).all() and torch.isfinite(y[~odd]).all()
        assert torch.equal(y[9, 0], bi)
        assert (y[12, 1] - bi).abs().max() <= 1e-24
        if kind == "layer":
            assert torch.equal(y[11, 1], bi)


def test_graph_of_a_training_step(cache):  # noqa: F811
    """Forward and backward captured once and replayed between eager work on other inputs."""
    log("norm training step in a graph")
    rot = cache.Rotary.make(64)
    pos = torch.arange(300, dtype=torch.int32, device="cuda")[:, None]
    x = normal(1, (300, 4, 64), BF).cuda().requires_grad_()
    ga = torch.ones(64, device="cuda").requires_grad_()
    bi = torch.zeros(64, device="cuda").requires_grad_()
    norm, g = cache.HeadNorm("layer", ga, bi), normal(2, (300, 4, 64), BF).cuda()

    def step():
        y = cache.norm_rotary(x, norm, pos, rot)
        return [y.detach()] + list(torch.autograd.grad(y, [x, ga, bi], g))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        with torch.no_grad():
            x.copy_(normal(10 + k, (300, 4, 64), BF))
            ga.copy_(1 + 0.1 * normal(20 + k, (64,), F32))
        graph.replay()
        got = [t.clone() for t in out]
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b), k


def test_saved_inputs_that_the_operators_overwrite(cache):  # noqa: F811
    """The library writes through addresses; a backward pass that saved what was overwritten refuses, as after torch's
    own in-place operations."""
    bf = lambda s, *shape: normal(s, shape, BF).cuda()
    pos = torch.arange(6, dtype=torch.int32, device="cuda")[:, None]
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    rot, other = cache.Rotary.make(64), cache.HeadNorm("rms")
    mk = lambda dt: cache.PagedCache.empty(2, 16, 16, dtype=dt)
    k = bf(2, 6, 16, 64)
    w = synth.make_block_weights((1, 0))
    w = {n: t.cuda() for n, t in w.items()}
    ws = torch.empty(vp.block_workspace_bytes(1, 6), dtype=torch.uint8, device="cuda")
    X, pos2 = bf(3, 6, 1024), torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    batch = cache.Batch(i32(0, 1)[None], i32(6), i32(0, 6), 6, 6, i32(6))

    def both(call):
        return [lambda x, pc=mk(dt): call(pc, x) for dt in (BF, torch.int8)]

    writers = [lambda x: cache.norm_rotary(x, other, out=x), lambda x: cache.rotary(x, pos, rot, out=x)]
    writers += both(lambda pc, x: cache.append(pc, batch, x, k, k, Q_out=x))
    writers += both(lambda pc, x: cache.attend(pc, batch, x, O=x))
    writers += both(lambda pc, x: cache.read(pc, batch, 6, K_out=x))
    writers += both(lambda pc, x: cache.read(pc, batch, 6, V_out=x))
    writers += [lambda x, i=i: vp.block_qkv(X, pos2, w, 1, 6, ws, *[x if j == i else None for j in range(3)]) for i in range(3)]
    writers += [lambda x: vp.block_out(X, k, w, 1, 6, ws, X_out=x.view(6, 1024))]
    for n, write in enumerate(writers):
        gain = torch.ones(64, device="cuda").requires_grad_()
        x = bf(1, 6, 16, 64)
        y = cache.norm_rotary(x, cache.HeadNorm("rms", gain), pos, rot)
        with torch.no_grad():
            write(x)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
        log("writer %d" % n)
    # positions and frequencies, which the gradient needs as the forward pass had them
    for call in (lambda x: cache.norm_rotary(x, cache.HeadNorm("rms"), pos, rot), lambda x: cache.rotary(x, pos, rot)):
        for t in (pos, rot.freq):
            x = bf(1, 6, 16, 64).requires_grad_()
            y = call(x)
            t.add_(1)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.sum().backward()
    # what the cache's own tensors are saved for
    for dt in (F32, torch.int8):
        pc = cache.PagedCache.empty(2, 16, 16, dtype=dt, rows=F32)
        for name in ("K", "V", "weight", "stamp", "scale"):
            t = getattr(pc, name)
            if t is None:
                continue
            before = t._version
            cache.append(pc, batch, None, k.float(), k.float())
            assert t._version > before, name
            before = t._version
            cache.evict(pc, batch.table, i32(6), i32(6), 3, 6)
            assert t._version > before, name
        before = pc.weight._version
        cache.attend(pc, batch, k.float(), weight_out=pc.weight)
        assert pc.weight._version > before
        lse = torch.empty(6, 16, device="cuda")
        before = lse._version
        cache.attend(pc, batch, k.float(), lse=lse)
        assert lse._version > before


def test_forward_mode_is_refused(cache):  # noqa: F811
    """Dual tensors, with and without requires_grad: nothing computes their tangents."""
    from torch.autograd import forward_ad
    pos = torch.arange(6, dtype=torch.int32, device="cuda")[:, None]
    rot, norm = cache.Rotary.make(64), cache.HeadNorm("rms", torch.ones(64, device="cuda"))
    x = normal(1, (6, 4, 64), F32).cuda()
    calls = [lambda x, n: cache.norm_rotary(x, n, pos, rot), lambda x, n: cache.norm_rotary(x, n),
             lambda x, n: cache.norm_rotary(x, n, out=torch.empty_like(x)), lambda x, n: cache.rotary(x, pos, rot)]
    for call in calls:
        with forward_ad.dual_level():
            call(x, norm)                                     # (no dual among them)
            for leaf in (x, x.clone().requires_grad_()):
                with pytest.raises((ValueError, RuntimeError, NotImplementedError)):
                    call(forward_ad.make_dual(leaf, torch.ones_like(x)), norm)
            with torch.no_grad(), pytest.raises(ValueError, match="forward-mode"):
                call(forward_ad.make_dual(x, torch.ones_like(x)), norm)
        call(x, norm)
    with forward_ad.dual_level():
        for name in ("gain", "bias"):
            t = torch.ones(64, device="cuda")
            with pytest.raises(ValueError, match="forward-mode"):
                cache.norm_rotary(x, cache.HeadNorm("layer", **{name: forward_ad.make_dual(t, t)}))
    # a dual gradient that comes back to the operators
    for call in calls[:2] + calls[3:]:
        leaf = x.clone().requires_grad_()
        y = call(leaf, norm)
        with forward_ad.dual_level():
            with pytest.raises(ValueError, match="forward-mode"):
                torch.autograd.grad(y, leaf, forward_ad.make_dual(torch.ones_like(x), x))


@pytest.mark.parametrize("dim", [None, 32, 10])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_infinities_past_the_turned_features(cache, dim, layout):  # noqa: F811
    """A bias, or a gradient, that is infinite in a feature that is not turned stays in it."""
    pos = torch.arange(7, dtype=torch.int32, device="cuda")[:, None]
    turn = () if dim is None else (pos, cache.Rotary.make(dim, layout=layout))
    bias = torch.zeros(64)
    bias[63], bias[40] = float("inf"), float("-inf")
    norm = cache.HeadNorm("layer", None, bias.cuda().requires_grad_())
    x, g = normal(1, (7, 3, 64), F32).cuda(), normal(2, (7, 3, 64), F32)
    g[2, 1, 62] = float("inf")
    y = cache.norm_rotary(x, norm, *turn)
    odd = torch.zeros(64, dtype=torch.bool)
    odd[63] = odd[40] = True
    assert torch.equal(torch.isinf(y.cpu()), odd.expand(7, 3, 64)) and not torch.isnan(y).any()
    d, = torch.autograd.grad(y, norm.bias, g.cuda())
    assert torch.isposinf(d[62]) and torch.isfinite(d).sum() == 63


def test_parameters_exchanged_for_others_at_their_address(cache):  # noqa: F811
    """Of as many elements, but of another shape, other strides or another type."""
    x = normal(1, (5, 4, 64), F32).cuda()
    G = (1 + normal(2, (64, 64), F32)).cuda()
    fresh = lambda g: cache.norm_rotary(x, cache.HeadNorm("rms", g))
    norm = cache.HeadNorm("rms", G[:1])
    with pytest.raises(ValueError, match="heads"):
        cache.norm_rotary(x, norm)                            # (one head's gain)
    norm.gain = G[0]
    assert torch.equal(cache.norm_rotary(x, norm), fresh(G[0].clone()))
    norm.gain = G[:1]
    with pytest.raises(ValueError, match="heads"):
        cache.norm_rotary(x, norm)
    for bad in (G[:, 0], G[0].view(torch.int32)):
        norm = cache.HeadNorm("rms", G[0])
        norm.gain = bad
        with pytest.raises(ValueError):
            cache.norm_rotary(x, norm)
        norm.gain, norm.bias = G[0], bad
        with pytest.raises(ValueError):
            cache.norm_rotary(x, norm)
        norm.bias = None
        assert torch.equal(cache.norm_rotary(x, norm), fresh(G[0].clone()))
