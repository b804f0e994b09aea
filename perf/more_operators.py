"""Heads normalised and rotated in one pass, and the paged key-value cache held in 8 bits: real sizes.

Views of P = 1,374 tokens with 16 heads of 64 (or single tokens) arrive in a paged cache whose keys
and values take a byte each: codes [pages, Hkv, page, 64], int8 or fp8 (e4m3), and per slot and key
head two scales in bf16, [pages, Hkv, page, 2], the key's and the value's.  A scale is the smallest
power of two for which the row's largest value stays within the largest code (127 or 448), at least 2^-100,
so code times scale is a bf16 value.  Codes are rounded to the nearest, ties to even.  Five operators:

  norm       queries or keys of every head normalised over their 64 features (mean and variance, or the mean
             square alone), with a gain and a bias, and turned by their positions
  norm_grad  a training step through it: the output, and the gradients of input, gain and bias
  append     a chunk of new tokens: Q and K normalised and turned, K and V quantised into the
             sequences' last slots; the chunk read back as the cache now holds it
  attend     softmax attention of the chunk's queries over the 8-bit slots (grouped heads, causal or
             whole chunks), the log-sum-exp of every row, and where asked the attention weights added to
             the slots they fall on
  read       the last slots of every sequence as plain rows in bf16 or fp32

A case is a dict of plain values; the lengths of a batch follow from `B`, `q`, `len` and `mix`.
"""
import math
import random

import numpy as np
import torch

own = False

D = 64
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
LARGEST = {"int8": 127.0, "e4m3": 448.0}
EPS = 1e-6


def listed():
    return [
        # queries of a few single tokens, fp32: the smallest call, latency only
        dict(name="norm_tokens", op="norm", T=13, H=16, dtype="f32", kind="layer", gain="shared", fused=False,
             dim=64, axes=1, layout="half", span=4096),
        # the keys of eight views, part of one projection's output: 2D positions of their patches
        dict(name="norm_views", op="norm", T=10992, H=16, dtype="bf16", kind="layer", gain="shared", fused=True,
             dim=64, axes=2, layout="half", span=38),
        # training in fp32 on one view: mean squares, a gain for every head, part of the head turned
        dict(name="norm_grad_view_f32", op="norm_grad", T=1374, H=16, dtype="f32", kind="rms", gain="heads",
             fused=False, dim=48, axes=1, layout="interleaved", span=100000),
        # training on a scene of 32 views: the ordinary large call
        dict(name="norm_grad_views", op="norm_grad", T=43968, H=16, dtype="bf16", kind="layer", gain="shared",
             fused=True, dim=64, axes=2, layout="half", span=38),
        # one token for each of 64 sequences, grouped heads, slices of one projection's output
        dict(name="append_tokens", op="append", B=64, q=1, len=2748, mix=2, Hq=16, Hkv=4, dtype="bf16",
             code="e4m3", page=16, kind="rms", gain="shared", fused=True, dim=32, axes=1, layout="interleaved",
             span=100000),
        # a view joins 31 others
        dict(name="append_view", op="append", B=1, q=1374, len=43968, mix=1, Hq=16, Hkv=16, dtype="bf16",
             code="int8", page=64, kind="layer", gain="shared", fused=False, dim=64, axes=2, layout="half",
             span=38),
        # a single token over a pair of views: latency
        dict(name="attend_token_s2", op="attend", B=1, q=1, len=2748, mix=3, Hq=16, Hkv=16, dtype="bf16",
             code="e4m3", page=64, causal=True, weights=False),
        # single tokens over eight ragged room scans of up to 100 views, four query heads to a key head,
        # their weights gathered for the eviction
        dict(name="attend_tokens_s100_weights", op="attend", B=8, q=1, len=137400, mix=5, Hq=16, Hkv=4,
             dtype="bf16", code="int8", page=128, causal=True, weights=True),
        # a view attends 32 views and itself: the largest call
        dict(name="attend_view_s32", op="attend", B=1, q=1374, len=43968, mix=6, Hq=16, Hkv=16, dtype="bf16",
             code="e4m3", page=64, causal=False, weights=False),
        # ragged causal chunks of four sequences with the weights gathered
        dict(name="attend_chunks_weights", op="attend", B=4, q=1031, len=10992, mix=7, Hq=16, Hkv=8,
             dtype="bf16", code="int8", page=32, causal=True, weights=True),
        # a scene of 32 views handed to a stage that takes plain rows
        dict(name="read_scene", op="read", B=1, q=43968, len=43968, mix=8, Hkv=16, dtype="bf16", code="e4m3",
             page=64),
        # the latest tokens of 16 ragged sequences in fp32
        dict(name="read_batch_f32", op="read", B=16, q=257, len=2748, mix=9, Hkv=4, dtype="f32", code="int8",
             page=16),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "append", "attend", "attend", "attend", "read"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    code = rng.choice(["int8", "e4m3"])
    mix = rng.randrange(1 << 30)
    rot = dict(axes=rng.choice([1, 1, 2]), layout=rng.choice(["half", "interleaved"]), span=_log(rng, 16, 1000000))
    rot["dim"] = rng.choice([16, 32, 48, 64]) if rot["axes"] == 1 else rng.choice([32, 64])
    norm = dict(kind=rng.choice(["layer", "rms"]), gain=rng.choice(["shared", "shared", "heads", "none"]),
                fused=rng.random() < 0.5)
    if op in ("norm", "norm_grad"):
        return dict(op=op, T=_log(rng, 1, 43968 if dtype == "bf16" else 20000), H=rng.choice([1, 3, 4, 8, 16]),
                    dtype=dtype, **norm, **rot)
    Hq, Hkv = rng.choice([(16, 16), (16, 16), (16, 8), (16, 4), (16, 1), (12, 4), (6, 2)])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "append":
        B = _log(rng, 1, 64)
        q = _log(rng, 1, max(1, 2748 // B))
        return dict(op=op, B=B, q=q, len=q + _log(rng, 1, 87936 // B), mix=mix, Hq=Hq, Hkv=Hkv, dtype=dtype,
                    code=code, page=page, **norm, **rot)
    if op == "read":
        B = _log(rng, 1, 32)
        n = _log(rng, 1, (43968 if dtype == "bf16" else 20000) // B)
        return dict(op=op, B=B, q=_log(rng, 1, n), len=n, mix=mix, Hkv=Hkv, dtype=dtype, code=code, page=page)
    # attend: a third single tokens, the others chunks; no more logits, and no more slots, than listed
    B = _log(rng, 1, 64)
    slots = (250000 if dtype == "bf16" else 100000) // B
    q = 1 if rng.random() < 0.35 else _log(rng, 1, 1500)
    most = (900000000 if dtype == "bf16" else 100000000) // (B * Hq * q)
    n = max(1, min(_log(rng, 1, 137400), slots, most))
    return dict(op=op, B=B, q=min(q, n), len=n, mix=mix, Hq=Hq, Hkv=Hkv, dtype=dtype, code=code, page=page,
                causal=rng.random() < 0.7, weights=rng.random() < 0.4)


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """Slots in use (the chunk's included) and new tokens of every sequence: the first has the
    most of both, the others are spread below; in batches of four and more the last is idle."""
    r = random.Random(case["mix"])
    B, n, q = case["B"], case["len"], case["q"]
    ln = [n] + [max(1, _log(r, max(1, n // 8), n)) for _ in range(B - 1)]
    qs = [q] + [min(v, 1 if q == 1 else _log(r, 1, q)) for v in ln[1:]]
    if B >= 4:
        qs[-1] = 0
    return [min(v, n) for v in ln], qs


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _rotation(case, seed, T):
    """Positions, and every pair's share of a revolution per position times 2^64."""
    n = case["dim"] // case["axes"] // 2
    base = 100.0 if case["axes"] == 2 else 10000.0
    f = [base ** (-j / n) for j in range(n)] * case["axes"]
    r = np.random.RandomState(seed % (1 << 31))
    pos = r.randint(0, case["span"], (T, case["axes"])).astype(np.int32)
    return {"radians": f, "pos": torch.from_numpy(pos).to("cuda"),
            "freq": torch.tensor([round(v / (2 * math.pi) * 2.0 ** 64) for v in f], dtype=torch.int64, device="cuda")}


def _gains(case, gen, H):
    """Gain and bias of a trained norm: [64], or [H, 64]; the mean square has no bias."""
    shape = (H, D) if case["gain"] == "heads" else (D,)
    gain = 1 + 0.2 * torch.randn(shape, generator=gen, device="cuda")
    bias = 0.2 * torch.randn(shape, generator=gen, device="cuda")
    if case["gain"] == "none":
        return None, None
    return gain, bias if case["kind"] == "layer" else None


def _pages(case, seed, ln):
    """A pool with a few pages to spare, the sequences' pages scattered over it; -1 where a
    sequence has none."""
    page = case["page"]
    need = [-(-n // page) for n in ln]
    r = np.random.RandomState((seed + 77) % (1 << 31))
    npages = sum(need) + 3
    ids = r.permutation(npages)
    table = np.full((len(ln), max(need)), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return npages, torch.from_numpy(table).to("cuda")


def _pool(case, gen, npages):
    """Codes of K and V and their scales, as appends of normal rows of unequal size leave them."""
    Hkv, page = case["Hkv"], case["page"]
    K, V = (torch.empty(npages, Hkv, page, D, dtype=CODES[case["code"]], device="cuda") for _ in range(2))
    scale = torch.empty(npages, Hkv, page, 2, dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 25) // (Hkv * page * D))
    for i in range(0, npages, step):
        n = min(step, npages - i)
        for j, pool in enumerate((K, V)):
            x = torch.randn(n, Hkv, page, D, generator=gen, device="cuda")
            x *= torch.exp(0.3 * torch.randn(n, Hkv, page, 1, generator=gen, device="cuda"))
            code, s = _quantised(x, case["code"])
            pool.view(torch.uint8)[i:i + n] = code.view(torch.uint8)
            scale[i:i + n, :, :, j] = s
    return K, V, scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed & ((1 << 62) - 1))
    op, dt = case["op"], DTYPES[case["dtype"]]
    st = {"op": op, "case": case}
    if op in ("norm", "norm_grad"):
        T, H, grad = case["T"], case["H"], op == "norm_grad"
        shape = (T, 3 * H if case["fused"] else H, D)
        x = _normal(g, shape, torch.float32) * torch.exp(0.3 * torch.randn(shape[1:], generator=g, device="cuda"))
        x = (x + 0.3 * torch.randn(shape[1:], generator=g, device="cuda")).to(dt)
        st["x"] = x[:, :H] if case["fused"] else x
        st["gain"], st["bias"] = _gains(case, g, H)
        st.update(_rotation(case, seed, T))
        if grad:
            st["g"] = _normal(g, (T, H, D), dt)
            st["leaves"] = [v.requires_grad_() for v in (st["x"], st["gain"], st["bias"]) if v is not None]
        else:
            st["y"] = torch.empty(T, H, D, dtype=dt, device="cuda")
        if own:
            from paper_2609_23733_amd import cache
            st["rot"] = cache.Rotary(st["freq"], layout=case["layout"], axes=case["axes"])
            st["norm"] = cache.HeadNorm(case["kind"], st["gain"], st["bias"], eps=EPS)
        return st
    ln, qs = _lengths(case)
    npages, table = _pages(case, seed, ln)
    page, Hkv = case["page"], case["Hkv"]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    q_start = np.concatenate([[0], np.cumsum(qs)]).tolist()
    T = q_start[-1]
    st["table"], st["length"], st["q_start"], st["T"] = table, i32(ln), i32(q_start), T
    st["K"], st["V"], st["scale"] = _pool(case, g, npages)
    st["weight"] = st["stamp"] = st["seen"] = None
    if op == "append":
        Hq = case["Hq"]
        if case["fused"]:
            x = _normal(g, (T, Hq + 2 * Hkv, D), dt)
            st["Qn"], st["Kn"], st["Vn"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        else:
            st["Qn"], st["Kn"], st["Vn"] = (_normal(g, (T, h, D), dt) for h in (Hq, Hkv, Hkv))
        st["q_gain"], st["q_bias"] = _gains(case, g, Hq)
        st["k_gain"], st["k_bias"] = _gains(case, g, Hkv)
        st.update(_rotation(case, seed, T))
        st["seen"] = st["length"] + 7
        st["weight"] = torch.rand(npages, Hkv, page, generator=g, device="cuda")
        st["stamp"] = torch.full((npages, Hkv, page), -1, dtype=torch.int32, device="cuda")
        st["Q_out"] = torch.empty(T, Hq, D, dtype=dt, device="cuda")
        st["K_out"], st["V_out"] = (torch.empty(T, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    elif op == "read":
        st["K_out"], st["V_out"] = (torch.empty(T, Hkv, D, dtype=dt, device="cuda") for _ in range(2))
    else:
        st["Q"] = _normal(g, (T, case["Hq"], D), dt)
        st["O"] = torch.empty_like(st["Q"])
        st["lse"] = torch.empty(T, case["Hq"], dtype=torch.float32, device="cuda")
        st["weight_out"] = None
        if case["weights"]:
            st["weight"] = torch.rand(npages, Hkv, page, generator=g, device="cuda") * 0.1
            st["weight_out"] = st["weight"].clone()
    if own:
        from paper_2609_23733_amd import cache
        st["pc"] = cache.PagedCache(st["K"], st["V"], st["weight"], st["stamp"], scale=st["scale"], rows=dt)
        st["batch"] = cache.Batch(st["table"], st["length"], st["q_start"], max(qs), max(ln), st["seen"])
        if op == "append":
            st["rot"] = cache.Rotary(st["freq"], layout=case["layout"], axes=case["axes"])
            st["q_norm"] = cache.HeadNorm(case["kind"], st["q_gain"], st["q_bias"], eps=EPS)
            st["k_norm"] = cache.HeadNorm(case["kind"], st["k_gain"], st["k_bias"], eps=EPS)
        elif op == "attend":
            st["ws"] = cache.attend_workspace(st["pc"], st["batch"], case["Hq"], T)
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    c = st["case"]
    if own:
        return _run_own(st, c)
    with torch.no_grad():
        return {"norm": _norm, "norm_grad": _norm_grad, "append": _append, "attend": _attend,
                "read": _read}[c["op"]](st, c)


def _run_own(st, c):
    from paper_2609_23733_amd import cache
    if c["op"] == "norm":
        return {"y": cache.norm_rotary(st["x"], st["norm"], st["pos"], st["rot"], out=st["y"])}
    if c["op"] == "norm_grad":
        y = cache.norm_rotary(st["x"], st["norm"], st["pos"], st["rot"])
        d = torch.autograd.grad(y, st["leaves"], st["g"])
        return {"y": y, "d": list(d)}
    if c["op"] == "append":
        q = cache.append(st["pc"], st["batch"], st["Qn"], st["Kn"], st["Vn"], st["pos"], st["rot"],
                         Q_out=st["Q_out"], q_norm=st["q_norm"], k_norm=st["k_norm"])
        K, V = cache.read(st["pc"], st["batch"], st["T"], K_out=st["K_out"], V_out=st["V_out"])
        return {"Q": q, "K": K, "V": V, "weight": st["weight"], "stamp": st["stamp"]}
    if c["op"] == "read":
        K, V = cache.read(st["pc"], st["batch"], st["T"], K_out=st["K_out"], V_out=st["V_out"])
        return {"K": K, "V": V}
    O, lse = cache.attend(st["pc"], st["batch"], st["Q"], causal=c["causal"], O=st["O"], lse=st["lse"],
                          weight_out=st["weight_out"], ws=st["ws"])
    return {"O": O, "lse": lse, "weight": st["weight_out"]}


def _angles(st, c, T):
    """Cosines and sines [T, 1, axes, pairs].  The angle in revolutions is the low 64 bits of
    pos * freq, of which the top 32 make the fp32 angle."""
    n = c["dim"] // c["axes"] // 2
    turn = st["pos"].long().repeat_interleave(n, dim=1) * st["freq"]
    ang = ((turn >> 32).float() * (2 * math.pi / 2.0 ** 32)).view(T, 1, c["axes"], n)
    return torch.cos(ang), torch.sin(ang)


def _turn(f, c, co, si):
    """[T, H, 64] fp32 with its pairs turned."""
    T, dim, n = f.shape[0], c["dim"], co.shape[3]
    r = f[..., :dim].reshape(T, -1, c["axes"], *((2, n) if c["layout"] == "half" else (n, 2)))
    k = 3 if c["layout"] == "half" else 4
    a, b = r.select(k, 0), r.select(k, 1)
    y = torch.stack([a * co - b * si, b * co + a * si], dim=k).reshape(T, -1, dim)
    return torch.cat([y, f[..., dim:]], dim=2)


def _normed(x, c):
    """Rows without mean (layer) and of mean square 1, and the factor that made them so."""
    f = x.float()
    if c["kind"] == "layer":
        f = f - f.mean(dim=2, keepdim=True)
    r = torch.rsqrt((f * f).mean(dim=2, keepdim=True) + EPS)
    return f * r, r


def _affine(f, gain, bias):
    f = f if gain is None else f * gain
    return f if bias is None else f + bias


def _norm(st, c):
    co, si = _angles(st, c, c["T"])
    return {"y": _turn(_affine(_normed(st["x"], c)[0], st["gain"], st["bias"]), c, co, si).to(st["x"].dtype)}


def _norm_grad(st, c):
    co, si = _angles(st, c, c["T"])
    f, r = _normed(st["x"], c)
    y = _turn(_affine(f, st["gain"], st["bias"]), c, co, si).to(st["x"].dtype)
    h = _turn(st["g"].float(), c, co, -si)                      # the rotation's transpose
    d = h if st["gain"] is None else h * st["gain"]
    dx = d - f * (d * f).mean(dim=2, keepdim=True)
    if c["kind"] == "layer":
        dx = dx - d.mean(dim=2, keepdim=True)
    over = (0,) if c["gain"] == "heads" else (0, 1)
    out = [(dx * r).to(st["x"].dtype)]
    if st["gain"] is not None:
        out.append((h * f).sum(dim=over, dtype=torch.float64).float())
    if st["bias"] is not None:
        out.append(h.sum(dim=over, dtype=torch.float64).float())
    return {"y": y, "d": out}


def _quantised(x, code):
    """Codes and scales of fp32 rows; the scale's exponent from 64 bits, as rows lie next to its borders."""
    m, e = torch.frexp(x.abs().amax(dim=-1).double() / LARGEST[code])
    e = torch.where(m == 0.5, e - 1, e).clamp(min=-100)         # (m 2^e with m from 0.5 to 1)
    s = torch.ldexp(torch.ones_like(m), e).float()
    v = x / s[..., None]
    v = torch.round(v).to(torch.int8) if code == "int8" else v.to(torch.float8_e4m3fn)
    return v, s.to(torch.bfloat16)


def _values(code, scale):
    return code.float() * scale.float()[..., None]


def _new_slots(st):
    """Page, place in it, and number of every new token."""
    c = st["case"]
    t = torch.arange(st["T"], device="cuda")
    b = torch.searchsorted(st["q_start"].long(), t, right=True) - 1
    past = t - st["q_start"].long()[b + 1]                      # -1 for a chunk's last
    s = st["length"].long()[b] + past
    return st["table"].long()[b, s // c["page"]], s % c["page"], b, past


def _read(st, c):
    page, s, _, _ = _new_slots(st)
    dt = st["K_out"].dtype
    out = {}
    scale = st["scale"][page, :, s]
    code = CODES[c["code"]]
    out["K"] = _values(st["K"].view(torch.uint8)[page, :, s].view(code), scale[..., 0]).to(dt)
    out["V"] = _values(st["V"].view(torch.uint8)[page, :, s].view(code), scale[..., 1]).to(dt)
    return out


def _append(st, c):
    page, s, b, past = _new_slots(st)
    co, si = _angles(st, c, st["T"])
    Q = _turn(_affine(_normed(st["Qn"], c)[0], st["q_gain"], st["q_bias"]), c, co, si).to(st["Qn"].dtype)
    k, ks = _quantised(_turn(_affine(_normed(st["Kn"], c)[0], st["k_gain"], st["k_bias"]), c, co, si), c["code"])
    v, vs = _quantised(st["Vn"].float(), c["code"])
    st["K"].view(torch.uint8)[page, :, s] = k.view(torch.uint8)
    st["V"].view(torch.uint8)[page, :, s] = v.view(torch.uint8)
    st["scale"][page, :, s] = torch.stack([ks, vs], dim=2)
    st["weight"][page, :, s] = 0.0
    st["stamp"][page, :, s] = (st["seen"][b] + past).to(torch.int32)[:, None].expand(-1, c["Hkv"])
    return {"Q": Q, **_read(st, c), "weight": st["weight"], "stamp": st["stamp"]}


def _rows(pool, st):
    """[B, Hkv, slots, ...] of the pages in every sequence's table."""
    x = pool[st["table"].clamp(min=0).long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])


def _attend(st, c):
    B, Hq, Hkv = c["B"], c["Hq"], c["Hkv"]
    G, q, T = Hq // Hkv, c["q"], st["T"]
    n = st["table"].shape[1] * c["page"]
    slot = torch.arange(n, device="cuda")
    t = torch.arange(q, device="cuda")
    ln = st["length"].long()
    nq = (st["q_start"][1:] - st["q_start"][:-1]).long()
    live = (slot < ln[:, None]) & (nq > 0)[:, None]                          # [B, slots]
    scale, code = _rows(st["scale"], st), CODES[c["code"]]
    K, V = (torch.where(live[:, None, :, None],
                        _values(_rows(st[k].view(torch.uint8), st).view(code), scale[..., j]), 0.0)
            for j, k in enumerate(("K", "V")))
    at = (st["q_start"].long()[:B, None] + t).clamp(max=T - 1)               # [B, q]
    Q = st["Q"].float()[at].view(B, q, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, q * G, D)
    x = torch.matmul(Q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(B, Hkv, q, G, n)
    sees = (live[:, None] & (t < nq[:, None])[..., None])[:, None, :, None]  # [B, 1, q, 1, slots]
    if c["causal"]:
        last = (ln - nq)[:, None] + t                                        # [B, q]
        sees = sees & (slot <= last[..., None])[:, None, :, None]
    x.masked_fill_(~sees, -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    x = x.sub_(m).exp_()
    s = x.sum(dim=-1, keepdim=True)
    lse = torch.where(s > 0, torch.log(s) + m, -math.inf)
    x = x.div_(torch.where(s > 0, s, 1.0))
    O = torch.matmul(x.view(B, Hkv, q * G, n), V).view(B, Hkv, q, G, D).transpose(1, 2)
    new = t < nq[:, None]
    out = {"O": O.reshape(B, q, Hq, D)[new].to(st["Q"].dtype),
           "lse": lse[..., 0].transpose(1, 2).reshape(B, q, Hq)[new], "weight": None}
    if c["weights"]:
        w = (_rows(st["weight"], st) + x.sum(dim=(2, 3))).transpose(1, 2)    # [B, slots, Hkv]
        page = st["table"].long().repeat_interleave(c["page"], dim=1)
        st["weight_out"][page[live], :, (slot % c["page"]).expand(B, n)[live]] = w[live]
        out["weight"] = st["weight_out"]
    return out


# ------------------------------------------------------------------ work

def work(case):
    e, op = SIZE[case["dtype"]], case["op"]
    turn = 3.0 * case.get("dim", 0)                                          # of a head's row
    if op in ("norm", "norm_grad"):
        rows, small = case["T"] * case["H"], 4 * case["T"] * case["axes"]
        if op == "norm":
            return {"bytes": 2 * rows * D * e + small, "flops": rows * (7.0 * D + turn)}
        return {"bytes": 4 * rows * D * e + small, "flops": rows * (20.0 * D + 2 * turn)}
    ln, qs = _lengths(case)
    Hkv, T = case["Hkv"], sum(qs)
    slot = 2 * D + 4                                                         # codes and scales
    if op == "read":
        return {"bytes": T * Hkv * (slot + 2 * D * e), "flops": 2.0 * T * Hkv * D}
    if op == "append":
        Hq = case["Hq"]
        return {"bytes": T * (2 * Hq * D * e + Hkv * (2 * D * e + slot + 4 * D + 8) + 4 * case["axes"]),
                "flops": T * ((Hq + Hkv) * (7.0 * D + turn) + 8.0 * Hkv * D)}
    slots = sum(n for n, q in zip(ln, qs) if q)
    pairs = sum(q * n - (q * (q - 1) // 2 if case["causal"] else 0) for n, q in zip(ln, qs))
    return {"bytes": Hkv * slots * slot + T * case["Hq"] * (2 * D * e + 4)
            + (8 * Hkv * slots if case["weights"] else 0), "flops": 4.0 * D * case["Hq"] * pairs}


# ------------------------------------------------------------------ in 64 bits, from the definitions

def exact(case, seed):
    """One sequence and head after the other, on the rows that the page table names."""
    st = prepare(case, seed)
    with torch.no_grad():
        if case["op"] in ("norm", "norm_grad"):
            return _exact_norm(st, case)
        ln, qs = _lengths(case)
        table = st["table"].cpu().numpy().astype(np.int64)

        def rows(b, n0, n1):
            s = np.arange(n0, n1)
            return (torch.from_numpy(table[b, s // case["page"]]).to("cuda"),
                    torch.from_numpy(s % case["page"]).to("cuda"))

        if case["op"] == "append":
            return _exact_append(st, case, ln, qs, rows)
        if case["op"] == "read":
            at = [rows(b, n - m, n) for b, (n, m) in enumerate(zip(ln, qs))]
            p, s = (torch.cat([a[i] for a in at]) for i in range(2))
            return {k: torch.stack([_held(st, case, j, p, h, s) for h in range(case["Hkv"])], dim=1)
                    for j, k in enumerate(("K", "V"))}
        G = case["Hq"] // case["Hkv"]
        O = torch.zeros(st["T"], case["Hq"], D, dtype=torch.float64, device="cuda")
        lse = torch.zeros(st["T"], case["Hq"], dtype=torch.float64, device="cuda")
        W = st["weight"].double() if case["weights"] else None
        t = 0
        for b, (n, m) in enumerate(zip(ln, qs)):
            if m == 0:
                continue
            p, s = rows(b, 0, n)
            hidden = None
            if case["causal"]:
                hidden = torch.arange(n, device="cuda") > torch.arange(n - m, n, device="cuda")[:, None]
            for hk in range(case["Hkv"]):
                k, v = _held(st, case, 0, p, hk, s), _held(st, case, 1, p, hk, s)
                for h in range(hk * G, (hk + 1) * G):
                    x = st["Q"][t:t + m, h].double() @ k.t() / 8.0
                    if hidden is not None:
                        x = x.masked_fill(hidden, -math.inf)
                    lse[t:t + m, h] = torch.logsumexp(x, dim=1)
                    a = torch.exp(x - lse[t:t + m, h, None])
                    O[t:t + m, h] = a @ v
                    if W is not None:
                        W[p, hk, s] += a.sum(dim=0)
            t += m
        return {"O": O, "lse": lse, "weight": W}


def _held(st, case, j, p, h, s):
    """Rows of K (j = 0) or V of one head, in 64 bits."""
    code = st["KV"[j]].view(torch.uint8)[p, h, s]
    if case["code"] == "int8":
        v = code.double() - 256.0 * (code >= 128)
    else:                                                                    # sign, four bits, three bits
        e, f = (code >> 3) & 15, (code & 7).double()
        v = torch.where(e == 0, f / 512, (8 + f) * torch.exp2(e.double() - 10))
        v = torch.where(code >= 128, -v, v)
    return v * st["scale"][p, h, s, j].double()[:, None]


def _exact_rows(x, st, case, gain, bias):
    """Normalised rows turned: pairs as complex numbers times e^(i pos freq), the angle from the real
    frequency.  Returns the rows, those before gain and bias, and the function that turns."""
    y = x.double()
    if case["kind"] == "layer":
        y = y - y.sum(dim=2, keepdim=True) / D
    rms = torch.sqrt((y ** 2).sum(dim=2, keepdim=True) / D + EPS)
    y = y / rms

    def turn(z, sign):
        z = z.clone()
        n = case["dim"] // case["axes"] // 2
        for a in range(case["axes"]):
            for j in range(n):
                o = a * 2 * n
                i0, i1 = (o + j, o + j + n) if case["layout"] == "half" else (o + 2 * j, o + 2 * j + 1)
                pos = st["pos"][:, a].double()
                w = torch.polar(torch.ones_like(pos), sign * pos * st["radians"][a * n + j])
                u = torch.complex(z[:, :, i0], z[:, :, i1]) * w[:, None]
                z[:, :, i0], z[:, :, i1] = u.real, u.imag
        return z

    z = y if gain is None else y * gain.double()
    return turn(z if bias is None else z + bias.double(), 1.0), y, rms, turn


def _exact_norm(st, case):
    """The gradients through the Jacobian of a row, J = (I - [1 1^T / 64] - n n^T / 64) / rms."""
    out, y, rms, turn = _exact_rows(st["x"], st, case, st["gain"], st["bias"])
    if case["op"] == "norm":
        return {"y": out}
    h = turn(st["g"].double(), -1.0)
    z = h if st["gain"] is None else h * st["gain"].double()
    dx = z - (y * z).sum(dim=2, keepdim=True) / D * y
    if case["kind"] == "layer":
        dx = dx - z.sum(dim=2, keepdim=True) / D
    d = [dx / rms]
    for v, k in ((h * y, "gain"), (h, "bias")):
        if st[k] is not None:
            v = v.sum(dim=0)
            d.append(v if case["gain"] == "heads" else v.sum(dim=0))
    return {"y": out, "d": d}


def _exact_codes(x, case):
    """Rows as the cache holds them: multiples of the step at each value."""
    top = LARGEST[case["code"]]
    big = x.abs().amax(dim=2, keepdim=True)
    e = torch.ceil(torch.log2(big / top)).clamp(min=-100)
    e = torch.where(torch.exp2(e - 1) * top >= big, e - 1, e)                # (a logarithm next to a whole number)
    s = torch.exp2(torch.where(torch.exp2(e) * top < big, e + 1, e).clamp(min=-100))
    if case["code"] == "int8":
        return torch.round(x / s) * s
    v = x / s
    step = torch.exp2((torch.frexp(v).exponent - 1).clamp(min=-6).double() - 3)
    return torch.round(v / step) * step * s


def _exact_append(st, case, ln, qs, rows):
    Q = _exact_rows(st["Qn"], st, case, st["q_gain"], st["q_bias"])[0]
    K = _exact_codes(_exact_rows(st["Kn"], st, case, st["k_gain"], st["k_bias"])[0], case)
    V = _exact_codes(st["Vn"].double(), case)
    W, S = st["weight"].double(), st["stamp"].clone()
    for b, (n, m) in enumerate(zip(ln, qs)):
        if m:
            p, s = rows(b, n - m, n)
            W[p, :, s] = 0.0
            S[p, :, s] = torch.arange(n + 7 - m, n + 7, dtype=torch.int32, device="cuda")[:, None]
    return {"Q": Q, "K": K, "V": V, "weight": W, "stamp": S}
