"""The paged key-value cache of views that arrive one after another: its operators, at real sizes.

A scene whose views (S views of P = 1,374 tokens, 16 heads of 64) arrive one at a time, or several
scenes at once, keep the keys and values of the views seen so far in pages of a common pool:
K, V [pages, Hkv, page, 64], and for every slot the attention weight that its key has gathered
and the number of the token it holds ("stamp"), [pages, Hkv, page].  Sequence b's slot s lies on
page table[b, s // page].  Four operators work on it:

  rotary   positions as rotations of feature pairs, y = mag R(pos * freq) x, or its transpose (the
           gradient); `freq` is a 64-bit fraction of a revolution per position, so the
           angle is reduced exactly at any position
  append   a chunk of new tokens: Q and K rotated, K and V written into the sequences' last slots,
           the slots' weight cleared and their stamps set
  attend   softmax attention of the chunk's queries over the cached slots (grouped heads, causal or
           whole chunks), the log-sum-exp of every row, and, where asked, the attention
           weights added to the slots they fall on
  evict    keeps `keep` slots of every sequence and head: protected ones (the first `sink` tokens, the
           latest `recent`) first, then by gathered weight, lower slots first among equals; kept
           slots past `keep` move into the holes below it, both in ascending order

A case is a dict of plain values; the lengths of a batch follow from `B`, `q`, `len` and `mix`.
"""
import math
import random

import numpy as np
import torch

own = False

D = 64
PATCHES_AND_SPECIAL = 1374
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def listed():
    return [
        # queries of a few single tokens, fp32: the smallest call, latency only
        dict(name="rotary_tokens", op="rotary", T=13, H=16, dtype="f32", dim=64, axes=1, layout="half",
             scaling="none", span=4096, transpose=False),
        # gradient through the positions of a batch of scenes, far past the trained range, part of the head
        dict(name="rotary_grad_long", op="rotary", T=43968, H=16, dtype="bf16", dim=48, axes=1,
             layout="interleaved", scaling="parts", span=1000000, transpose=True),
        # a view of an object scene joins 31 others: 2D positions of its patches
        dict(name="append_view", op="append", B=1, q=1374, len=43968, mix=1, Hq=16, Hkv=16, dtype="bf16",
             page=64, dim=64, axes=2, layout="half", scaling="none", span=38, fused=False),
        # one token for each of 64 sequences, grouped heads, slices of one projection's output
        dict(name="append_tokens", op="append", B=64, q=1, len=2748, mix=2, Hq=16, Hkv=4, dtype="f32",
             page=16, dim=32, axes=1, layout="interleaved", scaling="linear", span=100000, fused=True),
        # a single token over a pair of views: latency
        dict(name="attend_token_s2", op="attend", B=1, q=1, len=2748, mix=3, Hq=16, Hkv=16, dtype="bf16",
             page=64, causal=True, weights=False),
        # single tokens of 32 ragged sequences, four query heads to a key head, short pages
        dict(name="attend_tokens_batch", op="attend", B=32, q=1, len=10992, mix=4, Hq=16, Hkv=4,
             dtype="bf16", page=16, causal=True, weights=False),
        # single tokens over whole room scans (100 views), their weights gathered for the eviction
        dict(name="attend_token_s100_weights", op="attend", B=2, q=1, len=137400, mix=5, Hq=16, Hkv=16,
             dtype="bf16", page=128, causal=True, weights=True),
        # a view attends 32 views and itself: the ordinary large call
        dict(name="attend_view_s32", op="attend", B=1, q=1374, len=43968, mix=6, Hq=16, Hkv=16,
             dtype="bf16", page=64, causal=False, weights=False),
        # ragged causal chunks of four sequences with the weights gathered
        dict(name="attend_chunks_weights", op="attend", B=4, q=1031, len=10992, mix=7, Hq=16, Hkv=8,
             dtype="bf16", page=32, causal=True, weights=True),
        # ragged prompts in fp32
        dict(name="attend_prompts_f32", op="attend", B=3, q=777, len=2748, mix=8, Hq=16, Hkv=8,
             dtype="f32", page=32, causal=True, weights=False),
        # a room scan brought down to 32 views' worth of slots
        dict(name="evict_s100", op="evict", B=1, len=137400, keep=43968, sink=1374, recent=1374, mix=9,
             Hkv=16, dtype="bf16", page=64),
        # eight ragged sequences in fp32, some of them short enough to keep everything
        dict(name="evict_batch_f32", op="evict", B=8, len=8244, keep=2748, sink=5, recent=257, mix=10,
             Hkv=4, dtype="f32", page=16),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    op = rng.choice(["rotary", "append", "attend", "attend", "attend", "evict"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    mix = rng.randrange(1 << 30)
    rot = dict(axes=rng.choice([1, 1, 2]), layout=rng.choice(["half", "interleaved"]),
               scaling=rng.choice(["none", "linear", "parts"]), span=_log(rng, 64, 1000000))
    rot["dim"] = rng.choice([16, 32, 48, 64]) if rot["axes"] == 1 else rng.choice([32, 64])
    Hq, Hkv = rng.choice([(16, 16), (16, 16), (16, 8), (16, 4), (16, 1), (12, 4), (6, 2)])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "rotary":
        return dict(op=op, T=_log(rng, 1, 43968 if dtype == "bf16" else 20000), H=rng.choice([1, 3, 4, 8, 16]),
                    dtype=dtype, transpose=rng.random() < 0.4, **rot)
    if op == "append":
        B = _log(rng, 1, 64)
        q = _log(rng, 1, max(1, 2748 // B))
        return dict(op=op, B=B, q=q, len=q + _log(rng, 1, 87936 // B), mix=mix, Hq=Hq, Hkv=Hkv, dtype=dtype,
                    page=page, fused=Hq != Hkv and rng.random() < 0.6, **rot)
    if op == "evict":
        B = _log(rng, 1, 16)
        n = _log(rng, 64, (137400 if dtype == "bf16" else 60000) // B)
        keep = max(1, int(n * rng.uniform(0.1, 0.95)))
        return dict(op=op, B=B, len=n, keep=keep, sink=rng.choice([0, 1, 5, min(n, 1374)]),
                    recent=rng.choice([0, 1, 64, min(n, 1374)]), mix=mix, Hkv=Hkv, dtype=dtype, page=page)
    # attend: a third single tokens, the others chunks; no more logits, and no more slots, than listed
    B = _log(rng, 1, 64)
    slots = (250000 if dtype == "bf16" else 100000) // B
    q = 1 if rng.random() < 0.35 else _log(rng, 1, 1500)
    most = (900000000 if dtype == "bf16" else 150000000) // (B * Hq * q)
    n = max(1, min(_log(rng, 1, 137400), slots, most))
    q = min(q, n)
    return dict(op=op, B=B, q=q, len=n, mix=mix, Hq=Hq, Hkv=Hkv, dtype=dtype, page=page,
                causal=rng.random() < 0.7, weights=rng.random() < 0.4)


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """Slots in use (the chunk's included) and new tokens of every sequence: the first has the
    most of both, the others are spread below; in batches of four and more the last is idle."""
    r = random.Random(case["mix"])
    B, n, q = case["B"], case["len"], case.get("q", 0)
    ln = [n] + [max(1, _log(r, max(1, n // 8), n)) for _ in range(B - 1)]
    if case["op"] == "evict":
        return [min(v, n) for v in ln], [0] * B
    qs = [q] + [min(v, 1 if q == 1 else _log(r, 1, q)) for v in ln[1:]]
    if B >= 4:
        qs[-1] = 0
    return [min(v, n) for v in ln], qs


def _normal(gen, shape, std, dtype):
    """N(0, std^2); drawn in slices so that no fp32 copy of a large pool is held."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 26
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=gen, device="cuda") * std
    return out


def _frequencies(case):
    """Radians per position of every pair and the factor on the result.  Sections of the axes
    have the same frequencies.  "linear": positions divided by 8.  "parts": pairs that turn less than
    once over the trained 8,192 positions divided by 8, those that turn 32 times or more kept, in
    between blended, with the factor 0.1 ln 8 + 1."""
    n = case["dim"] // case["axes"] // 2
    base = 100.0 if case["axes"] == 2 else 10000.0
    f = [base ** (-j / n) for j in range(n)]
    mag = 1.0
    if case["scaling"] == "linear":
        f = [v / 8 for v in f]
    if case["scaling"] == "parts":
        keep = [min(1.0, max(0.0, (8192 * v / (2 * math.pi) - 1) / 31)) for v in f]
        f = [v * (k + (1 - k) / 8) for v, k in zip(f, keep)]
        mag = 0.1 * math.log(8) + 1
    return f * case["axes"], mag


def _rotation(case, seed, T):
    f, mag = _frequencies(case)
    fixed = [round(v / (2 * math.pi) * 2.0 ** 64) for v in f]   # below 2^62: at most one radian
    r = np.random.RandomState(seed % (1 << 31))
    pos = r.randint(0, case["span"], (T, case["axes"])).astype(np.int32)
    return {"freq": torch.tensor(fixed, dtype=torch.int64, device="cuda"), "mag": mag,
            "pos": torch.from_numpy(pos).to("cuda")}


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


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed & ((1 << 62) - 1))
    op, dt = case["op"], DTYPES[case["dtype"]]
    st = {"op": op, "case": case}
    if op == "rotary":
        st["x"] = _normal(g, (case["T"], case["H"], D), 1.0, dt)
        st["y"] = torch.empty_like(st["x"])
        st.update(_rotation(case, seed, case["T"]))
        if own:
            from paper_2609_23733_amd import cache
            st["rot"] = cache.Rotary(st["freq"], layout=case["layout"], axes=case["axes"], mag=st["mag"])
        return st
    ln, qs = _lengths(case)
    npages, table = _pages(case, seed, ln)
    page, Hkv = case["page"], case["Hkv"]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    st["table"], st["length"] = table, i32(ln)
    st["K"] = _normal(g, (npages, Hkv, page, D), 1.0, dt)
    st["V"] = _normal(g, (npages, Hkv, page, D), 1.0, dt)
    if op == "evict":
        B, n = case["B"], case["len"]
        past = n // 3                                      # tokens that earlier evictions took out
        st["seen"] = st["length"] + past
        w = torch.exp(1.5 * torch.randn(npages, Hkv, page, generator=g, device="cuda"))
        tied = torch.rand(npages, Hkv, page, generator=g, device="cuda")
        w = torch.where(tied < 0.1, 0.0, torch.where(tied < 0.2, torch.round(w), w))
        st["weight"], st["stamp"] = w, torch.zeros(npages, Hkv, page, dtype=torch.int32, device="cuda")
        # the kept tokens of every head in an order of its own: numbers below `sink` and from
        # `past` + `sink` on, each once
        for b in range(B):
            o = torch.rand(Hkv, ln[b], generator=g, device="cuda").argsort(dim=1).to(torch.int32)
            o = torch.where(o < case["sink"], o, o + past)
            s = torch.arange(ln[b], device="cuda")
            st["stamp"][table[b, s // page].long(), :, s % page] = o.t()
        st["weight_out"], st["stamp_out"] = w.clone(), st["stamp"].clone()
        st["length_out"] = st["length"].clone()
        if own:
            from paper_2609_23733_amd import cache
            st["pc"] = cache.PagedCache(st["K"], st["V"], st["weight"], st["stamp"])
            st["ws"] = cache.evict_workspace(st["pc"], B, n)
        return st
    q_start = np.concatenate([[0], np.cumsum(qs)]).tolist()
    T, Hq = q_start[-1], case["Hq"]
    st["q_start"], st["T"] = i32(q_start), T
    if op == "append":
        if case["fused"]:
            x = _normal(g, (T, Hq + 2 * Hkv, D), 1.0, dt)
            st["Qn"], st["Kn"], st["Vn"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        else:
            st["Qn"], st["Kn"], st["Vn"] = (_normal(g, (T, h, D), 1.0, dt) for h in (Hq, Hkv, Hkv))
        st.update(_rotation(case, seed, T))
        st["seen"] = st["length"] + 7
        st["weight"] = torch.rand(npages, Hkv, page, generator=g, device="cuda")
        st["stamp"] = torch.full((npages, Hkv, page), -1, dtype=torch.int32, device="cuda")
        st["Q_out"] = torch.empty(T, Hq, D, dtype=dt, device="cuda")
    else:
        st["Q"] = _normal(g, (T, Hq, D), 1.0, dt)
        st["O"] = torch.empty_like(st["Q"])
        st["lse"] = torch.empty(T, Hq, dtype=torch.float32, device="cuda")
        st["weight"] = st["weight_out"] = None
        if case["weights"]:
            st["weight"] = torch.rand(npages, Hkv, page, generator=g, device="cuda") * 0.1
            st["weight_out"] = st["weight"].clone()
    if own:
        from paper_2609_23733_amd import cache
        st["pc"] = cache.PagedCache(st["K"], st["V"], st["weight"], st.get("stamp"))
        st["batch"] = cache.Batch(st["table"], st["length"], st["q_start"], max(qs), max(ln), st.get("seen"))
        if op == "append":
            st["rot"] = cache.Rotary(st["freq"], layout=case["layout"], axes=case["axes"], mag=st["mag"])
        else:
            st["ws"] = cache.attend_workspace(st["pc"], st["batch"], Hq, T)
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    c = st["case"]
    if own:
        return _run_own(st, c)
    if c["op"] == "rotary":
        return {"y": _rotate(st["x"], st, c, c["transpose"])}
    return {"append": _append, "attend": _attend, "evict": _evict}[c["op"]](st, c)


def _run_own(st, c):
    from paper_2609_23733_amd import cache
    if c["op"] == "rotary":
        return {"y": cache.rotary(st["x"], st["pos"], st["rot"], out=st["y"], transpose=c["transpose"])}
    if c["op"] == "append":
        q = cache.append(st["pc"], st["batch"], st["Qn"], st["Kn"], st["Vn"], st["pos"], st["rot"],
                         Q_out=st["Q_out"])
        return {"Q": q, "K": st["K"], "V": st["V"], "weight": st["weight"], "stamp": st["stamp"]}
    if c["op"] == "attend":
        O, lse = cache.attend(st["pc"], st["batch"], st["Q"], causal=c["causal"], O=st["O"], lse=st["lse"],
                              weight_out=st["weight_out"], ws=st["ws"])
        return {"O": O, "lse": lse, "weight": st["weight_out"]}
    n = cache.evict(st["pc"], st["table"], st["length"], st["seen"], keep=c["keep"], max_len=c["len"],
                    sink=c["sink"], recent=c["recent"], weight_out=st["weight_out"],
                    stamp_out=st["stamp_out"], length_out=st["length_out"], ws=st["ws"])
    return {"K": st["K"], "V": st["V"], "weight": st["weight_out"], "stamp": st["stamp_out"], "length": n}


def _rotate(x, st, c, transpose):
    """[T, H, 64] rotated, rounded once.  The angle in revolutions is the low 64 bits of
    pos * freq, of which the top 32 make the fp32 angle."""
    T, dim, axes = x.shape[0], c["dim"], c["axes"]
    n = dim // axes // 2
    turn = st["pos"].long().repeat_interleave(n, dim=1) * st["freq"]
    ang = ((turn >> 32).float() * (2 * math.pi / 2.0 ** 32)).view(T, 1, axes, n)
    if transpose:
        ang = -ang
    co, si = torch.cos(ang) * st["mag"], torch.sin(ang) * st["mag"]
    f = x.float()
    r = f[..., :dim].reshape(T, -1, axes, *((2, n) if c["layout"] == "half" else (n, 2)))
    k = 3 if c["layout"] == "half" else 4
    a, b = r.select(k, 0), r.select(k, 1)
    y = torch.stack([a * co - b * si, b * co + a * si], dim=k).reshape(T, -1, dim)
    return torch.cat([y, f[..., dim:]], dim=2).to(x.dtype)


def _new_slots(st):
    """Sequence, number within the chunk, and slot of every new token."""
    t = torch.arange(st["T"], device="cuda")
    b = torch.searchsorted(st["q_start"].long(), t, right=True) - 1
    i = t - st["q_start"].long()[b]
    nq = (st["q_start"][1:] - st["q_start"][:-1]).long()[b]
    return b, i, st["length"].long()[b] - nq + i, st["seen"].long()[b] - nq + i


def _append(st, c):
    b, _, s, stamp = _new_slots(st)
    page = st["table"].long()[b, s // c["page"]]
    s = s % c["page"]
    st["K"][page, :, s] = _rotate(st["Kn"], st, c, False)
    st["V"][page, :, s] = st["Vn"]
    st["weight"][page, :, s] = 0.0
    st["stamp"][page, :, s] = stamp.to(torch.int32)[:, None].expand(-1, c["Hkv"])
    return {"Q": _rotate(st["Qn"], st, c, False), "K": st["K"], "V": st["V"], "weight": st["weight"],
            "stamp": st["stamp"]}


def _rows(pool, st, c):
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
    K = torch.where(live[:, None, :, None], _rows(st["K"], st, c).float(), 0.0)
    V = torch.where(live[:, None, :, None], _rows(st["V"], st, c).float(), 0.0)
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
        w = (_rows(st["weight"], st, c) + x.sum(dim=(2, 3))).transpose(1, 2)  # [B, slots, Hkv]
        page = st["table"].long().repeat_interleave(c["page"], dim=1)
        st["weight_out"][page[live], :, (slot % c["page"]).expand(B, n)[live]] = w[live]
        out["weight"] = st["weight_out"]
    return out


def _evict(st, c):
    B, Hkv, n = c["B"], c["Hkv"], st["table"].shape[1] * c["page"]
    slot = torch.arange(n, device="cuda")
    ln = st["length"].long()
    live = (slot < ln[:, None])[:, None]
    left = ln.clamp(max=c["keep"])                                           # [B]
    stamp, w = _rows(st["stamp"], st, c), _rows(st["weight"], st, c)
    safe = (stamp < c["sink"]) | (stamp >= (st["seen"] - c["recent"])[:, None, None])
    rank = torch.where(live, torch.where(safe, math.inf, w), -math.inf)
    order = rank.sort(dim=2, descending=True, stable=True).indices           # [B, Hkv, slots]
    keep = torch.zeros(B, Hkv, n, dtype=torch.bool, device="cuda")
    keep.scatter_(2, order, (slot < left[:, None])[:, None].expand(B, Hkv, n))
    low = (slot < left[:, None])[:, None]
    hole, mover = low & ~keep, keep & ~low
    # the j-th mover goes to the j-th hole
    b, hm, src = mover.nonzero(as_tuple=True)
    dst = hole.nonzero(as_tuple=True)[2]
    page = st["table"].long()
    ps, pd, s, d = page[b, src // c["page"]], page[b, dst // c["page"]], src % c["page"], dst % c["page"]
    for name in ("K", "V"):
        st[name][pd, hm, d] = st[name][ps, hm, s]
    b, h, o = low.expand(B, Hkv, n).nonzero(as_tuple=True)
    po = page[b, o // c["page"]]
    for name in ("weight", "stamp"):
        st[name + "_out"][po, h, o % c["page"]] = st[name][po, h, o % c["page"]]
        st[name + "_out"][pd, hm, d] = st[name][ps, hm, s]
    st["length_out"].copy_(left)
    return {"K": st["K"], "V": st["V"], "weight": st["weight_out"], "stamp": st["stamp_out"],
            "length": st["length_out"]}


# ------------------------------------------------------------------ work

def work(case):
    e, op = SIZE[case["dtype"]], case["op"]
    if op == "rotary":
        x = case["T"] * case["H"]
        return {"bytes": 2 * x * D * e + 4 * case["T"] * case["axes"], "flops": 3.0 * x * case["dim"]}
    ln, qs = _lengths(case)
    Hkv = case["Hkv"]
    if op == "append":
        T = sum(qs)
        return {"bytes": 2 * T * D * e * (case["Hq"] + 2 * Hkv) + T * (8 * Hkv + 4 * case["axes"]),
                "flops": 3.0 * T * (case["Hq"] + Hkv) * case["dim"]}
    if op == "evict":
        # weights and stamps read; those kept written; the keys and values of as many movers as
        # weights without order leave past `keep`, read and written
        k = [min(n, case["keep"]) for n in ln]
        return {"bytes": sum(Hkv * (8 * n + 8 * v + v * (n - v) / n * 4 * D * e) for n, v in zip(ln, k)),
                "flops": float(sum(Hkv * n for n in ln))}
    slots = sum(n for n, q in zip(ln, qs) if q)
    pairs = sum(q * n - (q * (q - 1) // 2 if case["causal"] else 0) for n, q in zip(ln, qs))
    T = sum(qs)
    return {"bytes": 2 * Hkv * slots * D * e + T * case["Hq"] * (2 * D * e + 4)
            + (8 * Hkv * slots if case["weights"] else 0), "flops": 4.0 * D * case["Hq"] * pairs}


# ------------------------------------------------------------------ in 64 bits, from the definitions

def exact(case, seed):
    """One sequence and head after the other, on the rows that the page table names."""
    st = prepare(case, seed)
    if case["op"] == "rotary":
        return {"y": _exact_rotation(st["x"], st, case, -1.0 if case["transpose"] else 1.0)}
    ln, qs = _lengths(case)
    table = st["table"].cpu().numpy().astype(np.int64)
    page, Hkv = case["page"], case["Hkv"]

    def rows(b, n0, n1):
        s = np.arange(n0, n1)
        return (torch.from_numpy(table[b, s // page]).to("cuda"), torch.from_numpy(s % page).to("cuda"))

    if case["op"] == "append":
        kr, q = (_exact_rotation(st[k], st, case, 1.0) for k in ("Kn", "Qn"))
        K, V, W, S = st["K"].double(), st["V"].double(), st["weight"].double(), st["stamp"].clone()
        t = 0
        for b, (n, m) in enumerate(zip(ln, qs)):
            p, s = rows(b, n - m, n)
            K[p, :, s], V[p, :, s], W[p, :, s] = kr[t:t + m], st["Vn"][t:t + m].double(), 0.0
            S[p, :, s] = torch.arange(n + 7 - m, n + 7, dtype=torch.int32, device="cuda")[:, None]
            t += m
        return {"Q": q, "K": K, "V": V, "weight": W, "stamp": S}
    if case["op"] == "evict":
        return _exact_eviction(st, case, ln, rows)
    G = case["Hq"] // Hkv
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
        for hk in range(Hkv):
            k, v = st["K"][p, hk, s].double(), st["V"][p, hk, s].double()
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


def _exact_rotation(x, st, case, sign):
    """Pairs as complex numbers times e^(i pos freq), the angle from the real frequency."""
    f, mag = _frequencies(case)
    n = case["dim"] // case["axes"] // 2
    y = x.double().clone()
    pos = st["pos"].double()
    for a in range(case["axes"]):
        for j in range(n):
            o = a * 2 * n
            i0, i1 = (o + j, o + j + n) if case["layout"] == "half" else (o + 2 * j, o + 2 * j + 1)
            w = torch.polar(torch.full_like(pos[:, a], mag), sign * pos[:, a] * f[a * n + j])
            z = torch.complex(y[:, :, i0], y[:, :, i1]) * w[:, None]
            y[:, :, i0], y[:, :, i1] = z.real, z.imag
    return y


def _exact_eviction(st, case, ln, rows):
    K, V, W, S = st["K"].clone(), st["V"].clone(), st["weight"].clone(), st["stamp"].clone()
    seen, left = st["seen"].tolist(), []
    for b, n in enumerate(ln):
        k = min(n, case["keep"])
        left.append(k)
        p, s = rows(b, 0, n)
        for h in range(case["Hkv"]):
            w, stamp = W[p, h, s].cpu().numpy(), S[p, h, s].cpu().numpy()
            safe = (stamp < case["sink"]) | (stamp >= seen[b] - case["recent"])
            kept = np.lexsort((np.arange(n), -np.where(safe, 0, w), ~safe))[:k]
            src = np.sort(kept[kept >= k])
            dst = np.setdiff1d(np.arange(k), kept)
            i, j = torch.from_numpy(src).to("cuda"), torch.from_numpy(dst).to("cuda")
            for x in (K, V, W, S):
                x[p[j], h, s[j]] = x[p[i], h, s[i]]
    return {"K": K, "V": V, "weight": W, "stamp": S,
            "length": torch.tensor(left, dtype=torch.int32, device="cuda")}
