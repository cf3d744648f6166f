"""Timed calls of the 4-bit cache and of eviction by accumulated attention weight, beside their plain forms.

Three kinds of work, as a program makes them:

  store   new rows of keys and values go into a cache held in 4 bits, and rows of it come out again as values
          (pc_q4_store, pc_q4_load)
  attn    queries over such a cache (pc_q4_attn): one token of each sequence, a few rows, a whole frame; with
          `weights` every key's attention weight is added to its running sum
  evict   a cache that has grown to Nk rows is cut to n_keep by those sums, in place (pc_evict for rows in bf16 or
          fp32, pc_q4_evict for rows in 4 bits)

A group of 32 neighbouring dims of a row shares the power of two 2^e, e the least integer for which the group's
largest magnitude is at most 7 * 2^e, from -120 to 125; an element is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times
2^e (ties to the even code).  The byte of the scale is e + 127; element 2i of a row is the low half of its byte i.

Head counts, frame sizes and cache lengths are those of this repository's configurations, tests and bench.py.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
FRAME_COST = 4 * 16 * 4032 * 29512 * 128    # flops of the largest listed attention


# ------------------------------------------------------------------------------ the cases
def listed() -> list[dict]:
    return [
        # one new token of a 28-layer stack with 4 KV heads, all layers in one call: launches are all there is
        dict(name="store_token_stack", kind="store", dtype="bf16", H=112, n=1, D=128),
        # one generated frame of 48 x 84 tokens enters the cache of a layer with 8 KV heads
        dict(name="store_frame", kind="store", dtype="bf16", H=8, n=4032, D=128),
        # frames of 24 x 42 tokens enter 28 layers x 4 heads, rows in fp32
        dict(name="store_stack_f32", kind="store", dtype="f32", H=112, n=1008, D=128),
        # one token over the packed cache of the small layer (ragged length): latency
        dict(name="token_attn_small", kind="attn", dtype="bf16", Hq=8, Hkv=2, D=128, n=1, Nk=1179, lse=False,
             weights=False, share=False, decay=1.0),
        # one token over the full cache of 48 frames: the cache's bytes
        dict(name="token_attn_long", kind="attn", dtype="bf16", Hq=16, Hkv=4, D=128, n=1, Nk=193792, lse=True,
             weights=False, share=False, decay=1.0),
        # one token over the packed cache of frame 48 in the 24/8-head layer, weights accumulated for the eviction
        dict(name="token_weights", kind="attn", dtype="bf16", Hq=24, Hkv=8, D=128, n=1, Nk=41800, lse=False,
             weights=True, share=False, decay=0.98),
        # a few rows at once (a block of text tokens) in fp32, D = 64, one sum for both heads
        dict(name="rows_f32_weights", kind="attn", dtype="f32", Hq=8, Hkv=2, D=64, n=37, Nk=1804, lse=True,
             weights=True, share=True, decay=1.0),
        # half-resolution frames over a packed cache of frame 24, weights accumulated over all rows
        dict(name="halfgrid_weights", kind="attn", dtype="bf16", Hq=16, Hkv=4, D=128, n=1008, Nk=7455, lse=True,
             weights=True, share=False, decay=0.9),
        # a whole frame over the packed cache of frame 24
        dict(name="frame_attn", kind="attn", dtype="bf16", Hq=16, Hkv=4, D=128, n=4032, Nk=29512, lse=False,
             weights=False, share=False, decay=1.0),
        # the small layer's 4-bit cache after a frame of 252 tokens has come in; the kept rows are read out
        dict(name="evict_small_q4", kind="evict", cache="q4", H=2, share=False, D=128, Nk=1431, n_keep=1179, n_anchor=40,
             recent=5),
        # steady state of token by token generation, 28 layers x 4 heads at once: one row in, one row out
        dict(name="evict_token_stack", kind="evict", cache="bf16", H=112, share=False, D=128, Nk=8321, n_keep=8320,
             n_anchor=256, recent=64),
        # the full cache of 48 frames cut to the size it is packed to
        dict(name="evict_layer", kind="evict", cache="bf16", H=4, share=False, D=128, Nk=193792, n_keep=41800,
             n_anchor=4288, recent=1),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng) -> dict:
    kind = rng.choice(["store", "attn", "attn", "evict"])
    D = rng.choice([64, 128, 128])
    if kind == "store":
        H = rng.choice([1, 2, 3, 4, 8, 112])
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), H=H, n=_spread(rng, 1, 112 * 1008 // H if H > 16 else 4032),
                    D=D)
    if kind == "attn":
        Hq, Hkv = rng.choice([(2, 1), (8, 2), (6, 2), (16, 4), (24, 8), (4, 4)])
        f32 = rng.random() < 0.3
        n = 1 if rng.random() < 0.4 else _spread(rng, 2, 300 if f32 else 4032)
        most = FRAME_COST // (4 * Hq * n * D) // (8 if f32 else 2)
        Nk = _spread(rng, 1, int(min(193792, max(1, most))))
        return dict(kind=kind, dtype="f32" if f32 else "bf16", Hq=Hq, Hkv=Hkv, D=D, n=n, Nk=Nk, lse=rng.random() < 0.5,
                    weights=rng.random() < 0.5, share=rng.random() < 0.3, decay=rng.choice([1.0, 0.98, 0.5]))
    H = rng.choice([1, 2, 4, 8, 112])
    Nk = _spread(rng, 2, 193792 if H <= 4 else 8321)
    n_keep = max(1, Nk - _spread(rng, 1, Nk - 1)) if rng.random() < 0.5 else rng.randint(1, Nk - 1)
    return dict(kind=kind, cache=rng.choice(["bf16", "f32", "q4"]) if H * Nk < 200000 else "bf16", H=H,
                share=rng.random() < 0.3, D=D, Nk=Nk, n_keep=n_keep,
                n_anchor=rng.choice([0, min(n_keep, rng.randint(1, 256))]), recent=rng.choice([0, 1, 64]))


# ------------------------------------------------------------------------------ inputs
def _rows(shape, gen, spread):
    """Rows of keys or values: N(0, 1) times a size of each channel (some channels of keys are far larger than
    others) and of each row."""
    x = torch.empty(shape, device=DEV).normal_(generator=gen)
    size = torch.exp(spread * torch.empty(shape[:-2] + (1, shape[-1]), device=DEV).normal_(generator=gen))
    return x.mul_(size)


def _pack(x):
    """Codes and scale bytes of rows x (finite), in the cache's layout."""
    g = x.float().unflatten(-1, (-1, 32))
    e = _exponent(g.abs().amax(-1))
    q = (_to_grid(torch.ldexp(g, -e[..., None])).abs() * 2).long()
    code = torch.tensor([0, 1, 2, 3, 4, 0, 5, 0, 6, 0, 0, 0, 7], device=x.device)[q] + 8 * torch.signbit(g).long()
    code = code.flatten(-2).unflatten(-1, (-1, 2))
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), (e + 127).to(torch.uint8)


def prepare(case: dict, seed: int):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, D = case["kind"], case["D"]
    st = dict(case=case)
    if kind == "store":
        H, n, dt = case["H"], case["n"], DTYPES[case["dtype"]]
        room, cap = (5, n + 9)       # the rows go behind 5 that are there
        st.update(K=_rows((H, n, D), gen, 0.8).to(dt), V=_rows((H, n, D), gen, 0.2).to(dt), row0=room,
                  cache=tuple(torch.zeros((H, cap, w), dtype=torch.uint8, device=DEV) for w in (D // 2, D // 32) * 2),
                  K_out=torch.empty((H, n, D), dtype=dt, device=DEV), V_out=torch.empty((H, n, D), dtype=dt, device=DEV))
        return st
    if kind == "attn":
        Hq, Hkv, n, Nk, dt = case["Hq"], case["Hkv"], case["n"], case["Nk"], DTYPES[case["dtype"]]
        K, V = _rows((Hkv, Nk, D), gen, 0.4), _rows((Hkv, Nk, D), gen, 0.2)
        Q = torch.empty((Hq, n, D), device=DEV).normal_(generator=gen)
        # each group of heads looks for a direction of its own, which some of its keys have: heavy hitters
        u = torch.empty((Hkv, 1, D), device=DEV).normal_(generator=gen) * D ** -0.5
        K += u * torch.empty((Hkv, Nk, 1), device=DEV).normal_(generator=gen) * 0.7
        Q += math.sqrt(D) * u.repeat_interleave(Hq // Hkv, 0)
        st.update(Q=Q.to(dt), cache=_pack(K) + _pack(V), scale=D ** -0.5, O=torch.empty((Hq, n, D), dtype=dt, device=DEV),
                  lse=torch.empty((Hq, n), device=DEV) if case["lse"] else None)
        if case["weights"]:
            hsel = 1 if case["share"] else Hkv
            st["w0"] = torch.empty((hsel, Nk), device=DEV).exponential_(Nk / 8, generator=gen)
            st["w"] = torch.empty_like(st["w0"])
        return st
    H, Nk = case["H"], case["Nk"]
    hsel = 1 if case["share"] else H
    K, V = _rows((H, Nk, D), gen, 0.8), _rows((H, Nk, D), gen, 0.2)
    st["rows"] = _pack(K) + _pack(V) if case["cache"] == "q4" else (K.to(DTYPES[case["cache"]]), V.to(DTYPES[case["cache"]]))
    if case["cache"] == "q4":
        st["out"] = tuple(torch.empty((H, case["n_keep"], D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    # coordinates (a row's place in time, a place in its frame) and weights in one buffer, so that one copy brings
    # both back to where they stood before the pass
    book = torch.empty((hsel * Nk * 4,), dtype=torch.int32, device=DEV)
    pos, w = book[:hsel * Nk * 3].view(hsel, Nk, 3), book[hsel * Nk * 3:].view(torch.float32).view(hsel, Nk)
    pos[..., 0] = torch.arange(Nk, device=DEV, dtype=torch.int32)
    pos[..., 1:] = torch.randint(0, 400, (hsel, Nk, 2), dtype=torch.int32, device=DEV, generator=gen)
    w.exponential_(1.0, generator=gen).mul_(torch.empty((hsel, Nk), device=DEV).normal_(generator=gen).exp_())
    w[torch.rand((hsel, Nk), device=DEV, generator=gen) < 0.05] = 0.0     # rows that nothing has looked at: ties
    st.update(book=book, book0=book.clone(), pos=pos, w=w)
    st["pos0"], st["w0"] = (st["book0"][:hsel * Nk * 3].view(hsel, Nk, 3),
                            st["book0"][hsel * Nk * 3:].view(torch.float32).view(hsel, Nk))
    return st


# ------------------------------------------------------------------------------ plain forms
def _exponent(a):
    """The least e with a <= 7 * 2^e, from -120 to 125."""
    m, x = torch.frexp(a)
    e = torch.where(m <= 0.875, x - 3, x - 2)
    return torch.where(a > 0, e, torch.full_like(e, -120)).clamp(-120, 125)


def _to_grid(v):
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp(max=6.0), v)


def _values(codes, scales):
    """What codes and scale bytes stand for, in fp32."""
    nibbles = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    return torch.ldexp(grid[nibbles].unflatten(-1, (-1, 32)), scales[..., None].int() - 127).flatten(-2)


def _round_trip(x):
    g = x.float().unflatten(-1, (-1, 32))
    e = _exponent(g.abs().amax(-1, keepdim=True))
    return torch.ldexp(_to_grid(torch.ldexp(g, -e)), e).flatten(-2).to(x.dtype)


def _attend(st):
    c, Q = st["case"], st["Q"]
    kc, ks, vc, vs = st["cache"]
    rows = Q.float().reshape(c["Hkv"], -1, c["D"])
    s = torch.matmul(rows, _values(kc, ks).transpose(1, 2)) * st["scale"]
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    del s
    l = p.sum(-1, keepdim=True)
    out = {"O": (torch.matmul(p, _values(vc, vs)) / l).reshape(Q.shape).to(Q.dtype)}
    if c["lse"]:
        out["lse"] = (m + torch.log(l)).reshape(Q.shape[:2])
    if c["weights"]:
        mass = (p / l).sum(1)
        out["w"] = c["decay"] * st["w0"] + (mass.sum(0, keepdim=True) if c["share"] else mass)
    return out


def _kept_rows(pos, w, c):
    """Which row stands where after the eviction: [Hsel][n_keep]."""
    Nk, n_keep = c["Nk"], c["n_keep"]
    j = torch.arange(Nk, device=w.device)
    safe = (j < c["n_anchor"]) | (pos[..., 0] > pos[:, -1:, 0] - c["recent"])
    rank = torch.where(safe, math.inf, w)
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices
    keep = torch.zeros_like(safe).scatter_(1, order[:, :n_keep], True)
    hole = ~keep[:, :n_keep]
    movers = torch.sort((~keep[:, n_keep:]).int(), dim=1, stable=True).indices + n_keep     # kept rows first, ascending
    nth = (torch.cumsum(hole.int(), 1) - 1).clamp(0, Nk - n_keep - 1)
    return torch.where(hole, movers.gather(1, nth), j[:n_keep])


def _evict(st):
    c, H = st["case"], st["case"]["H"]
    src = _kept_rows(st["pos0"], st["w0"], c)
    of_head = src.expand(H, -1)[..., None]
    rows = st["rows"]
    if c["cache"] == "q4":
        rows = tuple(_values(rows[i], rows[i + 1]).to(torch.bfloat16) for i in (0, 2))
    K, V = (x.gather(1, of_head.expand(-1, -1, c["D"])) for x in rows)
    return {"K": K, "V": V, "pos": st["pos0"].gather(1, src[..., None].expand(-1, -1, 3)), "w": st["w0"].gather(1, src)}


def run(st):
    c = st["case"]
    if not own:
        if c["kind"] == "store":
            return {"K": _round_trip(st["K"]), "V": _round_trip(st["V"])}
        return _attend(st) if c["kind"] == "attn" else _evict(st)

    import paper_2601_04359_amd as pk
    if c["kind"] == "store":
        pk.pc_q4_store(st["K"], st["V"], st["cache"], st["row0"])
        pk.pc_q4_load(st["cache"], st["row0"], st["K_out"], st["V_out"])
        return {"K": st["K_out"], "V": st["V_out"]}
    if c["kind"] == "attn":
        w = None
        if c["weights"]:
            w = st["w"].copy_(st["w0"])     # the sums as they stood before this token
        out = {"O": pk.pc_q4_attn(st["Q"], st["cache"], c["Nk"], st["scale"], O=st["O"], lse=st["lse"], weights=w,
                                  decay=c["decay"])}
        if c["lse"]:
            out["lse"] = st["lse"]
        if c["weights"]:
            out["w"] = w
        return out
    # coordinates and sums as they stood; the rows of K and V need no such copy: rows move from n_keep on to below it,
    # and a second eviction by the same sums moves the same ones to the same places
    st["book"].copy_(st["book0"])
    n = c["n_keep"]
    if c["cache"] == "q4":
        pk.pc_q4_evict(st["rows"], st["pos"], st["w"], c["Nk"], n, n_anchor=c["n_anchor"], recent_t=c["recent"])
        K, V = pk.pc_q4_load(st["rows"], 0, *st["out"])
    else:
        pk.pc_evict(*st["rows"], st["pos"], st["w"], c["Nk"], n, n_anchor=c["n_anchor"], recent_t=c["recent"])
        K, V = (x[:, :n] for x in st["rows"])
    return {"K": K, "V": V, "pos": st["pos"][:, :n], "w": st["w"][:, :n]}


# ------------------------------------------------------------------------------ work
def work(case: dict) -> dict:
    D = case["D"]
    packed = D // 2 + D // 32
    if case["kind"] == "store":
        size = {"bf16": 2, "f32": 4}[case["dtype"]]
        # in: rows read, codes written; out: the same the other way round
        return {"bytes": 2 * 2 * case["H"] * case["n"] * (D * size + packed), "flops": 2 * case["H"] * case["n"] * D}
    if case["kind"] == "attn":
        size = {"bf16": 2, "f32": 4}[case["dtype"]]
        Hq, Hkv, n, Nk = case["Hq"], case["Hkv"], case["n"], case["Nk"]
        data = 2 * Hkv * Nk * packed + 2 * Hq * n * D * size + (4 * Hq * n if case["lse"] else 0)
        if case["weights"]:
            data += 2 * 4 * Nk * (1 if case["share"] else Hkv)
        return {"bytes": data, "flops": 4 * Hq * n * Nk * D}
    H, Nk, n = case["H"], case["Nk"], case["n_keep"]
    hsel = 1 if case["share"] else H
    moved = (Nk - n) * n / Nk       # rows from n_keep on that are kept, of rows kept without order
    row = {"q4": packed, "bf16": 2 * D, "f32": 4 * D}[case["cache"]]
    data = 4 * hsel * Nk + (4 * hsel * Nk if case["recent"] else 0) + 2 * moved * (2 * row * H + 16 * hsel)
    if case["cache"] == "q4":
        data += 2 * H * n * (packed + 2 * D)
    return {"bytes": int(data), "flops": hsel * Nk}


# ------------------------------------------------------------------------------ in 64 bits
def _exact_grid(x):
    """The 4-bit value of every element, found by comparing distances in 64 bits."""
    g = x.double().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 7)).clamp(-120, 125)
    e = torch.where(top > 7 * torch.exp2(e), e + 1, e)                       # the logarithm may be off beside a border
    e = torch.where((top <= 7 * torch.exp2(e - 1)) & (e > -120), e - 1, e).clamp(-120, 125)
    v = (g / torch.exp2(e)).abs()
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    border = (grid[1:] + grid[:-1]) / 2
    code = (v[..., None] > border).sum(-1)                                   # below or at a border: the lower one ...
    tie = (v[..., None] == border).any(-1)
    code = torch.where(tie & (code % 2 == 1), code + 1, code)                # ... but at a border the even one
    return (grid[code] * torch.sign(g) * torch.exp2(e)).flatten(-2)


def _exact_values(codes, scales):
    low = codes.to(torch.int64)
    sign_and_code = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.int64, device=codes.device)
    sign_and_code[..., 0::2], sign_and_code[..., 1::2] = low % 16, low // 16
    grid = torch.tensor(GRID, dtype=torch.float64, device=codes.device)
    v = grid[sign_and_code % 8] * (1 - 2 * (sign_and_code // 8)).double()
    return v * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def exact(case: dict, seed: int):
    st = prepare(case, seed)
    if case["kind"] == "store":
        parts = {"K": [], "V": []}
        for name in parts:
            for h in range(case["H"]):
                parts[name].append(_exact_grid(st[name][h]))
        return {name: torch.stack(p) for name, p in parts.items()}
    if case["kind"] == "attn":
        Hq, Hkv, D, Nk = case["Hq"], case["Hkv"], case["D"], case["Nk"]
        rep = Hq // Hkv
        O, lse = torch.empty(st["Q"].shape, dtype=torch.float64, device=DEV), torch.empty(st["Q"].shape[:2], dtype=torch.float64, device=DEV)
        w = torch.zeros((Hkv, Nk), dtype=torch.float64, device=DEV)
        for g in range(Hkv):
            k, v = _exact_values(st["cache"][0][g], st["cache"][1][g]), _exact_values(st["cache"][2][g], st["cache"][3][g])
            kt = k.t().contiguous()
            for h in range(g * rep, (g + 1) * rep):
                logits = torch.mm(st["Q"][h].double(), kt) * st["scale"]
                lse[h] = torch.logsumexp(logits, 1)
                p = torch.exp(logits - lse[h][:, None])
                O[h] = torch.mm(p, v)
                w[g] += p.sum(0)
                del logits, p
        out = {"O": O}
        if case["lse"]:
            out["lse"] = lse
        if case["weights"]:
            out["w"] = case["decay"] * st["w0"].double() + (w.sum(0, keepdim=True) if case["share"] else w)
        return out
    Nk, n = case["Nk"], case["n_keep"]
    pos, w = st["pos0"].cpu().numpy(), st["w0"].cpu().numpy()
    rows = st["rows"]
    if case["cache"] == "q4":
        rows = (_exact_values(rows[0], rows[1]), _exact_values(rows[2], rows[3]))
    out = {"K": [], "V": [], "pos": [], "w": []}
    for s in range(w.shape[0]):
        level = np.zeros(Nk, np.int64)
        level[:case["n_anchor"]] = 1
        level[pos[s, :, 0].astype(np.int64) > int(pos[s, Nk - 1, 0]) - case["recent"]] = 1
        best = np.lexsort((np.arange(Nk), np.where(level == 1, 0.0, -w[s].astype(np.float64)), -level))[:n]
        kept = set(best.tolist())
        movers = iter(sorted(r for r in kept if r >= n))
        src = torch.tensor([r if r in kept else next(movers) for r in range(n)], device=DEV)
        out["pos"].append(st["pos0"][s][src])
        out["w"].append(st["w0"][s][src])
        for h in range(rows[0].shape[0]) if case["share"] else (s,):
            out["K"].append(rows[0][h][src])
            out["V"].append(rows[1][h][src])
    return {name: torch.stack(p) for name, p in out.items()}
