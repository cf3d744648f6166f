"""Timed calls of the operators that serve several sequences from one memory, beside their plain forms.

Three kinds of work, as a program makes them:

  prompt  causal attention over whole prompts, packed one behind the other (pc_prompt_attn).  Row i of a sequence with
          nq queries and nk keys sees keys 0 .. nk - nq + i
  store   the rows of a step go into a cache held in pages, keys and queries rotated by their (t, h, w) on the way
          (pc_page_store).  The last row of sequence s becomes its row lens[s] - 1
  attn    the rows of a step attend over that cache (pc_page_attn); the first n_shared rows of all sequences are the
          same pages, read once for all

The rotation turns dims (2i, 2i + 1) of a section of width w by pos_axis * 10000^(-2i/w).  Head counts, frame sizes and
cache lengths are those of this repository's configurations, tests and bench.py, or generic.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SECTIONS = {128: (32, 48, 48), 64: (16, 24, 24)}
BASE = 10000.0
LONGEST = 16384      # rows of the largest listed prompt, with 24 heads


# ------------------------------------------------------------------------------ the cases
def listed() -> list[dict]:
    return [
        # the small layer's text prompt: launches and latency are all there is
        dict(name="prompt_text", kind="prompt", dtype="bf16", Hq=8, Hkv=2, D=128, nq="40", nk="", lse=False),
        # prompts of ten requests at once, from none and one token to a frame's half
        dict(name="prompt_ragged", kind="prompt", dtype="bf16", Hq=16, Hkv=4, D=128, nq="1,17,256,300,1000,2049,777,64,0,5",
             nk="", lse=True),
        # 256 text tokens and the conditioning image of 48 x 84 tokens as one prompt
        dict(name="prompt_image", kind="prompt", dtype="bf16", Hq=16, Hkv=4, D=128, nq="4288", nk="", lse=False),
        # a long document in front of a video, in the rollout's 24/8-head layer
        dict(name="prompt_long", kind="prompt", dtype="bf16", Hq=24, Hkv=8, D=128, nq="16384", nk="", lse=False),
        # prompts that come in pieces: the rows in front are there already
        dict(name="prompt_pieces", kind="prompt", dtype="bf16", Hq=16, Hkv=4, D=128, nq="512,100,1008", nk="4288,612,1008",
             lse=True),
        # the correctness tier
        dict(name="prompt_f32", kind="prompt", dtype="f32", Hq=8, Hkv=2, D=128, nq="40,252,333,1", nk="", lse=True),
        # one token of each of 64 sequences
        dict(name="store_tokens", kind="store", dtype="bf16", Hq=16, Hkv=4, D=128, page=64, before=",".join(
            str(300 + 37 * i) for i in range(64)), n="1", keep=False),
        # prompts of eight requests enter the cache; their rotated keys are kept for the attention over them as well
        dict(name="store_prompts", kind="store", dtype="bf16", Hq=24, Hkv=8, D=128, page=128, before="0,0,0,0,512,0,64,0",
             n="256,1000,40,4032,333,1,1808,999", keep=True),
        # a token of each of 8 sequences of the small layer's lengths: latency
        dict(name="tokens_small", kind="attn", dtype="bf16", Hq=8, Hkv=2, D=128, page=64, n="1",
             lens="1179,40,292,544,1,796,1048,1300", n_shared=0),
        # a token of each of 16 sequences of very different lengths, up to the packed cache of frame 24
        dict(name="tokens_long", kind="attn", dtype="bf16", Hq=24, Hkv=8, D=128, page=256, n="1",
             lens="29512,16,4288,8191,256,20000,1000,12345,29000,7455,64,15000,4032,2200,25000,1", n_shared=0),
        # 64 continuations of one video: the packed cache of frame 48 is common to all, up to 512 rows are not
        dict(name="branches_tokens", kind="attn", dtype="bf16", Hq=16, Hkv=4, D=128, page=64, n="1",
             lens=",".join(str(41800 + 8 * (i + 1)) for i in range(64)), n_shared=41800),
        # eight continuations take a block of 64 rows each behind the packed cache of frame 24
        dict(name="branches_blocks", kind="attn", dtype="bf16", Hq=16, Hkv=4, D=128, page=128, n="64",
             lens=",".join(str(29512 + 64 * (1 + i % 4)) for i in range(8)), n_shared=29512),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _text(numbers) -> str:
    return ",".join(str(int(v)) for v in numbers)


def _numbers(text: str) -> list[int]:
    return [int(v) for v in text.split(",")] if text else []


def draw(rng) -> dict:
    kind = rng.choice(["prompt", "prompt", "store", "attn", "attn"])
    Hq, Hkv = rng.choice([(2, 1), (8, 2), (6, 2), (16, 4), (24, 8), (4, 4)])
    f32 = rng.random() < 0.25
    D = rng.choice([64, 128, 128])
    c = dict(kind=kind, dtype="f32" if f32 else "bf16", Hq=Hq, Hkv=Hkv, D=D)
    if kind == "prompt":
        n_seq = rng.choice([1, 1, 2, 3, 8, 30])
        most = (1200 if f32 or D == 64 else 5000) // (1 if n_seq < 8 else 4)
        nq = [_spread(rng, 1, most) for _ in range(n_seq)]
        nk = []
        if rng.random() < 0.4:
            nk = [q + rng.choice([0, _spread(rng, 1, most)]) for q in nq]
        return dict(c, nq=_text(nq), nk=_text(nk), lse=rng.random() < 0.5)
    c["page"] = rng.choice([64, 128, 256])
    n_seq = _spread(rng, 1, 100)
    if kind == "store":
        if rng.random() < 0.5:
            n, before = [rng.choice([1, 1, 2, 5])], [_spread(rng, 1, 3000) for _ in range(n_seq)]
        else:
            n = [_spread(rng, 1, 4032 if n_seq < 5 else 300) for _ in range(n_seq)]
            before = [rng.choice([0, _spread(rng, 1, 600)]) for _ in n]
        return dict(c, n=_text(n), before=_text(before), keep=rng.random() < 0.5)
    n_shared = rng.choice([0, 0, _spread(rng, 1, 41800 // (8 if f32 or D == 64 else 1))])
    if rng.random() < 0.7:
        n = [1] if rng.random() < 0.7 else [_spread(rng, 1, min(64, 2000 // n_seq))]
        rows = n * n_seq
    else:
        rows = n = [_spread(rng, 1, min(200, 2000 // n_seq)) for _ in range(n_seq)]
    most = 4096 // (8 if f32 or D == 64 else 1)
    if n_shared == 0 and n_seq <= 16 and len(n) == 1 and n[0] == 1:
        most = 29512
    lens = [n_shared + r + rng.choice([0, _spread(rng, 1, most)]) for r in rows]
    return dict(c, n=_text(n), lens=_text(lens), n_shared=n_shared)


def _rows(case) -> list[int]:
    """New rows of every sequence of a store or attn case: one number stands for all."""
    n, n_seq = _numbers(case["n"]), len(_numbers(case["before"] if case["kind"] == "store" else case["lens"]))
    return n * n_seq if len(n) == 1 else n


def _offsets(counts) -> list[int]:
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


# ------------------------------------------------------------------------------ inputs
def _normal(shape, gen):
    return torch.empty(shape, device=DEV).normal_(generator=gen)


def _q_and_k(Hq, Hkv, n, gen, D):
    """Queries for n keys' worth of heads: each group of heads looks for a direction of its own."""
    u = _normal((Hkv, 1, D), gen) * D ** -0.5
    return u, _normal((Hq, n, D), gen) + math.sqrt(D) * u.repeat_interleave(Hq // Hkv, 0)


def _pages(lens, page, gen, first=()):
    """Page numbers of every sequence, in no order; `first`: pages that all of them begin with.  A page that is only
    partly common is a copy in every sequence."""
    need = [max(0, -(-n // page) - len(first)) for n in lens]
    free = torch.randperm(sum(need) + 3, generator=torch.Generator().manual_seed(int(gen.initial_seed()))) + len(first)
    table = torch.zeros((len(lens), max(1, len(first) + max(need))), dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :len(first)] = torch.tensor(list(first), dtype=torch.int32)
        table[s, len(first):len(first) + n] = free[at:at + n]
        at += n
    return table, len(first) + sum(need) + 3


def prepare(case: dict, seed: int):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    Hq, Hkv, D, dt = case["Hq"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
    st = dict(case=case, scale=D ** -0.5)
    if case["kind"] == "prompt":
        nq = _numbers(case["nq"])
        nk = _numbers(case["nk"]) or nq
        Tq, Tk = sum(nq), sum(nk)
        u, Q = _q_and_k(Hq, Hkv, Tq, gen, D)
        K = _normal((Hkv, Tk, D), gen) + u * _normal((Hkv, Tk, 1), gen) * 0.7
        st.update(Q=Q.to(dt), K=K.to(dt), V=_normal((Hkv, Tk, D), gen).to(dt), offs_q=_offsets(nq),
                  offs_k=_offsets(nk) if case["nk"] else None, O=torch.empty((Hq, Tq, D), dtype=dt, device=DEV),
                  lse=torch.empty((Hq, Tq), device=DEV) if case["lse"] else None)
        return st
    page, rows = case["page"], _rows(case)
    T = sum(rows)
    st["offs_host"] = _offsets(rows)
    st["offs"] = None if len(_numbers(case["n"])) == 1 else st["offs_host"]
    if case["kind"] == "store":
        lens = [b + n for b, n in zip(_numbers(case["before"]), rows)]
        table, n_pages = _pages(lens, page, gen)
        pos = torch.empty((T, 3), dtype=torch.int32)
        for s, n in enumerate(rows):      # a frame's tokens: 8 rows and columns apart, every 84 a row, 4032 a frame
            i = torch.arange(lens[s] - n, lens[s])
            pos[st["offs_host"][s]:st["offs_host"][s + 1]] = torch.stack((256 + 4 * (i // 4032), 8 * (i % 4032 // 84), 8 * (i % 84)), 1)
        st.update(K=_normal((Hkv, T, D), gen).to(dt), V=_normal((Hkv, T, D), gen).to(dt), Q=_normal((Hq, T, D), gen).to(dt),
                  pos=pos.to(DEV), q_scale=st["scale"] * 1.4426950408889634,
                  Q_out=torch.empty((Hq, T, D), dtype=dt, device=DEV),
                  K_out=torch.empty((Hkv, T, D), dtype=dt, device=DEV) if case["keep"] else None)
    else:
        lens, ns = _numbers(case["lens"]), case["n_shared"]
        whole = ns // page       # pages that are common as they are
        table, n_pages = _pages(lens, page, gen, first=range(whole))
        u, Q = _q_and_k(Hq, Hkv, T, gen, D)
        st.update(Q=Q.to(dt), u=u, O=torch.empty((Hq, T, D), dtype=dt, device=DEV), max_len=max(lens))
    K, V = (_normal((n_pages, Hkv, page, D), gen) for _ in range(2))
    if case["kind"] == "attn":
        K += st.pop("u") * _normal((n_pages, Hkv, page, 1), gen) * 0.7
        if ns % page:            # the page that is common in part: every sequence has its copy of the common rows
            common = table[:, whole].long().to(DEV)
            for x in (K, V):
                x[common, :, :ns % page] = x[common[0], :, :ns % page]
        st["shared"] = table[0, :-(-ns // page)].to(DEV) if ns else None
    st.update(pages=(K.to(dt), V.to(dt)), table=table.to(DEV), lens=torch.tensor(lens, dtype=torch.int32, device=DEV), lens_host=lens)
    return st


# ------------------------------------------------------------------------------ plain forms
def _attend(q, k, v, scale, shift):
    """q [rep][nq][D] over k, v [nk][D], all fp32; row i sees keys up to shift + i -> (O, lse)."""
    rep, nq, D = q.shape
    s = torch.matmul(q.reshape(rep * nq, D), k.t().contiguous()).reshape(rep, nq, -1) * scale
    if shift < k.shape[0] - 1:
        seen = torch.arange(k.shape[0], device=k.device) <= shift + torch.arange(nq, device=k.device)[:, None]
        s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    del s
    l = p.sum(-1, keepdim=True)
    return torch.matmul(p.reshape(rep * nq, -1), v).reshape(rep, nq, D) / l, (m + torch.log(l))[..., 0]


def _turn(x, pos, scale):
    """Rows x [H][T][D] rotated by pos, times scale, in fp32; angles in 64 bits."""
    D = x.shape[-1]
    freq = torch.cat([BASE ** (-torch.arange(0, w, 2, dtype=torch.float64, device=x.device) / w) for w in SECTIONS[D]])
    axis = torch.cat([torch.full((w // 2,), a, device=x.device) for a, w in enumerate(SECTIONS[D])])
    ang = pos.double()[:, axis] * freq
    c, s = (torch.cos(ang) * scale).float(), (torch.sin(ang) * scale).float()
    a, b = x.float().unflatten(-1, (-1, 2)).unbind(-1)
    return torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2).to(x.dtype)


def _places(st):
    """(page, row in it) of every new row."""
    page = st["case"]["page"]
    s_of = torch.repeat_interleave(torch.arange(len(st["lens_host"])), torch.tensor(_rows(st["case"]))).to(DEV)
    ends = torch.tensor(st["offs_host"][1:], device=DEV)[s_of]
    at = st["lens"].long()[s_of] - ends + torch.arange(len(s_of), device=DEV)
    return st["table"].long()[s_of, at // page], at % page


def _plain(st):
    c = st["case"]
    Hkv, rep = c["Hkv"], c["Hq"] // c["Hkv"]
    if c["kind"] == "store":
        k, q = _turn(st["K"], st["pos"], 1.0), _turn(st["Q"], st["pos"], st["q_scale"])
        at = _places(st)
        K, V = st["pages"]
        K[at[0], :, at[1]] = k.transpose(0, 1)
        V[at[0], :, at[1]] = st["V"].transpose(0, 1)
        return dict({"K": K, "V": V, "Q": q}, **({"K_out": k} if c["keep"] else {}))
    Q = st["Q"]
    O, lse = torch.empty_like(Q), torch.empty(Q.shape[:2], device=DEV)
    if c["kind"] == "prompt":
        offs_q, offs_k = st["offs_q"], st["offs_k"] or st["offs_q"]
    else:
        offs_q = st["offs_host"]
    for s in range(len(offs_q) - 1):
        a, b = offs_q[s], offs_q[s + 1]
        if a == b:
            continue
        if c["kind"] == "prompt":
            k, v = (st[x][:, offs_k[s]:offs_k[s + 1]] for x in "KV")
        else:
            n = st["lens_host"][s]
            ids = st["table"][s, :-(-n // c["page"])].long()
            k, v = (x[ids].transpose(0, 1).flatten(1, 2)[:, :n] for x in st["pages"])
        for g in range(Hkv):
            h = slice(g * rep, (g + 1) * rep)
            o, e = _attend(Q[h, a:b].float(), k[g].float(), v[g].float(), st["scale"], k.shape[1] - (b - a))
            O[h, a:b], lse[h, a:b] = o.to(Q.dtype), e
    return dict({"O": O}, **({"lse": lse} if c.get("lse") else {}))


def run(st):
    if not own:
        return _plain(st)
    import paper_2601_04359_amd as pk
    c = st["case"]
    if c["kind"] == "prompt":
        pk.pc_prompt_attn(st["Q"], st["K"], st["V"], st["scale"], st["offs_q"], st["offs_k"], O=st["O"], lse=st["lse"])
        return dict({"O": st["O"]}, **({"lse": st["lse"]} if c["lse"] else {}))
    if c["kind"] == "store":
        pk.pc_page_store(st["K"], st["V"], st["pages"], st["table"], st["lens"], offs=st["offs"], pos=st["pos"],
                         sections=SECTIONS[c["D"]], base=BASE, K_out=st["K_out"], Q=st["Q"], Q_out=st["Q_out"],
                         out_scale=st["q_scale"])
        return dict({"K": st["pages"][0], "V": st["pages"][1], "Q": st["Q_out"]}, **({"K_out": st["K_out"]} if c["keep"] else {}))
    pk.pc_page_attn(st["Q"], st["pages"], st["table"], st["lens"], st["max_len"], st["scale"], offs=st["offs"],
                    shared=st["shared"], n_shared=c["n_shared"], O=st["O"])
    return {"O": st["O"]}


# ------------------------------------------------------------------------------ work
def _pairs(nq: int, nk: int) -> int:
    """(query, key) pairs of a sequence: row i sees nk - nq + i + 1 keys."""
    return nq * (nk - nq) + nq * (nq + 1) // 2


def work(case: dict) -> dict:
    Hq, Hkv, D, size = case["Hq"], case["Hkv"], case["D"], {"bf16": 2, "f32": 4}[case["dtype"]]
    if case["kind"] == "prompt":
        nq = _numbers(case["nq"])
        nk = _numbers(case["nk"]) or nq
        data = 2 * D * size * (Hq * sum(nq) + Hkv * sum(nk)) + (4 * Hq * sum(nq) if case["lse"] else 0)
        return {"bytes": data, "flops": 4 * Hq * D * sum(_pairs(a, b) for a, b in zip(nq, nk))}
    rows = _rows(case)
    T = sum(rows)
    if case["kind"] == "store":
        return {"bytes": T * (D * size * (4 * Hkv + 2 * Hq + (Hkv if case["keep"] else 0)) + 12), "flops": 3 * T * D * (Hq + Hkv)}
    lens, ns = _numbers(case["lens"]), case["n_shared"]
    keys = ns + sum(n - ns for n in lens)
    return {"bytes": 2 * D * size * (Hq * T + Hkv * keys), "flops": 4 * Hq * D * sum(_pairs(a, b) for a, b in zip(rows, lens))}


# ------------------------------------------------------------------------------ in 64 bits
def _exact_turn(x, pos, scale):
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    at = 0
    for axis, w in enumerate(SECTIONS[x.shape[-1]]):
        for i in range(w // 2):
            ang = pos[:, axis].double() * math.pow(BASE, -2.0 * i / w)
            a, b = x[..., at].double(), x[..., at + 1].double()
            out[..., at] = scale * (a * torch.cos(ang) - b * torch.sin(ang))
            out[..., at + 1] = scale * (a * torch.sin(ang) + b * torch.cos(ang))
            at += 2
    return out


def _exact_rows(q, k, v, scale, first):
    """One head: row i of q sees the first first + i keys; blocks of rows at a time."""
    o, e = [], []
    k, v = k.double(), v.double()
    kt = k.t().contiguous()
    for a in range(0, q.shape[0], 2048):
        z = torch.mm(q[a:a + 2048].double(), kt) * scale
        hidden = torch.arange(k.shape[0], device=k.device)[None] >= first + a + torch.arange(z.shape[0], device=k.device)[:, None]
        z.masked_fill_(hidden, -math.inf)
        e.append(torch.logsumexp(z, 1))
        o.append(torch.mm(torch.exp(z - e[-1][:, None]), v))
    return torch.cat(o), torch.cat(e)


def exact(case: dict, seed: int):
    st = prepare(case, seed)
    Hq, Hkv = case["Hq"], case["Hkv"]
    if case["kind"] == "store":
        k = _exact_turn(st["K"], st["pos"], 1.0)
        K, V = (x.double() for x in st["pages"])
        table, page = st["table"].cpu().tolist(), case["page"]
        for s, n in enumerate(_rows(case)):
            for i in range(n):
                t, j = st["offs_host"][s] + i, st["lens_host"][s] - n + i
                K[table[s][j // page], :, j % page] = k[:, t]
                V[table[s][j // page], :, j % page] = st["V"][:, t].double()
        out = {"K": K, "V": V, "Q": _exact_turn(st["Q"], st["pos"], st["q_scale"])}
        if case["keep"]:
            out["K_out"] = k
        return out
    O = torch.empty(st["Q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(st["Q"].shape[:2], dtype=torch.float64, device=DEV)
    counts = _numbers(case["nq"]) if case["kind"] == "prompt" else _rows(case)
    keys = (_numbers(case["nk"]) or counts) if case["kind"] == "prompt" else st["lens_host"]
    a = ka = 0
    for s, (n, m) in enumerate(zip(counts, keys)):
        for h in range(Hq if n else 0):
            g = h * Hkv // Hq
            if case["kind"] == "prompt":
                k, v = st["K"][g, ka:ka + m], st["V"][g, ka:ka + m]
            else:
                at = [int(p) for p in st["table"][s].cpu()][:(m + case["page"] - 1) // case["page"]]
                k, v = (torch.cat([x[p, g] for p in at])[:m] for x in st["pages"])
            O[h, a:a + n], lse[h, a:a + n] = _exact_rows(st["Q"][h, a:a + n], k, v, st["scale"], m - n + 1)
        a, ka = a + n, ka + m
    return dict({"O": O}, **({"lse": lse} if case.get("lse") else {}))
