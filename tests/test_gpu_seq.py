"""Prompts, a cache in pages and its attention (pc_prompt_attn, pc_page_store, pc_page_attn) against plain 64-bit forms.

Stored rows have to be equal bit for bit to what pc_rope3d makes of them.  Tolerances of the attention, element by element,
with u = 2^-24 (half a step of fp32), A = the largest sum_d |q_d k_d| * scale that a row meets, in units of the logits:
  * a logit: D products summed in fp32 in any order, the scale folded into base 2 (three roundings), the subtraction
    of the reference: |ds| <= (D + 8) u A; the exponential adds a step of its result (2 u) and its argument's rounding, up
    to u * 2 A * log2(e).  A probability is off by a factor of at most 1 + e, e = (D + 16) u A + 8 u.
  * O, fp32 inputs: (2 e + (Nk + 64) u) sum_j p_j |v_j|: probability and normaliser, sums of Nk terms, merges.
  * O, bf16 inputs: the probabilities are rounded to bf16 before the second product and O at the end, half a step each:
    2^-8 (|O| + sum_j p_j |v_j|) more.
  * lse: (D + 16) u A + (|lse| + Nk + 64) u.
(Nk u is the worst case of a serial sum.)
"""
import numpy as np
import pytest
import torch

import paper_2601_04359_amd as pk
from paper_2601_04359_amd.rollout import PagedStack

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SECTIONS = {128: (32, 48, 48), 64: (16, 24, 24)}
NAN = float("nan")


def offsets(counts, start=0):
    return [start + int(v) for v in np.concatenate([[0], np.cumsum(counts)])]


def normal(gen, *shape):
    return torch.empty(shape, device=DEV).normal_(generator=gen)


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def check_rows(dtype, got, got_lse, q, k, v, scale, first):
    """One head: row i of q [nq][D] sees keys below first + i of k, v [nk][D]; got [nq][D], got_lse [nq] or None."""
    nq, D = q.shape
    nk = k.shape[0]
    q, k, v, got = (x.detach().double() for x in (q, k, v, got))
    seen = torch.arange(nk, device=DEV)[None] < first + torch.arange(nq, device=DEV)[:, None]
    none = ~seen.any(1)
    assert (got[none] == 0).all()
    if got_lse is not None:
        assert (got_lse[none] == -float("inf")).all()
    if none.all():
        return
    z = torch.where(seen, q @ k.t().contiguous() * scale, -float("inf"))[~none]
    size = torch.where(seen, q.abs() @ k.abs().t().contiguous() * scale, 0.0)[~none].amax(1)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    O, mass = p @ v, p @ v.abs()
    e = ((D + 16) * U * size + 8 * U)[:, None]
    tol = (2 * e + (nk + 64) * U) * mass
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (O.abs() + mass)
    err = (got[~none] - O).abs()
    assert (err <= tol).all(), f"O off by {(err / tol).max().item():.2f} tolerances"
    if got_lse is not None:
        tol = (D + 16) * U * size + (lse.abs() + nk + 64) * U
        err = (got_lse[~none].double() - lse).abs()
        assert (err <= tol).all(), f"lse off by {(err / tol).max().item():.2f} tolerances"


# ------------------------------------------------------------------------------ prompts
def run_prompt(dtype, Hq, Hkv, D, nq, nk=None, *, seed=0, scale=None, start=0, spare=3, lse=True, make=None):
    """Packed prompts with `start` rows of nobody in front and `spare` behind, gaps between heads; checks every sequence."""
    gen, dt = generator(seed + sum(nq) * 7 + D), TYPES[dtype]
    scale = D ** -0.5 if scale is None else scale
    oq = offsets(nq, start)
    ok = None if nk is None else offsets(nk, 2)
    Tq, Tk = oq[-1] + spare, (oq[-1] if ok is None else ok[-1]) + spare
    Q = normal(gen, Hq, Tq + 1, D).to(dt)[:, :Tq]
    big = normal(gen, Hkv, Tk + 5, D), normal(gen, Hkv, Tk + 2, D)
    K, V = big[0].to(dt)[:, 2:Tk + 2], big[1].to(dt)[:, :Tk]
    if make is not None:
        make(Q, K, V)
    kq = oq if ok is None else ok
    for x in (K, V):      # rows of nobody
        x[:, :kq[0]], x[:, kq[-1]:] = NAN, NAN
    O = torch.full((Hq, Tq + 2, D), 7.0, dtype=dt, device=DEV)[:, :Tq]
    L = torch.full((Hq, Tq), 7.0, device=DEV) if lse else None
    got = pk.pc_prompt_attn(Q, K, V, scale, oq, ok, O=O, lse=L)
    assert got is O
    for s in range(len(nq)):
        a, b = oq[s], oq[s + 1]
        for h in range(Hq if b > a else 0):
            g = h // (Hq // Hkv)
            k, v = K[g, kq[s]:kq[s + 1]], V[g, kq[s]:kq[s + 1]]
            check_rows(dtype, O[h, a:b], None if L is None else L[h, a:b], Q[h, a:b], k, v, scale, k.shape[0] - (b - a) + 1)
    for rest in (slice(0, oq[0]), slice(oq[-1], Tq)):
        assert (O[:, rest] == 7.0).all() and (L is None or (L[:, rest] == 7.0).all())
    return Q, K, V, O, L


HEADS = [(2, 1), (8, 2), (6, 2), (4, 4), (5, 1)]


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
@pytest.mark.parametrize("nq", [[1], [17], [33, 1, 0, 5], [64, 63, 65, 127, 129], [300, 1], [0, 0, 2, 0]])
def test_prompt(dtype, D, Hq, Hkv, nq):
    run_prompt(dtype, Hq, Hkv, D, nq, start=len(nq) - 1)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("nq,nk", [([1], [1000]), ([5, 40], [700, 41]), ([64, 64], [64, 65]), ([7, 3, 200], [5, 0, 190]), ([100], [300]),
                                   ([3], [0]), ([130, 20, 1], [129, 500, 63])])
def test_prompt_with_other_keys(dtype, D, nq, nk):
    run_prompt(dtype, 8, 2, D, nq, nk)


@pytest.mark.parametrize("dtype,Hq,Hkv,nq", [("bf16", 4, 1, [1500]), ("bf16", 16, 4, [2049]), ("bf16", 24, 8, [777, 1300]), ("bf16", 16, 4, [4500]),
                                             ("bf16", 3, 3, [3001]), ("f32", 2, 1, [1100]), ("bf16", 32, 2, [600, 601, 3, 90])])
def test_prompt_long(dtype, Hq, Hkv, nq):
    run_prompt(dtype, Hq, Hkv, 128, nq)


@pytest.mark.parametrize("n_seq", [64, 65, 150])
def test_prompt_of_many_sequences(n_seq):
    rng = np.random.default_rng(n_seq)
    nq = [int(v) for v in rng.integers(0, 40, n_seq)]
    run_prompt("bf16", 4, 2, 128, nq, lse=n_seq != 65)
    run_prompt("bf16", 4, 2, 128, nq, [max(0, n + int(d)) for n, d in zip(nq, rng.integers(-3, 30, n_seq))])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,at", [([90], [(0, 40)]), ([200, 300], [(0, 199), (1, 17), (1, 280)]), ([700], [(0, 3), (0, 650)])])
def test_prompt_what_a_row_does_not_see_does_not_reach_it(dtype, nq, at):
    """NaN and infinity in keys and values that only later rows of the sequence see."""
    Hq, Hkv, D = 4, 2, 128
    oq = offsets(nq)
    where = [(s, oq[s] + i) for s, i in at]
    gen = generator(5)
    Q, K, V = (normal(gen, H, oq[-1], D).to(TYPES[dtype]) for H in (Hq, Hkv, Hkv))
    clean = pk.pc_prompt_attn(Q, K, V, D ** -0.5, oq)
    for i, (s, j) in enumerate(where):
        V[:, j, 5 + i], V[:, j, 77] = NAN, float("inf")
        if i % 2:
            K[:, j, 9] = NAN
    got = pk.pc_prompt_attn(Q, K, V, D ** -0.5, oq)
    hit = torch.zeros(oq[-1], dtype=torch.bool, device=DEV)
    for s, j in where:
        hit[j:oq[s + 1]] = True
    assert got[:, ~hit].isfinite().all()
    assert torch.equal(got[:, ~hit], clean[:, ~hit]) or (got[:, ~hit].float() - clean[:, ~hit].float()).abs().max() < 0.02
    for i, (s, j) in enumerate(where):
        assert not got[:, j:oq[s + 1], 5 + i].isfinite().any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("level", [1e8, 1e30])
def test_prompt_hidden_keys(dtype, level):
    """Keys that a coordinate of their own hides: rows that see others too weigh those alone, the rest are numbers."""
    Hq, Hkv, D, n = 4, 2, 128, 150
    gen = generator(3)
    Q, K, V = (normal(gen, H, n, D).to(TYPES[dtype]) for H in (Hq, Hkv, Hkv))
    Q[..., 0], K[..., 0] = 1.0, 0.0
    K[:, :40, 0] = -level
    L = torch.empty((Hq, n), device=DEV)
    O = pk.pc_prompt_attn(Q, K, V, D ** -0.5, [0, n], lse=L)
    assert O.isfinite().all() and L.isfinite().all()
    for h in range(Hq):
        check_rows(dtype, O[h, 40:], None, Q[h, 40:], K[h // 2, 40:], V[h // 2, 40:], D ** -0.5, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["rising", "falling"])
def test_prompt_reference_moves(dtype, order):
    def make(Q, K, V):
        n = K.shape[1]
        ramp = torch.linspace(0, 6, n, device=DEV)
        K.mul_((ramp if order == "rising" else 6 - ramp)[None, :, None].to(K.dtype))
    run_prompt(dtype, 8, 2, 128, [500], make=make)


def test_prompt_folded_scale():
    run_prompt("bf16", 8, 2, 128, [333, 70], scale=pk.PC_SCALE_FOLDED)
    run_prompt("f32", 8, 2, 128, [333, 70], scale=pk.PC_SCALE_FOLDED)


@pytest.mark.parametrize("dtype,nq", [("bf16", [300, 20]), ("bf16", [2300]), ("f32", [100, 30])])
def test_prompt_is_reproducible_and_captured(dtype, nq):
    Q, K, V, O, L = run_prompt(dtype, 8, 2, 128, nq)
    oq, out, lse = offsets(nq), torch.zeros_like(Q), torch.zeros(Q.shape[:2], device=DEV)
    pk.pc_prompt_attn(Q, K, V, 128 ** -0.5, oq, O=out, lse=lse)
    want, want_lse = out.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pk.pc_prompt_attn(Q, K, V, 128 ** -0.5, oq, O=out, lse=lse)
    for _ in range(3):
        out.zero_(), lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


# ------------------------------------------------------------------------------ pages
class Paged:
    """Sequences of given lengths, in 64-bit-free plain form (K, V [Hkv][len][D] each) and in pages: everything that no sequence
    owns is NaN, table entries behind a sequence's last page are out of range."""

    def __init__(self, dtype, Hkv, D, lens, page=64, shared=0, seed=0, strided=False, make=None, width_more=2):
        gen, dt = generator(seed + sum(max(n, 0) for n in lens) + D), TYPES[dtype]
        self.dtype, self.D, self.Hkv, self.page, self.n_shared = dtype, D, Hkv, page, shared
        self.lens_host = [max(0, n) for n in lens]
        longest = max(max(self.lens_host), shared, 1)
        common = [normal(gen, Hkv, shared, D).to(dt) for _ in range(2)]
        self.seqs = []
        for n in self.lens_host:
            kv = [torch.cat((c[:, :n], normal(gen, Hkv, max(0, n - shared), D).to(dt)), 1) for c in common]
            self.seqs.append(kv)
        if make is not None:
            make(self)
        need = [-(-n // page) for n in self.lens_host]
        n_common = -(-shared // page)
        n_pages = sum(need) + n_common + 3
        free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        width = -(-longest // page) + width_more
        self.table = torch.full((len(lens), width + 1), n_pages + 5, dtype=torch.int32)[:, :width]
        if strided:      # heads outside, pages inside: a cache of one sequence's layout seen as pages
            big = [torch.full((Hkv, n_pages + 1, page, D), NAN, dtype=dt, device=DEV) for _ in range(2)]
            self.pages = tuple(x[:, :n_pages].transpose(0, 1) for x in big)
        else:
            self.pages = tuple(torch.full((n_pages, Hkv, page, D), NAN, dtype=dt, device=DEV) for _ in range(2))
        self.shared = None
        if shared:
            ids = [free.pop() for _ in range(n_common)]
            self.shared = torch.tensor(ids, dtype=torch.int32, device=DEV)
            self.put(ids, common, 0, shared)
        for s, n in enumerate(self.lens_host):
            ids = [free.pop() for _ in range(need[s])]
            self.table[s, :need[s]] = torch.tensor(ids, dtype=torch.int32)
            self.put(ids, self.seqs[s], shared, n)     # the common rows in its own pages are nothing that is read
        self.table = self.table.to(DEV)
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)

    def put(self, ids, rows, begin, end):
        for i, p in enumerate(ids):
            a, b = max(i * self.page, begin), min((i + 1) * self.page, end)
            if a < b:
                for pool, x in zip(self.pages, rows):
                    pool[p, :, a - i * self.page:b - i * self.page] = x[:, a:b]


def run_pages(dtype, Hq, Hkv, D, lens, n, *, page=64, shared=0, ragged=None, seed=0, scale=None, max_len=None, lse=True, strided=False,
              make=None, ws=None, paged=None):
    """n rows of every sequence (ragged: that many of each) over pages; checks every row."""
    pg = paged or Paged(dtype, Hkv, D, lens, page, shared, seed, strided, make)
    scale = D ** -0.5 if scale is None else scale
    rows = ragged if ragged is not None else [n] * len(lens)
    offs = offsets(rows, 1 if ragged is not None else 0)
    T = offs[-1] + (2 if ragged is not None else 0)
    gen = generator(seed + 17)
    Q = normal(gen, Hq, T + 1, D).to(TYPES[dtype])[:, :T]
    O = torch.full((Hq, T + 1, D), 7.0, dtype=TYPES[dtype], device=DEV)[:, :T]
    L = torch.full((Hq, T), 7.0, device=DEV) if lse else None
    longest = max(max(pg.lens_host), 1) if max_len is None else max_len
    got = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, longest, scale, offs=offs if ragged is not None else None, shared=pg.shared,
                          n_shared=shared, O=O, lse=L, ws=ws)
    assert got is O
    for s, (k, v) in enumerate(pg.seqs):
        a, b = offs[s], offs[s + 1]
        for h in range(Hq if b > a else 0):
            g = h // (Hq // Hkv)
            check_rows(dtype, O[h, a:b], None if L is None else L[h, a:b], Q[h, a:b], k[g], v[g], scale, int(pg.lens[s]) - (b - a) + 1)
    for rest in (slice(0, offs[0]), slice(offs[-1], T)):
        assert (O[:, rest] == 7.0).all() and (L is None or (L[:, rest] == 7.0).all())
    return pg, Q, O, L


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (6, 2), (4, 4), (5, 1), (32, 2)])
@pytest.mark.parametrize("lens,n", [([1], 1), ([130, 64, 0, 1], 1), ([63, 200], 3), ([500, 65, 640], 1), ([40, 1000], 17)])
def test_page_attn(dtype, D, Hq, Hkv, lens, n):
    run_pages(dtype, Hq, Hkv, D, lens, n)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("page", [64, 192])
@pytest.mark.parametrize("shared", [1, 63, 64, 300, 777])
@pytest.mark.parametrize("n,more", [(1, [1, 5, 64]), (1, [700, 0, 1]), (4, [4, 90, 3])])
def test_page_attn_common_rows(dtype, D, page, shared, n, more):
    """more: rows of each sequence behind the common ones; fewer than n: some rows see common rows only."""
    run_pages(dtype, 8, 2, D, [shared + m for m in more], n, page=page, shared=shared)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,shared", [([0, 400, 5, 130], 128), ([300, 299, 0, 0], 300), ([0, 0], 70), ([-3, 100], 64), ([2, 1, 64], 200)])
def test_page_attn_sequences_shorter_than_the_common_rows(dtype, lens, shared):
    run_pages(dtype, 8, 2, 128, lens, 1, shared=shared)
    run_pages(dtype, 8, 2, 128, lens, 3, shared=shared, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shared", [0, 100])
def test_page_attn_ragged(dtype, shared):
    rng = np.random.default_rng(shared)
    rows = [1, 0, 40, 7, 130, 1]
    run_pages(dtype, 8, 2, 128, [shared + n + int(v) for n, v in zip(rows, (500, 30, 0, 64, 200, 0))], None, ragged=rows, shared=shared)
    rows = [int(v) for v in rng.integers(0, 6, 140)]        # three launches
    run_pages(dtype, 4, 2, 128, [shared + n + int(v) for n, v in zip(rows, rng.integers(0, 200, 140))], None, ragged=rows, shared=shared)


@pytest.mark.parametrize("dtype,Hq,Hkv,lens,n,shared", [
    ("bf16", 16, 4, [5000, 3, 2049], 1, 0), ("bf16", 16, 4, [9000 + i for i in range(20)], 1, 9000), ("bf16", 4, 1, [4100, 300], 1, 0),
    ("bf16", 16, 4, [3000 + 40 * i for i in range(3)], 40, 2900), ("bf16", 24, 8, [4500], 300, 0), ("f32", 8, 2, [2500 + i for i in range(5)], 1, 2400),
    ("bf16", 8, 2, [2100] * 130, 1, 2000), ("bf16", 4, 2, [70 + i % 90 for i in range(600)], 1, 64),
    ("f32", 4, 2, [1 + i % 300 for i in range(300)], 2, 0), ("bf16", 16, 4, [9000, 1, 64, 3000, 0, 200, 129, 5000], 1, 0), ("bf16", 16, 2, [1000 + i for i in range(70)], 2, 0)])
def test_page_attn_long(dtype, Hq, Hkv, lens, n, shared):
    run_pages(dtype, Hq, Hkv, 128, lens, n, shared=shared, page=128)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("Hq,Hkv,n_seq,n,shared", [(9, 3, 5, 40, 2600), (11, 11, 3, 9, 1500), (7, 1, 6, 30, 4100), (13, 13, 2, 70, 600), (20, 5, 33, 1, 3000)])
def test_page_attn_tiles_of_common_rows_in_any_number(dtype, D, Hq, Hkv, n_seq, n, shared):
    """Shares times heads that eight divide, do not divide, and are fewer than; several tiles of each."""
    run_pages(dtype, Hq, Hkv, D, [shared + n + 13 * i for i in range(n_seq)], n, shared=shared)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,n,shared,max_len", [([5, 900, 1, 0], 1, 0, 2000), ([310, 305, 1200, 300], 2, 300, 2200), ([40, 9000, 3], 1, 0, 30000),
                                                   ([500, 460, 420], 100, 400, 1300)])
def test_page_attn_what_the_workspace_holds_does_not_count(dtype, lens, n, shared, max_len):
    """Shares for rows up to max_len that the sequences do not have are not written by anybody: the memory may hold anything."""
    nws = pk.pc_page_attn_workspace_bytes(pk.PC_BF16 if dtype == "bf16" else pk.PC_F32, 8, 2, n * len(lens), 128, len(lens), max_len, shared)
    page = 64
    pg = Paged(dtype, 2, 128, lens, page, shared, width_more=-(-max_len // page))
    outs = []
    for fill in (255, 127, 0):      # NaN, 3e38, 0
        ws = torch.full((max(nws, 1),), fill, dtype=torch.uint8, device=DEV)
        outs.append(run_pages(dtype, 8, 2, 128, lens, n, shared=shared, max_len=max_len, ws=ws, paged=pg)[2:])
    for O, L in outs[1:]:
        assert torch.equal(O, outs[0][0]) and torch.equal(L, outs[0][1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_page_attn_launches_without_rows(dtype):
    """More sequences than a launch has, the first launch's (or all) without rows."""
    rows = [0] * 64 + [3, 0, 70]
    run_pages(dtype, 8, 2, 128, [100 + n for n in rows], None, ragged=rows, shared=50)
    pg = Paged(dtype, 2, 128, [90, 80], shared=70)
    Q, O = torch.randn(8, 4, 128, device=DEV).to(TYPES[dtype]), torch.full((8, 4, 128), 7.0, dtype=TYPES[dtype], device=DEV)
    for offs in ([0, 0, 0], [2, 2, 2]):
        pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, 90, 0.1, offs=offs, shared=pg.shared, n_shared=70, O=O)
    assert (O == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_page_attn_strided_pages_and_bounds(dtype):
    """Heads outside of the pages; a bound far above the lengths, and one below them."""
    lens = [300, 65, 128]
    pg, Q, O, L = run_pages(dtype, 8, 2, 128, lens, 1, strided=True, shared=40)
    O2 = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, 64 * pg.table.shape[1], 128 ** -0.5, shared=pg.shared, n_shared=40)
    assert (O2.float() - O.float()).abs().max() < 0.02
    cut = Paged(dtype, 2, 128, [min(n, 100) for n in lens], shared=40)
    got = pk.pc_page_attn(Q, cut.pages, cut.table, pg.lens, 100, 128 ** -0.5, shared=cut.shared, n_shared=40)
    want = pk.pc_page_attn(Q, cut.pages, cut.table, cut.lens, 100, 128 ** -0.5, shared=cut.shared, n_shared=40)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,shared", [(1, 0), (5, 0), (1, 200), (70, 130)])
def test_page_attn_pages_that_are_not_there(dtype, n, shared):
    """A page number out of range stands for rows that nobody sees."""
    lens = [400, 500]
    pg = Paged(dtype, 2, 128, lens, shared=shared)
    for at, bad in ((3, -1), (4, 2 ** 30)):
        pg.table[0, at] = bad
        if shared:
            pg.shared[1] = bad
    T = 2 * n
    Q = normal(generator(1), 8, T, 128).to(TYPES[dtype])
    L = torch.empty((8, T), device=DEV)
    O = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, 500, 128 ** -0.5, shared=pg.shared, n_shared=shared, lse=L)
    for s in range(2):
        gone = torch.zeros(lens[s], dtype=torch.bool, device=DEV)
        if s == 0:
            gone[max(192, shared):320] = True
        if shared:
            gone[64:min(128, shared)] = True
        for h in range(8):
            for i in range(n):
                at = s * n + i
                keep = ~gone & (torch.arange(lens[s], device=DEV) <= lens[s] - n + i)
                k, v = (x[h // 4][keep] for x in pg.seqs[s])
                check_rows(dtype, O[h, at:at + 1], L[h, at:at + 1], Q[h, at:at + 1], k, v, 128 ** -0.5, k.shape[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,shared", [(6, 0), (6, 128), (40, 0), (90, 70)])
def test_page_attn_what_a_row_does_not_see_does_not_reach_it(dtype, n, shared):
    def make(p):
        k, v = p.seqs[1]
        v[:, 190, 7], v[:, 193, 9], k[:, 192, 3] = NAN, float("inf"), NAN
    lens = [400, 194, 300]
    pg = Paged(dtype, 2, 128, lens, shared=shared, make=make)
    Q = normal(generator(2), 8, 3 * n, 128).to(TYPES[dtype])
    O = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, 400, 128 ** -0.5, shared=pg.shared, n_shared=shared)
    first = n + 190 - (194 - n)       # the row that is row 190 of its sequence, if it is among the new ones
    clean = [i for i in range(3 * n) if not max(first, n) <= i < 2 * n]
    assert O[:, clean].isfinite().all()
    assert not O[:, max(first, n):2 * n, 7].isfinite().any() and not O[:, 2 * n - 1].isfinite().any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_page_attn_hidden_keys(dtype):
    def make(p):
        for k, v in p.seqs:
            k[..., 0] = 0.0
            k[:, 30:150, 0] = -1e30
    for lens, shared in (([200, 151, 600], 0), ([200, 151, 600], 20)):
        pg = Paged(dtype, 2, 128, lens, shared=shared, make=make if not shared else None)
        Q = normal(generator(2), 8, len(lens), 128).to(TYPES[dtype])
        Q[..., 0] = 1.0
        L = torch.empty((8, len(lens)), device=DEV)
        O = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, 600, 128 ** -0.5, shared=pg.shared, n_shared=shared, lse=L)
        assert O.isfinite().all()
        for s in range(len(lens)):
            keep = torch.ones(lens[s], dtype=torch.bool, device=DEV)
            if not shared:
                keep[30:150] = False
            for h in range(8):
                k, v = (x[h // 4][keep] for x in pg.seqs[s])
                check_rows(dtype, O[h, s:s + 1], L[h, s:s + 1], Q[h, s:s + 1], k, v, 128 ** -0.5, k.shape[0])


@pytest.mark.parametrize("dtype,shared", [("bf16", 0), ("bf16", 700), ("f32", 100)])
def test_page_attn_is_reproducible_and_captured(dtype, shared):
    """The lengths grow between replays of one graph."""
    lens = [shared + 1, shared + 64, shared + 400]
    pg, Q, O, L = run_pages(dtype, 8, 2, 128, lens, 1, shared=shared)
    out = torch.zeros_like(O)
    nws = pk.pc_page_attn_workspace_bytes(pk.PC_BF16 if dtype == "bf16" else pk.PC_F32, 8, 2, 3, 128, 3, shared + 400, shared)
    ws = torch.full((max(nws, 16),), 0xA5, dtype=torch.uint8, device=DEV)
    call = lambda: pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, shared + 400, 128 ** -0.5, shared=pg.shared, n_shared=shared, O=out, ws=ws)
    call()
    assert torch.equal(out, O)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for d in (0, 1, 30):
        pg.lens.copy_(torch.tensor([max(1, n - d) for n in lens], dtype=torch.int32))
        out.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        call()
        assert torch.equal(got, out)


# ------------------------------------------------------------------------------ rows into pages
def turned(x, pos, D, scale=1.0):
    y = x.contiguous().clone()
    if y.shape[1]:
        pk.pc_rope3d(y, pos, SECTIONS[D], out_scale=scale)
    return y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,page,before,rows,ragged", [
    (8, 2, 64, [0], [1], False), (8, 2, 64, [63, 64, 0, 200], [1, 1, 1, 1], False), (6, 3, 128, [5, 130], [3, 3], False),
    (5, 1, 64, [0, 60, 0, 7], [70, 0, 1, 130], True), (16, 4, 192, [100] * 70, [2] * 70, True), (24, 8, 64, [0, 31], [257, 33], True)])
def test_store(dtype, D, Hq, Hkv, page, before, rows, ragged):
    gen, dt = generator(len(before) + D), TYPES[dtype]
    lens = [b + n for b, n in zip(before, rows)]
    pg = Paged(dtype, Hkv, D, lens, page, width_more=0, strided=Hkv == 2)
    offs = offsets(rows, 1 if ragged else 0)
    T = offs[-1] + (2 if ragged else 0)
    K, V = normal(gen, Hkv, T + 3, D).to(dt)[:, :T], normal(gen, Hkv, T + 1, D).to(dt)[:, :T]
    Q = normal(gen, Hq, T + 2, D).to(dt)[:, :T]
    pos = torch.randint(-50, 5000, (T, 3), dtype=torch.int32, device=DEV, generator=gen)
    o = offs if ragged else None
    mine = slice(offs[0], offs[-1])
    want_k, want_q = turned(K, pos, D), turned(Q, pos, D, 0.3)
    before_pages = [x.clone() for x in pg.pages]

    def check(k_rows):
        for pool, x, was in zip(pg.pages, (k_rows, V), before_pages):
            want = was.clone()
            for s in range(len(rows)):
                for i in range(rows[s]):
                    r = lens[s] - rows[s] + i
                    want[pg.table[s, r // page].item(), :, r % page] = x[:, offs[s] + i]
            assert torch.equal(torch.nan_to_num(pool.float(), 123.0), torch.nan_to_num(want.float(), 123.0))
    K_out, Q_out = torch.full_like(K, 7.0), torch.full_like(Q, 7.0)
    K_was, V_was = K.clone(), V.clone()
    pk.pc_page_store(K, V, pg.pages, pg.table, pg.lens, offs=o, pos=pos, sections=SECTIONS[D], K_out=K_out, Q=Q, Q_out=Q_out, out_scale=0.3)
    check(want_k)
    assert torch.equal(K_out[:, mine], want_k[:, mine]) and torch.equal(Q_out[:, mine], want_q[:, mine])
    for rest in (slice(0, offs[0]), slice(offs[-1], T)):
        assert (K_out[:, rest] == 7.0).all() and (Q_out[:, rest] == 7.0).all()
    assert torch.equal(K, K_was) and torch.equal(V, V_was)
    for pool, was in zip(pg.pages, before_pages):
        pool.copy_(was)
    pk.pc_page_store(K, V, pg.pages, pg.table, pg.lens, offs=o, pos=pos, sections=SECTIONS[D], K_out=K, Q=Q, Q_out=Q, out_scale=0.3)
    check(want_k)       # in place
    assert torch.equal(K[:, mine], want_k[:, mine]) and torch.equal(Q[:, mine], want_q[:, mine])
    for pool, was in zip(pg.pages, before_pages):
        pool.copy_(was)
    K.copy_(K_was)
    K[:, mine.start, 3] = NAN
    pk.pc_page_store(K, V, pg.pages, pg.table, pg.lens, offs=o)     # as they are
    check(K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_rows_without_a_page(dtype):
    """Pausing sequences, lengths beyond the table, page numbers out of range: nothing is stored, the rest is."""
    Hkv, D, page = 2, 128, 64
    pg = Paged(dtype, Hkv, D, [64, 1, 128, 60, 60], page, width_more=0)
    lens = torch.tensor([0, -5, 200, 60, 1], dtype=torch.int32, device=DEV)      # idle; negative; behind the table; bad page; fine
    pg.table[3, 0] = -2
    T, gen = 5, generator(4)
    K, V = normal(gen, Hkv, T, D).to(TYPES[dtype]), normal(gen, Hkv, T, D).to(TYPES[dtype])
    pos = torch.zeros((T, 3), dtype=torch.int32, device=DEV)
    was = [x.clone() for x in pg.pages]
    K_out = torch.zeros_like(K)
    pk.pc_page_store(K, V, pg.pages, pg.table, lens, pos=pos, sections=SECTIONS[D], K_out=K_out)
    for pool, w, x in zip(pg.pages, was, (K, V)):
        w[pg.table[4, 0].item(), :, 0] = x[:, 4]
        assert torch.equal(torch.nan_to_num(pool.float(), 123.0), torch.nan_to_num(w.float(), 123.0))
    assert torch.equal(K_out, K)


# ------------------------------------------------------------------------------ large offsets, streams
def test_offsets_beyond_32_bits():
    """Pages whose elements lie beyond 2^32 bytes and 2^31 elements, K and V of 4.5 GiB each."""
    Hkv, D, page = 2, 128, 64
    n_pages = (2 ** 31 + 2 ** 28) // (Hkv * page * D)
    K = torch.empty((n_pages, Hkv, page, D), dtype=torch.bfloat16, device=DEV)
    pages = (K, torch.empty_like(K))
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device=DEV)
    gen = generator(9)
    k, v = (normal(gen, Hkv, 150, D).to(torch.bfloat16) for _ in range(2))
    lens = torch.tensor([150], dtype=torch.int32, device=DEV)
    pk.pc_page_store(k, v, pages, table, lens)
    assert torch.equal(pages[0][n_pages - 2, :, :22], k[:, 128:]) and torch.equal(pages[1][n_pages - 1], v[:, :64])
    Q = normal(gen, 8, 1, D).to(torch.bfloat16)
    O = pk.pc_page_attn(Q, pages, table, lens, 150, D ** -0.5)
    for h in range(8):
        check_rows("bf16", O[h], None, Q[h], k[h // 4], v[h // 4], D ** -0.5, 150)


def test_calls_on_two_streams_do_not_meet():
    pgs = [Paged("bf16", 2, 128, [700 + i, 300], shared=200, seed=i) for i in range(2)]
    Qs = [normal(generator(i), 8, 2, 128).to(torch.bfloat16) for i in range(2)]
    call = lambda i: pk.pc_page_attn(Qs[i], pgs[i].pages, pgs[i].table, pgs[i].lens, 701, 128 ** -0.5, shared=pgs[i].shared, n_shared=200)
    want = [call(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        got = []
        for i, st in enumerate(streams):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                got.append(call(i))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_both_halves_of_the_binding_give_the_same_bits(monkeypatch):
    from paper_2601_04359_amd import binding
    assert binding._NATIVE
    results = []
    for native in (binding._NATIVE, False):
        monkeypatch.setattr(binding, "_NATIVE", native)
        _, _, _, O, L = run_prompt("bf16", 8, 2, 128, [40, 333], [40, 500], lse=True)
        out = [O, L]
        for ragged, shared in ((None, 0), (None, 200), ([1, 5, 2], 130)):
            _, _, O, L = run_pages("bf16", 8, 2, 128, [300, 210, 400], 1 if ragged is None else None, ragged=ragged, shared=shared)
            out += [O, L]
        test_store("bf16", 128, 8, 2, 64, [63, 64, 0, 200], [1, 1, 1, 1], False)
        test_store("f32", 64, 5, 1, 64, [0, 60, 0, 7], [70, 0, 1, 130], True)
        results.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*results))
    if native is False:
        monkeypatch.undo()
    Q = torch.zeros((8, 4, 128), dtype=torch.bfloat16, device=DEV)
    pages, table, lens = pk.page_cache(3, 2, 64, 128), torch.zeros((4, 2), dtype=torch.int32, device=DEV), torch.ones(4, dtype=torch.int32, device=DEV)
    for bad in (dict(max_len=129), dict(max_len=0), dict(lens=lens.long()), dict(table=table[:3]), dict(pages=pages[0]), dict(n_shared=5),
                dict(shared=table[0, :1], n_shared=65), dict(offs=[0, 2, 4]), dict(offs=[0, 1, 2, 3, 5]), dict(lens=lens.cpu()),
                dict(ws=torch.zeros(1, dtype=torch.uint8, device=DEV), shared=table[0], n_shared=65), dict(O=Q), dict(scale=-1.0)):
        kw = {**dict(pages=pages, table=table, lens=lens, max_len=128, scale=0.1, O=torch.empty_like(Q)), **bad}
        with pytest.raises(pk.PackCacheError):
            pk.pc_page_attn(Q, kw.pop("pages"), kw.pop("table"), kw.pop("lens"), kw.pop("max_len"), kw.pop("scale"), **kw)


# ------------------------------------------------------------------------------ the operators together
class Twin:
    """A PagedStack and its sequences in plain form; every attend() is checked row by row."""

    def __init__(self, dtype="bf16", layers=2, Hq=8, Hkv=2, D=128, n_pages=60, seed=0, **kw):
        self.s = PagedStack(layers, Hq, Hkv, D, n_pages, D ** -0.5, sections=SECTIONS[D], dtype=TYPES[dtype], fold_scale=False, **kw)
        for t in (self.s.K, self.s.V):
            t.fill_(NAN)
        self.dtype, self.gen, self.plain = dtype, generator(seed), {}

    def open(self):
        q = self.s.open()
        self.plain[q] = [[torch.empty((self.s.Hkv, 0, self.s.D), dtype=TYPES[self.dtype], device=DEV) for _ in range(2)] for _ in range(self.s.L)]
        return q

    def fork(self, q, n=1):
        out = self.s.fork(q, n)
        for f in out:
            self.plain[f] = [[x.clone() for x in kv] for kv in self.plain[q]]
        return out

    def step(self, seqs, rows, **kw):
        s = self.s
        counts = [rows] * len(seqs) if isinstance(rows, int) else rows
        offs = offsets(counts)
        T = offs[-1]
        s.begin(seqs, rows, **kw)
        for layer in range(s.L):
            Q, K, V = (normal(self.gen, H, T, s.D).to(TYPES[self.dtype]) for H in (s.Hq, s.Hkv, s.Hkv))
            pos = torch.randint(0, 900, (T, 3), dtype=torch.int32, device=DEV, generator=self.gen)
            k, q = turned(K, pos, s.D), turned(Q, pos, s.D)
            L = torch.empty((s.Hq, T), device=DEV)
            O = s.attend(layer, Q, K, V, pos, lse=L)
            assert torch.equal(Q, q)
            for i, seq in enumerate(seqs):
                a, b = offs[i], offs[i + 1]
                kv = self.plain[seq][layer]
                kv[0], kv[1] = torch.cat((kv[0], k[:, a:b]), 1), torch.cat((kv[1], V[:, a:b]), 1)
                for h in range(s.Hq if b > a else 0):
                    g = h // (s.Hq // s.Hkv)
                    check_rows(self.dtype, O[h, a:b], L[h, a:b], q[h, a:b], kv[0][g], kv[1][g], s.scale, kv[0].shape[1] - (b - a) + 1)
        for seq in seqs:
            assert s.rows(seq) == self.plain[seq][0][0].shape[1]


@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 64), ("bf16", 64, 64), ("f32", 128, 128)])
def test_stack_of_sequences(dtype, D, page):
    t = Twin(dtype, D=D, page_rows=page, n_pages=40)
    a, b, c = t.open(), t.open(), t.open()
    t.step([a, b, c], [130, 1, 64])               # prompts
    t.step([a, b, c], 1)
    d, e = t.fork(a, 2)                           # in the middle of a page
    t.step([a, d, e], 1)                          # copies; two pages are common
    assert t.s.n_shared == 131 // page * page
    t.step([d, e], [40, 1])
    t.step([a, b, c, d, e], [1, 0, 3, 70, 2])     # no page is common to all
    assert t.s.n_shared == 0
    free = t.s.free_pages()
    f, = t.fork(d)
    t.step([d, f], 0)                             # nothing new: the whole sequence is common, the page that is not full as well
    assert t.s.n_shared == t.s.rows(d) and t.s.free_pages() == free
    t.step([f], 5)
    t.step([d, f], 1)
    for q in (a, b, e, f):
        t.s.close(q)
    g = t.open()
    t.step([g], [200])                            # pages that others have left
    t.step([c, d, g], [1, 1, 1], max_len=page * 5)
    for q in (c, d, g):
        t.s.close(q)
    assert t.s.free_pages() == 40


def test_stack_of_many_branches():
    """A prompt continued 20 ways, token by token across the border of a page; then one of them 10 ways."""
    t = Twin(n_pages=90, layers=1, Hq=16, Hkv=4)
    a = t.open()
    t.step([a], [700])
    branches = [a] + t.fork(a, 19)
    for _ in range(3):
        t.step(branches, 1)
        assert t.s.n_shared == 640
    t.step(branches, 66)
    for q in branches[1:]:
        t.s.close(q)
    more = [a] + t.fork(a, 9)
    t.step(more, 2)
    assert t.s.n_shared == 768 and t.s.rows(a) == 771


def test_stack_step_in_a_graph():
    """Steps of one token, recorded once: begin() moves the lengths and tables between the replays."""
    layers, Hq, Hkv, D = 2, 8, 2, 128
    gen = generator(3)
    stacks = [PagedStack(layers, Hq, Hkv, D, 40, D ** -0.5, max_rows=512) for _ in range(2)]
    rows = lambda n: [normal(gen, layers, H, n, D).to(torch.bfloat16) for H in (Hq, Hkv, Hkv)]
    Q, K, V = rows(150)
    pos = torch.randint(0, 900, (150, 3), dtype=torch.int32, device=DEV, generator=gen)
    seqs = []
    for s in stacks:
        a = s.open()
        s.begin([a], 150)
        for l in range(layers):
            s.attend(l, Q[l].clone(), K[l].clone(), V[l], pos)
        seqs.append([a] + s.fork(a, 2))
        s.begin(seqs[-1], 1, max_len=512)
        for l in range(layers):
            s.attend(l, Q[l, :, :3].clone(), K[l, :, :3].clone(), V[l, :, :3], pos[:3])
    fixed = [x[:, :, :3].clone() for x in (Q, K, V)]
    p, O = pos[:3].clone(), torch.empty((layers, Hq, 3, D), dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    stacks[0].begin(seqs[0], 1, max_len=512)
    with torch.cuda.graph(graph):
        for l in range(layers):
            stacks[0].attend(l, fixed[0][l], fixed[1][l], fixed[2][l], p, O=O[l])
    for step in range(70):                        # across a page's border
        new = rows(3)
        if step:
            stacks[0].begin(seqs[0], 1, max_len=512)
        stacks[1].begin(seqs[1], 1, max_len=512)
        assert stacks[0].n_shared == stacks[1].n_shared == 128
        for x, y in zip(fixed, new):
            x.copy_(y)
        p.random_(0, 900, generator=gen)
        graph.replay()
        torch.cuda.synchronize()
        for l in range(layers):
            want = stacks[1].attend(l, new[0][l], new[1][l], new[2][l], p)
            assert torch.equal(O[l], want)


# ------------------------------------------------------------------------------ scores of -inf
def check_kept(dtype, O, L, Q, kv, keep, scale, none=0):
    """Rows one by one: row i of O, L, Q [Hq][n][..] weighs the keys of kv (K, V [Hkv][nk][D]) that keep [n][nk] has; `none` of the rows
    have no such key, and give 0 and -inf."""
    Hq, n, _ = O.shape
    for i in range(n):
        for h in range(Hq):
            k, v = (x[h // (Hq // kv[0].shape[0])][keep[i]] for x in kv)
            if k.shape[0] == 0:
                assert (O[h, i] == 0).all() and L[h, i] == -float("inf")
            else:
                check_rows(dtype, O[h, i:i + 1], L[h, i:i + 1], Q[h, i:i + 1], k, v, scale, k.shape[0])
    assert (~keep.any(1)).sum() == none


def causal(n, nk, gone):
    """keep [n][nk] of the last n rows of a sequence of nk, without the keys in `gone`."""
    at = torch.arange(nk, device=DEV)
    keep = at[None] <= nk - n + torch.arange(n, device=DEV)[:, None]
    return keep & ~torch.isin(at, torch.tensor(list(gone), dtype=torch.int64, device=DEV))[None]


OVERFLOWS = [17, 18, 40, 63, 64, 70]


def overflow(Q, K):
    """Products of these keys with every query are beyond the range of 32 bits."""
    Q[..., 0], K[..., 0] = 8.0, 0.0
    K[:, [j for j in OVERFLOWS if j < K.shape[1]], 0] = -3e38


def rewrite(pg, change):
    """change(K, V) of every sequence's rows, the common ones among them, in plain form and in the pages."""
    for K, V in pg.seqs:
        change(K, V)
    longest = max(range(len(pg.seqs)), key=lambda s: pg.lens_host[s])
    if pg.n_shared:
        pg.put(pg.shared.tolist(), [x[:, :pg.n_shared] for x in pg.seqs[longest]], 0, pg.n_shared)
    for s, n in enumerate(pg.lens_host):
        pg.put(pg.table[s, :-(-n // pg.page)].tolist(), pg.seqs[s], pg.n_shared, n)


@pytest.mark.parametrize("dtype,D", [("f32", 128), ("f32", 64), ("bf16", 128), ("bf16", 64)])
@pytest.mark.parametrize("scale", [128 ** -0.5, 0.1, 0.125, pk.PC_SCALE_FOLDED])
@pytest.mark.parametrize("n", [75, 700])
def test_prompt_scores_of_minus_infinity_weigh_nothing(dtype, D, scale, n):
    Hq, Hkv = 4, 2
    gen = generator(n)
    Q, K, V = (normal(gen, H, n, D).to(TYPES[dtype]) for H in (Hq, Hkv, Hkv))
    overflow(Q, K)
    L = torch.empty((Hq, n), device=DEV)
    O = pk.pc_prompt_attn(Q, K, V, scale, [0, n], lse=L)
    rows = list(range(0, 17, 5)) + list(range(17, 75, 3)) + [n - 1]
    check_kept(dtype, O[:, rows], L[:, rows], Q[:, rows], (K, V), causal(n, n, OVERFLOWS)[rows], scale)


@pytest.mark.parametrize("dtype,D", [("f32", 128), ("f32", 64), ("bf16", 128), ("bf16", 64)])
@pytest.mark.parametrize("scale", [128 ** -0.5, 0.1, 0.125, pk.PC_SCALE_FOLDED])
@pytest.mark.parametrize("lens,n,shared", [([100, 300], 1, 0), ([100, 300], 1, 66), ([120, 300], 30, 20)])
def test_page_attn_scores_of_minus_infinity_weigh_nothing(dtype, D, scale, lens, n, shared):
    pg = Paged(dtype, 2, D, lens, shared=shared)
    Q = normal(generator(1), 4, 2 * n, D).to(TYPES[dtype])
    rewrite(pg, lambda K, V: overflow(Q, K))
    L = torch.empty((4, 2 * n), device=DEV)
    O = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, max(lens), scale, shared=pg.shared, n_shared=shared, lse=L)
    for s in range(2):
        mine = slice(s * n, (s + 1) * n)
        check_kept(dtype, O[:, mine], L[:, mine], Q[:, mine], pg.seqs[s], causal(n, lens[s], OVERFLOWS), scale)


# ------------------------------------------------------------------------------ pages that are all missing
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("scale", [0.1, pk.PC_SCALE_FOLDED])
@pytest.mark.parametrize("lens,n,shared,missing,missing_shared", [
    ([1, 90], 1, 0, [(0, 0)], []),                                   # a padded place: one row, no page
    ([200, 90], 1, 0, [(0, 0), (0, 1), (0, 2), (0, 3)], []),
    ([100, 70], 70, 0, [(0, 0), (1, 0)], []),                        # the first page, and rows that begin in it
    ([600, 300], 300, 0, [(0, 0), (0, 4), (0, 5), (1, 0), (1, 1)], []),
    ([3000, 2900], 1, 0, [(1, i) for i in range(46)], []),           # joined shares
    ([230, 214], 2, 200, [(1, 3)], [0, 1, 2, 3]),                    # nothing in common, and nothing of one's own
    ([200, 200], 2, 200, [], [0, 1, 2, 3]),                          # common rows only
    ([2700, 2750], 150, 2600, [(0, i) for i in range(40, 43)], list(range(41)))])
def test_page_attn_rows_without_any_page(dtype, D, scale, lens, n, shared, missing, missing_shared):
    """A row all of whose keys lie in pages that are not there sees nothing: O = 0, lse = -inf."""
    pg = Paged(dtype, 2, D, lens, shared=shared)
    gone = [set(), set()]
    for s, i in missing:
        pg.table[s, i] = -1 if i % 2 else 2 ** 30
        gone[s] |= {j for j in range(i * 64, i * 64 + 64) if j >= shared}
    for i in missing_shared:
        pg.shared[i] = -1 if i % 2 else 2 ** 30
        for s in range(2):
            gone[s] |= {j for j in range(i * 64, i * 64 + 64) if j < shared}
    Q = normal(generator(1), 4, 2 * n, D).to(TYPES[dtype])
    L = torch.full((4, 2 * n), 7.0, device=DEV)
    O = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, max(lens), scale, shared=pg.shared, n_shared=shared, lse=L)
    empty = 0
    for s in range(2):
        keep = causal(n, lens[s], gone[s])
        nothing = ~keep.any(1)
        empty += int(nothing.sum())
        mine = slice(s * n, (s + 1) * n)
        rows = [i for i in range(n) if n < 40 or i % 17 == 0 or i in (63, 64, n - 1)]
        assert (O[:, mine][:, nothing] == 0).all() and (L[:, mine][:, nothing] == -float("inf")).all()
        check_kept(dtype, O[:, mine][:, rows], L[:, mine][:, rows], Q[:, mine][:, rows], pg.seqs[s], keep[rows], scale, int(nothing[rows].sum()))
    assert empty > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,n,shared", [([90, 70], 1, 0), ([90, 70], 70, 0), ([300, 320], 2, 200)])
def test_page_attn_rows_without_any_page_do_not_hide_a_nan(dtype, lens, n, shared):
    """A query that is not a number leaves none, with pages and beside rows without."""
    pg = Paged(dtype, 2, 128, lens, shared=shared)
    pg.table[0, :] = -1
    if shared:
        pg.shared[:] = -1
    Q = normal(generator(1), 4, 2 * n, 128).to(TYPES[dtype])
    Q[1, 2 * n - 1, 5], Q[2, 0, 5] = NAN, NAN
    O = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, max(lens), 0.1, shared=pg.shared, n_shared=shared)
    assert O[1, 2 * n - 1].isnan().all() and (O[:, :n] == 0).all()
    ok = torch.ones((4, 2 * n), dtype=torch.bool, device=DEV)
    ok[1, 2 * n - 1] = False
    assert O[ok].isfinite().all()


# ------------------------------------------------------------------------------ infinities that are seen
@pytest.mark.parametrize("dtype,D,Hq,Hkv,n", [("bf16", 128, 8, 2, 40), ("bf16", 64, 8, 2, 300), ("bf16", 128, 16, 4, 2049), ("bf16", 128, 3, 3, 3001),
                                              ("f32", 128, 4, 2, 150), ("f32", 64, 2, 1, 1100)])
@pytest.mark.parametrize("at", [0, 5, 31, 33, -1, -40])
@pytest.mark.parametrize("scale", [0.1, pk.PC_SCALE_FOLDED])
def test_prompt_an_infinity_that_is_seen_arrives_as_one(dtype, D, Hq, Hkv, n, at, scale):
    """A single infinite value in V: infinite in its dim in the rows that see it, whatever tile or form it is read by, and numbers
    everywhere else."""
    gen, at = generator(n), at % n
    Q, K, V = (normal(gen, H, n, D).to(TYPES[dtype]) for H in (Hq, Hkv, Hkv))
    V[:, at, 9], V[:, at, D - 1] = float("inf"), -float("inf")
    O = pk.pc_prompt_attn(Q, K, V, scale, [0, n])
    assert (O[:, at:, 9] == float("inf")).all() and (O[:, at:, D - 1] == -float("inf")).all()
    V[:, at, 9], V[:, at, D - 1] = 0.0, 0.0
    rest = torch.ones((n, D), dtype=torch.bool, device=DEV)
    rest[at:, 9], rest[at:, D - 1] = False, False
    assert torch.equal(O[:, rest], pk.pc_prompt_attn(Q, K, V, scale, [0, n])[:, rest])


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("n,shared", [(1, 0), (6, 0), (50, 0), (300, 0), (6, 40), (50, 40), (300, 40), (300, 1960)])
@pytest.mark.parametrize("back", [1, 2, 40, None])
@pytest.mark.parametrize("scale", [0.1, pk.PC_SCALE_FOLDED])
def test_page_attn_an_infinity_that_is_seen_arrives_as_one(dtype, D, n, shared, back, scale):
    """back: so many rows in front of the sequence's end; None: the first row behind the common ones."""
    lens = [shared + 330, shared + 400, shared + 301]
    at = lens[1] - back if back is not None else shared
    pg = Paged(dtype, 2, D, lens, shared=shared)
    Q = normal(generator(2), 8, 3 * n, D).to(TYPES[dtype])
    call = lambda: pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, max(lens), scale, shared=pg.shared, n_shared=shared)

    def put(x, y):
        pg.seqs[1][1][:, at, 9], pg.seqs[1][1][:, at, D - 1] = x, y
        rewrite(pg, lambda K, V: None)
    put(float("inf"), -float("inf"))
    O = call()
    first = n + max(0, at - (lens[1] - n))      # the rows of the sequence that see it
    assert (O[:, first:2 * n, 9] == float("inf")).all() and (O[:, first:2 * n, D - 1] == -float("inf")).all()
    put(0.0, 0.0)
    rest = torch.ones((3 * n, D), dtype=torch.bool, device=DEV)
    rest[first:2 * n, 9], rest[first:2 * n, D - 1] = False, False
    assert torch.equal(O[:, rest], call()[:, rest])


# ------------------------------------------------------------------------------ many query heads behind many keys
@pytest.mark.parametrize("dtype,D,Hq", [("bf16", 64, 2 ** 16), ("bf16", 128, 2 ** 19)])
def test_prompt_tiles_behind_more_than_32_bits_of_rows(dtype, D, Hq):
    """Two sequences of one token in very many heads of one KV head, one of them behind 2^20 keys: the keys in front of it, counted in
    row tiles (of 32 and of 128 rows), are beyond 2^31."""
    nk = [100, 2 ** 20 + 5000]
    gen, oq, ok = generator(6), [0, 1, 2], offsets(nk)
    Q = normal(gen, Hq, 2, D).to(TYPES[dtype])
    K, V = (normal(gen, 1, ok[-1], D).to(TYPES[dtype]) for _ in range(2))
    L = torch.empty((Hq, 2), device=DEV)
    O = pk.pc_prompt_attn(Q, K, V, D ** -0.5, oq, ok, lse=L)
    for h in (0, 1, 31, 32, 127, 128, 40000, Hq - 1):
        for s in range(2):
            mine = slice(ok[s], ok[s + 1])
            check_rows(dtype, O[h, s:s + 1], L[h, s:s + 1], Q[h, s:s + 1], K[0, mine], V[0, mine], D ** -0.5, nk[s])


# ------------------------------------------------------------------------------ rows beyond one launch
def test_store_of_more_rows_than_a_launch_has_threads_for():
    """2^26 + 1,000 rows of one sequence, of which the pages hold the last 500; four rows take 256 threads."""
    T, D, n = 2 ** 26 + 1000, 64, 500
    K, V = (torch.zeros((1, T, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    gen = generator(8)
    for x in (K, V):
        x[:, T - 600:] = normal(gen, 1, 600, D).to(torch.bfloat16)
    pages, table = pk.page_cache(9, 1, 64, D), torch.arange(8, 0, -1, dtype=torch.int32, device=DEV)[None].contiguous()
    K_out = torch.empty_like(K)
    for offs in (None, [0, T]):
        for x in (*pages, K_out):
            x.fill_(7.0)
        pk.pc_page_store(K, V, pages, table, torch.tensor([n], dtype=torch.int32, device=DEV), offs=offs, K_out=K_out)
        for pool, x in zip(pages, (K, V)):
            got = pool[table[0].long(), 0].reshape(-1, D)
            assert torch.equal(got[:n], x[0, T - n:]) and (got[n:] == 7.0).all() and (pool[0] == 7.0).all()
        assert torch.equal(K_out, K)


# ------------------------------------------------------------------------------ lengths that are no lengths
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("n,shared,max_len", [(3, 64, 64), (3, 0, 90), (40, 64, 64), (150, 500, 500), (3, 64, 90), (200, 64, 700)])
@pytest.mark.parametrize("ragged", [False, True])
def test_page_attn_any_number_as_a_length(dtype, D, n, shared, max_len, ragged):
    """Negative ones down to the lowest number are sequences without rows, the highest ones end at max_len."""
    lens = [max_len, 0, 0, max_len, 0]
    pg = Paged(dtype, 2, D, lens, shared=shared)
    pg.lens = torch.tensor([2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1, max_len, -1], dtype=torch.int32, device=DEV)
    T, Hq = 5 * n, 8
    Q = normal(generator(1), Hq, T, D).to(TYPES[dtype])
    L = torch.full((Hq, T), 7.0, device=DEV)
    O = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, max_len, 0.1, offs=offsets([n] * 5) if ragged else None, shared=pg.shared, n_shared=shared,
                        lse=L)
    for s, m in enumerate(lens):
        mine = slice(s * n, (s + 1) * n)
        if m == 0:
            assert (O[:, mine] == 0).all() and (L[:, mine] == -float("inf")).all()
        for h in range(Hq if m else 0):
            check_rows(dtype, O[h, mine], L[h, mine], Q[h, mine], pg.seqs[s][0][h // 4], pg.seqs[s][1][h // 4], 0.1, m - n + 1)


# ------------------------------------------------------------------------------ more of the same, where it could go wrong
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("level", [1e8, 1e30])
@pytest.mark.parametrize("scale", [128 ** -0.5, pk.PC_SCALE_FOLDED])
@pytest.mark.parametrize("lens,n,shared,hidden", [
    ([400, 351, 600], 1, 300, [(30, 150), (310, 340)]),           # some of both
    ([400, 351, 600], 1, 300, [(0, 300)]),                        # all common rows
    ([400, 351, 600], 40, 300, [(0, 290)]), ([400, 361, 600], 40, 300, [(300, 1000)]),      # all own rows
    ([2900, 2700, 2650], 1, 2600, [(0, 2500)]), ([2900, 2700, 2650], 1, 2600, [(2600, 3000)]),
    ([900, 860], 200, 600, [(64, 600)]), ([900, 860], 200, 600, [(0, 64), (600, 1000)]), ([3000, 2900, 70], 1, 0, [(0, 64), (200, 2800)])])
def test_page_attn_hidden_keys_in_any_share(dtype, D, level, scale, lens, n, shared, hidden):
    """Keys that a coordinate of their own hides, in common and in own rows: shares of very different references are joined."""
    at = [j for a, b in hidden for j in range(a, b)]

    def hide(K, V):
        K[..., 0] = 0.0
        K[:, [j for j in at if j < K.shape[1]], 0] = -level
    pg = Paged(dtype, 2, D, lens, shared=shared)
    rewrite(pg, hide)
    T = n * len(lens)
    Q = normal(generator(2), 4, T, D).to(TYPES[dtype])
    Q[..., 0] = 1.0
    L = torch.empty((4, T), device=DEV)
    O = pk.pc_page_attn(Q, pg.pages, pg.table, pg.lens, max(lens), scale, shared=pg.shared, n_shared=shared, lse=L)
    assert O.isfinite().all() and L.isfinite().all()
    for s, m in enumerate(lens):
        keep = causal(n, m, at)
        rows = [i for i in sorted({0, 1, n // 3, n // 2, n - 1}) if i < n and keep[i].any()]
        mine = [s * n + i for i in rows]
        check_kept(dtype, O[:, mine], L[:, mine], Q[:, mine], pg.seqs[s], keep[rows], scale)


@pytest.mark.parametrize("dtype,D,Hq,Hkv,nq,nk", [
    ("bf16", 64, 8, 2, [2300, 40], None), ("bf16", 64, 2, 1, [5000], None), ("bf16", 64, 6, 6, [700, 1, 900], [3000, 64, 900]), ("f32", 64, 2, 1, [1500], None),
    ("bf16", 128, 4, 1, [130, 700], [4000, 700]), ("bf16", 64, 64, 1, [90, 33], None), ("bf16", 128, 64, 1, [90, 33], [400, 30])])
@pytest.mark.parametrize("scale", [0.1, pk.PC_SCALE_FOLDED])
def test_prompt_longer_ones_of_every_head_size(dtype, D, Hq, Hkv, nq, nk, scale):
    run_prompt(dtype, Hq, Hkv, D, nq, nk, scale=scale)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("Hq,Hkv,lens,n,shared", [(8, 2, [130, 64, 0, 1], 1, 0), (8, 2, [5000, 300], 1, 0), (16, 4, [700 + 9 * i for i in range(9)], 40, 600),
                                                  (24, 8, [1500, 400], 300, 0), (16, 4, [4000 + i for i in range(30)], 1, 3900), (64, 1, [90, 500], 3, 60)])
def test_page_attn_folded_scale(dtype, D, Hq, Hkv, lens, n, shared):
    run_pages(dtype, Hq, Hkv, D, lens, n, shared=shared, scale=pk.PC_SCALE_FOLDED)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 70])
def test_page_attn_one_page_at_several_places(dtype, n):
    """Of one sequence, of two, and of the common rows."""
    pg = Paged(dtype, 2, 128, [300, 290], shared=128)
    pg.table[0, 3], pg.table[1, 2], pg.table[1, 3], pg.shared[1] = pg.table[0, 2].item(), pg.table[0, 2].item(), pg.shared[0].item(), pg.shared[0].item()
    for s in range(2):
        for x in (0, 1):
            own, common = pg.seqs[0][x][:, 128:192].clone(), pg.seqs[s][x][:, :64].clone()
            pg.seqs[s][x][:, 64:128] = common
            pg.seqs[s][x][:, 128:192] = own
            pg.seqs[s][x][:, 192:256] = own if s == 0 else common
    run_pages(dtype, 8, 2, 128, [300, 290], n, shared=128, paged=pg)


def test_two_graphs_that_share_a_workspace():
    """Recorded steps of different sizes on one workspace, replayed one behind the other on one stream."""
    pgs = [Paged("bf16", 2, 128, lens, shared=200, seed=i) for i, lens in enumerate(([700, 300], [260, 1900, 200]))]
    Qs = [normal(generator(i), 8, n, 128).to(torch.bfloat16) for i, n in enumerate((4, 3))]
    outs = [torch.zeros_like(q) for q in Qs]
    sizes = [pk.pc_page_attn_workspace_bytes(pk.PC_BF16, 8, 2, q.shape[1], 128, len(p.lens_host), max(p.lens_host), 200) for q, p in zip(Qs, pgs)]
    ws = torch.full((max(sizes),), 0xFF, dtype=torch.uint8, device=DEV)
    call = lambda i, **kw: pk.pc_page_attn(Qs[i], pgs[i].pages, pgs[i].table, pgs[i].lens, max(pgs[i].lens_host), 0.1, shared=pgs[i].shared, n_shared=200, **kw)
    want, graphs = [call(i) for i in range(2)], []
    for i in range(2):
        call(i, O=outs[i], ws=ws)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(i, O=outs[i], ws=ws)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1, 0)):
        for x in outs:
            x.zero_()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


@pytest.mark.parametrize("rows", [[5, 70], [1, 1]])
def test_stack_passes_over_one_step(rows):
    """Rows that are given anew replace those of the pass before: as if only the last pass had been."""
    results = []
    for passes in (1, 3):
        gen = generator(7)
        s = PagedStack(2, 8, 2, 128, 20, 128 ** -0.5)
        a, b = s.open(), s.open()
        draw = lambda n: [normal(gen, H, n, 128).to(torch.bfloat16) for H in (8, 2, 2)]
        for counts in ([130, 64], rows):
            s.begin([a, b], counts)
            T = sum(counts)
            pos = torch.arange(3 * T, dtype=torch.int32, device=DEV).reshape(T, 3)
            given = [[draw(T) for _ in range(2)] for _ in range(3)]
            for i in range(3 - passes, 3):
                out = [s.attend(l, *given[i][l], pos, again=i > 3 - passes) for l in range(2)]
            results.append(torch.stack(out))
        results[-2:] = [torch.cat(results[-2:], 2)]
        with pytest.raises(ValueError):
            s.attend(0, *draw(T), pos)
    assert torch.equal(*results)
