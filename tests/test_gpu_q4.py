"""The 4-bit cache (pc_q4_store, pc_q4_load, pc_q4_attn) and eviction by weight against plain 64-bit forms.

Codes, scales, moved rows and indices have to be equal bit for bit.  Tolerances of the attention, element by element,
with u = 2^-24 (half a step of fp32), A = the largest sum_d |q_d k_d| * scale of the call, in units of the logits:
  * a logit: D products summed in fp32 in any order, the scale folded into base 2 (three roundings), the subtraction
    of the reference: |ds| <= (D + 8) u A; the exponential adds a step of its result (v_exp_f32: 2 u) and its argument's
    rounding, up to u * 2 A * log2(e).  A probability is off by a factor of at most 1 + e, e = (D + 16) u A + 8 u.
  * O, fp32 inputs: (2 e + (Nk + 64) u) sum_j p_j |v_j|: probability and normaliser, sums of Nk terms, merges.
  * O, bf16 inputs: the probabilities are rounded to bf16 before the second product and O at the end, half a step each:
    2^-8 (|O| + sum_j p_j |v_j|) more.
  * lse: (D + 16) u A + (|lse| + Nk + 64) u;  weights: (2 e + (rows + 64) u) mass + 2 u (decay |w| + mass).
(Nk u is the worst case of a serial sum; the largest Nk here makes it 2^-11.)
"""
import numpy as np
import pytest
import torch

import paper_2601_04359_amd as pk
from oracle import q4_oracle as orc
from paper_2601_04359_amd.rollout import EvictingStack

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def packed(K, V, spare=3, head_gap=0):
    """A cache that holds float arrays K, V [H][n][D] in its first rows, quantised by the oracle; spare rows behind them
    hold NaN groups, head_gap more rows lie between heads."""
    H, n, D = K.shape
    out = []
    for x in (K, V):
        codes, scales = orc.q4_store(x)
        c = torch.full((H, n + spare + head_gap, D // 2), 0x77, dtype=torch.uint8)
        s = torch.full((H, n + spare + head_gap, D // 32), 255, dtype=torch.uint8)
        c[:, :n], s[:, :n] = torch.from_numpy(codes), torch.from_numpy(scales)
        out += [c.to(DEV)[:, :n + spare], s.to(DEV)[:, :n + spare]]
    return tuple(out)


def cache_values(cache, n):
    kc, ks, vc, vs = (t[:, :n].cpu().numpy() for t in cache)
    return orc.q4_load(kc, ks), orc.q4_load(vc, vs)


def rows(rng, shape, hard=True):
    """Rows with channels and groups of very different sizes, ties of the grid, zeros and tiny numbers."""
    x = rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[:-2] + (1, shape[-1])))
    if hard:
        flat = x.reshape(-1, shape[-1])
        n = len(flat)
        grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, -0.25, -2.5, -5.0, -7.0])
        flat[rng.integers(n), :32] = 0.0
        flat[rng.integers(n), :32] = np.resize(grid, 32)                 # every border between codes
        flat[rng.integers(n), 32:64] = np.resize(grid, 32) * 2.0 ** -100
        flat[rng.integers(n), 32:64] = np.resize(grid, 32) * 2.0 ** -122  # below the least scale
        flat[rng.integers(n), :32] = np.resize(grid, 32) * 2.0 ** 125     # the largest scale
        flat[rng.integers(n), 32:64] = 3.3e38
        flat[rng.integers(n), 0] = 1e-40
    return x


# ------------------------------------------------------------------------------ rows in, rows out
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,n,row0", [(1, 1, 0), (3, 7, 2), (112, 1, 5), (2, 129, 0), (5, 64, 31)])
def test_store_and_load(dtype, D, H, n, row0):
    rng = np.random.default_rng(H * n + D)
    big = [torch.from_numpy(rows(rng, (H, n + 4, D))).to(TYPES[dtype]).to(DEV) for _ in range(2)]
    K, V = big[0][:, :n], big[1][:, 2:n + 2]       # rows of longer heads
    K[0, 0, 3], V[-1, -1, 40], V[0, -1, 1] = float("nan"), float("inf"), -float("inf")
    cap = row0 + n + 3
    cache = tuple(torch.full((H, cap, w), 0xA5, dtype=torch.uint8, device=DEV) for w in (D // 2, D // 32) * 2)
    pk.pc_q4_store(K, V, cache, row0)
    for x, codes, scales in ((K, *cache[:2]), (V, *cache[2:])):
        want_c, want_s = orc.q4_store(f64(x))
        assert np.array_equal(scales[:, row0:row0 + n].cpu().numpy(), want_s)
        assert np.array_equal(codes[:, row0:row0 + n].cpu().numpy(), want_c)
        for t in (codes, scales):                   # the rows before and behind are as they were
            assert (t[:, :row0] == 0xA5).all() and (t[:, row0 + n:] == 0xA5).all()
    want = cache_values(tuple(t[:, row0:] for t in cache), n)
    for out in ("bf16", "f32"):
        Ko = torch.full((H, n + 1, D), 7.0, dtype=TYPES[out], device=DEV)
        Vo = Ko.clone()
        pk.pc_q4_load(cache, row0, Ko[:, :n], Vo[:, :n])
        for got, w in ((Ko, want[0]), (Vo, want[1])):
            assert np.array_equal(f64(got[:, :n]), w, equal_nan=True) and (got[:, n] == 7.0).all()
        one = torch.empty((H, n, D), dtype=TYPES[out], device=DEV)
        assert pk.pc_q4_load(cache, row0, V=one)[1] is one and np.array_equal(f64(one), want[1], equal_nan=True)
        assert pk.pc_q4_load(cache, row0, K=one)[0] is one and np.array_equal(f64(one), want[0], equal_nan=True)


@pytest.mark.parametrize("H,Hsel,n", [(4, 4, 3), (4, 1, 130), (6, 2, 1)])
def test_store_writes_the_rows_bookkeeping(H, Hsel, n):
    D, row0, cap = 128, 4, 4 + n + 2
    x = torch.randn((H, n, D), device=DEV, dtype=torch.bfloat16)
    cache = pk.q4_cache(H, cap, D)
    pos = torch.full((Hsel, cap, 3), -7, dtype=torch.int32, device=DEV)
    w = torch.full((Hsel, cap), 3.0, device=DEV)
    new = torch.arange(3 * n, dtype=torch.int32, device=DEV).view(n, 3)
    pk.pc_q4_store(x, x, cache, row0, pos_new=new, pos=pos, weights=w)
    assert torch.equal(pos[:, row0:row0 + n], new.expand(Hsel, n, 3)) and (w[:, row0:row0 + n] == 0).all()
    for rest in (slice(0, row0), slice(row0 + n, cap)):
        assert (pos[:, rest] == -7).all() and (w[:, rest] == 3.0).all()
    pk.pc_q4_store(x, x, cache, row0, weights=w.fill_(2.0))
    assert (w[:, row0:row0 + n] == 0).all() and (w[:, :row0] == 2.0).all()
    pk.pc_q4_store(x[:, :0], x[:, :0], cache, cap, weights=w)      # nothing to store


# ------------------------------------------------------------------------------ attention
def check_attn(dtype, Hq, Hkv, Nq, Nk, D, *, weights=None, decay=1.0, seed=0, scale=None, K=None, V=None, Q=None, q_gap=0,
               head_gap=0, lse=True, ws=None, visible=slice(None)):
    rng = np.random.default_rng(1000 * seed + Hq * 7 + Nq * 13 + Nk)
    scale = D ** -0.5 if scale is None else scale
    K = rng.standard_normal((Hkv, Nk, D)) if K is None else K
    V = rng.standard_normal((Hkv, Nk, D)) if V is None else V
    Q = rng.standard_normal((Hq, Nq, D)) * 1.5 if Q is None else Q
    cache = packed(K, V, head_gap=head_gap)
    Qd = torch.zeros((Hq, Nq + q_gap, D), dtype=TYPES[dtype], device=DEV)[:, :Nq]
    Qd.copy_(torch.from_numpy(Q))
    O = torch.full((Hq, Nq + q_gap, D), 9.0, dtype=TYPES[dtype], device=DEV)
    L = torch.empty((Hq, Nq), device=DEV) if lse else None
    w = None
    if weights is not None:
        w = torch.full((1 if weights == "one" else Hkv, Nk + 5), 3.0, device=DEV)
        w[:, :Nk] = torch.from_numpy(rng.exponential(1.0, (w.shape[0], Nk)))
        if decay == 0.0:
            w[:, :Nk] = float("nan")
        w0 = f64(w)
    pk.pc_q4_attn(Qd, cache, Nk, scale, O=O[:, :Nq], lse=L, weights=w, decay=decay, ws=ws)
    assert (O[:, Nq:] == 9.0).all()
    Kv, Vv = cache_values(cache, Nk)
    Qv = f64(Qd)
    want, want_l, mass = orc.attn(Qv, Kv, Vv, scale)
    spread = orc.attn(Qv, Kv, np.abs(Vv), scale)[0]            # sum_j p_j |v_j|
    rep = Hq // Hkv
    # keys that a call hides have probability 0 in either form: the bound is that of the others
    A = max(float((np.abs(Qv[h]) @ np.abs(Kv[h // rep][visible]).T).max()) for h in range(Hq)) * scale
    e = (D + 16) * U * A + 8 * U
    tol = (2 * e + (Nk + 64) * U) * spread
    if dtype == "bf16":
        tol += 2.0 ** -8 * (np.abs(want) + spread)
    err = np.abs(f64(O[:, :Nq]) - want)
    assert np.all(err <= tol + 1e-30), (err.max(), (err / (tol + 1e-30)).max())
    if lse:
        err = np.abs(f64(L) - want_l)
        assert np.all(err <= (D + 16) * U * A + (np.abs(want_l) + Nk + 64) * U), err.max()
    if w is not None:
        mass = mass.sum(0, keepdims=True) if weights == "one" else mass
        old = 0.0 if decay == 0.0 else decay * w0[:, :Nk]
        n = Hq * Nq if weights == "one" else rep * Nq
        tol = (2 * e + (n + 64) * U) * mass + 2 * U * (np.abs(old) + mass)
        err = np.abs(f64(w[:, :Nk]) - (old + mass))
        assert np.all(err <= tol + 1e-37), (err.max(), (err / (tol + 1e-37)).max())
        assert (w[:, Nk:] == 3.0).all()
    return O[:, :Nq], L, w


SHAPES = [   # Hq, Hkv, Nq, Nk
    (1, 1, 1, 1), (2, 1, 1, 2), (4, 4, 1, 15), (8, 2, 1, 16), (8, 2, 1, 17), (6, 2, 3, 31), (4, 1, 4, 32), (16, 4, 1, 33),
    (3, 1, 5, 64), (24, 8, 1, 255), (8, 2, 2, 257), (5, 1, 3, 511), (2, 2, 9, 1000), (16, 4, 4, 1179), (8, 8, 17, 300),
    (2, 1, 16, 777), (4, 2, 23, 90), (16, 1, 1, 5000), (32, 1, 1, 640), (6, 2, 40, 129), (4, 2, 64, 1804), (2, 2, 131, 515),
    (8, 2, 100, 260), (16, 4, 37, 2000),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,Nq,Nk", SHAPES)
def test_attn(dtype, D, Hq, Hkv, Nq, Nk):
    check_attn(dtype, Hq, Hkv, Nq, Nk, D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("weights", ["each", "one"])
@pytest.mark.parametrize("Hq,Hkv,Nq,Nk,D,decay", [
    (1, 1, 1, 1, 64, 1.0), (8, 2, 1, 17, 128, 0.98), (16, 4, 1, 1179, 128, 0.0), (6, 2, 11, 64, 64, 0.5), (24, 8, 1, 260, 128, 1.0),
    (4, 2, 23, 515, 64, 0.9), (8, 2, 37, 1804, 128, 0.0), (3, 1, 70, 33, 128, 1.0), (4, 4, 1, 4097, 64, 0.25),
    (8, 2, 100, 300, 128, 2.0)])
def test_attn_weights(dtype, weights, Hq, Hkv, Nq, Nk, D, decay):
    check_attn(dtype, Hq, Hkv, Nq, Nk, D, weights=weights, decay=decay, lse=Nk % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,Nq,Nk", [(16, 8, 20, 8300), (16, 8, 20, 16500), (24, 8, 9, 12289)])
def test_attn_weights_of_many_keys(dtype, D, Hq, Hkv, Nq, Nk):
    """Waves with keys of their own, one, two and four groups of them per work-group, 64 and 128 keys each, the last work-group's
    in part behind the last key."""
    check_attn(dtype, Hq, Hkv, Nq, Nk, D, weights="each", decay=0.75)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,Nq,Nk", [(128, 16, 1, 700), (128, 16, 1, 3000), (72, 6, 1, 1100), (36, 18, 4, 90)])
def test_attn_weights_of_many_heads_in_one_sum(dtype, Hq, Hkv, Nq, Nk):
    """More than 64 kept logit rows behind one sum, in one share of the keys and in several."""
    check_attn(dtype, Hq, Hkv, Nq, Nk, 64, weights="one", decay=0.9)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,Nq,Nk,first", [(128, 16, 1, 700, 350), (128, 16, 1, 3000, 1000), (16, 8, 20, 16500, 9000)])
def test_attn_hidden_keys_of_many_heads_and_keys(dtype, Hq, Hkv, Nq, Nk, first):
    check_hidden_rows(dtype, 128, Hq, Hkv, Nq, Nk, "one" if Nq == 1 else "each", 1e20, -2.0, 128 ** -0.5, first)


@pytest.mark.parametrize("weights", [None, "each", "one"])
@pytest.mark.parametrize("Hq,Hkv,Nq,Nk,gaps,decay", [
    (4, 1, 192, 33, 0, 1.0), (8, 2, 200, 300, 0, 0.9), (6, 2, 257, 1000, 5, 0.0), (4, 1, 1000, 1, 0, 0.5), (16, 4, 193, 130, 3, 2.0),
    (2, 2, 800, 515, 0, 1.0), (2, 2, 767, 400, 1, 0.3)])
def test_attn_many_rows(weights, Hq, Hkv, Nq, Nk, gaps, decay):
    """On both sides of the 768 rows per KV head from which on the cache is turned into bf16 rows."""
    check_attn("bf16", Hq, Hkv, Nq, Nk, 128, weights=weights, decay=decay, q_gap=gaps, head_gap=gaps, lse=weights != "one")


@pytest.mark.parametrize("Nq", [200, 400])
def test_attn_many_rows_hard(Nq):
    """Climbing logits, hidden keys and values that are not numbers, in the form for many rows."""
    Hq, Hkv, Nk, D = 8, 2, 500, 128
    rng = np.random.default_rng(6)
    K, Q = rng.standard_normal((Hkv, Nk, D)) * 0.1, rng.standard_normal((Hq, Nq, D)) * 0.1
    K[..., 0], Q[..., 0] = np.linspace(0, 6, Nk), 1000.0
    check_attn("bf16", Hq, Hkv, Nq, Nk, D, K=K, Q=Q, weights="each")
    hidden = np.arange(Nk) % 50 != 17
    K, Q = rng.standard_normal((Hkv, Nk, D)), rng.standard_normal((Hq, Nq, D))
    K[:, :, 127], K[:, :, 96:127], Q[..., 127] = np.where(hidden, -6.0, 0.0), 0.0, 2.0 ** 100
    _, _, w = check_attn("bf16", Hq, Hkv, Nq, Nk, D, K=K, Q=Q, weights="each", decay=0.0, visible=~hidden)
    assert (w[:, :Nk][:, torch.from_numpy(hidden).to(DEV)] == 0).all()
    V = rng.standard_normal((Hkv, Nk, D))
    V[1, 3, 70] = np.nan
    O = pk.pc_q4_attn(torch.randn((Hq, Nq, D), device=DEV).to(torch.bfloat16), packed(rng.standard_normal((Hkv, Nk, D)), V), Nk, 0.1)
    bad = torch.isnan(O)
    assert bad[4:, :, 64:96].all() and not bad[4:, :, :64].any() and not bad[4:, :, 96:].any() and not bad[:4].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Nq", [1, 30, 150])
def test_attn_long(dtype, Nq):
    """Many shares, and far more keys than a share."""
    check_attn(dtype, 4, 2, Nq, 20011, 128, weights="each", decay=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Nq,D", [(1, 128), (21, 64), (90, 128)])
def test_attn_strides(dtype, Nq, D):
    """Heads of the cache, the queries and the output further apart than their rows."""
    check_attn(dtype, 6, 3, Nq, 203, D, weights="each", q_gap=3, head_gap=17)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Nq", [1, 40, 130])
@pytest.mark.parametrize("order", ["up", "down", "peak"])
def test_attn_reference_moves(dtype, Nq, order):
    """Logits that climb through the keys by hundreds, fall, or peak at one key in the middle."""
    Hq, Hkv, Nk, D = 4, 2, 700, 128
    rng = np.random.default_rng(5)
    K, Q = rng.standard_normal((Hkv, Nk, D)) * 0.1, rng.standard_normal((Hq, Nq, D)) * 0.1
    K[..., 0] = {"up": np.linspace(0, 6, Nk), "down": np.linspace(6, 0, Nk), "peak": (np.arange(Nk) == 351) * 6.0}[order]
    Q[..., 0] = 1000.0 if order != "peak" else 300.0
    check_attn(dtype, Hq, Hkv, Nq, Nk, D, K=K, Q=Q, weights="each")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Nq", [1, 33, 130])
def test_attn_masked_by_a_coordinate(dtype, Nq):
    """Keys that a caller hides through a dimension of its own: logits of -1e30 in the first and the last shares, one
    key in a hundred visible.  Hidden keys get weight 0."""
    Hq, Hkv, Nk, D = 4, 2, 3000, 128
    rng = np.random.default_rng(9)
    K, Q = rng.standard_normal((Hkv, Nk, D)), rng.standard_normal((Hq, Nq, D))
    hidden = np.arange(Nk) % 100 != 57
    K[:, :, 127] = np.where(hidden, -6.0, 0.0)
    K[:, :, 96:127] = 0.0
    Q[..., 127] = 2.0 ** 100
    _, _, w = check_attn(dtype, Hq, Hkv, Nq, Nk, D, K=K, Q=Q, weights="each", decay=0.0, visible=~hidden)
    assert (w[:, :Nk][:, torch.from_numpy(hidden).to(DEV)] == 0).all()


def check_hidden_rows(dtype, D, Hq, Hkv, Nq, Nk, weights, big, level, scale, first_visible):
    """Keys hidden through dimensions of their own: a third of the rows sees the keys from first_visible on, one in three, a
    third sees none (all hidden alike: every key weighs the same), a third sees none and hides some twice (the others share).
    The rows without a visible key are zero in every other dimension, so that their logits are exact in any precision."""
    rng = np.random.default_rng(Nk + Nq + int(np.log2(big) - level))
    K, V, Q = (rng.standard_normal((h, n, D)) for h, n in ((Hkv, Nk), (Hkv, Nk), (Hq, Nq)))
    hidden = (np.arange(Nk) % 3 != 0) | (np.arange(Nk) < first_visible)
    K[..., D - 32:], Q[..., D - 32:] = 0.0, 0.0
    K[..., D - 1], K[..., D - 2] = np.where(hidden, level, 0.0), level
    kind = np.arange(Hq * Nq).reshape(Hq, Nq) % 3
    Q[kind > 0] = 0.0
    Q[..., D - 1], Q[..., D - 2] = np.where(kind != 1, big, 0.0), np.where(kind > 0, big, 0.0)
    cache, Qd = packed(K, V), torch.from_numpy(Q).to(TYPES[dtype]).to(DEV)
    lse = torch.empty((Hq, Nq), device=DEV)
    w = None if weights is None else torch.full((1 if weights == "one" else Hkv, Nk), 2.0, device=DEV)
    O = pk.pc_q4_attn(Qd, cache, Nk, scale, lse=lse, weights=w, decay=0.5)
    Kv, Vv = cache_values(cache, Nk)
    want, want_l, mass = orc.attn(f64(Qd), Kv, Vv, scale)
    spread = orc.attn(f64(Qd), Kv, np.abs(Vv), scale)[0]
    # the logits that are not hidden; those of the other rows are exact, 0 beside their reference, which leaves the logarithm of
    # the sum: log2(Nk) <= 15 in half a step of its own, less than (D + 16) u A
    A = max(15.0, float(np.abs(f64(Qd)[..., :D - 32]).sum(-1).max() * np.abs(Kv).max() * scale))
    e = (D + 16) * U * A + 8 * U
    tol = (2 * e + (Nk + 64) * U) * spread + (2.0 ** -8 * (np.abs(want) + spread) if dtype == "bf16" else 0)
    assert np.all(np.abs(f64(O) - want) <= tol + 1e-30), np.abs(f64(O) - want).max()
    # scale to base 2, the product, and back: 4 roundings of a far logit
    assert np.all(np.abs(f64(lse) - want_l) <= (D + 16) * U * A + (5 * np.abs(want_l) + Nk + 64) * U)
    if w is not None:
        mass = mass.sum(0, keepdims=True) if weights == "one" else mass
        n = Hq * Nq if weights == "one" else Hq // Hkv * Nq
        assert np.all(np.abs(f64(w) - (1.0 + mass)) <= (2 * e + (n + 64) * U) * mass + 2 * U * (1.0 + mass))


HIDDEN_BY = [(1e12, -2.0, 0.125), (1e20, -2.0, 128 ** -0.5), (1e30, -1.0, 0.125), (1e30, -3.0, 0.1)]     # a query's entry, a key's, the scale


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("weights", ["each", "one"])
@pytest.mark.parametrize("big,level,scale", HIDDEN_BY)
@pytest.mark.parametrize("D,Hq,Hkv,Nq,Nk,first", [(128, 4, 2, 1, 3000, 1500), (64, 6, 2, 5, 700, 300), (128, 4, 2, 33, 900, 290),
                                                  (128, 6, 3, 1, 90, 40), (64, 2, 1, 130, 3000, 1100)])
def test_attn_hidden_keys_and_rows_without_any_other(dtype, weights, big, level, scale, D, Hq, Hkv, Nq, Nk, first):
    check_hidden_rows(dtype, D, Hq, Hkv, Nq, Nk, weights, big, level, scale, first)


@pytest.mark.parametrize("weights", ["each", "one", None])
@pytest.mark.parametrize("big,level,scale", HIDDEN_BY)
@pytest.mark.parametrize("Hq,Hkv,Nq,Nk,first", [(4, 2, 400, 900, 290), (16, 8, 385, 130, 60), (6, 2, 1000, 33, 10), (2, 1, 800, 3000, 1500)])
def test_attn_many_rows_hidden_keys_and_rows_without_any_other(weights, big, level, scale, Hq, Hkv, Nq, Nk, first):
    check_hidden_rows("bf16", 128, Hq, Hkv, Nq, Nk, weights, big, level, scale, first)


@pytest.mark.parametrize("Nq", [1, 30, 400])
def test_attn_hidden_keys_of_queries_that_carry_the_scale(Nq):
    """ln 2 as the scale: the form for many rows takes pc_frame_attn's and pc_score's shorter loops."""
    check_hidden_rows("bf16", 128, 4, 2, Nq, 900, "each", 1e20, -2.0, pk.PC_SCALE_FOLDED, 290)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Nq", [1, 20, 130])
def test_attn_not_a_number(dtype, Nq):
    """A key group that holds a NaN spoils its KV head's rows, a value group its 32 dims; the other head is untouched."""
    Hq, Hkv, Nk, D = 4, 2, 400, 128
    rng = np.random.default_rng(2)
    K, V = rng.standard_normal((Hkv, Nk, D)), rng.standard_normal((Hkv, Nk, D))
    V[1, 399, 70] = np.inf
    cache, Q = packed(K, V), torch.randn((Hq, Nq, D), device=DEV).to(TYPES[dtype])
    O = pk.pc_q4_attn(Q, cache, Nk, 0.1)
    bad = torch.isnan(O)
    assert bad[2:, :, 64:96].all() and not bad[2:, :, :64].any() and not bad[2:, :, 96:].any() and not bad[:2].any()
    K[1, 17, 5] = np.nan
    L, w = torch.zeros((Hq, Nq), device=DEV), torch.zeros((Hkv, Nk), device=DEV)
    O = pk.pc_q4_attn(Q, packed(K, V), Nk, 0.1, lse=L, weights=w)
    assert torch.isnan(O[2:]).all() and not torch.isnan(O[:2]).any()
    assert torch.isnan(L[2:]).all() and not torch.isnan(L[:2]).any() and not torch.isnan(w[0]).any()


@pytest.mark.parametrize("Nq,Nk", [(1, 5000), (50, 700), (150, 700)])
def test_attn_is_reproducible_and_takes_a_workspace(Nq, Nk):
    Hq, Hkv, D = 8, 2, 128
    rng = np.random.default_rng(3)
    cache = packed(rng.standard_normal((Hkv, Nk, D)), rng.standard_normal((Hkv, Nk, D)))
    Q = torch.randn((Hq, Nq, D), device=DEV, dtype=torch.bfloat16)
    n = pk.pc_q4_attn_workspace_bytes(pk.PC_BF16, Hq, Hkv, Nq, Nk, D, True)
    assert n > 0
    outs = []
    for _ in range(3):
        ws = torch.randint(0, 255, (n,), dtype=torch.uint8, device=DEV)
        w = torch.ones((Hkv, Nk), device=DEV)
        outs.append((pk.pc_q4_attn(Q, cache, Nk, 0.09, weights=w, ws=ws), w))
    for O, w in outs[1:]:
        assert torch.equal(O, outs[0][0]) and torch.equal(w, outs[0][1])
    with pytest.raises(pk.PackCacheError) as e:
        pk.pc_q4_attn(Q, cache, Nk, 0.09, weights=w, ws=torch.empty(n - 1, dtype=torch.uint8, device=DEV))
    assert e.value.status == -6


# ------------------------------------------------------------------------------ eviction
def check_evict(kind, H, Hsel, Nk, n_keep, D=128, n_anchor=0, recent_t=0, w=None, t=None, with_pos=True, with_idx=True, seed=0):
    rng = np.random.default_rng(seed + Nk * 3 + n_keep)
    cap = Nk + 2
    w = rng.exponential(1.0, (Hsel, Nk)) if w is None else w
    wd = torch.full((Hsel, cap), 5.0, device=DEV)
    wd[:, :Nk] = torch.from_numpy(np.asarray(w, np.float64))
    pos = torch.from_numpy(rng.integers(-1000, 1000, (Hsel, cap, 3))).int().to(DEV)
    if t is not None:
        pos[:, :Nk, 0] = torch.from_numpy(np.asarray(t)).int().to(DEV)
    if kind == "q4":
        data = tuple(torch.randint(0, 255, (H, cap, b), dtype=torch.uint8, device=DEV) for b in (D // 2, D // 32) * 2)
    else:
        data = tuple(torch.randn((H, cap, D), device=DEV).to(TYPES[kind]) for _ in range(2))
    before = [x.clone() for x in data] + ([pos.clone()] if with_pos else []) + [wd.clone()]
    idx = torch.full((Hsel, n_keep + 1), -1, dtype=torch.int32, device=DEV)[:, :n_keep] if with_idx else None
    args = (pos if with_pos else None, wd, Nk, n_keep, n_anchor, recent_t)
    left = pk.pc_q4_evict(data, *args, idx=idx) if kind == "q4" else pk.pc_evict(*data, *args, idx=idx)
    assert left == min(n_keep, Nk)
    after = list(data) + ([pos] if with_pos else []) + [wd]
    t_host = pos_t = before[-2][..., 0].cpu().numpy() if with_pos else None
    w_host = before[-1].cpu().numpy()
    for s in range(Hsel):
        src = orc.evict_rows(w_host[s], None if pos_t is None else t_host[s], Nk, n_keep, n_anchor, recent_t)
        if with_idx:
            assert np.array_equal(idx[s].cpu().numpy(), src)
        src = torch.from_numpy(src).to(DEV)
        per = H // Hsel
        for a, b in zip(after, before):
            for h in range(s * per, (s + 1) * per) if a.shape[0] == H and a is not wd and a is not pos else (s,):
                assert torch.equal(a[h, :left].view(torch.uint8), b[h][src].view(torch.uint8))
                assert torch.equal(a[h, left:].view(torch.uint8), b[h, left:].view(torch.uint8))


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("f32", 64), ("q4", 128), ("q4", 64), ("bf16", 72)])
@pytest.mark.parametrize("H,Hsel,Nk,n_keep", [(1, 1, 2, 1), (2, 2, 65, 64), (4, 1, 300, 17), (4, 4, 1025, 1000), (6, 2, 1024, 512),
                                              (2, 2, 5000, 4999), (3, 3, 2049, 1), (112, 28, 33, 20)])
def test_evict(kind, D, H, Hsel, Nk, n_keep):
    check_evict(kind, H, Hsel, Nk, n_keep, D=D)


@pytest.mark.parametrize("Nk,n_keep", [(20000, 19999), (20000, 300), (70001, 35000), (33000, 32768)])
def test_evict_long(Nk, n_keep):
    check_evict("q4", 2, 2, Nk, n_keep, n_anchor=100, recent_t=40)


@pytest.mark.parametrize("Nk", [100, 3000, 40000])
@pytest.mark.parametrize("what", ["equal", "zeros", "few", "special", "narrow", "spread", "ramp"])
def test_evict_weights_that_tie(Nk, what):
    rng = np.random.default_rng(11)
    w = {"equal": np.full(Nk, 0.37), "zeros": np.where(rng.random(Nk) < 0.9, 0.0, -0.0), "few": rng.integers(0, 3, Nk) * 1.0,
         "special": rng.choice([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, 1.0, -1.0], Nk),
         "narrow": 1.0 + rng.integers(0, 50, Nk) * 2.0 ** -23, "spread": np.exp(rng.normal(0, 25, Nk)).clip(0, 3e38),
         "ramp": np.arange(Nk)[::-1] * 1.0}[what]
    for n_keep in (1, Nk // 3, Nk - 1):
        check_evict("q4", 2, 2, Nk, n_keep, w=np.stack([w, np.roll(w, 7)]))


@pytest.mark.parametrize("Nk", [5, 64, 1030, 4096, 4097, 8321, 24576, 24577, 30000, 100001])
@pytest.mark.parametrize("n_out", [1, 2, 3, 4, 5, 8, 9])
def test_evict_few(Nk, n_out):
    """A token or a few leave: found one by one up to eight, with ties, protected rows and rows of the newest among them."""
    rng = np.random.default_rng(Nk + n_out)
    if n_out >= Nk:
        return
    w = rng.integers(0, max(2, Nk // 3), (3, Nk)) * 0.5
    w[1] = rng.choice([np.nan, 0.0, -0.0, 1.0, np.inf], Nk)
    w[2, -n_out:] = -1.0                   # all that leave lie behind n_keep: nothing moves
    t = np.stack([np.arange(Nk), rng.integers(0, 9, Nk), np.arange(Nk)])
    check_evict("q4", 3, 3, Nk, Nk - n_out, w=w, t=t, n_anchor=min(2, Nk - n_out), recent_t=0 if n_out == 2 else 2)
    check_evict("bf16", 6, 3, Nk, Nk - n_out, w=w, with_pos=False, with_idx=n_out % 2 == 0)
    if Nk in (1030, 30000):
        check_evict("f32", 60, 1, Nk, Nk - n_out, D=128, w=w[:1])      # too much to move in the same launch
        check_evict("bf16", 2, 2, Nk, Nk - n_out, n_anchor=Nk - n_out, w=w[:2])     # every row below n_keep an anchor
        check_evict("q4", 1, 1, Nk, Nk - n_out, w=w[:1], t=np.zeros((1, Nk)), recent_t=1)     # every row recent


@pytest.mark.parametrize("Nk,n_keep,n_anchor,recent_t", [
    (50, 20, 20, 0), (50, 20, 0, 1), (50, 20, 5, 30), (50, 3, 3, 1000), (9000, 40, 10, 5), (9000, 8999, 4000, 2 ** 31 - 1)])
@pytest.mark.parametrize("order", ["up", "same", "mixed", "far"])
def test_evict_anchors_and_recent_rows(Nk, n_keep, n_anchor, recent_t, order):
    rng = np.random.default_rng(4)
    t = {"up": np.arange(Nk), "same": np.full(Nk, 3), "mixed": rng.integers(0, Nk, Nk),
         "far": rng.choice([-2 ** 31, 2 ** 31 - 1, 0], Nk)}[order]
    check_evict("bf16", 2, 2, Nk, n_keep, n_anchor=n_anchor, recent_t=recent_t, t=np.stack([t, t[::-1]]))


def test_evict_without_coordinates_or_index():
    check_evict("bf16", 4, 2, 900, 700, with_pos=False, n_anchor=10)
    check_evict("q4", 4, 4, 900, 5, with_pos=False, with_idx=False)
    check_evict("f32", 4, 1, 900, 899, with_idx=False)


def test_evict_nothing():
    for n_keep in (10, 11):
        check_evict("bf16", 2, 2, 10, n_keep, with_idx=False)
    data = torch.randn((2, 10, 128), device=DEV)
    w = torch.ones((2, 10), device=DEV)
    assert pk.pc_evict(data, data.clone(), None, w, 10, 0) == 0 and pk.pc_evict(data, data.clone(), None, w, 0, 4) == 0
    with pytest.raises(pk.PackCacheError):
        pk.pc_evict(data, data.clone(), None, w, 10, 10, idx=torch.empty((2, 10), dtype=torch.int32, device=DEV))


# ------------------------------------------------------------------------------ the calls together
def test_offsets_beyond_32_bits():
    """A cache whose rows pass 2^31 and whose heads pass 2^32 bytes: 36 million rows of 64 bytes, two heads.  All keys are
    zero but for a few far apart that every query looks at."""
    H, Nk, D = 2, 36_000_000, 128
    cache = tuple(torch.zeros((H, Nk, w), dtype=torch.uint8, device=DEV) for w in (D // 2, D // 32) * 2)
    rows = torch.tensor([5, 17_000_000, 33_600_000, Nk - 1], device=DEV)
    K = torch.zeros((H, 4, D), device=DEV)
    K[..., 3] = 6.0
    V = torch.arange(4, device=DEV)[None, :, None] % 2 * 2.0 + torch.arange(H, device=DEV)[:, None, None] * 4.0 + torch.zeros((H, 4, D), device=DEV)
    small = pk.q4_cache(H, 4, D)
    pk.pc_q4_store(K, V, small, 0)
    for big, part in zip(cache, small):
        big[:, rows] = part
    Q = torch.zeros((H, 1, D), device=DEV)
    Q[..., 3] = 20.0
    lse, w = torch.zeros((H, 1), device=DEV), torch.zeros((H, Nk), device=DEV)
    O = pk.pc_q4_attn(Q, cache, Nk, 1.0, lse=lse, weights=w)
    # logits 120 against 0: the others' mass is 36e6 e^-120
    assert torch.allclose(O, V.mean(1, keepdim=True), atol=1e-5) and torch.allclose(lse, torch.full_like(lse, 120 + np.log(4)), rtol=1e-6)
    assert torch.allclose(w[:, rows], torch.full((H, 4), 0.25, device=DEV), rtol=1e-5)
    w[:, 20:1020] = 1e-3      # and they are what an eviction keeps
    left = pk.pc_q4_evict(cache, None, w, Nk, 1004)
    want = torch.cat([torch.tensor([5], device=DEV), rows[1:], ])
    assert left == 1004 and torch.allclose(w[:, :1020].sum(1), torch.full((2,), 1.0 + 1000 * 1e-3 + 16 * 1e-3, device=DEV), rtol=1e-3)
    Ko, Vo = (torch.empty((H, 1004, D), device=DEV) for _ in range(2))
    pk.pc_q4_load(cache, 0, Ko, Vo)
    assert torch.equal((Ko[..., 3] == 6.0).sum(1), torch.full((H,), len(want), device=DEV))
    one = torch.empty((H, 1, D), device=DEV)
    pk.pc_q4_load(cache, Nk - 1, V=one)
    assert torch.equal(one, V[:, 3:])
    pk.pc_q4_store(K[:, :1], V[:, 1:2], cache, Nk - 2)
    pk.pc_q4_load(cache, Nk - 2, V=one)
    assert torch.equal(one, V[:, 1:2])


@pytest.mark.parametrize("Nq", [1, 30, 300])
def test_both_halves_of_the_binding_give_the_same_bits(monkeypatch, Nq):
    from paper_2601_04359_amd import binding
    H, Hq, D, n = 2, 6, 128, 200
    x = [torch.randn((H, n, D), device=DEV).to(torch.bfloat16) for _ in range(2)]
    Q = torch.randn((Hq, Nq, D), device=DEV).to(torch.bfloat16)
    new = torch.arange(3 * n, dtype=torch.int32, device=DEV).view(n, 3)
    results = []
    for native in (True, False):
        assert pk.lib() and binding._NATIVE
        with monkeypatch.context() as m:
            if not native:
                m.setattr(binding, "_NATIVE", False)
            cache, pos, w = pk.q4_cache(H, n + 4, D), torch.zeros((H, n + 4, 3), dtype=torch.int32, device=DEV), torch.ones((H, n + 4), device=DEV)
            pk.pc_q4_store(*x, cache, 2, new, pos, w)
            O, lse = torch.empty_like(Q), torch.empty((Hq, Nq), device=DEV)
            assert pk.pc_q4_attn(Q, cache, n + 2, 0.1, O=O, lse=lse, weights=w, decay=0.5) is O
            idx = torch.empty((H, 77), dtype=torch.int32, device=DEV)
            assert pk.pc_q4_evict(cache, pos, w, n + 2, 77, n_anchor=3, recent_t=20, idx=idx) == 77
            K, V = torch.empty((H, 77, D), device=DEV), torch.empty((H, 77, D), device=DEV)
            assert pk.pc_q4_load(cache, 0, K, V) == (K, V)
            rows_k, rows_v = x[0].clone(), x[1].clone()
            w2 = w[:, :n].contiguous()
            assert pk.pc_evict(rows_k, rows_v, None, w2, n, 50) == 50
            results.append([*cache, pos, w, O, lse, idx, K, V, rows_k, rows_v, w2])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("native", [True, False])
def test_one_row_of_any_stride(monkeypatch, native):
    """One token's heads as a projection leaves them, [1][H][D], seen as [H][1][D]."""
    from paper_2601_04359_amd import binding
    assert pk.lib() and binding._NATIVE
    if not native:
        monkeypatch.setattr(binding, "_NATIVE", False)
    H, Hq, D = 4, 8, 128
    x = torch.randn((3, 1, Hq, D), device=DEV).to(torch.bfloat16)
    K, V, Q = (t.transpose(0, 1) for t in (x[0, :, :H], x[1, :, 3:3 + H], x[2]))
    a, b = pk.q4_cache(H, 3, D), pk.q4_cache(H, 3, D)
    pk.pc_q4_store(K, V, a, 1)
    pk.pc_q4_store(K.contiguous(), V.contiguous(), b, 1)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    out = torch.zeros((1, Hq, D), device=DEV, dtype=torch.bfloat16)
    pk.pc_q4_attn(Q, a, 2, 0.1, O=out.transpose(0, 1))
    assert torch.equal(out.transpose(0, 1), pk.pc_q4_attn(Q.contiguous(), b, 2, 0.1))
    k = torch.zeros((1, H, D), device=DEV)
    pk.pc_q4_load(a, 1, K=k.transpose(0, 1))
    assert torch.equal(k.transpose(0, 1), pk.pc_q4_load(b, 1, K=torch.zeros((H, 1, D), device=DEV))[0])
    with pytest.raises(pk.PackCacheError):
        pk.pc_q4_store(x[0, 0, :H, ::2][:, None], x[0, 0, :H, ::2][:, None], pk.q4_cache(H, 3, 64), 0)      # dims apart


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("Nq", [1, 30, 767, 768])
def test_one_head_of_any_stride(Nq, weights):
    """A single head as a projection leaves it, [Nq][1][D], seen as [1][Nq][D]: its stride between heads is D, or anything."""
    D, Nk = 128, 300
    x, k, v = (torch.randn((n, 1, D), device=DEV).to(torch.bfloat16) for n in (Nq, Nk, Nk))
    Q, K, V = (t.transpose(0, 1) for t in (x, k, v))
    assert Q.stride(0) == D
    cache, w, wo = pk.q4_cache(1, Nk, D), torch.zeros((1, Nk), device=DEV), torch.zeros((1, Nk), device=DEV)
    pk.pc_q4_store(K, V, cache, 0)
    out = torch.zeros((Nq, 1, D), device=DEV, dtype=torch.bfloat16)
    pk.pc_q4_attn(Q, cache, Nk, 0.1, O=out.transpose(0, 1), weights=w if weights else None)
    want = pk.pc_q4_attn(x.view(1, Nq, D), cache, Nk, 0.1, weights=wo if weights else None)
    assert torch.equal(out.transpose(0, 1), want) and torch.equal(w, wo)
    back = torch.zeros((Nk, 1, D), device=DEV)
    pk.pc_q4_load(cache, 0, K=back.transpose(0, 1))
    assert torch.equal(back.transpose(0, 1), pk.pc_q4_load(cache, 0, K=torch.zeros((1, Nk, D), device=DEV))[0])
    odd = torch.as_strided(x, (1, Nq, D), (Nq * D + 1, D, 1))
    assert torch.equal(pk.pc_q4_attn(odd, cache, Nk, 0.1), pk.pc_q4_attn(x.view(1, Nq, D), cache, Nk, 0.1))


def step_inputs(rng, layers, Hq, Hkv, n, D, t):
    K, V = (torch.from_numpy(rng.standard_normal((layers, Hkv, n, D))).to(torch.bfloat16).to(DEV) for _ in range(2))
    Q = torch.from_numpy(rng.standard_normal((layers, Hq, n, D)) * 2).to(torch.bfloat16).to(DEV)
    pos = torch.stack([torch.arange(t, t + n), torch.arange(n) % 3, torch.arange(n) % 5], 1).int().to(DEV)
    return K, V, Q, pos


@pytest.mark.parametrize("share", [False, True])
@pytest.mark.parametrize("budget", [45, 24])
@pytest.mark.parametrize("n,n_anchor,recent,decay", [(1, 4, 6, 1.0), (3, 0, 0, 0.9), (7, 10, 14, 0.5)])
def test_stack_step_by_step(share, n, n_anchor, recent, decay, budget):
    """A prompt and a dozen steps of two layers; each step is checked from the state the device holds when it begins."""
    layers, Hq, Hkv, D = 2, 8, 2, 128
    rng = np.random.default_rng(n)
    s = EvictingStack(layers, Hq, Hkv, D, budget, D ** -0.5, step_rows=20, n_anchor=n_anchor, recent_t=recent, decay=decay,
                      share_heads=share)
    hsel = 1 if share else Hkv
    t = 0
    for step in range(12):
        rows_in = 20 if step == 0 else n
        K, V, Q, pos = step_inputs(rng, layers, Hq, Hkv, rows_in, D, t)
        t += rows_in
        w_before, before = f64(s.weights), s.nk
        for layer in range(layers):
            s.append(layer, K[layer], V[layer], pos)
            O = s.attend(layer, Q[layer], q_pos=pos)
            cache, p, w = s.layer(layer)
            nk = before + rows_in
            assert torch.equal(p[:, before:nk], pos.expand(hsel, rows_in, 3))
            Kv, Vv = cache_values(cache, nk)
            for x, v, c, sc in ((K, Kv, cache[0], cache[1]), (V, Vv, cache[2], cache[3])):
                codes, scales = orc.q4_store(f64(x[layer]))        # the rotated keys, as they lie in K now
                assert np.array_equal(c[:, before:nk].cpu().numpy(), codes) and np.array_equal(sc[:, before:nk].cpu().numpy(), scales)
            want, _, mass = orc.attn(f64(Q[layer]), Kv, Vv, s.scale)
            spread = orc.attn(f64(Q[layer]), Kv, np.abs(Vv), s.scale)[0]
            assert np.all(np.abs(f64(O) - want) <= 2.0 ** -8 * (np.abs(want) + spread) + 1e-4 * spread)
            mass = mass.sum(0, keepdims=True) if share else mass
            old = decay * w_before[layer * hsel:(layer + 1) * hsel, :nk]
            old[:, before:] = 0
            assert np.allclose(f64(w[:, :nk]), old + mass, rtol=1e-4, atol=1e-7)
        state = [x.clone() for x in (*s.cache, s.pos, s.weights)]
        left = s.end_step()
        nk = before + rows_in
        assert left == s.nk == min(nk, budget)
        for sel in range(layers * hsel):
            src = orc.evict_rows(state[5][sel].cpu().numpy(), state[4][sel, :, 0].cpu().numpy(), nk, left, n_anchor, recent)
            src = torch.from_numpy(src).to(DEV)
            per = Hkv // hsel
            for h in range(sel * per, (sel + 1) * per):
                for a, b in zip(s.cache, state):
                    assert torch.equal(a[h, :left], b[h][src])
            assert torch.equal(s.pos[sel, :left], state[4][sel][src]) and torch.equal(s.weights[sel, :left], state[5][sel][src])
    assert s.nk == min(20 + 11 * n, budget)


@pytest.mark.parametrize("n,budget", [(1, 700), (5, 90), (210, 400)])
def test_stack_step_in_a_graph(n, budget):
    """A step of the full cache, recorded once and replayed with eager work in between, leaves what eager steps leave."""
    layers, Hq, Hkv, D = 2, 8, 2, 128
    rng = np.random.default_rng(8)
    args = (layers, Hq, Hkv, D, budget, D ** -0.5)
    kw = dict(step_rows=max(n, budget), n_anchor=8, recent_t=4, decay=0.97)
    a, b = EvictingStack(*args, **kw), EvictingStack(*args, **kw)
    K, V, Q, pos = step_inputs(rng, layers, Hq, Hkv, budget, D, 0)
    for s in (a, b):
        for layer in range(layers):
            s.append(layer, K[layer].clone(), V[layer], pos)
        s.end_step()
    ins = [x.clone() for x in step_inputs(rng, layers, Hq, Hkv, n, D, 0)]
    Oa = torch.empty_like(ins[2])

    def one(s, K, V, Q, pos, O):
        for layer in range(layers):
            s.append(layer, K[layer], V[layer], pos)
            s.attend(layer, Q[layer], O=O[layer], q_pos=pos)
        assert s.end_step() == budget

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):            # the eager side first: nothing is lazily set up inside the capture
        outs = []
        fresh = [step_inputs(np.random.default_rng(50 + i), layers, Hq, Hkv, n, D, budget + i * n) for i in range(4)]
        for x in fresh:
            K, V, Q, pos = (y.clone() for y in x)
            O = torch.empty_like(Q)
            one(b, K, V, Q, pos, O)
            outs.append((O.clone(), *[y.clone() for y in (*b.cache, b.pos, b.weights)]))
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(a, *ins, Oa)
    for x, want in zip(fresh, outs):
        for to, y in zip(ins, x):
            to.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((Oa, *a.cache, a.pos, a.weights), want):
            assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))
        torch.randn((100, 100), device=DEV) @ torch.randn((100, 100), device=DEV)
        torch.cuda.synchronize()


def test_calls_on_two_streams_do_not_meet():
    """Attention with weights and eviction of two caches at once, each on a stream of its own."""
    def work(seed):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        cache = tuple(torch.randint(100, 130, (4, 30000, b), dtype=torch.uint8, device=DEV, generator=g) for b in (64, 4) * 2)
        Q = torch.empty((8, 3, 128), device=DEV, dtype=torch.bfloat16).normal_(generator=g)
        return cache, Q, torch.zeros((4, 30000), device=DEV)

    def run(state):
        cache, Q, w = state
        outs = []
        for k in range(6):
            outs.append(pk.pc_q4_attn(Q, cache, 30000 - 100 * k, 0.05, weights=w, decay=0.9))
            pk.pc_q4_evict(cache, None, w, 30000 - 100 * k, 29900 - 100 * k)
        return [*outs, *cache, w]

    want = [run(work(s)) for s in (1, 2)]
    torch.cuda.synchronize()
    states, got = [work(s) for s in (1, 2)], []
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    for st, stream in zip(states, streams):
        with torch.cuda.stream(stream):
            got.append(run(st))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))
