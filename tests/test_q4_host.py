"""The 4-bit cache and eviction on the CPU: the oracle against brute force, and what the entry points refuse.

The library checks its arguments before any device work, so refusals are asked for with made-up addresses here."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import paper_2601_04359_amd as pk
from oracle import q4_oracle as orc
from paper_2601_04359_amd import binding
from paper_2601_04359_amd.rollout import EvictingStack


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.lib_path()):
        from paper_2601_04359_amd.build import build_library
        build_library()
    return binding.lib()


# ------------------------------------------------------------------------------ the oracle
def test_oracle_codes_are_the_nearest():
    v = np.concatenate([np.arange(0, 8, 1 / 64), -np.arange(0, 8, 1 / 64)])
    x = np.zeros((len(v), 32))
    x[:, 0], x[:, 1] = 7.0, v              # the scale is 1
    x[np.abs(v) > 7, 1] = 0
    codes, scales = orc.q4_store(x)
    assert (scales == 127).all() and (codes[:, 0] & 15 == 7).all()
    got = codes[:, 0] >> 4
    for a, c in zip(x[:, 1], got):
        assert c & 7 == orc.q4_nearest(a) and (c >> 3 == int(np.signbit(a)))
        assert abs(abs(a) - orc.GRID[c & 7]) == np.min(np.abs(abs(a) - orc.GRID))


@pytest.mark.parametrize("top,e", [(7.0, 0), (7.0000001, 1), (3.5, -1), (3.6, 0), (6.0, 0), (1.75, -2), (0.0, -120), (1e-40, -120),
                                   (7 * 2.0 ** -120, -120), (8 * 2.0 ** -120, -119), (3.4e38, 125), (7 * 2.0 ** 124, 124)])
def test_oracle_scale(top, e):
    assert orc.q4_scale_exponent(top) == e
    x = np.zeros((1, 32))
    x[0, 5] = -top
    assert orc.q4_store(x)[1][0, 0] == e + 127


def test_oracle_round_trip_error():
    """An element is off by at most half a step of the group's scale: 1 (of a step of 2) times 2^e."""
    x = np.random.default_rng(0).standard_normal((40, 64)) * 10
    codes, scales = orc.q4_store(x)
    e = 2.0 ** (scales.astype(float) - 127)
    assert np.all(np.abs(orc.q4_load(codes, scales) - x).reshape(40, 2, 32) <= e[..., None])


@pytest.mark.parametrize("seed", range(8))
def test_oracle_eviction_keeps_the_right_set(seed):
    rng = np.random.default_rng(seed)
    Nk, n_keep = 60, int(rng.integers(1, 60))
    w, t = rng.integers(0, 6, Nk) * 1.0, rng.integers(0, 30, Nk)
    n_anchor, recent = int(rng.integers(0, min(5, n_keep) + 1)), int(rng.integers(0, 4))
    src = orc.evict_rows(w, t, Nk, n_keep, n_anchor, recent)
    assert len(set(src)) == n_keep
    safe = (np.arange(Nk) < n_anchor) | (t > t[-1] - recent) if recent else np.arange(Nk) < n_anchor
    best = sorted(range(Nk), key=lambda j: (not safe[j], 0 if safe[j] else -w[j], j))[:n_keep]
    assert set(src) == set(best)
    stay = src == np.arange(n_keep)
    assert all(stay[j] for j in best if j < n_keep) and np.all(np.diff(src[~stay]) > 0)


def test_attention_does_not_depend_on_the_order_of_the_rows():
    rng = np.random.default_rng(1)
    Q, K, V = rng.standard_normal((2, 3, 64)), rng.standard_normal((1, 50, 64)), rng.standard_normal((1, 50, 64))
    p = rng.permutation(50)
    a, b = orc.attn(Q, K, V, 0.125), orc.attn(Q, K[:, p], V[:, p], 0.125)
    assert np.allclose(a[0], b[0], atol=1e-13) and np.allclose(a[2][:, p], b[2], atol=1e-13)
    assert np.allclose(a[2].sum(), 2 * 3)


# ------------------------------------------------------------------------------ refusals of the library
A = 0x7f0000001000      # an address; nothing looks behind it


def cache(**kw):
    f = dict(k_codes=A, k_scales=A, v_codes=A, v_scales=A, code_stride_h=1 << 20, scale_stride_h=1 << 16)
    f.update(kw)
    return C.byref(binding._Q4(*f.values()))


def store(L, **kw):
    a = dict(K=A, V=A, dtype=1, H=4, n=8, D=128, ks=1 << 20, vs=1 << 20, cache=cache(), row0=0, pos_new=None, pos=None, ps=0,
             w=None, ws=0, Hsel=0, stream=None)
    a.update(kw)
    return L.pc_q4_store(*a.values())


def load(L, **kw):
    a = dict(cache=cache(), H=4, row0=0, n=8, D=128, dtype=1, K=A, V=A, ks=1 << 20, vs=1 << 20, stream=None)
    a.update(kw)
    return L.pc_q4_load(*a.values())


def attn(L, **kw):
    a = dict(Q=A + 4096, cache=cache(), dtype=1, Hq=8, Hkv=4, Nq=1, Nk=1000, D=128, qs=1 << 20, os=1 << 20, scale=0.1, O=A, lse=None,
             w=None, wst=0, Hsel=0, decay=1.0, ws=A, ws_bytes=1 << 40, stream=None)
    a.update(kw)
    return L.pc_q4_attn(*a.values())


def evict(L, **kw):
    a = dict(K=A, V=A, dtype=1, H=4, D=128, ks=1 << 24, vs=1 << 24, pos=A, ps=1 << 20, w=A, wst=1 << 20, Hsel=4, Nk=1000, n_keep=900,
             n_anchor=0, recent=0, idx=None, ist=0, ws=A, ws_bytes=1 << 40, stream=None)
    a.update(kw)
    return L.pc_evict(*a.values())


def q4_evict(L, **kw):
    a = dict(cache=cache(), H=4, D=128, pos=A, ps=1 << 20, w=A, wst=1 << 20, Hsel=4, Nk=1000, n_keep=900, n_anchor=0, recent=0,
             idx=None, ist=0, ws=A, ws_bytes=1 << 40, stream=None)
    a.update(kw)
    return L.pc_q4_evict(*a.values())


NULL, SHAPE, DTYPE, UNSUPPORTED, BUDGET, WORKSPACE = -1, -2, -3, -4, -5, -6
BAD_CACHES = [
    (dict(cache=None), NULL), (dict(cache=cache(k_codes=None)), NULL), (dict(cache=cache(v_scales=None)), NULL),
    (dict(cache=cache(k_codes=A + 8)), SHAPE), (dict(cache=cache(v_codes=A + 1)), SHAPE), (dict(cache=cache(k_scales=A + 2)), SHAPE),
    (dict(cache=cache(code_stride_h=(1 << 20) + 8)), SHAPE), (dict(cache=cache(scale_stride_h=(1 << 16) + 2)), SHAPE),
    (dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", BAD_CACHES + [
    (dict(dtype=2), DTYPE), (dict(H=0), SHAPE), (dict(n=-1), SHAPE), (dict(row0=-1), SHAPE), (dict(K=None), NULL), (dict(V=None), NULL),
    (dict(cache=cache(code_stride_h=7 * 64)), SHAPE), (dict(cache=cache(scale_stride_h=28)), SHAPE), (dict(row0=1 << 20), SHAPE),
    (dict(ks=8 * 128 - 8), SHAPE), (dict(ks=(1 << 20) + 4), SHAPE), (dict(K=A + 8), SHAPE), (dict(dtype=0, V=A + 2), SHAPE),
    (dict(pos=A, Hsel=4, ps=1 << 20), NULL), (dict(pos_new=A), NULL), (dict(pos=A, pos_new=A, Hsel=3, ps=1 << 20), SHAPE),
    (dict(w=A, Hsel=0), SHAPE), (dict(w=A, Hsel=4, ws=7), SHAPE), (dict(pos=A, pos_new=A, Hsel=4, ps=20), SHAPE),
    (dict(H=1, n=2 ** 30), SHAPE)])
def test_store_refuses(L, kw, status):
    assert store(L, **kw) == status and b"pc_q4_store" in L.pc_last_error_detail()


@pytest.mark.parametrize("kw,status", BAD_CACHES + [
    (dict(dtype=7), DTYPE), (dict(H=-1), SHAPE), (dict(n=-1), SHAPE), (dict(row0=-3), SHAPE), (dict(K=None, V=None), NULL),
    (dict(cache=cache(code_stride_h=7 * 64)), SHAPE), (dict(vs=8 * 128 - 8), SHAPE), (dict(V=A + 4), SHAPE), (dict(H=1, n=2 ** 30), SHAPE)])
def test_load_refuses(L, kw, status):
    assert load(L, **kw) == status and b"pc_q4_load" in L.pc_last_error_detail()


@pytest.mark.parametrize("kw,status", BAD_CACHES + [
    (dict(dtype=-1), DTYPE), (dict(Hq=6), SHAPE), (dict(Hkv=0), SHAPE), (dict(Hq=0), SHAPE), (dict(Nq=0), SHAPE), (dict(Nk=0), SHAPE),
    (dict(Nk=(1 << 30) + 1), SHAPE), (dict(Hq=2 ** 20, Hkv=2 ** 20, Nq=2 ** 20), SHAPE), (dict(scale=0.0), SHAPE),
    (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(Q=None), NULL), (dict(O=None), NULL),
    (dict(Nq=5, qs=4 * 128), SHAPE), (dict(Nq=5, os=4 * 128), SHAPE), (dict(qs=132), SHAPE), (dict(O=A + 4), SHAPE),
    (dict(Q=A), SHAPE), (dict(dtype=0, Q=A + 1), SHAPE), (dict(Nk=1 << 20), SHAPE), (dict(w=A, Hsel=2, wst=1000), SHAPE), (dict(w=A, Hsel=0), SHAPE),
    (dict(w=A, Hsel=4, wst=999), SHAPE), (dict(w=A, Hsel=1, decay=-0.5), BUDGET), (dict(w=A, Hsel=1, decay=float("nan")), BUDGET),
    (dict(w=A, Hsel=1, decay=float("inf")), BUDGET), (dict(w=A, Hsel=1, ws=None), WORKSPACE), (dict(w=A, Hsel=1, ws=A + 8), WORKSPACE),
    (dict(w=A, Hsel=1, ws_bytes=16), WORKSPACE), (dict(Nk=100000, cache=cache(code_stride_h=1 << 30, scale_stride_h=1 << 26), ws=None), WORKSPACE)])
def test_attn_refuses(L, kw, status):
    assert attn(L, **kw) == status and b"pc_q4_attn" in L.pc_last_error_detail()


BOOK = [(dict(H=0), SHAPE), (dict(Hsel=0), SHAPE), (dict(Hsel=3), SHAPE), (dict(Hsel=8), SHAPE), (dict(Nk=-1), SHAPE),
        (dict(n_keep=-1), BUDGET), (dict(n_anchor=-1), BUDGET), (dict(n_anchor=901), BUDGET), (dict(recent=-1), BUDGET),
        (dict(w=None), NULL), (dict(pos=None, recent=1), NULL), (dict(wst=999), SHAPE), (dict(ps=2999), SHAPE),
        (dict(idx=A, ist=899), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws=A + 4), WORKSPACE), (dict(ws_bytes=64), WORKSPACE),
        (dict(n_keep=1000, idx=A, ist=1000), BUDGET)]


@pytest.mark.parametrize("kw,status", BOOK + [
    (dict(dtype=3), DTYPE), (dict(D=12), UNSUPPORTED), (dict(D=2048), UNSUPPORTED), (dict(K=None), NULL), (dict(V=None), NULL),
    (dict(ks=999 * 128), SHAPE), (dict(K=A + 8), SHAPE), (dict(vs=(1 << 24) + 1), SHAPE), (dict(H=70000, Hsel=70000), SHAPE)])
def test_evict_refuses(L, kw, status):
    assert evict(L, **kw) == status and b"pc_evict" in L.pc_last_error_detail()


@pytest.mark.parametrize("kw,status", BOOK + BAD_CACHES + [(dict(cache=cache(code_stride_h=999 * 64 // 16 * 16)), SHAPE)])
def test_q4_evict_refuses(L, kw, status):
    assert q4_evict(L, **kw) == status and b"pc_q4_evict" in L.pc_last_error_detail()


def test_calls_that_do_nothing(L):
    assert store(L, n=0, K=None, V=None) == 0 and load(L, n=0) == 0
    assert evict(L, Nk=0) == 0 and evict(L, n_keep=1000, ws=None) == 0 and evict(L, n_keep=5000, ws=None) == 0
    assert q4_evict(L, n_keep=0, ws=None) == 0


HIP = -7


def test_one_head_has_no_stride_to_be_checked(L):
    """Each call gets past the strides: what is missing is the workspace, or a launch (there is no device to launch on)."""
    for st in (0, 128, 1001):
        assert attn(L, Hq=1, Hkv=1, Nq=5, qs=st, os=st, w=A, Hsel=1, ws=None) == WORKSPACE
        assert evict(L, H=1, Hsel=1, ks=st, vs=st, ws=None) == WORKSPACE
    if not torch.cuda.is_available():
        for st in (0, 128, 1001):
            assert store(L, H=1, ks=st, vs=st) == HIP and load(L, H=1, ks=st, vs=st) == HIP


def test_attn_refuses_an_output_that_overlaps_the_queries(L):
    """Against a comparison of every head with every head; interleaved heads do not overlap."""
    rng = np.random.default_rng(3)
    seen = [0, 0]
    for _ in range(3000):
        Hkv, rep, Nq, dtype = int(rng.integers(1, 4)), int(rng.integers(1, 4)), int(rng.integers(1, 4)), int(rng.integers(0, 2))
        elt, size = (4, 2)[dtype], Nq * 64
        qs, os_ = (size + int(rng.integers(0, 4)) * size // 2 // 8 * 8 for _ in range(2))
        if rng.random() < 0.5:
            os_ = qs
        gap = int(rng.integers(-Hkv * rep * 2 * size * elt // 16, Hkv * rep * 2 * size * elt // 16)) * 16
        if rng.random() < 0.5:
            gap = int(rng.integers(-4, 5)) * size * elt // 2
        q0, o0 = A, A + gap
        hits = any(q0 + i * qs * elt < o0 + j * os_ * elt + size * elt and o0 + j * os_ * elt < q0 + i * qs * elt + size * elt
                   for i in range(Hkv * rep) for j in range(Hkv * rep))
        status = attn(L, Q=q0, O=o0, dtype=dtype, D=64, Hq=Hkv * rep, Hkv=Hkv, Nq=Nq, qs=qs, os=os_, w=A, Hsel=1, ws=None)
        assert status == (SHAPE if hits else WORKSPACE), (Hkv * rep, Nq, dtype, qs, os_, gap)
        assert not hits or b"overlap" in L.pc_last_error_detail()
        seen[hits] += 1
    assert min(seen) > 300, seen


def test_calls_beyond_one_launch_are_refused(L):
    """A launch has fewer than 2^32 threads: refused just above, not by the runtime, and before anything is launched."""
    big = cache(code_stride_h=1 << 40, scale_stride_h=1 << 36)
    for D, n in ((128, 2 ** 27), (64, 2 ** 28)):            # n rows of K and of V, 8 elements per thread
        for H in (1, 4):
            kw = dict(D=D, H=H, n=n // H, cache=big)
            assert store(L, **kw, ks=1 << 40, vs=1 << 40) == SHAPE and b"pc_q4_store" in L.pc_last_error_detail()
            assert load(L, **kw, ks=1 << 40, vs=1 << 40) == SHAPE and b"pc_q4_load" in L.pc_last_error_detail()
    # 32 rows per work-group of 512 threads
    for dtype, Hkv in ((0, 1), (0, 4), (1, 2)):
        st = attn(L, D=64, dtype=dtype, Hq=Hkv, Hkv=Hkv, Nq=2 ** 28 // Hkv, qs=1 << 40, os=1 << 40, Q=A + (1 << 60), cache=big)
        assert st == SHAPE and b"pc_q4_attn" in L.pc_last_error_detail()


def test_a_cache_beyond_one_launch_is_not_expanded(L):
    """From 768 rows on a cache is expanded to bf16 rows (2 x 256 bytes for each), up to what one launch copies."""
    rows = lambda Hkv, Nk: pk.pc_q4_attn_workspace_bytes(pk.PC_BF16, 2 * Hkv, Hkv, 1000, Nk, 128) // (Hkv * Nk * 512)
    for Hkv in (1, 4):
        assert rows(Hkv, 2 ** 27 // Hkv - 16) == 1 and rows(Hkv, 2 ** 27 // Hkv) == 0 and rows(Hkv, 2 ** 27 // Hkv + 1) == 0


def test_workspaces(L):
    assert pk.pc_evict_workspace_bytes(4, 100, 100) == 0 and pk.pc_evict_workspace_bytes(4, 100, 0) == 0
    assert pk.pc_evict_workspace_bytes(0, 100, 50) == 0 and pk.pc_evict_workspace_bytes(4, 100, 99) > 0
    assert pk.pc_q4_attn_workspace_bytes(1, 8, 3, 1, 100, 128) == 0 and pk.pc_q4_attn_workspace_bytes(1, 8, 2, 1, 100, 96) == 0
    assert pk.pc_q4_attn_workspace_bytes(1, 8, 2, 1, 100000, 128) > 0
    assert pk.pc_q4_attn_workspace_bytes(1, 8, 2, 1, 10, 128, True) > pk.pc_q4_attn_workspace_bytes(1, 8, 2, 1, 10, 128, False)


# ------------------------------------------------------------------------------ refusals of the binding
def test_binding_refuses_what_does_not_fit(L):
    c = pk.q4_cache(2, 10, 128, device="cpu")
    x = torch.zeros((2, 3, 128), dtype=torch.bfloat16)
    w, pos = torch.zeros((2, 10)), torch.zeros((2, 10, 3), dtype=torch.int32)

    def refused(status, call, *args, **kw):
        with pytest.raises(pk.PackCacheError) as e:
            call(*args, **kw)
        assert e.value.status == status, e.value

    refused(-4, pk.q4_cache, 2, 10, 96, "cpu")
    # everything has to be on the current GPU
    refused(-2, pk.pc_q4_store, x, x, c, 0)
    refused(-2, pk.pc_q4_load, c, 0, x)
    refused(-2, pk.pc_q4_attn, x, c, 10, 0.1)
    refused(-2, pk.pc_q4_evict, c, pos, w, 10, 5)
    refused(-2, pk.pc_evict, x, x, None, w, 3, 2)
    # layouts
    for bad in (c[:3], 5, (c[0].int(), *c[1:]), (c[0][:, :, :32], *c[1:]), (c[0][:1], *c[1:]), (c[0], c[1][:, :5], *c[2:]),
                (c[0].transpose(0, 1), *c[1:]), (c[0], c[1], torch.zeros((4, 10, 64), dtype=torch.uint8)[::2], c[3])):
        refused(-2, pk.pc_q4_attn, x, bad, 10, 0.1)
    refused(-2, pk.pc_evict, x, x[:, :2], None, w, 3, 2)
    refused(-2, pk.pc_evict, x, x, None, w, 4, 2)
    refused(-1, pk.pc_evict, x, x, None, None, 3, 2)
    refused(-2, pk.pc_evict, x, x, pos[:1], w, 3, 2)
    refused(-2, pk.pc_evict, x, x, None, w.double(), 3, 2)


def test_stack_refuses():
    for kw in (dict(budget=0), dict(budget=5, n_anchor=6), dict(budget=5, step_rows=0), dict(budget=5, n_anchor=-1)):
        with pytest.raises(ValueError):
            EvictingStack(1, 2, 1, 128, scale=0.1, device="cpu", **kw)
    s = EvictingStack(2, 4, 2, 128, budget=8, scale=0.1, step_rows=2, device="cpu")
    with pytest.raises(ValueError):
        s.append(0, torch.zeros((2, 11, 128)), torch.zeros((2, 11, 128)), torch.zeros((11, 3), dtype=torch.int32))
    s.n_new = 1
    with pytest.raises(ValueError):
        s.append(1, torch.zeros((2, 2, 128)), torch.zeros((2, 2, 128)), torch.zeros((2, 3), dtype=torch.int32))


def test_a_cache_without_heads_is_refused():
    """Such a cache has no heads to share query heads among: refused before anything divides by their number."""
    empty = tuple(torch.zeros((0, 8, w), dtype=torch.uint8) for w in (64, 4, 64, 4))
    with pytest.raises(pk.PackCacheError, match="at least one head"):
        pk.pc_q4_attn(torch.zeros((2, 1, 128)), empty, 4, 0.1)
    with pytest.raises(pk.PackCacheError, match="at least one head"):
        pk.pc_q4_store(torch.zeros((0, 1, 128)), torch.zeros((0, 1, 128)), empty, 0)


def test_stack_refuses_layers_that_are_not_in_step(monkeypatch):
    """Every layer appends once per step: a second append, an attend in front of it and a step without one are errors, and a
    store that is refused leaves the step as it was."""
    from paper_2601_04359_amd import rollout
    calls = []

    def stored(*args, **kw):
        calls.append("store")
        if len(calls) == 1:
            raise pk.PackCacheError(-2, "refused")

    monkeypatch.setattr(rollout.pk, "pc_q4_store", stored)
    monkeypatch.setattr(rollout.pk, "pc_q4_attn", lambda *a, **kw: calls.append(("attn", a[2])))
    monkeypatch.setattr(rollout.pk, "pc_q4_evict", lambda *a, **kw: calls.append(("evict", a[3])) or a[4])
    s = EvictingStack(2, 4, 2, 128, budget=8, scale=0.1, step_rows=4, device="cpu")
    x, pos, q = torch.zeros((2, 3, 128)), torch.zeros((3, 3), dtype=torch.int32), torch.zeros((4, 3, 128))

    def append(layer):
        s.append(layer, x, x, pos, rotate=False)

    with pytest.raises(pk.PackCacheError):
        append(0)
    assert s.n_new == 0 and s.end_step() == 0
    for layer in (-1, 2):
        with pytest.raises(ValueError):
            append(layer)
        with pytest.raises(ValueError):
            s.attend(layer, q)
    with pytest.raises(ValueError):
        s.append(0, x[:, :0], x[:, :0], pos[:0], rotate=False)
    for step in (0, 1, 2):
        append(1)
        with pytest.raises(ValueError):
            append(1)
        with pytest.raises(ValueError):
            s.attend(0, q)
        with pytest.raises(ValueError):
            s.end_step()
        s.attend(1, q)
        assert calls[-1] == ("attn", min(3 * step + 3, 11))
        append(0)
        s.attend(0, q)
        s.attend(1, q, accumulate=False)
        assert s.end_step() == min(3 * step + 3, 8)
    assert calls[-1] == ("evict", 9) and s.nk == 8
    s.attend(0, q)                             # between steps: the cache as it stands
    assert calls[-1] == ("attn", 8)


@pytest.mark.parametrize("budget,n_anchor,rows_per_t", [(40, 0, 1), (41, 7, 1), (60, 4, 6), (13, 1, 6), (5, 4, 1), (9, 9, 1)])
def test_stack_keeps_the_newest_rows_by_default(budget, n_anchor, rows_per_t):
    """Attention that looks at all rows alike, over ten budgets' worth of single rows: the defaults keep the newest row at every
    step and let the window move with it.  (Without a window the newest row's sum is the least: nothing ever changes.)"""
    s = EvictingStack(1, 2, 1, 64, budget, 0.1, n_anchor=n_anchor, rows_per_t=rows_per_t, device="cpu")
    assert s.recent_t * rows_per_t <= budget - n_anchor and (s.recent_t > 0) == (budget - n_anchor >= rows_per_t)
    t, w = np.zeros(0, np.int64), np.zeros(0)
    for step in range(10 * budget):
        t, w = np.append(t, step // rows_per_t), np.append(w, 0.0)
        w = s.decay * w + 1.0 / len(w)
        src = orc.evict_rows(w, t, len(w), min(budget, len(w)), n_anchor, s.recent_t)
        t, w = t[src], w[src]
        if s.recent_t:
            assert step // rows_per_t in t
            assert (t == step // rows_per_t).sum() == step % rows_per_t + 1 or step < budget
    assert (np.sort(t)[::-1][:s.recent_t] >= (step - budget) // rows_per_t).all()


def test_stack_refuses_a_window_that_its_budget_cannot_hold():
    def stack(**kw):
        return EvictingStack(1, 2, 1, 64, scale=0.1, device="cpu", **kw)

    for kw in (dict(budget=10, recent_t=11), dict(budget=10, n_anchor=4, recent_t=7), dict(budget=10, recent_t=4, rows_per_t=3),
               dict(budget=10, recent_t=-1), dict(budget=10, rows_per_t=0), dict(budget=10, recent_t=2 ** 31 - 1)):
        with pytest.raises(ValueError):
            stack(**kw)
    assert stack(budget=10, n_anchor=4, recent_t=6).recent_t == 6 and stack(budget=10, recent_t=3, rows_per_t=3).recent_t == 3
    assert stack(budget=10, recent_t=0).recent_t == 0 and stack(budget=10, n_anchor=10).recent_t == 0
