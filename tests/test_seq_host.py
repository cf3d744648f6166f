"""Prompts and pages on the CPU: what the entry points refuse, and calls that do nothing.

The library checks its arguments before any device work, so refusals are asked for with made-up addresses here."""
import ctypes as C
import os

import pytest
import torch

import paper_2601_04359_amd as pk
from paper_2601_04359_amd import binding
from paper_2601_04359_amd.rollout import PagedStack

NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4, -6
A = 1 << 40       # made-up addresses, far apart


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.lib_path()):
        from paper_2601_04359_amd.build import build_library
        build_library()
    return binding.lib()


def ints(v):
    return None if v is None else (C.c_int32 * len(v))(*v)


def prompt(L, **kw):
    a = dict(Q=A, K=2 * A, V=3 * A, dtype=pk.PC_BF16, Hq=8, Hkv=2, Tq=100, Tk=100, D=128, qs=12800, ks=12800, vs=12800, os=12800,
             scale=0.1, oq=[0, 40, 100], ok=None, n=2, O=4 * A, lse=None)
    a.update(kw)
    return L.pc_prompt_attn(a["Q"], a["K"], a["V"], a["dtype"], a["Hq"], a["Hkv"], a["Tq"], a["Tk"], a["D"], a["qs"], a["ks"], a["vs"],
                            a["os"], a["scale"], ints(a["oq"]), ints(a["ok"]), a["n"], a["O"], a["lse"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(Q=None), NULL), (dict(K=None), NULL), (dict(V=None), NULL), (dict(O=None), NULL), (dict(oq=None), NULL),
    (dict(dtype=2), DTYPE), (dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED), (dict(Hq=7), SHAPE), (dict(Hkv=0), SHAPE),
    (dict(scale=0.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(Tq=-1), SHAPE), (dict(n=-1), SHAPE),
    (dict(oq=[0, 40, 101]), SHAPE), (dict(oq=[-1, 40, 100]), SHAPE), (dict(oq=[0, 60, 50]), SHAPE), (dict(ok=[0, 40, 101]), SHAPE),
    (dict(ok=[0, 60, 50]), SHAPE), (dict(qs=12792), SHAPE), (dict(os=12792), SHAPE), (dict(ks=12792), SHAPE), (dict(vs=12792), SHAPE),
    (dict(qs=12801), SHAPE), (dict(Q=A + 8), SHAPE), (dict(O=4 * A + 2), SHAPE), (dict(K=2 * A + 4), SHAPE),
    (dict(O=A), SHAPE), (dict(O=A + 2 * 12800 * 7), SHAPE), (dict(O=2 * A - 16), SHAPE), (dict(O=3 * A + 256), SHAPE),
    (dict(Tq=2 ** 30, qs=2 ** 38, os=2 ** 38), UNSUPPORTED), (dict(Tk=2 ** 31 - 1, ks=2 ** 40, vs=2 ** 40), UNSUPPORTED)])
def test_prompt_refuses(L, kw, status):
    assert prompt(L, **kw) == status, L.pc_last_error_detail()


def test_calls_that_do_nothing(L):
    assert prompt(L, n=0) == 0 and prompt(L, oq=[5, 5, 5], ok=[0, 3, 9]) == 0
    assert store(L, T=0) == 0 and store(L, n=0) == 0
    assert attn(L, T=0) == 0 and attn(L, n=0) == 0


def pages(**kw):
    a = dict(K=5 * A, V=6 * A, stride_page=2 * 64 * 128, stride_h=64 * 128, n_pages=10, page_rows=64)
    a.update(kw)
    return binding._Pages(*a.values())


def store(L, pg=None, **kw):
    a = dict(K=A, V=2 * A, dtype=pk.PC_BF16, Hkv=2, T=4, D=128, ks=512, vs=512, table=7 * A, width=3, ts=3, lens=8 * A, offs=None, n=4,
             pos=9 * A, sec=(32, 48, 48), base=1e4, Ko=None, kos=512, Q=3 * A, Qo=4 * A, Hq=8, qs=512, qos=512, out=1.0)
    a.update(kw)
    p = C.byref(pages() if pg is None else pg) if pg is not False else None
    return L.pc_page_store(a["K"], a["V"], a["dtype"], a["Hkv"], a["T"], a["D"], a["ks"], a["vs"], p, a["table"], a["width"], a["ts"],
                           a["lens"], ints(a["offs"]), a["n"], a["pos"], *a["sec"], a["base"], a["Ko"], a["kos"], a["Q"], a["Qo"], a["Hq"],
                           a["qs"], a["qos"], a["out"], None)


def attn(L, pg=None, **kw):
    a = dict(Q=A, dtype=pk.PC_BF16, Hq=8, Hkv=2, T=4, D=128, qs=512, os=512, scale=0.1, table=7 * A, width=3, ts=3, lens=8 * A, offs=None,
             n=4, max_len=100, shared=None, n_shared=0, O=2 * A, lse=None, ws=3 * A, wb=1 << 30)
    a.update(kw)
    p = C.byref(pages() if pg is None else pg) if pg is not False else None
    return L.pc_page_attn(a["Q"], p, a["dtype"], a["Hq"], a["Hkv"], a["T"], a["D"], a["qs"], a["os"], a["scale"], a["table"], a["width"],
                          a["ts"], a["lens"], ints(a["offs"]), a["n"], a["max_len"], a["shared"], a["n_shared"], a["O"], a["lse"], a["ws"],
                          a["wb"], None)


BAD_PAGES = [(pages(K=None), NULL), (pages(V=None), NULL), (False, NULL), (pages(n_pages=0), SHAPE), (pages(page_rows=32), SHAPE),
             (pages(page_rows=100), SHAPE), (pages(page_rows=0), SHAPE), (pages(stride_h=64 * 128 - 8), SHAPE),
             (pages(stride_page=64 * 128 - 8), SHAPE), (pages(K=5 * A + 2), SHAPE), (pages(V=6 * A + 8), SHAPE),
             (pages(stride_h=64 * 128 + 1), SHAPE), (pages(stride_page=2 * 64 * 128 + 4), SHAPE)]
BAD_SEQUENCES = [(dict(table=None), NULL), (dict(lens=None), NULL), (dict(width=0), SHAPE), (dict(ts=2), SHAPE), (dict(T=5), SHAPE),
                 (dict(offs=[0, 1, 2, 3, 5]), SHAPE), (dict(offs=[0, 2, 1, 3, 4]), SHAPE), (dict(offs=[-1, 1, 2, 3, 4]), SHAPE),
                 (dict(T=-1), SHAPE), (dict(n=-1), SHAPE), (dict(dtype=3), DTYPE), (dict(D=32), UNSUPPORTED)]


@pytest.mark.parametrize("pg,status", BAD_PAGES)
def test_pages_are_checked(L, pg, status):
    assert store(L, pg) == status and attn(L, pg) == status


@pytest.mark.parametrize("kw,status", BAD_SEQUENCES)
def test_sequences_are_checked(L, kw, status):
    assert store(L, **kw) == status and attn(L, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(K=None), NULL), (dict(V=None), NULL), (dict(Q=None), NULL), (dict(Qo=None), NULL), (dict(pos=None), NULL), (dict(Hkv=0), SHAPE),
    (dict(sec=(32, 48, 46)), SHAPE), (dict(sec=(31, 49, 48)), SHAPE), (dict(sec=(-2, 82, 48)), SHAPE), (dict(base=0.0), SHAPE),
    (dict(out=0.0), SHAPE), (dict(out=float("inf")), SHAPE), (dict(ks=504), SHAPE), (dict(vs=504), SHAPE), (dict(qs=504), SHAPE),
    (dict(qos=504), SHAPE), (dict(Ko=10 * A, kos=504), SHAPE), (dict(Ko=10 * A + 8), SHAPE), (dict(K=A + 2), SHAPE), (dict(Q=3 * A + 4), SHAPE),
    (dict(Hq=0), SHAPE), (dict(width=2 ** 26, ts=2 ** 26), SHAPE)])
def test_store_refuses(L, kw, status):
    assert store(L, **kw) == status, L.pc_last_error_detail()


@pytest.mark.parametrize("kw,status", [
    (dict(Q=None), NULL), (dict(O=None), NULL), (dict(Hq=7), SHAPE), (dict(scale=-1.0), SHAPE), (dict(max_len=0), SHAPE), (dict(max_len=193), SHAPE),
    (dict(shared=10 * A), SHAPE), (dict(n_shared=5), SHAPE), (dict(shared=10 * A, n_shared=-5), SHAPE), (dict(O=A), SHAPE),
    (dict(O=A + 512 * 2 * 8 - 16), SHAPE), (dict(qs=504), SHAPE), (dict(os=504), SHAPE), (dict(Q=A + 8), SHAPE), (dict(O=2 * A + 8), SHAPE),
    (dict(max_len=192, shared=10 * A, n_shared=100, ws=None), WORKSPACE), (dict(max_len=192, shared=10 * A, n_shared=100, wb=64), WORKSPACE),
    (dict(max_len=192, shared=10 * A, n_shared=100, ws=3 * A + 8), WORKSPACE),
    (dict(T=2 ** 23, n=2 ** 23, qs=2 ** 30, os=2 ** 30), UNSUPPORTED)])
def test_attn_refuses(L, kw, status):
    assert attn(L, **kw) == status, L.pc_last_error_detail()


def test_workspaces(L):
    size = lambda **kw: pk.pc_page_attn_workspace_bytes(**{**dict(dtype=pk.PC_BF16, Hq=8, Hkv=2, T=4, D=128, n_seq=4, max_len=100), **kw})
    assert size(n_shared=50) >= 2 * 8 * 4 * (128 * 4 + 8)          # the common rows and the others: two shares at least
    assert size(Hq=7) == 0 and size(D=96) == 0 and size(T=5) == 0 and size(max_len=0) == 0 and size(dtype=2) == 0
    assert size(offs=[0, 1, 2, 3, 9], T=9, n_shared=50) > 0 and size(offs=[0, 2, 1, 3, 4]) == 0


# ------------------------------------------------------------------------------ the binding
@pytest.mark.parametrize("dtype", [pk.PC_BF16, pk.PC_F32])
@pytest.mark.parametrize("shared", [0, 70])
def test_sequences_that_are_all_empty_need_nothing(L, dtype, shared):
    for offs in ([0, 0, 0], [2, 2, 2]):
        assert L.pc_page_attn_workspace_bytes(dtype, 8, 2, 4, 128, ints(offs), 2, 100, shared) >= 0


def test_workspaces_of_what_is_refused_are_nothing(L):
    big = 2 ** 31 - 1
    for Hq, Hkv, T, max_len, shared in [(64, 64, big, 100, 0), (64, 64, 2 ** 30, 100, 50), (1, 1, 4, big, 0), (1, 1, 4, 100, big),
                                        (2 ** 20, 2 ** 20, 2 ** 20, 100, 0)]:
        assert L.pc_page_attn_workspace_bytes(pk.PC_BF16, Hq, Hkv, T, 128, None, 1, max_len, shared) == 0


@pytest.mark.parametrize("dtype", [pk.PC_BF16, pk.PC_F32])
def test_workspaces_of_the_largest_calls_are_counted(L, dtype):
    """Every size that a call may have gets a plan: no overflow on the way to it, and never fewer bytes than the partial rows take."""
    for Hq, Hkv, T, n_seq, max_len, shared in [(1, 1, 1, 1, 1 << 29, 0), (1, 1, 1, 1, 1 << 29, 1 << 29), (32, 1, 1 << 20, 1 << 20, 1 << 20, 0),
                                               (32, 32, 1 << 20, 1, 1 << 29, 1 << 28), (128, 8, 1 << 18, 4, 1 << 24, 1 << 23), (1, 1, 1, 1, 1, 0),
                                               (33, 11, 7, 7, 65, 64), (64, 64, 1 << 19, 1 << 19, 64, 63)]:
        for D in (64, 128):
            size = L.pc_page_attn_workspace_bytes(dtype, Hq, Hkv, T, D, None, n_seq, max_len, shared)
            launch = T // n_seq * min(n_seq, 256)
            assert size < 1 << 62 and (size == 0 or size >= launch * Hq * D * 4)


def test_binding_refuses_what_does_not_fit(L):
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)

    def refused(f, *a, **kw):
        with pytest.raises(pk.PackCacheError) as e:
            f(*a, **kw)
        return e.value.status
    Q, K = bf(8, 10, 128), bf(2, 10, 128)
    assert refused(pk.pc_prompt_attn, Q[0], K, K, 0.1, [0, 10]) == SHAPE
    assert refused(pk.pc_prompt_attn, Q, K, K[:, :9], 0.1, [0, 10]) == SHAPE
    assert refused(pk.pc_prompt_attn, Q, K.float(), K, 0.1, [0, 10]) == DTYPE
    assert refused(pk.pc_prompt_attn, Q, K, K, 0.1, []) == SHAPE
    assert refused(pk.pc_prompt_attn, Q, K, K, 0.1, [0, 10], [0, 5, 10]) == SHAPE
    assert refused(pk.pc_prompt_attn, Q, K, K, 0.1, [0, 2 ** 31]) == SHAPE
    assert refused(pk.pc_prompt_attn, Q, K, K, 0.1, [0, 10], O=Q[:, :9]) == SHAPE
    assert refused(pk.pc_prompt_attn, Q, K, K, 0.1, [0, 10], lse=torch.zeros(8, 9)) == SHAPE
    assert refused(pk.pc_prompt_attn, Q, K.transpose(0, 1).contiguous().transpose(0, 1), K, 0.1, [0, 10]) == SHAPE     # rows not dense
    assert refused(pk.pc_prompt_attn, Q, K, K, 0.1, [0, 10]) == SHAPE                                                  # not on the GPU
    pg = (bf(3, 2, 64, 128), bf(3, 2, 64, 128))
    for f in (lambda *a, **k: pk.pc_page_store(K, K, *a, **k), lambda p, t, n, **k: pk.pc_page_attn(Q, p, t, n, 64, 0.1, **k)):
        assert refused(f, pg[0][0], i32(10, 2), i32(10)) == SHAPE
        assert refused(f, (pg[0], pg[1][:2]), i32(10, 2), i32(10)) == SHAPE
        assert refused(f, (pg[0].float(), pg[1].float()), i32(10, 2), i32(10)) == SHAPE
        assert refused(f, pg, i32(10, 2), i32(10)) == SHAPE                  # not on the GPU
    with pytest.raises(pk.PackCacheError):
        pk.page_cache(3, 2, 100, 128, device="cpu")
    k, v = pk.page_cache(3, 2, 128, 64, dtype=torch.float32, device="cpu")
    assert k.shape == v.shape == (3, 2, 128, 64) and k.dtype == torch.float32
    with pytest.raises(pk.PackCacheError):
        binding._sequences(i32(4, 2).long(), i32(4), None, 4)


# ------------------------------------------------------------------------------ the stack's bookkeeping
def stack(**kw):
    return PagedStack(**{**dict(n_layers=2, Hq=4, Hkv=2, D=64, n_pages=8, scale=0.1, device="cpu"), **kw})


def test_stack_pages_follow_the_sequences():
    s = stack()
    a, b = s.open(), s.open()
    s.begin([a, b], [130, 64])
    assert s.free_pages() == 4 and s.rows(a) == 130 and s.n_shared == 0 and s.max_len == 130
    s.K[:, s._pages[a][2], :, :2] = 3.0
    c, d = s.fork(a, 2)
    assert s.free_pages() == 4 and s.rows(c) == 130
    s.begin([c, d], 1)                      # both leave a's last page for copies of it
    assert s.free_pages() == 2 and s.n_shared == 128
    assert len({s._pages[q][2] for q in (a, c, d)}) == 3 and s._pages[a][:2] == s._pages[c][:2] == s._pages[d][:2]
    assert (s.K[:, s._pages[c][2], :, :2] == 3.0).all() and (s.K[:, s._pages[d][2], :, :2] == 3.0).all()
    assert s.lens[:2].tolist() == [131, 131] and s.table[0, :3].tolist() == s._pages[c] and s.shared[:2].tolist() == s._pages[c][:2]
    s.close(a)
    assert s.free_pages() == 3
    s.begin([c, d], [0, 0])
    assert s.n_shared == 128
    s.begin([c], 1)
    assert s.n_shared == 0
    s.close(c), s.close(d), s.close(b)
    assert s.free_pages() == 8 and sorted(s._free) == list(range(8))


def test_the_last_user_of_a_page_keeps_it():
    s = stack(n_pages=3)
    a = s.open()
    s.begin([a], 70)
    b, = s.fork(a)
    s.begin([a, b], 1)                      # one copy is enough for the two
    assert s.free_pages() == 0 and s._pages[a][1] != s._pages[b][1]


def test_stack_of_sequences_refuses():
    for bad in (dict(n_layers=0), dict(Hq=3), dict(n_pages=0), dict(max_seqs=0)):
        with pytest.raises(ValueError):
            stack(**bad)
    for bad in (dict(D=96), dict(page_rows=48)):
        with pytest.raises(pk.PackCacheError):
            stack(**bad)
    s = stack(max_seqs=2, max_rows=256)
    a, b, c = s.open(), s.open(), s.open()
    s.begin([a, b], [100, 256])
    free = s.free_pages()
    for seqs, rows, kw in (([a, b, c], 1, {}), ([a, a], 1, {}), ([], 1, {}), ([a, b], [1], {}), ([a], [-1], {}), ([b], 1, {}), ([99], 1, {}),
                           ([a, c], [100, 256], {}), ([a], 1, dict(max_len=100)), ([a], 1, dict(max_len=257))):
        with pytest.raises(ValueError):
            s.begin(seqs, rows, **kw)
        assert s.free_pages() == free and [s.rows(q) for q in (a, b, c)] == [100, 256, 0]      # as it was
    s.begin([a], 1)
    Q, K = torch.zeros((4, 1, 64), dtype=torch.bfloat16), torch.zeros((2, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        s.attend(2, Q, K, K, None)
    with pytest.raises(ValueError):
        s.attend(0, torch.zeros((4, 2, 64)), K, K, None)
    s.close(c)
    with pytest.raises(ValueError):
        s.attend(0, Q, K, K, None)           # the step is over
    for f in (s.close, s.fork, s.rows):
        with pytest.raises(ValueError):
            f(c)


# ------------------------------------------------------------------------------ launches
@pytest.mark.parametrize("dtype,D", [(pk.PC_BF16, 128), (pk.PC_BF16, 64), (pk.PC_F32, 128), (pk.PC_F32, 64)])
def test_more_work_groups_than_a_launch_has_threads_for(L, dtype, D):
    """Threads of a launch fit 32 bits: calls with more are refused, and not left to fail behind the checks."""
    H = 2 ** 24
    kw = dict(dtype=dtype, D=D, Hq=H, Hkv=H)
    assert prompt(L, **kw, Tq=1, Tk=1, n=1, oq=[0, 1], qs=D, ks=D, vs=D, os=D) == UNSUPPORTED, L.pc_last_error_detail()
    assert prompt(L, **kw, Tq=60, Tk=60, n=60, oq=list(range(61)), qs=60 * D, ks=60 * D, vs=60 * D, os=60 * D) == UNSUPPORTED
    pg = pages(stride_h=64 * D, stride_page=64 * D * H, n_pages=1)
    assert attn(L, pg, **kw, T=1, n=1, max_len=64, width=1, ts=1, qs=D, os=D, wb=1 << 40) == UNSUPPORTED, L.pc_last_error_detail()


# ------------------------------------------------------------------------------ workspaces
@pytest.mark.parametrize("dtype", [pk.PC_BF16, pk.PC_F32])
@pytest.mark.parametrize("shared", [0, 70])
@pytest.mark.parametrize("offs", [[0, 0, 0], [2, 2, 2], [3] * 131])
def test_calls_without_rows_need_no_workspace(L, dtype, shared, offs):
    n = len(offs) - 1
    assert L.pc_page_attn_workspace_bytes(dtype, 8, 2, 4, 64, ints(offs), n, 100, shared) == 0
    kw = dict(dtype=dtype, offs=offs, n=n, shared=10 * A if shared else None, n_shared=shared, ws=None, wb=0, D=64, qs=256, os=256)
    assert attn(L, pages(stride_h=64 * 64, stride_page=2 * 64 * 64), **kw) == 0, L.pc_last_error_detail()


@pytest.mark.parametrize("dtype", [pk.PC_BF16, pk.PC_F32])
@pytest.mark.parametrize("Hq,Hkv,T,n_seq,max_len,shared,joined", [
    (8, 2, 4, 4, 100, 50, True),                # common rows and others
    (8, 2, 4, 4, 64, 64, False),                # nothing but common rows, few
    (8, 2, 4, 4, 64, 0, False), (8, 2, 1, 1, 1, 0, False),
    (8, 2, 1, 1, 1 << 20, 0, True),             # one row behind many
    (8, 2, 1, 1, 40000, 40000, True), (16, 4, 64, 64, 42000, 41800, True), (1, 1, 1, 1, 1 << 29, 1 << 28, True)])
def test_workspaces_hold_the_shares_that_are_joined(L, dtype, Hq, Hkv, T, n_seq, max_len, shared, joined):
    for D in (64, 128):
        size = L.pc_page_attn_workspace_bytes(dtype, Hq, Hkv, T, D, None, n_seq, max_len, shared)
        assert size >= 2 * Hq * T * (D + 2) * 4 if joined else size == 0      # two shares of every row at least


# ------------------------------------------------------------------------------ tensors that overlap
R = 512 * 2             # bytes of a head of the rows in store() and attn()
P = 64 * 128 * 2        # of a page of one head


@pytest.mark.parametrize("kw", [
    dict(Ko=A + 16), dict(Ko=A + R), dict(Ko=A, kos=1024), dict(Ko=A - R), dict(Ko=2 * A), dict(Ko=2 * A + R), dict(Ko=3 * A),
    dict(Ko=3 * A + 7 * R), dict(Ko=4 * A + 16), dict(Qo=3 * A + R), dict(Qo=3 * A, qos=520), dict(Qo=3 * A - 8 * R + 16), dict(Qo=A),
    dict(Qo=2 * A + R), dict(Qo=5 * A), dict(Qo=5 * A + 19 * P), dict(Qo=6 * A + 7 * P), dict(Ko=6 * A + 20 * P - 16), dict(Ko=5 * A - 2 * R + 16)])
def test_store_refuses_outputs_that_overlap(L, kw):
    assert store(L, **kw) == SHAPE, L.pc_last_error_detail()


def passes(status):
    """Without a GPU a call that passes its checks ends as an error of HIP."""
    return status not in (NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE)


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where nothing can be launched")
def test_what_does_not_overlap_is_not_refused(L):
    """In place; heads, pages and outputs in the gaps of each other."""
    for kw in (dict(), dict(Ko=A), dict(Qo=3 * A), dict(Ko=A, Qo=3 * A), dict(Ko=A + 2 * R), dict(Ko=A - 2 * R), dict(Qo=3 * A + 8 * R),
               dict(ks=1024, Ko=A + R, kos=1024), dict(qs=2048, qos=2048, Qo=3 * A + R, Ko=3 * A + 2 * R, kos=2048),
               dict(Ko=5 * A - 2 * R), dict(Ko=5 * A + 20 * P), dict(K=5 * A, V=6 * A + P)):
        assert passes(store(L, **kw)), (kw, L.pc_last_error_detail())
    wide = pages(stride_page=4 * 64 * 128, stride_h=2 * 64 * 128, V=5 * A + P)       # K and V of a head beside each other
    assert passes(store(L, wide))
    gaps = pages(stride_page=3 * 64 * 128)                                           # room for a head behind each page
    assert passes(store(L, gaps, Ko=5 * A + 2 * P, kos=3 * 64 * 128)) and store(L, gaps, Ko=5 * A + 2 * P, kos=64 * 128) == SHAPE
    for kw in (dict(), dict(lse=4 * A), dict(O=A + 8 * R), dict(O=A + R, qs=1024, os=1024), dict(O=5 * A - 8 * R), dict(lse=2 * A + 8 * R)):
        assert passes(attn(L, **kw)), (kw, L.pc_last_error_detail())
    assert passes(attn(L, gaps, O=5 * A + 2 * P, os=3 * 64 * 128)) and attn(L, gaps, O=5 * A + 2 * P, os=64 * 128) == SHAPE
    need = -(-pk.pc_page_attn_workspace_bytes(pk.PC_BF16, 8, 2, 4, 128, 4, 192, 100) // 16) * 16
    kw = dict(max_len=192, shared=10 * A, n_shared=100)
    for at in (A - need, A + 8 * R, 5 * A + 20 * P, 5 * A - need):
        assert passes(attn(L, ws=at, **kw)), (at, L.pc_last_error_detail())
    for kw in (dict(), dict(lse=5 * A), dict(lse=4 * A + 8 * 25600), dict(O=A + 25600, qs=25600, os=25600), dict(K=2 * A, V=2 * A)):
        assert passes(prompt(L, **kw)), (kw, L.pc_last_error_detail())


@pytest.mark.parametrize("kw", [
    dict(lse=A), dict(lse=A + 8 * R - 4), dict(lse=2 * A), dict(lse=2 * A + R - 4), dict(lse=5 * A + 19 * P), dict(lse=6 * A), dict(O=5 * A),
    dict(O=5 * A + 20 * P - 16), dict(O=6 * A + 3 * P), dict(O=5 * A - 8 * R + 16)])
def test_attn_refuses_outputs_that_overlap(L, kw):
    assert attn(L, **kw) == SHAPE, L.pc_last_error_detail()


@pytest.mark.parametrize("kw", [dict(ws=A), dict(ws=2 * A), dict(ws=A - 16), dict(ws=2 * A + 8 * R - 16), dict(ws=5 * A + 3 * P), dict(ws=6 * A + 20 * P - 16),
                                dict(lse=4 * A, ws=4 * A), dict(lse=4 * A, ws=4 * A + 112)])
def test_attn_refuses_a_workspace_that_overlaps(L, kw):
    assert attn(L, **kw, max_len=192, shared=10 * A, n_shared=100) == WORKSPACE, L.pc_last_error_detail()


@pytest.mark.parametrize("kw", [dict(lse=A), dict(lse=2 * A + 16), dict(lse=3 * A + 2 * 25600 - 4), dict(lse=4 * A + 8 * 25600 - 4), dict(lse=4 * A - 3196),
                                dict(O=2 * A, os=25600), dict(O=A + 12800, qs=25600, os=25600)])
def test_prompt_refuses_outputs_that_overlap(L, kw):
    assert prompt(L, **kw) == SHAPE, L.pc_last_error_detail()


# ------------------------------------------------------------------------------ every layer of a step, once
@pytest.fixture
def launches(monkeypatch):
    """The stack's calls, noted down instead of made; `recording`: whether they go into a graph."""
    from paper_2601_04359_amd import rollout
    done = type("Done", (), dict(calls=[], recording=False))()
    monkeypatch.setattr(rollout.pk, "pc_page_store", lambda *a, **kw: done.calls.append("store"))
    monkeypatch.setattr(rollout.pk, "pc_prompt_attn", lambda *a, **kw: done.calls.append("prompt"))
    monkeypatch.setattr(rollout.pk, "pc_page_attn", lambda *a, **kw: done.calls.append("pages"))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: done.recording)
    return done


def step(s, seqs, rows, layers):
    s.begin(seqs, rows)
    attend(s, sum([rows] * len(seqs) if isinstance(rows, int) else rows), layers)


def attend(s, T, layers):
    for layer in layers:
        s.attend(layer, torch.zeros((4, T, 64)), torch.zeros((2, T, 64)), torch.zeros((2, T, 64)), None)


def test_a_layer_that_misses_a_step_is_an_error(launches):
    s = stack(n_layers=3)
    a, b = s.open(), s.open()
    step(s, [a, b], [3, 5], (0, 2))
    with pytest.raises(ValueError, match="1"):
        s.begin([a, b], 1)
    assert [s.rows(q) for q in (a, b)] == [3, 5]
    attend(s, 8, (1,))
    step(s, [a], 1, (2, 0, 1))
    assert launches.calls == ["store", "prompt"] * 3 + ["store", "pages"] * 3


def test_a_layer_that_is_attended_to_twice_is_an_error(launches):
    s = stack()
    a = s.open()
    step(s, [a], 3, (0,))
    with pytest.raises(ValueError):
        attend(s, 3, (0,))
    assert launches.calls == ["store", "prompt"]
    attend(s, 3, (1,))
    step(s, [a], 0, (0, 0, 0))          # nothing new: nothing is stored
    step(s, [a], 1, (0, 1))


def test_a_store_that_fails_may_be_made_again(launches, monkeypatch):
    from paper_2601_04359_amd import rollout
    s = stack()
    a = s.open()
    s.begin([a], 3)
    with monkeypatch.context() as m:
        m.setattr(rollout.pk, "pc_page_store", lambda *a, **kw: (_ for _ in ()).throw(pk.PackCacheError(-2, "no")))
        with pytest.raises(pk.PackCacheError):
            attend(s, 3, (0,))
    attend(s, 3, (0, 1))
    s.begin([a], 1)


def test_sequences_of_a_step_that_close_ends_can_only_be_closed(launches):
    s = stack()
    a, b, c, d = (s.open() for _ in range(4))
    step(s, [a, b, c, d], [3, 70, 0, 4], (0, 1))
    s.close(d)                                     # every layer has its rows: nobody loses any
    step(s, [a, b, c], [1, 1, 0], (0,))
    e, = s.fork(a)
    s.close(b)                                     # layer 1 has not
    for q in (a, e):
        for f in (lambda: s.begin([q], 1), lambda: s.begin([c, q], 1), lambda: s.fork(q)):
            with pytest.raises(ValueError, match="only be closed"):
                f()
        assert s.rows(q) == 4
    step(s, [c], 2, (0, 1))                        # had no new rows
    s.close(a), s.close(e), s.close(c)
    assert s.free_pages() == 8
    step(s, [s.open()], 3, (0, 1))


def test_steps_that_a_graph_replays(launches):
    """attend() is called once, while it is recorded, and not again."""
    s = stack()
    a = s.open()
    step(s, [a], 3, (0, 1))
    step(s, [a], 1, (0, 1))
    launches.recording = True
    attend(s, 1, (0, 1))                           # behind a first call of the same step
    launches.recording = False
    for _ in range(3):
        s.begin([a], 1)
    b, = s.fork(a)
    step(s, [a, b], 1, (0,))                       # a layer by itself, the other one in the graph
    s.begin([a], 1)
    s.close(b)
    s.begin([a], 1)


def test_a_further_pass_over_a_step_says_so(launches):
    s = stack()
    a = s.open()
    step(s, [a], 3, (0, 1))
    for _ in range(2):
        for layer in range(2):
            s.attend(layer, torch.zeros((4, 3, 64)), torch.zeros((2, 3, 64)), torch.zeros((2, 3, 64)), None, again=True)
    assert launches.calls == ["store", "prompt"] * 6 and s.rows(a) == 3
    s.begin([a], 1)


@pytest.mark.skipif(torch.cuda.is_available(), reason="tensors that are not on the GPU, and no GPU")
def test_attend_without_a_gpu_is_refused():
    s = stack()
    s.begin([s.open()], 3)
    bf = lambda *n: torch.zeros(n, dtype=torch.bfloat16)
    with pytest.raises(pk.PackCacheError):
        s.attend(0, bf(4, 3, 64), bf(2, 3, 64), bf(2, 3, 64), torch.zeros((3, 3), dtype=torch.int32))
