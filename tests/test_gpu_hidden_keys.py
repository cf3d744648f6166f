"""Keys that a caller hides through dimensions of their own, by logits from -1e8 to -1e30: pc_frame_attn and pc_score.

Rows of three kinds, a third each: some keys visible; all hidden alike (every key weighs the same); all hidden and some twice
(the others share).  The rows without a visible key are zero in every other dimension: their logits are exact in any precision.

Tolerances, with u = 2^-24 and A the largest sum_d |q_d k_d| * scale over visible keys: a logit is off by (D + 8) u A, a probability
by a factor of 1 + e, e = (D + 16) u A + 8 u, and by half a step of bf16 before the second product; O once more by half a step.
"""
import numpy as np
import pytest
import torch

import paper_2601_04359_amd as pk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
D = 128
# a query's entry, a key's, the scale (the exponent of the largest key's probability is far from 0 unless the product is rounded)
HIDDEN_BY = [(1e8, -3.0, 128 ** -0.5), (1e12, -2.0, 0.125), (1e20, -2.0, 128 ** -0.5), (1e30, -1.0, 0.125), (1e30, -3.0, 0.1),
             (1e20, -2.0, pk.PC_SCALE_FOLDED)]     # the shorter loops


def hidden_inputs(hq, hkv, nq, nk, big, level, first_visible, D=D, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV)
    g.manual_seed(nq + nk)
    Q, K, V = (torch.empty((h, n, D), device=DEV).normal_(generator=g) for h, n in ((hq, nq), (hkv, nk), (hkv, nk)))
    j = torch.arange(nk, device=DEV)
    hidden = (j % 3 != 0) | (j < first_visible)
    Q[..., D - 32:], K[..., D - 32:] = 0.0, 0.0
    K[..., D - 1], K[..., D - 2] = hidden * level, level
    kind = (torch.arange(hq * nq, device=DEV) % 3).view(hq, nq)
    Q[kind > 0] = 0.0
    Q[..., D - 1], Q[..., D - 2] = (kind != 1) * big, (kind > 0) * big
    return [x.to(dtype) for x in (Q, K, V)] + [kind, hidden]


def reference(Q, K, V, scale, rows):
    """O, lse, probabilities (per query head) and sum_j p_j |v_j| of these rows, in 64 bits."""
    rep = Q.shape[0] // K.shape[0]
    out = []
    for h in range(Q.shape[0]):
        s = Q[h, rows].double() @ K[h // rep].double().t().contiguous() * scale
        lse = torch.logsumexp(s, 1)
        m = s.amax(1, keepdim=True)
        p = torch.exp(s - m)
        p = p / p.sum(1, keepdim=True)
        v = V[h // rep].double()
        out.append((p @ v, lse, p, p @ v.abs()))
    return [torch.stack(x) for x in zip(*out)]


# 32 rows per work-group whole and in shares, 64, 128 and 256, the last also in shares
SHAPES = [(8, 2, 252, 1804), (2, 1, 184, 5000), (16, 4, 666, 1786), (6, 2, 1593, 1701), (16, 4, 4032, 2048), (16, 4, 1008, 7455), (4, 2, 7, 33)]


@pytest.mark.parametrize("big,level,scale", HIDDEN_BY)
@pytest.mark.parametrize("first", [0, 0.4, 0.9])
@pytest.mark.parametrize("hq,hkv,nq,nk", SHAPES)
def test_frame_attn_hidden_keys_and_rows_without_any_other(hq, hkv, nq, nk, first, big, level, scale):
    Q, K, V, kind, hidden = hidden_inputs(hq, hkv, nq, nk, big, level, int(first * nk))
    lse = torch.empty((hq, nq), device=DEV)
    O = pk.pc_frame_attn(Q, K, V, nk, scale, lse=lse)
    rows = torch.arange(0, nq, max(1, nq // 40), device=DEV)
    Ow, Lw, _, spread = reference(Q, K, V, scale, rows)
    A = max(15.0, float(Q[..., :96].float().abs().sum(-1).max() * K[..., :96].float().abs().max() * scale))
    e = (D + 16) * U * A + 8 * U
    tol = (2 * e + (nk + 64) * U) * spread + 2.0 ** -8 * (Ow.abs() + spread)
    err = (O[:, rows].double() - Ow).abs()
    assert (err <= tol).all(), (err.max().item(), O.isnan().sum().item())
    assert ((lse[:, rows].double() - Lw).abs() <= (D + 16) * U * A + (5 * Lw.abs() + nk + 64) * U).all()


@pytest.mark.parametrize("big,level,scale", HIDDEN_BY)
@pytest.mark.parametrize("first", [0, 0.4, 0.9])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("hq,hkv,nq,nk", [(8, 2, 100, 1804), (2, 1, 64, 300), (16, 4, 512, 12000), (4, 2, 7, 33), (16, 4, 330, 7300)])
def test_score_hidden_keys_and_rows_without_any_other(hq, hkv, nq, nk, given, first, big, level, scale):
    """A row that sees nothing but hidden keys adds nothing to any score; the others add nothing to hidden keys."""
    Q, K, V, kind, hidden = hidden_inputs(hq, hkv, nq, nk, big, level, int(first * nk))
    rows = torch.arange(nq, device=DEV)
    _, Lw, p, _ = reference(Q, K, V, scale, rows)
    score = pk.pc_score(Q, K, nk, scale, lse=Lw.float() if given else None).double()
    sees = (kind == 0).double()[..., None]
    want = (p * sees).view(hkv, hq // hkv * nq, nk).sum(1)
    assert (score[:, hidden] == 0).all()
    A = max(15.0, float(Q[..., :96].float().abs().sum(-1).max() * K[..., :96].float().abs().max() * scale))
    # a log-sum-exp of its own or a given one in fp32, and its change of base: three roundings of at most A
    rel = 2 * ((D + 16) * U * A + 8 * U) + 3 * U * A + (hq // hkv * nq + 64) * U
    assert ((score - want).abs() <= rel * want + 1e-30).all(), (score - want).abs().max().item()


@pytest.mark.parametrize("big,level,scale", HIDDEN_BY)
@pytest.mark.parametrize("first", [0, 0.9])
@pytest.mark.parametrize("D,hq,hkv,nq,nk", [(64, 2, 1, 64, 336), (128, 8, 2, 100, 700), (64, 4, 2, 7, 33), (128, 4, 1, 300, 90)])
def test_f32_hidden_keys_and_rows_without_any_other(D, hq, hkv, nq, nk, first, big, level, scale):
    Q, K, V, kind, hidden = hidden_inputs(hq, hkv, nq, nk, big, level, int(first * nk), D, torch.float32)
    lse = torch.empty((hq, nq), device=DEV)
    O = pk.pc_frame_attn(Q, K, V, nk, scale, lse=lse)
    Ow, Lw, p, spread = reference(Q, K, V, scale, torch.arange(nq, device=DEV))
    A = max(15.0, float(Q[..., :D - 32].abs().sum(-1).max() * K[..., :D - 32].abs().max() * scale))
    e = (D + 16) * U * A + 8 * U
    err = (O.double() - Ow).abs()
    assert (err <= (2 * e + (nk + 64) * U) * spread + 1e-30).all(), (err.max().item(), O.isnan().sum().item())
    assert ((lse.double() - Lw).abs() <= (D + 16) * U * A + (5 * Lw.abs() + nk + 64) * U).all()
    want = (p * (kind == 0).double()[..., None]).view(hkv, hq // hkv * nq, nk).sum(1)
    rel = 2 * e + 3 * U * A + (hq // hkv * nq + 64) * U
    for given in (None, lse):
        score = pk.pc_score(Q, K, nk, scale, lse=given).double()
        assert (score[:, hidden] == 0).all() and ((score - want).abs() <= rel * want + 1e-30).all(), (score - want).abs().max().item()
