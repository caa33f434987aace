"""The training operators (include/colbandit_train.h) against their formulas in 64 bits.

Tolerances are bounds on the rounding that the kernels do, worked out from the terms of each sum in the 64-bit
reference: a value rounded to the storage type is off by at most U of itself (2^-8 for bf16: eight significant bits,
to nearest; nothing for fp32, where it stays as it is), and 32-bit arithmetic by at most F = 2e-5 of the sum of the
absolute terms (scores below 32 in size carry an error of some 2^-23 * 32 * 3 into the exponential's argument, and sums
of a few thousand terms less than that)."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F = 2e-5
U = {"bf16": 2.0 ** -8, "f32": 0.0}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    from paper_2602_02827_amd import build, training
    build.build_library()
    training.lib()
    return training


@pytest.fixture(scope="module")
def dev(tr):
    assert torch.cuda.is_available(), "these tests need the GPU"
    return torch.device("cuda")


def offsets(lengths):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64))


# ---- the reference ---------------------------------------------------------------------------------------

def bucket(dist, n_buckets, max_distance, causal):
    """Bucket of a distance key - query in exact integer arithmetic: range i of a direction's wide ones begins at the
    first integer x with x^(n-s) >= s^(n-s-i) * max_distance^i (s single distances, n buckets)."""
    n = n_buckets if causal else n_buckets // 2
    base = n if not causal and dist > 0 else 0
    far = max(0, -dist) if causal else abs(dist)
    s = n // 2
    if far < s:
        return base + far
    return base + s + sum(far ** (n - s) >= s ** (n - s - i) * max_distance ** i for i in range(1, n - s))


class Attention:
    """Outputs, gradients and the bounds of both, in 64 bits on the CPU."""

    def __init__(self, q, k, v, ql, kl, dtype, causal=False, scale=None, keep=None, bias=None, max_distance=128, dout=None):
        u = U[dtype]
        q, k, v = (x.detach().double().cpu() for x in (q, k, v))
        H, Hk, d = q.shape[1], k.shape[1], q.shape[2]
        scale = 1.0 / math.sqrt(d) if scale is None else scale
        dout = None if dout is None else dout.detach().double().cpu()
        table = None if bias is None else bias.detach().double().cpu()
        zero = torch.zeros_like
        self.out, self.out_tol = zero(q), zero(q)
        self.lse = torch.full((H, q.shape[0]), -math.inf, dtype=torch.float64)
        self.dq, self.dq_tol, self.dk, self.dk_tol, self.dv, self.dv_tol = (zero(x) for x in (q, q, k, k, k, k))
        if table is not None:
            self.dbias, self.dbias_tol = zero(table), zero(table)
        qo, ko = offsets(ql).tolist(), offsets(kl).tolist()
        for s, (lq, lk) in enumerate(zip(ql, kl)):
            if lq == 0 or lk == 0:
                continue
            a, x = slice(qo[s], qo[s + 1]), slice(ko[s], ko[s + 1])
            dist = torch.arange(lk) - (torch.arange(lq)[:, None] + lk - lq)
            seen = torch.ones(lq, lk, dtype=torch.bool)
            if causal:
                seen &= dist <= 0
            if keep is not None:
                seen &= keep[x].cpu().bool()
            if table is not None:
                of = torch.tensor([bucket(t, table.shape[0], max_distance, causal) for t in range(-lk - lq, lk + lq + 1)])
                b = of[dist + lk + lq]
            for h in range(H):
                g = h // (H // Hk)
                visible = seen.any(0)[:, None]
                K, V = torch.where(visible, k[x, g], 0.0), torch.where(visible, v[x, g], 0.0)
                Q = torch.where(seen.any(1)[:, None], q[a, h], 0.0)
                S = Q @ K.T * scale
                if table is not None:
                    S = S + table[b, h]
                S[~seen] = -math.inf
                lse = torch.logsumexp(S, 1)
                P = torch.exp(S - torch.where(lse == -math.inf, 0.0, lse)[:, None])
                O = P @ V
                spread = P @ V.abs()
                self.out[a, h], self.lse[h, a] = O, lse
                self.out_tol[a, h] = u * (spread + O.abs()) + F * spread
                if dout is None:
                    continue
                G = torch.where(seen.any(1)[:, None], dout[a, h], 0.0)
                dP = G @ V.T
                delta = (G * O).sum(1, keepdim=True)
                E = P * (dP - delta)
                # delta comes from the rounded output; P and E are rounded as operands; the rest in 32 bits
                d_delta = (G.abs() * ((u + F) * spread + u * O.abs())).sum(1, keepdim=True)
                rough = P * (G.abs() @ V.abs().T + (G.abs() * spread).sum(1, keepdim=True))
                e_tol = P * d_delta + F * rough
                self.dq[a, h] = E @ K * scale
                self.dq_tol[a, h] = abs(scale) * ((u * E.abs() + e_tol) @ K.abs()) + u * (E @ K * scale).abs()
                self.dk[x, g] += E.T @ Q * scale
                self.dk_tol[x, g] += abs(scale) * ((u * E.abs() + e_tol).T @ Q.abs())
                self.dv[x, g] += P.T @ G
                self.dv_tol[x, g] += (u + F) * (P.T @ G.abs())
                if table is not None:
                    self.dbias[:, h].index_add_(0, b.reshape(-1), E.reshape(-1))
                    self.dbias_tol[:, h].index_add_(0, b.reshape(-1), e_tol.reshape(-1))
        self.dk_tol += u * self.dk.abs()
        self.dv_tol += u * self.dv.abs()
        if table is not None:
            self.dbias_tol += u * self.dbias.abs()


def within(got, want, tol, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape and bool(torch.isfinite(got).all()), what
    worst = (got - want).abs() - 1.05 * tol
    i = int(worst.argmax()) if worst.numel() else 0
    assert worst.numel() == 0 or float(worst.max()) <= 1e-9, (what, i, got.reshape(-1)[i], want.reshape(-1)[i], tol.reshape(-1)[i])


def problem(dev, dtype, ql, kl, H, Hk, d, seed=0, bias=None, keep=False, size=1.0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    p = dict(q=n(sum(ql), H, d) * size, k=n(sum(kl), Hk, d), v=n(sum(kl), Hk, d), dout=n(sum(ql), H, d) * 0.1)
    p = {x: t.to(DT[dtype]).to(dev) for x, t in p.items()}
    p["bias"] = None if bias is None else n(bias, H).to(DT[dtype]).to(dev)
    p["keep"] = None
    if keep:
        m = torch.rand(sum(kl), generator=g) >= 0.25
        ko = offsets(kl)
        m[ko[0]:ko[1]] = False                       # a sequence whose rows see nothing
        p["keep"] = m.to(dev)
    return p


def attend(tr, p, ql, kl, causal=False, scale=None, max_distance=128):
    qo, ko = offsets(ql).to(p["q"].device), offsets(kl).to(p["q"].device)
    how = dict(causal=causal, scale=scale, keep=p["keep"], bias=p["bias"], max_distance=max_distance)
    f = tr.colbandit_attention(p["q"], p["k"], p["v"], qo, ko, **how)
    b = tr.colbandit_attention_backward(p["dout"], p["q"], p["k"], p["v"], f["out"], f["lse"], qo, ko, **how)
    torch.cuda.synchronize()
    return f, b


def check_attention(tr, p, ql, kl, dtype, causal=False, scale=None, max_distance=128):
    f, b = attend(tr, p, ql, kl, causal, scale, max_distance)
    r = Attention(p["q"], p["k"], p["v"], ql, kl, dtype, causal, scale, p["keep"], p["bias"], max_distance, p["dout"])
    lse = f["lse"].double().cpu()
    assert torch.equal(lse == -math.inf, r.lse == -math.inf)
    fine = r.lse > -math.inf
    assert float((lse - r.lse)[fine].abs().max() if fine.any() else 0.0) <= F * 2
    within(f["out"], r.out, r.out_tol, "out")
    assert bool((f["out"].double().cpu()[~fine.T] == 0).all())
    within(b["dq"], r.dq, r.dq_tol, "dq")
    within(b["dk"], r.dk, r.dk_tol, "dk")
    within(b["dv"], r.dv, r.dv_tol, "dv")
    if p["bias"] is not None:
        within(b["dbias"], r.dbias, r.dbias_tol, "dbias")
    return f, b


EDGES = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]


# ---- attention -------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("causal,bias,keep", [(False, None, False), (True, 32, True), (False, 32, True), (True, None, False)])
def test_attention_at_the_edges_of_tiles(tr, dev, dtype, d, causal, bias, keep):
    p = problem(dev, dtype, EDGES, EDGES, 2, 2, d, bias=bias, keep=keep)
    check_attention(tr, p, EDGES, EDGES, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads", [(6, 3), (8, 1), (7, 1), (20, 1), (3, 1)])
@pytest.mark.parametrize("causal,bias,keep", [(True, None, True), (False, 8, False)])
def test_heads_that_share_keys(tr, dev, dtype, heads, kv_heads, causal, bias, keep):
    ql = [5, 0, 70, 33, 1]
    p = problem(dev, dtype, ql, ql, heads, kv_heads, 64, seed=1, bias=bias, keep=keep)
    check_attention(tr, p, ql, ql, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bias", [None, 32])
def test_queries_and_keys_of_different_lengths(tr, dev, dtype, causal, bias):
    """More queries than keys leave rows without keys under a causal limit; either side may be empty."""
    ql, kl = [1, 40, 7, 0, 130, 1, 33, 3], [300, 9, 0, 12, 64, 1, 257, 3]
    p = problem(dev, dtype, ql, kl, 4, 4, 64, seed=2, bias=bias)
    check_attention(tr, p, ql, kl, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_short_and_single_token_sequences(tr, dev, dtype):
    for lengths in ([1], [1, 1, 1], [5], [32] * 3, [0, 0, 4], list(range(1, 33)) * 3):
        p = problem(dev, dtype, lengths, lengths, 3, 3, 32, seed=3, bias=16)
        check_attention(tr, p, lengths, lengths, dtype)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences_are_found(tr, dev, dtype):
    """More sequences than one step of the search takes, and more than two."""
    g = np.random.default_rng(4)
    lengths = g.integers(0, 9, 5000).tolist()
    p = problem(dev, dtype, lengths, lengths, 1, 1, 32, seed=4)
    check_attention(tr, p, lengths, lengths, dtype)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,heads,kv_heads,bias,keep", [(128, 8, 2, None, False), (64, 4, 4, 32, True), (32, 20, 1, None, True)])
@pytest.mark.parametrize("causal", [True, False])
def test_single_tokens_over_long_keys(tr, dev, dtype, d, heads, kv_heads, bias, keep, causal):
    """Their keys are split and the parts joined; one sequence is short, so that most of its parts are empty."""
    ql, kl = [1, 1, 1, 3], [5000, 1, 37, 2051]
    p = problem(dev, dtype, ql, kl, heads, kv_heads, d, seed=5, bias=bias, keep=keep)
    check_attention(tr, p, ql, kl, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_sequences(tr, dev, dtype):
    lengths = [1030, 411]
    p = problem(dev, dtype, lengths, lengths, 2, 1, 64, seed=6, keep=True)
    check_attention(tr, p, lengths, lengths, dtype, True)
    p = problem(dev, dtype, lengths, lengths, 2, 2, 64, seed=6, bias=32)
    check_attention(tr, p, lengths, lengths, dtype)


@gpu
@pytest.mark.parametrize("n_buckets,max_distance,causal", [(4, 2, False), (8, 256, False), (128, 256, False), (2, 7, True), (3, 9, True),
                                                          (32, 128, True), (31, 200, True), (128, 65, True)])
def test_bias_tables_of_many_shapes(tr, dev, n_buckets, max_distance, causal):
    lengths = [300, 1, 150]
    p = problem(dev, "f32", lengths, lengths, 2, 2, 32, seed=7, bias=n_buckets)
    check_attention(tr, p, lengths, lengths, "f32", causal, max_distance=max_distance)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_of_a_packed_projection_and_of_heads_first(tr, dev, dtype):
    """q, k and v as views: of one [rows][(H + 2 Hk) d] tensor, and of [heads][rows][d] ones, NaN all around."""
    ql, H, Hk, d = [70, 3, 129], 4, 2, 64
    p = problem(dev, dtype, ql, ql, H, Hk, d, seed=8)
    n = sum(ql)
    want, want_grads = attend(tr, p, ql, ql)
    joint = torch.full((n, (H + 2 * Hk) * d + 16), math.nan, dtype=DT[dtype], device=dev)
    views = dict(p, q=joint[:, :H * d].view(n, H, d), k=joint[:, H * d:(H + Hk) * d].view(n, Hk, d),
                 v=joint[:, (H + Hk) * d:(H + 2 * Hk) * d].view(n, Hk, d))
    first = {x: torch.full((p[x].shape[1], n + 2, d + 8), math.nan, dtype=DT[dtype], device=dev) for x in "qkv"}
    heads_first = dict(p, **{x: first[x][:, 1:n + 1, :d].transpose(0, 1) for x in "qkv"})
    for other in (views, heads_first):
        for x in "qkv":
            other[x].copy_(p[x])
        f, b = attend(tr, other, ql, ql)
        for x in ("out", "lse"):
            assert torch.equal(f[x], want[x])
        for x in ("dq", "dk", "dv"):
            assert torch.equal(b[x], want_grads[x])


@gpu
@pytest.mark.parametrize("ql", [list(range(1, 18)), [128, 97, 65], [1, 2, 3, 40]])
@pytest.mark.parametrize("d,H,Hk", [(64, 3, 3), (128, 4, 2)])
@pytest.mark.parametrize("bias", [None, 32])
def test_short_rows_lose_nothing_but_the_results_rounding(tr, dev, ql, d, H, Hk, bias):
    """Rows that see up to 128 keys: delta in 32 bits and dS in two values of eight bits, 2^-17 of it, which over 128 keys is some
    2^-13.5 of the sum.  A stored value is the exact one's nearest, or off by no more than that and twice the error before it is
    rounded: the norm of the error is that of the exact gradients' own rounding and at most 2^-12 of their norm."""
    p = problem(dev, "bf16", ql, ql, H, Hk, d, seed=19, bias=bias)
    want = Attention(p["q"], p["k"], p["v"], ql, ql, "bf16", causal=True, bias=p["bias"], dout=p["dout"])
    _, b = attend(tr, p, ql, ql, causal=True)
    for name in ("dq",) if bias is None else ("dq", "dbias"):
        exact = getattr(want, name)
        error, own = float((b[name].double().cpu() - exact).norm()), float((exact.bfloat16().double() - exact).norm())
        assert error <= own + 2.0 ** -12 * float(exact.norm()), (name, error, own)


@gpu
@pytest.mark.parametrize("heads", [4, 2])
def test_rows_and_heads_beyond_32_bits(tr, dev, heads):
    """Rows 16 MiB apart and heads 3 GiB apart (packed heads' rows are addressed from their tile's first one in 32 bits: these are
    too far apart for that), so that offsets pass 2^32 bytes."""
    ql, H, Hk, d = [140, 60], heads, 2, 64
    n = sum(ql)
    p = problem(dev, "bf16", ql, ql, H, Hk, d, seed=16)
    want, want_grads = attend(tr, p, ql, ql, causal=True)
    room = torch.empty(H * (n << 23), dtype=torch.bfloat16, device=dev)
    for order in ("rows", "heads"):
        row, head = (1 << 23, d) if order == "rows" else (H * d, n << 23)
        for x in "qkv":
            far = dict(p)
            far[x] = torch.as_strided(room, p[x].shape, (row, head, 1))
            far[x].copy_(p[x])
            f, b = attend(tr, far, ql, ql, causal=True)
            for name in ("out", "lse"):
                assert torch.equal(f[name], want[name]), (order, x, name)
            if order == "rows" or x != "q" or H == Hk:          # (else other tiles, which add in another order)
                for name in ("dq", "dk", "dv"):
                    assert torch.equal(b[name], want_grads[name]), (order, x, name)


@gpu
@pytest.mark.parametrize("wild", [[0, 1 << 40, 90], [-7, 50, 1 << 40], [80, 20, 60], [0, 0, 0]])
def test_offsets_that_are_none_stay_in_bounds(tr, dev, wild):
    """The kernels clamp them to the tensors; results mean nothing, neighbours in memory stay as they are."""
    ql = [40, 50]
    p = problem(dev, "bf16", ql, ql, 2, 2, 32, seed=17, bias=8, keep=True)
    off, how = torch.tensor(wild, device=dev), dict(keep=p["keep"], bias=p["bias"])
    guard = torch.full((3, 90, 2, 32), 7.0, dtype=torch.bfloat16, device=dev)
    lse = torch.zeros(2, 90, device=dev)
    tr.colbandit_attention(p["q"], p["k"], p["v"], off, out={"out": guard[1], "lse": lse}, **how)
    b = tr.colbandit_attention_backward(p["dout"], p["q"], p["k"], p["v"], guard[1], lse, off, **how)
    Q, D, _ = embeddings(dev, "f32", 3, 7, [90], 32)
    f = tr.colbandit_maxsim_scores(Q, D, off)
    g = tr.colbandit_maxsim_backward(f["scores"].nan_to_num(), f["argmax"], Q, D, off)
    torch.cuda.synchronize()
    assert bool((guard[0] == 7).all()) and bool((guard[2] == 7).all()) and b["dq"].shape == p["q"].shape and g["dQ"].shape == Q.shape


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-20, 5.0])
def test_scales_of_any_sign_and_size(tr, dev, dtype, scale):
    """The products' sign is the columns', a scale of zero leaves only the bias; 5 makes rows that are nearly one key (scores up to
    80, whose 32-bit rounding is 2.5 times that of the bound's 32)."""
    ql = [70, 33]
    p = problem(dev, dtype, ql, ql, 2, 2, 32, seed=18, bias=8, size=0.4 if scale == 5.0 else 1.0)
    check_attention(tr, p, ql, ql, dtype, scale=scale)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("wild", [math.nan, math.inf, -math.inf, "lowest"])
def test_masked_keys_may_hold_anything(tr, dev, dtype, wild):
    wild = torch.finfo(DT[dtype]).min if wild == "lowest" else wild
    ql, kl = [40, 1, 100, 20], [9, 700, 100, 0]
    p = problem(dev, dtype, ql, kl, 2, 1, 64, seed=9, keep=True)
    f, b = check_attention(tr, p, ql, kl, dtype)
    q = dict(p, k=p["k"].clone(), v=p["v"].clone(), dout=p["dout"].clone(), q=p["q"].clone())
    for x in "kv":
        q[x][~p["keep"]] = wild
    q["dout"][:40] = wild                            # and so may rows that see nothing
    q["q"][:40] = wild
    q["dout"][141:] = wild
    f2, b2 = attend(tr, q, ql, kl)
    for x, y in ((f, f2), (b, b2)):
        for name in x:
            assert x[name] is None or torch.equal(x[name], y[name]), name


@gpu
def test_a_bias_of_the_lowest_value_hides_a_distance(tr, dev):
    """Rows that have other keys: the hidden ones get no weight; a row with nothing else shares it out."""
    lengths, low = [50, 1], torch.finfo(torch.float32).min
    p = problem(dev, "f32", lengths, lengths, 2, 2, 32, seed=10, bias=8)
    p["bias"][0] = low                               # distance 0
    f, b = attend(tr, p, lengths, lengths)
    r = Attention(p["q"], p["k"], p["v"], lengths, lengths, "f32", bias=p["bias"], dout=p["dout"])
    within(f["out"], r.out, r.out_tol, "out")
    for x in ("dq", "dk", "dv"):
        within(b[x][:50], getattr(r, x)[:50], getattr(r, x + "_tol")[:50], x)


def check_far(tr, p, ql, kl, dtype, causal=False, scale=None, like=None, by=1.0, lse_of=lambda x: x):
    """All results of rows whose log-sum-exp may be of any size: it has a 32-bit value's own rounding, and as much again for the
    product that it is the sum of.  The reference's probabilities are exp(S - lse), which in 64 bits lose a sum's logarithm too
    where lse is that large: it is then given a problem of the same probabilities (`like`: other inputs, q divided by `by`, a power
    of two, which is what the keys' gradient differs by), and `lse_of` its log-sum-exp."""
    f, b = attend(tr, p, ql, kl, causal, scale)
    a = dict(p, **(like or {}))
    r = Attention(a["q"], a["k"], a["v"], ql, kl, dtype, causal, scale, a["keep"], a["bias"], 128, a["dout"])
    r.dk, r.dk_tol, r.lse = r.dk * by, r.dk_tol * by, torch.where(r.lse == -math.inf, r.lse, lse_of(r.lse))
    lse = f["lse"].double().cpu()
    assert torch.equal(lse == -math.inf, r.lse == -math.inf)
    fine = r.lse > -math.inf
    assert bool(((lse - r.lse).abs() <= F * 2 + 2.0 ** -22 * r.lse.abs())[fine].all())
    within(f["out"], r.out, r.out_tol, "out")
    for x in ("dq", "dk", "dv") + (() if p["bias"] is None else ("dbias",)):
        within(b[x], getattr(r, x), getattr(r, x + "_tol"), x)


def extreme(value, dtype):
    return {"lowest": torch.finfo(DT[dtype]).min, "highest": torch.finfo(DT[dtype]).max}.get(value, value)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("low", [-1e4, -1e7, -1e9, -1e30, -1e38, "lowest"])
def test_rows_that_see_nothing_but_a_hidden_distance(tr, dev, dtype, d, causal, low):
    """A bucket of the table hides distance 0.  Rows that see other keys give it no weight; those that see only this one (the first
    of a causal sequence, sequences of one token) have all of it there, and all gradients."""
    lengths = [50, 1, 133, 1]
    p = problem(dev, dtype, lengths, lengths, 2, 2, d, seed=20, bias=8)
    p["bias"][0] = extreme(low, dtype)
    check_far(tr, p, lengths, lengths, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl", [([150, 1, 70], [150, 1, 70]), ([1, 3], [5000, 700])])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("value", ["lowest", -1e30, 1e30, "highest"])
def test_a_table_that_is_far_from_zero_everywhere(tr, dev, dtype, ql, kl, causal, value):
    """Products are below such a bias' rounding in 64 bits as well: all keys that are seen weigh the same, in one part or several."""
    p = problem(dev, dtype, ql, kl, 2, 2, 64, seed=21, bias=32, keep=True)
    p["bias"][:] = extreme(value, dtype)
    at, tiny = float(p["bias"][0, 0].double()), 2.0 ** -40
    check_far(tr, p, ql, kl, dtype, causal, like=dict(q=p["q"].double() * tiny, bias=torch.zeros_like(p["bias"])), by=1 / tiny,
              lse_of=lambda x: x + at)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_biases_beyond_the_powers_of_two_keep_their_order(tr, dev, dtype):
    """Values whose product with log2(e) is beyond 32 bits: a row that sees two of them has its weight at the higher one."""
    lengths = [2, 1, 2]
    p = problem(dev, dtype, lengths, lengths, 2, 2, 32, seed=22, bias=8)
    p["bias"][:] = extreme("lowest", dtype)
    p["bias"][1] = -2.5e38                           # the key before
    check_far(tr, p, lengths, lengths, dtype, True)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [None, 32])
@pytest.mark.parametrize("exponent", [10, 20, 30, 60])
@pytest.mark.parametrize("ql,kl", [([150, 1, 70], [150, 1, 70]), ([1, 3], [5000, 700])])
def test_scores_of_any_size(tr, dev, dtype, bias, exponent, ql, kl):
    """Whole numbers times a power of two: products are exact in 32 bits, and a row has one key, or equal ones that share it."""
    p = problem(dev, dtype, ql, kl, 4, 2, 64, seed=23, bias=bias)
    g = torch.Generator().manual_seed(24)
    for x, by in (("q", 2.0 ** exponent), ("k", 1.0)):
        p[x] = (torch.randint(-8, 9, p[x].shape, generator=g) * by).to(DT[dtype]).to(dev)
    if bias:
        p["bias"].zero_()
    by = 2.0 ** (exponent - 10)                      # (at 2^10 scores are multiples of 128: the next one has nothing)
    check_far(tr, p, ql, kl, dtype, like=dict(q=p["q"].double() / by), by=by, lse_of=lambda x: (x / 128).round() * 128 * by + (x - (x / 128).round() * 128))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [None, 32])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_of_any_size_that_are_rounded(tr, dev, dtype, bias, d):
    """Scores of some 2^30, whose rounding in 32 bits is 2^7: a row has one key, the gradients' kernels have to find the very scores
    of the forward pass.  Rows whose first two scores are closer than 2^-16 of their size take no part."""
    lengths = [150, 1, 70]
    p = problem(dev, dtype, lengths, lengths, 4, 2, d, seed=26, bias=bias, size=2.0 ** 30)
    S = torch.einsum("qhd,khd->hqk", p["q"].double().cpu(), p["k"].double().cpu().repeat_interleave(2, 1))
    own = torch.block_diag(*[torch.ones(n, n) for n in lengths]).bool()
    top = S.masked_fill(~own, -math.inf).topk(2, -1).values
    p["dout"][((top[..., 0] - top[..., 1]) < 2.0 ** -16 * top[..., 0].abs()).T.to(dev)] = 0
    f, b = attend(tr, p, lengths, lengths)
    r = Attention(p["q"], p["k"], p["v"], lengths, lengths, dtype, bias=p["bias"], dout=p["dout"])
    for x in ("dq", "dk", "dv") + (() if bias is None else ("dbias",)):
        within(b[x], getattr(r, x), getattr(r, x + "_tol"), x)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [None, 8])
def test_a_scale_near_zero(tr, dev, dtype, bias):
    """A log-sum-exp divided by it is beyond 32 bits."""
    lengths = [200, 33]
    p = problem(dev, dtype, lengths, lengths, 2, 1, 64, seed=25, bias=bias)
    check_far(tr, p, lengths, lengths, dtype, scale=1.2e-38)


@gpu
@pytest.mark.parametrize("size", [30.0, 1e-3])
def test_sharp_and_flat_rows(tr, dev, size):
    """Scores of some hundreds, where a row has one key, and rows whose keys all weigh the same."""
    lengths = [150, 20]
    p = problem(dev, "bf16", lengths, lengths, 2, 2, 64, seed=11, size=size)
    f, _ = attend(tr, p, lengths, lengths)
    r = Attention(p["q"], p["k"], p["v"], lengths, lengths, "bf16")
    within(f["out"], r.out, r.out_tol + 4e-4 * r.out.abs().max() * (size > 1), "out")


@gpu
@pytest.mark.parametrize("causal,bias", [(False, 32), (True, None)])
def test_attention_gradients_against_differences(tr, dev, causal, bias):
    """Central differences along a direction, step 1/64: the third-order term is some 1e-4 of the slope, the outputs'
    rounding (2^-23 of sums of size 100, over the step) less."""
    lengths = [60, 7]
    p = problem(dev, "f32", lengths, lengths, 2, 2, 32, seed=12, bias=bias)
    off = offsets(lengths).to(dev)
    how = dict(causal=causal, keep=None, max_distance=40)
    w = p["dout"].double()

    def value(**x):
        a = dict(p, **x)
        return float((tr.colbandit_attention(a["q"], a["k"], a["v"], off, bias=a["bias"], **how)["out"].double() * w).sum())

    leaves = {x: p[x].clone().requires_grad_(True) for x in ("q", "k", "v", "bias") if p[x] is not None}
    out = tr.attention(leaves["q"], leaves["k"], leaves["v"], off, causal=causal, bias=leaves.get("bias"), max_distance=40)
    out.backward(p["dout"])
    g = torch.Generator().manual_seed(13)
    for x, leaf in leaves.items():
        way = torch.randn(leaf.shape, generator=g).to(dev)
        h = 1.0 / 64
        slope = (value(**{x: p[x] + h * way}) - value(**{x: p[x] - h * way})) / (2 * h)
        size = float(leaf.grad.double().norm())
        got = float((leaf.grad.double() * way.double()).sum())
        assert abs(got - slope) <= 4e-3 * size, (x, got, slope, size)


@gpu
def test_the_same_inputs_give_the_same_bits_on_any_stream_and_in_graphs(tr, dev):
    ql = [180, 32, 77, 1030]
    p = problem(dev, "bf16", ql, ql, 4, 4, 64, seed=14, bias=32, keep=True)
    want = attend(tr, p, ql, ql)

    def same(f, b):
        for x, y in zip(want, (f, b)):
            for name in x:
                assert torch.equal(x[name], y[name]), name

    same(*attend(tr, p, ql, ql))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = attend(tr, p, ql, ql)
    s.synchronize()
    same(*got)
    off = offsets(ql).to(dev)
    how = dict(keep=p["keep"], bias=p["bias"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = tr.colbandit_attention(p["q"], p["k"], p["v"], off, **how)
        b = tr.colbandit_attention_backward(p["dout"], p["q"], p["k"], p["v"], f["out"], f["lse"], off, **how)
    for _ in range(3):
        for t in (f["out"], f["lse"], b["dq"], b["dk"], b["dv"], b["dbias"]):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        same(f, b)


@gpu
def test_given_outputs_and_workspaces(tr, dev):
    ql, kl = [1, 1], [3000, 10]
    p = problem(dev, "bf16", ql, kl, 2, 1, 64, seed=15)
    qo, ko = offsets(ql).to(dev), offsets(kl).to(dev)
    want = tr.colbandit_attention(p["q"], p["k"], p["v"], qo, ko)
    out = {x: torch.zeros_like(want[x]) for x in ("out", "lse")}
    ws = torch.empty(64 << 20, dtype=torch.uint8, device=dev)
    got = tr.colbandit_attention(p["q"], p["k"], p["v"], qo, ko, out=out, workspace=ws)
    assert got["out"] is out["out"] and all(torch.equal(got[x], want[x]) for x in want)
    with pytest.raises(tr.ColbanditError, match="workspace"):
        tr.colbandit_attention(p["q"], p["k"], p["v"], qo, ko, workspace=ws[:256])


# ---- MaxSim loss -----------------------------------------------------------------------------------------

def embeddings(dev, dtype, nq, T, lengths, d, seed=0, step=64):
    """Values on a coarse grid: products and sums are exact in 32 bits, and equal maxima are common."""
    g = torch.Generator().manual_seed(seed)
    grid = lambda *s: torch.randint(-3, 4, s, generator=g).float() / step  # noqa: E731
    return grid(nq, T, d).to(DT[dtype]).to(dev), grid(sum(lengths), d).to(DT[dtype]).to(dev), offsets(lengths).to(dev)


def maxsim_reference(Q, D, off):
    Q, D, off = Q.double().cpu().numpy(), D.double().cpu().numpy(), off.cpu().numpy()
    nq, T, d = Q.shape
    scores, arg = np.full((nq, len(off) - 1), -np.inf), np.full((nq, len(off) - 1, T), -1, dtype=np.int32)
    for i in range(len(off) - 1):
        if off[i + 1] > off[i]:
            c = Q.reshape(-1, d) @ D[off[i]:off[i + 1]].T
            arg[:, i] = c.argmax(1).reshape(nq, T)
            scores[:, i] = c.max(1).reshape(nq, T).sum(1)
    return scores, arg


def gradient_reference(g, arg, Q, D, off):
    """Gradients and the sums of their absolute terms."""
    g, Q, D, off = g.double().cpu(), Q.double().cpu(), D.double().cpu(), off.cpu().tolist()
    nq, T, d = Q.shape
    r = [torch.zeros_like(Q), torch.zeros_like(Q), torch.zeros_like(D), torch.zeros_like(D)]
    for i in range(len(off) - 1):
        if off[i + 1] == off[i]:
            continue
        rows = torch.from_numpy(arg[:, i].astype(np.int64)) + off[i]
        w = g[:, i, None, None]
        r[0] += w * D[rows]
        r[1] += (w * D[rows]).abs()
        r[2].index_add_(0, rows.reshape(-1), (w * Q).reshape(-1, d))
        r[3].index_add_(0, rows.reshape(-1), (w * Q).abs().reshape(-1, d))
    return r


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("nq,T,lengths", [(1, 1, [1]), (3, 21, EDGES), (5, 128, [70, 0, 3, 300]), (9, 24, [0, 1030, 65]),
                                          (40, 32, [5, 180, 64, 1, 33])])
def test_maxsim_scores_choices_and_gradients(tr, dev, dtype, d, nq, T, lengths):
    Q, D, off = embeddings(dev, dtype, nq, T, lengths, d, seed=d + nq)
    f = tr.colbandit_maxsim_scores(Q, D, off)
    scores, arg = maxsim_reference(Q, D, off)
    np.testing.assert_array_equal(f["argmax"].cpu().numpy(), arg)
    np.testing.assert_array_equal(f["scores"].double().cpu().numpy(), scores)
    g = torch.randn(nq, len(lengths), generator=torch.Generator().manual_seed(1)).to(dev)
    b = tr.colbandit_maxsim_backward(g, f["argmax"], Q, D, off)
    dQ, dQ_abs, dD, dD_abs = gradient_reference(g, arg, Q, D, off)
    within(b["dQ"], dQ, U[dtype] * dQ.abs() + F * dQ_abs, "dQ")
    within(b["ddocs"], dD, U[dtype] * dD.abs() + F * dD_abs, "ddocs")
    again = tr.colbandit_maxsim_backward(g, f["argmax"], Q, D, off)
    assert torch.equal(again["dQ"], b["dQ"]) and torch.equal(again["ddocs"], b["ddocs"])


@gpu
@pytest.mark.parametrize("same", ["tokens", "documents"])
def test_every_query_token_chooses_one_document_token(tr, dev, same):
    """The whole list of entries (more than are sorted at once) falls on one row; equal tokens: the first."""
    nq, T, lengths, d = 150, 32, [100, 3], 64
    Q, D, off = embeddings(dev, "bf16", nq, T, lengths, d, seed=3)
    if same == "documents":
        D[:] = D[0]
    else:
        Q[:] = Q[0, 0]
    f = tr.colbandit_maxsim_scores(Q, D, off)
    scores, arg = maxsim_reference(Q, D, off)
    np.testing.assert_array_equal(f["argmax"].cpu().numpy(), arg)
    g = torch.rand(nq, 2, generator=torch.Generator().manual_seed(2)).to(dev)
    b = tr.colbandit_maxsim_backward(g, f["argmax"], Q, D, off)
    dQ, dQ_abs, dD, dD_abs = gradient_reference(g, arg, Q, D, off)
    within(b["dQ"], dQ, U["bf16"] * dQ.abs() + F * dQ_abs, "dQ")
    within(b["ddocs"], dD, U["bf16"] * dD.abs() + F * dD_abs, "ddocs")


@gpu
def test_many_documents_and_choices_out_of_range(tr, dev):
    """Thousands of documents of 0 to 8 tokens; choices that name no row of the corpus add nothing."""
    lengths = np.random.default_rng(5).integers(0, 9, 6000).tolist()
    Q, D, off = embeddings(dev, "f32", 3, 5, lengths, 32, seed=5)
    f = tr.colbandit_maxsim_scores(Q, D, off)
    scores, arg = maxsim_reference(Q, D, off)
    np.testing.assert_array_equal(f["argmax"].cpu().numpy(), arg)
    np.testing.assert_array_equal(f["scores"].double().cpu().numpy(), scores)
    g = torch.randn(3, 6000, generator=torch.Generator().manual_seed(3)).to(dev)
    wild = torch.full_like(f["argmax"], 1 << 30)
    b = tr.colbandit_maxsim_backward(g, wild, Q, D, off)
    assert not b["dQ"].any() and not b["ddocs"].any()


@gpu
@pytest.mark.parametrize("N", [1, 2, 255, 256, 257, 5000])
@pytest.mark.parametrize("temperature", [0.02, 1.0, 30.0])
def test_contrastive_loss(tr, dev, N, temperature):
    """Differences of scores of size 10 have an error of 2^-22, which the temperature divides."""
    nq = 7
    g = torch.Generator().manual_seed(N)
    x = (torch.randn(nq, N, generator=g) * 3 + 10).to(dev)
    if N > 2:
        x[0, 1] = x[3, 0] = -math.inf
    t = torch.randint(0, N, (nq,), generator=g).to(dev)
    t[2], t[5] = -1, N
    if N > 2:
        t[0] = 0
        t[3] = 2
    r = tr.colbandit_contrastive_loss(x, t, temperature)
    z = x.double().cpu() / temperature
    tc = t.cpu()
    off_by = 4e-6 + 3e-6 / temperature
    for q in range(nq):
        loss, grad = float(r["loss"][q]), r["dscores"][q].double().cpu()
        if q in (2, 5):
            assert loss == 0 and not grad.any()
            continue
        want = torch.logsumexp(z[q], 0) - z[q, tc[q]]
        assert abs(loss - float(want)) <= off_by * 3 + 1e-6 * abs(float(want))
        p = torch.softmax(z[q], 0)
        p[tc[q]] -= 1.0
        assert float((grad * temperature * 5 - p).abs().max()) <= off_by


@gpu
def test_contrastive_loss_as_part_of_a_program(tr, dev):
    """Gradients of the mean loss against central differences along a direction, embeddings that are not on a grid (step 2^-8:
    choices that change within it are few, and their documents' scores are continuous)."""
    g = torch.Generator().manual_seed(6)
    lengths = [20, 35, 64, 7, 90]
    unit = lambda *s: torch.nn.functional.normalize(torch.randn(*s, generator=g), dim=-1).to(dev)  # noqa: E731
    Q, D, off = unit(4, 16, 64), unit(sum(lengths), 64), offsets(lengths).to(dev)
    t = torch.tensor([0, 2, -1, 4], device=dev)

    def value(Q, D):
        return float(tr.contrastive_maxsim(Q, D, off, t, 0.5).double())

    q, d = Q.clone().requires_grad_(True), D.clone().requires_grad_(True)
    (tr.contrastive_maxsim(q, d, off, t, 0.5) * 3.0).backward()
    for x, leaf in (("q", q), ("d", d)):
        way = torch.nn.functional.normalize(torch.randn(leaf.shape, generator=g), dim=-1).to(dev)
        h = 2.0 ** -8
        a, b = (Q + h * way, D) if x == "q" else (Q, D + h * way), (Q - h * way, D) if x == "q" else (Q, D - h * way)
        slope = 3.0 * (value(*a) - value(*b)) / (2 * h)
        got = float((leaf.grad.double() * way.double()).sum())
        assert abs(got - slope) <= 0.02 * float(leaf.grad.double().norm()) + 2e-3, (x, got, slope)


# ---- clipping --------------------------------------------------------------------------------------------

def clip_reference(grads, max_norm):
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    return norm, min(1.0, max_norm / (norm + 1e-6))


def check_clip(tr, grads, max_norm, in_place=False):
    before = [g.clone() for g in grads]
    norm, by = clip_reference(grads, max_norm)
    r = tr.colbandit_clip_gradients(grads, max_norm, out=None if in_place else [torch.full_like(g, 7.0) for g in grads])
    torch.cuda.synchronize()
    got = float(r["norm"])
    assert abs(got - norm) <= 2.0 ** -22 * norm if norm < 3.4028235e38 else got == math.inf   # it is written in 32 bits
    for x, y, g in zip(before, r["grads"], grads):
        assert (y is g) == in_place
        u = 2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -23
        assert bool(((y.double() - x.double() * by).abs() <= (u + 2.0 ** -21) * x.double().abs() * by + 1e-40).all())
    return r


@gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("max_norm", [0.5, 1e9, math.inf])
def test_clipping_many_tensors(tr, dev, in_place, max_norm):
    """Both types, sizes around the vectors' and chunks' ends, none at all, more tensors than one launch takes, and views that are
    aligned to nothing but their type."""
    g = torch.Generator().manual_seed(7)
    sizes = [0, 1, 7, 8, 9, 31, 129, 8191, 8192, 8193, 70001] * 25
    whole = [torch.randn(n + 3, generator=g).to(DT["bf16" if i % 3 else "f32"]).to(dev) for i, n in enumerate(sizes)]
    grads = [w[i % 3:i % 3 + n] for i, (w, n) in enumerate(zip(whole, sizes))]
    check_clip(tr, grads, max_norm, in_place)


@gpu
def test_clipping_leaves_what_is_small_enough(tr, dev):
    x = torch.randn(1000, generator=torch.Generator().manual_seed(8)).to(dev)
    y = x.clone()
    assert float(tr.clip_gradients_([torch.nn.Parameter(torch.zeros(3, device=dev))] + [_with_grad(y)], 1e6)) > 0
    assert torch.equal(x, y)
    z = torch.zeros(5, device=dev)
    r = tr.colbandit_clip_gradients([z], 1.0)
    assert float(r["norm"]) == 0 and not z.any()


def _with_grad(g):
    p = torch.nn.Parameter(torch.zeros_like(g))
    p.grad = g
    return p


@gpu
def test_clipping_extremes(tr, dev):
    """Squares beyond 32 bits, numbers below its normal range, and norms that are no numbers."""
    big = [torch.full((1000,), 1e30, device=dev), torch.full((10,), -3e38, device=dev)]
    check_clip(tr, big, 1.0)
    tiny = torch.full((100,), 1e-30, device=dev)
    assert abs(float(tr.colbandit_clip_gradients([tiny], 1.0)["norm"]) / 1e-29 - 1) < 1e-5
    r = tr.colbandit_clip_gradients([torch.tensor([1.0, math.inf], device=dev)], 1.0)
    assert float(r["norm"]) == math.inf and float(r["grads"][0][0]) == 0 and math.isnan(float(r["grads"][0][1]))
    r = tr.colbandit_clip_gradients([torch.tensor([1.0, math.nan], device=dev)], 1.0)
    assert math.isnan(float(r["norm"])) and bool(torch.isnan(r["grads"][0]).all())


@gpu
def test_loss_and_clipping_in_graphs(tr, dev):
    Q, D, off = embeddings(dev, "bf16", 6, 24, [40, 5, 130], 128, seed=9)
    t = torch.tensor([0, 1, 2, 0, 1, 2], device=dev)

    def step():
        f = tr.colbandit_maxsim_scores(Q, D, off)
        l = tr.colbandit_contrastive_loss(f["scores"], t, 0.3)
        b = tr.colbandit_maxsim_backward(l["dscores"], f["argmax"], Q, D, off)
        c = tr.colbandit_clip_gradients([b["dQ"], b["ddocs"]], 1e-2, out=[torch.empty_like(b["dQ"]), torch.empty_like(b["ddocs"])])
        return [f["scores"], l["loss"], b["dQ"], b["ddocs"], c["norm"], *c["grads"]]

    want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for x in got:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


# ---- together --------------------------------------------------------------------------------------------

@gpu
def test_fine_tuning_an_encoder(tr, dev):
    """The operators as a program uses them: the loss falls to less than half, more queries find their document, and the same
    seed gives the same losses."""
    from paper_2602_02827_amd import finetune
    r = finetune.train(steps=40, n_docs=128)
    assert all(math.isfinite(x) for x in r["losses"] + r["norms"])
    assert sum(r["losses"][-5:]) < 0.5 * sum(r["losses"][:5]), r["losses"]
    assert r["after"] > r["before"]
    assert finetune.train(steps=3, n_docs=128)["losses"] == r["losses"][:3]


# ---- boundary --------------------------------------------------------------------------------------------

def test_library_exports_every_declared_training_symbol(tr):
    hdr = open(os.path.join(ROOT, "include", "colbandit_train.h")).read()
    hdr = re.sub(r"/\*.*?\*/", "", hdr, flags=re.S)
    declared = set(re.findall(r"\b(colbandit_[a-z_0-9]+)\s*\(", hdr))
    assert declared == set(tr.EXPORTS)
    L = ctypes.CDLL(tr.binding.LIB_PATH)
    assert all(getattr(L, name) is not None for name in declared)
    assert tr.lib().colbandit_sizeof_attn() == ctypes.sizeof(tr.ColbanditAttn)


def test_training_header_is_plain_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "colbandit_train.h"\nint main(void) { colbandit_attn a; return (int)(sizeof a != colbandit_sizeof_attn()); }\n')
    for cc, std in (("gcc", "-std=c99"), ("g++", "-std=c++11")):
        r = subprocess.run([cc, std, "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only", "-x", "c" if cc == "gcc" else "c++",
                            "-I", os.path.join(ROOT, "include"), str(src)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr


def test_bias_buckets_are_those_of_exact_arithmetic(tr):
    for n_buckets, max_distance, causal in [(32, 128, 0), (32, 128, 1), (4, 2, 0), (2, 2, 1), (3, 9, 1), (128, 256, 0), (64, 100, 0),
                                            (31, 200, 1), (128, 65, 1), (10, 243, 0)]:
        starts = tr.colbandit_bias_buckets(n_buckets, max_distance, causal)
        for dist in range(-300, 1):
            got = int(np.searchsorted(starts, -dist, side="right")) - 1
            assert got == bucket(dist, n_buckets, max_distance, bool(causal)), (n_buckets, max_distance, causal, dist)
    L = tr.lib()
    s = (ctypes.c_int32 * 128)()
    assert L.colbandit_bias_buckets(32, 128, 0, None) == -1
    assert L.colbandit_bias_buckets(31, 128, 0, s) == -2 and L.colbandit_bias_buckets(0, 128, 1, s) == -2
    assert L.colbandit_bias_buckets(2, 128, 0, s) == -2 and L.colbandit_bias_buckets(32, 8, 0, s) == -2
    assert L.colbandit_bias_buckets(130, 128, 0, s) == -4 and L.colbandit_bias_buckets(32, 257, 0, s) == -4


def _attn_struct(tr, **kw):
    a = dict(dt=1, n_seqs=2, heads=4, kv_heads=2, d=64, causal=0, n_buckets=32, max_distance=128, scale=0.125, total_q=10, total_k=12,
             q_offsets=0x1000, k_offsets=0x2000, q=0x3000, k=0x4000, v=0x5000, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128,
             v_head=64, keep=None, bias=None)
    a.update(kw)
    return tr.ColbanditAttn(**a)


def test_attention_refusals(tr):
    """Every case fails validation, so nothing is ever launched (no GPU needed)."""
    L = tr.lib()

    def forward(out=0x10000, lse=0x20000, ws=None, nb=0, **kw):
        return L.colbandit_attention(_attn_struct(tr, **kw), out, lse, ws, nb, None)

    def backward(out=0x10000, lse=0x20000, dout=0x30000, dq=0x40000, dk=0x50000, dv=0x60000, dbias=None, ws=0x100000, nb=1 << 30, **kw):
        return L.colbandit_attention_backward(_attn_struct(tr, **kw), out, lse, dout, dq, dk, dv, dbias, ws, nb, None)

    for call in (forward, backward):
        assert call(q=None) == -1 and call(k=None) == -1 and call(v=None) == -1
        assert call(q_offsets=None) == -1 and call(k_offsets=None) == -1 and call(out=None) == -1 and call(lse=None) == -1
        assert call(n_seqs=0) == -2 and call(heads=0) == -2 and call(kv_heads=0) == -2 and call(d=0) == -2 and call(dt=5) == -2
        assert call(heads=5) == -2 and call(total_q=-1) == -2 and call(total_k=-1) == -2
        assert call(scale=math.nan) == -3 and call(scale=math.inf) == -3
        assert call(d=48) == -4 and call(d=256) == -4 and call(total_q=1 << 31) == -4 and call(total_k=1 << 31) == -4
        assert call(q=0x3008) == -6 and call(k=0x4002) == -6 and call(v=0x5004) == -6 and call(out=0x10008) == -6
        assert call(q_row=260) == -6 and call(k_head=4) == -6 and call(v_row=1) == -6 and call(q_offsets=0x1004) == -6
        more = {} if call is forward else {"dbias": 0x70000}
        assert call(bias=0x6000, n_buckets=31, **more) == -2 and call(bias=0x6000, max_distance=300, **more) == -4
        assert call(bias=0x6001, **more) == -6
    assert forward(n_seqs=1, total_q=1, total_k=5000) == -1                    # split keys need a workspace
    assert forward(n_seqs=1, total_q=1, total_k=5000, ws=0x100010, nb=1 << 30) == -6
    assert forward(n_seqs=1, total_q=1, total_k=5000, ws=0x100000, nb=256) == -5
    assert backward(dout=None) == -1 and backward(dq=None) == -1 and backward(dk=None) == -1 and backward(dv=None) == -1
    assert backward(bias=0x6000) == -1 and backward(ws=None) == -1 and backward(ws=0x100010) == -6 and backward(nb=16) == -5
    assert backward(dv=0x60008) == -6 and backward(bias=0x6000, dbias=0x70001) == -6
    assert L.colbandit_attention(None, 0x10000, 0x20000, None, 0, None) == -1
    assert L.colbandit_attention_workspace_bytes(_attn_struct(tr, d=48), 1) == 0


def test_loss_and_clip_refusals(tr):
    L = tr.lib()

    def scores(Q=0x1000, nq=2, T=8, d=64, dt=1, docs=0x2000, off=0x3000, N=3, total=20, s=0x4000, a=0x5000):
        return L.colbandit_maxsim_scores(Q, nq, T, d, dt, docs, off, N, total, s, a, None)

    def grads(g=0x4000, a=0x5000, Q=0x1000, nq=2, T=8, d=64, dt=1, docs=0x2000, off=0x3000, N=3, total=20, dQ=0x6000, dD=0x7000):
        return L.colbandit_maxsim_backward(g, a, Q, nq, T, d, dt, docs, off, N, total, dQ, dD, None)

    for call in (scores, grads):
        assert call(Q=None) == -1 and call(docs=None) == -1 and call(off=None) == -1 and call(a=None) == -1
        assert call(nq=0) == -2 and call(T=0) == -2 and call(N=0) == -2 and call(total=-1) == -2 and call(dt=3) == -2
        assert call(d=48) == -4 and call(T=129) == -4 and call(nq=65536) == -4
        assert call(Q=0x1008) == -6 and call(docs=0x2002) == -6 and call(off=0x3004) == -6 and call(a=0x5002) == -6
    assert scores(s=None) == -1 and grads(g=None) == -1 and grads(dQ=None) == -1 and grads(dD=None) == -1 and grads(dD=0x7008) == -6

    def loss(s=0x1000, nq=2, N=3, t=0x2000, temp=1.0, out=0x3000, g=0x4000):
        return L.colbandit_contrastive_loss(s, nq, N, t, temp, out, g, None)
    assert loss(s=None) == -1 and loss(t=None) == -1 and loss(out=None) == -1 and loss(g=None) == -1
    assert loss(nq=0) == -2 and loss(N=0) == -2 and loss(nq=65536) == -4 and loss(t=0x2004) == -6
    assert loss(temp=0.0) == -3 and loss(temp=-1.0) == -3 and loss(temp=math.nan) == -3 and loss(temp=math.inf) == -3

    def clip(n=2, g=(0x1000, 0x2000), o=(0x1000, 0x2000), sizes=(4, 5), dts=(0, 1), most=1.0, norm=0x3000, ws=0x10000, nb=1 << 20):
        arr = lambda t, v: None if v is None else (t * len(v))(*v)  # noqa: E731
        return L.colbandit_clip_gradients(n, arr(ctypes.c_void_p, g), arr(ctypes.c_void_p, o), arr(ctypes.c_int64, sizes),
                                          arr(ctypes.c_int32, dts), most, norm, ws, nb, None)
    assert clip(g=None) == -1 and clip(sizes=None) == -1 and clip(dts=None) == -1 and clip(norm=None) == -1 and clip(ws=None) == -1
    assert clip(n=0) == -2 and clip(sizes=(4, -1)) == -2 and clip(dts=(0, 2)) == -2 and clip(g=(0x1000, None)) == -1
    assert clip(o=(None, 0x2000)) == -1 and clip(most=0.0) == -3 and clip(most=math.nan) == -3 and clip(sizes=(4, 1 << 43)) == -4
    assert clip(g=(0x1002, 0x2000)) == -6 and clip(o=(0x1000, 0x2001)) == -6 and clip(ws=0x10010) == -6 and clip(nb=8) == -5


def test_python_refusals(tr):
    """Shapes, types and places are checked before the library is called."""
    q = torch.zeros(10, 2, 64)
    off = torch.tensor([0, 10])
    for bad in (dict(q=q.half()), dict(k=q.bfloat16()), dict(q=q[0]), dict(v=q[:, :1]), dict(off=off.int()), dict(off=off[:1]),
                dict(q=q.transpose(1, 2)), dict(keep=torch.zeros(9, dtype=torch.bool)), dict(keep=torch.zeros(10)),
                dict(bias=torch.zeros(32, 3)), dict(bias=torch.zeros(32, 2).bfloat16()), dict(k_off=torch.tensor([0, 5, 10])), {}):
        a = dict(q=q, k=q, v=q, off=off, keep=None, bias=None, k_off=None)
        a.update(bad)
        if not bad and torch.cuda.is_available():
            continue                                 # the last: tensors that are not on the device
        with pytest.raises((TypeError, ValueError, RuntimeError, AssertionError)):
            tr.colbandit_attention(a["q"], a["k"], a["v"], a["off"], a["k_off"], keep=a["keep"], bias=a["bias"])


def test_what_a_call_writes_must_be_on_the_device(tr, monkeypatch):
    """Outputs and workspaces that lie elsewhere are refused before the library is called (here by a stand-in of it, with the tensors'
    places made up, so that nothing is launched)."""
    class Library:
        def __getattr__(self, name):
            return (lambda *a: 256) if name.endswith("workspace_bytes") else lambda *a: pytest.fail(name + " was called")
    elsewhere = []
    monkeypatch.setattr(tr, "lib", Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: -1 if any(t is x for x in elsewhere) else 0)
    q, off = torch.zeros(10, 2, 64), torch.tensor([0, 10])
    g, out, lse, ws = [torch.zeros(5), torch.zeros(3)], torch.zeros_like(q), torch.zeros(2, 10), torch.zeros(256, dtype=torch.uint8)
    to = [torch.zeros(5), torch.zeros(3)]
    calls = {
        "out": (out, lambda: tr.colbandit_attention(q, q, q, off, out={"out": out, "lse": lse}, workspace=ws)),
        "lse": (lse, lambda: tr.colbandit_attention(q, q, q, off, out={"out": out, "lse": lse}, workspace=ws)),
        "workspace": (ws, lambda: tr.colbandit_attention(q, q, q, off, workspace=ws)),
        "backward workspace": (ws, lambda: tr.colbandit_attention_backward(q, q, q, q, out, lse, off, workspace=ws)),
        "clipped": (to[1], lambda: tr.colbandit_clip_gradients(g, 1.0, out=to, workspace=ws)),
        "clip workspace": (ws, lambda: tr.colbandit_clip_gradients(g, 1.0, workspace=ws)),
    }
    for name, (tensor, call) in calls.items():
        elsewhere[:] = [tensor]
        with pytest.raises(ValueError, match="current device"):
            call()
            pytest.fail(name)


def second_order_is_an_error(value, x):
    """First-order gradients as ever; a penalty on them is no term that is left out."""
    (value() * 2).backward()
    first, x.grad = x.grad, None
    g, = torch.autograd.grad(value(), x, create_graph=True)
    assert torch.equal(g * 2, first)
    with pytest.raises(RuntimeError, match="second-order"):
        (g.square().sum() + x.square().sum()).backward()


def test_second_order_gradients_are_refused(tr, monkeypatch):
    """The autograd forms over stand-ins of the library's calls."""
    monkeypatch.setattr(tr, "colbandit_attention", lambda q, *a, **k: {"out": q.detach() * 3, "lse": q.new_zeros(2, 10)})
    monkeypatch.setattr(tr, "colbandit_attention_backward", lambda dout, q, k, v, *a, bias=None, **h: {
        "dq": dout * 3, "dk": torch.zeros_like(k), "dv": torch.zeros_like(v), "dbias": None if bias is None else torch.zeros_like(bias)})
    monkeypatch.setattr(tr, "colbandit_maxsim_scores", lambda Q, docs, off: {"scores": Q.detach().sum((1, 2))[:, None], "argmax": off})
    monkeypatch.setattr(tr, "colbandit_contrastive_loss", lambda s, t, temp: {"loss": s[:, 0], "dscores": torch.ones_like(s) / len(s)})
    monkeypatch.setattr(tr, "colbandit_maxsim_backward", lambda d, a, Q, docs, off: {
        "dQ": d[:, :, None].expand(Q.shape).clone(), "ddocs": torch.zeros_like(docs)})
    q, off = torch.randn(10, 2, 64, requires_grad=True), torch.tensor([0, 10])
    for bias in (None, torch.zeros(32, 2, requires_grad=True)):
        q.grad = None
        second_order_is_an_error(lambda: tr.attention(q, q.detach(), q.detach(), off, bias=bias).sum(), q)
    Q, docs = torch.randn(3, 4, 32, requires_grad=True), torch.randn(7, 32)
    second_order_is_an_error(lambda: tr.contrastive_maxsim(Q, docs, torch.tensor([0, 7]), torch.zeros(3, dtype=torch.int64)), Q)


@gpu
def test_second_order_gradients_are_refused_on_the_device(tr, dev):
    q, off = torch.randn(10, 2, 64, device=dev, requires_grad=True), torch.tensor([0, 4, 10], device=dev)
    second_order_is_an_error(lambda: tr.attention(q, q.detach() * 0.5, q.detach(), off).sum(), q)
    Q, D, docs = embeddings(dev, "f32", 3, 7, [5, 6], 32)
    Q.requires_grad_()
    second_order_is_an_error(lambda: tr.contrastive_maxsim(Q, D, docs, torch.tensor([0, 1, 0], device=dev)), Q)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,H,Hk,d,bias", [([40, 3], [40, 3], 2, 2, 64, 8), ([1, 1, 1], [2000, 7, 900], 4, 1, 128, None),
                                               ([130, 0, 300, 64], [130, 0, 300, 64], 6, 2, 32, None), ([5], [5], 1, 1, 96, 32)])
@pytest.mark.parametrize("more", [1, 31, 64, 128, 333])
def test_rows_behind_the_last_sequence_get_zeros(tr, dev, dtype, ql, kl, H, Hk, d, bias, more):
    """A batch padded to a round size, with NaN: the sequences' results are those without it (the plan may be another), the other
    rows' are zeros, and minus infinity for the log-sum-exp."""
    p = problem(dev, dtype, ql, kl, H, Hk, d, seed=27, bias=bias, keep=True)
    r = Attention(p["q"], p["k"], p["v"], ql, kl, dtype, keep=p["keep"], bias=p["bias"], dout=p["dout"])
    nq, nk = sum(ql), sum(kl)
    far = {x: torch.full((p[x].shape[0] + more, *p[x].shape[1:]), math.nan, dtype=DT[dtype], device=dev) for x in ("q", "k", "v", "dout")}
    for x in far:
        far[x][:len(p[x])] = p[x]
    far["keep"] = torch.ones(nk + more, dtype=torch.bool, device=dev)
    far["keep"][:nk] = p["keep"]
    for x in ("q", "k", "v"):                        # what the allocator gives next held other values
        torch.full_like(far[x], 7.0)
    f, b = attend(tr, dict(far, bias=p["bias"]), ql, kl)
    within(f["out"][:nq], r.out, r.out_tol, "out")
    assert not f["out"][nq:].any() and bool((f["lse"][:, nq:] == -math.inf).all())
    for x, n in (("dq", nq), ("dk", nk), ("dv", nk)):
        within(b[x][:n], getattr(r, x), getattr(r, x + "_tol"), x)
        assert not b[x][n:].any(), x
    if bias is not None:
        within(b["dbias"], r.dbias, r.dbias_tol, "dbias")


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,T", [(3, 7), (150, 32)])
@pytest.mark.parametrize("lengths", [[50, 0, 64, 3], [1]])
@pytest.mark.parametrize("more", [1, 64, 200])
def test_tokens_behind_the_last_document_get_zeros(tr, dev, dtype, nq, T, lengths, more):
    Q, D, off = embeddings(dev, dtype, nq, T, lengths, 96, seed=28)
    padded = torch.cat([D, torch.full((more, 96), math.nan, dtype=D.dtype, device=dev)])
    f, g = tr.colbandit_maxsim_scores(Q, D, off), tr.colbandit_maxsim_scores(Q, padded, off)
    assert torch.equal(f["scores"], g["scores"]) and torch.equal(f["argmax"], g["argmax"])
    dscores = torch.randn(nq, len(lengths), generator=torch.Generator().manual_seed(1)).to(dev)
    want = tr.colbandit_maxsim_backward(dscores, f["argmax"], Q, D, off)
    torch.full_like(padded, 7.0)
    got = tr.colbandit_maxsim_backward(dscores, f["argmax"], Q, padded, off)
    assert torch.equal(got["dQ"], want["dQ"]) and torch.equal(got["ddocs"][:len(D)], want["ddocs"]) and not got["ddocs"][len(D):].any()


def test_what_no_launch_can_hold_is_refused(tr):
    """Launches of 2^32 threads and more are refused as what they are before anything is enqueued (the device would refuse them one
    by one, the second after the first has run)."""
    L = tr.lib()
    def both(**kw):
        a = _attn_struct(tr, **kw)
        return (L.colbandit_attention(a, 0x10000, 0x20000, 0x100000, 1 << 45, None),
                L.colbandit_attention_backward(a, 0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000, None, 0x100000, 1 << 45, None))

    assert both(n_seqs=6_000_000, total_q=6_000_000, total_k=6_000_000, heads=12, kv_heads=12) == (-4, -4)
    assert both(n_seqs=1, total_q=(1 << 31) - (1 << 17), total_k=64, heads=64, kv_heads=64) == (-4, -4)
    assert both(n_seqs=1, total_q=10, total_k=12, heads=8192, kv_heads=8192, q_row=64, k_row=64, v_row=64, d=32) == (-4, -4)

    def grads(nq=2, T=8, N=3, total=20):
        return L.colbandit_maxsim_backward(0x4000, 0x5000, 0x1000, nq, T, 64, 1, 0x2000, 0x3000, N, total, 0x6000, 0x7000, None)

    assert grads(N=1 << 24) == -4 and grads(total=1 << 30, N=3) == -4 and grads(nq=65535, T=128, N=9_000_000) == -4


def test_clipping_where_nothing_has_a_gradient(tr):
    assert float(tr.clip_gradients_([], 1.0)) == 0 and float(tr.clip_gradients_(iter([torch.nn.Parameter(torch.ones(3))]), 1.0)) == 0


def test_a_parameter_that_is_listed_twice_is_clipped_once(tr, monkeypatch):
    """Two entries of one tensor would be scaled in place by two workgroups at once."""
    monkeypatch.setattr(tr, "colbandit_clip_gradients", lambda grads, most: {"norm": len(grads)})
    p, q = (torch.nn.Parameter(torch.ones(3)) for _ in range(2))
    p.grad, q.grad = torch.ones(3), torch.ones(3)
    assert tr.clip_gradients_([p, q, p], 1.0) == 2


@gpu
def test_fine_tuning_on_fewer_documents_than_a_batch(tr, dev):
    from paper_2602_02827_amd import finetune
    r = finetune.train(steps=2, n_docs=5)
    assert all(math.isfinite(x) for x in r["losses"] + r["norms"])


# ---- forms that large calls take -------------------------------------------------------------------------

def heads_in_a_row(ql, kl, heads, kv_heads, bias):
    """Whether the plan's workgroups go on to a second head: units (key heads) in pairs leave 1,536 workgroups or more, of short
    sequences; for the queries' tiles and for the keys'."""
    n, group = len(ql), heads // kv_heads
    pack = 1 if bias or group > 16 else group
    units, q_slots, k_slots = heads // pack, sum(ql) // (128 // pack) + n, sum(kl) // 128 + n
    short = sum(kl) // n <= 384 and sum(ql) * group // n <= 384
    return short and units > 1 and q_slots * (units // 2) >= 1536, short and kv_heads > 1 and k_slots * (kv_heads // 2) >= 1536


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("bias,keep,causal", [(None, False, False), (32, True, False), (8, False, True)])
def test_two_heads_a_workgroup_of_many_sequences(tr, dev, dtype, d, bias, keep, causal):
    """Three heads: the last workgroup of a tile has one."""
    lengths = np.random.default_rng(30).integers(0, 10, 1600).tolist()
    assert heads_in_a_row(lengths, lengths, 3, 3, bias) == (True, True)
    p = problem(dev, dtype, lengths, lengths, 3, 3, d, seed=30, bias=bias, keep=keep)
    check_attention(tr, p, lengths, lengths, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype,d,bias,keep,causal", [("bf16", 64, 32, True, False), ("bf16", 32, None, True, True), ("f32", 32, 32, False, True)])
def test_two_heads_a_workgroup_of_several_tiles(tr, dev, dtype, d, bias, keep, causal):
    lengths = [1 + i * 179 // 127 for i in range(128)]
    assert heads_in_a_row(lengths, lengths, 25, 25, bias) == (True, True)
    p = problem(dev, dtype, lengths, lengths, 25, 25, d, seed=31, bias=bias, keep=keep)
    check_attention(tr, p, lengths, lengths, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias,keep,causal", [(None, True, True), (None, False, False), (32, True, False)])
def test_two_heads_a_workgroup_that_share_keys(tr, dev, dtype, bias, keep, causal):
    g = np.random.default_rng(32)
    kl = g.integers(0, 21, 800).tolist()
    ql = [int(x) for x in np.minimum(g.integers(0, 30, 800), 25)]
    assert heads_in_a_row(ql, kl, 10, 5, bias) == (True, True)
    p = problem(dev, dtype, ql, kl, 10, 5, 64, seed=32, bias=bias, keep=keep)
    check_attention(tr, p, ql, kl, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("n_buckets,causal", [(64, False), (128, False), (31, True)])
def test_tables_that_reach_beyond_128(tr, dev, dtype, d, n_buckets, causal):
    """Their histograms leave a workgroup one head, where there are many sequences too."""
    lengths = [9, 0, 4] * 60 + [600]
    p = problem(dev, dtype, lengths, lengths, 3, 3, d, seed=33, bias=n_buckets, keep=True)
    starts = tr.colbandit_bias_buckets(n_buckets, 256, causal)
    assert starts[-1] > 128
    check_attention(tr, p, lengths, lengths, dtype, causal, max_distance=256)


@gpu
def test_tables_that_reach_beyond_128_over_many_sequences(tr, dev):
    lengths = [9, 0, 4] * 533 + [500]
    assert heads_in_a_row(lengths, lengths, 3, 3, 128) == (True, True)
    p = problem(dev, "bf16", lengths, lengths, 3, 3, 64, seed=34, bias=128)
    check_attention(tr, p, lengths, lengths, "bf16", max_distance=256)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("nq,T", [(24, 32), (11, 24), (3, 128)])
def test_maxsim_of_many_documents(tr, dev, dtype, d, nq, T):
    """Two columns a lane: groups of queries times documents are 1,024 or more."""
    lengths = np.random.default_rng(35).integers(0, 80, 700).tolist()
    assert -(-nq // (256 // T)) * len(lengths) >= 1024
    Q, D, off = embeddings(dev, dtype, nq, T, lengths, d, seed=35)
    f = tr.colbandit_maxsim_scores(Q, D, off)
    scores, arg = maxsim_reference(Q, D, off)
    np.testing.assert_array_equal(f["argmax"].cpu().numpy(), arg)
    np.testing.assert_array_equal(f["scores"].double().cpu().numpy(), scores)
    g = torch.randn(nq, len(lengths), generator=torch.Generator().manual_seed(2)).to(dev)
    b = tr.colbandit_maxsim_backward(g, f["argmax"], Q, D, off)
    dQ, dQ_abs, dD, dD_abs = gradient_reference(g, arg, Q, D, off)
    within(b["dQ"], dQ, U[dtype] * dQ.abs() + F * dQ_abs, "dQ")
    within(b["ddocs"], dD, U[dtype] * dD.abs() + F * dD_abs, "ddocs")


@gpu
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("nq,T,n", [(5, 24, 40), (24, 32, 400)])
@pytest.mark.parametrize("spread", [0, 3])
def test_maxsim_scores_of_full_width_numbers(tr, dev, d, nq, T, n, spread):
    """fp32 values of 24 significant bits, of sizes up to 10^spread apart.  A product's pieces that are left out are 2^-22 of it; six
    products of pieces for sixteen elements are added one after the other, each sum off by at most 2^-23 of the absolute terms.  The
    chosen token is one whose cell is within both cells' bounds of the best."""
    g = torch.Generator().manual_seed(36 + d)
    lengths = np.random.default_rng(36).integers(1, 60, n).tolist()
    size = 10.0 ** (torch.rand(d, generator=g) * spread)
    Q = (torch.randn(nq, T, d, generator=g) * size / d ** 0.5).to(dev)
    D = (torch.randn(sum(lengths), d, generator=g) / size).to(dev)
    off = offsets(lengths).to(dev)
    f = tr.colbandit_maxsim_scores(Q, D, off)
    q, x, arg = Q.double().cpu().reshape(nq * T, d), D.double().cpu(), f["argmax"].cpu().long()
    rate = 2.0 ** -22 + 6 * d / 16 * 2.0 ** -23
    o = off.tolist()
    for i in range(n):
        S, A = q @ x[o[i]:o[i + 1]].T, rate * (q.abs() @ x[o[i]:o[i + 1]].abs().T)
        at = arg[:, i].reshape(-1, 1)
        best = S.max(1, keepdim=True)
        assert bool((S.gather(1, at) >= best.values - A.gather(1, at) - A.gather(1, best.indices)).all())
        want, tol = best.values.view(nq, T).sum(1), A.max(1).values.view(nq, T).sum(1)
        tol = tol + T * 2.0 ** -24 * best.values.abs().view(nq, T).sum(1)
        assert bool(((f["scores"][:, i].double().cpu() - want).abs() <= tol).all()), i


# ---- refusals of the binding on tensors that are on the device -----------------------------------------------

def refused(call, base, bad):
    """The call takes `base`, and refuses each change of it by its own error and words."""
    call(**base)
    for change, error, words in bad:
        with pytest.raises(error, match=words):
            call(**dict(base, **change))
            pytest.fail(str(change))


@gpu
def test_attention_refusals_on_the_device(tr, dev):
    q, off = torch.zeros(10, 2, 64, device=dev), torch.tensor([0, 10], device=dev)
    cpu = q.cpu()
    base = dict(q=q, k=q, v=q, q_offsets=off, k_offsets=None, keep=torch.ones(10, dtype=torch.bool, device=dev),
                bias=torch.zeros(32, 2, device=dev), max_distance=128, scale=None)
    E = tr.ColbanditError
    bad = [
        (dict(q=q.half()), TypeError, "float32 or bfloat16"), (dict(k=q.bfloat16()), TypeError, "one type"),
        (dict(v=q.double()), TypeError, "one type"), (dict(q=q[0]), ValueError, "total_q, heads, d"),
        (dict(v=q[:, :1]), ValueError, "total_k, kv_heads, d"), (dict(k=q[:, :, :32], v=q[:, :, :32]), ValueError, "total_k, kv_heads, d"),
        (dict(q=torch.zeros(10, 64, 2, device=dev).transpose(1, 2)), ValueError, "consecutive"),
        (dict(q_offsets=off.int()), ValueError, "offsets"), (dict(q_offsets=off[:1]), ValueError, "offsets"),
        (dict(q_offsets=torch.tensor([0, 1, 10, 1], device=dev)[::2]), ValueError, "offsets"),
        (dict(k_offsets=torch.tensor([0, 5, 10], device=dev)), ValueError, "equally many"),
        (dict(keep=torch.ones(9, dtype=torch.bool, device=dev)), ValueError, "keep"), (dict(keep=torch.ones(10, device=dev)), ValueError, "keep"),
        (dict(bias=torch.zeros(32, 3, device=dev)), ValueError, "n_buckets, heads"),
        (dict(bias=torch.zeros(2, 32, device=dev).t()), ValueError, "n_buckets, heads"),
        (dict(bias=torch.zeros(32, 2, device=dev).bfloat16()), TypeError, "type of q"),
        (dict(q=cpu), ValueError, "current device"), (dict(k=cpu), ValueError, "current device"), (dict(v=cpu), ValueError, "current device"),
        (dict(q_offsets=off.cpu()), ValueError, "current device"), (dict(k_offsets=off.cpu()), ValueError, "current device"),
        (dict(keep=torch.ones(10, dtype=torch.bool)), ValueError, "current device"), (dict(bias=torch.zeros(32, 2)), ValueError, "current device"),
        (dict(scale=math.nan), E, "knob"), (dict(bias=torch.zeros(31, 2, device=dev)), E, "invalid size"), (dict(max_distance=300), E, "kernels cover"),
    ]
    refused(tr.colbandit_attention, base, bad)
    f = tr.colbandit_attention(q, q, q, off)
    back = dict(base, dout=torch.zeros_like(q), out=f["out"], lse=f["lse"])
    more = [(dict(dout=q[:9]), ValueError, "dout"), (dict(out=q.bfloat16()), ValueError, "out"), (dict(lse=f["lse"].t().contiguous()), ValueError, "lse"),
            (dict(dout=cpu), ValueError, "current device"), (dict(out=cpu), ValueError, "current device"), (dict(lse=f["lse"].cpu()), ValueError, "current device")]
    refused(tr.colbandit_attention_backward, back, bad + more)
    for out, words in ((dict(out=q.clone(), lse=f["lse"].cpu()), "current device"), (dict(out=cpu, lse=f["lse"]), "current device"),
                       (dict(out=q[:9].clone(), lse=f["lse"]), "out"), (dict(out=q.clone(), lse=f["lse"].double()), "lse")):
        with pytest.raises(ValueError, match=words):
            tr.colbandit_attention(q, q, q, off, out=out)


@gpu
def test_loss_and_clip_refusals_on_the_device(tr, dev):
    Q, D, off = embeddings(dev, "f32", 3, 7, [5, 6], 64)
    base = dict(Q=Q, docs=D, offsets=off)
    bad = [(dict(Q=Q.half()), TypeError, "float32 or bfloat16"), (dict(docs=D.bfloat16()), TypeError, "one type"),
           (dict(Q=Q[0]), ValueError, "n_queries"), (dict(docs=D[:, :32]), ValueError, "n_queries"), (dict(Q=Q[:, ::2]), ValueError, "contiguous"),
           (dict(docs=D[::2]), ValueError, "contiguous"), (dict(offsets=off.int()), ValueError, "offsets"), (dict(offsets=off[:1]), ValueError, "offsets"),
           (dict(Q=Q.cpu()), ValueError, "current device"), (dict(docs=D.cpu()), ValueError, "current device"),
           (dict(offsets=off.cpu()), ValueError, "current device"),
           (dict(Q=Q[:, :, :48].contiguous(), docs=D[:, :48].contiguous()), tr.ColbanditError, "kernels cover")]
    refused(tr.colbandit_maxsim_scores, base, bad)
    f = tr.colbandit_maxsim_scores(Q, D, off)
    g = torch.zeros_like(f["scores"])
    more = [(dict(dscores=g[:2]), ValueError, "dscores"), (dict(dscores=g.double()), ValueError, "dscores"), (dict(argmax=f["argmax"].long()), ValueError, "argmax"),
            (dict(dscores=g.cpu()), ValueError, "current device"), (dict(argmax=f["argmax"].cpu()), ValueError, "current device")]
    refused(tr.colbandit_maxsim_backward, dict(base, dscores=g, argmax=f["argmax"]), bad + more)
    t = torch.tensor([0, 1, 0], device=dev)
    refused(tr.colbandit_contrastive_loss, dict(scores=g, targets=t, temperature=1.0), [
        (dict(scores=g.double()), ValueError, "scores"), (dict(scores=g.t()), ValueError, "scores"), (dict(targets=t.int()), ValueError, "targets"),
        (dict(targets=t[:2]), ValueError, "targets"), (dict(scores=g.cpu()), ValueError, "current device"),
        (dict(targets=t.cpu()), ValueError, "current device"), (dict(temperature=0.0), tr.ColbanditError, "knob")])
    x = [torch.ones(5, device=dev), torch.ones(3, device=dev).bfloat16()]
    to = [torch.empty_like(a) for a in x]
    refused(tr.colbandit_clip_gradients, dict(grads=x, max_norm=1.0, out=to), [
        (dict(grads=[]), ValueError, "list of tensors"), (dict(out=to[:1]), ValueError, "as many"), (dict(grads=[x[0].half(), x[1]]), TypeError, "float32 or bfloat16"),
        (dict(out=[to[1], to[0]]), TypeError, "of their types"), (dict(out=[to[0][:4], to[1]]), ValueError, "of their shapes"),
        (dict(grads=[torch.ones(10, device=dev)[::2], x[1]]), ValueError, "contiguous"), (dict(grads=[x[0].cpu(), x[1]]), ValueError, "current device"),
        (dict(out=[to[0].cpu(), to[1]]), ValueError, "current device"), (dict(max_norm=0.0), tr.ColbanditError, "knob")])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl", [([40, 200], [40, 200]), ([1, 1], [700, 3000])])
@pytest.mark.parametrize("bias", [None, 8])
def test_a_nan_that_is_seen_is_in_every_result(tr, dev, dtype, ql, kl, bias):
    """A key of the second sequence is NaN: so are all results of its rows, and the first sequence's are as they were."""
    p = problem(dev, dtype, ql, kl, 2, 2, 64, seed=40, bias=bias)
    f, b = attend(tr, p, ql, kl)
    p["k"] = p["k"].clone()
    p["k"][kl[0] + 2] = math.nan
    g, c = attend(tr, p, ql, kl)
    for x, y, rows in ((f["out"], g["out"], ql[0]), (f["lse"].t(), g["lse"].t(), ql[0]), (b["dq"], c["dq"], ql[0]), (b["dk"], c["dk"], kl[0]), (b["dv"], c["dv"], kl[0])):
        assert torch.equal(x[:rows], y[:rows]) and bool(torch.isnan(y[rows:]).all())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl", [([40, 200], [40, 200]), ([1, 1], [700, 3000])])
@pytest.mark.parametrize("bias", [None, 8])
def test_a_query_that_is_nan_is_in_every_result(tr, dev, dtype, ql, kl, bias):
    """The last row of the second sequence: all its scores are NaN, so it is no row that sees nothing."""
    p = problem(dev, dtype, ql, kl, 2, 2, 64, seed=41, bias=bias)
    p["q"][-1] = math.nan
    f, b = attend(tr, p, ql, kl)
    for x in (f["out"][-1], f["lse"][:, -1], b["dq"][-1], b["dk"][kl[0]:], b["dv"][kl[0]:]):
        assert bool(torch.isnan(x).all())
    for x in (f["out"][:-1], f["lse"][:, :-1], b["dq"][:-1], b["dk"][:kl[0]], b["dv"][:kl[0]]):
        assert bool(torch.isfinite(x).all())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("head", [0, 1, 2])
def test_one_head_of_several_in_a_row_is_far_from_zero(tr, dev, dtype, d, causal, head):
    """Workgroups that go on from a head whose rows see nothing but a hidden distance to one whose do not, and the other way."""
    lengths = np.random.default_rng(43).integers(0, 4, 1600).tolist()
    assert heads_in_a_row(lengths, lengths, 3, 3, 8) == (True, True)
    p = problem(dev, dtype, lengths, lengths, 3, 3, d, seed=43, bias=8)
    p["bias"][0, head] = torch.finfo(DT[dtype]).min
    check_far(tr, p, lengths, lengths, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,heads,kv_heads", [(64, 4, 4), (128, 4, 2), (96, 3, 1)])
@pytest.mark.parametrize("ql,kl", [([150, 3, 70], [150, 3, 70]), ([40, 1], [1100, 900])])
@pytest.mark.parametrize("causal", [False, True])
def test_rows_on_both_sides_of_where_they_are_normalised_again(tr, dev, monkeypatch, dtype, d, heads, kv_heads, ql, kl, causal):
    """Ordinary rows with biases that move them to 240 and to 280: log-sum-exps below and above 256 in one call.  Scores of up to 290
    carry nine times the error of the file's bound, which is for up to 32."""
    monkeypatch.setitem(globals(), "F", F * 290 / 32)
    p = problem(dev, dtype, ql, kl, heads, kv_heads, d, seed=44, bias=32, keep=True)
    p["bias"] += torch.tensor([240.0, 280.0], device=dev).repeat(2)[:heads].to(DT[dtype])
    check_attention(tr, p, ql, kl, dtype, causal)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_a_table_of_minus_infinity_hides_a_distance(tr, dev, dtype, d, causal):
    """Rows that see nothing else see nothing."""
    lengths = [50, 1, 133, 1]
    p = problem(dev, dtype, lengths, lengths, 2, 2, d, seed=45, bias=8)
    p["bias"][0] = -math.inf
    check_attention(tr, p, lengths, lengths, dtype, causal)


def test_a_temperature_whose_inverse_is_infinite_is_refused(tr):
    L = tr.lib()
    for temperature in (1e-39, 1e-45):
        assert L.colbandit_contrastive_loss(0x1000, 2, 3, 0x2000, temperature, 0x3000, 0x4000, None) == -3


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,Hk,bias", [(64, 2, 2, 8), (64, 6, 2, None), (128, 4, 2, None), (96, 2, 2, 32)])
def test_rows_before_all_keys_may_hold_anything(tr, dev, dtype, d, H, Hk, bias):
    """More queries than keys under a causal limit, and none at all: rows that see nothing, without a mask."""
    ql, kl = [140, 40, 7, 300], [9, 39, 0, 150]
    p = problem(dev, dtype, ql, kl, H, Hk, d, seed=46, bias=bias)
    f, b = check_attention(tr, p, ql, kl, dtype, True)
    wild = dict(p, q=p["q"].clone(), dout=p["dout"].clone())
    a = 0
    for lq, lk in zip(ql, kl):
        wild["q"][a:a + lq - lk] = math.nan
        wild["dout"][a:a + lq - lk] = math.inf
        a += lq
    f2, b2 = attend(tr, wild, ql, kl, True)
    for x, y in ((f, f2), (b, b2)):
        for name in x:
            assert x[name] is None or torch.equal(x[name], y[name]), name
