"""Token lookup, norms with rotation, attention through a window and orthogonalised updates (include/colbandit_train.h)
against their formulas in 64 bits.

Tolerances are bounds on the rounding that the kernels do: a value rounded to the storage type is off by at most U of itself
(2^-8 for bf16, eight significant bits, to nearest; 2^-24 for fp32), a sum of n terms in 32 bits by at most n 2^-24 of the
sum of the absolute terms, whatever its order, and the few operations that a rotated value takes by F = 2e-5 of the absolute terms
(a mean of up to 128 squares in 32 bits is off by 2^-18 at most)."""
import ctypes
import math

import numpy as np
import pytest
import torch

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
F = 2e-5
E32 = 2.0 ** -24
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


def within(got, want, tol, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape and bool(torch.isfinite(got).all()), what
    worst = (got - want).abs() - tol
    i = int(worst.argmax()) if worst.numel() else 0
    assert worst.numel() == 0 or float(worst.max()) <= 1e-30, (what, i, got.reshape(-1)[i], want.reshape(-1)[i], tol.reshape(-1)[i])


def captured(dev, call):
    """Outputs of `call` from a graph, replayed three times with eager work in between, each compared with the eager ones."""
    want = call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        for t in got.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x in want:
            assert torch.equal(got[x], want[x]), x
        again = call()
        torch.cuda.synchronize()
        assert all(torch.equal(again[x], want[x]) for x in want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert all(torch.equal(got[x], want[x]) for x in want)


# ---- token lookup ------------------------------------------------------------------------------------------

def tokens_of(kind, n, vocab, seed=0):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        t = torch.full((n,), vocab // 2, dtype=torch.int64)
    elif kind == "few":                               # some long runs, a chunk's worth and one more, and single ones
        t = torch.cat([torch.full((c,), i % vocab, dtype=torch.int64) for i, c in enumerate([64, 65, 63, 1, 200, 128, 129, 2])])
        t = t[torch.randperm(len(t), generator=g)][:n]
    else:
        t = torch.randint(0, vocab, (n,), generator=g)
        t[torch.rand(n, generator=g) < 0.3] = vocab - 1
    if kind == "padded":
        t[torch.rand(n, generator=g) < 0.2] = -1
        t[::7] = vocab
        t[1::11] = 1 << 40
        t[2::11] = -(1 << 40)
    return t


def check_embedding(tr, dev, tokens, vocab, width, table, out, scale=1.0, seed=0):
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(vocab, width, generator=g).to(DT[table]).to(dev)
    G = torch.randn(len(tokens), width, generator=g).to(DT[out]).to(dev)
    t = tokens.to(dev)
    got = tr.colbandit_embedding(W, t, scale=scale, dtype=DT[out])["out"]
    grad = tr.colbandit_embedding_backward(G, t, vocab, scale=scale, dtype=DT[table])["dtable"]
    torch.cuda.synchronize()
    real = (tokens >= 0) & (tokens < vocab)
    want = torch.zeros(len(tokens), width, dtype=torch.float64)
    s = float(np.float32(scale))
    want[real] = W.double().cpu()[tokens[real]] * s
    within(got, want, (U[out] + E32) * want.abs(), "out")
    Gd = G.double().cpu()
    sums, size = torch.zeros(vocab, width, dtype=torch.float64), torch.zeros(vocab, width, dtype=torch.float64)
    sums.index_add_(0, tokens[real], Gd[real])
    size.index_add_(0, tokens[real], Gd[real].abs())
    count = torch.bincount(tokens[real], minlength=vocab).double()[:, None]
    within(grad, sums * s, (U[table] * sums.abs() + (count + 2) * E32 * size) * abs(s), "dtable")
    return got, grad


@gpu
@pytest.mark.parametrize("table,out", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("width", [1, 7, 8, 129, 256])
@pytest.mark.parametrize("n,vocab,kind", [(1, 1, "one"), (63, 5, "any"), (65, 3, "one"), (652, 9, "few"), (1000, 700, "padded"), (1500, 1, "any")])
def test_embedding_rows_and_gradients(tr, dev, table, out, width, n, vocab, kind):
    check_embedding(tr, dev, tokens_of(kind, n, vocab), vocab, width, table, out, scale=1.7)


@gpu
@pytest.mark.parametrize("n,vocab,width,kind", [(70001, 300, 16, "any"), (70001, 3, 24, "one"), (20011, 250007, 8, "padded"), (5, 1 << 20, 1, "any")])
def test_embedding_of_many_tokens_and_rows(tr, dev, n, vocab, width, kind):
    check_embedding(tr, dev, tokens_of(kind, n, vocab), vocab, width, "f32", "bf16", scale=-0.25)


@gpu
def test_embedding_of_no_tokens(tr, dev):
    none = torch.zeros(0, dtype=torch.int64, device=dev)
    W = torch.randn(5, 24, device=dev)
    assert tr.colbandit_embedding(W, none)["out"].shape == (0, 24)
    g = tr.colbandit_embedding_backward(W[:0], none, 5)["dtable"]
    assert g.shape == (5, 24) and not bool(g.any())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_embedding_takes_rows_that_lie_apart(tr, dev, dtype):
    """Table and gradient as parts of wider tensors, aligned to 16 bytes and not."""
    t = tokens_of("any", 300, 40).to(dev)
    for first, row in ((0, 96), (8, 96), (1, 97), (4, 100)):
        whole = torch.randn(300, row, device=dev).to(DT[dtype])
        part = whole[:, first:first + 64]
        assert torch.equal(tr.colbandit_embedding(part[:40], t)["out"], part[:40][t])
        got = tr.colbandit_embedding_backward(part, t, 40)["dtable"]
        assert torch.equal(got, tr.colbandit_embedding_backward(part.contiguous(), t, 40)["dtable"])


@gpu
def test_embedding_padding_may_hold_anything(tr, dev):
    t = tokens_of("padded", 1000, 20)
    G = torch.randn(1000, 32)
    G[(t < 0) | (t >= 20)] = math.nan
    got = tr.colbandit_embedding_backward(G.to(dev), t.to(dev), 20)["dtable"]
    assert bool(torch.isfinite(got).all())
    W = torch.full((20, 32), math.inf, device=dev)
    out = tr.colbandit_embedding(W, t.to(dev))["out"].cpu()
    real = (t >= 0) & (t < 20)
    assert bool((out[~real] == 0).all()) and bool((out[real] == math.inf).all())


@gpu
def test_embedding_table_beyond_32_bits(tr, dev):
    vocab, width = (1 << 24) - 3, 264                 # 8.9 GB
    W = torch.zeros(vocab, width, dtype=torch.bfloat16, device=dev)
    rows = [0, 8135000, vocab - 1]                    # byte offsets on both sides of 2^32, elements on both sides of 2^31
    for i, r in enumerate(rows):
        W[r] = i + 1
    t = torch.tensor(rows * 40, device=dev)
    out = tr.colbandit_embedding(W, t, scale=2.0)["out"]
    assert torch.equal(out[:, 0].float().cpu(), torch.tensor([2.0, 4.0, 6.0] * 40))
    g = tr.colbandit_embedding_backward(out, t, vocab, out=W)["dtable"]
    assert torch.equal(g[rows][:, -1].float().cpu(), torch.tensor([80.0, 160.0, 240.0])) and float(g.sum(dtype=torch.float64)) == 480.0 * width


@gpu
def test_embedding_in_graphs_and_as_part_of_a_program(tr, dev):
    t = tokens_of("padded", 3000, 100).to(dev)
    W = torch.randn(100, 96, device=dev, requires_grad=True)
    G = torch.randn(3000, 96, device=dev)
    captured(dev, lambda: tr.colbandit_embedding(W.detach(), t, scale=3.0) | tr.colbandit_embedding_backward(G, t, 100, scale=3.0))
    out = tr.embedding(W, t.view(30, 100), scale=3.0, dtype=torch.bfloat16)
    assert out.shape == (30, 100, 96) and out.dtype == torch.bfloat16
    (out.float() * G.view(30, 100, 96)).sum().backward()
    want = tr.colbandit_embedding_backward(G.bfloat16(), t, 100, scale=3.0, dtype=torch.float32)["dtable"]
    assert torch.equal(W.grad, want)
    W.grad = None
    tr.embedding(W, t).sum().backward()               # an expanded gradient
    real = t[(t >= 0) & (t < 100)]
    assert torch.equal(W.grad[:, 0], torch.bincount(real, minlength=100).float())


# ---- norms and rotation ------------------------------------------------------------------------------------

def rotation_problem(dev, dtype, rows, H, Hk, d, seed=0, longest=50, weights=True):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    qkv = n(rows, (H + 2 * Hk) * d).to(DT[dtype]).to(dev)
    p = dict(q=qkv[:, :H * d].view(rows, H, d), k=qkv[:, H * d:(H + Hk) * d].view(rows, Hk, d),
             positions=torch.randint(0, longest, (rows,), generator=g).to(dev),
             q_weight=(1 + 0.2 * n(d)).to(dev) if weights else None, k_weight=(1 + 0.2 * n(d)).to(dev) if weights else None)
    return p, (n(rows, H, d) * 0.1).to(DT[dtype]).to(dev), (n(rows, Hk, d) * 0.1).to(DT[dtype]).to(dev)


def rotation_reference(x, w, positions, base, eps, interleaved, dy):
    """Outputs and gradients in 64 bits by autograd, and the absolute terms that bound their rounding."""
    x = x.detach().double().cpu()
    d = x.shape[2]
    w = torch.ones(d, dtype=torch.float64) if w is None else w.double().cpu()
    i = torch.arange(d // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
    if positions is None:
        angle = torch.zeros(x.shape[0], d // 2, dtype=torch.float64)
    else:
        angle = positions.double().cpu()[:, None] * base ** (-2.0 * i.double() / d)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

    def turned(y, s):
        out = torch.zeros_like(y)
        return out.index_copy(2, a, y[..., a] * c - y[..., b] * s).index_copy(2, b, y[..., b] * c + y[..., a] * s)

    def spread(y):                                    # of a pair, what both values are made of
        both = y[..., a].abs() + y[..., b].abs()
        return torch.zeros_like(y).index_copy(2, a, both).index_copy(2, b, both)

    x.requires_grad_()
    w.requires_grad_()
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    out = turned(x * r * w, s)
    dy = dy.double().cpu()
    dx, dw = torch.autograd.grad(out, (x, w), dy)
    with torch.no_grad():
        n = x * r
        u = spread(dy)
        e = u * w.abs()
        return dict(out=out.detach(), out_tol=spread(n * w), dx=dx, dx_tol=r * (e + n.abs() * (e * n.abs()).mean(-1, keepdim=True)), dw=dw,
                    dw_tol=(u * n.abs()).sum((0, 1)))


def check_rotation(tr, p, dq, dk, dtype, base=10000.0, eps=1e-6, interleaved=False, longest=50):
    table = tr.colbandit_rotary_table(longest, p["q"].shape[2], base) if p["positions"] is not None else None
    how = dict(p, table=table, eps=eps, interleaved=interleaved)
    q, k = how.pop("q"), how.pop("k")
    f = tr.colbandit_norm_rotate(q, k, **how)
    b = tr.colbandit_norm_rotate_backward(dq, dk, q, k, **how)
    torch.cuda.synchronize()
    for name, x, g in (("q", q, dq), ("k", k, dk)):
        r = rotation_reference(x, p[name + "_weight"], p["positions"], base, eps, interleaved, g)
        terms = x.shape[0] * x.shape[1]
        within(f[name], r["out"], U[dtype] * r["out"].abs() + F * r["out_tol"], name)
        within(b["d" + name], r["dx"], U[dtype] * r["dx"].abs() + F * r["dx_tol"], "d" + name)
        within(b["d" + name + "_weight"], r["dw"], (F + terms * E32) * r["dw_tol"], "weight of " + name)
    return f, b


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,H,Hk,weights", [(1, 1, 1, True), (3, 8, 2, False), (70, 5, 5, True), (701, 12, 3, True)])
def test_norms_and_rotation(tr, dev, dtype, d, interleaved, rows, H, Hk, weights):
    p, dq, dk = rotation_problem(dev, dtype, rows, H, Hk, d, weights=weights)
    check_rotation(tr, p, dq, dk, dtype, interleaved=interleaved)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_of_many_rows(tr, dev, dtype):
    p, dq, dk = rotation_problem(dev, dtype, 30011, 3, 1, 64, seed=3, longest=16384)
    check_rotation(tr, p, dq, dk, dtype, longest=16384)


@gpu
def test_far_positions_and_other_bases(tr, dev):
    p, dq, dk = rotation_problem(dev, "f32", 40, 2, 2, 64, seed=4, longest=200000)
    check_rotation(tr, p, dq, dk, "f32", base=500000.0, longest=200000)
    check_rotation(tr, p, dq, dk, "f32", base=0.5, eps=0.25, longest=200000)


@gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_norms_alone(tr, dev, interleaved):
    p, dq, dk = rotation_problem(dev, "f32", 33, 4, 2, 96, seed=5)
    check_rotation(tr, dict(p, positions=None), dq, dk, "f32", interleaved=interleaved)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_position_get_zeros(tr, dev, dtype):
    """Padding: positions outside of the table, whatever the rows hold."""
    p, dq, dk = rotation_problem(dev, dtype, 64, 4, 2, 64, seed=6)
    none = torch.zeros(64, dtype=torch.bool)
    none[5:20] = none[60:] = True
    none = none.to(dev)
    p["positions"][none] = torch.tensor([-1, 50, 1 << 40, -(1 << 40)], device=dev)[torch.arange(int(none.sum()), device=dev) % 4]
    clean = tr.colbandit_rotary_table(50, 64)
    how = {x: p[x] for x in ("positions", "q_weight", "k_weight")} | dict(table=clean)
    p["q"][none] = p["k"][none] = dq[none] = dk[none] = math.nan
    f = tr.colbandit_norm_rotate(p["q"], p["k"], **how)
    b = tr.colbandit_norm_rotate_backward(dq, dk, p["q"], p["k"], **how)
    for t in (f["q"], f["k"], b["dq"], b["dk"]):
        assert bool((t[none] == 0).all()) and bool(torch.isfinite(t).all())
    some = {x: (y[~none].contiguous() if x == "positions" else y) for x, y in how.items()}
    g = tr.colbandit_norm_rotate(p["q"][~none], p["k"][~none], **some)
    assert torch.equal(g["q"], f["q"][~none]) and torch.equal(g["k"], f["k"][~none])
    w = tr.colbandit_norm_rotate_backward(dq[~none], dk[~none], p["q"][~none], p["k"][~none], **some)
    for x in ("dq_weight", "dk_weight"):              # the same terms in another order
        assert bool(torch.isfinite(b[x]).all()) and float((b[x] - w[x]).abs().max()) <= 1e-5


@gpu
def test_norms_of_no_rows_and_of_zeros(tr, dev):
    q = torch.zeros(0, 2, 64, device=dev)
    assert tr.colbandit_norm_rotate(q, q)["q"].shape == (0, 2, 64)
    b = tr.colbandit_norm_rotate_backward(q, q, q, q)
    assert not bool(b["dq_weight"].any()) and not bool(b["dk_weight"].any())
    z = torch.zeros(3, 2, 64, device=dev)
    assert not bool(tr.colbandit_norm_rotate(z, z)["q"].any())


@gpu
def test_rotated_products_depend_on_distances_alone(tr, dev):
    """What the rotation is for: of one query and one key, the product at positions p + x and p does not depend on p."""
    g = torch.Generator().manual_seed(7)
    x, y = torch.randn(1, 1, 64, generator=g), torch.randn(1, 1, 64, generator=g)
    at = torch.tensor([0, 1, 500, 4000])
    table = tr.colbandit_rotary_table(5000, 64)
    for interleaved in (False, True):
        q = tr.colbandit_norm_rotate(x.expand(4, 1, 64).contiguous().to(dev), y.expand(4, 1, 64).contiguous().to(dev),
                                     positions=(at + 17).to(dev), table=table, interleaved=interleaved)["q"]
        k = tr.colbandit_norm_rotate(x.expand(4, 1, 64).contiguous().to(dev), y.expand(4, 1, 64).contiguous().to(dev),
                                     positions=at.to(dev), table=table, interleaved=interleaved)["k"]
        s = (q.double() * k.double()).sum((1, 2))
        # (terms of both of size 1, 64 of them, each off by a few 2^-24)
        assert float((s - s[0]).abs().max()) <= 64 * 4 * 8 * E32


@gpu
def test_rotation_in_graphs_and_as_part_of_a_program(tr, dev):
    p, dq, dk = rotation_problem(dev, "bf16", 300, 6, 3, 64, seed=8)
    how = {x: p[x] for x in ("positions", "q_weight", "k_weight")} | dict(table=tr.colbandit_rotary_table(50, 64))
    captured(dev, lambda: tr.colbandit_norm_rotate(p["q"], p["k"], **how) | tr.colbandit_norm_rotate_backward(dq, dk, p["q"], p["k"], **how))
    leaves = [p["q"].clone().requires_grad_(), p["k"].clone().requires_grad_(), p["q_weight"].clone().requires_grad_(), None]
    q, k = tr.norm_rotate(leaves[0], leaves[1], positions=how["positions"], table=how["table"], q_weight=leaves[2])
    ((q * dq).sum() + (k * dk).sum()).backward()
    b = tr.colbandit_norm_rotate_backward(dq, dk, p["q"], p["k"], positions=how["positions"], table=how["table"], q_weight=p["q_weight"])
    assert torch.equal(leaves[0].grad, b["dq"]) and torch.equal(leaves[1].grad, b["dk"]) and torch.equal(leaves[2].grad, b["dq_weight"])
    for t in leaves[:3]:
        t.grad = None
    q, k = tr.norm_rotate(leaves[0], leaves[1], positions=how["positions"], table=how["table"], q_weight=leaves[2])
    q.float().sum().backward()                        # one output's gradient alone, and expanded
    assert bool(torch.isfinite(leaves[0].grad).all()) and not bool(leaves[1].grad.any())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_in_place(tr, dev, dtype, interleaved):
    p, _, _ = rotation_problem(dev, dtype, 130, 5, 2, 96, seed=12)
    how = dict(positions=p["positions"], table=tr.colbandit_rotary_table(50, 96), q_weight=p["q_weight"], interleaved=interleaved)
    q, k = p["q"].contiguous(), p["k"].contiguous()
    want = tr.colbandit_norm_rotate(q, k, **how)
    got = tr.colbandit_norm_rotate(q, k, out={"q": q, "k": k}, **how)
    assert got["q"] is q and torch.equal(q, want["q"]) and torch.equal(k, want["k"])


@gpu
def test_rotation_gradients_against_differences(tr, dev):
    p, dq, dk = rotation_problem(dev, "f32", 9, 2, 1, 32, seed=9)
    table = tr.colbandit_rotary_table(50, 32)
    how = dict(positions=p["positions"], table=table)
    leaves = {x: p[x].detach().clone() for x in ("q", "k", "q_weight", "k_weight")}

    def value(**other):
        a = {**leaves, **other}
        f = tr.colbandit_norm_rotate(a["q"], a["k"], q_weight=a["q_weight"], k_weight=a["k_weight"], **how)
        return float((f["q"].double() * dq.double()).sum() + (f["k"].double() * dk.double()).sum())

    b = tr.colbandit_norm_rotate_backward(dq, dk, leaves["q"], leaves["k"], q_weight=leaves["q_weight"], k_weight=leaves["k_weight"], **how)
    g = torch.Generator().manual_seed(10)
    h = 1e-2
    for x in leaves:
        way = torch.randn(leaves[x].shape, generator=g).to(dev)
        slope = (value(**{x: leaves[x] + h * way}) - value(**{x: leaves[x] - h * way})) / (2 * h)
        size = float(b["d" + x].double().norm())
        # a third-order term of h^2 times some tens, and the rounding of the values over h
        assert abs(float((b["d" + x].double() * way.double()).sum()) - slope) <= 4e-2 * size, x


# ---- attention through a window ------------------------------------------------------------------------------

def bucket(dist, n_buckets, max_distance, causal):
    n = n_buckets if causal else n_buckets // 2
    base = n if not causal and dist > 0 else 0
    far = max(0, -dist) if causal else abs(dist)
    s = n // 2
    if far < s:
        return base + far
    return base + s + sum(far ** (n - s) >= s ** (n - s - i) * max_distance ** i for i in range(1, n - s))


def seen_by(lq, lk, causal, before, after, sinks, keep):
    p, j = torch.arange(lq)[:, None] + lk - lq, torch.arange(lk)[None]
    seen = ((j >= p - before) & (j <= p + after)) | (j < sinks)
    if causal:
        seen &= j <= p
    return seen if keep is None else seen & keep.cpu().bool()


def window_reference(p, ql, kl, dtype, causal, window, sinks, max_distance=128):
    """Outputs, gradients and the bounds of both, in 64 bits on the CPU: of bf16, probabilities and their gradients are rounded as
    operands, as results are."""
    u = U["bf16"] if dtype == "bf16" else 0.0
    q, k, v, dout = (p[x].detach().double().cpu() for x in ("q", "k", "v", "dout"))
    H, Hk, d = q.shape[1], k.shape[1], q.shape[2]
    scale = 1.0 / math.sqrt(d)
    table = None if p["bias"] is None else p["bias"].double().cpu()
    r = {x: torch.zeros_like(y) for x, y in (("out", q), ("dq", q), ("dk", k), ("dv", k))}
    r |= {x + "_tol": torch.zeros_like(y) for x, y in list(r.items())}
    r["lse"] = torch.full((H, q.shape[0]), -math.inf, dtype=torch.float64)
    if table is not None:
        r["dbias"], r["dbias_tol"] = torch.zeros_like(table), torch.zeros_like(table)
    qo, ko = offsets(ql).tolist(), offsets(kl).tolist()
    for s, (lq, lk) in enumerate(zip(ql, kl)):
        if lq == 0 or lk == 0:
            continue
        a, x = slice(qo[s], qo[s + 1]), slice(ko[s], ko[s + 1])
        seen = seen_by(lq, lk, causal, *window, sinks, None if p["keep"] is None else p["keep"][x])
        dist = torch.arange(lk) - (torch.arange(lq)[:, None] + lk - lq)
        if table is not None:
            of = torch.tensor([bucket(t, table.shape[0], max_distance, causal) for t in range(-lk - lq, lk + lq + 1)])
            at = of[dist + lk + lq]
        kept = torch.ones(lk, 1, dtype=torch.bool) if p["keep"] is None else p["keep"][x].cpu()[:, None]
        rows = seen.any(1)[:, None]
        for h in range(H):
            g = h // (H // Hk)
            K, V = torch.where(kept, k[x, g], 0.0), torch.where(kept, v[x, g], 0.0)
            Q, G = torch.where(rows, q[a, h], 0.0), torch.where(rows, dout[a, h], 0.0)
            S = Q @ K.T * scale
            if table is not None:
                S = S + table[at, h]
            S[~seen] = -math.inf
            lse = torch.logsumexp(S, 1)
            P = torch.exp(S - torch.where(lse == -math.inf, 0.0, lse)[:, None])
            O, spread = P @ V, P @ V.abs()
            r["out"][a, h], r["lse"][h, a] = O, lse
            r["out_tol"][a, h] = u * (spread + O.abs()) + F * spread
            dP = G @ V.T
            E = P * (dP - (G * O).sum(1, keepdim=True))
            d_delta = (G.abs() * ((u + F) * spread + u * O.abs())).sum(1, keepdim=True)
            rough = P * (G.abs() @ V.abs().T + (G.abs() * spread).sum(1, keepdim=True))
            e_tol = P * d_delta + F * rough
            r["dq"][a, h] = E @ K * scale
            r["dq_tol"][a, h] = scale * ((u * E.abs() + e_tol) @ K.abs()) + u * (E @ K * scale).abs()
            r["dk"][x, g] += E.T @ Q * scale
            r["dk_tol"][x, g] += scale * ((u * E.abs() + e_tol).T @ Q.abs())
            r["dv"][x, g] += P.T @ G
            r["dv_tol"][x, g] += (u + F) * (P.T @ G.abs())
            if table is not None:
                r["dbias"][:, h].index_add_(0, at.reshape(-1), E.reshape(-1))
                r["dbias_tol"][:, h].index_add_(0, at.reshape(-1), e_tol.reshape(-1))
    r["dk_tol"] += u * r["dk"].abs()
    r["dv_tol"] += u * r["dv"].abs()
    if table is not None:
        r["dbias_tol"] += u * r["dbias"].abs()
    return r


def window_problem(dev, dtype, ql, kl, H, Hk, d, seed=0, bias=None, keep=False):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    p = dict(q=n(sum(ql), H, d), k=n(sum(kl), Hk, d), v=n(sum(kl), Hk, d), dout=n(sum(ql), H, d) * 0.1)
    p = {x: t.to(DT[dtype]).to(dev) for x, t in p.items()}
    p["bias"] = None if bias is None else n(bias, H).to(DT[dtype]).to(dev)
    p["keep"] = None
    if keep:
        m = torch.rand(sum(kl), generator=g) >= 0.25
        ko = offsets(kl)
        m[ko[0]:ko[1]] = False
        p["keep"] = m.to(dev)
    return p


def attend(tr, p, ql, kl, causal, window, sinks):
    qo, ko = offsets(ql).to(p["q"].device), offsets(kl).to(p["q"].device)
    how = dict(causal=causal, keep=p["keep"], bias=p["bias"], window=window, sinks=sinks)
    f = tr.colbandit_attention(p["q"], p["k"], p["v"], qo, ko, **how)
    b = tr.colbandit_attention_backward(p["dout"], p["q"], p["k"], p["v"], f["out"], f["lse"], qo, ko, **how)
    torch.cuda.synchronize()
    return f, b


def check_window(tr, p, ql, kl, dtype, causal, window, sinks):
    f, b = attend(tr, p, ql, kl, causal, window, sinks)
    r = window_reference(p, ql, kl, dtype, causal, window, sinks)
    lse = f["lse"].double().cpu()
    assert torch.equal(lse == -math.inf, r["lse"] == -math.inf)
    fine = r["lse"] > -math.inf
    assert float((lse - r["lse"])[fine].abs().max() if fine.any() else 0.0) <= F * 2
    assert bool((f["out"].double().cpu()[~fine.T] == 0).all())
    more = lambda t: 1.05 * t + 1e-9  # noqa: E731
    within(f["out"], r["out"], more(r["out_tol"]), "out")
    for x in ("dq", "dk", "dv") + (() if p["bias"] is None else ("dbias",)):
        within(b[x], r[x], more(r[x + "_tol"]), x)
    return f, b


EDGES = [1, 2, 31, 32, 33, 64, 65, 127, 129, 200]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("causal,bias,keep,window,sinks", [
    (True, None, False, (31, 0), 0), (False, None, True, (0, 0), 0), (False, 32, False, (10, 33), 3), (True, 32, True, (64, 9), 70),
    (False, None, False, (300, 5), 1), (True, None, True, (1, 0), 150)])
def test_windows_at_the_edges_of_tiles(tr, dev, dtype, d, causal, bias, keep, window, sinks):
    p = window_problem(dev, dtype, EDGES, EDGES, 2, 2, d, seed=1, bias=bias, keep=keep)
    check_window(tr, p, EDGES, EDGES, dtype, causal, window, sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,Hk", [(64, 6, 3), (128, 8, 2), (32, 7, 1), (96, 20, 1)])
@pytest.mark.parametrize("causal,window,sinks", [(True, (47, 0), 5), (False, (3, 40), 0), (False, (130, 0), 40)])
def test_windows_of_heads_that_share_keys(tr, dev, dtype, d, H, Hk, causal, window, sinks):
    ql = [3, 0, 150, 70]
    check_window(tr, window_problem(dev, dtype, ql, ql, H, Hk, d, seed=2), ql, ql, dtype, causal, window, sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("window,sinks,bias", [((20, 0), 4, None), ((0, 7), 0, 8), ((5, 5), 129, None)])
def test_windows_over_queries_and_keys_of_different_lengths(tr, dev, dtype, causal, window, sinks, bias):
    """Few rows at the end of many keys, and rows that stand before the first key."""
    ql, kl = [1, 5, 200, 40, 0, 3, 130], [300, 5, 60, 0, 9, 1000, 131]
    p = window_problem(dev, dtype, ql, kl, 4, 2, 64, seed=3, bias=bias)
    check_window(tr, p, ql, kl, dtype, causal, window, sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal,window,sinks,keep", [(True, (255, 0), 4, False), (False, (64, 64), 1, True), (False, (700, 3), 33, False)])
def test_windows_in_long_sequences(tr, dev, dtype, causal, window, sinks, keep):
    """More than one workgroup's rows for the first keys."""
    ql = [1500, 513, 512]
    p = window_problem(dev, dtype, ql, ql, 2, 1, 64, seed=4, keep=keep)
    check_window(tr, p, ql, ql, dtype, causal, window, sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql", [[513, 512, 514, 511], [1, 600, 2, 1100, 0, 513], [700, 700]])
def test_first_keys_of_sequences_of_several_chunks(tr, dev, dtype, ql):
    """Chunks of 256 rows: sequences of two, of three, and of a row more, one after the other."""
    kl = [n + 3 for n in ql]
    p = window_problem(dev, dtype, ql, kl, 2, 2, 32, seed=14)
    check_window(tr, p, ql, kl, dtype, False, (3, 2), 5)


@gpu
@pytest.mark.parametrize("dtype,d,sinks,rows", [("bf16", 128, 64, 128), ("bf16", 96, 5, 128), ("f32", 128, 5, 256), ("bf16", 64, 3, 256),
                                                ("bf16", 128, 65, 256), ("bf16", 64, 257, 512), ("f32", 64, 256, 256)])
@pytest.mark.parametrize("causal", [True, False])
def test_first_keys_at_the_edges_of_chunks(tr, dev, dtype, d, sinks, rows, causal):
    """Rows that one workgroup adds up for the first keys: as many, one less and more, twice as many, none and one."""
    ql = [rows, rows + 1, 0, rows - 1, 2 * rows, 2 * rows + 1, 1, rows]
    p = window_problem(dev, dtype, ql, ql, 2, 1, d, seed=19)
    check_window(tr, p, ql, ql, dtype, causal, (7, 5), sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,sinks,keep", [(32, 0, False), (64, 5, True), (96, 300, False), (128, 3, False)])
def test_long_sums_of_heads_that_share_keys(tr, dev, dtype, d, sinks, keep):
    """Keys that more than a thousand rows see, those of all heads together, some of them by a whole multiple of that."""
    ql = [640, 385, 1, 256, 128]
    p = window_problem(dev, dtype, ql, ql, 16, 2, d, seed=23, keep=keep)
    check_window(tr, p, ql, ql, dtype, True, (255, 0), sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,Hk,keep", [(128, 8, 2, False), (64, 4, 4, True)])
@pytest.mark.parametrize("window,sinks", [((1023, 0), 4), ((3, 0), 0), ((100000, 0), 0)])
def test_single_tokens_through_a_window(tr, dev, dtype, d, H, Hk, keep, window, sinks):
    ql, kl = [1] * 6, [1, 5000, 1024, 1025, 3, 2600]
    p = window_problem(dev, dtype, ql, kl, H, Hk, d, seed=5, keep=keep)
    check_window(tr, p, ql, kl, dtype, True, window, sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
def test_a_window_over_everything_is_no_window(tr, dev, dtype, causal):
    """Windows beyond every sequence, and first keys that are all of them."""
    ql = [180, 32, 77, 515]
    p = window_problem(dev, dtype, ql, ql, 4, 2, 64, seed=6, keep=True)
    off = offsets(ql).to(dev)
    f = tr.colbandit_attention(p["q"], p["k"], p["v"], off, causal=causal, keep=p["keep"])
    for window, sinks in (((1 << 62, 1 << 40), 0), ((600, 600), 7), ((0, 0), 600)):
        g, _ = check_window(tr, p, ql, ql, dtype, causal, window, sinks)
        assert float((g["out"].float() - f["out"].float()).abs().max()) <= 2 * U[dtype] * 4 + 1e-4
    wide = tr.colbandit_attention(p["q"], p["k"], p["v"], off, causal=causal, keep=p["keep"], window=(1 << 70, 1 << 64))
    whole = tr.colbandit_attention(p["q"], p["k"], p["v"], off, causal=causal, keep=p["keep"], window=(1 << 62, 1 << 62))
    assert torch.equal(wide["out"], whole["out"]) and torch.equal(wide["lse"], whole["lse"])


@gpu
@pytest.mark.parametrize("wild", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_keys_in_windows_may_hold_anything(tr, dev, dtype, wild):
    ql = [90, 33, 200]
    p = window_problem(dev, dtype, ql, ql, 2, 2, 64, seed=7, keep=True)
    p["k"][~p["keep"]] = p["v"][~p["keep"]] = wild
    p["q"][:90] = p["dout"][:90] = wild               # a sequence whose rows see nothing
    check_window(tr, p, ql, ql, dtype, True, (16, 0), 40)
    check_window(tr, p, ql, ql, dtype, False, (2, 5), 3)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("more", [1, 64, 333])
def test_rows_behind_the_last_sequence_of_a_window_get_zeros(tr, dev, dtype, more):
    ql = [40, 3, 129]
    p = window_problem(dev, dtype, [sum(ql) + more], [sum(ql) + more], 4, 2, 64, seed=8)
    off = offsets(ql).to(dev)
    n = sum(ql)
    for t in ("q", "k", "v", "dout"):
        p[t][n:] = math.nan
    how = dict(causal=True, window=(20, 0), sinks=30)
    f = tr.colbandit_attention(p["q"], p["k"], p["v"], off, **how)
    b = tr.colbandit_attention_backward(p["dout"], p["q"], p["k"], p["v"], f["out"], f["lse"], off, **how)
    part = {x: (y[:n] if y is not None else None) for x, y in p.items()}
    g, c = check_window(tr, part, ql, ql, dtype, True, (20, 0), 30)
    assert bool((f["lse"][:, n:] == -math.inf).all()) and torch.equal(f["out"][:n], g["out"])
    for x, y in ((f["out"], g["out"]), (b["dq"], c["dq"]), (b["dk"], c["dk"]), (b["dv"], c["dv"])):
        assert not bool(x[n:].any()) and torch.equal(x[:n], y)


@gpu
@pytest.mark.parametrize("wild", [[0, 1 << 40, 90], [-7, 50, 1 << 40], [80, 20, 60], [0, 0, 0]])
def test_offsets_that_are_none_stay_in_bounds_through_a_window(tr, dev, wild):
    p = window_problem(dev, "bf16", [90], [90], 4, 2, 64, seed=9)
    off = torch.tensor(wild, device=dev)
    how = dict(window=(5, 9), sinks=40)
    f = tr.colbandit_attention(p["q"], p["k"], p["v"], off, **how)
    tr.colbandit_attention_backward(p["dout"], p["q"], p["k"], p["v"], f["out"], f["lse"], off, **how)
    torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("bias,sinks", [(32, 0), (None, 9)])
def test_windows_in_graphs_and_as_part_of_a_program(tr, dev, bias, sinks):
    ql = [180, 32, 1030]
    p = window_problem(dev, "bf16", ql, ql, 4, 4, 64, seed=10, bias=bias, keep=True)
    off = offsets(ql).to(dev)
    how = dict(keep=p["keep"], bias=p["bias"], window=(40, 17), sinks=sinks)

    def call():
        f = tr.colbandit_attention(p["q"], p["k"], p["v"], off, **how)
        b = tr.colbandit_attention_backward(p["dout"], p["q"], p["k"], p["v"], f["out"], f["lse"], off, **how)
        return f | {x: y for x, y in b.items() if y is not None}

    captured(dev, call)
    leaves = [p[x].clone().requires_grad_() for x in ("q", "k", "v")]
    out = tr.attention(*leaves, off, keep=p["keep"], bias=p["bias"], window=(40, 17), sinks=sinks)
    out.backward(p["dout"])
    want = call()
    assert torch.equal(out, want["out"]) and all(torch.equal(t.grad, want["d" + x]) for t, x in zip(leaves, "qkv"))


def two_heads_a_workgroup(ql, kl, heads, kv_heads, bias, window, sinks):
    """Whether the plan's workgroups go on to a second head through a window: units (key heads) in pairs leave 1,536 workgroups or
    more, and a tile of 128 sees up to 384 rows; for the queries' tiles and for the keys'.  (Heads of up to 64.)"""
    n, group, span = len(ql), heads // kv_heads, sum(window) + 128
    pack = 1 if bias or group > 16 else group
    units, q_slots, k_slots = heads // pack, sum(ql) // (128 // pack) + n, sum(kl) // 128 + n
    k_rows, q_rows = min(span + sinks, sum(kl) // n), min(span * group, sum(ql) * group // n)
    return k_rows <= 384 and units > 1 and q_slots * (units // 2) >= 1536, q_rows <= 384 and kv_heads > 1 and k_slots * (kv_heads // 2) >= 1536


@gpu
@pytest.mark.parametrize("dtype,d,H", [("bf16", 64, 25), ("bf16", 32, 24), ("f32", 64, 24), ("f32", 32, 25)])
@pytest.mark.parametrize("causal,bias,keep,window,sinks", [
    (False, None, False, (64, 64), 1), (True, None, True, (47, 0), 0), (False, 32, True, (20, 33), 0), (True, 32, False, (90, 0), 130)])
def test_two_heads_a_workgroup_through_a_window(tr, dev, dtype, d, H, causal, bias, keep, window, sinks):
    """Sequences of 1 to 180 rows; with an odd number of heads the last workgroup of a tile has one."""
    lengths = [1 + i * 179 // 127 for i in range(128)]
    assert two_heads_a_workgroup(lengths, lengths, H, H, bias, window, sinks) == (True, True)
    p = window_problem(dev, dtype, lengths, lengths, H, H, d, seed=31, bias=bias, keep=keep)
    check_window(tr, p, lengths, lengths, dtype, causal, window, sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,sinks,keep", [(64, 0, False), (32, 5, True), (64, 5, False)])
def test_two_heads_a_workgroup_with_long_sums(tr, dev, dtype, d, sinks, keep):
    """Many short sequences and a long one, whose keys more than a thousand rows of the heads that share them see: the second key
    head of a workgroup begins its sums anew.  Five heads to a key head: so are the first keys' sums."""
    lengths = (np.random.default_rng(33).integers(0, 5, 1540).tolist()) + [900]
    assert two_heads_a_workgroup(lengths, lengths, 10, 2, None, (700, 300), sinks)[1]
    p = window_problem(dev, dtype, lengths, lengths, 10, 2, d, seed=32, keep=keep)
    check_window(tr, p, lengths, lengths, dtype, False, (700, 300), sinks)


def check_far_window(tr, p, ql, kl, dtype, causal, window, sinks, scale=None, like=None, by=1.0, lse_of=lambda x: x):
    """All results of rows whose log-sum-exp may be of any size: it has a 32-bit value's own rounding, and as much again for the
    product that it is the sum of.  The reference's probabilities are exp(S - lse), which in 64 bits lose a sum's logarithm too
    where lse is that large: it is then given a problem of the same probabilities (`like`: other inputs, q divided by `by`, a power
    of two, which is what the keys' gradient differs by), and `lse_of` its log-sum-exp.  A scale is its queries' factor."""
    qo, ko = offsets(ql).to(p["q"].device), offsets(kl).to(p["q"].device)
    how = dict(causal=causal, keep=p["keep"], bias=p["bias"], window=window, sinks=sinks, scale=scale)
    f = tr.colbandit_attention(p["q"], p["k"], p["v"], qo, ko, **how)
    b = tr.colbandit_attention_backward(p["dout"], p["q"], p["k"], p["v"], f["out"], f["lse"], qo, ko, **how)
    torch.cuda.synchronize()
    a = dict(p, **(like or {}))
    factor = 1.0 if scale is None else float(np.float32(scale)) * math.sqrt(p["q"].shape[2])
    if scale is not None:
        a["q"] = a["q"].double() * factor
    r = window_reference(a, ql, kl, dtype, causal, window, sinks)
    r["dq"], r["dq_tol"] = r["dq"] * factor, r["dq_tol"] * abs(factor)
    r["dk"], r["dk_tol"] = r["dk"] * by, r["dk_tol"] * by
    r["lse"] = torch.where(r["lse"] == -math.inf, r["lse"], lse_of(r["lse"]))
    lse = f["lse"].double().cpu()
    assert torch.equal(lse == -math.inf, r["lse"] == -math.inf)
    fine = r["lse"] > -math.inf
    assert bool(((lse - r["lse"]).abs() <= F * 2 + 2.0 ** -22 * r["lse"].abs())[fine].all())
    more = lambda t: 1.05 * t + 1e-9  # noqa: E731
    within(f["out"], r["out"], more(r["out_tol"]), "out")
    for x in ("dq", "dk", "dv") + (() if p["bias"] is None else ("dbias",)):
        within(b[x], r[x], more(r[x + "_tol"]), x)


LOWEST = {"bf16": torch.finfo(torch.bfloat16).min, "f32": torch.finfo(torch.float32).min}


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("causal,window,sinks", [(True, (3, 0), 0), (False, (0, 0), 0), (False, (2, 40), 1), (True, (64, 0), 3)])
@pytest.mark.parametrize("low", [-1e4, -1e30, "lowest", -math.inf])
def test_rows_that_see_a_hidden_distance_through_a_window(tr, dev, dtype, d, causal, window, sinks, low):
    """A bucket of the table hides distance 0: of rows that see only this one, and beside others.  With minus infinity the former see
    nothing."""
    lengths = [50, 1, 133, 1]
    p = window_problem(dev, dtype, lengths, lengths, 2, 2, d, seed=33, bias=8)
    p["bias"][0] = LOWEST[dtype] if low == "lowest" else low
    check_far_window(tr, p, lengths, lengths, dtype, causal, window, sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ql,kl,window,sinks", [([150, 1, 70], [150, 1, 70], (31, 20), 5), ([1, 3], [5000, 700], (1023, 0), 4)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("value", ["lowest", -1e30, 1e30])
def test_tables_far_from_zero_through_a_window(tr, dev, dtype, d, ql, kl, window, sinks, causal, value):
    """Products are below such a bias' rounding in 64 bits as well: all keys that are seen weigh the same, in one part or several."""
    p = window_problem(dev, dtype, ql, kl, 2, 2, d, seed=34, bias=32, keep=True)
    p["bias"][:] = LOWEST[dtype] if value == "lowest" else value
    at, tiny = float(p["bias"][0, 0].double()), 2.0 ** -40
    check_far_window(tr, p, ql, kl, dtype, causal, window, sinks, like=dict(q=p["q"].double() * tiny, bias=torch.zeros_like(p["bias"])),
                     by=1 / tiny, lse_of=lambda x: x + at)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,heads,kv_heads", [(64, 4, 4), (128, 4, 2), (96, 3, 1)])
@pytest.mark.parametrize("ql,kl,window,sinks", [([150, 3, 70], [150, 3, 70], (40, 9), 2), ([40, 1], [1100, 900], (600, 0), 70)])
@pytest.mark.parametrize("causal", [False, True])
def test_rows_on_both_sides_of_where_they_are_normalised_again_through_a_window(tr, dev, monkeypatch, dtype, d, heads, kv_heads, ql, kl,
                                                                                window, sinks, causal):
    """Ordinary rows with biases that move them to 240 and to 280: log-sum-exps below and above 256 in one call.  Scores of up to 290
    carry nine times the error of the file's bound, which is for up to 32."""
    monkeypatch.setitem(globals(), "F", F * 290 / 32)
    p = window_problem(dev, dtype, ql, kl, heads, kv_heads, d, seed=35, bias=32, keep=True)
    p["bias"] += torch.tensor([240.0, 280.0], device=dev).repeat(2)[:heads].to(DT[dtype])
    check_far_window(tr, p, ql, kl, dtype, causal, window, sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head", [0, 1, 2])
@pytest.mark.parametrize("d,causal,window,sinks", [(64, True, (2, 0), 0), (32, False, (0, 1), 1)])
def test_one_head_of_several_is_far_from_zero_through_a_window(tr, dev, dtype, head, d, causal, window, sinks):
    """Workgroups that go on from a head whose rows see nothing but a hidden distance to one whose do not, and the other way."""
    lengths = np.random.default_rng(43).integers(0, 4, 1600).tolist()
    assert two_heads_a_workgroup(lengths, lengths, 3, 3, 8, window, sinks) == (True, True)
    p = window_problem(dev, dtype, lengths, lengths, 3, 3, d, seed=36, bias=8)
    p["bias"][0, head] = LOWEST[dtype]
    check_far_window(tr, p, lengths, lengths, dtype, causal, window, sinks)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [None, 32])
@pytest.mark.parametrize("scale", [0.0, -0.125, -3e-3])
@pytest.mark.parametrize("d,heads,kv_heads,ql,kl", [(64, 2, 1, [150, 1, 70], [150, 1, 70]), (128, 4, 2, [90, 33], [90, 33]), (128, 2, 2, [1, 2], [3000, 400])])
def test_scales_of_zero_and_below_through_a_window(tr, dev, dtype, bias, scale, d, heads, kv_heads, ql, kl):
    p = window_problem(dev, dtype, ql, kl, heads, kv_heads, d, seed=37, bias=bias)
    check_far_window(tr, p, ql, kl, dtype, True, (300, 0), 5, scale=scale)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,causal,window,sinks", [(128, True, (1023, 0), 4), (64, False, (2000, 2000), 0)])
def test_single_tokens_with_a_bias_through_a_window(tr, dev, dtype, d, causal, window, sinks):
    """Keys in several parts."""
    ql, kl = [1] * 6, [1, 5000, 1024, 1025, 3, 2600]
    p = window_problem(dev, dtype, ql, kl, 3, 3, d, seed=38, bias=32, keep=True)
    check_window(tr, p, ql, kl, dtype, causal, window, sinks)


# ---- orthogonalised updates ------------------------------------------------------------------------------------

POLYNOMIAL = (3.4445, -4.7750, 2.0315)


def polynomial_steps(g, steps, k, dtype):
    a, b, c = k
    x = g.to(dtype)
    x = x if g.shape[0] <= g.shape[1] else x.T
    x = x / x.double().norm().clamp(min=1e-300).to(dtype)
    for _ in range(steps):
        A = x @ x.T
        x = a * x + (b * A + c * (A @ A)) @ x
    return x if g.shape[0] <= g.shape[1] else x.T


def check_orthogonal(matrices, out, steps=5, k=POLYNOMIAL):
    """Pieces hold 22 bits of a value where 32-bit arithmetic holds 24, so the steps' error is at most four times that of the same
    steps in plain 32-bit products; results are rounded once."""
    for g, o in zip(matrices, out):
        g = g.detach().cpu()
        k32 = [float(np.float32(x)) for x in k]
        want = polynomial_steps(g.double(), steps, k32, torch.float64)
        plain = float((polynomial_steps(g.float(), steps, k32, torch.float32).double() - want).norm())
        size = float(want.norm())
        tol = 4 * plain + 4 * steps * E32 * size + (U["bf16"] if g.dtype == torch.bfloat16 else E32) * size
        got = o.detach().double().cpu()
        assert got.shape == want.shape and bool(torch.isfinite(got).all())
        assert float((got - want).norm()) <= tol, (tuple(g.shape), float((got - want).norm()), tol, size)


def updates(shapes, dtype, dev, seed=0, rank=None, noise=1.0):
    g = torch.Generator().manual_seed(seed)
    r = []
    for i, (m, n) in enumerate(shapes):
        few = min(16 if rank is None else rank, m, n)
        x = (torch.randn(m, few, generator=g) * torch.logspace(0, -1, few)) @ torch.randn(few, n, generator=g)
        r.append(((x + noise * torch.randn(m, n, generator=g)) * 10.0 ** (i % 5 - 3)).to(DT[dtype]).to(dev))
    return r


SHAPES = [(1, 1), (1, 77), (77, 1), (2, 3), (31, 33), (64, 64), (65, 63), (64, 65), (96, 255), (128, 300), (300, 129), (256, 256), (17, 1000)]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matrices_of_many_shapes_are_orthogonalised_together(tr, dev, dtype):
    m = updates(SHAPES, dtype, dev)
    out = tr.colbandit_orthogonalise(m)["out"]
    torch.cuda.synchronize()
    check_orthogonal(m, out)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matrices_of_large_tiles(tr, dev, dtype):
    """Enough of them that tiles are of 128, among them one smaller than a tile and one with a row more."""
    m = updates([(384, 400)] * 37 + [(5, 9), (385, 700), (640, 129)], dtype, dev, seed=1)
    out = tr.colbandit_orthogonalise(m)["out"]
    torch.cuda.synchronize()
    check_orthogonal(m[::9] + m[-3:], out[::9] + out[-3:])
    assert all(torch.equal(a, b) for a, b in zip(out[30:], tr.colbandit_orthogonalise(m[30:] + m[:30])["out"]))


@gpu
def test_more_matrices_than_one_launch_takes(tr, dev):
    m = updates([(8, 24), (30, 7)] * 50, "f32", dev, seed=2)
    out = tr.colbandit_orthogonalise(m)["out"]
    torch.cuda.synchronize()
    check_orthogonal(m, out)


@gpu
@pytest.mark.parametrize("steps,k", [(1, POLYNOMIAL), (2, POLYNOMIAL), (12, (1.875, -1.25, 0.375)), (3, (1.5, -0.5, 0.0)), (2, (-1.0, 0.0, 0.0)), (64, (1.5, -0.5, 0.0))])
def test_other_polynomials_and_steps(tr, dev, steps, k):
    m = updates([(40, 60), (70, 50)], "f32", dev, seed=3)
    out = tr.colbandit_orthogonalise(m, steps=steps, coefficients=k)["out"]
    check_orthogonal(m, out, steps, k)


@gpu
def test_singular_values_come_near_to_one(tr, dev):
    g = torch.Generator().manual_seed(4)
    m = [torch.randn(100, 200, generator=g).to(dev), torch.randn(130, 90, generator=g).to(dev)]
    for x in tr.colbandit_orthogonalise(m)["out"]:
        s = torch.linalg.svdvals(x.double().cpu())
        assert 0.6 <= float(s.min()) and float(s.max()) <= 1.3
    for x in tr.colbandit_orthogonalise(m, steps=15, coefficients=(1.875, -1.25, 0.375))["out"]:
        s = torch.linalg.svdvals(x.double().cpu())
        assert float((s - 1).abs().max()) <= 1e-4


@gpu
@pytest.mark.parametrize("rank,noise", [(1, 0.0), (3, 1e-4)])
def test_matrices_of_low_rank(tr, dev, rank, noise):
    m = updates([(60, 200), (128, 128)], "f32", dev, seed=5, rank=rank, noise=noise)
    check_orthogonal(m, tr.colbandit_orthogonalise(m)["out"])


def graded(kind, by, shape, seed=9):
    """Rows or columns that fall to 10^-by of the first, or one row and others that are all that small."""
    x = torch.randn(shape, generator=torch.Generator().manual_seed(seed))
    if kind == "one":
        x[1:] *= 10.0 ** -by
        return x
    n = shape[0 if kind == "rows" else 1]
    fall = torch.logspace(0, -by, n)
    return x * (fall[:, None] if kind == "rows" else fall)


@gpu
@pytest.mark.parametrize("kind,by", [("rows", 6), ("rows", 8), ("rows", 10), ("columns", 6), ("columns", 10), ("one", 4), ("one", 8)])
@pytest.mark.parametrize("steps,k", [(5, POLYNOMIAL), (6, POLYNOMIAL), (8, POLYNOMIAL), (12, POLYNOMIAL), (20, POLYNOMIAL),
                                     (12, (1.875, -1.25, 0.375)), (64, (1.5, -0.5, 0.0))])
def test_graded_matrices(tr, dev, kind, by, steps, k):
    """What is small beside a matrix' norm counts as much as the rest once enough steps have raised it."""
    m = [graded(kind, by, shape).to(dev) for shape in ((128, 512), (300, 129), (64, 70))]
    out = tr.colbandit_orthogonalise(m, steps=steps, coefficients=k)["out"]
    check_orthogonal(m, out, steps, k)


def rows_are_right(g, o, steps, k):
    """Each row on its own: 32-bit values and sums, whose products lose 2^-26, are off by what plain 32-bit products are off by."""
    g, o = g.cpu(), o.double().cpu()
    k32 = [float(np.float32(x)) for x in k]
    want = polynomial_steps(g.double(), steps, k32, torch.float64)
    plain = ((polynomial_steps(g.float(), steps, k32, torch.float32).double() - want).norm(dim=1) / want.norm(dim=1)).max()
    assert float(((o - want).norm(dim=1) / want.norm(dim=1)).max()) <= 4 * float(plain) + 4 * steps * E32


@gpu
@pytest.mark.parametrize("kind,by", [("rows", 8), ("columns", 8), ("one", 8)])
@pytest.mark.parametrize("steps,k", [(12, POLYNOMIAL), (64, (1.5, -0.5, 0.0)), (5, (0.5, 0.0, 0.0)), (40, (0.6, 0.2, 0.0))])
def test_rows_of_graded_matrices(tr, dev, kind, by, steps, k):
    """Where steps raise what is small far, or make all of a matrix small, values are held in 32 bits."""
    for shape in ((128, 512), (300, 129)):
        m = graded(kind, by, shape).to(dev)
        rows_are_right(m, tr.colbandit_orthogonalise([m], steps=steps, coefficients=k)["out"][0], steps, k)


@gpu
@pytest.mark.parametrize("dtype,steps", [("bf16", 5), ("f32", 5), ("f32", 9)])
def test_matrices_with_long_sides(tr, dev, dtype, steps):
    """Sides above 1,000, tiles of 64 and, with enough of them, of 128: pieces and, of nine steps, 32 bits."""
    m = updates([(1030, 1100), (33, 5000), (2100, 70)], dtype, dev, seed=10)
    check_orthogonal(m, tr.colbandit_orthogonalise(m, steps=steps)["out"], steps)
    m += updates([(1030, 1029)] * 6, dtype, dev, seed=11)
    out = tr.colbandit_orthogonalise(m, steps=steps)["out"]
    check_orthogonal(m[:4], out[:4], steps)


@gpu
def test_extreme_matrices(tr, dev):
    """Zeros stay zeros, any finite size is normalised, what is not finite is NaN, and neither touches the others of the list."""
    base = updates([(40, 50)], "f32", dev, seed=6)[0]
    bad = base.clone()
    bad[3, 4] = math.inf
    nan = base.clone()
    nan[39, 49] = math.nan
    big, small = base / base.abs().max() * 3e38, base * 1e-38
    out = tr.colbandit_orthogonalise([base, torch.zeros_like(base), bad, big, nan, small, base[:0], base[:, :0].contiguous()])["out"]
    want = tr.colbandit_orthogonalise([base])["out"][0]
    assert torch.equal(out[0], want) and not bool(out[1].any()) and bool(out[2].isnan().all()) and bool(out[4].isnan().all())
    check_orthogonal([big, small], [out[3], out[5]])
    assert out[6].shape == (0, 50) and out[7].shape == (40, 0)


@gpu
def test_extreme_matrices_of_many_steps(tr, dev):
    """The same of values that are held in 32 bits, and in place, in a graph and on another stream."""
    base = updates([(40, 50)], "f32", dev, seed=6)[0]
    bad, nan = base.clone(), base.clone()
    bad[3, 4], nan[39, 49] = -math.inf, math.nan
    big, small = base / base.abs().max() * 3e38, base * 1e-38
    m, how = [base, torch.zeros_like(base), bad, big, nan, small], dict(steps=12)
    out = tr.colbandit_orthogonalise(m, **how)["out"]
    assert torch.equal(out[0], tr.colbandit_orthogonalise([base], **how)["out"][0])
    assert not bool(out[1].any()) and bool(out[2].isnan().all()) and bool(out[4].isnan().all())
    check_orthogonal([base, big, small], [out[0], out[3], out[5]], 12)
    m = updates([(50, 90), (200, 64), (700, 720)], "bf16", dev, seed=7)
    want = tr.colbandit_orthogonalise(m, **how)["out"]
    copies = [x.clone() for x in m]
    tr.colbandit_orthogonalise(copies, out=copies, **how)
    assert all(torch.equal(a, b) for a, b in zip(copies, want))
    captured(dev, lambda: dict(enumerate(tr.colbandit_orthogonalise(m, **how)["out"])))


@gpu
def test_orthogonalising_in_place_in_graphs_and_steps(tr, dev):
    m = updates([(50, 90), (200, 64), (64, 64)], "bf16", dev, seed=7)
    want = tr.colbandit_orthogonalise(m)["out"]
    copies = [x.clone() for x in m]
    tr.colbandit_orthogonalise(copies, out=copies)
    assert all(torch.equal(a, b) for a, b in zip(copies, want))
    captured(dev, lambda: dict(enumerate(tr.colbandit_orthogonalise(m)["out"])))
    p = [torch.nn.Parameter(torch.zeros(30, 20, device=dev)), torch.nn.Parameter(torch.zeros(20, 30, device=dev)),
         torch.nn.Parameter(torch.zeros(4, 4, device=dev))]
    momenta = {}
    with pytest.raises(ValueError, match="two-dimensional"):
        flat = torch.nn.Parameter(torch.zeros(4, device=dev))
        flat.grad = torch.ones(4, device=dev)
        p[0].grad = torch.ones(30, 20, device=dev)
        tr.orthogonal_step_([p[0], flat], momenta, rate=0.1)
    assert not momenta and not bool(p[0].any())
    empty = torch.nn.Parameter(torch.zeros(0, 4, device=dev))
    empty.grad = torch.zeros(0, 4, device=dev)
    tr.orthogonal_step_([empty], momenta, rate=0.1)
    grads = updates([(30, 20), (20, 30)], "f32", dev, seed=8)
    for _ in range(2):
        p[0].grad, p[1].grad = grads[0].clone(), grads[1].clone()
        tr.orthogonal_step_(p + p[:1], momenta, rate=0.1, momentum=0.5)
    assert not bool(p[2].any()) and p[2] not in momenta
    # momenta g and 1.5 g; the updates point the same way, and their sizes do not matter
    for x, g in zip(p[:2], grads):
        assert float((momenta[x] - 1.5 * g).abs().max()) <= 4 * E32 * float(g.abs().max())
        step = tr.colbandit_orthogonalise([g])["out"][0] * (-0.2 * math.sqrt(max(1.0, g.shape[0] / g.shape[1])))
        assert float((x.detach() - step).norm()) <= 1e-4 * float(step.norm())


@gpu
@pytest.mark.parametrize("bad", ["coefficients", "steps", "many", "size", "momentum", "sparse"])
def test_refused_steps_change_nothing(tr, dev, bad):
    """Neither momenta nor parameters, nor is a momentum made."""
    p = [torch.nn.Parameter(torch.randn(30, 20, device=dev)), torch.nn.Parameter(torch.randn(20, 30, device=dev))]
    for x in p:
        x.grad = torch.randn_like(x)
    momenta, how = {}, {}
    tr.orthogonal_step_(p[:1], momenta, rate=0.1)
    if bad == "coefficients":
        how = dict(coefficients=(5.0, 0.0, 0.0))
    elif bad in ("steps", "many"):
        how = dict(steps=0 if bad == "steps" else 65)
    elif bad == "size":
        p.append(torch.nn.Parameter(torch.zeros(16385, 16385, device=dev, dtype=torch.bfloat16)))
        p[-1].grad = torch.zeros_like(p[-1])
    elif bad == "momentum":
        momenta[p[1]] = torch.ones(30, 20, device=dev)
    else:
        p[1].grad = p[1].grad.to_sparse()
    before = {x: m.clone() for x, m in momenta.items()}
    values = [x.detach().clone() for x in p]
    with pytest.raises((ValueError, RuntimeError)):
        tr.orthogonal_step_(p, momenta, rate=0.1, **how)
    assert [id(x) for x in momenta] == [id(x) for x in before] and all(torch.equal(momenta[x], m) for x, m in before.items())
    assert all(torch.equal(x, y) for x, y in zip(p, values))


@gpu
def test_momenta_of_16_bit_parameters_are_32_bits(tr, dev):
    """A gradient of 2^-10 of the momentum, which 16 bits would leave out, counts in every step."""
    p = torch.nn.Parameter(torch.zeros(24, 40, device=dev, dtype=torch.bfloat16))
    momenta = {}
    for x in [1.0] + [2.0 ** -10] * 4:
        p.grad = torch.full_like(p, x)
        tr.orthogonal_step_([p], momenta, rate=0.1, momentum=1.0)
    assert momenta[p].dtype == torch.float32 and p.dtype == torch.bfloat16
    assert torch.equal(momenta[p], torch.full_like(momenta[p], 1.0 + 2.0 ** -8))
    assert bool((p < 0).all())


# ---- together --------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("positions", ["bias", "rotary"])
def test_an_encoder_of_all_of_them(tr, dev, positions):
    """The example with a window and orthogonalised updates runs, and the same seed gives the same steps."""
    from paper_2602_02827_amd import finetune

    def run():
        return finetune.train(steps=3, n_docs=48, batch=16, positions=positions, window=24, optimiser="orthogonal")

    a, b = run(), run()
    assert all(math.isfinite(x) for x in a["losses"] + a["norms"]) and a["losses"] == b["losses"] and a["norms"] == b["norms"]


@pytest.mark.parametrize("window", [None, 7])
@pytest.mark.parametrize("positions", ["bias", "rotary"])
def test_the_examples_encoder_says_what_it_means(tr, monkeypatch, positions, window):
    """What the example's encoder asks of the operators, by stand-ins: each row's place in its own sequence, empty ones among them, the
    window to both sides with the first key, the mask and the bias."""
    from paper_2602_02827_amd import finetune
    asked = {}

    def rotate(q, k, **how):
        asked.update(how)
        return q, k

    def attend(q, k, v, off, **how):
        asked.update(how, off=off)
        return v

    monkeypatch.setattr(tr, "embedding", lambda W, t: W[t])
    monkeypatch.setattr(tr, "norm_rotate", rotate)
    monkeypatch.setattr(tr, "attention", attend)
    encoder = finetune.Encoder(positions, window)
    lengths = [20, 0, 150, 1, 33]
    off, tokens = offsets(lengths), torch.randint(0, 2 * finetune.WORDS, (sum(lengths),), generator=torch.Generator().manual_seed(3))
    out = encoder(tokens, off)
    assert out.shape == (sum(lengths), finetune.EMBED) and asked["off"] is off
    assert torch.equal(asked["keep"], tokens >= finetune.PUNCTUATION)
    assert asked.get("window") == (None if window is None else (window, window)) and asked.get("sinks", 0) == (0 if window is None else 1)
    if positions == "rotary":
        assert torch.equal(asked["positions"], torch.cat([torch.arange(n) for n in lengths])) and asked["table"].shape[0] >= max(lengths)
        assert asked["q_weight"] is encoder.q_weight and asked["k_weight"] is encoder.k_weight and "bias" not in asked
    else:
        assert torch.equal(asked["bias"], encoder.bias.bfloat16()) and asked["max_distance"] == finetune.MAX_DISTANCE
    out.float().square().sum().backward()
    assert bool(encoder.tokens.grad.any()) and bool(encoder.qkv.weight.grad.any())


@gpu
def test_gradients_through_lookup_rotation_and_window(tr, dev):
    """Token table to attention's output and back, against the same by torch in 64 bits."""
    g = torch.Generator().manual_seed(11)
    lengths, H, d, vocab = [70, 1, 45], 2, 32, 30
    off = offsets(lengths)
    t = torch.randint(0, vocab, (sum(lengths),), generator=g)
    positions = torch.cat([torch.arange(n) for n in lengths])
    W = torch.randn(vocab, H * d, generator=g)
    M = torch.randn(H * d, 3 * H * d, generator=g) / math.sqrt(H * d)
    wq, wk = 1 + 0.1 * torch.randn(d, generator=g), 1 + 0.1 * torch.randn(d, generator=g)
    dout = torch.randn(sum(lengths), H, d, generator=g)
    table = tr.colbandit_rotary_table(70, d)
    ours = [x.to(dev).requires_grad_() for x in (W, M, wq, wk)]
    x = tr.embedding(ours[0], t.to(dev), scale=0.5)
    # (a product in full 32 bits, not in a shortened type)
    q, k, v = (x[:, :, None] * ours[1][None]).sum(1).view(-1, 3, H, d).unbind(1)
    q, k = tr.norm_rotate(q, k, positions=positions.to(dev), table=table, q_weight=ours[2], k_weight=ours[3])
    tr.attention(q, k, v, off.to(dev), window=(9, 4), sinks=2).backward(dout.to(dev))

    theirs = [x.double().requires_grad_() for x in (W, M, wq, wk)]
    x = theirs[0][t] * 0.5
    q, k, v = (x @ theirs[1]).view(-1, 3, H, d).unbind(1)
    cs = torch.view_as_complex(table.double().cpu())[positions][:, None]

    def turned(x, w):
        y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        z = torch.complex(y[..., :d // 2], y[..., d // 2:]) * cs
        return torch.cat([z.real, z.imag], -1)

    q, k = turned(q, theirs[2]), turned(k, theirs[3])
    out = []
    for a, b in zip(off[:-1].tolist(), off[1:].tolist()):
        S = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b]) / math.sqrt(d)
        S = S.masked_fill(~seen_by(b - a, b - a, False, 9, 4, 2, None), -math.inf)
        out.append(torch.einsum("hij,jhd->ihd", torch.softmax(S, -1), v[a:b]))
    torch.cat(out).backward(dout.double())
    for a, b in zip(ours, theirs):                    # a chain of some ten sums in 32 bits, each within F of its terms
        assert float((a.grad.double().cpu() - b.grad).norm()) <= 10 * F * float(b.grad.norm())


# ---- refusals --------------------------------------------------------------------------------------------------

def test_window_refusals(tr):
    """Nothing is ever launched: every case fails validation."""
    L = tr.lib()

    def struct(**kw):
        a = dict(dt=1, n_seqs=2, heads=4, kv_heads=2, d=64, causal=0, n_buckets=32, max_distance=128, scale=0.125, total_q=10, total_k=12,
                 q_offsets=0x1000, k_offsets=0x2000, q=0x3000, k=0x4000, v=0x5000, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128,
                 v_head=64, keep=None, bias=None)
        return tr.ColbanditAttn(**{**a, **kw})

    def forward(w=(1, 1, 1), out=0x10000, **kw):
        return L.colbandit_attention_window(struct(**kw), tr.ColbanditWindow(*w) if w else None, out, 0x20000, None, 0, None)

    def backward(w=(1, 1, 1), out=0x10000, ws=0x100000, nb=1 << 30, **kw):
        return L.colbandit_attention_window_backward(struct(**kw), tr.ColbanditWindow(*w) if w else None, out, 0x20000, 0x30000, 0x40000,
                                                     0x50000, 0x60000, None, ws, nb, None)

    for call in (forward, backward):
        assert call(w=None) == -1 and call(w=(-1, 0, 0)) == -2 and call(w=(0, -1, 0)) == -2 and call(w=(0, 0, -1)) == -2
        assert call(w=(0, 0, 1025)) == -4 and call(total_q=(1 << 28) + 1) == -4 and call(total_k=(1 << 28) + 1) == -4
        assert call(out=None) == -1 and call(q=None) == -1 and call(d=48) == -4 and call(heads=5) == -2 and call(scale=math.nan) == -3
        assert call(q=0x3008) == -6
    assert backward(ws=None) == -1 and backward(ws=0x100010) == -6 and backward(nb=16) == -5
    # a launch of 2^32 threads for the first keys
    assert backward(w=(1, 1, 1024), n_seqs=1 << 20, kv_heads=4, nb=1 << 62) == -4
    assert L.colbandit_attention_window_workspace_bytes(struct(d=48), tr.ColbanditWindow(1, 1, 1), 1) == 0
    assert L.colbandit_attention_window_workspace_bytes(struct(), tr.ColbanditWindow(1, -1, 1), 1) == 0
    plain = L.colbandit_attention_workspace_bytes(struct(), 1)
    assert L.colbandit_attention_window_workspace_bytes(struct(), tr.ColbanditWindow(1, 1, 0), 1) == plain
    assert L.colbandit_attention_window_workspace_bytes(struct(), tr.ColbanditWindow(1, 1, 3), 1) > plain


def test_embedding_refusals(tr):
    L = tr.lib()

    def rows(table=0x1000, tdt=0, row=64, tokens=0x2000, n=5, vocab=10, width=64, scale=1.0, out=0x3000, odt=1):
        return L.colbandit_embedding(table, tdt, row, tokens, n, vocab, width, scale, out, odt, None)

    def grads(dout=0x1000, ddt=0, row=64, tokens=0x2000, n=5, vocab=10, width=64, scale=1.0, table=0x3000, tdt=1, ws=0x10000, nb=1 << 30):
        return L.colbandit_embedding_backward(dout, ddt, row, tokens, n, vocab, width, scale, table, tdt, ws, nb, None)

    for call in (rows, grads):
        assert call(table=None) == -1 and call(tokens=None) == -1
        assert call(n=-1) == -2 and call(vocab=0) == -2 and call(width=0) == -2 and call(row=63) == -2 and call(tdt=2) == -2
        assert call(n=1 << 31) == -4 and call(vocab=(1 << 24) + 1) == -4 and call(width=65537, row=65537) == -4
        assert call(tokens=0x2004) == -6 and call(table=0x3001) == -6
    assert rows(n=1 << 30, width=17, row=17) == -4 and grads(vocab=1 << 24, width=257, row=257, nb=1 << 62) == -4
    assert rows(out=None) == -1 and rows(out=0x3001) == -6 and grads(dout=None) == -1 and grads(dout=0x1002) == -6
    assert grads(ws=None) == -1 and grads(ws=0x10010) == -6 and grads(nb=64) == -5
    assert L.colbandit_embedding_workspace_bytes(-1, 10, 64) == 0 and L.colbandit_embedding_workspace_bytes(0, 10, 64) > 0


def test_rotation_refusals(tr):
    L = tr.lib()

    def struct(**kw):
        a = dict(dt=1, heads=4, kv_heads=2, d=64, interleaved=0, eps=1e-6, rows=10, n_positions=50, q=0x1000, k=0x2000, q_row=512, q_head=64,
                 k_row=512, k_head=64, q_weight=0x3000, k_weight=0x4000, table=0x5000, positions=0x6000)
        return tr.ColbanditRotation(**{**a, **kw})

    def forward(q=0x10000, k=0x20000, **kw):
        return L.colbandit_norm_rotate(struct(**kw), q, k, None)

    def backward(gq=0x10000, gk=0x20000, dq=0x30000, dk=0x40000, wq=0x50000, wk=0x60000, ws=0x100000, nb=1 << 30, **kw):
        return L.colbandit_norm_rotate_backward(struct(**kw), gq, gk, dq, dk, wq, wk, ws, nb, None)

    def inputs(call, **kw):                           # (forward's own q and k are outputs)
        return L.colbandit_norm_rotate(struct(**kw), 0x10000, 0x20000, None) if call is forward else backward(**kw)

    for call in (forward, backward):
        assert inputs(call, q=None) == -1 and inputs(call, k=None) == -1 and inputs(call, positions=None) == -1
        assert inputs(call, heads=0) == -2 and inputs(call, kv_heads=0) == -2 and inputs(call, rows=-1) == -2 and inputs(call, dt=2) == -2
        assert inputs(call, n_positions=0) == -2 and inputs(call, d=0) == -2 and inputs(call, q_row=-8) == -2
        assert inputs(call, eps=-1.0) == -3 and inputs(call, eps=math.nan) == -3 and inputs(call, eps=math.inf) == -3
        assert inputs(call, d=48) == -4 and inputs(call, rows=1 << 31) == -4 and inputs(call, heads=5000) == -4
        assert inputs(call, q=0x1008) == -6 and inputs(call, q_row=260) == -6 and inputs(call, k_head=4) == -6
        assert inputs(call, table=0x5008) == -6 and inputs(call, positions=0x6004) == -6 and inputs(call, q_weight=0x3002) == -6
    assert forward(q=None) == -1 and forward(k=0x20008) == -6
    assert backward(gq=None) == -1 and backward(dk=None) == -1 and backward(dq=0x30008) == -6 and backward(wq=0x50002) == -6
    assert backward(ws=None) == -1 and backward(ws=0x100010) == -6 and backward(nb=16) == -5
    assert L.colbandit_norm_rotate(None, 0x10000, 0x20000, None) == -1
    t = (ctypes.c_float * 64)()
    assert L.colbandit_rotary_table(1, 64, 1e4, None) == -1 and L.colbandit_rotary_table(0, 64, 1e4, t) == -2
    assert L.colbandit_rotary_table(1, 63, 1e4, t) == -2 and L.colbandit_rotary_table(1, 64, 0.0, t) == -3
    assert L.colbandit_rotary_table(1, 64, math.inf, t) == -3


def test_orthogonalising_refusals(tr):
    L = tr.lib()

    def call(n=2, g=(0x1000, 0x2000), o=(0x1000, 0x2000), rows=(4, 5), cols=(6, 7), dts=(0, 1), steps=5, k=POLYNOMIAL, ws=0x10000, nb=1 << 40):
        arr = lambda t, v: None if v is None else (t * len(v))(*v)  # noqa: E731
        i64 = ctypes.c_int64
        return L.colbandit_orthogonalise(n, arr(ctypes.c_void_p, g), arr(ctypes.c_void_p, o), arr(i64, rows), arr(i64, cols),
                                         arr(ctypes.c_int32, dts), steps, arr(ctypes.c_float, k), ws, nb, None)

    assert call(g=None) == -1 and call(o=None) == -1 and call(rows=None) == -1 and call(cols=None) == -1 and call(dts=None) == -1
    assert call(k=None) == -1 and call(g=(0x1000, None)) == -1 and call(o=(None, 0x2000)) == -1 and call(ws=None) == -1
    assert call(n=0) == -2 and call(rows=(-1, 5)) == -2 and call(cols=(4, -5)) == -2 and call(dts=(0, 2)) == -2 and call(steps=0) == -2
    assert call(steps=65) == -3 and call(k=(math.nan, 0.0, 0.0)) == -3
    assert call(k=(5.0, 0.0, 0.0)) == -3 and call(k=(2.0, 0.0, 0.0)) == -3 and call(k=(1.0, 40.0, -40.0)) == -3 and call(k=(-3.0, 0.0, 2.5)) == -3
    assert call(rows=(16385, 5), cols=(16385, 7)) == -4 and call(cols=((1 << 26) + 1, 7)) == -4
    assert call(g=(0x1002, 0x2000)) == -6 and call(o=(0x1000, 0x2001)) == -6 and call(ws=0x10010) == -6 and call(nb=64) == -5


def test_polynomials_with_a_small_leading_coefficient_are_refused_too(tr):
    """An extreme between the ends, where the quadratic formula's own cancellation loses it."""
    for k in ((30.0, -30.0, 1e-30), (30.0, -30.0, 0.0), (30.0, -30.0, -1e-25), (-30.0, 30.0, 1e-20)):
        arr = lambda t, *v: (t * len(v))(*v)  # noqa: E731
        assert tr.lib().colbandit_orthogonalise(1, arr(ctypes.c_void_p, 0x1000), arr(ctypes.c_void_p, 0x1000), arr(ctypes.c_int64, 4),
                                                arr(ctypes.c_int64, 5), arr(ctypes.c_int32, 0), 1, arr(ctypes.c_float, *k), None, 0, None) == -3


def test_rotation_takes_as_many_rows_as_it_says(tr):
    """More than a launch of a thread for every value would have threads: refused for what is missing and not for their number."""
    for d in (32, 64, 96, 128):
        r = tr.ColbanditRotation(1, 1, 1, d, 0, 1e-6, (1 << 31) - (1 << 16) - 1, 1, 0x1000, 0x2000, d, d, d, d, None, None, None, None)
        assert tr.lib().colbandit_norm_rotate(r, None, None, None) == -1
        assert tr.lib().colbandit_norm_rotate_backward(r, None, None, None, None, None, None, None, 0, None) == -1


def test_numbers_beyond_the_librarys_types_keep_their_sign(tr, monkeypatch):
    w = tr._window((-(1 << 64) + 5, 1 << 64), 3)
    assert w.before < 0 and w.after == 1 << 62
    assert tr._window((1, 1), -(1 << 64) + 1).sinks < 0
    monkeypatch.setattr(tr, "_on_device", lambda *t: 0)
    monkeypatch.setattr(tr, "_workspace", lambda *a: (None, 0))
    monkeypatch.setattr(tr, "_stream", lambda *a: None)
    for steps in ((1 << 32) + 5, -(1 << 32) + 5):
        with pytest.raises(tr.ColbanditError, match="-[23]"):
            tr.colbandit_orthogonalise([torch.zeros(4, 5)], steps=steps)


def test_an_orthogonal_steps_workspace_lives_until_it_is_used(tr, monkeypatch):
    """From the checks, through what is done before the call, to the call."""
    import gc
    import types
    import weakref
    held, calls = [], []

    def call(*args):
        gc.collect()
        calls.append((args[-2], [x() is not None for x in held]))
        return 0 if args[-2] else -5

    def workspace(ws, need, device):
        ws = torch.zeros(need, dtype=torch.uint8)
        held.append(weakref.ref(ws))
        return ws, need

    monkeypatch.setattr(tr, "_on_device", lambda *t: 0)
    monkeypatch.setattr(tr, "_stream", lambda *a: None)
    monkeypatch.setattr(tr, "_workspace", workspace)
    monkeypatch.setattr(tr, "lib", lambda: types.SimpleNamespace(colbandit_orthogonalise=call, colbandit_orthogonalise_workspace_bytes=lambda *a: 64))
    p = torch.nn.Parameter(torch.zeros(4, 5))
    p.grad = torch.ones(4, 5)
    tr.orthogonal_step_([p], {}, rate=0.1)
    tr.colbandit_orthogonalise([p.grad])
    assert [room for room, _ in calls] == [0, 64, 64] and [alive[-1] for _, alive in calls] == [True] * 3


def test_python_refusals(tr):
    """Shapes, types and places are checked before the library is called."""
    W, t = torch.zeros(5, 8), torch.zeros(3, dtype=torch.int64)
    q, w = torch.zeros(4, 2, 64), torch.ones(64)
    table, positions = torch.zeros(9, 32, 2), torch.zeros(4, dtype=torch.int64)
    off = torch.tensor([0, 4])
    for bad in (lambda: tr.colbandit_embedding(W.half(), t), lambda: tr.colbandit_embedding(W[0], t),
                lambda: tr.colbandit_embedding(W.T, t), lambda: tr.colbandit_embedding(W, t.int()),
                lambda: tr.colbandit_embedding(W, t[:, None]), lambda: tr.colbandit_embedding(W, t, dtype=torch.float16),
                lambda: tr.colbandit_embedding(W, t, out=torch.zeros(3, 7)),
                lambda: tr.colbandit_embedding_backward(W, t, 5), lambda: tr.colbandit_embedding_backward(W[:1].expand(3, 8), t, 5),
                lambda: tr.colbandit_embedding_backward(W[:3], t, 5, out=torch.zeros(4, 8)),
                lambda: tr.colbandit_norm_rotate(q.half(), q.half()), lambda: tr.colbandit_norm_rotate(q, q.bfloat16()),
                lambda: tr.colbandit_norm_rotate(q, q[:3]), lambda: tr.colbandit_norm_rotate(q, q[:, :, :32]),
                lambda: tr.colbandit_norm_rotate(q, q, q_weight=w[:32]), lambda: tr.colbandit_norm_rotate(q, q, q_weight=w.bfloat16()),
                lambda: tr.colbandit_norm_rotate(q, q, table=table), lambda: tr.colbandit_norm_rotate(q, q, table=table[:, :16], positions=positions),
                lambda: tr.colbandit_norm_rotate(q, q, table=table, positions=positions[:3]),
                lambda: tr.colbandit_norm_rotate(q.transpose(1, 2), q.transpose(1, 2)),
                lambda: tr.colbandit_norm_rotate_backward(q[:3], q, q, q),
                lambda: tr.colbandit_attention(q, q, q, off, sinks=2), lambda: tr.colbandit_attention(q, q, q, off, window=3),
                lambda: tr.colbandit_orthogonalise([]), lambda: tr.colbandit_orthogonalise([w]), lambda: tr.colbandit_orthogonalise([W.half()]),
                lambda: tr.colbandit_orthogonalise([W.T]), lambda: tr.colbandit_orthogonalise([W], out=[W.bfloat16()]),
                lambda: tr.colbandit_orthogonalise([W], out=[W, W])):
        with pytest.raises((TypeError, ValueError)):
            bad()
    if not torch.cuda.is_available():                 # tensors that are not on the device
        for bad in (lambda: tr.colbandit_embedding(W, t), lambda: tr.colbandit_norm_rotate(q, q), lambda: tr.colbandit_orthogonalise([W])):
            with pytest.raises((ValueError, RuntimeError, AssertionError)):
                bad()


def test_rotary_tables_are_those_of_64_bits(tr):
    for n, d, base in ((1, 2, 1e4), (50, 64, 1e4), (7, 96, 123.0), (300, 128, 5e5)):
        got = tr.colbandit_rotary_table(n, d, base, device="cpu").double()
        a = torch.arange(n).double()[:, None] * torch.tensor([base ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64)
        # rounded to 32 bits once; angles of a few hundred in 64 bits differ in their last places
        assert float((got - torch.stack([a.cos(), a.sin()], 2)).abs().max()) <= 2.0 ** -25 + 1e-12


def test_second_order_gradients_are_refused(tr, monkeypatch):
    """The autograd forms over stand-ins of the library's calls."""
    monkeypatch.setattr(tr, "colbandit_embedding", lambda W, t, **how: {"out": W[t] * how["scale"]})
    monkeypatch.setattr(tr, "colbandit_embedding_backward",
                        lambda g, t, vocab, **how: {"dtable": torch.zeros(vocab, g.shape[1]).index_add(0, t, g.detach()) * how["scale"]})
    W, t = torch.randn(5, 4, requires_grad=True), torch.tensor([1, 1, 3])
    g, = torch.autograd.grad((tr.embedding(W, t, scale=2.0) ** 2).sum(), W, create_graph=True)
    with pytest.raises(RuntimeError, match="second-order"):
        g.square().sum().backward()
    monkeypatch.setattr(tr, "colbandit_norm_rotate", lambda q, k, **how: {"q": q * 2, "k": k * 3})
    monkeypatch.setattr(tr, "colbandit_norm_rotate_backward", lambda a, b, q, k, **how: {
        "dq": a.detach() * 2, "dk": b.detach() * 3, "dq_weight": torch.zeros(64), "dk_weight": torch.zeros(64)})
    q = torch.randn(3, 2, 64, requires_grad=True)
    a, b = tr.norm_rotate(q, q)
    g, = torch.autograd.grad(((a + b) ** 2).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="second-order"):
        g.square().sum().backward()
