"""Timed cases of the training operators: one fine-tuning step of a late-interaction encoder, piece by
piece, over the ragged packed layout that the scoring calls use (rows of all sequences one after the
other, int64 offsets).

A case is a dict of plain values:
  op        attn   attention over packed sequences, with a learned bias by buckets of distance where
                   `bias`: its outputs and the rows' log-sum-exp
            train  the same and its backward pass: outputs and all gradients, the bias table's among them
            loss   MaxSim scores of every (query, document) pair, the contrastive loss over them and the
                   gradients of queries and documents
            clip   the global norm of a list of gradients, and the list clipped to a largest norm
  attn, train: dtype, n (sequences), kmin, kmax (their lengths), qmin, qmax (query rows of each; 0: the
            sequence's own), heads, kv_heads, d, causal, bias, keep (a tenth of the keys and one whole
            sequence are masked)
  loss:     dtype, nq, T, N, kmin, kmax (tokens of a document), d
  clip:     dtype, hidden, layers, vocab

`run` computes an operator in its plain form, by elementary torch operations in 32 bits, or calls the
framework where `own` is set.
"""
import math
import random

import numpy as np
import torch

own = False

BUCKETS, MAX_DISTANCE = 32, 128
TEMPERATURE = 0.7


def _attn(name, op, dtype, n, k, heads, kv_heads, d, q=(0, 0), causal=False, bias=False, keep=False):
    c = dict(op=op, dtype=dtype, n=n, kmin=k[0], kmax=k[1], qmin=q[0], qmax=q[1], heads=heads,
             kv_heads=kv_heads, d=d, causal=causal, bias=bias, keep=keep)
    return dict(c, name=name) if name else c


def _loss(name, dtype, nq, T, N, k, d):
    c = dict(op="loss", dtype=dtype, nq=nq, T=T, N=N, kmin=k[0], kmax=k[1], d=d)
    return dict(c, name=name) if name else c


def _clip(name, dtype, hidden, layers, vocab):
    c = dict(op="clip", dtype=dtype, hidden=hidden, layers=layers, vocab=vocab)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the query encoder answers one query of 32 tokens: the smallest call, where latency is all
        _attn("attn_one_query", "attn", "bf16", 1, (32, 32), 12, 12, 64, bias=True),
        # sixteen sequences each take one new token, over what they have read so far (1 to 16,385 keys)
        _attn("attn_single_tokens", "attn", "bf16", 16, (1, 16385), 8, 2, 128, q=(1, 1), causal=True),
        # a candidate list of short passages through a small fp32 encoder, punctuation masked
        _attn("attn_candidates_f32", "attn", "f32", 61, (1, 181), 6, 6, 32, keep=True),
        # page images of 1,030 patch tokens are indexed
        _attn("attn_pages", "attn", "bf16", 48, (1030, 1030), 16, 8, 128),
        # a training batch of passages of 32 to 180 tokens: bias by buckets, punctuation masked
        _attn("train_passages", "train", "bf16", 512, (32, 180), 12, 12, 64, bias=True, keep=True),
        # a training batch of pages, causal backbone whose heads share keys
        _attn("train_pages", "train", "bf16", 24, (1030, 1030), 8, 2, 128, causal=True),
        # odd lengths, an odd number of heads, fp32
        _attn("train_odd_f32", "train", "f32", 37, (1, 301), 5, 5, 96, bias=True),
        # a few queries against their few candidates (a step of gradient accumulation, odd sizes)
        _loss("loss_few_f32", "f32", 3, 21, 10, (5, 64), 64),
        # in-batch negatives: 64 queries, 8 passages for each
        _loss("loss_in_batch", "bf16", 64, 32, 512, (32, 180), 128),
        # the same for pages, vision queries of 24 tokens
        _loss("loss_pages", "bf16", 16, 24, 128, (1030, 1030), 128),
        # only the projection to the embedding width is tuned
        _clip("clip_head", "f32", 768, 0, 0),
        # all of an encoder: 67 million parameters
        _clip("clip_encoder", "f32", 768, 6, 32000),
    ]


# limits of a drawn case: visible pairs times heads times width, of what the plain form holds for the
# padded batch, and of the loss's products, each that of the largest listed case
MAX_PAIRS_D = 48 * 1030 * 1030 * 16 * 128
MAX_PADDED = 512 * 180 * 180 * 12 * 6
MAX_PRODUCTS = 64 * 32 * 512 * 106 * 128


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    op = rng.choice(["attn", "attn", "attn", "train", "train", "train", "loss", "loss", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "clip":
        layers = rng.randint(0, 6)
        return _clip(None, dtype, rng.choice([128, 256, 384, 512, 768]), layers,
                     log(1000, 32000) | 1 if layers else 0)
    if op == "loss":
        T = rng.choice([32, 24, rng.randint(1, 64), rng.randint(5, 128)])
        k = rng.choice([(32, 180), (1, 2 * rng.randint(5, 150) + 1), (1030, 1030), (729, 729)])
        d = rng.choice([128, 128, 64, 96, 32])
        nq, N = log(1, 128), log(2, 1500)
        most = MAX_PRODUCTS // (3 if dtype == "f32" else 1)
        while nq * T * N * (k[0] + k[1]) / 2 * d > most:
            nq, N = max(1, nq * 3 // 4), max(2, N * 3 // 4)
        return _loss(None, dtype, nq, T, N, k, d)
    d, heads, kv_heads = rng.choice([(32, 6, 6), (32, 12, 4), (64, 12, 12), (64, 8, 2), (64, 7, 1), (96, 5, 5),
                                     (96, 6, 3), (128, 8, 2), (128, 16, 8), (128, 4, 4)])
    n = log(1, 512)
    k = rng.choice([(32, 180), (32, 64), (1, log(8, 600) | 1), (1030, 1030), (1, log(64, 4096) | 1)])
    q = (0, 0)
    if op == "attn" and rng.random() < 0.4:
        q = rng.choice([(1, 1), (1, 32), (32, 32)])
        if q == (1, 1):
            k = (1, log(64, 16384) | 1)
    longest = k[1] if q == (0, 0) else q[1]
    most = MAX_PAIRS_D // (5 if op == "train" else 1) // (6 if dtype == "f32" else 1)
    while n > 1 and (n * longest * k[1] * heads * d > most or n * longest * k[1] * heads > MAX_PADDED):
        n = n * 3 // 4
    return _attn(None, op, dtype, n, k, heads, kv_heads, d, q=q, causal=rng.random() < 0.5,
                 bias=rng.random() < 0.6, keep=rng.random() < 0.4)


# ---- inputs ----------------------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _spread(n, lo, hi):
    """n lengths from lo to hi, evenly spread."""
    return [hi] if n == 1 else [lo + i * (hi - lo) // (n - 1) for i in range(n)]


def _lengths(case):
    k = _spread(case.get("n") or case["N"], case["kmin"], case["kmax"])
    if not case.get("qmax"):
        return k, k
    return _spread(case["n"], case["qmin"], case["qmax"]), k


def _offsets(lengths):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)).cuda()


def _shapes(case):
    """Shapes of an encoder's gradients: with no layers, of its projection to the embedding width."""
    h = case["hidden"]
    layer = [(h, 3 * h), (h, h), (2 * h + h // 2, h), (h, 2 * h + h // 2), (3 * h,), (h,), (h,), (2 * h + h // 2,)]
    table = [(case["vocab"], h), (BUCKETS, h // 64 or 1)] if case["layers"] else []
    return table + layer * case["layers"] + [(h, 128), (129,), (1,)]


def prepare(case, seed):
    """The activations, masks, tables, gradients and offsets that a training program has in hand."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dtype(case)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    if case["op"] == "clip":
        # gradients differ in size from tensor to tensor by orders of magnitude
        grads = [(normal(*s) * 10.0 ** (-4 + i % 3)).to(dt) for i, s in enumerate(_shapes(case))]
        return dict(case=case, grads=grads, out=[torch.empty_like(t) for t in grads], max_norm=0.01)
    order = random.Random(seed)
    ql, kl = _lengths(case)
    pairs = list(zip(ql, kl))
    order.shuffle(pairs)
    off = _offsets([b for _, b in pairs])
    total = sum(kl)
    if case["op"] == "loss":
        nq, T, N, d = (case[x] for x in ("nq", "T", "N", "d"))
        Q = torch.nn.functional.normalize(normal(nq, T, d), dim=-1)
        D = torch.nn.functional.normalize(normal(total, d), dim=-1)
        # every query's own document holds noisy copies of some of its tokens, as far as it has room
        own_doc = torch.arange(nq, device="cuda") % N
        near = torch.nn.functional.normalize(Q[:N, ::6] + normal(min(nq, N), -(-T // 6), d) * (1.6 / math.sqrt(d)), dim=-1)
        rows = off[:min(nq, N), None] + torch.arange(near.shape[1], device="cuda")
        room = rows < off[1:min(nq, N) + 1, None]
        D[rows[room]] = near[room]
        # embeddings as an 8-bit index holds them (a step of 1/512): the products of such values and
        # their sums have no rounding in 32 bits, and equal maxima do occur
        grid = lambda x: (x * 512.0).round().clamp(-127, 127) / 512.0  # noqa: E731
        return dict(case=case, Q=grid(Q).to(dt), D=grid(D).to(dt), off=off, longest=max(kl), targets=own_doc)
    H, Hk, d = case["heads"], case["kv_heads"], case["d"]
    # one projection's output, of which queries, keys and values are views
    self_attn = not case["qmax"]
    qoff = off if self_attn else _offsets([a for a, _ in pairs])
    kv = normal(total, (2 * Hk + (H if self_attn else 0)) * d).to(dt)
    at = H * d if self_attn else 0
    k = kv[:, at:at + Hk * d].view(total, Hk, d)
    v = kv[:, at + Hk * d:].view(total, Hk, d)
    q = kv[:, :at].view(total, H, d) if self_attn else normal(sum(ql), H, d).to(dt)
    # some heads look sharply, some broadly
    sharp = torch.linspace(0.3, 2.0, H, device="cuda")[:, None]
    q.mul_(sharp.to(dt))
    keep = None
    if case["keep"]:
        keep = torch.rand(total, generator=g, device="cuda") >= 0.1
        if case["n"] > 1:
            keep[off[0]:off[1]] = False
    bias = normal(BUCKETS, H).to(dt) if case["bias"] else None
    dout = (normal(q.shape[0], H, d) * 1e-2).to(dt) if case["op"] == "train" else None
    return dict(case=case, q=q, k=k, v=v, qoff=qoff, koff=off, keep=keep, bias=bias, dout=dout,
                longest_q=max(ql), longest_k=max(kl), scale=1.0 / math.sqrt(d))


# ---- plain forms -----------------------------------------------------------------------------------

def _rows(off, longest):
    """Row numbers of the padded batch, and which of them are rows of their sequence."""
    r = off[:-1, None] + torch.arange(longest, device="cuda")
    real = r < off[1:, None]
    return torch.where(real, r, 0), real


def _bucket(rel, causal):
    """Buckets of a distance key - query: half of them of single distances, the others of ranges that widen
    up to MAX_DISTANCE; both directions have half of all buckets each unless only one is visible."""
    n = BUCKETS if causal else BUCKETS // 2
    far = (-rel).clamp(min=0) if causal else rel.abs()
    exact_ones = n // 2
    wide = exact_ones + (torch.log(far.clamp(min=1).double() / exact_ones) / math.log(MAX_DISTANCE / exact_ones)
                         * (n - exact_ones) + 1e-9).floor().long().clamp(max=n - exact_ones - 1)
    b = torch.where(far < exact_ones, far, wide)
    return b if causal else b + torch.where(rel > 0, n, 0)


def _plain_attention(s):
    c = s["case"]
    H, Hk, d, group = c["heads"], c["kv_heads"], c["d"], c["heads"] // c["kv_heads"]
    qr, q_real = _rows(s["qoff"], s["longest_q"])
    kr, k_real = _rows(s["koff"], s["longest_k"])

    def padded(x, rows, real):                      # [n, heads, length, d]
        return (x[rows].float() * real[..., None, None]).transpose(1, 2).contiguous()

    Q = padded(s["q"], qr, q_real)
    K = padded(s["k"], kr, k_real).repeat_interleave(group, 1)
    V = padded(s["v"], kr, k_real).repeat_interleave(group, 1)
    S = torch.matmul(Q, K.transpose(2, 3).contiguous()) * s["scale"]
    shift = (s["koff"].diff() - s["qoff"].diff())[:, None, None]
    rel = torch.arange(s["longest_k"], device="cuda") - torch.arange(s["longest_q"], device="cuda")[:, None] - shift
    seen = q_real[:, :, None] & k_real[:, None, :]
    if s["keep"] is not None:
        seen = seen & s["keep"][kr][:, None, :]
    if c["causal"]:
        seen = seen & (rel <= 0)
    bucket = None
    if s["bias"] is not None:
        bucket = _bucket(rel[:1] if not c["qmax"] else rel, c["causal"])
        S = S + s["bias"].float()[bucket].permute(0, 3, 1, 2)
    S = S.masked_fill(~seen[:, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    P = torch.exp(S - m)
    del S
    total = P.sum(-1, keepdim=True)
    P = P / torch.where(total == 0, 1.0, total)
    O = torch.matmul(P, V)
    lse = (m + torch.log(total))[..., 0]
    dt = s["q"].dtype
    out = {"out": O.transpose(1, 2)[q_real].to(dt), "lse": lse.transpose(1, 2)[q_real].t().contiguous()}
    if s["dout"] is None:
        return out
    dO = padded(s["dout"], qr, q_real)
    dP = torch.matmul(dO, V.transpose(2, 3).contiguous())
    dS = P * (dP - (P * dP).sum(-1, keepdim=True))
    del dP
    shared = lambda x: x.view(x.shape[0], Hk, group, -1, d).sum(2)  # noqa: E731
    out["dq"] = (torch.matmul(dS, K) * s["scale"]).transpose(1, 2)[q_real].to(dt)
    out["dk"] = (shared(torch.matmul(dS.transpose(2, 3).contiguous(), Q)) * s["scale"]).transpose(1, 2)[k_real].to(dt)
    out["dv"] = shared(torch.matmul(P.transpose(2, 3).contiguous(), dO)).transpose(1, 2)[k_real].to(dt)
    if bucket is not None:                          # one distance has one bucket in every sequence
        one_hot = (bucket.reshape(-1, 1) == torch.arange(BUCKETS, device="cuda")).float()
        out["dbias"] = torch.matmul(dS.sum(0).reshape(H, -1), one_hot).t().contiguous().to(dt)
    return out


def _plain_loss(s):
    c = s["case"]
    nq, T, N, d, dt = c["nq"], c["T"], c["N"], c["d"], s["Q"].dtype
    rows, real = _rows(s["off"], s["longest"])
    Q = s["Q"].float().view(nq * T, d)
    D = s["D"][rows].float() * real[..., None]      # [N, longest, d]
    S = torch.matmul(D, Q.t().contiguous()).masked_fill(~real[..., None], -math.inf)
    cells = S.amax(1, keepdim=True)                 # [N, 1, nq * T]
    at = torch.arange(s["longest"], device="cuda")[:, None]
    arg = torch.where(S == cells, at, s["longest"]).amin(1, keepdim=True)
    scores = cells.view(N, nq, T).sum(2).t().contiguous()
    x = scores / TEMPERATURE
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    z = e.sum(1, keepdim=True)
    targets = s["targets"][:, None]
    loss = (top + torch.log(z) - x.gather(1, targets))[:, 0]
    hit = (torch.arange(N, device="cuda") == targets).float()
    g = (e / z - hit) / (TEMPERATURE * nq)          # [nq, N]
    W = (at == arg).float() * g.t()[:, None, :, None].expand(N, 1, nq, T).reshape(N, 1, nq * T)
    dD = torch.matmul(W, Q)
    dQ = torch.matmul(W.reshape(-1, nq * T).t().contiguous(), D.view(-1, d))
    return {"scores": scores, "loss": loss, "dQ": dQ.view(nq, T, d).to(dt), "ddocs": dD[real].to(dt)}


def _plain_clip(s):
    flat = torch.cat([t.reshape(-1).float() for t in s["grads"]])
    norm = flat.square().sum().sqrt()
    flat = flat * (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    parts = flat.split([t.numel() for t in s["grads"]])
    return {"norm": norm, "grads": [p.view(t.shape).to(t.dtype) for p, t in zip(parts, s["grads"])]}


# ---- one pass --------------------------------------------------------------------------------------

def _own(s):
    from paper_2602_02827_amd import training as t
    c = s["case"]
    if c["op"] == "clip":
        return t.colbandit_clip_gradients(s["grads"], s["max_norm"], out=s["out"])
    if c["op"] == "loss":
        f = t.colbandit_maxsim_scores(s["Q"], s["D"], s["off"])
        l = t.colbandit_contrastive_loss(f["scores"], s["targets"], TEMPERATURE)
        b = t.colbandit_maxsim_backward(l["dscores"], f["argmax"], s["Q"], s["D"], s["off"])
        return {"scores": f["scores"], "loss": l["loss"], "dQ": b["dQ"], "ddocs": b["ddocs"]}
    how = dict(causal=c["causal"], scale=s["scale"], keep=s["keep"], bias=s["bias"], max_distance=MAX_DISTANCE)
    f = t.colbandit_attention(s["q"], s["k"], s["v"], s["qoff"], s["koff"], **how)
    if c["op"] == "attn":
        return {"out": f["out"], "lse": f["lse"]}
    b = t.colbandit_attention_backward(s["dout"], s["q"], s["k"], s["v"], f["out"], f["lse"], s["qoff"], s["koff"], **how)
    r = {"out": f["out"], "lse": f["lse"], "dq": b["dq"], "dk": b["dk"], "dv": b["dv"]}
    return dict(r, dbias=b["dbias"]) if s["bias"] is not None else r


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_clip(state) if op == "clip" else _plain_loss(state) if op == "loss" else _plain_attention(state)


def work(case):
    """Bytes and operations of one pass: inputs read once, outputs written once; a product's operations for
    the pairs that are visible (those of masked single keys are counted)."""
    c, b = case, 2 if case["dtype"] == "bf16" else 4
    if c["op"] == "clip":
        n = sum(math.prod(s) for s in _shapes(c))
        return {"bytes": 2 * n * b, "flops": 3 * n}
    ql, kl = _lengths(c)
    if c["op"] == "loss":
        rows, total, d, N = c["nq"] * c["T"], sum(kl), c["d"], c["N"]
        # products for the scores; a row added for each (query token, document) in either gradient
        return {"bytes": 2 * (rows + total) * d * b + 4 * c["nq"] * (N + 1) + 8 * (N + 1 + c["nq"]),
                "flops": 2 * rows * total * d + 4 * rows * N * d}
    H, Hk, d, nq, nk = c["heads"], c["kv_heads"], c["d"], sum(ql), sum(kl)
    if c["causal"]:
        pairs = sum(sum(max(0, min(k, i + 1 + k - q)) for i in range(q)) for q, k in zip(ql, kl))
    else:
        pairs = sum(q * k for q, k in zip(ql, kl))
    rows = nq * H * d * b
    keys = nk * Hk * d * b
    table = BUCKETS * H * b if c["bias"] else 0
    small = 16 * (c["n"] + 1) + (nk if c["keep"] else 0) + table + 4 * nq * H
    if c["op"] == "attn":
        return {"bytes": 2 * rows + 2 * keys + small, "flops": 4 * d * H * pairs}
    # what a step reads and writes: q, k, v, the outputs' gradient; out, the three gradients, the table's
    return {"bytes": 4 * rows + 4 * keys + small + table, "flops": 14 * d * H * pairs}


# ---- the definition, in 64 bits --------------------------------------------------------------------

def _host_bucket(dist, causal):
    """Bucket of one distance, from the ranges' first distances."""
    n = BUCKETS if causal else BUCKETS // 2
    base = 0 if causal or dist <= 0 else n
    far = max(0, -dist) if causal else abs(dist)
    single = n // 2
    first = [single * (MAX_DISTANCE / single) ** (i / (n - single)) for i in range(n - single)]
    return base + (far if far < single else single + sum(far >= f - 1e-9 for f in first) - 1)


def _exact_attention(case, s):
    c, H, Hk = case, case["heads"], case["kv_heads"]
    group = H // Hk
    qo, ko = s["qoff"].tolist(), s["koff"].tolist()
    wide = lambda x: None if x is None else x.double()  # noqa: E731
    q, k, v, dout, table = (wide(s[x]) for x in ("q", "k", "v", "dout", "bias"))
    far = max(s["longest_q"], s["longest_k"]) + 1
    of = torch.tensor([_host_bucket(x, c["causal"]) for x in range(-far, far + 1)], device="cuda")
    O, L = torch.zeros_like(q), torch.full((H, q.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dtable = torch.zeros(BUCKETS, H, dtype=torch.float64, device="cuda")
    for a, b, x, y in zip(qo[:-1], qo[1:], ko[:-1], ko[1:]):
        if a == b or x == y:
            continue
        i = torch.arange(b - a, device="cuda")[:, None] + (y - x) - (b - a)
        dist = torch.arange(y - x, device="cuda") - i
        hidden = torch.zeros_like(dist, dtype=torch.bool)
        if c["causal"]:
            hidden |= dist > 0
        if s["keep"] is not None:
            hidden |= ~s["keep"][x:y]
        for h in range(H):
            Q, K, V = q[a:b, h], k[x:y, h // group], v[x:y, h // group]
            Z = (Q @ K.t().contiguous()) * s["scale"]
            if table is not None:
                Z = Z + table[of[dist + far], h]
            Z[hidden] = -math.inf
            lse = torch.logsumexp(Z, 1)
            P = torch.exp(Z - torch.where(lse == -math.inf, 0.0, lse)[:, None])
            O[a:b, h], L[h, a:b] = P @ V, lse
            if dout is None:
                continue
            G = dout[a:b, h]
            E = P * (G @ V.t().contiguous() - (G * O[a:b, h]).sum(1, keepdim=True))
            dq[a:b, h] = E @ K * s["scale"]
            dk[x:y, h // group] += E.t().contiguous() @ Q * s["scale"]
            dv[x:y, h // group] += P.t().contiguous() @ G
            if table is not None:
                dtable[:, h].index_add_(0, of[dist + far].reshape(-1), E.reshape(-1))
    r = {"out": O, "lse": L}
    if dout is not None:
        r |= {"dq": dq, "dk": dk, "dv": dv}
        if table is not None:
            r["dbias"] = dtable
    return r


def _exact_loss(case, s):
    nq, T, N, d = (case[x] for x in ("nq", "T", "N", "d"))
    Q, D, off = s["Q"].double().view(nq * T, d), s["D"].double(), s["off"].tolist()
    scores = torch.zeros(nq, N, dtype=torch.float64, device="cuda")
    best = []
    for i in range(N):
        Z = (Q @ D[off[i]:off[i + 1]].t().contiguous()).cpu().numpy()
        best.append(torch.from_numpy(Z.argmax(1)).cuda())      # the first of equal ones
        scores[:, i] = torch.from_numpy(Z.max(1).reshape(nq, T).sum(1))
    x = scores / TEMPERATURE
    loss = torch.logsumexp(x, 1) - x[torch.arange(nq), s["targets"]]
    g = torch.softmax(x, 1)
    g[torch.arange(nq), s["targets"]] -= 1.0
    g = g / (TEMPERATURE * nq)
    dQ, dD = torch.zeros_like(Q), torch.zeros_like(D)
    for i in range(N):
        w = g[:, i].repeat_interleave(T)[:, None]
        rows = off[i] + best[i]
        dQ += w * D[rows]
        dD.index_add_(0, rows, w * Q)
    return {"scores": scores, "loss": loss, "dQ": dQ.view(nq, T, d), "ddocs": dD}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        g = [t.double() for t in s["grads"]]
        norm = torch.sqrt(sum((t * t).sum() for t in g))
        c = min(1.0, s["max_norm"] / (float(norm) + 1e-6))
        return {"norm": norm, "grads": [t * c for t in g]}
    if case["op"] == "loss":
        return None if case["nq"] * case["T"] * sum(_lengths(case)[1]) > 3e9 else _exact_loss(case, s)
    return None if case["n"] * case["heads"] > 8000 else _exact_attention(case, s)
