"""Measured cases of the operators between the embedding and the loss of a
training step: rotary positions, attention with its gradient, and distillation
from a teacher's top logits with its gradient.

Each case is one pass as a training step makes it.  ``run`` computes it either
in plain torch operations (``own`` false: binary32 whatever the inputs' type,
angles in binary64, one rounding at the end) or through this repository's entry
points (``own`` true).

* rotary     query and key heads of one buffer turned by their positions, and
             the gradient turned back: rope, rope_grad.
* attn       attention over packed sequences with its log-sum-exp: attn.
* attn_grad  the gradients of q, k and v from what the forward pass kept:
             attn_grad.
* distill    loss and gradient of the logits against a teacher's top logits,
             in one call (``joint``: distill with dloss) or in two as where the
             loss comes first (distill, distill_grad).

Matrices have tokens in rows and heads side by side.  Sequences are packed one
after the other; the rows behind the last one are padding.  A query of a
sequence with more keys than queries stands at the keys' end (keys kept from
earlier tokens).

Widths are those of the Qwen2.5-1.5B and 7B parameter lists of ``synth``
(hidden 1536 / 3584 and keys 256 / 512 as heads of 128, vocabulary 151936 /
152064) and its small sets; token counts are generic.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # one decoded token's 12 query and 2 key heads: launch latency
        dict(name="rotary_token", op="rotary", tokens=1, heads=14, dim=128, turned=128, axes=1, pairs="halves",
             dtype="bf16"),
        # a micro-batch of text and pictures in 7B geometry: three axes, queries and keys of one projection's output
        dict(name="rotary_7b", op="rotary", tokens=16384, heads=32, dim=128, turned=128, axes=3, pairs="halves",
             dtype="bf16"),
        # one new token over 4096 kept ones, 1.5B
        dict(name="attn_token", op="attn", tokens=1, seqs=1, kept=4095, pad=0, heads=12, kv=2, dim=128, causal=True,
             window=0, dtype="bf16"),
        # a short odd batch in full precision, heads of 40
        dict(name="attn_short_f32", op="attn", tokens=333, seqs=3, kept=0, pad=5, heads=8, kv=8, dim=40, causal=True,
             window=0, dtype="f32"),
        # one long prompt scored under 7B, nothing to be trained
        dict(name="attn_prompt_7b", op="attn", tokens=8192, seqs=1, kept=0, pad=0, heads=28, kv=4, dim=128,
             causal=True, window=0, dtype="bf16"),
        # a micro-batch of packed answers, 1.5B
        dict(name="attn_grad_packed_1.5b", op="attn_grad", tokens=8192, seqs=13, kept=0, pad=77, heads=12, kv=2,
             dim=128, causal=True, window=0, dtype="bf16"),
        # a few short sequences in full precision
        dict(name="attn_grad_short_f32", op="attn_grad", tokens=333, seqs=3, kept=0, pad=5, heads=8, kv=8, dim=40,
             causal=True, window=0, dtype="f32"),
        # one long sequence, 7B: the largest part of a step's attention
        dict(name="attn_grad_7b", op="attn_grad", tokens=8192, seqs=1, kept=0, pad=0, heads=28, kv=4, dim=128,
             causal=True, window=0, dtype="bf16"),
        # one token's logits, 1.5B: launch latency and one long row
        dict(name="distill_token", op="distill", tokens=1, vocab=151936, top=64, tau=1.0, dtype="bf16", joint=True),
        # a short odd batch in full precision at temperature 2, loss first
        dict(name="distill_small_f32", op="distill", tokens=333, vocab=18993, top=20, tau=2.0, dtype="f32",
             joint=False),
        # a micro-batch of 7B logits
        dict(name="distill_7b", op="distill", tokens=4096, vocab=152064, top=64, tau=1.0, dtype="bf16", joint=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "attn", "attn_grad", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "rotary":
        dim = rng.choice([64, 80, 96, 128])
        turned = dim if rng.random() < 0.7 else dim // 2
        heads = _log(rng, 1, 40)
        return dict(op=op, tokens=_log(rng, 1, min(16384, 16384 * 16 * 128 // (heads * dim))), heads=heads, dim=dim,
                    turned=turned, axes=rng.choice([1, 1, 2, 3]), pairs=rng.choice(["halves", "neighbours"]),
                    dtype=dtype)
    if op == "distill":
        vocab = _log(rng, 500, 152064)
        return dict(op=op, tokens=_log(rng, 1, min(8192, 4096 * 76032 // vocab)), vocab=vocab,
                    top=_log(rng, 1, min(200, vocab)), tau=rng.choice([1.0, 1.0, 2.0, 0.7]), dtype=dtype,
                    joint=rng.random() < 0.5)
    dim = rng.choice([64, 128, 128, 40, 72, 96]) if dtype == "bf16" else rng.choice([40, 64, 96, 128])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 4, 6, 7])
    # binary32 products run on the CUDA cores: these are drawn shorter
    most = 8192 * math.sqrt(28 * 128 / (heads * dim) / (24 if dtype == "f32" else 2))
    tokens = _log(rng, 1, int(min(8192, most)))
    kept = _log(rng, 1, int(min(8192, most * most / tokens))) if rng.random() < 0.3 else 0
    seqs = _log(rng, 1, max(1, min(32, tokens // 8)))
    return dict(op=op, tokens=tokens, seqs=seqs, kept=kept // seqs, pad=rng.choice([0, 0, 3, 40]), heads=heads, kv=kv,
                dim=dim, causal=rng.random() < 0.8, window=0 if rng.random() < 0.8 else _log(rng, 16, 2048),
                dtype=dtype)


def _lengths(case):
    """Queries of each sequence: uneven parts of the tokens."""
    T, n = case["tokens"], case["seqs"]
    w = [1 + 7919 * i % 13 for i in range(n)]
    ends = [T * sum(w[:i + 1]) // sum(w) for i in range(n)]
    return [b - a for a, b in zip([0] + ends, ends)]


def _spans(case):
    """(first query, queries, first key, keys) of each sequence."""
    out, q0, k0 = [], 0, 0
    for n in _lengths(case):
        out.append((q0, n, k0, n + case["kept"]))
        q0, k0 = q0 + n, k0 + n + case["kept"]
    return out


def _window(case):
    return case["window"] if case["causal"] else 0


def _pairs(case):
    """Visible (query, key) pairs of one head."""
    total = 0
    for _, nq, _, nk in _spans(case):
        if not case["causal"]:
            total += nq * nk
            continue
        w = _window(case) or nk
        lo, hi = nk - nq + 1, nk               # keys up to the query: lo .. hi of them
        short = max(0, min(hi, w) - lo + 1)    # queries that see fewer keys than the window
        total += (lo + min(hi, w)) * short // 2 + w * (hi - lo + 1 - short)
    return total


def _offsets(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def _sections(case):
    """Pairs of each axis: the first axis has half of them or more."""
    n, axes = case["turned"] // 2, case["axes"]
    rest = n // (axes + 1) if axes > 1 else 0
    return (n - rest * (axes - 1),) + (rest,) * (axes - 1)


def _frequencies(case):
    """The angle per position of each pair, and the pair's axis (binary64, on the host)."""
    n = case["turned"] // 2
    freq = [1e6 ** (-i / n) for i in range(n)]
    axis = [a for a, c in enumerate(_sections(case)) for _ in range(c)]
    return freq, axis


def _positions(gen, case):
    """A text's positions far into a long context; pictures' rows and columns on the further axes."""
    T, axes = case["tokens"], case["axes"]
    first = int(torch.randint(0, 100000, (1,), generator=gen, device="cuda").item())
    p = torch.arange(first, first + T, device="cuda")[None].repeat(axes, 1)
    if axes > 1:
        picture = torch.arange(T, device="cuda") % 1024 < 576
        for a in range(1, axes):
            p[a] = torch.where(picture, first + torch.randint(0, 24, (T,), generator=gen, device="cuda"), p[a])
    return p[0].contiguous() if axes == 1 else p


def _heads_of(gen, rows, heads, dim, dtype):
    """Queries or keys as a trained model has them: a few channels larger than the others."""
    x = torch.randn(rows, heads * dim, generator=gen, device="cuda")
    big = torch.rand(heads * dim, generator=gen, device="cuda") < 0.02
    return (x * torch.where(big, 4.0, 1.0)).to(DTYPES[dtype])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, T, dtype = case["op"], case["tokens"], DTYPES[case["dtype"]]
    state = dict(case)
    if op == "rotary":
        H, D = case["heads"], case["dim"]
        # queries and keys stand in front of the values of one projection's output
        state["x"] = _heads_of(gen, T, H + 2, D, case["dtype"])[:, :H * D]
        state["dy"] = (torch.randn(T, H * D, generator=gen, device="cuda") * 1e-2).to(dtype)
        state["positions"] = _positions(gen, case)
        freq, axis = _frequencies(case)
        state["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
        state["axis"] = torch.tensor(axis, device="cuda")
        if own:
            import paper_2607_19331_gb300 as iso
            state["plan"] = iso.rope_plan(D, base=1e6, sections=_sections(case), rot_dim=case["turned"],
                                          pairs=case["pairs"])
        return state
    if op == "distill":
        V, K = case["vocab"], case["top"]
        z = torch.empty(T, V, dtype=torch.float32, device="cuda").normal_(0.0, 2.0, generator=gen)
        u = torch.rand(T, K, generator=gen, device="cuda", dtype=torch.float64)
        ids = ((torch.exp(u * math.log(V + 1.0)) - 1.0).to(torch.int64) * 7919 % V)
        z.scatter_reduce_(1, ids, 6.0 + 2.0 * torch.randn(T, K, generator=gen, device="cuda"), "amax")
        state["logits"] = z.to(dtype)
        state["teacher"] = (6.0 + 2.0 * torch.randn(T, K, generator=gen, device="cuda")).to(dtype)
        # the nearest entries only: a row has as many as the teacher's nucleus held
        kept = torch.randint(1, K + 1, (T, 1), generator=gen, device="cuda")
        state["ids"] = torch.where(torch.arange(K, device="cuda")[None] < kept, ids, -1)
        counted = torch.rand(T, generator=gen, device="cuda") < 0.9
        counted[0] = True
        state["dloss"] = torch.where(counted, 1.0 / T, 0.0)
        return state
    H, KV, D = case["heads"], case["kv"], case["dim"]
    lengths, spans = _lengths(case), _spans(case)
    rows, krows = T + case["pad"], T + case["kept"] * case["seqs"] + case["pad"]
    if case["kept"] == 0:      # one projection's output
        qkv = _heads_of(gen, rows, H + 2 * KV, D, case["dtype"])
        state["q"], state["k"], state["v"] = qkv.split([H * D, KV * D, KV * D], dim=1)
    else:
        state["q"] = _heads_of(gen, rows, H, D, case["dtype"])
        kv = _heads_of(gen, krows, 2 * KV, D, case["dtype"])
        state["k"], state["v"] = kv.split([KV * D, KV * D], dim=1)
    state["spans"] = spans
    packed = case["seqs"] > 1 or case["pad"] > 0
    state["q_ends"] = _offsets(lengths) if packed else None
    state["k_ends"] = _offsets([n + case["kept"] for n in lengths]) if packed and case["kept"] else None
    if op == "attn_grad":
        state["out"], state["lse"] = _attention(state)
        state["dout"] = (torch.randn(rows, H * D, generator=gen, device="cuda") * 1e-2).to(dtype)
    return state


def _hidden(case, nq, nk):
    """Where a query of one sequence does not see a key."""
    if not case["causal"]:
        return None
    i = torch.arange(nk - nq, nk, device="cuda")[:, None]
    j = torch.arange(nk, device="cuda")[None]
    far = j > i
    return far | (j <= i - _window(case)) if _window(case) else far


def _groups(s):
    """Query heads, key and value head of every group of every sequence, binary32 [heads, tokens, dim], and the rows."""
    H, KV, D = s["heads"], s["kv"], s["dim"]
    G = H // KV
    for q0, nq, k0, nk in s["spans"]:
        if nq == 0:
            continue
        hidden = _hidden(s, nq, nk)
        for h in range(KV):
            q = s["q"][q0:q0 + nq, h * G * D:(h + 1) * G * D].float().view(nq, G, D).transpose(0, 1)
            k = s["k"][k0:k0 + nk, h * D:(h + 1) * D].float()
            v = s["v"][k0:k0 + nk, h * D:(h + 1) * D].float()
            yield q, k, v, hidden, h, slice(q0, q0 + nq), slice(k0, k0 + nk)


def _attention(s):
    H, KV, D = s["heads"], s["kv"], s["dim"]
    G = H // KV
    out = torch.zeros(s["q"].shape[0], H * D, dtype=s["q"].dtype, device="cuda")
    lse = torch.zeros(H, s["q"].shape[0], dtype=torch.float32, device="cuda")
    for q, k, v, hidden, h, rows, _ in _groups(s):
        S = torch.matmul(q, k.t()).mul_(D ** -0.5)
        if hidden is not None:
            S.masked_fill_(hidden, -math.inf)
        top = S.amax(dim=2, keepdim=True)
        S = S.sub_(top).exp_()
        total = S.sum(dim=2, keepdim=True)
        o = torch.matmul(S, v) / total
        out[rows, h * G * D:(h + 1) * G * D] = o.transpose(0, 1).reshape(-1, G * D).to(out.dtype)
        lse[h * G:(h + 1) * G, rows] = (top + torch.log(total))[:, :, 0]
    return out, lse


def _attention_grad(s):
    H, KV, D = s["heads"], s["kv"], s["dim"]
    G = H // KV
    dq, dk, dv = (torch.zeros(s[n].shape, dtype=s[n].dtype, device="cuda") for n in ("q", "k", "v"))
    for q, k, v, hidden, h, rows, keys in _groups(s):
        cols = slice(h * G * D, (h + 1) * G * D)
        do = s["dout"][rows, cols].float().view(-1, G, D).transpose(0, 1)
        o = s["out"][rows, cols].float().view(-1, G, D).transpose(0, 1)
        P = torch.matmul(q, k.t()).mul_(D ** -0.5).sub_(s["lse"][h * G:(h + 1) * G, rows, None]).exp_()
        if hidden is not None:
            P.masked_fill_(hidden, 0.0)
        dv[keys, h * D:(h + 1) * D] = torch.matmul(P.transpose(1, 2), do).sum(0).to(dv.dtype)
        dS = torch.matmul(do, v.t()).sub_((do * o).sum(dim=2, keepdim=True)).mul_(P)
        dk[keys, h * D:(h + 1) * D] = torch.matmul(dS.transpose(1, 2), q).sum(0).mul(D ** -0.5).to(dk.dtype)
        dq[rows, cols] = torch.matmul(dS, k).mul_(D ** -0.5).transpose(0, 1).reshape(-1, G * D).to(dq.dtype)
    return {"dq": dq, "dk": dk, "dv": dv}


def _turn(x, positions, s, sign):
    T, H, D, R = x.shape[0], s["heads"], s["dim"], s["turned"]
    p = positions[None] if positions.dim() == 1 else positions
    angle = p[s["axis"]].t().double() * s["freq"]                    # [T, pairs]
    c, n = angle.cos().float()[:, None], (sign * angle.sin()).float()[:, None]
    out = x.float().view(T, H, D).clone()
    if s["pairs"] == "halves":
        a, b = slice(0, R // 2), slice(R // 2, R)
    else:
        a, b = slice(0, R, 2), slice(1, R, 2)
    u, w = out[:, :, a].clone(), out[:, :, b].clone()
    out[:, :, a] = u * c - w * n
    out[:, :, b] = u * n + w * c
    return out.view(T, H * D).to(x.dtype)


def _distillation(s):
    z, ids, tau, g = s["logits"].float(), s["ids"], s["tau"], s["dloss"]
    used = ids >= 0
    at = ids.clamp(min=0)
    t = torch.where(used, s["teacher"].float() / tau, -math.inf)
    log_p = t - torch.logsumexp(t, dim=1, keepdim=True)
    p = torch.where(used, log_p.exp(), 0.0)
    z = z / tau
    top = z.amax(dim=1, keepdim=True)
    q = (z - top).exp_()
    total = q.sum(dim=1, keepdim=True)
    lse = top + total.log()
    log_q = z.gather(1, at) - lse
    loss = tau * tau * torch.where(used, p * (log_p - log_q), 0.0).sum(dim=1)
    grad = q.div_(total).scatter_add_(1, at, -p).mul_((g * tau)[:, None])
    return {"loss": loss, "lse": lse[:, 0], "dlogits": grad.to(s["logits"].dtype)}


def _plain(s):
    op = s["op"]
    if op == "rotary":
        return {"y": _turn(s["x"], s["positions"], s, 1.0), "dx": _turn(s["dy"], s["positions"], s, -1.0)}
    if op == "attn":
        out, lse = _attention(s)
        return {"out": out, "lse": lse}
    if op == "attn_grad":
        return _attention_grad(s)
    return _distillation(s)


def run(state):
    if not own:
        return _plain(state)
    import paper_2607_19331_gb300 as iso
    s, op = state, state["op"]
    if op == "rotary":
        return {"y": iso.rope(s["x"], s["positions"], s["plan"]), "dx": iso.rope_grad(s["dy"], s["positions"], s["plan"])}
    if op == "attn":
        out, lse = iso.attn(s["q"], s["k"], s["v"], s["heads"], s["kv"], causal=s["causal"], window=_window(s),
                            seqs=s["q_ends"], kv_seqs=s["k_ends"])
        return {"out": out, "lse": lse}
    if op == "attn_grad":
        dq, dk, dv = iso.attn_grad(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["heads"], s["kv"],
                                   causal=s["causal"], window=_window(s), seqs=s["q_ends"], kv_seqs=s["k_ends"])
        return {"dq": dq, "dk": dk, "dv": dv}
    if s["joint"]:
        loss, lse, dlogits = iso.distill(s["logits"], s["ids"], s["teacher"], temperature=s["tau"], dloss=s["dloss"])
    else:
        loss, lse = iso.distill(s["logits"], s["ids"], s["teacher"], temperature=s["tau"])
        dlogits = iso.distill_grad(s["dloss"], s["logits"], s["ids"], s["teacher"], lse, temperature=s["tau"])
    return {"loss": loss, "lse": lse, "dlogits": dlogits}


def work(case):
    """Bytes and operations of one pass.  Logits count once where loss and
    gradient are one call and twice where they are two: the loss is returned
    before the gradient is asked for."""
    op, T, b = case["op"], case["tokens"], BYTES[case["dtype"]]
    if op == "rotary":
        n = T * case["heads"] * case["dim"]
        return {"bytes": 4 * n * b + 8 * T * case["axes"], "flops": 6 * n}
    if op == "distill":
        V, K = case["vocab"], case["top"]
        return {"bytes": (2 if case["joint"] else 3) * T * V * b + T * K * (8 + b) + 12 * T, "flops": 8 * T * V}
    H, KV, D = case["heads"], case["kv"], case["dim"]
    kt = T + case["kept"] * case["seqs"]
    q, kv, lse = T * H * D * b, 2 * kt * KV * D * b, 4 * T * H
    if op == "attn":
        return {"bytes": 2 * q + kv + lse, "flops": 4 * _pairs(case) * H * D}
    return {"bytes": 4 * q + 2 * kv + lse, "flops": 10 * _pairs(case) * H * D}


def _exact_turn(x, positions, s, sign):
    """Pairs as complex numbers, turned by the angles' unit vectors."""
    T, H, D, R = x.shape[0], s["heads"], s["dim"], s["turned"]
    freq, axis = _frequencies(s)
    p = positions.reshape(s["axes"], T).double()
    angle = torch.stack([p[a] * f for f, a in zip(freq, axis)], dim=1)
    unit = torch.polar(torch.ones_like(angle), sign * angle)[:, None]
    v = x.double().view(T, H, D)
    if s["pairs"] == "halves":
        first, second = torch.arange(R // 2), torch.arange(R // 2) + R // 2
    else:
        first, second = 2 * torch.arange(R // 2), 2 * torch.arange(R // 2) + 1
    w = torch.complex(v[:, :, first], v[:, :, second]) * unit
    out = v.clone()
    out[:, :, first], out[:, :, second] = w.real, w.imag
    return out.view(T, H * D)


def _exact_attention(s, grad):
    """Query head by query head, sequence by sequence."""
    H, KV, D = s["heads"], s["kv"], s["dim"]
    q, k, v = (s[n].double().unflatten(1, (-1, D)) for n in ("q", "k", "v"))
    out, lse = torch.zeros_like(q), torch.zeros(H, q.shape[0], dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for q0, nq, k0, nk in filter(lambda span: span[1], s["spans"]):
        rows, keys = slice(q0, q0 + nq), slice(k0, k0 + nk)
        sees = torch.ones(nq, nk, dtype=torch.bool, device="cuda")
        if s["causal"]:
            sees = sees.tril(nk - nq)
            if _window(s):
                sees = sees.triu(nk - nq - _window(s) + 1)
        for h in range(H):
            g = h // (H // KV)
            logits = torch.einsum("id,jd->ij", q[rows, h], k[keys, g]) / math.sqrt(D)
            logits = torch.where(sees, logits, torch.full_like(logits, -math.inf))
            if not grad:
                out[rows, h] = torch.softmax(logits, dim=1) @ v[keys, g]
                lse[h, rows] = torch.logsumexp(logits, dim=1)
                continue
            prob = torch.exp(logits - s["lse"][h, rows].double()[:, None])
            do = s["dout"].unflatten(1, (-1, D))[rows, h].double()
            delta = torch.einsum("id,id->i", do, s["out"].unflatten(1, (-1, D))[rows, h].double())
            ds = prob * (torch.einsum("id,jd->ij", do, v[keys, g]) - delta[:, None]) / math.sqrt(D)
            dv[keys, g] += torch.einsum("ij,id->jd", prob, do)
            dk[keys, g] += torch.einsum("ij,id->jd", ds, q[rows, h])
            dq[rows, h] = torch.einsum("ij,jd->id", ds, k[keys, g])
    if not grad:
        return {"out": out.flatten(1), "lse": lse}
    return {"dq": dq.flatten(1), "dk": dk.flatten(1), "dv": dv.flatten(1)}


def _exact_distillation(s):
    """Row by row where rows are few, in blocks of rows otherwise: the
    teacher's distribution is laid out over the vocabulary."""
    T, V = s["logits"].shape
    tau, loss, lse = s["tau"], [], []
    grad = torch.empty(T, V, dtype=torch.float64, device="cuda")
    for a in range(0, T, 256):
        ids, z = s["ids"][a:a + 256], s["logits"][a:a + 256].double() / tau
        t = s["teacher"][a:a + 256].double() / tau
        weight = torch.where(ids >= 0, torch.exp(t - t.amax(dim=1, keepdim=True)), torch.zeros_like(t))
        weight = weight / weight.sum(dim=1, keepdim=True)
        log_q = torch.log_softmax(z, dim=1)
        lse.append(torch.logsumexp(z, dim=1))
        dense = torch.zeros_like(z).index_put_((torch.arange(len(z), device="cuda")[:, None].expand_as(ids),
                                                ids.clamp(min=0)), weight, accumulate=True)
        entropy = torch.special.xlogy(weight, weight).sum(dim=1)
        loss.append((entropy - (dense * log_q).sum(dim=1)) * tau ** 2)
        grad[a:a + 256] = (torch.exp(log_q) - dense) * (tau * s["dloss"][a:a + 256].double())[:, None]
    return {"loss": torch.cat(loss), "lse": torch.cat(lse), "dlogits": grad}


def exact(case, seed):
    op, s = case["op"], prepare(case, seed)
    if op == "rotary":
        return {"y": _exact_turn(s["x"], s["positions"], s, 1.0), "dx": _exact_turn(s["dy"], s["positions"], s, -1.0)}
    if op == "distill":
        return _exact_distillation(s)
    return _exact_attention(s, op == "attn_grad")
