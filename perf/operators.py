"""Measured cases of the training-step operators: 8-bit activation checkpoints
with the weight and SwiGLU gradients taken from them, and the token embedding
with its gradient by sorted tokens.

Each case is one pass as a training step makes it.  ``run`` computes it either
in plain torch operations (``own`` false: binary32 whatever the inputs' type,
one rounding at the end) or through this repository's entry points (``own``
true).

* checkpoint   x is packed to 8 bits in the forward pass and read back in the
               backward pass: act_pack, act_unpack.
* linear_grad  the weight gradient G_W = dY^T X_hat of a linear layer whose
               input was kept as a checkpoint: act_pack, act_wgrad.
* swiglu       h = silu(gate) up with both inputs kept as checkpoints, then the
               gradients and h again from them: swiglu_pack, swiglu_grad.
* embed        rows of the embedding table times a scale: embed.
* embed_grad   the dense gradient of the table: embed_grad.

The checkpoint format: groups of 32 consecutive channels of a token share a
power of two 2^e, e the least integer >= -126 with max |x| <= 127 2^e, and
hold round-half-even(x / 2^e); a group with a NaN or an infinity decodes to
NaN.  Every decoded value is exact in bfloat16.

Widths are those of the Qwen2.5-1.5B and 7B parameter lists of ``synth``
(hidden 1536 / 3584, intermediate 8960 / 18944, vocabulary 151936 / 152064)
and its small sets (widths divided by 8); token counts are generic.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
GROUP = 32


def listed():
    return [
        # one decoded token's hidden state: launch latency
        dict(name="checkpoint_token", op="checkpoint", tokens=1, cols=1536, dtype="bf16", gap=0),
        # the MLP activations of one micro-batch of prompts in 1.5B geometry
        dict(name="checkpoint_inter_1.5b", op="checkpoint", tokens=16384, cols=8960, dtype="bf16", gap=0),
        # a short odd batch in full precision (a small set's projection, rows of an odd-width buffer)
        dict(name="linear_grad_short_f32", op="linear_grad", tokens=333, rows=1120, cols=451, dtype="f32",
             out="f32", gap=3),
        # attention output projection of 1.5B: a small weight under many tokens
        dict(name="linear_grad_attn_1.5b", op="linear_grad", tokens=8192, rows=1536, cols=1536, dtype="bf16",
             out="f32", gap=0),
        # gate projection of 7B under one micro-batch: the largest product of a step
        dict(name="linear_grad_gate_7b", op="linear_grad", tokens=8192, rows=18944, cols=3584, dtype="bf16",
             out="bf16", gap=0),
        # one token through the activation of 1.5B: launch latency
        dict(name="swiglu_token", op="swiglu", tokens=1, cols=8960, dtype="bf16", fused=True),
        # the activation of 7B for a micro-batch, gate and up as halves of one projection's output
        dict(name="swiglu_7b", op="swiglu", tokens=8192, cols=18944, dtype="bf16", fused=True),
        # decoding: one token id per step
        dict(name="embed_token", op="embed", tokens=1, vocab=151936, cols=1536, dtype="bf16", scale=1.0, pad=False),
        # a large micro-batch of packed prompts with padding, 7B
        dict(name="embed_prompts_7b", op="embed", tokens=32768, vocab=152064, cols=3584, dtype="bf16",
             scale=1.0, pad=True),
        # a short odd batch against a small set's table, full precision
        dict(name="embed_grad_small_f32", op="embed_grad", tokens=333, vocab=18992, cols=192, dtype="f32",
             out="f32", scale=13.856406460551018, pad=True),
        # a micro-batch against the 1.5B table, gradient in the weights' type
        dict(name="embed_grad_1.5b", op="embed_grad", tokens=8192, vocab=151936, cols=1536, dtype="bf16",
             out="bf16", scale=1.0, pad=True),
        # a large micro-batch against the 7B table, binary32 gradient
        dict(name="embed_grad_7b", op="embed_grad", tokens=32768, vocab=152064, cols=3584, dtype="bf16",
             out="f32", scale=1.0, pad=True),
    ]


def _log(rng, lo, hi):
    n = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n + 1 if n % 1024 == 0 else n  # the listed cases have the round token counts


def draw(rng):
    op = rng.choice(["checkpoint", "linear_grad", "swiglu", "embed", "embed_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    odd = rng.random() < 0.5

    def width(lo, hi):
        c = _log(rng, lo, hi)
        return c if odd else max(lo, c // 16 * 16 + 8)

    if op == "checkpoint":
        cols = width(64, 18944)
        tokens = _log(rng, 1, min(16384, 8192 * 18944 // (2 * cols)))
        return dict(op=op, tokens=tokens, cols=cols, dtype=dtype, gap=rng.choice([0, 0, 5, 8]))
    if op == "linear_grad":
        rows, cols = width(64, 18944), width(64, 18944)
        # binary32 gradients take three products per element: they are drawn shorter
        most = 8192 * 18944 * 3584 // (4 if dtype == "f32" else 1)
        return dict(op=op, tokens=_log(rng, 1, max(1, min(16384, most // (rows * cols)))), rows=rows, cols=cols,
                    dtype=dtype, out=rng.choice(["bf16", "f32"]), gap=rng.choice([0, 0, 3, 8]))
    if op == "swiglu":
        cols = width(64, 18944)
        tokens = _log(rng, 1, min(16384, 8192 * 18944 // (2 * cols)))
        return dict(op=op, tokens=tokens, cols=cols, dtype=dtype, fused=rng.random() < 0.5)
    vocab, cols = _log(rng, 500, 152064), width(64, 3584)
    scale = rng.choice([1.0, math.sqrt(cols)])
    case = dict(op=op, tokens=_log(rng, 1, 32768), vocab=vocab, cols=cols, dtype=dtype, scale=scale,
                pad=rng.random() < 0.7)
    if op == "embed_grad":
        case["out"] = rng.choice(["bf16", "f32"])
    return case


def _activations(gen, tokens, cols, dtype, gap):
    """Activations as a trained model has them: most near N(0, 1), tokens of
    different size, and a few channels tens of times larger.  A row stride of
    cols + gap."""
    x = torch.randn(tokens, cols + gap, generator=gen, device="cuda")
    x *= torch.exp(0.5 * torch.randn(tokens, 1, generator=gen, device="cuda"))
    big = torch.rand(cols + gap, generator=gen, device="cuda") < 0.005
    x *= torch.where(big, 30.0, 1.0)
    return x.to(DTYPES[dtype])[:, :cols]


def _gradient(gen, tokens, cols, dtype):
    return (torch.randn(tokens, cols, generator=gen, device="cuda") * 1e-2).to(DTYPES[dtype])


def _token_ids(gen, case):
    """Token ids with the 1 / rank frequencies of text, the ranks spread over
    the vocabulary; with padding, a run of pad ids at the end."""
    T, V = case["tokens"], case["vocab"]
    u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0).to(torch.int64).clamp_(0, V - 1)
    ids = torch.randperm(V, generator=gen, device="cuda")[rank]
    if case["pad"]:
        ids[T - T // 16:] = V - 1
    return ids


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, T = case["op"], case["tokens"]
    state = dict(case)
    if op == "checkpoint":
        state["x"] = _activations(gen, T, case["cols"], case["dtype"], case["gap"])
    elif op == "linear_grad":
        state["x"] = _activations(gen, T, case["cols"], case["dtype"], case["gap"])
        state["dy"] = _gradient(gen, T, case["rows"] + case["gap"], case["dtype"])[:, :case["rows"]]
    elif op == "swiglu":
        c = case["cols"]
        if case["fused"]:
            gate_up = _activations(gen, T, 2 * c, case["dtype"], 0)
            state["gate"], state["up"] = gate_up[:, :c], gate_up[:, c:]
        else:
            state["gate"] = _activations(gen, T, c, case["dtype"], 0)
            state["up"] = _activations(gen, T, c, case["dtype"], 0)
        state["dh"] = _gradient(gen, T, c, case["dtype"])
    else:
        state["ids"] = _token_ids(gen, case)
        state["pad_id"] = case["vocab"] - 1 if case["pad"] else None
        if op == "embed":
            w = torch.empty(case["vocab"], case["cols"], dtype=DTYPES[case["dtype"]], device="cuda")
            state["table"] = w.normal_(0.0, 0.02, generator=gen)
        else:
            state["dy"] = _gradient(gen, T, case["cols"], case["dtype"])
    return state


def _two_to(e):
    """2^e in binary32, exactly (torch.ldexp goes through pow, which is not): e in -126 .. 127."""
    return ((e.clamp(-126, 127) + 127) << 23).to(torch.int32).view(torch.float32)


def _decoded(x):
    """The values that a checkpoint of x stands for, in binary32."""
    T, C = x.shape
    groups = -(-C // GROUP)
    v = torch.zeros(T, groups * GROUP, dtype=torch.float32, device=x.device)
    v[:, :C] = x
    v = v.view(T, groups, GROUP)
    amax = v.abs().amax(dim=2, keepdim=True)
    mant, exp = torch.frexp(amax)
    e = (exp - torch.where(mant <= 127.0 / 128.0, 7, 6)).clamp(min=-126)
    e = torch.where(amax == 0, torch.zeros_like(e), e)
    code = torch.round(v * _two_to(-e))
    out = torch.where(torch.isfinite(amax), code * _two_to(e), torch.full_like(v, math.nan))
    return out.view(T, groups * GROUP)[:, :C]


def _plain(s):
    op = s["op"]
    if op == "checkpoint":
        return _decoded(s["x"]).to(s["x"].dtype)
    if op == "linear_grad":
        return torch.matmul(s["dy"].float().t(), _decoded(s["x"])).to(DTYPES[s["out"]])
    if op == "swiglu":
        dtype = s["gate"].dtype
        g, u = s["gate"].float(), s["up"].float()
        h = (g / (1.0 + torch.exp(-g)) * u).to(dtype)
        g, u, dh = _decoded(s["gate"]), _decoded(s["up"]), s["dh"].float()
        sig = 1.0 / (1.0 + torch.exp(-g))
        d_gate = (dh * u * sig * (1.0 + g * (1.0 - sig))).to(dtype)
        d_up = (dh * g * sig).to(dtype)
        return {"h": h, "d_gate": d_gate, "d_up": d_up, "h_hat": (g * sig * u).to(dtype)}
    ids, pad_id = s["ids"], s["pad_id"]
    if op == "embed":
        out = s["table"][ids].float() * s["scale"]
        if pad_id is not None:
            out = torch.where((ids == pad_id)[:, None], torch.zeros_like(out), out)
        return out.to(s["table"].dtype)
    dy = s["dy"].float() * s["scale"]
    if pad_id is not None:
        dy = torch.where((ids == pad_id)[:, None], torch.zeros_like(dy), dy)
    grad = torch.zeros(s["vocab"], s["cols"], dtype=torch.float32, device=dy.device)
    return grad.index_add_(0, ids, dy).to(DTYPES[s["out"]])


def run(state):
    if not own:
        return _plain(state)
    import paper_2607_19331_gb300 as iso
    s, op = state, state["op"]
    if op == "checkpoint":
        return iso.act_unpack(iso.act_pack(s["x"]))
    if op == "linear_grad":
        return iso.act_wgrad(s["dy"], iso.act_pack(s["x"]), dtype=DTYPES[s["out"]])
    if op == "swiglu":
        h, gate, up = iso.swiglu_pack(s["gate"], s["up"])
        d_gate, d_up, h_hat = iso.swiglu_grad(s["dh"], gate, up)
        return {"h": h, "d_gate": d_gate, "d_up": d_up, "h_hat": h_hat}
    if op == "embed":
        return iso.embed(s["table"], s["ids"], scale=s["scale"], pad_id=s["pad_id"])
    return iso.embed_grad(s["dy"], s["ids"], s["vocab"], scale=s["scale"], pad_id=s["pad_id"],
                          dtype=DTYPES[s["out"]])


def work(case):
    """Bytes and operations of one pass.  A checkpoint is an output of the
    forward call and an input of the backward call (it is what stays in memory
    between them), so its codes and exponents count once each way."""
    op, T, b = case["op"], case["tokens"], BYTES[case["dtype"]]
    if op in ("embed", "embed_grad"):
        C = case["cols"]
        if op == "embed":
            # every token's row is written; rows are read once each, at most the table
            return {"bytes": min(T, case["vocab"]) * C * b + T * C * b + 8 * T, "flops": T * C}
        return {"bytes": T * C * b + 8 * T + case["vocab"] * C * BYTES[case["out"]], "flops": 2 * T * C}
    C = case["cols"]
    kept = T * C + T * -(-C // GROUP)
    if op == "checkpoint":
        return {"bytes": 2 * T * C * b + 2 * kept, "flops": 6 * T * C}
    if op == "linear_grad":
        M = case["rows"]
        return {"bytes": T * C * b + 2 * kept + T * M * b + M * C * BYTES[case["out"]], "flops": 2 * T * M * C}
    # gate, up, h | dh, d_gate, d_up, h_hat, and both checkpoints each way
    return {"bytes": 7 * T * C * b + 4 * kept, "flops": 40 * T * C}


def _exact_decoded(x):
    """The checkpoint's values in binary64, from the format's definition."""
    x = x.double()
    T, C = x.shape
    out = torch.empty_like(x)
    for c in range(0, C, GROUP):
        g = x[:, c:c + GROUP]
        amax = g.abs().amax(dim=1, keepdim=True)
        # the least e with amax <= 127 2^e: up from below, as log2 may be a rounding off at a power of two
        e = (torch.round(torch.log2(amax / 127.0)) - 1.0).clamp(min=-126.0)
        for _ in range(2):
            e = e + (amax > 127.0 * torch.exp2(e)).double()
        step = torch.exp2(torch.where(torch.isfinite(e), e, torch.zeros_like(e)))
        code = torch.round(g / step)
        out[:, c:c + GROUP] = torch.where(torch.isfinite(amax), code * step, torch.full_like(g, math.nan))
    return out


def exact(case, seed):
    op = case["op"]
    if op == "linear_grad" and work(case)["flops"] > 3e12:
        return None  # minutes at the card's binary64 rate
    s = prepare(case, seed)
    if op == "checkpoint":
        return _exact_decoded(s["x"])
    if op == "linear_grad":
        return s["dy"].double().t() @ _exact_decoded(s["x"])
    if op == "swiglu":
        if case["tokens"] * case["cols"] > 1 << 26:
            return None
        g, u = s["gate"].double(), s["up"].double()
        h = g * torch.sigmoid(g) * u
        g, u, dh = _exact_decoded(s["gate"]), _exact_decoded(s["up"]), s["dh"].double()
        sig = torch.sigmoid(g)
        return {"h": h, "d_gate": dh * u * (sig + g * sig * torch.sigmoid(-g)), "d_up": dh * g * sig,
                "h_hat": g * sig * u}
    ids, keep = s["ids"], torch.ones_like(s["ids"], dtype=torch.float64)
    if s["pad_id"] is not None:
        keep[ids == s["pad_id"]] = 0.0
    if op == "embed":
        return s["table"][ids].double() * (s["scale"] * keep)[:, None]
    # tokens in ascending order of their id; row v is the difference of the
    # running sums at the two ends of its run
    order = torch.argsort(ids, stable=True)
    rows = (s["dy"].double() * (s["scale"] * keep)[:, None])[order]
    run_sum = torch.cumsum(rows, dim=0)
    last = torch.searchsorted(ids[order], torch.arange(case["vocab"], device=ids.device), right=True)
    run_sum = torch.cat([torch.zeros_like(run_sum[:1]), run_sum])
    ends = torch.cat([torch.zeros_like(last[:1]), last])
    return run_sum[ends[1:]] - run_sum[ends[:-1]]
