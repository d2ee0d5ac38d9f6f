"""Operators of the LM head next to the policy loss, at the sizes a trainer or a rollout engine runs them at: the supervised loss
with its gradient (from bf16 hidden states, or from states stored in 8 bits), and the head held in 8-bit integers (logits of a few
or of many tokens, scoring of given tokens).

`run` computes them in plain torch, or, with `own` set, by the library's calls.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _case(op, T, d, V, **kw):
    base = dict(op=op, T=T, d=d, V=V, w_std=0.02)
    if op in ("ce", "ce_stored"):
        base |= dict(smooth=0.0, z_coef=0.0, turn=0, grad_W=True)
    elif op == "score8":
        base |= dict(turn=0)
    else:
        base |= dict(out="bf16")
    return base | kw


def listed():
    def case(name, op, T, d, V, **kw):
        return dict(_case(op, T, d, V, **kw), name=name)

    return [
        # supervised loss of a unit-test sized policy, where launches and host time are all there is
        case("ce_tiny", "ce", 256, 256, 4096),
        # one micro-batch of supervised warm start on a 3B-class head: a few conversations, prompts left out of the loss, smoothed labels
        case("ce_micro_3b", "ce", 1283, 2048, 151936, turn=200, smooth=0.1),
        # an ordinary step of it, packed conversations with a z term
        case("ce_step_3b", "ce", 16384, 2048, 151936, turn=512, z_coef=1e-4),
        # a 7B-class head that is frozen: the trunk's gradient alone
        case("ce_frozen_7b", "ce", 4096, 3584, 152064, turn=1024, grad_W=False, w_std=0.015),
        # hidden states of one rollout stored in 8 bits, then a step on them: a short batch on a narrow head
        case("stored_short", "ce_stored", 777, 896, 151936, turn=111),
        # and a batch of long multi-turn rollouts
        case("stored_long", "ce_stored", 8192, 2560, 151936, turn=4096),
        # the next token's logits of one sequence, and of a ragged batch of them
        case("next_token", "linear8", 1, 2048, 151936),
        case("next_tokens_7b", "linear8", 13, 3584, 152064, out="fp32", w_std=0.015),
        # odd sizes: a trimmed vocabulary, a width that is no multiple of a tile
        case("odd_head", "linear8", 333, 1000, 4099, out="fp16"),
        # logits of a whole prompt batch
        case("prompt_logits", "linear8", 4096, 2048, 151936),
        # scoring one short turn, and a batch, under a reference model whose head is held in 8 bits
        case("score8_turn", "score8", 77, 2560, 151936),
        case("score8_batch", "score8", 16384, 2048, 151936, turn=512),
    ]


def draw(rng):
    """Another case of the same ranges: one row to sixteen thousand, narrow to 7B-class heads, small to full vocabularies."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["ce", "ce", "ce_stored", "linear8", "linear8", "score8"])
    V = rng.choice([log(1000, 152064), log(30000, 152064), 151936, 152064])
    if op in ("ce", "ce_stored"):
        d = 64 * log(4, 56)
        T = log(32, min(16384, max(64, int(16384 * 2048 * 151936 * 0.75 / (d * V)))))
        return _case(op, T, d, V, turn=rng.choice([0, rng.randint(16, max(17, T))]), smooth=rng.choice([0.0, 0.05, 0.1]),
                     z_coef=rng.choice([0.0, 1e-4]), grad_W=rng.random() < 0.75)
    if op == "score8":
        d = 64 * log(4, 56)
        T = log(1, min(16384, int(16384 * 2048 * 151936 / (d * V))))
        return _case(op, T, d, V, turn=rng.choice([0, rng.randint(16, max(17, T))]))
    d = rng.choice([64 * log(4, 56), 8 * log(16, 448), log(100, 3584)])
    T = rng.choice([log(1, 64), log(1, 6000)])
    return _case(op, T, d, V, out=rng.choice(["bf16", "fp16", "fp32"]))


def _valid(case):
    """Rows that count: of every `turn` rows the first few, more or fewer, are a prompt."""
    rows = torch.ones(case["T"], dtype=torch.uint8)
    if case["turn"]:
        for i, at in enumerate(range(0, case["T"], case["turn"])):
            rows[at:at + (1 + i * 7 % 4) * case["turn"] // 10] = 0
    return rows


def _quantize(x):
    """Rows of x in 8 bits: integers of -127 .. 127 and one scale each.  An element is multiplied by 127 / (the row's largest), kept
    in 32 bits, and the product rounded to the nearest integer, half to even: in 64 bits, where it is exact."""
    x = x.float()
    most = x.abs().amax(1)
    some, full = most >= 2.0 ** -100, torch.full_like(most, 127)   # (not the number 127: a quotient, rounded once)
    q = torch.round(x.double() * torch.where(some, full / most, 0.0).double()[:, None]).float()
    return q, torch.where(some, most / full, 0.0)


def prepare(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    T, d, V, std = case["T"], case["d"], case["V"], case["w_std"]
    W = (torch.randn(V, d, generator=g, device=DEVICE) * std).to(torch.bfloat16)
    # ids with the skew of natural text; a trained model is sure of many of its tokens
    y = (torch.rand(T, generator=g, device=DEVICE) ** 3 * V).long().clamp(max=V - 1)
    sure = torch.rand(T, generator=g, device=DEVICE) * 16 / (std * std * d)
    H = (torch.randn(T, d, generator=g, device=DEVICE) + sure[:, None] * W[y].float()).to(torch.bfloat16)
    state = dict(case, H=H)
    if case["op"] in ("linear8", "score8"):
        # the weights are laid out once: rows of 8-bit integers that start on multiples of 16 bytes
        q, scale = _quantize(W)
        rows = torch.zeros(V, (d + 15) // 16 * 16, dtype=torch.int8, device=DEVICE)
        rows[:, :d] = q.to(torch.int8)
        state |= dict(Wq=rows[:, :d], w_scale=scale)
    else:
        state |= dict(W=W)
    if case["op"] != "linear8":
        state |= dict(tokens=y.int(), mask=_valid(case).to(DEVICE))
    return state


def _cross_entropy(H, W, s):
    mask, y, e, zc, V = s["mask"].bool(), s["tokens"].long(), s["smooth"], s["z_coef"], s["V"]
    h, w = torch.where(mask[:, None], H, 0.0), W.float()
    z = h @ w.T
    m = z.amax(1, keepdim=True)
    zy, zbar = z.gather(1, y[:, None])[:, 0], z.sum(1, dtype=torch.float64).float() / V
    p = z.sub_(m).exp_()
    total = p.sum(1)
    lse = m[:, 0] + total.log()
    weight = mask.float() / mask.sum().clamp(min=1)
    each = (1 - e) * (lse - zy) + e * (lse - zbar) + zc * lse * lse
    loss = (weight.double() * each).sum().float()
    G = p.mul_((weight * (1 + 2 * zc * lse) / total)[:, None]).sub_((weight * e / V)[:, None])
    G.scatter_add_(1, y[:, None], (-weight * (1 - e))[:, None])
    out = dict(loss=loss.reshape(1), logp=torch.where(mask, zy - lse, 0.0), dH=(G @ w).to(torch.bfloat16))
    if s["grad_W"]:
        out["dW"] = (G.T @ h).to(torch.bfloat16)
    return out


def _int8_product(s):
    q, scale = _quantize(s["H"])
    return (q @ s["Wq"].float().T).mul_(scale[:, None]).mul_(s["w_scale"])


def run(state):
    s, op = state, state["op"]
    if own:
        import paper_2512_21450_b200 as rl
        if op == "linear8":
            return rl.rl_int8_linear(s["H"], s["Wq"], s["w_scale"], out_dtype=DTYPES[s["out"]])
        if op == "score8":
            logp, entropy, lse = rl.rl_token_logprobs_int8(s["H"], s["Wq"], s["w_scale"], s["tokens"], s["mask"])
            return dict(logp=logp, entropy=entropy, lse=lse)
        H, H_scale = s["H"], None
        if op == "ce_stored":
            H, H_scale = rl.rl_quantize_rows(H)
        out = rl.rl_cross_entropy_fwd_bwd(H, s["W"], s["tokens"], s["mask"], label_smoothing=s["smooth"], z_coef=s["z_coef"],
                                          H_scale=H_scale, want_dW=s["grad_W"], dW_bf16=True)
        return {k: out[k] for k in ("loss", "logp", "dH", "dW") if k in out}
    if op == "linear8":
        return _int8_product(s).to(DTYPES[s["out"]])
    if op == "score8":
        mask = s["mask"].bool()
        z = _int8_product(s)
        m = z.amax(1, keepdim=True)
        zy = z.gather(1, s["tokens"].long()[:, None])[:, 0]
        p = (z - m).exp_()
        total = p.sum(1)
        lse = m[:, 0] + total.log()
        entropy = lse - p.mul_(z).sum(1) / total
        return dict(logp=torch.where(mask, zy - lse, 0.0), entropy=torch.where(mask, entropy, 0.0), lse=torch.where(mask, lse, 0.0))
    H = s["H"].float()
    if op == "ce_stored":
        # what is stored stands for scale * integer in bf16, the type that the head's products take
        q, scale = _quantize(H)
        H = (q * scale[:, None]).to(torch.bfloat16).float()
    return _cross_entropy(H, s["W"], s)


def work(case):
    T, d, V = case["T"], case["d"], case["V"]
    if case["op"] == "linear8":
        return dict(bytes=T * d * 2 + V * (d + 4) + T * V * DTYPES[case["out"]].itemsize, flops=2 * T * d * V)
    n = int(_valid(case).sum())
    if case["op"] == "score8":
        return dict(bytes=n * d * 2 + V * (d + 4) + T * 17, flops=2 * n * d * V)
    # logits, dH and, where asked for, dW
    grads = 2 if case["grad_W"] else 1
    stored = T * d * 4 if case["op"] == "ce_stored" else 0
    return dict(bytes=n * d * 2 + T * d * 2 + V * d * 2 * grads + T * 9 + stored, flops=2 * (1 + grads) * n * d * V)


def exact(case, seed):
    """From the definitions, in 64 bits, a few rows of logits at a time."""
    s = prepare(case, seed)
    T, d, V, op = case["T"], case["d"], case["V"], case["op"]
    H = s["H"].double()
    if op != "ce":
        # scale and reciprocal are kept in 32 bits
        most = H.abs().amax(1)
        H = torch.round(H * (torch.full_like(most, 127) / most).float().double()[:, None]) * (most / 127).float().double()[:, None]
    W = s["Wq"].double() * s["w_scale"].double()[:, None] if "Wq" in s else s["W"].double()
    step = max(1, (1 << 28) // V)
    if op == "linear8":
        if T * V > 1 << 29:
            out = torch.empty(T, V, device=DEVICE, dtype=torch.float32)   # to a few 1e-8
        else:
            out = torch.empty(T, V, device=DEVICE, dtype=torch.float64)
        for a in range(0, T, step):
            out[a:a + step] = H[a:a + step] @ W.T
        return out
    if op == "ce_stored":
        H = H.float().bfloat16().double()
    mask, y = s["mask"].bool(), s["tokens"].long()
    logp, entropy, lse = (torch.zeros(T, dtype=torch.float64, device=DEVICE) for _ in range(3))
    backward = op != "score8"
    if backward:
        e, zc, n = case["smooth"], case["z_coef"], int(mask.sum())
        loss, dH = torch.zeros(1, dtype=torch.float64, device=DEVICE), torch.zeros_like(H)
        dW = torch.zeros_like(W) if case["grad_W"] else None
    rows = mask.nonzero()[:, 0]
    for r in rows.split(step):
        z = H[r] @ W.T
        lse[r] = torch.logsumexp(z, 1)
        lp = z - lse[r][:, None]
        p = lp.exp()
        logp[r] = lp.gather(1, y[r][:, None])[:, 0]
        if not backward:
            entropy[r] = -(p * lp).sum(1)
            continue
        # the target distribution: one on the label, smoothed over the vocabulary
        t = torch.full_like(p, e / V)
        t[torch.arange(len(r), device=DEVICE), y[r]] += 1 - e
        loss += (-(t * lp).sum(1) + zc * lse[r] ** 2).sum() / n
        g = ((1 + 2 * zc * lse[r])[:, None] * p - t) / n
        dH[r] = g @ W
        if dW is not None:
            dW += g.T @ H[r]
    if not backward:
        return dict(logp=logp, entropy=entropy, lse=lse)
    out = dict(loss=loss, logp=logp, dH=dH)
    if dW is not None:
        out["dW"] = dW
    return out
