"""Cases of the language-model operators around the inner step, for measuring them.

The inner phase of DiLoCo trains a decoder on every replica; between its matrix products stand
four operators, each with its gradient: the scaled embedding lookup, layer norm (over the model
width, and over every head of q and k), causal attention over packed sequences, and the loss
against a teacher's top logits (K = 1 is the cross-entropy of a target token).  `run` makes one
pass through one of them: in elementary torch operations in 32 bits, or, where `own` is true,
through the package's `ops` module.  `exact` computes the same from the definitions in 64 bits.

Sizes: vocabulary 32 000 and model widths 512 to 2048 are those of the 35M ... 1B decoders that
the package's synthetic vectors are sized by; head sizes and token counts are generic.
"""
import math

import torch

own = False

F32, BF16 = "float32", "bfloat16"
DEV = "cuda"


def _dt(name):
    return torch.bfloat16 if name == BF16 else torch.float32


# ------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a handful of tokens looked up for a probe of a model in training: latency alone
        dict(name="embed-17-tokens", op="embedding", train=False, M=1, tokens=17, vocab=32000, d=512, dtype=F32, grad=F32),
        # one inner step's tokens of four 35M replicas, fp32 gradients for AdamW
        dict(name="embed-step-35m", op="embedding", train=True, M=4, tokens=8192, vocab=32000, d=512, dtype=BF16, grad=F32),
        # one inner step's tokens of two 1B replicas, bf16 gradients
        dict(name="embed-step-1b", op="embedding", train=True, M=2, tokens=32768, vocab=32000, d=2048, dtype=BF16, grad=BF16),
        # the norm before a block for a short batch: latency alone
        dict(name="norm-48-rows", op="norm", train=False, M=1, rows=48, groups=1, d=512, dtype=BF16, param=F32),
        # the norm before a block in one inner step of two 1B replicas
        dict(name="norm-step-1b", op="norm", train=True, M=2, rows=16384, groups=1, d=2048, dtype=BF16, param=F32),
        # QKNorm: every head of q, read out of a fused projection's rows, an odd number of tokens
        dict(name="qk-norm-step", op="norm", train=True, M=2, rows=8191, groups=16, d=128, dtype=BF16, param=BF16),
        # a few short documents in evaluation: latency
        dict(name="attn-5-short", op="attention", train=False, tokens=300, sequences=5, heads=8, kv_heads=8, d=64),
        # one inner step of a 35M model: documents of many lengths packed into one row of tokens
        dict(name="attn-step-35m", op="attention", train=True, tokens=8192, sequences=11, heads=8, kv_heads=8, d=64),
        # long documents, grouped heads, 1B width
        dict(name="attn-step-1b", op="attention", train=True, tokens=16384, sequences=3, heads=16, kv_heads=4, d=128),
        # the loss of a short evaluation batch
        dict(name="loss-24-rows", op="distill", train=False, rows=24, vocab=32000, k=1, dtype=F32, temperature=1.0, z=1e-4),
        # next-token cross-entropy with z-loss, fp32 logits
        dict(name="cross-entropy-step", op="distill", train=True, rows=8192, vocab=32000, k=1, dtype=F32, temperature=1.0, z=1e-4),
        # a student trained on a teacher's 64 largest logits, odd vocabulary
        dict(name="distill-step", op="distill", train=True, rows=16384, vocab=50021, k=64, dtype=BF16, temperature=2.0, z=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embedding", "norm", "attention", "distill"])
    train = rng.random() < 0.7
    dtype = rng.choice([F32, BF16, BF16])
    if op == "embedding":
        d = rng.choice([512, 768, 1000, 1024, 1280, 2048])
        M = rng.choice([1, 2, 4, 8])
        tokens = max(1, _log(rng, 8, 65536) // M)
        vocab = min(_log(rng, 1000, 64000), (2 * 32000 * 2048) // (M * d))
        return dict(op=op, train=train, M=M, tokens=tokens, vocab=vocab, d=d, dtype=dtype, grad=rng.choice([F32, BF16]))
    if op == "norm":
        groups = rng.choice([1, 1, 4, 8, 16])
        d = rng.choice([64, 80, 128]) if groups > 1 else rng.choice([512, 768, 1001, 1024, 2048, 4096, 8192])
        M = rng.choice([1, 2, 4])
        rows = max(1, _log(rng, 16, (1 << 26) // (groups * d)) // M)
        return dict(op=op, train=train, M=M, rows=rows, groups=groups, d=d, dtype=dtype, param=rng.choice([F32, BF16]))
    if op == "attention":
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 4])
        while heads > 16:
            heads -= kv
        tokens = _log(rng, 64, 16384 if heads <= 8 else 12288)
        return dict(op=op, train=train, tokens=tokens, sequences=rng.randint(1, min(tokens, 40)), heads=heads, kv_heads=kv,
                    d=rng.choice([64, 64, 80, 96, 128, 128]))
    vocab = rng.choice([32000, 32000, _log(rng, 2000, 100000)])
    rows = _log(rng, 8, 6e8 / vocab)
    return dict(op=op, train=train, rows=rows, vocab=vocab, k=rng.choice([1, 1, 8, 20, 64, 100]), dtype=dtype,
                temperature=rng.choice([1.0, 2.0, 1.5]), z=rng.choice([0.0, 1e-4]))


# ------------------------------------------------------------------------------------ inputs
def _lengths(case, gen):
    """Document lengths of a packed row: a heavy-tailed split of the tokens, every document non-empty."""
    T, B = case["tokens"], case["sequences"]
    w = torch.rand(B, generator=gen, dtype=torch.float64).mul(3.0).exp()
    n = (w / w.sum() * (T - B)).floor().to(torch.int64) + 1
    n[-1] += T - int(n.sum())
    return n


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    c, op, train = dict(case), case["op"], case["train"]

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)

    if op == "embedding":
        M, T, V, d, dt = c["M"], c["tokens"], c["vocab"], c["d"], _dt(c["dtype"])
        # ranks of a text's tokens: the r-th most frequent one appears in proportion to 1/r
        u = torch.rand((M, T), generator=g, device=DEV, dtype=torch.float64)
        c["ids"] = (torch.exp(u * math.log(V + 1.0)) - 1.0).to(torch.int64).clamp_(0, V - 1).to(torch.int32)
        c["table"] = normal(M, V, d, std=0.02, dtype=dt)
        c["scale"] = math.sqrt(d)
        if train:
            c["dout"] = normal(M, T, d, std=1e-3, dtype=dt)
            c["dtable"] = torch.zeros((M, V, d), dtype=_dt(c["grad"]), device=DEV)   # this tensor's part of the gradients
    elif op == "norm":
        M, N, G, d, dt, pt = c["M"], c["rows"], c["groups"], c["d"], _dt(c["dtype"]), _dt(c["param"])
        # heads are read in place from rows that also hold the other projections
        x = normal(M, N, G if G == 1 else 3 * G, d, std=2.0).add_(0.3).to(dt)
        c["x"] = x[:, :, :G]
        c["weight"] = normal(M, d, std=0.1).add_(1.0).to(pt)
        c["bias"] = normal(M, d, std=0.1, dtype=pt)
        c["eps"] = 1e-5
        if train:
            c["dy"] = normal(M, N, G, d, dtype=dt)
            c["dweight"], c["dbias"] = (torch.zeros((M, d), dtype=torch.float32, device=DEV) for _ in range(2))
    elif op == "attention":
        T, H, K, D = c["tokens"], c["heads"], c["kv_heads"], c["d"]
        host = torch.Generator()
        host.manual_seed(int(seed))
        n = _lengths(c, host)
        c["cu"] = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32).to(DEV)
        c["seq"] = torch.repeat_interleave(torch.arange(len(n)), n).to(DEV)
        qkv = normal(T, H + 2 * K, D, dtype=torch.bfloat16)       # one fused projection
        c["q"], c["k"], c["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
        c["scale"] = 1.0 / math.sqrt(D)
        if train:
            c["dout"] = normal(T, H, D, dtype=torch.bfloat16)
    else:
        N, V, k, dt = c["rows"], c["vocab"], c["k"], _dt(c["dtype"])
        c["logits"] = normal(N, V, std=2.0, dtype=dt)
        if k == 1:
            c["ids"] = torch.randint(0, V, (N, 1), generator=g, device=DEV, dtype=torch.int32)
            c["ids"][::16] = -1                                    # places without a target
        else:
            # k different tokens: a random start and a stride that does not divide the vocabulary
            a = torch.randint(0, V, (N, 1), generator=g, device=DEV)
            b = torch.arange(k, device=DEV) * (V // (k + 1)) + a
            c["ids"] = (b % V).to(torch.int32)
        c["teacher"] = normal(N, k, std=2.0).add_(3.0).to(dt)
        c["row_weight"] = torch.full((N,), 1.0 / N, device=DEV)
    return c


# --------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2502_12996_b200 import ops
    op, train = s["op"], s["train"]
    if op == "embedding":
        out = {"out": ops.embedding_forward(s["ids"], s["table"], scale=s["scale"])}
        if train:
            out["dtable"] = ops.embedding_backward(s["ids"], s["dout"], s["dtable"], scale=s["scale"])
        return out
    if op == "norm":
        y, mean, rstd = ops.layer_norm_forward(s["x"], s["weight"], s["bias"], eps=s["eps"])
        out = {"y": y, "mean": mean, "rstd": rstd}
        if train:
            out["dx"] = ops.layer_norm_backward(s["dy"], s["x"], s["weight"], mean, rstd, s["dweight"], s["dbias"])
            out["dweight"], out["dbias"] = s["dweight"], s["dbias"]
        return out
    if op == "attention":
        o, lse = ops.attention_forward(s["q"], s["k"], s["v"], s["cu"], scale=s["scale"])
        out = {"out": o, "lse": lse}
        if train:
            out["dq"], out["dk"], out["dv"] = ops.attention_backward(s["dout"], s["q"], s["k"], s["v"], o, lse, s["cu"],
                                                                     scale=s["scale"])
        return out
    loss, lse, grad = ops.distill_loss(s["logits"], s["ids"], s["teacher"], temperature=s["temperature"], z_coef=s["z"],
                                       row_weight=s["row_weight"], grad=train)
    return {"loss": loss, "lse": lse, "dlogits": grad} if train else {"loss": loss, "lse": lse}


def _run_plain(s):
    op, train = s["op"], s["train"]
    if op == "embedding":
        M, V, d = s["M"], s["vocab"], s["d"]
        flat = (s["ids"].long() + torch.arange(M, device=DEV)[:, None] * V).reshape(-1)
        rows = s["table"].reshape(M * V, d)[flat].float() * s["scale"]
        out = {"out": rows.to(s["table"].dtype).view(M, -1, d)}
        if train:
            dt = torch.zeros((M * V, d), device=DEV)
            dt.index_add_(0, flat, s["dout"].reshape(-1, d).float() * s["scale"])
            out["dtable"] = dt.view(M, V, d).to(s["dtable"].dtype)
        return out
    if op == "norm":
        x, w, b = s["x"].float(), s["weight"].float()[:, None, None], s["bias"].float()[:, None, None]
        mean = x.mean(-1, keepdim=True)
        xc = x - mean
        rstd = ((xc * xc).mean(-1, keepdim=True) + s["eps"]).rsqrt()
        xh = xc * rstd
        out = {"y": (xh * w + b).to(s["x"].dtype), "mean": mean.squeeze(-1), "rstd": rstd.squeeze(-1)}
        if train:
            dy = s["dy"].float()
            dxh = dy * w
            dx = rstd * (dxh - dxh.mean(-1, keepdim=True) - xh * (dxh * xh).mean(-1, keepdim=True))
            out["dx"] = dx.to(s["x"].dtype)
            out["dweight"] = (dy * xh).sum((1, 2))
            out["dbias"] = dy.sum((1, 2))
        return out
    if op == "attention":
        T, H, K, D = s["tokens"], s["heads"], s["kv_heads"], s["d"]
        q = s["q"].float().view(T, K, H // K, D).permute(1, 2, 0, 3)
        k, v = (t.float().permute(1, 0, 2)[:, None] for t in (s["k"], s["v"]))
        at = torch.arange(T, device=DEV)
        hidden = (s["seq"][:, None] != s["seq"][None, :]) | (at[None, :] > at[:, None])
        z = (q @ k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(hidden, -math.inf)
        top = z.amax(-1, keepdim=True)
        p = z.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        p.div_(total)
        o = p @ v
        lse = (top + total.log()).reshape(H, T)

        def rows(t):
            return t.reshape(-1, T, D).permute(1, 0, 2).to(torch.bfloat16).contiguous()

        out = {"out": rows(o), "lse": lse}
        if train:
            do = s["dout"].float().view(T, K, H // K, D).permute(1, 2, 0, 3)
            out["dv"] = rows((p.transpose(-1, -2) @ do).sum(1))
            dz = (do @ v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
            out["dq"] = rows(dz @ k)
            out["dk"] = rows((dz.transpose(-1, -2) @ q).sum(1))
        return out
    tau, dt = s["temperature"], s["logits"].dtype
    x = s["logits"].float() / tau
    top = x.amax(-1, keepdim=True)
    e = (x - top).exp()
    total = e.sum(-1, keepdim=True)
    lse = top + total.log()
    there = s["ids"] >= 0
    ids = s["ids"].long().clamp_min(0)
    t = (s["teacher"].float() / tau).masked_fill(~there, -math.inf)
    any_ = there.any(-1, keepdim=True)
    t = torch.where(any_, t, torch.zeros_like(t))
    t = t - t.amax(-1, keepdim=True)
    logp = t - t.exp().sum(-1, keepdim=True).log()
    p = torch.where(there, logp.exp(), torch.zeros_like(logp))
    kl = torch.where(there, p * (logp - (x.gather(1, ids) - lse)), torch.zeros_like(p)).sum(-1, keepdim=True)
    w = s["row_weight"][:, None] * any_
    out = {"loss": (w * (tau * tau * kl + s["z"] * lse * lse)).squeeze(-1), "lse": lse.squeeze(-1)}
    if train:
        d = e.div_(total).mul_(w * (tau + 2.0 * s["z"] * lse / tau))
        d.scatter_add_(1, ids, -w * tau * p)
        out["dlogits"] = d.to(dt)
    return out


# --------------------------------------------------------------------------------- the floor
def work(case):
    c, op, train = case, case["op"], case["train"]
    size = {F32: 4, BF16: 2}
    if op == "embedding":
        n, e = c["M"] * c["tokens"], size[c["dtype"]]
        # ids, the rows looked up (at most the whole table), the outputs
        moved = n * 4 + (min(n, c["M"] * c["vocab"]) + n) * c["d"] * e
        if train:
            moved += n * c["d"] * e + c["M"] * c["vocab"] * c["d"] * size[c["grad"]]
        return {"bytes": moved, "flops": n * c["d"] * (3 if train else 1)}
    if op == "norm":
        rows, e = c["M"] * c["rows"] * c["groups"], size[c["dtype"]]
        params = 2 * c["M"] * c["d"]
        moved = 2 * rows * c["d"] * e + rows * 8 + params * size[c["param"]]
        if train:                                                 # x, dy read again and dx written, the weights' gradients
            moved += 3 * rows * c["d"] * e + rows * 8 + params * 4
        return {"bytes": moved, "flops": rows * c["d"] * (20 if train else 7)}
    if op == "attention":
        # the lengths are drawn with the seed; as many pairs as equal ones give, which is the least
        T, B, H, K, D = c["tokens"], c["sequences"], c["heads"], c["kv_heads"], c["d"]
        pairs = H * T * (T / B + 1) / 2
        moved = 2 * T * D * (2 * H + 2 * K) + 4 * T * H
        if train:
            moved += 2 * T * D * (4 * H + 4 * K) + 4 * T * H
        return {"bytes": moved, "flops": pairs * D * (14 if train else 4)}
    n, e = c["rows"] * c["vocab"], size[c["dtype"]]
    return {"bytes": n * e * (2 if train else 1) + c["rows"] * (12 + c["k"] * (4 + e)), "flops": n * (7 if train else 4)}


# ---------------------------------------------------------------------- the definitions, 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, train = s["op"], s["train"]
    if op == "embedding":
        M = s["M"]
        out = {"out": torch.stack([s["table"][m].double().index_select(0, s["ids"][m].long()) for m in range(M)]) * s["scale"]}
        if train:
            grad = torch.zeros(s["dtable"].shape, dtype=torch.float64, device=DEV)
            for m in range(M):
                grad[m].index_put_((s["ids"][m].long(),), s["dout"][m].double(), accumulate=True)
            out["dtable"] = grad * s["scale"]
        return out
    if op == "norm":
        x, w, b = s["x"].double(), s["weight"].double()[:, None, None], s["bias"].double()[:, None, None]
        var, mean = torch.var_mean(x, dim=-1, correction=0)
        rstd = 1.0 / torch.sqrt(var + s["eps"])
        xh = (x - mean[..., None]) * rstd[..., None]
        out = {"y": xh * w + b, "mean": mean, "rstd": rstd}
        if train:
            dy, d = s["dy"].double(), s["d"]
            # the gradient as the projection of w dy off the constant vector and off xh
            h = dy * w
            c1 = torch.einsum("...d->...", h) / d
            c2 = torch.einsum("...d,...d->...", h, xh) / d
            out["dx"] = (h - c1[..., None] - xh * c2[..., None]) * rstd[..., None]
            out["dweight"] = torch.einsum("mngd,mngd->md", dy, xh)
            out["dbias"] = torch.einsum("mngd->md", dy)
        return out
    if op == "attention":
        T, H, K, D = s["tokens"], s["heads"], s["kv_heads"], s["d"]
        shape = {"out": H, "dq": H, "dk": K, "dv": K}
        out = {n: torch.zeros((T, h, D), dtype=torch.float64, device=DEV) for n, h in shape.items() if train or n == "out"}
        out["lse"] = torch.zeros((H, T), dtype=torch.float64, device=DEV)
        cu = s["cu"].tolist()
        for a, b in zip(cu, cu[1:]):
            for h in range(H):
                g = h // (H // K)
                q, k, v = s["q"][a:b, h].double(), s["k"][a:b, g].double(), s["v"][a:b, g].double()
                z = torch.tril(q @ k.T * s["scale"]) + torch.triu(torch.full((b - a, b - a), -math.inf, dtype=torch.float64, device=DEV), 1)
                lse = torch.logsumexp(z, 1)
                p = torch.exp(z - lse[:, None])
                out["out"][a:b, h] = p @ v
                out["lse"][h, a:b] = lse
                if train:
                    do = s["dout"][a:b, h].double()
                    dp = do @ v.T
                    dz = p * (dp - (p * dp).sum(1, keepdim=True)) * s["scale"]
                    out["dv"][a:b, g] += p.T @ do
                    out["dk"][a:b, g] += dz.T @ q
                    out["dq"][a:b, h] = dz @ k
        return out
    tau, z, w = s["temperature"], s["z"], s["row_weight"].double()
    N = s["rows"]
    loss, lses, grads = [], [], []
    for r in range(0, N, 2048):                                   # bounded pieces: 64 bits of the whole would not fit beside it
        x = s["logits"][r:r + 2048].double().requires_grad_(train)
        ids, t = s["ids"][r:r + 2048].long(), s["teacher"][r:r + 2048].double()
        with torch.enable_grad():
            lse = torch.logsumexp(x / tau, 1)
            keep = ids >= 0
            some = keep.any(1)
            p = torch.softmax(torch.where(keep, t / tau, torch.full_like(t, -1e300)), 1) * keep
            logq = x.gather(1, ids.clamp_min(0)) / tau - lse[:, None]
            kl = (torch.special.xlogy(p, p) - p * logq).sum(1)
            row = (tau * tau * kl + z * lse * lse) * w[r:r + 2048] * some
        if train:
            grads.append(torch.autograd.grad(row.sum(), x)[0])
        loss.append(row.detach())
        lses.append(lse.detach())
    out = {"loss": torch.cat(loss), "lse": torch.cat(lses)}
    if train:
        out["dlogits"] = torch.cat(grads)
    return out
