"""The attention's and the layer norm's workloads: what a training or serving step asks of them, in a plain form and
through the library, with the work that each cannot do without.

Shapes are those of the parameter sets that the optimizer steps: 768 wide with 12 heads of 64 (ViT-B/16 with 197 patches,
GPT-2 small with 1024 positions) and 2048 wide with 16 heads of 128 (the 1.3B decoder).
"""
import math
import random

import torch

own = False


def listed():
    return [
        # --- attention, forward
        # a short prompt of a serving loop through the 768-wide decoder: latency alone
        dict(name="attn_short", op="attention", train=False, tokens=37, sequences=1, ragged=False, behind=0, mix=0, heads=12, kv=12, dim=64, causal=True),
        # evaluation of 64 images: every patch attends all 197 of its image
        dict(name="attn_images", op="attention", train=False, tokens=64 * 197, sequences=64, ragged=False, behind=0, mix=0, heads=12, kv=12, dim=64, causal=False),
        # 32 prompts of different lengths in one pass, four query heads to a key head
        dict(name="attn_prompts", op="attention", train=False, tokens=9001, sequences=32, ragged=True, behind=0, mix=3, heads=16, kv=4, dim=128, causal=True),
        # --- attention, forward and backward
        # one image of a fine-tuning step
        dict(name="attn_train_image", op="attention", train=True, tokens=197, sequences=1, ragged=False, behind=0, mix=0, heads=12, kv=12, dim=64, causal=False),
        # eight sequences of the 768-wide decoder's 1024 positions
        dict(name="attn_train_1024", op="attention", train=True, tokens=8192, sequences=8, ragged=False, behind=0, mix=0, heads=12, kv=12, dim=64, causal=True),
        # documents packed into a batch of 8192 rows, the last 113 of which are padding
        dict(name="attn_train_packed", op="attention", train=True, tokens=8192, sequences=11, ragged=True, behind=113, mix=5, heads=16, kv=4, dim=128, causal=True),
        # one long document through the 2048-wide decoder
        dict(name="attn_train_long", op="attention", train=True, tokens=16384, sequences=1, ragged=False, behind=0, mix=0, heads=16, kv=16, dim=128, causal=True),
        # --- layer norm, forward
        # one token of a serving loop
        dict(name="norm_token", op="norm", train=False, m=1, n=768, f32=False, residual=False),
        # evaluation, 2048 wide
        dict(name="norm_eval", op="norm", train=False, m=16384, n=2048, f32=False, residual=False),
        # --- layer norm, forward and backward
        # one image
        dict(name="norm_train_image", op="norm", train=True, m=197, n=768, f32=False, residual=True),
        # an odd width, the residual stream and the gradients in binary32
        dict(name="norm_train_odd", op="norm", train=True, m=4097, n=1001, f32=True, residual=True),
        # 16384 tokens of the 2048-wide decoder, the skip's gradient added
        dict(name="norm_train_large", op="norm", train=True, m=16384, n=2048, f32=False, residual=True),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.35:
        n = rng.choice([768, 2048, _spread(rng, 64, 8192)])
        f32 = rng.random() < 0.3
        m = min(_spread(rng, 1, 32768), 16384 * (1024 if f32 else 2048) // n)
        return dict(op="norm", train=rng.random() < 0.6, m=m, n=n, f32=f32, residual=rng.random() < 0.6)
    train = rng.random() < 0.6
    heads, kv = rng.choice([(12, 12), (16, 16), (16, 4), (16, 1), (8, 2), (6, 3), (25, 25)])
    dim = rng.choice([64, 64, 128, 128, 80, 96, 32])
    sequences = _spread(rng, 1, 128)
    ragged = rng.random() < 0.6
    tokens = max(sequences, _spread(rng, 16, 16384))
    if heads * dim * tokens > 16384 * 2048:
        tokens = max(sequences, 16384 * 2048 // (heads * dim))
    if not ragged:
        tokens -= tokens % sequences
    behind = rng.choice([0, 0, tokens // 50]) if ragged else 0
    return dict(op="attention", train=train, tokens=tokens, sequences=sequences, ragged=ragged, behind=behind, mix=rng.randrange(1 << 20),
                heads=heads, kv=kv, dim=dim, causal=rng.random() < 0.7 or tokens > 3000 * sequences)


def _lengths(case):
    """The sequences' lengths: equal, or cut at random places of the rows that hold sequences."""
    count, rows = case["sequences"], case["tokens"] - case["behind"]
    if not case["ragged"]:
        return [rows // count] * count
    rng = random.Random(case["mix"])
    cuts = sorted(rng.randint(0, rows) for _ in range(count - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [rows])]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    bf = torch.bfloat16

    def normal(*shape, std=1.0, mean=0.0, dtype=bf):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)

    s = dict(case=case)
    if case["op"] == "norm":
        m, n = case["m"], case["n"]
        stream = torch.float32 if case["f32"] else bf
        s["x"] = normal(m, n, std=2.0, mean=0.3, dtype=stream)
        s["weight"], s["bias"] = normal(n, std=0.2, mean=1.0), normal(n, std=0.1)
        if case["train"]:
            s["dy"] = normal(m, n, std=1e-2)
            if case["residual"]:
                s["residual"] = normal(m, n, std=1e-2, dtype=stream)
        return s
    t, h, kv, d = case["tokens"], case["heads"], case["kv"], case["dim"]
    qkv = normal(t, h + 2 * kv, d)             # as one product leaves them
    s["qkv"], s["q"], s["k"], s["v"] = qkv, qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
    s["lengths"] = _lengths(case)
    ends = torch.tensor([0] + s["lengths"]).cumsum(0)
    s["offsets"] = ends.to(device="cuda", dtype=torch.int32) if case["ragged"] else None
    if case["train"]:
        s["do"] = normal(t, h, d, std=1e-2)
    return s


# ---------------------------------------------------------------- the plain form: 32 bits, elementary operations
EPS = 1e-5


def _plain_norm(s):
    case, bf = s["case"], torch.bfloat16
    x, w, b = s["x"].float(), s["weight"].float(), s["bias"].float()
    mean = x.sum(1, keepdim=True) / case["n"]
    centred = x - mean
    rstd = 1.0 / torch.sqrt((centred * centred).sum(1, keepdim=True) / case["n"] + EPS)
    hat = centred * rstd
    y = (hat * w + b).to(bf)
    stats = torch.cat([mean, rstd], 1).t()
    if not case["train"]:
        return y, stats
    dy = s["dy"].float()
    wdy = dy * w
    dx = rstd * (wdy - wdy.sum(1, keepdim=True) / case["n"] - hat * ((wdy * hat).sum(1, keepdim=True) / case["n"]))
    if case["residual"]:
        dx = dx + s["residual"].float()
    gt = torch.float32 if case["f32"] else bf
    return y, stats, dx.to(s["x"].dtype), (dy * hat).sum(0).to(gt), dy.sum(0).to(gt)


def _plain_attention(s):
    case, bf = s["case"], torch.bfloat16
    t, h, kv, d = case["tokens"], case["heads"], case["kv"], case["dim"]
    scale, group = 1.0 / math.sqrt(d), h // kv
    out = torch.zeros(t, h, d, device="cuda", dtype=bf)
    lse = torch.zeros(h, t, device="cuda")
    grads = torch.zeros(t, h + 2 * kv, d, device="cuda", dtype=bf) if case["train"] else None
    at = 0
    for n in s["lengths"]:
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        hidden = torch.ones(n, n, device="cuda", dtype=torch.bool).triu(1) if case["causal"] else None
        step = max(1, min(kv, (1 << 30) // (n * n * group)))       # key heads at a time
        for a in range(0, kv, step):
            b = min(kv, a + step)
            q = s["q"][rows, a * group:b * group].float().reshape(n, b - a, group, d).permute(1, 2, 0, 3)      # [kv, group, n, d]
            k, v = (s[c][rows, a:b].float().permute(1, 0, 2).unsqueeze(1) for c in "kv")
            e = (q @ k.transpose(-1, -2)) * scale
            if hidden is not None:
                e.masked_fill_(hidden, -math.inf)
            top = e.amax(-1, keepdim=True)
            e = torch.exp(e - top)
            z = e.sum(-1, keepdim=True)
            p = e / z
            o = p @ v
            out[rows, a * group:b * group] = o.permute(2, 0, 1, 3).reshape(n, -1, d).to(bf)
            lse[a * group:b * group, rows] = (torch.log(z) + top).reshape(-1, n)
            if not case["train"]:
                continue
            do = s["do"][rows, a * group:b * group].float().reshape(n, b - a, group, d).permute(1, 2, 0, 3)
            ds = do @ v.transpose(-1, -2)
            ds -= (do * o).sum(-1, keepdim=True)
            ds *= p
            ds *= scale
            grads[rows, a * group:b * group] = (ds @ k).permute(2, 0, 1, 3).reshape(n, -1, d).to(bf)
            grads[rows, h + a:h + b] = (ds.transpose(-1, -2) @ q).sum(1).permute(1, 0, 2).to(bf)
            grads[rows, h + kv + a:h + kv + b] = (p.transpose(-1, -2) @ do).sum(1).permute(1, 0, 2).to(bf)
    return (out, lse, grads) if case["train"] else (out, lse)


# ---------------------------------------------------------------- the library's calls
def _library(s):
    from paper_2404_00438_b200 import layers
    case = s["case"]
    if case["op"] == "norm":
        y, stats = layers.norm_forward(s["x"], s["weight"], s["bias"], eps=EPS)
        if not case["train"]:
            return y, stats
        dx, dw, db = layers.norm_backward(s["dy"], s["x"], s["weight"], stats, residual=s.get("residual"),
                                          grad_dtype=torch.float32 if case["f32"] else torch.bfloat16)
        return y, stats, dx, dw, db
    h, kv = case["heads"], case["kv"]
    length = None if case["ragged"] else case["tokens"] // case["sequences"]
    out, lse = layers.attention_forward(s["q"], s["k"], s["v"], causal=case["causal"], offsets=s["offsets"], length=length)
    if not case["train"]:
        return out, lse
    grads = torch.empty_like(s["qkv"])         # as the backward pass of the product before takes them
    layers.attention_backward(s["do"], s["q"], s["k"], s["v"], out, lse, causal=case["causal"], offsets=s["offsets"], length=length,
                              dq=grads[:, :h], dk=grads[:, h:h + kv], dv=grads[:, h + kv:], zero_rest=True)
    return out, lse, grads


def run(state):
    if own:
        return _library(state)
    return _plain_norm(state) if state["case"]["op"] == "norm" else _plain_attention(state)


def work(case):
    if case["op"] == "norm":
        m, n, e = case["m"], case["n"], 4 if case["f32"] else 2
        if not case["train"]:                  # x in, y and the rows' statistics out
            return {"bytes": m * n * (e + 2) + 4 * n + 8 * m, "flops": 8 * m * n}
        # x, dy and the skip's gradient in, y and dx out; weight and bias in, their gradients out
        return {"bytes": m * n * (2 * e + 4 + (e if case["residual"] else 0)) + 4 * n + 2 * n * e + 8 * m, "flops": 22 * m * n}
    t, h, kv, d = case["tokens"], case["heads"], case["kv"], case["dim"]
    pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in _lengths(case))
    b = 2 * t * d * (2 * h + 2 * kv) + 4 * t * h                     # q, k, v in, out and lse out
    if not case["train"]:
        return {"bytes": b, "flops": 4 * pairs * h * d}
    return {"bytes": b + 2 * t * d * (2 * h + 2 * kv), "flops": 14 * pairs * h * d}      # do in, dq, dk, dv out; seven products


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    d = {key: v.to(f64) for key, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["op"] == "norm":
        x = d["x"]
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = torch.rsqrt(var + EPS)
        hat = torch.addcmul(-(mean * rstd)[:, None], x, rstd[:, None])
        y = torch.addcmul(d["bias"], hat, d["weight"])
        stats = torch.stack([mean, rstd])
        if not case["train"]:
            return y, stats
        u = torch.mul(d["dy"], d["weight"])
        along = torch.einsum("ij,ij->i", u, hat) / case["n"]
        dx = torch.mul(u - u.mean(1, keepdim=True) - torch.mul(hat, along[:, None]), rstd[:, None])
        if case["residual"]:
            dx += d["residual"]
        return y, stats, dx, torch.einsum("ij,ij->j", d["dy"], hat), torch.einsum("ij->j", d["dy"])
    t, h, kv, dim = case["tokens"], case["heads"], case["kv"], case["dim"]
    group = h // kv
    out = torch.zeros(t, h, dim, dtype=f64, device="cuda")
    lse = torch.zeros(h, t, dtype=f64, device="cuda")
    grads = torch.zeros(t, h + 2 * kv, dim, dtype=f64, device="cuda")
    at = 0
    for n in s["lengths"]:
        if n:
            index = torch.arange(n, device="cuda")
            for head in range(h):              # a head's square of scores at a time
                q, k, v = d["q"][at:at + n, head], d["k"][at:at + n, head // group], d["v"][at:at + n, head // group]
                score = torch.einsum("ic,jc->ij", q, k) / dim ** 0.5
                if case["causal"]:
                    score = torch.where(index[:, None] < index[None, :], torch.full((), -math.inf, dtype=f64, device="cuda"), score)
                total = torch.logsumexp(score, dim=1)
                p = score.sub_(total[:, None]).exp_()
                o = torch.einsum("ij,jc->ic", p, v)
                out[at:at + n, head], lse[head, at:at + n] = o, total
                if case["train"]:
                    do = d["do"][at:at + n, head]
                    grads[at:at + n, h + kv + head // group] += torch.einsum("ij,ic->jc", p, do)
                    slope = torch.einsum("ic,jc->ij", do, v).sub_(torch.einsum("ic,ic->i", do, o)[:, None]).mul_(p)
                    grads[at:at + n, head] = torch.einsum("ij,jc->ic", slope, k) / dim ** 0.5
                    grads[at:at + n, h + head // group] += torch.einsum("ij,ic->jc", slope, q) / dim ** 0.5
        at += n
    return (out, lse, grads) if case["train"] else (out, lse)
