"""The layer operators' workloads: what a training or serving step asks of them, in a plain form and
through the library, with the work that each cannot do without.

Shapes are those of the parameter sets that the optimizer steps: 768 wide with 2304, 768 and 3072 columns and a
1000-class head (ViT-B/16, GPT-2 small), 2048 wide with 8192 columns (the 1.3B decoder), 50257 words.
"""
import math

import torch

own = False

NONE, RELU, GELU, SILU = "none", "relu", "gelu", "silu"
IGNORE = -100


def listed():
    return [
        # --- forward product
        # one token of a serving loop through the qkv product of the 768-wide model: latency alone
        dict(name="fwd_token", op="forward", m=1, k=768, n=2304, act=NONE, residual=False, transposed=False, f32=False),
        # eight sequences' next-word logits, fp32, the tied embedding (stored words x width) as the weight
        dict(name="fwd_logits", op="forward", m=8, k=2048, n=50257, act=NONE, residual=False, transposed=True, f32=True),
        # a ragged batch (777 rows) and a class head's odd number of columns, everything in the epilogue
        dict(name="fwd_odd", op="forward", m=777, k=768, n=1001, act=SILU, residual=True, transposed=False, f32=False),
        # the 1.3B model's down product with the residual stream, 8192 tokens
        dict(name="fwd_large", op="forward", m=8192, k=8192, n=2048, act=NONE, residual=True, transposed=False, f32=False),
        # --- backward product
        # one image (197 patches) through the ViT attention output product
        dict(name="bwd_small", op="backward", m=197, k=768, n=768, act=NONE, transposed=False, f32=False),
        # qkv product of the 768-wide model, four sequences of 1024, weight gradient in fp32
        dict(name="bwd_f32", op="backward", m=4096, k=768, n=2304, act=NONE, transposed=True, f32=True),
        # --- 8-bit checkpoints: an MLP block trained from them
        # a short ragged sequence through the 768-wide MLP
        dict(name="mlp8_small", op="mlp8", m=257, k=768, n=3072),
        # 8192 tokens through the 1.3B model's MLP
        dict(name="mlp8_large", op="mlp8", m=8192, k=2048, n=8192),
        # the residual stream of 8192 tokens stored in 8 bits and restored
        dict(name="keep8", op="keep8", m=8192, k=2048),
        # --- loss over the vocabulary
        # fine-tuning a 1000-class head on a few images
        dict(name="loss_small", op="loss", m=197, k=768, n=1000, grads=True),
        # evaluation of the 768-wide model on one odd-length sequence: no gradients
        dict(name="loss_eval", op="loss", m=1023, k=768, n=50257, grads=False),
        # the 1.3B model's head, 8192 tokens, with gradients
        dict(name="loss_large", op="loss", m=8192, k=2048, n=50257, grads=True),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["forward", "forward", "backward", "backward", "mlp8", "keep8", "loss", "loss"])
    m = _spread(rng, 1, 8192)
    if op == "forward":
        transposed = rng.random() < 0.4
        n = 50257 if transposed and m <= 64 else _spread(rng, 257, 8192)
        return dict(op=op, m=m, k=_spread(rng, 255, 8192), n=n, act=rng.choice([NONE, RELU, GELU, SILU]),
                    residual=rng.random() < 0.5, transposed=transposed, f32=rng.random() < 0.3)
    if op == "backward":
        f32 = rng.random() < 0.3
        return dict(op=op, m=m, k=_spread(rng, 255, 8192), n=_spread(rng, 255, 4096),
                    act=NONE if f32 else rng.choice([NONE, RELU, GELU, SILU]), transposed=rng.random() < 0.5, f32=f32)
    if op == "mlp8":
        k = rng.choice([768, 2048, _spread(rng, 255, 2048)])
        return dict(op=op, m=m, k=k, n=rng.choice([4 * k, _spread(rng, 255, 8192)]))
    if op == "keep8":
        return dict(op=op, m=max(64, m), k=_spread(rng, 255, 8192))
    return dict(op=op, m=m, k=rng.choice([768, 2048, _spread(rng, 255, 2048)]),
                n=rng.choice([50257, 1000, _spread(rng, 100, 50257)]), grads=rng.random() < 0.7)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    bf = torch.bfloat16

    def normal(*shape, std=1.0, dtype=bf):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    op, m, k = case["op"], case["m"], case["k"]
    n = case.get("n", 0)
    s = dict(case=case, x=normal(m, k))
    if op in ("forward", "backward"):
        std = 1.0 / math.sqrt(k)
        s["w"] = normal(n, k, std=std).t() if case["transposed"] else normal(k, n, std=std)
        s["bias"] = normal(n, std=0.1)
        if op == "backward":
            s["dy"] = normal(m, n, std=1e-2)
        elif case["residual"]:
            s["residual"] = normal(m, n)
    elif op == "mlp8":
        s["w1"], s["b1"] = normal(k, n, std=1.0 / math.sqrt(k)), normal(n, std=0.1)
        s["w2"], s["b2"] = normal(n, k, std=1.0 / math.sqrt(n)), normal(k, std=0.1)
        s["dy"] = normal(m, k, std=1e-2)
    elif op == "loss":
        s["w"] = normal(n, k, std=2.0 / math.sqrt(k))
        y = torch.randint(0, n, (m,), generator=g, device="cuda")
        drop = torch.rand(m, generator=g, device="cuda") < 0.05
        drop[:1] = False
        s["targets"] = torch.where(drop, torch.full_like(y, IGNORE), y)
    return s


# ---------------------------------------------------------------- the plain form: 32 bits, elementary operations
def _act(z, act):
    if act == RELU:
        return z.clamp_min(0.0)
    if act == SILU:
        return z / (1.0 + torch.exp(-z))
    if act == GELU:
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(z, act):
    if act == RELU:
        return (z > 0).to(z.dtype)
    if act == SILU:
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    if act == GELU:
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _keep8(v):
    """What 8 bits keep of v: blocks of 32 along the row share the smallest power of two 2^e with max|v| <= 127 2^e."""
    m, k = v.shape
    blocks = torch.nn.functional.pad(v, (0, -k % 32)).view(m, -1, 32)
    frac, exp = torch.frexp(blocks.abs().amax(-1, keepdim=True))
    e = torch.where(frac <= 127.0 / 128.0, exp - 7, exp - 6).clamp_min(-126)
    step = ((e + 127) << 23).view(torch.float32)          # 2^e, by its exponent field: exact
    return (torch.round(blocks / step) * step).view(m, -1)[:, :k]


def _plain(s):
    case, op, bf = s["case"], s["case"]["op"], torch.bfloat16
    x = s["x"].float()
    if op == "forward":
        y = _act(x @ s["w"].float() + s["bias"].float(), case["act"])
        if case["residual"]:
            y = y + s["residual"].float()
        return y if case["f32"] else y.to(bf)
    if op == "backward":
        dy = s["dy"].float()
        dx = (dy @ s["w"].float().t()) * _act_grad(x, case["act"])
        a = _act(x, case["act"])
        dw = (dy.t() @ a).t() if case["transposed"] else a.t() @ dy
        gt = torch.float32 if case["f32"] else bf
        return dx.to(bf), dw.to(gt), dy.sum(0).to(gt)
    if op == "mlp8":
        w1, w2, dy = s["w1"].float(), s["w2"].float(), s["dy"].float()
        z = x @ w1 + s["b1"].float()
        y = _act(z, GELU) @ w2 + s["b2"].float() + x
        z8, x8 = _keep8(z), _keep8(x)
        du = (dy @ w2.t()) * _act_grad(z8, GELU)
        dx = du @ w1.t() + dy
        return [t.to(bf) for t in (y, dx, x8.t() @ du, du.sum(0), _act(z8, GELU).t() @ dy, dy.sum(0))]
    if op == "keep8":
        return _keep8(x).to(bf)
    w, t = s["w"].float(), s["targets"]
    keep = t != IGNORE
    logits = x @ w.t()
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    z = e.sum(1, keepdim=True)
    at = t.clamp_min(0).unsqueeze(1)
    zero = torch.zeros((), device=x.device)
    rows = torch.where(keep, (torch.log(z) + top - logits.gather(1, at)).squeeze(1), zero)
    count = keep.sum()
    loss = rows.sum() / count
    if not case["grads"]:
        return loss, rows
    del logits
    d = e.div_(z)
    d.scatter_add_(1, at, torch.full_like(z, -1.0))
    d *= torch.where(keep, 1.0 / count, zero).unsqueeze(1)
    return loss, rows, (d @ w).to(bf), (d.t() @ x).to(bf)


# ---------------------------------------------------------------- the library's calls
def _library(s):
    from paper_2404_00438_b200 import layers
    case, op = s["case"], s["case"]["op"]
    if op == "forward":
        return layers.linear_forward(s["x"], s["w"], s["bias"], act=case["act"], residual=s.get("residual"),
                                     out_dtype=torch.float32 if case["f32"] else torch.bfloat16)
    if op == "backward":
        return layers.linear_backward(s["dy"], s["w"], s["x"], act=case["act"],
                                      grad_dtype=torch.float32 if case["f32"] else torch.bfloat16)
    if op == "mlp8":
        x8 = layers.checkpoint8(s["x"])
        h, z8 = layers.linear_forward(s["x"], s["w1"], s["b1"], act=GELU, keep="8bit")
        y = layers.linear_forward(h, s["w2"], s["b2"], residual=s["x"])
        du, dw2, db2 = layers.linear_backward(s["dy"], s["w2"], z8, act=GELU)
        dx, dw1, db1 = layers.linear_backward(du, s["w1"], x8, residual=s["dy"])
        return [y, dx, dw1, db1, dw2, db2]
    if op == "keep8":
        return layers.restore8(layers.checkpoint8(s["x"]))
    if not case["grads"]:
        r = layers.lm_loss(s["x"], s["w"], s["targets"], ignore_index=IGNORE, grads=False)
        return r.loss, r.rows
    r = layers.lm_loss(s["x"], s["w"], s["targets"], ignore_index=IGNORE)
    return r.loss, r.rows, r.dx, r.dw


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    op, m, k = case["op"], case["m"], case["k"]
    n = case.get("n", 0)
    if op == "forward":
        b = 2 * (m * k + k * n + n) + m * n * (4 if case["f32"] else 2) + (2 * m * n if case["residual"] else 0)
        return {"bytes": b, "flops": 2 * m * k * n}
    if op == "backward":
        g = 4 if case["f32"] else 2
        return {"bytes": 2 * (m * n + k * n + 2 * m * k) + g * (k * n + n), "flops": 4 * m * k * n}
    if op == "mlp8":     # x, dy in, y, dx out; both weights and biases in, their gradients out
        return {"bytes": 8 * m * k + 8 * k * n + 4 * (k + n), "flops": 12 * m * k * n}
    if op == "keep8":    # values in, 8 bits and exponents written and read, values out
        return {"bytes": 4 * m * k + 2 * m * k * 33 / 32, "flops": 4 * m * k}
    if case["grads"]:
        return {"bytes": 4 * (m * k + n * k) + 12 * m + 4, "flops": 6 * m * k * n}
    return {"bytes": 2 * (m * k + n * k) + 12 * m + 4, "flops": 2 * m * k * n}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, f64 = case["op"], torch.float64
    d = {key: v.to(f64) for key, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    root = math.sqrt(2.0 / math.pi)

    def act(z, kind):
        if kind == RELU:
            return torch.where(z > 0, z, torch.zeros_like(z))
        if kind == SILU:
            return z * torch.special.expit(z)
        if kind == GELU:        # half of 1 + tanh(u) is the logistic function of 2u
            return z * torch.special.expit(2.0 * root * (z + 0.044715 * z ** 3))
        return z

    def slope(z, kind):
        if kind == RELU:
            return torch.where(z > 0, torch.ones_like(z), torch.zeros_like(z))
        if kind == SILU:
            p = torch.special.expit(z)
            return p + z * p * (1 - p)
        if kind == GELU:
            p = torch.special.expit(2.0 * root * (z + 0.044715 * z ** 3))
            return p + z * p * (1 - p) * 2.0 * root * (1 + 0.134145 * z ** 2)
        return torch.ones_like(z)

    def eight(v):
        out = torch.empty_like(v)
        for a in range(0, v.shape[1], 32):
            top = v[:, a:a + 32].abs().max(1, keepdim=True).values
            e = torch.ceil(torch.log2(torch.clamp(top, min=2.0 ** -110) / 127.0))
            e = torch.where(127.0 * 2.0 ** (e - 1) >= top, e - 1, e)
            e = torch.where(127.0 * 2.0 ** e < top, e + 1, e)
            step = ((torch.clamp(e, min=-126.0).to(torch.int64) + 1023) << 52).view(f64)
            out[:, a:a + 32] = torch.round(v[:, a:a + 32] / step) * step
        return out

    if op == "forward":
        y = act(torch.addmm(d["bias"], d["x"], d["w"]), case["act"])
        return y + d["residual"] if case["residual"] else y
    if op == "backward":
        dx = torch.mm(d["dy"], d["w"].mT) * slope(d["x"], case["act"])
        return dx, torch.mm(act(d["x"], case["act"]).mT, d["dy"]), d["dy"].sum(dim=0)
    if op == "mlp8":
        z = torch.addmm(d["b1"], d["x"], d["w1"])
        y = torch.addmm(d["b2"], act(z, GELU), d["w2"]) + d["x"]
        z8 = eight(z)
        du = torch.mm(d["dy"], d["w2"].mT) * slope(z8, GELU)
        dx = torch.addmm(d["dy"], du, d["w1"].mT)
        return [y, dx, torch.mm(eight(d["x"]).mT, du), du.sum(dim=0), torch.mm(act(z8, GELU).mT, d["dy"]), d["dy"].sum(dim=0)]
    if op == "keep8":
        return eight(d["x"])
    m, n = case["m"], case["n"]
    rows = torch.zeros(m, dtype=f64, device="cuda")
    valid = s["targets"] != IGNORE
    count = int(valid.sum())
    dx, dw = torch.zeros_like(d["x"]), torch.zeros_like(d["w"])
    for a in range(0, m, 1024):       # a piece of the rows at a time, so that the logits fit in 64 bits
        t, x = s["targets"][a:a + 1024], d["x"][a:a + 1024]
        logits = torch.mm(x, d["w"].mT)
        lse = torch.logsumexp(logits, dim=1)
        ok = valid[a:a + 1024]
        at = torch.where(ok, t, torch.zeros_like(t))
        pick = torch.arange(len(t), device="cuda")
        rows[a:a + 1024] = torch.where(ok, lse - logits[pick, at], torch.zeros_like(lse))
        if case["grads"]:
            p = torch.exp(logits - lse[:, None])
            p[pick, at] -= 1.0
            p = torch.where(ok[:, None], p / count, torch.zeros_like(p))
            dx[a:a + 1024] = torch.mm(p, d["w"])
            dw += torch.mm(p.mT, x)
    loss = rows.sum() / count
    return (loss, rows, dx, dw) if case["grads"] else (loss, rows)
