"""The operators at the two ends of a training step whose speed is measured, in
their plain form and as a user calls them.

The last pipeline stage turns the hidden state that crossed the boundary into a
loss over the vocabulary and into the gradients of the hidden state and of the
vocabulary's weights; every stage then clips its gradients by their global norm
and updates its parameters.

A case is a dict of plain values:
  op      score   loss and log-sum-exp of each token (no gradients)
          step    the same with the gradients of x and w for given token weights
          norm    global norm of a list of gradients and the clip factor
          adamw   one AdamW step over a list of parameters
  dt      f32 | bf16 | f16: x and w; the gradients (and parameters) of a list
score, step:
  n, v, h   tokens, vocabulary, hidden size
  skipped   share of the tokens that carry no target (padding, prompts)
norm, adamw: the tensors of a stack of transformer blocks with an embedding
  layers, width, vocab   blocks, hidden size, rows of the embedding
  shift     elements by which every tensor's address is off a 16-byte boundary
adamw:
  pdt     the parameters' dtype (dt is the gradients')
  bits    32: moments in binary32; 8: in 8 bits with a power of two per 256
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEV = "cuda"
IGNORE = -100
BLOCK = 256                                    # state positions that share one power of two
LR, B1, B2, EPS, WD, MAX_NORM, STEP0 = 2.5e-4, 0.9, 0.999, 1e-8, 0.01, 1.0, 10


def _head(name, op, dt, n, v, h, skipped):
    return {"name": name, "op": op, "dt": dt, "n": n, "v": v, "h": h, "skipped": skipped}


def _list(name, op, dt, layers, width, vocab, shift, **more):
    return {"name": name, "op": op, "dt": dt, "layers": layers, "width": width, "vocab": vocab, "shift": shift, **more}


def listed():
    return [
        # one token scored against a whole vocabulary (a serving stage that ranks continuations)
        _head("score 1 token", "score", "bf16", 1, 50257, 768, 0.0),
        # evaluation of a batch of 8 sequences of 512, one in ten tokens padding
        _head("score batch", "score", "bf16", 4096, 50257, 768, 0.1),
        # a small model's step where the number of launches counts; odd sizes
        _head("step small odd", "step", "f32", 61, 1009, 97, 0.1),
        # fine-tuning, the batch of 8 x 512 tokens of the transformer workload
        _head("step batch", "step", "bf16", 4096, 50257, 768, 0.1),
        # instruction data: half of the tokens are prompts; odd sizes throughout
        _head("step odd half skipped", "step", "f16", 1531, 30011, 1001, 0.5),
        # the same in binary32
        _head("step binary32", "step", "f32", 2048, 32000, 768, 0.0),
        # a wide stage with a large vocabulary and many tokens
        _head("step wide", "step", "bf16", 8192, 131072, 4096, 0.0),
        # gradients of a small stage, 26 tensors
        _list("norm small", "norm", "f32", 2, 129, 1000, 1),
        # gradients of the whole 12 block stack
        _list("norm stack", "norm", "bf16", 12, 896, 50257, 0),
        # a small stage's update, where the launch counts
        _list("adamw small", "adamw", "f32", 2, 129, 1000, 1, pdt="f32", bits=8),
        # the whole 12 block stack in binary32
        _list("adamw stack", "adamw", "f32", 12, 896, 50257, 0, pdt="f32", bits=32),
        # a wide stage with 8 bit moments
        _list("adamw wide 8 bit", "adamw", "bf16", 24, 2048, 50257, 0, pdt="bf16", bits=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["score", "step", "step", "norm", "adamw", "adamw"])
    dt = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op in ("score", "step"):
        most = 8192 * 131072 * 4096 // (6 if dt == "f32" else 1)
        while True:
            n, v, h = _log_int(rng, 1, 8192), _log_int(rng, 2, 131072), _log_int(rng, 8, 4096)
            if rng.random() < 0.5:
                h = max(8, h // 64 * 64)
            if n * v * h <= most and 3072 not in (n, v, h):
                break
        return {"op": op, "dt": dt, "n": n, "v": v, "h": h, "skipped": rng.choice([0.0, 0.1, 0.5, 0.9])}
    while True:
        layers, width, vocab = rng.randint(0, 24), _log_int(rng, 16, 2048), _log_int(rng, 2, 50257)
        if 12 * layers * width * width + vocab * width <= 1_300_000_000 and not {3 * width, 4 * width, vocab} & {3072}:
            break
    c = {"op": op, "dt": dt, "layers": layers, "width": width, "vocab": vocab, "shift": rng.choice([0, 0, 1, 3])}
    if op == "adamw":
        c["pdt"] = rng.choice([dt, dt, "f32", "bf16"])
        c["bits"] = rng.choice([8, 32])
    return c


# ------------------------------------------------------------------ inputs
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000 + salt)
    return g


def _randn(shape, seed, salt, dt=torch.float32):
    return torch.randn(shape, generator=_gen(seed, salt), device=DEV, dtype=dt)


def _rand(shape, seed, salt):
    return torch.rand(shape, generator=_gen(seed, salt), device=DEV)


def _shapes(c):
    """the parameters of the stack, in the order a module lists them"""
    d, out = c["width"], [(c["vocab"], c["width"])]
    for _ in range(c["layers"]):
        out += [(d,), (d,), (3 * d, d), (3 * d,), (d, d), (d,), (d,), (d,), (4 * d, d), (4 * d,), (d, 4 * d), (d,)]
    return out + [(d,), (d,)]


def _places(c):
    """(first position, elements, shape) of each tensor, and the positions in all: every tensor starts on a block"""
    at, out = 0, []
    for s in _shapes(c):
        n = math.prod(s)
        out.append((at, n, s))
        at += -(-n // BLOCK) * BLOCK
    return out, at


def _flat(size, shift, dt):
    """a zero buffer whose first element is `shift` elements off a 16-byte boundary"""
    return torch.zeros(size + 16, dtype=dt, device=DEV)[shift:shift + size]


def _fill(flat, places, make):
    """normal values in the tensors' places, zeros between them"""
    make(flat)
    for (a, n, _), b in zip(places, [p[0] for p in places[1:]] + [flat.numel()]):
        flat[a + n:b].zero_()


def _prepare_list(c, seed):
    places, size = _places(c)
    g = _flat(size, c["shift"], DTYPES[c["dt"]])
    # per-tensor scales of a real step differ: each block of positions has its own
    scale = torch.exp(_randn((size // BLOCK, 1), seed, 1)) * 1e-3
    _fill(g, places, lambda t: t.view(-1, BLOCK).copy_(_randn((size // BLOCK, BLOCK), seed, 2, torch.float32 if size < 1 << 28 else torch.bfloat16)).mul_(scale.to(t.dtype)))
    s = {"c": c, "grads": [g[a:a + n].view(sh) for a, n, sh in places], "g": g}
    if c["op"] == "norm":
        return s
    p = _flat(size, c["shift"], DTYPES[c["pdt"]])
    _fill(p, places, lambda t: t.copy_(_randn((size,), seed, 3, torch.bfloat16)).mul_(0.02))
    s["p"], s["params"], s["t"], s["seed"] = p, [p[a:a + n].view(sh) for a, n, sh in places], STEP0, seed & 0x7FFFFFFF
    # moments after a few steps: near the gradients that were seen; the norm that the step before this one left
    m = g.float() * 0.3
    v = g.float().square() * (0.5 + _rand((size,), seed, 4)) * 1e-2
    if c["bits"] == 8:
        m, em = _encode_m(m, seed & 0x7FFFFFFF)
        v, ev = _encode_v(v, seed & 0x7FFFFFFF)
        s["state"] = {"m": m, "em": em, "v": v, "ev": ev}
    else:
        s["state"] = {"m": m, "v": v}
    norm = torch.linalg.vector_norm(g, dtype=torch.float32)
    s["clip"] = torch.stack([norm, (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)])
    return s


def _prepare_head(c, seed):
    n, v, h, dt = c["n"], c["v"], c["h"], DTYPES[c["dt"]]
    w = _randn((v, h), seed, 1, torch.float32 if v * h < 1 << 27 else torch.bfloat16).mul_(1.5 / math.sqrt(h)).to(dt)
    t = torch.randint(0, v, (n,), generator=_gen(seed, 2), device=DEV)
    # a model that has learned something: the target's logit stands out by 0 to 12
    wt = w[t].float()
    x = _randn((n, h), seed, 3) + wt * (12 * _rand((n, 1), seed, 4) / wt.square().sum(1, keepdim=True).clamp(min=1e-6))
    x = x.to(dt)
    skip = _rand((n,), seed, 5) < c["skipped"]
    if n > 0:
        skip[0] = False
    t = torch.where(skip, torch.full_like(t, IGNORE), t)
    s = {"c": c, "x": x, "w": w, "t": t}
    if c["op"] == "step":
        s["weight"] = torch.where(skip, 0.0, 1.0 / (~skip).sum().float()).float()
    return s


def prepare(case, seed):
    return _prepare_head(case, seed) if case["op"] in ("score", "step") else _prepare_list(case, seed)


# --------------------------------------------------- moments held in 8 bits
def _exponents(x):
    """per block, the exponent of the power of two that its largest magnitude
    lies under once it is rounded up to 3 mantissa bits (-127 for none)"""
    return ((x.view(-1, BLOCK).abs().amax(1).view(torch.int32) + 0xFFFFF) >> 23) - 127


def _scaled(x, e, bias):
    """x * 2^(-bias - e), block by block, rounded once to binary32"""
    return (x.view(-1, BLOCK).double() * torch.exp2((-bias - e).double())[:, None]).float().view(-1)


def _encode_m(m, seed):
    """sign, 4 exponent bits, 3 mantissa bits, up or down at random"""
    e = _exponents(m)
    bits = _scaled(m.abs(), e, 112).view(torch.int32)
    u = ((bits + _noise(m.numel(), seed, swap=True)) >> 20).clamp(max=127)
    return (u | torch.where(m.view(torch.int32) < 0, 128, 0)).to(torch.uint8), e.to(torch.int8)


def _noise(size, seed, swap=False):
    """20 random bits per position: a hash of the position's pair and the seed, 16 bits of it (swap: the other
    position's) and a half"""
    j = torch.arange((size + 1) // 2, device=DEV, dtype=torch.int64)
    h = ((j ^ seed) * 0x9E3779B9) & 0xFFFFFFFF
    h = ((h ^ (h >> 15)) * 0xB7E15163) & 0xFFFFFFFF
    h = h ^ (h >> 16)
    h = torch.stack([h >> 16, h & 0xFFFF] if swap else [h & 0xFFFF, h >> 16], 1).view(-1)[:size]
    return ((h << 4) | 8).to(torch.int32)


def _encode_v(v, seed):
    """5 exponent bits, 3 mantissa bits, up or down at random; what is not zero stays so"""
    e = _exponents(v)
    u = ((_scaled(v, e, 96).view(torch.int32) + _noise(v.numel(), seed)) >> 20).clamp(max=255)
    return torch.where(v > 0, u.clamp(min=1), 0).to(torch.uint8), e.to(torch.int8)


def _decode(code, e, bits, bias):
    u = code.to(torch.int32)
    x = ((u & ((1 << bits) - 1)) << 20).view(torch.float32).view(-1, BLOCK).double()
    x = (x * torch.exp2((bias + e.int()).double())[:, None]).float().view(-1)
    return torch.where(u >= 128, -x, x) if bits == 7 else x


# -------------------------------------------------------------- plain forms
def _plain_head(s):
    x, w, t = s["x"], s["w"], s["t"]
    keep = t != IGNORE
    xf, wf = torch.where(keep[:, None], x.float(), 0.0), w.float()
    at = torch.where(keep, t, 0)[:, None]
    z = xf @ wf.t()
    top = z.amax(1, keepdim=True)
    zt = z.gather(1, at)[:, 0]
    p = z.sub_(top).exp_()
    total = p.sum(1, keepdim=True)
    lse = (top + total.log())[:, 0]
    out = {"loss": torch.where(keep, lse - zt, 0.0), "lse": torch.where(keep, lse, 0.0)}
    if s["c"]["op"] == "step":
        g = torch.where(keep, s["weight"], 0.0)[:, None]
        p.div_(total).scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32)).mul_(g)
        out["dx"] = (p @ wf).to(x.dtype)
        out["dw"] = (p.t() @ xf).to(w.dtype)
    return out


def _plain_norm(s):
    norm = s["g"].float().square().sum().sqrt()
    return torch.stack([norm, (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)])


def _plain_adamw(s):
    c, st = s["c"], s["state"]
    s["t"] += 1
    g = s["g"].float() * s["clip"][1]
    eight = c["bits"] == 8
    m = _decode(st["m"], st["em"], 7, 112) if eight else st["m"]
    v = _decode(st["v"], st["ev"], 8, 96) if eight else st["v"]
    m = m * B1 + g * (1 - B1)
    v = v * B2 + g * g * (1 - B2)
    denom = (v * (1 / (1 - B2 ** s["t"]))).sqrt() + EPS
    p = s["p"].float() * (1 - LR * WD) - m / denom * (LR / (1 - B1 ** s["t"]))
    s["p"].copy_(p)
    if eight:
        s["seed"] = (s["seed"] + 1) & 0x7FFFFFFF
        st["m"], st["em"] = _encode_m(m, s["seed"])
        st["v"], st["ev"] = _encode_v(v, s["seed"])
        m, v = _decode(st["m"], st["em"], 7, 112), _decode(st["v"], st["ev"], 8, 96)
    else:
        st["m"], st["v"] = m, v
    return {"p": s["p"], "m": m, "v": v}


# ------------------------------------------------------- the user's own calls
def _own(s):
    from paper_2401_07788_amd import head, optim
    op = s["c"]["op"]
    if op == "score":
        loss, lse = head.linear_xent(s["x"], s["w"], s["t"], ignore_index=IGNORE)
        return {"loss": loss, "lse": lse}
    if op == "step":
        r = head.linear_xent_step(s["x"], s["w"], s["t"], s["weight"], ignore_index=IGNORE)
        return {"loss": r.loss, "lse": r.lse, "dx": r.dx, "dw": r.dw}
    if op == "norm":
        if "list" not in s:
            s["list"] = optim.TensorList(s["grads"])
        return optim.grad_norm(s["list"], MAX_NORM)
    if "opt" not in s:
        s["opt"] = optim.AdamW(s["params"], lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, state_bits=s["c"]["bits"],
                               state=s["state"], t=s["t"], seed=s["seed"])
    s["opt"].step(s["grads"], clip=s["clip"])
    m, v = s["opt"].moments()
    return {"p": s["p"], "m": m, "v": v}


def run(state):
    if own:
        return _own(state)
    op = state["c"]["op"]
    return _plain_norm(state) if op == "norm" else _plain_adamw(state) if op == "adamw" else _plain_head(state)


# -------------------------------------------------------------------- costs
def work(case):
    c, size = case, {"f32": 4, "bf16": 2, "f16": 2}
    if c["op"] in ("score", "step"):
        n, v, h, e = c["n"], c["v"], c["h"], size[c["dt"]]
        counted = max(1, round(n * (1 - c["skipped"])))
        if c["op"] == "score":
            return {"bytes": (counted + v) * h * e + 16 * n, "flops": 2 * counted * v * h}
        return {"bytes": (counted + v + n + v) * h * e + 20 * n, "flops": 6 * counted * v * h}
    n, e = sum(math.prod(s) for s in _shapes(c)), size[c["dt"]]
    if c["op"] == "norm":
        return {"bytes": n * e, "flops": 2 * n}
    # 8 bits: codes read and written, and the moments returned as the values they stand for
    moments = 2 * (1 + 1 + 4) if c["bits"] == 8 else 16
    return {"bytes": n * (e + 2 * size[c["pdt"]] + moments), "flops": 16 * n}


# ------------------------------------------------------------------ 64 bits
def _exact_head(s):
    keep = s["t"] != IGNORE
    rows = keep.nonzero()[:, 0]
    x, w, t = s["x"][rows].double(), s["w"].double(), s["t"][rows]
    z = torch.mm(x, w.t().contiguous())
    lse = torch.logsumexp(z, 1)
    n = keep.numel()
    loss, full = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
    loss[rows] = lse - z[torch.arange(rows.numel(), device=DEV), t]
    full[rows] = lse
    out = {"loss": loss, "lse": full}
    if s["c"]["op"] == "step":
        d = torch.exp(z.sub_(lse[:, None]))
        d[torch.arange(rows.numel(), device=DEV), t] -= 1
        d *= s["weight"][rows].double()[:, None]
        dx = torch.zeros(n, w.shape[1], dtype=torch.float64, device=DEV)
        dx[rows] = torch.mm(d, w)
        out["dx"], out["dw"] = dx, torch.mm(d.t().contiguous(), x)
    return out


def _exact_adamw(s):
    eight, st, k = s["c"]["bits"] == 8, s["state"], s["t"] + 1
    g = s["g"].double() * s["clip"][1].double()
    m = (_decode(st["m"], st["em"], 7, 112) if eight else st["m"]).double()
    v = (_decode(st["v"], st["ev"], 8, 96) if eight else st["v"]).double()
    m, v = m * B1 + g * (1 - B1), v * B2 + g.square() * (1 - B2)
    p = s["p"].double()
    p = p - LR * WD * p - LR * (m / (1 - B1 ** k)) / ((v / (1 - B2 ** k)).sqrt() + EPS)
    # moments that are rounded to 8 bits at random have no value in 64 bits
    return {"p": p, "m": None if eight else m, "v": None if eight else v}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        norm = s["g"].double().square().sum().sqrt()
        return torch.stack([norm, (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)])
    return _exact_adamw(s) if case["op"] == "adamw" else _exact_head(s)
