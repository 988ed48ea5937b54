"""Adapters on a ternary model, as work that can be timed and compared: serving them, training them, and the two
operators that stand before and behind them.

Kinds of case (key "kind"):
  lora        ternary pointwise layer with the low-rank adapters of many requests      prom_pw_conv_lora
  lora_grad   its gradients: of the activations and of every adapter's two factors     prom_pw_conv_lora_backward
  norm        layer norm                                                               prom_layernorm
  norm_quant  layer norm whose rows leave as int8 with a step each                     prom_layernorm_quant
  norm_grad   its gradients: of the rows, the weight and the bias                      prom_layernorm_backward
  adamw       one AdamW step over many tensors, moments in 32 or in 8 bits             AdamWTensors.step

Where `own` is false a pass computes the same from elementary torch operations: the adapters as masked products over
all of them at once, the moments in 8 bits in the float32 operations that the interface fixes."""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 256  # elements that share a scale in the 8-bit form of the moments
LR, BETA1, BETA2, EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 100
NORM_EPS, QUANT_EPS = 1e-5, 1e-5


def listed():
    return [
        # one request writes its next token: one row, one adapter, nothing but latency
        dict(name="lora 1 token 4096-4096 r16", kind="lora", n=1, hw=1, cin=4096, cout=4096, rank=16, adapters=8, type="bf16", out="bf16", runs=False),
        # 64 requests write a token each, every one through its own adapter: the adapters are the bytes
        dict(name="lora 64 tokens 4096-4096 r16", kind="lora", n=64, hw=1, cin=4096, cout=4096, rank=16, adapters=64, type="bf16", out="bf16", runs=False),
        # a projection of MobileNetV2 (14x14, 960 to 160) on images that each bring an adapter, float32 out
        dict(name="lora 64 images 960-160 r8", kind="lora", n=64, hw=196, cin=960, cout=160, rank=8, adapters=12, type="f16", out="f32", runs=False),
        # prompts of a few requests in one batch, some of them without an adapter
        dict(name="lora 8192 tokens 4096-4096 r32", kind="lora", n=8192, hw=1, cin=4096, cout=4096, rank=32, adapters=16, type="bf16", out="bf16", runs=True),
        # a small fine-tuning step of odd sizes, float32 gradients in and out
        dict(name="lora grad 500 tokens 1000-1030 r12", kind="lora_grad", n=500, hw=1, cin=1000, cout=1030, rank=12, adapters=5, type="bf16", out="f32", runs=True),
        # a training batch that several adapters share
        dict(name="lora grad 8192 tokens 4096-4096 r16", kind="lora_grad", n=8192, hw=1, cin=4096, cout=4096, rank=16, adapters=8, type="bf16", out="bf16", runs=True),
        # one token's norm
        dict(name="norm 1x4096", kind="norm", rows=1, cols=4096, type="f16"),
        # the norm before a quantised projection
        dict(name="norm quant 2048x2048", kind="norm_quant", rows=2048, cols=2048, type="bf16"),
        # a training batch's norm, backwards
        dict(name="norm grad 8192x4096", kind="norm_grad", rows=8192, cols=4096, type="bf16"),
        # few rows of an odd width
        dict(name="norm grad 777x1031", kind="norm_grad", rows=777, cols=1031, type="f32"),
        # the two factors of a few adapters
        dict(name="adamw 12 tensors 32 bits", kind="adamw", tensors=12, mean=40000, bits=32, type="f32"),
        # a whole model's tensors, small vectors beside large matrices, moments in 8 bits
        dict(name="adamw 150 tensors 8 bits", kind="adamw", tensors=150, mean=500000, bits=8, type="bf16"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):  # channels: half of them whole tiles, the others anything
        v = log(lo, hi)
        return max(lo, v // 64 * 64) if rng.random() < 0.5 else v

    kind = rng.choice(["lora", "lora", "lora_grad", "norm", "norm_quant", "norm_grad", "adamw"])
    if kind in ("lora", "lora_grad"):
        hw = rng.choice([1, 1, 1, 49, 196])
        n = max(1, log(1, 8192) // hw)
        type = rng.choice(["bf16", "f16"])
        return dict(kind=kind, n=n, hw=hw, cin=width(64, 4096), cout=width(64, 4096), rank=rng.choice([4, 8, 12, 16, 16]),
                    adapters=rng.randint(1, 16 if kind == "lora" else 8), type=type, out=rng.choice([type, type, "f32"]) if kind == "lora" else rng.choice([type, "f32"]) if n * hw < 2000 else type,
                    runs=rng.random() < 0.5)
    if kind == "adamw":
        tensors = log(1, 150)
        return dict(kind=kind, tensors=tensors, mean=log(1000, min(2000000, 75000000 // tensors)), bits=rng.choice([8, 32]), type=rng.choice(["f32", "bf16"]))
    return dict(kind=kind, rows=log(1, 8192), cols=width(64, 4096), type=rng.choice(["f32", "bf16", "f16"]) if kind != "norm_grad" else rng.choice(["bf16", "f16", "f32"]))


def sizes(case):
    """Elements of each tensor of an AdamW case: one large matrix in four, vectors between them; the sum does not depend on the seed."""
    n, mean = case["tensors"], case["mean"]
    part = [(0.13, 1.9, 0.47, 1.5)[i % 4] for i in range(n)]
    return [max(1, int(mean * n * p / sum(part)) + i % 7) for i, p in enumerate(part)]


def spread(case, r, device):
    """Which adapter each batch element takes, -1 for none: in runs as prompts lie in a batch, or mixed."""
    n, adapters = case["n"], case["adapters"]
    if case["runs"]:
        cuts = torch.rand(adapters + 1, generator=r, device=device).cumsum(0)
        edge = (cuts / cuts[-1] * n).long()
        which = torch.bucketize(torch.arange(n, device=device), edge[:-1], right=True)
        which = torch.where(which >= adapters, torch.full_like(which, -1), which)
    else:
        which = torch.arange(n, device=device) % adapters
        which = which[torch.randperm(n, generator=r, device=device)]
    return which.int()


def pack(w):
    """Ternary [rows][k] codes in the library's packed form: 16 to a word, weight 16j+4d+b at bits 8b+2d, 8b+2d+1."""
    rows, k = w.shape
    padded = torch.zeros(rows, (k + 15) // 16 * 16, dtype=torch.int64, device=w.device)
    padded[:, :k] = w.long() & 3
    at = (8 * torch.arange(4, device=w.device)[None, :] + 2 * torch.arange(4, device=w.device)[:, None]).reshape(-1)
    words = (padded.view(rows, -1, 16) << at).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int().view(torch.uint8).reshape(-1)


def prepare(case, seed):
    device = torch.device("cuda")
    r = torch.Generator(device=device)
    r.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=r, device=device)  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=r, device=device)  # noqa: E731
    kind = case["kind"]
    if kind in ("lora", "lora_grad"):
        n, hw, cin, cout, rank, adapters = (case[k] for k in ("n", "hw", "cin", "cout", "rank", "adapters"))
        type, m = TYPES[case["type"]], n * hw
        s = dict(case=case)
        s["x"] = (randn(n, hw, 1, cin) * 40).round().clamp(-127, 127).to(torch.int8)
        s["w"] = torch.randint(-1, 2, (cout, cin), generator=r, device=device, dtype=torch.int8)
        s["step"] = 0.02 + 0.02 * rand(n)
        s["w_scale"] = (0.5 + rand(cout)) / math.sqrt(cin)
        s["a"] = (randn(adapters, rank, cin) / math.sqrt(cin)).to(type)
        s["b"] = (randn(adapters, rank, cout) / math.sqrt(rank)).to(type)
        s["scale"] = 0.5 + rand(adapters)
        s["index"] = spread(case, r, device)
        if kind == "lora":
            s["bias"] = randn(cout) * 0.1
            s["packed"] = pack(s["w"])
        else:
            s["packed"] = pack(s["w"].t())
            s["dy"] = randn(n, hw, 1, cout).to(TYPES[case["out"]])
            hid = torch.zeros(n, hw, rank, device=device)
            for l in range(adapters):
                at = s["index"] == l
                hid[at] = (s["x"][at].reshape(-1, cin).float() @ s["a"][l].float().t()).view(-1, hw, rank) * s["step"][at][:, None, None]
            s["hid"] = hid.view(m, rank)
        return s
    if kind.startswith("norm"):
        rows, cols, type = case["rows"], case["cols"], TYPES[case["type"]]
        s = dict(case=case, x=(randn(rows, cols) * (0.5 + rand(rows, 1)) + 0.3 * randn(rows, 1)).to(type), weight=1 + 0.2 * randn(cols), bias=0.2 * randn(cols))
        if kind == "norm_grad":
            s["dy"] = randn(rows, cols).to(type)
            x = s["x"].double()
            s["mean"] = x.mean(1).float()
            s["rstd"] = (1 / (x.var(1, unbiased=False) + NORM_EPS).sqrt()).float()
        return s
    count = sizes(case)
    blocks = [(k + BLOCK - 1) // BLOCK for k in count]
    total = sum(blocks)
    live = torch.zeros(total * BLOCK, device=device)
    at = 0
    s = dict(case=case, start=[], count=count, blocks=total)
    for k, b in zip(count, blocks):
        live[at * BLOCK:at * BLOCK + k] = 1
        s["start"].append(at * BLOCK)
        at += b
    s["p"] = randn(total * BLOCK) * 0.02 * live
    s["g"] = (randn(total * BLOCK) * 1e-3 * live).to(TYPES[case["type"]])
    m = randn(total * BLOCK) * 1e-4 * live
    v = (randn(total * BLOCK) * 1e-3 * live).square() + 1e-8 * live
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["m_scale"], s["v"], s["v_scale"] = encode(m.view(-1, BLOCK), v.sqrt().view(-1, BLOCK))
    return s


def encode(m, root):
    """The moments of whole blocks in 8 bits: signed codes whose squares stand for m, unsigned ones whose squares stand for the root of v."""
    top, high = m.abs().amax(1), root.amax(1)
    m_scale, v_scale = top * (1 / 16129), high * (1 / 65025)
    m_inv, v_inv = torch.full_like(top, 16129) / top, torch.full_like(high, 65025) / high
    small, low = top < 2.0 ** -100, high < 2.0 ** -100
    code = (m.abs() * m_inv[:, None]).sqrt().round().clamp(max=127) * m.sign()
    coder = torch.maximum((root * v_inv[:, None]).sqrt().round().clamp(max=255), (root > 0).float())
    code = torch.where(small[:, None], torch.zeros_like(code), code).to(torch.int8)
    coder = torch.where(low[:, None], torch.zeros_like(coder), coder).to(torch.uint8)
    zero = torch.zeros_like(top)
    return code.view(-1), torch.where(small, zero, m_scale), coder.view(-1), torch.where(low, zero, v_scale)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2505_03254_amd as P
        if kind == "lora":
            y, hid = P.prom_pw_conv_lora(s["x"], s["packed"], case["cout"], s["step"], s["w_scale"], s["bias"],
                                         P.Lora(s["a"], s["b"], s["scale"], s["index"]), dtype=TYPES[case["out"]], want_hid=True)
            return y, hid
        if kind == "lora_grad":
            return P.prom_pw_conv_lora_backward(s["dy"], s["x"], s["step"], s["packed"], s["w_scale"], P.Lora(s["a"], s["b"], s["scale"], s["index"]), s["hid"])
        if kind == "norm":
            return P.prom_layernorm(s["x"], s["weight"], s["bias"], NORM_EPS)
        if kind == "norm_quant":
            q, step, mean, rstd = P.prom_layernorm_quant(s["x"], s["weight"], s["bias"], NORM_EPS, QUANT_EPS)
            return q * step[:, None], step, mean, rstd
        if kind == "norm_grad":
            return P.prom_layernorm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"])
        if "tensors" not in s:
            part = lambda t, i: t[s["start"][i]:s["start"][i] + s["count"][i]]  # noqa: E731
            block = lambda t, i: t[s["start"][i] // BLOCK:(s["start"][i] + s["count"][i] + BLOCK - 1) // BLOCK]  # noqa: E731
            s["tensors"] = P.AdamWTensors([
                P.AdamWTensor(part(s["p"], i), part(s["g"], i), part(s["m"], i), part(s["v"], i),
                              *((block(s["m_scale"], i), block(s["v_scale"], i)) if case["bits"] == 8 else ()))
                for i in range(len(s["count"]))])
        s["tensors"].step(STEP, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY)
        if case["bits"] == 32:
            return s["p"], s["m"], s["v"]
        if "m32" not in s:
            s["m32"], s["v32"] = torch.zeros_like(s["p"]), torch.zeros_like(s["p"])
            s["to"] = s["tensors"].moment_targets([(s["m32"][a:a + k], s["v32"][a:a + k]) for a, k in zip(s["start"], s["count"])])
        s["tensors"].moments(s["to"])
        return s["p"], s["m32"], s["v32"]
    if kind in ("lora", "lora_grad"):
        hw, cin, cout, rank, adapters = (case[k] for k in ("hw", "cin", "cout", "rank", "adapters"))
        x = s["x"].view(-1, cin).float()
        w = s["w"].float()
        a, b = s["a"].view(-1, cin).float(), s["b"].view(-1, cout).float()
        which = s["index"].long().repeat_interleave(hw)
        step = s["step"].repeat_interleave(hw)[:, None]
        mask = (which[:, None] == torch.arange(adapters, device=x.device)).repeat_interleave(rank, 1)  # [m][adapters * rank]
        scale = s["scale"].repeat_interleave(rank)
        if kind == "lora":
            hid = x @ a.t() * step * mask
            y = (x @ w.t()) * s["w_scale"] * step + s["bias"] + (hid * scale) @ b
            return y.to(TYPES[case["out"]]).view(case["n"], hw, 1, cout), hid.view(-1, adapters, rank).sum(1)
        dy = s["dy"].view(-1, cout).float()
        g = dy @ b.t() * mask * scale
        dx = (dy * s["w_scale"]) @ w + g @ a
        da = (g * step).t() @ x
        db = (s["hid"].repeat(1, adapters) * mask * scale).t() @ dy
        return dx.to(s["dy"].dtype).view(s["x"].shape), da.view(adapters, rank, cin), db.view(adapters, rank, cout)
    if kind == "norm":
        x = s["x"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = 1 / (d.square().mean(1) + NORM_EPS).sqrt()
        return (d * rstd[:, None] * s["weight"] + s["bias"]).to(s["x"].dtype), mean, rstd
    if kind == "norm_quant":  # the moments in 64 bits: a code must not hang on the order of a sum
        x = s["x"].double()
        mean = x.mean(1)
        rstd = (1 / ((x - mean[:, None]).square().mean(1) + NORM_EPS).sqrt()).float()
        mean = mean.float()
        y = (s["x"].float() - mean[:, None]) * rstd[:, None] * s["weight"] + s["bias"]
        top = y.abs().amax(1).clamp(min=QUANT_EPS)
        most = torch.full_like(top, 127)
        q = (y * (most / top)[:, None]).round().clamp(-128, 127)
        step = top / most
        return q * step[:, None], step, mean, rstd
    if kind == "norm_grad":
        dy = s["dy"].float()
        hat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"]
        dx = (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True)) * s["rstd"][:, None]
        return dx.to(s["dy"].dtype), (dy * hat).sum(0), dy.sum(0)
    g = s["g"].float()
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        c, r = s["m"].float().view(-1, BLOCK), s["v"].float().view(-1, BLOCK)
        m = (c * c.abs() * s["m_scale"][:, None]).view(-1)
        v = (r * r * s["v_scale"][:, None]).view(-1)
        v = v * v
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * (1 - BETA2) * g
    root = v.sqrt()
    denom = root * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS
    s["p"].copy_(s["p"] * (1 - LR * DECAY) - m * (LR / (1 - BETA1 ** STEP)) / denom)
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return s["p"], s["m"], s["v"]
    s["m"], s["m_scale"], s["v"], s["v_scale"] = encode(m.view(-1, BLOCK), root.view(-1, BLOCK))
    c, r = s["m"].float().view(-1, BLOCK), s["v"].float().view(-1, BLOCK)
    root = (r * r * s["v_scale"][:, None]).view(-1)
    return s["p"], (c * c.abs() * s["m_scale"][:, None]).view(-1), root * root


def work(case):
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if kind in ("lora", "lora_grad"):
        m = case["n"] * case["hw"]
        cin, cout, rank = case["cin"], case["cout"], case["rank"]
        used = min(case["adapters"], case["n"])
        both, out = cin + cout, size[case["out"]]
        weights = (cin * cout) // 4 + 4 * cout + used * rank * both * size[case["type"]]
        if kind == "lora":
            return {"bytes": m * cin + m * cout * out + weights + 4 * m * rank + 4 * cout + 8 * case["n"], "flops": 2 * m * (cin * cout + rank * both)}
        return {"bytes": m * cin + m * both * out + weights + 4 * m * rank + 8 * case["n"] + 4 * case["adapters"] * rank * both,
                "flops": 2 * m * (cin * cout + 2 * rank * both)}
    if kind.startswith("norm"):
        rows, cols, each = case["rows"], case["cols"], size[case["type"]]
        if kind == "norm_grad":
            return {"bytes": 3 * rows * cols * each + 8 * rows + 12 * cols, "flops": 14 * rows * cols}
        return {"bytes": rows * cols * (each + (each if kind == "norm" else 4)) + 8 * rows + 8 * cols, "flops": 8 * rows * cols}
    total = sum(sizes(case))
    return {"bytes": total * (8 + size[case["type"]] + (16 if case["bits"] == 32 else 4 + 8)), "flops": 16 * total}


def exact(case, seed):
    """From the definitions, in 64 bits: adapter by adapter, tensor by tensor."""
    s = prepare(case, seed)
    kind = case["kind"]
    D = torch.float64
    if kind in ("lora", "lora_grad"):
        n, hw, cin, cout, rank, adapters = (case[k] for k in ("n", "hw", "cin", "cout", "rank", "adapters"))
        real = s["x"].to(D).view(n, hw, cin) * s["step"].to(D)[:, None, None]  # what the int8 activations stand for
        kernel = s["w"].to(D) * s["w_scale"].to(D)[:, None]
        if kind == "lora":
            y = torch.matmul(real.view(-1, cin), kernel.t().contiguous()).view(n, hw, cout) + s["bias"].to(D)
            hid = torch.zeros(n, hw, rank, dtype=D, device=y.device)
            for l in range(adapters):
                rows = (s["index"] == l).nonzero().view(-1)
                if rows.numel():
                    h = torch.matmul(real[rows].reshape(-1, cin), s["a"][l].to(D).t().contiguous())
                    hid[rows] = h.view(-1, hw, rank)
                    y[rows] += s["scale"][l].to(D) * torch.matmul(h, s["b"][l].to(D)).view(-1, hw, cout)
            return y.view(n, hw, 1, cout), hid.view(-1, rank)
        dy = s["dy"].to(D).view(n, hw, cout)
        dx = torch.matmul(dy.view(-1, cout), kernel).view(n, hw, cin)
        da = torch.zeros(adapters, rank, cin, dtype=D, device=dx.device)
        db = torch.zeros(adapters, rank, cout, dtype=D, device=dx.device)
        for l in range(adapters):
            rows = (s["index"] == l).nonzero().view(-1)
            if rows.numel():
                d = dy[rows].reshape(-1, cout)
                g = s["scale"][l].to(D) * torch.matmul(d, s["b"][l].to(D).t().contiguous())
                dx[rows] += torch.matmul(g, s["a"][l].to(D)).view(-1, hw, cin)
                da[l] = torch.matmul(g.t().contiguous(), real[rows].reshape(-1, cin))
                db[l] = s["scale"][l].to(D) * torch.matmul(s["hid"].to(D).view(n, hw, rank)[rows].reshape(-1, rank).t().contiguous(), d)
        return dx.view(n, hw, 1, cin), da, db
    if kind.startswith("norm"):
        x, weight, bias = (s[k].to(D) for k in ("x", "weight", "bias"))
        if kind == "norm_grad":
            dy, mean, rstd = s["dy"].to(D), s["mean"].to(D)[:, None], s["rstd"].to(D)[:, None]
            hat, g, cols = (x - mean) * rstd, dy * weight, case["cols"]
            along = (g * hat).sum(1, keepdim=True) / cols
            return rstd * (g - g.sum(1, keepdim=True) / cols - hat * along), (dy * hat).sum(0), dy.sum(0)
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = (var + NORM_EPS).rsqrt()
        y = (x - mean[:, None]) * rstd[:, None] * weight + bias
        if kind == "norm":
            return y, mean, rstd
        step = y.abs().amax(1).clamp(min=QUANT_EPS) / 127
        return None, step, mean, rstd  # the codes are fixed by float32 operations: no value of their own
    p, g = s["p"].to(D), s["g"].to(D)
    if case["bits"] == 32:
        m, v = s["m"].to(D), s["v"].to(D)
    else:
        spread_m, spread_v = s["m_scale"].to(D).repeat_interleave(BLOCK), s["v_scale"].to(D).repeat_interleave(BLOCK)
        m = s["m"].to(D).abs().square() * s["m"].to(D).sign() * spread_m
        v = (s["v"].to(D).square() * spread_v).square()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    hat = m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
    p = p - LR * DECAY * p - LR * hat
    return (p, m, v) if case["bits"] == 32 else (p, None, None)  # the 8-bit moments are codes: fixed by float32 operations
