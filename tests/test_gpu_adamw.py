"""AdamW over many tensors: equal, bit for bit, to the float32 operations of the interface made one by one on the CPU, and near the
definition in 64 bits."""
import math

import numpy as np
import pytest

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2505_03254_amd as P
    P.load_library()
    return P


SIZES = [1, 3, 4, 255, 256, 257, 1000, 4095, 4096, 4097, 50000, 131]
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


def sqrt(t):
    """Correctly rounded; torch's own on the CPU is off by one step for 6 in 1000 values."""
    import torch
    return torch.from_numpy(np.sqrt(t.numpy()))


def decode(c, scale, n):
    import torch
    c = c.float()
    return c * c.abs() * scale.repeat_interleave(256)[:n]


def blocks(t):
    import torch
    n = t.numel()
    out = torch.zeros((n + 255) // 256 * 256)
    out[:n] = t
    return out.view(-1, 256)


def encode(t, most):
    """t: m (most 127) or the root of v (most 255)."""
    import torch
    n, b = t.numel(), blocks(t)
    top = b.abs().amax(1)
    small = top < 2.0 ** -100
    inv = torch.full_like(top, most * most) / top
    c = sqrt(b.abs() * inv[:, None]).round().clamp(max=most)
    if most == 255:
        c = torch.maximum(c, (b > 0).float())
    c = torch.where(small[:, None], torch.zeros_like(c), c * b.sign())
    scale = torch.where(small, torch.zeros_like(top), top * torch.tensor(1 / (most * most), dtype=torch.float32))
    return c.view(-1)[:n].to(torch.int8 if most == 127 else torch.uint8), scale


def step_by_hand(s, t, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """One step in float32, one rounding per operation (what float32 tensors on the CPU do, operation by operation)."""
    import torch
    f = lambda v: torch.tensor(v, dtype=torch.float64).float()  # noqa: E731
    p, g = s["p"].float(), s["g"].float() * f(grad_scale)
    n = p.numel()
    if s["bits"] == 8:
        m, root = decode(s["m"], s["ms"], n), decode(s["v"], s["vs"], n)
        v = root * root
    else:
        m, v = s["m"], s["v"]
    m = m * f(beta1) + g * f(1 - beta1)
    v = v * f(beta2) + g * f(1 - beta2) * g
    root = sqrt(v)
    denom = root * f(1 / math.sqrt(1 - beta2 ** t)) + f(eps)
    p = p * f(1 - lr * weight_decay) - m * f(lr / (1 - beta1 ** t)) / denom
    out = dict(s, p=p.to(s["p"].dtype), p32=p)
    if s["bits"] == 8:
        out["m"], out["ms"] = encode(m, 127)
        out["v"], out["vs"] = encode(root, 255)
    else:
        out["m"], out["v"] = m, v
    return out


def make(seed, n, bits, ptype, gtype, copy=None):
    import torch
    r = torch.Generator().manual_seed(seed)
    s = dict(bits=bits, p=torch.randn(n, generator=r).to(ptype), g=(torch.randn(n, generator=r) * 10.0 ** (torch.rand(n, generator=r) * 4 - 4)).to(gtype))
    m, v = torch.randn(n, generator=r) * 0.01, torch.rand(n, generator=r) * 1e-4
    if bits == 8:
        s["m"], s["ms"] = encode(m, 127)
        s["v"], s["vs"] = encode(v.sqrt(), 255)
    else:
        s["m"], s["v"] = m, v
    if copy is not None:
        s["copy"] = torch.zeros(n, dtype=copy)
    return s


def upload(P, s):
    c = {k: v.cuda() if hasattr(v, "cuda") else v for k, v in s.items()}
    return c, P.AdamWTensor(c["p"], c["g"], c["m"], c["v"], c.get("ms"), c.get("vs"), c.get("copy"))


def same(got, want, what=""):
    import torch
    for k in ("p", "m", "v", "ms", "vs"):
        if k in want:
            assert torch.equal(got[k].cpu(), want[k]), f"{what}{k}: {int((got[k].cpu() != want[k]).sum())} differ"
    if "copy" in want:
        assert torch.equal(got["copy"].cpu(), want["p32"].to(want["copy"].dtype)), what + "copy"


def test_many_tensors_of_every_kind_at_once(P):
    torch = torch_cuda()
    f32, bf16, f16 = torch.float32, torch.bfloat16, torch.float16
    kinds = [(f32, f32, None), (f32, bf16, bf16), (f32, f16, f16), (bf16, bf16, None), (f16, f32, None)]
    sets = [make(100 * i + j, n, bits, *kinds[(i + j) % 5]) for i, n in enumerate(SIZES) for j, bits in enumerate((8, 32))]
    up = [upload(P, s) for s in sets]
    opt = P.AdamWTensors([t for _, t in up])
    for step in (1, 2, 3, 1000):
        sets = [step_by_hand(s, step, **HYPER) for s in sets]
        opt.step(step, **HYPER)
        for i, ((c, _), s) in enumerate(zip(up, sets)):
            same(c, s, f"step {step} tensor {i} of {s['p'].numel()} in {s['bits']} bits: ")
    targets = opt.moment_targets([(torch.empty(s["p"].numel(), device="cuda"), torch.empty(s["p"].numel(), device="cuda")) for s in sets])
    for (m, v), s in zip(opt.moments(targets), sets):
        n = s["p"].numel()
        if s["bits"] == 8:
            root = decode(s["v"], s["vs"], n)
            assert torch.equal(m.cpu(), decode(s["m"], s["ms"], n)) and torch.equal(v.cpu(), root * root)
        else:
            assert torch.equal(m.cpu(), s["m"]) and torch.equal(v.cpu(), s["v"])


def test_against_the_definition(P):
    """In 32 bits: p' is made of four float32 operations beyond p and the update, the moments of three: 8 roundings of 2^-24 of the parts."""
    torch = torch_cuda()
    s = make(5, 5000, 32, torch.float32, torch.float32)
    c, t = upload(P, s)
    P.AdamWTensors([t]).step(7, **HYPER)
    D = torch.float64
    g, m, v, p = (s[k].to(D) for k in ("g", "m", "v", "p"))
    m1, v1 = 0.9 * m + 0.1 * g, 0.99 * v + 0.01 * g * g
    up = HYPER["lr"] * (m1 / (1 - 0.9 ** 7)) / ((v1 / (1 - 0.99 ** 7)).sqrt() + 1e-8)
    part = HYPER["lr"] * ((0.9 * m.abs() + 0.1 * g.abs()) / (1 - 0.9 ** 7)) / ((v1 / (1 - 0.99 ** 7)).sqrt() + 1e-8)
    e = 8 * 2.0 ** -24
    assert ((c["m"].cpu().to(D) - m1).abs() <= e * (m.abs() + g.abs())).all()
    assert ((c["v"].cpu().to(D) - v1).abs() <= e * v1).all()
    assert ((c["p"].cpu().to(D) - (p * (1 - 3e-4) - up)).abs() <= e * (p.abs() + 2 * part)).all()


def test_state_from_zero_zero_gradients_and_tiny_ones(P):
    torch = torch_cuda()
    n = 1024
    s = dict(bits=8, p=torch.ones(n), g=torch.zeros(n), m=torch.zeros(n, dtype=torch.int8), v=torch.zeros(n, dtype=torch.uint8), ms=torch.zeros(4), vs=torch.zeros(4))
    s["g"][300] = 1e-3       # alone in its block
    s["g"][512:768] = 1e-35  # moments below what a block holds
    s["g"][800] = 1.0        # beside it, a value 1e-6 of it: a code of at least 1 in v
    s["g"][801] = 1e-6
    c, t = upload(P, s)
    opt = P.AdamWTensors([t])
    for step in (1, 2, 3):
        s = step_by_hand(s, step, **HYPER)
        opt.step(step, **HYPER)
        same(c, s, f"step {step} ")
    assert c["v"][801] >= 1 and not c["m"][512:768].any() and c["ms"][2] == 0 and c["p"].isfinite().all()


def test_not_finite(P):
    """A NaN or an infinite gradient: in 32 bits its element's, in 8 bits its block's moments are lost, no other block's."""
    torch = torch_cuda()
    for bits in (8, 32):
        s = make(9, 1000, bits, torch.float32, torch.float32)
        want = dict(s)
        s = dict(s, g=s["g"].clone())
        s["g"][10], s["g"][600] = float("nan"), float("inf")
        c, t = upload(P, s)
        opt = P.AdamWTensors([t])
        opt.step(3, **HYPER)
        want = step_by_hand(want, 3, **HYPER)
        other = torch.ones(1000, dtype=torch.bool)
        other[[10, 600]] = False
        assert torch.equal(c["p"].cpu()[other], want["p"][other]) and not c["p"][10].isfinite() and not c["p"][600].isfinite()
        if bits == 8:
            assert c["ms"].isnan().tolist() == [True, False, True, False] and c["vs"].isnan().tolist() == [True, False, True, False]
            opt.step(4, **HYPER)
            assert c["p"][:256].isnan().all() and c["p"][512:768].isnan().all() and c["p"][256:512].isfinite().all()


def test_gradients_scaled_and_schedule_on_the_device_captured(P):
    """step, lr and grad_scale in device memory, changed between the replays of one captured step, against the same
    values given by the host."""
    torch = torch_cuda()
    s = [make(i, n, bits, torch.float32, torch.bfloat16) for i, (n, bits) in enumerate(((700, 8), (5000, 32), (33, 32)))]
    one, two = [upload(P, k) for k in s], [upload(P, k) for k in s]
    a, b = P.AdamWTensors([t for _, t in one]), P.AdamWTensors([t for _, t in two])
    step, lr, gs = torch.ones(1, dtype=torch.int32, device="cuda"), torch.full((1,), 0.0, device="cuda"), torch.ones(1, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(step, lr=lr, grad_scale=gs, beta1=0.9, beta2=0.99)
    for t in range(1, 6):
        step.fill_(t)
        lr.fill_(0.5 ** t)
        gs.fill_(1.0 / t)
        graph.replay()
        b.step(t, lr=0.5 ** t, grad_scale=gs, beta1=0.9, beta2=0.99)
        torch.cuda.synchronize()
        for (c, _), (d, _) in zip(one, two):
            for k in ("p", "m", "v", "ms", "vs"):
                if k in c:
                    assert torch.equal(c[k], d[k]), (t, k)


def test_neighbours_of_a_tensor_stay_as_they_were(P):
    """Tensors at odd places of larger ones."""
    torch = torch_cuda()
    for n in (1, 255, 1027):
        s = make(n, n, 8, torch.bfloat16, torch.float16)
        flat = {k: torch.full((v.numel() + 3,), 9, dtype=v.dtype, device="cuda") for k, v in s.items() if k != "bits"}
        for k, v in flat.items():
            v[1:-2] = s[k].cuda()
        part = {k: v[1:-2] for k, v in flat.items()}
        P.AdamWTensors([P.AdamWTensor(part["p"], part["g"], part["m"], part["v"], part["ms"], part["vs"])]).step(2, **HYPER)
        same(part, step_by_hand(s, 2, **HYPER), f"{n} ")
        for k, v in flat.items():
            assert v[0] == 9 and (v[-2:] == 9).all(), k
