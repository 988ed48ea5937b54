"""The calls of the float side at sizes that take their large tiles, and where offsets pass 32 bits."""
import numpy as np
import pytest

from gpu_util import torch_cuda
from test_gpu_lora import check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2505_03254_amd as P
    P.load_library()
    return P


@pytest.mark.parametrize("ti", range(3))
@pytest.mark.parametrize("rows,cin,cout,rank", [
    (16400, 200, 1030, 20), (4100, 200, 1030, 20), (2100, 72, 1030, 12),   # forward: 128, 64 and 32 rows x 256 channels
    (16400, 1030, 72, 20), (4100, 1030, 200, 20), (2100, 1030, 72, 12),    # and the gradient of the activations
    (900, 1030, 1200, 40)])                                               # both by two groups of wavefronts
def test_tiles(P, rows, cin, cout, rank, ti):
    torch = torch_cuda()
    t, o = [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32), (torch.float16, torch.float16)][ti]
    check(P, make(rows + rank, rows, 1, 1, cin, cout, rank, 5, t, dy_type=o), f"{rows} {cin} {cout} {t} {o} ")


def test_adapter_layer_beyond_2_31_elements(P):
    """y and dy of 2.2e9 elements: the first and the last rows against the definition in 64 bits, relative to the magnitudes of the sums:
    y is rounded once (2^-8), with hid in two planes (2^-16) and float32 sums of 68 terms; dx twice (dy * w_scale and the result, 2^-7)."""
    torch = torch_cuda()
    rows, cin, cout, rank = (1 << 20) + 64, 64, 2112, 4
    r = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-128, 128, (rows, 1, 1, cin), generator=r, device="cuda", dtype=torch.int8)
    wt = torch.randint(-1, 2, (cout, cin), generator=r, device="cuda", dtype=torch.int8)
    step, ws = torch.rand(rows, generator=r, device="cuda") * 0.02 + 0.01, torch.rand(cout, generator=r, device="cuda") * 0.1 + 0.05
    lora = P.Lora(torch.randn(2, rank, cin, generator=r, device="cuda").bfloat16(), torch.randn(2, rank, cout, generator=r, device="cuda").bfloat16() * 0.1,
                  torch.ones(2, device="cuda"), torch.randint(-1, 2, (rows,), generator=r, device="cuda", dtype=torch.int32))
    wp, wtp = (torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(v))).cuda() for v in (wt.cpu().numpy(), wt.cpu().numpy().T))
    y, hid = P.prom_pw_conv_lora(x, wp, cout, step, ws, None, lora, want_hid=True)
    assert y.numel() > 1 << 31
    dy = torch.randn(rows, 1, 1, cout, generator=r, device="cuda", dtype=torch.bfloat16)
    dx, da, db = P.prom_pw_conv_lora_backward(dy, x, step, wtp, ws, lora, hid)
    torch.cuda.synchronize()
    D = torch.float64
    w = wt.to(D) * ws.to(D)[:, None]
    for at in (slice(0, 40), slice(rows - 40, rows)):
        real = x[at].view(40, cin).to(D) * step[at].to(D)[:, None]
        idx = lora.index[at].long()
        has = (idx >= 0).to(D)[:, None]
        a, b = lora.a.to(D)[idx.clamp(min=0)], lora.b.to(D)[idx.clamp(min=0)]
        h = (a * real[:, None, :]).sum(2) * has
        want = real @ w.t().contiguous() + (b * h[:, :, None]).sum(1)
        size = real.abs() @ w.abs().t().contiguous() + (b.abs() * h.abs()[:, :, None]).sum(1)
        assert ((y[at].view(40, cout).to(D) - want).abs() <= (2.0 ** -8 + 2.0 ** -15) * size).all()
        d = dy[at].view(40, cout).to(D)
        g = (b * d[:, None, :]).sum(2) * has
        want = d @ w + (a * g[:, :, None]).sum(1)
        size = d.abs() @ w.abs() + (a.abs() * g.abs()[:, :, None]).sum(1)
        assert ((dx[at].view(40, cin).to(D) - want).abs() <= (2.0 ** -7 + 2.0 ** -11) * size).all()
    # db of a million rows in float32: sums of 128 rows, then of their 4000 sums: (128 + 4100) * 2^-24 of the magnitudes
    for l in range(2):
        at = (lora.index == l).nonzero().view(-1)
        want, size = torch.zeros(rank, cout, dtype=D, device="cuda"), torch.zeros(rank, cout, dtype=D, device="cuda")
        for part in at.split(1 << 16):
            hh, dd = hid[part].to(D).t().contiguous(), dy.view(rows, cout)[part].to(D)
            want += hh @ dd
            size += hh.abs() @ dd.abs()
        assert ((db[l].to(D) - want).abs() <= 4300 * 2.0 ** -24 * size).all()


def test_norm_beyond_2_31_elements(P):
    torch = torch_cuda()
    rows, cols = 66000, 32768
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 1 << 31
    r = torch.Generator(device="cuda").manual_seed(2)
    row = torch.randn(64, cols, generator=r, device="cuda").bfloat16()
    x[:64], x[-64:] = row, row
    x[64:-64] = row[0]
    y, mean, rstd = P.prom_layernorm(x)
    small = P.prom_layernorm(row)
    assert torch.equal(y[:64], small[0]) and torch.equal(y[-64:], small[0]) and torch.equal(y[rows // 2], small[0][0])
    dx, _, db = P.prom_layernorm_backward(y, x, None, mean, rstd)
    ds, _, _ = P.prom_layernorm_backward(small[0], row, None, *small[1:])
    assert torch.equal(dx[:64], ds) and torch.equal(dx[-64:], ds) and torch.equal(dx[rows // 2], ds[0])
    del dx, y
    q, step, _, _ = P.prom_layernorm_quant(x)
    qs, ss, _, _ = P.prom_layernorm_quant(row)
    assert torch.equal(q[-64:], qs) and torch.equal(step[-64:], ss)


def test_adamw_beyond_2_31_elements(P):
    torch = torch_cuda()
    n = (1 << 31) + 3000
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = (torch.zeros((n + 255) // 256, device="cuda") for _ in range(2))
    k = 3000 + 512  # from a block's start, 2^31 - 512, on
    g[-k:] = torch.randn(k, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()
    p[-k:] = 1.0
    small = [t[-k:].clone() for t in (p, g, m, v)] + [torch.zeros((k + 255) // 256, device="cuda") for _ in range(2)]
    one, two = P.AdamWTensors([P.AdamWTensor(p, g, m, v, ms, vs)]), P.AdamWTensors([P.AdamWTensor(*small)])
    for t in (1, 2):
        one.step(t)
        two.step(t)
    for a, b in zip((p, m, v), (small[0], small[2], small[3])):
        assert torch.equal(a[-k:], b) and not a[:1 << 20].any() and not a[1 << 30:(1 << 30) + 4096].any()
    assert torch.equal(ms[-small[4].numel():], small[4]) and torch.equal(vs[-small[5].numel():], small[5])
