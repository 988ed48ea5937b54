"""Layer norm, its int8 form and its gradients against the definition in 64 bits.

Tolerances: h = (x - mean) * rstd carries the float32 errors of mean (n/2 additions deep at most 2^-24 each of mean|x|) and
rstd, all relative to |x| + |mean| over the spread; with sums taken pairwise over lanes, 64 * 2^-24 covers every width here.
Results are rounded once to their type (eps / 2)."""
import pytest

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu

SUM = 64 * 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    import paper_2505_03254_amd as P
    P.load_library()
    return P


def make(seed, rows, cols, dtype, offset=0.5):
    torch = torch_cuda()
    r = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, cols, generator=r) * (0.2 + torch.rand(rows, 1, generator=r)) + offset * torch.randn(rows, 1, generator=r)).to(dtype)
    return x, 1 + 0.3 * torch.randn(cols, generator=r), torch.randn(cols, generator=r), torch.randn(rows, cols, generator=r).to(dtype)


def moments(x, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    return mean, 1 / (var + eps).sqrt()


SIZES = [(1, 1), (1, 2), (3, 7), (1, 4096), (5, 64), (1030, 65), (4, 511), (9, 512), (2, 513), (7, 1031), (3, 2049), (1025, 1030), (2, 4097), (3, 8192),
         (2, 16385), (1, 32768), (4100, 33)]


@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(P, rows, cols, t):
    torch = torch_cuda()
    dtype = getattr(torch, t)
    x, w, b, _ = make(rows * 7 + cols, rows, cols, dtype)
    for weight, bias in ((w, b), (None, b), (w, None)):
        y, mean, rstd = P.prom_layernorm(x.cuda(), None if weight is None else weight.cuda(), None if bias is None else bias.cuda(), 1e-5)
        m, r = moments(x, 1e-5)
        ww = torch.ones(cols).double() if weight is None else weight.double()
        bb = torch.zeros(cols).double() if bias is None else bias.double()
        h = (x.double() - m) * r
        want = h * ww + bb
        size = (x.double().abs() + x.double().abs().mean(1, keepdim=True)) * r * ww.abs() + h.abs() * ww.abs() + bb.abs()
        assert ((y.cpu().double() - want).abs() <= torch.finfo(dtype).eps / 2 * want.abs() + SUM * size + torch.finfo(dtype).tiny).all()
        assert ((mean.cpu().double() - m[:, 0]).abs() <= SUM * x.double().abs().mean(1)).all()
        spread = (x.double().abs().mean(1) * r[:, 0]).clamp(min=1)  # the mean's error moves the variance in proportion
        assert ((rstd.cpu().double() / r[:, 0] - 1).abs() <= SUM * spread).all()


@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantised_rows(P, rows, cols, t):
    """Codes and steps equal the float32 operations of the interface, made one by one on the CPU from the kernel's own mean
    and rstd; those are the 64-bit moments rounded once (one step of float32 either way where 64 bits end at a border)."""
    torch = torch_cuda()
    dtype = getattr(torch, t)
    x, w, b, _ = make(rows * 5 + cols, rows, cols, dtype, offset=3.0)
    q, step, mean, rstd = (v.cpu() for v in P.prom_layernorm_quant(x.cuda(), w.cuda(), b.cuda(), 1e-5, 1e-5))
    m, r = moments(x, 1e-5)
    assert ((mean.double() - m[:, 0]).abs() <= 2.0 ** -24 * (1 + 1e-6) * m[:, 0].abs() + 1e-14).all()
    assert ((rstd.double() / r[:, 0] - 1).abs() <= 2.0 ** -24 * (1 + 1e-6) + 1e-9 * (m[:, 0] * r[:, 0]).square() * 2.0 ** -20).all()
    y = (x.float() - mean[:, None]) * rstd[:, None] * w + b
    top = y.abs().amax(1).clamp(min=1e-5)
    most = torch.full_like(top, 127)
    assert torch.equal(step, top / most)
    assert torch.equal(q, (y * (most / top)[:, None]).round().clamp(-128, 127).to(torch.int8))


@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,cols", SIZES + [(3000, 130)])
def test_gradients(P, rows, cols, t):
    torch = torch_cuda()
    dtype = getattr(torch, t)
    x, w, _, dy = make(rows * 3 + cols, rows, cols, dtype)
    m, r = moments(x, 1e-5)
    mean, rstd = m[:, 0].float(), r[:, 0].float()
    m, r = mean.double()[:, None], rstd.double()[:, None]
    h = (x.double() - m) * r
    for weight in (w, None):
        ww = torch.ones(cols).double() if weight is None else weight.double()
        g = dy.double() * ww
        want = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        hs = (x.double().abs() + m.abs()) * r
        size = r * (g.abs() + g.abs().mean(1, keepdim=True) + 2 * hs * (g.abs() * hs).mean(1, keepdim=True))
        dx, dw, db = P.prom_layernorm_backward(dy.cuda(), x.cuda(), None if weight is None else weight.cuda(), mean.cuda(), rstd.cuda())
        assert ((dx.cpu().double() - want).abs() <= torch.finfo(dtype).eps / 2 * want.abs() + SUM * size + torch.finfo(dtype).tiny).all()
        deep = (rows + 16) * 2.0 ** -24
        assert ((dw.cpu().double() - (dy.double() * h).sum(0)).abs() <= deep * (dy.double().abs() * hs).sum(0)).all()
        assert ((db.cpu().double() - dy.double().sum(0)).abs() <= deep * dy.double().abs().sum(0)).all()
        for k in range(1, 7):
            parts = P.prom_layernorm_backward(dy.cuda(), x.cuda(), None if weight is None else weight.cuda(), mean.cuda(), rstd.cuda(), bool(k & 1), bool(k & 2), bool(k & 4))
            for have, whole in zip(parts, (dx, dw, db)):
                assert have is None or torch.equal(have, whole)


def test_gradient_against_differences(P):
    """Along a random direction, by central differences of the 64-bit definition (error h^2 of its third derivative: 1e-8 of the parts)."""
    torch = torch_cuda()
    x, w, b, dy = make(1, 6, 200, torch.float32)
    d = torch.randn(x.shape, generator=torch.Generator().manual_seed(2)).double()

    def loss(x):
        m, r = moments(x, 1e-5)
        return (((x - m) * r * w.double() + b.double()) * dy.double()).sum()

    e = 1e-4
    want = (loss(x.double() + e * d) - loss(x.double() - e * d)) / (2 * e)
    y, mean, rstd = P.prom_layernorm(x.cuda(), w.cuda(), b.cuda())
    dx, _, _ = P.prom_layernorm_backward(dy.cuda(), x.cuda(), w.cuda(), mean, rstd)
    size = float((dx.cpu().double() * d).abs().sum())
    assert abs(float((dx.cpu().double() * d).sum() - want)) <= (1e-6 + 2 * SUM) * size


def test_rows_with_infinities_and_nan_stay_alone(P):
    torch = torch_cuda()
    x, w, b, dy = make(4, 40, 300, torch.float32)
    clean = P.prom_layernorm(x.cuda(), w.cuda(), b.cuda())
    cq = P.prom_layernorm_quant(x.cuda(), w.cuda(), b.cuda())
    x[3, 7], x[9, 299], x[20] = float("nan"), float("inf"), 0.0
    y, mean, rstd = P.prom_layernorm(x.cuda(), w.cuda(), b.cuda())
    q, step, _, _ = P.prom_layernorm_quant(x.cuda(), w.cuda(), b.cuda())
    keep = torch.ones(40, dtype=torch.bool)
    keep[[3, 9, 20]] = False
    keep = keep.cuda()
    assert torch.equal(y[keep], clean[0][keep]) and torch.equal(q[keep], cq[0][keep])
    assert y[3].isnan().all() and not step[3].isfinite() and not step[9].isfinite()
    assert torch.equal(y[20].cpu(), b)  # a constant row: the bias


def test_rows_behind_the_last_stay_as_they_were(P):
    torch = torch_cuda()
    x, w, b, dy = make(8, 6, 1031, torch.bfloat16)
    big = torch.full((7, 1031), 5.0, dtype=torch.bfloat16, device="cuda")
    y, _, _ = P.prom_layernorm(x[:5].cuda(), w.cuda(), b.cuda(), y=big[:5])
    assert (big[5:] == 5).all() and torch.equal(y, P.prom_layernorm(x.cuda(), w.cuda(), b.cuda())[0][:5])
    q = torch.full((7, 1031), 9, dtype=torch.int8, device="cuda")
    P.prom_layernorm_quant(x[:5].cuda(), w.cuda(), b.cuda(), q=q[:5])
    assert (q[5:] == 9).all()


def test_captured(P):
    torch = torch_cuda()
    x, w, b, dy = (v.cuda() for v in make(6, 300, 1000, torch.bfloat16))

    def run():
        y, mean, rstd = P.prom_layernorm(x, w, b)
        return (y,) + P.prom_layernorm_backward(dy, x, w, mean, rstd) + P.prom_layernorm_quant(x, w, b)

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    for i in range(3):
        x.add_(0.25)
        g.replay()
        torch.cuda.synchronize()
        for u, v in zip(got, run()):
            assert torch.equal(u, v)
