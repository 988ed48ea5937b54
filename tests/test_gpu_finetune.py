"""The calls together, as fine-tuning the adapters of a ternary layer makes them: float weights quantised once, then norm with int8 rows, layer
with adapters, gradients back through both, AdamW over adapters and norm; every step checked against the same step in 64 bits from the same
parameters (the int8 rows, which rounding decides, are taken from the run)."""
import numpy as np
import pytest

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu

ROWS, CIN, COUT, RANK, ADAPTERS = 150, 192, 136, 8, 3
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.01)


@pytest.fixture(scope="module")
def P():
    import paper_2505_03254_amd as P
    P.load_library()
    return P


class Model:
    """Frozen ternary weights, float32 master adapters with bf16 copies that the kernels read, norm weight and bias."""

    def __init__(self, P, bits):
        torch = torch_cuda()
        r = torch.Generator().manual_seed(3)
        randn = lambda *s: torch.randn(*s, generator=r).cuda()  # noqa: E731
        self.P, self.torch, self.bits = P, torch, bits
        self.packed, scale, codes = P.prom_quantize_pw_absmean(randn(COUT, CIN) / CIN ** 0.5, want_codes=True)
        self.codes = codes
        self.packed_t = torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(codes.cpu().numpy().T))).cuda()
        self.w_scale = 1 / scale
        self.params = dict(a=randn(ADAPTERS, RANK, CIN) / CIN ** 0.5, b=randn(ADAPTERS, RANK, COUT) * 0.1, weight=1 + 0.1 * randn(CIN), bias=0.1 * randn(CIN))
        self.copies = {k: self.params[k].bfloat16() for k in "ab"}
        self.grads = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self.scale = torch.rand(ADAPTERS, generator=r).cuda() + 0.5
        self.index = torch.randint(-1, ADAPTERS, (ROWS,), generator=r, dtype=torch.int32).cuda()
        self.x, self.target = randn(ROWS, CIN).bfloat16(), randn(ROWS, COUT).bfloat16()
        tensors = []
        self.state = {}
        for k, v in self.params.items():
            n = v.numel()
            if bits == 8:
                s = [torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros((n + 255) // 256, device="cuda"),
                     torch.zeros((n + 255) // 256, device="cuda")]
            else:
                s = [torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), None, None]
            self.state[k] = s
            tensors.append(P.AdamWTensor(v, self.grads[k], s[0], s[1], s[2], s[3], self.copies.get(k)))
        self.opt = P.AdamWTensors(tensors)
        self.step_no = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(self):
        P, p = self.P, self.params
        self.step_no += 1
        q, step, mean, rstd = P.prom_layernorm_quant(self.x, p["weight"], p["bias"])
        lora = P.Lora(self.copies["a"], self.copies["b"], self.scale, self.index)
        y, hid = P.prom_pw_conv_lora(q.view(ROWS, 1, 1, CIN), self.packed, COUT, step, self.w_scale, None, lora, want_hid=True)
        dy = (y.view(ROWS, COUT) - self.target) * (1.0 / ROWS)
        dx, da, db = P.prom_pw_conv_lora_backward(dy.view(ROWS, 1, 1, COUT), q.view(ROWS, 1, 1, CIN), step, self.packed_t, self.w_scale, lora, hid)
        dn, dweight, dbias = P.prom_layernorm_backward(dx.view(ROWS, CIN), self.x, p["weight"], mean, rstd)
        for k, g in dict(a=da, b=db, weight=dweight, bias=dbias).items():
            self.grads[k].copy_(g)
        self.opt.step(self.step_no, **HYPER)
        return dict(q=q, step=step, y=y.view(ROWS, COUT), dy=dy, dx=dn)

    def check(self, before, copies, out):
        """The gradients of this step in 64 bits from the parameters before it."""
        torch, D = self.torch, torch_cuda().float64
        c = lambda t: t.detach().cpu().to(D)  # noqa: E731
        x, w = c(self.x), c(self.codes) * c(self.w_scale)[:, None]
        mean = x.mean(1, keepdim=True)
        rstd = 1 / ((x - mean).square().mean(1, keepdim=True) + 1e-5).sqrt()
        h = (x - mean) * rstd
        real = c(out["q"]) * c(out["step"])[:, None]
        assert ((real - (h * c(before["weight"]) + c(before["bias"]))).abs() <= 0.5001 * c(out["step"])[:, None]).all()  # half a code
        a, b, scale = c(copies["a"]), c(copies["b"]), c(self.scale)
        y, dy = real @ w.t(), c(out["dy"])
        dreal = dy @ w
        da, db = torch.zeros_like(a), torch.zeros_like(b)
        for l in range(ADAPTERS):
            at = (self.index == l).cpu()
            y[at] += scale[l] * real[at] @ a[l].t() @ b[l]
            g = scale[l] * dy[at] @ b[l].t()
            dreal[at] += g @ a[l]
            da[l] = g.t() @ real[at]
            db[l] = scale[l] * (real[at] @ a[l].t()).t() @ dy[at]
        g = dreal * c(before["weight"])
        dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        # dx of the layer is rounded to bf16 (2^-8) after dy * w_scale was (2^-8); float32 sums of under 256 terms are far below
        rows = 2.0 ** -7
        norm = lambda t: float(t.norm())  # noqa: E731
        assert norm(c(out["y"]) - y) <= 2.0 ** -8 * norm(y)
        assert norm(c(self.grads["a"]) - da) <= 2.0 ** -16 * norm(da) and norm(c(self.grads["b"]) - db) <= 2.0 ** -16 * norm(db)
        assert norm(c(self.grads["bias"]) - dreal.sum(0)) <= rows * norm(dreal.abs().sum(0))
        assert norm(c(self.grads["weight"]) - (dreal * h).sum(0)) <= rows * norm((dreal * h).abs().sum(0))
        assert norm(c(out["dx"]) - dx) <= 2 * rows * norm(dx)


@pytest.mark.parametrize("bits", [8, 32])
def test_steps_against_64_bits(P, bits):
    m = Model(P, bits)
    for t in range(3):
        before, copies = {k: v.clone() for k, v in m.params.items()}, {k: v.clone() for k, v in m.copies.items()}
        m.check(before, copies, m.step())
        for k in "ab":
            assert m.torch.equal(m.copies[k], m.params[k].bfloat16())
        for k in m.params:
            assert m.params[k].isfinite().all() and not m.torch.equal(m.params[k], before[k])


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_steps_are_the_eager_ones(P, bits):
    """One captured step replayed, beside the same model stepped eagerly: every parameter and moment equal after each."""
    one, two = Model(P, bits), Model(P, bits)
    torch = one.torch
    one.step()
    two.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.step()
    for _ in range(4):
        graph.replay()
        two.step()
        torch.cuda.synchronize()
        for k in one.params:
            assert torch.equal(one.params[k], two.params[k]), k
            for u, v in zip(one.state[k], two.state[k]):
                assert u is None or torch.equal(u, v), k


def test_two_calls_at_once_on_two_streams(P):
    """Two models stepped on streams of their own, interleaved: the results of one after the other."""
    ref = [Model(P, 32), Model(P, 8)]
    for m in ref:
        for _ in range(3):
            m.step()
    got = [Model(P, 32), Model(P, 8)]
    torch = got[0].torch
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for m, s in zip(got, streams):
            with torch.cuda.stream(s):
                m.step()
    torch.cuda.synchronize()
    for m, r in zip(got, ref):
        for k in m.params:
            assert torch.equal(m.params[k], r.params[k]), k


def test_a_stream_given_to_the_calls(P):
    """stream=: work enqueued behind it on the current stream does not get the call's workspace while it runs."""
    m = Model(P, 32)
    torch = m.torch
    q, step, mean, rstd = P.prom_layernorm_quant(m.x, m.params["weight"], m.params["bias"])
    lora = P.Lora(m.copies["a"], m.copies["b"], m.scale, m.index)
    x4 = q.view(ROWS, 1, 1, CIN)
    y, hid = P.prom_pw_conv_lora(x4, m.packed, COUT, step, m.w_scale, None, lora, want_hid=True)
    dy = m.target.view(ROWS, 1, 1, COUT)
    want = P.prom_pw_conv_lora_backward(dy, x4, step, m.packed_t, m.w_scale, lora, hid)
    wn = P.prom_layernorm_backward(want[0].view(ROWS, CIN), m.x, m.params["weight"], mean, rstd)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(4):
        got = P.prom_pw_conv_lora_backward(dy, x4, step, m.packed_t, m.w_scale, lora, hid, stream=side)
        gn = P.prom_layernorm_backward(got[0].view(ROWS, CIN), m.x, m.params["weight"], mean, rstd, stream=side)
        gy, gh = P.prom_pw_conv_lora(x4, m.packed, COUT, step, m.w_scale, None, lora, want_hid=True, stream=side)
        gq = P.prom_layernorm_quant(m.x, m.params["weight"], m.params["bias"], stream=side)
        for size in (1 << 14, 1 << 18, 1 << 20, 1 << 21):
            torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        for u, v in zip(got + gn + (gy, gh) + gq, want + wn + (y, hid) + (q, step, mean, rstd)):
            assert torch.equal(u, v)
