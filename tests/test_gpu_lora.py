"""The ternary pointwise layer with adapters, forward and backward, against its definition in 64 bits.

Tolerances, relative to what a result is made of (the same sums with every term's magnitude, `size` below): a rounding is off by half a step,
eps / 2 of the value (bf16 2^-8, f16 2^-11) and never less than half of the type's smallest step (2^-25 in f16).  A number in p bf16 planes is off by
(2^-8)^p, since each plane rounds what the ones before it left: dx carries dy * w_scale in 1, 2 or 3 planes (bf16, f16, float32), and hid and g enter
with 2 (16-bit results) or 3.  float32 sums of K terms are off by at most K * 2^-24 of `size`."""
import numpy as np
import pytest

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2505_03254_amd as P
    P.load_library()
    return P


def make(seed, n, h, w, cin, cout, rank, adapters, type, index=None, dy_type=None):
    torch = torch_cuda()
    r = torch.Generator().manual_seed(seed)
    s = dict(n=n, h=h, w=w, cin=cin, cout=cout, rank=rank, adapters=adapters)
    s["x"] = torch.randint(-128, 128, (n, h, w, cin), generator=r, dtype=torch.int8)
    s["wt"] = torch.randint(-1, 2, (cout, cin), generator=r, dtype=torch.int8)
    s["step"] = 0.01 + 0.05 * torch.rand(n, generator=r)
    s["ws"] = (0.2 + torch.rand(cout, generator=r)) / cin ** 0.5
    s["bias"] = torch.randn(cout, generator=r)
    s["a"] = (torch.randn(adapters, rank, cin, generator=r) / cin ** 0.5).to(type)
    s["b"] = torch.randn(adapters, rank, cout, generator=r).to(type)
    s["scale"] = 0.25 + torch.rand(adapters, generator=r)
    s["index"] = torch.randint(-1, adapters, (n,), generator=r, dtype=torch.int32) if index is None else torch.tensor(index, dtype=torch.int32)
    s["dy"] = torch.randn(n, h, w, cout, generator=r).to(dy_type or type)
    return s


def definition(s):
    """Everything in 64 bits, row by adapter; the same with magnitudes."""
    import torch
    D = torch.float64
    m, hw = s["n"] * s["h"] * s["w"], s["h"] * s["w"]
    x = s["x"].to(D).view(m, -1)
    step = s["step"].to(D).repeat_interleave(hw)[:, None]
    which = s["index"].long().repeat_interleave(hw)
    dy = s["dy"].to(D).view(m, -1)

    def go(f):
        y = f(x) @ f(s["wt"].to(D)).t() * f(s["ws"].to(D)) * step + f(s["bias"].to(D))
        dx = f(dy) * f(s["ws"].to(D)) @ f(s["wt"].to(D))
        hid = torch.zeros(m, s["rank"], dtype=D)
        da, db = torch.zeros(s["a"].shape, dtype=D), torch.zeros(s["b"].shape, dtype=D)
        for l in range(s["adapters"]):
            at = which == l
            a, b, scale = f(s["a"][l].to(D)), f(s["b"][l].to(D)), float(s["scale"][l])
            hid[at] = f(x)[at] @ a.t() * step[at]
            y[at] += scale * hid[at] @ b
            g = scale * f(dy)[at] @ b.t()
            dx[at] += g @ a
            da[l] = (g * step[at]).t() @ f(x)[at]
            db[l] = scale * hid[at].t() @ f(dy)[at]
        return dict(y=y, hid=hid, dx=dx, da=da, db=db)

    return go(lambda t: t), go(lambda t: t.abs())


def near(got, want, size, rel, what):
    import torch
    off = (got.double().cpu().view(want.shape) - want).abs()
    least = torch.finfo(got.dtype).tiny * torch.finfo(got.dtype).eps / 2
    lim = rel * size + least + 1e-30
    bad = off > lim
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, the worst by {float((off / lim).max()):.2f} times the bound"


def rounding(t):
    torch = torch_cuda()
    return torch.finfo(t).eps / 2


def run_both(P, s, **more):
    torch = torch_cuda()
    c = {k: v.cuda() if hasattr(v, "cuda") else v for k, v in s.items()}
    lora = P.Lora(c["a"], c["b"], c["scale"], c["index"])
    wp = torch.from_numpy(P.prom_pack_ternary(s["wt"].numpy())).cuda()
    wtp = torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(s["wt"].numpy().T))).cuda()
    y, hid = P.prom_pw_conv_lora(c["x"], wp, s["cout"], c["step"], c["ws"], c["bias"], lora, dtype=s["dy"].dtype, want_hid=True)
    dx, da, db = P.prom_pw_conv_lora_backward(c["dy"], c["x"], c["step"], wtp, c["ws"], lora, hid)
    torch.cuda.synchronize()
    return dict(y=y, hid=hid, dx=dx, da=da, db=db)


def check(P, s, what=""):
    torch = torch_cuda()
    got = run_both(P, s)
    want, size = definition(s)
    t = s["dy"].dtype
    m = s["n"] * s["h"] * s["w"]
    sum_of = lambda k: (k + 8) * 2.0 ** -24  # noqa: E731
    hid_bits = 2.0 ** -16 if t != torch.float32 else 2.0 ** -24
    planes = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -16, torch.float32: 2.0 ** -24}[t]
    near(got["hid"], want["hid"], size["hid"], sum_of(s["cin"]), what + "hid")
    near(got["y"], want["y"], size["y"], rounding(t) + sum_of(s["cin"] + s["rank"]) + hid_bits, what + "y")
    near(got["dx"], want["dx"], size["dx"], rounding(t) + planes + sum_of(s["cout"] + s["rank"]) + hid_bits, what + "dx")
    # three planes hold 24 bits of a coefficient, and so do the products that are taken of them
    near(got["da"], want["da"], size["da"], sum_of(m + s["cout"]) + 2.0 ** -22, what + "da")
    near(got["db"], want["db"], size["db"], sum_of(m + s["cin"]) + 2.0 ** -22, what + "db")
    none = ((s["index"] < 0) | (s["index"] >= s["adapters"])).repeat_interleave(s["h"] * s["w"])
    assert not got["hid"][none.cuda()].any()
    for l in range(s["adapters"]):
        if not (s["index"] == l).any():
            assert not got["da"][l].any() and not got["db"][l].any()
    return got


def types():
    import torch
    return [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float16, torch.float32)]


@pytest.mark.parametrize("ti", range(4))
@pytest.mark.parametrize("shape", [
    (1, 1, 1, 64, 64, 16, 1), (1, 1, 1, 1, 1, 1, 1), (3, 1, 1, 17, 5, 3, 2), (16, 1, 1, 256, 48, 8, 4), (17, 1, 1, 100, 130, 12, 3),
    (64, 1, 1, 300, 66, 16, 64), (65, 1, 1, 300, 66, 16, 64), (5, 7, 7, 96, 100, 4, 3), (2, 6, 5, 960, 160, 20, 2), (130, 1, 1, 33, 257, 33, 5),
    (9, 3, 11, 129, 65, 64, 4), (300, 1, 1, 1000, 70, 128, 7), (257, 1, 1, 2048, 384, 40, 2)])
def test_types_and_sizes(P, shape, ti):
    t, o = types()[ti]
    check(P, make(hash(shape) % 1000, *shape, t, dy_type=o), f"{shape} {t} {o} ")


@pytest.mark.parametrize("rows,rank", [(1, 32), (2, 16), (3, 10), (16, 2), (17, 1), (31, 1), (32, 1), (33, 1), (5, 7), (33, 20), (48, 128), (64, 5)])
@pytest.mark.parametrize("cin,cout", [(256, 40), (4640, 33), (70, 16)])
def test_few_rows(P, rows, rank, cin, cout):
    """On both sides of what a few rows' product does itself, and of its two shapes."""
    torch = torch_cuda()
    check(P, make(rows * rank, rows, 1, 1, cin, cout, rank, 3, torch.bfloat16, dy_type=torch.float32), f"{rows} {rank} ")


@pytest.mark.parametrize("rows", [40, 200, 1000])
@pytest.mark.parametrize("kind", ["none", "one", "last", "outside", "in turn", "runs"])
def test_who_takes_what(P, rows, kind):
    torch = torch_cuda()
    L = 6
    index = {"none": [-1] * rows, "one": [2] * rows, "last": [-1] * (rows - 1) + [L - 1], "outside": [[-5, L, 2 ** 31 - 1, -2 ** 31, 0][i % 5] for i in range(rows)],
             "in turn": [i % L for i in range(rows)], "runs": sorted([(i * i) % (L + 1) - 1 for i in range(rows)])}[kind]
    check(P, make(rows, rows, 1, 1, 160, 200, 16, L, torch.bfloat16, index), f"{kind} ")


@pytest.mark.parametrize("rows", [30, 300])
def test_what_an_adapter_holds_stays_with_its_rows(P, rows):
    """Infinities and NaN in one adapter reach the rows that take it and no others, bit for bit."""
    torch = torch_cuda()
    s = make(5, rows, 1, 1, 200, 144, 16, 4, torch.bfloat16)
    clean = run_both(P, s)
    bad = dict(s, a=s["a"].clone(), b=s["b"].clone())
    bad["a"][1] = float("nan")
    bad["b"][1] = float("inf")
    got = run_both(P, bad)
    others = (s["index"] != 1).cuda()
    for k in ("y", "dx"):
        assert torch.equal(got[k][others], clean[k][others]), k
        assert not torch.isfinite(got[k][~others].float()).any(), k
    assert torch.equal(got["hid"][others], clean["hid"][others])
    for l in (0, 2, 3):
        assert torch.equal(got["da"][l], clean["da"][l]) and torch.equal(got["db"][l], clean["db"][l])


def test_the_base_is_that_of_the_integer_kernel(P):
    """Without adapters y is (acc * w_scale) * x_step + bias, three float32 operations, acc from prom_pw_accum_i32."""
    torch = torch_cuda()
    for n, hw in ((3, 1), (20, 9)):
        s = make(n, n, hw, 1, 448, 96, 8, 2, torch.bfloat16, [-1] * n, dy_type=torch.float32)
        c = {k: v.cuda() if hasattr(v, "cuda") else v for k, v in s.items()}
        wp = torch.from_numpy(P.prom_pack_ternary(s["wt"].numpy())).cuda()
        y = P.prom_pw_conv_lora(c["x"], wp, 96, c["step"], c["ws"], c["bias"], P.Lora(c["a"], c["b"], c["scale"], c["index"]), dtype=torch.float32)
        acc = P.prom_pw_accum_i32(c["x"], wp, 96)
        want = acc.float() * c["ws"] * c["step"][:, None, None, None] + c["bias"]
        assert torch.equal(y, want)


def test_same_bits_every_time_and_outputs_given_by_the_caller(P):
    torch = torch_cuda()
    for n in (48, 700):
        s = make(n, n, 1, 1, 320, 272, 24, 5, torch.float16)
        one, two = run_both(P, s), run_both(P, s)
        for k in one:
            assert torch.equal(one[k], two[k]), k
        c = {k: v.cuda() if hasattr(v, "cuda") else v for k, v in s.items()}
        wp = torch.from_numpy(P.prom_pack_ternary(s["wt"].numpy())).cuda()
        big = torch.full((n + 2, 1, 1, 272), 7.0, dtype=torch.float16, device="cuda")
        hid = torch.empty(n, 24, device="cuda")
        y, h = P.prom_pw_conv_lora(c["x"], wp, 272, c["step"], c["ws"], c["bias"], P.Lora(c["a"], c["b"], c["scale"], c["index"]), y=big[1:n + 1], hid=hid)
        assert torch.equal(y, one["y"]) and torch.equal(h, one["hid"])
        assert (big[0] == 7).all() and (big[n + 1] == 7).all()


def test_unaligned_tensors(P):
    """Tensors that start at any element: x one byte, adapters, y and dy one element into their memory."""
    torch = torch_cuda()

    def shifted(t):
        t = t.cuda()
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        flat[1:] = t.reshape(-1)
        return flat[1:].view(t.shape)

    for n in (20, 150):
        s = make(n, n, 1, 1, 192, 112, 16, 3, torch.bfloat16)
        want = run_both(P, s)
        c = {k: shifted(v) if hasattr(v, "cuda") else v for k, v in s.items()}
        lora = P.Lora(c["a"], c["b"], c["scale"], c["index"])
        wp = torch.from_numpy(P.prom_pack_ternary(s["wt"].numpy())).cuda()
        wtp = torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(s["wt"].numpy().T))).cuda()
        flat = torch.empty(n * 112 + 1, dtype=torch.bfloat16, device="cuda")
        y, hid = P.prom_pw_conv_lora(c["x"], wp, 112, c["step"], c["ws"], c["bias"], lora, y=flat[1:].view(n, 1, 1, 112), want_hid=True)
        dx, da, db = P.prom_pw_conv_lora_backward(c["dy"], c["x"], c["step"], wtp, c["ws"], lora, hid)
        for k, v in dict(y=y, hid=hid, dx=dx, da=da, db=db).items():
            assert torch.equal(v, want[k]), k


def test_parts_of_the_gradient(P):
    torch = torch_cuda()
    s = make(3, 90, 1, 1, 128, 96, 8, 3, torch.bfloat16)
    want = run_both(P, s)
    c = {k: v.cuda() if hasattr(v, "cuda") else v for k, v in s.items()}
    lora = P.Lora(c["a"], c["b"], c["scale"], c["index"])
    wtp = torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(s["wt"].numpy().T))).cuda()
    for k in range(1, 8):
        f = dict(want_dx=bool(k & 1), want_da=bool(k & 2), want_db=bool(k & 4))
        got = P.prom_pw_conv_lora_backward(c["dy"], c["x"], c["step"], wtp if k & 1 else None, c["ws"] if k & 1 else None, lora, want["hid"] if k & 4 else None, **f)
        for name, v in zip(("dx", "da", "db"), got):
            assert (v is None) == (not f["want_" + name])
            assert v is None or torch.equal(v, want[name]), name


def test_gradient_against_differences(P):
    """sum(dy * y) moved along random directions of a and b, by central differences of the float32 forward pass: along a line y is a
    polynomial of degree 1 in a and in b, so that the difference is exact up to the rounding of y (2^-23 of its parts, over 2 h)."""
    torch = torch_cuda()
    s = make(11, 96, 1, 1, 128, 80, 8, 3, torch.bfloat16, dy_type=torch.float32)
    got = run_both(P, s)
    dy = s["dy"].double().view(96, -1)
    r = torch.Generator().manual_seed(1)
    for name, grad in (("a", got["da"]), ("b", got["db"])):
        # a direction that keeps both ends exact in bf16: a power of two at some places
        d = (torch.randint(0, 50, s[name].shape, generator=r) == 0).double() * 0.0
        for _ in range(40):
            i = tuple(int(torch.randint(0, k, (1,), generator=r)) for k in s[name].shape)
            d[i] = 1.0
        lo, hi = s[name].double() - d, s[name].double() + d
        lo, hi = lo.to(s[name].dtype), hi.to(s[name].dtype)
        y = [run_both(P, dict(s, **{name: v}))["y"].double().cpu().view(96, -1) for v in (lo, hi)]
        want = (dy * (y[1] - y[0])).sum()
        moved = hi.double() - lo.double()
        have = (grad.double().cpu() * moved).sum()
        size = (dy.abs() * (y[1].abs() + y[0].abs())).sum()
        assert abs(float(want - have)) <= 2.0 ** -20 * float(size)


def test_another_stream_and_a_captured_pass(P):
    torch = torch_cuda()
    for n in (32, 260):
        s = make(n, n, 1, 1, 256, 192, 16, 4, torch.bfloat16)
        want = run_both(P, s)
        c = {k: v.cuda() if hasattr(v, "cuda") else v for k, v in s.items()}
        lora = P.Lora(c["a"], c["b"], c["scale"], c["index"])
        wp = torch.from_numpy(P.prom_pack_ternary(s["wt"].numpy())).cuda()
        wtp = torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(s["wt"].numpy().T))).cuda()

        def both(stream=None):
            y, hid = P.prom_pw_conv_lora(c["x"], wp, 192, c["step"], c["ws"], c["bias"], lora, want_hid=True, stream=stream)
            return (y, hid) + P.prom_pw_conv_lora_backward(c["dy"], c["x"], c["step"], wtp, c["ws"], lora, hid, stream=stream)

        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            got = both()
        side.synchronize()
        for k, v in zip(("y", "hid", "dx", "da", "db"), got):
            assert torch.equal(v, want[k]), k
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = both()
        x0, i0 = c["x"].clone(), c["index"].clone()
        for turn in range(3):
            c["x"].copy_(x0.roll(turn, 0))
            c["index"].copy_(i0.roll(turn, 0))
            graph.replay()
            torch.cuda.synchronize()
            eager = both()
            torch.cuda.synchronize()
            for k, u, v in zip(("y", "hid", "dx", "da", "db"), got, eager):
                assert torch.equal(u, v), (turn, k)
