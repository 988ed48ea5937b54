"""Calls that are given a stream, beside work of the current stream's that is still under way on the memory which the allocator would hand out next."""
import numpy as np
import pytest

from gpu_util import torch_cuda
from test_gpu_lora import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2505_03254_amd as P
    P.load_library()
    return P


class Busy:
    """Some milliseconds of products on the current stream."""

    def __init__(self):
        torch = torch_cuda()
        self.a = torch.randn(4096, 4096, device="cuda")
        self.out = torch.empty_like(self.a)

    def enqueue(self):
        for _ in range(12):
            torch_cuda().matmul(self.a, self.a, out=self.out)


def freed_after(busy, tensors):
    """Blocks like these, overwritten on the current stream once the products are done, and given back to the allocator at once."""
    torch = torch_cuda()
    busy.enqueue()
    old = [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in tensors]
    for t in old:
        t.view(torch.uint8).fill_(0x7B)


@pytest.mark.parametrize("name", ["norm", "quant", "norm back", "lora", "lora back"])
def test_memory_that_the_current_stream_still_works_on(P, name):
    torch = torch_cuda()
    n, cin, cout = 150, 192, 112
    s = make(1, n, 1, 1, cin, cout, 16, 3, torch.bfloat16)
    c = {k: v.cuda() if hasattr(v, "cuda") else v for k, v in s.items()}
    lora = P.Lora(c["a"], c["b"], c["scale"], c["index"])
    wp = torch.from_numpy(P.prom_pack_ternary(s["wt"].numpy())).cuda()
    wtp = torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(s["wt"].numpy().T))).cuda()
    x = torch.randn(3000, 1030, device="cuda").bfloat16()
    weight = torch.rand(1030, device="cuda")
    dyn = torch.randn_like(x)
    _, mean, rstd = P.prom_layernorm(x, weight)
    hid = P.prom_pw_conv_lora(c["x"], wp, cout, c["step"], c["ws"], c["bias"], lora, want_hid=True)[1]
    call, space = {
        "norm": (lambda **k: P.prom_layernorm(x, weight, **k), 0),
        "quant": (lambda **k: P.prom_layernorm_quant(x, weight, **k), 0),
        "norm back": (lambda **k: P.prom_layernorm_backward(dyn, x, weight, mean, rstd, **k), P.prom_layernorm_backward_workspace_size(x.dtype, 3000, 1030)),
        "lora": (lambda **k: P.prom_pw_conv_lora(c["x"], wp, cout, c["step"], c["ws"], c["bias"], lora, want_hid=True, **k),
                 P.prom_pw_conv_lora_workspace_size(n, 1, 1, cin, cout, 3, 16, True)),
        "lora back": (lambda **k: P.prom_pw_conv_lora_backward(c["dy"], c["x"], c["step"], wtp, c["ws"], lora, hid, **k),
                      P.prom_pw_conv_lora_backward_workspace_size(n, 1, 1, cin, cout, 3, 16, torch.bfloat16)),
    }[name]
    want = call()
    like = list(want) + ([torch.empty(space, dtype=torch.uint8, device="cuda")] if space else [])
    busy, side = Busy(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        freed_after(busy, like)
        got = call(stream=side)
        torch.cuda.synchronize()
        for u, v in zip(got, want):
            assert torch.equal(u, v)
        # and the results' memory is not handed out while the current stream still reads them
        busy.enqueue()
        kept = [u.clone() for u in got]
        del got, u
        call(stream=side)
        torch.cuda.synchronize()
        for u, v in zip(kept, want):
            assert torch.equal(u, v)
        del kept, u


def test_a_captured_pass_with_a_side_stream(P):
    """A stream that joins the capture, and several replays of it."""
    torch = torch_cuda()
    x, w = torch.randn(300, 1000, device="cuda").bfloat16(), torch.rand(1000, device="cuda")
    side = torch.cuda.Stream()

    def run():
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        y, mean, rstd = P.prom_layernorm(x, w, stream=side)
        q = P.prom_layernorm_quant(x, w)
        here.wait_stream(side)
        return (y,) + q + P.prom_layernorm_backward(y, x, w, mean, rstd)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(4):
        x.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(got, run()):
            assert torch.equal(u, v)
        torch.cuda.synchronize()


@pytest.mark.parametrize("how", ["given", "current"])
def test_a_table_that_nobody_holds_any_more(P, how):
    """A step and the reading of its moments wait on a busy stream; table and targets' addresses are given back meanwhile."""
    torch = torch_cuda()
    sizes = (5000, 33, 257)

    def make():
        g = torch.Generator().manual_seed(4)
        return [P.AdamWTensor(torch.randn(n, generator=g).cuda(), torch.randn(n, generator=g).cuda(), torch.zeros(n, dtype=torch.int8, device="cuda"),
                              torch.zeros(n, dtype=torch.uint8, device="cuda"), *(torch.zeros((n + 255) // 256, device="cuda") for _ in range(2))) for n in sizes]

    def targets():
        return [(torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")) for n in sizes]

    ref, mref = make(), targets()
    opt = P.AdamWTensors(ref)
    opt.step(1)
    opt.moments(opt.moment_targets(mref))
    busy, side = Busy(), torch.cuda.Stream()
    for _ in range(3):
        got, mgot = make(), targets()
        opt = P.AdamWTensors(got)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            busy.enqueue()
        at = opt.moment_targets(mgot)
        if how == "given":
            opt.step(1, stream=side)
            opt.moments(at, stream=side)
        else:
            with torch.cuda.stream(side):
                opt.step(1)
                opt.moments(at)
        del opt, at
        others = [torch.full((k,), 0, dtype=torch.uint8, device="cuda") for k in (24, 48, 128, 256, 512, 1024, 4096) for _ in range(3)]
        torch.cuda.synchronize()
        del others
        for a, b in zip(got, ref):
            for k in ("param", "exp_avg", "exp_avg_sq", "avg_scale", "sq_scale"):
                assert torch.equal(getattr(a, k), getattr(b, k)), k
        for a, b in zip(mgot, mref):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
