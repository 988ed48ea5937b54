"""The fine-tuning example of README.md, run as it stands there: the step has to move every parameter against its gradient."""
import os
import re

import numpy as np
import pytest

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def test_the_fine_tuning_example():
    torch = torch_cuda()
    import paper_2505_03254_amd as P
    P.load_library()
    block = next(b for b in re.findall(r"```python\n(.*?)```", open(README).read(), re.S) if "prom_pw_conv_lora_backward" in b)
    r = torch.Generator().manual_seed(1)
    randn = lambda *s: torch.randn(*s, generator=r).cuda()  # noqa: E731
    n, cin, cout, adapters, rank = 90, 96, 72, 3, 8
    codes = torch.randint(-1, 2, (cout, cin), generator=r, dtype=torch.int8).numpy()
    # the gradients' order in the example: a, b, norm weight, norm bias
    params = [randn(adapters, rank, cin) * 0.1, randn(adapters, rank, cout) * 0.1, 1 + 0.1 * randn(cin), 0.1 * randn(cin)]
    copies = [params[0].bfloat16(), params[1].bfloat16(), None, None]
    grads = [torch.zeros_like(p) for p in params]
    tensors = [P.AdamWTensor(p, g, torch.zeros_like(p), torch.zeros_like(p), copy=c) for p, g, c in zip(params, grads, copies)]
    before = [p.clone() for p in params]
    space = dict(P=P, torch=torch, n=n, cin=cin, cout=cout, x=randn(n, cin).bfloat16(), norm_w=params[2], norm_b=params[3], a=copies[0], b=copies[1],
                 scale=torch.ones(adapters, device="cuda"), index=torch.arange(n, dtype=torch.int32).cuda() % adapters, w_scale=torch.full((cout,), 0.1, device="cuda"),
                 wp=torch.from_numpy(P.prom_pack_ternary(codes)).cuda(), wtp=torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(codes.T))).cuda(),
                 dy=randn(n, 1, 1, cout).bfloat16(), params=params, grads=grads, opt=P.AdamWTensors(tensors), t=1)
    exec(block, space)
    torch.cuda.synchronize()
    assert space["y"].isfinite().all()
    # the first step from zero moments: p (1 - 1e-3 * 0.01) - 1e-3 sign(g), float32
    for p, old, g in zip(params, before, (space["da"], space["db"], space["dw"], space["dbias"])):
        moved = old.double() * (1 - 1e-5) - p.double()
        assert (g.abs() > 1e-4).float().mean() > 0.9
        at = g.abs() > 1e-4  # eps is 1e-8 beside it: 1e-4 of the step
        assert ((moved - 1e-3 * g.sign()).abs()[at] <= 1e-3 * 1e-3 + 2.0 ** -22 * old.abs().double()[at]).all()
