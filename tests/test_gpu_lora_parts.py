"""Parts of the gradient of the adapters' layer from tensors that start at any element."""
import numpy as np
import pytest

from gpu_util import torch_cuda
from test_gpu_lora import make, run_both, types

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2505_03254_amd as P
    P.load_library()
    return P


@pytest.mark.parametrize("ti", range(4))
@pytest.mark.parametrize("n", [20, 150])
def test_parts_of_unaligned_tensors(P, n, ti):
    torch = torch_cuda()
    t, o = types()[ti]
    s = make(n, n, 1, 1, 193, 111, 16, 3, t, dy_type=o)
    want = run_both(P, s)
    c = {k: v.cuda() if hasattr(v, "cuda") else v for k, v in s.items()}
    for k in ("dy", "x"):
        flat = torch.empty(c[k].numel() + 1, dtype=c[k].dtype, device="cuda")
        flat[1:] = c[k].reshape(-1)
        c[k] = flat[1:].view(c[k].shape)
    lora = P.Lora(c["a"], c["b"], c["scale"], c["index"])
    wtp = torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(s["wt"].numpy().T))).cuda()
    for k in range(1, 8):
        f = dict(want_dx=bool(k & 1), want_da=bool(k & 2), want_db=bool(k & 4))
        got = P.prom_pw_conv_lora_backward(c["dy"], c["x"], c["step"], wtp if k & 1 else None, c["ws"] if k & 1 else None, lora, want["hid"] if k & 4 else None, **f)
        for name, v in zip(("dx", "da", "db"), got):
            assert v is None if not f["want_" + name] else torch.equal(v, want[name]), (k, name)
