"""The gradients of the adapters over a million rows of one adapter."""
import pytest

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2505_03254_amd as P
    P.load_library()
    return P


@pytest.mark.parametrize("value", [1.3, 0.9])
def test_a_million_rows_of_one_adapter(P, value):
    """Equal terms, whose roundings all go the same way: a chunk's 128 rows are at most 3 * 128 + 16 float32 additions deep, and the chunks must
    add no more than another such sum does."""
    torch = torch_cuda()
    rows, c = 1 << 20, 16
    v = torch.tensor(value, device="cuda")
    x, dy = torch.ones(rows, 1, 1, c, dtype=torch.int8, device="cuda"), torch.ones(rows, 1, 1, c, dtype=torch.bfloat16, device="cuda")
    lora = P.Lora(torch.zeros(1, 1, c, dtype=torch.bfloat16, device="cuda"), torch.full((1, 1, c), 1 / c, dtype=torch.bfloat16, device="cuda"),
                  torch.ones(1, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"))
    _, da, db = P.prom_pw_conv_lora_backward(dy, x, v.expand(rows).contiguous(), None, None, lora, v.expand(rows, 1).contiguous(), want_dx=False)
    want = rows * float(v)
    for g in (da, db):
        assert float((g.double() / want - 1).abs().max()) <= 2 * (3 * 128 + 16) * 2.0 ** -24
