"""How many bits the results of the adapters' layer keep, element by element and on average.

A 16-bit result is rounded once: half a step of the value itself, eps / 2 (bf16 2^-8, f16 2^-11).  What lies below that is relative to the
magnitudes of the sums (`size`): dy * w_scale goes into the product with half a step of 2^-11 (bf16), 2^-16 (f16) or 2^-24 (float32), hid and g with
2^-16 for 16-bit results, and a float32 sum of K terms is off by at most K * 2^-24."""
import numpy as np
import pytest

from gpu_util import torch_cuda
from test_gpu_lora import definition, make, run_both

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2505_03254_amd as P
    P.load_library()
    return P


def dx_alone(P, dy, codes, ws):
    """dx of rows without an adapter.  dy [rows, cout], codes [cout, cin] on the host."""
    torch = torch_cuda()
    rows, (cout, cin) = dy.shape[0], codes.shape
    lora = P.Lora(torch.zeros(1, 1, cin, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 1, cout, dtype=torch.bfloat16, device="cuda"),
                  torch.ones(1, device="cuda"), torch.full((rows,), -1, dtype=torch.int32, device="cuda"))
    wtp = torch.from_numpy(P.prom_pack_ternary(np.ascontiguousarray(codes.numpy().T))).cuda()
    dx, _, _ = P.prom_pw_conv_lora_backward(dy.cuda().view(rows, 1, 1, cout), torch.zeros(rows, 1, 1, cin, dtype=torch.int8, device="cuda"),
                                            torch.ones(rows, device="cuda"), wtp, ws.cuda(), lora, None, want_da=False, want_db=False)
    return dx.cpu().view(rows, cin)


def test_a_scale_between_two_bf16_values(P):
    """257 terms that would all lose nearly 2^-8 in the same direction if dy * w_scale were rounded to bf16: 256 instead of 258.  Rows of
    every magnitude beside each other."""
    torch = torch_cuda()
    e = torch.tensor([-126, -110, -60, -20, -3, 0, 1, 9, 40, 100, 118])
    scale = 1 + 2.0 ** -8 - 2.0 ** -16
    dy = torch.ldexp(torch.ones(len(e), 257), e[:, None]).bfloat16()
    codes = torch.ones(257, 20, dtype=torch.int8)
    dx = dx_alone(P, dy, codes, torch.full((257,), scale)).double()
    want = torch.ldexp(torch.full((len(e), 20), 257 * scale, dtype=torch.float64), e[:, None])
    off = ((dx - want).abs() / want).max(1).values
    assert (off <= 2.0 ** -8 + 2.0 ** -11 + 265 * 2.0 ** -24).all(), off.tolist()


def test_a_large_element_beside_small_ones(P):
    """Outputs that an element 2^20 times its neighbours does not reach keep their bits."""
    torch = torch_cuda()
    r = torch.Generator().manual_seed(1)
    dy = torch.randn(100, 300, generator=r).bfloat16()
    dy[:, 77] = 2.0 ** 20
    codes = torch.randint(-1, 2, (300, 64), generator=r, dtype=torch.int8)
    codes[77, :32] = 0
    ws = 0.5 + torch.rand(300, generator=r)
    dx = dx_alone(P, dy, codes, ws).double()
    D = torch.float64
    want = dy.to(D) * ws.to(D) @ codes.to(D)
    size = (dy.to(D) * ws.to(D)).abs() @ codes.to(D).abs()
    assert ((dx - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -11 + 308 * 2.0 ** -24) * size).all()


@pytest.mark.parametrize("e", [24, 28, 32, 36])
def test_elements_far_below_the_rows_largest(P, e):
    """2^-28 of the largest product and less is held in steps of 2^-38 of it, half of one off at most per term, and not as zero."""
    torch = torch_cuda()
    r = torch.Generator().manual_seed(e)
    dy = (1 + torch.rand(70, 200, generator=r)).bfloat16()
    dy[:, 3] = 2.0 ** e
    codes = torch.randint(0, 2, (200, 40), generator=r, dtype=torch.int8)
    codes[3] = 0
    codes[3, 20:] = 1
    dx = dx_alone(P, dy, codes, torch.ones(200)).double()
    want = dy.double() @ codes.double()
    terms = codes.double().sum(0)
    lost = 2.0 ** (e - 39) * terms if e >= 28 else 0.0 * terms
    assert ((dx - want).abs() <= (2.0 ** -8 + 208 * 2.0 ** -24) * want + 2.0 ** -11 * want + lost).all()
    assert (dx[:, :20] > 0.5 * want[:, :20]).all()


def test_rows_of_zeros_and_rows_that_are_not_finite(P):
    torch = torch_cuda()
    r = torch.Generator().manual_seed(2)
    dy = torch.randn(90, 130, generator=r).bfloat16()
    codes = torch.randint(-1, 2, (130, 70), generator=r, dtype=torch.int8)
    codes[5] = 1
    ws = 0.5 + torch.rand(130, generator=r)
    clean = dx_alone(P, dy, codes, ws)
    bad = dy.clone()
    bad[7], bad[20, 5], bad[33, 5], bad[34, 5] = 0, float("nan"), float("inf"), -float("inf")
    dx = dx_alone(P, bad, codes, ws)
    rest = torch.ones(90, dtype=torch.bool)
    rest[[7, 20, 33, 34]] = False
    assert torch.equal(dx[rest], clean[rest]) and not dx[7].any()
    assert dx[20].isnan().all() and (dx[33] == float("inf")).all() and (dx[34] == -float("inf")).all()


@pytest.mark.parametrize("index", [-1, 0])
@pytest.mark.parametrize("rows,cin,cout", [(300, 72, 1030), (2100, 1030, 72), (500, 512, 4096)])
def test_the_average_error_is_that_of_one_rounding(P, rows, cin, cout, index):
    """The result's own rounding r has the norm that bf16(want) - want has.  dy * w_scale adds at most 2^-11 / sqrt(3) = 0.00028 of the norm of
    want (independent errors of random signs), against r's 0.0016: sqrt(1 + 0.031) = 1.015 of r, and 1.5 % for the sample."""
    torch = torch_cuda()
    s = make(rows, rows, 1, 1, cin, cout, 8, 1, torch.bfloat16, [index] * rows)
    want = definition(s)[0]["dx"]
    got = run_both(P, s)["dx"].cpu().double().view(want.shape)
    once = (want.float().bfloat16().double() - want).norm()
    assert float((got - want).norm()) <= 1.03 * float(once), float((got - want).norm() / once)


@pytest.mark.parametrize("ti", range(4))
@pytest.mark.parametrize("rows,cin,cout,rank", [
    (1, 64, 64, 16), (20, 300, 66, 5), (65, 1030, 72, 8), (300, 129, 1031, 33), (16400, 1030, 72, 20), (4100, 1030, 200, 20), (2100, 1030, 72, 12),
    (4100, 200, 1030, 20), (900, 1030, 1200, 40)])
def test_every_element(P, rows, cin, cout, rank, ti):
    torch = torch_cuda()
    t, o = [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float16, torch.float32)][ti]
    s = make(rows + cin, rows, 1, 1, cin, cout, rank, 5, t, dy_type=o)
    got = run_both(P, s)
    want, size = definition(s)
    half = torch.finfo(o).eps / 2
    low = 2.0 ** -16 if o != torch.float32 else 2.0 ** -24
    planes = {torch.bfloat16: 2.0 ** -11, torch.float16: 2.0 ** -16, torch.float32: 2.0 ** -24}[o]
    least = torch.finfo(o).tiny * torch.finfo(o).eps / 2
    for name, below in (("y", low + (cin + rank + 8) * 2.0 ** -24), ("dx", planes + low + (cout + rank + 8) * 2.0 ** -24)):
        off = (got[name].double().cpu().view(want[name].shape) - want[name]).abs()
        limit = half * want[name].abs() + below * size[name] + least
        assert (off <= limit).all(), (name, float((off / limit).max()))
