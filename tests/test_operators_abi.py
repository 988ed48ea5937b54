"""What the calls of the float side refuse, on the host and before any launch (the addresses are never dereferenced), and the tables they
write there."""
import ctypes

import numpy as np
import pytest

X, W, Y, A, B, S, I, H, WS = (0x100000000 * k for k in range(1, 10))


@pytest.fixture(scope="module")
def lib():
    import paper_2505_03254_amd as P
    return P.load_library()


def lora(**k):
    from paper_2505_03254_amd.binding import _LoraC
    v = dict(a=A, b=B, scale=S, index=I, adapters=3, rank=8, type=1)
    v.update(k)
    return _LoraC(**v)


def forward(lib, lo=None, **k):
    v = dict(x=X, n=100, h=1, w=1, cin=64, wp=W, cout=48, step=S + 4096, ws=S + 8192, bias=S + 12288, y=Y, yt=1, hid=H, space=WS, bytes=1 << 24)
    v.update(k)
    return lib.prom_pw_conv_lora(v["x"], v["n"], v["h"], v["w"], v["cin"], v["wp"], v["cout"], v["step"], v["ws"], v["bias"], lo if lo is not None else lora(),
                                 v["y"], v["yt"], v["hid"], v["space"], v["bytes"], None)


def backward(lib, lo=None, **k):
    v = dict(dy=Y, t=1, x=X, n=100, h=1, w=1, cin=64, wp=W, cout=48, step=S + 4096, ws=S + 8192, hid=H, dx=Y + (1 << 28), da=Y + (2 << 28), db=Y + (3 << 28),
             space=WS, bytes=1 << 24)
    v.update(k)
    return lib.prom_pw_conv_lora_backward(v["dy"], v["t"], v["x"], v["n"], v["h"], v["w"], v["cin"], v["wp"], v["cout"], v["step"], v["ws"],
                                          lo if lo is not None else lora(), v["hid"], v["dx"], v["da"], v["db"], v["space"], v["bytes"], None)


@pytest.mark.parametrize("k,code", [
    (dict(x=None), -1), (dict(wp=None), -1), (dict(step=None), -1), (dict(ws=None), -1), (dict(y=None), -1), (dict(n=0), -1), (dict(h=-1), -1),
    (dict(cin=0), -1), (dict(cout=-3), -1), (dict(yt=2), -1), (dict(yt=3), -1), (dict(wp=W + 2), -1), (dict(y=Y + 1), -1), (dict(yt=0, y=Y + 2), -1),
    (dict(hid=H + 2), -1), (dict(bias=S + 2), -1), (dict(cin=65537), -2), (dict(cout=65537), -2), (dict(n=1 << 30), -2), (dict(n=(1 << 26) + 1), -2), (dict(n=1 << 16, h=1 << 10, w=1 << 10), -2),
    (dict(space=None), -4), (dict(bytes=100), -4), (dict(space=WS + 8), -4), (dict(y=X + 10), -3), (dict(y=A + 2), -3), (dict(hid=Y + 64), -3), (dict(y=WS), -3),
    (dict(hid=I), -3), (dict(n=64, hid=None, space=None), -4)])
def test_forward_refuses(lib, k, code):
    assert forward(lib, **k) == code


@pytest.mark.parametrize("k,code", [
    (dict(dy=None), -1), (dict(step=None), -1), (dict(dx=None, da=None, db=None), -1), (dict(ws=None), -1), (dict(wp=None), -1), (dict(hid=None), -1),
    (dict(x=None), -1), (dict(t=2), -1), (dict(dy=Y + 1), -1), (dict(da=Y + 2), -1), (dict(n=-1), -1), (dict(cin=65537), -2), (dict(bytes=1000), -4),
    (dict(space=None), -4), (dict(dx=Y + 100), -3), (dict(da=H), -3), (dict(db=WS + 256), -3), (dict(da=B), -3), (dict(dx=Y + (2 << 28)), -3), (dict(da=S), -3)])
def test_backward_refuses(lib, k, code):
    assert backward(lib, **k) == code


@pytest.mark.parametrize("k,code", [
    (dict(a=None), -1), (dict(b=None), -1), (dict(scale=None), -1), (dict(index=None), -1), (dict(adapters=0), -1), (dict(rank=0), -1), (dict(type=0), -1),
    (dict(type=7), -1), (dict(a=A + 1), -1), (dict(index=I + 2), -1), (dict(rank=129), -2), (dict(adapters=65536), -2)])
def test_adapters_refused(lib, k, code):
    assert forward(lib, lora(**k)) == code
    assert backward(lib, lora(**k)) == code
    assert lib.prom_pw_conv_lora(X, 1, 1, 1, 64, W, 48, S, S, None, None, Y, 1, None, WS, 1 << 24, None) == -1


def test_workspace_sizes(lib):
    f, b = lib.prom_pw_conv_lora_workspace_size, lib.prom_pw_conv_lora_backward_workspace_size
    assert f(64, 1, 1, 64, 48, 3, 8, 1) == 0 and f(64, 1, 1, 64, 48, 3, 8, 0) >= 64 * 8 * 4 and f(65, 1, 1, 64, 48, 3, 8, 1) > 0
    for bad in ((0, 1, 1, 64, 48, 3, 8), (4, 1, 1, 65537, 48, 3, 8), (4, 1, 1, 64, 48, 3, 129), (4, 1, 1, 64, 48, 65536, 8), (1 << 16, 1 << 10, 1 << 10, 8, 8, 1, 1)):
        assert f(*bad, 0) == 0 and b(*bad, 1) == 0
    assert b(4, 1, 1, 64, 48, 3, 8, 3) == 0
    assert b(1000, 1, 1, 64, 48, 3, 8, 0) > b(1000, 1, 1, 64, 48, 3, 8, 2) > b(1000, 1, 1, 64, 48, 3, 8, 1) > 0


def norm(lib, **k):
    v = dict(x=X, t=1, rows=10, cols=100, w=W, b=W + 4096, eps=1e-5, y=Y, mean=S, rstd=S + 4096)
    v.update(k)
    return lib.prom_layernorm(v["x"], v["t"], v["rows"], v["cols"], v["w"], v["b"], v["eps"], v["y"], v["mean"], v["rstd"], None)


@pytest.mark.parametrize("k,code", [
    (dict(x=None), -1), (dict(y=None), -1), (dict(t=3), -1), (dict(t=-1), -1), (dict(rows=0), -1), (dict(cols=0), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
    (dict(x=X + 1), -1), (dict(t=0, y=Y + 2), -1), (dict(w=W + 1), -1), (dict(mean=S + 2), -1), (dict(cols=32769), -2), (dict(rows=1 << 31), -2),
    (dict(y=X + 20), -3), (dict(y=X), -3), (dict(mean=X), -3), (dict(rstd=S + 4), -3), (dict(y=W), -3)])
def test_norm_refuses(lib, k, code):
    assert norm(lib, **k) == code


def test_norm_quant_refuses(lib):
    def go(q=Y, step=S, eps=1e-5, qe=1e-5, mean=S + 4096, cols=100):
        return lib.prom_layernorm_quant(X, 1, 10, cols, W, None, eps, qe, q, step, mean, None, None)
    assert go(q=None) == -1 and go(step=None) == -1 and go(qe=0.0) == -1 and go(qe=float("nan")) == -1 and go(eps=-1.0) == -1 and go(step=S + 1) == -1
    assert go(q=X + 1999) == -3 and go(step=Y + 996) == -3 and go(mean=S + 36) == -3 and go(cols=40000) == -2


def test_norm_backward_refuses(lib):
    need = lib.prom_layernorm_backward_workspace_size(1, 10, 100)
    assert need >= 800 and lib.prom_layernorm_backward_workspace_size(3, 10, 100) == 0 and lib.prom_layernorm_backward_workspace_size(1, 10, 32769) == 0

    def go(dy=X, x=X + 8192, dx=Y, dw=Y + 8192, db=Y + 16384, mean=S, rstd=S + 64, ws=WS, nb=need, t=1):
        return lib.prom_layernorm_backward(dy, x, t, 10, 100, W, mean, rstd, dx, dw, db, ws, nb, None)
    assert go(dy=None) == -1 and go(mean=None) == -1 and go(rstd=None) == -1 and go(dx=None, dw=None, db=None) == -1 and go(t=9) == -1 and go(dw=Y + 8193) == -1
    assert go(ws=None) == -4 and go(nb=need - 1) == -4 and go(ws=WS + 16) == -4
    assert go(dx=X) == -3 and go(dw=Y + 1000) == -3 and go(db=WS) == -3 and go(dw=S) == -3


def tensor(**k):
    from paper_2505_03254_amd.binding import _AdamWTensorC
    v = dict(param=X, grad=W, exp_avg=Y, exp_avg_sq=A, avg_scale=S, sq_scale=S + 4096, copy=None, n=1000, param_type=0, grad_type=1, copy_type=0, state_bits=8)
    v.update(k)
    return _AdamWTensorC(**v)


@pytest.mark.parametrize("k,code", [
    (dict(param=None), -1), (dict(grad=None), -1), (dict(exp_avg=None), -1), (dict(exp_avg_sq=None), -1), (dict(avg_scale=None), -1), (dict(sq_scale=None), -1),
    (dict(n=0), -1), (dict(param_type=3), -1), (dict(grad_type=-1), -1), (dict(state_bits=16), -1), (dict(copy=B, copy_type=5), -1), (dict(param=X + 2), -1),
    (dict(state_bits=32, exp_avg=Y + 2), -1), (dict(avg_scale=S + 2), -1), (dict(n=(1 << 42) + 1), -2), (dict(param=W), -3), (dict(exp_avg_sq=Y + 999), -3),
    (dict(copy=X + 4, copy_type=0), -3), (dict(sq_scale=S + 12), -3)])
def test_adamw_table_refuses(lib, k, code):
    from paper_2505_03254_amd.binding import _AdamWPlanC, _AdamWTensorC
    arr = (_AdamWTensorC * 2)(tensor(), tensor(**k))
    plan, bad, host = _AdamWPlanC(), ctypes.c_int(-7), np.zeros(4096, dtype=np.uint8)
    assert lib.prom_adamw_table(arr, 2, host.ctypes.data, host.size, plan, bad) == code and bad.value == 1
    assert lib.prom_adamw_table_size(arr, 2) == 0 and not host.any()


def test_adamw_table(lib):
    """One entry per tensor, then the tensor of every workgroup of 4096 elements."""
    from paper_2505_03254_amd.binding import _AdamWPlanC, _AdamWTensorC
    sizes = (1, 4096, 4097, 20000)
    arr = (_AdamWTensorC * 4)(*[tensor(n=n, state_bits=32, param=X + (k << 20), grad=W + (k << 20), exp_avg=Y + (k << 20), exp_avg_sq=A + (k << 20)) for k, n in enumerate(sizes)])
    size = lib.prom_adamw_table_size(arr, 4)
    host = np.zeros(size + 4, dtype=np.uint8)
    plan, bad = _AdamWPlanC(), ctypes.c_int(-7)
    assert lib.prom_adamw_table(arr, 4, host.ctypes.data, size - 1, plan, bad) == -4
    assert lib.prom_adamw_table(arr, 4, host.ctypes.data, size, plan, bad) == 0 and bad.value == -1
    assert (plan.tensors, plan.workgroups) == (4, 9) and size == 4 * 72 + 9 * 4
    assert host[4 * 72:size].view(np.int32).tolist() == [0, 1, 2, 2, 3, 3, 3, 3, 3] and not host[size:].any()
    assert lib.prom_adamw_table(arr, 0, host.ctypes.data, size, plan, None) == -1 and lib.prom_adamw_table(None, 4, host.ctypes.data, size, plan, None) == -1
    assert lib.prom_adamw_table(arr, 4, None, size, plan, None) == -1


def test_adamw_step_refuses(lib):
    from paper_2505_03254_amd.binding import _AdamWHyperC, _AdamWPlanC

    def go(table=X, plan=None, **k):
        v = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, step_dev=None, lr_dev=None, grad_scale=None)
        v.update(k)
        return lib.prom_adamw_step(table, plan if plan is not None else _AdamWPlanC(4, 9), _AdamWHyperC(**v), None)
    nan = float("nan")
    for k in (dict(step=0), dict(step=-5), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.5), dict(beta2=nan), dict(eps=-1.0), dict(eps=nan), dict(weight_decay=-1.0), dict(lr=-1.0),
              dict(lr=nan), dict(step_dev=X + 2), dict(lr_dev=X + 1), dict(grad_scale=X + 2), dict(table=None), dict(table=X + 4), dict(plan=_AdamWPlanC(0, 9)), dict(plan=_AdamWPlanC(4, 0))):
        assert go(**k) == -1, k
    assert lib.prom_adamw_step(X, None, None, None) == -1
    assert lib.prom_adamw_moments(None, _AdamWPlanC(4, 9), X, X, None) == -1 and lib.prom_adamw_moments(X, _AdamWPlanC(4, 9), None, X, None) == -1
    assert lib.prom_adamw_moments(X, _AdamWPlanC(4, 9), X + 4, X, None) == -1


def test_binding_refuses_tensors_off_the_gpu():
    torch = pytest.importorskip("torch")
    import paper_2505_03254_amd as P
    x = torch.zeros(2, 8)
    with pytest.raises(TypeError):
        P.prom_layernorm(x)
    with pytest.raises(TypeError):
        P.prom_layernorm_quant(x)
    with pytest.raises(TypeError):
        P.prom_pw_conv_lora(torch.zeros(2, 1, 1, 8, dtype=torch.int8), x, 4, x, x, None, P.Lora(x, x, x, x))
    with pytest.raises(TypeError):
        P.AdamWTensors([P.AdamWTensor(x, x, x, x)])
    with pytest.raises(ValueError):
        P.AdamWTensors([])
