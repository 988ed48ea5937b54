"""Which alignment the gradients of the adapters' layer ask for, on the host: every call here ends at the workspace check, before any launch (the
addresses are never dereferenced)."""
import pytest

from test_operators_abi import S, W, X, Y, H, WS, backward, lib, lora  # noqa: F401

EWORKSPACE, EINVAL = -4, -1


@pytest.mark.parametrize("parts", [dict(dx=None), dict(dx=None, da=None), dict(dx=None, db=None), dict(da=None, db=None), dict()])
@pytest.mark.parametrize("t,step", [(1, 2), (2, 2), (0, 4)])
def test_tensors_start_at_any_element(lib, parts, t, step):  # noqa: F811
    lo = lora(type=t or 1)
    for k in range(4):
        assert backward(lib, lo, t=t, dy=Y + k * step, space=None, **parts) == EWORKSPACE, k


def test_packed_weights_are_words_where_they_are_looked_at(lib):  # noqa: F811
    for off in (1, 2, 3):
        assert backward(lib, wp=W + off, space=None) == EINVAL
        assert backward(lib, wp=W + off, dx=None, space=None) == EWORKSPACE
    assert backward(lib, wp=None, dx=None, space=None) == EWORKSPACE and backward(lib, wp=None, space=None) == EINVAL
