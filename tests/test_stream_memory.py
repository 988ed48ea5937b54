"""What a call does with device memory when it is given a stream, shown on the host: tensors and streams that only note what is done with them.

A kernel on another stream than the current one must not get memory of the current stream's (its last user there may still be at work on it),
and memory that it uses must not be handed out again before it is done."""
import contextlib
import types

import pytest

torch = pytest.importorskip("torch")


class Stream:
    def __init__(self, handle):
        self.cuda_stream, self.device = handle, torch.device("cuda", 0)
        self.device_index = 0


class Mem:
    """A device tensor: which stream's memory it is, and which streams it was recorded on."""

    def __init__(self, world, shape, dtype, brought=False):
        self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, torch.device("cuda", 0), True
        self.of, self.recorded, self.brought = world.now[-1], [], brought
        world.made.append(self)
        self.ptr = 0x10000000 * len(world.made)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.ptr

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def dim(self):
        return len(self.shape)

    def record_stream(self, s):
        self.recorded.append(s)

    def to(self, _):
        return self


@pytest.fixture()
def world(monkeypatch):
    from paper_2505_03254_amd import binding as B
    w = types.SimpleNamespace(now=[Stream(0x11)], made=[], launched=[], side=Stream(0x22), B=B)

    @contextlib.contextmanager
    def stream(s):
        w.now.append(s)
        yield
        w.now.pop()

    shape = lambda a: (a,) if isinstance(a, int) else tuple(a)  # noqa: E731
    fake = types.SimpleNamespace(
        float32=torch.float32, bfloat16=torch.bfloat16, float16=torch.float16, int8=torch.int8, uint8=torch.uint8, int32=torch.int32, int64=torch.int64, Tensor=Mem,
        empty=lambda s, dtype=None, device=None: Mem(w, shape(s), dtype), empty_like=lambda t: Mem(w, t.shape, t.dtype),
        tensor=lambda v, dtype=None, device=None: Mem(w, (len(v), len(v[0])), dtype), from_numpy=lambda a: Mem(w, a.shape, torch.uint8),
        cuda=types.SimpleNamespace(stream=stream, current_stream=lambda device=None: w.now[-1], set_device=lambda d: None))

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_size"):
                return lambda *a: 4096

            def call(*a):
                w.launched.append((name, a[-1]))
                return 0
            return call

    monkeypatch.setattr(B, "_torch", fake)
    monkeypatch.setattr(B, "_lib", Lib())
    monkeypatch.setattr(B, "load_library", lambda: B._lib)
    monkeypatch.setattr(B, "_raw_stream", lambda d: w.now[-1].cuda_stream)
    monkeypatch.setattr(B, "_get_device", lambda: 0)
    for f in ("_norm_workspace", "prom_pw_conv_lora_workspace_size", "prom_pw_conv_lora_backward_workspace_size"):
        getattr(B, f).cache_clear()
    yield w
    for f in ("_norm_workspace", "prom_pw_conv_lora_workspace_size", "prom_pw_conv_lora_backward_workspace_size"):
        getattr(B, f).cache_clear()


def calls(w):
    """name -> (what it is called with, the places of outputs and workspaces that the caller may bring)"""
    B, f32 = w.B, torch.float32
    have = lambda *s, dtype=f32: Mem(w, s, dtype, brought=True)  # noqa: E731
    rows, cols, cin, cout, rank = 10, 64, 64, 48, 8
    x, i8 = have(rows, cols, dtype=torch.bfloat16), have(rows, 1, 1, cin, dtype=torch.int8)
    lora = B.Lora(have(2, rank, cin, dtype=torch.bfloat16), have(2, rank, cout, dtype=torch.bfloat16), have(2), have(rows, dtype=torch.int32))
    wp = have(4096, dtype=torch.uint8)
    dy = have(rows, 1, 1, cout, dtype=torch.bfloat16)
    return {
        "norm": (lambda **k: B.prom_layernorm(x, have(cols), None, **k), dict(y=have(rows, cols, dtype=torch.bfloat16), mean=have(rows))),
        "quant": (lambda **k: B.prom_layernorm_quant(x, have(cols), None, **k), dict(q=have(rows, cols, dtype=torch.int8), step=have(rows))),
        "norm back": (lambda **k: B.prom_layernorm_backward(x, have(rows, cols, dtype=torch.bfloat16), None, have(rows), have(rows), **k), dict(workspace=have(4096, dtype=torch.uint8))),
        "lora": (lambda **k: B.prom_pw_conv_lora(i8, wp, cout, have(rows), have(cout), None, lora, want_hid=True, **k),
                 dict(y=have(rows, 1, 1, cout, dtype=torch.bfloat16), workspace=have(4096, dtype=torch.uint8))),
        "lora without hid": (lambda **k: B.prom_pw_conv_lora(i8, wp, cout, have(rows), have(cout), None, lora, **k), dict(workspace=have(4096, dtype=torch.uint8))),
        "lora back": (lambda **k: B.prom_pw_conv_lora_backward(dy, i8, have(rows), wp, have(cout), lora, have(rows, rank), **k), dict(workspace=have(4096, dtype=torch.uint8))),
    }


@pytest.mark.parametrize("name", ["norm", "quant", "norm back", "lora", "lora without hid", "lora back"])
@pytest.mark.parametrize("bring", [False, True])
def test_a_call_on_a_given_stream_allocates_there(world, name, bring):
    go, theirs = calls(world)[name]
    home, side = world.now[-1], world.side
    out = go(stream=side, **(theirs if bring else {}))
    assert [s for _, s in world.launched] == [side.cuda_stream] and world.now == [home]
    new = [t for t in world.made if not t.brought]
    assert new and all(t.of is side for t in new)                          # memory of the stream that works on it
    for t in out if isinstance(out, tuple) else (out,):
        assert home in t.recorded                                          # which the caller goes on to use on its own
    for t in theirs.values() if bring else ():
        assert t.of is home and side in t.recorded


@pytest.mark.parametrize("name", ["norm", "quant", "norm back", "lora", "lora without hid", "lora back"])
def test_a_call_on_the_current_stream_records_nothing(world, name):
    go, _ = calls(world)[name]
    go()
    assert [s for _, s in world.launched] == [world.now[-1].cuda_stream] and not any(t.recorded for t in world.made)
    go(stream=world.now[-1])
    assert not any(t.recorded for t in world.made)


def test_a_stream_of_another_device_is_refused(world):
    world.side.device, world.side.device_index = torch.device("cuda", 1), 1
    for name, (go, _) in calls(world).items():
        with pytest.raises(ValueError):
            go(stream=world.side)
    assert not world.launched


def tensors(w, n=1000, bits=8):
    have = lambda k, dtype: Mem(w, (k,), dtype, brought=True)  # noqa: E731
    m = (torch.int8, torch.uint8) if bits == 8 else (torch.float32, torch.float32)
    scales = [have((n + 255) // 256, torch.float32) for _ in range(2)] if bits == 8 else []
    return w.B.AdamWTensor(have(n, torch.float32), have(n, torch.bfloat16), have(n, m[0]), have(n, m[1]), *scales, copy=have(n, torch.bfloat16))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("how", ["given", "current"])
def test_the_table_of_a_step_on_another_stream(world, how, bits):
    """The table, which the kernel takes its addresses from, and the tensors that it points at, once for each stream that a step runs on."""
    w = world
    home, side, third = w.now[-1], w.side, Stream(0x33)
    brought = tensors(w, bits=bits)
    opt = w.B.AdamWTensors([brought])
    table = next(t for t in w.made if not t.brought)

    def step(s, t):
        if how == "given":
            opt.step(t, stream=s)
        else:
            w.now.append(s)
            opt.step(t)
            w.now.pop()

    opt.step(1)
    assert not any(t.recorded for t in w.made)
    step(side, 2)
    step(side, 3)
    step(third, 4)
    opt.step(5)
    pointed = [t for t in vars(brought).values() if t is not None]
    for t in [table] + pointed:
        assert t.recorded == [side, third]
    assert [h for name, h in w.launched if name == "prom_adamw_step"] == [home.cuda_stream, side.cuda_stream, side.cuda_stream, third.cuda_stream, home.cuda_stream]


@pytest.mark.parametrize("how", ["given", "current"])
def test_the_targets_of_moments_on_another_stream(world, how):
    w = world
    home, side = w.now[-1], w.side
    opt = w.B.AdamWTensors([tensors(w), tensors(w)])
    pairs = [tuple(Mem(w, (1000,), torch.float32, brought=True) for _ in range(2)) for _ in range(2)]
    before = len(w.made)
    targets = opt.moment_targets(pairs)
    addresses = w.made[before]
    opt.moments(targets)
    assert not any(t.recorded for t in w.made)
    if how == "given":
        opt.moments(targets, stream=side)
    else:
        w.now.append(side)
        opt.moments(targets)
        w.now.pop()
    table = next(t for t in w.made if not t.brought)
    for t in [table, addresses] + [t for pair in pairs for t in pair]:
        assert side in t.recorded
    assert [h for name, h in w.launched if name == "prom_adamw_moments"] == [home.cuda_stream, side.cuda_stream]


def test_a_step_on_a_stream_of_another_device_is_refused(world):
    w = world
    opt = w.B.AdamWTensors([tensors(w)])
    targets = opt.moment_targets([tuple(Mem(w, (1000,), torch.float32, brought=True) for _ in range(2))])
    w.side.device = torch.device("cuda", 1)
    w.launched.clear()
    for go in (lambda: opt.step(1, stream=w.side), lambda: opt.moments(targets, stream=w.side)):
        with pytest.raises(ValueError):
            go()
    assert not w.launched


@pytest.mark.parametrize("name,dtype", [("step", torch.int32), ("lr", torch.float32), ("grad_scale", torch.float32)])
@pytest.mark.parametrize("shape", [(0,), (3, 0)])
def test_a_hyperparameter_on_the_device_holds_a_number(world, name, dtype, shape):
    """An empty tensor has no address: as lr it would stand for a rate of 0, as grad_scale for none."""
    w = world
    opt = w.B.AdamWTensors([tensors(w)])
    w.launched.clear()
    bad = Mem(w, shape, dtype, brought=True)
    with pytest.raises(ValueError):
        opt.step(**dict(dict(step=1), **{name: bad}))
    assert not w.launched
    for one in ((), (1,), (4,)):
        opt.step(**dict(dict(step=1), **{name: Mem(w, one, dtype, brought=True)}))
    assert len(w.launched) == 3
