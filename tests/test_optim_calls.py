"""What the Python calls over many tensors refuse before the library sees it, without a GPU: buffers are
stand-ins, and the library notes its calls instead of making them."""
import pytest

ap = pytest.importorskip("paper_2108_02416_gb300")
torch = pytest.importorskip("torch")


class Buffer:
    """A device tensor as far as the calls look at it."""
    is_cuda = True

    def __init__(self, n=1, dtype=torch.float32, device=0):
        self.n, self.dtype, self.index, self.device = n, dtype, device, torch.device("cuda", device)

    def numel(self):
        return self.n

    def data_ptr(self):
        return 1 << 30

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.index


LAUNCHES = ("aspis_grad_norm", "aspis_clip_grads", "aspis_adamw")


class Library:
    """Notes the calls that launch; the others go to the real one."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name in LAUNCHES:
            def call(*args):
                self.calls.append(name)
                return ap.OK
            return call
        return getattr(self.real, name)


def current(monkeypatch, device):
    monkeypatch.setattr(torch.cuda, "current_device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", device, raising=False)


@pytest.fixture
def library(monkeypatch):
    lib = Library(ap.lib)
    monkeypatch.setattr(ap, "lib", lib)
    current(monkeypatch, lambda: 0)
    return lib


def buffers(device=0):
    return Buffer(device=device), Buffer(ap.NORM_WORKSPACE_BYTES, torch.uint8, device)


def test_lists_of_the_other_kind(library):
    """the library would read one kind's memory as the other's"""
    grads, params = ap.TensorList([]), ap.ParamList([], [], [], [])
    norm, work = buffers()
    ap.aspis_grad_norm(grads, norm, work, stream=0)
    ap.aspis_clip_grads(grads, 1.0, norm, work, stream=0)
    ap.aspis_adamw(params, 1, 1e-3, max_norm=1.0, norm=norm, work=work, stream=0)
    assert library.calls == list(LAUNCHES)
    for wrong in (params, [], None):
        with pytest.raises(ValueError):
            ap.aspis_grad_norm(wrong, norm, work, stream=0)
        with pytest.raises(ValueError):
            ap.aspis_clip_grads(wrong, 1.0, norm, work, stream=0)
    for wrong in (grads, [], None):
        with pytest.raises(ValueError):
            ap.aspis_adamw(wrong, 1, 1e-3, stream=0)
    assert len(library.calls) == 3


class Devices:
    """Two devices: which one is current, and which was at each call of the library."""

    def __init__(self, monkeypatch, library):
        self.current, self.at, self.streams = 0, [], []
        devices = self

        class Guard:
            def __init__(self, index):
                self.index = index

            def __enter__(self):
                self.before, devices.current = devices.current, self.index

            def __exit__(self, *_):
                devices.current = self.before

        class Noting:
            def __getattr__(self, name):
                call = getattr(library, name)
                if name not in LAUNCHES:
                    return call

                def noted(*args):
                    devices.at.append(devices.current)
                    devices.streams.append(getattr(args[-1], "value", args[-1]) or 0)
                    return call(*args)
                return noted

        monkeypatch.setattr(ap, "lib", Noting())
        monkeypatch.setattr(torch.cuda, "device", Guard)
        current(monkeypatch, lambda: self.current)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)


class Stream:
    def __init__(self, index):
        self.cuda_stream, self.device = 200 + index, torch.device("cuda", index)


@pytest.fixture
def devices(monkeypatch, library):
    return Devices(monkeypatch, library)


def lists(index):
    """lists whose tensors lie on a device (empty ones: nothing would be launched on any address)"""
    out = ap.TensorList([]), ap.ParamList([], [], [], [])
    for x in out:
        x._index, x.device = index, torch.device("cuda", index)
    return out


def every_call(grads, params, norm, work, each=None, stream=None):
    return [lambda: ap.aspis_grad_norm(grads, norm, work, tensor_norms=each, stream=stream),
            lambda: ap.aspis_clip_grads(grads, 1.0, norm, work, stream=stream),
            lambda: ap.aspis_adamw(params, 1, 1e-3, max_norm=1.0, norm=norm, work=work, stream=stream)]


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("own", [0, 1])
def test_calls_run_on_the_lists_device(devices, own, current):
    devices.current = current
    for call in every_call(*lists(own), *buffers(own)):
        call()
    for call in every_call(*lists(own), *buffers(own), stream=Stream(own)):
        call()
    ap.aspis_adamw(lists(own)[1], 1, 1e-3)                   # no buffers
    assert devices.at == [own] * 7 and devices.current == current
    assert devices.streams == [100 + own] * 3 + [200 + own] * 3 + [100 + own]


def test_an_empty_list_runs_where_its_buffers_are(devices):
    for call in every_call(ap.TensorList([]), ap.ParamList([], [], [], []), *buffers(1)):
        call()
    assert devices.at == [1] * 3 and devices.streams == [101] * 3


def test_buffers_and_streams_of_another_device(devices):
    (norm0, work0), (norm1, work1) = buffers(0), buffers(1)
    for norm, work in ((norm0, work1), (norm1, work0), (norm0, work0)):
        for call in every_call(*lists(1), norm, work):
            with pytest.raises(ValueError):
                call()
    for call in every_call(*lists(1), norm1, work1, stream=Stream(0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        ap.aspis_grad_norm(lists(1)[0], norm1, work1, tensor_norms=Buffer(device=0))
    assert devices.at == []


@pytest.mark.parametrize("eps,code", [(3.4e38, "OK"), (3.5e38, "E_INVAL"), (1e300, "E_INVAL"), (0.0, "OK")])
def test_eps_ends_where_fp32_does(eps, code):
    """it is used in fp32, where these would be infinite and stop every parameter (an empty list: nothing is launched)"""
    params, args = ap.ParamList([], [], [], []), ap._AdamwArgs(1e-3, 0.9, 0.999, eps, 1, -1.0, 1.0, 0, 0)
    assert ap.lib.aspis_adamw(params._h, ap.ctypes.byref(args), None, None, None) == getattr(ap, code)


class OnDevice:
    """A host tensor that says it lies on a device: lists look at tensors and read none."""

    def __init__(self, t):
        self.t, self.device = t, torch.device("cuda", 0)

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


def strided(shape, strides):
    return OnDevice(torch.zeros(4096).as_strided(shape, strides))


@pytest.mark.parametrize("shape,one,other,same", [
    ((1, 5, 4, 3), (60, 1, 15, 5), (7, 1, 15, 5), True),         # channels last; a dimension of one has any stride
    ((4, 1, 3), (1, 12, 4), (1, 1, 4), True),
    ((4, 1, 3, 1), (1, 99, 4, 5), (1, 4, 4, 12), True),
    ((4, 5, 3), (1, 12, 4), (1, 12, 4), True),
    ((4, 5, 3), (1, 12, 4), (5, 1, 20), False),
    ((4, 1, 3), (1, 12, 4), (3, 3, 1), False),                   # one in the other order
    ((4, 1, 3), (3, 3, 1), (1, 12, 4), False),
    ((2, 2), (1, 2), (2, 1), False),
    ((1, 1), (9, 7), (1, 1), True),
])
def test_orders_in_memory(shape, one, other, same):
    """element i of one tensor goes with element i of the other, wherever a dimension of length one claims to step to"""
    def make():
        a, b = strided(shape, one), strided(shape, other)
        ap.TensorList([a], [b])
        ap.ParamList([a], [b], [strided(shape, other)], [strided(shape, one)])
    if same:
        make()
    else:
        with pytest.raises(ValueError):
            make()
