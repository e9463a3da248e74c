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


class Library:
    """Notes the calls that launch; the others go to the real one."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name in ("aspis_grad_norm", "aspis_clip_grads", "aspis_adamw"):
            def call(*args):
                self.calls.append(name)
                return ap.OK
            return call
        return getattr(self.real, name)


@pytest.fixture
def library(monkeypatch):
    lib = Library(ap.lib)
    monkeypatch.setattr(ap, "lib", lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
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
    assert library.calls == ["aspis_grad_norm", "aspis_clip_grads", "aspis_adamw"]
    for wrong in (params, [], None):
        with pytest.raises(ValueError):
            ap.aspis_grad_norm(wrong, norm, work, stream=0)
        with pytest.raises(ValueError):
            ap.aspis_clip_grads(wrong, 1.0, norm, work, stream=0)
    for wrong in (grads, [], None):
        with pytest.raises(ValueError):
            ap.aspis_adamw(wrong, 1, 1e-3, stream=0)
    assert len(library.calls) == 3
