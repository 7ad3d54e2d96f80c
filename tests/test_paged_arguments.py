"""What the Python calls of the paged cache do with their arguments before anything is launched: host tensors
that say they are on a GPU, and a stand-in for the library."""
import types

import pytest

import paper_2311_08252_b200 as rest

torch = pytest.importorskip("torch")
OK = 0


class OnGpu(torch.Tensor):
    """A host tensor that says that it is on GPU 1."""

    def get_device(self):
        return 1


def gpu(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


class Library:
    """Notes every call with the device that was current."""

    def __init__(self, devices):
        self.calls, self.devices = [], devices

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.devices[-1], args))
            return 64 if name.endswith("_bytes") else OK
        return call


@pytest.fixture
def library(monkeypatch):
    """GPU 0 is current."""
    devices = [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            devices.append(self.index)

        def __exit__(self, *_):
            devices.pop()

    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(OnGpu))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: devices[-1])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index, raising=False)
    lib = Library(devices)
    monkeypatch.setattr(rest, "_lib", lib)
    return lib


def attend(mask=None, **kw):
    q, pages = gpu(2, 3, 4, 64, dtype=torch.bfloat16), gpu(5, 2, 16, 64, dtype=torch.bfloat16)
    return rest.rest_paged_attention(q, pages, pages, gpu(2, 4), gpu(2), mask, 0.125, **kw)


@pytest.mark.parametrize("dtype", [torch.int32, torch.uint32])
def test_masks_are_words(library, dtype):
    attend(gpu(2, 3, 1, dtype=dtype))
    name, device, args = library.calls[-1]
    assert name == "rest_paged_attention" and device == 1 and args[-1] == 1001


@pytest.mark.parametrize("dtype", [torch.float32, torch.bool, torch.int64, torch.int16])
def test_masks_of_other_types_are_refused(library, dtype):
    with pytest.raises(rest.RestError, match="mask"):
        attend(gpu(2, 3, 1, dtype=dtype))
    assert not library.calls


def accept(**kw):
    i, f = (lambda *s: gpu(*s)), (lambda *s: gpu(*s, dtype=torch.float32))
    return rest.rest_accept_sampled(f(2, 4, 9), i(2, 3), i(2, 3), i(2), f(2, 4), f(2), f(2), 2, **kw)


@pytest.mark.parametrize("call", [attend, accept])
def test_scratch_sizes_are_asked_for_on_the_tensors_device(library, call):
    """They go by the device's number of SMs; GPU 0 is current, the tensors are on GPU 1."""
    call()
    assert [(name.endswith("_bytes"), device) for name, device, _ in library.calls] == [(True, 1), (False, 1)]


def every_call():
    pages, rows, i = gpu(5, 2, 16, 64, dtype=torch.bfloat16), gpu(2, 3, 2, 64, dtype=torch.bfloat16), gpu(2)
    return {
        "attention": attend, "accept": accept,
        "write": lambda **kw: rest.rest_paged_kv_write(pages, pages, gpu(2, 4), i, rows, rows, **kw),
        "commit": lambda **kw: rest.rest_paged_kv_commit(pages, pages, gpu(2, 4), i, gpu(2, 3), i, 3, **kw),
        "fork": lambda **kw: rest.rest_pages_fork(gpu(5), gpu(2, 4), i, i, gpu(1), gpu(1), 16, **kw),
        "copy": lambda **kw: rest.rest_pages_copy(pages, pages, i, i, **kw),
        "reserve": lambda **kw: rest.rest_pages_reserve(gpu(5), gpu(2, 4), i, i, 16, **kw),
        "release": lambda **kw: rest.rest_pages_release(gpu(5), gpu(2, 4), i, i, 16, **kw),
    }


@pytest.mark.parametrize("name", ["attention", "accept", "write", "commit", "fork", "copy", "reserve", "release"])
def test_streams_of_another_device_are_refused(library, name):
    """Tensors on GPU 1, a stream of GPU 0: the launch would go to GPU 1's own current stream, or fail."""
    call = every_call()[name]
    call()
    n = len(library.calls)
    with pytest.raises(rest.RestError, match="stream"):
        call(stream=types.SimpleNamespace(cuda_stream=64, device_index=0))
    assert len(library.calls) == n


@pytest.mark.parametrize("name", ["attention", "release"])
def test_windows_beyond_32_bits_are_refused(library, name):
    """2^32 + 5 would otherwise become a window of 5."""
    call = every_call()[name]
    call(window=(1 << 31) - 1, sinks=(1 << 31) - 1)
    n = len(library.calls)
    for kw in (dict(window=(1 << 32) + 5), dict(window=1 << 31), dict(window=7, sinks=1 << 32), dict(window=-1)):
        with pytest.raises(rest.RestError, match="window"):
            call(**kw)
    assert len(library.calls) == n
