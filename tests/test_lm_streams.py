"""The package's calls on a stream that is not torch's current one, on the CPU: stand-ins for torch's streams, tensors
and the library's launches record which memory is taken, marked and used where."""
import pytest

import paper_1901_02244_amd as cb

torch = pytest.importorskip("torch")

K, N, D, V, OUT = 2, 6, 64, 40, 24


class Stream:
    def __init__(self, handle, device_index=0):
        self.cuda_stream, self.device_index = handle, device_index
        self.device = torch.device("cuda", device_index)

    def __eq__(self, other):
        return self.cuda_stream == other.cuda_stream

    __hash__ = None


class Cuda:
    """torch.cuda of two devices."""

    def __init__(self):
        self.device, self.streams, self.blocks = 0, [Stream(0, 0), Stream(0, 1)], []

    def current_device(self):
        return self.device

    def set_device(self, index):
        self.device = index

    def current_stream(self, index=None):
        return self.streams[self.device if index is None else index]

    def set_stream(self, stream):
        self.device = stream.device_index
        self.streams[stream.device_index] = stream

    def tensor(self, shape, dtype=torch.float32, index=0):
        return Tensor(self, shape, dtype, index)


class Tensor:
    """A contiguous tensor: the stream whose memory it took, and those it was marked for."""

    def __init__(self, cuda, shape, dtype, index):
        self.cuda, self.shape, self.dtype, self.index = cuda, torch.Size(shape), dtype, index
        self.device, self.is_cuda = torch.device("cuda", index), True
        self.home, self.marked = cuda.streams[index].cuda_stream, []
        cuda.blocks.append(self)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def stride(self, i):
        return self.shape[i + 1:].numel()

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 1 << 40

    def new_empty(self, shape, dtype):
        return Tensor(self.cuda, shape, dtype, self.index)

    def record_stream(self, stream):
        if not self.is_cuda:
            raise NotImplementedError
        self.marked.append(stream.cuda_stream)


class Torch:
    uint8, int32, float32 = torch.uint8, torch.int32, torch.float32

    def __init__(self):
        self.cuda, self._C = Cuda(), object()

    def empty_like(self, t):
        return t.new_empty(t.shape, t.dtype)


class Library:
    """The library's sizes; its launches succeed (or fail with `rc`) and note their stream."""

    def __init__(self, cuda):
        self.cuda, self.launches, self.rc = cuda, [], 0
        self.sizes = cb.lib()

    def __getattr__(self, name):
        if name.endswith("_bytes") or name == "cb_last_error":
            return getattr(self.sizes, name)

        def launch(*args):
            self.launches.append((name, args[-1], self.cuda.device))
            return self.rc

        return launch


@pytest.fixture
def fake(monkeypatch):
    cb._type_code("test", torch.float32)  # the package has seen torch
    t = Torch()
    library = Library(t.cuda)
    monkeypatch.setattr(cb, "_torch", t)
    monkeypatch.setattr(cb, "lib", lambda: library)
    return t.cuda, library


def calls(cuda):
    """{name: (call of a stream, its input tensors)} of every operator."""
    new = cuda.tensor
    h, w, y = new((K, N, D)), new((K, V, D)), new((K, N), torch.int32)
    lse, ws = new((K, N)), new((1 << 28,), torch.uint8)
    x, o, gate, dy, dres = new((K, N, D)), new((K, N, D)), new((K, N, D)), new((K, N, D)), new((K, N, D))
    post, pre, dpost, dpre = (new((K, D)) for _ in range(4))
    dw, dy2, dw2 = new((K, V, D)), new((K, N, OUT)), new((K, OUT, D))
    kept = cb.Kept(new((cb.lib().cb_ckpt_bytes(K * N, D),), torch.uint8), (K, N, D), torch.float32)
    how = dict(block=o, gate=gate, post=post, pre=pre)
    return {
        "xent_fwd": (lambda s: cb.cb_vocab_xent_fwd(h, w, y, stream=s), [h, w, y]),
        "xent_fwd, workspace": (lambda s: cb.cb_vocab_xent_fwd(h, w, y, workspace=ws, stream=s), [h, w, y, ws]),
        "xent_bwd": (lambda s: cb.cb_vocab_xent_bwd(h, w, y, lse, stream=s), [h, w, y, lse]),
        "xent_bwd, dw": (lambda s: cb.cb_vocab_xent_bwd(h, w, y, lse, dw=dw, stream=s), [h, w, y, lse, dw]),
        "norm_fwd": (lambda s: cb.cb_gated_norm_fwd(x, **how, keep=True, stream=s), [x, o, gate, post, pre]),
        "norm_fwd, no block": (lambda s: cb.cb_gated_norm_fwd(x, pre=pre, stream=s), [x, pre]),
        "norm_bwd": (lambda s: cb.cb_gated_norm_bwd(x, dy, dres=dres, **how, stream=s),
                     [x, dy, dres, o, gate, post, pre]),
        "norm_bwd, gammas": (lambda s: cb.cb_gated_norm_bwd(x, dy, **how, dpost=dpost, dpre=dpre, stream=s),
                             [x, dy, o, gate, post, pre, dpost, dpre]),
        "pack": (lambda s: cb.cb_ckpt_pack(x, stream=s), [x]),
        "unpack": (lambda s: cb.cb_ckpt_unpack(kept, stream=s), [kept.data]),
        "wgrad": (lambda s: cb.cb_ckpt_wgrad(kept, dy2, stream=s), [kept.data, dy2]),
        "wgrad, dw": (lambda s: cb.cb_ckpt_wgrad(kept, dy2, dw=dw2, workspace=ws, stream=s),
                      [kept.data, dy2, dw2, ws]),
    }


NAMES = ["xent_fwd", "xent_fwd, workspace", "xent_bwd", "xent_bwd, dw", "norm_fwd", "norm_fwd, no block", "norm_bwd",
         "norm_bwd, gammas", "pack", "unpack", "wgrad", "wgrad, dw"]


def test_every_operator_is_here(fake):
    assert list(calls(fake[0])) == NAMES


def tensors(result):
    if isinstance(result, (tuple, list)):
        return [t for r in result for t in tensors(r)]
    if isinstance(result, dict):
        return tensors(list(result.values()))
    if isinstance(result, cb.Kept):
        return [result.data]
    return [result] if isinstance(result, Tensor) else []


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_a_given_stream(name, fake):
    """What a call on another stream takes is that stream's memory: a block of torch's current stream that was just
    freed may still be read by work queued there, and the other stream does not wait for it.  Results are marked
    for the current stream, where the caller goes on with them."""
    cuda, library = fake
    f, inputs = calls(cuda)[name]
    before = len(cuda.blocks)
    result = f(Stream(77))
    new = cuda.blocks[before:]
    assert [handle for _, handle, _ in library.launches] == [77]
    assert all(t.home == 77 for t in new)
    results = [t for t in tensors(result) if not any(t is i for i in inputs)]
    assert all(t.marked == [0] for t in results)
    assert all(not t.marked for t in new if not any(t is r for r in results))  # workspaces
    assert cuda.current_stream().cuda_stream == 0 and cuda.device == 0  # and the caller's stream is back


@pytest.mark.parametrize("name", NAMES)
def test_a_failed_call_leaves_the_streams_as_they_were(name, fake):
    cuda, library = fake
    f, _ = calls(cuda)[name]
    library.rc = cb.CB_EDEVICE
    with pytest.raises(cb.CBError):
        f(Stream(77))
    assert cuda.current_stream().cuda_stream == 0 and cuda.device == 0


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_the_current_stream(name, fake):
    """Without a stream, or with the current one, nothing changes hands."""
    cuda, library = fake
    for s in (None, Stream(0)):
        f, inputs = calls(cuda)[name]
        before = len(cuda.blocks)
        f(s)
        assert all(t.home == 0 and not t.marked for t in cuda.blocks[before:] + inputs)
    assert [handle for _, handle, _ in library.launches] == [0, 0]


@pytest.mark.parametrize("name", NAMES)
def test_device_of_the_inputs(name, fake):
    """Inputs of a device that is not the current one: the call runs there and comes back."""
    cuda, library = fake
    cuda.device = 1
    f, _ = calls(cuda)[name]
    f(Stream(77, 0))
    f(None)
    assert [(handle, device) for _, handle, device in library.launches] == [(77, 0), (0, 0)]
    assert cuda.device == 1 and cuda.streams[1].cuda_stream == 0 and cuda.streams[0].cuda_stream == 0


@pytest.mark.parametrize("name", NAMES)
def test_inputs_of_a_given_stream(name, fake):
    """Inputs, given outputs and a given workspace are marked for the other stream: a caller who drops one after the
    call does not have its memory taken while the work there still uses it."""
    cuda, _ = fake
    f, inputs = calls(cuda)[name]
    f(Stream(77))
    assert all(77 in t.marked for t in inputs)


@pytest.mark.parametrize("what", ["type", "device", "host"])
def test_a_refused_workspace_leaves_the_streams_as_they_were(what, fake):
    cuda, library = fake
    h, w, y = cuda.tensor((K, N, D)), cuda.tensor((K, V, D)), cuda.tensor((K, N), torch.int32)
    ws = cuda.tensor((1 << 28,), torch.float32 if what == "type" else torch.uint8, 1 if what == "device" else 0)
    if what == "host":
        ws.is_cuda, ws.device = False, torch.device("cpu")
    with pytest.raises(cb.CBError) as e:
        cb.cb_vocab_xent_fwd(h, w, y, workspace=ws, stream=Stream(77))
    assert e.value.code == cb.CB_EINVAL
    assert cuda.current_stream().cuda_stream == 0 and cuda.device == 0 and not library.launches


@pytest.mark.parametrize("handle", [0, 77])
@pytest.mark.parametrize("name", NAMES)
def test_a_stream_of_another_device_is_refused(name, handle, fake):
    """The default streams of all devices have the handle 0: the device tells them apart."""
    cuda, library = fake
    f, inputs = calls(cuda)[name]
    with pytest.raises(cb.CBError) as e:
        f(Stream(handle, 1))
    assert e.value.code == cb.CB_EINVAL and "stream" in str(e.value)
    assert not library.launches and not any(t.marked for t in inputs)
    assert cuda.device == 0 and [s.cuda_stream for s in cuda.streams] == [0, 0]
