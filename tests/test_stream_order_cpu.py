"""Memory that a call takes is ordered on the stream that it launches on.

torch's allocator hands a block out again as soon as the stream that it was taken on
has the work queued that used it.  A result that is taken on the current stream and
written by another one can be overwritten by what the current stream still does with the
block, and a result that is given back can be overwritten while the other stream reads
it.  Shown with a torch of plain CPU tensors that say they are on a GPU, and a library
that launches nothing: no GPU is needed, and none could show it each time."""
import contextlib
import ctypes
import types

import pytest
import torch

import paper_2502_01637_amd as S

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="replaces torch's GPU functions: for a process without one")


class Stream:
    def __init__(self, handle, device=None):
        self.cuda_stream, self.waits = handle, []

    def wait_stream(self, other):
        self.waits.append(other.cuda_stream)

    def synchronize(self):
        pass


class Tensor(torch.Tensor):
    """A CPU tensor that says it is on cuda:0 and remembers the streams of its memory."""
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", 0))

    def get_device(self):
        return 0

    def record_stream(self, stream):
        self.also = stream.cuda_stream

    def item(self):
        Tensor.read_on.append(torch.cuda.current_stream().cuda_stream)
        return super().item()


@pytest.fixture
def gpu(monkeypatch):
    state = types.SimpleNamespace(current=Stream(5), taken=[], launched=[])
    Tensor.read_on = []

    def memory(make):
        def new(*size, dtype=None, device=None, **_):
            t = make(*size, dtype=dtype).as_subclass(Tensor)
            t.on, t.also = state.current.cuda_stream, None
            state.taken.append(t)
            return t
        return new

    @contextlib.contextmanager
    def switch(stream):
        old, state.current = state.current, stream
        yield
        state.current = old

    real = S.scone.lib()

    class Library:
        def __getattr__(self, name):
            f = getattr(real, name)
            if f.argtypes is None or f.restype is not ctypes.c_int or f.argtypes[-1] is not ctypes.c_void_p \
                    or name.endswith("layout"):
                return f

            def call(*args):
                assert len(args) == len(f.argtypes), name
                state.launched.append((name, args[-1]))
                return 0
            return call

    monkeypatch.setattr(S.scone, "_lib", Library())
    monkeypatch.setattr(S.scone, "_raw_stream", lambda index: state.current.cuda_stream)
    monkeypatch.setattr(S.scone, "_current_device", lambda: 0)
    for name, fake in [("Stream", Stream), ("ExternalStream", Stream), ("stream", switch),
                       ("current_stream", lambda device=None: state.current),
                       ("current_device", lambda: 0), ("synchronize", lambda *_: None)]:
        monkeypatch.setattr(torch.cuda, name, fake)
    state.tensor = lambda *size, dtype: torch.zeros(*size, dtype=dtype).as_subclass(Tensor)
    state.monkeypatch = monkeypatch
    monkeypatch.setattr(torch, "empty", memory(torch.empty))
    return state


def new_rows(gpu, n=6, cols=100):
    return S.Mx4Rows(gpu.tensor(n, S.mx4_row_bytes(cols), dtype=torch.uint8), cols)


def quantize(gpu, stream):
    return S.quantize_mx4(gpu.tensor(4, 100, dtype=torch.bfloat16), stream=stream).data


def gather(gpu, stream):
    return S.gather_mx4(gpu.tensor(3, dtype=torch.int32), new_rows(gpu), stream=stream)


def dequantize(gpu, stream):
    return S.dequantize_mx4(new_rows(gpu), stream=stream)


def linear(gpu, stream):
    return S.linear_mx4(gpu.tensor(100, 100, dtype=torch.bfloat16), new_rows(gpu), stream=stream)


CALLS = [quantize, gather, dequantize, linear]


def check(gpu, call, stream, handle):
    result = call(gpu, stream)
    assert [h for _, h in gpu.launched] == [handle]
    assert gpu.taken and all(t.on == handle for t in gpu.taken)
    # the program uses the result on its own stream: it is given back there too
    assert result.also == (None if handle == 5 else 5)


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__)
@pytest.mark.parametrize("kind", ["none", "current", "current handle", "other", "other handle"])
def test_results_are_taken_on_the_launch_stream(gpu, call, kind):
    stream, handle = {"none": (None, 5), "current": (gpu.current, 5), "current handle": (5, 5),
                      "other": (Stream(8), 8), "other handle": (8, 8)}[kind]
    check(gpu, call, stream, handle)


@pytest.mark.parametrize("stream", [Stream(8), 8], ids=["object", "handle"])
def test_4bit_model_waits_for_the_model_it_is_made_from(gpu, stream):
    """The parameters may still be on their way on the current stream."""
    made = [stream] if isinstance(stream, Stream) else []
    gpu.monkeypatch.setattr(torch.cuda, "ExternalStream",
                            lambda *a, **k: made.append(Stream(*a, **k)) or made[-1])
    model = types.SimpleNamespace(d=512, n_heads=8, d_ff=1024, n_layers=2, max_len=3,
                                  blob=gpu.tensor(100, dtype=torch.int16))
    four = S.FgramModelMx4(model, stream=stream)
    assert gpu.launched == [("scone_fgram_model_quantize", 8)]
    assert four.weights.on == 8 and four.weights.also == 5
    assert [h for s in made for h in s.waits] == [5]
    gpu.launched.clear()
    assert S.FgramModelMx4(model).weights.on == 5 and gpu.launched[0][1] == 5


# ------------------------------------------------------- rows of any bytes ----

def tokens(gpu):
    return gpu.tensor(3, 20, dtype=torch.int32)


TABLE = types.SimpleNamespace(handle=ctypes.c_void_p(64), device=torch.device("cuda", 0))


def lookup(gpu, stream):
    return S.lookup(TABLE, tokens(gpu), 3, want_len=True, stream=stream)


def tag(gpu, stream):
    return S.tag(TABLE, tokens(gpu), 3, stream=stream)[:1]


def discover(gpu, stream):
    gpu.monkeypatch.setattr(ctypes, "c_int64", lambda f=ctypes.c_int64: f(4))
    return S.discover_fgrams(tokens(gpu), 3, 4, stream=stream)


def gather_bytes(gpu, stream):
    return [S.gather(tokens(gpu), gpu.tensor(9, 16, dtype=torch.float32), stream=stream)]


def embed(gpu, stream):
    return [S.embed(TABLE, tokens(gpu), 3, gpu.tensor(9, 16, dtype=torch.float32), stream=stream)]


def embed_pipelined(gpu, stream):
    return [S.embed_pipelined(TABLE, None, 3, None, tokens(gpu),
                              gpu.tensor(9, 16, dtype=torch.float32), stream=stream)]


def gather_split(gpu, stream):
    far = S.HostRows.__new__(S.HostRows)
    far.device_ptr, far.n_rows, far.row_bytes, far.row_shape = 4096, 9, 64, (16,)
    far.dtype, far._closed = torch.float32, True
    return [S.gather_split(tokens(gpu), gpu.tensor(9, 16, dtype=torch.float32), far,
                           gpu.tensor(1 << 16, dtype=torch.uint8), stream=stream)]


@pytest.mark.parametrize("call", [lookup, tag, discover, gather_bytes, embed, embed_pipelined,
                                  gather_split], ids=lambda f: f.__name__)
@pytest.mark.parametrize("kind", ["none", "current", "current handle", "other", "other handle"])
def test_results_of_the_byte_calls(gpu, call, kind):
    stream, handle = {"none": (None, 5), "current": (gpu.current, 5), "current handle": (5, 5),
                      "other": (Stream(8), 8), "other handle": (8, 8)}[kind]
    results = call(gpu, stream)
    assert [h for _, h in gpu.launched] == [handle]
    assert gpu.taken and all(t.on == handle for t in gpu.taken)
    assert [t.also for t in gpu.taken] == [None if handle == 5 else 5] * len(gpu.taken)
    assert len(results) > 0


@pytest.mark.parametrize("kind", ["none", "other", "other handle"])
def test_count_is_cleared_and_read_on_the_launch_stream(gpu, kind):
    stream, handle = {"none": (None, 5), "other": (Stream(8), 8), "other handle": (8, 8)}[kind]
    cleared = []
    real = torch.zeros

    def zeros(*size, dtype=None, device=None):
        cleared.append(gpu.current.cuda_stream)
        return real(*size, dtype=dtype).as_subclass(Tensor)

    tok = tokens(gpu)
    gpu.monkeypatch.setattr(torch, "zeros", zeros)
    S.scone.lookup_counted(TABLE, tok, 3, stream=stream)
    assert [h for _, h in gpu.launched] == cleared == Tensor.read_on == [handle]
    assert all(t.on == handle for t in gpu.taken) and len(gpu.taken) == 2
