"""Workspaces that the binding allocates belong to the stream that works on them.

torch's allocator hands a freed block to the next tensor of the stream it was allocated on, without a
wait. Here torch and the library are stand-ins: what is checked is on which stream the block was taken."""
import contextlib
import types

import pytest

import paper_2608_02560_gb300 as pg


class Tensor:
    is_cuda = True
    device = "cuda:0"

    def __init__(self, shape, dtype, stream=None):
        self.shape, self.dtype, self.stream = tuple(shape), dtype, stream

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    element_size = staticmethod(lambda: 1)
    is_contiguous = staticmethod(lambda: True)
    data_ptr = staticmethod(lambda: 0x10000)

    def dim(self):
        return len(self.shape)

    def stride(self):
        out, n = [], 1
        for s in reversed(self.shape):
            out.insert(0, n)
            n *= s
        return tuple(out)


class Stream:
    def __init__(self, number):
        self.cuda_stream = number


class Lib:
    """The stream argument of each call, and a workspace size for each size call."""

    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        if name.endswith("_size"):
            return lambda *a: 4096
        return lambda *a: self.streams.append(a[-1]) or 0


@pytest.fixture
def world(monkeypatch):
    now, made = [1], []          # the current stream, and the blocks that were taken

    @contextlib.contextmanager
    def on(stream):
        before, now[0] = now[0], stream.cuda_stream
        yield
        now[0] = before

    def empty(n, dtype=None, device=None):
        made.append(Tensor((n,), dtype, now[0]))
        return made[-1]

    class External(Stream):
        def __init__(self, number, device=None):
            Stream.__init__(self, number)

    dtypes = {n: n for n in ("float32", "bfloat16", "float16", "complex64", "int64", "uint8")}
    cuda = types.SimpleNamespace(stream=on, Stream=Stream, ExternalStream=External, is_initialized=lambda: True,
                                 current_stream=lambda: Stream(now[0]), current_device=lambda: 0)
    torch = types.SimpleNamespace(empty=empty, cuda=cuda, _C=types.SimpleNamespace(), **dtypes)
    lib = Lib()
    for name, value in (("_torch_module", torch), ("_dtype_codes", None), ("_raw_stream", None), ("_lib", lib)):
        monkeypatch.setattr(pg, name, value)
    return made, lib


def _calls(stream):
    t = Tensor
    index, queries = t((500, 64), "float16"), t((3, 64), "float16")
    rows, best = t((3,), "int64"), t((3, 2), "int64")
    T = 5000
    inputs = pg.delta_inputs(None, t((T, 1, 64), "bfloat16"), t((T, 1, 64), "bfloat16"), t((T, 1), "float32"),
                             t((T, 1), "float32"))
    states = t((1, 1, 1, 64, 64), "float32")
    return {"retrieve": lambda: pg.precog_retrieve(index, queries, rows, stream=stream),
            "retrieve_keys": lambda: pg.precog_retrieve_keys(index, queries, 0, rows, stream=stream),
            "retrieve_topk": lambda: pg.precog_retrieve_topk(index, queries, 2, best, stream=stream),
            "delta_scan": lambda: pg.precog_delta_scan(inputs, t((2,), "int64"), T, states_out=states, stream=stream)}


@pytest.mark.parametrize("call", ["retrieve", "retrieve_keys", "retrieve_topk", "delta_scan"])
@pytest.mark.parametrize("stream", [None, "torch", "raw"])
def test_a_workspace_is_taken_on_the_stream_that_uses_it(world, call, stream):
    made, lib = world
    other = {None: None, "torch": Stream(7), "raw": types.SimpleNamespace(cuda_stream=9)}[stream]
    _calls(other)[call]()
    assert len(made) == 1 and len(lib.streams) == 1
    assert made[0].stream == lib.streams[0] == {None: 1, "torch": 7, "raw": 9}[stream]
