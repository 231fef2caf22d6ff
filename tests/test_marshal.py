"""The binding's host side without a GPU: what counts as a stream, in Python and in the compiled argument checks."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2506_07366_b200 import binding, build


class Held:
    """A stream object of another library: has a handle."""

    def __init__(self, handle):
        self.cuda_stream = handle


STREAMS = [0, 4096, True, np.int64(4096), np.uint64(2 ** 40 + 16), torch.tensor(4096), ctypes.c_void_p(4096).value, "4096",
           Held(4096), Held(np.int64(4096))]
NO_STREAMS = [object(), [], {}]


def compiled_stream():
    """stream -> the handle that an entry point without tensors gets from the compiled checks."""
    build.build_marshal()
    got = []

    @ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p)
    def entry(context, stream):
        got.append(stream or 0)
        return 0

    call = binding._marshal().Call(ctypes.cast(entry, ctypes.c_void_p).value, 0, binding._ptr, ())

    def handle(stream):
        assert call(stream) == 0, entry                   # (keeps entry alive)
        return got.pop()

    return handle


@pytest.mark.parametrize("of", [lambda: binding._stream, compiled_stream], ids=["python", "compiled"])
def test_stream_arguments(of):
    handle = of()
    for stream in STREAMS:
        want = stream.cuda_stream if isinstance(stream, Held) else stream
        assert handle(stream) == int(want), stream
    for stream in NO_STREAMS:
        with pytest.raises(AttributeError):
            handle(stream)
    with pytest.raises(ValueError):
        handle("four")
