"""What the host decides for experts in 4 bits (csrc/mx4.cuh): blocks, the cut of the rows, the workspace."""
import ctypes

import pytest

from paper_2506_07366_b200 import binding
from tests import host_code

SOURCE = """
#include "mx4.cuh"
extern "C" int short_blocks(int sms) { return mx4::short_blocks(sms); }
extern "C" int max_blocks() { return mx4::kMaxCtas; }
extern "C" void cut(const moegps_shape_t* s, int* out) {
  const mx4::Cut c = mx4::cut_of(*s);
  out[0] = c.tile_rows;
  out[1] = c.short_rows;
}
extern "C" long long partial_bytes(const moegps_shape_t* s) {
  const mx4::Layout l = mx4::layout_of(*s);
  return (long long)(l.x_code - l.partial);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    lib = host_code.compiled(tmp_path_factory.mktemp("experts4"), SOURCE)
    lib.partial_bytes.restype = ctypes.c_longlong
    return lib


def test_blocks_that_wait_for_one_another(lib):
    """As many as SMs: with fewer, those of another launch could begin beside them and be counted with them.  Every one has its place in
    the workspace, or the call is refused."""
    most = lib.max_blocks()
    for sms in (1, 108, 132, 148, 152, 160, most):
        assert lib.short_blocks(sms) == sms
    for sms in (most + 1, 256):
        assert lib.short_blocks(sms) == 0
    for T in (1, 4096):
        s = binding.Shape(T, 256, 384, 8, 2, 8)
        out = (ctypes.c_int * 2)()
        lib.cut(ctypes.byref(s.c_struct()), out)
        # three parts, two weight tiles of 128 outputs each, for the rows of a tile, fp32
        assert lib.partial_bytes(ctypes.byref(s.c_struct())) == most * 3 * 2 * out[0] * 128 * 4
