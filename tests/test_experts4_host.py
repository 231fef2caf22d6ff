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


def cut(lib, E, D, F, K, T, align=16):
    """'short' (with the rows of a tile), 'long' or 'both'."""
    out = (ctypes.c_int * 2)()
    lib.cut(ctypes.byref(binding.Shape(T, D, F, E, K, E, 0, align).c_struct()), out)
    if out[1] == 2 ** 31 - 1:
        return f"short {out[0]}"
    return "both" if out[1] else "long"


LAYERS = dict(fine=(256, 7168, 2048, 8), mixtral=(8, 4096, 14336, 2), many=(64, 2048, 1408, 6), light=(8, 1024, 2048, 2))


@pytest.mark.parametrize("align", [64, 128, 256])
def test_padding_is_rows_like_others(lib, align):
    """Few tokens whose slots are aligned to more rows than a tile has: as many rows an expert as the alignment."""
    for name, (E, D, F, K) in LAYERS.items():
        for T in (1, 2, 8, 32):
            whole = max(1, align * min(E, T * K) // K)   # tokens that fill as many rows
            few, full = cut(lib, E, D, F, K, T, align), cut(lib, E, D, F, K, align * E // K, align)
            assert few == full, (name, T, whole)
    assert cut(lib, *LAYERS["fine"], 1, align) == "long"
    if align > 96:
        assert cut(lib, *LAYERS["mixtral"], 1, align) == cut(lib, *LAYERS["many"], 8, align) == "long"
    assert cut(lib, *LAYERS["light"], 1, align) == "short 48"


@pytest.mark.parametrize("align", [1, 16, 32])
def test_cut_of_layers(lib, align):
    for name, T, want in (("fine", 1, "short 32"), ("fine", 64, "short 32"), ("fine", 128, "both"), ("fine", 4096, "both"),
                          ("mixtral", 1, "short 32"), ("mixtral", 96, "short 32"), ("mixtral", 128, "short 48"),
                          ("mixtral", 384, "short 48"), ("mixtral", 400, "long"), ("mixtral", 16384, "long"),
                          ("many", 48, "short 32"), ("many", 512, "short 48"), ("many", 8192, "long"),
                          ("light", 1, "short 32"), ("light", 256, "short 48"), ("light", 2048, "long")):
        assert cut(lib, *LAYERS[name], T, align) == want, (name, T)
    # few experts, whatever their weights, are not worked in both ways before they have dozens of rows each; many are
    assert cut(lib, 24, 4096, 14336, 2, 288) == "short 32" and cut(lib, 24, 4096, 14336, 2, 576) == "short 48"
    assert cut(lib, 160, 4096, 1536, 8, 960) == "both" and cut(lib, 128, 4096, 1280, 8, 768) == "both"


@pytest.mark.parametrize("E", [8, 32, 64, 160, 256])
def test_cut_does_not_jump_with_the_weights(lib, E):
    """A few columns more change the rows an expert from which both ways are taken by as little."""
    first = []
    for F in range(1024, 16385, 256):
        first.append(next((per for per in range(1, 600) if not cut(lib, E, 4096, F, 1, per * E).startswith("short")), 600))
    assert all(b <= a and a - b <= 1 + a * 0.25 for a, b in zip(first, first[1:])), first
