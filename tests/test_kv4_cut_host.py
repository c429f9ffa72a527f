"""Which form of attention over the 4-bit cache a call takes, on the host: the tests of a form reach it, and the workspace is what the
form needs.  The library keeps the choice to itself; a few lines compiled against its header ask for it."""
import ctypes as C
import subprocess

import pytest

from paper_2105_01827_amd import binding, build as lib_build
from tests import test_gpu_kv4_unseen_scales as unseen, test_gpu_kv4_wide as wide
from tests.test_gpu_kv4_attention import _many

READER = """
#include "gala_attention4_cut.h"
extern "C" int read_cut(int heads, int dim, int count, int max_new, int max_len, int table_stride, int heads_q, int window, int sinks, float scale,
                        int q_type, int out_type, long *places) {
    gala::KvArgs kv{};
    kv.heads = heads, kv.dim = dim, kv.count = count, kv.max_new = max_new, kv.max_len = max_len, kv.table_stride = table_stride;
    const bool fine = !gala::in_halves(scale, q_type, out_type);
    const gala::Cut c = gala::cut_of(kv, heads_q, window, sinks, fine || !gala::fits_wide(q_type, dim));
    *places = c.splits == 1 ? 0 : c.places();
    return c.many;
}
"""
KINDS = {"f32": 0, "f16": 1, "bf16": 2, "residue": 3}


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    at = tmp_path_factory.mktemp("reader")
    (at / "reader.cpp").write_text(READER)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", lib_build.CSRC, str(at / "reader.cpp"), "-o", str(at / "reader.so")])
    lib = C.CDLL(str(at / "reader.so"))

    def read(new, lens, heads, group, dim, kind, out, window, sinks):
        """(whether a wavefront has 32 queries, bytes of workspace)"""
        places, count, max_new, max_len = C.c_long(), len(new), max(new), max(lens)
        many = lib.read_cut(heads, dim, count, max_new, max_len, -(-max_len // 64), heads * group, window, sinks, C.c_float(dim ** -0.5),
                            KINDS[kind], KINDS[out], C.byref(places))
        return bool(many), count * heads * places.value * (dim + 2) * 4
    return read


def test_cases_of_the_wide_form_take_it(cut):
    for args in [*wide.ALL_ROWS.values(), *wide.LONG.values(), wide.RISING]:
        assert cut(*args)[0], args
    for new in (1, 60, 130):
        assert cut([new, new], [300, 500], _many(new), 2, 64, "bf16", "bf16", unseen.WINDOW, unseen.SINKS)[0] == (new == 130)


@pytest.mark.parametrize("dim", [1, 32, 64, 80, 128, 160, 192, 200, 256])
def test_types_that_the_wide_form_does_not_have(cut, dim):
    many = [300, 300], [300, 300], 64, 4, dim
    for kind in KINDS:
        for out in KINDS:
            wanted = {kind, out} <= {"f16", "bf16"} and not (kind == "f16" and dim > 192)
            assert cut(*many, kind, out, 0, 0)[0] == wanted
    assert not cut([31], [300], 64, 4, dim, "bf16", "bf16", 0, 0)[0]         # fewer than 128 queries of a head


@pytest.mark.parametrize("dim", [33, 64, 128, 256])
def test_the_workspace_is_what_shares_need(cut, dim):
    for count, new, length, window in ((1, 1, 131072, 0), (1, 1, 4000, 0), (64, 1, 8192, 0), (3, 7, 20000, 5000), (1, 300, 6000, 0), (2, 2000, 5207, 0), (1, 1, 64, 0)):
        batch = binding.KvBatchArg(count, new, length, -(-length // 64), 1 << 20, 1 << 20, 1 << 20)
        cache = binding.Kv4CacheArg(8, dim, 4, 0, 1 << 20)
        need = binding.load().gala_kv4_attention_workspace(C.byref(cache), C.byref(batch), 16, window, 0)
        assert need == cut([new] * count, [length] * count, 8, 2, dim, "f32", "f32", window, 0)[1]
        for kind in ("f16", "bf16"):                                         # whatever the types are
            assert need >= cut([new] * count, [length] * count, 8, 2, dim, kind, kind, window, 0)[1]
