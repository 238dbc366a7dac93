"""The cache's 8-bit form, branching, dropping and rotation without a GPU: sizes, refusals that come before any device call, the
binding's structure, and how 8-bit attention is cut into parts."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2503_14153_amd as sd
from paper_2503_14153_amd import binding
from tests.test_abi import _defines, _struct_fields, lib  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def config(**more):
    return binding._Config(**{**dict(n_layers=32, d_model=4096, n_heads=32, head_dim=128, d_ffn=11008, vocab=32016, n_medusa=4, topk=10,
                                     dtype=1, trunc_fallback=0, rope_theta=1e6, rms_eps=1e-5), **more})


def test_the_rope_structure_mirrors_the_header():
    assert _struct_fields("sd_rope") == [f[0] for f in binding._Rope._fields_]
    d = _defines()
    assert (d["SD_ROPE_HALF"], d["SD_ROPE_INTERLEAVED"]) == (0, 1)
    assert (d["SD_ROPE_PLAIN"], d["SD_ROPE_LINEAR"], d["SD_ROPE_BY_PARTS"]) == (0, 1, 2)
    assert d["SD_MAX_DROP_RANGES"] == 16


def test_bytes_of_a_cache_in_8_bits(lib):  # noqa: F811
    # layers * (K and V) * batch * heads * rows rounded up to blocks of 32 * head_dim, and two exponents per block and head (whole
    # words of two blocks)
    assert lib.sd_kv8_bytes(C.byref(config()), 1, 2048) == 32 * 32 * (2 * 2048 * 128 + 64 * 2)
    assert lib.sd_kv8_bytes(C.byref(config()), 8, 4097) == 32 * 8 * 32 * (2 * 4128 * 128 + 130 * 2)
    assert lib.sd_kv8_bytes(None, 1, 16) == 0 and lib.sd_kv8_bytes(C.byref(config()), 0, 16) == 0
    assert lib.sd_kv8_bytes(C.byref(config(dtype=0)), 1, 16) == 0          # float32 models have no such cache


def test_null_arguments_are_refused(lib):  # noqa: F811
    null, code = None, _defines()["SD_ERR_NULL"]
    one = (C.c_int32 * 1)(0)
    assert lib.sd_kv8_create(null, 1, 64, null, 0, null) == code
    assert lib.sd_kv_write_layers(null, 0, 0, 1, null, null, null) == code
    assert lib.sd_kv_read_layers(null, 0, 0, 1, null, null, null) == code
    assert lib.sd_kv_fork(null, 0, null, one, 1, null) == code
    assert lib.sd_kv_drop_rows(null, 0, one, one, 1, null) == code
    assert lib.sd_tree_attention(null, null, null, 0, null, null, null, 0, null, 0, null) == code
    assert lib.sd_set_rope(null, null, null) == code
    assert lib.sd_rope_rows(null, 1, null, 64, null, 64, null, 1, 1, 64, 0, null) == code
    r = sd.Rope(1e4, 64)._c()
    assert lib.sd_rope_rows(C.byref(r), 1, null, 64, null, 64, null, 1, 1, 64, 0, null) == code
    assert lib.sd_rope_rows(C.byref(r), 1, null, 64, null, 64, null, 0, 1, 64, 0, null) == 0         # no rows: nothing to do


GOOD = dict(theta=1e4, rotary_dim=64, layout=0, scaling=0, factor=1.0, low=1.0, high=4.0, trained_len=4096, magnitude=1.0)


@pytest.mark.parametrize("bad", [dict(theta=0.0), dict(theta=-1.0), dict(theta=float("inf")), dict(theta=float("nan")), dict(rotary_dim=0),
                                 dict(rotary_dim=7), dict(rotary_dim=258), dict(rotary_dim=128), dict(layout=2), dict(scaling=3),
                                 dict(scaling=-1), dict(magnitude=0.0), dict(magnitude=float("nan")), dict(scaling=1, factor=0.0),
                                 dict(scaling=2, factor=float("inf")), dict(scaling=2, low=4.0), dict(scaling=2, trained_len=0)])
def test_bad_rotations_are_refused(lib, bad):  # noqa: F811
    r = binding._Rope(**{**GOOD, **bad})
    assert lib.sd_rope_rows(C.byref(r), 1, 16, 64, 16, 64, 16, 4, 1, 64, 0, None) == _defines()["SD_ERR_SHAPE"]


@pytest.mark.parametrize("dtype,ld_x,ld_y,n,heads,dim,x,y", [
    (2, 64, 64, 4, 1, 64, 16, 32), (1, 63, 64, 4, 1, 64, 16, 32), (1, 64, 63, 4, 1, 64, 16, 32), (1, 64, 64, -1, 1, 64, 16, 32),
    (1, 64, 64, 4, 0, 64, 16, 32), (1, 64, 64, 4, 1, 32, 16, 32), (1, 64, 128, 4, 1, 64, 16, 16), (1, 64, 64, 4, 1, 64, 17, 32),
    (0, 64, 64, 4, 1, 64, 16, 34), (1, 10 ** 6, 10 ** 6, 4, 1025, 64, 16, 32), (1, 2048, 2048, 4, 1, 2048, 16, 32)])
def test_bad_rows_are_refused(lib, dtype, ld_x, ld_y, n, heads, dim, x, y):  # noqa: F811
    r = binding._Rope(**GOOD)
    assert lib.sd_rope_rows(C.byref(r), dtype, x, ld_x, y, ld_y, 16, n, heads, dim, 0, None) == _defines()["SD_ERR_SHAPE"]


# ---------------------------------------------------------------------------------------------- parts of 8-bit attention
CODE = """
#include "attn_geom.h"
extern "C" int split(int groups, int resident, int B, int TB, const int* len, int most, unsigned* slot, int* each, int* share, int* max_parts) {
    Attn8Split s = attn8_split(groups, resident, B, TB, len, most);
    for (int i = 0; i < s.n; ++i) { slot[i] = s.slot[i]; each[i] = s.each[i]; share[i] = s.share[i]; }
    *max_parts = s.max_parts;
    return s.n;
}
"""


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    d = tmp_path_factory.mktemp("split8")
    (d / "split.cpp").write_text(CODE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2503_14153_amd", "csrc"), str(d / "split.cpp"), "-o", str(d / "split.so")], check=True)
    f = C.CDLL(str(d / "split.so")).split

    def call(groups, resident, TB, lens, most):
        slot, each, share, parts = (C.c_uint * 64)(), (C.c_int * 64)(), (C.c_int * 64)(), C.c_int()
        n = f(groups, resident, len(lens), TB, (C.c_int * len(lens))(*lens), most, slot, each, share, C.byref(parts))
        assert 1 <= n <= 64
        return [(slot[i] & 255, slot[i] >> 8 & 255, slot[i] >> 16, each[i], share[i]) for i in range(n)], parts.value
    return call


@pytest.mark.parametrize("groups", [1, 4, 32, 40, 128, 512])
@pytest.mark.parametrize("TB", [1, 2, 8])
@pytest.mark.parametrize("lens", [[0], [1], [500], [16873], [10 ** 6], [0, 0, 0], [4096, 1024, 7, 0], [5] * 32, [17000] * 32,
                                  [0] * 31 + [16896]])
def test_every_sequence_has_its_parts_once_and_they_cover_its_blocks(split, groups, TB, lens):
    most = 15 if len(lens) > 1 else 65
    entries, max_parts = split(groups, 256 if TB > 1 else 512, TB, lens, most)
    assert max_parts == max(e[2] for e in entries) <= most
    for b, bound in enumerate(lens):
        mine = [e for e in entries if e[0] == b]
        own = mine[0][2]
        assert [e[1] for e in mine] == list(range(own)) and all(e[2] == own for e in mine)
        # what the waves take of it, at lengths up to the bound and (a launch that is replayed) beyond it
        for n in {0, 1, bound // 2, max(0, bound - 33), bound, bound + 40, 3 * bound + 1000}:
            nblk, seen = (n + 31) // 32, 0
            for _, part, _, each, share in mine:
                end = nblk if part == own - 1 else min(nblk, (part + 1) * each)
                for quarter in range(4):
                    first = part * each + quarter * share
                    last = end if quarter == 3 else min(end, first + share)
                    if first < last:
                        assert first == seen               # one after the other, nothing twice, nothing left out
                        seen = last
            assert seen == nblk
        if bound:                                      # at the bound itself the waves have about the same
            most_blocks = max(e[4] for e in mine)
            assert most_blocks <= -(-(-(-(-(-bound // 32) + TB) // own)) // 4)
