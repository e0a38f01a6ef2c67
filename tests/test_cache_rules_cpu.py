"""How the cache's attention deals out its work (csrc/rules.hpp), compiled for the host."""

import ctypes
import shutil
import subprocess

import pytest

from paper_2605_06206_amd import build as build_mod


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not found")
    tmp = tmp_path_factory.mktemp("rules")
    # walks a range through tiles of np pages, the first entered at page blk0: units taken
    (tmp / "r.cpp").write_text(
        '#include "rules.hpp"\n'
        'extern "C" long long per(long long total, int ranges, int least, int round) {\n'
        '  return foe::range_units(total, ranges, least, round);\n}\n'
        'extern "C" long long walk(int np, int blk0, long long left) {\n'
        '  long long taken = 0;\n'
        '  for (; left > 0; blk0 = 0) {\n'
        '    const int end = foe::segment_end(np, blk0, left);\n'
        '    if (end <= blk0 || end > np) return -1;\n'
        '    taken += end - blk0;\n'
        '    left -= end - blk0;\n'
        '  }\n'
        '  return taken;\n}\n')
    lib = ctypes.CDLL(str(_compiled(gxx, tmp)))
    for name in ("per", "walk"):
        getattr(lib, name).restype = ctypes.c_longlong
    lib.per.argtypes = [ctypes.c_longlong] + [ctypes.c_int] * 3
    lib.walk.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_longlong]
    return lib


def _compiled(gxx, tmp):
    out = tmp / "r.so"
    subprocess.run([gxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-I", build_mod.CSRC,
                    str(tmp / "r.cpp"), "-o", str(out)], check=True)
    return out


@pytest.mark.parametrize("total,ranges,least,round_", [
    (1, 256, 2, 0), (511, 256, 2, 0), (513, 256, 2, 0), (1 << 37, 1024, 4, 512),
    (22 * 512, 1024, 4, 512), (22 * 512 + 1, 1024, 4, 512), (3, 1, 4, 1),
])
def test_ranges_hold_all_units(rules, total, ranges, least, round_):
    per = rules.per(total, ranges, least, round_)
    assert per >= least and per * ranges >= total
    if round_ and total <= 22 * round_:
        assert per * round_ >= total and (per - 1) * round_ < max(total, least * round_)


def test_ranges_of_the_largest_batch(rules):
    """The most units that the entry point's limits allow: 8192 sequences with tables of 2^18
    pages, 64 groups, 33 heads (tiles of 4 rows) and 127100 rows, 13 or 17 of a sequence."""
    rows = [13] * 8192
    for i in range((127100 - sum(rows)) // 4):
        rows[i] = 17
    tiles = sum(-(-n // 4) for n in rows)
    total = tiles * (1 << 18) * 64
    assert total > 1 << 39
    per = rules.per(total, 256, 2, 0)
    assert per > 1 << 31 and per * 256 >= total
    for blk0 in (0, 1, (1 << 18) - 1):
        assert rules.walk(1 << 18, blk0, per) == per


@pytest.mark.parametrize("np_,blk0,left", [(1, 0, 1), (7, 3, 2), (7, 3, 4), (7, 3, 5), (7, 6, 100)])
def test_a_range_ends_inside_a_tile(rules, np_, blk0, left):
    assert rules.walk(np_, blk0, left) == left
