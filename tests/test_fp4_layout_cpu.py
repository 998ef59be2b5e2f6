"""csrc/fp4_layout.h itself, compiled for the host: where the kernels of the 4-bit cache write, read and convert a page, and the
transposition of values in LDS."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2207_10284_amd import ops
from paper_2207_10284_amd.build import CSRC

WIDTHS = (32, 64, 128)
SOURCE = """
#include "fp4_layout.h"
using namespace mra;
template <int D, int C> void row_unit(int unit, int slot, int size, int* o) {
  const Fp4RowUnit<D, C> u(unit);
  const int x[] = {u.value, u.r, u.c, u.codes_at(slot, size), u.step_at(slot, size), Fp4RowUnit<D, C>::kUnits};
  for (int i = 0; i < 6; ++i) o[i] = x[i];
}
template <int D, int T> void stage_unit(int n, int tid, int* o) {
  const Fp4StageUnit<D, T> u(n, tid);
  o[0] = u.x; o[1] = u.r; o[2] = u.blk; o[3] = Fp4StageUnit<D, T>::N;
}
extern "C" {
int row_tokens() { return kFp4RowTokens; }
int row_tiles(int n) { return fp4_row_tiles(n); }
int tile_row(int value, int x, int i) { return fp4_tile_row(value, x, i); }
#define WIDTH(D) \\
  int codes_##D(int x, int size) { return Fp4Page<D>::codes(x, size); } \\
  int steps_##D(int x, int size) { return Fp4Page<D>::steps(x, size); } \\
  int place_##D(int r, int c) { return fp4_value_place<D>(r, c); } \\
  void write_##D(int unit, int slot, int size, int* o) { row_unit<D, 16>(unit, slot, size, o); } \\
  void read_##D(int unit, int slot, int size, int* o) { row_unit<D, 8>(unit, slot, size, o); } \\
  void stage_##D##_256(int n, int tid, int* o) { stage_unit<D, 256>(n, tid, o); }
WIDTH(32) WIDTH(64) WIDTH(128)
void stage_128_512(int n, int tid, int* o) { stage_unit<128, 512>(n, tid, o); }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cc = shutil.which("g++") or shutil.which("c++")
    if cc is None:
        pytest.skip("no host compiler")
    at = tmp_path_factory.mktemp("layout")
    (at / "layout.cpp").write_text(SOURCE)
    subprocess.run([cc, "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(at / "layout.cpp"), "-o", str(at / "layout.so")],
                   check=True)
    return ctypes.CDLL(str(at / "layout.so"))


def call(f, *args, n):
    out = (ctypes.c_int * n)()
    f(*args, out)
    return list(out)


def test_the_kernels_use_it():
    for name in ("fp4_cache.hip", "fp4_attention.hip"):
        text = open(os.path.join(CSRC, name)).read()
        assert "fp4_tile.h" in text and '#include "fp4_layout.h"' in open(os.path.join(CSRC, "fp4_tile.h")).read()
        for own in (("Fp4RowUnit<D, 16>", "Fp4RowUnit<D, 8>", "fp4_row_tiles") if name == "fp4_cache.hip" else
                    ("Fp4StageUnit<D, T>", "fp4_tile_row", "fp4_value_place<D>")):
            assert own in text


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("size", [32, 64, 1024])
@pytest.mark.parametrize("kind,chunk", [("write", 16), ("read", 8)])
def test_writing_and_reading_reach_every_byte_once(lib, d, size, kind, chunk):
    """All units of a page's tokens: of keys and values each byte of codes, each step, and nothing else; a token's
    codes lie together, by channel, as the ABI's header has them."""
    f, tokens = getattr(lib, f"{kind}_{d}"), lib.row_tokens()
    total = ops.fp4_page_bytes(size, d)
    units = call(f, 0, 0, size, n=6)[5]
    assert units == 2 * tokens * d // chunk and units % 256 == 0
    codes, steps = {}, {}
    for unit in range(units):
        value, r, c = call(f, unit, 0, size, n=6)[:3]
        assert value in (0, 1) and 0 <= r < tokens and 0 <= c < d // chunk
        if r >= size:
            continue
        for slot in range(r, size, tokens):                # token r of each tile of the page
            at, step = call(f, unit, slot, size, n=6)[3:5]
            assert at == value * size * d // 2 + slot * d // 2 + c * chunk // 2
            assert step == size * d + value * size * d // 32 + slot * d // 32 + c * chunk // 32
            assert at % (chunk // 2) == 0
            for byte in range(at, at + chunk // 2):
                assert byte not in codes
                codes[byte] = unit
            steps.setdefault(step, set()).add(unit)
    assert sorted(codes) == list(range(size * d)) and sorted(steps) == list(range(size * d, total))
    assert all(len(s) == 32 // chunk for s in steps.values())


def test_tiles_that_tokens_touch(lib):
    t = lib.row_tokens()
    for n in (1, 2, 3, 31, 62, 63, 64, 65, 66, 127, 128, 129, 1000, 4097):
        assert lib.row_tiles(n) == max((start + n - 1) // t + 1 for start in range(t))
    assert lib.row_tiles(1 << 26) == (1 << 20) + 1


@pytest.mark.parametrize("d,threads", [(32, 256), (64, 256), (128, 256), (128, 512)])
def test_a_stage_converts_every_block_once(lib, d, threads):
    f = getattr(lib, f"stage_{d}_{threads}")
    per = call(f, 0, 0, n=4)[3]
    seen = [tuple(u[:3]) for u in (call(f, n, tid, n=4) for tid in range(threads) for n in range(per)) if u[0] < 2]
    assert sorted(seen) == [(x, r, b) for x in range(2) for r in range(64) for b in range(d // 32)]
    for size in (32, 64, 1024):                            # 16 bytes of codes and a step of each, in the page
        for x, r, b in seen:
            slot = size - 32 + r % 32
            at = getattr(lib, f"codes_{d}")(x, size) + slot * (d // 2) + b * 16
            assert at % 16 == 0 and at + 16 <= (x + 1) * size * d // 2
            assert getattr(lib, f"steps_{d}")(x, size) + slot * (d // 32) + b < ops.fp4_page_bytes(size, d)


@pytest.mark.parametrize("d", WIDTHS)
def test_values_come_back_transposed(lib, d):
    """What lanes put and get in a wave's value tile: every place once, lane (g, i) of the transposing read t has channel
    16 t + i of rows 8 g .. 8 g + 7, whose weights the first product left in the same lane group."""
    place = getattr(lib, f"place_{d}")
    assert sorted(place(r, c) for r in range(32) for c in range(0, d, 4)) == list(range(0, 64 * d, 8))
    lds = {}
    for lane in range(64):                                 # row 16 x + i of the values, chunk n of eight channels
        g, i = lane >> 4, lane & 15
        for x in range(2):
            row = lib.tile_row(1, x, i)
            for n in range(d // 32):
                at = (place(i, g * (d // 4)) ^ 16 * n) + x * 16 * 2 * d
                for e in range(8):
                    lds[at + 2 * e] = (row, g * (d // 4) + 8 * n + e)
    assert len(lds) == 32 * d
    for t in range(d // 16):                               # lane i of 16 receives element i % 4 of the 8 bytes of lane 4 k + i / 4
        for lane in range(64):
            g, i = lane >> 4, lane & 15
            for e in range(2):
                for k in range(4):
                    j = 4 * k + i // 4
                    at = place(8 * g + 4 * e + (j >> 2), 4 * (j & 3)) ^ 32 * t
                    assert lds[at + 2 * (i % 4)] == (8 * g + 4 * e + k, 16 * t + i)


def test_scores_meet_their_keys(lib):
    """Row 4 g + r of the first product's part x is the key that lane i = 4 g + r loaded: of group g the eight keys 8 g .."""
    for g in range(4):
        keys = [lib.tile_row(0, x, 4 * g + r) for x in range(2) for r in range(4)]
        assert keys == list(range(8 * g, 8 * g + 8))
