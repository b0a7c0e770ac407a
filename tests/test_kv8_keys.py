"""Which keys a tile of query rows sees and how they are dealt out to CTAs
(csrc/kv8_keys.h), compiled for the host, against counting token by token; and the
size of an append's launch."""
import ctypes
import os
import subprocess

import pytest

from paper_2609_14991_gb300 import _build

UNIT = 16


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("keys")
    (d / "k.cpp").write_text('''#include "kv8_keys.h"
extern "C" int share(int units, int tile, int step, int split, int splits, int* out) {
  const tsd::KeyShare s = tsd::key_share(units, tile, step, split, splits);
  out[0] = s.lo, out[1] = s.n, out[2] = s.steps;
  return 0;
}
extern "C" long long blocks(int n, int rows, int starts, int max_new, int block) {
  return tsd::append_blocks(n, rows, starts, max_new, block);
}
extern "C" int units(int pos0, int pos1, int window, int sinks, int* tokens) {
  const tsd::KeyTiles k = tsd::key_tiles(pos0, pos1, window, sinks);
  for (int i = 0; i < k.total; ++i) tokens[i] = k.token(i);
  return k.total;
}
''')
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-shared", "-fPIC", "-I", _build.CSRC, "-o", str(d / "k.so"),
                    str(d / "k.cpp")], check=True)
    k = ctypes.CDLL(str(d / "k.so"))
    k.blocks.restype = ctypes.c_longlong
    return k


def test_shares_of_keys(lib):
    """Every total and split: shares adjoin, hold all units once, and take as many steps as their units need, none if empty."""
    out = (ctypes.c_int * 3)()
    for splits in range(1, 65):
        for units in range(1, 300):
            at = 0
            for split in range(splits):
                lib.share(units, 8, 4, split, splits, out)
                lo, n, steps = out
                assert lo == at and n >= 0
                at += n
                mine = [u for u in range(8 * lo, 8 * (lo + n)) if u < units]
                assert steps == -(-len(mine) // 4), (units, split, splits, steps)
            assert at == -(-units // 8)


def test_units_hold_every_key_that_is_seen(lib):
    """A rows' list of units: ascending, each with a key that some row sees, and all such keys."""
    out = (ctypes.c_int * 64)()
    for pos0 in (0, 1, 15, 16, 40, 130):
        for rows in (1, 5, 33):
            for window in (0, 1, 2, 16, 17, 50, 2 ** 31 - 1):
                for sinks in (0, 1, 16, 17, 40, 2 ** 31 - 1):
                    pos1 = pos0 + rows - 1
                    n = lib.units(pos0, pos1, window, sinks, out)
                    seen = {j // UNIT for p in range(pos0, pos1 + 1) for j in range(p + 1)
                            if window == 0 or j > p - window or j < sinks}
                    assert [t // UNIT for t in out[:n]] == sorted(seen), (pos0, rows, window, sinks)


@pytest.mark.parametrize("block", [16, 32, 64])
def test_an_appends_launch_grows_with_its_rows(lib, block):
    """A row each takes one block's CTAs, however many sequences; without bounds a launch is linear in rows and
    sequences; a given bound has CTAs for every block that as many rows may touch."""
    for n in (1, 2, 64, 1024, 65535):
        assert lib.blocks(n, n, 0, 0, block) == 1
        for rows in (1, n // 2 + 1, n, 3 * n, 1 << 22):
            per = lib.blocks(n, rows, 1, 0, block)
            assert 1 <= per and n * per <= 16 * (rows + n) / block + 2 * n
            touched = max((start + rows - 1) // block - start // block + 1 for start in range(block))
            assert lib.blocks(1, rows, 1, 0, block) == touched
            for most in (1, 2, block, block + 1, 1000, 1 << 30):
                c = min(most, rows)
                assert lib.blocks(n, rows, 1, most, block) == max((s + c - 1) // block - s // block + 1 for s in range(block))
