"""Which keys a tile of query rows sees and how they are dealt out to CTAs
(csrc/kv8_keys.h), compiled for the host, against counting token by token."""
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
extern "C" int units(int pos0, int pos1, int window, int sinks, int* tokens) {
  const tsd::KeyTiles k = tsd::key_tiles(pos0, pos1, window, sinks);
  for (int i = 0; i < k.total; ++i) tokens[i] = k.token(i);
  return k.total;
}
''')
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-shared", "-fPIC", "-I", _build.CSRC, "-o", str(d / "k.so"),
                    str(d / "k.cpp")], check=True)
    return ctypes.CDLL(str(d / "k.so"))


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
