"""The launcher of a pass over the shared prefix refuses shapes that its kernels would read out of range with: each is
refused on the host, before anything is launched.  CPU only (a shim calls the library's launcher)."""
import ctypes
import os
import subprocess

import pytest

from paper_2502_00085_amd import binding, build

SHIM = """
#include "prefix.h"
// 2 of 4 layers, 4 KV heads, 3 row blocks of 32 rows; the call's own fields from x
extern "C" int launch(int four, int layer_begin, int n_layers, int splits, int records, int xcd_group, int trie_splits, int prefix_wgs) {
  td::DevState s{};
  s.T = 2;
  s.L = 4;
  s.Hq = 16;
  s.Hkv = 4;
  s.D = 128;
  s.dtype = TD_BF16;
  td::PrefixArgs a{};
  a.rows = td::PrefixRows::kLeaves;
  a.four = four;
  a.layer_begin = layer_begin;
  a.n_layers = n_layers;
  a.tries = 2;
  a.per_trie = 12;
  a.row_blocks = 3;
  a.splits = splits;
  a.records = records;
  a.xcd_group = xcd_group;
  a.trie_splits = trie_splits;
  a.trie_blocks = 1;
  a.prefix_wgs = prefix_wgs;
  return td::launch_prefix(s, a, nullptr, nullptr, nullptr);
}
"""


@pytest.fixture(scope="module")
def launch(tmp_path_factory):
    binding.lib()  # (built)
    d = tmp_path_factory.mktemp("prefix_launch")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run([build.hipcc(), "-O1", "-std=c++17", "-fPIC", "-shared", "--cuda-host-only", "-I", os.path.join(build.ROOT, "include"),
                    "-I", build.CSRC, str(d / "shim.cpp"), "-L", build.PKG, "-l:libtriedecode.so", "-Wl,-rpath," + build.PKG,
                    "-o", str(d / "shim.so")],
                   check=True, capture_output=True)
    return ctypes.CDLL(str(d / "shim.so")).launch


@pytest.mark.parametrize("four", [0, 1])
@pytest.mark.parametrize("case", [
    # (layer_begin, n_layers, splits, records, xcd_group, trie_splits, prefix_wgs)
    (0, 1, 3, 3, 1, 0, 0),  # 12 (layer, KV head, split) triples: not eights
    (0, 2, 5, 8, 1, 3, 120 + 1),
    (0, 1, 0, 1, 0, 0, 0), (0, 0, 2, 2, 0, 0, 0),
    (3, 2, 2, 2, 0, 0, 0), (-1, 2, 2, 2, 0, 0, 0),  # past the layers
    (0, 2, 4, 3, 0, 0, 0), (0, 2, 4, 5, 0, 2, 96),  # more splits than records
    (0, 2, 4, 6, 0, 2, 95), (0, 2, 4, 6, 1, 2, 48),  # another number of the pass's WGs
])
def test_a_launch_that_does_not_fit_is_refused(launch, four, case):
    assert launch(four, *case) == 1  # hipErrorInvalidValue
