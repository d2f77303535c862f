"""The launch shape of a pass over the shared prefix (csrc/prefix_rule.h), a pure function of what the host knows:
its limits over a grid of batches.  Compiled with the host compiler (CPU only)."""
import ctypes
import itertools
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_00085_amd", "csrc")
WRAP = """
#include "prefix_rule.h"
using namespace td;
extern "C" void shape(int tries, int heads, int kv, int dim, int f32, int four, int layers, int queries, long keys, long fit, int most,
                      long nodes, int* out) {
  const PassShape a = prefix_pass_shape(PrefixHeads{tries, heads, kv, dim, f32 != 0}, four != 0, layers, queries, keys, fit, most, nodes);
  const int x[6] = {a.row_blocks, a.splits, a.xcd_group, a.trie_splits, a.trie_blocks, (int)a.prefix_wgs};
  for (int i = 0; i < 6; ++i) out[i] = x[i];
}
"""


class Shape:
    def __init__(self, x):
        self.row_blocks, self.splits, self.xcd_group, self.trie_splits, self.trie_blocks, self.prefix_wgs = x

    def __eq__(self, other):
        return vars(self) == vars(other)

    def __repr__(self):
        return str(vars(self))


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    d = tmp_path_factory.mktemp("prefix_rule")
    (d / "w.cpp").write_text(WRAP)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "w.cpp"),
                    "-o", str(d / "w.so")], check=True)
    L = ctypes.CDLL(str(d / "w.so"))
    L.shape.argtypes = [ctypes.c_int] * 8 + [ctypes.c_long] * 2 + [ctypes.c_int, ctypes.c_long, ctypes.c_void_p]

    def call(tries, beams, G, kv, dim, keys, nodes, layers=1, four=True, f32=False):
        records = max((16 << 20) // dim, tries * kv * max(beams * G, 128))  # (as td_set_prefix reserves)
        out = (ctypes.c_int * 6)()
        L.shape(tries, G * kv, kv, dim, f32, four, layers, beams, keys, records // (layers * tries * beams * G * kv), 64, nodes, out)
        return Shape(out)

    return call


GRID = list(itertools.product((1, 2, 3, 5, 7, 10, 16), (1, 4, 8, 16), (1, 4), (1, 4, 8, 32), (64, 1000, 2000, 4096, 20000, 50000),
                              (30, 300, 868, 4000, 8000), (1, 4), (True, False)))


def test_a_pass_without_the_tries_has_its_own_splits(shape):
    """Where the tries' nodes do not join the launch, they change nothing of it."""
    joined = 0
    for tries, beams, G, kv, keys, nodes, layers, four in GRID:
        a = shape(tries, beams, G, kv, 128, keys, nodes, layers, four)
        if a.trie_splits == 0:
            assert a == shape(tries, beams, G, kv, 128, keys, 0, layers, four), (tries, beams, G, kv, keys, nodes, layers, four)
        joined += a.trie_splits > 0
    assert 0 < joined < len(GRID)
    # 5 tries of 4 beams and 4,000 nodes, 8 heads: 63 tiles of a trie are too many for the launch, the pass has 8 splits
    assert shape(5, 4, 1, 8, 128, 2000, 4000).splits == 8


def test_limits_of_a_launch(shape):
    for tries, beams, G, kv, keys, nodes, layers, four in GRID:
        a = shape(tries, beams, G, kv, 128, keys, nodes, layers, four)
        case = (tries, beams, G, kv, keys, nodes, layers, four, a)
        assert a.splits >= 1 and a.row_blocks >= 1, case
        fit = max((16 << 20) // 128, tries * kv * max(beams * G, 128)) // (layers * tries * beams * G * kv)
        assert a.splits + a.trie_splits <= max(1, fit), case
        if a.xcd_group:  # (how the kernels take a block's number apart)
            assert layers * kv * a.splits % 8 == 0, case
        if a.trie_splits:
            assert a.prefix_wgs == layers * kv * a.row_blocks * a.splits, case
            assert a.prefix_wgs + layers * tries * kv * a.trie_blocks * a.trie_splits <= 512, case  # two per CU
            assert ((nodes + 63) // 64 + a.trie_splits - 1) // a.trie_splits <= 8, case
            rows = 64 if four else (32 if tries * beams * G <= 32 else 64 if tries * beams * G <= 64 else 128)
            if not four or tries * beams * G <= 512:
                assert a.trie_blocks * rows >= beams * G, case


def test_a_short_pass_stays_short_as_the_tries_grow(shape):
    """A captured call goes by the tries' capacity, the same call outside a graph by the nodes that they have: a few more
    nodes change a short pass's splits by little, and it stays within a workgroup per CU."""
    # 4 x 8 beams of 32 heads (8 KV heads) over 4,096 positions, 736 nodes stored, room for 868
    for nodes in (736, 868):
        a = shape(4, 8, 4, 8, 128, 4096, nodes)
        assert (a.splits, a.trie_splits) == (4, 4), nodes
    for tries, beams, G, kv, keys in ((4, 8, 4, 8, 4096), (4, 16, 4, 8, 2500), (8, 8, 4, 8, 1000), (4, 8, 4, 8, 6000), (2, 4, 1, 32, 1000)):
        before, tiles = None, 0
        while True:
            tiles += 1
            a = shape(tries, beams, G, kv, 128, keys, 64 * tiles)
            wgs = a.prefix_wgs + tries * kv * a.trie_blocks * a.trie_splits
            if a.trie_splits == 0 or wgs > 256:
                break  # (the tries are too large for it)
            case = (tries, beams, G, kv, keys, tiles, a)
            assert a.splits >= min(shape(tries, beams, G, kv, 128, keys, 0).splits, -(-keys // 64 // 16)), case
            assert before is None or abs(a.splits - before) <= 2, case
            before = a.splits
        assert tiles > 12, (tries, beams, keys, tiles)
