"""A prefix in 4 bits and positions of several axes without a GPU: the reference's rounding, and what the
binding and the library refuse before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2502_00085_amd.binding as B
from prefix4_ref import SIZES, pack64, turn_axes, values64
from prefix_ref import turn


def test_rounding_of_a_block():
    """Values between two sizes go to the nearer, ties to the even code; the unit by the largest."""
    y = torch.zeros(32, dtype=torch.float64)
    y[:12] = torch.tensor([6, 5.1, 5, 4.9, 3.5, 3.49, 2.5, 1.75, 1.25, 0.75, 0.25, -0.26])
    e, s = pack64(y)
    assert int(s[0]) == 127
    assert values64(e, s)[:12].tolist() == [6, 6, 4, 4, 4, 3, 2, 2, 1, 1, 0, -0.5]
    for most, unit in ((6.9, 1.0), (7.0, 2.0), (7.9, 2.0), (8.0, 2.0), (4.0, 1.0), (3.99, 1.0), (3.5, 1.0), (3.49, 0.5), (2.0 ** -200, 2.0 ** -125),
                       (2.0 ** 127.9, 2.0 ** 125), (0.0, 2.0 ** -125)):
        y[:] = 0
        y[3] = -most
        e, s = pack64(y)
        assert 2.0 ** (int(s[0]) - 127) == unit, most
        assert abs(float(values64(e, s)[3])) / unit in SIZES.tolist()
    for bad in (float("nan"), float("inf"), -float("inf")):
        y[5] = bad
        e, s = pack64(y)
        assert int(s[0]) == 255 and bool(torch.isnan(values64(e, s)).all())


def test_every_code_stands_for_itself():
    e = torch.arange(256, dtype=torch.uint8).view(16, 16)
    s = torch.full((16, 1), 100, dtype=torch.uint8)
    y = values64(e, s)
    assert sorted(set(y.abs().flatten().tolist())) == (SIZES * 2.0 ** -27).tolist()
    top = y.clone()
    top[:, 0] = 6 * 2.0 ** -27  # (with a 6 in it a block keeps its unit)
    again = values64(*pack64(top))
    assert torch.equal(again, top)


@pytest.mark.parametrize("inter", [False, True])
def test_one_axis_is_the_plain_rotation(inter):
    gen = torch.Generator().manual_seed(0)
    x, f = torch.randn((3, 5, 2, 64), generator=gen), torch.linspace(1, 0.01, 16)
    pos = np.array([0, 3, 100, 7, 12345])
    want = turn(x, pos, f, inter)
    assert float((turn_axes(x, pos[:, None], f, [0] * 16, inter) - want).abs().max()) < 1e-12
    assert float((turn_axes(x, np.stack([pos * 0 + 9, pos], 1), f, [1] * 16, inter) - want).abs().max()) < 1e-12


def test_calls_reject_a_null_context():
    L = B.lib()
    assert L.td_set_prefix4(None, None) == B.TD_EINVAL
    assert L.td_set_prefix4(None, ctypes.byref(B.TdPrefix4())) == B.TD_EINVAL
    assert L.trie_prefix_load(None, 0, 1, 0, 1, None, None, None) == B.TD_EINVAL
    assert L.trie_prefix_store_axes(None, 0, 1, 0, 1, None, None, 0, None, 0, None, 0, None, None) == B.TD_EINVAL
    assert L.trie_store_kv_axes(None, 0, 1, 1, None, None, None, 0, None, 0, None, 0, None, None) == B.TD_EINVAL


class Dev:
    """A host tensor dressed as a device one."""

    def __init__(self, t):
        self.t, self.is_cuda, self.dtype, self.shape = t, True, t.dtype, t.shape

    def is_contiguous(self):
        return self.t.is_contiguous()

    def numel(self):
        return self.t.numel()

    def dim(self):
        return self.t.dim()

    def data_ptr(self):
        return 4096


def dims(**kw):
    d = B.TdDesc(1, 8, 4096, 1000, 2, 8, 2, 128, 0, B.TD_BF16, 0, 1, -1, 1.0, 0, 0x10000, 0x20000)
    for k, v in kw.items():
        setattr(d, k, v)
    return B.Dims(d)


def test_pages_are_checked_before_the_library():
    u8 = dict(dtype=torch.uint8)
    k, s = torch.zeros((3, 2, 2, 16, 64), **u8), torch.zeros((3, 2, 2, 16, 4), **u8)
    for kk, ks, vv, vs in ((k, s, k, s),  # (host tensors)
                           (Dev(k.to(torch.int8)), Dev(s), Dev(k), Dev(s)), (Dev(k), Dev(s.float()), Dev(k), Dev(s)),
                           (Dev(k[:, :1].contiguous()), Dev(s), Dev(k), Dev(s)), (Dev(torch.zeros((3, 2, 2, 16, 128), **u8)), Dev(s), Dev(k), Dev(s)),
                           (Dev(k), Dev(s[:2].contiguous()), Dev(k), Dev(s)), (Dev(k), Dev(s), Dev(k[:2].contiguous()), Dev(s)),
                           (Dev(k), Dev(s), Dev(k), Dev(torch.zeros((3, 2, 2, 16, 8), **u8))), (Dev(k.transpose(0, 1)), Dev(s), Dev(k), Dev(s)),
                           (Dev(k.transpose(3, 4)), Dev(s), Dev(k), Dev(s))):
        with pytest.raises(ValueError):
            B.td_set_prefix4(None, dims(), kk, ks, vv, vs, (0,), 1)
    with pytest.raises(ValueError):
        B.td_set_prefix4(None, dims(), Dev(k), Dev(s), Dev(k), Dev(s), (0.5,), 1)


def test_axes_are_checked_before_the_library():
    freq = Dev(torch.ones(16))
    for axis in ([0] * 15, [0] * 17, [0] * 15 + [4], [0] * 15 + [-1], [[0] * 16]):
        with pytest.raises(ValueError):
            B.RopeAxes(freq, axis)
    with pytest.raises(ValueError):
        B.RopeAxes(Dev(torch.ones(16, dtype=torch.float64)), [0] * 16)
    rope = B.RopeAxes(freq, [i % 3 for i in range(16)])
    i32 = dict(dtype=torch.int32)
    pos, shift = torch.zeros((2, 5, 3), **i32), torch.zeros((2, 3), **i32)
    c = rope.c((2, 5), 2, Dev(pos), None)
    assert (c.n_axes, c.d_pos, c.d_shift, c.rope.dim) == (3, 4096, None, 32)
    assert [c.h_axis[i] for i in range(16)] == [i % 3 for i in range(16)]
    c = rope.c((2, 5), 2, None, Dev(torch.zeros((2, 4), **i32)))
    assert (c.n_axes, c.d_pos, c.d_shift) == (4, None, 4096)
    assert rope.c((2, 5), 2, None, None).n_axes == 3
    for p, s in ((Dev(pos), Dev(shift)), (Dev(pos[:, :4].contiguous()), None), (Dev(pos[..., :2].contiguous()), None), (Dev(pos.long()), None),
                 (Dev(pos.transpose(1, 2)), None), (None, Dev(torch.zeros((5, 3), **i32))), (None, Dev(torch.zeros((2, 5), **i32))), (pos, None)):
        with pytest.raises(ValueError):
            rope.c((2, 5), 2, p, s)
    with pytest.raises(ValueError):
        B._rope_call(B.Rope(freq), (5,), 1, Dev(torch.zeros((5, 3), **i32)), None)
    with pytest.raises(ValueError):
        B._rope_call(None, (5,), 1, None, Dev(torch.zeros((1, 3), **i32)))
