"""A captured decode step over a prefix in 4 bits.  A captured call's launch goes by the tries' capacity, the same
call's outside a graph by the nodes that they have: both are checked against 64 bits, and each replay gives what the
first gave.  The second capacity of a case has other splits, the third a launch of the tries' own."""
import pytest
import torch

from gpu_harness import log
from prefix_ref import check
from test_gpu_prefix4_attn import Batch
from test_gpu_prefix_attn import randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,Hq,Hkv,b,tries,S,window,caps", [
    (128, 32, 8, 8, [(200, 5), (90, 3), (140, 4), (7, 2)], 4096, 0, (500, 1400, 6000)),
    (128, 32, 8, 8, [(200, 5), (90, 3), (140, 4), (7, 2)], 4500, 3000, (500, 1400, 6000)),
    (96, 32, 32, 4, [(150, 6), (31, 2)], 1000, 0, (300, 900, 5000)),
    (64, 8, 2, 16, [(64, 3), (30, 1), (5, 2)], 900, 400, (200, 900, 5000)),
    (64, 4, 1, 3, [(9, 2)], 65, 40, (40, 700, 5000))])
def test_captured_step(D, Hq, Hkv, b, tries, S, window, caps):
    for cap in caps:
        log(f"captured d={D} {Hq}/{Hkv} b={b} S={S} W={window} cap={cap}")
        bt = Batch("bf16", D, Hq, Hkv, S, 32, tries, b, window=window, cap=cap)
        q, eager = bt.decode(sample=0.1)
        out = torch.full_like(q, 5.0)
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            bt.dec.attn_decode(0, 1, q, None, None, out, bt.scale)
        first = None
        for _ in range(3):
            out.fill_(5.0)
            graph.replay()
            torch.cuda.synchronize()
            if first is None:
                first = out.clone()
            assert torch.equal(out, first)
            again = torch.full_like(q, 5.0)  # (eager work between the replays)
            bt.dec.attn_decode(0, 1, q, None, None, again, bt.scale)
            torch.cuda.synchronize()
            assert torch.equal(again, eager)
        for t, s in enumerate(bt.tries):
            for j in range(b):
                if j >= s["n_live"]:
                    assert bool((first[0, t, j] == 0).all())
                elif bt.rng.random() < 0.25:
                    want, tol = bt.expect(q[0, t, j], 0, t, int(s["leaf_slot"][j]))
                    check(first[0, t, j][None], want, tol, (cap, t, j))
        # new queries through the same graph
        q.copy_(randn(bt.gen, tuple(q.shape), q.dtype))
        graph.replay()
        torch.cuda.synchronize()
        t, j = len(bt.tries) - 1, 0
        want, tol = bt.expect(q[0, t, j], 0, t, int(bt.tries[t]["leaf_slot"][j]))
        check(out[0, t, j][None], want, tol, "new queries")
        assert bt.dec.status() == 0
        bt.dec.close()
