"""What lies in front of a sequence's first slot, behind its last and in other sequences' parts of a page: the outputs
have the same bits whether it is finite or NaN.  (A row that has to be computed again, over its own slots alone, rounds
differently: none is.)"""
import math

import pytest
import torch

from paper_2609_03515_gb300 import ikv
from rows_ref import Cache
from test_gpu_prefix import Call
from test_gpu_window import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 24, 64, 128])
@pytest.mark.parametrize("group", [1, 4, 7])
@pytest.mark.parametrize("start", [0, 5, 40, 127])
def test_windows(d, page, group, start):
    """Prompts whose last unit has few queries, so that the unit in front of it ends a few slots before the sequence does;
    sequences that begin inside a page."""
    lens = [128 // group * 2 * 2 + 3, 128 // group * 2 + 1, 61, 130]
    outs = []
    for hidden in (9.0, math.nan):
        c = Cache(lens, 2, group, d, "bf16", page, seed=41, starts=[start, 0, start + 1, start]).device(hidden)
        outs.append([run(c, counts, window, sinks)[0]
                     for counts in (lens, [3, 66, 1, 40]) for window, sinks in ((0, 0), (50, 3), (20, 0))])
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("plen", [1, 100, 125, 128, 190])
@pytest.mark.parametrize("ahead", [0, 1, 5, 40])
@pytest.mark.parametrize("start", [0, 3])
def test_prefixes(d, page, plen, ahead, start):
    """The first member a few slots longer than the prefix (the first steps behind a fork), and members whose own pages
    hold nothing in the prefix's slots."""
    lens = [plen + ahead, plen + 70, plen + 3]
    outs = []
    for hidden in (9.0, math.nan):
        c = Cache(lens, 2, 4, d, "bf16", page, seed=42, starts=[start, start + 6, 0], share=[(0, [1, 2], plen)])
        for b in (1, 2):
            c.k[b][:, :, :plen] = hidden
            c.v[b][:, :, :plen] = hidden
        call = Call(c.device(hidden), [[0, 1, 2]], [plen])
        call.run()
        call.done()
        outs.append((call.out.cpu(), call.score.cpu()))
    assert bool(outs[0][0].isfinite().all())
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
