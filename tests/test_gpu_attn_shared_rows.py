"""Attention over shared prefixes: what one sequence holds is nothing to the others, under every schedule."""
import math

import numpy as np
import pytest
import torch

from paper_2605_21603_amd import binding as B
from workloads import gen

from gpu_util import GpuRun
from test_gpu_attn_shared import Case, forward, group, shared_step, SHAPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", ["fast", "fast_g3", "fast_p48", "bf16_64", "f32_64"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("poisoned", [0, 3, 6])
def test_other_sequences_keep_their_bits(shape, value, poisoned):
    """The last token of one sequence - a draft, a longer draft, a prompt - holds NaN or infinities: every row of the other sequences has the bits it
    had, whichever launch or dispatch they share, and the sequence's earlier rows are right."""
    ps = SHAPES[shape][3]
    c = Case(shape, group("a", 5, [4, 9, 33, 150], new=4) + [(None, 0, 20, 3), ("a", 5, 70, 70), (None, 0, 1100, 90), (None, 0, 65, 64, 2), (None, 0, 40, 1), ("a", 5, 3, 1)])
    want = c.run()
    rows = np.flatnonzero((c.seq == poisoned) & (c.pos >= 0))
    last = rows[-1]
    page, slot = c.table[poisoned, c.pos[last] // ps], c.pos[last] % ps
    c.v[page, :, 3::7, slot] = value
    c.k[page, :, slot, 2::5] = value
    got = c.run()
    others = torch.from_numpy(np.flatnonzero((c.seq != poisoned) | (c.pos < 0))).to(got.device)
    assert torch.equal(got[others], want[others])
    c.check(got, without={int(last)})
    again = c.run()
    assert torch.equal(again[others], got[others]) and torch.equal(again[rows[:-1]], got[rows[:-1]])
    if shape.startswith("fast"):
        assert torch.equal(got[rows[:-1]], want[rows[:-1]])


@pytest.mark.parametrize("shape", ["fast", "fast_g3", "fast_g1", "fast_g16", "fast_p48", "fast_p512", "bf16_p32"])
@pytest.mark.parametrize("sequence", [0, 1, 2, 3, 4])
def test_rows_from_a_bad_value_on_see_it_where_it_is(shape, sequence):
    """Values of tokens in the middle of a step - +inf, -inf, NaN, +inf and -inf at different ones - are in the rows that attend them, in their head-dim indices, which
    are not finite; everything else, of those rows and of the ones before, has the bits that it has with other values in their place."""
    ps = SHAPES[shape][3]
    seqs = group("a", 5, [9, 33], new=4) + [("a", 5, 70, 70), (None, 0, 1100, 90), (None, 0, 50, 3), ("a", 5, 20, 1), (None, 0, 40, 1)]
    c = Case(shape, seqs)
    new = seqs[sequence][3]
    rows = np.flatnonzero(c.seq == sequence)
    first, second = rows[new // 3], rows[new // 2]
    at = lambda t: (c.table[sequence, c.pos[t] // ps], c.pos[t] % ps)

    def place(values):
        for t, dim, value in values:
            page, slot = at(t)
            c.v[page, :, dim::16, slot] = value

    bad = [(first, 1, math.inf), (first, 2, -math.inf), (first, 3, math.nan), (first, 4, math.inf), (second, 4, -math.inf), (second, 5, math.inf)]
    place([(t, dim, 0.5) for t, dim, _ in bad])
    want = c.run().float()
    place(bad)
    got = c.run().float()
    for t in range(len(c.seq)):
        odd = [] if c.seq[t] != sequence or t < first else [1, 2, 3, 4] if t < second else [1, 2, 3, 4, 5]
        expect = want[t].clone()
        for dim in odd:
            expect[:, dim::16] = math.inf                    # (an infinity met by a merge's weight of zero is NaN)
        assert torch.equal(torch.isfinite(got[t]), torch.isfinite(expect)), (t, first, second)
        assert torch.equal(got[t][torch.isfinite(expect)], expect[torch.isfinite(expect)]), (t, first, second)


@pytest.mark.parametrize("name,prefixes,poisoned", [("stack_mixed", {0: (40, [0, 1, 5]), 6: (18, [6])}, [0]), ("stack_mixed", {0: (40, [0, 1, 5]), 6: (18, [6])}, [3, 6]),
                                                    ("c3_small", {1: (3, [1, 2, 3])}, [0]), ("c3_small", {1: (3, [1, 2, 3])}, [2]), ("f32_small", {1: (1, [1, 2, 3])}, [3])])
def test_one_bad_token_in_the_layer(name, prefixes, poisoned):
    """The last token of a sequence comes in with infinities, so its row and its cached keys and values are NaN.  All other rows are finite and the
    same bits under every schedule; those of other sequences are the ones of the step without it."""
    w = gen.config(name)
    prefixes = {f: (n, [s for s in members if w.seqs[s][1] - w.seqs[s][0] >= n * w.shape.page_size]) for f, (n, members) in prefixes.items()}
    w, data, prefix = shared_step(name, prefixes)
    clean = forward(GpuRun(w, data), data, prefix, B.sequential())[0]
    starts = np.concatenate([[0], np.cumsum([q for q, _ in w.seqs])])
    bad = [int(starts[s + 1]) - 1 for s in poisoned]
    x = data["x"].clone()
    x[bad] = math.inf
    data = dict(data, x=x)
    run = GpuRun(w, data)
    y = forward(run, data, prefix, B.sequential())[0]
    good = torch.tensor([t for t in range(len(y)) if t not in bad])
    others = torch.tensor([t for s in range(len(w.seqs)) if s not in poisoned for t in range(starts[s], starts[s + 1])])
    assert torch.isfinite(y[good].float()).all() and torch.isnan(y[bad].float()).all()
    assert torch.equal(y[others], clean[others])
    if w.shape.dtype == "bf16":
        assert torch.equal(y[good], clean[good])
    every_sequence = [int(t) for t in starts]
    for sched in (B.nano_schedule(w.nano_rows), B.nano_schedule(w.nano_rows, stagger=2), B.nano_schedule(every_sequence, stagger=1), B.nano_schedule(w.nano_rows, use_graph=True),
                  B.sequential(use_graph=True), B.nano_schedule(w.nano_rows, merged_ops=[B.DYN_OP_QKV], stagger=1)):
        for repeat in (1, 3):
            got = forward(run, data, prefix, sched, repeat=repeat)[0]
            assert torch.equal(got[good], y[good])
