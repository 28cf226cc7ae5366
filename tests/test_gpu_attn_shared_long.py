"""Attention over shared prefixes: a long prompt's own keys are cut as they are without sharing."""
import numpy as np
import pytest
import torch

from paper_2605_21603_amd import binding as B
from workloads import gen

import test_gpu_attn_shared as shared
from gpu_util import GpuRun
from test_gpu_attn_shared import Case, forward, shared_step

pytestmark = pytest.mark.gpu


def plain_rule(reach):
    ct = 1024
    while reach > 8 * ct and ct < 8192:
        ct *= 2
    return ct


def run_rule(reach, tg, n_kv, rows, mean):
    ct, cu, most = plain_rule(reach), n_kv * rows * mean // (256 * tg), 8192 if reach <= 8192 else 4096
    while ct < most and ct < reach and 4 * ct <= cu:
        ct *= 2
    return ct


def chunks_of_own_keys(att):
    """The chunk length of every row's own keys, from the plan that the call left in its workspace: partials (o, then m and l) of C chunks a token, then
    six arrays of a word per row - the sixth of them this - and the lists."""
    T, n_q, hd = att.out.shape
    up = lambda n: (n + 255) & ~255
    parts = lambda c: up(T * c * n_q * hd * 4) + up(T * c * n_q * 2 * 4)
    c = next(c for c in range(1, 500) if parts(c) + up((6 * T + 8 + 4 * c * T) * 4) == att.batch.workspace_bytes)
    at = att.batch.workspace - att.workspace.data_ptr() + parts(c)
    return att.workspace[at:at + 6 * T * 4].view(torch.int32).view(6, T)[5].cpu().numpy()


def test_prompts_of_more_and_of_fewer_rows(monkeypatch):
    monkeypatch.setitem(shared.SHAPES, "layer", (32, 8, 128, 16, torch.bfloat16))
    seqs = [(None, 0, 5000, 2600), ("a", 3, 4800, 2700), ("a", 3, 40, 1), (None, 0, 5000, 2560), (None, 0, 30, 1), ("a", 3, 600, 40)]
    c = Case("layer", seqs)
    got = c.run()
    ct, row = chunks_of_own_keys(c.att), 0
    for key, pages, own, new in seqs:
        p = np.arange(own - new, own)
        if new > 4:
            want = [run_rule((x // 64 + 1) * 64, 64, 8, new, own - new + (new + 1) // 2) if new > 2560 else plain_rule((x // 64 + 1) * 64) for x in p]
            assert np.array_equal(ct[row:row + new], want), (own, new)
            assert (max(want) > 1024) == (new > 2560)
        row += new
    keep = np.zeros(len(c.seq), bool)
    keep[::97] = keep[-45:] = keep[2598:2602] = True
    got[torch.from_numpy(~keep).to(got.device)] = 0
    c.pos[~keep] = -1
    c.check(got)


def test_a_long_prompt_in_the_layer_under_every_schedule():
    """2700 tokens beside decodes that share a page: the prompt's rows are one dispatch's or lie beside the others', the bits are the same."""
    w = gen.config("c3_mid")
    members = [s for s, (q, ctx) in enumerate(w.seqs) if q == 1 and ctx > 16]
    w, data, prefix = shared_step("c3_mid", {members[0]: (1, members)})
    run = GpuRun(w, data)
    want = forward(run, data, prefix, B.sequential())
    starts = [0] + [int(x) for x in np.cumsum([q for q, _ in w.seqs])]
    for sched in (B.nano_schedule(w.nano_rows, stagger=1), B.nano_schedule([0, starts[1], starts[6], starts[-1]]), B.sequential(use_graph=True)):
        for a, b in zip(forward(run, data, prefix, sched), want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
