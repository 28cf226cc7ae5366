"""Attention over shared prefixes on the GPU: against every row's own attention in 64 bits, and inside the layer."""
import dataclasses
import math

import numpy as np
import pytest
import torch

from paper_2605_21603_amd import binding as B
from workloads import gen

from gpu_util import GpuRun, check_against_oracle, say
from test_gpu_parity import cu_masks_halves

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# q heads, kv heads, head dim, page size, type: the fast forms with groups of 4, 3, 1 and 16 q heads, the general one on the matrix
# cores, and what runs without sharing
SHAPES = {
    "fast": (8, 2, 128, 16, torch.bfloat16), "fast_g3": (6, 2, 128, 16, torch.bfloat16), "fast_g1": (3, 3, 128, 16, torch.bfloat16),
    "fast_g16": (16, 1, 128, 16, torch.bfloat16),
    "fast_p48": (8, 2, 128, 48, torch.bfloat16), "fast_p512": (4, 2, 128, 512, torch.bfloat16),
    "bf16_64": (8, 2, 64, 16, torch.bfloat16), "bf16_p32": (8, 2, 128, 32, torch.bfloat16), "bf16_256": (4, 2, 256, 16, torch.bfloat16),
    "f32_64": (8, 2, 64, 16, torch.float32), "f32_32": (3, 1, 32, 48, torch.float32), "f32_128": (4, 4, 128, 16, torch.float32),
    "odd_page": (4, 2, 64, 5, torch.float32), "narrow": (4, 2, 8, 16, torch.bfloat16), "many_heads": (34, 2, 32, 16, torch.bfloat16),
}


class Case:
    """seqs: (prefix key or None, shared pages, keys of its own, new tokens, [rows of padding behind]) per sequence, in batch order.
    Everything that no row attends - other slots of a last page, unused pages - holds NaN or infinities."""

    def __init__(self, shape, seqs, seed=0, lead=None, pages=None, spare=3, width=0, pitch=0, scale=1.0):
        n_q, n_kv, hd, ps, dt = SHAPES[shape]
        self.dims = n_q, n_kv, hd, ps
        gen_ = torch.Generator(device=DEV).manual_seed(seed)
        rs = np.random.RandomState(seed)
        prefixes, n_pages, table = {}, 0, []
        first = {}
        for s, (key, shared, own, new, *_) in enumerate(seqs):
            row = []
            if key is not None:
                have = prefixes.setdefault(key, [])
                while len(have) < shared:
                    have.append(n_pages)
                    n_pages += 1
                row = have[:shared]
                first.setdefault((key, shared), s)
            n = -(-own // ps)
            table.append(row + list(range(n_pages, n_pages + n)))
            n_pages += n
        n_pages += spare
        perm = rs.permutation(n_pages)
        width = max(width, max(len(r) for r in table))
        self.table = np.full((len(seqs), width), int(perm[-1]), np.int32)
        for s, r in enumerate(table):
            self.table[s, :len(r)] = perm[r]
        self.ctx = np.array([(sh if key is not None else 0) * ps + own for key, sh, own, *_ in seqs])
        seq, pos = [], []
        for s, (key, sh, own, new, *pad) in enumerate(seqs):
            seq += [s] * new
            pos += list(range(self.ctx[s] - new, self.ctx[s]))
            if pad:
                seq += [int(rs.randint(len(seqs)))] * pad[0]
                pos += [-1] * pad[0]
        self.seq, self.pos = np.array(seq, np.int32), np.array(pos, np.int32)
        if lead is None:
            lead = [first[(key, sh)] if key is not None else s for s, (key, sh, *_) in enumerate(seqs)]
            pages = [sh if key is not None else 0 for key, sh, *_ in seqs]
        T = len(seq)
        k = torch.full((n_pages, n_kv, ps, hd), math.nan, device=DEV, dtype=dt)
        v = torch.full((n_pages, n_kv, hd, ps), math.inf, device=DEV, dtype=dt)
        live = np.zeros((n_pages, ps), bool)
        for s in range(len(seqs)):
            for j in range(-(-int(self.ctx[s]) // ps)):
                live[self.table[s, j], :min(ps, self.ctx[s] - j * ps)] = True
        mask = torch.from_numpy(live).to(DEV)
        kr = torch.randn(k.shape, generator=gen_, device=DEV) * scale
        vr = torch.randn(v.shape, generator=gen_, device=DEV)
        k = torch.where(mask[:, None, :, None], kr.to(dt), k)
        v = torch.where(mask[:, None, None, :], vr.to(dt), v)
        pitch = pitch or n_q * hd
        self.q = torch.randn((T, pitch), generator=gen_, device=DEV).to(dt)[:, :n_q * hd].view(T, n_q, hd)
        self.out = torch.full((T + 2, pitch), 7.0, device=DEV, dtype=dt)
        self.k, self.v = k, v
        to = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
        self.args = dict(seq_of_token=to(self.seq), pos_of_token=to(self.pos), block_table=to(self.table), prefix_lead=to(lead), prefix_pages=to(pages))
        self.att = None

    def attention(self, **change):
        n_q, n_kv, hd, ps = self.dims
        T = len(self.seq)
        return B.SharedAttention(self.q, self.out[:T, :n_q * hd].view(T, n_q, hd), self.k, self.v, **dict(self.args, **change))

    def run(self, **change):
        self.att = self.attention(**change)
        self.att.workspace.fill_(0xFF)                # nothing in it may matter
        self.att.forward()
        torch.cuda.synchronize()
        T = len(self.seq)
        assert (self.out[T:] == 7).all() and (self.out[:, self.q.shape[1] * self.q.shape[2]:] == 7).all()      # rows and columns that are not the call's
        return self.att.out.clone()

    def check(self, got, without=()):
        """|got - exact| of every element within what the roundings on the way allow.

        bf16: a probability is rounded to bf16 (half a step, 2^-8 of it) before it meets its value and in the sum that divides, so
        each element is off by at most 2 * 2^-8 * A with A = sum p |v| / sum p, and the result by 2^-8 of itself.  In 32 bits: a
        score of d products and its scaling by (d + 8) 2^-24 of the sum S of their magnitudes, which moves a probability by twice that (numerator
        and sum), sums over n keys by n 2^-24 each, exponentials and merge factors by a few 2^-23."""
        n_q, n_kv, hd, ps = self.dims
        G, worst = n_q // n_kv, 0.0
        low = got.dtype == torch.bfloat16
        kept = [t for t in range(len(self.seq)) if t not in without]
        assert torch.isfinite(got[kept].float()).all()
        for t in kept:
            if self.pos[t] < 0:
                assert (got[t] == 0).all()
                continue
            s, n = self.seq[t], int(self.pos[t]) + 1
            pages = torch.from_numpy(self.table[s, :-(-n // ps)]).long().to(DEV)
            K = self.k[pages].double().transpose(0, 1).reshape(n_kv, -1, hd)[:, :n]
            V = self.v[pages].double().permute(1, 0, 3, 2).reshape(n_kv, -1, hd)[:, :n]
            q = self.q[t].double().view(n_kv, G, hd)
            scores = (q[:, :, None, :] * K[:, None]).sum(-1) / math.sqrt(hd)
            S = (q[:, :, None, :].abs() * K[:, None].abs()).sum(-1).amax(-1, keepdim=True) / math.sqrt(hd)
            p = torch.softmax(scores, -1)
            want = (p[..., None] * V[:, None]).sum(2)
            A = (p[..., None] * V[:, None].abs()).sum(2)
            bound = A * (4 * (hd + 8) * S + 2 * n + 64) * 2.0 ** -24
            if low:
                bound = bound + 2.0 ** -8 * (want.abs() + 2 * A)
            err = (got[t].double().view(n_kv, G, hd) - want).abs()
            assert (err <= bound * 1.001 + 1e-30).all(), (t, (err / bound).max().item())
            worst = max(worst, (err / bound).max().item())
        return worst


def group(key, shared, owns, new=1):
    return [(key, shared, own, min(own, new)) for own in owns]


@pytest.mark.parametrize("shape", list(SHAPES))
def test_groups_of_every_size_beside_sequences_alone(shape):
    """Groups of 2 to 70 sequences, a run that is cut by others, one lead with two page counts, padding between and behind."""
    rs = np.random.RandomState(5)
    own = lambda n, hi=80: rs.randint(1, hi, n).tolist()
    seqs = (group("a", 5, own(2)) + [(None, 0, 33, 1, 2)] + group("b", 17, own(9)) + group("a", 5, own(3)) + group("c", 1, own(70)) + group("b", 16, own(4)) +
            [(None, 0, 1, 1), (None, 0, 100, 1)] + group("d", 9, own(8) + [1, 16, 17]) + [("e", 4, 7, 1, 5)])
    c = Case(shape, seqs)
    say("%s: worst share of the bound %.2f" % (shape, c.check(c.run())))


@pytest.mark.parametrize("shape", ["fast", "fast_g3", "fast_p48", "bf16_p32", "bf16_64", "f32_64", "odd_page"])
def test_several_tokens_a_sequence(shape):
    """Drafts of a few tokens, prompts of many, behind a shared prefix, beside decodes of the same group."""
    seqs = (group("a", 9, [5, 1, 90, 200, 3, 64]) + group("a", 9, [30, 150, 4], new=3) + [("a", 9, 170, 150), ("a", 9, 40, 40)] + group("b", 3, [25] * 12, new=5) +
            [(None, 0, 70, 70), (None, 0, 9, 2, 1)])
    c = Case(shape, seqs)
    c.check(c.run())


@pytest.mark.parametrize("shape", ["fast", "fast_g3", "fast_g1", "fast_g16", "fast_p48", "bf16_64", "f32_64"])
@pytest.mark.parametrize("new", [2, 3, 4, 5, 17])
def test_drafts_behind_long_keys_of_their_own(shape, new):
    """Few tokens a sequence: their own keys end inside a tile, a chunk or a page, each token's one further."""
    owns = [new, new + 1, 15 + new, 16, 64, 64 + new, 65, 129, 500 + new, 1024, 1030]
    c = Case(shape, group("a", 6, [max(o, new) for o in owns], new=new) + [(None, 0, 900, new, 1), (None, 0, new, new), ("a", 6, 800, 1)])
    c.check(c.run())


@pytest.mark.parametrize("shape", ["fast", "fast_g3", "bf16_64", "f32_64", "odd_page"])
def test_positions_that_repeat_or_skip(shape):
    """Rows of one sequence that do not follow one another each attend the keys up to their own position; the last page of the
    table's last row is full, so one key more would be read past it."""
    ps = SHAPES[shape][3]
    own = 6 * ps
    c = Case(shape, group("a", 4, [own, own, own], new=6) + [(None, 0, own, 3), ("a", 4, own, 30)], spare=0)
    at = 0
    for s, pos in enumerate([[-1, -1, -1, -1, -1, -1], [-6, -4, -4, -4, -2, -1], [-9, -8, -3, -3, -2, -2], [-7, -7, -1], [-30 + i // 2 for i in range(30)]]):
        c.pos[at:at + len(pos)] = c.ctx[s] + np.array(pos)
        at += len(pos)
    c.args["pos_of_token"].copy_(torch.from_numpy(c.pos))
    c.check(c.run())


@pytest.mark.parametrize("shape", ["fast", "fast_g3", "fast_g16", "fast_p48", "bf16_64", "f32_64", "odd_page"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_what_later_tokens_hold_does_not_reach_earlier_ones(shape, value):
    """Keys and values of a sequence's last tokens are NaN or infinite: the rows before them are as they were."""
    ps = SHAPES[shape][3]
    seqs = group("a", 5, [4, 9, 33, 150], new=4) + [(None, 0, 20, 3), ("a", 5, 70, 70), (None, 0, 1100, 90), (None, 0, 65, 64, 2), (None, 0, 40, 1)]
    c = Case(shape, seqs)
    poisoned = set()
    for s, (*_, last) in enumerate([[1], [2], [3], [1], [1], [30], [60], [3], [0]]):
        rows = [t for t in range(len(c.seq)) if c.seq[t] == s and c.pos[t] >= 0]
        for t in rows[len(rows) - last:]:
            poisoned.add(t)
            page, slot = c.table[s, c.pos[t] // ps], c.pos[t] % ps
            c.v[page, :, t % 7::7, slot] = value
            c.k[page, :, slot, t % 5::5] = -value
    c.check(c.run(), without=poisoned)


@pytest.mark.parametrize("shape,keys", [("fast", 4096), ("fast", 4097), ("fast", 4159), ("fast", 8255), ("fast_p48", 4100), ("bf16_64", 8193), ("f32_64", 8200)])
@pytest.mark.parametrize("new", [1, 3])
def test_lengths_just_past_what_the_most_chunks_hold(shape, keys, new):
    """As many chunks as a token has partials for: neither the rows around it nor what lies behind the partials is written."""
    c = Case(shape, [(None, 0, 9, 1), (None, 0, keys, new), (None, 0, 17, 1), (None, 0, keys, new)])
    c.check(c.run())


@pytest.mark.parametrize("shape,shared", [("fast", 256), ("fast", 257), ("fast", 4097), ("fast_p48", 86), ("bf16_64", 257)])
@pytest.mark.parametrize("n", [3, 90])
def test_prefixes_just_past_what_the_most_chunks_hold(shape, shared, n):
    if n > 3 and shared > 1000:
        n = 20
    c = Case(shape, group("a", shared, [3] * n) + [(None, 0, 5, 1)])
    c.check(c.run())


@pytest.mark.parametrize("shape,shared", [("fast", 300), ("fast", 531), ("fast_p48", 111), ("bf16_64", 150), ("f32_64", 70)])
@pytest.mark.parametrize("n", [2, 7, 9, 40])
def test_long_prefixes(shape, shared, n):
    """Prefixes of many chunks, odd page counts, few and many sharers."""
    c = Case(shape, group("a", shared, list(range(1, n + 1))) + [(None, 0, 700, 1)])
    c.check(c.run())


@pytest.mark.parametrize("shape", ["fast", "bf16_64", "f32_64"])
def test_what_is_no_prefix_is_not_shared(shape):
    """Leads and page counts outside the table, a whole row, tokens that stand inside the shared pages, leads nobody else names: the
    rows' own attention all the same."""
    ps = SHAPES[shape][3]
    seqs = group("a", 6, [20, 1, 30, 7, 9, 11, 5, 8])
    for lead, pages in (([-1] * 8, [6] * 8), ([8] * 8, [6] * 8), ([1 << 30] * 8, [6] * 8), ([0] * 8, [-3] * 8), ([0] * 8, [1 << 30] * 8), ([0] * 8, [8] * 8), (list(range(8)), [6] * 8),
                        ([0] * 8, [0] * 8), ([0, 0, 1, 1, 7, 7, 7, -5], [6, 5, 6, 6, 1, 2, 3, 4])):
        c = Case(shape, seqs, lead=lead, pages=pages)
        c.check(c.run())
    # a step whose tokens begin inside the shared pages: those rows attend alone, the ones behind them share
    seqs = [("a", 6, 20, 20 + 2 * ps), ("a", 6, 9, 1), ("a", 6, 3, 1), ("a", 6, 3, 3 + ps)]
    c = Case(shape, seqs)
    c.check(c.run())


def test_without_prefixes_and_rows_of_padding_alone():
    c = Case("fast", [(None, 0, 40, 1), (None, 0, 300, 7, 4), (None, 0, 1, 1)])
    c.check(c.run(prefix_lead=None, prefix_pages=None))
    c.args["pos_of_token"].fill_(-1)
    c.pos[:] = -1
    c.check(c.run())
    one = Case("fast", [(None, 0, 1, 1)])
    one.check(one.run())


@pytest.mark.parametrize("shape", ["fast", "f32_64", "bf16_64"])
def test_rows_of_a_wider_pitch_a_wider_table_and_large_scores(shape):
    n_q, n_kv, hd, ps, _ = SHAPES[shape]
    c = Case(shape, group("a", 12, [5, 40, 3, 17, 1, 9, 100, 2, 8, 31]) + [(None, 0, 50, 1)], width=700, pitch=(n_q + 2 * n_kv) * hd, scale=8.0)
    c.check(c.run())


@pytest.mark.parametrize("chunk", [64, 1024])
def test_chunk_sizes(chunk):
    c = Case("fast", group("a", 40, [5, 400, 3, 700, 1]) + group("b", 30, [70] * 12) + [(None, 0, 1500, 1)])
    c.check(c.run(kv_chunk_positions=chunk))


def test_the_same_batch_gives_the_same_bits():
    """Whatever the workspace held, and however the launches' workgroups come to their work."""
    for shape in ("fast", "bf16_64", "f32_64"):
        seqs = group("a", 20, [3, 50, 17, 90, 4, 33, 61, 2, 9, 12, 14]) + group("b", 7, [10, 20, 30]) + [("b", 7, 90, 70)]
        c = Case(shape, seqs)
        first = c.run()
        for _ in range(5):
            assert torch.equal(c.run(), first), shape


def test_more_sequences_than_are_counted_attend_without_sharing():
    """4097 sequences: every row over its own table row; 4096: shared."""
    for n in (4096, 4097):
        c = Case("f32_32", group("a", 1, [1] * 40) + [(None, 0, 1, 1)])
        table = np.zeros((n, c.table.shape[1]), np.int32)
        table[:41] = c.table
        lead, pages = np.full(n, -1), np.zeros(n)
        lead[:40], pages[:40] = 0, 1
        to = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
        c.check(c.run(block_table=to(table), prefix_lead=to(lead), prefix_pages=to(pages)))


def test_more_rows_than_the_plan_looks_at_in_one_round():
    """1500 decodes in groups across the rounds' borders, and a prompt of 2700 tokens behind a shared prefix (its lists are built by another
    search); every 37th row is compared."""
    rs = np.random.RandomState(0)
    for shape, seqs in (("fast", group("a", 3, rs.randint(1, 30, 1000).tolist()) + group("b", 2, rs.randint(1, 30, 70).tolist()) + group("c", 4, rs.randint(1, 30, 430).tolist())),
                        ("fast", group("a", 8, [4, 5, 6]) + [("a", 8, 2700, 2700)] + group("a", 8, [7, 8])),
                        ("f32_32", group("a", 1, rs.randint(1, 30, 1030).tolist()) + group("b", 2, rs.randint(1, 30, 70).tolist()))):
        c = Case(shape, seqs)
        got = c.run()
        keep = np.zeros(len(c.seq), bool)
        keep[::37] = keep[1000:1100] = keep[-6:] = True
        got[torch.from_numpy(~keep).to(DEV)] = 0
        c.pos[~keep] = -1
        c.check(got)


@pytest.mark.parametrize("rows", [255, 256, 257, 1023, 1024, 1025])
def test_rows_around_the_plans_rounds(rows):
    """As many rows as one round of the plan holds, one fewer and one more; a draft and a query block lie across the border."""
    head = group("a", 2, [3] * (rows - 40)) + [("a", 2, 37, 37)]
    c = Case("fast", head + [("b", 1, 9, 3), ("b", 1, 5, 1)] if rows > 1000 else head + group("b", 1, [9, 5, 7]))
    got = c.run()
    keep = np.zeros(len(c.seq), bool)
    keep[::29] = keep[-50:] = True
    got[torch.from_numpy(~keep).to(DEV)] = 0
    c.pos[~keep] = -1
    c.check(got)


@pytest.mark.parametrize("shape", ["fast", "fast_p48", "bf16_64", "f32_32", "odd_page"])
def test_rows_outside_the_table_attend_nothing(shape):
    """Sequences that are none and positions past the table's width, between rows that are read as ever."""
    c = Case(shape, group("a", 3, [5, 40, 7]) + group("a", 3, [30, 20], new=9) + [(None, 0, 50, 20), ("a", 3, 4, 1)])
    n, most = len(c.ctx), c.table.shape[1] * SHAPES[shape][3]
    for t, (seq, pos) in {1: (n, 3), 4: (-1, 0), 8: (0, most), 15: (2 ** 31 - 1, 9), 16: (1, 2 ** 31 - 1), 25: (-2 ** 31, 5), 40: (n, most), 41: (3, -7)}.items():
        c.args["seq_of_token"][t], c.args["pos_of_token"][t], c.pos[t] = seq, pos, -1
    c.check(c.run())


@pytest.mark.parametrize("n_seqs", [1024, 1025])
def test_few_rows_of_many_sequences(n_seqs):
    """The plan of few rows counts up to 1024 sequences' leads; a batch may have many more sequences than rows."""
    c = Case("fast", group("a", 3, [5, 40, 7]) + group("b", 1, [1, 2]) + [(None, 0, 1, 0)] * (n_seqs - 5))
    c.check(c.run())


@pytest.mark.parametrize("shape", ["bf16_256", "f32_128", "bf16_64", "narrow", "fast"])
@pytest.mark.parametrize("copies", [1, 60])
def test_merges_by_a_half_wave_and_by_a_workgroup(shape, copies):
    """Few rows and many, one chunk a row to as many as there are."""
    c = Case(shape, group("a", 24, [1, 700, 30] * copies) + [(None, 0, 3, 1), (None, 0, 3000, 1)])
    got = c.run()
    keep = np.zeros(len(c.seq), bool)
    keep[::17] = keep[-3:] = True
    got[torch.from_numpy(~keep).to(DEV)] = 0
    c.pos[~keep] = -1
    c.check(got)


@pytest.mark.parametrize("shape", ["fast", "fast_p48", "bf16_64", "f32_32"])
def test_offsets_beyond_32_bits(shape):
    """A pool whose last pages lie beyond 2^32 bytes and 2^31 elements: the same bits as with these pages at the front."""
    c = Case(shape, group("a", 7, [5, 300, 33]) + group("a", 7, [90, 20], new=15) + [(None, 0, 100, 1)])
    want = c.run()
    used = c.k.shape[0]
    n = (1 << 31) // c.k[0].numel() + used + 7
    for name in ("k", "v"):
        small = getattr(c, name)
        big = torch.zeros((n,) + small.shape[1:], device=DEV, dtype=small.dtype)
        big[n - used:] = small
        setattr(c, name, big)
    c.args["block_table"] += n - used
    assert torch.equal(c.run(), want)


def test_captured_call_follows_the_arrays_and_two_graphs_share_a_workspace():
    a, b = Case("fast", group("a", 20, [3, 50, 17, 90, 4, 33, 61, 2, 9, 12, 14])), Case("fast", group("a", 9, [30, 5, 7]) + [(None, 0, 90, 1)], seed=1)
    atts = [c.attention() for c in (a, b)]
    big = max(atts, key=lambda x: x.workspace.numel()).workspace
    atts = [c.attention(workspace=big) for c in (a, b)]
    for att in atts:
        att.forward()
    torch.cuda.synchronize()
    graphs = []
    for att in atts:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            att.forward()
        graphs.append(g)
    lead, pages = a.args["prefix_lead"], a.args["prefix_pages"]
    for step in range(4):
        a.pos -= 1 if step else 0                                   # every row one key less; those left without stand inside the prefix
        a.args["pos_of_token"].copy_(torch.from_numpy(a.pos).to(DEV))
        pages.fill_([20, 20, 7, 0][step])
        big.fill_(0xFF)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        a.check(atts[0].out)
        b.check(atts[1].out)
        want = atts[0].out.clone()
        atts[0].forward()
        assert torch.equal(want, atts[0].out)


def test_on_a_stream_of_its_own():
    c = Case("fast", group("a", 20, [3, 50, 17, 90, 4, 33, 61, 2, 9, 12, 14]))
    att, s = c.attention(), torch.cuda.Stream()
    torch.cuda.synchronize()
    att.forward(s)
    s.synchronize()
    c.check(att.out)


# ---------------------------------------------------------------------------------- inside the layer

def shared_step(name, prefixes, seed=None):
    """A generated step whose sequences share prefixes: {first sequence: (pages, members)}; the block table's rows begin alike."""
    w = gen.config(name)
    data = gen.generate(w)
    lead, pages = np.arange(w.n_seqs), np.zeros(w.n_seqs, np.int64)
    table = data["block_table"].copy()
    for first, (n, members) in prefixes.items():
        for s in members:
            q, ctx = w.seqs[s]
            assert ctx - q >= n * w.shape.page_size
            lead[s], pages[s] = first, n
            table[s, :n] = table[first, :n]
    data["block_table"] = table
    return w, data, (lead, pages)


def forward(run, data, prefix, sched, repeat=1, noalloc=False, exact=False):
    step = B.DeviceStep(run.layer, data, prefix=prefix, sched=sched if exact else None)
    step.workspace.fill_(0xFF)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(repeat):
        if noalloc:
            run.layer.forward_noalloc(step.batch, st)
        else:
            run.layer.forward(step.batch, sched, st)
    st.synchronize()
    return step.y.cpu(), step.k_cache.cpu(), step.v_cache.cpu()


LAYERS = [
    ("c2_small", {0: (6, [0, 1, 5, 6, 7]), 2: (13, [2, 3, 9, 10, 12][:2] + [10])}),
    ("c2_small", {0: (1, [0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12])}),
    ("c5_small", {0: (7, [0, 1, 2, 3, 4, 5, 6, 8, 9, 10]), 12: (5, list(range(12, 24)))}),
    ("c4_small", {0: (1, [i for i in range(40) if i not in (8, 18)])}),
    ("stack_mixed", {0: (40, [0, 1, 5]), 6: (18, [6])}),
    ("c3_small", {1: (3, [1, 2, 3])}),
    ("f32_small", {1: (1, [1, 2, 3])}),
]


@pytest.mark.parametrize("name,prefixes", LAYERS)
def test_layer_with_shared_prefixes(name, prefixes):
    """Against the oracle, which knows nothing of sharing; every schedule the same bits; graph, exact workspace, static workspace."""
    prefixes = {f: (n, [s for s in members if gen.config(name).seqs[s][1] - gen.config(name).seqs[s][0] >= n * gen.config(name).shape.page_size]) for f, (n, members) in prefixes.items()}
    w, data, prefix = shared_step(name, prefixes)
    run = GpuRun(w, data)
    chain = B.MOE_CHAIN if w.shape.n_experts else B.DENSE_CHAIN
    y, k, v = forward(run, data, prefix, B.sequential())
    if w.shape.n_layers == 1:
        say("%s: max rel err vs oracle %.3e" % (name, check_against_oracle(w, data, y, k, v)))
    plain, kp, vp = forward(run, data, None, B.sequential())
    # without the promise the first layer's caches are the same bits (they are written before any attention), and the output agrees: per
    # layer both are within the layer's bound of the exact one
    assert torch.equal(k[0].view(torch.uint8), kp[0].view(torch.uint8)) and torch.equal(v[0].view(torch.uint8), vp[0].view(torch.uint8))
    tol = (2e-2 if w.shape.dtype == "bf16" else 1e-4) * 2 * w.shape.n_layers
    rel = ((y - plain).abs().amax(1) / plain.abs().amax(1)).max().item()
    assert rel <= tol or w.shape.n_experts, rel
    scheds = [B.nano_schedule(w.nano_rows, chain), B.nano_schedule(w.nano_rows, chain, stagger=2),
              B.nano_schedule(w.nano_rows, chain, merged_ops=[B.DYN_OP_QKV, B.DYN_OP_OPROJ], stagger=1),
              B.nano_schedule(w.nano_rows, chain, use_graph=True), B.sequential(use_graph=True)]
    for i, sched in enumerate(scheds):
        for exact in (False, True):
            got = forward(run, data, prefix, sched, repeat=3 if sched.use_graph else 1, exact=exact)
            for a, b in zip(got, (y, k, v)):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (i, exact)
    got = forward(run, data, prefix, B.sequential(), noalloc=True)
    for a, b in zip(got, (y, k, v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("name,prefixes", [LAYERS[0], LAYERS[2], LAYERS[6]])
def test_layer_with_shared_prefixes_on_partitions(name, prefixes):
    """Micro-batches, or all attention, on half of the CUs: the same bits."""
    prefixes = {f: (n, [s for s in members if gen.config(name).seqs[s][1] - gen.config(name).seqs[s][0] >= n * gen.config(name).shape.page_size]) for f, (n, members) in prefixes.items()}
    w, data, prefix = shared_step(name, prefixes)
    run = GpuRun(w, data)
    want = forward(run, data, prefix, B.sequential())
    k = len(w.nano_rows) - 1
    for sched in (B.nano_schedule(w.nano_rows, stagger=1, partitions=[1 + i % 2 for i in range(k)], cu_masks=cu_masks_halves()),
                  B.nano_schedule(w.nano_rows, stagger=2, partitions=[2] * k, op_partitions={B.DYN_OP_ATTN: 1}, cu_masks=cu_masks_halves())):
        for a, b in zip(forward(run, data, prefix, sched), want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_graphs_with_and_without_prefixes_are_not_taken_for_one_another():
    w, data, prefix = shared_step("c2_small", {0: (6, [0, 1, 5, 6, 7][:2])})
    run = GpuRun(w, data)
    step = B.DeviceStep(run.layer, data, prefix=prefix)
    st, sched = torch.cuda.Stream(), B.sequential(use_graph=True)
    out = []
    for with_prefix in (True, False, True, False):
        step.batch.prefix_lead = step.prefix_lead.data_ptr() if with_prefix else None
        step.batch.prefix_pages = step.prefix_pages.data_ptr() if with_prefix else None
        step.y.zero_()
        torch.cuda.synchronize()
        run.layer.forward(step.batch, sched, st)
        st.synchronize()
        out.append(step.y.cpu())
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    want = [forward(run, data, p, B.sequential())[0] for p in (prefix, None)]
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_a_prompt_is_forked_and_decoded_and_the_pool_compacted():
    """The calls together, as a program makes them: a prompt is read by the layer, forked into answers that share its pages, each answer
    takes a few steps through the layer with the shared pages read once, ends, and the pool is compacted; every step against the same step
    without sharing, on pools of the same contents."""
    w = gen.config("c2_small")
    data = gen.generate(w)
    run = GpuRun(w, data)
    sh = w.shape
    ps, n_pages, rows, width = sh.page_size, 120, 12, 12
    torch.manual_seed(0)
    k = torch.randn((1, n_pages, sh.n_kv, ps, sh.head_dim)).to(torch.bfloat16).to(DEV)
    v = torch.randn((1, n_pages, sh.n_kv, sh.head_dim, ps)).to(torch.bfloat16).to(DEV)
    ints = lambda a: torch.tensor(list(a), dtype=torch.int32, device=DEV)
    table, lens, ref = torch.zeros((rows, width), dtype=torch.int32, device=DEV), ints([0] * rows), ints([0] * n_pages)
    pool = B.PagePool(k, v, table, lens, ref, rows)

    def step(active, new, prefix):
        """`new` tokens of each row in `active`, which already has room for them."""
        ctx = lens.cpu().numpy()
        d = dict(x=x[:len(active) * new], k_cache=k, v_cache=v, block_table=table[active].cpu().numpy(),
                 seq_of_token=np.repeat(np.arange(len(active), dtype=np.int32), new),
                 pos_of_token=np.concatenate([np.arange(ctx[r] - new, ctx[r], dtype=np.int32) for r in active]),
                 q_start=np.arange(len(active) + 1, dtype=np.int32) * new)
        s = B.DeviceStep(run.layer, d, prefix=prefix)
        run.layer.forward(s.batch, B.sequential(), torch.cuda.current_stream())
        torch.cuda.synchronize()
        return s.y.clone()

    prompt = 3 * ps + 5
    pool.resize(ints([4]), ints([2 * ps]))                      # some other sequence
    assert pool.resize(ints([0]), ints([prompt])).tolist() == [0]
    x = torch.randn((prompt, sh.hidden), device=DEV).to(torch.bfloat16)
    step([0], prompt, None)
    kids = [1, 2, 3, 5, 6, 7, 8]
    assert pool.fork(ints([0] * 7), ints(kids)).tolist() == [0] * 7
    for i in range(4):
        x = torch.randn((8, sh.hidden), device=DEV).to(torch.bfloat16)
        active = [0] + kids
        assert pool.resize(ints(active), ints([prompt + i + 1] * 8)).tolist() == [0] * 8
        before = k.clone(), v.clone()
        plain = step(active, 1, None)
        after = k.clone(), v.clone()
        k.copy_(before[0])
        v.copy_(before[1])
        y = step(active, 1, ([0] * 8, [3] * 8))
        assert torch.equal(k, after[0]) and torch.equal(v, after[1])
        # each is within 2e-2 of the exact row
        assert ((y.float() - plain.float()).abs().amax(1) <= 4e-2 * plain.float().abs().amax(1)).all()
    assert pool.resize(ints([4, 0, 1, 2]), ints([0, 0, 0, 0])).tolist() == [0] * 4
    y = step(kids[3:], 1, ([0] * 4, [3] * 4))
    new_page, n_live = pool.compact()
    assert n_live.item() == 3 + 5 and (ref[:8] > 0).all() and (ref[8:] == 0).all()
    assert torch.equal(step(kids[3:], 1, ([0] * 4, [3] * 4)), y)
