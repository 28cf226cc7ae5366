"""The plain forms of the timed calls (perf/operators.py), on the CPU: the pages' ones leave what a program that cares for one page after another
leaves, bit for bit, whatever lies in the tables behind a row's pages."""
import random

import numpy as np
import pytest
import torch

from pages_model import Model
from perf import operators as O


@pytest.fixture(autouse=True)
def small_heads(monkeypatch):
    monkeypatch.setattr(O, "SHAPES", {"8b": dict(dtype="bf16", n_q=2, n_kv=1, head_dim=8), "hd64": dict(dtype="bf16", n_q=2, n_kv=1, head_dim=8),
                                      "f32": dict(dtype="f32", n_q=2, n_kv=1, head_dim=8)})


def compare(c, seed):
    got = O.run(dict(case=c, **O._pool_inputs(c, seed, "cpu")))
    want = O._exact_pages(c, O._pool_inputs(c, seed, "cpu"))
    assert set(got) == set(want)
    for name, w in want.items():
        assert torch.equal(got[name].double(), w), (c, seed, name)


@pytest.mark.parametrize("case", [c for c in O.listed() if c["op"] != "attention"], ids=lambda c: c["name"])
@pytest.mark.parametrize("seed", range(6))
def test_listed_calls(case, seed):
    compare(dict(case, layers=min(case["layers"], 2)), seed)


@pytest.mark.parametrize("seed", range(40))
def test_forks_whose_parents_end_with_a_page(seed):
    """Among 64 parents of 100 to 1024 positions five fill their last page: there is no part of one to copy."""
    compare(O._fork("f32", layers=1, parents=64, children=4, len_lo=100, len_hi=1024, draft=9), seed)
    compare(O._fork("f32", layers=1, parents=3, children=5, len_lo=32, len_hi=32, draft=20), seed)


def test_drawn_calls():
    rng, seen = random.Random(3), 0
    while seen < 25:
        c = O.draw(rng)
        if c["op"] != "attention" and c.get("pages", 0) * c["layers"] <= 40000:
            compare(dict(c, layers=min(c["layers"], 2)), seen)
            seen += 1


@pytest.mark.parametrize("seed", range(30))
def test_forks_and_new_lengths_against_the_model(seed):
    """Rows forked, grown, cut back - into pages that others name, too - and freed; the tables hold old entries behind every row's pages."""
    rs = np.random.RandomState(seed)
    rows, width, pages, ps = 9, 6, 60, 4
    k, v = torch.randn(2, pages, 1, ps, 8), torch.randn(2, pages, 1, 8, ps)
    ref, lens = np.zeros(pages, np.int32), np.zeros(rows, np.int32)
    table = rs.randint(0, pages, (rows, width)).astype(np.int32)
    free = rs.permutation(pages)
    for r in range(4):
        lens[r] = rs.randint(1, width * ps + 1)
        n = -(-int(lens[r]) // ps)
        table[r, :n], free = free[:n], free[n:]
        ref[table[r, :n]] = 1
    m = Model(k.numpy(), v.numpy(), table, lens, ref, ps)
    to = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32)
    s = dict(case=dict(page=ps), k_cache=k.clone(), v_cache=v.clone(), block_table=to(table), seq_len=to(lens), ref_count=to(ref))

    def check():
        for name, want in (("k_cache", m.k), ("v_cache", m.v), ("block_table", m.table), ("seq_len", m.lens), ("ref_count", m.ref)):
            assert np.array_equal(s[name].numpy(), want), name

    parents, children = rs.randint(0, 4, 4), np.array([4, 5, 6, 7])
    assert O._plain_fork(s, to(parents), to(children)).tolist() == m.fork(list(parents), list(children))
    check()
    for _ in range(3):
        some = rs.permutation(8)[:5]
        lengths = rs.randint(0, width * ps + 1, 5)
        assert O._plain_resize(s, to(some), to(lengths)).tolist() == m.resize(list(some), list(lengths))
        check()
