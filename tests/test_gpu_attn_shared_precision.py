"""Attention over shared prefixes: where the layer attends with all of a probability's bits, so does the call that shares."""
import math

import pytest
import torch

import test_gpu_attn_shared as shared
from test_gpu_attn_shared import Case, group
from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", ["fast_p48", "bf16_p32", "fast_p512", "bf16_64", "bf16_256"])
@pytest.mark.parametrize("what", ["decodes", "drafts", "prompts"])
def test_probabilities_are_not_rounded_to_bf16(shape, what):
    """Queries and keys are -1, 0 and 1, so a score's products and their sum are exact.  Against 64 bits an element is then off by
      its own rounding to bf16: 2^-8 of itself;
      the two bf16 parts of a probability, which leave 2^-16 of it, once in the numerator, once in the sum: 2 x 2^-16 A, A = sum p |v| / sum p;
      the scale (a constant, a root, a quotient, a product: 5 x 2^-24 of a score s in the exp2 domain, ln 2 of which moves a probability) and the reference's
      product (2^-24 of s): 2 x 6 x 0.7 |s| 2^-24 A;
      sums over n keys and merges: (2 n + 64) 2^-24 A.
    A probability rounded to one bf16 number is off by up to 2^-8: two orders of magnitude more for the few keys of these rows."""
    seqs = {"decodes": group("a", 1, [5, 40, 3, 17, 1, 9, 31]) + [(None, 0, 50, 1), (None, 0, 2, 1)],
            "drafts": group("a", 1, [5, 40, 4, 17, 31], new=4) + [(None, 0, 50, 3)],
            "prompts": [("a", 1, 40, 40), ("a", 1, 90, 33), (None, 0, 70, 70), (None, 0, 100, 20)]}[what]
    c = Case(shape, seqs)
    signs = lambda t: torch.where(torch.isfinite(t), t.float().round().clamp(-1, 1).to(t.dtype), t)
    c.q, c.k = signs(c.q).contiguous(), signs(c.k)
    got = c.run()
    n_q, n_kv, hd, ps = c.dims
    worst = 0.0
    for t in range(len(c.seq)):
        s, n = c.seq[t], int(c.pos[t]) + 1
        pages = torch.from_numpy(c.table[s, :-(-n // ps)]).long().to(got.device)
        K = c.k[pages].double().transpose(0, 1).reshape(n_kv, -1, hd)[:, :n]
        V = c.v[pages].double().permute(1, 0, 3, 2).reshape(n_kv, -1, hd)[:, :n]
        scores = (c.q[t].double().view(n_kv, n_q // n_kv, 1, hd) * K[:, None]).sum(-1) / math.sqrt(hd)
        p = torch.softmax(scores, -1)
        want, A = (p[..., None] * V[:, None]).sum(2), (p[..., None] * V[:, None].abs()).sum(2)
        top = scores.abs().amax(-1, keepdim=True) * math.log2(math.e)
        bound = 2.0 ** -8 * want.abs() + A * (2 * 2.0 ** -16 + (2 * n + 64 + 2 * 6 * 0.7 * top) * 2.0 ** -24)
        err = (got[t].double().view(n_kv, n_q // n_kv, hd) - want).abs()
        assert (err <= bound).all(), (t, (err / bound).max().item())
        worst = max(worst, (err / bound).max().item())
    say("%s %s: worst share of the bound %.2f" % (shape, what, worst))


@pytest.mark.parametrize("name,prefixes", [("bf16_ps32", {0: (1, [0, 1, 2, 3])}), ("bf16_max", {0: (1, [0, 2, 3])}), ("bf16_hd64", {1: (2, [1, 2, 3])})])
def test_layers_on_larger_pages_and_other_heads(name, prefixes):
    """Against the oracle, under every schedule, as the layers of 16-position pages are."""
    shared.test_layer_with_shared_prefixes(name, prefixes)
