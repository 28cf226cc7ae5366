"""Timed calls of the paged cache's operators: attention over shared prefixes, and the pages' own care.

A serving program keeps one pool of cache pages for many sequences.  Sequences that begin with the same
tokens name the same pages; the attention then reads those pages once for all of them.  Between steps
pages are copied, sequences are forked from others, grown, cut back and freed, and a fragmented pool is
compacted.  Each case is one such call (or the few that belong together) on tensors in device memory.
"""
from __future__ import annotations

import functools
import math
import random

import numpy as np
import torch

own = False

# Heads and storage of the layers that the benchmark's decode steps use ("8b"), of a smaller layer with 64-wide
# heads, and of one kept in 32 bits.
SHAPES = {
    "8b": dict(dtype="bf16", n_q=32, n_kv=8, head_dim=128),
    "hd64": dict(dtype="bf16", n_q=32, n_kv=8, head_dim=64),
    "f32": dict(dtype="f32", n_q=16, n_kv=4, head_dim=64),
}


def _attention(shape, *, seqs, groups, prefix_lo, prefix_hi, suffix_lo, suffix_hi, new_lo=1, new_hi=1, alone=0, padding=0, page=16, name=None):
    """`seqs` sequences in `groups` groups; a group's prefix has prefix_lo..prefix_hi shared positions (whole pages), each
    sequence suffix_lo..suffix_hi more of its own, of which new_lo..new_hi are this step's tokens; `alone` sequences
    without a shared prefix behind them, and `padding` rows that attend nothing."""
    c = dict(op="attention", shape=shape, seqs=seqs, groups=groups, prefix_lo=prefix_lo, prefix_hi=prefix_hi, suffix_lo=suffix_lo,
             suffix_hi=suffix_hi, new_lo=new_lo, new_hi=new_hi, alone=alone, padding=padding, page=page)
    return dict(c, name=name) if name else c


def _copy(shape, *, layers, pages, copies, page=16, name=None):
    c = dict(op="copy", shape=shape, layers=layers, pages=pages, copies=copies, page=page)
    return dict(c, name=name) if name else c


def _fork(shape, *, layers, parents, children, len_lo, len_hi, draft, page=16, name=None):
    """Every one of `parents` sequences of len_lo..len_hi positions is forked `children` times, the forks grow by up to
    `draft` positions, and are freed."""
    c = dict(op="fork", shape=shape, layers=layers, parents=parents, children=children, len_lo=len_lo, len_hi=len_hi, draft=draft, page=page)
    return dict(c, name=name) if name else c


def _compact(shape, *, layers, pages, live, rows, page=16, name=None):
    """A pool of `pages` pages of which `live` are named by `rows` sequences, scattered."""
    c = dict(op="compact", shape=shape, layers=layers, pages=pages, live=live, rows=rows, page=page)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a few answers sampled from one short prompt: what a step costs when little is in it
        _attention("8b", seqs=5, groups=1, prefix_lo=512, prefix_hi=512, suffix_lo=1, suffix_hi=60, name="attn_5_samples_of_512"),
        # a server whose requests all begin with the same instructions, beside some that do not
        _attention("8b", seqs=64, groups=1, prefix_lo=2048, prefix_hi=2048, suffix_lo=16, suffix_hi=1024, alone=7, padding=3, name="attn_64_behind_2048"),
        # several long documents, many questions to each
        _attention("8b", seqs=256, groups=4, prefix_lo=4096, prefix_hi=8192, suffix_lo=33, suffix_hi=2048, name="attn_256_on_4_documents"),
        # requests that begin with the same instructions, their own prompts being read
        _attention("8b", seqs=12, groups=1, prefix_lo=4096, prefix_hi=4096, suffix_lo=40, suffix_hi=300, new_lo=33, new_hi=300, name="attn_12_prompts_behind_4096"),
        # 64-wide heads, pages of 32 positions, a few drafted tokens a sequence
        _attention("hd64", seqs=41, groups=3, prefix_lo=640, prefix_hi=1500, suffix_lo=9, suffix_hi=700, new_lo=1, new_hi=5, page=32, name="attn_hd64_41_drafts"),
        # a 32-bit layer as one runs it to check a model
        _attention("f32", seqs=24, groups=2, prefix_lo=160, prefix_hi=900, suffix_lo=1, suffix_hi=300, name="attn_f32_24_in_2_groups"),
        # one page written to while another sequence still reads it, in a whole model
        _copy("8b", layers=32, pages=64, copies=1, name="copy_1_page_32_layers"),
        # a sequence moved to other pages
        _copy("8b", layers=32, pages=1024, copies=389, name="copy_389_pages_32_layers"),
        # best of seven for one chat
        _fork("8b", layers=32, parents=1, children=7, len_lo=2901, len_hi=2901, draft=33, name="fork_1_into_7"),
        # beams of a loaded server, a few tokens drafted on each
        _fork("8b", layers=8, parents=64, children=4, len_lo=100, len_hi=1024, draft=9, name="fork_64_into_4"),
        # a small pool in 32 bits
        _compact("f32", layers=2, pages=200, live=120, rows=9, name="compact_f32_200_pages"),
        # a large pool after many sequences have ended
        _compact("8b", layers=8, pages=4000, live=2417, rows=70, name="compact_4000_pages"),
    ]


def _spread(rng, lo, hi):
    """An integer of lo..hi, uniform over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    kind = rng.choice(["attention", "attention", "attention", "attention", "copy", "fork", "compact"])
    shape = rng.choice(["8b", "8b", "8b", "hd64", "f32"])
    page = rng.choice([16, 16, 16, 32, 64]) if shape == "8b" else rng.choice([16, 32])
    if kind == "attention":
        seqs = _spread(rng, 1, 256)
        groups = min(seqs, _spread(rng, 1, 8))
        hi = _spread(rng, 64, min(16384, 32768 // groups))
        suffix = _spread(rng, 1, min(4096, max(8, 131072 // seqs)))
        new = rng.choice([1, 1, 1, _spread(rng, 1, max(1, min(suffix, 300, 12_000_000 // (seqs * (hi + suffix)))))])
        return _attention(shape, seqs=seqs, groups=groups, prefix_lo=_spread(rng, 32, hi), prefix_hi=hi, suffix_lo=_spread(rng, 1, suffix), suffix_hi=suffix,
                          new_lo=_spread(rng, 1, new), new_hi=new, alone=rng.choice([0, 0, _spread(rng, 1, 32)]), padding=rng.choice([0, 0, _spread(rng, 1, 16)]), page=page)
    layers = _spread(rng, 1, 32)
    most = 16384 * 16 // (layers * page)
    if kind == "copy":
        pages = _spread(rng, 2, most)
        return _copy(shape, layers=layers, pages=pages, copies=_spread(rng, 1, pages // 2), page=page)
    if kind == "fork":
        parents = _spread(rng, 1, 64)
        hi = _spread(rng, 1, min(4096, max(64, 262144 // (layers * parents))))
        return _fork(shape, layers=layers, parents=parents, children=_spread(rng, 1, min(32, max(1, 256 // parents))), len_lo=_spread(rng, 1, hi), len_hi=hi,
                     draft=_spread(rng, 1, 64), page=page)
    pages = _spread(rng, 16, most)
    live = rng.randint(max(1, pages // 8), pages)
    return _compact(shape, layers=layers, pages=pages, live=live, rows=_spread(rng, 1, min(live, 256)), page=page)


# ---------------------------------------------------------------------------------- the structure of a case

def _even(i, lo, hi):
    """The i-th of a run of values that cover lo..hi evenly, in no order."""
    return lo + int((hi - lo + 1) * ((i * 0.6180339887498949 + 0.5) % 1.0))


def _seqs(c):
    """(group or -1, prefix positions, context, new tokens) of every sequence."""
    ps, out = c["page"], []
    for i in range(c["seqs"]):
        g = i * c["groups"] // c["seqs"]
        prefix = _even(g, c["prefix_lo"], c["prefix_hi"]) // ps * ps
        suffix = _even(i, c["suffix_lo"], c["suffix_hi"])
        out.append((g, prefix, prefix + suffix, min(suffix, _even(i + 3, c["new_lo"], c["new_hi"]))))
    for i in range(c["alone"]):
        ctx = _even(i + 1, c["suffix_lo"], c["suffix_hi"])
        out.append((-1, 0, ctx, 1))
    return out


def _dtype(c):
    return torch.float32 if SHAPES[c["shape"]]["dtype"] == "f32" else torch.bfloat16


def _up(n, ps):
    return (n + ps - 1) // ps


def _generator(seed, device="cuda:0"):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    return gen


def _caches(c, seed, layers, pages, device="cuda:0"):
    sh, gen = SHAPES[c["shape"]], _generator(seed, device)
    k = torch.randn((layers, pages, sh["n_kv"], c["page"], sh["head_dim"]), generator=gen, device=device, dtype=_dtype(c))
    v = torch.randn((layers, pages, sh["n_kv"], sh["head_dim"], c["page"]), generator=gen, device=device, dtype=_dtype(c))
    return k, v


def _attention_inputs(c, seed, device="cuda:0"):
    sh, ps, seqs = SHAPES[c["shape"]], c["page"], _seqs(c)
    rs = np.random.RandomState(seed % (1 << 31))
    leads, n_pages = {}, 0
    shared = {}
    for s, (g, prefix, ctx, _) in enumerate(seqs):
        if g >= 0 and g not in shared:
            shared[g] = np.arange(n_pages, n_pages + prefix // ps)
            n_pages += prefix // ps
            leads[g] = s
    own_pages = []
    for g, prefix, ctx, _ in seqs:
        n = _up(ctx, ps) - prefix // ps
        own_pages.append(np.arange(n_pages, n_pages + n))
        n_pages += n
    perm = rs.permutation(n_pages).astype(np.int32)
    table = np.zeros((len(seqs), max(_up(s[2], ps) for s in seqs)), dtype=np.int32)
    for s, (g, prefix, ctx, _) in enumerate(seqs):
        row = np.concatenate([shared[g], own_pages[s]]) if g >= 0 else own_pages[s]
        table[s, :len(row)] = perm[row]
    new = [n for _, _, _, n in seqs]
    seq_of_token = np.concatenate([np.repeat(np.arange(len(seqs)), new), np.zeros(c["padding"], dtype=np.int64)]).astype(np.int32)
    pos_of_token = np.concatenate([np.arange(ctx - n, ctx) for _, _, ctx, n in seqs] + [np.full(c["padding"], -1)]).astype(np.int32)
    lead = np.array([leads[g] if g >= 0 else s for s, (g, _, _, _) in enumerate(seqs)], dtype=np.int32)
    pages = np.array([prefix // ps for _, prefix, _, _ in seqs], dtype=np.int32)
    k, v = _caches(c, seed, 1, n_pages, device)
    # what the projections before it leave: rows with the q heads first, k and v behind them
    width = (sh["n_q"] + 2 * sh["n_kv"]) * sh["head_dim"]
    qkv = torch.randn((len(seq_of_token), width), generator=_generator(seed + 1, device), device=device, dtype=_dtype(c))
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
    return dict(qkv=qkv, k_cache=k[0], v_cache=v[0], seq_of_token=to(seq_of_token), pos_of_token=to(pos_of_token), block_table=to(table),
                prefix_lead=to(lead), prefix_pages=to(pages))


@functools.lru_cache(maxsize=64)
def _scattered(pages, live, rows):
    """Which pages are live, as the rows' page lists: a pool's history, the same for every seed."""
    rs = np.random.RandomState(pages * 31 + live * 7 + rows)
    used = rs.permutation(pages)[:live].astype(np.int32)
    cuts = np.sort(rs.choice(np.arange(1, live), rows - 1, replace=False)) if rows > 1 else np.array([], dtype=np.int64)
    return np.split(used, cuts)


def _moves(c):
    used = np.concatenate(_scattered(c["pages"], c["live"], c["rows"]))
    return int((used >= c["live"]).sum())


def _pool_inputs(c, seed, device="cuda:0"):
    """A pool of pages: both caches, block table, positions of every row, references to every page; and the calls' own arrays."""
    ps, to = c["page"], lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
    rs = np.random.RandomState(seed % (1 << 31))
    if c["op"] == "copy":
        k, v = _caches(c, seed, c["layers"], c["pages"], device)
        perm = rs.permutation(c["pages"]).astype(np.int32)
        return dict(k_cache=k, v_cache=v, block_table=to(np.zeros((1, 1), np.int32)), seq_len=to(np.zeros(1, np.int32)), ref_count=to(np.ones(c["pages"], np.int32)),
                    src=to(perm[:c["copies"]]), dst=to(perm[c["copies"]:2 * c["copies"]]))
    if c["op"] == "fork":
        lens = np.array([_even(i, c["len_lo"], c["len_hi"]) for i in range(c["parents"])], dtype=np.int32)
        n_child = c["parents"] * c["children"]
        width = _up(c["len_hi"] + c["draft"], ps)
        n_pages = int(sum(_up(int(n), ps) for n in lens))
        spare = n_child * (_up(c["draft"], ps) + 1)
        perm = rs.permutation(n_pages + spare).astype(np.int32)
        table = np.zeros((c["parents"] + n_child, width), dtype=np.int32)
        ref = np.zeros(n_pages + spare, dtype=np.int32)
        at = 0
        for p, n in enumerate(lens):
            m = _up(int(n), ps)
            table[p, :m] = perm[at:at + m]
            ref[perm[at:at + m]] = 1
            at += m
        parent = np.tile(np.arange(c["parents"]), c["children"]).astype(np.int32)
        grown = (lens[parent] + np.array([_even(i, 1, c["draft"]) for i in range(n_child)])).astype(np.int32)
        k, v = _caches(c, seed, c["layers"], n_pages + spare, device)
        return dict(k_cache=k, v_cache=v, block_table=to(table), seq_len=to(np.concatenate([lens, np.zeros(n_child, np.int32)])), ref_count=to(ref),
                    parent=to(parent), child=to(np.arange(c["parents"], c["parents"] + n_child, dtype=np.int32)), grown=to(grown),
                    nothing=to(np.zeros(n_child, np.int32)))
    lists = _scattered(c["pages"], c["live"], c["rows"])
    table = np.zeros((c["rows"], max(len(r) for r in lists)), dtype=np.int32)
    ref = np.zeros(c["pages"], dtype=np.int32)
    for r, used in enumerate(lists):
        table[r, :len(used)] = used
        ref[used] += 1
    lens = np.array([(len(r) - 1) * ps + rs.randint(1, ps + 1) for r in lists], dtype=np.int32)
    k, v = _caches(c, seed, c["layers"], c["pages"], device)
    return dict(k_cache=k, v_cache=v, block_table=to(table), seq_len=to(lens), ref_count=to(ref), table_before=to(table), ref_before=to(ref))


# ---------------------------------------------------------------------------------- one pass

def prepare(c, seed):
    """The tensors of a call in device memory; with the framework's operators the handle that a program keeps beside them."""
    if c["op"] == "attention":
        d, sh = _attention_inputs(c, seed), SHAPES[c["shape"]]
        T = d["qkv"].shape[0]
        d["q"] = d["qkv"][:, :sh["n_q"] * sh["head_dim"]].view(T, sh["n_q"], sh["head_dim"])
        d["out"] = torch.empty((T, sh["n_q"], sh["head_dim"]), dtype=d["q"].dtype, device=d["q"].device)
        if own:
            from paper_2605_21603_amd import binding as B
            d["call"] = B.SharedAttention(d["q"], d["out"], d["k_cache"], d["v_cache"], d["seq_of_token"], d["pos_of_token"], d["block_table"],
                                          d["prefix_lead"], d["prefix_pages"])
        else:
            d["groups"] = _plain_groups(c, d["q"].device)
    else:
        d = _pool_inputs(c, seed)
        if own:
            from paper_2605_21603_amd import binding as B
            d["pool"] = B.PagePool(d["k_cache"], d["v_cache"], d["block_table"], d["seq_len"], d["ref_count"],
                                   max_requests=max(1, c["parents"] * c["children"] if c["op"] == "fork" else 1))
            d["status"] = torch.zeros((3, max(1, c["parents"] * c["children"] if c["op"] == "fork" else 1)), dtype=torch.int32, device=d["k_cache"].device)
            if c["op"] == "compact":
                d["new_page"] = torch.empty(c["pages"], dtype=torch.int32, device=d["k_cache"].device)
                d["n_live"] = torch.empty(1, dtype=torch.int32, device=d["k_cache"].device)
    return dict(case=c, **d)


def run(s):
    """One pass: the attention's rows; or the pool as the calls leave it, with what they answer."""
    op = s["case"]["op"]
    if op == "attention":
        if own:
            s["call"].forward()
            return s["out"]
        return _plain_attention(s)
    if op == "copy":
        if own:
            s["pool"].copy(s["src"], s["dst"])
        else:
            _plain_copy(s, s["src"], s["dst"])
        return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
    if op == "fork":
        if own:
            forked = s["pool"].fork(s["parent"], s["child"], s["status"][0])
            grown = s["pool"].resize(s["child"], s["grown"], s["status"][1])
            freed = s["pool"].resize(s["child"], s["nothing"], s["status"][2])
        else:
            forked = _plain_fork(s, s["parent"], s["child"])
            grown = _plain_resize(s, s["child"], s["grown"])
            freed = _plain_resize(s, s["child"], s["nothing"])
        return dict(k_cache=s["k_cache"], v_cache=s["v_cache"], block_table=s["block_table"], seq_len=s["seq_len"], ref_count=s["ref_count"],
                    forked=forked, grown=grown, freed=freed)
    # the pool is fragmented again: what moved away is still where it was
    s["block_table"].copy_(s["table_before"])
    s["ref_count"].copy_(s["ref_before"])
    if own:
        s["pool"].compact(s["new_page"], s["n_live"])
        new_page, n_live = s["new_page"], s["n_live"]
    else:
        new_page, n_live = _plain_compact(s)
    return dict(k_cache=s["k_cache"], v_cache=s["v_cache"], block_table=s["block_table"], ref_count=s["ref_count"], new_page=new_page, n_live=n_live)


# ---------------------------------------------------------------------------------- the plain forms

def _plain_groups(c, device):
    """Runs of sequences that are computed together: (first sequence, end, prefix pages, suffix positions, tokens, and the rows
    as [sequence, token], short ones filled up with their last row)."""
    seqs, out, row = _seqs(c), [], 0
    s = 0
    while s < len(seqs):
        e = s + 1
        while e < len(seqs) and e - s < 64 and seqs[e][:2] == seqs[s][:2]:
            e += 1
        members = seqs[s:e]
        new, at = max(m[3] for m in members), []
        for _, _, _, n in members:
            at.append([row + min(j, n - 1) for j in range(new)])
            row += n
        out.append((s, e, members[0][1] // c["page"], max(m[2] - m[1] for m in members), new, torch.tensor(at, device=device)))
        s = e
    return out


def _plain_attention(s):
    c = s["case"]
    sh, ps = SHAPES[c["shape"]], c["page"]
    n_q, n_kv, d = sh["n_q"], sh["n_kv"], sh["head_dim"]
    G, dev, scale = n_q // n_kv, s["q"].device, 1.0 / math.sqrt(d)
    out = torch.zeros(s["q"].shape, dtype=torch.float32, device=dev)
    for s0, s1, prefix_pages, suffix, new, at in s["groups"]:
        n, P = s1 - s0, prefix_pages * ps
        q = s["q"][at].float().view(n, new, n_kv, G, d).permute(2, 0, 1, 3, 4).contiguous()                  # [kv, seq, token, head, d]
        pos = s["pos_of_token"][at].long()
        scores, values = [], []
        if P:
            table = s["block_table"][s0, :prefix_pages].long()
            K = s["k_cache"][table].float().permute(1, 0, 2, 3).reshape(n_kv, P, d)
            V = s["v_cache"][table].float().permute(1, 0, 3, 2).reshape(n_kv, P, d)
            scores.append((q.view(n_kv, -1, d) @ K.transpose(1, 2)).view(n_kv, n, new, G, P) * scale)
            values.append(V)
        own_pages = _up(suffix, ps)
        cols = (prefix_pages + torch.arange(own_pages, device=dev)).clamp_(max=s["block_table"].shape[1] - 1)
        table = s["block_table"][s0:s1, cols].long()
        K = s["k_cache"][table].float().permute(2, 0, 1, 3, 4).reshape(n_kv * n, own_pages * ps, d)
        V = s["v_cache"][table].float().permute(2, 0, 1, 4, 3).reshape(n_kv * n, own_pages * ps, d)
        sc = (q.view(n_kv * n, new * G, d) @ K.transpose(1, 2)).view(n_kv, n, new, G, own_pages * ps) * scale
        key = P + torch.arange(own_pages * ps, device=dev)
        hidden = key[None, None, :] > pos[:, :, None]                                                         # [seq, token, key]
        scores.append(sc.masked_fill(hidden[None, :, :, None, :], -math.inf))
        m = scores[-1].amax(-1, keepdim=True)
        if P:
            m = torch.maximum(m, scores[0].amax(-1, keepdim=True))
        p = torch.exp(scores[-1] - m)
        total = p.sum(-1, keepdim=True)
        o = (p.view(n_kv * n, new * G, -1) @ V).view(n_kv, n, new, G, d)
        if P:
            p = torch.exp(scores[0] - m)
            total = total + p.sum(-1, keepdim=True)
            o = o + (p.view(n_kv, -1, P) @ values[0]).view(n_kv, n, new, G, d)
        out[at] = (o / total).permute(1, 2, 0, 3, 4).reshape(n, new, n_q, d)
    return out.to(s["q"].dtype)


def _plain_copy(s, src, dst):
    src, dst = src.long(), dst.long()
    for cache in (s["k_cache"], s["v_cache"]):
        cache[:, dst] = cache[:, src]


def _plain_take(s, need):
    """Which requests get their pages, and the free pages in order with the place of each request's first."""
    free = s["ref_count"] == 0
    order = torch.sort(free.logical_not().to(torch.int32), stable=True).indices
    upto = need.cumsum(0)
    return (need == 0) | (upto <= free.sum()), order, upto - need


def _add_refs(s, pages, mask, by):
    """ref_count[page] += by for every masked entry."""
    ref = torch.cat([s["ref_count"], s["ref_count"].new_zeros(1)])
    ref.index_add_(0, torch.where(mask, pages, len(s["ref_count"])).flatten().long(), torch.full((pages.numel(),), by, dtype=ref.dtype, device=ref.device))
    s["ref_count"].copy_(ref[:-1])


def _plain_fork(s, parent, child):
    ps, parent, child = s["case"]["page"], parent.long(), child.long()
    table, lens = s["block_table"], s["seq_len"][parent]
    full, tail = lens // ps, (lens % ps != 0).to(torch.int64)
    ok, order, first = _plain_take(s, tail)
    cols = torch.arange(table.shape[1], device=table.device)[None, :]
    rows = table[parent]
    fresh = order[first.clamp(max=len(order) - 1)].to(torch.int32)
    has_tail = ok & (tail > 0)
    last = rows.gather(1, full[:, None].clamp(max=table.shape[1] - 1).long())[:, 0]
    shared = ok[:, None] & (cols < full[:, None])
    _add_refs(s, rows, shared, 1)
    _add_refs(s, fresh, has_tail, 1)
    entry = has_tail[:, None] & (cols == full[:, None])
    table[child] = torch.where(shared, rows, torch.where(entry, fresh[:, None], table[child]))
    s["seq_len"][child] = torch.where(ok, lens, 0)
    _plain_copy(s, last[has_tail], fresh[has_tail])
    return torch.where(ok, 0, 1).to(torch.int32)


def _plain_resize(s, row, length):
    ps, row = s["case"]["page"], row.long()
    table, before = s["block_table"], s["seq_len"][row]
    had, has = (before + ps - 1) // ps, (length + ps - 1) // ps
    cols = torch.arange(table.shape[1], device=table.device)[None, :]
    rows = table[row]
    # a last page that stays, partly filled, must be the row's own
    last = rows.gather(1, (has - 1)[:, None].clamp(0, table.shape[1] - 1).long())[:, 0]
    part = (length < before) & (length % ps != 0) & (s["ref_count"][last.long()] > 1)
    ok, order, first = _plain_take(s, torch.where(part, 1, (has - had).clamp(min=0)).to(torch.int64))
    taken = order[(first[:, None] + (cols - had[:, None]).clamp(min=0)).clamp(max=len(order) - 1)].to(torch.int32)
    grown = ok[:, None] & (cols >= had[:, None]) & (cols < has[:, None])
    split = ok & part
    fresh = order[first.clamp(max=len(order) - 1)].to(torch.int32)
    entry = split[:, None] & (cols == (has - 1)[:, None])
    _add_refs(s, rows, (ok[:, None] & (cols >= has[:, None]) & (cols < had[:, None])) | entry, -1)
    _add_refs(s, taken, grown, 1)
    _add_refs(s, fresh, split, 1)
    table[row] = torch.where(grown, taken, torch.where(entry, fresh[:, None], rows))
    s["seq_len"][row] = torch.where(ok, length, before)
    _plain_copy(s, last[split], fresh[split])
    return torch.where(ok, 0, 1).to(torch.int32)


def _plain_compact(s):
    ref, ps = s["ref_count"], s["case"]["page"]
    n, dev = len(ref), ref.device
    page = torch.arange(n, device=dev)
    live = ref > 0
    n_live = live.sum()
    moving, hole = live & (page >= n_live), (~live) & (page < n_live)
    src, dst = moving.nonzero()[:, 0], hole.nonzero()[:, 0]                           # as many holes as pages behind them
    to = page.clone()
    to[src] = dst
    used = torch.arange(s["block_table"].shape[1], device=dev)[None, :] < ((s["seq_len"] + ps - 1) // ps)[:, None]
    s["block_table"].copy_(torch.where(used, to[s["block_table"].long()].to(torch.int32), s["block_table"]))
    ref[dst] = ref[src]
    ref[src] = 0
    _plain_copy(s, src, dst)
    new_page = torch.where(live, to, -1)
    return new_page.to(torch.int32), n_live.to(torch.int32).view(1)


# ---------------------------------------------------------------------------------- what a pass needs, and what it should give

def work(c):
    sh = SHAPES[c["shape"]]
    e = 4 if sh["dtype"] == "f32" else 2
    position = 2 * sh["n_kv"] * sh["head_dim"] * e                            # K and V of one position and layer
    if c["op"] == "attention":
        seqs = _seqs(c)
        prefixes = {g: prefix for g, prefix, _, _ in seqs if g >= 0}
        T = sum(n for _, _, _, n in seqs) + c["padding"]
        cached = sum(prefixes.values()) + sum(ctx - prefix for _, prefix, ctx, _ in seqs)
        keys = sum(n * (ctx - n) + n * (n + 1) // 2 for _, _, ctx, n in seqs)
        return {"bytes": cached * position + 2 * T * sh["n_q"] * sh["head_dim"] * e, "flops": 4 * sh["n_q"] * sh["head_dim"] * keys}
    page = position * c["page"] * c["layers"]
    if c["op"] == "copy":
        return {"bytes": 2 * c["copies"] * page, "flops": 0}
    if c["op"] == "compact":
        return {"bytes": 2 * _moves(c) * page + 16 * c["pages"] + 8 * c["live"], "flops": 0}
    lens = [_even(i, c["len_lo"], c["len_hi"]) for i in range(c["parents"])]
    tails = [n % c["page"] != 0 for n in lens]
    tables = sum(_up(n, c["page"]) for n in lens) * c["children"]
    return {"bytes": (1 + c["children"]) * sum(tails) * page + 4 * 8 * tables, "flops": 0}


def exact(c, seed):
    """Attention of every row over its own sequence's keys, in 64 bits; for the pages' operators what a program that cares for
    one page after another on the host would leave."""
    if c["op"] != "attention":
        return _exact_pages(c, _pool_inputs(c, seed))
    d, sh, ps = _attention_inputs(c, seed), SHAPES[c["shape"]], c["page"]
    n_q, n_kv, hd = sh["n_q"], sh["n_kv"], sh["head_dim"]
    T = d["qkv"].shape[0]
    q = d["qkv"][:, :n_q * hd].double().view(T, n_kv, n_q // n_kv, hd)
    out = torch.zeros((T, n_q, hd), dtype=torch.float64, device=q.device)
    row = 0
    for s, (_, _, ctx, n) in enumerate(_seqs(c)):
        pages = d["block_table"][s, :_up(ctx, ps)].long()
        K = d["k_cache"][pages].double().transpose(0, 1).reshape(n_kv, -1, hd)[:, :ctx]
        V = d["v_cache"][pages].double().permute(1, 0, 3, 2).reshape(n_kv, -1, hd)[:, :ctx]
        for t in range(n):
            seen = ctx - n + t + 1
            score = (q[row + t] @ K[:, :seen].transpose(1, 2).contiguous()) / math.sqrt(hd)
            out[row + t] = (torch.softmax(score, -1) @ V[:, :seen]).view(n_q, hd)
        row += n
    return out


def _exact_pages(c, d):
    ps = c["page"]
    table, lens, ref = (d[n].cpu().numpy().copy() for n in ("block_table", "seq_len", "ref_count"))
    copies = {}                                          # page -> the page whose content at the start it has in the end
    host = lambda n: d[n].cpu().tolist()

    def lowest_free(taken):
        for p in range(len(ref)):
            if ref[p] == 0 and p not in taken:
                return p
        return None

    out = {}
    if c["op"] == "copy":
        copies = dict(zip(host("dst"), host("src")))
    elif c["op"] == "fork":
        taken, answer = set(), []
        after = ref.copy()
        for parent, child in zip(host("parent"), host("child")):
            pages = table[parent, :_up(int(lens[parent]), ps)].copy()
            answer.append(0)
            if lens[parent] % ps:
                fresh = lowest_free(taken)
                if fresh is None:
                    answer[-1] = 1
                    continue
                taken.add(fresh)
                copies[fresh] = int(pages[-1])
                pages[-1] = fresh
            np.add.at(after, pages, 1)
            table[child, :len(pages)] = pages
            lens[child] = lens[parent]
        ref, taken, grown = after, set(), []
        after = ref.copy()
        for child, n in zip(host("child"), host("grown")):
            had, has = _up(int(lens[child]), ps), _up(n, ps)
            fresh = []
            while len(fresh) < has - had and (p := lowest_free(taken)) is not None:
                fresh.append(p)
                taken.add(p)
            grown.append(0 if len(fresh) == max(0, has - had) else 1)
            if not grown[-1]:
                table[child, had:has] = fresh
                after[fresh] = 1
                lens[child] = n
        ref = after
        for child in host("child"):
            np.subtract.at(ref, table[child, :_up(int(lens[child]), ps)], 1)
            lens[child] = 0
        out = dict(forked=answer, grown=grown, freed=[0] * len(answer))
    else:
        live = [p for p in range(len(ref)) if ref[p] > 0]
        holes = [p for p in range(len(live)) if ref[p] == 0]
        new_page = np.full(len(ref), -1, dtype=np.int64)
        new_page[live] = live
        for src, dst in zip([p for p in live if p >= len(live)], holes):
            new_page[src], copies[dst] = dst, src
            ref[dst], ref[src] = ref[src], 0
        for r in range(len(table)):
            n = _up(int(lens[r]), ps)
            table[r, :n] = new_page[table[r, :n]]
        out = dict(new_page=new_page, n_live=[len(live)])
    at = torch.arange(d["k_cache"].shape[1])
    for dst, src in copies.items():
        at[dst] = src
    at = at.to(d["k_cache"].device)
    want = dict(k_cache=d["k_cache"][:, at].double(), v_cache=d["v_cache"][:, at].double())
    if c["op"] == "copy":
        return want
    want.update(block_table=table, seq_len=lens, ref_count=ref)
    if c["op"] == "compact":
        del want["seq_len"]
    want.update(out)
    return {n: v if isinstance(v, torch.Tensor) else torch.as_tensor(np.asarray(v), device=at.device).double() for n, v in want.items()}
