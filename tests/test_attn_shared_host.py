"""Attention over shared prefixes without a GPU: what the entry point and the layer refuse, and the workspace they ask for."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_21603_amd import binding as B
from workloads import gen

GOOD = dict(dtype=B.DYN_BF16, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_tokens=5, n_seqs=5, q=0x10000, ld_q=1024, out=0x20000, ld_out=1024,
            seq_of_token=0x30000, pos_of_token=0x30100, block_table=0x30200, max_pages_per_seq=9, prefix_lead=0x30300, prefix_pages=0x30400, k_cache=0x40000,
            v_cache=0x50000, workspace=0x60000, workspace_bytes=1 << 30)


def batch(**change):
    b = B.dyn_attn_batch()
    for name, value in dict(GOOD, **change).items():
        setattr(b, name, value)
    return b


@pytest.mark.parametrize("change,status,text", [
    (dict(dtype=2), B.DYN_ERR_INVALID_ARG, "dtype"),
    (dict(n_kv_heads=3), B.DYN_ERR_INVALID_ARG, "multiple"),
    (dict(n_q_heads=0), B.DYN_ERR_INVALID_ARG, "non-positive"),
    (dict(head_dim=96), B.DYN_ERR_UNSUPPORTED, "power of two"),
    (dict(head_dim=512), B.DYN_ERR_UNSUPPORTED, "power of two"),
    (dict(page_size=513), B.DYN_ERR_UNSUPPORTED, "page_size"),
    (dict(kv_chunk_positions=40), B.DYN_ERR_INVALID_ARG, "kv_chunk_positions"),
    (dict(n_tokens=-1), B.DYN_ERR_INVALID_ARG, "negative"),
    (dict(n_tokens=1 << 24), B.DYN_ERR_UNSUPPORTED, "tokens"),
    (dict(n_seqs=0), B.DYN_ERR_INVALID_ARG, "without sequences"),
    (dict(max_pages_per_seq=0), B.DYN_ERR_INVALID_ARG, "without sequences"),
    (dict(n_seqs=1 << 20, max_pages_per_seq=1 << 9), B.DYN_ERR_UNSUPPORTED, "2^29"),
    (dict(n_seqs=1, max_pages_per_seq=1 << 27), B.DYN_ERR_UNSUPPORTED, "2^30 positions"),
    (dict(q=None), B.DYN_ERR_INVALID_ARG, "NULL"),
    (dict(v_cache=None), B.DYN_ERR_INVALID_ARG, "NULL"),
    (dict(out=0x10000), B.DYN_ERR_INVALID_ARG, "alias"),
    (dict(prefix_pages=None), B.DYN_ERR_INVALID_ARG, "go together"),
    (dict(ld_q=1000), B.DYN_ERR_INVALID_ARG, "fit"),
    (dict(ld_out=1028), B.DYN_ERR_INVALID_ARG, "16-byte"),
    (dict(k_cache=0x40008), B.DYN_ERR_INVALID_ARG, "16-byte"),
    (dict(workspace=None), B.DYN_ERR_WORKSPACE, "workspace"),
    (dict(workspace_bytes=1 << 12), B.DYN_ERR_WORKSPACE, "needs"),
])
def test_refusals(change, status, text):
    assert B.lib().dyn_attn_shared(C.byref(batch(**change)), None) == status and text in B.dyn_last_error(), B.dyn_last_error()


def test_no_tokens_is_no_work():
    assert B.lib().dyn_attn_shared(C.byref(batch(n_tokens=0, n_seqs=0, q=None, workspace=None)), None) == B.DYN_OK
    assert B.lib().dyn_attn_shared(None, None) == B.DYN_ERR_INVALID_ARG


def test_workspace_grows_with_the_batch():
    size = lambda **change: B.lib().dyn_attn_shared_workspace_bytes(C.byref(batch(**change)))
    assert 0 < size() < size(n_tokens=9) < size(n_tokens=9, max_pages_per_seq=900)
    assert size(dtype=7) == 0
    # long rows: the shared keys have at most 32 chunks of up to 8192 positions, and more chunks only beyond that
    a, b = (size(n_tokens=1, max_pages_per_seq=n) for n in (16384, 32768))
    assert a < b < 2.2 * a


def test_binding_checks_tensors():
    q, cache = torch.zeros(3, 4, 32), torch.zeros(6, 2, 16, 32)
    ok = dict(q=q, out=torch.zeros(3, 4, 32), k_cache=cache, v_cache=cache.view(6, 2, 32, 16), seq_of_token=torch.zeros(3, dtype=torch.int32),
              pos_of_token=torch.zeros(3, dtype=torch.int32), block_table=torch.zeros(2, 3, dtype=torch.int32))
    for bad in (dict(out=torch.zeros(3, 4, 16)), dict(q=q.double()), dict(q=torch.zeros(3, 32, 4).transpose(1, 2)), dict(v_cache=cache), dict(pos_of_token=torch.zeros(3)),
                dict(pos_of_token=torch.zeros(4, dtype=torch.int32)), dict(prefix_lead=torch.zeros(2, dtype=torch.int32)),
                dict(prefix_lead=torch.zeros(3, dtype=torch.int32), prefix_pages=torch.zeros(3, dtype=torch.int32)),
                dict(q=torch.zeros(1, 4, 32).expand(3, 4, 32))):
        with pytest.raises(ValueError):
            B.SharedAttention(**dict(ok, **bad))
    with pytest.raises(ValueError, match="on a GPU"):
        B.SharedAttention(**ok)


def layer_and_batch(name="c2_small", **fields):
    w = gen.config(name)
    fake = {n: 0x1000 for n in ("w_qkv", "w_o", "w_gate_up", "w_down", "g_norm1", "g_norm2")}
    layer = B.DynLayer(B.make_config(w.shape), [fake] * w.shape.n_layers)
    md = gen.metadata(w)
    q = np.ascontiguousarray(md["q_start"])
    b = B.dyn_batch(w.n_tokens, w.n_seqs, 0x10000, 0x20000, 0x30000, 0x30000, 0x30000, md["max_pages_per_seq"], q.ctypes.data, 0x40000, 0x50000, 1 << 20, None, 0)
    b._keep = q
    for field, value in fields.items():
        setattr(b, field, value)
    return w, layer, b


def test_layer_refuses_half_a_prefix_and_too_large_a_table():
    for fields, status, text in ((dict(prefix_lead=0x1000), B.DYN_ERR_INVALID_ARG, "go together"), (dict(prefix_pages=0x1000), B.DYN_ERR_INVALID_ARG, "go together"),
                                 (dict(prefix_lead=0x1000, prefix_pages=0x1000, max_pages_per_seq=1 << 26), B.DYN_ERR_UNSUPPORTED, "2^29")):
        _, layer, b = layer_and_batch(**fields)
        sc = B.sequential().to_c()
        assert B.lib().dyn_layer_forward(layer.handle, C.addressof(b), C.addressof(sc), None) == status and text in B.dyn_last_error()


@pytest.mark.parametrize("name", ["c2_small", "c3_small", "f32_small", "stack_mixed"])
def test_schedules_with_shared_prefixes_have_room_of_their_own(name):
    """The workspace holds the partials of the shared keys beside those of the own ones, for every schedule; a batch without them
    needs what it always did."""
    w, layer, plain = layer_and_batch(name)
    _, _, b = layer_and_batch(name, prefix_lead=0x1000, prefix_pages=0x1000)
    scheds = [B.sequential(), B.nano_schedule(w.nano_rows, stagger=1)]
    for sched in scheds:
        assert layer.schedule_workspace_bytes(b, sched) > layer.schedule_workspace_bytes(plain, sched)
        report = layer.memory(b, sched)
        assert report["workspace_bytes"] >= report["workspace_bytes_schedule"] >= report["peak_live_bytes"]
        regions = {(r["kind"], r["slot"]): r for r in layer.schedule_regions(b, sched)}
        for key, r in {(r["kind"], r["slot"]): r for r in layer.schedule_regions(plain, sched)}.items():
            assert regions[key]["bytes"] > r["bytes"] if key[0] in ("part_o", "part_ml", "plan") else regions[key]["bytes"] == r["bytes"]
    assert layer.memory(plain, scheds[0])["workspace_bytes"] == layer.workspace_bytes(w.n_tokens, plain.max_pages_per_seq)
