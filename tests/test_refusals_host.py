"""Sizes that the shared attention's entry point cannot count."""
import ctypes as C

import pytest

from paper_2605_21603_amd import binding as B
from test_attn_shared_host import batch


@pytest.mark.parametrize("heads,head_dim", [(1 << 24, 256), (1 << 24, 128), ((1 << 28) - 1, 16)])
def test_rows_of_more_elements_than_32_bits_count(heads, head_dim):
    b = batch(n_q_heads=heads, n_kv_heads=heads, head_dim=head_dim, ld_q=1 << 30, ld_out=1 << 30, workspace_bytes=1 << 62)
    assert B.lib().dyn_attn_shared(C.byref(b), None) == B.DYN_ERR_UNSUPPORTED and "elements" in B.dyn_last_error()
    assert B.lib().dyn_attn_shared_workspace_bytes(C.byref(b)) == 0
