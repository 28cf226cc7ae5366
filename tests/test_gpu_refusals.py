"""What the handles of the shared attention and the page operators refuse when they are made: with the library's own status and words."""
import pytest
import torch

from paper_2605_21603_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEV)


def attention(hd=32, ps=16, **change):
    k, q = torch.zeros((2, 1, ps, hd), device=DEV), torch.zeros((1, 1, hd), device=DEV)
    return B.SharedAttention(q, q.clone(), k, k.view(2, 1, hd, ps), ints(1), ints(1), ints(1, 1), **change)


def pool(hd=8, ps=16, max_requests=1):
    k = torch.zeros((1, 2, 1, ps, hd), device=DEV)
    return B.PagePool(k, k.view(1, 2, 1, hd, ps), ints(1, 1), ints(1), ints(2), max_requests)


@pytest.mark.parametrize("make,status,text", [
    (lambda: attention(hd=96), B.DYN_ERR_UNSUPPORTED, "power of two"),
    (lambda: attention(ps=1024), B.DYN_ERR_UNSUPPORTED, "page_size"),
    (lambda: attention(kv_chunk_positions=40), B.DYN_ERR_INVALID_ARG, "kv_chunk_positions"),
    (lambda: pool(ps=1, hd=2), B.DYN_ERR_UNSUPPORTED, "multiple of 16"),
    (lambda: pool(ps=1024), B.DYN_ERR_UNSUPPORTED, "page_size"),
    (lambda: pool(max_requests=-1), B.DYN_ERR_INVALID_ARG, "max_requests = -1"),
])
def test_status_and_words(make, status, text):
    with pytest.raises(B.DynError, match=text) as e:
        make()
    assert e.value.status == status


def test_no_words_of_an_earlier_refusal():
    with pytest.raises(B.DynError, match="power of two"):
        attention(hd=96)
    with pytest.raises(B.DynError, match="max_requests = -3"):
        pool(max_requests=-3)
    attention().forward()
    pool(max_requests=0).compact()
    torch.cuda.synchronize()
