"""Calls on a stream that is not torch's current one: memory that they still write is nobody else's."""
import pytest
import torch

from paper_2605_21603_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(a):
    return torch.tensor(list(a), dtype=torch.int32, device=DEV)


def page_pool(max_requests=8):
    k, v = torch.zeros((2, 40, 1, 16, 8), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 40, 1, 8, 16), dtype=torch.bfloat16, device=DEV)
    return B.PagePool(k, v, ints([0] * 80).view(8, 10), ints([0] * 8), ints([0] * 40), max_requests)


def taken_again(ptr, nbytes):
    """Whether torch gives the block at `ptr` to one of the next tensors of that size on the current stream (all small blocks of a segment among them)."""
    held = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(max(4, 9000 * 512 // max(nbytes, 512)))]
    return any(t.data_ptr() <= ptr < t.data_ptr() + max(nbytes, 512) for t in held)


def results_of(pool, what, stream):
    if what == "compact":
        return list(pool.compact(stream=stream))
    return [pool.resize(ints([0, 1]), ints([40, 100]), stream=stream) if what == "resize" else pool.fork(ints([0, 1]), ints([4, 5]), stream=stream)]


@pytest.mark.parametrize("what", ["resize", "fork", "compact"])
def test_results_belong_to_the_calls_stream(what):
    """Dropped at once, or kept: a tensor made on the current stream meanwhile does not lie where the call writes, and the answer is right."""
    pool, other, s = page_pool(), page_pool(), torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)                       # the current stream is behind; the call's own stream is not
    results = results_of(pool, what, s)
    s.synchronize()
    want = {"resize": [[0, 0]], "fork": [[0, 0]], "compact": [[-1] * 40, [0]]}[what]
    assert [r.tolist() for r in results] == want
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(800_000_000)                  # the call lies behind this
    ptrs = [(r.data_ptr(), r.numel() * 4) for r in results_of(other, what, s)]
    assert not s.query()
    for ptr, nbytes in ptrs:
        assert not taken_again(ptr, nbytes)
    torch.cuda.synchronize()


@pytest.mark.parametrize("what", ["resize", "fork", "compact"])
def test_results_that_the_current_stream_still_reads(what):
    """Dropped before the current stream has come to the copy of it: the call's stream does not get the memory back until then."""
    pool, s = page_pool(), torch.cuda.Stream()
    torch.cuda.synchronize()
    results = results_of(pool, what, s)
    s.synchronize()
    want = [(r + 0).tolist() for r in results]          # (the kernel is loaded)
    torch.cuda._sleep(800_000_000)
    read = [r + 0 for r in results]
    ptrs = [(r.data_ptr(), r.numel() * 4) for r in results]
    del results
    assert not torch.cuda.current_stream().query()
    with torch.cuda.stream(s):
        assert not any(taken_again(*p) for p in ptrs)
    torch.cuda.synchronize()
    assert [r.tolist() for r in read] == want


def test_arrays_of_a_call_are_kept_until_it_has_read_them():
    """Rows and lengths that the program drops while the call waits in its stream."""
    pool, s = page_pool(), torch.cuda.Stream()
    rows, lengths = ints([2, 3, 6]), ints([33, 160, 1])
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(800_000_000)
    status = pool.resize(rows, lengths, stream=s)
    ptrs = [rows.data_ptr(), lengths.data_ptr()]
    del rows, lengths
    assert not s.query()
    assert not any(taken_again(p, 12) for p in ptrs)
    s.synchronize()
    assert status.tolist() == [0, 0, 0] and pool.seq_len.tolist() == [0, 0, 33, 160, 0, 0, 1, 0]


def attention():
    T, n_q, hd = 3, 2, 32
    cache = torch.randn((6, 1, 16, hd), device=DEV)
    q, out = torch.randn((T, n_q, hd), device=DEV), torch.empty((T, n_q, hd), device=DEV)
    return B.SharedAttention(q, out, cache, cache.view(6, 1, hd, 16).clone(), ints([0, 1, 2]), ints([20, 3, 31]), ints([0, 1, 2, 3, 4, 5]).view(3, 2))


@pytest.mark.parametrize("make,use", [(page_pool, lambda h, s: h.compact(stream=s)), (attention, lambda h, s: h.forward(s))], ids=["pages", "attention"])
@pytest.mark.parametrize("current", [False, True])
def test_a_handle_dropped_while_its_call_waits(make, use, current):
    """The workspace is the call's until it is done, whether its stream is given or torch's current one."""
    handle, s = make(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(800_000_000)
        if current:
            use(handle, None)
    if not current:
        use(handle, s)
    block = handle._workspace.bytes
    ptr, nbytes = block.data_ptr(), block.numel()
    del handle, block
    assert not s.query()
    assert not taken_again(ptr, nbytes)
    torch.cuda.synchronize()


def test_a_new_handles_first_call_on_another_stream_waits_for_what_its_memory_was_used_for():
    """A fill on the current stream still writes the block that the new handle's workspace gets: the plan of the call is not overwritten."""
    pool = page_pool()
    nbytes = pool._workspace.bytes.numel()
    del pool
    torch.cuda.synchronize()
    pools = page_pool()                                 # (its tensors; the handle itself is made again below)
    args = (pools.k_cache, pools.v_cache, pools.block_table, pools.seq_len, pools.ref_count)
    rows, lengths, s = ints([0, 1]), ints([40, 100]), torch.cuda.Stream()
    torch.cuda.synchronize()
    scratch = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(8)]
    torch.cuda._sleep(50_000_000)
    for t in scratch:
        t.fill_(0xFF)
    del scratch, t
    pool = B.PagePool(*args, 8)
    status = pool.resize(rows, lengths, stream=s)
    s.synchronize()
    assert status.tolist() == [0, 0] and pool.seq_len.tolist()[:2] == [40, 100] and pool.block_table[0, :3].tolist() == [0, 1, 2]
    torch.cuda.synchronize()


def test_two_handles_captured_on_streams_of_their_own():
    """A capture waits for no event of another stream; eager calls on the handle before, between and behind."""
    att = attention()
    want = att.forward().clone()
    pool = page_pool()
    rows, lengths, status = ints([0, 1]), ints([40, 100]), ints([9, 9])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        att.forward()
        pool.resize(rows, lengths, status)
    for i in range(3):
        att.out.zero_()
        status.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(att.out, want) and status.tolist() == [0, 0]
        att.out.zero_()
        torch.cuda.synchronize()
        att.forward(side)
        side.synchronize()
        assert torch.equal(att.out, want)
        assert pool.resize(rows, lengths, stream=side).tolist() == [0, 0]
