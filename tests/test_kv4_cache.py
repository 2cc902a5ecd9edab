"""What a cache of keys and values in 4 bits does with the calls that its
documentation allows and refuses (see test_gpu_kv4.py for its results)."""
import ctypes

import pytest
import torch

import paper_2609_32420_amd as P
from test_gpu_kv4 import DEV, _bf16, _i32


@pytest.mark.gpu
def test_a_refused_append_leaves_entries_made_ahead():
    # pages of a history entered behind the lengths, in a request that gets tokens and in one that does not
    heads, d = 1, 64
    cache = P.Kv4Cache(9, 3, 5, heads, d, 64)
    k = _bf16(140, heads, d, seed=1)
    assert cache.append(k, k, _i32([70, 5, 65]))[2] == 0
    cache.table[0, 3] = cache.table[2, 0]
    cache.table[1, 1:4] = cache.table[0, :3]
    before = cache.table.clone(), cache.kv_len.clone(), cache.free.clone()
    odd = _bf16(91 * d + 4)[4:].view(91, heads, d)  # 8 bytes off
    for v, error in ((k[:90].float(), ValueError), (k[:60], ValueError), (odd[:90], P.CarnatorError)):
        with pytest.raises(error):
            cache.append(k[:90], v, _i32([90, 0, 0]))
        for got, want in zip((cache.table, cache.kv_len, cache.free), before):
            assert torch.equal(got, want)
    assert cache.append(k[:90], k[:90], _i32([90, 0, 0]))[2] == 0
    assert torch.equal(cache.table[1:], before[0][1:]) and int(cache.kv_len[0]) == 160


@pytest.mark.parametrize("requests", [[1, 2], (slice(1, 3)), slice(-2, None), torch.tensor([1, 2]),
                                      torch.tensor([False, True, True]), [1, -1, 1], range(1, 3)])
def test_release_takes_indices_of_every_kind(requests):
    cache = P.Kv4Cache(8, 3, 3, 1, 64, 64, device="cpu")  # page tables alone: no kernel runs
    cache.table[:] = torch.tensor([[0, 1, 2], [3, 1, -1], [4, 5, 8]])
    cache.kv_len[:] = torch.tensor([192, 100, 150])
    cache.free = torch.tensor([6, 7], dtype=torch.int32)
    cache.release(requests)
    assert cache.table.tolist() == [[0, 1, 2], [-1] * 3, [-1] * 3] and cache.kv_len.tolist() == [192, 0, 0]
    assert sorted(cache.free.tolist()) == [3, 4, 5, 6, 7] and cache.free.dtype is torch.int32


@pytest.mark.parametrize("request_", [1, -2, torch.tensor(1), slice(1, 2)])
def test_release_of_one_request(request_):
    cache = P.Kv4Cache(8, 3, 3, 1, 64, 64, device="cpu")
    cache.table[:] = torch.tensor([[0, 1, 2], [3, 1, -1], [4, 5, 8]])
    cache.free = torch.tensor([6, 7], dtype=torch.int32)
    cache.release(request_)
    assert cache.table[1].tolist() == [-1] * 3 and sorted(cache.free.tolist()) == [3, 6, 7]


@pytest.mark.gpu
def test_a_workspace_that_the_kernels_cannot_use_is_refused():
    pool, table = P.kv4_pool(60, 2, 64, 64), _i32([list(range(60))])
    q, args = _bf16(2, 8, 64, seed=1), (_i32([0, 2]), _i32([3800]), 2, 64)
    want = P.kv4_attn(q, pool, table, *args)
    ws = P.kv4_attn_workspace(q, pool, table, 2, 64)
    assert ws.numel() > 1
    for bad in (ws.cpu(), ws[:1].expand(ws.numel()), torch.empty(2 * ws.numel(), dtype=torch.uint8, device=DEV)[::2]):
        with pytest.raises(ValueError):
            P.kv4_attn(q, pool, table, *args, workspace=bad)
    with pytest.raises(P.CarnatorError):
        P.kv4_attn(q, pool, table, *args, workspace=ws[:-256])
    # in bytes, whatever the type
    floats = torch.empty(ws.numel() // 4, device=DEV)
    assert torch.equal(P.kv4_attn(q, pool, table, *args, workspace=floats), want)


@pytest.mark.gpu
def test_an_lse_that_is_passed_is_written():
    pool = P.kv4_pool(3, 2, 64, 64)
    x = _bf16(150, 2, 64, seed=1)
    P.kv4_store(pool, x, x, torch.arange(150, dtype=torch.int32, device=DEV), 64)
    q, args = _bf16(3, 4, 64, seed=2), (_i32([[0, 1, 2]]), _i32([0, 3]), _i32([150]), 3, 64)
    o, want = P.kv4_attn(q, pool, *args, return_lse=True)
    lse = torch.full_like(want, 7.0)
    got = P.kv4_attn(q, pool, *args, lse=lse)
    assert torch.equal(got, o) and torch.equal(lse, want)
    with pytest.raises(ValueError):
        P.kv4_attn(q, pool, *args, lse=lse.double())


@pytest.mark.gpu
def test_an_append_is_not_captured():
    cache = P.Kv4Cache(6, 2, 3, 1, 64, 64)
    k = _bf16(2, 1, 64, seed=1)
    cache.append(k, k, _i32([1, 1]))
    before = cache.table.clone(), cache.kv_len.clone(), cache.free.clone()
    new, x = _i32([1, 1]), torch.zeros(4, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        with pytest.raises(RuntimeError, match="captured"):
            cache.append(k, k, new)
        x.add_(1)
    g.replay()
    torch.cuda.synchronize()
    for got, want in zip((cache.table, cache.kv_len, cache.free), before):
        assert torch.equal(got, want)
    assert (x == 1).all() and cache.append(k, k, new)[2] == 0 and cache.kv_len.tolist() == [2, 2]


@pytest.mark.gpu
def test_a_captured_plan_takes_pages_from_a_list_that_is_kept_in_place():
    # decoding captured whole: plan, store and attention; the free list and the lengths
    # are moved on in place before each replay
    cache = P.Kv4Cache(8, 2, 4, 1, 64, 64)
    k, v = _bf16(130, 1, 64, seed=1), _bf16(130, 1, 64, seed=2)
    assert cache.append(k, v, _i32([63, 64]))[2] == 0
    other = P.Kv4Cache(8, 2, 4, 1, 64, 64)
    assert other.append(k, v, _i32([63, 64]))[2] == 0
    free, ones, q = cache.free.clone(), _i32([1, 1]), _bf16(2, 2, 64, seed=3)
    k1, v1 = k[:2].clone(), v[:2].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        start, kv, slots, _, counts = P.page_plan(cache.kv_len, ones, cache.table, free, 64, 2)
        P.kv4_store(cache.pool, k1, v1, slots, 64)
        cache.kv_len.copy_(kv)
        out = cache.attn(q, start, 1, causal=True)
    for i in range(70):
        k1.copy_(_bf16(2, 1, 64, seed=10 + i))
        v1.copy_(_bf16(2, 1, 64, seed=99 + i))
        g.replay()
        free.copy_(free.roll(-int(counts[1])))
        q_start, _, lacking = other.append(k1, v1, ones)
        assert lacking == 0
        want = other.attn(q, q_start, 1, causal=True)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(cache.kv_len, other.kv_len) and torch.equal(cache.table, other.table)


@pytest.mark.gpu
@pytest.mark.parametrize("most", [1, 100, 2 ** 31, 2 ** 33])
def test_no_queries_at_all(most):
    pool = P.kv4_pool(3, 2, 64, 64)
    q, args = _bf16(2, 4, 64)[:0], (_i32([[0, 1, 2]]), _i32([0, 0]), _i32([150]), most, 64)
    o, lse = P.kv4_attn(q, pool, *args, return_lse=True)
    assert o.shape == (0, 4, 64) and lse.shape == (0, 4)
    assert P.kv4_attn(q, pool, *args, workspace=P.kv4_attn_workspace(q, pool, args[0], most, 64)).shape == (0, 4, 64)


def _load_strides(batch, heads, k, v):
    c = P.Kv4(0x100000, 4, heads, 128, 64)
    return P.lib().carnator_kv4_load(ctypes.byref(c), 0x10000, batch, 3, 0x10000, 100, 0x40000, *k, 0x50000, *v, None)


@pytest.mark.parametrize("batch,heads,bad", [(2, 2, (0, 12800, 128)), (2, 2, (25600, 0, 128)), (2, 1, (0, 12800, 128)),
                                             (1, 2, (0, 0, 128)), (2, 2, (64, 12800, 128)), (2, 2, (25600, 120, 128)),
                                             (1, 1, (-8, 0, 128)), (1, 1, (0, -8, 128)), (1, 1, (0, 0, 120))])
def test_load_refuses_outputs_whose_rows_share_memory(batch, heads, bad):
    good = (25600, 12800, 128)
    assert _load_strides(batch, heads, bad, good) == -2 and _load_strides(batch, heads, good, bad) == -2


@pytest.mark.gpu
def test_load_into_one_head_of_any_stride():
    pool = P.kv4_pool(3, 1, 64, 64)
    x = _bf16(150, 1, 64, seed=1)
    P.kv4_store(pool, x, x, torch.arange(150, dtype=torch.int32, device=DEV), 64)
    args = (_i32([[0, 1, 2]]), _i32([150]), 64)
    want = P.kv4_load(pool, *args, n=150)
    out = [torch.zeros(150, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    P.kv4_load(pool, *args, out=[t.as_strided((1, 1, 150, 64), (0, 0, 64, 1)) for t in out])
    for a, b in zip(out, want):
        assert torch.equal(a, b[0, 0])
    two = P.kv4_pool(3, 2, 64, 64)
    with pytest.raises(P.CarnatorError):
        P.kv4_load(two, *args, out=[t.expand(1, 2, 150, 64) for t in out])


def test_a_cache_in_host_memory_refuses_what_runs_kernels():
    cache = P.Kv4Cache(4, 1, 2, 1, 64, 64, device="cpu")
    x, two = torch.zeros(2, 1, 64, dtype=torch.bfloat16), torch.tensor([2], dtype=torch.int32)
    for f in (lambda: cache.append(x, x, two), lambda: cache.load(), lambda: cache.attn(x, torch.tensor([0, 2]), 2)):
        with pytest.raises(ValueError):
            f()
