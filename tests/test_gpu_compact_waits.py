"""Compactions whose chains have several segments, which wait for each other by flags in the pool's workspace: captured ones after the
workspace has grown, and waits that do not end."""
import numpy as np
import pytest
import torch

import paper_2506_15155_amd as E
from tests.test_gpu_fp4 import Cache
from tests.test_gpu_tokens import read, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [E.ELLM_BF16, E.ELLM_MXFP4])
def test_replays_after_the_workspace_has_grown(dtype):
    """A partition override makes a decode call allocate a larger workspace; what was captured before keeps the one that it has."""
    c = Cache([3000, 0, 40000], 2, 2, 128, 100, dtype, room=3000)
    E.ellm_pool_prepare(c.pool)
    # a wave for every 64 tokens leaves more partial results than SIMDs + n_kv * (tensors - 1), what the workspace is made for
    assert 2 * 40000 // 64 > E.ellm_workspace_bytes(4, 2, 128, 5) // (2 * 130 * 4)
    keep = torch.arange(3, 3000, 2, dtype=torch.int32, device="cuda")
    q, dq = c.queries()
    small, out = dq[:1].contiguous(), torch.full_like(dq[:1], 77)
    want = c.decode(small, [c.ids[0]])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        E.ellm_kv_copy(c.pool, [c.ids[0]], [c.ids[1]])
        E.ellm_kv_compact(c.pool, [c.ids[1]], keep=keep, n_keep=[len(keep)])
        E.ellm_decode_attention(c.pool, [c.ids[0]], small, out)
    c.k[1], c.v[1] = c.k[0][3::2], c.v[0][3::2]
    g.replay()
    same(c)
    assert torch.equal(out, want)
    E.ellm_pool_set_split_tokens(c.pool, 64)
    large = dq[2:].contiguous()
    c.check(c.decode(large, [c.ids[2]]), q[2:], [2])
    E.ellm_pool_set_split_tokens(c.pool, 0)
    others = [torch.full((1 << 20,), 0x55, dtype=torch.uint8, device="cuda") for _ in range(40)]    # whoever gets freed memory next
    for _ in range(3):
        out.fill_(77)
        g.replay()
        same(c)
        assert torch.equal(out, want)
        c.check(c.decode(large, [c.ids[2]]), q[2:], [2])
    assert all(bool((x == 0x55).all()) for x in others)
    c.close()


@pytest.mark.parametrize("dtype,dim", [(E.ELLM_BF16, 128), (E.ELLM_MXFP4, 64)])
def test_a_wait_that_gives_up_is_reported_and_stores_nothing(dtype, dim):
    """With no look at a flag every segment that has to wait leaves its rows alone; the pool says so until it is told to go on."""
    n, first = 9000, 5
    c = Cache([300, n, 40], 2, 2, dim, 100, dtype)
    rows = (64 << 10) // (2 * dim if dtype == E.ELLM_BF16 else dim // 2)        # of a segment
    assert n > 3 * rows
    q, dq = c.queries()
    keep = torch.arange(first + 1, n, dtype=torch.int32, device="cuda")
    E.ellm_debug_set_compact_looks(c.pool, 0)
    # a move of one segment waits for nothing
    E.ellm_kv_compact(c.pool, [c.ids[0]], keep=torch.arange(0, 300, 3, dtype=torch.int32, device="cuda"), n_keep=[100])
    c.k[0], c.v[0] = c.k[0][::3], c.v[0][::3]
    c.decode(dq)
    E.ellm_kv_compact(c.pool, [c.ids[1]], first=[first], keep=keep, n_keep=[len(keep)])
    torch.cuda.synchronize()
    lens = [E.ellm_tensor_get_table(c.pool, t)[1] for t in c.ids]
    assert lens == [100, n - 1, 40]
    out, rows_out = torch.empty_like(dq), torch.empty(100, 2, dim, dtype=torch.bfloat16, device="cuda")
    refused = [lambda: E.ellm_decode_attention(c.pool, c.ids, dq, out, check=False), lambda: E.ellm_decode_attention_noalloc(c.pool, c.ids, dq, out, check=False),
               lambda: E.ellm_kv_append(c.pool, c.ids, dq, dq, [1, 1, 1], check=False), lambda: E.ellm_kv_append_decode(c.pool, c.ids, dq, dq, dq, out, check=False),
               lambda: E.ellm_kv_read(c.pool, [c.ids[0]], rows_out, rows_out, check=False), lambda: E.ellm_kv_copy(c.pool, [c.ids[2]], [c.ids[0]], n_tokens=[1], check=False),
               lambda: E.ellm_kv_compact(c.pool, [c.ids[0]], keep=keep, n_keep=[1], check=False), lambda: E.ellm_pool_sync(c.pool, check=False)]
    for call in refused:
        assert call() == E.ERR.HIP and f"tensor {c.ids[1]} " in E.ellm_last_error()
    assert [E.ellm_tensor_get_table(c.pool, t)[1] for t in c.ids] == lens
    E.ellm_pool_reset_counters(c.pool)
    E.ellm_pool_sync(c.pool)
    # every row is the one that was to move there, or the one that was there: the first segment's all moved, the others' all not
    for got, held in zip(read(c, [c.ids[1]]), (c.k[1], c.v[1])):
        moved = first + rows
        assert np.array_equal(got, np.concatenate([held[:first], held[first + 1:moved + 1], held[moved:n - 1]]))
    # as good as new: lengths are cut, tokens appended, and the same move waits and moves
    E.ellm_debug_set_compact_looks(c.pool, -1)
    E.ellm_kv_compact(c.pool, [c.ids[1]])
    c.k[1], c.v[1] = c.k[1][:0], c.v[1][:0]
    c.append(*c.draw(n), [0, n, 0])
    E.ellm_kv_compact(c.pool, [c.ids[1]], first=[first], keep=keep, n_keep=[len(keep)])
    c.k[1], c.v[1] = (np.concatenate([x[1][:first], x[1][first + 1:]]) for x in (c.k, c.v))
    same(c)
    c.check(c.decode(dq), q)
    assert E.ellm_debug_set_compact_looks(c.pool, -2, check=False) == E.ERR.INVALID
    c.close()
