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
