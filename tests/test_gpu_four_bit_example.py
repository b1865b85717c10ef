"""The example of a serving loop over a 4-bit cache: what its attention calls return is attention over the rows that the cache says
it holds, and the chunks are all free in the end."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2506_15155_amd as E
from tests import plain

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# half a step of the result's rounding, and the scores', weights' and sums' share, of the largest |value| of V
TOL = 2.0 ** -8 + 2.0 ** -10


def test_loop():
    spec = importlib.util.spec_from_file_location("four_bit_cache", os.path.join(ROOT, "examples", "four_bit_cache.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    lens = [300, 77, 420]
    loop = ex.Loop(lens, samples=3, budget=400, seed=5)
    (k, v), held = loop.prompt(lens)
    for x, y in zip((k, v), held):
        want = plain.held(*plain.quantise(x.cpu().double().numpy()))
        assert np.array_equal(y.cpu().double().numpy(), want)
    loop.fork()
    freed = 0
    for s in range(12):
        q, out = loop.step()
        n = loop.len[loop.forks]
        kk, vv = (torch.empty(int(n.sum()), ex.N_KV, ex.DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        E.ellm_kv_read(loop.pool, loop.handles(loop.forks), kk, vv)
        if s % 4 == 3:
            kk, vv, qq, got = (x.cpu().double().numpy() for x in (kk, vv, q, out))
            at = np.concatenate([[0], np.cumsum(n)])
            for i in range(len(n)):
                ki, vi = kk[at[i]:at[i + 1]], vv[at[i]:at[i + 1]]
                assert (np.abs(got[i] - plain.attention(qq[i], ki, vi)) <= TOL * np.abs(vi).max()).all()
        freed += loop.evict()
        for i in loop.forks:
            assert E.ellm_tensor_get_table(loop.pool, loop.ids[i])[1] == loop.len[i]
    assert freed > 0
    loop.end()
    assert loop.free() == loop.buf.shape[0] and E.ellm_pool_self_check(loop.pool) == 0
    loop.close()
