"""Plans of decode launches over 4-bit rows: pools without a device cut a batch as an MI355X does, two waves for every SIMD where the
kernel has room for them."""
import numpy as np
import pytest
import torch

import paper_2506_15155_amd as E


def lengths(p, lens):
    """A pool's tensors of these lengths (their rows, if there is a device, are whatever its memory holds)."""
    T = E.ellm_pool_get_geometry(p)["tokens_per_chunk"]
    ids = []
    for n in lens:
        ids.append(E.ellm_tensor_create(p, n))
        E.ellm_tensor_map_chunks(p, ids[-1], 0, -(-n // T))
    return ids


def without_device(n_kv, group, dim, lens, tokens=2048):
    cb = tokens * 2 * n_kv * (dim // 2 + dim // 32)
    slots = [-(-n // tokens) for n in lens]
    p = E.ellm_pool_create(None, None, cb, n_kv * group, n_kv, dim, len(lens), max(slots), flags=E.ELLM_POOL_METADATA_ONLY, device_bytes=sum(slots) * cb,
                           dtype=E.ELLM_MXFP4)
    ids = lengths(p, lens)
    E.ellm_kv_append(p, ids, 16, 16, np.array(lens, np.int32))
    return p, ids


# kv heads, q heads of each, head size, waves of a SIMD: up to 16 heads of 64 and 8 of 128 two workgroups have room in LDS
SHAPES = [(8, 1, 128, 2), (8, 4, 128, 2), (1, 8, 128, 2), (2, 9, 128, 1), (4, 16, 128, 1), (2, 17, 128, 1), (1, 64, 64, 1), (2, 16, 64, 2), (4, 5, 64, 2)]


@pytest.mark.parametrize("n_kv,group,dim,waves", SHAPES)
def test_waves_of_a_launch(n_kv, group, dim, waves):
    p, ids = without_device(n_kv, group, dim, [100000])
    assert E.ellm_decode_plan(p, ids)[0].tolist() == [1024 * waves // n_kv]
    E.ellm_debug_set_compute_units(p, 64)
    assert E.ellm_decode_plan(p, ids)[0].tolist() == [256 * waves // n_kv]
    E.ellm_debug_set_compute_units(p, 0)
    assert E.ellm_decode_plan(p, ids)[0].tolist() == [1024 * waves // n_kv]
    E.ellm_pool_destroy(p)


@pytest.mark.gpu
@pytest.mark.parametrize("n_kv,group,dim,waves", SHAPES)
def test_plans_with_and_without_a_device_are_the_same(n_kv, group, dim, waves):
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("not a whole MI355X")
    for lens in ([100000], [5, 300, 20, 4096], [3000] * 20, [40 + 100 * i for i in range(100)]):
        p, ids = without_device(n_kv, group, dim, lens)
        want = E.ellm_decode_plan(p, ids)
        cb = 2048 * 2 * n_kv * (dim // 2 + dim // 32)
        slots = [-(-n // 2048) for n in lens]
        buf = torch.zeros(sum(slots), cb, dtype=torch.uint8, device="cuda")
        d = E.ellm_pool_create(buf, None, cb, n_kv * group, n_kv, dim, len(lens), max(slots), dtype=E.ELLM_MXFP4)
        on_device = lengths(d, lens)
        rows = torch.zeros(sum(lens), n_kv, dim, dtype=torch.bfloat16, device="cuda")
        E.ellm_kv_append(d, on_device, rows, rows, np.array(lens, np.int32))
        got = E.ellm_decode_plan(d, on_device)
        assert got[0].tolist() == want[0].tolist() and got[1] == want[1]
        assert E.ellm_debug_decode_kernel(d, on_device) == E.ellm_debug_decode_kernel(p, ids)
        torch.cuda.synchronize()
        E.ellm_pool_destroy(d)
        E.ellm_pool_destroy(p)
