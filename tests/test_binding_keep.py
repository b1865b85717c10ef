"""The list of kept positions is read by the GPU: a host array, which the counts beside it are, is refused."""
import numpy as np
import pytest
import torch  # noqa: F401  (ahead of the package: both then use one HIP runtime, which the tests after this one need)

import paper_2506_15155_amd as E


@pytest.mark.parametrize("ids_as", [list, lambda x: np.array(x, np.int32)])
def test_host_arrays_of_positions_are_refused(ids_as):
    p = E.ellm_pool_create(None, None, 4096, 2, 2, 64, 2, 8, flags=E.ELLM_POOL_METADATA_ONLY, device_bytes=16 * 4096)
    t = E.ellm_tensor_create(p, 40)
    E.ellm_tensor_map_chunks(p, t, 0, 5)
    E.ellm_kv_append(p, [t], 16, 16, [30])
    n = np.array([3], np.int64)
    for dtype in (np.int32, np.int64):
        with pytest.raises(ValueError, match="device"):
            E.ellm_kv_compact(p, ids_as([t]), keep=np.arange(3, dtype=dtype), n_keep=n)
    assert E.ellm_tensor_get_table(p, t)[1] == 30
    E.ellm_kv_compact(p, ids_as([t]), keep=0x1000, n_keep=n)
    assert E.ellm_tensor_get_table(p, t)[1] == 3
    E.ellm_pool_destroy(p)
