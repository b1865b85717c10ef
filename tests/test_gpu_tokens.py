"""Reading, copying and compacting tokens on the GPU, in pools of bf16 and of 4-bit rows: every value against a plain model
of the tensors, bit for bit; nothing outside them is touched."""
import numpy as np
import pytest
import torch

import paper_2506_15155_amd as E
from tests import plain
from tests.test_gpu_fp4 import Cache, dev, host

pytestmark = pytest.mark.gpu

KINDS = [(E.ELLM_MXFP4, 2, 128, 16), (E.ELLM_MXFP4, 3, 64, 24), (E.ELLM_MXFP4, 1, 128, 300), (E.ELLM_BF16, 2, 128, 24), (E.ELLM_BF16, 8, 64, 16),
         (E.ELLM_BF16, 1, 128, 200), (E.ELLM_MXFP4, 8, 128, 7)]


def read(c, ids, first=None, n_tokens=None):
    n = sum(n_tokens) if n_tokens is not None else sum(E.ellm_tensor_get_table(c.pool, t)[1] - (first[i] if first is not None else 0) for i, t in enumerate(ids))
    k, v = (torch.full((n, c.n_kv, c.dim), 77, dtype=torch.int16, device="cuda") for _ in range(2))
    E.ellm_kv_read(c.pool, ids, k, v, first=first, n_tokens=n_tokens)
    torch.cuda.synchronize()
    return plain.values(host(k)), plain.values(host(v))


def same(c):
    """Every tensor holds what the model says."""
    k, v = read(c, c.ids)
    assert np.array_equal(k, np.concatenate(c.k)) and np.array_equal(v, np.concatenate(c.v))


def outside(c):
    """The bytes of the pool that belong to no token."""
    torch.cuda.synchronize()
    buf = c.buf.cpu().numpy()
    mask = np.ones(buf.shape, bool)
    for t in c.ids:
        table, n = E.ellm_tensor_get_table(c.pool, t)
        for s in range(-(-n // c.T)):
            m = min(c.T, n - s * c.T)
            parts = [(0, 4 * c.n_kv * c.T * c.dim)]
            if c.fp4:
                end = c.n_kv * c.T * c.dim
                parts = [(0, end), (end, end + 2 * c.n_kv * c.T * (c.dim // 32))]
            for lo, hi in parts:
                mask[table[s]][lo:hi].reshape(c.n_kv, 2, c.T, -1)[:, :, :m] = False
    return buf[mask]


@pytest.mark.parametrize("driver", [False, True])
@pytest.mark.parametrize("dtype,n_kv,dim,tokens", KINDS)
def test_read(dtype, n_kv, dim, tokens, driver):
    lens = [1, 31, 32, 33, 200, 7, 1000]
    c = Cache(lens, n_kv, 2, dim, tokens, dtype, driver=driver, align=65536 if driver else 256)
    same(c)
    which = [4, 4, 0, 6, 1, 6]
    first, n = [3, 199, 1, 31, 0, 64], [100, 1, 0, 700, 31, 33]
    k, v = read(c, [c.ids[i] for i in which], first, n)
    for got, held in ((k, c.k), (v, c.v)):
        assert np.array_equal(got, np.concatenate([held[i][f:f + m] for i, f, m in zip(which, first, n)]))
    c.close()


def test_read_of_many_requests():
    c = Cache([5 + i % 60 for i in range(300)], 1, 1, 64, 16)
    same(c)
    c.close()


@pytest.mark.parametrize("driver", [False, True])
@pytest.mark.parametrize("dtype,n_kv,dim,tokens", KINDS)
def test_copy(dtype, n_kv, dim, tokens, driver):
    lens = [300, 0, 5, 0, 0, 129, 17, 0]
    c = Cache(lens, n_kv, 2, dim, tokens, dtype, room=600, driver=driver, align=65536 if driver else 256)
    for src, dst, first, n in (([0, 0, 0], [1, 2, 3], [0, 0, 0], [300, 300, 300]),       # one range, to tensors of other lengths
                               ([0, 5, 5, 0], [1, 2, 4, 6], [299, 0, 0, 7], [1, 129, 129, 33]),
                               ([6, 6], [7, 3], [0, 1], [1, 0]),
                               ([1], [7], [31], [65])):
        E.ellm_kv_copy(c.pool, [c.ids[i] for i in src], [c.ids[i] for i in dst], first=first, n_tokens=n)
        for i, j, f, m in zip(src, dst, first, n):
            c.k[j], c.v[j] = (np.concatenate([x[j], x[i][f:f + m]]) for x in (c.k, c.v))
        same(c)
        if not driver:
            assert (outside(c) == 0xFF).all()
    c.close()


def test_copy_of_whole_tensors_to_many():
    c = Cache([77] + [0] * 200, 2, 1, 64, 16, room=100)
    E.ellm_kv_copy(c.pool, [c.ids[0]] * 200, c.ids[1:])
    c.k[1:], c.v[1:] = [c.k[0]] * 200, [c.v[0]] * 200
    same(c)
    c.close()


@pytest.mark.parametrize("driver", [False, True])
@pytest.mark.parametrize("dtype,n_kv,dim,tokens", KINDS)
def test_compact(dtype, n_kv, dim, tokens, driver):
    lens = [1, 2, 64, 700, 3000, 33, 500, 257]
    c = Cache(lens, n_kv, 2, dim, tokens, dtype, driver=driver, align=65536 if driver else 256)
    rng = np.random.default_rng(8)
    for share in (1.0, 0.9, 0.5, 0.03):
        first = [int(rng.integers(0, len(k) + 1)) if i % 2 else 0 for i, k in enumerate(c.k)]
        lists = [f + np.sort(rng.permutation(len(k) - f)[:int(np.ceil(share * (len(k) - f)))]) for f, k in zip(first, c.k)]
        keep = torch.from_numpy(np.concatenate(lists).astype(np.int32)).cuda()
        E.ellm_kv_compact(c.pool, c.ids, first=first, keep=keep, n_keep=[len(x) for x in lists], flags=E.ELLM_COMPACT_UNMAP)
        for i, (f, x) in enumerate(zip(first, lists)):
            at = np.concatenate([np.arange(f), x]).astype(np.int64)
            c.k[i], c.v[i] = c.k[i][at], c.v[i][at]
        same(c)
        for t in c.ids:
            table, n = E.ellm_tensor_get_table(c.pool, t)
            assert int((table >= 0).sum()) == -(-n // c.T)
    c.close()


def test_compact_moves_nothing_else():
    """Chunks of other tensors and free ones keep their bytes."""
    c = Cache([400, 90, 256], 2, 2, 128, 32)
    torch.cuda.synchronize()
    before = c.buf.cpu().numpy().copy()
    mine = set(E.ellm_tensor_get_table(c.pool, c.ids[0])[0])
    keep = torch.arange(1, 400, 3, dtype=torch.int32, device="cuda")
    E.ellm_kv_compact(c.pool, [c.ids[0]], keep=keep, n_keep=[len(keep)])
    torch.cuda.synchronize()
    after = c.buf.cpu().numpy()
    others = [i for i in range(c.n_chunks) if i not in mine]
    assert np.array_equal(before[others], after[others])
    c.close()


def test_positions_that_break_the_rules_stay_inside():
    """Positions past the end, negative, out of order: no byte outside the tensor's tokens from `first` on changes."""
    c = Cache([300, 50], 2, 2, 64, 48, E.ELLM_BF16)
    torch.cuda.synchronize()
    before = c.buf.cpu().numpy().copy()
    bad = np.array([2**31 - 1, -2**31, 5, 299, 300, 100000, -1, 0, 250, 20] * 10, np.int32)
    E.ellm_kv_compact(c.pool, [c.ids[0]], first=[100], keep=torch.from_numpy(bad).cuda(), n_keep=[100])
    torch.cuda.synchronize()
    after = c.buf.cpu().numpy()
    table = E.ellm_tensor_get_table(c.pool, c.ids[0])[0]
    for s in range(c.n_chunks):
        old, new = (plain.chunk_rows(x[s], 2, 64, c.T, False) for x in (before, after))
        where = list(table).index(s) if s in table else -1
        for r in range(c.T):
            pos = where * c.T + r
            if where < 0 or pos < 100 or pos >= 200:
                assert np.array_equal(old[r], new[r]), (s, r)
    c.close()


def test_calls_behind_each_other_on_changing_streams():
    """Append, copy, compact, read of the same tensors, each on another stream than the one before."""
    c = Cache([100, 0], 2, 2, 128, 24, room=300)
    s = [torch.cuda.Stream() for _ in range(3)]
    keep = torch.arange(0, 100, 2, dtype=torch.int32, device="cuda")
    k, v = c.draw(30)
    dk, dv = dev(plain.bits(k)), dev(plain.bits(v))
    torch.cuda.synchronize()
    E.ellm_kv_copy(c.pool, [c.ids[0]], [c.ids[1]], stream=s[0])
    E.ellm_kv_compact(c.pool, [c.ids[0]], keep=keep, n_keep=[50], stream=s[1])
    E.ellm_kv_append(c.pool, c.ids, dk, dv, [10, 20], stream=s[2])
    E.ellm_kv_copy(c.pool, [c.ids[0]], [c.ids[1]], first=[40], stream=s[0])
    c.k[1], c.v[1] = c.k[0], c.v[0]
    c.k[0], c.v[0] = c.k[0][::2], c.v[0][::2]
    c.note(k, v, [10, 20])
    c.k[1], c.v[1] = (np.concatenate([x[1], x[0][40:]]) for x in (c.k, c.v))
    same(c)
    c.close()


def test_chunks_freed_by_a_compaction_are_offloaded_and_reused_in_order():
    """Chunks given back are written by whoever gets them next, behind the compaction that still reads them."""
    c = Cache([900, 40], 2, 2, 128, 32, host_chunks=4)
    keep = torch.arange(800, 900, dtype=torch.int32, device="cuda")
    E.ellm_kv_compact(c.pool, [c.ids[0]], keep=keep, n_keep=[100], flags=E.ELLM_COMPACT_UNMAP)
    E.ellm_chunk_deflate_to_host(c.pool, c.ids[1], 0, 2)
    E.ellm_chunk_inflate_from_host(c.pool, c.ids[1], 0, 2)         # into chunks that the compaction has just given back
    c.k[0], c.v[0] = c.k[0][800:], c.v[0][800:]
    same(c)
    assert E.ellm_pool_self_check(c.pool) == 0
    c.close()


def test_a_captured_copy_and_compaction():
    """Launches with fixed lengths can be replayed: the graph holds the lengths of the capture."""
    c = Cache([70, 0], 2, 2, 128, 32, room=200)
    E.ellm_pool_prepare(c.pool)
    keep = torch.arange(10, 70, 3, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        E.ellm_kv_copy(c.pool, [c.ids[0]], [c.ids[1]])
        E.ellm_kv_compact(c.pool, [c.ids[1]], keep=keep, n_keep=[20])
    c.k[1], c.v[1] = c.k[0][10::3], c.v[0][10::3]
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        same(c)
    c.close()


@pytest.mark.parametrize("dtype,n_kv,dim,lens,share", [
    (E.ELLM_BF16, 1, 128, [20000, 700, 9000], 0.8), (E.ELLM_BF16, 4, 64, [6000] * 40, 0.5), (E.ELLM_MXFP4, 2, 128, [30000, 40, 2000], 0.9),
    (E.ELLM_MXFP4, 1, 64, [60000, 5000], 0.3), (E.ELLM_BF16, 8, 128, [3000] * 20, 0.97), (E.ELLM_MXFP4, 8, 128, [1500] * 130, 0.7)])
def test_compactions_of_many_segments(dtype, n_kv, dim, lens, share):
    """Rows that move far and near, in chains of many segments whose stores wait for others' reads; three times in a row."""
    rng = np.random.default_rng(4)
    total = sum(lens)
    k, v = (torch.randn(total, n_kv, dim, device="cuda").to(torch.bfloat16) for _ in range(2))
    row = dim // 2 + dim // 32 if dtype == E.ELLM_MXFP4 else 2 * dim
    cb = -(-300 * 2 * n_kv * row // 256) * 256
    T = plain.tokens_per_chunk(cb, n_kv, dim, dtype == E.ELLM_MXFP4)
    slots = [-(-n // T) for n in lens]
    buf = torch.zeros(sum(slots), cb, dtype=torch.uint8, device="cuda")
    pool = E.ellm_pool_create(buf, None, cb, n_kv, n_kv, dim, len(lens), max(slots), dtype=dtype)
    place, ids = rng.permutation(sum(slots)).astype(np.int32), []
    for n, s in zip(lens, slots):
        ids.append(E.ellm_tensor_create(pool, n))
        E.ellm_tensor_map_chunks(pool, ids[-1], 0, s, place[:s])
        place = place[s:]
    E.ellm_kv_append(pool, ids, k, v, lens)
    want = []
    for x in (k, v):
        out = torch.empty_like(x)
        want.append(out)
    E.ellm_kv_read(pool, ids, *want)
    n = list(lens)
    for turn in range(3):
        # scattered positions; all but some at the beginning; the last ones
        keep = [np.sort(rng.permutation(m)[:max(1, int(m * share))]) if turn == 0 else np.arange(min(m - 1, 5 + m // 10), m) if turn == 1 else
                np.concatenate([np.arange(m // 3), np.arange(m - m // 3, m)]) if m > 3 else np.arange(1) for m in n]
        at = np.concatenate([b + x for b, x in zip(np.concatenate([[0], np.cumsum(n)[:-1]]), keep)])
        want = [x[torch.from_numpy(at).cuda()] for x in want]
        n = [len(x) for x in keep]
        E.ellm_kv_compact(pool, ids, keep=torch.from_numpy(np.concatenate(keep).astype(np.int32)).cuda(), n_keep=n)
        got = [torch.empty_like(x) for x in want]
        E.ellm_kv_read(pool, ids, *got)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    torch.cuda.synchronize()
    E.ellm_pool_destroy(pool)


def test_a_compaction_without_room_for_flags():
    """Chains of so many segments that the workspace has no room for a flag each go one segment after the other."""
    n_kv, dim, n = 16, 64, 1100000
    cb = 1 << 21
    T = plain.tokens_per_chunk(cb, n_kv, dim, False)
    slots = -(-n // T)
    buf = torch.empty(slots, cb, dtype=torch.uint8, device="cuda")
    pool = E.ellm_pool_create(buf, None, cb, n_kv, n_kv, dim, 1, slots)
    marks = E.ellm_workspace_bytes(n_kv, n_kv, dim, 1) // 4
    assert 2 * n_kv * (16 + (n - 1) // 512) > marks
    t = E.ellm_tensor_create(pool, n)
    E.ellm_tensor_map_chunks(pool, t, 0, slots)
    k, v = (torch.randn(n, n_kv, dim, device="cuda", dtype=torch.float16).view(torch.bfloat16) for _ in range(2))
    E.ellm_kv_append(pool, [t], k, v, [n])
    keep = torch.arange(1, n, dtype=torch.int32, device="cuda")
    E.ellm_kv_compact(pool, [t], keep=keep, n_keep=[n - 1])
    got = [torch.empty_like(k[1:]) for _ in range(2)]
    E.ellm_kv_read(pool, [t], *got)
    assert torch.equal(got[0].view(torch.int16), k[1:].view(torch.int16)) and torch.equal(got[1].view(torch.int16), v[1:].view(torch.int16))
    torch.cuda.synchronize()
    E.ellm_pool_destroy(pool)


def test_decode_after_a_compaction_in_its_workspace():
    """Both use the workspace of partial results, one behind the other."""
    c = Cache([5000, 300], 2, 4, 128, 64)
    q, dq = c.queries()
    for step in range(3):
        m = [len(x) for x in c.k]
        keep = [np.arange(0, x) for x in m]
        keep[0] = np.delete(keep[0], 7)
        E.ellm_kv_compact(c.pool, c.ids, keep=torch.from_numpy(np.concatenate(keep).astype(np.int32)).cuda(), n_keep=[len(x) for x in keep])
        c.k[0], c.v[0] = c.k[0][keep[0]], c.v[0][keep[0]]
        c.check(c.decode(dq), q)
    c.close()
