"""Pools of 4-bit rows on the GPU, through the C ABI: the bytes that appending writes, decode attention over them, plain and
fused, against the plain format and attention in 64 bits; what holds for every pool (bit equality of runs, of remapped chunks, of
the two entry points, of the fused call and the two it stands for, host round trips, graphs, streams)."""
import numpy as np
import pytest
import torch

import paper_2506_15155_amd as E
from tests import plain

pytestmark = pytest.mark.gpu

# What an output may be off, of the largest |value| of V that the head sees (weights sum to 1, so no output is larger): half a
# step for the result's rounding, 2^-8 of it; the weights are two bf16 values (to 2^-16); scores in 32 bits, 128 products at
# 2^-24 each of |q||k| / sqrt(D), which is under 60 here, and the exponential's 2^-23: under 2^-10 of a weight all together.
TOL = 2.0 ** -8 + 2.0 ** -10


def dev(b):
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).cuda()


def host(t):
    return t.cpu().numpy().view(np.uint16)


class Cache:
    """A pool over a poisoned buffer, tensors on scattered chunks, and beside them the values they hold."""

    def __init__(self, lens, n_kv, group, dim, tokens, dtype=E.ELLM_MXFP4, room=8, driver=False, host_chunks=0, seed=0, align=256):
        self.rng = np.random.default_rng(seed)
        self.n_kv, self.group, self.dim, self.fp4 = n_kv, group, dim, dtype == E.ELLM_MXFP4
        row = dim // 2 + dim // 32 if self.fp4 else 2 * dim
        self.chunk = -(-tokens * 2 * n_kv * row // align) * align
        self.T = plain.tokens_per_chunk(self.chunk, n_kv, dim, self.fp4)
        slots = [-(-(n + room) // self.T) for n in lens]
        self.n_chunks = sum(slots) + 3
        self.buf = self.pinned = None
        if host_chunks:
            self.pinned = torch.zeros(host_chunks * self.chunk, dtype=torch.uint8, pin_memory=True)
        shape = (self.chunk, n_kv * group, n_kv, dim, len(lens) + 2, max(slots) + 1)
        if driver:
            self.pool = E.ellm_pool_create(None, self.pinned, *shape, flags=E.ELLM_POOL_DRIVER_MAPPED, device_bytes=self.n_chunks * self.chunk, dtype=dtype)
        else:
            self.buf = torch.full((self.n_chunks, self.chunk), 0xFF, dtype=torch.uint8, device="cuda")      # scales of NaN
            self.pool = E.ellm_pool_create(self.buf, self.pinned, *shape, dtype=dtype)
        place = self.rng.permutation(self.n_chunks)
        self.ids, self.k, self.v = [], [], []
        for n, s in zip(lens, slots):
            t = E.ellm_tensor_create(self.pool, n + room)
            E.ellm_tensor_map_chunks(self.pool, t, 0, s, place[:s].astype(np.int32))
            place = place[s:]
            self.ids.append(t)
            self.k.append(np.zeros((0, n_kv, dim)))
            self.v.append(np.zeros((0, n_kv, dim)))
        if any(lens):
            self.append(*self.draw(sum(lens)), list(lens))

    def draw(self, n, spread=3):
        """K and V rows, bf16 values, of magnitudes that differ from block to block."""
        def one():
            x = self.rng.standard_normal((n, self.n_kv, self.dim // 32, 32)) * np.exp2(self.rng.integers(-spread, 2, (n, self.n_kv, self.dim // 32, 1)))
            return plain.bf16(x.reshape(n, self.n_kv, self.dim))
        return one(), one()

    def kept(self, x):
        return plain.held(*plain.quantise(x)) if self.fp4 else x

    def note(self, k, v, n_new):
        at = 0
        for b, n in enumerate(n_new):
            self.k[b] = np.concatenate([self.k[b], self.kept(k[at:at + n])])
            self.v[b] = np.concatenate([self.v[b], self.kept(v[at:at + n])])
            at += n

    def append(self, k, v, n_new):
        E.ellm_kv_append(self.pool, self.ids, dev(plain.bits(k)), dev(plain.bits(v)), np.array(n_new, np.int32))
        self.note(k, v, n_new)

    def queries(self):
        q = plain.bf16(self.rng.standard_normal((len(self.ids), self.n_kv * self.group, self.dim)))
        return q, dev(plain.bits(q))

    def decode(self, dq, ids=None, scale=0.0, call=E.ellm_decode_attention):
        out = torch.full_like(dq, 77)
        call(self.pool, self.ids if ids is None else ids, dq, out, scale)
        torch.cuda.synchronize()
        return out

    def check(self, out, q, which=None, scale=None):
        got = plain.values(host(out))
        for i, b in enumerate(range(len(self.ids)) if which is None else which):
            want = plain.attention(q[i], self.k[b], self.v[b], scale)
            top = np.repeat(np.abs(self.v[b]).max((0, 2)), self.group)[:, None]
            assert (np.abs(got[i] - want) <= TOL * top + 1e-30).all(), (b, np.abs(got[i] - want).max(), top.max())

    def close(self):
        torch.cuda.synchronize()
        E.ellm_pool_destroy(self.pool)


# kv heads, q heads of each, head size, tokens that a chunk is made for: groups that fill 4, 8 and 16 columns, that take two passes; chunks
# smaller than a unit, that end inside one, of whole units, larger than a request
SHAPES = [(8, 1, 64, 16), (2, 4, 128, 16), (1, 3, 128, 24), (2, 8, 128, 5), (2, 6, 64, 40), (1, 16, 128, 100), (2, 16, 64, 300),
          (8, 4, 128, 1920), (1, 20, 128, 33), (5, 2, 64, 64), (1, 64, 64, 48), (3, 5, 128, 257)]
LENS = [[1], [2, 15, 16, 17], [31, 32, 33, 1], [63, 64, 65, 200, 7], [129, 500, 1, 255, 256, 257], [1000, 3000]]


@pytest.mark.parametrize("driver", [False, True])
@pytest.mark.parametrize("n_kv,group,dim,tokens", SHAPES)
def test_append_and_decode(n_kv, group, dim, tokens, driver):
    for i, lens in enumerate(LENS):
        c = Cache(lens, n_kv, group, dim, tokens, driver=driver, seed=i, align=65536 if driver else 256)
        q, dq = c.queries()
        out = c.decode(dq)
        c.check(out, q)
        assert torch.equal(c.decode(dq), out)
        assert torch.equal(c.decode(dq, call=E.ellm_decode_attention_noalloc), out)
        c.close()


@pytest.mark.parametrize("n_kv,group,dim,tokens", [(2, 4, 128, 16), (1, 3, 64, 24), (8, 1, 128, 300)])
def test_bytes_of_the_cache(n_kv, group, dim, tokens):
    """Codes and scales where the header says, equal to the plain format's, whatever the appends' sizes; nothing else is written."""
    c = Cache([0, 0, 0], n_kv, group, dim, tokens, room=200)
    rows = [np.zeros((0, n_kv, 2, dim))] * 3
    for n_new in ([1, 40, 0], [31, 1, 3], [1, 1, 1], [64, 100, 17], [5, 0, 33]):
        k, v = c.draw(sum(n_new), spread=30)
        k[0, 0, :5] = [0.0, -0.0, 6.0, -5.0, 2.5]
        c.append(k, v, n_new)
        at = 0
        for b, n in enumerate(n_new):
            rows[b] = np.concatenate([rows[b], np.stack([k[at:at + n], v[at:at + n]], 2)])
            at += n
    torch.cuda.synchronize()
    buf = c.buf.cpu().numpy()
    untouched = np.ones(buf.shape, bool)
    for b, t in enumerate(c.ids):
        table, n = E.ellm_tensor_get_table(c.pool, t)
        assert n == len(rows[b])
        codes, scales = plain.quantise(rows[b])
        for s in range(-(-n // c.T)):
            m = min(c.T, n - s * c.T)
            got_c, got_s = plain.chunk_rows(buf[table[s]], n_kv, dim, c.T, True)
            assert np.array_equal(got_c[:m], codes[s * c.T:s * c.T + m]) and np.array_equal(got_s[:m], scales[s * c.T:s * c.T + m])
            end = n_kv * c.T * dim
            untouched[table[s]][:end].reshape(n_kv, 2, c.T, dim // 2)[:, :, :m] = False
            untouched[table[s]][end:end + 2 * n_kv * c.T * (dim // 32)].reshape(n_kv, 2, c.T, dim // 32)[:, :, :m] = False
    assert (buf[untouched] == 0xFF).all()
    c.close()


@pytest.mark.parametrize("dim", [64, 128])
def test_values_at_the_format_s_edges(dim):
    """The smallest and largest magnitudes, ties, and blocks with NaN or infinities, as codes and in attention."""
    c = Cache([0], 1, 2, dim, 16, room=64)
    n = 40
    rng = np.random.default_rng(3)
    k, v = np.zeros((n, 1, dim)), np.zeros((n, 1, dim))
    for i in range(n):
        ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]) * 2.0 ** rng.integers(-120, 120)
        v[i, 0] = rng.choice(ties, dim) * rng.choice([-1, 1], dim)
    v[0, 0], v[1, 0] = 2.0 ** -133, -3.3895313892515355e38             # the smallest and largest bf16 values
    v[2, 0] = 2.0 ** -126
    v[3, 0, :32] = np.nan
    v[4, 0, 3] = -np.inf
    c.append(k, v, [n])
    codes, scales = plain.quantise(v)
    table, _ = E.ellm_tensor_get_table(c.pool, c.ids[0])
    torch.cuda.synchronize()
    got = [plain.chunk_rows(c.buf[table[s]].cpu().numpy(), 1, dim, c.T, True) for s in range(-(-n // c.T))]
    assert np.array_equal(np.concatenate([x[0] for x in got])[:n, 0, 1], codes[:, 0])
    assert np.array_equal(np.concatenate([x[1] for x in got])[:n, 0, 1], scales[:, 0])
    q, dq = c.queries()
    out = plain.values(host(c.decode(dq)))
    # K is 0, so every weight is 1 / n: a NaN block makes its 32 dims of the result NaN, and no others
    assert np.isnan(out[0, :, :32]).all() and not np.isnan(out[0, :, 32:]).any()
    c.close()


@pytest.mark.parametrize("n_kv,group,dim", [(2, 4, 128), (2, 16, 64), (1, 1, 64)])
def test_a_key_that_is_nan_makes_its_head_nan(n_kv, group, dim):
    c = Cache([70], n_kv, group, dim, 16)
    k, v = c.draw(1)
    k[0, n_kv - 1, 5] = np.inf
    c.append(k, v, [1])
    q, dq = c.queries()
    out = plain.values(host(c.decode(dq)))[0].reshape(n_kv, group, dim)
    assert np.isnan(out[n_kv - 1]).all() and np.isfinite(out[:n_kv - 1]).all()
    c.close()


@pytest.mark.parametrize("driver", [False, True])
@pytest.mark.parametrize("n_kv,group,dim,tokens", [(2, 4, 128, 16), (1, 3, 64, 24), (8, 1, 128, 1920), (2, 16, 64, 100), (1, 20, 128, 40), (2, 12, 128, 64)])
def test_fused_step_equals_append_and_decode(n_kv, group, dim, tokens, driver):
    """Same bytes, lengths and output bits; requests that begin, cross units, chunks and tiles with the new token."""
    lens = [0, 1, 15, 16, 31, 63, 64, 127, 128, 255, 300, 511, 700, tokens - 1, tokens]
    a, b = (Cache(lens, n_kv, group, dim, tokens, driver=driver, seed=5, align=65536 if driver else 256) for _ in range(2))
    for step in range(3):
        k, v = a.draw(len(lens))
        q, dq = a.queries()
        out = torch.full_like(dq, 77)
        E.ellm_kv_append_decode(a.pool, a.ids, dev(plain.bits(k)), dev(plain.bits(v)), dq, out)
        a.note(k, v, [1] * len(lens))
        b.append(k, v, [1] * len(lens))
        want = b.decode(dq)
        assert torch.equal(out, want)
        a.check(out, q)
        if not driver:
            assert torch.equal(a.buf, b.buf)
        for x, y in zip(a.ids, b.ids):
            assert E.ellm_tensor_get_table(a.pool, x)[1] == E.ellm_tensor_get_table(b.pool, y)[1]
    a.close()
    b.close()


@pytest.mark.parametrize("dim", [64, 128])
def test_the_new_row_s_edges(dim):
    """The fused call quantises a row of its own: NaN, infinities, zeros and extreme magnitudes as the append does."""
    lens = [40] * 6
    a, b = (Cache(lens, 2, 4, dim, 24, seed=9) for _ in range(2))
    k, v = a.draw(6, spread=100)
    k[0], v[1], v[2, 1, 7], k[3] = 0, 0, np.nan, 3.3e38
    v[4], k[5, 0, dim - 1] = 2.0 ** -133, -np.inf
    k, v = plain.bf16(k), plain.bf16(v)
    q, dq = a.queries()
    out = torch.full_like(dq, 77)
    E.ellm_kv_append_decode(a.pool, a.ids, dev(plain.bits(k)), dev(plain.bits(v)), dq, out)
    b.append(k, v, [1] * 6)
    want = b.decode(dq)
    assert np.array_equal(host(out), host(want)) and torch.equal(a.buf, b.buf)
    a.close()
    b.close()


@pytest.mark.parametrize("n_kv,group,dim,tokens,lens", [
    (8, 4, 128, 512, [9000]), (8, 4, 128, 512, [3000] * 5), (1, 8, 128, 16, [40000, 3]), (2, 16, 64, 1000, [20000, 900, 1, 7000]),
    (4, 1, 128, 300, [2000] * 40), (2, 6, 64, 64, [300] * 130), (8, 4, 128, 100, [100 + 37 * i for i in range(70)]), (1, 33, 64, 48, [700] * 9),
    (8, 2, 128, 64, [1500 + i for i in range(24)])])
def test_large_launches(n_kv, group, dim, tokens, lens):
    """Requests shared by many waves and workgroups, shares that run over several requests, launches of two groups."""
    c = Cache(lens, n_kv, group, dim, tokens)
    q, dq = c.queries()
    out = c.decode(dq)
    some = sorted(set(range(0, len(lens), max(1, len(lens) // 6))) | {len(lens) - 1})
    c.check(out[some], q[some], some)
    assert torch.equal(c.decode(dq), out)
    # chunk by chunk on the driver's side of the same numbers of waves: other cuts agree to rounding
    for percent in (50, 300):
        E.ellm_debug_set_waves(c.pool, percent)
        c.check(c.decode(dq)[some], q[some], some)
    E.ellm_debug_set_waves(c.pool, 100)
    E.ellm_pool_set_split_tokens(c.pool, 192)
    c.check(c.decode(dq)[some], q[some], some)
    c.close()


def test_batches_of_two_groups_equal_two_calls():
    lens = [3 + (i * 37) % 400 for i in range(200)]
    c = Cache(lens, 4, 4, 128, 64)
    q, dq = c.queries()
    out = c.decode(dq)
    parts = [c.decode(dq[a:b].contiguous(), c.ids[a:b]) for a, b in ((0, 128), (128, 200))]
    assert torch.equal(out, torch.cat(parts))
    c.check(out[[0, 127, 128, 199]], q[[0, 127, 128, 199]], [0, 127, 128, 199])
    c.close()


def test_scale_and_large_scores():
    c = Cache([333, 17], 2, 4, 128, 64)
    q, dq = c.queries()
    for scale in (0.5, 1e-3, -0.25):
        c.check(c.decode(dq, scale=scale), q, scale=scale)
    c.close()


@pytest.mark.parametrize("n_kv,group,dim,tokens,lens", [(2, 4, 128, 64, [333, 17]), (1, 16, 64, 24, [333, 70]), (8, 4, 128, 512, [3000] * 5)])
def test_scores_of_any_size(n_kv, group, dim, tokens, lens):
    """Scores that differ by far more than 2^24: the result is the V row of the largest one. Scores that are all alike: the mean
    of V, of however large scores."""
    c = Cache(lens, n_kv, group, dim, tokens, room=40)
    q, dq = c.queries()
    for exponent in (16, 20, 23, 24, 26, 27, 30, 33, 60, 100):
        for sign in (1, -1):
            scale = sign * 1.37 * 2.0 ** exponent
            got = plain.values(host(c.decode(dq, scale=scale)))
            for i in range(len(lens)):
                for h in range(n_kv * group):
                    k, v = c.k[i][:, h // group], c.v[i][:, h // group]
                    s = k @ q[i, h] * sign
                    # (a score of 128 products in 32 bits is 2^-17 of the sum of their magnitudes off, which is under 1000; 0.02 * 2^16 is far
                    # more than any exponential needs)
                    near = v[s >= s.max() - 0.02]
                    tol = TOL * np.abs(v).max()
                    assert ((got[i, h] >= near.min(0) - tol) & (got[i, h] <= near.max(0) + tol)).all(), (scale, i, h)
    c.close()
    c = Cache([0] * len(lens), n_kv, group, dim, tokens, room=max(lens))
    k, v = c.draw(sum(lens))
    k[:] = k[0]
    c.append(k, v, lens)
    for exponent in (16, 20, 23, 24, 26, 27, 30, 33, 60, 100):
        for sign in (1, -1):
            c.check(c.decode(dq, scale=sign * 1.37 * 2.0 ** exponent), q, scale=0)
    c.close()


@pytest.mark.parametrize("n_kv,group,dim,tokens,lens", [(2, 4, 128, 64, [333, 17, 1]), (1, 16, 64, 24, [333, 70]), (8, 4, 128, 512, [3000] * 5), (1, 20, 128, 16, [100])])
def test_blocks_of_very_different_magnitudes(n_kv, group, dim, tokens, lens):
    """Each block of 32 dims of V has its result to the same part of its own largest value, whatever the others' are."""
    c = Cache([0] * len(lens), n_kv, group, dim, tokens, room=max(lens))
    k, v = c.draw(sum(lens))
    v *= np.repeat(2.0 ** c.rng.permutation([-90, 70, 0, -25])[:dim // 32], 32)
    c.append(k, plain.bf16(v), lens)
    q, dq = c.queries()
    got = plain.values(host(c.decode(dq)))
    for i in range(len(lens)):
        want = plain.attention(q[i], c.k[i], c.v[i])
        top = np.repeat(np.abs(c.v[i]).reshape(-1, n_kv, dim // 32, 32).max((0, 3)), group, 0)
        assert (np.abs(got[i] - want) <= TOL * np.repeat(top, 32, -1)).all(), i
    c.close()


def test_remapped_chunks_and_host_round_trips_keep_the_bits():
    lens = [100, 500, 33]
    a, b = Cache(lens, 2, 4, 128, 48, seed=1, host_chunks=16), Cache(lens, 2, 4, 128, 48, seed=1)
    q, dq = a.queries()
    want = a.decode(dq)
    for t in a.ids:
        table, n = E.ellm_tensor_get_table(a.pool, t)
        E.ellm_chunk_deflate_to_host(a.pool, t, 0, min(3, int((table >= 0).sum())))
    with pytest.raises(E.EllmError):
        a.decode(dq)
    for t in reversed(a.ids):
        table, n = E.ellm_tensor_get_table(a.pool, t)
        E.ellm_chunk_inflate_from_host(a.pool, t, 0, int((table <= -2).sum()))
    assert torch.equal(a.decode(dq), want)
    assert torch.equal(b.decode(dq), want)
    a.close()
    b.close()


def test_calls_on_changing_streams():
    c = Cache([200, 90], 2, 4, 128, 32, room=64)
    s = [torch.cuda.Stream() for _ in range(2)]
    for i in range(6):
        k, v = c.draw(2)
        dk, dv = dev(plain.bits(k)), dev(plain.bits(v))
        q, dq = c.queries()
        out = torch.full_like(dq, 77)
        torch.cuda.synchronize()
        E.ellm_kv_append(c.pool, c.ids, dk, dv, stream=s[i % 2])
        E.ellm_decode_attention(c.pool, c.ids, dq, out, stream=s[1 - i % 2])
        torch.cuda.synchronize()
        c.note(k, v, [1, 1])
        c.check(out, q)
    c.close()


def test_replays_of_a_captured_decode():
    lens = [50, 700, 3000, 9]
    c = Cache(lens, 2, 4, 128, 128, room=16)
    qs = [c.queries() for _ in range(4)]
    want = [c.decode(dq) for _, dq in qs]
    E.ellm_pool_prepare(c.pool)
    dq = qs[0][1].clone()
    out = torch.full_like(dq, 77)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        E.ellm_decode_attention_noalloc(c.pool, c.ids, dq, out)
    for i in (1, 2, 3, 0):
        dq.copy_(qs[i][1])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        c.decode(dq)
    c.close()


def test_offsets_past_32_bits():
    """A pool of 5 GB: the chunks of one request lie at both its ends."""
    n_kv, dim, cb = 2, 128, 1 << 20
    n = 5 << 10
    buf = torch.full((n, cb), 0xFF, dtype=torch.uint8, device="cuda")
    T = plain.tokens_per_chunk(cb, n_kv, dim, True)
    pool = E.ellm_pool_create(buf, None, cb, 8, n_kv, dim, 1, 3, dtype=E.ELLM_MXFP4)
    t = E.ellm_tensor_create(pool, 3 * T)
    E.ellm_tensor_map_chunks(pool, t, 0, 3, np.array([n - 1, 0, n - 2], np.int32))
    rng = np.random.default_rng(0)
    m = 2 * T + 100
    k, v = (plain.bf16(rng.standard_normal((m, n_kv, dim))) for _ in range(2))
    E.ellm_kv_append(pool, [t], dev(plain.bits(k)), dev(plain.bits(v)), [m])
    q = plain.bf16(rng.standard_normal((1, 8, dim)))
    dq = dev(plain.bits(q))
    out = torch.empty_like(dq)
    E.ellm_decode_attention(pool, [t], dq, out)
    got = plain.values(host(out))[0]
    kk, vv = plain.held(*plain.quantise(k)), plain.held(*plain.quantise(v))
    want = plain.attention(q[0], kk, vv)
    assert (np.abs(got - want) <= TOL * np.abs(vv).max()).all()
    E.ellm_pool_destroy(pool)


def test_chunk_stream_is_for_bf16_rows():
    c = Cache([20], 1, 1, 64, 16)
    sink = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert E.ellm_debug_kv_stream_read(c.pool, c.ids, sink, check=False) == E.ERR.INVALID
    assert E.ellm_debug_decode_kernel(c.pool, c.ids) == "decode_fp4_block_kernel"
    c.close()
