"""The operators around a 4-bit cache and the pages of a cache, as cases that can be timed and compared:

  decode   one layer's decode attention over a batch of requests whose K and V are held in 4 bits;
  step     the decode iteration of several layers: new rows quantised and written, attention over all, in one
           call per layer; the rows that the cache now holds are read back, and the tokens dropped again (a
           draft that was not accepted);
  append   new tokens' K and V rows are quantised into the cache, and read back as the dense rows that a prompt's
           own attention takes; the requests then end;
  copy     requests are forked: each source's tokens become the beginning of several other tensors;
  compact  tokens are evicted: the kept ones move together, and new ones are appended behind them (or, "accept",
           drafts are appended, the accepted ones kept and the rest dropped).

A cache in 4 bits holds blocks of 32 dims of a row: an 8-bit power of two s, the smallest one with max |x| <= 6 s, and
for every dim the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 times s with a sign (ties to the even code). The values of cases
are normal with a magnitude of its own for every channel, as K has it; chunks are scattered over the pool.

The plain form works on the same chunks, through the same table, with elementary operations in 32 bits.
"""
from __future__ import annotations

import math
import sys

import numpy as np
import torch

own = False
MIB = 1 << 20
PIECE = 1 << 18            # tokens whose rows are generated at a time


def listed():
    return [
        # the smallest call: four short requests of a small MHA model, 16-token chunks, where allocating is not allowed
        _case("decode_tiny", "decode", batch=4, n_kv=8, group=1, dim=64, chunk_tokens=16, dist="uniform", lo=16, hi=256, entry="noalloc"),
        # one user's request, interactive: an 8B-shaped layer over a few thousand tokens
        _case("decode_one", "decode", batch=1, n_kv=8, group=4, dim=128, dist="uniform", lo=3000, hi=3500),
        # the serving batch: 64 requests with long-tailed lengths
        _case("decode_8b", "decode", batch=64, n_kv=8, group=4, dim=128, dist="lognormal", lo=64, hi=8192),
        # few kv heads of 64 shared by 16 q heads each
        _case("decode_g16", "decode", batch=64, n_kv=2, group=16, dim=64, dist="uniform", lo=512, hi=24576),
        # a 70B-shaped layer over long contexts: the largest call
        _case("decode_long", "decode", batch=16, n_kv=8, group=8, dim=128, dist="uniform", lo=32768, hi=131072),
        # the whole decode iteration, 4 layers of the 8B shape
        _case("step_8b", "step", batch=64, n_kv=8, group=4, dim=128, dist="lognormal", lo=64, hi=8192, layers=4),
        # prompts of four new requests
        _case("append_prompt", "append", batch=4, n_kv=8, group=4, dim=128, dist="uniform", lo=4096, hi=32768),
        # one token for each request of a batch
        _case("append_token", "append", batch=64, n_kv=8, group=4, dim=128, dist="lognormal", lo=64, hi=8192, new=1),
        # four prompts, each sampled from four times, in a bf16 cache
        _case("fork_beams", "copy", batch=4, n_kv=8, group=4, dim=128, dist="uniform", lo=2000, hi=8192, copies=4, dtype="bf16"),
        # one short prompt forked for eight samples in a 4-bit cache of small chunks, and read back
        _case("fork_small", "copy", batch=1, n_kv=8, group=4, dim=128, chunk_tokens=64, dist="uniform", lo=200, hi=300, copies=8),
        # eviction from a bf16 cache: four fifths of every request's tokens are kept, new ones take the others' place
        _case("compact_evict", "compact", batch=8, n_kv=8, group=4, dim=128, dist="uniform", lo=4096, hi=16384, keep=80, dtype="bf16"),
        # speculative decoding over a 4-bit cache: of 8 drafts for every request 3 are accepted
        _case("compact_accept", "compact", batch=64, n_kv=8, group=4, dim=128, dist="lognormal", lo=64, hi=8192, new=8, keep=38, entry="accept"),
    ]


def _case(name, kind, batch, n_kv, group, dim, dist, lo, hi, chunk_tokens=0, layers=1, new=0, copies=0, keep=0, dtype="mxfp4", pool="table",
          entry="plain", lens_seed=1):
    c = {"kind": kind, "batch": batch, "n_kv": n_kv, "group": group, "dim": dim, "chunk_tokens": chunk_tokens, "dist": dist, "lo": lo,
         "hi": hi, "layers": layers, "new": new, "copies": copies, "keep": keep, "dtype": dtype, "pool": pool, "entry": entry,
         "lens_seed": lens_seed}
    return {"name": name, **c} if name else c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges: every size at random, odd ones included."""
    kind = rng.choice(["decode"] * 5 + ["step", "append", "append", "copy", "copy", "compact", "compact"])
    dim = rng.choice([64, 128, 128])
    n_kv, group = rng.choice([1, 2, 4, 5, 8, 8, 8, 10, 16, 40]), rng.choice([1, 1, 2, 3, 4, 4, 5, 6, 7, 8, 8, 12, 16, 20])
    if n_kv * group > 128:
        group = 128 // n_kv
    dtype = "mxfp4" if kind in ("decode", "step", "append") else rng.choice(["mxfp4", "bf16"])
    chunk_tokens = rng.choice([0, 0, 0, 16, 24, 40, 64, 100, 128, 333])
    most = {"decode": 512 << 20, "step": 48 << 20, "append": 96 << 20, "copy": 64 << 20, "compact": 128 << 20}[kind]    # values of K and V
    while True:
        batch = _log(rng, 1, {"decode": 200, "step": 80, "append": 100, "copy": 8, "compact": 80}[kind])
        mean = _log(rng, 16 if kind == "decode" else 40, 65536 if kind == "decode" else 8192)
        if batch * mean * n_kv * dim * 2 <= most and (not chunk_tokens or mean <= 8192):
            break
    dist = rng.choice(["uniform", "lognormal"])
    lo, hi = (max(1, mean // 3), mean * 5 // 3) if dist == "uniform" else (max(1, mean // 4), mean * 3)
    pool = "driver" if kind == "decode" and not chunk_tokens and rng.random() < 0.25 else "table"
    partials = (1024 + n_kv * (min(batch, 128) - 1)) * group * (dim + 2) * 4
    entry = "noalloc" if kind == "decode" and partials <= 16 * MIB and rng.random() < 0.2 else "plain"
    new = rng.choice([0, 1, 1, 5, 64]) if kind == "append" else 0
    keep = rng.choice([10, 25, 50, 80, 95]) if kind == "compact" else 0
    if kind == "compact" and rng.random() < 0.4:
        entry, new, keep = "accept", rng.choice([4, 7, 8, 16]), rng.choice([10, 30, 60])
    return _case("", kind, batch, n_kv, group, dim, dist, lo, hi, chunk_tokens, rng.choice([2, 3]) if kind == "step" else 1, new,
                 rng.choice([1, 2, 3, 5]) if kind == "copy" else 0, keep, dtype, pool, entry, rng.randrange(1 << 20))


# ---- shapes -----------------------------------------------------------------------------------------
def _lens(case):
    """Context lengths of the batch (append with all tokens new: of the prompts)."""
    rng = np.random.default_rng(case["lens_seed"])
    lo, hi, n = case["lo"], case["hi"], case["batch"]
    if case["dist"] == "uniform":
        return rng.integers(lo, hi + 1, size=n).astype(np.int64)
    return np.clip(np.rint(np.exp(math.log(math.sqrt(lo * hi)) + rng.standard_normal(n))), lo, hi).astype(np.int64)


def _bytes_per_token(case):
    return 2 * case["n_kv"] * (case["dim"] // 2 + case["dim"] // 32 if case["dtype"] == "mxfp4" else case["dim"] * 2)


def _chunk(case):
    """(tokens per chunk, bytes of a chunk)"""
    bpt = _bytes_per_token(case)
    size = -(-case["chunk_tokens"] * bpt // 256) * 256 if case["chunk_tokens"] else 2 * MIB
    tokens = size // bpt
    return (tokens // 16 * 16 if case["dtype"] == "mxfp4" and tokens >= 256 else tokens), size


def _kept(case):
    """compact: (tokens before the kept ones, tokens to choose from, kept) of every request."""
    lens = _lens(case)
    if case["entry"] == "accept":
        n = np.full_like(lens, case["new"])
        return lens, n, np.minimum(n, np.maximum(1, n * case["keep"] // 100))
    first = np.minimum(4, lens)                     # the first few tokens always stay
    return first, lens - first, (lens - first) * case["keep"] // 100


# ---- values -----------------------------------------------------------------------------------------
def _gen(seed, *what):
    g = torch.Generator(device="cuda")
    s = seed & 0xFFFFFFFF
    for w in what:
        s = (s * 1000003 + w + 1) & 0x7FFFFFFFFFFF
    return g.manual_seed(s)


def _rows(case, g, n):
    """K and V rows of n tokens."""
    shape = (n, case["n_kv"], case["dim"])
    channel = torch.exp(0.5 * torch.randn(shape[1:], generator=g, device="cuda"))
    k = (torch.randn(shape, generator=g, device="cuda") * channel).to(torch.bfloat16)
    return k, torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _history(case, seed, lens):
    """The K and V rows that are in the cache before the pass, some requests at a time: (first, end, k, v)."""
    b = 0
    while b < len(lens):
        e, n = b + 1, int(lens[b])
        while e < len(lens) and n + int(lens[e]) <= PIECE:
            n += int(lens[e])
            e += 1
        yield (b, e, *_rows(case, _gen(seed, 1, b), n))
        b = e


def _queries(case, seed, rows):
    return torch.randn(rows, case["n_kv"] * case["group"], case["dim"], generator=_gen(seed, 2), device="cuda").to(torch.bfloat16)


def _keep_lists(case, seed):
    """Positions of the kept tokens, in ascending order, request after request."""
    rng = np.random.default_rng(seed + 5)
    first, n, kept = _kept(case)
    return np.concatenate([f + np.sort(rng.permutation(m)[:k]) for f, m, k in zip(first, n, kept)]).astype(np.int32)


# ---- what a program keeps ---------------------------------------------------------------------------
class _State:
    """The cache: chunks, a table, the tensors' lengths; the pool's handle; the buffers of the loop around it."""

    pool = None

    def __init__(self, case, seed, lens, room):
        """lens: tokens of each tensor that are there before the pass; room: most tokens it will hold"""
        self.case, self.len = case, lens.copy()
        self.tokens, self.chunk = _chunk(case)
        need = -(-room // self.tokens)
        place = np.random.default_rng(seed).permutation(int(need.sum()) + 2)
        ends = np.cumsum(need)
        self.table_host = np.zeros((len(lens), int(need.max())), np.int64)
        for b in range(len(lens)):
            self.table_host[b, :need[b]] = place[ends[b] - need[b]:ends[b]]
        self.n_chunks, self.room, self.need = len(place), room, need
        self.buf = torch.zeros(self.n_chunks, self.chunk, dtype=torch.uint8, device="cuda") if case["pool"] == "table" or not own else None
        self.table = torch.from_numpy(self.table_host).cuda()
        if own:
            self._open()

    def _open(self):
        import paper_2506_15155_amd as E
        self.E, case = E, self.case
        dtype = E.ELLM_MXFP4 if case["dtype"] == "mxfp4" else E.ELLM_BF16
        shape = (self.chunk, case["n_kv"] * case["group"], case["n_kv"], case["dim"], len(self.len), int(self.need.max()))
        if self.buf is None:
            self.pool = E.ellm_pool_create(None, None, *shape, flags=E.ELLM_POOL_DRIVER_MAPPED, device_bytes=self.n_chunks * self.chunk, dtype=dtype)
        else:
            self.pool = E.ellm_pool_create(self.buf, None, *shape, dtype=dtype)
        self.ids = np.empty(len(self.len), np.int32)
        for b in range(len(self.len)):
            self.ids[b] = E.ellm_tensor_create(self.pool, int(self.room[b]))
            E.ellm_tensor_map_chunks(self.pool, int(self.ids[b]), 0, int(self.need[b]), self.table_host[b, :self.need[b]].astype(np.int32))

    def fill(self, b, e, k, v):
        """Tensors b .. e - 1 get their first tokens."""
        if own:
            self.E.ellm_kv_append(self.pool, self.ids[b:e], k, v, self.len[b:e].astype(np.int32))
        else:
            _write(self, *_each(torch.arange(b, e, device="cuda"), torch.zeros(e - b, dtype=torch.int64, device="cuda"),
                                torch.from_numpy(self.len[b:e]).cuda()), k, v)

    def __del__(self):
        if self.pool is not None and not sys.is_finalizing():
            torch.cuda.synchronize()
            self.E.ellm_pool_destroy(self.pool)
            self.pool = None


def prepare(case, seed):
    kind, lens, B = case["kind"], _lens(case), case["batch"]
    lens = np.tile(lens, case["layers"])
    before, room = lens, lens
    if kind == "step":
        room = lens + 1
    elif kind == "append":
        before, room = (lens, lens + case["new"]) if case["new"] else (np.zeros_like(lens), lens)
    elif kind == "copy":
        before, room = np.concatenate([lens, np.zeros(B * case["copies"], np.int64)]), np.concatenate([lens, np.repeat(lens, case["copies"])])
    elif kind == "compact" and case["entry"] == "accept":
        room = lens + case["new"]
    st = _State(case, seed, before, room)
    n_full = B if kind == "copy" else 0 if kind == "append" and not case["new"] else len(before)
    for b, e, k, v in _history(case, seed, before[:n_full]):
        st.fill(b, e, k, v)
    if kind in ("decode", "step"):
        st.q = _queries(case, seed, len(lens))
        st.out = torch.empty_like(st.q)
    st.new = {"step": np.ones_like(lens), "append": np.full_like(lens, case["new"]) if case["new"] else lens}.get(kind)
    if kind == "compact":
        st.first, choice, st.n_keep = _kept(case)
        st.keep = torch.from_numpy(_keep_lists(case, seed)).cuda()
        st.new = choice if case["entry"] == "accept" else choice - st.n_keep
    if st.new is not None:
        st.k_new, st.v_new = _rows(case, _gen(seed, 3), int(st.new.sum()))
    if kind == "copy":
        st.src = np.repeat(np.arange(B), case["copies"]).astype(np.int64)
        st.dst = np.arange(B, B + B * case["copies"]).astype(np.int64)
    read = {"step": st.new, "append": st.new, "copy": lens[st.src] if kind == "copy" else None, "compact": getattr(st, "n_keep", None)}.get(kind)
    if read is not None and case["dtype"] == "mxfp4" and (kind != "compact" or case["entry"] == "accept"):
        st.k_out, st.v_out = (torch.empty(int(read.sum()), case["n_kv"], case["dim"], dtype=torch.bfloat16, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    return st


# ---- a pass -----------------------------------------------------------------------------------------
def run(st):
    return (_OWN if own else _PLAIN)[st.case["kind"]](st)


def _values(st):
    """What the whole cache holds: a bf16 one as it lies there, of one in 4 bits the values of all tokens."""
    if st.case["dtype"] == "bf16":
        return [st.buf.view(torch.bfloat16)]
    return _read_all(st) if own else _read(st, *_all_tokens(st))


def _read_all(st):
    n = int(st.len.sum())
    k, v = (torch.empty(n, st.case["n_kv"], st.case["dim"], dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st.E.ellm_kv_read(st.pool, st.ids, k, v)
    return [k, v]


def _own_decode(st):
    call = st.E.ellm_decode_attention_noalloc if st.case["entry"] == "noalloc" else st.E.ellm_decode_attention
    call(st.pool, st.ids, st.q, st.out)
    return [st.out]


def _own_step(st):
    E, B = st.E, st.case["batch"]
    for i in range(0, len(st.ids), B):
        E.ellm_kv_append_decode(st.pool, st.ids[i:i + B], st.k_new[i:i + B], st.v_new[i:i + B], st.q[i:i + B], st.out[i:i + B])
    E.ellm_kv_read(st.pool, st.ids, st.k_out, st.v_out, first=st.len)
    E.ellm_kv_compact(st.pool, st.ids, first=st.len)
    return [st.out, st.k_out, st.v_out]


def _own_append(st):
    E = st.E
    E.ellm_kv_append(st.pool, st.ids, st.k_new, st.v_new, st.new.astype(np.int32))
    E.ellm_kv_read(st.pool, st.ids, st.k_out, st.v_out, first=st.len)
    E.ellm_kv_compact(st.pool, st.ids, first=st.len)
    return [st.k_out, st.v_out]


def _own_copy(st):
    E = st.E
    dst = st.ids[st.dst]
    E.ellm_kv_copy(st.pool, st.ids[st.src], dst)
    if st.case["dtype"] == "mxfp4":
        E.ellm_kv_read(st.pool, dst, st.k_out, st.v_out)
    E.ellm_kv_compact(st.pool, dst)
    return [st.k_out, st.v_out] if st.case["dtype"] == "mxfp4" else _values(st)


def _own_compact(st):
    E, new = st.E, st.new.astype(np.int32)
    if st.case["entry"] == "accept":
        E.ellm_kv_append(st.pool, st.ids, st.k_new, st.v_new, new)
        E.ellm_kv_compact(st.pool, st.ids, first=st.first, keep=st.keep, n_keep=st.n_keep)
        if st.case["dtype"] == "mxfp4":
            E.ellm_kv_read(st.pool, st.ids, st.k_out, st.v_out, first=st.first)
        E.ellm_kv_compact(st.pool, st.ids, first=st.len)
        return [st.k_out, st.v_out] if st.case["dtype"] == "mxfp4" else _values(st)
    E.ellm_kv_compact(st.pool, st.ids, first=st.first, keep=st.keep, n_keep=st.n_keep)
    E.ellm_kv_append(st.pool, st.ids, st.k_new, st.v_new, new)
    return _values(st)


_OWN = {"decode": _own_decode, "step": _own_step, "append": _own_append, "copy": _own_copy, "compact": _own_compact}


# ---- the plain form ---------------------------------------------------------------------------------
def _each(which, first, n):
    """Tensor and position of tokens first[i] .. first[i] + n[i] - 1 of tensors which[i], one after the other."""
    b = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n)
    t = torch.arange(len(b), device="cuda") - torch.repeat_interleave(torch.cumsum(n, 0) - n, n)
    return which[b], first[b] + t


def _all_tokens(st):
    n = torch.from_numpy(st.len).cuda()
    return _each(torch.arange(len(n), device="cuda"), torch.zeros_like(n), n)


def _planes(st):
    """The chunks as [chunk][kv head][K, V][row][..]: the rows (4 bits: two dims a byte), and the scales of 4-bit ones."""
    H, D, T = st.case["n_kv"], st.case["dim"], st.tokens
    if st.case["dtype"] == "bf16":
        return st.buf.view(torch.bfloat16)[:, :2 * H * T * D].unflatten(1, (H, 2, T, D)), None
    end = H * T * D
    return st.buf[:, :end].unflatten(1, (H, 2, T, D // 2)), st.buf[:, end:end + 2 * H * T * (D // 32)].unflatten(1, (H, 2, T, D // 32))


def _quantised(x):
    """[..][D] -> bytes of two codes [..][D / 2], scales [..][D / 32]"""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    finite = torch.isfinite(top)
    top = torch.where(finite, top, 0)
    # the exponent of the smallest power of two that max |x| is at most 6 times of: max |x| = m 2^e, 1 <= m < 2, and 6 = 1.5 * 4
    bits = top.view(torch.int32)
    e = ((bits + 0x3FFFFF) >> 23) - 2
    e = e.clamp(0, 252)
    # (multiplied by the power's inverse in two halves: either is a normal number)
    half = (127 - e) >> 1
    power = lambda n: ((n + 127) << 23).view(torch.float32)  # noqa: E731
    y = (x * power(half)[..., None] * power(127 - e - half)[..., None]).abs()
    code = (y > .25).to(torch.uint8) + (y >= .75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)
    code = torch.where(finite[..., None], code + 8 * torch.signbit(x), 0).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, torch.where(finite, e, 255).to(torch.uint8)


def _held(codes, scales):
    """The values that codes and scales stand for."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    s = scales.int()
    s = torch.where(s == 0, 1 << 22, s << 23).view(torch.float32)
    s = torch.where(scales == 255, math.nan, s)
    return (grid[c.int()].unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def _at(st, b, t):
    return st.table[b, t // st.tokens], t % st.tokens


def _write(st, b, t, k, v):
    """New rows to tokens t of tensors b."""
    chunk, row = _at(st, b, t)
    rows, scales = _planes(st)
    x = torch.stack([k, v], 2)                        # [token][kv head][K, V][dim]
    if scales is None:
        rows[chunk, :, :, row] = x
    else:
        rows[chunk, :, :, row], scales[chunk, :, :, row] = _quantised(x)


def _read(st, b, t):
    chunk, row = _at(st, b, t)
    rows, scales = _planes(st)
    x = rows[chunk, :, :, row]
    x = x if scales is None else _held(x, scales[chunk, :, :, row]).to(torch.bfloat16)
    return [x[:, :, 0].contiguous(), x[:, :, 1].contiguous()]


def _move(st, from_, to):
    """Rows of tokens from_ = (tensors, positions) to tokens `to`."""
    (c0, r0), (c1, r1) = _at(st, *from_), _at(st, *to)
    rows, scales = _planes(st)
    rows[c1, :, :, r1] = rows[c0, :, :, r0]
    if scales is not None:
        scales[c1, :, :, r1] = scales[c0, :, :, r0]


def _attention(st, lens):
    """Every tensor's tokens t < lens[b], padded to the longest."""
    H, G, D = st.case["n_kv"], st.case["group"], st.case["dim"]
    t = torch.arange(int(lens.max()), device="cuda")
    n = torch.from_numpy(lens).cuda()[:, None]
    there = t < n
    chunk, row = _at(st, torch.arange(len(lens), device="cuda")[:, None], torch.minimum(t, n - 1))
    rows, scales = _planes(st)
    side = lambda p: _held(rows[chunk, :, p, row], scales[chunk, :, p, row]).transpose(1, 2).contiguous()  # noqa: E731
    q = st.q.float().view(-1, H, G, D)
    s = torch.matmul(q, side(0).transpose(2, 3)) / math.sqrt(D)
    s = torch.where(there[:, None, None], s, -math.inf)
    w = torch.exp(s - s.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    st.out.copy_(torch.matmul(w, side(1)).view(-1, H * G, D))
    return st.out


def _new_tokens(st):
    return _each(torch.arange(len(st.new), device="cuda"), torch.from_numpy(st.len).cuda(), torch.from_numpy(st.new).cuda())


def _plain_decode(st):
    return [_attention(st, st.len)]


def _plain_step(st):
    to = _new_tokens(st)
    _write(st, *to, st.k_new, st.v_new)
    return [_attention(st, st.len + 1), *_read(st, *to)]


def _plain_append(st):
    to = _new_tokens(st)
    _write(st, *to, st.k_new, st.v_new)
    return _read(st, *to)


def _plain_copy(st):
    src, dst = torch.from_numpy(st.src).cuda(), torch.from_numpy(st.dst).cuda()
    n = torch.from_numpy(st.len[st.src]).cuda()
    from_, to = _each(src, torch.zeros_like(n), n), _each(dst, torch.zeros_like(n), n)
    _move(st, from_, to)
    return _read(st, *to) if st.case["dtype"] == "mxfp4" else _values(st)


def _plain_compact(st):
    which, first, n = torch.arange(len(st.first), device="cuda"), torch.from_numpy(st.first).cuda(), torch.from_numpy(st.n_keep).cuda()
    to = _each(which, first, n)
    new = torch.from_numpy(st.new).cuda()
    if st.case["entry"] == "accept":
        _write(st, *_each(which, first, new), st.k_new, st.v_new)
    _move(st, (to[0], st.keep.long()), to)
    if st.case["entry"] == "accept":
        return _read(st, *to) if st.case["dtype"] == "mxfp4" else _values(st)
    _write(st, *_each(which, first + n, new), st.k_new, st.v_new)
    return _values(st)


_PLAIN = {"decode": _plain_decode, "step": _plain_step, "append": _plain_append, "copy": _plain_copy, "compact": _plain_compact}


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    lens, B, H, D = np.tile(_lens(case), case["layers"]), case["batch"], case["n_kv"], case["dim"]
    n, held, dense = int(lens.sum()), _bytes_per_token(case), 4 * H * D
    kind = case["kind"]
    if kind in ("decode", "step"):
        io = 2 * 2 * len(lens) * H * case["group"] * D
        flops = 4 * n * H * case["group"] * D
        new = len(lens) * (2 * dense + 2 * held) if kind == "step" else 0
        return {"bytes": n * held + io + new, "flops": flops}
    if kind == "append":
        new = int(len(lens) * case["new"] if case["new"] else n)
        return {"bytes": new * (2 * dense + 2 * held), "flops": 0}
    read = (held + dense) if case["dtype"] == "mxfp4" else 0
    if kind == "copy":
        return {"bytes": n * held + case["copies"] * n * (held + read), "flops": 0}
    first, choice, kept = (int(x.sum()) for x in _kept(case))
    if case["entry"] == "accept":
        return {"bytes": choice * (dense + held) + kept * (2 * held + read), "flops": 0}
    return {"bytes": kept * 2 * held + (choice - kept) * (dense + held) + n * read, "flops": 0}


# ---- the same in 64 bits ----------------------------------------------------------------------------
def _held64(x):
    """The values that rows have in 4 bits: a power of two by the logarithm, then the nearest multiple of the spacing there."""
    x = x.double().unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(-1) / 6)
    e = torch.where(m == 0.5, e - 1, e).clamp(-127, 125)[..., None].double()
    y = x * torch.exp2(-e)
    spacing = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return ((torch.round(y / spacing) * spacing).clamp(-6, 6) * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    kind, H, G, D = case["kind"], case["n_kv"], case["group"], case["dim"]
    if case["dtype"] == "bf16":
        return None                                   # moved, not computed
    lens = np.tile(_lens(case), case["layers"])
    if kind in ("append", "step") or kind == "compact" and case["entry"] == "accept":
        count = lens if kind == "append" and not case["new"] else np.full_like(lens, case["new"] or 1)
        k, v = (_held64(x) for x in _rows(case, _gen(seed, 3), int(count.sum())))
        if kind == "append":
            return [k, v]
        if kind == "compact":
            base = np.repeat(np.arange(len(lens)) * case["new"] - lens, _kept(case)[2])
            at = torch.from_numpy(_keep_lists(case, seed) + base).cuda()
            return [k[at], v[at]]
    if kind == "compact":
        first, choice, kept = _kept(case)
        lists = np.split(_keep_lists(case, seed), np.cumsum(kept)[:-1])
        new = [torch.split(_held64(x), (choice - kept).tolist()) for x in _rows(case, _gen(seed, 3), int((choice - kept).sum()))]
        got = [[], []]
        for b, e, *rows in _history(case, seed, lens):
            for x, n, out in zip(rows, new, got):
                for i, y in zip(range(b, e), torch.split(_held64(x), lens[b:e].tolist())):
                    out += [y[:int(first[i])], y[torch.from_numpy(lists[i]).cuda().long()], n[i]]
        return [torch.cat(x) for x in got]
    if kind == "copy":
        ks, vs = [], []
        for b, e, hk, hv in _history(case, seed, lens):
            ks += list(torch.split(_held64(hk), lens[b:e].tolist()))
            vs += list(torch.split(_held64(hv), lens[b:e].tolist()))
        return [torch.cat([x for x in xs for _ in range(case["copies"])]) for xs in (ks, vs)]
    q = _queries(case, seed, len(lens)).double() / math.sqrt(D)
    out = torch.empty(len(lens), H, G, D, dtype=torch.float64, device="cuda")
    for b, e, hk, hv in _history(case, seed, lens):
        at = 0
        for i in range(b, e):
            n = int(lens[i])
            ki, vi = _held64(hk[at:at + n]), _held64(hv[at:at + n])
            if kind == "step":
                ki, vi = torch.cat([ki, k[i:i + 1]]), torch.cat([vi, v[i:i + 1]])
            for h in range(H):
                s = ki[:, h].contiguous() @ q[i, h * G:(h + 1) * G].t().contiguous()
                out[i, h] = torch.softmax(s, 0).t().contiguous() @ vi[:, h].contiguous()
            at += n
    out = out.view(len(lens), H * G, D)
    return [out, k, v] if kind == "step" else [out]
