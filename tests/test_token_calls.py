"""Reading, copying and compacting tokens, and pools of 4-bit rows: what the calls do to the host's state, and what they
refuse, on pools without a device. Also the plain 4-bit format that the GPU tests compare with."""
import os
import re
import subprocess

import numpy as np
import pytest

import paper_2506_15155_amd as E
from tests import plain

ERR = E.ERR
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def pool(n_chunks=32, tensors=8, slots=8, tokens=16, host=0, dtype=E.ELLM_MXFP4, n_kv=2, dim=64, flags=E.ELLM_POOL_METADATA_ONLY):
    row = dim // 2 + dim // 32 if dtype == E.ELLM_MXFP4 else 2 * dim
    cb = -(-tokens * 2 * n_kv * row // 256) * 256
    return E.ellm_pool_create(None, None, cb, 2 * n_kv, n_kv, dim, tensors, slots, flags=flags, device_bytes=n_chunks * cb,
                              host_bytes=host * cb, dtype=dtype)


def grown(p, n, room=None):
    """A tensor of n tokens with chunks for `room`."""
    T = E.ellm_pool_get_geometry(p)["tokens_per_chunk"]
    t = E.ellm_tensor_create(p, max(room or n, 1))
    E.ellm_tensor_map_chunks(p, t, 0, -(-(room or n) // T))
    if n:
        E.ellm_kv_append(p, [t], 16, 16, [n])
    return t


def length(p, t):
    return E.ellm_tensor_get_table(p, t)[1]


def state(p, n):
    o, s, mt, ms = E.ellm_pool_get_owner_state(p)
    return [(tuple(tab), ln) for tab, ln in (E.ellm_tensor_get_table(p, t) for t in range(n))], tuple(o), tuple(s), tuple(mt), tuple(ms)


@pytest.mark.parametrize("n_kv,dim,tokens", [(1, 64, 16), (2, 64, 16), (8, 128, 24), (40, 128, 100), (5, 64, 255), (8, 128, 300), (2, 64, 257)])
def test_geometry_of_four_bit_pools(n_kv, dim, tokens):
    bpt = 2 * n_kv * (dim // 2 + dim // 32)
    cb = -(-tokens * bpt // 256) * 256
    p = E.ellm_pool_create(None, None, cb, n_kv, n_kv, dim, 2, 2, flags=1, device_bytes=4 * cb, dtype=E.ELLM_MXFP4)
    g = E.ellm_pool_get_geometry(p)
    assert g["bytes_per_token"] == bpt and g["tokens_per_chunk"] == plain.tokens_per_chunk(cb, n_kv, dim, True)
    T = g["tokens_per_chunk"]
    assert T * bpt <= cb and (T < 256 or T % 16 == 0)
    E.ellm_pool_destroy(p)


def test_pool_refuses_other_types():
    for dtype in (0, 3, 65535):
        rc, p = E.ellm_pool_create(None, None, 4096, 2, 2, 64, 2, 2, flags=1, device_bytes=65536, dtype=dtype, check=False)
        assert rc == ERR.INVALID and not p
    # a chunk has to hold a token: 136 bytes of one head of 128, 17 heads are 2312
    rc, p = E.ellm_pool_create(None, None, 2304, 17, 17, 128, 2, 2, flags=1, device_bytes=65536, dtype=E.ELLM_MXFP4, check=False)
    assert rc == ERR.INVALID and not p


@pytest.mark.parametrize("dtype", [E.ELLM_MXFP4, E.ELLM_BF16])
def test_copies_and_cuts_change_lengths_and_slots(dtype):
    p = pool(dtype=dtype)
    T = E.ellm_pool_get_geometry(p)["tokens_per_chunk"]
    a, b, c = grown(p, 3 * T + 5), grown(p, 0, 8 * T), grown(p, 7, 8 * T)
    E.ellm_kv_copy(p, [a, a], [b, c])
    assert (length(p, a), length(p, b), length(p, c)) == (3 * T + 5, 3 * T + 5, 3 * T + 12)
    E.ellm_kv_copy(p, [a, a], [b, c], first=[T, 3 * T + 5], n_tokens=[2, 0])
    assert (length(p, b), length(p, c)) == (3 * T + 7, 3 * T + 12)
    E.ellm_kv_copy(p, [a], [b], first=[3 * T])
    assert length(p, b) == 3 * T + 12
    # kept: 3 of the tokens from T on
    E.ellm_kv_compact(p, [a, b], first=[T, 0], keep=4096, n_keep=[3, 1])
    assert (length(p, a), length(p, b)) == (T + 3, 1)
    free = int((E.ellm_pool_get_owner_state(p)[1] == E.ELLM_CHUNK_FREE).sum())
    E.ellm_kv_compact(p, [b, c], flags=E.ELLM_COMPACT_UNMAP)
    assert (length(p, b), length(p, c)) == (0, 0)
    for t in (b, c):
        assert (E.ellm_tensor_get_table(p, t)[0] == -1).all()
    assert int((E.ellm_pool_get_owner_state(p)[1] == E.ELLM_CHUNK_FREE).sum()) == free + 16
    E.ellm_kv_compact(p, [a], first=[T], n_keep=[0], flags=E.ELLM_COMPACT_UNMAP)
    table, n = E.ellm_tensor_get_table(p, a)
    assert n == T and (table >= 0).tolist() == [True, False, False, False]
    assert E.ellm_pool_self_check(p) == 0
    E.ellm_pool_destroy(p)


def test_cut_slots_give_host_copies_back():
    p = pool(host=4)
    T = E.ellm_pool_get_geometry(p)["tokens_per_chunk"]
    a = grown(p, 3 * T)
    E.ellm_chunk_deflate_to_host(p, a, 1, 2)
    assert E.ellm_kv_compact(p, [a], first=[T + 1], keep=4096, n_keep=[1], check=False) == ERR.NOT_RESIDENT
    E.ellm_kv_compact(p, [a], first=[T], flags=E.ELLM_COMPACT_UNMAP)      # nothing moves: what lies behind may be anywhere
    assert (E.ellm_pool_get_host_slots(p)[0] == -1).all() and length(p, a) == T
    assert E.ellm_pool_self_check(p) == 0
    E.ellm_pool_destroy(p)


def test_refusals_change_nothing():
    p = pool(host=2, tensors=6)
    T = E.ellm_pool_get_geometry(p)["tokens_per_chunk"]
    a, b, c, d = grown(p, 2 * T + 3), grown(p, 4, 4 * T), grown(p, T, 3 * T), grown(p, 2 * T)
    gone = grown(p, T)
    E.ellm_tensor_release(p, gone)
    E.ellm_chunk_deflate_to_host(p, d, 1, 1)
    hole = E.ellm_tensor_create(p, 2 * T)
    E.ellm_tensor_map_chunks(p, hole, 0, 1)
    before = state(p, 6)
    read = lambda *x, k=16, v=16, **y: E.ellm_kv_read(p, *x, k, v, check=False, **y)  # noqa: E731
    copy = lambda *x, **y: E.ellm_kv_copy(p, *x, check=False, **y)  # noqa: E731
    compact = lambda *x, **y: E.ellm_kv_compact(p, *x, check=False, **y)  # noqa: E731
    for call in (read, lambda ids, **y: copy(ids, [b] * len(ids), **y) if len(ids) == 1 else ERR.INVALID):
        assert call([17]) == call([-1]) == call([gone]) == ERR.INVALID
        assert call([a], first=[-1]) == call([a], n_tokens=[-1]) == ERR.INVALID
        assert call([a], first=[2 * T + 4]) == call([a], n_tokens=[2 * T + 4]) == call([a], first=[5], n_tokens=[2 * T - 1]) == ERR.RANGE
        assert call([a], first=[2**62], n_tokens=[2**62]) == call([a], first=[1], n_tokens=[2**63 - 1]) == ERR.RANGE
        assert call([d]) == call([d], first=[T + 2]) == ERR.NOT_RESIDENT
    assert read([a], k=None) == read([a], v=None) == ERR.INVALID
    assert read([a, a]) == ERR.NO_DEVICE and read([hole]) == read([a], first=[2 * T + 3]) == ERR.OK
    assert E.lib.ellm_kv_read(p, None, 1, None, None, 16, 16, None) == ERR.INVALID == E.lib.ellm_kv_read(p, None, -1, None, None, 16, 16, None)
    assert copy([a], [gone]) == copy([a], [99]) == copy([a, a], [b, b]) == copy([a, b], [b, c]) == copy([b], [b]) == ERR.INVALID
    assert copy([a, c], [c, b], n_tokens=[1, 1]) == ERR.INVALID
    assert copy([a], [hole]) == ERR.RANGE                     # 2 T + 3 tokens into room for 2 T
    assert copy([a], [hole], n_tokens=[T + 1]) == ERR.UNMAPPED
    assert copy([a], [c], n_tokens=[2 * T + 1]) == ERR.RANGE
    assert copy([c], [d]) == ERR.RANGE
    assert E.lib.ellm_kv_copy(p, None, None, 1, None, None, None) == ERR.INVALID == E.lib.ellm_kv_copy(p, None, None, -1, None, None, None)
    assert compact([a], flags=2) == compact([a, a]) == compact([55]) == compact([gone]) == ERR.INVALID
    assert compact([a], first=[-1]) == compact([a], n_keep=[-1], keep=16) == ERR.INVALID
    assert compact([a], first=[2 * T + 4]) == compact([a], first=[2 * T], n_keep=[4], keep=16) == compact([a], n_keep=[2**62], keep=16) == ERR.RANGE
    assert compact([a], n_keep=[1]) == ERR.INVALID            # nothing that names the token
    assert compact([d], n_keep=[1], keep=16) == ERR.NOT_RESIDENT
    assert E.lib.ellm_kv_compact(p, None, 1, None, None, None, 0, None) == ERR.INVALID
    assert E.lib.ellm_kv_compact(None, None, 0, None, None, None, 0, None) == ERR.INVALID
    assert E.lib.ellm_kv_copy(None, None, None, 0, None, None, None) == E.lib.ellm_kv_read(None, None, 0, None, None, None, None, None) == ERR.INVALID
    assert state(p, 6) == before and E.ellm_pool_self_check(p) == 0
    # nothing to do is done
    assert read([]) == copy([], []) == compact([]) == compact([a], first=[2 * T + 3]) == 0
    assert state(p, 6) == before
    E.ellm_pool_destroy(p)


def test_tensors_of_2_to_the_31_tokens():
    """The kernels number positions in 32 bits: what would pass them is refused; lengths can be cut all the same."""
    most = 3 << 30
    for dtype in (E.ELLM_BF16, E.ELLM_MXFP4):
        cb = 1 << 31
        p = E.ellm_pool_create(None, None, cb, 1, 1, 64, 3, 400, flags=1, device_bytes=800 * cb, dtype=dtype)
        T = E.ellm_pool_get_geometry(p)["tokens_per_chunk"]
        t = E.ellm_tensor_create(p, most)
        E.ellm_tensor_map_chunks(p, t, 0, -(-most // T))
        small = E.ellm_tensor_create(p, 100)
        E.ellm_tensor_map_chunks(p, small, 0, 1)
        add = lambda n: E.ellm_kv_append(p, [t], 16, 16, [n], check=False)  # noqa: E731
        assert add(1 << 30) == ERR.RANGE
        assert add((1 << 30) - 1) == add((1 << 30) - 1) == add(1) == 0 and length(p, t) == (1 << 31) - 1
        assert add(1) == (ERR.RANGE if dtype == E.ELLM_MXFP4 else 0)
        assert E.ellm_kv_read(p, [t], 16, 16, first=[5], n_tokens=[1], check=False) == ERR.RANGE
        assert E.ellm_kv_copy(p, [t], [small], first=[5], n_tokens=[1], check=False) == ERR.RANGE
        assert E.ellm_kv_compact(p, [t], keep=16, n_keep=[1], check=False) == ERR.RANGE
        assert E.ellm_kv_compact(p, [t], first=[(1 << 31) - 1], check=False) == E.ellm_kv_compact(p, [t], first=[7], check=False) == 0
        assert length(p, t) == 7 and E.ellm_kv_copy(p, [t], [small], check=False) == 0 and length(p, small) == 7
        E.ellm_pool_destroy(p)


def test_binding_refuses_short_arrays():
    import torch
    p = pool()
    a, b = grown(p, 5), grown(p, 5)
    with pytest.raises(ValueError):
        E.ellm_kv_read(p, [a, b], 16, 16, first=[0])
    with pytest.raises(ValueError):
        E.ellm_kv_copy(p, [a, b], [a])
    with pytest.raises(ValueError):
        E.ellm_kv_compact(p, [a, b], first=[0], keep=16, n_keep=[1, 1])
    with pytest.raises(ValueError):
        E.ellm_kv_compact(p, [a, b], keep=torch.zeros(3, dtype=torch.int32), n_keep=[2, 2])
    with pytest.raises(ValueError):
        E.ellm_kv_compact(p, [a], keep=torch.zeros(3, dtype=torch.int64), n_keep=[2])
    assert length(p, a) == length(p, b) == 5
    E.ellm_pool_destroy(p)


@pytest.mark.parametrize("call", ["append", "copy", "compact"])
def test_a_refused_launch_leaves_whole_groups(call):
    """Groups of 128 requests before the refused one are done, those behind it untouched."""
    n = 300
    p = pool(n_chunks=2 * n + 2, tensors=n + 1, slots=2)
    T = E.ellm_pool_get_geometry(p)["tokens_per_chunk"]
    src = grown(p, 9, 2 * T)
    ids = [grown(p, 5, 2 * T) for _ in range(n)]
    E.ellm_debug_fail_launch(p, 2)
    flags = E.ELLM_COMPACT_UNMAP
    rc = {"append": lambda: E.ellm_kv_append(p, ids, 16, 16, [3] * n, check=False),
          "copy": lambda: E.ellm_kv_copy(p, [src] * n, ids, n_tokens=[3] * n, check=False),
          "compact": lambda: E.ellm_kv_compact(p, ids, first=[1] * n, keep=16, n_keep=[2] * n, flags=flags, check=False)}[call]()
    assert rc == ERR.HIP and "refused" in E.ellm_last_error()
    done = 3 if call == "compact" else 8
    assert [length(p, t) for t in ids] == [done] * 128 + [5] * (n - 128)
    mapped = [int((E.ellm_tensor_get_table(p, t)[0] >= 0).sum()) for t in ids]
    assert mapped == ([1] * 128 if call == "compact" else [2] * 128) + [2] * (n - 128)
    assert E.ellm_pool_self_check(p) == 0
    E.ellm_pool_destroy(p)


class Nothing:
    """In the place of the native calls: handles no form of these."""

    def __getattr__(self, name):
        return (lambda *a: None) if name in ("read", "copy", "compact") else getattr(REAL, name)


REAL = E.binding._calls


def forms(values, dtype):
    a = np.asarray(values, dtype)
    wide = np.zeros(2 * len(a), dtype)
    wide[::2] = a
    return {"array": a, "list": list(values), "other width": a.astype(np.int32 if dtype == np.int64 else np.int64), "strided": wide[::2],
            "swapped": a.astype(a.dtype.newbyteorder()), "longer": np.concatenate([a, a])}


@pytest.mark.parametrize("ids_form", ["array", "list", "other width", "strided", "swapped"])
@pytest.mark.parametrize("n_form", ["array", "list", "other width", "strided", "swapped", "longer"])
def test_native_conversion_and_the_general_one(monkeypatch, ids_form, n_form):
    """Every form of arguments gives the same results, tables and refusals either way."""
    import torch

    class Address:
        def data_ptr(self):
            return 0x2000

    def walk():
        p = pool(tensors=4)
        t = [grown(p, 40, 120), grown(p, 20, 120), grown(p, 0, 120)]
        ids = lambda *v: forms([t[i] if i < 3 else i for i in v], np.int32)[ids_form]  # noqa: E731
        n = lambda *v: forms(v, np.int64)[n_form]  # noqa: E731
        seen = []

        def call(f, *a, **k):
            try:
                seen.append(f(p, *a, stream=0, **k))
            except Exception as e:
                seen.append((type(e).__name__, getattr(e, "code", None)))

        for at in (0x1000, None, Address(), torch.zeros(4)):
            call(E.ellm_kv_read, ids(0, 1), at, 0x3000, first=n(1, 20), n_tokens=n(2, 0))
            call(E.ellm_kv_read, ids(2), 0x3000, at)
        call(E.ellm_kv_read, ids(9), 16, 16, check=False)
        call(E.ellm_kv_copy, ids(0, 1), ids(2), first=n(1, 2))
        call(E.ellm_kv_copy, ids(0), ids(2))
        call(E.ellm_kv_copy, ids(0), ids(1, 2), first=n(7), n_tokens=n(3))
        call(E.ellm_kv_copy, ids(0), ids(0), check=False)
        for keep in (0x1000, Address(), torch.zeros(4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int64),
                     torch.zeros(8, dtype=torch.int32)[::2], None, "x"):
            call(E.ellm_kv_compact, ids(0, 1), first=n(1, 2), keep=keep, n_keep=n(3, 1))
        for flags in (0, 1, 2, True):
            call(E.ellm_kv_compact, ids(0, 1), first=n(2, 1), flags=flags, check=False)
        call(E.ellm_kv_compact, ids(0, 1), first=n(1))
        call(E.ellm_kv_compact, ids(0, 1))
        after = state(p, 3)
        E.ellm_pool_destroy(p)
        return seen, after

    native = walk()
    assert native[0].count(0) >= 5
    monkeypatch.setattr(E.binding, "_calls", Nothing())
    assert walk() == native


def test_plain_arguments_are_converted_natively():
    p = pool()
    a, b = grown(p, 9, 40), grown(p, 0, 40)
    ids, other, one = np.array([a], np.int32), np.array([b], np.int32), np.array([1], np.int64)
    assert REAL.read(p, ids, 16, 16, None, one, 0) == ERR.NO_DEVICE
    assert REAL.copy(p, ids, other, one, None, 0) == 0 and REAL.compact(p, ids, one, 16, one, 0, 0) == 0
    assert (length(p, a), length(p, b)) == (2, 8)
    with pytest.raises(TypeError):
        REAL.copy(p, ids)
    E.ellm_pool_destroy(p)


# ---- the format that GPU tests compare with ---------------------------------------------------------
def test_plain_format():
    one = lambda *x: np.array(list(x) + [0.0] * (32 - len(x)))  # noqa: E731
    c, s = plain.quantise(one(6.0, -6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.2500001))
    assert s[0] == 127 and c[:10].tolist() == [7, 15, 0, 2, 2, 4, 4, 6, 6, 9]
    assert plain.quantise(one(6.0000001))[1][0] == 128 and plain.quantise(one(3.0))[1][0] == 126
    assert plain.quantise(one(0.0))[1][0] == 0 and plain.quantise(one(2.0**-126))[1][0] == 0
    c, s = plain.quantise(one(3.0e38))
    assert s[0] == 252 and c[0] == 7 and np.isfinite(plain.held(c, s)).all()
    c, s = plain.quantise(one(1.0, np.nan, np.inf))
    assert s[0] == 255 and not c.any() and np.isnan(plain.held(c, s)).all()
    rng = np.random.default_rng(0)
    x = plain.bf16(rng.standard_normal((50, 128)) * np.exp2(rng.integers(-20, 20, (50, 1))))
    c, s = plain.quantise(x)
    v = plain.held(c, s)
    top = np.repeat(np.abs(x).reshape(50, 4, 32).max(-1), 32, -1)
    assert (np.abs(v - x) <= top / 5 + 1e-300).all()                    # 5 is held as 4
    again = plain.quantise(v)
    assert np.array_equal(plain.held(*again), v)                        # what is held is held exactly


def test_no_kernel_of_any_file_needs_scratch_memory(tmp_path):
    """As the test of the same property of the first file of kernels, for the code objects of all of them."""
    tools = "/opt/rocm/llvm/bin/"
    if not os.path.exists(tools + "clang-offload-bundler"):
        pytest.skip("no LLVM tools")
    section = str(tmp_path / "fatbin")
    subprocess.run([tools + "llvm-objcopy", "--dump-section", ".hip_fatbin=" + section, E.LIB_PATH, str(tmp_path / "unused")], check=True)
    data = open(section, "rb").read()
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)]
    assert len(starts) == 3
    found = []
    for i, (a, b) in enumerate(zip(starts, starts[1:] + [len(data)])):
        bundle, code = str(tmp_path / f"bundle{i}"), str(tmp_path / f"code{i}")
        open(bundle, "wb").write(data[a:b])
        subprocess.run([tools + "clang-offload-bundler", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", "--input=" + bundle,
                        "--output=" + code, "--unbundle"], check=True)
        notes = subprocess.run([tools + "llvm-readelf", "--notes", code], check=True, capture_output=True, text=True).stdout
        found += zip(*(re.findall(rf"^    \.{key}: +(\S+)$", notes, flags=re.M) for key in ("name", "private_segment_fixed_size", "vgpr_spill_count")))
    names = " ".join(n for n, _, _ in found)
    for kernel in ("decode_fp4_kernel", "decode_fp4_block_kernel", "fp4_append_kernel", "read_tokens_kernel", "copy_tokens_kernel", "compact_kernel"):
        assert kernel in names
    assert [n for n, a, b in found if int(a) or int(b)] == []
