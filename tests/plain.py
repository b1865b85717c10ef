"""Plain implementations in 64 bits of what tests of the 4-bit cache compare with: the format, and attention."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def bf16(x):
    """float32/64 values rounded to nearest-even bf16, as float64."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    r = ((u.astype(np.uint64) + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint32) << 16
    return np.where(np.isnan(x), np.float32(np.nan), r.view(np.float32)).astype(np.float64)


def bits(x):
    """bf16 bit patterns of values that bf16 has."""
    return (np.ascontiguousarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def values(b):
    return (np.ascontiguousarray(b).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def quantise(x):
    """[..., D] bf16 values -> (codes 0..15 [..., D], scale codes [..., D / 32]), by search over the grid."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(blocks).max(-1)
    bad = ~np.isfinite(blocks).all(-1)
    top = np.where(bad, 0, top)
    # the smallest power of two that the maximum is at most 6 times of: about where the logarithm says, then by comparison
    e = np.clip(np.floor(np.log2(np.maximum(top, 1e-300) / 6)), -127, 125).astype(int)
    for _ in range(2):
        e = np.where((top > 6.0 * 2.0 ** e.astype(float)) & (e < 125), e + 1, e)
        e = np.where((top <= 6.0 * 2.0 ** (e - 1.0)) & (e > -127), e - 1, e)
    y = np.abs(np.where(bad[..., None], 0, blocks)) / (2.0 ** e.astype(float))[..., None]
    d = np.abs(y[..., None] - GRID)
    near = d.min(-1, keepdims=True)
    # of two at the same distance the even code
    pick = np.where(d == near, np.arange(8) % 2, 9).argmin(-1)
    codes = np.where(bad[..., None], 0, pick + 8 * np.signbit(blocks))
    return codes.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def held(codes, scales):
    """The values that codes and scales stand for."""
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def attention(q, k, v, scale=None):
    """q [Hq][D], k and v [tokens][Hkv][D], all float64 -> [Hq][D]"""
    hq, dim = q.shape
    hkv = k.shape[1]
    g = hq // hkv
    out = np.empty((hq, dim))
    for h in range(hq):
        s = k[:, h // g] @ q[h] * (1 / np.sqrt(dim) if scale is None else scale)
        w = np.exp(s - s.max())
        out[h] = (w / w.sum()) @ v[:, h // g]
    return out


def tokens_per_chunk(chunk_bytes, n_kv, dim, fp4):
    if not fp4:
        return chunk_bytes // (4 * n_kv * dim)
    t = chunk_bytes // (2 * n_kv * (dim // 2 + dim // 32))
    return t // 16 * 16 if t >= 256 else t


def chunk_rows(chunk, n_kv, dim, tokens, fp4):
    """A chunk's bytes -> [token][kv head][K, V] of rows: bf16 bits, or (codes, scales)."""
    if not fp4:
        rows = chunk.view(np.uint16)[:2 * n_kv * tokens * dim].reshape(n_kv, 2, tokens, dim)
        return rows.transpose(2, 0, 1, 3)
    end = n_kv * tokens * dim
    b = chunk[:end].reshape(n_kv, 2, tokens, dim // 2)
    codes = np.stack([b & 15, b >> 4], -1).reshape(n_kv, 2, tokens, dim)
    scales = chunk[end:end + 2 * n_kv * tokens * (dim // 32)].reshape(n_kv, 2, tokens, dim // 32)
    return codes.transpose(2, 0, 1, 3), scales.transpose(2, 0, 1, 3)
