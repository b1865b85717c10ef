"""Decode over 4-bit rows whose values lie at either end of what the format holds (exponents -127 .. 125): the result is a mean of V, so
it is in range wherever V is, however many tokens it is taken over and however their work is divided."""
import numpy as np
import pytest
import torch

import paper_2506_15155_amd as E
from tests import plain
from tests.test_gpu_fp4 import Cache, dev, host

pytestmark = pytest.mark.gpu

# What an output may be off, of the largest |V| of its block of 32 dims. The result's rounding: half a step, 2^-8. Weights as fp16 values:
# 2^-12 of each, those under 2^-37 of the largest wholly, which for under 2^15 tokens are 2^-22 together. V is exact down to 2^-36 of the largest scale of
# its block. Scores: 128 products in 32 bits, each up to 2^-24 of the sum of magnitudes off, 2^-17 of it together; |q||k| / sqrt(D) log2 e is
# under 60 here, so an exponential's argument is 2^-11 and a weight 2^-11.5 off, which moves a mean by up to twice that.
TOL = 2.0 ** -8 + 2.0 ** -12 + 2.0 ** -10

# requests of one wave and of several, in blocks, in shares that meet in LDS, through the workspace and in the combine pass, of waves
# that leave their results by themselves (over 16 heads), in runs and by units
SHAPES = [(2, 4, 128, 64, [1, 2, 40]), (2, 4, 128, 64, [333, 17, 1]), (8, 4, 128, 512, [3000] * 5), (1, 20, 128, 16, [100]), (1, 33, 64, 48, [700] * 9),
          (4, 1, 128, 300, [2000] * 16), (1, 8, 128, 16, [10000, 3]), (2, 16, 64, 1000, [20000, 900, 1, 7000]), (1, 12, 128, 600, [9000, 50])]


def wanted(q, k, v):
    """Attention with V as parts of its own largest value, which is put back at the end: no sum is out of range in any precision."""
    top = np.abs(v).max()
    return plain.attention(q, k, v / top) * top


@pytest.mark.parametrize("n_kv,group,dim,tokens,lens", SHAPES)
@pytest.mark.parametrize("exponent", [125, 100, -110])
def test_means_of_very_large_and_small_values(n_kv, group, dim, tokens, lens, exponent):
    c = Cache([0] * len(lens), n_kv, group, dim, tokens, room=max(lens))
    k, v = c.draw(sum(lens))
    # every block's largest value between 3 and 6 times 2^exponent; block 1 some powers of two below, of the same sign everywhere
    v = v / np.abs(v).reshape(*v.shape[:2], -1, 32).max(-1).repeat(32, -1).reshape(v.shape) * 6 * 2.0 ** exponent * c.rng.uniform(0.5, 1, (sum(lens), n_kv, 1))
    v[:, :, 32:64] = np.abs(v[:, :, 32:64]) * 2.0 ** -5
    v = plain.bf16(np.clip(v, -6 * 2.0 ** 125, 6 * 2.0 ** 125))
    c.append(k, v, lens)
    q, dq = c.queries()
    out = c.decode(dq)
    assert torch.equal(c.decode(dq, call=E.ellm_decode_attention_noalloc), out)
    got = plain.values(host(out))
    for i in range(len(lens)):
        want = wanted(q[i], c.k[i], c.v[i])
        top = np.repeat(np.abs(c.v[i]).reshape(-1, n_kv, dim // 32, 32).max((0, 3)), group, 0)
        assert (np.abs(got[i] - want) <= TOL * np.repeat(top, 32, -1)).all(), (i, np.abs(got[i] - want).max() / top.max())
    c.close()


def test_values_at_the_format_s_ends_in_one_request():
    """Means over the smallest, ordinary and the largest magnitudes side by side (the request whose codes another test compares)."""
    for dim in (64, 128):
        c = Cache([0], 1, 2, dim, 16, room=64)
        n, rng = 40, np.random.default_rng(3)
        v = rng.choice([0.25, 0.75, 1.25, 5.0, 6.0], (n, 1, dim)) * 2.0 ** rng.integers(-120, 120, (n, 1, 1))
        v[0, 0], v[1, 0], v[2, 0] = 2.0 ** -133, -3.3895313892515355e38, 2.0 ** -126
        c.append(np.zeros((n, 1, dim)), v, [n])
        q, dq = c.queries()
        got = plain.values(host(c.decode(dq)))[0]
        want = wanted(q[0], c.k[0], c.v[0])              # (every weight is 1 / n)
        assert np.isfinite(got).all() and (np.abs(got - want) <= TOL * np.abs(c.v[0]).max()).all()
        assert (got < -5e36).all()
        c.close()


def test_the_fused_step_and_a_second_group_of_requests():
    for lens in ([300, 16, 1000, 1], [20 + i % 70 for i in range(150)]):
        a, b = (Cache(lens, 2, 4, 128, 300, seed=5) for _ in range(2))
        k, v = a.draw(len(lens))
        v = plain.bf16(v / np.abs(v).max() * 6 * 2.0 ** 125)
        q, dq = a.queries()
        out = torch.full_like(dq, 77)
        E.ellm_kv_append_decode(a.pool, a.ids, dev(plain.bits(k)), dev(plain.bits(v)), dq, out)
        b.append(k, v, [1] * len(lens))
        assert torch.equal(out, b.decode(dq))
        a.note(k, v, [1] * len(lens))
        got = plain.values(host(out))
        for i in range(len(lens)):
            want = wanted(q[i], a.k[i], a.v[i])
            assert (np.abs(got[i] - want) <= TOL * np.abs(a.v[i]).max()).all(), i
        a.close()
        b.close()


@pytest.mark.parametrize("n_kv,group,dim,tokens,lens", SHAPES)
def test_scores_without_end(n_kv, group, dim, tokens, lens):
    """Scores that are -infinity: a token of no weight is left out, wherever in the request it lies; where all are, there is no mean (0 / 0)."""
    c = Cache([0] * len(lens), n_kv, group, dim, tokens, room=max(lens))
    k, v = c.draw(sum(lens))
    k[:], at = 0, 0
    left = []
    for n in lens:
        mask = c.rng.random(n) < 0.5
        if n > 600:
            mask[:] = False                              # whole waves without a weight
            mask[-30:] = True
        k[at:at + n, :, 0] = np.where(mask, 0, -(2.0 ** 100))[:, None]
        left.append(mask)
        at += n
    c.append(k, v, lens)
    q = np.zeros((len(lens), n_kv * group, dim))
    q[:, :, 0] = 2.0 ** 100                              # (a product of 2^200 is infinity in 32 bits)
    got = plain.values(host(c.decode(dev(plain.bits(q)))))
    for i, mask in enumerate(left):
        if not mask.any():
            assert np.isnan(got[i]).all()
            continue
        want = wanted(q[i] * 0, c.k[i][mask], c.v[i][mask])
        assert (np.abs(got[i] - want) <= TOL * np.abs(c.v[i]).max()).all(), i
    c.close()
