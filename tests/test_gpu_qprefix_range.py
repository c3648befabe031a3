"""wise_qcache_attn on the GPU where numbers are very large: scores of 2^14 to fp32's largest, against the
fp64 definition over scores that fp32 holds exactly, and values whose sums reach the end of its range."""

import numpy as np
import pytest
import torch

from kept_model import attend, pack, quantise
from cache_model import bf16_values
from parity_util import say
from test_gpu_qprefix import Batch, WIDTHS

pytestmark = pytest.mark.gpu

# (groups, key-value heads, query heads of each, q_len): one row, 17 to 32 rows, and shared pages of few and of more than 64 rows.
KINDS = {"one": ([(0, [300, 33])], 2, 1, 1), "rows": ([(0, [300, 70])], 1, 20, 1), "few": ([(20, [40, 5, 70])], 2, 4, 2),
         "many": ([(20, [30] * 10)], 1, 8, 2)}


def set_keys(b, x):
    """The keys x [pages][kv][page][d] in place of the cache's, exact in its width."""
    pool = b.pool.copy()
    pool[0] = pack(*quantise(x, b.bits), b.bits, 0)
    b.set_pool(pool, b.page, x.shape[-1], b.bits)
    assert np.array_equal(b.k, x)
    b.cache.pool.copy_(torch.tensor(pool))


def exact_scores(b, scale):
    """kept_model.attend where every score is a number that fp32 holds exactly, as no rounding of a sum changes it.  What is then off
    in a probability: its own half step of 2^-12; the scale's rounding, 2^-23 of a difference of up to 2^7 (past it
    the weight is below 2^-128), 2^-16; the exponentials and partial sums, 2^-18 + n 2^-24.  o's rounding, 2^-8 |o|."""
    q = bf16_values(b.q.view(torch.int16).numpy())
    o, lse, _, _ = attend(q, b.k, b.v, b.tables, b.lens, b.ids, b.page, scale)
    most = np.abs(b.v[np.isfinite(b.v)]).max()
    n = b.lens.max()
    a, _, _, _ = attend(q, b.k, np.abs(b.v), b.tables, b.lens, b.ids, b.page, scale)      # sum p |v|
    part = 2.0 ** -12 + 2.0 ** -16 + 2.0 ** -18 + n * 2.0 ** -24
    bound = 2.0 ** -8 * np.abs(o) + (1 + 2.0 ** -8) * (part * a + n * 2.0 ** -31 * most)
    return o, lse, bound, 2.0 ** -16 + 2.0 ** -18 + n * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse)


@WIDTHS
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores(gpu_lib, kind, d, sign, bits):
    """Row maxima of 2^14 to 2^120 of either sign: scores one to twelve fp32 steps apart while these tell weights apart, far apart beyond."""
    groups, kv, gq, q_len = KINDS[kind]
    b = Batch(groups, 16, d, kv, gq, bits, q_len, seed=d)
    rng = np.random.default_rng(d)
    step = rng.choice([0, 0.5, 1, 1.5, 2, 3, 4, 6], size=b.k.shape[:3])
    first = b.tables[:, :4]
    step[first[first >= 0]] = 0                       # the first keys lie below: later ones raise the reference
    x = np.zeros(b.k.shape)
    x[..., 0], x[..., 32] = 1, step
    set_keys(b, x)
    for power in (14, 16, 18, 21, 23, 24, 25, 26, 27, 29, 30, 31, 32, 35, 60, 120):
        q = torch.zeros(b.q.shape)
        q[..., 0] = sign * 2.0 ** 27
        q[..., 32] = 2.0 ** 5 if power < 28 else 2.0 ** 24   # of a step of 0.5: one of fp32's at 2^27, or 2^-4 of the score
        b.q = q.to(torch.bfloat16)
        scale = 2.0 ** (power - 27)
        truth = exact_scores(b, scale)
        for cache in (b.cache, b.roomy()):
            for shared in (True, False):
                out, lse = b.run(shared, scale, cache=cache)
                say(f"2^{power} d {d} bits {bits} {kind} shared {shared}")
                assert torch.isfinite(out).all() and torch.isfinite(lse).all()
                b.check(out, lse, truth)


@WIDTHS
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("gain", [0.0, 1.0, 8.0, 60.0])
def test_large_values(gpu_lib, kind, d, gain, bits):
    """Values that add up to just under 2^127 in a row's dims, in every scale or in one of them: o is finite."""
    groups, kv, gq, q_len = KINDS[kind]
    b = Batch(groups, 16, d, kv, gq, bits, q_len, seed=d, gain=gain)
    n = int(b.lens.max())
    largest = 127 + int(np.floor(127 - np.log2(n * (6 if bits == 4 else 448))))
    pool = b.pool.copy()
    at = 16 * d * bits // 8
    scales = pool[1][..., at:]
    live = scales != 255
    of = np.zeros(scales.shape[-1], int)              # which 32 dims a scale is of
    of[:] = np.arange(of.size) % (4 * d // 32) // 4
    for which in (None, 0, d // 32 - 1):
        new = scales.copy()
        new[live & (of == which if which is not None else True)] = largest
        pool[1][..., at:] = new
        b.set_pool(pool, 16, d, bits)
        b.cache.pool.copy_(torch.tensor(pool))
        truth = b.truth()
        assert np.abs(truth[0]).max() > 2.0 ** 100
        for cache in (b.cache, b.roomy()):
            for shared in (True, False):
                out, lse = b.run(shared, cache=cache)
                say(f"scale {which} d {d} bits {bits} {kind} gain {gain} shared {shared}")
                assert torch.isfinite(out).all()
                b.check(out, lse, truth)


@WIDTHS
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("first", [False, True])
def test_scores_that_overflow(gpu_lib, kind, d, first, bits):
    """Keys of the largest values there are, whose scores are past fp32's range below or next to its end: they have weight 0, whether the
    rows meet them first or last, and a row whose every score is -inf, like one that sees nothing, is 0."""
    groups, kv, gq, q_len = KINDS[kind]
    b = Batch(groups, 16, d, kv, gq, bits, q_len, seed=d)
    big = {4: 6 * 2.0 ** 125, 8: 448 * 2.0 ** 119}[bits]
    b.q[..., 0] = 1 + b.q[..., 0].abs()
    b.q[0, :, :, 0] = 0.5                             # scores that stay finite
    x = b.k.copy()
    x[~np.isfinite(x)] = 0
    x[..., 0] = np.abs(x[..., 0])
    for s in b.ids:
        at = 0 if first else int(b.lens[s] - 1) // 16
        x[int(b.tables[s, at]), :, :, 0] = -big
    codes, scales = quantise(x, bits)
    pool = b.pool.copy()
    pool[0] = pack(codes, scales, bits, 0)
    b.set_pool(pool, 16, d, bits)
    b.cache.pool.copy_(torch.tensor(pool))
    near = b.k.copy()                                 # the definition, and bounds that know of no overflow, with scores of -80 and less
    near[near == -big] = -2000
    hold, b.k = b.k, near
    o, _, bound, _ = b.truth()
    b.k = hold
    for cache in (b.cache, b.roomy()):
        for shared in (True, False):
            out, lse = b.run(shared, cache=cache)
            say(f"d {d} bits {bits} {kind} first {first} shared {shared}")
            got = out.double().cpu().numpy()
            seen = np.isfinite(lse.cpu().numpy())     # a row may see those keys alone
            assert np.isfinite(got).all() and np.all(got[~seen] == 0)
            assert np.all(np.abs(got - o)[seen] <= bound[seen])
