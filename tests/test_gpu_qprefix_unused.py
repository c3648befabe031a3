"""wise_qcache_attn on the GPU: what lies in places that no row sees changes neither its results nor its time."""

import numpy as np
import pytest
import torch

from parity_util import say
from test_gpu_qprefix import Batch, WIDTHS, ints

pytestmark = pytest.mark.gpu


def used(b, d):
    """Which bytes of the pool's pages belong to a token that is there: [2][pages][bytes]."""
    from kept_model import places
    out = np.zeros((2, b.pool.shape[1], b.pool.shape[3]), bool)
    tokens = np.zeros(b.pool.shape[1], int)
    for s, n in enumerate(b.lens):
        for c, p in enumerate(b.tables[s]):
            if p >= 0:
                tokens[p] = max(tokens[p], min(b.page, n - c * b.page))
    for plane in (0, 1):
        code, _, scale = places(b.page, d, b.bits, plane)
        for p, n in enumerate(tokens):
            out[plane, p, code[:n].reshape(-1)] = True
            out[plane, p, scale[:n].reshape(-1)] = True
    return out


def time_of(cache, q, shared, ids):
    """us of a call, the median of 9 runs of 20."""
    out = torch.empty_like(q)
    times = []
    for _ in range(9):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        for _ in range(20):
            cache.attend(0, q, out, seq_ids=ids, shared=shared)
        end.record()
        end.synchronize()
        times.append(start.elapsed_time(end) / 20 * 1e3)
    return sorted(times)[4]


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("fill", [0, 127, 255, None])
def test_unused_bytes(gpu_lib, d, fill, bits):
    """The same bits whatever unused bytes hold: zeros, NaN codes under ordinary scales, NaN, anything."""
    b = Batch([(8, [30, 45, 7]), (0, [2033, 1, 300])], 16, d, 2, 4, bits, 2, seed=d)
    mine = used(b, d)[:, :, None]
    want = [b.run(shared, cache=cache) for cache in (b.cache, b.roomy()) for shared in (True, False)]
    truth = b.truth()
    rng = np.random.default_rng(d)
    other = rng.integers(0, 256, b.pool.shape, dtype=np.uint8) if fill is None else np.full_like(b.pool, fill)
    b.cache.pool.copy_(torch.tensor(np.where(mine, b.pool, other)))
    got = [b.run(shared, cache=cache) for cache in (b.cache, b.roomy()) for shared in (True, False)]
    for (o, lse), (o2, lse2) in zip(want, got):
        b.check(o, lse, truth)
        assert torch.equal(o.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse, lse2)


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
def test_unused_bytes_cost_nothing(gpu_lib, d, bits):
    """A last page that is partly filled takes the same time over zeros and over NaN: at most three times as long, as only a walk
    over the sequence's keys for these would exceed (2033 reads one after another, half a millisecond)."""
    b = Batch([(0, [2033] * 8)], 16, d, 8, 4, bits, 1, seed=d)
    mine = used(b, d)[:, :, None]
    q, ids = b.q.cuda(), ints(b.ids)
    times = []
    for fill in (0, 127, 255):
        b.cache.pool.copy_(torch.tensor(np.where(mine, b.pool, np.full_like(b.pool, fill))))
        times.append(time_of(b.cache, q, None, ids))
    say(f"d {d} bits {bits}: {times} us")
    assert max(times[1:]) < 3 * times[0]
