"""wise_qcache_attn on the GPU: what lies in places that no row sees changes neither its results nor its time, and NaN that rows do
see costs little."""

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


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
def test_a_nan_costs_little(gpu_lib, d, bits):
    """A NaN in the newest token's value: at most three times the time of none, as above."""
    b = Batch([(0, [2033] * 8)], 16, d, 8, 4, bits, 1, seed=d)
    q, ids = b.q.cuda(), ints(b.ids)
    b.cache.pool.copy_(torch.tensor(np.where(used(b, d)[:, :, None], b.pool, 0)))
    times = [time_of(b.cache, q, None, ids)]
    for s in b.ids:
        b.cache.pool[1, int(b.tables[s, 2032 // 16]), :, 16 * d * bits // 8] = 255      # the first scale of the page's first token
    times.append(time_of(b.cache, q, None, ids))
    out, _ = b.run()
    nan = torch.isnan(out)
    assert nan[..., :32].all() and not nan[..., 32:].any()
    say(f"d {d} bits {bits}: {times} us")
    assert times[1] < 3 * times[0]


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("lens", [[700, 130, 40], [700, 3000]])
def test_nan_beside_missing_pages(gpu_lib, d, lens, bits):
    """NaN values in tiles that have a mask in the middle of a sequence, as half of their keys have no page, and in later ones."""
    page, q_len = 16, 3
    b = Batch([(0, lens)], page, d, 2, 4, bits, q_len, seed=d)
    missing = [(s, c) for s, n in enumerate(lens) for c in (1, 6, 30) if c * page < n - page]
    for s, c in missing:
        b.tables[s, c] = -1
    b.cache.tables.copy_(ints(b.tables.tolist()))
    o, lse, bound, zb = b.truth()
    row, g = d * bits // 8, d // 32
    for hit in ([(0, 0, 0, 0)], [(0, 7 * page + 3, 1, 1), (0, 20 * page, 0, 0)], [(0, 699, 1, g - 1), (1, 7 * page + 1, 0, 1)],
                [(s, n - q_len + 1, 0, 1) for s, n in enumerate(lens)]):      # sequence, position, head, scale
        pool, want = b.pool.copy(), o.copy()
        for s, pos, h, i in hit:
            p, t = b.tables[s, pos // page], pos % page
            assert p >= 0
            pool[1, p, h, page * row + t // 4 * 4 * g + 4 * i + t % 4] = 255
            for r in range(q_len):
                if pos <= lens[s] - q_len + r:
                    want[s, 4 * h:4 * h + 4, r, 32 * i:32 * i + 32] = np.nan
        b.cache.pool.copy_(torch.tensor(pool))
        for cache in (b.cache, b.roomy()):
            got = b.run(False, cache=cache)[0].double().cpu().numpy()
            assert np.array_equal(np.isnan(got), np.isnan(want)), hit
            ok = ~np.isnan(want)
            assert np.all(np.abs(got - want)[ok] <= bound[ok])
