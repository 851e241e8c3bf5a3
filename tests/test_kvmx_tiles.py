"""That tests/test_gpu_kvmx_tiles.py sees a tile left out, taken twice or taken from another page: the mistakes
made in its oracle."""
import numpy as np
import pytest

from test_gpu_kvmx_tiles import BOUND, T, page_weights, times


@pytest.mark.parametrize("d,frames,last", [(128, 272, 56), (64, 332, 56), (64, 513, 64), (128, 403, 24), (64, 31, 1)])
def test_one_wrong_tile_is_seen(d, frames, last):
    """In every row, whichever tile it is (at d dims a page is one of up to nine frames)."""
    rng = np.random.default_rng(1)
    table = np.arange(frames) % d
    n = (frames - 1) * T + last
    keys, q = rng.standard_normal((d, T, d)), rng.standard_normal((4, d))
    right = page_weights(q, keys, times(d, table, n))
    whole = np.zeros((d, T))
    for t in range(frames if last > 8 else frames - 1):
        part = whole.copy()
        part[table[t], :T if t + 1 < frames else last] = 1.0
        other = np.roll(part, 1, 0)
        for wrong in (-part, part, other - part):
            got = page_weights(q, keys, times(d, table, n) + wrong)
            assert np.all(np.any(np.abs(got - right) > 2 * BOUND * right, -1)), t
