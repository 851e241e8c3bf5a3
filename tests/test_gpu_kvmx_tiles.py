"""Attention over a microscaled cache takes every key tile once, in every schedule.

A frame is a tile of 64 keys, and a page's values are one in a dim of its own and zero in the others, so an
output's dim is the weight of the frames that hold the page.  Each dim is a few frames of hundreds: a tile left
out, taken twice or taken from another page moves one by a fifteenth and more, the bound is about an eightieth."""
import numpy as np
import pytest

from harness import dev_bf16, dev_i32, host_f32
from test_gpu_kvmx import Pool, _attend, _sync
from workloads import make_rng, normal_bf16

pytestmark = pytest.mark.gpu

T = 64
# the weights and their sum 2^-8 each, the store 2^-8, scores and exp2 2^-10
BOUND = 3 * 2.0 ** -8 + 2.0 ** -10


def times(d, table, n):
    """How often each key of each of the d pages is among the first n keys of a table of pages."""
    count = np.zeros((d, T))
    np.add.at(count, table[:n // T], 1.0)
    if n % T:
        count[table[n // T], :n % T] += 1.0
    return count


def page_weights(q, keys, count):
    """What rows q [m, d] give to each page: keys [pages, T, d] of one head, attended to `count` times each."""
    s = q @ keys.reshape(-1, q.shape[-1]).T / np.sqrt(q.shape[-1])
    p = (np.exp(s - s.max(-1, keepdims=True)) * count.reshape(-1)).reshape(len(q), *count.shape)
    return p.sum(-1) / p.sum((-2, -1))[:, None]


@pytest.fixture(scope="module")
def A(gpu):
    from paper_2606_15319_amd import ardit
    return ardit


def _pages(A, H, d, bits, rows, cached, shared=0):
    """A pool of d pages, page j with ones in dim j, and per stream a table that names them in turn, each from
    another page on; returns the pool, the keys [d, 64, H, d] and the tables."""
    pool = Pool(A, H, d, (8, 8), 1, bits, [d * T], seed=23)
    rng = make_rng(301)
    keys = np.zeros((d, T, H, d))
    for j, page in enumerate(pool.ids[0]):
        v = np.zeros((T, H, d))
        v[:, :, j] = 1.0
        keys[j], held = pool.host.pack(page, normal_bf16(rng, (T, H, d)).astype(np.float64), v)
        assert np.array_equal(held, v)
    pool.upload()
    pool.span = max(c + -(-m // T) for c, m in zip(cached, rows))
    first = 7 * np.arange(len(rows))[:, None] * (np.arange(pool.span) >= shared)
    pick = (np.arange(pool.span) + first) % d
    pool.table = dev_i32(np.array(pool.ids[0], np.int32)[pick])
    return pool, keys, pick


def _check(A, H, d, bits, rows, cached, shared=0):
    pool, keys, pick = _pages(A, H, d, bits, rows, cached, shared)
    q = normal_bf16(make_rng(302), (sum(rows), H, d))
    o = _attend(A, pool, rows, [c * T for c in cached], dev_bf16(q.reshape(-1, H * d)), shared)
    _sync()
    got = host_f32(o).astype(np.float64).reshape(-1, H, d)
    assert np.isfinite(got).all()
    rng = np.random.default_rng(303)
    at = 0
    for b, m in enumerate(rows):
        n = cached[b] * T + m
        count = times(d, pick[b], n)
        assert count.sum() == n
        # rows of every 256-row tile, and the last
        some = [at + int(rng.integers(r, min(r + 256, m))) for r in range(0, m, 256)] + [at + m - 1] if m else []
        for h in range(H):
            ref = page_weights(q[some, h].astype(np.float64), keys[:, :, h], count)
            assert np.all(np.abs(got[some, h] - ref) <= BOUND * ref), h
        at += m


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,d,rows,cached", [
    (12, 128, [4600], [200]),                   # items that shed their tails
    (10, 128, [2300, 2290], [180, 180]),
    (12, 64, [4600], [260]),
    (20, 64, [4600], [100]),                    # a full round, and a split one
    (20, 128, [4600], [330]),
    (8, 128, [2048, 1024], [300, 64]),          # split, of two lengths
    (4, 64, [300, 513], [300, 130]),
    (64, 64, [1275, 505], [120, 130]),          # two to a CU
    (8, 64, [6240, 780, 4608], [432, 216, 48]),   # one to a CU
    (8, 64, [4600, 4607], [440, 148]),          # 32 rows each
    (12, 128, [4608], [72]),                    # whole
])
def test_chunks(A, bits, H, d, rows, cached):
    _check(A, H, d, bits, rows, cached)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,d,rows,cached,shared", [
    (3, 128, [1, 40, 0, 9], [300, 171, 2, 130], 0),       # cuts, joined
    (10, 64, [17, 192, 1, 65], [300, 64, 210, 90], 0),
    (2, 128, [1] * 30 + [40], [25] * 30 + [31], 0),       # a wave each
    (8, 64, [2000, 1], [100, 1000], 0),                   # beside the other kernel, joined
    (8, 128, [3000, 3, 40], [200, 400, 200], 0),
    (4, 128, [3, 1, 24, 7, 12, 1], [200, 204, 201, 230, 200, 210], 200),
    (2, 64, [1] * 40, [130 + i % 3 for i in range(40)], 130),
])
def test_few_rows(A, bits, H, d, rows, cached, shared):
    _check(A, H, d, bits, rows, cached, shared)
