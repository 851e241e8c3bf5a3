"""Keys next to the border of two codes: an append into a microscaled cache takes the nearer."""
import numpy as np
import pytest

import oracle as O
from harness import dev_bf16, host_f32
from oracle import mxkv_ref as M
from test_gpu_kvmx import Pool, _sync
from workloads import make_rng, normal_bf16

pytestmark = pytest.mark.gpu

EPS = float(np.float32(1e-6))


@pytest.fixture(scope="module")
def A(gpu):
    from paper_2606_15319_amd import ardit
    return ardit


def _bf16(x):
    """x to bf16, towards zero."""
    return (np.asarray(x, np.float32).view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)


def _near(rng, bits, border, delta, top):
    """A row of 128 (two heads of 64): its first element's key is border (1 + delta) of its block's scale, and the
    block's largest, two on, about `top` of the norm (None: that one's key is `border` itself).  What is left of the
    norm goes to the second head by the largest squares that fit, so that it is right to 2^-50."""
    D = 128
    row = np.zeros(D)
    lead = float(_bf16(rng.uniform(1, 2)))
    rms = lead / (border * (1 + delta))
    if top is None:
        row[2] = lead
        row[0:32:4] = _bf16(rng.uniform(0.02, 0.3, 8) * lead)
    else:
        row[0] = lead
        row[2] = float(_bf16(top * rms))
    left = D * (rms * rms - EPS) - float(np.sum(row * row))
    assert left > 0
    for i in range(64, 74):
        row[i] = float(_bf16(np.sqrt(left)))
        left -= row[i] ** 2
    return row * rng.choice([-1.0, 1.0], D)


def _append(A, bits, qkv, gain, eps=EPS):
    """Keys of one stream of frames of 8 x 8 tokens, two heads of 64, from position 0: what its pages hold, and the pool."""
    import torch
    n, H, d, T = len(qkv), 2, 64, 64
    pool = Pool(A, H, d, (8, 8), 1, bits, [T] * (n // T), fill=0)
    pool.dims = A.make_dims(H * d, H, d, 128, 1, 8, 8, eps)
    pool.upload()
    q = torch.empty((n, H * d), dtype=torch.bfloat16, device="cuda")
    B = n // T
    A.ardit_kv_append_mx(None, pool.dims, A.Batch([T] * B, [0] * B, [0] * B), dev_bf16(qkv), dev_bf16(np.ones(H * d, np.float32)),
                         dev_bf16(gain), pool.kv(), q)
    _sync()
    pool.download()
    return np.concatenate([pool.host.unpack(i[0])[0] for i in pool.ids]), q


def _want(rows, gain, eps=EPS):
    """Keys of _append in 64 bits."""
    k = O.rms_norm(rows.astype(np.float64), eps, gain.astype(np.float64)).reshape(-1, 2, 64)
    return np.concatenate([O.rope3d(k[t:t + 64], O.chunk_positions(1, 8, 8, 0), 10000.0) for t in range(0, len(k), 64)])


@pytest.mark.parametrize("bits", [8, 4])
def test_the_nearer_code(A, bits):
    """Borders of codes and of scales, missed by 2^-26 and 2^-36 on either side: less than fp32 tells apart."""
    rng = np.random.default_rng(200 + bits)
    g = M.grid(bits)
    unit = 2.0 ** -5 if bits == 8 else 1.0         # the scale of blocks whose largest is between 4 and 6
    rows, deltas = [], []
    for i in range(192):
        delta = (1 if i & 1 else -1) * 2.0 ** (-26 if i & 2 else -36)
        if i % 4 == 3 and i > 96:
            # the largest of its block just below 256 2^e, or just above 6 2^e
            border, top = (8.0 if bits == 8 else 6.0), None
            delta = -abs(delta) if bits == 8 else abs(delta)
            if i & 4:                              # and on the side where nothing changes
                delta = -delta
        else:
            c = int(rng.integers(0, np.searchsorted(g, 5.0 / unit)))
            border, top = (g[c] + g[c + 1]) / 2 * unit, rng.uniform(5.3, 5.9)
        rows.append(_near(rng, bits, border, delta, top))
        deltas.append((border, delta, top))
    rows = np.array(rows, np.float32)
    assert np.array_equal(rows, _bf16(rows))
    qkv = normal_bf16(make_rng(7), (len(rows), 3 * 128)).astype(np.float32)
    qkv[:, 128:256] = rows
    one = np.ones(128, np.float32)
    kr = _want(rows, one)
    for r, (border, delta, top) in enumerate(deltas):      # the rows are what they are meant to be
        key = abs(kr[r, 0, 0 if top else 2])
        assert abs(key / border - 1 - delta) < 2.0 ** -46
    got, _ = _append(A, bits, qkv, one)
    want = M.rounded(kr, bits, -1)
    bad = np.unique(np.nonzero(got[:, 0, :32] != want[:, 0, :32])[0])
    assert not len(bad), [deltas[b] for b in bad[:8]]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,d,lat", [(12, 128, (30, 52)), (20, 64, (6, 12))])
def test_every_key_takes_the_nearest_code(A, bits, H, d, lat):
    """Two chunks of random projections near the stream's start, where the rotation's angles are exact to 2^-48: a
    key may only be off by what 64 bits leave open."""
    import torch
    D, T = H * d, lat[0] * lat[1]
    pool = Pool(A, H, d, lat, 1, bits, [T, T], seed=1, fill=0)
    pool.upload()
    rng = make_rng(201)
    qkv = normal_bf16(rng, (2 * T, 3 * D))
    g = dev_bf16(1 + 0.02 * normal_bf16(rng, (D,)))
    q = torch.empty((2 * T, D), dtype=torch.bfloat16, device="cuda")
    A.ardit_kv_append_mx(None, pool.dims, A.Batch([T, T], [0, 0], [0, 5]), dev_bf16(qkv), g, g, pool.kv(), q)
    _sync()
    pool.download()
    for b, pos in enumerate((0, 5)):
        x = qkv[b * T:(b + 1) * T, D:2 * D].astype(np.float64)
        kr = O.rope3d(O.rms_norm(x, EPS, host_f32(g)).reshape(T, H, d), O.chunk_positions(1, *lat, pos), 10000.0)
        got = pool.host.unpack(pool.ids[b][0])[0]
        assert np.all(np.abs(got - kr) - np.abs(M.rounded(kr, bits, -1) - kr) <= 1e-12)


@pytest.mark.parametrize("bits", [8, 4])
def test_projections_at_the_end_of_bf16(A, bits):
    """Keys of a usual size from projections near the largest bf16 number, whose product with the gain, as their
    square, is past fp32."""
    rng = np.random.default_rng(211)
    qkv = normal_bf16(make_rng(212), (64, 3 * 128)).astype(np.float32)
    rows = _bf16(rng.standard_normal((64, 128)).astype(np.float32))
    rows[::2] *= np.float32(2.0 ** 125)
    rows[5] = 0
    rows[5, 2] = -1.5 * 2.0 ** 127
    rows[7] = 2.0 ** 127
    qkv[:, 128:256] = rows
    gain = np.where(np.arange(128) % 2, 1.75, 3.0).astype(np.float32)
    kr = _want(rows, gain)
    assert np.isfinite(rows).all() and np.abs(kr).max() < 40
    got, q = _append(A, bits, qkv, gain)
    assert np.isfinite(host_f32(q)).all()
    assert np.all(np.abs(got - kr) - np.abs(M.rounded(kr, bits, -1) - kr) <= 1e-12)


@pytest.mark.parametrize("bits", [8, 4])
def test_projections_at_bf16s_small_end(A, bits):
    """Subnormal projections whose product with the gain is less than fp32 holds to its last bit, over a small eps."""
    rng = np.random.default_rng(213)
    qkv = normal_bf16(make_rng(214), (64, 3 * 128)).astype(np.float32)
    rows = np.ldexp(rng.integers(-127, 128, (64, 128)).astype(np.float32), -133)
    qkv[:, 128:256] = rows
    gain = _bf16(rng.uniform(1, 2, 128) * 2.0 ** -14)
    eps = float(np.float32(1e-36))
    kr = _want(rows, gain, eps)
    assert 2.0 ** -90 < np.abs(kr).max() < 2.0 ** -70
    got, _ = _append(A, bits, qkv, gain, eps)
    assert np.array_equal(got, M.rounded(kr, bits, -1))
