"""The microscaled key/value cache without a GPU: pins of its reference, and the
refusals of its entry points (the fake device addresses are never dereferenced,
every call fails a host check first)."""
import numpy as np
import pytest

from oracle import mxkv_ref as M
from oracle.ardit_ref import rms_norm  # noqa: F401

A = pytest.importorskip("paper_2606_15319_amd.ardit",
                        reason="libardit.so not built (python -m paper_2606_15319_amd.build)")

FAKE = 1 << 20


# ------------------------------------------------------------------- pins
def test_grids_from_the_formats():
    assert list(M.grid(4)) == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    g = M.grid(8)
    assert len(g) == 127 and g[0] == 0 and g[1] == 2.0 ** -9 and g[-1] == 448
    assert np.all(np.diff(g) > 0)


@pytest.mark.parametrize("bits,limit", [(8, 256.0), (4, 6.0)])
def test_exponent_is_the_smallest_that_fits(bits, limit):
    rng = np.random.default_rng(1)
    a = np.concatenate([2.0 ** rng.uniform(-100, 100, 500), 2.0 ** np.arange(-20, 20), 6 * 2.0 ** np.arange(-20, 20),
                        1.5 * 2.0 ** np.arange(-20, 20), np.nextafter(6 * 2.0 ** np.arange(-20, 20), np.inf)])
    for x in a:
        fits = (lambda e: x / 2.0 ** e < limit) if bits == 8 else (lambda e: x / 2.0 ** e <= limit)
        e = next(e for e in range(-140, 140) if fits(e))
        assert M.exponent(x, bits) == max(e, -117)
    assert M.exponent(0.0, bits) == -117 and M.exponent(1e-300, bits) == -117


def test_worked_ties():
    x = np.zeros(32)
    x[:9] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5]
    assert list(M.rounded(x, 4)[:9]) == [6, 0, 1, 1, 2, 2, 4, 4, -4]
    x = np.zeros(32)
    x[:5] = [255, 1.0625, 1.1875, 248, 136]      # e = 0: quantum 1/8 from 1, 16 from 128
    assert list(M.rounded(x, 8)[:5]) == [256, 1.0, 1.25, 256, 128]


@pytest.mark.parametrize("bits", [8, 4])
def test_round_trip_and_half_a_step(bits):
    rng = np.random.default_rng(2)
    x = rng.standard_normal((50, 3, 64)) * 2.0 ** rng.integers(-30, 30, (50, 3, 1))
    y = M.rounded(x, bits)
    assert np.array_equal(M.rounded(y, bits), y)              # what a code stands for is kept
    _, e = M.quantize(x, bits)
    g = M.grid(bits)
    top = 2 ** 4 if bits == 8 else 2                          # the step at the top of the range
    assert np.all(np.abs(y - x) <= np.ldexp(1.0, e) * top / 2)
    step = np.diff(g)[np.clip(np.searchsorted(g, np.abs(x) / np.ldexp(1.0, e)) - 1, 0, len(g) - 2)]
    assert np.all(np.abs(y - x) <= np.ldexp(step, e) / 2)


def test_short_last_block_zero_and_not_finite():
    x = np.ones(40)
    x[32:] = 3.0
    x[3] = np.inf
    y = M.rounded(x, 8)
    assert np.isnan(y[:32]).all() and np.array_equal(y[32:], x[32:])
    assert np.array_equal(M.rounded(np.zeros(5), 4), np.zeros(5))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("T,n", [(72, 72), (64, 64), (72, 65), (32, 1)])
def test_pages_pack_and_unpack(bits, T, n):
    rng = np.random.default_rng(3)
    H, d = 2, 64
    k, v = rng.standard_normal((2, n, H, d))
    p = M.Pages(3, H, d, T, bits)
    p.pack(1, k, v)
    ku, vu = p.unpack(1, n)
    assert np.array_equal(ku, M.rounded(k, bits, -1)) and np.array_equal(vu, M.rounded(v, bits, 0))
    assert (p.k_codes[[0, 2]] == 0xFF).all() and (p.v_scales[[0, 2]] == 0xFF).all()


# --------------------------------------------------------------- refusals
def _dims(**kw):
    d = dict(dim=256, n_heads=4, head_dim=64, ffn_dim=1024, frames_per_chunk=3, lat_h=8, lat_w=8)
    d.update(kw)
    return A.make_dims(**d)


def _mx(fmt=1, k=FAKE, ks=FAKE, v=FAKE, vs=FAKE, table=FAKE, n_pages=9, max_frames=9):
    return A.kv_mx(k, ks, v, vs, table, n_pages, max_frames, fmt)


def _kv(max_frames=9, n_pages=9):
    return A.kv_paged(FAKE, FAKE, FAKE, n_pages, max_frames)


def _status(fn, *args):
    with pytest.raises(A.ArditError) as e:
        fn(*args)
    return e.value.status


def test_bytes():
    d = _dims(lat_h=6, lat_w=12)                  # T = 72, two tiles
    assert A.ardit_kv_mx_bytes(d, A.KV_E4M3, 5) == (5 * 128 * 256, 5 * 128 * 8)
    assert A.ardit_kv_mx_bytes(d, A.KV_E2M1, 5) == (5 * 128 * 128, 5 * 128 * 8)
    assert _status(A.ardit_kv_mx_bytes, d, 0, 5) == -1
    assert _status(A.ardit_kv_mx_bytes, d, 1, 0) == -1
    assert _status(A.ardit_kv_mx_bytes, _dims(n_heads=3), 1, 1) == -2
    p = M.Pages(5, 4, 64, 72, 4)
    assert A.ardit_kv_mx_bytes(d, A.KV_E2M1, 5) == (p.k_codes.size, p.k_scales.size)
    assert A.ardit_kv_mx_bytes(d, A.KV_E2M1, 5) == (p.v_codes.size, p.v_scales.size)


BAD_POOLS = [(dict(fmt=0), -1), (dict(fmt=3), -1), (dict(k=0), -1), (dict(ks=0), -1), (dict(v=0), -1),
             (dict(vs=0), -1), (dict(table=0), -1), (dict(k=FAKE + 8), -1), (dict(ks=FAKE + 4), -1),
             (dict(v=FAKE + 2), -1), (dict(vs=FAKE + 1), -1), (dict(n_pages=0), -1),
             (dict(max_frames=0), -1), (dict(max_frames=8), -3), (dict(n_pages=1 << 30), -3)]


@pytest.mark.parametrize("kw,code", BAD_POOLS)
def test_bad_pools(kw, code):
    d = _dims()
    b = A.Batch([192], [384], [6])
    n = A.ardit_workspace_size(d, b)
    assert _status(A.ardit_kv_append_mx, FAKE, d, b, FAKE, FAKE, FAKE, _mx(**kw), FAKE) == code
    assert _status(A.ardit_kv_read_mx, FAKE, d, b, _mx(**kw), _kv()) == code
    assert _status(A.ardit_attn_fwd_mx, FAKE, d, b, FAKE, _mx(**kw), 0, FAKE, FAKE, n) == code


def test_append_refusals():
    d = _dims()
    ok = A.Batch([192], [384], [6])
    f = A.ardit_kv_append_mx
    assert _status(f, FAKE, d, A.Batch([100], [384], [6]), FAKE, FAKE, FAKE, _mx(), FAKE) == -2   # no chunk
    assert _status(f, FAKE, d, A.Batch([192], [100], [6]), FAKE, FAKE, FAKE, _mx(), FAKE) == -2   # no frames
    assert _status(f, FAKE, d, A.Batch([192], [384], [-1]), FAKE, FAKE, FAKE, _mx(), FAKE) == -1
    assert _status(f, FAKE, d, A.Batch([192], [384]), FAKE, FAKE, FAKE, _mx(), FAKE) == -1        # no positions
    for i in range(4):
        for bad in (0, FAKE + 8):
            p = [FAKE] * 4
            p[i] = bad
            assert _status(f, FAKE, d, ok, p[0], p[1], p[2], _mx(), p[3]) == -1


def test_read_refusals():
    d = _dims()
    f = A.ardit_kv_read_mx
    assert _status(f, FAKE, d, A.Batch([10], [100]), _mx(), _kv()) == -2
    assert _status(f, FAKE, d, A.Batch([-1], [64]), _mx(), _kv()) == -2
    assert _status(f, FAKE, d, A.Batch([600], [0]), _mx(max_frames=10, n_pages=10), _kv()) == -3
    assert _status(f, FAKE, d, A.Batch([10], [64]), _mx(), A.kv_paged(0, FAKE, FAKE, 9, 9)) == -1
    assert _status(f, FAKE, d, A.Batch([10], [64]), _mx(), A.kv_paged(FAKE + 2, FAKE, FAKE, 9, 9)) == -1


def test_attention_refusals():
    d = _dims()
    b = A.Batch([5, 0, 7], [384, 0, 192])
    n = A.ardit_workspace_size(d, b)
    f = A.ardit_attn_fwd_mx

    def call(batch=b, q=FAKE, shared=0, o=FAKE, ws=FAKE, nbytes=n, kv=None, dims=d):
        return _status(f, FAKE, dims, batch, q, kv or _mx(), shared, o, ws, nbytes)

    assert call(shared=-1) == -1
    assert call(shared=4) == -2                  # stream 2 caches three frames; stream 1 has no queries
    assert call(shared=1 << 30) == -2
    assert call(nbytes=n - 1) == -4
    assert call(q=0) == -1 and call(o=0) == -1 and call(ws=0) == -1
    assert call(q=FAKE + 8) == -1 and call(o=FAKE + 2) == -1 and call(ws=FAKE + 16) == -1
    assert call(batch=A.Batch([5], [384], sparsity=[0.5])) == -5
    assert call(batch=A.Batch([5], [384], sparsity=[1.5])) == -1
    assert call(batch=A.Batch([5], [100])) == -2
    wide = _dims(dim=512, head_dim=128)
    assert call(dims=wide, batch=A.Batch([5], [384], quant=[1]), nbytes=1 << 40) == -5
    # T = 32: 2^30 keys and half of every tile is padding
    small = _dims(lat_h=4, lat_w=8)
    assert call(dims=small, batch=A.Batch([5], [1 << 30]), nbytes=1 << 40,
                kv=_mx(max_frames=1 << 26)) == -3


def _stack(batch=None, kv=None, dims=None, nbytes=1 << 40, x=FAKE, out=FAKE + 4096, mod=FAKE, ctx=FAKE):
    d = dims or _dims()
    w = A.block_weights({k: FAKE for k in A._BLOCK_FIELDS})
    b = batch or A.Batch([192], [384], [6], [32])
    A.ardit_stack_fwd_mx(FAKE, d, b, x, [kv or _mx()], mod, [ctx], [ctx], [w], out, FAKE, nbytes)


def _chunk(batch=None, kv=None, steps=(2,), ts=((900.0, 400.0),), x0=1 << 30, nbytes=1 << 28, noise=FAKE):
    d = _dims()
    w = A.block_weights({k: FAKE for k in A._BLOCK_FIELDS})
    tw = A.time_weights({k: FAKE for k in A._TIME_FIELDS})
    b = batch or A.Batch([192], [384], [6], [32])
    A.ardit_chunk_generate_mx(FAKE, d, b, list(steps), ts, FAKE, noise, [kv or _mx()], tw, [FAKE], [FAKE], [w], x0,
                              FAKE, nbytes)


@pytest.mark.parametrize("call", [_stack, _chunk])
def test_model_path_refusals(call):
    assert _status(lambda: call(kv=_mx(fmt=7))) == -1
    assert _status(lambda: call(kv=_mx(vs=0))) == -1
    assert _status(lambda: call(kv=_mx(max_frames=8))) == -3
    assert _status(lambda: call(batch=A.Batch([192], [384], [6], [32], sparsity=[0.5]))) == -5
    assert _status(lambda: call(batch=A.Batch([100], [384], [6], [32]))) == -2
    assert _status(lambda: call(batch=A.Batch([192], [100], [6], [32]))) == -2
    assert _status(lambda: call(batch=A.Batch([192], [384], [6], [0]))) == -2
    assert _status(lambda: call(nbytes=1024)) == -4


def test_stack_and_chunk_refusals():
    assert _status(lambda: _stack(x=FAKE, out=FAKE)) == -1
    assert _status(lambda: _stack(mod=0)) == -1
    assert _status(lambda: _stack(ctx=0)) == -1
    wide = _dims(dim=512, head_dim=128)
    assert _status(lambda: _stack(dims=wide, batch=A.Batch([192], [384], [6], [32], quant=[1]))) == -5
    assert _status(lambda: _chunk(steps=(17,), ts=((0.0,) * 17,))) == -1
    assert _status(lambda: _chunk(ts=((900.0, 1400.0),))) == -1
    assert _status(lambda: _chunk(noise=0)) == -1
    assert _status(lambda: _chunk(x0=FAKE)) == -1            # over x_init
