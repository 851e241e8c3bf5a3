"""Linear layers in 8-bit integers on the CPU: the reference's pins and the calls' refusals."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import int_ref as I
from workloads import normal_bf16

A = pytest.importorskip("paper_2606_15319_amd.ardit",
                        reason="libardit.so not built (python -m paper_2606_15319_amd.build)")
FAKE = 1 << 20


# ------------------------------------------------------------------ reference
def _rational(row):
    m = max(abs(Fraction(float(v))) for v in row)
    out = []
    for v in row:
        t = 127 * Fraction(float(v)) / m
        k = t.numerator // t.denominator
        rest = t - k
        out.append(k + (rest > Fraction(1, 2) or (rest == Fraction(1, 2) and k % 2 == 1)))
    return out


@pytest.mark.parametrize("kind", ["normal", "halves", "tiny", "huge"])
def test_codes_equal_those_of_rational_arithmetic(kind):
    rng = np.random.default_rng(3)
    x = normal_bf16(rng, (20, 37)).astype(np.float32)
    if kind == "halves":
        x = rng.integers(-254, 255, (20, 37)).astype(np.float32) * 0.5
        x[:, 5] = 127.0
    elif kind == "tiny":
        x = x * np.float32(1e-41)
    elif kind == "huge":
        x = x * np.float32(2.0 ** 124)
    codes, scales, _ = I.quantize(x)
    for r in range(len(x)):
        if np.abs(x[r]).max() > 0:
            assert codes[r].tolist() == _rational(x[r])
    assert np.array_equal(scales, (np.abs(x).max(1).astype(np.float64) / 127).astype(np.float32))


def test_rows_without_a_scale():
    x = np.ones((3, 4))
    x[0] = 0.0
    x[1, 2] = np.inf
    x[2, 0] = np.nan
    codes, scales, _ = I.quantize(x)
    assert not codes.any() and scales[0] == 0 and np.isnan(scales[1:]).all()


def test_worked_ties():
    codes, _, margin = I.quantize(np.array([[127.0, 63.5, 62.5, -0.5, -1.5, 126.5, 126.4]]))
    assert codes[0].tolist() == [127, 64, 62, 0, -2, 126, 126]
    assert margin[0, 1] == 0 and margin[0, 6] > 0.09


def test_values_of_codes_keep_their_codes():
    rng = np.random.default_rng(4)
    q = rng.integers(-127, 128, (9, 50))
    q[:, 0] = 127
    s = rng.uniform(0.01, 3.0, 9)
    codes, scales, _ = I.quantize(I.dequantize(q, s))
    assert np.array_equal(codes, q)
    assert np.allclose(scales, s, rtol=2.0 ** -23)


def test_product_by_loops():
    rng = np.random.default_rng(5)
    qx, qw = rng.integers(-127, 128, (3, 11)), rng.integers(-127, 128, (4, 11))
    sx, sw, b = rng.uniform(0.1, 1, 3), rng.uniform(0.1, 1, 4), rng.normal(size=4)
    got, _ = I.linear(qx, sx, qw, sw, b)
    for i in range(3):
        for j in range(4):
            s = sum(int(qx[i, k]) * int(qw[j, k]) for k in range(11))
            assert got[i, j] == pytest.approx(s * sx[i] * sw[j] + b[j], rel=1e-14)


# ------------------------------------------------------------------- refusals
def _status(fn, *a):
    with pytest.raises(A.ArditError) as e:
        fn(*a)
    return e.value.status


EINVAL, ESHAPE, ECAPACITY, EUNSUPPORTED = -1, -2, -3, -5


@pytest.mark.parametrize("change,status", [
    (dict(x=0), EINVAL), (dict(x=FAKE + 1), EINVAL), (dict(x=FAKE + 2, x_type=1), EINVAL), (dict(x_type=2), EINVAL),
    (dict(rows=-1), ESHAPE), (dict(rows=(1 << 22) + 1), ECAPACITY), (dict(cols=0), ESHAPE),
    (dict(cols=65537, ldx=65537, ldc=65552), ESHAPE), (dict(ldx=99), ESHAPE), (dict(ldx=(1 << 32) + 1), ESHAPE),
    (dict(codes=0), EINVAL), (dict(codes=FAKE + 8), EINVAL), (dict(ldc=96), ESHAPE), (dict(ldc=120), ESHAPE),
    (dict(ldc=(1 << 20) + 16), ESHAPE), (dict(scales=0), EINVAL), (dict(scales=FAKE + 2), EINVAL)])
def test_quantize_refuses(change, status):
    a = dict(x=FAKE, x_type=A.BF16, rows=4, cols=100, ldx=100, codes=FAKE, ldc=112, scales=FAKE)
    a.update(change)
    assert _status(A.ardit_int_quantize, 0, *a.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(codes=0), EINVAL), (dict(rows=-1), ESHAPE), (dict(cols=0), ESHAPE), (dict(ldc=100), ESHAPE),
    (dict(scales=0), EINVAL), (dict(y=0), EINVAL), (dict(y=FAKE + 1), EINVAL), (dict(y_type=7), EINVAL),
    (dict(ldy=99), ESHAPE)])
def test_dequantize_refuses(change, status):
    a = dict(codes=FAKE, rows=4, cols=100, ldc=112, scales=FAKE, y=FAKE, y_type=A.BF16, ldy=100)
    a.update(change)
    assert _status(A.ardit_int_dequantize, 0, *a.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(x=0), EINVAL), (dict(x_type=3), EINVAL), (dict(ldx=99), ESHAPE), (dict(delta=FAKE + 1, ldd=100), EINVAL),
    (dict(delta=FAKE, ldd=50), ESHAPE), (dict(h=FAKE + 2, ldh=100), EINVAL), (dict(h=FAKE << 1, ldh=99), ESHAPE),
    (dict(h=FAKE, ldh=100), EINVAL),                              # over a bf16 x
    (dict(x_type=1, h=FAKE, ldh=104), EINVAL),                    # over x with another stride
    (dict(delta=FAKE * 3, ldd=100, h=FAKE * 3, ldh=100), EINVAL),  # over a bf16 delta
    (dict(shift_row=6), EINVAL), (dict(scale_row=-2), EINVAL), (dict(scale_row=1), EINVAL),   # (no mod)
    (dict(gate_row=2, mod=FAKE), EINVAL),                         # no delta
    (dict(scale_row=1, mod=FAKE, rows_per_stream=0), EINVAL), (dict(scale_row=1, mod=FAKE + 2), EINVAL),
    (dict(scale_row=1, mod=FAKE, gain=FAKE), EINVAL), (dict(scale_row=1, mod=FAKE, mod_table=FAKE + 1), EINVAL),
    (dict(gain=FAKE + 1), EINVAL), (dict(eps=0.0), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(eps=1e-71), EINVAL), (dict(eps=1e301), EINVAL), (dict(eps=-1e-6), EINVAL)])
def test_norm_refuses(change, status):
    a = dict(x=FAKE, x_type=A.BF16, ldx=100)
    a.update(change)
    d = A.norm_desc(**a)
    assert _status(A.ardit_int_norm, 0, 4, 100, d, FAKE, 112, FAKE) == status


def test_norm_refuses_its_sizes_and_outputs():
    d = A.norm_desc(FAKE, A.BF16, 9000)
    for rows, dim, codes, ldc, scales, status in [(-1, 100, FAKE, 112, FAKE, ESHAPE), (4, 0, FAKE, 112, FAKE, ESHAPE),
                                                  (4, 8193, FAKE, 9008, FAKE, ESHAPE), (4, 100, 0, 112, FAKE, EINVAL),
                                                  (4, 100, FAKE, 100, FAKE, ESHAPE), (4, 100, FAKE, 112, 0, EINVAL),
                                                  ((1 << 22) + 1, 100, FAKE, 112, FAKE, ECAPACITY)]:
        assert _status(A.ardit_int_norm, 0, rows, dim, d, codes, ldc, scales) == status


@pytest.mark.parametrize("change,status", [
    (dict(m=-1), ESHAPE), (dict(m=(1 << 22) + 1), ECAPACITY), (dict(n=0), ESHAPE), (dict(n=(1 << 20) + 1), ESHAPE),
    (dict(k=0), ESHAPE), (dict(k=65537, ldx=65552, ldw=65552), ESHAPE), (dict(x_codes=0), EINVAL),
    (dict(x_codes=FAKE + 8), EINVAL), (dict(ldx=100), ESHAPE), (dict(ldw=104), ESHAPE), (dict(w_codes=0), EINVAL),
    (dict(x_scales=0), EINVAL), (dict(w_scales=0), EINVAL), (dict(bias=FAKE + 1), EINVAL), (dict(act=2), EINVAL),
    (dict(act=1, res=FAKE * 3, ldr=64), EUNSUPPORTED), (dict(res=FAKE * 3, ldr=63), ESHAPE),
    (dict(res=FAKE * 3, ldr=64, res_type=5), EINVAL), (dict(gate_row=2), EINVAL), (dict(gate_row=6), EINVAL),
    (dict(gate_row=2, res=FAKE * 3, ldr=64), EINVAL),             # no mod
    (dict(gate_row=2, res=FAKE * 3, ldr=64, mod=FAKE, rows_per_stream=0), EINVAL),
    (dict(res=FAKE * 2, ldr=64, res_type=1), EINVAL),             # y over res of another type
    (dict(res=FAKE * 2, ldr=72), EINVAL)])                        # ... or stride
def test_linear_refuses(change, status):
    a = dict(m=4, n=64, k=100, x_codes=FAKE, ldx=112, x_scales=FAKE, w_codes=FAKE, ldw=112, w_scales=FAKE)
    a.update(change)
    assert _status(A.ardit_int_linear, 0, A.linear_desc(**a), FAKE * 2, A.BF16, 64) == status


def test_linear_refuses_its_output():
    d = A.linear_desc(4, 64, 100, FAKE, 112, FAKE, FAKE, 112, FAKE)
    g = A.linear_desc(4, 64, 100, FAKE, 112, FAKE, FAKE, 112, FAKE, act=A.ACT_GELU)
    assert _status(A.ardit_int_linear, 0, d, 0, A.BF16, 64) == EINVAL
    assert _status(A.ardit_int_linear, 0, d, FAKE, A.BF16, 63) == ESHAPE
    assert _status(A.ardit_int_linear, 0, d, FAKE, 9, 64) == EINVAL
    assert _status(A.ardit_int_linear, 0, g, FAKE, A.F32, 64) == EUNSUPPORTED


def test_no_rows_is_no_work():
    A.ardit_int_quantize(0, None, A.BF16, 0, 100, 100, None, 112, None)
    A.ardit_int_dequantize(0, None, 0, 100, 112, None, None, A.F32, 100)
    A.ardit_int_norm(0, 0, 100, A.norm_desc(None, A.F32, 100), None, 112, None)
    A.ardit_int_linear(0, A.linear_desc(0, 64, 100, None, 112, None, FAKE, 112, FAKE), None, A.BF16, 64)


def _stack_args(**kw):
    dims = dict(dim=256, n_heads=4, head_dim=64, ffn_dim=1024, frames_per_chunk=3, lat_h=8, lat_w=8)
    dims.update({k: v for k, v in kw.items() if k in dims})
    d = A.make_dims(**dims)
    b = A.Batch([192], [384], [6], [32])
    n = A.ardit_workspace_size(d, b)
    names = [k for k in A._BLOCK_FIELDS if k not in A._INT_MATRICES]
    w = A.block_weights({k: FAKE for k in names if k != kw.get("without")})
    w8 = A.block_weights_int({k: FAKE for k in A._INT_MATRICES + A._INT_SCALES if k != kw.get("without8")})
    kv = A.kv_paged(FAKE, FAKE, FAKE, 9, 9)
    return [0, d, b, FAKE, [kv], FAKE, [FAKE], [FAKE], [w], [w8], FAKE * 2, FAKE, kw.get("ws_bytes", n)]


@pytest.mark.parametrize("change,status", [
    (dict(without="b_qkv"), EINVAL), (dict(without="mod_table"), EINVAL), (dict(without8="w_o"), EINVAL),
    (dict(without8="s_2"), EINVAL), (dict(ffn_dim=256 * 15 + 128), EUNSUPPORTED), (dict(ws_bytes=100), -4)])
def test_the_stack_refuses(change, status):
    # (matrices of the bf16 weights are NULL throughout: they are not read)
    assert _status(A.ardit_stack_fwd_int, *_stack_args(**change)) == status


def test_the_chunk_refuses():
    a = _stack_args(without8="s_qkv")
    tw = A.time_weights({k: FAKE for k in A._TIME_FIELDS})
    call = [0, a[1], a[2], [2], [[1000.0, 500.0]], FAKE, FAKE * 3, a[4], tw, a[6], a[7], a[8], a[9], FAKE * 512, FAKE, a[12]]
    assert _status(A.ardit_chunk_generate_int, *call) == EINVAL
