"""Linear layers in 8-bit integers on the GPU against their float64 reference.

Tolerances, in units of u = 2^-24 (half a step of fp32):
  - codes of given rows, their scales, values read back: equal;
  - a norm's codes: equal wherever 127 |y| / m of the reference lies further than 1e-9 from a
    half (both sides compute y in fp64), and next to it one of the two;
  - a product p = sum sx sw: the sum's conversion, two products: 3 u |p|; the bias: u |z|; a
    gate: its own rounding u and the fma's; bf16 half a step more (2^-8 of the value);
  - GELU: its slope is at most 1.13, and z sigmoid(2 v) through exp2 and a reciprocal of 2 steps
    each whose argument is off by 6 u: (8 + 14 |v|) u of the value, v = 0.798 (z + 0.0447 z^3).
"""
import numpy as np
import pytest

from harness import dev_bf16, dev_f32, host_f32
from oracle import int_ref as I
from workloads import bf16_round, normal_bf16

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
GUARD = 0x55


@pytest.fixture(scope="module")
def A(gpu):
    from paper_2606_15319_amd import ardit
    return ardit


def _sync():
    import torch
    torch.cuda.synchronize()


def _strided(a, f32, ld, shift=0, fill=np.nan):
    """Rows of a on the device, ld elements apart, starting `shift` elements into their buffer."""
    import torch
    rows, cols = a.shape
    whole = np.full(shift + rows * ld, fill, np.float32)
    v = whole[shift:shift + rows * ld].reshape(rows, ld)
    v[:, :cols] = a
    t = (dev_f32 if f32 else dev_bf16)(whole)
    return t, t[shift:] if rows * ld else t


class Codes:
    """Codes and scales on the device, guarded on all sides."""

    def __init__(self, rows, cols, extra=0):
        import torch
        self.rows, self.cols, self.pad = rows, cols, -(-cols // 16) * 16
        self.ld = self.pad + extra
        self.all = torch.full((rows + 2, self.ld), GUARD, dtype=torch.int8, device="cuda")
        self.s_all = torch.full((rows + 2,), -7.0, dtype=torch.float32, device="cuda")
        self.q, self.s = self.all[1:], self.s_all[1:]

    def host(self):
        _sync()
        q, s = self.all.cpu().numpy(), self.s_all.cpu().numpy()
        assert (q[0] == GUARD).all() and (q[-1] == GUARD).all() and (q[:, self.pad:] == GUARD).all()
        assert s[0] == -7.0 and s[-1] == -7.0
        assert not q[1:-1, self.cols:self.pad].any()
        return q[1:-1, :self.cols], s[1:-1]


def _rows(kind, rows, cols, f32, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols))
    if kind == "ties":      # whole and half numbers under a maximum of 127
        x = rng.integers(-253, 254, (rows, cols)) * 0.5
        x[:, cols // 2] = 127.0
    elif kind == "tiny":
        x = x * 2.0 ** -138
    elif kind == "huge":
        x = x * 2.0 ** 124
    elif kind == "odd":     # rows of zeros, infinities, NaN, one element
        x[0::5] = 0.0
        x[1::5, 0] = np.inf
        x[2::5, cols - 1] = np.nan
        x[3::5] = 0.0
        x[3::5, cols // 3] = -1e-3
    x = x.astype(np.float32)
    return x if f32 else bf16_round(x).astype(np.float32)


QUANTIZE = [(1, 1, 0, 0), (3, 7, 0, 0), (5, 16, 0, 0), (2, 17, 3, 1), (9, 256, 0, 0), (33, 520, 8, 0), (6, 1315, 13, 0),
            (4, 2049, 0, 1), (4, 2056, 0, 0), (3, 8192, 0, 0), (2, 13824, 8, 8), (5, 16392, 0, 0), (1, 65536, 0, 0),
            (3, 65533, 3, 0)]


@pytest.mark.parametrize("kind", ["normal", "ties", "tiny", "huge", "odd"])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,cols,pad,shift", QUANTIZE)
def test_quantize_and_read_back(A, rows, cols, pad, shift, f32, kind):
    import torch
    x = _rows(kind, rows, cols, f32, rows * cols)
    keep, xd = _strided(x, f32, cols + pad, shift)
    c = Codes(rows, cols, extra=16 * (pad > 0))
    A.ardit_int_quantize(None, xd, A.F32 if f32 else A.BF16, rows, cols, cols + pad, c.q, c.ld, c.s)
    q, s = c.host()
    want, ws, _ = I.quantize(x)
    assert np.array_equal(q, want)
    assert np.array_equal(s, ws, equal_nan=True)
    for y_f32 in (False, True):
        y = torch.full((rows + 1, cols + pad), 3.0, dtype=torch.float32 if y_f32 else torch.bfloat16, device="cuda")
        A.ardit_int_dequantize(None, c.q, rows, cols, c.ld, c.s, y, A.F32 if y_f32 else A.BF16, cols + pad)
        _sync()
        got = host_f32(y)
        v = q.astype(np.float32) * s[:, None]
        if not y_f32:
            v = np.where(np.isnan(v), v, bf16_round(np.nan_to_num(v)))
        assert np.array_equal(got[:rows, :cols], v.astype(np.float32), equal_nan=True)
        assert (got[rows] == 3.0).all() and (got[:, cols:] == 3.0).all()


def _check_norm(A, rows, dim, f32=False, delta="", gate=False, by="gain", per=None, keep=True, pad=0, kind="normal",
                table=True, eps=1e-6, over=""):
    import torch
    rng = np.random.default_rng(rows * 7 + dim)
    x = _rows(kind, rows, dim, f32, rows + dim) if kind != "loud" else None
    if x is None:
        x = 3.0 * rng.standard_normal((rows, dim)) * np.where(rng.random(dim) < 0.02, 20, 1)
        x = x.astype(np.float32) if f32 else bf16_round(x.astype(np.float32)).astype(np.float32)
    per = per or rows
    streams = -(-rows // per)
    ld = dim + pad
    _, xd = _strided(x, f32, ld)
    mod = (0.3 * rng.standard_normal((streams, 6, dim))).astype(np.float32)
    tab = (0.02 * rng.standard_normal((6, dim))).astype(np.float32)
    gain = bf16_round((1 + 0.1 * rng.standard_normal(dim)).astype(np.float32)).astype(np.float32)
    md, td, gd = dev_f32(mod), dev_f32(tab), dev_bf16(gain)
    kw = {}
    row_of = np.arange(rows) // per

    def vector(r):
        return (mod[:, r] + tab[r] if table else mod[:, r])[row_of].astype(np.float64)

    h = x.astype(np.float64)
    if delta:
        d = rng.standard_normal((rows, dim)).astype(np.float32)
        if delta == "bf16":
            d = bf16_round(d).astype(np.float32)
        _, dd = _strided(d, delta == "f32", ld)
        kw.update(delta=dd, delta_type=A.F32 if delta == "f32" else A.BF16, ldd=ld)
        if gate:
            kw.update(gate_row=5)
        h = h + (vector(5) * d.astype(np.float64) if gate else d.astype(np.float64))
    hd = None
    if keep:
        hd = {"": torch.full((rows, ld), 9.0, dtype=torch.float32, device="cuda"), "x": xd, "delta": kw.get("delta")}[over]
        kw.update(h=hd, ldh=ld)
    if by == "gain":
        kw.update(gain=gd)
    if by in ("mod", "scale"):
        kw.update(scale_row=1)
    if by in ("mod", "shift"):
        kw.update(shift_row=3)
    if by != "gain" and by != "plain" or gate:
        kw.update(mod=md, mod_table=td if table else None, rows_per_stream=per)
    desc = A.norm_desc(xd, A.F32 if f32 else A.BF16, ld, eps=eps, **kw)
    c = Codes(rows, dim, extra=16 * (pad > 0))
    A.ardit_int_norm(None, rows, dim, desc, c.q, c.ld, c.s)
    q, s = c.host()
    with np.errstate(invalid="ignore", over="ignore"):
        h32 = h.astype(np.float32)
    if keep:
        got = host_f32(hd).ravel()[:rows * ld].reshape(rows, ld)
        if not over:
            assert (got[:, dim:] == 9.0).all()
        got = got[:, :dim]
        # one rounding, of a sum that fp64 may already have rounded
        step = np.spacing(np.abs(h32).astype(np.float32)).astype(np.float64)
        with np.errstate(invalid="ignore"):
            ok = (np.abs(got - h) <= 0.5 * step * (1 + 1e-6)) | (got == h32) | (np.isnan(got) & np.isnan(h32))
        assert ok.all()
        h32 = got
    with np.errstate(invalid="ignore", over="ignore"):
        y = I.norm(h32, eps, gain if by == "gain" else None, vector(1) if by in ("mod", "scale") else None,
                   vector(3) if by in ("mod", "shift") else None)
        want, ws, margin = I.quantize(y)
    sure = margin > 1e-9
    assert np.array_equal(q[sure], want[sure]), (np.argwhere((q != want) & sure)[:4], rows, dim)
    assert (np.abs(q.astype(int) - want)[~sure] <= 1).all()
    assert np.array_equal(np.isnan(s), np.isnan(ws))
    fin = ~np.isnan(ws)
    assert (np.abs(s[fin].astype(np.float64) - ws[fin]) <= np.spacing(ws[fin])).all()


@pytest.mark.parametrize("by", ["gain", "mod", "scale", "shift", "plain"])
@pytest.mark.parametrize("rows,dim,pad", [(1, 1, 0), (3, 8, 0), (9, 100, 0), (17, 256, 8), (5, 1000, 0), (2, 1536, 0),
                                          (11, 2051, 2), (9, 5120, 0), (3, 8192, 0), (2, 8185, 0)])
def test_norm(A, rows, dim, pad, by):
    _check_norm(A, rows, dim, by=by, pad=pad, keep=False)


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("delta", ["bf16", "f32"])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,dim,pad,by,per", [(1, 64, 0, "gain", None), (24, 257, 0, "mod", 8), (23, 512, 8, "mod", 5),
                                                 (6, 1536, 0, "mod", 1), (10, 5120, 0, "mod", 7), (3, 8192, 0, "mod", None)])
def test_norm_of_a_sum(A, rows, dim, pad, by, per, f32, delta, gate):
    _check_norm(A, rows, dim, f32=f32, delta=delta, gate=gate, by=by, per=per, pad=pad, kind="loud")


def test_norm_halves_go_to_the_even_code(A):
    """With a gain or alone the codes are those of h gain, exactly: a half of the largest is 63.5, and becomes 64."""
    import torch
    rng = np.random.default_rng(9)
    rows, D = 200, 512
    h = bf16_round(rng.standard_normal((rows, D)).astype(np.float32)).astype(np.float32)
    gain = bf16_round((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)).astype(np.float32)
    gain[[0, 1]] = gain[2]
    h[:, 2] = np.abs(h * gain).max(1) * 2
    h = bf16_round(h).astype(np.float32)
    h[:, 0], h[:, 1] = h[:, 2] / 2, -h[:, 2] / 2
    for g in (gain, None):
        c = Codes(rows, D)
        xd, gd = dev_bf16(h), dev_bf16(gain)
        A.ardit_int_norm(None, rows, D, A.norm_desc(xd, A.BF16, D, gain=gd if g is not None else None), c.q, D, c.s)
        q, _ = c.host()
        want, _, _ = I.quantize(h.astype(np.float64) * (gain if g is not None else 1.0))
        assert np.array_equal(q, want)
        assert (q[:, 0] == np.sign(h[:, 2]) * 64).all() and (q[:, 1] == -np.sign(h[:, 2]) * 64).all()


@pytest.mark.parametrize("over", ["x", "delta"])
def test_norm_in_place(A, over):
    _check_norm(A, 13, 640, f32=True, delta="f32", gate=True, by="mod", per=4, over=over)
    _check_norm(A, 5, 77, f32=True, delta="f32", by="mod", per=4, over=over)


@pytest.mark.parametrize("kind", ["odd", "tiny", "huge", "ties"])
@pytest.mark.parametrize("by", ["gain", "mod", "plain", "scale"])
@pytest.mark.parametrize("f32", [False, True])
def test_norm_of_unusual_rows(A, kind, by, f32):
    _check_norm(A, 10, 384, f32=f32, by=by, kind=kind, keep=False)
    _check_norm(A, 10, 77, f32=f32, by=by, kind=kind, keep=False, table=False)


@pytest.mark.parametrize("kind", ["odd", "tiny", "huge"])
@pytest.mark.parametrize("by", ["gain", "mod", "plain", "shift"])
@pytest.mark.parametrize("eps", [1e-70, 1e4])
def test_norm_with_the_ends_of_eps(A, kind, by, eps):
    """Rows of zeros and of subnormal numbers beside 1 / rms at both ends."""
    _check_norm(A, 10, 384, f32=True, by=by, kind=kind, keep=False, eps=eps)


def test_norm_too_small_for_a_scale(A):
    """1 / rms of 1e-150: y is 0 in 32 bits, so the scale is; with a shift y is the shift."""
    x = np.random.default_rng(4).standard_normal((7, 300)).astype(np.float32)
    mod = np.random.default_rng(5).standard_normal((1, 6, 300)).astype(np.float32)
    xd, md = dev_f32(x), dev_f32(mod)
    c = Codes(7, 300)
    A.ardit_int_norm(None, 7, 300, A.norm_desc(xd, A.F32, 300, eps=1e300), c.q, c.ld, c.s)
    assert (c.host()[1] == 0.0).all()
    A.ardit_int_norm(None, 7, 300, A.norm_desc(xd, A.F32, 300, mod=md, rows_per_stream=7, shift_row=3, eps=1e300),
                     c.q, c.ld, c.s)
    q, s = c.host()
    want, ws, margin = I.quantize(np.broadcast_to(mod[:, 3], (7, 300)).astype(np.float64))
    assert np.array_equal(q[margin > 1e-9], want[margin > 1e-9])
    assert (np.abs(s.astype(np.float64) - ws) <= np.spacing(ws)).all()


def test_norm_whose_terms_cancel(A):
    """Shift against scale: y is small beside its terms, where fp32 alone would take other codes."""
    import torch
    rng = np.random.default_rng(8)
    D, rows = 1024, 6
    x = rng.standard_normal((rows, D)).astype(np.float32)
    x[1:] = x[0] * 2.0 ** np.arange(1, rows)[:, None]
    u = x[0].astype(np.float64) / np.sqrt((x[0].astype(np.float64) ** 2).mean() + 1e-30)
    mod = np.zeros((1, 6, D), np.float32)
    mod[0, 0] = (-u * (1 + 1e-5 * rng.standard_normal(D))).astype(np.float32)
    c = Codes(rows, D)
    xd, md = dev_f32(x), dev_f32(mod)
    d = A.norm_desc(xd, A.F32, D, mod=md, rows_per_stream=rows, shift_row=0, eps=1e-30)
    A.ardit_int_norm(None, rows, D, d, c.q, c.ld, c.s)
    q, s = c.host()
    want, ws, margin = I.quantize(I.norm(x, 1e-30, shift=mod[0, 0]))
    sure = margin > 1e-8        # (fp64 steps of 1e-16 beside y of 1e-5: 1e-11 of m, 127 of them)
    assert sure.mean() > 0.999 and np.array_equal(q[sure], want[sure])


def _norm_of(A, x, eps, gain=None, scale=None, shift=None):
    """Codes and scales of rows x (fp32) beside those of the reference, vectors shared by all rows."""
    rows, D = x.shape
    mod = np.zeros((1, 6, D), np.float32)
    kw = {}
    keep = [dev_f32(x)]
    if gain is not None:
        keep.append(dev_bf16(gain))
        kw.update(gain=keep[-1])
    if scale is not None:
        mod[0, 1] = scale
        kw.update(scale_row=1)
    if shift is not None:
        mod[0, 3] = shift
        kw.update(shift_row=3)
    keep.append(dev_f32(mod))
    if scale is not None or shift is not None:
        kw.update(mod=keep[-1], rows_per_stream=rows)
    c = Codes(rows, D)
    A.ardit_int_norm(None, rows, D, A.norm_desc(keep[0], A.F32, D, eps=eps, **kw), c.q, c.ld, c.s)
    q, s = c.host()
    with np.errstate(over="ignore"):
        want, ws, margin = I.quantize(I.norm(x, eps, gain, scale, shift))
    sure = margin > 1e-9
    assert np.array_equal(q[sure], want[sure]), (int((q != want)[sure].sum()), int(sure.sum()))
    assert (np.abs(q.astype(int) - want)[~sure] <= 1).all()
    assert (np.abs(s.astype(np.float64) - ws) <= np.spacing(ws)).all()
    return q, s


@pytest.mark.parametrize("by", ["gain", "scale", "mod"])
@pytest.mark.parametrize("h,eps,vec", [(1e-22, 1e40, 1e6), (1e-21, 1e40, 3e5), (1e-43, 1e-6, 3e5), (1e-22, 1e40, 1e10),
                                       (1e-30, 1e32, 1e30), (1e-26, 1e40, 1e14), (1e30, 1e80, 1.0), (1e30, 1e92, 1.0),
                                       (1e-20, 1e40, 1e4)])
def test_norm_whose_unit_is_no_normal_number(A, h, eps, vec, by):
    """h / rms or 1 / rms below 2^-126, where 32 bits hold few of its bits or none, in rows whose y is a
    normal number."""
    rng = np.random.default_rng(12)
    rows, D = 20, 1024
    x = (h * rng.standard_normal((rows, D))).astype(np.float32)
    x[3] = 0.0
    v = (vec * rng.standard_normal(D)).astype(np.float32)
    if by == "gain":
        _norm_of(A, x, eps, gain=bf16_round(v).astype(np.float32))
    else:
        shift = (h / eps ** 0.5 * vec * rng.standard_normal(D)).astype(np.float32)
        _norm_of(A, x, eps, scale=v, shift=shift if by == "mod" else None)


@pytest.mark.parametrize("eps", [1e85, 1e300])
def test_norm_too_small_for_a_scale_has_its_codes(A, eps):
    """m / 127 of about 1e-44 (a few of fp32's least steps) and of 1e-152 (the scale is 0)."""
    x = np.random.default_rng(6).standard_normal((9, 300)).astype(np.float32)
    q, s = _norm_of(A, x, eps)
    assert (np.abs(q).max(1) == 127).all() and (s == 0).all() == (eps > 1e90)


def test_norm_of_subnormal_rows_below_a_scale(A):
    """1 / rms is a normal number, h / rms 1e-50: 0 in 32 bits throughout, with scales of up to 2^20 too."""
    x = (1e-40 * np.random.default_rng(7).standard_normal((9, 300))).astype(np.float32)
    for scale in (None, (1e5 * np.random.default_rng(8).standard_normal(300)).astype(np.float32)):
        q, s = _norm_of(A, x, 1e20, scale=scale)
        assert (np.abs(q).max(1) == 127).all() and not s.any()


def test_norm_whose_terms_pass_the_range(A):
    """u (1 + scale) past fp32's largest number, which the shift brings back: y is a number, and has codes.
    Without the shift, or with one of the other sign, y is an infinity."""
    rng = np.random.default_rng(21)
    rows, D = 5, 264
    x = rng.standard_normal((1, D)).astype(np.float32)
    x[0, :40] *= 4
    x = x * np.float32(2.0) ** np.arange(rows, dtype=np.float32)[:, None]
    u = (x[0].astype(np.float64) / np.sqrt((x[0].astype(np.float64) ** 2).mean()))
    far = np.argsort(-np.abs(u))[:7]
    scale = rng.standard_normal(D).astype(np.float32)
    shift = (1e38 * rng.standard_normal(D)).clip(-2e38, 2e38).astype(np.float32)
    scale[far] = (5e38 / u[far]).astype(np.float32)       # p = 5e38
    shift[far] = -3e38 + 1e37 * np.arange(7, dtype=np.float32)
    _norm_of(A, x, 1e-30, scale=scale, shift=shift)
    for other in (None, -shift):
        c = Codes(rows, D)
        mod = np.zeros((1, 6, D), np.float32)
        mod[0, 1] = scale
        if other is not None:
            mod[0, 3] = other
        xd, md = dev_f32(x), dev_f32(mod)
        A.ardit_int_norm(None, rows, D, A.norm_desc(xd, A.F32, D, eps=1e-30, mod=md, rows_per_stream=rows, scale_row=1,
                                                    shift_row=-1 if other is None else 3), c.q, c.ld, c.s)
        q, s = c.host()
        assert np.isnan(s).all() and not q.any()


# ---------------------------------------------------------------------- linear
def _linear_case(A, M, N, K, epi="bias", out="bf16", res="f32", per=None, pad=0, seed=0, ends=False, bias=True):
    import torch
    rng = np.random.default_rng(seed + M * 31 + N * 7 + K)
    kp = -(-K // 16) * 16
    qx, qw = rng.integers(-127, 128, (M, K)), rng.integers(-127, 128, (N, K))
    if ends:
        qx[:], qw[:] = -128, -128
    sx = (rng.uniform(0.5, 2, M) * 0.01).astype(np.float32)
    sw = (rng.uniform(0.5, 2, N) * 0.01).astype(np.float32)
    b = bf16_round(rng.standard_normal(N).astype(np.float32)).astype(np.float32)
    ldx, ldw, ldy = kp + 16 * pad, kp + 32 * pad, N + 3 * pad

    def codes(q, ld, junk):
        a = rng.integers(-128, 128, (q.shape[0], ld))
        a[:, :K] = q
        if not junk:            # zeros in one of the two are enough
            a[:, K:kp] = 0
        return torch.from_numpy(a.astype(np.int8)).to("cuda")

    t = {"x": codes(qx, ldx, True), "w": codes(qw, ldw, False), "sx": dev_f32(sx), "sw": dev_f32(sw), "b": dev_bf16(b)}
    kw = {}
    r = g = None
    if epi in ("res", "gate"):
        r = rng.standard_normal((M, N)).astype(np.float32)
        if res == "bf16":
            r = bf16_round(r).astype(np.float32)
        _, t["r"] = _strided(r, res == "f32", N + 5 * pad)
        kw.update(res=t["r"], res_type=A.F32 if res == "f32" else A.BF16, ldr=N + 5 * pad)
    if epi == "gate":
        per = per or M
        mod = rng.standard_normal((-(-M // per), 6, N)).astype(np.float32)
        tab = rng.standard_normal((6, N)).astype(np.float32)
        t["m"], t["t"] = dev_f32(mod), dev_f32(tab)
        kw.update(mod=t["m"], mod_table=t["t"], gate_row=2, rows_per_stream=per)
        g = (mod[:, 2].astype(np.float64) + tab[2])[np.arange(M) // per]
    desc = A.linear_desc(M, N, K, t["x"], ldx, t["sx"], t["w"], ldw, t["sw"], bias=t["b"] if bias else None,
                         act=A.ACT_GELU if epi == "gelu" else A.ACT_NONE, **kw)
    y = torch.full((M + 1, ldy), 5.0, dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    A.ardit_int_linear(None, desc, y, A.F32 if out == "f32" else A.BF16, ldy)
    _sync()
    got = host_f32(y)
    assert (got[M] == 5.0).all() and (got[:, N:] == 5.0).all()
    got = got[:M, :N].astype(np.float64)
    bb = b.astype(np.float64) if bias else 0.0
    want, p = I.linear(qx, sx, qw, sw, bb, epi == "gelu", r, g)
    z = p + bb
    tol = 3.1 * U * np.abs(p) + 1.1 * U * np.abs(z)
    if epi == "gelu":
        v = np.abs(0.7978845608 * (z + 0.044715 * z ** 3))
        tol = 1.13 * tol + (8 + 14 * v) * U * np.abs(want) + 1e-36
    elif epi == "res":
        tol = tol + 1.1 * U * np.abs(want)
    elif epi == "gate":
        tol = np.abs(g) * tol + 1.1 * U * (np.abs(g * z) + np.abs(want))
    if out == "bf16":
        tol = tol * 1.01 + 2.0 ** -8 * np.abs(want)
    err = np.abs(got - want)
    assert (err <= tol).all(), (float((err / (tol + 1e-300)).max()), np.argwhere(err > tol)[:4].tolist())
    return got


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 64, 130, 300])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 16), (64, 128), (100, 100), (129, 129), (257, 1000), (516, 240), (1536, 384)])
def test_linear_sizes(A, M, N, K):
    _linear_case(A, M, N, K, out="f32")
    _linear_case(A, M, N, K, out="bf16", pad=1, epi="gelu")


@pytest.mark.parametrize("epi,out,res", [("bias", "bf16", ""), ("bias", "f32", ""), ("gelu", "bf16", "")] +
                         [(e, o, r) for e in ("res", "gate") for o in ("bf16", "f32") for r in ("bf16", "f32")])
@pytest.mark.parametrize("M,N,K,pad", [(1, 256, 512, 0), (7, 130, 70, 1), (24, 640, 1280, 0), (70, 384, 256, 0),
                                       (200, 520, 144, 1), (389, 1280, 640, 0), (521, 776, 272, 0)])
def test_linear_results(A, M, N, K, pad, epi, out, res):
    _linear_case(A, M, N, K, epi=epi, out=out, res=res, pad=pad, per=max(1, M // 3))


@pytest.mark.parametrize("M,N,K", [(1, 640, 13824), (40, 200, 8960), (260, 300, 4096), (5, 64, 65536), (130, 129, 65535)])
def test_linear_long(A, M, N, K):
    _linear_case(A, M, N, K, out="f32")
    _linear_case(A, M, N, K, out="f32", ends=True, bias=False)


# sizes that reach every tile of the large products, with steps of K from one to many and cut short
@pytest.mark.parametrize("M,N,K", [(130, 129, 1000), (389, 1280, 640), (500, 1500, 1600), (300, 5000, 2000),
                                   (2000, 1990, 1315), (1000, 5120, 144), (1500, 4500, 300), (3000, 5000, 128),
                                   (2400, 4000, 272), (4000, 2600, 260), (9000, 3900, 200), (2890, 5125, 400),
                                   (2800, 5120, 1290), (2500, 640, 256), (4680, 300, 128)])
def test_linear_tiles(A, M, N, K):
    _linear_case(A, M, N, K, epi="gate", out="bf16", per=1000)
    _linear_case(A, M, N, K, out="f32", bias=False, pad=1)


# one to four blocks of 16 columns a workgroup, over more and fewer steps of K than it has waves
@pytest.mark.parametrize("K", [150, 1300])
@pytest.mark.parametrize("M", [1, 16, 20, 50, 64])
@pytest.mark.parametrize("N", [4000, 4100, 8200, 12300, 17001])
def test_linear_few_rows(A, M, N, K):
    _linear_case(A, M, N, K, epi="res", out="f32", res="f32")


def test_linear_scales_at_their_ends(A):
    """Scales whose product leaves fp32 although the result does not; zero and NaN rows."""
    import torch
    K, N = 256, 128
    rng = np.random.default_rng(2)
    qx, qw = rng.integers(-127, 128, (6, K)), rng.integers(-127, 128, (N, K))
    sx = np.array([3e36, 1e-40, 1.0, 0.0, np.nan, 2e-38], np.float32)
    sw = np.full(N, 1e-30, np.float32)
    sw[::2] = 1e5
    sw[0] = np.nan
    t = [torch.from_numpy(a.astype(np.int8)).to("cuda") for a in (qx, qw)] + [dev_f32(sx), dev_f32(sw)]
    d = A.linear_desc(6, N, K, t[0], K, t[2], t[1], K, t[3])
    y = torch.empty((6, N), dtype=torch.float32, device="cuda")
    A.ardit_int_linear(None, d, y, A.F32, N)
    _sync()
    got = host_f32(y).astype(np.float64)
    want = I.product(qx, sx, qw, sw)
    with np.errstate(over="ignore"):
        w32 = want.astype(np.float32)
    fine = np.isfinite(w32)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[np.isinf(w32)], w32[np.isinf(w32)])
    assert (np.abs(got - want)[fine] <= 3.1 * U * np.abs(want[fine]) + 2.0 ** -149).all()


def test_residual_in_place(A):
    import torch
    M, N, K = 150, 384, 256
    rng = np.random.default_rng(6)
    q = [torch.from_numpy(rng.integers(-127, 128, s).astype(np.int8)).to("cuda") for s in ((M, K), (N, K))]
    s = [dev_f32(rng.uniform(0.001, 0.002, n)) for n in (M, N)]
    r = dev_f32(rng.standard_normal((M, N)))
    y = torch.empty_like(r)
    A.ardit_int_linear(None, A.linear_desc(M, N, K, q[0], K, s[0], q[1], K, s[1], res=r, res_type=A.F32, ldr=N), y, A.F32, N)
    A.ardit_int_linear(None, A.linear_desc(M, N, K, q[0], K, s[0], q[1], K, s[1], res=r, res_type=A.F32, ldr=N), r, A.F32, N)
    _sync()
    assert torch.equal(y, r)


@pytest.mark.parametrize("N,K", [(640, 512), (5120, 1280), (1990, 1315)])
def test_a_row_has_the_same_bits_in_any_batch(A, N, K):
    """Rows alone, in a few, in a tile, in many: whichever kernel runs."""
    import torch
    M = 2000
    rng = np.random.default_rng(7)
    kp = -(-K // 16) * 16
    x = np.zeros((M, kp), np.int8)
    w = np.zeros((N, kp), np.int8)
    x[:, :K], w[:, :K] = rng.integers(-127, 128, (M, K)), rng.integers(-127, 128, (N, K))
    xd, wd = torch.from_numpy(x).to("cuda"), torch.from_numpy(w).to("cuda")
    sx, sw = dev_f32(rng.uniform(0.001, 0.002, M)), dev_f32(rng.uniform(0.001, 0.002, N))
    b = dev_bf16(rng.standard_normal(N))

    def rows(at, n):
        y = torch.empty((n, N), dtype=torch.bfloat16, device="cuda")
        d = A.linear_desc(n, N, K, xd[at:], kp, sx[at:], wd, kp, sw, bias=b, act=A.ACT_GELU)
        A.ardit_int_linear(None, d, y, A.BF16, N)
        _sync()
        return y.view(torch.int16)

    whole = rows(0, M)
    for at, n in [(0, 1), (1999, 1), (37, 5), (100, 16), (555, 40), (600, 100), (900, 300), (3, 777)]:
        assert torch.equal(rows(at, n), whole[at:at + n]), (at, n)


# -------------------------------------------------------------------- together
def _ffn(A, t, stream=None):
    """The FFN half of a block through the calls: sum, norm, up with GELU, codes, down with the gated residual."""
    M, D, F = t["M"], t["D"], t["F"]
    A.ardit_int_norm(stream, M, D, A.norm_desc(t["x"], A.F32, D, delta=t["delta"], delta_type=A.BF16, ldd=D, h=t["h"], ldh=D,
                                               mod=t["mod"], mod_table=t["tab"], rows_per_stream=M // 2, shift_row=3,
                                               scale_row=4, gate_row=2), t["c"], D, t["s"])
    A.ardit_int_linear(stream, A.linear_desc(M, F, D, t["c"], D, t["s"], t["w1"], D, t["s1"], bias=t["b1"],
                                             act=A.ACT_GELU), t["u"], A.BF16, F)
    A.ardit_int_quantize(stream, t["u"], A.BF16, M, F, F, t["cu"], F, t["su"])
    A.ardit_int_linear(stream, A.linear_desc(M, D, F, t["cu"], F, t["su"], t["w2"], F, t["s2"], bias=t["b2"], res=t["h"],
                                             res_type=A.F32, ldr=D, mod=t["mod"], mod_table=t["tab"], gate_row=5,
                                             rows_per_stream=M // 2), t["y"], A.BF16, D)


def _ffn_state(A, M, D, F, seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rn = lambda *s: torch.randn(s, device="cuda", generator=g)
    t = {"M": M, "D": D, "F": F, "x": rn(M, D), "delta": rn(M, D).bfloat16(), "mod": 0.3 * rn(2, 6, D), "tab": 0.02 * rn(6, D),
         "b1": (0.02 * rn(F)).bfloat16(), "b2": (0.02 * rn(D)).bfloat16()}
    i8 = lambda *s: torch.empty(s, dtype=torch.int8, device="cuda")
    t.update(h=torch.empty(M, D, device="cuda"), c=i8(M, D), s=torch.empty(M, device="cuda"), cu=i8(M, F),
             su=torch.empty(M, device="cuda"), u=torch.empty(M, F, dtype=torch.bfloat16, device="cuda"),
             y=torch.empty(M, D, dtype=torch.bfloat16, device="cuda"), w1=i8(F, D), w2=i8(D, F),
             s1=torch.empty(F, device="cuda"), s2=torch.empty(D, device="cuda"))
    t["W1"], t["W2"] = (0.05 * rn(F, D)).bfloat16(), (0.05 * rn(D, F)).bfloat16()
    A.ardit_int_quantize(None, t["W1"], A.BF16, F, D, D, t["w1"], D, t["s1"])
    A.ardit_int_quantize(None, t["W2"], A.BF16, D, F, F, t["w2"], F, t["s2"])
    return t


@pytest.mark.parametrize("M,D,F", [(2, 256, 512), (20, 640, 1536), (194, 256, 1024), (1100, 512, 1280)])
def test_calls_together(A, M, D, F):
    """Each step against the reference of what the step before it left."""
    t = _ffn_state(A, M, D, F, M)
    _ffn(A, t)
    _sync()
    n = {k: (host_f32(v) if v.dtype.is_floating_point else v.cpu().numpy()) for k, v in t.items() if hasattr(v, "dtype")}
    row = np.arange(M) // (M // 2)
    vec = lambda r: (n["mod"][:, r] + n["tab"][r])[row].astype(np.float64)
    h = n["x"].astype(np.float64) + vec(2) * n["delta"]
    assert (np.abs(n["h"] - h) <= 1.01 * U * np.abs(h)).all()
    q, s, margin = I.quantize(I.norm(n["h"], 1e-6, scale=vec(4), shift=vec(3)))
    assert np.array_equal(n["c"][margin > 1e-9], q[margin > 1e-9]) and np.allclose(n["s"], s, rtol=2 * U, atol=0)
    u, p = I.linear(n["c"], n["s"], n["w1"], n["s1"], n["b1"], gelu=True)
    z = p + n["b1"]
    tol = 1.2 * U * (3.1 * np.abs(p) + 1.1 * np.abs(z)) + (2.0 ** -8 + (8 + 14 * (np.abs(z) + np.abs(z) ** 3)) * U) * np.abs(u)
    assert (np.abs(n["u"] - u) <= tol + 1e-36).all()
    q, s, _ = I.quantize(n["u"])
    assert np.array_equal(n["cu"], q) and np.array_equal(n["su"], s)
    y, p = I.linear(n["cu"], n["su"], n["w2"], n["s2"], n["b2"], res=n["h"], gate=vec(5))
    z = p + n["b2"]
    tol = np.abs(vec(5)) * U * (3.1 * np.abs(p) + 2.2 * np.abs(z)) + (1.1 * U + 2.0 ** -8) * np.abs(y)
    assert (np.abs(n["y"] - y) <= 1.02 * tol).all()


def test_captured_and_replayed(A):
    """The run in one graph, replayed with new inputs between eager calls, on a stream of its own."""
    import torch
    t = _ffn_state(A, 322, 384, 1280, 5)
    _ffn(A, t)
    _sync()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _ffn(A, t)
    for i in range(4):
        t["x"].normal_()
        t["x"][7] = 0
        t["y"].zero_()
        g.replay()
        _sync()
        got = t["y"].clone()
        t["y"].zero_()
        _ffn(A, t)
        _sync()
        assert torch.equal(got, t["y"]) and bool(got.any())


def test_two_streams_at_once(A):
    import torch
    states = [_ffn_state(A, m, 512, 1536, 8 + m) for m in (40, 600)]
    want = []
    for t in states:
        _ffn(A, t)
        _sync()
        want.append(t["y"].clone())
        t["y"].zero_()
    streams = [torch.cuda.Stream() for _ in states]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for t, s in zip(states, streams):
            _ffn(A, t, s)
    _sync()
    for t, w in zip(states, want):
        assert torch.equal(t["y"], w)
